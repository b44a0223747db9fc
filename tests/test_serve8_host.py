"""Serving from the 8-bit cache without a GPU: the oracle's pins, and the host checks of
the entry points (refusals return before anything is enqueued; no compute call runs here)."""
import ctypes
import math
import os
import random

import numpy as np
import pytest
import torch

import paper_2609_14717_amd as co
from oracle import SKIP, serve8

F8 = torch.float8_e4m3fn
needs_lib = pytest.mark.skipif(not os.path.exists(co.LIB_PATH), reason="library not built")


# ------------------------------------------------------------------ the oracle

def test_codes_stand_for_the_values_that_torch_reads():
    t = torch.arange(256, dtype=torch.uint8).view(F8).double().numpy()
    np.testing.assert_array_equal(serve8.VALUES, t)


def test_rounding_is_to_the_nearest_code_ties_to_even():
    """Every value, every midpoint of two neighbours and points next to it."""
    v = serve8.VALUES[:127]
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e3)])
    code = serve8.e4m3_code(x)
    np.testing.assert_array_equal(code[:127], np.arange(127))
    np.testing.assert_array_equal(code[127:253] % 2, 0)
    np.testing.assert_array_equal(code[253:379], np.arange(126))
    np.testing.assert_array_equal(code[379:], np.arange(1, 127))
    near = np.concatenate([v, mid])          # these are exact in 32 bits: torch agrees
    near = near[near.astype(np.float32) == near]
    t = torch.tensor(near, dtype=torch.float32).to(F8).view(torch.uint8).numpy()
    np.testing.assert_array_equal(serve8.e4m3_code(near), t)
    assert list(serve8.e4m3_code([math.inf, -math.inf, math.nan])) == [127] * 3
    np.testing.assert_array_equal(serve8.e4m3_code(-x), code | 128)


@pytest.mark.parametrize("top,k", [(448.0, 0), (449.0, 1), (1.75, -8), (1.76, -7), (1.0, -8),
                                   (3e38, 120), (1e-38, -126), (0.0, -126)])
def test_scale_is_the_smallest_power_that_fits(top, k):
    b = serve8.scale_byte([[top, -top / 2, math.inf, math.nan]])
    assert b - 127 == k
    assert top <= 448 * 2.0 ** k
    if k > -126:
        assert top > 448 * 2.0 ** (k - 1)


def test_store_keeps_and_clears_slots():
    new = lambda *s: np.zeros(s, np.uint8)  # noqa: E731
    c = serve8.Cache8(new(1, 2, 1, 16, 64), new(1, 2, 1, 16, 64), new(1, 2, 1), new(1, 2, 1))
    c.k[:] = 0x38                            # 1.0 in every slot
    one = np.ones((1, 3, 1, 64))
    assert c.store(one, one * 500, [17, 18, SKIP], 2) == 0
    assert c.ks[0, 1, 0] == 119              # 1.0 under 2^-8; the old scale, 2^-127, was finer
    x = c.values("k", 0, 1, 0)
    assert np.all(x[1:3] == 1.0) and np.all(x[0] == 0.0)    # 2^-127 is below the smallest code
    assert np.all(c.values("v", 0, 1, 0)[1:3] == 512.0)     # 500 under 2: 250 -> 256
    assert c.store(one, one, [0, 1, 2], 2) == 0
    assert np.all(c.values("k", 0, 0, 0)[:3] == 1.0) and np.all(c.k[0, 0, 0, 3:] == 0)
    assert c.store(one, one, [32, -3, 19], 2) == serve8.ERR_PAGE_RANGE


def test_going_back_undoes_an_assignment():
    r = random.Random(5)
    for trial in range(60):
        S, P = r.randint(1, 9), r.randint(1, 6)
        n = S * P + r.randint(0, 5)
        table, held = np.full((S, P), -1, np.int64), [0] * S
        free = list(range(n))
        r.shuffle(free)
        a = [r.randint(0, P * 16) for _ in range(S)]
        b = [r.randint(0, P * 16) for _ in range(S)]
        table, held, free, st = serve8.assign_pages(a, 0, table, held, free, P, n)
        assert st == 0 and held == [-(-x // 16) for x in a]
        t2, h2, f2, st = serve8.assign_pages(b, 0, table, held, free, P, n)
        owned = sorted(int(x) for x in t2[t2 >= 0]) + f2
        assert st == 0 and sorted(owned) == list(range(n))
        t3, h3, f3, st = serve8.assign_pages(a, 0, t2, h2, f2, P, n)
        assert st == 0 and h3 == held and f3 == free
        np.testing.assert_array_equal(t3, table)


def test_a_pool_that_runs_out_serves_in_order():
    table = np.full((4, 4), -1)
    table[0, :2] = [7, 8]
    t, held, free, st = serve8.assign_pages([0, 32, 48, 16], 0, table, [2, 0, 0, 0], [5], 4, 9)
    assert st == serve8.ERR_POOL and held == [0, 2, 0, 0] and free == [5]
    assert t[1].tolist() == [7, 8, -1, -1] and np.all(t[2:] == -1)


def test_slot_map_pins():
    pos, dst, st = serve8.slot_map(7, [1, 3, 3, 6], [15, 0, 2], [[4, 9], [1, 1], [0, 3]], 2, 10)
    assert st == 0 and pos.tolist() == [0, 15, 16, 2, 3, 4, 0]
    assert dst.tolist() == [SKIP, 79, 144, 2, 3, 4, SKIP]
    assert serve8.slot_map(1, [0, 1], [-1], [[0]], 1, 1)[2] == serve8.ERR_LENGTH
    assert serve8.slot_map(1, [0, 1], [16], [[0]], 1, 1)[2] == serve8.ERR_CAPACITY
    assert serve8.slot_map(1, [0, 1], [3], [[1]], 1, 1)[2] == serve8.ERR_PAGE_RANGE


# --------------------------------------------------------------- host refusals

FAKE = 1 << 20      # an aligned, non-null address that is never dereferenced here


def _dims(**kw):
    base = dict(S=2, B=16, Dcat=768, d=256, L=1, Hq=4, Hkv=2, hd=64, max_pages_per_seq=8,
                num_pages=16, dtype="bf16", theta=1e4)
    base.update(kw)
    return co.make_dims(**base)


def _state(**kw):
    return dict({k: FAKE for k in ("ctx_len", "carry_len", "page_table", "k_carry", "v_carry",
                                   "status")}, k_cache=None, v_cache=None, **kw)


def _cache(**kw):
    return dict({k: FAKE for k in ("k_pages", "v_pages", "k_scale", "v_scale")}, **kw)


def _pool(**kw):
    return dict({k: FAKE for k in ("page_table", "held", "free_pages", "free_count")}, **kw)


ROUTE = {k: FAKE for k in ("accept_len", "row_pos", "row_dst")}
BIG = 1 << 34


def assign(d, want=FAKE, reserve=0, pool=None, status=FAKE, ws=FAKE, nb=BIG):
    return co.carryover_assign_pages(d, want, reserve, pool or _pool(), status, ws, stream=0,
                                     ws_bytes=nb)


def slots(d, n=8, start=FAKE, pos0=FAKE, table=FAKE, pos=FAKE, dst=FAKE, status=FAKE):
    return co.carryover_slot_map(d, n, start, pos0, table, pos, dst, status, stream=0)


def store(d, n=8, k=FAKE, v=FAKE, dst=FAKE, cache=None, status=FAKE):
    return co.carryover_store_kv8(d, n, k, v, dst, cache or _cache(), status, stream=0)


def attend(d, layers=1, q=FAKE, ks=None, vs=None, st=None, cache=None, out=FAKE, lse=None, mass=None,
           ws=FAKE, nb=BIG, l0=0):
    return co.drafter_block_attention_kv8(d, l0, layers, q, ks, vs, st or _state(), cache or _cache(),
                                          out, lse, mass, 0, ws, stream=0, ws_bytes=nb)


def project(d, w=None, st=None, cache=None, ws=FAKE, nb=BIG):
    return co.carryover_project_kv8(d, w or co.weights(FAKE, FAKE, FAKE), FAKE, ROUTE,
                                    st or _state(), cache or _cache(), ws, stream=0, ws_bytes=nb)


def round_(d, w=None, q=FAKE, st=None, cache=None, lse=None, nb=BIG):
    return co.carryover_round_kv8(d, w or co.weights(FAKE, FAKE, FAKE), FAKE, FAKE, FAKE, q,
                                  st or _state(), cache or _cache(), ROUTE, FAKE, lse, 0, FAKE,
                                  stream=0, ws_bytes=nb)


EVERY = (assign, slots, store, attend, project, round_)


def _rc(fn, *a, **kw):
    try:
        fn(*a, **kw)
    except co.CarryoverError as e:
        return e.code
    return co.CO_OK


@needs_lib
@pytest.mark.parametrize("kw,code", [(dict(hd=96), co.CO_ERR_UNSUPPORTED),
                                     (dict(Hq=6, Hkv=4), co.CO_ERR_UNSUPPORTED),
                                     (dict(num_pages=0), co.CO_ERR_INVALID_ARG),
                                     (dict(num_pages=1 << 27), co.CO_ERR_UNSUPPORTED)])
def test_bad_dims_are_refused_by_every_call(kw, code):
    for call in EVERY:
        assert _rc(call, _dims(**kw)) == code, call.__name__


@needs_lib
def test_the_cache_is_of_bf16_drafters():
    d = _dims(dtype="f32")
    for call in (store, attend, project, round_):
        assert _rc(call, d) == co.CO_ERR_UNSUPPORTED, call.__name__
    for which in (co.CO_WS_PROJECT_KV8, co.CO_WS_ATTENTION_KV8, co.CO_WS_ROUND_KV8):
        assert co.workspace_bytes(d, which) == 0
    d = _dims(B=32, Hq=8)                   # 128 query rows per KV head
    assert _rc(attend, d) == _rc(round_, d) == co.CO_ERR_UNSUPPORTED
    assert co.workspace_bytes(d, co.CO_WS_ATTENTION_KV8) == 0
    assert co.workspace_bytes(d, co.CO_WS_PROJECT_KV8) > 0


@needs_lib
@pytest.mark.parametrize("call,kw", [
    (assign, dict(want=None)), (assign, dict(reserve=-1)), (assign, dict(want=FAKE + 2)),
    (assign, dict(status=None)), (assign, dict(ws=None)), (assign, dict(ws=FAKE + 16)),
    (assign, dict(pool=_pool(held=None))), (assign, dict(pool=_pool(page_table=None))),
    (assign, dict(pool=_pool(free_pages=FAKE + 1))), (assign, dict(pool=_pool(free_count=None))),
    (slots, dict(n=-1)), (slots, dict(start=None)), (slots, dict(pos0=FAKE + 2)),
    (slots, dict(table=None)), (slots, dict(pos=None)), (slots, dict(dst=FAKE + 1)),
    (slots, dict(status=None)),
    (store, dict(n=-1)), (store, dict(k=None)), (store, dict(v=FAKE + 8)), (store, dict(dst=None)),
    (store, dict(cache=_cache(k_pages=FAKE + 8))), (store, dict(cache=_cache(v_scale=None))),
    (store, dict(status=None)),
    (attend, dict(layers=2)), (attend, dict(layers=-1)), (attend, dict(q=None)),
    (attend, dict(q=FAKE + 2)), (attend, dict(out=None)), (attend, dict(lse=FAKE + 2)),
    (attend, dict(mass=FAKE + 1)), (attend, dict(ks=FAKE)), (attend, dict(vs=FAKE)),
    (attend, dict(ks=FAKE, vs=FAKE + 8)), (attend, dict(ws=FAKE + 128)), (attend, dict(ws=None)),
    (attend, dict(cache=_cache(k_scale=None))), (attend, dict(cache=_cache(v_pages=None))),
    (attend, dict(st=_state(ctx_len=None))),
    (project, dict(cache=_cache(v_pages=FAKE + 4))), (project, dict(ws=None)),
    (project, dict(w=co.weights(FAKE, FAKE, None))),
    (round_, dict(cache=_cache(k_pages=None))), (round_, dict(q=FAKE + 2)), (round_, dict(lse=FAKE + 2)),
    (round_, dict(w=co.weights(FAKE, FAKE, FAKE, FAKE + 2))),
], ids=lambda x: x.__name__ if callable(x) else "-".join(x))
def test_null_and_misaligned_arguments_are_refused(call, kw):
    assert _rc(call, _dims(), **kw) == co.CO_ERR_INVALID_ARG


@needs_lib
@pytest.mark.parametrize("call,which", [(assign, co.CO_WS_ASSIGN_PAGES),
                                        (attend, co.CO_WS_ATTENTION_KV8),
                                        (project, co.CO_WS_PROJECT_KV8),
                                        (round_, co.CO_WS_ROUND_KV8)])
def test_small_workspaces_are_refused(call, which):
    need = co.workspace_bytes(_dims(), which)
    assert need > 0 and need % 256 == 0
    assert _rc(call, _dims(), nb=need - 1) == co.CO_ERR_WORKSPACE
    assert _rc(call, _dims(), nb=0) == co.CO_ERR_WORKSPACE


@needs_lib
def test_round_workspace_is_its_steps():
    d = _dims(L=3, S=5)
    size = lambda w: co.workspace_bytes(d, w)  # noqa: E731
    assert size(co.CO_WS_ROUND_KV8) == size(co.CO_WS_PROJECT_KV8) + size(co.CO_WS_ATTENTION_KV8)
    rows = 3 * 5 * 16 * 2 * 64 * 2
    assert size(co.CO_WS_PROJECT_KV8) >= size(co.CO_WS_PROJECT) + 2 * rows


@needs_lib
def test_tables_beyond_32_bits_are_refused():
    d = _dims(S=1 << 16, max_pages_per_seq=1 << 15, B=1)
    assert _rc(assign, d) == co.CO_ERR_UNSUPPORTED
    d = _dims(L=8192, Hkv=8, Hq=8)
    assert _rc(store, d) == co.CO_ERR_UNSUPPORTED


@needs_lib
def test_sizes_beyond_a_launch_are_refused():
    assert _rc(assign, _dims(S=1 << 23, B=1, max_pages_per_seq=1)) == co.CO_ERR_UNSUPPORTED
    assert _rc(assign, _dims(S=1, max_pages_per_seq=1 << 23)) == co.CO_ERR_UNSUPPORTED
    assert _rc(store, _dims(), n=1 << 28) == co.CO_ERR_UNSUPPORTED
    d = _dims(S=1 << 24, B=16, L=1)
    assert _rc(project, d) == _rc(round_, d) == co.CO_ERR_UNSUPPORTED
    assert co.workspace_bytes(d, co.CO_WS_PROJECT_KV8) == 0


@needs_lib
def test_layer_ranges_that_pass_32_bits_are_refused():
    big = 2 ** 31 - 1
    for l0, n in ((1, big), (big, 1), (big, big)):
        assert _rc(attend, _dims(), l0=l0, layers=n) == co.CO_ERR_INVALID_ARG


@needs_lib
def test_empty_batches_and_no_rows_succeed():
    d = _dims(S=0)
    for which in range(9):
        co.workspace_bytes(d, which)
    for call in EVERY:
        kw = dict(n=0) if call in (slots, store) else {}
        assert _rc(call, d, **kw) == co.CO_OK, call.__name__
    assert _rc(attend, _dims(), layers=0) == co.CO_OK
    assert _rc(slots, _dims(), n=0) == _rc(store, _dims(), n=0) == co.CO_OK


@needs_lib
def test_pool_status_has_a_message():
    assert co.status_string(co.CO_ERR_POOL) != "unknown status"
    assert ctypes.sizeof(co.co_kv8) == ctypes.sizeof(co.co_page_pool) == 32
