"""GPU parity of serving from the 8-bit cache (page tables and slot maps, rows into the
cache, attention over it, and the round of all of them) with the fp64 oracle.

Whole numbers, codes and scale bytes are equal to the oracle's.  Attention is held to
the rule of the other bf16 paths, 2e-2 of a head vector's largest entry and 2e-2 of a
log-sum-exp or share: the queries are rounded to two codes after their rotation (2^-9 of
the value: a logit of a few units moves by a few 2^-9), the softmax weights to fp16 against
codes (half a step, 2^-11 of their size) and to two bf16 parts against carry and own rows
(2^-16), and the output to bf16 (2^-8).  The codes are exact in fp16 under the largest value
scale of the sequence and head, down to 2^-35 of the largest entry that it allows.
"""
import math
import random

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import oracle  # noqa: E402
import paper_2609_14717_amd as co  # noqa: E402
from helpers import assert_heads_close, head_err  # noqa: E402
from oracle import PAGE, SKIP, serve8  # noqa: E402

TOL = 2e-2
DEV = "cuda"


def ints(x):
    return torch.tensor(np.array(x), dtype=torch.int32, device=DEV)


def zero():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def space(d, which):
    return torch.full((max(256, co.workspace_bytes(d, which)),), 0xA5, dtype=torch.uint8, device=DEV)


def np_(t):
    return t.cpu().numpy()


# ------------------------------------------------------------- page tables

def dims(S, max_pages, num_pages, B=1, L=1, Hq=1, Hkv=1, hd=64, theta=1e4):
    return co.make_dims(S, B, 64, 64, L, Hq, Hkv, hd, max_pages, num_pages, "bf16", theta)


class Pool:
    """A pool on the device beside the oracle's."""

    def __init__(self, S, max_pages, num_pages, seed):
        self.d = dims(S, max_pages, num_pages)
        self.t = co.alloc_page_pool(self.d)
        ids = list(range(num_pages))
        random.Random(seed).shuffle(ids)
        self.t["free_pages"].copy_(ints(ids))
        self.table, self.held, self.free = np.full((S, max_pages), -1), [0] * S, ids
        self.ws, self.status = space(self.d, co.CO_WS_ASSIGN_PAGES), zero()

    def assign(self, want, reserve=0, stream=None):
        self.status.zero_()
        co.carryover_assign_pages(self.d, ints(want), reserve, self.t, self.status, self.ws, stream)
        d = self.d
        self.table, self.held, self.free, status = serve8.assign_pages(
            want, reserve, self.table, self.held, self.free, d.max_pages_per_seq, d.num_pages)
        assert int(self.status) == status
        np.testing.assert_array_equal(np_(self.t["held"]), self.held)
        np.testing.assert_array_equal(np_(self.t["page_table"]), self.table)
        assert int(self.t["free_count"]) == len(self.free)
        np.testing.assert_array_equal(np_(self.t["free_pages"])[:len(self.free)], self.free)


# the last three in two launches: more than 32768 entries, or more than 1024 sequences
@pytest.mark.parametrize("S,max_pages", [(1, 1), (1, 300), (2, 5), (7, 3), (33, 65), (1024, 4),
                                         (1025, 3), (130, 520), (1, 70000)])
def test_pages_follow_lengths(S, max_pages):
    r = random.Random(S * 1000 + max_pages)
    p = Pool(S, max_pages, max(4, S * min(max_pages, 40) // 2), S)
    top = min(max_pages, 60) * PAGE
    for step in range(6):
        lengths = [r.choice((0, 1, 15, 16, 17, top, r.randint(0, top), r.randint(0, top) // 4))
                   for _ in range(S)]
        p.assign([min(top, x) for x in lengths], r.choice((0, 0, 1, 16)))   # may run out
    p.assign([0] * S)
    assert sorted(p.free) == list(range(p.d.num_pages))


def test_going_back_restores_table_and_free_list():
    p = Pool(40, 30, 1200, 3)
    r = random.Random(9)
    a, b = ([r.randint(0, 480) for _ in range(40)] for _ in range(2))
    p.assign(a)
    before = {k: v.clone() for k, v in p.t.items()}
    p.assign(b)
    p.assign(a)
    n = int(p.t["free_count"])
    for k in ("page_table", "held", "free_count"):
        assert torch.equal(p.t[k], before[k])
    assert torch.equal(p.t["free_pages"][:n], before["free_pages"][:n])


@pytest.mark.parametrize("S,max_pages", [(6, 8), (6, 11000)], ids=["one launch", "two"])
def test_pages_of_bad_lengths_stay(S, max_pages):
    p = Pool(S, max_pages, 60, 1)
    p.assign([20, 30, 40, 0, 50, 60])
    p.assign([33, -1, 10, 5, 50, 60])                               # CO_ERR_LENGTH
    p.assign([33, 33, max_pages * PAGE + 1, 5, 0, 1])               # CO_ERR_CAPACITY
    p.assign([2 ** 31 - 1, 3, 40, 5, 0, 1], 2 ** 31 - 1)
    p.t["held"][1] = max_pages + 1                                  # a holding it cannot have
    p.status.zero_()
    co.carryover_assign_pages(p.d, ints([0] * 6), 0, p.t, p.status, p.ws)
    assert int(p.status) == co.CO_ERR_LENGTH
    assert np_(p.t["held"]).tolist() == [0, max_pages + 1, 0, 0, 0, 0]


@pytest.mark.parametrize("max_pages", [8, 11000], ids=["one launch", "two"])
@pytest.mark.parametrize("count", [-1, 61])
def test_a_free_count_out_of_range_changes_nothing(count, max_pages):
    p = Pool(6, max_pages, 60, 1)
    p.assign([20, 30, 40, 0, 50, 60])
    p.t["free_count"].fill_(count)
    before = {k: v.clone() for k, v in p.t.items()}
    p.status.zero_()
    co.carryover_assign_pages(p.d, ints([0, 99, 0, 9, 9, 9]), 0, p.t, p.status, p.ws)
    assert int(p.status) == co.CO_ERR_POOL
    assert all(torch.equal(p.t[k], before[k]) for k in before)


@pytest.mark.parametrize("S,lo,hi,extra", [(1, 0, 0, 3), (1, 1, 1, 0), (5, 0, 3, 2), (64, 0, 50, 9),
                                           (300, 0, 1, 0), (4096, 0, 3, 5), (4097, 0, 3, 5),
                                           (3, 900, 2100, 1)])
def test_slot_map(S, lo, hi, extra):
    r = random.Random(S + hi)
    P = -(-(hi + 40) // PAGE)
    n = [r.randint(lo, hi) for _ in range(S)]
    start = np.concatenate([[0], np.cumsum(n)]) + extra // 2          # padding in front and behind
    pos0 = [r.randint(0, 40) for _ in range(S)]
    table = np.random.RandomState(S).permutation(S * P).reshape(S, P)
    rows = int(start[-1]) + extra
    d, status = dims(S, P, S * P), zero()
    pos, dst = torch.full((2, rows + 1), 77, dtype=torch.int32, device=DEV)
    co.carryover_slot_map(d, rows, ints(start), ints(pos0), ints(table), pos, dst, status)
    wp, wd, st = serve8.slot_map(rows, start, pos0, table, P, S * P)
    assert int(status) == st == 0
    np.testing.assert_array_equal(np_(pos)[:rows], wp)
    np.testing.assert_array_equal(np_(dst)[:rows], wd)
    assert int(pos[rows]) == int(dst[rows]) == 77                     # nothing past the last row


@pytest.mark.parametrize("off", [1, 2, 3])
def test_slot_map_into_unaligned_arrays(off):
    d, status, rows = dims(3, 9, 27), zero(), 300
    start, pos0, table = [0, 120, 121, 300], [0, 5, 11], np.arange(26, -1, -1).reshape(3, 9)
    pos, dst = torch.full((2, rows + 8), 77, dtype=torch.int32, device=DEV)
    dst = torch.cat([dst, dst])[:rows + 8]
    co.carryover_slot_map(d, rows, ints(start), ints(pos0), ints(table), pos[off:], dst[off:], status)
    wp, wd, st = serve8.slot_map(rows, start, pos0, table, 9, 27)
    assert int(status) == st
    np.testing.assert_array_equal(np_(pos)[off:off + rows], wp)
    np.testing.assert_array_equal(np_(dst)[off:off + rows], wd)
    assert np.all(np_(pos)[:off] == 77) and np.all(np_(dst)[off + rows:] == 77)


@pytest.mark.parametrize("pos0,page,code", [(-1, 0, co.CO_ERR_LENGTH), (30, 0, co.CO_ERR_CAPACITY),
                                            (3, 9, co.CO_ERR_PAGE_RANGE), (3, -1, co.CO_ERR_PAGE_RANGE)])
def test_slot_map_errors_skip_the_row(pos0, page, code):
    d, status = dims(2, 2, 9), zero()
    table = [[page, 1], [2, 3]]
    pos, dst = torch.zeros((2, 9), dtype=torch.int32, device=DEV)
    co.carryover_slot_map(d, 9, ints([0, 4, 9]), ints([pos0, 14]), ints(table), pos, dst, status)
    wp, wd, st = serve8.slot_map(9, [0, 4, 9], [pos0, 14], table, 2, 9)
    assert int(status) == st == code
    np.testing.assert_array_equal(np_(pos), wp)
    np.testing.assert_array_equal(np_(dst), wd)
    assert wd[4:].tolist() == [46, 47, 48, 49, 50]


def test_slot_map_of_starts_that_decrease():
    """Rows that no sequence holds by the starts get no slot; the status says so."""
    d, status = dims(3, 4, 12), zero()
    pos, dst = torch.zeros((2, 8), dtype=torch.int32, device=DEV)
    co.carryover_slot_map(d, 8, ints([0, 6, 2, 8]), ints([0, 0, 0]), ints(np.arange(12).reshape(3, 4)),
                          pos, dst, status)
    assert np.all((np_(dst) == SKIP) | ((np_(dst) >= 0) & (np_(dst) < 192)))


# -------------------------------------------------------------------- store

def rows_of(kind, shape, g):
    x = torch.randn(shape, generator=g, device=DEV)
    if kind == "ordinary":
        x *= torch.exp2(3 * torch.rand(shape[0], 1, shape[2], 1, generator=g, device=DEV))
    elif kind == "wide":           # magnitudes over the whole range of the type
        x = torch.exp2(torch.rand(shape, generator=g, device=DEV) * 250 - 125) * x.sign()
    elif kind == "ties":           # multiples of half a code's step, and the largest code
        x = torch.randint(-896, 897, shape, generator=g, device=DEV).float() / 2
    elif kind == "bad":            # infinities, NaN, zeros and a head of nothing else
        m = torch.randint(0, 12, shape, generator=g, device=DEV)
        x = torch.where(m == 0, math.inf, torch.where(m == 1, -math.inf, torch.where(m == 2, math.nan, x)))
        x[:, :, 0] = torch.where(m[:, :, 0] < 6, math.nan, 0.0)
    elif kind == "small":          # below the smallest scale
        x *= 2.0 ** -130
    return x.bfloat16()


def same_codes(got, want):
    """Equal codes; a NaN of either sign."""
    a, b = np.asarray(got), np.asarray(want)
    nan = ((a & 127) == 127) & ((b & 127) == 127)
    assert np.array_equal(np.where(nan, 0, a), np.where(nan, 0, b))


def check_cache(cache, orc):
    got = serve8.Cache8.read(cache)
    np.testing.assert_array_equal(got.ks, orc.ks)
    np.testing.assert_array_equal(got.vs, orc.vs)
    same_codes(got.k, orc.k)
    same_codes(got.v, orc.v)


def earlier(cache, g):
    """Codes of any value but NaN, and scales on both sides of the rows' own."""
    for k in ("k_pages", "v_pages"):
        c = torch.randint(0, 127, cache[k].shape, generator=g, device=DEV)
        cache[k].copy_(c + 128 * torch.randint(0, 2, c.shape, generator=g, device=DEV))
    for k in ("k_scale", "v_scale"):
        cache[k].copy_(torch.randint(105, 130, cache[k].shape, generator=g, device=DEV))


LAYOUTS = {
    "one": [5 * PAGE + 3],
    "first": [2 * PAGE],
    "last": [2 * PAGE + 15],
    "page": list(range(48, 64)),
    "over pages": [PAGE * 3 + 14, PAGE * 3 + 15, PAGE * 1, PAGE * 1 + 1, PAGE * 1 + 2],
    "window": [SKIP, -1, 35, 36, -1, -2, -3, 16, 17, 18, -1, SKIP, 0, 1, 2, 3, 4, 95, -1],
    "prompt": [*range(0, 32), *range(80, 96), *range(32, 45), *range(66, 80), *range(48, 56)],
    "tokens": [7, 16 + 15, 32, 48 + 1, 64 + 8, 80],
    "nothing": [SKIP, -1, -7],
    "out of range": [96, 97, 3, 2 ** 31 - 1, -5, 1600],
}


@pytest.mark.parametrize("hd,H,L", [(64, 1, 1), (128, 3, 2)])
@pytest.mark.parametrize("kind", ["ordinary", "wide", "ties", "bad", "small"])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_store(layout, kind, hd, H, L):
    dst = LAYOUTS[layout]
    g = torch.Generator(device=DEV).manual_seed(len(dst) * 7 + hd)
    d, status = dims(1, 6, 6, L=L, Hq=H, Hkv=H, hd=hd), zero()
    cache = co.alloc_kv8(d)
    earlier(cache, g)
    orc = serve8.Cache8.read(cache)
    k, v = (rows_of(kind, (L, len(dst), H, hd), g) for _ in range(2))
    co.carryover_store_kv8(d, len(dst), k, v, ints(dst), cache, status)
    st = orc.store(k.double().cpu().numpy(), v.double().cpu().numpy(), dst, 6)
    assert int(status) == st == (co.CO_ERR_PAGE_RANGE if layout == "out of range" else 0)
    check_cache(cache, orc)


@pytest.mark.parametrize("hd", [64, 128])
def test_store_token_by_token(hd):
    """A page that fills one token at a time, magnitudes rising and falling."""
    g = torch.Generator(device=DEV).manual_seed(hd)
    d, status = dims(2, 2, 4, L=2, Hq=2, Hkv=2, hd=hd), zero()
    cache = co.alloc_kv8(d)
    orc = serve8.Cache8.read(cache)
    for t in range(20):
        size = 2.0 ** (6 * math.sin(t))
        k, v = ((torch.randn((2, 2, 2, hd), generator=g, device=DEV) * size).bfloat16() for _ in range(2))
        dst = [16 + t if t < 16 else t - 16, 3 * 16 + t if t < 16 else SKIP]
        co.carryover_store_kv8(d, 2, k, v, ints(dst), cache, status)
        orc.store(k.double().cpu().numpy(), v.double().cpu().numpy(), dst, 4)
        check_cache(cache, orc)
    assert int(status) == 0


@pytest.mark.parametrize("M,L,H", [(700, 5, 8), (3000, 5, 8), (8000, 4, 8)])
def test_store_of_many_rows(M, L, H):
    """More wavefronts than fit at once: several rows to each, and pages that start in
    one wavefront's rows and end in the next one's."""
    hd, pages = 64, M // PAGE + 40
    r = random.Random(M)
    g = torch.Generator(device=DEV).manual_seed(M)
    dst, page = [], 0
    while len(dst) < M:                       # prompts, single tokens and skipped rows in turn
        n, t0 = r.choice(((1, r.randrange(16)), (r.randint(1, 200), 0), (r.randint(1, 30), r.randrange(16))))
        n = min(n, (pages - page) * PAGE - t0)
        if n <= 0:
            break
        dst += [page * PAGE + t0 + i for i in range(n)] + [SKIP] * r.choice((0, 0, 1))
        page += -(-(t0 + n) // PAGE)
    dst = dst[:M]
    d, status = dims(1, pages, pages, L=L, Hq=H, Hkv=H, hd=hd), zero()
    cache = co.alloc_kv8(d)
    earlier(cache, g)
    before = {k: v.clone() for k, v in cache.items()}
    k, v = (torch.randn((L, len(dst), H, hd), generator=g, device=DEV).bfloat16() for _ in range(2))
    co.carryover_store_kv8(d, len(dst), k, v, ints(dst), cache, status)
    assert int(status) == 0
    for layer, head in ((0, 0), (L - 1, H - 1), (1, 3)):     # some heads, all pages
        part = lambda t: {n: x[layer:layer + 1, :, head:head + 1] for n, x in t.items()}  # noqa: E731
        orc = serve8.Cache8.read(part(before))
        orc.store(*(x[layer:layer + 1, :, head:head + 1].double().cpu().numpy() for x in (k, v)), dst, pages)
        check_cache(part(cache), orc)
    again = {n: x.clone() for n, x in before.items()}
    co.carryover_store_kv8(d, len(dst), k, v, ints(dst), again, status)
    assert all(torch.equal(again[n], cache[n]) for n in cache)


# ------------------------------------------------------------------- attention

class Serve:
    """A drafter state over an 8-bit cache, with the oracle's view of it."""

    def __init__(self, S, B, L, Hq, Hkv, hd, ctx, carry, seed=0, own=False, wide=0, theta=1e4,
                 num_pages=None, ids=None, size=1.0):
        r = np.random.RandomState(seed)
        g = torch.Generator(device=DEV).manual_seed(seed)
        need = [-(-n // PAGE) for n in ctx]
        P = max(max(need), wide, 1)
        N = num_pages or sum(need) + 3
        order = np.asarray(ids) if ids is not None else r.permutation(N)
        table, at = np.full((S, P), -1), 0       # an entry past the context is never read
        for s, n in enumerate(need):
            table[s, :n] = order[at:at + n]
            at += n
        self.d = co.make_dims(S, B, 64, 64, L, Hq, Hkv, hd, P, N, "bf16", theta)
        self.S, self.B, self.L, self.Hq, self.Hkv, self.hd, self.theta = S, B, L, Hq, Hkv, hd, theta
        self.ctx, self.carry, self.table = list(ctx), list(carry), table
        self.cache = co.alloc_kv8(self.d)
        used = torch.tensor(order[:max(at, 1)], device=DEV)
        for x in ("k", "v"):                     # any finite codes, scales of their own
            shape = (L, len(used)) + self.cache[x + "_pages"].shape[2:]
            code = torch.randint(0, 127, shape, generator=g, device=DEV)
            code = code * (torch.rand(shape, generator=g, device=DEV) < 0.5) + 40    # few large ones
            code = code.clamp_max(100) + 128 * torch.randint(0, 2, shape, generator=g, device=DEV)
            self.cache[x + "_pages"][:, used] = code.to(torch.uint8)
            b = torch.randint(118, 124, (L, len(used), Hkv), generator=g, device=DEV)
            self.cache[x + "_scale"][:, used] = b.to(torch.uint8)
        self.st = co.alloc_state(self.d, np.where(table < 0, -1, table), committed=False)
        for k in ("k_carry", "v_carry"):
            self.st[k].normal_(generator=g)
        self.st["ctx_len"].copy_(ints(ctx))
        self.st["carry_len"].copy_(ints(carry))
        self.q = (size * torch.randn((L, S, B, Hq, hd), generator=g, device=DEV)).bfloat16()
        self.own = [torch.randn((L, S, B, Hkv, hd), generator=g, device=DEV).bfloat16() if own else None
                    for _ in range(2)]
        self.ws = space(self.d, co.CO_WS_ATTENTION_KV8)
        self.poison()

    def poison(self):
        """NaN codes in the slots past every context, NaN in the carry slots past every length."""
        for s, n in enumerate(self.ctx):
            if n % PAGE:
                p, t = int(self.table[s][n // PAGE]), n % PAGE
                self.cache["k_pages"][:, p, :, t:] = 0x7F
                self.cache["v_pages"][:, p, :, :, t:] = 0xFF
        CP = -(-self.B // PAGE)
        for s, u in enumerate(self.carry):
            for c in range(CP):
                t = max(0, min(PAGE, u - c * PAGE))
                self.st["k_carry"][:, s, c, :, t:] = math.nan
                self.st["v_carry"][:, s, c, :, :, t:] = math.nan

    def run(self, l0=0, ln=None, lse=True, mass=False, flags=0, stream=None, out=None):
        ln = self.L if ln is None else ln
        q = self.q[l0:l0 + ln].contiguous()
        out = torch.full_like(q, 9.0) if out is None else out
        z = torch.full(q.shape[:-1], 9.0, device=DEV) if lse else None
        m = torch.full(q.shape[:-1], 9.0, device=DEV) if mass else None
        own = [None if x is None else x[l0:l0 + ln].contiguous() for x in self.own]
        co.drafter_block_attention_kv8(self.d, l0, ln, q, *own, self.st, self.cache, out, z, m, flags,
                                       self.ws, stream)
        return out, z, m

    def check(self, got, l0=0, seqs=None, hidden=(), rotated=False, rounded=False):
        """Against the oracle, every sequence or some; ``hidden``: (s, page) left out;
        ``rounded``: the oracle takes the queries as the kernels hold them, two codes
        per dim after rotation and scaling (see the test that asks for it)."""
        out, z, m = (None if t is None else t.double().cpu().numpy() for t in got)
        orc, G = serve8.Cache8.read(self.cache), self.Hq // self.Hkv
        kc, vc = (self.st[k].double().cpu().numpy() for k in ("k_carry", "v_carry"))
        q = self.q.double().cpu().numpy()
        own = [None if x is None else x.double().cpu().numpy() for x in self.own]
        worst = 0.0
        for s in range(self.S) if seqs is None else seqs:
            n, u = self.ctx[s], self.carry[s]
            pos = n + np.arange(self.B)
            keep = np.ones(n, bool)
            for at, p in hidden:
                if at == s:
                    keep[p * PAGE:(p + 1) * PAGE] = False
            for i in range(out.shape[0]):
                layer = l0 + i
                for h in range(self.Hkv):
                    table = [[max(0, x) for x in row] for row in self.table[s:s + 1]]
                    k, v = orc.context(table, 0, layer, h, n)
                    k, v = k[keep], v[keep]
                    rows = np.arange(u)
                    ku = kc[layer, s, rows // PAGE, h, rows % PAGE]
                    vu = vc[layer, s, rows // PAGE, h, :, rows % PAGE]
                    ks, vs = [k, ku], [v, vu]
                    if own[0] is not None:
                        ks.append(oracle.rope(own[0][layer, s, :, h], pos, self.theta))
                        vs.append(own[1][layer, s, :, h])
                    ks, vs = np.concatenate(ks), np.concatenate(vs)
                    qs = q[layer, s, :, h * G:(h + 1) * G].reshape(self.B * G, self.hd)
                    qp = np.repeat(0 * pos if rotated else pos, G)
                    if rounded:
                        c = math.log2(math.e) / math.sqrt(self.hd)
                        qs, qp = two_codes(oracle.rope(qs, qp, self.theta) * c) / c, 0 * qp
                    o, lse = oracle.attend(qs, qp, ks, vs, self.theta)
                    go = out[i, s, :, h * G:(h + 1) * G].reshape(self.B * G, self.hd)
                    assert np.all(np.isfinite(go)), (s, layer, h)
                    worst = max(worst, head_err(go, o))
                    if z is not None:
                        gz = z[i, s, :, h * G:(h + 1) * G].ravel()
                        assert np.array_equal(np.isinf(gz), np.isinf(lse))
                        fine = np.isfinite(lse)
                        off = np.abs(gz[fine] - lse[fine]).max(initial=0)
                        assert off <= TOL * max(1, np.abs(lse[fine]).max(initial=0))
                    if m is not None:
                        want = oracle.carry_mass(qs, qp, k, ku, self.theta)
                        gm = m[i, s, :, h * G:(h + 1) * G].ravel()
                        assert np.abs(gm - want).max() <= TOL, (s, layer, h)
        assert worst <= TOL, worst
        assert int(self.st["status"]) == (co.CO_ERR_PAGE_RANGE if hidden else 0)
        return worst


def two_codes(rows):
    """Rows as the sum of two e4m3 codes per entry: one under the row's scale, one for the
    rest under a sixteenth of it."""
    out = np.empty_like(rows)
    for i, x in enumerate(rows):
        unit = 2.0 ** (max(5, serve8.scale_byte(x)) - 127)
        hi = serve8.VALUES[serve8.e4m3_code(x / unit)]
        out[i] = (hi + serve8.VALUES[serve8.e4m3_code((x / unit - hi) * 16)] / 16) * unit
    return out


def spread(lo, hi, n, seed):
    r = random.Random(seed)
    return [lo, hi][:n] + [r.randint(lo, hi) for _ in range(n - 2)]


EDGES = [0, 1, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 127, 128, 129]
CASES = [
    # S, B, L, Hq, Hkv, hd, contexts, carry rows up to, wide table
    (17, 1, 1, 1, 1, 64, EDGES, 1, 0),                   # one token, one head: every page and tile edge
    (17, 1, 1, 2, 2, 128, EDGES, 0, 0),
    (17, 16, 1, 4, 1, 128, EDGES, 16, 0),                # 64 rows
    (17, 16, 1, 4, 1, 64, EDGES, 16, 0),
    (17, 16, 1, 2, 1, 128, EDGES, 16, 40),               # 32 rows
    (1, 16, 1, 8, 2, 128, [2100], 16, 0),                # one sequence over the whole chip
    (1, 7, 1, 6, 2, 128, [2100], 7, 0),                  # 21 rows
    (2, 1, 1, 8, 1, 128, [1, 130], 1, 300),              # multi-query single tokens
    (3, 1, 2, 16, 1, 64, [5000, 1, 700], 1, 0),
    (3, 16, 2, 2, 1, 64, [33, 600, 350], 16, 0),
    (5, 11, 1, 3, 1, 128, spread(100, 9000, 5, 1), 11, 0),   # 33 rows, uneven
    (5, 11, 1, 3, 1, 64, spread(100, 9000, 5, 2), 11, 0),
    (64, 4, 1, 8, 8, 128, spread(1, 40, 64, 3), 4, 0),   # one sequence per lane
    (65, 4, 1, 8, 8, 64, spread(1, 40, 65, 4), 4, 0),    # two per lane
    (130, 16, 1, 4, 1, 128, spread(0, 300, 130, 5), 16, 0),
    (300, 1, 1, 4, 2, 64, spread(0, 200, 300, 6), 1, 0),
    (32, 15, 1, 4, 4, 64, spread(80, 140, 32, 7), 15, 300),
    (2, 40, 1, 1, 1, 128, [100, 300], 40, 0),            # carry segments of several pages
    (2, 64, 1, 1, 1, 64, [70, 0], 64, 0),
    (3, 48, 2, 1, 1, 64, [1000, 20, 3], 48, 0),
]


def case(i, **kw):
    S, B, L, Hq, Hkv, hd, ctx, most, wide = CASES[i]
    r = random.Random(i)
    carry = [r.choice((0, most, r.randint(0, most))) for _ in range(S)]
    return Serve(S, B, L, Hq, Hkv, hd, ctx, carry, seed=i, wide=wide, theta=1e6 if i % 2 else 1e4, **kw)


@pytest.mark.parametrize("i", range(len(CASES)), ids=lambda i: "-".join(map(str, CASES[i][:6])))
def test_attention(i):
    sv = case(i)
    sv.check(sv.run())


@pytest.mark.parametrize("i", range(len(CASES)), ids=lambda i: "-".join(map(str, CASES[i][:6])))
def test_attention_with_own_rows_and_mass(i):
    sv = case(i, own=True)
    sv.check(sv.run(mass=True))
    lone = case(i)
    lone.check(lone.run(mass=True, lse=False))


def test_attention_of_some_layers():
    sv = Serve(3, 5, 4, 6, 3, 64, [100, 0, 37], [5, 2, 0], seed=5)
    sv.check(sv.run(1, 2), l0=1)


def test_attention_takes_rotated_queries():
    sv = Serve(2, 5, 1, 2, 1, 128, [100, 40], [5, 2], seed=6)
    sv.check(sv.run(flags=co.CO_Q_PREROTATED), rotated=True)
    sv.check(sv.run(flags=co.CO_ATTN_SHARED_PREFIX))       # no effect


@pytest.mark.parametrize("hd,B,G", [(64, 1, 1), (64, 16, 4), (128, 16, 2), (128, 16, 4)])
@pytest.mark.parametrize("size", [0.0, 6.0, 60.0])
def test_attention_of_flat_and_peaked_softmaxes(hd, B, G, size):
    """Queries of nothing (all weights equal), and logits far from each other, which
    move the reference at every tile; keys small on some pages and large on others.
    The rounding of the queries (the second code's half step: 2^-9 of an entry) moves a
    logit by up to 2^-9 sum |q_d k_d| / sqrt(hd): at queries of 6 that sum is near
    128 * (6 * 0.8) * 0.6 / 11 = 33, so 0.06 of the logit and of a weight.  The oracle
    therefore takes the rounded queries, which leaves the rounding of the weights and
    the output to the rule.  At queries of 60 a query that rounds the other way (a
    tie, to the sine's last bit: one step, 2^-8 of 200 or so, times a key of 3) would
    move a logit by a fifth of a unit: only finite results are asked for."""
    sv = Serve(2, B, 1, G, 1, hd, [700, 90], [B, 0], seed=8, size=size)
    got = sv.run()
    if size < 60:
        sv.check(got, rounded=True)
    else:
        assert torch.isfinite(got[0].float()).all() and torch.isfinite(got[1]).all()


@pytest.mark.parametrize("hd,B,G", [(64, 1, 2), (64, 16, 4), (128, 1, 2), (128, 16, 4)])
@pytest.mark.parametrize("bytes_", [(0, 40), (100, 150), (200, 240), "up", "down"])
def test_attention_over_values_of_any_scale(bytes_, hd, B, G):
    """Value pages whose scales differ from page to page: by up to 2^50, or by 2^3 a page
    up or down (the largest, which the outputs show, first or last)."""
    sv = Serve(3, B, 1, G, 1, hd, [700, 77, 16], [0, 0, 0], seed=12, size=0.3)
    N = sv.d.num_pages
    if isinstance(bytes_, tuple):
        g = torch.Generator(device=DEV).manual_seed(12)
        b = torch.randint(*bytes_, (N,), generator=g, device=DEV)
    else:
        b = torch.full((N,), 120, device=DEV)
        row = torch.tensor([int(p) for p in sv.table[0] if p >= 0], device=DEV)
        b[row] = 40 + 3 * torch.arange(len(row), device=DEV)
        if bytes_ == "down":
            b[row] = b[row].flip(0)
    sv.cache["v_scale"][0, :, 0] = b.to(torch.uint8)
    sv.check(sv.run())


@pytest.mark.parametrize("hd,B,G", [(64, 1, 2), (128, 16, 4)])
@pytest.mark.parametrize("below", [12, 22])
def test_attention_reads_small_values_beside_large_ones(below, hd, B, G):
    """The key that has all the weight has values 2^-below of another page's: subnormal
    beside them, and still exact.  Its score is 128 (head_dim 64: 64 * 2^4 / 8) or 90.5
    (128 * 2^3 / 11.3) and the others' 0, whose weights of 2^-130 leave nothing of 2^35
    times as large values: each row is one value row, rounded once to bf16."""
    sv = Serve(1, B, 1, G, 1, hd, [32], [0], seed=14)
    sv.q.fill_(1.0)
    a, b = (int(x) for x in sv.table[0, :2])
    one = 0x38                                                     # e4m3 1.0
    sv.cache["k_pages"][0, a], sv.cache["k_pages"][0, b] = 0, 0
    sv.cache["k_pages"][0, b, 0, 5] = one
    sv.cache["k_scale"][0, b, 0] = 127 + (4 if hd == 64 else 3)
    sv.cache["v_scale"][0, a, 0], sv.cache["v_scale"][0, b, 0] = 140, 140 - below
    out, _, _ = sv.run(flags=co.CO_Q_PREROTATED)
    v = serve8.Cache8.read(sv.cache).context(sv.table, 0, 0, 0, 32)[1]
    want = torch.from_numpy(v[16 + 5]).to(DEV).float()
    assert torch.all((out[0, 0].float() - want).abs() <= want.abs() * 2 ** -8)


@pytest.mark.parametrize("hd,B,G", [(64, 1, 8), (64, 16, 4), (128, 1, 8), (128, 16, 4)])
def test_attention_is_as_exact_as_its_output_type(hd, B, G):
    """Rounding an exact result to bf16 leaves 1.7e-3 (half a step is 2^-9 to 2^-8 of an
    entry, evenly spread: 2^-8 / sqrt(12) of the entries' 1.0 .. 2.0 is 1.1e-3 to 2.3e-3);
    queries of two codes 0.7e-3, fp16 weights 0.3e-3: 1.9e-3 together, and 2.1e-3 allowed
    (bf16 weights would leave 2.4e-3)."""
    sv = Serve(4, B, 1, G, 1, hd, [3000, 2000, 1000, 300], [0, 0, 0, 0], seed=13)
    g = torch.Generator(device=DEV).manual_seed(13)
    r = lambda *n: torch.randn(n, generator=g, device=DEV).bfloat16()  # noqa: E731
    dst = [sv.table[s][t // PAGE] * PAGE + t % PAGE for s in range(4) for t in range(sv.ctx[s])]
    co.carryover_store_kv8(sv.d, len(dst), r(1, len(dst), 1, hd), r(1, len(dst), 1, hd), ints(dst),
                           sv.cache, sv.st["status"])
    out, _, _ = sv.run()
    orc, off, all_ = serve8.Cache8.read(sv.cache), 0.0, 0.0
    for s, n in enumerate(sv.ctx):
        k, v = orc.context(sv.table, s, 0, 0, n)
        q = sv.q[0, s].double().cpu().numpy().reshape(B * G, hd)
        o, _ = oracle.attend(q, np.repeat(n + np.arange(B), G), k, v, sv.theta)
        d = out[0, s].double().cpu().numpy().reshape(B * G, hd) - o
        off, all_ = off + np.sum(d * d), all_ + np.sum(o * o)
    assert math.sqrt(off / all_) <= 2.1e-3, math.sqrt(off / all_)


@pytest.mark.parametrize("hd,B,G", [(64, 1, 2), (128, 16, 4)])
def test_attention_leaves_out_pages_out_of_range(hd, B, G):
    sv = Serve(3, B, 1, G, 1, hd, [200, 77, 64], [B, 0, 0], seed=9)
    for s, p, to in ((0, 2, -5), (0, 11, sv.d.num_pages), (1, 4, 2 ** 31 - 1), (2, 0, -1), (2, 1, -1),
                     (2, 2, -1), (2, 3, -1)):
        sv.table[s][p] = to
    sv.st["page_table"].copy_(ints(sv.table))
    hidden = [(0, 2), (0, 11), (1, 4), (2, 0), (2, 1), (2, 2), (2, 3)]
    sv.table[sv.table >= sv.d.num_pages] = 0
    sv.check(sv.run(), hidden=hidden)


@pytest.mark.parametrize("hd,B,G", [(64, 1, 2), (64, 16, 4), (128, 1, 2), (128, 16, 4)])
def test_a_page_left_out_reads_nothing_of_another(hd, B, G):
    """The cache's first page was never written: codes and scales that read as NaN."""
    sv = Serve(2, B, 1, G, 1, hd, [200, 64], [B, 0], seed=9, num_pages=30, ids=range(29, 0, -1))
    for x in sv.cache.values():
        x[:, 0] = 0xFF
    for s, p in ((0, 1), (0, 6), (1, 0)):
        sv.table[s][p] = -1
    sv.st["page_table"].copy_(ints(sv.table))
    sv.check(sv.run(), hidden=[(0, 1), (0, 6), (1, 0)])


@pytest.mark.parametrize("i", [3, 4, 10, 13, 14, 15, 17])
@pytest.mark.parametrize("workgroups", [1, 3, 7])
def test_attention_in_few_slices(i, workgroups, tune):
    """A few streams walk many segments in turn, parts of them at both ends."""
    tune("attn_workgroups", workgroups)
    sv = case(i, own=i % 2 == 1)
    sv.check(sv.run(mass=i % 2 == 1))


@pytest.mark.parametrize("bad", [(-1, 0), (16 * 13 + 1, 0), (5, -1), (5, 17)])
def test_attention_of_bad_lengths_is_empty(bad):
    sv = Serve(3, 16, 1, 2, 1, 128, [200, 40, 100], [3, 0, 9], seed=10)
    out, z, _ = sv.run()
    sv.check((out, z, None))
    sv.st["ctx_len"][1], sv.st["carry_len"][1] = bad
    got, gz, gm = sv.run(mass=True)
    assert int(sv.st["status"]) == co.CO_ERR_LENGTH
    assert torch.all(got[:, 1] == 0) and torch.all(gz[:, 1] == -math.inf) and torch.all(gm[:, 1] == 0)
    # the others: the split may differ, the result not by more than both sides' rounding
    for s in (0, 2):
        assert_heads_close(got[:, s].double().cpu().numpy(), out[:, s].double().cpu().numpy(), TOL, "others")


@pytest.mark.parametrize("hd", [64, 128])
def test_attention_past_32_bit_offsets(hd):
    """Pages whose bytes lie more than 2^32 into the cache."""
    Hkv = 8
    page = Hkv * PAGE * hd
    N = 2 ** 32 // page + 600
    sv = Serve(2, 16, 1, 4 * Hkv, Hkv, hd, [300, 100], [16, 3], seed=11, num_pages=N,
               ids=list(range(N - 1, N - 40, -1)))
    small = Serve(2, 16, 1, 4 * Hkv, Hkv, hd, [300, 100], [16, 3], seed=11, num_pages=50,
                  ids=list(range(39)))
    a, b = sv.run()[0], small.run()[0]
    assert torch.equal(a, b)
    small.check((b, None, None))


def test_store_past_32_bit_offsets():
    hd, Hkv = 128, 8
    N = 2 ** 32 // (Hkv * PAGE * hd) + 3
    d, status = dims(1, 1, N, L=1, Hq=Hkv, Hkv=Hkv, hd=hd), zero()
    g = torch.Generator(device=DEV).manual_seed(1)
    cache = co.alloc_kv8(d)
    k, v = (torch.randn((1, 5, Hkv, hd), generator=g, device=DEV).bfloat16() for _ in range(2))
    dst = [(N - 1) * PAGE + 15] + [(N - 2) * PAGE + i for i in range(4)]
    co.carryover_store_kv8(d, 5, k, v, ints(dst), cache, status)
    last = {n: x[:, N - 2:] for n, x in cache.items()}
    orc = serve8.Cache8(*(np.zeros((1, 2, Hkv, PAGE, hd), np.uint8) for _ in range(2)),
                        *(np.zeros((1, 2, Hkv), np.uint8) for _ in range(2)))
    orc.store(k.double().cpu().numpy(), v.double().cpu().numpy(), [31, 0, 1, 2, 3], 2)
    check_cache(last, orc)
    assert int(status) == 0 and int(cache["k_pages"][:, :N - 2].count_nonzero()) == 0


def test_attention_repeats_bit_for_bit_and_on_another_stream():
    sv = case(5, own=True)
    first = sv.run(mass=True)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        again = sv.run(mass=True)
    torch.cuda.current_stream().wait_stream(other)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_stand_alone_mass_and_self_merge_serve_the_result():
    sv = Serve(4, 9, 2, 6, 2, 128, [150, 0, 33, 800], [9, 4, 0, 2], seed=12, own=True)
    want, wz, wm = sv.run(mass=True)
    keys = sv.own
    sv.own = [None, None]
    out, z, _ = sv.run()
    m = torch.empty_like(z)
    co.drafter_carry_mass(sv.d, 0, 2, sv.q, sv.st, z, m)
    co.drafter_self_merge(sv.d, 0, 2, sv.q, *keys, sv.st, out, z)
    assert_heads_close(out.double().cpu().numpy(), want.double().cpu().numpy(), TOL, "self merge")
    assert float((m - wm).abs().max()) <= TOL
    assert float((z - wz).abs().max()) <= TOL
