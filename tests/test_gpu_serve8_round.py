"""Serving from the 8-bit cache, the calls together as a program makes them: ragged
prompts projected to pages assigned on the device, chained rounds, requests that end
and enter; captured into a graph; on two streams at once.

Codes are compared exactly with the oracle's store of the rows that the bf16 path
writes for the same inputs (both take the same projection); attention by the rule
of tests/test_gpu_serve8.py over the cache's own contents."""
import numpy as np
import pytest

from synth import workloads as wl

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import oracle  # noqa: E402
import paper_2609_14717_amd as co  # noqa: E402
from helpers import gather_carry, head_err  # noqa: E402
from oracle import PAGE, SKIP, serve8  # noqa: E402
from synth.scenario import Scenario, Scenario8  # noqa: E402
from test_gpu_serve8 import TOL, check_cache, ints, np_, space  # noqa: E402

BASE = wl.RAGGED32.replace(S=5, L=2, Dcat=256, d=128, ctx_lo=20, ctx_hi=400, rounds=6,
                           accept=("geom", 0.25))
WORKLOADS = {
    "64": BASE,
    "128": BASE.replace(hd=128, Hq=8, Hkv=2, L=3, S=3, theta=1e6),
    "one row": BASE.replace(B=1, Hq=6, Hkv=3, S=7),
    "wide": BASE.replace(hd=128, Hq=16, Hkv=8, Dcat=1536, d=768, L=1, S=9, B=7, ctx_lo=1, theta=1e6),
}


def attend_check(sc, out, lse, q, seqs=None):
    """The round's attention against the oracle over what cache and carry segment hold."""
    w, st = sc.w, sc.st
    orc, table = serve8.Cache8.read(sc.cache), np_(st["page_table"])
    ctx, car = np_(st["ctx_len"]), np_(st["carry_len"])
    G, worst = w.Hq // w.Hkv, 0.0
    go, gz, qd = (t.double().cpu().numpy() for t in (out, lse, q))
    for s in range(w.S):
        n, pos = int(ctx[s]), int(ctx[s]) + np.arange(w.B)
        for layer in range(w.L):
            ku, vu = gather_carry(st, s, layer, int(car[s]))
            for h in range(w.Hkv):
                k, v = orc.context(table, s, layer, h, n)
                rows = qd[layer, s, :, h * G:(h + 1) * G].reshape(w.B * G, w.hd)
                o, z = oracle.attend(rows, np.repeat(pos, G), np.concatenate([k, ku[:, h]]),
                                     np.concatenate([v, vu[:, h]]), w.theta)
                worst = max(worst, head_err(go[layer, s, :, h * G:(h + 1) * G].reshape(w.B * G, w.hd), o))
                fine = np.isfinite(z)
                assert np.abs(gz[layer, s, :, h * G:(h + 1) * G].ravel() - z)[fine].max(initial=0) <= TOL
    assert worst <= TOL, worst
    return worst


def rows_of_round(sc, rt):
    """Keys and values [L][S * B][Hkv][hd] that a round wrote to the bf16 cache."""
    w = sc.w
    dst = np_(rt["row_dst"]).reshape(-1)
    k, v = (np.zeros((w.L, len(dst), w.Hkv, w.hd)) for _ in range(2))
    keep = dst >= 0
    p, t = torch.tensor(dst[keep] // PAGE).cuda(), torch.tensor(dst[keep] % PAGE).cuda()
    for layer in range(w.L):
        k[layer, keep] = sc.st["k_cache"][layer][p, :, t].double().cpu().numpy()
        v[layer, keep] = sc.st["v_cache"][layer][p, :, :, t].double().cpu().numpy()
    return k, v, dst


@pytest.mark.parametrize("name", WORKLOADS)
def test_rounds(name):
    """Chained rounds: the bf16 path's rounds give the route, the carry segment and the
    rows, bit for bit; the oracle's store of those rows gives the codes."""
    w = WORKLOADS[name]
    ref, sc = Scenario(w), Scenario8(w)
    assert co.carryover_read_status(sc.st) == 0
    for r in range(4):
        ref_in = ref.round_inputs(r)
        out, lse = ref.new_output()
        co.carryover_round(ref.dims, ref.W, *ref_in[:1], *ref_in[2:4], ref_in[1], ref.st, ref.rt, out,
                           lse, 0, ref.ws)
        orc = serve8.Cache8.read(sc.cache)
        out8, lse8 = sc.new_output()
        sc.round(ref_in, out8, lse8)
        assert co.carryover_read_status(sc.st) == 0
        for x in ("accept_len", "row_pos"):
            assert torch.equal(ref.rt[x], sc.rt[x])
        for x in ("ctx_len", "carry_len", "k_carry", "v_carry"):
            assert torch.equal(ref.st[x], sc.st[x]), x
        k, v, _ = rows_of_round(ref, ref.rt)
        dst = np_(sc.rt["row_dst"]).reshape(-1)
        table = np_(sc.st["page_table"])
        pos = np_(sc.rt["row_pos"])
        acc = np_(sc.rt["accept_len"])
        for s in range(w.S):
            for j in range(w.B):
                want = (table[s][pos[s, j] // PAGE] * PAGE + pos[s, j] % PAGE if j < acc[s]
                        else -1 - (j - acc[s]))
                assert dst[s * w.B + j] == want
        assert orc.store(k, v, dst, sc.dims.num_pages) == 0
        check_cache(sc.cache, orc)
        attend_check(sc, out8, lse8, ref_in[1])


def test_round_is_its_steps_bit_for_bit():
    w = WORKLOADS["128"]
    a, b = Scenario8(w), Scenario8(w)
    for x in a.cache:
        assert torch.equal(a.cache[x], b.cache[x])
    for r in range(2):
        hidden, q, draft, target = a.round_inputs(r)[:4]
        out, lse = a.new_output()
        out2, lse2 = b.new_output()
        a.round((hidden, q, draft, target), out, lse)
        b.assign(b.st["ctx_len"], w.B)
        co.carryover_route(b.dims, draft, target, 0, b.st, b.rt)
        co.carryover_project_kv8(b.dims, b.W, hidden, b.rt, b.st, b.cache, b.ws)
        ws = space(b.dims, co.CO_WS_ATTENTION_KV8)
        co.drafter_block_attention_kv8(b.dims, 0, w.L, q, None, None, b.st, b.cache, out2, lse2, None, 0, ws)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
        assert all(torch.equal(a.cache[x], b.cache[x]) for x in a.cache)
        assert all(torch.equal(a.rt[x], b.rt[x]) for x in a.rt)


@pytest.mark.parametrize("flags", [co.CO_BASELINE_MODE, co.CO_ROUTE_CARRY_ONLY, co.CO_ROUTE_ACCEPT_ALL])
def test_round_modes(flags):
    w = WORKLOADS["64"]
    sc = Scenario8(w)
    before = {x: sc.cache[x].clone() for x in sc.cache}
    inputs = sc.round_inputs(0)
    out, lse = sc.new_output()
    sc.round(inputs, out, lse, flags)
    assert co.carryover_read_status(sc.st) == 0
    if flags == co.CO_ROUTE_CARRY_ONLY:       # nothing is committed
        assert all(torch.equal(before[x], sc.cache[x]) for x in before)
    if flags != co.CO_ROUTE_CARRY_ONLY:
        attend_check(sc, out, lse, inputs[1])


def test_variants_of_the_projection_reach_the_rows():
    """Separate projector and both norms: the rows of the bf16 path, in codes."""
    w = WORKLOADS["64"].replace(ctx_lo=40, ctx_hi=90)
    for kw in (dict(separate_projector=True), dict(z_norm=True, k_norm=True), dict(fold_e=False)):
        ref, sc = Scenario(w, **kw), Scenario8(w, **kw)
        inputs = ref.round_inputs(0)
        out, lse = ref.new_output()
        co.carryover_round(ref.dims, ref.W, inputs[0], inputs[2], inputs[3], inputs[1], ref.st, ref.rt,
                           out, lse, 0, ref.ws)
        orc = serve8.Cache8.read(sc.cache)
        sc.round(inputs, out, lse)
        k, v, _ = rows_of_round(ref, ref.rt)
        orc.store(k, v, np_(sc.rt["row_dst"]).reshape(-1), sc.dims.num_pages)
        check_cache(sc.cache, orc)
        assert torch.equal(ref.st["k_carry"], sc.st["k_carry"])


def prompts(lengths, w, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((sum(lengths), w.Dcat), generator=g, device="cuda").bfloat16()


@pytest.mark.parametrize("lengths", [[1], [17, 0, 33, 1, 16], [700, 3, 0, 129, 64]])
def test_ragged_prompts_enter_and_leave(lengths):
    """Prompts of any lengths: pages assigned, rows mapped and projected in one call over
    packed rows; then they end and others enter on the same pages."""
    w = BASE.replace(S=len(lengths), Dcat=256, d=128, ctx_lo=0, ctx_hi=0, ctx_mode="projected")
    P = 60
    d = co.make_dims(w.S, w.B, w.Dcat, w.d, w.L, w.Hq, w.Hkv, w.hd, P, 130, "bf16", w.theta)
    sc = Scenario8(w.replace(ctx_lo=0, ctx_hi=0))      # weights
    pool, cache = co.alloc_page_pool(d), co.alloc_kv8(d)
    st = co.alloc_state(d, np.full((w.S, P), -1), committed=False)
    st["page_table"] = pool["page_table"]
    ws = space(d, co.CO_WS_ASSIGN_PAGES)
    for turn, n in enumerate((lengths, lengths[::-1])):
        st["ctx_len"].zero_()
        co.carryover_assign_pages(d, ints([0] * w.S), 0, pool, st["status"], ws)   # the ones before end
        assert int(pool["free_count"]) == 130
        co.carryover_assign_pages(d, ints(n), w.B, pool, st["status"], ws)
        rows, pad = sum(n), 5
        h = torch.cat([prompts(n, w, turn), torch.full((pad, w.Dcat), float("nan")).cuda().bfloat16()])
        start = ints(np.concatenate([[0], np.cumsum(n)]))
        rt = co.alloc_route(1, rows + pad)
        co.carryover_slot_map(d, rows + pad, start, st["ctx_len"], st["page_table"], rt["row_pos"],
                              rt["row_dst"], st["status"])
        assert np.all(np_(rt["row_dst"])[0, rows:] == SKIP)
        pd = co.make_dims(1, rows + pad, w.Dcat, w.d, w.L, w.Hq, w.Hkv, w.hd, P, 130, "bf16", w.theta)
        orc = serve8.Cache8.read(cache)
        co.carryover_project_kv8(pd, sc.W, h, rt, st, cache, space(pd, co.CO_WS_PROJECT_KV8))
        # the bf16 path's rows, by the same route
        full = co.alloc_state(pd, np.zeros((1, P)))
        co.carryover_project_kv(pd, sc.W, h, rt, full, space(pd, co.CO_WS_PROJECT))
        dst = np_(rt["row_dst"])[0]
        keep = dst >= 0
        k, v = (np.zeros((w.L, rows + pad, w.Hkv, w.hd)) for _ in range(2))
        p, t = torch.tensor(dst[keep] // PAGE).cuda(), torch.tensor(dst[keep] % PAGE).cuda()
        for layer in range(w.L):
            k[layer, keep] = full["k_cache"][layer][p, :, t].double().cpu().numpy()
            v[layer, keep] = full["v_cache"][layer][p, :, :, t].double().cpu().numpy()
        orc.store(k, v, dst, 130)
        check_cache(cache, orc)
        assert int(st["status"]) == 0 and int(full["status"]) == 0


def test_captured_in_a_graph():
    """Assignment, slot map, store, round and attention in one graph, replayed with eager
    work in between; every replay equals the eager calls from the same state."""
    w = WORKLOADS["128"]
    sc = Scenario8(w)
    inputs = sc.round_inputs(0)
    out, lse = sc.new_output()
    out2, lse2 = sc.new_output()
    n = torch.from_numpy(sc.ctx0.astype(np.int32)).cuda()
    longer = n + 40
    rows = 40 * w.S
    start = ints(np.arange(w.S + 1) * 40)
    k, v = (torch.randn((w.L, rows, w.Hkv, w.hd), device="cuda").bfloat16() for _ in range(2))
    pos, dst = torch.zeros((2, rows), dtype=torch.int32, device="cuda")
    ws = space(sc.dims, co.CO_WS_ATTENTION_KV8)
    snap = {x: sc.cache[x].clone() for x in sc.cache}

    def work():
        for x in snap:
            sc.cache[x].copy_(snap[x])
        sc.st["ctx_len"].copy_(n)
        sc.assign(n)
        sc.assign(longer, w.B)
        co.carryover_slot_map(sc.dims, rows, start, n, sc.st["page_table"], pos, dst, sc.st["status"])
        co.carryover_store_kv8(sc.dims, rows, k, v, dst, sc.cache, sc.st["status"])
        sc.st["ctx_len"].copy_(longer)
        sc.round(inputs, out, lse)
        co.drafter_block_attention_kv8(sc.dims, 0, w.L, inputs[1], None, None, sc.st, sc.cache, out2,
                                       lse2, None, 0, ws)

    seen = lambda: [t.clone() for t in (out, lse, out2, lse2, pos, dst, *sc.cache.values(),  # noqa: E731
                                        *sc.st.values(), *sc.rt.values(), sc.pool["held"],
                                        sc.pool["free_count"]) if t is not None]
    work()
    work()
    want = seen()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            work()
    torch.cuda.current_stream().wait_stream(side)
    for replay in range(4):
        for t in (out, lse, out2, pos):
            t.fill_(5)
        g.replay()
        torch.cuda.synchronize()
        assert co.carryover_read_status(sc.st) == 0
        got = seen()
        assert all(torch.equal(x, y) for x, y in zip(want, got)), replay
        if replay == 1:
            work()                                   # the program's own eager work
            torch.cuda.synchronize()


def test_two_streams_at_once():
    """Calls on distinct states and workspaces, in flight together."""
    a, b = (Scenario8(WORKLOADS[x]) for x in ("128", "wide"))
    jobs = []
    for sc in (a, b):
        inputs = sc.round_inputs(0)
        out, lse = sc.new_output()
        ctx = sc.st["ctx_len"].clone()
        jobs.append((sc, inputs, out, lse, ctx, torch.cuda.Stream()))
    want = []
    for sc, inputs, out, lse, ctx, _ in jobs:
        sc.round(inputs, out, lse)
        sc.st["ctx_len"].copy_(ctx)
        sc.round(inputs, out, lse)                   # the same rows again: the same pages
        want.append((out.clone(), lse.clone()))
    torch.cuda.synchronize()
    for _ in range(5):
        for sc, inputs, out, lse, ctx, stream in jobs:
            with torch.cuda.stream(stream):
                out.fill_(3)
                sc.st["ctx_len"].copy_(ctx)
                sc.round(inputs, out, lse)
    torch.cuda.synchronize()
    for (sc, _, out, lse, *_), (o, z) in zip(jobs, want):
        assert torch.equal(out, o) and torch.equal(lse, z)


def test_pool_that_runs_out_leaves_rounds_safe():
    """A sequence without a page for its window reports it and is left as it was."""
    w = WORKLOADS["64"].replace(S=3, ctx_lo=100, ctx_hi=100)
    sc = Scenario8(w)
    sc.pool["free_count"].zero_()                    # every other page is someone else's
    inputs = sc.round_inputs(0)
    out, lse = sc.new_output()
    longer = sc.st["ctx_len"] + 100
    sc.assign(longer, w.B)
    assert co.carryover_read_status(sc.st) == co.CO_ERR_POOL
    sc.st["status"].zero_()
    sc.st["ctx_len"].copy_(longer)                   # a program that goes on regardless
    sc.round(inputs, out, lse)
    assert co.carryover_read_status(sc.st) in (co.CO_ERR_POOL, co.CO_ERR_PAGE_RANGE)
    assert torch.isfinite(out.float()).all()
