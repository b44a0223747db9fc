"""GPU: calls on the 8-bit cache at the edge of what they take, against the oracle."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2609_14717_amd as co  # noqa: E402
from oracle import serve8  # noqa: E402
from synth.scenario import Scenario8  # noqa: E402
from test_gpu_serve8 import check_cache, dims, ints, zero  # noqa: E402
from test_gpu_serve8_round import WORKLOADS, attend_check  # noqa: E402


def test_store_for_more_sequences_than_a_window_has_rows():
    g = torch.Generator(device="cuda").manual_seed(3)
    small = dims(1, 4, 4, L=2, Hq=2, Hkv=2)
    cache, status = co.alloc_kv8(small), zero()
    orc = serve8.Cache8.read(cache)
    k, v = (torch.randn((2, 5, 2, 64), generator=g, device="cuda").bfloat16() for _ in range(2))
    dst = [17, 18, -1, 32, 33]
    d = dims(1 << 24, 4, 4, B=16, L=2, Hq=2, Hkv=2)
    co.carryover_store_kv8(d, 5, k, v, ints(dst), cache, status)
    orc.store(k.double().cpu().numpy(), v.double().cpu().numpy(), dst, 4)
    check_cache(cache, orc)
    assert int(status) == 0


@pytest.mark.parametrize("name", WORKLOADS)
def test_a_round_that_only_carries(name):
    """CO_ROUTE_CARRY_ONLY: every row of the window that was not accepted goes to the carry
    segment, the cache stays, and the round attends over both."""
    w = WORKLOADS[name]
    sc = Scenario8(w)
    before, ctx = {x: sc.cache[x].clone() for x in sc.cache}, sc.st["ctx_len"].clone()
    inputs = sc.round_inputs(0)
    out, lse = sc.new_output()
    sc.round(inputs, out, lse, co.CO_ROUTE_CARRY_ONLY)
    assert co.carryover_read_status(sc.st) == 0
    assert all(torch.equal(before[x], sc.cache[x]) for x in before)
    assert w.B == 1 or int(sc.st["carry_len"].max()) > 0
    attend_check(sc, out, lse, inputs[1])
