"""Host checks of the calls on the 8-bit cache and next to them, at the edge of what they
take (no compute call runs here: no GPU is needed)."""
import pytest

import paper_2609_14717_amd as co
from test_serve8_host import BIG, FAKE, _dims, _rc, _state, attend, needs_lib, project, round_, store


@needs_lib
def test_a_store_is_bounded_by_its_own_rows():
    """Its rows are num_rows, whatever num_seqs and block say; a window's are the others'."""
    for S, B in ((1 << 24, 16), (1 << 28, 1), (1, 1 << 28), (1 << 14, 1 << 14)):
        d = _dims(S=S, B=B)
        assert _rc(store, d, n=0) == co.CO_OK
        assert _rc(store, d, n=1 << 28) == co.CO_ERR_UNSUPPORTED
        assert _rc(project, d) == _rc(round_, d) == _rc(attend, d) == co.CO_ERR_UNSUPPORTED
        for which in (co.CO_WS_PROJECT_KV8, co.CO_WS_ATTENTION_KV8, co.CO_WS_ROUND_KV8):
            assert co.workspace_bytes(d, which) == 0
    assert _rc(store, _dims(S=(1 << 30) - 1, B=1), n=0) == co.CO_OK    # every call's bound


FULL = dict(_state(), k_cache=FAKE, v_cache=FAKE)
LAYERS = {
    "attention": lambda d, l0, n: co.drafter_block_attention(
        d, l0, n, FAKE, FULL, FAKE, None, 0, FAKE, stream=0, ws_bytes=BIG),
    "ext": lambda d, l0, n: co.drafter_block_attention_ext(
        d, l0, n, FAKE, FAKE, FAKE, FULL, FAKE, None, None, 0, FAKE, stream=0, ws_bytes=BIG),
    "kv8": lambda d, l0, n: attend(d, l0=l0, layers=n),
    "backward": lambda d, l0, n: co.drafter_block_attention_backward(
        d, l0, n, FAKE, FULL, FAKE, FAKE, FAKE, 1, *[FAKE] * 5, FAKE, stream=0, ws_bytes=BIG),
    "mass": lambda d, l0, n: co.drafter_carry_mass(d, l0, n, FAKE, _state(), FAKE, FAKE, stream=0),
    "merge": lambda d, l0, n: co.drafter_self_merge(
        d, l0, n, FAKE, FAKE, FAKE, _state(), FAKE, FAKE, stream=0),
}


@needs_lib
@pytest.mark.parametrize("call", LAYERS.values(), ids=LAYERS)
def test_layer_ranges_past_32_bits_are_refused_by_every_call(call):
    big, d = 2 ** 31 - 1, _dims(L=3)
    for l0, n in ((0, 4), (3, 1), (1, big), (big, 1), (big, big), (big - 1, 3), (-1, 1), (0, -1)):
        assert _rc(call, d, l0, n) == co.CO_ERR_INVALID_ARG, (l0, n)
    for l0 in range(4):
        assert _rc(call, _dims(L=3, S=0), l0, 3 - l0) == co.CO_OK


@needs_lib
@pytest.mark.parametrize("call", LAYERS.values(), ids=LAYERS)
@pytest.mark.parametrize("S", [0, 1])
def test_query_rows_past_32_bits_are_refused(call, S):
    """block * heads of a group = 2^32 and 2^32 + 17: neither no row nor 17."""
    for B, G in ((1 << 29, 8), (1 << 28, 16), (613566759, 7)):
        d = _dims(S=S, B=B, Hq=G, Hkv=1)
        assert _rc(call, d, 0, 1) == co.CO_ERR_UNSUPPORTED, (B, G)
        for which in (co.CO_WS_ATTENTION, co.CO_WS_ROUND, co.CO_WS_ATTENTION_KV8, co.CO_WS_ROUND_KV8):
            assert co.workspace_bytes(d, which) == 0
