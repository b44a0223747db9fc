"""Host checks of the calls on the 8-bit cache and next to them, at the edge of what they
take (no compute call runs here: no GPU is needed)."""
import pytest

import paper_2609_14717_amd as co
from test_serve8_host import _dims, _rc, attend, needs_lib, project, round_, store


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
