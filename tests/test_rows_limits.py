"""Layer norm's limits and workspaces, on the host alone (test_rows_refusals.py says how)."""
import ctypes as C

import pytest

from paper_2103_00686_amd import binding as B
from test_rows_refusals import _bwd, _fwd, _norm, host


@host
@pytest.mark.parametrize("parts", [1, 2, 3, 7, 26, 64])
def test_the_most_rows(parts):
    """n_rows * n_parts < 2^31, also where the parts do not divide it: a null buffer is what such a call is refused for."""
    most = ((1 << 31) - 1) // parts
    n = _norm(n_rows=most, n_parts=parts, width=1)
    rc, text = _fwd(n, x=0, xs=parts, ys=parts)
    assert rc == B.FAE_EINVAL and "null x" in text
    assert B.load().fae_layer_norm_bwd_workspace_bytes(C.byref(n)) > 0
    n.n_rows = most + 1
    rc, text = _fwd(n, x=0, xs=parts, ys=parts)
    assert rc == B.FAE_EINVAL and "n_rows" in text
    assert B.load().fae_layer_norm_bwd_workspace_bytes(C.byref(n)) == 0


@host
@pytest.mark.parametrize("n_rows", [1 << 31, 1 << 58, (1 << 63) - 1])
def test_products_that_overflow(n_rows):
    for parts in (1, 64):
        n = _norm(n_rows=n_rows, n_parts=parts, width=1)
        assert _fwd(n)[0] == B.FAE_EINVAL and _bwd(n) == B.FAE_EINVAL
        assert B.load().fae_layer_norm_bwd_workspace_bytes(C.byref(n)) == 0
