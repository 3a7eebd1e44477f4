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


@host
@pytest.mark.parametrize("x_type,y_type", [(B.FAE_F32, B.FAE_F32), (B.FAE_BF16, B.FAE_BF16)])
@pytest.mark.parametrize("parts,width", [(1, 16), (1, 64), (1, 100), (1, 513), (1, 1664), (1, 9001), (2, 7), (3, 40), (4, 100), (5, 128), (7, 16), (8, 64), (13, 64),
                                         (26, 64), (26, 256), (33, 20), (63, 512), (64, 8)])
def test_a_workspace_is_enough_for_fewer_rows(parts, width, x_type, y_type):
    """A program sizes it for its largest batch and has a smaller one at the end."""
    lib, n, before = B.load(), _norm(n_parts=parts, width=width, x_type=x_type, y_type=y_type), 0
    rows = sorted({*range(0, 3000), *range(3000, 70_000, 13), *(1 << k for k in range(16, 24)), ((1 << 31) - 1) // parts})
    for n.n_rows in rows:
        need = lib.fae_layer_norm_bwd_workspace_bytes(C.byref(n))
        assert need >= max(before, 256)
        before = need
    assert before <= 2 * 4 * (1024 + 64) * parts * (width + 3) + 512  # a row of sums for each part and workgroup, whatever the rows
