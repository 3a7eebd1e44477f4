"""What the softmax loss's backward with the forward's losses refuses, before anything is launched (test_rows_refusals.py says how)."""
import ctypes as C

import pytest

from paper_2103_00686_amd import binding as B
from test_rows_refusals import _ctx, host

X, W, T, L, E, M, G, GX, GW, GB, WS = (k << 40 for k in range(1, 12))  # far apart


def _what(**kw):
    s = B._SoftmaxLoss(10, 500, 64, B.FAE_F32, 1.0, 32, T, None)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _kept(what, x=X, xs=64, w=W, ws=64, lse=E, loss=L, mean=M, g=G, gx=GX, gxs=64, gw=GW, gws=64, gb=GB, at=WS, n=1 << 38):
    return B.load().fae_softmax_loss_bwd_kept(_ctx(), C.byref(what) if what else None, C.c_void_p(x), C.c_int64(xs), C.c_void_p(w), C.c_int64(ws),
                                              C.c_void_p(lse), C.c_void_p(loss), C.c_void_p(mean), C.c_void_p(g), C.c_void_p(gx), C.c_int64(gxs),
                                              C.c_void_p(gw), C.c_int64(gws), C.c_void_p(gb), C.c_void_p(at), C.c_size_t(n))


@host
@pytest.mark.parametrize("bad", [dict(loss=L + 2), dict(loss=GX), dict(loss=GW + 400 * 256), dict(loss=GB - 4), dict(at=L - 64), dict(lse=0), dict(g=0), dict(x=0), dict(gx=X),
                                 dict(gw=W), dict(gxs=63), dict(gb=E), dict(at=WS + 8)])
def test_buffers(bad):
    assert _kept(_what(), **bad) == B.FAE_EINVAL


@host
def test_workspace_and_nulls():
    assert _kept(_what(), n=64) == B.FAE_ENOSPC and _kept(_what(), loss=0, n=64) == B.FAE_ENOSPC
    assert _kept(None) == B.FAE_EINVAL and _kept(_what(width=0)) == B.FAE_EINVAL


def _refused(what, **kw):
    """The library's text: a refusal of sizes, or of the workspace behind it."""
    ctx = _ctx()
    args = dict(x=1 << 45, w=1 << 46, lse=1 << 47, g=1 << 48, gx=1 << 49, gw=1 << 50, gb=1 << 51, mean=1 << 52)
    args.update(kw)
    rc = B.load().fae_softmax_loss_bwd(ctx, C.byref(what), C.c_void_p(args["x"]), C.c_int64(what.width), C.c_void_p(args["w"]), C.c_int64(what.width),
                                       C.c_void_p(args["lse"]), C.c_void_p(args["mean"]), C.c_void_p(args["g"]), C.c_void_p(args["gx"]), C.c_int64(what.width),
                                       C.c_void_p(args["gw"]), C.c_int64(what.width), C.c_void_p(args["gb"]), C.c_void_p(1 << 53), C.c_size_t(64))
    assert rc in (B.FAE_EINVAL, B.FAE_ENOSPC)
    return rc


@host
@pytest.mark.parametrize("type", [B.FAE_F32, B.FAE_BF16, B.FAE_F16])
def test_more_held_rows_than_a_grid_takes(type):
    """512 threads for 128 rows of a width above 128: from 2^30 - 127 on they are 2^32."""
    most = (1 << 30) - 128
    assert (most + 127) // 128 * 512 < 1 << 32 <= (most + 1 + 127) // 128 * 512
    for width, n, rc in ((129, most, B.FAE_ENOSPC), (129, most + 1, B.FAE_EINVAL), (256, 1 << 30, B.FAE_EINVAL), (128, 0x7ffeffff, B.FAE_ENOSPC)):
        what = _what(n_classes=n, width=width, type=type)
        assert _refused(what) == rc and _refused(what, gw=0) == rc and _refused(what, gw=0, gb=0) == B.FAE_ENOSPC
        what = _what(n_rows=n, width=width, type=type, targets=1 << 54)
        assert _refused(what) == B.FAE_ENOSPC and _refused(what, gx=0, mean=0) == B.FAE_ENOSPC and _refused(what, mean=0) == rc
        assert B.load().fae_softmax_loss_fwd(_ctx(), C.byref(what), C.c_void_p(1 << 45), C.c_int64(width), C.c_void_p(1 << 46), C.c_int64(width), None, None,
                                             C.c_void_p(1 << 52), C.c_void_p(1 << 53), C.c_size_t(64)) == rc
