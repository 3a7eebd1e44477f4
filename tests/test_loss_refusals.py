"""What the softmax loss and the gradients' norm and clipping refuse, before anything is launched (test_rows_refusals.py says how)."""
import ctypes as C

import pytest
import torch

from paper_2103_00686_amd import binding as B
from test_rows_refusals import _ctx, host

X, W, T, L, E, M, G, GX, GW, GB, WS = (k << 40 for k in range(1, 12))  # far apart
BIG = 1 << 38


def _what(**kw):
    s = B._SoftmaxLoss(10, 500, 64, B.FAE_F32, 1.0, 32, T, None)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _fwd(what, x=X, xs=64, w=W, ws=64, loss=L, lse=E, mean=M, at=WS, n=BIG):
    return B.load().fae_softmax_loss_fwd(_ctx(), C.byref(what) if what else None, C.c_void_p(x), C.c_int64(xs), C.c_void_p(w), C.c_int64(ws),
                                         C.c_void_p(loss), C.c_void_p(lse), C.c_void_p(mean), C.c_void_p(at), C.c_size_t(n))


def _bwd(what, x=X, xs=64, w=W, ws=64, lse=E, mean=M, g=G, gx=GX, gxs=64, gw=GW, gws=64, gb=GB, at=WS, n=BIG):
    return B.load().fae_softmax_loss_bwd(_ctx(), C.byref(what) if what else None, C.c_void_p(x), C.c_int64(xs), C.c_void_p(w), C.c_int64(ws),
                                         C.c_void_p(lse), C.c_void_p(mean), C.c_void_p(g), C.c_void_p(gx), C.c_int64(gxs), C.c_void_p(gw),
                                         C.c_int64(gws), C.c_void_p(gb), C.c_void_p(at), C.c_size_t(n))


@host
@pytest.mark.parametrize("bad", [dict(n_rows=-1), dict(n_rows=1 << 31), dict(n_rows=1 << 62), dict(n_classes=0), dict(n_classes=-4), dict(n_classes=1 << 31), dict(width=0),
                                 dict(width=B.FAE_LOSS_MAX_WIDTH + 1), dict(width=-1), dict(type=3), dict(type=-1), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(target_bits=0), dict(target_bits=16), dict(targets=0), dict(targets=T + 2),
                                 dict(targets=T + 4, target_bits=64), dict(bias=X + 2)])
def test_descriptions(bad):
    assert _fwd(_what(**bad)) == B.FAE_EINVAL
    assert _bwd(_what(**bad)) == B.FAE_EINVAL


@host
@pytest.mark.parametrize("bad", [dict(x=0), dict(w=0), dict(x=X + 2), dict(w=W + 1), dict(xs=63), dict(ws=0), dict(xs=1 << 62), dict(at=WS + 8)])
def test_inputs(bad):
    assert _fwd(_what(), **bad) == B.FAE_EINVAL
    assert _bwd(_what(), **bad) == B.FAE_EINVAL


@host
@pytest.mark.parametrize("bad", [dict(loss=L + 2), dict(lse=E + 1), dict(mean=M + 3), dict(loss=E), dict(loss=E + 36), dict(mean=X), dict(mean=W + 499 * 256), dict(lse=T),
                                 dict(at=X), dict(at=M - 16)])
def test_outputs(bad):
    assert _fwd(_what(), **bad) == B.FAE_EINVAL


@host
@pytest.mark.parametrize("bad", [dict(lse=0), dict(g=0), dict(lse=E + 1), dict(gx=GX + 1), dict(gw=GW + 2), dict(gb=GB + 1), dict(gxs=63), dict(gws=10), dict(gx=X), dict(gx=GW),
                                 dict(gw=W), dict(gw=X), dict(gb=E), dict(gb=G - 4), dict(gx=M), dict(at=GW)])
def test_backward_buffers(bad):
    assert _bwd(_what(), **bad) == B.FAE_EINVAL


@host
def test_workspaces():
    lib = B.load()
    for what in (_what(), _what(n_rows=100_000, n_classes=7), _what(n_rows=1, n_classes=1 << 24, type=B.FAE_BF16)):
        f, b = lib.fae_softmax_loss_fwd_workspace_bytes(C.byref(what)), lib.fae_softmax_loss_bwd_workspace_bytes(C.byref(what))
        assert 0 < f < b
        far = dict(x=X, w=1 << 50)
        assert _fwd(what, n=f - 1, **far) == B.FAE_ENOSPC and _fwd(what, at=0, **far) == B.FAE_ENOSPC
        assert _bwd(what, n=b - 1, gw=1 << 51, **far) == B.FAE_ENOSPC and _bwd(what, at=0, gw=1 << 51, **far) == B.FAE_ENOSPC
    for bad in (_what(width=0), _what(n_rows=-1), _what(n_classes=0), _what(type=9)):
        assert lib.fae_softmax_loss_fwd_workspace_bytes(C.byref(bad)) == 0 and lib.fae_softmax_loss_bwd_workspace_bytes(C.byref(bad)) == 0
    assert lib.fae_softmax_loss_fwd_workspace_bytes(None) == 0 and lib.fae_softmax_loss_bwd_workspace_bytes(None) == 0


@host
@pytest.mark.parametrize("type", [B.FAE_F32, B.FAE_BF16])
@pytest.mark.parametrize("width", [16, 100, 256])
def test_a_workspace_is_enough_for_smaller_calls(type, width):
    lib = B.load()
    sizes = [0, 1, 5, 31, 32, 33, 100, 127, 128, 129, 1000, 2048, 5003, 16384, 30_000, 65_536, 70_000, 131_072, 1_000_000, 40_000_000, 0x7ffeffff]
    for query in (lib.fae_softmax_loss_fwd_workspace_bytes, lib.fae_softmax_loss_bwd_workspace_bytes):
        need = {(n, v): query(C.byref(_what(n_rows=n, n_classes=v, width=width, type=type))) for n in sizes for v in sizes[1:]}
        for (n, v), k in need.items():
            assert k > 0
            i, j = sizes.index(n), sizes.index(v)
            if i:
                assert need[sizes[i - 1], v] <= k
            if j > 1:
                assert need[n, sizes[j - 1]] <= k


@host
def test_nulls():
    lib = B.load()
    assert _fwd(None) == B.FAE_EINVAL and _bwd(None) == B.FAE_EINVAL
    what = _what()
    assert lib.fae_softmax_loss_fwd(None, C.byref(what), None, C.c_int64(64), None, C.c_int64(64), None, None, None, None, C.c_size_t(0)) == B.FAE_EINVAL
    assert lib.fae_grad_norm(None, C.c_int32(0), None, C.c_float(1), None, None, C.c_size_t(0)) == B.FAE_EINVAL
    assert lib.fae_grad_clip(None, C.c_int32(0), None, C.c_float(1), C.c_float(1), None, None, C.c_size_t(0)) == B.FAE_EINVAL


def _grads(*tensors):
    arr = (B._Grad * max(len(tensors), 1))()
    for i, (g, o, n, t) in enumerate(tensors):
        arr[i] = B._Grad(g, o, n, t)
    return arr, len(tensors)


def _norm(tensors, scale=1.0, norm=L, ws=WS, n=1 << 20, count=None):
    arr, k = _grads(*tensors)
    return B.load().fae_grad_norm(_ctx(), C.c_int32(k if count is None else count), arr, C.c_float(scale), C.c_void_p(norm), C.c_void_p(ws), C.c_size_t(n))


def _clip(tensors, scale=1.0, most=1.0, norm=L, ws=WS, n=1 << 20, count=None):
    arr, k = _grads(*tensors)
    return B.load().fae_grad_clip(_ctx(), C.c_int32(k if count is None else count), arr, C.c_float(scale), C.c_float(most), C.c_void_p(norm), C.c_void_p(ws), C.c_size_t(n))


@host
@pytest.mark.parametrize("bad", [(0, X, 5, 0), (X + 2, X + 2, 5, 0), (X + 1, X + 1, 5, 1), (X, X, -1, 0), (X, X, 1 << 36, 0), (X, X, 5, 3), (X, X, 5, -1)])
def test_gradients(bad):
    assert _norm([bad]) == B.FAE_EINVAL and _clip([bad]) == B.FAE_EINVAL


@host
def test_gradients_arguments():
    fine = [(X, X, 5, 0)]
    for call in (_norm, _clip):
        assert call(fine, scale=float("nan")) == B.FAE_EINVAL and call(fine, scale=float("inf")) == B.FAE_EINVAL
        assert call(fine, norm=L + 2) == B.FAE_EINVAL and call(fine, ws=WS + 8) == B.FAE_EINVAL
        assert call(fine, ws=0) == B.FAE_ENOSPC and call(fine, n=8) == B.FAE_ENOSPC
        assert call(fine, count=-1) == B.FAE_EINVAL and call(fine, count=B.FAE_MAX_GRADS + 1) == B.FAE_EINVAL
    assert _norm(fine, norm=0) == B.FAE_EINVAL
    assert _norm(fine, norm=X + 8) == B.FAE_EINVAL and _norm(fine, ws=X) == B.FAE_EINVAL
    assert _clip(fine, most=-1.0) == B.FAE_EINVAL and _clip(fine, most=float("nan")) == B.FAE_EINVAL
    assert _clip([(X, 0, 5, 0)]) == B.FAE_EINVAL and _clip([(X, W + 2, 5, 0)]) == B.FAE_EINVAL


@host
@pytest.mark.parametrize("tensors", [[(X, X, 5, 0), (X, X, 5, 0)], [(X, W, 5, 0), (G, W, 5, 0)], [(X, X + 4, 5, 0)], [(X, W, 5, 0), (W + 16, G, 5, 0)],
                                     [(X, X, 500, 0), (X + 100, X + 100, 5, 1)], [(X, L, 5, 0)], [(X, WS, 5, 0)], [(X, X, 5, 0), (X + 8, W, 2, 0), (X, G, 1, 0)]])
def test_outputs_on_other_tensors(tensors):
    assert _clip(tensors) == B.FAE_EINVAL
    assert _clip(tensors[::-1]) == B.FAE_EINVAL


def test_tensors_of_another_kind():
    """The binding's own checks."""
    cpu = torch.zeros((4, 64))
    with pytest.raises(TypeError):
        B.SoftmaxLoss(4, 4, 64, torch.zeros(4)).c(0)
    with pytest.raises(ValueError):
        B.SoftmaxLoss(4, 4, 64, torch.zeros(5, dtype=torch.int32)).c(0)
    with pytest.raises(TypeError):
        B.SoftmaxLoss(4, 4, 64, torch.zeros(4, dtype=torch.int32)).c(0)  # on the host
    with pytest.raises(ValueError):
        B._loss_rows(cpu, 5, B.SoftmaxLoss(4, 4, 64, None), 0)
    with pytest.raises(TypeError):
        B._grads([cpu], None, 0)
    with pytest.raises(ValueError):
        B._grads([cpu], [], 0)
    for t, dense in ((cpu, True), (cpu.t(), True), (cpu[:, :3], False), (cpu[:2], True), (torch.zeros(3, 1, 5)[:, 0], True), (torch.zeros(()), True),
                     (torch.zeros(4).expand(3, 4), False), (torch.zeros(2, 3, 4).permute(2, 0, 1), True), (torch.zeros(8)[::2], False)):
        assert B._dense(t) == dense
