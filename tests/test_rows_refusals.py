"""What layer norm and dropout refuse, before anything is launched.  The library's checks run on the host alone: a block of
zeros stands for the context (a refusal only writes its text there), and the buffers are addresses that nothing reads."""
import ctypes as C

import numpy as np
import pytest
import torch

import rows_ref as R
from paper_2103_00686_amd import binding as B

host = pytest.mark.skipif(torch.cuda.is_available(), reason="a call that is not refused would run")
X, Y, G, WS = 1 << 40, 2 << 40, 3 << 40, 4 << 40  # far apart


def _ctx():
    return C.create_string_buffer(1 << 16)


def _norm(**kw):
    n = B._Norm(10, 2, 64, B.FAE_F32, B.FAE_F32, 1e-5, None, None)
    for k, v in kw.items():
        setattr(n, k, v)
    return n


def _drop(**kw):
    d = B._Drop(0.1, 1, 2, None)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _fwd(norm, x=X, xs=128, y=Y, ys=128, drop=None, ctx=None):
    ctx = ctx or _ctx()
    rc = B.load().fae_layer_norm_fwd(ctx, C.byref(norm) if norm else None, C.c_void_p(x), C.c_int64(xs), C.c_void_p(y), C.c_int64(ys),
                                     C.byref(drop) if drop else None)
    return rc, B.load().fae_last_error(C.cast(ctx, C.c_void_p)).decode()


def _bwd(norm, x=X, xs=128, gy=G, gs=128, gx=Y, os=128, dg=None, db=None, drop=None, ws=WS, ws_bytes=1 << 30):
    ctx = _ctx()
    return B.load().fae_layer_norm_bwd(ctx, C.byref(norm) if norm else None, C.c_void_p(x), C.c_int64(xs), C.c_void_p(gy), C.c_int64(gs),
                                       C.c_void_p(gx), C.c_int64(os), C.c_void_p(dg), C.c_void_p(db), C.byref(drop) if drop else None,
                                       C.c_void_p(ws), C.c_size_t(ws_bytes))


def _dropout(fn, drop, n=10, parts=2, width=64, x=X, xt=0, xs=128, y=Y, yt=0, ys=128):
    return getattr(B.load(), fn)(_ctx(), C.byref(drop) if drop else None, C.c_int64(n), C.c_int32(parts), C.c_int32(width), C.c_void_p(x),
                                 C.c_int32(xt), C.c_int64(xs), C.c_void_p(y), C.c_int32(yt), C.c_int64(ys))


@host
@pytest.mark.parametrize("bad", [dict(n_rows=-1), dict(n_rows=1 << 30), dict(n_rows=1 << 40), dict(n_parts=0), dict(n_parts=65), dict(n_parts=-3), dict(width=0),
                                 dict(width=-5), dict(width=B.FAE_NORM_MAX_WIDTH + 1), dict(x_type=3), dict(y_type=-1), dict(x_type=B.FAE_BF16),
                                 dict(x_type=B.FAE_BF16, y_type=B.FAE_F16), dict(eps=0.0), dict(eps=-1e-5), dict(eps=float("nan")),
                                 dict(eps=float("inf")), dict(gamma=X + 2), dict(beta=X + 1)])
def test_norms(bad):
    assert _fwd(_norm(**bad))[0] == B.FAE_EINVAL
    assert _bwd(_norm(**bad)) == B.FAE_EINVAL


@host
@pytest.mark.parametrize("bad", [dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(p=1e-6), dict(p=1 - 1e-6), dict(d_offset=X + 4)])
def test_drops(bad):
    assert _fwd(_norm(), drop=_drop(**bad))[0] == B.FAE_EINVAL
    assert _bwd(_norm(), drop=_drop(**bad)) == B.FAE_EINVAL
    for fn in ("fae_dropout_fwd", "fae_dropout_bwd"):
        assert _dropout(fn, _drop(**bad)) == B.FAE_EINVAL


@host
@pytest.mark.parametrize("bad", [dict(x=0), dict(y=0), dict(x=X + 1), dict(y=Y + 2), dict(xs=127), dict(ys=0), dict(xs=-128), dict(xs=1 << 62),
                                 dict(y=X + 4), dict(y=X, ys=129), dict(y=X + 128 * 4), dict(y=X + 64 * 4, xs=160, ys=160)])
def test_buffers(bad):
    rc, text = _fwd(_norm(), **bad)
    assert rc == B.FAE_EINVAL and "fae_layer_norm_fwd" in text
    assert _dropout("fae_dropout_fwd", _drop(), **bad) == B.FAE_EINVAL
    assert _dropout("fae_dropout_bwd", _drop(), **bad) == B.FAE_EINVAL


@host
@pytest.mark.parametrize("bad", [dict(x=0), dict(gy=0), dict(gx=0), dict(gx=X + 4), dict(gx=G + 4), dict(gs=5), dict(os=5), dict(dg=X + 1), dict(db=X + 2)])
def test_backward_buffers(bad):
    assert _bwd(_norm(), **bad) == B.FAE_EINVAL


@host
def test_an_output_of_another_type_is_not_in_place():
    assert _fwd(_norm(y_type=B.FAE_BF16), y=X)[0] == B.FAE_EINVAL
    assert _bwd(_norm(y_type=B.FAE_BF16), gx=G) == B.FAE_EINVAL
    assert _dropout("fae_dropout_fwd", _drop(), y=X, yt=B.FAE_F16) == B.FAE_EINVAL


@host
def test_workspaces():
    need = B.fae_layer_norm_bwd_workspace_bytes(B.Norm(10, 2, 64))
    assert need > 0
    assert _bwd(_norm(), dg=1 << 20, db=2 << 20, ws_bytes=need - 1) == B.FAE_ENOSPC
    assert _bwd(_norm(), dg=1 << 20, db=2 << 20, ws=0) == B.FAE_ENOSPC
    assert B.load().fae_layer_norm_bwd_workspace_bytes(None) == 0


@host
@pytest.mark.parametrize("bad", [dict(n=-1), dict(n=1 << 32), dict(parts=0), dict(width=0), dict(width=-8), dict(parts=1 << 16, width=1 << 15), dict(n=1 << 31, parts=2),
                                 dict(xt=3), dict(yt=-1), dict(xt=B.FAE_BF16, yt=B.FAE_F16)])
def test_dropout_shapes(bad):
    assert _dropout("fae_dropout_fwd", _drop(), **bad) == B.FAE_EINVAL
    assert _dropout("fae_dropout_bwd", _drop(), **bad) == B.FAE_EINVAL


@host
def test_nulls():
    lib = B.load()
    assert _fwd(None)[0] == B.FAE_EINVAL and _bwd(None) == B.FAE_EINVAL and _dropout("fae_dropout_fwd", None) == B.FAE_EINVAL
    n, d = _norm(), _drop()
    assert lib.fae_layer_norm_fwd(None, C.byref(n), None, C.c_int64(0), None, C.c_int64(0), None) == B.FAE_EINVAL
    assert lib.fae_layer_norm_bwd(None, C.byref(n), None, C.c_int64(0), None, C.c_int64(0), None, C.c_int64(0), None, None, None, None,
                                  C.c_size_t(0)) == B.FAE_EINVAL
    assert lib.fae_dropout_fwd(None, C.byref(d), C.c_int64(1), C.c_int32(1), C.c_int32(1), None, 0, C.c_int64(1), None, 0, C.c_int64(1)) == B.FAE_EINVAL


@host
def test_no_rows_need_no_buffers():
    assert _fwd(_norm(n_rows=0), x=0, y=0)[0] == B.FAE_OK
    assert _dropout("fae_dropout_fwd", _drop(), n=0, x=0, y=0) == B.FAE_OK


def test_tensors_of_another_kind():
    """The binding's own checks: type, device, shape, values of a sample side by side."""
    cpu = torch.zeros((4, 64))
    with pytest.raises(TypeError):
        B._rows(cpu, 1, 64, torch.float32, 0)
    with pytest.raises(TypeError):
        B._type(torch.float64)
    with pytest.raises(ValueError):
        B.Norm(4, 2, 64, gamma=torch.zeros(64)).c(0)
    with pytest.raises(TypeError):
        B.Norm(4, 1, 64, gamma=torch.zeros(64)).c(0)
    with pytest.raises(TypeError):
        B.Drop(0.1, 1, 2, torch.zeros(2, dtype=torch.int64)).c(0)

    class Fake:  # what _rows looks at, as if on a device
        is_cuda, dtype = True, torch.float32

        def __init__(self, shape, stride, index=0):
            self.shape, self._s, self.device = torch.Size(shape), stride, torch.device("cuda", index)

        def stride(self, i=None):
            return self._s if i is None else self._s[i]

        def data_ptr(self):
            return 4096
    assert B._rows(Fake((4, 3, 8), (40, 8, 1)), 3, 8, torch.float32, 0)[1].value == 40
    assert B._rows(Fake((1, 3, 8), (7, 8, 1)), 3, 8, torch.float32, 0)[1].value == 24
    assert B._rows(Fake((4, 1, 8), (9, 999, 1)), 1, 8, torch.float32, 0)[1].value == 9
    for shape, stride, index in (((4, 3, 8), (40, 9, 1), 0), ((4, 3, 8), (40, 8, 2), 0), ((4, 24), (24, 1), 1), ((4, 25), (25, 1), 0), ((4,), (1,), 0)):
        with pytest.raises(ValueError):
            B._rows(Fake(shape, stride, index), 3, 8, torch.float32, 0)


def test_generator_against_published_outputs():
    """Philox4x32-10's known answers (Salmon et al., the authors' test vectors) for a counter and a key of zeros."""
    got = R.philox_numbers(1, 8, 0, 0).view(np.uint32)[0]
    assert [hex(v) for v in got] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]
