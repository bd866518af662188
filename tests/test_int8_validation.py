"""8-bit layers, refusals (no GPU): bad sizes, types and combinations come back as errors before any device work."""
import ctypes

import pytest
import torch

from paper_2607_04461_amd import flashbon as fb

P = ctypes.c_void_p(256)   # never dereferenced: every call here is refused on the host
BF, F32 = fb.BF16, fb.FP32


def _quant(dtype=BF, M=2, K=8, x=P, xs=8, q=P, scale=P):
    return fb.load().flashbon_op_quant_rows(dtype, M, K, x, xs, q, scale, None)


def _linear(dtype=BF, M=2, N=4, K=8, A=P, sa=P, W=P, sw=P, bias=None, epi=0, out=P, gate=None, res=None, cache=None):
    return fb.load().flashbon_op_linear_i8(dtype, M, N, K, A, sa, W, sw, bias, epi, out, gate, res, cache, None)


def _norm(dtype=BF, M=2, D=8, eps=1e-6, x=P, alpha=1.0, y=None, post=0, gain=None, gate=None, x_out=P, pre=1, shift=None,
          scale=None, out=P, q=None, qs=None):
    return fb.load().flashbon_op_norm_residual(dtype, M, D, eps, x, alpha, y, post, gain, gate, x_out, pre, shift, scale,
                                               out, q, qs, None)


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("call,kw,status", [
    (_quant, dict(dtype=2), fb.EINVAL), (_quant, dict(M=0), fb.ESHAPE), (_quant, dict(M=-1), fb.ESHAPE),
    (_quant, dict(K=0, xs=0), fb.ESHAPE), (_quant, dict(K=65537, xs=65537), fb.ESHAPE), (_quant, dict(xs=7), fb.ESHAPE),
    (_quant, dict(xs=-8), fb.ESHAPE), (_quant, dict(x=None), fb.EINVAL), (_quant, dict(q=None), fb.EINVAL),
    (_quant, dict(scale=None), fb.EINVAL),
    (_linear, dict(dtype=-1), fb.EINVAL), (_linear, dict(M=0), fb.ESHAPE), (_linear, dict(N=0), fb.ESHAPE),
    (_linear, dict(K=0), fb.ESHAPE), (_linear, dict(K=65537), fb.ESHAPE), (_linear, dict(N=(1 << 20) + 1), fb.ESHAPE),
    (_linear, dict(A=None), fb.EINVAL), (_linear, dict(sa=None), fb.EINVAL), (_linear, dict(W=None), fb.EINVAL),
    (_linear, dict(sw=None), fb.EINVAL), (_linear, dict(out=None), fb.EINVAL), (_linear, dict(epi=4), fb.EINVAL),
    (_linear, dict(epi=-1), fb.EINVAL),
    (_norm, dict(dtype=7), fb.EINVAL), (_norm, dict(M=0), fb.ESHAPE), (_norm, dict(D=0), fb.ESHAPE),
    (_norm, dict(D=6145), fb.ESHAPE), (_norm, dict(x=None), fb.EINVAL), (_norm, dict(x_out=None, out=None), fb.EINVAL),
    (_norm, dict(q=P, qs=P), fb.EINVAL), (_norm, dict(out=None, q=P), fb.EINVAL), (_norm, dict(out=None, qs=P), fb.EINVAL),
    (_norm, dict(post=3), fb.EINVAL), (_norm, dict(pre=-1), fb.EINVAL), (_norm, dict(eps=0.0), fb.EINVAL),
    (_norm, dict(eps=-1.0), fb.EINVAL), (_norm, dict(eps=INF), fb.EINVAL), (_norm, dict(eps=NAN), fb.EINVAL),
    (_norm, dict(alpha=INF), fb.EINVAL), (_norm, dict(alpha=NAN), fb.EINVAL),
])
def test_library_refuses(call, kw, status):
    assert call(**kw) == status
    assert fb.load().flashbon_last_error().decode() != ""


def _t(shape, dtype):
    return torch.zeros(shape, dtype=dtype)


I8, F, B = torch.int8, torch.float32, torch.bfloat16


def test_binding_takes_what_fits():
    fb.validate_quant_rows(BF, 3, 8, _t((3, 8), B), 8, _t((3, 8), I8), _t(3, F), require_device=False)
    fb.validate_quant_rows(F32, 3, 8, _t((3, 20), F)[:, 4:12], 20, _t((3, 8), I8), _t(3, F), require_device=False)
    fb.validate_linear_i8(BF, 3, 4, 8, _t((3, 8), I8), _t(3, F), _t((4, 8), I8), _t(4, F), None, fb.EPI_STORE,
                          _t((3, 4), B), require_device=False)
    fb.validate_linear_i8(BF, 3, 4, 8, _t((3, 8), I8), _t(3, F), _t((4, 8), I8), _t(4, F), _t(4, F), fb.EPI_RESIDUAL,
                          _t((3, 4), F), _t(4, F), _t((3, 4), F), _t((3, 4), F), require_device=False)
    fb.validate_norm_residual(F32, 3, 8, _t((3, 8), F), _t((3, 8), F), q=_t((3, 8), I8), q_scale=_t(3, F),
                              x_out=_t((3, 8), F), gate=_t(8, F), require_device=False)


@pytest.mark.parametrize("kw", [
    dict(x=_t((3, 8), F)), dict(x=_t((2, 8), B)), dict(x=_t((8, 3), B).t()), dict(q=_t((3, 8), torch.uint8)),
    dict(q=_t((3, 7), I8)), dict(q=_t((8, 3), I8).t()), dict(scale=_t(2, F)), dict(scale=_t(3, torch.float64)),
    dict(scale=None), dict(xs=4), dict(dtype=3), dict(M=0),
])
def test_binding_refuses_rows(kw):
    a = dict(dtype=BF, M=3, x=_t((3, 8), B), xs=8, q=_t((3, 8), I8), scale=_t(3, F))
    a.update(kw)
    with pytest.raises(ValueError):
        fb.validate_quant_rows(a["dtype"], a["M"], 8, a["x"], a["xs"], a["q"], a["scale"], require_device=False)


@pytest.mark.parametrize("kw", [
    dict(A=_t((3, 8), B)), dict(A=_t((2, 8), I8)), dict(A=None), dict(W=_t((8, 4), I8).t()), dict(W=_t((3, 8), I8)),
    dict(a_scale=_t(2, F)), dict(w_scale=_t(3, F)), dict(w_scale=_t(4, B)), dict(bias=_t(3, F)), dict(out=_t((3, 4), F)),
    dict(out=_t((2, 4), B)), dict(epilogue=fb.EPI_STORE_F32), dict(dtype=5),
    dict(epilogue=fb.EPI_RESIDUAL, out=_t((3, 4), F), gate=_t(3, F)),
    dict(epilogue=fb.EPI_RESIDUAL, out=_t((3, 4), F), residual_in=_t((3, 3), F)),
    dict(epilogue=fb.EPI_RESIDUAL, out=_t((3, 4), F), cache_out=_t((3, 4), B)),
])
def test_binding_refuses_linear(kw):
    a = dict(dtype=BF, M=3, N=4, K=8, A=_t((3, 8), I8), a_scale=_t(3, F), W=_t((4, 8), I8), w_scale=_t(4, F), bias=None,
             epilogue=fb.EPI_STORE, out=_t((3, 4), B))
    a.update(kw)
    with pytest.raises(ValueError):
        fb.validate_linear_i8(**a, require_device=False)


@pytest.mark.parametrize("kw", [
    dict(x=_t((3, 8), B)), dict(x=None), dict(y=_t((3, 8), F)), dict(y=_t((2, 8), B)), dict(out=_t((3, 8), F)),
    dict(q=_t((3, 8), torch.uint8)), dict(q_scale=_t(2, F)), dict(x_out=_t((3, 7), F)), dict(gate=_t(7, F)),
    dict(post_gain=_t(8, B)), dict(shift=_t((16,), F)[::2]), dict(scale=_t(4, F)),
])
def test_binding_refuses_norm(kw):
    a = dict(dtype=BF, M=3, D=8, x=_t((3, 8), F))
    a.update(kw)
    with pytest.raises(ValueError):
        fb.validate_norm_residual(**a, require_device=False)


@pytest.mark.parametrize("M", [1 << 31, (1 << 32) + 1])
def test_binding_refuses_sizes_that_would_wrap(M):
    def m(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="meta")
    with pytest.raises(ValueError, match="2\\^31"):
        fb.validate_quant_rows(BF, M, 1, m((M, 1), B), 1, m((M, 1), I8), m(M, F), require_device=False)
    with pytest.raises(ValueError, match="2\\^31"):
        fb.validate_linear_i8(BF, M, 1, 1, m((M, 1), I8), m(M, F), m((1, 1), I8), m(1, F), None, fb.EPI_STORE, m((M, 1), B),
                              require_device=False)
    with pytest.raises(ValueError, match="2\\^31"):
        fb.validate_norm_residual(BF, M, 1, m((M, 1), F), out=m((M, 1), B), require_device=False)


def test_binding_wants_the_current_device():
    with pytest.raises(ValueError):
        fb._pointers(0, ("x", _t(4, F), F, 4, True))
