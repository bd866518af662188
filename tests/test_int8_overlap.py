"""8-bit layers, buffers that share memory: an output on an input, or on another output, is refused before any device work.
The addresses here are never dereferenced: every call is refused on the host.  Calls of buffers next to each other, which
are taken, run on the GPU's own tensors (the last tests)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import int8 as o8
from paper_2607_04461_amd import flashbon as fb

BF, F32 = fb.BF16, fb.FP32
M, N, K, D = 6, 20, 24, 40
STEP = 1 << 16           # between buffers that are not meant to touch


def _address(names):
    return {name: (i + 1) * STEP for i, name in enumerate(names)}


def _p(a):
    return None if a is None else ctypes.c_void_p(a)


def _refused(status):
    assert status == fb.EINVAL and "overlap" in fb.load().flashbon_last_error().decode()


# sizes in bytes, of what a call of the sizes above reads and writes
QUANT = dict(x=M * K * 2, q=M * K, scale=4 * M)
LINEAR = dict(A=M * K, sa=4 * M, W=N * K, sw=4 * N, bias=4 * N, out=4 * M * N, gate=4 * N, res=4 * M * N, cache=4 * M * N)
NORM = dict(x=4 * M * D, y=2 * M * D, gain=4 * D, gate=4 * D, x_out=4 * M * D, shift=4 * D, scale=4 * D, out=2 * M * D)
CODES = {**{k: v for k, v in NORM.items() if k != "out"}, "q": M * D, "qs": 4 * M}


def _quant(a, stride=K):
    return fb.load().flashbon_op_quant_rows(BF, M, K, _p(a["x"]), stride, _p(a["q"]), _p(a["scale"]), None)


def _linear(a, epi=fb.EPI_RESIDUAL):
    return fb.load().flashbon_op_linear_i8(BF, M, N, K, *(_p(a[k]) for k in ("A", "sa", "W", "sw", "bias")), epi,
                                           *(_p(a[k]) for k in ("out", "gate", "res", "cache")), None)


def _norm(a):
    return fb.load().flashbon_op_norm_residual(
        BF, M, D, 1e-6, _p(a["x"]), 1.0, _p(a.get("y")), 1, _p(a.get("gain")), _p(a.get("gate")), _p(a.get("x_out")), 1,
        _p(a.get("shift")), _p(a.get("scale")), _p(a.get("out")), _p(a.get("q")), _p(a.get("qs")), None)


def _pairs(sizes, outputs):
    return [(o, i) for o in outputs for i in sizes if i != o]


@pytest.mark.parametrize("call,sizes,out,other", [
    (c, s, o, i) for c, s, outs in ((_quant, QUANT, ("q", "scale")), (_linear, LINEAR, ("out", "cache")),
                                    (_norm, NORM, ("x_out", "out")), (_norm, CODES, ("x_out", "q", "qs")))
    for o, i in _pairs(s, outs)])
def test_an_output_on_another_buffer_is_refused(call, sizes, out, other):
    a = _address(sizes)
    for at in (a[other] + sizes[other] - 1, a[other] - sizes[out] + 1, a[other] + 1):     # last byte, first byte, inside
        _refused(call({**a, out: at}))


@pytest.mark.parametrize("epi,out,other", [(fb.EPI_STORE, "out", k) for k in ("A", "sa", "W", "sw", "bias")])
def test_activations_on_an_input_are_refused(epi, out, other):
    a = _address(LINEAR)
    for at in (a[other] + LINEAR[other] - 1, a[other] - 2 * M * N + 1):
        _refused(_linear({**a, out: at}, epi))


def test_codes_on_a_row_of_a_slice_are_refused():
    """Rows of 48 bytes, 4000 apart: scales of 24 bytes fit between two of them, codes of 144 as well; on a row they do not."""
    a, stride = _address(QUANT), 2000
    for m in range(M):
        row = a["x"] + 2 * m * stride
        for name, size in (("q", M * K), ("scale", 4 * M)):
            for at in (row - size + 1, row, row + 47):
                _refused(_quant({**a, name: at}, stride))


@pytest.mark.gpu
def test_buffers_next_to_each_other_are_taken():
    """Everything a call takes in one allocation, end to end: codes and scales in the gaps of a slice's rows, a residual
    layer and its cache, a seam in place."""
    stride = 512
    wide = torch.zeros(M * stride, dtype=torch.bfloat16, device="cuda")
    x = wide.view(M, stride)[:, 8:8 + K]
    x.copy_(torch.randn(M, K, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda"))
    ref, rs = o8.quant_rows(x.double().cpu().numpy())
    bytes_ = wide.view(torch.int8)
    for row in (0, 2):      # right behind a row's last element, and up to the next row's first
        lo, hi = 2 * (row * stride + 8 + K), 2 * ((row + 1) * stride + 8)
        q, s = bytes_[lo:lo + M * K], bytes_[hi - 4 * M:hi].view(torch.float32)
        fb.flashbon_op_quant_rows(BF, M, K, x, q, s)
        assert np.array_equal(q.view(M, K).cpu().numpy(), ref) and np.array_equal(s.cpu().numpy(), rs)
    g = torch.Generator(device="cuda").manual_seed(2)
    ones = torch.ones(64, device="cuda")
    a = torch.randint(-9, 9, (M, K), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-9, 9, (N, K), generator=g, device="cuda", dtype=torch.int8)
    acc = a.float() @ w.float().t()                                        # whole numbers below 2^11
    three = torch.zeros(3, M, N, device="cuda")
    three[2].normal_()
    fb.flashbon_op_linear_i8(BF, M, N, K, a, ones, w, ones, None, fb.EPI_RESIDUAL, three[1], residual_in=three[2], cache_out=three[0])
    assert torch.equal(three[1], acc + three[2]) and torch.equal(three[0], three[1])
    fb.flashbon_op_linear_i8(BF, M, N, K, a, ones, w, ones, None, fb.EPI_RESIDUAL, three[1], residual_in=three[1], cache_out=three[0])
    assert torch.equal(three[1], acc + (acc + three[2])) and torch.equal(three[0], three[1])
    h = torch.randn(2, M, D, generator=g, device="cuda")
    before = h.clone()
    fb.flashbon_op_norm_residual(F32, M, D, 1e-6, h[0], h[1], alpha=0.5, x_out=h[0], pre_norm=fb.NORM_NONE)
    assert torch.equal(h[0], (0.5 * before[0].double() + before[1].double()).float()) and torch.equal(h[1], before[1])
