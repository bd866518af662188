"""8-bit layers, what the Python binding hands on (no GPU): calls that it has to refuse before the library sees them."""
import pytest
import torch

from paper_2607_04461_amd import flashbon as fb

BF, F32 = fb.BF16, fb.FP32
I8, F, B = torch.int8, torch.float32, torch.bfloat16


def _t(shape, dtype):
    return torch.zeros(shape, dtype=dtype)


# The ABI's integers have 32 bits, and ctypes keeps the low ones: 5 - 2^32 would arrive as five rows of tensors that hold none.
WRAPPED = [5 - (1 << 32), -(1 << 31) - 1, -(1 << 40) + 1]


@pytest.mark.parametrize("n", WRAPPED)
def test_sizes_below_32_bits_are_refused(n):
    empty = _t(0, I8), _t(0, F), _t(0, B)
    with pytest.raises(ValueError):
        fb.validate_quant_rows(BF, n, 1, empty[2], 1, empty[0], empty[1], require_device=False)
    for sizes in ((n, 4, 8), (3, n, 8), (3, 4, n)):
        with pytest.raises(ValueError, match="2\\^31"):
            fb.validate_linear_i8(BF, *sizes, _t((3, 8), I8), _t(3, F), _t((4, 8), I8), _t(4, F), None, fb.EPI_STORE,
                                  _t((3, 4), B), require_device=False)
    for sizes in ((n, 8), (3, n)):
        with pytest.raises(ValueError, match="2\\^31"):
            fb.validate_norm_residual(BF, *sizes, _t((3, 8), F), out=_t((3, 8), B), require_device=False)


@pytest.mark.parametrize("epilogue", [(1 << 32) + fb.EPI_GELU, fb.EPI_RESIDUAL - (1 << 32)])
def test_an_epilogue_that_would_wrap_is_refused(epilogue):
    with pytest.raises(ValueError, match="2\\^31"):
        fb.validate_linear_i8(BF, 3, 4, 8, _t((3, 8), I8), _t(3, F), _t((4, 8), I8), _t(4, F), None, epilogue, _t((3, 4), F),
                              require_device=False)


@pytest.mark.parametrize("missing", ["x", "q", "scale"])
def test_rows_need_their_tensors(missing):
    a = dict(x=_t((3, 8), B), q=_t((3, 8), I8), scale=_t(3, F))
    a[missing] = None
    with pytest.raises(ValueError, match=f"{missing} is required"):
        fb.validate_quant_rows(BF, 3, 8, a["x"], 8, a["q"], a["scale"], require_device=False)


@pytest.mark.parametrize("stride", [None, 8])
def test_a_call_without_rows_is_refused(stride, monkeypatch):
    monkeypatch.setattr(fb, "_current_device", lambda require_device: None)
    with pytest.raises(ValueError, match="x is required"):
        fb.flashbon_op_quant_rows(BF, 3, 8, None, _t((3, 8), I8), _t(3, F), x_row_stride=stride)


def test_the_stream_where_torch_lacks_the_short_way_to_it(monkeypatch):
    fb._with_torch()
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(fb, "_stream", lambda stream: 4321 if stream is None else int(stream))
    assert fb._raw_stream(None, 0) == 4321
    assert fb._raw_stream(77, 0) == 77
