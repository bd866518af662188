"""The seam between two blocks where its rounding decides: ties between two codes, rows that a norm leaves nothing of,
vectors whose product no fp32 holds, rows at the end of the range, and the same rows among many and among few."""
import numpy as np
import pytest
import torch

from oracle import int8 as o8
from paper_2607_04461_amd import flashbon as F

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                                     # half a step of fp32, relative
ACT = {F.BF16: torch.bfloat16, F.FP32: torch.float32}
EPS = 1e-6
# fewer rows than two a CU and more: widths of 513 to 2048 are laid out otherwise
FEW, MANY = 6, 530
WIDTHS = [(FEW, 40), (FEW, 41), (FEW, 500), (FEW, 1000), (MANY, 1000), (MANY, 1536), (MANY, 1601), (FEW, 2100), (FEW, 5003)]


def _dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(dtype)


def _f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _to_codes(x, y=None, dtype=F.FP32, **kw):
    M, D = x.shape
    q, s = torch.empty(M, D, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    h = torch.empty(M, D, device="cuda")
    F.flashbon_op_norm_residual(dtype, M, D, EPS, x, y, x_out=h, q=q, q_scale=s, **kw)
    return h, q.cpu().numpy(), s.cpu().numpy()


def _to_act(x, y=None, dtype=F.FP32, **kw):
    a, h = torch.empty_like(x, dtype=ACT[dtype]), torch.empty_like(x)
    F.flashbon_op_norm_residual(dtype, *x.shape, EPS, x, y, x_out=h, out=a, **kw)
    return h, a


# ------------------------------------------------------------------------------------------------- ties
def _ties(M, D):
    """Rows whose elements are (k + 1/2) s, s whole numbers and thirds of powers of two that fp32 holds; every third one
    step below, every third one above.  The largest is 127 s."""
    r = np.random.default_rng(3)
    scales = np.array([3, 5, 7, 11, 49, 99, 197, 3 * 2.0 ** -70, 5 * 2.0 ** 40])[np.arange(M) % 9]
    v = ((r.integers(-127, 127, (M, D)) + 0.5) * scales[:, None]).astype(np.float32)
    v[:, 1::3] = np.nextafter(v[:, 1::3], np.float32(0))
    v[:, 2::3] = np.nextafter(v[:, 2::3], np.float32(np.inf))
    v[:, D // 2] = 127 * scales
    return v


@pytest.mark.parametrize("M,D", WIDTHS)
def test_ties_go_to_the_even_code(M, D):
    v = _ties(M, D)
    rq, rs = o8.quant_rows(v)
    _, q, s = _to_codes(_dev(v), pre_norm=F.NORM_NONE)
    assert np.array_equal(s, rs) and np.array_equal(q, rq)


@pytest.mark.parametrize("M,D", WIDTHS)
def test_ties_made_of_a_branch_and_a_shift(M, D):
    """Whole halves: the stream, the branch, its gate and the shift add to (k + 1/2) s without a rounding."""
    r = np.random.default_rng(4)
    scales = np.array([3, 5, 7, 11, 49, 99])[np.arange(M) % 6]
    k = r.integers(-120, 120, (M, D))
    k[:, 0], half = 127, np.full((M, D), 0.5)
    half[:, 0] = 0.0
    a = (k + half) * scales[:, None]
    shift, gate = r.integers(-9, 10, D).astype(np.float64), r.choice([-2.0, 0.5, 1.0], D)
    y = r.integers(-50, 50, (M, D)).astype(np.float64)
    x = (a - shift - gate * y) * 2                                    # alpha 1/2
    h, q, s = _to_codes(_dev(x), _dev(y, torch.bfloat16), F.BF16, alpha=0.5, gate=_dev(gate), shift=_dev(shift),
                        pre_norm=F.NORM_NONE)
    rq, rs = o8.quant_rows(a)
    assert np.array_equal(_f64(h), a - shift)
    assert np.array_equal(s, rs) and np.array_equal(q, rq)


# ------------------------------------------------------------------------------------------ constant rows
CONSTANTS = [0.3, -7.7, 1e-3, 33333.3, 1e30, -1e-30]


@pytest.mark.parametrize("M,D", WIDTHS)
def test_layer_norm_leaves_nothing_of_a_constant_row(M, D):
    c = np.array(CONSTANTS, np.float32)[np.arange(M) % len(CONSTANTS)]
    x = _dev(np.repeat(c[:, None], D, 1))
    h, q, s = _to_codes(x, pre_norm=F.NORM_LAYER)
    assert torch.equal(h, x)
    assert (s == np.float32(2.0 ** -126)).all() and (q == 0).all()
    _, a = _to_act(x, pre_norm=F.NORM_LAYER)
    assert (a == 0).all()


@pytest.mark.parametrize("M,D", WIDTHS)
def test_a_constant_branch_adds_nothing(M, D):
    c = np.array(CONSTANTS, np.float32)[np.arange(M) % len(CONSTANTS)]
    x, y = torch.zeros(M, D, device="cuda"), _dev(np.repeat(c[:, None], D, 1))
    for run in (_to_codes, _to_act):
        assert (run(x, y, post_norm=F.NORM_LAYER, pre_norm=F.NORM_NONE)[0] == 0).all()


# ------------------------------------------------------------------------------------- the stream's rounding
@pytest.mark.parametrize("y,gain,gate", [(1e-30, 1e30, 1e30), (1e30, 1e-30, 1e-30), (1e30, 1e30, 1e-30), (1e-30, 1e-30, 1e30),
                                         (1e-20, 1e30, -1e20)])
def test_a_gate_and_a_gain_whose_product_no_fp32_holds(y, gain, gate):
    D = 77
    v = lambda c: _dev(np.full(D, c))  # noqa: E731
    x = _dev(np.full((3, D), 1e-31))
    rh, _ = o8.seam(_f64(x), np.full((3, D), np.float32(y)), 1.0, o8.NONE, _f64(v(gain)), _f64(v(gate)), o8.NONE, None, None, EPS)
    for run in (_to_codes, _to_act):
        h = run(x, _dev(np.full((3, D), y)), post_gain=v(gain), gate=v(gate), pre_norm=F.NORM_NONE)[0]
        np.testing.assert_allclose(_f64(h), rh, rtol=1.001 * U)      # rounded once


@pytest.mark.parametrize("post", [F.NORM_NONE, F.NORM_LAYER, F.NORM_RMS])
@pytest.mark.parametrize("M,D", WIDTHS)
@pytest.mark.parametrize("dtype", [F.BF16, F.FP32])
def test_the_stored_stream_does_not_depend_on_the_output(M, D, dtype, post):
    g = torch.Generator(device="cuda").manual_seed(5)
    x, y = torch.randn(M, D, generator=g, device="cuda"), torch.randn(M, D, generator=g, device="cuda").to(ACT[dtype])
    kw = dict(alpha=0.7, post_norm=post, post_gain=torch.randn(D, generator=g, device="cuda"),
              gate=torch.randn(D, generator=g, device="cuda"))
    alone = torch.empty_like(x)
    F.flashbon_op_norm_residual(dtype, M, D, EPS, x, y, x_out=alone, **kw)
    assert torch.equal(alone, _to_codes(x, y, dtype, **kw)[0])
    assert torch.equal(alone, _to_act(x, y, dtype, **kw)[0])
    kw = dict(alpha=0.7)
    F.flashbon_op_norm_residual(dtype, M, D, EPS, x, x_out=alone, **kw)
    assert torch.equal(alone, _to_codes(x, dtype=dtype, **kw)[0])
    assert torch.equal(alone, _to_act(x, dtype=dtype, **kw)[0])


# --------------------------------------------------------------------------------- rows at the end of the range
@pytest.mark.parametrize("D", [40, 1000, 2100])
@pytest.mark.parametrize("dtype", [F.BF16, F.FP32])
def test_norms_of_rows_at_the_end_of_the_range(D, dtype):
    """Rows whose differences from their mean, or whose reciprocal standard deviation, no fp32 holds."""
    r = np.random.default_rng(6)
    x = np.empty((4, D), np.float32)
    x[0] = np.where(np.arange(D) % 8 == 1, 3e38, -3e38)
    x[1] = np.where(np.arange(D) % 2, 3e38, -3e38)
    x[2] = 3e38 * r.uniform(0.5, 1, D)
    x[3] = 1e-38 * r.standard_normal(D)
    for pre, kind in ((F.NORM_LAYER, o8.LAYER), (F.NORM_RMS, o8.RMS)):
        h, a = _to_act(_dev(x), dtype=dtype, pre_norm=pre)
        assert torch.equal(h, _dev(x))
        ref = o8.norm(x, kind, EPS)
        # the output's rounding; of fp32 at most five more (the difference, the reciprocal, their product) and the mean's
        v = x.astype(np.float64)
        mean = v.mean(1, keepdims=True) if pre == F.NORM_LAYER else 0.0
        rstd = 1 / np.sqrt(((v - mean) ** 2).mean(1, keepdims=True) + EPS)
        # Below 2^-126 a type holds multiples of its smallest value alone, 2^-133 in bf16 and 2^-149 in fp32, and rounds by half
        # of that at most: the outputs next to zero in the last row, and that row's mean, whose rounding rstd multiplies.
        half, least = (2.0 ** -8, 2.0 ** -134) if dtype == F.BF16 else (U, 2.0 ** -150)
        off = U * np.abs(mean) + 2.0 ** -150
        assert (np.abs(_f64(a) - ref) <= (half + 5.1 * U) * 1.01 * np.abs(ref) + off * rstd + least).all()


# --------------------------------------------------------------------------------------- many rows and few
@pytest.mark.parametrize("D", [520, 1000, 1024, 1025, 1536, 1537, 1999, 2048])
@pytest.mark.parametrize("norm", [F.NORM_LAYER, F.NORM_RMS])
def test_a_rows_bits_are_the_same_among_many_rows_and_few(D, norm):
    """The stream is what a rounding to fp32 leaves of the branch's norm, so that it shows the last bits of the norm's 64."""
    r = np.random.default_rng(7)
    y = r.standard_normal((700, D)).astype(np.float32)
    x = o8.norm(y, {F.NORM_LAYER: o8.LAYER, F.NORM_RMS: o8.RMS}[norm], EPS)
    tx, ty = _dev(x), _dev(y)

    def run(m0, m1):
        return _to_codes(tx[m0:m1], ty[m0:m1], alpha=-1.0, post_norm=norm, pre_norm=F.NORM_LAYER)

    many = run(0, 700)
    for m0, m1 in ((0, 500), (500, 700), (333, 334)):
        for whole, part in zip(many, run(m0, m1)):
            assert torch.equal(whole[m0:m1], part) if torch.is_tensor(part) else np.array_equal(whole[m0:m1], part)
    a = _to_act(tx, ty, alpha=-1.0, post_norm=norm, pre_norm=F.NORM_LAYER)
    b = _to_act(tx[:500], ty[:500], alpha=-1.0, post_norm=norm, pre_norm=F.NORM_LAYER)
    assert all(torch.equal(p[:500], q) for p, q in zip(a, b))


# ------------------------------------------------------------------------------------ vectors of no branch
@pytest.mark.parametrize("M,D", [(FEW, 40), (FEW, 500), (FEW, 1536), (MANY, 1536), (FEW, 5003)])
def test_a_branchs_vectors_are_ignored_without_one(M, D):
    """The library's call with the addresses of one element each: nothing of them is to be read, where y is null."""
    import ctypes

    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    x, one = torch.randn(M, D, device="cuda"), torch.full((1,), float("nan"), device="cuda")
    h, a, ref = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    F.flashbon_op_norm_residual(F.FP32, M, D, EPS, x, alpha=0.5, out=ref)
    status = F.load().flashbon_op_norm_residual(F.FP32, M, D, EPS, p(x), 0.5, None, F.NORM_LAYER, p(one), p(one), p(h),
                                                F.NORM_LAYER, None, None, p(a), None, None,
                                                ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert status == F.OK and torch.equal(h, 0.5 * x) and torch.equal(a, ref)
