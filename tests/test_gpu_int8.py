"""8-bit layers on the GPU against the 64-bit oracle: codes to the bit, products and seams within derived bounds."""
import numpy as np
import pytest
import torch

from oracle import dit as odit
from oracle import int8 as o8
from paper_2607_04461_amd import flashbon as F

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                                     # half a step of fp32, relative
HALF = {F.BF16: 2.0 ** -8, F.FP32: U}              # of the stored types
ACT = {F.BF16: torch.bfloat16, F.FP32: torch.float32}
CODE = {"bf16": F.BF16, "fp32": F.FP32}


def _rng(*seed):
    return np.random.default_rng([88, *seed])


def _f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(dtype)


GUARD = 96


class Out:
    """An output of `n` elements at `offset`, its surroundings filled, to be found as they were."""

    def __init__(self, n, dtype, offset=0):
        self.buf = torch.full((GUARD + offset + n + GUARD,), 77, dtype=dtype, device="cuda")
        self.lo, self.hi = GUARD + offset, GUARD + offset + n
        self.view = self.buf[self.lo:self.hi]

    def check(self):
        assert (self.buf[:self.lo] == 77).all() and (self.buf[self.hi:] == 77).all()


def _placed(a, dtype, offset):
    """The array on the device, `offset` elements past an allocation's start."""
    buf = torch.zeros(a.size + offset, dtype=dtype, device="cuda")
    buf[offset:].copy_(_dev(a.reshape(-1), dtype))
    return buf[offset:]


# --------------------------------------------------------------------------------------------- rows to codes
def _quant(x, dtype, M, K, stride=None, offset=0):
    q, s = Out(M * K, torch.int8, offset), Out(M, torch.float32)
    F.flashbon_op_quant_rows(dtype, M, K, x, q.view, s.view, x_row_stride=stride)
    torch.cuda.synchronize()
    q.check()
    s.check()
    return q.view.cpu().numpy().reshape(M, K), s.view.cpu().numpy()


# both sides of every change in threads and pieces per row, odd lengths, the longest
LENGTHS = [1, 2, 7, 8, 9, 64, 511, 512, 513, 1024, 1536, 2047, 2049, 4096, 4099, 8192, 8960, 13824, 16385, 32768, 32777, 65535,
           65536]


@pytest.mark.parametrize("K", LENGTHS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_codes_equal_the_oracles(K, dtype):
    d, M = CODE[dtype], 5
    x = _dev(_rng(1, K).standard_normal((M, K)) * np.array([1e-3, 1, 40, 1e20, 3e-30])[:, None], ACT[d])
    q, s = _quant(x, d, M, K)
    rq, rs = o8.quant_rows(_f64(x))
    assert np.array_equal(s, rs) and np.array_equal(q, rq)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("K", [40, 41, 3000])
def test_codes_at_the_borders(K, dtype):
    """Every quotient a tie or next to one: scales 1, 3, 2^-60 and the floor."""
    d = CODE[dtype]
    rows = []
    for s in (1.0, 3.0, 2.0 ** -60, 2.0 ** -126):
        k = _rng(2, K).integers(-127, 127, K) + 0.5
        v = k * s
        v[0] = 127 * s if s > 2.0 ** -126 else 100 * s
        if dtype == "fp32":   # one step beside a third of the ties each
            v = v.astype(np.float32)
            v[1::3] = np.nextafter(v[1::3], np.float32(0))
            v[2::3] = np.nextafter(v[2::3], np.float32(np.inf))
        rows.append(v)
    x = _dev(np.stack(rows).astype(np.float32), ACT[d])
    q, s = _quant(x, d, 4, K)
    rq, rs = o8.quant_rows(_f64(x))
    assert np.array_equal(s, rs) and np.array_equal(q, rq)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("K", [13, 520, 9000])
def test_rows_of_zeros_and_extremes(K, dtype):
    d = CODE[dtype]
    x = np.zeros((9, K), np.float32)
    x[1, K // 2] = 1e-45                      # below the smallest scale (bf16: zero)
    x[2, -1] = -1e-38
    x[3] = np.finfo(np.float32).max if dtype == "fp32" else 3.3e38
    x[4, 3], x[5, K - 1], x[6, 0] = np.inf, -np.inf, np.nan
    x[7, 5], x[7, 6] = np.nan, np.inf
    x[8] = -2.0
    t = _dev(x, ACT[d])
    q, s = _quant(t, d, 9, K)
    rq, rs = o8.quant_rows(_f64(t))
    assert np.array_equal(s, rs, equal_nan=True) and np.array_equal(q, rq)
    assert np.isnan(s[4:8]).all() and np.isfinite(np.delete(s, range(4, 8))).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("K,ld,col,offset", [(64, 200, 16, 0), (65, 201, 3, 1), (1536, 4608, 1536, 3), (8957, 9001, 7, 5)])
def test_rows_within_wider_rows(K, ld, col, offset, dtype):
    d, M = CODE[dtype], 6
    wide = _dev(_rng(3, K).standard_normal((M, ld)), ACT[d])
    q, s = _quant(wide[:, col:col + K], d, M, K, offset=offset)
    rq, rs = o8.quant_rows(_f64(wide)[:, col:col + K])
    assert np.array_equal(s, rs) and np.array_equal(q, rq)


def test_a_rows_codes_do_not_depend_on_the_other_rows():
    x = torch.randn(301, 2050, device="cuda")
    q, s = _quant(x, F.FP32, 301, 2050)
    for m in (0, 150, 300):
        q1, s1 = _quant(x[m:m + 1].contiguous(), F.FP32, 1, 2050)
        assert np.array_equal(q1[0], q[m]) and s1[0] == s[m]


# --------------------------------------------------------------------------------------------- linear layers
def _codes(rng, rows, k, wide):
    if wide:   # all of -128 .. 127
        return rng.integers(-128, 128, (rows, k)).astype(np.int8)
    return np.clip(np.rint(rng.standard_normal((rows, k)) * 30), -127, 127).astype(np.int8)


def _linear(M, N, K, dtype, epi, offset=0, bias=True, gate=True, cache=True, in_place=False, wide=True):
    """One layer compared with the oracle, every element within the bound of its own roundings; returns the output."""
    d, r = CODE[dtype], _rng(4, M, N, K)
    a, w = _codes(r, M, K, wide), _codes(r, N, K, wide)
    sa, sw = np.exp(r.standard_normal(M) - 4).astype(np.float32), np.exp(r.standard_normal(N) - 5).astype(np.float32)
    b, g = r.standard_normal(N).astype(np.float32), r.standard_normal(N).astype(np.float32)
    h0 = r.standard_normal((M, N)).astype(np.float32)
    A, W = _placed(a, torch.int8, offset), _placed(w, torch.int8, offset)
    db, dg = (_dev(b) if bias else None), (_dev(g) if gate else None)
    stores_act = epi in ("store", "gelu")
    out = Out(M * N, ACT[d] if stores_act else torch.float32, offset)
    code = {"store": F.EPI_STORE, "gelu": F.EPI_GELU, "store_f32": F.EPI_STORE_F32, "residual": F.EPI_RESIDUAL}[epi]
    copy = Out(M * N, torch.float32, offset) if cache else None
    if in_place:
        out.view.copy_(_dev(h0.reshape(-1)))
    F.flashbon_op_linear_i8(d, M, N, K, A, _dev(sa), W, _dev(sw), db, code, out.view, gate=dg,
                            residual_in=None if in_place else _placed(h0, torch.float32, offset),
                            cache_out=copy.view if cache else None)
    torch.cuda.synchronize()
    out.check()
    got = _f64(out.view).reshape(M, N)
    t = o8.linear(a, sa, w, sw)                       # the scaled sum; the bias comes in the last rounding
    v = t + (b if bias else 0.0)
    # conversion, product with w_scale, and the last product with the bias added: half a step each
    err = 2.01 * U * np.abs(t) + 1.01 * U * np.abs(v)
    if epi == "gelu":
        # GELU is 1.13-Lipschitz; x / (1 + 2^-z), z off by 5 half steps, moves by at most 0.25 of them; the two hardware
        # functions (a step each), the sum and the product round
        v, err = odit.gelu_tanh(v), 1.13 * err + 0.25 * 5 * U + 6 * U * np.abs(odit.gelu_tanh(v))
    elif epi == "residual":
        ref = h0 + (g if gate else 1.0) * v
        err = np.abs(g if gate else 1.0) * err + 1.01 * U * np.abs(ref)
        v = ref
    if stores_act:
        err = err + HALF[d] * np.abs(v) * 1.01
    assert (np.abs(got - v) <= err + 1e-37).all(), np.abs(got - v).max()
    if cache and epi == "residual":
        assert torch.equal(copy.view, out.view)
    if copy is not None:
        copy.check()
    return out.view.clone()


# single rows and columns, sums of one product, edges of the tiles, sizes off every multiple
SHAPES = [(1, 1, 1), (1, 5, 16), (2, 3, 15), (3, 16, 17), (16, 16, 64), (17, 33, 130), (33, 40, 127), (64, 64, 128), (65, 66, 129),
          (1, 300, 1536), (5, 1000, 512), (16, 256, 2048), (31, 96, 4096), (100, 264, 272), (130, 136, 96), (257, 129, 255),
          (260, 520, 384)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("epi", ["store", "gelu", "store_f32", "residual"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_linear_against_the_oracle(M, N, K, epi, dtype):
    _linear(M, N, K, dtype, epi)


@pytest.mark.parametrize("M,N,K", [(70, 72, 80), (300, 520, 192), (9, 48, 512)])
@pytest.mark.parametrize("kw", [dict(bias=False), dict(gate=False), dict(cache=False), dict(in_place=True),
                                dict(in_place=True, bias=False, gate=False, cache=False)])
def test_linear_options(M, N, K, kw):
    _linear(M, N, K, "bf16", "residual", **kw)


FEW = ["few:16x16", "few:32x16", "few:32x32", "few:64x32"]
TILES = ["split:16x16", "split:32x16", "split:32x32", "split:64x32", "any", "256x256", "128x256", "128x128:two", "128x128",
         "96x128", "64x128", *FEW]


# a K of one, two, three and more of the ring's K tiles, K tails of 16 to 112, rows and columns on and beside the tiles' edges
@pytest.mark.parametrize("M,N,K", [(1, 8, 16), (129, 136, 112), (260, 264, 128), (255, 256, 240), (257, 512, 256), (300, 520, 400),
                                   (128, 248, 528), (513, 264, 1040)])
@pytest.mark.parametrize("epi", ["store", "gelu", "residual"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_every_kernel_gives_the_same_bits(M, N, K, epi, dtype, monkeypatch):
    first = None
    for tile in TILES:
        monkeypatch.setenv("FLASHBON_I8_TILE", tile)
        got = _linear(M, N, K, dtype, epi)
        first = got if first is None else first
        assert torch.equal(got, first), tile
    for w in (8, 7, 6):   # row blocks of two heights: all of the one or the other, mixed, and more than the rows need
        lo = 32 * (w - 1)
        for blocks in {-(-M // (lo + 32)), -(-M // lo), min(M, -(-M // lo) + 2)}:
            for tall in {max(0, -(-(M - lo * blocks) // 32)), blocks // 2, blocks}:
                if 0 <= tall <= blocks and lo * blocks + 32 * tall >= M:
                    monkeypatch.setenv("FLASHBON_I8_TILE", f"mix:{w}:{blocks}:{tall}")
                    assert torch.equal(_linear(M, N, K, dtype, epi), first), (w, blocks, tall)


# waves with none, one, two, three and more of the pieces of K, a last piece of 16 to 128 bytes; columns that the tiles take
# and no ring tile does
@pytest.mark.parametrize("M,N,K", [(1, 1, 16), (65, 33, 1008), (31, 15, 1040), (17, 47, 2064), (130, 129, 2688), (3, 70, 8976)])
@pytest.mark.parametrize("epi", ["store", "gelu", "residual"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_few_rows_any_columns(M, N, K, epi, dtype, monkeypatch):
    monkeypatch.setenv("FLASHBON_I8_TILE", "split:16x16")
    first = _linear(M, N, K, dtype, epi)
    for tile in FEW:
        monkeypatch.setenv("FLASHBON_I8_TILE", tile)
        assert torch.equal(_linear(M, N, K, dtype, epi), first), tile


@pytest.mark.parametrize("M,N", [(2, 40), (40000, 16)])
def test_more_rows_than_a_launch_takes(M, N):
    _linear(M, N, 48, "bf16", "residual")


def test_more_outputs_than_a_launch_takes():
    """1030 x 2^20: the widest layer, its rows in two launches."""
    M, N, K = 1030, 1 << 20, 5
    g = torch.Generator(device="cuda").manual_seed(21)
    a = torch.randint(-128, 128, (M, K), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    sa, sw = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    F.flashbon_op_linear_i8(F.BF16, M, N, K, a, sa, w, sw, None, F.EPI_STORE, out)
    for m in (0, 1023, 1024, 1029):
        acc = (a[m].float() * w.float()).sum(1)            # whole numbers below 2^17
        assert torch.equal(out[m], ((acc * sw) * sa[m]).bfloat16())


@pytest.mark.parametrize("offset", [1, 4, 8])
@pytest.mark.parametrize("M,N,K", [(70, 72, 80), (5, 48, 512), (300, 264, 256)])
@pytest.mark.parametrize("epi", ["store", "residual"])
def test_linear_on_any_address(M, N, K, offset, epi):
    assert torch.equal(_linear(M, N, K, "bf16", epi, offset=offset), _linear(M, N, K, "bf16", epi))


@pytest.mark.parametrize("M,N,K", [(40, 48, 65536), (3, 20, 65536), (3, 20, 65533)])
def test_longest_sums_of_the_largest_codes(M, N, K):
    a = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    w[1::2] = 127
    out = torch.empty(M, N, device="cuda")
    one = torch.ones(max(M, N), device="cuda")
    F.flashbon_op_linear_i8(F.FP32, M, N, K, a, one, w, one, None, F.EPI_STORE, out)
    torch.cuda.synchronize()
    exact = np.array([16384.0 * K, -16256.0 * K]).astype(np.float32)
    assert (out[:, 0::2].cpu().numpy() == exact[0]).all() and (out[:, 1::2].cpu().numpy() == exact[1]).all()


def test_a_row_without_a_scale_is_nan_and_no_other():
    x = torch.randn(40, 200, device="cuda")
    x[7, 3], x[21, 9] = float("inf"), float("nan")
    q, s = torch.empty(40, 200, dtype=torch.int8, device="cuda"), torch.empty(40, device="cuda")
    F.flashbon_op_quant_rows(F.FP32, 40, 200, x, q, s)
    w, sw = torch.ones(24, 200, dtype=torch.int8, device="cuda"), torch.ones(24, device="cuda")
    out = torch.empty(40, 24, device="cuda")
    F.flashbon_op_linear_i8(F.FP32, 40, 24, 200, q, s, w, sw, None, F.EPI_STORE, out)
    nan = torch.isnan(out).all(1).cpu().tolist()
    assert nan == [m in (7, 21) for m in range(40)]
    assert int(torch.isnan(out).sum()) == 48


def test_a_rows_bits_do_not_depend_on_the_other_rows():
    g = torch.Generator(device="cuda").manual_seed(5)
    a = torch.randint(-127, 128, (700, 640), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-127, 128, (520, 640), generator=g, device="cuda", dtype=torch.int8)
    sa, sw = torch.rand(700, generator=g, device="cuda") * 0.01, torch.rand(520, generator=g, device="cuda") * 0.01
    bias = torch.randn(520, generator=g, device="cuda")

    def run(m0, m1):
        out = torch.empty(m1 - m0, 520, dtype=torch.bfloat16, device="cuda")
        F.flashbon_op_linear_i8(F.BF16, m1 - m0, 520, 640, a[m0:m1], sa[m0:m1].contiguous(), w, sw, bias, F.EPI_GELU, out)
        return out

    whole = run(0, 700)
    for m0, m1 in ((0, 1), (3, 12), (100, 133), (650, 700), (0, 400)):
        assert torch.equal(run(m0, m1), whole[m0:m1])


# --------------------------------------------------------------------------------------------- the seam
KIND = {"none": F.NORM_NONE, "layer": F.NORM_LAYER, "rms": F.NORM_RMS}
EPS = 1e-6


def _seam(M, D, dtype, post="rms", pre="layer", out="i8", alpha=0.75, vectors=True, branch=True, x_out="new", x=None, y=None,
          offset=0):
    """One seam compared with the oracle; returns what it wrote."""
    d, r = CODE[dtype], _rng(6, M, D)
    x = (r.standard_normal((M, D)) + 0.5 * r.standard_normal(D)).astype(np.float32) if x is None else x
    y = r.standard_normal((M, D)) * 0.7 if y is None else y
    vec = [r.standard_normal(D).astype(np.float32) * k + c for k, c in ((0.1, 1.0), (0.5, 0.0), (0.3, 0.0), (0.3, 0.0))]
    gain, gate, shift, scale = [v.astype(np.float32) for v in vec] if vectors else [None] * 4
    dx = _placed(x, torch.float32, offset)
    dy = _placed(y, ACT[d], offset) if branch else None
    dv = [None if v is None else _placed(v, torch.float32, offset) for v in (gain, gate, shift, scale)]
    h = Out(M * D, torch.float32, offset) if x_out == "new" else None
    act = Out(M * D, ACT[d], offset) if out == "act" else None
    q = Out(M * D, torch.int8, offset) if out == "i8" else None
    qs = Out(M, torch.float32) if out == "i8" else None
    target = h.view if h else (dx if x_out == "x" else None)
    F.flashbon_op_norm_residual(d, M, D, EPS, dx, dy, alpha=alpha, post_norm=KIND[post], post_gain=dv[0], gate=dv[1],
                                x_out=target, pre_norm=KIND[pre], shift=dv[2], scale=dv[3],
                                out=act.view if act else None, q=q.view if q else None, q_scale=qs.view if qs else None)
    torch.cuda.synchronize()
    for o in (h, act, q, qs):
        if o is not None:
            o.check()
    ry = _f64(dy).reshape(M, D) if branch else None
    rh, ra = o8.seam(x, ry, alpha, KIND[post], gain, gate, KIND[pre], shift, scale, EPS)
    got = {}
    if target is not None:
        got["h"] = target.clone()
        gh = _f64(target).reshape(M, D)
        if out == "i8":
            np.testing.assert_allclose(gh, rh, rtol=U * 1.001, atol=1e-37)      # rounded once
        else:
            assert (np.abs(gh - rh) <= _h_bound(x, ry, alpha, KIND[post], gain, gate, rh)).all()
    if out == "i8":
        rq, rs = o8.quant_rows(ra)
        assert np.array_equal(qs.view.cpu().numpy(), rs, equal_nan=True)
        assert np.array_equal(q.view.cpu().numpy().reshape(M, D), rq)
        got["q"], got["s"] = q.view.clone(), qs.view.clone()
    if act is not None:
        ga = _f64(act.view).reshape(M, D)
        # from the stream as the kernel stored it, where it did: what is left is the second norm's own rounding
        hs = _f64(target).reshape(M, D) if target is not None else rh
        _, ra = o8.seam(hs, None, 1.0, 0, None, None, KIND[pre], shift, scale, EPS)
        bound = _a_bound(hs, KIND[pre], scale, shift, ra)
        if target is None:   # the stream's own error, through the norm
            s1 = np.abs(1.0 + (scale if scale is not None else 0.0))
            e = _h_bound(x, ry, alpha, KIND[post], gain, gate, rh)
            rstd = 1.0 if pre == "none" else 1 / np.sqrt(((hs - (hs.mean(1, keepdims=True) if pre == "layer" else 0)) ** 2).mean(1, keepdims=True) + EPS)
            bound = bound + 3 * s1 * rstd * e.max(1, keepdims=True)
        assert (np.abs(ga - ra) <= bound + HALF[d] * 1.01 * np.abs(ra)).all()
        got["a"] = act.view.clone()
    return got


def _h_bound(x, y, alpha, post, gain, gate, ref):
    """Roundings of h = alpha x + gate (y - mean) rstd gain in fp32: mean and rstd rounded from 64 bits, then one rounding
    an operation."""
    if y is None:
        return 1.01 * U * np.abs(ref) + 1e-37
    mean = y.mean(1, keepdims=True) if post == o8.LAYER else np.zeros((len(y), 1))
    rstd = 1.0 if post == o8.NONE else 1 / np.sqrt(((y - mean) ** 2).mean(1, keepdims=True) + EPS)
    k = np.abs((gate if gate is not None else 1.0) * (np.asarray(gain, np.float64) if gain is not None else 1.0)) * rstd
    # y - mean: the mean's rounding and the difference's; the product with rstd (itself rounded), with the gain, with the gate
    return k * (U * np.abs(mean) + 5.1 * U * np.abs(y - mean)) + U * (1.01 * np.abs(alpha * x) + 1.01 * np.abs(ref)) + 1e-37


def _a_bound(h, pre, scale, shift, ref):
    mean = h.mean(1, keepdims=True) if pre == o8.LAYER else np.zeros((len(h), 1))
    rstd = 1.0 if pre == o8.NONE else 1 / np.sqrt(((h - mean) ** 2).mean(1, keepdims=True) + EPS)
    s1 = np.abs(1.0 + (np.asarray(scale, np.float64) if scale is not None else 0.0))
    one = U * 1.01 * (1.0 + (np.abs(scale) if scale is not None else 0.0))    # 1 + scale rounds by half a step of itself
    # h as stored, rounded once more where only the kernel holds it
    return rstd * ((s1 + one) * (U * np.abs(mean) + 5.1 * U * np.abs(h - mean)) + s1 * U * np.abs(h)) + 2.02 * U * np.abs(ref) + 1e-37


DIMS = [1, 2, 7, 8, 63, 64, 257, 512, 513, 1024, 1031, 1536, 1537, 2048, 4096, 4104, 5120, 6143, 6144]


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("out", ["i8", "act"])
def test_seam_against_the_oracle(D, dtype, out):
    _seam(5, D, dtype, out=out)


@pytest.mark.parametrize("post", ["none", "layer", "rms"])
@pytest.mark.parametrize("pre", ["none", "layer", "rms"])
@pytest.mark.parametrize("out", ["i8", "act", "none"])
@pytest.mark.parametrize("D", [72, 2100])
def test_seam_norms(post, pre, out, D):
    _seam(9, D, "bf16", post, pre, out)


@pytest.mark.parametrize("kw", [dict(vectors=False), dict(branch=False), dict(x_out="x"), dict(x_out=None), dict(alpha=0.0),
                                dict(branch=False, vectors=False, alpha=1.0), dict(offset=1), dict(offset=3, x_out="x")])
@pytest.mark.parametrize("out", ["i8", "act"])
@pytest.mark.parametrize("D", [96, 1000, 3001])
def test_seam_options(kw, out, D):
    _seam(6, D, "bf16", out=out, **kw)


def test_seam_of_constant_wide_and_offset_rows():
    """Rows of one value (a variance of zero), of a large common offset, of huge and of tiny values."""
    r = _rng(7)
    for D in (48, 1536, 2056):
        x = r.standard_normal((6, D)).astype(np.float32)
        y = r.standard_normal((6, D))
        x[0], y[0] = 3.25, 0.0
        x[1], y[1] = 0.0, 0.0
        x[2] += 1e4
        y[3] += 300.0
        x[4] *= 1e15
        x[5] *= 1e-20
        y[5] *= 1e-20
        _seam(6, D, "fp32", "layer", "layer", "i8", x=x, y=y)
        _seam(6, D, "fp32", "rms", "rms", "i8", x=x, y=y)


@pytest.mark.parametrize("D", [40, 1500, 2501])
def test_seam_of_rows_that_are_not_finite(D):
    x, y = torch.randn(6, D, device="cuda"), torch.randn(6, D, device="cuda")
    x[1, 3], x[2, D - 1], y[4, 0] = float("nan"), float("inf"), float("-inf")
    h, q, s = torch.empty_like(x), torch.empty(6, D, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    F.flashbon_op_norm_residual(F.FP32, 6, D, EPS, x, y, post_norm=F.NORM_RMS, x_out=h, q=q, q_scale=s)
    assert torch.isnan(s).cpu().tolist() == [False, True, True, False, True, False]
    assert (q[[1, 2, 4]] == 0).all() and (q[[0, 3, 5]].abs().amax(1) == 127).all()
    a = torch.empty_like(x)
    F.flashbon_op_norm_residual(F.FP32, 6, D, EPS, x, y, post_norm=F.NORM_RMS, out=a)
    assert torch.isnan(a).any(1).cpu().tolist() == [False, True, True, False, True, False]


def test_a_rows_seam_does_not_depend_on_the_other_rows():
    x, y = torch.randn(203, 1536, device="cuda"), torch.randn(203, 1536, device="cuda").bfloat16()

    def run(m0, m1):
        n = m1 - m0
        h, q, s = torch.empty(n, 1536, device="cuda"), torch.empty(n, 1536, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        F.flashbon_op_norm_residual(F.BF16, n, 1536, EPS, x[m0:m1], y[m0:m1], post_norm=F.NORM_LAYER, x_out=h, q=q, q_scale=s)
        return h, q, s

    whole = run(0, 203)
    for m0, m1 in ((0, 1), (7, 9), (100, 203)):
        assert all(torch.equal(a, b[m0:m1]) for a, b in zip(run(m0, m1), whole))


# --------------------------------------------------------------------------------------------- together
class Branch:
    """The MLP branch of a block with 8-bit layers, between the seams on its two sides."""

    def __init__(self, M, D, H, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        n = lambda *s, std=1.0: torch.randn(*s, generator=g, device="cuda") * std  # noqa: E731
        self.M, self.D, self.H = M, D, H
        self.w1, self.b1, self.w2, self.b2 = n(H, D, std=D ** -0.5), n(H, std=0.1), n(D, H, std=H ** -0.5), n(D, std=0.1)
        self.gate, self.scale, self.shift, self.gain = n(D, std=0.5), n(D, std=0.2), n(D, std=0.2), 1 + n(D, std=0.1)
        i8 = lambda *s: torch.empty(*s, dtype=torch.int8, device="cuda")  # noqa: E731
        f = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
        bf = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.q1, self.s1, self.q2, self.s2 = i8(H, D), f(H), i8(D, H), f(D)
        F.flashbon_op_quant_rows(F.FP32, H, D, self.w1, self.q1, self.s1)
        F.flashbon_op_quant_rows(F.FP32, D, H, self.w2, self.q2, self.s2)
        self.x, self.a, self.sa, self.u, self.qu, self.su, self.y = f(M, D), i8(M, D), f(M), bf(M, H), i8(M, H), f(M), bf(M, D)
        self.out, self.next, self.sn = f(M, D), i8(M, D), f(M)

    def run(self, stream=None):
        M, D, H = self.M, self.D, self.H
        F.flashbon_op_norm_residual(F.BF16, M, D, EPS, self.x, pre_norm=F.NORM_LAYER, shift=self.shift, scale=self.scale,
                                    q=self.a, q_scale=self.sa, stream=stream)
        F.flashbon_op_linear_i8(F.BF16, M, H, D, self.a, self.sa, self.q1, self.s1, self.b1, F.EPI_GELU, self.u, stream=stream)
        F.flashbon_op_quant_rows(F.BF16, M, H, self.u, self.qu, self.su, stream=stream)
        F.flashbon_op_linear_i8(F.BF16, M, D, H, self.qu, self.su, self.q2, self.s2, self.b2, F.EPI_STORE, self.y, stream=stream)
        F.flashbon_op_norm_residual(F.BF16, M, D, EPS, self.x, self.y, alpha=1.0, post_norm=F.NORM_RMS, post_gain=self.gain,
                                    gate=self.gate, x_out=self.out, pre_norm=F.NORM_LAYER, q=self.next, q_scale=self.sn,
                                    stream=stream)

    def results(self):
        return [t.clone() for t in (self.a, self.sa, self.u, self.qu, self.su, self.y, self.out, self.next, self.sn)]

    def float_branch(self):
        """The same branch in 64 bits without 8-bit operands."""
        d = lambda t: _f64(t)  # noqa: E731
        _, a = o8.seam(d(self.x), None, 1.0, 0, None, None, o8.LAYER, d(self.shift), d(self.scale), EPS)
        u = odit.gelu_tanh(a @ d(self.w1).T + d(self.b1))
        y = u @ d(self.w2).T + d(self.b2)
        return d(self.x) + d(self.gate) * (o8.norm(y, o8.RMS, EPS) * d(self.gain))


@pytest.mark.parametrize("M,D,H", [(1, 64, 256), (37, 136, 520), (390, 256, 704), (65, 101, 203)])
def test_the_branch_as_a_whole(M, D, H):
    b = Branch(M, D, H, 11)
    b.x.copy_(torch.randn(M, D, generator=torch.Generator(device="cuda").manual_seed(12), device="cuda"))
    b.run()
    torch.cuda.synchronize()
    # every stage from the operands the stage before left
    _, a = o8.seam(_f64(b.x), None, 1.0, 0, None, None, o8.LAYER, _f64(b.shift), _f64(b.scale), EPS)
    rq, rs = o8.quant_rows(a)
    assert np.array_equal(_f64(b.a), rq) and np.array_equal(b.sa.cpu().numpy(), rs)
    t = o8.linear(_f64(b.a), _f64(b.sa), _f64(b.q1), _f64(b.s1), _f64(b.b1))
    assert np.abs(_f64(b.u) - odit.gelu_tanh(t)).max() <= 1.02 * 2.0 ** -8 * np.abs(t).max()
    rq, rs = o8.quant_rows(_f64(b.u))
    assert np.array_equal(_f64(b.qu), rq) and np.array_equal(b.su.cpu().numpy(), rs)
    rh, ra = o8.seam(_f64(b.x), _f64(b.y), 1.0, o8.RMS, _f64(b.gain), _f64(b.gate), o8.LAYER, None, None, EPS)
    np.testing.assert_allclose(_f64(b.out), rh, rtol=1.001 * U, atol=1e-37)
    rq, rs = o8.quant_rows(ra)
    assert np.array_equal(_f64(b.next), rq) and np.array_equal(b.sn.cpu().numpy(), rs)
    # Against the branch without 8-bit operands.  An operand's step is max / 127 and its error at most half of that,
    # uniform: max / (127 sqrt 12) in the root mean square.  Rows of these lengths have max <= 4.5 rms (GELU outputs and
    # short rows less than 6), so each of the four quantised operands is off by at most 6 / 440 = 1.4 %, and the two
    # products of two such operands by at most sqrt(4) 1.4 % = 2.8 % of the branch; bf16 adds 0.3 %.
    ref, got, x = b.float_branch(), _f64(b.out), _f64(b.x)
    assert np.linalg.norm(got - ref) <= 0.031 * np.linalg.norm(ref - x)


def test_the_branch_on_another_stream():
    b = Branch(130, 256, 704, 13)
    b.x.normal_()
    b.run()
    torch.cuda.synchronize()
    ref = b.results()
    side = torch.cuda.Stream()
    for t in (b.u, b.y, b.out):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    b.run(stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ref, b.results()))


def test_the_branch_captured_and_replayed():
    """Two graphs of two branches, replayed in turn with new inputs between the replays, against eager runs."""
    branches = [Branch(130, 256, 704, 14), Branch(5, 96, 200, 15)]
    side = torch.cuda.Stream()
    graphs = []
    for b in branches:
        b.x.normal_()
        b.run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            b.run()
        graphs.append(graph)
    for _ in range(3):
        for b, graph in zip(branches, graphs):
            b.x.normal_()
            b.run()
            torch.cuda.synchronize()
            ref = b.results()
            for t in (b.a, b.u, b.qu, b.y, b.out, b.next):
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(ref, b.results()))


# ------------------------------------------------------------------------- tensors past 2^31 elements and 2^32 bytes
def _spread(M):
    """Rows on both sides of a launch's part of the rows, and the last."""
    return [0, (1 << 20) - 1, 1 << 20, M - 1]


def test_rows_past_32_bits():
    M, K = (1 << 20) + 77, 2100
    g = torch.Generator(device="cuda").manual_seed(31)
    x = torch.empty(M, K, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    q, s = torch.empty(M, K, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    F.flashbon_op_quant_rows(F.BF16, M, K, x, q, s)
    for m in _spread(M):
        rq, rs = o8.quant_rows(_f64(x[m:m + 1]))
        assert np.array_equal(_f64(q[m:m + 1]), rq) and s[m].item() == rs[0]


def test_a_row_stride_past_32_bits():
    stride, K = (1 << 31) + 24, 1000
    x = torch.zeros(2 * stride, dtype=torch.bfloat16, device="cuda").view(2, stride)[:, :K]
    x.copy_(torch.randn(2, K, generator=torch.Generator(device="cuda").manual_seed(32), device="cuda"))
    q, s = _quant(x, F.BF16, 2, K)
    rq, rs = o8.quant_rows(_f64(x))
    assert np.array_equal(q, rq) and np.array_equal(s, rs)


@pytest.mark.parametrize("out", ["i8", "act"])
def test_a_stream_past_32_bits(out):
    M, D = (1 << 20) + 77, 2100
    g = torch.Generator(device="cuda").manual_seed(33)
    x = torch.empty(M, D, device="cuda").normal_(generator=g)
    y = torch.empty(M, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)

    def run(x, y):
        n = x.shape[0]
        h = torch.empty(n, D, device="cuda")
        a = torch.empty(n, D, dtype=torch.int8 if out == "i8" else torch.bfloat16, device="cuda")
        s = torch.empty(n, device="cuda")
        F.flashbon_op_norm_residual(F.BF16, n, D, EPS, x, y, post_norm=F.NORM_RMS, x_out=h,
                                    **(dict(q=a, q_scale=s) if out == "i8" else dict(out=a)))
        return (h, a, s) if out == "i8" else (h, a)

    whole, rows = run(x, y), _spread(M)
    few = run(x[rows].contiguous(), y[rows].contiguous())   # held to the oracle by the tests above
    assert all(torch.equal(p[rows], r) for p, r in zip(whole, few))


@pytest.mark.parametrize("K", [65536, 65533])
def test_layers_past_32_bits(K):
    """Rows that begin past 2^31 bytes of A, and weights that do."""
    for M, N in ((34000, 8), (5, 34000)):
        g = torch.Generator(device="cuda").manual_seed(34)
        a = torch.randint(-128, 128, (M, K), generator=g, device="cuda", dtype=torch.int8)
        w = torch.randint(-128, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
        sa, sw = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
        out = torch.empty(M, N, device="cuda")
        F.flashbon_op_linear_i8(F.FP32, M, N, K, a, sa, w, sw, None, F.EPI_STORE, out)
        for m in (0, 32767, 32768, M - 1) if M > N else range(M):
            for n in range(N) if M > N else (0, 32767, 32768, N - 1):
                acc = int((_f64(a[m]) * _f64(w[n])).sum())   # whole numbers below 2^30
                assert out[m, n].item() == np.float32(np.float32(acc) * np.float32(sw[n].item())) * np.float32(sa[m].item())


# ------------------------------------------------------------------------------------------- two threads at once
def test_two_threads_at_once():
    """Two branches, each on a thread and a stream of its own."""
    import threading

    branches = [Branch(130, 256, 704, 41), Branch(390, 136, 520, 42)]
    refs, failed = [], []
    for b in branches:
        b.x.normal_()
        b.run()
        torch.cuda.synchronize()
        refs.append(b.results())
        for t in (b.a, b.u, b.qu, b.y, b.out, b.next):
            t.zero_()
    torch.cuda.synchronize()

    def work(b):
        try:
            stream = torch.cuda.Stream()
            for _ in range(20):
                b.run(stream=stream.cuda_stream)
            stream.synchronize()
        except Exception as e:   # noqa: BLE001 - reported by the test's own thread
            failed.append(e)

    threads = [threading.Thread(target=work, args=(b,)) for b in branches]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
    for b, ref in zip(branches, refs):
        assert all(torch.equal(p, q) for p, q in zip(ref, b.results()))
