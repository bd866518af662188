"""8-bit layers: every layout of the row kernels, and the kernels that large layers take by themselves, against the
64-bit oracle and against each other."""
import numpy as np
import pytest
import torch

from oracle import int8 as o8
from paper_2607_04461_amd import flashbon as F
from test_gpu_int8 import ACT, CODE, EPS, Out, _codes, _dev, _f64, _linear, _quant, _seam

pytestmark = pytest.mark.gpu

MANY = 530          # more rows than two a CU


# ------------------------------------------------------------------------------------------ rows to codes
# the longest and the shortest row of every number of threads and pieces a row, whole pieces and not
BOUNDS = [128, 256, 512, 768, 1024, 1536, 2048, 4096, 6144, 8192, 10240, 12288, 16384, 24576, 32768, 49152, 65536]
LENGTHS = sorted({k for b in BOUNDS for k in (b, b - 3, b + 1, b + 8) if k <= 65536} | {5, 5120, 8960, 13824})


@pytest.mark.parametrize("K", LENGTHS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_codes_of_every_layout(K, dtype):
    d, M = CODE[dtype], 19
    x = _dev(np.random.default_rng([1, K]).standard_normal((M, K)) * np.exp(np.arange(M) - 9.0)[:, None], ACT[d])
    x[7, K - 1], x[11, K // 2], x[13] = float("inf"), float("nan"), 0.0
    q, s = _quant(x, d, M, K)
    rq, rs = o8.quant_rows(_f64(x))
    assert np.array_equal(s, rs, equal_nan=True) and np.array_equal(q, rq)


# ------------------------------------------------------------------------------------------------ seams
# threads and pieces a row change past 128, 256, 512, 1024, 1536, 2048 and 4096; whole rows, whole pieces, neither
NARROW = [120, 125, 128, 130, 250, 256, 264, 400, 509, 512]
WIDE = [2050, 2056, 2500, 4090, 4096, 4097, 4104, 5120, 6141, 6144]
LAYERED = [513, 520, 1000, 1024, 1027, 1032, 1528, 1536, 1537, 1544, 1600, 2040, 2045, 2048]   # by the number of rows, too


@pytest.mark.parametrize("M,D", [(21, d) for d in NARROW] + [(5, d) for d in WIDE + LAYERED] + [(MANY, d) for d in LAYERED])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("out", ["i8", "act", "none"])
def test_seam_of_every_layout(M, D, dtype, out):
    _seam(M, D, dtype, out=out)


@pytest.mark.parametrize("post,pre", [("none", "layer"), ("layer", "rms"), ("layer", "none")])
@pytest.mark.parametrize("out", ["i8", "act"])
@pytest.mark.parametrize("D", [1024, 1536, 1537, 2040, 2048])
def test_seam_norms_of_many_rows(D, out, post, pre):
    _seam(MANY, D, "bf16", post, pre, out)


@pytest.mark.parametrize("kw", [dict(vectors=False), dict(branch=False), dict(x_out="x"), dict(x_out=None),
                                dict(branch=False, x_out="x"), dict(offset=3, x_out="x")])
@pytest.mark.parametrize("out", ["i8", "act"])
@pytest.mark.parametrize("D", [1536, 1541, 1600])
def test_seam_options_of_many_rows(kw, out, D):
    _seam(MANY, D, "bf16", out=out, **kw)


# streams of 64 MiB and more, which are stored past the caches: rows of whole pieces that fill their threads, and that do not
@pytest.mark.parametrize("M,D,dtype,kw", [
    (10925, 1536, "bf16", dict(out="i8")), (10925, 1536, "fp32", dict(out="act", x_out="x")),
    (16400, 1024, "bf16", dict(out="act")), (8200, 2048, "bf16", dict(out="i8", x_out="x")),
    (16780, 1000, "bf16", dict(out="i8")), (16780, 1000, "bf16", dict(out="act", branch=False)),
    (3280, 5120, "bf16", dict(out="act")), (3280, 5120, "fp32", dict(out="i8")), (4110, 4088, "bf16", dict(out="none")),
    (131100, 128, "bf16", dict(out="i8")), (7000, 2400, "bf16", dict(out="act"))])
def test_seams_of_large_streams(M, D, dtype, kw):
    assert M * D * 4 >= 64 << 20
    _seam(M, D, dtype, **kw)


# ------------------------------------------------------------------------------------------------ products
RING = ["256x256", "128x256", "128x128:two", "128x128", "96x128", "64x128"]


class Layer:
    """A layer's operands, and its outputs by a kernel of choice (None: the library's)."""

    def __init__(self, M, N, K, dtype, epi, monkeypatch):
        r = np.random.default_rng([9, M, N, K])
        self.shape, self.dtype, self.env = (M, N, K), CODE[dtype], monkeypatch
        self.epi = {"store": F.EPI_STORE, "gelu": F.EPI_GELU, "store_f32": F.EPI_STORE_F32, "residual": F.EPI_RESIDUAL}[epi]
        f = lambda *s: r.standard_normal(s, dtype=np.float32)  # noqa: E731
        self.A, self.W = _dev(_codes(r, M, K, True), torch.int8), _dev(_codes(r, N, K, True), torch.int8)
        self.sa, self.sw, self.bias, self.gate = _dev(np.exp(f(M) - 4)), _dev(np.exp(f(N) - 5)), _dev(f(N)), _dev(f(N))
        self.h = _dev(f(M, N)) if epi == "residual" else None
        self.stores = ACT[self.dtype] if epi in ("store", "gelu") else torch.float32

    def run(self, tile=None, cache=True):
        M, N, K = self.shape
        if tile is None:
            self.env.delenv("FLASHBON_I8_TILE", raising=False)
        else:
            self.env.setenv("FLASHBON_I8_TILE", tile)
        out = Out(M * N, self.stores, 32)                    # on 16 bytes
        copy = Out(M * N, torch.float32, 32) if cache and self.h is not None else None
        F.flashbon_op_linear_i8(self.dtype, M, N, K, self.A, self.sa, self.W, self.sw, self.bias, self.epi, out.view,
                                gate=self.gate, residual_in=self.h, cache_out=copy.view if copy else None)
        torch.cuda.synchronize()
        out.check()
        if copy:
            copy.check()
            assert torch.equal(copy.view, out.view)
        return out.view


# what the library takes by itself, more than one round of workgroups and groups of row blocks whose last is not whole:
# 256x256 and 128x256 tiles, two 128x128 a CU, blocks of two heights (32 rows times 8 or 7, 7 or 6, 6 or 5); and an odd one
@pytest.mark.parametrize("M,N,K,epi", [
    (2600, 2312, 272, "store"), (2600, 4104, 4112, "residual"), (4000, 2056, 400, "gelu"), (6453, 2408, 272, "store"),
    (4680, 1536, 1552, "residual"), (5684, 2400, 144, "gelu"), (8849, 1288, 144, "gelu"), (9000, 3584, 272, "store_f32"),
    (2500, 2501, 1003, "residual")])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_layers_against_the_oracle(M, N, K, epi, dtype, monkeypatch):
    first = _linear(M, N, K, dtype, epi)
    monkeypatch.setenv("FLASHBON_I8_TILE", "any")
    assert torch.equal(_linear(M, N, K, dtype, epi), first)


def test_the_pools_layers_by_two_kernels(monkeypatch):
    """Whole outputs of the library's own choice and of the tiles for any size."""
    for M, N, K, epi in ((24960, 4608, 1536, "store"), (24960, 1536, 1536, "residual"), (24960, 8960, 1536, "gelu"),
                         (24960, 1536, 8960, "residual"), (65536, 1536, 256, "store")):
        layer = Layer(M, N, K, "bf16", epi, monkeypatch)
        own = layer.run()
        print(M, N, K, epi, flush=True)
        assert torch.equal(own, layer.run("any")), (M, N, K, epi)


# outputs of 64 MiB and more, which are stored past the caches, and of less: every tile, row blocks of every two heights
LARGE = [(4100, 4104, 272, "residual", "bf16"), (8200, 4104, 400, "gelu", "bf16"), (8200, 4104, 400, "store", "bf16"),
         (4100, 4104, 144, "store", "fp32"), (4100, 4104, 528, "gelu", "fp32"), (2100, 2312, 272, "residual", "bf16"),
         (2100, 4104, 4112, "store", "bf16")]


@pytest.mark.parametrize("M,N,K,epi,dtype", LARGE)
def test_every_kernel_gives_the_same_bits_of_large_layers(M, N, K, epi, dtype, monkeypatch):
    layer = Layer(M, N, K, dtype, epi, monkeypatch)
    first = layer.run("any")
    for tile in RING:
        assert torch.equal(layer.run(tile), first), tile
    for w in (8, 7, 6):
        lo = 32 * (w - 1)
        least, most = -(-M // (lo + 32)), -(-M // lo)
        for blocks in {least, (least + most) // 2, most}:
            tall = max(0, -(-(M - lo * blocks) // 32))
            assert torch.equal(layer.run(f"mix:{w}:{blocks}:{tall}"), first), (w, blocks, tall)


def test_every_kernel_gives_the_oracles_large_layers(monkeypatch):
    """The bits of the test above are those of the kernel that the oracle holds here, on the same shapes."""
    monkeypatch.setenv("FLASHBON_I8_TILE", "any")
    for M, N, K, epi, dtype in LARGE:
        print(M, N, K, epi, dtype, flush=True)
        _linear(M, N, K, dtype, epi, offset=32)
