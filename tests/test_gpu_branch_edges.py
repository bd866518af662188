"""The cross-attention branch's kernels at the ends of their ranges, against 64 bits.

Tolerances count roundings as in test_gpu_branch: E is half a step of fp32, U[t] of the type t.
"""
import numpy as np
import pytest
import torch

import test_gpu_branch as base
from oracle import branch
from paper_2607_04461_amd import flashbon as fb
from test_gpu_branch import ACT, CODE, E, U, cuda, gen, near, normal, wide

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------ LayerNorm
def rows_at_the_ends(d):
    """Rows whose differences from their mean, their squares or their reciprocal deviation no fp32 holds, and ordinary ones."""
    r = np.random.default_rng(51)
    x = np.empty((7, d), np.float32)
    x[0] = np.where(np.arange(d) % 8 == 1, 3e38, -3e38)
    x[1] = np.where(np.arange(d) % 2, 3e38, -3e38)
    x[2] = 3e38 * r.uniform(0.5, 1, d)
    x[3] = 1e20 * r.standard_normal(d)
    x[4] = 1e-38 * r.standard_normal(d)
    x[5] = 3e18 * r.standard_normal(d) - 1e21
    x[6] = r.standard_normal(d)
    return torch.from_numpy(x)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [1, 2, 40, 701, 1536, 2100, 5120, 6143])
def test_layer_norm_at_the_ends_of_the_range(dtype, d):
    x, w, b = rows_at_the_ends(d), normal(gen(52), 1, d), normal(gen(53), 1, d)
    m = len(x)
    out, mean, rstd = torch.empty(m, d, dtype=ACT[dtype], device="cuda"), torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    fb.flashbon_op_layer_norm(CODE[dtype], m, d, 1e-6, cuda(x), out, weight=cuda(w), bias=cuda(b), mean=mean, rstd=rstd)
    y, mu, rs = branch.layer_norm(x, w, b, m, False, 1e-6)
    xh, f = base.norm_spread(x, w, False, m)
    # as in test_layer_norm; 1 / 3e38 lies below fp32's normal numbers, where a rounding is off by 2^-150 at most
    off = 2.0 ** -48 * np.abs(mu)[:, None] * rs[:, None]
    near(mean, mu, E * np.abs(mu) + 2.0 ** -52 * np.abs(wide(x)).sum(1), "mean")
    assert (np.abs(wide(rstd) - rs) <= 24 * E * rs + 2.0 ** -150).all(), "rstd"
    near(out, y, U[ACT[dtype]] * np.abs(y) + 32 * E * xh * f + 2 * E * np.abs(y) + off * f, "out")


@pytest.mark.parametrize("d", [40, 701, 2100])
def test_layer_norm_of_a_tiny_eps(d):
    """Variances and an eps below fp32's normal numbers."""
    x = normal(gen(54), 5, d) * torch.tensor([1e-21, 1e-22, 3e-20, 1e-30, 1.0])[:, None]
    eps = float(np.float32(1e-42))
    out, rstd = torch.empty(5, d, device="cuda"), torch.empty(5, device="cuda")
    fb.flashbon_op_layer_norm(fb.FP32, 5, d, eps, cuda(x), out, rstd=rstd)
    y, mu, rs = branch.layer_norm(x, None, None, 5, False, eps)
    xh, _ = base.norm_spread(x, None, False, 5)
    # a mean below the normal numbers is taken off in parts that are off by 2^-150 at most
    near(rstd, rs, 24 * E * rs, "rstd")
    near(out, y, 40 * E * np.abs(y) + 2.0 ** -48 * np.abs(mu)[:, None] * rs[:, None] + 2.0 ** -149 * rs[:, None], "out")
