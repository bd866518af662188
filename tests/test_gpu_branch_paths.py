"""The cross-attention branch's kernels at sizes that reach their rarer variants: prompts of many blocks of keys, many ranges of
keys, rows 2^23 elements apart, rows gathered by their adapters on wide layers, weight gradients alone.

Tolerances are those of test_gpu_branch, derived there.
"""
import numpy as np
import pytest
import torch

import test_gpu_branch as base
from oracle import branch
from paper_2607_04461_amd import flashbon as fb
from test_gpu_branch import E, U, near, wide

pytestmark = pytest.mark.gpu

#        batch heads kv dh  tq   tk  prompts lengths
LONG = [(2, 4, 2, 128, 130, 700, 2, [700, 70]),       # blocks of keys wholly past a prompt's end
        (2, 2, 1, 64, 130, 600, 2, [600, 40]),
        (3, 1, 1, 128, 70, 1030, 2, [1030, 0]),
        (3, 2, 2, 32, 70, 300, 3, [300, 100, 129]),
        (2, 1, 1, 16, 200, 520, 1, [513]),
        (2, 1, 1, 64, 3, 8200, 1, [8100]),            # more ranges of keys than a round of the join
        (1, 2, 1, 128, 1, 8192, 1, [8192]),
        (1, 1, 1, 8, 40, 4100, 1, [4099])]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", LONG, ids=str)
def test_long_prompts(dtype, shape):
    base.test_cross_attention(dtype, shape)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", LONG, ids=str)
def test_long_prompts_grad(dtype, shape):
    base.test_cross_attention_grad(dtype, shape)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(9, 2046, 4), (6, 4094, 6), (7, 5117, 2)], ids=str)
def test_layer_norm_rows_in_single_elements(dtype, shape):
    """Odd rows of every number of pieces a lane."""
    base.test_layer_norm(dtype, *shape)
    base.test_layer_norm_grad(dtype, *shape)


@pytest.mark.parametrize("dh", [32, 64, 128])
def test_keys_farther_apart_than_tiles_take(dh):
    """Key rows past 2^23 elements apart, whose offsets within a tile pass 31 bits."""
    heads, tq, tk, n, far = 2, 100, 67, 66, (1 << 23) + 8
    q, kv, _, _ = base.cross_inputs("bf16", 1, heads, heads, dh, tq, tk, 1, [n], 72)
    wide_ = heads * dh
    flat = torch.zeros((tk - 1) * far + 2 * wide_, dtype=torch.bfloat16, device="cuda")
    flat.as_strided((tk, 2 * wide_), (far, 1)).copy_(kv.reshape(tk, -1))
    out, lse = torch.empty(tq, wide_, dtype=torch.bfloat16, device="cuda"), torch.empty(1, heads, tq, device="cuda")
    fb.flashbon_op_cross_attention(fb.BF16, 1, heads, heads, dh, tq, tk, q.cuda(), 0, wide_, flat, flat[wide_:], 0, far, None, 1,
                                   torch.tensor([n], dtype=torch.int32, device="cuda"), out, 0, wide_, lse=lse)
    k, v = (base.clean(kv, [n])[:, :, i] for i in (0, 1))
    want, wl = branch.cross_attention(wide(q), wide(k), wide(v), [0], [n])
    rel = base.p_error(q, k, [0], wl)
    near(lse, wl, rel + 8 * E * np.abs(wl), "lse")
    mass, _ = branch.cross_attention(wide(q), wide(k), np.abs(wide(v)), [0], [n])
    u = U[torch.bfloat16]
    near(out.reshape(q.shape), want, u * np.abs(want) + (u + 2 * rel.transpose(0, 2, 1)[..., None] + (n + 8) * E) * (1 + 2 * u) * mass, "out")


def grad_bounds(q, k, v, out, lse, dout, n, u):
    """How far dq, dk and dv of one candidate may be off before they are rounded, as in test_cross_attention_grad."""
    _, tq, heads, dh = q.shape
    rel = base.p_error(q, k, [0], wide(lse))
    eq, ek, ev = np.zeros(q.shape), np.zeros(k.shape), np.zeros(k.shape)
    for h in range(heads):
        kh = h // (heads // k.shape[2])
        qb, kb, vb, do, ob = wide(q[0, :, h]), wide(k[0, :n, kh]), wide(v[0, :n, kh]), wide(dout[0, :, h]), wide(out[0, :, h])
        p = np.exp(qb @ kb.T / np.sqrt(dh) - wide(lse[0, h])[:, None])
        r = rel[0, h][:, None]
        d = do @ vb.T - (do * ob).sum(1, keepdims=True)
        ed = (dh + 4) * E * (np.abs(do) @ np.abs(vb).T + (np.abs(do) * np.abs(ob)).sum(1, keepdims=True))
        ds, es = p * np.abs(d), p * (np.abs(d) * (r + u + 4 * E) + 2 * ed)
        m = (n + 8) * E
        eq[0, :, h] = ((es + m * ds) @ np.abs(kb)) / np.sqrt(dh)
        m = (tq * heads + 16) * E
        ek[0, :n, kh] += ((es + m * ds).T @ np.abs(qb)) / np.sqrt(dh)
        ev[0, :n, kh] += (p * (r + u + m)).T @ np.abs(do)
    return eq, ek, ev


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("which", ["q", "kv"])
def test_gradients_of_rows_far_apart(which, dh):
    """Rows 2^23 elements apart: all gradients, from fused keys and values, by the kernels whose offsets are 64 bits."""
    heads, kvh, tq, tk, n, far = 2, 1, 70, 133, 130, 1 << 23
    q, kv, _, dout = base.cross_inputs("bf16", 1, heads, kvh, dh, tq, tk, 1, [n], 71)
    k, v = (base.clean(kv, [n])[:, :, i] for i in (0, 1))
    out, lse = branch.cross_attention(wide(q), wide(k), wide(v), [0], [n])
    out, lse = torch.tensor(out).to(torch.bfloat16), torch.tensor(lse, dtype=torch.float32)
    wide_, narrow = heads * dh, kvh * dh

    def rows(t, width, apart):
        """t's rows of `width` elements, `apart` elements from one to the next."""
        flat = torch.zeros((t.numel() // width - 1) * apart + width, dtype=torch.bfloat16, device="cuda")
        view = flat.as_strided((t.numel() // width, width), (apart, 1))
        view.copy_(t.reshape(-1, width))
        return view

    q_rs, kv_rs = (far, 2 * narrow) if which == "q" else (wide_, far)
    qd, kvd, dq, dkv = rows(q, wide_, q_rs), rows(kv, 2 * narrow, kv_rs), rows(q, wide_, q_rs), rows(kv, 2 * narrow, kv_rs)
    sizes = (fb.BF16, 1, heads, kvh, dh, tq, tk)
    ws = torch.full((fb.flashbon_op_cross_attention_grad_workspace(*sizes, 1),), 255, dtype=torch.uint8, device="cuda")
    fb.flashbon_op_cross_attention_grad(*sizes, qd, 0, q_rs, kvd[:, :narrow], kvd[:, narrow:], 0, kv_rs, None, 1,
                                        torch.tensor([n], dtype=torch.int32, device="cuda"), out.cuda(), 0, wide_, lse.cuda(), dout.cuda(), dq,
                                        dkv[:, :narrow], dkv[:, narrow:], workspace=ws)
    tq_, tk_, tv_ = branch.cross_attention_grad(wide(q), wide(k), wide(v), wide(out), wide(lse), wide(dout), [0], [n])
    u = U[torch.bfloat16]
    eq, ek, ev = grad_bounds(q, k, v, out, lse, dout, n, u)
    near(dq.reshape(q.shape), tq_, u * np.abs(tq_) + 1.01 * eq, "dq")
    got = dkv.reshape(tk, 2, kvh, dh)
    near(got[:, 0], tk_[0], u * np.abs(tk_[0]) + 1.01 * ek[0], "dk")
    near(got[:, 1], tv_[0], u * np.abs(tv_[0]) + 1.01 * ev[0], "dv")


#             M    N    K   rank count per
GATHERED = [(64, 2056, 264, 32, 3, 1), (70, 136, 264, 128, 3, 1), (66, 2072, 136, 64, 3, 2), (70, 2056, 72, 24, 2, 3), (300, 72, 2120, 40, 7, 5)]
FORMS = [("bf16", "store"), ("bf16", "f32"), ("fp32", "store")]


@pytest.mark.parametrize("dtype,epi", FORMS + [("bf16", "residual"), ("fp32", "residual")])
@pytest.mark.parametrize("shape", GATHERED, ids=str)
def test_adapters_of_gathered_rows(dtype, epi, shape):
    """Single rows of a few adapters on layers or ranks too large for one launch."""
    base.test_adapters(dtype, epi, shape)


@pytest.mark.parametrize("dtype,epi", FORMS)
@pytest.mark.parametrize("shape", GATHERED, ids=str)
def test_adapters_grad_of_gathered_rows(dtype, epi, shape):
    base.test_adapters_grad(dtype, epi, shape)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rank", [16, 24, 64, 72])
def test_weight_gradients_alone_of_many_rows(dtype, rank):
    """Without dx the first product runs by itself, on up to 64 rows a tile."""
    base.test_adapters_grad(dtype, "store", (16500, 40, 24, rank, 2, 4130))
    base.test_adapters_grad(dtype, "store", (16384, 24, 72, rank, 1, 16384))


@pytest.mark.parametrize("dtype,epi", FORMS)
@pytest.mark.parametrize("shape", [(8300, 72, 40, 16, 2, 4150), (8300, 40, 72, 32, 2, 4150), (4400, 72, 40, 32, 2, 2200),
                                   (4400, 40, 72, 64, 2, 2200), (4400, 72, 40, 128, 2, 2200), (130, 2056, 264, 32, 2, 65)], ids=str)
def test_adapters_by_rows_of_a_tile(dtype, epi, shape):
    """32 rows a tile, 16, and so few that both products run by themselves."""
    base.test_adapters(dtype, epi, shape)
    base.test_adapters_grad(dtype, epi, shape)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [8300, 16500])
def test_adapters_of_rank_above_64_in_tiles_of_32_rows(dtype, m):
    base.test_adapters(dtype, "store", (m, 72, 40, 96, 2, 4130))
