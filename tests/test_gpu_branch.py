"""The cross-attention branch's kernels against 64 bits: LayerNorm, attention to prompts of their own lengths and low-rank
adapters, forward and backward, and a branch of all of them.

Tolerances count roundings: a value rounded to a type is off by at most ``finfo.eps / 2`` of itself (U below), and a sum of n
fp32 products by at most n 2^-24 of the sum of their magnitudes, whatever the order.  Where a value that was rounded (P and
dS of attention, the split factors of adapters) is summed, its rounding counts against the magnitudes it meets.
"""
import numpy as np
import pytest
import torch

from oracle import branch
from paper_2607_04461_amd import flashbon as fb

pytestmark = pytest.mark.gpu

CODE = {"bf16": fb.BF16, "fp32": fb.FP32}
ACT = {"bf16": torch.bfloat16, "fp32": torch.float32}
U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
E = 2.0 ** -24


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(*shape, generator=g) * std).to(dtype)


def cuda(t):
    return None if t is None else t.cuda()


def wide(t):
    return None if t is None else t.detach().cpu().double().numpy()


def near(got, want, tol, what):
    """Every element within its tolerance (or the same infinity)."""
    g, want, tol = wide(got), np.broadcast_to(want, got.shape), np.broadcast_to(tol, got.shape)
    fine = np.isfinite(want)
    assert np.array_equal(g[~fine], want[~fine]), f"{what}: infinities"
    bad = ~(np.abs(g - np.where(fine, want, 0)) <= tol + 1e-37) & fine
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0]}: {g[bad][0]} for {want[bad][0]} +- {tol[bad][0]}"


# ------------------------------------------------------------------------------------------------------ LayerNorm
NORMS = [(1, 1, 1), (1, 1536, 1), (3, 2, 2), (5, 7, 1), (17, 64, 5), (33, 512, 33), (70, 516, 20), (9, 1535, 4), (130, 1536, 100),
         (41, 2048, 7), (13, 2052, 13), (19, 4096, 6), (21, 5120, 8), (7, 6143, 3), (6, 6144, 6), (2100, 40, 700), (1500, 96, 1500)]


def norm_inputs(dtype, m, d, per, seed, modulated):
    g, groups = gen(seed), -(-m // per)
    x = normal(g, m, d) * torch.exp(normal(g, m, 1)) + normal(g, m, 1, std=3.0)
    w, b = normal(g, groups, d, std=0.5) + (0 if modulated else 1), normal(g, groups, d)
    return x, w, b, normal(g, m, d, dtype=ACT[dtype]), normal(g, m, d)


def norm_spread(x, w, modulated, per):
    """|xhat f| of each element, and the rows' |f|."""
    xh, _, _ = branch.layer_norm(wide(x), None, None, 1, False, 1e-6)
    f = 1.0 if w is None else np.abs(wide(w)[np.arange(len(x)) // per] + (1 if modulated else 0))
    return np.abs(xh), f


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m,d,per", NORMS)
def test_layer_norm(dtype, m, d, per):
    modulated = (m + d) % 2 == 0
    x, w, b, _, _ = norm_inputs(dtype, m, d, per, 1, modulated)
    out, mean, rstd = torch.empty(m, d, dtype=ACT[dtype], device="cuda"), torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    fb.flashbon_op_layer_norm(CODE[dtype], m, d, 1e-6, cuda(x), out, weight=cuda(w), bias=cuda(b), rows_per_group=per,
                              modulated=modulated, mean=mean, rstd=rstd)
    y, mu, rs = branch.layer_norm(x, w, b, per, modulated, 1e-6)
    xh, f = norm_spread(x, w, modulated, per)
    # a row's squares: at most 24 on a lane, then 8 levels, each value off by 3 roundings: 38 in the sum, half in rstd, 4 more;
    # the mean in two parts of fp32 is off by 2^-48, the values by 2^-48 |mean| rstd
    off = 2.0 ** -48 * np.abs(mu)[:, None] * rs[:, None]
    near(mean, mu, E * np.abs(mu) + 2.0 ** -52 * np.abs(wide(x)).sum(1), "mean")
    near(rstd, rs, 24 * E * rs, "rstd")
    near(out, y, U[ACT[dtype]] * np.abs(y) + 32 * E * xh * f + 2 * E * np.abs(y) + off * f, "out")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m,d,per", NORMS)
def test_layer_norm_grad(dtype, m, d, per):
    modulated = (m + d) % 2 == 1
    x, w, _, dy, res = norm_inputs(dtype, m, d, per, 2, modulated)
    _, mu, rs = branch.layer_norm(x, w, None, per, modulated, 1e-6)
    mean, rstd = torch.tensor(mu, dtype=torch.float32), torch.tensor(rs, dtype=torch.float32)
    groups = -(-m // per)
    dx, dw, db = torch.empty(m, d, device="cuda"), torch.empty(groups, d, device="cuda"), torch.empty(groups, d, device="cuda")
    ws = torch.full((fb.flashbon_op_layer_norm_grad_workspace(m, d, per),), 255, dtype=torch.uint8, device="cuda")
    fb.flashbon_op_layer_norm_grad(CODE[dtype], m, d, cuda(x), cuda(mean), cuda(rstd), cuda(dy), dx, weight=cuda(w),
                                   rows_per_group=per, modulated=modulated, residual=cuda(res), dweight=dw, dbias=db, workspace=ws)
    tx, tw, tb = branch.layer_norm_grad(x, w, per, modulated, wide(mean), wide(rstd), dy.float(), res)
    xh = np.abs((wide(x) - wide(mean)[:, None]) * wide(rstd)[:, None])
    f = np.abs(wide(w)[np.arange(m) // per] + (1 if modulated else 0))
    g, ay = np.abs(wide(dy)) * f, np.abs(wide(dy))
    n = 24 + 8 + 4           # sums along a row: 24 on a lane, 8 levels, products' roundings
    mean_g, mean_gx = g.mean(1, keepdims=True), (g * xh).mean(1, keepdims=True)
    tol = E * (2 * np.abs(tx) + wide(rstd)[:, None] * (6 * g + (n + 4) * mean_g + xh * (n + 8) * mean_gx))
    near(dx, tx, tol, "dx")
    rows = [slice(i * per, min(m, (i + 1) * per)) for i in range(groups)]
    # sums over rows: 16 rows (or a 1024th of them) in fp32, then four waves, chunks in 64 bits; three roundings each before
    n = max(16, m // 1024 + 1) + 4 + 4
    near(dw, tw, n * E * np.stack([(ay * xh)[r].sum(0) for r in rows]), "dweight")
    near(db, tb, n * E * np.stack([ay[r].sum(0) for r in rows]), "dbias")


def test_layer_norm_without_vectors_and_parts():
    m, d = 40, 200
    x, _, _, dy, _ = norm_inputs("bf16", m, d, m, 3, False)
    out = torch.empty(m, d, dtype=torch.bfloat16, device="cuda")
    fb.flashbon_op_layer_norm(fb.BF16, m, d, 1e-6, cuda(x), out)
    y, mu, rs = branch.layer_norm(x, None, None, m, False, 1e-6)
    near(out, y, (U[torch.bfloat16] + 40 * E) * np.abs(y) + 2.0 ** -40, "out")
    mean, rstd = torch.tensor(mu, dtype=torch.float32).cuda(), torch.tensor(rs, dtype=torch.float32).cuda()
    dx, only = torch.empty(m, d, device="cuda"), torch.empty(m, d, device="cuda")
    db, dw = torch.empty(1, d, device="cuda"), torch.empty(1, d, device="cuda")
    ws = torch.empty(fb.flashbon_op_layer_norm_grad_workspace(m, d), dtype=torch.uint8, device="cuda")
    fb.flashbon_op_layer_norm_grad(fb.BF16, m, d, cuda(x), mean, rstd, cuda(dy), dx, dweight=dw, dbias=db, workspace=ws)
    fb.flashbon_op_layer_norm_grad(fb.BF16, m, d, cuda(x), mean, rstd, cuda(dy), only)
    assert torch.equal(dx, only)
    other = torch.empty(1, d, device="cuda")
    fb.flashbon_op_layer_norm_grad(fb.BF16, m, d, cuda(x), mean, rstd, cuda(dy), dbias=other, workspace=ws)
    assert torch.equal(other, db)
    # in place onto the residual stream's gradient
    res = normal(gen(4), m, d).cuda()
    want, inplace = torch.empty(m, d, device="cuda"), res.clone()
    fb.flashbon_op_layer_norm_grad(fb.BF16, m, d, cuda(x), mean, rstd, cuda(dy), want, residual=res)
    fb.flashbon_op_layer_norm_grad(fb.BF16, m, d, cuda(x), mean, rstd, cuda(dy), inplace, residual=inplace)
    assert torch.equal(want, inplace)


@pytest.mark.parametrize("d", [1536, 5120, 701])
def test_layer_norm_rows_far_from_zero_and_flat(d):
    """Rows whose mean is 10^4 times their deviation keep their digits; rows of one value become the bias."""
    x = normal(gen(5), 6, d, std=0.5) + 5000.0
    x[2] = 7.25
    b = normal(gen(6), 1, d)
    out = torch.empty(6, d, device="cuda")
    fb.flashbon_op_layer_norm(fb.FP32, 6, d, 1e-6, cuda(x), out, bias=cuda(b))
    y, mu, rs = branch.layer_norm(x, None, b, 6, False, 1e-6)
    near(out, y, 40 * E * (np.abs(y) + np.abs(wide(b))) + 2.0 ** -46 * np.abs(mu)[:, None] * rs[:, None], "out")
    assert torch.equal(out[2].cpu(), b[0])


@pytest.mark.parametrize("d", [96, 5120])
def test_layer_norm_rows_stand_alone(d):
    """A row's bits do not depend on the others, nor on the place of the buffers; NaN stays in its row."""
    x, w, b, dy, _ = norm_inputs("fp32", 37, d, 37, 7, False)
    x[5, 3] = float("nan")
    whole, one = torch.empty(37, d, device="cuda"), torch.empty(1, d, device="cuda")
    fb.flashbon_op_layer_norm(fb.FP32, 37, d, 1e-6, cuda(x), whole, weight=cuda(w), bias=cuda(b))
    for row in (0, 11, 36):
        fb.flashbon_op_layer_norm(fb.FP32, 1, d, 1e-6, cuda(x[row:row + 1]), one, weight=cuda(w), bias=cuda(b))
        assert torch.equal(one[0], whole[row])
    bad = torch.isnan(whole).any(1).cpu()
    assert bad.nonzero().flatten().tolist() == [5]


def test_layer_norm_off_sixteen_bytes():
    m, d = 21, 64
    x, w, b, dy, res = norm_inputs("bf16", m, d, 7, 8, True)
    shifted = lambda t: torch.cat([t.flatten()[:1], t.flatten()]).cuda()[1:].view(t.shape)  # noqa: E731
    out = torch.empty(m, d, dtype=torch.bfloat16, device="cuda")
    fb.flashbon_op_layer_norm(fb.BF16, m, d, 1e-6, shifted(x), out, weight=shifted(w), bias=shifted(b), rows_per_group=7, modulated=True)
    y, _, _ = branch.layer_norm(x, w, b, 7, True, 1e-6)
    xh, f = norm_spread(x, w, True, 7)
    near(out, y, U[torch.bfloat16] * np.abs(y) + 32 * E * xh * f + 2 * E * np.abs(y) + 2.0 ** -40, "out")


# ------------------------------------------------------------------------------------------------ cross-attention
#         batch heads kv dh  tq   tk  prompts lengths
CROSSES = [(1, 1, 1, 8, 1, 1, 1, [1]),
           (1, 2, 1, 16, 3, 5, 1, [4]),
           (2, 4, 4, 32, 17, 33, 2, [33, 0]),
           (3, 4, 2, 64, 65, 64, 2, [64, 1]),
           (3, 6, 2, 128, 70, 65, 3, [65, 64, 63]),
           (2, 2, 2, 128, 129, 130, 1, [129]),
           (5, 3, 1, 64, 130, 200, 2, [7, 200]),
           (2, 8, 1, 128, 33, 97, 2, [96, 97]),
           (1, 5, 5, 128, 1, 700, 1, [641]),
           (2, 2, 1, 32, 5, 1100, 2, [1100, 300]),
           (4, 1, 1, 8, 300, 20, 3, [20, 5, 20]),
           (1, 12, 12, 128, 200, 77, 1, [77])]


def cross_inputs(dtype, batch, heads, kvh, dh, tq, tk, prompts, lengths, seed):
    """q, fused keys and values with NaN and infinities past each prompt's end, and the prompt of each batch row."""
    g, act = gen(seed), ACT[dtype]
    q, kv = normal(g, batch, tq, heads, dh, dtype=act), normal(g, prompts, tk, 2, kvh, dh, dtype=act)
    for c, n in enumerate(lengths):
        kv[c, n:] = float("nan")
        kv[c, n::2] = float("inf")
    index = [(2 * b + 1) % prompts for b in range(batch)]
    return q, kv, index, normal(g, batch, tq, heads, dh, dtype=act)


def clean(kv, lengths):
    kv = kv.clone()
    for c, n in enumerate(lengths):
        kv[c, n:] = 0
    return kv


def cross_call(dtype, q, kv, index, lengths, lse=True, workspace=True):
    batch, tq, heads, dh = q.shape
    prompts, tk, _, kvh, _ = kv.shape
    sizes = (CODE[dtype], batch, heads, kvh, dh, tq, tk)
    qd, kvd = q.cuda(), kv.cuda()
    out = torch.empty_like(qd)
    ls = torch.empty(batch, heads, tq, device="cuda") if lse else None
    ws = torch.full((fb.flashbon_op_cross_attention_workspace(*sizes),), 255, dtype=torch.uint8, device="cuda") if workspace else None
    i32 = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    q_strides, kv_strides = (tq * heads * dh, heads * dh), (tk * 2 * kvh * dh, 2 * kvh * dh)
    fb.flashbon_op_cross_attention(*sizes, qd, *q_strides, kvd[:, :, 0], kvd[:, :, 1], *kv_strides, i32(index), prompts,
                                   i32(lengths), out, *q_strides, lse=ls, workspace=ws)
    return out, ls


def score_error(q, k, index):
    """How far a score may be off, for each batch row and head: fp32 products and their scaling, on the largest rows."""
    a, b = np.abs(wide(q)), np.abs(wide(k))
    dh, per = q.shape[3], q.shape[2] // k.shape[2]
    top_q, top_k = a.sum(3).max(1), b.max((1, 3))
    top_k = np.repeat(top_k, per, 1)[index]
    return (dh + 8) * E * top_q * top_k / np.sqrt(dh)


def p_error(q, k, index, lse):
    """How far exp(score - lse) may be off, relative: the score's error, that of lse twice, and the exponential's steps."""
    s = score_error(q, k, index)[:, :, None]
    return 2 * s + 4 * E * np.where(np.isfinite(lse), np.abs(lse), 0) + 16 * E


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", CROSSES, ids=str)
def test_cross_attention(dtype, shape):
    *sizes, lengths = shape
    q, kv, index, _ = cross_inputs(dtype, *sizes, lengths, 11)
    got, lse = cross_call(dtype, q, kv, index, lengths)
    kv = clean(kv, lengths)
    k, v = kv[:, :, 0], kv[:, :, 1]
    out, want = branch.cross_attention(wide(q), wide(k), wide(v), index, lengths)
    rel = p_error(q, k, index, want)
    near(lse, want, rel + 8 * E * np.where(np.isfinite(want), np.abs(want), 0), "lse")
    mass, _ = branch.cross_attention(wide(q), wide(k), np.abs(wide(v)), index, lengths)      # sum p |v|
    u = U[ACT[dtype]]
    tol = u * np.abs(out) + (u + 2 * rel.transpose(0, 2, 1)[..., None] + (max(lengths) + 8) * E) * (1 + 2 * u) * mass
    near(got, out, tol, "out")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", CROSSES, ids=str)
def test_cross_attention_grad(dtype, shape):
    (batch, heads, kvh, dh, tq, tk, prompts), lengths = shape[:-1], shape[-1]
    q, kv, index, dout = cross_inputs(dtype, *shape[:-1], lengths, 12)
    zero = clean(kv, lengths)
    k, v = zero[:, :, 0], zero[:, :, 1]
    out, lse = branch.cross_attention(wide(q), wide(k), wide(v), index, lengths)
    out, lse = torch.tensor(out).to(ACT[dtype]), torch.tensor(lse, dtype=torch.float32)
    sizes = (CODE[dtype], batch, heads, kvh, dh, tq, tk)
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device="cuda")  # noqa: E731
    dq, dkv = torch.full_like(q, 9.0).cuda(), torch.full_like(kv, 9.0).cuda()
    ws = torch.full((fb.flashbon_op_cross_attention_grad_workspace(*sizes, prompts),), 255, dtype=torch.uint8, device="cuda")
    kvd, qs, ks = kv.cuda(), (tq * heads * dh, heads * dh), (tk * 2 * kvh * dh, 2 * kvh * dh)
    args = (*sizes, q.cuda(), *qs, kvd[:, :, 0], kvd[:, :, 1], *ks, i32(index), prompts, i32(lengths), out.cuda(), *qs, lse.cuda(), dout.cuda())
    fb.flashbon_op_cross_attention_grad(*args, dq, dkv[:, :, 0], dkv[:, :, 1], workspace=ws)
    tq_, tk_, tv_ = branch.cross_attention_grad(wide(q), wide(k), wide(v), wide(out), wide(lse), wide(dout), index, lengths)
    # errors: of P relative (rel), of dS absolute; sums over keys, and over queries, heads and candidates
    u = U[ACT[dtype]]
    rel = p_error(q, k, index, wide(lse))
    eq, ek, ev = np.zeros(q.shape), np.zeros(k.shape), np.zeros(k.shape)
    for b in range(batch):
        c = index[b]
        n = lengths[c]
        if n == 0:
            continue
        for h in range(heads):
            kh = h // (heads // kvh)
            qb, kb, vb, do, ob = wide(q[b, :, h]), wide(k[c, :n, kh]), wide(v[c, :n, kh]), wide(dout[b, :, h]), wide(out[b, :, h])
            p = np.exp(qb @ kb.T / np.sqrt(dh) - wide(lse[b, h])[:, None])
            r = rel[b, h][:, None]
            d = do @ vb.T - (do * ob).sum(1, keepdims=True)
            ed = (dh + 4) * E * (np.abs(do) @ np.abs(vb).T + (np.abs(do) * np.abs(ob)).sum(1, keepdims=True))
            ds, es = p * np.abs(d), p * (np.abs(d) * (r + u + 4 * E) + 2 * ed)
            m = (n + 8) * E
            eq[b, :, h] = ((es + m * ds) @ np.abs(kb)) / np.sqrt(dh)
            m = (tq * batch * heads + 16) * E
            ek[c, :n, kh] += ((es + m * ds).T @ np.abs(qb)) / np.sqrt(dh)
            ev[c, :n, kh] += (p * (r + u + m)).T @ np.abs(do)
    near(dq, tq_, u * np.abs(tq_) + 1.01 * eq, "dq")
    near(dkv[:, :, 0], tk_, u * np.abs(tk_) + 1.01 * ek, "dk")
    near(dkv[:, :, 1], tv_, u * np.abs(tv_) + 1.01 * ev, "dv")
    # one part alone has the same bits
    alone, alone_kv = torch.empty_like(dq), torch.empty_like(dkv)
    fb.flashbon_op_cross_attention_grad(*args, alone, workspace=ws)
    fb.flashbon_op_cross_attention_grad(*args, None, alone_kv[:, :, 0], alone_kv[:, :, 1], workspace=ws)
    assert torch.equal(alone, dq) and torch.equal(alone_kv, dkv)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dh", [16, 64, 128])
def test_cross_attention_grad_of_one_key(dtype, dh):
    """One key has probability 1 whatever its score: nothing reaches q and k, and dv is the sum of dout."""
    q, kv, _, dout = cross_inputs(dtype, 2, 2, 1, dh, 70, 3, 2, [1, 1], 19)
    out, lse = cross_call(dtype, q, kv, [0, 1], [1, 1])
    sizes, qs, ks = (CODE[dtype], 2, 2, 1, dh, 70, 3), (70 * 2 * dh, 2 * dh), (3 * 2 * dh, 2 * dh)
    dq, dkv = torch.full_like(q, 9.0).cuda(), torch.full_like(kv, 9.0).cuda()
    ws = torch.empty(fb.flashbon_op_cross_attention_grad_workspace(*sizes, 2), dtype=torch.uint8, device="cuda")
    kvd, i32 = kv.cuda(), lambda t: torch.tensor(t, dtype=torch.int32, device="cuda")  # noqa: E731
    fb.flashbon_op_cross_attention_grad(*sizes, q.cuda(), *qs, kvd[:, :, 0], kvd[:, :, 1], *ks, i32([0, 1]), 2, i32([1, 1]), out, *qs, lse,
                                        dout.cuda(), dq, dkv[:, :, 0], dkv[:, :, 1], workspace=ws)
    assert not dq.any() and not dkv[:, :, 0].any() and not dkv[:, 1:].any()
    want = wide(dout).sum((1, 2))
    # 140 terms of P = 1 within 16 E and a rounding, summed in fp32
    near(dkv[:, 0, 1, 0], want, U[ACT[dtype]] * np.abs(want) + (U[ACT[dtype]] + 170 * E) * np.abs(wide(dout)).sum((1, 2)), "dv")


@pytest.mark.parametrize("tk,pad,swap", [(1, 0, False), (1, 8, True), (5, 8, False), (5, 24, True), (1, 0, True)])
def test_cross_attention_grad_into_fused_rows(tk, pad, swap):
    """dk and dv in one buffer of alternating rows, one key a prompt among them, and prompts further apart than their rows:
    the same as in two buffers, and what lies between is left as it was."""
    heads, dh, tq, prompts = 2, 16, 9, 3
    d, g = heads * dh, gen(18)
    bs = tk * 2 * d + pad
    store = normal(g, prompts * bs, dtype=torch.bfloat16).cuda()
    first, second = store[: prompts * bs - d], store[d:]
    k, v = (second, first) if swap else (first, second)
    q, dout = normal(g, prompts, tq, d, dtype=torch.bfloat16).cuda(), normal(g, prompts, tq, d, dtype=torch.bfloat16).cuda()
    out, lse = torch.empty_like(q), torch.empty(prompts, heads, tq, device="cuda")
    sizes, qs = (fb.BF16, prompts, heads, heads, dh, tq, tk), (tq * d, d)
    fb.flashbon_op_cross_attention(*sizes, q, *qs, k, v, bs, 2 * d, None, prompts, None, out, *qs, lse=lse)
    ws = torch.empty(fb.flashbon_op_cross_attention_grad_workspace(*sizes, prompts), dtype=torch.uint8, device="cuda")
    args = (*sizes, q, *qs, k, v, bs, 2 * d, None, prompts, None, out, *qs, lse, dout)
    fused = torch.full_like(store, 9.0)
    one, two = fused[: prompts * bs - d], fused[d:]
    dk, dv = (two, one) if swap else (one, two)
    fb.flashbon_op_cross_attention_grad(*args, None, dk, dv, workspace=ws)
    apart = [torch.full_like(store, 9.0) for _ in range(2)]
    fb.flashbon_op_cross_attention_grad(*args, None, *apart, workspace=ws)
    rows = lambda t: torch.stack([t[c * bs:c * bs + tk * 2 * d].view(tk, 2, d) for c in range(prompts)])  # noqa: E731
    got, half = rows(fused), 1 if swap else 0
    assert torch.equal(got[:, :, half], rows(apart[0])[:, :, 0]) and torch.equal(got[:, :, 1 - half], rows(apart[1])[:, :, 0])
    if pad:
        assert all(bool((fused[c * bs + tk * 2 * d:(c + 1) * bs] == 9.0).all()) for c in range(prompts))


def test_cross_attention_without_tables():
    """No index: batch row b has prompt b; no lengths: all keys; no lse, no workspace."""
    q, kv, _, _ = cross_inputs("bf16", 3, 2, 2, 128, 40, 30, 3, [30, 30, 30], 13)
    got, _ = cross_call("bf16", q, kv, None, None, lse=False, workspace=False)
    want, _ = cross_call("bf16", q, kv, [0, 1, 2], [30, 30, 30])
    assert torch.equal(got, want)


@pytest.mark.parametrize("which", ["q", "kv"])
def test_cross_attention_rows_far_apart(which):
    """Rows 2^23 elements apart take the kernels whose offsets are 64 bits: within the tolerance of the others, whose rounding of
    P and dS they share or better."""
    batch, heads, dh, tq, tk = 1, 1, 128, 70, 67
    q, kv, _, dout = cross_inputs("bf16", batch, heads, heads, dh, tq, tk, 1, [tk], 20)
    want, lse = cross_call("bf16", q, kv, [0], [tk])
    far = 1 << 23
    room = torch.zeros(70 * far, dtype=torch.bfloat16, device="cuda")
    view = room.view(70, far)[:, :dh]
    sizes = (fb.BF16, batch, heads, heads, dh, tq, tk)
    qd, kd, vd, dd = q.cuda().view(tq, dh), kv[0, :, 0, 0].contiguous().cuda(), kv[0, :, 1, 0].contiguous().cuda(), dout.cuda()
    strides = {"q": (0, dh), "kv": (0, dh)}
    if which == "q":
        view[:tq] = qd
        qd, strides["q"] = view, (0, far)
    else:
        view[:tk] = kd
        other = torch.zeros(70 * far, dtype=torch.bfloat16, device="cuda").view(70, far)[:, :dh]
        other[:tk] = vd
        kd, vd, strides["kv"] = view, other, (0, far)
    out, ls = torch.empty(tq, dh, dtype=torch.bfloat16, device="cuda"), torch.empty(tq, device="cuda")
    fb.flashbon_op_cross_attention(*sizes, qd, *strides["q"], kd, vd, *strides["kv"], None, 1, None, out, 0, dh, lse=ls)
    exact, _ = branch.cross_attention(wide(q), wide(kv[:, :, 0]), wide(kv[:, :, 1]), [0], [tk])
    mass, _ = branch.cross_attention(wide(q), wide(kv[:, :, 0]), np.abs(wide(kv[:, :, 1])), [0], [tk])
    near(out, exact[0, :, 0], 2.0 ** -8 * np.abs(exact[0, :, 0]) + (2.0 ** -8 + 500 * E) * mass[0, :, 0], "out")
    ws = torch.empty(fb.flashbon_op_cross_attention_grad_workspace(*sizes, 1), dtype=torch.uint8, device="cuda")
    dq, dk, dv = torch.zeros_like(room).view(70, far)[:, :dh] if which == "q" else torch.zeros_like(out), None, None
    fb.flashbon_op_cross_attention_grad(*sizes, qd, *strides["q"], kd, vd, *strides["kv"], None, 1, None, out, 0, dh, ls, dd, dq, workspace=ws)
    tq_, _, _ = branch.cross_attention_grad(wide(q), wide(kv[:, :, 0]), wide(kv[:, :, 1]), wide(out).reshape(1, tq, 1, dh), wide(ls).reshape(1, 1, tq),
                                            wide(dout), [0], [tk])
    err = np.linalg.norm(wide(dq)[:tq] - tq_[0, :, 0]) / np.linalg.norm(tq_)
    assert err <= 2 * 2.0 ** -8, err          # two roundings of 2^-8 at most each, of independent signs


def test_cross_attention_values_of_tables_are_clamped():
    q, kv, _, _ = cross_inputs("bf16", 2, 2, 2, 64, 40, 30, 2, [30, 30], 14)
    got, _ = cross_call("bf16", q, kv, [-5, 99], [1000, -3])
    want, _ = cross_call("bf16", q, kv, [0, 1], [30, 0])
    assert torch.equal(got, want)


@pytest.mark.parametrize("dh,tq,tk", [(128, 1, 1000), (64, 3, 2000), (128, 100, 77), (32, 50, 40)])
def test_cross_attention_candidates_stand_alone(dh, tq, tk):
    q, kv, index, _ = cross_inputs("bf16", 6, 4, 2, dh, tq, tk, 2, [tk, tk - 9], 15)
    whole, lse = cross_call("bf16", q, kv, index, [tk, tk - 9])
    for b in (0, 5):
        one, l1 = cross_call("bf16", q[b:b + 1].contiguous(), kv, [index[b]], [tk, tk - 9])
        assert torch.equal(one[0], whole[b]) and torch.equal(l1[0], lse[b])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_cross_attention_large_scores(dtype):
    """Scores of some hundreds, rising along the keys, one row of equal keys: the running maximum moves at every tile."""
    q, kv, index, _ = cross_inputs(dtype, 1, 2, 2, 64, 20, 150, 1, [150], 16)
    kv[0, :, 0] = (kv[0, :, 0].float() * torch.linspace(0, 60, 150)[:, None, None]).to(kv.dtype)
    got, lse = cross_call(dtype, q, kv, index, [150])
    k, v = kv[:, :, 0], kv[:, :, 1]
    out, want = branch.cross_attention(wide(q), wide(k), wide(v), index, [150])
    rel = p_error(q, k, index, want)
    near(lse, want, rel + 8 * E * np.abs(want), "lse")
    mass, _ = branch.cross_attention(wide(q), wide(k), np.abs(wide(v)), index, [150])
    u = U[ACT[dtype]]
    near(got, out, u * np.abs(out) + (u + 2 * rel.transpose(0, 2, 1)[..., None] + 160 * E) * (1 + 2 * u) * mass, "out")


def test_cross_attention_strides():
    """Queries out of a fused buffer, the output into one: what lies between the rows is left as it was."""
    q, kv, index, _ = cross_inputs("bf16", 2, 2, 2, 64, 37, 50, 2, [50, 20], 17)
    want, _ = cross_call("bf16", q, kv, index, [50, 20])
    fused, target = torch.full((2, 40, 384), 3.0, dtype=torch.bfloat16, device="cuda"), torch.full((2, 41, 256), 5.0, dtype=torch.bfloat16, device="cuda")
    fused[:, :37, 128:256] = q.cuda().flatten(2)
    kvd = kv.cuda()
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device="cuda")  # noqa: E731
    fb.flashbon_op_cross_attention(fb.BF16, 2, 2, 2, 64, 37, 50, fused[:, :, 128:], 40 * 384, 384, kvd[:, :, 0], kvd[:, :, 1], 50 * 256, 256,
                                   i32(index), 2, i32([50, 20]), target[:, :, 64:], 41 * 256, 256)
    assert torch.equal(target[:, :37, 64:192], want.flatten(2))
    target[:, :37, 64:192] = 5.0
    assert bool((target == 5.0).all())


# ------------------------------------------------------------------------------------------------------- adapters
#            M    N    K   rank count per
ADAPTERS = [(1, 8, 8, 8, 1, 1), (7, 24, 40, 8, 3, 2), (64, 136, 264, 32, 5, 1), (65, 256, 64, 16, 2, 33), (200, 520, 328, 24, 4, 50),
            (130, 64, 1032, 64, 2, 130), (300, 264, 96, 128, 3, 70), (33, 72, 56, 40, 40, 1), (1000, 128, 256, 32, 1, 1000),
            (517, 392, 136, 104, 2, 17)]


def adapter_inputs(dtype, m, n, k, rank, count, per, seed):
    g, act = gen(seed), ACT[dtype]
    groups = -(-m // per)
    index = torch.tensor([(5 * i + 1) % (count + 1) - (i % 7 == 6) for i in range(groups)], dtype=torch.int32)   # count and -1: none
    if count == 1:
        index.zero_()
    return (normal(g, m, k, dtype=act), normal(g, count, rank, k, dtype=act, std=k ** -0.5), normal(g, count, n, rank, dtype=act, std=0.3),
            torch.exp(normal(g, count)), index, g)


EPIS = {"store": fb.EPI_STORE, "f32": fb.EPI_STORE_F32, "residual": fb.EPI_RESIDUAL}


@pytest.mark.parametrize("dtype,epi", [("bf16", "store"), ("bf16", "f32"), ("bf16", "residual"), ("fp32", "store"), ("fp32", "residual")])
@pytest.mark.parametrize("shape", ADAPTERS, ids=str)
def test_adapters(dtype, epi, shape):
    m, n, k, rank, count, per = shape
    x, down, up, s, index, g = adapter_inputs(dtype, *shape, 21)
    outs = ACT[dtype] if epi == "store" else torch.float32
    base, gate = normal(g, m, n, dtype=outs), normal(g, n) if epi == "residual" else None
    out, u = torch.empty(m, n, dtype=outs, device="cuda"), torch.empty(m, rank, device="cuda")
    args = (CODE[dtype], m, n, k, rank, count, x.cuda(), down.cuda(), up.cuda(), s.cuda(), index.cuda(), per, EPIS[epi])
    fb.flashbon_op_adapters(*args, base.cuda(), out, u, gate=cuda(gate))
    want, wu = branch.adapters(wide(x), wide(down), wide(up), s, index, per, wide(base), wide(gate))
    ab = [np.abs(wide(t)) for t in (x, down, up)]
    ag = None if gate is None else np.abs(wide(gate))
    _, mu = branch.adapters(*ab, s, index, per)                     # sum |x| |down|
    eu = (k + 8) * E * mu
    near(u, wu, eu, "u")
    # u is off by eu; next to bf16 weights it goes in parts, 2^-16 of it lost where out is bf16, 2^-24 where it is fp32
    lost = 2.0 ** -16 if outs is torch.bfloat16 else 2 * E
    terms = np.zeros((m, n))
    for a, rows in branch._groups(m, per, index, count):
        terms[rows] = float(s[a]) * (1.0 if ag is None else ag) * ((eu[rows] + np.abs(wu[rows]) * (lost + (4 * rank + 8) * E)) @ ab[2][a].T)
    near(out, want, U[outs] * np.abs(want) + 2 * E * np.abs(wide(base)) + 1.01 * terms, "out")
    # onto the projection's output in place, and without one
    inplace, only, zero = base.cuda(), torch.empty_like(out), torch.empty_like(out)
    fb.flashbon_op_adapters(*args, inplace, inplace, u, gate=cuda(gate))
    assert torch.equal(inplace, out)
    fb.flashbon_op_adapters(*args, None, only, u, gate=cuda(gate))
    fb.flashbon_op_adapters(*args, torch.zeros_like(out), zero, u, gate=cuda(gate))
    assert torch.equal(only, zero)


@pytest.mark.parametrize("dtype,epi", [("bf16", "store"), ("bf16", "f32"), ("fp32", "store")])
@pytest.mark.parametrize("shape", ADAPTERS, ids=str)
def test_adapters_grad(dtype, epi, shape):
    m, n, k, rank, count, per = shape
    x, down, up, s, index, g = adapter_inputs(dtype, *shape, 22)
    outs = ACT[dtype] if epi == "store" else torch.float32
    base, dy = normal(g, m, k, dtype=outs), normal(g, m, n, dtype=ACT[dtype])
    u = torch.tensor(branch.adapters(wide(x), wide(down), wide(up), s, index, per)[1], dtype=torch.float32)
    dx = torch.empty(m, k, dtype=outs, device="cuda")
    dd, du = torch.full(down.shape, 7.0, device="cuda"), torch.full(up.shape, 7.0, device="cuda")
    sizes = (CODE[dtype], m, n, k, rank, count)
    ws = torch.full((fb.flashbon_op_adapters_grad_workspace(*sizes, per),), 255, dtype=torch.uint8, device="cuda")
    args = (*sizes, x.cuda(), down.cuda(), up.cuda(), s.cuda(), index.cuda(), per, u.cuda(), dy.cuda(), EPIS[epi])
    fb.flashbon_op_adapters_grad(*args, base.cuda(), dx, dd, du, workspace=ws)
    tx, td, tu = branch.adapters_grad(wide(x), wide(down), wide(up), wide(u), wide(dy), s, index, per, wide(base))
    ax, ad, au, amid, ay = (np.abs(wide(t)) for t in (x, down, up, u, dy))
    lost = 2.0 ** -16 if outs is torch.bfloat16 else 2 * E
    ex, ed, eu = np.zeros((m, k)), np.zeros(down.shape), np.zeros(up.shape)
    for a, rows in branch._groups(m, per, index, count):
        sc = float(s[a])
        mid = sc * (ay[rows] @ au[a])                               # sum |dy| |up|: du is off by (n + 8) E of it
        true = sc * np.abs(wide(dy)[rows] @ wide(up)[a])
        ex[rows] = (mid * (n + 8) * E + true * (lost + (4 * rank + 8) * E)) @ ad[a]
        ed[a] += (mid * (n + 8) * E + true * (m * 3 + 16) * E).T @ ax[rows]
        eu[a] += sc * (ay[rows].T @ amid[rows]) * (m * 3 + 16) * E
    near(dx, tx, U[outs] * np.abs(tx) + 2 * E * np.abs(wide(base)) + 1.01 * ex, "dx")
    near(dd, td, E * np.abs(td) + 1.01 * ed, "d_down")
    near(du, tu, E * np.abs(tu) + 1.01 * eu, "d_up")
    inplace, parts = base.cuda(), (torch.empty_like(dd), torch.empty_like(du))
    fb.flashbon_op_adapters_grad(*args, inplace, inplace, workspace=ws)
    fb.flashbon_op_adapters_grad(*args, None, None, parts[0], workspace=ws)
    fb.flashbon_op_adapters_grad(*args, None, None, None, parts[1], workspace=ws)
    assert torch.equal(inplace, dx) and torch.equal(parts[0], dd) and torch.equal(parts[1], du)


@pytest.mark.parametrize("dtype,epi", [("bf16", "store"), ("bf16", "f32"), ("fp32", "store")])
@pytest.mark.parametrize("shape", [(8300, 136, 72, 128, 3, 997), (8250, 1160, 1096, 104, 2, 1031), (8300, 264, 1032, 64, 3, 8300)], ids=str)
def test_adapters_of_many_rows(dtype, epi, shape):
    """Enough rows that a workgroup takes 32 of them."""
    test_adapters(dtype, epi, shape)
    test_adapters_grad(dtype, epi, shape)


def test_adapters_without_tables():
    x, down, up, _, _, _ = adapter_inputs("bf16", 50, 64, 48, 16, 1, 50, 23)
    a, b = (torch.empty(50, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    u = torch.empty(50, 16, device="cuda")
    args = (fb.BF16, 50, 64, 48, 16, 1, x.cuda(), down.cuda(), up.cuda())
    fb.flashbon_op_adapters(*args, None, None, 7, fb.EPI_STORE, None, a, u)
    fb.flashbon_op_adapters(*args, torch.ones(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), 50, fb.EPI_STORE, None, b, u)
    assert torch.equal(a, b)


def test_adapters_rows_stand_alone():
    """A row's bits do not depend on the rows beside it, nor on how they are grouped."""
    m, n, k, rank = 150, 264, 520, 32
    x, down, up, s, _, g = adapter_inputs("bf16", m, n, k, rank, 1, m, 24)
    base = normal(g, m, n, dtype=torch.bfloat16).cuda()
    results = []
    for per in (m, 64, 16, 1):
        out, u = torch.empty_like(base), torch.empty(m, rank, device="cuda")
        fb.flashbon_op_adapters(fb.BF16, m, n, k, rank, 1, x.cuda(), down.cuda(), up.cuda(), s.cuda(), None, per, fb.EPI_STORE, base, out, u)
        results.append((out, u))
    for out, u in results[1:]:
        assert torch.equal(out, results[0][0]) and torch.equal(u, results[0][1])


# --------------------------------------------------------------------------------------- together, and in a graph
class Branch:
    """h + gate W_o' attention(W_q' LN(h), kv) with adapters beside W_q and W_o, forward and backward, through the library."""

    def __init__(self, seed, batch=3, tokens=50, heads=2, dh=64, text=40, rank=16):
        g, self.bf = gen(seed), torch.bfloat16
        d = self.d = heads * dh
        self.batch, self.tokens, self.heads, self.dh, self.text, self.rank, self.m = batch, tokens, heads, dh, text, rank, batch * tokens
        self.h = normal(g, self.m, d)
        self.w, self.b = normal(g, batch, d, std=0.3), normal(g, batch, d, std=0.3)
        self.wq, self.wo = normal(g, d, d, dtype=self.bf, std=d ** -0.5), normal(g, d, d, dtype=self.bf, std=d ** -0.5)
        self.kv = normal(g, 2, text, 2 * d, dtype=self.bf)
        self.lengths, self.prompts = torch.tensor([text, 13], dtype=torch.int32), torch.tensor([1, 0, 1], dtype=torch.int32)
        self.aq, self.bq = normal(g, 2, rank, d, dtype=self.bf, std=d ** -0.5), normal(g, 2, d, rank, dtype=self.bf, std=rank ** -0.5)
        self.ao, self.bo = normal(g, 2, rank, d, dtype=self.bf, std=d ** -0.5), normal(g, 2, d, rank, dtype=self.bf, std=rank ** -0.5)
        self.scales, self.index = torch.tensor([0.5, 2.0]), torch.tensor([1, -1, 0], dtype=torch.int32)
        self.gate, self.dh_out = normal(g, d), normal(g, self.m, d)

    def device(self):
        for name, t in list(vars(self).items()):
            if torch.is_tensor(t):
                setattr(self, name, t.cuda())
        e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        m, d, r, bf = self.m, self.d, self.rank, self.bf
        self.wqt, self.wot = self.wq.t().contiguous(), self.wo.t().contiguous()
        self.c, self.q, self.att, self.uq, self.uo = e(m, d, dtype=bf), e(m, d, dtype=bf), e(m, d, dtype=bf), e(m, r), e(m, r)
        self.mean, self.rstd, self.lse, self.y = e(m), e(m), e(self.batch, self.heads, self.tokens), e(m, d)
        self.dy, self.datt, self.dq, self.dc = e(m, d, dtype=bf), e(m, d, dtype=bf), e(m, d, dtype=bf), e(m, d, dtype=bf)
        self.dx, self.dkv, self.dw, self.db = e(m, d), e(2, self.text, 2 * d, dtype=bf), e(self.batch, d), e(self.batch, d)
        self.daq, self.dbq, self.dao, self.dbo = e(2, r, d), e(2, d, r), e(2, r, d), e(2, d, r)
        self.sizes = (fb.BF16, self.batch, self.heads, self.heads, self.dh, self.tokens, self.text)
        self.ad = (fb.BF16, m, d, d, r, 2)
        need = max(fb.flashbon_op_cross_attention_grad_workspace(*self.sizes, 2), fb.flashbon_op_adapters_grad_workspace(*self.ad, self.tokens),
                   fb.flashbon_op_layer_norm_grad_workspace(m, d, self.tokens), fb.flashbon_op_cross_attention_workspace(*self.sizes))
        self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        return self

    def step(self):
        m, d, t = self.m, self.d, self.tokens
        qs, ks, k, v = (t * d, d), (self.text * 2 * d, 2 * d), self.kv[:, :, :d], self.kv[:, :, d:]
        fb.flashbon_op_layer_norm(fb.BF16, m, d, 1e-6, self.h, self.c, weight=self.w, bias=self.b, rows_per_group=t, modulated=True,
                                  mean=self.mean, rstd=self.rstd)
        fb.flashbon_op_linear(fb.BF16, m, d, d, self.c, self.wq, None, fb.EPI_STORE, self.q)
        fb.flashbon_op_adapters(*self.ad, self.c, self.aq, self.bq, self.scales, self.index, t, fb.EPI_STORE, self.q, self.q, self.uq)
        fb.flashbon_op_cross_attention(*self.sizes, self.q, *qs, k, v, *ks, self.prompts, 2, self.lengths, self.att, *qs, lse=self.lse, workspace=self.ws)
        fb.flashbon_op_linear_residual(fb.BF16, m, d, d, self.att, self.wo, None, self.gate, self.h, self.y)
        fb.flashbon_op_adapters(*self.ad, self.att, self.ao, self.bo, self.scales, self.index, t, fb.EPI_RESIDUAL, self.y, self.y, self.uo, gate=self.gate)
        # backward
        self.dy.copy_(self.dh_out * self.gate)
        fb.flashbon_op_linear(fb.BF16, m, d, d, self.dy, self.wot, None, fb.EPI_STORE, self.datt)
        fb.flashbon_op_adapters_grad(*self.ad, self.att, self.ao, self.bo, self.scales, self.index, t, self.uo, self.dy, fb.EPI_STORE, self.datt,
                                     self.datt, self.dao, self.dbo, workspace=self.ws)
        fb.flashbon_op_cross_attention_grad(*self.sizes, self.q, *qs, k, v, *ks, self.prompts, 2, self.lengths, self.att, *qs, self.lse, self.datt,
                                            self.dq, self.dkv[:, :, :d], self.dkv[:, :, d:], workspace=self.ws)
        fb.flashbon_op_linear(fb.BF16, m, d, d, self.dq, self.wqt, None, fb.EPI_STORE, self.dc)
        fb.flashbon_op_adapters_grad(*self.ad, self.c, self.aq, self.bq, self.scales, self.index, t, self.uq, self.dq, fb.EPI_STORE, self.dc,
                                     self.dc, self.daq, self.dbq, workspace=self.ws)
        fb.flashbon_op_layer_norm_grad(fb.BF16, m, d, self.h, self.mean, self.rstd, self.dc, self.dx, weight=self.w, rows_per_group=t, modulated=True,
                                       residual=self.dh_out, dweight=self.dw, dbias=self.db, workspace=self.ws)

    RESULTS = ("y", "dx", "dw", "db", "daq", "dbq", "dao", "dbo", "dkv")

    def results(self):
        return {name: getattr(self, name).clone() for name in self.RESULTS}


def reference_branch(b):
    """The same branch in 64 bits, its gradients by torch's."""
    f = {n: t.double() for n, t in vars(b).items() if torch.is_tensor(t) and t.is_floating_point()}
    for n in ("h", "w", "b", "kv", "aq", "bq", "ao", "bo"):
        f[n].requires_grad_()
    rows = torch.arange(b.m) // b.tokens
    c = torch.nn.functional.layer_norm(f["h"], (b.d,), eps=1e-6) * (1 + f["w"][rows]) + f["b"][rows]
    has = (b.index[rows] >= 0).double()[:, None] * f["scales"][b.index[rows].clamp_min(0).long()][:, None]
    a = b.index[rows].clamp_min(0).long()

    def adapted(x, w, down, up):
        low = (down[a] @ x[:, :, None]) * has[:, :, None]
        return x @ w.t() + (up[a] @ low)[:, :, 0]
    q = adapted(c, f["wq"], f["aq"], f["bq"]).view(b.batch, b.tokens, b.heads, b.dh)
    att = []
    for i in range(b.batch):
        p = int(b.prompts[i])
        n = int(b.lengths[p])
        k, v = (t.reshape(n, b.heads, b.dh) for t in f["kv"][p, :n].chunk(2, 1))
        s = torch.softmax(torch.einsum("qhd,khd->hqk", q[i], k) / b.dh ** 0.5, 2)
        att.append(torch.einsum("hqk,khd->qhd", s, v).reshape(b.tokens, b.d))
    y = f["h"] + f["gate"] * adapted(torch.cat(att), f["wo"], f["ao"], f["bo"])
    (y * f["dh_out"]).sum().backward()
    return {"y": y.detach(), "dx": f["h"].grad, "dw": f["w"].grad, "db": f["b"].grad, "daq": f["aq"].grad, "dbq": f["bq"].grad,
            "dao": f["ao"].grad, "dbo": f["bo"].grad, "dkv": f["kv"].grad}


def test_branch_together():
    """The operators in turn as a training step runs them, against the whole branch in 64 bits.

    Up to nine activations in a row are rounded to bf16 (c, q twice, P, att, dy, datt twice, dS, dq, dc twice), each by a
    random 2^-8 / sqrt(12) or less of itself: some 4e-3 in the root mean square of a result; three times that is allowed."""
    b = Branch(31)
    want = reference_branch(b)
    b.device().step()
    for name, got in b.results().items():
        e = float((got.double().cpu() - want[name]).norm() / want[name].norm())
        assert e <= 1.2e-2, (name, e)
    assert not b.dkv[1, 13:].any()


def test_branch_in_a_graph():
    """Two captured steps that share a workspace, replayed in turn with eager steps between: always the same bits."""
    a, b = Branch(32).device(), Branch(33).device()
    b.ws = a.ws
    a.step()
    b.step()
    want = [a.results(), b.results()]
    torch.cuda.synchronize()
    graphs = []
    for x in (a, b):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            x.step()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.step()
        graphs.append(g)
    for _ in range(4):
        for x, g, w in zip((a, b), graphs, want):
            for name in x.RESULTS:
                getattr(x, name).zero_()
            g.replay()
            torch.cuda.synchronize()
            for name, t in x.results().items():
                assert torch.equal(t, w[name]), name
        a.step()


def test_branch_on_another_stream():
    a = Branch(34).device()
    a.step()
    want = a.results()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for name in a.RESULTS:
            getattr(a, name).zero_()
        a.step()
    side.synchronize()
    for name, t in a.results().items():
        assert torch.equal(t, want[name]), name


# ------------------------------------------------------------------------------------- offsets past 32 bits
def room(elements, dtype=torch.bfloat16):
    return torch.zeros(elements, dtype=dtype, device="cuda")


def test_layer_norm_past_32_bits():
    """The last rows of 2^31 elements and more have the bits that they have alone."""
    d, tail = 4104, 3
    m = (1 << 31) // d + 5
    g = gen(41)
    rows, dy, w = normal(g, tail, d).cuda(), normal(g, tail, d, dtype=torch.bfloat16).cuda(), normal(g, 1, d).cuda()
    x, out = room(m * d, torch.float32).view(m, d), room(m * d).view(m, d)
    x[-tail:] = rows
    mean, rstd = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    fb.flashbon_op_layer_norm(fb.BF16, m, d, 1e-6, x, out, weight=w, mean=mean, rstd=rstd)
    alone, mu, rs = torch.empty(tail, d, dtype=torch.bfloat16, device="cuda"), torch.empty(tail, device="cuda"), torch.empty(tail, device="cuda")
    fb.flashbon_op_layer_norm(fb.BF16, tail, d, 1e-6, rows, alone, weight=w, mean=mu, rstd=rs)
    assert torch.equal(out[-tail:], alone) and torch.equal(mean[-tail:], mu) and torch.equal(rstd[-tail:], rs)
    out.zero_()
    out[-tail:] = dy
    dx, one = room(m * d, torch.float32).view(m, d), torch.empty(tail, d, device="cuda")
    fb.flashbon_op_layer_norm_grad(fb.BF16, m, d, x, mean, rstd, out, dx, weight=w)
    fb.flashbon_op_layer_norm_grad(fb.BF16, tail, d, rows, mu, rs, dy, one, weight=w)
    assert torch.equal(dx[-tail:], one) and not dx[:-tail].any()


@pytest.mark.parametrize("dh,tq,tk", [(128, 70, 70), (128, 2, 300), (32, 70, 20)])
def test_cross_attention_past_32_bits(dh, tq, tk):
    """Batch rows and prompts 2^31 elements apart: the bits of a call on dense buffers."""
    q, kv, _, dout = cross_inputs("bf16", 2, 1, 1, dh, tq, tk, 2, [tk, tk - 1], 42)
    kv = clean(kv, [tk, tk - 1])
    far = (1 << 31) + 64
    sizes, i32 = (fb.BF16, 2, 1, 1, dh, tq, tk), lambda t: torch.tensor(t, dtype=torch.int32, device="cuda")  # noqa: E731
    index, lengths = i32([1, 0]), i32([tk, tk - 1])
    dense = [t.contiguous().cuda() for t in (q[:, :, 0], kv[:, :, 0, 0], kv[:, :, 1, 0], dout[:, :, 0])]

    def spread(t):
        n, rows, _ = t.shape
        view = room(far + rows * dh).as_strided((n, rows, dh), (far, dh, 1))
        view.copy_(t)
        return view

    def run(tensors, q_bs, kv_bs):
        qq, kk, vv, dd = tensors
        # out, dq, dk and dv like the inputs whose strides they have
        out, dq, dk, dv = (spread(torch.zeros(t.shape, dtype=t.dtype, device="cuda")) if q_bs > 1 << 20 else torch.zeros_like(t) for t in (qq, qq, kk, vv))
        lse, ws = torch.empty(2, 1, tq, device="cuda"), torch.empty(fb.flashbon_op_cross_attention_workspace(*sizes), dtype=torch.uint8, device="cuda")
        fb.flashbon_op_cross_attention(*sizes, qq, q_bs, dh, kk, vv, kv_bs, dh, index, 2, lengths, out, q_bs, dh, lse=lse, workspace=ws)
        ws = torch.empty(fb.flashbon_op_cross_attention_grad_workspace(*sizes, 2), dtype=torch.uint8, device="cuda")
        fb.flashbon_op_cross_attention_grad(*sizes, qq, q_bs, dh, kk, vv, kv_bs, dh, index, 2, lengths, out, q_bs, dh, lse, dd, dq, dk, dv, workspace=ws)
        return [t.clone() for t in (out, lse, dq, dk, dv)]
    want = run(dense, tq * dh, tk * dh)
    for a, b in zip(run([spread(t) for t in dense], far, far), want):
        assert torch.equal(a.contiguous(), b)


def test_adapters_past_32_bits():
    """The last rows of outputs (and of inputs) of 2^31 elements have the bits that they have alone."""
    wide_, rank, tail = 1032, 8, 5
    m = (1 << 31) // wide_ + 20
    g = gen(43)
    down, up = normal(g, 1, rank, 8, dtype=torch.bfloat16).cuda(), normal(g, 1, wide_, rank, dtype=torch.bfloat16).cuda()
    x, base = room(m * 8).view(m, 8), room(m * wide_).view(m, wide_)
    x[-tail:], base[-tail:] = normal(g, tail, 8, dtype=torch.bfloat16).cuda(), normal(g, tail, wide_, dtype=torch.bfloat16).cuda()
    last, u, mid = base[-tail:].clone(), torch.empty(m, rank, device="cuda"), torch.empty(tail, rank, device="cuda")
    alone = torch.empty_like(last)
    fb.flashbon_op_adapters(fb.BF16, tail, wide_, 8, rank, 1, x[-tail:].contiguous(), down, up, None, None, tail, fb.EPI_STORE, last, alone, mid)
    fb.flashbon_op_adapters(fb.BF16, m, wide_, 8, rank, 1, x, down, up, None, None, 1000, fb.EPI_STORE, base, base, u)
    assert torch.equal(base[-tail:], alone) and torch.equal(u[-tail:], mid) and not base[:-tail].any()
    # the wide side as the input: dx of x [m][1032], dy [m][8]
    down, up = up.transpose(1, 2).contiguous(), normal(g, 1, 8, rank, dtype=torch.bfloat16).cuda()
    dd, du = torch.empty(1, rank, wide_, device="cuda"), torch.empty(1, 8, rank, device="cuda")
    sizes = (m, 8, wide_, rank, 1)
    ws = torch.empty(fb.flashbon_op_adapters_grad_workspace(fb.BF16, *sizes, 1000), dtype=torch.uint8, device="cuda")
    dx = room(m * wide_).view(m, wide_)
    fb.flashbon_op_adapters_grad(fb.BF16, *sizes, base, down, up, None, None, 1000, u, x, fb.EPI_STORE, None, dx, dd, du, workspace=ws)
    one, d1, u1 = torch.empty_like(alone), torch.empty_like(dd), torch.empty_like(du)
    sizes = (tail, 8, wide_, rank, 1)
    fb.flashbon_op_adapters_grad(fb.BF16, *sizes, alone, down, up, None, None, tail, mid, x[-tail:].contiguous(), fb.EPI_STORE, None, one, d1, u1,
                                 workspace=ws)
    assert torch.equal(dx[-tail:], one) and not dx[:-tail].any()
    # every other row is zero: the sums are those of the last rows, in another order of
    # five terms, whose magnitudes stay below sixty-four times the largest sum
    for a, b in ((dd, d1), (du, u1)):
        assert float((a - b).abs().max()) <= 5 * 64 * E * float(b.abs().max())
