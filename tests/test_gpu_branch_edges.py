"""The cross-attention branch's kernels at the ends of their ranges, against 64 bits.

Tolerances count roundings as in test_gpu_branch: E is half a step of fp32, U[t] of the type t.
"""
import threading

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


def norm_grad_case(x, dtype, per, modulated, eps=1e-6):
    """The gradient of rows x from statistics saved in fp32, against that of the mean before its rounding."""
    m, d = x.shape
    groups, g = -(-m // per), gen(55)
    w, dy, res = normal(g, groups, d), normal(g, m, d, dtype=ACT[dtype]), normal(g, m, d)
    _, mu, rs = branch.layer_norm(x, w, None, per, modulated, eps)
    mean, rstd = torch.tensor(mu, dtype=torch.float32), torch.tensor(rs, dtype=torch.float32)
    dx, dw, db = torch.empty(m, d, device="cuda"), torch.empty(groups, d, device="cuda"), torch.empty(groups, d, device="cuda")
    ws = torch.full((fb.flashbon_op_layer_norm_grad_workspace(m, d, per),), 255, dtype=torch.uint8, device="cuda")
    fb.flashbon_op_layer_norm_grad(CODE[dtype], m, d, cuda(x), cuda(mean), cuda(rstd), cuda(dy), dx, weight=cuda(w),
                                   rows_per_group=per, modulated=modulated, residual=cuda(res), dweight=dw, dbias=db, workspace=ws)
    tx, tw, tb = branch.layer_norm_grad(x, w, per, modulated, mu, wide(rstd), dy.float(), res)
    xh = np.abs((wide(x) - mu[:, None]) * wide(rstd)[:, None])
    f = np.abs(wide(w)[np.arange(m) // per] + (1 if modulated else 0))
    gr, ay = np.abs(wide(dy)) * f, np.abs(wide(dy))
    n = 24 + 8 + 4           # sums along a row, as in test_layer_norm_grad
    mean_g, mean_gx = gr.mean(1, keepdims=True), (gr * xh).mean(1, keepdims=True)
    near(dx, tx, E * (2 * np.abs(tx) + wide(rstd)[:, None] * (6 * gr + (n + 4) * mean_g + xh * (n + 8) * mean_gx)), "dx")
    rows = [slice(i * per, min(m, (i + 1) * per)) for i in range(groups)]
    n = 16 + 4 + 4
    near(dw, tw, n * E * np.stack([(ay * xh)[r].sum(0) for r in rows]), "dweight")
    near(db, tb, n * E * np.stack([ay[r].sum(0) for r in rows]), "dbias")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [2, 40, 701, 2100, 6143])
def test_layer_norm_grad_at_the_ends_of_the_range(dtype, d):
    x = rows_at_the_ends(d)
    norm_grad_case(x[:3], dtype, 3, False)
    norm_grad_case(torch.cat([x[1:2], x[:1]]), dtype, 1, True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 701, 1536, 2100, 5120])
def test_layer_norm_grad_of_rows_far_from_zero(dtype, d):
    """A mean of 10^4 deviations, saved in fp32, is off by 2^-11 of one, which every element of the row would share."""
    x = normal(gen(56), 40, d, std=0.5) + 5000.0 + torch.arange(40)[:, None] / 7.0
    norm_grad_case(x, dtype, 40, False)
    norm_grad_case(x, dtype, 7, True)


# ------------------------------------------------------------------------------------------------ cross-attention
#          heads kv dh  tq   tk  the keys before which all count for nothing
NOTHING = [(2, 1, 16, 70, 90, 70), (2, 2, 32, 3, 40, 33), (2, 2, 64, 100, 200, 130), (4, 2, 128, 70, 70, 64), (2, 2, 128, 129, 200, 129),
           (2, 1, 128, 70, 700, 640), (1, 1, 128, 2, 900, 512)]


def inputs_of_dead_keys(dtype, shape, seed):
    """Three prompts whose first keys, all keys and every other key have scores of -infinity."""
    heads, kvh, dh, tq, tk, first = shape
    lengths = [tk, tk, tk - 1]
    q, kv, index, dout = base.cross_inputs(dtype, 3, heads, kvh, dh, tq, tk, 3, lengths, seed)
    q[..., 0] = q[..., 0].abs() + 0.25
    kv[0, :first, 0, :, 0] = -float("inf")
    kv[1, :, 0, :, 0] = -float("inf")
    kv[2, 3::2, 0, :, 0] = -float("inf")
    return q, kv, index, lengths, dout


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", NOTHING, ids=str)
def test_cross_attention_of_keys_that_count_for_nothing(dtype, shape):
    """Keys whose scores are -infinity have probability 0, be they whole tiles, and rows of no other keys are those of an empty
    prompt, on every path."""
    tk = shape[4]
    q, kv, index, lengths, _ = inputs_of_dead_keys(dtype, shape, 57)
    got, lse = base.cross_call(dtype, q, kv, index, lengths)
    kv = base.clean(kv, lengths)
    k, v = kv[:, :, 0], kv[:, :, 1]
    out, want = branch.cross_attention(wide(q), wide(k), wide(v), index, lengths)
    row = index.index(1)
    assert not out[row].any() and np.isneginf(want[row]).all() and np.isfinite(want[index.index(0)]).all()
    finite = torch.where(torch.isinf(k), torch.zeros_like(k), k)
    rel = base.p_error(q, finite, index, want)
    near(lse, want, rel + 8 * E * np.where(np.isfinite(want), np.abs(want), 0), "lse")
    mass, _ = branch.cross_attention(wide(q), wide(k), np.abs(wide(v)), index, lengths)
    u = U[ACT[dtype]]
    near(got, out, u * np.abs(out) + (u + 2 * rel.transpose(0, 2, 1)[..., None] + (tk + 8) * E) * (1 + 2 * u) * mass, "out")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", NOTHING, ids=str)
def test_cross_attention_grad_of_keys_that_count_for_nothing(dtype, shape):
    """Such keys take no gradient, whatever the number of queries: rows past the last query meet them with zeros."""
    heads, kvh, dh, tq, tk, first = shape
    q, kv, index, lengths, dout = inputs_of_dead_keys(dtype, shape, 58)
    out, lse = base.cross_call(dtype, q, kv, index, lengths)
    kv = base.clean(kv, lengths)
    sizes, qs, ks = (CODE[dtype], 3, heads, kvh, dh, tq, tk), (tq * heads * dh, heads * dh), (tk * 2 * kvh * dh, 2 * kvh * dh)
    dkv, kvd = torch.full_like(kv, 9.0).cuda(), kv.cuda()
    ws = torch.empty(fb.flashbon_op_cross_attention_grad_workspace(*sizes, 3), dtype=torch.uint8, device="cuda")
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device="cuda")  # noqa: E731
    fb.flashbon_op_cross_attention_grad(*sizes, q.cuda(), *qs, kvd[:, :, 0], kvd[:, :, 1], *ks, i32(index), 3, i32(lengths), out, *qs, lse,
                                        dout.cuda(), None, dkv[:, :, 0], dkv[:, :, 1], workspace=ws)
    assert not dkv[0, :first].any() and not dkv[1].any() and not dkv[2, 3::2].any()
    assert bool(torch.isfinite(dkv).all()) and bool(dkv[0, first:].any()) and bool(dkv[2, :3].any())
    # the keys that count have the gradient of a prompt of them alone
    some = torch.arange(tk) % 2 == 0
    some[:3], some[tk - 1:] = True, False
    for c, rows in ((0, torch.arange(tk) >= first), (2, some)):
        b = index.index(c)
        k1, v1 = (kv[c:c + 1, rows, i] for i in (0, 1))
        _, tk_, tv = branch.cross_attention_grad(wide(q[b:b + 1]), wide(k1), wide(v1), wide(out[b:b + 1]), wide(lse[b:b + 1]), wide(dout[b:b + 1]))
        for got, want in ((dkv[c, rows.cuda(), 0], tk_[0]), (dkv[c, rows.cuda(), 1], tv[0])):
            # P and dS rounded once and results once, and fp32's sums of order 10^3 terms
            assert np.linalg.norm(wide(got) - want) <= (2 * U[ACT[dtype]] + 1000 * E) * np.linalg.norm(want)


# ------------------------------------------------------------------------------- sums over many tiles, large scores
def equal_keys(dtype, dh, tq, tk, score, seed):
    """Queries of ones and keys whose scores (before the scale) are all `score`, exactly; values of order one."""
    q = torch.zeros(1, tq, 2, dh, dtype=ACT[dtype])
    q[..., 0] = 1.0
    kv = torch.zeros(1, tk, 2, 1, dh, dtype=ACT[dtype])
    kv[:, :, 0, :, 0] = score
    kv[:, :, 1] = normal(gen(seed), 1, tk, 1, dh, dtype=ACT[dtype])
    return q, kv


PATHS = [(16, 70, 4096), (64, 100, 4096), (128, 70, 4096), (128, 100, 300), (128, 2, 4096), (32, 3, 8000)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dh,tq,tk", PATHS)
@pytest.mark.parametrize("workspace", [False, True])
def test_cross_attention_weighs_all_tiles_alike(dtype, dh, tq, tk, workspace):
    """Values of 1 before the middle and of -1 behind it, under equal scores: their sums are whole multiples of one probability,
    exact in fp32, and cancel."""
    for score in (37.0, 117.0, 1000.0):
        q, kv = equal_keys(dtype, dh, tq, tk, score, 73)
        kv[:, :tk // 2, 1], kv[:, tk // 2:, 1] = 1.0, -1.0
        got, lse = base.cross_call(dtype, q, kv, [0], [tk], workspace=workspace)
        want = score / np.sqrt(dh) + np.log(tk)
        near(lse, np.full(lse.shape, want), 8 * E * want, "lse")
        assert float(got.abs().max()) <= 8 * E       # ranges of keys are joined with factors of one rounding each


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dh,tq,tk", PATHS)
@pytest.mark.parametrize("score", [-1e37, -1e12, 1e10, 1e37, 2.0 ** 31, -2.0 ** 30, 2.0 ** 24, 3e9, -1.1e9, 1.7e7, -3e6])
def test_cross_attention_of_large_scores(dtype, dh, tq, tk, score):
    """Scores of any finite size: equal ones have equal probabilities, lower ones none."""
    u = U[ACT[dtype]]
    q, kv = equal_keys(dtype, dh, tq, tk, score, 74)
    score = float(kv[0, 0, 0, 0, 0])
    got, lse = base.cross_call(dtype, q, kv, [0], [tk])
    v = wide(kv[0, :, 1, 0])
    want = score / np.sqrt(dh) + np.log(tk)
    near(lse, np.full(lse.shape, want), 8 * E * abs(want), "lse")
    tol = u * np.abs(v.mean(0)) + (2 * u + (tk + 8) * E) * np.abs(v).mean(0)
    near(got, np.broadcast_to(v.mean(0), got.shape), tol, "out")
    # most keys far below, in whole tiles and between the others
    low = score * 1.5 if score < 0 else score * 0.5
    kv[0, :tk // 2, 0, 0, 0] = low
    kv[0, tk // 2::3, 0, 0, 0] = low
    got, lse = base.cross_call(dtype, q, kv, [0], [tk])
    on = wide(kv[0, :, 0, 0, 0]) == score
    want, v = score / np.sqrt(dh) + np.log(on.sum()), v[on]
    near(lse, np.full(lse.shape, want), 8 * E * abs(want), "lse")
    near(got, np.broadcast_to(v.mean(0), got.shape), u * np.abs(v.mean(0)) + (2 * u + (tk + 8) * E) * np.abs(v).mean(0), "out")
    # and one ordinary key above them all where they are negative
    if score < 0:
        kv[0, tk - 1, 0, 0, 0] = 1.0
        got, lse = base.cross_call(dtype, q, kv, [0], [tk])
        near(lse, np.full(lse.shape, 1 / np.sqrt(dh)), 8 * E, "lse")
        near(got, np.broadcast_to(wide(kv[0, tk - 1, 1, 0]), got.shape), 4 * E, "out")


# ------------------------------------------------------------------------------------------------- other layouts
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dh,tq,tk", [(16, 9, 7), (64, 70, 66), (128, 70, 66), (128, 3, 300)])
@pytest.mark.parametrize("order", [("t", "n", "two"), ("t", "two", "n"), ("n", "two", "t"), ("two", "n", "t")], ids="-".join)
def test_cross_attention_of_rows_side_by_side(dtype, dh, tq, tk, order):
    """Queries as [tq][batch][width], keys and values in one buffer in any order of prompts, rows and the two: the bits of
    dense buffers, and what lies between the rows is left as it was."""
    batch, heads, kvh, prompts, lengths = 3, 2, 1, 2, [tk, tk - 2]
    q, kv, index, dout = base.cross_inputs(dtype, batch, heads, kvh, dh, tq, tk, prompts, lengths, 63)
    kv = base.clean(kv, lengths).cuda()
    wide_, narrow, pad = heads * dh, kvh * dh, 16
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device="cuda")  # noqa: E731
    sizes = (CODE[dtype], batch, heads, kvh, dh, tq, tk)
    counts, strides, step = {"n": prompts, "t": tk, "two": 2}, {}, narrow
    for axis in reversed(order):
        strides[axis] = step
        step = step * counts[axis] + pad
    room = step

    def fused():
        """A buffer of nines, and a view of it as [prompts][tk][2][narrow]."""
        flat = torch.full((room,), 9.0, dtype=ACT[dtype], device="cuda")
        return flat, flat.as_strided((prompts, tk, 2, narrow), (strides["n"], strides["t"], strides["two"], 1))

    def run(side):
        """Outputs as [batch][tq] and [prompts][tk][2] rows."""
        qs = (wide_, batch * wide_) if side else (tq * wide_, wide_)
        rows = lambda t: t.transpose(0, 1).contiguous() if side else t  # noqa: E731
        qq, dd = (rows(t.flatten(2)).cuda() for t in (q, dout))
        out, dq = torch.empty_like(qq), torch.empty_like(qq)
        lse = torch.empty(batch, heads, tq, device="cuda")
        if side:
            (flat, keys), (dflat, dkeys), ks = fused(), fused(), (strides["n"], strides["t"])
            keys.copy_(kv.flatten(3))
            k, v, dk, dv = flat, flat[strides["two"]:], dflat, dflat[strides["two"]:]
        else:
            keys, dkeys, ks = kv.flatten(3), torch.empty_like(kv).flatten(3), (tk * 2 * narrow, 2 * narrow)
            k, v, dk, dv = keys[:, :, 0], keys[:, :, 1], dkeys[:, :, 0], dkeys[:, :, 1]
        ws = torch.empty(fb.flashbon_op_cross_attention_workspace(*sizes), dtype=torch.uint8, device="cuda")
        fb.flashbon_op_cross_attention(*sizes, qq, *qs, k, v, *ks, i32(index), prompts, i32(lengths), out, *qs, lse=lse, workspace=ws)
        ws = torch.empty(fb.flashbon_op_cross_attention_grad_workspace(*sizes, prompts), dtype=torch.uint8, device="cuda")
        fb.flashbon_op_cross_attention_grad(*sizes, qq, *qs, k, v, *ks, i32(index), prompts, i32(lengths), out, *qs, lse, dd, dq, dk, dv, workspace=ws)
        result = [rows(out), lse, rows(dq), dkeys.clone()]
        if side:
            dkeys.fill_(9.0)
            assert bool((dflat == 9.0).all())
        return result

    for a, b in zip(run(True), run(False)):
        assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------------------- adapters
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rank", [8, 128])
@pytest.mark.parametrize("per,scale", [(1, float("inf")), (7, float("nan")), (40, -float("inf"))])
def test_adapters_that_no_row_uses(dtype, rank, per, scale):
    """Weights and a scale of anything: they reach no row, and their gradients are 0."""
    m, n, k, count = 75, 72, 40, 4
    x, down, up, s, _, g = base.adapter_inputs(dtype, m, n, k, rank, count, per, 75)
    index = torch.tensor([2 if i % 3 else -1 if i % 2 else 0 for i in range(-(-m // per))], dtype=torch.int32)
    b, dy, bx = (normal(g, m, w, dtype=ACT[dtype]).cuda() for w in (n, n, k))
    sizes, results = (CODE[dtype], m, n, k, rank, count), []
    for bad in (False, True):
        if bad:
            for a in (1, 3):
                s[a], down[a], up[a] = scale, float("nan"), float("inf")
        args = (x.cuda(), down.cuda(), up.cuda(), s.cuda(), index.cuda(), per)
        out, u = torch.empty_like(b), torch.empty(m, rank, device="cuda")
        fb.flashbon_op_adapters(*sizes, *args, fb.EPI_STORE, b, out, u)
        dx, dd, du = torch.empty_like(bx), torch.empty(count, rank, k, device="cuda"), torch.empty(count, n, rank, device="cuda")
        ws = torch.full((fb.flashbon_op_adapters_grad_workspace(*sizes, per),), 255, dtype=torch.uint8, device="cuda")
        fb.flashbon_op_adapters_grad(*sizes, *args, u, dy, fb.EPI_STORE, bx, dx, dd, du, workspace=ws)
        results.append((out, u, dx, dd, du))
    for clean, got in zip(*results):
        assert torch.equal(clean, got)
    assert not results[1][3][1::2].any() and not results[1][4][1::2].any()


# ------------------------------------------------------------------------------------------- two threads at once
def together(works):
    """Runs each of the works on a thread and a stream of its own, twenty times."""
    failed = []

    def run(work):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(20):
                    work()
            stream.synchronize()
        except Exception as e:   # noqa: BLE001 - reported by the test's own thread
            failed.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=run, args=(w,)) for w in works]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("tq,tk", [(2, 5), (65, 66)])
def test_cross_attention_grad_of_two_batches_at_once(dh, tq, tk):
    """The least and the largest batch, whose kernels ask for different amounts of LDS."""
    works, results = [], []
    for batch in (1, 4096):
        q, kv, _, dout = base.cross_inputs("bf16", batch, 1, 1, dh, tq, tk, 1, [tk], 59 + batch)
        index = torch.zeros(batch, dtype=torch.int32, device="cuda")
        out, lse = base.cross_call("bf16", q, kv, [0] * batch, [tk])
        sizes, qs, ks = (fb.BF16, batch, 1, 1, dh, tq, tk), (tq * dh, dh), (tk * 2 * dh, 2 * dh)
        ws = torch.empty(fb.flashbon_op_cross_attention_grad_workspace(*sizes, 1), dtype=torch.uint8, device="cuda")
        dq, dkv, q, kv, dout = torch.empty_like(out), torch.empty_like(kv).cuda(), q.cuda(), kv.cuda(), dout.cuda()

        def work(sizes=sizes, qs=qs, ks=ks, q=q, kv=kv, index=index, out=out, lse=lse, dout=dout, dq=dq, dkv=dkv, ws=ws):
            fb.flashbon_op_cross_attention_grad(*sizes, q, *qs, kv[:, :, 0], kv[:, :, 1], *ks, index, 1, None, out, *qs, lse, dout, dq,
                                                dkv[:, :, 0], dkv[:, :, 1], workspace=ws)
        work()
        works.append(work)
        results.append((dq, dkv, dq.clone(), dkv.clone()))
    for dq, dkv, _, _ in results:
        dq.zero_(), dkv.zero_()
    together(works)
    for dq, dkv, a, b in results:
        assert torch.equal(dq, a) and torch.equal(dkv, b)


def test_two_branches_at_once():
    branches = [base.Branch(61).device(), base.Branch(62, tokens=70, heads=3, dh=128, text=90, rank=48).device()]
    want = []
    for b in branches:
        b.step()
        want.append(b.results())
        for name in b.RESULTS:
            getattr(b, name).zero_()
    together([b.step for b in branches])
    for b, w in zip(branches, want):
        for name, t in b.results().items():
            assert torch.equal(t, w[name]), name
