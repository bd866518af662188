"""The cross-attention branch with a prompt and an adapter per candidate, and its gradients, in 64 bits.

LayerNorm with statistics, attention to prompts of their own lengths and low-rank adapters, forward and backward, written
from the formulas as loops over groups, candidates and heads.
"""
import numpy as np


def _wide(x):
    return None if x is None else np.asarray(x, np.float64)


def _factor(weight, rows, per, modulated):
    if weight is None:
        return 1.0
    f = _wide(weight)[np.arange(rows) // per]
    return 1.0 + f if modulated else f


def layer_norm(x, weight, bias, per, modulated, eps):
    """(y, mean, rstd) of rows x [M][D]; weight and bias [groups][D] or None, one for each ``per`` rows."""
    x = _wide(x)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None] * _factor(weight, len(x), per, modulated)
    if bias is not None:
        y = y + _wide(bias)[np.arange(len(x)) // per]
    return y, mean, rstd


def layer_norm_grad(x, weight, per, modulated, mean, rstd, dy, residual=None):
    """(dx, dweight, dbias) from the gradient dy of y and the saved statistics."""
    x, dy, rstd = _wide(x), _wide(dy), _wide(rstd)[:, None]
    xhat = (x - _wide(mean)[:, None]) * rstd
    g = dy * _factor(weight, len(x), per, modulated)
    dx = rstd * (g - g.mean(1, keepdims=True) - xhat * (g * xhat).mean(1, keepdims=True))
    if residual is not None:
        dx = dx + _wide(residual)
    groups = -(-len(x) // per)
    rows = [slice(i * per, (i + 1) * per) for i in range(groups)]
    return dx, np.stack([(dy[r] * xhat[r]).sum(0) for r in rows]), np.stack([dy[r].sum(0) for r in rows])


def _prompt(index, b, n):
    return b if index is None else min(max(int(index[b]), 0), n - 1)


def _keys(lengths, c, tk):
    return tk if lengths is None else min(max(int(lengths[c]), 0), tk)


def cross_attention(q, k, v, index=None, lengths=None):
    """(out, lse [b][h][tq]) for q [b][tq][h][dh], k and v [n][tk][kv heads][dh]."""
    q, k, v = _wide(q), _wide(k), _wide(v)
    batch, tq, heads, dh = q.shape
    out, lse = np.zeros_like(q), np.full((batch, heads, tq), -np.inf)
    for b in range(batch):
        c = _prompt(index, b, len(k))
        n = _keys(lengths, c, k.shape[1])
        if n == 0:
            continue
        for h in range(heads):
            kh = h * k.shape[2] // heads
            s = q[b, :, h] @ k[c, :n, kh].T / np.sqrt(dh)
            top = s.max(1, keepdims=True)
            live = ~np.isneginf(top[:, 0])       # a row whose scores are all -infinity is that of an empty prompt
            e = np.exp(s[live] - top[live])
            out[b, live, h] = e @ v[c, :n, kh] / e.sum(1, keepdims=True)
            lse[b, h, live] = top[live, 0] + np.log(e.sum(1))
    return out, lse


def cross_attention_grad(q, k, v, out, lse, dout, index=None, lengths=None):
    """(dq, dk, dv) from the gradient dout of out, with out and lse of the forward pass."""
    q, k, v, out, lse, dout = (_wide(t) for t in (q, k, v, out, lse, dout))
    batch, tq, heads, dh = q.shape
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for b in range(batch):
        c = _prompt(index, b, len(k))
        n = _keys(lengths, c, k.shape[1])
        if n == 0:
            continue
        for h in range(heads):
            kh = h * k.shape[2] // heads
            keys, values, do = k[c, :n, kh], v[c, :n, kh], dout[b, :, h]
            p = np.exp(q[b, :, h] @ keys.T / np.sqrt(dh) - np.where(np.isneginf(lse[b, h]), np.inf, lse[b, h])[:, None])
            ds = p * (do @ values.T - (do * out[b, :, h]).sum(1, keepdims=True)) / np.sqrt(dh)
            dq[b, :, h] = ds @ keys
            dk[c, :n, kh] += ds.T @ q[b, :, h]
            dv[c, :n, kh] += p.T @ do
    return dq, dk, dv


def _groups(rows, per, index, count):
    """(adapter, rows) of each group that has an adapter."""
    for i in range(-(-rows // per)):
        a = 0 if index is None else int(index[i])
        if 0 <= a < count:
            yield a, slice(i * per, min((i + 1) * per, rows))


def adapters(x, down, up, scales=None, index=None, per=1, base=None, gate=None):
    """(out, u): out = base + gate s (x down^T) up^T, u = x down^T, for x [M][K], down [n][r][K], up [n][N][r]."""
    x, down, up, scales, gate = (_wide(t) for t in (x, down, up, scales, gate))
    out = np.zeros((len(x), up.shape[1])) if base is None else _wide(base).copy()
    u = np.zeros((len(x), down.shape[1]))
    for a, rows in _groups(len(x), per, index, len(down)):
        u[rows] = x[rows] @ down[a].T
        out[rows] += (1.0 if scales is None else scales[a]) * (1.0 if gate is None else gate) * (u[rows] @ up[a].T)
    return out, u


def adapters_grad(x, down, up, u, dy, scales=None, index=None, per=1, base=None):
    """(dx, d_down, d_up) from the gradient dy of out (times the gate, where there is one) and u."""
    x, down, up, u, dy, scales = (_wide(t) for t in (x, down, up, u, dy, scales))
    dx = np.zeros_like(x) if base is None else _wide(base).copy()
    d_down, d_up = np.zeros_like(down), np.zeros_like(up)
    for a, rows in _groups(len(x), per, index, len(down)):
        s = 1.0 if scales is None else scales[a]
        du = s * (dy[rows] @ up[a])
        dx[rows] += du @ down[a]
        d_down[a] += du.T @ x[rows]
        d_up[a] += s * (dy[rows].T @ u[rows])
    return dx, d_down, d_up
