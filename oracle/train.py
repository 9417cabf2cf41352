"""Operators of a policy update in 64 bits for the oracle (test infrastructure): attention over packed documents, the
modulated LayerNorm, the gradient of the clipped objective (Eq. 5) and AdamW, each written from its formula.

Pins (tests/test_oracle_train.py): gradients against differences of the forward value; codes of 8-bit states against
a search over all codes.
"""
import numpy as np

from oracle import philox


def spans(off, rows):
    """[(first, end)] of the documents of an offset array, held within [0, rows]."""
    o = np.clip(np.asarray(off, np.int64), 0, rows)
    return [(int(a), int(max(a, b))) for a, b in zip(o, o[1:])]


def attention(q, k, v, q_off, k_off, scale):
    """q [Tq, NH, d], k, v [Tk, NKV, d] -> out [Tq, NH, d], lse [NH, Tq], and per (document, head) what the gradient needs."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    Tq, NH, _ = q.shape
    share = NH // k.shape[1]
    out, lse, kept = np.zeros_like(q), np.full((NH, Tq), -np.inf), []
    for (a, b), (x, y) in zip(spans(q_off, Tq), spans(k_off, k.shape[0])):
        if a == b or x == y:
            continue
        for h in range(NH):
            s = q[a:b, h] @ k[x:y, h // share].T * scale
            top = s.max(1, keepdims=True)
            e = np.exp(s - np.where(np.isinf(top), 0, top))
            t = e.sum(1, keepdims=True)
            p = e / np.where(t == 0, 1, t)
            with np.errstate(divide="ignore"):
                lse[h, a:b] = (top + np.log(t))[:, 0]
            out[a:b, h] = p @ v[x:y, h // share]
            kept.append((a, b, x, y, h, p))
    return out, lse, kept


def attention_grad(dout, q, k, v, q_off, k_off, scale):
    """-> dq, dk, dv, and for each a bound of the terms that rounding touches: sums of |p dout|, |ds k| and |ds q| with
    |p| sum |dout out| added to every |ds| (what an error in dout . out weighs)."""
    dout, q, k, v = (np.asarray(x, np.float64) for x in (dout, q, k, v))
    out, _, kept = attention(q, k, v, q_off, k_off, scale)
    share = q.shape[1] // k.shape[1]
    dq, dk, dv, wq, wk, wv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for a, b, x, y, h, p in kept:
        g, do, o = h // share, dout[a:b, h], out[a:b, h]
        ds = p * (do @ v[x:y, g].T - (do * o).sum(1, keepdims=True)) * scale
        w = (np.abs(ds) + p * (np.abs(do) @ np.abs(v[x:y, g]).T + (np.abs(do) * np.abs(o)).sum(1, keepdims=True)) * scale)
        dq[a:b, h], wq[a:b, h] = ds @ k[x:y, g], w @ np.abs(k[x:y, g])
        dk[x:y, g] += ds.T @ q[a:b, h]
        wk[x:y, g] += w.T @ np.abs(q[a:b, h])
        dv[x:y, g] += p.T @ do
        wv[x:y, g] += p.T @ np.abs(do)
    return (dq, dk, dv), (wq, wk, wv)


def layer_norm(x, mods, shift_off, scale_off, row_off, group, eps=1e-6):
    """-> out (NaN in rows of no document or of a group that is none), mean, rstd."""
    x, mods = np.asarray(x, np.float64), np.asarray(mods, np.float64)
    H, out = x.shape[1], np.full(np.shape(x), np.nan)
    mean = x.mean(1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    for (a, b), g in zip(spans(row_off, len(x)), group):
        if 0 <= g < len(mods):
            out[a:b] = (x[a:b] - mean[a:b, None]) * rstd[a:b, None] * (1 + mods[g, scale_off:scale_off + H]) + mods[g, shift_off:shift_off + H]
    return out, mean, rstd


def layer_norm_grad(dout, x, mean, rstd, mods, shift_off, scale_off, row_off, group, residual):
    """-> dx (NaN in rows that the operator leaves alone), dshift, dscale [groups, H]."""
    dout, x, mean, rstd, mods = (np.asarray(t, np.float64) for t in (dout, x, mean, rstd, mods))
    H, dx = x.shape[1], np.full(x.shape, np.nan)
    dshift, dscale = np.zeros((len(mods), H)), np.zeros((len(mods), H))
    for (a, b), k in zip(spans(row_off, len(x)), group):
        if not 0 <= k < len(mods):
            continue
        y = (x[a:b] - mean[a:b, None]) * rstd[a:b, None]
        g = dout[a:b] * (1 + mods[k, scale_off:scale_off + H])
        dx[a:b] = rstd[a:b, None] * (g - g.mean(1, keepdims=True) - y * (g * y).mean(1, keepdims=True)) + (0 if residual is None else residual[a:b])
        dshift[k] += dout[a:b].sum(0)
        dscale[k] += (dout[a:b] * y).sum(0)
    return dx, dshift, dscale


def objective_grad(z, v_rows, edge_ids, row_parent, row_first, row_coef, logp_old, adv, clip_eps, n_total):
    """-> J, logp_new [edges], d(-J)/dv [rows, D], clipped [edges]."""
    z, v_rows = np.asarray(z, np.float64), np.asarray(v_rows, np.float64)
    n, J, grad = len(edge_ids), 0.0, np.zeros(v_rows.shape)
    logp, clipped = np.zeros(n), np.zeros(n, bool)
    for r, (a_z, a_v, h, c0) in enumerate(row_coef):
        mu = a_z * z[row_parent[r]] + a_v * v_rows[r]
        for e in range(row_first[r], row_first[r + 1]):
            d = z[edge_ids[e]] - mu
            logp[e] = c0 - h * (d ** 2).sum()
            rho, a = np.exp(logp[e] - np.float64(logp_old[edge_ids[e]])), np.float64(adv[edge_ids[e]])
            held = np.clip(rho, 1 - clip_eps, 1 + clip_eps) * a
            clipped[e] = held < rho * a
            J += min(rho * a, held) / n_total
            if not clipped[e]:
                grad[r] -= rho * a / n_total * 2 * h * a_v * d
    return J, logp, grad, clipped


# ---------------------------------------------------------------------------------------------------- AdamW, states in 8 bits
TAG_ADAMW = 4


def code_values(bits):
    """Values of the codes without a sign: 4 bits of exponent, `bits` of mantissa."""
    c = np.arange(16 << bits)
    e, f = c >> bits, c & ((1 << bits) - 1)
    return np.where(e > 0, (f + (1 << bits)) * 2.0 ** (e - 1.0), f)


def decode(code, scale, bits, sign):
    """fp32 values, as an update reads them."""
    table = code_values(bits).astype(np.float32)
    x = table[code & 127] * np.where(code & 128, np.float32(-1), np.float32(1)) if sign else table[code]
    return (x.astype(np.float32) * np.repeat(np.asarray(scale, np.float32), 256)[:len(code)]).astype(np.float32)


def encode(x, bits, random16, sign):
    """Codes and scales of fp32 values, in fp32 operations that each round once."""
    x, n = np.asarray(x, np.float32), len(x)
    most = np.float32(code_values(bits)[-1])
    a = np.zeros(-(-n // 256) * 256, np.float32)
    a[:n] = np.abs(x)
    top = a.reshape(-1, 256).max(1)
    some = top > np.float32(2.0 ** -96)
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        scale = np.where(np.isfinite(top), np.where(some, top / most, np.float32(0)), np.float32(np.nan)).astype(np.float32)
        up = np.where(np.isfinite(top) & some, most / top, np.float32(0)).astype(np.float32)
        y = np.minimum(np.nan_to_num(a * np.repeat(up, 256), nan=0.0), most)[:n]
    e = np.maximum(np.frexp(y)[1] - 1 - bits, 0)
    q = np.floor(np.ldexp(y, -e).astype(np.float32) + random16.astype(np.float32) * np.float32(1 / 65536)).astype(np.int64)
    code = (e << bits) + q
    if sign:
        code = code | np.where(x < 0, 128, 0)
    return code.astype(np.uint8), scale


def adamw_words(seed, index, step, n):
    """The 32 random bits of the elements of tensor `index`."""
    quads = np.arange(-(-n // 4), dtype=np.uint64)
    counter = np.stack([quads, np.full_like(quads, index), np.full_like(quads, step), np.full_like(quads, TAG_ADAMW)], -1)
    return philox.philox4x32_10(counter, seed).reshape(-1)[:n]


def adamw(p, g, m, v, step, lr, beta1, beta2, eps, weight_decay, f=np.float64):
    """One step in the type f, every operation rounded by itself -> p, m, v, sqrt(v)."""
    p, g, m, v = (np.asarray(x).astype(f) for x in (p, g, m, v))
    m = m * f(beta1) + g * f(1 - beta1)
    v = v * f(beta2) + (g * f(1 - beta2)) * g
    root = np.sqrt(v)
    p = p * f(1 - lr * weight_decay) - (m / (root * f(1 / np.sqrt(1 - beta2 ** step)) + f(eps))) * f(lr / (1 - beta1 ** step))
    return p, m, v, root
