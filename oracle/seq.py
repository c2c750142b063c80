"""The sequence operators from their definitions, in 64 bits, on numpy arrays; and how far an fp32 evaluation may be off.

Each function returns (result, bound): the bound is what rounding every operation to fp32 can add up to, without the rounding of
the result to its own type.  `U` is half a unit in the last place of 1; the counts of operations are generous by two or three."""
import numpy as np

U = 2.0 ** -24
E4M3_MAX, MIN_SCALE, BLOCK = 448.0, 2.0 ** -126, 128


def silu(v):
    with np.errstate(over="ignore"):
        return v / (1 + np.exp(-v))


def softplus(v):
    return np.maximum(v, 0) + np.log1p(np.exp(-np.abs(v)))


def causal_conv(x, weight, bias, state, lengths, act):
    """x [batch, length, channels], state [batch, taps - 1, channels]; returns y, bound, new state."""
    batch, length, channels = x.shape
    taps = weight.shape[1]
    y, bound = np.zeros(x.shape), np.zeros(x.shape)
    new = np.zeros((batch, taps - 1, channels))
    for b in range(batch):
        wide = np.concatenate([state[b], x[b, :lengths[b]]]) if state is not None else np.concatenate([np.zeros((taps - 1, channels)), x[b, :lengths[b]]])
        for t in range(lengths[b]):
            s, m = np.array(bias, copy=True), np.abs(bias)
            for j in range(taps):
                s = s + weight[:, j] * wide[t + j]
                m = m + np.abs(weight[:, j] * wide[t + j])
            e = (taps + 2) * U * m
            # silu's slope is at most 1.1; the hardware exponential and reciprocal are good to a few units
            y[b, t], bound[b, t] = (silu(s), 1.1 * e + 8 * U * (1 + np.abs(s)) * np.abs(silu(s))) if act else (s, e)
        new[b] = wide[lengths[b]:]
    return y, bound, new


def selective_scan(u, delta, A, B, C, D, z, delta_bias, state, lengths, plus):
    """Returns y, its bound, the new state, its bound."""
    batch, length, channels = u.shape
    states = A.shape[1]
    y, bound = np.zeros(u.shape), np.zeros(u.shape)
    new, new_bound = np.zeros((batch, channels, states)), np.zeros((batch, channels, states))
    for b in range(batch):
        h = np.zeros((channels, states)) if state is None else state[b].copy()
        mag, err = np.abs(h), np.zeros_like(h)      # of the sums of magnitudes, and what has gone wrong so far
        for t in range(lengths[b]):
            raw = delta[b, t] + delta_bias
            d = softplus(raw) if plus else raw
            # relative error of d: the sum's rounding moves the exponential, then some ten operations
            rd = (12 + 2 * (np.abs(delta[b, t]) + np.abs(delta_bias))) * U if plus else 2 * U * (np.abs(delta[b, t]) + np.abs(delta_bias)) / np.maximum(np.abs(raw), 1e-30)
            a = np.exp(d[:, None] * A)
            ra = (4 * U + rd[:, None]) * np.abs(d[:, None] * A) + 4 * U
            put = (d * u[b, t])[:, None] * B[b, t][None]
            err = a * err + ra * a * mag + (rd[:, None] + 4 * U) * np.abs(put) + 2 * U * (a * mag + np.abs(put))
            h = a * h + put
            mag = a * mag + np.abs(put)
            out = (h * C[b, t]).sum(1)
            e = (np.abs(C[b, t]) * (err + (states + 4) * U * mag)).sum(1)
            if D is not None:
                out, e = out + D * u[b, t], e + 3 * U * np.abs(D * u[b, t])
            if z is not None:
                g = silu(z[b, t])
                out, e = out * g, e * np.abs(g) + (10 + 2 * np.abs(z[b, t])) * U * np.abs(out * g)
            y[b, t], bound[b, t] = out, e
        new[b], new_bound[b] = h, err
    return y, bound, new, new_bound


def quantize(x, block_rows):
    """x / scale before it is rounded to eight bits, and the scales; fp32 as the definition has them."""
    rows, k = x.shape
    rb, kb = -(-rows // block_rows), -(-k // BLOCK)
    scales, q = np.zeros((rb, kb), np.float32), np.zeros((rows, k), np.float32)
    with np.errstate(all="ignore"):
        for i in range(rb):
            for j in range(kb):
                part = x[i * block_rows:(i + 1) * block_rows, j * BLOCK:(j + 1) * BLOCK].astype(np.float32)
                s = np.abs(part).max() / np.float32(E4M3_MAX)
                scales[i, j] = s if np.isnan(s) else max(s, np.float32(MIN_SCALE))
                q[i * block_rows:(i + 1) * block_rows, j * BLOCK:(j + 1) * BLOCK] = part / scales[i, j]
    return q, scales


def block_matmul(a, a_scales, b, b_scales, bias):
    """a [m, k], b [n, k] as the numbers they stand for; returns y and the sum of the magnitudes of what is added."""
    m, k = a.shape
    n = b.shape[0]
    y, mag = np.tile(bias, (m, 1)), np.tile(np.abs(bias), (m, 1))
    for j in range(-(-k // BLOCK)):
        at = slice(j * BLOCK, (j + 1) * BLOCK)
        s = a_scales[:, j, None] * np.repeat(b_scales[:, j], BLOCK)[None, :n]
        y = y + s * (a[:, at] @ b[:, at].T)
        mag = mag + np.abs(s) * (np.abs(a[:, at]) @ np.abs(b[:, at]).T)
    return y, mag


def rms_norm(x, residual, weight, eps):
    """y, its bound, and the sum x + residual."""
    r = x if residual is None else x + residual
    root = np.sqrt((r ** 2).mean(1, keepdims=True) + eps)
    y = r / root * weight
    # the sum's rounding, at most 64 squares one after the other in each of some lanes that meet in pairs (half of it: a root), root, three products
    return y, (52 + 10) * U * np.abs(y) + 2.0 ** -149, r


def add_adapters(y, x, down, up, scales, index, lengths, parts):
    """out and its bound; with `parts` it allows for a down x that is rounded to 16 bits."""
    out, bound = np.array(y, copy=True), np.zeros(y.shape)
    k, rank = x.shape[2], up.shape[2]
    for b, n in enumerate(lengths):
        e = index[b]
        if 0 <= e < len(down):
            s = 1.0 if scales is None else scales[e]
            t, mag = x[b, :n] @ down[e].T * s, np.abs(x[b, :n]) @ np.abs(down[e]).T * abs(s)
            off = (k + 6) * U * mag + (2.0 ** -16 if parts else 0) * np.abs(t)
            more = np.abs(t) @ np.abs(up[e]).T
            out[b, :n] += t @ up[e].T
            bound[b, :n] = off @ np.abs(up[e]).T + (rank + 6) * U * (more + np.abs(y[b, :n]))
        out[b, n:] = 0
    return out, bound


def gated_delta_rule(q, k, v, g, beta, scale, normalize, state, lengths, parts):
    """y, its bound, the new states, and the bound of their columns' 2-norms.

    A token multiplies what the columns of the states are off by with exp(g) (I - beta k k^T), whose 2-norm is max(1, |1 - beta k.k|), and adds
    its own rounding: sums over the numbers of a key and over the up to 64 tokens that are worked on together, of the states' and the correction's size.
    With `parts` it allows for operands rounded to 16 bits in the result's own sums."""
    batch, length, heads, dv = v.shape
    dk, group = q.shape[3], heads // q.shape[2]
    if normalize:
        q, k = (t / np.sqrt((t ** 2).sum(-1, keepdims=True) + 1e-6) for t in (q, k))
    y, bound = np.zeros(v.shape), np.zeros(v.shape)
    new, new_bound = np.zeros((batch, heads, dk, dv)), np.zeros((batch, heads, dv))
    c = 2 * (dk + 64) * U
    at = np.arange(heads) // group
    with np.errstate(under="ignore"):
        for b in range(batch):
            S = np.zeros((heads, dk, dv)) if state is None else state[b].copy()
            off = np.zeros((heads, dv))
            recent = np.sqrt((S ** 2).sum(1))           # the largest states of the last 64 tokens, decayed: what is added up inside a chunk
            for t in range(lengths[b]):
                gt = np.clip(g[b, t], -128, 0)
                e = np.exp(gt)[:, None]
                S = S * e[..., None]
                kt, qt, bt = k[b, t, at], q[b, t, at], beta[b, t][:, None]
                nk, nq = np.sqrt((kt ** 2).sum(1))[:, None], np.sqrt((qt ** 2).sum(1))[:, None]
                size = np.sqrt((S ** 2).sum(1))
                d = bt * (v[b, t] - np.einsum("hij,hi->hj", S, kt))
                grow = np.maximum(1, np.abs(1 - bt * nk ** 2))
                recent = np.maximum(recent * e, size) + np.abs(bt) * nk * np.abs(v[b, t])
                off = grow * e * off + c * (recent + np.abs(bt) * nk * (nk * recent + np.abs(v[b, t])))
                S = S + kt[..., None] * d[:, None, :]
                y[b, t] = scale * np.einsum("hij,hi->hj", S, qt)
                bound[b, t] = abs(scale) * nq * (off + (c + (3 * 2.0 ** -16 if parts else 0)) * (recent + np.abs(d) * nk))
            new[b], new_bound[b] = S, off
    return y, bound, new, new_bound
