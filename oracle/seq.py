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
