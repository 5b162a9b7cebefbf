"""The ends of a training step in binary64 (numpy): token embedding and its gradient, the clipped policy loss with its
gradient, AdamW with states in 32 or 8 bits.  Written from the formulas of include/symi.h; shares no code with the GPU path."""
import numpy as np

BLOCK = 256
WORD = 0xffffffff


def embed(tokens, table, scale):
    V = len(table)
    out = np.zeros((len(tokens), table.shape[1]))
    live = (tokens >= 0) & (tokens < V)
    out[live] = scale * table[tokens[live]].astype(np.float64)
    return out


def embed_gradient(tokens, dX, V, scale):
    """(gradient [V, d], the sum of the summands' sizes [V, d], their number [V]): the last two for error bounds."""
    out, size, count = np.zeros((V, dX.shape[1])), np.zeros((V, dX.shape[1])), np.zeros(V)
    for t, v in enumerate(tokens):
        if 0 <= v < V:
            out[v] += scale * dX[t].astype(np.float64)
            size[v] += abs(scale) * np.abs(dX[t].astype(np.float64))
            count[v] += 1
    return out, size, count


def policy(z, V, action, old, ref, advantage, weight, clip_low, clip_high, kl_coef, inv_temp, grad_scale=1.0):
    """dict of logp [T], stats [4], dlogits [T, ld], and p, slope, kl, ratio, e per token; a token that does not count has zeros."""
    T, ld = z.shape
    out = {"logp": np.zeros(T), "dlogits": np.zeros((T, ld)), "terms": np.zeros((T, 4)), "p": np.zeros((T, V)),
           "ratio": np.zeros(T), "e": np.zeros(T)}
    with np.errstate(all="ignore"):
        for t in range(T):
            a = int(action[t])
            if weight[t] == 0 or not 0 <= a < V:
                continue
            x = z[t, :V].astype(np.float64) * inv_temp
            m = x.max()
            s = np.exp(x - m).sum()
            lp = (x[a] - m) - np.log(s)
            out["logp"][t] = lp
            if old is None:
                continue
            A, w = float(advantage[t]), float(weight[t])
            r = np.exp(lp - float(old[t]))
            bounded = min(max(r, 1 - clip_low), 1 + clip_high)
            gain = -min(r * A, bounded * A)
            clipped = bounded * A < r * A
            far = float(ref[t]) - lp if ref is not None else 0.0
            e = np.expm1(far)
            kl = e - far
            slope = (0.0 if clipped else -A * r) - kl_coef * e
            out["terms"][t] = w * (gain + kl_coef * kl), w * gain, w * kl, w * clipped
            out["ratio"][t], out["e"][t] = r, e
            out["p"][t] = np.exp(x - m) / s
            u = grad_scale * w * inv_temp * slope
            out["dlogits"][t, :V] = -u * out["p"][t]
            out["dlogits"][t, a] += u
    out["stats"] = out["terms"].sum(axis=0)
    return out


# ---- AdamW

def _mix(x):
    x = x ^ (x >> 16)
    x = (x * 0xBB67AE85) & WORD
    x = x ^ (x >> 15)
    x = (x * 0x6A09E667) & WORD
    return x ^ (x >> 16)


def random_numbers(seed, step, first_block, n):
    """The two numbers in (0, 1) of every element of a tensor whose first block is `first_block` of all."""
    key = _mix((_mix(seed & WORD) + step) & WORD)
    i = np.arange(first_block * BLOCK, first_block * BLOCK + n, dtype=np.uint64)
    times = np.array([0x3C6EF373, 0xA54FF53B, 0x510E527F, 0x9B05688D], dtype=np.uint64)[i & 3]
    h = _mix((((i >> 2) & WORD) * 0x9E3779B1 + key) & WORD)
    r = (h * times) & WORD
    r = r ^ (r >> 15)
    return ((r & 0xffff) + 0.5) / 65536, ((r >> 16) + 0.5) / 65536


def m_values(codes, scale):
    c = codes.astype(np.float64)
    return np.sign(c) * (c / 127) ** 2 * np.repeat(scale.astype(np.float64), BLOCK)[:len(c)]


def v_values(codes, scale):
    return (codes.astype(np.float64) / 255) ** 4 * np.repeat(scale.astype(np.float64), BLOCK)[:len(codes)]


def block_max(x):
    pad = np.zeros(-len(x) % BLOCK)
    return np.abs(np.concatenate([x, pad])).reshape(-1, BLOCK).max(axis=1)


def encode(x, power, top, u):
    """(codes without sign, how near the choice was: the distance of the random number to the threshold) of x >= 0."""
    a = np.repeat(block_max(x), BLOCK)[:len(x)]
    part = x / np.where(a > 0, a, 1)
    lo = np.clip(np.floor(top * part ** (1 / power)), 0, top - 1)
    below, above = (lo / top) ** power, ((lo + 1) / top) ** power
    share = (part - below) / (above - below)
    return lo + (share > u), np.minimum(np.abs(share - u), np.minimum(np.abs(share), np.abs(1 - share)))


def adamw(w, g, m, v, lr, beta1, beta2, eps, wd, step, gscale=1.0):
    """(w, m, v) after the step; the states before they are rounded to codes."""
    g = gscale * g.astype(np.float64)
    m = beta1 * m.astype(np.float64) + (1 - beta1) * g
    v = beta2 * v.astype(np.float64) + (1 - beta2) * g * g
    w = w.astype(np.float64)
    return w - lr * (m / (1 - beta1 ** step) / (np.sqrt(v / (1 - beta2 ** step)) + eps) + wd * w), m, v
