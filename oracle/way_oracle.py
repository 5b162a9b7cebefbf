"""The way into the experts in binary64 (numpy): norms and their gradients, routing by scores, values in 8 bits and the experts'
products of them.  Written from the formulas of include/symi.h; shares no code with the GPU path."""
import numpy as np

BLOCK = 128


# ---- norm

def norm(R, center, eps, w=None, b=None):
    """dict of Y, mean, rstd, var of rows R [T, d] (the residual sum already taken)."""
    R = R.astype(np.float64)
    mean = R.mean(axis=1) if center else np.zeros(len(R))
    x = R - mean[:, None]
    var = (x * x).mean(axis=1)
    with np.errstate(all="ignore"):
        rstd = 1 / np.sqrt(var + eps)
        y = x * rstd[:, None]
    y = y * (1.0 if w is None else w.astype(np.float64)) + (0.0 if b is None else b.astype(np.float64))
    return {"Y": y, "mean": mean, "rstd": rstd, "var": var}


def norm_gradient(dY, R, mean, rstd, center, w=None, dR=None):
    dY, R = dY.astype(np.float64), R.astype(np.float64)
    xh = (R - (mean.astype(np.float64)[:, None] if center else 0.0)) * rstd.astype(np.float64)[:, None]
    g = dY * (1.0 if w is None else w.astype(np.float64))
    level = g.mean(axis=1, keepdims=True) if center else np.zeros((len(g), 1))
    along = (g * xh).mean(axis=1, keepdims=True)
    dX = (g - level - xh * along) * rstd.astype(np.float64)[:, None]
    if dR is not None:
        dX = dX + dR.astype(np.float64)
    return {"dX": dX, "dw": (dY * xh).sum(axis=0), "db": dY.sum(axis=0), "xh": xh, "g": g, "level": level, "along": along}


# ---- routing by scores

def scores(z, sigmoid):
    """Scores of a row, masked classes with 0."""
    live = z > -np.inf
    s = np.zeros(len(z))
    if sigmoid:
        with np.errstate(over="ignore"):
            s[live] = 1 / (1 + np.exp(-z[live]))
    elif live.any():
        e = np.exp(z[live] - z[live].max())
        s[live] = e / e.sum()
    return s


def route(logits, bias, k, renorm, sigmoid, groups, top_groups, group_top, scale):
    """dict of idx [T, k], gate [T, k], hist [E], real [T, k]: whether a choice was one (else it filled up)."""
    T, E = logits.shape
    per = E // groups
    idx, gate, real = np.zeros((T, k), dtype=np.int64), np.zeros((T, k)), np.zeros((T, k), dtype=bool)
    with np.errstate(all="ignore"):
        for t in range(T):
            z = logits[t].astype(np.float64)
            s = scores(z, sigmoid)
            c = s + bias.astype(np.float64) if bias is not None else z
            live = (z > -np.inf) & (c > -np.inf)
            value = c if bias is not None or group_top == 1 else s
            if groups > 1:
                of = []
                for g in range(groups):
                    mine = sorted((value[e] for e in range(g * per, g * per + per) if live[e]), reverse=True)[:group_top]
                    of.append(sum(mine) if mine else -np.inf)
                kept = sorted(range(groups), key=lambda g: (-of[g], g))[:top_groups]
                live = live & np.isin(np.arange(E) // per, kept)
            best = sorted((e for e in range(E) if live[e]), key=lambda e: (-c[e], e))[:k]
            chosen = best + [e for e in range(E) if e not in best and not live[e]][:k - len(best)]
            idx[t], real[t, :len(best)] = chosen, True
            if not best:
                pass
            elif renorm:     # relative to the largest of the chosen
                low = np.minimum(z[best], 0) - np.log1p(np.exp(-np.abs(z[best]))) if sigmoid else z[best]
                part = np.exp(low - low.max())
                gate[t, :len(best)] = scale * part / part.sum()
            else:
                gate[t, :len(best)] = scale * s[best]
            if np.isnan(z).any() or (not sigmoid and (z == np.inf).any()):
                gate[t] = np.nan
    return {"idx": idx, "gate": gate, "hist": np.bincount(idx.reshape(-1), minlength=E), "real": real}


def route_gradient(logits, idx, real, dgate, renorm, sigmoid, scale):
    """(dlogits [T, E], the sum of the sizes of what each is a difference of)."""
    T, E = logits.shape
    out, size = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        z = logits[t].astype(np.float64)
        s = scores(z, sigmoid)
        j = idx[t][real[t]]
        dg = scale * dgate[t][real[t]].astype(np.float64)
        if not len(j):
            continue
        if renorm:
            low = np.minimum(z[j], 0) - np.log1p(np.exp(-np.abs(z[j]))) if sigmoid else z[j]
            g = np.exp(low - low.max())
            g /= g.sum()
            out[t, j] = g * (dg - (g * dg).sum())
            size[t, j] = g * (np.abs(dg) + np.abs(g * dg).sum())
        elif sigmoid:
            out[t, j], size[t, j] = s[j] * dg, s[j] * np.abs(dg)
        else:
            out[t] = -s * (s[j] * dg).sum()
            size[t] = s * np.abs(s[j] * dg).sum()
            out[t, j] += s[j] * dg
            size[t, j] += s[j] * np.abs(dg)
        if sigmoid:
            keep = np.exp(-np.logaddexp(0, np.where(z > -np.inf, z, 0)))
            out[t], size[t] = out[t] * np.where(z > -np.inf, keep, 1), size[t] * np.where(z > -np.inf, keep, 1)
    return out, size


# ---- values in 8 bits

def power(most):
    """s of a block whose largest finite |x| is `most`: the smallest byte with most <= 448 * 2 ** (s - 127)."""
    s = 0
    if most > 0:
        s = max(0, int(np.floor(np.log2(most))) - 10 + 127)
        while most > 448 * 2.0 ** (s - 127):
            s += 1
    return s


def to_e4m3(y):
    """|y| <= 448 to the nearest value of e4m3, ties to the even one."""
    step = 2.0 ** (np.maximum(np.frexp(y)[1] - 1, -6) - 3)
    return np.rint(y / step) * step


def quant(x, block):
    """(q as numbers [R, n], s [ceil(R / block), ceil(n / 128)]) of one group of rows."""
    x = x.astype(np.float64)
    R, n = x.shape
    rb, cb = -(-R // block), -(-n // BLOCK)
    q, s = np.zeros((R, n)), np.zeros((rb, cb), dtype=np.int64)
    for i in range(rb):
        for j in range(cb):
            part = x[i * block:(i + 1) * block, j * BLOCK:(j + 1) * BLOCK]
            fine = np.isfinite(part)
            s[i, j] = power(np.abs(part[fine]).max() if fine.any() else 0.0)
            y = np.where(fine, part, 0) * 2.0 ** (127 - s[i, j])
            q[i * block:(i + 1) * block, j * BLOCK:(j + 1) * BLOCK] = np.where(fine, to_e4m3(y), np.nan)
    return q, s


def values(q, s, block):
    """What codes (as numbers) and scales stand for."""
    R, n = q.shape
    scale = 2.0 ** (s.astype(np.float64) - 127)
    return q * np.repeat(np.repeat(scale, block, axis=0)[:R], BLOCK, axis=1)[:, :n]


def product(a, w, offsets):
    """(Y, the sum of the summands' sizes) of rows a [A, n] and weights w [S, R, n], both as the values they stand for."""
    Y, size = np.zeros((len(a), w.shape[1])), np.zeros((len(a), w.shape[1]))
    for p in range(len(w)):
        rows = slice(offsets[p], offsets[p + 1])
        Y[rows], size[rows] = a[rows] @ w[p].T, np.abs(a[rows]) @ np.abs(w[p]).T
    return Y, size


def silu_product(u, v):
    with np.errstate(over="ignore"):
        return u / (1 + np.exp(-u)) * v
