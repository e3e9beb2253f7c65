"""Microscaled 4 bits and layers of experts in float64, written from their definitions (NumPy): the truth that the tests compare the device with."""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def width(n):
    return (n + 127) // 128 * 128


def quantize(x, mdiag=None):
    """x: rows x n (numbers of at most 32 bits).  (codes rows x width, one a byte; scale bytes rows x width / 32)."""
    u = np.asarray(x, np.float32)
    if mdiag is not None:
        with np.errstate(all="ignore"):
            u = u / np.asarray(mdiag, np.float32)            # the quotient is one of 32 bits
    rows, n = u.shape
    full = np.zeros((rows, width(n)), np.float64)
    full[:, :n] = u
    b = full.reshape(rows, -1, 32)
    bad = ~np.isfinite(b).all(-1)
    top = np.where(bad, 0.0, np.abs(np.where(np.isfinite(b), b, 0.0)).max(-1))
    e = np.maximum(np.frexp(top)[1] - 1 - 2, -127)           # top = f 2^p, f in [0.5, 1): floor(log2 top) = p - 1
    e = np.where(top == 0.0, -127, e)
    scaled = np.abs(np.where(bad[..., None], 0.0, b)) / np.exp2(e.astype(np.float64))[..., None]
    distance = np.abs(np.minimum(scaled, 6.0)[..., None] - MAGNITUDES)
    nearest = distance.min(-1, keepdims=True)
    tied = distance == nearest                               # of two as near, the even code
    code = np.where(tied.sum(-1) > 1, np.where(tied[..., 0::2].any(-1), 2 * tied[..., 0::2].argmax(-1), tied.argmax(-1)), tied.argmax(-1))
    code = code + 8 * np.signbit(b)
    code[bad] = 0
    return code.reshape(rows, -1).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales):
    """The numbers that codes (one a byte) and scale bytes stand for, rows x width."""
    v = MAGNITUDES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    power = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127.0))
    return (v.reshape(codes.shape[0], -1, 32) * power[..., None]).reshape(codes.shape[0], -1)


def pack(codes, scales):
    """codes rows x width / 2 and scales width / 128 x rows x 4 as the library keeps them."""
    return codes[:, 0::2] | (codes[:, 1::2] << 4), np.ascontiguousarray(scales.reshape(scales.shape[0], -1, 4).transpose(1, 0, 2))


def unpack(codes, scales):
    out = np.empty((codes.shape[0], 2 * codes.shape[1]), np.uint8)
    out[:, 0::2], out[:, 1::2] = codes & 15, codes >> 4
    return out, scales.transpose(1, 0, 2).reshape(codes.shape[0], -1)


def product(x, w, L_A=None, L_B=None):
    """(Z, bound on sums of magnitudes) of x (rows x n) and w (m x n) with the low-rank branch."""
    z, size = x @ w.T, np.abs(x) @ np.abs(w).T
    if L_A is not None:
        z = z + (x @ L_B.T) @ L_A.T
        size = size + (np.abs(x) @ np.abs(L_B).T) @ np.abs(L_A).T
    return z, size


def gated(z):
    m = z.shape[-1] // 2
    with np.errstate(over="ignore"):
        return z[:, :m] / (1.0 + np.exp(-z[:, :m])) * z[:, m:]


def route(logits, top_k, bias=None, sigmoid=False, groups=1, top_groups=1, group_top=1, renormalize=True, scale=1.0):
    """(ids, weights) row by row."""
    l = np.asarray(logits, np.float64).copy()
    l[np.isnan(l)] = -np.inf
    l[l == np.inf] = float(np.finfo(np.float32).max)
    rows, experts = l.shape
    ids, weights = np.full((rows, top_k), -1, np.int64), np.zeros((rows, top_k))
    size = experts // groups
    for t in range(rows):
        off = l[t] == -np.inf
        with np.errstate(over="ignore"):
            if sigmoid:
                s = np.where(off, 0.0, 1.0 / (1.0 + np.exp(-l[t])))
            else:
                s = np.where(off, 0.0, np.exp(l[t] - (l[t].max() if not off.all() else 0.0)))
                s = s / s.sum() if s.sum() > 0 else s
        c = l[t].copy() if bias is None and (groups == 1 or group_top == 1) else s + (0.0 if bias is None else np.asarray(bias, np.float64))
        c[off | np.isnan(c)] = -np.inf
        if groups > 1:
            worth = []
            for i in range(groups):
                best = np.sort(c[i * size:(i + 1) * size])[::-1][:group_top]
                worth.append(best[best > -np.inf].sum() if best[0] > -np.inf else -np.inf)
            taken = sorted(range(groups), key=lambda i: (-worth[i], i))[:top_groups]
            for i in range(groups):
                if i not in taken:
                    c[i * size:(i + 1) * size] = -np.inf
        chosen = [e for e in sorted(range(experts), key=lambda e: (-c[e], e))[:top_k] if c[e] > -np.inf]
        ids[t, :len(chosen)] = chosen
        w = s[chosen]
        if renormalize and w.sum() > 0:
            w = w / w.sum()
        weights[t, :len(chosen)] = w * scale
    return ids, weights


def plan(ids, experts):
    """(offsets, order, place) of ids, rows x top_k."""
    flat = ids.reshape(-1)
    order, offsets, place = [], [0], np.full(flat.size, -1)
    for e in range(experts):
        mine = np.nonzero(flat == e)[0]
        place[mine] = len(order) + np.arange(mine.size)
        order += mine.tolist()
        offsets.append(len(order))
    return np.array(offsets), np.array(order + [-1] * (flat.size - len(order))), place
