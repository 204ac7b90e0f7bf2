"""Dropout, adapters and the softmax loss in numpy and 64 bits, from their definitions (test infrastructure only)."""
import numpy as np


def philox(seed, block, place):
    """Philox4x32-10 in Python's whole numbers: four 32-bit words."""
    c, k = [block & 0xFFFFFFFF, block >> 32, place & 0xFFFFFFFF, place >> 32], [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p, q = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(q >> 32) ^ c[1] ^ k[0], q & 0xFFFFFFFF, (p >> 32) ^ c[3] ^ k[1], p & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def draws(count, seed, place):
    """The 16-bit numbers of elements 0 .. count - 1."""
    with np.errstate(over="ignore"):
        b = np.arange((count + 7) // 8, dtype=np.uint64)
        m, h = np.uint64(0xFFFFFFFF), np.uint64(32)
        c = [b & m, b >> h, np.full_like(b, place & 0xFFFFFFFF), np.full_like(b, place >> 32)]
        k = [seed & 0xFFFFFFFF, seed >> 32]
        for _ in range(10):
            p, q = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
            c = [(q >> h) ^ c[1] ^ np.uint64(k[0]), q & m, (p >> h) ^ c[3] ^ np.uint64(k[1]), p & m]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    words = np.stack(c, 1)
    return np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], 2).reshape(-1)[:count].astype(np.int64)


def border(p):
    return int(np.floor(float(np.float32(p)) * 65536 + 0.5))


def mask(shape, p, seed, place):
    """What dropout multiplies by, in the shape of a dense tensor."""
    t = border(p)
    if t == 0:
        return np.ones(shape)
    if t == 65536:
        return np.zeros(shape)
    return (draws(int(np.prod(shape)), seed, place) >= t).reshape(shape) * (65536.0 / (65536 - t))


def adapter_fwd(x, w, bias, a, b, ids, scales, m):
    """y, inner of x (pixels, c_in); ids: one per pixel; m: dropout's mask, like x."""
    y = x @ w.T + (0 if bias is None else bias)
    inner = np.zeros((len(x), a.shape[1]))
    for i, k in enumerate(ids):
        if 0 <= k < len(a):
            inner[i] = scales[k] * (a[k] @ (x[i] * m[i]))
            y[i] = y[i] + b[k] @ inner[i]
    return y, inner


def adapter_bwd(dy, x, w, a, b, ids, scales, m, inner):
    dx, da, db = dy @ w, np.zeros(a.shape), np.zeros(b.shape)
    for i, k in enumerate(ids):
        if 0 <= k < len(a):
            u = scales[k] * (b[k].T @ dy[i])
            dx[i] += m[i] * (a[k].T @ u)
            da[k] += np.outer(u, x[i] * m[i])
            db[k] += np.outer(dy[i], inner[i])
    return dx, da, db


def softmax_loss(z, labels, smoothing, mean):
    """loss, row_loss, dz."""
    rows, c = z.shape
    row, dz = np.zeros(rows), np.zeros(z.shape)
    has = [0 <= t < c for t in labels]
    g = 1.0 / max(sum(has), 1) if mean else 1.0
    for i in range(rows):
        if not has[i]:
            continue
        top = z[i].max()
        lse = top + np.log(np.exp(z[i] - top).sum())
        target = np.full(c, smoothing / c)
        target[labels[i]] += 1 - smoothing
        row[i] = lse - (target[target > 0] * z[i][target > 0]).sum()
        dz[i] = g * (np.exp(z[i] - lse) - target)
    return row.sum() * g, row, dz
