"""The training operators' definitions in 64 bits (numpy), and the error bounds that their float32 arithmetic may have.

U is half a unit in the last place of float32; ROUND the same for each output type. A sum of n float32 terms in any order has
an error of at most (n - 1) U times the sum of the terms' sizes; the kernels add in at least 32 chains, joined by a tree, so
a row of H elements takes at most H / 32 + 40 additions one after the other."""
import numpy as np

U = 2.0 ** -24
ROUND = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
SMALL = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}      # spacing of the smallest numbers
BLOCK = 256
TINY = 2.0 ** -126


def chain(H):
    return H / 32 + 40


def norm_forward(x, gamma, beta, eps):
    """y, mean, rstd and the bounds of their errors before y is rounded to its type."""
    mean = x.mean(1, keepdims=True)
    var = ((x - mean) ** 2).mean(1, keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    xh = (x - mean) * rstd
    y = xh * gamma + beta
    n, size = chain(x.shape[1]), np.abs(x).mean(1, keepdims=True)
    off_mean = n * U * size
    # the variance: its terms' rounding, the sum's, and the mean's own error squared (first order cancels in the sum)
    off_rstd = rstd * (n * U + 4 * U) + rstd ** 3 * off_mean ** 2
    off_y = np.abs(gamma) * (rstd * (off_mean + U * np.abs(x - mean)) + np.abs(x - mean) * off_rstd + 2 * U * np.abs(xh)) + 2 * U * (np.abs(y) + np.abs(beta))
    return (y, mean[:, 0], rstd[:, 0]), (off_y, off_mean[:, 0], off_rstd[:, 0])


def holders(rows, P, splits):
    """First and last + 1 row of each process."""
    if splits is None:
        return [(p * rows // P, (p + 1) * rows // P) for p in range(P)]
    s = np.minimum(np.asarray(splits), rows)
    return [(int(s[p]), int(max(s[p], s[p + 1]))) for p in range(P)]


def messages(sums, k):
    """[P][H] as [ceil(H/k)][P][k], filled up with zeros."""
    P, H = sums.shape
    out = np.zeros((P, -(-H // k) * k))
    out[:, :H] = sums
    return out.reshape(P, -1, k).transpose(1, 0, 2)


def norm_backward(dy, x, gamma, mean, rstd, P, k, splits):
    """dx, dgamma, dbeta (messages) and the bounds of their errors before dx is rounded to its type."""
    mean, rstd = mean[:, None], rstd[:, None]
    xh = (x - mean) * rstd
    a = dy * gamma
    c1, c2 = a.mean(1, keepdims=True), (a * xh).mean(1, keepdims=True)
    dx = rstd * (a - c1 - xh * c2)
    n = chain(x.shape[1]) + 8
    off_dx = rstd * (n * U * (np.abs(a).mean(1, keepdims=True) + np.abs(xh) * np.abs(a * xh).mean(1, keepdims=True)) +
                     8 * U * (np.abs(a) + np.abs(c1) + np.abs(xh * c2)))
    outs = []
    for terms in (dy * xh, dy):
        total = np.stack([terms[lo:hi].sum(0) for lo, hi in holders(len(x), P, splits)])
        off = np.stack([(hi - lo + 8) * U * np.abs(terms[lo:hi]).sum(0) for lo, hi in holders(len(x), P, splits)])
        outs.append((messages(total, k), messages(off, k)))
    return (dx, outs[0][0], outs[1][0]), (off_dx, outs[0][1], outs[1][1])


def assert_within(got, want, off, dtype="float32", what=""):
    """got (rounded to dtype) against want, whose float32 error is at most off."""
    got = np.asarray(got, dtype=np.float64)
    room = off + ROUND[dtype] * (np.abs(want) + off) + SMALL[dtype]
    bad = ~(np.abs(got - want) <= room)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} outside, worst {np.nanmax(np.abs(got - want) / room):.3g} of its room, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}"


def shares(status, k, n):
    """1 / included for each element, 0 where its message was not delivered."""
    if status is None:
        return np.ones(n)
    ok = ((status[:, 0] & 0xFF) == 0) & (status[:, 1] > 0)
    return np.repeat(np.where(ok, 1.0 / np.maximum(status[:, 1], 1), 0.0), k)[:n]


def decode(m, v, ms, vs):
    """8-bit states as numbers."""
    m, v = m.astype(np.float64).reshape(-1, BLOCK), v.astype(np.float64).reshape(-1, BLOCK)
    return (m * np.abs(m) * ms[:, None] / 127 ** 2).ravel(), ((v * v * vs[:, None] / 255 ** 2) ** 2).ravel()


def adamw(p, g, m, v, lr, beta1, beta2, eps, step, decay, share, scale=1.0):
    """New p, m, v of one tensor, and the bounds of their errors in float32."""
    g = g * share * scale
    there = share > 0
    m1, v1 = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    mh, root = m1 / (1 - beta1 ** step), np.sqrt(v1 / (1 - beta2 ** step))
    move = np.divide(lr * mh, root + eps, out=np.zeros_like(m), where=(root + eps) > 0)
    p1 = p - lr * decay * p - move
    off_m = 6 * U * (np.abs(beta1 * m) + np.abs((1 - beta1) * g)) + 2.0 ** -147
    off_v = 10 * U * v1 + 2.0 ** -147
    # the move: its own roundings (the constants' among them), what m's error and what v's error (half of it, under the root) make of it
    off_p = 4 * U * np.abs(p) + 16 * U * np.abs(move) + np.divide(lr * off_m / (1 - beta1 ** step), root + eps, out=np.zeros_like(m), where=(root + eps) > 0) + 2.0 ** -147
    keep = lambda new, old: np.where(there, new, old)
    none = lambda off: np.where(there, off, 0.0)
    return (keep(p1, p), keep(m1, m), keep(v1, v)), (none(off_p), none(off_m), none(off_v))
