"""The AdamW step in plain float32 (numpy), every operation rounded once: the bits that the kernels' states must have."""
import numpy as np

F = np.float32
BLOCK = 256
TINY = F(2.0 ** -126)


def factors(beta1, beta2, step):
    """beta1, beta2, 1 - beta1, 1 - beta2 and both bias corrections as the call rounds them."""
    return F(beta1), F(beta2), F(1 - beta1), F(1 - beta2), F(1 / (1 - beta1 ** step)), F(1 / np.sqrt(1 - beta2 ** step))


def moments(g, m, v, beta1, beta2, step):
    """New m and v."""
    b1, b2, r1, r2, _, _ = factors(beta1, beta2, step)
    return m * b1 + g * r1, v * b2 + (g * g) * r2


def weights(p, m, v, lr, beta1, beta2, eps, step, decay=0.0):
    """New weights from the new m and v in 64 bits, and the bound of what float32 with an approximate root and quotient (each 2^-23
    off at most) makes of them: the factors' roundings (3 half units), root and quotient (4), three products and a sum (4), rounded
    up to 16 of the move; two roundings of p's factor, one product and one sum."""
    _, _, _, _, c1, c2 = (np.float64(x) for x in factors(beta1, beta2, step))
    lr = np.float64(F(lr))
    move = m.astype(np.float64) / (np.sqrt(v.astype(np.float64)) * c2 + np.float64(F(eps))) * (lr * c1)
    out = p.astype(np.float64) * (1 - lr * np.float64(F(decay))) - move
    return out, 2.0 ** -24 * (16 * np.abs(move) + 4 * np.abs(p.astype(np.float64)))


def nearest_root(x, most):
    """The whole number c with (c - 1/2)^2 <= x < (c + 1/2)^2, at most `most`."""
    x = x.astype(np.float64)
    c = np.floor(np.sqrt(x) + 0.5)
    c = np.where((c - 0.5) ** 2 > x, c - 1, c)
    c = np.where((c + 0.5) ** 2 <= x, c + 1, c)
    return np.clip(c, 0, most)                                       # at c = 0 the lower border says nothing


def squares_of_codes(m, v):
    """x = code^2 before it is rounded for both states, and the blocks' scales."""
    m, r = m.reshape(-1, BLOCK), np.sqrt(v).reshape(-1, BLOCK)
    ms, vs = np.maximum(np.abs(m).max(1), TINY), np.maximum(r.max(1), TINY)
    return np.abs(m) * (F(1) / ms)[:, None] * F(16129), r * (F(1) / vs)[:, None] * F(65025), ms, vs


def encode(m, v):
    """Codes of whole blocks, nearest, and their scales."""
    xm, xv, ms, vs = squares_of_codes(m, v)
    cm, cv = nearest_root(xm, 127), nearest_root(xv, 255)
    cv = np.where(v.reshape(-1, BLOCK) > 0, np.maximum(cv, 1), cv)
    return np.where(m.reshape(-1, BLOCK) < 0, -cm, cm).astype(np.int8).ravel(), cv.astype(np.uint8).ravel(), ms, vs


def decode(m, v, ms, vs):
    """What codes stand for, in float32."""
    c, d = m.astype(F).reshape(-1, BLOCK), v.astype(F).reshape(-1, BLOCK)
    r = d * d * (vs * (F(1) / F(65025)))[:, None]
    return (c * np.abs(c) * (ms * (F(1) / F(16129)))[:, None]).ravel(), (r * r).ravel()


def dither(places, step):
    """u of each place in the states' arrays."""
    return (((places.astype(np.uint64) * 0x6A09E667 + step * 0x9E3779B9) & 0xFFFFFFFF) >> 9).astype(np.float64) * 2.0 ** -23


def dithered_root(x, u, most, power):
    """The whole number c with c^2 <= x < (c + 1)^2, or c + 1 where x lies more than u of the way from c to it, by what they stand for (the
    codes' square, or with power 4 their fourth power)."""
    x = x.astype(np.float64)
    c = np.floor(np.sqrt(x))
    part = (x ** (power / 2) - c ** power) / ((c + 1) ** power - c ** power)
    return np.minimum(np.where(part > u, c + 1, c), most)
