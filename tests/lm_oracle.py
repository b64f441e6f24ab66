"""Definitions in 64 bits of the embedding, the token log probabilities and the orthogonalised update, in numpy, and how far a float32
computation of them may be off."""
import numpy as np

U32 = 2.0 ** -24                                     # half a step of float32, relative
QUINTIC = (3.4445, -4.7750, 2.0315)


def half_step(name):
    return {"float32": U32, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[name]


def least(name):
    """Smallest normal number: rounding below it is off by a fixed amount."""
    return {"float32": 2.0 ** -126, "bfloat16": 2.0 ** -126, "float16": 2.0 ** -14}[name]


def embedding_forward(tokens, table, scale):
    there = (tokens >= 0) & (tokens < table.shape[0])
    return np.where(there[:, None], scale * table[np.where(there, tokens, 0)], 0.0)


def holders(n, P, splits):
    """The process that holds each token, -1: none."""
    splits = [p * n // P for p in range(P + 1)] if splits is None else [min(int(s), n) for s in splits]
    held = np.full(n, -1)
    for p in range(P):
        held[splits[p]:splits[p + 1]] = p
    return held


def messages(sums, k):
    """[P][n] as [ceil(n/k)][P][k]."""
    P, n = sums.shape
    S = -(-n // k)
    out = np.zeros((P, S * k))
    out[:, :n] = sums
    return out.reshape(P, S, k).transpose(1, 0, 2)


def embedding_backward(tokens, dy, V, scale, P, k, splits=None):
    """The gradient's messages, and how far float32 sums in any order may be off (a term more than there are additions, for the scale)."""
    n, H = dy.shape
    held = holders(n, P, splits)
    sums, sizes, count = np.zeros((P, V, H)), np.zeros((P, V, H)), np.zeros((P, V, 1))
    for t in range(n):
        if 0 <= tokens[t] < V and held[t] >= 0:
            sums[held[t], tokens[t]] += dy[t]
            sizes[held[t], tokens[t]] += abs(dy[t])
            count[held[t], tokens[t]] += 1
    off = abs(scale) * sizes * (count + 1) * U32
    return messages((scale * sums).reshape(P, V * H), k), messages(off.reshape(P, V * H), k)


def logprobs(x, tokens, scale, top=0):
    """lse, logprob, entropy, top values and tokens of each row, and the sum of p * |z - max z| (which rounding is in proportion to)."""
    z = scale * x
    with np.errstate(invalid="ignore", divide="ignore"):
        m = z.max(1, keepdims=True)
        d = z - np.where(np.isfinite(m), m, 0)
        e = np.exp(d)
        s = e.sum(1)
        lse = m[:, 0] + np.log(s)
        p = np.where(s[:, None] > 0, e / np.where(s > 0, s, 1)[:, None], 0)
        spread = np.where(p > 0, p * -np.where(p > 0, d, 0), 0).sum(1)
        entropy = np.where(s > 0, np.log(np.where(s > 0, s, 1)) + spread, 0)
        bad = ~(z < np.inf).all(1)
        lse, entropy = np.where(bad, np.nan, lse), np.where(bad, np.nan, entropy)
        there = (tokens >= 0) & (tokens < x.shape[1])
        ln_s = np.where(bad, np.nan, np.log(np.where(s > 0, s, 1)))          # z - max z first: 64 bits hold no 1e38 + 1 either
        given = np.where(there, d[np.arange(len(z)), np.where(there, tokens, 0)] - ln_s, 0)
        given = np.where(there & (s == 0) & ~bad, -np.inf, given)
        order = np.argsort(-x, axis=1, kind="stable")[:, :top]
        best = np.take_along_axis(d, order, 1) - ln_s[:, None]
        best = np.where(((s == 0) & ~bad)[:, None], -np.inf, best)
    return lse, given, entropy, best, order, spread


def sum_off(spread, V):
    """How far ln(sum exp) in float32 may be off: each term by its exponent's three roundings (in proportion to |z - max|, whose mean is `spread`)
    and the approximate power's 2^-22, and the additions: at most V of them in a row."""
    return 2.0 ** -22 + U32 * (4 * spread + min(V, 4096) + 64)


def logprobs_backward(x, tokens, scale, lse, entropy, up, de):
    """The logits' gradient from the lse and entropy given, and how far float32 may be off before the result is rounded."""
    z = scale * x
    with np.errstate(invalid="ignore"):
        logp = np.where(np.isneginf(lse)[:, None], -np.inf, z - lse[:, None])
    p = np.exp(logp)
    there = (tokens >= 0) & (tokens < x.shape[1])
    up = np.where(there, up, 0)
    fine = np.where(p > 0, logp, 0)
    g = -p * (up[:, None] + de[:, None] * (fine + entropy[:, None]))
    far = abs(np.where(p > 0, z, 0))
    size = p * (abs(up)[:, None] + abs(de)[:, None] * (far + abs(np.where(np.isfinite(lse), lse, 0))[:, None] + abs(entropy)[:, None]))
    off = scale * size * (2.0 ** -22 + 4 * U32 * (1 + abs(fine) + far)) + scale * 2.0 ** -120
    rows = np.nonzero(there & ~np.isneginf(lse))[0]
    g[rows, tokens[rows]] += up[rows]
    off[rows, tokens[rows]] += scale * abs(up[rows]) * 4 * U32
    return scale * g, off


def _largest_slope(s):
    """The most that a change of X (its root of the sum of squares) grows in a step: the divided differences of the quintic, which is odd, over
    X's singular values s."""
    a, b, c = QUINTIC
    f, slope = a * s + b * s ** 3 + c * s ** 5, a + 3 * b * s ** 2 + 5 * c * s ** 4
    with np.errstate(invalid="ignore", divide="ignore"):
        apart = abs((f[:, None] - f) / (s[:, None] - s))
        both = abs((f[:, None] + f) / (s[:, None] + s))
    return max(np.nanmax(np.where(np.isfinite(apart), apart, 0)), np.nanmax(np.where(np.isfinite(both), both, 0)), abs(slope).max(), abs(a))\
        if s.min() < 0.1 else max(np.nanmax(np.where(abs(s[:, None] - s) > 1e-6, apart, 0)), np.nanmax(both), abs(slope).max())


def muon(p, m, g, there, lr, lr_scale, decay, mu, nesterov, eps, steps, products):
    """Weights, momentum and the update X of one matrix, and how far X may be off (the root of the sum of squares, to first order); `there`: the
    elements that were delivered.

    A step's operands are X, A without its diagonal and B with 3.4445 on its diagonal, each entry off by half a step of float16 (u) or, of two float16 numbers, of their
    22 bits. X's change grows by the step's slope; A's passes through b + 2 c |A|, then like B's through |X| (largest singular values). The sums
    are float32, 16 products at a time: as many additions in a row as there are sixteens (and a few), each off by 2^-24 of the sum of sizes."""
    m1 = np.where(there, mu * m + g, m)
    u = np.where(there, g + mu * m1 if nesterov else m1, m)
    l = lr * lr_scale
    if not there.any():
        return p, m1, np.zeros_like(p), 0.0
    x = u / (np.sqrt((u * u).sum()) + eps)
    turned = x.shape[0] > x.shape[1]
    x = x.T if turned else x
    a, b, c = QUINTIC
    h = 2.0 ** -11 if products == 16 else 2.0 ** -22
    norm = np.linalg.norm
    rows, cols = x.shape
    off = h * norm(x) + 4 * U32 * norm(x)
    for _ in range(steps):
        q = x @ x.T
        r = b * q + c * (q @ q)
        s = np.linalg.svd(x, compute_uv=False)
        top = s.max()
        q_off = h * norm(q - np.diag(np.diag(q))) + (cols / 16 + 4) * U32 * norm(x) ** 2
        r_off = h * norm(r + a * np.eye(rows)) + q_off * (abs(b) + 2 * c * top ** 2) + c * (rows / 16 + 4) * U32 * norm(q) ** 2
        y = a * x + r @ x
        off = _largest_slope(s) * off + r_off * top + (rows / 16 + 4) * U32 * norm(r) * norm(x) + h * norm(y)
        x = y
    x = x.T if turned else x
    return p * (1 - l * decay) - l * x, m1, x, off
