"""Orthogonalised updates with the roundings that the kernels make, on the host (numpy): fp16 operands in one or two parts, fp32 sums and everything else in
fp32.  The sums' order differs from the kernels', so single results do, but not how far they are from 64 bits on the whole."""
import numpy as np

from more_operators_ref import COEF, _triples, ortho_ref

F = np.float32
SX, SA, SB = 4096.0, 256.0, 1024.0


def parts(x, scale=1.0):
    y = (x * F(scale)).astype(F)
    hi = y.astype(np.float16).astype(F)
    return hi, (y - hi).astype(np.float16).astype(F)


def product(p, q, planes=2):
    """Rows of p times columns of q: high x high, and with two planes high x low and low x high."""
    s = p[0] @ q[0]
    return s if planes == 1 else ((s + p[0] @ q[1]) + p[1] @ q[0]).astype(F)


def start(G, eps):
    G = np.asarray(G, np.float64)
    X = G.T if G.shape[0] > G.shape[1] else G
    return parts((X * (SX / (np.sqrt((X * X).sum()) + float(F(eps))))).astype(F))


def tiled(G, steps=5, coef=COEF, eps=1e-7, planes=2, without=()):
    """Matrices of more than 128 rows and columns.  without: "low" of the operands, or "linear" (the low part of a X), as a kernel that lost them would be."""
    x = start(G, eps)
    C = _triples(coef, steps)
    if "low" in without:
        planes = 1
    for k, (a, b, c) in enumerate(F(C)):
        turned = tuple(p.T.copy() for p in x)
        s = product(x, turned, planes)
        d = (np.diag(s) * F(1 / (SX * SX))).astype(F)
        f = parts((s - np.diag(np.diag(s))) * F(SA / (SX * SX)))
        sq = (product(f, f, planes) * F(1 / (SA * SA))).astype(F)  # (f is symmetric)
        fv = ((f[0] + f[1] if planes == 2 else f[0]) * F(1 / SA)).astype(F)
        e = (c * (d * d + np.diag(sq)) + b * d).astype(F)
        h = (c * ((d[:, None] + d[None, :]) * fv + sq) + b * fv).astype(F)
        h = parts((h - np.diag(np.diag(h))) * F(SB))
        linear = x[0] if "linear" in without else x[0] + x[1]
        y = ((a + e)[:, None] * linear + product(h, x, planes) * F(1 / SB)).astype(F)
        if k + 1 < steps:
            x = parts(y)
    y = (y * F(1 / SX)).astype(np.float64)
    return y.T if np.shape(G)[0] > np.shape(G)[1] else y


def _plan(steps, coef, limit):
    def scale(most, s=4096.0):
        while s > 1.0 and most * s > 16384.0:
            s *= 0.5
        return s
    out, top, last, factors = [], 1.002, 1.002, 1.0
    for k, (a, b, c) in enumerate(_triples(coef, steps)):
        x = top * np.arange(257) / 256
        p = np.abs(a + b * x ** 2 + c * x ** 4)
        if k:
            out[-1]["end"] = factors * p.max() > limit
            factors = 1.0 if out[-1]["end"] else factors
        factors *= max(1.0, p.max())
        out.append({"a": F(a), "b": F(b), "c": F(c), "sa": scale(top * max(top, last)), "sp": scale(p.max()), "sq": scale(factors), "end": k + 1 == steps})
        last, top = top, 1.002 * (p * x).max()
    return out


def small(G, steps=5, coef=COEF, eps=1e-7, limit=1.0):
    """Matrices of up to 128 rows: runs of steps on A = X X^T, of which the product of the largest factors is at most limit."""
    def rows(M, s):  # off the diagonal in two parts, the diagonal in fp32
        d = np.diag(M).copy()
        return (*parts(M - np.diag(d), s), d)

    def times(r, s, M, t):
        return (r[2][:, None] * M + product(r, parts(M, t)) * F(1 / (s * t))).astype(F)

    x, A, plan = start(G, eps), None, _plan(steps, coef, limit)
    for k, s in enumerate(plan):
        if A is None:
            A, Q = (product(x, tuple(p.T.copy() for p in x)) * F(1 / (SX * SX))).astype(F), None
        P = (s["b"] * A + s["c"] * times(rows(A, s["sa"]), s["sa"], A, s["sa"])).astype(F)
        P[np.diag_indices(len(P))] += s["a"]
        rp = rows(P, s["sp"])
        Q = P if Q is None else times(rp, s["sp"], Q, plan[k - 1]["sq"])
        if not s["end"]:
            A = times(rp, s["sp"], times(rp, s["sp"], A, s["sa"]), plan[k + 1]["sa"])
        else:
            r = rows(Q, s["sq"])
            y = (r[2][:, None] * (x[0] + x[1]) + product(r, x) * F(1 / s["sq"])).astype(F)
            x, A = parts(y), None
    y = (y * F(1 / SX)).astype(np.float64)
    return y.T if np.shape(G)[0] > np.shape(G)[1] else y


def with_values(rows, cols, s, rng):
    """A matrix (fp32 values) of these singular values and random directions."""
    m = min(rows, cols)
    q, _ = np.linalg.qr(rng.standard_normal((m, m)))
    p, _ = np.linalg.qr(rng.standard_normal((max(rows, cols), m)))
    G = (q * s) @ p.T
    return (G.T if rows > cols else G).astype(np.float32).astype(np.float64)


def off(got, G, **how):
    """Distance from the definition in 64 bits, of its norm."""
    want = ortho_ref(G, **how)
    return float(np.linalg.norm(got - want) / np.linalg.norm(want))


def few_rows():
    """Lists of small matrices of one shape whose smaller singular values are a fifth of the largest: a step brings them near 0 (where a s + b s^3 + c s^5 crosses it),
    and what runs of two steps lose there is four times what single steps do."""
    lists = []
    for m, n in [(2, 2), (2, 5), (5, 2), (4, 4), (3, 30), (8, 40)]:
        rng = np.random.default_rng(100 * m + n)
        k = min(m, n)
        lists.append([with_values(m, n, np.r_[1.0, np.full(k - 1, 0.2)], rng) for _ in range(64)])
    return lists


def two_decades(rows, cols):
    return with_values(rows, cols, np.logspace(0, -2, min(rows, cols)), np.random.default_rng(rows + cols))


LARGER = [(134, 176), (300, 200), (257, 900), (520, 513)]
SMALLER = [(20, 60), (64, 100), (128, 300), (600, 40)]
rms = lambda v: float(np.sqrt(np.mean(np.square(v))))  # noqa: E731
