"""Orthogonalised updates and scores of rows of logits from their definitions, in 64 bits on the host (numpy)."""
import numpy as np

COEF = (3.4445, -4.7750, 2.0315)


def _triples(coef, steps):
    c = np.asarray(np.float32(coef), np.float64).reshape(-1, 3)  # as the calls take them
    return np.broadcast_to(c, (steps, 3)) if len(c) == 1 else c


def ortho_ref(G, steps=5, coef=COEF, eps=1e-7):
    G = np.asarray(G, np.float64)
    X = G.T if G.shape[0] > G.shape[1] else G
    with np.errstate(all="ignore"):
        X = X / (np.sqrt((X * X).sum()) + float(np.float32(eps)))
        for a, b, c in _triples(coef, steps):
            A = X @ X.T
            X = a * X + (b * A + c * (A @ A)) @ X
    return X.T if G.shape[0] > G.shape[1] else X


def _high(x, scale):
    return (x * scale).astype(np.float16).astype(np.float64) / scale


def _both(x, scale):
    hi = (x * scale).astype(np.float16).astype(np.float64)
    return (hi + (x * scale - hi).astype(np.float16).astype(np.float64)) / scale


def ortho_rounded(G, steps=5, coef=COEF, eps=1e-7, planes=1):
    """The same with what is stored in 11 or 22 bits rounded to them, and nothing else: the linear term in 22, diagonals not at all."""
    G = np.asarray(G, np.float64)
    flip = G.shape[0] > G.shape[1]
    X = G.T if flip else G
    X = _both(X / (np.sqrt((X * X).sum()) + float(np.float32(eps))), 4096)
    q = _high if planes == 1 else _both
    for k, (a, b, c) in enumerate(_triples(coef, steps)):
        Xq = q(X, 4096)
        A = Xq @ Xq.T
        d = np.diag(A).copy()
        F = q(A - np.diag(d), 256)
        B = b * F + c * (F @ F + (d[:, None] + d[None, :]) * F)
        e = b * d + c * (d * d + np.diag(F @ F))
        H = q(B - np.diag(np.diag(B)), 1024)
        X = (a + e)[:, None] * X + H @ Xq
        if k + 1 < steps:
            X = _both(X, 4096)
    return X.T if flip else X


def runs_of(coef, steps, limit):
    """Where runs of steps end that are made on A = X X^T alone: the product of the largest factors |a + b s^2 + c s^4| is at most limit."""
    ends, top, product = [False] * steps, 1.002, 1.0
    for k, (a, b, c) in enumerate(_triples(coef, steps)):
        x = top * np.arange(257) / 256
        p = np.abs(a + b * x ** 2 + c * x ** 4)
        if k and product * p.max() > limit:
            ends[k - 1], product = True, 1.0
        product *= max(1.0, p.max())
        top = 1.002 * (p * x).max()
    ends[-1] = True
    return ends


def ortho_runs(G, steps=5, coef=COEF, eps=1e-7, limit=12.0):
    """The definition by runs of steps on A, with everything rounded to 22 bits as it is stored."""
    G = np.asarray(G, np.float64)
    flip = G.shape[0] > G.shape[1]
    X = G.T if flip else G
    X = _both(X / (np.sqrt((X * X).sum()) + float(np.float32(eps))), 4096)
    I, A = np.eye(len(X)), None
    for (a, b, c), end in zip(_triples(coef, steps), runs_of(coef, steps, limit)):
        if A is None:
            A, Q = X @ X.T, None
        Aq = _both(A, 4096)
        P = a * I + b * A + c * (Aq @ Aq)
        Pq = _both(P, 4096)
        Q = P if Q is None else Pq @ _both(Q, 32)
        if not end:
            A = Pq @ _both(Pq @ Aq, 4096)
        else:
            X, A = _both(_both(Q, 32) @ X, 4096), None
    return X.T if flip else X


def fp32_sums(G, steps=5, coef=COEF, eps=1e-7, limit=0.0):
    """What the fp32 sums of the products may add to the result, in Frobenius norm.  A sum of n terms in chains of n / 32 rounds about that often
    plus a few times; roundings of many entries are independent, so those of a matrix add up like sqrt(n / 32 + 8) 2^-24 of its norm, 4
    times that at most.  A later step multiplies what is there by at most max |p'| = p'(0) = a (usual steps; the divided
    differences of the odd p bound the derivative of the matrix function in this norm).  In a run of steps on A (limit) what A is off by goes on to the next A by at most the slope of
    l p(l)^2."""
    G = np.asarray(G, np.float64)
    X = G.T if G.shape[0] > G.shape[1] else G
    norm = np.sqrt((X * X).sum()) + float(np.float32(eps))
    s = np.linalg.svd(X / norm, compute_uv=False)
    m, n = X.shape
    u = 4 * np.sqrt(max(m, n) / 32 + 8) * 2.0 ** -24
    off, carried = 2.0 ** -24, 0.0
    for (a, b, c), end in zip(_triples(coef, steps), runs_of(coef, steps, limit)):
        top, size = s.max(), np.sqrt((s * s).sum())
        slope = np.abs(a + 3 * b * np.linspace(0, top, 100) ** 2 + 5 * c * np.linspace(0, top, 100) ** 4).max()
        dA = u * top * size + carried
        at = np.linspace(0, top, 100) ** 2
        p, dp = a + b * at + c * at ** 2, b + 2 * c * at
        carried = 0.0 if end else np.abs(p * p + 2 * at * p * dp).max() * dA
        dB = (abs(b) + 2 * abs(c) * top ** 2) * dA + u * (abs(b) + abs(c) * top ** 2) * top * size
        s = np.abs(a * s + b * s ** 3 + c * s ** 5)
        off = slope * off + dB * top + 2 * u * (abs(a) + abs(b) * top ** 2 + abs(c) * top ** 4) * size
    return off


def muon_ref(W, G, M, lr, momentum=0.95, nesterov=True, weight_decay=0.0, scale=1.0, steps=5, coef=COEF, eps=1e-7, ortho=ortho_ref):
    """(W, M, O) after a step."""
    f = lambda v: float(np.float32(v))  # noqa: E731
    W, G, M = (np.asarray(t, np.float64) for t in (W, G, M))
    M = f(momentum) * M + G
    O = ortho(G + f(momentum) * M if nesterov else M, steps, coef, eps)
    return W - f(lr) * f(weight_decay) * W - f(lr) * f(scale) * O, M, O


def scores_ref(Z, y, top):
    """part, logp, lse, entropy, classes, their log-probabilities, p, log p: all in 64 bits, row by row from the definitions."""
    Z = np.asarray(Z, np.float64)
    B, K = Z.shape
    part = np.ones(B, bool) if y is None else (np.asarray(y) >= 0) & (np.asarray(y) < K)
    logp, lse, H = np.zeros(B), np.zeros(B), np.zeros(B)
    classes, tops = np.full((B, top), -1), np.zeros((B, top))
    p, lp = np.zeros((B, K)), np.zeros((B, K))
    for i in np.nonzero(part)[0]:
        z = Z[i]
        order = np.argsort(-np.where(np.isnan(z), -np.inf, z), kind="stable")
        order = order[(z[order] > -np.inf)][:top]
        classes[i, :len(order)] = order
        tops[i] = -np.inf
        if np.isnan(z).any() or (z == np.inf).any():
            logp[i] = lse[i] = H[i] = p[i] = lp[i] = np.nan
            tops[i, :len(order)] = np.nan
            continue
        if (z == -np.inf).all():
            logp[i] = lse[i] = -np.inf
            lp[i] = -np.inf
            continue
        w = int(np.argmax(z))
        d = z - z[w]
        e = np.exp(d)
        o = np.delete(e, w).sum()
        lp[i] = d - np.log1p(o)
        p[i] = e / (1 + o)
        lse[i] = z[w] + np.log1p(o)
        few = np.where(e > 0, d, 0.0)
        H[i] = np.log1p(o) - (e * few).sum() / (1 + o)
        tops[i, :len(order)] = lp[i, order]
        if y is not None:
            logp[i] = lp[i, y[i]]
    return part, logp, lse, H, classes, tops, p, lp


def scores_grad_ref(ref, y, g_logp, g_entropy):
    """From what scores_ref gives; 1 - p_y as the sum of the others."""
    part, _, _, H, _, _, p, lp = ref
    B, K = p.shape
    d = np.zeros((B, K))
    for i in range(B):
        gl, gh = (0.0 if g is None else float(g[i]) for g in (g_logp, g_entropy))
        if not part[i] or (gl == 0 and gh == 0) or (p[i] == 0).all():
            continue
        d[i] = -gl * p[i] - gh * p[i] * (np.where(p[i] == 0, 0.0, lp[i]) + H[i])
        if gl:
            q = p[i].copy()
            q[y[i]] = 0
            d[i, y[i]] += gl * (p[i, y[i]] + q.sum())
    return d
