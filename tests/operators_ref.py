"""The operators on device tensors from their definitions, in 64 bits on the host (numpy): what the tests compare with."""
import numpy as np

M32 = np.uint64(0xFFFFFFFF)


def philox(counter, key, rounds=10):
    """Philox4x32: counter (..., 4), key (2) of 32-bit words in uint64 arrays."""
    c = [counter[..., i].astype(np.uint64) for i in range(4)]
    k = [np.uint64(key[0]), np.uint64(key[1])]
    for _ in range(rounds):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ k[0], p1 & M32, (p0 >> np.uint64(32)) ^ c[3] ^ k[1], p0 & M32]
        k = [(k[0] + np.uint64(0x9E3779B9)) & M32, (k[1] + np.uint64(0xBB67AE85)) & M32]
    return np.stack(c, -1)


def dropout_keep(rows, cols, p, seed, offset):
    """Which elements are kept, and the factor of those."""
    groups = (cols + 7) // 8
    ctr = np.empty((rows, groups, 4), np.uint64)
    ctr[..., 0] = np.arange(groups, dtype=np.uint64)
    ctr[..., 1] = np.arange(rows, dtype=np.uint64)[:, None]
    ctr[..., 2], ctr[..., 3] = np.uint64(offset & 0xFFFFFFFF), np.uint64(offset >> 32)
    w = philox(ctr, (seed & 0xFFFFFFFF, seed >> 32))
    halves = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1).reshape(rows, groups * 8)[:, :cols]
    t = int(np.floor(65536.0 * float(np.float32(p)) + 0.5))
    return halves >= np.uint64(t), 65536.0 / (65536 - t)


def rows_ref(Z, y, weight=None):
    """part, lp, lse, p (zero where a row takes no part), all in 64 bits."""
    Z = np.asarray(Z, np.float64)
    B, K = Z.shape
    y = np.asarray(y)
    part = (y >= 0) & (y < K)
    if weight is not None:
        part &= np.asarray(weight) != 0
    lp, lse, p = np.zeros(B), np.zeros(B), np.zeros((B, K))
    for i in np.nonzero(part)[0]:
        z = Z[i]
        if np.all(z == -np.inf):
            part[i], lp[i], lse[i] = False, -np.inf, -np.inf
            continue
        with np.errstate(all="ignore"):
            m = z.max()
            e = np.exp(z - m)
            s = e.sum()
            lse[i], p[i] = m + np.log(s), e / s
            others = np.delete(z, y[i])
            if e[y[i]] > 0.5 * s:  # all but certain: the digits are in what is left
                lp[i] = -np.log1p(np.exp(others - z[y[i]]).sum())
            else:
                lp[i] = z[y[i]] - lse[i]
            if np.isnan(z).any():
                lp[i] = lse[i] = np.nan
                p[i] = np.nan
    return part, lp, lse, p


def grad_ref(part, p, y, g):
    """g ([k = y] - p) per row; 1 - p_y as the sum of the others."""
    B, K = p.shape
    d = np.zeros((B, K))
    for i in np.nonzero(part)[0]:
        q = p[i].copy()
        q[y[i]] = 0.0
        d[i] = -g[i] * q
        d[i, y[i]] = g[i] * q.sum()
    return d


def policy_ref(Z, y, old, adv, ref, weight, clip, kl_coef):
    """stats, lp, dZ, g (per row, weighted)."""
    B = len(y)
    w = np.full(B, 1.0 / max(B, 1)) if weight is None else np.asarray(weight, np.float64)
    part, lp, _, p = rows_ref(Z, y, weight)
    stats, g = np.zeros(4), np.zeros(B)
    for i in np.nonzero(part)[0]:
        A, pg, kl, cut, gi = float(adv[i]), 0.0, 0.0, False, 0.0
        if A != 0.0:
            r = np.exp(lp[i] - float(old[i]))
            pg = -min(r * A, min(max(r, 1 - clip[0]), 1 + clip[1]) * A)
            cut = (A > 0 and r > 1 + clip[1]) or (A < 0 and r < 1 - clip[0])
            gi = 0.0 if cut else -r * A
        if ref is not None:
            d = float(ref[i]) - lp[i]
            kl = np.expm1(d) - d
            gi += kl_coef * -np.expm1(d)
        stats += w[i] * np.array([pg + (kl_coef * kl if kl_coef else 0.0), pg, kl, float(cut)])
        g[i] = w[i] * gi
    return stats, lp, grad_ref(part, p, y, g), g


def preference_ref(Z, y, seq, ref, beta, smoothing):
    """stats, s, dZ (rows outside of the sequences: NaN), g per row."""
    part, lp, _, p = rows_ref(Z, y)
    pairs = (len(seq) - 1) // 2
    s = np.array([lp[seq[q]:seq[q + 1]][part[seq[q]:seq[q + 1]]].sum() for q in range(2 * pairs)])
    gain = s - (0.0 if ref is None else np.asarray(ref, np.float64))
    h = gain[0::2] - gain[1::2]
    softplus = lambda v: np.logaddexp(0.0, v)  # noqa: E731
    loss = (1 - smoothing) * softplus(-beta * h) + smoothing * softplus(beta * h)
    slope = beta / pairs * (smoothing / (1 + np.exp(-beta * h)) - (1 - smoothing) / (1 + np.exp(beta * h)))
    g = np.zeros(len(y))
    for q in range(2 * pairs):
        g[seq[q]:seq[q + 1]] = slope[q // 2] * (1 if q % 2 == 0 else -1)
    d = grad_ref(part, p, y, g)
    d[:seq[0]] = np.nan
    d[seq[-1]:] = np.nan
    return np.array([loss.mean(), (h > 0).mean(), beta * gain[0::2].mean(), beta * gain[1::2].mean()]), s, d, g
