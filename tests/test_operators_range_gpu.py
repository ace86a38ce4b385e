"""Log-probabilities and the losses on logits of any finite size: rows masked throughout with a large negative value, rows far from
0, one class far above the others.

Tolerances, with u = 2^-24: (z - max) is rounded, its product with log2 e, the exponential twice: an exponential of T = max - z is
off by (2 T + 4) u relative, where T <= 104 counts (below that it is 0 in fp32).  eps(K) adds the sum's chains as in the tests of
ordinary logits: K / 64 + 64 terms and a tree of 16.  log2 e is off by 0.22 u, the result rounded: 1.25 u of a log-probability.
Exponentials below 2^-126 are flushed: 2^-125 absolute.  A bf16 result adds 2^-8 relative.
A gradient is a product of fp32 values: where |g p| < 2^-126 (a pair whose loss is flat has g of 1e-33 and less), it is not a normal
value, and is 0 or off by up to 2^-126 itself, however exact g and p are.
"""
import numpy as np
import pytest
import torch

import operators_ref as ref
import paper_2004_08771_amd as hb

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -125
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = [1e4, 1e9, 1e10, 1e12, 1e20, 1e30, 3.3e38]
LEVELS = [s * c for c in SIZES for s in (-1.0, 1.0)]
KINDS = 6
# (rows, classes): every number of lanes a row, and rows in chunks (64 rows and less of more than 32768 classes, and rows too long for registers)
SHAPES = [(84, 4), (84, 7), (84, 16), (84, 40), (84, 100), (84, 255), (84, 510), (84, 983), (84, 2049), (84, 4100), (84, 8200), (84, 16385),
          (84, 33000), (60, 33000), (36, 70001), (84, 82003), (24, 300007)]


def eps(K):
    return (2 * 17 + 2 * np.log(K) + 4 + K / 64 + 64 + 16) * U


def rows(B, K, dtype, rng):
    """B rows over all levels and kinds, as stored, and a chosen class each."""
    z, y = np.empty((B, K), np.float32), rng.integers(0, K, B).astype(np.int32)
    low = float(torch.finfo(TYPES[dtype]).min)
    for i in range(B):
        c = np.float32(LEVELS[(3 * (i // KINDS) + 4) % len(LEVELS)])
        kind, other = i % KINDS, (y[i] + 1 + rng.integers(0, max(1, K - 1))) % K
        if kind == 0:      # masked throughout, or one value throughout
            z[i] = c
        elif kind == 1:    # one class far from the rest: the chosen one
            z[i] = 0.0
            z[i, y[i]] = c
        elif kind == 2:    # ... another one
            z[i] = 0.0
            z[i, other] = c
        elif kind == 3:    # ordinary logits as far from 0 as they can be told apart
            z[i] = np.clip(c, -1e4, 1e4) + rng.standard_normal(K)
        elif kind == 4:    # a tie of the chosen class and another, the rest masked
            z[i] = low
            z[i, y[i]] = z[i, other] = c
        else:              # neighbouring values
            z[i] = c * (1 + 2.0 ** -7 * rng.integers(0, 3, K)) if abs(c) < 1e38 else c
    return torch.as_tensor(z).to(TYPES[dtype]).double().numpy(), y


def softmax_ref(z, y):
    """lp, lse, p in 64 bits, from differences to the maximum."""
    B, K = z.shape
    at = np.arange(B)
    m = z.max(1)
    d = z - m[:, None]
    e = np.exp(d)
    s = e.sum(1)
    chosen = e[at, y]
    e[at, y] = 0.0
    others = e.sum(1)
    e[at, y] = chosen
    with np.errstate(all="ignore"):
        lp = np.where(chosen > others, -np.log1p(others / chosen), d[at, y] - np.log(s))
    return lp, m + np.log(s), e / s[:, None], m


def device(z, dtype):
    return torch.as_tensor(z).to(TYPES[dtype]).cuda()


def vec(a, dtype=torch.float32):
    return torch.as_tensor(np.asarray(a)).to(dtype).cuda()


def ws(B, pairs=0):
    return torch.full((hb.choice_workspace_bytes(B, pairs),), 0xFF, dtype=torch.uint8, device="cuda")


def near(got, want, tol, what):
    got = got.double().cpu().numpy() if torch.is_tensor(got) else got
    with np.errstate(over="ignore"):
        want32 = want.astype(np.float32).astype(np.float64)
    past = np.isinf(want32)                      # beyond fp32
    assert np.array_equal(got[past], want32[past]), what
    off = np.abs(got[~past] - want[~past]) - np.broadcast_to(tol, want.shape)[~past]
    assert not (~(off <= 0)).any(), f"{what}: {int((~(off <= 0)).sum())} of {off.size} off, by {np.nanmax(off):.3g}"


def lp_tol(lp, K):
    return eps(K) + 1.25 * U * np.abs(lp) + TINY


def unit_grad(p, y):
    """[k = y] - p, 1 - p_y as the sum of the others."""
    at = np.arange(len(y))
    u = -p
    u[at, y] = 0.0
    u[at, y] = -u.sum(1)
    return u


def grad_tol(unit, z, m, g, K, dtype, g_off=0.0):
    rel = eps(K) + (2 * np.minimum(m[:, None] - z, 104.0) + 16) * U
    tol = np.abs(g)[:, None] * (rel * np.abs(unit) + TINY) + np.abs(unit) * np.reshape(g_off, (-1, 1)) + 2.0 ** -126
    return tol + (2.0 ** -8 * np.abs(unit * g[:, None]) + 2.0 ** -133 if dtype == "bf16" else 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K", SHAPES)
def test_logprob_of_logits_of_any_size(B, K, dtype):
    z, y = rows(B, K, dtype, np.random.default_rng(B + K))
    lp, lse, _, _ = softmax_ref(z, y)
    a, b = torch.full((B,), 7.0, device="cuda"), torch.full((B,), 7.0, device="cuda")
    hb.logprob(device(z, dtype), vec(y, torch.int32), a, b, ws=ws(B))
    near(a, lp, lp_tol(lp, K), "logp")
    near(b, lse, eps(K) + 1.25 * U * np.abs(lse), "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K", SHAPES + [(84, 9001), (300, 20011)])
def test_gradient_of_log_probabilities_of_any_size(B, K, dtype):
    """exp(z - lse) from lse or z_y - logp, n the smaller of |logp| and |lse|: what n is rounded to, what is subtracted from it and its
    product with log2 e add 4 u n to an exponent.  Where that is not small the probability is still at most 1 - p_y."""
    rng = np.random.default_rng(B + 7 * K)
    z, y = rows(B, K, dtype, rng)
    lp, lse, p, m = softmax_ref(z, y)
    g = rng.standard_normal(B).astype(np.float32).astype(np.float64)
    g[1::13] = 0.0
    unit = unit_grad(p.copy(), y)
    others = unit[np.arange(B), y]
    off = eps(K) + (2 * np.minimum(m[:, None] - z, 104.0) + 16 + 4 * np.minimum(np.abs(lp), np.abs(lse))[:, None]) * U
    off = np.minimum(np.abs(unit) * np.expm1(np.minimum(off, 80.0)), np.maximum(others, p.max(1))[:, None] + 0.0 * unit)
    off[np.arange(B), y] = (2 * eps(K) + 16 * U) * others
    tol = np.abs(g)[:, None] * (off + 4 * U * np.abs(unit) + TINY) + 2.0 ** -126
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (np.abs(unit * g[:, None]) + tol)
    Z, dy, a, b = device(z, dtype), vec(y, torch.int32), torch.zeros(B, device="cuda"), torch.zeros(B, device="cuda")
    hb.logprob(Z, dy, a, b, ws=ws(B))
    dZ = torch.full_like(Z, 7.0)
    hb.logprob_grad(Z, dy, a, b, vec(g), dZ)
    near(dZ, unit * g[:, None], tol, "dZ")
    assert torch.isfinite(dZ).all()
    wide = torch.full((B, K + 5), 7.0, device="cuda", dtype=TYPES[dtype])     # in place, other edges
    wide[:, 3:K + 3] = Z
    hb.logprob_grad(wide[:, 3:K + 3], dy, a, b, vec(g), wide[:, 3:K + 3])
    near(wide[:, 3:K + 3], unit * g[:, None], tol, "dZ in place")
    assert bool((wide[:, :3] == 7.0).all()) and bool((wide[:, K + 3:] == 7.0).all())
    hb.logprob_grad(Z, dy, a, b, vec(g), Z)
    assert torch.equal(Z, dZ)


@pytest.mark.parametrize("c", [0.0, 1e4, 1e5, 1e7, -1e7])
def test_an_offset_of_the_logits_costs_a_gradient_nothing(c):
    """Three classes at c, c + 1, c + 2: softmax 0.0900, 0.2447, 0.6652, whatever c; off by the exponentials' roundings."""
    z = np.array([[c, c + 1, c + 2]] * 3)
    y = np.arange(3, dtype=np.int32)
    a, b, dZ = torch.zeros(3, device="cuda"), torch.zeros(3, device="cuda"), torch.zeros(3, 3, device="cuda")
    hb.logprob(device(z, "f32"), vec(y, torch.int32), a, b, ws=ws(3))
    hb.logprob_grad(device(z, "f32"), vec(y, torch.int32), a, b, torch.ones(3, device="cuda"), dZ)
    p = np.exp([0.0, 1.0, 2.0])
    near(dZ, np.eye(3) - p / p.sum(), 32 * U, "dZ")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K", SHAPES)
def test_policy_loss_on_logits_of_any_size(B, K, dtype):
    """Advantages of both signs, log-ratios away from the borders of the clip; a choice that is all but impossible has ratio 0."""
    rng = np.random.default_rng(B + 3 * K)
    z, y = rows(B, K, dtype, rng)
    lp, _, p, m = softmax_ref(z, y)
    plain = np.abs(lp) < 100
    old = np.where(plain, lp - rng.choice([-0.7, -0.1, 0.0, 0.1, 0.7], B), 0.0).astype(np.float32).astype(np.float64)
    adv = np.where(rng.random(B) < 0.5, -1.0, 1.0) * rng.uniform(0.5, 1.5, B).astype(np.float32)
    refs = np.where(plain, lp + 0.3 * rng.standard_normal(B), 0.0).astype(np.float32).astype(np.float64)
    w = np.where(plain, 1.0, 0.0) / B           # without a reference: all of them
    for use_ref, w in [(True, w.astype(np.float32).astype(np.float64)), (False, np.full(B, float(np.float32(1.0 / B))))]:
        kl_coef = 0.04 if use_ref else 0.0
        r = np.exp(np.minimum(lp - old, 80.0))
        d = np.where(w > 0, refs - lp, 0.0) if use_ref else np.zeros(B)
        cut = ((adv > 0) & (r > 1.2)) | ((adv < 0) & (r < 0.8))
        pg = -np.minimum(r * adv, np.clip(r, 0.8, 1.2) * adv)
        g = w * (np.where(cut, 0.0, -r * adv) - kl_coef * np.expm1(d))
        kl = np.expm1(d) - d
        stats = np.array([(w * (pg + kl_coef * kl)).sum(), (w * pg).sum(), (w * kl).sum(), (w * cut).sum()])
        e = np.where(r > 0, lp_tol(np.where(plain, lp, 0.0), K) + 8 * U, 0.0)
        g_off = w * (r * np.abs(adv) + kl_coef * np.exp(d)) * 2 * e
        s_tol = (w * (r * np.abs(adv) + np.exp(d)) * 2 * e).sum() + 8 * U * np.abs(stats).max() + 8 * U
        Z, dZ = device(z, dtype), torch.full((B, K), 7.0, device="cuda", dtype=TYPES[dtype])
        st, st2, a = torch.full((4,), 7.0, device="cuda"), torch.full((4,), 7.0, device="cuda"), torch.full((B,), 7.0, device="cuda")
        args = dict(ref=vec(refs) if use_ref else None, weight=vec(w) if use_ref else None, kl_coef=kl_coef, ws=ws(B))
        head = (Z, vec(y, torch.int32), vec(old), vec(adv))
        hb.policy_loss(*head, st, dZ=dZ, logp=a, **args)
        near(a, np.where(w > 0, lp, 0.0), lp_tol(lp, K), "logp")
        near(st, stats, s_tol, "stats")
        unit = unit_grad(p.copy(), y)
        near(dZ, unit * g[:, None], grad_tol(unit, z, m, g, K, dtype, g_off), "dZ")
        hb.policy_loss(*head, st2, **args)
        near(st2, stats, s_tol, "stats of the loss alone")
        hb.policy_loss(*head, st, dZ=Z, **args)   # in place
        assert torch.equal(Z, dZ)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K", SHAPES)
def test_preference_loss_on_logits_of_any_size(B, K, dtype):
    rng = np.random.default_rng(B + 5 * K)
    pairs, beta = 2, 0.1
    z, y = rows(B, K, dtype, rng)
    lp, _, p, m = softmax_ref(z, y)
    choice = np.abs(lp) < 100
    seq = np.array([0, B // 5, B // 2, B - 3, B], np.int32)
    live = np.where(choice, lp, 0.0)
    s = np.array([live[seq[q]:seq[q + 1]].sum() for q in range(4)])
    refs = (s + 3 * rng.standard_normal(4)).astype(np.float32).astype(np.float64)
    e = np.where(choice, lp_tol(live, K), 0.0)
    se = np.array([e[seq[q]:seq[q + 1]].sum() for q in range(4)])
    gain = s - refs
    h = gain[0::2] - gain[1::2]
    slope = -beta / pairs / (1 + np.exp(beta * h))
    stats = np.array([np.logaddexp(0, -beta * h).mean(), (h > 0).mean(), beta * gain[0::2].mean(), beta * gain[1::2].mean()])
    g, g_off = np.zeros(B), np.zeros(B)
    for q in range(4):
        g[seq[q]:seq[q + 1]] = slope[q // 2] * (1 if q % 2 == 0 else -1)
        g_off[seq[q]:seq[q + 1]] = beta / pairs * (beta / 4 * (se[0::2] + se[1::2])[q // 2] + 4 * U)
    g, g_off = g * choice, g_off * choice
    dZ = torch.full((B, K), 7.0, device="cuda", dtype=TYPES[dtype])
    st, sl = torch.full((4,), 7.0, device="cuda"), torch.full((4,), 7.0, device="cuda")
    hb.preference_loss(device(z, dtype), vec(np.where(choice, y, -1), torch.int32), vec(seq, torch.int32), st, dZ=dZ, ref=vec(refs), beta=beta,
                       seq_logp=sl, ws=ws(B, pairs))
    near(sl, s, se + U * np.abs(s), "seq_logp")
    near(st, stats, beta * 2 * se.max() + 8 * U * (1 + np.abs(stats).max()), "stats")
    unit = unit_grad(p.copy(), y)
    near(dZ, unit * g[:, None], grad_tol(unit, z, m, g, K, dtype, g_off), "dZ")


def test_a_plain_implementation_agrees_with_its_own_definition():
    """The reference above against the one of ordinary logits, where both hold."""
    rng = np.random.default_rng(2)
    z, y = 2 * rng.standard_normal((9, 33)), rng.integers(0, 33, 9)
    lp, lse, p, _ = softmax_ref(z, y)
    part, lp2, lse2, p2 = ref.rows_ref(z, y)
    assert np.allclose(lp, lp2, atol=1e-13) and np.allclose(lse, lse2, atol=1e-13) and np.allclose(p, p2, atol=1e-15)
    assert np.allclose(unit_grad(p, y), ref.grad_ref(part, p2, y, np.ones(9)), atol=1e-15)


def test_matrices_side_by_side_in_one_buffer():
    """Input and output as the two halves of a buffer's columns: as apart (the logits aligned alike: a row's sum is made in pieces that
    begin at 16-byte boundaries), and nothing else is written."""
    rng = np.random.default_rng(4)
    B, K = 37, 203
    z, y = rows(B, K, "f32", rng)
    buf = torch.full((B, 2 * K + 7), 7.0, device="cuda")
    left, right = buf[:, 1:K + 1], buf[:, K + 1:2 * K + 1]
    left.copy_(torch.as_tensor(z))
    Z, dy, apart = buf.clone()[:, 1:K + 1], vec(y, torch.int32), torch.full((B, K), 7.0, device="cuda")
    a, b, g = torch.zeros(B, device="cuda"), torch.zeros(B, device="cuda"), torch.ones(B, device="cuda")
    st = torch.zeros(4, device="cuda")
    hb.logprob(left, dy, a, b, ws=ws(B))
    for call in (lambda z, d: hb.dropout(z, d, 0.25, 3, 1), lambda z, d: hb.logprob_grad(z, dy, a, b, g, d),
                 lambda z, d: hb.policy_loss(z, dy, a, g, st, dZ=d, ws=ws(B))):
        call(left, right)
        call(Z, apart)
        assert torch.equal(right, apart) and torch.equal(left, Z)
        assert bool((buf[:, 0] == 7.0).all()) and bool((buf[:, 2 * K + 1:] == 7.0).all())
