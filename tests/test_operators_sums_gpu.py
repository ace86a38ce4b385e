"""That every class of a row is counted, once, in every form: rows whose sum is known to the last digit.

With all logits equal every exponential is 2^0 = 1 and every partial sum a whole number of at most 2^24, exact in fp32.  What is left is the
logarithm (an integer, and one of fp32 off by 2 u, u = 2^-24) and the rounding of the result: log K off by (2 + 1.25 log K) u, 1 / K by 4 u
relative (1 / s, its product with g).  A piece of 16 bytes left out of a row of 2^20 classes is 4e-6.
"""
import numpy as np
import pytest
import torch

import paper_2004_08771_amd as hb

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CLASSES = [1, 2, 5, 8, 9, 17, 31, 40, 64, 65, 100, 129, 257, 400, 513, 983, 1025, 1500, 2049, 3001, 4099, 6000, 8193, 12001, 16385, 20000, 27003,
           32771, 40961, 49157, 53001, 60007, 65537, 81925, 98309, 110001, 131073, 163841, 200003]
VOCABULARIES = [(1, 300007, "bf16"), (2, 1 << 20, "f32"), (3, 700001, "bf16"), (1, 1 << 24, "f32"), (1, 1 << 24, "bf16"), (1030, 50001, "f32"),
                (300, 170003, "bf16"), (2100, 98400, "bf16"), (2100, 49300, "f32")]


def ws(B, pairs=0):
    return torch.full((hb.choice_workspace_bytes(B, pairs),), 0xFF, dtype=torch.uint8, device="cuda")


def view(B, K, dtype, base, fill):
    """B rows with a pitch that puts each at another place in a 16-byte piece; around them what must neither count nor change."""
    ld = K + 3
    flat = torch.full((B * ld + base + 16,), 50.0, dtype=TYPES[dtype], device="cuda")
    m = flat[base:base + B * ld].view(B, ld)[:, :K]
    m.fill_(fill)
    return m, flat


def check(B, K, dtype, base, c):
    Z, _ = view(B, K, dtype, base, c)
    y = (torch.arange(B, device="cuda") * 7919 % K).to(torch.int32)
    y[0], y[-1] = K - 1, 0
    lp = -np.log(K)
    tol = (2 + 1.25 * abs(lp)) * U + (2.0 ** -30 if K == 1 else 0.0)
    out = 2.0 ** -8 if dtype == "bf16" else 0.0
    a, b = torch.full((B,), 7.0, device="cuda"), torch.full((B,), 7.0, device="cuda")
    hb.logprob(Z, y, a, b, ws=ws(B))
    c = float(Z[0, 0])
    assert float((a.double() - lp).abs().max()) <= tol
    assert float((b.double() - (c - lp)).abs().max()) <= tol + U * abs(c - lp)

    def gradient(dZ, g, what):
        """g ([k = y] - 1 / K), rounded."""
        want = -g / K
        rest = dZ.double()
        mine = rest.gather(1, y.long()[:, None])[:, 0]
        assert float((mine - g * (1 - 1 / K)).abs().max()) <= abs(g) * (16 * U + out) * (1 - 1 / K), what
        rest = rest.scatter(1, y.long()[:, None], want)
        assert float((rest - want).abs().max()) <= abs(want) * (16 * U + 4 * U * abs(lp) + out), what

    d, flat = view(B, K, dtype, base + 1, 7.0)
    hb.logprob_grad(Z, y, a, b, torch.full((B,), -0.5, device="cuda"), d)
    gradient(d, -0.5, "log-probabilities")
    one = torch.ones(B, device="cuda")
    st = torch.zeros(4, device="cuda")
    hb.policy_loss(Z, y, a, one, st, dZ=d, weight=one, ws=ws(B))      # ratio 1 but for the rounding of a log-probability
    gradient(d, -1.0, "policy")
    assert abs(float(st[0]) + B) <= B * (2 * tol + 4 * U)
    hb.policy_loss(Z, y, a, one, st, weight=one, ws=ws(B))
    assert abs(float(st[0]) + B) <= B * (2 * tol + 4 * U)
    if B >= 2:
        n = B // 2
        seq, sl = torch.tensor([0, n, B], dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda")
        ref = torch.tensor([n * lp, (B - n) * lp], device="cuda", dtype=torch.float32)
        hb.preference_loss(Z, y, seq, st, dZ=d, ref=ref, seq_logp=sl, beta=0.001, ws=ws(B, 1))
        assert float((sl.double() - ref.double()).abs().max()) <= B * tol + 2 * U * B * abs(lp)
        # h = 0 but for the sums' error and the reference's rounding: a slope of beta / 2
        rows = d.double() * 2000
        mine = rows.gather(1, y.long()[:, None])[:, 0].clone()
        sign = torch.where(torch.arange(B, device="cuda") < n, -1.0, 1.0).double()
        rel = 16 * U + out + 0.001 * (B * tol + 2 * U * B * abs(lp))
        assert float((mine - sign * (1 - 1 / K)).abs().max()) <= rel * (1 - 1 / K)
        rows = rows.scatter(1, y.long()[:, None], 0.0) + sign[:, None] / K
        rows = rows.scatter(1, y.long()[:, None], 0.0)
        assert float(rows.abs().max()) <= rel / K
    around = torch.ones_like(flat, dtype=torch.bool)
    around[base + 1:base + 1 + B * (K + 3)].view(B, K + 3)[:, :K] = False
    assert bool((flat[around] == 50.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", CLASSES)
def test_every_class_is_counted(K, dtype):
    for B, base, c in [(1, 0, 0.0), (5, 3, -2.0), (67, 6, 1.5)] + ([(300, 1, 0.25)] if K < 20000 else []):
        check(B, K, dtype, base, c)


@pytest.mark.parametrize("B,K,dtype", VOCABULARIES)
def test_every_class_of_long_rows_is_counted(B, K, dtype):
    check(B, K, dtype, 5, 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K", [(24, 1 << 24), (48, 300007), (300, 150001), (60, 61003), (80, 4099)])
def test_a_large_class_is_found_wherever_it_is(B, K, dtype):
    """One logit of log K + 3 among zeros, at the ends, at the borders of pieces, lanes and chunks, in turn: a class left out there
    changes log-probabilities by 3."""
    V = 4 if dtype == "f32" else 8
    rng = np.random.default_rng(K)
    per = -(-(K // V) // max(1, min(-(-(K // V) // 1024), 2048 // B)))     # pieces of a chunk
    spots = list(range(V)) + list(range(K - V, K))
    for piece in [64, 256, 1024, per, 2 * per, K // V - 1]:
        spots += [piece * V + i for i in (-1, 0, V - 1, V)]
    spots = [s for s in spots if 0 <= s < K] + list(rng.integers(0, K, B))
    high = float(torch.tensor(np.log(K) + 3.0).to(TYPES[dtype]))
    for start in range(0, max(1, len(spots) - B + 1), B):
        at = np.array(spots[start:start + B])
        at = np.concatenate([at, at[:B - len(at)]])
        Z = torch.zeros(B, K, dtype=TYPES[dtype], device="cuda")
        cols = torch.as_tensor(at, device="cuda")
        Z[torch.arange(B, device="cuda"), cols] = high
        y = ((cols + 1) % K).to(torch.int32)
        lse = np.log(np.exp(high) + K - 1)
        a, b = torch.zeros(B, device="cuda"), torch.zeros(B, device="cuda")
        hb.logprob(Z, y, a, b, ws=ws(B))
        # ones are added up exactly, the large exponential is off by (2 T + 4) u of itself, T = high
        tol = (2 * high + 8 + 1.25 * lse) * U
        assert float((a.double() + lse).abs().max()) <= tol, at[int((a.double() + lse).abs().argmax())]
        st, old, one = torch.zeros(4, device="cuda"), a.clone(), torch.ones(B, device="cuda")
        hb.policy_loss(Z, y, old, one, st, weight=one, dZ=Z, ws=ws(B))      # in place
        p = np.exp(high - lse)
        got = Z[torch.arange(B, device="cuda"), cols].double()
        assert float((got / p - 1).abs().max()) <= tol + 16 * U + (2.0 ** -8 if dtype == "bf16" else 0.0)
        del Z
