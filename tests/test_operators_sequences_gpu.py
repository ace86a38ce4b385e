"""The preference loss: rows outside of all sequences, and many pairs."""
import numpy as np
import pytest
import torch

import paper_2004_08771_amd as hb

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def rows_of_workspace(ws, B, pairs):
    """What the call has kept of each row: its log-probability, 0 where it has taken no part (sums of 32 bytes for each pair, 1024 at
    least, and coefficients of 16 bytes a row stand in front of them)."""
    at = 32 * max(pairs, 1024) + 16 * B
    return ws[at:at + 8 * B].view(torch.float64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K", [(50, 3), (50, 40), (50, 700), (50, 5000), (1500, 30), (40, 33001), (70, 130001), (3000, 9)])
def test_rows_outside_of_the_sequences_are_not_looked_at(B, K, dtype):
    """They have classes and ordinary logits: a call that reads them has log-probabilities for them."""
    g = torch.Generator(device="cuda").manual_seed(B + K)
    Z = torch.randn(B, K, device="cuda", generator=g).to(TYPES[dtype])
    y = torch.randint(0, K, (B,), device="cuda", generator=g, dtype=torch.int32)
    lo, mid, hi = B // 5, B // 3, B - B // 4
    seq = torch.tensor([lo, mid, hi], dtype=torch.int32, device="cuda")
    for grad in (False, True):
        ws = torch.zeros(hb.choice_workspace_bytes(B, 1), dtype=torch.uint8, device="cuda")
        rows_of_workspace(ws, B, 1).fill_(7.0)
        st, sl, dZ = torch.zeros(4, device="cuda"), torch.zeros(2, device="cuda"), torch.full_like(Z, 7.0)
        hb.preference_loss(Z, y, seq, st, dZ=dZ if grad else None, seq_logp=sl, ws=ws)
        kept = rows_of_workspace(ws, B, 1)
        assert bool((kept[lo:hi] < 0).all())
        assert not kept[:lo].any() and not kept[hi:].any()
        # the sums of what is kept, rounded to fp32
        want = torch.stack([kept[lo:mid].sum(), kept[mid:hi].sum()])
        assert float(((sl.double() - want) / want).abs().max()) <= 2.0 ** -24 + 1e-12
        if grad:
            assert bool((dZ[:lo] == 7.0).all()) and bool((dZ[hi:] == 7.0).all()) and not bool((dZ[lo:hi] == 7.0).any())


@pytest.mark.parametrize("pairs,per", [(1025, 3), (16384, 2), (16385, 2), (65536, 1), (65537, 1), (300000, 1), (1 << 21, 1)])
def test_many_pairs(pairs, per):
    """Sums over more pairs than one block adds up, in 64 bits: off by the rounding of the result; a log-probability of few classes by 32 u."""
    B, K, beta, eps, u = 2 * pairs * per, 5, 0.3, 0.1, 2.0 ** -24
    g = torch.Generator(device="cuda").manual_seed(pairs)
    Z = torch.randn(B, K, device="cuda", generator=g)
    y = torch.randint(-1, K, (B,), device="cuda", generator=g, dtype=torch.int32)
    # lengths of 0 to 2 per
    cuts = torch.randint(0, B + 1, (2 * pairs - 1,), device="cuda", generator=g).sort().values
    seq = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), B)])
    refs = torch.randn(2 * pairs, device="cuda", generator=g)
    lsm = torch.log_softmax(Z.double(), 1)
    part = y >= 0
    lp = torch.where(part, lsm.gather(1, y.clamp(min=0).long()[:, None])[:, 0], 0.0)
    cum = torch.cat([lp.new_zeros(1), lp.cumsum(0)])
    s = cum[seq[1:]] - cum[seq[:-1]]
    gain = (s - refs.double()).view(pairs, 2)
    h = gain[:, 0] - gain[:, 1]
    softplus = lambda v: v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))  # noqa: E731
    stats = torch.stack([((1 - eps) * softplus(-beta * h) + eps * softplus(beta * h)).mean(), (h > 0).double().mean(),
                         beta * gain[:, 0].mean(), beta * gain[:, 1].mean()])
    slope = beta / pairs * (eps * torch.sigmoid(beta * h) - (1 - eps) * torch.sigmoid(-beta * h))
    rows = torch.searchsorted(seq[1:], torch.arange(B, device="cuda"), right=True)
    gr = torch.stack([slope, -slope], 1).view(-1)[rows]
    unit = -lsm.exp()
    unit.scatter_add_(1, y.clamp(min=0).long()[:, None], torch.ones(B, 1, device="cuda", dtype=torch.float64))
    want = unit * (gr * part)[:, None]
    ws = torch.full((hb.choice_workspace_bytes(B, pairs),), 0xFF, dtype=torch.uint8, device="cuda")
    st, sl, dZ = torch.zeros(4, device="cuda"), torch.zeros(2 * pairs, device="cuda"), torch.full_like(Z, 7.0)
    args = dict(ref=refs, beta=beta, smoothing=eps, ws=ws)
    longest = int((seq[1:] - seq[:-1]).max())
    seq = seq.to(torch.int32)
    for grad in (True, False):
        hb.preference_loss(Z, y, seq, st, dZ=dZ if grad else None, seq_logp=sl, **args)
        assert float(((st.double() - stats).abs() - (8 + 64 * per * beta) * u * (1 + stats.abs())).max()) <= 0
        assert float(((sl.double() - s).abs() - longest * 32 * u - 2 * u * s.abs()).max()) <= 0
        st.fill_(7.0)
    # an exponential and 1 / s: 64 u of a probability; the slope by beta / 4 times the sums' error
    tol = 64 * u * want.abs() + (beta / pairs) * (64 * u + beta / 4 * 2 * longest * 32 * u) * unit.abs() + 1e-30
    assert float(((dZ.double() - want).abs() - tol).max()) <= 0
