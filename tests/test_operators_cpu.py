"""What the operators on device tensors refuse, before any device call, and the generator behind dropout."""
import numpy as np
import pytest
import torch

import operators_ref as ref
import paper_2004_08771_amd as hb

Z = torch.zeros(6, 10)
Y = torch.zeros(6, dtype=torch.int32)
ROW = torch.zeros(6)
WS = torch.zeros(1 << 17, dtype=torch.uint8)
STATS = torch.zeros(4)
SEQ = torch.tensor([0, 2, 6], dtype=torch.int32)


def refused(call, code=hb.HB_ERR_INVALID, text=None):
    with pytest.raises(hb.HbError) as e:
        call()
    assert e.value.code == code, e.value
    if text:
        assert text in str(e.value)


def test_known_answers_of_the_generator():
    """The three published vectors of Philox4x32-10 (Random123)."""
    for ctr, key, out in [
        ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
        ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
        ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
         (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)),
    ]:
        assert tuple(int(v) for v in ref.philox(np.array(ctr, np.uint64), key)) == out


@pytest.mark.parametrize("p", [-0.1, 1.0, 1.5, float("nan"), float("inf"), 1.0 - 2.0 ** -20])
def test_dropout_refuses_probabilities(p):
    refused(lambda: hb.dropout(Z, torch.zeros_like(Z), p, 1))


def test_dropout_refuses_operands():
    out = torch.zeros_like(Z)
    for x, o in [(Z.double(), out.double()), (Z, out.bfloat16()), (Z, torch.zeros(6, 11)), (Z.t(), torch.zeros(10, 6)),
                 (Z[0], out[0]), (Z.expand(6, 10)[:1].expand(6, 10), out)]:
        refused(lambda: hb.dropout(x, o, 0.5, 1))
    big = torch.zeros(7, 10)
    refused(lambda: hb.dropout(big[:6], big[1:], 0.5, 1), text="overlaps")
    wide = torch.zeros(6, 30)
    refused(lambda: hb.dropout(wide[:, :10], wide[:, 5:15], 0.5, 1), text="overlaps")
    call = hb.lib().hb_dropout_async
    a = Z.data_ptr()
    for args in [(a, 10, a, 10, 2, 6, 10), (a, 9, a, 9, 0, 6, 10), (a, 10, a, 9, 0, 6, 10), (None, 10, a, 10, 0, 6, 10),
                 (a, 10, None, 10, 0, 6, 10), (a + 2, 10, a + 2, 10, 0, 6, 10), (a, 10, a, 10, 0, -1, 10),
                 (a, 10, a, 10, 0, 6, -1), (a, 1 << 31, a, 1 << 31, 0, 1 << 31, 10), (a, 1 << 31, a, 1 << 31, 0, 6, 10)]:
        assert call(*args, 0.5, 1, 0, None) == hb.HB_ERR_INVALID, args
    assert call(None, 0, None, 0, 0, 0, 10, 0.5, 1, 0, None) == hb.HB_OK      # nothing to do
    assert call(None, 0, None, 0, 0, 3, 0, 0.5, 1, 0, None) == hb.HB_OK


def test_workspace_sizes():
    need = hb.choice_workspace_bytes
    assert 0 < need(0) <= need(1) <= need(4096) < need(8192) and need(16, 1 << 20) > need(16, 64) >= need(16)
    assert need(-1) == 0 and need((1 << 22) + 1) == 0 and need(4, -1) == 0 and need(4, (1 << 22) + 1) == 0
    small = WS[:need(6) - 1]
    refused(lambda: hb.logprob(Z, Y, ROW, ROW, ws=small), text="workspace")
    refused(lambda: hb.logprob(Z, Y, ROW, ROW, ws=None))
    refused(lambda: hb.policy_loss(Z, Y, ROW, ROW, STATS, ws=small), text="workspace")
    refused(lambda: hb.preference_loss(Z, Y, SEQ, STATS, ws=small), text="workspace")
    refused(lambda: hb.logprob(Z, Y, ROW, ROW, ws=WS[4:]), text="aligned")


def test_losses_refuse_operands():
    for call in (lambda z, y: hb.logprob(z, y, ROW, ROW, ws=WS),
                 lambda z, y: hb.logprob_grad(z, y, ROW, ROW, ROW, torch.zeros_like(z)),
                 lambda z, y: hb.policy_loss(z, y, ROW, ROW, STATS, ws=WS),
                 lambda z, y: hb.preference_loss(z, y, SEQ, STATS, ws=WS)):
        for z, y in [(Z.double(), Y), (Z, Y.long()), (Z, Y[:5]), (Z.half(), Y), (Z[0], Y), (Z[:, ::2], Y),
                     (Z, torch.zeros(12, dtype=torch.int32)[::2]), (torch.zeros(6, 0), Y)]:
            refused(lambda: call(z, y))
    big = torch.zeros(7, 10)
    refused(lambda: hb.logprob_grad(big[:6], Y, ROW, ROW, ROW, big[1:]), text="overlaps")
    refused(lambda: hb.policy_loss(big[:6], Y, ROW, ROW, STATS, dZ=big[1:], ws=WS), text="overlaps")
    refused(lambda: hb.preference_loss(big[:6], Y, SEQ, STATS, dZ=big[1:], ws=WS), text="overlaps")
    refused(lambda: hb.policy_loss(Z, Y, ROW, ROW, STATS, dZ=Z.bfloat16(), ws=WS))
    refused(lambda: hb.logprob(Z, Y, None, ROW, ws=WS), text="d_logp")
    refused(lambda: hb.policy_loss(Z, Y, ROW, ROW, None, ws=WS), text="d_stats")
    refused(lambda: hb.policy_loss(Z, Y, None, ROW, STATS, ws=WS), text="d_old_logp")
    refused(lambda: hb.policy_loss(Z, Y, ROW, None, STATS, ws=WS), text="d_adv")
    refused(lambda: hb.logprob_grad(Z, Y, None, ROW, ROW, torch.zeros_like(Z)))
    refused(lambda: hb.policy_loss(Z, Y, ROW, ROW[:3], STATS, ws=WS))
    refused(lambda: hb.policy_loss(Z, Y, ROW, ROW, STATS[:3], ws=WS))


def test_losses_refuse_outputs_that_overlap():
    r, d = torch.zeros(4, 6), torch.zeros_like(Z)
    far = torch.zeros(64)
    both, four = far[:6], far[3:7]
    for call in (lambda: hb.logprob(Z, Y, r[0], r[0], ws=WS), lambda: hb.logprob(Z, Y, both, far[5:11], ws=WS),
                 lambda: hb.logprob(Z, Y, Z.view(-1)[54:], None, ws=WS), lambda: hb.logprob(Z, Y, WS.view(torch.float32)[:6], None, ws=WS),
                 lambda: hb.logprob_grad(Z, Y, r[0], r[1], d.view(-1)[:6], d), lambda: hb.logprob_grad(Z, Y, d.view(-1)[54:], r[1], r[2], d),
                 lambda: hb.policy_loss(Z, Y, r[0], r[1], STATS, logp=r[0], ws=WS),
                 lambda: hb.policy_loss(Z, Y, r[0], r[1], STATS, logp=r[1], ws=WS),
                 lambda: hb.policy_loss(Z, Y, r[0], r[1], STATS, logp=r[2], ref=r[2], ws=WS),
                 lambda: hb.policy_loss(Z, Y, r[0], r[1], STATS, logp=r[2], weight=r[2], ws=WS),
                 lambda: hb.policy_loss(Z, Y, r[0], r[1], four, logp=both, ws=WS),
                 lambda: hb.policy_loss(Z, Y, r[0], r[1], d.view(-1)[:4], dZ=d, ws=WS),
                 lambda: hb.policy_loss(Z, Y, r[0], r[1], STATS, dZ=d, logp=Z.view(-1)[:6], ws=WS),
                 lambda: hb.preference_loss(Z, Y, SEQ, STATS, seq_logp=STATS[:2], ws=WS),
                 lambda: hb.preference_loss(Z, Y, SEQ, STATS, seq_logp=r[0][:2], ref=r[0][:2], ws=WS),
                 lambda: hb.preference_loss(Z, Y, SEQ, d.view(-1)[:4], dZ=d, ws=WS)):
        refused(call, text="overlaps")


@pytest.mark.parametrize("more", [dict(clip=(-0.1, 0.2)), dict(clip=(1.1, 0.2)), dict(clip=(0.2, -0.2)),
                                  dict(clip=(float("nan"), 0.2)), dict(clip=(0.2, float("inf"))), dict(kl_coef=0.1),
                                  dict(kl_coef=-0.1, ref=ROW), dict(kl_coef=float("nan"), ref=ROW)])
def test_policy_refuses_settings(more):
    refused(lambda: hb.policy_loss(Z, Y, ROW, ROW, STATS, ws=WS, **more))


@pytest.mark.parametrize("more", [dict(beta=0.0), dict(beta=-1.0), dict(beta=float("nan")), dict(beta=float("inf")),
                                  dict(smoothing=-0.1), dict(smoothing=0.6), dict(smoothing=float("nan")),
                                  dict(ref=ROW[:3])])
def test_preference_refuses_settings(more):
    refused(lambda: hb.preference_loss(Z, Y, SEQ, STATS, ws=WS, **more))


def test_preference_refuses_offsets():
    for seq in (SEQ[:1], SEQ[:2], torch.zeros(4, dtype=torch.int32), SEQ.long()):
        refused(lambda: hb.preference_loss(Z, Y, seq, STATS, ws=WS))
    p = hb.binding.Preference(None, None, 1, 0.1, 0.0)
    call = hb.lib().hb_preference_loss_async
    args = lambda p: (Z.data_ptr(), 10, 0, Y.data_ptr(), 6, 10, p, STATS.data_ptr(), None, None, 0, WS.data_ptr(), 1 << 17, None)
    assert call(*args(p)) == hb.HB_ERR_INVALID
    for pairs in (0, -1, (1 << 22) + 1):
        assert call(*args(hb.binding.Preference(SEQ.data_ptr(), None, pairs, 0.1, 0.0))) == hb.HB_ERR_INVALID
    assert call(*args(None)) == hb.HB_ERR_INVALID


def test_limits_of_rows_and_classes():
    z, y, w = Z.data_ptr(), Y.data_ptr(), WS.data_ptr()
    call = hb.lib().hb_logprob_async
    for B, K, ld in [(-1, 10, 10), ((1 << 22) + 1, 10, 10), (6, 0, 10), (6, (1 << 24) + 1, 1 << 25), (6, 10, 9), (6, 10, 1 << 31)]:
        assert call(z, ld, 0, y, B, K, y, y, w, 1 << 40, None) == hb.HB_ERR_INVALID, (B, K, ld)
    assert call(z, 10, 7, y, 6, 10, y, y, w, 1 << 17, None) == hb.HB_ERR_INVALID
    assert call(None, 10, 0, None, 0, 10, None, None, w, 1 << 17, None) == hb.HB_OK   # no rows
