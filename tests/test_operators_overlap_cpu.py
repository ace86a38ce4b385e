"""Which matrices overlap: rows, not the ranges from their first to their last element.  Nothing is launched: the check comes before
anything that needs a device, and the addresses are made up."""
import random

import pytest
import torch

import paper_2004_08771_amd as hb

BASE = 1 << 40


def overlaps(x, ldx, out, ldo, rows, cols, size):
    rc = hb.lib().hb_dropout_async(x, ldx, out, ldo, {4: hb.HB_TENSOR_F32, 2: hb.HB_TENSOR_BF16}[size], rows, cols, 0.5, 1, 0, None)
    assert rc != hb.HB_OK
    return "overlaps" in hb.binding.last_error()


def elements(first, ld, rows, cols):
    return {first + i * ld + j for i in range(rows) for j in range(cols)}


@pytest.mark.parametrize("size", [2, 4])
def test_overlap_of_matrices_is_that_of_their_elements(size):
    rng = random.Random(size)
    seen = {True: 0, False: 0}
    for _ in range(6000):
        rows, cols = rng.randint(1, 12), rng.randint(1, 9)
        ldx, ldo = (cols + rng.choice([0, 1, 2, 5, rng.randint(0, 40), rng.randint(0, 200)]) for _ in range(2))
        if rng.random() < 0.3:
            ldo = ldx
        span = max(ldx, ldo) * rows
        at = rng.randint(-span, span) if rng.random() < 0.5 else rng.randint(-ldx, ldx)
        if at == 0 and ldx == ldo:
            continue
        want = bool(elements(0, ldx, rows, cols) & elements(at, ldo, rows, cols))
        seen[want] += 1
        assert overlaps(BASE, ldx, BASE + at * size, ldo, rows, cols, size) == want, (rows, cols, ldx, ldo, at)
    assert min(seen.values()) > 1000


def test_overlap_of_large_matrices():
    """Pitches and rows up to the limits: rows of one in the gaps of the other, up to the last element of a gap and past it."""
    rows, ld, half = 1 << 30, (1 << 31) - 1, (1 << 30) - 1
    for cols, shift, want in [(1000, 1000, False), (1000, 999, True), (half, half, False), (half, half - 1, True), (half, half + 1, False),
                              (half, half + 2, True), (7, 8, False), (7, ld - 6, True)]:
        assert overlaps(BASE, ld, BASE + 4 * shift, ld, rows, cols, 4) == want, (cols, shift)
    # pitches of 1000 and 1001, 100 columns: row j of one begins at 100 + j behind row j of the other and ends in row j + 1 from
    # j = 801 on, which is there from 803 rows on
    assert not overlaps(BASE, 1000, BASE + 4 * 100, 1001, 802, 100, 4)
    assert overlaps(BASE, 1000, BASE + 4 * 100, 1001, 803, 100, 4)


def test_halves_of_a_buffer():
    """As a user has them: the left columns of a buffer to the right ones, log-probabilities beside gradients."""
    buf = torch.zeros(6, 20)
    y, row, ws = torch.zeros(6, dtype=torch.int32), torch.zeros(6), torch.zeros(1 << 17, dtype=torch.uint8)
    for call in (lambda a, b: hb.dropout(a, b, 0.5, 1), lambda a, b: hb.logprob_grad(a, y, row, row, row, b),
                 lambda a, b: hb.policy_loss(a, y, row, row, torch.zeros(4), dZ=b, ws=ws)):
        for a, b, meet in [(buf[:, :10], buf[:, 10:], False), (buf[:, 10:], buf[:, :10], False), (buf[:, :10], buf[:, 9:19], True),
                           (buf[::2, :10], buf[1::2, :10], False), (buf[:3], buf[2:5], True)]:
            with pytest.raises(hb.HbError) as e:
                call(a, b) if len(a) == 6 else hb.dropout(a, b, 0.5, 1)
            assert ("overlaps" in str(e.value)) == meet


def test_what_is_empty_overlaps_nothing():
    """No rows: the pointers to what a row has may be anything, inside the statistics as well."""
    st, ws = torch.zeros(4), torch.zeros(1 << 17, dtype=torch.uint8)
    inside = st.data_ptr() + 4
    policy = hb.binding.Policy(inside, None, inside, None, 0.2, 0.2, 0.0)
    rc = hb.lib().hb_policy_loss_async(inside, 5, hb.HB_TENSOR_F32, inside, 0, 5, policy, st.data_ptr(), inside, inside, 5, ws.data_ptr(),
                                       ws.nbytes, None)
    assert rc != hb.HB_OK and "overlaps" not in hb.binding.last_error()      # (there is no device here)
