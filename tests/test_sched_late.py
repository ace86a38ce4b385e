"""The scheduler hands out the rest of an epoch to whoever asks: a worker that asks late gets nothing, so nothing that two workers do at their own pace may count on a
share for each."""
import pytest

from oracle.sched import AdaptiveSchedule


def _of_the_library(*args):
    import paper_2004_08771_amd as hb
    return hb.Sched(*args)


@pytest.mark.parametrize("make", [AdaptiveSchedule, _of_the_library])
def test_a_worker_that_asks_late_gets_nothing(make):
    """Two workers, 60000 examples: the first is served 117 batches of 512 before the other asks, and 96 examples are left, fewer than the other's smallest
    batch that it would be given."""
    s = make(60000, [64, 64], [512, 256], [512, 256], 2.0)
    steps = 0
    while s.request(0, float(steps))[1]:
        steps += 1
    assert steps == 117 and s.remaining() == 96
    assert s.request(1, 0.0)[1] == 0
    s.new_epoch()
    assert s.request(1, 0.0)[1] > 0
