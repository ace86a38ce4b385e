"""Two GPU workers on host threads of their own, each handle on its own stream: what holds whatever their pace is.  With a scheduler each, both train their whole epoch, with the
bits that they have alone; with one scheduler between them, what the algorithm fixes holds, and a share for each is not asked for."""
import threading

import numpy as np
import pytest

import hb_inputs as hi
import oracle

pytestmark = pytest.mark.gpu

DIMS, ACT, LOSS = (32, 64, 32, 6), hi.ACT_SIGMOID, hi.LOSS_SOFTMAX_CE


def data(n, seed=14):
    rng = np.random.default_rng(seed)
    X = rng.standard_normal((n, DIMS[0])).astype(np.float32)
    y = np.argmax(X @ rng.standard_normal((DIMS[0], DIMS[-1])), axis=1).astype(np.int32)
    return X, y, hi.xavier_uniform_params(DIMS, rng)


def handles(params, muon):
    import torch
    import paper_2004_08771_amd as hb
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ms = [hb.Model(DIMS, ACT, LOSS).configure(hb.HB_F32, 512, stream=s.cuda_stream) for s in streams]
    for m in ms:
        m.set_params(params)
        if muon:
            m.set_muon(hb.muon_args(weight_decay=0.1))
    return streams, ms


def together(*calls):
    """The results of the calls, on a thread each, which meet before the first."""
    out, meet = {}, threading.Barrier(len(calls))

    def work(w):
        try:
            meet.wait(timeout=60)
            out[w] = calls[w]()
        except Exception as e:  # shown by the assertion below
            out[w] = e

    th = [threading.Thread(target=work, args=(w,)) for w in range(len(calls))]
    for t in th:
        t.start()
    for t in th:
        t.join(timeout=100)
    assert all(isinstance(out.get(w), tuple) for w in range(len(calls))), out
    return [out[w] for w in range(len(calls))]


def params_of(m):
    p = np.empty(m.num_params, np.float32)
    m.get_params(p)
    return p


@pytest.mark.parametrize("muon", [False, True])
def test_a_scheduler_each(muon):
    import paper_2004_08771_amd as hb
    n = 30000
    X, y, params = data(n)
    rates, sizes = (0.02 / 64, 0.01 / 64), (256, 200)

    def epoch(m, w):
        return m.worker_run_epoch(hb.Sched(n, [sizes[w]], [sizes[w]], [sizes[w]]), 0, X, y, rates[w])

    _, alone = handles(params, muon)
    want = [epoch(m, w) for w, m in enumerate(alone)]
    _, ms = handles(params, muon)
    got = together(*[lambda m=m, w=w: epoch(m, w) for w, m in enumerate(ms)])
    for w, m in enumerate(ms):
        assert got[w] == want[w] and got[w][1] == n // sizes[w]
        assert np.array_equal(params_of(m), params_of(alone[w])) and not np.array_equal(params_of(m), params)
        m.destroy()
        alone[w].destroy()


def test_one_scheduler_between_them():
    import paper_2004_08771_amd as hb
    n = 60000
    X, y, params = data(n)
    before = oracle.batch_loss(DIMS, ACT, LOSS, params, X, y)
    H = params.copy()
    s = hb.Sched(n, [64, 64], [512, 256], [512, 256], 2.0)
    _, ms = handles(params, False)
    got = together(*[lambda m=m, w=w: m.worker_run_epoch(s, w, X, y, 0.02 / 64, host_model=H, merge_every=1, merge_weight=0.5) for w, m in enumerate(ms)])
    for u, steps, _ in got:
        assert u == steps
    # as many steps as the smallest and the largest batches make of the examples
    assert (n - s.remaining()) / 512 <= got[0][1] + got[1][1] <= (n - s.remaining()) / 64
    assert s.remaining() < min(s.batch_size(0), s.batch_size(1))
    assert 64 <= s.batch_size(0) <= 512 and 64 <= s.batch_size(1) <= 256
    assert np.all(np.isfinite(H)) and oracle.batch_loss(DIMS, ACT, LOSS, H, X, y) < before
    for m in ms:
        m.destroy()
