"""Rates that hb_muon_async refuses are refused by a handle's orthogonalised steps too, before anything of the step runs."""
import numpy as np
import pytest
import torch

import paper_2004_08771_amd as hb
from test_model_muon_gpu import batch, model, momenta, params
from test_operators_gpu import vec

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("how,scale,lr", [({}, 1e3, 1e38), ({}, -1e3, 1e38), ({"weight_decay": 1e30}, 0.2, 1e30), ({}, 3e38, 0.0), ({}, 3e38, 1e-3)])
def test_a_rate_whose_products_are_not_finite(how, scale, lr, bf16):
    dims, B = (20, 70, 40, 11), 60
    X, y = batch(dims, B, bf16)
    m, flat = model(dims, bf16=bf16)
    m.set_muon(hb.muon_args(**how), 2, 3, scale)  # factors scale sqrt(70), scale sqrt(40)
    seed = np.arange(m.num_params, dtype=np.float32)
    m.set_momenta(seed)
    rng = np.random.default_rng(2)
    old, adv, seq = vec(-2 + 0.1 * rng.standard_normal(B)), vec(rng.standard_normal(B)), vec([0, 20, 30, 50, 60], torch.int32)
    policy, preference = hb.policy_args(B, old, adv), hb.preference_args(seq)
    loss, stats = torch.full((1,), 7.0, device="cuda"), torch.full((4,), 7.0, device="cuda")
    for step in (lambda r: m.batch_step_async(X, y, B, r, loss), lambda r: m.policy_step_async(X, y, B, r, policy, stats),
                 lambda r: m.preference_step_async(X, y, B, r, preference, stats)):
        with pytest.raises(hb.HbError) as e:
            step(lr)
        assert e.value.code == hb.HB_ERR_INVALID and "not finite" in str(e.value)
        assert np.array_equal(params(m), flat) and np.array_equal(momenta(m), seed)
        assert bool((loss == 7).all()) and bool((stats == 7).all())
    # gradients need no rate, and a rate that is fine is taken (the usual factor again)
    grad = torch.zeros(m.num_params, device="cuda")
    assert np.isfinite(m.batch_grad(X, y, B, grad))
    m.set_muon(hb.muon_args(), 2, 3, 0.2)
    m.batch_step_async(X, y, B, 0.01, loss)
    assert np.isfinite(params(m)).all() and not np.array_equal(params(m), flat) and float(loss) != 7


def test_an_epoch_of_such_a_rate():
    dims, n = (12, 24, 4), 600
    rng = np.random.default_rng(0)
    X, y = rng.standard_normal((n, dims[0])).astype(np.float32), rng.integers(0, 4, n).astype(np.int32)
    m, flat = model(dims)
    m.set_muon(hb.muon_args(), scale=1e10)
    with pytest.raises(hb.HbError) as e:
        m.worker_run_epoch(hb.Sched(n, [100], [100], [100]), 0, X, y, 1e30)
    assert e.value.code == hb.HB_ERR_INVALID
    assert np.array_equal(params(m), flat) and not momenta(m).any()
