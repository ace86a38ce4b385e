"""The worker loop of a handle with orthogonalised updates trains the steps that its batches make one by one."""
import numpy as np
import pytest
import torch

import paper_2004_08771_amd as hb
from test_model_muon_gpu import model, momenta, params
from test_operators_gpu import vec

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("dims", [(12, 24, 4), (40, 150, 140, 9)])
def test_an_epoch_is_its_steps(dims, bf16):
    n, B, rate = 650, 100, np.float32(1e-4)
    rng = np.random.default_rng(0)
    X = torch.as_tensor(rng.standard_normal((n, dims[0]))).to(torch.bfloat16 if bf16 else torch.float32)
    y = rng.integers(0, dims[-1], n).astype(np.int32)
    how = hb.muon_args(momentum=0.9, weight_decay=0.1, products=hb.HB_TENSOR_BF16 if bf16 else hb.HB_TENSOR_F32)
    (a, flat), (b, _), (plain, _) = (model(dims, bf16=bf16) for _ in range(3))
    for m in (a, b):
        m.set_muon(how, 1, len(dims) - 1, 0.3)
    for m in (a, plain):
        _, steps, loss = m.worker_run_epoch(hb.Sched(n, [B], [B], [B]), 0, X.contiguous(), y, rate)
        assert steps == 6 and np.isfinite(loss)
        if m is a:
            of_epoch = loss
    each = torch.zeros(6, device="cuda")
    dX, dy = X.cuda(), vec(y, torch.int32)
    for k in range(6):
        b.batch_step_async(dX[k * B:(k + 1) * B], dy[k * B:(k + 1) * B], B, float(rate * np.float32(B)), each[k:k + 1])
    assert np.array_equal(params(a), params(b)) and np.array_equal(momenta(a), momenta(b)) and np.abs(momenta(a)).max() > 0
    assert of_epoch == float(each.double().sum())
    assert not np.array_equal(params(a), params(plain)) and not np.array_equal(params(a), flat)


def test_momenta_stay_where_updates_are_switched_off():
    dims, B = (30, 20, 5), 40
    m, flat = model(dims)
    rng = np.random.default_rng(1)
    X, y = torch.as_tensor(rng.standard_normal((B, dims[0]))).float().cuda(), vec(rng.integers(0, 5, B), torch.int32)
    m.set_muon(hb.muon_args())
    m.batch_step_async(X, y, B, 0.01)
    kept = momenta(m)
    assert kept.any()
    m.set_muon(None)
    m.batch_step_async(X, y, B, 0.01)
    assert np.array_equal(momenta(m), kept)
    m.set_muon(hb.muon_args())
    assert not momenta(m).any()
