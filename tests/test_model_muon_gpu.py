"""Orthogonalised updates and scores on a handle, and the operators as a training step uses them together.

An update is compared with its definition on the gradient that the handle itself gives for the same batch (the same kernels make it in a step): the
tolerances are those of the operators' tests, for the update lr scale sqrt(max(d_l, d_l-1)) times that of the orthogonalised matrix, for
weights three roundings of 2^-24 each.
"""
import numpy as np
import pytest
import torch

import more_operators_ref as ref
import paper_2004_08771_amd as hb
from test_model_operators_gpu import unpack
from test_operators_gpu import U, host, vec
from test_ortho_gpu import norm, tolerance, work

pytestmark = pytest.mark.gpu


def model(dims, act=hb.HB_ACT_RELU, loss=hb.HB_LOSS_SOFTMAX_CE, bf16=False, max_B=300, seed=0):
    m = hb.Model(dims, act, loss).configure(hb.HB_BF16_F32MASTER if bf16 else hb.HB_F32, max_B, False, torch.cuda.current_stream().cuda_stream)
    rng = np.random.default_rng(seed)
    flat = np.concatenate([np.concatenate([(rng.standard_normal(o * i) * np.sqrt(2 / (i + o))), 0.1 * rng.standard_normal(o)])
                           for i, o in zip(dims[:-1], dims[1:])]).astype(np.float32)
    m.set_params(flat)
    return m, flat


def batch(dims, B, bf16=False, seed=1):
    rng = np.random.default_rng(seed)
    X = torch.as_tensor(rng.standard_normal((B, dims[0]))).to(torch.bfloat16 if bf16 else torch.float32).cuda()
    return X, vec(rng.integers(0, dims[-1], B), torch.int32)


def params(m):
    out = np.empty(m.num_params, np.float32)
    m.get_params(out)
    return out


def momenta(m):
    out = np.empty(m.num_params, np.float32)
    m.get_momenta(out)
    return out


def check_step(dims, before, after, grad, m0, m1, lr, first, last, scale, products, momentum, nesterov, decay, tiles):
    W0, b0 = unpack(dims, before)
    W1, b1 = unpack(dims, after)
    G, gb = unpack(dims, grad)
    M0, _ = unpack(dims, m0)
    M1, _ = unpack(dims, m1)
    f = lambda v: float(np.float32(v))  # noqa: E731
    for l in range(1, len(dims)):
        assert (np.abs(b1[l] - (b0[l] - f(lr) * gb[l])) <= 2 * U * (np.abs(b0[l]) + abs(lr) * np.abs(gb[l]))).all()
        if not first <= l <= last:
            assert (np.abs(W1[l] - (W0[l] - f(lr) * G[l])) <= 2 * U * (np.abs(W0[l]) + abs(lr) * np.abs(G[l]))).all()
            assert np.array_equal(M1[l], M0[l])
            continue
        s = f(scale) * np.sqrt(max(dims[l], dims[l - 1]))
        want_w, want_m, O = ref.muon_ref(W0[l], G[l], M0[l], lr, momentum, nesterov, decay, s)
        assert (np.abs(M1[l] - want_m) <= 2 * U * (momentum * np.abs(M0[l]) + np.abs(G[l])) + 1e-30).all()
        u = G[l] + f(momentum) * want_m if nesterov else want_m
        _, tol = tolerance(u, products, tiles=tiles)
        off = norm(W1[l] - want_w)
        assert off <= lr * s * (tol + 485 * 3 * U) + 3 * U * (norm(W0[l]) + lr * s * norm(O)), (l, off)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("dims,B", [((54, 32, 7), 64), ((54, 160, 96, 7), 200), ((40, 150, 150, 33), 300), ((17, 5), 9)])
def test_steps(dims, B, bf16):
    products = "bf16" if bf16 else "f32"
    first, last = (1, len(dims) - 1) if B != 200 else (2, len(dims) - 2)
    tiles = any(min(dims[l], dims[l - 1]) > 128 for l in range(first, last + 1))
    m, flat = model(dims, bf16=bf16)
    how = hb.muon_args(momentum=0.9, nesterov=B != 64, weight_decay=0.1, products=hb.HB_TENSOR_BF16 if bf16 else hb.HB_TENSOR_F32)
    m.set_muon(how, first, last, 0.3)
    loss = torch.zeros(1, device="cuda")
    for k in range(2):
        X, y = batch(dims, B, bf16, seed=k)
        before, m0, grad = params(m), momenta(m), torch.zeros(m.num_params, device="cuda")
        want_loss = m.batch_grad(X, y, B, grad)
        m.batch_step_async(X, y, B, 0.02, loss)
        after, m1 = params(m), momenta(m)
        assert float(loss) == pytest.approx(want_loss, abs=0)
        check_step(dims, before, after, grad.cpu().numpy(), m0, m1, 0.02, first, last, 0.3, products, 0.9, B != 64, 0.1, tiles)
    # what is derived from the weights follows them
    other, _ = model(dims, bf16=bf16)
    other.set_params(params(m))
    assert m.batch_loss(X, y, B) == other.batch_loss(X, y, B)
    # off: plain steps again, as a handle's that never had it
    m.set_muon(None)
    m.batch_step_async(X, y, B, 0.02)
    other.batch_step_async(X, y, B, 0.02)
    assert np.array_equal(params(m), params(other))


def test_policy_preference_and_dropout_steps():
    dims, B = (20, 70, 40, 11), 120
    X, y = batch(dims, B)
    rng = np.random.default_rng(2)
    old, adv = vec(-2 + 0.1 * rng.standard_normal(B)), vec(rng.standard_normal(B))
    seq = vec([0, 30, 60, 80, 120], torch.int32)
    policy, preference = hb.policy_args(B, old, adv), hb.preference_args(seq)
    stats, stats2 = torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda")
    for step, grad in [(lambda m: m.policy_step_async(X, y, B, 0.01, policy, stats), lambda m, g: m.policy_grad_async(X, y, B, policy, g, stats2)),
                       (lambda m: m.preference_step_async(X, y, B, 0.01, preference, stats),
                        lambda m, g: m.preference_grad_async(X, y, B, preference, g, stats2))]:
        for p in (0.0, 0.25):
            m, flat = model(dims)
            g = torch.zeros(m.num_params, device="cuda")
            m.set_dropout(p, 5, 3)
            grad(m, g)
            m.set_muon(hb.muon_args(), scale=0.2)
            m.set_dropout(p, 5, 3)
            step(m)
            assert torch.equal(stats, stats2)
            zero = np.zeros_like(flat)
            check_step(dims, flat, params(m), g.cpu().numpy(), zero, momenta(m), 0.01, 1, 3, 0.2, "f32", 0.95, True, 0.0, False)


def test_momenta_of_a_checkpoint():
    dims, B = (30, 20, 5), 40
    X, y = batch(dims, B)
    a, flat = model(dims)
    a.set_muon(hb.muon_args(coef=[(3.4445, -4.775, 2.0315)] * 3, steps=3))
    for _ in range(3):
        a.batch_step_async(X, y, B, 0.01)
    b, _ = model(dims)
    b.set_muon(hb.muon_args(coef=[(3.4445, -4.775, 2.0315)] * 3, steps=3))
    b.set_params(params(a))
    b.set_momenta(momenta(a))
    for m in (a, b):
        m.batch_step_async(X, y, B, 0.01)
    assert np.array_equal(params(a), params(b)) and np.array_equal(momenta(a), momenta(b))
    assert np.abs(momenta(a)).max() > 0
    a.set_muon(hb.muon_args())
    assert not momenta(a).any()


def test_steps_in_a_graph():
    dims, B = (30, 40, 5), 50
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        X, y = batch(dims, B)
        (a, flat), (b, _) = model(dims), model(dims)
        for m in (a, b):
            m.set_muon(hb.muon_args())
            m.batch_step_async(X, y, B, 0.01)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        a.batch_step_async(X, y, B, 0.01)
    for _ in range(3):
        with torch.cuda.stream(stream):
            X.normal_()
            graph.replay()
            b.batch_step_async(X, y, B, 0.01)
        stream.synchronize()
        assert np.array_equal(params(a), params(b))


def test_worker_loop_and_profile():
    dims, n = (12, 24, 4), 600
    rng = np.random.default_rng(0)
    X, y = rng.standard_normal((n, dims[0])).astype(np.float32), rng.integers(0, 4, n).astype(np.int32)
    m, flat = model(dims)
    m.set_muon(hb.muon_args())
    s = hb.Sched(n, [100], [100], [100])
    _, steps, loss = m.worker_run_epoch(s, 0, X, y, 1e-4)
    assert steps == 6 and np.isfinite(loss) and np.isfinite(params(m)).all() and not np.array_equal(params(m), flat)
    dX, dy = torch.as_tensor(X[:100]).cuda(), vec(y[:100], torch.int32)
    m.profile_enable()
    m.batch_step_async(dX, dy, 100, 0.01)
    kinds = {(r["kind"], r["layer"]) for r in m.profile_read()}
    assert (7, 8) in kinds and (4, 0) in kinds


def test_refusals():
    dims = (12, 24, 4)
    m, _ = model(dims)
    buf = np.zeros(m.num_params, np.float32)

    def code(call):
        with pytest.raises(hb.HbError) as e:
            call()
        return e.value.code

    assert code(lambda: m.get_momenta(buf)) == code(lambda: m.set_momenta(buf)) == hb.HB_ERR_STATE
    for first, last, scale in [(0, 1, 0.2), (2, 1, 0.2), (1, 3, 0.2), (1, 2, float("nan"))]:
        assert code(lambda: m.set_muon(hb.muon_args(), first, last, scale)) == hb.HB_ERR_INVALID
    for how in (hb.muon_args(momentum=1.0), hb.muon_args(steps=0, coef=(1, 0, 0)), hb.muon_args(weight_decay=-1.0)):
        assert code(lambda: m.set_muon(how)) == hb.HB_ERR_INVALID
    sparse = hb.Model(dims, hb.HB_ACT_RELU, hb.HB_LOSS_LOGISTIC if dims[-1] <= 2 else hb.HB_LOSS_SOFTMAX_CE).configure(hb.HB_F32, 64, True)
    assert code(lambda: sparse.set_muon(hb.muon_args())) == hb.HB_ERR_UNSUPPORTED
    X, y = batch(dims, 20)
    row, c = torch.zeros(20, device="cuda"), torch.zeros(20, 2, dtype=torch.int32, device="cuda")
    assert code(lambda: m.batch_scores_async(X, None, 20, d_logp=row)) == hb.HB_ERR_INVALID
    assert code(lambda: m.batch_scores_async(X, y, 20, d_logp=row, d_lse=row)) == hb.HB_ERR_INVALID
    assert code(lambda: m.batch_scores_async(X, y, 20, d_entropy=X.view(-1)[:20])) == hb.HB_ERR_INVALID
    assert code(lambda: m.batch_scores_async(X, y, 20, d_top_class=torch.zeros(20, 65, dtype=torch.int32, device="cuda"))) == hb.HB_ERR_INVALID
    assert code(lambda: m.batch_scores_async(X, y, 301, d_top_class=c)) == hb.HB_ERR_INVALID
    logistic = hb.Model((12, 2), hb.HB_ACT_RELU, hb.HB_LOSS_LOGISTIC).configure(hb.HB_F32, 64)
    assert code(lambda: logistic.batch_scores_async(X, y, 20, d_top_class=c)) == hb.HB_ERR_INVALID


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("dims,B", [((54, 32, 7), 64), ((20, 70, 983), 77)])
def test_scores_of_a_network(dims, B, bf16):
    """The classes and the normalisers of the network's logits, which a network in torch gives to 1e-4 (bf16 mode 2e-2); the log-probabilities are those
    of the call that has only them."""
    m, flat = model(dims, bf16=bf16)
    X, y = batch(dims, B, bf16)
    y[::7] = -1
    logp, logp2, lse, lse2, H = (torch.zeros(B, device="cuda") for _ in range(5))
    c, t = torch.zeros(B, 5, dtype=torch.int32, device="cuda"), torch.zeros(B, 5, device="cuda")
    m.batch_logprob_async(X, y, B, logp2, lse2)
    m.batch_scores_async(X, y, B, logp, lse, H, c, t)
    assert float((logp - logp2).abs().max()) < 1e-5 and float((lse - lse2).abs().max()) < 1e-5
    W, b = unpack(dims, flat)
    a = host(X)
    for l in range(1, len(dims)):
        a = a @ W[l].T + b[l]
        a = np.maximum(a, 0) if l < len(dims) - 1 else a
    tol = 2e-2 * np.abs(a).max() if bf16 else 1e-4
    part, _, _, want_H, classes, tops, _, _ = ref.scores_ref(a, y.cpu().numpy(), 5)
    assert np.abs(host(H) - want_H).max() < 4 * tol * (1 + np.log(dims[-1])) and np.abs(host(t) - tops)[part].max() < 4 * tol
    got = c.cpu().numpy()
    assert (got[~part] == -1).all()
    for i in np.nonzero(part)[0]:  # in order but for logits that are as near as that
        assert len(set(got[i])) == 5 and np.abs(a[i][got[i]] - a[i][classes[i]]).max() < 4 * tol
    m.batch_scores_async(X, None, B, d_top_class=c)
    assert (c[:, 0] >= 0).all()


def test_a_policy_step_of_a_network_elsewhere():
    """Scores, their gradient and the orthogonalised update together, as a training step with an entropy bonus makes it, against the step in 64 bits."""
    rng = np.random.default_rng(4)
    B, d, h, K = 50, 40, 60, 30
    x = rng.standard_normal((B, d)).astype(np.float32)
    W = [(rng.standard_normal((h, d)) * 0.2).astype(np.float32), (rng.standard_normal((K, h)) * 0.2).astype(np.float32)]
    y, adv = rng.integers(0, K, B), rng.standard_normal(B).astype(np.float32) / B
    X, V, M = vec(x), [vec(w) for w in W], [torch.zeros(w.shape, device="cuda") for w in W]
    scores_ws = torch.empty(hb.scores_workspace_bytes(B, K, 3), dtype=torch.uint8, device="cuda")
    ws = work([w.shape for w in W], "f32")
    W64 = [w.astype(np.float64) for w in W]
    M64 = [np.zeros(w.shape) for w in W]
    g_h = np.full(B, 0.01 / B, np.float32)
    for step in range(2):
        A = X @ V[0].T
        R = torch.relu(A)
        Z = (R @ V[1].T).contiguous()
        logp, H, top = torch.zeros(B, device="cuda"), torch.zeros(B, device="cuda"), torch.zeros(B, 3, dtype=torch.int32, device="cuda")
        hb.scores(Z, vec(y, torch.int32), logp=logp, entropy=H, top_class=top, ws=scores_ws)
        dZ = torch.empty_like(Z)
        hb.scores_grad(Z, dZ, vec(y, torch.int32), -vec(adv), -vec(g_h), ws=scores_ws)
        dA = (dZ @ V[1]) * (A > 0)
        G = [(dA.T @ X).contiguous(), (dZ.T @ R).contiguous()]
        hb.muon_update(V, G, M, 0.02, ws=ws)

        a = x.astype(np.float64) @ W64[0].T
        r = np.maximum(a, 0)
        z = r @ W64[1].T
        s = ref.scores_ref(z, y, 3)
        assert np.abs(host(logp) - s[1]).max() < 1e-3 and np.abs(host(H) - s[3]).max() < 1e-3 and top.shape == (B, 3)
        dz = ref.scores_grad_ref(s, y, -adv, -g_h)
        da = (dz @ W64[1]) * (a > 0)
        for i, g in enumerate([da.T @ x.astype(np.float64), dz.T @ r]):
            # fp32 products of depth 60 and the logits' roundings: 1e-5 of the gradient, which small singular values have 485 times
            assert norm(host(G[i]) - g) < 1e-4 * norm(g), (step, i)
            W64[i], M64[i], O = ref.muon_ref(W64[i], g, M64[i], 0.02, scale=0.2 * np.sqrt(max(W[i].shape)))
            assert norm(host(V[i]) - W64[i]) < 0.02 * 0.2 * np.sqrt(max(W[i].shape)) * 485 * 1e-4 * norm(O) * (step + 1)
