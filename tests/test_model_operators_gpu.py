"""Dropout, the policy loss and the preference loss on a handle: against a network in 64 bits (numpy) with the same masks.

Tolerances are the handle's own: relative 2-norm of every gradient tensor 1e-4 in fp32, 2e-2 in the bf16 mode (losses the same,
log-probabilities absolute).  ReLU decisions are the kernels' (read back), asserted where they are not within rounding of 0:
an activation is stored with a relative error of `step` (bf16 half a step, 2^-8; fp32 sums of up to 1024 terms 2^-14), the error of
layer l's sums is at most |W_l| times that of its inputs, and that of its activations theirs and a rounding more.
"""
import numpy as np
import pytest
import torch

import hb_inputs as hi
import operators_ref as ref
import paper_2004_08771_amd as hb

pytestmark = pytest.mark.gpu

SIG, RELU = hi.ACT_SIGMOID, hi.ACT_RELU
CE = hi.LOSS_SOFTMAX_CE


def unpack(dims, flat):
    W, b, at = [None], [None], 0
    for d_in, d_out in zip(dims[:-1], dims[1:]):
        W.append(np.asarray(flat[at:at + d_in * d_out], np.float64).reshape(d_out, d_in))
        at += d_in * d_out
        b.append(np.asarray(flat[at:at + d_out], np.float64))
        at += d_out
    return W, b


class Net:
    """Forward and backward pass in 64 bits, with the dropout masks of call `call` where p > 0."""

    def __init__(self, dims, act, flat, X, p=0.0, seed=0, call=0, on=None, step=2.0 ** -14):
        self.dims, self.act, (self.W, self.b) = dims, act, unpack(dims, flat)
        L, B = len(dims) - 1, X.shape[0]
        self.inp, self.A, self.mask = [np.asarray(X, np.float64)], [None], [None]
        self.on = [None]
        off = np.zeros_like(self.inp[0]) if step == 2.0 ** -8 else step * np.abs(self.inp[0])
        for l in range(1, L + 1):
            z = self.inp[l - 1] @ self.W[l].T + self.b[l]
            if l == L:
                self.Z = z
                return
            if act == SIG:
                a = 1 / (1 + np.exp(-z))
            else:
                off = off @ np.abs(self.W[l]).T + 2.0 ** -20
                if on is not None:
                    sure = np.abs(z) > off
                    assert sure.mean() > 0.5
                    assert np.array_equal((z > 0)[sure], on[l][sure])
                self.on.append(z > 0 if on is None else on[l])
                a = np.where(self.on[l], z, 0.0)
            keep, scale = ref.dropout_keep(B, dims[l], p, seed, 32 * call + l) if p > 0 else (np.ones_like(a), 1.0)
            self.A.append(a)
            self.mask.append(keep * scale)
            if act == RELU:
                off = (off + step * np.abs(a)) * keep * scale
            self.inp.append(a * keep * scale)

    def grads(self, delta):
        L, out = len(self.dims) - 1, []
        for l in range(L, 0, -1):
            out = [(delta.T @ self.inp[l - 1]).reshape(-1), delta.sum(0)] + out
            if l > 1:
                a = self.A[l - 1]
                d = delta @ self.W[l] * self.mask[l - 1]
                delta = d * (a * (1 - a) if self.act == SIG else self.on[l - 1])
        return out


def tensors(dims, flat):
    out, at = [], 0
    for d_in, d_out in zip(dims[:-1], dims[1:]):
        for n in (d_in * d_out, d_out):
            out.append(np.asarray(flat[at:at + n], np.float64))
            at += n
    return out


def near(got, want, tol, what):
    for i, (g, w) in enumerate(zip(got, want)):
        n = np.linalg.norm(w)
        assert np.linalg.norm(g - w) <= tol * max(n, 1e-6), f"{what}, tensor {i}: {np.linalg.norm(g - w) / max(n, 1e-30):.3g}"


def make(dims, act, dtype, B, rng, p=0.0, seed=0, call=0):
    flat = hi.xavier_uniform_params(dims, rng, bias_scale=0.2)
    X = rng.standard_normal((B, dims[0]), dtype=np.float32)
    m = hb.Model(dims, act, CE).configure(dtype, B + 3)
    if dtype == hb.HB_BF16_F32MASTER:
        dX = torch.from_numpy(X).cuda().bfloat16()
        X = dX.float().cpu().numpy()
        t = torch.from_numpy(flat)
        at, ref_flat = 0, flat.copy()
        for d_in, d_out in zip(dims[:-1], dims[1:]):   # the products read bf16 weights
            ref_flat[at:at + d_in * d_out] = t[at:at + d_in * d_out].bfloat16().float().numpy()
            at += d_in * d_out + d_out
    else:
        dX, ref_flat = torch.from_numpy(X).cuda(), flat
    m.set_params(flat)
    if p:
        m.set_dropout(p, seed, call)
    return m, flat, ref_flat, X, dX


def decisions(m, dims, B, act):
    if act != RELU:
        return None
    on = [None]
    for l in range(1, len(dims) - 1):
        a = np.empty((B, dims[l]), np.float32)
        m.get_activations(l, B, a)
        on.append(a > 0)
    return on


F32, BF16 = hb.HB_F32, hb.HB_BF16_F32MASTER
STEP = {F32: 2.0 ** -14, BF16: 2.0 ** -8}
NETS = [
    ((54, 32, 7), SIG, F32, 64), ((54, 32, 7), RELU, F32, 1), ((54, 96, 7), SIG, F32, 1000), ((40, 72, 100), RELU, F32, 333),
    ((70, 65, 129, 67, 12), RELU, F32, 321), ((54, 512, 512, 7), SIG, F32, 2048), ((300, 257, 257, 983), SIG, F32, 130), ((33, 5), SIG, F32, 77),
    ((64, 128, 96, 40), SIG, BF16, 300), ((33, 70, 51, 9), SIG, BF16, 127), ((33, 70, 51, 9), RELU, BF16, 127), ((512, 768, 512, 200), RELU, BF16, 2048),
    ((300, 1024, 1024, 33), SIG, BF16, 1001), ((128, 256, 1000), SIG, BF16, 200), ((64, 20, 24, 20, 16, 10), SIG, BF16, 65),
]

# outputs so wide that few rows are cut into chunks; bf16: their padding
WIDE = [((24, 16, 33001), SIG, F32, 6), ((24, 16, 33001), SIG, BF16, 6), ((24, 16, 50003), SIG, BF16, 70)]


@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("dims,act,dtype,B", NETS + WIDE)
def test_policy_gradient_of_a_network(dims, act, dtype, B, p):
    rng = np.random.default_rng(B + len(dims))
    seed, call, K = 987654321012345, 11, dims[-1]
    m, flat, ref_flat, X, dX = make(dims, act, dtype, B, rng, p, seed, call)
    y = rng.integers(0, K, B).astype(np.int32)
    if B > 5:
        y[3::10] = -1
    adv = rng.standard_normal(B).astype(np.float32)
    # log-ratios away from the borders of the clip by more than either precision moves them
    base = Net(dims, act, ref_flat, X, p, seed, call)
    _, lp, _, _ = ref.rows_ref(base.Z, y)
    old = (lp - rng.choice([-0.8, -0.05, 0.0, 0.05, 0.8], B)).astype(np.float32)
    refs = (lp + 0.3 * rng.standard_normal(B)).astype(np.float32)
    w = (rng.uniform(0.5, 1.5, B) / B).astype(np.float32)
    vec = lambda a, t=torch.float32: torch.as_tensor(np.asarray(a)).to(t).cuda()  # noqa: E731
    keep_alive = [vec(old), vec(adv), vec(refs), vec(w)]
    args = hb.policy_args(B, keep_alive[0], keep_alive[1], ref=keep_alive[2], weight=keep_alive[3], clip=(0.2, 0.3), kl_coef=0.05)
    dy, g = vec(y, torch.int32), torch.full((m.num_params,), float("nan"), device="cuda")
    stats, logp = torch.zeros(4, device="cuda"), torch.zeros(B, device="cuda")
    m.policy_grad_async(dX, dy, B, args, g, stats, logp)
    torch.cuda.synchronize()
    on = decisions(m, dims, B, act)
    net = Net(dims, act, ref_flat, X, p, seed, call, on, STEP[dtype])
    want_stats, want_lp, dZ, _ = ref.policy_ref(net.Z, y, old, adv, refs, w, (0.2, 0.3), 0.05)
    tol = 1e-4 if dtype == F32 else 2e-2
    near(tensors(dims, g.cpu().numpy()), net.grads(dZ), tol, "gradient")
    assert np.abs(logp.cpu().numpy() - want_lp).max() <= tol * (1 + np.abs(want_lp).max())
    assert np.abs(stats.cpu().numpy() - want_stats).max() <= tol * max(1.0, np.abs(want_stats).max())
    after = np.empty_like(flat)
    m.get_params(after)
    assert np.array_equal(after, flat)                       # a gradient leaves the replica
    # the step applies it; its masks are those of the next call
    lr = 0.05
    if p:
        m.set_dropout(p, seed, call)
    m.policy_step_async(dX, dy, B, lr, args, stats)
    m.get_params(after)
    near([a - f for a, f in zip(tensors(dims, after), tensors(dims, flat))], [-lr * t for t in net.grads(dZ)],
         2 * tol if dtype == BF16 else 1e-3, "step")         # a difference of stored parameters: their rounding, too
    m.destroy()


@pytest.mark.parametrize("p", [0.0, 0.2])
@pytest.mark.parametrize("dims,act,dtype,B", [NETS[0], NETS[3], NETS[5], NETS[8], NETS[9], NETS[12]] + WIDE)
def test_preference_gradient_of_a_network(dims, act, dtype, B, p):
    rng = np.random.default_rng(7 * B + len(dims))
    seed, call, K, pairs = 5, 2 ** 40, dims[-1], 3
    m, flat, ref_flat, X, dX = make(dims, act, dtype, B, rng, p, seed, call)
    y = rng.integers(0, K, B).astype(np.int32)
    y[5::9] = K
    seq = np.concatenate([[2], np.sort(rng.integers(2, B - 1, 2 * pairs - 1)), [B - 2]]).astype(np.int32)
    refs = None
    net = Net(dims, act, ref_flat, X, p, seed, call)
    _, s, _, _ = ref.preference_ref(net.Z, y, seq, None, 0.1, 0.0)
    refs = (s + 2 * rng.standard_normal(2 * pairs)).astype(np.float32)
    dseq, dref = torch.from_numpy(seq).cuda(), torch.from_numpy(refs).cuda()
    args = hb.preference_args(dseq, dref, beta=0.2, smoothing=0.1)
    g, stats, sl = torch.zeros(m.num_params, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(2 * pairs, device="cuda")
    m.preference_grad_async(dX, torch.from_numpy(y).cuda(), B, args, g, stats, sl)
    torch.cuda.synchronize()
    net = Net(dims, act, ref_flat, X, p, seed, call, decisions(m, dims, B, act), STEP[dtype])
    want, s, dZ, _ = ref.preference_ref(net.Z, y, seq, refs, 0.2, 0.1)
    tol = 1e-4 if dtype == F32 else 2e-2
    near(tensors(dims, g.cpu().numpy()), net.grads(np.nan_to_num(dZ)), tol, "gradient")
    assert np.abs(sl.cpu().numpy() - s).max() <= tol * (1 + np.abs(s).max())
    m.preference_step_async(dX, torch.from_numpy(y).cuda(), B, 0.1, args, stats)
    after = np.empty_like(flat)
    m.get_params(after)
    assert np.isfinite(after).all() and not np.array_equal(after, flat)
    m.destroy()


@pytest.mark.parametrize("dims,act,dtype,B", NETS)
def test_dropout_of_the_labelled_loss(dims, act, dtype, B):
    rng = np.random.default_rng(3 * B + len(dims))
    p, seed, K = 0.25, 77, dims[-1]
    m, flat, ref_flat, X, dX = make(dims, act, dtype, B, rng, p, seed, 0)
    y = rng.integers(0, K, B).astype(np.int32)
    dy, g = torch.from_numpy(y).cuda(), torch.zeros(m.num_params, device="cuda")
    tol = 1e-4 if dtype == F32 else 2e-2
    for call in range(2):                                   # the second call has other masks
        loss = m.batch_grad(dX, dy, B, g)
        net = Net(dims, act, ref_flat, X, p, seed, call, decisions(m, dims, B, act), STEP[dtype])
        part, lp, _, prob = ref.rows_ref(net.Z, y)
        near(tensors(dims, g.cpu().numpy()), net.grads(ref.grad_ref(part, prob, y, np.full(B, -1.0 / B))), tol, f"call {call}")
        assert abs(loss + lp.mean()) <= tol * abs(lp.mean())
    plain = Net(dims, act, ref_flat, X)
    _, lp, _, _ = ref.rows_ref(plain.Z, y)
    assert abs(m.batch_loss(dX, dy, B) + lp.mean()) <= tol * abs(lp.mean())   # a loss has no dropout
    out = torch.zeros(B, device="cuda")
    m.batch_logprob_async(dX, dy, B, out)
    assert np.abs(out.cpu().numpy() - lp).max() <= tol * (1 + np.abs(lp).max())
    m.set_dropout(0.0)
    loss = m.batch_grad(dX, dy, B, g)
    other = hb.Model(dims, act, CE).configure(dtype, B + 3)
    other.set_params(flat)
    h = torch.zeros_like(g)
    assert other.batch_grad(dX, dy, B, h) == loss and torch.equal(g, h)       # off: what a handle without it gives
    m.destroy()
    other.destroy()


def test_dropout_of_a_csr_step():
    rng = np.random.default_rng(6)
    dims, B, p, seed = (200, 64, 48, 3), 150, 0.4, 21
    dense = np.where(rng.random((B, dims[0])) < 0.1, rng.standard_normal((B, dims[0])), 0.0).astype(np.float32)
    rows = np.concatenate([[0], np.cumsum((dense != 0).sum(1))]).astype(np.int32)
    cols, vals = np.nonzero(dense)[1].astype(np.int32), dense[dense != 0]
    flat = hi.xavier_uniform_params(dims, rng, bias_scale=0.2)
    y = rng.integers(0, 3, B).astype(np.int32)
    m = hb.Model(dims, SIG, CE).configure(F32, B, sparse_first_layer=True)
    m.set_params(flat)
    m.set_dropout(p, seed, 4)
    t = [torch.from_numpy(a).cuda() for a in (rows, cols, vals, y)]
    g = torch.zeros(m.num_params, device="cuda")
    m.batch_grad_csr(t[0], t[1], t[2], len(vals), t[3], B, g)
    net = Net(dims, SIG, flat, dense, p, seed, 4)
    part, _, _, prob = ref.rows_ref(net.Z, y)
    near(tensors(dims, g.cpu().numpy()), net.grads(ref.grad_ref(part, prob, y, np.full(B, -1.0 / B))), 1e-4, "csr")
    m.destroy()


def test_dropout_in_the_worker_loop():
    """An epoch of the GPU worker's loop with dropout is its steps, one call each."""
    rng = np.random.default_rng(8)
    dims, n, b = (20, 40, 4), 256, 32
    X, y = rng.standard_normal((n, 20), dtype=np.float32), rng.integers(0, 4, n).astype(np.int32)
    flat = hi.xavier_uniform_params(dims, rng, bias_scale=0.2)
    out = []
    for loop in (True, False):
        m = hb.Model(dims, RELU, CE).configure(F32, b)
        m.set_params(flat)
        m.set_dropout(0.3, 9, 100)
        if loop:
            m.worker_run_epoch(hb.Sched(n, [b], [b], [b]), 0, X, y, 0.01)
        else:
            for i in range(0, n, b):
                m.batch_step_async(torch.from_numpy(X[i:i + b]).cuda(), torch.from_numpy(y[i:i + b]).cuda(), b, np.float32(0.01) * b)
        out.append(np.empty_like(flat))
        m.get_params(out[-1])
        m.destroy()
    near(tensors(dims, out[0]), tensors(dims, out[1]), 1e-6, "epoch")


def test_a_policy_learns_from_itself():
    """As it is used: the log-probabilities of the policy when it acted and of a reference, then steps with dropout."""
    rng = np.random.default_rng(12)
    dims, act, B, p, seed, lr = (30, 48, 48, 6), SIG, 200, 0.1, 3, 0.5
    m, flat, _, X, dX = make(dims, act, F32, B, rng)
    reference, flat_ref, _, _, _ = make(dims, act, F32, B, rng)
    y, adv = rng.integers(0, 6, B).astype(np.int32), rng.standard_normal(B).astype(np.float32)
    dy, dadv = torch.from_numpy(y).cuda(), torch.from_numpy(adv).cuda()
    old, refs, stats = torch.zeros(B, device="cuda"), torch.zeros(B, device="cuda"), torch.zeros(4, device="cuda")
    m.batch_logprob_async(dX, dy, B, old)
    reference.batch_logprob_async(dX, dy, B, refs)
    m.set_dropout(p, seed)
    args = hb.policy_args(B, old, dadv, ref=refs, clip=(0.9, 3.0), kl_coef=0.02)
    host = flat.astype(np.float64)
    h_old = ref.rows_ref(Net(dims, act, flat, X).Z, y)[1]
    h_ref = ref.rows_ref(Net(dims, act, flat_ref, X).Z, y)[1]
    for step in range(3):
        m.policy_step_async(dX, dy, B, lr, args, stats)
        net = Net(dims, act, host, X, p, seed, step)
        want, _, dZ, _ = ref.policy_ref(net.Z, y, h_old, adv, h_ref, None, (0.9, 3.0), 0.02)
        assert np.abs(stats.cpu().numpy() - want).max() <= 1e-4
        host = host - lr * np.concatenate(net.grads(dZ))
    after = np.empty_like(flat)
    m.get_params(after)
    near(tensors(dims, after), tensors(dims, host), 1e-4, "after three steps")
    m.destroy()
    reference.destroy()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_captured_step_with_dropout(dtype):
    rng = np.random.default_rng(4)
    dims, B, p, lr = (64, 96, 64, 40), 129, 0.2, 0.1
    st = torch.cuda.Stream()
    flat = hi.xavier_uniform_params(dims, rng, bias_scale=0.2)
    ms = [hb.Model(dims, RELU, CE).configure(dtype, B, stream=st.cuda_stream) for _ in range(2)]
    X = torch.from_numpy(rng.standard_normal((B, 64), dtype=np.float32)).cuda().to(torch.bfloat16 if dtype == BF16 else torch.float32)
    dy = torch.from_numpy(rng.integers(0, 40, B).astype(np.int32)).cuda()
    old, adv = torch.full((B,), -3.7, device="cuda"), torch.from_numpy(rng.standard_normal(B).astype(np.float32)).cuda()
    args = hb.policy_args(B, old, adv)
    stats = [torch.zeros(4, device="cuda") for _ in ms]
    torch.cuda.synchronize()
    for m in ms:
        m.set_params(flat)
        m.policy_step_async(X, dy, B, lr, args, stats[0])    # the first call allocates
        m.set_dropout(p, 8, 50)
        m.set_params(flat)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        ms[0].policy_step_async(X, dy, B, lr, args, stats[0])
    a, b = np.empty_like(flat), np.empty_like(flat)
    for k in range(5):
        g.replay()
        torch.cuda.synchronize()
        ms[1].set_dropout(p, 8, 50)                          # a replay has the masks of the captured call
        ms[1].policy_step_async(X, dy, B, lr, args, stats[1])
        ms[0].get_params(a)
        ms[1].get_params(b)
        assert np.array_equal(a, b) and torch.equal(stats[0], stats[1]), k
    for m in ms:
        m.destroy()


def test_refusals_of_a_handle():
    m = hb.Model((8, 16, 4), SIG, CE).configure(F32, 32)
    log = hb.Model((8, 16, 2), SIG, hi.LOSS_LOGISTIC).configure(F32, 32)
    csr = hb.Model((8, 16, 4), SIG, CE).configure(F32, 32, sparse_first_layer=True)
    X, y, v = torch.zeros(32, 8, device="cuda"), torch.zeros(32, dtype=torch.int32, device="cuda"), torch.zeros(32, device="cuda")
    st, seq = torch.zeros(4, device="cuda"), torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    pol, prf = hb.policy_args(32, v, v), hb.preference_args(seq)
    bad_pol = hb.policy_args(32, v, v, clip=(-1.0, 0.2))
    many = hb.preference_args(torch.zeros(2 * 33 + 1, dtype=torch.int32, device="cuda"))
    g = torch.zeros(m.num_params, device="cuda")
    for call in (lambda: log.policy_step_async(X, y, 32, 0.1, pol, st), lambda: log.batch_logprob_async(X, y, 32, v),
                 lambda: csr.policy_step_async(X, y, 32, 0.1, pol, st), lambda: csr.preference_step_async(X, y, 32, 0.1, prf, st),
                 lambda: m.policy_step_async(X, y, 33, 0.1, pol, st), lambda: m.policy_step_async(X, y, 0, 0.1, pol, st),
                 lambda: m.policy_step_async(None, y, 32, 0.1, pol, st), lambda: m.policy_step_async(X, None, 32, 0.1, pol, st),
                 lambda: m.policy_step_async(X, y, 32, float("nan"), pol, st), lambda: m.policy_step_async(X, y, 32, 0.1, pol, None),
                 lambda: m.policy_step_async(X, y, 32, 0.1, bad_pol, st), lambda: m.policy_grad_async(X, y, 32, pol, None, st),
                 lambda: m.preference_step_async(X, y, 32, 0.1, many, st), lambda: m.preference_grad_async(X, y, 32, prf, None, st),
                 lambda: m.preference_grad_async(X, y, 32, prf, g, None), lambda: m.batch_logprob_async(X, y, 32, None),
                 lambda: m.policy_step_async(X, y, 32, 0.1, pol, st, v), lambda: m.policy_step_async(X, y, 32, 0.1, pol, v),
                 lambda: m.preference_step_async(X, y, 32, 0.1, prf, st, st), lambda: m.batch_logprob_async(X, y, 32, v, v),
                 lambda: m.set_dropout(1.0), lambda: m.set_dropout(-0.1), lambda: m.set_dropout(0.1, 0, 1 << 59)):
        with pytest.raises(hb.HbError) as e:
            call()
        assert e.value.code == hb.HB_ERR_INVALID
    fresh = hb.Model((8, 16, 4), SIG, CE)
    for call in (lambda: fresh.set_dropout(0.5), lambda: fresh.policy_step_async(X, y, 32, 0.1, pol, st),
                 lambda: fresh.batch_logprob_async(X, y, 32, v), lambda: fresh.preference_grad_async(X, y, 32, prf, g, st)):
        with pytest.raises(hb.HbError) as e:
            call()
        assert e.value.code == hb.HB_ERR_STATE
    for t in (m, log, csr):
        t.destroy()
