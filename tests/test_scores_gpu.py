"""Scores of rows of logits and their gradient against the definitions in 64 bits.

Tolerances, with U = 2^-24 and eps_s, lp_tol of the log-probabilities' tests (an exponential is off by (T + 4) U relative, sums in chains add up):
  log s is off by eps_s absolute, and by eps_s relative where it is small (the sum without the largest term has that relative error).
  h / s = sum of p u: every term off by (T + 6) U + its exponential's error, relative: 2 eps_s relative of the sum of |terms|, which is the
  entropy less log s.  So an entropy is off by 3 eps_s relative, and by the rounding of the result.  (T of a term that counts: 17 + log K.)
  dz = -p (gl + gh (log p + H)) + [k = y] gl: p off by eps_s + (T' + 8) U relative with T' the distance from the maximum; log p + H by its terms' errors,
  (T' + H + 1) 3 eps_s.  A bf16 result adds 2^-8 relative (2^-133 absolute near zero).
Classes are equal.  Their logits are compared as stored, so nothing is lost there.
"""
import numpy as np
import pytest
import torch

import more_operators_ref as ref
import paper_2004_08771_amd as hb
from test_operators_gpu import TYPES, U, check, eps_s, host, lp_tol, matrix, outside_is_nan, vec

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (3, 2), (64, 7), (257, 3), (5, 63), (9, 64), (7, 65), (130, 100), (33, 255), (6, 257), (11, 300), (50, 983), (3, 1030),
          (5, 2049), (4, 4100), (3, 8200), (2, 9001), (2, 17000), (65, 20001), (2, 33000), (66, 33003), (1, 50257), (65, 53300), (3, 65600),
          (65, 70001), (1, 131072), (65, 131100), (1, 165000), (66, 90001)]
TOPS = [0, 1, 2, 5, 20, 64]


def logits(B, K, rng, dtype, plain=False):
    z = (2.0 * rng.standard_normal((B, K))).astype(np.float32)
    y = rng.integers(0, K, B).astype(np.int32)
    if not plain:
        if K > 2:
            z[rng.random((B, K)) < 0.15] = -np.inf
            z[rng.random((B, K)) < 0.05] = torch.finfo(TYPES[dtype]).min
        for i in range(B):
            kind = (i + K) % 13
            if kind == 3:
                y[i] = [-1, K, -2 ** 31, 2 ** 31 - 1][(i // 13) % 4]
                z[i, rng.integers(0, K)] = np.nan
            elif kind == 5:
                z[i] = -np.inf
            elif kind == 7:
                z[i, rng.integers(0, K)] = 40.0       # all but certain
            elif kind == 8:
                z[i, y[i]] = 40.0
            elif kind == 9:
                z[i] = rng.integers(-1, 3, K)          # many equal
            elif kind == 10:
                z[i] = 1.5
            elif kind == 11:
                z[i] = np.sort(rng.standard_normal(K))[::1 if i % 2 else -1]
            elif kind == 12:
                z[i] = np.where(rng.random(K) < 0.5, 0.0, -0.0)
    return torch.as_tensor(z).to(TYPES[dtype]).double().numpy(), y


def work(B, K, top=0):
    return torch.full((hb.scores_workspace_bytes(B, K, top),), 0xFF, dtype=torch.uint8, device="cuda")


def entropy_tol(H, K):
    return 3 * eps_s(K) * np.abs(np.where(np.isfinite(H), H, 0.0)) + U * np.abs(np.where(np.isfinite(H), H, 0.0)) + 1e-37


def run(Z, y, top, ws=None):
    B, K = Z.shape
    out = [torch.full((B,), 7.0, device="cuda") for _ in range(3)]
    c, t = torch.full((B, top), 7, dtype=torch.int32, device="cuda"), torch.full((B, top), 7.0, device="cuda")
    hb.scores(Z, y, logp=None if y is None else out[0], lse=out[1], entropy=out[2], top_class=c, top_logp=t, ws=work(B, K, top) if ws is None else ws)
    return (*out, c, t)


def compare(got, want, y, K, what):
    _, logp, lse, H, classes, tops, _, _ = want
    if y is not None:
        check(got[0], logp, lp_tol(logp, K), (what, "logp"))
    check(got[1], lse, lp_tol(lse, K), (what, "lse"))
    check(got[2], H, entropy_tol(H, K), (what, "entropy"))
    assert np.array_equal(got[3].cpu().numpy(), classes), (what, "classes")
    check(got[4], tops, lp_tol(tops, K), (what, "alternatives"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K", SHAPES)
def test_scores(B, K, dtype):
    rng = np.random.default_rng(B + 17 * K)
    for n, (plain, with_y, ld, base) in enumerate([(True, True, K, 0), (False, True, K + 3, 1), (False, False, K + 8, 0)]):
        z, y = logits(B, K, rng, dtype, plain)
        Z, flat = matrix(z, dtype, ld, base)
        top = TOPS[(B + K + n) % 6] if K > 300 else TOPS[(n + B) % 6]
        yy = y if with_y else None
        got = run(Z, vec(y, torch.int32) if with_y else None, top)
        compare(got, ref.scores_ref(z, yy, top), yy, K, (plain, with_y, top))


@pytest.mark.parametrize("top", TOPS)
@pytest.mark.parametrize("dtype,B,K", [("f32", 30, 7), ("bf16", 30, 500), ("f32", 30, 260), ("bf16", 30, 3000), ("f32", 14, 10007), ("f32", 13, 40000),
                                       ("bf16", 2, 100003)])
def test_alternatives_of_every_kind_of_row(dtype, B, K, top):
    rng = np.random.default_rng(top + K)
    z, y = logits(B, K, rng, dtype)
    Z, _ = matrix(z, dtype)
    compare(run(Z, vec(y, torch.int32), top), ref.scores_ref(z, y, top), y, K, top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [7, 300, 5000, 70000])
def test_nan_and_infinity_stay_in_their_row(K, dtype):
    rng = np.random.default_rng(K)
    z, y = logits(6, K, rng, dtype, plain=True)
    z[1, K - 1], z[2, 0], z[4, K // 2] = np.nan, np.inf, np.nan
    z[3, :] = np.nan
    y[0], y[2] = K - 1, 0
    Z, _ = matrix(z, dtype)
    got = run(Z, vec(y, torch.int32), 3)
    want = ref.scores_ref(z, y, 3)
    compare(got, want, y, K, K)
    dZ = torch.full_like(Z, 7.0)
    g = rng.standard_normal(6).astype(np.float32)
    hb.scores_grad(Z, dZ, vec(y, torch.int32), vec(g), vec(g), ws=work(6, K))
    d = host(dZ)
    assert np.isfinite(d[[0, 5]]).all() and np.isnan(d[[1, 2, 3, 4]]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [0.0, 1e4, -3e7, 1e30])
def test_logits_far_from_zero(offset, dtype):
    """Only differences count: rows whose logits are large steps of their type apart."""
    rng = np.random.default_rng(5)
    step = max(1.0, abs(offset) * 2.0 ** (-7 if dtype == "bf16" else -23))
    z, y = offset + step * rng.integers(-4, 1, (40, 50)), rng.integers(0, 50, 40).astype(np.int32)
    z = torch.as_tensor(z).to(TYPES[dtype]).double().numpy()
    Z, _ = matrix(z, dtype)
    compare(run(Z, vec(y, torch.int32), 5), ref.scores_ref(z, y, 5), y, 50, offset)


def grad_tol(want, r, z, y, gl, gh, K, dtype):
    part, _, _, H, _, _, p, lp = r
    far = np.where(p > 0, z.max(1, keepdims=True) - np.where(np.isfinite(z), z, 0.0), 0.0)
    rel = eps_s(K) + (far + 8) * U
    gl, gh = np.abs(gl)[:, None], np.abs(gh)[:, None]
    inner = gl + gh * np.abs(np.where(p > 0, lp, 0.0) + H[:, None])
    tol = p * (rel * inner + gh * (far + H[:, None] + 1) * 3 * eps_s(K) + 4 * U * gl)
    if y is not None:
        for i in np.nonzero(part)[0]:
            q = p[i].copy()
            q[y[i]] = 0
            tol[i, y[i]] += gl[i, 0] * (eps_s(K) * q.sum() + (8 * U if p[i, y[i]] < p[i].max() else 0.0))
    tol = tol * 2 + 4 * U * np.abs(want) + 1e-30
    return tol + (2.0 ** -8 * np.abs(want) + 2.0 ** -133 if dtype == "bf16" else 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K", SHAPES)
def test_gradient(B, K, dtype):
    rng = np.random.default_rng(B + 19 * K)
    for use_l, use_h, ld, ldd, base in [(True, True, K, K, 0), (True, False, K + 3, K + 1, 1), (False, True, K + 8, K + 8, 0)]:
        z, y = logits(B, K, rng, dtype)
        gl, gh = rng.standard_normal(B).astype(np.float32), rng.standard_normal(B).astype(np.float32)
        gl[::5] = 0
        gh[::3] = 0
        idle = (gl * use_l == 0) & (gh * use_h == 0)
        z[idle, 0] = np.nan  # not looked at
        Z, _ = matrix(z, dtype, ld, base)
        dZ, flat = matrix(np.zeros((B, K)), dtype, ldd, base)
        a, b = (gl if use_l else None), (gh if use_h else None)
        yy = y if use_l else None
        hb.scores_grad(Z, dZ, None if yy is None else vec(y, torch.int32), None if a is None else vec(a), None if b is None else vec(b), ws=work(B, K))
        z[idle] = 0.0  # for the reference, whose gradient there is zeros
        r = ref.scores_ref(z, yy, 0)
        want = ref.scores_grad_ref(r, y, a, b)
        check(dZ, want, grad_tol(want, r, z, yy, gl * use_l, gh * use_h, K, dtype), (use_l, use_h))
        assert outside_is_nan(flat, dZ)
        if ldd == ld and not np.isnan(want).any():  # in place
            hb.scores_grad(Z, Z, None if yy is None else vec(y, torch.int32), None if a is None else vec(a), None if b is None else vec(b), ws=work(B, K))
            assert torch.equal(Z, dZ)


@pytest.mark.parametrize("dtype,B,K", [("f32", 1030, 5001), ("f32", 1024, 8000), ("bf16", 1025, 9001), ("f32", 257, 30001), ("bf16", 256, 50257), ("bf16", 300, 50257),
                                       ("bf16", 259, 65536), ("f32", 64, 32771), ("bf16", 64, 40001), ("bf16", 64, 65543)])
def test_both_sides_of_what_rows_decide(dtype, B, K):
    rng = np.random.default_rng(B + K)
    z, y = logits(B, K, rng, dtype)
    gl, gh = rng.standard_normal(B).astype(np.float32), rng.standard_normal(B).astype(np.float32)
    Z, _ = matrix(z, dtype, K + 1, 1)
    Y = vec(y, torch.int32)
    want = ref.scores_ref(z, y, 5)
    compare(run(Z, Y, 5), want, y, K, (dtype, B, K))
    dZ, flat = matrix(np.zeros((B, K)), dtype, K + 1, 1)
    hb.scores_grad(Z, dZ, Y, vec(gl), vec(gh), ws=work(B, K))
    g = ref.scores_grad_ref(want, y, gl, gh)
    check(dZ, g, grad_tol(g, want, z, y, gl, gh, K, dtype), (dtype, B, K))
    assert outside_is_nan(flat, dZ)


def test_gradient_against_differences():
    rng = np.random.default_rng(2)
    B, K = 4, 9
    z, y = rng.standard_normal((B, K)), rng.integers(0, K, B)
    gl, gh = rng.standard_normal(B), rng.standard_normal(B)
    value = lambda v: (lambda r: (gl * r[1] + gh * r[3]).sum())(ref.scores_ref(v, y, 0))  # noqa: E731
    want = np.zeros((B, K))
    for i in range(B):
        for k in range(K):
            h = np.zeros((B, K))
            h[i, k] = 1e-5
            want[i, k] = (value(z + h) - value(z - h)) / 2e-5
    dZ = torch.empty(B, K, device="cuda")
    hb.scores_grad(torch.as_tensor(z).float().cuda(), dZ, vec(y, torch.int32), vec(gl), vec(gh), ws=work(B, K))
    assert np.abs(host(dZ) - want).max() < 1e-5
    assert np.abs(ref.scores_grad_ref(ref.scores_ref(z, y, 0), y, gl, gh) - want).max() < 1e-8


def test_many_rows_and_the_same_bits():
    g = torch.Generator(device="cuda").manual_seed(1)
    Z = torch.randn(100001, 7, device="cuda", generator=g).bfloat16()
    y = torch.randint(-1, 7, (100001,), device="cuda", generator=g, dtype=torch.int32)
    a, b = run(Z, y, 3), run(Z, y, 3)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    part = y >= 0
    lp = torch.log_softmax(Z.double(), 1)
    H = -(lp.exp() * lp).sum(1)
    assert float((a[2].double() - torch.where(part, H, 0.0)).abs().max()) < 1e-6
    c = Z.float().sort(dim=1, descending=True, stable=True).indices
    assert torch.equal(a[3], torch.where(part[:, None], c[:, :3], -1).int())


def test_more_chunks_than_the_workspace_holds_at_a_time():
    """Rows too long for a block, several launches of them one after the other."""
    B, K = 700, 400000
    g = torch.Generator(device="cuda").manual_seed(4)
    Z = torch.randn(B, K, device="cuda", generator=g).bfloat16()
    y = torch.randint(0, K, (B,), device="cuda", generator=g, dtype=torch.int32)
    got = run(Z, y, 2)
    dZ = torch.empty_like(Z)
    one = torch.ones(B, device="cuda")
    hb.scores_grad(Z, dZ, y, one, one, ws=work(B, K))
    for i in list(range(0, B, 53)) + [B - 1]:
        lp = torch.log_softmax(Z[i].double(), 0)
        H = -(lp.exp() * lp).sum()
        assert abs(float(got[0][i]) - float(lp[y[i]])) < eps_s(K) + U * 40 and abs(float(got[2][i]) - float(H)) < 3 * eps_s(K) * float(H)
        top = Z[i].float().topk(2).values
        assert torch.equal(Z[i].float()[got[3][i].long()], top)
        want = -lp.exp() * (1 + lp + H)
        want[y[i]] += 1
        assert float((dZ[i].double() - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max())


def test_two_calls_at_once_and_captured():
    torch.manual_seed(3)
    for B, K in [(40, 300), (3, 70001)]:
        Z, other = torch.randn(B, K, device="cuda"), torch.randn(B, K, device="cuda")
        y = torch.randint(0, K, (B,), device="cuda", dtype=torch.int32)
        one = torch.ones(B, device="cuda")
        ws, ws2, ws3 = work(B, K, 5), work(B, K, 5), work(B, K)
        out = [torch.zeros(B, device="cuda") for _ in range(3)] + [torch.zeros(B, 5, dtype=torch.int32, device="cuda"), torch.zeros(B, 5, device="cuda")]
        dZ = torch.zeros(B, K, device="cuda")

        def call():
            hb.scores(Z, y, logp=out[0], lse=out[1], entropy=out[2], top_class=out[3], top_logp=out[4], ws=ws)
            hb.scores_grad(Z, dZ, y, out[0], one, ws=ws3)

        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        side = torch.cuda.Stream()
        for k in range(4):
            Z.normal_()
            other.normal_()
            side.wait_stream(torch.cuda.current_stream())
            graph.replay()
            with torch.cuda.stream(side):
                b = run(other, y, 5, ws2)
            torch.cuda.synchronize()
            a = run(Z, y, 5)
            d = torch.zeros(B, K, device="cuda")
            hb.scores_grad(Z, d, y, a[0], one, ws=work(B, K))
            c = run(other, y, 5)
            torch.cuda.synchronize()
            assert all(torch.equal(s, t) for s, t in zip(a, out)) and torch.equal(d, dZ) and all(torch.equal(s, t) for s, t in zip(b, c)), k


def test_scores_agree_with_log_probabilities():
    """The calls that give the same numbers."""
    torch.manual_seed(1)
    for B, K in [(300, 983), (20, 40000)]:
        Z, y = torch.randn(B, K, device="cuda"), torch.randint(-1, K, (B,), device="cuda", dtype=torch.int32)
        logp, lse, g = torch.empty(B, device="cuda"), torch.empty(B, device="cuda"), torch.randn(B, device="cuda")
        hb.logprob(Z, y, logp, lse, ws=torch.empty(hb.choice_workspace_bytes(B), dtype=torch.uint8, device="cuda"))
        got = run(Z, y, 1)
        assert float((got[0] - logp).abs().max()) <= 2 * eps_s(K) + 40 * U and float((got[1] - lse).abs().max()) <= 2 * eps_s(K) + 40 * U
        d, e = torch.empty_like(Z), torch.empty_like(Z)
        hb.logprob_grad(Z, y, logp, lse, g, d)
        hb.scores_grad(Z, e, y, g_logp=g, ws=work(B, K))
        assert float((d - e).abs().max()) <= 4 * (eps_s(K) + 60 * U) * float(g.abs().max())
