"""Orthogonalised updates against their definition in 64 bits.

Tolerances, in Frobenius norm: what the roundings of stored operands do is found by making the same roundings in the 64-bit computation
(ortho_rounded, for small matrices ortho_runs); others may fall elsewhere by the order of fp32 sums, so twice its distance from the definition is allowed, and on top what fp32 sums
may add (fp32_sums).  A bf16 result adds its rounding, 2^-8 relative to each entry.  Weights: the update's tolerance times lr scale, and three
roundings of 2^-24 of |w| and of the update; momenta: one rounding of each term.
"""
import numpy as np
import pytest
import torch

import more_operators_ref as ref
import paper_2004_08771_amd as hb
from test_operators_gpu import U, host, matrix, outside_is_nan

pytestmark = pytest.mark.gpu

KINDS = {"f32": hb.HB_TENSOR_F32, "bf16": hb.HB_TENSOR_BF16}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def work(shapes, products):
    """A workspace that holds NaN."""
    return torch.full((hb.ortho_workspace_bytes(shapes, KINDS[products]),), 0xFF, dtype=torch.uint8, device="cuda")


def gradient(rows, cols, rng, kind="spread"):
    g = rng.standard_normal((rows, cols))
    if kind == "spread":
        g *= np.exp(rng.standard_normal((rows, 1))) * np.exp(rng.standard_normal((1, cols)))
        g += 3 * rng.standard_normal((rows, 1)) * rng.standard_normal((1, cols))
    elif kind == "low":  # few directions
        k = max(1, min(rows, cols) // 8)
        g = rng.standard_normal((rows, k)) @ rng.standard_normal((k, cols))
    elif kind == "holes":  # units without a gradient
        g[rng.random(rows) < 0.3] = 0.0
        g[:, rng.random(cols) < 0.3] = 0.0
    return g


def norm(x):
    return float(np.sqrt((x * x).sum()))


def tolerance(G, products, out="f32", tiles=False, **how):
    """(result, how far one may be from it in norm); tiles: beside larger matrices in a list"""
    want = ref.ortho_ref(G, **how)
    limit = 0.0
    if min(G.shape) <= 128 and not tiles:  # small matrices, by themselves: runs of steps
        limit = 12.0 if products == "f32" else 500.0
        rounded = ref.ortho_runs(G, limit=limit, **how)
    else:
        rounded = ref.ortho_rounded(G, planes=2 if products == "f32" else 1, **how)
    tol = 2 * norm(rounded - want) + ref.fp32_sums(G, limit=limit, **how)
    return want, tol + (2.0 ** -8 * norm(want) if out == "bf16" else 2.0 ** -24 * norm(want)) + 2.0 ** -36 * np.sqrt(want.size)


def check(got, want, tol, what):
    got = host(got) if torch.is_tensor(got) else got
    assert got.shape == want.shape and np.isfinite(got).all(), what
    off = norm(got - want)
    assert off <= tol, f"{what}: off by {off:.3g}, {tol:.3g} is allowed (norm {norm(want):.3g})"


SHAPES = [(1, 1), (1, 7), (7, 1), (2, 2), (3, 64), (64, 3), (17, 33), (54, 32), (63, 65), (64, 64), (65, 64), (127, 200), (200, 129),
          (512, 54), (7, 512), (300, 257), (512, 512)]


@pytest.mark.parametrize("products", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_orthogonalize(rows, cols, products):
    rng = np.random.default_rng(rows * 1000 + cols)
    for kind, g_type, o_type, ldg, ldo, base in [("spread", "f32", "f32", cols, cols, 0), ("low", "bf16", "bf16", cols + 3, cols + 1, 1),
                                                 ("holes", "f32", "bf16", cols + 5, cols, 3)]:
        G = torch.as_tensor(gradient(rows, cols, rng, kind)).to(TYPES[g_type]).double().numpy()
        dG, flat_g = matrix(G, g_type, ldg, base)
        out, flat_o = matrix(np.zeros((rows, cols)), o_type, ldo, base)
        hb.orthogonalize(dG, out, products=KINDS[products], ws=work([(rows, cols)], products))
        want, tol = tolerance(G, products, o_type)
        check(out, want, tol, (kind, rows, cols))
        assert outside_is_nan(flat_o, out) and outside_is_nan(flat_g, dG) and np.array_equal(host(dG), G)


@pytest.mark.parametrize("products", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1100, 1000), (700, 2100), (2049, 1025)])
def test_orthogonalize_larger(rows, cols, products):
    rng = np.random.default_rng(rows)
    G = gradient(rows, cols, rng).astype(np.float32).astype(np.float64)
    dG, _ = matrix(G, "f32")
    out = torch.empty(rows, cols, device="cuda")
    hb.orthogonalize(dG, out, products=KINDS[products], ws=work([(rows, cols)], products))
    check(out, *tolerance(G, products), (rows, cols))


@pytest.mark.parametrize("products", ["f32", "bf16"])
@pytest.mark.parametrize("shapes", [[(140, 9000)], [(5000, 200), (130, 131)], [(190, 3001), (150, 8192), (1, 1)], [(100, 20000)], [(12, 30000), (16, 5)],
                                    [(64, 32768)], [(16384, 128)]])
def test_few_rows_and_many_columns(shapes, products):
    """A long axis is split: what is joined again gives the definition, the same every time."""
    rng = np.random.default_rng(shapes[0][1])
    tiles = max(min(s) for s in shapes) > 128
    G = [gradient(*s, rng).astype(np.float32).astype(np.float64) for s in shapes]
    dG = [torch.as_tensor(g).float().cuda() for g in G]
    out, again = [torch.empty_like(g) for g in dG], [torch.empty_like(g) for g in dG]
    for o in (out, again):
        hb.orthogonalize(dG, o, products=KINDS[products], ws=work(shapes, products))
    for g, o, p in zip(G, out, again):
        check(o, *tolerance(g, products, tiles=tiles), g.shape)
        assert torch.equal(o, p)


@pytest.mark.parametrize("n", [1, 2, 5, 6, 31, 82])
def test_one_row_keeps_its_digits(n):
    """One singular value of 1 with exact arithmetic: f(s) = s p(s) five times.  Errors of a step relative to X: its planes 2^-22; products 2^-24 each of the
    scale and the result; p by what A is off (2^-22 of dropped terms, (n + 2) 2^-24 of sums) and three roundings of up to |p's terms|; each times what later steps make of it."""
    rng = np.random.default_rng(n)
    G = rng.standard_normal((1, n)).astype(np.float32).astype(np.float64)
    out = torch.empty(1, n, device="cuda")
    hb.orthogonalize(torch.as_tensor(G).float().cuda(), out, products=KINDS["f32"], ws=work([(1, n)], "f32"))
    a, b, c = 3.4445, -4.7750, 2.0315
    s, tol = 1.0, 2.0 ** -22
    for _ in range(5):
        p = a + b * s ** 2 + c * s ** 4
        slope = abs(a + 3 * b * s ** 2 + 5 * c * s ** 4) / abs(p)
        terms = (a + abs(b) * s ** 2 + c * s ** 4) / abs(p)
        off_a = 2.0 ** -22 + (n + 2) * 2.0 ** -24
        tol = tol * max(1.0, slope) + 2.0 ** -22 + 2 * 2.0 ** -24 + abs(b * s ** 2 + 2 * c * s ** 4) / abs(p) * off_a + 3 * 2.0 ** -24 * terms
        s *= p
    want = s * G / np.linalg.norm(G)
    assert np.abs(out.cpu().double().numpy() - want).max() <= tol * np.abs(want).max()


def test_large_matrix_against_products_on_the_device():
    """Sizes of the largest tiles: the definition in 64-bit products on the device."""
    g = torch.Generator(device="cuda").manual_seed(1)
    for rows, cols in [(4096, 4000), (2300, 6000), (8192, 2048)]:
        G = torch.randn(rows, cols, device="cuda", generator=g) * torch.exp(torch.randn(1, cols, device="cuda", generator=g))
        X = G.double().T.contiguous() if rows > cols else G.double()
        X = X / X.norm()
        for _ in range(5):
            A = X @ X.T.contiguous()
            a, b, c = (float(np.float32(v)) for v in ref.COEF)
            X = a * X + (b * A + c * (A @ A)) @ X
        want = X.T if rows > cols else X
        for products, tol in (("f32", 2e-5), ("bf16", 5e-3)):
            # of the norm: 485 roundings of 2^-22 and fp32 sums of depth 8192 / 32; roundings of 2^-11 in each of three products of the last steps
            out = torch.empty_like(G)
            hb.orthogonalize(G, out, products=KINDS[products], ws=work([(rows, cols)], products))
            assert float((out.double() - want).norm() / want.norm()) <= tol, (rows, cols, products)


SMALL = [(1, 1), (3, 40), (16, 16), (16, 1025), (17, 100), (32, 1024), (33, 5), (64, 512), (64, 513), (65, 65), (128, 128), (128, 129), (100, 1000), (5, 8192),
         (9000, 20), (700, 128), (60, 3000), (127, 2000), (31, 33)]


@pytest.mark.parametrize("products", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SMALL)
def test_small_matrices(shape, products):
    """One block of columns, several, and several matrices of which the largest decides."""
    rng = np.random.default_rng(shape[0] + 7 * shape[1])
    for shapes, how in [([shape], {}), ([shape, (shape[0], 2), (1, 1)], {"steps": 7}), ([shape[::-1], shape], {"steps": 1}),
                        ([shape], {"steps": 9, "coef": (1.5, -0.5, 0.0)})]:
        G = [gradient(r, c, rng, ("spread", "low", "holes")[(r + i) % 3]).astype(np.float32).astype(np.float64) for i, (r, c) in enumerate(shapes)]
        out = [matrix(np.zeros(s), "f32", s[1] + 1, 1) for s in shapes]
        hb.orthogonalize([matrix(x, "f32", x.shape[1] + 2, 3)[0] for x in G], [o[0] for o in out], products=KINDS[products],
                         ws=work(shapes, products), **how)
        for x, (o, flat) in zip(G, out):
            check(o, *tolerance(x, products, **how), (shapes, how))
            assert outside_is_nan(flat, o)


def test_coefficients_that_grow_go_through_the_products():
    """Factors too large for the runs of small matrices."""
    rng = np.random.default_rng(8)
    G = gradient(20, 30, rng, "plain").astype(np.float32).astype(np.float64)
    how = {"steps": 2, "coef": ((30.0, 0.0, 0.0), (1.0, 0.0, 0.0))}
    out = torch.empty(20, 30, device="cuda")
    hb.orthogonalize(torch.as_tensor(G).float().cuda(), out, ws=work([(20, 30)], "f32"), **how)
    check(out, *tolerance(G, "f32", tiles=True, **how), "grown")


def test_lists_of_mixed_shapes():
    """More matrices than go through the same launches, tall and wide, some without rows."""
    rng = np.random.default_rng(5)
    shapes = [(int(rng.integers(1, 150)), int(rng.integers(1, 150))) for _ in range(37)] + [(0, 5), (5, 0), (300, 20)]
    G = [gradient(r, c, rng).astype(np.float32).astype(np.float64) for r, c in shapes]
    dG = [torch.as_tensor(x).float().cuda() for x in G]
    out = [torch.full((r, c), 7.0, device="cuda") for r, c in shapes]
    hb.orthogonalize(dG, out, ws=work(shapes, "f32"))
    for x, o, s in zip(G, out, shapes):
        if 0 not in s:
            check(o, *tolerance(x, "f32", tiles=True), s)


@pytest.mark.parametrize("how", [{"steps": 1}, {"steps": 2, "coef": (1.5, -0.5, 0.0)}, {"steps": 12, "coef": (1.5, -0.5, 0.0)},
                                 {"steps": 3, "coef": ((4.0, -8.0, 5.0), (3.4445, -4.775, 2.0315), (1.875, -1.25, 0.375))},
                                 {"steps": 5, "eps": 0.5}])
def test_steps_and_coefficients(how):
    rng = np.random.default_rng(3)
    for rows, cols in [(40, 70), (130, 90)]:
        G = gradient(rows, cols, rng, "plain").astype(np.float32).astype(np.float64)
        for products in ("f32", "bf16"):
            out = torch.empty(rows, cols, device="cuda")
            hb.orthogonalize(torch.as_tensor(G).float().cuda(), out, products=KINDS[products], ws=work([(rows, cols)], products), **how)
            check(out, *tolerance(G, products, **how), (how, rows, cols, products))


def test_singular_values_come_near_one():
    rng = np.random.default_rng(9)
    G = rng.standard_normal((120, 300))
    out = torch.empty(120, 300, device="cuda")
    hb.orthogonalize(torch.as_tensor(G).float().cuda(), out, steps=12, coef=(1.5, -0.5, 0.0), ws=work([(120, 300)], "f32"))
    s = np.linalg.svd(host(out), compute_uv=False)
    assert np.abs(s - 1).max() < 1e-4


def test_sizes_of_values():
    """Only the direction counts: G near the ends of fp32's range; zeros; inf and NaN."""
    rng = np.random.default_rng(4)
    G = gradient(50, 70, rng).astype(np.float32)
    want, tol = tolerance(G.astype(np.float64), "f32", eps=0.0)
    ws = work([(50, 70)], "f32")
    for scale in (2.0 ** 100, 2.0 ** -100, 1.0):
        out = torch.empty(50, 70, device="cuda")
        hb.orthogonalize(torch.as_tensor(G * np.float32(scale)).cuda(), out, eps=0.0, ws=ws)
        check(out, want, tol, scale)
    hb.orthogonalize(torch.zeros(50, 70, device="cuda"), out, ws=ws)
    assert bool((out == 0).all())
    for bad in (float("nan"), float("inf")):
        g = torch.as_tensor(G).cuda()
        g[3, 5] = bad
        hb.orthogonalize(g, out, ws=ws)
        assert bool(torch.isnan(out).all())
    hb.orthogonalize(torch.as_tensor(G).cuda(), out, eps=0.0, ws=ws)  # nothing of it stays in the workspace
    check(out, want, tol, "after")


def test_in_place_and_again():
    rng = np.random.default_rng(6)
    G = torch.as_tensor(gradient(190, 130, rng)).float().cuda()
    ws = work([(190, 130)], "f32")
    want = torch.empty_like(G)
    hb.orthogonalize(G, want, ws=ws)
    for _ in range(3):
        again = torch.empty_like(G)
        hb.orthogonalize(G, again, ws=ws)
        assert torch.equal(again, want)
    hb.orthogonalize(G, G, ws=ws)
    assert torch.equal(G, want)


@pytest.mark.parametrize("products", ["f32", "bf16"])
@pytest.mark.parametrize("g_type", ["f32", "bf16"])
@pytest.mark.parametrize("nesterov", [True, False])
def test_muon(nesterov, g_type, products):
    rng = np.random.default_rng(11)
    shapes = [(32, 54), (7, 32), (200, 100), (129, 300), (1, 5)]
    lr, momentum, decay = 0.02, 0.9, 0.1
    state = []
    for r, c in shapes:
        W, M = rng.standard_normal((r, c)).astype(np.float32) * 0.1, gradient(r, c, rng).astype(np.float32)
        state.append([W.astype(np.float64), M.astype(np.float64)])
    dW = [matrix(w, "f32", w.shape[1] + 3, 2) for w, _ in state]
    dM = [matrix(m, "f32", m.shape[1] + 1, 1) for _, m in state]
    scale = [0.5, 1.0, -1.0, 2.0, 0.25]
    ws = work(shapes, products)
    for _ in range(2):
        G = [torch.as_tensor(gradient(r, c, rng)).to(TYPES[g_type]) for r, c in shapes]
        dG = [matrix(g.double().numpy(), g_type, g.shape[1] + 2, 1)[0] for g in G]
        before = [(host(w[0]), host(m[0])) for w, m in zip(dW, dM)]
        hb.muon_update([w[0] for w in dW], dG, [m[0] for m in dM], lr, momentum, nesterov, decay, scale, products=KINDS[products], ws=ws)
        for (w, fw), (m, fm), g, (w0, m0), s in zip(dW, dM, G, before, scale):
            g = g.double().numpy()
            want_w, want_m, O = ref.muon_ref(w0, g, m0, lr, momentum, nesterov, decay, s)
            size = np.abs(momentum * m0) + np.abs(g)
            assert (np.abs(host(m) - want_m) <= 2 * U * size + 1e-30).all()
            u = g + float(np.float32(momentum)) * want_m if nesterov else want_m
            _, tol = tolerance(u, products, tiles=True)
            tol += 485 * 3 * U  # U from an M that has been rounded
            check(w, want_w, lr * abs(s) * tol + 3 * U * (norm(w0) + lr * abs(s) * norm(O)), w0.shape)
            assert outside_is_nan(fw, w) and outside_is_nan(fm, m)


def test_update_in_a_graph_and_on_a_stream():
    """Replays between eager updates of other weights, each compared with the eager result from the same state."""
    torch.manual_seed(2)
    shapes = [(64, 54), (64, 64), (10, 64)]
    make = lambda: [torch.randn(s, device="cuda") for s in shapes]  # noqa: E731
    W, G, M = make(), make(), make()
    V, H, N = make(), make(), make()
    ws, ws2 = work(shapes, "f32"), work(shapes, "f32")
    side = torch.cuda.Stream()
    call = lambda w, g, m, x: hb.muon_update(w, g, m, 0.01, weight_decay=0.1, ws=x)  # noqa: E731
    call(W, G, M, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(W, G, M, ws)
    for k in range(4):
        for t in G + H:
            t.normal_()
        w0, m0 = [w.clone() for w in W], [m.clone() for m in M]
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(V, H, N, ws2)
            call(w0, G, m0, ws2)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(W + M, w0 + m0)), k
