"""Orthogonalised updates of matrices that begin at a boundary of their vector loads while their rows do not (pitches that are no multiple of four), in
several blocks of columns and in tiles.  Tolerances are those of test_ortho_gpu."""
import numpy as np
import pytest
import torch

import more_operators_ref as ref
import paper_2004_08771_amd as hb
from test_operators_gpu import U, host, matrix, outside_is_nan
from test_ortho_gpu import KINDS, TYPES, gradient, norm, tolerance, work

pytestmark = pytest.mark.gpu

SHAPES = [(100, 1000), (9000, 20), (16, 1025), (61, 1001), (1, 2049), (200, 301)]


@pytest.mark.parametrize("g_type", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalize(shape, g_type):
    rows, cols = shape
    rng = np.random.default_rng(rows + cols)
    G = torch.as_tensor(gradient(rows, cols, rng)).to(TYPES[g_type]).double().numpy()
    want, tol = tolerance(G, "f32")
    first = None
    for ldg, ldo in [(cols, cols), (cols + 1, cols), (cols + 2, cols + 3), (cols + 3, cols + 4)]:
        dG, flat_g = matrix(G, g_type, ldg)
        out, flat_o = matrix(np.zeros(shape), "f32", ldo)
        hb.orthogonalize(dG, out, products=KINDS["f32"], ws=work([shape], "f32"))
        assert norm(host(out) - want) <= tol, (shape, ldg)
        assert outside_is_nan(flat_g, dG) and outside_is_nan(flat_o, out)
        # G is divided by the same number but for the order of a sum in 64 bits
        first = host(out) if first is None else first
        assert norm(host(out) - first) <= tol, (shape, ldg)


@pytest.mark.parametrize("g_type", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_update(shape, g_type):
    """Gaps in the gradient, in the momenta, and in one of them beside the other without."""
    rows, cols = shape
    rng = np.random.default_rng(rows * 3 + cols)
    lr, momentum, decay, s = 0.02, 0.9, 0.1, 0.5
    G = torch.as_tensor(gradient(rows, cols, rng)).to(TYPES[g_type]).double().numpy()
    W = (rng.standard_normal(shape) * 0.1).astype(np.float32).astype(np.float64)
    M = gradient(rows, cols, rng).astype(np.float32).astype(np.float64)
    want_w, want_m, O = ref.muon_ref(W, G, M, lr, momentum, True, decay, s)
    u = G + float(np.float32(momentum)) * want_m
    _, tol = tolerance(u, "f32")
    tol += 485 * 3 * U  # U from an M that has been rounded
    for ldg, ldm, ldw in [(cols + 1, cols, cols), (cols, cols + 1, cols), (cols, cols + 2, cols + 1), (cols + 3, cols + 3, cols + 3), (cols + 4, cols + 1, cols)]:
        dG, flat_g = matrix(G, g_type, ldg)
        dM, flat_m = matrix(M, "f32", ldm)
        dW, flat_w = matrix(W, "f32", ldw)
        hb.muon_update(dW, dG, dM, lr, momentum, True, decay, s, ws=work([shape], "f32"))
        assert (np.abs(host(dM) - want_m) <= 2 * U * (np.abs(momentum * M) + np.abs(G)) + 1e-30).all(), (shape, ldg, ldm)
        assert norm(host(dW) - want_w) <= lr * s * tol + 3 * U * (norm(W) + lr * s * norm(O)), (shape, ldg, ldm)
        assert outside_is_nan(flat_m, dM) and outside_is_nan(flat_w, dW) and outside_is_nan(flat_g, dG)
