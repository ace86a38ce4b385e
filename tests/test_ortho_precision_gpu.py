"""How far the orthogonalised updates are from 64 bits, against the host's forms of the same roundings (ortho_roundings; test_ortho_precision_cpu has which mistakes
these tolerances show), and that a call repeats itself."""
import numpy as np
import pytest
import torch

import ortho_roundings as r
import paper_2004_08771_amd as hb
from test_ortho_gpu import KINDS, work
from test_operators_gpu import host

pytestmark = pytest.mark.gpu


def result(G, products, beside=()):
    """The results of the matrices G in one call, `beside` others of these shapes."""
    dG = [torch.as_tensor(np.ascontiguousarray(g)).float().cuda() for g in G] + [torch.ones(s, device="cuda") for s in beside]
    out = [torch.empty_like(g) for g in dG]
    hb.orthogonalize(dG, out, products=KINDS[products], ws=work([tuple(g.shape) for g in dG], products))
    return [host(o) for o in out[:len(G)]]


@pytest.mark.parametrize("G", r.few_rows(), ids=lambda G: "x".join(map(str, G[0].shape)))
def test_few_rows_go_step_by_step(G):
    allowed = 2 * r.rms([r.off(r.small(g, limit=1.0), g) for g in G])
    assert r.rms([r.off(o, g) for o, g in zip(result(G, "f32"), G)]) < allowed


@pytest.mark.parametrize("shape", r.LARGER)
def test_tiles(shape):
    G = r.two_decades(*shape)
    assert r.off(result([G], "f32")[0], G) < 3 * r.off(r.tiled(G), G)
    assert r.off(result([G], "bf16")[0], G) < 2 * r.off(r.tiled(G, planes=1), G)


@pytest.mark.parametrize("shape", r.SMALLER)
def test_small_matrices_by_themselves_and_beside_larger_ones(shape):
    G = r.two_decades(*shape)
    assert r.off(result([G], "f32")[0], G) < 3 * r.off(r.small(G, limit=12.0), G)
    assert r.off(result([G], "bf16")[0], G) < 2 * r.off(r.small(G, limit=500.0), G)
    assert r.off(result([G], "f32", beside=[(130, 129)])[0], G) < 3 * r.off(r.tiled(G), G)
    assert r.off(result([G], "bf16", beside=[(130, 129)])[0], G) < 2 * r.off(r.tiled(G, planes=1), G)


@pytest.mark.parametrize("products", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1000, 4096), (2048, 2000), (61, 1712), (134, 176)])
def test_a_call_repeats_itself(rows, cols, products):
    """The same bits, whatever the workspace holds and whatever went through it in between."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    G, other = (torch.randn(rows, cols, device="cuda", generator=g).bfloat16() for _ in range(2))
    ws = work([(rows, cols)], products)
    want, out = torch.empty_like(G), torch.empty_like(G)
    hb.orthogonalize(G, want, products=KINDS[products], ws=ws)
    for fill in (0, 255, None):
        hb.orthogonalize(other, out, products=KINDS[products], ws=ws)
        if fill is not None:
            ws.fill_(fill)
        hb.orthogonalize(G, out, products=KINDS[products], ws=ws)
        assert torch.equal(out, want)


@pytest.mark.parametrize("low", [1e-2, 3e-3, 1e-4])
@pytest.mark.parametrize("shape", r.SMALLER + [(64, 512), (100, 1000)])
def test_singular_values_near_zero(shape, low):
    """Three times the host's form: a step multiplies what a rounding leaves beside them, so a few roundings count more than the others."""
    G = r.with_values(*shape, np.r_[1.0, np.full(min(shape) - 1, low)], np.random.default_rng(1))
    for products, beside, form in [("f32", (), lambda: r.small(G, limit=12.0)), ("f32", [(130, 129)], lambda: r.tiled(G)),
                                   ("bf16", (), lambda: r.small(G, limit=500.0)), ("bf16", [(130, 129)], lambda: r.tiled(G, planes=1))]:
        assert r.off(result([G], products, beside)[0], G) < 3 * r.off(form(), G), (products, beside)
