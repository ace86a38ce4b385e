"""Which mistakes the precision tests of the orthogonalised updates would see: the host's forms of the kernels' roundings, with the mistake and without.

The tests on the device allow three times what the host's form of fp32-like products is off by, and twice where a list of 64 small matrices is taken together (root
mean square) or operands have 11 bits.  Both are sums of many independent roundings, so another order of the sums moves them by a tenth or so."""
import numpy as np
import pytest

import ortho_roundings as r


@pytest.mark.parametrize("G", r.few_rows(), ids=lambda G: "x".join(map(str, G[0].shape)))
def test_runs_of_two_steps_with_few_rows_are_seen(G):
    single, double = (r.rms([r.off(r.small(g, limit=limit), g) for g in G]) for limit in (1.0, 12.0))
    assert single < 1.5e-6 and double > 2.5 * single


@pytest.mark.parametrize("shape", r.LARGER)
def test_lost_low_parts_are_seen(shape):
    G = r.two_decades(*shape)
    right = r.off(r.tiled(G), G)
    assert right < 3e-6
    assert r.off(r.tiled(G, without=("low",)), G) > 100 * right and r.off(r.tiled(G, without=("linear",)), G) > 100 * right
    right = r.off(r.tiled(G, planes=1), G)
    assert right < 1e-3 and r.off(r.tiled(G, planes=1, without=("linear",)), G) > 2.5 * right


@pytest.mark.parametrize("shape", r.SMALLER)
def test_runs_of_five_steps_are_seen(shape):
    G = r.two_decades(*shape)
    right = r.off(r.small(G, limit=12.0), G)
    assert right < 6e-6 and r.off(r.small(G, limit=500.0), G) > 8 * right


@pytest.mark.parametrize("shape", r.SMALLER + [(64, 512), (100, 1000)])
def test_what_singular_values_near_zero_cost(shape):
    """The figures that the documentation has for operands of 11 bits: small matrices by themselves, and as they go beside larger ones."""
    for low, alone, beside in [(1e-2, 1e-4, 6e-4), (3e-3, 2e-3, 2e-3), (1e-4, 1e-3, 1.5e-2)]:
        G = r.with_values(*shape, np.r_[1.0, np.full(min(shape) - 1, low)], np.random.default_rng(1))
        assert r.off(r.small(G, limit=500.0), G) < alone and r.off(r.tiled(G, planes=1), G) < beside, low
        assert r.off(r.small(G, limit=12.0), G) < 1e-4 and r.off(r.tiled(G), G) < 1e-4
