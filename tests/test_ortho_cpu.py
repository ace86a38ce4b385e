"""What the orthogonalised updates refuse, before any device call."""
import ctypes

import numpy as np
import pytest
import torch

import more_operators_ref as ref
import paper_2004_08771_amd as hb
from test_operators_cpu import refused

G, OUT = torch.zeros(6, 10), torch.zeros(6, 10)
WS = torch.zeros(1 << 20, dtype=torch.uint8)


def test_workspace_sizes():
    need = hb.ortho_workspace_bytes
    assert 0 < need([]) <= need([(1, 1)]) <= need([(512, 512)]) < need([(4096, 512)])
    assert need([(512, 512)], hb.HB_TENSOR_BF16) < need([(512, 512)])
    assert need([(64, 64)] * 16) > need([(64, 64)]) and need([(64, 64)] * 32) == need([(64, 64)] * 16)
    assert need([(-1, 5)]) == 0 and need([(32769, 1)]) == 0 and need([(32768, 32769)]) == 0 and need([(0, 0)]) > 0
    assert need([(5, 5)], 7) == 0
    small = WS[:need([(6, 10)]) - 1]
    refused(lambda: hb.orthogonalize(G, OUT, ws=small), text="workspace")
    refused(lambda: hb.orthogonalize(G, OUT, ws=None))
    refused(lambda: hb.orthogonalize(G, OUT, ws=WS[4:]), text="aligned")
    refused(lambda: hb.muon_update(G, G.clone(), OUT, 0.1, ws=small), text="workspace")


@pytest.mark.parametrize("how", [{"steps": 0}, {"steps": 33}, {"steps": -1}, {"coef": (1, 2)}, {"coef": ((1, 2, 3),) * 4}, {"coef": (33, 0, 0)},
                                 {"coef": (float("nan"), 0, 0)}, {"coef": (1, float("inf"), 0)}, {"eps": -1e-9}, {"eps": float("nan")},
                                 {"eps": float("inf")}, {"products": 2}])
def test_steps_are_refused(how):
    refused(lambda: hb.orthogonalize(G, OUT, ws=WS, **how))
    refused(lambda: hb.muon_update(G, G.clone(), OUT, 0.1, ws=WS, **how))


@pytest.mark.parametrize("how", [{"lr": -0.1}, {"lr": float("nan")}, {"lr": float("inf")}, {"momentum": -0.1}, {"momentum": 1.0},
                                 {"momentum": float("nan")}, {"weight_decay": -1.0}, {"weight_decay": float("inf")}, {"scale": float("nan")},
                                 {"scale": [1.0, 2.0]}, {"lr": 1e30, "weight_decay": 1e30}, {"lr": 1e30, "scale": 1e30}])
def test_updates_are_refused(how):
    refused(lambda: hb.muon_update(G, G.clone(), OUT, **{"lr": 0.1, "ws": WS, **how}))


def test_operands_are_refused():
    for g, o in [(G.double(), OUT), (G, OUT.half()), (G[0], OUT[0]), (G, torch.zeros(10, 6)), (G.t(), torch.zeros(10, 6)), ([G, G], [OUT]),
                 ([G, G.bfloat16()], [OUT, torch.zeros(6, 10)]), (G, torch.zeros(6, 1).expand(6, 10))]:
        refused(lambda: hb.orthogonalize(g, o, ws=WS))
    big = torch.zeros(14, 20)
    for g, o in [(big[:6], big[1:7]), ([big[:6], big[6:12]], [torch.zeros(6, 20), big[5:11]]), ([G, G], [OUT, OUT]),
                 (big[:7], big.view(-1)[:140].view(14, 10)[:7, :5].expand(7, 5))]:
        if (o[0] if isinstance(o, list) else o).shape == (g[0] if isinstance(g, list) else g).shape:
            refused(lambda: hb.orthogonalize(g, o, ws=WS), text="overlaps")
    # the result over its own G as another type, and over another's G
    raw = torch.zeros(6 * 10, dtype=torch.float32)
    refused(lambda: hb.orthogonalize(raw.view(6, 10), raw.view(torch.bfloat16)[:60].view(6, 10), ws=WS), text="overlaps")
    refused(lambda: hb.orthogonalize([big[:6], big[6:12]], [big[6:12], torch.zeros(6, 20)], ws=WS), text="overlaps")
    refused(lambda: hb.orthogonalize(G, WS.view(torch.float32)[:60].view(6, 10), ws=WS), text="overlaps")
    for w, g, m in [(G, G, OUT), (G, OUT, G), (G, OUT, OUT), ([G, G], [OUT, OUT], [torch.zeros(6, 10), torch.zeros(6, 10)])]:
        refused(lambda: hb.muon_update(w, g, m, 0.1, ws=WS), text="overlaps")
    for w, g, m in [(G.bfloat16(), OUT, torch.zeros(6, 10)), (G, OUT, torch.zeros(6, 10).bfloat16()), (G, OUT, torch.zeros(6, 11))]:
        refused(lambda: hb.muon_update(w, g, m, 0.1, ws=WS))
    # halves of the columns of one buffer are apart: refused only for where they are
    with pytest.raises(hb.HbError) as e:
        hb.orthogonalize(big[:, :10], big[:, 10:], ws=WS)
    assert "overlaps" not in str(e.value)


def test_the_library_refuses_what_the_binding_cannot_say():
    call = hb.lib().hb_orthogonalize_async
    how = hb.ortho_args()
    one = lambda **k: ctypes.byref(hb.binding.OrthoMatrix(**{"rows": 6, "cols": 10, "d_g": G.data_ptr(), "ldg": 10,  # noqa: E731
                                                             "d_out": OUT.data_ptr(), "ldo": 10, **k}))
    tail = (ctypes.byref(how), WS.data_ptr(), WS.nbytes, None)
    for k in [{"rows": -1}, {"cols": -1}, {"rows": 1 << 40}, {"d_g": None}, {"d_out": None}, {"ldg": 9}, {"ldo": 9}, {"ldg": 1 << 31},
              {"d_g": G.data_ptr() + 2}]:
        assert call(one(**k), 1, 0, 0, *tail) == hb.HB_ERR_INVALID, k
    assert call(one(), 1, 3, 0, *tail) == hb.HB_ERR_INVALID and call(one(), 1, 0, -1, *tail) == hb.HB_ERR_INVALID
    assert call(one(), -1, 0, 0, *tail) == hb.HB_ERR_INVALID and call(one(), 4097, 0, 0, *tail) == hb.HB_ERR_INVALID
    assert call(None, 1, 0, 0, *tail) == hb.HB_ERR_INVALID and call(one(), 1, 0, 0, None, *tail[1:]) == hb.HB_ERR_INVALID
    for k in [{"rows": 0}, {"cols": 0, "d_g": None, "d_out": None}]:
        assert call(one(**k), 1, 0, 0, *tail) == hb.HB_OK, k  # nothing to do
    assert call(None, 0, 0, 0, *tail) == hb.HB_OK
    bad = hb.ortho_args()
    bad.n_coef = 0
    assert call(one(), 1, 0, 0, ctypes.byref(bad), *tail[1:]) == hb.HB_ERR_INVALID


def test_the_definition():
    """The polynomial of the singular values, on a matrix whose singular vectors are known."""
    rng = np.random.default_rng(0)
    q, _ = np.linalg.qr(rng.standard_normal((8, 8)))
    p, _ = np.linalg.qr(rng.standard_normal((12, 8)))
    s = np.linspace(0.2, 3, 8)
    for flip in (False, True):
        G = q @ np.diag(s) @ p.T
        t = s / (np.sqrt((s * s).sum()) + float(np.float32(1e-7)))
        a, b, c = (float(np.float32(v)) for v in ref.COEF)
        for _ in range(5):
            t = a * t + b * t ** 3 + c * t ** 5
        want = q @ np.diag(t) @ p.T
        got = ref.ortho_ref(G.T).T if flip else ref.ortho_ref(G)
        assert np.abs(got - want).max() < 1e-12
        assert np.abs(ref.ortho_rounded(G, planes=2) - want).max() < 1e-4


def test_a_model_that_is_not_configured():
    m = hb.Model((8, 4, 2))
    buf = np.zeros(m.num_params, np.float32)
    for call in (lambda: m.set_muon(hb.muon_args()), lambda: m.set_muon(None), lambda: m.get_momenta(buf), lambda: m.set_momenta(buf),
                 lambda: m.batch_scores_async(1, 1, 4)):
        refused(call, hb.HB_ERR_STATE)
