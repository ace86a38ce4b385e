"""What the scores refuse, before any device call."""
import numpy as np
import torch

import more_operators_ref as ref
import paper_2004_08771_amd as hb
from test_operators_cpu import ROW, Y, Z, refused

WS = torch.zeros(1 << 16, dtype=torch.uint8)
TC, TL = torch.zeros(6, 3, dtype=torch.int32), torch.zeros(6, 3)


def test_workspace_sizes():
    need = hb.scores_workspace_bytes
    assert 0 < need(0, 1) <= need(1, 10) <= need(1, 1 << 20) < need(1, 1 << 20, 20) and need(1 << 22, 1 << 24, 64) < 1 << 24
    for args in [(-1, 5), ((1 << 22) + 1, 5), (5, 0), (5, (1 << 24) + 1), (5, 5, -1), (5, 5, 65)]:
        assert need(*args) == 0
    small = WS[:need(6, 10, 3) - 1]
    refused(lambda: hb.scores(Z, Y, ROW, top_class=TC, ws=small), text="workspace")
    refused(lambda: hb.scores(Z, Y, ROW, ws=None))
    refused(lambda: hb.scores(Z, Y, ROW, ws=WS[4:]), text="aligned")
    refused(lambda: hb.scores_grad(Z, torch.zeros_like(Z), Y, ROW, ws=WS[:need(6, 10) - 1]), text="workspace")


def test_operands_are_refused():
    for z, y in [(Z.double(), Y), (Z, Y.long()), (Z, Y[:5]), (Z.half(), Y), (Z[0], Y), (Z[:, ::2], Y), (torch.zeros(6, 0), Y)]:
        refused(lambda: hb.scores(z, y, ROW.clone(), ws=WS))
        refused(lambda: hb.scores_grad(z, torch.zeros_like(z), y, ROW, ws=WS))
    refused(lambda: hb.scores(Z, None, logp=ROW, ws=WS), text="d_y")
    refused(lambda: hb.scores(Z, Y, logp=ROW[:5], ws=WS))
    refused(lambda: hb.scores(Z, Y, top_logp=TL, ws=WS))
    refused(lambda: hb.scores(Z, Y, top_class=TC.long(), ws=WS))
    refused(lambda: hb.scores(Z, Y, top_class=TC[:5], ws=WS))
    refused(lambda: hb.scores(Z, Y, top_class=TC[:, :2], ws=WS))
    refused(lambda: hb.scores(Z, Y, top_class=TC, top_logp=TL[:, :2].contiguous(), ws=WS))
    refused(lambda: hb.scores(Z, Y, top_class=torch.zeros(6, 65, dtype=torch.int32), ws=WS), text="top")
    refused(lambda: hb.scores_grad(Z, torch.zeros_like(Z), None, g_logp=ROW, ws=WS), text="d_y")
    refused(lambda: hb.scores_grad(Z, torch.zeros_like(Z), Y, ws=WS), text="d_g")
    refused(lambda: hb.scores_grad(Z, torch.zeros(6, 11), Y, ROW, ws=WS))
    refused(lambda: hb.scores_grad(Z, torch.zeros(6, 10, dtype=torch.bfloat16), Y, ROW, ws=WS))


def test_overlaps_are_refused():
    row = ROW.clone()
    refused(lambda: hb.scores(Z, Y, logp=row, lse=row, ws=WS), text="overlaps")
    refused(lambda: hb.scores(Z, Y, entropy=Z.view(-1)[:6], ws=WS), text="overlaps")
    refused(lambda: hb.scores(Z, Y, entropy=Y.view(torch.float32), ws=WS), text="overlaps")
    refused(lambda: hb.scores(Z, Y, top_class=TC, top_logp=TC.view(torch.float32), ws=WS), text="overlaps")
    refused(lambda: hb.scores(Z, Y, lse=WS.view(torch.float32)[:6], ws=WS), text="overlaps")
    big = torch.zeros(7, 10)
    refused(lambda: hb.scores_grad(big[:6], big[1:], Y, ROW, ws=WS), text="overlaps")
    refused(lambda: hb.scores_grad(Z, torch.zeros_like(Z), Y, WS.view(torch.float32)[:6], ws=WS), text="overlaps")
    g = torch.zeros(6, 10)
    refused(lambda: hb.scores_grad(Z, g, Y, g.view(-1)[:6], ws=WS), text="overlaps")


def test_the_library_refuses_what_the_binding_cannot_say():
    call, grad = hb.lib().hb_scores_async, hb.lib().hb_scores_grad_async
    z, y, r, w, n = Z.data_ptr(), Y.data_ptr(), ROW.data_ptr(), WS.data_ptr(), WS.nbytes
    for ldz, t, b, k, top in [(9, 0, 6, 10, 0), (10, 2, 6, 10, 0), (10, 0, -1, 10, 0), (10, 0, 6, 0, 0), (10, 0, 6, 10, -1), (10, 0, 6, 10, 65),
                              (10, 0, 6, 10, 3), (1 << 31, 0, 6, 10, 0), (10, 0, (1 << 22) + 1, 10, 0)]:
        assert call(z, ldz, t, y, b, k, top, r, None, None, None, None, w, n, None) == hb.HB_ERR_INVALID, (ldz, t, b, k, top)
    assert call(None, 10, 0, y, 6, 10, 0, r, None, None, None, None, w, n, None) == hb.HB_ERR_INVALID
    assert call(z + 2, 10, 0, y, 6, 10, 0, r, None, None, None, None, w, n, None) == hb.HB_ERR_INVALID
    assert grad(z, 10, 0, y, 6, 10, r, None, None, 10, w, n, None) == hb.HB_ERR_INVALID
    assert grad(z, 10, 0, y, 6, 10, r, None, z, 9, w, n, None) == hb.HB_ERR_INVALID
    assert call(None, 10, 0, None, 0, 10, 0, None, None, None, None, None, w, n, None) == hb.HB_OK  # nothing to do
    assert grad(None, 10, 0, None, 0, 10, None, None, None, 10, w, n, None) == hb.HB_OK


def test_the_definitions():
    """Uniform rows, a row of two classes, and a certain one."""
    z = np.array([[0.0, 0, 0, 0], [np.log(3), 0, -np.inf, -np.inf], [50, 0, 0, 0]])
    _, logp, lse, H, classes, tops, _, _ = ref.scores_ref(z, np.array([2, 1, 0]), 3)
    assert np.allclose(H[:2], [np.log(4), np.log(4) - 0.75 * np.log(3)]) and np.isclose(H[2], 153 * np.exp(-50), rtol=1e-10)
    assert np.allclose(logp[:2], [-np.log(4), -np.log(4)]) and np.isclose(logp[2], -3 * np.exp(-50))
    assert classes.tolist() == [[0, 1, 2], [0, 1, -1], [0, 1, 2]] and tops[1, 2] == -np.inf
