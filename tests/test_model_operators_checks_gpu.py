"""What the calls of a handle with a loss of their own refuse, and what its profile says of them."""
import pytest
import torch

import hb_inputs as hi
import paper_2004_08771_amd as hb
import test_model_operators_gpu as networks

pytestmark = pytest.mark.gpu

F32, BF16 = hb.HB_F32, hb.HB_BF16_F32MASTER
CE = hi.LOSS_SOFTMAX_CE


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_outputs_of_a_handle_that_overlap_are_refused(dtype):
    """One allocation cut into pieces that meet: outputs with each other, with the labels, the input, and what a row has besides."""
    B, dims = 32, (8, 16, 4)
    m = hb.Model(dims, hi.ACT_SIGMOID, CE).configure(dtype, B)
    P = m.num_params
    X = torch.zeros(B, 8, device="cuda", dtype=torch.float32 if dtype == F32 else torch.bfloat16)
    flat_x = X.view(-1).view(torch.float32)
    y = torch.zeros(B, dtype=torch.int32, device="cuda")
    buf = torch.zeros(P + 100, device="cuda")
    v, w, r, st = [torch.zeros(B, device="cuda") for _ in range(4)]
    seq, pref = torch.tensor([0, 5, 32], dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda")
    pol = hb.policy_args(B, v, w, ref=r, weight=buf[:B], kl_coef=0.1)
    prf = hb.preference_args(seq, pref)
    labels = y.view(torch.float32)
    refused = [
        lambda: m.batch_logprob_async(X, y, B, buf[:B], buf[B - 1:2 * B - 1]), lambda: m.batch_logprob_async(X, y, B, buf[1:], buf[:B]),
        lambda: m.batch_logprob_async(X, y, B, labels), lambda: m.batch_logprob_async(X, y, B, v, labels),
        lambda: m.batch_logprob_async(X, y, B, flat_x[-B:]), lambda: m.batch_logprob_async(X, y, B, v, flat_x),
        lambda: m.policy_step_async(X, y, B, 0.1, pol, flat_x[-4:]), lambda: m.policy_step_async(X, y, B, 0.1, pol, st, labels),
        lambda: m.policy_step_async(X, y, B, 0.1, pol, st, buf[B - 1:]), lambda: m.policy_step_async(X, y, B, 0.1, pol, st[4:], st[:B]),
        lambda: m.policy_grad_async(X, y, B, pol, buf, st), lambda: m.policy_grad_async(X, y, B, pol, buf[B:], buf[B + P - 1:]),
        lambda: m.policy_grad_async(X, y, B, pol, buf[B:], st, buf[B + 3:]),
        lambda: m.preference_step_async(X, y, B, 0.1, prf, st, st[3:]), lambda: m.preference_step_async(X, y, B, 0.1, prf, labels),
        lambda: m.preference_step_async(X, y, B, 0.1, prf, st, pref), lambda: m.preference_grad_async(X, y, B, prf, buf, buf[P - 1:]),
        lambda: m.preference_grad_async(X, y, B, prf, buf, st, buf[7:]), lambda: m.preference_grad_async(X, y, B, prf, flat_x[-1:], st),
    ]
    for i, call in enumerate(refused):
        with pytest.raises(hb.HbError) as e:
            call()
        assert e.value.code == hb.HB_ERR_INVALID and "overlaps" in str(e.value), i
    # side by side is fine
    m.batch_logprob_async(X, y, B, buf[:B], buf[B:2 * B])
    m.policy_grad_async(X, y, B, pol, buf[B:B + P], buf[B + P:B + P + 4], buf[B + P + 4:B + P + 4 + B])
    m.preference_grad_async(X, y, B, prf, buf[B:B + P], buf[B + P:B + P + 4], buf[B + P + 4:B + P + 6])
    torch.cuda.synchronize()
    assert torch.isfinite(buf).all()
    m.destroy()


# calls whose rows go through registers once, are cut into chunks that the gradient's kernel or one of their own joins; few pairs, whose
# sums the gradient's kernel makes, and many
PROFILED = [
    ("policy", (24, 16, 1000), 200, 0, {0: "rw", 1: ""}), ("policy", (24, 16, 7), 32, 0, {0: "rw"}), ("policy", (24, 16, 50003), 20, 0, {0: "r", 2: "rw"}),
    ("logprob", (24, 16, 1000), 200, 0, {0: "r"}), ("logprob", (24, 16, 50003), 20, 0, {0: "r", 1: ""}),
    ("preference", (24, 16, 1000), 200, 2, {0: "r", 2: "rw"}), ("preference", (24, 16, 7), 3000, 2, {0: "r", 1: "", 2: "rw"}),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind,dims,B,pairs,passes", PROFILED)
def test_profile_has_every_launch_of_a_loss(kind, dims, B, pairs, passes, dtype):
    """An entry for each pass, with what it has to move: the logits are fp32, the gradient is of the handle's type."""
    K = dims[-1]
    m = hb.Model(dims, hi.ACT_SIGMOID, CE).configure(dtype, B)
    m.set_params(torch.zeros(m.num_params).numpy())
    X = torch.randn(B, dims[0], device="cuda").to(torch.float32 if dtype == F32 else torch.bfloat16)
    y = torch.zeros(B, dtype=torch.int32, device="cuda")
    v, st, g = torch.zeros(B, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(m.num_params, device="cuda")
    seq = torch.linspace(0, B, 2 * pairs + 1).to(torch.int32).cuda() if pairs else None

    def call():
        if kind == "policy":
            m.policy_grad_async(X, y, B, hb.policy_args(B, v, v), g, st)
        elif kind == "preference":
            m.preference_grad_async(X, y, B, hb.preference_args(seq), g, st)
        else:
            m.batch_logprob_async(X, y, B, v)

    call()
    m.profile_enable(True)
    call()
    call()
    got = {s["layer"]: s for s in m.profile_read() if s["kind"] == 3}
    m.profile_enable(False)
    assert set(got) == set(passes)
    for i, moved in passes.items():
        s = got[i]
        assert s["launches"] == 2 and s["total_ms"] > 0
        want = (4 * B * (K + 1) if "r" in moved else 0) + ((4 if dtype == F32 else 2) * B * K if "w" in moved else 0)
        assert s["bytes_per_launch"] == want or (not moved and s["bytes_per_launch"] > 0)
    m.destroy()


@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("dims,act,dtype,B", [((24, 16, 53001), hi.ACT_SIGMOID, F32, 6), ((24, 16, 53001), hi.ACT_SIGMOID, BF16, 6),
                                              ((24, 16, 40003), hi.ACT_SIGMOID, BF16, 20)])
def test_losses_of_networks_whose_rows_are_cut_into_chunks(dims, act, dtype, B, p):
    """The tests of a handle's gradients, with outputs so wide that few rows go in chunks whatever they are read for."""
    networks.test_policy_gradient_of_a_network(dims, act, dtype, B, p)
    networks.test_preference_gradient_of_a_network(dims, act, dtype, B, p)


def test_dropout_leaves_the_backward_products_as_fast():
    """Sigmoid networks in bf16: the derivative's activations come from their transposed copy with dropout, too.  Read across the rows they
    make these products 1.5 to 2.2 times as long; the bound is half way."""
    dims, B = (512, 4096, 4096, 1024), 8192
    m = hb.Model(dims, hi.ACT_SIGMOID, CE).configure(BF16, B)
    m.set_params((torch.randn(m.num_params) * 0.02).numpy())
    X = torch.randn(B, dims[0], device="cuda").bfloat16()
    y = torch.randint(0, dims[-1], (B,), dtype=torch.int32, device="cuda")
    g = torch.zeros(m.num_params, device="cuda")
    times = {}
    for p in (0.0, 0.2):
        m.set_dropout(p, 3)
        m.batch_grad(X, y, B, g)
        best = []
        for _ in range(5):
            m.profile_enable(True)
            m.batch_grad(X, y, B, g)
            best.append(sum(s["total_ms"] for s in m.profile_read() if s["kind"] == 1))
            m.profile_enable(False)
        times[p] = min(best)
    assert times[0.0] > 0 and times[0.2] < 1.3 * times[0.0], times
    m.destroy()
