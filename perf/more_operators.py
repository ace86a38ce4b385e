"""More operators on device tensors whose speed is measured, with their plain forms.

  ortho        a matrix with its singular values brought near 1 by Newton-Schulz products: X = G / (|G| + eps), then
               steps of A = X X^T, X = a X + (b A + c A^2) X (on the transpose where there are more rows than columns)
  muon         a step of training with it, for all matrices of a network in one call: momentum, the orthogonalised
               update, weight decay
  scores       log-probabilities of given classes, the normaliser, the entropy and the top alternatives of rows of logits
  scores_grad  the gradient in the logits of a weighted sum of log-probabilities and entropies

`own` false computes the plain forms with elementary torch operations, true calls the framework.
"""
import math

import torch

own = False

F32, BF16 = "f32", "bf16"
TYPES = {F32: (torch.float32, 4), BF16: (torch.bfloat16, 2)}
COEF, STEPS, EPS = (3.4445, -4.7750, 2.0315), 5, 1e-7
LR, MOMENTUM, DECAY = 5e-5, 0.95, 0.1  # of a schedule's end
PAD = 0.1  # share of rows without a given class


def listed():
    return [
        # the first layer of the covtype network: latency
        {"name": "ortho-512x54-f32", "kind": "ortho", "rows": 512, "cols": 54, "dtype": F32},
        # the output layer of the 983-way network: more rows than columns, odd
        {"name": "ortho-983x512-f32", "kind": "ortho", "rows": 983, "cols": 512, "dtype": F32},
        # the output layer of the bf16 workload
        {"name": "ortho-1000x4096-bf16", "kind": "ortho", "rows": 1000, "cols": 4096, "dtype": BF16},
        # a hidden layer of the bf16 workload, the most work in one matrix
        {"name": "ortho-4096x4096-bf16", "kind": "ortho", "rows": 4096, "cols": 4096, "dtype": BF16},
        # a training step of the covtype network: small matrices, all at once
        {"name": "muon-54-512x4-7-f32", "kind": "muon", "dims": "54,512,512,512,512,7", "dtype": F32},
        # a training step of the 300-1024x3-2 network
        {"name": "muon-300-1024x3-2-f32", "kind": "muon", "dims": "300,1024,1024,1024,2", "dtype": F32},
        # a training step of the bf16 workload with its fp32 master weights
        {"name": "muon-2048-4096x3-1000-bf16", "kind": "muon", "dims": "2048,4096,4096,4096,1000", "dtype": BF16},
        # the answers of a small policy network with their runners-up: latency
        {"name": "scores-256x7-top3-f32", "kind": "scores", "rows": 256, "classes": 7, "top": 3, "dtype": F32},
        # one token over a long vocabulary, as it is served
        {"name": "scores-1x131072-top20-f32", "kind": "scores", "rows": 1, "classes": 131072, "top": 20, "dtype": F32},
        # a batch of texts over an odd vocabulary, as they are judged
        {"name": "scores-8192x50257-top5-bf16", "kind": "scores", "rows": 8192, "classes": 50257, "top": 5, "dtype": BF16},
        # a policy's gradient with an entropy bonus: the 983-way network at a ragged batch, and a vocabulary
        {"name": "scores-grad-2047x983-f32", "kind": "scores_grad", "rows": 2047, "classes": 983, "dtype": F32},
        {"name": "scores-grad-4096x32000-bf16", "kind": "scores_grad", "rows": 4096, "classes": 32000, "dtype": BF16},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: matrices of 1 .. 8192 rows and columns, networks of up to six layers; rows of 2 .. 2^18 classes, one row to many."""
    kind = rng.choice(["ortho", "ortho", "muon", "scores", "scores", "scores_grad"])
    dtype = rng.choice([F32, BF16])
    if kind == "ortho":
        rows, cols = _log_int(rng, 1, 8192), _log_int(rng, 1, 8192)
        if min(rows, cols) ** 2 * max(rows, cols) > 1 << 36:
            rows = rows // 2
        return {"kind": kind, "rows": rows, "cols": cols, "dtype": dtype}
    if kind == "muon":
        dims = [_log_int(rng, 2, 2560) for _ in range(rng.randint(2, 7))]
        return {"kind": kind, "dims": ",".join(map(str, dims)), "dtype": dtype}
    most = (780 << 20) // TYPES[dtype][1]  # elements
    classes = _log_int(rng, 2, 1000) if rng.random() < 0.4 else _log_int(rng, 1000, 1 << 18)
    if rng.random() < 0.3:
        classes = max(8, classes // 8 * 8)
    case = {"kind": kind, "rows": _log_int(rng, 1, min(1 << 15, most // classes)), "classes": classes, "dtype": dtype}
    if kind == "scores":
        case["top"] = rng.choice([0, 1, 5, 20, 64])
    return case


def _shapes(case):
    """(rows, columns) of the case's matrices: out x in, as a layer has them."""
    if case["kind"] == "ortho":
        return [(case["rows"], case["cols"])]
    dims = [int(d) for d in case["dims"].split(",")]
    return list(zip(dims[1:], dims[:-1]))


def work(case):
    size = TYPES[case["dtype"]][1]
    if case["kind"] in ("ortho", "muon"):
        n = sum(r * c for r, c in _shapes(case))
        # of the products X X^T and A A^T, which are symmetric, half
        flops = sum(STEPS * (3 * min(s) ** 2 * max(s) + min(s) ** 3) for s in _shapes(case))
        # muon: weights and momenta there and back, the gradient
        return {"bytes": (2 * size if case["kind"] == "ortho" else 16 + size) * n, "flops": flops}
    B, K = case["rows"], case["classes"]
    if case["kind"] == "scores":
        live = B - int(PAD * B)
        return {"bytes": size * K * live + (16 + 8 * case["top"]) * B, "flops": 5 * K * live}
    live = B - int(PAD * B)
    return {"bytes": size * K * (live + B) + 12 * B, "flops": 9 * K * live}


def _gradient(r, c, dev):
    """As a layer's gradient: units of different sizes and two directions that stand out."""
    G = torch.randn(r, c, **dev)
    G *= torch.exp(0.5 * torch.randn(r, 1, **dev)) * torch.exp(0.5 * torch.randn(1, c, **dev))
    for s in (8.0, 4.0):
        G += s * (r ** -0.5 + c ** -0.5) * torch.randn(r, 1, **dev) * torch.randn(1, c, **dev)
    return G * 1e-3


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype, _ = TYPES[case["dtype"]]
    dev = {"device": "cuda", "generator": g}
    if case["kind"] in ("ortho", "muon"):
        shapes = _shapes(case)
        # the padded halves of every matrix that the products go through, twice over: generous
        ws = torch.empty(sum(64 * (r + 512) * (c + 512) + 32 * (min(r, c) + 512) ** 2 for r, c in shapes), dtype=torch.uint8, device="cuda")
        state = {"case": case, "ws": ws, "G": [_gradient(r, c, dev).to(dtype) for r, c in shapes]}
        if case["kind"] == "ortho":
            state["out"] = [torch.empty_like(G) for G in state["G"]]
        else:
            state["W"] = [torch.randn(r, c, **dev) * (2.0 / (r + c)) ** 0.5 for r, c in shapes]
            state["M"] = [4.0 * _gradient(r, c, dev) for r, c in shapes]
            state["scale"] = [0.2 * max(s) ** 0.5 for s in shapes]
        return state
    B, K = case["rows"], case["classes"]
    Z = torch.randn(B, K, **dev).mul_(2.0).to(dtype)
    # classes with the odds of the logits, as sampled; a part of the rows has none
    y = (Z.float() - torch.empty(B, K, device="cuda").exponential_(generator=g).log_()).argmax(1).to(torch.int32)
    y[torch.randperm(B, **dev)[:int(PAD * B)]] = -1
    state = {"case": case, "Z": Z, "y": y, "ws": torch.empty(65536 + (64 + 2048 * (K // 4096 + 1)) * B, dtype=torch.uint8, device="cuda")}
    if case["kind"] == "scores":
        for name in ("logp", "lse", "entropy"):
            state[name] = torch.zeros(B, device="cuda")
        state["top_class"] = torch.zeros(B, case["top"], dtype=torch.int32, device="cuda")
        state["top_logp"] = torch.zeros(B, case["top"], device="cuda")
    else:
        state["g_logp"] = torch.randn(B, **dev) / B
        state["g_entropy"] = torch.full((B,), -0.01 / B, device="cuda")
        state["dZ"] = torch.zeros_like(Z)
    return state


def _newton_schulz(G):
    """In 32 bits; sums of squares in 64."""
    X = G.T if G.shape[0] > G.shape[1] else G
    X = (X.double() / (X.double().square().sum().sqrt() + EPS)).float()
    a, b, c = COEF
    for _ in range(STEPS):
        A = X @ X.T
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.T if G.shape[0] > G.shape[1] else X


def _row_terms(Z, y):
    """Of every row: whether it takes part, z - max, exp of it, and in 64 bits the sum of exponentials without the largest logit,
    the whole sum, the log-probability of its class, the normaliser and the entropy."""
    z = Z.float()
    part = (y >= 0) & (y < Z.shape[1])
    first = z.argmax(1, keepdim=True)
    top = z.gather(1, first)
    d = z - top
    e = torch.exp(d)
    others = e.scatter(1, first, 0.0).sum(1, dtype=torch.float64)
    log_s = torch.log1p(others)
    entropy = log_s - (e * d).sum(1, dtype=torch.float64) / (1 + others)
    at = torch.where(part, y, 0).long()[:, None]
    lp = d.gather(1, at)[:, 0].double() - log_s
    return part, at, d, e, others, log_s, lp, top[:, 0].double() + log_s, entropy


def run(state):
    if own:
        import paper_2004_08771_amd as hb
    case = state["case"]
    if case["kind"] == "ortho":
        if own:
            hb.orthogonalize(state["G"], state["out"], steps=STEPS, coef=COEF, eps=EPS, ws=state["ws"])
            return {"out": state["out"]}
        return {"out": [_newton_schulz(G.float()).to(G.dtype) for G in state["G"]]}
    if case["kind"] == "muon":
        W, M, G, scale = state["W"], state["M"], state["G"], state["scale"]
        if own:
            hb.muon_update(W, G, M, LR, momentum=MOMENTUM, nesterov=True, weight_decay=DECAY, scale=scale, steps=STEPS, coef=COEF, eps=EPS,
                           products=hb.HB_TENSOR_F32 if case["dtype"] == F32 else hb.HB_TENSOR_BF16, ws=state["ws"])
            return {"W": W, "M": M}
        for w, m, g, s in zip(W, M, G, scale):
            m.mul_(MOMENTUM).add_(g.float())
            o = _newton_schulz(m * MOMENTUM + g.float())
            w.copy_(w.double() * (1 - LR * DECAY) - LR * s * o.double())
        return {"W": W, "M": M}
    Z, y, ws = state["Z"], state["y"], state["ws"]
    if case["kind"] == "scores":
        if own:
            hb.scores(Z, y, logp=state["logp"], lse=state["lse"], entropy=state["entropy"], top_class=state["top_class"],
                      top_logp=state["top_logp"], ws=ws)
            return {name: state[name] for name in ("logp", "lse", "entropy", "top_class", "top_logp")}
        part, _, d, _, _, log_s, lp, lse, entropy = _row_terms(Z, y)
        zero = lambda v, no: torch.where(part.view(-1, *[1] * (v.dim() - 1)), v, no)  # noqa: E731
        # the order of fp32 numbers as whole numbers, and behind it the class, the lowest first
        bits = (Z.float() + 0.0).view(torch.int32).long()
        key = (torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) << 32) + (0x7FFFFFFF - torch.arange(Z.shape[1], device=Z.device))
        k = min(case["top"], Z.shape[1])
        classes = 0x7FFFFFFF - (key.topk(k, 1).values & 0xFFFFFFFF)
        out = {"logp": zero(lp, 0.0).float(), "lse": zero(lse, 0.0).float(), "entropy": zero(entropy, 0.0).float()}
        tops = d.gather(1, classes).double() - log_s[:, None]
        gone = case["top"] - k  # there are no more classes
        out["top_class"] = torch.nn.functional.pad(zero(classes, -1), (0, gone), value=-1).to(torch.int32)
        out["top_logp"] = zero(torch.nn.functional.pad(tops, (0, gone), value=-math.inf), 0.0).float()
        return out
    if own:
        hb.scores_grad(Z, state["dZ"], y, g_logp=state["g_logp"], g_entropy=state["g_entropy"], ws=ws)
        return {"dZ": state["dZ"]}
    part, at, d, e, others, log_s, lp, _, entropy = _row_terms(Z, y)
    s = 1 + others
    g, h = state["g_logp"].double(), state["g_entropy"].double()
    p = e * (1 / s).float()[:, None]
    dZ = p * -((d + (entropy - log_s).float()[:, None]) * h.float()[:, None] + g.float()[:, None])
    # the class itself: 1 - p from the sum without it, where it is the largest
    p_at, d_at = torch.exp(lp), d.gather(1, at)[:, 0].double()
    rest = torch.where(d_at == 0, others / s, 1 - p_at)
    dZ = dZ.scatter(1, at, (g * rest - h * p_at * (d_at + entropy - log_s)).float()[:, None])
    return {"dZ": torch.where(part[:, None], dZ, 0.0).to(Z.dtype)}


def exact(case, seed):
    """From the definitions in 64 bits."""
    state = prepare(case, seed)
    a, b, c = COEF

    def orthogonal(U):
        flip = U.shape[0] > U.shape[1]
        X = U.t().contiguous() if flip else U
        X = X / (torch.linalg.norm(X) + EPS)
        for _ in range(STEPS):
            S = X.mm(X.t())
            P = (b * S).addmm_(S, S, alpha=c)
            P.diagonal().add_(a)
            X = P.mm(X)
        return X.t() if flip else X

    if case["kind"] == "ortho":
        return {"out": [orthogonal(G.double()) for G in state["G"]]}
    if case["kind"] == "muon":
        M = [MOMENTUM * m.double() + g.double() for m, g in zip(state["M"], state["G"])]
        W = [w.double() - LR * (DECAY * w.double() + s * orthogonal(g.double() + MOMENTUM * m))
             for w, m, g, s in zip(state["W"], M, state["G"], state["scale"])]
        return {"W": W, "M": M}
    Z, y = state["Z"], state["y"].long()
    (B, K), part = Z.shape, y >= 0
    step = max(1, (1 << 26) // K)
    rows = torch.arange(B, device="cuda")
    if case["kind"] == "scores":
        out = {n: torch.zeros(B, dtype=torch.float64, device="cuda") for n in ("logp", "lse", "entropy")}
        out["top_logp"] = torch.zeros(B, case["top"], dtype=torch.float64, device="cuda")
        for i in range(0, B, step):
            z, at = Z[i:i + step].double(), rows[i:i + step]
            L = torch.log_softmax(z, 1)
            out["logp"][at] = L.gather(1, y[at].clamp(min=0)[:, None])[:, 0]
            out["lse"][at] = torch.logsumexp(z, 1)
            out["entropy"][at] = -(L.exp() * L).sum(1)
            out["top_logp"][at] = torch.nn.functional.pad(L, (0, case["top"]), value=-math.inf).topk(case["top"], 1).values
        for v in out.values():
            v[~part] = 0.0
        return {**out, "top_class": None}
    dZ = torch.zeros(B, K, dtype=torch.float64, device="cuda")
    for i in range(0, B, step):
        at = rows[i:i + step][part[i:i + step]]
        L = torch.log_softmax(Z[at].double(), 1)
        p = L.exp()
        H = -(p * L).sum(1, keepdim=True)
        # d log p_y / dz_k = [k = y] - p_k and d H / dz_k = -p_k (log p_k + H)
        D = -state["g_entropy"][at].double()[:, None] * p * (L + H) - state["g_logp"][at].double()[:, None] * p
        D[torch.arange(len(at), device="cuda"), y[at]] += state["g_logp"][at].double()
        dZ[at] = D
    return {"dZ": dZ}
