"""The operators on device tensors whose speed is measured, with their plain forms.

  dropout     every element is kept with probability 1 - p, by a counter-based generator (Philox4x32-10): the mask is never
              stored, and the backward pass is the same call on the gradient
  logprob     log-probabilities of the chosen classes of B rows of logits, and with `grad` the gradient of a weighted sum of them
  policy      the clipped policy loss with a KL term to a reference, and its gradient in the logits
  preference  the loss over paired log ratios of sequences of rows, and its gradient in the logits

Where a row of logits has a label outside [0, K), it takes no part (padding): its log-probability and its gradient are zero.
`own` false computes the plain forms with elementary torch operations, true calls the framework.
"""
import math

import torch

own = False

F32, BF16 = "f32", "bf16"
TYPES = {F32: (torch.float32, 4), BF16: (torch.bfloat16, 2)}
P_DROP, CLIP, KL_COEF, BETA, SMOOTHING = 0.1, (0.2, 0.28), 0.04, 0.1, 0.05
PAD = 0.1  # share of rows without a choice


def listed():
    return [
        # a ragged hidden layer and a few rows: latency
        {"name": "dropout-61x983-f32", "kind": "dropout", "rows": 61, "cols": 983, "dtype": F32},
        # a hidden layer of the covtype network at the headline batch
        {"name": "dropout-4096x512-f32", "kind": "dropout", "rows": 4096, "cols": 512, "dtype": F32},
        # a hidden layer of the bf16 workload
        {"name": "dropout-16384x4096-bf16", "kind": "dropout", "rows": 16384, "cols": 4096, "dtype": BF16},
        # the actions of a small policy network, as they are taken
        {"name": "logprob-4096x7-f32", "kind": "logprob", "rows": 4096, "classes": 7, "dtype": F32, "grad": False},
        # a reference's log-probabilities over a vocabulary
        {"name": "logprob-8192x32000-bf16", "kind": "logprob", "rows": 8192, "classes": 32000, "dtype": BF16, "grad": False},
        # both directions: the 983-way network at a ragged batch, and a vocabulary
        {"name": "logprob-grad-2047x983-f32", "kind": "logprob", "rows": 2047, "classes": 983, "dtype": F32, "grad": True},
        {"name": "logprob-grad-4096x32000-bf16", "kind": "logprob", "rows": 4096, "classes": 32000, "dtype": BF16, "grad": True},
        # a policy step of a small network: latency
        {"name": "policy-256x7-f32", "kind": "policy", "rows": 256, "classes": 7, "dtype": F32},
        # a micro-batch of sampled tokens over an odd vocabulary, the largest call
        {"name": "policy-8192x50257-bf16", "kind": "policy", "rows": 8192, "classes": 50257, "dtype": BF16},
        # fewer rows than compute units, each of half a megabyte
        {"name": "policy-24x131072-f32", "kind": "policy", "rows": 24, "classes": 131072, "dtype": F32},
        # a few short compared trajectories
        {"name": "preference-4x983-f32", "kind": "preference", "pairs": 4, "rows": 167, "classes": 983, "dtype": F32},
        # compared answers over a vocabulary
        {"name": "preference-16x32000-bf16", "kind": "preference", "pairs": 16, "rows": 8111, "classes": 32000, "dtype": BF16},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: networks' outputs of 2 .. 1000 classes and vocabularies up to 2^18, one row to many, any remainder."""
    kind = rng.choice(["dropout", "logprob", "logprob", "policy", "policy", "preference"])
    dtype = rng.choice([F32, BF16])
    most = (780 << 20) // TYPES[dtype][1]  # elements
    if kind == "dropout":
        cols = _log_int(rng, 1, 1 << 17)
        if rng.random() < 0.5:
            cols = max(8, cols // 8 * 8)
        return {"kind": kind, "rows": _log_int(rng, 1, min(1 << 16, (1 << 26) // cols)), "cols": cols, "dtype": dtype}
    classes = _log_int(rng, 2, 1000) if rng.random() < 0.4 else _log_int(rng, 1000, 1 << 18)
    if rng.random() < 0.3:
        classes = max(8, classes // 8 * 8)
    rows = _log_int(rng, 1, min(1 << 15, most // classes))
    case = {"kind": kind, "rows": rows, "classes": classes, "dtype": dtype}
    if kind == "logprob":
        case["grad"] = rng.random() < 0.5
    if kind == "preference":
        case["pairs"] = _log_int(rng, 1, max(1, min(64, rows // 4)))
    return case


def _counts(case):
    """(rows that take part, rows of the sequences): the rest is padding, or stands behind the last sequence."""
    used = case["rows"] - (case["rows"] // 50 if case["kind"] == "preference" else 0)
    return used - int(PAD * used), used


def work(case):
    size = TYPES[case["dtype"]][1]
    if case["kind"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * size * n, "flops": n}
    live, used = _counts(case)
    K = case["classes"]
    if case["kind"] == "logprob":  # logits, labels, log-probabilities and normalisers; with grad the incoming and outgoing gradients
        return {"bytes": size * K * (live + (used if case["grad"] else 0)) + (16 if case["grad"] else 12) * used,
                "flops": (6 if case["grad"] else 3) * K * live}
    rows = 20 if case["kind"] == "policy" else 4  # label and what a row has besides
    return {"bytes": size * K * (live + used) + rows * used, "flops": 6 * K * live}


def _seeded(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    g = _seeded(seed)
    dtype, _ = TYPES[case["dtype"]]
    dev = {"device": "cuda", "generator": g}
    if case["kind"] == "dropout":
        x = torch.randn(case["rows"], case["cols"], **dev).to(dtype)
        return {"case": case, "x": x, "out": torch.empty_like(x), "seed": seed * 0x9E3779B97F4A7C15 % (1 << 64), "offset": (3 + seed) % (1 << 63)}
    B, K = case["rows"], case["classes"]
    Z = torch.randn(B, K, **dev).mul_(2.0).to(dtype)
    # choices with the odds of the logits, as sampled; a part of the rows has none
    y = (Z.float() - torch.empty(B, K, device="cuda").exponential_(generator=g).log_()).argmax(1).to(torch.int32)
    live, used = _counts(case)
    none = torch.randperm(used, **dev)[:used - live]
    y[none] = -1
    ws = torch.empty(65536 + 64 * B, dtype=torch.uint8, device="cuda")
    state = {"case": case, "Z": Z, "y": y, "ws": ws, "logp": torch.zeros(B, device="cuda"), "dZ": torch.zeros_like(Z)}
    if case["kind"] == "logprob":
        state["lse"] = torch.zeros(B, device="cuda")
        state["g"] = torch.randn(B, **dev)
        return state
    state["stats"] = torch.zeros(4, device="cuda")
    at = y.long().clamp(min=0)
    lp = Z.float().gather(1, at[:, None])[:, 0] - torch.logsumexp(Z.float(), 1)
    if case["kind"] == "policy":  # sampled by a policy a few steps old, a reference further off, advantages of unit variance
        state["old"] = lp + 0.15 * torch.randn(B, **dev)
        state["ref"] = lp + 0.4 * torch.randn(B, **dev)
        state["adv"] = torch.randn(B, **dev)
        state["weight"] = torch.full((B,), 1.0 / max(1, live), device="cuda")
        return state
    N = case["pairs"]  # 2 N sequences of any lengths, one after the other
    cuts = torch.sort(torch.randint(0, used + 1, (2 * N - 1,), **dev)).values
    state["seq"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), used)]).to(torch.int32)
    run_sum = torch.cat([lp.new_zeros(1, dtype=torch.float64), torch.where(y >= 0, lp, 0.0).double().cumsum(0)])
    sums = run_sum[state["seq"][1:].long()] - run_sum[state["seq"][:-1].long()]
    state["ref"] = sums.float() + 6.0 * torch.randn(2 * N, **dev)
    state["seq_logp"] = torch.zeros(2 * N, device="cuda")
    return state


def _keep(rows, cols, seed, offset, device):
    """16 bits of Philox4x32-10 for every element: columns in groups of eight, counter (group, row, offset), key `seed`."""
    low = 0xFFFFFFFF
    groups = (cols + 7) // 8
    c0 = torch.arange(groups, device=device).expand(rows, groups)
    c1 = torch.arange(rows, device=device)[:, None].expand(rows, groups)
    c2, c3 = torch.full_like(c0, offset & low), torch.full_like(c0, offset >> 32)
    k0, k1 = seed & low, seed >> 32

    def product(a, x):  # high and low half of a 32 x 32 -> 64 bit product, in 64 signed bits
        u, v = a * (x >> 16), a * (x & 0xFFFF)
        return (u + (v >> 16)) >> 16, (((u & 0xFFFF) << 16) + v) & low

    for _ in range(10):
        h0, l0 = product(0xD2511F53, c0)
        h1, l1 = product(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], -1)
    return torch.stack([words & 0xFFFF, words >> 16], -1).reshape(rows, groups * 8)[:, :cols]


def _row_terms(Z, y, weight=None):
    """Of every row: whether it takes part, its choice, exp(z - max), and in 64 bits the sum without the choice, the whole sum,
    the log-probability and the logarithm of the sum of exponentials."""
    z = Z.float()
    top = z.amax(1)
    part = (y >= 0) & (y < Z.shape[1]) & (top != -math.inf)
    if weight is not None:
        part = part & (weight != 0)
    z, top = torch.where(part[:, None], z, 0.0), torch.where(part, top, 0.0)
    at = torch.where(part, y, 0).long()[:, None]
    e = torch.exp(z - top[:, None])
    d = (z.gather(1, at)[:, 0] - top).double()
    chosen = torch.exp(d)
    others = e.scatter(1, at, 0.0).sum(1, dtype=torch.float64)
    s = others + chosen
    lp = torch.where(others < chosen, -torch.log1p(others / chosen), d - torch.log(s))
    return part, at, e, others, s, torch.where(part, lp, 0.0), torch.where(part, top.double() + torch.log(s), 0.0)


def _logit_grad(terms, g, dtype):
    """g ([k = y] - p_k) for every row, zero where a row takes no part; 1 - p_y from the sum without the choice."""
    part, at, e, others, s, _, _ = terms
    p = (e * (1 / s).float()[:, None]).scatter(1, at, (-others / s).float()[:, None])
    return torch.where(part[:, None], p * -g.float()[:, None], 0.0).to(dtype)


def run(state):
    if own:
        import paper_2004_08771_amd as hb
    case = state["case"]
    if case["kind"] == "dropout":
        x, seed, offset = state["x"], state["seed"], state["offset"]
        if own:
            hb.dropout(x, state["out"], P_DROP, seed, offset)
            return {"out": state["out"]}
        t = int(P_DROP * 65536 + 0.5)
        keep = _keep(*x.shape, seed, offset, x.device) >= t
        return {"out": torch.where(keep, x.float() * (65536 / (65536 - t)), 0.0).to(x.dtype)}
    Z, y, ws = state["Z"], state["y"], state["ws"]
    if case["kind"] == "logprob":
        if own:
            hb.logprob(Z, y, state["logp"], state["lse"], ws=ws)
            out = {"logp": state["logp"], "lse": state["lse"]}
            if case["grad"]:
                hb.logprob_grad(Z, y, state["logp"], state["lse"], state["g"], state["dZ"])
                out["dZ"] = state["dZ"]
            return out
        terms = _row_terms(Z, y)
        out = {"logp": terms[5].float(), "lse": terms[6].float()}
        if case["grad"]:
            out["dZ"] = _logit_grad(terms, state["g"], Z.dtype)
        return out
    if case["kind"] == "policy":
        if own:
            hb.policy_loss(Z, y, state["old"], state["adv"], state["stats"], dZ=state["dZ"], ref=state["ref"], weight=state["weight"],
                           clip=CLIP, kl_coef=KL_COEF, logp=state["logp"], ws=ws)
            return {"stats": state["stats"], "logp": state["logp"], "dZ": state["dZ"]}
        terms = _row_terms(Z, y, state["weight"])
        part, lp = terms[0], terms[5]
        adv, w = state["adv"].double(), torch.where(part, state["weight"], 0.0).double()
        r = torch.exp(torch.where(part, lp - state["old"].double(), 0.0))
        pg = -torch.minimum(r * adv, r.clamp(1 - CLIP[0], 1 + CLIP[1]) * adv)
        cut = ((adv > 0) & (r > 1 + CLIP[1])) | ((adv < 0) & (r < 1 - CLIP[0]))
        d = torch.where(part, state["ref"].double() - lp, 0.0)
        kl = torch.expm1(d) - d
        g = w * (torch.where(cut, 0.0, -r * adv) - KL_COEF * torch.expm1(d))
        sums = torch.stack([(w * pg).sum(), (w * kl).sum(), (w * cut).sum()])
        stats = torch.stack([sums[0] + KL_COEF * sums[1], sums[0], sums[1], sums[2]]).float()
        return {"stats": stats, "logp": lp.float(), "dZ": _logit_grad(terms, g, Z.dtype)}
    seq, N = state["seq"], case["pairs"]
    if own:
        hb.preference_loss(Z, y, seq, state["stats"], dZ=state["dZ"], ref=state["ref"], beta=BETA, smoothing=SMOOTHING,
                           seq_logp=state["seq_logp"], ws=ws)
        return {"stats": state["stats"], "seq_logp": state["seq_logp"], "dZ": state["dZ"]}
    used = _counts(case)[1]  # the rows behind the last sequence stay as they are
    terms = _row_terms(Z[:used], y[:used])
    run_sum = torch.cat([terms[5].new_zeros(1), terms[5].cumsum(0)])
    at = seq.long()
    sums = run_sum[at[1:]] - run_sum[at[:-1]]
    gain = (sums - state["ref"].double()).view(N, 2)
    h = gain[:, 0] - gain[:, 1]
    softplus = lambda v: v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))  # noqa: E731
    loss = (1 - SMOOTHING) * softplus(-BETA * h) + SMOOTHING * softplus(BETA * h)
    dh = BETA / N * (SMOOTHING / (1 + torch.exp(-BETA * h)) - (1 - SMOOTHING) / (1 + torch.exp(BETA * h)))
    rows = torch.searchsorted(at[1:], torch.arange(used, device=Z.device), right=True)
    g = torch.stack([dh, -dh], 1).view(-1)[rows]
    state["dZ"][:used] = _logit_grad(terms, g, Z.dtype)
    stats = torch.stack([loss.mean(), (h > 0).double().mean(), BETA * gain[:, 0].mean(), BETA * gain[:, 1].mean()]).float()
    return {"stats": stats, "seq_logp": sums.float(), "dZ": state["dZ"]}


def exact(case, seed):
    """From the definitions in 64 bits, a block of rows at a time."""
    state = prepare(case, seed)
    if case["kind"] == "dropout":
        x, key, off, m32 = state["x"], state["seed"], state["offset"], (1 << 32) - 1
        rows, cols = x.shape
        if cols > 1 << 15:
            return None
        t, keep = int(P_DROP * 65536 + 0.5), torch.empty(rows, cols, dtype=torch.bool, device="cuda")
        for j in range(0, cols, 8):  # a counter block for a column of groups
            ctr = [torch.full((rows,), j // 8, device="cuda"), torch.arange(rows, device="cuda"),
                   torch.full((rows,), off & m32, device="cuda"), torch.full((rows,), off >> 32, device="cuda")]
            for n in range(10):
                ka, kb = (key + n * 0x9E3779B9) & m32, ((key >> 32) + n * 0xBB67AE85) & m32
                wide = []
                for a, x0 in ((0xD2511F53, ctr[0]), (0xCD9E8D57, ctr[2])):
                    # 64-bit products wrap: the low 32 bits are right, the high ones from 11-bit pieces
                    pieces = [(x0 >> s) & 0x7FF for s in (0, 11, 22)]
                    acc = a * pieces[0]
                    lowest, acc = acc & 0x7FF, (acc >> 11) + a * pieces[1]
                    middle, acc = acc & 0x7FF, (acc >> 11) + a * pieces[2]
                    wide.append((acc >> 10, ((acc & 0x3FF) << 22) | (middle << 11) | lowest))
                ctr = [wide[1][0] ^ ctr[1] ^ ka, wide[1][1], wide[0][0] ^ ctr[3] ^ kb, wide[0][1]]
            for e in range(min(8, cols - j)):
                keep[:, j + e] = ((ctr[e // 2] >> (16 * (e % 2))) & 0xFFFF) >= t
        return {"out": x.double() * keep / (1 - t / 65536)}
    Z, y, K = state["Z"], state["y"].long(), case["classes"]
    used = _counts(case)[1]
    part = (y >= 0)[:used]
    grad = case["kind"] != "logprob" or case["grad"]
    logp, lse = torch.zeros(len(y), dtype=torch.float64, device="cuda"), torch.zeros(len(y), dtype=torch.float64, device="cuda")
    step = max(1, (1 << 27) // K)

    def blocks():
        for a in range(0, used, step):
            b = min(used, a + step)
            yield a, b, torch.log_softmax(Z[a:b].double(), 1)

    for a, b, lsm in blocks():
        logp[a:b] = torch.where(part[a:b], lsm.gather(1, y[a:b].clamp(min=0)[:, None])[:, 0], 0.0)
        lse[a:b] = torch.where(part[a:b], Z[a:b, 0].double() - lsm[:, 0], 0.0)
    if case["kind"] == "logprob":
        g, out = state["g"].double(), {"logp": logp, "lse": lse}
    elif case["kind"] == "policy":
        A, w = state["adv"].double(), state["weight"].double() * part
        ratio, d = torch.exp(logp - state["old"].double()), state["ref"].double() - logp
        held = torch.where(A > 0, ratio.clamp(max=1 + CLIP[1]), ratio.clamp(min=1 - CLIP[0]))
        cut = (held != ratio) & (A != 0)
        obj, kl = -(w * held * A).sum(), (w * (torch.exp(d) - d - 1)).sum()
        g = w * (-(ratio * A) * ~cut + KL_COEF * (1 - torch.exp(d)))
        out = {"stats": torch.stack([obj + KL_COEF * kl, obj, kl, (w * cut).sum()]), "logp": logp}
    else:
        at, N = state["seq"].tolist(), case["pairs"]
        sums = torch.stack([logp[at[q]:at[q + 1]].sum() for q in range(2 * N)])
        up, down = [(sums - state["ref"].double())[i::2] for i in (0, 1)]
        z = BETA * (up - down)
        loss = -(1 - SMOOTHING) * torch.nn.functional.logsigmoid(z) - SMOOTHING * torch.nn.functional.logsigmoid(-z)
        slope = BETA / N * (torch.sigmoid(z) - (1 - SMOOTHING))
        g = torch.zeros(len(y), dtype=torch.float64, device="cuda")
        for q in range(2 * N):
            g[at[q]:at[q + 1]] = slope[q // 2] * (1 - 2 * (q % 2))
        out = {"stats": torch.stack([loss.mean(), (z > 0).double().mean(), BETA * up.mean(), BETA * down.mean()]), "seq_logp": sums}
    if grad:
        dZ = torch.zeros(len(y), K, dtype=torch.float64, device="cuda")
        for a, b, lsm in blocks():
            p = lsm.exp_()
            p[torch.arange(b - a, device="cuda"), y[a:b].clamp(min=0)] -= 1
            dZ[a:b] = -(g[a:b] * part[a:b])[:, None] * p
        out["dZ"] = dZ
    return out
