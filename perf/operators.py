"""The update half of a GRPO step, as timed and compared cases: from the policy's logits to clipped gradients.

Kinds of case (one entry point each):
  policy   sr_policy_loss: the clipped policy loss with its KL term over ragged token sequences, and the gradient of the
           loss with respect to the logits ("grad": false = the loss alone, as an evaluation pass has it).
  pairs    sr_preference_loss: the paired log-ratio loss over (chosen, rejected) sequences, and its gradient.
  clip     sr_clip_grad_norm: the global 2-norm over a list of gradient tensors, and the list scaled down to a largest norm.

Sizes: vocabularies and hidden sizes of the benchmark configuration (152064, 3584, FFN 18944) and of the small test
configuration (1024, 256, FFN 688), their numbers of sequences and action lengths, and odd sizes between them.
"""
import math

import torch

own = False

F32, BF16, F16 = "float32", "bfloat16", "float16"
BYTES = {F32: 4, BF16: 2, F16: 2}
# hidden, query and kv dims, FFN, vocabulary
MODELS = {"wide": (3584, 3584, 512, 18944, 152064), "tiny": (256, 256, 128, 688, 1024)}
MOST_LOGITS = 4096 * 152064        # of the largest policy case
MOST_PAIR_LOGITS = 2400 * 152064
MOST_GRADS = 1_000_000_000


def _policy(name, seqs, rows, vocab, dtype, reduce, kl, grad=True, masked=0.0, pad=0, grad_scale=1.0):
    return {"name": name, "kind": "policy", "seqs": seqs, "rows": rows, "vocab": vocab, "dtype": dtype, "reduce": reduce, "kl": kl,
            "grad": grad, "masked": masked, "pad": pad, "grad_scale": grad_scale, "clip_low": 0.2, "clip_high": 0.28}


def _pairs(name, pairs, rows, vocab, dtype, masked=0.0, pad=0, smoothing=0.0, grad_scale=1.0):
    return {"name": name, "kind": "pairs", "pairs": pairs, "rows": rows, "vocab": vocab, "dtype": dtype, "masked": masked, "pad": pad,
            "smoothing": smoothing, "grad_scale": grad_scale, "beta": 0.1}


def _clip(name, source, dtype, out, std, model="", layers=0, embed=False, tensors=0, most=0, shapes=0, scale=1.0):
    return {"name": name, "kind": "clip", "source": source, "dtype": dtype, "out": out, "std": std, "model": model, "layers": layers,
            "embed": embed, "tensors": tensors, "most": most, "shapes": shapes, "scale": scale, "max_norm": 1.0}


def listed():
    return [
        # one turn of the small test configuration, 32 sequences of 8 action tokens: launches and host calls count
        _policy("policy-tiny", 32, 256, 1024, F32, "tokens", 0.04),
        # one token of each of the benchmark's 128 sequences, on the single-precision logits that the decoder leaves
        _policy("policy-128x1", 128, 128, 152064, F32, "sequences", 0.04),
        # a turn of the benchmark's rollout as a training program holds it: ragged actions, 32 tokens on average, bf16
        _policy("policy-rollout", 128, 4096, 152064, BF16, "sequences", 0.04),
        # an odd vocabulary in padded rows, half precision with a loss scale, a tenth of the rows masked, no KL term
        _policy("policy-odd-half", 23, 1531, 32011, F16, "tokens", 0.0, masked=0.1, pad=5, grad_scale=4096.0),
        # the loss alone, over the sums of whole sequences: an evaluation pass
        _policy("policy-loss-only", 64, 2048, 152064, BF16, "sums", 0.04, grad=False),
        # a few short pairs of the small configuration
        _pairs("pairs-tiny", 8, 203, 1024, F32),
        # ragged pairs at an odd vocabulary, prompts masked, rows that begin at odd addresses, smoothed labels
        _pairs("pairs-odd", 24, 1701, 50021, BF16, masked=0.3, smoothing=0.1),
        # pairs of the benchmark's vocabulary
        _pairs("pairs-wide", 16, 2400, 152064, BF16),
        # every gradient of the small test configuration: 27 tensors, far below one launch's worth of work
        _clip("clip-tiny", "model", F32, F32, 0.004, model="tiny", layers=2, embed=True),
        # several hundred adapters and vectors of odd lengths, which begin at odd addresses
        _clip("clip-ragged", "ragged", F32, F32, 0.01, tensors=339, most=300_000, shapes=5),
        # one layer at the benchmark's width, bf16 gradients into single precision for the optimizer
        _clip("clip-layer", "model", BF16, F32, 0.002, model="wide", layers=1, scale=0.25),
        # two layers and the embedding at the benchmark's width
        _clip("clip-wide", "model", BF16, BF16, 0.002, model="wide", layers=2, embed=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["policy", "policy", "pairs", "clip"])
    if kind == "clip":
        dtype = rng.choice([F32, BF16, F16])
        out = rng.choice([dtype, F32])
        std = 0.02 * math.exp(rng.uniform(-2.0, 1.0))
        if rng.random() < 0.3:
            return _clip("", "model", dtype, out, std, model=rng.choice(["wide", "tiny"]), layers=1, embed=rng.random() < 0.5) | {
                "scale": rng.choice([1.0, 0.125])}
        tensors = _log(rng, 1, 500)
        most = min(_log(rng, 10, 20_000_000), MOST_GRADS // tensors)
        return _clip("", "ragged", dtype, out, std, tensors=tensors, most=most, shapes=rng.randrange(1 << 20), scale=rng.choice([1.0, 0.125]))
    dtype = rng.choice([F32, BF16, BF16, F16])
    vocab = rng.choice([1024, 152064, 0, 0, 0]) or _log(rng, 500, 152064)
    most = (MOST_LOGITS if kind == "policy" else MOST_PAIR_LOGITS) // vocab * 2 // BYTES[dtype]
    rows = _log(rng, 1 if kind == "policy" else 2, max(4, min(most, 32768)))
    scale = 4096.0 if dtype == F16 else 1.0
    masked, pad = rng.choice([0.0, 0.0, 0.3]), rng.choice([0, 0, 8, 3])
    if kind == "policy":
        return _policy("", min(rows, _log(rng, 1, 512)), rows, vocab, dtype, rng.choice(["tokens", "sequences", "sums"]),
                       rng.choice([0.0, 0.04]), grad=rng.random() < 0.8, masked=masked, pad=pad, grad_scale=scale)
    return _pairs("", min(max(1, rows // 2), _log(rng, 1, 64)), rows, vocab, dtype, masked=masked, pad=pad,
                  smoothing=rng.choice([0.0, 0.1]), grad_scale=scale)


def _sizes(case):
    """Elements of each tensor of a clip case."""
    if case["source"] == "ragged":
        g = torch.Generator().manual_seed(case["shapes"])
        u = torch.rand(case["tensors"], generator=g, dtype=torch.float64)
        return [max(1, int(math.exp(float(x) * math.log(case["most"])))) for x in u]
    H, q, kv, ffn, vocab = MODELS[case["model"]]
    layer = [q * H, kv * H, kv * H, q, kv, kv, H * q, ffn * H, ffn * H, H * ffn, H, H]
    ends = [vocab * H, H] + ([vocab * H] if case["model"] == "tiny" else []) if case["embed"] else []
    return layer * case["layers"] + ends


def work(case):
    if case["kind"] == "clip":
        n = sum(_sizes(case))
        return {"bytes": n * (BYTES[case["dtype"]] + BYTES[case["out"]]), "flops": 3 * n}
    n, b = case["rows"] * case["vocab"], BYTES[case["dtype"]]
    grad = case.get("grad", True)
    # per logit: difference and exponential, sum, comparison; for the gradient difference, exponential and product again
    return {"bytes": n * b * (1 - case["masked"]) + (n * b if grad else 0) + 24 * case["rows"],
            "flops": n * (1 - case["masked"]) * (7 if grad else 4)}


def _cuts(rows, seqs, gen):
    """Row ranges of `seqs` ragged sequences that fill `rows` rows."""
    cuts = torch.sort(torch.randint(0, rows + 1, (seqs - 1,), generator=gen)).values
    even = torch.arange(1, seqs) * rows // seqs
    inner = (cuts + 2 * even) // 3                                 # ragged, but of one order
    return torch.cat([torch.zeros(1, dtype=torch.long), inner, torch.tensor([rows])]).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    if case["kind"] == "clip":
        sizes = _sizes(case)
        n = sum(sizes)
        grads = torch.empty(n, dtype=getattr(torch, case["dtype"]), device="cuda").normal_(0.0, case["std"], generator=gen)
        out = torch.empty(n, dtype=getattr(torch, case["out"]), device="cuda")
        state = {"case": case, "grads": grads, "out": out, "norm": torch.empty(1, dtype=torch.float32, device="cuda"),
                 "workspace": torch.empty(65536, dtype=torch.uint8, device="cuda")}
        if own:                                                    # the list of tensors that a training program keeps
            import paper_2605_05802_amd as sr
            state["list"] = sr.tensor_list(grads.split(sizes), out.split(sizes))
        return state
    rows, vocab = case["rows"], case["vocab"]
    dtype = getattr(torch, case["dtype"])
    logits = torch.empty(rows, vocab + case["pad"], dtype=dtype, device="cuda")[:, :vocab]
    logits.normal_(0.0, 2.5, generator=gen)
    targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    at = targets.long()[:, None]
    likely = math.log(vocab) + 1.0 + 2.0 * torch.randn(rows, 1, generator=gen, device="cuda")       # sampled tokens are likely ones
    logits.scatter_(1, at, likely.to(dtype))
    logprob = torch.empty(rows, device="cuda")
    for r in range(0, rows, 512):
        x = logits[r:r + 512].float()
        logprob[r:r + 512] = x.gather(1, at[r:r + 512])[:, 0] - torch.logsumexp(x, 1)
    normal = lambda n, s: s * torch.randn(n, generator=gen, device="cuda")
    n_seq = case["seqs"] if case["kind"] == "policy" else 2 * case["pairs"]
    state = {"case": case, "logits": logits, "targets": targets, "seq_start": _cuts(rows, n_seq, host).cuda(),
             "mask": (torch.rand(rows, generator=gen, device="cuda") >= case["masked"]).to(torch.uint8) if case["masked"] else None,
             "ref_logprob": logprob + normal(rows, 0.3), "token_logprob": torch.empty(rows, device="cuda"),
             "stats": torch.empty(4, device="cuda"), "grad": torch.empty(rows, vocab, dtype=dtype, device="cuda") if case.get("grad", True) else None,
             "workspace": torch.empty(65536 + 64 * rows + 32 * n_seq, dtype=torch.uint8, device="cuda")}
    if case["kind"] == "policy":
        ratio = normal(rows, 0.15)                                 # logarithms, none at an end of the clipping range itself
        for end in (math.log(1 - case["clip_low"]), math.log(1 + case["clip_high"])):
            ratio = torch.where((ratio - end).abs() < 1e-3, ratio + 4e-3, ratio)
        state["old_logprob"] = logprob - ratio
        if not case["kl"]:
            state["ref_logprob"] = None
        adv = normal(n_seq, 1.0)
        state["advantages"] = torch.where(torch.rand(n_seq, generator=gen, device="cuda") < 0.2, torch.zeros_like(adv), adv)
    else:
        state["log_ratio"] = torch.empty(n_seq, device="cuda")
    return state


def run(state):
    case = state["case"]
    if case["kind"] == "clip":
        return _run_clip(state, case)
    if case["kind"] == "policy":
        return _run_policy(state, case)
    return _run_pairs(state, case)


def _outputs(state, names):
    return {k: state[k] for k in names if state[k] is not None}


def _run_clip(state, case):
    if own:
        import paper_2605_05802_amd as sr
        sr.sr_clip_grad_norm(state["list"], case["max_norm"], state["norm"], state["workspace"], scale=case["scale"])
        return _outputs(state, ("norm", "out"))
    x = state["grads"].float() * case["scale"]
    norm = (x * x).sum().sqrt()
    return {"norm": norm.reshape(1), "out": (x * torch.clamp(case["max_norm"] / norm, max=1.0)).to(state["out"].dtype)}


def _softmax_rows(state):
    """(exponentials, their sums, log-probability of the target) per row, in 32 bits."""
    x = state["logits"].float()
    largest = x.max(1, keepdim=True).values
    chosen = x.gather(1, state["targets"].long()[:, None]) - largest
    e = torch.exp(x - largest)
    total = e.sum(1, keepdim=True)
    return e, total, (chosen - torch.log(total))[:, 0]


def _members(state):
    """[sequences, rows]: whether a row counts for a sequence."""
    row = torch.arange(state["logits"].shape[0], device="cuda")
    start = state["seq_start"]
    inside = (row >= start[:-1, None]) & (row < start[1:, None])
    return inside if state["mask"] is None else inside & (state["mask"] != 0)


def _logit_grad(state, e, total, slope, counts):
    """slope * (onehot - softmax) per row, rounded once."""
    g = e * (-slope / total[:, 0])[:, None]
    g.scatter_add_(1, state["targets"].long()[:, None], slope[:, None])
    return torch.where(counts[:, None], g, torch.zeros_like(g)).to(state["logits"].dtype)


def _run_policy(state, case):
    if own:
        import paper_2605_05802_amd as sr
        sr.sr_policy_loss(state["logits"], state["targets"], state["seq_start"], state["old_logprob"], state["advantages"], state["stats"],
                          state["workspace"], mask=state["mask"], ref_logprob=state["ref_logprob"], grad=state["grad"],
                          token_logprob=state["token_logprob"], clip_low=case["clip_low"], clip_high=case["clip_high"], kl_coef=case["kl"],
                          reduce=case["reduce"], grad_scale=case["grad_scale"])
        return _outputs(state, ("stats", "token_logprob", "grad"))
    e, total, logprob = _softmax_rows(state)
    member = _members(state)
    counts = member.any(0)
    tokens = member.sum(1).float()                                 # of every sequence
    some = (tokens > 0).float().sum()
    per_seq = {"tokens": (1.0 / tokens.sum()).expand_as(tokens), "sequences": 1.0 / (tokens * some), "sums": (1.0 / some).expand_as(tokens)}[case["reduce"]]
    seq = member.float().argmax(0)
    zero = torch.zeros_like(logprob)
    weight = torch.where(counts, per_seq[seq], zero)
    adv = state["advantages"][seq]
    ratio = torch.exp(logprob - state["old_logprob"])
    plain, clipped = ratio * adv, torch.clamp(ratio, 1 - case["clip_low"], 1 + case["clip_high"]) * adv
    active = plain <= clipped
    surrogate = torch.where(active, plain, clipped)
    slope = torch.where(active, -plain, zero)
    kl = zero
    if case["kl"]:
        d = state["ref_logprob"] - logprob
        kl = torch.exp(d) - d - 1
        slope = slope + case["kl"] * (1 - torch.exp(d))
    mean = lambda v: torch.where(counts, weight * v, zero).sum()
    stats = torch.stack([mean(case["kl"] * kl - surrogate), mean(surrogate), mean(kl), mean((~active).float())])
    out = {"stats": stats, "token_logprob": torch.where(counts, logprob, zero)}
    if case["grad"]:
        out["grad"] = _logit_grad(state, e, total, weight * slope * case["grad_scale"], counts)
    return out


def _run_pairs(state, case):
    if own:
        import paper_2605_05802_amd as sr
        sr.sr_preference_loss(state["logits"], state["targets"], state["seq_start"], state["stats"], state["workspace"], mask=state["mask"],
                              ref_logprob=state["ref_logprob"], grad=state["grad"], token_logprob=state["token_logprob"],
                              log_ratio=state["log_ratio"], beta=case["beta"], label_smoothing=case["smoothing"], grad_scale=case["grad_scale"])
        return _outputs(state, ("stats", "log_ratio", "token_logprob", "grad"))
    e, total, logprob = _softmax_rows(state)
    member = _members(state)
    counts = member.any(0)
    zero = torch.zeros_like(logprob)
    log_ratio = torch.where(member, (logprob - state["ref_logprob"])[None], zero[None]).sum(1)
    reward = case["beta"] * log_ratio
    margin = reward[0::2] - reward[1::2]
    softplus = lambda v: torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs()))
    s = case["smoothing"]
    loss = (1 - s) * softplus(-margin) + s * softplus(margin)
    stats = torch.stack([loss.mean(), (margin > 0).float().mean(), reward[0::2].mean(), reward[1::2].mean()])
    slope = case["beta"] / case["pairs"] * (s / (1 + torch.exp(-margin)) - (1 - s) / (1 + torch.exp(margin)))
    slope = torch.stack([slope, -slope], 1).reshape(-1)[member.float().argmax(0)]
    return {"stats": stats, "log_ratio": log_ratio, "token_logprob": torch.where(counts, logprob, zero),
            "grad": _logit_grad(state, e, total, torch.where(counts, slope * case["grad_scale"], zero), counts)}


def exact(case, seed):
    """The same outputs in 64 bits, the gradients by differentiating the definitions."""
    state = prepare(case, seed)
    if case["kind"] == "clip":
        if state["grads"].numel() > 3 * MOST_GRADS:
            return None
        x = state["grads"].double() * case["scale"]
        norm = torch.linalg.vector_norm(x)
        return {"norm": norm.reshape(1), "out": x * (case["max_norm"] / norm) if norm > case["max_norm"] else x}
    z = state["logits"].double().requires_grad_(True)
    rows, n_seq = z.shape[0], state["seq_start"].numel() - 1
    logprob = torch.cat([torch.log_softmax(x, 1).gather(1, t.long()[:, None])[:, 0]
                         for x, t in zip(z.split(256), state["targets"].split(256))])
    seq = torch.repeat_interleave(torch.arange(n_seq, device="cuda"), state["seq_start"].diff().long())
    keep = torch.ones(rows, dtype=torch.float64, device="cuda") if state["mask"] is None else state["mask"].double()
    by_seq = lambda v: torch.zeros(n_seq, dtype=torch.float64, device="cuda").index_add(0, seq, v * keep)
    if case["kind"] == "policy":
        ratio = torch.exp(logprob - state["old_logprob"].double())
        adv = state["advantages"].double()[seq]
        clipped = ratio.clamp(1 - case["clip_low"], 1 + case["clip_high"])
        surrogate = torch.minimum(ratio * adv, clipped * adv)
        d = state["ref_logprob"].double() - logprob if case["kl"] else torch.zeros_like(logprob)
        kl = torch.expm1(d) - d
        length = by_seq(torch.ones_like(keep))
        used = (length > 0).sum()

        def mean(v):
            s = by_seq(v)
            if case["reduce"] == "tokens":
                return s.sum() / length.sum()
            return (s / length.clamp(min=1)).sum() / used if case["reduce"] == "sequences" else s.sum() / used

        loss = mean(case["kl"] * kl - surrogate)
        stats = torch.stack([loss, mean(surrogate), mean(kl), mean((ratio * adv > clipped * adv).double())])
        out = {"stats": stats.detach(), "token_logprob": (logprob * keep).detach()}
    else:
        log_ratio = by_seq(logprob - state["ref_logprob"].double())
        reward = case["beta"] * log_ratio
        margin = reward[0::2] - reward[1::2]
        s = case["smoothing"]
        loss = -((1 - s) * torch.nn.functional.logsigmoid(margin) + s * torch.nn.functional.logsigmoid(-margin)).mean()
        stats = torch.stack([loss, (margin > 0).double().mean(), reward[0::2].mean(), reward[1::2].mean()])
        out = {"stats": stats.detach(), "log_ratio": log_ratio.detach(), "token_logprob": (logprob * keep).detach()}
    if case.get("grad", True):
        (g,) = torch.autograd.grad(loss * case["grad_scale"], z)
        out["grad"] = g
    return out
