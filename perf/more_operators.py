"""What surrounds the matrix products of the policy that is trained, as timed and compared cases: embedding, residual and norm, dropout.

Kinds of case (one entry point each):
  embed       sr_embed: rows of the token table, scaled, for a list of tokens.
  embed_grad  sr_embed_grad: the gradient of that table, the rows of equal tokens added up.
  norm        sr_add_norm: residual + branch (dropped out or not), root-mean-square norm of the sum; output of the branch's type or
              in 8 bits with scales.
  norm_grad   sr_add_norm_grad: the gradients of residual, branch and gain.
  dropout     sr_dropout: a counter-based mask on rows, alone or on the way into a residual.

Sizes: vocabularies and hidden sizes of the benchmark configuration (152064, 3584, FFN 18944) and of the small test
configuration (1024, 256, FFN 688), their numbers of sequences and prefill rows, and odd sizes between them.
"""
import math

import numpy as np
import torch

own = False

F32, BF16, F16, E4M3, E5M2 = "float32", "bfloat16", "float16", "float8_e4m3fn", "float8_e5m2"
BYTES = {F32: 4, BF16: 2, F16: 2, E4M3: 1, E5M2: 1}
LARGEST = {E4M3: 448.0, E5M2: 57344.0}
TABLE = 152064 * 3584              # elements of the largest table
ROWS = 65536 * 3584                # elements of the largest batch of rows
MOST_BYTES = 1119e6                # of the largest listed case
EPS = 1e-6


def _embed(name, tokens, vocab, width, dtype, out, scale=1.0, pad=0, outside=0.0):
    return {"name": name, "kind": "embed", "tokens": tokens, "vocab": vocab, "width": width, "dtype": dtype, "out": out, "scale": scale,
            "pad": pad, "outside": outside}


def _embed_grad(name, tokens, vocab, width, dtype, out, spread, scale=1.0, hot=0.0, outside=0.0):
    return {"name": name, "kind": "embed_grad", "tokens": tokens, "vocab": vocab, "width": width, "dtype": dtype, "out": out,
            "spread": spread, "scale": scale, "hot": hot, "outside": outside}


def _norm(name, rows, width, dtype, residual, out, p=0.0, block=0, pad=0):
    return {"name": name, "kind": "norm", "rows": rows, "width": width, "dtype": dtype, "residual": residual, "out": out, "p": p,
            "block": block, "pad": pad}


def _norm_grad(name, rows, width, dtype, residual, p=0.0, pad=0):
    return {"name": name, "kind": "norm_grad", "rows": rows, "width": width, "dtype": dtype, "residual": residual, "p": p, "pad": pad}


def _dropout(name, rows, width, dtype, p, residual="", pad=0):
    return {"name": name, "kind": "dropout", "rows": rows, "width": width, "dtype": dtype, "p": p, "residual": residual, "pad": pad}


def listed():
    return [
        # one token of each of the benchmark's 128 sequences, into the single-precision residual
        _embed("embed-step", 128, 152064, 3584, BF16, F32),
        # 128 trajectories of 512 tokens of a training batch, a twentieth of it padding, with the scaling that some decoders have
        _embed("embed-batch", 65536, 152064, 3584, BF16, BF16, scale=math.sqrt(3584), outside=0.05),
        # the small test configuration's gradient: 32 sequences of 8 tokens; launches and host calls count
        _embed_grad("embed-grad-tiny", 256, 1024, 256, F32, F32, "even"),
        # a turn's 4096 action tokens into the whole table of the benchmark's vocabulary: mostly zeros to write
        _embed_grad("embed-grad-wide", 4096, 152064, 3584, BF16, BF16, "natural"),
        # tokens as text has them, half of them one observation marker, at an odd vocabulary and width, summed for the optimizer
        _embed_grad("embed-grad-hot", 49153, 32011, 1031, F16, F32, "natural", scale=1 / 1024, hot=0.5, outside=0.05),
        # a decode step's norm: 128 rows
        _norm("norm-step", 128, 3584, BF16, F32, BF16),
        # a prefill pass of 8192 rows with its output in 8 bits, a scale for each 128 columns
        _norm("norm-8bit", 8192, 3584, BF16, F32, E4M3, block=128),
        # half precision throughout, an odd width in padded rows, dropout on the branch
        _norm("norm-odd-half", 1531, 2047, F16, F16, F16, p=0.1, pad=9),
        # the small test configuration's backward pass
        _norm_grad("norm-grad-tiny", 256, 256, F32, F32),
        # a training batch of 16384 tokens with dropout on the branch, bf16 beside a single-precision residual
        _norm_grad("norm-grad-batch", 16384, 3584, BF16, F32, p=0.1),
        # a ragged batch, added into the residual
        _dropout("dropout-odd", 203, 1031, F16, 0.2, residual=F16, pad=3),
        # the activations between the feed-forward products of a prefill-sized batch
        _dropout("dropout-wide", 8192, 18944, BF16, 0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        case = _draw(rng)
        if work(case)["bytes"] <= MOST_BYTES:
            return case


def _draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_grad", "norm", "norm", "norm_grad", "norm_grad", "dropout"])
    dtype = rng.choice([F32, BF16, BF16, F16])
    wide = rng.choice([dtype, F32])
    pad = rng.choice([0, 0, 8, 3])
    if kind == "dropout":
        width = rng.choice([256, 3584, 18944, 0, 0]) or _log(rng, 1, 20000)
        rows = _log(rng, 1, max(2, min(65536, 8192 * 18944 // width * 2 // BYTES[dtype] // (2 if wide == F32 else 1))))
        return _dropout("", rows, width, dtype, rng.choice([0.05, 0.1, 0.5]), residual=rng.choice(["", wide]), pad=pad)
    if kind in ("embed", "embed_grad"):
        width = rng.choice([256, 3584, 0, 0]) or _log(rng, 16, 8192)
        vocab = rng.choice([1024, 152064, 0, 0]) or _log(rng, 500, 152064)
        vocab = min(vocab, TABLE // width * 2 // BYTES[dtype])
        scale, outside = rng.choice([1.0, math.sqrt(width)]), rng.choice([0.0, 0.05])
        if kind == "embed":
            tokens = _log(rng, 1, max(2, min(65536, ROWS // width * 2 // BYTES[wide])))
            return _embed("", tokens, vocab, width, dtype, wide, scale=scale, pad=pad, outside=outside)
        vocab = min(vocab, TABLE // width * 2 // BYTES[wide])
        tokens = _log(rng, 1, max(2, min(65536, TABLE // 8 // width)))
        return _embed_grad("", tokens, vocab, width, dtype, wide, rng.choice(["even", "natural"]), scale=scale if dtype != F16 else 0.01,
                           hot=rng.choice([0.0, 0.0, 0.5]), outside=outside)
    width = rng.choice([256, 3584, 0, 0]) or _log(rng, 16, 8192)
    p = rng.choice([0.0, 0.0, 0.1])
    if kind == "norm_grad":
        rows = _log(rng, 1, max(2, min(65536, 16384 * 3584 // width * 4 // BYTES[wide] // 2)))
        return _norm_grad("", rows, width, dtype, wide, p=p, pad=pad)
    rows = _log(rng, 1, max(2, min(65536, 16384 * 3584 // width)))
    out = rng.choice([dtype, dtype, E4M3, E5M2])
    return _norm("", rows, width, dtype, wide, out, p=p, block=rng.choice([0, 32, 128]) if out in LARGEST else 0, pad=pad)


def _blocks(case):
    """Scales of a row."""
    return -(-case["width"] // case["block"]) if case["block"] else 1


def work(case):
    b = BYTES[case["dtype"]]
    if case["kind"] == "dropout":
        n, r = case["rows"] * case["width"], BYTES.get(case["residual"], 0)
        return {"bytes": n * (b + (2 * r if r else b)), "flops": 2 * n}
    if case["kind"] == "embed":
        n = case["tokens"] * case["width"]
        # rows of the table that the tokens name, each once
        named = case["vocab"] * -math.expm1(-case["tokens"] * (1 - case["outside"]) / case["vocab"])
        return {"bytes": named * case["width"] * b + n * BYTES[case["out"]] + 4 * case["tokens"], "flops": n}
    if case["kind"] == "embed_grad":
        n, kept = case["tokens"] * case["width"], 1 - case["outside"]
        return {"bytes": n * b * kept + case["vocab"] * case["width"] * BYTES[case["out"]] + 4 * case["tokens"], "flops": 2 * n}
    n, r = case["rows"] * case["width"], BYTES[case["residual"]]
    if case["kind"] == "norm":
        return {"bytes": n * (b + 2 * r + BYTES[case["out"]]) + 4 * case["rows"] * (1 + (_blocks(case) if case["out"] in LARGEST else 0)),
                "flops": 6 * n}
    return {"bytes": n * (b + 3 * r + b) + 4 * case["rows"], "flops": 14 * n}


def _rows(rows, width, pad, dtype, gen, std=1.0):
    """Rows of `width` columns, `pad` unused ones behind each."""
    x = torch.empty(rows, width + pad, dtype=getattr(torch, dtype), device="cuda").normal_(0.0, std, generator=gen)
    return x[:, :width]


def _tokens(case, gen):
    n, vocab = case["tokens"], case["vocab"]
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    if case.get("spread") == "natural":                            # the r-th commonest token has a share of about 1 / r
        t = torch.randperm(vocab, generator=gen, device="cuda")[(torch.exp(u * math.log(vocab + 1)).long() - 1).clamp(0, vocab - 1)]
    else:
        t = (u * vocab).long().clamp(max=vocab - 1)
    share = torch.rand(n, generator=gen, device="cuda")
    t = torch.where(share < case.get("hot", 0.0), vocab // 2, t)
    return torch.where(torch.rand(n, generator=gen, device="cuda") < case["outside"], -1, t).int()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": case}
    new = lambda rows, width, dtype: torch.empty(rows, width, dtype=getattr(torch, dtype), device="cuda")
    width, dtype = case["width"], case["dtype"]
    if case["kind"] in ("embed", "embed_grad"):
        state["tokens"] = _tokens(case, gen)
        if case["kind"] == "embed":
            state["table"] = _rows(case["vocab"], width, 0, dtype, gen, 0.02)
            state["out"] = new(case["tokens"], width + case["pad"], case["out"])[:, :width]
        else:
            state["d_out"] = _rows(case["tokens"], width, 0, dtype, gen, 0.01 / case["scale"])
            state["d_table"] = new(case["vocab"], width, case["out"])
            state["workspace"] = torch.empty(_grad_workspace(case["tokens"], width), dtype=torch.uint8, device="cuda")
        return state
    rows = case["rows"]
    # which mask: a number of the program's, and a count of its steps that lies on the device
    state["seed"], state["mask"] = seed * 0x10001 + 7, seed % 13
    state["step"] = torch.full((1,), seed % 101, dtype=torch.int64, device="cuda")
    if case["kind"] == "dropout":
        state["x"] = _rows(rows, width, case["pad"], dtype, gen)
        state["base"] = _rows(rows, width, case["pad"], case["residual"], gen) if case["residual"] else None
        state["out"] = new(rows, width, case["residual"] or dtype)
        return state
    state["gain"] = (1.0 + 0.1 * torch.randn(width, generator=gen, device="cuda")).to(getattr(torch, dtype))
    if case["kind"] == "norm":
        state["x"] = _rows(rows, width, case["pad"], dtype, gen)
        state["base"] = _rows(rows, width, case["pad"], case["residual"], gen, 2.0)
        state["total"], state["out"] = new(rows, width, case["residual"]), new(rows, width, case["out"])
        state["rstd"] = torch.empty(rows, device="cuda")
        state["scales"] = torch.empty(rows, _blocks(case), device="cuda") if case["out"] in LARGEST else None
        return state
    state["total"] = _rows(rows, width, case["pad"], case["residual"], gen, 2.0)
    state["rstd"] = torch.rsqrt(state["total"].double().square().mean(1) + EPS).float()
    state["d_out"] = _rows(rows, width, case["pad"], dtype, gen, 0.01)
    state["d_total"] = _rows(rows, width, case["pad"], case["residual"], gen, 0.01)
    state["d_residual"], state["d_x"] = new(rows, width, case["residual"]), new(rows, width, dtype)
    state["d_gain"] = torch.empty(width, device="cuda")
    state["workspace"] = torch.empty(_norm_workspace(rows, width), dtype=torch.uint8, device="cuda")
    return state


def _grad_workspace(tokens, width):
    return (1 << 20) + 64 * tokens + (tokens // 8 + 64) * 4 * width


def _norm_workspace(rows, width):
    return min(rows, 2048) * width * 4 + 65536


def run(state):
    return RUN[state["case"]["kind"]](state, state["case"])


def _outputs(state, names):
    return {k: state[k] for k in names if state[k] is not None}


def _signed(x):
    return x - (1 << 64) if x >= 1 << 63 else x


def _mix(z):
    """SplitMix64's finishing function on 64-bit patterns held as signed integers."""
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(0x94D049BB133111EB)
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _keep(state, case):
    """What multiplies each element: 0, or 1 over the share that is kept."""
    rows, width = case["rows"], case["width"]
    golden = _signed(0x9E3779B97F4A7C15)
    dropped = int(case["p"] * 65536 + 0.5)
    key = _mix(_mix(torch.full((1,), state["seed"], dtype=torch.int64, device="cuda") + golden)
               ^ ((state["step"] + state["mask"]) * _signed(0xD1342543DE82EF95) + 1))
    each = -(-width // 4)
    at = torch.arange(rows, device="cuda")[:, None] * each + torch.arange(each, device="cuda") + 1
    bits = _mix(key + at * golden)
    u = torch.stack([(bits >> s) & 0xffff for s in (0, 16, 32, 48)], 2).reshape(rows, 4 * each)[:, :width]
    return (u >= dropped).float() * (65536.0 / (65536 - dropped))


def _run_embed(state, case):
    if own:
        import paper_2605_05802_amd as sr
        sr.sr_embed(state["table"], state["tokens"], state["out"], scale=case["scale"])
        return _outputs(state, ("out",))
    t = state["tokens"].long()
    inside = ((t >= 0) & (t < case["vocab"])).float()
    return {"out": (state["table"][t.clamp(0, case["vocab"] - 1)].float() * (inside * case["scale"])[:, None]).to(state["out"].dtype)}


def _run_embed_grad(state, case):
    if own:
        import paper_2605_05802_amd as sr
        sr.sr_embed_grad(state["d_out"], state["tokens"], state["d_table"], state["workspace"], scale=case["scale"])
        return _outputs(state, ("d_table",))
    t = state["tokens"].long()
    inside = ((t >= 0) & (t < case["vocab"])).float()
    table = torch.zeros(case["vocab"], case["width"], device="cuda")
    table.index_add_(0, t.clamp(0, case["vocab"] - 1), state["d_out"].float() * inside[:, None])
    return {"d_table": (table * case["scale"]).to(state["d_table"].dtype)}


def _dropout_options(sr, state, case):
    return sr.Dropout(case["p"], state["seed"], mask=state["mask"], step=state["step"]) if case["p"] else None


def _run_norm(state, case):
    if own:
        import paper_2605_05802_amd as sr
        sr.sr_add_norm(state["base"], state["gain"], state["out"], x=state["x"], total=state["total"], rstd=state["rstd"],
                       scales=state["scales"], scale_block=case["block"], dropout=_dropout_options(sr, state, case), eps=EPS)
        return _outputs(state, ("total", "out", "rstd", "scales"))
    x = state["x"].float()
    if case["p"]:
        x = x * _keep(state, case)
    total = (state["base"].float() + x).to(state["total"].dtype)
    h = total.float()
    rstd = 1.0 / torch.sqrt((h * h).mean(1) + EPS)
    y = h * rstd[:, None] * state["gain"].float()
    out = {"total": total, "rstd": rstd}
    if case["out"] not in LARGEST:
        return out | {"out": y.to(state["out"].dtype)}
    block, blocks = case["block"] or case["width"], _blocks(case)
    y = torch.cat([y, y.new_zeros(y.shape[0], block * blocks - case["width"])], 1).view(-1, blocks, block)
    scales = torch.clamp(y.abs().amax(2) / LARGEST[case["out"]], min=2.0 ** -126)
    codes = (y / scales[:, :, None]).reshape(-1, block * blocks)[:, :case["width"]].to(state["out"].dtype)
    return out | {"out": codes, "scales": scales}


def _run_norm_grad(state, case):
    if own:
        import paper_2605_05802_amd as sr
        sr.sr_add_norm_grad(state["d_out"], state["total"], state["rstd"], state["gain"], state["workspace"], d_total=state["d_total"],
                            d_residual=state["d_residual"], d_x=state["d_x"], d_gain=state["d_gain"],
                            dropout=_dropout_options(sr, state, case))
        return _outputs(state, ("d_residual", "d_x", "d_gain"))
    dy, rstd = state["d_out"].float(), state["rstd"][:, None]
    normed = state["total"].float() * rstd
    g = dy * state["gain"].float()
    dh = rstd * (g - normed * (g * normed).mean(1, keepdim=True)) + state["d_total"].float()
    dx = dh * _keep(state, case) if case["p"] else dh
    return {"d_residual": dh.to(state["d_residual"].dtype), "d_x": dx.to(state["d_x"].dtype), "d_gain": (dy * normed).sum(0)}


def _run_dropout(state, case):
    if own:
        import paper_2605_05802_amd as sr
        sr.sr_dropout(state["x"], state["out"], sr.Dropout(case["p"], state["seed"], mask=state["mask"], step=state["step"]),
                      residual=state["base"])
        return _outputs(state, ("out",))
    y = state["x"].float() * _keep(state, case)
    if state["base"] is not None:
        y = y + state["base"].float()
    return {"out": y.to(state["out"].dtype)}


RUN = {"embed": _run_embed, "embed_grad": _run_embed_grad, "norm": _run_norm, "norm_grad": _run_norm_grad, "dropout": _run_dropout}


def _exact_keep(state, case):
    """The mask's factors in 64 bits, from unsigned integers on the host."""
    u64 = np.uint64
    golden = 0x9E3779B97F4A7C15
    whole = (1 << 64) - 1

    def finish(z):
        z = (z ^ (z >> u64(30))) * u64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> u64(27))) * u64(0x94D049BB133111EB)
        return z ^ (z >> u64(31))

    rows, width, each = case["rows"], case["width"], (case["width"] + 3) // 4
    first = finish(np.array([(state["seed"] + golden) & whole], dtype=u64))
    which = ((state["mask"] + int(state["step"].item())) * 0xD1342543DE82EF95 + 1) & whole
    key = finish(first ^ u64(which))
    bits = finish(key + (np.arange(rows * each, dtype=u64) + u64(1)) * u64(golden))
    parts = bits.astype("<u8").view("<u2").reshape(rows, 4 * each)[:, :width]
    dropped = math.floor(case["p"] * 65536 + 0.5)
    kept = torch.from_numpy(parts >= dropped).cuda()
    return kept.double() / (1.0 - dropped / 65536)


def exact(case, seed):
    """The same outputs in 64 bits, gradients by differentiating the definitions; codes of 8 bits have no such value."""
    state = prepare(case, seed)
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    if case["kind"] in ("embed", "embed_grad"):
        t = state["tokens"].long()
        valid = (t >= 0) & (t < case["vocab"])
        if case["kind"] == "embed":
            out = torch.zeros(case["tokens"], case["width"], dtype=torch.float64, device="cuda")
            out[valid] = state["table"].index_select(0, t[valid]).double() * case["scale"]
            return {"out": out}
        # sums over the tokens' places in ascending order of the tokens
        order = torch.sort(t[valid], stable=True)
        found, count = torch.unique_consecutive(order.values, return_counts=True)
        ends = count.cumsum(0)
        out = torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device="cuda")
        d = state["d_out"][valid][order.indices]
        for c in range(0, case["width"], 256):
            run = d[:, c:c + 256].double().cumsum(0)
            upto = run[ends - 1]
            out[found, c:c + 256] = torch.cat([upto[:1], upto[1:] - upto[:-1]]) if len(found) else upto
        return {"d_table": out.mul_(case["scale"])}
    keep = _exact_keep(state, case) if case["p"] else None
    if case["kind"] == "dropout":
        y = state["x"].double() * keep
        return {"out": y if state["base"] is None else state["base"].double() + y}
    gain = state["gain"].double()
    if case["kind"] == "norm":
        x = state["x"].double()
        total = state["base"].double() + (x if keep is None else x * keep)
        h = total.to(state["total"].dtype).double()                # the norm is that of the sum as it is stored
        rstd = (h.square().sum(1) / case["width"] + EPS) ** -0.5
        y = torch.einsum("ij,i,j->ij", h, rstd, gain)
        if case["out"] not in LARGEST:
            return {"total": total, "rstd": rstd, "out": y}
        block = case["block"] or case["width"]
        scales = torch.stack([torch.linalg.vector_norm(part, math.inf, dim=1) for part in y.split(block, 1)], 1) / LARGEST[case["out"]]
        return {"total": total, "rstd": rstd, "out": None, "scales": scales.clamp(min=2.0 ** -126)}
    h = state["total"].double().requires_grad_(True)
    g = gain.requires_grad_(True)
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * g
    d_total, d_gain = torch.autograd.grad((y * state["d_out"].double()).sum() + (h * state["d_total"].double()).sum(), (h, g))
    return {"d_residual": d_total, "d_x": d_total if keep is None else torch.where(keep > 0, d_total * keep, zero), "d_gain": d_gain}
