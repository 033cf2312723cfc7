"""sr_policy_loss and sr_preference_loss against a plain evaluation in 64 bits.

Tolerances.  u = 2^-24.  The sum of exponentials of a row is a chain of at most vocab / 64 + 64 additions (a wavefront a row is
the shortest one the library may take), every exponential's argument carries two roundings relative to D = the largest
difference from the maximum that still counts (below -40 a term is 4e-18), the instruction itself and its scaling a few more:
    rel(s) <= u (vocab / 64 + 64 + 3 * 40 + 8) = S.
l = (x_y - m) - log s: abs(l) <= S + 2 u (|x_y - m| + |log s| + 1) = E.  From there to first order
    r = exp(l - old): rel 2 E + 8 u;  exp(d) the same;  slope: weight * scale * (r |A| + kl_coef (exp(d) + 1)) (2 E + 8 u),
    gradient: |onehot - p| * that + |slope| p (S + 3 u (D + 4)) + 4 u |slope| + half a unit in the last place of its type.
Sums over tokens are in double over single-precision terms."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2605_05802_amd as sr

U = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24}
LOW, HIGH = 0.2, 0.28


def make(rows, n_seq, vocab, dtype, seed, *, pad=0, shift=0, masked=0.0, lead=0, tail=0, cuts=None):
    """Inputs as a dict of device tensors.  pad: unused columns; shift: elements in front of the first row; lead, tail: rows
    outside every sequence; cuts: sequence starts."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    host = np.random.default_rng(seed)
    ld = vocab + pad
    buf = torch.full((rows * ld + shift,), float("nan"), dtype=dtype, device="cuda")
    logits = buf[shift:].view(rows, ld)[:, :vocab]
    logits.copy_(torch.randn(rows, vocab, generator=g, device="cuda") * 2.5)
    targets = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    at = targets.long()[:, None]
    logits.scatter_(1, at, (math.log(vocab) + 1 + 2 * torch.randn(rows, 1, generator=g, device="cuda")).to(dtype))
    if cuts is None:
        cuts = np.sort(host.integers(lead, rows - tail + 1, n_seq - 1))
        cuts = [lead, *cuts.tolist(), rows - tail]
    logprob = torch.log_softmax(logits.double(), 1).gather(1, at)[:, 0]
    ratio = 0.2 * torch.randn(rows, generator=g, device="cuda", dtype=torch.float64)
    for end in (math.log(1 - LOW), math.log(1 + HIGH)):            # none so near an end that rounding decides
        ratio = torch.where((ratio - end).abs() < 1e-3, ratio + 4e-3, ratio)
    adv = torch.randn(n_seq, generator=g, device="cuda")
    adv[::5] = 0.0
    return {"logits": logits, "targets": targets, "seq_start": torch.tensor(cuts, dtype=torch.int32, device="cuda"),
            "mask": (torch.rand(rows, generator=g, device="cuda") >= masked).to(torch.uint8) if masked else None,
            "old_logprob": (logprob - ratio).float(), "advantages": adv,
            "ref_logprob": (logprob + 0.3 * torch.randn(rows, generator=g, device="cuda", dtype=torch.float64)).float()}


def counting(x):
    """(counts [rows], sequence of every row)."""
    rows = x["logits"].shape[0]
    start = x["seq_start"].long()
    row = torch.arange(rows, device="cuda")
    inside = (row[None] >= start[:-1, None]) & (row[None] < start[1:, None])
    counts = inside.any(0)
    if x["mask"] is not None:
        counts &= x["mask"] != 0
    return counts, inside.float().argmax(0)


def row_terms(x, counts):
    z = torch.where(counts[:, None], x["logits"].double(), torch.zeros((), dtype=torch.float64, device="cuda"))
    m = z.max(1).values
    s = torch.exp(z - m[:, None]).sum(1)
    at = x["targets"].long()[:, None]
    off = z.gather(1, at)[:, 0] - m
    p = torch.exp(z - m[:, None]) / s[:, None]
    hot = torch.zeros_like(p).scatter_(1, at, 1.0)
    vocab = z.shape[1]
    S = U * (vocab / 64 + 64 + 128)
    E = S + 2 * U * (off.abs() + torch.log(s) + 1)
    return off - torch.log(s), p, hot, S, E


def policy_reference(x, reduce, kl_coef, use_ref, scale=1.0):
    counts, seq = counting(x)
    l, p, hot, S, E = row_terms(x, counts)
    n_seq = x["advantages"].numel()
    length = torch.zeros(n_seq, dtype=torch.float64, device="cuda").index_add_(0, seq, counts.double())
    used = (length > 0).sum().clamp(min=1)
    w = {"tokens": (1 / length.sum().clamp(min=1)).expand(n_seq), "sequences": 1 / (used * length.clamp(min=1)),
         "sums": (1.0 / used).double().expand(n_seq)}[reduce][seq]
    w = torch.where(counts, w, 0.0)
    A = x["advantages"].double()[seq]
    r = torch.exp(l - x["old_logprob"].double())
    lo, hi = float(np.float32(1) - np.float32(LOW)), float(np.float32(1) + np.float32(HIGH))
    plain, clipped = r * A, r.clamp(lo, hi) * A
    out = plain > clipped
    sur = torch.minimum(plain, clipped)
    d = x["ref_logprob"].double() - l if use_ref else torch.zeros_like(l)
    kl = torch.expm1(d) - d
    slope = torch.where(out, 0.0, -plain) - kl_coef * torch.expm1(d)
    mean = lambda v: torch.where(counts, w * v, 0.0).sum()
    stats = torch.stack([mean(kl_coef * kl - sur), mean(sur), mean(kl), mean(out.double())])
    e = 2 * E + 8 * U
    slope_tol = (plain.abs() + kl_coef * (torch.exp(d) + 1)) * e
    stat_tol = mean(kl_coef * ((torch.exp(d) + 1) * e)) + mean(plain.abs() * e) + mean((torch.exp(d) + 1) * e) + 4 * U * stats.abs().max()
    return {"stats": stats, "stat_tol": stat_tol, "logprob": torch.where(counts, l, 0.0), "E": E, "slope": torch.where(counts, w * slope * scale, 0.0),
            "slope_tol": torch.where(counts, w * slope_tol * scale, 0.0), "p": p, "hot": hot, "S": S, "counts": counts}


def check_grad(grad, ref):
    slope, p, hot = ref["slope"][:, None], ref["p"], ref["hot"]
    want = torch.where(ref["counts"][:, None], slope * (hot - p), 0.0)
    tol = (hot - p).abs() * ref["slope_tol"][:, None] + slope.abs() * p * (ref["S"] + 3 * U * 44) + 4 * U * slope.abs() * hot
    tol = tol + ROUND[grad.dtype] * (want.abs() + tol) + SMALLEST[grad.dtype]
    off = (grad.double() - want).abs()
    assert bool((off <= tol).all()), f"gradient: worst excess {(off - tol).max().item():.3e}, at {int((off - tol).argmax())}"
    assert bool((grad[~ref["counts"]] == 0).all())


def run_policy(x, reduce, kl_coef, *, grad=True, in_place=False, use_ref=True, scale=1.0, stream=None):
    rows, vocab = x["logits"].shape
    n_seq = x["advantages"].numel()
    if in_place:
        g = x["logits"]
    else:
        g = torch.full((rows, vocab), 7.0, dtype=x["logits"].dtype, device="cuda") if grad else None
    stats = torch.full((4,), 7.0, device="cuda")
    lp = torch.full((rows,), 7.0, device="cuda")
    ws = torch.full((sr.token_loss_workspace(rows, n_seq),), 255, dtype=torch.uint8, device="cuda")
    sr.sr_policy_loss(x["logits"], x["targets"], x["seq_start"], x["old_logprob"], x["advantages"], stats, ws, mask=x["mask"],
                      ref_logprob=x["ref_logprob"] if use_ref else None, grad=g, token_logprob=lp, clip_low=LOW, clip_high=HIGH,
                      kl_coef=kl_coef, reduce=reduce, grad_scale=scale, stream=stream)
    return stats, lp, g


def check_policy(x, reduce, kl_coef, **kw):
    ref = policy_reference(x, reduce, kl_coef, kw.get("use_ref", True), kw.get("scale", 1.0))
    stats, lp, g = run_policy(x, reduce, kl_coef, **kw)
    assert bool(((lp.double() - ref["logprob"]).abs() <= ref["E"]).all())
    assert bool((lp[~ref["counts"]] == 0).all())
    assert bool(((stats.double() - ref["stats"]).abs() <= ref["stat_tol"]).all()), (stats, ref["stats"], ref["stat_tol"])
    if g is not None:
        check_grad(g, ref)
    return stats, lp, g


TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_seq,vocab,pad,shift", [
    (1, 1, 1, 0, 0), (1, 1, 2, 0, 0), (3, 2, 7, 0, 1), (5, 5, 8, 8, 0), (17, 3, 9, 3, 0), (64, 8, 63, 1, 1), (9, 4, 255, 0, 3),
    (256, 32, 1000, 24, 0), (300, 7, 1024, 0, 0), (33, 9, 4097, 0, 1), (40, 6, 5003, 5, 2), (70, 3, 20011, 0, 0), (1, 1, 152064, 0, 0),
    (3, 2, 152064, 0, 0), (300, 11, 9000, 0, 0), (5000, 100, 130, 0, 0), (700, 20, 33333, 0, 1), (258, 4, 152064, 0, 0)])
def test_policy_loss_over_sizes(dtype, rows, n_seq, vocab, pad, shift):
    x = make(rows, n_seq, vocab, dtype, rows + vocab, pad=pad, shift=shift)
    check_policy(x, "sequences", 0.04, scale=4096.0 if dtype == torch.float16 else 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("reduce", ["tokens", "sequences", "sums"])
@pytest.mark.parametrize("kl,use_ref", [(0.0, False), (0.0, True), (0.3, True)])
@pytest.mark.parametrize("masked", [0.0, 0.4])
@pytest.mark.parametrize("rows,vocab", [(91, 777), (301, 12001)])
def test_policy_loss_over_means_and_masks(reduce, kl, use_ref, masked, rows, vocab):
    check_policy(make(rows, 13, vocab, torch.bfloat16, 3, masked=masked, lead=4, tail=9), reduce, kl, use_ref=use_ref)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(12, 515), (12, 30001), (300, 12001), (260, 152064)])
def test_gradient_in_place_and_the_loss_alone(dtype, rows, vocab):
    x = make(rows, 4, vocab, dtype, 8, pad=3, masked=0.3)
    stats, lp, g = check_policy(x, "tokens", 0.04)
    s1, l1, none = run_policy(x, "tokens", 0.04, grad=False)
    assert none is None and torch.equal(lp, l1) and torch.equal(s1, stats)
    s2, l2, g2 = run_policy(x, "tokens", 0.04, in_place=True)
    assert torch.equal(lp, l2) and torch.equal(s2, stats) and torch.equal(g2, g)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab", [(30, 999), (30, 40001), (290, 20003)])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_the_mask_leaves_out_are_not_read(rows, vocab, dtype):
    """NaN and infinity in rows that do not count, in their old and reference values, and behind every row's end."""
    x = make(rows, 6, vocab, dtype, 5, pad=4, masked=0.5, lead=3, tail=2, cuts=[3, 3, 9, 9, 20, 20, rows - 2])
    counts, _ = counting(x)
    x["mask"][9:20] = 0                                            # a sequence that the mask leaves empty
    counts, _ = counting(x)
    for i, bad in enumerate((float("nan"), float("inf"), float("-inf"))):
        x["logits"][(~counts).nonzero()[i::3, 0]] = bad
        x["old_logprob"][(~counts).nonzero()[i::3, 0]] = bad
        x["ref_logprob"][(~counts).nonzero()[i::3, 0]] = bad
    x["targets"][~counts] = 1 << 30
    y = dict(x, targets=torch.where(counts, x["targets"], 0), ref_logprob=torch.where(counts, x["ref_logprob"], 0.0),
             old_logprob=torch.where(counts, x["old_logprob"], 0.0))
    for reduce in ("tokens", "sequences", "sums"):
        ref = policy_reference(y, reduce, 0.04, True)
        stats, lp, g = run_policy(x, reduce, 0.04)
        assert bool(((lp.double() - ref["logprob"]).abs() <= ref["E"]).all())
        assert bool(((stats.double() - ref["stats"]).abs() <= ref["stat_tol"]).all())
        check_grad(g, ref)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(11, 700), (11, 33003), (280, 16001)])
def test_masked_vocabulary_entries(dtype, rows, vocab):
    """-infinity and the type's lowest value among the logits, rows of nothing but the lowest value, and rows of one entry."""
    x = make(rows, 3, vocab, dtype, 2)
    g = torch.Generator(device="cuda").manual_seed(0)
    gone = torch.rand(rows, vocab, generator=g, device="cuda") < 0.5
    gone.scatter_(1, x["targets"].long()[:, None], False)
    low = torch.finfo(dtype).min
    x["logits"][0:4] = torch.where(gone[0:4], torch.tensor(float("-inf"), dtype=dtype, device="cuda"), x["logits"][0:4])
    x["logits"][4:8] = torch.where(gone[4:8], torch.tensor(low, dtype=dtype, device="cuda"), x["logits"][4:8])
    x["logits"][8] = low
    x["logits"][9] = float("-inf")
    x["logits"][9, int(x["targets"][9])] = 0.5
    x["old_logprob"][8] = x["ref_logprob"][8] = -math.log(vocab)
    x["old_logprob"][9] = x["ref_logprob"][9] = 0.0
    fresh = torch.log_softmax(x["logits"][:8].double(), 1).gather(1, x["targets"][:8].long()[:, None])[:, 0]
    x["old_logprob"][:8] = (fresh + 0.05).float()
    x["ref_logprob"][:8] = (fresh - 0.1).float()
    stats, lp, _ = check_policy(x, "tokens", 0.04)
    assert bool(torch.isfinite(lp).all()) and bool(torch.isfinite(stats).all())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab", [(9, 800), (9, 33003), (270, 16001)])
def test_rows_without_a_distribution_say_nan(rows, vocab):
    """NaN, +infinity, nothing but -infinity, a target outside the vocabulary: NaN in that row and in the loss, nowhere else."""
    x = make(rows, 2, vocab, torch.float32, 4)
    x["logits"][1, vocab // 2] = float("nan")
    x["logits"][2, vocab - 1] = float("inf")
    x["logits"][3] = float("-inf")
    x["targets"][4], x["targets"][5] = vocab, -1
    stats, lp, g = run_policy(x, "tokens", 0.0, use_ref=False)
    assert bool(torch.isnan(lp[1:6]).all()) and bool(torch.isfinite(lp[6:]).all()) and bool(torch.isfinite(lp[0]))
    assert bool(torch.isnan(stats[0]))
    assert bool(torch.isnan(g[1:6]).any(1).all()) and bool(torch.isfinite(g[6:]).all()) and bool(torch.isfinite(g[0]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab", [(9, 800), (9, 33003), (200, 60001), (9, 152064)])
def test_a_token_that_cannot_occur(rows, vocab):
    """Log-probability -infinity, ratio 0: no gradient without a KL term whatever the advantage, an infinite KL term with one."""
    x = make(rows, 2, vocab, torch.bfloat16, 6)
    x["logits"][2, int(x["targets"][2])] = float("-inf")
    x["advantages"].copy_(torch.tensor([1.5, -0.5], device="cuda"))
    stats, lp, g = run_policy(x, "tokens", 0.0, use_ref=True)
    assert lp[2].item() == float("-inf") and bool(torch.isfinite(lp[3:]).all())
    assert bool((g[2] == 0).all()) and bool(torch.isfinite(g).all())
    assert bool(torch.isfinite(stats[:2]).all()) and stats[2].item() == float("inf")
    stats, _, g = run_policy(x, "tokens", 0.04)
    assert stats[0].item() == float("inf") and bool(torch.isfinite(g[3:]).all()) and bool(torch.isfinite(g[:2]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab,n_seq", [(300, 500, 6), (40, 9000, 2), (5000, 64, 1500), (260, 50001, 4)])
def test_starts_that_make_no_sense_stay_inside_the_buffers(rows, vocab, n_seq):
    """Decreasing, negative and huge sequence starts: unspecified results, nothing else written."""
    x = make(rows, n_seq, vocab, torch.bfloat16, 6, masked=0.3)
    rng = np.random.default_rng(1)
    top = 2 ** 31 - 1
    for starts in ([top] * (n_seq + 1), [-top - 1] * (n_seq + 1), rng.integers(-5, rows + 5, n_seq + 1).tolist(),
                   [rows] + [0] * (n_seq - 1) + [top], [-3] + [top] * (n_seq - 1) + [rows // 2], [top] + [5] * n_seq):
        y = dict(x, seq_start=torch.tensor(starts, dtype=torch.int64, device="cuda").to(torch.int32))
        for run in (lambda: run_policy(y, "sequences", 0.04), lambda: run_policy(y, "sequences", 0.04, grad=False), lambda: run_pairs(y, 0.1, 0.0)):
            before = [x["logits"].clone(), x["targets"].clone(), x["old_logprob"].clone()]
            run()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(before, (x["logits"], x["targets"], x["old_logprob"])))


@pytest.mark.gpu
def test_nothing_counts():
    for rows, vocab in ((5, 50), (5, 20000), (300, 9000)):
        x = make(rows, 2, vocab, torch.bfloat16, 1, masked=0.5)
        x["mask"].zero_()
        stats, lp, g = run_policy(x, "sequences", 0.04)
        assert bool((stats == 0).all()) and bool((lp == 0).all()) and bool((g == 0).all())
    empty = {"logits": torch.empty(0, 10, device="cuda"), "targets": torch.empty(0, dtype=torch.int32, device="cuda"),
             "seq_start": torch.zeros(3, dtype=torch.int32, device="cuda"), "mask": None, "old_logprob": torch.empty(0, device="cuda"),
             "ref_logprob": torch.empty(0, device="cuda"), "advantages": torch.ones(2, device="cuda")}
    stats, _, _ = run_policy(empty, "tokens", 0.04)
    assert bool((stats == 0).all())
    stats = torch.full((4,), 7.0, device="cuda")
    ws = torch.empty(sr.token_loss_workspace(0, 2), dtype=torch.uint8, device="cuda")
    sr.sr_preference_loss(empty["logits"], empty["targets"], empty["seq_start"], stats, ws)
    assert stats[0].item() == pytest.approx(math.log(2), rel=1e-6) and bool((stats[1:] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_that_lie_more_than_2_to_the_31_elements_apart(dtype):
    rows, vocab, ld = 4, 1003, (1 << 30) + 1
    small = make(rows, 2, vocab, dtype, 6)
    stats, lp, g = run_policy(small, "tokens", 0.04)
    far = torch.empty((rows - 1) * ld + vocab, dtype=dtype, device="cuda").as_strided((rows, vocab), (ld, 1))
    far.copy_(small["logits"])
    x = dict(small, logits=far)
    s2, l2, g2 = run_policy(x, "tokens", 0.04, in_place=True)
    assert torch.equal(stats, s2) and torch.equal(lp, l2) and torch.equal(g2, g)


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [200, 20000])
def test_policy_gradient_against_differences(vocab):
    """The loss in 64 bits, differenced along random directions, against the kernel's gradient."""
    x = make(24, 5, vocab, torch.float32, 9, masked=0.2)
    _, _, g = run_policy(x, "sequences", 0.2)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(4):
        v = torch.randn(g.shape, generator=gen, device="cuda", dtype=torch.float64)
        h = 1e-5
        f = [policy_reference(dict(x, logits=x["logits"].double() + s * h * v), "sequences", 0.2, True)["stats"][0].item() for s in (1, -1)]
        want = (f[0] - f[1]) / (2 * h)
        # third derivatives of the loss are O(|slope|): h^2 of them, and 64-bit cancellation of 1e-16 / h
        assert (g.double() * v).sum().item() == pytest.approx(want, rel=1e-4, abs=1e-6)


@pytest.mark.gpu
def test_sums_at_ratio_one_give_the_gradient_of_the_policy_gradient_loss():
    """Section 2.1: L = -(1/N) sum_i A_i log p(tau_i), with the advantages that sr_grpo_loss writes."""
    n_groups, G, vocab, tokens = 3, 4, 500, 6
    n = n_groups * G
    x = make(n * tokens, n, vocab, torch.float32, 12, cuts=[tokens * i for i in range(n + 1)])
    z = x["logits"].double().requires_grad_(True)
    lp = torch.log_softmax(z, 1).gather(1, x["targets"].long()[:, None])[:, 0]
    rewards = torch.tensor(np.random.default_rng(0).integers(0, 2, n), dtype=torch.float32, device="cuda")
    rewards[:G] = 1.0                                              # a group without variance
    adv = torch.empty(n, device="cuda")
    loss = torch.empty(1, dtype=torch.float64, device="cuda")
    seq_lp = lp.detach().view(n, tokens).sum(1).contiguous()
    sr.sr_grpo_loss(seq_lp, rewards, G, 1e-6, adv, torch.empty(n_groups, dtype=torch.float64, device="cuda"), loss)
    x["advantages"], x["old_logprob"] = adv, lp.detach().float()
    _, _, g = run_policy(x, "sums", 0.0, use_ref=False)
    want = torch.autograd.grad(-(adv.double() * lp.view(n, tokens).sum(1)).sum() / n, z)[0]
    assert bool((g[:G * tokens] == 0).all())
    assert float((g.double() - want).abs().max()) <= 1e-5 * float(want.abs().max())


# ---------------------------------------------------------------------------------------------
# preference loss
# ---------------------------------------------------------------------------------------------
def run_pairs(x, beta, smoothing, *, use_ref=True, in_place=False, grad=True, scale=1.0, stream=None):
    rows, vocab = x["logits"].shape
    n_seq = x["seq_start"].numel() - 1
    g = x["logits"] if in_place else torch.full((rows, vocab), 7.0, dtype=x["logits"].dtype, device="cuda") if grad else None
    stats, lr = torch.full((4,), 7.0, device="cuda"), torch.full((n_seq,), 7.0, device="cuda")
    lp = torch.full((rows,), 7.0, device="cuda")
    ws = torch.full((sr.token_loss_workspace(rows, n_seq),), 255, dtype=torch.uint8, device="cuda")
    sr.sr_preference_loss(x["logits"], x["targets"], x["seq_start"], stats, ws, mask=x["mask"], ref_logprob=x["ref_logprob"] if use_ref else None,
                          grad=g, token_logprob=lp, log_ratio=lr, beta=beta, label_smoothing=smoothing, grad_scale=scale, stream=stream)
    return stats, lr, lp, g


def pairs_reference(x, beta, smoothing, use_ref, scale):
    counts, seq = counting(x)
    l, p, hot, S, E = row_terms(x, counts)
    n_seq = x["seq_start"].numel() - 1
    ref = x["ref_logprob"].double() if use_ref else torch.zeros_like(l)
    by = lambda v: torch.zeros(n_seq, dtype=torch.float64, device="cuda").index_add_(0, seq, torch.where(counts, v, 0.0))
    ratio, ratio_tol = by(l - ref), by(E)
    b = float(np.float32(beta))
    s = float(np.float32(smoothing))
    m = b * (ratio[0::2] - ratio[1::2])
    m_tol = b * (ratio_tol[0::2] + ratio_tol[1::2])
    logsig = torch.nn.functional.logsigmoid
    pairs = n_seq // 2
    loss = -(1 - s) * logsig(m) - s * logsig(-m)
    stats = torch.stack([loss.mean(), (m > 0).double().mean(), b * ratio[0::2].mean(), b * ratio[1::2].mean()])
    stat_tol = m_tol.max() + 4 * U * (stats.abs().max() + (b * ratio).abs().max() + loss.abs().max())
    slope = b / pairs * (s * torch.sigmoid(m) - (1 - s) * torch.sigmoid(-m)) * scale
    slope_tol = b / pairs * scale * m_tol + 4 * U * slope.abs()    # sigmoid' <= 1/4, twice
    both = lambda v, sign: torch.stack([v, sign * v], 1).reshape(-1)[seq]
    return {"stats": stats, "stat_tol": stat_tol, "ratio": ratio, "ratio_tol": ratio_tol + 2 * U * ratio.abs(), "logprob": torch.where(counts, l, 0.0),
            "E": E, "p": p, "hot": hot, "S": S, "counts": counts, "slope": torch.where(counts, both(slope, -1), 0.0),
            "slope_tol": torch.where(counts, both(slope_tol, 1), 0.0)}


def check_pairs(x, beta, smoothing, **kw):
    ref = pairs_reference(x, beta, smoothing, kw.get("use_ref", True), kw.get("scale", 1.0))
    stats, lr, lp, g = run_pairs(x, beta, smoothing, **kw)
    assert bool(((lp.double() - ref["logprob"]).abs() <= ref["E"]).all()) and bool((lp[~ref["counts"]] == 0).all())
    assert bool(((lr.double() - ref["ratio"]).abs() <= ref["ratio_tol"]).all())
    assert bool(((stats.double() - ref["stats"]).abs() <= ref["stat_tol"]).all()), (stats, ref["stats"], ref["stat_tol"])
    if g is not None:
        check_grad(g, ref)
    return stats, lr, lp, g


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,pairs,vocab,pad,shift", [
    (2, 1, 1, 0, 0), (2, 1, 9, 0, 1), (40, 6, 77, 3, 0), (203, 8, 1024, 0, 0), (33, 3, 4097, 0, 1), (50, 2, 20011, 5, 0), (4, 1, 152064, 0, 0),
    (600, 40, 10007, 0, 0), (3000, 500, 100, 0, 0), (270, 5, 152064, 0, 0)])
def test_preference_loss_over_sizes(dtype, rows, pairs, vocab, pad, shift):
    x = make(rows, 2 * pairs, vocab, dtype, rows, pad=pad, shift=shift)
    check_pairs(x, 0.1, 0.0, scale=4096.0 if dtype == torch.float16 else 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab", [(91, 777), (301, 12001)])
@pytest.mark.parametrize("smoothing", [0.0, 0.2, 1.0])
@pytest.mark.parametrize("use_ref", [True, False])
def test_preference_loss_over_masks_and_labels(rows, vocab, smoothing, use_ref):
    x = make(rows, 8, vocab, torch.bfloat16, 3, masked=0.5, cuts=[5, 20, 40, 40, 40, 41, 50, 60, rows - 6])
    x["mask"][41:50] = 0
    counts, _ = counting(x)
    x["logits"][~counts] = float("nan")
    x["ref_logprob"][~counts] = float("nan")
    x["targets"][~counts] = -5
    y = dict(x, targets=torch.where(counts, x["targets"], 0), ref_logprob=torch.where(counts, x["ref_logprob"], 0.0))
    ref = pairs_reference(y, 0.3, smoothing, use_ref, 1.0)
    stats, lr, lp, g = run_pairs(x, 0.3, smoothing, use_ref=use_ref)
    assert bool(((lr.double() - ref["ratio"]).abs() <= ref["ratio_tol"]).all()) and bool((lp[~counts] == 0).all())
    assert bool(((stats.double() - ref["stats"]).abs() <= ref["stat_tol"]).all())
    check_grad(g, ref)
    s1, r1, l1, none = run_pairs(x, 0.3, smoothing, use_ref=use_ref, grad=False)
    assert none is None and torch.equal(s1, stats) and torch.equal(r1, lr) and torch.equal(l1, lp)
    s2, r2, l2, g2 = run_pairs(x, 0.3, smoothing, use_ref=use_ref, in_place=True)
    assert torch.equal(s2, stats) and torch.equal(r2, lr) and torch.equal(l2, lp) and torch.equal(g2, g)


@pytest.mark.gpu
def test_a_target_that_cannot_occur_decides_its_pair():
    """The other sequence has probability 0: the margin is infinite, the loss 0, and no gradient is NaN."""
    x = make(6, 2, 300, torch.float32, 3, cuts=[0, 3, 6])
    x["logits"][4, int(x["targets"][4])] = float("-inf")
    stats, lr, lp, g = run_pairs(x, 0.1, 0.0)
    assert stats[0].item() == 0.0 and stats[1].item() == 1.0 and lr[1].item() == float("-inf") and lp[4].item() == float("-inf")
    assert bool((g == 0).all())


@pytest.mark.gpu
def test_preference_gradient_against_differences():
    x = make(30, 6, 400, torch.float32, 9, masked=0.2)
    _, _, _, g = run_pairs(x, 0.2, 0.1)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(4):
        v = torch.randn(g.shape, generator=gen, device="cuda", dtype=torch.float64)
        h = 1e-5
        f = [pairs_reference(dict(x, logits=x["logits"].double() + s * h * v), 0.2, 0.1, True, 1.0)["stats"][0].item() for s in (1, -1)]
        assert (g.double() * v).sum().item() == pytest.approx((f[0] - f[1]) / (2 * h), rel=1e-4, abs=1e-6)


# ---------------------------------------------------------------------------------------------
# both
# ---------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("rows,n_seq,vocab", [(20011, 3, 40), (20000, 1, 17), (33001, 2, 300), (5000, 3001, 50), (4097, 1024, 600), (4096, 1024, 2100),
                                              (1100, 1100, 6001), (2049, 40, 9001)])
@pytest.mark.parametrize("masked", [0.0, 0.4])
def test_many_rows_and_many_sequences(rows, n_seq, vocab, masked):
    """On both sides of the numbers of rows and sequences up to which one workgroup counts, looks weights up and adds."""
    x = make(rows, n_seq, vocab, torch.bfloat16, 11, masked=masked, lead=1, tail=2)
    for reduce in ("tokens", "sequences", "sums"):
        check_policy(x, reduce, 0.04)
    run = run_policy(x, "sequences", 0.04, grad=False)
    assert torch.equal(run[0], run_policy(x, "sequences", 0.04)[0])
    if n_seq % 2 == 0:
        check_pairs(x, 0.1, 0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_seq,vocab", [(7, 2, 100), (3, 2, 50003), (40, 4, 2049), (300, 8, 30001), (260, 2, 90001), (1030, 4, 9999)])
@pytest.mark.parametrize("shift", [0, 1, 5])
def test_nothing_but_the_outputs_is_written(dtype, rows, n_seq, vocab, shift):
    """Columns between the gradient's rows, elements in front of and behind it, bytes behind the workspace and the small outputs."""
    x = make(rows, n_seq, vocab, dtype, 13, pad=3, masked=0.2)
    ld = vocab + 7
    for pairs in (False, True):
        buf = torch.full((rows * ld + 64,), 3.0, dtype=dtype, device="cuda")
        g = buf[shift:shift + rows * ld].view(rows, ld)[:, :vocab]
        need = sr.token_loss_workspace(rows, n_seq)
        ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
        small = torch.full((4 + rows + n_seq + 16,), 5.0, device="cuda")
        stats, lp, lr = small[:4], small[4:4 + rows], small[4 + rows:4 + rows + n_seq]
        before = x["logits"].clone()
        if pairs:
            sr.sr_preference_loss(x["logits"], x["targets"], x["seq_start"], stats, ws[:need], mask=x["mask"], ref_logprob=x["ref_logprob"],
                                  grad=g, token_logprob=lp, log_ratio=lr)
            check_grad(g, pairs_reference(x, 0.1, 0.0, True, 1.0))
        else:
            sr.sr_policy_loss(x["logits"], x["targets"], x["seq_start"], x["old_logprob"], x["advantages"], stats, ws[:need], mask=x["mask"],
                              ref_logprob=x["ref_logprob"], grad=g, token_logprob=lp, clip_low=LOW, clip_high=HIGH, kl_coef=0.04)
            check_grad(g, policy_reference(x, "tokens", 0.04, True))
            assert bool((lr == 5.0).all())
        assert bool((ws[need:] == 77).all()) and bool((small[4 + rows + n_seq:] == 5.0).all())
        rest = buf.clone()
        rest[shift:shift + rows * ld].view(rows, ld)[:, :vocab] = 3.0
        assert bool((rest == 3.0).all())
        assert torch.equal(before, x["logits"])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab", [(20, 900), (6, 60001), (300, 30001)])
def test_side_streams_repetitions_and_graphs(rows, vocab):
    """Bit-identical from call to call, on another stream, and in every replay of a captured graph, also with new inputs."""
    x = make(rows, 4, vocab, torch.bfloat16, 7, masked=0.2)
    stats, lp, g = run_policy(x, "tokens", 0.04)
    ps, plr, plp, pg = run_pairs(x, 0.1, 0.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s1, l1, g1 = run_policy(x, "tokens", 0.04)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(s1, stats) and torch.equal(l1, lp) and torch.equal(g1, g)
    n_seq = 4
    out = [torch.empty(4, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(g), torch.empty(4, device="cuda"), torch.empty_like(g)]
    ws = torch.empty(sr.token_loss_workspace(rows, n_seq), dtype=torch.uint8, device="cuda")

    def both():
        sr.sr_policy_loss(x["logits"], x["targets"], x["seq_start"], x["old_logprob"], x["advantages"], out[0], ws, mask=x["mask"],
                          ref_logprob=x["ref_logprob"], grad=out[2], token_logprob=out[1], clip_low=LOW, clip_high=HIGH, kl_coef=0.04)
        sr.sr_preference_loss(x["logits"], x["targets"], x["seq_start"], out[3], ws, mask=x["mask"], ref_logprob=x["ref_logprob"], grad=out[4])

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(3):
        if k == 2:
            x["logits"].mul_(0.5)
            stats, lp, g = run_policy(x, "tokens", 0.04)
            ps, _, _, pg = run_pairs(x, 0.1, 0.0)
        for o in out:
            o.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, (stats, lp, g, ps, pg)):
            assert torch.equal(a, b), k


def _rows(**kw):
    r = dict(logits=4096, grad=8192, ld_logits=100, ld_grad=100, targets=4096, mask=None, seq_start=4096, token_logprob=None, dtype=1,
             n_rows=4, vocab=100, n_seq=2, grad_scale=1.0, reserved=0)
    r.update(kw)
    return sr.TokenRows(*[r[n] for n, _ in sr.TokenRows._fields_])


@pytest.mark.parametrize("bad", [dict(logits=None), dict(targets=None), dict(seq_start=None), dict(dtype=3), dict(dtype=-1), dict(n_rows=-1), dict(vocab=0),
                                 dict(n_seq=0), dict(ld_logits=99), dict(ld_grad=99), dict(logits=4097), dict(grad=8193), dict(grad_scale=math.nan),
                                 dict(dtype=0, logits=4098), dict(grad=4096, ld_grad=104), dict(vocab=(1 << 30) + 1, ld_logits=1 << 31, ld_grad=1 << 31),
                                 dict(targets=4097), dict(seq_start=4098), dict(token_logprob=4099)])
def test_refusals_of_rows(bad):
    L, fake = sr.lib(), ctypes.c_void_p(4096)                      # never dereferenced: validation fails first
    big = 1 << 20
    opt = sr.PolicyOptions(0.2, 0.2, 0.0, 0)
    assert L.sr_policy_loss(ctypes.byref(_rows(**bad)), fake, None, fake, ctypes.byref(opt), fake, fake, big, None) == sr.SR_E_ARG
    assert L.sr_preference_loss(ctypes.byref(_rows(**bad)), fake, 0.1, 0.0, None, fake, fake, big, None) == sr.SR_E_ARG


def test_refusals_of_options_and_workspaces():
    L, fake = sr.lib(), ctypes.c_void_p(4096)
    big, need = 1 << 20, sr.token_loss_workspace(4, 2)
    rows = ctypes.byref(_rows())
    good = sr.PolicyOptions(0.2, 0.2, 0.0, 0)
    p = lambda o, old=fake, ref=None, adv=fake, stats=fake, ws=fake, n=big: L.sr_policy_loss(rows, old, ref, adv, ctypes.byref(o), stats, ws, n, None)
    for o in (sr.PolicyOptions(-0.1, 0.2, 0.0, 0), sr.PolicyOptions(1.1, 0.2, 0.0, 0), sr.PolicyOptions(0.2, -0.2, 0.0, 0),
              sr.PolicyOptions(0.2, math.inf, 0.0, 0), sr.PolicyOptions(math.nan, 0.2, 0.0, 0), sr.PolicyOptions(0.2, 0.2, math.nan, 0),
              sr.PolicyOptions(0.2, 0.2, 0.0, 3), sr.PolicyOptions(0.2, 0.2, 0.0, -1), sr.PolicyOptions(0.2, 0.2, 0.1, 0)):
        assert p(o) == sr.SR_E_ARG
    assert p(good, old=None) == p(good, adv=None) == p(good, stats=None) == p(good, ws=None) == sr.SR_E_ARG
    odd = ctypes.c_void_p(4098)
    assert p(good, old=odd) == p(good, ref=odd) == p(good, adv=odd) == p(good, stats=odd) == sr.SR_E_ARG
    assert p(good, ws=ctypes.c_void_p(4104)) == p(good, n=need - 1) == sr.SR_E_ARG
    assert L.sr_policy_loss(None, fake, None, fake, ctypes.byref(good), fake, fake, big, None) == sr.SR_E_ARG
    assert L.sr_policy_loss(rows, fake, None, fake, None, fake, fake, big, None) == sr.SR_E_ARG
    q = lambda r=rows, beta=0.1, s=0.0, stats=fake, n=big: L.sr_preference_loss(r, None, beta, s, None, stats, fake, n, None)
    assert q(r=ctypes.byref(_rows(n_seq=3))) == q(beta=math.inf) == q(s=-0.1) == q(s=1.1) == q(s=math.nan) == sr.SR_E_ARG
    assert q(stats=None) == q(n=need - 1) == q(r=None) == sr.SR_E_ARG


def test_sizes_beyond_a_launch():
    L, fake = sr.lib(), ctypes.c_void_p(4096)
    opt = sr.PolicyOptions(0.2, 0.2, 0.0, 0)
    for bad in (dict(n_rows=(1 << 26) + 1), dict(n_seq=(1 << 23) + 2)):
        rows = ctypes.byref(_rows(**bad))
        assert L.sr_policy_loss(rows, fake, None, fake, ctypes.byref(opt), fake, fake, 1 << 40, None) == sr.SR_E_LIMIT
        assert L.sr_preference_loss(rows, fake, 0.1, 0.0, None, fake, fake, 1 << 40, None) == sr.SR_E_LIMIT


RULES = """
#include "token_plan.h"
extern "C" void rows_plan(int policy, int n_rows, int vocab, int bytes, int *out) {
    const sr::RowPlan p = policy ? sr::plan_policy_rows(n_rows, vocab, bytes) : sr::plan_streamed_rows(n_rows, vocab, bytes);
    const int v[] = {p.waves, p.resident, p.parts, p.elems, p.grad_waves, p.grad_parts, p.grad_elems};
    for (int i = 0; i < 7; ++i) out[i] = v[i];
}
"""


def test_parts_cover_rows_and_fit_the_workspace(tmp_path):
    """Over sizes around every limit: parts are whole vectors, cover the row exactly, are none of them empty, and number at most what
    the workspace holds; a resident row fits the registers that its kernel has."""
    import subprocess
    from paper_2605_05802_amd.build import CSRC
    (tmp_path / "rules.cpp").write_text(RULES)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + CSRC, str(tmp_path / "rules.cpp"), "-o", str(tmp_path / "rules.so")])
    lib, out = ctypes.CDLL(str(tmp_path / "rules.so")), (ctypes.c_int * 7)()
    rng = np.random.default_rng(0)
    vocabs = sorted({1, 2, 7, 8, 9, 4095, 4096, 4097, 40959, 40960, 40961, 81920, 81921, 163839, 163840, 163841, 152064, 1 << 20, 1 << 30,
                     *np.exp(rng.uniform(0, math.log(1 << 21), 200)).astype(int).tolist()})
    for n_rows in (1, 2, 3, 100, 111, 112, 191, 256, 257, 320, 321, 1000, 1023, 1024, 1025, 4096, 8192, 8193, 100000, 1 << 26):
        for vocab in vocabs:
            for size in (2, 4):
                for policy in (0, 1):
                    lib.rows_plan(policy, n_rows, vocab, size, out)
                    waves, resident, parts, elems, grad_waves, grad_parts, grad_elems = out
                    per = 16 // size
                    assert waves in (1, 4, 16) and parts >= 1 and elems % per == 0
                    assert (parts - 1) * elems < vocab <= parts * elems
                    assert parts == 1 or parts * n_rows <= 8192
                    if resident:
                        assert policy and parts == 1 and resident <= (8 if waves == 1 else 20)
                        assert 64 * waves * (resident - 1) < max(vocab // per, 1) <= 64 * waves * resident
                    else:
                        assert grad_waves in (1, 4) and grad_elems % per == 0 and (grad_parts - 1) * grad_elems < vocab <= grad_parts * grad_elems


def test_the_binding_refuses_wrong_tensors():
    t = lambda *s, d=torch.float32: torch.zeros(*s, dtype=d)
    i32 = torch.int32
    ws = t(sr.token_loss_workspace(4, 2), d=torch.uint8)
    good = dict(logits=t(4, 10), targets=t(4, d=i32), seq_start=t(3, d=i32), old_logprob=t(4), advantages=t(2), stats=t(4), workspace=ws)
    for bad in (dict(logits=t(4, 10, d=torch.float64)), dict(logits=t(10, 4).t()), dict(logits=t(40)), dict(targets=t(4, d=torch.int64)),
                dict(targets=t(5, d=i32)), dict(old_logprob=t(8)[::2]), dict(advantages=t(3)), dict(stats=t(3)), dict(grad=t(4, 11)),
                dict(grad=t(4, 10, d=torch.float16)), dict(mask=t(4)), dict(token_logprob=t(3)), dict(ref_logprob=t(4, d=torch.float64))):
        with pytest.raises(sr.SrError) as e:
            sr.sr_policy_loss(**{**good, **bad}, stream=0)
        assert e.value.status == sr.SR_E_ARG


def test_host_tensors_are_refused():
    i32 = torch.int32
    rows = dict(logits=torch.zeros(4, 10), targets=torch.zeros(4, dtype=i32), seq_start=torch.zeros(3, dtype=i32), stats=torch.zeros(4),
                workspace=torch.zeros(sr.token_loss_workspace(4, 2), dtype=torch.uint8))
    with pytest.raises(sr.SrError, match="device tensors expected"):
        sr.sr_policy_loss(old_logprob=torch.zeros(4), advantages=torch.zeros(2), **rows)
    with pytest.raises(sr.SrError, match="device tensors expected"):
        sr.sr_preference_loss(**rows)


def test_more_threads_than_a_launch_has():
    L, fake = sr.lib(), ctypes.c_void_p(4096)
    opt = sr.PolicyOptions(0.2, 0.2, 0.0, 0)
    for n_rows, vocab in (((1 << 26) - 3, 4), (1 << 24, 5000), (1 << 26, 3000)):
        rows = ctypes.byref(_rows(n_rows=n_rows, vocab=vocab, ld_logits=vocab, ld_grad=vocab, grad=4096))
        assert L.sr_policy_loss(rows, fake, None, fake, ctypes.byref(opt), fake, fake, 1 << 40, None) == sr.SR_E_LIMIT
        assert L.sr_preference_loss(rows, fake, 0.1, 0.0, None, fake, fake, 1 << 40, None) == sr.SR_E_LIMIT
    rows = ctypes.byref(_rows(n_rows=1 << 23, vocab=50000, ld_logits=50000, ld_grad=50000, grad=4096))
    assert L.sr_preference_loss(rows, fake, 0.1, 0.0, None, fake, fake, 1 << 40, None) == sr.SR_E_LIMIT


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_seq,vocab,pad,shift", [
    (7, 3, 45056, 0, 0),        # parts of one wavefront, bf16
    (50, 60, 22528, 0, 0),      # ... fp32; more sequences than rows
    (120, 1024, 43001, 7, 1), (121, 1025, 43001, 0, 0), (159, 9, 60000, 0, 3), (160, 9, 41000, 0, 0), (127, 5, 21003, 1, 2),
    (257, 300, 41001, 0, 1), (352, 8, 41000, 8, 0), (353, 8, 41000, 0, 0), (2, 2, 400001, 0, 5), (1023, 40, 164001, 0, 0), (1024, 40, 164001, 0, 0)])
def test_few_rows_in_parts(dtype, rows, n_seq, vocab, pad, shift):
    x = make(rows, n_seq, vocab, dtype, rows + vocab, pad=pad, shift=shift, masked=0.25 if rows > 7 else 0.0, lead=min(rows // 9, 5), tail=min(rows // 7, 3))
    scale = 4096.0 if dtype == torch.float16 else 1.0
    for reduce in ("tokens", "sequences", "sums") if rows < 200 else ("sequences",):
        stats, lp, g = check_policy(x, reduce, 0.04, scale=scale)
    s1, l1, none = run_policy(x, reduce, 0.04, grad=False, scale=scale)
    assert torch.equal(s1, stats) and torch.equal(l1, lp)
    s2, l2, g2 = run_policy(x, reduce, 0.04, in_place=True, scale=scale)
    assert torch.equal(s2, stats) and torch.equal(l2, lp) and torch.equal(g2, g)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_seq,vocab,pad,shift", [
    (520, 30, 41001, 0, 1), (769, 7, 45056, 1, 0), (400, 3, 81921, 0, 0), (513, 600, 100000, 3, 1), (600, 40, 152064, 0, 1)])
def test_workgroups_of_several_rows(dtype, rows, n_seq, vocab, pad, shift):
    """Rows held in registers, two or more a workgroup, which begin at and inside words."""
    x = make(rows, n_seq, vocab, dtype, rows, pad=pad, shift=shift, masked=0.3, lead=5, tail=7)
    scale = 4096.0 if dtype == torch.float16 else 1.0
    stats, lp, g = check_policy(x, "sequences", 0.04, scale=scale)
    s2, l2, g2 = run_policy(x, "sequences", 0.04, in_place=True, scale=scale)
    assert torch.equal(s2, stats) and torch.equal(l2, lp) and torch.equal(g2, g)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [3, 70, 1030])
@pytest.mark.parametrize("vocab", [1, 2, 8, 9, 15, 16, 17, 512, 4096, 4097, 16384])
def test_rows_that_begin_inside_words(dtype, rows, vocab):
    """Gradient and logits apart by a word, by half of one, and every row differently."""
    for shift, pad in ((1, 0), (1, 1), (0, 1), (3, 2)):
        x = make(rows, 2, vocab, dtype, vocab, pad=pad, shift=shift)
        check_policy(x, "tokens", 0.04, scale=4096.0 if dtype == torch.float16 else 1.0)
        check_pairs(x, 0.2, 0.1, scale=4096.0 if dtype == torch.float16 else 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,pairs,vocab,pad,shift", [
    (2, 1, 3, 0, 1), (256, 1, 515, 0, 0), (257, 1, 515, 0, 0), (256, 8, 2001, 0, 1), (256, 9, 2001, 1, 0), (255, 2, 3500, 0, 3), (10, 4, 50021, 0, 0),
    (300, 1, 515, 0, 0), (512, 16, 2001, 0, 1), (513, 16, 2001, 0, 1), (512, 17, 2001, 1, 0), (500, 2, 7000, 0, 3), (65, 13, 50021, 0, 0),
    (130, 1, 12288, 0, 0), (7, 3, 45056, 0, 0), (31, 16, 152064, 0, 1)])
def test_few_pairs(dtype, rows, pairs, vocab, pad, shift):
    """Either side of the sizes up to which the loss has two kernels; the sums are the same with and without a gradient."""
    scale = 4096.0 if dtype == torch.float16 else 1.0
    for masked, lead, tail in ((0.0, 0, 0), (0.3, rows // 9, rows // 7)):
        x = make(rows, 2 * pairs, vocab, dtype, rows + vocab, pad=pad, shift=shift, masked=masked, lead=lead, tail=tail)
        stats, lr, lp, g = check_pairs(x, 0.1, 0.2, scale=scale)
        s1, r1, l1, none = run_pairs(x, 0.1, 0.2, grad=False, scale=scale)
        assert torch.equal(s1, stats) and torch.equal(r1, lr) and torch.equal(l1, lp)
        s2, r2, l2, g2 = run_pairs(x, 0.1, 0.2, in_place=True, scale=scale)
        assert torch.equal(s2, stats) and torch.equal(r2, lr) and torch.equal(l2, lp) and torch.equal(g2, g)


def test_refusals_of_log_probabilities_that_are_read_and_written():
    """The whole array, and one element of four, on either side."""
    L, fake, base = sr.lib(), ctypes.c_void_p(4096), 1 << 20
    opt = sr.PolicyOptions(0.2, 0.2, 0.1, 0)
    for at in (base, base - 12, base + 12):
        rows, same = ctypes.byref(_rows(token_logprob=base)), ctypes.c_void_p(at)
        policy = lambda old, ref: L.sr_policy_loss(rows, old, ref, fake, ctypes.byref(opt), fake, fake, 1 << 20, None)
        assert policy(same, fake) == policy(fake, same) == policy(same, same) == sr.SR_E_ARG
        assert L.sr_preference_loss(rows, same, 0.1, 0.0, None, fake, fake, 1 << 20, None) == sr.SR_E_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab", [(6, 300), (6, 50021), (300, 20003)])
def test_log_probabilities_beside_the_ones_they_are_compared_with(rows, vocab):
    """Three neighbours in one array."""
    x = make(rows, 2, vocab, torch.bfloat16, 17)
    stats, lp, g = run_policy(x, "tokens", 0.04)
    _, _, plp, pg = run_pairs(x, 0.1, 0.0)
    three = torch.cat([x["old_logprob"], torch.full_like(lp, 7.0), x["ref_logprob"]])
    old, out, ref = three.split(rows)
    ws = torch.empty(sr.token_loss_workspace(rows, 2), dtype=torch.uint8, device="cuda")
    grad, s = torch.empty_like(g), torch.empty(4, device="cuda")
    sr.sr_policy_loss(x["logits"], x["targets"], x["seq_start"], old, x["advantages"], s, ws, ref_logprob=ref, grad=grad, token_logprob=out,
                      clip_low=LOW, clip_high=HIGH, kl_coef=0.04)
    assert torch.equal(s, stats) and torch.equal(out, lp) and torch.equal(grad, g)
    sr.sr_preference_loss(x["logits"], x["targets"], x["seq_start"], s, ws, ref_logprob=ref, grad=grad, token_logprob=out.fill_(7.0))
    assert torch.equal(out, plp) and torch.equal(grad, pg)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(40, 900), (40, 33003), (260, 16001), (300, 152064)])
def test_advantage_zero_leaves_a_row_out_whatever_its_ratio(dtype, rows, vocab):
    """exp(l - old) beyond single precision, times 0: the surrogate and the slope are 0, as the formula has them."""
    x = make(rows, 5, vocab, dtype, 21, cuts=[0, rows // 4, rows // 2, rows // 2, rows - 3, rows])
    x["old_logprob"][:rows // 4] = -150.0                          # the advantage of sequence 0 is 0
    assert x["advantages"][0].item() == 0.0
    for kl in (0.0, 0.04):
        for grad in (True, False):
            stats, lp, g = check_policy(x, "sequences", kl, grad=grad, scale=4096.0 if dtype == torch.float16 else 1.0)
            assert bool(torch.isfinite(stats).all()) and (g is None or bool(torch.isfinite(g).all()))
            assert kl or g is None or bool((g[:rows // 4] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("pairs,rows,n_seq,vocab,dtype", [(False, 128, 4, 152064, torch.float32), (False, 16, 4, 400000, torch.float16),
                                                          (True, 64, 4, 10200, torch.float32), (True, 62, 16, 20400, torch.bfloat16)])
def test_few_rows_that_do_not_count_cost_no_reading(pairs, rows, n_seq, vocab, dtype):
    """The logits in pinned memory of the host, some hundred times as slow to read: a call in which no row counts, by the mask or because
    every row lies outside the sequences, takes nothing like the time of one in which all do (both readings of every row)."""
    x = make(rows, n_seq, vocab, dtype, 5)
    far = torch.empty(rows, vocab, dtype=dtype, pin_memory=True)
    far.copy_(x["logits"])
    lp, stats, grad = torch.empty(rows, device="cuda"), torch.empty(4, device="cuda"), torch.empty_like(x["logits"])
    ws = torch.empty(sr.token_loss_workspace(rows, n_seq), dtype=torch.uint8, device="cuda")
    opt, L = sr.PolicyOptions(LOW, HIGH, 0.04, 0), sr.lib()
    at = lambda t: None if t is None else t.data_ptr()

    def microseconds(mask, seq_start):
        r = sr.TokenRows(at(far), at(grad), vocab, vocab, at(x["targets"]), at(mask), at(seq_start), at(lp),
                         {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[dtype], rows, vocab, n_seq, 1.0, 0)
        times = []
        for _ in range(12):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            torch.cuda.synchronize()
            a.record()
            stream = torch.cuda.current_stream().cuda_stream
            if pairs:
                status = L.sr_preference_loss(r, at(x["ref_logprob"]), 0.1, 0.0, None, at(stats), at(ws), ws.nbytes, stream)
            else:
                status = L.sr_policy_loss(r, at(x["old_logprob"]), at(x["ref_logprob"]), at(x["advantages"]), opt, at(stats), at(ws), ws.nbytes, stream)
            b.record()
            torch.cuda.synchronize()
            assert status == sr.SR_OK
            times.append(1000.0 * a.elapsed_time(b))
        return min(times[1:])

    all_rows = microseconds(None, x["seq_start"])
    assert bool(torch.isfinite(grad).all()) and bool((grad != 0).any(1).all())
    masked = microseconds(torch.zeros(rows, dtype=torch.uint8, device="cuda"), x["seq_start"])
    assert bool((grad == 0).all()) and bool((lp == 0).all())
    grad.fill_(7.0)
    outside = microseconds(None, torch.full_like(x["seq_start"], rows))
    assert bool((grad == 0).all()) and bool((lp == 0).all())
    # the second reading alone, or as much of it as a thread asks for ahead, is a third of it at the least
    assert max(masked, outside) < all_rows / 4, (masked, outside, all_rows)


THREADS = """
import importlib, sys, threading
import torch
import paper_2605_05802_amd as sr

def call():
    try:
        sr.sr_grad_norm([], torch.zeros(1), torch.zeros(1))
    except sr.SrError:
        return                                                     # host tensors
    except Exception as e:
        bad.append(repr(e))

bad, k, lines = [], 0, 1
while k < lines:
    importlib.reload(sr)                                           # nothing called yet
    lines = 0

    def trace(frame, event, arg):
        global lines
        if frame.f_code.co_filename != sr.__file__:
            return None
        if event == "line":
            lines += 1
            if lines == k + 1:
                other = threading.Thread(target=call)
                other.start()
                other.join()
        return trace

    sys.settrace(trace)
    call()
    sys.settrace(None)
    k += 1
print(k, bad)
sys.exit(1 if bad or k < 5 else 0)
"""


def test_a_first_call_in_the_middle_of_another_threads_first_call():
    """At every line of the binding that the first call passes, another thread makes one of its own from beginning to end."""
    import os
    import subprocess
    import sys
    r = subprocess.run([sys.executable, "-c", THREADS], capture_output=True, text=True, timeout=120,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0, r.stdout + r.stderr


def test_workspaces_of_fewer_bytes_than_elements_are_refused():
    i32, ws = torch.int32, torch.zeros(1, dtype=torch.uint8).expand(1 << 20)
    rows = dict(logits=torch.zeros(4, 10), targets=torch.zeros(4, dtype=i32), seq_start=torch.zeros(3, dtype=i32), stats=torch.zeros(4), workspace=ws)
    for call in (lambda: sr.sr_policy_loss(old_logprob=torch.zeros(4), advantages=torch.zeros(2), **rows), lambda: sr.sr_preference_loss(**rows),
                 lambda: sr.sr_grad_norm([], torch.zeros(1), ws), lambda: sr.sr_clip_grad_norm([], 1.0, torch.zeros(1), ws)):
        with pytest.raises(sr.SrError, match="workspace: contiguous") as e:
            call()
        assert e.value.status == sr.SR_E_ARG


@pytest.mark.parametrize("reduce", ["token", "mean", None, 0])
def test_a_mean_that_does_not_exist_is_refused(reduce):
    i32 = torch.int32
    with pytest.raises(sr.SrError, match="reduce: one of tokens, sequences, sums") as e:
        sr.sr_policy_loss(torch.zeros(4, 10), torch.zeros(4, dtype=i32), torch.zeros(3, dtype=i32), torch.zeros(4), torch.zeros(2), torch.zeros(4),
                          torch.zeros(sr.token_loss_workspace(4, 2), dtype=torch.uint8), reduce=reduce)
    assert e.value.status == sr.SR_E_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab,n_seq", [(300, 500, 6), (40, 9000, 2), (5000, 64, 1500), (260, 50001, 4), (20, 900, 16), (5, 300, 2)])
@pytest.mark.parametrize("masked", [0.0, 0.3])
def test_starts_that_make_no_sense_write_nothing_beside_the_outputs(rows, vocab, n_seq, masked):
    """Elements around and between the gradient's rows, bytes around the workspace and elements around every small output."""
    x = make(rows, n_seq, vocab, torch.bfloat16, 6, masked=masked)
    rng = np.random.default_rng(2)
    top, ld, need = 2 ** 31 - 1, vocab + 7, sr.token_loss_workspace(rows, n_seq)
    for starts in ([top] * (n_seq + 1), [-top - 1] * (n_seq + 1), rng.integers(-5, rows + 5, n_seq + 1).tolist(),
                   [rows] + [0] * (n_seq - 1) + [top], [-3] + [top] * (n_seq - 1) + [rows // 2], [top] + [5] * n_seq,
                   [-rows] * n_seq + [top], [0] * n_seq + [rows + 1], [-1] + [rows + 1] * n_seq):
        seq_start = torch.tensor(starts, dtype=torch.int64, device="cuda").to(torch.int32)
        for pairs, grad in ((False, True), (False, False), (True, True), (True, False)):
            around = torch.full((64 + rows * ld + 64,), 3.0, dtype=torch.bfloat16, device="cuda")
            g = around[64:64 + rows * ld].view(rows, ld)[:, :vocab]
            ws = torch.full((4096 + need + 4096,), 77, dtype=torch.uint8, device="cuda")
            sizes, small, at = [4, rows, n_seq], torch.full((4 + rows + n_seq + 4 * 1024,), 5.0, device="cuda"), 0
            outs, gaps = [], torch.ones_like(small, dtype=torch.bool)
            for n in sizes:
                at += 1024
                outs.append(small[at:at + n])
                gaps[at:at + n] = False
                at += n
            inputs = [x[k] for k in ("logits", "targets", "old_logprob", "ref_logprob", "advantages")] + [seq_start]
            before = [t.clone() for t in inputs]
            common = dict(mask=x["mask"], ref_logprob=x["ref_logprob"], grad=g if grad else None, token_logprob=outs[1])
            if pairs:
                sr.sr_preference_loss(x["logits"], x["targets"], seq_start, outs[0], ws[4096:4096 + need], log_ratio=outs[2], **common)
            else:
                sr.sr_policy_loss(x["logits"], x["targets"], seq_start, x["old_logprob"], x["advantages"], outs[0], ws[4096:4096 + need],
                                  kl_coef=0.04, reduce="sequences", **common)
            g.fill_(3.0)
            assert bool((around == 3.0).all()) and bool((small[gaps] == 5.0).all())
            assert bool((ws[:4096] == 77).all()) and bool((ws[4096 + need:] == 77).all())
            assert all(torch.equal(a, b) for a, b in zip(inputs, before))


BOUNDS = """
#include "token_plan.h"
extern "C" int bound(int row, int n_rows) { return sr::row_bound(row, n_rows); }
extern "C" int sequence(const int *seq_start, int n_seq, int row) { return sr::sequence_of(seq_start, n_seq, row); }
"""


def test_ranges_of_rows_stay_inside_the_rows(tmp_path):
    """Starts of every kind: each range of rows lies in [0, rows], each row's sequence is -1 or one of the sequences whatever surrounds
    the array, and for starts that make sense it is the one that owns the row."""
    import subprocess
    from paper_2605_05802_amd.build import CSRC
    (tmp_path / "bounds.cpp").write_text(BOUNDS)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + CSRC, str(tmp_path / "bounds.cpp"), "-o", str(tmp_path / "bounds.so")])
    lib, rng, top = ctypes.CDLL(str(tmp_path / "bounds.so")), np.random.default_rng(3), 2 ** 31 - 1
    for rows, n_seq in ((1, 1), (5, 2), (20, 16), (300, 6), (4096, 1024), (5000, 1500), (1 << 26, 3)):
        some = sorted({0, 1, rows // 2, rows - 1, *rng.integers(0, rows, 30).tolist()} & set(range(rows)))
        good = np.sort(rng.integers(0, rows + 1, n_seq + 1))
        for starts in ([top] * (n_seq + 1), [-top - 1] * (n_seq + 1), rng.integers(-5, rows + 5, n_seq + 1), [rows] + [0] * (n_seq - 1) + [top],
                       [-3] + [top] * (n_seq - 1) + [rows // 2], [top] + [5] * n_seq, [-rows] * n_seq + [top], [-1] + [rows + 1] * n_seq, good):
            starts = np.array(starts, dtype=np.int64)
            assert all(0 <= lib.bound(int(s), rows) <= rows for s in starts)
            assert [lib.bound(int(s), rows) for s in starts] == np.clip(starts, 0, rows).tolist()
            answers = []
            for poison in (-top - 1, top):
                field = np.full(n_seq + 1 + 2 * (n_seq + 8), poison, dtype=np.int32)
                field[n_seq + 8:2 * n_seq + 9] = starts
                at = field.ctypes.data_as(ctypes.POINTER(ctypes.c_int))
                at = ctypes.cast(ctypes.addressof(at.contents) + 4 * (n_seq + 8), ctypes.POINTER(ctypes.c_int))
                answers.append([lib.sequence(at, n_seq, r) for r in some])
            assert answers[0] == answers[1] and all(-1 <= a < n_seq for a in answers[0])
            if np.array_equal(starts, good):
                for r, a in zip(some, answers[0]):
                    inside = (starts[:-1] <= r) & (r < starts[1:])
                    assert a == (int(inside.argmax()) if inside.any() else -1)


row_terms_of_any_order = row_terms


def tight_row_terms(chain):
    """row_terms with the error of a row's sum as its kernel adds it up.  Every exponential: the difference, its product with log2(e) and
    that constant 3.2 u of |x - m| together, however many rescalings that distance is made of, and one unit in the last place; sixteen
    additions in a group; then `chain` steps (groups of a lane, wavefronts, parts) of an exponential and a sum, 5 u each, and ten
    additions over lanes.  The distance enters with its mean D over the row's distribution:
        rel(s) <= u (28 + 5 (chain + 2) + 3.2 D)."""
    def terms(x, counts):
        l, p, hot, _, _ = row_terms_of_any_order(x, counts)
        z = torch.where(counts[:, None], x["logits"].double(), torch.zeros((), dtype=torch.float64, device="cuda"))
        off = z.gather(1, x["targets"].long()[:, None])[:, 0] - z.max(1).values
        D = float((p * (z.max(1, keepdim=True).values - z)).sum(1).max())
        S = U * (28 + 5 * (chain + 2) + 3.2 * D)
        return l, p, hot, S, S + 2 * U * (off.abs() + (off - l).abs() + 1)
    return terms


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rows,n_seq,vocab,chain,pair_chain", [
    (torch.bfloat16, 400, 4, 152064, 11, 22),  # 20 vectors a thread of 16 wavefronts: 10 groups; 2 parts of 40 vectors: 20
    (torch.float32, 130, 4, 152064, 13, 13),   # 7 parts of 22 vectors a thread: 6 groups
    (torch.bfloat16, 5, 2, 152064, 39, 39),    # 37 parts of 3 vectors a thread: 2 groups
    (torch.float16, 300, 6, 32011, 9, 7),      # 16 vectors a thread of 4 wavefronts: 8 groups; 3 parts of 6 vectors: 4
    (torch.float32, 64, 8, 1024, 2, 2)])       # 4 vectors a thread of one wavefront: 1 group
def test_sums_of_wide_rows_keep_single_precision(monkeypatch, dtype, rows, n_seq, vocab, chain, pair_chain):
    """Log-probabilities, loss and gradient of both losses, with bounds that follow the kernels' own order of additions."""
    x = make(rows, n_seq, vocab, dtype, 27, masked=0.2)
    scale = 4096.0 if dtype == torch.float16 else 1.0
    monkeypatch.setitem(globals(), "row_terms", tight_row_terms(chain))
    check_policy(x, "tokens", 0.04, scale=scale)
    monkeypatch.setitem(globals(), "row_terms", tight_row_terms(pair_chain))
    check_pairs(x, 0.1, 0.1, scale=scale)
