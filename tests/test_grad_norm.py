"""sr_grad_norm and sr_clip_grad_norm against a plain evaluation in 64 bits.

Tolerances.  Squares are formed and added in 64 bits (at most 2^31 terms: relative 1e-7 at the very worst, 1e-12 as a rule), so the
norm carries one rounding to single precision; the factor another, the product a third and, for 16-bit outputs, a fourth to
the output's type: 4 * 2^-24 relative, plus half a unit in the last place of the output's type."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2605_05802_amd as sr

U = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 1.5e-45, torch.bfloat16: 1e-40, torch.float16: 2.0 ** -24}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def work():
    return torch.full((1,), 7.0, device="cuda"), torch.full((sr.GRAD_NORM_WORKSPACE,), 255, dtype=torch.uint8, device="cuda")


def tensors_of(sizes, dtypes, seed, std=0.01, shift=0):
    """Tensors that begin `shift` elements behind an aligned address."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        d = dtypes[i % len(dtypes)]
        buf = torch.empty(n + shift, dtype=d, device="cuda")
        buf.copy_(torch.randn(n + shift, generator=g, device="cuda") * std)
        out.append(buf[shift:])
    return out


def norm_of(ts, scale=1.0):
    return abs(scale) * math.sqrt(sum(float((t.double() ** 2).sum()) for t in ts))


def check(ts, max_norm, scale=1.0, out_dtype=None, in_place=False):
    want = norm_of(ts, scale)
    c = scale * (max_norm / want if want > max_norm else 1.0)
    expect = [t.double() * c for t in ts]
    norm, ws = work()
    sr.sr_grad_norm(ts, norm, ws, scale=scale)
    assert norm.item() == pytest.approx(want, rel=4 * U)
    norm.fill_(7.0)
    outs = None if in_place else [torch.full_like(t, 5.0, dtype=out_dtype or t.dtype) for t in ts]
    sr.sr_clip_grad_norm(sr.tensor_list(ts, outs), max_norm, norm, ws, scale=scale)
    assert norm.item() == pytest.approx(want, rel=4 * U)
    for got, e in zip(ts if in_place else outs, expect):
        tol = e.abs() * (4 * U + ROUND[got.dtype]) + SMALLEST[got.dtype]
        assert bool(((got.double() - e).abs() <= tol).all())
    return norm, outs


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("sizes", [[1], [7], [8], [0, 3, 0], [8191, 8192, 8193], [1 << 20], [5, 100003, 1, 64, 262147], list(range(1, 400))])
@pytest.mark.parametrize("shift", [0, 1])
def test_sizes_types_and_alignment(dtype, out, sizes, shift):
    ts = tensors_of(sizes, [dtype], 1, shift=shift)
    norm = norm_of(ts)
    for limit in (0.5 * norm, 2 * norm):
        check(ts, limit, out_dtype=out)
    if out == dtype:
        check(ts, 2 * norm, in_place=True)
        check(ts, 0.5 * norm, in_place=True)


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.125, -2.0, 1.0, 0.0])
def test_mixed_types_scales_and_limits(scale):
    ts = tensors_of([1000, 33, 20001, 4096], [F32, BF16, F16], 2)
    for limit in (0.0, 1e-3, 1e9):
        check(ts, limit, scale=scale, out_dtype=F32)
    check(ts, 1e-3, scale=scale, in_place=True)


@pytest.mark.gpu
def test_magnitudes_whose_squares_leave_single_precision():
    for std in (1e-30, 1e30):
        check(tensors_of([5000, 77], [F32, BF16], 3, std=std), 1.0, out_dtype=F32)


@pytest.mark.gpu
def test_a_limit_that_is_met_changes_no_bit():
    ts = tensors_of([1000, 5], [BF16, F32], 4)
    before = [t.clone() for t in ts]
    norm, ws = work()
    sr.sr_clip_grad_norm(ts, norm_of(ts) * 1.001, norm, ws)
    assert all(torch.equal(a, b) for a, b in zip(ts, before))


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_norm_that_is_not_finite_is_reported_and_nothing_is_scaled(bad):
    ts = tensors_of([10000, 50], [F32], 5)
    ts[0][7777] = bad
    before = [t.clone() for t in ts]
    norm, ws = work()
    sr.sr_clip_grad_norm(ts, 0.1, norm, ws)
    assert math.isnan(norm.item()) if math.isnan(bad) else norm.item() == math.inf
    assert all(torch.equal(a.view(torch.int32), b.view(torch.int32)) for a, b in zip(ts, before))
    outs = [torch.empty_like(t) for t in ts]
    sr.sr_clip_grad_norm(sr.tensor_list(ts, outs), 0.1, norm, ws, scale=2.0)
    assert torch.equal(outs[1], 2 * ts[1])


@pytest.mark.gpu
def test_more_tensors_than_any_launch_takes():
    """Several thousand small tensors among large ones: the sums of many launches share the workspace."""
    sizes = [3 + i % 5 for i in range(1500)] + ([20_000_001] + [9] * 130) * 7
    ts = tensors_of(sizes, [F32], 6)
    check(ts, 0.3)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16)])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_nothing_but_the_outputs_is_written(dtype, out, shift):
    sizes = [1, 8192, 5, 8191, 20000, 3]
    ts = tensors_of(sizes, [dtype], 9, shift=shift)
    before = [t.clone() for t in ts]
    buf = torch.full((sum(sizes) + 16 * len(sizes) + 64,), 3.0, dtype=out, device="cuda")
    outs, at, gaps = [], shift, torch.ones_like(buf, dtype=torch.bool)
    for n in sizes:
        outs.append(buf[at:at + n])
        gaps[at:at + n] = False
        at += n + 3
    norm = torch.full((3,), 7.0, device="cuda")
    ws = torch.full((sr.GRAD_NORM_WORKSPACE + 512,), 77, dtype=torch.uint8, device="cuda")
    want = norm_of(ts)
    sr.sr_clip_grad_norm(sr.tensor_list(ts, outs), 0.5 * want, norm[1:2], ws[:sr.GRAD_NORM_WORKSPACE])
    for o, t in zip(outs, ts):
        e = t.double() * 0.5
        assert bool(((o.double() - e).abs() <= e.abs() * (4 * U + ROUND[out]) + SMALLEST[out]).all())
    assert bool((buf[gaps] == 3.0).all()) and all(torch.equal(a, b) for a, b in zip(ts, before))
    assert norm[0].item() == norm[2].item() == 7.0 and bool((ws[sr.GRAD_NORM_WORKSPACE:] == 77).all())


@pytest.mark.gpu
def test_nothing_at_all():
    norm, ws = work()
    sr.sr_clip_grad_norm([], 1.0, norm, ws)
    assert norm.item() == 0.0
    norm.fill_(7.0)
    sr.sr_grad_norm([torch.empty(0, device="cuda")], norm, ws)
    assert norm.item() == 0.0
    check([torch.zeros(100, device="cuda")], 0.0)


@pytest.mark.gpu
def test_one_tensor_of_more_than_2_to_the_31_elements():
    n = (1 << 31) + 12345
    t = torch.zeros(n, dtype=BF16, device="cuda")
    t[5], t[n - 1], t[1 << 31] = 3.0, 4.0, 12.0
    norm, ws = work()
    sr.sr_clip_grad_norm([t], 1.0, norm, ws)
    assert norm.item() == 13.0
    want = torch.tensor([3 / 13, 4 / 13, 12 / 13], dtype=F32).to(BF16)
    assert [t[5].item(), t[n - 1].item(), t[1 << 31].item()] == want.tolist() and t[1000].item() == 0.0


@pytest.mark.gpu
def test_repetitions_streams_and_graphs():
    ts = tensors_of([100000, 33, 9_000_001], [F32, BF16], 8)
    outs = [torch.empty_like(t) for t in ts]
    listed = sr.tensor_list(ts, outs)
    norm, ws = work()
    sr.sr_clip_grad_norm(listed, 0.5, norm, ws)
    want, first = norm.clone(), [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sr.sr_clip_grad_norm(listed, 0.5, norm, ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(norm, want) and all(torch.equal(a, b) for a, b in zip(outs, first))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sr.sr_clip_grad_norm(listed, 0.5, norm, ws)
    for k in range(3):
        if k == 2:
            ts[0].mul_(3.0)
            sr.sr_clip_grad_norm(listed, 0.5, norm, ws)
            want, first = norm.clone(), [o.clone() for o in outs]
        norm.fill_(7.0)
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, want) and all(torch.equal(a, b) for a, b in zip(outs, first))


def test_refusals():
    L, fake = sr.lib(), ctypes.c_void_p(4096)                      # never dereferenced: validation fails first
    one = lambda data=4096, out=None, n=5, dtype=0, out_dtype=0: (sr.Tensor * 1)(sr.Tensor(data, out, n, dtype, out_dtype))
    clip = lambda a=one(), n=1, scale=1.0, limit=1.0, norm=fake, ws=fake, size=sr.GRAD_NORM_WORKSPACE: L.sr_clip_grad_norm(
        a, n, scale, limit, norm, ws, size, None)
    for r in (clip(a=None), clip(n=-1), clip(scale=math.nan), clip(limit=math.inf), clip(limit=-1.0), clip(norm=None), clip(norm=ctypes.c_void_p(4098)), clip(ws=None),
              clip(ws=ctypes.c_void_p(4100)), clip(size=sr.GRAD_NORM_WORKSPACE - 1), clip(a=one(data=None)), clip(a=one(data=4098)),
              clip(a=one(n=-1)), clip(a=one(n=1 << 50)), clip(a=one(n=(1 << 36) + 1)), clip(a=one(dtype=3)), clip(a=one(dtype=1, out=8192, out_dtype=2)),
              clip(a=one(out=8192, out_dtype=1)), clip(a=one(dtype=1, out=8193, out_dtype=1)), clip(a=one(dtype=1, out=4096, out_dtype=0))):
        assert r == sr.SR_E_ARG
    assert L.sr_grad_norm(one(data=None), 1, 1.0, fake, fake, sr.GRAD_NORM_WORKSPACE, None) == sr.SR_E_ARG
    with pytest.raises(sr.SrError):
        sr.tensor_list([torch.zeros(3, dtype=torch.float64)])
    with pytest.raises(sr.SrError):
        sr.tensor_list([torch.zeros(4, 4).t()])
    with pytest.raises(sr.SrError):
        sr.tensor_list([torch.zeros(3)], [torch.zeros(4)])
    with pytest.raises(sr.SrError):
        sr.tensor_list([torch.zeros(3)], [])


@pytest.mark.gpu
@pytest.mark.parametrize("count", [1, 64, 511, 512, 513, 4096, 4097, 9000])
def test_planned_lists_of_any_length(count):
    """One table on the device: up to 512 tensors are copied to LDS, more are searched, 64 at a time.  Empty tensors, several
    chunks in some of them and all three types among them."""
    sizes = [(i * 7919) % 23 if i % 97 else 8192 * (i % 5) + i % 3 for i in range(count)]
    sizes[0] = 40000
    ts = tensors_of(sizes, [F32, BF16, F16], 11)
    check(ts, 0.3 * norm_of(ts))
    listed, (norm, ws) = sr.tensor_list(ts), work()
    sr.sr_grad_norm(listed, norm, ws, scale=-0.5)
    assert norm.item() == pytest.approx(0.5 * norm_of(ts), rel=4 * U)


@pytest.mark.gpu
def test_a_plan_writes_its_table_and_nothing_else():
    ts = tensors_of([0, 5, 10000, 0, 7], [F32], 12)
    rows = (sr.Tensor * 5)(*[sr.Tensor(t.data_ptr(), None, t.numel(), 0, 0) for t in ts])
    table = torch.full((64 + 24 * 5 + 64,), 99, dtype=torch.uint8, device="cuda")
    plan = sr.TensorPlan()
    assert sr.lib().sr_plan_tensors(rows, 5, table.data_ptr(), 64 + 24 * 5, plan, None) == sr.SR_OK
    assert bool((table[-64:] == 99).all()) and plan.n_tensors == 3 and plan.chunks == 4
    assert sr.lib().sr_plan_tensors(rows, 0, table.data_ptr(), 64, plan, None) == sr.SR_OK
    norm, ws = work()
    assert sr.lib().sr_planned_clip_grad_norm(plan, 1.0, 1.0, norm.data_ptr(), ws.data_ptr(), ws.nbytes, None) == sr.SR_OK
    torch.cuda.synchronize()
    assert norm.item() == 0.0


def test_refusals_of_plans():
    L, fake = sr.lib(), ctypes.c_void_p(4096)                      # never dereferenced: validation fails first
    one = (sr.Tensor * 1)(sr.Tensor(4096, None, 5, 0, 0))
    plan = sr.TensorPlan()
    make = lambda a=one, n=1, table=fake, size=88, to=plan: L.sr_plan_tensors(a, n, table, size, to, None)
    for r in (make(a=None), make(n=-1), make(table=None), make(table=ctypes.c_void_p(4104)), make(size=87), make(to=None),
              make(a=(sr.Tensor * 1)(sr.Tensor(None, None, 5, 0, 0))), make(a=(sr.Tensor * 1)(sr.Tensor(4096, 4096, 5, 1, 0)))):
        assert r == sr.SR_E_ARG
    many = (sr.Tensor * 256)(*[sr.Tensor(4096, None, 1 << 36, 1, 0)] * 256)
    assert make(a=many, n=256, size=64 + 24 * 256) == sr.SR_E_LIMIT
    good = dict(table=4096, chunks=3, keep=0, n_tensors=2, reserved=0)
    clip = lambda scale=1.0, limit=1.0, norm=fake, ws=fake, size=sr.GRAD_NORM_WORKSPACE, **k: L.sr_planned_clip_grad_norm(
        sr.TensorPlan(**{**good, **k}), scale, limit, norm, ws, size, None)
    for r in (clip(scale=math.nan), clip(limit=-1.0), clip(norm=None), clip(ws=None), clip(size=100), clip(table=None),
              clip(n_tensors=-1), clip(chunks=1), clip(chunks=1 << 31)):
        assert r == sr.SR_E_ARG
    assert L.sr_planned_clip_grad_norm(None, 1.0, 1.0, fake, fake, sr.GRAD_NORM_WORKSPACE, None) == sr.SR_E_ARG
    assert L.sr_planned_grad_norm(None, 1.0, fake, fake, sr.GRAD_NORM_WORKSPACE, None) == sr.SR_E_ARG


def test_host_tensors_are_refused():
    for make in (lambda t: sr.TensorList([t]), lambda t: sr.tensor_list([t]), lambda t: sr.sr_grad_norm([], t, t)):
        with pytest.raises(sr.SrError, match="device tensors expected"):
            make(torch.zeros(1))


@pytest.mark.gpu
@pytest.mark.parametrize("plan", [False, True])
@pytest.mark.parametrize("value,scale", [(1e38, 1.0), (1e30, 1e9), (3e38, -2.0)])
def test_a_norm_beyond_single_precision_scales_nothing(plan, value, scale):
    """A hundred elements whose norm is finite in 64 bits and infinite as it is written: the factor is 1, in place and not."""
    ts = [torch.full((n,), value, device="cuda") for n in (93, 7)]
    assert norm_of(ts, scale) > torch.finfo(F32).max
    before, outs = [t.clone() for t in ts], [torch.empty_like(t) for t in ts]
    norm, ws = work()
    sr.sr_grad_norm(ts, norm, ws, scale=scale)
    assert norm.item() == math.inf
    sr.sr_clip_grad_norm(sr.TensorList(ts, outs, plan=plan), 0.1, norm.fill_(7.0), ws, scale=scale)
    assert norm.item() == math.inf
    assert all(torch.equal(o, b * scale) for o, b in zip(outs, before)) and all(torch.equal(a, b) for a, b in zip(ts, before))
    sr.sr_clip_grad_norm(sr.TensorList(ts, plan=plan), 0.1, norm.fill_(7.0), ws, scale=scale)
    assert norm.item() == math.inf and all(torch.equal(a, b * scale) for a, b in zip(ts, before))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out,std,limit", [
    (F32, F32, 1e30, 1e-10), (F32, F32, 1e30, 1e-25), (F32, F32, 1e36, 0.3), (BF16, F32, 1e30, 1e-10), (BF16, BF16, 1e30, 1e-25),
    (F16, F32, 1e3, 1e-36), (F32, F32, 1.0, 1e-36), (BF16, BF16, 1e36, 0.3)])
def test_factors_below_the_normal_numbers(dtype, out, std, limit):
    """limit / norm is subnormal or 0 in single precision, the products are not."""
    sizes = [5000, 77, 8192, 20001]
    ts = tensors_of(sizes, [dtype], 13, std=std)
    for scale in (1.0, -0.25):
        assert limit / norm_of(ts) < 2.0 ** -126
        check(ts, limit, scale=scale, out_dtype=out)
    if out == dtype:
        check(ts, limit, in_place=True)


@pytest.mark.gpu
def test_the_largest_norm_that_single_precision_holds_is_scaled():
    top = torch.finfo(F32).max
    check([torch.full((1,), top, device="cuda")], 1.0)
    check([torch.full((1,), top, device="cuda")], 1.0, in_place=True)


def clip_direct(ts, max_norm, norm, ws, outs=None, scale=1.0, stream=None):
    """The call over a list that is not planned: the tensors travel in the arguments of launches of at most 184."""
    listed = sr.TensorList(ts, outs)
    assert listed.plan is None
    sr.sr_clip_grad_norm(listed, max_norm, norm, ws, scale=scale, stream=stream)


def check_direct(ts, max_norm, scale=1.0, out_dtype=None, in_place=False):
    want = norm_of(ts, scale)
    c = scale * (max_norm / want if want > max_norm else 1.0)
    expect = [t.double() * c for t in ts]
    norm, ws = work()
    outs = None if in_place else [torch.full_like(t, 5.0, dtype=out_dtype or t.dtype) for t in ts]
    clip_direct(ts, max_norm, norm, ws, outs, scale)
    assert norm.item() == pytest.approx(want, rel=4 * U)
    for got, e in zip(ts if in_place else outs, expect):
        assert bool(((got.double() - e).abs() <= e.abs() * (4 * U + ROUND[got.dtype]) + SMALLEST[got.dtype]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("sizes", [[1], [0, 3, 0], [8191, 8192, 8193], [5, 100003, 1, 64, 262147], list(range(1, 400)), [1 << 24, 77]])
@pytest.mark.parametrize("shift", [0, 1])
def test_lists_in_the_arguments(dtype, out, sizes, shift):
    ts = tensors_of(sizes, [dtype], 21, shift=shift)
    norm = norm_of(ts)
    for limit, scale in ((0.5 * norm, 1.0), (2 * norm, 1.0), (0.1 * norm, -0.5)):
        check_direct(ts, limit, scale, out)
    if out == dtype:
        check_direct(ts, 2 * norm, in_place=True)
        check_direct(ts, 0.5 * norm, in_place=True)


@pytest.mark.gpu
@pytest.mark.parametrize("count", [183, 184, 185, 368, 369, 1500])
@pytest.mark.parametrize("most", [9, 30000])
def test_lists_of_several_launches(count, most):
    """Either side of what one launch takes, empty tensors and all three types among them; few chunks, whose workgroups add the squares
    up for themselves and of which the first launch writes the norm, and many."""
    sizes = [(i * 7919) % most for i in range(count)]
    ts = tensors_of(sizes, [F32, BF16, F16], 22)
    check_direct(ts, 0.3 * norm_of(ts), scale=0.5, out_dtype=F32)
    check_direct(ts, 0.3 * norm_of(ts), in_place=True)


@pytest.mark.gpu
def test_launches_that_share_the_workspace_and_read_past_the_caches():
    """Several thousand tensors, 560 MB of them: sums of many launches, and the part that the second pass finds in the caches begins
    inside one of them."""
    ts = tensors_of([3 + i % 5 for i in range(1500)] + ([20_000_001] + [9] * 130) * 7, [F32], 23)
    check_direct(ts, 0.3)
    check_direct(ts, 0.2, in_place=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16)])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_lists_in_the_arguments_write_nothing_but_the_outputs(dtype, out, shift):
    sizes = [1, 8192, 5, 8191, 20000, 3] * 40
    ts = tensors_of(sizes, [dtype], 24, shift=shift)
    before = [t.clone() for t in ts]
    buf = torch.full((sum(sizes) + 3 * len(sizes) + 64,), 3.0, dtype=out, device="cuda")
    outs, at, gaps = [], shift, torch.ones_like(buf, dtype=torch.bool)
    for n in sizes:
        outs.append(buf[at:at + n])
        gaps[at:at + n] = False
        at += n + 3
    norm = torch.full((3,), 7.0, device="cuda")
    ws = torch.full((512 + sr.GRAD_NORM_WORKSPACE + 512,), 77, dtype=torch.uint8, device="cuda")
    want = norm_of(ts)
    clip_direct(ts, 0.5 * want, norm[1:2], ws[512:-512], outs)
    for o, t in zip(outs, ts):
        e = t.double() * 0.5
        assert bool(((o.double() - e).abs() <= e.abs() * (4 * U + ROUND[out]) + SMALLEST[out]).all())
    assert bool((buf[gaps] == 3.0).all()) and all(torch.equal(a, b) for a, b in zip(ts, before))
    assert norm[0].item() == norm[2].item() == 7.0 and norm[1].item() == pytest.approx(want, rel=4 * U)
    assert bool((ws[:512] == 77).all()) and bool((ws[-512:] == 77).all())


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[100000, 33, 9_000_001], [50, 9000] * 150])
def test_lists_in_the_arguments_on_streams_and_in_graphs(sizes):
    """A captured call holds its list: every replay gives what an eager call does, also with new values."""
    ts = tensors_of(sizes, [F32, BF16], 25)
    outs = [torch.empty_like(t) for t in ts]
    norm, ws = work()
    clip_direct(ts, 0.5, norm, ws, outs)
    want, first = norm.clone(), [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    norm.fill_(7.0)
    side.wait_stream(torch.cuda.current_stream())
    clip_direct(ts, 0.5, norm, ws, outs, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(norm, want) and all(torch.equal(a, b) for a, b in zip(outs, first))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        clip_direct(ts, 0.5, norm, ws, outs)
    for k in range(4):
        if k == 2:
            ts[0].mul_(3.0)
            clip_direct(ts, 0.5, norm, ws, outs)
            want, first = norm.clone(), [o.clone() for o in outs]
        norm.fill_(7.0)
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, want) and all(torch.equal(a, b) for a, b in zip(outs, first))
