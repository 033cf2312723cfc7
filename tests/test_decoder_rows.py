"""sr_embed, sr_embed_grad, sr_dropout, sr_add_norm, sr_add_norm_grad against plain evaluations in 64 bits.

Tolerances.  u = 2^-24 is half a unit of single precision, R half a unit of an output's type relative to its value.
  embed       one product, one rounding: |e| (u + R).
  embed_grad  a sum of m terms in any order is off by at most m u sum|d|; a product, a sum with what was there: (m + 3) u |scale| sum|d| + u |old|
              + R |e|.  Long sums have chains of at most chunk + ceil(chunks / 4) + 4 additions, with `chunk` as row_plan.h cuts.
  dropout     x keep: keep's rounding and the product, 2 u; the sum u; R.
  total       the same.  It is compared first; what follows is compared with the evaluation from the stored total.
  rstd        a row's squares: chains of at most 32 (a thread's) + 6 + 16 additions and a product each, all positive: 55 u relative; quotient, eps
              3 u; the root halves it, root and reciprocal u each: 55 / 2 + 4 < 32 u.
  out         rstd, two products: 34 u + R.  Scales: the largest of these over a constant: 36 u.  Codes: half a step of their type relative to
              value / scale, at least half the smallest one, 72 u |value / scale| from the two of them.
  gradients   n = h rstd: u.  g = dy gain: u.  c = mean(g n): (55 + 4) u mean|g n|.  rstd (g - n c) + dt:
              u (rstd (5 |g| + |n| (6 |c| + 64 mean|g n|)) + 2 |dt| + 2 |e|) + R |e|; dropout adds 2 u |e|.
  d_gain      rows in turn: chains of at most rows / min(rows, 512) + 1, then 32 parts and 64 groups: (rows / 512 + 100) u sum|dy n| + R |e|.
"""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2605_05802_amd as sr

F32, BF16, F16, E4M3, E5M2 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.float8_e5m2
U = 2.0 ** -24
ROUND = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11, E4M3: 2.0 ** -4, E5M2: 2.0 ** -3}
SMALLEST = {F32: 1e-37, BF16: 1e-37, F16: 2.0 ** -25, E4M3: 2.0 ** -10, E5M2: 2.0 ** -17}      # half the smallest step
LARGEST = {E4M3: 448.0, E5M2: 57344.0}
PAIRS = [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)]
WIDTHS = [1, 2, 3, 5, 7, 8, 9, 11, 63, 64, 65, 127, 250, 256, 257, 511, 512, 513, 1031, 2047, 2048, 2049, 3584, 4095, 4097, 8192, 8201, 16384]


class Field:
    """Rows with `pad` unused columns behind each and `shift` elements in front, all of which hold a value that nothing may change."""

    def __init__(self, rows, width, dtype, pad=0, shift=0, fill=None):
        self.guard = 3.0 if fill is None else fill
        self.buf = torch.full((shift + rows * (width + pad) + 8,), self.guard, dtype=F32, device="cuda").to(dtype)
        self.at = torch.zeros(self.buf.numel(), dtype=torch.bool, device="cuda")
        view = lambda b: b[shift:shift + rows * (width + pad)].view(rows, width + pad)[:, :width]
        self.t = view(self.buf)
        view(self.at).fill_(True)

    def check(self):
        assert bool((self.buf.float()[~self.at] == self.guard).all()), "written between rows"


def randn(gen, rows, width, dtype, std=1.0, pad=0, shift=0):
    f = Field(rows, width, dtype, pad, shift)
    f.t.copy_(std * torch.randn(rows, width, generator=gen, device="cuda"))
    return f


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def close(got, want, tol):
    got, want = got.double(), want.double()
    bad = ~((got - want).abs() <= tol)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, the first at {bad.nonzero()[0].tolist()}: " \
                                f"{got[bad][0].item()!r} for {want[bad][0].item()!r}, worst {((got - want).abs() / tol)[bad].max().item():.3g} tolerances"


def mask_words(seed, which, words):
    """Words `words` (uint64 array) of the stream, by unsigned arithmetic on the host."""
    u, golden = np.uint64, np.uint64(0x9E3779B97F4A7C15)
    with np.errstate(over="ignore"):
        def finish(z):
            z = (z ^ (z >> u(30))) * u(0xBF58476D1CE4E5B9)
            z = (z ^ (z >> u(27))) * u(0x94D049BB133111EB)
            return z ^ (z >> u(31))
        key = finish(finish(np.array([seed], dtype=u) + golden) ^ (np.array([which], dtype=u) * u(0xD1342543DE82EF95) + u(1)))
        return finish(key + (words + u(1)) * golden)


def kept(rows, width, p, seed, mask=0, first_row=0, step=0):
    """Factors of the mask: 0, or 1 over the kept share, in 64 bits."""
    each = (width + 3) // 4
    at = np.arange(rows * each, dtype=np.uint64) + np.uint64(first_row * each % 2 ** 64)
    parts = mask_words(seed % 2 ** 64, (mask + step) % 2 ** 64, at).view("<u2").reshape(rows, 4 * each)[:, :width]
    drop = min(65535, int(float(np.float32(p)) * 65536 + 0.5))
    return (parts >= drop) * (65536.0 / (65536 - drop))


# ------------------------------------------------------------------------------------------------------------------
# on the CPU
# ------------------------------------------------------------------------------------------------------------------
FAKE = 4096                            # never read: everything below fails before


def rows_of(**k):
    return sr.Rows(**{**dict(data=FAKE, ld=64, dtype=0, reserved=0), **k})


def test_mask_keeps_the_share_that_it_says():
    """The reference's mask, of which the kernels' is a copy bit for bit: shares, neighbours and masks of one seed."""
    n = 1 << 18
    for p in (0.1, 0.5):
        k = [(kept(n // 512, 512, p, 3, mask=m) > 0).astype(float) for m in (0, 1)]
        bound = 5 * math.sqrt(p * (1 - p) / n)
        assert abs(k[0].mean() - (1 - p)) < bound + 2 ** -16
        for a, b in ((k[0], k[1]), (k[0][:, 1:], k[0][:, :-1]), (k[0][1:], k[0][:-1]), (k[0][:, 4:], k[0][:, :-4])):
            assert abs(((a - 1 + p) * (b - 1 + p)).mean()) < 5 * p * (1 - p) / math.sqrt(a.size) + 2 ** -15


def test_sizes_of_the_structures():
    assert ctypes.sizeof(sr.Rows) == 24 and ctypes.sizeof(sr.Mask) == 40
    assert ctypes.sizeof(sr.NormRows) == 4 * 24 + 4 * 8 + 6 * 4 and ctypes.sizeof(sr.NormGradRows) == 5 * 24 + 4 * 8 + 6 * 4


def test_embed_refusals():
    L = sr.lib()
    call = lambda t=rows_of(), vocab=10, width=64, tokens=FAKE, n=4, scale=1.0, o=rows_of(data=8192): L.sr_embed(t, vocab, width, tokens, n, scale, o, None)
    for r in (call(t=None), call(o=None), call(vocab=0), call(width=0), call(n=-1), call(tokens=None), call(tokens=FAKE + 2), call(scale=math.nan),
              call(scale=math.inf), call(t=rows_of(data=None)), call(o=rows_of(data=None)), call(t=rows_of(ld=63)), call(o=rows_of(ld=63)),
              call(t=rows_of(data=FAKE + 2)), call(t=rows_of(dtype=3), o=rows_of(dtype=3)), call(t=rows_of(dtype=-1)), call(t=rows_of(dtype=1), o=rows_of(dtype=2)),
              call(o=rows_of(dtype=1)), call(o=rows_of()), call(t=rows_of(ld=-64)), call(t=rows_of(ld=1 << 41))):
        assert r == sr.SR_E_ARG
    wide = rows_of(ld=1 << 21)
    assert call(t=wide, o=wide, width=(1 << 20) + 1) == sr.SR_E_LIMIT
    wide8 = rows_of(ld=1 << 20, data=8192)
    assert call(t=wide, o=wide8, width=1 << 20, n=1 << 20) == sr.SR_E_LIMIT
    assert call(n=0, tokens=None, o=rows_of(data=None)) == sr.SR_OK


def test_embed_grad_refusals():
    L = sr.lib()
    big = 1 << 40

    def call(d=rows_of(), tokens=FAKE, n=4, scale=1.0, t=rows_of(data=8192), vocab=10, width=64, accumulate=0, ws=FAKE, size=big):
        return L.sr_embed_grad(d, tokens, n, scale, t, vocab, width, accumulate, ws, size, None)
    need = sr.embed_grad_workspace(4, 64)
    for r in (call(d=None), call(t=None), call(tokens=None), call(tokens=FAKE + 1), call(n=-1), call(vocab=0), call(width=0), call(scale=math.inf),
              call(ws=None), call(ws=FAKE + 8), call(size=need - 1), call(d=rows_of(data=None)), call(t=rows_of(data=None)), call(t=rows_of()),
              call(d=rows_of(ld=60)), call(t=rows_of(data=8192, ld=60)), call(d=rows_of(dtype=1), t=rows_of(data=8192, dtype=2)),
              call(t=rows_of(data=8192, dtype=1)), call(d=rows_of(dtype=3))):
        assert r == sr.SR_E_ARG
    assert call(n=(1 << 20) + 1) == sr.SR_E_LIMIT
    wide = rows_of(ld=1 << 21)
    assert call(d=wide, t=wide, width=(1 << 20) + 1) == sr.SR_E_LIMIT
    assert call(vocab=(1 << 31) - 1) == sr.SR_E_LIMIT
    assert call(n=0, tokens=None, accumulate=1, d=rows_of(data=None)) == sr.SR_OK            # nothing to add


ROW_PLAN = """
#include "row_plan.h"
#include "sr.h"
extern "C" {
void norm_shape(int width, int single, int *out) {
    const sr::RowShape s = sr::norm_shape(width, single);
    out[0] = s.per_vec; out[1] = s.vecs; out[2] = s.threads; out[3] = s.lanes;
}
int norm_parts(int rows, int width, int single) { return sr::norm_grad_parts(rows, sr::norm_shape(width, single)); }
void grad_plan(int n, int width, int single, int bytes, long long *out) {
    const sr::EmbedGradPlan p = sr::embed_grad_plan(n, width, single, bytes);
    const sr::EmbedGradRoom r = sr::embed_grad_room(n, width, p);
    const long long v[] = {p.per_vec, p.slices, p.chunk, p.spans, p.zero_rows, (long long)r.parts, (long long)r.end, (long long)SR_EMBED_GRAD_WORKSPACE(n, width)};
    for (int i = 0; i < 8; ++i) out[i] = v[i];
}
size_t norm_workspace(int rows, int width) { return SR_NORM_GRAD_WORKSPACE(rows, width); }
}
"""


@pytest.fixture(scope="module")
def row_plan(tmp_path_factory):
    import subprocess
    from paper_2605_05802_amd.build import CSRC, INCLUDE
    d = tmp_path_factory.mktemp("row_plan")
    (d / "p.cpp").write_text(ROW_PLAN)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + CSRC, "-I" + INCLUDE, str(d / "p.cpp"), "-o", str(d / "p.so")])
    lib = ctypes.CDLL(str(d / "p.so"))
    lib.norm_workspace.restype = ctypes.c_size_t
    return lib


def test_every_width_fits_the_threads_of_its_rows(row_plan):
    out = (ctypes.c_int * 4)()
    for single in (0, 1):
        for width in range(1, 16385):
            row_plan.norm_shape(width, single, out)
            per_vec, vecs, threads, lanes = out
            assert width >= per_vec and threads * vecs * per_vec >= width and vecs in (1, 2, 4)
            assert (lanes == threads and vecs == 1 and lanes in (16, 32, 64)) if lanes else (threads % 64 == 0 and 64 < threads <= 1024)
            assert per_vec > 1 or lanes == 16                       # columns one by one: one kernel


def test_partial_sums_fit_their_workspaces(row_plan):
    for width in (1, 7, 64, 65, 256, 257, 1031, 3584, 4097, 16384):
        for rows in (0, 1, 2, 63, 512, 2047, 2048, 2049, 10 ** 6, 2 ** 31 - 1):
            for single in (0, 1):
                parts = row_plan.norm_parts(rows, width, single)
                assert min(rows, 1) <= parts <= min(rows, 2048) and 4 * parts * width <= row_plan.norm_workspace(rows, width) == sr.norm_grad_workspace(rows, width)
    out = (ctypes.c_longlong * 8)()
    for width in (1, 7, 8, 63, 256, 257, 1031, 3584, 16384, 1 << 20):
        for n in [*range(0, 300), 1023, 2047, 2048, 2049, 4096, 8191, 8192, 8193, 50001, 2 ** 20 - 1, 2 ** 20]:
            for single, bytes_ in ((0, 2), (1, 4)):
                row_plan.grad_plan(n, width, single, bytes_, out)
                per_vec, slices, chunk, spans, zero_rows, parts, end, room = out
                assert width >= per_vec and slices * 64 * per_vec >= width and spans * 8 * chunk >= n > (spans - 1) * 8 * chunk - (n == 0)
                assert parts % 16 == 0 and end <= room == sr.embed_grad_workspace(n, width) and 1 <= zero_rows <= 512


def mask_of(**k):
    return sr.Mask(**{**dict(p=0.5, reserved=0, seed=1, mask=0, first_row=0, step=None), **k})


def test_dropout_refusals():
    L = sr.lib()
    call = lambda x=rows_of(), r=None, o=rows_of(data=8192), rows=4, width=64, m=mask_of(): L.sr_dropout(x, r, o, rows, width, m, None)
    for r in (call(x=None), call(o=None), call(m=None), call(rows=-1), call(width=0), call(m=mask_of(p=1.0)), call(m=mask_of(p=-0.1)),
              call(m=mask_of(p=math.nan)), call(m=mask_of(step=FAKE + 4)), call(x=rows_of(data=None)), call(o=rows_of(data=None)), call(x=rows_of(ld=63)),
              call(x=rows_of(dtype=3), o=rows_of(dtype=3)), call(o=rows_of(dtype=1)), call(x=rows_of(dtype=1), r=rows_of(dtype=2), o=rows_of(dtype=2)),
              call(r=rows_of(dtype=0, data=12288), x=rows_of(dtype=1), o=rows_of(dtype=1)), call(o=rows_of(ld=128)),       # in place with another distance
              call(x=rows_of(dtype=1), r=rows_of(data=12288), o=rows_of())):                                  # ... another type
        assert r == sr.SR_E_ARG
    far = lambda data: rows_of(ld=1 << 31, data=data)
    assert call(x=far(FAKE), o=far(8192), width=(1 << 30) + 1) == sr.SR_E_LIMIT
    assert call(x=far(FAKE), o=far(8192), width=1 << 30, rows=1 << 20) == sr.SR_E_LIMIT
    assert call(rows=0, x=rows_of(data=None), o=rows_of(data=None)) == sr.SR_OK


def test_add_norm_refusals():
    L = sr.lib()
    good = dict(x=rows_of(), residual=rows_of(data=8192), total=rows_of(data=12288), out=rows_of(data=16384), gain=FAKE, rstd=None, scales=None,
                dropout=None, gain_dtype=0, rows=4, width=64, scale_block=0, eps=1e-6, reserved=0)
    call = lambda **k: L.sr_add_norm(sr.NormRows(**{**good, **k}), None)
    e4 = rows_of(data=16384, dtype=3)
    for r in (L.sr_add_norm(None, None), call(rows=-1), call(width=0), call(eps=-1.0), call(eps=math.nan), call(eps=math.inf), call(gain=None), call(gain=FAKE + 2),
              call(rstd=FAKE + 2), call(gain_dtype=1), call(gain_dtype=7), call(x=rows_of(dtype=1)), call(x=rows_of(dtype=3)), call(residual=rows_of(dtype=1)),
              call(residual=rows_of(data=None)), call(total=rows_of(data=12288, dtype=1)), call(out=rows_of(data=16384, dtype=1)), call(out=rows_of(data=None)),
              call(out=rows_of(data=16384, dtype=5)), call(out=rows_of(data=16384, ld=63)), call(x=rows_of(ld=63)), call(total=rows_of(data=12288, ld=63)),
              call(out=e4), call(scales=FAKE), call(out=e4, scales=FAKE, scale_block=16), call(out=e4, scales=FAKE, scale_block=-32),
              call(scale_block=32), call(out=e4, scales=FAKE + 1), call(total=rows_of(data=16384)), call(out=rows_of(data=8192)),
              call(total=rows_of(data=FAKE)), call(total=rows_of(data=8192, ld=128)), call(out=rows_of(ld=128)),
              call(dropout=ctypes.pointer(mask_of(p=1.0)))):
        assert r == sr.SR_E_ARG
    wide = {k: rows_of(data=v.data, ld=1 << 15) for k, v in good.items() if isinstance(v, sr.Rows)}
    assert call(width=16385, **wide) == sr.SR_E_LIMIT
    assert call(width=16384, rows=(1 << 31) - 1, **wide) == sr.SR_E_LIMIT
    assert call(width=1, rows=(1 << 31) - 1) == sr.SR_E_LIMIT
    assert call(rows=0) == sr.SR_OK


def test_add_norm_grad_refusals():
    L = sr.lib()
    good = dict(d_out=rows_of(), total=rows_of(data=8192), d_total=rows_of(data=12288), d_residual=rows_of(data=16384), d_x=rows_of(data=20480), rstd=FAKE,
                gain=FAKE, d_gain=24576, dropout=None, gain_dtype=0, d_gain_dtype=0, rows=4, width=64, accumulate=0, reserved=0)
    call = lambda ws=FAKE, size=1 << 30, **k: L.sr_add_norm_grad(sr.NormGradRows(**{**good, **k}), ws, size, None)
    need = sr.norm_grad_workspace(4, 64)
    none = rows_of(data=None)
    for r in (L.sr_add_norm_grad(None, FAKE, 1 << 30, None), call(rows=-1), call(width=0), call(ws=None), call(ws=FAKE + 4), call(size=need - 1), call(rstd=None),
              call(rstd=FAKE + 2), call(gain=None), call(gain=FAKE + 1), call(gain_dtype=2), call(d_gain_dtype=2), call(d_gain=24578), call(d_out=none), call(total=none),
              call(d_out=rows_of(dtype=1)), call(d_out=rows_of(dtype=4)), call(d_total=rows_of(data=12288, dtype=1)), call(d_residual=rows_of(data=16384, dtype=2)),
              call(d_x=rows_of(data=20480, dtype=1)), call(d_x=rows_of(data=20480, ld=1)), call(d_residual=none, d_x=none, d_gain=None),
              call(d_residual=rows_of(data=8192)), call(d_x=rows_of(data=8192)), call(d_x=rows_of(data=16384)), call(d_x=rows_of(data=12288)),
              call(d_residual=rows_of()), call(d_gain=FAKE), call(d_residual=rows_of(data=12288, ld=128)), call(d_x=rows_of(ld=128)), call(dropout=ctypes.pointer(mask_of(p=-1.0)))):
        assert r == sr.SR_E_ARG
    wide = {k: rows_of(data=v.data, ld=1 << 15) for k, v in good.items() if isinstance(v, sr.Rows)}
    assert call(width=16385, **wide) == sr.SR_E_LIMIT
    assert call(width=16384, rows=(1 << 31) - 1, **wide) == sr.SR_E_LIMIT
    assert call(width=1, rows=(1 << 31) - 1) == sr.SR_E_LIMIT


def test_the_binding_refuses_host_tensors_and_other_shapes():
    z = lambda *s, t=F32: torch.zeros(*s, dtype=t)
    tok = z(4, t=torch.int32)
    ws = z(1 << 20, t=torch.uint8)
    for call, text in (
            (lambda: sr.sr_embed(z(10, 8), tok, z(4, 8)), "device tensors"),
            (lambda: sr.sr_embed(z(10, 8), tok, z(4, 9)), "out"),
            (lambda: sr.sr_embed(z(10, 8), tok, z(4, 8, t=torch.float64)), "out"),
            (lambda: sr.sr_embed(z(80), tok, z(4, 8)), "table"),
            (lambda: sr.sr_embed(z(8, 10).t(), tok, z(4, 8)), "adjacent"),
            (lambda: sr.sr_embed_grad(z(4, 8), tok, z(10, 8), ws), "device tensors"),
            (lambda: sr.sr_embed_grad(z(5, 8), tok, z(10, 8), ws), "d_out"),
            (lambda: sr.sr_embed_grad(z(4, 8), tok, z(10, 8), ws[::2]), "workspace"),
            (lambda: sr.sr_dropout(z(4, 8), z(4, 8), sr.Dropout(0.1, 1)), "device tensors"),
            (lambda: sr.sr_dropout(z(4, 8), z(4, 8), sr.Dropout(0.1, 1), residual=z(4, 9)), "residual"),
            (lambda: sr.sr_dropout(z(4, 8), z(4, 8), 0.1), "a Dropout"),
            (lambda: sr.Dropout(1.0, 1), "p < 1"), (lambda: sr.Dropout(0.1, 1, step=z(1, t=torch.int64)), "step"),
            (lambda: sr.sr_add_norm(z(4, 8), z(8), z(4, 8)), "device tensors"),
            (lambda: sr.sr_add_norm(z(4, 8), z(9), z(4, 8)), "gain"),
            (lambda: sr.sr_add_norm(z(4, 8), z(8), z(4, 8, t=E4M3), scales=z(4, 2), scale_block=32), "scales|device"),
            (lambda: sr.sr_add_norm_grad(z(4, 8), z(4, 8), z(4), z(8), ws, d_x=z(4, 8)), "device tensors"),
            (lambda: sr.sr_add_norm_grad(z(4, 8), z(4, 8), z(5), z(8), ws, d_x=z(4, 8)), "rstd|device")):
        with pytest.raises(sr.SrError, match=text):
            call()


# ------------------------------------------------------------------------------------------------------------------
# embedding
# ------------------------------------------------------------------------------------------------------------------
def some_tokens(gen, n, vocab, hot=0.0, outside=0.0):
    t = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    t = torch.where(torch.rand(n, generator=gen, device="cuda") < hot, vocab // 2, t)
    bad = torch.tensor([-1, vocab, 2 ** 31 - 1, -2 ** 31], device="cuda")[torch.randint(0, 4, (n,), generator=gen, device="cuda")]
    return torch.where(torch.rand(n, generator=gen, device="cuda") < outside, bad, t).int()


@pytest.mark.gpu
@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("width", WIDTHS + [30000])
def test_embed(types, width):
    T, O = types
    for n, vocab, pad, shift, scale in ((1, 5, 0, 0, 1.0), (131, 37, 3, 1, 0.75), (64, 1000, 8, 0, -1.5)):
        gen = rng(width + n)
        table, out = randn(gen, vocab, width, T, pad=pad, shift=shift), Field(n, width, O, pad, shift)
        tokens = some_tokens(gen, n, vocab, outside=0.2)
        sr.sr_embed(table.t, tokens, out.t, scale=scale)
        t = tokens.long()
        inside = (t >= 0) & (t < vocab)
        want = torch.where(inside[:, None], table.t.double()[t.clamp(0, vocab - 1)] * scale, 0.0)
        close(out.t, want, want.abs() * (U + ROUND[O]) + SMALLEST[O])
        out.check()


def grad_of_table(d, tokens, vocab, scale):
    """(gradient, sum of magnitudes, terms of every row) in 64 bits"""
    t = tokens.long()
    inside = (t >= 0) & (t < vocab)
    d, t = d.double()[inside], t[inside]
    zero = torch.zeros(vocab, d.shape[1], dtype=torch.float64, device="cuda")
    count = torch.zeros(vocab, dtype=torch.float64, device="cuda").index_add_(0, t, torch.ones(len(t), dtype=torch.float64, device="cuda"))
    return zero.index_add(0, t, d) * scale, zero.index_add(0, t, d.abs()) * abs(scale), count[:, None]


def check_embed_grad(gen, n, vocab, width, T, O, pad=0, shift=0, scale=1.0, accumulate=False, hot=0.0, outside=0.0, tokens=None):
    d, table = randn(gen, n, width, T, pad=pad, shift=shift), Field(vocab, width, O, pad, shift, fill=5.0)
    if tokens is None:
        tokens = some_tokens(gen, n, vocab, hot, outside)
    if accumulate:
        table.t.copy_(torch.randn(vocab, width, generator=gen, device="cuda"))
    old = table.t.double()
    ws = torch.full((sr.embed_grad_workspace(n, width) + 512,), 77, dtype=torch.uint8, device="cuda")
    sr.sr_embed_grad(d.t, tokens, table.t, ws[256:-256], scale=scale, accumulate=accumulate)
    want, size, m = grad_of_table(d.t, tokens, vocab, scale)
    tol = size * (m + 3) * U
    if accumulate:
        want, tol = want + old, tol + old.abs() * U
    close(table.t, want, tol + want.abs() * ROUND[O] + SMALLEST[O])
    table.check()
    if accumulate:
        assert torch.equal(table.t.double()[m[:, 0] == 0], old[m[:, 0] == 0])
    else:
        assert bool((table.t[m[:, 0] == 0] == 0).all())
    assert bool((ws[:256] == 77).all()) and bool((ws[-256:] == 77).all())
    return table.t


@pytest.mark.gpu
@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("width", WIDTHS)
def test_embed_grad(types, width):
    for k, (n, vocab) in enumerate(((1, 3), (131, 37), (64, 1000), (700, 2))):
        gen = rng(width + n)
        check_embed_grad(gen, n, vocab, width, *types, pad=(0, 3, 8, 1)[k], shift=k % 2, scale=(1.0, -0.5, 2.0, 0.25)[k], accumulate=k % 2 == 1,
                         hot=0.3 if k == 1 else 0.0, outside=0.2)


@pytest.mark.gpu
@pytest.mark.parametrize("types", [(BF16, F32), (F16, F16)])
@pytest.mark.parametrize("n", [0, 1, 15, 16, 17, 63, 64, 65, 255, 256, 257, 1023, 1024, 1025, 2047, 2048, 2049, 4096, 4097, 8192, 8193, 16385, 20000])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_grad_of_any_number_of_tokens(types, n, accumulate):
    """One token of all, halves of them one token, every token its own; padding alone."""
    for k, (vocab, hot, outside) in enumerate(((300, 0.0, 0.1), (50, 0.5, 0.0), (1, 0.0, 0.0), (7, 0.0, 1.0), (n + 1, 0.0, 0.0))):
        gen = rng(n * 5 + k)
        tokens = torch.randperm(n, generator=gen, device="cuda").int() if k == 4 else None
        check_embed_grad(gen, n, vocab, 72, *types, accumulate=accumulate, hot=hot, outside=outside, tokens=tokens)


@pytest.mark.gpu
@pytest.mark.parametrize("n,width", [(70001, 64), (262144, 16), (100000, 260), (1 << 20, 8)])
def test_embed_grad_of_many_tokens(n, width):
    """Sums of whole batches in chunks: chains as long as the docstring says, and so exact."""
    gen = rng(n)
    tokens = some_tokens(gen, n, 40, hot=0.6, outside=0.05)
    d = randn(gen, n, width, BF16)
    table = torch.empty(40, width, device="cuda")
    sr.sr_embed_grad(d.t, tokens, table, torch.empty(sr.embed_grad_workspace(n, width), dtype=torch.uint8, device="cuda"))
    want, size, m = grad_of_table(d.t, tokens, 40, 1.0)
    slices = -(-width // 256)
    chunk = max(16, -(-n * slices // 8192) + 15)
    depth = min(n, chunk + n / chunk / 4 + 4)
    close(table, want, size * (depth + 3) * U + SMALLEST[F32])


@pytest.mark.gpu
@pytest.mark.parametrize("types", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("vocab,width,pad,shift", [(60000, 1031, 0, 0), (60000, 1031, 0, 1), (60001, 1031, 0, 3), (60000, 1031, 5, 1), (50000, 2048, 0, 0),
                                                   (700000, 64, 0, 7), (700000, 64, 8, 0), (3000000, 24, 1, 0)])
def test_embed_grad_of_large_tables(types, vocab, width, pad, shift):
    """Tables that are filled with zeros before the sums are written, at any address and distance of rows."""
    for n in (0, 1, 777, 9000):
        check_embed_grad(rng(vocab + n), n, vocab, width, *types, pad=pad, shift=shift, hot=0.3, outside=0.1)


@pytest.mark.gpu
@pytest.mark.parametrize("n,vocab,width,accumulate", [(200, 100, 64, False), (5000, 300, 72, False), (5000, 300, 72, True), (9001, 1000, 40, False), (30000, 50, 33, False),
                                                      (3000, 60000, 1031, False), (12000, 100000, 520, False)])
def test_embed_grad_in_graphs_that_run_beside_each_other(n, vocab, width, accumulate):
    """Two captured calls, a workspace each, replayed on two streams at once over tokens that change; each gives what an eager call does."""
    gen = rng(n)
    calls = []
    for k in range(2):
        tokens, d = some_tokens(gen, n, vocab, hot=0.4 * k, outside=0.1), torch.randn(n, width, generator=gen, device="cuda")
        table, ws = torch.zeros(vocab, width, device="cuda"), torch.empty(sr.embed_grad_workspace(n, width), dtype=torch.uint8, device="cuda")
        call = lambda t=tokens, d=d, table=table, ws=ws: sr.sr_embed_grad(d, t, table, ws, accumulate=accumulate)
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        calls.append((tokens, table, call, graph, torch.cuda.Stream()))
    for turn in range(3):
        want = []
        for tokens, table, call, graph, stream in calls:
            tokens.copy_(some_tokens(gen, n, vocab, hot=0.3 * turn, outside=0.1))
            table.fill_(1.0)
            call()
            want.append(table.clone())
            table.fill_(1.0)
        torch.cuda.synchronize()
        for tokens, table, call, graph, stream in calls:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for w, (tokens, table, call, graph, stream) in zip(want, calls):
            assert torch.equal(table, w)


@pytest.mark.gpu
@pytest.mark.parametrize("n,hot", [(300, 0.2), (5000, 0.5), (20000, 0.9)])
def test_embed_grad_is_the_same_every_time(n, hot):
    gen = rng(n)
    tokens, d = some_tokens(gen, n, 100, hot=hot), randn(gen, n, 200, F32)
    ws = torch.empty(sr.embed_grad_workspace(n, 200), dtype=torch.uint8, device="cuda")
    first = None
    for k in range(4):
        table = torch.full((100, 200), float(k), device="cuda")
        ws.fill_(k * 85)
        sr.sr_embed_grad(d.t, tokens, table, ws)
        assert first is None or torch.equal(first, table)
        first = table


@pytest.mark.gpu
def test_embed_grad_is_that_of_differences():
    """(f(table + e) - f(table - e)) / 2 e of a linear function, through the lookup itself."""
    gen = rng(1)
    vocab, width, n = 9, 12, 40
    table, d = torch.randn(vocab, width, generator=gen, device="cuda"), torch.randn(n, width, generator=gen, device="cuda")
    tokens = some_tokens(gen, n, vocab, outside=0.1)
    grad, out = torch.empty_like(table), torch.empty_like(d)
    sr.sr_embed_grad(d, tokens, grad, torch.empty(sr.embed_grad_workspace(n, width), dtype=torch.uint8, device="cuda"), scale=0.5)

    def f(t):
        sr.sr_embed(t, tokens, out, scale=0.5)
        return (out.double() * d.double()).sum().item()
    for at in ((0, 0), (3, 7), (8, 11)):
        e = torch.zeros_like(table)
        e[at] = 1.0
        # linear, and no entry is rounded by more than u max|table + e|
        assert (f(table + e) - f(table - e)) / 2 == pytest.approx(grad[at].item(), abs=40 * 3 * 2 * U * 4 * 4)


@pytest.mark.gpu
def test_embed_grad_keeps_infinities_to_their_tokens():
    d = torch.ones(6, 16, device="cuda")
    d[0], d[1], d[5] = math.inf, math.nan, math.inf
    tokens = torch.tensor([1, 2, 3, 3, 0, 9], dtype=torch.int32, device="cuda")
    table = torch.empty(5, 16, device="cuda")
    sr.sr_embed_grad(d, tokens, table, torch.empty(sr.embed_grad_workspace(6, 16), dtype=torch.uint8, device="cuda"))
    assert bool((table[0] == 1).all()) and bool((table[1] == math.inf).all()) and bool(table[2].isnan().all()) and bool((table[3] == 2).all())
    assert bool((table[4] == 0).all())


# ------------------------------------------------------------------------------------------------------------------
# dropout
# ------------------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("width", WIDTHS + [18944, 33333])
def test_dropout(types, width):
    T, O = types
    for rows, pad, shift, p, add, first in ((1, 0, 0, 0.1, False, 0), (37, 3, 1, 0.5, True, 10 ** 12), (6, 8, 0, 0.0, True, 3), (5, 1, 0, 0.999, False, 7)):
        gen = rng(width + rows)
        O2 = O if add else T
        x, base, out = randn(gen, rows, width, T, pad=pad, shift=shift), randn(gen, rows, width, O2, pad=pad, shift=shift), Field(rows, width, O2, pad, shift)
        drop = sr.Dropout(p, 2 ** 63 + 11, mask=2 ** 40 + 5, first_row=first)
        sr.sr_dropout(x.t, out.t, drop, residual=base.t if add else None)
        k = torch.from_numpy(kept(rows, width, p, 2 ** 63 + 11, 2 ** 40 + 5, first)).cuda()
        part = x.t.double() * k
        want = part + base.t.double() if add else part
        close(out.t, want, part.abs() * 2 * U + (part.abs() + (base.t.double().abs() if add else 0)) * U + want.abs() * ROUND[O2] + SMALLEST[O2])
        out.check()
        if not add:
            assert torch.equal(out.t != 0, (k > 0) & (x.t != 0))
        # in the place of its inputs
        keep = out.t.clone()
        if add:
            sr.sr_dropout(x.t, base.t, drop, residual=base.t)
            assert torch.equal(base.t, keep)
            base.check()
        elif T == O2:
            sr.sr_dropout(x.t, x.t, drop)
            assert torch.equal(x.t, keep)
            x.check()


@pytest.mark.gpu
def test_dropped_elements_are_zeros_whatever_they_held():
    x = torch.full((50, 37), math.nan, device="cuda")
    x[:, 1::2] = math.inf
    out = torch.empty_like(x)
    sr.sr_dropout(x, out, sr.Dropout(0.5, 4))
    k = torch.from_numpy(kept(50, 37, 0.5, 4)).cuda() > 0
    assert bool((out[~k] == 0).all()) and torch.equal(out[k].isnan(), x[k].isnan()) and bool((out[k & ~x.isnan()] == math.inf).all())


@pytest.mark.gpu
def test_a_batch_in_parts_has_the_mask_of_the_whole():
    x = torch.ones(101, 203, device="cuda")
    whole, parts = torch.empty_like(x), torch.empty_like(x)
    step = torch.full((1,), 9, dtype=torch.int64, device="cuda")
    sr.sr_dropout(x, whole, sr.Dropout(0.3, 5, mask=2, step=step))
    for a, b in ((0, 1), (1, 40), (40, 101)):
        sr.sr_dropout(x[a:b], parts[a:b], sr.Dropout(0.3, 5, mask=2, first_row=a, step=step))
    assert torch.equal(whole, parts) and torch.equal(whole > 0, torch.from_numpy(kept(101, 203, 0.3, 5, 2, 0, 9)).cuda() > 0)


# ------------------------------------------------------------------------------------------------------------------
# residual + norm
# ------------------------------------------------------------------------------------------------------------------
def check_norm(gen, rows, width, T, R, out_type=None, gain_type=None, block=0, p=0.0, pad=0, shift=0, has_x=True, in_place=False, eps=1e-6, std=1.0,
               has_total=True, has_rstd=True):
    out_type = out_type or T
    x, base = randn(gen, rows, width, T, pad=pad, shift=shift), randn(gen, rows, width, R, std, pad=pad, shift=shift)
    gain = (1 + 0.5 * torch.randn(width, generator=gen, device="cuda")).to(gain_type or T)
    out = Field(rows, width, F32 if out_type in LARGEST else out_type, pad, shift)
    if out_type in LARGEST:
        out.buf = out.buf.to(out_type)
        out.t = out.buf[shift:shift + rows * (width + pad)].view(rows, width + pad)[:, :width]
    total = base if in_place else Field(rows, width, R, pad, shift)
    before = base.t.double()
    blocks = -(-width // block) if block else 1
    scales = torch.full((rows, blocks), -7.0, device="cuda") if out_type in LARGEST else None
    rstd = torch.full((rows,), -7.0, device="cuda")
    drop = sr.Dropout(p, 99, mask=3, first_row=5) if p else None
    sr.sr_add_norm(base.t, gain, out.t, x=x.t if has_x else None, total=total.t if has_total else None, rstd=rstd if has_rstd else None, scales=scales,
                   scale_block=block, dropout=drop, eps=eps)
    part = x.t.double() if has_x else torch.zeros_like(before)
    if p and has_x:
        part = part * torch.from_numpy(kept(rows, width, p, 99, 3, 5)).cuda()
    want = before + part
    if has_total:
        close(total.t, want, part.abs() * 2 * U + (before.abs() + part.abs()) * U + want.abs() * ROUND[R] + SMALLEST[R])
        total.check()
        h = total.t.double()
    else:
        h = want.float().to(R).double()              # a rounding may fall to the other side: the caller leaves room for it
    r = 1 / (h.square().mean(1) + eps).sqrt()
    if has_rstd:
        close(rstd, r, r * 32 * U)
    y = h * r[:, None] * gain.double()
    loose = 0.0 if has_total else 2 * ROUND[R]
    if out_type not in LARGEST:
        close(out.t, y, y.abs() * (34 * U + ROUND[out_type] + loose) + SMALLEST[out_type])
    else:
        wide = torch.cat([y.abs(), y.new_zeros(rows, blocks * (block or width) - width)], 1).view(rows, blocks, -1)
        s = (wide.amax(2) / LARGEST[out_type]).clamp(min=2.0 ** -126)
        close(scales, s, s * 36 * U)
        v = y / scales.double().repeat_interleave(block or width, 1)[:, :width]
        close(out.t.float(), v, v.abs() * (ROUND[out_type] + 72 * U) + SMALLEST[out_type])
        assert bool((out.buf.float()[~out.at] == 3.0).all())
    if out_type not in LARGEST:
        out.check()
    return total, rstd, gain, out


@pytest.mark.gpu
@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("width", WIDTHS)
def test_add_norm(types, width):
    for k, (rows, pad, shift) in enumerate(((1, 0, 0), (5, 3, 1), (131, 8, 0))):
        check_norm(rng(width + rows), rows, width, *types, pad=pad, shift=shift, p=(0.0, 0.3, 0.1)[k], gain_type=(None, F32, None)[k], in_place=k == 2)


@pytest.mark.gpu
@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("width", [1, 7, 8, 33, 256, 1031, 4100])
def test_add_norm_with_parts_left_out(types, width):
    check_norm(rng(width), 7, width, *types, has_x=False, pad=1)
    check_norm(rng(width), 7, width, *types, has_total=False, has_rstd=False)
    check_norm(rng(width), 7, width, *types, has_x=False, has_total=False, gain_type=F32)


@pytest.mark.gpu
@pytest.mark.parametrize("out_type", [E4M3, E5M2])
@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("width", [1, 5, 8, 31, 32, 33, 63, 100, 128, 129, 256, 513, 1031, 2048, 3584, 4097, 8192, 16384])
def test_add_norm_in_8_bits(out_type, types, width):
    for k, block in enumerate((0, 32, 64, 128)):
        check_norm(rng(width + block), 6 + k, width, *types, out_type=out_type, block=block, pad=k, shift=k % 2, p=0.2 if k == 1 else 0.0)


@pytest.mark.gpu
def test_8_bit_output_of_every_size_of_value():
    """Rows of one large value and small ones: subnormal codes, and zeros below half the smallest."""
    for out_type in (E4M3, E5M2):
        h = torch.logspace(0, -9, 512, device="cuda")[None].repeat(3, 1) * torch.tensor([1.0, -1.0], device="cuda").repeat(256)
        h[1] *= 1e-6
        h[2] *= 1e6
        gain, out, scales = torch.ones(512, device="cuda"), torch.empty(3, 512, dtype=out_type, device="cuda"), torch.empty(3, device="cuda")
        sr.sr_add_norm(h, gain, out, scales=scales, eps=0.0)
        y = h.double() / h.double().square().mean(1, keepdim=True).sqrt()
        v = y / scales.double()[:, None]
        close(out.float(), v, v.abs() * (ROUND[out_type] + 72 * U) + SMALLEST[out_type])
        assert bool((out.float()[:, 0].abs() == LARGEST[out_type]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("width", [6, 256, 1031, 3584])
def test_rows_of_zeros_and_rows_that_are_not_finite(width):
    """Each row for itself: zeros stay zeros, what is not finite does not leave its row."""
    h = torch.randn(6, width, generator=rng(3), device="cuda")
    h[1], h[2, 3], h[3, 2], h[4] = 0.0, math.nan, math.inf, 3e38
    gain = torch.ones(width, device="cuda")
    out, rstd = torch.empty_like(h), torch.empty(6, device="cuda")
    sr.sr_add_norm(h, gain, out, rstd=rstd, eps=1e-6)
    for r in (0, 5):
        y = h[r].double() / (h[r].double().square().mean() + 1e-6).sqrt()
        close(out[r], y, y.abs() * 35 * U + 1e-37)
    assert bool((out[1] == 0).all()) and rstd[1].item() == pytest.approx(1e3, rel=8 * U)
    assert bool(out[2].isnan().all()) and rstd[3].item() == 0 and bool(out[3, 2].isnan()) and bool((out[3][torch.arange(width, device="cuda") != 2] == 0).all())
    assert rstd[4].item() == 0 and bool((out[4] == 0).all())
    codes, scales = torch.empty(6, width, dtype=E4M3, device="cuda"), torch.empty(6, device="cuda")
    sr.sr_add_norm(h, gain, codes, scales=scales, eps=1e-6)
    assert bool((codes[1].float() == 0).all()) and scales[1].item() == 2.0 ** -126 and bool(codes[2].float().isnan().all())
    assert bool(codes[3, 2].float().isnan()) and scales[3].item() == 2.0 ** -126


def check_norm_grad(gen, rows, width, T, R, gain_type=None, grad_type=F32, p=0.0, pad=0, shift=0, has_d_total=True, in_place=False, accumulate=False,
                    wanted=("d_residual", "d_x", "d_gain"), std=1.0):
    dy, h = randn(gen, rows, width, T, pad=pad, shift=shift), randn(gen, rows, width, R, std, pad=pad, shift=shift)
    dt = randn(gen, rows, width, R, pad=pad, shift=shift) if has_d_total else None
    gain = (1 + 0.5 * torch.randn(width, generator=gen, device="cuda")).to(gain_type or T)
    rstd = (h.t.double().square().mean(1) + 1e-6).rsqrt().float()
    y, t = dy.t.double(), torch.zeros(rows, width, dtype=torch.float64, device="cuda") if dt is None else dt.t.double()
    to_r = dt if in_place else Field(rows, width, R, pad, shift)
    to_x = dy if in_place else Field(rows, width, T, pad, shift)
    d_gain = torch.randn(width, generator=gen, device="cuda").to(grad_type)
    old = d_gain.double() if accumulate else torch.zeros(width, dtype=torch.float64, device="cuda")
    ws = torch.full((sr.norm_grad_workspace(rows, width) + 512,), 77, dtype=torch.uint8, device="cuda")
    sr.sr_add_norm_grad(dy.t, h.t, rstd, gain, ws[256:-256] if "d_gain" in wanted else None, d_total=None if dt is None else dt.t,
                        d_residual=to_r.t if "d_residual" in wanted else None, d_x=to_x.t if "d_x" in wanted else None,
                        d_gain=d_gain if "d_gain" in wanted else None, dropout=sr.Dropout(p, 99, mask=3, first_row=5) if p else None, accumulate=accumulate)
    r = rstd.double()[:, None]
    n, g = h.t.double() * r, y * gain.double()
    c, size = (g * n).mean(1, keepdim=True), (g * n).abs().mean(1, keepdim=True)
    dh = r * (g - n * c) + t
    tol = U * (r * (5 * g.abs() + n.abs() * (6 * c.abs() + 64 * size)) + 2 * t.abs() + 2 * dh.abs())
    if "d_residual" in wanted:
        close(to_r.t, dh, tol + dh.abs() * ROUND[R] + SMALLEST[R])
        to_r.check()
    if "d_x" in wanted:
        k = torch.from_numpy(kept(rows, width, p, 99, 3, 5)).cuda() if p else 1.0
        close(to_x.t, dh * k, (tol + 2 * U * dh.abs()) * k + (dh * k).abs() * ROUND[T] + SMALLEST[T])
        to_x.check()
    if "d_gain" in wanted:
        want = (y * n).sum(0) + old
        close(d_gain, want, (rows / 512 + 100) * U * (y * n).abs().sum(0) + U * old.abs() + want.abs() * ROUND[grad_type] + SMALLEST[grad_type])
        assert bool((ws[:256] == 77).all()) and bool((ws[-256:] == 77).all())


@pytest.mark.gpu
@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("width", WIDTHS)
def test_add_norm_grad(types, width):
    T, R = types
    for k, (rows, pad, shift) in enumerate(((1, 0, 0), (5, 3, 1), (131, 8, 0))):
        check_norm_grad(rng(width + rows), rows, width, T, R, pad=pad, shift=shift, p=(0.0, 0.3, 0.1)[k], gain_type=(None, F32, None)[k],
                        grad_type=(F32, T, F32)[k], in_place=k == 2, accumulate=k == 1)


@pytest.mark.gpu
@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("width", [1, 7, 8, 33, 256, 1031, 4100])
def test_add_norm_grad_with_parts_left_out(types, width):
    for wanted in (("d_residual",), ("d_x",), ("d_gain",), ("d_residual", "d_gain")):
        check_norm_grad(rng(width), 9, width, *types, has_d_total="d_gain" in wanted, wanted=wanted, pad=1, p=0.2)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width", [(2047, 24), (2048, 500), (2049, 8), (8193, 64), (5000, 257), (3000, 2050), (1025, 4100), (700, 16384)])
def test_add_norm_grad_of_many_rows(rows, width):
    check_norm_grad(rng(rows), rows, width, BF16, F32, p=0.1)
    check_norm_grad(rng(rows), rows, width, F16, F16, grad_type=F16)


@pytest.mark.gpu
def test_no_rows():
    e = torch.empty(0, 24, device="cuda")
    gain, d_gain = torch.ones(24, device="cuda"), torch.full((24,), 3.0, device="cuda")
    ws = torch.empty(sr.norm_grad_workspace(0, 24), dtype=torch.uint8, device="cuda")
    sr.sr_add_norm(e, gain, torch.empty_like(e), x=e.clone(), total=torch.empty_like(e), rstd=e[:, 0].contiguous())
    sr.sr_dropout(e, torch.empty_like(e), sr.Dropout(0.1, 1))
    sr.sr_embed(torch.ones(3, 24, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), e)
    sr.sr_add_norm_grad(e, e, e[:, 0].contiguous(), gain, None, d_x=torch.empty_like(e))
    sr.sr_add_norm_grad(e, e, e[:, 0].contiguous(), gain, ws, d_gain=d_gain, accumulate=True)
    assert bool((d_gain == 3).all())
    sr.sr_add_norm_grad(e, e, e[:, 0].contiguous(), gain, ws, d_gain=d_gain)
    assert bool((d_gain == 0).all())


@pytest.mark.gpu
def test_norm_gradients_are_those_of_differences():
    """Central differences of the forward operator itself, in directions: f = <out, v> + <total, w>.  The third derivative of a row's norm is at most a few
    over the cube of its root mean square (1 here), steps are 2^-7, so that differences are good to 2^-14 |v| plus rounding over the step."""
    gen = rng(8)
    rows, width, e = 5, 40, 2.0 ** -7
    N = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, base, gain, v, w = N(rows, width), N(rows, width), 1 + 0.2 * N(width), N(rows, width), N(rows, width)
    drop = sr.Dropout(0.25, 3)

    def f(x, base, gain):
        out, total, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda")
        sr.sr_add_norm(base, gain, out, x=x, total=total, rstd=rstd, dropout=drop)
        return ((out.double() * v).sum() + (total.double() * w).sum()).item(), total, rstd
    _, total, rstd = f(x, base, gain)
    dr, dx, dg = torch.empty_like(x), torch.empty_like(x), torch.empty_like(gain)
    sr.sr_add_norm_grad(v, total, rstd, gain, torch.empty(sr.norm_grad_workspace(rows, width), dtype=torch.uint8, device="cuda"), d_total=w, d_residual=dr,
                        d_x=dx, d_gain=dg, dropout=drop)
    for which, grad in ((0, dx), (1, dr), (2, dg)):
        for _ in range(3):
            args = [x, base, gain]
            way = N(*args[which].shape)
            way /= way.norm()
            at = lambda s: [a + s * e * way if i == which else a for i, a in enumerate(args)]
            slope = (f(*at(1))[0] - f(*at(-1))[0]) / (2 * e)
            assert slope == pytest.approx((grad.double() * way).sum().item(), abs=2 ** -14 * v.norm().item() + 200 * 40 * U / e)


# ------------------------------------------------------------------------------------------------------------------
# far offsets, streams, graphs, all of them together
# ------------------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
def test_rows_that_lie_further_apart_than_32_bits_reach():
    """2100 rows, 2^20 elements apart: the last begin beyond 2^31 elements."""
    rows, width, far = 2100, 40, 1 << 20
    gen = rng(2)
    room = lambda: torch.empty((rows - 1) * far + width, dtype=BF16, device="cuda").as_strided((rows, width), (far, 1))
    x, y, z, w = (room() for _ in range(4))
    near = lambda: torch.randn(rows, width, generator=gen, device="cuda").bfloat16()
    a, b = near(), near()
    x.copy_(a)
    y.copy_(b)
    tokens = torch.randint(0, rows, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    gain, rstd = torch.ones(width, dtype=BF16, device="cuda"), torch.empty(rows, device="cuda")
    drop = sr.Dropout(0.2, 1)
    e = torch.empty_like(a)
    sr.sr_embed(x, tokens, z)
    sr.sr_embed(a, tokens, e)
    assert torch.equal(z, e)
    sr.sr_dropout(x, z, drop, residual=y)
    sr.sr_dropout(a, e, drop, residual=b)
    assert torch.equal(z, e)
    t = torch.empty_like(a)
    sr.sr_add_norm(y, gain, w, x=x, total=z, rstd=rstd, dropout=drop)
    sr.sr_add_norm(b, gain, e, x=a, total=t, rstd=rstd, dropout=drop)
    assert torch.equal(w, e) and torch.equal(z, t)
    sr.sr_add_norm_grad(x, z, rstd, gain, None, d_total=y, d_residual=w, dropout=drop)
    sr.sr_add_norm_grad(a, t, rstd, gain, None, d_total=b, d_residual=e, dropout=drop)
    assert torch.equal(w, e)
    ws = torch.empty(sr.embed_grad_workspace(rows, width), dtype=torch.uint8, device="cuda")
    sr.sr_embed_grad(x, tokens, w, ws)
    sr.sr_embed_grad(a, tokens, e, ws)
    assert torch.equal(w, e)


@pytest.mark.gpu
def test_a_stream_that_is_named():
    """The calls go where `stream` says: work of that stream before them is seen, and the current stream does not wait."""
    gen = rng(6)
    n, width, vocab = 3000, 320, 500
    d, tokens = torch.randn(n, width, generator=gen, device="cuda"), some_tokens(gen, n, vocab)
    gain, drop = torch.randn(width, generator=gen, device="cuda"), sr.Dropout(0.3, 2)
    ws = torch.empty(max(sr.embed_grad_workspace(n, width), sr.norm_grad_workspace(n, width)), dtype=torch.uint8, device="cuda")
    E = lambda *s: torch.zeros(*s, device="cuda")

    def run(x, stream):
        out, total, rstd, dx, dg, table, rows = E(n, width), E(n, width), E(n), E(n, width), E(width), E(vocab, width), E(n, width)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            x.mul_(2.0)
        sr.sr_dropout(x, x, drop, stream=stream)
        sr.sr_add_norm(d, gain, out, x=x, total=total, rstd=rstd, stream=stream)
        sr.sr_add_norm_grad(x, total, rstd, gain, ws, d_x=dx, d_gain=dg, stream=stream.cuda_stream)
        sr.sr_embed_grad(dx, tokens, table, ws, stream=stream)
        sr.sr_embed(table, tokens, rows, stream=stream)
        stream.synchronize()
        return out, dg, table, rows
    x = torch.randn(n, width, generator=gen, device="cuda")
    want = run(x.clone(), torch.cuda.current_stream())
    got = run(x.clone(), torch.cuda.Stream())
    assert all(torch.equal(p, q) for p, q in zip(got, want))


class Block:
    """embedding -> dropout -> [residual + norm -> product] twice -> norm, and back, with every buffer made beforehand"""

    def __init__(self, dtype, n=150, vocab=61, width=96, seed=0, outside=0.1):
        gen = rng(seed)
        N = lambda *s: 0.3 * torch.randn(*s, generator=gen, device="cuda")
        self.dtype, self.n, self.vocab, self.width = dtype, n, vocab, width
        self.table, self.W = N(vocab, width).to(dtype), [N(width, width).to(dtype) for _ in range(2)]
        self.gain = [(1 + N(width)).to(dtype) for _ in range(3)]
        self.tokens = some_tokens(gen, n, vocab, hot=0.3, outside=outside)
        self.d_last = N(n, width).to(dtype)
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        E = lambda t, *s: torch.empty(*s, dtype=t, device="cuda")
        self.h = [E(F32, n, width) for _ in range(4)]
        self.y, self.b = [E(dtype, n, width) for _ in range(3)], [E(dtype, n, width) for _ in range(3)]
        self.rstd = [E(F32, n) for _ in range(3)]
        self.dh, self.db = [E(F32, n, width) for _ in range(3)], [E(dtype, n, width) for _ in range(3)]
        self.dy = [E(dtype, n, width) for _ in range(3)]
        self.d_gain, self.dW = [E(F32, width) for _ in range(3)], [E(dtype, width, width) for _ in range(2)]
        self.d_table = E(F32, vocab, width)
        self.ws = E(torch.uint8, max(sr.embed_grad_workspace(n, width), sr.norm_grad_workspace(n, width)))
        self.drop = [sr.Dropout(0.1, 7, mask=k, step=self.step) for k in range(4)]

    def run(self):
        sr.sr_embed(self.table, self.tokens, self.h[3], scale=2.0)
        sr.sr_dropout(self.h[3], self.h[0], self.drop[3])
        for k in range(3):
            before = self.h[max(k - 1, 0)]
            sr.sr_add_norm(before, self.gain[k], self.y[k], x=self.b[k - 1] if k else None, total=self.h[k] if k else None, rstd=self.rstd[k],
                           dropout=self.drop[k] if k else None)
            if k < 2:
                torch.mm(self.y[k], self.W[k], out=self.b[k])
        dy, dt = self.d_last, None
        for k in (2, 1, 0):
            sr.sr_add_norm_grad(dy, self.h[k], self.rstd[k], self.gain[k], self.ws, d_total=dt, d_residual=self.dh[k], d_x=self.db[k] if k else None,
                                d_gain=self.d_gain[k], dropout=self.drop[k] if k else None)
            dt = self.dh[k]
            if k:
                torch.mm(self.y[k - 1].t(), self.db[k], out=self.dW[k - 1])
                torch.mm(self.db[k], self.W[k - 1].t().contiguous(), out=self.dy[k - 1])
                dy = self.dy[k - 1]
        sr.sr_dropout(dt, self.h[3], self.drop[3])
        sr.sr_embed_grad(self.h[3], self.tokens, self.d_table, self.ws, scale=2.0)
        return [*self.d_gain, *self.dW, self.d_table, self.y[2]]

    def reference(self):
        leaf = lambda t: t.double().cpu().requires_grad_(True)
        table, W, gain = leaf(self.table), [leaf(w) for w in self.W], [leaf(g) for g in self.gain]
        t = self.tokens.long().cpu()
        inside = ((t >= 0) & (t < self.vocab)).double()[:, None]
        step = int(self.step.item())
        keep = [torch.from_numpy(kept(self.n, self.width, 0.1, 7, k, step=step)) for k in range(4)]
        h = table[t.clamp(0, self.vocab - 1)] * inside * 2.0 * keep[3]
        branches = []
        for k in range(3):
            if k:
                branches.append(y @ W[k - 1])
                h = h + branches[-1] * keep[k]
            y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6) * gain[k]
        *grads, d1, d2 = torch.autograd.grad((y * self.d_last.double().cpu()).sum(), [*gain, *W, table, *branches])
        self.largest_branch_gradient = max(d1.abs().max().item(), d2.abs().max().item())
        return [*grads, y.detach()]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,outside", [(F32, 0.1), (BF16, 0.1), (F16, 0.1), (F16, 0.0)])
def test_a_training_pass_of_all_of_them(dtype, outside):
    """Against differentiation in 64 bits on the CPU.  Seven roundings of 16-bit tensors lie between (y, b, db, dy twice): 2-norms within 32 half units; in
    single precision the products' sums of 96 and 150 terms add theirs.

    A token outside the vocabulary has a row of zeros, whose rstd is 1 / sqrt(eps) = 1000 at each norm: gradients of its branches reach 0.3 * 1000 * (0.3
    sqrt(96) = 3) * 1000 = 9e5, which half precision does not hold.  Infinite rows times zeros then make NaN of the gains' and products' gradients;
    the table's gradient leaves those rows out, and the output does not depend on gradients: these two are compared there."""
    b = Block(dtype, outside=outside)
    b.step.fill_(4)
    got, want = b.run(), b.reference()
    if dtype == F16 and outside:
        assert b.largest_branch_gradient > torch.finfo(F16).max
        got, want = got[-2:], want[-2:]
    for g, w in zip(got, want):
        off = (g.double().cpu() - w).norm() / w.norm()
        assert off <= (32 * ROUND[dtype] if dtype != F32 else 200 * U)


@pytest.mark.gpu
def test_a_training_pass_in_a_graph_and_on_another_stream():
    """Every replay draws the masks of its own step, and gives what the eager pass gives, bit for bit."""
    b = Block(BF16, seed=3)
    want = []
    for step in range(4):
        b.step.fill_(step)
        want.append([t.clone() for t in b.run()])
    assert not torch.equal(want[0][-1], want[1][-1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [t.clone() for t in b.run()]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want[3]))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = b.run()
    for turn in range(2):
        for step in range(4):
            b.step.fill_(step)
            for t in out:
                t.zero_()
            b.ws.fill_(turn * 255)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(out, want[step]))
    b.step.fill_(1)
    assert all(torch.equal(p, q) for p, q in zip(b.run(), want[1]))


@pytest.mark.gpu
@pytest.mark.parametrize("dropout,norm", [(0.0, False), (0.25, False), (0.0, True), (0.25, True)])
def test_gradients_of_the_policy_step_s_adapter(dropout, norm):
    """Against differentiation in 64 bits, at the second update's mask.  A chain of five operators in single precision, products of 1024 terms among them:
    2-norms within 2000 u."""
    from paper_2605_05802_amd.policy_step import SHAPE, Adapter
    gen = rng(4)
    rows, rank = 300, 16
    a = Adapter(rank, 3, dropout, norm)
    a.step.fill_(1)
    a.B.copy_(torch.randn(rank, SHAPE.vocab, generator=gen, device="cuda"))
    if norm:
        a.gain.copy_(1 + 0.3 * torch.randn(rank, generator=gen, device="cuda"))
    before = torch.randint(0, 40, (rows,), generator=gen, device="cuda")
    base, d = torch.randn(rows, SHAPE.vocab, generator=gen, device="cuda"), torch.randn(rows, SHAPE.vocab, generator=gen, device="cuda")
    logits = a.logits(base, before)
    got = a.gradients(d, before)
    leaves = [w.double().requires_grad_(True) for w in a.weights]
    x = leaves[0][before]
    if norm:
        x = x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-6) * leaves[3]
    if dropout:
        x = x * torch.from_numpy(kept(rows, rank, dropout, 3, step=1)).cuda()
    want = base.double() + x @ leaves[1] + leaves[2]
    for g, w in zip([logits, *got], [want.detach(), *torch.autograd.grad((want * d.double()).sum(), leaves)]):
        assert (g.double() - w).norm() <= 2000 * U * w.norm()


@pytest.mark.gpu
def test_the_policy_step_runs_with_norm_and_dropout():
    from paper_2605_05802_amd.policy_step import train
    losses, pair_losses, norms = train(groups=3, G=4, updates=2, pair_updates=1, dropout=0.1, norm=True)
    assert len(losses) == 2 and all(math.isfinite(x) for x in [*losses, *pair_losses, *norms])
