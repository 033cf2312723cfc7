"""sr_add_norm without a branch: what it reads, and that it is the norm of the residual alone."""
import ctypes
import subprocess

import pytest
import torch

import paper_2605_05802_amd as sr
from test_decoder_rows import E4M3, F32, PAIRS, ROUND, SMALLEST, U, close, rng

SOURCE = """
#include "row_plan.h"
extern "C" void branch_rows(const void *x, long long ld, const void *gain, long long *out) {
    const sr::BranchRows b = sr::branch_rows(x, ld, gain);
    out[0] = (long long)b.data;
    out[1] = b.ld;
}
"""


def test_no_branch_is_looked_for_in_the_gain_alone(tmp_path):
    """Element c of row r is asked for at data + size of T * (r * ld + c): within the gain, of T or wider, for every row; a branch's in its rows."""
    from paper_2605_05802_amd.build import CSRC
    (tmp_path / "b.cpp").write_text(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + CSRC, str(tmp_path / "b.cpp"), "-o", str(tmp_path / "b.so")])
    at, out = ctypes.CDLL(str(tmp_path / "b.so")).branch_rows, (ctypes.c_longlong * 2)()
    at.argtypes = [ctypes.c_void_p, ctypes.c_longlong, ctypes.c_void_p, ctypes.c_void_p]
    for width in (1, 7, 256, 16384):
        for rows in (1, 2, 1 << 20):
            for size, gain_size in ((2, 2), (2, 4), (4, 4)):
                at(None, 77, 4096, out)
                first, last = out[0], out[0] + size * ((rows - 1) * out[1] + width)
                assert first == 4096 and last <= 4096 + gain_size * width
                at(8192, width + 3, 4096, out)
                assert list(out) == [8192, width + 3]


@pytest.mark.gpu
@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("width", [1, 5, 8, 33, 64, 250, 257, 1031, 3584, 4100, 16384])
@pytest.mark.parametrize("gain_single", [False, True])
def test_the_norm_of_a_residual_alone(types, width, gain_single):
    """The same bit for bit as with a branch of zeros, whatever lies between the residual's rows (NaN here), stored beside it and in its place, in 16 and in 8
    bits; and the formula in 64 bits (34 u + R: rstd 32 u, two products, one rounding)."""
    T, R = types
    gen = rng(width)
    rows, pad = 37, 5
    buf = torch.full((rows, width + pad), float("nan"), dtype=R, device="cuda")
    base = buf[:, :width]
    base.copy_(torch.randn(rows, width, generator=gen, device="cuda"))
    gain = (1 + 0.5 * torch.randn(width, generator=gen, device="cuda")).to(F32 if gain_single else T)
    zeros = torch.zeros(rows, width, dtype=T, device="cuda")
    drop = sr.Dropout(0.5, 3)
    for out_type in (T, E4M3):
        E = lambda t: torch.empty(rows, width, dtype=t, device="cuda")
        scales = [torch.empty(rows, device="cuda") if out_type is E4M3 else None for _ in range(3)]
        out, total, rstd = [E(out_type) for _ in range(3)], [E(R) for _ in range(2)], [torch.empty(rows, device="cuda") for _ in range(3)]
        sr.sr_add_norm(base, gain, out[0], x=zeros, total=total[0], rstd=rstd[0], scales=scales[0])
        # a mask has nothing to drop; the type of the branch that there is none of follows from the output, or the gain
        if out_type is E4M3 and gain_single and R is F32 and T is not F32:
            continue                                 # nothing names T: a call with T = fp32, another one
        sr.sr_add_norm(base, gain, out[1], total=total[1], rstd=rstd[1], scales=scales[1], dropout=drop)
        place = buf.clone()
        sr.sr_add_norm(place[:, :width], gain, out[2], total=place[:, :width], rstd=rstd[2], scales=scales[2])
        for k in (1, 2):
            assert torch.equal(out[0].view(torch.uint8), out[k].view(torch.uint8)) and torch.equal(rstd[0], rstd[k])
            assert scales[0] is None or torch.equal(scales[0], scales[k])
        assert torch.equal(total[1], base) and torch.equal(total[0], base) and torch.equal(place[:, :width], base)
        assert bool(place[:, width:].isnan().all()) and bool(buf[:, width:].isnan().all())
        if out_type is T:
            h = base.double()
            y = h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * gain.double()
            close(out[1], y, y.abs() * (34 * U + ROUND[T]) + SMALLEST[T])
