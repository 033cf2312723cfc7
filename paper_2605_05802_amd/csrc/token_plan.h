// Which kernels the losses over token rows run on, and the rows of a sequence, in plain C++ so that the rules can be evaluated without a GPU.
#pragma once
#include <cstdint>

#include "plan.h"

namespace sr {

struct RowPlan {
    int waves;           // wavefronts per row or part: 1, 4 or 16
    int resident;        // > 0: vectors of a row that a thread of the register-resident kernel holds (at most kMostResident)
    int parts, elems;    // parts of a row that the streaming kernels give to workgroups of their own, and their elements
    int grad_waves, grad_parts, grad_elems;    // the same of the gradient
};
constexpr int kMostResident = 20, kMostOneWave = 8;
// Many small parts in the order of the memory: 2400 rows of 152064 bf16 take 244 us in parts of 101 KB, 231 of 32 KB, 214 of 16 KB, 220 of 9 KB.
constexpr int kGradPartBytes = 16384;

// A row of `vecs` vectors in at most `parts` equal ones
inline void split_row(int vecs, int per_vec, int parts, int *n, int *elems) {
    if (parts < 1) parts = 1;
    const int each = vecs > 0 ? ceil_div(vecs, parts) : 1;
    *n = vecs > 0 ? ceil_div(vecs, each) : 1;
    *elems = each * per_vec;
}

// Rows that are read twice.  Few rows: parts for about 1024 workgroups (128 rows of 152064 fp32 in 8 parts 16 + 24 us for maximum and
// gradient, in 16 parts 16 + 27; where a kernel between them merges the parts, 16, 32 and 64 of them take it 1, 4 and 9 us longer).  Many: 8192 parts even out the end
// (2400 rows of 152064 bf16 in 3 parts each 129 us, in one 136; 1701 rows of 50021 in 4, 30 us, 34).
inline RowPlan plan_streamed_rows(int n_rows, int vocab, int elem_bytes) {
    const int per_vec = 16 / elem_bytes, vecs = ceil_div(vocab, per_vec);
    int parts = n_rows > 0 ? (n_rows < 1024 ? 1024 : 8192) / n_rows : 1;
    const int most = vecs / 512;                         // 8 KiB each at least
    if (parts > most) parts = most;
    if (parts > 64) parts = 64;
    RowPlan p{};
    split_row(vecs, per_vec, parts, &p.parts, &p.elems);
    p.waves = p.elems <= 512 * per_vec ? 1 : 4;
    const int grad_parts = n_rows < 1024 ? parts : vecs / (kGradPartBytes / 16);
    split_row(vecs, per_vec, grad_parts, &p.grad_parts, &p.grad_elems);
    p.grad_waves = p.grad_elems <= 512 * per_vec ? 1 : 4;
    return p;
}

// Rows of the policy loss: held in registers between maximum and gradient where they fit.  Rows of sixteen wavefronts are one to a
// compute unit: with few of them too few compute units work (rows of 152064 bf16: 64 take 27 us, streamed 18; 128, 28 and 24; 160, 28 and 29;
// 192, 31 and 35; of 75000 fp32: 112 take 23 and 21; 128, 24 and 25; 192, 29 and 34), and a few more than 256 wait for a second round
// (152064 bf16: 288 rows take 58 us, streamed 46; 352, 59 and 54; 448, 60 and 66; 75000 fp32: 51 and 46, 57 and 56, 61 and 71).
inline RowPlan plan_policy_rows(int n_rows, int vocab, int elem_bytes) {
    const int per_vec = 16 / elem_bytes, vecs = vocab / per_vec;
    const int waves = vecs <= 64 * kMostOneWave ? 1 : vecs <= 256 * kMostResident ? 4 : 16, each = ceil_div(vecs, 64 * waves);
    const bool uneven = n_rows < (elem_bytes == 2 ? 160 : 128) || (n_rows > 256 && n_rows <= 352);
    if (each > kMostResident || (waves == 16 && uneven)) return plan_streamed_rows(n_rows, vocab, elem_bytes);
    RowPlan p{waves, each > 0 ? each : 1};
    split_row(ceil_div(vocab, per_vec), per_vec, 1, &p.parts, &p.elems);
    return p;
}

// An entry of seq_start as an end of a range of rows, whatever it holds
constexpr int row_bound(int row, int n_rows) { return row < 0 ? 0 : row < n_rows ? row : n_rows; }
// The sequence of a row, or -1: the last one that begins at or before it, found among seq_start[0 .. n_seq - 1] whatever they hold; then one
// entry more is read, at most seq_start[n_seq].
constexpr int sequence_of(const int32_t *seq_start, int n_seq, int row) {
    int lo = -1, hi = n_seq;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (seq_start[mid] <= row) lo = mid;
        else hi = mid;
    }
    return lo >= 0 && row < seq_start[lo + 1] ? lo : -1;
}

// A launch has at most 2^32 - 1 threads
inline bool launches_fit(const RowPlan &p, int n_rows, bool grad) {
    auto threads = [](int64_t units, int waves) { return waves == 1 ? (units + 3) / 4 * 256 : units * 64 * waves; };
    if (p.resident && grad) return p.waves == 16 || threads(n_rows, p.waves) <= UINT32_MAX;
    return threads((int64_t)n_rows * p.parts, p.waves) <= UINT32_MAX &&
           (!grad || threads((int64_t)n_rows * p.grad_parts, p.grad_waves) <= UINT32_MAX);
}

}  // namespace sr
