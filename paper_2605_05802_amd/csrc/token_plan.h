// Which kernels the losses over token rows run on, in plain C++ so that the rules can be evaluated without a GPU.
#pragma once
#include "plan.h"

namespace sr {

struct RowPlan {
    int waves;           // wavefronts per row or part: 1, 4 or 16
    int resident;        // > 0: vectors of a row that a thread of the register-resident kernel holds (at most kMostResident)
    int parts, elems;    // parts of a row that the streaming kernels give to workgroups of their own, and their elements
};
constexpr int kMostResident = 20, kMostOneWave = 8;

// Rows that are read twice
inline RowPlan plan_streamed_rows(int n_rows, int vocab, int elem_bytes) {
    const int per_vec = 16 / elem_bytes, vecs = ceil_div(vocab, per_vec);
    int parts = n_rows > 0 ? 1024 / n_rows : 1;
    const int most = vecs / 512;                         // 8 KiB each at least
    if (parts > most) parts = most;
    if (parts > 64) parts = 64;
    if (parts < 1) parts = 1;
    const int each = ceil_div(vecs, parts);
    return RowPlan{each <= 512 ? 1 : 4, 0, ceil_div(vecs, each), each * per_vec};
}

// Rows of the policy loss: held in registers between maximum and gradient where they fit
inline RowPlan plan_policy_rows(int n_rows, int vocab, int elem_bytes) {
    const int per_vec = 16 / elem_bytes, vecs = vocab / per_vec;
    const int waves = vecs <= 64 * kMostOneWave ? 1 : vecs <= 256 * kMostResident ? 4 : 16, each = ceil_div(vecs, 64 * waves);
    if (each > kMostResident || (waves == 16 && n_rows < 192)) return plan_streamed_rows(n_rows, vocab, elem_bytes);
    return RowPlan{waves, each > 0 ? each : 1, 1, ceil_div(vocab, per_vec) * per_vec};
}

}  // namespace sr
