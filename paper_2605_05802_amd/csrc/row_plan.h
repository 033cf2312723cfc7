// Which kernels the row operators of training run on (embedding, residual + norm, dropout), in plain C++ so that the rules can be
// evaluated without a GPU.
#pragma once
#include <cstdint>

#include "plan.h"

namespace sr {

// A thread takes `per_vec` adjacent columns at a time: 16 bytes of the wider operand, so that a wavefront reads and writes whole lines
// of every operand.
// Rows narrower than a vector go column by column.
constexpr int row_vec(int width, bool single) { return width < 8 ? 1 : single ? 4 : 8; }

struct RowShape {
    int per_vec, vecs;       // vectors that a thread holds: 1, 2 or 4
    int threads;             // of a row
    bool wave;               // a wavefront a row, four rows to a workgroup, no barrier
};
constexpr int kMostNormWidth = 16384, kMostDropWidth = 1 << 30, kMostEmbedWidth = 1 << 20;

inline RowShape norm_shape(int width, bool single) {
    RowShape s{row_vec(width, single), 1, 64, true};
    const int n = ceil_div(width, s.per_vec);
    if (n <= 64) return s;
    s.wave = false;
    s.vecs = n <= 512 ? 1 : n <= 1024 ? 2 : 4;
    s.threads = round_up(ceil_div(n, s.vecs), 64);
    return s;
}

// Rows of the partial sums of a gain's gradient: workgroups (wavefronts, where each has a row of its own) that take rows in turn
constexpr int kMostNormParts = 2048;
inline int norm_grad_parts(int rows, const RowShape &s) {
    int parts = s.wave ? 2048 : 256 * (2048 / s.threads > 8 ? 8 : 2048 / s.threads);
    if (parts > kMostNormParts) parts = kMostNormParts;
    return rows < parts ? rows : parts;
}

// The gradient of an embedding: sorted tokens in spans of kSpanChunks chunks of `chunk`, a wavefront for 64 * per_vec columns of each
// chunk, a workgroup for those of a span
constexpr int kSpanChunks = 4;
constexpr int kMostTokens = 1 << 20;
struct EmbedGradPlan {
    int per_vec, slices, chunk, spans;
    int zero_rows;           // rows of zeros of a wavefront: about 8 KB of them, and at most 32
};
inline EmbedGradPlan embed_grad_plan(int n, int width, bool single, int table_bytes) {
    EmbedGradPlan p{};
    p.per_vec = row_vec(width, single);
    p.slices = ceil_div(ceil_div(width, p.per_vec), 64);
    const int64_t want = ((int64_t)n * p.slices + 8191) / 8192;
    p.chunk = want <= 16 ? 16 : round_up((int)(want < n ? want : n), 16);
    p.spans = ceil_div(n, kSpanChunks * p.chunk);
    const int rows = 8192 / (table_bytes * (width < 8192 ? width : 8192));
    p.zero_rows = rows < 1 ? 1 : rows > 32 ? 32 : rows;
    return p;
}

}  // namespace sr
