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
    int lanes;               // 16, 32 or 64 where rows are a part of a wavefront or a whole one, 0 where they are workgroups
};
constexpr int kMostNormWidth = 16384, kMostDropWidth = 1 << 30, kMostEmbedWidth = 1 << 20;

// As few vectors a thread as 1024 threads allow, but two of four columns from 512 threads on.  (Gradients: 4096 rows of 3584 bf16 beside fp32 51.4 us, one
// each 52.8; 4096 rows of 4100 bf16 44 us in one each and 71 in two, 1500 of 16384 69 in two and 199 in four.  Registers of the gradient's kernels: one vector of
// four columns 64, two 104, one of eight 90, two of eight 121, without the next row's beside them, with which 23 would spill; four of four, beyond 8192 columns
// beside fp32, 128, and 8 spilled.)
inline RowShape norm_shape(int width, bool single) {
    RowShape s{row_vec(width, single), 1, 0, 0};
    const int n = ceil_div(width, s.per_vec);
    if (n <= 64) {
        s.threads = s.lanes = n <= 16 ? 16 : n <= 32 ? 32 : 64;
        return s;
    }
    s.vecs = single ? n <= 512 ? 1 : n <= 2048 ? 2 : 4 : n <= 1024 ? 1 : 2;
    s.threads = round_up(ceil_div(n, s.vecs), 64);
    return s;
}

// A norm without a branch loads its rows' worth of one all the same and leaves it out (the kernel has one form): the gain, again and again, which it
// reads anyway.  The residual's rows would do where the types are equal; elements of 16 bits beside a residual in single precision lie
// elsewhere in it, between its rows too.  (16384 rows of 3584 bf16 beside fp32, nothing stored but the norm: 66 us, by way of the residual 71.)
struct BranchRows {
    const void *data;
    int64_t ld;
};
inline BranchRows branch_rows(const void *x, int64_t ld, const void *gain) { return x ? BranchRows{x, ld} : BranchRows{gain, 0}; }

// Rows of the partial sums of a gain's gradient: workgroups (wavefronts, for rows that are not) that take rows in turn.  Workgroups: 1024
// threads to a compute unit, two at least, while each has two rows under way (16384 rows of 3584 bf16 beside fp32 186 us, with 2048 threads 191;
// 30000 of 1031 83 and 91).  Wavefronts: as many as fit (60000 rows of 256 bf16 beside fp32 52 us, with half of them
// 58, with a quarter 96).
// However many rows there are, the sums take 8 MB at most, or 512 rows of more than 4096 columns: a workgroup's 1024 / threads come to 8192 / width.
constexpr int kMostNormParts = 2048;
inline int norm_grad_parts(int rows, const RowShape &s) {
    const int each = 1024 / (s.lanes ? 64 : s.threads), some = rows < 4 * kMostNormParts ? rows : 4 * kMostNormParts;
    const int units = s.lanes ? ceil_div(some, 64 / s.lanes) : some;
    const int parts = s.lanes ? kMostNormParts : 256 * (each > 8 ? 8 : each < 2 ? 2 : each);
    return units < parts ? units : parts;
}

// Few rows: the gain's gradient from the rows themselves, by workgroups for sixteen columns in the same launch
// (with the call: 256 rows of 256 fp32 8.2 us instead of 10.9, 128 of 3584 bf16 beside fp32 8.2 and 10.7, 512 12.5 and 14.0, 128 of 16384 bf16 32 and 37;
// 512 of 8192 23.0 and 22.4)
inline bool gain_grad_direct(int rows, int width) { return rows <= 512 && (int64_t)rows * width <= 1 << 21; }

// Whether the gradient of a short list of tokens goes row by row of the table: not more workgroups than run at once
inline bool embed_few(int vocab, int slices) { return ((int64_t)vocab + 15) / 16 * slices <= 512; }

// Whether a whole table is filled with zeros before the sums are written over them: that saves 0.036 us a MB of the table and costs a second
// writing of up to n rows, 0.18 us a MB, and a launch, 6 us (152064 x 3584 fp32: 4096 tokens 354 us instead of 410, 16384 422 and 445, 38000 513 and
// 488; 152064 x 256 fp32: 1500 tokens 33 and 29)
inline bool zeros_go_first(int n, int vocab, int64_t row_bytes) { return ((int64_t)vocab - 5 * (int64_t)n) * row_bytes > 170000000; }

// The gradient of an embedding: sorted tokens in spans of kSpanChunks chunks of `chunk`, a wavefront for 64 * per_vec columns of each
// chunk, a workgroup for those of a span
constexpr int kSpanChunks = 8, kMostZeroRows = 64 * kSpanChunks;
constexpr int kMostTokens = 1 << 20;
struct EmbedGradPlan {
    int per_vec, slices, chunk, spans;
    int zero_rows;           // rows of the table of a workgroup that writes zeros: about 64 KB of them (76000 tokens into 152064 x 1024
                             // fp32 184 us, with 32 KB, and so twice the searches, 204)
};
inline EmbedGradPlan embed_grad_plan(int n, int width, bool single, int table_bytes) {
    EmbedGradPlan p{};
    p.per_vec = row_vec(width, single);
    p.slices = ceil_div(ceil_div(width, p.per_vec), 64);
    const int64_t want = ((int64_t)n * p.slices + 8191) / 8192;      // 8192 wavefronts run at once
    p.chunk = want <= 8 ? 8 : round_up((int)(want < n ? want : n), 8);
    p.spans = ceil_div(n, kSpanChunks * p.chunk);
    const int64_t rows = 65536 / ((int64_t)table_bytes * width);
    p.zero_rows = rows < 4 ? 4 : rows > kMostZeroRows ? kMostZeroRows : (int)rows;
    return p;
}

// Where things lie in the workspace, in bytes: sorted tokens and their places, the same between passes of the sort, digit counts of every tile, and
// two rows of partial sums for every span.  These are 4 MB and two rows at most: chunks grow with the list, so that there are no more than 1024 / slices spans and
// one, of slices that are 512 columns at most.
constexpr int kMostDigitBits = 11, kSortTile = 2048;
struct EmbedGradRoom {
    size_t places, other_sorted, other_places, counts, parts, end;
};
inline EmbedGradRoom embed_grad_room(int n, int width, const EmbedGradPlan &p) {
    const size_t list = 4 * (size_t)n;
    EmbedGradRoom r{list, 2 * list, 3 * list, 4 * list, 0, 0};
    r.parts = r.counts + ((size_t)4 << kMostDigitBits) * ceil_div(n, kSortTile);
    r.end = r.parts + (size_t)8 * width * p.spans;
    return r;
}

}  // namespace sr
