// Internal declarations of the operators that fill a worker's gradient buffer: embedding tables, activation
// checkpoints in 8 bits and the gradients made from them.  Nothing here is exported.
#pragma once

#include <cstddef>
#include <cstdint>

#include "adasum_host.h"

namespace adasum {

constexpr int64_t kMostTokens = (1ll << 31) - 65536;   // rows of an activation matrix, or of a table
constexpr int64_t kMostChannels = 1ll << 24;
constexpr int kBlock = ADASUM_CHECKPOINT_BLOCK;

// Storage types that may stand beside each other in one operator.
inline bool types_go_together(int a, int b) {
    return known_dtype(a) && known_dtype(b) && (a == ADASUM_F64) == (b == ADASUM_F64);
}

// ---- embedding tables (adasum_embedding.hip) ----------------------------------

struct Ids {
    const void* p;
    int wide;        // 64-bit ids
    int64_t n;
};

// The sorted tokens are cut into chunks of 32, or of 16 up to kFewTokens tokens, which make too few waves otherwise (whole calls in bf16 with 16
// and 32: 8192 tokens of 30522 rows x 1024 36 and 43 us, of 512 rows x 64 27 and 32; 32768 tokens 49 and 50, 37 and 39, but of 512 rows x
// 1024 54 and 50; 131072 tokens 117 and 100, 82 and 76).  A run (the tokens
// of one row) that is no longer than a chunk is summed by the wave in whose chunk it starts; of a longer one every chunk sums its part,
// and a second launch adds the parts.
constexpr int64_t kFewTokens = 32768;
// Workgroups that sort: each takes an equal range of rows, at most kSortRows where it reads all tokens itself and at most kGatherRows
// where the tokens have been sorted by range before, in parts of kPartTokens.
constexpr int kSortGroups = 256;
constexpr int kSortRows = 1008;   // (their counts take just under 64 KB)
constexpr int kGatherRows = 1024;
constexpr int kPartTokens = 2048;
inline int64_t sort_rows(int64_t rows) {
    const int64_t r = (rows + kSortGroups - 1) / kSortGroups;
    return r < 1 ? 1 : r > kSortRows ? kSortRows : r;
}
// Whether the tokens are sorted by range first.  (Not for tables of more rows than their workgroups have lanes for; each of the others reads
// all ids then, which many tokens feel: x 64 in bf16, 262144 and 262145 rows, 16384 tokens 32 and 51 us, 131072 tokens 51 and 305.)
inline bool in_parts(int64_t rows, int64_t n_ids) { return n_ids > 4096 && rows <= kSortGroups * kGatherRows; }

// Workspace of the table's gradient (byte offsets).
struct EmbeddingLayout {
    int run = 0;              // tokens of a chunk
    int64_t chunks = 0;
    size_t off_totals = 0;    // int32: tokens whose id names a row; runs of more than a chunk's tokens
    size_t off_listed = 0;    // int32 [chunk]: the chunks in which those start
    size_t off_place = 0;     // int32 [n]: tokens in the order of their ids
    size_t off_row = 0;       // int32 [n]: their ids
    size_t off_begins = 0;    // where they are sorted by range first: int32 [range + 1][part]
    size_t off_part_place = 0, off_part_row = 0;   // int32 [part][kPartTokens]
    size_t off_parts = 0;     // [chunk][2][width]: sums of the run that comes from the chunk before, and of the one that goes on into the next
    size_t total = 0;
};
EmbeddingLayout embedding_layout(int64_t rows, int64_t width, int64_t n_ids, int dtype);

int launch_lookup(int dtype, int out_dtype, const void* table, int64_t rows, int64_t width, const Ids& ids, double scale,
                  void* out, int64_t out_stride, void* stream);

struct EmbeddingGrad {
    const void* dy;
    int dtype;
    int64_t dy_stride;
    Ids ids;
    double scale;
    void* grad;              // the table
    int grad_dtype;
    int64_t rows, width;
    int accumulate;
    char* ws;
    EmbeddingLayout lay;
};
int launch_embedding_grad(const EmbeddingGrad& g, void* stream);

// ---- checkpoints (adasum_checkpoint.hip) ---------------------------------------

inline int64_t checkpoint_pitch(int64_t width) { return (width + kBlock - 1) / kBlock * kBlock; }

struct Kept {
    const int8_t* q;
    const int8_t* e;
    int64_t rows, width, pitch;
};
inline Kept kept_view(const void* checkpoint, int64_t rows, int64_t width) {
    Kept k;
    k.rows = rows;
    k.width = width;
    k.pitch = checkpoint_pitch(width);
    k.q = static_cast<const int8_t*>(checkpoint);
    k.e = k.q + rows * k.pitch;
    return k;
}

int launch_store(const void* x, int dtype, int64_t x_stride, const Kept& to, void* stream);
int launch_load(const Kept& k, void* out, int dtype, int64_t out_stride, void* stream);
int launch_act_grad(const Kept& k, int act, const void* dy, int dtype, int64_t dy_stride, void* dx, int64_t dx_stride,
                    void* stream);

// ---- weight gradients (adasum_weight_grad.hip, adasum_weight_split.cpp) -----------

// A workgroup computes a square of the weight, `tile` wide, over one of `parts` parts of the tokens, each `steps` steps of the kernel (of
// 64 tokens, 32 in fp32).
struct WeightSplit {
    int tile = 0;
    int64_t parts = 1, steps = 0;
    size_t off_bias = 0;      // fp32 [parts][outputs], behind fp32 [parts][outputs][width] (with more than one part)
    size_t total = 0;
};
WeightSplit weight_split(int64_t rows, int64_t width, int64_t outputs, int dtype);

struct WeightGrad {
    Kept x;
    const void* dy;
    int dtype;
    int64_t dy_stride, outputs;
    void* grad;              // the weight
    void* bias;              // or null
    int grad_dtype, accumulate;
    char* ws;
    WeightSplit split;
};
int launch_weight_grad(const WeightGrad& g, void* stream);

}  // namespace adasum
