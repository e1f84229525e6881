// Internal declarations of the operators that fill a worker's gradient buffer (embedding tables, activation
// checkpoints in 8 bits and the gradients made from them) and of those between the layers (dropout, the join of a
// block with its residual stream, products in 8-bit floating point).  Nothing here is exported.
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

// ---- dropout (adasum_dropout.hip) ---------------------------------------------

int launch_dropout(const void* x, int dtype, int64_t x_stride, int64_t rows, int64_t width, double p, uint64_t seed, const void* step,
                   void* out, int64_t out_stride, void* stream);

// ---- the join of a block with its residual stream (adasum_join.hip) -------------

constexpr int64_t kMostJoined = 8192;   // channels of a row: what the lanes of a workgroup hold
struct Matrix {
    const void* p;
    int64_t stride;
};
struct JoinCall {
    const adasum_join_form* form;
    const void* params;
    int param_dtype;
    const void* step;
    int64_t rows;
};
struct JoinRows {
    Matrix x, residual, h, y;
};
struct JoinGradRows {
    Matrix x, h, dy, dh, dx, dresidual;
};
// The sums of the parameters' gradients: fp32 [group][kind][width].
struct JoinLayout {
    int groups = 0, kinds = 0;
    size_t total = 0;
};
// Rows that a workgroup has in its lanes at once.
inline int joined_at_once(int64_t width) { return width <= 64 ? 32 : width <= 128 ? 16 : width <= 256 ? 8 : width <= 1024 ? 4 : 1; }
// Workgroups that go round the rows: what the chip holds at once, by the registers that a row's lanes take; the gradient has half of that
// where the sums of more would cost what the rest gains.  16.8 million elements in bf16, no operand in a cache, with 512, 768, 1024, 1280 and
// 2048: width 512 33, 29, 28, 28 and 30 us; 1024 27, 28, 27, 31 and 30, with two norms and a gate 30, 29, 33, 33 and 33; 8192 28, 31, 31, 32
// and 32.  Gradients with 256, 512 and 1024: width 512 75, 50 and 43, with two norms and a gate 68, 49 and 57; 1024 51, 41 and 47;
// 8192 49, 59 and 77.
inline int join_groups(int64_t width, bool full, bool gradient) {
    const bool one = width <= 512 || (width > 1024 && width <= 2048);   // granule a lane
    if (gradient) return one && !full ? 1024 : width <= 4096 ? 512 : 256;
    return one ? 1024 : width <= 4096 ? 768 : 512;
}
inline JoinLayout join_layout(const adasum_join_form& f, int64_t rows) {
    JoinLayout lay;
    const bool full = f.after || f.gate >= 0;
    const bool any = f.gate >= 0 || (f.after && (f.after_weight >= 0 || f.after_bias >= 0)) ||
                     (f.before && (f.before_weight >= 0 || f.before_bias >= 0));
    const int64_t needed = (rows + joined_at_once(f.width) - 1) / joined_at_once(f.width);
    const int64_t most = join_groups(f.width, full, true);
    lay.groups = static_cast<int>(needed < most ? needed : most);
    lay.kinds = !any ? 0 : full ? 4 : 2;
    lay.total = static_cast<size_t>(lay.groups) * lay.kinds * f.width * 4;
    return lay;
}
struct JoinSums {
    JoinLayout layout;
    void* ws;
    void* grads[5];          // after weight and bias, gate, before weight and bias; null: none
    int dtype, accumulate;
};
// By the storage types of activations and stream: 0 fp32, 1 bf16, 2 fp16, and 3 bf16, 4 fp16 with a stream of fp32.
template <int TYPES> int launch_join(const JoinCall& c, const JoinRows& m, void* stream);
template <int TYPES> int launch_join_grad(const JoinCall& c, const JoinGradRows& m, const JoinSums& to, void* stream);
template <> int launch_join<0>(const JoinCall&, const JoinRows&, void*);
template <> int launch_join<1>(const JoinCall&, const JoinRows&, void*);
template <> int launch_join<2>(const JoinCall&, const JoinRows&, void*);
template <> int launch_join<3>(const JoinCall&, const JoinRows&, void*);
template <> int launch_join<4>(const JoinCall&, const JoinRows&, void*);
template <> int launch_join_grad<0>(const JoinCall&, const JoinGradRows&, const JoinSums&, void*);
template <> int launch_join_grad<1>(const JoinCall&, const JoinGradRows&, const JoinSums&, void*);
template <> int launch_join_grad<2>(const JoinCall&, const JoinGradRows&, const JoinSums&, void*);
template <> int launch_join_grad<3>(const JoinCall&, const JoinGradRows&, const JoinSums&, void*);
template <> int launch_join_grad<4>(const JoinCall&, const JoinGradRows&, const JoinSums&, void*);

// ---- linear layers in 8-bit floating point (adasum_linear.hip) ------------------

constexpr int kBlock8 = ADASUM_LINEAR_BLOCK;
inline int64_t blocks8(int64_t n) { return (n + kBlock8 - 1) / kBlock8; }
// A weight: its rows in panels of 64 channels, [blocks of width * 2][outputs][64] bytes, those of its transpose, [blocks of outputs * 2]
// [width][64], and a byte for each block, [blocks of outputs][blocks of width], e + 127.
struct Weight8 {
    unsigned char *q, *turned, *e;
    int64_t outputs, width;
};
inline size_t weight8_bytes(int64_t outputs, int64_t width) {
    return static_cast<size_t>(outputs) * blocks8(width) * kBlock8 + static_cast<size_t>(width) * blocks8(outputs) * kBlock8 +
           align_up(static_cast<size_t>(blocks8(outputs)) * blocks8(width), 16);
}
inline Weight8 weight8_view(const void* weight, int64_t outputs, int64_t width) {
    Weight8 w;
    w.q = static_cast<unsigned char*>(const_cast<void*>(weight));
    w.turned = w.q + outputs * blocks8(width) * kBlock8;
    w.e = w.turned + width * blocks8(outputs) * kBlock8;
    w.outputs = outputs;
    w.width = width;
    return w;
}
int launch_weight8_store(const void* w, int dtype, const Weight8& to, void* stream);

// out [rows][outputs] = x [rows][depth] times the transpose of w [outputs][depth] in 8 bits, and a bias.
struct Product8 {
    const unsigned char *w, *e;          // panels of 64 channels; the exponent of block (output, depth) is e[output * e_output + depth * e_depth]
    int64_t outputs, depth, e_output, e_depth;
    const void* x;
    int dtype;
    int64_t x_stride, rows;
    const void* bias;                    // or null
    int bias_dtype;
    void* out;
    int out_dtype;
    int64_t out_stride;
    char* ws;
};
size_t product8_workspace(int64_t rows, int64_t outputs, int64_t depth, int out_dtype);
int launch_product8(const Product8& p, void* stream);

}  // namespace adasum
