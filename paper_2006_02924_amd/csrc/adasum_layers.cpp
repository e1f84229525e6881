// C-ABI layer of the operators that fill a worker's gradient buffer: argument checks, then the launches.
#include "adasum_layers.h"

namespace adasum {
namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Bytes from `first` on, as addresses; an empty range overlaps nothing.
struct Range {
    uintptr_t first = 0;
    unsigned __int128 bytes = 0;
    bool meets(const Range& o) const {
        return bytes != 0 && o.bytes != 0 && first < static_cast<unsigned __int128>(o.first) + o.bytes &&
               o.first < static_cast<unsigned __int128>(first) + bytes;
    }
};
Range rows_range(const void* p, int64_t n, int64_t width, int64_t stride, int dtype) {
    Range r;
    r.first = reinterpret_cast<uintptr_t>(p);
    if (n > 0 && width > 0)
        r.bytes = (static_cast<unsigned __int128>(n - 1) * static_cast<uint64_t>(stride) + static_cast<uint64_t>(width)) * elem_bytes(dtype);
    return r;
}
Range bytes_range(const void* p, unsigned __int128 bytes) {
    Range r;
    r.first = reinterpret_cast<uintptr_t>(p);
    r.bytes = bytes;
    return r;
}

// Offsets and strides beyond this cannot be addresses; the products below stay inside 64 bits.
constexpr int64_t kMostElements = 1ll << 44;

int check_sizes(int64_t n, int64_t width) {
    return n < 0 || width < 0 || n > kMostTokens || width > kMostChannels ? ADASUM_ERR_INVALID_ARG : ADASUM_OK;
}
// A matrix of n rows; `written`: its rows must lie apart.
int check_rows(const void* p, int64_t n, int64_t width, int64_t stride, bool written) {
    if (stride < 0 || stride > kMostElements || (written && n > 1 && stride < width)) return ADASUM_ERR_INVALID_ARG;
    if (n == 0 || width == 0) return ADASUM_OK;
    if (p == nullptr) return ADASUM_ERR_INVALID_ARG;
    return aligned16(p) ? ADASUM_OK : ADASUM_ERR_MISALIGNED;
}
int check_flat(const void* p, int64_t offset, int64_t elems) {
    if (offset < 0 || offset > kMostElements || elems > kMostElements) return ADASUM_ERR_INVALID_ARG;
    if (elems == 0) return ADASUM_OK;
    if (p == nullptr) return ADASUM_ERR_INVALID_ARG;
    return aligned16(p) ? ADASUM_OK : ADASUM_ERR_MISALIGNED;
}
int check_ids(const void* ids, int id_type, int64_t n) {
    if (id_type != ADASUM_ID_I32 && id_type != ADASUM_ID_I64) return ADASUM_ERR_UNSUPPORTED;
    if (n == 0) return ADASUM_OK;
    if (ids == nullptr) return ADASUM_ERR_INVALID_ARG;
    return aligned16(ids) ? ADASUM_OK : ADASUM_ERR_MISALIGNED;
}
int check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return ADASUM_OK;
    return ws == nullptr || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0 || have < need ? ADASUM_ERR_WORKSPACE : ADASUM_OK;
}
int check_checkpoint(const void* checkpoint, int64_t rows, int64_t width) {
    const int rc = check_sizes(rows, width);
    if (rc != ADASUM_OK) return rc;
    if (rows == 0 || width == 0) return ADASUM_OK;
    if (checkpoint == nullptr) return ADASUM_ERR_INVALID_ARG;
    return aligned16(checkpoint) ? ADASUM_OK : ADASUM_ERR_MISALIGNED;
}
bool kept_type(int dtype) { return known_dtype(dtype) && dtype != ADASUM_F64; }
int64_t checkpoint_bytes(int64_t rows, int64_t width) { return rows * (checkpoint_pitch(width) / kBlock) * (kBlock + 1); }

char* at(void* base, int64_t offset, int dtype) { return static_cast<char*>(base) + offset * elem_bytes(dtype); }

#define ADASUM_CHECK(expr)                      \
    do {                                        \
        const int rc_ = (expr);                 \
        if (rc_ != ADASUM_OK) return rc_;       \
    } while (0)

int launched(int hip_error) { return hip_error == 0 ? ADASUM_OK : hip_failure(hip_error); }

}  // namespace
}  // namespace adasum

using namespace adasum;

extern "C" {

int adasum_embedding(const void* params, int dtype, int64_t offset, int64_t rows, int64_t width, const void* ids, int id_type,
                     int64_t n_ids, double scale, void* out, int out_dtype, int64_t out_stride, void* stream) {
    if (!types_go_together(dtype, out_dtype)) return ADASUM_ERR_UNSUPPORTED;
    ADASUM_CHECK(check_sizes(rows, width));
    ADASUM_CHECK(check_sizes(n_ids, width));
    ADASUM_CHECK(check_flat(params, offset, n_ids == 0 ? 0 : rows * width));
    ADASUM_CHECK(check_ids(ids, id_type, n_ids));
    ADASUM_CHECK(check_rows(out, n_ids, width, out_stride, true));
    if (n_ids == 0 || width == 0) return ADASUM_OK;
    if (rows == 0) return ADASUM_ERR_INVALID_ARG;
    const void* const table = static_cast<const char*>(params) + offset * elem_bytes(dtype);
    const Range result = rows_range(out, n_ids, width, out_stride, out_dtype);
    if (result.meets(rows_range(table, rows, width, width, dtype)) ||
        result.meets(bytes_range(ids, static_cast<unsigned __int128>(n_ids) * (id_type == ADASUM_ID_I64 ? 8 : 4))))
        return ADASUM_ERR_ALIAS;
    const Ids named{ids, id_type == ADASUM_ID_I64, n_ids};
    return launched(launch_lookup(dtype, out_dtype, table, rows, width, named, scale, out, out_stride, stream));
}

int adasum_embedding_grad_workspace_bytes(int64_t rows, int64_t width, int64_t n_ids, int dtype, size_t* bytes) {
    if (bytes == nullptr) return ADASUM_ERR_INVALID_ARG;
    if (!known_dtype(dtype)) return ADASUM_ERR_UNSUPPORTED;
    ADASUM_CHECK(check_sizes(rows, width));
    ADASUM_CHECK(check_sizes(n_ids, width));
    *bytes = n_ids == 0 || rows == 0 || width == 0 ? 0 : embedding_layout(rows, width, n_ids, dtype).total;
    return ADASUM_OK;
}

int adasum_embedding_grad(const void* dy, int dtype, int64_t dy_stride, const void* ids, int id_type, int64_t n_ids, double scale,
                          void* grad, int grad_dtype, int64_t offset, int64_t rows, int64_t width, int accumulate, void* workspace,
                          size_t workspace_bytes, void* stream) {
    if (!types_go_together(dtype, grad_dtype)) return ADASUM_ERR_UNSUPPORTED;
    if (accumulate != 0 && accumulate != 1) return ADASUM_ERR_INVALID_ARG;
    ADASUM_CHECK(check_sizes(rows, width));
    ADASUM_CHECK(check_sizes(n_ids, width));
    ADASUM_CHECK(check_flat(grad, offset, rows * width));
    ADASUM_CHECK(check_ids(ids, id_type, n_ids));
    ADASUM_CHECK(check_rows(dy, n_ids, width, dy_stride, false));
    if (rows == 0 || width == 0) return ADASUM_OK;
    EmbeddingGrad g{};
    if (n_ids > 0) g.lay = embedding_layout(rows, width, n_ids, dtype);
    ADASUM_CHECK(check_workspace(workspace, workspace_bytes, g.lay.total));
    g.grad = at(grad, offset, grad_dtype);
    const Range result = rows_range(g.grad, rows, width, width, grad_dtype), scratch = bytes_range(workspace, g.lay.total);
    const Range named = bytes_range(ids, static_cast<unsigned __int128>(n_ids) * (id_type == ADASUM_ID_I64 ? 8 : 4));
    const Range given = rows_range(dy, n_ids, width, dy_stride, dtype);
    if (result.meets(given) || result.meets(named) || result.meets(scratch) || scratch.meets(given) || scratch.meets(named))
        return ADASUM_ERR_ALIAS;
    g.dy = dy;
    g.dtype = dtype;
    g.dy_stride = dy_stride;
    g.ids = Ids{ids, id_type == ADASUM_ID_I64, n_ids};
    g.scale = scale;
    g.grad_dtype = grad_dtype;
    g.rows = rows;
    g.width = width;
    g.accumulate = accumulate;
    g.ws = static_cast<char*>(workspace);
    return launched(launch_embedding_grad(g, stream));
}

int adasum_checkpoint_bytes(int64_t rows, int64_t width, size_t* bytes) {
    if (bytes == nullptr) return ADASUM_ERR_INVALID_ARG;
    ADASUM_CHECK(check_sizes(rows, width));
    *bytes = static_cast<size_t>(checkpoint_bytes(rows, width));
    return ADASUM_OK;
}

int adasum_checkpoint_store(const void* x, int dtype, int64_t x_stride, int64_t rows, int64_t width, void* checkpoint, void* stream) {
    if (!kept_type(dtype)) return ADASUM_ERR_UNSUPPORTED;
    ADASUM_CHECK(check_checkpoint(checkpoint, rows, width));
    ADASUM_CHECK(check_rows(x, rows, width, x_stride, false));
    if (rows == 0 || width == 0) return ADASUM_OK;
    if (rows_range(x, rows, width, x_stride, dtype).meets(bytes_range(checkpoint, checkpoint_bytes(rows, width)))) return ADASUM_ERR_ALIAS;
    return launched(launch_store(x, dtype, x_stride, kept_view(checkpoint, rows, width), stream));
}

int adasum_checkpoint_load(const void* checkpoint, int64_t rows, int64_t width, void* out, int dtype, int64_t out_stride, void* stream) {
    if (!kept_type(dtype)) return ADASUM_ERR_UNSUPPORTED;
    ADASUM_CHECK(check_checkpoint(checkpoint, rows, width));
    ADASUM_CHECK(check_rows(out, rows, width, out_stride, true));
    if (rows == 0 || width == 0) return ADASUM_OK;
    if (rows_range(out, rows, width, out_stride, dtype).meets(bytes_range(checkpoint, checkpoint_bytes(rows, width))))
        return ADASUM_ERR_ALIAS;
    return launched(launch_load(kept_view(checkpoint, rows, width), out, dtype, out_stride, stream));
}

int adasum_checkpoint_act_grad(const void* checkpoint, int64_t rows, int64_t width, int act, const void* dy, int dtype,
                               int64_t dy_stride, void* dx, int64_t dx_stride, void* stream) {
    if (!kept_type(dtype) || act < ADASUM_ACT_RELU || act > ADASUM_ACT_SILU) return ADASUM_ERR_UNSUPPORTED;
    ADASUM_CHECK(check_checkpoint(checkpoint, rows, width));
    ADASUM_CHECK(check_rows(dy, rows, width, dy_stride, false));
    ADASUM_CHECK(check_rows(dx, rows, width, dx_stride, true));
    if (rows == 0 || width == 0) return ADASUM_OK;
    const Range result = rows_range(dx, rows, width, dx_stride, dtype);
    const bool in_place = dx == dy && (dx_stride == dy_stride || rows == 1);
    if (result.meets(bytes_range(checkpoint, checkpoint_bytes(rows, width))) ||
        (!in_place && result.meets(rows_range(dy, rows, width, dy_stride, dtype))))
        return ADASUM_ERR_ALIAS;
    return launched(launch_act_grad(kept_view(checkpoint, rows, width), act, dy, dtype, dy_stride, dx, dx_stride, stream));
}

int adasum_checkpoint_weight_grad_workspace_bytes(int64_t rows, int64_t width, int64_t outputs, int dtype, size_t* bytes) {
    if (bytes == nullptr) return ADASUM_ERR_INVALID_ARG;
    if (!kept_type(dtype)) return ADASUM_ERR_UNSUPPORTED;
    ADASUM_CHECK(check_sizes(rows, width));
    ADASUM_CHECK(check_sizes(0, outputs));
    *bytes = weight_split(rows, width, outputs, dtype).total;
    return ADASUM_OK;
}

int adasum_checkpoint_weight_grad(const void* checkpoint, int64_t rows, int64_t width, const void* dy, int dtype, int64_t dy_stride,
                                  int64_t outputs, void* grad, int grad_dtype, int64_t offset, int64_t bias_offset, int accumulate,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    if (!kept_type(dtype) || !kept_type(grad_dtype)) return ADASUM_ERR_UNSUPPORTED;
    if (accumulate != 0 && accumulate != 1) return ADASUM_ERR_INVALID_ARG;
    ADASUM_CHECK(check_checkpoint(checkpoint, rows, width));
    ADASUM_CHECK(check_sizes(0, outputs));
    ADASUM_CHECK(check_rows(dy, rows, outputs, dy_stride, false));
    ADASUM_CHECK(check_flat(grad, offset, outputs * width));
    const bool with_bias = bias_offset >= 0;
    if (with_bias) ADASUM_CHECK(check_flat(grad, bias_offset, outputs));
    if (outputs == 0) return ADASUM_OK;
    if (width == 0) return with_bias ? ADASUM_ERR_INVALID_ARG : ADASUM_OK;
    WeightGrad g{};
    g.split = weight_split(rows, width, outputs, dtype);
    ADASUM_CHECK(check_workspace(workspace, workspace_bytes, g.split.total));
    g.x = kept_view(checkpoint, rows, width);
    g.grad = at(grad, offset, grad_dtype);
    g.bias = with_bias ? at(grad, bias_offset, grad_dtype) : nullptr;
    const Range results[2] = {rows_range(g.grad, outputs, width, width, grad_dtype),
                              with_bias ? rows_range(g.bias, 1, outputs, outputs, grad_dtype) : Range{}};
    const Range scratch = bytes_range(workspace, g.split.total);
    const Range reads[2] = {bytes_range(checkpoint, checkpoint_bytes(rows, width)), rows_range(dy, rows, outputs, dy_stride, dtype)};
    if (results[0].meets(results[1])) return ADASUM_ERR_ALIAS;
    for (const Range& r : results)
        if (r.meets(reads[0]) || r.meets(reads[1]) || r.meets(scratch)) return ADASUM_ERR_ALIAS;
    if (scratch.meets(reads[0]) || scratch.meets(reads[1])) return ADASUM_ERR_ALIAS;
    g.dy = dy;
    g.dtype = dtype;
    g.dy_stride = dy_stride;
    g.outputs = outputs;
    g.grad_dtype = grad_dtype;
    g.accumulate = accumulate;
    g.ws = static_cast<char*>(workspace);
    return launched(launch_weight_grad(g, stream));
}

}  // extern "C"
