// C-ABI layer of the operators that fill a worker's gradient buffer and of those between the layers: argument checks, then the launches.
#include "adasum_layers.h"

#include <cmath>

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

bool in_place(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int64_t rows) {
    return a == b && (a_stride == b_stride || rows == 1);
}
// The step of a mask: read by the kernel.
int check_step(const void* step) { return (reinterpret_cast<uintptr_t>(step) & 7u) == 0 ? ADASUM_OK : ADASUM_ERR_MISALIGNED; }
bool is_share(double p) { return p >= 0.0 && p <= 1.0; }

// What a join's form says by itself.
int check_form(const adasum_join_form* f) {
    if (f == nullptr || f->struct_bytes != sizeof(adasum_join_form)) return ADASUM_ERR_INVALID_ARG;
    if (!kept_type(f->dtype) || (f->stream_dtype != f->dtype && f->stream_dtype != ADASUM_F32)) return ADASUM_ERR_UNSUPPORTED;
    if (f->norm != ADASUM_NORM_LAYER && f->norm != ADASUM_NORM_RMS) return ADASUM_ERR_UNSUPPORTED;
    if ((f->after != 0 && f->after != 1) || (f->before != 0 && f->before != 1) || f->width < 0) return ADASUM_ERR_INVALID_ARG;
    if (f->width > kMostJoined) return ADASUM_ERR_UNSUPPORTED;
    // (the square root's argument has to be a normal number for a row of zeros too)
    if (!(f->eps >= 1.2e-38 && f->eps < 3.4e38) || !std::isfinite(f->residual_scale) || std::fabs(f->residual_scale) > 3.4e38 ||
        !is_share(f->dropout))
        return ADASUM_ERR_INVALID_ARG;
    return ADASUM_OK;
}
// The vectors that a form names, in the order of their gradients; -1: none.
struct Vectors {
    int64_t offset[5];
    explicit Vectors(const adasum_join_form& f)
        : offset{f.after ? f.after_weight : -1, f.after ? f.after_bias : -1, f.gate, f.before ? f.before_weight : -1, f.before ? f.before_bias : -1} {}
    int check(const void* flat, int64_t width) const {
        for (int64_t o : offset)
            if (o >= 0) {
                const int rc = check_flat(flat, o, width);
                if (rc != ADASUM_OK) return rc;
            }
        return ADASUM_OK;
    }
    Range range(int i, const void* flat, int64_t width, int dtype) const {
        return offset[i] < 0 ? Range{} : rows_range(static_cast<const char*>(flat) + offset[i] * elem_bytes(dtype), 1, width, width, dtype);
    }
    bool any() const {
        for (int64_t o : offset)
            if (o >= 0) return true;
        return false;
    }
};
int join_types(const adasum_join_form& f) {
    return f.dtype == f.stream_dtype ? (f.dtype == ADASUM_F32 ? 0 : f.dtype == ADASUM_BF16 ? 1 : 2) : f.dtype == ADASUM_BF16 ? 3 : 4;
}
template <typename F>
int with_join_types(const adasum_join_form& f, F&& go) {
    switch (join_types(f)) {
        case 0: return go(std::integral_constant<int, 0>{});
        case 1: return go(std::integral_constant<int, 1>{});
        case 2: return go(std::integral_constant<int, 2>{});
        case 3: return go(std::integral_constant<int, 3>{});
        default: return go(std::integral_constant<int, 4>{});
    }
}

int check_weight8(const void* weight, int64_t outputs, int64_t width) {
    if (outputs < 0 || outputs > kMostChannels || width < 0 || width > kMostChannels) return ADASUM_ERR_INVALID_ARG;
    if (outputs == 0 || width == 0) return ADASUM_OK;
    if (weight == nullptr) return ADASUM_ERR_INVALID_ARG;
    return aligned16(weight) ? ADASUM_OK : ADASUM_ERR_MISALIGNED;
}
// One of a layer's two products: x [rows][depth] with the weight's rows, or with those of its transpose.
int product8(const void* weight, int64_t outputs, int64_t width, bool turned, const void* x, int dtype, int64_t x_stride, int64_t rows,
             const void* params, int param_dtype, int64_t bias_offset, void* out, int out_dtype, int64_t out_stride, void* workspace,
             size_t workspace_bytes, void* stream) {
    if (!kept_type(dtype) || !kept_type(out_dtype) || (bias_offset >= 0 && !kept_type(param_dtype))) return ADASUM_ERR_UNSUPPORTED;
    ADASUM_CHECK(check_weight8(weight, outputs, width));
    Product8 p{};
    p.outputs = turned ? width : outputs;
    p.depth = turned ? outputs : width;
    ADASUM_CHECK(check_sizes(rows, p.depth));
    ADASUM_CHECK(check_rows(x, rows, p.depth, x_stride, false));
    ADASUM_CHECK(check_rows(out, rows, p.outputs, out_stride, true));
    if (bias_offset >= 0) ADASUM_CHECK(check_flat(params, bias_offset, p.outputs));
    if (rows == 0 || p.outputs == 0) return ADASUM_OK;
    const size_t need = product8_workspace(rows, p.outputs, p.depth, out_dtype);
    ADASUM_CHECK(check_workspace(workspace, workspace_bytes, need));
    const Range result = rows_range(out, rows, p.outputs, out_stride, out_dtype), scratch = bytes_range(workspace, need);
    const Range reads[2] = {rows_range(x, rows, p.depth, x_stride, dtype), bytes_range(weight, weight8_bytes(outputs, width))};
    p.bias = bias_offset >= 0 ? static_cast<const char*>(params) + bias_offset * elem_bytes(param_dtype) : nullptr;
    const Range bias = bias_offset >= 0 ? rows_range(p.bias, 1, p.outputs, p.outputs, param_dtype) : Range{};
    if (result.meets(reads[0]) || result.meets(reads[1]) || result.meets(bias) || result.meets(scratch) || scratch.meets(reads[0]) ||
        scratch.meets(reads[1]) || scratch.meets(bias))
        return ADASUM_ERR_ALIAS;
    const Weight8 w = weight8_view(weight, outputs, width);
    p.w = turned ? w.turned : w.q;
    p.e = w.e;
    p.e_output = turned ? 1 : blocks8(width);
    p.e_depth = turned ? blocks8(width) : 1;
    p.x = x;
    p.dtype = dtype;
    p.x_stride = x_stride;
    p.rows = rows;
    p.bias_dtype = param_dtype;
    p.out = out;
    p.out_dtype = out_dtype;
    p.out_stride = out_stride;
    p.ws = static_cast<char*>(workspace);
    return launched(launch_product8(p, stream));
}

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

int adasum_dropout(const void* x, int dtype, int64_t x_stride, int64_t rows, int64_t width, double p, uint64_t seed, const uint64_t* step,
                   void* out, int64_t out_stride, void* stream) {
    if (!kept_type(dtype)) return ADASUM_ERR_UNSUPPORTED;
    if (!is_share(p)) return ADASUM_ERR_INVALID_ARG;
    ADASUM_CHECK(check_sizes(rows, width));
    ADASUM_CHECK(check_rows(x, rows, width, x_stride, false));
    ADASUM_CHECK(check_rows(out, rows, width, out_stride, true));
    ADASUM_CHECK(check_step(step));
    if (rows == 0 || width == 0) return ADASUM_OK;
    const Range result = rows_range(out, rows, width, out_stride, dtype);
    if ((!in_place(out, out_stride, x, x_stride, rows) && result.meets(rows_range(x, rows, width, x_stride, dtype))) ||
        (step != nullptr && result.meets(bytes_range(step, 8))))
        return ADASUM_ERR_ALIAS;
    return launched(launch_dropout(x, dtype, x_stride, rows, width, p, seed, step, out, out_stride, stream));
}

int adasum_join(const adasum_join_form* form, const void* params, int param_dtype, const uint64_t* step, const void* x, int64_t x_stride,
                const void* residual, int64_t residual_stride, int64_t rows, void* h, int64_t h_stride, void* y, int64_t y_stride, void* stream) {
    ADASUM_CHECK(check_form(form));
    const adasum_join_form& f = *form;
    const Vectors named(f);
    if (named.any() && !kept_type(param_dtype)) return ADASUM_ERR_UNSUPPORTED;
    ADASUM_CHECK(check_sizes(rows, f.width));
    ADASUM_CHECK(named.check(params, f.width));
    ADASUM_CHECK(check_step(step));
    ADASUM_CHECK(check_rows(x, rows, f.width, x_stride, false));
    if (residual != nullptr) ADASUM_CHECK(check_rows(residual, rows, f.width, residual_stride, false));
    if (h != nullptr) ADASUM_CHECK(check_rows(h, rows, f.width, h_stride, true));
    if (f.before) ADASUM_CHECK(check_rows(y, rows, f.width, y_stride, true));
    else if (y != nullptr) return ADASUM_ERR_INVALID_ARG;
    if (rows == 0 || f.width == 0) return ADASUM_OK;
    if (!f.before && h == nullptr) return ADASUM_ERR_INVALID_ARG;
    const Range results[2] = {h != nullptr ? rows_range(h, rows, f.width, h_stride, f.stream_dtype) : Range{},
                              f.before ? rows_range(y, rows, f.width, y_stride, f.dtype) : Range{}};
    const Range stream_in = residual != nullptr ? rows_range(residual, rows, f.width, residual_stride, f.stream_dtype) : Range{};
    const Range block_out = rows_range(x, rows, f.width, x_stride, f.dtype), counted = step != nullptr ? bytes_range(step, 8) : Range{};
    if (results[0].meets(results[1])) return ADASUM_ERR_ALIAS;
    for (int r = 0; r < 2; ++r) {
        if (results[r].meets(block_out) || results[r].meets(counted)) return ADASUM_ERR_ALIAS;
        if (results[r].meets(stream_in) && !(r == 0 && in_place(h, h_stride, residual, residual_stride, rows))) return ADASUM_ERR_ALIAS;
        for (int i = 0; i < 5; ++i)
            if (results[r].meets(named.range(i, params, f.width, param_dtype))) return ADASUM_ERR_ALIAS;
    }
    const JoinCall call{form, params, param_dtype, step, rows};
    const JoinRows m{{x, x_stride}, {residual, residual_stride}, {h, h_stride}, {y, y_stride}};
    return launched(with_join_types(f, [&](auto types) { return launch_join<decltype(types)::value>(call, m, stream); }));
}

int adasum_join_grad_workspace_bytes(const adasum_join_form* form, int64_t rows, size_t* bytes) {
    if (bytes == nullptr) return ADASUM_ERR_INVALID_ARG;
    ADASUM_CHECK(check_form(form));
    ADASUM_CHECK(check_sizes(rows, form->width));
    *bytes = join_layout(*form, rows).total;
    return ADASUM_OK;
}

int adasum_join_grad(const adasum_join_form* form, const void* params, int param_dtype, const uint64_t* step, const void* x, int64_t x_stride,
                     const void* h, int64_t h_stride, const void* dy, int64_t dy_stride, const void* dh, int64_t dh_stride, int64_t rows, void* dx,
                     int64_t dx_stride, void* dresidual, int64_t dresidual_stride, void* grad, int grad_dtype, int accumulate, void* workspace,
                     size_t workspace_bytes, void* stream) {
    ADASUM_CHECK(check_form(form));
    const adasum_join_form& f = *form;
    const Vectors named(f);
    if (named.any() && (!kept_type(param_dtype) || !kept_type(grad_dtype))) return ADASUM_ERR_UNSUPPORTED;
    if (accumulate != 0 && accumulate != 1) return ADASUM_ERR_INVALID_ARG;
    ADASUM_CHECK(check_sizes(rows, f.width));
    ADASUM_CHECK(named.check(params, f.width));
    ADASUM_CHECK(named.check(grad, f.width));
    ADASUM_CHECK(check_step(step));
    const bool reads_x = f.after || f.gate >= 0;
    if (reads_x) ADASUM_CHECK(check_rows(x, rows, f.width, x_stride, false));
    if (f.before) {
        ADASUM_CHECK(check_rows(h, rows, f.width, h_stride, false));
        ADASUM_CHECK(check_rows(dy, rows, f.width, dy_stride, false));
    }
    if (dh != nullptr || !f.before) ADASUM_CHECK(check_rows(dh, rows, f.width, dh_stride, false));
    ADASUM_CHECK(check_rows(dx, rows, f.width, dx_stride, true));
    if (dresidual != nullptr) ADASUM_CHECK(check_rows(dresidual, rows, f.width, dresidual_stride, true));
    if (f.width == 0) return ADASUM_OK;
    JoinSums to{join_layout(f, rows), workspace, {}, grad_dtype, accumulate};
    ADASUM_CHECK(check_workspace(workspace, workspace_bytes, to.layout.total));
    const Range scratch = bytes_range(workspace, to.layout.total);
    // what is read (dh apart, in whose place the stream's gradient may come), and what is written
    Range reads[9] = {reads_x ? rows_range(x, rows, f.width, x_stride, f.dtype) : Range{},
                      f.before ? rows_range(h, rows, f.width, h_stride, f.stream_dtype) : Range{},
                      f.before ? rows_range(dy, rows, f.width, dy_stride, f.dtype) : Range{}, step != nullptr ? bytes_range(step, 8) : Range{}};
    Range results[8] = {rows_range(dx, rows, f.width, dx_stride, f.dtype),
                        dresidual != nullptr ? rows_range(dresidual, rows, f.width, dresidual_stride, f.stream_dtype) : Range{}, scratch};
    for (int i = 0; i < 5; ++i) {
        reads[4 + i] = named.range(i, params, f.width, param_dtype);
        results[3 + i] = named.range(i, grad, f.width, grad_dtype);
        to.grads[i] = named.offset[i] < 0 ? nullptr : at(grad, named.offset[i], grad_dtype);
    }
    const Range carried = dh != nullptr ? rows_range(dh, rows, f.width, dh_stride, f.stream_dtype) : Range{};
    for (int r = 0; r < 8; ++r) {
        for (const Range& g : reads)
            if (results[r].meets(g)) return ADASUM_ERR_ALIAS;
        if (results[r].meets(carried) && !(r == 1 && in_place(dresidual, dresidual_stride, dh, dh_stride, rows))) return ADASUM_ERR_ALIAS;
        for (int o = 0; o < r; ++o)
            if (results[r].meets(results[o])) return ADASUM_ERR_ALIAS;
    }
    const JoinCall call{form, params, param_dtype, step, rows};
    const JoinGradRows m{{x, x_stride}, {h, h_stride}, {dy, dy_stride}, {dh, dh_stride}, {dx, dx_stride}, {dresidual, dresidual_stride}};
    return launched(with_join_types(f, [&](auto types) { return launch_join_grad<decltype(types)::value>(call, m, to, stream); }));
}

int adasum_linear_bytes(int64_t outputs, int64_t width, size_t* bytes) {
    if (bytes == nullptr) return ADASUM_ERR_INVALID_ARG;
    if (outputs < 0 || outputs > kMostChannels || width < 0 || width > kMostChannels) return ADASUM_ERR_INVALID_ARG;
    *bytes = outputs == 0 || width == 0 ? 0 : weight8_bytes(outputs, width);
    return ADASUM_OK;
}

int adasum_linear_store(const void* params, int dtype, int64_t offset, int64_t outputs, int64_t width, void* weight, void* stream) {
    if (!kept_type(dtype)) return ADASUM_ERR_UNSUPPORTED;
    ADASUM_CHECK(check_weight8(weight, outputs, width));
    ADASUM_CHECK(check_flat(params, offset, outputs * width));
    if (outputs == 0 || width == 0) return ADASUM_OK;
    const void* const w = static_cast<const char*>(params) + offset * elem_bytes(dtype);
    if (rows_range(w, outputs, width, width, dtype).meets(bytes_range(weight, weight8_bytes(outputs, width)))) return ADASUM_ERR_ALIAS;
    return launched(launch_weight8_store(w, dtype, weight8_view(weight, outputs, width), stream));
}

int adasum_linear_workspace_bytes(int64_t rows, int64_t width, int64_t outputs, int out_dtype, size_t* bytes) {
    if (bytes == nullptr) return ADASUM_ERR_INVALID_ARG;
    if (!kept_type(out_dtype)) return ADASUM_ERR_UNSUPPORTED;
    ADASUM_CHECK(check_sizes(rows, width));
    ADASUM_CHECK(check_sizes(rows, outputs));
    const size_t forward = product8_workspace(rows, outputs, width, out_dtype), back = product8_workspace(rows, width, outputs, out_dtype);
    *bytes = rows == 0 ? 0 : forward > back ? forward : back;
    return ADASUM_OK;
}

int adasum_linear(const void* weight, int64_t outputs, int64_t width, const void* x, int dtype, int64_t x_stride, int64_t rows,
                   const void* params, int param_dtype, int64_t bias_offset, void* out, int out_dtype, int64_t out_stride, void* workspace,
                   size_t workspace_bytes, void* stream) {
    return product8(weight, outputs, width, false, x, dtype, x_stride, rows, params, param_dtype, bias_offset, out, out_dtype, out_stride, workspace,
                    workspace_bytes, stream);
}

int adasum_linear_grad(const void* weight, int64_t outputs, int64_t width, const void* dy, int dtype, int64_t dy_stride, int64_t rows, void* dx,
                        int dx_dtype, int64_t dx_stride, void* workspace, size_t workspace_bytes, void* stream) {
    return product8(weight, outputs, width, true, dy, dtype, dy_stride, rows, nullptr, ADASUM_F32, -1, dx, dx_dtype, dx_stride, workspace,
                    workspace_bytes, stream);
}

}  // extern "C"
