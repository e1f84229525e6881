// gfx950 kernels of the place where a block's output joins the residual stream, and of its gradient:
//   v = N(x) w + b  (or x),   h = scale residual + gate D(v),   y = N(h) w' + b'
// with N the norm of a row (its mean and spread, or its spread alone) and D dropout.  (Compiled once for each pair of storage types.)
//
// A row lies in the registers of a run of lanes, eight channels a granule, from its loads to its stores: the statistics are sums over the
// lanes, first the mean, then the squares of what is left, so that nothing cancels.  A workgroup goes from row to row with the
// parameters' vectors in registers; the gradient adds those of the parameters up there too, each lane its own channels' in fp32 over the
// workgroup's rows, and a second launch adds the workgroups' in fp64.  The gradient works the statistics out again from the rows that it
// reads anyhow: nothing is kept for it but the rows themselves.
#include <hip/hip_runtime.h>

#include "adasum_layers.h"
#include "adasum_mask.h"

namespace adasum {
namespace {

#if ADASUM_JOIN_TYPES == 0
typedef float T; typedef float S;
#elif ADASUM_JOIN_TYPES == 1
typedef bf16_t T; typedef bf16_t S;
#elif ADASUM_JOIN_TYPES == 2
typedef f16_t T; typedef f16_t S;
#elif ADASUM_JOIN_TYPES == 3
typedef bf16_t T; typedef float S;
#else
typedef f16_t T; typedef float S;
#endif

// ---- sums over the lanes of a row ---------------------------------------------

template <int N>
__device__ __forceinline__ float turned(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + N, 0xf, 0xf, true));
}
// Over each run of 16 or 64 lanes, in every lane of it.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
    v += turned<8>(v);
    v += turned<4>(v);
    v += turned<2>(v);
    v += turned<1>(v);
    if constexpr (LANES > 16) {
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
        const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(b[0]) + __uint_as_float(b[1]);
    }
    return v;
}
// Over the LANES lanes of a row, N sums at a time.  Rows of several waves meet in LDS, in one of two places in turn: a wave that writes the
// next but one sum has passed the barrier behind which all have read this one.
template <int LANES>
struct RowSums {
    static constexpr int kWaves = LANES > 64 ? LANES / 64 : 1;
    float (*shared)[2][kWaves];   // [2]
    int turn = 0;
    template <int N>
    __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lanes_sum<LANES>(v[i]);
        if constexpr (LANES > 64) {
            float(&at)[2][kWaves] = shared[turn];
            turn ^= 1;
            const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
            if (lane == 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) at[i][wave] = v[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = 0.f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) v[i] += at[i][w];
            }
        }
    }
    __device__ __forceinline__ float operator()(float v) {
        float a[1] = {v};
        (*this)(a);
        return a[0];
    }
};

// ---- a row's part in a lane ---------------------------------------------------

template <int LANES, int V, RowForm FORM>
struct Row {
    typedef float Part[V][kG];
    static constexpr int threads = LANES > 256 ? LANES : 256;
    static constexpr int rows_at_once = threads / LANES;
    int width, lane;
    __device__ __forceinline__ int at(int k) const { return (k * LANES + lane) * kG; }
    __device__ __forceinline__ bool there(int k, int i) const { return FORM == kWhole ? at(k) < width : at(k) + i < width; }
    template <typename E>
    __device__ __forceinline__ void load(Granule<E, kG> (&raw)[V], const E* row) const {
#pragma unroll
        for (int k = 0; k < V; ++k) load_row<FORM>(raw[k], row, at(k), width);
    }
    // zeros where there is no channel
    template <typename E>
    __device__ __forceinline__ void values(Part& v, const Granule<E, kG> (&raw)[V]) const {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            unpack(raw[k], v[k]);
#pragma unroll
            for (int i = 0; i < kG; ++i)
                if (!there(k, i)) v[k][i] = 0.f;
        }
    }
    template <typename E>
    __device__ __forceinline__ void store(E* row, const Part& v) const {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (at(k) < width) store_row<FORM>(row, v[k], at(k), width);
    }
    // a vector of parameters, or `instead`
    __device__ __forceinline__ void param(Part& v, const void* p, int type, float instead) const {
#pragma unroll
        for (int k = 0; k < V; ++k) {
#pragma unroll
            for (int i = 0; i < kG; ++i) v[k][i] = instead;
            const int left = width - at(k);
            if (p == nullptr || left <= 0) continue;
            if (type == ADASUM_F32) load_some(v[k], static_cast<const float*>(p) + at(k), left);
            else if (type == ADASUM_BF16) load_some(v[k], static_cast<const bf16_t*>(p) + at(k), left);
            else load_some(v[k], static_cast<const f16_t*>(p) + at(k), left);
        }
    }
    // v normed (hat); returns one over its spread
    __device__ __forceinline__ float normed(Part& v, RowSums<LANES>& sums, bool centred, float eps, float each) const {
        if (centred) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) s += v[k][i];
            const float mean = sums(s) * each;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) v[k][i] = there(k, i) ? v[k][i] - mean : 0.f;
        }
        float q = 0.f;
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < kG; ++i) q = __builtin_fmaf(v[k][i], v[k][i], q);
        const float r = 1.f / __builtin_sqrtf(__builtin_fmaf(sums(q), each, eps));
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < kG; ++i) v[k][i] *= r;
        return r;
    }
    // the gradient d of normed rows (hat, r) times w, back to before the norm
    __device__ __forceinline__ void norm_grad(Part& d, const Part& w, const Part& hat, float r, RowSums<LANES>& sums, bool centred, float each) const {
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < kG; ++i) {
                d[k][i] *= w[k][i];
                s[0] += d[k][i];
                s[1] = __builtin_fmaf(d[k][i], hat[k][i], s[1]);
            }
        sums(s);
        const float mean = centred ? s[0] * each : 0.f, inner = s[1] * each;
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < kG; ++i) d[k][i] = r * (d[k][i] - __builtin_fmaf(hat[k][i], inner, mean));
    }
    __device__ __forceinline__ void mask(unsigned (&w)[V][4], const Mask& m, Step step, long long row) const {
#pragma unroll
        for (int k = 0; k < V; ++k) mask_words(w[k], m, step, static_cast<unsigned>(at(k)) / kG, static_cast<unsigned>(row));
    }
};

struct Args {
    const T* x;
    const S* residual;          // or null
    const S* h;                 // of the gradient
    const T* dy;
    const S* dh;
    S* to_h;
    T* to_y;
    T* dx;
    S* dresidual;
    long long x_stride, residual_stride, h_stride, dy_stride, dh_stride, to_h_stride, to_y_stride, dx_stride, dresidual_stride, rows;
    const void *after_weight, *after_bias, *gate, *before_weight, *before_bias;
    int param_type, width, after, before, centred, drop;
    float eps, scale, each;     // each: one over the width
    Mask mask;
    float* parts;               // sums of the parameters' gradients: [workgroup][kind][width]
    int kinds;
};

// FULL: with a norm of x, or a gate.
template <int LANES, int V, RowForm FORM, bool FULL>
__global__ void __launch_bounds__((Row<LANES, V, FORM>::threads))
join_kernel(Args a) {
    typedef Row<LANES, V, FORM> R;
    typedef typename R::Part Part;
    __shared__ float shared[2][2][RowSums<LANES>::kWaves];
    RowSums<LANES> sums{shared};
    R r;
    r.width = a.width;
    r.lane = threadIdx.x % LANES;
    const Step step = step_of(a.mask);
    Part aw, ab, gate, bw, bb;
    if constexpr (FULL) {
        r.param(aw, a.after_weight, a.param_type, 1.f);
        r.param(ab, a.after_bias, a.param_type, 0.f);
        r.param(gate, a.gate, a.param_type, 1.f);
    }
    r.param(bw, a.before_weight, a.param_type, 1.f);
    r.param(bb, a.before_bias, a.param_type, 0.f);
    // (rows of several waves: the workgroup's lanes go round together)
    for (long long row = static_cast<long long>(blockIdx.x) * R::rows_at_once + threadIdx.x / LANES; row < a.rows;
         row += static_cast<long long>(gridDim.x) * R::rows_at_once) {
        Granule<T, kG> raw_x[V];
        Granule<S, kG> raw_r[V];
        r.load(raw_x, a.x + row * a.x_stride);
        if (a.residual != nullptr) r.load(raw_r, a.residual + row * a.residual_stride);
        Part v;
        r.values(v, raw_x);
        if constexpr (FULL) {
            if (a.after) {
                r.normed(v, sums, a.centred, a.eps, a.each);
#pragma unroll
                for (int k = 0; k < V; ++k)
#pragma unroll
                    for (int i = 0; i < kG; ++i) v[k][i] = __builtin_fmaf(v[k][i], aw[k][i], ab[k][i]);
            }
        }
        if (a.drop) {
            unsigned w[V][4];
            r.mask(w, a.mask, step, row);
#pragma unroll
            for (int k = 0; k < V; ++k) drop(v[k], w[k], a.mask);
        }
        if constexpr (FULL) {
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) v[k][i] *= gate[k][i];
        }
        if (a.residual != nullptr) {
            Part res;
            r.values(res, raw_r);
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) v[k][i] = __builtin_fmaf(a.scale, res[k][i], v[k][i]);
        }
        if (a.to_h != nullptr) r.store(a.to_h + row * a.to_h_stride, v);
        if (a.before) {
            // (a bias of the norm of x is there behind the row's end too)
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i)
                    if (!r.there(k, i)) v[k][i] = 0.f;
            r.normed(v, sums, a.centred, a.eps, a.each);
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) v[k][i] = __builtin_fmaf(v[k][i], bw[k][i], bb[k][i]);
            r.store(a.to_y + row * a.to_y_stride, v);
        }
    }
}

// The kinds of parameters in the order of their sums.
enum { kAfterWeight, kAfterBias, kGate, kBeforeWeight, kBeforeBias };

template <int LANES, int V, RowForm FORM, bool FULL>
__global__ void __launch_bounds__((Row<LANES, V, FORM>::threads))
join_grad_kernel(Args a) {
    typedef Row<LANES, V, FORM> R;
    typedef typename R::Part Part;
    constexpr int kFirst = FULL ? 0 : kBeforeWeight, kSums = kBeforeBias + 1 - kFirst;
    __shared__ float shared[2][2][RowSums<LANES>::kWaves];
    RowSums<LANES> sums{shared};
    R r;
    r.width = a.width;
    r.lane = threadIdx.x % LANES;
    const Step step = step_of(a.mask);
    Part aw, ab, gate, bw;
    if constexpr (FULL) {
        r.param(aw, a.after_weight, a.param_type, 1.f);
        r.param(ab, a.after_bias, a.param_type, 0.f);
        r.param(gate, a.gate, a.param_type, 1.f);
    }
    r.param(bw, a.before_weight, a.param_type, 1.f);
    Part total[kSums] = {};
    for (long long row = static_cast<long long>(blockIdx.x) * R::rows_at_once + threadIdx.x / LANES; row < a.rows;
         row += static_cast<long long>(gridDim.x) * R::rows_at_once) {
        Granule<T, kG> raw_x[V], raw_dy[V];
        Granule<S, kG> raw_h[V], raw_dh[V];
        if (a.before) {
            r.load(raw_dy, a.dy + row * a.dy_stride);
            r.load(raw_h, a.h + row * a.h_stride);
        }
        if (a.dh != nullptr) r.load(raw_dh, a.dh + row * a.dh_stride);
        if constexpr (FULL) r.load(raw_x, a.x + row * a.x_stride);
        Part d = {};
        if (a.before) {
            Part hat;
            r.values(hat, raw_h);
            r.values(d, raw_dy);
            const float spread = r.normed(hat, sums, a.centred, a.eps, a.each);
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) {
                    total[kBeforeWeight - kFirst][k][i] = __builtin_fmaf(d[k][i], hat[k][i], total[kBeforeWeight - kFirst][k][i]);
                    total[kBeforeBias - kFirst][k][i] += d[k][i];
                }
            r.norm_grad(d, bw, hat, spread, sums, a.centred, a.each);
        }
        if (a.dh != nullptr) {
            Part dh;
            r.values(dh, raw_dh);
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) d[k][i] += dh[k][i];
        }
        if (a.dresidual != nullptr) {
            Part scaled;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) scaled[k][i] = a.scale * d[k][i];
            r.store(a.dresidual + row * a.dresidual_stride, scaled);
        }
        // (what dropout leaves of d; its gradient is taken through the gate)
        unsigned w[V][4];
        if (a.drop) {
            r.mask(w, a.mask, step, row);
#pragma unroll
            for (int k = 0; k < V; ++k) drop(d[k], w[k], a.mask);
        }
        if constexpr (FULL) {
            Part hat;
            r.values(hat, raw_x);
            float spread = 1.f;
            if (a.after) spread = r.normed(hat, sums, a.centred, a.eps, a.each);
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) {
                    const bool here = r.there(k, i);
                    // (dropped places of x add nothing, whatever it holds there)
                    const float v = a.after ? __builtin_fmaf(hat[k][i], aw[k][i], ab[k][i]) : hat[k][i];
                    if (here && (!a.drop || keeps(w[k], i, a.mask.limit)))
                        total[kGate - kFirst][k][i] = __builtin_fmaf(d[k][i], v, total[kGate - kFirst][k][i]);
                    d[k][i] = here ? d[k][i] * gate[k][i] : 0.f;
                }
            if (a.after) {
#pragma unroll
                for (int k = 0; k < V; ++k)
#pragma unroll
                    for (int i = 0; i < kG; ++i) {
                        total[kAfterWeight - kFirst][k][i] = __builtin_fmaf(d[k][i], hat[k][i], total[kAfterWeight - kFirst][k][i]);
                        total[kAfterBias - kFirst][k][i] += d[k][i];
                    }
                r.norm_grad(d, aw, hat, spread, sums, a.centred, a.each);
            }
        }
        r.store(a.dx + row * a.dx_stride, d);
    }
    if (a.parts == nullptr) return;
    // the workgroup's rows together, where it has several at once, then its sums to memory
    float* const to = a.parts + static_cast<long long>(blockIdx.x) * a.kinds * a.width;
    if constexpr (R::rows_at_once > 1) {
        constexpr int kWidth = LANES * V * kG;
        __shared__ float meet[R::rows_at_once][kWidth];
#pragma unroll
        for (int s = 0; s < kSums; ++s) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) meet[threadIdx.x / LANES][r.at(k) + i] = total[s][k][i];
            __syncthreads();
            for (int j = threadIdx.x; j < a.width; j += R::threads) {
                float sum = 0.f;
#pragma unroll
                for (int w = 0; w < R::rows_at_once; ++w) sum += meet[w][j];
                to[s * a.width + j] = sum;
            }
        }
    } else {
#pragma unroll
        for (int s = 0; s < kSums; ++s)
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (r.at(k) < a.width) store_some<kG>(to + s * a.width + r.at(k), total[s][k], a.width - r.at(k));
    }
}

// The parameters' gradients out of the workgroups' sums: a workgroup takes 64 channels of a kind, four waves a quarter of the sums each.
struct Finish {
    const float* parts;
    int groups, kinds, width, accumulate;
    void* to[5];                 // by place among the sums; null: not asked for
};
template <typename G>
__global__ void __launch_bounds__(256) join_finish_kernel(Finish f) {
    __shared__ double shared[4][64];
    const int kind = blockIdx.y, lane = threadIdx.x & 63, way = threadIdx.x >> 6, j = blockIdx.x * 64 + lane;
    G* const to = static_cast<G*>(f.to[kind]);
    if (to == nullptr) return;
    double sum = 0;
    if (j < f.width) {
#pragma unroll 4
        for (int g = way; g < f.groups; g += 4) sum += f.parts[(static_cast<long long>(g) * f.kinds + kind) * f.width + j];
    }
    shared[way][lane] = sum;
    __syncthreads();
    if (way == 0 && j < f.width) {
        sum = shared[0][lane] + shared[1][lane] + shared[2][lane] + shared[3][lane];
        if (f.accumulate) sum += load_elem(to + j);
        store_elem(to + j, static_cast<float>(sum));
    }
}

template <typename F>
int with_lanes(int64_t width, F&& f) {
    auto whole_or_not = [&](auto lanes, auto items) -> int {
        if (width % kG == 0) return f(lanes, items, std::integral_constant<RowForm, kWhole>{});
        if constexpr (decltype(lanes)::value == 16) {
            if (width < kG) return f(lanes, items, std::integral_constant<RowForm, kShort>{});
        }
        return f(lanes, items, std::integral_constant<RowForm, kRagged>{});
    };
    typedef std::integral_constant<int, 1> One;
    typedef std::integral_constant<int, 2> Two;
    if (width <= 128) return whole_or_not(std::integral_constant<int, 16>{}, One{});
    if (width <= 512) return whole_or_not(std::integral_constant<int, 64>{}, One{});
    if (width <= 1024) return whole_or_not(std::integral_constant<int, 64>{}, Two{});
    if (width <= 2048) return whole_or_not(std::integral_constant<int, 256>{}, One{});
    if (width <= 4096) return whole_or_not(std::integral_constant<int, 256>{}, Two{});
    return whole_or_not(std::integral_constant<int, 1024>{}, One{});
}

Args args_of(const JoinCall& c) {
    const adasum_join_form& f = *c.form;
    Args a{};
    auto vector = [&](int64_t offset) -> const void* {
        return offset < 0 ? nullptr : static_cast<const char*>(c.params) + offset * elem_bytes(c.param_dtype);
    };
    if (f.after) {
        a.after_weight = vector(f.after_weight);
        a.after_bias = vector(f.after_bias);
    }
    a.gate = vector(f.gate);
    if (f.before) {
        a.before_weight = vector(f.before_weight);
        a.before_bias = vector(f.before_bias);
    }
    a.param_type = c.param_dtype;
    a.rows = c.rows;
    a.width = static_cast<int>(f.width);
    a.after = f.after;
    a.before = f.before;
    a.centred = f.norm == ADASUM_NORM_LAYER;
    a.eps = static_cast<float>(f.eps);
    a.scale = static_cast<float>(f.residual_scale);
    a.each = static_cast<float>(1.0 / static_cast<double>(f.width));
    a.mask = make_mask(f.dropout, f.seed, c.step);
    a.drop = a.mask.limit != 0;
    return a;
}
bool is_full(const adasum_join_form& f) { return f.after || f.gate >= 0; }

}  // namespace

template <>
int launch_join<ADASUM_JOIN_TYPES>(const JoinCall& c, const JoinRows& m, void* stream) {
    Args a = args_of(c);
    a.x = static_cast<const T*>(m.x.p);
    a.x_stride = m.x.stride;
    a.residual = static_cast<const S*>(m.residual.p);
    a.residual_stride = m.residual.stride;
    a.to_h = static_cast<S*>(const_cast<void*>(m.h.p));
    a.to_h_stride = m.h.stride;
    a.to_y = static_cast<T*>(const_cast<void*>(m.y.p));
    a.to_y_stride = m.y.stride;
    return with_lanes(c.form->width, [&](auto lanes, auto items, auto form) -> int {
        constexpr int L = decltype(lanes)::value, V = decltype(items)::value;
        constexpr RowForm F = decltype(form)::value;
        typedef Row<L, V, F> R;
        const int64_t needed = (c.rows + R::rows_at_once - 1) / R::rows_at_once, most = 2048;
        return launch(is_full(*c.form) ? join_kernel<L, V, F, true> : join_kernel<L, V, F, false>, needed < most ? needed : most, 1, R::threads, 0,
                      stream, a);
    });
}

template <>
int launch_join_grad<ADASUM_JOIN_TYPES>(const JoinCall& c, const JoinGradRows& m, const JoinSums& to, void* stream) {
    Args a = args_of(c);
    a.x = static_cast<const T*>(m.x.p);
    a.x_stride = m.x.stride;
    a.h = static_cast<const S*>(m.h.p);
    a.h_stride = m.h.stride;
    a.dy = static_cast<const T*>(m.dy.p);
    a.dy_stride = m.dy.stride;
    a.dh = static_cast<const S*>(m.dh.p);
    a.dh_stride = m.dh.stride;
    a.dx = static_cast<T*>(const_cast<void*>(m.dx.p));
    a.dx_stride = m.dx.stride;
    a.dresidual = static_cast<S*>(const_cast<void*>(m.dresidual.p));
    a.dresidual_stride = m.dresidual.stride;
    a.kinds = to.layout.kinds;
    a.parts = to.layout.kinds > 0 ? static_cast<float*>(to.ws) : nullptr;
    const bool full = is_full(*c.form);
    const int groups = to.layout.groups;
    if (groups > 0) {
        const int rc = with_lanes(c.form->width, [&](auto lanes, auto items, auto form) -> int {
            constexpr int L = decltype(lanes)::value, V = decltype(items)::value;
            constexpr RowForm F = decltype(form)::value;
            return launch(full ? join_grad_kernel<L, V, F, true> : join_grad_kernel<L, V, F, false>, groups, 1, Row<L, V, F>::threads, 0, stream, a);
        });
        if (rc != 0) return rc;
    }
    if (to.layout.kinds == 0) return 0;
    Finish f{a.parts, groups, to.layout.kinds, a.width, to.accumulate, {}};
    for (int s = 0; s < to.layout.kinds; ++s) f.to[s] = to.grads[full ? s : s + kBeforeWeight];
    return with_type(to.dtype, [&](auto g) -> int {
        return launch(join_finish_kernel<decltype(g)>, (a.width + 63) / 64, to.layout.kinds, 256, 0, stream, f);
    });
}

}  // namespace adasum
