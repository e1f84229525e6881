// gfx950 kernels of the place where a block's output joins the residual stream, and of its gradient:
//   v = N(x) w + b  (or x),   h = scale residual + gate D(v),   y = N(h) w' + b'
// with N the norm of a row (its mean and spread, or its spread alone) and D dropout.  (Compiled once for each pair of storage types.)
//
// A row lies in the registers of a run of lanes, eight channels a granule, from its loads to its stores: the statistics are sums over the
// lanes, first the mean, then the squares of what is left, so that nothing cancels.  A workgroup goes from row to row with the
// parameters' vectors in registers; the gradient adds those of the parameters up there too, each lane its own channels' in fp32 over the
// workgroup's rows, which meet in fp64 (rounded once into the workspace), and a second launch adds the workgroups' in fp64.  The gradient
// works the statistics out again from the rows that it reads anyhow: nothing is kept for it but the rows themselves.
//
// Memory bounds it: 16384 x 1024 in bf16 with dropout (134 MB) 29 us, its gradient 31 and 4 for the second launch; 32749 x 1024 with an fp32 stream and
// all parts (604 MB), gradient 116 - 119 us, 5.1 TB/s.  The vector units take half to two thirds of that, so that what they do counts: rows that fill their
// lanes have no masks, two sums serve three parameters, weight and gate are one vector (gradient 134 us with five sums and three vectors).  Above 4096 channels with
// all parts the gradient's registers do not suffice: 512 lanes have 256 each, in fp32 24 (filled lanes), 69 (whole granules) and some 480 (ragged rows)
// are kept in memory, in bf16 none, 1 and 27.
#include <hip/hip_runtime.h>

#include "adasum_layers.h"
#include "adasum_mask.h"

#define ADASUM_INLINE __attribute__((always_inline))

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

template <int ORDER>
__device__ __forceinline__ float moved(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), ORDER, 0xf, 0xf, true));
}
// Over each run of 8, 16, 32 or 64 lanes, in every lane of it.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
    if constexpr (LANES == 8) {
        v += moved<0xb1>(v);       // 1 0 3 2 of every four lanes
        v += moved<0x4e>(v);       // 2 3 0 1
        v += moved<0x141>(v);      // the eight lanes from the last to the first
    } else {
        v += moved<0x128>(v);      // eight, four, two and one on, round the sixteen
        v += moved<0x124>(v);
        v += moved<0x122>(v);
        v += moved<0x121>(v);
    }
    if constexpr (LANES > 16) {
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    }
    if constexpr (LANES > 32) {
        const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(b[0]) + __uint_as_float(b[1]);
    }
    return v;
}
// Over the LANES lanes of a row, N sums at a time.  Rows of several waves meet in LDS, in one of two places in turn: a wave that writes the
// next but one sum has passed the barrier behind which all have read this one.
template <int LANES>
struct RowSums {
    static constexpr int kWaves = LANES > 64 ? LANES / 64 : 1, kRows = LANES > 64 && LANES < 256 ? 256 / LANES : 1;
    float (*shared)[2][kRows][kWaves];   // [2]
    int turn = 0;
    template <int N>
    __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lanes_sum<LANES>(v[i]);
        if constexpr (LANES > 64) {
            float(&at)[2][kRows][kWaves] = shared[turn];
            turn ^= 1;
            const int lane = threadIdx.x & 63, row = threadIdx.x / LANES, wave = threadIdx.x % LANES / 64;
            if (lane == 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) at[i][row][wave] = v[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = 0.f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) v[i] += at[i][row][w];
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

// (FILLED: whole granules, as many as there are lanes for: no lane has to ask whether its channels are there)
template <int LANES, int V, RowForm FORM, bool FILLED>
struct Row {
    typedef float Part[V][kG];
    static constexpr int lanes = LANES, threads = LANES > 256 ? LANES : 256;
    static constexpr int rows_at_once = threads / LANES;
    int width, lane;
    __device__ __forceinline__ int at(int k) const { return (k * LANES + lane) * kG; }
    __device__ __forceinline__ bool there(int k, int i) const { return FILLED || (FORM == kWhole ? at(k) < width : at(k) + i < width); }
    // (a last granule that is shorter is loaded as the row's last eight channels, and moved down when it is needed: nothing waits here)
    template <typename E>
    __device__ __forceinline__ void load(Granule<E, kG> (&raw)[V], const E* row) const {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if constexpr (FILLED) load_any(raw[k], row + at(k));
            else if constexpr (FORM == kRagged) load_any(raw[k], row + min(at(k), width - kG));
            else load_row<FORM>(raw[k], row, at(k), width);
        }
    }
    // zeros where there is no channel
    template <typename E>
    __device__ __forceinline__ void values(Part& v, const Granule<E, kG> (&raw)[V]) const {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if constexpr (FORM == kRagged) {
                Granule<E, kG> g = raw[k];
                if (__any(at(k) < width && at(k) > width - kG)) move_down(g, at(k) - min(at(k), width - kG));
                unpack(g, v[k]);
            } else {
                unpack(raw[k], v[k]);
            }
#pragma unroll
            for (int i = 0; i < kG; ++i)
                if (!there(k, i)) v[k][i] = 0.f;
        }
    }
    template <typename E>
    __device__ __forceinline__ void store(E* row, const Part& v) const {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if (FILLED) store_any<kG>(row + at(k), v[k]);
            else if (at(k) < width) store_row<FORM>(row, v[k], at(k), width);
        }
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
        auto sum = [&]() ADASUM_INLINE {
            float t = 0.f;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) t += v[k][i];
            return sums(t);
        };
        auto squares = [&]() ADASUM_INLINE {
            float t = 0.f;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) t = __builtin_fmaf(v[k][i], v[k][i], t);
            return sums(t);
        };
        auto take = [&](float mean) ADASUM_INLINE {
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) v[k][i] = there(k, i) ? v[k][i] - mean : 0.f;
        };
        // Where the mean is above sixteen times the spread, what its own rounding left counts, and is the whole of a row of equal values: the mean of
        // that is taken off too.  (All lanes go round together; to other rows it makes no difference.  For every row it would take 1 - 3 % of
        // batches of 1024 channels, 5 - 17 % of 4096 and 8192 with all parts; as a branch behind the first round 20 - 30 registers.)
        static_assert(LANES <= 64 || rows_at_once == 1, "waves that meet at a barrier have the same row");
        float q = 0.f;
        bool again = true;
        for (int round = 0; round < 2 && __any(again); ++round) {
            float mean = 0.f;
            if (centred) {
                mean = sum() * each;
                take(again ? mean : 0.f);
            }
            q = squares();
            again = again && 256.f * (q * each) < mean * mean;
        }
        const float square = __builtin_fmaf(q, each, eps);
        // (one over an infinity would be 0, and the row its bias)
        const float r = square < __builtin_inff() ? 1.f / __builtin_sqrtf(square) : __builtin_nanf("");
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
            for (int i = 0; i < kG; ++i) d[k][i] = there(k, i) ? r * (d[k][i] - __builtin_fmaf(hat[k][i], inner, mean)) : 0.f;
    }
    // two vectors' product, in the first one's place
    __device__ __forceinline__ void times(Part& v, const Part& w) const {
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < kG; ++i) v[k][i] *= w[k][i];
    }
    __device__ __forceinline__ void mask(bool (&keep)[V][kG], const Mask& m, Step step, long long row) const {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            unsigned w[4];
            mask_words(w, m, step, static_cast<unsigned>(at(k)) / kG, static_cast<unsigned>(row));
            kept(keep[k], w, m.below);
        }
    }
};

// A workgroup's rows: those that it has at once, and the ones after them, whose loads are issued before they are worked on.  All lanes go round
// together; where there are no rows left, lanes take the last one again and store nothing of it.
template <typename R>
struct Rounds {
    long long row, rows;
    bool there;
    __device__ __forceinline__ explicit Rounds(long long n) : rows(n) { at(static_cast<long long>(blockIdx.x) * R::rows_at_once); }
    __device__ __forceinline__ void at(long long first) {
        const long long r = first + threadIdx.x / R::lanes;
        there = r < rows;
        row = there ? r : rows - 1;
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
    int param_type, width, after, before, centred;
    float eps, scale, each;     // each: one over the width
    Mask mask;
    float* parts;               // sums of the parameters' gradients: [workgroup][kind][width]
    int kinds;
};

// FULL: with a norm of x, or a gate.
template <int LANES, int V, RowForm FORM, bool FILLED, bool FULL>
__global__ void __launch_bounds__((Row<LANES, V, FORM, FILLED>::threads))
join_kernel(Args a) {
    typedef Row<LANES, V, FORM, FILLED> R;
    typedef typename R::Part Part;
    __shared__ float shared[2][2][RowSums<LANES>::kRows][RowSums<LANES>::kWaves];
    RowSums<LANES> sums{shared};
    R r;
    r.width = a.width;
    r.lane = threadIdx.x % LANES;
    if (a.rows == 0) return;
    const Step step = step_of(a.mask);
    // (gate * dropout(hat * weight + bias) is taken as dropout(hat * (gate * weight) + gate * bias), two vectors in registers instead of three: either
    // way three roundings to fp32, of products of the gate instead of what it multiplies)
    Part aw, ab, bw, bb;
    if constexpr (FULL) {
        r.param(aw, a.after_weight, a.param_type, 1.f);
        r.param(ab, a.after_bias, a.param_type, 0.f);
        r.param(bw, a.gate, a.param_type, 1.f);
        r.times(aw, bw);
        r.times(ab, bw);
    }
    r.param(bw, a.before_weight, a.param_type, 1.f);
    r.param(bb, a.before_bias, a.param_type, 0.f);
    Granule<T, kG> raw_x[V];
    Granule<S, kG> raw_r[V];
    auto load = [&](long long row) {
        r.load(raw_x, a.x + row * a.x_stride);
        if (a.residual != nullptr) r.load(raw_r, a.residual + row * a.residual_stride);
    };
    Rounds<R> now(a.rows);
    load(now.row);
    const long long each = static_cast<long long>(gridDim.x) * R::rows_at_once;
    for (long long first = static_cast<long long>(blockIdx.x) * R::rows_at_once; first < a.rows; first += each) {
        const long long row = now.row;
        const bool there = now.there;
        Part v, res;
        r.values(v, raw_x);
        if (a.residual != nullptr) r.values(res, raw_r);
        if (first + each < a.rows) {
            now.at(first + each);
            load(now.row);
        }
        if constexpr (FULL) {
            if (a.after) r.normed(v, sums, a.centred, a.eps, a.each);
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) v[k][i] = __builtin_fmaf(v[k][i], aw[k][i], ab[k][i]);
        }
        if (a.mask.drops) {
            bool keep[V][kG];
            r.mask(keep, a.mask, step, row);
#pragma unroll
            for (int k = 0; k < V; ++k) drop(v[k], keep[k], a.mask.factor);
        }
        if (a.residual != nullptr) {
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) v[k][i] = __builtin_fmaf(a.scale, res[k][i], v[k][i]);
        }
        if (a.to_h != nullptr && there) r.store(a.to_h + row * a.to_h_stride, v);
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
            if (there) r.store(a.to_y + row * a.to_y_stride, v);
        }
    }
}

// What is summed over the rows, with D the gradient that comes to dropout, as it leaves of it, and v what the gate and the norm of x get to
// see: x, normed where there is a norm.  The gradients of the weight and bias of that norm are gate * (sum of D v) and gate * (sum of D),
// the gate's is weight * (sum of D v) + bias * (sum of D), both in fp64 by then: where those nearly cancel its error is that of the two sums, of
// the same kind as the rounding of each row's hat * weight + bias would leave.
enum { kAfterProduct, kAfter, kBeforeWeight, kBeforeBias };

template <int LANES, int V, RowForm FORM, bool FILLED, bool FULL>
__global__ void __launch_bounds__((Row<LANES, V, FORM, FILLED>::threads))
join_grad_kernel(Args a) {
    typedef Row<LANES, V, FORM, FILLED> R;
    typedef typename R::Part Part;
    constexpr int kFirst = FULL ? 0 : kBeforeWeight, kSums = kBeforeBias + 1 - kFirst;
    __shared__ float shared[2][2][RowSums<LANES>::kRows][RowSums<LANES>::kWaves];
    RowSums<LANES> sums{shared};
    R r;
    r.width = a.width;
    r.lane = threadIdx.x % LANES;
    if (a.rows == 0) return;
    const Step step = step_of(a.mask);
    Part aw, bw;
    if constexpr (FULL) {
        r.param(aw, a.after_weight, a.param_type, 1.f);
        r.param(bw, a.gate, a.param_type, 1.f);
        r.times(aw, bw);
    }
    r.param(bw, a.before_weight, a.param_type, 1.f);
    Part total[kSums] = {};
    Granule<T, kG> raw_x[V], raw_dy[V];
    Granule<S, kG> raw_h[V], raw_dh[V];
    auto load = [&](long long row) {
        if (a.before) {
            r.load(raw_dy, a.dy + row * a.dy_stride);
            r.load(raw_h, a.h + row * a.h_stride);
        }
        if (a.dh != nullptr) r.load(raw_dh, a.dh + row * a.dh_stride);
        if constexpr (FULL) r.load(raw_x, a.x + row * a.x_stride);
    };
    Rounds<R> now(a.rows);
    load(now.row);
    const long long each = static_cast<long long>(gridDim.x) * R::rows_at_once;
    for (long long first = static_cast<long long>(blockIdx.x) * R::rows_at_once; first < a.rows; first += each) {
        const long long row = now.row;
        const bool there = now.there;
        Part d = {}, dh = {}, hat, v;
        if (a.before) {
            r.values(hat, raw_h);
            r.values(d, raw_dy);
        }
        if (a.dh != nullptr) r.values(dh, raw_dh);
        if constexpr (FULL) r.values(v, raw_x);
        if (first + each < a.rows) {
            now.at(first + each);
            load(now.row);
        }
        // (a row that is not there adds zeros)
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < kG; ++i) {
                if (!there) d[k][i] = dh[k][i] = 0.f;
            }
        if (a.before) {
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
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) d[k][i] += dh[k][i];
        }
        if (a.dresidual != nullptr && there) {
            Part scaled;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) scaled[k][i] = a.scale * d[k][i];
            r.store(a.dresidual + row * a.dresidual_stride, scaled);
        }
        bool keep[V][kG];
        if (a.mask.drops) {
            r.mask(keep, a.mask, step, row);
#pragma unroll
            for (int k = 0; k < V; ++k) drop(d[k], keep[k], a.mask.factor);
        }
        if constexpr (FULL) {
            float spread = 1.f;
            if (a.after) {
                spread = r.normed(v, sums, a.centred, a.eps, a.each);
            } else {
                // (what x holds in dropped places, or a row that is not there, adds nothing)
#pragma unroll
                for (int k = 0; k < V; ++k)
#pragma unroll
                    for (int i = 0; i < kG; ++i)
                        if (!there || (a.mask.drops && !keep[k][i])) v[k][i] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < kG; ++i) {
                    total[kAfterProduct - kFirst][k][i] = __builtin_fmaf(d[k][i], v[k][i], total[kAfterProduct - kFirst][k][i]);
                    total[kAfter - kFirst][k][i] += d[k][i];
                }
            if (a.after) r.norm_grad(d, aw, v, spread, sums, a.centred, a.each);
            else r.times(d, aw);
        }
        if (there) r.store(a.dx + row * a.dx_stride, d);
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
                double sum = 0.0;
#pragma unroll
                for (int w = 0; w < R::rows_at_once; ++w) sum += meet[w][j];
                to[s * a.width + j] = static_cast<float>(sum);
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

// The parameters' gradients out of the workgroups' sums: a workgroup takes 16 channels, sixteen lanes of each share the sums; those of D v
// and D together, as the gate's gradient is made of both.
struct Finish {
    const float* parts;
    int groups, kinds, width, accumulate, param_type;
    const void *after_weight, *after_bias, *gate;     // parameters
    void* to[5];                                      // gradients of after weight and bias, gate, before weight and bias; null: not asked for
};
__device__ __forceinline__ double param_at(const void* p, int type, int j, double instead) {
    if (p == nullptr) return instead;
    if (type == ADASUM_F32) return load_elem(static_cast<const float*>(p) + j);
    return type == ADASUM_BF16 ? load_elem(static_cast<const bf16_t*>(p) + j) : load_elem(static_cast<const f16_t*>(p) + j);
}
template <typename G>
__global__ void __launch_bounds__(256) join_finish_kernel(Finish f) {
    __shared__ double shared[2][16][17];
    const int lane = threadIdx.x & 15, way = threadIdx.x >> 4, j = blockIdx.x * 16 + lane;
    // (the sums of the norm before the next block are the last two)
    const bool of_block = f.kinds == 4 && blockIdx.y == 0;
    const float* const parts = f.parts + (of_block ? 0 : f.kinds - 2) * f.width;
    double sum[2] = {};
    if (j < f.width) {
#pragma unroll 8
        for (int g = way; g < f.groups; g += 16) {
            const float* const at = parts + static_cast<long long>(g) * f.kinds * f.width + j;
            sum[0] += at[0];
            sum[1] += at[f.width];
        }
    }
    shared[0][way][lane] = sum[0];
    shared[1][way][lane] = sum[1];
    __syncthreads();
    if (way != 0 || j >= f.width) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) {
        sum[0] += shared[0][w][lane];
        sum[1] += shared[1][w][lane];
    }
    auto put = [&](void* grad, double v) {
        if (grad == nullptr) return;
        G* const to = static_cast<G*>(grad) + j;
        store_elem(to, static_cast<float>(f.accumulate ? v + load_elem(to) : v));
    };
    if (of_block) {
        const double gate = param_at(f.gate, f.param_type, j, 1.0);
        put(f.to[0], gate * sum[0]);
        put(f.to[1], gate * sum[1]);
        // (without a bias the second sum is not asked for, whatever it is)
        const double weighed = param_at(f.after_weight, f.param_type, j, 1.0) * sum[0];
        put(f.to[2], f.after_bias == nullptr ? weighed : weighed + param_at(f.after_bias, f.param_type, j, 0.0) * sum[1]);
    } else {
        put(f.to[3], sum[0]);
        put(f.to[4], sum[1]);
    }
}

// f(lanes of a row, granules of a lane, form of the row, whether it fills the lanes), as constants.  No more lanes than the row has granules, and a wave
// alone where it can be: no barriers.  (16.8 million elements in bf16, forward and gradient: width 64 in 16 lanes 38 and 63 us, in 8 24 and 37; 256
// in 64 lanes 38 and 64, in 32 25 and 38; 1024 in 128 lanes 32 and 38, in 64 28 and 30 (no operand in a cache); 4096 with all parts in 512 lanes 42 and 72, in 256 with two
// granules 30 and 63; 8192 in 1024 lanes 42 and 101, in 512 39 and 65.)
template <typename F>
int with_lanes(int64_t width, F&& f) {
    auto chosen = [&](auto lanes, auto items) -> int {
        constexpr int kChannels = decltype(lanes)::value * decltype(items)::value * kG;
        const std::integral_constant<RowForm, kWhole> whole;
        if (width == kChannels) return f(lanes, items, whole, std::true_type{});
        if (width % kG == 0) return f(lanes, items, whole, std::false_type{});
        if constexpr (decltype(lanes)::value == 8) {
            if (width < kG) return f(lanes, items, std::integral_constant<RowForm, kShort>{}, std::false_type{});
        }
        return f(lanes, items, std::integral_constant<RowForm, kRagged>{}, std::false_type{});
    };
    typedef std::integral_constant<int, 1> One;
    typedef std::integral_constant<int, 2> Two;
    if (width <= 64) return chosen(std::integral_constant<int, 8>{}, One{});
    if (width <= 128) return chosen(std::integral_constant<int, 16>{}, One{});
    if (width <= 256) return chosen(std::integral_constant<int, 32>{}, One{});
    if (width <= 512) return chosen(std::integral_constant<int, 64>{}, One{});
    if (width <= 1024) return chosen(std::integral_constant<int, 64>{}, Two{});
    if (width <= 2048) return chosen(std::integral_constant<int, 256>{}, One{});
    if (width <= 4096) return chosen(std::integral_constant<int, 256>{}, Two{});
    return chosen(std::integral_constant<int, 512>{}, Two{});
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
    return with_lanes(c.form->width, [&](auto lanes, auto items, auto form, auto filled) -> int {
        constexpr int L = decltype(lanes)::value, V = decltype(items)::value;
        constexpr RowForm F = decltype(form)::value;
        constexpr bool E = decltype(filled)::value;
        typedef Row<L, V, F, E> R;
        const int64_t needed = (c.rows + R::rows_at_once - 1) / R::rows_at_once;
        // (fewer than two rounds: each workgroup takes its rows and goes, so that the chip stays full to the end)
        const int64_t most = join_groups(c.form->width, is_full(*c.form), false);
        return launch(is_full(*c.form) ? join_kernel<L, V, F, E, true> : join_kernel<L, V, F, E, false>, needed < 2 * most ? needed : most, 1, R::threads, 0,
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
        const int rc = with_lanes(c.form->width, [&](auto lanes, auto items, auto form, auto filled) -> int {
            constexpr int L = decltype(lanes)::value, V = decltype(items)::value;
            constexpr RowForm F = decltype(form)::value;
            constexpr bool E = decltype(filled)::value;
            return launch(full ? join_grad_kernel<L, V, F, E, true> : join_grad_kernel<L, V, F, E, false>, groups, 1, Row<L, V, F, E>::threads, 0, stream, a);
        });
        if (rc != 0) return rc;
    }
    if (to.layout.kinds == 0) return 0;
    Finish f{a.parts, groups, to.layout.kinds, a.width, to.accumulate, a.param_type, a.after_weight, a.after_bias, a.gate, {}};
    for (int s = 0; s < 5; ++s) f.to[s] = to.grads[s];
    return with_type(to.dtype, [&](auto g) -> int {
        return launch(join_finish_kernel<decltype(g)>, (a.width + 15) / 16, to.layout.kinds / 2, 256, 0, stream, f);
    });
}

}  // namespace adasum
