// gfx950 kernels of activation checkpoints in 8 bits: store, load, and the gradient through an activation function whose input is
// a checkpoint.  (The gradients of a linear layer from one are in adasum_weight_grad.hip.)
//
// All three stream: a lane takes eight channels of a row, four lanes a block of 32 that shares an exponent.  The exponent comes
// from the bits of the block's largest magnitude, scaling by a power of two is exact, and the sum with 3 * 2^22 rounds to nearest
// even and leaves the whole number in the low byte.  Memory bounds them: 32768 x 4096 bf16 stored and loaded again (406 MB each) take 80 and
// 67 us, the gradient (675 MB) through relu and silu 109 - 112 us, through gelu 117 and its other form 122, where the vector units are
// as busy: 5.1 - 6.2 TB/s.  In fp32 116 us each (675 MB) and 207 us for every gradient (1.21 GB), 5.8 TB/s.
#include <hip/hip_runtime.h>

#include "adasum_layers.h"
#include "adasum_rows.h"

namespace adasum {
namespace {

__device__ __forceinline__ unsigned quad_max(unsigned v) {
    v = max(v, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0xb1, 0xf, 0xf, true)));   // lanes 1 0 3 2
    return max(v, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x4e, 0xf, 0xf, true)));   // 2 3 0 1
}

__device__ __forceinline__ unsigned low_bytes(unsigned a, unsigned b, unsigned c, unsigned d) {
    const unsigned ab = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), cd = __builtin_amdgcn_perm(d, c, 0x04000c0cu);
    return ab | cd;
}

// 2^e; NaN for the mark of a block that is not finite.
__device__ __forceinline__ float step_of(int e) {
    return __uint_as_float(e == -128 ? 0x7fc00000u : static_cast<unsigned>(e + 127) << 23);
}

__device__ __forceinline__ void kept_values(float (&x)[kG], u32x2 q, float step) {
    const unsigned w[2] = {q.x, q.y};
#pragma unroll
    for (int i = 0; i < kG; ++i) x[i] = static_cast<float>(static_cast<signed char>(w[i / 4] >> (8 * (i % 4)))) * step;
}

// Slopes of the activation functions.  A lane of the stream has some 40 instructions per element before the vector units bound it, so each
// takes one exponential and one reciprocal (of the hardware, one unit in the last place each).
//
// gelu: with the normal density f and its upper tail Q, the slope at -a is Q(a) - a f(a) = f(a) (M(a) - a), M = Q / f, and that at
// a is 1 minus it.  M falls smoothly from 1.25 to 1 / a: a polynomial in t = 1 / (1 + a / 4), fitted here for the least largest
// error relative to what fp32's own roundings leave (M + a) at 0 <= a <= 16; 1.7 % of that.  What is evaluated is M / sqrt(2 pi).
// Against fp64 the slope is off by 1.1e-7 at most.  Relative to f(a) (M(a) + a) on the negative side, the rounding of the exponential's
// argument and that of its constant show: 4.4e-7 below 4, 1.4e-6 at 9, 7.6e-6 at 12, which is far below the rounding of a result of
// 16 bits.  For results in fp32 (FINE) a^2 is exact, as kept values have seven bits, and what its product with the constant loses,
// and the constant itself, multiplies the exponential: 4.5e-7 down to -12.5, where the terms leave fp32's range.  (32768 x 4096:
// 207 us in fp32 with and without that, where memory bounds it; for 16 bits it would cost 123 us instead of 117.)
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// s(z) + f s(z) s(-z) for s(z) = 1 / (1 + exp(-z)), from e = exp(-|z|): s is 1 / (1 + e), or e / (1 + e) below zero, and the product
// e / (1 + e)^2 on both sides.  (e is held times 2^16: its product with f may be a normal number where e is none.)
__device__ __forceinline__ float logistic_slope(float z, float f) {
    const float e = exp2_fast(__builtin_fmaf(__builtin_fabsf(z), -1.4426950408889634f, 16.f)), less = e * 0x1p-16f;
    const float r = __builtin_amdgcn_rcpf(1.f + less);
    return __builtin_fmaf(f * 0x1p-16f, e * r * r, z < 0.f ? less * r : r);
}
template <int ACT, bool FINE>
__device__ __forceinline__ float slope(float x) {
    if constexpr (ACT == ADASUM_ACT_RELU) {
        return x != x ? x : x > 0.f ? 1.f : 0.f;
    } else if constexpr (ACT == ADASUM_ACT_GELU) {
        const float a = __builtin_fabsf(x), t = __builtin_amdgcn_rcpf(__builtin_fmaf(a, 0.25f, 1.f));
        float m = -0.09283597022294998f;
        m = __builtin_fmaf(m, t, 0.34739378094673157f);
        m = __builtin_fmaf(m, t, -0.27806541323661804f);
        m = __builtin_fmaf(m, t, 0.2922147512435913f);
        m = __builtin_fmaf(m, t, 0.01876537874341011f);
        m = __builtin_fmaf(m, t, 0.11390205472707748f);
        m = __builtin_fmaf(m, t, 0.09862539917230606f);
        constexpr double kPower = -0.72134752044448170;   // - log2(e) / 2
        constexpr float kHigh = static_cast<float>(kPower), kLow = static_cast<float>(kPower - static_cast<double>(kHigh));
        const float b = FINE ? fminf(a, 64.f) : a, bb = b * b, power = bb * kHigh;   // (beyond, nothing is left; NaN comes in with m)
        float e = exp2_fast(power);
        if constexpr (FINE) e = __builtin_fmaf(e, __builtin_fmaf(bb, kLow, __builtin_fmaf(bb, kHigh, -power)) * 0.6931471805599453f, e);
        const float s = e * __builtin_fmaf(a, -0.3989422804014327f, m * t);
        return x < 0.f ? s : 1.f - s;
    } else if constexpr (ACT == ADASUM_ACT_GELU_TANH) {
        // beyond 30 the slope is 0 or 1 to the last bit, and the cube may overflow
        const float y = x > 30.f ? 30.f : x < -30.f ? -30.f : x;
        const float yy = y * y;
        return logistic_slope(1.5957691216057308f * y * __builtin_fmaf(yy, 0.044715f, 1.f),
                              1.5957691216057308f * y * __builtin_fmaf(yy, 3 * 0.044715f, 1.f));
    } else {
        return logistic_slope(x, x);
    }
}

template <typename T, RowForm FORM, int ITEMS>
__global__ void __launch_bounds__(kThreadsRow)
store_kernel(const T* __restrict__ x, long long stride, int width, long long pitch, signed char* __restrict__ q, signed char* __restrict__ e,
             RowWork work) {
    // (of large tensors only x: eight bytes a lane are slower so)
    constexpr bool NT = ITEMS > 1;
    every_rows(work, [&](long long first, unsigned n) {
        for (unsigned base = threadIdx.x; base < n; base += kThreadsRow * ITEMS) {
            Granule<T, kG> raw[ITEMS];
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const Place p = place_of(work, first, min(base + kThreadsRow * k, n - 1));
                load_row<FORM, NT>(raw[k], x + p.row * stride, p.at, width);
            }
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                // (n and the step are multiples of four: the lanes of a block are here together)
                const unsigned g = base + kThreadsRow * k;
                if (g < n) {
                    const Place p = place_of(work, first, g);
                    float v[kG];
                    unpack(raw[k], v);
                    // (channels up to the pitch that do not exist)
#pragma unroll
                    for (int i = 0; i < kG; ++i)
                        if (FORM == kWhole ? p.at >= width : p.at + i >= width) v[i] = 0.f;
                    unsigned most = 0;
#pragma unroll
                    for (int i = 0; i < kG; ++i) most = max(most, __float_as_uint(v[i]) & 0x7fffffffu);
                    most = quad_max(most);
                    const bool bad = most >= 0x7f800000u;
                    const int exponent = max(static_cast<int>(most >> 23) - 133, -120);
                    const float scale = __uint_as_float(static_cast<unsigned>(127 - exponent) << 23);
                    unsigned b[kG];
#pragma unroll
                    for (int i = 0; i < kG; ++i) b[i] = __float_as_uint(fminf(fmaxf(v[i] * scale, -127.f), 127.f) + 12582912.f);
                    u32x2 packed;
                    packed.x = bad ? 0u : low_bytes(b[0], b[1], b[2], b[3]);
                    packed.y = bad ? 0u : low_bytes(b[4], b[5], b[6], b[7]);
                    *reinterpret_cast<u32x2*>(q + p.row * pitch + p.at) = packed;
                    if ((g & 3) == 0) e[p.row * (pitch / kBlock) + p.at / kBlock] = static_cast<signed char>(bad ? -128 : exponent);
                }
            }
        }
    });
}

template <typename T, RowForm FORM, int ITEMS>
__global__ void __launch_bounds__(kThreadsRow)
load_kernel(const signed char* __restrict__ q, const signed char* __restrict__ e, int width, long long pitch, T* __restrict__ out,
            long long stride, RowWork work) {
    constexpr bool NT = ITEMS > 1;
    every_rows(work, [&](long long first, unsigned n) {
        for (unsigned base = threadIdx.x; base < n; base += kThreadsRow * ITEMS) {
            u32x2 kept[ITEMS];
            int exponent[ITEMS];
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const Place p = place_of(work, first, min(base + kThreadsRow * k, n - 1));
                kept[k] = *reinterpret_cast<const u32x2*>(q + p.row * pitch + p.at);
                exponent[k] = e[p.row * (pitch / kBlock) + p.at / kBlock];
            }
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const unsigned g = base + kThreadsRow * k;
                if (g < n) {
                    const Place p = place_of(work, first, g);
                    float v[kG];
                    kept_values(v, kept[k], step_of(exponent[k]));
                    store_row<FORM, NT>(out + p.row * stride, v, p.at, width);
                }
            }
        }
    });
}

// (dy and dx may be the same rows: a lane loads what it stores before it does)
template <typename T, int ACT, RowForm FORM, int ITEMS>
__global__ void __launch_bounds__(kThreadsRow)
act_grad_kernel(const signed char* __restrict__ q, const signed char* __restrict__ e, int width, long long pitch, const T* dy,
                long long dy_stride, T* dx, long long dx_stride, RowWork work) {
    constexpr bool NT = ITEMS > 1;
    every_rows(work, [&](long long first, unsigned n) {
        for (unsigned base = threadIdx.x; base < n; base += kThreadsRow * ITEMS) {
            u32x2 kept[ITEMS];
            int exponent[ITEMS];
            Granule<T, kG> raw[ITEMS];
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const Place p = place_of(work, first, min(base + kThreadsRow * k, n - 1));
                kept[k] = *reinterpret_cast<const u32x2*>(q + p.row * pitch + p.at);
                exponent[k] = e[p.row * (pitch / kBlock) + p.at / kBlock];
                load_row<FORM, NT>(raw[k], dy + p.row * dy_stride, p.at, width);
            }
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const unsigned g = base + kThreadsRow * k;
                if (g < n) {
                    const Place p = place_of(work, first, g);
                    float v[kG], d[kG];
                    kept_values(v, kept[k], step_of(exponent[k]));
                    unpack(raw[k], d);
#pragma unroll
                    for (int i = 0; i < kG; ++i) v[i] = d[i] * slope<ACT, sizeof(T) == 4>(v[i]);
                    store_row<FORM, NT>(dx + p.row * dx_stride, v, p.at, width);
                }
            }
        }
    });
}

// Four granules of a lane in flight, past the caches, or one through them.  Rows of 1024 (in thousands of granules: microseconds with one and
// with four of them), operands that no cache holds: loads of bf16 524: 4.7 and 4.3; 4194: 21.2 and 19.7; 16777: 73 and 67.  Stores 524: 5.0 and
// 5.5; 2097: 13.6 and 12.3; 16777: 77 and 79.  In fp32, where a granule is 32 bytes, four are slower: loads 4194: 35 and 40; 16777: 116
// and 137, stores 116 and 124.  Gradients of relu in bf16 524: 6.0 and 6.3; 1049: 10.5 and 9.7; 16777: 114 and 109, of silu 4194: 31.7 and
// 32.1; 16777: 115 and 110; gelu, whose vector instructions take as long as its memory, 4194: 32 and 34; 16777: 118 and 122, and its
// other form 34 and 37, 124 and 129.  fp16 is like bf16.  Operands that were just used are faster with one (4194, bf16: stores 18.5 and 21).
constexpr int64_t kMany = 1 << 19, kManyOfSilu = 1 << 21;

}  // namespace

int launch_store(const void* x, int dtype, int64_t x_stride, const Kept& to, void* stream) {
    const RowGrid g = row_grid(to.rows, to.pitch, dtype, kMany);
    return with_type(dtype, [&](auto t) -> int {
        typedef decltype(t) T;
        return with_form(row_form(to.width, kG), [&](auto form) -> int {
            constexpr RowForm F = decltype(form)::value;
            return with_items<T>(g, [&](auto items) -> int {
                return launch(store_kernel<T, F, decltype(items)::value>, g.groups, 1, kThreadsRow, 0, stream, static_cast<const T*>(x), x_stride,
                              to.width, to.pitch, reinterpret_cast<signed char*>(const_cast<int8_t*>(to.q)),
                              reinterpret_cast<signed char*>(const_cast<int8_t*>(to.e)), g.work);
            });
        });
    });
}

int launch_load(const Kept& k, void* out, int dtype, int64_t out_stride, void* stream) {
    const RowGrid g = row_grid(k.rows, k.pitch, dtype, kMany);
    return with_type(dtype, [&](auto t) -> int {
        typedef decltype(t) T;
        auto go = [&](auto form) -> int {
            constexpr RowForm F = decltype(form)::value;
            return with_items<T>(g, [&](auto items) -> int {
                return launch(load_kernel<T, F, decltype(items)::value>, g.groups, 1, kThreadsRow, 0, stream,
                              reinterpret_cast<const signed char*>(k.q), reinterpret_cast<const signed char*>(k.e), k.width, k.pitch,
                              static_cast<T*>(out), out_stride, g.work);
            });
        };
        // (short rows are stored like ragged ones)
        return k.width % kG == 0 ? go(std::integral_constant<RowForm, kWhole>{}) : go(std::integral_constant<RowForm, kRagged>{});
    });
}

int launch_act_grad(const Kept& k, int act, const void* dy, int dtype, int64_t dy_stride, void* dx, int64_t dx_stride, void* stream) {
    const RowGrid g = row_grid(k.rows, k.pitch, dtype, act == ADASUM_ACT_RELU ? kMany : act == ADASUM_ACT_SILU ? kManyOfSilu : INT64_MAX);
    return with_type(dtype, [&](auto t) -> int {
        typedef decltype(t) T;
        return with_form(row_form(k.width, kG), [&](auto form) -> int {
            constexpr RowForm F = decltype(form)::value;
            auto go = [&](auto chosen) -> int {
                constexpr int ACT = decltype(chosen)::value;
                auto run = [&](auto items) -> int {
                    return launch(act_grad_kernel<T, ACT, F, decltype(items)::value>, g.groups, 1, kThreadsRow, 0, stream,
                                  reinterpret_cast<const signed char*>(k.q), reinterpret_cast<const signed char*>(k.e), k.width, k.pitch,
                                  static_cast<const T*>(dy), dy_stride, static_cast<T*>(dx), dx_stride, g.work);
                };
                if constexpr (ACT == ADASUM_ACT_GELU || ACT == ADASUM_ACT_GELU_TANH) return run(std::integral_constant<int, 1>{});
                else return with_items<T>(g, run);
            };
            switch (act) {
                case ADASUM_ACT_RELU: return go(std::integral_constant<int, ADASUM_ACT_RELU>{});
                case ADASUM_ACT_GELU: return go(std::integral_constant<int, ADASUM_ACT_GELU>{});
                case ADASUM_ACT_GELU_TANH: return go(std::integral_constant<int, ADASUM_ACT_GELU_TANH>{});
                default: return go(std::integral_constant<int, ADASUM_ACT_SILU>{});
            }
        });
    });
}

}  // namespace adasum
