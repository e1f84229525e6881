// gfx950 kernels of a linear layer's gradients from an activation checkpoint: dW = dy^T x over the tokens, and dy's sums.
#include <hip/hip_runtime.h>

#include "adasum_layers.h"
#include "adasum_rows.h"

namespace adasum {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mfma(bf16_t, u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma(f16_t, u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// What the matrix cores multiply: the 16-bit types as they are; fp32 as three bf16 parts, each the leading eight bits of what the
// parts before it leave, which is exact (infinities and NaN are the first part alone).
template <typename T> struct Products { typedef T type; static constexpr int planes = 1; };
template <> struct Products<float> { typedef bf16_t type; static constexpr int planes = 3; };

__device__ __forceinline__ void part_of(float x, unsigned (&p)[3]) {
    const unsigned a = __float_as_uint(x);
    p[0] = a >> 16;
    if ((a & 0x7f800000u) == 0x7f800000u) {
        if ((a & 0x7fffffu) != 0) p[0] |= 0x40u;
        p[1] = p[2] = 0;
        return;
    }
    const float r = x - __uint_as_float(a & 0xffff0000u);
    const unsigned b = __float_as_uint(r);
    p[1] = b >> 16;
    p[2] = __float_as_uint(r - __uint_as_float(b & 0xffff0000u)) >> 16;
}

constexpr int kPad = 8;
constexpr int kRowLds = kStepTokens + kPad;

// A workgroup of four waves: 128 x 128 of dW over the steps of one part of the tokens, each wave a quarter.  Both operands are staged
// with the tokens innermost, as the matrix cores want them.
template <typename D, typename T>
__global__ void __launch_bounds__(256)
weight_grad_kernel(const signed char* __restrict__ q, const signed char* __restrict__ e, long long rows, int width, long long pitch,
                   const D* __restrict__ dy, long long dy_stride, int outputs, T* __restrict__ grad, int accumulate,
                   float* __restrict__ parts, long long steps, int tiles_i) {
    typedef typename Products<D>::type E;
    constexpr int P = Products<D>::planes;
    __shared__ __align__(16) unsigned short as[P][kGradTile][kRowLds];
    __shared__ __align__(16) unsigned short bs[kGradTile][kRowLds];
    const int o0 = static_cast<int>(blockIdx.x / tiles_i) * kGradTile, i0 = static_cast<int>(blockIdx.x % tiles_i) * kGradTile;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wo = (wave >> 1) * 64, wi = (wave & 1) * 64;
    const int st = threadIdx.x >> 3, sc = (threadIdx.x & 7) * 16;   // what this lane stages: a token, 16 channels
    f32x16 acc[2][2] = {};
    const long long t_begin = static_cast<long long>(blockIdx.y) * steps * kStepTokens;
    const long long t_end = min(rows, t_begin + steps * kStepTokens);
    for (long long t0 = t_begin; t0 < t_end; t0 += kStepTokens) {
        const long long t = t0 + st;
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v[8];
            const int o = o0 + sc + 8 * h;
            load_some<8>(v, dy + t * dy_stride + o, t < t_end ? outputs - o : 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (P == 3) {
                    unsigned p[3];
                    part_of(v[j], p);
#pragma unroll
                    for (int k = 0; k < 3; ++k) as[k][sc + 8 * h + j][st] = static_cast<unsigned short>(p[k]);
                } else {
                    as[0][sc + 8 * h + j][st] = static_cast<unsigned short>(bits_of(E{}, v[j]));
                }
            }
        }
        const int i = i0 + sc;
        u32x4 kept = {0, 0, 0, 0};
        float step = 0.f;
        if (t < t_end && i < pitch) {
            kept = *reinterpret_cast<const u32x4*>(q + t * pitch + i);
            const int ex = e[t * (pitch / kBlock) + i / kBlock];
            step = __uint_as_float(ex == -128 ? 0x7fc00000u : static_cast<unsigned>(ex + 127) << 23);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float x = static_cast<float>(static_cast<signed char>(kept[j / 4] >> (8 * (j % 4)))) * step;
            bs[sc + j][st] = static_cast<unsigned short>(bits_of(E{}, x));
        }
        __syncthreads();
#pragma unroll
        for (int k0 = 0; k0 < kStepTokens; k0 += 16) {
            u32x4 b[2];
#pragma unroll
            for (int n = 0; n < 2; ++n)
                b[n] = *reinterpret_cast<const u32x4*>(&bs[wi + 32 * n + (lane & 31)][k0 + 8 * (lane >> 5)]);
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const u32x4 a = *reinterpret_cast<const u32x4*>(&as[p][wo + 32 * m + (lane & 31)][k0 + 8 * (lane >> 5)]);
#pragma unroll
                    for (int n = 0; n < 2; ++n) acc[m][n] = mfma(E{}, a, b[n], acc[m][n]);
                }
        }
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int o = o0 + wo + 32 * m + 8 * (r / 4) + 4 * (lane >> 5) + r % 4, i = i0 + wi + 32 * n + (lane & 31);
                if (o < outputs && i < width) {
                    const long long at = static_cast<long long>(o) * width + i;
                    if (parts != nullptr) {
                        parts[static_cast<long long>(blockIdx.y) * outputs * width + at] = acc[m][n][r];
                    } else {
                        store_elem(grad + at, accumulate ? acc[m][n][r] + load_elem(grad + at) : acc[m][n][r]);
                    }
                }
            }
}

// dy's sums: a workgroup takes 64 outputs over one part of the tokens.
template <typename D, typename T>
__global__ void __launch_bounds__(256)
bias_kernel(long long rows, const D* __restrict__ dy, long long dy_stride, int outputs, T* __restrict__ bias, int accumulate,
            float* __restrict__ parts, long long tokens) {
    __shared__ double sums[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int o = static_cast<int>(blockIdx.x) * 64 + lane;
    const long long t_begin = blockIdx.y * tokens, t_end = min(rows, t_begin + tokens);
    double sum = 0;
    if (o < outputs)
        for (long long t = t_begin + wave; t < t_end; t += 4) sum += load_elem(dy + t * dy_stride + o);
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || o >= outputs) return;
    const float s = static_cast<float>(sums[0][lane] + sums[1][lane] + (sums[2][lane] + sums[3][lane]));
    if (parts != nullptr) parts[static_cast<long long>(blockIdx.y) * outputs + o] = s;
    else store_elem(bias + o, accumulate ? s + load_elem(bias + o) : s);
}

// out (+)= the sum of the parts, in their order.
template <typename T>
__global__ void __launch_bounds__(256)
join_parts_kernel(const float* __restrict__ parts, int n_parts, long long n, T* __restrict__ out, int accumulate) {
    for (long long at = blockIdx.x * 256ll + threadIdx.x; at < n; at += 256ll * gridDim.x) {
        float s = 0.f;
        for (int p = 0; p < n_parts; ++p) s += parts[p * n + at];
        store_elem(out + at, accumulate ? s + load_elem(out + at) : s);
    }
}

template <typename T>
int join(const float* parts, int64_t n_parts, int64_t n, T* out, int accumulate, void* stream) {
    return launch(join_parts_kernel<T>, at_most_groups((n + 255) / 256), 1, 256, 0, stream, parts, n_parts, n, out, accumulate);
}

}  // namespace

WeightSplit weight_split(int64_t rows, int64_t width, int64_t outputs, int dtype) {
    (void)dtype;
    WeightSplit s;
    const int64_t tiles = ((outputs + kGradTile - 1) / kGradTile) * ((width + kGradTile - 1) / kGradTile);
    const int64_t steps = (rows + kStepTokens - 1) / kStepTokens;
    int64_t parts = tiles > 0 ? 512 / tiles : 1;
    if (parts > steps / 8) parts = steps / 8;
    if (parts < 1) parts = 1;
    s.steps = (steps + parts - 1) / parts;
    s.parts = s.steps > 0 ? (steps + s.steps - 1) / s.steps : 1;
    if (s.parts > 1) {
        s.off_bias = align_up(static_cast<size_t>(s.parts) * outputs * width * 4, 256);
        s.total = s.off_bias + static_cast<size_t>(s.parts) * outputs * 4;
    }
    return s;
}

int launch_weight_grad(const WeightGrad& g, void* stream) {
    return with_types(g.dtype, g.grad_dtype, [&](auto d, auto t) -> int {
        typedef decltype(d) D;
        typedef decltype(t) T;
        if constexpr (sizeof(D) == 8 || sizeof(T) == 8) {
            return static_cast<int>(hipErrorInvalidValue);   // (refused before)
        } else {
            const bool split = g.split.parts > 1;
            float* const parts = split ? reinterpret_cast<float*>(g.ws) : nullptr;
            float* const bias_parts = split ? reinterpret_cast<float*>(g.ws + g.split.off_bias) : nullptr;
            const D* const dy = static_cast<const D*>(g.dy);
            const int64_t tiles_o = (g.outputs + kGradTile - 1) / kGradTile, tiles_i = (g.x.width + kGradTile - 1) / kGradTile;
            int rc = 0;
            if (tiles_i > 0) {
                T* const grad = static_cast<T*>(g.grad);
                rc = launch(weight_grad_kernel<D, T>, tiles_o * tiles_i, g.split.parts, 256, 0, stream, reinterpret_cast<const signed char*>(g.x.q),
                            reinterpret_cast<const signed char*>(g.x.e), g.x.rows, g.x.width, g.x.pitch, dy, g.dy_stride, g.outputs, grad,
                            g.accumulate, parts, g.split.steps, tiles_i);
                if (rc == 0 && split) rc = join(parts, g.split.parts, g.outputs * g.x.width, grad, g.accumulate, stream);
            }
            if (rc != 0 || g.bias == nullptr) return rc;
            T* const bias = static_cast<T*>(g.bias);
            rc = launch(bias_kernel<D, T>, (g.outputs + 63) / 64, g.split.parts, 256, 0, stream, g.x.rows, dy, g.dy_stride, g.outputs, bias,
                        g.accumulate, bias_parts, g.split.steps * kStepTokens);
            return rc == 0 && split ? join(bias_parts, g.split.parts, g.outputs, bias, g.accumulate, stream) : rc;
        }
    });
}

}  // namespace adasum
