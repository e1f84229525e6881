// gfx950 kernels of linear layers whose products are taken in 8-bit floating point with an exponent for each block of 128: the matrix cores
// multiply e4m3 numbers and apply a power of two for each operand's block by themselves.
#include <hip/hip_runtime.h>

#include "adasum_layers.h"
#include "adasum_rows.h"

namespace adasum {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// ---- into 8 bits ----------------------------------------------------------------

__device__ __forceinline__ unsigned finite_size(float v) {
    const unsigned b = __float_as_uint(v) & 0x7fffffffu;
    return b >= 0x7f800000u ? 0u : b;
}
// e + 127 for a block whose largest finite value has these bits: the least e >= -120 with |x| <= 448 * 2^e = 1.75 * 2^(e + 8).
__device__ __forceinline__ unsigned exponent_of(unsigned most) {
    const int e = static_cast<int>(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);
    return static_cast<unsigned>(max(e, 7));
}
// Four values by 2^-e as e4m3 numbers.
__device__ __forceinline__ unsigned in_8_bits(const float* v, unsigned exponent) {
    const float scale = __uint_as_float((254u - exponent) << 23);
    float s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = (__float_as_uint(v[i]) & 0x7f800000u) == 0x7f800000u ? __uint_as_float(0x7fc00000u) : v[i] * scale;
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(s[0], s[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(s[2], s[3], w, true);
    return static_cast<unsigned>(w);
}

// What eight e4m3 numbers by 2^e stand for, in bf16, which holds them all.
__device__ __forceinline__ u32x4 in_bf16(u32x2 q, unsigned exponent) {
    const float scale = __uint_as_float(exponent << 23);
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int from = static_cast<int>(i < 2 ? q.x : q.y);
        const auto two = i % 2 ? __builtin_amdgcn_cvt_pk_f32_fp8(from, true) : __builtin_amdgcn_cvt_pk_f32_fp8(from, false);
        w[i] = __builtin_amdgcn_perm(__float_as_uint(two[1] * scale), __float_as_uint(two[0] * scale), 0x07060302u);
    }
    return w;
}
// The largest over each 16 lanes.
__device__ __forceinline__ unsigned most_of_16(unsigned v) {
    v = max(v, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x128, 0xf, 0xf, true)));
    v = max(v, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x124, 0xf, 0xf, true)));
    v = max(v, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x122, 0xf, 0xf, true)));
    return max(v, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x121, 0xf, 0xf, true)));
}
// Where a token's exponent lies among those of one block of channels: of each 64 tokens, those 16 apart are together, so that a lane of the
// matrix cores' operand has its four tokens' in a word.
__device__ __forceinline__ long long exponent_place(long long t) { return (t & ~63ll) + (t & 15) * 4 + (t >> 4 & 3); }

// Rows of activations into 8 bits (EXACT: into the values those stand for, in bf16), sixteen lanes a block of channels.
template <typename X, RowForm FORM, bool EXACT, int ITEMS>
__global__ void __launch_bounds__(kThreadsRow)
rows8_kernel(const X* __restrict__ x, long long stride, int width, unsigned char* __restrict__ to, unsigned char* __restrict__ e, long long pitch,
             long long tokens, RowWork work) {
    constexpr bool NT = ITEMS > 1;
    every_rows(work, [&](long long first, unsigned n) {
        for (unsigned base = threadIdx.x; base < n; base += kThreadsRow * ITEMS) {
            Granule<X, kG> raw[ITEMS];
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const Place p = place_of(work, first, min(base + kThreadsRow * k, n - 1));
                load_row<FORM, NT>(raw[k], x + p.row * stride, p.at, width);
            }
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                // (n and the step are multiples of sixteen: the lanes of a block are here together)
                const unsigned g = base + kThreadsRow * k;
                if (g < n) {
                    const Place p = place_of(work, first, g);
                    float v[kG];
                    unpack(raw[k], v);
                    unsigned most = 0;
#pragma unroll
                    for (int i = 0; i < kG; ++i) {
                        if (FORM == kWhole ? p.at >= width : p.at + i >= width) v[i] = 0.f;
                        most = max(most, finite_size(v[i]));
                    }
                    const unsigned exponent = exponent_of(most_of_16(most));
                    u32x2 q;
                    q.x = in_8_bits(v, exponent);
                    q.y = in_8_bits(v + 4, exponent);
                    if constexpr (EXACT) {
                        *reinterpret_cast<u32x4*>(to + (p.row * pitch + p.at) * 2) = in_bf16(q, exponent);
                    } else {
                        *reinterpret_cast<u32x2*>(to + p.row * pitch + p.at) = q;
                        if ((g & 15) == 0) e[p.at / kBlock8 * tokens + exponent_place(p.row)] = static_cast<unsigned char>(exponent);
                    }
                }
            }
        }
    });
}
// A weight's rows in 8 bits into the values they stand for.
__global__ void __launch_bounds__(kThreadsRow)
weight_values_kernel(const unsigned char* __restrict__ q, const unsigned char* __restrict__ e, long long e_output, long long e_depth, long long pitch,
                     unsigned char* __restrict__ to, RowWork work) {
    every_rows(work, [&](long long first, unsigned n) {
        for (unsigned g = threadIdx.x; g < n; g += kThreadsRow) {
            const Place p = place_of(work, first, g);
            *reinterpret_cast<u32x4*>(to + (p.row * pitch + p.at) * 2) =
                in_bf16(*reinterpret_cast<const u32x2*>(q + p.row * pitch + p.at), e[p.row / kBlock8 * e_output + p.at / kBlock8 * e_depth]);
        }
    });
}

// A workgroup puts a block of 128 outputs x 128 inputs into 8 bits, as it is and transposed (through LDS).
template <typename T>
__global__ void __launch_bounds__(256) weight8_store_kernel(const T* __restrict__ from, Weight8 w, int blocks_i, long long blocks) {
    __shared__ unsigned most_of[4];
    __shared__ __align__(16) unsigned char turned[kBlock8][kBlock8 + 4];   // [input][output]
    const long long pitch = static_cast<long long>(blocks_i) * kBlock8, pitch_turned = (w.outputs + kBlock8 - 1) / kBlock8 * kBlock8;
    const int r = threadIdx.x / 16, c = threadIdx.x % 16 * 8;
    for (long long block = blockIdx.x; block < blocks; block += gridDim.x) {
        const long long o0 = block / blocks_i * kBlock8, i0 = block % blocks_i * kBlock8;
        float v[8][8];
        unsigned most = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const long long o = o0 + 16 * k + r, left = w.width - (i0 + c);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = 0.f;
            if (o < w.outputs && left > 0) load_some(v[k], from + o * w.width + i0 + c, static_cast<int>(min(left, 8ll)));
#pragma unroll
            for (int i = 0; i < 8; ++i) most = max(most, finite_size(v[k][i]));
        }
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) most = max(most, static_cast<unsigned>(__shfl_xor(static_cast<int>(most), m, 64)));
        __syncthreads();   // (the last block's have been read)
        if ((threadIdx.x & 63) == 0) most_of[threadIdx.x / 64] = most;
        __syncthreads();
        most = max(max(most_of[0], most_of[1]), max(most_of[2], most_of[3]));
        const unsigned exponent = exponent_of(most);
        if (threadIdx.x == 0) w.e[block] = static_cast<unsigned char>(exponent);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            u32x2 q;
            q.x = in_8_bits(v[k], exponent);
            q.y = in_8_bits(v[k] + 4, exponent);
            const long long o = o0 + 16 * k + r;
            if (o < w.outputs) *reinterpret_cast<u32x2*>(w.q + o * pitch + i0 + c) = q;
#pragma unroll
            for (int i = 0; i < 8; ++i) turned[c + i][16 * k + r] = static_cast<unsigned char>((i < 4 ? q.x : q.y) >> (8 * (i % 4)));
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int in = 16 * k + r;
            if (i0 + in < w.width) {
                u32x2 q;
                q.x = *reinterpret_cast<const unsigned*>(&turned[in][c]);
                q.y = *reinterpret_cast<const unsigned*>(&turned[in][c + 4]);
                *reinterpret_cast<u32x2*>(w.turned + (i0 + in) * pitch_turned + o0 + c) = q;
            }
        }
    }
}

// ---- products -------------------------------------------------------------------
//
// The matrix cores multiply e4m3 numbers exactly, but add the products of eight consecutive channels with what lies 2^-13 below the largest's
// power of two cut off (measured: of one large product and a small one beside it, that is what is kept; further apart all of fp32 is). Random
// operands come out off by 1.5e-5 of the result's size.  16-bit results are rounded by far more (2^-9 and 2^-12).  fp32 results are
// therefore computed from the same operands as bf16 numbers, which hold what they stand for: exact products, sums in fp32, half the rate.

// 16 outputs x 16 tokens of a workgroup.  Its four waves share the depth, block by block: a wave reads 128 channels of 16 rows of the weight as
// they are, puts those of the tokens into 8 bits where the matrix cores want them, and multiplies.
template <typename X, typename O, RowForm FORM>
__global__ void __launch_bounds__(256) few_tokens_kernel(Product8 p, long long tiles_o, long long tiles) {
    __shared__ float meet[4][16][17];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, group = lane >> 4;
    const int blocks = static_cast<int>((p.depth + kBlock8 - 1) / kBlock8), depth = static_cast<int>(p.depth);
    const long long pitch = static_cast<long long>(blocks) * kBlock8;
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const long long o0 = tile % tiles_o * 16, t0 = tile / tiles_o * 16;
        const unsigned char* const w = p.w + min(o0 + row, static_cast<long long>(p.outputs) - 1) * pitch + 32 * group;
        const X* const x = static_cast<const X*>(p.x) + min(t0 + row, static_cast<long long>(p.rows) - 1) * p.x_stride;
        const unsigned char* const e = p.e + o0 / kBlock8 * p.e_output;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int b = wave; b < blocks; b += 4) {
            i32x8 a, q;
            const u32x4 lo = *reinterpret_cast<const u32x4*>(w + static_cast<long long>(b) * kBlock8);
            const u32x4 hi = *reinterpret_cast<const u32x4*>(w + static_cast<long long>(b) * kBlock8 + 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a[i] = static_cast<int>(lo[i]);
                a[4 + i] = static_cast<int>(hi[i]);
            }
            Granule<X, 8> raw[4];
            float v[4][8];
            unsigned most = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) load_row<FORM>(raw[k], x, b * kBlock8 + 32 * group + 8 * k, depth);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                unpack(raw[k], v[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (b * kBlock8 + 32 * group + 8 * k + (FORM == kWhole ? 0 : i) >= depth) v[k][i] = 0.f;
                    most = max(most, finite_size(v[k][i]));
                }
            }
            most = max(most, static_cast<unsigned>(__shfl_xor(static_cast<int>(most), 16, 64)));
            most = max(most, static_cast<unsigned>(__shfl_xor(static_cast<int>(most), 32, 64)));
            const unsigned exponent = exponent_of(most);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                q[2 * k] = static_cast<int>(in_8_bits(v[k], exponent));
                q[2 * k + 1] = static_cast<int>(in_8_bits(v[k] + 4, exponent));
            }
            const unsigned of_weight = e[b * p.e_depth];
            if constexpr (sizeof(O) == 4) {
                // (the same eight channels of both, whichever they are)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    u32x2 l, m;
                    l.x = static_cast<unsigned>(a[2 * k]);
                    l.y = static_cast<unsigned>(a[2 * k + 1]);
                    m.x = static_cast<unsigned>(q[2 * k]);
                    m.y = static_cast<unsigned>(q[2 * k + 1]);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, in_bf16(l, of_weight)),
                                                                  __builtin_bit_cast(bf16x8, in_bf16(m, exponent)), acc, 0, 0, 0);
                }
            } else {
                acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q, acc, 0, 0, 0, static_cast<int>(of_weight), 0, static_cast<int>(exponent));
            }
        }
        __syncthreads();   // (the last tile's sums have been read)
#pragma unroll
        for (int i = 0; i < 4; ++i) meet[wave][row][4 * group + i] = acc[i];
        __syncthreads();
        const int t = threadIdx.x / 16, o = threadIdx.x % 16;
        if (t0 + t < p.rows && o0 + o < p.outputs) {
            float sum = (meet[0][t][o] + meet[1][t][o]) + (meet[2][t][o] + meet[3][t][o]);
            if (p.bias != nullptr) {
                if (p.bias_dtype == ADASUM_F32) sum += load_elem(static_cast<const float*>(p.bias) + o0 + o);
                else if (p.bias_dtype == ADASUM_BF16) sum += load_elem(static_cast<const bf16_t*>(p.bias) + o0 + o);
                else sum += load_elem(static_cast<const f16_t*>(p.bias) + o0 + o);
            }
            store_elem(static_cast<O*>(p.out) + (t0 + t) * p.out_stride + o0 + o, sum);
        }
    }
}

// TILE x TILE of the result: what a workgroup of four waves computes.  Both operands come in rows along the depth, 128 bytes a step (a block
// of 8-bit numbers, 64 of 16 bits), and go to LDS past the registers.  A row's eight pieces of 16 bytes lie in LDS at their number
// exclusive-or half the row's, so that sixteen rows' same piece lies in all banks.
template <int TILE>
struct ProductShape {
    static constexpr int threads = 256, frags = TILE / 32;                 // of 16 rows, a wave along each side
    static constexpr int operand_bytes = TILE * kBlock8, buffer_bytes = 2 * operand_bytes, lds_bytes = 2 * buffer_bytes;
    static constexpr int loads = operand_bytes / (threads * 16);           // of an operand, a lane
};

struct Large {
    const unsigned char *w, *x;           // rows `pitch` bytes apart
    const unsigned char *e_w, *e_x;       // exponents (not EXACT): [output / 128 * e_output + block * e_depth], [block * tokens + place]
    long long outputs, rows, e_output, e_depth, tokens;
    const void* bias;
    unsigned pitch;
    int bias_dtype, steps;
    long long out_stride;
    unsigned tiles_o, tiles_t;
};

// Sixteen bytes a lane from base + offset to LDS, a wave's one after the other from `to` on.  (The builtin makes every later read of LDS wait
// for it, of whatever place.  There is no register that the load writes; the loop below waits for it by itself.)
__device__ __forceinline__ void load_to_lds(const unsigned char* base, unsigned offset, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void wait_for_all() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt 0, lgkmcnt 0
    asm volatile("" ::: "memory");
}

// f(0) .. f(N - 1), as constants.
template <int N, int I = 0, typename F>
__device__ __forceinline__ void every(F&& f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        every<N, I + 1>(f);
    }
}

template <bool EXACT, int TILE, typename O>
__global__ void __launch_bounds__(256, TILE == 256 ? 1 : 2) product_kernel(Large p, O* __restrict__ out) {
    typedef ProductShape<TILE> S;
    constexpr int F = S::frags;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned n = die_order(blockIdx.x, gridDim.x);
    const long long o0 = static_cast<long long>(n % p.tiles_o) * TILE, t0 = static_cast<long long>(n / p.tiles_o) * TILE;
    const int wo = wave % 2 * (16 * F), wt = wave / 2 * (16 * F);

    // what a lane loads: a piece of each 32nd row
    const unsigned char *w_base = p.w + o0 * p.pitch, *x_base = p.x + t0 * p.pitch;
    const int w_last = static_cast<int>(min(p.outputs - o0, static_cast<long long>(TILE))) - 1;
    const int x_last = static_cast<int>(min(p.rows - t0, static_cast<long long>(TILE))) - 1;
    unsigned w_at[S::loads], x_at[S::loads];
#pragma unroll
    for (int k = 0; k < S::loads; ++k) {
        const int row = k * 32 + wave * 8 + (lane >> 3), piece = (lane & 7) ^ (row >> 1 & 7);
        w_at[k] = min(row, w_last) * p.pitch + 16 * piece;
        x_at[k] = min(row, x_last) * p.pitch + 16 * piece;
    }
    const unsigned char* e_w = EXACT ? nullptr : p.e_w + min(o0 + wo, p.outputs - 1) / kBlock8 * p.e_output;
    const unsigned char* e_x = EXACT ? nullptr : p.e_x + t0 + wt + (lane & 15) * 4;
    // exponents of this step, of the next, and those that are being loaded; of the tokens, a word for each 64
    constexpr int WORDS = F / 4;
    unsigned of_w = 0, next_w = 0, coming_w = 0, of_x[WORDS] = {}, next_x[WORDS] = {}, coming_x[WORDS] = {};
    const unsigned to = static_cast<unsigned>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)(lds))) + wave * 1024;
    auto load = [&](int buffer) {
        if constexpr (!EXACT) {
            coming_w = *e_w;
#pragma unroll
            for (int k = 0; k < WORDS; ++k) coming_x[k] = *reinterpret_cast<const unsigned*>(e_x + 64 * k);
        }
#pragma unroll
        for (int k = 0; k < S::loads; ++k) {
            load_to_lds(w_base, w_at[k], to + buffer * S::buffer_bytes + k * 4096);
            load_to_lds(x_base, x_at[k], to + buffer * S::buffer_bytes + S::operand_bytes + k * 4096);
        }
    };
    // (behind the last step it is loaded again, and not used)
    int ahead = 0;
    auto next = [&] {
        if (ahead + 1 < p.steps) {
            ++ahead;
            w_base += kBlock8;
            x_base += kBlock8;
            if constexpr (!EXACT) {
                e_w += p.e_depth;
                e_x += p.tokens;
            }
        }
    };
    // what it reads: of a row, pieces g and g + 4 for its group g of lanes
    const int row = lane & 15, group = lane >> 4, first = 16 * (group ^ (row >> 1)), second = 16 * ((group + 4) ^ (row >> 1));
    const char* const w_read = lds + (wo + row) * kBlock8;
    const char* const x_read = lds + S::operand_bytes + (wt + row) * kBlock8;
    u32x4 fw[F][2], fx[F][2];
    auto read_w = [&](int i, int from) {
        fw[i][0] = *reinterpret_cast<const u32x4*>(w_read + from + i * 16 * kBlock8 + first);
        fw[i][1] = *reinterpret_cast<const u32x4*>(w_read + from + i * 16 * kBlock8 + second);
    };
    auto read_x = [&](int j, int from) {
        fx[j][0] = *reinterpret_cast<const u32x4*>(x_read + from + j * 16 * kBlock8 + first);
        fx[j][1] = *reinterpret_cast<const u32x4*>(x_read + from + j * 16 * kBlock8 + second);
    };
    auto whole = [](const u32x4 (&f)[2]) {
        i32x8 r;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            r[k] = static_cast<int>(f[0][k]);
            r[4 + k] = static_cast<int>(f[1][k]);
        }
        return r;
    };
    f32x4 acc[F][F] = {};
    auto multiply = [&](int i, auto number) {
        constexpr int j = decltype(number)::value;
        if constexpr (EXACT) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fw[i][h]), __builtin_bit_cast(bf16x8, fx[j][h]), acc[i][j],
                                                                    0, 0, 0);
        } else {
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(whole(fw[i]), whole(fx[j]), acc[i][j], 0, 0, 0, static_cast<int>(of_w), j % 4,
                                                                         static_cast<int>(of_x[j / 4]));
        }
    };
    auto came = [&] {
        next_w = coming_w;
#pragma unroll
        for (int k = 0; k < WORDS; ++k) next_x[k] = coming_x[k];
    };
    auto turn = [&] {
        of_w = next_w;
#pragma unroll
        for (int k = 0; k < WORDS; ++k) of_x[k] = next_x[k];
    };
    load(0);
    wait_for_all();
    came();
    turn();
    next();
    load(1);
    __builtin_amdgcn_s_barrier();
#pragma unroll
    for (int i = 0; i < F; ++i) {
        read_x(i, 0);
        read_w(i, 0);
    }
    // A step's products come out of registers.  Beside them the next step's operands are read, into the registers of those that have been
    // used for the last time, and the loads of the step after are issued, into the buffer that this step's operands were in.
    for (int s = 0; s < p.steps; ++s) {
        const int other = ~s & 1, from = other * S::buffer_bytes;
        every<F>([&](auto j) { multiply(0, j); });
        __builtin_amdgcn_sched_barrier(0);
        wait_for_all();
        __builtin_amdgcn_s_barrier();
        came();
        next();
        load(other ^ 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 1; i < F - 2; ++i) {
            read_w(i - 1, from);
            every<F>([&](auto j) { multiply(i, j); });
            __builtin_amdgcn_sched_barrier(0);
        }
        read_w(F - 3, from);
        every<F>([&](auto j) {
            multiply(F - 2, j);
            multiply(F - 1, j);
            __builtin_amdgcn_sched_barrier(0);
            read_x(j, from);
        });
        read_w(F - 2, from);
        read_w(F - 1, from);
        __builtin_amdgcn_sched_barrier(0);
        turn();
    }
    // A lane has four consecutive outputs of a token in each 16 x 16.  Through LDS, some tokens of a wave at a time, sixteen lanes get a token's
    // consecutive outputs to store.
    wait_for_all();
    __builtin_amdgcn_s_barrier();
    constexpr int kOutputs = 16 * F, kRow = kOutputs * static_cast<int>(sizeof(O)) + 16;     // bytes of a token's row
    constexpr int kOfLane = 16 / static_cast<int>(sizeof(O)), kLanes = kOutputs / kOfLane;   // outputs that a lane stores, lanes of a token
    char* const mine = lds + wave * (S::lds_bytes / 4);
    constexpr int kTogether = S::lds_bytes / 4 / (16 * kRow) < F ? S::lds_bytes / 4 / (16 * kRow) : F;   // of the token's sixteens
    static_assert(kTogether >= 1, "");
    float bias[F][4] = {};
    if (p.bias != nullptr) {
#pragma unroll
        for (int i = 0; i < F; ++i) {
            const long long o = o0 + wo + 16 * i + 4 * group;
            const int there = static_cast<int>(min(p.outputs - o, 4ll));
            if (there <= 0) continue;
            if (p.bias_dtype == ADASUM_F32) load_some<4>(bias[i], static_cast<const float*>(p.bias) + o, there);
            else if (p.bias_dtype == ADASUM_BF16) load_some<4>(bias[i], static_cast<const bf16_t*>(p.bias) + o, there);
            else load_some<4>(bias[i], static_cast<const f16_t*>(p.bias) + o, there);
        }
    }
#pragma unroll
    for (int j0 = 0; j0 < F; j0 += kTogether) {
#pragma unroll
        for (int j = j0; j < F && j < j0 + kTogether; ++j)
#pragma unroll
            for (int i = 0; i < F; ++i) {
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = acc[i][j][k] + bias[i][k];
                store_any<4>(reinterpret_cast<O*>(mine + (16 * (j - j0) + row) * kRow) + 16 * i + 4 * group, v);
            }
        __builtin_amdgcn_wave_barrier();
        const int tokens = 16 * (F - j0 < kTogether ? F - j0 : kTogether);
#pragma unroll 4
        for (int k = lane; k < tokens * kLanes; k += 64) {
            const int token = k / kLanes, at = k % kLanes * kOfLane;
            const long long t = t0 + wt + 16 * j0 + token, o = o0 + wo + at;
            const u32x4 w = *reinterpret_cast<const u32x4*>(mine + token * kRow + at * static_cast<int>(sizeof(O)));
            if (t >= p.rows || o >= p.outputs) continue;
            O* const to_out = out + t * p.out_stride + o;
            const int there = static_cast<int>(min(p.outputs - o, static_cast<long long>(kOfLane)));
            if (there == kOfLane) {
                store_at<false>(w, reinterpret_cast<u32x4_any*>(to_out));
            } else {
                unsigned words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int e = 0; e < kOfLane; ++e)
                    if (e < there) {
                        if constexpr (sizeof(O) == 4) to_out[e] = __uint_as_float(words[e]);
                        else to_out[e].v = static_cast<unsigned short>(words[e / 2] >> (16 * (e & 1)));
                    }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// The kernel of few tokens does the large ones' work where there are none to fill a tile.
// (A tile's rows are addressed with 32 bits.)
bool is_large(int64_t rows, int64_t outputs, int64_t depth) { return rows > 64 && depth > 0 && depth <= (1 << 22) && outputs >= 16; }
constexpr int64_t kTokenPad = 256;
struct Workspace8 {
    size_t off_more = 0, total = 0;    // the exponents, or the weight's values
};
Workspace8 workspace8(int64_t rows, int64_t outputs, int64_t depth, int out_dtype) {
    Workspace8 w;
    if (!is_large(rows, outputs, depth)) return w;
    const size_t pitch = static_cast<size_t>(blocks8(depth)) * kBlock8;
    const bool exact = out_dtype == ADASUM_F32;
    w.off_more = static_cast<size_t>(rows) * pitch * (exact ? 2 : 1);
    w.total = w.off_more + (exact ? static_cast<size_t>(outputs) * pitch * 2
                                  : static_cast<size_t>(blocks8(depth)) * align_up(static_cast<size_t>(rows), kTokenPad));
    return w;
}

template <bool EXACT, int TILE, typename O>
int launch_large(const Product8& p, const Large& l, void* stream) {
    typedef ProductShape<TILE> S;
    const auto kernel = product_kernel<EXACT, TILE, O>;
    const int rc = static_cast<int>(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::lds_bytes));
    if (rc != 0) return rc;
    return launch(kernel, static_cast<int64_t>(l.tiles_o) * l.tiles_t, 1, S::threads, S::lds_bytes, stream, l, static_cast<O*>(p.out));
}

constexpr int64_t kMany8 = 1 << 19;

// Rows into 8 bits (fp32 results: both operands into the values those stand for), then the product.
template <bool EXACT, typename O>
int large_product(const Product8& p, void* stream) {
    const int64_t blocks = blocks8(p.depth), pitch = blocks * kBlock8, tokens = align_up(static_cast<size_t>(p.rows), kTokenPad);
    const Workspace8 ws = workspace8(p.rows, p.outputs, p.depth, p.out_dtype);
    unsigned char* const x = reinterpret_cast<unsigned char*>(p.ws);
    unsigned char* const more = x + ws.off_more;
    int rc = with_type(p.dtype, [&](auto t) -> int {
        typedef decltype(t) X;
        const RowGrid g = row_grid(p.rows, pitch, p.dtype, kMany8);
        return with_form(row_form(p.depth, kG), [&](auto form) -> int {
            constexpr RowForm F = decltype(form)::value;
            return with_items<X>(g, [&](auto items) -> int {
                return launch(rows8_kernel<X, F, EXACT, decltype(items)::value>, g.groups, 1, kThreadsRow, 0, stream, static_cast<const X*>(p.x),
                              p.x_stride, p.depth, x, EXACT ? nullptr : more, pitch, tokens, g.work);
            });
        });
    });
    if (rc != 0) return rc;
    if (EXACT) {
        const RowGrid g = row_grid(p.outputs, pitch, ADASUM_F32, 0);
        rc = launch(weight_values_kernel, g.groups, 1, kThreadsRow, 0, stream, p.w, p.e, p.e_output, p.e_depth, pitch, more, g.work);
        if (rc != 0) return rc;
    }
    Large l{};
    l.w = EXACT ? more : p.w;
    l.x = x;
    l.e_w = p.e;
    l.e_x = EXACT ? nullptr : more;
    l.pitch = pitch * (EXACT ? 2 : 1);
    l.outputs = p.outputs;
    l.rows = p.rows;
    l.e_output = p.e_output;
    l.e_depth = p.e_depth;
    l.tokens = tokens;
    l.bias = p.bias;
    l.bias_dtype = p.bias_dtype;
    l.steps = static_cast<int>(l.pitch / kBlock8);
    l.out_stride = p.out_stride;
    auto tiles = [&](int64_t n, int tile) { return static_cast<unsigned>((n + tile - 1) / tile); };
    const bool wide = static_cast<int64_t>(tiles(p.outputs, 256)) * tiles(p.rows, 256) >= 192;
    l.tiles_o = tiles(p.outputs, wide ? 256 : 128);
    l.tiles_t = tiles(p.rows, wide ? 256 : 128);
    return wide ? launch_large<EXACT, 256, O>(p, l, stream) : launch_large<EXACT, 128, O>(p, l, stream);
}

}  // namespace

int launch_weight8_store(const void* w, int dtype, const Weight8& to, void* stream) {
    const int64_t blocks_i = blocks8(to.width), blocks = blocks8(to.outputs) * blocks_i;
    return with_type(dtype, [&](auto t) -> int {
        typedef decltype(t) T;
        return launch(weight8_store_kernel<T>, at_most_groups(blocks), 1, 256, 0, stream, static_cast<const T*>(w), to, blocks_i, blocks);
    });
}

size_t product8_workspace(int64_t rows, int64_t outputs, int64_t depth, int out_dtype) { return workspace8(rows, outputs, depth, out_dtype).total; }

int launch_product8(const Product8& p, void* stream) {
    if (is_large(p.rows, p.outputs, p.depth)) {
        switch (p.out_dtype) {
            case ADASUM_F32: return large_product<true, float>(p, stream);
            case ADASUM_BF16: return large_product<false, bf16_t>(p, stream);
            default: return large_product<false, f16_t>(p, stream);
        }
    }
    return with_type(p.dtype, [&](auto x) -> int {
        typedef decltype(x) X;
        return with_type(p.out_dtype, [&](auto out) -> int {
            typedef decltype(out) O;
            return with_form(row_form(p.depth, 8), [&](auto form) -> int {
                constexpr RowForm F = decltype(form)::value;
                const int64_t tiles_o = (p.outputs + 15) / 16, tiles = tiles_o * ((p.rows + 15) / 16);
                return launch(few_tokens_kernel<X, O, F>, at_most_groups(tiles), 1, 256, 0, stream, p, tiles_o, tiles);
            });
        });
    });
}

}  // namespace adasum
