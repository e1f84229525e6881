// gfx950 kernels of linear layers whose products are taken in 8-bit floating point with an exponent for each block of 128: the matrix cores
// multiply e4m3 numbers and apply a power of two for each operand's block by themselves.
//
// Times (bf16): 8192 -> 8192, 8192 rows 410 us for the product alone (2.68 PFLOP/s; a library product with one scale 2.74); 4096 -> 1024, 16384
// rows 61 (2.25; library 2.42) and 41 to put the rows into 8 bits (201 MB, 4.9 TB/s); 1024 -> 4096, 32768 rows 175 and 25; one row of
// 1024 -> 4096 4.4.  fp32: 4096 -> 1024, 4093 rows 40, 19 and 5 (the weight's values).  A weight of 4096 x 1024 into 8 bits 7 - 10.
#include <hip/hip_runtime.h>

#include "adasum_layers.h"
#include "adasum_rows.h"

namespace adasum {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Where operands lie: in panels of 64 bytes of the depth, all rows of a panel one after the other, so that sixteen rows' pieces of a panel are
// a kilobyte of memory in one.
constexpr int kPanel = 64;
__device__ __forceinline__ long long panel_place(long long rows, long long row, int byte) {
    return (byte / kPanel * rows + row) * kPanel + byte % kPanel;
}

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
// Where a token's exponent lies among those of one block of channels: of each 128 tokens, those 32 apart are together, so that a lane of the
// matrix cores' operand has its four tokens' in a word.
__device__ __forceinline__ long long exponent_place(long long t) { return (t & ~127ll) + (t & 31) * 4 + (t >> 5 & 3); }

// Rows of activations into 8 bits (EXACT: into the values those stand for, in bf16), sixteen lanes a block of channels.
template <typename X, RowForm FORM, bool EXACT, int ITEMS>
__global__ void __launch_bounds__(kThreadsRow)
rows8_kernel(const X* __restrict__ x, long long stride, int width, unsigned char* __restrict__ to, unsigned char* __restrict__ e, long long tokens,
             RowWork work) {
    static_assert(EXACT || FORM != kShort, "a depth below 8 is EXACT");
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
                        *reinterpret_cast<u32x4*>(to + panel_place(work.rows, p.row, 2 * p.at)) = in_bf16(q, exponent);
                    } else {
                        *reinterpret_cast<u32x2*>(to + panel_place(work.rows, p.row, p.at)) = q;
                        if ((g & 15) == 0) e[p.at / kBlock8 * tokens + exponent_place(p.row)] = static_cast<unsigned char>(exponent);
                    }
                }
            }
        }
    });
}
// A weight's rows in 8 bits into the values they stand for.
__global__ void __launch_bounds__(kThreadsRow)
weight_values_kernel(const unsigned char* __restrict__ q, const unsigned char* __restrict__ e, long long e_output, long long e_depth,
                     unsigned char* __restrict__ to, RowWork work) {
    every_rows(work, [&](long long first, unsigned n) {
        for (unsigned g = threadIdx.x; g < n; g += kThreadsRow) {
            const Place p = place_of(work, first, g);
            *reinterpret_cast<u32x4*>(to + panel_place(work.rows, p.row, 2 * p.at)) =
                in_bf16(*reinterpret_cast<const u32x2*>(q + panel_place(work.rows, p.row, p.at)),
                        e[p.row / kBlock8 * e_output + p.at / kBlock8 * e_depth]);
        }
    });
}

// A workgroup puts a block of 128 outputs x 128 inputs into 8 bits, as it is and transposed (through LDS).
template <typename T, RowForm FORM>
__global__ void __launch_bounds__(1024) weight8_store_kernel(const T* __restrict__ from, Weight8 w, int blocks_i, long long blocks) {
    __shared__ unsigned most_of[16];
    __shared__ __align__(16) unsigned char turned[kBlock8][kBlock8 + 4];   // [input][output]
    const int r = threadIdx.x / 16, c = threadIdx.x % 16 * 8;
    for (long long block = blockIdx.x; block < blocks; block += gridDim.x) {
        const long long o0 = block / blocks_i * kBlock8, i0 = block % blocks_i * kBlock8;
        // (without branches: both are loaded before either is waited for)
        Granule<T, 8> raw[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
            load_row<FORM>(raw[k], from + min(o0 + 64 * k + r, static_cast<long long>(w.outputs) - 1) * w.width, static_cast<int>(i0) + c, static_cast<int>(w.width));
        float v[2][8];
        unsigned most = 0;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            unpack(raw[k], v[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (o0 + 64 * k + r >= w.outputs || i0 + c + (FORM == kWhole ? 0 : i) >= w.width) v[k][i] = 0.f;
                most = max(most, finite_size(v[k][i]));
            }
        }
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) most = max(most, static_cast<unsigned>(__shfl_xor(static_cast<int>(most), m, 64)));
        __syncthreads();   // (the last block's have been read)
        if ((threadIdx.x & 63) == 0) most_of[threadIdx.x / 64] = most;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k) most = max(most, most_of[k]);
        const unsigned exponent = exponent_of(most);
        if (threadIdx.x == 0) w.e[block] = static_cast<unsigned char>(exponent);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            u32x2 q;
            q.x = in_8_bits(v[k], exponent);
            q.y = in_8_bits(v[k] + 4, exponent);
            const long long o = o0 + 64 * k + r;
            if (o < w.outputs) *reinterpret_cast<u32x2*>(w.q + panel_place(w.outputs, o, static_cast<int>(i0) + c)) = q;
#pragma unroll
            for (int i = 0; i < 8; ++i) turned[c + i][64 * k + r] = static_cast<unsigned char>((i < 4 ? q.x : q.y) >> (8 * (i % 4)));
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int in = 64 * k + r;
            if (i0 + in < w.width) {
                u32x2 q;
                q.x = *reinterpret_cast<const unsigned*>(&turned[in][c]);
                q.y = *reinterpret_cast<const unsigned*>(&turned[in][c + 4]);
                *reinterpret_cast<u32x2*>(w.turned + panel_place(w.width, i0 + in, static_cast<int>(o0) + c)) = q;
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

// 16 OUTPUTS outputs x 16 tokens of a workgroup.  Its waves share the depth, block by block: a wave reads 128 channels of the weight's rows as
// they are, puts those of the tokens into 8 bits where the matrix cores want them, and multiplies.
template <typename X, typename O, RowForm FORM, int WAVES, int OUTPUTS>
__global__ void __launch_bounds__(64 * WAVES) few_tokens_kernel(Product8 p, long long tiles_o, long long tiles) {
    static_assert(WAVES == 4 || FORM != kShort, "a depth below 8 is one block, which needs no sixteen waves");
    constexpr int kOutputs = 16 * OUTPUTS;
    __shared__ float meet[WAVES][16][kOutputs + 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, group = lane >> 4;
    const int blocks = static_cast<int>((p.depth + kBlock8 - 1) / kBlock8), depth = static_cast<int>(p.depth);
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const long long o0 = tile % tiles_o * kOutputs, t0 = tile / tiles_o * 16;
        const unsigned char* w[OUTPUTS];
#pragma unroll
        for (int i = 0; i < OUTPUTS; ++i)
            w[i] = p.w + ((group >> 1) * static_cast<long long>(p.outputs) + min(o0 + 16 * i + row, static_cast<long long>(p.outputs) - 1)) * kPanel +
                   32 * (group & 1);
        const X* const x = static_cast<const X*>(p.x) + min(t0 + row, static_cast<long long>(p.rows) - 1) * p.x_stride;
        const unsigned char* const e = p.e + o0 / kBlock8 * p.e_output;
        f32x4 acc[OUTPUTS] = {};
        // (a block's loads are issued before the products of the one before it)
        u32x4 lo[OUTPUTS], hi[OUTPUTS];
        Granule<X, 8> raw[4];
        unsigned weight_exponent = 0;
        auto load = [&](int b) {
#pragma unroll
            for (int i = 0; i < OUTPUTS; ++i) {
                const unsigned char* const here = w[i] + b * static_cast<long long>(p.outputs) * kBlock8;
                lo[i] = *reinterpret_cast<const u32x4*>(here);
                hi[i] = *reinterpret_cast<const u32x4*>(here + 16);
            }
            weight_exponent = e[b * p.e_depth];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int at = b * kBlock8 + 32 * group + 8 * k;
                if constexpr (FORM == kRagged) load_any(raw[k], x + min(at, depth - 8));
                else load_row<FORM>(raw[k], x, at, depth);
            }
        };
        if (wave < blocks) load(wave);
        for (int b = wave; b < blocks; b += WAVES) {
            i32x8 a[OUTPUTS], q;
#pragma unroll
            for (int n = 0; n < OUTPUTS; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    a[n][i] = static_cast<int>(lo[n][i]);
                    a[n][4 + i] = static_cast<int>(hi[n][i]);
                }
            const unsigned of_weight = weight_exponent;
            float v[4][8];
            unsigned most = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int at = b * kBlock8 + 32 * group + 8 * k;
                if constexpr (FORM == kRagged) {
                    // (the row's last eight channels, moved down)
                    if (b == blocks - 1) move_down(raw[k], at - min(at, depth - 8));
                }
                unpack(raw[k], v[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (at + (FORM == kWhole ? 0 : i) >= depth) v[k][i] = 0.f;
                    most = max(most, finite_size(v[k][i]));
                }
            }
            if (b + WAVES < blocks) load(b + WAVES);
            most = max(most, static_cast<unsigned>(__shfl_xor(static_cast<int>(most), 16, 64)));
            most = max(most, static_cast<unsigned>(__shfl_xor(static_cast<int>(most), 32, 64)));
            const unsigned exponent = exponent_of(most);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                q[2 * k] = static_cast<int>(in_8_bits(v[k], exponent));
                q[2 * k + 1] = static_cast<int>(in_8_bits(v[k] + 4, exponent));
            }
            if constexpr (sizeof(O) == 4) {
                // (the same eight channels of both, whichever they are)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const u32x2 m = {static_cast<unsigned>(q[2 * k]), static_cast<unsigned>(q[2 * k + 1])};
                    const bf16x8 token = __builtin_bit_cast(bf16x8, in_bf16(m, exponent));
#pragma unroll
                    for (int n = 0; n < OUTPUTS; ++n) {
                        const u32x2 l = {static_cast<unsigned>(a[n][2 * k]), static_cast<unsigned>(a[n][2 * k + 1])};
                        acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, in_bf16(l, of_weight)), token, acc[n], 0, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int n = 0; n < OUTPUTS; ++n)
                    acc[n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a[n], q, acc[n], 0, 0, 0, static_cast<int>(of_weight), 0,
                                                                              static_cast<int>(exponent));
            }
        }
        __syncthreads();   // (the last tile's sums have been read)
#pragma unroll
        for (int n = 0; n < OUTPUTS; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) meet[wave][row][16 * n + 4 * group + i] = acc[n][i];
        __syncthreads();
        for (int at = threadIdx.x; at < 16 * kOutputs; at += 64 * WAVES) {
            const int t = at / kOutputs, o = at % kOutputs;
            if (t0 + t >= p.rows || o0 + o >= p.outputs) continue;
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < WAVES; k += 4) sum += (meet[k][t][o] + meet[k + 1][t][o]) + (meet[k + 2][t][o] + meet[k + 3][t][o]);
            if (p.bias != nullptr) {
                if (p.bias_dtype == ADASUM_F32) sum += load_elem(static_cast<const float*>(p.bias) + o0 + o);
                else if (p.bias_dtype == ADASUM_BF16) sum += load_elem(static_cast<const bf16_t*>(p.bias) + o0 + o);
                else sum += load_elem(static_cast<const f16_t*>(p.bias) + o0 + o);
            }
            store_elem(static_cast<O*>(p.out) + (t0 + t) * p.out_stride + o0 + o, sum);
        }
    }
}

// TILE x TILE of the result: what a workgroup of four waves computes at a time.  A step is a panel of both operands, 64 bytes of the depth (64
// numbers of 8 bits, 32 of 16).  Panels go to LDS past the registers, into one of four places in turn.  A row's four pieces of 16 bytes lie
// there at their number exclusive-or a quarter of the row's, so that sixteen rows' same piece lies in all banks.
template <bool EXACT, int TILE, typename O>
struct ProductShape {
    static constexpr int threads = 256, frags = TILE / 64;                 // of 32 rows, a wave along each side
    static constexpr int panel_bytes = TILE * kPanel, step_bytes = 2 * panel_bytes, places = 4;
    static constexpr int loads = panel_bytes / (threads * 16);             // of an operand, a wave
    // what a wave loads of PANELS panels in a row behind one that begins a block: both operands', and the exponents with every second
    static constexpr int loads_of(int panels) { return 2 * loads * panels + (EXACT ? 0 : panels / 2); }
    static constexpr int exponents = EXACT ? 0 : 256;                      // bytes of a block's exponents, a wave
    // results pass through LDS, 32 tokens of a wave at a time, as many of its outputs as there is room for, in whole fragments
    static constexpr int frag_bytes = 32 * static_cast<int>(sizeof(O));
    static constexpr int row_bytes = (TILE == 256 || EXACT) && frags * frag_bytes >= 128 ? 128 : 64, result_bytes = 32 * row_bytes;
    static constexpr int frags_at_once = row_bytes / frag_bytes;
    static_assert(frags_at_once >= 1 && frags % frags_at_once == 0, "a wave has no other fragments than its own");
    static constexpr int off_exponents = places * step_bytes, off_results = off_exponents + 4 * places * exponents;
    static constexpr int lds_bytes = off_results + 4 * result_bytes;
};

constexpr unsigned kStrip = 4;
struct Large {
    const unsigned char *w, *x;           // panels
    const unsigned char *e_w, *e_x;       // exponents (not EXACT): [output / 128 * e_output + block * e_depth], [block * tokens + place]
    long long outputs, rows, e_output, e_depth, tokens;
    const void* bias;
    int bias_dtype, steps;                // steps of a tile: an even number
    long long out_stride;
    unsigned tiles_o, tiles;
};

// (Scalars that the vector unit writes may be read as addresses five instructions later, m0 one later: nobody but this file sees to that in
// the assembly below.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // (that nobody keeps m0 for later across these: nobody is to)
// Sixteen (or four) bytes a lane from base + offset to LDS, a wave's one after the other from `to` on.  (The builtin makes every later read of
// LDS wait for it, of whatever place.  There is no register that the load writes; the loop below waits for it by itself.)
__device__ __forceinline__ void load_to_lds(const unsigned char* base, unsigned offset, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "m0", "memory");
}
__device__ __forceinline__ void load_word_to_lds(const unsigned char* at, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(at) : "m0", "memory");
}
#pragma clang diagnostic pop
// An address that all lanes have, in scalar registers.
__device__ __forceinline__ const unsigned char* in_scalars(const unsigned char* p) {
    const unsigned long long a = reinterpret_cast<unsigned long long>(p);
    const unsigned lo = __builtin_amdgcn_readfirstlane(static_cast<unsigned>(a)), hi = __builtin_amdgcn_readfirstlane(static_cast<unsigned>(a >> 32));
    return reinterpret_cast<const unsigned char*>(static_cast<unsigned long long>(hi) << 32 | lo);
}
// Until at most LOADS of the wave's accesses to memory are under way, and none to LDS.
template <int LOADS>
__device__ __forceinline__ void wait_for_loads() {
    static_assert(LOADS <= 63, "");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (LOADS & 15) | (LOADS >> 4) << 14);
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

#define ADASUM_INLINE __attribute__((always_inline))
// What bounds it: a step's loads (64 KB of a block of 128 in 0.9 us; a step ahead, as far as a third place would let them be, they were late: 4096
// -> 1024, 16384 rows 66 us for 60) and the matrix cores, 1.0 us at the clock that the card has then.  A tile of 1024's depth spends as long
// again on its start and its results.  Loads run three steps ahead of the products.  A step's operands are in registers when it begins; beside its products the next step's are
// read, into the registers of those that have been used for the last time.
template <bool EXACT, int TILE, typename O>
__global__ void __launch_bounds__(256, TILE == 256 ? 1 : 2) product_kernel(Large p, O* __restrict__ out) {
    typedef ProductShape<EXACT, TILE, O> S;
    constexpr int F = S::frags, L = S::loads;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wo = wave % 2 * (32 * F), wt = wave / 2 * (32 * F);
    const unsigned lds_base = static_cast<unsigned>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)(lds)));

    // Tiles go by four along the outputs, then along the tokens: what one die has at a time is near a square, and shares operands both ways.
    const unsigned n = die_order(blockIdx.x, gridDim.x), tiles_t = gridDim.x / p.tiles_o;
    const unsigned strip = n / (kStrip * tiles_t), across = min(p.tiles_o - strip * kStrip, kStrip), at = n - strip * kStrip * tiles_t;
    const long long o0 = static_cast<long long>(strip * kStrip + at % across) * TILE, t0 = static_cast<long long>(at / across) * TILE;

    // ---- loads: a lane's piece of each 64th row
    int load_place = 0;
    const unsigned char *w_base = in_scalars(p.w + o0 * kPanel), *x_base = in_scalars(p.x + t0 * kPanel);
    const int w_last = static_cast<int>(min(p.outputs - o0, static_cast<long long>(TILE))) - 1;
    const int x_last = static_cast<int>(min(p.rows - t0, static_cast<long long>(TILE))) - 1;
    unsigned w_at[L], x_at[L];
#pragma unroll
    for (int k = 0; k < L; ++k) {
        const int row = (k * 4 + wave) * 16 + (lane >> 2), piece = (lane & 3) ^ (lane >> 4);
        w_at[k] = min(row, w_last) * kPanel + 16 * piece;
        x_at[k] = min(row, x_last) * kPanel + 16 * piece;
    }
    // (of the exponents, the first half of the lanes load the tokens', the others the word that has the weight's)
    const unsigned char* const of_x0 = EXACT ? nullptr : p.e_x + ((t0 + wt) & ~127ll) + 4 * (lane & 31);
    const unsigned char* const of_w0 = EXACT ? nullptr : p.e_w + min(o0 + wo, p.outputs - 1) / kBlock8 * p.e_output;
    const unsigned char* e_at = lane < 32 ? of_x0 : of_w0;
    const long long of_tokens = p.tokens, of_weight = p.e_depth, e_next = lane < 32 ? of_tokens : of_weight;
    // a panel, the first of a block of the depth or its second
    auto load = [&](auto odd) ADASUM_INLINE {
        if constexpr (!EXACT && !decltype(odd)::value) {
            load_word_to_lds(reinterpret_cast<const unsigned char*>(reinterpret_cast<uintptr_t>(e_at) & ~static_cast<uintptr_t>(3)),
                             lds_base + S::off_exponents + (wave * S::places + (load_place >> 1 & (S::places - 1))) * S::exponents);
            e_at += e_next;
        }
        const unsigned to = lds_base + (load_place & (S::places - 1)) * S::step_bytes + wave * 1024;
        asm volatile("s_nop 4" : "+s"(w_base), "+s"(x_base));   // (whoever wrote them last)
#pragma unroll
        for (int k = 0; k < L; ++k) {
            load_to_lds(w_base, w_at[k], to + k * 4096);
            load_to_lds(x_base, x_at[k], to + S::panel_bytes + k * 4096);
        }
        ++load_place;
        w_base += p.outputs * kPanel;
        x_base += p.rows * kPanel;
    };

    // ---- products
    const int row = lane & 31, group = lane >> 5, turn = row >> 2 & 3;
    const char* const w_read = lds + (wo + row) * kPanel;
    const char* const x_read = lds + S::panel_bytes + (wt + row) * kPanel;
    const int piece[2] = {16 * (group ^ turn), 16 * ((group + 2) ^ turn)};
    u32x4 fw[F][2], fx[F][2];
    auto read_w = [&](int i, int from) ADASUM_INLINE {
#pragma unroll
        for (int h = 0; h < 2; ++h) fw[i][h] = *reinterpret_cast<const u32x4*>(w_read + from + i * 32 * kPanel + piece[h]);
    };
    auto read_x = [&](int j, int from) ADASUM_INLINE {
#pragma unroll
        for (int h = 0; h < 2; ++h) fx[j][h] = *reinterpret_cast<const u32x4*>(x_read + from + j * 32 * kPanel + piece[h]);
    };
    // the exponents of this block of the depth, and of the next
    unsigned of_w = 0, of_x = 0, next_w = 0, next_x = 0;
    auto whole = [](const u32x4 (&f)[2]) ADASUM_INLINE {
        i32x8 r;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            r[k] = static_cast<int>(f[0][k]);
            r[4 + k] = static_cast<int>(f[1][k]);
        }
        return r;
    };
    f32x16 acc[F][F] = {};
    auto multiply = [&](int i, auto number) ADASUM_INLINE {
        constexpr int j = decltype(number)::value;
        f32x16 sum = acc[i][j];
        if constexpr (EXACT) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fw[i][h]), __builtin_bit_cast(bf16x8, fx[j][h]), sum, 0, 0, 0);
        } else {
            sum = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(whole(fw[i]), whole(fx[j]), sum, 0, 0, 0, static_cast<int>(of_w), j,
                                                                  static_cast<int>(of_x));
        }
        acc[i][j] = sum;
    };
    int place = 0;                        // of the panels that are multiplied; a tile begins with an even one
    // where the weight's exponent lies in its word
    unsigned e_shift = static_cast<unsigned>(reinterpret_cast<uintptr_t>(of_w0) & 3) * 8;
    const unsigned e_shift_next = static_cast<unsigned>(p.e_depth & 3) * 8;
    auto read_exponents = [&](int block) ADASUM_INLINE {
        if constexpr (!EXACT) {
            const char* const at = lds + S::off_exponents + (wave * S::places + (block & (S::places - 1))) * S::exponents;
            // (of a wave with fewer than the 128 tokens, its bytes)
            next_x = *reinterpret_cast<const unsigned*>(at + 4 * row) >> (8 * (static_cast<int>(t0 + wt) & 127) / 32);
            next_w = *reinterpret_cast<const unsigned*>(at + 128) >> e_shift;
            e_shift = (e_shift + e_shift_next) & 31;
        }
    };
    // One step.  What is waited for is the next step's panel; all others that there are places for came after it and may be under way.
    auto step = [&](auto odd, auto more) ADASUM_INLINE {
        every<F>([&](auto j) { multiply(0, j); });
        __builtin_amdgcn_sched_barrier(0);
        wait_for_loads<decltype(more)::value ? S::loads_of(S::places - 2) : 0>();
        __builtin_amdgcn_s_barrier();
        if constexpr (decltype(more)::value) load(odd);
        ++place;
        const int from = (place & (S::places - 1)) * S::step_bytes;
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (decltype(odd)::value) read_exponents(place >> 1);
#pragma unroll
        for (int i = 1; i < F - 2; ++i) {
            read_w(i - 1, from);
            every<F>([&](auto j) { multiply(i, j); });
            __builtin_amdgcn_sched_barrier(0);
        }
        constexpr int kLeft = F > 2 ? F - 2 : 1;   // the rows that are left, column by column
        read_w(kLeft - 1, from);
        every<F>([&](auto j) {
#pragma unroll
            for (int i = kLeft; i < F; ++i) multiply(i, j);
            __builtin_amdgcn_sched_barrier(0);
            read_x(j, from);
        });
#pragma unroll
        for (int i = kLeft; i < F; ++i) read_w(i, from);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (decltype(odd)::value) {
            of_w = next_w;
            of_x = next_x;
        }
    };

    // ---- results: a lane has four times four consecutive outputs of a token in each 32 x 32; through LDS consecutive lanes get a token's
    // consecutive outputs to store
    char* const mine = lds + S::off_results + wave * S::result_bytes;
    constexpr int kPieces = S::row_bytes / 16, kFrags = S::frags_at_once;   // of 32 outputs, at a time
    auto piece_at = [&](int token, int n) {
        return mine + token * S::row_bytes + 16 * (n ^ (kPieces == 8 ? token >> 1 & 7 : token >> 2 & 3));
    };
    auto store = [&](bool all) ADASUM_INLINE {
#pragma unroll
        for (int i0 = 0; i0 < F; i0 += kFrags) {
            float bias[kFrags][4][4] = {};
            if (p.bias != nullptr) {
#pragma unroll
                for (int i = 0; i < kFrags; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const long long o = o0 + wo + 32 * (i0 + i) + 8 * q + 4 * group;
                        const int there = static_cast<int>(min(p.outputs - o, 4ll));
                        if (there <= 0) continue;
                        if (p.bias_dtype == ADASUM_F32) load_some<4>(bias[i][q], static_cast<const float*>(p.bias) + o, there);
                        else if (p.bias_dtype == ADASUM_BF16) load_some<4>(bias[i][q], static_cast<const bf16_t*>(p.bias) + o, there);
                        else load_some<4>(bias[i][q], static_cast<const f16_t*>(p.bias) + o, there);
                    }
            }
#pragma unroll
            for (int j = 0; j < F; ++j) {
#pragma unroll
                for (int i = 0; i < kFrags; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float v[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] = acc[i0 + i][j][4 * q + k] + bias[i][q][k];
                        if constexpr (sizeof(O) == 4) store_any<4>(reinterpret_cast<O*>(piece_at(row, 2 * q + group)), v);
                        else store_any<4>(reinterpret_cast<O*>(piece_at(row, 4 * i + q) + 8 * group), v);
                    }
                asm volatile("" ::: "memory");   // (a wave's own accesses to LDS keep their order)
                constexpr int kOfLane = 16 / static_cast<int>(sizeof(O));
#pragma unroll
                for (int k = 0; k < kPieces / 2; ++k) {
                    const int token = k * (64 / kPieces) + lane / kPieces, n = lane % kPieces;
                    const u32x4 v = *reinterpret_cast<const u32x4*>(piece_at(token, n));
                    const long long t = t0 + wt + 32 * j + token, o = o0 + wo + 32 * i0 + n * kOfLane;
                    O* const to = out + t * p.out_stride + o;
                    // (past the caches: 32768 x 1024 -> 4096 in bf16 206 -> 202 us, in fp32 346 -> 318)
                    if (all) {
                        store_at<true>(v, reinterpret_cast<u32x4_any*>(to));
                    } else if (t < p.rows && o < p.outputs) {
                        if (p.outputs - o >= kOfLane) {
                            store_at<false>(v, reinterpret_cast<u32x4_any*>(to));
                        } else {
                            const unsigned words[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int e = 0; e < kOfLane; ++e)
                                if (o + e < p.outputs) {
                                    if constexpr (sizeof(O) == 4) to[e] = __uint_as_float(words[e]);
                                    else to[e].v = static_cast<unsigned short>(words[e / 2] >> (16 * (e & 1)));
                                }
                        }
                    }
                }
                asm volatile("" ::: "memory");
            }
        }
    };

    const std::true_type yes;
    const std::false_type no;
    // (there are at least as many steps as places)
#pragma unroll
    for (int k = 0; k < S::places; k += 2) {
        load(no);
        load(yes);
    }
    wait_for_loads<S::loads_of(S::places - 1)>();
    __builtin_amdgcn_s_barrier();
    read_exponents(0);
    of_w = next_w;
    of_x = next_x;
#pragma unroll
    for (int i = 0; i < F; ++i) {
        read_x(i, 0);
        read_w(i, 0);
    }
    for (int s = S::places; s < p.steps; s += 2) {
        step(no, yes);
        step(yes, yes);
    }
    // (the last find all their panels loaded)
    for (int s = 0; s < S::places; s += 2) {
        step(no, no);
        step(yes, no);
    }
    if (o0 + TILE <= p.outputs && t0 + TILE <= p.rows) store(true);
    else store(false);
}

// From how many tiles of 16 x 16 on a workgroup takes two, and four, along the outputs: the tokens' operands are made once for them.  (4096 -> 1024 in
// bf16, 64 rows with one 9.5 us, with two 7.2; 256 rows 28, 19 and with four 14; 1000 -> 2048, 128 rows 9.6 and 9.6.)
constexpr int64_t kSomeTiles = 512, kManyTiles = 1024;
// 16-bit results of one block of depth: the other kernel's workgroups are on the chip at once up to 4096 tiles of 16 x 16 (16 x 64 for each of four a
// compute unit).  128 -> 1024 in bf16, 1024 rows (4096 tiles) 7.3 and 7.4 with tiles, 1088 rows 9.4 and 7.6, 2048 rows 12.9 and 8.2; 128 -> 128, 8192
// rows 7.2 and 8.0, 9216 rows 9.5 and 8.6; but 128 -> 32, 36864 rows (4608 tiles) 15.0 and 15.6.  (Three launches, of operands as bf16 numbers.)
constexpr double kShallowTiles = 4096;
// Whether the products go by tiles of 64 to 256, by what a call takes (microseconds) beside 3.5 either way: the kernel of few tokens 0.3 for each
// thousand blocks of 16 x 16 x 128, the other, with the launch before it, 1.5 and 0.33 for each block of the depth; for fp32 results 0.48, and
// 3 and 0.75.  (Fitted; both ways:)  1024 -> 4096 in bf16, 64 rows 6.0 and 7.0, 128 rows 8.1 and 7.2; 2048 -> 1000, 256 rows 10 and 10, 512 rows
// 12.2 and 10.8; 8192 -> 8192, 32 rows 21 and 26, 64 rows 35 and 26; 256 -> 256, 2048 rows 5.1 and 5.3, 4096 rows 8.4 and 5.8; fp32 1024 -> 4096, 128
// rows 12 and 15, 256 rows 20 and 16; 2048 -> 1000, 512 rows 20 and 20.  It does not count the values of a large weight, which fp32 results
// take a launch more for: 8192 -> 8192 in fp32, 64 rows 54 and 83, by tiles all the same.
bool is_large(int64_t rows, int64_t outputs, int64_t depth, int out_dtype) {
    const double blocks = static_cast<double>(blocks8(depth)), tiles = static_cast<double>((rows + 15) / 16) * static_cast<double>((outputs + 15) / 16);
    if (out_dtype != ADASUM_F32 && blocks == 1) return tiles > kShallowTiles;
    return depth > 0 && (out_dtype == ADASUM_F32 ? 0.00048 * tiles * blocks > 3 + 0.75 * blocks : 0.0003 * tiles * blocks > 1.5 + 0.33 * blocks);
}
// Whether operands are multiplied as the bf16 numbers that they stand for: for fp32 results, and where a tile would have two steps only (the
// kernel's loads are three ahead).
bool is_exact(int64_t depth, int out_dtype) { return out_dtype == ADASUM_F32 || depth <= kBlock8; }
constexpr int64_t kTokenPad = 256;
struct Workspace8 {
    size_t off_more = 0, total = 0;    // the exponents, or the weight's values
};
Workspace8 workspace8(int64_t rows, int64_t outputs, int64_t depth, int out_dtype) {
    Workspace8 w;
    if (!is_large(rows, outputs, depth, out_dtype)) return w;
    const size_t pitch = static_cast<size_t>(blocks8(depth)) * kBlock8;
    const bool exact = is_exact(depth, out_dtype);
    w.off_more = static_cast<size_t>(rows) * pitch * (exact ? 2 : 1);
    w.total = w.off_more + (exact ? static_cast<size_t>(outputs) * pitch * 2
                                  : static_cast<size_t>(blocks8(depth)) * align_up(static_cast<size_t>(rows), kTokenPad));
    return w;
}

template <bool EXACT, int TILE, typename O>
int launch_large(const Product8& p, const Large& l, void* stream) {
    typedef ProductShape<EXACT, TILE, O> S;
    static_assert(S::lds_bytes * (TILE == 256 ? 1 : 2) <= 160 << 10, "what a compute unit has");
    const auto kernel = product_kernel<EXACT, TILE, O>;
    const int rc = static_cast<int>(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::lds_bytes));
    if (rc != 0) return rc;
    return launch(kernel, l.tiles, 1, S::threads, S::lds_bytes, stream, l, static_cast<O*>(p.out));
}

// (granules from which a lane has four in flight, past the caches: with the product behind it, 4194 thousand in bf16 29 us with one and 33 with
// four, 16777 127 and 116)
constexpr int64_t kMany8 = 1 << 23;

// Tiles of edge 128 up to which those of 64 are faster: a compute unit's own loads bound these calls (some 60 GB/s), and more of them share a
// product.  8192 -> 8192 in bf16, 256 rows (128 tiles) 39 us with 128 and 35 with 64, 512 rows (256 tiles) 44 and 64; 4096 -> 1024, 128 rows 19.7 and
// 14.8, 2048 rows (128 tiles) 27.6 and 26.1.
constexpr int64_t kFewSmall = 128;
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
            // (a depth below 8 is EXACT)
            constexpr RowForm F = !EXACT && decltype(form)::value == kShort ? kRagged : decltype(form)::value;
            return with_items<X>(g, [&](auto items) -> int {
                return launch(rows8_kernel<X, F, EXACT, decltype(items)::value>, g.groups, 1, kThreadsRow, 0, stream, static_cast<const X*>(p.x),
                              p.x_stride, p.depth, x, EXACT ? nullptr : more, tokens, g.work);
            });
        });
    });
    if (rc != 0) return rc;
    if (EXACT) {
        const RowGrid g = row_grid(p.outputs, pitch, ADASUM_F32, 0);
        rc = launch(weight_values_kernel, g.groups, 1, kThreadsRow, 0, stream, p.w, p.e, p.e_output, p.e_depth, more, g.work);
        if (rc != 0) return rc;
    }
    Large l{};
    l.w = EXACT ? more : p.w;
    l.x = x;
    l.e_w = p.e;
    l.e_x = EXACT ? nullptr : more;
    l.outputs = p.outputs;
    l.rows = p.rows;
    l.e_output = p.e_output;
    l.e_depth = p.e_depth;
    l.tokens = tokens;
    l.bias = p.bias;
    l.bias_dtype = p.bias_dtype;
    l.steps = static_cast<int>(pitch * (EXACT ? 2 : 1) / kPanel);
    l.out_stride = p.out_stride;
    auto tiles = [&](int64_t n, int tile) { return (n + tile - 1) / tile; };
    // A round of 256 tiles of edge 256 takes as long as 1.75 rounds of 512 of edge 128, of which it has two's work.  (8192 -> 8192 in bf16, 1024 rows:
    // 80 us with 128 and 100 with 256, 2048: 148 and 137; 4096 -> 1024, 8192 rows 61 and 77, 16384: 116 and 108.)
    const int64_t wide_tiles = tiles(p.outputs, 256) * tiles(p.rows, 256), small_tiles = tiles(p.outputs, 128) * tiles(p.rows, 128);
    const bool wide = 7 * tiles(wide_tiles, 256) < 4 * tiles(small_tiles, 512);
    const int tile = wide ? 256 : small_tiles > kFewSmall ? 128 : 64;
    l.tiles_o = static_cast<unsigned>(tiles(p.outputs, tile));
    l.tiles = static_cast<unsigned>(l.tiles_o * tiles(p.rows, tile));
    return tile == 256 ? launch_large<EXACT, 256, O>(p, l, stream)
                       : tile == 128 ? launch_large<EXACT, 128, O>(p, l, stream) : launch_large<EXACT, 64, O>(p, l, stream);
}

}  // namespace

int launch_weight8_store(const void* w, int dtype, const Weight8& to, void* stream) {
    const int64_t blocks_i = blocks8(to.width), blocks = blocks8(to.outputs) * blocks_i;
    return with_type(dtype, [&](auto t) -> int {
        typedef decltype(t) T;
        return with_form(row_form(to.width, 8), [&](auto form) -> int {
            return launch(weight8_store_kernel<T, decltype(form)::value>, at_most_groups(blocks), 1, 1024, 0, stream, static_cast<const T*>(w), to,
                          blocks_i, blocks);
        });
    });
}

size_t product8_workspace(int64_t rows, int64_t outputs, int64_t depth, int out_dtype) { return workspace8(rows, outputs, depth, out_dtype).total; }

int launch_product8(const Product8& p, void* stream) {
    if (is_large(p.rows, p.outputs, p.depth, p.out_dtype)) {
        const bool exact = is_exact(p.depth, p.out_dtype);
        switch (p.out_dtype) {
            case ADASUM_F32: return large_product<true, float>(p, stream);
            case ADASUM_BF16: return exact ? large_product<true, bf16_t>(p, stream) : large_product<false, bf16_t>(p, stream);
            default: return exact ? large_product<true, f16_t>(p, stream) : large_product<false, f16_t>(p, stream);
        }
    }
    return with_type(p.dtype, [&](auto x) -> int {
        typedef decltype(x) X;
        return with_type(p.out_dtype, [&](auto out) -> int {
            typedef decltype(out) O;
            return with_form(row_form(p.depth, 8), [&](auto form) -> int {
                constexpr RowForm F = decltype(form)::value;
                const int64_t tiles_t = (p.rows + 15) / 16, tiles = (p.outputs + 15) / 16 * tiles_t, blocks = blocks8(p.depth);
                auto go = [&](auto waves, auto outputs) -> int {
                    constexpr int W = decltype(waves)::value, N = decltype(outputs)::value;
                    const int64_t tiles_o = (p.outputs + 16 * N - 1) / (16 * N);
                    return launch(few_tokens_kernel<X, O, F, W, N>, at_most_groups(tiles_o * tiles_t), 1, 64 * W, 0, stream, p, tiles_o,
                                  tiles_o * tiles_t);
                };
                const std::integral_constant<int, 1> one;
                const std::integral_constant<int, 2> two;
                const std::integral_constant<int, 4> four;
                const std::integral_constant<int, 16> sixteen;
                // (sixteen waves share a depth that four would go through in turn: 4096 -> 1024 in bf16, one row 10.0 and 7.9 us; fp32, whose
                // operands take longer to make, 12.1 and 10.5, but 2048 -> 1000, 16 rows 8.4 and 9.6)
                if constexpr (F != kShort) {
                    if (p.out_dtype == ADASUM_F32 ? tiles <= 64 && blocks > 16 : tiles <= 256 && blocks > 8) return go(sixteen, one);
                }
                return tiles >= kManyTiles ? go(four, four) : tiles >= kSomeTiles ? go(four, two) : go(four, one);
            });
        });
    });
}

}  // namespace adasum
