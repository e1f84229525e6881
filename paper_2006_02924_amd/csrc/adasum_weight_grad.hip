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

// What the matrix cores multiply: the 16-bit types as they are; fp32 as three bf16 parts, each what the parts before it leave, rounded to
// nearest.  The three add up to the value (9 + 9 + 6 bits; of values below 2^-110 what lies below 2^-133 is lost).  Rounded rather than
// cut off, so that the smaller parts of values of one sign have either sign: a sum of some thousand tokens is too large for a run of
// third parts to change it, and what is lost must not add up (8192 positive tokens came out 46 steps of fp32 too small on average
// with parts cut off, 0.7 with parts rounded).
template <typename T> struct Products { typedef T type; static constexpr int planes = 1; };
template <> struct Products<float> { typedef bf16_t type; static constexpr int planes = 3; };

// The parts of two values.  (Near the end of the range the first two are limited, so that no part and no sum of them is an infinity that the
// value is not.  Infinities and NaN leave the limits as they are and are in the third part.)
__device__ __forceinline__ void parts_of(unsigned (&p)[3], unsigned a, unsigned b) {
    constexpr float kMost = 0x1.fep127f, kRest = 0x1.fep119f;   // bf16's largest number, and its largest below what fp32 has beyond that
    const float x = __uint_as_float(a), y = __uint_as_float(b);
    p[0] = rounded_pair(bf16_t{}, __builtin_amdgcn_fmed3f(x, -kMost, kMost), __builtin_amdgcn_fmed3f(y, -kMost, kMost));
    const float rx = x - __uint_as_float(p[0] << 16), ry = y - __uint_as_float(p[0] & 0xffff0000u);
    p[1] = rounded_pair(bf16_t{}, __builtin_amdgcn_fmed3f(rx, -kRest, kRest), __builtin_amdgcn_fmed3f(ry, -kRest, kRest));
    p[2] = rounded_pair(bf16_t{}, rx - __uint_as_float(p[1] << 16), ry - __uint_as_float(p[1] & 0xffff0000u));
}

// Two values that their type holds exactly.
__device__ __forceinline__ unsigned exact_pair(bf16_t, float a, float b) {
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ unsigned exact_pair(f16_t, float a, float b) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_pkrtz(a, b));
}

// c and the sum of eight values.  The instruction multiplies with one, exactly, and adds with truncation: a step's run of them is then
// added to the rest with rounding.  (40000 positive tokens come out within 3 steps of fp32, 0.1 on average.  Additions on the vector
// unit would take four instructions for one.)
__device__ __forceinline__ float plus_eight(bf16_t, u32x4 a, float c) {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    const pair one = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned w = a[i];
        c = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair, w), one, c, false);
    }
    return c;
}
__device__ __forceinline__ float plus_eight(f16_t, u32x4 a, float c) {
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    const pair one = {static_cast<_Float16>(1.f), static_cast<_Float16>(1.f)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned w = a[i];
        c = __builtin_amdgcn_fdot2(__builtin_bit_cast(pair, w), one, c, false);
    }
    return c;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

// Workgroup `b` of n as the eight dies see it: consecutive workgroups go to dies in turn, and those of one die should share operands.
__device__ __forceinline__ unsigned die_order(unsigned b, unsigned n) {
    const unsigned die = b & 7, at = b >> 3, each = n >> 3, more = n & 7;
    return die * each + (die < more ? die : more) + at;
}

// What a workgroup does, by the edge of its square of dW (TILE) and the storage type of dy.
template <typename D, int TILE>
struct GradShape {
    // waves along the outputs and the channels, and the 32 x 32 blocks each has along them
    static constexpr int waves_o = TILE == 256 ? 4 : 2, waves_i = 2;
    static constexpr int frags_o = TILE / 32 / waves_o, frags_i = TILE / 32 / waves_i;
    static constexpr int threads = 64 * waves_o * waves_i;
    static constexpr int planes = Products<D>::planes;
    static constexpr int step = planes == 3 ? 32 : 64;          // tokens of a step
    static constexpr int subs = step / 16;                      // matrix instructions' share of it
    // LDS: [token][channel], rows TILE channels and 64 bytes apart, so that the transposing read's four rows of 32 bytes lie in
    // different banks
    static constexpr int pitch = 2 * TILE + 64;
    static constexpr int plane_bytes = step * pitch;
    static constexpr int buffer_bytes = (planes + 1) * plane_bytes;
    // a lane stages eight channels of dy, and sixteen of x, of a token at a time
    static constexpr int a_rows = threads / (TILE / 8), b_rows = threads / (TILE / 16);
    static constexpr int a_passes = step / a_rows, b_passes = step / b_rows;
    static constexpr int lds_bytes = 2 * buffer_bytes;
};

// Eight elements of dy, and sixteen of x (zeros where there is no such token), to LDS.
template <typename D>
__device__ __forceinline__ void to_lds(char* at, int plane_bytes, const Granule<D, 8>& g) {
    if constexpr (sizeof(D) == 2) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = g.w[i];
        *reinterpret_cast<u32x4*>(at) = w;
    } else {
        unsigned s[4][3];
#pragma unroll
        for (int i = 0; i < 4; ++i) parts_of(s[i], g.w[2 * i], g.w[2 * i + 1]);
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = s[i][k];
            *reinterpret_cast<u32x4*>(at + k * plane_bytes) = w;
        }
    }
}
template <typename E>
__device__ __forceinline__ void to_lds(E, char* at, u32x4 q, int e, bool there) {
    unsigned word[4] = {q.x, q.y, q.z, q.w};
    // (here and not before: the compiler would take the bytes apart where they are loaded, and wait for the load there)
    asm volatile("" : "+v"(word[0]), "+v"(word[1]), "+v"(word[2]), "+v"(word[3]), "+v"(e));
    const float step = !there ? 0.f : __uint_as_float(e == -128 ? 0x7fc00000u : static_cast<unsigned>(e + 127) << 23);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned from = word[2 * h + i / 2];
            const float a = static_cast<float>(static_cast<signed char>(i & 1 ? from >> 16 : from)) * step;
            const float b = static_cast<float>(static_cast<signed char>(i & 1 ? from >> 24 : from >> 8)) * step;
            w[i] = exact_pair(E{}, a, b);
        }
        *reinterpret_cast<u32x4*>(at + 16 * h) = w;
    }
}

// TILE x TILE of dW over one part of the tokens: eight waves of 64 x 128 or four of 64 x 64.
//
// Both operands lie with the tokens in rows, and the matrix cores want eight tokens of a channel in a lane: a step of both is staged in
// LDS as it lies in memory (x as the values it stands for), and read with the transposing LDS read.  While a step is multiplied out of
// one buffer, the next one, which is in registers by then, is written into the other and the loads of the one after are issued, a
// part of them beside every sixteen tokens' products.  One barrier a step.
//
// What bounds it: the products.  65536 x 4096 x 4096 in bf16 takes 1.80 - 2.03 ms (1.08 - 1.22 PFLOP/s; a library product of 8192^3 reaches
// 1.19 on this card, and 0.83 on the 16384 x 4096 x 1024 that this kernel does at 0.92 - 0.98 with the join), fp32, three products for one,
// 4096 x 1024 x 4096 113 - 118 us (0.9 PFLOP/s of bf16 products).  The matrix cores are busy 60 % of the cycles, of which there are 1.6e9 a
// second then: the card lowers its clock, so what is taken off the other units pays little.  Four waves of 128 x 128 read a third less LDS
// but leave the vector unit's 280 instructions a step beside 64 of the matrix core to one wave, which cannot issue both (44 % of the
// cycles).  With parts, what they store and the join reads is 16 bytes per weight for four parts: some 25 us of 16384 x 4096 x 1024's
// 141 - 168.  Products of the two 16-bit types are exact in fp32; the cores' sums were not found to drift (40000 terms of one sign).
// RAGGED: outputs that are no multiple of eight; the last ones' eight are loaded as the last eight there are, and moved down where they are
// staged (4096 x 30522 x 1024 bf16 370 -> 324 us, 8192 x 2047 x 2048 fp16 169 -> 94, against element by element without a pipeline).
template <typename D, typename T, int TILE, bool RAGGED>
__global__ void __launch_bounds__((GradShape<D, TILE>::threads), 2)
weight_grad_kernel(const signed char* __restrict__ q, const signed char* __restrict__ e, long long rows, int width, long long pitch,
                   const D* __restrict__ dy, long long dy_stride, int outputs, T* __restrict__ grad, int accumulate,
                   float* __restrict__ parts, long long steps, unsigned tiles_o, unsigned tiles_i, T* __restrict__ bias,
                   float* __restrict__ bias_parts) {
    typedef typename Products<D>::type E;
    typedef GradShape<D, TILE> S;
    constexpr int P = S::planes, FO = S::frags_o, FI = S::frags_i;
    extern __shared__ __align__(16) char lds[];
    const unsigned n = die_order(blockIdx.x, gridDim.x), tile = n % (tiles_o * tiles_i), part = n / (tiles_o * tiles_i);
    const int o0 = static_cast<int>(tile / tiles_i) * TILE, i0 = static_cast<int>(tile % tiles_i) * TILE;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wo = wave / S::waves_i * (32 * FO), wi = wave % S::waves_i * (32 * FI);
    const long long t_begin = part * steps * S::step, t_end = min(rows, t_begin + steps * S::step);
    const int whole = static_cast<int>((t_end - t_begin) / S::step);

    // what this lane stages.  Lanes behind the last channel load the first ones again: what comes of them is not stored.
    const int a_row = threadIdx.x / (TILE / 8), a_col = threadIdx.x % (TILE / 8) * 8;
    const int b_row = threadIdx.x / (TILE / 16), b_col = threadIdx.x % (TILE / 16) * 16;
    const int o = o0 + a_col, i = i0 + b_col < pitch ? i0 + b_col : 0;
    const int a_there = outputs - o;          // elements of this lane's eight that exist
    const int o_safe = a_there >= 8 ? o : RAGGED ? max(outputs - 8, 0) : 0;
    const D* a_at = dy + (t_begin + a_row) * dy_stride + o_safe;
    const signed char* b_at = q + (t_begin + b_row) * pitch + i;
    const signed char* e_at = e + (t_begin + b_row) * (pitch / kBlock) + i / kBlock;
    char* const a_lds = lds + a_row * S::pitch + a_col * 2;
    char* const b_lds = lds + P * S::plane_bytes + b_row * S::pitch + b_col * 2;
    // what it reads: of a run of 16 lanes, four lanes one token's sixteen channels
    const int r_row = 8 * (lane >> 5) + ((lane & 15) >> 2), r_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const char* const a_read = lds + r_row * S::pitch + (wo + r_col) * 2;
    const char* const b_read = lds + P * S::plane_bytes + r_row * S::pitch + (wi + r_col) * 2;

    f32x16 acc[FO][FI] = {};
    // dy's sums over this lane's tokens, of a step and of all (every workgroup and wave along the weight's rows has them, one stores them)
    float run[FO] = {}, total[FO] = {};
    Granule<D, 8> a_reg[S::a_passes];
    u32x4 b_reg[S::b_passes];
    int e_reg[S::b_passes];

    auto load_a = [&](int k) { load_any(a_reg[k], a_at + k * S::a_rows * dy_stride); };
    auto load_b = [&](int k) {
        b_reg[k] = *reinterpret_cast<const u32x4*>(b_at + k * S::b_rows * pitch);
        e_reg[k] = e_at[k * S::b_rows * (pitch / kBlock)];
    };
    auto write_a = [&](int k, int buffer, int down) {
        Granule<D, 8> g = a_reg[k];
        if constexpr (RAGGED) move_down(g, down);
        to_lds<D>(a_lds + buffer * S::buffer_bytes + k * S::a_rows * S::pitch, S::plane_bytes, g);
    };
    auto write_b = [&](int k, int buffer, bool there) {
        to_lds(E{}, b_lds + buffer * S::buffer_bytes + k * S::b_rows * S::pitch, b_reg[k], e_reg[k], there);
    };
    auto next = [&] {
        a_at += S::step * dy_stride;
        b_at += S::step * pitch;
        e_at += S::step * (pitch / kBlock);
    };
    auto fragment = [&](const char* at) -> u32x4 {
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + 4 * S::pitch));
        u32x4 f;
        const u32x2 l = __builtin_bit_cast(u32x2, lo), h = __builtin_bit_cast(u32x2, hi);
        f.x = l.x;
        f.y = l.y;
        f.z = h.x;
        f.w = h.y;
        return f;
    };
    // two sets of operands: the next sixteen tokens' are read beside this one's products.  (With fp32's three parts there is enough to
    // do beside one set's reads: 117 us for 122, 4096 x 1024 x 4096.)
    constexpr int SETS = P == 3 ? 1 : 2;
    u32x4 fa[SETS][FO], fb[SETS][FI];
    auto read = [&](int set, int sub, int buffer) {
        const int from = buffer * S::buffer_bytes + sub * 16 * S::pitch;
#pragma unroll
        for (int k = 0; k < FI; ++k) fb[set % SETS][k] = fragment(b_read + from + 64 * k);
#pragma unroll
        for (int m = 0; m < FO; ++m) fa[set % SETS][m] = fragment(a_read + from + 64 * m);
    };
    // (the first part of dy is in registers already; the others of fp32 follow)
    auto multiply = [&](int set, int sub, int buffer) {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int m = 0; m < FO; ++m) {
                const u32x4 a = p == 0 ? fa[set % SETS][m]
                                       : fragment(a_read + buffer * S::buffer_bytes + sub * 16 * S::pitch + p * S::plane_bytes + 64 * m);
#pragma unroll
                for (int k = 0; k < FI; ++k) acc[m][k] = mfma(E{}, fb[set % SETS][k], a, acc[m][k]);
                run[m] = plus_eight(E{}, a, run[m]);
            }
    };

    // (no eight to load: such layers go without the pipeline, bf16 16384 x 1024 with 1, 2, 7 and 8 outputs 17, 18, 20 and 16 us, 65536 x 256
    // 25, 27, 31 and 20.5; fp32, 27 and 37 us, does not feel it)
    const bool few = RAGGED && outputs < 8;
    auto end_run = [&] {
#pragma unroll
        for (int m = 0; m < FO; ++m) {
            total[m] += run[m];
            run[m] = 0.f;
        }
    };
    // which passes are staged beside which sixteen tokens' products: all before the last ones, which the barrier comes before
    auto staged = [&](int sub, auto&& a, auto&& b) {
#pragma unroll
        for (int k = 0; k < S::a_passes; ++k)
            if (k * (S::subs - (SETS == 2)) / S::a_passes == sub) a(k);
#pragma unroll
        for (int k = 0; k < S::b_passes; ++k)
            if (k * (S::subs - (SETS == 2)) / S::b_passes == sub) b(k);
    };
    if (whole > 0 && !few) {
#pragma unroll
        for (int sub = 0; sub < S::subs; ++sub) staged(sub, load_a, load_b);
#pragma unroll
        for (int sub = 0; sub < S::subs; ++sub)
            staged(sub, [&](int k) { write_a(k, 0, o - o_safe); }, [&](int k) { write_b(k, 0, true); });
        if (whole > 1) next();
        // (the loads are in flight in the order in which the loop issues them: what waits for one waits for no later one)
#pragma unroll
        for (int sub = 0; sub < S::subs; ++sub) {
            __builtin_amdgcn_sched_barrier(0);
            staged(sub, load_a, load_b);
        }
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();
        if constexpr (SETS == 2) read(0, 0, 0);
        for (int s = 0; s < whole; ++s) {
            const int buffer = s & 1;
            if (s + 2 < whole) next();     // (else the last whole step is loaded again, and not used)
#pragma unroll
            for (int sub = 0; sub < S::subs; ++sub) {
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (SETS == 2) {
                    // the next sixteen tokens' operands, of the next step's buffer behind the last ones
                    if (sub + 1 < S::subs) {
                        read(sub + 1, sub + 1, buffer);
                    } else {
                        __syncthreads();
                        read(0, 0, buffer ^ 1);
                    }
                } else {
                    read(0, sub, buffer);
                }
                multiply(sub, sub, buffer);
                staged(sub,
                       [&](int k) {
                           write_a(k, buffer ^ 1, o - o_safe);
                           load_a(k);
                       },
                       [&](int k) {
                           write_b(k, buffer ^ 1, true);
                           load_b(k);
                       });
                // what there is to do on the vector units, six instructions at a time, between the matrix cores': left to itself the
                // compiler puts much of it before or behind them (32768 x 4096 x 4096 bf16 1038 -> 1017 us)
                if constexpr (P == 1) {
#pragma unroll
                    for (int k = 0; k < FO * FI; ++k) {
                        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x2, 6, 0);
                    }
                }
            }
            end_run();
            if constexpr (SETS == 1) __syncthreads();
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // the steps that are left: the last one, which may be short; all of them of fewer than eight outputs
    for (int s = few ? 0 : whole; t_begin + static_cast<long long>(s) * S::step < t_end; ++s) {
        const long long t0 = t_begin + static_cast<long long>(s) * S::step;
#pragma unroll
        for (int k = 0; k < S::a_passes; ++k) {
            const long long t = t0 + k * S::a_rows + a_row;
            Granule<D, 8> g;
#pragma unroll
            for (int w = 0; w < Granule<D, 8>::NW; ++w) g.w[w] = 0;
            if (t < t_end) {
                const D* const at = dy + t * dy_stride + o;
                if (a_there >= 8) {
                    load_any(g, at);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j < a_there) {
                            if constexpr (sizeof(D) == 2) g.w[j / 2] |= static_cast<unsigned>(at[j].v) << (16 * (j & 1));
                            else g.w[j] = __float_as_uint(at[j]);
                        }
                }
            }
            a_reg[k] = g;
        }
#pragma unroll
        for (int k = 0; k < S::b_passes; ++k) {
            const long long t = min(t0 + k * S::b_rows + b_row, t_end - 1);
            b_reg[k] = *reinterpret_cast<const u32x4*>(q + t * pitch + i);
            e_reg[k] = e[t * (pitch / kBlock) + i / kBlock];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < S::a_passes; ++k) write_a(k, 0, 0);
#pragma unroll
        for (int k = 0; k < S::b_passes; ++k) write_b(k, 0, t0 + k * S::b_rows + b_row < t_end);
        __syncthreads();
#pragma unroll
        for (int sub = 0; sub < S::subs; ++sub) {
            read(0, sub, 0);
            multiply(0, sub, 0);
        }
        end_run();
    }

    if (bias != nullptr && i0 == 0 && wi == 0) {
#pragma unroll
        for (int m = 0; m < FO; ++m) {
            const float v = total[m] + __shfl_xor(total[m], 32, 64);
            const int at = o0 + wo + 32 * m + lane;
            if (lane < 32 && at < outputs) {
                if (bias_parts != nullptr) bias_parts[static_cast<long long>(part) * outputs + at] = v;
                else store_elem(bias + at, accumulate ? v + load_elem(bias + at) : v);
            }
        }
    }
    // four consecutive channels of one output
    auto put = [&](int to, int ti, float (&v)[4]) {
        if (to >= outputs || ti >= width) return;
        const long long at = static_cast<long long>(to) * width + ti;
        if (parts != nullptr) {
            store_some<4>(parts + static_cast<long long>(part) * outputs * width + at, v, width - ti);
        } else {
            if (accumulate) {
                float old[4];
                load_some<4>(old, grad + at, width - ti);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] += old[j];
            }
            store_some<4>(grad + at, v, width - ti);
        }
    };
    // A lane has such fours of 32 outputs apart.  Through LDS, a wave's 32 outputs at a time, consecutive lanes get consecutive channels
    // to store: 16384 x 4096 x 1024 bf16 175 -> 168 us.  The smaller square, whose workgroups come and
    // go beside another's products, is faster without (1024 x 4096 x 1024: 20.6 us and 22.1).
    if constexpr (TILE == 256) {
        constexpr int kRow = 32 * FI + 4, kLanes = 8 * FI;   // floats a row takes; lanes that store one
        static_assert(S::threads / 64 * 32 * kRow * 4 <= S::lds_bytes, "the waves' rows fit");
        float* const rows_of_wave = reinterpret_cast<float*>(lds) + wave * (32 * kRow);
#pragma unroll
        for (int m = 0; m < FO; ++m) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < FI; ++k)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    u32x4 w;
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(acc[m][k][4 * r + j]);
                    *reinterpret_cast<u32x4*>(rows_of_wave + (lane & 31) * kRow + 32 * k + 8 * r + 4 * (lane >> 5)) = w;
                }
            __syncthreads();
#pragma unroll 4
            for (int n = lane; n < 32 * kLanes; n += 64) {
                const int row = n / kLanes, col = 4 * (n % kLanes);
                const u32x4 w = *reinterpret_cast<const u32x4*>(rows_of_wave + row * kRow + col);
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(w[j]);
                put(o0 + wo + 32 * m + row, i0 + wi + col, v);
            }
        }
    } else {
#pragma unroll
        for (int m = 0; m < FO; ++m)
#pragma unroll
            for (int k = 0; k < FI; ++k)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = acc[m][k][4 * r + j];
                    put(o0 + wo + 32 * m + (lane & 31), i0 + wi + 32 * k + 8 * r + 4 * (lane >> 5), v);
                }
    }
}

// out (+)= the sum of the parts, in a fixed order: the weight's in the first `groups` workgroups, the bias's in the others.  WAYS waves
// share the parts of 256 elements, where there are many parts of few.
template <typename T>
struct Joined {
    const float* parts;
    int n_parts;
    long long n;
    T* out;
};
template <typename T, int WAYS>
__global__ void __launch_bounds__(256) join_parts_kernel(Joined<T> weight, int groups, Joined<T> bias, int accumulate) {
    __shared__ float shared[WAYS][WAYS > 1 ? 256 : 1];
    const bool first = static_cast<int>(blockIdx.x) < groups;
    const Joined<T> j = first ? weight : bias;
    const long long block = first ? blockIdx.x : blockIdx.x - groups, blocks = first ? groups : gridDim.x - groups;
    const int way = WAYS > 1 ? threadIdx.x >> 6 : 0, lane = WAYS > 1 ? threadIdx.x & 63 : threadIdx.x;
    constexpr int kElems = 1024 / WAYS;
    for (long long base = block * kElems; base < j.n; base += kElems * blocks) {
        const long long at = base + 4 * lane;
        const int there = static_cast<int>(min(4ll, j.n - at));
        float s[4] = {}, v[4];
        if (there > 0) {
#pragma unroll 4
            for (int p = way; p < j.n_parts; p += WAYS) {
                load_some<4>(v, j.parts + p * j.n + at, there);
#pragma unroll
                for (int k = 0; k < 4; ++k) s[k] += v[k];
            }
        }
        if constexpr (WAYS > 1) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 4; ++k) shared[way][4 * lane + k] = s[k];
            __syncthreads();
            if (way != 0) continue;
#pragma unroll
            for (int w = 1; w < WAYS; ++w)
#pragma unroll
                for (int k = 0; k < 4; ++k) s[k] += shared[w][4 * lane + k];
        }
        if (there > 0) {
            if (accumulate) {
                load_some<4>(v, j.out + at, there);
#pragma unroll
                for (int k = 0; k < 4; ++k) s[k] += v[k];
            }
            store_some<4>(j.out + at, s, there);
        }
    }
}

}  // namespace

int launch_weight_grad(const WeightGrad& g, void* stream) {
    return with_types(g.dtype, g.grad_dtype, [&](auto d, auto t) -> int {
        typedef decltype(d) D;
        typedef decltype(t) T;
        if constexpr (sizeof(D) == 8 || sizeof(T) == 8) {
            return static_cast<int>(hipErrorInvalidValue);   // (refused before)
        } else {
            const WeightSplit& w = g.split;
            float* const parts = w.parts > 1 ? reinterpret_cast<float*>(g.ws) : nullptr;
            float* const bias_parts = w.parts > 1 ? reinterpret_cast<float*>(g.ws + w.off_bias) : nullptr;
            T* const grad = static_cast<T*>(g.grad);
            T* const bias = static_cast<T*>(g.bias);
            const int64_t tiles_o = (g.outputs + w.tile - 1) / w.tile, tiles_i = (g.x.width + w.tile - 1) / w.tile;
            const bool wide = w.tile == 256;
            const int lds = wide ? GradShape<D, 256>::lds_bytes : GradShape<D, 128>::lds_bytes;
            const int threads = wide ? GradShape<D, 256>::threads : GradShape<D, 128>::threads;
            const bool ragged = g.outputs % 8 != 0;
            const auto kernel = wide ? (ragged ? weight_grad_kernel<D, T, 256, true> : weight_grad_kernel<D, T, 256, false>)
                                     : (ragged ? weight_grad_kernel<D, T, 128, true> : weight_grad_kernel<D, T, 128, false>);
            int rc = static_cast<int>(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
            if (rc != 0) return rc;
            rc = launch(kernel, tiles_o * tiles_i * w.parts, 1, threads, lds, stream, reinterpret_cast<const signed char*>(g.x.q),
                        reinterpret_cast<const signed char*>(g.x.e), g.x.rows, g.x.width, g.x.pitch, static_cast<const D*>(g.dy), g.dy_stride,
                        g.outputs, grad, g.accumulate, parts, w.steps, tiles_o, tiles_i, bias, bias_parts);
            if (rc != 0 || parts == nullptr) return rc;
            const Joined<T> weights{parts, static_cast<int>(w.parts), g.outputs * g.x.width, grad};
            const Joined<T> sums{bias_parts, static_cast<int>(w.parts), bias != nullptr ? g.outputs : 0, bias};
            const bool few = w.parts >= 8 && weights.n < (1 << 19);
            const int64_t elems = few ? 256 : 1024, groups = at_most_groups((weights.n + elems - 1) / elems);
            return launch(few ? join_parts_kernel<T, 4> : join_parts_kernel<T, 1>, groups + (sums.n + elems - 1) / elems, 1, 256, 0, stream,
                          weights, groups, sums, g.accumulate);
        }
    });
}

}  // namespace adasum
