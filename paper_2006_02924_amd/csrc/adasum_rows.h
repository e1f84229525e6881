// Device code shared by the operators on rows: 16-byte accesses at any element's alignment, values in fp32 or fp64.
#pragma once

#include <tuple>

#include "adasum_device.h"

namespace adasum {
namespace {

// Launches a kernel and says how that went, whatever error an earlier call of this thread left behind.
template <typename... P, typename... A>
int launch(void (*kernel)(P...), int64_t groups, int64_t parts, int threads, size_t lds, void* stream, const A&... args) {
    std::tuple<P...> values(static_cast<P>(args)...);
    return std::apply(
        [&](P&... v) {
            void* pointers[] = {const_cast<void*>(reinterpret_cast<const void*>(&v))...};
            return static_cast<int>(hipLaunchKernel(reinterpret_cast<const void*>(kernel),
                                                    dim3(static_cast<unsigned>(groups), static_cast<unsigned>(parts)), dim3(threads), pointers,
                                                    lds, static_cast<hipStream_t>(stream)));
        },
        values);
}
// Workgroups of a launch at most: the kernels go round.
constexpr int64_t kMostGroups = 1 << 20;
inline int64_t at_most_groups(int64_t groups) { return groups < kMostGroups ? groups : kMostGroups; }

// A row may start anywhere (a layer of a flat buffer, a slice of a wider matrix): the memory system takes 16-byte accesses at
// every element's alignment, the type only has to say so.
typedef unsigned int u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned int u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

// (Not through templates of any type: as a template's argument a type loses the alignment that it was declared with.)
template <bool NT>
__device__ __forceinline__ u32x4 load_at(const u32x4_any* p) {
    if constexpr (NT && ADASUM_NT_LOAD) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool NT>
__device__ __forceinline__ u32x2 load_at(const u32x2_any* p) {
    if constexpr (NT && ADASUM_NT_LOAD) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool NT>
__device__ __forceinline__ void store_at(u32x4 v, u32x4_any* p) {
    if constexpr (NT && ADASUM_NT_STORE) __builtin_nontemporal_store(v, p);
    else *p = v;
}
template <bool NT>
__device__ __forceinline__ void store_at(u32x2 v, u32x2_any* p) {
    if constexpr (NT && ADASUM_NT_STORE) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// NT: what is used once passes the caches by (streams of many megabytes; see the kernels for what that gave).
template <bool NT = false, typename T, int G>
__device__ __forceinline__ void load_any(Granule<T, G>& r, const T* p) {
    constexpr int NW = Granule<T, G>::NW;
    if constexpr (NW == 2) {
        const u32x2 q = load_at<NT>(reinterpret_cast<const u32x2_any*>(p));
        r.w[0] = q.x;
        r.w[1] = q.y;
    } else {
#pragma unroll
        for (int i = 0; i < NW / 4; ++i) {
            const u32x4 q = load_at<NT>(reinterpret_cast<const u32x4_any*>(p) + i);
            r.w[4 * i + 0] = q.x;
            r.w[4 * i + 1] = q.y;
            r.w[4 * i + 2] = q.z;
            r.w[4 * i + 3] = q.w;
        }
    }
}

template <bool NT = false, int NW>
__device__ __forceinline__ void store_words_any(void* p, const unsigned int (&w)[NW]) {
    if constexpr (NW == 2) {
        u32x2 q;
        q.x = w[0];
        q.y = w[1];
        store_at<NT>(q, reinterpret_cast<u32x2_any*>(p));
    } else {
#pragma unroll
        for (int i = 0; i < NW / 4; ++i) {
            u32x4 q;
            q.x = w[4 * i + 0];
            q.y = w[4 * i + 1];
            q.z = w[4 * i + 2];
            q.w = w[4 * i + 3];
            store_at<NT>(q, reinterpret_cast<u32x4_any*>(p) + i);
        }
    }
}

// Two values rounded to a 16-bit type (to nearest even, by the conversion instructions).
__device__ __forceinline__ unsigned int rounded_pair(bf16_t, float a, float b) {
    bf16x2_t p;
    p.x = static_cast<__bf16>(a);
    p.y = static_cast<__bf16>(b);
    return __builtin_bit_cast(unsigned int, p);
}
__device__ __forceinline__ unsigned int rounded_pair(f16_t, float a, float b) {
    return f32_to_f16_bits(a) | f32_to_f16_bits(b) << 16;
}

// G values to consecutive elements of T.
template <int G, bool NT = false, typename T, typename A>
__device__ __forceinline__ void store_any(T* p, const A (&v)[G]) {
    unsigned int w[Granule<T, G>::NW];
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < G / 2; ++i) w[i] = rounded_pair(T{}, v[2 * i], v[2 * i + 1]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < G; ++i) w[i] = __float_as_uint(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const long long b = __double_as_longlong(v[i]);
            w[2 * i] = static_cast<unsigned int>(b);
            w[2 * i + 1] = static_cast<unsigned int>(b >> 32);
        }
    }
    store_words_any<NT>(p, w);
}

// `there` (1 .. G) elements of T as values, zeros behind them.  (What is loaded in a branch is waited for at its end: for kernels that keep
// many loads in flight see load_row.)
template <int G, typename T, typename A>
__device__ __forceinline__ void load_some(A (&v)[G], const T* p, int there) {
    if (there >= G) {
        Granule<T, G> r;
        load_any(r, p);
        unpack(r, v);
    } else {
#pragma unroll
        for (int i = 0; i < G; ++i) v[i] = i < there ? load_elem(p + i) : A(0);
    }
}
template <int G, bool NT = false, typename T, typename A>
__device__ __forceinline__ void store_some(T* p, const A (&v)[G], int there) {
    if (there >= G) {
        store_any<G, NT>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < G; ++i)
            if (i < there) store_elem(p + i, v[i]);
    }
}

// How rows of `width` elements fall into granules of G: whole ones; a last one that is shorter, which is loaded as the row's last G elements
// and moved down, without a branch; rows shorter than a granule, element by element.
enum RowForm { kWhole, kRagged, kShort };
inline RowForm row_form(int64_t width, int G) { return width % G == 0 ? kWhole : width >= G ? kRagged : kShort; }

// Moves a granule's elements `by` places down.
template <typename T, int G>
__device__ __forceinline__ void move_down(Granule<T, G>& r, int by) {
    constexpr int NW = Granule<T, G>::NW;
    const int halves = by * static_cast<int>(sizeof(T) / 2);
#pragma unroll
    for (int step = NW / 2; step >= 1; step /= 2) {
        const bool yes = (halves / 2) & step;
#pragma unroll
        for (int i = 0; i + step < NW; ++i) {
            const unsigned here = r.w[i], there = r.w[i + step];   // (values: a choice between places would put the granule in memory)
            r.w[i] = yes ? there : here;
        }
    }
    if constexpr (sizeof(T) == 2) {
        const bool yes = halves & 1;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const unsigned here = r.w[i], moved = here >> 16 | (i + 1 < NW ? r.w[i + 1] << 16 : 0u);
            r.w[i] = yes ? moved : here;
        }
    }
}

// The granule at element `at` of a row; what lies behind the row's end is not defined (`at` may lie there too).
template <RowForm FORM, bool NT = false, typename T, int G>
__device__ __forceinline__ void load_row(Granule<T, G>& r, const T* row, int at, int width) {
    if constexpr (FORM == kWhole) {
        load_any<NT>(r, row + (at < width ? at : 0));
    } else if constexpr (FORM == kRagged) {
        const int from = min(at, width - G);
        load_any<NT>(r, row + from);
        move_down(r, at - from);
    } else {
#pragma unroll
        for (int w = 0; w < Granule<T, G>::NW; ++w) r.w[w] = 0;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const T* const p = row + min(at + i, width - 1);
            if constexpr (sizeof(T) == 2) {
                r.w[i / 2] |= static_cast<unsigned>(p->v) << (16 * (i & 1));
            } else if constexpr (sizeof(T) == 4) {
                r.w[i] = __float_as_uint(*p);
            } else {
                const long long b = __double_as_longlong(*p);
                r.w[2 * i] = static_cast<unsigned>(b);
                r.w[2 * i + 1] = static_cast<unsigned>(b >> 32);
            }
        }
    }
}
template <RowForm FORM, bool NT = false, int G, typename T, typename A>
__device__ __forceinline__ void store_row(T* row, const A (&v)[G], int at, int width) {
    if constexpr (FORM == kWhole) {
        if (at < width) store_any<G, NT>(row + at, v);
    } else {
        store_some<G, NT>(row + at, v, width - at);
    }
}

// Division of numbers below 2^31 by a fixed one, by a multiplication: q = (n * m) >> (32 + s) with
// m = ceil(2^(32 + s) / d), 2^s >= d; the product is taken with a 33-bit m (its top bit is always set).
struct Divider {
    unsigned d, m, s;
};
inline Divider make_divider(unsigned d) {
    Divider r{d, 0, 0};
    while ((1ull << r.s) < d) ++r.s;
    const unsigned long long top = (1ull << 32) * ((1ull << r.s) - d) / d + 1;
    r.m = static_cast<unsigned>(top);
    return r;
}
__device__ __forceinline__ unsigned divide(unsigned n, const Divider& v) {
    return static_cast<unsigned>((static_cast<unsigned long long>(__umulhi(n, v.m)) + n) >> v.s);
}

// f(form) as a constant.
template <typename F>
int with_form(RowForm form, F&& f) {
    switch (form) {
        case kWhole: return f(std::integral_constant<RowForm, kWhole>{});
        case kRagged: return f(std::integral_constant<RowForm, kRagged>{});
        default: return f(std::integral_constant<RowForm, kShort>{});
    }
}
// f(type of a, type of b) for storage types that go together.
template <typename F>
int with_type(int dtype, F&& f) {
    switch (dtype) {
        case ADASUM_F32: return f(float{});
        case ADASUM_BF16: return f(bf16_t{});
        default: return f(f16_t{});
    }
}
template <typename F>
int with_types(int a, int b, F&& f) {
    if (a == ADASUM_F64) return f(double{}, double{});
    return with_type(a, [&](auto ta) { return with_type(b, [&](auto tb) { return f(ta, tb); }); });
}

}  // namespace
}  // namespace adasum
