// gfx950 kernels of embedding tables that lie in a worker's flat buffer: rows looked up, and the table's gradient by sorted tokens.
#include <hip/hip_runtime.h>

#include "adasum_layers.h"
#include "adasum_rows.h"

namespace adasum {
namespace {

// An id as a number that is below 2^31 - 65536 for every row there may be, and far above for ids that name none.
__device__ __forceinline__ unsigned row_of(const Ids& ids, int64_t t) {
    if (ids.wide) {
        const u32x2 id = static_cast<const u32x2*>(ids.p)[t];
        return id.y == 0 ? id.x : ~0u;
    }
    return static_cast<const unsigned*>(ids.p)[t];
}

// ---- rows of the table -----------------------------------------------------------
//
// out[t] = scale * table[ids[t]]: every byte moves once, nothing is computed to speak of.  A workgroup takes consecutive tokens, a
// lane G elements of a row at a time (16 bytes of the narrower type), ITEMS of them in flight.  65536 tokens of 30522 rows of 1024 in fp32
// to bf16: 49 us, 7.6 TB/s with the rows that several tokens name counted as often; stores past the caches give 2 us of that.
template <typename T, typename U, RowForm FORM, int ITEMS>
__global__ void __launch_bounds__(256)
lookup_kernel(const T* __restrict__ table, unsigned rows, int width, Ids ids, typename Traits<T>::acc_t scale, U* __restrict__ out,
              long long out_stride, int tokens, Divider granules) {
    typedef typename Traits<T>::acc_t A;
    constexpr int G = 16 / (sizeof(T) < sizeof(U) ? sizeof(T) : sizeof(U));
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * tokens; first < ids.n; first += static_cast<int64_t>(gridDim.x) * tokens) {
        const int here = static_cast<int>(min(static_cast<int64_t>(tokens), ids.n - first));
        const unsigned work = static_cast<unsigned>(here) * granules.d;
        for (unsigned base = threadIdx.x; base < work; base += 256 * ITEMS) {
            Granule<T, G> raw[ITEMS];
            unsigned id[ITEMS], t[ITEMS];
            int at[ITEMS];
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const unsigned g = min(base + 256 * k, work - 1);
                t[k] = divide(g, granules);
                at[k] = static_cast<int>((g - t[k] * granules.d) * G);
                id[k] = row_of(ids, first + t[k]);
            }
            // (ids that name no row load the first one)
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) load_row<FORM>(raw[k], table + static_cast<long long>(id[k] < rows ? id[k] : 0) * width, at[k], width);
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                A v[G];
                unpack(raw[k], v);
#pragma unroll
                for (int i = 0; i < G; ++i) v[i] = id[k] < rows ? v[i] * scale : A(0);
                if (base + 256 * k < work) store_row<FORM, (ITEMS > 1)>(out + (first + t[k]) * out_stride, v, at[k], width);
            }
        }
    }
}

// ---- sorting the tokens -----------------------------------------------------------
//
// Workgroup j lists the tokens whose id lies in its range of rows, in the order of their ids and, for one id, of the tokens.  It
// reads all ids twice (they stay in L2): once to count how many lie below its range, which is where its list starts, and how many
// tokens of a sixteenth of the input every row has; then, with the places that follow from those counts, to write.  No workgroup
// waits for another.  Workgroups behind the last one clear the table meanwhile.  512
// tokens of 30522 rows: 7.0 us; 4096: 13.4; of 16384 it took 20.6 where sorting in parts takes 17, of 65501 63 and 18.
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortBatch = 16;                   // ids a lane has in flight
constexpr int kClearBytes = 64 * kSortThreads;   // per workgroup

// Counts in LDS that the lanes of a wave write for each other: volatile, and known to be LDS all the same.
typedef volatile __attribute__((address_space(3))) int* lds_counts;

// Zeros over the workgroups' share of the table.
__device__ __forceinline__ void clear_table(long long block, long long blocks, char* __restrict__ clear, long long clear_bytes) {
    const unsigned zero[4] = {0, 0, 0, 0};
    for (long long from = block * kClearBytes; from < clear_bytes; from += blocks * kClearBytes)
        for (int k = threadIdx.x; k < kClearBytes / 16; k += static_cast<int>(blockDim.x)) {
            const long long at = from + 16ll * k;
            if (at + 16 <= clear_bytes) {
                store_words_any<true>(clear + at, zero);
            } else {
                for (long long b = at; b < clear_bytes; b += 2) *reinterpret_cast<unsigned short*>(clear + b) = 0;
            }
        }
}

__global__ void __launch_bounds__(kSortThreads)
sort_kernel(Ids ids, unsigned rows, unsigned per_group, int groups, int* __restrict__ totals, int* __restrict__ place,
            int* __restrict__ row, char* __restrict__ clear, long long clear_bytes) {
    extern __shared__ int counts[];   // [wave][row of the range], then what the scan needs
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (static_cast<int>(blockIdx.x) >= groups) {
        clear_table(blockIdx.x - groups, gridDim.x - groups, clear, clear_bytes);
        return;
    }
    const unsigned lo = blockIdx.x * per_group, mine = min(per_group, rows - lo);
    int* const scan = counts + kSortWaves * per_group;
    for (unsigned i = threadIdx.x; i < kSortWaves * per_group; i += kSortThreads) counts[i] = 0;
    __syncthreads();
    const int64_t segment = ((ids.n + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
    const int64_t begin = min(segment * wave, ids.n), end = min(begin + segment, ids.n);
    const lds_counts my_counts = (lds_counts)(counts + wave * per_group);
    unsigned batch[kSortBatch];
    auto load = [&](int64_t from) {
#pragma unroll
        for (int k = 0; k < kSortBatch; ++k) {
            const int64_t t = from + 64 * k + lane;
            batch[k] = t < end ? row_of(ids, t) : ~0u;
        }
    };
    int below = 0;
    for (int64_t from = begin; from < end; from += 64 * kSortBatch) {
        load(from);
#pragma unroll
        for (int k = 0; k < kSortBatch; ++k) {
            below += batch[k] < lo;
            if (batch[k] - lo < mine) atomicAdd(counts + wave * per_group + (batch[k] - lo), 1);
        }
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) below += __shfl_xor(below, m, 64);
    if (lane == 0) scan[wave] = below;
    __syncthreads();
    int base = 0;
    for (int w = 0; w < kSortWaves; ++w) base += scan[w];
    // one row of the range per thread (per_group is at most kSortThreads): its tokens, and those of the rows before it
    const unsigned r = threadIdx.x;
    int sum = 0;
    if (r < mine)
        for (int w = 0; w < kSortWaves; ++w) sum += counts[w * per_group + r];
    int upto = sum;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int before = __shfl_up(upto, m, 64);
        if (lane >= m) upto += before;
    }
    __syncthreads();
    if (lane == 63) scan[wave] = upto;
    __syncthreads();
    int at = base + upto - sum;
    for (int w = 0; w < wave; ++w) at += scan[w];
    if (r < mine)
        for (int w = 0; w < kSortWaves; ++w) {
            const int n = counts[w * per_group + r];
            counts[w * per_group + r] = at;
            at += n;
        }
    if (blockIdx.x == static_cast<unsigned>(groups) - 1 && r == mine - 1) {
        totals[0] = at;
        totals[1] = 0;   // runs that sum_kernel lists
    }
    __syncthreads();
    const bool kept = end - begin <= 64 * kSortBatch;   // the ids are in registers still
    for (int64_t from = begin; from < end; from += 64 * kSortBatch) {
        if (!kept) load(from);
#pragma unroll
        for (int k = 0; k < kSortBatch; ++k) {
            const unsigned b_mine = batch[k] - lo;
            unsigned long long left = __ballot(b_mine < mine);
            while (left != 0) {
                const int leader = __ffsll(left) - 1;
                const unsigned b = __builtin_amdgcn_readlane(b_mine, leader);
                const unsigned long long same = __ballot(b_mine == b);
                if (b_mine == b) {
                    const int p = my_counts[b] + __popcll(same & ((1ull << lane) - 1));
                    place[p] = static_cast<int>(from) + 64 * k + lane;
                    row[p] = static_cast<int>(batch[k]);
                }
                // (a wave's LDS operations are done in order: the reads above come before this write)
                if (lane == leader) my_counts[b] = my_counts[b] + __popcll(same);
                left &= ~same;
            }
        }
    }
}

// ---- sorting many tokens -------------------------------------------------------------
//
// Where the tokens are many, reading all of them in every workgroup costs more than a launch.  (Equal ids must come to lie together, the
// order of the rows does not matter.)  A row belongs to the range that its lowest bits say: vocabularies often are in the order of
// frequency.  First, workgroups of kPartTokens tokens each sort theirs by range, for themselves, and write down where each range
// begins; what lies below a range in all of them together is where its list starts.  Then one workgroup per range gathers its tokens,
// in order, and sorts them by row.
//
// 65501 tokens of 30522 rows: 6.8 and 10.8 us, most of it one memory access or barrier after another; 131072 take 7.5 and 14.8.
// Both sort in registers: a wave takes 64 tokens at a time, finds by one vote per bit which lanes have the same key, and so ranks them
// behind those of the same key that it has seen before.
constexpr int kRowBits = 10;
static_assert(kGatherRows == 1 << kRowBits && kGatherRows <= kSortThreads, "a range's rows have as many bits, and a lane each");
constexpr int kPartThreads = 512, kPartWaves = kPartThreads / 64, kPartBatch = kPartTokens / kPartThreads;
constexpr int kGatherBatch = 16;   // tokens of a lane that are in registers at most

// The lanes with the same key of BITS bits, among those of `valid`.
template <int BITS>
__device__ __forceinline__ unsigned long long same_key(unsigned key, unsigned long long valid, int bits) {
    unsigned long long same = valid;
#pragma unroll
    for (int b = 0; b < BITS; ++b) {
        if (b >= bits) break;
        const bool one = (key >> b) & 1;
        const unsigned long long ones = __ballot(one);
        same &= one ? ones : ~ones;
    }
    return same;
}

// Sums over the lanes before this one, of every lane's value, across a workgroup of WAVES waves; the sum of all comes back in `all`.
template <int WAVES>
__device__ __forceinline__ int scan_before(int v, int* shared, int& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int upto = v;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int before = __shfl_up(upto, m, 64);
        if (lane >= m) upto += before;
    }
    __syncthreads();
    if (lane == 63) shared[wave] = upto;
    __syncthreads();
    int sum = upto - v;
    all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) sum += shared[w];
        all += shared[w];
    }
    return sum;
}

// The tokens of each part by range: part_place / part_row[part * kPartTokens + i], and begins[range][part], the index of the part's
// first token of that range (range kSortGroups: its tokens that name a row).
__global__ void __launch_bounds__(kPartThreads)
part_kernel(Ids ids, unsigned rows, int n_parts, int* __restrict__ begins, int* __restrict__ part_place,
            int* __restrict__ part_row, char* __restrict__ clear, long long clear_bytes) {
    __shared__ int counts[kPartWaves][kSortGroups];
    __shared__ int first[kSortGroups];
    __shared__ int scan[kPartWaves];
    if (static_cast<int>(blockIdx.x) >= n_parts) {
        clear_table(blockIdx.x - n_parts, gridDim.x - n_parts, clear, clear_bytes);
        return;
    }
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t from = static_cast<int64_t>(blockIdx.x) * kPartTokens + wave * (64 * kPartBatch) + lane;
    unsigned id[kPartBatch];
    int rank[kPartBatch], group[kPartBatch];
#pragma unroll
    for (int k = 0; k < kPartBatch; ++k) id[k] = from + 64 * k < ids.n ? row_of(ids, from + 64 * k) : ~0u;
    for (int i = threadIdx.x; i < kPartWaves * kSortGroups; i += kPartThreads) (&counts[0][0])[i] = 0;
    __syncthreads();
    const lds_counts mine = (lds_counts)(counts[wave]);
#pragma unroll
    for (int k = 0; k < kPartBatch; ++k) {
        const bool valid = id[k] < rows;
        group[k] = valid ? static_cast<int>(id[k] % kSortGroups) : 0;
        const unsigned long long same = same_key<8>(group[k], __ballot(valid), 8);
        const int before = __popcll(same & ((1ull << lane) - 1));
        const int seen = mine[group[k]];
        rank[k] = valid ? seen + before : -1;
        if (valid && before == 0) mine[group[k]] = seen + __popcll(same);
    }
    __syncthreads();
    static_assert(kSortGroups <= kPartThreads, "one range per lane");
    const int r = threadIdx.x;
    int sum = 0;
    if (r < kSortGroups)
        for (int w = 0; w < kPartWaves; ++w) {
            const int n = counts[w][r];
            counts[w][r] = sum;
            sum += n;
        }
    int all = 0;
    const int start = scan_before<kPartWaves>(sum, scan, all);
    if (r < kSortGroups) {
        first[r] = start;
        begins[static_cast<int64_t>(r) * n_parts + blockIdx.x] = start;
    }
    if (r == 0) begins[static_cast<int64_t>(kSortGroups) * n_parts + blockIdx.x] = all;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPartBatch; ++k)
        if (rank[k] >= 0) {
            const int64_t to = static_cast<int64_t>(blockIdx.x) * kPartTokens + first[group[k]] + counts[wave][group[k]] + rank[k];
            part_place[to] = static_cast<int>(from + 64 * k);
            part_row[to] = static_cast<int>(id[k]);
        }
}

// Range blockIdx.x: gathers its tokens from the parts and sorts them by row.
__global__ void __launch_bounds__(kSortThreads)
gather_kernel(unsigned per_group, int row_bits, int n_parts, const int* __restrict__ begins, const int* __restrict__ part_place,
              const int* __restrict__ part_row, int* __restrict__ totals, int* __restrict__ place, int* __restrict__ row,
              char* __restrict__ clear, long long clear_bytes) {
    if (blockIdx.x >= kSortGroups) {
        clear_table(blockIdx.x - kSortGroups, gridDim.x - kSortGroups, clear, clear_bytes);
        return;
    }
    extern __shared__ int counts[];                 // [wave][row of the range], then [row]: where the row's next token goes
    __shared__ int length[kSortThreads];            // of the parts in hand: tokens of this range before them
    __shared__ int source[kSortThreads];            // where theirs begin
    __shared__ int scan[kSortWaves];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int* const begin_here = begins + static_cast<int64_t>(blockIdx.x) * n_parts;
    const int* const begin_next = begin_here + n_parts;
    int* const next = counts + kSortWaves * per_group;
    const lds_counts mine = (lds_counts)(counts + wave * per_group);
    // tokens of the ranges before this one, and of those up to it
    int below = 0, upto = 0, first_here = 0, first_next = 0;
    for (int p = threadIdx.x; p < n_parts; p += kSortThreads) {
        const int b = begin_here[p], e = begin_next[p];
        if (p < kSortThreads) {
            first_here = b;
            first_next = e;
        }
        below += b;
        upto += e;
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
        below += __shfl_xor(below, m, 64);
        upto += __shfl_xor(upto, m, 64);
    }
    if (lane == 0) {
        length[wave] = below;
        source[wave] = upto;
    }
    __syncthreads();
    int all_below = 0, all_here = 0;
    for (int w = 0; w < kSortWaves; ++w) {
        all_below += length[w];
        all_here += source[w];
    }
    all_here -= all_below;
    // 64 tokens of a wave at a time: how often, and how many waves have any
    const int rounds = min(kGatherBatch, (all_here + kSortThreads - 1) / kSortThreads), at_once = kSortThreads * rounds;
    const int ways = min(kSortWaves, (all_here + 64 * rounds - 1) / (64 * rounds));
    if (blockIdx.x == kSortGroups - 1 && threadIdx.x == 0) {
        totals[0] = all_below + all_here;
        totals[1] = 0;   // runs that sum_kernel lists
    }
    if (all_here == 0) return;
    for (unsigned r = threadIdx.x; r < per_group; r += kSortThreads) next[r] = 0;
    // the search for a token's part begins with half of a power of two that is no less than the parts in hand
    const int half_parts = n_parts >= kSortThreads ? kSortThreads / 2 : n_parts > 1 ? 1 << (31 - __builtin_clz(n_parts - 1)) : 0;
    int token[kGatherBatch], rank[kGatherBatch];
    unsigned key[kGatherBatch];
    // f() for every `at_once` tokens of the range, in order: then a wave has consecutive ones, 64 at a time
    auto every = [&](auto&& f) {
        for (int p0 = 0; p0 < n_parts; p0 += kSortThreads) {
            const int p = p0 + static_cast<int>(threadIdx.x);
            const bool later = p0 > 0 && p < n_parts;
            const int b = later ? begin_here[p] : p0 > 0 ? 0 : first_here, n = (later ? begin_next[p] : p0 > 0 ? 0 : first_next) - b;
            int all = 0;
            const int before = scan_before<kSortWaves>(n, scan, all);
            length[threadIdx.x] = before;
            source[threadIdx.x] = b;
            __syncthreads();
            for (int e0 = 0; e0 < all; e0 += at_once) {
#pragma unroll
                for (int k = 0; k < kGatherBatch; ++k) {
                    const int e = e0 + wave * (64 * rounds) + 64 * k + lane;
                    token[k] = -1;
                    key[k] = 0;
                    if (k < rounds && e < all) {
                        // the part that has it: the last one that begins at or before it
                        int q = 0;
                        for (int step = half_parts; step > 0; step >>= 1)
                            if (length[q + step] <= e) q += step;
                        const int64_t from = static_cast<int64_t>(p0 + q) * kPartTokens + source[q] + (e - length[q]);
                        token[k] = part_place[from];
                        key[k] = static_cast<unsigned>(part_row[from]) / kSortGroups;
                    }
                }
                f();
            }
            __syncthreads();
        }
    };
    // from how many tokens the rows have to where theirs begin
    auto rows_begin = [&] {
        const unsigned r = threadIdx.x;
        __syncthreads();
        const int n = r < per_group ? next[r] : 0;
        int all = 0;
        const int before = scan_before<kSortWaves>(n, scan, all);
        if (r < per_group) next[r] = all_below + before;
        __syncthreads();
    };
    const bool once = all_here <= at_once && n_parts <= kSortThreads;
    if (!once) {
        // a hot range, whose tokens come in several batches: first count them all
        every([&] {
#pragma unroll
            for (int k = 0; k < kGatherBatch; ++k) {
                const unsigned long long valid = __ballot(token[k] >= 0);
                if (valid == 0) continue;
                const unsigned long long same = same_key<kRowBits>(key[k], valid, row_bits);
                if (token[k] >= 0 && __popcll(same & ((1ull << lane) - 1)) == 0) atomicAdd(next + key[k], __popcll(same));
            }
        });
        rows_begin();
    }
    every([&] {
        for (unsigned i = threadIdx.x; i < ways * per_group; i += kSortThreads) counts[i] = 0;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kGatherBatch; ++k) {
            const unsigned long long valid = __ballot(token[k] >= 0);
            if (valid == 0) continue;
            const unsigned long long same = same_key<kRowBits>(key[k], valid, row_bits);
            const int before = __popcll(same & ((1ull << lane) - 1)), seen = mine[key[k]];
            rank[k] = seen + before;
            if (token[k] >= 0 && before == 0) mine[key[k]] = seen + __popcll(same);
        }
        __syncthreads();
        const unsigned r = threadIdx.x;
        if (once) {
            if (r < per_group)
                for (int w = 0; w < ways; ++w) next[r] += counts[w * per_group + r];
            rows_begin();
        }
        if (r < per_group) {
            int to = next[r];
            for (int w = 0; w < ways; ++w) {
                const int n = counts[w * per_group + r];
                counts[w * per_group + r] = to;
                to += n;
            }
            next[r] = to;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kGatherBatch; ++k)
            if (token[k] >= 0) {
                const int to = mine[key[k]] + rank[k];
                place[to] = token[k];
                row[to] = static_cast<int>(key[k] * kSortGroups + blockIdx.x);
            }
        __syncthreads();
    });
}

// Where every range has one row only, its tokens are sorted as they are: workgroup (range, piece) moves those of the parts of its piece, a
// wave a part, and at most kPieces pieces.
constexpr int kPieces = 1024;
__global__ void __launch_bounds__(256)
move_kernel(int n_parts, int pieces, int piece_parts, const int* __restrict__ begins, const int* __restrict__ part_place, int* __restrict__ totals,
            int* __restrict__ place, int* __restrict__ row, int groups, char* __restrict__ clear, long long clear_bytes) {
    if (static_cast<int>(blockIdx.x) >= groups) {
        clear_table(blockIdx.x - groups, gridDim.x - groups, clear, clear_bytes);
        return;
    }
    __shared__ int shared[3][4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int range = static_cast<int>(blockIdx.x) / pieces, first = static_cast<int>(blockIdx.x) % pieces * piece_parts;
    const int* const begin_here = begins + static_cast<int64_t>(range) * n_parts;
    const int* const begin_next = begin_here + n_parts;
    // tokens of the ranges before this one, of this one in the parts before, and of all ranges
    int sums[3] = {};
    for (int p = threadIdx.x; p < n_parts; p += 256) {
        sums[0] += begin_here[p];
        if (p < first) sums[1] += begin_next[p] - begin_here[p];
        sums[2] += begins[static_cast<int64_t>(kSortGroups) * n_parts + p];
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) sums[k] += __shfl_xor(sums[k], m, 64);
        if (lane == 0) shared[k][wave] = sums[k];
    }
    __syncthreads();
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        totals[0] = shared[2][0] + shared[2][1] + shared[2][2] + shared[2][3];
        totals[1] = 0;   // runs that sum_kernel lists
    }
    int to = 0;
    for (int w = 0; w < 4; ++w) to += shared[0][w] + shared[1][w];
    for (int p = first; p < min(first + piece_parts, n_parts); ++p) {
        const int b = begin_here[p], n = begin_next[p] - b;
        if ((p & 3) == wave)
#pragma unroll 8
            for (int i = lane; i < n; i += 64) {
                place[to + i] = part_place[static_cast<int64_t>(p) * kPartTokens + b + i];
                row[to + i] = range;
            }
        to += n;
    }
}

// ---- sums over runs of equal ids ----------------------------------------------------
//
// Work is split over the sorted tokens, so a token that half the batch shares costs no more than others.  A wave has a chunk and 64 lanes'
// worth of the elements, eight rows of dy in flight: the row that has been added makes room for the load of the one eight places on.
// What bounds it is memory: 65501 tokens x 1024 (15 % padding) bf16 to fp32, 212 MB, 47 us; added to a table, 314 MB, 70 us; 16384 tokens
// of two rows x 1024 fp32, 67 MB, 14 us.  The code of a flush is there eight times and no more: with sixteen (and all three forms of
// rows in one kernel) it no longer fitted the instruction cache, and 131072 tokens x 64 took 94 us instead of 28.

// A wave's look at a chunk of R sorted tokens: index i stands for place i - R of the chunk, 0 <= i < 3 R.
template <int R>
struct Window {
    int row0, row1;               // of index lane, and of index 64 + lane
    unsigned long long start;     // bit i: a run starts at index i (i < 64)
    unsigned later;               // the same for index 64 + i
    __device__ __forceinline__ int row_at(int i) const {
        return i < 64 ? __builtin_amdgcn_readlane(row0, i) : __builtin_amdgcn_readlane(row1, i - 64);
    }
    // Whether the run that starts at index a (a < 2 R) has more than R tokens.
    __device__ __forceinline__ bool is_long(int a) const { return row_at(a + R) == row_at(a); }
    // The runs that start before the chunk, and in its first `there` tokens, as bits; the index of the first start behind a full chunk.
    __device__ __forceinline__ unsigned before() const { return static_cast<unsigned>(start) & (~0u >> (32 - R)); }
    __device__ __forceinline__ unsigned inside(int there) const { return static_cast<unsigned>(start >> R) & (~0u >> (32 - there)); }
    __device__ __forceinline__ int behind() const {
        const unsigned bits = R == 32 ? later : static_cast<unsigned>(start >> (R == 32 ? 0 : 2 * R));
        return 2 * R + __builtin_ctz(bits | 0x80000000u);
    }
};
template <int R>
__device__ __forceinline__ Window<R> look(const int* row, int total, int64_t chunk, int lane) {
    static_assert(R == 16 || R == 32, "the window is 48 or 96 places");
    Window<R> w;
    const int64_t p0 = chunk * R - R + lane, p1 = p0 + 64;
    w.row0 = p0 >= 0 && p0 < total ? row[p0] : p0 < 0 ? -1 : -2;
    const int left = __shfl_up(w.row0, 1, 64);
    w.start = __ballot(lane > 0 && w.row0 != left);
    w.row1 = -2;
    w.later = 0;
    if constexpr (R == 32) {
        const int last = __shfl(w.row0, 63, 64);
        if (lane < R && p1 < total) w.row1 = row[p1];
        const int left1 = __shfl_up(w.row1, 1, 64);
        w.later = static_cast<unsigned>(__ballot(lane < R && w.row1 != (lane == 0 ? last : left1)));
    }
    return w;
}

// One wave: chunk `chunk`, the elements of `slice`.  The chunks in which a run of more than R tokens
// starts are listed (`longs` counts them), in no certain order.
constexpr int kBatch = 8;   // rows of dy in flight
template <int R, typename D, typename T, RowForm FORM, bool ADD>
__device__ __forceinline__ void
sum_chunk(long long chunk, int slice, int lane, const D* __restrict__ dy, long long dy_stride, int width, int total,
          const int* __restrict__ place, const int* __restrict__ row, typename Traits<D>::acc_t scale, T* __restrict__ grad,
          typename Traits<D>::acc_t* __restrict__ parts, int* __restrict__ longs, int* __restrict__ listed) {
    typedef typename Traits<D>::acc_t A;
    constexpr int G = Traits<D>::VEC;
    const Window<R> w = look<R>(row, total, chunk, lane);
    const int there = static_cast<int>(min(static_cast<long long>(R), total - chunk * R));
    // the tokens of index R and on
    const int64_t pp = chunk * R + lane;
    const int token = pp < total ? place[pp] : 0;
    int from = R, until = R + there;
    // runs that start here (behind the last token is no run)
    const unsigned starts = w.inside(there);
    bool carried = false;   // the first run is a long one that comes from the chunk before
    if (!(starts & 1)) {
        const unsigned before = w.before();
        const int a = before != 0 ? 31 - __builtin_clz(before) : -1;
        carried = a < 0 || w.is_long(a);
        if (!carried) {
            if (starts == 0) return;   // all of the chunk belongs to a run that the wave before has
            from = R + __builtin_ctz(starts);
        }
    }
    // the last run that starts here: whole if it is not long, else as far as the chunk goes
    bool open = false;
    if (starts != 0) {
        open = w.is_long(R + 31 - __builtin_clz(starts));
        // (not long: the next run, or the end of the tokens, is in the window)
        if (!open && there == R) until = w.behind();
        if (open && slice == 0 && lane == 0) listed[atomicAdd(longs, 1)] = static_cast<int>(chunk);
    }
    const int at = (slice * 64 + lane) * G;
    auto ends_at = [&](int i) { return i + 1 == until || (i + 1 < 64 ? (w.start >> (i + 1)) & 1 : (w.later >> (i + 1 - 64)) & 1); };
    auto goes_on = [&](int i) { return open && i + 1 == until; };
    A sum[G];
#pragma unroll
    for (int i = 0; i < G; ++i) sum[i] = A(0);
    bool first_run = carried;
    Granule<D, G> v[kBatch];
    Granule<T, G> old[ADD ? kBatch : 1];
    auto load = [&](int k, int index) {
        // (the last one again behind the last: a branch here would have the loads waited for at its end)
        const int i = min(index, until - 1);
        const int t = __builtin_amdgcn_readlane(token, i - R);
        load_row<FORM>(v[k], dy + static_cast<long long>(t) * dy_stride, at, width);
        if constexpr (ADD) load_row<FORM>(old[k], grad + static_cast<long long>(w.row_at(i)) * width, at, width);
    };
#pragma unroll
    for (int k = 0; k < kBatch; ++k) load(k, from + k);
    for (int i0 = from; i0 < until; i0 += kBatch) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int i = i0 + k;
            A x[G];
            unpack(v[k], x);
#pragma unroll
            for (int j = 0; j < G; ++j) sum[j] += x[j];
            if (i < until && ends_at(i)) {
                if (first_run || goes_on(i)) {
                    // (the one that comes from before and goes on lies in the first place)
                    store_row<FORM>(parts + (2 * chunk + (first_run ? 0 : 1)) * width, sum, at, width);
                } else {
#pragma unroll
                    for (int j = 0; j < G; ++j) sum[j] *= scale;
                    if constexpr (ADD) {
                        A o[G];
                        unpack(old[k], o);
#pragma unroll
                        for (int j = 0; j < G; ++j) sum[j] += o[j];
                    }
                    store_row<FORM>(grad + static_cast<long long>(w.row_at(i)) * width, sum, at, width);
                }
#pragma unroll
                for (int j = 0; j < G; ++j) sum[j] = A(0);
                first_run = false;
            }
            load(k, i + kBatch);
        }
    }
}

template <int R, typename D, typename T, RowForm FORM, bool ADD>
__global__ void __launch_bounds__(256)
sum_kernel(const D* __restrict__ dy, long long dy_stride, int width, int* __restrict__ totals, const int* __restrict__ place,
           const int* __restrict__ row, typename Traits<D>::acc_t scale, T* __restrict__ grad, typename Traits<D>::acc_t* __restrict__ parts,
           int* __restrict__ listed, int slices, long long n_chunks) {
    const int lane = threadIdx.x & 63;
    const int total = totals[0];
    const long long units = min(n_chunks, (static_cast<long long>(total) + R - 1) / R) * slices;
    for (long long unit = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 6); unit < units; unit += 4ll * gridDim.x) {
        const int slice = static_cast<int>(unit % slices);
        const long long chunk = unit / slices;
        sum_chunk<R, D, T, FORM, ADD>(chunk, slice, lane, dy, dy_stride, width, total, place, row, scale, grad, parts, totals + 1, listed);
    }
}

// A sum in fp64 to the result's type, with one rounding: on the way to 16 bits fp32 takes what is cut off into its last bit (rounding to
// odd; it has more than two bits more than either type, at all magnitudes), so that the second rounding sees on which side of half a
// step the sum lies.
__device__ __forceinline__ float to_odd(double s) {
    const float f = static_cast<float>(s);
    if (!(static_cast<double>(f) != s) || s != s) return f;
    const unsigned bits = __float_as_uint(f);
    return __uint_as_float((fabs(static_cast<double>(f)) > fabs(s) ? bits - 1 : bits) | 1u);
}
__device__ __forceinline__ void store_sum(double* p, double s) { *p = s; }
__device__ __forceinline__ void store_sum(float* p, double s) { *p = static_cast<float>(s); }
template <typename T>
__device__ __forceinline__ void store_sum(T* p, double s) { store_elem(p, to_odd(s)); }

// The parts of long runs.  A compute unit alone reads little, so a workgroup takes 64 elements only: groups of sixteen lanes share a
// run's chunks, four elements a lane.
constexpr int64_t kMostJoins = 8192;   // workgroups
template <int R, int THREADS, typename D, typename T>
__global__ void __launch_bounds__(THREADS)
join_kernel(int width, const int* __restrict__ totals, const int* __restrict__ row, typename Traits<D>::acc_t scale, T* __restrict__ grad,
            int accumulate, const typename Traits<D>::acc_t* __restrict__ parts, const int* __restrict__ listed) {
    typedef typename Traits<D>::acc_t A;
    constexpr int kJoinGroups = THREADS / 16;
    __shared__ double shared[kJoinGroups][64];
    const int lane = threadIdx.x & 63, group = threadIdx.x >> 4, col = 4 * (threadIdx.x & 15);
    const int total = totals[0];
    const long long slices = (width + 63) / 64, units = totals[1] * slices, n_chunks = (static_cast<long long>(total) + R - 1) / R;
    for (long long unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const long long chunk = listed[unit / slices];
        const Window<R> w = look<R>(row, total, chunk, lane);
        const int key = w.row_at(R + 31 - __builtin_clz(w.inside(R)));
        // the last chunk that begins with this row (the next one does): the chunks up to `lo` do, those from `hi` on do not
        long long lo = chunk + 1, hi = n_chunks;
        while (hi - lo > 1) {
            const long long step = (hi - lo + 63) / 64, c = lo + (lane + 1) * step;
            const unsigned long long same = __ballot(c < hi && row[c < hi ? c * R : 0] == key);
            const int yes = same == ~0ull ? 64 : __ffsll(~same) - 1;
            const long long next = lo + yes * step;
            hi = min(hi, next + step);
            lo = next;
        }
        const int at = static_cast<int>(unit % slices) * 64 + col, have = width - at;
        const long long n = lo - chunk + 1;
        double sum[4] = {};
        if (have > 0) {
#pragma unroll 8
            for (long long c = group; c < n; c += kJoinGroups) {
                A v[4];
                load_some<4>(v, parts + (2 * (chunk + c) + (c == 0 ? 1 : 0)) * width + at, have);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] += v[j];
            }
        }
        __syncthreads();   // (all have read what the last round left there)
#pragma unroll
        for (int j = 0; j < 4; ++j) shared[group][col + j] = sum[j];
        __syncthreads();
        if (threadIdx.x < 64) {
            const int e = static_cast<int>(unit % slices) * 64 + lane;
            if (e < width) {
                double s = 0;
#pragma unroll
                for (int g = 0; g < kJoinGroups; ++g) s += shared[g][lane];
                s *= scale;
                T* const to = grad + static_cast<long long>(key) * width + e;
                store_sum(to, accumulate ? s + load_elem(to) : s);
            }
        }
    }
}

int slices_of(int64_t width, int dtype) {
    const int per = 64 * 16 / elem_bytes(dtype);
    return static_cast<int>((width + per - 1) / per);
}

}  // namespace

EmbeddingLayout embedding_layout(int64_t rows, int64_t width, int64_t n_ids, int dtype) {
    EmbeddingLayout l;
    l.run = n_ids <= kFewTokens ? 16 : 32;
    l.chunks = (n_ids + l.run - 1) / l.run;
    l.off_listed = 256;
    l.off_place = align_up(l.off_listed + 4 * static_cast<size_t>(l.chunks), 256);
    l.off_row = align_up(l.off_place + 4 * static_cast<size_t>(n_ids), 256);
    size_t end = align_up(l.off_row + 4 * static_cast<size_t>(n_ids), 256);
    if (in_parts(rows, n_ids)) {
        const size_t n_parts = (static_cast<size_t>(n_ids) + kPartTokens - 1) / kPartTokens;
        l.off_begins = end;
        l.off_part_place = align_up(l.off_begins + 4 * (kSortGroups + 1) * n_parts, 256);
        l.off_part_row = l.off_part_place + 4 * n_parts * kPartTokens;
        end = l.off_part_row + 4 * n_parts * kPartTokens;
    }
    l.off_parts = end;
    l.total = l.off_parts + static_cast<size_t>(l.chunks) * 2 * width * (dtype == ADASUM_F64 ? 8 : 4);
    return l;
}

int launch_lookup(int dtype, int out_dtype, const void* table, int64_t rows, int64_t width, const Ids& ids, double scale, void* out,
                  int64_t out_stride, void* stream) {
    return with_types(dtype, out_dtype, [&](auto t, auto u) -> int {
        typedef decltype(t) T;
        typedef decltype(u) U;
        constexpr int G = 16 / (sizeof(T) < sizeof(U) ? sizeof(T) : sizeof(U));
        const int64_t granules = (width + G - 1) / G;
        // one granule of a lane in flight, or four, stored past the caches (rows of 1024, in thousands of granules): 131: 2.6 and 3.4 us; 262: 3.6
        // and 3.8, in fp32 4.8 and 4.5; 4194: 25.4 and 21.7; 16777: 93 and 77, in fp32 192 and 153
        const bool large = ids.n * granules > (1 << 18);
        const int64_t per_block = large ? 1024 : 256;
        const int64_t tokens = granules >= per_block ? 1 : per_block / granules;
        const int64_t blocks = (ids.n + tokens - 1) / tokens;
        return with_form(row_form(width, G), [&](auto form) -> int {
            constexpr RowForm F = decltype(form)::value;
            return launch(large ? lookup_kernel<T, U, F, 4> : lookup_kernel<T, U, F, 1>, at_most_groups(blocks), 1, 256, 0, stream,
                          static_cast<const T*>(table), rows, width, ids, scale, static_cast<U*>(out), out_stride, tokens,
                          make_divider(static_cast<unsigned>(granules)));
        });
    });
}

int launch_embedding_grad(const EmbeddingGrad& g, void* stream) {
    const int64_t clear_bytes = g.accumulate ? 0 : g.rows * g.width * elem_bytes(g.grad_dtype);
    int* const totals = reinterpret_cast<int*>(g.ws + g.lay.off_totals);
    int* const listed = reinterpret_cast<int*>(g.ws + g.lay.off_listed);
    int* const place = reinterpret_cast<int*>(g.ws + g.lay.off_place);
    int* const row = reinterpret_cast<int*>(g.ws + g.lay.off_row);
    char* const clear = static_cast<char*>(g.grad);
    int rc = 0;
    if (in_parts(g.rows, g.ids.n)) {
        const int64_t per_group = (g.rows + kSortGroups - 1) / kSortGroups, n_parts = (g.ids.n + kPartTokens - 1) / kPartTokens;
        int row_bits = 0;
        while ((1 << row_bits) < per_group) ++row_bits;
        int* const begins = reinterpret_cast<int*>(g.ws + g.lay.off_begins);
        int* const part_place = reinterpret_cast<int*>(g.ws + g.lay.off_part_place);
        int* const part_row = reinterpret_cast<int*>(g.ws + g.lay.off_part_row);
        // each launch clears half of the table
        const int64_t half = clear_bytes / 2 / kClearBytes * kClearBytes;
        rc = launch(part_kernel, n_parts + at_most_groups((half + kClearBytes - 1) / kClearBytes), 1, kPartThreads, 0, stream, g.ids, g.rows, n_parts, begins, part_place, part_row, clear, half);
        if (rc != 0) return rc;
        const int64_t clearing = at_most_groups((clear_bytes - half + kClearBytes - 1) / kClearBytes);
        if (per_group == 1) {
            const int64_t piece_parts = n_parts <= 4 * kPieces ? 4 : (n_parts + kPieces - 1) / kPieces;
            const int64_t pieces = (n_parts + piece_parts - 1) / piece_parts, groups = g.rows * pieces;
            rc = launch(move_kernel, groups + clearing, 1, 256, 0, stream, n_parts, pieces, piece_parts, begins, part_place, totals, place, row, groups,
                        clear + half, clear_bytes - half);
        } else {
            rc = static_cast<int>(hipFuncSetAttribute(reinterpret_cast<const void*>(gather_kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                      static_cast<int>(sizeof(int) * (kSortWaves + 1) * kGatherRows)));
            if (rc != 0) return rc;
            rc = launch(gather_kernel, kSortGroups + clearing, 1, kSortThreads, sizeof(int) * (kSortWaves + 1) * per_group, stream, per_group,
                        row_bits, n_parts, begins, part_place, part_row, totals, place, row, clear + half, clear_bytes - half);
        }
    } else {
        const int64_t per_group = sort_rows(g.rows);
        const int64_t groups = g.ids.n == 0 ? 0 : (g.rows + per_group - 1) / per_group;
        const int64_t clearing = at_most_groups((clear_bytes + kClearBytes - 1) / kClearBytes);
        if (groups + clearing == 0) return 0;
        const size_t lds = sizeof(int) * (static_cast<size_t>(kSortWaves) * per_group + kSortWaves);
        rc = launch(sort_kernel, groups + clearing, 1, kSortThreads, lds, stream, g.ids, g.rows, per_group, groups, totals, place, row, clear,
                    clear_bytes);
    }
    if (rc != 0 || g.ids.n == 0) return rc;
    return with_types(g.dtype, g.grad_dtype, [&](auto d, auto t) -> int {
        typedef decltype(d) D;
        typedef decltype(t) T;
        typedef typename Traits<D>::acc_t A;
        const int slices = slices_of(g.width, g.dtype);
        const int64_t units = g.lay.chunks * slices;
        A* const parts = reinterpret_cast<A*>(g.ws + g.lay.off_parts);
        auto go = [&](auto run) -> int {
            constexpr int R = decltype(run)::value;
            const int rc2 = with_form(row_form(g.width, Traits<D>::VEC), [&](auto form) -> int {
                constexpr RowForm F = decltype(form)::value;
                return launch(g.accumulate ? sum_kernel<R, D, T, F, true> : sum_kernel<R, D, T, F, false>, at_most_groups((units + 3) / 4), 1, 256,
                              0, stream, static_cast<const D*>(g.dy), g.dy_stride, g.width, totals, place, row, g.scale,
                              static_cast<T*>(g.grad), parts, listed, slices, g.lay.chunks);
            });
            if (rc2 != 0 || g.ids.n <= R) return rc2;   // (so few tokens make no long run)
            // Runs times slices, at most; workgroups that find nothing cost less than workgroups that take turns (512 rows x 1024, 65536 tokens: 66.0 us
            // with up to 8192 of them, 70.4 with 1024; 32768 rows 63.7 and 64.3; 4096 tokens of 30522 rows 29.0 both).
            const int64_t slices64 = (g.width + 63) / 64, most = (g.ids.n / (R + 1)) * slices64;
            // Workgroups of 1024 lanes shorten the way through a run's parts, but need the room of four: they are better where few runs share
            // many tokens (whole calls, bf16, 256 and 1024 lanes: 16384 tokens, two rows x 1024 35.7 and 30.0 us; 131072, 8 rows x 1024 75.6 and
            // 70.6; 131072, 16 rows x 64 33.5 and 29.5) and worse elsewhere (16384 tokens, 16 rows x 1024 25.2 and 31.2; 65536, 32 rows x 256
            // 27.5 and 30.6; 131072, 16 rows x 1024 69 and 72.5; 65536, 64 rows x 64 24.7 and 24.9).
            const bool few = static_cast<double>(g.ids.n) >= 64.0 * static_cast<double>(g.rows) * static_cast<double>(g.rows * slices64);
            return launch(few ? join_kernel<R, 1024, D, T> : join_kernel<R, 256, D, T>, most < kMostJoins ? most : kMostJoins, 1, few ? 1024 : 256, 0,
                          stream, g.width, totals, row, g.scale, static_cast<T*>(g.grad), g.accumulate, parts, listed);
        };
        return g.lay.run == 16 ? go(std::integral_constant<int, 16>{}) : go(std::integral_constant<int, 32>{});
    });
}

}  // namespace adasum
