// gfx950 kernel of dropout whose mask is never stored: a stream like those of the checkpoints, eight channels a lane.  Memory bounds it: 32768 x
// 4096 in bf16 (537 MB) take 90 us, 5.9 TB/s.  The mask's products, ten rounds of two for eight elements, take the vector units some 65 us of
// that; with 32 bits an element instead of 16 they would be twice as many, and the longer ones.
#include <hip/hip_runtime.h>

#include "adasum_layers.h"
#include "adasum_mask.h"

namespace adasum {
namespace {

// (x and out may be the same rows: a lane loads what it stores before it does)
template <typename T, RowForm FORM, int ITEMS>
__global__ void __launch_bounds__(kThreadsRow)
dropout_kernel(const T* x, long long x_stride, int width, T* out, long long out_stride, Mask mask, RowWork work) {
    constexpr bool NT = ITEMS > 1;
    const Step step = step_of(mask);
    every_rows(work, [&](long long first, unsigned n) {
        for (unsigned base = threadIdx.x; base < n; base += kThreadsRow * ITEMS) {
            Granule<T, kG> raw[ITEMS];
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const Place p = place_of(work, first, min(base + kThreadsRow * k, n - 1));
                load_row<FORM, NT>(raw[k], x + p.row * x_stride, p.at, width);
            }
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const unsigned g = base + kThreadsRow * k;
                if (g < n) {
                    const Place p = place_of(work, first, g);
                    float v[kG];
                    unpack(raw[k], v);
                    if (mask.drops) {
                        unsigned w[4];
                        bool keep[kG];
                        mask_words(w, mask, step, static_cast<unsigned>(p.at) / kG, static_cast<unsigned>(p.row));
                        kept(keep, w, mask.below);
                        drop(v, keep, mask.factor);
                    }
                    store_row<FORM, NT>(out + p.row * out_stride, v, p.at, width);
                }
            }
        }
    });
}

// Four granules of a lane in flight, past the caches, or one through them (thousands of granules in bf16, microseconds with one and with four):
// 1049 7.9 and 8.4, 2097 12.8 and 15.0, 4194 22.6 and 26.0, where the caches hold something; 16777 97 and 91, and 91 and 91 with other operands in between.
constexpr int64_t kMany = 1 << 23;

}  // namespace

int launch_dropout(const void* x, int dtype, int64_t x_stride, int64_t rows, int64_t width, double p, uint64_t seed, const void* step, void* out,
                   int64_t out_stride, void* stream) {
    const RowGrid g = row_grid(rows, (width + kG - 1) / kG * kG, dtype, kMany);
    const Mask mask = make_mask(p, seed, step);
    return with_type(dtype, [&](auto t) -> int {
        typedef decltype(t) T;
        return with_form(row_form(width, kG), [&](auto form) -> int {
            constexpr RowForm F = decltype(form)::value;
            return with_items<T>(g, [&](auto items) -> int {
                return launch(dropout_kernel<T, F, decltype(items)::value>, g.groups, 1, kThreadsRow, 0, stream, static_cast<const T*>(x), x_stride,
                              width, static_cast<T*>(out), out_stride, mask, g.work);
            });
        });
    });
}

}  // namespace adasum
