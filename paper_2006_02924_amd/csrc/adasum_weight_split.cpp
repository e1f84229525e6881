// How a weight gradient is split over workgroups (host only).
#include "adasum_layers.h"

namespace adasum {

// The edge of a workgroup's square and the number of parts, by what a call would take (microseconds): a fixed time, the steps of a
// workgroup, and the second launch where there are parts.  A workgroup of edge 256 has a compute unit to itself, two of edge 128 share
// one.  Measured, a step takes 1.8 us (fp32: 2.5) with edge 256; with edge 128, which reads more for its products, 0.85 (1.25)
// alone on its compute unit and 1.4 (1.95) beside another.  Examples (bf16, edge / parts): 256 x 2048 x 1000 10.3 us with 128 / 1, 17.3
// with 256 / 1, 18.8 with 128 / 2; 2048 x 1024 x 1024 23 with 128 / 4, 30 with 256 / 8; 16384 x 1024 x 1024 54 with 256 / 16, 56
// with 128 / 8; 16384 x 1024 x 4096 139 with 256 / 4, 200 with 128 / 2; 65536 x 64 x 64 21.5 with 128 / 128, 27.3 with 256 / 128.
WeightSplit weight_split(int64_t rows, int64_t width, int64_t outputs, int dtype) {
    const bool f32 = dtype == ADASUM_F32;
    const int64_t step = f32 ? 32 : 64, steps = (rows + step - 1) / step;
    static constexpr int kCounts[] = {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 32, 48, 64, 96, 128, 192, 256};
    WeightSplit best;
    double least = 0;
    for (int tile : {256, 128}) {
        const int64_t tiles = ((outputs + tile - 1) / tile) * ((width + tile - 1) / tile);
        for (int count : kCounts) {
            if (count > 1 && count > steps) break;
            const int64_t each = (steps + count - 1) / count, parts = each > 0 ? (steps + each - 1) / each : 1, groups = tiles * parts;
            const double a_step = tile == 256 ? (f32 ? 2.5 : 1.8) : groups <= 256 ? (f32 ? 1.25 : 0.85) : (f32 ? 1.95 : 1.4);
            const int64_t slots = tile == 256 || groups <= 256 ? 256 : 512;
            double time = (tile == 256 ? 12.0 : 8.6) + static_cast<double>((groups + slots - 1) / slots) * static_cast<double>(each) * a_step;
            if (parts > 1) time += 5.0 + 0.02 * static_cast<double>(parts) + 0.9e-6 * static_cast<double>(parts) * static_cast<double>(outputs * width);
            if (best.tile == 0 || time < least) {
                least = time;
                best.tile = tile;
                best.parts = parts;
                best.steps = each;
            }
        }
    }
    if (best.parts > 1) {
        best.off_bias = align_up(static_cast<size_t>(best.parts) * outputs * width * 4, 256);
        best.total = best.off_bias + static_cast<size_t>(best.parts) * outputs * 4;
    }
    return best;
}

}  // namespace adasum
