// Dropout's mask, never stored: element j of row t is kept by a 16-bit number that both passes compute from a seed, a step and its place.
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers, as easy as 1, 2, 3; 2011): ten rounds of two 32 x 32-bit products turn
// a counter of 128 bits and a key of 64 into four words.  A counter stands for eight channels of a row, a half of a word for each: the
// rounds' products are quarter-rate instructions, and a word for each channel would take longer than a stream of 16-bit elements.
#pragma once

#include "adasum_rows.h"

namespace adasum {
namespace {

struct Mask {
    unsigned k0, k1;                   // the seed
    bool drops;                        // else everything is kept
    unsigned below;                    // kept: numbers above it (65535: none)
    float factor;                      // of what is kept
    const unsigned* step;              // 64 bits on the device, or null (0)
};
inline Mask make_mask(double p, unsigned long long seed, const void* step) {
    Mask m;
    m.k0 = static_cast<unsigned>(seed);
    m.k1 = static_cast<unsigned>(seed >> 32);
    const unsigned limit = static_cast<unsigned>(65536.0 * p + 0.5);
    m.drops = limit != 0;
    m.below = m.drops ? limit - 1 : 0;
    m.factor = limit == 65536 ? 0.f : static_cast<float>(65536.0 / (65536.0 - limit));
    m.step = static_cast<const unsigned*>(step);
    return m;
}
struct Step {
    unsigned lo = 0, hi = 0;
};
__device__ __forceinline__ Step step_of(const Mask& m) {
    Step s;
    if (m.step != nullptr) {
        s.lo = m.step[0];
        s.hi = m.step[1];
    }
    return s;
}

// The eight numbers of channels 8 * granule .. 8 * granule + 7 of a row, two a word.
__device__ __forceinline__ void mask_words(unsigned (&w)[4], const Mask& m, Step step, unsigned granule, unsigned row) {
    unsigned c0 = granule, c1 = row, c2 = step.lo, c3 = step.hi, k0 = m.k0, k1 = m.k1;
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const unsigned long long a = static_cast<unsigned long long>(c0) * 0xd2511f53u, b = static_cast<unsigned long long>(c2) * 0xcd9e8d57u;
        c0 = static_cast<unsigned>(b >> 32) ^ c1 ^ k0;
        c1 = static_cast<unsigned>(b);
        c2 = static_cast<unsigned>(a >> 32) ^ c3 ^ k1;
        c3 = static_cast<unsigned>(a);
        k0 += 0x9e3779b9u;
        k1 += 0xbb67ae85u;
    }
    w[0] = c0;
    w[1] = c1;
    w[2] = c2;
    w[3] = c3;
}
// (one comparison each: of the lower half by itself, of the upper one with what is below it in tow)
__device__ __forceinline__ void kept(bool (&keep)[kG], const unsigned (&w)[4], unsigned below) {
    const unsigned short half = static_cast<unsigned short>(below);
    const unsigned top = below << 16 | 0xffffu;
#pragma unroll
    for (int i = 0; i < kG; ++i) keep[i] = i & 1 ? w[i / 2] > top : static_cast<unsigned short>(w[i / 2]) > half;
}
// (a choice and no product: what is dropped is 0 also where it was no number)
__device__ __forceinline__ void drop(float (&v)[kG], const bool (&keep)[kG], float factor) {
#pragma unroll
    for (int i = 0; i < kG; ++i) v[i] = keep[i] ? v[i] * factor : 0.f;
}

}  // namespace
}  // namespace adasum
