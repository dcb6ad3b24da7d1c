// sample_bins.h - running sums over the bins of a row's histogram of weights, and which thread has a border in its bins.
// Host and device code; no CUDA types.
#pragma once

#include <math.h>
#include <stdint.h>

#ifdef __CUDACC__
#define RPD_BINS_HD __host__ __device__ __forceinline__
#else
#define RPD_BINS_HD inline
#endif

namespace rpd {

// Weights are added up in whole units of 2^-30 of the row's sum.  Sums of integers do not depend on the order of the additions:
// what is before a thread's bins is exactly what is behind those of the thread before it, whichever warp and CTA added it
// up, and running sums never fall.  So one thread of the row has a border, and one alone.  (With fp32 sums, each rounded in its own
// order, about one target in 10^6 lay between the two sides of a thread's border: two threads had it, or none.)  4096 bins'
// roundings are 2^-19 of the sum at most.
constexpr float kBinUnits = 0x1p30f;

RPD_BINS_HD uint32_t bin_units(float weight, float units) {
    return static_cast<uint32_t>(fminf(weight * units, 2.f * kBinUnits) + 0.5f);
}

// What a border is told by: the first bin up to whose end there are `least` tokens (by_count), or a sum of weights of `least` or
// more (`more`: of more than it).  Holds for every bin from the border's on: counts and units never fall, nor do their products with
// `unit`, the weight of one, as fp32 rounds them.
struct BinBorder {
    bool by_count, more;
    float least, unit;
    RPD_BINS_HD float weight(uint32_t units) const { return static_cast<float>(units) * unit; }
    RPD_BINS_HD bool holds(int count, uint32_t units) const {
        return by_count ? count >= static_cast<int>(least) : more ? weight(units) > least : weight(units) >= least;
    }
    // Whether it is in the bins of a thread, which has the row's first ones or follows `count0` tokens and `units0`.
    RPD_BINS_HD bool within(bool first, int count0, uint32_t units0, int count1, uint32_t units1) const {
        return (first || !holds(count0, units0)) && holds(count1, units1);
    }
};

}  // namespace rpd
