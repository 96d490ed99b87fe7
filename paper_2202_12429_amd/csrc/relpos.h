// Buckets of distances, shared by the bias kernels and by attention over bags.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "common.h"

namespace bp {

// A bp_relpos as a kernel argument: the borders by value, so that no call depends on host memory after it returns.
struct Relpos {
    int32_t buckets = 1, two_sided = 1;
    int32_t borders[BP_RELPOS_MAX_BUCKETS] = {};        // buckets - 1 of them, then values no distance reaches
    __host__ __device__ int rows() const { return buckets * (two_sided ? 2 : 1); }
};

int check_relpos(const bp_relpos* rp, Relpos* out);

// The table row of a distance: a binary search over the borders (in LDS, BP_RELPOS_MAX_BUCKETS values, the unused ones above
// every distance), which wavefronts whose distances all lie behind the last border need not make.  -1: not seen.  Distances are
// differences of int32 positions and may need 33 bits.
__device__ __forceinline__ int relpos_row(int64_t distance, const int32_t* borders, int buckets, int two_sided) {
    const bool later = distance < 0;
    const int64_t away = later ? -distance : distance;
    const int32_t n = away > 0x7ffffffe ? 0x7ffffffe : (int32_t)away;
    int at = buckets - 1;
    if (buckets > 1 && __any(n < borders[buckets - 2])) {
        at = 0;
#pragma unroll
        for (int step = BP_RELPOS_MAX_BUCKETS / 2; step >= 1; step >>= 1)
            if (borders[at + step - 1] <= n) at += step;
    }
    return !later ? at : two_sided ? at + buckets : -1;
}

}  // namespace bp
