// What the forward and backward kernels of attention over bags share: their arguments, a bag's entries, an entry's score.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "common.h"
#include "relpos.h"
#include "row_access.h"

namespace bp {

struct AttnArgs {
    Relpos rp;
    const void* cache_w;
    const int32_t* slots;
    const int64_t* bag_off;
    const int32_t* bag_len;
    const float* q;
    const int32_t* q_pos;
    const int32_t* lookup_pos;
    const float* bias;             // NULL: no bias, and every entry of the bag is seen
    int64_t n, bags, C;
    int64_t wst;                   // elements from one cache row to the next
    int32_t q_heads, kv_heads, d, value_at, dim;
    float scale, cap;
};

int attn_check(const bp_config* cfg, const bp_attn* at, const bp_relpos* rp, const void* cache_w, const int32_t* lookup_slots,
               const int64_t* bag_offsets, const int32_t* bag_lengths, int64_t n_lookups, int64_t bags, const float* q,
               const int32_t* q_pos, const int32_t* lookup_pos, const float* bias_table, AttnArgs* out);
int attn_check_shape(const bp_config* cfg, const bp_attn* at);

// The entries [first, first + count) that a bag uses; offsets and lengths that point outside the lookups use nothing there.
struct BagSpan {
    int64_t first, count;
};
__device__ __forceinline__ BagSpan bag_span(const AttnArgs& a, int64_t bag) {
    int64_t first = a.bag_off[bag], end = a.bag_off[bag + 1];
    if (first < 0) first = 0;
    if (end > a.n) end = a.n;
    int64_t count = end > first ? end - first : 0;
    if (a.bag_len) {
        const int64_t used = a.bag_len[bag];
        if (used < count) count = used > 0 ? used : 0;
    }
    return {first, count};
}

__device__ __forceinline__ float row_value(const float* row, int64_t i) { return row[i]; }
__device__ __forceinline__ float row_value(const uint16_t* row, int64_t i) { return bf16_bits_to_f32(row[i]); }

}  // namespace bp
