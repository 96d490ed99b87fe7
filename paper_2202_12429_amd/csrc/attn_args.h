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

int attn_check_workspace(const void* workspace, size_t have, size_t need);
int attn_check_sizes(int64_t n, int64_t bags, size_t* bytes);

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

// Bags are handed out in pieces of 1 << shift entries.  Piece numbers need no scan over the bags: bag b's begin at
// (its offset >> shift) + b, which leaves every bag room for all its pieces (and some numbers without one).
__device__ __forceinline__ uint32_t first_piece(const AttnArgs& a, int shift, uint32_t bag) {
    int64_t at = a.bag_off[bag];
    if (at < 0) at = 0;
    if (at > a.n) at = a.n;
    return (uint32_t)(at >> shift) + bag;
}
inline int64_t piece_count(int64_t n, int64_t bags, int shift) { return (n >> shift) + bags; }

struct BagPiece {
    uint32_t bag, number, of;         // piece `number` of the bag's `of` (0 for an empty bag, which has the piece 0 all the same)
    uint32_t first_id;                // the number of the bag's first piece among all
    int64_t first;                    // its entries
    int count;
};
// The piece with number `id` among `all`: the last bag that begins no later, found 64 bags a step by every wavefront.
__device__ __forceinline__ BagPiece find_piece(const AttnArgs& a, int shift, uint32_t id, uint32_t all) {
    const uint32_t lane = threadIdx.x % 64;
    uint32_t lo = 0, hi = (uint32_t)a.bags;
    while (hi - lo > 1) {
        const uint32_t step = (hi - lo + 63) / 64, i = lo + (lane + 1) * step;
        const bool starts = i < hi && first_piece(a, shift, i) <= id;
        lo += __popcll(__ballot(starts)) * step;
        hi = min(hi, lo + step);
    }
    const BagSpan s = bag_span(a, lo);
    BagPiece p;
    p.bag = lo;
    p.first_id = first_piece(a, shift, lo);
    p.number = id - p.first_id;
    p.of = min((uint32_t)((s.count + (1 << shift) - 1) >> shift), all - min(all, p.first_id));
    p.first = s.first + ((int64_t)p.number << shift);
    p.count = p.number < p.of ? (int)min(int64_t(1) << shift, s.count - ((int64_t)p.number << shift)) : 0;
    return p;
}

// exp of a difference: scores stay in natural units up to here, so that the lowest fp32 value, which masks give, does not become
// an infinity by a change of base.
__device__ __forceinline__ float exp_few_ulp(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// tanh to a few units of the last place: the series up to x^13 where 1 - 2 / (e^2x + 1) cancels.
__device__ __forceinline__ float tanh_few_ulp(float x) {
    const float y = x * x;
    float s = 21844.f / 6081075.f;
    s = fmaf(s, y, -1382.f / 155925.f);
    s = fmaf(s, y, 62.f / 2835.f);
    s = fmaf(s, y, -17.f / 315.f);
    s = fmaf(s, y, 2.f / 15.f);
    s = fmaf(s, y, -1.f / 3.f);
    const float e = __builtin_amdgcn_exp2f(x * 2.8853900817779268f);
    const float far = fmaf(-2.f, __builtin_amdgcn_rcpf(e + 1.f), 1.f);
    return fabsf(x) < 0.4f ? fmaf(x * y, s, x) : far;
}

}  // namespace bp
