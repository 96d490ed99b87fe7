// What the forward and backward kernels of attention over bags share: their arguments, a bag's entries, an entry's score.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "common.h"
#include "relpos.h"

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
__device__ __forceinline__ BagSpan bag_span(const AttnArgs& a, int64_t first, int64_t end, int64_t used) {
    if (first < 0) first = 0;
    if (end > a.n) end = a.n;
    int64_t count = end > first ? end - first : 0;
    if (used < count) count = used > 0 ? used : 0;
    return {first, count};
}
__device__ __forceinline__ BagSpan bag_span(const AttnArgs& a, int64_t bag) {
    return bag_span(a, a.bag_off[bag], a.bag_off[bag + 1], a.bag_len ? a.bag_len[bag] : a.n);
}

// Bags are handed out in pieces of 1 << shift entries, numbered without a scan over the bags: numbers below `bags` are the bags'
// first pieces; the others of bag b begin at bags + (its offset >> shift), which leaves every bag room for all of its pieces (and
// some numbers without one).
inline int64_t piece_count(int64_t n, int64_t bags, int shift) { return (n >> shift) + bags; }
__device__ __forceinline__ uint32_t more_pieces(const AttnArgs& a, int shift, int64_t at) {
    if (at < 0) at = 0;
    if (at > a.n) at = a.n;
    return (uint32_t)(at >> shift);
}

struct BagPiece {
    uint32_t bag, number, of;         // piece `number` of the bag's `of` (at least 1); a number without a piece has number >= of
    uint32_t more;                    // the bag's pieces 1, 2, ... have the numbers more, more + 1, ...
    int64_t first;                    // its entries
    int count;
};
__device__ __forceinline__ BagPiece bag_piece(const AttnArgs& a, int shift, uint32_t bag, uint32_t number, const BagSpan& s, int64_t offset) {
    BagPiece p;
    const uint32_t at = more_pieces(a, shift, offset), extra = (uint32_t)(a.n >> shift);
    p.bag = bag;
    p.number = number;
    p.more = (uint32_t)a.bags + at;
    p.of = max(1u, min((uint32_t)((s.count + (1 << shift) - 1) >> shift), 1 + extra - at));
    p.first = s.first + ((int64_t)number << shift);
    p.count = number < p.of ? (int)min(int64_t(1) << shift, s.count - ((int64_t)number << shift)) : 0;
    return p;
}
// The piece with number `id`; behind the first pieces the bag is looked for, 64 bags a step by every wavefront.
__device__ __forceinline__ BagPiece find_piece(const AttnArgs& a, int shift, uint32_t id) {
    if (id < (uint32_t)a.bags) return bag_piece(a, shift, id, 0, bag_span(a, id), a.bag_off[id]);
    const uint32_t lane = threadIdx.x % 64, x = id - (uint32_t)a.bags;
    uint32_t lo = 0, hi = (uint32_t)a.bags;
    while (hi - lo > 1) {             // the last bag whose numbers begin no later
        const uint32_t step = (hi - lo + 63) / 64, i = lo + (lane + 1) * step;
        lo += __popcll(__ballot(i < hi && more_pieces(a, shift, a.bag_off[i]) <= x)) * step;
        hi = min(hi, lo + step);
    }
    return bag_piece(a, shift, lo, x - more_pieces(a, shift, a.bag_off[lo]) + 1, bag_span(a, lo), a.bag_off[lo]);
}

// exp of a difference: scores stay in natural units up to here, so that the lowest fp32 value, which masks give, does not become
// an infinity by a change of base.  The product with log2(e) is rounded once, so the result is off by up to |x| * 2^-24 of itself: for
// x = -16, where it is 1e-7, by 1e-6.
__device__ __forceinline__ float exp_few_ulp(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }
// exp(x) * 2^shift; the same bits as above for a shift of 0
__device__ __forceinline__ float exp_few_ulp(float x, float shift) { return __builtin_amdgcn_exp2f(fmaf(x, 1.4426950408889634f, shift)); }

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
