// bp_evict_by_weight: lists over their budget lose the entries of the lowest accumulated weight.
#include <algorithm>

#include "common.h"

namespace bp {
namespace {

constexpr int kEvictBlock = 256;
constexpr int64_t kMaxLists = int64_t(1) << 24;

struct EvictArgs {
    const int64_t* bag_off;
    const int32_t* bag_len;
    int64_t n, bags;
    int32_t budget, sinks, recent;
    const float* weight;
    const int64_t* ids;
    const int32_t *slots, *pos;
    float* kept_weight;
    int64_t* kept_ids;
    int32_t *kept_slots, *kept_pos, *kept_len;
    int64_t* evict_ids;
    int32_t* evict_slots;
    int64_t list_capacity;
    int64_t* evict_off;
};

// The entries [first, first + count) of a list; offsets and lengths that point outside the arrays use nothing there.
__device__ __forceinline__ void list_span(const EvictArgs& a, int64_t bag, int64_t* first, int64_t* count) {
    int64_t f = a.bag_off[bag], e = a.bag_off[bag + 1];
    if (f < 0) f = 0;
    if (e > a.n) e = a.n;
    int64_t c = e > f ? e - f : 0;
    if (a.bag_len) {
        const int64_t used = a.bag_len[bag];
        if (used < c) c = used > 0 ? used : 0;
    }
    *first = f;
    *count = c;
}

// Weights as unsigned keys of the same order: -0 as 0, NaN above everything.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0xffffffffu;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int64_t block_sum(int64_t v, int64_t* scratch) {
    __syncthreads();
    scratch[threadIdx.x] = v;
    __syncthreads();
    for (int off = kEvictBlock / 2; off >= 1; off >>= 1) {
        if ((int)threadIdx.x < off) scratch[threadIdx.x] += scratch[threadIdx.x + off];
        __syncthreads();
    }
    const int64_t r = scratch[0];
    __syncthreads();
    return r;
}

// A workgroup a list.  The weight up to which entries leave is found eight bits at a time by counting; of the entries that have
// exactly that weight the earliest leave.
__global__ __launch_bounds__(kEvictBlock) void evict_kernel(EvictArgs a) {
    __shared__ int64_t scratch[kEvictBlock];
    __shared__ uint32_t hist[256];
    __shared__ uint32_t found, rest;
    __shared__ uint32_t scan[2][kEvictBlock];
    const int64_t bag = blockIdx.x;
    int64_t before = 0;
    for (int64_t b = threadIdx.x; b < bag; b += kEvictBlock) {
        int64_t f, c;
        list_span(a, b, &f, &c);
        before += max(int64_t(0), c - a.budget);
    }
    before = block_sum(before, scratch);
    int64_t first = 0, count = 0;
    if (bag < a.bags) list_span(a, bag, &first, &count);
    const int64_t over = max(int64_t(0), count - a.budget);
    if (threadIdx.x == 0) {
        if (bag < a.bags) a.kept_len[bag] = (int32_t)(count - over);
        a.evict_off[bag] = before;
        if (bag == a.bags - 1) a.evict_off[a.bags] = before + over;
    }
    if (bag >= a.bags - 1)                                  // the last list, or none at all
        for (int64_t e = before + over + threadIdx.x; e < a.list_capacity; e += kEvictBlock) {
            if (a.evict_ids) a.evict_ids[e] = -1;
            a.evict_slots[e] = -1;
        }
    const int64_t may0 = a.sinks, may1 = count - a.recent;
    uint32_t prefix = 0, need = (uint32_t)over;            // the need-th smallest key that starts with the bits found so far
    if (over) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            hist[threadIdx.x] = 0;
            __syncthreads();
            for (int64_t e = may0 + threadIdx.x; e < may1; e += kEvictBlock) {
                const uint32_t key = weight_key(a.weight[first + e]);
                if (shift == 24 || key >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&hist[key >> shift & 255], 1u);
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                uint32_t left = need, d = 0;
                while (left > hist[d]) left -= hist[d++];
                found = d;
                rest = left;
            }
            __syncthreads();
            prefix |= found << shift;
            need = rest;
            __syncthreads();
        }
    }
    // the kept entries and the others, each in order
    int64_t kept = 0, gone = 0, ties = 0;
    for (int64_t e0 = 0; e0 < count; e0 += kEvictBlock) {
        const int64_t e = e0 + threadIdx.x;
        const bool may = over && e >= may0 && e < may1;
        const float w = e < count ? a.weight[first + e] : 0.f;
        const uint32_t key = weight_key(w);
        const bool tie = may && key == prefix;
        int cur = 0;
        uint32_t all[2];
        for (int round = 0; round < 2; ++round) {          // first the ties are numbered, then what leaves
            const bool leaves = may && (key < prefix || (tie && round && (uint64_t)ties + all[0] < need));
            scan[cur][threadIdx.x] = round ? leaves : tie;
            __syncthreads();
            for (int off = 1; off < kEvictBlock; off <<= 1) {
                scan[cur ^ 1][threadIdx.x] = scan[cur][threadIdx.x] + ((int)threadIdx.x >= off ? scan[cur][threadIdx.x - off] : 0);
                cur ^= 1;
                __syncthreads();
            }
            const uint32_t incl = scan[cur][threadIdx.x], total = scan[cur][kEvictBlock - 1];
            if (round == 0) {
                all[0] = incl - tie;
                all[1] = total;
                __syncthreads();
                continue;
            }
            const int64_t in_tile = min((int64_t)kEvictBlock, count - e0);
            if (e < count) {
                const int64_t from = first + e;
                if (leaves) {
                    const int64_t to = before + gone + incl - 1;
                    if (to < a.list_capacity) {
                        if (a.evict_ids) a.evict_ids[to] = a.ids[from];
                        a.evict_slots[to] = a.slots[from];
                    }
                } else {
                    const int64_t to = first + kept + threadIdx.x - incl;
                    if (a.kept_weight) a.kept_weight[to] = w;
                    if (a.kept_ids) a.kept_ids[to] = a.ids[from];
                    a.kept_slots[to] = a.slots[from];
                    if (a.kept_pos) a.kept_pos[to] = a.pos[from];
                }
            }
            gone += total;
            kept += in_tile - total;
            ties += all[1];
            __syncthreads();
        }
    }
}

}  // namespace
}  // namespace bp

using namespace bp;

BP_EXPORT int bp_evict_by_weight_workspace_bytes(int64_t n, int64_t bags, size_t* bytes) {
    if (!bytes) return fail(BP_ERR_INVALID_ARG, "bytes is NULL");
    if (n < 0 || bags < 0) return fail(BP_ERR_INVALID_ARG, "negative size");
    if (n >= (int64_t(1) << 31) || bags >= kMaxLists) return fail(BP_ERR_UNSUPPORTED, "n >= 2^31 or bags >= 2^24");
    *bytes = 0;
    return BP_OK;
}

BP_EXPORT int bp_evict_by_weight(const int64_t* bag_offsets, const int32_t* bag_lengths, int64_t n, int64_t bags, int32_t budget, int32_t sinks,
                                 int32_t recent, const float* weight, const int64_t* ids, const int32_t* slots, const int32_t* pos,
                                 float* kept_weight, int64_t* kept_ids, int32_t* kept_slots, int32_t* kept_pos, int32_t* kept_lengths,
                                 int64_t* evict_ids, int32_t* evict_slots, int64_t list_capacity, int64_t* evict_offsets, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    size_t need = 0;
    BP_TRY(bp_evict_by_weight_workspace_bytes(n, bags, &need));
    if (budget < 1 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget)
        return fail(BP_ERR_INVALID_ARG, "budget %d, sinks %d, recent %d: at least 1, 0 and 0, sinks + recent <= budget", budget, sinks, recent);
    if (list_capacity < 0) return fail(BP_ERR_INVALID_ARG, "negative list_capacity");
    if (!evict_offsets || (bags && (!bag_offsets || !kept_lengths))) return fail(BP_ERR_INVALID_ARG, "NULL pointer");
    if (n && bags && (!weight || !slots || !kept_slots)) return fail(BP_ERR_INVALID_ARG, "NULL pointer");
    if (n && ((ids != nullptr) != (kept_ids != nullptr) || (pos != nullptr) != (kept_pos != nullptr)))
        return fail(BP_ERR_INVALID_ARG, "kept_ids goes with ids, kept_pos with pos");
    if (list_capacity && (!evict_slots || (n && (ids != nullptr) != (evict_ids != nullptr))))
        return fail(BP_ERR_INVALID_ARG, "evict_slots is NULL, or only one of ids and evict_ids is given");
    if ((((uintptr_t)bag_offsets | (uintptr_t)ids | (uintptr_t)kept_ids | (uintptr_t)evict_ids | (uintptr_t)evict_offsets) & 7) ||
        (((uintptr_t)bag_lengths | (uintptr_t)weight | (uintptr_t)slots | (uintptr_t)pos | (uintptr_t)kept_weight | (uintptr_t)kept_slots |
          (uintptr_t)kept_pos | (uintptr_t)kept_lengths | (uintptr_t)evict_slots) & 3))
        return fail(BP_ERR_INVALID_ARG, "an array is not aligned to its elements");
    const void* const from[4] = {weight, ids, slots, pos};
    const void* const to[4] = {kept_weight, kept_ids, kept_slots, kept_pos};
    const size_t wide[4] = {4, 8, 4, 4};
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j)
            if (from[i] && to[j] && (uintptr_t)from[i] < (uintptr_t)to[j] + n * wide[j] && (uintptr_t)to[j] < (uintptr_t)from[i] + n * wide[i])
                return fail(BP_ERR_INVALID_ARG, "the kept arrays overlap the input arrays");
    if (bags && kept_lengths == bag_lengths) return fail(BP_ERR_INVALID_ARG, "kept_lengths is bag_lengths");
    const EvictArgs a{bag_offsets, bag_lengths, n, bags, budget, sinks, recent, weight, ids, slots, pos, kept_weight, kept_ids, kept_slots,
                      kept_pos, kept_lengths, evict_ids, evict_slots, list_capacity, evict_offsets};
    BP_LAUNCH(K_EVICT_SELECT, evict_kernel, dim3((unsigned)std::max<int64_t>(bags, 1)), dim3(kEvictBlock), 0, (hipStream_t)stream, a);
    return BP_OK;
}
