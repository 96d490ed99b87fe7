// bp_embbag_attn_fwd: bags pooled by attention over their cached rows.
//
// One pass over a bag's rows with the running maximum and sum of a softmax, both fp32.  Four layouts, chosen by sizes (FwdPlan): a
// workgroup a piece of up to 512 entries of a bag; short bags a wavefront a piece; the same without the matrix instructions where a key has
// one query; and few long bags shared evenly over the chip.  The parts of a bag of several meet in a second launch.  Weights, if asked
// for, are made of the scores, which are kept: by the workgroup itself where it has all heads of a whole bag, else by a launch of their own.
#include <algorithm>
#include <cmath>

#include "attn_tile.h"

namespace bp {

int attn_check_shape(const bp_config* cfg, const bp_attn* at) {
    BP_TRY(check_config(cfg));
    if (!at) return fail(BP_ERR_INVALID_ARG, "at is NULL");
    if (at->kv_heads < 1 || at->kv_heads > 64) return fail(BP_ERR_INVALID_ARG, "kv_heads %d outside [1, 64]", at->kv_heads);
    if (at->q_heads < 1 || at->q_heads % at->kv_heads != 0 || at->q_heads / at->kv_heads > 16)
        return fail(BP_ERR_INVALID_ARG, "q_heads %d: a multiple of kv_heads %d, at most 16 times as many", at->q_heads, at->kv_heads);
    if (at->head_dim < 8 || at->head_dim > 256 || at->head_dim % 8 != 0)
        return fail(BP_ERR_INVALID_ARG, "head_dim %d: a multiple of 8 in [8, 256]", at->head_dim);
    const int64_t span = (int64_t)at->kv_heads * at->head_dim;
    if (at->value_offset != 0 && (at->value_offset < span || at->value_offset % 8 != 0))
        return fail(BP_ERR_INVALID_ARG, "value_offset %d: 0, or a multiple of 8 that is at least %lld", at->value_offset, (long long)span);
    if (at->value_offset + span > cfg->dim)
        return fail(BP_ERR_INVALID_ARG, "keys and values end at element %lld of rows of %d", (long long)(at->value_offset + span), cfg->dim);
    if (!std::isfinite(at->scale)) return fail(BP_ERR_INVALID_ARG, "scale is not finite");
    if (!std::isfinite(at->cap) || at->cap < 0) return fail(BP_ERR_INVALID_ARG, "cap is negative or not finite");
    // the kernels multiply by it: a score of 0 would be NaN
    if (at->cap > 0 && !std::isfinite(at->scale / at->cap)) return fail(BP_ERR_INVALID_ARG, "scale / cap is not finite");
    return BP_OK;
}

int attn_check(const bp_config* cfg, const bp_attn* at, const bp_relpos* rp, const void* cache_w, const int32_t* lookup_slots,
               const int64_t* bag_offsets, const int32_t* bag_lengths, int64_t n_lookups, int64_t bags, const float* q,
               const int32_t* q_pos, const int32_t* lookup_pos, const float* bias_table, AttnArgs* out) {
    BP_TRY(attn_check_shape(cfg, at));
    if (bags < 0 || n_lookups < 0) return fail(BP_ERR_INVALID_ARG, "negative size");
    if (bags >= (int64_t(1) << 31) || n_lookups >= (int64_t(1) << 31)) return fail(BP_ERR_UNSUPPORTED, "size >= 2^31");
    AttnArgs a{};
    if (rp) {
        BP_TRY(check_relpos(rp, &a.rp));
        if (bags && (!q_pos || !bias_table || (n_lookups && !lookup_pos)))
            return fail(BP_ERR_INVALID_ARG, "rp is given without q_pos, lookup_pos and bias_table");
    } else if (q_pos || lookup_pos || bias_table) {
        return fail(BP_ERR_INVALID_ARG, "q_pos, lookup_pos and bias_table go with rp");
    }
    if (bags && (!cache_w || !bag_offsets || !q || (n_lookups && !lookup_slots))) return fail(BP_ERR_INVALID_ARG, "NULL pointer");
    if (((uintptr_t)cache_w | (uintptr_t)q | (uintptr_t)bias_table) & 15)
        return fail(BP_ERR_INVALID_ARG, "cache_w, q and bias_table must be 16-byte aligned");
    if (((uintptr_t)bag_offsets & 7) || (((uintptr_t)lookup_slots | (uintptr_t)bag_lengths | (uintptr_t)q_pos | (uintptr_t)lookup_pos) & 3))
        return fail(BP_ERR_INVALID_ARG, "an array is not aligned to its elements");
    a.cache_w = cache_w;
    a.slots = lookup_slots;
    a.bag_off = bag_offsets;
    a.bag_len = bag_lengths;
    a.q = q;
    a.q_pos = q_pos;
    a.lookup_pos = lookup_pos;
    a.bias = bias_table;
    a.n = n_lookups;
    a.bags = bags;
    a.C = cfg->capacity;
    a.wst = cache_w_stride16(cfg) * (16 / (int64_t)elem_bytes(cfg->weight_dtype));
    a.q_heads = at->q_heads;
    a.kv_heads = at->kv_heads;
    a.d = at->head_dim;
    a.value_at = at->value_offset;
    a.dim = cfg->dim;
    a.scale = at->scale;
    a.cap = at->cap;
    *out = a;
    return BP_OK;
}

int attn_check_workspace(const void* workspace, size_t have, size_t need) {
    if (need && (!workspace || ((uintptr_t)workspace & 255))) return fail(BP_ERR_INVALID_ARG, "workspace NULL or not 256-byte aligned");
    if (have < need) return fail(BP_ERR_WORKSPACE_TOO_SMALL, "workspace %zu < required %zu bytes", have, need);
    return BP_OK;
}
int attn_check_sizes(int64_t n, int64_t bags, size_t* bytes) {
    if (!bytes) return fail(BP_ERR_INVALID_ARG, "bytes is NULL");
    if (bags < 0 || n < 0) return fail(BP_ERR_INVALID_ARG, "negative size");
    if (bags >= (int64_t(1) << 31) || n >= (int64_t(1) << 31)) return fail(BP_ERR_UNSUPPORTED, "size >= 2^31");
    return BP_OK;
}


namespace {

struct FwdArgs {
    AttnArgs a;
    int32_t shift;              // log2 of a piece's entries
    uint32_t pieces;
    uint32_t groups;            // workgroups that share all entries evenly; 0: a workgroup a piece
    uint32_t* blocks;           // [bags + 1] running count of the bags' blocks, written by the first of these workgroups
    int32_t weighed;            // bags of one piece have their weights from the first launch
    float* scores;              // [q_heads][score_stride]; NULL when no weights are asked for
    int64_t score_stride;
    float2* norms;              // [bags][q_heads], with the scores: the maximum and one over the sum, 0 where nothing is seen
    float* part_ml;             // [parts][q_heads][2]: maximum and sum of a part of a bag
    float* part_o;              // [parts][q_heads][d]: its weighted values, not divided by the sum
    float* out;
    float* lse;
    const float* weight_in;
    float* weight_out;
};

// weight_out of a piece's entries, a thread each, from the scores and the bag's norms: not from lse, which no longer holds the sum where
// scores are large (a mask of low values over a whole bag).  A bag without a norm (nothing seen) has scores of -infinity alone.
template <int BLOCK>
__device__ __forceinline__ void add_weights(const FwdArgs& f, uint32_t bag, int64_t first, int count) {
    constexpr int AHEAD = BLOCK == 64 ? 1 : 8;                       // heads whose loads are in flight: wavefronts by themselves have no registers for more
    const float2* const norms = f.norms + (int64_t)bag * f.a.q_heads;
    for (int i = threadIdx.x % BLOCK; i < count; i += BLOCK) {
        const int64_t k = first + i;
        float add = 0.f;
#pragma unroll AHEAD
        for (int h = 0; h < f.a.q_heads; ++h) {
            const float c = f.scores[h * f.score_stride + k];
            const float2 norm = norms[h];
            add += c == -INFINITY ? 0.f : exp_few_ulp(c - norm.x) * norm.y;
        }
        f.weight_out[k] = (f.weight_in ? f.weight_in[k] : 0.f) + add;
    }
}

// LDS of a workgroup, in this order: borders, every wavefront's slots and table rows of a tile, its maxima and sums, the bias
// table's columns of the workgroup's heads, and (over the table, once it is done with) the wavefronts' weighted values.
template <int WAVES>
struct AttnLds {
    static constexpr int BORDERS = 0, TILE = BP_RELPOS_MAX_BUCKETS, ML = TILE + WAVES * 128, FREE = ML + WAVES * 32;
    static size_t bytes(int flat, int table_floats) { return (size_t)(FREE + std::max(table_floats, WAVES * (flat / 4) * 64)) * 4; }
};

// Entries [first, first + count) of a bag: all that it uses, or the part with this number.
struct Segment {
    uint32_t bag, part;
    int64_t first;
    int count;
    bool whole;
};

// The borders, and the bias table's columns of the workgroup's heads.
template <int WAVES>
__device__ __forceinline__ void read_table(const AttnArgs& a, float* lds, int first_head, int cols) {
    if (!a.bias) return;
    float* const table = lds + AttnLds<WAVES>::FREE;
    if (threadIdx.x < BP_RELPOS_MAX_BUCKETS) ((int32_t*)lds)[AttnLds<WAVES>::BORDERS + threadIdx.x] = a.rp.borders[threadIdx.x];
    if (cols == a.q_heads)
        for (int e = threadIdx.x; e < a.rp.rows() * cols; e += WAVES * 64) table[e] = a.bias[e];
    else
        for (int e = threadIdx.x; e < a.rp.rows() * cols; e += WAVES * 64) table[e] = a.bias[(e / cols) * a.q_heads + first_head + e % cols];
}

// What the first tile of a wavefront's next segment begins with, on its way during the one before.
struct Ahead {
    int32_t slot, pos;
    int64_t q_pos;
};

// One segment: the workgroup's wavefronts take its tiles in turn, or (ALONE) each has a segment of its own.
constexpr int kFwdWaves = 4, kFwdBlock = kFwdWaves * 64;
template <typename T, int DP, int PACK, bool FULL, bool ALONE>
__device__ __forceinline__ void attend(const FwdArgs& f, const Segment& p, float* lds, const Ahead& ahead = Ahead{}) {
    typedef AttnLds<kFwdWaves> L;
    constexpr int kLdsBorders = L::BORDERS, kLdsTile = L::TILE, kLdsMl = L::ML, kLdsFree = L::FREE;
    typedef AttnTile<T, DP, PACK> X;
    typedef typename Bytes<X::VW * sizeof(T)>::type VRaw;
    const AttnArgs& a = f.a;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, g = lane / 16;
    const int group = a.q_heads / a.kv_heads, kv0 = blockIdx.y * PACK, heads = FULL ? PACK : min(PACK, a.kv_heads - kv0), d = FULL ? DP : a.d;
    constexpr int stripes = ALONE ? 1 : kFwdWaves;
    const int stripe = ALONE ? 0 : wave, first_head = kv0 * group, cols = heads * group, table_cols = cols, flat = heads * d;
    const int head = first_head + min(col, cols - 1), own = min(col, cols - 1) / group;        // the column's query head, its kv head

    int32_t* const borders = (int32_t*)lds + kLdsBorders;
    int32_t* const tiles_of = (int32_t*)lds + kLdsTile + wave * 128;          // two tiles: slots, table offsets
    float* const table = lds + kLdsFree;

    // entry `lane` of a tile: its slot and position, fetched ahead
    const int tiles = (p.count + X::ROWS - 1) / X::ROWS;
    int32_t slot_n = -1, pos_n = 0;
    const auto fetch = [&](int t) {
        const int e = t * X::ROWS + lane;
        const bool have = lane < X::ROWS && e < p.count;
        slot_n = have ? a.slots[p.first + e] : -1;
        pos_n = have && a.bias ? a.lookup_pos[p.first + e] : 0;
    };
    if (ALONE) slot_n = ahead.slot, pos_n = ahead.pos;
    else fetch(stripe);
    const int64_t q_pos = ALONE ? ahead.q_pos : a.bias ? a.q_pos[p.bag] : 0;
    if (!ALONE) read_table<kFwdWaves>(a, lds, first_head, cols);

    // the queries: lane col has the column's
    const float* const q = a.q + ((int64_t)p.bag * a.q_heads + head) * d;
    std::conditional_t<X::BF16, Split3, f32x4> qf[X::KM];
#pragma unroll
    for (int m = 0; m < X::KM; ++m) {
        const int at = m * X::KC + g * (X::KC / 4);
        const bool have = col < cols && at < d;
        if constexpr (X::BF16) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 t = or_zeros(*reinterpret_cast<const float4*>(q + (FULL || at < d ? at : 0) + 4 * i), have);
                v[4 * i] = t.x, v[4 * i + 1] = t.y, v[4 * i + 2] = t.z, v[4 * i + 3] = t.w;
            }
            qf[m].set(v);
        } else {
            const float4 t = or_zeros(*reinterpret_cast<const float4*>(q + (FULL || at < d ? at : 0)), have);
            qf[m] = f32x4{t.x, t.y, t.z, t.w};
        }
    }
    if (!ALONE && a.bias) __syncthreads();

    f32x4 o[X::MB][X::VW];
#pragma unroll
    for (int m = 0; m < X::MB; ++m)
#pragma unroll
        for (int j = 0; j < X::VW; ++j) o[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float top = -INFINITY, sum = 0.f;             // of the lane's query head; the sum over the lane's own entries
    const T* const w = (const T*)a.cache_w + (int64_t)kv0 * d;

    // What a tile takes, a step ahead of its use: slots and table offsets into LDS, keys as soon as the tile before has its scores,
    // values as soon as it has pooled, so that one or the other is always on its way, in the registers that it falls free of.
    bool all_seen_n = true;
    const auto place = [&](int t) {               // what fetch() brought, for tile t
        int row_of = -1;
        if ((uint32_t)slot_n < (uint64_t)a.C) row_of = a.bias ? relpos_row(q_pos - pos_n, borders, a.rp.buckets, a.rp.two_sided) : 0;
        all_seen_n = __ballot(row_of >= 0 || lane >= X::ROWS) == ~0ull;
        int32_t* const tile = tiles_of + (t / stripes & 1) * 64;
        __builtin_amdgcn_wave_barrier();
        if (lane < X::ROWS) {
            tile[lane] = row_of >= 0 ? slot_n : 0;                    // what is not seen reads row 0, and leaves it out
            tile[32 + lane] = row_of >= 0 ? row_of * table_cols : -1;
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    // row `col` of S tile u is entry PER * (col / 4) + 4u + col % 4, so that lane (col, g)'s scores are of the entries PER * g ...
    uint4 kraw[PACK][X::NU][X::KM];
    const auto load_keys = [&](int t) {
        const int32_t* const tile = tiles_of + (t / stripes & 1) * 64;
#pragma unroll
        for (int u = 0; u < X::NU; ++u) {
            const T* const row = w + (int64_t)tile[X::PER * (col / 4) + 4 * u + col % 4] * a.wst;
#pragma unroll
            for (int k = 0; k < PACK; ++k)
#pragma unroll
                for (int m = 0; m < X::KM; ++m) {
                    const int at = m * X::KC + g * (X::KC / 4);
                    kraw[k][u][m] = row_bytes_at<FULL>(row + (FULL ? k : min(k, heads - 1)) * d, at, d);      // (a head that is not there is nobody's)
                }
        }
    };
    VRaw vraw[X::PER][X::MB];
    const auto load_values = [&](int t) {
        const int32_t* const tile = tiles_of + (t / stripes & 1) * 64;
#pragma unroll
        for (int e = 0; e < X::PER; ++e) {
            const T* const row = w + (int64_t)tile[X::PER * g + e] * a.wst + a.value_at;
#pragma unroll
            for (int m = 0; m < X::MB; ++m) {
                const int at = m * 16 * X::VW + col * X::VW;
                vraw[e][m] = *reinterpret_cast<const VRaw*>(row + (FULL || at < flat ? at : 0));
            }
        }
    };
    const float by_cap = a.cap > 0 ? a.scale / a.cap : 0.f;
    const float* const column = table + min(col, cols - 1);
    if (stripe < tiles) {
        place(stripe);
        load_keys(stripe);
        load_values(stripe);
        fetch(stripe + stripes);
    }
    for (int t = stripe; t < tiles; t += stripes) {
        const bool all_seen = all_seen_n, more = t + stripes < tiles;
        const int32_t* const tile = tiles_of + (t / stripes & 1) * 64;
        if (more) {
            place(t + stripes);
            fetch(t + 2 * stripes);
        }
        float z[X::PER];
#pragma unroll
        for (int u = 0; u < X::NU; ++u) {
#pragma unroll
            for (int k = 0; k < PACK; ++k) {
                f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int m = 0; m < X::KM; ++m) {
                    if constexpr (X::BF16) {
                        const bf16x8 key = __builtin_bit_cast(bf16x8, kraw[k][u][m]);
#pragma unroll
                        for (int part = 2; part >= 0; --part) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, qf[m].part[part], s, 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(word(kraw[k][u][m], e)), qf[m][e], s, 0, 0, 0);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) z[4 * u + i] = k == 0 || own == k ? s[i] : z[4 * u + i];
            }
        }
        if (more) load_keys(t + stripes);
        int32_t row_t[X::PER];
#pragma unroll
        for (int e = 0; e < X::PER; ++e) row_t[e] = tile[32 + X::PER * g + e];
        float most = -INFINITY;
        if (a.cap > 0) {                          // (tests of what the call has stay outside the loops over entries)
#pragma unroll
            for (int e = 0; e < X::PER; ++e) z[e] = a.cap * tanh_few_ulp(z[e] * by_cap);
        } else {
#pragma unroll
            for (int e = 0; e < X::PER; ++e) z[e] *= a.scale;
        }
        if (a.bias) {
#pragma unroll
            for (int e = 0; e < X::PER; ++e) z[e] += column[max(row_t[e], 0)];
        }
        if (!all_seen) {
#pragma unroll
            for (int e = 0; e < X::PER; ++e) z[e] = row_t[e] >= 0 ? z[e] : -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < X::PER; ++e) most = fmaxf(most, z[e]);
        if (f.scores && col < cols) {
            const int e0 = t * X::ROWS + X::PER * g;
            float* const to = f.scores + head * f.score_stride + p.first + e0;
            if (e0 + X::PER <= p.count) {
#pragma unroll
                for (int e = 0; e < X::PER; e += 4) __builtin_memcpy(to + e, z + e, 16);        // aligned to a float
            } else {
#pragma unroll
                for (int e = 0; e < X::PER; ++e)
                    if (e0 + e < p.count) to[e] = z[e];
            }
        }
        // The reference of the exponentials moves only when a score exceeds it by more than 7 (a factor of 1,100, nothing to fp32).
        if (__ballot(most > top + 7.f || (top == -INFINITY && most > top))) {
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            const float next = fmaxf(top, most), from = next == -INFINITY ? 0.f : next;
            const float shrink = exp_few_ulp(top - from);
            sum *= shrink;
#pragma unroll
            for (int m = 0; m < X::MB; ++m)
#pragma unroll
                for (int j = 0; j < X::VW; ++j) o[m][j] *= shrink;
            top = next;
        }
        const float from = top == -INFINITY ? 0.f : top;
        float pr[X::PER];
#pragma unroll
        for (int e = 0; e < X::PER; ++e) {
            pr[e] = exp_few_ulp(z[e] - from);
            sum += pr[e];
        }
        if (!all_seen) {
#pragma unroll
            for (int e = 0; e < X::PER; ++e)
#pragma unroll
                for (int m = 0; m < X::MB; ++m) vraw[e][m] = masked(vraw[e][m], row_t[e] >= 0 ? ~0u : 0u);
        }
        if constexpr (X::BF16) {
            Split3 pf;
            pf.set(pr);
#pragma unroll
            for (int m = 0; m < X::MB; ++m)
#pragma unroll
                for (int j = 0; j < X::VW; ++j) {
                    uint32_t v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[i] = __builtin_amdgcn_perm(word(vraw[2 * i + 1][m], j / 2), word(vraw[2 * i][m], j / 2), j % 2 ? 0x07060302u : 0x05040100u);
                    const bf16x8 vf = __builtin_bit_cast(bf16x8, make_uint4(v[0], v[1], v[2], v[3]));
#pragma unroll
                    for (int part = 2; part >= 0; --part) o[m][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf.part[part], o[m][j], 0, 0, 0);
                }
        } else {
#pragma unroll
            for (int e = 0; e < X::PER; ++e)
#pragma unroll
                for (int m = 0; m < X::MB; ++m)
#pragma unroll
                    for (int j = 0; j < X::VW; ++j)
                        o[m][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(word(vraw[e][m], j)), pr[e], o[m][j], 0, 0, 0);
        }
        if (more) load_values(t + stripes);
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);

    float* const to = (p.whole ? f.out + ((int64_t)p.bag * a.q_heads + head) * d : f.part_o + ((int64_t)p.part * a.q_heads + head) * d) - own * d;
    const auto write_norm = [&](float best, float l, float by) {     // by: one over l, 0 for 0
        if (p.whole) {
            f.lse[(int64_t)p.bag * a.q_heads + head] = l == 0.f ? -INFINITY : best + __builtin_amdgcn_logf(l) * kLn2;
            if (f.scores) f.norms[(int64_t)p.bag * a.q_heads + head] = make_float2(best, by);
        } else {
            f.part_ml[((int64_t)p.part * a.q_heads + head) * 2] = best;
            f.part_ml[((int64_t)p.part * a.q_heads + head) * 2 + 1] = l;
        }
    };
    const auto write = [&](int at, const float (&v)[X::VW]) {        // VW elements that lie side by side, if they are the column's head's
        if (col < cols && at >= own * d && at < (own + 1) * d) __builtin_memcpy(__builtin_assume_aligned(to + at, X::VW >= 4 ? 16 : 4 * X::VW), v, sizeof(v));
    };
    if constexpr (ALONE) {
        const float by = !p.whole ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
        if (g == 0 && col < cols) write_norm(top, sum, by);
#pragma unroll
        for (int m = 0; m < X::MB; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v[X::VW];
#pragma unroll
                for (int j = 0; j < X::VW; ++j) v[j] = o[m][j][i] * by;
                write((m * 16 + 4 * g + i) * X::VW, v);
            }
        return;
    }

    // the wavefronts meet: every lane leaves its sums, and takes up a fourth of the lane's own place of all four
    float* const ml = lds + kLdsMl;
    float* const ox = lds + kLdsFree;
    constexpr int kWaveO = X::OREGS * 64;
    __syncthreads();                                                 // done with the table
    if (g == 0) {
        ml[wave * 32 + col] = top;
        ml[wave * 32 + 16 + col] = sum;
    }
#pragma unroll
    for (int m = 0; m < X::MB; ++m)
#pragma unroll
        for (int j = 0; j < X::VW; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) ox[wave * kWaveO + ((m * X::VW + j) * 4 + i) * 64 + lane] = o[m][j][i];
    __syncthreads();
    float best = -INFINITY, l = 0.f, k[kFwdWaves];
#pragma unroll
    for (int x = 0; x < kFwdWaves; ++x) best = fmaxf(best, ml[x * 32 + col]);
#pragma unroll
    for (int x = 0; x < kFwdWaves; ++x) {
        k[x] = exp_few_ulp(ml[x * 32 + col] - (best == -INFINITY ? 0.f : best));
        l = fmaf(k[x], ml[x * 32 + 16 + col], l);
    }
    const float by = l == 0.f ? 0.f : 1.f / l;
    if (p.whole) {
#pragma unroll
        for (int x = 0; x < kFwdWaves; ++x) k[x] = l == 0.f ? 0.f : k[x] * by;
    }
    if (wave == 0 && g == 0 && col < cols) write_norm(best, l, by);
#pragma unroll
    for (int m = 0; m < X::MB; ++m) {
        float v[X::VW];
#pragma unroll
        for (int j = 0; j < X::VW; ++j) {
            v[j] = 0.f;
#pragma unroll
            for (int x = 0; x < kFwdWaves; ++x) v[j] = fmaf(k[x], ox[x * kWaveO + ((m * X::VW + j) * 4 + wave) * 64 + lane], v[j]);
        }
        write((m * 16 + 4 * g + wave) * X::VW, v);
    }
    __syncthreads();                                                 // LDS is free again, the bag's norms there
}

// A workgroup a piece: calls whose bags are short, or so many that they even out.
template <typename T, int DP, int PACK, bool FULL>
__global__ __launch_bounds__(kFwdBlock, DP * PACK > 128 ? 1 : DP * PACK > 64 ? 2 : 3) void embbag_attn_fwd_kernel(FwdArgs f) {
    extern __shared__ float lds[];
    const uint32_t id = blockIdx.z * gridDim.x + blockIdx.x;
    if (id >= f.pieces) return;
    const BagPiece p = find_piece(f.a, f.shift, id);
    if (p.number >= p.of) return;
    attend<T, DP, PACK, FULL, false>(f, Segment{p.bag, id, p.first, p.count, p.of == 1}, lds);
    if (f.scores && p.of == 1 && f.weighed) add_weights<kFwdBlock>(f, p.bag, p.first, p.count);       // all heads were this workgroup's
}

// Short bags: every wavefront takes whole pieces, so that none waits for the others of a workgroup (20,000 bags of up to 50 rows, 4 heads of
// 16 through the matrix instructions: 88 us by workgroups, 58 so; of up to 200: 46 and 48), and has the next piece's entries on their way
// meanwhile.  body(segment, ahead); `rows`: entries whose slots it wants ahead.
template <bool AHEAD, typename F>                                         // AHEAD: where registers are not what is short
__device__ __forceinline__ void for_own_pieces(const FwdArgs& f, int rows, F&& body) {
    const AttnArgs& a = f.a;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t waves = gridDim.x * kFwdWaves;
    uint32_t id = blockIdx.x * kFwdWaves + wave;
    if (id >= f.pieces) return;
    const auto begin = [&](const BagPiece& p) {
        const bool have = lane < rows && lane < p.count;
        return Ahead{have ? a.slots[p.first + lane] : -1, have && a.bias ? a.lookup_pos[p.first + lane] : 0, a.bias ? a.q_pos[p.bag] : 0};
    };
    BagPiece p = find_piece(a, f.shift, id);
    Ahead ahead = begin(p);
    for (;;) {
        const bool more = waves < f.pieces - id;
        BagPiece next{};
        Ahead next_ahead{};
        if (AHEAD && more) {
            next = find_piece(a, f.shift, id + waves);
            next_ahead = begin(next);
        }
        if (p.number < p.of) {
            body(Segment{p.bag, id, p.first, p.count, p.of == 1}, ahead);
            if (f.scores && p.of == 1 && f.weighed) {
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
                add_weights<64>(f, p.bag, p.first, p.count);
            }
        }
        if (!more) break;
        id += waves;
        p = AHEAD ? next : find_piece(a, f.shift, id);
        ahead = AHEAD ? next_ahead : begin(p);
    }
}

template <typename T, int DP, int PACK, bool FULL>
__global__ __launch_bounds__(kFwdBlock, DP * PACK > 128 ? 1 : DP * PACK > 64 ? 2 : 3) void embbag_attn_short_kernel(FwdArgs f) {
    extern __shared__ float lds[];
    const AttnArgs& a = f.a;
    const int group = a.q_heads / a.kv_heads, kv0 = blockIdx.y * PACK;
    read_table<kFwdWaves>(a, lds, kv0 * group, min(PACK, a.kv_heads - kv0) * group);
    if (a.bias) __syncthreads();
    for_own_pieces<true>(f, AttnTile<T, DP, PACK>::ROWS, [&](const Segment& p, const Ahead& ahead) { attend<T, DP, PACK, FULL, true>(f, p, lds, ahead); });
}

// One query head a kv head, and rows that are their own values: the matrix instructions would run 16 columns for one, and read a row
// twice.  A lane holds 16 bytes of a row, LANES lanes a head, 64 / (heads * LANES) rows side by side; a score is a sum over a head's
// lanes, and every lane pools its own elements, rows side by side each with their own maximum and sum up to the end.  Bound by the way
// from a slot to its row, with as many wavefronts as their registers let a CU hold.  (20,000 bags of up to 50 rows, 4 heads of 16: 34 us in
// fp32 and 27 in bf16, through the matrix instructions 58 and 65; keys and values apart, 2 heads of 64 in bf16: 75 and 70, with two query
// heads a kv head 151 and 71.)
template <typename T, int LANES>
__global__ __launch_bounds__(kFwdBlock, sizeof(T) == 4 ? 6 : 5) void embbag_attn_narrow_kernel(FwdArgs f) {
    extern __shared__ float lds[];
    constexpr int kSteps = 2;
    typedef Narrow<T, LANES> N;
    const AttnArgs& a = f.a;
    const int lane = threadIdx.x % 64, width = a.kv_heads * LANES, r = lane / width, head = lane % width / LANES, at = lane % LANES * N::VE;
    const int side = 64 / width, d = N::D;
    const int32_t* const borders = (const int32_t*)lds;
    const float* const table = lds + AttnLds<kFwdWaves>::FREE;
    const T* const w = (const T*)a.cache_w + (int64_t)head * d + at;
    const float by_cap = a.cap > 0 ? a.scale / a.cap : 0.f;
    read_table<kFwdWaves>(a, lds, 0, a.q_heads);
    if (a.bias) __syncthreads();
    for_own_pieces<false>(f, 64, [&](const Segment& p, const Ahead& ahead) {
        float q[N::VE], o[N::VE], top = -INFINITY, sum = 0.f;
        N::read(a.q + ((int64_t)p.bag * a.q_heads + head) * d + at, q);
#pragma unroll
        for (int i = 0; i < N::VE; ++i) o[i] = 0.f;
        int32_t slot_n = ahead.slot, pos_n = ahead.pos;
        for (int e0 = 0; e0 < p.count; e0 += 64) {
            int row_of = -1;
            if ((uint32_t)slot_n < (uint64_t)a.C) row_of = a.bias ? relpos_row(ahead.q_pos - pos_n, borders, a.rp.buckets, a.rp.two_sided) : 0;
            const int slot = row_of >= 0 ? slot_n : 0, here = min(64, p.count - e0);
            if (e0 + 64 < p.count) {
                const bool have = e0 + 64 + lane < p.count;
                slot_n = have ? a.slots[p.first + e0 + 64 + lane] : -1;
                pos_n = have && a.bias ? a.lookup_pos[p.first + e0 + 64 + lane] : 0;
            }
            for (int s0 = 0; s0 < here; s0 += kSteps * side) {
                uint4 raw[kSteps];
                int row[kSteps];
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    const int e = s0 + s * side + r;                         // (behind the 64th: an entry that is not there)
                    row[s] = __shfl(row_of, e & 63);
                    if (e >= here) row[s] = -1;
                    const T* const from = w + (int64_t)__shfl(slot, e & 63) * a.wst;
                    if (s0 + s * side < here) raw[s] = *reinterpret_cast<const uint4*>(from);
                }
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    if (s0 + s * side >= here) break;
                    float v[N::VE];
                    N::widen(masked(raw[s], row[s] >= 0 ? ~0u : 0u), v);
                    float z = N::dot(q, v);
                    z = a.cap > 0 ? a.cap * tanh_few_ulp(z * by_cap) : z * a.scale;
                    if (a.bias) z += table[max(row[s], 0) * a.q_heads + head];
                    if (row[s] < 0) z = -INFINITY;
                    if (f.scores && at == 0 && s0 + s * side + r < here) f.scores[head * f.score_stride + p.first + e0 + s0 + s * side + r] = z;
                    if (__ballot(z > top + 7.f || (top == -INFINITY && z > top))) {
                        const float next = fmaxf(top, z), shrink = exp_few_ulp(top - (next == -INFINITY ? 0.f : next));
                        sum *= shrink;
#pragma unroll
                        for (int i = 0; i < N::VE; ++i) o[i] *= shrink;
                        top = next;
                    }
                    const float pr = exp_few_ulp(z - (top == -INFINITY ? 0.f : top));
                    sum += pr;
#pragma unroll
                    for (int i = 0; i < N::VE; ++i) o[i] = fmaf(pr, v[i], o[i]);
                }
            }
        }
        for (int off = width; off < 64; off <<= 1) {
            const float other = __shfl_xor(top, off), next = fmaxf(top, other), from = next == -INFINITY ? 0.f : next;
            const float ka = exp_few_ulp(top - from), kb = exp_few_ulp(other - from);
            sum = fmaf(sum, ka, __shfl_xor(sum, off) * kb);
#pragma unroll
            for (int i = 0; i < N::VE; ++i) o[i] = fmaf(o[i], ka, __shfl_xor(o[i], off) * kb);
            top = next;
        }
        if (r) return;
        const int64_t to = (int64_t)(p.whole ? p.bag : p.part) * a.q_heads + head;
        const float by = !p.whole ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int i = 0; i < N::VE; ++i) o[i] *= by;
        N::write((p.whole ? f.out : f.part_o) + to * d + at, o);
        if (at == 0) {
            if (p.whole) {
                f.lse[to] = sum == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(sum) * kLn2;
                if (f.scores) f.norms[to] = make_float2(top, by);
            } else {
                f.part_ml[to * 2] = top;
                f.part_ml[to * 2 + 1] = sum;
            }
        }
    });
}

// Few long bags: as many workgroups as the chip holds share all entries evenly, in blocks of kBlock, wherever bags begin and end;
// a part's fixed cost (the way to its first rows, the meeting of its wavefronts: 8 us in a busy memory) is then paid once and at
// the same time everywhere, and no CU is left with a part more than another.  (Rows of 1 KB, 64 bags
// of up to 8,192 entries: 67 us, by pieces 99; all of 4,096: 67 and 71; 1,024 bags of up to 700: 92 and 98.)  Bag b's blocks have the numbers [blocks[b], blocks[b + 1]), an empty bag's
// one block among them; workgroup w takes those from w * all / groups on.  Workgroups beyond the number of blocks (lists that use little of
// their room) take nothing: each of the others has a block, so every one between a bag's first and last owner has written its part.
constexpr int kBlockShift = 7, kBlock = 1 << kBlockShift, kEvenBags = 2048;
__device__ __forceinline__ uint32_t bag_blocks(const AttnArgs& a, uint32_t bag) {
    return max(1u, (uint32_t)((bag_span(a, bag).count + kBlock - 1) >> kBlockShift));
}
__device__ __forceinline__ uint32_t even_start(uint32_t w, uint32_t all, uint32_t groups) { return (uint32_t)((uint64_t)w * all / groups); }
__device__ __forceinline__ uint32_t even_owner(uint32_t block, uint32_t all, uint32_t groups) { return (uint32_t)(((uint64_t)(block + 1) * groups - 1) / all); }

template <typename T, int DP, int PACK, bool FULL>
__global__ __launch_bounds__(kFwdBlock, DP * PACK > 128 ? 1 : DP * PACK > 64 ? 2 : 3) void embbag_attn_even_kernel(FwdArgs f) {
    extern __shared__ float lds[];
    __shared__ uint32_t wave_sums[kFwdWaves], start_bag, start_block;
    const AttnArgs& a = f.a;
    const uint32_t bags = (uint32_t)a.bags, per = (bags + kFwdBlock - 1) / kFwdBlock;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    // running counts: a thread up to kEvenBags / kFwdBlock bags side by side
    uint32_t c[kEvenBags / kFwdBlock], sum = 0;
#pragma unroll
    for (uint32_t i = 0; i < kEvenBags / kFwdBlock; ++i) {
        const uint32_t b = threadIdx.x * per + i;
        c[i] = i < per && b < bags ? bag_blocks(a, b) : 0;
        sum += c[i];
    }
    uint32_t upto = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t x = __shfl_up(upto, off);
        if (lane >= off) upto += x;
    }
    if (lane == 63) wave_sums[wave] = upto;
    if (threadIdx.x == 0) start_bag = bags;
    __syncthreads();
    uint32_t before = upto - sum, all = 0;
#pragma unroll
    for (int x = 0; x < kFwdWaves; ++x) {
        if (x < wave) before += wave_sums[x];
        all += wave_sums[x];
    }
    all = __builtin_amdgcn_readfirstlane(all);
    const uint32_t groups = min(f.groups, all), share = min(blockIdx.x, groups);
    uint32_t at = even_start(share, all, groups);
    const uint32_t end = even_start(min(share + 1, groups), all, groups);
#pragma unroll
    for (uint32_t i = 0; i < kEvenBags / kFwdBlock; ++i) {
        const uint32_t b = threadIdx.x * per + i;
        if (i < per && b < bags) {
            if (blockIdx.x == 0 && blockIdx.y == 0) f.blocks[b] = before;
            if (before <= at && at < before + c[i]) {
                start_bag = b;
                start_block = at - before;
            }
            before += c[i];
            if (b == bags - 1 && blockIdx.x == 0 && blockIdx.y == 0) f.blocks[bags] = before;
        }
    }
    __syncthreads();
    uint32_t bag = __builtin_amdgcn_readfirstlane(start_bag), block = __builtin_amdgcn_readfirstlane(start_block);
    while (at < end && bag < bags) {
        const BagSpan s = bag_span(a, bag);
        const uint32_t mine = max(1u, (uint32_t)((s.count + kBlock - 1) >> kBlockShift)), take = min(mine - block, end - at);
        const int64_t skip = (int64_t)block << kBlockShift;
        attend<T, DP, PACK, FULL, false>(f, Segment{bag, 2 * blockIdx.x + (block == 0), s.first + skip, (int)min(s.count - skip, (int64_t)take << kBlockShift), take == mine}, lds);
        at += take;
        block = 0;
        ++bag;
    }
}

// The parts of a bag of several: a workgroup sums 64 elements of their pooled rows, four a thread and 16 parts side by side, each
// with the maximum and sum of its head, online as within a part.  Workgroups look through `each` bags for such bags.  (64 bags of 12
// parts, 16 heads of 64: 4.8 us, by 16 elements and 64 parts side by side 10.3; two bags of 384: 5.2 and 4.4.)
constexpr int kJoinBlock = 256, kShare = 64;
__global__ __launch_bounds__(kJoinBlock) void embbag_attn_join_kernel(FwdArgs f, int each) {
    constexpr int ACROSS = kShare / 4;
    __shared__ float part[kJoinBlock / 64][ACROSS][6];
    const AttnArgs& a = f.a;
    const int hq = a.q_heads, width = hq * a.d, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int at = blockIdx.y * kShare + threadIdx.x % ACROSS * 4, h = min(at / a.d, hq - 1);
    const int64_t bag0 = (int64_t)(blockIdx.z * gridDim.x + blockIdx.x) * each, mine = bag0 + lane;
    // the parts of a bag, and the number of its i-th
    const auto parts_of = [&](uint32_t bag, uint32_t* first) -> uint32_t {
        if (f.groups) {
            const uint32_t all = f.blocks[a.bags], groups = min(f.groups, all);
            *first = even_owner(f.blocks[bag], all, groups);
            return even_owner(f.blocks[bag + 1] - 1, all, groups) - *first + 1;
        }
        const BagPiece p = bag_piece(a, f.shift, bag, 0, bag_span(a, bag), a.bag_off[bag]);
        *first = p.more;
        return p.of;
    };
    uint32_t first_of = 0;
    uint64_t several = __ballot(lane < each && mine < a.bags && parts_of((uint32_t)min(mine, a.bags - 1), &first_of) > 1);
    for (; several; several &= several - 1) {
        const uint32_t bag = (uint32_t)(bag0 + __ffsll((unsigned long long)several) - 1);
        uint32_t first;
        const uint32_t of = parts_of(bag, &first);
        const auto part_id = [&](uint32_t i) -> int64_t {
            return f.groups ? 2 * (int64_t)(first + i) + (i == 0) : i == 0 ? bag : (int64_t)first + i - 1;
        };
        float top = -INFINITY, l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        const auto take = [&](float m, float x, const float4& v) {
            const float next = fmaxf(top, m), from = next == -INFINITY ? 0.f : next;
            const float ka = exp_few_ulp(top - from), kb = exp_few_ulp(m - from);
            l = fmaf(l, ka, x * kb);
            o.x = fmaf(o.x, ka, v.x * kb);
            o.y = fmaf(o.y, ka, v.y * kb);
            o.z = fmaf(o.z, ka, v.z * kb);
            o.w = fmaf(o.w, ka, v.w * kb);
            top = next;
        };
        constexpr int AHEAD = 4;
        for (uint32_t i0 = threadIdx.x / ACROSS; i0 < of; i0 += kJoinBlock / ACROSS * AHEAD) {
            float2 ml[AHEAD];
            float4 v[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const uint32_t i = i0 + j * (kJoinBlock / ACROSS);
                const bool have = i < of && at < width;
                const int64_t id = part_id(i);
                ml[j] = have ? *reinterpret_cast<const float2*>(f.part_ml + (id * hq + h) * 2) : make_float2(-INFINITY, 0.f);
                v[j] = have ? *reinterpret_cast<const float4*>(f.part_o + id * width + at) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) take(ml[j].x, ml[j].y, v[j]);
        }
#pragma unroll
        for (int off = ACROSS; off < 64; off <<= 1)
            take(__shfl_xor(top, off), __shfl_xor(l, off), make_float4(__shfl_xor(o.x, off), __shfl_xor(o.y, off), __shfl_xor(o.z, off), __shfl_xor(o.w, off)));
        if (lane < ACROSS) {
            float* const x = part[wave][lane];
            x[0] = top, x[1] = l, x[2] = o.x, x[3] = o.y, x[4] = o.z, x[5] = o.w;
        }
        __syncthreads();
        if (threadIdx.x < ACROSS && at < width) {
            for (int w = 1; w < kJoinBlock / 64; ++w) {
                const float* const x = part[w][lane];
                take(x[0], x[1], make_float4(x[2], x[3], x[4], x[5]));
            }
            const bool none = l == 0.f;
            *reinterpret_cast<float4*>(f.out + (int64_t)bag * width + at) =
                none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o.x / l, o.y / l, o.z / l, o.w / l);
            if (at % a.d == 0) {
                f.lse[(int64_t)bag * hq + h] = none ? -INFINITY : top + __builtin_amdgcn_logf(l) * kLn2;
                if (f.scores) f.norms[(int64_t)bag * hq + h] = make_float2(top, none ? 0.f : 1.f / l);
            }
        }
        __syncthreads();
    }
}

// Weights of the entries of the bags that were not whole in one workgroup, from the scores and the bags' final norms: an entry a
// thread.
constexpr int kWeightShift = 8;
__global__ __launch_bounds__(kJoinBlock) void embbag_attn_weight_kernel(FwdArgs f) {
    const uint32_t id = blockIdx.z * gridDim.x + blockIdx.x;
    if (id >= (uint64_t)(f.a.n >> kWeightShift) + f.a.bags) return;
    const BagPiece p = find_piece(f.a, kWeightShift, id);
    if (p.number >= p.of || (f.weighed && bag_piece(f.a, f.shift, p.bag, 0, bag_span(f.a, p.bag), f.a.bag_off[p.bag]).of == 1)) return;
    add_weights<kJoinBlock>(f, p.bag, p.first, p.count);
}

// How a call is laid out.
constexpr int kPieceShift = 9, kLongMean = 1 << kPieceShift, kShortMean = 64, kNarrowMean = 128, kManyBags = 2560;
struct FwdPlan {
    int dp, pack, chunks;      // head_dim rounded up; kv heads a workgroup takes, and how many such shares there are
    bool alone;                // a wavefront a piece
    bool narrow;               // heads without the matrix instructions
    bool even;                 // bags of 512 entries and more in the mean, and not so many that each workgroup could not count them
    uint32_t resident, groups; // workgroups that the chip holds at once; and no more than have a block of entries
    FwdPlan(const bp_attn* at, int dtype, int64_t n, int64_t bags) {
        dp = attn_dp(at, dtype);
        pack = attn_pack(at, dp);
        chunks = (at->kv_heads + pack - 1) / pack;
        even = bags <= kEvenBags && n >= kLongMean * std::max<int64_t>(bags, 1);
        const int flat = pack * dp;
        resident = std::max(1, 256 * (flat > 128 ? 1 : flat > 64 ? 2 : 3) / chunks);
        narrow = attn_narrow(at, dtype);
        // More bags than workgroups at once, and short ones.  Without the matrix instructions also longer ones, if there are enough for half of
        // the chip's wavefronts (heads of 16 fp32, bags of 250 entries in the mean: 8,000 141 us by workgroups and 126, 2,000 45 and 73).
        alone = bags > resident && n < (!narrow ? kShortMean : bags > kManyBags ? kLongMean : kNarrowMean) * bags;
        if (narrow && alone) chunks = 1;
        groups = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(resident, (n >> kBlockShift) + bags));
    }
    // parts that a workspace for n has room for, whatever smaller call it serves
    static int64_t parts(int64_t n, int64_t bags) { return std::max((n >> kPieceShift) + bags, 2 * std::min<int64_t>(768, (n >> kBlockShift) + std::min<int64_t>(bags, kEvenBags))); }
};

// From one head's scores to the next: whole lines, and no power of two.
int64_t score_stride(int64_t n) { return ceil_div(n, 64) * 64 + 192; }

struct FwdScratch {
    float *scores, *part_ml, *part_o;
    float2* norms;
    uint32_t* blocks;
    size_t bytes;
    FwdScratch(void* ws, const bp_attn* at, int64_t n, int64_t bags, bool with_weights) {
        const int64_t parts = FwdPlan::parts(n, bags);
        Carver c(ws, 0);
        scores = c.take<float>(with_weights ? (size_t)score_stride(n) * at->q_heads : 0);
        norms = c.take<float2>(with_weights ? (size_t)bags * at->q_heads : 0);
        part_ml = c.take<float>((size_t)parts * at->q_heads * 2);
        part_o = c.take<float>((size_t)parts * at->q_heads * at->head_dim);
        blocks = c.take<uint32_t>((size_t)std::min<int64_t>(bags, kEvenBags) + 1);
        bytes = c.used();
    }
};

struct FwdLaunch {
    const FwdArgs& f;
    const FwdPlan& l;
    hipStream_t stream;
    template <typename T, int DP, int PACK, bool FULL>
    int run() {
        const int table = f.a.bias ? f.a.rp.rows() * std::min(PACK, f.a.kv_heads) * (f.a.q_heads / f.a.kv_heads) : 0;
        const size_t shared = AttnLds<kFwdWaves>::bytes(DP * PACK, table);
        if (l.even)
            BP_LAUNCH(K_ATTN_FWD, (embbag_attn_even_kernel<T, DP, PACK, FULL>), dim3(f.groups, (unsigned)l.chunks), dim3(kFwdBlock), shared, stream, f);
        else if (l.narrow && l.alone)
            return dispatch_narrow<T>(f.a, *this);
        else if (l.alone)
            BP_LAUNCH(K_ATTN_FWD, (embbag_attn_short_kernel<T, DP, PACK, FULL>), dim3(std::min(l.resident, (unsigned)ceil_div(f.pieces, kFwdWaves)), (unsigned)l.chunks), dim3(kFwdBlock), shared, stream, f);
        else
            BP_LAUNCH(K_ATTN_FWD, (embbag_attn_fwd_kernel<T, DP, PACK, FULL>), spread_grid(f.pieces, (unsigned)l.chunks), dim3(kFwdBlock), shared, stream, f);
        return BP_OK;
    }
    template <typename T, int LANES>
    int run_narrow() {
        const size_t shared = AttnLds<kFwdWaves>::FREE * 4 + (f.a.bias ? (size_t)f.a.rp.rows() * f.a.q_heads * 4 : 0);
        BP_LAUNCH(K_ATTN_FWD, (embbag_attn_narrow_kernel<T, LANES>), dim3(std::min(4096u, (unsigned)ceil_div(f.pieces, kFwdWaves))), dim3(kFwdBlock), shared, stream, f);
        return BP_OK;
    }
};

}  // namespace
}  // namespace bp

using namespace bp;

BP_EXPORT int bp_embbag_attn_fwd_workspace_bytes(const bp_config* cfg, const bp_attn* at, int64_t n_lookups, int64_t bags,
                                                 int32_t with_weights, size_t* bytes) {
    BP_TRY(attn_check_shape(cfg, at));
    BP_TRY(attn_check_sizes(n_lookups, bags, bytes));
    *bytes = FwdScratch(nullptr, at, n_lookups, bags, with_weights != 0).bytes;
    return BP_OK;
}

BP_EXPORT int bp_embbag_attn_fwd(const bp_config* cfg, const bp_attn* at, const bp_relpos* rp, const void* cache_w, const int32_t* lookup_slots,
                                 const int64_t* bag_offsets, const int32_t* bag_lengths, int64_t n_lookups, int64_t bags, const float* q,
                                 const int32_t* q_pos, const int32_t* lookup_pos, const float* bias_table, float* out, float* lse,
                                 const float* weight_in, float* weight_out, void* workspace, size_t workspace_bytes, void* stream_) {
    FwdArgs f{};
    size_t need = 0;
    hipStream_t stream = (hipStream_t)stream_;
    BP_TRY(attn_check(cfg, at, rp, cache_w, lookup_slots, bag_offsets, bag_lengths, n_lookups, bags, q, q_pos, lookup_pos, bias_table, &f.a));
    if (weight_in && !weight_out) return fail(BP_ERR_INVALID_ARG, "weight_in without weight_out");
    if (bags == 0) return BP_OK;
    if (!out || !lse) return fail(BP_ERR_INVALID_ARG, "NULL pointer");
    if (((uintptr_t)out & 15) || (((uintptr_t)lse | (uintptr_t)weight_in | (uintptr_t)weight_out) & 3))
        return fail(BP_ERR_INVALID_ARG, "out must be 16-byte aligned, lse and the weights aligned to their elements");
    const bool weights = weight_out != nullptr && n_lookups > 0;
    BP_TRY(bp_embbag_attn_fwd_workspace_bytes(cfg, at, n_lookups, bags, weights, &need));
    BP_TRY(attn_check_workspace(workspace, workspace_bytes, need));
    const FwdScratch w(workspace, at, n_lookups, bags, weights);
    const FwdPlan l(at, cfg->weight_dtype, n_lookups, bags);
    f.shift = kPieceShift;
    f.pieces = (uint32_t)piece_count(n_lookups, bags, f.shift);
    f.groups = l.even ? l.groups : 0;
    f.blocks = w.blocks;
    f.scores = weights ? w.scores : nullptr;
    f.norms = w.norms;
    f.score_stride = score_stride(n_lookups);
    f.weighed = l.chunks == 1 && !l.even;
    f.part_ml = w.part_ml;
    f.part_o = w.part_o;
    f.out = out;
    f.lse = lse;
    f.weight_in = weight_in;
    f.weight_out = weight_out;
    FwdLaunch launch{f, l, stream};
    BP_TRY(cfg->weight_dtype == BP_F32 ? dispatch_attn<float>(f.a, l.dp, l.pack, launch) : dispatch_attn<uint16_t>(f.a, l.dp, l.pack, launch));
    const bool several = l.even ? l.groups > 1 : n_lookups > (int64_t(1) << f.shift);          // else no bag can have two parts
    if (several) {
        const int64_t shares = ceil_div((int64_t)at->q_heads * at->head_dim, kShare);
        const int64_t each = std::min(std::max<int64_t>(bags * shares / 8192, 1), (int64_t)64);
        BP_LAUNCH(K_ATTN_JOIN, embbag_attn_join_kernel, spread_grid(ceil_div(bags, each), (unsigned)shares), dim3(kJoinBlock), 0, stream, f, (int)each);
    }
    if (weights && (several || !f.weighed))
        BP_LAUNCH(K_ATTN_WEIGHT, embbag_attn_weight_kernel, spread_grid(piece_count(n_lookups, bags, kWeightShift), 1), dim3(kJoinBlock), 0, stream, f);
    return BP_OK;
}
