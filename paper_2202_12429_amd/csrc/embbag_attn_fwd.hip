// bp_embbag_attn_fwd: bags pooled by attention over their cached rows.
//
// One pass over a bag's rows with the running maximum and sum of a softmax.  A bag is cut into pieces of a power of two of
// entries, a workgroup each; the pieces of a bag of several are joined by a second launch, which also turns scores into weights.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_args.h"

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

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct FwdArgs {
    AttnArgs a;
    int32_t shift;              // log2 of a piece's entries
    int32_t heads;              // kv heads of a workgroup: 1, 2 or 4 of its four wavefronts' worth
    uint32_t pieces;
    float* scores;              // [n][q_heads]; NULL when no weights are asked for
    float* part_ml;             // [pieces][q_heads][2]: maximum and sum of a piece
    float* part_o;              // [pieces][q_heads][d]: its weighted values, not divided by the sum
    float* out;
    float* lse;
    const float* weight_in;
    float* weight_out;
};

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kFwdBlock = 256, kFwdWaves = kFwdBlock / 64;

// Three bf16 parts of an fp32 value whose sum it is exactly: the leading eight bits of what the parts before leave.
__device__ __forceinline__ float leading(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
__device__ __forceinline__ uint32_t upper_halves(float lo, float hi) {
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
struct Split3 {
    bf16x8 part[3];             // 8 values: leading, middle and last bits
    __device__ __forceinline__ void set(const float (&x)[8]) {
        uint32_t w[3][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
            for (int s = 0; s < 3; ++s) {
                w[s][i] = upper_halves(a, b);
                a -= leading(a);
                b -= leading(b);
            }
        }
#pragma unroll
        for (int s = 0; s < 3; ++s) part[s] = __builtin_bit_cast(bf16x8, make_uint4(w[s][0], w[s][1], w[s][2], w[s][3]));
    }
};

// How a wavefront takes a tile of rows with the matrix instructions (rows down, the group's query heads across, of which it has
// up to 16).  DP: head_dim rounded up.  Scores: S[row][head] = K Q^T, a lane loads 16 bytes of a row and its neighbours 16 rows
// away the next 16.  Pooling: O^T[d][head] = V^T P^T; a row of S that a lane holds is an entry whose p that lane is asked for, so
// p never leaves its lane, and V comes in whole rows: a lane loads VW elements, which serve VW products of 16 dims each.
// bf16 rows go through the bf16 instruction: q and p are cut into three bf16 parts, whose products are exact in fp32, so that
// what is computed is fp32 (and the instruction's adder is idle for most of the time anyway: 8 TB/s of rows need a sixth of it).
template <typename T, int DP>
struct AttnTile {
    static constexpr bool BF16 = sizeof(T) == 2;
    static constexpr int ROWS = BF16 ? 32 : 16;        // entries of a tile
    static constexpr int NU = ROWS / 16;               // S tiles
    static constexpr int PER = ROWS / 4;               // entries a lane holds scores of
    static constexpr int KC = BF16 ? 32 : 16, KM = (DP + KC - 1) / KC;
    static constexpr int VW = DP / 16 < (BF16 ? 8 : 4) ? DP / 16 : BF16 ? 8 : 4, MB = DP / (16 * VW);
    static constexpr int OREGS = MB * VW * 4;
};

template <int BYTES>
struct Bytes {
    typedef std::conditional_t<BYTES == 16, uint4, std::conditional_t<BYTES == 8, uint2, uint32_t>> type;
};
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t word(const uint2& v, int i) { return i == 0 ? v.x : v.y; }
__device__ __forceinline__ uint32_t word(uint32_t v, int) { return v; }
__device__ __forceinline__ uint4 masked(const uint4& v, uint32_t m) { return make_uint4(v.x & m, v.y & m, v.z & m, v.w & m); }
__device__ __forceinline__ uint2 masked(const uint2& v, uint32_t m) { return make_uint2(v.x & m, v.y & m); }
__device__ __forceinline__ uint32_t masked(uint32_t v, uint32_t m) { return v & m; }

// LDS of a workgroup, in this order: borders, every wavefront's slots and table rows of a tile, its maxima and sums, the bias
// table's columns of the workgroup's heads, and (over the table, once it is done with) the wavefronts' weighted values.
constexpr int kLdsBorders = 0, kLdsTile = BP_RELPOS_MAX_BUCKETS, kLdsMl = kLdsTile + kFwdWaves * 64, kLdsFree = kLdsMl + kFwdWaves * 32;
inline size_t attn_fwd_lds(int dp, int table_floats) {
    return (size_t)(kLdsFree + std::max(table_floats, kFwdWaves * (dp / 4) * 65)) * 4;
}

template <typename T, int DP>
__global__ __launch_bounds__(kFwdBlock) void embbag_attn_fwd_kernel(FwdArgs f) {
    typedef AttnTile<T, DP> X;
    typedef typename Bytes<X::VW * sizeof(T)>::type VRaw;
    extern __shared__ float lds[];
    const AttnArgs& a = f.a;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, col = lane % 16, g = lane / 16;
    const BagPiece p = find_piece(a, f.shift, blockIdx.x, f.pieces);
    if (p.number > 0 && p.number >= p.of) return;
    const int group = a.q_heads / a.kv_heads, heads = f.heads, stripes = kFwdWaves / heads;
    const int kv0 = blockIdx.y * heads, kv = kv0 + wave % heads, stripe = wave / heads;
    const int first_head = kv0 * group, table_cols = heads * group;

    int32_t* const borders = (int32_t*)lds + kLdsBorders;
    int32_t* const tile = (int32_t*)lds + kLdsTile + wave * 64;
    float* const table = lds + kLdsFree;
    if (a.bias) {
        if (threadIdx.x < BP_RELPOS_MAX_BUCKETS) borders[threadIdx.x] = a.rp.borders[threadIdx.x];
        for (int e = threadIdx.x; e < a.rp.rows() * table_cols; e += kFwdBlock)
            table[e] = a.bias[(e / table_cols) * a.q_heads + first_head + e % table_cols];
    }

    // the group's queries: lane col has query head col
    const int head = kv * group + min(col, group - 1);
    const float* const q = a.q + ((int64_t)p.bag * a.q_heads + head) * a.d;
    std::conditional_t<X::BF16, Split3, f32x4> qf[X::KM];
#pragma unroll
    for (int m = 0; m < X::KM; ++m) {
        const int at = m * X::KC + g * (X::KC / 4);
        const bool have = col < group && at < a.d;
        if constexpr (X::BF16) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 t = have ? *reinterpret_cast<const float4*>(q + at + 4 * i) : make_float4(0.f, 0.f, 0.f, 0.f);
                v[4 * i] = t.x, v[4 * i + 1] = t.y, v[4 * i + 2] = t.z, v[4 * i + 3] = t.w;
            }
            qf[m].set(v);
        } else {
            const float4 t = have ? *reinterpret_cast<const float4*>(q + at) : make_float4(0.f, 0.f, 0.f, 0.f);
            qf[m] = f32x4{t.x, t.y, t.z, t.w};
        }
    }
    const int64_t q_pos = a.bias ? a.q_pos[p.bag] : 0;
    __syncthreads();

    f32x4 o[X::MB][X::VW];
#pragma unroll
    for (int m = 0; m < X::MB; ++m)
#pragma unroll
        for (int j = 0; j < X::VW; ++j) o[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float top = -INFINITY, sum = 0.f;             // of the lane's query head; the sum over the lane's own entries
    const T* const w = (const T*)a.cache_w + (int64_t)kv * a.d;
    const int tiles = (p.count + X::ROWS - 1) / X::ROWS;

    // entry `lane` of the tile: its slot and position, one tile ahead
    int32_t slot_n = -1, pos_n = 0;
    const auto fetch = [&](int t) {
        const int e = t * X::ROWS + lane;
        const bool have = lane < X::ROWS && e < p.count;
        slot_n = have ? a.slots[p.first + e] : -1;
        pos_n = have && a.bias ? a.lookup_pos[p.first + e] : 0;
    };
    fetch(stripe);
    for (int t = stripe; t < tiles; t += stripes) {
        int row_of = -1;
        if ((uint32_t)slot_n < (uint64_t)a.C) row_of = a.bias ? relpos_row(q_pos - pos_n, borders, a.rp.buckets, a.rp.two_sided) : 0;
        const bool all_seen = __ballot(row_of >= 0 || lane >= X::ROWS) == ~0ull;
        if (lane < X::ROWS) {
            tile[lane] = row_of >= 0 ? slot_n : 0;                    // what is not seen reads row 0, and leaves it out
            tile[32 + lane] = row_of;
        }
        fetch(t + stripes);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        // row `col` of S tile u is entry PER * (col / 4) + 4u + col % 4, so that lane (col, g)'s scores are of the entries PER * g ...
        uint4 kraw[X::NU][X::KM];
#pragma unroll
        for (int u = 0; u < X::NU; ++u) {
            const T* const row = w + (int64_t)tile[X::PER * (col / 4) + 4 * u + col % 4] * a.wst;
#pragma unroll
            for (int m = 0; m < X::KM; ++m) {
                const int at = m * X::KC + g * (X::KC / 4);
                kraw[u][m] = at < a.d ? *reinterpret_cast<const uint4*>(row + at) : make_uint4(0, 0, 0, 0);
            }
        }
        VRaw vraw[X::PER][X::MB];
        int32_t row_t[X::PER];
#pragma unroll
        for (int e = 0; e < X::PER; ++e) {
            const T* const row = w + (int64_t)tile[X::PER * g + e] * a.wst + a.value_at;
            row_t[e] = tile[32 + X::PER * g + e];
#pragma unroll
            for (int m = 0; m < X::MB; ++m) {
                const int at = m * 16 * X::VW + col * X::VW;
                vraw[e][m] = *reinterpret_cast<const VRaw*>(row + (at < a.d ? at : 0));
            }
        }
        float z[X::PER];
#pragma unroll
        for (int u = 0; u < X::NU; ++u) {
            f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < X::KM; ++m) {
                if constexpr (X::BF16) {
                    const bf16x8 k = __builtin_bit_cast(bf16x8, kraw[u][m]);
#pragma unroll
                    for (int part = 2; part >= 0; --part) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[m].part[part], s, 0, 0, 0);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(word(kraw[u][m], e)), qf[m][e], s, 0, 0, 0);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) z[4 * u + i] = s[i];
        }
        float most = -INFINITY;
#pragma unroll
        for (int e = 0; e < X::PER; ++e) {
            float c = z[e] * a.scale;
            if (a.cap > 0) c = a.cap * tanh_few_ulp(c / a.cap);
            if (a.bias) c += table[max(row_t[e], 0) * table_cols + (wave % heads) * group + min(col, group - 1)];
            z[e] = row_t[e] >= 0 ? c : -INFINITY;
            most = fmaxf(most, z[e]);
        }
        if (f.scores && col < group) {
#pragma unroll
            for (int e = 0; e < X::PER; ++e)
                if (t * X::ROWS + X::PER * g + e < p.count)
                    f.scores[(p.first + t * X::ROWS + X::PER * g + e) * a.q_heads + head] = z[e];
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
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);

    // the wavefronts of a head meet
    float* const ml = lds + kLdsMl;
    float* const ox = lds + kLdsFree;
    constexpr int kWaveO = X::OREGS * 65;
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
            for (int i = 0; i < 4; ++i) ox[wave * kWaveO + ((m * X::VW + j) * 4 + i) * 65 + lane] = o[m][j][i];
    __syncthreads();
    const bool whole = p.of <= 1;
    for (int e = threadIdx.x; e < heads * group * a.d; e += kFwdBlock) {
        const int at = e % a.d, qh = e / a.d, c = qh % group, wh = qh / group;
        const int row = at % (16 * X::VW) / X::VW, reg = (at / (16 * X::VW) * X::VW + at % X::VW) * 4 + row % 4, from = row / 4 * 16 + c;
        float best = -INFINITY;
        for (int s = 0; s < stripes; ++s) best = fmaxf(best, ml[(wh + s * heads) * 32 + c]);
        const float ref = best == -INFINITY ? 0.f : best;
        float l = 0.f, v = 0.f;
        for (int s = 0; s < stripes; ++s) {
            const int x = wh + s * heads;
            const float k = exp_few_ulp(ml[x * 32 + c] - ref);
            l = fmaf(k, ml[x * 32 + 16 + c], l);
            v = fmaf(k, ox[x * kWaveO + reg * 65 + from], v);
        }
        const int h = first_head + qh;
        if (whole) {
            f.out[((int64_t)p.bag * a.q_heads + h) * a.d + at] = l == 0.f ? 0.f : v / l;
            if (at == 0) f.lse[(int64_t)p.bag * a.q_heads + h] = l == 0.f ? -INFINITY : best + __builtin_amdgcn_logf(l) * kLn2;
        } else {
            f.part_o[((int64_t)blockIdx.x * a.q_heads + h) * a.d + at] = v;
        }
        if (at == 0 && (!whole || f.scores)) {
            f.part_ml[((int64_t)blockIdx.x * a.q_heads + h) * 2] = best;
            f.part_ml[((int64_t)blockIdx.x * a.q_heads + h) * 2 + 1] = l;
        }
    }
}

// A workgroup a piece again: the bag's maxima and sums over its pieces, then this piece's share of the pooled rows and its own
// entries' weights.
constexpr int kShare = 16;                        // elements of the pooled rows that a workgroup sums at a time, 64 bytes
__global__ __launch_bounds__(kFwdBlock) void embbag_attn_join_kernel(FwdArgs f) {
    extern __shared__ float lds[];
    const AttnArgs& a = f.a;
    const BagPiece p = find_piece(a, f.shift, blockIdx.x, f.pieces);
    if (p.number >= p.of || (p.of == 1 && !f.scores)) return;
    const int hq = a.q_heads, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    float* const best = lds;                      // [hq]
    float* const total = lds + hq;                // [hq]
    float* const part = lds + 2 * hq;             // [kFwdBlock]
    const float* const ml = f.part_ml + (int64_t)p.first_id * hq * 2;
    for (int h = wave; h < hq; h += kFwdWaves) {
        float top = -INFINITY;
        for (uint32_t i = lane; i < p.of; i += 64) top = fmaxf(top, ml[((int64_t)i * hq + h) * 2]);
        for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
        const float from = top == -INFINITY ? 0.f : top;
        float l = 0.f;
        for (uint32_t i = lane; i < p.of; i += 64) l = fmaf(exp_few_ulp(ml[((int64_t)i * hq + h) * 2] - from), ml[((int64_t)i * hq + h) * 2 + 1], l);
        for (int off = 32; off >= 1; off >>= 1) l += __shfl_xor(l, off);
        if (lane == 0) {
            best[h] = from;
            total[h] = l;
            if (p.number == 0 && p.of > 1) f.lse[(int64_t)p.bag * hq + h] = l == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(l) * kLn2;
        }
    }
    __syncthreads();
    if (p.of > 1) {
        const int width = hq * a.d;               // a multiple of 8
        const float* const po = f.part_o + (int64_t)p.first_id * width;
        for (int e0 = p.number * kShare; e0 < width; e0 += p.of * kShare) {
            const int e = e0 + threadIdx.x % kShare, h = min(e / a.d, hq - 1);
            float v = 0.f;
            for (uint32_t i = threadIdx.x / kShare; i < p.of && e < width; i += kFwdBlock / kShare)
                v = fmaf(exp_few_ulp(ml[((int64_t)i * hq + h) * 2] - best[h]), po[(int64_t)i * width + e], v);
            part[threadIdx.x] = v;
            __syncthreads();
            if (threadIdx.x < kShare && e < width) {
                for (int i = 1; i < kFwdBlock / kShare; ++i) v += part[i * kShare + threadIdx.x];
                f.out[(int64_t)p.bag * width + e] = total[h] == 0.f ? 0.f : v / total[h];
            }
            __syncthreads();
        }
    }
    if (!f.scores) return;
    for (int i = threadIdx.x; i < p.count; i += kFwdBlock) {
        const int64_t k = p.first + i;
        float add = 0.f;
        for (int h = 0; h < hq; ++h) {
            const float e = exp_few_ulp(f.scores[k * hq + h] - best[h]);
            add += total[h] == 0.f ? 0.f : e / total[h];
        }
        f.weight_out[k] = (f.weight_in ? f.weight_in[k] : 0.f) + add;
    }
}

// kv heads that share a workgroup's four wavefronts: whole rows are then read by one workgroup where heads are few.
int fwd_heads(int kv_heads) { return kv_heads % 4 == 0 ? 4 : kv_heads % 2 == 0 ? 2 : 1; }
// Pieces so small that the launch has two workgroups for every CU, within limits.
constexpr int kShiftLeast = 7, kShiftMost = 10, kPiecesEnough = 1024;
int64_t fwd_enough(const bp_attn* at) { return kPiecesEnough / (at->kv_heads / fwd_heads(at->kv_heads)); }
int fwd_shift(const bp_attn* at, int64_t n) {
    int shift = kShiftLeast;
    while (shift < kShiftMost && (n >> shift) > fwd_enough(at)) ++shift;
    return shift;
}

struct FwdScratch {
    float *scores, *part_ml, *part_o;
    size_t bytes;
    FwdScratch(void* ws, const bp_attn* at, int64_t n, int64_t bags, bool with_weights) {
        // room for the pieces of any n up to this one: a workspace for the largest call serves the smaller ones
        const int64_t pieces = bags + std::max(std::min(n >> kShiftLeast, fwd_enough(at)), n >> kShiftMost);
        Carver c(ws, 0);
        scores = c.take<float>(with_weights ? (size_t)n * at->q_heads : 0);
        part_ml = c.take<float>((size_t)pieces * at->q_heads * 2);
        part_o = c.take<float>((size_t)pieces * at->q_heads * at->head_dim);
        bytes = c.used();
    }
};

template <typename T, int DP>
int launch_fwd(const FwdArgs& f, hipStream_t stream) {
    const int table = f.a.bias ? f.a.rp.rows() * f.heads * (f.a.q_heads / f.a.kv_heads) : 0;
    BP_LAUNCH(K_ATTN_FWD, (embbag_attn_fwd_kernel<T, DP>), dim3(f.pieces, (unsigned)(f.a.kv_heads / f.heads)), dim3(kFwdBlock), attn_fwd_lds(DP, table),
              stream, f);
    return BP_OK;
}
template <typename T>
int launch_fwd(const FwdArgs& f, hipStream_t stream) {
    if constexpr (sizeof(T) == 4) {
        if (f.a.d <= 16) return launch_fwd<T, 16>(f, stream);
    }
    if (f.a.d <= 32) return launch_fwd<T, 32>(f, stream);
    if (f.a.d <= 64) return launch_fwd<T, 64>(f, stream);
    if (f.a.d <= 128) return launch_fwd<T, 128>(f, stream);
    return launch_fwd<T, 256>(f, stream);
}

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
    f.shift = fwd_shift(at, n_lookups);
    f.heads = fwd_heads(at->kv_heads);
    f.pieces = (uint32_t)piece_count(n_lookups, bags, f.shift);
    f.scores = weights ? w.scores : nullptr;
    f.part_ml = w.part_ml;
    f.part_o = w.part_o;
    f.out = out;
    f.lse = lse;
    f.weight_in = weight_in;
    f.weight_out = weight_out;
    BP_TRY(cfg->weight_dtype == BP_F32 ? launch_fwd<float>(f, stream) : launch_fwd<uint16_t>(f, stream));
    if (weights || n_lookups > (int64_t(1) << f.shift))         // else no bag can have two pieces
        BP_LAUNCH(K_ATTN_JOIN, embbag_attn_join_kernel, dim3(f.pieces), dim3(kFwdBlock), (size_t)(2 * at->q_heads + kFwdBlock) * 4, stream, f);
    return BP_OK;
}
