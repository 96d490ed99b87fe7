// bp_embbag_attn_bwd: the gradients of bags pooled by attention over their cached rows.
//
// One pass over a bag's rows.  With lse and the pooled rows from the forward pass a score's gradient needs no other entry:
//     p = exp(c - lse),  dz = p * (<grad_out, value> - <grad_out, out>),  ds = dz * (the cap's slope) * scale
// grad of the key = sum over its heads of ds * q, of the value = sum of p * grad_out, of q = sum over the entries of ds * key,
// of the bias table = sum of dz by table row.  Bound by memory: a row is read once and its gradient, in fp32, written.
#include <algorithm>
#include <cmath>

#include "attn_tile.h"

namespace bp {
namespace {

// Wavefronts work by themselves: all entries are numbered in units of 32, bag b's from (its offset >> 5) + b on, and shared out
// evenly, wherever bags begin and end.  A bag that is one wavefront's has its grad_q from there; parts of others meet in a launch
// of their own.
constexpr int kUnitShift = 5, kUnit = 1 << kUnitShift;
// A share's gradient of the bias table is summed in fp32, a lane a quarter of the entries (without matrix instructions: of the rows side by
// side), and in fp64 from there on: up to this many units, 4,096 entries, a share.
constexpr int kMostUnits = 128;
constexpr int kBwdWaves = 4, kBwdBlock = kBwdWaves * 64;

struct BwdArgs {
    AttnArgs a;
    const float* out;
    const float* lse;
    const float* grad_out;
    float* grad_q;
    float* grad_rows;
    uint32_t units, waves;      // (n >> kUnitShift) + bags; wavefronts that share them
    float* parts;               // [2 * waves][q_heads][d]: grad_q of a bag's part: [2w] of the bag that is under way as wavefront w
                                // begins, [2w + 1] of the one it begins and does not end
    double* bias_parts;         // [workgroups][table rows][q_heads]
};

__device__ __forceinline__ uint32_t first_unit(const AttnArgs& a, uint32_t bag) {
    int64_t at = a.bag_off[bag];
    if (at < 0) at = 0;
    if (at > a.n) at = a.n;
    return (uint32_t)(at >> kUnitShift) + bag;
}
__device__ __forceinline__ uint32_t share_start(uint32_t wave, uint32_t units, uint32_t waves) { return (uint32_t)((uint64_t)wave * units / waves); }
__device__ __forceinline__ uint32_t share_of(uint32_t unit, uint32_t units, uint32_t waves) {
    return min((uint32_t)(((uint64_t)(unit + 1) * waves - 1) / units), waves - 1);
}

// A wavefront's bags, or parts of them: body(bag, first entry, entries, all that the bag uses?, its beginning?).
template <typename F>
__device__ __forceinline__ void for_own_bags(const BwdArgs& f, uint32_t share, F&& body) {
    const AttnArgs& a = f.a;
    const int lane = threadIdx.x % 64;
    uint32_t at = share < f.waves ? share_start(share, f.units, f.waves) : f.units;
    const uint32_t end = share < f.waves ? share_start(share + 1, f.units, f.waves) : f.units;
    uint32_t bag = 0;
    if (at < end) {
        uint32_t hi = (uint32_t)a.bags;
        while (hi - bag > 1) {                                           // the last bag that begins no later, 64 bags a step
            const uint32_t step = (hi - bag + 63) / 64, i = bag + (lane + 1) * step;
            bag += __popcll(__ballot(i < hi && first_unit(a, i) <= at)) * step;
            hi = min(hi, bag + step);
        }
    }
    for (; at < end && bag < (uint32_t)a.bags; ++bag) {
        // the bag's units from `at` on that are this wavefront's
        const BagSpan s = bag_span(a, bag);
        const uint32_t from = first_unit(a, bag), mine = max(1u, (uint32_t)((s.count + kUnit - 1) >> kUnitShift));
        const uint32_t begin = at - min(at, from), stop = min(mine, end - min(end, from));
        const bool starts = begin == 0, whole = starts && stop == mine;
        at = bag + 1 < (uint32_t)a.bags ? max(at, first_unit(a, bag + 1)) : end;
        if (begin >= stop) continue;                                     // numbers without a unit
        body(bag, s.first + ((int64_t)begin << kUnitShift), (int)min(s.count - ((int64_t)begin << kUnitShift), (int64_t)(stop - begin) << kUnitShift), whole, starts);
    }
}
// Where a mask of low values in the bias table covers a whole bag, lse is that value: rounded, it no longer holds the sum of the
// exponentials, and every weight exp(score - lse) would be 1.  So from kFarLse on, where lse is off by 2^-8 or more, the sum over the bag's
// entries (a lane's: from, from + step ...) is made again, plainly, and divides the weights; but not where the scores before the bias
// are no longer small against lse (-infinity then): those have lost more to their own rounding, and add up in another order here.  Every
// wavefront that has a part of such a bag reads all of its keys once more (64 bags of 4,096, 16 heads on 4 of 64: 2.3 ms, without the mask
// 0.18).  The arguments are read anew, so that nothing of this stays in registers along the kernel.
constexpr float kFarLse = 65536.f, kSmall = 64.f;
__device__ __forceinline__ bool far_lse(float lse) { return fabsf(lse) >= kFarLse && fabsf(lse) < INFINITY; }
typedef const __attribute__((address_space(4))) AttnArgs* Again;         // the kernels' only argument begins with them
__device__ __forceinline__ Again arguments_again() {
    auto at = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return (Again)at;
}
template <typename T>
__device__ __forceinline__ float sum_of_weights(uint32_t bag, int64_t first, int64_t count, int head, int kv_head, float lse, int from, int step,
                                                const int32_t* borders, const float* column, int columns) {
    typedef Narrow<T, 1> N;                                              // 16 bytes of a row
    const Again a = arguments_again();
    const int32_t *const slots = a->slots + first, *const pos = a->lookup_pos + first;
    const int d = a->d;
    const float* const q = a->q + ((int64_t)bag * a->q_heads + head) * d;
    const int64_t q_pos = a->q_pos[bag];
    float sum = 0.f;
#pragma unroll 1
    for (int64_t e = from; e < count; e += step) {
        const int32_t slot = slots[e];
        if ((uint32_t)slot >= (uint64_t)a->C) continue;
        const int row_of = relpos_row(q_pos - pos[e], borders, a->rp.buckets, a->rp.two_sided);
        if (row_of < 0) continue;
        const T* const key = (const T*)a->cache_w + (int64_t)slot * a->wst + (int64_t)kv_head * d;
        float c = 0.f;
#pragma unroll 1
        for (int x = 0; x < d; x += N::VE) {
            float k[N::VE], y[N::VE];
            N::widen(*reinterpret_cast<const uint4*>(key + x), k);
            N::read(q + x, y);
#pragma unroll
            for (int i = 0; i < N::VE; ++i) c = fmaf(y[i], k[i], c);
        }
        c = a->cap > 0 ? a->cap * tanh_few_ulp(c * (a->scale / a->cap)) : c * a->scale;
        if (!(fabsf(c) * kSmall < fabsf(lse))) return -INFINITY;
        c += column[row_of * columns];
        if (c != -INFINITY) sum += exp_few_ulp(c - lse);
    }
    return sum;
}
__device__ __forceinline__ float shift_of(float sum) { return sum > 0.f && sum < INFINITY ? -__builtin_amdgcn_logf(sum) : 0.f; }

// Elements of the rows that are neither key nor value.
__device__ __forceinline__ void clear_rest(const BwdArgs& f, int64_t first, int count) {
    const AttnArgs& a = f.a;
    const int span = a.kv_heads * a.d, behind = a.value_at + span, gap = a.value_at == 0 ? 0 : a.value_at - span;
    if (gap + a.dim - behind > 0)
        for (int64_t e = threadIdx.x % 64; e < (int64_t)count * (gap + a.dim - behind); e += 64) {
            const int x = (int)(e % (gap + a.dim - behind));
            f.grad_rows[(first + e / (gap + a.dim - behind)) * a.dim + (x < gap ? span + x : behind + x - gap)] = 0.f;
        }
}

// LDS: borders, the bias table's columns of the workgroup's heads; of every wavefront two tiles' slots and table rows, a tile's ds and p
// entry by entry, and four tables of sums, one for each quarter of the wavefront, in which a column is one lane's.
// STAGE: 16 entries' row gradients, to be written out a row at a time: keys' and values', or, of wide heads, a stretch of either.
template <typename T, int DP, int PACK, bool FULL>
struct BwdLds {
    static constexpr int FLAT = DP * PACK, ROWS = sizeof(T) == 2 ? 32 : 16, WIDE = 17;
    static constexpr bool STAGED = FULL, APART = DP > 64;
    static constexpr int STRETCH = APART ? 128 : FLAT, STAGE_WIDE = (APART ? 1 : 2) * STRETCH + 4, STAGE = STAGED ? 16 * STAGE_WIDE : 0;
    static constexpr int EACH = 128 + 2 * ROWS * WIDE + STAGE;                          // of a wavefront behind the borders
    static size_t floats(int table_rows, int cols) { return 64 + (size_t)kBwdWaves * EACH + (size_t)table_rows * cols + (size_t)kBwdWaves * 4 * table_rows * 16; }
};

// Workgroups that a CU holds, by their registers.
constexpr int bwd_groups_a_cu(size_t elem, int dp, int flat) { return flat <= 32 || (elem == 4 && dp <= 32 && flat <= 64) ? 2 : 1; }

constexpr int kNarrowGroups = 4;         // of the kernel without matrix instructions

template <typename T, int DP, int PACK, bool FULL>
__global__ __launch_bounds__(kBwdBlock, bwd_groups_a_cu(sizeof(T), DP, DP * PACK)) void embbag_attn_bwd_kernel(BwdArgs f) {
    typedef AttnTile<T, DP, PACK> X;
    typedef BwdLds<T, DP, PACK, FULL> L;
    typedef typename Bytes<X::VW * sizeof(T)>::type VRaw;
    constexpr int STEPS = PACK == 1 ? 4 : PACK == 2 ? 2 : 1;             // of four columns, in a head's group
    constexpr int BLOCKS = DP / 16, SOME = BLOCKS < 8 ? BLOCKS : 8;      // of 16 elements of a head; blocks whose gradients are in work at a time
    // q and grad_out in registers all along a bag, where they fit; else from the caches, tile by tile (400,000 rows of 2 x 256 bf16: 460 us so,
    // 1370 with registers spilled)
    constexpr bool KEEP = DP <= 128;
    extern __shared__ float lds[];
    const AttnArgs& a = f.a;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, g = lane / 16;
    const int d = FULL ? DP : a.d;
    const int group = a.q_heads / a.kv_heads, kv0 = blockIdx.y * PACK, heads = FULL ? PACK : min(PACK, a.kv_heads - kv0);
    const int first_head = kv0 * group, cols = heads * group, flat = heads * d;
    const int head = first_head + min(col, cols - 1), own = min(col, cols - 1) / group;
    const int table_rows = a.bias ? a.rp.rows() : 0;

    int32_t* const borders = (int32_t*)lds;
    int32_t* const tiles_of = (int32_t*)lds + 64 + wave * L::EACH;       // two tiles: slots, then table rows
    float* const turn_ds = lds + 64 + wave * L::EACH + 128;              // [entry][column]
    float* const turn_p = turn_ds + L::ROWS * L::WIDE;
    float* const stage = turn_p + L::ROWS * L::WIDE;                     // [entry][key, value][element]
    float* const table = lds + 64 + kBwdWaves * L::EACH;
    float* const sums = table + table_rows * cols + wave * 4 * table_rows * 16 + g * table_rows * 16 + col;      // this lane's column
    if (a.bias) {
        if (threadIdx.x < BP_RELPOS_MAX_BUCKETS) borders[threadIdx.x] = a.rp.borders[threadIdx.x];
        for (int e = threadIdx.x; e < table_rows * cols; e += kBwdBlock) table[e] = a.bias[(e / cols) * a.q_heads + first_head + e % cols];
        for (int r = 0; r < table_rows; ++r) sums[r * 16] = 0.f;
        __syncthreads();
    }

    const uint32_t share = blockIdx.x * kBwdWaves + wave;
    const T* const w = (const T*)a.cache_w + (int64_t)kv0 * d;
    const float by_cap = a.cap > 0 ? a.scale / a.cap : 0.f;
    int sum_row = -1;                                                    // the lane's running sum for the bias table, and its row
    float sum_dz = 0.f;

    for_own_bags(f, share, [&](uint32_t bag, int64_t first, int count, bool whole, bool starts) {
        // A tile's slots come two tiles ahead of their rows' use (the first tile's before all else: 20,000 bags of up to 50, 8 heads on 2 of 32:
        // 170 us so, behind the bag's own products 177), its rows as soon as the tile before has its scores.
        int32_t slot_n = -1, pos_n = 0;
        const auto fetch = [&](int e0) {
            const bool have = lane < X::ROWS && e0 + lane < count;
            slot_n = have ? a.slots[first + e0 + lane] : -1;
            pos_n = have && a.bias ? a.lookup_pos[first + e0 + lane] : 0;
        };
        fetch(0);
        // q and grad_out: for the products with rows, and (a column a quarter) for those with ds and p
        const float* const q = a.q + ((int64_t)bag * a.q_heads + head) * d;
        const float* const go = f.grad_out + ((int64_t)bag * a.q_heads + head) * d;
        const float* const po = f.out + ((int64_t)bag * a.q_heads + head) * d;
        typedef std::conditional_t<X::BF16, Split3, f32x4> Frag;
        const auto columns = [&](const float* of, int m, float (&v)[X::KC / 4]) {       // elements of the column's head that are this lane's
            const int x = m * X::KC + g * (X::KC / 4);
#pragma unroll
            for (int i = 0; i < X::KC / 16; ++i) {
                const int place = (FULL || x < d ? x : 0) + 4 * i;       // inside the row in any case, as below: no branch a load
                const float4 t = or_zeros(*reinterpret_cast<const float4*>(of + place), col < cols && x < d);
                v[4 * i] = t.x, v[4 * i + 1] = t.y, v[4 * i + 2] = t.z, v[4 * i + 3] = t.w;
            }
        };
        const auto fragment = [&](Frag& to, const float (&v)[X::KC / 4]) {
            if constexpr (X::BF16) to.set(v);
            else to = f32x4{v[0], v[1], v[2], v[3]};
        };
        // scores and <grad_out, value>, each entry's against every column
        const auto product = [&](const uint4& rows, const Frag& with, f32x4& sum) {
            if constexpr (X::BF16) {
#pragma unroll
                for (int part = 2; part >= 0; --part)
                    sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, rows), with.part[part], sum, 0, 0, 0);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(word(rows, i)), with[i], sum, 0, 0, 0);
            }
        };
        // <grad_out, out> of the column: the same products in the same order, out in the place of a value, so that where a bag sees one entry
        // (whose value out then is, bit for bit) it equals <grad_out, value> and the score has no gradient: not the noise of two roundings,
        // which a step of Adagrad would blow up.  All loads first (2,000 bags of up to 400 rows of 1 KB: 156 us; 161 with every step's products
        // between its loads and the next one's).
        Frag qf[KEEP ? X::KM : 1], gf[KEEP ? X::KM : 1];
        float us[X::KM][X::KC / 4], os[X::KM][X::KC / 4], qs[KEEP ? X::KM : 1][X::KC / 4];
#pragma unroll
        for (int m = 0; m < X::KM; ++m) {
            columns(go, m, us[m]);
            columns(po, m, os[m]);
            if constexpr (KEEP) columns(q, m, qs[m]);
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (KEEP) {
#pragma unroll
            for (int m = 0; m < X::KM; ++m) {
                fragment(gf[m], us[m]);
                fragment(qf[m], qs[m]);
            }
        }
        constexpr int SUMS = X::BF16 ? 3 : 1;                            // a part of out each; the leading one's is all of it for a bf16 value
        f32x4 sa[SUMS];                                                  // of heads 4g ... with the column's grad_out
#pragma unroll
        for (int x = 0; x < SUMS; ++x) sa[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int m = 0; m < X::KM; ++m) {
            Frag of_out;
            if constexpr (!KEEP) fragment(gf[0], us[m]);
            fragment(of_out, os[m]);
#pragma unroll
            for (int x = 0; x < SUMS; ++x) {
                if constexpr (X::BF16) product(__builtin_bit_cast(uint4, of_out.part[x]), gf[KEEP ? m : 0], sa[x]);
                else product(__builtin_bit_cast(uint4, of_out), gf[KEEP ? m : 0], sa[x]);
            }
        }
        if constexpr (X::BF16) sa[0] += sa[1] + sa[2];
        const float against = __shfl(col % 4 == 0 ? sa[0][0] : col % 4 == 1 ? sa[0][1] : col % 4 == 2 ? sa[0][2] : sa[0][3], col / 4 * 16 + col);
        const float lse = f.lse[(int64_t)bag * a.q_heads + head];
        float shift = 0.f;
        if (a.bias && __any(far_lse(lse))) {
            const BagSpan span = bag_span(a, bag);
            float sum = sum_of_weights<T>(bag, span.first, span.count, head, head / group, lse, g, 4, borders, table + min(col, cols - 1), cols);
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (far_lse(lse)) shift = shift_of(sum);
        }
        const auto element = [&](const float* of, int k, int b, int t) { // 16 * block + col of head k's column 4 * step + g
            const int c = 4 * t + g, x = 16 * b + col;
            const int64_t place = ((int64_t)bag * a.q_heads + first_head + (FULL ? k : min(k, heads - 1)) * group + min(c, group - 1)) * d + (FULL ? x : min(x, d - 1));
            const float v = of[place];
            return k < heads && c < group && x < d ? v : 0.f;
        };
        float qt[KEEP ? PACK : 1][BLOCKS][STEPS], gt[KEEP ? PACK : 1][BLOCKS][STEPS];
        if constexpr (KEEP) {
#pragma unroll
            for (int k = 0; k < PACK; ++k)
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int t = 0; t < STEPS; ++t) {
                        qt[k][b][t] = element(a.q, k, b, t);
                        gt[k][b][t] = element(f.grad_out, k, b, t);
                    }
        }
        const int64_t q_pos = a.bias ? a.q_pos[bag] : 0;

        f32x4 dq[X::MB][X::VW];
#pragma unroll
        for (int m = 0; m < X::MB; ++m)
#pragma unroll
            for (int j = 0; j < X::VW; ++j) dq[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};

        uint64_t seen_n = 0;
        int one_row_n = -1;                                              // the table row, where all entries have the same: far away, mostly
        const auto place = [&](int e0) {
            int row_of = -1;
            if ((uint32_t)slot_n < (uint64_t)a.C) row_of = a.bias ? relpos_row(q_pos - pos_n, borders, a.rp.buckets, a.rp.two_sided) : 0;
            seen_n = __ballot(row_of >= 0);
            const int one = __builtin_amdgcn_readfirstlane(row_of);
            one_row_n = __all(row_of == one || lane >= X::ROWS) ? one : -1;
            int32_t* const tile = tiles_of + (e0 / X::ROWS & 1) * 64;
            __builtin_amdgcn_wave_barrier();
            if (lane < X::ROWS) {
                tile[lane] = row_of >= 0 ? slot_n : 0;                   // what is not seen reads row 0, and leaves it out
                tile[32 + lane] = row_of;
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        };
        const auto row_of_tile = [&](int e0, int u) {
            return w + (int64_t)(tiles_of + (e0 / X::ROWS & 1) * 64)[X::PER * (col / 4) + 4 * u + col % 4] * a.wst;
        };
        const auto row_part = [&](const T* row, int k, int m) {          // (a head that is not there is nobody's)
            return row_bytes_at<FULL>(row + (FULL ? k : min(k, heads - 1)) * d, m * X::KC + g * (X::KC / 4), d);
        };
        uint4 kr[X::NU][PACK][X::KM], vr[X::NU][PACK][X::KM];
        const auto load_rows = [&](int e0) {
#pragma unroll
            for (int u = 0; u < X::NU; ++u) {
                const T* const row = row_of_tile(e0, u);
#pragma unroll
                for (int k = 0; k < PACK; ++k)
#pragma unroll
                    for (int m = 0; m < X::KM; ++m) {
                        kr[u][k][m] = row_part(row, k, m);
                        vr[u][k][m] = row_part(row + a.value_at, k, m);
                    }
            }
        };
        place(0);
        load_rows(0);
        fetch(X::ROWS);
        for (int e0 = 0; e0 < count; e0 += X::ROWS) {
            const int32_t* const tile = tiles_of + (e0 / X::ROWS & 1) * 64;
            const uint64_t seen = seen_n;
            const int one_row = one_row_n;
            const bool all_seen = seen == (X::ROWS == 32 ? 0xffffffffull : 0xffffull);
            // the keys again, in whole rows (from the caches)
            VRaw kv[X::PER][X::MB];
            const auto whole_keys = [&]() {
#pragma unroll
                for (int e = 0; e < X::PER; ++e) {
                    const T* const row = w + (int64_t)tile[X::PER * g + e] * a.wst;
#pragma unroll
                    for (int m = 0; m < X::MB; ++m) {
                        const int x = m * 16 * X::VW + col * X::VW;
                        kv[e][m] = *reinterpret_cast<const VRaw*>(row + (FULL || x < flat ? x : 0));
                    }
                }
            };
            whole_keys();
            float c[X::PER], dp[X::PER];
            if constexpr (KEEP) {
#pragma unroll
                for (int u = 0; u < X::NU; ++u)
#pragma unroll
                    for (int k = 0; k < PACK; ++k) {
                        f32x4 sc = {0.f, 0.f, 0.f, 0.f}, sp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int m = 0; m < X::KM; ++m) {
                            product(kr[u][k][m], qf[m], sc);
                            product(vr[u][k][m], gf[m], sp);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            c[4 * u + i] = k == 0 || own == k ? sc[i] : c[4 * u + i];
                            dp[4 * u + i] = k == 0 || own == k ? sp[i] : dp[4 * u + i];
                        }
                    }
            } else {                                                     // (heads this wide are alone in their wavefront)
                f32x4 sc[X::NU], sp[X::NU];
#pragma unroll
                for (int u = 0; u < X::NU; ++u) sc[u] = sp[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int m0 = 0; m0 < X::KM; m0 += 2) {
                    __builtin_amdgcn_sched_barrier(0);
                    float v[2][X::KC / 4], o[2][X::KC / 4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        columns(q, m0 + h, v[h]);
                        columns(go, m0 + h, o[h]);
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        fragment(qf[0], v[h]);
                        fragment(gf[0], o[h]);
#pragma unroll
                        for (int u = 0; u < X::NU; ++u) {
                            product(kr[u][0][m0 + h], qf[0], sc[u]);
                            product(vr[u][0][m0 + h], gf[0], sp[u]);
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < X::NU; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) c[4 * u + i] = sc[u][i], dp[4 * u + i] = sp[u][i];
            }
            if (e0 + X::ROWS < count) {
                place(e0 + X::ROWS);
                load_rows(e0 + X::ROWS);
                fetch(e0 + 2 * X::ROWS);
            }
            float z[X::PER], bend[X::PER], ds[X::PER], dzs[X::PER];
            if (a.cap > 0) {                                             // (tests of what the call has stay outside the loops over entries)
#pragma unroll
                for (int e = 0; e < X::PER; ++e) {
                    const float t = tanh_few_ulp(c[e] * by_cap);
                    z[e] = a.cap * t;
                    bend[e] = a.scale * fmaxf(fmaf(-t, t, 1.f), 0.f);    // (0 for a NaN, which a row that nobody sees may give; one that is seen has p NaN)
                }
            } else {
#pragma unroll
                for (int e = 0; e < X::PER; ++e) {
                    z[e] = c[e] * a.scale;
                    bend[e] = a.scale;
                }
            }
            if (a.bias) {
#pragma unroll
                for (int e = 0; e < X::PER; ++e) z[e] += table[max(tile[32 + X::PER * g + e], 0) * cols + min(col, cols - 1)];
            }
#pragma unroll
            for (int e = 0; e < X::PER; ++e) {
                const bool in = (seen >> (X::PER * g + e) & 1) && z[e] != -INFINITY;      // (a score of -infinity weighs nothing, also in a bag of them alone)
                const float p = in ? exp_few_ulp(z[e] - lse, shift) : 0.f, dz = in ? p * (dp[e] - against) : 0.f;
                ds[e] = dz * bend[e];
                turn_ds[(X::PER * g + e) * L::WIDE + col] = ds[e];
                turn_p[(X::PER * g + e) * L::WIDE + col] = p;
                dzs[e] = dz;
            }
            if (a.bias) {
                const auto turn_to = [&](int r) {
                    if (r != sum_row) {
                        if (sum_row >= 0) sums[sum_row * 16] += sum_dz;
                        sum_row = r;
                        sum_dz = 0.f;
                    }
                };
                if (one_row >= 0) {
                    turn_to(one_row);
#pragma unroll
                    for (int e = 0; e < X::PER; ++e) sum_dz += dzs[e];
                } else {
#pragma unroll
                    for (int e = 0; e < X::PER; ++e) {
                        const int r = tile[32 + X::PER * g + e];
                        if (r >= 0) {
                            turn_to(r);
                            sum_dz += dzs[e];
                        }
                    }
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            // Gradients of the rows: elements down (four side by side a lane), entries across.  Straight from the registers a store would
            // write 64 bytes of 16 rows each, which memory takes at half the rate of whole rows (400,000 rows of 1 KB: 161 us so, 140 this).
            const auto row_gradients = [&](auto steps) {
                constexpr int N = decltype(steps)::value;
                // a head's gradients of the keys or of the values, added to `to`: from its columns' elements and what the entries have of them
                const auto of_head = [&](const float (&y)[SOME][STEPS], const float* turn, int u, int k, f32x4 (&to)[SOME]) {
                    float x[N];
#pragma unroll
                    for (int t = 0; t < N; ++t) {
                        const bool have = (FULL || k < heads) && 4 * t + g < group;
                        const float v = turn[(16 * u + col) * L::WIDE + (have ? k * group + 4 * t + g : 0)];
                        x[t] = have ? v : 0.f;
                    }
#pragma unroll
                    for (int b = 0; b < SOME; ++b)
#pragma unroll
                        for (int t = 0; t < N; ++t) to[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[b][t], x[t], to[b], 0, 0, 0);
                };
                const auto with_rows = [&](int u, auto&& then) {
                    const int entry = 16 * u + col;
                    float* const rows_at = f.grad_rows + (first + e0 + 16 * u) * a.dim + kv0 * d;
                    const bool blank = !all_seen && !(seen >> entry & 1);
                    const auto zero = [&](f32x4 (&to)[SOME]) {
#pragma unroll
                        for (int b = 0; b < SOME; ++b) to[b] = f32x4{0.f, 0.f, 0.f, 0.f};
                    };
                    const auto to_stage = [&](const f32x4 (&from)[SOME], int at) {
#pragma unroll
                        for (int b = 0; b < SOME; ++b) *reinterpret_cast<f32x4*>(stage + col * L::STAGE_WIDE + at + 16 * b + 4 * g) = from[b];
                    };
                    const auto to_rows = [&](const f32x4 (&from)[SOME], int at, int b0) {
                        if (e0 + entry >= count) return;
#pragma unroll
                        for (int b = 0; b < SOME; ++b)
                            if (FULL || 16 * (b0 + b) + 4 * g < d) *reinterpret_cast<f32x4*>(rows_at + (int64_t)col * a.dim + at + 16 * b + 4 * g) = from[b];
                    };
                    const auto write_rows = [&](auto parts, int at) {
                        constexpr int UNITS = L::STRETCH / 4, EVERY = decltype(parts)::value * UNITS, ROWS_A_TIME = 64 / EVERY, TIMES = 16 / ROWS_A_TIME;      // units of 16 bytes
                        constexpr int AHEAD = TIMES < 4 ? TIMES : 4;
                        static_assert(EVERY <= 64);
                        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                        __builtin_amdgcn_wave_barrier();
                        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                        const int my_row = lane / EVERY, part = lane % EVERY / UNITS, unit = lane % UNITS, left = count - e0 - 16 * u - my_row;
                        const uint32_t lane_at = my_row * a.dim + part * a.value_at + 4 * unit;
                        const float* const from = stage + my_row * L::STAGE_WIDE + part * L::STRETCH + 4 * unit;
#pragma unroll
                        for (int i0 = 0; i0 < TIMES; i0 += AHEAD) {
                            f32x4 v[AHEAD];
#pragma unroll
                            for (int j = 0; j < AHEAD; ++j) v[j] = *reinterpret_cast<const f32x4*>(from + (i0 + j) * ROWS_A_TIME * L::STAGE_WIDE);
#pragma unroll
                            for (int j = 0; j < AHEAD; ++j)
                                if ((i0 + j) * ROWS_A_TIME < left) *reinterpret_cast<f32x4*>(rows_at + at + (int64_t)((i0 + j) * ROWS_A_TIME) * a.dim + lane_at) = v[j];
                        }
                        __builtin_amdgcn_wave_barrier();
                    };
                    then(blank, zero, to_stage, to_rows, write_rows);
                };
                const std::integral_constant<int, 1> one;
                if constexpr (L::APART) {
                    const auto of_part = [&](const float (&y)[SOME][STEPS], const float (&also)[SOME][STEPS], bool values, int b0) {
#pragma unroll
                        for (int u = 0; u < X::NU; ++u)
                            with_rows(u, [&](bool blank, auto zero, auto to_stage, auto to_rows, auto write_rows) {
                                f32x4 of[SOME];
                                zero(of);
                                of_head(y, values ? turn_p : turn_ds, u, 0, of);
                                if (a.value_at == 0) of_head(also, turn_p, u, 0, of);
                                if (blank) zero(of);
                                if constexpr (L::STAGED) {
                                    to_stage(of, 0);
                                    write_rows(one, (values ? a.value_at : 0) + 16 * b0);
                                } else {
                                    to_rows(of, (values ? a.value_at : 0) + 16 * b0, b0);
                                }
                            });
                    };
                    if constexpr (KEEP) {
                        of_part(qt[0], gt[0], false, 0);
                        if (a.value_at) of_part(gt[0], gt[0], true, 0);
                    } else {
#pragma unroll 1
                        for (int b0 = 0; b0 < BLOCKS; b0 += SOME) {
                            float y[SOME][STEPS], also[SOME][STEPS];
#pragma unroll
                            for (int b = 0; b < SOME; ++b)
#pragma unroll
                                for (int t = 0; t < N; ++t) {
                                    y[b][t] = element(a.q, 0, b0 + b, t);
                                    also[b][t] = element(f.grad_out, 0, b0 + b, t);
                                }
                            __builtin_amdgcn_sched_barrier(0);           // all on their way before the first is used
                            of_part(y, also, false, b0);
                            if (a.value_at) of_part(also, also, true, b0);
                        }
                    }
                } else {
#pragma unroll
                    for (int u = 0; u < X::NU; ++u)
                        with_rows(u, [&](bool blank, auto zero, auto to_stage, auto to_rows, auto write_rows) {
#pragma unroll
                            for (int k = 0; k < PACK; ++k) {
                                f32x4 gk[SOME], gv[SOME];
                                zero(gk);
                                zero(gv);
                                of_head(qt[k], turn_ds, u, k, gk);
                                of_head(gt[k], turn_p, u, k, gv);
                                if (!all_seen && blank) {
                                    zero(gk);
                                    zero(gv);
                                }
                                if (a.value_at == 0) {
#pragma unroll
                                    for (int b = 0; b < SOME; ++b) gk[b] += gv[b];
                                }
                                if constexpr (L::STAGED) {
                                    to_stage(gk, k * DP);
                                    if (a.value_at) to_stage(gv, L::STRETCH + k * DP);
                                } else if (FULL || k < heads) {
                                    to_rows(gk, k * d, 0);
                                    if (a.value_at) to_rows(gv, a.value_at + k * d, 0);
                                }
                            }
                            if constexpr (L::STAGED) {
                                if (a.value_at) write_rows(std::integral_constant<int, 2>(), 0);
                                else write_rows(one, 0);
                            }
                        });
                }
            };
            if (STEPS > 1 && group <= 4) row_gradients(std::integral_constant<int, 1>());
            else row_gradients(std::integral_constant<int, STEPS>());
            // of q: as the forward pass pools values
            if (!all_seen) {
#pragma unroll
                for (int e = 0; e < X::PER; ++e)
#pragma unroll
                    for (int m = 0; m < X::MB; ++m) kv[e][m] = masked(kv[e][m], seen >> (X::PER * g + e) & 1 ? ~0u : 0u);
            }
            if constexpr (X::BF16) {
                Split3 df;
                df.set(ds);
#pragma unroll
                for (int m = 0; m < X::MB; ++m)
#pragma unroll
                    for (int j = 0; j < X::VW; ++j) {
                        uint32_t v[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            v[i] = __builtin_amdgcn_perm(word(kv[2 * i + 1][m], j / 2), word(kv[2 * i][m], j / 2), j % 2 ? 0x07060302u : 0x05040100u);
                        const bf16x8 kf = __builtin_bit_cast(bf16x8, make_uint4(v[0], v[1], v[2], v[3]));
#pragma unroll
                        for (int part = 2; part >= 0; --part) dq[m][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, df.part[part], dq[m][j], 0, 0, 0);
                    }
            } else {
#pragma unroll
                for (int e = 0; e < X::PER; ++e)
#pragma unroll
                    for (int m = 0; m < X::MB; ++m)
#pragma unroll
                        for (int j = 0; j < X::VW; ++j)
                            dq[m][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(word(kv[e][m], j)), ds[e], dq[m][j], 0, 0, 0);
            }
        }
        if (blockIdx.y == 0) clear_rest(f, first, count);
        float* const to = (whole ? f.grad_q + ((int64_t)bag * a.q_heads + head) * d
                                 : f.parts + ((2 * (int64_t)share + starts) * a.q_heads + head) * d) - own * d;
#pragma unroll
        for (int m = 0; m < X::MB; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int x = (m * 16 + 4 * g + i) * X::VW;
                float v[X::VW];
#pragma unroll
                for (int j = 0; j < X::VW; ++j) v[j] = dq[m][j][i];
                if (col < cols && x >= own * d && x < (own + 1) * d) __builtin_memcpy(__builtin_assume_aligned(to + x, X::VW >= 4 ? 16 : 4 * X::VW), v, sizeof(v));
            }
    });
    if (!a.bias) return;
    if (sum_row >= 0 && col < cols) sums[sum_row * 16] += sum_dz;
    __syncthreads();
    const float* const all = table + table_rows * cols;
    for (int e = threadIdx.x; e < table_rows * cols; e += kBwdBlock) {
        double sum = 0;
        for (int x = 0; x < kBwdWaves * 4; ++x) sum += all[(x * table_rows + e / cols) * 16 + e % cols];
        f.bias_parts[((int64_t)blockIdx.x * table_rows + e / cols) * a.q_heads + first_head + e % cols] = sum;
    }
}

// One query head a kv head, and rows that are their own values, without the matrix instructions, as in the forward pass: a lane holds 16
// bytes of a row and writes their gradients, rows side by side.  (8,192 bags of up to 50 rows, 4 heads of 16: 40 us in fp32 and 29 in
// bf16, through the matrix instructions 63 and 108.)
template <typename T, int LANES>
__global__ __launch_bounds__(kBwdBlock, kNarrowGroups) void embbag_attn_bwd_narrow_kernel(BwdArgs f) {
    extern __shared__ float lds[];
    constexpr int kSteps = 4;
    typedef Narrow<T, LANES> N;
    const AttnArgs& a = f.a;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int width = a.kv_heads * LANES, r = lane / width, head = lane % width / LANES, at = lane % LANES * N::VE;
    const int side = 64 / width, d = N::D, heads = a.q_heads, table_rows = a.bias ? a.rp.rows() : 0;
    int32_t* const borders = (int32_t*)lds;
    float* const table = lds + 64;
    float* const all_sums = table + table_rows * heads;                  // [wavefront][row side by side][table row][head]
    float* const sums = all_sums + (wave * side + r) * table_rows * heads + head;
    if (a.bias) {
        if (threadIdx.x < BP_RELPOS_MAX_BUCKETS) borders[threadIdx.x] = a.rp.borders[threadIdx.x];
        for (int e = threadIdx.x; e < table_rows * heads; e += kBwdBlock) table[e] = a.bias[e];
        for (int e = threadIdx.x; e < kBwdWaves * side * table_rows * heads; e += kBwdBlock) all_sums[e] = 0.f;
        __syncthreads();
    }
    const T* const w = (const T*)a.cache_w + (int64_t)head * d + at;
    const float by_cap = a.cap > 0 ? a.scale / a.cap : 0.f;
    const uint32_t share = blockIdx.x * kBwdWaves + wave;
    for_own_bags(f, share, [&](uint32_t bag, int64_t first, int count, bool whole, bool starts) {
        const int64_t place = ((int64_t)bag * heads + head) * d + at;
        float q[N::VE], go[N::VE], out[N::VE], dq[N::VE];
        N::read(a.q + place, q);
        N::read(f.grad_out + place, go);
        N::read(f.out + place, out);
        const float lse = f.lse[(int64_t)bag * heads + head], against = N::dot(go, out);
        float shift = 0.f;
        if (a.bias && __any(far_lse(lse))) {                             // (the scores add up as below, so their size does not matter)
            const Again b = arguments_again();
            const BagSpan span = bag_span(a, bag);
            float sum = 0.f;
#pragma unroll 1
            for (int64_t e = r; e < span.count; e += side) {
                const int32_t slot = b->slots[span.first + e];
                if ((uint32_t)slot >= (uint64_t)b->C) continue;
                const int row_of = relpos_row((int64_t)b->q_pos[bag] - b->lookup_pos[span.first + e], borders, b->rp.buckets, b->rp.two_sided);
                if (row_of < 0) continue;
                float v[N::VE];
                N::widen(*reinterpret_cast<const uint4*>((const T*)b->cache_w + (int64_t)slot * b->wst + (int64_t)head * d + at), v);
                float z = N::dot(q, v);
                z = (b->cap > 0 ? b->cap * tanh_few_ulp(z * (b->scale / b->cap)) : z * b->scale) + table[row_of * heads + head];
                if (z != -INFINITY) sum += exp_few_ulp(z - lse);
            }
            for (int off = width; off < 64; off <<= 1) sum += __shfl_xor(sum, off);
            if (far_lse(lse)) shift = shift_of(sum);
        }
        const int64_t q_pos = a.bias ? a.q_pos[bag] : 0;
#pragma unroll
        for (int i = 0; i < N::VE; ++i) dq[i] = 0.f;
        int32_t slot_n = -1, pos_n = 0;
        const auto fetch = [&](int e) {
            slot_n = e + lane < count ? a.slots[first + e + lane] : -1;
            pos_n = e + lane < count && a.bias ? a.lookup_pos[first + e + lane] : 0;
        };
        fetch(0);
        for (int e0 = 0; e0 < count; e0 += 64) {
            int row_of = -1;
            if ((uint32_t)slot_n < (uint64_t)a.C) row_of = a.bias ? relpos_row(q_pos - pos_n, borders, a.rp.buckets, a.rp.two_sided) : 0;
            const int slot = row_of >= 0 ? slot_n : 0, here = min(64, count - e0);
            if (e0 + 64 < count) fetch(e0 + 64);
            for (int s0 = 0; s0 < here; s0 += kSteps * side) {
                uint4 raw[kSteps];
                int row[kSteps];
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    const int e = s0 + s * side + r;                     // (behind the 64th: an entry that is not there)
                    row[s] = __shfl(row_of, e & 63);
                    if (e >= here) row[s] = -1;
                    const T* const from = w + (int64_t)__shfl(slot, e & 63) * a.wst;
                    if (s0 + s * side < here) raw[s] = *reinterpret_cast<const uint4*>(from);
                }
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    if (s0 + s * side >= here) break;
                    float v[N::VE], grad[N::VE];
                    N::widen(masked(raw[s], row[s] >= 0 ? ~0u : 0u), v);
                    float z = N::dot(q, v), bend = a.scale;
                    if (a.cap > 0) {
                        const float t = tanh_few_ulp(z * by_cap);
                        z = a.cap * t;
                        bend = a.scale * fmaxf(fmaf(-t, t, 1.f), 0.f);
                    } else {
                        z *= a.scale;
                    }
                    if (a.bias) z += table[max(row[s], 0) * heads + head];
                    const float dp = N::dot(go, v);
                    const bool in = row[s] >= 0 && z != -INFINITY;       // (as in the kernel above; both dots add in the same order)
                    const float p = in ? exp_few_ulp(z - lse, shift) : 0.f, dz = in ? p * (dp - against) : 0.f, ds = dz * bend;
                    if (a.bias && at == 0 && row[s] >= 0) sums[row[s] * heads] += dz;
#pragma unroll
                    for (int i = 0; i < N::VE; ++i) {
                        grad[i] = row[s] >= 0 ? fmaf(ds, q[i], p * go[i]) : 0.f;
                        dq[i] = fmaf(ds, v[i], dq[i]);
                    }
                    if (s0 + s * side + r < here) N::write(f.grad_rows + (first + e0 + s0 + s * side + r) * a.dim + head * d + at, grad);
                }
            }
        }
        clear_rest(f, first, count);
        for (int off = width; off < 64; off <<= 1)
#pragma unroll
            for (int i = 0; i < N::VE; ++i) dq[i] += __shfl_xor(dq[i], off);
        if (r == 0) N::write((whole ? f.grad_q + place : f.parts + ((2 * (int64_t)share + starts) * heads + head) * d + at), dq);
    });
    if (!a.bias) return;
    __syncthreads();
    for (int e = threadIdx.x; e < table_rows * heads; e += kBwdBlock) {
        double sum = 0;
        for (int x = 0; x < kBwdWaves * side; ++x) sum += all_sums[x * table_rows * heads + e];
        f.bias_parts[(int64_t)blockIdx.x * table_rows * heads + e] = sum;
    }
}

// grad_q of the bags that several wavefronts had a part of.  Workgroups look through `each` bags for such bags.  Up to kFewParts
// parts: one workgroup, four elements a thread; more: a workgroup 64 elements, 16 parts of them side by side.
constexpr int kJoinBlock = 256, kShare = 64, kFewParts = 8;
__global__ __launch_bounds__(kJoinBlock) void embbag_attn_bwd_join_kernel(BwdArgs f, int each) {
    __shared__ float4 part[kJoinBlock];
    const AttnArgs& a = f.a;
    const int width = a.q_heads * a.d, lane = threadIdx.x % 64;
    const int64_t bag0 = (int64_t)(blockIdx.z * gridDim.x + blockIdx.x) * each, mine = bag0 + lane;
    const auto parts_of = [&](uint32_t bag, uint32_t* first) -> uint32_t {
        const uint32_t from = first_unit(a, bag), units = max(1u, (uint32_t)((bag_span(a, bag).count + kUnit - 1) >> kUnitShift));
        *first = share_of(from, f.units, f.waves);
        return share_of(min(from + units, f.units) - 1, f.units, f.waves) - *first + 1;
    };
    uint32_t my_first = 0, my_of = 0;
    if (lane < each && mine < a.bags) my_of = parts_of((uint32_t)mine, &my_first);
    const auto add = [](float4& v, const float4& x) { v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w; };
    for (uint64_t several = __ballot(my_of > 1); several; several &= several - 1) {
        const int which = __ffsll((unsigned long long)several) - 1;
        const uint32_t bag = (uint32_t)(bag0 + which), of = __shfl(my_of, which), first = __shfl(my_first, which);
        const auto from = [&](uint32_t i, int at) { return *reinterpret_cast<const float4*>(f.parts + (2 * (int64_t)(first + i) + (i == 0)) * width + at); };
        float* const to = f.grad_q + (int64_t)bag * width;
        if (of <= kFewParts) {
            if (blockIdx.y > 0) continue;
            for (int at = 4 * threadIdx.x; at < width; at += 4 * kJoinBlock) {
                float4 v = from(0, at);
#pragma unroll
                for (uint32_t i = 1; i < kFewParts; ++i)
                    if (i < of) add(v, from(i, at));
                *reinterpret_cast<float4*>(to + at) = v;
            }
            continue;
        }
        const int at = blockIdx.y * kShare + threadIdx.x % 16 * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (uint32_t i = threadIdx.x / 16; i < of && at < width; i += kJoinBlock / 16) add(v, from(i, at));
        part[threadIdx.x] = v;
        __syncthreads();
        if (threadIdx.x < 16 && at < width) {
            for (int i = 1; i < kJoinBlock / 16; ++i) add(v, part[16 * i + threadIdx.x]);
            *reinterpret_cast<float4*>(to + at) = v;
        }
        __syncthreads();
    }
}

// grad_bias from the workgroups' parts: 16 elements of the table a workgroup, 64 parts of them side by side
constexpr int kBiasJoinBlock = 1024;
__global__ __launch_bounds__(kBiasJoinBlock) void embbag_attn_bias_join_kernel(const double* __restrict__ parts, int count, int groups, float* __restrict__ grad_bias) {
    __shared__ double part[kBiasJoinBlock / 16][16];
    const int c = threadIdx.x % 16, e = blockIdx.x * 16 + c, share = threadIdx.x / 16;
    double sum = 0;
    if (e < count) {
#pragma unroll 4
        for (int x = share; x < groups; x += kBiasJoinBlock / 16) sum += parts[(int64_t)x * count + e];
    }
    part[share][c] = sum;
    __syncthreads();
    if (share == 0 && e < count) {
        for (int x = 1; x < kBiasJoinBlock / 16; ++x) sum += part[x][c];
        grad_bias[e] = (float)sum;
    }
}

struct BwdPlan {
    int dp, pack, chunks;
    uint32_t units, waves, groups;
    bool narrow;
    BwdPlan(const bp_attn* at, int dtype, int64_t n, int64_t bags) {
        narrow = attn_narrow(at, dtype);
        dp = attn_dp(at, dtype);
        pack = attn_pack(at, dp);
        chunks = narrow ? 1 : (at->kv_heads + pack - 1) / pack;
        units = (uint32_t)((n >> kUnitShift) + bags);
        // what the chip holds at once, or shares of kMostUnits
        const int64_t held = std::max(1, 256 * kBwdWaves * (narrow ? kNarrowGroups : bwd_groups_a_cu(elem_bytes(dtype), dp, dp * pack)) / chunks);
        waves = (uint32_t)std::min<int64_t>(units, std::max<int64_t>(held, ceil_div(units, kMostUnits)));
        groups = (waves + kBwdWaves - 1) / kBwdWaves;
    }
};

struct BwdScratch {
    float* parts;
    double* bias_parts;
    size_t bytes;
    BwdScratch(void* ws, const BwdPlan& l, const bp_attn* at, int table_rows) {
        Carver c(ws, 0);
        parts = c.take<float>((size_t)2 * l.waves * at->q_heads * at->head_dim);
        bias_parts = c.take<double>((size_t)l.groups * table_rows * at->q_heads);
        bytes = c.used();
    }
};

constexpr size_t kLdsMost = 160 << 10;            // of a workgroup
struct BwdLaunch {
    const BwdArgs& f;
    const BwdPlan& l;
    hipStream_t stream;
    template <typename T, int DP, int PACK, bool FULL>
    int run() {
        const int cols = std::min(PACK, f.a.kv_heads) * (f.a.q_heads / f.a.kv_heads);
        const size_t shared = BwdLds<T, DP, PACK, FULL>::floats(f.a.bias ? f.a.rp.rows() : 0, cols) * 4;
        if constexpr (FULL) {
            if (shared > kLdsMost) return run<T, DP, PACK, false>();     // the largest tables leave no room for whole rows
        }
        BP_LAUNCH(K_ATTN_BWD, (embbag_attn_bwd_kernel<T, DP, PACK, FULL>), dim3(l.groups, (unsigned)l.chunks), dim3(kBwdBlock), shared, stream, f);
        return BP_OK;
    }
    template <typename T, int LANES>
    int run_narrow() {
        const size_t shared = (64 + (f.a.bias ? (size_t)f.a.rp.rows() * (f.a.q_heads + kBwdWaves * 64 / LANES) : 0)) * 4;
        BP_LAUNCH(K_ATTN_BWD, (embbag_attn_bwd_narrow_kernel<T, LANES>), dim3(l.groups), dim3(kBwdBlock), shared, stream, f);
        return BP_OK;
    }
    template <typename T>
    int start() {
        return l.narrow ? dispatch_narrow<T>(f.a, *this) : dispatch_attn<T>(f.a, l.dp, l.pack, *this);
    }
};

}  // namespace
}  // namespace bp

using namespace bp;

BP_EXPORT int bp_embbag_attn_bwd_workspace_bytes(const bp_config* cfg, const bp_attn* at, const bp_relpos* rp, int64_t n_lookups, int64_t bags,
                                                 size_t* bytes) {
    Relpos r;
    BP_TRY(attn_check_shape(cfg, at));
    BP_TRY(attn_check_sizes(n_lookups, bags, bytes));
    if (rp) BP_TRY(check_relpos(rp, &r));
    *bytes = BwdScratch(nullptr, BwdPlan(at, cfg->weight_dtype, n_lookups, bags), at, rp ? r.rows() : 0).bytes;
    return BP_OK;
}

BP_EXPORT int bp_embbag_attn_bwd(const bp_config* cfg, const bp_attn* at, const bp_relpos* rp, const void* cache_w, const int32_t* lookup_slots,
                                 const int64_t* bag_offsets, const int32_t* bag_lengths, int64_t n_lookups, int64_t bags, const float* q,
                                 const int32_t* q_pos, const int32_t* lookup_pos, const float* bias_table, const float* out, const float* lse,
                                 const float* grad_out, float* grad_q, float* grad_rows, float* grad_bias, void* workspace,
                                 size_t workspace_bytes, void* stream_) {
    BwdArgs f{};
    size_t need = 0;
    hipStream_t stream = (hipStream_t)stream_;
    BP_TRY(attn_check(cfg, at, rp, cache_w, lookup_slots, bag_offsets, bag_lengths, n_lookups, bags, q, q_pos, lookup_pos, bias_table, &f.a));
    if ((rp != nullptr) != (grad_bias != nullptr)) return fail(BP_ERR_INVALID_ARG, "grad_bias goes with rp");
    if (bags && (!out || !lse || !grad_out || !grad_q || (n_lookups && !grad_rows))) return fail(BP_ERR_INVALID_ARG, "NULL pointer");
    if ((((uintptr_t)out | (uintptr_t)grad_out | (uintptr_t)grad_q | (uintptr_t)grad_rows) & 15) || (((uintptr_t)lse | (uintptr_t)grad_bias) & 3))
        return fail(BP_ERR_INVALID_ARG, "out, grad_out, grad_q and grad_rows must be 16-byte aligned, lse and grad_bias aligned to their elements");
    BP_TRY(bp_embbag_attn_bwd_workspace_bytes(cfg, at, rp, n_lookups, bags, &need));
    BP_TRY(attn_check_workspace(workspace, workspace_bytes, need));
    const BwdPlan l(at, cfg->weight_dtype, n_lookups, bags);
    const int table_rows = rp ? f.a.rp.rows() : 0, count = table_rows * at->q_heads;
    const BwdScratch w(workspace, l, at, table_rows);
    f.out = out;
    f.lse = lse;
    f.grad_out = grad_out;
    f.grad_q = grad_q;
    f.grad_rows = grad_rows;
    f.units = l.units;
    f.waves = l.waves;
    f.parts = w.parts;
    f.bias_parts = w.bias_parts;
    if (bags) {
        BwdLaunch launch{f, l, stream};
        BP_TRY(cfg->weight_dtype == BP_F32 ? launch.start<float>() : launch.start<uint16_t>());
        if (l.waves > 1) {
            const int64_t shares = ceil_div((int64_t)at->q_heads * at->head_dim, kShare);
            const int64_t each = std::min(std::max<int64_t>(bags * shares / 8192, 1), (int64_t)64);
            BP_LAUNCH(K_ATTN_JOIN, embbag_attn_bwd_join_kernel, spread_grid(ceil_div(bags, each), (unsigned)shares), dim3(kJoinBlock), 0, stream, f,
                      (int)each);
        }
    }
    if (rp)
        BP_LAUNCH(K_ATTN_JOIN, embbag_attn_bias_join_kernel, dim3((unsigned)ceil_div(count, 16)), dim3(kBiasJoinBlock), 0, stream, w.bias_parts, count,
                  bags ? (int)l.groups : 0, grad_bias);
    return BP_OK;
}
