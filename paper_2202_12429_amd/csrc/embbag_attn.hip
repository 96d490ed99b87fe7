// bp_embbag_attn_fwd / bp_embbag_attn_bwd: bags pooled by attention over their cached rows.
#include <algorithm>
#include <cmath>

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

namespace {

// The table row of an entry's distance: -1 when it is not seen, 0 where no bias is asked for.
__device__ __forceinline__ int entry_row(const AttnArgs& a, int64_t bag, int64_t k, const int32_t* borders) {
    if ((uint32_t)a.slots[k] >= (uint64_t)a.C) return -1;
    if (!a.bias) return 0;
    return relpos_row((int64_t)a.q_pos[bag] - a.lookup_pos[k], borders, a.rp.buckets, a.rp.two_sided);
}

constexpr int kAttnBlock = 256;
constexpr int kMaxQHeads = 1024;

// A workgroup a bag: scores to the workspace, softmax head by head, then weights and pooled rows.
template <typename T>
__global__ __launch_bounds__(kAttnBlock) void embbag_attn_fwd_kernel(AttnArgs a, float* __restrict__ scores, float* __restrict__ out,
                                                                     float* __restrict__ lse, const float* weight_in, float* weight_out) {
    __shared__ int32_t borders[BP_RELPOS_MAX_BUCKETS];
    __shared__ float norm[kMaxQHeads];
    if (threadIdx.x < BP_RELPOS_MAX_BUCKETS) borders[threadIdx.x] = a.rp.borders[threadIdx.x];
    __syncthreads();
    const int64_t bag = blockIdx.x;
    const BagSpan s = bag_span(a, bag);
    const T* const w = (const T*)a.cache_w;
    const int hq = a.q_heads, group = hq / a.kv_heads;
    for (int64_t e = threadIdx.x; e < s.count * hq; e += kAttnBlock) {
        const int64_t k = s.first + e / hq;
        const int h = (int)(e % hq);
        const int row = entry_row(a, bag, k, borders);
        float c = -INFINITY;
        if (row >= 0) {
            const T* const key = w + a.slots[k] * a.wst + (h / group) * a.d;
            const float* const q = a.q + (bag * hq + h) * a.d;
            float dot = 0.f;
            for (int i = 0; i < a.d; ++i) dot = fmaf(q[i], row_value(key, i), dot);
            c = a.scale * dot;
            if (a.cap > 0) c = a.cap * tanhf(c / a.cap);
            if (a.bias) c += a.bias[row * hq + h];
        }
        scores[k * hq + h] = c;
    }
    __syncthreads();
    for (int h = threadIdx.x / 64; h < hq; h += kAttnBlock / 64) {
        const int lane = threadIdx.x % 64;
        float top = -INFINITY;
        for (int64_t e = lane; e < s.count; e += 64) top = fmaxf(top, scores[(s.first + e) * hq + h]);
        for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
        if (top == -INFINITY) top = 0.f;
        float sum = 0.f;
        for (int64_t e = lane; e < s.count; e += 64) sum += expf(scores[(s.first + e) * hq + h] - top);
        for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off);
        if (lane == 0) {
            norm[h] = sum == 0.f ? 0.f : top + logf(sum);            // nothing seen: every weight below is exp(-inf)
            lse[bag * hq + h] = sum == 0.f ? -INFINITY : top + logf(sum);
        }
    }
    __syncthreads();
    if (weight_out)
        for (int64_t e = threadIdx.x; e < s.count; e += kAttnBlock) {
            const int64_t k = s.first + e;
            float sum = 0.f;
            for (int h = 0; h < hq; ++h) sum += expf(scores[k * hq + h] - norm[h]);
            weight_out[k] = (weight_in ? weight_in[k] : 0.f) + sum;
        }
    for (int t = threadIdx.x; t < hq * a.d; t += kAttnBlock) {
        const int h = t / a.d, i = t % a.d;
        float sum = 0.f;
        for (int64_t k = s.first; k < s.first + s.count; ++k) {
            const float c = scores[k * hq + h];
            if (c == -INFINITY) continue;                            // an entry that is not seen is not read
            sum = fmaf(expf(c - norm[h]), row_value(w + a.slots[k] * a.wst + a.value_at + (h / group) * a.d, i), sum);
        }
        out[bag * hq * a.d + t] = sum;
    }
}

// A workgroup a bag: p and the gradient of the scores to the workspace, then the gradients that they are summed into.
template <typename T>
__global__ __launch_bounds__(kAttnBlock) void embbag_attn_bwd_kernel(AttnArgs a, const float* __restrict__ out, const float* __restrict__ lse,
                                                                     const float* __restrict__ grad_out, float* __restrict__ ps,
                                                                     float* __restrict__ dzs, int32_t* __restrict__ rows,
                                                                     float* __restrict__ grad_q, float* __restrict__ grad_rows) {
    __shared__ int32_t borders[BP_RELPOS_MAX_BUCKETS];
    __shared__ float against[kMaxQHeads];
    if (threadIdx.x < BP_RELPOS_MAX_BUCKETS) borders[threadIdx.x] = a.rp.borders[threadIdx.x];
    const int64_t bag = blockIdx.x;
    const BagSpan s = bag_span(a, bag);
    const T* const w = (const T*)a.cache_w;
    const int hq = a.q_heads, group = hq / a.kv_heads;
    for (int h = threadIdx.x; h < hq; h += kAttnBlock) {
        float sum = 0.f;
        for (int i = 0; i < a.d; ++i) sum = fmaf(grad_out[(bag * hq + h) * a.d + i], out[(bag * hq + h) * a.d + i], sum);
        against[h] = sum;
    }
    __syncthreads();
    for (int64_t e = threadIdx.x; e < s.count * hq; e += kAttnBlock) {
        const int64_t k = s.first + e / hq;
        const int h = (int)(e % hq);
        const int row = entry_row(a, bag, k, borders);
        if (h == 0) rows[k] = row;
        float p = 0.f, dz = 0.f, ds = 0.f;
        if (row >= 0) {
            const T* const key = w + a.slots[k] * a.wst + (h / group) * a.d;
            const T* const val = key + a.value_at;
            const float* const q = a.q + (bag * hq + h) * a.d;
            const float* const g = grad_out + (bag * hq + h) * a.d;
            float dot = 0.f, dp = 0.f;
            for (int i = 0; i < a.d; ++i) {
                dot = fmaf(q[i], row_value(key, i), dot);
                dp = fmaf(g[i], row_value(val, i), dp);
            }
            float c = a.scale * dot, bend = 1.f;
            if (a.cap > 0) {
                const float t = tanhf(c / a.cap);
                c = a.cap * t;
                bend = 1.f - t * t;
            }
            if (a.bias) c += a.bias[row * hq + h];
            p = c == -INFINITY ? 0.f : expf(c - lse[bag * hq + h]);
            dz = p * (dp - against[h]);
            ds = dz * bend * a.scale;
        }
        ps[k * hq + h] = p;
        dzs[(k * hq + h) * 2] = dz;
        dzs[(k * hq + h) * 2 + 1] = ds;
    }
    __syncthreads();
    for (int t = threadIdx.x; t < hq * a.d; t += kAttnBlock) {
        const int h = t / a.d, i = t % a.d;
        float sum = 0.f;
        for (int64_t k = s.first; k < s.first + s.count; ++k)
            if (rows[k] >= 0) sum = fmaf(dzs[(k * hq + h) * 2 + 1], row_value(w + a.slots[k] * a.wst + (h / group) * a.d, i), sum);
        grad_q[bag * hq * a.d + t] = sum;
    }
    const int span = a.kv_heads * a.d;
    for (int64_t t = threadIdx.x; t < s.count * a.dim; t += kAttnBlock) {
        const int64_t k = s.first + t / a.dim;
        const int i = (int)(t % a.dim);
        float sum = 0.f;
        if (rows[k] >= 0) {
            if (i < span)
                for (int h = i / a.d * group; h < (i / a.d + 1) * group; ++h)
                    sum = fmaf(dzs[(k * hq + h) * 2 + 1], a.q[(bag * hq + h) * a.d + i % a.d], sum);
            const int v = i - a.value_at;
            if (v >= 0 && v < span)
                for (int h = v / a.d * group; h < (v / a.d + 1) * group; ++h)
                    sum = fmaf(ps[k * hq + h], grad_out[(bag * hq + h) * a.d + v % a.d], sum);
        }
        grad_rows[k * a.dim + i] = sum;
    }
}

__global__ __launch_bounds__(256) void attn_clear_rows_kernel(int32_t* __restrict__ rows, int64_t n) {
    const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (k < n) rows[k] = -1;
}

// Table gradient of one head over one share of the entries: a column a lane, so that no two lanes meet.
constexpr int kBiasShares = 256;
__global__ __launch_bounds__(64) void attn_bias_grad_kernel(const float* __restrict__ dzs, const int32_t* __restrict__ rows, int64_t n, int hq,
                                                            int table_rows, double* __restrict__ partial) {
    __shared__ float sums[2 * BP_RELPOS_MAX_BUCKETS][64];
    const int lane = threadIdx.x, h = blockIdx.y;
    for (int r = 0; r < table_rows; ++r) sums[r][lane] = 0.f;
    const int64_t share = (n + kBiasShares - 1) / kBiasShares;
    for (int64_t k = blockIdx.x * share + lane; k < min(n, (blockIdx.x + 1) * share); k += 64) {
        const int r = rows[k];
        if (r >= 0) sums[r][lane] += dzs[(k * hq + h) * 2];
    }
    __syncthreads();
    for (int r = lane; r < table_rows; r += 64) {
        double sum = 0;
        for (int j = 0; j < 64; ++j) sum += sums[r][j];
        partial[((int64_t)blockIdx.x * table_rows + r) * hq + h] = sum;
    }
}

__global__ __launch_bounds__(256) void attn_bias_join_kernel(const double* __restrict__ partial, int count, float* __restrict__ grad_bias) {
    const int e = blockIdx.x * 256 + threadIdx.x;
    if (e >= count) return;
    double sum = 0;
    for (int s = 0; s < kBiasShares; ++s) sum += partial[(int64_t)s * count + e];
    grad_bias[e] = (float)sum;
}

struct BwdScratch {
    float *ps, *dzs;
    int32_t* rows;
    double* partial;
    size_t bytes;
    BwdScratch(void* ws, int64_t n, int hq, int table_rows) {
        Carver c(ws, 0);
        ps = c.take<float>((size_t)n * hq);
        dzs = c.take<float>((size_t)n * hq * 2);
        rows = c.take<int32_t>((size_t)n);
        partial = c.take<double>((size_t)kBiasShares * table_rows * hq);
        bytes = c.used();
    }
};

int check_workspace(const void* workspace, size_t have, size_t need) {
    if (need && (!workspace || ((uintptr_t)workspace & 255))) return fail(BP_ERR_INVALID_ARG, "workspace NULL or not 256-byte aligned");
    if (have < need) return fail(BP_ERR_WORKSPACE_TOO_SMALL, "workspace %zu < required %zu bytes", have, need);
    return BP_OK;
}
int check_sizes(int64_t n, int64_t bags, size_t* bytes) {
    if (!bytes) return fail(BP_ERR_INVALID_ARG, "bytes is NULL");
    if (bags < 0 || n < 0) return fail(BP_ERR_INVALID_ARG, "negative size");
    if (bags >= (int64_t(1) << 31) || n >= (int64_t(1) << 31)) return fail(BP_ERR_UNSUPPORTED, "size >= 2^31");
    return BP_OK;
}

}  // namespace
}  // namespace bp

using namespace bp;

BP_EXPORT int bp_embbag_attn_fwd_workspace_bytes(const bp_config* cfg, const bp_attn* at, int64_t n_lookups, int64_t bags,
                                                 int32_t with_weights, size_t* bytes) {
    BP_TRY(attn_check_shape(cfg, at));
    BP_TRY(check_sizes(n_lookups, bags, bytes));
    *bytes = (size_t)n_lookups * at->q_heads * sizeof(float);
    return BP_OK;
}

BP_EXPORT int bp_embbag_attn_fwd(const bp_config* cfg, const bp_attn* at, const bp_relpos* rp, const void* cache_w, const int32_t* lookup_slots,
                                 const int64_t* bag_offsets, const int32_t* bag_lengths, int64_t n_lookups, int64_t bags, const float* q,
                                 const int32_t* q_pos, const int32_t* lookup_pos, const float* bias_table, float* out, float* lse,
                                 const float* weight_in, float* weight_out, void* workspace, size_t workspace_bytes, void* stream) {
    AttnArgs a;
    size_t need = 0;
    BP_TRY(attn_check(cfg, at, rp, cache_w, lookup_slots, bag_offsets, bag_lengths, n_lookups, bags, q, q_pos, lookup_pos, bias_table, &a));
    if (weight_in && !weight_out) return fail(BP_ERR_INVALID_ARG, "weight_in without weight_out");
    if (bags == 0) return BP_OK;
    if (!out || !lse) return fail(BP_ERR_INVALID_ARG, "NULL pointer");
    if (((uintptr_t)out & 15) || (((uintptr_t)lse | (uintptr_t)weight_in | (uintptr_t)weight_out) & 3))
        return fail(BP_ERR_INVALID_ARG, "out must be 16-byte aligned, lse and the weights aligned to their elements");
    BP_TRY(bp_embbag_attn_fwd_workspace_bytes(cfg, at, n_lookups, bags, weight_out != nullptr, &need));
    BP_TRY(check_workspace(workspace, workspace_bytes, need));
    const dim3 grid((unsigned)bags), block(kAttnBlock);
    if (cfg->weight_dtype == BP_F32)
        BP_LAUNCH(K_ATTN_FWD, embbag_attn_fwd_kernel<float>, grid, block, 0, (hipStream_t)stream, a, (float*)workspace, out, lse, weight_in, weight_out);
    else
        BP_LAUNCH(K_ATTN_FWD, embbag_attn_fwd_kernel<uint16_t>, grid, block, 0, (hipStream_t)stream, a, (float*)workspace, out, lse, weight_in,
                  weight_out);
    return BP_OK;
}

BP_EXPORT int bp_embbag_attn_bwd_workspace_bytes(const bp_config* cfg, const bp_attn* at, const bp_relpos* rp, int64_t n_lookups, int64_t bags,
                                                 size_t* bytes) {
    Relpos r;
    BP_TRY(attn_check_shape(cfg, at));
    BP_TRY(check_sizes(n_lookups, bags, bytes));
    if (rp) BP_TRY(check_relpos(rp, &r));
    *bytes = BwdScratch(nullptr, n_lookups, at->q_heads, rp ? r.rows() : 0).bytes;
    return BP_OK;
}

BP_EXPORT int bp_embbag_attn_bwd(const bp_config* cfg, const bp_attn* at, const bp_relpos* rp, const void* cache_w, const int32_t* lookup_slots,
                                 const int64_t* bag_offsets, const int32_t* bag_lengths, int64_t n_lookups, int64_t bags, const float* q,
                                 const int32_t* q_pos, const int32_t* lookup_pos, const float* bias_table, const float* out, const float* lse,
                                 const float* grad_out, float* grad_q, float* grad_rows, float* grad_bias, void* workspace,
                                 size_t workspace_bytes, void* stream_) {
    AttnArgs a;
    size_t need = 0;
    hipStream_t stream = (hipStream_t)stream_;
    BP_TRY(attn_check(cfg, at, rp, cache_w, lookup_slots, bag_offsets, bag_lengths, n_lookups, bags, q, q_pos, lookup_pos, bias_table, &a));
    if ((rp != nullptr) != (grad_bias != nullptr)) return fail(BP_ERR_INVALID_ARG, "grad_bias goes with rp");
    if (bags && (!out || !lse || !grad_out || !grad_q || (n_lookups && !grad_rows))) return fail(BP_ERR_INVALID_ARG, "NULL pointer");
    if ((((uintptr_t)out | (uintptr_t)grad_out | (uintptr_t)grad_q | (uintptr_t)grad_rows) & 15) || (((uintptr_t)lse | (uintptr_t)grad_bias) & 3))
        return fail(BP_ERR_INVALID_ARG, "out, grad_out, grad_q and grad_rows must be 16-byte aligned, lse and grad_bias aligned to their elements");
    BP_TRY(bp_embbag_attn_bwd_workspace_bytes(cfg, at, rp, n_lookups, bags, &need));
    BP_TRY(check_workspace(workspace, workspace_bytes, need));
    const int table_rows = rp ? a.rp.rows() : 0;
    const BwdScratch w(workspace, n_lookups, a.q_heads, table_rows);
    if (n_lookups)
        BP_LAUNCH(K_FILL, attn_clear_rows_kernel, dim3((unsigned)ceil_div(n_lookups, 256)), dim3(256), 0, stream, w.rows, n_lookups);
    if (bags) {
        const dim3 grid((unsigned)bags), block(kAttnBlock);
        if (cfg->weight_dtype == BP_F32)
            BP_LAUNCH(K_ATTN_BWD, embbag_attn_bwd_kernel<float>, grid, block, 0, stream, a, out, lse, grad_out, w.ps, w.dzs, w.rows, grad_q, grad_rows);
        else
            BP_LAUNCH(K_ATTN_BWD, embbag_attn_bwd_kernel<uint16_t>, grid, block, 0, stream, a, out, lse, grad_out, w.ps, w.dzs, w.rows, grad_q,
                      grad_rows);
    }
    if (rp) {
        const int count = table_rows * a.q_heads;
        BP_LAUNCH(K_ATTN_JOIN, attn_bias_grad_kernel, dim3(kBiasShares, (unsigned)a.q_heads), dim3(64), 0, stream, w.dzs, w.rows, n_lookups,
                  a.q_heads, table_rows, w.partial);
        BP_LAUNCH(K_ATTN_JOIN, attn_bias_join_kernel, dim3((unsigned)ceil_div(count, 256)), dim3(256), 0, stream, w.partial, count, grad_bias);
    }
    return BP_OK;
}
