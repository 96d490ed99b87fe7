// bp_embbag_attn_bwd: the gradients of bags pooled by attention over their cached rows.
#include <algorithm>
#include <cmath>

#include "attn_args.h"

namespace bp {
namespace {

// The table row of an entry's distance: -1 when it is not seen, 0 where no bias is asked for.
__device__ __forceinline__ int entry_row(const AttnArgs& a, int64_t bag, int64_t k, const int32_t* borders) {
    if ((uint32_t)a.slots[k] >= (uint64_t)a.C) return -1;
    if (!a.bias) return 0;
    return relpos_row((int64_t)a.q_pos[bag] - a.lookup_pos[k], borders, a.rp.buckets, a.rp.two_sided);
}

constexpr int kAttnBlock = 256;
constexpr int kMaxQHeads = 1024;

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

}  // namespace
}  // namespace bp

using namespace bp;

BP_EXPORT int bp_embbag_attn_bwd_workspace_bytes(const bp_config* cfg, const bp_attn* at, const bp_relpos* rp, int64_t n_lookups, int64_t bags,
                                                 size_t* bytes) {
    Relpos r;
    BP_TRY(attn_check_shape(cfg, at));
    BP_TRY(attn_check_sizes(n_lookups, bags, bytes));
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
    BP_TRY(attn_check_workspace(workspace, workspace_bytes, need));
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
