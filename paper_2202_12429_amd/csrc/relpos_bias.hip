// Bias by distance: out[h, i, j] = table[row((q_start + i) - j)][h], its gradient and the step on the table.
#include <algorithm>
#include <cmath>
#include <vector>

#include "common.h"
#include "relpos.h"
#include "row_access.h"

namespace bp {

int check_relpos(const bp_relpos* rp, Relpos* out) {
    if (!rp) return fail(BP_ERR_INVALID_ARG, "rp is NULL");
    if (rp->buckets < 1 || rp->buckets > BP_RELPOS_MAX_BUCKETS)
        return fail(BP_ERR_INVALID_ARG, "buckets %d outside [1, %d]", rp->buckets, BP_RELPOS_MAX_BUCKETS);
    if (rp->buckets > 1 && !rp->borders) return fail(BP_ERR_INVALID_ARG, "borders is NULL");
    Relpos r;
    r.buckets = rp->buckets;
    r.two_sided = rp->two_sided != 0;
    for (int i = 0; i < BP_RELPOS_MAX_BUCKETS; ++i) r.borders[i] = 0x7fffffff;
    for (int i = 0; i + 1 < rp->buckets; ++i) {
        const int32_t b = rp->borders[i];
        if (b < 1 || b >= (1 << 30) || (i > 0 && b <= rp->borders[i - 1]))
            return fail(BP_ERR_INVALID_ARG, "border %d is %d: ascending, in [1, 2^30)", i, b);
        r.borders[i] = b;
    }
    *out = r;
    return BP_OK;
}

namespace {

// Whole numbers of any size, for comparing products of powers exactly: base 2^32, lowest word first.
typedef std::vector<uint32_t> Whole;
void multiply(Whole& w, uint32_t by) {
    uint64_t carry = 0;
    for (auto& d : w) {
        carry += (uint64_t)d * by;
        d = (uint32_t)carry;
        carry >>= 32;
    }
    if (carry) w.push_back((uint32_t)carry);
}
Whole product(uint32_t a, int times_a, uint32_t b, int times_b) {
    Whole w{1};
    for (int i = 0; i < times_a; ++i) multiply(w, a);
    for (int i = 0; i < times_b; ++i) multiply(w, b);
    return w;
}
bool at_least(const Whole& a, const Whole& b) {
    if (a.size() != b.size()) return a.size() > b.size();
    for (size_t i = a.size(); i-- > 0;)
        if (a[i] != b[i]) return a[i] > b[i];
    return true;
}

constexpr int64_t kBiasMost = int64_t(1) << 40;

// One element a thread.
template <typename T>
__global__ __launch_bounds__(256) void relpos_bias_fwd_kernel(Relpos rp, const float* __restrict__ table, int heads, int64_t lq,
                                                              int64_t lk, int64_t q_start, T* __restrict__ out, int64_t row_stride,
                                                              int64_t head_stride) {
    __shared__ int32_t borders[BP_RELPOS_MAX_BUCKETS];
    if (threadIdx.x < BP_RELPOS_MAX_BUCKETS) borders[threadIdx.x] = rp.borders[threadIdx.x];
    __syncthreads();
    const int64_t n = heads * lq * lk;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (int64_t)gridDim.x * 256) {
        const int64_t j = e % lk, i = e / lk % lq, h = e / lk / lq;
        const int row = relpos_row(q_start + i - j, borders, rp.buckets, rp.two_sided);
        const float v = row < 0 ? -INFINITY : table[(int64_t)row * heads + h];
        T* const to = out + h * head_stride + i * row_stride + j;
        if constexpr (sizeof(T) == 2) *to = (T)f32_to_bf16_bits(v);
        else *to = v;
    }
}

// A bucket's pairs lie in a stretch of a query's keys, so a wavefront adds a query's stretches one by one.
constexpr int kGradRows = 16;          // queries of one (batch, head) a wavefront takes
template <typename T>
__global__ __launch_bounds__(64) void relpos_bias_bwd_kernel(Relpos rp, const T* __restrict__ grad, int64_t lq, int64_t lk,
                                                             int64_t row_stride, int64_t head_stride, int64_t batch_stride,
                                                             int64_t q_start, double* __restrict__ partial) {
    const int lane = threadIdx.x, rows = rp.rows();
    const T* const g = grad + blockIdx.z * batch_stride + blockIdx.y * head_stride;
    const int64_t part = ((int64_t)blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x;
    for (int r = 0; r < rows; ++r) {
        const bool later = r >= rp.buckets;
        const int b = later ? r - rp.buckets : r;
        const int64_t near = b ? rp.borders[b - 1] : later ? 1 : 0, far = b + 1 < rp.buckets ? rp.borders[b] : int64_t(1) << 40;
        double sum = 0;
        for (int64_t i = (int64_t)blockIdx.x * kGradRows; i < min(lq, ((int64_t)blockIdx.x + 1) * kGradRows); ++i) {
            const int64_t q = q_start + i;
            const int64_t first = max(int64_t(0), later ? q + near : q - far + 1), end = min(lk, later ? q + far : q - near + 1);
            float run = 0.f;
            for (int64_t j = first + lane; j < end; j += 64) {
                if constexpr (sizeof(T) == 2) run += bf16_bits_to_f32(g[i * row_stride + j]);
                else run += g[i * row_stride + j];
            }
            sum += run;
        }
        for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off);
        if (lane == 0) partial[part * rows + r] = sum;
    }
}

// grad_table[r][h] = the partial sums of head h, batch by batch and stretch by stretch
__global__ __launch_bounds__(256) void relpos_bias_join_kernel(const double* __restrict__ partial, int rows, int heads, int64_t batch,
                                                               int64_t stretches, float* __restrict__ grad_table) {
    const int e = blockIdx.x * 256 + threadIdx.x;
    if (e >= rows * heads) return;
    const int r = e / heads, h = e % heads;
    double sum = 0;
    for (int64_t b = 0; b < batch; ++b)
        for (int64_t s = 0; s < stretches; ++s) sum += partial[((b * heads + h) * stretches + s) * rows + r];
    grad_table[e] = (float)sum;
}

// One thread an element; the row-wise rule takes a workgroup a row.
__global__ __launch_bounds__(256) void relpos_update_kernel(int rule, float lr, float eps, int rows, int heads, float* __restrict__ table,
                                                            float* __restrict__ state, const float* __restrict__ grad) {
    if (rule == BP_ADAGRAD_ROWWISE) {
        __shared__ double part[256];
        const float* const g = grad + (int64_t)blockIdx.x * heads;
        double sq = 0;
        for (int h = threadIdx.x; h < heads; h += 256) sq += (double)g[h] * g[h];
        part[threadIdx.x] = sq;
        __syncthreads();
        for (int off = 128; off >= 1; off >>= 1) {
            if ((int)threadIdx.x < off) part[threadIdx.x] += part[threadIdx.x + off];
            __syncthreads();
        }
        const float s = state[blockIdx.x] + (float)(part[0] / heads);
        __syncthreads();
        if (threadIdx.x == 0) state[blockIdx.x] = s;
        const float den = sqrtf(s) + eps;
        for (int h = threadIdx.x; h < heads; h += 256) table[(int64_t)blockIdx.x * heads + h] -= lr * g[h] / den;
        return;
    }
    const int e = blockIdx.x * 256 + threadIdx.x;
    if (e >= rows * heads) return;
    const float g = grad[e];
    float step = lr * g;
    if (rule == BP_ADAGRAD) {
        const float s = state[e] + g * g;
        state[e] = s;
        step /= sqrtf(s) + eps;
    }
    table[e] -= step;
}

// Sizes and strides of a [batch][heads][lq][lk] array; 0 strides become the dense ones.
struct Grid4 {
    int64_t batch, lq, lk, row, head, bat;
    int32_t heads;
};
int check_grid(int64_t batch, int32_t heads, int64_t lq, int64_t lk, int64_t row_stride, int64_t head_stride, int64_t batch_stride,
               int64_t q_start, Grid4* out) {
    if (batch < 0 || heads < 0 || lq < 0 || lk < 0) return fail(BP_ERR_INVALID_ARG, "negative size");
    if (heads > 65'535 || batch > 65'535 || lq >= (1 << 30) || lk >= (1 << 30))
        return fail(BP_ERR_UNSUPPORTED, "more than 65,535 heads or batch entries, or a length >= 2^30");
    if (lq && lk && (batch * heads > kBiasMost / lq || batch * heads * lq > kBiasMost / lk))
        return fail(BP_ERR_UNSUPPORTED, "more than 2^40 pairs");
    if (q_start <= -(int64_t(1) << 30) || q_start >= (int64_t(1) << 30)) return fail(BP_ERR_INVALID_ARG, "q_start outside (-2^30, 2^30)");
    const int64_t row = row_stride ? row_stride : lk, need_head = lq ? (lq - 1) * row + lk : 0;
    const int64_t most = int64_t(1) << 45;
    if (row < lk || row > most) return fail(BP_ERR_INVALID_ARG, "row_stride %lld: 0, or at least lk and at most 2^45", (long long)row_stride);
    const int64_t head = head_stride ? head_stride : lq * row;
    if (head < need_head || head > most)
        return fail(BP_ERR_INVALID_ARG, "head_stride %lld: 0, or at least the span of a head's rows and at most 2^45", (long long)head_stride);
    const int64_t need_batch = heads ? (heads - 1) * head + need_head : 0, bat = batch_stride ? batch_stride : heads * head;
    if (bat < need_batch || bat > (int64_t(1) << 46))
        return fail(BP_ERR_INVALID_ARG, "batch_stride %lld: 0, or at least the span of the heads", (long long)batch_stride);
    *out = Grid4{batch, lq, lk, row, head, bat, heads};
    return BP_OK;
}
int64_t grad_stretches(int64_t lq) { return ceil_div(lq, kGradRows); }

}  // namespace
}  // namespace bp

using namespace bp;

BP_EXPORT int bp_relpos_borders(int32_t buckets, int32_t far, int32_t* borders) {
    if (buckets < 1 || buckets > BP_RELPOS_MAX_BUCKETS)
        return fail(BP_ERR_INVALID_ARG, "buckets %d outside [1, %d]", buckets, BP_RELPOS_MAX_BUCKETS);
    if (far < 1 || far >= (1 << 24)) return fail(BP_ERR_INVALID_ARG, "far %d outside [1, 2^24)", far);
    if (buckets == 1) return BP_OK;
    if (!borders) return fail(BP_ERR_INVALID_ARG, "borders is NULL");
    const int e = std::max(1, buckets / 2), k = buckets - e;
    const uint32_t to = (uint32_t)std::max(far, e + 1);
    for (int b = 1; b < e; ++b) borders[b - 1] = b;
    for (int t = 0; t < k; ++t) {
        // the smallest n with n >= e * (to / e)^(t / k), that is n^k * e^t >= to^t * e^k: from a guess, put right in whole numbers
        const Whole goal = product(to, t, (uint32_t)e, k);
        const auto reaches = [&](uint32_t n) { return at_least(product(n, k, (uint32_t)e, t), goal); };
        uint32_t n = (uint32_t)std::max(1.0, std::floor(e * std::pow((double)to / e, (double)t / k)));
        while (n > 1 && reaches(n - 1)) --n;
        while (!reaches(n)) ++n;
        const int at = e - 1 + t;
        if (at > 0) n = std::max(n, (uint32_t)borders[at - 1] + 1);
        borders[at] = (int32_t)n;
    }
    return BP_OK;
}

BP_EXPORT int bp_relpos_bias_fwd(const bp_relpos* rp, const float* table, int32_t heads, int64_t lq, int64_t lk, int64_t q_start, void* out,
                                 int32_t out_dtype, int64_t row_stride, int64_t head_stride, void* stream) {
    Relpos r;
    Grid4 g;
    BP_TRY(check_relpos(rp, &r));
    BP_TRY(check_grid(1, heads, lq, lk, row_stride, head_stride, 0, q_start, &g));
    if (out_dtype != BP_F32 && out_dtype != BP_BF16) return fail(BP_ERR_INVALID_ARG, "unknown out_dtype %d", out_dtype);
    if (heads == 0 || lq == 0 || lk == 0) return BP_OK;
    if (!table || !out) return fail(BP_ERR_INVALID_ARG, "NULL pointer");
    if (((uintptr_t)table & 3) || (uintptr_t)out % elem_bytes(out_dtype)) return fail(BP_ERR_INVALID_ARG, "table or out is not aligned to its element");
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(heads * lq * lk, 256), 1 << 20));
    if (out_dtype == BP_F32)
        BP_LAUNCH(K_RELPOS_FWD, relpos_bias_fwd_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, r, table, heads, lq, lk, q_start,
                  (float*)out, g.row, g.head);
    else
        BP_LAUNCH(K_RELPOS_FWD, relpos_bias_fwd_kernel<uint16_t>, grid, dim3(256), 0, (hipStream_t)stream, r, table, heads, lq, lk, q_start,
                  (uint16_t*)out, g.row, g.head);
    return BP_OK;
}

BP_EXPORT int bp_relpos_bias_bwd_workspace_bytes(const bp_relpos* rp, int64_t batch, int32_t heads, int64_t lq, int64_t lk, size_t* bytes) {
    Relpos r;
    Grid4 g;
    if (!bytes) return fail(BP_ERR_INVALID_ARG, "bytes is NULL");
    BP_TRY(check_relpos(rp, &r));
    BP_TRY(check_grid(batch, heads, lq, lk, 0, 0, 0, 0, &g));
    *bytes = (size_t)(batch * heads * grad_stretches(lq) * r.rows()) * sizeof(double);
    return BP_OK;
}

BP_EXPORT int bp_relpos_bias_bwd(const bp_relpos* rp, const void* grad_out, int32_t grad_dtype, int64_t batch, int32_t heads, int64_t lq,
                                 int64_t lk, int64_t row_stride, int64_t head_stride, int64_t batch_stride, int64_t q_start,
                                 float* grad_table, void* workspace, size_t workspace_bytes, void* stream_) {
    Relpos r;
    Grid4 g;
    size_t need = 0;
    hipStream_t stream = (hipStream_t)stream_;
    BP_TRY(check_relpos(rp, &r));
    BP_TRY(check_grid(batch, heads, lq, lk, row_stride, head_stride, batch_stride, q_start, &g));
    if (grad_dtype != BP_F32 && grad_dtype != BP_BF16) return fail(BP_ERR_INVALID_ARG, "unknown grad_dtype %d", grad_dtype);
    if (heads == 0) return BP_OK;
    if (!grad_table || (batch && lq && lk && !grad_out)) return fail(BP_ERR_INVALID_ARG, "NULL pointer");
    if (((uintptr_t)grad_table & 3) || (uintptr_t)grad_out % elem_bytes(grad_dtype))
        return fail(BP_ERR_INVALID_ARG, "grad_out or grad_table is not aligned to its element");
    BP_TRY(bp_relpos_bias_bwd_workspace_bytes(rp, batch, heads, lq, lk, &need));
    if (need && (!workspace || ((uintptr_t)workspace & 255))) return fail(BP_ERR_INVALID_ARG, "workspace NULL or not 256-byte aligned");
    if (workspace_bytes < need) return fail(BP_ERR_WORKSPACE_TOO_SMALL, "workspace %zu < required %zu bytes", workspace_bytes, need);
    double* const partial = (double*)workspace;
    const int64_t stretches = grad_stretches(lq);
    if (batch && lq) {
        const dim3 grid((unsigned)stretches, (unsigned)heads, (unsigned)batch);
        if (grad_dtype == BP_F32)
            BP_LAUNCH(K_RELPOS_BWD, relpos_bias_bwd_kernel<float>, grid, dim3(64), 0, stream, r, (const float*)grad_out, lq, lk, g.row, g.head,
                      g.bat, q_start, partial);
        else
            BP_LAUNCH(K_RELPOS_BWD, relpos_bias_bwd_kernel<uint16_t>, grid, dim3(64), 0, stream, r, (const uint16_t*)grad_out, lq, lk, g.row,
                      g.head, g.bat, q_start, partial);
    }
    BP_LAUNCH(K_RELPOS_JOIN, relpos_bias_join_kernel, dim3((unsigned)ceil_div((int64_t)r.rows() * heads, 256)), dim3(256), 0, stream, partial,
              r.rows(), heads, lq ? batch : 0, stretches, grad_table);
    return BP_OK;
}

BP_EXPORT int bp_relpos_update(const bp_config* cfg, const bp_relpos* rp, int32_t heads, float* table, float* state, const float* grad_table,
                               void* stream) {
    Relpos r;
    if (!cfg) return fail(BP_ERR_INVALID_ARG, "cfg is NULL");
    BP_TRY(check_relpos(rp, &r));
    const int rule = cfg->optimizer;
    if (rule != BP_SGD && rule != BP_ADAGRAD && rule != BP_ADAGRAD_ROWWISE) return fail(BP_ERR_INVALID_ARG, "unknown optimizer %d", rule);
    if (heads < 0 || heads > 65'535) return fail(BP_ERR_INVALID_ARG, "heads %d outside [0, 65535]", heads);
    if (heads == 0) return BP_OK;
    if (!table || !grad_table || (rule != BP_SGD && !state)) return fail(BP_ERR_INVALID_ARG, "NULL pointer");
    if (((uintptr_t)table | (uintptr_t)grad_table | (uintptr_t)state) & 3) return fail(BP_ERR_INVALID_ARG, "arrays must be aligned to their elements");
    const int64_t blocks = rule == BP_ADAGRAD_ROWWISE ? r.rows() : ceil_div((int64_t)r.rows() * heads, 256);
    BP_LAUNCH(K_RELPOS_UPDATE, relpos_update_kernel, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, rule, cfg->lr, cfg->eps, r.rows(),
              heads, table, state, grad_table);
    return BP_OK;
}
