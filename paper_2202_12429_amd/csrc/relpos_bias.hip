// Bias by distance: out[h, i, j] = table[row((q_start + i) - j)][h], its gradient and the step on the table.
#include <algorithm>
#include <cmath>
#include <type_traits>

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

// Whole numbers for comparing products of powers exactly: base 2^32, lowest word first.  The products are below n^32 * 32^32 for n up to
// `far`, 2^24, and a little more: 2^1024 is room enough, and no entry point of C allocates here, which might throw.
struct Whole {
    uint32_t word[32] = {1};
    int size = 1;
};
void multiply(Whole& w, uint32_t by) {
    uint64_t carry = 0;
    for (int i = 0; i < w.size; ++i) {
        carry += (uint64_t)w.word[i] * by;
        w.word[i] = (uint32_t)carry;
        carry >>= 32;
    }
    if (carry && w.size < 32) w.word[w.size++] = (uint32_t)carry;
}
Whole product(uint32_t a, int times_a, uint32_t b, int times_b) {
    Whole w;
    for (int i = 0; i < times_a; ++i) multiply(w, a);
    for (int i = 0; i < times_b; ++i) multiply(w, b);
    return w;
}
bool at_least(const Whole& a, const Whole& b) {
    if (a.size != b.size) return a.size > b.size;
    for (int i = a.size; i-- > 0;)
        if (a.word[i] != b.word[i]) return a.word[i] > b.word[i];
    return true;
}

constexpr int64_t kBiasMost = int64_t(1) << 40;

// A workgroup writes a stretch of keys for up to kBiasRows queries of one head.  What it writes depends on j - i alone, so the
// looked-up values lie in LDS as one line, of which every query takes a stretch, shifted by one from the query before.  16
// bytes a store, aligned in memory (the first and last of a row's chunks may be cut), whatever a row's own alignment.  bf16 lines
// are kept as pairs, once from every even and once from every odd element on.  Bound by the stores (15 heads,
// 2,048 queries, 1,999 keys, bf16: 36 us, with non-temporal stores 40).
constexpr int kBiasBlock = 256, kBiasRows = 32, kBiasChunks = 256;
template <typename T>
__global__ __launch_bounds__(kBiasBlock) void relpos_bias_fwd_kernel(Relpos rp, const float* __restrict__ table, int heads, int64_t lq,
                                                                     int64_t lk, int64_t q_start, T* __restrict__ out, int64_t row_stride,
                                                                     int64_t head_stride, int chunks, int64_t tiles) {
    constexpr int PER = 16 / sizeof(T), MOST = kBiasChunks * PER + 2 * PER + kBiasRows + 8;
    __shared__ int32_t borders[BP_RELPOS_MAX_BUCKETS];
    __shared__ float column[2 * BP_RELPOS_MAX_BUCKETS];
    __shared__ uint32_t line[MOST];                       // fp32: a value a word; bf16: words 0 .. MOST/2 even pairs, then odd ones
    const int64_t id = (int64_t)blockIdx.z * gridDim.x + blockIdx.x, j0 = id % tiles * chunks * PER, i0 = id / tiles * kBiasRows;
    if (i0 >= lq) return;
    const int h = blockIdx.y, rows = (int)min((int64_t)kBiasRows, lq - i0);
    if (threadIdx.x < BP_RELPOS_MAX_BUCKETS) borders[threadIdx.x] = rp.borders[threadIdx.x];
    for (int r = threadIdx.x; r < rp.rows(); r += kBiasBlock) column[r] = table[(int64_t)r * heads + h];
    __syncthreads();
    // line[x] is the value of key j for query i with x = (j - j0 + PER) + (rows - 1 - (i - i0)): a cut chunk begins up to PER - 1
    // keys before j0
    const int width = chunks * PER + PER + rows - 1;
    const int64_t nearest = q_start + i0 + rows - 1 - j0 + PER;
    const auto value = [&](int x) {
        const int row = relpos_row(nearest - x, borders, rp.buckets, rp.two_sided);
        return row < 0 ? -INFINITY : column[row];
    };
    if constexpr (sizeof(T) == 2) {
        uint16_t* const even = (uint16_t*)line;
        uint16_t* const odd = (uint16_t*)(line + MOST / 2);
        for (int x = threadIdx.x; x < width; x += kBiasBlock) {
            const uint16_t v = (uint16_t)f32_to_bf16_bits(value(x));
            even[x] = v;
            if (x) odd[x - 1] = v;
        }
    } else {
        for (int x = threadIdx.x; x < width; x += kBiasBlock) line[x] = __float_as_uint(value(x));
    }
    __syncthreads();
    // a row's chunks side by side, and as many rows side by side as the workgroup has threads for
    int wide = 1;
    while (wide < chunks + 1 && wide < kBiasBlock) wide <<= 1;
    T* const base = out + h * head_stride + i0 * row_stride + j0;
    for (int r = threadIdx.x / wide; r < rows; r += kBiasBlock / wide) {
        T* const row = base + r * row_stride;
        const int cut = (int)(((uintptr_t)row & 15) / sizeof(T));      // keys by which the row's first aligned chunk begins before it
        const int64_t left = lk - j0;
        const int end = (int)min(left, (int64_t)chunks * PER);         // the workgroup's keys are [0, end) of the row
        for (int c = threadIdx.x % wide; c * PER - cut < end; c += wide) {
            const int j = c * PER - cut, x = j + PER + rows - 1 - r;
            uint32_t v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = sizeof(T) == 4 ? line[x + i] : x % 2 ? line[MOST / 2 + x / 2 + i] : line[x / 2 + i];
            if (j >= 0 && j + PER <= end) {
                *reinterpret_cast<uint4*>(row + j) = make_uint4(v[0], v[1], v[2], v[3]);
            } else {
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (j + i >= 0 && j + i < end) {
                        if constexpr (sizeof(T) == 2) row[j + i] = (T)(v[i / 2] >> (16 * (i % 2)));
                        else row[j + i] = __uint_as_float(v[i]);
                    }
            }
        }
    }
}

// The gradient's sums run along the diagonals: a wavefront takes 64 blocks of NB x NB pairs side by side, a block a lane (NB
// keys are 16 bytes), and walks down the diagonal with them, so that a lane adds the same 2 NB - 1 diagonals all the way, in
// registers, and what is not seen (later keys of a one-sided bias) is a matter of whole diagonals: they are dropped behind the
// walk, whatever they hold.  Bound by the loads: a step's NB rows of 16 bytes a lane are in flight together, its
// additions wait for them, and other wavefronts fill the time.
constexpr int kGradWaves = 4;

template <typename T>
struct GradBlock {
    static constexpr int NB = 16 / sizeof(T), STEPS = 128 / NB, DIAGONALS = 64 * NB + 8;      // (the last ones unused)
    typedef uint32_t Vec __attribute__((ext_vector_type(4)));
    // fp64 from the first addition on for fp32, which costs nothing (2 x 16 grids of 2,048 x 2,048: 115 us, with fp32 runs 123); bf16
    // values, of eight bits each, in fp32 over a segment's 128 queries, and in fp64 from there on
    typedef std::conditional_t<sizeof(T) == 4, double, float> Sum;
    Vec raw[NB];
    // The block at `at`, of which `rows` x `cols` pairs exist; `left`: elements from `at` to the end of the array.  A row's 16 bytes
    // are read as long as they lie in the array, and cut after that.
    __device__ __forceinline__ void load(const T* at, int64_t row_stride, int64_t left, int rows, int cols) {
        // zeros first, for every lane: written behind the branch they would have to wait for the loads of the lanes inside it
#pragma unroll
        for (int i = 0; i < NB; ++i) raw[i] = Vec{0, 0, 0, 0};
        if (rows >= NB && cols >= NB) {
#pragma unroll
            for (int i = 0; i < NB; ++i) __builtin_memcpy(&raw[i], at + i * row_stride, 16);           // aligned to their elements only
        }
        if (rows <= 0 || cols <= 0 || (rows >= NB && cols >= NB)) return;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            if (i >= rows) continue;
            const T* const row = at + i * row_stride;
            if (i * row_stride + NB <= left) {
                __builtin_memcpy(&raw[i], row, 16);
            } else {
                uint64_t lo = 0, hi = 0;                               // the array's last few elements, one by one
#pragma unroll 1
                for (int j = 0; j < cols; ++j) {
                    uint32_t bits;
                    if constexpr (sizeof(T) == 2) bits = row[j];
                    else bits = __float_as_uint(row[j]);
                    const uint64_t v = (uint64_t)bits << (j % (NB / 2) * (8 * sizeof(T)));
                    if (j < NB / 2) lo |= v;
                    else hi |= v;
                }
                raw[i] = Vec{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if constexpr (sizeof(T) == 2) raw[i][w] &= (2 * w < cols ? 0xffffu : 0u) | (2 * w + 1 < cols ? 0xffff0000u : 0u);
                else raw[i][w] = w < cols ? raw[i][w] : 0u;
            }
        }
    }
    __device__ __forceinline__ float value(int i, int j) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(raw[i][j]);
        else return __uint_as_float(j % 2 ? raw[i][j / 2] & 0xffff0000u : raw[i][j / 2] << 16);
    }
};

struct GradArgs {
    Relpos rp;
    int64_t lq, lk, row, head, bat, q_start;
    int64_t blocks_q, blocks_k;            // blocks down and across
    int64_t span;                          // elements from the first pair to the last one, and one more
    int64_t first_band;                    // block diagonal (block column - block row) of band 0's lane 0
    int32_t bands, segments, steps;        // of 64 block diagonals; of `steps` block rows
    int32_t heads;
    double* partial;                       // [batch][heads][bands][segments][table rows]
};

template <typename T>
__global__ __launch_bounds__(kGradWaves * 64) void relpos_bias_bwd_kernel(GradArgs a, const T* __restrict__ grad) {
    typedef GradBlock<T> B;
    constexpr int NB = B::NB;
    __shared__ double diag[kGradWaves][B::DIAGONALS], eights[kGradWaves][B::DIAGONALS / 8], more[kGradWaves][B::DIAGONALS / 64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t job = (int64_t)blockIdx.x * kGradWaves + wave, jobs = (int64_t)a.bands * a.segments;
    const bool have = job < jobs;
    const int64_t band0 = a.first_band + job / a.segments * 64, seg0 = job % a.segments * a.steps;
    const int64_t kd = band0 + lane;                                   // the lane's block diagonal
    typename B::Sum acc[2 * NB - 1];
#pragma unroll
    for (int d = 0; d < 2 * NB - 1; ++d) acc[d] = 0;
    if (have) {
        // block rows in which some lane has a block
        const int64_t from = max(seg0, -(band0 + 63)), to = min(min(seg0 + a.steps, a.blocks_q), a.blocks_k - band0);
        // a one-sided bias sees nothing of a block whose keys are all later
        const bool seen = a.rp.two_sided || kd * NB - (NB - 1) <= a.q_start;
        const int64_t base = blockIdx.z * a.bat + blockIdx.y * a.head;
        B cur;
        const auto fetch = [&](B& b, int64_t row) {
            const int64_t col = row + kd, i = row * NB, j = col * NB;
            const bool in = seen && row < to && col >= 0 && col < a.blocks_k;
            const int64_t at = base + i * a.row + j;
            b.load(grad + at, a.row, a.span - at, in ? (int)min(a.lq - i, (int64_t)NB) : 0, in ? (int)min(a.lk - j, (int64_t)NB) : 0);
        };
        const auto add = [&](const B& b) {
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[j - i + NB - 1] += b.value(i, j);
        };
        for (int64_t row = from; row < to; ++row) {
            fetch(cur, row);
            add(cur);
        }
    }
    // diagonals (j - i) of the wavefront from band0 * NB - (NB - 1) on: neighbours share NB - 1 of theirs
    double* const d = diag[wave];
#pragma unroll
    for (int k = 0; k < NB; ++k) d[NB * lane + k] = acc[k];
    if (lane < 8) d[64 * NB + lane] = 0;
    __syncthreads();
#pragma unroll
    for (int k = NB; k < 2 * NB - 1; ++k) d[NB * lane + k] += acc[k];
    __syncthreads();
    // A bucket is a stretch of diagonals: single ones at both ends, sums of eight and of sixty-four in between, so that no lane
    // adds more than 36 values one behind the other.  (A NaN where nothing is seen stays in its own sums: a seen bucket takes no
    // part of a sum that it does not hold whole.)
    for (int e = lane; e < B::DIAGONALS / 8; e += 64) {
        double sum = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += d[8 * e + k];
        eights[wave][e] = sum;
    }
    __syncthreads();
    if (lane < B::DIAGONALS / 64) {
        double sum = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += eights[wave][8 * lane + k];
        more[wave][lane] = sum;
    }
    __syncthreads();
    if (!have) return;
    const int rows = a.rp.rows();
    double* const out = a.partial + (((int64_t)blockIdx.z * a.heads + blockIdx.y) * jobs + job) * rows;
    const int64_t zero = band0 * NB - (NB - 1);                        // the diagonal d[0] is
    for (int r = lane; r < rows; r += 64) {
        const bool later = r >= a.rp.buckets;
        const int b = later ? r - a.rp.buckets : r;
        const int64_t near = b ? a.rp.borders[b - 1] : later ? 1 : 0, far = b + 1 < a.rp.buckets ? a.rp.borders[b] : int64_t(1) << 40;
        // distance q_start - diagonal in [near, far), or its negative for later keys
        const int64_t lo = later ? a.q_start + near : a.q_start - far + 1, hi = later ? a.q_start + far : a.q_start - near + 1;
        int x = (int)min(max(lo - zero, int64_t(0)), (int64_t)B::DIAGONALS);
        const int end = (int)min(max(hi - zero, int64_t(0)), (int64_t)B::DIAGONALS);
        double sum = 0;
        while (x < end && x % 8) sum += d[x++];
        for (; x + 8 <= end && x % 64; x += 8) sum += eights[wave][x / 8];
        for (; x + 64 <= end; x += 64) sum += more[wave][x / 64];
        for (; x + 8 <= end; x += 8) sum += eights[wave][x / 8];
        while (x < end) sum += d[x++];
        out[r] = sum;
    }
}

// grad_table[r][h] = the sum over the wavefronts' parts: a workgroup 16 rows of a head, 64 shares of the parts side by side
constexpr int kJoinRows = 16, kJoinShares = 64;
__global__ __launch_bounds__(kJoinRows * kJoinShares) void relpos_bias_join_kernel(const double* __restrict__ partial, int rows, int heads,
                                                                                   int64_t batch, int64_t jobs, float* __restrict__ grad_table) {
    __shared__ double part[kJoinShares][kJoinRows];
    const int h = blockIdx.x, c = threadIdx.x % kJoinRows, r = blockIdx.y * kJoinRows + c, share = threadIdx.x / kJoinRows;
    double sum = 0;
    if (r < rows)
        for (int64_t b = 0; b < batch; ++b)
            for (int64_t s = share; s < jobs; s += kJoinShares) sum += partial[((b * heads + h) * jobs + s) * rows + r];
    part[share][c] = sum;
    __syncthreads();
    for (int off = kJoinShares / 2; off >= 1; off >>= 1) {
        if (share < off) part[share][c] += part[share + off][c];
        __syncthreads();
    }
    if (share == 0 && r < rows) grad_table[(int64_t)r * heads + h] = (float)part[0][c];
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
    const int64_t row = row_stride ? row_stride : lk, most = int64_t(1) << 45;
    if (row < lk || row > most / std::max<int64_t>(lq, 1))
        return fail(BP_ERR_INVALID_ARG, "row_stride %lld: 0, or at least lk and at most 2^45 / lq", (long long)row_stride);
    const int64_t need_head = lq ? (lq - 1) * row + lk : 0;
    const int64_t head = head_stride ? head_stride : lq * row;
    if (head < need_head || head > most)
        return fail(BP_ERR_INVALID_ARG, "head_stride %lld: 0, or at least the span of a head's rows and at most 2^45", (long long)head_stride);
    const int64_t need_batch = heads ? (heads - 1) * head + need_head : 0, bat = batch_stride ? batch_stride : heads * head;
    if (bat < need_batch || bat > (int64_t(1) << 46))
        return fail(BP_ERR_INVALID_ARG, "batch_stride %lld: 0, or at least the span of the heads", (long long)batch_stride);
    *out = Grid4{batch, lq, lk, row, head, bat, heads};
    return BP_OK;
}

// Bands and segments of the walk.  Segments of 128 queries where those make 4,096 wavefronts or more, shorter ones in smaller
// launches (3 x 5 grids of 777 x 1,001 fp32, enough being 1,024: 21.6 us; 4,096: 13.6;
// 16,384: 13.2, but 2 x 16 grids of 2,048 x 2,048 bf16 then take 37.4 for 36.5).
constexpr int kGradEnough = 4096;
int grad_plan(const Relpos& r, int32_t dtype, int64_t batch, int32_t heads, int64_t lq, int64_t lk, int64_t q_start, GradArgs* a) {
    const int block = 16 / (int)elem_bytes(dtype), shift = dtype == BP_F32 ? 2 : 3;
    a->blocks_q = ceil_div(lq, block);
    a->blocks_k = ceil_div(lk, block);
    a->first_band = -(a->blocks_q - 1);
    int64_t last = a->blocks_k - 1;
    if (!r.two_sided) last = std::min(last, (q_start + block - 1) >> shift);            // rounded down
    const int64_t bands = lq == 0 || lk == 0 || last < a->first_band ? 0 : ceil_div(last - a->first_band + 1, 64);
    a->steps = 128 / block;
    while (a->steps > 4 && batch * heads * bands * ceil_div(a->blocks_q, a->steps) < kGradEnough) a->steps /= 2;
    const int64_t segments = ceil_div(a->blocks_q, a->steps);
    if (bands * segments >= (int64_t(1) << 26)) return fail(BP_ERR_UNSUPPORTED, "more than 2^26 pieces of work a head");       // a launch's threads
    a->bands = (int32_t)bands;
    a->segments = (int32_t)segments;
    return BP_OK;
}

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
    const int per = 16 / (int)elem_bytes(out_dtype), chunks = kBiasChunks;         // a workgroup's keys
    const int64_t row_blocks = ceil_div(lq, kBiasRows), all_chunks = ceil_div(lk, per);
    const int64_t tiles = ceil_div(all_chunks, chunks);
    const dim3 grid = spread_grid(tiles * row_blocks, (unsigned)heads);
    if (out_dtype == BP_F32)
        BP_LAUNCH(K_RELPOS_FWD, relpos_bias_fwd_kernel<float>, grid, dim3(kBiasBlock), 0, (hipStream_t)stream, r, table, heads, lq, lk, q_start,
                  (float*)out, g.row, g.head, chunks, tiles);
    else
        BP_LAUNCH(K_RELPOS_FWD, relpos_bias_fwd_kernel<uint16_t>, grid, dim3(kBiasBlock), 0, (hipStream_t)stream, r, table, heads, lq, lk,
                  q_start, (uint16_t*)out, g.row, g.head, chunks, tiles);
    return BP_OK;
}

BP_EXPORT int bp_relpos_bias_bwd_workspace_bytes(const bp_relpos* rp, int64_t batch, int32_t heads, int64_t lq, int64_t lk, size_t* bytes) {
    Relpos r;
    Grid4 g;
    if (!bytes) return fail(BP_ERR_INVALID_ARG, "bytes is NULL");
    BP_TRY(check_relpos(rp, &r));
    BP_TRY(check_grid(batch, heads, lq, lk, 0, 0, 0, 0, &g));
    const int rows = r.rows();
    r.two_sided = 1;                                   // room for every q_start: as if all keys were seen
    *bytes = 0;
    for (int32_t dtype : {BP_F32, BP_BF16}) {
        GradArgs a{};
        BP_TRY(grad_plan(r, dtype, batch, heads, lq, lk, 0, &a));
        // (shorter segments come to less than twice the wavefronts that are enough)
        const int64_t walks = batch * heads * a.bands, block = 16 / (int64_t)elem_bytes(dtype);
        const int64_t most = std::max(walks * ceil_div(a.blocks_q, 128 / block), std::min<int64_t>(2 * kGradEnough, walks * ceil_div(a.blocks_q, 4)));
        *bytes = std::max(*bytes, (size_t)(most * rows) * sizeof(double));
    }
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
    GradArgs a{};
    BP_TRY(grad_plan(r, grad_dtype, batch, heads, lq, lk, q_start, &a));
    a.rp = r;
    a.lq = lq;
    a.lk = lk;
    a.row = g.row;
    a.head = g.head;
    a.bat = g.bat;
    a.span = batch && heads && lq ? (batch - 1) * g.bat + (heads - 1) * g.head + (lq - 1) * g.row + lk : 0;
    a.q_start = q_start;
    a.heads = heads;
    a.partial = (double*)workspace;
    const int64_t jobs = (int64_t)a.bands * a.segments;
    if (batch && jobs) {
        const dim3 grid((unsigned)ceil_div(jobs, kGradWaves), (unsigned)heads, (unsigned)batch), block(kGradWaves * 64);
        if (grad_dtype == BP_F32)
            BP_LAUNCH(K_RELPOS_BWD, relpos_bias_bwd_kernel<float>, grid, block, 0, stream, a, (const float*)grad_out);
        else
            BP_LAUNCH(K_RELPOS_BWD, relpos_bias_bwd_kernel<uint16_t>, grid, block, 0, stream, a, (const uint16_t*)grad_out);
    }
    BP_LAUNCH(K_RELPOS_JOIN, relpos_bias_join_kernel, dim3((unsigned)heads, (unsigned)ceil_div(r.rows(), kJoinRows)),
              dim3(kJoinRows * kJoinShares), 0, stream, a.partial, r.rows(), heads, batch, jobs, grad_table);
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
