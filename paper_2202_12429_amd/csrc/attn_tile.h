// A tile of a bag's rows in the matrix instructions: what the forward and backward kernels of attention over bags share.
#pragma once

#include <type_traits>

#include "attn_args.h"

namespace bp {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLn2 = 0.6931471805599453f;

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

// How a wavefront takes a tile of rows with the matrix instructions: the rows' entries down, query heads across, of which there
// are up to 16 columns: the groups of PACK kv heads, so that what is done with a score is done for all of them at once.
// Scores: S[entry][column] = K Q^T for every kv head, of which a column takes its own head's; a lane loads 16 bytes of a row and
// its neighbours 16 lanes away the next 16.  (A product of all heads' keys with a query padded by zeros would do without the
// choice, but a NaN of one head would be another's too.)  Pooling: O^T[element][column] = V^T P^T over the heads' values side by
// side, of which a column's own are taken at the end; an entry whose scores a lane holds is one whose p that lane is asked for,
// so p never leaves its lane, and V comes in whole rows: a lane loads VW elements, which serve VW products of 16 elements each.
// bf16 rows go through the bf16 instruction: q and p are cut into three bf16 parts, whose products are exact in fp32, so that
// what is computed is fp32.  DP: head_dim rounded up.
template <typename T, int DP, int PACK>
struct AttnTile {
    static constexpr bool BF16 = sizeof(T) == 2;
    static constexpr int ROWS = BF16 ? 32 : 16;        // entries of a tile
    static constexpr int NU = ROWS / 16;               // S tiles
    static constexpr int PER = ROWS / 4;               // entries a lane holds scores of
    static constexpr int KC = BF16 ? 32 : 16, KM = (DP + KC - 1) / KC;
    static constexpr int FLAT = PACK * DP;             // elements of the heads' values
    static constexpr int VW = FLAT / 16 < (BF16 ? 8 : 4) ? FLAT / 16 : BF16 ? 8 : 4, MB = FLAT / (16 * VW);
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

// head_dim rounded up, and the kv heads that share a wavefront's columns: as many as have columns, and registers for two
// workgroups a CU (forward, four heads of 64, rows of 1 KB: 67 us by twos, 70 one by one).
inline int attn_dp(const bp_attn* at, int dtype) {
    int dp = dtype == BP_F32 ? 16 : 32;
    while (dp < at->head_dim) dp *= 2;
    return dp;
}
inline int attn_pack(const bp_attn* at, int dp) {
    int pack = 1;
    const int group = at->q_heads / at->kv_heads;
    while (pack < at->kv_heads && 2 * pack * group <= 16 && 2 * pack * dp <= 128 && pack < 8) pack *= 2;
    return pack;
}

// Calls f.template run<T, DP, PACK, FULL>() for a layout.  FULL: heads of exactly DP elements, PACK of them in every wavefront, for
// which the kernels need no test of what lies inside a row (backward, heads of 64: those tests took half of a tile's instructions).
template <typename T, int DP, int PACK, typename F>
int dispatch_attn_full(const AttnArgs& a, F&& f) {
    return a.d == DP && a.kv_heads % PACK == 0 ? f.template run<T, DP, PACK, true>() : f.template run<T, DP, PACK, false>();
}
template <typename T, int DP, typename F>
int dispatch_attn_pack(const AttnArgs& a, int pack, F&& f) {
    switch (pack) {
        case 1: return dispatch_attn_full<T, DP, 1>(a, f);
        case 2: if constexpr (DP <= 64) return dispatch_attn_full<T, DP, 2>(a, f); break;
        case 4: if constexpr (DP <= 32) return dispatch_attn_full<T, DP, 4>(a, f); break;
        case 8: if constexpr (DP <= 16) return dispatch_attn_full<T, DP, 8>(a, f); break;
    }
    return fail(BP_ERR_UNSUPPORTED, "no layout for %d heads of %d", pack, DP);
}
template <typename T, typename F>
int dispatch_attn(const AttnArgs& a, int dp, int pack, F&& f) {
    switch (dp) {
        case 16: if constexpr (sizeof(T) == 4) return dispatch_attn_pack<T, 16>(a, pack, f); break;
        case 32: return dispatch_attn_pack<T, 32>(a, pack, f);
        case 64: return dispatch_attn_pack<T, 64>(a, pack, f);
        case 128: return dispatch_attn_pack<T, 128>(a, pack, f);
        case 256: return dispatch_attn_pack<T, 256>(a, pack, f);
    }
    return fail(BP_ERR_UNSUPPORTED, "no layout for heads of %d", dp);
}

// Rows without the matrix instructions: a lane holds 16 bytes, LANES lanes a head.
template <typename T, int LANES>
struct Narrow {
    static constexpr int VE = 16 / sizeof(T), D = LANES * VE;
    static __device__ __forceinline__ void read(const float* from, float (&v)[VE]) {
#pragma unroll
        for (int i = 0; i < VE; i += 4) __builtin_memcpy(v + i, __builtin_assume_aligned(from + i, 16), 16);
    }
    static __device__ __forceinline__ void write(float* to, const float (&v)[VE]) {
#pragma unroll
        for (int i = 0; i < VE; i += 4) __builtin_memcpy(__builtin_assume_aligned(to + i, 16), v + i, 16);
    }
    static __device__ __forceinline__ void widen(const uint4& x, float (&v)[VE]) {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (VE == 4) {
                v[i] = __uint_as_float(w[i]);
            } else {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
    // the same sum in all of the head's lanes
    static __device__ __forceinline__ float dot(const float (&x)[VE], const float (&y)[VE]) {
        float s = x[0] * y[0];
#pragma unroll
        for (int i = 1; i < VE; ++i) s = fmaf(x[i], y[i], s);
#pragma unroll
        for (int off = 1; off < LANES; off <<= 1) s += __shfl_xor(s, off);
        return s;
    }
};
// One query head a kv head, rows that are their own values, and lanes that heads and rows divide evenly.
inline bool attn_narrow(const bp_attn* at, int dtype) {
    const int lanes = at->head_dim * (dtype == BP_F32 ? 4 : 2) / 16, width = lanes * at->kv_heads;
    const auto power = [](int x) { return x > 0 && (x & (x - 1)) == 0; };
    return at->q_heads == at->kv_heads && at->value_offset == 0 && at->head_dim >= 16 && power(at->head_dim) && power(at->kv_heads) && width <= 64;
}
template <typename T, typename F>
int dispatch_narrow(const AttnArgs& a, F&& f) {
    switch (a.d * (int)sizeof(T) / 16) {
        case 2: if constexpr (sizeof(T) == 2) return f.template run_narrow<T, 2>(); break;
        case 4: return f.template run_narrow<T, 4>();
        case 8: return f.template run_narrow<T, 8>();
        case 16: return f.template run_narrow<T, 16>();
        case 32: return f.template run_narrow<T, 32>();
        case 64: if constexpr (sizeof(T) == 4) return f.template run_narrow<T, 64>(); break;
    }
    return fail(BP_ERR_UNSUPPORTED, "no layout for heads of %d", a.d);
}

__device__ __forceinline__ float4 or_zeros(const float4& v, bool have) {
    return make_float4(have ? v.x : 0.f, have ? v.y : 0.f, have ? v.z : 0.f, have ? v.w : 0.f);
}

// 16 bytes of a row, or zeros: the address is one inside the row in any case, so that no load waits for a mask.
template <bool FULL, typename T>
__device__ __forceinline__ uint4 row_bytes_at(const T* row, int x, int d) {
    const uint4 v = *reinterpret_cast<const uint4*>(row + (FULL || x < d ? x : 0));
    return FULL ? v : masked(v, x < d ? ~0u : 0u);
}

}  // namespace
}  // namespace bp
