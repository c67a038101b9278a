// Shared by the kernels of attention with modified scores: the score function, the rows a CTA has to
// walk, and the tensor maps over hi/lo planes.
#pragma once
#include "common.cuh"
#include "tc_common.cuh"

namespace bt {
namespace mod {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// tanh for the cap.  A capped score is cap * tanh(u), u = score / cap: for the usual small u its error
// has to be relative to u, so below 0.6 an odd polynomial is used (least-squares fit of (tanh(u)/u - 1) / u^2
// reweighted to the smallest largest relative error, 2.8e-9, one FP32 rounding in all); above,
// 1 - 2 / (1 + e^2|u|), which is good to 2^-22 there.
constexpr float kTanhSmall = 0.6f;
__device__ __forceinline__ float tanh_small(float u) {
    const float w = u * u;
    float q = fmaf(w, -0.005895158275961876f, 0.020795971155166626f);
    q = fmaf(w, q, -0.053783830255270004f);
    q = fmaf(w, q, 0.13331924378871918f);
    q = fmaf(w, q, -0.33333298563957214f);
    return fmaf(u * w, q, u);
}
__device__ __forceinline__ float tanh_any(float u) {
    const float t = fmaf(-2.0f, rcp_fast(1.0f + ex2_fast(2.8853900817779268f * fabsf(u))), 1.0f);
    return fabsf(u) < kTanhSmall ? tanh_small(u) : copysignf(t, u);
}
// u <- tanh(u).  The exponential and the reciprocal run at an eighth of the rate of a multiplication and are
// needed only where some score of the row's tile is beyond 0.6 caps.
template <int N>
__device__ __forceinline__ void tanh_tile(float (&u)[N]) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(u[i]));
    if (top < kTanhSmall) {
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] = tanh_small(u[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] = tanh_any(u[i]);
    }
}

// Score modification in base-2 units.  `unit` turns a dot product q k into cap units (u = unit * dot) or,
// without a cap, straight into base-2 units; `to_log2` turns tanh into base-2 units.  The backward kernels
// multiply their own rows by `unit` before the product instead of the scores after it.
struct Score {
    float unit, to_log2, slope2;
};
template <bool CAP, bool SLOPE>
__device__ __forceinline__ Score make_score(float scale, float cap, const float* slopes, int h) {
    Score s;
    s.unit = CAP ? scale / cap : scale * kLog2e;
    s.to_log2 = CAP ? cap * kLog2e : 1.0f;
    s.slope2 = SLOPE ? slopes[h] * kLog2e : 0.f;
    return s;
}
// x: N neighbouring dot products of one row -> modified scores in base-2 units.  |first - i| is the distance of
// position i.  Without a modification x stays as it is (the exponent's multiplication takes `unit`).
template <bool CAP, bool SLOPE, int N>
__device__ __forceinline__ void score_tile(float (&x)[N], const Score& s, int first) {
    if (CAP || SLOPE) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= s.unit;
    }
    if (CAP) {
        tanh_tile<N>(x);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= s.to_log2;
    }
    if (SLOPE) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = fmaf(-s.slope2, fabsf((float)(first - i)), x[i]);
    }
}
// The same for dot products already multiplied by s.unit, keeping 1 - tanh^2 (`grad` untouched without a cap).
template <bool CAP, bool SLOPE, int N>
__device__ __forceinline__ void score_tile_grad(float (&x)[N], float (&grad)[N], const Score& s, int first) {
    if (CAP) {
        tanh_tile<N>(x);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            grad[i] = fmaf(-x[i], x[i], 1.0f);
            x[i] *= s.to_log2;
        }
    }
    if (SLOPE) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = fmaf(-s.slope2, fabsf((float)(first - i)), x[i]);
    }
}

// Rows [lo, hi) that `rows` own rows from r0 on have to walk (64-row blocks; without spans: causal).
__device__ __forceinline__ int2 block_range(const int2* blocks, int b, int T, int r0, int rows, bool keys) {
    if (!blocks) return keys ? make_int2(r0, T) : make_int2(0, min(r0 + rows, T));
    const int nb = (T + 63) >> 6;
    int2 u = make_int2(0x7fffffff, 0);
    for (int k = r0 >> 6; k < min((r0 + rows + 63) >> 6, nb); ++k) {
        const int2 v = blocks[(int64_t)b * nb + k];
        if (v.x < v.y) u = make_int2(min(u.x, v.x), max(u.y, v.y));
    }
    return u.y ? u : make_int2(0, 0);
}
// The range of one own row; empty past the end of the sequence.
__device__ __forceinline__ int2 row_range(const int2* spans, int b, int T, int row, bool keys) {
    if (row >= T) return make_int2(0, 0);
    if (!spans) return keys ? make_int2(row, T) : make_int2(0, row + 1);
    return spans[(int64_t)b * T + row];
}

// Tensor map over a row-major [rows][cols] array of hi/lo planes: boxes of 32 columns x box_rows rows x both
// planes, K-major (128-byte swizzle) or MN-major (128-byte swizzle with 32-byte atoms).
inline bool plane_map(CUtensorMap* tm, const float* base, int64_t cols, int64_t rows, uint32_t box_rows, bool mn_major) {
    tc::EncodeTiledFn enc = tc::tensor_map_encoder();
    if (!enc) return false;
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, 2};
    cuuint64_t strides[2] = {(cuuint64_t)cols * 4, (cuuint64_t)(rows * cols) * 4};
    cuuint32_t box[3] = {32, box_rows, 2};
    cuuint32_t estr[3] = {1, 1, 1};
    return enc(tm, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, (void*)base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               mn_major ? CU_TENSOR_MAP_SWIZZLE_128B_ATOM_32B : CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Runs `stmt` with kCap and kSlope the constants of the call's modification.
#define BT_FOR_MOD(g, stmt)                                                             \
    do {                                                                                \
        if ((g).cap > 0.f && (g).slopes) { constexpr bool kCap = true, kSlope = true; stmt; }   \
        else if ((g).cap > 0.f) { constexpr bool kCap = true, kSlope = false; stmt; }   \
        else if ((g).slopes) { constexpr bool kCap = false, kSlope = true; stmt; }      \
        else { constexpr bool kCap = false, kSlope = false; stmt; }                     \
    } while (0)

}  // namespace mod
}  // namespace bt
