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
// reweighted to the smallest largest relative error, 4.7e-9, a tenth of an FP32 rounding); above,
// 1 - 2 / (1 + e^2|u|), which is good to 2^-22 there.
constexpr float kTanhSmall = 0.6f;
constexpr float kTanh0 = -0.33333298563957214f, kTanh1 = 0.13331924378871918f, kTanh2 = -0.053783830255270004f,
                kTanh3 = 0.020795971155166626f, kTanh4 = -0.005895158275961876f;
__device__ __forceinline__ float tanh_small(float u) {
    const float w = u * u;
    float q = fmaf(w, kTanh4, kTanh3);
    q = fmaf(w, q, kTanh2);
    q = fmaf(w, q, kTanh1);
    q = fmaf(w, q, kTanh0);
    return fmaf(u * w, q, u);
}
// `grad`: 1 - tanh^2.  From a rounded tanh it would cancel as |u| grows (wrong by 1e-3 at 6, zero from 9 on); above 0.6 it is
// 4 r (1 - r), r = 1 / (1 + e^2|u|), without a difference of nearly equal numbers.
__device__ __forceinline__ float tanh_any(float u, float& grad) {
    const float r = rcp_fast(1.0f + ex2_fast(2.8853900817779268f * fabsf(u))), small = tanh_small(u);
    const bool is_small = fabsf(u) < kTanhSmall;
    grad = is_small ? fmaf(-small, small, 1.0f) : 4.0f * fmaf(-r, r, r);
    return is_small ? small : copysignf(fmaf(-2.0f, r, 1.0f), u);
}
__device__ __forceinline__ float tanh_any(float u) {
    float unused;
    return tanh_any(u, unused);
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
// x: N neighbouring scores of one row -> modified scores in base-2 units, less ref.  UNIT: x holds plain dot products;
// otherwise they carry s.unit already.  |first - i| is the distance of position i; `grad` (GRAD and CAP) receives
// 1 - tanh^2.  The exponential and the reciprocal of tanh run at an eighth of the rate of a multiplication and are
// needed only where some score of the N is beyond 0.6 caps.  A distance is linear in i unless the row lies inside the N
// positions (no integer conversion per element: it runs at an eighth of the rate too); counted down to a position near
// the row, a distance would keep the rounding of the far end, so there each is formed by itself.  __fadd_rn: the same roundings
// whether ref is known to be zero or not (a sum fused with the bias's product would have another).
template <bool CAP, bool SLOPE, bool GRAD, bool UNIT, int N>
__device__ __forceinline__ void score_tile(float (&x)[N], float (&grad)[N], const Score& s, int first, float ref) {
    if (CAP) {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (UNIT) x[i] *= s.unit;
            top = fmaxf(top, fabsf(x[i]));
        }
        if (top < kTanhSmall) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[i] = tanh_small(x[i]);
                if (GRAD) grad[i] = fmaf(-x[i], x[i], 1.0f);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float f;
                x[i] = tanh_any(x[i], f);
                if (GRAD) grad[i] = f;
            }
        }
    }
    constexpr bool kScale = CAP || UNIT;
    const float scale = CAP ? s.to_log2 : s.unit;
    if (SLOPE) {
        const float d = (float)first;
        if (first >= 2 * N || first <= 0) {
            const float step = first <= 0 ? -s.slope2 : s.slope2, start = fmaf(-step, d, -ref);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float bias = fmaf(step, (float)i, start);
                x[i] = kScale ? fmaf(x[i], scale, bias) : __fadd_rn(x[i], bias);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float bias = fmaf(-s.slope2, fabsf(d - (float)i), -ref);
                x[i] = kScale ? fmaf(x[i], scale, bias) : __fadd_rn(x[i], bias);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = kScale ? fmaf(x[i], scale, -ref) : x[i] - ref;
    }
}

// The reference that a tile's scores are taken less of before the exponential.  Usually score_tile subtracts it inside a fused
// operation, unrounded.  Where it or a bias reaches 2^24, a score's own rounding is a unit of the exponent or more, and the
// fused difference would be that rounding's, up to any size; there the rounded score less the reference, which is the largest
// of the same rounded scores: never above zero (tanh may be a rounding out of order), and zero for the largest.
struct Reference {
    float now, later;
    bool far;               // some row of the warp: uniform
};
// slope2, distance: the bias of no column of the tile is larger than their product.
__device__ __forceinline__ Reference make_reference(float ref, float slope2, int distance) {
    const bool far = __any_sync(0xffffffffu, fmaxf(fabsf(ref), fabsf(slope2) * (float)distance) >= 16777216.0f);
    return {far ? 0.f : ref, ref, far};
}
template <int N>
__device__ __forceinline__ void less_reference(float (&z)[N], const Reference& r) {
    if (!r.far) return;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        z[i] -= r.later;
        z[i] = z[i] > 0.f ? 0.f : z[i];     // not fminf: NaN stays
    }
}

// Rows [lo, hi) that `rows` own rows from r0 on have to walk (64-row blocks; without spans: causal).  Whatever the table
// holds -- it may have been built for other lengths -- a walk stays inside the sequence.
__device__ __forceinline__ int2 block_range(const int2* blocks, int b, int T, int r0, int rows, bool keys) {
    if (!blocks) return keys ? make_int2(r0, T) : make_int2(0, min(r0 + rows, T));
    const int nb = (T + 63) >> 6;
    int2 u = make_int2(0x7fffffff, 0);
    for (int k = r0 >> 6; k < min((r0 + rows + 63) >> 6, nb); ++k) {
        const int2 v = blocks[(int64_t)b * nb + k];
        if (v.x < v.y) u = make_int2(min(u.x, v.x), max(u.y, v.y));
    }
    return make_int2(max(min(u.x, T), 0), max(min(u.y, T), 0));
}
// The range of one own row, inside the sequence too; empty past its end.
__device__ __forceinline__ int2 row_range(const int2* spans, int b, int T, int row, bool keys) {
    if (row >= T) return make_int2(0, 0);
    if (!spans) return keys ? make_int2(row, T) : make_int2(0, row + 1);
    const int2 s = spans[(int64_t)b * T + row];
    return make_int2(max(s.x, 0), min(s.y, T));
}

// The factor of a row's output and its lse, from its maximum (base 2) and sum.  A row that reads nothing has weight zero
// and lse -inf; one whose scores left FP32's range is not a number in both, also if every one of them is -inf.
__device__ __forceinline__ float row_factor(float l, int2 span) {
    return l != 0.f ? 1.0f / l : span.x < span.y ? __int_as_float(0x7fffffff) : 0.f;
}
__device__ __forceinline__ float row_lse(float m, float l, int2 span) {
    return l != 0.f ? (m + log2f(l)) * kLn2 : span.x < span.y ? __int_as_float(0x7fffffff) : -INFINITY;
}

// ---------------------------------------------------------------- pieces of the persistent kernels
// One lane of a converged warp.  The issuing roles run on whole warps and put only the products behind this: the
// compiler then keeps their descriptors in uniform registers, and an MMA is issued every 16 clocks at N = 32 and every 32 at N = 64,
// which is the pipe's own rate.  (Behind a test of the lane number each descriptor is moved there by
// itself: 45 to 60 clocks an MMA, whatever its shape.)
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
    return p != 0;
}

// Register split of a kernel of several warpgroups: each gives up or takes registers of the block's launch total.
template <int N>
__device__ __forceinline__ void set_regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void set_regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

__device__ __forceinline__ void tmem_ldn(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr));
}
__device__ __forceinline__ void tmem_stn(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_ldn(uint32_t taddr, uint32_t (&r)[32]) { tc::tmem_ld32(taddr, r); }
__device__ __forceinline__ void tmem_stn(uint32_t taddr, const uint32_t (&r)[32]) { tc::tmem_st32(taddr, r); }

// A thread that owns a row reads and writes it in whole 32-byte sectors: no staging through shared memory, which the
// next work item's tiles already occupy.
__device__ __forceinline__ void ld_sector(const float* p, float (&v)[8]) {
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "l"(p));
}
__device__ __forceinline__ void st_sector(float* p, const float (&v)[8]) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
                 "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
}

__device__ __forceinline__ void load_sector(const float* p, float (&v)[8]) {
    if ((reinterpret_cast<uintptr_t>(p) & 31u) == 0) {
        ld_sector(p, v);
    } else {
        const float4 a = ld4(p, 0), b = ld4(p, 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
}
// Eight values of a row to the raw array and / or the planes.  Rows start on 16 bytes only (C is a multiple of 16
// floats, and so is every head's first column, but the caller's pointer need not be 32-byte aligned).
__device__ __forceinline__ void store_sector(const float (&v)[8], int64_t at, float* raw, float* hi, float* lo) {
    auto put = [](float* p, const float (&x)[8]) {
        if ((reinterpret_cast<uintptr_t>(p) & 31u) == 0) {
            st_sector(p, x);
        } else {
            *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
            *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
        }
    };
    if (raw) put(raw + at, v);
    if (hi) {
        float a[8], b[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) split_tf32(v[e], a[e], b[e]);
        put(hi + at, a);
        put(lo + at, b);
    }
}

// Work items of a persistent kernel are the CTAs of its grid: a running CTA takes over one that has not started
// (cluster launch control), so that a free SM always gets the next item and an item's prologue and epilogue
// overlap its neighbours.  One thread asks; the answer is 16 bytes in shared memory.
__device__ __forceinline__ void ask_next(uint32_t answer, uint32_t bar) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the previous answer has been read
    tc::mbar_expect_tx(bar, 16u);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(answer), "r"(bar) : "memory");
}
// Whether there is a next item; x, y its block index.  Not to be asked again after a "no".
__device__ __forceinline__ bool next_item(uint32_t answer, int& x, int& y) {
    uint32_t ok, cx = 0, cy = 0;
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b128 h;\n\t.reg .b32 z;\n\t"
        "ld.shared.b128 h, [%3];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n\t"
        "selp.u32 %2, 1, 0, p;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%0, %1, z, _}, h;\n\t}"
        : "+r"(cx), "+r"(cy), "=r"(ok) : "r"(answer) : "memory");
    x = (int)cx;
    y = (int)cy;
    return ok != 0;
}
// grouped_block for a given linear block index.
__device__ __forceinline__ void grouped_item(int head_group, int id, int& bh, int& y) {
    const int nh = (int)gridDim.x, ny = (int)gridDim.y;
    const int G = (head_group > 0 && head_group < nh) ? head_group : nh;
    const int per = G * ny, grp = id / per, rem = id - grp * per;
    const int first = grp * G, heads = min(G, nh - first);
    y = rem / heads;
    bh = first + (rem - y * heads);
}
// What an item is, for all roles: written by the scheduling thread, two deep.
struct Item {
    int bh, blk, t0, n;      // n tiles from tile t0 on; n < 0: no more items
};
// Item i for one role (a thread, or a whole warp); false when the wait ran out.
__device__ __forceinline__ bool get_item(const volatile Item* info, uint32_t full, uint32_t empty, int i, Item& it, int* err, bool whole_warp) {
    const uint32_t parity = (uint32_t)(i >> 1) & 1u, at = 8u * (uint32_t)(i & 1);
    if (!(whole_warp ? tc::mbar_wait_warp(full + at, parity, err, 110) : tc::mbar_wait(full + at, parity, err, 110))) return false;
    it.bh = info[i & 1].bh; it.blk = info[i & 1].blk; it.t0 = info[i & 1].t0; it.n = info[i & 1].n;
    if (whole_warp) __syncwarp();
    if (!whole_warp || (threadIdx.x & 31) == 0) tc::mbar_arrive(empty + at);
    return true;
}
// Hands item i to the other roles.
__device__ __forceinline__ bool put_item(volatile Item* info, uint32_t full, uint32_t empty, int i, const Item& it, int* err) {
    const uint32_t at = 8u * (uint32_t)(i & 1);
    if (!tc::mbar_wait(empty + at, ((uint32_t)(i >> 1) & 1u) ^ 1u, err, 119)) return false;
    info[i & 1].bh = it.bh; info[i & 1].blk = it.blk; info[i & 1].t0 = it.t0; info[i & 1].n = it.n;
    tc::mbar_arrive(full + at);
    return true;
}
// The item of block (x, y): its rows' range as tiles of `tile` rows.
__device__ __forceinline__ Item make_item(const AttnModArgs& g, int head_group, int x, int y, bool keys, int rows, int tile) {
    Item it;
    int yb;
    grouped_item(head_group, y * (int)gridDim.x + x, it.bh, yb);
    it.blk = keys ? yb : (int)gridDim.y - 1 - yb;        // causal walks: the longest first
    const int2 r = block_range(keys ? g.spans.qblock : g.spans.kblock, it.bh / g.H, g.T, it.blk * rows, rows, keys);
    it.t0 = r.x / tile;
    it.n = r.x < r.y ? (r.y - 1) / tile + 1 - it.t0 : 0;
    return it;
}

// Bit k set: column k0 + k lies in the range (N <= 32 columns; the tests of single bits are an instruction each).
template <int N>
__device__ __forceinline__ uint32_t column_bits(int2 span, int k0) {
    const int lo = min(max(span.x - k0, 0), N), hi = min(max(span.y - k0, 0), N);
    const uint32_t below_hi = hi >= 32 ? 0xffffffffu : (1u << hi) - 1u, below_lo = lo >= 32 ? 0xffffffffu : (1u << lo) - 1u;
    return below_hi & ~below_lo;
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
#define BT_FOR_MOD(g, ...)                                                             \
    do {                                                                                \
        if ((g).cap > 0.f && (g).slopes) { constexpr bool kCap = true, kSlope = true; __VA_ARGS__; }   \
        else if ((g).cap > 0.f) { constexpr bool kCap = true, kSlope = false; __VA_ARGS__; }   \
        else if ((g).slopes) { constexpr bool kCap = false, kSlope = true; __VA_ARGS__; }      \
        else { constexpr bool kCap = false, kSlope = false; __VA_ARGS__; }                     \
    } while (0)

}  // namespace mod
}  // namespace bt
