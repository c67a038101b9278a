// Attention with modified scores on warp-level MMA, 3xTF32: short sequences of heads of 16 and 32 columns.
//
// One CTA owns 64 rows of one head, 16 per warp, and walks the 64-row tiles of the other side between the ends
// of its rows' ranges; a warp skips the tiles none of its rows reads.  Streamed tiles go through
// double-buffered shared memory (row stride head_dim + 4 floats: conflict-free fragments), raw
// arrays by cp.async, planes added on the way in.  Every product is m16n8k8 TF32 three times on hi/lo
// splits.  The tensor core truncates as it accumulates, so the sums over a walk are taken per tile and added in
// FP32, the small terms (lo hi, hi lo) in accumulators of their own: 7e-6 of the output at 4,096 positions without.
//   forward  rows = queries, online softmax in base 2
//   dq       rows = queries; also D = rowsum(dO o O), which dkv reads
//   dkv      rows = keys
// Bound by issue: the splits in front of the products and the score function, on top of the legacy tensor pipe
// (gradients at 2,000 positions: pipe 47 % busy, 2.0 instructions a clock; 64 sequences of 128, 16 heads of 32: 31 %, 1.5 to 1.9, forward
// 61 us, gradients 203).  They serve calls that are over before that counts.
#include "attention_mod.cuh"

namespace bt {

using namespace mod;
using tc::ex2_approx;

namespace {

constexpr int kRows = 64, kThreads = 128;

__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void split_u(float x, uint32_t& hi, uint32_t& lo) {
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(hi) : "f"(x));
    lo = __float_as_uint(x - __uint_as_float(hi));
}

// 64 rows x HD floats from row0 on (rows past the last are read as the last: masked or never stored) into a
// shared tile of row stride HD + 4.  Raw arrays arrive asynchronously; the caller commits and waits.
template <int HD>
__device__ __forceinline__ void stage(const float* hi, const float* lo, int64_t stride, int row0, int T, float* dst) {
    constexpr int V4 = HD / 4;
    for (int i = threadIdx.x; i < kRows * V4; i += kThreads) {
        const int r = i / V4, c = 4 * (i - r * V4);
        const int64_t at = (int64_t)min(row0 + r, T - 1) * stride + c;
        float* d = dst + r * (HD + 4) + c;
        if (lo) {
            *reinterpret_cast<float4*>(d) = add4(ld4(hi + at, 0), ld4(lo + at, 0));
        } else {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(d)), "l"(hi + at) : "memory");
        }
    }
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_groups() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// This warp's 16 rows (r0 and r1 = r0 + 8 in this thread) times `mul` as split A fragments.
template <int HD>
__device__ __forceinline__ void row_frags(const float* hi, const float* lo, int64_t stride, int r0, int r1, int T, float mul,
                                          int t4, uint32_t (&a_hi)[HD / 8][4], uint32_t (&a_lo)[HD / 8][4]) {
    const int64_t at[2] = {(int64_t)min(r0, T - 1) * stride, (int64_t)min(r1, T - 1) * stride};
#pragma unroll
    for (int ks = 0; ks < HD / 8; ++ks)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t i = at[e & 1] + ks * 8 + t4 + 4 * (e >> 1);
            split_u((lo ? hi[i] + lo[i] : hi[i]) * mul, a_hi[ks][e], a_lo[ks][e]);
        }
}

// acc (16 x 64) = A . X^T, X a shared tile: B element (k, n) = X[n][k].
template <int HD>
__device__ __forceinline__ void rows_times_tile(float (&acc)[8][4], const uint32_t (&a_hi)[HD / 8][4],
                                                const uint32_t (&a_lo)[HD / 8][4], const float* x, int g, int t4) {
#pragma unroll
    for (int nt = 0; nt < 8; ++nt) acc[nt][0] = acc[nt][1] = acc[nt][2] = acc[nt][3] = 0.f;
#pragma unroll
    for (int ks = 0; ks < HD / 8; ++ks) {
        uint32_t bh[8][2], bl[8][2];
#pragma unroll
        for (int nt = 0; nt < 8; ++nt) {
            const int o = (nt * 8 + g) * (HD + 4) + ks * 8 + t4;
            split_u(x[o], bh[nt][0], bl[nt][0]);
            split_u(x[o + 4], bh[nt][1], bl[nt][1]);
        }
#pragma unroll
        for (int nt = 0; nt < 8; ++nt) mma_tf32(acc[nt], a_lo[ks], bh[nt][0], bh[nt][1]);
#pragma unroll
        for (int nt = 0; nt < 8; ++nt) mma_tf32(acc[nt], a_hi[ks], bl[nt][0], bl[nt][1]);
#pragma unroll
        for (int nt = 0; nt < 8; ++nt) mma_tf32(acc[nt], a_hi[ks], bh[nt][0], bh[nt][1]);
    }
}

// sum (16 x HD) += Z (16 x 64, in the accumulator layout) . X.  Columns 2 t4, 2 t4 + 1 of Z serve as the contraction
// indices t4, t4 + 4, so B element (k, n) = X[nt * 8 + 2 t4 (+ 1)][n].
template <int HD>
__device__ __forceinline__ void add_z_times_tile(float (&sum)[HD / 8][4], const float (&z)[32], const float* x, int g, int t4) {
    float big[HD / 8][4], small[HD / 8][4];
#pragma unroll
    for (int dt = 0; dt < HD / 8; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) big[dt][e] = small[dt][e] = 0.f;
#pragma unroll
    for (int nt = 0; nt < 8; ++nt) {
        uint32_t a_hi[4], a_lo[4], bh[HD / 8][2], bl[HD / 8][2];
        split_u(z[4 * nt], a_hi[0], a_lo[0]);
        split_u(z[4 * nt + 2], a_hi[1], a_lo[1]);
        split_u(z[4 * nt + 1], a_hi[2], a_lo[2]);
        split_u(z[4 * nt + 3], a_hi[3], a_lo[3]);
#pragma unroll
        for (int dt = 0; dt < HD / 8; ++dt) {
            const int o = (nt * 8 + 2 * t4) * (HD + 4) + dt * 8 + g;
            split_u(x[o], bh[dt][0], bl[dt][0]);
            split_u(x[o + HD + 4], bh[dt][1], bl[dt][1]);
        }
#pragma unroll
        for (int dt = 0; dt < HD / 8; ++dt) mma_tf32(small[dt], a_lo, bh[dt][0], bh[dt][1]);
#pragma unroll
        for (int dt = 0; dt < HD / 8; ++dt) mma_tf32(small[dt], a_hi, bl[dt][0], bl[dt][1]);
#pragma unroll
        for (int dt = 0; dt < HD / 8; ++dt) mma_tf32(big[dt], a_hi, bh[dt][0], bh[dt][1]);
    }
#pragma unroll
    for (int dt = 0; dt < HD / 8; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[dt][e] += big[dt][e] + small[dt][e];
}

__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
    return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
}
__device__ __forceinline__ float quad_sum(float v) {
    v += __shfl_xor_sync(0xffffffffu, v, 1);
    return v + __shfl_xor_sync(0xffffffffu, v, 2);
}

// Element 4 nt + e of a thread's 16 x 64 tile: row r0 (e < 2) or r1, column 8 nt + 2 t4 + (e & 1).
__device__ __forceinline__ int column(int i, int t4) { return 8 * (i >> 2) + 2 * t4 + (i & 1); }

// Score products (own rows already times the score unit) -> modified scores in base-2 units, and 1 - tanh^2.
template <bool CAP, bool SLOPE>
__device__ __forceinline__ void modify(float (&x)[32], float (&grad)[32], const Score& sc, int r0, int tile0, int t4) {
    score_tile<CAP, false, true, false, 32>(x, grad, sc, 0, 0.f);
    if (SLOPE) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            x[i] = fmaf(-sc.slope2, fabsf((float)(r0 + ((i & 2) ? 8 : 0) - tile0 - column(i, t4))), x[i]);
    }
}
__device__ __forceinline__ bool reads(int i, int t4, int tile0, const int2 (&span)[2]) {
    const int c = tile0 + column(i, t4);
    const int2 s = span[(i >> 1) & 1];
    return c >= s.x && c < s.y;
}
// Whether this warp's rows read any, or all, of the 64 rows from tile0 on.
__device__ __forceinline__ bool any_reads(int tile0, const int2 (&span)[2]) {
    return __any_sync(0xffffffffu, (span[0].x < tile0 + 64 && span[0].y > tile0) || (span[1].x < tile0 + 64 && span[1].y > tile0));
}
__device__ __forceinline__ bool all_read(int tile0, const int2 (&span)[2]) {
    return span[0].x <= tile0 && span[0].y >= tile0 + 64 && span[1].x <= tile0 && span[1].y >= tile0 + 64;
}

template <int HD>
__device__ __forceinline__ void store(const float (&v)[HD / 8][4], float m0, float m1, int r0, int r1, int T, int t4, int64_t at,
                                      int64_t stride, float* raw, float* hi, float* lo) {
#pragma unroll
    for (int dt = 0; dt < HD / 8; ++dt)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int r = half ? r1 : r0;
            if (r >= T) continue;
            const float m = half ? m1 : m0;
            const float2 x = make_float2(v[dt][2 * half] * m, v[dt][2 * half + 1] * m);
            const int64_t i = at + (int64_t)r * stride + dt * 8 + 2 * t4;
            if (raw) *reinterpret_cast<float2*>(raw + i) = x;
            if (hi) {
                float2 h, l;
                split_tf32(x.x, h.x, l.x);
                split_tf32(x.y, h.y, l.y);
                *reinterpret_cast<float2*>(hi + i) = h;
                *reinterpret_cast<float2*>(lo + i) = l;
            }
        }
}

// What the three kernels share: the CTA's head and rows, and the tiles it walks.
struct Work {
    int b, h, r0, r1, tile, tiles, warp, g, t4;
    int64_t ld, head, stat;     // row stride of qkv, its row 0 of this head, row 0 of lse / dvec
    int2 span[2];
};
__device__ __forceinline__ Work make_work(const AttnModArgs& g, int hd, bool keys) {
    Work w;
    w.b = (int)blockIdx.y / g.H;
    w.h = (int)blockIdx.y % g.H;
    const int lane = threadIdx.x & 31;
    w.warp = threadIdx.x >> 5;
    w.g = lane >> 2;
    w.t4 = lane & 3;
    // causal walks: the longest first
    const int blk = keys ? (int)blockIdx.x : (int)gridDim.x - 1 - (int)blockIdx.x;
    w.r0 = blk * kRows + w.warp * 16 + w.g;
    w.r1 = w.r0 + 8;
    w.ld = 3 * (int64_t)g.C;
    w.head = (int64_t)w.b * g.T * w.ld + (int64_t)w.h * hd;
    w.stat = ((int64_t)w.b * g.H + w.h) * g.T;
    const int2 range = block_range(keys ? g.spans.qblock : g.spans.kblock, w.b, g.T, blk * kRows, kRows, keys);
    w.tile = range.x / 64;
    w.tiles = range.x < range.y ? (range.y - 1) / 64 + 1 - w.tile : 0;
    w.span[0] = row_range(keys ? g.spans.q : g.spans.k, w.b, g.T, w.r0, keys);
    w.span[1] = row_range(keys ? g.spans.q : g.spans.k, w.b, g.T, w.r1, keys);
    return w;
}
__device__ __forceinline__ const float* plus(const float* p, int64_t n) { return p ? p + n : nullptr; }

template <int HD, bool CAP, bool SLOPE>
__global__ void __launch_bounds__(kThreads, 2) fwd_kernel(const AttnModArgs g) {
    constexpr int TILE = kRows * (HD + 4);
    extern __shared__ float sm[];   // K[2], V[2]
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *g.err = 0;
    const Work w = make_work(g, HD, false);
    const Score sc = make_score<CAP, SLOPE>(1.0f / sqrtf((float)HD), g.cap, g.slopes, w.h);
    const float *q = g.qkv + w.head, *q_lo = plus(g.qkv_lo, w.head);
    auto load = [&](int t) {
        stage<HD>(q + g.C, plus(q_lo, g.C), w.ld, (w.tile + t) * 64, g.T, sm + (t & 1) * TILE);
        stage<HD>(q + 2 * (int64_t)g.C, plus(q_lo, 2 * (int64_t)g.C), w.ld, (w.tile + t) * 64, g.T, sm + (2 + (t & 1)) * TILE);
        commit();
    };
    if (w.tiles > 0) load(0);
    uint32_t q_hi[HD / 8][4], q_l[HD / 8][4];
    row_frags<HD>(q, q_lo, w.ld, w.r0, w.r1, g.T, sc.unit, w.t4, q_hi, q_l);
    float o[HD / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < HD / 8; ++dt) o[dt][0] = o[dt][1] = o[dt][2] = o[dt][3] = 0.f;
    for (int t = 0; t < w.tiles; ++t) {
        if (t + 1 < w.tiles) {
            load(t + 1);
            wait_groups<1>();
        } else {
            wait_groups<0>();
        }
        __syncthreads();
        const int k0 = (w.tile + t) * 64;
        if (any_reads(k0, w.span)) {
            float s[8][4], x[32], none[32];
            rows_times_tile<HD>(s, q_hi, q_l, sm + (t & 1) * TILE, w.g, w.t4);
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = s[i >> 2][i & 3];
            modify<CAP, SLOPE>(x, none, sc, w.r0, k0, w.t4);
            if (!all_read(k0, w.span)) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (!reads(i, w.t4, k0, w.span)) x[i] = -INFINITY;
            }
            float top[2] = {-INFINITY, -INFINITY}, use[2];
#pragma unroll
            for (int i = 0; i < 32; ++i) top[(i >> 1) & 1] = fmaxf(top[(i >> 1) & 1], x[i]);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float mn = fmaxf(m[r], quad_max(top[r]));
                use[r] = mn == -INFINITY ? 0.f : mn;         // a row that has read nothing yet
                const float corr = ex2_approx(m[r] - use[r]);
                m[r] = mn;
                l[r] *= corr;
#pragma unroll
                for (int dt = 0; dt < HD / 8; ++dt) {
                    o[dt][2 * r] *= corr;
                    o[dt][2 * r + 1] *= corr;
                }
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                x[i] = ex2_approx(x[i] - use[(i >> 1) & 1]);
                l[(i >> 1) & 1] += x[i];
            }
            add_z_times_tile<HD>(o, x, sm + (2 + (t & 1)) * TILE, w.g, w.t4);
        }
        __syncthreads();   // everyone is done with this buffer before it is refilled
    }
    float inv[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] = quad_sum(l[r]);
        inv[r] = row_factor(l[r], w.span[r]);
        const int row = r ? w.r1 : w.r0;
        if (w.t4 == 0 && row < g.T) g.lse[w.stat + row] = row_lse(m[r], l[r], w.span[r]);
    }
    store<HD>(o, inv[0], inv[1], w.r0, w.r1, g.T, w.t4, (int64_t)w.b * g.T * g.C + (int64_t)w.h * HD, g.C, g.o, g.o_hi, g.o_lo);
}

template <int HD, bool CAP, bool SLOPE>
__global__ void __launch_bounds__(kThreads, 2) dq_kernel(const AttnModArgs g) {
    constexpr int TILE = kRows * (HD + 4);
    extern __shared__ float sm[];   // K[2], V[2]
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *g.err = 0;
    const Work w = make_work(g, HD, false);
    const float scale = 1.0f / sqrtf((float)HD);
    const Score sc = make_score<CAP, SLOPE>(scale, g.cap, g.slopes, w.h);
    const float *q = g.qkv + w.head, *q_lo = plus(g.qkv_lo, w.head);
    auto load = [&](int t) {
        stage<HD>(q + g.C, plus(q_lo, g.C), w.ld, (w.tile + t) * 64, g.T, sm + (t & 1) * TILE);
        stage<HD>(q + 2 * (int64_t)g.C, plus(q_lo, 2 * (int64_t)g.C), w.ld, (w.tile + t) * 64, g.T, sm + (2 + (t & 1)) * TILE);
        commit();
    };
    if (w.tiles > 0) load(0);
    uint32_t q_hi[HD / 8][4], q_l[HD / 8][4], d_hi[HD / 8][4], d_l[HD / 8][4];
    row_frags<HD>(q, q_lo, w.ld, w.r0, w.r1, g.T, sc.unit, w.t4, q_hi, q_l);
    const int64_t oat = (int64_t)w.b * g.T * g.C + (int64_t)w.h * HD;
    row_frags<HD>(g.d_o + oat, plus(g.d_o_lo, oat), g.C, w.r0, w.r1, g.T, 1.0f, w.t4, d_hi, d_l);
    float D[2] = {0.f, 0.f}, L[2], dq[HD / 8][4];
#pragma unroll
    for (int ks = 0; ks < HD / 8; ++ks)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = min((e & 1) ? w.r1 : w.r0, g.T - 1);
            D[e & 1] = fmaf(__uint_as_float(d_hi[ks][e]) + __uint_as_float(d_l[ks][e]),
                            g.o[oat + (int64_t)row * g.C + ks * 8 + w.t4 + 4 * (e >> 1)], D[e & 1]);
            dq[ks][e] = 0.f;
        }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = r ? w.r1 : w.r0;
        D[r] = quad_sum(D[r]);
        L[r] = g.lse[w.stat + min(row, g.T - 1)] * kLog2e;
        if (w.t4 == 0 && row < g.T) g.dvec[w.stat + row] = D[r];
    }
    for (int t = 0; t < w.tiles; ++t) {
        if (t + 1 < w.tiles) {
            load(t + 1);
            wait_groups<1>();
        } else {
            wait_groups<0>();
        }
        __syncthreads();
        const int k0 = (w.tile + t) * 64;
        if (any_reads(k0, w.span)) {
            float s[8][4], dp[8][4], x[32], f[32];
            rows_times_tile<HD>(s, q_hi, q_l, sm + (t & 1) * TILE, w.g, w.t4);
            rows_times_tile<HD>(dp, d_hi, d_l, sm + (2 + (t & 1)) * TILE, w.g, w.t4);
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = s[i >> 2][i & 3];
            modify<CAP, SLOPE>(x, f, sc, w.r0, k0, w.t4);
            const bool whole = all_read(k0, w.span);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                float p = ex2_approx(x[i] - L[(i >> 1) & 1]);
                if (!whole && !reads(i, w.t4, k0, w.span)) p = 0.f;
                x[i] = p * (dp[i >> 2][i & 3] - D[(i >> 1) & 1]);
                if (CAP) x[i] *= f[i];
            }
            add_z_times_tile<HD>(dq, x, sm + (t & 1) * TILE, w.g, w.t4);
        }
        __syncthreads();
    }
    store<HD>(dq, scale, scale, w.r0, w.r1, g.T, w.t4, w.head, w.ld, g.dqkv, g.dqkv_hi, g.dqkv_lo);
}

template <int HD, bool CAP, bool SLOPE>
__global__ void __launch_bounds__(kThreads, 2) dkv_kernel(const AttnModArgs g) {
    constexpr int TILE = kRows * (HD + 4);
    extern __shared__ float sm[];   // Q[2], dO[2], then lse[2][64], D[2][64]
    pdl_wait();
    pdl_trigger();
    const Work w = make_work(g, HD, true);
    const float scale = 1.0f / sqrtf((float)HD);
    const Score sc = make_score<CAP, SLOPE>(scale, g.cap, g.slopes, w.h);
    const float *q = g.qkv + w.head, *q_lo = plus(g.qkv_lo, w.head);
    const int64_t oat = (int64_t)w.b * g.T * g.C + (int64_t)w.h * HD;
    float* stats = sm + 4 * TILE;
    auto load = [&](int t) {
        const int q0 = (w.tile + t) * 64;
        stage<HD>(q, q_lo, w.ld, q0, g.T, sm + (t & 1) * TILE);
        stage<HD>(g.d_o + oat, plus(g.d_o_lo, oat), g.C, q0, g.T, sm + (2 + (t & 1)) * TILE);
        commit();
        const int r = min(q0 + (int)(threadIdx.x & 63), g.T - 1);      // rows past the end are masked below
        stats[(t & 1) * 128 + threadIdx.x] = threadIdx.x < 64 ? g.lse[w.stat + r] * kLog2e : g.dvec[w.stat + r];
    };
    if (w.tiles > 0) load(0);
    uint32_t k_hi[HD / 8][4], k_l[HD / 8][4], v_hi[HD / 8][4], v_l[HD / 8][4];
    row_frags<HD>(q + g.C, plus(q_lo, g.C), w.ld, w.r0, w.r1, g.T, sc.unit, w.t4, k_hi, k_l);
    row_frags<HD>(q + 2 * (int64_t)g.C, plus(q_lo, 2 * (int64_t)g.C), w.ld, w.r0, w.r1, g.T, 1.0f, w.t4, v_hi, v_l);
    float dk[HD / 8][4], dv[HD / 8][4];
#pragma unroll
    for (int dt = 0; dt < HD / 8; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) dk[dt][e] = dv[dt][e] = 0.f;
    for (int t = 0; t < w.tiles; ++t) {
        if (t + 1 < w.tiles) {
            load(t + 1);
            wait_groups<1>();
        } else {
            wait_groups<0>();
        }
        __syncthreads();
        const int q0 = (w.tile + t) * 64;
        if (any_reads(q0, w.span)) {
            const float *q_s = sm + (t & 1) * TILE, *do_s = sm + (2 + (t & 1)) * TILE;
            const float *Ls = stats + (t & 1) * 128, *Ds = Ls + 64;
            float s[8][4], x[32], f[32];
            rows_times_tile<HD>(s, k_hi, k_l, q_s, w.g, w.t4);              // S^T = K Q^T
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = s[i >> 2][i & 3];
            modify<CAP, SLOPE>(x, f, sc, w.r0, q0, w.t4);
            const bool whole = all_read(q0, w.span);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                x[i] = ex2_approx(x[i] - Ls[column(i, w.t4)]);
                if (!whole && !reads(i, w.t4, q0, w.span)) x[i] = 0.f;
            }
            add_z_times_tile<HD>(dv, x, do_s, w.g, w.t4);                   // dV += P^T dO
            rows_times_tile<HD>(s, v_hi, v_l, do_s, w.g, w.t4);             // dP^T = V dO^T
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                x[i] *= s[i >> 2][i & 3] - Ds[column(i, w.t4)];
                if (CAP) x[i] *= f[i];
            }
            add_z_times_tile<HD>(dk, x, q_s, w.g, w.t4);                    // dK += dS^T Q
        }
        __syncthreads();
    }
    store<HD>(dk, scale, scale, w.r0, w.r1, g.T, w.t4, w.head + g.C, w.ld, g.dqkv, g.dqkv_hi, g.dqkv_lo);
    store<HD>(dv, 1.0f, 1.0f, w.r0, w.r1, g.T, w.t4, w.head + 2 * (int64_t)g.C, w.ld, g.dqkv, g.dqkv_hi, g.dqkv_lo);
}

template <int HD>
constexpr int smem_bytes() { return (4 * kRows * (HD + 4) + 256) * (int)sizeof(float); }

template <auto KERNEL>
cudaError_t go(int smem, const AttnModArgs& g, cudaStream_t s) {
    const cudaError_t e = allow_smem<KERNEL>(smem);
    if (e != cudaSuccess) return e;
    BT_KERNEL_LAUNCH(KERNEL, dim3((g.T + kRows - 1) / kRows, g.B * g.H), kThreads, smem, s, g);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

template <int HD>
cudaError_t fwd(const AttnModArgs& g, cudaStream_t s) {
    BT_FOR_MOD(g, return (go<fwd_kernel<HD, kCap, kSlope>>(smem_bytes<HD>(), g, s)));
}
template <int HD>
cudaError_t bwd(const AttnModArgs& g, cudaStream_t s) {
    cudaError_t e;
    BT_FOR_MOD(g, {
        if ((e = go<dq_kernel<HD, kCap, kSlope>>(smem_bytes<HD>(), g, s)) != cudaSuccess) return e;   // first: it forms D
        return go<dkv_kernel<HD, kCap, kSlope>>(smem_bytes<HD>(), g, s);
    });
}

}  // namespace

// grid.y is the sequence-head: at most 65,535 of them.
bool attention_mod_mma_supports(const AttnModArgs& g) { return g.C / g.H <= 32 && (int64_t)g.B * g.H <= 65535; }

cudaError_t launch_attention_mod_fwd_mma(const AttnModArgs& g, cudaStream_t s) {
    return g.C / g.H == 16 ? fwd<16>(g, s) : fwd<32>(g, s);
}
cudaError_t launch_attention_mod_bwd_mma(const AttnModArgs& g, cudaStream_t s) {
    return g.C / g.H == 16 ? bwd<16>(g, s) : bwd<32>(g, s);
}

}  // namespace bt
