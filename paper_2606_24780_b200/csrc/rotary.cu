// Rotary position embedding on the fused qkv array: every pair (a, b) of the first rot_dim
// columns of each query and key head is turned by the angle position * theta_i,
//     a' = m (a cos - b sin),  b' = m (a sin + b cos),
// i the index of the pair, m the magnitude factor; the values, and the columns past rot_dim, pass
// through.  The backward is the same turn by the negative angle (a rotation's transpose).
//
// Bound by HBM: 8 bytes per element, and 6 operations per pair.  The angles are the only work beyond
// that: a row's rot_dim / 2 sines and cosines are formed once per CTA, in shared memory, and shared by
// its 2H heads.  The angle is reduced in 64 bits -- position * theta / 2 pi, the whole turns
// dropped -- because a 32-bit product is 0.01 radian off at position 131,072; the remaining fraction
// of a turn, at most 1/2, then goes through sincospif in 32 bits (relative error 2^-23).  The 64-bit product's own
// rounding grows with the position: 3e-7 radian at 2^31, below an FP32 rounding up to 2^28.
// 8,192 rows, 12 heads of 64: 27 us, 5.6 TB/s of a copy's 6.45; 32,762 rows, 16 heads of 64, half turned: 140 us, 5.7 TB/s.
#include "common.cuh"

namespace bt {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxRows = 8;      // rows of one CTA
constexpr int kMaxPairs = 64;    // rot_dim / 2

// n / d for n < 2^31 by multiplication: with 2^s < d <= 2^(s + 1), m = ceil(2^(32 + s) / d) has 32 bits, and its excess, below
// 2^-(32 + s) n of a quotient, is less than the 1 / d that a quotient may be off.  A row has at most 2 C units, C <= 2^26.
__device__ __forceinline__ uint32_t quotient(uint32_t n, const RopeArgs::Divisor& d) { return d.m ? __umulhi(n, d.m) >> d.s : n; }

// A thread group of the CTA owns a row.  First the columns that only move (the values, the tails of partly rotated
// heads), while the angles are formed; then the rotated ones.  Pieces are float4 (VEC) or single columns, kUnroll of them
// requested before the first is used.  In place the first part falls away.
template <bool VEC>
__global__ void __launch_bounds__(kThreads) rope_kernel(const RopeArgs g) {
    constexpr int W = VEC ? 4 : 1, kUnroll = VEC ? 4 : 8;
    __shared__ float2 cs[kMaxRows * kMaxPairs];
    pdl_wait();
    pdl_trigger();
    const int64_t n0 = (int64_t)blockIdx.x * g.rows;
    const int group = kThreads / g.rows, r = (int)threadIdx.x / group, t0 = (int)threadIdx.x - r * group;
    const int half = g.rot >> 1, d = g.C / g.H;
    for (int i = threadIdx.x; i < g.rows * half; i += kThreads) {
        const int row = i / half, k = i - row * half;
        const int64_t n = min(n0 + row, g.N - 1);
        const int pos = g.pos ? g.pos[n] : (int)(n % g.T);
        const double turns = (double)pos * g.turns[k];
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        cs[i] = make_float2(c * g.mscale, s * g.sin_sign * g.mscale);
    }
    const bool live = n0 + r < g.N;
    const int64_t row = (n0 + r) * 3 * (int64_t)g.C;
    auto get = [&](int64_t at) -> float4 { return VEC ? __ldcs(reinterpret_cast<const float4*>(g.x + at)) : make_float4(g.x[at], 0.f, 0.f, 0.f); };
    auto put = [&](int64_t at, const float4& v) {
        if (VEC) {
            store_raw_split(v, g.y, g.y_hi, g.y_lo, at >> 2);
        } else {
            if (g.y) g.y[at] = v.x;
            if (g.y_hi) split_tf32(v.x, g.y_hi[at], g.y_lo[at]);
        }
    };
    if (live && g.y != g.x) {
        const int pass = (d - g.rot) / W, heads = 2 * g.H * pass, total = heads + g.C / W;
        for (int t = t0; t < total; t += group * kUnroll) {
            float4 v[kUnroll];
            int64_t at[kUnroll];
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                const int u = t + k * group;
                if (u < heads) {
                    const uint32_t hd = quotient(u, g.pass);
                    at[k] = row + (int64_t)hd * d + g.rot + (u - (int)hd * pass) * W;
                } else {
                    at[k] = row + 2 * (int64_t)g.C + (int64_t)(u - heads) * W;
                }
                if (u < total) v[k] = get(at[k]);
            }
#pragma unroll
            for (int k = 0; k < kUnroll; ++k)
                if (t + k * group < total) put(at[k], v[k]);
        }
    }
    __syncthreads();
    if (!live) return;
    // a unit: W pairs of a head -- two pieces half a rotation apart, or (interleaved) next to one another
    const int per_head = half / W, total = 2 * g.H * per_head;
    const float2* angle = cs + r * half;
    for (int t = t0; t < total; t += group * kUnroll) {
        float4 a[kUnroll], b[kUnroll];
        int64_t at[kUnroll];
        int pair[kUnroll];
        const int64_t apart = g.interleaved ? W : half;
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            const int u = t + k * group;
            const uint32_t hd = quotient(u, g.head);
            pair[k] = (u - (int)hd * per_head) * W;
            at[k] = row + (int64_t)hd * d + (g.interleaved ? 2 * pair[k] : pair[k]);
            if (u < total) {
                a[k] = get(at[k]);
                b[k] = get(at[k] + apart);
            }
        }
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            if (t + k * group >= total) break;
            const float2* c = angle + pair[k];
            float4 oa, ob;
            if (!VEC) {
                oa.x = a[k].x * c[0].x - b[k].x * c[0].y;
                ob.x = a[k].x * c[0].y + b[k].x * c[0].x;
            } else if (g.interleaved) {
                const float2 c0 = c[0], c1 = c[1], c2 = c[2], c3 = c[3];
                oa = make_float4(a[k].x * c0.x - a[k].y * c0.y, a[k].x * c0.y + a[k].y * c0.x, a[k].z * c1.x - a[k].w * c1.y, a[k].z * c1.y + a[k].w * c1.x);
                ob = make_float4(b[k].x * c2.x - b[k].y * c2.y, b[k].x * c2.y + b[k].y * c2.x, b[k].z * c3.x - b[k].w * c3.y, b[k].z * c3.y + b[k].w * c3.x);
            } else {
                const float2 c0 = c[0], c1 = c[1], c2 = c[2], c3 = c[3];
                oa = make_float4(a[k].x * c0.x - b[k].x * c0.y, a[k].y * c1.x - b[k].y * c1.y, a[k].z * c2.x - b[k].z * c2.y, a[k].w * c3.x - b[k].w * c3.y);
                ob = make_float4(a[k].x * c0.y + b[k].x * c0.x, a[k].y * c1.y + b[k].y * c1.x, a[k].z * c2.y + b[k].z * c2.x, a[k].w * c3.y + b[k].w * c3.x);
            }
            put(at[k], oa);
            put(at[k] + apart, ob);
        }
    }
}

}  // namespace

cudaError_t launch_rope(RopeArgs g, cudaStream_t s) {
    // Rows per CTA (a power of two): 2,304 float4 of work (9 per thread) or more, while a short array still spreads over
    // the SMs.
    const int64_t row4 = 3 * (int64_t)g.C / 4;
    int rows = 1;
    while (rows < kMaxRows && rows * row4 < 2304 && (g.N + 2 * rows - 1) / (2 * rows) >= 148) rows *= 2;
    g.rows = rows;
    const int64_t grid = (g.N + rows - 1) / rows;
    if (grid > 0x7fffffff) return cudaErrorInvalidValue;
    const int w = g.rot % 8 == 0 ? 4 : 1;
    auto divisor = [](uint32_t d) -> RopeArgs::Divisor {
        if (d < 2) return {0u, 0u};
        uint32_t s = 0;
        while ((2u << s) < d) ++s;
        return {(uint32_t)(((0x100000000ull << s) + d - 1) / d), s};
    };
    g.head = divisor(g.rot / 2 / w);
    g.pass = divisor((g.C / g.H - g.rot) / w);
    if (g.rot % 8 == 0) BT_KERNEL_LAUNCH((rope_kernel<true>), (unsigned)grid, kThreads, 0, s, g);
    else BT_KERNEL_LAUNCH((rope_kernel<false>), (unsigned)grid, kThreads, 0, s, g);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

}  // namespace bt
