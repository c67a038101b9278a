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
// of a turn, at most 1/2, then goes through sincospif in 32 bits (relative error 2^-23).
#include "common.cuh"

namespace bt {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxRows = 8;      // rows of one CTA
constexpr int kMaxPairs = 64;    // rot_dim / 2

template <bool VEC>
__global__ void __launch_bounds__(kThreads) rope_kernel(const RopeArgs g) {
    __shared__ float2 cs[kMaxRows * kMaxPairs];
    pdl_wait();
    pdl_trigger();
    const int64_t n0 = (int64_t)blockIdx.x * g.rows;
    const int rows = (int)min((int64_t)g.rows, g.N - n0);
    const int half = g.rot >> 1;
    for (int i = threadIdx.x; i < rows * half; i += kThreads) {
        const int r = i / half, k = i - r * half;
        const int64_t n = n0 + r;
        const int pos = g.pos ? g.pos[n] : (int)(n % g.T);
        const double turns = (double)pos * g.turns[k];
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        cs[r * half + k] = make_float2(c * g.mscale, s * g.sin_sign * g.mscale);
    }
    __syncthreads();

    const int d = g.C / g.H;
    const int64_t ld = 3 * (int64_t)g.C;
    const bool raw_in_place = g.y == g.x;
    // One unit of the vector form is four pairs of a head (half layout: two float4 a half apart;
    // interleaved: two neighbouring float4) or one float4 that passes through; of the scalar form one
    // pair or one element.  The units of a head come first the rotated, then the others; heads of q and
    // k before the values.  In place only the rotated ones exist.
    constexpr int W = VEC ? 4 : 1;
    const int rot_units = half / W, pass_units = raw_in_place ? 0 : (d - g.rot) / W;
    const int per_head = rot_units + pass_units, v_units = raw_in_place ? 0 : g.C / W;
    const int per_row = 2 * g.H * per_head + v_units;
#pragma unroll 4
    for (int u = threadIdx.x; u < rows * per_row; u += kThreads) {
        const int r = u / per_row, w = u - r * per_row;
        const int64_t row = (n0 + r) * ld;
        int64_t at;        // first (or only) piece
        int k = -1;        // first pair of the unit, -1: passes through
        if (w < 2 * g.H * per_head) {
            const int hd = w / per_head, j = w - hd * per_head;
            at = row + (int64_t)hd * d;     // heads of k follow those of q
            if (j < rot_units) {
                k = j * W;
                at += g.interleaved ? 2 * k : k;
            } else {
                at += g.rot + (j - rot_units) * W;
            }
        } else {
            at = row + 2 * (int64_t)g.C + (int64_t)(w - 2 * g.H * per_head) * W;
        }
        if (VEC) {
            float4 a = *reinterpret_cast<const float4*>(g.x + at);
            if (k < 0) {
                store_raw_split(a, g.y, g.y_hi, g.y_lo, at >> 2);
                continue;
            }
            const int64_t at2 = at + (g.interleaved ? 4 : half);
            float4 b = *reinterpret_cast<const float4*>(g.x + at2);
            const float2* t = cs + r * half + k;
            const float2 t0 = t[0], t1 = t[1], t2 = t[2], t3 = t[3];
            float4 oa, ob;
            if (g.interleaved) {
                oa = make_float4(a.x * t0.x - a.y * t0.y, a.x * t0.y + a.y * t0.x, a.z * t1.x - a.w * t1.y, a.z * t1.y + a.w * t1.x);
                ob = make_float4(b.x * t2.x - b.y * t2.y, b.x * t2.y + b.y * t2.x, b.z * t3.x - b.w * t3.y, b.z * t3.y + b.w * t3.x);
            } else {
                oa = make_float4(a.x * t0.x - b.x * t0.y, a.y * t1.x - b.y * t1.y, a.z * t2.x - b.z * t2.y, a.w * t3.x - b.w * t3.y);
                ob = make_float4(a.x * t0.y + b.x * t0.x, a.y * t1.y + b.y * t1.x, a.z * t2.y + b.z * t2.x, a.w * t3.y + b.w * t3.x);
            }
            store_raw_split(oa, g.y, g.y_hi, g.y_lo, at >> 2);
            store_raw_split(ob, g.y, g.y_hi, g.y_lo, at2 >> 2);
        } else {
            auto put = [&](int64_t i, float v) {
                if (g.y) g.y[i] = v;
                if (g.y_hi) {
                    float h, l;
                    split_tf32(v, h, l);
                    g.y_hi[i] = h;
                    g.y_lo[i] = l;
                }
            };
            const float a = g.x[at];
            if (k < 0) {
                put(at, a);
                continue;
            }
            const int64_t at2 = at + (g.interleaved ? 1 : half);
            const float b = g.x[at2];
            const float2 t = cs[r * half + k];
            put(at, a * t.x - b * t.y);
            put(at2, a * t.y + b * t.x);
        }
    }
}

}  // namespace

cudaError_t launch_rope(RopeArgs g, cudaStream_t s) {
    // Rows per CTA: at least 2,304 float4 of work (9 per thread), while a short array still spreads over
    // the SMs.
    const int64_t row4 = 3 * (int64_t)g.C / 4;
    int rows = (int)max((int64_t)1, min((int64_t)kMaxRows, (2304 + row4 - 1) / row4));
    while (rows > 1 && (g.N + rows - 1) / rows < 148) rows >>= 1;
    g.rows = rows;
    const int64_t grid = (g.N + rows - 1) / rows;
    if (grid > 0x7fffffff) return cudaErrorInvalidValue;
    if (g.rot % 8 == 0) BT_KERNEL_LAUNCH((rope_kernel<true>), (unsigned)grid, kThreads, 0, s, g);
    else BT_KERNEL_LAUNCH((rope_kernel<false>), (unsigned)grid, kThreads, 0, s, g);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

}  // namespace bt
