// Attention with modified scores in plain FP32: the reference for the tensor-core kernels, selected
// with BT_FLAG_ATTN_SIMT.  One warp owns one (sequence, head,
// position); lanes own head columns; every dot product is a warp-shuffle reduction.  The forward is the
// textbook two-pass softmax, deliberately not the one-pass recurrence of the fast kernels.
//     z_ij = c tanh(q_i k_j / (c sqrt d)) - slope |i - j|     (c = 0: z_ij = q_i k_j / sqrt d - slope |i - j|)
//     dz_ij / d(q_i k_j) = (1 - tanh^2) / sqrt d
#include "attention_mod.cuh"

namespace bt {

namespace {

constexpr int kWarps = 8;

// Value of an array given raw (lo null) or as hi/lo planes.
template <int DPL>
__device__ __forceinline__ void load_row(const float* hi, const float* lo, int64_t at, int d, int lane, float (&r)[DPL]) {
#pragma unroll
    for (int k = 0; k < DPL; ++k) {
        const int c = lane + 32 * k;
        r[k] = 0.f;
        if (c < d) r[k] = lo ? hi[at + c] + lo[at + c] : hi[at + c];
    }
}
template <int DPL>
__device__ __forceinline__ float dot(const float (&a)[DPL], const float (&b)[DPL]) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < DPL; ++k) s = fmaf(a[k], b[k], s);
    return warp_sum(s);
}
template <int DPL>
__device__ __forceinline__ void store_row(const float (&v)[DPL], int d, int lane, int64_t at, float* raw, float* hi, float* lo) {
#pragma unroll
    for (int k = 0; k < DPL; ++k) {
        const int c = lane + 32 * k;
        if (c >= d) continue;
        if (raw) raw[at + c] = v[k];
        if (hi) split_tf32(v[k], hi[at + c], lo[at + c]);
    }
}
// Modified score of raw score s (already scaled by 1/sqrt d); t receives 1 - tanh^2 (1 without a cap), from e^-2|u|: formed from
// the tanh it would cancel.
__device__ __forceinline__ float mod_score(float s, float cap, float slope, int distance, float& t) {
    t = 1.f;
    if (cap > 0.f) {
        const float u = s / cap, e = expf(-2.0f * fabsf(u));
        t = 4.0f * e / ((1.0f + e) * (1.0f + e));
        s = cap * tanhf(u);
    }
    return s - slope * fabsf((float)distance);
}

struct Pos { int i, h, b; int64_t gw; };
__device__ __forceinline__ bool position(const AttnModArgs& g, Pos& p) {
    p.gw = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (p.gw >= (int64_t)g.B * g.H * g.T) return false;
    p.i = (int)(p.gw % g.T);
    p.h = (int)((p.gw / g.T) % g.H);
    p.b = (int)(p.gw / ((int64_t)g.T * g.H));
    return true;
}

template <int DPL>
__global__ void __launch_bounds__(kWarps * 32) fwd_kernel(const AttnModArgs g) {
    pdl_wait();
    pdl_trigger();
    Pos p;
    if (!position(g, p)) return;
    const int lane = threadIdx.x & 31, d = g.C / g.H;
    const float scale = 1.0f / sqrtf((float)d), slope = g.slopes ? g.slopes[p.h] : 0.f;
    const int64_t ld = 3 * (int64_t)g.C, head = (int64_t)p.b * g.T * ld + (int64_t)p.h * d;
    const int2 span = mod::row_range(g.spans.k, p.b, g.T, p.i, false);
    float q[DPL], kv[DPL], acc[DPL], t;
    load_row<DPL>(g.qkv, g.qkv_lo, head + p.i * ld, d, lane, q);
    float mx = -INFINITY, l = 0.f;
    for (int j = span.x; j < span.y; ++j) {
        load_row<DPL>(g.qkv, g.qkv_lo, head + j * ld + g.C, d, lane, kv);
        mx = fmaxf(mx, mod_score(dot<DPL>(q, kv) * scale, g.cap, slope, p.i - j, t));
    }
#pragma unroll
    for (int k = 0; k < DPL; ++k) acc[k] = 0.f;
    for (int j = span.x; j < span.y; ++j) {
        load_row<DPL>(g.qkv, g.qkv_lo, head + j * ld + g.C, d, lane, kv);
        const float w = expf(mod_score(dot<DPL>(q, kv) * scale, g.cap, slope, p.i - j, t) - mx);
        l += w;
        load_row<DPL>(g.qkv, g.qkv_lo, head + j * ld + 2 * (int64_t)g.C, d, lane, kv);
#pragma unroll
        for (int k = 0; k < DPL; ++k) acc[k] = fmaf(w, kv[k], acc[k]);
    }
    const float inv = l > 0.f ? 1.0f / l : 0.f;      // a row that reads nothing is zero, its lse -inf
#pragma unroll
    for (int k = 0; k < DPL; ++k) acc[k] *= inv;
    store_row<DPL>(acc, d, lane, ((int64_t)p.b * g.T + p.i) * g.C + (int64_t)p.h * d, g.o, g.o_hi, g.o_lo);
    if (lane == 0 && g.lse) g.lse[p.gw] = span.x < span.y ? mx + logf(l) : -INFINITY;
}

template <int DPL>
__global__ void __launch_bounds__(kWarps * 32) dq_kernel(const AttnModArgs g) {
    pdl_wait();
    pdl_trigger();
    Pos p;
    if (!position(g, p)) return;
    const int lane = threadIdx.x & 31, d = g.C / g.H;
    const float scale = 1.0f / sqrtf((float)d), slope = g.slopes ? g.slopes[p.h] : 0.f;
    const int64_t ld = 3 * (int64_t)g.C, row = (int64_t)p.b * g.T, head = row * ld + (int64_t)p.h * d;
    const int2 span = mod::row_range(g.spans.k, p.b, g.T, p.i, false);
    float q[DPL], go[DPL], kk[DPL], vv[DPL], acc[DPL], t;
    load_row<DPL>(g.qkv, g.qkv_lo, head + p.i * ld, d, lane, q);
    load_row<DPL>(g.d_o, g.d_o_lo, (row + p.i) * g.C + (int64_t)p.h * d, d, lane, go);
    const float L = g.lse[p.gw], D = g.dvec[p.gw];
#pragma unroll
    for (int k = 0; k < DPL; ++k) acc[k] = 0.f;
    for (int j = span.x; j < span.y; ++j) {
        load_row<DPL>(g.qkv, g.qkv_lo, head + j * ld + g.C, d, lane, kk);
        load_row<DPL>(g.qkv, g.qkv_lo, head + j * ld + 2 * (int64_t)g.C, d, lane, vv);
        const float w = expf(mod_score(dot<DPL>(q, kk) * scale, g.cap, slope, p.i - j, t) - L);
        const float ds = w * (dot<DPL>(go, vv) - D) * t * scale;
#pragma unroll
        for (int k = 0; k < DPL; ++k) acc[k] = fmaf(ds, kk[k], acc[k]);
    }
    store_row<DPL>(acc, d, lane, head + p.i * ld, g.dqkv, g.dqkv_hi, g.dqkv_lo);
}

template <int DPL>
__global__ void __launch_bounds__(kWarps * 32) dkv_kernel(const AttnModArgs g) {
    pdl_wait();
    pdl_trigger();
    Pos p;
    if (!position(g, p)) return;
    const int lane = threadIdx.x & 31, d = g.C / g.H;
    const float scale = 1.0f / sqrtf((float)d), slope = g.slopes ? g.slopes[p.h] : 0.f;
    const int64_t ld = 3 * (int64_t)g.C, row = (int64_t)p.b * g.T, head = row * ld + (int64_t)p.h * d;
    const int64_t stat = ((int64_t)p.b * g.H + p.h) * g.T;
    const int2 span = mod::row_range(g.spans.q, p.b, g.T, p.i, true);
    float q[DPL], go[DPL], kk[DPL], vv[DPL], dk[DPL], dv[DPL], t;
    load_row<DPL>(g.qkv, g.qkv_lo, head + p.i * ld + g.C, d, lane, kk);
    load_row<DPL>(g.qkv, g.qkv_lo, head + p.i * ld + 2 * (int64_t)g.C, d, lane, vv);
#pragma unroll
    for (int k = 0; k < DPL; ++k) dk[k] = dv[k] = 0.f;
    for (int i = span.x; i < span.y; ++i) {
        load_row<DPL>(g.qkv, g.qkv_lo, head + i * ld, d, lane, q);
        load_row<DPL>(g.d_o, g.d_o_lo, (row + i) * g.C + (int64_t)p.h * d, d, lane, go);
        const float w = expf(mod_score(dot<DPL>(q, kk) * scale, g.cap, slope, i - p.i, t) - g.lse[stat + i]);
        const float ds = w * (dot<DPL>(go, vv) - g.dvec[stat + i]) * t * scale;
#pragma unroll
        for (int k = 0; k < DPL; ++k) {
            dv[k] = fmaf(w, go[k], dv[k]);
            dk[k] = fmaf(ds, q[k], dk[k]);
        }
    }
    store_row<DPL>(dk, d, lane, head + p.i * ld + g.C, g.dqkv, g.dqkv_hi, g.dqkv_lo);
    store_row<DPL>(dv, d, lane, head + p.i * ld + 2 * (int64_t)g.C, g.dqkv, g.dqkv_hi, g.dqkv_lo);
}

unsigned warps_grid(const AttnModArgs& g) {
    return (unsigned)(((int64_t)g.B * g.H * g.T + kWarps - 1) / kWarps);
}

}  // namespace

cudaError_t launch_attention_mod_fwd_simt(const AttnModArgs& g, cudaStream_t s) {
    const int d = g.C / g.H;
    const unsigned grid = warps_grid(g);
    if (d <= 32) BT_KERNEL_LAUNCH((fwd_kernel<1>), grid, kWarps * 32, 0, s, g);
    else if (d <= 64) BT_KERNEL_LAUNCH((fwd_kernel<2>), grid, kWarps * 32, 0, s, g);
    else BT_KERNEL_LAUNCH((fwd_kernel<4>), grid, kWarps * 32, 0, s, g);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

cudaError_t launch_attention_mod_bwd_simt(const AttnModArgs& g, cudaStream_t s) {
    const int d = g.C / g.H;
    const unsigned grid = warps_grid(g);
    if (d <= 32) {
        BT_KERNEL_LAUNCH((dq_kernel<1>), grid, kWarps * 32, 0, s, g);
        BT_KERNEL_LAUNCH((dkv_kernel<1>), grid, kWarps * 32, 0, s, g);
    } else if (d <= 64) {
        BT_KERNEL_LAUNCH((dq_kernel<2>), grid, kWarps * 32, 0, s, g);
        BT_KERNEL_LAUNCH((dkv_kernel<2>), grid, kWarps * 32, 0, s, g);
    } else {
        BT_KERNEL_LAUNCH((dq_kernel<4>), grid, kWarps * 32, 0, s, g);
        BT_KERNEL_LAUNCH((dkv_kernel<4>), grid, kWarps * 32, 0, s, g);
    }
    BT_COUNT_LAUNCH();
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

}  // namespace bt
