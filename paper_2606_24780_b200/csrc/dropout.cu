// Dropout whose mask is never stored: element i is kept where word i mod 4 of the counter-based
// generator's block i / 4 is at least p 2^32, in the forward and again in the backward.
//     y_i = keep_i x_i / (1 - p) (+ residual_i),        dx_i = keep_i dy_i / (1 - p)
// The generator is Philox-4x32 with ten rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", 2011): counter (block low, block high, offset low, offset high), key
// (seed low, seed high).  Two calls with different offsets share no counter.
//
// Bound by HBM: 8 bytes per element (12 with a residual).  A block costs 20 wide multiplications and 40
// exclusive ors for four elements, a third of what the memory time leaves an SM for.
#include "common.cuh"

namespace bt {

namespace {

constexpr int kThreads = 256;
constexpr int kItems = 4;   // float4 per thread: all loads in flight before the first is used

__device__ __forceinline__ uint4 philox4x32(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
        const uint32_t n0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0, n2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)p1;
        c3 = (uint32_t)p0;
        c0 = n0;
        c2 = n2;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

__global__ void __launch_bounds__(kThreads) dropout_kernel(const DropoutArgs g) {
    pdl_wait();
    pdl_trigger();
    const uint64_t offset = g.offset + (g.d_step ? *g.d_step : 0ull);
    const int64_t n4 = g.n >> 2, first = (int64_t)blockIdx.x * (kThreads * kItems) + threadIdx.x;
    auto words = [&](int64_t blk) {
        return philox4x32((uint32_t)blk, (uint32_t)((uint64_t)blk >> 32), (uint32_t)offset, (uint32_t)(offset >> 32),
                          (uint32_t)g.seed, (uint32_t)(g.seed >> 32));
    };
    auto one = [&](float x, uint32_t w, float res) { return (w >= g.threshold ? x * g.scale : 0.f) + res; };
    float4 x[kItems], res[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int64_t i = first + (int64_t)k * kThreads;
        x[k] = res[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < n4) {
            x[k] = ld4(g.x, i);
            if (g.residual) res[k] = ld4(g.residual, i);
        }
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int64_t i = first + (int64_t)k * kThreads;
        if (i < n4) {
            const uint4 w = words(i);
            store_raw_split(make_float4(one(x[k].x, w.x, res[k].x), one(x[k].y, w.y, res[k].y),
                                        one(x[k].z, w.z, res[k].z), one(x[k].w, w.w, res[k].w)),
                            g.y, g.y_hi, g.y_lo, i);
        }
    }
    // the last one to three elements (raw output only: planes need n % 4 == 0)
    if (blockIdx.x == 0 && threadIdx.x == 0 && (g.n & 3)) {
        const uint4 w = words(n4);
        const uint32_t ws[3] = {w.x, w.y, w.z};
        for (int e = 0; e < (int)(g.n & 3); ++e) {
            const int64_t i = 4 * n4 + e;
            g.y[i] = one(g.x[i], ws[e], g.residual ? g.residual[i] : 0.f);
        }
    }
}

}  // namespace

cudaError_t launch_dropout(const DropoutArgs& g, cudaStream_t s) {
    const int64_t per = 4 * (int64_t)kThreads * kItems;
    const int64_t grid = (g.n + per - 1) / per;
    if (grid > 0x7fffffff) return cudaErrorInvalidValue;
    BT_KERNEL_LAUNCH((dropout_kernel), (unsigned)grid, kThreads, 0, s, g);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

}  // namespace bt
