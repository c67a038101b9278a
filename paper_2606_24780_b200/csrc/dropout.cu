// Dropout whose mask is never stored: element i is kept where word i mod 4 of the counter-based
// generator's block i / 4 is at least p 2^32, in the forward and again in the backward.
//     y_i = keep_i x_i / (1 - p) (+ residual_i),        dx_i = keep_i dy_i / (1 - p)
// The generator is Philox-4x32 with ten rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", 2011): counter (block low, block high, offset low, offset high), key
// (seed low, seed high).  Two calls with different offsets share no counter.
//
// Bound by HBM: 8 bytes per element (12 with a residual).  A block costs 20 wide multiplications and 20 three-way
// exclusive ors for four elements, which the memory time covers as long as little comes on top: with the round keys as kernel
// arguments, a 32-bit threshold and no bounds inside whole CTAs 33.6 M elements take 44 us (6.05 TB/s of a copy's 6.45), 51 us
// without; 6.3 M and a residual 13.4 us, 5.6 TB/s.
#include "common.cuh"

namespace bt {

namespace {

constexpr int kThreads = 256;
constexpr int kItems = 4;   // float4 per thread: all loads in flight before the first is used

// `key`: the keys of the ten rounds, two words each (kernel arguments: an operand of the exclusive ors, not an addition).
__device__ __forceinline__ uint4 philox4x32(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, const uint32_t (&key)[20]) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
        const uint32_t n0 = (uint32_t)(p1 >> 32) ^ c1 ^ key[2 * r], n2 = (uint32_t)(p0 >> 32) ^ c3 ^ key[2 * r + 1];
        c1 = (uint32_t)p1;
        c3 = (uint32_t)p0;
        c0 = n0;
        c2 = n2;
    }
    return make_uint4(c0, c1, c2, c3);
}

// RES: with a residual; RAW: the raw array is the only output.
template <bool RES, bool RAW>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const DropoutArgs g) {
    pdl_wait();
    pdl_trigger();
    const uint64_t offset = g.offset + (g.d_step ? *g.d_step : 0ull);
    const int64_t n4 = g.n >> 2, first = (int64_t)blockIdx.x * (kThreads * kItems) + threadIdx.x;
    const bool whole = (int64_t)(blockIdx.x + 1) * (kThreads * kItems) <= n4;      // no bounds inside this CTA
    const uint32_t threshold = (uint32_t)g.threshold;
    const bool any = (g.threshold >> 32) == 0;                                    // p rounds to one: nothing is kept
    auto words = [&](int64_t blk) {
        return philox4x32((uint32_t)blk, (uint32_t)((uint64_t)blk >> 32), (uint32_t)offset, (uint32_t)(offset >> 32), g.key);
    };
    auto one = [&](float x, uint32_t w, float res) {
        const float y = any && w >= threshold ? x * g.scale : 0.f;
        return RES ? y + res : y;
    };
    float4 x[kItems], res[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int64_t i = first + (int64_t)k * kThreads;
        if (whole || i < n4) {
            x[k] = ld4(g.x, i);
            if (RES) res[k] = ld4(g.residual, i);
        }
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int64_t i = first + (int64_t)k * kThreads;
        if (whole || i < n4) {
            const uint4 w = words(i);
            const float4 y = make_float4(one(x[k].x, w.x, res[k].x), one(x[k].y, w.y, res[k].y), one(x[k].z, w.z, res[k].z),
                                         one(x[k].w, w.w, res[k].w));
            if (RAW)
                reinterpret_cast<float4*>(g.y)[i] = y;
            else
                store_raw_split(y, g.y, g.y_hi, g.y_lo, i);
        }
    }
    // the last one to three elements (raw output only: planes need n % 4 == 0)
    if (RAW && blockIdx.x == 0 && threadIdx.x == 0 && (g.n & 3)) {
        const uint4 w = words(n4);
        const uint32_t ws[3] = {w.x, w.y, w.z};
        for (int e = 0; e < (int)(g.n & 3); ++e) {
            const int64_t i = 4 * n4 + e;
            g.y[i] = one(g.x[i], ws[e], RES ? g.residual[i] : 0.f);
        }
    }
}

}  // namespace

cudaError_t launch_dropout(const DropoutArgs& args, cudaStream_t s) {
    DropoutArgs g = args;
    for (int r = 0; r < 10; ++r) {
        g.key[2 * r] = (uint32_t)g.seed + (uint32_t)r * 0x9E3779B9u;
        g.key[2 * r + 1] = (uint32_t)(g.seed >> 32) + (uint32_t)r * 0xBB67AE85u;
    }
    const int64_t per = 4 * (int64_t)kThreads * kItems;
    const int64_t grid = (g.n + per - 1) / per;
    if (grid > 0x7fffffff) return cudaErrorInvalidValue;
    if (g.y_hi) {
        if (g.residual)
            BT_KERNEL_LAUNCH((dropout_kernel<true, false>), (unsigned)grid, kThreads, 0, s, g);
        else
            BT_KERNEL_LAUNCH((dropout_kernel<false, false>), (unsigned)grid, kThreads, 0, s, g);
    } else {
        if (g.residual)
            BT_KERNEL_LAUNCH((dropout_kernel<true, true>), (unsigned)grid, kThreads, 0, s, g);
        else
            BT_KERNEL_LAUNCH((dropout_kernel<false, true>), (unsigned)grid, kThreads, 0, s, g);
    }
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

}  // namespace bt
