// The head's products with W for some dozens of rows of x: W goes through the SMs as it is, and becomes FP16 pairs on the way.
//
//     kStats  z = x W^T, (maximum, sum of exponentials) over a CTA's share of the vocabulary; kStatsTop the same with a teacher's entries
//     kGrad   the same z, u = 2^15 (q - [v = target]) as pairs (q to an absolute 2^-40, see head_tc.cu)
//     kDx     dx = u W, a range of the vocabulary each, joined by head_direct_dx_kernel
//
// With so few rows the weights' bytes bound the call, and a pass that makes pairs of W (read, written and read again) costs three times
// as much.  Here a tile of W is the A operand of tcgen05.mma.kind::f16, in tensor memory: 128 rows of W by 64 columns, lane = row, or
// for dx 128 columns by 64 rows, lane = column.  A thread takes the 64 values of its own lane out of shared memory, scales them by a
// power of two of their own, and stores the pairs.  The same lanes hold the products, so the scale comes out again where the thread of
// the lane adds the block to its sums in FP32.
//
//     warps 0, 2 (a lane) TMA: W tiles (FP32, raw or planes); the pairs of x or u
//     warp 1 (one lane)   MMA: += W x^T per 64 of the contraction index (l h' + h l' + h h')
//     warps 4-7, 8-11     pairs of even and odd blocks
//     warps 12-15         sums, then the mode's last step
//
// W 50,257 x 1,024: statistics of 9 rows take 56 us, of 100 68 (all launches, L2 cold; 3.7 and 3.0 TB/s of W), gradients 155 and 188.  Few rows are bound by the
// copies; with more, x comes to every SM as often as W and from L2, and a block's chain of copy, pairs, product and sum shows.
//
// W's ring has an even number of stages: a stage then always belongs to the same warps.  (Two groups that took turns on one
// stage could take the fill that the other still waits for to be theirs: a parity tells neighbouring phases apart, not more.)
// Every wait is bounded: one that runs out sets the error word and the CTA drains and exits, still releasing its tensor memory.
#include <cuda.h>

#include "head.cuh"
#include "tc_common.cuh"

namespace bt {

using namespace tc;

namespace {

constexpr int kTileRows = 128, kGroup = 32, kBlock = 64, kMostX = 128;
constexpr int kThreads = 512;
constexpr int kRegsIssue = 40, kRegsPairs = 120, kRegsSums = 224;      // of the launch's 4 x 128

// W by boxes of one to four groups (boxes of one group alone, up to sixteen to a stage, take half as long again).
struct WMaps {
    CUtensorMap of[4];
};

// What becomes of the products of x and W (kStats with targets, kStatsTop with a teacher's entries, kGrad), and the product of u and W.
enum Mode { kStats, kStatsTop, kGrad, kDx };

struct Args {
    int N, C, V, groups, blocks, Nr;        // groups of 32 rows of W; Nr: rows of x, up to a multiple of 16
    int x_stages, per;                      // groups of a CTA that has one pass over them
    const float* rowf;                      // [N]
    float2* stats;                          // kStats, kStatsTop: [N][4 CTAs]
    HeadScores scores;                      // kStats, kStatsTop
    const RowParams* rows;                  // kGrad
    int v0;                                 // kGrad: first column of this piece
    __half* u;                              // kGrad: [2][N][ldu]
    long long u_plane, ldu;
    int c_tiles, splits;                    // kDx: of 128 columns of W, and of the vocabulary
    float* parts;                           // kDx: [splits][N][C]
    float grow;
    int* err;
};

template <bool PLANES>
struct Cfg {
    static constexpr uint32_t kForms = PLANES ? 2u : 1u, kBox = kGroup * 32u * 4u;       // a stage: [2 halves of the block][forms][groups]
    static constexpr uint32_t kW = 8u * kForms * kBox;
    static constexpr int kStages = PLANES ? 2 : 4;                      // of W; those of x are as many as fit
    static constexpr uint32_t kScales = (2u * kTileRows + kMostX + 24u * kMostX) * 4u;     // scales, rowf; references, sums, spans and entries of four warps
    static constexpr uint32_t kFixed = 1024 + kStages * kW + kScales + 256;
};
constexpr uint32_t kSmemMost = 227u * 1024u;
constexpr int kMostXStages = 4;
__host__ __device__ constexpr uint32_t x_bytes(int Nr) { return 2u * Nr * kBlock * 2u; }

__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void tma_prefetch_3d(const CUtensorMap* tm, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];" ::"l"(tm), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld1(uint32_t taddr, uint32_t& r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(taddr));
}

__device__ __forceinline__ void copy4(uint32_t* dst, const uint32_t* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy8(int2* dst, const int2* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

// Maxima (MAX) or sums over the warp's lanes of 32 values per lane: lane l gets that of value l.
template <bool MAX>
__device__ __forceinline__ float across(float (&v)[32], int lane) {
#pragma unroll
    for (int half = 16; half >= 1; half /= 2) {
        const bool up = lane & half;
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const float keep = up ? v[i + half] : v[i], give = up ? v[i] : v[i + half], got = __shfl_xor_sync(0xffffffffu, give, half);
            v[i] = MAX ? fmaxf(keep, got) : keep + got;
        }
    }
    return v[0];
}

template <bool PLANES, int MODE>
__global__ void __launch_bounds__(kThreads, 1)
head_direct_kernel(const __grid_constant__ WMaps tmW, const __grid_constant__ CUtensorMap tmX, const Args g) {
    using C = Cfg<PLANES>;
    constexpr bool kSums = MODE == kStats || MODE == kStatsTop;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const base_ptr = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t x_size = x_bytes(g.Nr), x_ring = base + C::kStages * C::kW;
    float* const scales = reinterpret_cast<float*>(base_ptr + C::kStages * C::kW + g.x_stages * x_size);
    float* const row_f = scales + 2 * kTileRows;
    float* const refs = row_f + kMostX;
    const uint32_t bars = x_ring + g.x_stages * x_size + C::kScales;
    auto full_bar = [&](int s) { return bars + 8u * s; };
    auto empty_bar = [&](int s) { return bars + 8u * (C::kStages + s); };
    auto pairs_bar = [&](int a) { return bars + 8u * (2 * C::kStages + a); };
    auto done_bar = [&](int a) { return bars + 8u * (2 * C::kStages + 2 + a); };
    auto drained_bar = [&](int a) { return bars + 8u * (2 * C::kStages + 4 + a); };
    auto x_full_bar = [&](int s) { return bars + 8u * (2 * C::kStages + 6 + s); };
    auto x_empty_bar = [&](int s) { return bars + 8u * (2 * C::kStages + 6 + kMostXStages + s); };
    const uint32_t tmem_slot = bars + 8u * (2 * C::kStages + 6 + 2 * kMostXStages);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // The CTA's share of W: four groups in every complete round of all CTAs, and an even part of what is left, if there were any.
    // kDx: one tile of columns, and every splits-th block of rows, from the end of W, which the call before has left in L2.
    const int ctas = gridDim.x, full = g.per < 4 ? 0 : g.groups / (4 * ctas), rest = g.groups - 4 * ctas * full;
    const int r0 = full == 0 ? g.per * blockIdx.x : 4 * ctas * full + (int)((int64_t)blockIdx.x * rest / ctas);
    const int r1 = full == 0 ? min(g.groups, r0 + g.per) : 4 * ctas * full + (int)((blockIdx.x + 1LL) * rest / ctas);
    const int c_tile = MODE == kDx ? (int)blockIdx.x % g.c_tiles : 0, split = MODE == kDx ? (int)blockIdx.x / g.c_tiles : 0;
    const int passes = MODE == kDx ? 1 : full + (r1 > r0 ? 1 : 0), blocks = MODE == kDx ? (g.blocks - split + g.splits - 1) / g.splits : g.blocks;
    auto first_of = [&](int p) { return MODE == kDx ? 0 : p < full ? 4 * ((int)blockIdx.x + p * ctas) : r0; };
    auto groups_of = [&](int p) { return MODE == kDx ? min(4, (g.C - c_tile * kTileRows) / kGroup) : p < full ? 4 : r1 - r0; };
    auto block_of = [&](int b) { return MODE == kDx ? g.blocks - 1 - split - b * g.splits : b; };

    if (threadIdx.x == 0) {
        prefetch_tensormap(&tmW.of[MODE == kDx ? 0 : groups_of(0) - 1]);
        prefetch_tensormap(&tmX);
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 4);     // the warps that make pairs of it
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(pairs_bar(a), 4);
            mbar_init(done_bar(a), 1);
            mbar_init(drained_bar(a), 4);
        }
        for (int s = 0; s < g.x_stages; ++s) {
            mbar_init(x_full_bar(s), 1);
            mbar_init(x_empty_bar(s), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(tmem_slot) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(base_ptr + (tmem_slot - base));
    // the first of W on their way into L2 while the kernel before makes x's pairs (100 rows against 50,257 x 1,024: 73.6 us to 71.8, L2 cold)
    if (MODE != kDx && threadIdx.x == 0)
        for (int b = 0; b < min(g.blocks, 2 * C::kStages); ++b) {
            tma_prefetch_3d(&tmW.of[groups_of(0) - 1], b * kBlock, first_of(0) * kGroup, 0);
            if (b * kBlock + 32 < g.C) tma_prefetch_3d(&tmW.of[groups_of(0) - 1], b * kBlock + 32, first_of(0) * kGroup, 0);
        }
    pdl_wait();
    pdl_trigger();
    // tensor memory: products 0-127 and 128-255, pairs (32 columns of h, 32 of l) from 256 and 320, a tile's sums from 384
    auto t_sum = [&](int a) { return tmem + 128u * a; };
    auto t_pair = [&](int a) { return tmem + 256u + 64u * a; };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
        if ((warp == 0 || warp == 2) && lane == 0) {
            uint32_t it = 0, xs = 0, xp = 0;           // stage of x and how often it has come round
            bool ok = true;
            for (int p = 0; p < passes && ok; ++p)
                for (int i = 0; i < blocks; ++i, ++it) {
                    const int b = block_of(i);
                    if (warp == 0) {
                        const int s = it % C::kStages, n = groups_of(p), first = first_of(p);
                        if (!mbar_wait(empty_bar(s), ((it / C::kStages) & 1u) ^ 1u, g.err, 41)) { ok = false; break; }
                        mbar_expect_tx(full_bar(s), MODE == kDx ? C::kW : 2u * C::kForms * n * C::kBox);
                        const CUtensorMap* tm = MODE == kDx ? &tmW.of[0] : &tmW.of[n - 1];
                        if (MODE == kDx) {
                            tma_load_3d(base + s * C::kW, tm, full_bar(s), c_tile * kTileRows, b * kBlock, 0);
                        } else {
                            tma_load_3d(base + s * C::kW, tm, full_bar(s), b * kBlock, first * kGroup, 0);
                            tma_load_3d(base + s * C::kW + C::kW / 2, tm, full_bar(s), b * kBlock + 32, first * kGroup, 0);
                        }
                    } else {
                        if (!mbar_wait(x_empty_bar(xs), (xp & 1u) ^ 1u, g.err, 47)) { ok = false; break; }
                        mbar_expect_tx(x_full_bar(xs), x_size);
                        tma_load_3d(x_ring + xs * x_size, &tmX, x_full_bar(xs), b * kBlock, 0, 0);
                        if (++xs == (uint32_t)g.x_stages) xs = 0, ++xp;
                    }
                }
            if (!ok)                        // copies in flight land before the shared memory is given back
                for (int i = 0; i < 2000; ++i) __nanosleep(1000);
        }
        if (warp == 1) {
            // FP16 operands, A with rows of K in lanes, B K-major
            const uint32_t idesc = (1u << 4) | ((uint32_t)(g.Nr >> 3) << 17) | ((uint32_t)(kTileRows >> 4) << 24);
            uint32_t it = 0, xs = 0, xp = 0;
            bool ok = true;
            for (int p = 0; p < passes && ok; ++p)
                for (int b = 0; b < blocks; ++b, ++it) {
                    const int a = it & 1;
                    if (!mbar_wait_warp(x_full_bar(xs), xp & 1u, g.err, 48) || !mbar_wait_warp(pairs_bar(a), (it >> 1) & 1u, g.err, 42)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t x_base = x_ring + xs * x_size;
                    if (elect_one()) {
#pragma unroll
                        for (int j = 0; j < kBlock / 16; ++j) {
                            const uint64_t xh = make_desc(x_base + j * 32u, 16u, 1024u, 2u), xl = make_desc(x_base + g.Nr * 128u + j * 32u, 16u, 1024u, 2u);
                            mma_f16_ts(t_sum(a), t_pair(a) + 32u + 8u * j, xh, idesc, j > 0 ? 1u : 0u);
                            mma_f16_ts(t_sum(a), t_pair(a) + 8u * j, xl, idesc, 1u);
                            mma_f16_ts(t_sum(a), t_pair(a) + 8u * j, xh, idesc, 1u);
                        }
                        umma_commit(x_empty_bar(xs));
                        umma_commit(done_bar(a));
                    }
                    __syncwarp();
                    if (++xs == (uint32_t)g.x_stages) xs = 0, ++xp;
                }
        }
    } else if (warp < 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsPairs));
        const int a = (warp - 4) >> 2, quad = warp & 3, row = quad * kGroup + lane;
        const uint32_t t_row = t_pair(a) + ((uint32_t)(quad * 32) << 16);
        uint32_t it = 0;
        bool ok = true;
        for (int p = 0; p < passes && ok; ++p) {
            const int groups = groups_of(p);
            const bool mine = quad < groups;
            for (int b = 0; b < blocks; ++b, ++it) {
                if ((int)(it & 1u) != a) continue;
                const int s = it % C::kStages;
                if (!mbar_wait_warp(full_bar(s), (it / C::kStages) & 1u, g.err, 43)) { ok = false; break; }
                if (!mine) {                // behind the share: these lanes' products are not looked at
                    if (!mbar_wait_warp(drained_bar(a), ((it >> 1) & 1u) ^ 1u, g.err, 44)) { ok = false; break; }
                    if (lane == 0) {
                        mbar_arrive(empty_bar(s));
                        mbar_arrive(pairs_bar(a));
                    }
                    continue;
                }
                float v[kBlock];
                if (MODE == kDx) {          // a column of [64][128]
#pragma unroll
                    for (int i = 0; i < kBlock; ++i) {
                        const float* p = reinterpret_cast<const float*>(base_ptr + s * C::kW) + i * kTileRows + row;
                        v[i] = PLANES ? p[0] + p[kBlock * kTileRows] : p[0];
                    }
                }
                // the 16-byte units of a row of 128 bytes lie swizzled by the row
#pragma unroll
                for (int h = 0; MODE != kDx && h < 2; ++h)
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const uint8_t* p = base_ptr + s * C::kW + (4 * C::kForms * h + quad) * C::kBox + lane * 128 + ((q ^ (lane & 7)) << 4);
                        float4 w = *reinterpret_cast<const float4*>(p);
                        if (PLANES) w = add4(w, *reinterpret_cast<const float4*>(p + groups * C::kBox));
                        v[h * 32 + 4 * q] = w.x; v[h * 32 + 4 * q + 1] = w.y; v[h * 32 + 4 * q + 2] = w.z; v[h * 32 + 4 * q + 3] = w.w;
                    }
                __syncwarp();
                if (lane == 0) mbar_arrive(empty_bar(s));
                float top[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < kBlock; ++i) top[i & 3] = fmaxf(top[i & 3], fabsf(v[i]));
                const float m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                const int k = pair_exponent(m);
                const float sc = pow2(k);
                uint32_t hi[32], lo[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) to_pairs(v[2 * i] * sc, v[2 * i + 1] * sc, hi[i], lo[i]);
                // the sums of the block before last have been taken, and with them its scales and pairs
                if (!mbar_wait_warp(drained_bar(a), ((it >> 1) & 1u) ^ 1u, g.err, 44)) { ok = false; break; }
                tc_fence_after();
                tmem_st32(t_row, hi);
                tmem_st32(t_row + 32u, lo);
                scales[a * kTileRows + row] = ldexpf(1.0f, -k - 15);      // the sums stay near W's size whatever x's
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pairs_bar(a));
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSums));
        const int quad = warp & 3, row = quad * 32 + lane;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        float *const ref = refs + quad * kMostX, *const sum = refs + (4 + quad) * kMostX;     // over the tiles, in units of the reference
        float* const row_l = refs;          // kGrad
        int* const hit = reinterpret_cast<int*>(refs + kMostX);
        uint32_t it = 0;
        bool ok = true;
        for (int n = lane; n < kMostX; n += 32) {
            if (MODE != kDx && quad == 0) row_f[n] = n < g.N ? g.rowf[n] * g.grow : 0.f;
            if (kSums) {
                ref[n] = -INFINITY;
                sum[n] = 0.f;
            }
            if (MODE == kGrad && quad == 0) {
                const RowParams r = n < g.N ? g.rows[n] : RowParams{INFINITY, 0.f, 0.f, -1};
                row_l[n] = (r.L - 15.0f) + r.L_rest;           // see kGrad in head_tc.cu
                hit[n] = r.target < 0 ? -1 : r.target - g.v0;
            }
        }
        int target[4] = {-1, -1, -1, -1};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (MODE == kStats && q * 32 + lane < g.N) target[q] = g.scores.targets[q * 32 + lane];
            if (target[q] >= g.V) target[q] = 0;
        }
        // kStatsTop: a row's entries among the warp's rows of W, of this pass and the next, and the first of them; each lane copies
        // what it reads
        uint32_t* const span = reinterpret_cast<uint32_t*>(refs + 8 * kMostX) + quad * 2 * kMostX;
        int2* const entry = reinterpret_cast<int2*>(refs + 16 * kMostX) + quad * kMostX;
        auto fetch_spans = [&](int p) {
            for (int n = lane; n < g.N; n += 32) {
                if (quad < groups_of(p)) copy4(span + (p & 1) * kMostX + n, g.scores.spans + (long long)n * g.groups + first_of(p) + quad);
                else span[(p & 1) * kMostX + n] = 0u;
            }
        };
        if (MODE == kStatsTop) fetch_spans(0);
        asm volatile("bar.sync 1, 128;" ::: "memory");         // these four warps
        for (int p = 0; p < passes && ok; ++p) {
            const int first = first_of(p);
            const bool mine = quad < groups_of(p);
            if (MODE == kStatsTop) {        // the pass's spans are here; its first entries and the next pass's spans on their way
                asm volatile("cp.async.wait_all;" ::: "memory");
                for (int n = lane; n < g.N; n += 32) {
                    const uint32_t m = span[(p & 1) * kMostX + n];
                    if ((m & 0xffffu) < m >> 16) copy8(entry + n, g.scores.entries + (long long)n * g.scores.K + (m & 0xffffu));
                }
                if (p + 1 < passes) fetch_spans(p + 1);
            }
            float z[4][32];
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int j = 0; j < 32; ++j) z[q][j] = 0.f;
            for (int b = 0; b < blocks; ++b, ++it) {
                const int a = it & 1;
                // the products are there, and the block's scales before them
                if (!mbar_wait_warp(done_bar(a), (it >> 1) & 1u, g.err, 45) || !mbar_wait_warp(pairs_bar(a), (it >> 1) & 1u, g.err, 46)) { ok = false; break; }
                tc_fence_after();
                const float sc = scales[a * kTileRows + row];
#pragma unroll
                for (int q = 0; q < 4; q += 2) {        // two loads under way at a time
                    if (q * 32 >= g.Nr || !mine) continue;
                    uint32_t r0[32], r1[32];
                    tmem_ld32(t_sum(a) + lanes + q * 32u, r0);
                    const bool more = q * 32 + 32 < g.Nr;
                    if (more) tmem_ld32(t_sum(a) + lanes + q * 32u + 32u, r1);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 32; ++j) z[q][j] = fmaf(__uint_as_float(r0[j]), sc, z[q][j]);
                    if (more) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) z[q + 1][j] = fmaf(__uint_as_float(r1[j]), sc, z[q + 1][j]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(drained_bar(a));
            }
            if (!ok) break;
            if (!mine) continue;
            const int v_at = (first + quad) * kGroup + lane;
            const bool there = v_at < g.V;
            // through tensor memory, which takes an index: what follows is one small piece of code for a few columns at a time (all of
            // them in line are fetched anew for every tile: 79 us against 70 for statistics of 100 rows, V 50,257, C 1,024)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t r[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(z[q][j]);
                if (q * 32 < g.N) tmem_st32(tmem + 384u + lanes + q * 32u, r);
            }
            tmem_st_wait();
            if (MODE == kDx) {
                float* dst = g.parts + (long long)split * g.N * g.C + c_tile * kTileRows + row;
#pragma unroll 1
                for (int n0 = 0; n0 < g.N; n0 += 8, dst += 8 * g.C) {
                    uint32_t zr[8];
                    tmem_ld8(tmem + 384u + lanes + n0, zr);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (n0 + j < g.N) dst[j * g.C] = __uint_as_float(zr[j]) * g.grow;
                }
            }
            if (MODE == kGrad) {
                __half* dst = g.u + (lane & 3) * g.ldu + (v_at & ~3);
#pragma unroll 1
                for (int n0 = 0; n0 < g.N; n0 += 8, dst += 8 * g.ldu) {
                    uint32_t zr[8];
                    tmem_ld8(tmem + 384u + lanes + n0, zr);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 8; j += 4) {
                        const float4 f = *reinterpret_cast<const float4*>(row_f + n0 + j), l = *reinterpret_cast<const float4*>(row_l + n0 + j);
                        const int4 t = *reinterpret_cast<const int4*>(hit + n0 + j);
                        const float fs[4] = {f.x, f.y, f.z, f.w}, ls[4] = {l.x, l.y, l.z, l.w};
                        const int ts[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float e = ex2_fast(fmaf(__uint_as_float(zr[j + i]) * fs[i], 32768.0f, -ls[i]));
                            if (ls[i] == INFINITY) e = 0.f;    // whatever the row holds
                            if (ts[i] == v_at) e -= 32768.0f;
                            const __half h = __float2half_rn(e), r = __float2half_rn(e - __half2float(h));
                            zr[j + i] = (uint32_t)__half_as_ushort(h) | (uint32_t)__half_as_ushort(r) << 16;
                        }
                    }
                    // four lanes trade their values of four rows for four columns of a row each: 8 bytes to a store, columns behind
                    // the piece into the padding of u
#pragma unroll
                    for (int j = 0; j < 8; j += 4) {
                        uint32_t a[4];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t keep = lane & 2 ? zr[j + 2 + i] : zr[j + i], got = __shfl_xor_sync(0xffffffffu, lane & 2 ? zr[j + i] : zr[j + 2 + i], 2);
                            a[i] = lane & 2 ? got : keep;              // columns 0, 1 (after the next step) ...
                            a[2 + i] = lane & 2 ? keep : got;          // ... and 2, 3 of the lane's two rows
                        }
                        const uint32_t k0 = lane & 1 ? a[1] : a[0], k1 = lane & 1 ? a[3] : a[2];
                        const uint32_t g0 = __shfl_xor_sync(0xffffffffu, lane & 1 ? a[0] : a[1], 1), g1 = __shfl_xor_sync(0xffffffffu, lane & 1 ? a[2] : a[3], 1);
                        const uint32_t c0 = lane & 1 ? g0 : k0, c1 = lane & 1 ? k0 : g0, c2 = lane & 1 ? g1 : k1, c3 = lane & 1 ? k1 : g1;
                        if (n0 + j + (lane & 3) < g.N) {
                            *reinterpret_cast<uint2*>(dst + j * g.ldu) = make_uint2(__byte_perm(c0, c1, 0x5410), __byte_perm(c2, c3, 0x5410));
                            *reinterpret_cast<uint2*>(dst + j * g.ldu + g.u_plane) = make_uint2(__byte_perm(c0, c1, 0x7632), __byte_perm(c2, c3, 0x7632));
                        }
                    }
                }
            }
#pragma unroll 1
            for (int q = 0; kSums && q * 32 < g.N; ++q) {
                uint32_t zr[32];
                tmem_ld32(tmem + 384u + lanes + q * 32u, zr);
                tmem_ld_wait();
                const int n = q * 32 + lane;
                float v[32], most = -INFINITY;
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    const float4 f = *reinterpret_cast<const float4*>(row_f + q * 32 + j), r = *reinterpret_cast<const float4*>(ref + q * 32 + j);
                    const float fs[4] = {f.x, f.y, f.z, f.w}, rs[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float zs = __uint_as_float(zr[j + i]) * fs[i] * 32768.0f;
                        zr[j + i] = __float_as_uint(zs);
                        v[j + i] = zs - rs[i];
                        most = fmaxf(most, v[j + i]);
                    }
                }
                // a row's reference is its maximum over the warp's part of an earlier tile, as long as that is near enough: values
                // of 2^20 and more take a new one, those that vanish beside it add nothing that counts
                if (__any_sync(0xffffffffu, there && !(most <= 20.f))) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = there ? __uint_as_float(zr[j]) : -INFINITY;
                    const float m = fmaxf(across<true>(v, lane), ref[n]);
                    __syncwarp();
                    if (m != ref[n]) {
                        sum[n] = sum[n] != 0.f ? sum[n] * ex2_fast(ref[n] - m) : 0.f;
                        ref[n] = m;
                    }
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(zr[j]) - ref[q * 32 + j];
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = there ? ex2_fast(v[j]) : 0.f;
                sum[n] += across<false>(v, lane);
            }
            // the scores that the losses need, as the sums have them: few of a warp's groups of W have any
            auto score = [&](int n, int at, long long to) {
                uint32_t r;
                tmem_ld1(tmem + 384u + lanes + n, r);
                tmem_ld_wait();
                if (lane == at) g.scores.zk[to] = __uint_as_float(r) * row_f[n] * 32768.0f;
            };
            if (MODE == kStats) {
                const int v_first = (first + quad) * kGroup;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    for (unsigned left = __ballot_sync(0xffffffffu, target[q] >= v_first && target[q] < v_first + kGroup); left; left &= left - 1) {
                        const int j = __ffs(left) - 1;
                        score(q * 32 + j, __shfl_sync(0xffffffffu, target[q], j) - v_first, q * 32 + j);
                    }
            }
            if (MODE == kStatsTop) {
                asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll 1
                for (int q = 0; q * 32 < g.N; ++q) {        // a lane's row of x has its entries in turn, the next on its way meanwhile
                    const int n = q * 32 + lane;
                    const uint32_t m = n < g.N ? span[(p & 1) * kMostX + n] : 0u;
                    int e = m & 0xffffu;
                    const int e_end = m >> 16;
                    int2 now = e < e_end ? entry[n] : make_int2(0, 0);
                    for (unsigned left; (left = __ballot_sync(0xffffffffu, e < e_end)) != 0; ++e) {
                        const int2 next = e + 1 < e_end ? g.scores.entries[(long long)n * g.scores.K + e + 1] : make_int2(0, 0);
                        for (; left; left &= left - 1) {
                            const int j = __ffs(left) - 1, col = __shfl_sync(0xffffffffu, now.x, j), place = __shfl_sync(0xffffffffu, now.y, j);
                            score(q * 32 + j, col & (kGroup - 1), (long long)(q * 32 + j) * g.scores.K + place);
                        }
                        now = next;
                    }
                }
            }
        }
        if (MODE == kStatsTop) asm volatile("cp.async.wait_all;" ::: "memory");       // where a wait ran out
        // a warp without rows of W has the sum zero
        for (int n = lane; kSums && n < g.N; n += 32) g.stats[(long long)n * (4 * gridDim.x) + 4 * blockIdx.x + quad] = make_float2(ref[n], sum[n]);
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// kGrad and kDx: `rows` of W from row v0 on.
template <bool PLANES, int MODE>
cudaError_t launch(const HeadArgs& h, int v0, int rows, const HalfMat& x, int grid, const Args& g, cudaStream_t s) {
    using C = Cfg<PLANES>;
    if (!tensor_map_encoder()) return cudaErrorNotSupported;
    WMaps tmW;
    CUtensorMap tmX;
    const cuuint32_t one[3] = {1, 1, 1};
    const cuuint64_t w_dims[3] = {(cuuint64_t)h.C, (cuuint64_t)rows, PLANES ? 2u : 1u}, w_strides[2] = {(cuuint64_t)h.C * 4, (cuuint64_t)h.V * h.C * 4};
    const cuuint32_t x_box[3] = {kBlock, (cuuint32_t)g.Nr, 2};
    const cuuint64_t x_dims[3] = {(cuuint64_t)x.cols, (cuuint64_t)x.rows, 2}, x_strides[2] = {(cuuint64_t)x.ld * 2, (cuuint64_t)x.plane * 2};
    bool ok = tensor_map_encoder()(&tmX, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, (void*)x.hi, x_dims, x_strides, x_box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    for (int n = 1; ok && n <= (MODE == kDx ? 1 : 4); ++n) {
        const cuuint32_t w_box[3] = {MODE == kDx ? (cuuint32_t)kTileRows : 32u, MODE == kDx ? (cuuint32_t)kBlock : (cuuint32_t)(n * kGroup), C::kForms};
        ok = tensor_map_encoder()(&tmW.of[n - 1], CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, (void*)(h.w + (int64_t)v0 * h.C), w_dims, w_strides, w_box, one,
                                  CU_TENSOR_MAP_INTERLEAVE_NONE, MODE == kDx ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B,
                                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    }
    if (!ok) return cudaErrorInvalidValue;
    const uint32_t fit = (kSmemMost - C::kFixed) / x_bytes(g.Nr);
    Args a = g;
    a.x_stages = fit < (uint32_t)kMostXStages ? (int)fit : kMostXStages;       // two and more: 128 rows take 32 KB
    const cudaError_t e = allow_smem<head_direct_kernel<PLANES, MODE>>(kSmemMost);
    if (e != cudaSuccess) return e;
    BT_KERNEL_LAUNCH((head_direct_kernel<PLANES, MODE>), grid, kThreads, (size_t)(C::kFixed + a.x_stages * x_bytes(g.Nr)), s,
                     tmW, tmX, a);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

// dx of the rows from the splits' sums, 32 columns of four per CTA, an eighth of the splits to a warp.  The sums over earlier pieces
// of the vocabulary lie where the result will be.
__global__ void __launch_bounds__(256) head_direct_dx_kernel(const HeadArgs g, const RowParams* __restrict__ rows, int splits, const float* __restrict__ parts,
                                                             bool onto, bool last) {
    __shared__ float4 sm[8][32];
    pdl_wait();
    pdl_trigger();
    const int C4 = g.C / 4, lane = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t i = blockIdx.x * 32LL + lane, n4 = g.N * C4;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < n4) {
#pragma unroll 8
        for (int k = y; k < splits; k += 8) t = add4(t, ld4(parts, k * n4 + i));
    }
    sm[y][lane] = t;
    __syncthreads();
    if (y > 0 || i >= n4) return;
    for (int k = 1; k < 8; ++k) t = add4(t, sm[k][lane]);
    const float rg = rows[i / C4].g;
    t = rg == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(t.x * rg, t.y * rg, t.z * rg, t.w * rg);      // zero: the row has no part in the loss
    float* const sums = g.dx ? g.dx : g.dx_hi;
    if (onto) t = add4(t, ld4(sums, i));
    if (last) store_raw_split(t, g.dx, g.dx_hi, g.dx_lo, i);
    else reinterpret_cast<float4*>(sums)[i] = t;
}

// Four groups to a CTA, or fewer where that leaves SMs idle and a CTA keeps 64 KB of W: x has to come to every CTA, and the next
// kernel starts earlier where SMs are free.  9 rows against planes of 3,000 x 2,048 35 us, four groups each 40; against 5,000 x 256
// 14.5, on 148 SMs 17.0.
struct Share {
    int per, ctas;
};
Share share_of(int C, int rows) {
    const int groups = (rows + kGroup - 1) / kGroup, sms = sm_count();
    Share s{4, 0};
    while (s.per > 1 && (groups + s.per / 2 - 1) / (s.per / 2) <= sms && s.per / 2 * kGroup * C * 4 >= 64 * 1024) s.per /= 2;
    s.ctas = (groups + s.per - 1) / s.per < sms ? (groups + s.per - 1) / s.per : sms;
    return s;
}

Args args_for(const HeadArgs& h, int rows, int* err) {
    Args g{};
    g.per = share_of(h.C, rows).per;
    g.N = (int)h.N; g.C = h.C; g.V = rows;
    g.groups = (rows + kGroup - 1) / kGroup;
    g.blocks = (h.C + kBlock - 1) / kBlock;
    g.Nr = ((int)h.N + 15) / 16 * 16;
    g.err = err;
    g.grow = head_growth(3 * kBlock / 16);
    return g;
}

}  // namespace

bool head_direct_fits(int64_t N) { return N <= kMostX; }
int head_direct_strips(int C, int V) { return 4 * share_of(C, V).ctas; }

cudaError_t launch_head_direct(const HeadArgs& h, const HalfMat& x, const float* rowf, const HeadScores& scores, float2* stats, int* err, cudaStream_t s) {
    Args g = args_for(h, h.V, err);
    g.rowf = rowf; g.stats = stats; g.scores = scores;
    const int grid = share_of(h.C, h.V).ctas;
    if (scores.targets) return h.w_lo ? launch<true, kStats>(h, 0, h.V, x, grid, g, s) : launch<false, kStats>(h, 0, h.V, x, grid, g, s);
    return h.w_lo ? launch<true, kStatsTop>(h, 0, h.V, x, grid, g, s) : launch<false, kStatsTop>(h, 0, h.V, x, grid, g, s);
}

cudaError_t launch_head_direct_grad(const HeadArgs& h, const HalfMat& x, int v0, int cols, const float* rowf, const RowParams* rows, __half* u, int64_t ldu,
                                    int64_t u_plane, int* err, cudaStream_t s) {
    Args g = args_for(h, cols, err);
    g.rowf = rowf; g.rows = rows; g.v0 = v0; g.u = u; g.ldu = ldu; g.u_plane = u_plane;
    const int grid = share_of(h.C, cols).ctas;
    return h.w_lo ? launch<true, kGrad>(h, v0, cols, x, grid, g, s) : launch<false, kGrad>(h, v0, cols, x, grid, g, s);
}

cudaError_t launch_head_direct_dx(const HeadArgs& h, const HalfMat& u, int v0, const RowParams* rows, bool onto, bool last, float* partials, int* err,
                                  cudaStream_t s) {
    const int cols = (int)u.cols, sms = sm_count() < 148 ? sm_count() : 148;       // head_partial_bytes() counts on 148
    Args g = args_for(h, cols, err);
    g.blocks = (cols + kBlock - 1) / kBlock;
    g.c_tiles = (h.C + kTileRows - 1) / kTileRows;
    g.splits = sms / g.c_tiles < g.blocks ? sms / g.c_tiles : g.blocks;
    g.parts = partials;
    const int grid = g.c_tiles * g.splits;
    const cudaError_t e = h.w_lo ? launch<true, kDx>(h, v0, cols, u, grid, g, s) : launch<false, kDx>(h, v0, cols, u, grid, g, s);
    if (e != cudaSuccess) return e;
    BT_KERNEL_LAUNCH((head_direct_dx_kernel), (unsigned)((h.N * h.C / 4 + 31) / 32), 256, 0, s, h, rows, g.splits, (const float*)partials, onto, last);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

}  // namespace bt
