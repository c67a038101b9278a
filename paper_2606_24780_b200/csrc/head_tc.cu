// Matrix products of the language-model head on the tensor cores, on pairs of FP16 numbers.
//
// An FP32 value v is held as s v = h + l with FP16 h = rn(s v), l = rn(s v - h) and a power of two s that brings the largest
// value of its row (or array) to [2^14, 2^15): 22 bits of every value down to 2^-18 of the largest, an absolute 2^-40 of
// the largest below.  A product is l h' + h l' + h h' in FP32.  tcgen05.mma.kind::f16 runs at twice the rate of kind::tf32
// and a pair takes 4 bytes where two TF32 planes take 8, so that both the tensor pipe and the copies take half the time
// of the library's three-product TF32 GEMM, at the same 22 bits.
//
// Three products share one kernel; NT z = x W^T, NN dx = u W, TN dW = u^T y, with three epilogues:
//     kStats  (maximum, sum of exponentials) of a strip, half a tile's columns, of a row
//     kGrad   u = 2^15 (q - [v = target]) as pairs, the operand of the two others.  One power of two for all of u: dx sums over its
//             columns and dW over its rows, and 2^15 brings its largest, 1, to the top of FP16.  q is then held to an absolute
//             2^-40; a power of two per column, which dW could take, needs the whole column before its first pair
//     kOut    FP32, scaled by a power of two and by the row's own factor, over or onto what is there
//
// Warp 0 copies tiles (TMA), warp 1 issues MMAs, warps 4 to 11 take accumulators out of tensor memory.  Tiles are 256 rows on a
// pair of CTAs (cta_group::2; each CTA brings its own rows of A and half of B's) or 128 on one where there are no more.
// The tensor core truncates when it adds, so sums are taken over in registers after 384 of the contraction index (72
// instructions): a warp holds 32 rows of 128 columns there, which also frees the accumulator before the epilogue's arithmetic.
// Every such step takes some 500 clocks from the MMAs, which read and write tensor memory at its full rate: at 768 columns sums
// after 128, 256, 384 and 512 take 1,230, 1,105, 1,105 and 1,100 us for z of 8,192 x 50,304, and 388, 330, 290 and 288 for a
// quarter of u, whose epilogue has to end within two steps; the error grows with the step.
#include <cuda.h>
#include <cuda_fp16.h>

#include "head.cuh"
#include "tc_common.cuh"

namespace bt {

using namespace tc;

namespace {

enum Epi { kStats, kGrad, kOut };

constexpr int BM = 128;                     // rows of a CTA
constexpr int BK = 32;                      // contraction per stage: 64-byte rows of K-major tiles
constexpr int kChunk = 384 / BK;            // stages between two sums in registers
constexpr int kEpiWarps = 8;
constexpr int kParts = kEpiWarps / 4;       // of a tile's columns, one to a warp
// Three warpgroups: TMA, MMA and two idle warps, then the epilogue's.  They share the launch's registers (168 each) as
// 56 + 2 x 224.
constexpr int kThreads = 128 + 32 * kEpiWarps;
constexpr int kRegsFew = 56, kRegsMany = 224;
constexpr uint32_t kSmemBudget = 227u * 1024u;

template <bool PAIR, int BN>
struct Cfg {
    static constexpr int kBRows = PAIR ? BN / 2 : BN;                   // of B in one CTA
    static constexpr uint32_t kABytes = 2u * BM * BK * 2u, kBBytes = 2u * kBRows * BK * 2u, kStage = kABytes + kBBytes;
    static constexpr uint32_t kFixed = 1024u + 256u;
    static constexpr int kFit = (int)((kSmemBudget - kFixed) / kStage);
    static constexpr int kStages = kFit > 8 ? 8 : kFit;
    static constexpr size_t kSmem = kFixed + (size_t)kStages * kStage;
};

struct Args {
    int M, N;                               // of the result
    int tiles_m, tiles_n, group_m, kb_total;
    float grow;                             // see head_growth()
    // The tiles of the complete rounds run over all of K; the tail_tiles of the last, partly filled one (all, where there
    // are fewer tiles than CTAs) are cut into tail_splits ranges of tail_kb stages, whose sums are joined by join_kernel.
    int tail_tiles, tail_splits, tail_kb;
    float* partials;                        // [tail_splits][tail_tiles][rows of a tile][BN]
    int* err;
    const float* rowf;                      // [M] factor from accumulator to units of log 2
    const float* colf;                      // kStats: [N] the columns' part of it
    HeadScores scores;                      // kStats
    float2* stats;                          // kStats: [M][kParts tiles_n]
    const RowParams* rows;                  // kGrad
    int v0;                                 // kGrad: first column of this piece
    __half* u;                              // kGrad: [2][M][ldu]
    long long u_plane, ldu;
    float* out;                             // kOut: [M][N]
    const RowParams* row_g;                 // kOut: factor of the row (nullable)
    const float* scale;                     // kOut
    int onto;                               // kOut: add to what is there
};

struct Unit {
    int tm, tn, kb0, kb1, slot;             // slot: of a partial tile, -1: the whole of K
};
__host__ __device__ __forceinline__ void tile_at(const Args& g, int t, int& tm, int& tn) {
    // groups of group_m row tiles, rows fastest inside: CTAs that run together share their tiles through L2
    const int per = g.group_m * g.tiles_n, grp = t / per, rem = t - grp * per, first = grp * g.group_m;
    const int rows = g.tiles_m - first < g.group_m ? g.tiles_m - first : g.group_m;
    tn = rem / rows;
    tm = first + (rem - tn * rows);
}
__device__ __forceinline__ Unit unit_at(const Args& g, int u) {
    Unit w{0, 0, 0, g.kb_total, -1};
    const int whole = g.tiles_m * g.tiles_n - g.tail_tiles;
    int tile = u;
    if (u >= whole) {
        const int v = u - whole, sp = v / g.tail_tiles;
        tile = whole + (v - sp * g.tail_tiles);
        w.kb0 = sp * g.tail_kb;
        w.kb1 = min(g.kb_total, w.kb0 + g.tail_kb);
        w.slot = v;
    }
    tile_at(g, tile, w.tm, w.tn);
    return w;
}
__host__ __device__ __forceinline__ int units_of(const Args& g) {
    return g.tiles_m * g.tiles_n - g.tail_tiles + g.tail_tiles * g.tail_splits;
}

// Descriptor of a step of 16 of the contraction index.  K-major: rows of 64 bytes, 64-byte swizzle.  MN-major: groups of 64
// columns, 128-byte rows of one k each, 128-byte swizzle.
template <bool MN>
__device__ __forceinline__ uint64_t step_desc(uint32_t tile, int rows, bool lo, int ks) {
    if (MN) return make_desc(tile + (lo ? BK * 128u : 0u) + ks * 2048u, 2u * BK * 128u, 1024u, 2u);
    return make_desc(tile + (lo ? rows * 64u : 0u) + ks * 32u, 16u, 512u, 4u);
}

// FP16 operands (formats 0), FP32 accumulators.
__host__ __device__ constexpr uint32_t make_idesc_f16(int m, int n, bool a_mn, bool b_mn) {
    return (1u << 4) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

template <bool PAIR>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void commit(uint32_t bar) {
    if (PAIR) umma2_commit(bar, (uint16_t)3);
    else umma_commit(bar);
}

__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
    return p != 0;
}

// A thread's own 32 bytes of its row: a full sector, so that rows go out of registers as they are.  (Through shared memory and
// out as whole lines the gradient's epilogue held the products up: MMAs and copies leave little of the shared memory's rate.)
__device__ __forceinline__ void store32(void* p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
                 "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
// The same where `p` may lie on a multiple of 16 only.
__device__ __forceinline__ void store32(void* p, const uint32_t (&v)[8], bool whole) {
    if (whole) return store32(p, v);
    reinterpret_cast<uint4*>(p)[0] = make_uint4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void load32(const void* p, uint32_t (&v)[8]) {
    const uint4 a = reinterpret_cast<const uint4*>(p)[0], b = reinterpret_cast<const uint4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

template <bool PAIR, bool A_MN, bool B_MN, int BN, int EPI>
__device__ __forceinline__ void run(const CUtensorMap* tmA, const CUtensorMap* tmB, const Args& g) {
    using C = Cfg<PAIR, BN>;
    constexpr int kCols = BN / kParts;      // columns of one epilogue warp
    constexpr int kTileRows = PAIR ? 2 * BM : BM;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const base_ptr = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t bars = base + C::kStages * C::kStage;
    auto full_bar = [&](int s) { return bars + 8u * s; };
    auto empty_bar = [&](int s) { return bars + 8u * (C::kStages + s); };
    auto tfull_bar = [&](int a) { return bars + 8u * (2 * C::kStages + a); };
    auto tempty_bar = [&](int a) { return bars + 8u * (2 * C::kStages + 2 + a); };
    const uint32_t tmem_slot = bars + 8u * (2 * C::kStages + 4);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    const int first = PAIR ? blockIdx.x >> 1 : blockIdx.x, step = PAIR ? gridDim.x >> 1 : gridDim.x;

    if (threadIdx.x == 0) {
        prefetch_tensormap(tmA);
        prefetch_tensormap(tmB);
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(tfull_bar(a), 1);
            mbar_init(tempty_bar(a), (PAIR ? 2 : 1) * kEpiWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(tmem_slot) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(tmem_slot) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(base_ptr + (tmem_slot - base));
    pdl_wait();
    pdl_trigger();
    const int units = units_of(g);

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsFew));
        if (warp == 0 && lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            for (int u = first; u < units && ok; u += step) {
                const Unit w = unit_at(g, u);
                const int a_row = w.tm * kTileRows + (int)rank * BM, b_col = w.tn * BN + (int)rank * C::kBRows;
                for (int kb = w.kb0; kb < w.kb1; ++kb, ++it) {
                    const int s = it % C::kStages;
                    if (!mbar_wait(empty_bar(s), ((it / C::kStages) & 1u) ^ 1u, g.err, 31)) { ok = false; break; }
                    const uint32_t a_dst = base + s * C::kStage, b_dst = a_dst + C::kABytes;
                    // a pair's copies are all counted by the leader's barrier
                    const uint32_t bar = PAIR ? mapa_shared(full_bar(s), 0) : full_bar(s);
                    if (rank == 0) mbar_expect_tx(full_bar(s), (PAIR ? 2u : 1u) * C::kStage);
                    auto load = [&](uint32_t dst, const CUtensorMap* tm, int c0, int c1) {
                        if (PAIR) tma_load_3d_pair(dst, tm, bar, c0, c1, 0);
                        else tma_load_3d(dst, tm, bar, c0, c1, 0);
                    };
                    if (A_MN) {
#pragma unroll
                        for (int a = 0; a < BM / 64; ++a) load(a_dst + a * 2 * BK * 128, tmA, a_row + 64 * a, kb * BK);
                    } else {
                        load(a_dst, tmA, kb * BK, a_row);
                    }
                    if (B_MN) {
#pragma unroll
                        for (int a = 0; a < C::kBRows / 64; ++a) load(b_dst + a * 2 * BK * 128, tmB, b_col + 64 * a, kb * BK);
                    } else {
                        load(b_dst, tmB, kb * BK, b_col);
                    }
                }
            }
            if (!ok)                        // copies in flight land before the shared memory is given back
                for (int i = 0; i < 2000; ++i) __nanosleep(1000);
        }
        if (warp == 1 && rank == 0) {
            constexpr uint32_t idesc = make_idesc_f16(kTileRows, BN, A_MN, B_MN);
            uint32_t it = 0, at = 0;
            bool ok = true;
            for (int u = first; u < units && ok; u += step) {
                const Unit w = unit_at(g, u);
                for (int k0 = w.kb0; k0 < w.kb1 && ok; k0 += kChunk, ++at) {
                    const int acc = at & 1, k1 = min(w.kb1, k0 + kChunk);
                    if (!mbar_wait_warp(tempty_bar(acc), ((at >> 1) & 1u) ^ 1u, g.err, 32)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t d = tmem + (uint32_t)acc * 256u;
                    for (int kb = k0; kb < k1; ++kb, ++it) {
                        const int s = it % C::kStages;
                        if (!mbar_wait_warp(full_bar(s), (it / C::kStages) & 1u, g.err, 33)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t a_base = base + s * C::kStage, b_base = a_base + C::kABytes;
                        if (elect_one()) {
#pragma unroll
                            for (int j = 0; j < BK / 16; ++j) {
                                const uint64_t ah = step_desc<A_MN>(a_base, BM, false, j), al = step_desc<A_MN>(a_base, BM, true, j);
                                const uint64_t bh = step_desc<B_MN>(b_base, C::kBRows, false, j), bl = step_desc<B_MN>(b_base, C::kBRows, true, j);
                                mma_f16<PAIR>(d, al, bh, idesc, (kb > k0 || j > 0) ? 1u : 0u);
                                mma_f16<PAIR>(d, ah, bl, idesc, 1u);
                                mma_f16<PAIR>(d, ah, bh, idesc, 1u);
                            }
                            commit<PAIR>(empty_bar(s));
                            if (kb == k1 - 1) commit<PAIR>(tfull_bar(acc));
                        }
                        __syncwarp();
                    }
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsMany));
        const int quad = warp & 3, part = (warp - 4) >> 2;
        const uint32_t t_row = tmem + ((uint32_t)(quad * 32) << 16) + part * kCols;
        const uint32_t drained[2] = {PAIR ? mapa_shared(tempty_bar(0), 0) : tempty_bar(0), PAIR ? mapa_shared(tempty_bar(1), 0) : tempty_bar(1)};
        const float scale = EPI == kOut ? *g.scale * g.grow : 0.f;
        uint32_t at = 0;
        bool ok = true;
        for (int u = first; u < units && ok; u += step) {
            const Unit w = unit_at(g, u);
            const int row0 = w.tm * kTileRows + (int)rank * BM + quad * 32, row = row0 + lane;
            const int col0 = w.tn * BN + part * kCols, cols = g.N - col0;      // cols may be below zero
            int e_at = 0, e_end = 0;
            int2 entry = make_int2(0, 0), next = entry;
            if (EPI == kStats && row < g.M) {
                if (g.scores.targets) {     // one entry at most
                    int t = g.scores.targets[row];
                    if (t >= g.N) t = 0;
                    entry.x = t;
                    e_end = t >= col0 && t < col0 + kCols ? 1 : 0;
                } else {
                    const uint32_t span = g.scores.spans[(long long)row * (kParts * g.tiles_n) + kParts * w.tn + part];
                    e_at = span & 0xffffu;
                    e_end = span >> 16;
                    if (e_at < e_end) entry = g.scores.entries[(long long)row * g.scores.K + e_at];
                    if (e_at + 1 < e_end) next = g.scores.entries[(long long)row * g.scores.K + e_at + 1];
                }
            }
            RowParams rp{INFINITY, 0.f, 0.f, -1};
            float f = 0.f;
            if (EPI != kOut && row < g.M) f = g.rowf[row] * g.grow;
            if (EPI == kGrad && row < g.M) rp = g.rows[row];
            float v[kCols];
            for (int k0 = w.kb0; k0 < w.kb1; k0 += kChunk, ++at) {
                const int acc = at & 1;
                if (!mbar_wait_warp(tfull_bar(acc), (at >> 1) & 1u, g.err, 34)) { ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < kCols / 32; ++c) {
                    uint32_t rr[32];
                    tmem_ld32(t_row + acc * 256u + c * 32, rr);
                    tmem_ld_wait();
                    if (k0 == w.kb0) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[c * 32 + j] = __uint_as_float(rr[j]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[c * 32 + j] += __uint_as_float(rr[j]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR) mbar_arrive_cluster(drained[acc]);
                    else mbar_arrive(drained[acc]);
                }
            }
            if (!ok) break;
            if (EPI == kStats) {
                if (cols > 0) {
                    const float4* cf = reinterpret_cast<const float4*>(g.colf + col0);     // padded to a multiple of 256 columns
#pragma unroll
                    for (int j = 0; j < kCols / 4; ++j) {
                        const float4 t = cf[j];
                        // rounded here, and not inside the differences below: the maximum is one of these numbers
                        v[4 * j] = __fmul_rn(v[4 * j], t.x * f);
                        v[4 * j + 1] = __fmul_rn(v[4 * j + 1], t.y * f);
                        v[4 * j + 2] = __fmul_rn(v[4 * j + 2], t.z * f);
                        v[4 * j + 3] = __fmul_rn(v[4 * j + 3], t.w * f);
                    }
                }
                // scores of the row's target or entries in this strip, the first two of which are here already
                while (__any_sync(0xffffffffu, e_at < e_end)) {
                    const int c = e_at < e_end ? entry.x - col0 : -1;
                    float z = 0.f;
#pragma unroll
                    for (int q = 0; q < kCols / 16; ++q) {
                        if (!__any_sync(0xffffffffu, (c >> 4) == q)) continue;
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (c == q * 16 + j) z = v[q * 16 + j];
                    }
                    if (e_at < e_end) {
                        g.scores.zk[g.scores.targets ? row : (long long)row * g.scores.K + entry.y] = z;
                        ++e_at;
                        entry = next;
                        if (e_at + 1 < e_end) next = g.scores.entries[(long long)row * g.scores.K + e_at + 1];
                    }
                }
                if (row < g.M && cols > 0) {
                    if (cols < kCols) {
#pragma unroll
                        for (int j = 0; j < kCols; ++j)
                            if (j >= cols) v[j] = -INFINITY;
                    }
                    float m = v[0], s = 0.f;
#pragma unroll
                    for (int j = 1; j < kCols; ++j) m = fmaxf(m, v[j]);
#pragma unroll
                    for (int j = 0; j < kCols; ++j) s += ex2_fast(v[j] - m);
                    g.stats[(long long)row * (kParts * g.tiles_n) + kParts * w.tn + part] = make_float2(m, s);
                } else if (row < g.M) {
                    g.stats[(long long)row * (kParts * g.tiles_n) + kParts * w.tn + part] = make_float2(-INFINITY, 0.f);
                }
            } else if (EPI == kGrad) {
                // 2^15 q = 2^(z - L): what L - 15 is rounded by, and z - L at a q of one, is 2^-22
                const float L = (rp.L - 15.0f) + rp.L_rest;
                const bool live = rp.L != INFINITY, all_live = __all_sync(0xffffffffu, live);
                const int hit = rp.target < 0 ? -1 : rp.target - g.v0 - col0;
                __half* dst = g.u + row * g.ldu + col0;
#pragma unroll
                for (int c = 0; c < kCols / 16; ++c) {
                    if (c * 16 >= cols) break;
                    float e[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) e[j] = ex2_fast(fmaf(v[c * 16 + j], f, -L));
                    if (!all_live) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) e[j] = live ? e[j] : 0.f;
                    }
                    if (__any_sync(0xffffffffu, hit >= c * 16 && hit < c * 16 + 16)) {
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (hit == c * 16 + j) e[j] -= 32768.0f;
                    }
                    uint32_t h[8], l[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) to_pairs(e[2 * j], e[2 * j + 1], h[j], l[j]);
                    if (row < g.M) {
                        store32(dst + c * 16, h);
                        store32(dst + g.u_plane + c * 16, l);
                    }
                }
            } else {
                float rg = 1.f;
                if (g.row_g && w.slot < 0) rg = row < g.M ? g.row_g[row].g : 0.f;
                // a partial tile keeps bare sums
                float* dst = w.slot < 0 ? g.out + (long long)row * g.N + col0
                                        : g.partials + ((long long)w.slot * kTileRows + (int)rank * BM + quad * 32 + lane) * BN + part * kCols;
                const bool onto = g.onto && w.slot < 0, whole = (reinterpret_cast<uintptr_t>(dst) & 31u) == 0;
                const float sc = w.slot < 0 ? scale : 1.f;
                if (row < g.M) {
#pragma unroll
                    for (int c = 0; c < kCols / 8; ++c) {
                        if (c * 8 >= cols) break;
                        uint32_t t[8], old[8];
                        if (onto) load32(dst + c * 8, old);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            float o = rg == 0.f ? 0.f : v[c * 8 + j] * sc * rg;     // zero: the row has no part in the loss
                            if (onto) o += __uint_as_float(old[j]);
                            t[j] = __float_as_uint(o);
                        }
                        store32(dst + c * 8, t, whole);
                    }
                }
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();           // the partner's memory stays in use until both are done
    if (warp == 1) {
        if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

template <bool A_MN, bool B_MN, int BN, int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
head_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ Args g) {
    run<true, A_MN, B_MN, BN, EPI>(&tmA, &tmB, g);
}
template <bool A_MN, bool B_MN, int BN, int EPI>
__global__ void __launch_bounds__(kThreads, 1)
head_single_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ Args g) {
    run<false, A_MN, B_MN, BN, EPI>(&tmA, &tmB, g);
}

// The tail's partial tiles through kOut's last step: LANES threads add every LANES-th range in order, then their sums.
template <int LANES>
__global__ void __launch_bounds__(256) join_kernel(const Args g, int tile_rows, int bn) {
    __shared__ float4 sm[LANES][256 / LANES];
    pdl_wait();
    pdl_trigger();
    constexpr int kOuts = 256 / LANES;
    const int bn4 = bn / 4, y = threadIdx.x / kOuts, at = threadIdx.x % kOuts;
    const long long per = (long long)tile_rows * bn4, total = g.tail_tiles * per;
    const float sc = *g.scale * g.grow;
    for (long long base = (long long)blockIdx.x * kOuts; base < total; base += (long long)gridDim.x * kOuts) {     // total is a multiple of kOuts
        const long long i = base + at;
        const int j = (int)(i / per);
        const long long r = i - j * per;
        const int lr = (int)(r / bn4), c = 4 * (int)(r - (long long)lr * bn4);
        int tm, tn;
        tile_at(g, g.tiles_m * g.tiles_n - g.tail_tiles + j, tm, tn);
        const int row = tm * tile_rows + lr, col = tn * bn + c;
        const bool there = row < g.M && col < g.N;
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
        if (there) {
#pragma unroll 4
            for (int sp = y; sp < g.tail_splits; sp += LANES) t = add4(t, ld4(g.partials, sp * total + i));
        }
        if (LANES > 1) {
            sm[y][at] = t;
            __syncthreads();
            for (int k = 1; y == 0 && k < LANES; ++k) t = add4(t, sm[k][at]);
            __syncthreads();
        }
        if (!there || y > 0) continue;
        const float rg = g.row_g ? g.row_g[row].g : 1.f;
        t = rg == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(t.x * sc * rg, t.y * sc * rg, t.z * sc * rg, t.w * sc * rg);
        float4* p = reinterpret_cast<float4*>(g.out + (long long)row * g.N + col);
        if (g.onto) t = add4(t, *p);
        *p = t;
    }
}

// ------------------------------------------------------------------ host side

bool encode(CUtensorMap* tm, const HalfMat& m, bool mn, int box_rows) {
    const cuuint64_t dims[3] = {(cuuint64_t)m.cols, (cuuint64_t)m.rows, 2};
    const cuuint64_t strides[2] = {(cuuint64_t)m.ld * 2, (cuuint64_t)m.plane * 2};
    const cuuint32_t box[3] = {mn ? 64u : (cuuint32_t)BK, mn ? (cuuint32_t)BK : (cuuint32_t)box_rows, 2}, one[3] = {1, 1, 1};
    return tensor_map_encoder()(tm, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, (void*)m.hi, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                mn ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

float growth(int kb_total) {
    double n = 0.0, nn = 0.0;               // the mean over the contraction index of the instructions in its sum
    for (int left = kb_total; left > 0; left -= kChunk) {
        const double c = 3.0 * (BK / 16) * (left < kChunk ? left : kChunk);
        n += c;
        nn += c * c;
    }
    return head_growth(nn / n);
}

// Ranges of K for each tile of the last round: as many as it has CTAs for, of at least one sum in registers each.
int ranges_of(int tail, int slots, int kb_total) {
    const int sp = slots / tail < kb_total / kChunk ? slots / tail : kb_total / kChunk;
    return sp > 1 ? sp : 1;
}

template <bool PAIR, bool A_MN, bool B_MN, int BN, int EPI>
cudaError_t launch(Args& g, const HalfMat& A, const HalfMat& B, int64_t K, cudaStream_t s) {
    using C = Cfg<PAIR, BN>;
    constexpr int rows = PAIR ? 2 * BM : BM;
    if (!tensor_map_encoder()) return cudaErrorNotSupported;
    CUtensorMap tmA, tmB;
    if (!encode(&tmA, A, A_MN, BM) || !encode(&tmB, B, B_MN, C::kBRows)) return cudaErrorInvalidValue;
    const int sms = sm_count() < 148 ? sm_count() : 148, slots = PAIR ? sms / 2 : sms;      // head_partial_bytes() counts on 148
    g.tiles_m = (g.M + rows - 1) / rows;
    g.tiles_n = (g.N + BN - 1) / BN;
    g.group_m = 4 * g.tiles_n <= slots ? 4 : 16;
    if (g.group_m > g.tiles_m) g.group_m = g.tiles_m;
    g.kb_total = (int)((K + BK - 1) / BK);
    g.grow = growth(g.kb_total);
    g.tail_tiles = g.tail_splits = g.tail_kb = 0;
    const int tiles = g.tiles_m * g.tiles_n;
    if (EPI == kOut && g.partials && tiles % slots) {
        const int tail = tiles % slots, sp = ranges_of(tail, slots, g.kb_total);
        if (sp > 1) {
            g.tail_kb = (g.kb_total + sp - 1) / sp;
            g.tail_splits = (g.kb_total + g.tail_kb - 1) / g.tail_kb;
            g.tail_tiles = tail;
        }
    }
    const int units = units_of(g), n = units < slots ? units : slots;
    if (PAIR) {
        const cudaError_t e = allow_smem<head_pair_kernel<A_MN, B_MN, BN, EPI>>(C::kSmem);
        if (e != cudaSuccess) return e;
        BT_KERNEL_LAUNCH((head_pair_kernel<A_MN, B_MN, BN, EPI>), 2 * n, kThreads, C::kSmem, s, tmA, tmB, g);
    } else {
        const cudaError_t e = allow_smem<head_single_kernel<A_MN, B_MN, BN, EPI>>(C::kSmem);
        if (e != cudaSuccess) return e;
        BT_KERNEL_LAUNCH((head_single_kernel<A_MN, B_MN, BN, EPI>), n, kThreads, C::kSmem, s, tmA, tmB, g);
    }
    BT_COUNT_LAUNCH();
    if (g.tail_tiles) {
        const long long want = ((long long)g.tail_tiles * rows * BN / 4 + 255) / 256;
        if (g.tail_splits >= 8) BT_KERNEL_LAUNCH((join_kernel<8>), (int)(8 * want < 148 * 8 ? 8 * want : 148 * 8), 256, 0, s, g, rows, BN);
        else BT_KERNEL_LAUNCH((join_kernel<1>), (int)(want < 148 * 8 ? want : 148 * 8), 256, 0, s, g, rows, BN);
        BT_COUNT_LAUNCH();
    }
    return cudaGetLastError();
}

// Tiles of a product.  A CTA's share of 256 columns takes one unit of time per stage, of 128 half of that and some of its operands
// again; CTAs on their own (128 rows) bring twice as much of B per row as pairs (256 rows) but are twice as many.  A tile
// costs some ten stages more for filling and emptying.  The shape of the least time over all rounds is taken (the last one counts
// in part where it is cut along K): pairs and 256 columns where there is work for all SMs, smaller ones where there is not.
// Gradients of 372 rows, C 1,440, V 835 take 60 us, with 256-wide pairs alone 75; of 595 rows, C 224, V 1,607 41 and 55.
struct Tiles {
    bool pair;
    int bn;
};
Tiles choose_tiles(int64_t M, int64_t N, int64_t K, bool cut) {
    const double kb = (double)((K + BK - 1) / BK);
    Tiles best{true, 256};
    double least = 1e300;
    for (const Tiles t : {Tiles{true, 256}, Tiles{true, 128}, Tiles{false, 256}, Tiles{false, 128}}) {
        if (t.pair && t.bn == 128 && !cut) continue;       // not compiled
        const int64_t rows = t.pair ? 2 * BM : BM, units = ((M + rows - 1) / rows) * ((N + t.bn - 1) / t.bn), slots = t.pair ? 74 : 148;
        const double stage = t.bn == 256 ? (t.pair ? 1.0 : 1.2) : (t.pair ? 0.7 : 0.85);
        double rounds = (double)((units + slots - 1) / slots);
        if (cut && units % slots) rounds += 1.0 / ranges_of((int)(units % slots), (int)slots, (int)kb) - 1.0;
        const double cost = rounds * (kb * stage + (t.bn == 256 ? 12 : 8));
        if (cost < least) {
            least = cost;
            best = t;
        }
    }
    return best;
}

template <int EPI>
cudaError_t launch_wide(Args& g, const HalfMat& A, const HalfMat& B, int64_t K, cudaStream_t s) {
    const Tiles t = choose_tiles(g.M, g.N, K, false);
    if (t.pair) return launch<true, false, false, 256, EPI>(g, A, B, K, s);
    return t.bn == 256 ? launch<false, false, false, 256, EPI>(g, A, B, K, s) : launch<false, false, false, 128, EPI>(g, A, B, K, s);
}

template <bool A_MN>
cudaError_t launch_out(Args& g, const HalfMat& A, const HalfMat& B, int64_t K, cudaStream_t s) {
    const Tiles t = choose_tiles(g.M, g.N, K, true);
    if (t.pair) return t.bn == 256 ? launch<true, A_MN, true, 256, kOut>(g, A, B, K, s) : launch<true, A_MN, true, 128, kOut>(g, A, B, K, s);
    return t.bn == 256 ? launch<false, A_MN, true, 256, kOut>(g, A, B, K, s) : launch<false, A_MN, true, 128, kOut>(g, A, B, K, s);
}

}  // namespace

HeadStrips head_stats_strips(int64_t N, int C, int V) {
    const int bn = choose_tiles(N, V, C, false).bn;
    return HeadStrips{bn / kParts, kParts * ((V + bn - 1) / bn)};
}
size_t head_partial_bytes() { return (size_t)148 * BM * 256 * sizeof(float); }

cudaError_t launch_head_stats(const HalfMat& x, const HalfMat& w, const float* rowf, const float* colf, const HeadScores& scores, float2* stats,
                              int* err, cudaStream_t s) {
    Args g{};
    g.M = (int)x.rows; g.N = (int)w.rows;
    g.rowf = rowf; g.colf = colf; g.scores = scores; g.stats = stats; g.err = err;
    return launch_wide<kStats>(g, x, w, x.cols, s);
}

cudaError_t launch_head_grad(const HalfMat& x, const HalfMat& w, int v0, const float* rowf, const RowParams* rows, __half* u, int64_t ldu,
                             int64_t u_plane, int* err, cudaStream_t s) {
    Args g{};
    g.M = (int)x.rows; g.N = (int)w.rows;
    g.rowf = rowf; g.rows = rows; g.v0 = v0; g.u = u; g.ldu = ldu; g.u_plane = u_plane; g.err = err;
    return launch_wide<kGrad>(g, x, w, x.cols, s);
}

cudaError_t launch_head_dx(const HalfMat& u, const HalfMat& w, const RowParams* rows, const float* scale, bool onto, float* dx, float* partials,
                           int* err, cudaStream_t s) {
    Args g{};
    g.M = (int)u.rows; g.N = (int)w.cols;
    g.out = dx; g.row_g = rows; g.scale = scale; g.onto = onto; g.partials = partials; g.err = err;
    return launch_out<false>(g, u, w, u.cols, s);
}

cudaError_t launch_head_dw(const HalfMat& u, const HalfMat& y, const float* scale, float* dw, float* partials, int* err, cudaStream_t s) {
    Args g{};
    g.M = (int)u.cols; g.N = (int)y.cols;
    g.out = dw; g.scale = scale; g.partials = partials; g.err = err;
    return launch_out<true>(g, u, y, u.rows, s);
}

}  // namespace bt
