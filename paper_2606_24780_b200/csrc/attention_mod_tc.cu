// Attention with modified scores on the 5th-generation tensor cores, head_dim 64, 3xTF32.
//
// The division of the work is that of the plain causal kernels (one CTA = 128 rows of one head, one
// row per tensor-memory lane, 64-row tiles of the other side, products spread over several issuing
// threads, bounded mbarrier waits): see attention_tc.cu and attention_tc_bwd.cu.  What differs:
//
//   Tiles      A CTA walks the tiles between the ends of its rows' ranges (SpanView): with packed documents
//              the work is that of the documents.  A thread owns a row, so the mask is two comparisons
//              with the row's own range, made only in tiles that the range does not cover.
//   Scores     z = cap tanh(u) - slope |i - j| in base-2 units (attention_mod.cuh), at compile time with or
//              without cap and slope.  The backward multiplies its own rows by 1 / (cap sqrt d) before
//              the product, so u comes out of the tensor core.
//   Rounding   The tensor core truncates when it adds to its accumulator, so sums that run over a whole walk
//              drift: by 3.2e-6 of dK over 1,024 causal positions and 1.7e-5 over 8,192.  Here no accumulator outlives a
//              tile: the products of a tile start from zero and are added to registers in FP32, rounded
//              to nearest.  And the two small terms of a split product (lo hi, hi lo) go in before
//              the large one, or into columns of their own, so that a tile's sum is truncated eight times at its full size, not 24 times.
#include "attention_mod.cuh"

namespace bt {

using namespace tc;
using namespace mod;

namespace {

constexpr int HD = 64, BR = 128, BT64 = 64;
constexpr uint32_t kResBytes = 2u * 2u * BR * 128u;    // 128 own rows: 2 k-blocks x (hi, lo) x 128 rows x 128 B
constexpr uint32_t kTile = 2u * 2u * BT64 * 128u;      // one streamed 64-row tile (hi, lo) in one layout
//  MN-major 64-row tile: 2 column groups of [hi | lo][64 rows][128 B]; a k-step is 8 rows
__device__ __forceinline__ constexpr uint32_t mn_off(int ks, bool lo) { return (lo ? BT64 * 128u : 0u) + (uint32_t)ks * 1024u; }
__device__ __forceinline__ DescBase mn_base(uint32_t tile) { return make_desc_base(tile, 2u * BT64 * 128u, 512u, 1u); }

struct ModTcArgs {
    AttnModArgs a;
    int head_group;          // heads per group of the CTA order (grouped_block)
};

__device__ __forceinline__ void alloc_tmem(uint32_t slot) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void free_tmem(uint32_t tmem) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}
// A role whose wait ran out lets copies in flight land before the CTA exits.
__device__ __forceinline__ void settle() {
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
}

// ------------------------------------------------------------------------------------------ forward
//
//   warps 0-3, 4-7   softmax warpgroups on alternate key tiles, each with its own running maximum, sum and output
//                    in registers, merged at the end
//   warp 8           TMA producer (Q once; K and V tiles through one ring of five slots in the order
//                    K0 K1 V0 K2 V1 ...);  warp 9 issues S = Q K^T, warp 10 O_tile = P V (P from tensor memory)
//   tensor memory    per buffer b: S at 256b, P_hi at 256b + 64, P_lo at 256b + 128, O_tile at 256b + 192
constexpr int kFwdThreads = 352, kWarpLoad = 8, kWarpS = 9, kWarpO = 10, kSlots = 5;
constexpr uint32_t kFwdSmem = 1024u + kResBytes + kSlots * kTile + 256u;
static_assert(kFwdSmem <= 232448u, "shared memory");
__device__ __forceinline__ int pos_k(int t) { return t == 0 ? 0 : 2 * t - 1; }
__device__ __forceinline__ int pos_v(int t) { return 2 * t + 2; }

template <bool CAP, bool SLOPE>
__global__ void __launch_bounds__(kFwdThreads, 1)
attn_mod_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                    const __grid_constant__ CUtensorMap tmV, const ModTcArgs args) {
    const AttnModArgs& g = args.a;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_s = base, ring_s = q_s + kResBytes, bars = ring_s + kSlots * kTile;
    const uint32_t q_full = bars;
    auto slot_full = [&](int i) { return bars + 8u * (1 + i); };
    auto slot_empty = [&](int i) { return bars + 8u * (6 + i); };
    auto s_full = [&](int b) { return bars + 8u * (11 + b); };
    auto p_full = [&](int b) { return bars + 8u * (13 + b); };
    auto o_full = [&](int b) { return bars + 8u * (15 + b); };
    const uint32_t merge_full = bars + 8u * 17, all_done = bars + 8u * 18, tmem_slot = bars + 8u * 19;
    auto smem_ptr = [&](uint32_t addr) { return smem_raw + (addr - smem_u32(smem_raw)); };

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int bh, yb;
    grouped_block(args.head_group, bh, yb);
    const int qt = (int)gridDim.y - 1 - yb;
    const int b = bh / g.H, h = bh % g.H, q0 = qt * BR;
    const int row_base = b * g.T;

    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(slot_full(i), 1);
            mbar_init(slot_empty(i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(s_full(i), 1);
            mbar_init(p_full(i), 4);
            mbar_init(o_full(i), 1);
        }
        mbar_init(merge_full, 4);
        mbar_init(all_done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kWarpS) alloc_tmem(tmem_slot);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem_ptr(tmem_slot));
    pdl_wait();      // set-up done; global memory is touched from here on
    pdl_trigger();
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *g.err = 0;
    const int2 range = block_range(g.spans.kblock, b, g.T, q0, BR, false);
    const int kt0 = range.x / BT64, n_kt = range.x < range.y ? (range.y - 1) / BT64 + 1 - kt0 : 0;

    if (warp == kWarpLoad) {
        if (lane == 0 && n_kt > 0) {
            mbar_expect_tx(q_full, kResBytes);
            for (int kb = 0; kb < 2; ++kb)
                tma_load_3d(q_s + kb * (kResBytes / 2), &tmQ, q_full, h * HD + kb * 32, row_base + q0, 0);
            bool ok = true;
            const int n_pos = pos_v(n_kt - 1) + 1;
            int slot = 0;
            uint32_t round = 0;
            for (int p = 0; p < n_pos && ok; ++p) {
                const bool is_k = p == 0 || (p & 1);
                const int t = p == 0 ? 0 : (is_k ? (p + 1) >> 1 : (p - 2) >> 1);
                if (t < n_kt) {                          // only K(n_kt) near the end falls outside
                    if (!mbar_wait(slot_empty(slot), (round & 1u) ^ 1u, g.err, 111)) { ok = false; break; }
                    mbar_expect_tx(slot_full(slot), kTile);
                    for (int kb = 0; kb < 2; ++kb)
                        tma_load_3d(ring_s + (uint32_t)slot * kTile + kb * (kTile / 2), is_k ? &tmK : &tmV, slot_full(slot),
                                    (is_k ? g.C : 2 * g.C) + h * HD + kb * 32, row_base + (kt0 + t) * BT64, 0);
                }
                if (++slot == kSlots) { slot = 0; ++round; }
            }
            if (!ok) settle();
        }
    } else if (warp == kWarpS) {
        if (lane == 0 && n_kt > 0) {
            constexpr uint32_t idesc = make_idesc_tf32(BR, BT64, false, false);
            bool ok = mbar_wait(q_full, 0, g.err, 113);
            const DescBase qd = kmaj_base(q_s);
            for (int t = 0; t < n_kt && ok; ++t) {
                const int buf = t & 1, pk = pos_k(t), slot = pk % kSlots;
                if (!mbar_wait(slot_full(slot), (uint32_t)(pk / kSlots) & 1u, g.err, 114)) { ok = false; break; }
                // S[buf] is free once the softmax of tile t - 2 has read it (it then publishes P)
                if (t >= 2 && !mbar_wait(p_full(buf), ((t - 2) >> 1) & 1u, g.err, 120)) { ok = false; break; }
                tc_fence_after();
                const uint32_t d = tmem + (uint32_t)buf * 256u;
                const DescBase kd = kmaj_base(ring_s + (uint32_t)slot * kTile);
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    umma_tf32(d, qd.at(kmaj_off(BR, ks, true)), kd.at(kmaj_off(BT64, ks, false)), idesc, ks > 0 ? 1u : 0u);
                    umma_tf32(d, qd.at(kmaj_off(BR, ks, false)), kd.at(kmaj_off(BT64, ks, true)), idesc, 1u);
                }
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    umma_tf32(d, qd.at(kmaj_off(BR, ks, false)), kd.at(kmaj_off(BT64, ks, false)), idesc, 1u);
                umma_commit(slot_empty(slot));
                umma_commit(s_full(buf));
            }
        }
    } else if (warp == kWarpO) {
        if (lane == 0 && n_kt > 0) {
            constexpr uint32_t idesc = make_idesc_tf32(BR, HD, false, true);
            bool ok = true;
            for (int t = 0; t < n_kt && ok; ++t) {
                const int buf = t & 1, pv = pos_v(t), slot = pv % kSlots;
                // P(t) published; the softmax warps read O[buf] of tile t - 2 before publishing it
                if (!mbar_wait(p_full(buf), (t >> 1) & 1u, g.err, 115)) { ok = false; break; }
                if (!mbar_wait(slot_full(slot), (uint32_t)(pv / kSlots) & 1u, g.err, 116)) { ok = false; break; }
                tc_fence_after();
                const uint32_t t0 = tmem + (uint32_t)buf * 256u, d = t0 + 192u;
                const DescBase vd = mn_base(ring_s + (uint32_t)slot * kTile);
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    umma_tf32_ts(d, t0 + 128u + ks * 8u, vd.at(mn_off(ks, false)), idesc, ks > 0 ? 1u : 0u);  // P_lo V_hi
                    umma_tf32_ts(d, t0 + 64u + ks * 8u, vd.at(mn_off(ks, true)), idesc, 1u);                  // P_hi V_lo
                }
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) umma_tf32_ts(d, t0 + 64u + ks * 8u, vd.at(mn_off(ks, false)), idesc, 1u);
                umma_commit(slot_empty(slot));
                umma_commit(o_full(buf));
            }
            if (ok) umma_commit(all_done);
        }
    } else if (warp < 8) {
        const int wg = warp >> 2, lane_group = warp & 3;
        const int rloc = lane_group * 32 + lane, row = q0 + rloc;
        const uint32_t t_lane = tmem + ((uint32_t)(lane_group * 32) << 16) + (uint32_t)wg * 256u;
        const Score sc = make_score<CAP, SLOPE>(1.0f / sqrtf((float)HD), g.cap, g.slopes, h);
        const float c = (CAP || SLOPE) ? 1.0f : sc.unit;       // from score_tile's result to base-2 units
        const int2 span = row_range(g.spans.k, b, g.T, row, false);
        float m = -INFINITY, l = 0.f, corr_prev = 0.f;
        float o_reg[HD];
#pragma unroll
        for (int i = 0; i < HD; ++i) o_reg[i] = 0.f;
        bool ok = true;

        auto add_output = [&](int t, float corr) -> bool {
            if (!mbar_wait_warp(o_full(wg), (t >> 1) & 1u, g.err, 117)) return false;
            tc_fence_after();
            uint32_t r0[32], r1[32];
            tmem_ld32(t_lane + 192u, r0);
            tmem_ld32(t_lane + 224u, r1);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                o_reg[i] = fmaf(o_reg[i], corr, __uint_as_float(r0[i]));
                o_reg[32 + i] = fmaf(o_reg[32 + i], corr, __uint_as_float(r1[i]));
            }
            return true;
        };

        int last = -1;
        for (int t = wg; t < n_kt && ok; t += 2) {
            // this warpgroup's previous tile first: the P V product of this tile overwrites O[wg]
            if (last >= 0 && !add_output(last, corr_prev)) { ok = false; break; }
            if (!mbar_wait_warp(s_full(wg), (t >> 1) & 1u, g.err, 118)) { ok = false; break; }
            tc_fence_after();
            float s0[32], s1[32];
            {
                uint32_t r0[32], r1[32];
                tmem_ld32(t_lane, r0);
                tmem_ld32(t_lane + 32u, r1);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    s0[i] = __uint_as_float(r0[i]);
                    s1[i] = __uint_as_float(r1[i]);
                }
            }
            const int key0 = (kt0 + t) * BT64;
            score_tile<CAP, SLOPE, 32>(s0, sc, row - key0);
            score_tile<CAP, SLOPE, 32>(s1, sc, row - key0 - 32);
            if (key0 < span.x || key0 + BT64 > span.y) {      // this row does not read the whole tile
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    if (key0 + i < span.x || key0 + i >= span.y) s0[i] = -INFINITY;
                    if (key0 + 32 + i < span.x || key0 + 32 + i >= span.y) s1[i] = -INFINITY;
                }
            }
            float mx = -INFINITY;
#pragma unroll
            for (int i = 0; i < 32; ++i) mx = fmaxf(mx, fmaxf(s0[i], s1[i]));
            // a row that has read nothing yet keeps its maximum at -inf; the arithmetic stays finite
            const float m_new = fmaxf(m, mx);
            const float m_use = (m_new == -INFINITY) ? 0.f : m_new;
            const float corr = ex2_approx((m - m_use) * c);
            const float mc = m_use * c;
            float sum = 0.f;
            uint32_t hi[32], lo[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const float p = ex2_approx(fmaf(s0[i], c, -mc));
                sum += p;
                split_tf32_int(p, hi[i], lo[i]);
            }
            tmem_st32(t_lane + 64u, hi);
            tmem_st32(t_lane + 128u, lo);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const float p = ex2_approx(fmaf(s1[i], c, -mc));
                sum += p;
                split_tf32_int(p, hi[i], lo[i]);
            }
            tmem_st32(t_lane + 96u, hi);
            tmem_st32(t_lane + 160u, lo);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full(wg));
            l = fmaf(l, corr, sum);
            m = m_new;
            corr_prev = corr;
            last = t;
        }
        if (ok && last >= 0) ok = add_output(last, corr_prev);

        // merge: warpgroup 1 hands (m, l, O) of its rows to warpgroup 0 through the first ring slots, idle once
        // every product has completed
        float* xch = reinterpret_cast<float*>(smem_ptr(ring_s));   // [128][66]
        if (wg == 1) {
            if (ok && n_kt > 0) ok = mbar_wait_warp(all_done, 0, g.err, 121);
            float* dst = xch + rloc * 66;
            dst[64] = m;
            dst[65] = l;
#pragma unroll
            for (int i = 0; i < HD; ++i) dst[i] = o_reg[i];
            __threadfence_block();
            __syncwarp();
            if (lane == 0) mbar_arrive(merge_full);
        } else {
            if (ok) ok = mbar_wait_warp(merge_full, 0, g.err, 119);
            if (ok) {
                const float* src = xch + rloc * 66;
                const float m1 = src[64], l1 = src[65];
                const float mm = fmaxf(m, m1), m_use = mm == -INFINITY ? 0.f : mm;
                const float f0 = ex2_approx((m - m_use) * c), f1 = ex2_approx((m1 - m_use) * c);
                l = l * f0 + l1 * f1;
                const float inv = l > 0.f ? 1.0f / l : 0.f;             // a row that reads nothing is zero
#pragma unroll
                for (int i = 0; i < HD; ++i) o_reg[i] = (o_reg[i] * f0 + src[i] * f1) * inv;
                const int wrow0 = q0 + lane_group * 32, nvalid = max(0, min(32, g.T - wrow0));
                const int64_t off0 = ((int64_t)(row_base + wrow0)) * g.C + h * HD;
                float* tile = reinterpret_cast<float*>(smem_ptr(ring_s + 2u * kTile) + (uint32_t)lane_group * kRowTileBytes);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float v[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = o_reg[half * 32 + i];
                    warp_rows_store(v, tile, lane, nvalid, g.o ? g.o + off0 + half * 32 : nullptr,
                                    g.o_hi ? g.o_hi + off0 + half * 32 : nullptr, g.o_hi ? g.o_lo + off0 + half * 32 : nullptr,
                                    g.C, nullptr);
                }
                if (row < g.T) g.lse[((int64_t)b * g.H + h) * g.T + row] = l > 0.f ? (mm * c + log2f(l)) * kLn2 : -INFINITY;
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == kWarpS) free_tmem(tmem);
}

// -------------------------------------------------------------------------------------- backward, dK and dV
//
// One CTA owns 128 keys and walks the 64-row query tiles that read them.
//     S^T = K' Q^T | dP^T = V dO^T | dV_tile = P^T dO | dK_tile = dS^T Q,  P^T = exp2(z - lse), dS^T = P^T o (dP^T - D) (1 - tanh^2)
// Warp 1 issues dV(t), S^T(t+1), ..., warp 10 dK(t), dP^T(t+1), ...: within a chain the product that overwrites a
// region follows the one that last read it.  dV(t) is complete when S^T(t+1) is (one thread's products
// complete in order), so the element-wise threads add it to their registers between those two
// waits, before they publish P^T(t+1), which lets dV(t+1) overwrite it; dK likewise with dP^T and dS^T.
//   tensor memory: K' hi|lo 0-127, dK 128-191, dV 192-255, S^T -> P^T_hi 256-319, P^T_lo 320-383,
//                  dP^T -> dS^T_hi 384-447, dS^T_lo 448-511
//   warps 2-9: both warpgroups on every tile, 32 of its queries each; of the accumulators 32 columns each
constexpr int kDkvThreads = 352, kWarpMma2 = 10;
constexpr uint32_t kDkvSmem = 1024u + kResBytes + 4u * kTile + 256u + 4u * kRowTileBytes + 1024u;
static_assert(kDkvSmem <= 232448u, "shared memory");

template <bool CAP, bool SLOPE>
__global__ void __launch_bounds__(kDkvThreads, 1)
attn_mod_dkv_kernel(const __grid_constant__ CUtensorMap tmQk, const __grid_constant__ CUtensorMap tmQm,
                    const __grid_constant__ CUtensorMap tmDOk, const __grid_constant__ CUtensorMap tmDOm,
                    const __grid_constant__ CUtensorMap tmVres, const ModTcArgs args) {
    const AttnModArgs& g = args.a;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t v_s = base, qk_s = base + kResBytes, dok_s = qk_s + kTile, dom_s = dok_s + kTile, qm_s = dom_s + kTile;
    const uint32_t bars = qm_s + kTile;
    enum { V_FULL = 0, QK_FULL, QK_EMPTY, DOK_FULL, DOK_EMPTY, DOM_FULL, DOM_EMPTY, QM_FULL, QM_EMPTY, S_FULL,
           DP_FULL, ACC_FULL, P_READY, DS_READY, K_READY, STAT_READY, N_BARS };
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    const uint32_t tmem_slot = bars + 8u * N_BARS;
    auto smem_ptr = [&](uint32_t addr) { return smem_raw + (addr - smem_u32(smem_raw)); };

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int bh, yb;
    grouped_block(args.head_group, bh, yb);
    const int b = bh / g.H, h = bh % g.H, j0 = yb * BR;
    const int row_base = b * g.T;

    if (threadIdx.x == 0) {
        for (int i = 0; i < P_READY; ++i) mbar_init(bar(i), i == ACC_FULL ? 2 : 1);   // both issuing threads commit at the end
        mbar_init(bar(P_READY), 8);
        mbar_init(bar(DS_READY), 8);
        mbar_init(bar(K_READY), 4);
        mbar_init(bar(STAT_READY), 8);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) alloc_tmem(tmem_slot);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem_ptr(tmem_slot));
    pdl_wait();      // set-up done; global memory is touched from here on
    pdl_trigger();
    const uint32_t tK_hi = tmem, tK_lo = tmem + 64, tdK = tmem + 128, tdV = tmem + 192;
    const uint32_t tS = tmem + 256, tPlo = tmem + 320, tdP = tmem + 384, tdSlo = tmem + 448;
    const int2 range = block_range(g.spans.qblock, b, g.T, j0, BR, true);
    const int qt0 = range.x / BT64, n_t = range.x < range.y ? (range.y - 1) / BT64 + 1 - qt0 : 0;
    auto q_row0 = [&](int t) { return (qt0 + t) * BT64; };

    if (warp == 0) {
        if (lane == 0 && n_t > 0) {
            mbar_expect_tx(bar(V_FULL), kResBytes);
            for (int kb = 0; kb < 2; ++kb)
                tma_load_3d(v_s + kb * (kResBytes / 2), &tmVres, bar(V_FULL), 2 * g.C + h * HD + kb * 32, row_base + j0, 0);
            bool ok = true;
            // in the order the products consume them: S^T(0), dP^T(0), then per tile dV(t), S^T(t+1), dK(t), dP^T(t+1)
            for (int i = 0; i < 4 * n_t + 2 && ok; ++i) {
                // j: 0 dO MN-major (t), 1 Q K-major (t+1), 2 Q MN-major (t), 3 dO K-major (t+1); first Q(0), dO(0) K-major
                const int j = i == 0 ? 1 : i == 1 ? 3 : (i - 2) & 3;
                const int t = i < 2 ? 0 : ((i - 2) >> 2) + (j & 1);
                if (t >= n_t) continue;
                const uint32_t dst = j == 0 ? dom_s : j == 1 ? qk_s : j == 2 ? qm_s : dok_s;
                const CUtensorMap* tm = j == 0 ? &tmDOm : j == 1 ? &tmQk : j == 2 ? &tmQm : &tmDOk;
                const int full = j == 0 ? DOM_FULL : j == 1 ? QK_FULL : j == 2 ? QM_FULL : DOK_FULL;
                ok = mbar_wait_ool(bar(full + 1), (uint32_t)(t & 1) ^ 1u, g.err, 131);   // every EMPTY barrier follows its FULL barrier
                if (!ok) break;
                mbar_expect_tx(bar(full), kTile);
                for (int part = 0; part < 2; ++part)
                    tma_load_3d(dst + part * (kTile / 2), tm, bar(full), h * HD + part * 32, row_base + q_row0(t), 0);
            }
            if (!ok) settle();
        }
    } else if (warp == 1 || warp == kWarpMma2) {
        if (lane == 0 && n_t > 0) {
            constexpr uint32_t idesc_a = make_idesc_tf32(BR, BT64, false, false);
            constexpr uint32_t idesc_a2 = make_idesc_tf32(BR, 2 * BT64, false, false);   // B = [hi rows | lo rows]
            constexpr uint32_t idesc_b = make_idesc_tf32(BR, HD, false, true);
            const bool score_chain = warp == 1;
            bool ok = score_chain ? mbar_wait_ool(bar(K_READY), 0, g.err, 134) : mbar_wait_ool(bar(V_FULL), 0, g.err, 133);
            const DescBase vd = kmaj_base(v_s), qd = kmaj_base(qk_s), od = kmaj_base(dok_s);
            const DescBase omd = mn_base(dom_s), qmd = mn_base(qm_s);
            // Score products: a tile's lo rows follow its hi rows, so [hi | lo] is one operand of 128 rows whose
            // second half lands in the neighbouring 64 columns; A_lo hi joins it there, the small terms
            // apart from the large one, and the reader adds the halves.
            auto issue_s = [&](int t) -> bool {
                if (!mbar_wait_ool(bar(QK_FULL), (uint32_t)(t & 1), g.err, 135)) return false;
                tc_fence_after();
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    const uint64_t q_hl = qd.at(kmaj_off(BT64, ks, false));
                    umma_tf32_ts(tS, tK_hi + ks * 8, q_hl, idesc_a2, ks > 0 ? 1u : 0u);   // K'_hi Q_hi | K'_hi Q_lo
                    umma_tf32_ts(tPlo, tK_lo + ks * 8, q_hl, idesc_a, 1u);                // + K'_lo Q_hi
                }
                umma_commit(bar(QK_EMPTY));
                umma_commit(bar(S_FULL));
                return true;
            };
            auto issue_dp = [&](int t) -> bool {
                if (!mbar_wait_ool(bar(DOK_FULL), (uint32_t)(t & 1), g.err, 136)) return false;
                tc_fence_after();
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    const uint64_t v_hi = vd.at(kmaj_off(BR, ks, false)), v_lo = vd.at(kmaj_off(BR, ks, true));
                    const uint64_t o_hl = od.at(kmaj_off(BT64, ks, false));
                    umma_tf32(tdP, v_hi, o_hl, idesc_a2, ks > 0 ? 1u : 0u);    // V_hi dO_hi | V_hi dO_lo
                    umma_tf32(tdSlo, v_lo, o_hl, idesc_a, 1u);                 // + V_lo dO_hi
                }
                umma_commit(bar(DOK_EMPTY));
                umma_commit(bar(DP_FULL));
                return true;
            };
            // Accumulating products, from zero in every tile, the small terms first.
            auto issue_acc = [&](int t, uint32_t acc, uint32_t a_hi, uint32_t a_lo, const DescBase& bd, int ready, int full) -> bool {
                if (!mbar_wait_ool(bar(ready), (uint32_t)(t & 1), g.err, 137)) return false;
                if (!mbar_wait_ool(bar(full), (uint32_t)(t & 1), g.err, 138)) return false;
                tc_fence_after();
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    umma_tf32_ts(acc, a_lo + ks * 8, bd.at(mn_off(ks, false)), idesc_b, ks > 0 ? 1u : 0u);
                    umma_tf32_ts(acc, a_hi + ks * 8, bd.at(mn_off(ks, true)), idesc_b, 1u);
                }
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) umma_tf32_ts(acc, a_hi + ks * 8, bd.at(mn_off(ks, false)), idesc_b, 1u);
                umma_commit(bar(full + 1));
                return true;
            };
            if (score_chain) {
                for (int t = 0; t <= n_t && ok; ++t) {
                    if (t > 0) ok = issue_acc(t - 1, tdV, tS, tPlo, omd, P_READY, DOM_FULL);   // dV += P^T dO
                    if (ok && t < n_t) ok = issue_s(t);
                }
            } else {
                for (int t = 0; t <= n_t && ok; ++t) {
                    if (t > 0) ok = issue_acc(t - 1, tdK, tdP, tdSlo, qmd, DS_READY, QM_FULL); // dK += dS^T Q
                    if (ok && t < n_t) ok = issue_dp(t);
                }
            }
            if (ok) umma_commit(bar(ACC_FULL));
        }
    } else if (warp < kWarpMma2) {
        const int wg = (warp - 2) >> 2, lane_group = warp & 3;
        const int etid = lane_group * 32 + lane, key = j0 + etid;
        const uint32_t t_lane = ((uint32_t)(lane_group * 32) << 16);
        const float scale = 1.0f / sqrtf((float)HD);
        const Score sc = make_score<CAP, SLOPE>(scale, g.cap, g.slopes, h);
        const int64_t gs = 3 * (int64_t)g.C;
        const int64_t lb = ((int64_t)b * g.H + h) * g.T;
        if (wg == 0 && n_t > 0) {   // K' = K * unit into tensor memory
            const int wrow0 = min(j0 + lane_group * 32, g.T - 1);
            const int64_t off = (int64_t)(row_base + wrow0) * gs + g.C + h * HD;
            float* tile = reinterpret_cast<float*>(smem_ptr(bars + 256u) + (uint32_t)lane_group * kRowTileBytes);
            rows_to_tmem(g.qkv + off, g.qkv_lo + off, gs, max(1, min(32, g.T - wrow0)), sc.unit, tK_hi + t_lane, tK_lo + t_lane,
                         tile, lane);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(K_READY));
        }
        const int2 span = row_range(g.spans.q, b, g.T, key, true);
        bool ok = true;
        const uint32_t c0 = 32u * (uint32_t)wg;
        // Statistics of a tile's 64 queries (lse in base-2 units, D) through shared memory, one tile ahead.  All
        // eight warps arrive, those without a value too: no warp can be two phases behind.
        float* stat = reinterpret_cast<float*>(smem_ptr(bars + 256u + 4u * kRowTileBytes));
        const int sidx = (warp - 2) * 32 + lane;
        auto fetch_stat = [&](int t) -> float {
            const int r = min(q_row0(t) + (sidx & 63), g.T - 1);   // rows past the end are masked below
            return sidx < 64 ? __ldg(g.lse + lb + r) * kLog2e : __ldg(g.dvec + lb + r);
        };
        auto publish_stat = [&](int t, float v) {
            if (sidx < 128) {
                stat[(t & 1) * 128 + sidx] = v;
                __threadfence_block();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(STAT_READY));
        };
        float acc_v[32], acc_k[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) acc_v[i] = acc_k[i] = 0.f;
        auto add_tile = [&](uint32_t t_acc, float (&acc)[32]) {
            uint32_t r[32];
            tmem_ld32(t_acc + t_lane + c0, r);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[i] += __uint_as_float(r[i]);
        };
        if (n_t > 0) publish_stat(0, sidx < 128 ? fetch_stat(0) : 0.f);
        for (int t = 0; t < n_t && ok; ++t) {
            const int q0 = q_row0(t) + 32 * wg;
            float next_stat = 0.f;
            if (sidx < 128 && t + 1 < n_t) next_stat = fetch_stat(t + 1);   // in flight during this tile
            if (!mbar_wait_warp_ool(bar(STAT_READY), (uint32_t)(t & 1), g.err, 142)) { ok = false; break; }
            const float4* Ls = reinterpret_cast<const float4*>(stat + (t & 1) * 128 + 32 * wg);
            const float4* Ds = Ls + 16;
            if (!mbar_wait_warp_ool(bar(S_FULL), (uint32_t)(t & 1), g.err, 141)) { ok = false; break; }
            tc_fence_after();
            float p[32], f[32];
            uint32_t s[32], lo[32];
            tmem_ld32(tS + t_lane + c0, s);
            tmem_ld32(tPlo + t_lane + c0, lo);        // the small half of the score product
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) p[i] = __uint_as_float(s[i]) + __uint_as_float(lo[i]);
            score_tile_grad<CAP, SLOPE, 32>(p, f, sc, key - q0);
            const bool whole = q0 >= span.x && q0 + 32 <= span.y;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float4 l4 = Ls[i];
                p[4 * i] = ex2_approx(p[4 * i] - l4.x);
                p[4 * i + 1] = ex2_approx(p[4 * i + 1] - l4.y);
                p[4 * i + 2] = ex2_approx(p[4 * i + 2] - l4.z);
                p[4 * i + 3] = ex2_approx(p[4 * i + 3] - l4.w);
            }
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (q0 + i < span.x || q0 + i >= span.y) p[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                split_tf32_int(p[i], s[i], lo[i]);
                if (CAP) p[i] *= f[i];
            }
            if (t > 0) add_tile(tdV, acc_v);         // dV(t - 1): complete, as S^T(t) is
            tmem_st32(tS + t_lane + c0, s);          // P^T hi over S^T
            tmem_st32(tPlo + t_lane + c0, lo);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(P_READY));
            if (!mbar_wait_warp_ool(bar(DP_FULL), (uint32_t)(t & 1), g.err, 143)) { ok = false; break; }
            tc_fence_after();
            tmem_ld32(tdP + t_lane + c0, s);
            tmem_ld32(tdSlo + t_lane + c0, lo);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float4 d4 = Ds[i];
                const float dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int k = 4 * i + e;
                    const float ds = p[k] * ((__uint_as_float(s[k]) + __uint_as_float(lo[k])) - dd[e]);
                    split_tf32_int(ds, s[k], lo[k]);
                }
            }
            if (t > 0) add_tile(tdK, acc_k);         // dK(t - 1): complete, as dP^T(t) is
            tmem_st32(tdP + t_lane + c0, s);         // dS^T hi over dP^T
            tmem_st32(tdSlo + t_lane + c0, lo);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(DS_READY));
            if (t + 1 < n_t) publish_stat(t + 1, next_stat);
        }
        if (ok && n_t > 0) {
            ok = mbar_wait_warp_ool(bar(ACC_FULL), 0, g.err, 144);
            if (ok) {   // warp-uniform: the tensor-memory loads need the whole warp
                tc_fence_after();
                add_tile(tdV, acc_v);
                add_tile(tdK, acc_k);
            }
        }
        if (ok) {
            const int wrow0 = j0 + lane_group * 32, nvalid = max(0, min(32, g.T - wrow0));
            // the streamed-tile buffers are idle by now: each warp stages its rows in a slice of them
            float* tile = reinterpret_cast<float*>(smem_ptr(qk_s) + (uint32_t)(warp - 2) * kRowTileBytes);
#pragma unroll
            for (int i = 0; i < 32; ++i) acc_k[i] *= scale;
#pragma unroll
            for (int part = 1; part < 3; ++part) {
                const int64_t off = (int64_t)(row_base + wrow0) * gs + (int64_t)part * g.C + h * HD + c0;
                warp_rows_store(part == 1 ? acc_k : acc_v, tile, lane, nvalid, g.dqkv ? g.dqkv + off : nullptr,
                                g.dqkv_hi ? g.dqkv_hi + off : nullptr, g.dqkv_hi ? g.dqkv_lo + off : nullptr, gs, nullptr);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) free_tmem(tmem);
}

// --------------------------------------------------------------------------------------------- backward, dQ
//
// One CTA owns 128 queries and walks the 64-key tiles they read; it also forms D = rowsum(dO o O), which the dkv
// kernel reads.
//     S = Q' K^T | dP = dO V^T | dS = P o (dP - D) (1 - tanh^2) | dQ_tile = dS K
//   warp 0 TMA; warps 1, 10, 11 issue S, dP, dQ; warps 2-5 / 6-9 the element-wise pass on alternate tiles;
//   warps 12-15 add every dQ tile to registers (64 columns of a row per thread) and write the result.
//   tensor memory: Q' hi|lo 0-127, dQ tile 128-255, buffer b at 256 + 128b: S -> dS_hi, dP -> dS_lo
// The dQ tile is 128 wide: the column groups [K_hi g0 | K_lo g0 | K_hi g1 | K_lo g1] (g = 32 head columns) as
// one operand of dS_hi, and dS_lo K_hi 32 columns further, on the second and third group; head columns
// 0-31 are the sum of groups 0 and 1, 32-63 that of 2 and 3.
constexpr int kDqThreads = 512, kWarpMma3 = 11, kWarpAdd = 12;
constexpr uint32_t kDqSmem = 1024u + kResBytes + 5u * kTile + 256u + 512u;
static_assert(kDqSmem <= 232448u, "shared memory");

// rowsum(dO o O) over one head for the warp's 32 rows; lane r returns row r's.
__device__ __forceinline__ float rows_dot(const float* o, const float* do_hi, const float* do_lo, long long stride, int nvalid, int lane) {
    const int sub = lane >> 3, cq = lane & 7;
    float acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        acc[i] = 0.f;
        const long long row = (long long)max(0, min(sub + 4 * i, nvalid - 1)) * stride + 4 * cq;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const float4 x = ld4(o + row + half * 32, 0);
            const float4 y = add4(ld4(do_hi + row + half * 32, 0), ld4(do_lo + row + half * 32, 0));
            acc[i] += (x.x * y.x + x.y * y.y) + (x.z * y.z + x.w * y.w);
        }
    }
    float d = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float v = acc[i];
        v += __shfl_xor_sync(0xffffffffu, v, 1);
        v += __shfl_xor_sync(0xffffffffu, v, 2);
        v += __shfl_xor_sync(0xffffffffu, v, 4);
        v = __shfl_sync(0xffffffffu, v, 8 * (lane & 3));     // row sub + 4 i lives in the lanes of slice `sub`
        if ((lane >> 2) == i) d = v;                          // lane r wants row r = (r & 3) + 4 (r >> 2)
    }
    return d;
}

template <bool CAP, bool SLOPE>
__global__ void __launch_bounds__(kDqThreads, 1)
attn_mod_dq_kernel(const __grid_constant__ CUtensorMap tmKk, const __grid_constant__ CUtensorMap tmKm,
                   const __grid_constant__ CUtensorMap tmVk, const __grid_constant__ CUtensorMap tmDOres, const ModTcArgs args) {
    const AttnModArgs& g = args.a;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t do_s = base;
    auto kk_s = [&](int st) { return base + kResBytes + (uint32_t)st * 2u * kTile; };
    auto vk_s = [&](int st) { return kk_s(st) + kTile; };
    const uint32_t km_s = base + kResBytes + 4u * kTile;
    const uint32_t bars = base + kResBytes + 5u * kTile;
    // the S and the dP issuing threads both commit to KEMPTY and SDP
    enum { DO_FULL = 0, KFULL0, KFULL1, KEMPTY0, KEMPTY1, MFULL, MEMPTY, SDP0, SDP1, DONE0, DONE1, DQ_FULL, DS0, DS1, Q_READY, DQ_FREE, N_BARS };
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    const uint32_t tmem_slot = bars + 8u * N_BARS;
    auto smem_ptr = [&](uint32_t addr) { return smem_raw + (addr - smem_u32(smem_raw)); };

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int bh, yb;
    grouped_block(args.head_group, bh, yb);
    const int qt = (int)gridDim.y - 1 - yb;
    const int b = bh / g.H, h = bh % g.H, q0 = qt * BR;
    const int row_base = b * g.T;

    if (threadIdx.x == 0) {
        for (int i = 0; i < N_BARS; ++i)
            mbar_init(bar(i), (i == KEMPTY0 || i == KEMPTY1 || i == SDP0 || i == SDP1) ? 2 : i >= DS0 ? 4 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) alloc_tmem(tmem_slot);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem_ptr(tmem_slot));
    pdl_wait();      // set-up done; global memory is touched from here on
    pdl_trigger();
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *g.err = 0;
    const uint32_t tQ_hi = tmem, tQ_lo = tmem + 64, tdQ = tmem + 128;
    auto tbuf = [&](int bb) { return tmem + 256u + 128u * (uint32_t)bb; };
    const int2 range = block_range(g.spans.kblock, b, g.T, q0, BR, false);
    const int kt0 = range.x / BT64, n_t = range.x < range.y ? (range.y - 1) / BT64 + 1 - kt0 : 0;

    if (warp == 0) {
        if (lane == 0 && n_t > 0) {
            mbar_expect_tx(bar(DO_FULL), kResBytes);
            for (int kb = 0; kb < 2; ++kb)
                tma_load_3d(do_s + kb * (kResBytes / 2), &tmDOres, bar(DO_FULL), h * HD + kb * 32, row_base + q0, 0);
            auto load_kmajor = [&](int t) -> bool {
                const int st = t & 1, k0 = row_base + (kt0 + t) * BT64;
                if (!mbar_wait_ool(bar(KEMPTY0 + st), ((t >> 1) & 1u) ^ 1u, g.err, 151)) return false;
                mbar_expect_tx(bar(KFULL0 + st), 2u * kTile);
                for (int kb = 0; kb < 2; ++kb) {
                    tma_load_3d(kk_s(st) + kb * (kTile / 2), &tmKk, bar(KFULL0 + st), g.C + h * HD + kb * 32, k0, 0);
                    tma_load_3d(vk_s(st) + kb * (kTile / 2), &tmVk, bar(KFULL0 + st), 2 * g.C + h * HD + kb * 32, k0, 0);
                }
                return true;
            };
            // the K-major tiles of t + 1 go out before the wait for the single MN-major buffer
            bool ok = load_kmajor(0);
            for (int t = 0; t < n_t && ok; ++t) {
                if (t + 1 < n_t) ok = load_kmajor(t + 1);
                // the MN-major buffer first stages the query rows
                if (ok && t == 0) ok = mbar_wait_ool(bar(Q_READY), 0, g.err, 152);
                if (ok) ok = mbar_wait_ool(bar(MEMPTY), (t & 1u) ^ 1u, g.err, 153);
                if (!ok) break;
                mbar_expect_tx(bar(MFULL), kTile);
                for (int grp = 0; grp < 2; ++grp)
                    tma_load_3d(km_s + grp * (kTile / 2), &tmKm, bar(MFULL), g.C + h * HD + grp * 32, row_base + (kt0 + t) * BT64, 0);
            }
            if (!ok) settle();
        }
    } else if (warp == 1 || warp == kWarpMma2) {
        if (lane == 0 && n_t > 0) {
            constexpr uint32_t idesc = make_idesc_tf32(BR, BT64, false, false);
            const bool s_product = warp == 1;
            bool ok = s_product ? mbar_wait_ool(bar(Q_READY), 0, g.err, 154) : mbar_wait_ool(bar(DO_FULL), 0, g.err, 155);
            const DescBase dod = kmaj_base(do_s);
            for (int t = 0; t < n_t && ok; ++t) {
                const int st = t & 1;
                if (!mbar_wait_ool(bar(KFULL0 + st), (t >> 1) & 1u, g.err, 156)) { ok = false; break; }
                // buffer t & 1: the dQ product of tile t - 2 has read it
                if (t >= 2 && !mbar_wait_ool(bar(DONE0 + st), ((t - 2) >> 1) & 1u, g.err, 157)) { ok = false; break; }
                tc_fence_after();
                if (s_product) {
                    const uint32_t d = tbuf(st);
                    const DescBase kd = kmaj_base(kk_s(st));
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) {
                        umma_tf32_ts(d, tQ_lo + ks * 8, kd.at(kmaj_off(BT64, ks, false)), idesc, ks > 0 ? 1u : 0u);
                        umma_tf32_ts(d, tQ_hi + ks * 8, kd.at(kmaj_off(BT64, ks, true)), idesc, 1u);
                    }
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) umma_tf32_ts(d, tQ_hi + ks * 8, kd.at(kmaj_off(BT64, ks, false)), idesc, 1u);
                } else {
                    const uint32_t d = tbuf(st) + 64u;
                    const DescBase vd = kmaj_base(vk_s(st));
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) {
                        umma_tf32(d, dod.at(kmaj_off(BR, ks, true)), vd.at(kmaj_off(BT64, ks, false)), idesc, ks > 0 ? 1u : 0u);
                        umma_tf32(d, dod.at(kmaj_off(BR, ks, false)), vd.at(kmaj_off(BT64, ks, true)), idesc, 1u);
                    }
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        umma_tf32(d, dod.at(kmaj_off(BR, ks, false)), vd.at(kmaj_off(BT64, ks, false)), idesc, 1u);
                }
                umma_commit(bar(KEMPTY0 + st));
                umma_commit(bar(SDP0 + st));
            }
        }
    } else if (warp == kWarpMma3) {
        if (lane == 0 && n_t > 0) {
            constexpr uint32_t idesc = make_idesc_tf32(BR, HD, false, true), idesc2 = make_idesc_tf32(BR, 2 * HD, false, true);
            bool ok = true;
            const DescBase kmd = mn_base(km_s), kmd4 = make_desc_base(km_s, BT64 * 128u, 512u, 1u);
            for (int t = 0; t < n_t && ok; ++t) {
                const int bb = t & 1;
                if (!mbar_wait_ool(bar(DS0 + bb), (t >> 1) & 1u, g.err, 158)) { ok = false; break; }
                if (!mbar_wait_ool(bar(MFULL), t & 1u, g.err, 159)) { ok = false; break; }
                if (t > 0 && !mbar_wait_ool(bar(DQ_FREE), (t - 1) & 1u, g.err, 160)) { ok = false; break; }
                tc_fence_after();
                const uint32_t s_hi = tbuf(bb), s_lo = tbuf(bb) + 64u;
                // one large term, to set all columns, then the small ones, then the other large ones
                umma_tf32_ts(tdQ, s_hi, kmd4.at(mn_off(0, false)), idesc2, 0u);
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) umma_tf32_ts(tdQ + 32u, s_lo + ks * 8, kmd.at(mn_off(ks, false)), idesc, 1u);
#pragma unroll
                for (int ks = 1; ks < 8; ++ks) umma_tf32_ts(tdQ, s_hi + ks * 8, kmd4.at(mn_off(ks, false)), idesc2, 1u);
                umma_commit(bar(MEMPTY));
                umma_commit(bar(DONE0 + bb));
                umma_commit(bar(DQ_FULL));
            }
        }
    } else if (warp >= kWarpAdd) {
        const int lane_group = warp & 3;
        const uint32_t t_row = tdQ + ((uint32_t)(lane_group * 32) << 16);
        float acc[2][32];
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[0][i] = acc[1][i] = 0.f;
        bool ok = true;
        for (int t = 0; t < n_t && ok; ++t) {
            if (!mbar_wait_warp_ool(bar(DQ_FULL), t & 1u, g.err, 161)) { ok = false; break; }
            tc_fence_after();
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t r[32], r2[32];
                tmem_ld32(t_row + half * 64, r);
                tmem_ld32(t_row + half * 64 + 32, r2);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i) acc[half][i] += __uint_as_float(r[i]) + __uint_as_float(r2[i]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(DQ_FREE));
        }
        if (ok) {
            const float scale = 1.0f / sqrtf((float)HD);
            const int wrow0 = q0 + lane_group * 32, nvalid = max(0, min(32, g.T - wrow0));
            const int64_t gs = 3 * (int64_t)g.C, off = (int64_t)(row_base + wrow0) * gs + h * HD;
            // every product has completed: the K-major tiles are idle
            float* tile = reinterpret_cast<float*>(smem_ptr(kk_s(0)) + (uint32_t)lane_group * kRowTileBytes);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int i = 0; i < 32; ++i) acc[half][i] *= scale;
                warp_rows_store(acc[half], tile, lane, nvalid, g.dqkv ? g.dqkv + off + half * 32 : nullptr,
                                g.dqkv_hi ? g.dqkv_hi + off + half * 32 : nullptr, g.dqkv_hi ? g.dqkv_lo + off + half * 32 : nullptr,
                                gs, nullptr);
            }
        }
    } else {
        const int wg = (warp - 2) >> 2, lane_group = warp & 3;
        const int row = q0 + lane_group * 32 + lane;
        const uint32_t t_lane = ((uint32_t)(lane_group * 32) << 16);
        const Score sc = make_score<CAP, SLOPE>(1.0f / sqrtf((float)HD), g.cap, g.slopes, h);
        const int64_t gs = 3 * (int64_t)g.C;
        const int64_t lb = ((int64_t)b * g.H + h) * g.T;
        const int wrow0 = min(q0 + lane_group * 32, g.T - 1), wvalid = max(1, min(32, g.T - wrow0));
        if (wg == 0 && n_t > 0) {
            const int64_t off = (int64_t)(row_base + wrow0) * gs + h * HD;
            float* tile = reinterpret_cast<float*>(smem_ptr(km_s) + (uint32_t)lane_group * kRowTileBytes);
            rows_to_tmem(g.qkv + off, g.qkv_lo + off, gs, wvalid, sc.unit, tQ_hi + t_lane, tQ_lo + t_lane, tile, lane);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the tile is next written by TMA
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(Q_READY));
        }
        float* dsm = reinterpret_cast<float*>(smem_ptr(bars + 256u));
        if (wg == 1) {
            const long long off = (long long)(row_base + wrow0) * g.C + h * HD;
            const float d = rows_dot(g.o + off, g.d_o + off, g.d_o_lo + off, g.C, wvalid, lane);
            dsm[lane_group * 32 + lane] = d;
            if (row < g.T) g.dvec[lb + row] = d;
        }
        asm volatile("bar.sync 2, 256;" ::: "memory");    // the eight element-wise warps, exactly once
        const float L = g.lse[lb + min(row, g.T - 1)] * kLog2e, D = dsm[lane_group * 32 + lane];
        const int2 span = row_range(g.spans.k, b, g.T, row, false);
        bool ok = true;
        const uint32_t tb = tbuf(wg) + t_lane;
        for (int t = wg; t < n_t && ok; t += 2) {
            const int k0 = (kt0 + t) * BT64;
            if (!mbar_wait_warp_ool(bar(SDP0 + wg), (t >> 1) & 1u, g.err, 162)) { ok = false; break; }
            tc_fence_after();
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int kh = k0 + half * 32;
                float x[32], f[32];
                uint32_t s[32], dp[32];
                tmem_ld32(tb + half * 32u, s);
                tmem_ld32(tb + 64u + half * 32u, dp);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(s[i]);
                score_tile_grad<CAP, SLOPE, 32>(x, f, sc, row - kh);
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] = ex2_approx(x[i] - L);
                if (kh < span.x || kh + 32 > span.y) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (kh + i < span.x || kh + i >= span.y) x[i] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    float ds = x[i] * (__uint_as_float(dp[i]) - D);
                    if (CAP) ds *= f[i];
                    split_tf32_int(ds, s[i], dp[i]);
                }
                tmem_st32(tb + half * 32u, s);                      // dS hi over S
                tmem_st32(tb + 64u + half * 32u, dp);               // dS lo over dP
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(DS0 + wg));
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) free_tmem(tmem);
}

}  // namespace

bool attention_mod_tc_supports(const AttnModArgs& g) { return g.C / g.H == HD && g.qkv_lo; }

cudaError_t launch_attention_mod_fwd_tc(const AttnModArgs& g, cudaStream_t s) {
    const int64_t rows = (int64_t)g.B * g.T, cols = 3 * (int64_t)g.C;
    CUtensorMap q, k, v;
    if (!plane_map(&q, g.qkv, cols, rows, BR, false) || !plane_map(&k, g.qkv, cols, rows, BT64, false) ||
        !plane_map(&v, g.qkv, cols, rows, BT64, true))
        return cudaErrorInvalidValue;
    const dim3 grid(g.B * g.H, (g.T + BR - 1) / BR);
    const ModTcArgs a{g, attn_head_group((int)grid.x, (int)grid.y)};
    BT_FOR_MOD(g, {
        cudaError_t e = cudaFuncSetAttribute(attn_mod_fwd_kernel<kCap, kSlope>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFwdSmem);
        if (e != cudaSuccess) return e;
        BT_KERNEL_LAUNCH((attn_mod_fwd_kernel<kCap, kSlope>), grid, kFwdThreads, kFwdSmem, s, q, k, v, a);
    });
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

cudaError_t launch_attention_mod_bwd_tc(const AttnModArgs& g, cudaStream_t s) {
    const int64_t rows = (int64_t)g.B * g.T, cols = 3 * (int64_t)g.C;
    CUtensorMap qkv_k, qkv_m, qkv_res, do_k, do_m, do_res;
    if (!plane_map(&qkv_k, g.qkv, cols, rows, BT64, false) || !plane_map(&qkv_m, g.qkv, cols, rows, BT64, true) ||
        !plane_map(&qkv_res, g.qkv, cols, rows, BR, false) || !plane_map(&do_k, g.d_o, g.C, rows, BT64, false) ||
        !plane_map(&do_m, g.d_o, g.C, rows, BT64, true) || !plane_map(&do_res, g.d_o, g.C, rows, BR, false))
        return cudaErrorInvalidValue;
    const dim3 grid(g.B * g.H, (g.T + BR - 1) / BR);
    const ModTcArgs a{g, attn_head_group((int)grid.x, (int)grid.y)};
    BT_FOR_MOD(g, {
        cudaError_t e = cudaFuncSetAttribute(attn_mod_dq_kernel<kCap, kSlope>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kDqSmem);
        if (e == cudaSuccess)
            e = cudaFuncSetAttribute(attn_mod_dkv_kernel<kCap, kSlope>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kDkvSmem);
        if (e != cudaSuccess) return e;
        // the dq kernel goes first: it also forms D
        BT_KERNEL_LAUNCH((attn_mod_dq_kernel<kCap, kSlope>), grid, kDqThreads, kDqSmem, s, qkv_k, qkv_m, qkv_k, do_res, a);
        BT_KERNEL_LAUNCH((attn_mod_dkv_kernel<kCap, kSlope>), grid, kDkvThreads, kDkvSmem, s, qkv_k, qkv_m, do_k, do_m, qkv_res, a);
    });
    BT_COUNT_LAUNCH();
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

}  // namespace bt
