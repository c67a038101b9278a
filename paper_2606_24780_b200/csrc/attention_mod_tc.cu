// Attention with modified scores on the 5th-generation tensor cores, head_dim 64, 32 and 16, 3xTF32.
//
// As in the plain causal kernels an item of work is 128 rows of one head, one row per tensor-memory lane, against 64-row
// tiles of the other side, with bounded mbarrier waits.  Unlike there the kernels are persistent: every role walks the
// items at its own pace, and what each does is written at each kernel.
//
//   Tiles      An item walks the tiles between the ends of its rows' ranges (SpanView): with packed documents
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
//   Launches   No programmatic trigger here: the next kernel's CTAs would take SMs from items that have not begun (3 % of the
//              gradients at 8,192 positions), and its set-up is short beside these kernels.
#include "attention_mod.cuh"

namespace bt {

using namespace tc;
using namespace mod;

namespace {

// HD: columns of a head as the tiles hold them, 64 or 32; a head of 16 is a tile of 32 whose other half the copies fill with zeros
constexpr int BR = 128, BT64 = 64;
template <int HD> constexpr uint32_t kRes = HD / 32 * 2u * BR * 128u;         // 128 own rows: k-blocks of 32 columns x (hi, lo) x 128 rows x 128 B
template <int HD> constexpr uint32_t kTileBytes = HD / 32 * 2u * BT64 * 128u; // one streamed 64-row tile (hi, lo) in one layout
//  MN-major 64-row tile: column groups of [hi | lo][64 rows][128 B]; a k-step is 8 rows
__device__ __forceinline__ constexpr uint32_t mn_off(int ks, bool lo) { return (lo ? BT64 * 128u : 0u) + (uint32_t)ks * 1024u; }
__device__ __forceinline__ DescBase mn_base(uint32_t tile) { return make_desc_base(tile, 2u * BT64 * 128u, 512u, 1u); }

struct ModTcArgs {
    AttnModArgs a;
    int d;                   // the heads' own columns
    int head_group;          // heads per group of the CTA order (grouped_block)
};

__device__ __forceinline__ void alloc_tmem(uint32_t slot) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void free_tmem(uint32_t tmem) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}
// Box of head_map: columns from c0 on of one head (of q, k and v heads counted through), rows from row on, both planes.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* tm, uint32_t bar, int c0, int head, int row) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"((unsigned long long)tm), "r"(c0), "r"(head), "r"(row), "r"(0), "r"(bar) : "memory");
}
// Brings a box into L2: the operands that an item begins with are 200 to 300 KB, and all SMs start theirs at about the same time.
__device__ __forceinline__ void prefetch_box(const CUtensorMap* tm, int c0, int head, int row) {
    asm volatile("cp.async.bulk.prefetch.tensor.4d.L2.global.tile [%0, {%1, %2, %3, %4}];"
                 ::"l"((unsigned long long)tm), "r"(c0), "r"(head), "r"(row), "r"(0) : "memory");
}
// A role whose wait ran out lets copies in flight land before the CTA exits.
__device__ __forceinline__ void settle() {
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
}

// ------------------------------------------------------------------------------------------ forward
//
// Persistent: the roles run over the work items (128 queries of one head) one after the other, each at its own pace, so
// an item's loads, first products, last sums and stores overlap its neighbours'.
//   warp 0      TMA producer and scheduler: the next item and its range of tiles; Q once per item, K and V tiles through one
//               ring of four slots, K one tile ahead of V
//   warp 1      S = Q K^T, the small terms first
//   warps 2, 3  O_tile = P V on alternate tiles, P from tensor memory, from zero in every tile
//   warps 4-15  three softmax warpgroups on tiles in turn, thread = row.  Every tile is normalised by its own row
//               maximum, so they carry nothing from tile to tile: a pass over the scores for the maximum (whole ones: their
//               small terms reach hundreds at 1e5), then P = exp2(z - r)
//   warps 16-19 add up: O = O 2^(m - m') + O_tile 2^(r - m'), l likewise; the row's output and lse
//   tensor memory  buffer i at 128 i: S -> P_hi, P_lo; O_tile at 384 and 448
// Two tiles in the softmax at a time are not enough to hide its latency; short rolled passes over the columns keep
// the code in the instruction cache (32 columns unrolled cost a third more time than 16).
// 8 packed sequences of 1,024, 12 heads, distance bias: 69 us, tensor pipe 40 % busy; the products of a tile are about 1,900
// clocks, the element-wise warps, at 1.7 to 2.1 instructions a clock of all four schedulers, need 2,700 with a cap.  S as two halves,
// [K_hi | K_lo] as one operand, is 250 clocks less of products, but both passes of the element-wise warps have to add them:
// 448 us in place of 437 at 8,192 positions, causal.
constexpr int kFwdThreads = 640, kSlots = 4, kSoft = 3, CH = 16;
constexpr int kRegsIssue = 56, kRegsSoft = 88, kRegsAdd = 160;
static_assert(kRegsIssue + kSoft * kRegsSoft + kRegsAdd <= 480, "registers: 640 threads get 96 each at launch");
constexpr uint32_t kStatBytes = 8u * 2u * BR * 4u;            // (r, sum) of the last eight tiles
template <int HD> constexpr uint32_t kFwdSmem = 1024u + kRes<HD> + kSlots * kTileBytes<HD> + 512u + kStatBytes;
static_assert(kFwdSmem<64> <= 232448u, "shared memory");
// Place of K(t) and V(t) among an item's 2n tile loads: K0 K1 V0 K2 V1 ... K(n-1) V(n-2) V(n-1).
__device__ __forceinline__ int pos_k(int t) { return t == 0 ? 0 : 2 * t - 1; }
__device__ __forceinline__ int pos_v(int t, int n) { return min(2 * t + 2, 2 * n - 1); }

template <int HD, bool CAP, bool SLOPE>
__global__ void __launch_bounds__(kFwdThreads, 1)
attn_mod_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                    const __grid_constant__ CUtensorMap tmV, const ModTcArgs args) {
    const AttnModArgs& g = args.a;
    constexpr uint32_t kResBytes = kRes<HD>, kTile = kTileBytes<HD>;
    constexpr int KB = HD / 32, KS = HD / 8;             // k-blocks, and k-steps of a product over the head's columns
    const int d = HD == 64 ? HD : args.d;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_s = base, ring_s = q_s + kResBytes, bars = ring_s + kSlots * kTile;
    enum { Q_FULL = 0, Q_EMPTY, SLOT_FULL, SLOT_EMPTY = SLOT_FULL + kSlots, S_FULL = SLOT_EMPTY + kSlots, P_DONE = S_FULL + kSoft,
           P_FULL = P_DONE + kSoft, O_FULL = P_FULL + kSoft, O_FREE = O_FULL + 2, INFO_FULL = O_FREE + 2, INFO_EMPTY = INFO_FULL + 2,
           NEXT = INFO_EMPTY + 2, N_BARS };
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    constexpr uint32_t kInfo = (8u * N_BARS + 15u) & ~15u;            // two Items, the scheduler's answer, the TMEM address
    static_assert(kInfo + 2 * sizeof(Item) + 32 <= 512, "barrier region");
    auto smem_ptr = [&](uint32_t addr) { return smem_raw + (addr - smem_u32(smem_raw)); };
    volatile Item* info = reinterpret_cast<volatile Item*>(smem_ptr(bars + kInfo));
    const uint32_t answer = bars + kInfo + 2u * (uint32_t)sizeof(Item), tmem_slot = answer + 16u;
    float* tile_stat = reinterpret_cast<float*>(smem_ptr(bars + 512u));

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < N_BARS; ++i)
            mbar_init(bar(i), (i >= O_FULL && i < O_FREE) ? 2 : (i >= O_FREE && i < INFO_FULL) || (i >= P_FULL && i < O_FULL) ? 4
                              : i >= INFO_EMPTY && i < NEXT ? 3 + 4 * kSoft + 4 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) alloc_tmem(tmem_slot);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem_ptr(tmem_slot));
    pdl_wait();      // set-up done; global memory is touched from here on
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *g.err = 0;

    auto next = [&](int i, Item& it, bool whole_warp) -> bool {     // every role walks the same items
        return get_item(info, bar(INFO_FULL), bar(INFO_EMPTY), i, it, g.err, whole_warp);
    };

    if (warp < 4) {
        set_regs_down<kRegsIssue>();
        if (warp == 0 && lane == 0) {
            uint32_t c = 0, qi = 0;                     // loads and non-empty items so far
            Item it = make_item(g, args.head_group, (int)blockIdx.x, (int)blockIdx.y, false, BR, BT64);
            bool ok = put_item(info, bar(INFO_FULL), bar(INFO_EMPTY), 0, it, g.err);
            for (int i = 0; ok && it.n >= 0; ++i) {
                // The next item is asked for five loads before this one's last and looked up before the last, so that its
                // loads follow at once (a boundary cost 6,000 clocks when it was asked for only then; asked for at the
                // start, the last items of long walks are spread worse: 10 % at 8,192 positions).
                const int last = 2 * it.n - 1;
                if (it.n == 0) ask_next(answer, bar(NEXT));
                Item follows{0, 0, 0, -1};
                auto look_up = [&]() -> bool {
                    if (!mbar_wait(bar(NEXT), (uint32_t)i & 1u, g.err, 120)) return false;
                    int x, y;
                    if (next_item(answer, x, y)) follows = make_item(g, args.head_group, x, y, false, BR, BT64);
                    if (follows.n > 0) {
                        const int h = follows.bh % g.H, row0 = (follows.bh / g.H) * g.T;
                        for (int kb = 0; kb < KB; ++kb) {
                            prefetch_box(&tmQ, kb * 32, h, row0 + follows.blk * BR);
                            prefetch_box(&tmK, kb * 32, g.H + h, row0 + follows.t0 * BT64);
                            prefetch_box(&tmV, kb * 32, 2 * g.H + h, row0 + follows.t0 * BT64);
                        }
                    }
                    return put_item(info, bar(INFO_FULL), bar(INFO_EMPTY), i + 1, follows, g.err);
                };
                if (it.n == 0) ok = look_up();
                const int h = it.bh % g.H, row0 = (it.bh / g.H) * g.T;
                for (int p = 0; p < 2 * it.n && ok; ++p, ++c) {
                    const bool is_k = p == 0 || ((p & 1) && p < 2 * it.n - 1);
                    const int t = p == 0 ? 0 : p == 2 * it.n - 1 ? it.n - 1 : is_k ? (p + 1) >> 1 : (p - 2) >> 1;
                    if (p == max(0, last - 8)) ask_next(answer, bar(NEXT));
                    if (p == max(1, last - 4)) ok = look_up();
                    if (!ok) break;
                    const uint32_t slot = c % kSlots;
                    ok = mbar_wait(bar(SLOT_EMPTY + slot), ((c / kSlots) & 1u) ^ 1u, g.err, 111);
                    if (!ok) break;
                    mbar_expect_tx(bar(SLOT_FULL + slot), kTile);
                    for (int kb = 0; kb < KB; ++kb)
                        load_box(ring_s + slot * kTile + kb * (kTile / KB), is_k ? &tmK : &tmV, bar(SLOT_FULL + slot),
                                    kb * 32, (is_k ? g.H : 2 * g.H) + h, row0 + (it.t0 + t) * BT64);
                    if (p == 0) {                       // behind the first K: the previous item's last S has to be done with Q
                        ok = mbar_wait(bar(Q_EMPTY), (qi & 1u) ^ 1u, g.err, 112);
                        if (!ok) break;
                        mbar_expect_tx(bar(Q_FULL), kResBytes);
                        for (int kb = 0; kb < KB; ++kb)
                            load_box(q_s + kb * (kResBytes / KB), &tmQ, bar(Q_FULL), kb * 32, h, row0 + it.blk * BR);
                    }
                }
                if (it.n > 0) ++qi;
                it = follows;
            }
            if (!ok) settle();
        } else if (warp == 1) {
            constexpr uint32_t idesc = make_idesc_tf32(BR, BT64, false, false);
            const DescBase qd = kmaj_base(q_s);
            uint32_t c = 0, qi = 0, gt = 0;             // loads, non-empty items, tiles before this item
            Item it;
            bool ok = true;
            for (int i = 0; ok && (ok = next(i, it, true)) && it.n >= 0; ++i) {
                if (it.n == 0) continue;
                ok = mbar_wait_warp(bar(Q_FULL), qi & 1u, g.err, 113);
                for (int t = 0; t < it.n && ok; ++t, ++gt) {
                    const uint32_t ck = c + (uint32_t)pos_k(t), slot = ck % kSlots, buf = gt % kSoft;
                    // In this order: K and V share the slots, and a wait on a slot's phase is only sound once the load before it
                    // in the slot has landed.  That was K(t - 2), waited for here, or, next to an item's edge, the V of a
                    // tile at least three back (P_DONE) or of one whose slot K(0) took over (Q_FULL).
                    if (gt >= kSoft && !mbar_wait_warp(bar(P_DONE + buf), (gt / kSoft - 1u) & 1u, g.err, 115)) { ok = false; break; }
                    if (!mbar_wait_warp(bar(SLOT_FULL + slot), (ck / kSlots) & 1u, g.err, 114)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t tS = tmem + buf * 128u;
                    const DescBase kd = kmaj_base(ring_s + slot * kTile);
                    if (elect_one()) {
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) {
                            umma_tf32(tS, qd.at(kmaj_off(BR, ks, true)), kd.at(kmaj_off(BT64, ks, false)), idesc, ks > 0 ? 1u : 0u);
                            umma_tf32(tS, qd.at(kmaj_off(BR, ks, false)), kd.at(kmaj_off(BT64, ks, true)), idesc, 1u);
                        }
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) umma_tf32(tS, qd.at(kmaj_off(BR, ks, false)), kd.at(kmaj_off(BT64, ks, false)), idesc, 1u);
                        umma_commit(bar(SLOT_EMPTY + slot));
                        umma_commit(bar(S_FULL + buf));
                        if (t == it.n - 1) umma_commit(bar(Q_EMPTY));
                    }
                    __syncwarp();
                }
                c += 2u * (uint32_t)it.n;
                ++qi;
            }
        } else if (warp >= 2) {
            // two issuing warps, tiles of their own parity; each O_tile buffer belongs to one of them
            constexpr uint32_t idesc = make_idesc_tf32(BR, HD, false, true);
            const uint32_t ob = (uint32_t)warp - 2u, tO = tmem + 384u + 64u * ob;
            uint32_t c = 0, gt = 0;
            Item it;
            bool ok = true;
            for (int i = 0; ok && (ok = next(i, it, true)) && it.n >= 0; ++i) {
                for (int t = (int)((gt ^ ob) & 1u); t < it.n && ok; t += 2) {
                    const uint32_t ga = gt + (uint32_t)t, cv = c + (uint32_t)pos_v(t, it.n), slot = cv % kSlots, buf = ga % kSoft;
                    // In this order: O_FREE says that the tile two back has been added, so that the buffer's P of three tiles
                    // back, which the other thread waited for, is past; P_FULL that every K up to this tile's has landed; the load
                    // before V(t) in its slot was one of those or a V of this thread's.
                    if (ga >= 2 && !mbar_wait_warp(bar(O_FREE + ob), ((ga >> 1) - 1u) & 1u, g.err, 118)) { ok = false; break; }
                    if (!mbar_wait_warp(bar(P_FULL + buf), (ga / kSoft) & 1u, g.err, 116)) { ok = false; break; }
                    if (!mbar_wait_warp(bar(SLOT_FULL + slot), (cv / kSlots) & 1u, g.err, 117)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t p_hi = tmem + buf * 128u, p_lo = p_hi + 64u;
                    const DescBase vd = mn_base(ring_s + slot * kTile);
                    if (elect_one()) {
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks) {
                            umma_tf32_ts(tO, p_lo + ks * 8u, vd.at(mn_off(ks, false)), idesc, ks > 0 ? 1u : 0u);
                            umma_tf32_ts(tO, p_hi + ks * 8u, vd.at(mn_off(ks, true)), idesc, 1u);
                        }
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks) umma_tf32_ts(tO, p_hi + ks * 8u, vd.at(mn_off(ks, false)), idesc, 1u);
                        umma_commit(bar(SLOT_EMPTY + slot));
                        umma_commit(bar(P_DONE + buf));
                        mbar_arrive(bar(O_FULL + ob));      // hands on what P_FULL published: the tile's (r, sum)
                        umma_commit(bar(O_FULL + ob));
                    }
                    __syncwarp();
                }
                c += 2u * (uint32_t)it.n;
                gt += (uint32_t)it.n;
            }
        }
    } else if (warp < 4 + 4 * kSoft) {
        set_regs_down<kRegsSoft>();
        const int wg = (warp - 4) >> 2, lane_group = warp & 3, rloc = lane_group * 32 + lane;
        const uint32_t t_s = tmem + ((uint32_t)(lane_group * 32) << 16) + (uint32_t)wg * 128u;
        uint32_t gt = 0, use = 0;
        Item it;
        bool ok = true;
        for (int i = 0; ok && (ok = next(i, it, true)) && it.n >= 0; ++i) {
            const int b = it.bh / g.H, h = it.bh % g.H, row = it.blk * BR + rloc;
            const Score sc = make_score<CAP, SLOPE>(1.0f / sqrtf((float)d), g.cap, g.slopes, h);
            const int2 span = row_range(g.spans.k, b, g.T, row, false);
            for (int t = (wg + kSoft - (int)(gt % kSoft)) % kSoft; t < it.n; t += kSoft, ++use) {
                if (!mbar_wait_warp(bar(S_FULL + wg), use & 1u, g.err, 121)) { ok = false; break; }
                tc_fence_after();
                const int key0 = (it.t0 + t) * BT64;
                const bool whole = key0 >= span.x && key0 + BT64 <= span.y;
                auto mask = [&](float (&z)[CH], int k0) {
                    if (!whole) {
                        const uint32_t bits = column_bits<CH>(span, k0);
#pragma unroll
                        for (int k = 0; k < CH; ++k)
                            if (!(bits >> k & 1u)) z[k] = -INFINITY;
                    }
                };
                float top = -INFINITY;
#pragma unroll 1
                for (int c0 = 0; c0 < BT64; c0 += CH) {
                    float z[CH], none[CH];
                    uint32_t r[CH];
                    tmem_ldn(t_s + c0, r);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < CH; ++k) z[k] = __uint_as_float(r[k]);
                    if (SLOPE) score_tile<CAP, SLOPE, false, true, CH>(z, none, sc, row - key0 - c0, 0.f);   // else the maximum is at that of the product
                    mask(z, key0 + c0);
#pragma unroll
                    for (int k = 0; k < CH; ++k) top = fmaxf(top, z[k]);
                }
                const bool none_read = top == -INFINITY;                // every P of this tile is zero
                float ref = 0.f, sum = 0.f;
                if (!none_read) ref = SLOPE ? top : CAP ? sc.to_log2 * tanh_any(top * sc.unit) : top * sc.unit;
                const Reference rf = make_reference(ref, sc.slope2, abs(row - key0) + BT64);
#pragma unroll 1
                for (int c0 = 0; c0 < BT64; c0 += CH) {
                    float z[CH], none[CH];
                    uint32_t hi[CH], lo[CH];
                    tmem_ldn(t_s + c0, hi);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < CH; ++k) z[k] = __uint_as_float(hi[k]);
                    score_tile<CAP, SLOPE, false, true, CH>(z, none, sc, row - key0 - c0, rf.now);
                    less_reference(z, rf);
                    mask(z, key0 + c0);
#pragma unroll
                    for (int k = 0; k < CH; ++k) {
                        const float p = ex2_approx(z[k]);
                        sum += p;
                        split_tf32_int(p, hi[k], lo[k]);
                    }
                    tmem_stn(t_s + c0, hi);                             // P_hi over S, P_lo beside it
                    tmem_stn(t_s + 64u + c0, lo);
                }
                float* stat = tile_stat + ((gt + (uint32_t)t) & 7u) * (2 * BR) + rloc;
                stat[0] = none_read ? -INFINITY : ref;
                stat[BR] = sum;
                __threadfence_block();
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(P_FULL + wg));
            }
            gt += (uint32_t)it.n;
        }
    } else {
        set_regs_up<kRegsAdd>();
        const int lane_group = warp & 3, rloc = lane_group * 32 + lane;
        const uint32_t t_o = tmem + 384u + ((uint32_t)(lane_group * 32) << 16);
        uint32_t gt = 0;
        Item it;
        bool ok = true;
        for (int i = 0; ok && (ok = next(i, it, true)) && it.n >= 0; ++i) {
            float acc[HD], m = -INFINITY, l = 0.f;
#pragma unroll
            for (int k = 0; k < HD; ++k) acc[k] = 0.f;
            for (int t = 0; t < it.n; ++t, ++gt) {
                const uint32_t ob = gt & 1u;
                if (!mbar_wait_warp(bar(O_FULL + ob), (gt >> 1) & 1u, g.err, 122)) { ok = false; break; }
                tc_fence_after();
                uint32_t r[KB][32];
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) tmem_ld32(t_o + 64u * ob + 32u * kb, r[kb]);
                const float* stat = tile_stat + (gt & 7u) * (2 * BR) + rloc;
                const float ref = stat[0], sum = stat[BR];
                tmem_ld_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(O_FREE + ob));           // before the arithmetic: a product waits for this
                const float top = fmaxf(m, ref), use = top == -INFINITY ? 0.f : top;
                const float keep = ex2_approx(m - use), join = ex2_approx(ref - use);
                l = l * keep + sum * join;
                m = top;
#pragma unroll
                for (int k = 0; k < HD; ++k) acc[k] = fmaf(acc[k], keep, __uint_as_float(r[k >> 5][k & 31]) * join);
            }
            const int b = it.bh / g.H, h = it.bh % g.H, row = it.blk * BR + rloc;
            if (ok && row < g.T) {
                const int2 span = l != 0.f ? make_int2(0, 0) : row_range(g.spans.k, b, g.T, row, false);
                const float inv = row_factor(l, span);
                const int64_t at = ((int64_t)b * g.T + row) * g.C + (int64_t)h * d;
#pragma unroll
                for (int q = 0; q < HD; q += 8) {
                    if (q >= d) break;
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = acc[q + e] * inv;
                    store_sector(v, at + q, g.o, g.o_hi, g.o_lo);
                }
                g.lse[((int64_t)b * g.H + h) * g.T + row] = row_lse(m, l, span);
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) free_tmem(tmem);
}

// -------------------------------------------------------------------------------------- backward, dK and dV
//
// Persistent as the forward; an item is 128 keys of one head and the 64-row query tiles that read them.
//     S^T = K' Q^T | dP^T = V dO^T | dV_tile = P^T dO | dK_tile = dS^T Q,  P^T = exp2(z - lse), dS^T = P^T o (dP^T - D) (1 - tanh^2)
//   warp 0      TMA producer and scheduler
//   warp 1      dV(t), S^T(t+1), dV(t+1), ...;   warp 2  dK(t), dP^T(t+1), ...: within a chain the product that overwrites a
//               region follows the one that last read it
//   warps 4-19  four element-wise warpgroups on every tile, thread = key, 16 of the tile's queries each, and 16 columns of
//               dK and of dV each.  dV(t) is complete when S^T(t+1) is (one thread's products complete in order): they
//               read it between that wait and publishing P^T(t+1), which lets dV(t+1) overwrite it; dK likewise
//   tensor memory  K' hi|lo 0-127, dK 128-191, dV 192-255, S^T -> P^T_hi 256-319, small half -> P^T_lo 320-383,
//               dP^T -> dS^T_hi 384-447, small half -> dS^T_lo 448-511
// That is all of it, so a tile's chain S^T -> P^T -> dV has no second buffer to overlap: 4,750 clocks a tile (5,400 with a cap)
// for 3,200 of products.  8 packed sequences of 1,024, 12 heads, cap: 133 us, tensor pipe 42 % busy.
constexpr int kDkvThreads = 640, kRegsIssueDkv = 64, kRegsElemDkv = 104;
static_assert(kRegsIssueDkv + 4 * kRegsElemDkv <= 480, "registers: 640 threads get 96 each at launch");
template <int HD> constexpr uint32_t kDkvSmem = 1024u + kRes<HD> + 4u * kTileBytes<HD> + 512u + 1024u;
static_assert(kDkvSmem<64> <= 232448u, "shared memory");

template <int HD, bool CAP, bool SLOPE>
__global__ void __launch_bounds__(kDkvThreads, 1)
attn_mod_dkv_kernel(const __grid_constant__ CUtensorMap tmQk, const __grid_constant__ CUtensorMap tmQm,
                    const __grid_constant__ CUtensorMap tmDOk, const __grid_constant__ CUtensorMap tmDOm,
                    const __grid_constant__ CUtensorMap tmVres, const ModTcArgs args) {
    const AttnModArgs& g = args.a;
    constexpr uint32_t kResBytes = kRes<HD>, kTile = kTileBytes<HD>;
    constexpr int KB = HD / 32, KS = HD / 8;             // k-blocks, and k-steps of a product over the head's columns
    const int d = HD == 64 ? HD : args.d;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t v_s = base, qk_s = base + kResBytes, dok_s = qk_s + kTile, dom_s = dok_s + kTile, qm_s = dom_s + kTile;
    const uint32_t bars = qm_s + kTile;
    enum { V_FULL = 0, V_EMPTY, QK_FULL, QK_EMPTY, DOK_FULL, DOK_EMPTY, DOM_FULL, DOM_EMPTY, QM_FULL, QM_EMPTY, S_FULL, DP_FULL, ACC_V, ACC_K,
           NEXT, INFO_FULL, INFO_EMPTY = INFO_FULL + 2, P_READY = INFO_EMPTY + 2, DS_READY, K_READY, STAT_READY, N_BARS };
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    constexpr uint32_t kInfo = (8u * N_BARS + 15u) & ~15u;
    static_assert(kInfo + 2 * sizeof(Item) + 32 <= 512, "barrier region");
    auto smem_ptr = [&](uint32_t addr) { return smem_raw + (addr - smem_u32(smem_raw)); };
    volatile Item* info = reinterpret_cast<volatile Item*>(smem_ptr(bars + kInfo));
    const uint32_t answer = bars + kInfo + 2u * (uint32_t)sizeof(Item), tmem_slot = answer + 16u;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < N_BARS; ++i) mbar_init(bar(i), i >= P_READY ? 16 : i >= INFO_EMPTY ? 2 + 16 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) alloc_tmem(tmem_slot);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem_ptr(tmem_slot));
    pdl_wait();      // set-up done; global memory is touched from here on
    const uint32_t tK_hi = tmem, tK_lo = tmem + 64, tdK = tmem + 128, tdV = tmem + 192;
    const uint32_t tS = tmem + 256, tPlo = tmem + 320, tdP = tmem + 384, tdSlo = tmem + 448;
    auto next = [&](int i, Item& it, bool whole_warp) -> bool {     // every role walks the same items
        return get_item(info, bar(INFO_FULL), bar(INFO_EMPTY), i, it, g.err, whole_warp);
    };

    if (warp < 4) {
        set_regs_down<kRegsIssueDkv>();
        if (warp == 0 && lane == 0) {
            uint32_t gt = 0, vi = 0;                    // tiles and non-empty items before this item
            Item it = make_item(g, args.head_group, (int)blockIdx.x, (int)blockIdx.y, true, BR, BT64);
            bool ok = put_item(info, bar(INFO_FULL), bar(INFO_EMPTY), 0, it, g.err);
            for (int i = 0; ok && it.n >= 0; ++i) {
                const int last = 4 * it.n + 1;          // asked for and looked up as in the forward
                if (it.n == 0) ask_next(answer, bar(NEXT));
                Item follows{0, 0, 0, -1};
                auto look_up = [&]() -> bool {
                    if (!mbar_wait(bar(NEXT), (uint32_t)i & 1u, g.err, 120)) return false;
                    int x, y;
                    if (next_item(answer, x, y)) follows = make_item(g, args.head_group, x, y, true, BR, BT64);
                    if (follows.n > 0) {
                        const int h = follows.bh % g.H, row0 = (follows.bh / g.H) * g.T, k0 = row0 + follows.blk * BR;
                        for (int kb = 0; kb < KB; ++kb) {
                            prefetch_box(&tmQk, kb * 32, g.H + h, k0);             // K, 64 rows at a time
                            prefetch_box(&tmQk, kb * 32, g.H + h, k0 + BT64);
                            prefetch_box(&tmVres, kb * 32, 2 * g.H + h, k0);
                            prefetch_box(&tmQk, kb * 32, h, row0 + follows.t0 * BT64);
                            prefetch_box(&tmDOk, kb * 32, h, row0 + follows.t0 * BT64);
                        }
                    }
                    return put_item(info, bar(INFO_FULL), bar(INFO_EMPTY), i + 1, follows, g.err);
                };
                if (it.n == 0) ok = look_up();
                const int h = it.bh % g.H, row0 = (it.bh / g.H) * g.T;
                // in the order the products consume them: S^T(0), dP^T(0), then per tile dV(t), S^T(t+1), dK(t), dP^T(t+1)
                for (int p = 0; it.n > 0 && p <= last && ok; ++p) {
                    if (p == max(0, last - 16)) ask_next(answer, bar(NEXT));
                    if (p == max(1, last - 11)) ok = look_up();
                    if (!ok) break;
                    // j: 0 dO MN-major (t), 1 Q K-major (t+1), 2 Q MN-major (t), 3 dO K-major (t+1); first Q(0), dO(0) K-major
                    const int j = p == 0 ? 1 : p == 1 ? 3 : (p - 2) & 3;
                    const int t = p < 2 ? 0 : ((p - 2) >> 2) + (j & 1);
                    if (t < it.n) {
                        const uint32_t dst = j == 0 ? dom_s : j == 1 ? qk_s : j == 2 ? qm_s : dok_s;
                        const CUtensorMap* tm = j == 0 ? &tmDOm : j == 1 ? &tmQk : j == 2 ? &tmQm : &tmDOk;
                        const int full = j == 0 ? DOM_FULL : j == 1 ? QK_FULL : j == 2 ? QM_FULL : DOK_FULL;
                        ok = mbar_wait(bar(full + 1), ((gt + (uint32_t)t) & 1u) ^ 1u, g.err, 131);   // every EMPTY barrier follows its FULL barrier
                        if (!ok) break;
                        mbar_expect_tx(bar(full), kTile);
                        for (int kb = 0; kb < KB; ++kb)
                            load_box(dst + kb * (kTile / KB), tm, bar(full), kb * 32, h, row0 + (it.t0 + t) * BT64);
                    }
                    if (p == 0) {                       // V, once the previous item's last dP^T is done with it
                        ok = mbar_wait(bar(V_EMPTY), (vi & 1u) ^ 1u, g.err, 132);
                        if (!ok) break;
                        mbar_expect_tx(bar(V_FULL), kResBytes);
                        for (int kb = 0; kb < KB; ++kb)
                            load_box(v_s + kb * (kResBytes / KB), &tmVres, bar(V_FULL), kb * 32, 2 * g.H + h, row0 + it.blk * BR);
                    }
                }
                gt += (uint32_t)it.n;
                if (it.n > 0) ++vi;
                it = follows;
            }
            if (!ok) settle();
        } else if (warp == 1 || warp == 2) {
            constexpr uint32_t idesc_a = make_idesc_tf32(BR, BT64, false, false);
            constexpr uint32_t idesc_a2 = make_idesc_tf32(BR, 2 * BT64, false, false);   // B = [hi rows | lo rows]
            constexpr uint32_t idesc_b = make_idesc_tf32(BR, HD, false, true);
            const bool score_chain = warp == 1;
            const DescBase vd = kmaj_base(v_s), qd = kmaj_base(score_chain ? qk_s : dok_s), bd = mn_base(score_chain ? dom_s : qm_s);
            const uint32_t t_x = score_chain ? tS : tdP, t_xlo = score_chain ? tPlo : tdSlo, t_acc = score_chain ? tdV : tdK;
            const int x_full = score_chain ? QK_FULL : DOK_FULL, x_done = score_chain ? S_FULL : DP_FULL;
            const int acc_in = score_chain ? P_READY : DS_READY, acc_b = score_chain ? DOM_FULL : QM_FULL;
            uint32_t gt = 0, ni = 0;
            Item it;
            bool ok = true;
            for (int i = 0; ok && (ok = next(i, it, true)) && it.n >= 0; ++i) {
                if (it.n == 0) continue;
                ok = mbar_wait_warp(bar(score_chain ? K_READY : V_FULL), ni & 1u, g.err, 133);
                for (int t = 0; t <= it.n && ok; ++t) {
                    if (t > 0) {
                        // dV += P^T dO or dK += dS^T Q of tile t - 1: from zero, the small terms first; it frees the
                        // region that the next score product overwrites
                        const uint32_t ph = (gt + (uint32_t)t - 1u) & 1u;
                        if (!mbar_wait_warp(bar(acc_in), ph, g.err, 137) || !mbar_wait_warp(bar(acc_b), ph, g.err, 138)) { ok = false; break; }
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int ks = 0; ks < 8; ++ks) {
                                umma_tf32_ts(t_acc, t_xlo + ks * 8, bd.at(mn_off(ks, false)), idesc_b, ks > 0 ? 1u : 0u);
                                umma_tf32_ts(t_acc, t_x + ks * 8, bd.at(mn_off(ks, true)), idesc_b, 1u);
                            }
#pragma unroll
                            for (int ks = 0; ks < 8; ++ks) umma_tf32_ts(t_acc, t_x + ks * 8, bd.at(mn_off(ks, false)), idesc_b, 1u);
                            umma_commit(bar(acc_b + 1));
                            if (t == it.n) umma_commit(bar(score_chain ? ACC_V : ACC_K));
                        }
                        __syncwarp();
                    }
                    if (t < it.n) {
                        // A tile's lo rows follow its hi rows, so [hi | lo] is one operand of 128 rows whose second half lands in
                        // the neighbouring 64 columns; A_lo hi joins it there, the small terms apart from the
                        // large one, and the reader adds the halves.
                        if (!mbar_wait_warp(bar(x_full), (gt + (uint32_t)t) & 1u, g.err, 135)) { ok = false; break; }
                        tc_fence_after();
                        if (elect_one()) {
                            if (score_chain) {
#pragma unroll
                                for (int ks = 0; ks < KS; ++ks) {
                                    const uint64_t b_hl = qd.at(kmaj_off(BT64, ks, false));
                                    umma_tf32_ts(t_x, tK_hi + ks * 8, b_hl, idesc_a2, ks > 0 ? 1u : 0u);      // K'_hi Q_hi | K'_hi Q_lo
                                    umma_tf32_ts(t_xlo, tK_lo + ks * 8, b_hl, idesc_a, 1u);                   // + K'_lo Q_hi
                                }
                            } else {
#pragma unroll
                                for (int ks = 0; ks < KS; ++ks) {
                                    const uint64_t b_hl = qd.at(kmaj_off(BT64, ks, false));
                                    umma_tf32(t_x, vd.at(kmaj_off(BR, ks, false)), b_hl, idesc_a2, ks > 0 ? 1u : 0u);   // V_hi dO_hi | V_hi dO_lo
                                    umma_tf32(t_xlo, vd.at(kmaj_off(BR, ks, true)), b_hl, idesc_a, 1u);                 // + V_lo dO_hi
                                }
                            }
                            umma_commit(bar(x_full + 1));
                            umma_commit(bar(x_done));
                            if (!score_chain && t == it.n - 1) umma_commit(bar(V_EMPTY));
                        }
                        __syncwarp();
                    }
                }
                gt += (uint32_t)it.n;
                ++ni;
            }
        }
    } else {
        set_regs_up<kRegsElemDkv>();
        const int wg = (warp - 4) >> 2, lane_group = warp & 3, rloc = lane_group * 32 + lane;
        const uint32_t t_lane = ((uint32_t)(lane_group * 32) << 16), c0 = 16u * (uint32_t)wg;
        const float scale = 1.0f / sqrtf((float)d);
        const int64_t gs = 3 * (int64_t)g.C;
        const bool tile_cols = HD == 64 || c0 < (uint32_t)HD, own_cols = HD == 64 || c0 < (uint32_t)d;   // narrow heads: the first warpgroups hold all columns
        // Statistics of a tile's 64 queries (lse in base-2 units, D) through shared memory, one tile ahead, from the
        // first warpgroup's threads.  All sixteen warps arrive: no warp can be two phases behind.
        float* stat = reinterpret_cast<float*>(smem_ptr(bars + 512u));
        const int sidx = (int)threadIdx.x - 128;
        auto fetch_stat = [&](const Item& it, int t) -> float {
            const int64_t lb = (int64_t)it.bh * g.T;
            const int r = min((it.t0 + t) * BT64 + (sidx & 63), g.T - 1);   // rows past the end are masked below
            return sidx >= 128 ? 0.f : sidx < 64 ? __ldg(g.lse + lb + r) * kLog2e : __ldg(g.dvec + lb + r);
        };
        auto publish_stat = [&](uint32_t ga, float v) {
            if (sidx < 128) {
                stat[(ga & 1u) * 128u + sidx] = v;
                __threadfence_block();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(STAT_READY));
        };
        // K' = K * unit of an item into tensor memory (16 columns here), and its first tile's statistics
        auto begin_item = [&](const Item& it, const Score& sc, uint32_t ga) {
            const float st0 = fetch_stat(it, 0);
            const int row = min(it.blk * BR + rloc, g.T - 1);
            const int64_t off = ((int64_t)(it.bh / g.H) * g.T + row) * gs + g.C + (int64_t)(it.bh % g.H) * d + c0;
            float a[2][8] = {}, e[2][8] = {};
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                if (!own_cols) break;
                load_sector(g.qkv + off + 8 * q, a[q]);
                load_sector(g.qkv_lo + off + 8 * q, e[q]);
            }
            if (tile_cols) {
                uint32_t hi[16], lo[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) split_tf32_int((a[k >> 3][k & 7] + e[k >> 3][k & 7]) * sc.unit, hi[k], lo[k]);
                tmem_stn(tK_hi + t_lane + c0, hi);   // the last S^T of the item before has been read
                tmem_stn(tK_lo + t_lane + c0, lo);
                tmem_st_wait();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(K_READY));
            publish_stat(ga, st0);
        };
        auto score_of = [&](const Item& it) { return make_score<CAP, SLOPE>(scale, g.cap, g.slopes, it.bh % g.H); };
        uint32_t gt = 0, ni = 0;
        Item it;
        bool ok = next(0, it, true);
        Score sc = score_of(it);
        if (ok && it.n > 0) begin_item(it, sc, 0);
        for (int i = 0; ok && it.n >= 0; ++i) {
            const int b = it.bh / g.H, h = it.bh % g.H, key = it.blk * BR + rloc;
            const int2 span = row_range(g.spans.q, b, g.T, key, true);
            float acc_v[16], acc_k[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) acc_v[k] = acc_k[k] = 0.f;
            for (int t = 0; t < it.n; ++t) {
                const uint32_t ga = gt + (uint32_t)t, ph = ga & 1u;
                const int q0 = (it.t0 + t) * BT64 + (int)c0;
                float next_stat = 0.f;
                if (t + 1 < it.n) next_stat = fetch_stat(it, t + 1);        // in flight during this tile
                if (!mbar_wait_warp(bar(STAT_READY), ph, g.err, 142)) { ok = false; break; }
                const float4* Ls = reinterpret_cast<const float4*>(stat + ph * 128u + c0);
                const float4* Ds = Ls + 16;
                if (!mbar_wait_warp(bar(S_FULL), ph, g.err, 141)) { ok = false; break; }
                tc_fence_after();
                float p[16], f[16];
                uint32_t s[16], lo[16];
                tmem_ldn(tS + t_lane + c0, s);
                tmem_ldn(tPlo + t_lane + c0, lo);
                tmem_ld_wait();
#pragma unroll
                for (int k = 0; k < 16; ++k) p[k] = __uint_as_float(s[k]) + __uint_as_float(lo[k]);
                score_tile<CAP, SLOPE, true, false, 16>(p, f, sc, key - q0, 0.f);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float4 l4 = Ls[q];
                    p[4 * q] = ex2_approx(p[4 * q] - l4.x);
                    p[4 * q + 1] = ex2_approx(p[4 * q + 1] - l4.y);
                    p[4 * q + 2] = ex2_approx(p[4 * q + 2] - l4.z);
                    p[4 * q + 3] = ex2_approx(p[4 * q + 3] - l4.w);
                }
                if (q0 < span.x || q0 + 16 > span.y) {
                    const uint32_t bits = column_bits<16>(span, q0);
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (!(bits >> k & 1u)) p[k] = 0.f;
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) split_tf32_int(p[k], s[k], lo[k]);
                tmem_stn(tS + t_lane + c0, s);           // P^T over S^T
                tmem_stn(tPlo + t_lane + c0, lo);
                if (tile_cols) tmem_ldn(tdV + t_lane + c0, s);   // dV(t - 1): complete, as S^T(t) is (not used at t = 0)
                tmem_ld_wait();
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(P_READY));
                if (CAP) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) p[k] *= f[k];
                }
                if (tile_cols && t > 0) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) acc_v[k] += __uint_as_float(s[k]);
                }
                if (!mbar_wait_warp(bar(DP_FULL), ph, g.err, 143)) { ok = false; break; }
                tc_fence_after();
                tmem_ldn(tdP + t_lane + c0, s);
                tmem_ldn(tdSlo + t_lane + c0, lo);
                tmem_ld_wait();
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float4 d4 = Ds[q];
                    const float dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int k = 4 * q + e;
                        split_tf32_int(p[k] * ((__uint_as_float(s[k]) + __uint_as_float(lo[k])) - dd[e]), s[k], lo[k]);
                    }
                }
                tmem_stn(tdP + t_lane + c0, s);          // dS^T over dP^T
                tmem_stn(tdSlo + t_lane + c0, lo);
                if (tile_cols) tmem_ldn(tdK + t_lane + c0, s);   // dK(t - 1): complete, as dP^T(t) is
                tmem_ld_wait();
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(DS_READY));
                if (tile_cols && t > 0) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) acc_k[k] += __uint_as_float(s[k]);
                }
                if (t + 1 < it.n) publish_stat(ga + 1u, next_stat);
            }
            if (!ok) break;
            // the next item's operand first, then what is left of this one
            gt += (uint32_t)it.n;
            Item follows;
            if (!next(i + 1, follows, true)) { ok = false; break; }
            const Score sc_next = score_of(follows);
            if (follows.n > 0) begin_item(follows, sc_next, gt);
            if (it.n > 0) {
                if (!mbar_wait_warp(bar(ACC_V), ni & 1u, g.err, 144) || !mbar_wait_warp(bar(ACC_K), ni & 1u, g.err, 145)) { ok = false; break; }
                ++ni;
                tc_fence_after();
                if (tile_cols) {
                    uint32_t r[16], r2[16];
                    tmem_ldn(tdV + t_lane + c0, r);
                    tmem_ldn(tdK + t_lane + c0, r2);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        acc_v[k] += __uint_as_float(r[k]);
                        acc_k[k] = (acc_k[k] + __uint_as_float(r2[k])) * scale;
                    }
                }
                tc_fence_before();
            }
            if (key < g.T && own_cols) {
                const int64_t at = ((int64_t)b * g.T + key) * gs + g.C + (int64_t)h * d + c0;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = acc_k[8 * q + e];
                    store_sector(v, at + 8 * q, g.dqkv, g.dqkv_hi, g.dqkv_lo);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = acc_v[8 * q + e];
                    store_sector(v, at + g.C + 8 * q, g.dqkv, g.dqkv_hi, g.dqkv_lo);
                }
            }
            it = follows;
            sc = sc_next;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) free_tmem(tmem);
}

// --------------------------------------------------------------------------------------------- backward, dQ
//
// Persistent as the others; an item is 128 queries of one head and the 64-key tiles they read.  It also forms D = rowsum(dO o O),
// which the dkv kernel reads.
//     S = Q' K^T | dP = dO V^T | dS = P o (dP - D) (1 - tanh^2) | dQ_tile = dS K
//   warp 0      TMA producer and scheduler;   warps 1, 2, 3 issue S, dP, dQ
//   warps 4-11, 12-19  two pairs of element-wise warpgroups on alternate tiles, thread = row, 32 of the tile's keys each.  The
//               pair whose tile an item begins with loads the item's Q' and forms its D while the other is at the
//               last tile of the item before
//   warps 20-23 add every dQ tile to registers (64 columns of a row per thread) and write the result
//   tensor memory  Q' hi|lo 0-127, dQ tile 128-255, buffer b at 256 + 128b: S -> dS_hi, dP -> dS_lo
// The dQ tile is 128 wide (heads of 32 and fewer: the first half of this): the column groups [K_hi g0 | K_lo g0 | K_hi g1 | K_lo g1] (g = 32 head columns) as
// one operand of dS_hi, and dS_lo K_hi 32 columns further, on the second and third group; head columns
// 0-31 are the sum of groups 0 and 1, 32-63 that of 2 and 3.
// 8 packed sequences of 1,024, 12 heads, cap: 124 us, tensor pipe 35 % busy: seven tiles an item there, and an item's Q' and D
// (5,000 to 8,000 clocks) overlap only the last tile before.
constexpr int kDqThreads = 768, kRegsIssueDq = 56, kRegsElemDq = 72, kRegsAddDq = 128;
static_assert(kRegsIssueDq + 4 * kRegsElemDq + kRegsAddDq <= 480, "registers: 768 threads get 80 each at launch");
template <int HD> constexpr uint32_t kDqSmem = 1024u + kRes<HD> + 5u * kTileBytes<HD> + 512u + 1024u;
static_assert(kDqSmem<64> <= 232448u, "shared memory");

template <int HD, bool CAP, bool SLOPE>
__global__ void __launch_bounds__(kDqThreads, 1)
attn_mod_dq_kernel(const __grid_constant__ CUtensorMap tmKk, const __grid_constant__ CUtensorMap tmKm,
                   const __grid_constant__ CUtensorMap tmVk, const __grid_constant__ CUtensorMap tmDOres, const ModTcArgs args) {
    const AttnModArgs& g = args.a;
    constexpr uint32_t kResBytes = kRes<HD>, kTile = kTileBytes<HD>;
    constexpr int KB = HD / 32, KS = HD / 8;             // k-blocks, and k-steps of a product over the head's columns
    const int d = HD == 64 ? HD : args.d;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t do_s = base, kv_s = base + kResBytes, km_s = kv_s + 4u * kTile, bars = km_s + kTile;   // kv_s: stage st: K at 2 st, V at 2 st + 1
    // the S and the dP issuing warps both commit to KEMPTY and SDP
    enum { DO_FULL = 0, DO_EMPTY, KFULL, MFULL = KFULL + 2, MEMPTY, DONE, DQ_FULL = DONE + 2, Q_FREE, NEXT, INFO_FULL, INFO_EMPTY = INFO_FULL + 2,
           KEMPTY = INFO_EMPTY + 2, SDP = KEMPTY + 2, DQ_FREE = SDP + 2, DS, Q_READY = DS + 2, D_FREE, N_BARS };
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    constexpr uint32_t kInfo = (8u * N_BARS + 15u) & ~15u;
    static_assert(kInfo + 2 * sizeof(Item) + 32 <= 512, "barrier region");
    auto smem_ptr = [&](uint32_t addr) { return smem_raw + (addr - smem_u32(smem_raw)); };
    volatile Item* info = reinterpret_cast<volatile Item*>(smem_ptr(bars + kInfo));
    const uint32_t answer = bars + kInfo + 2u * (uint32_t)sizeof(Item), tmem_slot = answer + 16u;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < N_BARS; ++i)
            mbar_init(bar(i), i == DO_EMPTY ? 9 : i == D_FREE ? 16 : i >= DS ? 8 : i == DQ_FREE ? 4 : i >= KEMPTY ? 2 : i >= INFO_EMPTY ? 3 + 16 + 4 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) alloc_tmem(tmem_slot);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem_ptr(tmem_slot));
    pdl_wait();      // set-up done; global memory is touched from here on
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *g.err = 0;
    const uint32_t tQ_hi = tmem, tQ_lo = tmem + 64, tdQ = tmem + 128;
    auto tbuf = [&](uint32_t bb) { return tmem + 256u + 128u * bb; };
    auto next = [&](int i, Item& it, bool whole_warp) -> bool {     // every role walks the same items
        return get_item(info, bar(INFO_FULL), bar(INFO_EMPTY), i, it, g.err, whole_warp);
    };

    if (warp < 4) {
        set_regs_down<kRegsIssueDq>();
        if (warp == 0) {
            if (lane == 0) {
                uint32_t gt = 0, di = 0;                // tiles and non-empty items before this item
                Item it = make_item(g, args.head_group, (int)blockIdx.x, (int)blockIdx.y, false, BR, BT64);
                bool ok = put_item(info, bar(INFO_FULL), bar(INFO_EMPTY), 0, it, g.err);
                for (int i = 0; ok && it.n >= 0; ++i) {
                    if (it.n == 0) ask_next(answer, bar(NEXT));
                    Item follows{0, 0, 0, -1};
                    auto look_up = [&]() -> bool {      // asked for and looked up as in the forward
                        if (!mbar_wait(bar(NEXT), (uint32_t)i & 1u, g.err, 120)) return false;
                        int x, y;
                        if (next_item(answer, x, y)) follows = make_item(g, args.head_group, x, y, false, BR, BT64);
                        if (follows.n > 0) {
                            const int h = follows.bh % g.H, row0 = (follows.bh / g.H) * g.T, q0 = row0 + follows.blk * BR;
                            for (int kb = 0; kb < KB; ++kb) {
                                prefetch_box(&tmDOres, kb * 32, h, q0);
                                prefetch_box(&tmKk, kb * 32, h, q0);               // Q, 64 rows at a time
                                prefetch_box(&tmKk, kb * 32, h, q0 + BT64);
                                prefetch_box(&tmKk, kb * 32, g.H + h, row0 + follows.t0 * BT64);
                                prefetch_box(&tmVk, kb * 32, 2 * g.H + h, row0 + follows.t0 * BT64);
                            }
                        }
                        return put_item(info, bar(INFO_FULL), bar(INFO_EMPTY), i + 1, follows, g.err);
                    };
                    if (it.n == 0) ok = look_up();
                    const int h = it.bh % g.H, row0 = (it.bh / g.H) * g.T;
                    // K and V (K-major) of tile t + 1 go out before the single MN-major K buffer is waited for
                    for (int t = -1; t < it.n && it.n > 0 && ok; ++t) {
                        if (t == max(-1, it.n - 5)) ask_next(answer, bar(NEXT));
                        if (t == max(0, it.n - 4)) ok = look_up();
                        if (!ok) break;
                        if (t + 1 < it.n) {
                            const uint32_t ga = gt + (uint32_t)(t + 1), st = ga & 1u;
                            ok = mbar_wait(bar(KEMPTY + st), ((ga >> 1) & 1u) ^ 1u, g.err, 151);
                            if (!ok) break;
                            mbar_expect_tx(bar(KFULL + st), 2u * kTile);
                            for (int kb = 0; kb < KB; ++kb) {
                                load_box(kv_s + 2u * st * kTile + kb * (kTile / KB), &tmKk, bar(KFULL + st), kb * 32, g.H + h, row0 + (it.t0 + t + 1) * BT64);
                                load_box(kv_s + (2u * st + 1u) * kTile + kb * (kTile / KB), &tmVk, bar(KFULL + st), kb * 32, 2 * g.H + h, row0 + (it.t0 + t + 1) * BT64);
                            }
                        }
                        if (t < 0) {                    // dO, once the previous item's last dP is done with it
                            ok = mbar_wait(bar(DO_EMPTY), (di & 1u) ^ 1u, g.err, 152);
                            if (!ok) break;
                            mbar_expect_tx(bar(DO_FULL), kResBytes);
                            for (int kb = 0; kb < KB; ++kb)
                                load_box(do_s + kb * (kResBytes / KB), &tmDOres, bar(DO_FULL), kb * 32, h, row0 + it.blk * BR);
                        } else {
                            ok = mbar_wait(bar(MEMPTY), ((gt + (uint32_t)t) & 1u) ^ 1u, g.err, 153);
                            if (!ok) break;
                            mbar_expect_tx(bar(MFULL), kTile);
                            for (int kb = 0; kb < KB; ++kb)
                                load_box(km_s + kb * (kTile / KB), &tmKm, bar(MFULL), kb * 32, g.H + h, row0 + (it.t0 + t) * BT64);
                        }
                    }
                    gt += (uint32_t)it.n;
                    if (it.n > 0) ++di;
                    it = follows;
                }
                if (!ok) settle();
            }
        } else if (warp < 3) {
            constexpr uint32_t idesc = make_idesc_tf32(BR, BT64, false, false);
            const bool s_product = warp == 1;
            const DescBase dod = kmaj_base(do_s);
            uint32_t gt = 0, ni = 0;
            Item it;
            bool ok = true;
            for (int i = 0; ok && (ok = next(i, it, true)) && it.n >= 0; ++i) {
                if (it.n == 0) continue;
                ok = mbar_wait_warp(bar(s_product ? Q_READY : DO_FULL), ni & 1u, g.err, 154);
                for (int t = 0; t < it.n && ok; ++t, ++gt) {
                    const uint32_t st = gt & 1u;
                    if (!mbar_wait_warp(bar(KFULL + st), (gt >> 1) & 1u, g.err, 156)) { ok = false; break; }
                    // buffer st: the dQ product of two tiles before has read it
                    if (gt >= 2 && !mbar_wait_warp(bar(DONE + st), ((gt >> 1) - 1u) & 1u, g.err, 157)) { ok = false; break; }
                    tc_fence_after();
                    if (elect_one()) {
                        if (s_product) {
                            const uint32_t dst = tbuf(st);
                            const DescBase kd = kmaj_base(kv_s + 2u * st * kTile);
#pragma unroll
                            for (int ks = 0; ks < KS; ++ks) {
                                umma_tf32_ts(dst, tQ_lo + ks * 8, kd.at(kmaj_off(BT64, ks, false)), idesc, ks > 0 ? 1u : 0u);
                                umma_tf32_ts(dst, tQ_hi + ks * 8, kd.at(kmaj_off(BT64, ks, true)), idesc, 1u);
                            }
#pragma unroll
                            for (int ks = 0; ks < KS; ++ks) umma_tf32_ts(dst, tQ_hi + ks * 8, kd.at(kmaj_off(BT64, ks, false)), idesc, 1u);
                        } else {
                            const uint32_t dst = tbuf(st) + 64u;
                            const DescBase vd = kmaj_base(kv_s + (2u * st + 1u) * kTile);
#pragma unroll
                            for (int ks = 0; ks < KS; ++ks) {
                                umma_tf32(dst, dod.at(kmaj_off(BR, ks, true)), vd.at(kmaj_off(BT64, ks, false)), idesc, ks > 0 ? 1u : 0u);
                                umma_tf32(dst, dod.at(kmaj_off(BR, ks, false)), vd.at(kmaj_off(BT64, ks, true)), idesc, 1u);
                            }
#pragma unroll
                            for (int ks = 0; ks < KS; ++ks)
                                umma_tf32(dst, dod.at(kmaj_off(BR, ks, false)), vd.at(kmaj_off(BT64, ks, false)), idesc, 1u);
                        }
                        umma_commit(bar(KEMPTY + st));
                        umma_commit(bar(SDP + st));
                        if (t == it.n - 1) umma_commit(bar(s_product ? Q_FREE : DO_EMPTY));
                    }
                    __syncwarp();
                }
                ++ni;
            }
        } else {
            constexpr uint32_t idesc = make_idesc_tf32(BR, HD, false, true), idesc2 = make_idesc_tf32(BR, 2 * HD, false, true);
            const DescBase kmd = mn_base(km_s), kmd4 = make_desc_base(km_s, BT64 * 128u, 512u, 1u);
            uint32_t gt = 0;
            Item it;
            bool ok = true;
            for (int i = 0; ok && (ok = next(i, it, true)) && it.n >= 0; ++i) {
                for (int t = 0; t < it.n && ok; ++t, ++gt) {
                    const uint32_t bb = gt & 1u;
                    if (!mbar_wait_warp(bar(MFULL), gt & 1u, g.err, 159)) { ok = false; break; }
                    if (gt > 0 && !mbar_wait_warp(bar(DQ_FREE), (gt - 1u) & 1u, g.err, 160)) { ok = false; break; }
                    if (!mbar_wait_warp(bar(DS + bb), (gt >> 1) & 1u, g.err, 158)) { ok = false; break; }
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t s_hi = tbuf(bb), s_lo = s_hi + 64u;
                        // one large term, to set all columns, then the small ones, then the other large ones
                        umma_tf32_ts(tdQ, s_hi, kmd4.at(mn_off(0, false)), idesc2, 0u);
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks) umma_tf32_ts(tdQ + 32u, s_lo + ks * 8, kmd.at(mn_off(ks, false)), idesc, 1u);
#pragma unroll
                        for (int ks = 1; ks < 8; ++ks) umma_tf32_ts(tdQ, s_hi + ks * 8, kmd4.at(mn_off(ks, false)), idesc2, 1u);
                        umma_commit(bar(MEMPTY));
                        umma_commit(bar(DONE + bb));
                        umma_commit(bar(DQ_FULL));
                    }
                    __syncwarp();
                }
            }
        }
    } else if (warp < 20) {
        set_regs_down<kRegsElemDq>();
        const uint32_t pair = (uint32_t)(warp - 4) >> 3, part = ((uint32_t)(warp - 4) >> 2) & 1u;   // 32 part .. of a tile's keys
        const int lane_group = warp & 3, rloc = lane_group * 32 + lane;
        const uint32_t t_lane = (uint32_t)(lane_group * 32) << 16, c0 = 32u * part;
        const uint32_t tb = tbuf(pair) + t_lane + c0;
        float* dsm = reinterpret_cast<float*>(smem_ptr(bars + 512u));        // [2][128]: D over each half of the head's columns
        uint32_t gt = 0, ni = 0;
        Item it;
        bool ok = true;
        for (int i = 0; ok && (ok = next(i, it, true)) && it.n >= 0; ++i) {
            const int b = it.bh / g.H, h = it.bh % g.H, row = it.blk * BR + rloc, rc = min(row, g.T - 1);
            const Score sc = make_score<CAP, SLOPE>(1.0f / sqrtf((float)d), g.cap, g.slopes, h);
            const int64_t lb = (int64_t)it.bh * g.T;
            if (it.n == 0) {                            // rows that read nothing: D only has to be finite
                if (pair == 0 && part == 0 && row < g.T) g.dvec[lb + row] = 0.f;
                continue;
            }
            if (pair == (gt & 1u)) {
                // this pair has the item's first tile: D over half the columns here (dO lies in shared memory), and Q' = Q * unit
                // into tensor memory; all loads of a half are on their way together
                constexpr int kCols = HD / 2;
                const int h0 = (int)part * kCols;
                const int64_t at = ((int64_t)b * g.T + rc) * g.C + (int64_t)h * d + h0;
                const int64_t qat = ((int64_t)b * g.T + rc) * 3 * (int64_t)g.C + (int64_t)h * d + h0;
                const uint8_t* do_row = smem_ptr(do_s + (uint32_t)(h0 >> 5) * (kResBytes / KB)) + rloc * 128;
                float dot = 0.f;
#pragma unroll 1
                for (int q = 0; q < kCols; q += 16) {
                    float o[2][8] = {}, x[2][8] = {}, y[2][8] = {};
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        if (HD < 64 && h0 >= d) break;  // a head of 16: the second part's columns are zeros
                        load_sector(g.o + at + q + 8 * k, o[k]);
                        load_sector(g.qkv + qat + q + 8 * k, x[k]);
                        load_sector(g.qkv_lo + qat + q + 8 * k, y[k]);
                    }
                    if (q == 0) {
                        // dO has landed; everyone has read the D, and the last S is done with the Q', of the item before
                        if (!mbar_wait_warp(bar(DO_FULL), ni & 1u, g.err, 155) ||
                            (ni > 0 && (!mbar_wait_warp(bar(D_FREE), (ni - 1u) & 1u, g.err, 163) ||
                                        !mbar_wait_warp(bar(Q_FREE), (ni - 1u) & 1u, g.err, 164)))) { ok = false; break; }
                        tc_fence_after();
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {       // 16-byte pieces of the row, swizzled by its number
                        const uint32_t piece = ((((uint32_t)(h0 + q) & 31u) >> 2) + (uint32_t)k) ^ ((uint32_t)rloc & 7u);
                        const float4 v = add4(*reinterpret_cast<const float4*>(do_row + piece * 16u),
                                              *reinterpret_cast<const float4*>(do_row + BR * 128u + piece * 16u));
                        const float* ok4 = &o[k >> 1][4 * (k & 1)];
                        dot = fmaf(v.x, ok4[0], fmaf(v.y, ok4[1], fmaf(v.z, ok4[2], fmaf(v.w, ok4[3], dot))));
                    }
                    uint32_t hi[16], lo[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) split_tf32_int((x[k >> 3][k & 7] + y[k >> 3][k & 7]) * sc.unit, hi[k], lo[k]);
                    tmem_stn(tQ_hi + t_lane + (uint32_t)(h0 + q), hi);
                    tmem_stn(tQ_lo + t_lane + (uint32_t)(h0 + q), lo);
                }
                if (!ok) break;
                dsm[part * 128u + (uint32_t)rloc] = dot;
                __threadfence_block();
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(bar(DO_EMPTY));
                    mbar_arrive(bar(Q_READY));
                }
            }
            const float L = __ldg(g.lse + lb + rc) * kLog2e;
            const int2 span = row_range(g.spans.k, b, g.T, row, false);
            if (!mbar_wait_warp(bar(Q_READY), ni & 1u, g.err, 165)) { ok = false; break; }   // both pairs: no phase is missed
            ++ni;
            const float D = dsm[rloc] + dsm[128 + rloc];
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(D_FREE));
            if (pair == (gt & 1u) && part == 0 && row < g.T) g.dvec[lb + row] = D;
            for (int t = (int)(pair ^ (gt & 1u)); t < it.n; t += 2) {
                const uint32_t ga = gt + (uint32_t)t;
                const int k0 = (it.t0 + t) * BT64 + (int)c0;
                if (!mbar_wait_warp(bar(SDP + pair), (ga >> 1) & 1u, g.err, 162)) { ok = false; break; }
                tc_fence_after();
                const bool whole = k0 >= span.x && k0 + 32 <= span.y;
#pragma unroll 1
                for (int q = 0; q < 32; q += 16) {
                    float x[16], f[16];
                    uint32_t s[16], dp[16];
                    tmem_ldn(tb + q, s);
                    tmem_ldn(tb + 64u + q, dp);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 16; ++k) x[k] = __uint_as_float(s[k]);
                    score_tile<CAP, SLOPE, true, false, 16>(x, f, sc, row - k0 - q, L);
#pragma unroll
                    for (int k = 0; k < 16; ++k) x[k] = ex2_approx(x[k]);
                    if (!whole) {
                        const uint32_t bits = column_bits<16>(span, k0 + q);
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (!(bits >> k & 1u)) x[k] = 0.f;
                    }
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        float ds = x[k] * (__uint_as_float(dp[k]) - D);
                        if (CAP) ds *= f[k];
                        split_tf32_int(ds, s[k], dp[k]);
                    }
                    tmem_stn(tb + q, s);                                // dS hi over S
                    tmem_stn(tb + 64u + q, dp);                         // dS lo over dP
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(DS + pair));
            }
            gt += (uint32_t)it.n;
        }
    } else {
        set_regs_up<kRegsAddDq>();
        const int lane_group = warp & 3, rloc = lane_group * 32 + lane;
        const uint32_t t_row = tdQ + ((uint32_t)(lane_group * 32) << 16);
        const float scale = 1.0f / sqrtf((float)d);
        const int64_t gs = 3 * (int64_t)g.C;
        uint32_t gt = 0;
        Item it;
        bool ok = true;
        for (int i = 0; ok && (ok = next(i, it, true)) && it.n >= 0; ++i) {
            float acc[HD];
#pragma unroll
            for (int k = 0; k < HD; ++k) acc[k] = 0.f;
            for (int t = 0; t < it.n; ++t, ++gt) {
                if (!mbar_wait_warp(bar(DQ_FULL), gt & 1u, g.err, 161)) { ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int q = 0; q < HD / 16; ++q) {
                    uint32_t r[16], r2[16];
                    tmem_ldn(t_row + (uint32_t)(64 * (q >> 1) + 16 * (q & 1)), r);
                    tmem_ldn(t_row + (uint32_t)(64 * (q >> 1) + 16 * (q & 1) + 32), r2);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 16; ++k) acc[16 * q + k] += __uint_as_float(r[k]) + __uint_as_float(r2[k]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(DQ_FREE));
            }
            const int b = it.bh / g.H, h = it.bh % g.H, row = it.blk * BR + rloc;
            if (ok && row < g.T) {
                const int64_t at = ((int64_t)b * g.T + row) * gs + (int64_t)h * d;
#pragma unroll
                for (int q = 0; q < HD; q += 8) {
                    if (q >= d) break;
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = acc[q + e] * scale;
                    store_sector(v, at + q, g.dqkv, g.dqkv_hi, g.dqkv_lo);
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) free_tmem(tmem);
}

}  // namespace

namespace {

// Tensor map over the hi/lo planes [2][rows][heads][d] of whole heads: boxes of 32 columns (zeros past d) x one head x box_rows rows x
// both planes, K-major (128-byte swizzle) or MN-major (128-byte swizzle with 32-byte atoms).
bool head_map(CUtensorMap* tm, const float* base, int d, int64_t heads, int64_t rows, uint32_t box_rows, bool mn_major) {
    EncodeTiledFn enc = tensor_map_encoder();
    if (!enc) return false;
    cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)rows, 2};
    cuuint64_t strides[3] = {(cuuint64_t)d * 4, (cuuint64_t)(heads * d) * 4, (cuuint64_t)(rows * heads * d) * 4};
    cuuint32_t box[4] = {32, 1, box_rows, 2};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    return enc(tm, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, (void*)base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               mn_major ? CU_TENSOR_MAP_SWIZZLE_128B_ATOM_32B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD>
cudaError_t launch_fwd(const AttnModArgs& g, cudaStream_t s) {
    const int64_t rows = (int64_t)g.B * g.T;
    const int d = g.C / g.H;
    CUtensorMap q, k, v;
    if (!head_map(&q, g.qkv, d, 3 * g.H, rows, BR, false) || !head_map(&k, g.qkv, d, 3 * g.H, rows, BT64, false) ||
        !head_map(&v, g.qkv, d, 3 * g.H, rows, BT64, true))
        return cudaErrorInvalidValue;
    const dim3 grid(g.B * g.H, (g.T + BR - 1) / BR);
    const ModTcArgs a{g, d, attn_head_group((int)grid.x, (int)grid.y)};
    BT_FOR_MOD(g, {
        cudaError_t e = allow_smem<attn_mod_fwd_kernel<HD, kCap, kSlope>>(kFwdSmem<HD>);
        if (e != cudaSuccess) return e;
        BT_KERNEL_LAUNCH((attn_mod_fwd_kernel<HD, kCap, kSlope>), grid, kFwdThreads, kFwdSmem<HD>, s, q, k, v, a);
    });
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

template <int HD>
cudaError_t launch_bwd(const AttnModArgs& g, cudaStream_t s) {
    const int64_t rows = (int64_t)g.B * g.T;
    const int d = g.C / g.H;
    CUtensorMap qkv_k, qkv_m, qkv_res, do_k, do_m, do_res;
    if (!head_map(&qkv_k, g.qkv, d, 3 * g.H, rows, BT64, false) || !head_map(&qkv_m, g.qkv, d, 3 * g.H, rows, BT64, true) ||
        !head_map(&qkv_res, g.qkv, d, 3 * g.H, rows, BR, false) || !head_map(&do_k, g.d_o, d, g.H, rows, BT64, false) ||
        !head_map(&do_m, g.d_o, d, g.H, rows, BT64, true) || !head_map(&do_res, g.d_o, d, g.H, rows, BR, false))
        return cudaErrorInvalidValue;
    const dim3 grid(g.B * g.H, (g.T + BR - 1) / BR);
    const ModTcArgs a{g, d, attn_head_group((int)grid.x, (int)grid.y)};
    BT_FOR_MOD(g, {
        cudaError_t e = allow_smem<attn_mod_dq_kernel<HD, kCap, kSlope>>(kDqSmem<HD>);
        if (e == cudaSuccess)
            e = allow_smem<attn_mod_dkv_kernel<HD, kCap, kSlope>>(kDkvSmem<HD>);
        if (e != cudaSuccess) return e;
        // the dq kernel goes first: it also forms D
        BT_KERNEL_LAUNCH((attn_mod_dq_kernel<HD, kCap, kSlope>), grid, kDqThreads, kDqSmem<HD>, s, qkv_k, qkv_m, qkv_k, do_res, a);
        BT_KERNEL_LAUNCH((attn_mod_dkv_kernel<HD, kCap, kSlope>), grid, kDkvThreads, kDkvSmem<HD>, s, qkv_k, qkv_m, do_k, do_m, qkv_res, a);
    });
    BT_COUNT_LAUNCH();
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_mod_fwd_tc(const AttnModArgs& g, cudaStream_t s) {
    return g.C / g.H == 64 ? launch_fwd<64>(g, s) : launch_fwd<32>(g, s);
}

cudaError_t launch_attention_mod_bwd_tc(const AttnModArgs& g, cudaStream_t s) {
    return g.C / g.H == 64 ? launch_bwd<64>(g, s) : launch_bwd<32>(g, s);
}

}  // namespace bt
