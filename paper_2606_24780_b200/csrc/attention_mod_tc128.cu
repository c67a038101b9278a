// Attention with modified scores on the 5th-generation tensor cores, head_dim 128, 3xTF32.
//
// One small pipeline serves the forward and the three gradients (a 128-row operand of this width takes 128 KB
// as hi/lo planes: one fits in shared memory, one in tensor memory):
//
//     X = A1 B1^T     A1: the CTA's own 128 rows times the score unit, hi/lo in TENSOR MEMORY
//     Y = A2 B2^T     A2: the CTA's own rows of a second tensor, resident in shared memory
//     Z = f(X, Y)     element-wise, thread = own row;   Out_tile = Z B3;   Out += Out_tile in registers
//
//   pass  rows     A1  B1  A2  B2   f                                    B3   Out
//   FWD   queries  Q'  K   -   -    P = exp2(z - r), r the tile's maximum  V    O (rescaled), lse
//   DQ    queries  Q'  K   dO  V    dS = P o (Y - D) (1 - tanh^2)          K    dQ (x 1/sqrt d)
//   DK    keys     K'  Q   V   dO   dS^T                                  Q    dK (x 1/sqrt d)
//   DV    keys     K'  Q   -   -    P^T                                   dO   dV
//
// Every tile of the forward is normalised by its own row maximum, so the element-wise threads carry no state;
// the threads that add the tiles up rescale by the running maximum.  Tiles, masks, score function and the
// reason why no accumulator outlives a tile are those of attention_mod_tc.cu.
//
//   warp 0 TMA; warps 1, 2, 3 issue X, Y, Out; warps 4-7, 8-11 the element-wise pass on alternate
//   tiles; warps 12-15 add the Out tiles: 128 columns of a row per thread, for which the other
//   warpgroups give up registers.
//   tensor memory: A1 hi 0-127, lo 128-255, Out tile 256-383, buffer b at 384 + 64 b: X -> Z_hi, Y -> Z_lo
//   shared memory: with A2 one buffer per stream; without, its 128 KB are two more stages of B1 and two of B3
// Waits are inlined: a call would hold a warpgroup to the registers of the callee.
// Two sequences of 1,000, 16 heads, prefix and cap: forward 66 us (tensor pipe 29 % busy), gradients 320 us (30 to 31 %).  256 blocks
// for 148 SMs are two rounds, and inside a block the chain X -> f -> Out of two tiles in flight is longer than its products.
#include "attention_mod.cuh"

namespace bt {

using namespace tc;
using namespace mod;

cudaError_t launch_attention_dvec(const float* o, const float* o_lo, const float* d_o, const float* d_o_lo, int B,
                                  int T, int C, int H, float* dvec, cudaStream_t s);

namespace {

constexpr int HD = 128, BR = 128, BT_ = 32, kThreads = 512;
constexpr uint32_t kRes = 4u * 2u * BR * 128u;     // 128 own rows: 4 k-blocks x (hi, lo) x 128 rows x 128 B
constexpr uint32_t kTile = 4u * 2u * BT_ * 128u;   // streamed tile: 4 blocks x (hi, lo) x 32 rows x 128 B
constexpr uint32_t kSmem = 1024u + kRes + 3u * kTile + 256u;
static_assert(kSmem <= 232448u, "shared memory");
// registers of a lane by warpgroup: issuing, element-wise (two), adding; the passes with Y issue more products
__host__ __device__ constexpr int regs_issue(bool y) { return y ? 80 : 64; }
__host__ __device__ constexpr int regs_element(bool y) { return y ? 104 : 112; }
constexpr int kRegsAdd = 208;
static_assert(regs_issue(true) + 2 * regs_element(true) + kRegsAdd <= 512 && regs_issue(false) + 2 * regs_element(false) + kRegsAdd <= 512,
              "registers: 512 threads get 128 each at launch");

enum Pass { P_FWD = 0, P_DQ = 1, P_DK = 2, P_DV = 3 };

struct Mod128Args {
    AttnModArgs a;
    const float* own;         // hi plane of the array the CTA's own rows (A1) come from, lo plane at own_lo
    const float* own_lo;
    int a1_col, a2_col, b1_col, b2_col, b3_col;   // column of head 0 in the arrays behind the operands
    float *out, *out_hi, *out_lo;
    long long out_stride;
    int out_col;
    float out_mul;
};

//  MN-major 32-row tile: 4 column groups of [hi | lo][32 rows][128 B]; a k-step is 8 rows
__device__ __forceinline__ constexpr uint32_t mn_off(int ks, bool lo) { return (lo ? BT_ * 128u : 0u) + (uint32_t)ks * 1024u; }

template <int PASS, bool CAP, bool SLOPE>
__global__ void __launch_bounds__(kThreads, 1)
attn_mod128_kernel(const __grid_constant__ CUtensorMap tmA2, const __grid_constant__ CUtensorMap tmB1,
                   const __grid_constant__ CUtensorMap tmB2, const __grid_constant__ CUtensorMap tmB3, const Mod128Args args) {
    constexpr bool kKeys = (PASS == P_DK || PASS == P_DV);    // own rows are keys, streamed rows queries
    constexpr bool kHasY = (PASS == P_DQ || PASS == P_DK);
    constexpr int S1 = kHasY ? 1 : 3, S3 = kHasY ? 1 : 2;     // stages of B1 and B3
    const AttnModArgs& g = args.a;

    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t a2_s = base, b1_s = base + kRes, b2_s = b1_s + kTile, b3_s = b2_s + kTile, bars = b3_s + kTile;
    enum { A2_FULL = 0, B1_FULL, B1_EMPTY = B1_FULL + 3, B2_FULL = B1_EMPTY + 3, B2_EMPTY, B3_FULL, B3_EMPTY = B3_FULL + 2,
           OUT_FULL = B3_EMPTY + 2, Z_DONE0, Z_DONE1, XY_FULL0, XY_FULL1, Z_READY0, Z_READY1, OUT_FREE, A1_READY, N_BARS };
    static_assert(8 * N_BARS + 4 <= 256, "barriers");
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    auto b1_stage = [&](int st) { return (kHasY || st == 0) ? b1_s : a2_s + (uint32_t)(st - 1) * kTile; };
    auto b3_stage = [&](int st) { return kHasY ? b3_s : a2_s + (uint32_t)(2 + st) * kTile; };
    const uint32_t tmem_slot = bars + 8u * N_BARS;
    auto smem_ptr = [&](uint32_t addr) { return smem_raw + (addr - smem_u32(smem_raw)); };
    // FWD: maximum and sum of each row's tile, four tiles deep ([4][2][128]).  It lies in the B2 buffer, which
    // this pass only uses to stage the own rows.
    float* tile_stat = reinterpret_cast<float*>(smem_ptr(b2_s));

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int bh = blockIdx.x, b = bh / g.H, h = bh % g.H;
    // causal walks: the longest first
    const int blk = kKeys ? (int)blockIdx.y : (int)gridDim.y - 1 - (int)blockIdx.y;
    const int r0 = blk * BR, row_base = b * g.T;

    if (threadIdx.x == 0) {
        for (int i = 0; i < N_BARS; ++i)
            mbar_init(bar(i), i == A1_READY ? 8 : i >= Z_READY0 ? 4 : (kHasY && (i == XY_FULL0 || i == XY_FULL1)) ? 2 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem_ptr(tmem_slot));
    pdl_wait();      // set-up done; global memory is touched from here on
    pdl_trigger();
    if ((PASS == P_FWD || PASS == P_DQ) && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *g.err = 0;
    const uint32_t tA1_hi = tmem, tA1_lo = tmem + 128, tOut = tmem + 256;
    auto tbuf = [&](int bb) { return tmem + 384u + 64u * (uint32_t)bb; };
    const int2 range = block_range(kKeys ? g.spans.qblock : g.spans.kblock, b, g.T, r0, BR, kKeys);
    const int t0 = range.x / BT_, n_t = range.x < range.y ? (range.y - 1) / BT_ + 1 - t0 : 0;

    if (warp < 4) {
        set_regs_down<regs_issue(kHasY)>();
        if (warp == 0 && lane == 0 && n_t > 0) {
            if (kHasY) {
                mbar_expect_tx(bar(A2_FULL), kRes);
                for (int kb = 0; kb < 4; ++kb)
                    tma_load_3d(a2_s + kb * (kRes / 4), &tmA2, bar(A2_FULL), args.a2_col + h * HD + kb * 32, row_base + r0, 0);
            }
            auto load = [&](uint32_t dst, const CUtensorMap* tm, int full, int empty, int col, int t, int stages) -> bool {
                const int st = t % stages;
                if (!mbar_wait(bar(empty + st), ((uint32_t)(t / stages) & 1u) ^ 1u, g.err, 171)) return false;
                mbar_expect_tx(bar(full + st), kTile);
                for (int part = 0; part < 4; ++part)
                    tma_load_3d(dst + part * (kTile / 4), tm, bar(full + st), col + h * HD + part * 32, row_base + (t0 + t) * BT_, 0);
                return true;
            };
            constexpr int kAhead = kHasY ? 1 : 2;           // B1 runs this many tiles ahead of B3
            bool ok = true;
            for (int t = 0; t < min(kAhead, n_t) && ok; ++t) ok = load(b1_stage(t % S1), &tmB1, B1_FULL, B1_EMPTY, args.b1_col, t, S1);
            if (kHasY) {
                // the B2 / B3 buffers first stage the own rows on their way into tensor memory
                if (ok) ok = mbar_wait(bar(A1_READY), 0, g.err, 172);
                if (ok) ok = load(b2_s, &tmB2, B2_FULL, B2_EMPTY, args.b2_col, 0, 1);
            }
            for (int t = 0; t < n_t && ok; ++t) {
                if (t + kAhead < n_t) ok = load(b1_stage((t + kAhead) % S1), &tmB1, B1_FULL, B1_EMPTY, args.b1_col, t + kAhead, S1);
                if (ok && kHasY && t + 1 < n_t) ok = load(b2_s, &tmB2, B2_FULL, B2_EMPTY, args.b2_col, t + 1, 1);
                if (ok) ok = load(b3_stage(t % S3), &tmB3, B3_FULL, B3_EMPTY, args.b3_col, t, S3);
            }
            if (!ok)
                for (int i = 0; i < 2000; ++i) __nanosleep(1000);   // let loads in flight land
        } else if (warp == 1 && n_t > 0) {
            // ---- X.  Without Y the 64 columns of a buffer are free: [B1_hi | B1_lo] is one operand of 64 rows, A1_lo B1_hi
            // joins the small half, and the reader adds the halves.  With Y: the small terms first.
            constexpr uint32_t idesc = make_idesc_tf32(BR, BT_, false, false), idesc2 = make_idesc_tf32(BR, 2 * BT_, false, false);
            bool ok = mbar_wait_warp(bar(A1_READY), 0, g.err, 173);
            for (int t = 0; t < n_t && ok; ++t) {
                const int st = t % S1;
                const uint32_t tX = tbuf(t & 1);
                if (!mbar_wait_warp(bar(B1_FULL + st), (uint32_t)(t / S1) & 1u, g.err, 175)) { ok = false; break; }
                // the Out product of tile t - 2 has read this buffer
                if (t >= 2 && !mbar_wait_warp(bar(Z_DONE0 + (t & 1)), (uint32_t)((t - 2) >> 1) & 1u, g.err, 176)) { ok = false; break; }
                tc_fence_after();
                const DescBase bd = kmaj_base(b1_stage(st));
                if (elect_one()) {
                if (kHasY) {
#pragma unroll
                    for (int ks = 0; ks < 16; ++ks) {
                        umma_tf32_ts(tX, tA1_lo + ks * 8, bd.at(kmaj_off(BT_, ks, false)), idesc, ks > 0 ? 1u : 0u);
                        umma_tf32_ts(tX, tA1_hi + ks * 8, bd.at(kmaj_off(BT_, ks, true)), idesc, 1u);
                    }
#pragma unroll
                    for (int ks = 0; ks < 16; ++ks) umma_tf32_ts(tX, tA1_hi + ks * 8, bd.at(kmaj_off(BT_, ks, false)), idesc, 1u);
                } else {
#pragma unroll
                    for (int ks = 0; ks < 16; ++ks) {
                        umma_tf32_ts(tX, tA1_hi + ks * 8, bd.at(kmaj_off(BT_, ks, false)), idesc2, ks > 0 ? 1u : 0u);
                        umma_tf32_ts(tX + 32u, tA1_lo + ks * 8, bd.at(kmaj_off(BT_, ks, false)), idesc, 1u);
                    }
                }
                umma_commit(bar(B1_EMPTY + st));
                umma_commit(bar(XY_FULL0 + (t & 1)));
                }
                __syncwarp();
            }
        } else if (kHasY && warp == 2 && n_t > 0) {
            constexpr uint32_t idesc = make_idesc_tf32(BR, BT_, false, false);
            bool ok = mbar_wait_warp(bar(A2_FULL), 0, g.err, 174);
            const DescBase ad = kmaj_base(a2_s), bd = kmaj_base(b2_s);
            for (int t = 0; t < n_t && ok; ++t) {
                const uint32_t tY = tbuf(t & 1) + 32u;
                if (!mbar_wait_warp(bar(B2_FULL), (uint32_t)t & 1u, g.err, 177)) { ok = false; break; }
                if (t >= 2 && !mbar_wait_warp(bar(Z_DONE0 + (t & 1)), (uint32_t)((t - 2) >> 1) & 1u, g.err, 178)) { ok = false; break; }
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                for (int ks = 0; ks < 16; ++ks) {
                    umma_tf32(tY, ad.at(kmaj_off(BR, ks, true)), bd.at(kmaj_off(BT_, ks, false)), idesc, ks > 0 ? 1u : 0u);
                    umma_tf32(tY, ad.at(kmaj_off(BR, ks, false)), bd.at(kmaj_off(BT_, ks, true)), idesc, 1u);
                }
#pragma unroll
                for (int ks = 0; ks < 16; ++ks)
                    umma_tf32(tY, ad.at(kmaj_off(BR, ks, false)), bd.at(kmaj_off(BT_, ks, false)), idesc, 1u);
                umma_commit(bar(B2_EMPTY));
                umma_commit(bar(XY_FULL0 + (t & 1)));
                }
                __syncwarp();
            }
        } else if (warp == 3 && n_t > 0) {
            // ---- Out_tile = Z B3, from zero, the small terms first
            constexpr uint32_t idesc = make_idesc_tf32(BR, HD, false, true);
            bool ok = true;
            for (int t = 0; t < n_t && ok; ++t) {
                const int st = t % S3;
                const uint32_t z_hi = tbuf(t & 1), z_lo = z_hi + 32u;
                if (!mbar_wait_warp(bar(Z_READY0 + (t & 1)), (uint32_t)(t >> 1) & 1u, g.err, 179)) { ok = false; break; }
                if (!mbar_wait_warp(bar(B3_FULL + st), (uint32_t)(t / S3) & 1u, g.err, 180)) { ok = false; break; }
                if (!mbar_wait_warp(bar(OUT_FREE), (uint32_t)t & 1u, g.err, 181)) { ok = false; break; }
                tc_fence_after();
                const DescBase bd = make_desc_base(b3_stage(st), 2u * BT_ * 128u, 512u, 1u);
                if (elect_one()) {
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) {
                    umma_tf32_ts(tOut, z_lo + ks * 8, bd.at(mn_off(ks, false)), idesc, ks > 0 ? 1u : 0u);
                    umma_tf32_ts(tOut, z_hi + ks * 8, bd.at(mn_off(ks, true)), idesc, 1u);
                }
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) umma_tf32_ts(tOut, z_hi + ks * 8, bd.at(mn_off(ks, false)), idesc, 1u);
                umma_commit(bar(B3_EMPTY + st));
                umma_commit(bar(Z_DONE0 + (t & 1)));
                umma_commit(bar(OUT_FULL));
                }
                __syncwarp();
            }
        }
    } else if (warp < 12) {
        // ---------------------------------------------------------------- element-wise warpgroups
        set_regs_down<regs_element(kHasY)>();
        const int wg = (warp - 4) >> 2, lane_group = warp & 3;
        const int rloc = lane_group * 32 + lane, own = r0 + rloc;
        const uint32_t t_lane = ((uint32_t)(lane_group * 32) << 16);
        const int64_t lb = ((int64_t)b * g.H + h) * g.T;
        const Score sc = make_score<CAP, SLOPE>(1.0f / sqrtf((float)HD), g.cap, g.slopes, h);
        if (n_t > 0) {   // own rows -> tensor memory: warpgroup 0 takes columns 0-63, warpgroup 1 64-127
            const int wrow0 = min(r0 + lane_group * 32, g.T - 1);
            const long long stride = 3 * (long long)g.C, off = (long long)(row_base + wrow0) * stride + args.a1_col + h * HD + 64 * wg;
            float* tile = reinterpret_cast<float*>(smem_ptr(b2_s) + (uint32_t)(warp - 4) * kRowTileBytes);
            rows_to_tmem(args.own + off, args.own_lo + off, stride, max(1, min(32, g.T - wrow0)), sc.unit,
                         tA1_hi + t_lane + 64u * wg, tA1_lo + t_lane + 64u * wg, tile, lane);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the staging tiles are next written by TMA
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(A1_READY));
            // FWD: the staging tiles become tile_stat, written by both warpgroups
            if (PASS == P_FWD) asm volatile("bar.sync 1, 256;" ::: "memory");
        }
        const int2 span = row_range(kKeys ? g.spans.q : g.spans.k, b, g.T, own, kKeys);
        const int rc = min(own, g.T - 1);
        float L = 0.f, D = 0.f;                           // DQ: this row's statistics
        if (PASS == P_DQ) {
            L = g.lse[lb + rc] * kLog2e;
            D = g.dvec[lb + rc];
        }
        const uint32_t tb = tbuf(wg) + t_lane;
        bool ok = true;
        for (int t = wg; t < n_t && ok; t += 2) {
            const int s0 = (t0 + t) * BT_;                // first streamed row of the tile
            float Lq = 0.f, Dq = 0.f;                     // DK, DV: query s0 + lane's statistics
            if (kKeys) {
                const int r = min(s0 + lane, g.T - 1);    // rows past the end are masked below
                Lq = __ldg(g.lse + lb + r) * kLog2e;
                if (PASS == P_DK) Dq = __ldg(g.dvec + lb + r);
            }
            if (!mbar_wait_warp(bar(XY_FULL0 + wg), (uint32_t)(t >> 1) & 1u, g.err, 182)) { ok = false; break; }
            tc_fence_after();
            const bool whole = s0 >= span.x && s0 + BT_ <= span.y;
            if (PASS == P_FWD) {
                // the reference from whole scores: the small half grows with them
                float top = -INFINITY, sum = 0.f;
#pragma unroll 1
                for (int q = 0; q < 32; q += 16) {
                    float z[16], none[16];
                    uint32_t hi[16], lo[16];
                    tmem_ldn(tb + q, hi);
                    tmem_ldn(tb + 32u + q, lo);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[i] = __uint_as_float(hi[i]) + __uint_as_float(lo[i]);
                    if (SLOPE) score_tile<CAP, SLOPE, false, false, 16>(z, none, sc, own - s0 - q, 0.f);   // else the maximum is at that of the product
                    const uint32_t bits = whole ? 0xffffu : column_bits<16>(span, s0 + q);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (bits >> i & 1u) top = fmaxf(top, z[i]);
                }
                const bool none_read = top == -INFINITY;                // every P of this tile is zero
                const float ref = none_read ? 0.f : (CAP && !SLOPE) ? sc.to_log2 * tanh_any(top) : top;
                const Reference rf = make_reference(ref, sc.slope2, abs(own - s0) + BT_);
#pragma unroll 1
                for (int q = 0; q < 32; q += 16) {
                    float z[16], none[16];
                    uint32_t hi[16], lo[16];
                    tmem_ldn(tb + q, hi);
                    tmem_ldn(tb + 32u + q, lo);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[i] = __uint_as_float(hi[i]) + __uint_as_float(lo[i]);
                    score_tile<CAP, SLOPE, false, false, 16>(z, none, sc, own - s0 - q, rf.now);
                    less_reference(z, rf);
                    const uint32_t bits = whole ? 0xffffu : column_bits<16>(span, s0 + q);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float p = (bits >> i & 1u) ? ex2_approx(z[i]) : 0.f;
                        sum += p;
                        split_tf32_int(p, hi[i], lo[i]);
                    }
                    tmem_stn(tb + q, hi);
                    tmem_stn(tb + 32u + q, lo);
                }
                tile_stat[(t & 3) * 256 + rloc] = none_read ? -INFINITY : ref;
                tile_stat[(t & 3) * 256 + 128 + rloc] = sum;
                __threadfence_block();
            } else {
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    const int sh = s0 + 16 * half;
                    float x[16], f[16];
                    uint32_t r[16], y[16];
                    tmem_ldn(tb + 16u * half, r);
                    tmem_ldn(tb + 32u + 16u * half, y);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = kHasY ? __uint_as_float(r[i]) : __uint_as_float(r[i]) + __uint_as_float(y[i]);
                    score_tile<CAP, SLOPE, true, false, 16>(x, f, sc, own - sh, kKeys ? 0.f : L);
                    const uint32_t bits = whole ? 0xffffu : column_bits<16>(span, sh);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float a = kKeys ? x[i] - __shfl_sync(0xffffffffu, Lq, 16 * half + i) : x[i];
                        float z = (bits >> i & 1u) ? ex2_approx(a) : 0.f;
                        if (kHasY) {
                            z *= __uint_as_float(y[i]) - (PASS == P_DK ? __shfl_sync(0xffffffffu, Dq, 16 * half + i) : D);
                            if (CAP) z *= f[i];
                        }
                        split_tf32_int(z, r[i], y[i]);
                    }
                    tmem_stn(tb + 16u * half, r);            // Z hi over X
                    tmem_stn(tb + 32u + 16u * half, y);      // Z lo over Y
                }
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(Z_READY0 + wg));
        }
    } else {
        // ---------------------------------------------------------------- the warpgroup that adds the tiles
        set_regs_up<kRegsAdd>();
        const int lane_group = warp & 3, rloc = lane_group * 32 + lane;
        const uint32_t t_row = tOut + ((uint32_t)(lane_group * 32) << 16);
        float acc[4][32];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[q][i] = 0.f;
        float m = -INFINITY, l = 0.f;                     // FWD: running maximum and sum of the row
        // OUT_FREE phase t lets Out(t) be issued: tile t - 1 has been read and, in the forward, the wait for Z_READY(t)
        // is over (it could otherwise be overtaken by two phases).
        auto release = [&](int t) -> bool {
            if (PASS == P_FWD && t < n_t && !mbar_wait_warp(bar(Z_READY0 + (t & 1)), (uint32_t)(t >> 1) & 1u, g.err, 183)) return false;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(OUT_FREE));
            return true;
        };
        bool ok = release(0);
        for (int t = 0; t < n_t && ok; ++t) {
            float keep = 1.f, join = 1.f;
            if (PASS == P_FWD) {
                const float mt = tile_stat[(t & 3) * 256 + rloc], lt = tile_stat[(t & 3) * 256 + 128 + rloc];
                const float top = fmaxf(m, mt), use = top == -INFINITY ? 0.f : top;
                keep = ex2_approx(m - use);
                join = ex2_approx(mt - use);
                l = l * keep + lt * join;
                m = top;
            }
            if (!mbar_wait_warp(bar(OUT_FULL), (uint32_t)t & 1u, g.err, 184)) { ok = false; break; }
            tc_fence_after();
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t r[32];
                tmem_ld32(t_row + 32u * q, r);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    acc[q][i] = PASS == P_FWD ? fmaf(acc[q][i], keep, __uint_as_float(r[i]) * join) : acc[q][i] + __uint_as_float(r[i]);
            }
            ok = release(t + 1);
        }
        if (ok) {
            // every product has completed: the stream buffers are idle
            const int wrow0 = r0 + lane_group * 32, nvalid = max(0, min(32, g.T - wrow0));
            const long long off = (long long)(row_base + wrow0) * args.out_stride + args.out_col + h * HD;
            float* tile = reinterpret_cast<float*>(smem_ptr(b1_s) + (uint32_t)lane_group * kRowTileBytes);
            const int2 span = PASS == P_FWD && l == 0.f ? row_range(g.spans.k, b, g.T, r0 + rloc, false) : make_int2(0, 0);
            const float mul = PASS == P_FWD ? row_factor(l, span) : args.out_mul;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
#pragma unroll
                for (int i = 0; i < 32; ++i) acc[q][i] *= mul;
                warp_rows_store(acc[q], tile, lane, nvalid, args.out ? args.out + off + 32 * q : nullptr,
                                args.out_hi ? args.out_hi + off + 32 * q : nullptr, args.out_hi ? args.out_lo + off + 32 * q : nullptr,
                                args.out_stride, nullptr);
            }
            if (PASS == P_FWD && r0 + rloc < g.T)
                g.lse[((int64_t)b * g.H + h) * g.T + r0 + rloc] = row_lse(m, l, span);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

template <int PASS>
cudaError_t launch_pass(const CUtensorMap& a2, const CUtensorMap& b1, const CUtensorMap& b2, const CUtensorMap& b3,
                        const Mod128Args& args, cudaStream_t s) {
    const AttnModArgs& g = args.a;
    const dim3 grid(g.B * g.H, (g.T + BR - 1) / BR);
    BT_FOR_MOD(g, {
        const cudaError_t e = allow_smem<attn_mod128_kernel<PASS, kCap, kSlope>>(kSmem);
        if (e != cudaSuccess) return e;
        BT_KERNEL_LAUNCH((attn_mod128_kernel<PASS, kCap, kSlope>), grid, kThreads, kSmem, s, a2, b1, b2, b3, args);
    });
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_mod_fwd_tc128(const AttnModArgs& g, cudaStream_t s) {
    const int64_t rows = (int64_t)g.B * g.T, cols = 3 * (int64_t)g.C;
    CUtensorMap k, v;
    if (!plane_map(&k, g.qkv, cols, rows, BT_, false) || !plane_map(&v, g.qkv, cols, rows, BT_, true)) return cudaErrorInvalidValue;
    Mod128Args a{};
    a.a = g;
    a.own = g.qkv; a.own_lo = g.qkv_lo;
    a.b1_col = g.C; a.b3_col = 2 * g.C;
    a.out = g.o; a.out_hi = g.o_hi; a.out_lo = g.o_lo; a.out_stride = g.C; a.out_mul = 1.0f;
    return launch_pass<P_FWD>(k, k, k, v, a, s);
}

cudaError_t launch_attention_mod_bwd_tc128(const AttnModArgs& g, cudaStream_t s) {
    cudaError_t e = launch_attention_dvec(g.o, nullptr, g.d_o, g.d_o_lo, g.B, g.T, g.C, g.H, g.dvec, s);
    if (e != cudaSuccess) return e;
    const int64_t rows = (int64_t)g.B * g.T, cols = 3 * (int64_t)g.C;
    CUtensorMap qkv_k, qkv_m, qkv_res, do_k, do_m, do_res;
    if (!plane_map(&qkv_k, g.qkv, cols, rows, BT_, false) || !plane_map(&qkv_m, g.qkv, cols, rows, BT_, true) ||
        !plane_map(&qkv_res, g.qkv, cols, rows, BR, false) || !plane_map(&do_k, g.d_o, g.C, rows, BT_, false) ||
        !plane_map(&do_m, g.d_o, g.C, rows, BT_, true) || !plane_map(&do_res, g.d_o, g.C, rows, BR, false))
        return cudaErrorInvalidValue;
    Mod128Args a{};
    a.a = g;
    a.own = g.qkv; a.own_lo = g.qkv_lo;
    a.out = g.dqkv; a.out_hi = g.dqkv_hi; a.out_lo = g.dqkv_lo; a.out_stride = cols;
    const float scale = 1.0f / sqrtf((float)HD);
    a.a1_col = 0; a.a2_col = 0; a.b1_col = g.C; a.b2_col = 2 * g.C; a.b3_col = g.C; a.out_col = 0; a.out_mul = scale;
    if ((e = launch_pass<P_DQ>(do_res, qkv_k, qkv_k, qkv_m, a, s)) != cudaSuccess) return e;
    a.a1_col = g.C; a.a2_col = 2 * g.C; a.b1_col = 0; a.b2_col = 0; a.b3_col = 0; a.out_col = g.C;
    if ((e = launch_pass<P_DK>(qkv_res, qkv_k, do_k, qkv_m, a, s)) != cudaSuccess) return e;
    a.out_col = 2 * g.C; a.out_mul = 1.0f;
    return launch_pass<P_DV>(qkv_res, qkv_k, do_k, do_m, a, s);
}

}  // namespace bt
