// Losses at the language-model head without the logits.
//
//     z_nv = x_n . W_v / tau,   lse_n = log sum_v exp z_nv,   q_nv = exp(z_nv - lse_n)
//     cross entropy (tau = 1):  loss_n = lse_n - z_{n, y_n}
//     distillation:             loss_n = tau^2 sum_k p_nk (log p_nk - z_{n, i_nk} + lse_n)
//     both:                     dz_nv = g_n (q_nv - a_nv),   dx = dz W,   dW = dz^T x
// where a_nv is the row's aim (1 at the target; the sum of p_nk / S_n over the entries with i_nk = v, S_n = sum_k p_nk) and
// g_n = inv_count w_n tau S_n.  The forward keeps one (maximum, sum) pair per row and strip of the vocabulary, joined
// by the finish kernels, and the few scores that the loss needs by themselves; the backward forms z again.
//
// Up to four rows, or eight (see few_rows), go through head_rows.cu in plain FP32, where the weights are read once; up to 128 through head_direct.cu, where the
// products with W (z, dx) read it as it is and make pairs of FP16 numbers on the way to the tensor cores; more rows to head_tc.cu,
// after kernels here have made such pairs of all of x and W.  dW of more than eight rows is head_tc.cu's.
#include <climits>

#include "head.cuh"

namespace bt {

namespace {

// The backward's look at the rows and at the largest of W, on CTAs of 256 threads; on 64 for rows of a teacher's entries that would not
// all be under way at once.  All gradients of 6,545 rows of 64 values, V 7,270, with 53 entries 221 us, on 256 threads 268; of 5,320 rows
// of 192 with targets, V 1,880, 111 on 256 and 126 on 64.
__host__ __device__ constexpr int row_threads(int64_t N, int K) { return N <= 1184 || K == 0 ? 256 : 64; }
__host__ __device__ constexpr int w_parts(int64_t N, int K) { return 592 * 256 / row_threads(N, K); }      // CTAs that look for the largest of W
__host__ __device__ constexpr int row_ctas(int64_t N, int K) {                                              // and those that look at the rows
    return N < 1184 * 256 / row_threads(N, K) ? (int)N : 1184 * 256 / row_threads(N, K);
}
__host__ __device__ inline int entries_of(const HeadArgs& g) { return g.aim.targets ? 0 : g.aim.K; }
constexpr int kThreads = 256;
constexpr int kFinishThreads = 256;

// Powers of two of the FP16 pairs: W and y are held times 2^kw and 2^ky.
struct Scales {
    float dx, dw;                           // from accumulators of u W and u^T y to the results
};

struct Scratch {
    HeadHeader* head;
    float2* stats;                          // forward: [N][strips]
    float* colf;                            // forward, tensor cores: [V] up to a multiple of 256
    int2* entries;                          // [N][K]
    uint32_t* spans;                        // [N][strips]
    float* zk;                              // [N] scores of the targets, or of a teacher's entries: [N][K], few rows [V][kFewRows]
    RowParams* rows;                        // backward: [N]
    int* eid;                               // [N][K] columns of the aim, each once; below zero: none
    float* ep;                              // [N][K] its weights there
    // few rows
    float* aim;                             // [V][kFewRows]
    float* dx_part;                         // [parts][kFewRows][C]
    // tensor cores
    Scales* scales;
    float *wpart, *ypart;                   // [w_parts(N, K)], [row_ctas(N, K)] largest values
    float* rowf;                            // [N]
    __half *x16, *y16, *w16, *u16;          // pairs: [2][N][C], [2][N][C], [2][V][C], [2][N][ldu]
    float* partials;
};

// Rows up to which the plain kernels are used, on the same inputs as the tensor cores from W as it is.  Forward: 3 rows against 50,257 x
// 768 35 us and 40, 5 rows 44 and 40, but against 9,000 x 2,048, too few rows of W for a tile to every SM, 27 and 32.  Backward: as
// long as one launch carries them (8 rows against 50,257 x 768 105 us and 122, against 5,000 x 4,096 in two launches 129 and 103).
bool few_rows(int64_t N, int C, int V, bool back) {
    return N <= kFewRows && (back ? N <= head_few_at_once(C) : N <= 4 || V < 148 * 128);
}

// Columns of one piece of the vocabulary, a multiple of 256: pieces of about the same size, of at most `piece` columns (or as many
// as u has in 512 MB) rounded up to the next 256.  u takes 4 N bytes per column, so 1,024 N at least: 1 GB from 2^20 rows on.
int piece_columns(int64_t N, int V, int piece) {
    int64_t most = piece > 0 ? piece : ((int64_t)1 << 27) / N;
    most = most < 256 ? 256 : (most + 255) / 256 * 256;
    const int64_t pieces = (V + most - 1) / most;
    return (int)(((V + pieces - 1) / pieces + 255) / 256 * 256);
}

template <typename T>
T* take(uint8_t* base, size_t& at, size_t n) {
    T* p = (T*)(base + at);
    at += head_pad(n * sizeof(T));
    return p;
}

void tc_layout(Scratch& s, uint8_t* base, size_t& at, int64_t N, int C, int V) {
    s.scales = take<Scales>(base, at, 1);
    s.rowf = take<float>(base, at, N);
    s.x16 = take<__half>(base, at, 2 * (size_t)N * C);
    if (V) s.w16 = take<__half>(base, at, 2 * (size_t)V * C);
}

// Which kernels form the forward's statistics: plain FP32, tensor cores straight from W, or from pairs of all of W.
enum Forward { kFew, kDirect, kPairs };
Forward forward_of(int64_t N, int C, int V) { return few_rows(N, C, V, false) ? kFew : head_direct_fits(N) ? kDirect : kPairs; }
int strips_of(int64_t N, int C, int V) {
    const Forward f = forward_of(N, C, V);
    return f == kFew ? head_few_strips(N, C, V) : f == kDirect ? head_direct_strips(C, V) : head_stats_strips(N, C, V).count;
}

// Those that a teacher's entries are sorted into.
HeadStrips entry_strips(int64_t N, int C, int V) {
    return forward_of(N, C, V) == kDirect ? head_direct_entry_strips(V) : head_stats_strips(N, C, V);
}

size_t fwd_layout(Scratch& s, uint8_t* base, int64_t N, int C, int V, int K) {
    size_t at = kHeadHeader;
    const Forward f = forward_of(N, C, V);
    s = Scratch{};
    s.head = (HeadHeader*)base;
    s.stats = take<float2>(base, at, (size_t)N * strips_of(N, C, V));
    s.zk = take<float>(base, at, K == 0 ? (size_t)N : f == kFew ? (size_t)V * kFewRows : (size_t)N * K);
    if (f == kFew) return at;
    tc_layout(s, base, at, N, C, f == kDirect ? 0 : V);
    if (f == kPairs) s.colf = take<float>(base, at, (V + 255) / 256 * 256);
    s.entries = take<int2>(base, at, (size_t)N * K);
    if (K) s.spans = take<uint32_t>(base, at, (size_t)N * entry_strips(N, C, V).count);
    return at;
}

size_t bwd_layout(Scratch& s, uint8_t* base, int64_t N, int C, int V, int K, int piece) {
    size_t at = kHeadHeader;
    s = Scratch{};
    s.head = (HeadHeader*)base;
    s.rows = take<RowParams>(base, at, N);
    s.eid = take<int>(base, at, (size_t)N * K);
    s.ep = take<float>(base, at, (size_t)N * K);
    if (few_rows(N, C, V, true)) {
        if (K) s.aim = take<float>(base, at, (size_t)V * kFewRows);
        s.dx_part = take<float>(base, at, (size_t)head_few_strips(N, C, V) * kFewRows * C);
        return at;
    }
    const bool direct = head_direct_fits(N);
    tc_layout(s, base, at, N, C, direct ? 0 : V);
    if (!direct) s.wpart = take<float>(base, at, w_parts(N, K));
    s.ypart = take<float>(base, at, row_ctas(N, K));
    s.y16 = take<__half>(base, at, 2 * (size_t)N * C);
    s.u16 = take<__half>(base, at, 2 * (size_t)N * piece_columns(N, V, piece));
    s.partials = take<float>(base, at, head_partial_bytes() / sizeof(float));
    return at;
}

__device__ __forceinline__ float4 ld_value(const float* hi, const float* lo, int64_t i4) {
    const float4 a = ld4(hi, i4);
    return lo ? add4(a, ld4(lo, i4)) : a;
}

// The sum of a row's exponentials: 2^m s.
struct RowSum {
    float m, s;
};
__device__ __forceinline__ float lse_of(RowSum r) { return (r.m + log2f(r.s)) * kLn2; }
// How far log sum exp lies above a score z (in units of log 2) that is part of the sum.  m is such a score too, and s the sum beside it:
// where z is the largest, m - z is an exact zero and s a number from 1 on.  The straight path's m may lie below the largest score, by 20 at
// most; the sum is then formed beside z.
__device__ __forceinline__ float above_score(RowSum r, float z) { return (z > r.m ? log2f(r.s * ex2_fast(r.m - z)) : r.m - z + log2f(r.s)) * kLn2; }

// A row's sum from its strips, by one warp or all (WARPS) of a CTA.
template <int WARPS>
__device__ __forceinline__ RowSum row_sum(const float2* st, int strips, float* sm) {
    float m = -INFINITY, s = 0.f;
#pragma unroll 4
    for (int i = WARPS == 1 ? threadIdx.x & 31 : threadIdx.x; i < strips; i += 32 * WARPS) {
        const float2 p = st[i];
        if (p.y != 0.f) {                   // a strip without columns has the sum zero
            const float m1 = fmaxf(m, p.x);
            s = s * ex2_fast(m - m1) + p.y * ex2_fast(p.x - m1);
            m = m1;
        }
    }
    const float top = WARPS == 1 ? warp_max(m) : block_all<32 * WARPS>(m, sm, MaxOp()), t = s != 0.f ? s * ex2_fast(m - top) : 0.f;
    return RowSum{top, WARPS == 1 ? warp_sum(t) : block_all<32 * WARPS>(t, sm, SumOp())};
}

// The loss against targets, a row per warp, or per CTA where there are few rows of many strips (100 rows of 592: 7.4 us, by a
// warp each 9.4; 8,192 rows of 394 37 us so, most of it barriers, and 19 by a warp each).
template <int WARPS>
__global__ void __launch_bounds__(kFinishThreads) head_finish_target_kernel(const HeadArgs g, const float2* __restrict__ stats, int strips,
                                                                            const float* __restrict__ zk, HeadHeader* head) {
    __shared__ double smd[kFinishThreads / 32];
    __shared__ float smf[kFinishThreads / 32];
    pdl_wait();
    pdl_trigger();
    const int64_t row = WARPS == 1 ? blockIdx.x * (int64_t)(kFinishThreads / 32) + (threadIdx.x >> 5) : blockIdx.x;
    const int lane = WARPS == 1 ? threadIdx.x & 31 : threadIdx.x;
    if (row < g.N) {
        int t = g.aim.targets[row];
        if (t >= g.V) {
            if (g.bad && lane == 0) atomicCAS(g.bad, 0, (int)row + 1);
            t = 0;
        }
        const RowSum r = row_sum<WARPS>(stats + row * strips, strips, smf);
        if (lane == 0) {
            if (g.lse) g.lse[row] = lse_of(r);
            const float loss = t >= 0 ? above_score(r, zk[row]) : 0.f;
            g.losses[row] = loss < 0.f ? 0.f : loss;           // exponentials rounded: 2^-21 below zero at most
        }
    }
    if (g.loss_mean) mean_by_last<kFinishThreads>(g.aim, g.losses, g.N, &head->rows_done, gridDim.x, g.loss_mean, smd);
}

// Up to some dozens of rows against a teacher, one per CTA.
template <bool FEW>
__global__ void __launch_bounds__(kFinishThreads) head_finish_kernel(const HeadArgs g, const float2* __restrict__ stats, int strips,
                                                                     const float* __restrict__ zk, HeadHeader* head) {
    __shared__ float smf[kFinishThreads / 32];
    __shared__ double smd[kFinishThreads / 32];
    pdl_wait();
    pdl_trigger();
    const int64_t row = blockIdx.x;
    const RowSum r = row_sum<kFinishThreads / 32>(stats + row * strips, strips, smf);
    bool any;
    const TeacherNorm norm = teacher_norm<kFinishThreads>(g.aim, row, g.V, g.bad, smf, any);
    float t = 0.f;
    for (int k = threadIdx.x; any && k < g.aim.K; k += kFinishThreads) {
        int id;
        const float lp = log_weight(entry_logit(g.aim, row, k, g.V, nullptr, id), norm), p = expf(lp);
        // NaN is not zero: such a row has no finite loss.  Where the norm is NaN, so is p of an entry that is not there
        if (id >= 0 && p != 0.f) t += p * (lp + above_score(r, zk[FEW ? (int64_t)id * kFewRows + row : row * g.aim.K + k]));
    }
    const float loss = block_all<kFinishThreads>(t, smf, SumOp()) * (g.aim.tau * g.aim.tau);
    if (threadIdx.x == 0) {
        if (g.lse) g.lse[row] = lse_of(r);
        g.losses[row] = loss;
    }
    if (g.loss_mean) mean_by_last<kFinishThreads>(g.aim, g.losses, g.N, &head->rows_done, gridDim.x, g.loss_mean, smd);
}

// More rows, one per warp.
__global__ void __launch_bounds__(kFinishThreads) head_finish_entries_kernel(const HeadArgs g, const float2* __restrict__ stats, int strips,
                                                                             const float* __restrict__ zk, HeadHeader* head) {
    __shared__ double smd[kFinishThreads / 32];
    pdl_wait();
    pdl_trigger();
    const int64_t row = blockIdx.x * (int64_t)(kFinishThreads / 32) + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (row < g.N) {
        const LossAim& a = g.aim;
        const RowSum r = row_sum<1>(stats + row * strips, strips, nullptr);
        float top = -INFINITY, sum = 0.f, loss = 0.f;
        int id;
        bool any = false;
        for (int k = lane; k < a.K; k += 32) {
            const float t = entry_logit(a, row, k, g.V, nullptr, id);
            any |= t != -INFINITY;          // a logit that is not a number counts: the row then has no finite loss
            top = fmaxf(top, t);
        }
        any = __any_sync(0xffffffffu, any);
        if (any) {
            top = warp_max(top);
            for (int k = lane; k < a.K; k += 32) sum += expf(entry_logit(a, row, k, g.V, nullptr, id) - top);
            const TeacherNorm norm = a.lse ? TeacherNorm{a.lse[row], 0.f} : TeacherNorm{top, logf(warp_sum(sum))};
            for (int k = lane; k < a.K; k += 32) {
                const float lp = log_weight(entry_logit(a, row, k, g.V, nullptr, id), norm), p = expf(lp);
                if (p != 0.f) loss += p * (lp + above_score(r, zk[row * a.K + k]));
            }
        }
        loss = warp_sum(loss) * (a.tau * a.tau);
        if (lane == 0) {
            if (g.lse) g.lse[row] = lse_of(r);
            g.losses[row] = loss;
        }
    }
    if (g.loss_mean) mean_by_last<kFinishThreads>(g.aim, g.losses, g.N, &head->rows_done, gridDim.x, g.loss_mean, smd);
}

// Planes: the hi plane stands for the value, whose largest it bounds within 2^-11 of itself.
__device__ __forceinline__ float max4(float m, float4 v) {
    return fmaxf(fmaxf(m, fmaxf(fabsf(v.x), fabsf(v.y))), fmaxf(fabsf(v.z), fabsf(v.w)));
}

// What the backward needs to know of the rows, one at a time per CTA, and the largest values of W and of y_nc = g_n x_nc.  Entries with the same id are joined into the first of them.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) head_rows_kernel(const HeadArgs g, RowParams* rows, int* eid, float* ep,
                                                                   float* wpart, float* ypart, HeadHeader* head) {
    extern __shared__ int ids[];            // [K], then the weights [K] and id_places(K)
    __shared__ float smf[THREADS / 32];
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && threadIdx.x == 0) *head = HeadHeader{0, 0u};
    const int w_ctas = wpart ? w_parts(g.N, entries_of(g)) : 0;
    if ((int)blockIdx.x < w_ctas) {         // the largest of W, a part per CTA
        const int64_t n4 = (int64_t)g.V * (g.C / 4), step = (int64_t)w_ctas * THREADS;
        float m = 0.f;
#pragma unroll 8
        for (int64_t i = blockIdx.x * (int64_t)THREADS + threadIdx.x; i < n4; i += step) m = max4(m, ld4(g.w, i));
        m = block_all<THREADS>(m, smf, MaxOp());
        if (threadIdx.x == 0) wpart[blockIdx.x] = m;
        return;
    }
    const int ctas = gridDim.x - w_ctas;
    float ymax = 0.f;
    for (int64_t row = blockIdx.x - w_ctas; row < g.N; row += ctas) {
        const LossAim& a = g.aim;
        RowParams r;
        const double L = (double)g.lse_in[row] * 1.4426950408889634;
        r.L = (float)L;
        r.L_rest = isfinite(r.L) ? (float)(L - (double)r.L) : 0.f;
        r.g = a.inv_count * row_weight(a, row) * a.tau;
        r.target = -1;
        bool live = r.g != 0.f;
        if (a.targets) {
            const int t = a.targets[row];
            live = live && t >= 0;
            r.target = t >= g.V ? 0 : t;
        } else {
            float* p = (float*)(ids + a.K);
            int* table = ids + 2 * a.K;
            const int places = id_places(a.K);
            for (int k = threadIdx.x; k < places; k += THREADS) table[k] = -1;
            bool any, twice = false;
            const TeacherNorm norm = teacher_norm<THREADS>(a, row, g.V, nullptr, smf, any);
            float sum = 0.f;
            for (int k = threadIdx.x; k < a.K; k += THREADS) {
                int id = -1;
                const float t = any ? entry_logit(a, row, k, g.V, nullptr, id) : -INFINITY;
                p[k] = any ? expf(log_weight(t, norm)) : 0.f;
                ids[k] = p[k] != 0.f ? id : -1;
                twice |= seen_before(table, places, a.K, ids[k]);
                sum += p[k];
            }
            twice = __syncthreads_or(twice);
            sum = block_all<THREADS>(sum, smf, SumOp());
            live = live && sum != 0.f;
            r.g *= sum;
            for (int k = threadIdx.x; k < a.K; k += THREADS) {
                const int id = ids[k];
                bool first = live && id >= 0;
                float w = twice ? 0.f : p[k];
                for (int j = 0; twice && first && j < a.K; ++j) {
                    if (ids[j] != id) continue;
                    if (j < k) first = false;
                    else w += p[j];
                }
                eid[row * a.K + k] = first ? id : -1;
                ep[row * a.K + k] = w / sum;
            }
        }
        if (!live) {
            r.L = INFINITY;
            r.L_rest = 0.f;
            r.g = 0.f;
            r.target = -1;
        }
        if (threadIdx.x == 0) rows[row] = r;
        if (ypart && live && r.g != 0.f) {      // the same for all threads
            float m = 0.f;
            for (int c = threadIdx.x; c < g.C / 4; c += THREADS) m = max4(m, ld4(g.x, row * (g.C / 4) + c));
            ymax = fmaxf(ymax, fabsf(r.g) * block_all<THREADS>(m, smf, MaxOp()));
        }
        __syncthreads();                        // the entries in shared memory have been read
    }
    if (ypart && threadIdx.x == 0) ypart[blockIdx.x - w_ctas] = ymax;
}

// ---------------------------------------------------------------- FP16 pairs

// Four values times s as pairs.
__device__ __forceinline__ void pairs4(float4 v, float s, uint2& hi, uint2& lo) {
    const float t[4] = {v.x * s, v.y * s, v.z * s, v.w * s};
    const __half2 a = __floats2half2_rn(t[0], t[1]), b = __floats2half2_rn(t[2], t[3]);
    const float2 fa = __half22float2(a), fb = __half22float2(b);
    const __half2 c = __floats2half2_rn(t[0] - fa.x, t[1] - fa.y), d = __floats2half2_rn(t[2] - fb.x, t[3] - fb.y);
    hi = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    lo = make_uint2(*reinterpret_cast<const uint32_t*>(&c), *reinterpret_cast<const uint32_t*>(&d));
}

// A row of C values as pairs at its own power of two, which it returns; by LANES neighbouring lanes.  Rows of up to 32 LANES values
// stay in registers between the search for the largest and the conversion.
template <int LANES>
__device__ __forceinline__ int row_to_pairs(const float* v, const float* v_lo, int64_t row, bool there, int C4, __half* out, int64_t plane4) {
    constexpr int kHeld = 8;
    const int lane = threadIdx.x % LANES;
    const bool held = C4 <= kHeld * LANES;
    float4 t[kHeld];
    float m = 0.f;
    if (held) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            t[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (there && lane + LANES * i < C4) t[i] = ld4(v, row * C4 + lane + LANES * i);
        }
        if (v_lo) {
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (there && lane + LANES * i < C4) t[i] = add4(t[i], ld4(v_lo, row * C4 + lane + LANES * i));
        }
#pragma unroll
        for (int i = 0; i < kHeld; ++i) m = max4(m, t[i]);
    } else if (there) {
        for (int c = lane; c < C4; c += LANES) m = max4(m, ld4(v, row * C4 + c));
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const int k = pair_exponent(m);
    const float s = pow2(k);
    auto put = [&](int c, float4 x) {
        uint2 h, l;
        pairs4(x, s, h, l);
        reinterpret_cast<uint2*>(out)[row * C4 + c] = h;
        reinterpret_cast<uint2*>(out)[plane4 + row * C4 + c] = l;
    };
    if (held) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (there && lane + LANES * i < C4) put(lane + LANES * i, t[i]);
    } else if (there) {
        for (int c = lane; c < C4; c += LANES) put(c, ld_value(v, v_lo, row * C4 + c));
    }
    return k;
}

// A teacher's entries of a row by ascending column, those that are not there behind all columns, and where each strip's begin.  A CTA
// sorts 512 entries at once, of several rows where they are shorter (3,740 rows of 101 one by one: 30 us).
constexpr int kSorted = 512;
__host__ __device__ inline int sorted_size(int K) {
    int n = 1;
    while (n < K) n *= 2;
    return n;
}
// Rows of a CTA: no more than leave four CTAs to an SM, whose threads search for the strips' first entries afterwards.
__host__ __device__ inline int rows_sorted(int64_t N, int K) {
    int rows = 1;
    while (2 * rows * sorted_size(K) <= kSorted && N / (2 * rows) >= 592) rows *= 2;
    return rows;
}
__device__ __forceinline__ void sort_entries(const HeadArgs& g, int2* entries, uint32_t* spans, HeadStrips strips, unsigned long long* key) {
    const LossAim& a = g.aim;
    const int n = sorted_size(a.K), rows = rows_sorted(g.N, a.K), all = n * rows;
    const int64_t row0 = blockIdx.x * (int64_t)rows;
    for (int i = threadIdx.x; i < all; i += kThreads) {
        const int k = i & (n - 1);
        const int64_t row = row0 + i / n;
        const int id = k < a.K && row < g.N ? entry_id(a, row, k, g.V, g.bad) : -1;
        key[i] = ((unsigned long long)(id < 0 ? INT_MAX : id) << 32) | (unsigned)k;
    }
    for (int size = 2; size <= n; size *= 2)
        for (int d = size / 2; d > 0; d /= 2) {
            __syncthreads();
            for (int i = threadIdx.x; i < all / 2; i += kThreads) {
                const int lo = 2 * i - (i & (d - 1)), hi = lo + d;
                const unsigned long long x = key[lo], y = key[hi];
                if ((x > y) == ((lo & (n - 1) & size) == 0)) {
                    key[lo] = y;
                    key[hi] = x;
                }
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < all; i += kThreads) {
        const int k = i & (n - 1);
        const int64_t row = row0 + i / n;
        if (k < a.K && row < g.N) entries[row * a.K + k] = make_int2((int)(key[i] >> 32), (int)(unsigned)key[i]);
    }
    for (int i = threadIdx.x; i < rows * (strips.count + 1); i += kThreads) {
        const int r = i / (strips.count + 1), t = i - r * (strips.count + 1);
        const int64_t row = row0 + r;
        if (row >= g.N) break;
        const unsigned long long from = (unsigned long long)t * strips.cols << 32, *own = key + r * n;
        int lo = 0, left = a.K;             // the first entry from there on
        while (left > 0) {
            const int h = left / 2;
            if (own[lo + h] < from) {
                lo += h + 1;
                left -= h + 1;
            } else {
                left = h;
            }
        }
        uint16_t* half = reinterpret_cast<uint16_t*>(spans + row * strips.count);       // where a strip's begin, those of the one before end
        if (t < strips.count) half[2 * t] = (uint16_t)lo;
        if (t > 0) half[2 * t - 1] = (uint16_t)lo;
    }
}

// Forward: the rows of W (the first w_rows) and x as pairs, each at its own power of two, which the epilogue takes out of its
// column or row; the first sort_ctas CTAs sort a teacher's entries meanwhile.  Planes of 16,384 + 2,048 rows of 768 take 39 us, 4.4 TB/s.
template <int LANES, bool SORT>
__global__ void __launch_bounds__(kThreads) head_row_pairs_kernel(const HeadArgs g, int64_t w_rows, const Scratch s, int sort_ctas,
                                                                    const HeadStrips strips) {
    __shared__ unsigned long long key[SORT ? kMaxEntries : 1];
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && threadIdx.x == 0) *s.head = HeadHeader{0, 0u};
    if (SORT && (int)blockIdx.x < sort_ctas) {
        sort_entries(g, s.entries, s.spans, strips, key);
        return;
    }
    const int C4 = g.C / 4;
    constexpr int kAtOnce = kThreads / LANES;
    // whole warps stay together: they share a base, and lanes whose row does not exist go along
    for (int64_t base = (blockIdx.x - sort_ctas) * (int64_t)kAtOnce; base < w_rows + g.N; base += (gridDim.x - sort_ctas) * (int64_t)kAtOnce) {
        const int64_t at = base + threadIdx.x / LANES;
        const bool of_w = at < w_rows, there = at < w_rows + g.N;
        const int64_t row = of_w ? at : at - w_rows;
        const int k = row_to_pairs<LANES>(of_w ? g.w : g.x, of_w ? g.w_lo : g.x_lo, row, there, C4, of_w ? s.w16 : s.x16, (of_w ? (int64_t)g.V : g.N) * C4);
        // 2^-k reaches 2^-126: the factor of a row of x is log2 e / tau 2^-k, a number of FP32 in any case
        if (there && threadIdx.x % LANES == 0) (of_w ? s.colf[row] : s.rowf[row]) = of_w ? ldexpf(1.0f, -k) : ldexpf(kLog2e / g.aim.tau, -k);
    }
}

// Backward: W and y at one power of two each, since they are summed over their rows, the rows of x each at its own.  The same planes 33 us.
__global__ void __launch_bounds__(kThreads) head_pairs_kernel(const HeadArgs g, const RowParams* __restrict__ rows, const Scratch s) {
    __shared__ float smf[kThreads / 32];
    pdl_wait();
    pdl_trigger();
    float m = 0.f, my = 0.f;
    for (int i = threadIdx.x; i < w_parts(g.N, entries_of(g)); i += kThreads) m = fmaxf(m, s.wpart[i]);
    for (int i = threadIdx.x; i < row_ctas(g.N, entries_of(g)); i += kThreads) my = fmaxf(my, s.ypart[i]);
    const int kw = pair_exponent(block_all<kThreads>(m, smf, MaxOp())), ky = pair_exponent(block_all<kThreads>(my, smf, MaxOp()));
    if (blockIdx.x == 0 && threadIdx.x == 0) *s.scales = Scales{ldexpf(1.0f, -15 - kw), ldexpf(1.0f, -15 - ky)};
    const int64_t n8 = (int64_t)g.V * g.C / 8, step = (int64_t)gridDim.x * kThreads;
    const float sw = pow2(kw), sy = pow2(ky);
#pragma unroll 4
    for (int64_t k = blockIdx.x * (int64_t)kThreads + threadIdx.x; k < n8; k += step) {
        const int64_t i = n8 - 1 - k;       // backwards: the end of W is what head_rows_kernel has left in L2
        uint2 h0, l0, h1, l1;
        pairs4(ld_value(g.w, g.w_lo, 2 * i), sw, h0, l0);
        pairs4(ld_value(g.w, g.w_lo, 2 * i + 1), sw, h1, l1);
        reinterpret_cast<uint4*>(s.w16)[i] = make_uint4(h0.x, h0.y, h1.x, h1.y);
        reinterpret_cast<uint4*>(s.w16)[n8 + i] = make_uint4(l0.x, l0.y, l1.x, l1.y);
    }
    const int C4 = g.C / 4, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t nx = g.N * C4;
    for (int64_t row = blockIdx.x * (int64_t)(kThreads / 32) + warp; row < g.N; row += gridDim.x * (int64_t)(kThreads / 32)) {
        const int kx = row_to_pairs<32>(g.x, g.x_lo, row, true, C4, s.x16, nx);
        const float gr = rows[row].g;
        for (int c = lane; c < C4; c += 32) {
            const float4 v = ld_value(g.x, g.x_lo, row * C4 + c);
            uint2 h, l;
            pairs4(make_float4(v.x * gr, v.y * gr, v.z * gr, v.w * gr), sy, h, l);
            if (gr == 0.f) h = l = make_uint2(0u, 0u);          // whatever the row holds
            reinterpret_cast<uint2*>(s.y16)[row * C4 + c] = h;
            reinterpret_cast<uint2*>(s.y16)[nx + row * C4 + c] = l;
        }
        // scores whose factor leaves this range are zero to FP32, or beyond it
        if (lane == 0) s.rowf[row] = ldexpf(kLog2e / g.aim.tau, max(-120, min(120, -kx - kw)));
    }
}

// The same without W, a row per CTA.
__global__ void __launch_bounds__(kThreads) head_pairs_of_rows_kernel(const HeadArgs g, const RowParams* __restrict__ rows, const Scratch s) {
    constexpr int kHeld = 4;                // C4 is at most 1,024
    __shared__ float smf[kThreads / 32];
    pdl_wait();
    pdl_trigger();
    const int64_t row = blockIdx.x;
    const int C4 = g.C / 4;
    float4 t[kHeld];
    float m = 0.f, my = 0.f;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        t[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (threadIdx.x + kThreads * i < C4) t[i] = ld_value(g.x, g.x_lo, row * C4 + threadIdx.x + kThreads * i);
        m = max4(m, t[i]);
    }
    for (int i = threadIdx.x; i < row_ctas(g.N, entries_of(g)); i += kThreads) my = fmaxf(my, s.ypart[i]);
    const int kx = pair_exponent(block_all<kThreads>(m, smf, MaxOp())), ky = pair_exponent(block_all<kThreads>(my, smf, MaxOp()));
    const float sx = pow2(kx), sy = pow2(ky), gr = rows[row].g;
    uint2 *const x = reinterpret_cast<uint2*>(s.x16) + row * C4, *const y = reinterpret_cast<uint2*>(s.y16) + row * C4;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int c = threadIdx.x + kThreads * i;
        if (c >= C4) continue;
        uint2 h, l;
        pairs4(t[i], sx, h, l);
        x[c] = h;
        x[g.N * C4 + c] = l;
        pairs4(make_float4(t[i].x * gr, t[i].y * gr, t[i].z * gr, t[i].w * gr), sy, h, l);
        if (gr == 0.f) h = l = make_uint2(0u, 0u);              // whatever the row holds
        y[c] = h;
        y[g.N * C4 + c] = l;
    }
    if (threadIdx.x > 0) return;
    s.rowf[row] = ldexpf(kLog2e / g.aim.tau, -kx);
    if (row == 0) *s.scales = Scales{0.f, ldexpf(1.0f, -15 - ky)};
}

// The teacher's part of a piece of u.
__global__ void __launch_bounds__(256) head_pair_entries_kernel(int64_t N, int K, const int* __restrict__ eid, const float* __restrict__ ep, int v0,
                                                                int cols, __half* u, int64_t ldu, int64_t plane) {
    pdl_wait();
    pdl_trigger();
    for (int64_t i = blockIdx.x * 256LL + threadIdx.x; i < N * K; i += gridDim.x * 256LL) {
        const int c = eid[i] - v0;
        if (eid[i] < 0 || c < 0 || c >= cols) continue;
        __half* p = u + i / K * ldu + c;
        const float t = (__half2float(p[0]) + __half2float(p[plane])) - 32768.0f * ep[i];
        p[0] = __float2half_rn(t);
        p[plane] = __float2half_rn(t - __half2float(p[0]));
    }
}

// Raw values at `hi` as planes.
__global__ void __launch_bounds__(256) head_planes_kernel(const float* x, float* hi, float* lo, int64_t n4) {
    pdl_wait();
    pdl_trigger();
    for (int64_t i = blockIdx.x * 256LL + threadIdx.x; i < n4; i += gridDim.x * 256LL) store_raw_split(ld4(x, i), nullptr, hi, lo, i);
}

int grid_for(int64_t threads, int most) {
    const int64_t n = (threads + 255) / 256;
    return (int)(n < 1 ? 1 : n < most ? n : most);
}

HalfMat pair_matrix(const __half* p, int64_t rows, int64_t cols) { return HalfMat{p, rows * cols, rows, cols, cols}; }

cudaError_t backward_in_pieces(const HeadArgs& g, const Scratch& w, int K, cudaStream_t s) {
    const bool direct = head_direct_fits(g.N);
    if (direct) BT_KERNEL_LAUNCH((head_pairs_of_rows_kernel), (unsigned)g.N, kThreads, 0, s, g, (const RowParams*)w.rows, w);
    else BT_KERNEL_LAUNCH((head_pairs_kernel), 148 * 8, kThreads, 0, s, g, (const RowParams*)w.rows, w);
    BT_COUNT_LAUNCH();
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const HalfMat x = pair_matrix(w.x16, g.N, g.C), y = pair_matrix(w.y16, g.N, g.C);
    const int ldu = piece_columns(g.N, g.V, g.piece);
    float* dx = g.dx ? g.dx : g.dx_hi;      // sums over the pieces go where the result will be
    for (int v0 = 0; v0 < g.V; v0 += ldu) {
        const int cols = g.V - v0 < ldu ? g.V - v0 : ldu;
        const HalfMat wp{w.w16 + (int64_t)v0 * g.C, (int64_t)g.V * g.C, cols, g.C, g.C}, u{w.u16, g.N * ldu, g.N, cols, ldu};
        e = direct ? launch_head_direct_grad(g, x, v0, cols, w.rowf, w.rows, w.u16, ldu, u.plane, &w.head->err, s)
                   : launch_head_grad(x, wp, v0, w.rowf, w.rows, w.u16, ldu, u.plane, &w.head->err, s);
        if (e == cudaSuccess && K) {
            BT_KERNEL_LAUNCH((head_pair_entries_kernel), grid_for(g.N * K, 148 * 8), 256, 0, s, g.N, K, (const int*)w.eid, (const float*)w.ep, v0,
                             cols, w.u16, (int64_t)ldu, u.plane);
            BT_COUNT_LAUNCH();
        }
        if (e == cudaSuccess && dx && direct) e = launch_head_direct_dx(g, u, v0, w.rows, v0 > 0, v0 + cols == g.V, w.partials, &w.head->err, s);
        else if (e == cudaSuccess && dx) e = launch_head_dx(u, wp, w.rows, &w.scales->dx, v0 > 0, dx, w.partials, &w.head->err, s);
        if (e == cudaSuccess && g.dw) e = launch_head_dw(u, y, &w.scales->dw, g.dw + (int64_t)v0 * g.C, w.partials, &w.head->err, s);
        if (e != cudaSuccess) return e;
    }
    if (g.dx_hi && !direct) {
        BT_KERNEL_LAUNCH((head_planes_kernel), grid_for(g.N * g.C / 4, 148 * 8), 256, 0, s, (const float*)dx, g.dx_hi, g.dx_lo, g.N * g.C / 4);
        BT_COUNT_LAUNCH();
    }
    return cudaGetLastError();
}

}  // namespace

size_t head_fwd_scratch_bytes(int64_t N, int C, int V, int K) {
    if (N < 1) return kHeadHeader;
    Scratch s;
    return fwd_layout(s, nullptr, N, C, V, K);
}

size_t head_bwd_scratch_bytes(int64_t N, int C, int V, int K, int piece) {
    if (N < 1) return kHeadHeader;
    Scratch s;
    return bwd_layout(s, nullptr, N, C, V, K, piece);
}

namespace {

template <int LANES>
cudaError_t launch_row_pairs_by(const HeadArgs& g, int64_t w_rows, const Scratch& w, cudaStream_t s) {
    const int K = entries_of(g), sort_ctas = K ? (int)((g.N + rows_sorted(g.N, K) - 1) / rows_sorted(g.N, K)) : 0;
    const int grid = sort_ctas + grid_for((w_rows + g.N) * LANES, 148 * 8);
    // the sort's shared memory, where there is none, keeps the next kernel's CTAs off the SM: 3 us
    if (sort_ctas) BT_KERNEL_LAUNCH((head_row_pairs_kernel<LANES, true>), grid, kThreads, 0, s, g, w_rows, w, sort_ctas, entry_strips(g.N, g.C, g.V));
    else BT_KERNEL_LAUNCH((head_row_pairs_kernel<LANES, false>), grid, kThreads, 0, s, g, w_rows, w, 0, HeadStrips{});
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}
// As few lanes to a row as hold it: many rows in flight.
cudaError_t launch_row_pairs(const HeadArgs& g, int64_t w_rows, const Scratch& w, cudaStream_t s) {
    return g.C <= 128   ? launch_row_pairs_by<4>(g, w_rows, w, s)
           : g.C <= 256 ? launch_row_pairs_by<8>(g, w_rows, w, s)
           : g.C <= 512 ? launch_row_pairs_by<16>(g, w_rows, w, s)
                        : launch_row_pairs_by<32>(g, w_rows, w, s);
}

}  // namespace

cudaError_t launch_head_fwd(const HeadArgs& g, cudaStream_t s) {
    Scratch w;
    const int K = entries_of(g);
    fwd_layout(w, g.scratch, g.N, g.C, g.V, K);
    const Forward f = forward_of(g.N, g.C, g.V);
    const int strips = strips_of(g.N, g.C, g.V);
    const HalfMat x = pair_matrix(w.x16, g.N, g.C);
    const HeadScores scores{g.aim.targets, K, w.entries, w.spans, w.zk};
    cudaError_t e = cudaSuccess;
    if (f == kFew) {
        e = launch_head_few_stats(g, w.stats, w.zk, w.head, s);
    } else if (f == kDirect) {
        e = launch_row_pairs(g, 0, w, s);
        if (e == cudaSuccess) e = launch_head_direct(g, x, w.rowf, scores, w.stats, &w.head->err, s);
    } else {
        e = launch_row_pairs(g, g.V, w, s);
        if (e == cudaSuccess)
            e = launch_head_stats(x, pair_matrix(w.w16, g.V, g.C), w.rowf, w.colf, scores, w.stats, &w.head->err, s);
    }
    if (e != cudaSuccess) return e;
    const unsigned ctas = (unsigned)((g.N + kFinishThreads / 32 - 1) / (kFinishThreads / 32));
    if (!K && g.N <= 148 * 8 && strips > 256)
        BT_KERNEL_LAUNCH((head_finish_target_kernel<kFinishThreads / 32>), (unsigned)g.N, kFinishThreads, 0, s, g, (const float2*)w.stats, strips, (const float*)w.zk,
                         w.head);
    else if (!K)
        BT_KERNEL_LAUNCH((head_finish_target_kernel<1>), ctas, kFinishThreads, 0, s, g, (const float2*)w.stats, strips, (const float*)w.zk, w.head);
    else if (f == kPairs)
        BT_KERNEL_LAUNCH((head_finish_entries_kernel), ctas, kFinishThreads, 0, s, g, (const float2*)w.stats, strips, (const float*)w.zk, w.head);
    else if (f == kFew)
        BT_KERNEL_LAUNCH((head_finish_kernel<true>), (unsigned)g.N, kFinishThreads, 0, s, g, (const float2*)w.stats, strips, (const float*)w.zk, w.head);
    else
        BT_KERNEL_LAUNCH((head_finish_kernel<false>), (unsigned)g.N, kFinishThreads, 0, s, g, (const float2*)w.stats, strips, (const float*)w.zk, w.head);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

cudaError_t launch_head_bwd(const HeadArgs& g, cudaStream_t s) {
    Scratch w;
    const int K = entries_of(g);
    bwd_layout(w, g.scratch, g.N, g.C, g.V, K, g.piece);
    const bool few = few_rows(g.N, g.C, g.V, true);
    const int ctas = row_ctas(g.N, K) + (w.wpart ? w_parts(g.N, K) : 0);
    const size_t smem = (size_t)(2 * K + id_places(K)) * 4;
    if (row_threads(g.N, K) == 64) BT_KERNEL_LAUNCH((head_rows_kernel<64>), ctas, 64, smem, s, g, w.rows, w.eid, w.ep, w.wpart, w.ypart, w.head);
    else BT_KERNEL_LAUNCH((head_rows_kernel<256>), ctas, 256, smem, s, g, w.rows, w.eid, w.ep, w.wpart, w.ypart, w.head);
    BT_COUNT_LAUNCH();
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    if (!few) return backward_in_pieces(g, w, K, s);
    return launch_head_few_grad(g, w.rows, K, w.eid, w.ep, w.aim, w.dx_part, s);
}

}  // namespace bt
