// Distillation from a teacher's top logits, on the student's logits: losses and gradient in one kernel.
//
//     z' = z / tau, q = softmax(z'), p_k = softmax_k(t_k / tau) (or exp(t_k / tau - lse))
//     loss = tau^2 sum_k p_k (log p_k - log q_{i_k}),   dz_v = g tau (S q_v - sum_{k: i_k = v} p_k),   S = sum_k p_k
//
// A CTA, or a cluster of up to eight with a slice of the columns each, walks over a row twice: once for its maximum and sum,
// once for the gradient, and the second walk reads what the first has left in L2, three quarters of it (1,184 rows: 300 MB read for 238).
// Holding the row in registers instead (one read, the next row on its way into shared memory) leaves no room for a second and third
// CTA per SM, whose loads run while this one reduces: 867 us against 681 at 8,192 x 50,257 when it was tried, where the copies
// alone take 502 (681 to 702 by the run, 4.7 TB/s; what is left is the latency of two walks).  The entries touch few columns: every
// thread stores its columns of g tau S q, and behind a barrier the threads that own an entry store the columns of the aim
// once more, from the logits that they have read before.
#include <cooperative_groups.h>

#include "head.cuh"

namespace bt {

namespace {

namespace cg = cooperative_groups;

constexpr int kBatch = 4;                   // float4 in flight per thread

struct Four {
    float a, b, c, d;
};

// Sums (MAX false: of a, b, c, d) or maxima (MAX: of a and b, sums of c) over the row's threads; two barriers.
template <int THREADS, int CS, bool MAX>
__device__ __forceinline__ Four row_all(Four v, Four* sm, Four* all) {
    auto join = [](Four x, Four y) {
        return MAX ? Four{fmaxf(x.a, y.a), fmaxf(x.b, y.b), x.c + y.c, 0.f} : Four{x.a + y.a, x.b + y.b, x.c + y.c, x.d + y.d};
    };
    auto fold = [&](Four x, int lanes) {
#pragma unroll
        for (int o = lanes / 2; o > 0; o >>= 1)
            x = join(x, Four{__shfl_xor_sync(0xffffffffu, x.a, o), __shfl_xor_sync(0xffffffffu, x.b, o), __shfl_xor_sync(0xffffffffu, x.c, o),
                             MAX ? 0.f : __shfl_xor_sync(0xffffffffu, x.d, o)});
        return x;
    };
    v = fold(v, 32);
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
    __syncthreads();
    Four r = fold(sm[threadIdx.x & (THREADS / 32 - 1)], THREADS / 32);     // the warps' values, once more in every warp
    if (CS == 1) {
        __syncthreads();
        return r;
    }
    cg::cluster_group c = cg::this_cluster();
    if (threadIdx.x < CS) *c.map_shared_rank(all + c.block_rank(), threadIdx.x) = r;
    c.sync();
    r = all[0];
#pragma unroll
    for (int k = 1; k < CS; ++k) r = join(r, all[k]);
    return r;
}

struct Entries {
    int id[kMaxEntries];                    // below zero: none
    float t[kMaxEntries], z[kMaxEntries];   // the teacher's logit, later its weight; the student's, in units of log 2 from the row's largest
};

template <int THREADS, int CS>
__global__ void __launch_bounds__(THREADS, 1536 / THREADS) distill_kernel(const DistillArgs g, int slice4, int mean_here) {
    __shared__ Four sm[2][THREADS / 32], all[2][CS];
    __shared__ Entries en;
    extern __shared__ int table[];                                  // [places]
    if (CS > 1) cg::this_cluster().barrier_arrive();                // waited for before the first store into another CTA's memory
    pdl_wait();
    pdl_trigger();
    const LossAim& a = g.aim;
    const int rank = CS > 1 ? (int)cg::this_cluster().block_rank() : 0;
    const int64_t row = blockIdx.x / CS;
    const int c0 = rank * slice4;                                   // columns in units of four
    const int n4 = min(slice4, (int)(g.ld / 4) - c0);               // columns that this CTA writes
    const int whole = max(0, min(n4, g.V / 4 - c0));                // and fours of them that lie inside the vocabulary
    const int rest = g.V / 4 - c0 >= 0 && g.V / 4 - c0 < n4 ? g.V & 3 : 0;      // columns behind those
    const float* z = g.z + row * g.ld + 4 * c0;
    const float4* z4 = reinterpret_cast<const float4*>(z);
    const float f = kLog2e / a.tau;

    const int places = id_places(a.K);
    for (int k = threadIdx.x; k < places; k += THREADS) table[k] = -1;      // row_all has a barrier before their use
    // the row's entries
    Four m{-INFINITY, -INFINITY, 0.f, 0.f};
#pragma unroll 1
    for (int k = threadIdx.x; k < a.K; k += THREADS) {
        int id;
        const float t = entry_logit(a, row, k, g.V, rank == 0 ? g.bad : nullptr, id);
        if (t == -INFINITY) id = -1;                                // a logit that is not a number counts
        en.id[k] = id;
        en.t[k] = t;
        if (id >= 0) en.z[k] = g.z[row * g.ld + id];                // before anything is written over it
        m.b = fmaxf(m.b, t);
        m.c += id >= 0 ? 1.f : 0.f;
    }
    // maximum and sum of exponentials of this thread's columns
    float s = 0.f;
    for (int i = threadIdx.x; i < whole; i += THREADS * kBatch) {
        float4 v[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (i + THREADS * k < whole) v[k] = z4[i + THREADS * k];
        float top = m.a;
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (i + THREADS * k < whole) top = fmaxf(top, fmaxf(fmaxf(v[k].x, v[k].y), fmaxf(v[k].z, v[k].w)));
        // columns of -inf alone leave the reference at zero: they add nothing to it
        const float ref = top == -INFINITY ? 0.f : top;
        s *= ex2_fast((m.a - ref) * f);
        m.a = top;
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (i + THREADS * k < whole)
                s += (ex2_fast((v[k].x - ref) * f) + ex2_fast((v[k].y - ref) * f)) + (ex2_fast((v[k].z - ref) * f) + ex2_fast((v[k].w - ref) * f));
    }
    if ((int)threadIdx.x < rest) {
        const float v = z[4 * whole + threadIdx.x], top = fmaxf(m.a, v), ref = top == -INFINITY ? 0.f : top;
        s = s * ex2_fast((m.a - ref) * f) + ex2_fast((v - ref) * f);
        m.a = top;
    }
    const float mine = m.a;
    if (CS > 1) cg::this_cluster().barrier_wait();                  // every CTA of the cluster has started, however short its slice
    m = row_all<THREADS, CS, true>(m, sm[0], all[0]);
    if (mine != m.a && s != 0.f) s *= ex2_fast((mine - m.a) * f);
    const bool any = m.c != 0.f;
    const float norm = !any ? 0.f : a.lse ? a.lse[row] : m.b;
    Four t{s, 0.f, 0.f, 0.f};
    bool twice = false;
#pragma unroll 1
    for (int k = threadIdx.x; k < a.K; k += THREADS) {
        const int id = en.id[k];
        const float lp = en.t[k] - norm, p = id >= 0 ? expf(lp) : 0.f;
        if (id >= 0) en.z[k] = (en.z[k] - m.a) * f;
        twice |= seen_before(table, places, a.K, id);
        if (p != 0.f && rank == 0) {
            t.b += p;
            t.c += p * (lp - en.z[k] * kLn2);
        }
        en.t[k] = p;                                                // only this thread has read it
    }
    t.d = twice ? 1.f : 0.f;
    t = row_all<THREADS, CS, false>(t, sm[1], all[1]);
    const float share = a.lse ? 1.f : any ? 1.0f / t.b : 0.f, S = a.lse ? t.b : any ? 1.f : 0.f;
    const float w = row_weight(a, row), G = a.inv_count * w * a.tau;
    if (rank == 0 && threadIdx.x == 0) {
        // sum_k p_k (log p_k + log sum exp - z_k), the teacher's normaliser taken out of the sum
        const float loss = !any || (a.lse && S == 0.f) ? 0.f : (a.lse ? t.c + S * logf(t.a) : t.c * share - logf(t.b) + logf(t.a)) * (a.tau * a.tau);
        g.losses[row] = loss;
        if (mean_here) *g.loss_mean = w != 0.f ? (float)((double)loss * (double)w * (double)a.inv_count) : 0.f;
    }
    if (g.dz || g.dz_hi) {
        const bool live = G != 0.f && S != 0.f;
        const float sc = G * S / t.a;
        const int64_t at = row * g.ld / 4 + c0;
        auto put4 = [&](int i, float4 d) {
            if (g.dz) __stcs(reinterpret_cast<float4*>(g.dz) + at + i, d);
            if (g.dz_hi) {
                float4 h, l;
                split_tf32(d, h, l);
                __stcs(reinterpret_cast<float4*>(g.dz_hi) + at + i, h);
                __stcs(reinterpret_cast<float4*>(g.dz_lo) + at + i, l);
            }
        };
        for (int i = threadIdx.x; i < whole; i += THREADS * kBatch) {
            float4 v[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                if (i + THREADS * k < whole) v[k] = __ldcs(z4 + i + THREADS * k);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (i + THREADS * k >= whole) continue;
                float4 d = make_float4(sc * ex2_fast((v[k].x - m.a) * f), sc * ex2_fast((v[k].y - m.a) * f),
                                       sc * ex2_fast((v[k].z - m.a) * f), sc * ex2_fast((v[k].w - m.a) * f));
                if (!live) d = make_float4(0.f, 0.f, 0.f, 0.f);
                put4(i + THREADS * k, d);
            }
        }
        // the last columns of the vocabulary, and those behind it
        for (int i = whole + threadIdx.x; i < n4; i += THREADS) {
            float d[4] = {0.f, 0.f, 0.f, 0.f};
            for (int j = 0; live && i == whole && j < rest; ++j) d[j] = sc * ex2_fast((z[4 * i + j] - m.a) * f);
            put4(i, make_float4(d[0], d[1], d[2], d[3]));
        }
        __syncthreads();
#pragma unroll 1
        for (int k = threadIdx.x; live && k < a.K; k += THREADS) {
            const int id = en.id[k];
            if (id < 4 * c0 || id >= 4 * (c0 + n4)) continue;       // none, or another CTA's column
            float sum = en.t[k];
            bool one = true;
            if (t.d != 0.f) {                                       // the first entry of an id takes all of its weight
                sum = 0.f;
                for (int j = 0; one && j < a.K; ++j) {
                    if (en.id[j] != id) continue;
                    if (j < k) one = false;
                    else sum += en.t[j];
                }
            }
            if (!one) continue;
            const float d = sc * ex2_fast(en.z[k]) - G * (sum * share);
            if (g.dz) g.dz[row * g.ld + id] = d;
            if (g.dz_hi) split_tf32(d, g.dz_hi[row * g.ld + id], g.dz_lo[row * g.ld + id]);
        }
    }
    if (CS > 1) cg::this_cluster().sync();                          // no CTA leaves while another may write to its memory
}

__global__ void __launch_bounds__(1024) weighted_mean_kernel(const float* __restrict__ losses, const LossAim a, int64_t N,
                                                             float* __restrict__ mean) {
    __shared__ double sm[32];
    pdl_wait();
    pdl_trigger();
    double t = 0.0;
#pragma unroll 8
    for (int64_t n = threadIdx.x; n < N; n += 1024) {
        const float w = row_weight(a, n);
        t += w != 0.f ? (double)losses[n] * (double)w : 0.0;
    }
    t = block_all<1024>(t, sm, SumOp());
    if (threadIdx.x == 0) *mean = (float)(t * (double)a.inv_count);
}

template <int THREADS, int CS>
cudaError_t launch_rows(const DistillArgs& g, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(g.N * CS));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = sizeof(int) * id_places(g.aim.K);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CS;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CS > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, distill_kernel<THREADS, CS>, g, (int)((g.ld / 4 + CS - 1) / CS), g.N == 1 && g.loss_mean ? 1 : 0);
}

}  // namespace

cudaError_t launch_softmax_distill(const DistillArgs& g, cudaStream_t s) {
    int dev = 0, sms = 148;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    const int64_t n4 = g.ld / 4;
    // CTAs per row: more while SMs would be idle and a thread keeps a batch, and while the rows that are walked over at the
    // same time (three CTAs per SM) would leave L2: 131,071 columns 123 us on pairs of CTAs, 149 with two CTAs per SM and longer batches
    int cs = 1;
    while (cs < 8 && ((g.N * cs * 2 <= 2 * sms && n4 > 512 * kBatch / 2 * cs) || 3 * sms / cs * n4 * 16 > ((int64_t)100 << 20))) cs *= 2;
    cudaError_t e;
    // short rows: more of them at a time on CTAs of 128 threads.  5,171 x 3,321 39 us against 81 on 512 threads, 8,000 x 8,000 105
    // against 148, 8,000 x 16,000 217 on 512 threads, 196 on 256, whose wide rows are slower (762 us against 717 at 50,257)
    if (cs == 1) e = n4 > 128 * 40 ? launch_rows<512, 1>(g, s) : n4 > 128 * 16 ? launch_rows<256, 1>(g, s) : launch_rows<128, 1>(g, s);
    else e = cs == 2 ? launch_rows<512, 2>(g, s) : cs == 4 ? launch_rows<512, 4>(g, s) : launch_rows<512, 8>(g, s);
    if (e != cudaSuccess) return e;
    BT_COUNT_LAUNCH();
    if (g.loss_mean && g.N > 1) {
        BT_KERNEL_LAUNCH((weighted_mean_kernel), 1, 1024, 0, s, (const float*)g.losses, g.aim, g.N, g.loss_mean);
        BT_COUNT_LAUNCH();
    }
    return cudaGetLastError();
}

}  // namespace bt
