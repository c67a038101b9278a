// Distillation from a teacher's top logits, on the student's logits: losses and gradient in one kernel.
//
//     z' = z / tau, q = softmax(z'), p_k = softmax_k(t_k / tau) (or exp(t_k / tau - lse))
//     loss = tau^2 sum_k p_k (log p_k - log q_{i_k}),   dz_v = g tau (S q_v - sum_{k: i_k = v} p_k),   S = sum_k p_k
//
// A row is read once, into registers, by one CTA or by a cluster of up to eight (a slice of the columns each; the row's
// maximum and sums cross the cluster through shared memory): rows of many columns do not fit one SM, and few rows would leave
// most SMs idle.  Where there are many rows per SM, the next one is on its way into shared memory while the current
// one is reduced and its gradient stored.  The entries touch few columns: every thread stores its columns of g tau S q,
// and behind a barrier the threads that own an entry store the columns of the aim once more, from the logits that they
// have read before.
#include <cooperative_groups.h>

#include "head.cuh"

namespace bt {

namespace {

namespace cg = cooperative_groups;

constexpr int kMostItems = 25;              // float4 per thread of the widest variant

__device__ __forceinline__ void copy16(float4* dst, const float4* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}

struct Entries {
    int id[kMaxEntries];                    // below zero: none
    float t[kMaxEntries], z[kMaxEntries];   // the teacher's logit, later its weight; the student's logit
};

struct Four {
    float a, b, c, d;
};

// Sums (MAX false: of a, b, c, d) or maxima (MAX: of a and b, sums of c) over the row's threads; two barriers.
template <int THREADS, int CS, bool MAX>
__device__ __forceinline__ Four row_all(Four v, Four* sm, Four* all) {
    auto join = [](Four x, Four y) {
        return MAX ? Four{fmaxf(x.a, y.a), fmaxf(x.b, y.b), x.c + y.c, 0.f} : Four{x.a + y.a, x.b + y.b, x.c + y.c, x.d + y.d};
    };
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        v = join(v, Four{__shfl_xor_sync(0xffffffffu, v.a, o), __shfl_xor_sync(0xffffffffu, v.b, o), __shfl_xor_sync(0xffffffffu, v.c, o),
                         MAX ? 0.f : __shfl_xor_sync(0xffffffffu, v.d, o)});
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
    __syncthreads();
    Four r = sm[0];
#pragma unroll
    for (int w = 1; w < THREADS / 32; ++w) r = join(r, sm[w]);
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

template <int THREADS, int ITEMS, int CS, bool STREAM>
__global__ void __launch_bounds__(THREADS) distill_kernel(const DistillArgs g, int slice4, int mean_here) {
    extern __shared__ float4 row_s[];       // STREAM: the next row's slice
    __shared__ Four sm[2][THREADS / 32], all[2][CS];
    __shared__ Entries en;
    pdl_wait();
    pdl_trigger();
    const LossAim& a = g.aim;
    const int rank = CS > 1 ? (int)cg::this_cluster().block_rank() : 0;
    const int64_t first = blockIdx.x / CS, step = gridDim.x / CS;
    const int c0 = rank * slice4, ld4_ = (int)(g.ld / 4);           // columns in units of four
    const int n4 = min(slice4, ld4_ - c0);                          // columns that this CTA writes
    const float f = kLog2e / a.tau, inv_tau = 1.0f / a.tau;
    auto fetch = [&](int64_t row) {
        const float4* src = reinterpret_cast<const float4*>(g.z + row * g.ld) + c0;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int i = threadIdx.x + THREADS * k;
            if (i < n4) copy16(row_s + i, src + i);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (STREAM && first < g.N) fetch(first);
    for (int64_t row = first; row < g.N; row += step) {
        const float* z = g.z + row * g.ld;
        // the row's entries: logit of the teacher, logit of the student (before anything is written over it)
        Four m{-INFINITY, -INFINITY, 0.f, 0.f};
#pragma unroll 1
        for (int k = threadIdx.x; k < a.K; k += THREADS) {
            int id;
            const float t = entry_logit(a, row, k, g.V, rank == 0 ? g.bad : nullptr, id);
            const bool there = t != -INFINITY;                      // a logit that is not a number counts
            en.id[k] = there ? id : -1;
            en.t[k] = t;
            en.z[k] = there ? z[id] : 0.f;
            m.b = fmaxf(m.b, t);
            m.c += there ? 1.f : 0.f;
        }
        if (STREAM) asm volatile("cp.async.wait_group 0;" ::: "memory");
        float4 v[ITEMS];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int i = threadIdx.x + THREADS * k, left = g.V - 4 * (c0 + i);      // columns of the vocabulary from here on
            v[k] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            if (i < n4 && left > 0) {
                const float4 x = STREAM ? row_s[i] : __ldcs(reinterpret_cast<const float4*>(z) + c0 + i);
                v[k].x = x.x;
                if (left > 1) v[k].y = x.y;
                if (left > 2) v[k].z = x.z;
                if (left > 3) v[k].w = x.w;
            }
            m.a = fmaxf(m.a, fmaxf(fmaxf(v[k].x, v[k].y), fmaxf(v[k].z, v[k].w)));
        }
        // this thread's part of the row is in registers, and its places in shared memory may take the next one's
        if (STREAM && row + step < g.N) fetch(row + step);
        m = row_all<THREADS, CS, true>(m, sm[0], all[0]);
        if (CS > 1) m.c *= 1.0f / CS;                               // every CTA of the cluster has counted all entries
        const bool any = m.c != 0.f;
        const float norm = !any ? 0.f : a.lse ? a.lse[row] : m.b;
        Four s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            v[k].x = ex2_fast((v[k].x - m.a) * f);
            v[k].y = ex2_fast((v[k].y - m.a) * f);
            v[k].z = ex2_fast((v[k].z - m.a) * f);
            v[k].w = ex2_fast((v[k].w - m.a) * f);
            s.a += (v[k].x + v[k].y) + (v[k].z + v[k].w);
        }
        bool twice = false;
#pragma unroll 1
        for (int k = threadIdx.x; k < a.K; k += THREADS) {
            const float lp = en.t[k] - norm, p = en.id[k] >= 0 ? expf(lp) : 0.f;
            if (p != 0.f && rank == 0) {
                s.b += p;
                s.c += p * (lp - (en.z[k] - m.a) * inv_tau);
            }
            en.t[k] = p;                                            // only this thread has read it
        }
#pragma unroll 1
        for (int k = threadIdx.x >> 5; k < a.K; k += THREADS / 32)  // does an id come twice?
            for (int j = threadIdx.x & 31; j < k; j += 32) twice |= en.id[j] == en.id[k] && en.id[k] >= 0;
        s.d = twice ? 1.f : 0.f;
        s = row_all<THREADS, CS, false>(s, sm[1], all[1]);
        const float share = a.lse ? 1.f : any ? 1.0f / s.b : 0.f, S = a.lse ? s.b : any ? 1.f : 0.f;
        const float w = row_weight(a, row), G = a.inv_count * w * a.tau;
        if (rank == 0 && threadIdx.x == 0) {
            // sum_k p_k (log p_k + log sum exp - z_k), the teacher's normaliser taken out of the sum
            const float loss = !any || (a.lse && S == 0.f) ? 0.f : (a.lse ? s.c + S * logf(s.a) : s.c * share - logf(s.b) + logf(s.a)) * (a.tau * a.tau);
            g.losses[row] = loss;
            if (mean_here) *g.loss_mean = w != 0.f ? (float)((double)loss * (double)w * (double)a.inv_count) : 0.f;
        }
        if (!g.dz && !g.dz_hi) continue;
        const bool live = G != 0.f && S != 0.f;
        const float sc = G * S / s.a;
        float4 *dz = reinterpret_cast<float4*>(g.dz ? g.dz + row * g.ld : nullptr), *hi = reinterpret_cast<float4*>(g.dz_hi ? g.dz_hi + row * g.ld : nullptr),
               *lo = reinterpret_cast<float4*>(g.dz_hi ? g.dz_lo + row * g.ld : nullptr);
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int i = threadIdx.x + THREADS * k;
            if (i >= n4) continue;
            const int left = g.V - 4 * (c0 + i);
            float4 d = make_float4(0.f, 0.f, 0.f, 0.f);
            if (live) {
                if (left > 0) d.x = v[k].x * sc;
                if (left > 1) d.y = v[k].y * sc;
                if (left > 2) d.z = v[k].z * sc;
                if (left > 3) d.w = v[k].w * sc;
            }
            if (dz) __stcs(dz + c0 + i, d);
            if (hi) {
                float4 h, l;
                split_tf32(d, h, l);
                __stcs(hi + c0 + i, h);
                __stcs(lo + c0 + i, l);
            }
        }
        __syncthreads();
        if (live) {
#pragma unroll 1
            for (int k = threadIdx.x; k < a.K; k += THREADS) {
                const int id = en.id[k];
                if (id < 4 * c0 || id >= 4 * (c0 + n4)) continue;   // none, or another CTA's column
                float sum = en.t[k];
                bool one = true;
                if (s.d != 0.f) {                                   // the first entry of an id takes all of its weight
                    sum = 0.f;
                    for (int j = 0; one && j < a.K; ++j) {
                        if (en.id[j] != id) continue;
                        if (j < k) one = false;
                        else sum += en.t[j];
                    }
                }
                if (!one) continue;
                const float d = sc * ex2_fast((en.z[k] - m.a) * f) - G * (sum * share);
                if (g.dz) g.dz[row * g.ld + id] = d;
                if (g.dz_hi) split_tf32(d, g.dz_hi[row * g.ld + id], g.dz_lo[row * g.ld + id]);
            }
        }
        __syncthreads();                                            // the entries in shared memory have been read
    }
    if (CS > 1) cg::this_cluster().sync();                          // no CTA leaves while another may write to its memory
}

// Rows of more columns than a cluster holds: three passes over global memory.
constexpr int kWideThreads = 1024;

__global__ void __launch_bounds__(kWideThreads) distill_wide_kernel(const DistillArgs g) {
    constexpr int T = kWideThreads;
    __shared__ int id_s[kMaxEntries];
    __shared__ float p_s[kMaxEntries], smf[T / 32];
    pdl_wait();
    pdl_trigger();
    const int64_t row = blockIdx.x;
    const LossAim& a = g.aim;
    const float* z = g.z + row * g.ld;
    const float f = kLog2e / a.tau;
    float m = -INFINITY;
    for (int v = threadIdx.x; v < g.V; v += T) m = fmaxf(m, z[v]);
    m = block_all<T>(m, smf, MaxOp());
    float s = 0.f;
    for (int v = threadIdx.x; v < g.V; v += T) s += ex2_fast((z[v] - m) * f);
    s = block_all<T>(s, smf, SumOp());
    bool any;
    const float norm = teacher_norm<T>(a, row, g.V, g.bad, smf, any), log_s = logf(s);
    const int k = threadIdx.x;                                      // one entry per thread
    int id = -1;
    float p = 0.f, zk = 0.f, loss = 0.f;
    if (k < a.K && any) {
        const float lp = entry_logit(a, row, k, g.V, nullptr, id) - norm;
        p = expf(lp);
        if (p == 0.f) id = -1;
        else {
            zk = z[id];
            loss = p * (lp + (log_s - (zk - m) * (1.0f / a.tau)));
        }
    }
    if (k < a.K) {
        id_s[k] = id;
        p_s[k] = p;
    }
    const float S = block_all<T>(p, smf, SumOp());
    loss = block_all<T>(loss, smf, SumOp());
    if (threadIdx.x == 0) g.losses[row] = loss * (a.tau * a.tau);
    if (!g.dz && !g.dz_hi) return;
    const float G = a.inv_count * row_weight(a, row) * a.tau, sc = G * S / s;
    const bool live = G != 0.f && S != 0.f;
    auto put = [&](int64_t v, float d) {
        if (g.dz) g.dz[row * g.ld + v] = d;
        if (g.dz_hi) split_tf32(d, g.dz_hi[row * g.ld + v], g.dz_lo[row * g.ld + v]);
    };
    for (int64_t v = threadIdx.x; v < g.ld; v += T) put(v, live && v < g.V ? sc * ex2_fast((z[v] - m) * f) : 0.f);
    __syncthreads();
    if (!live || id < 0) return;
    float sum = 0.f;
    for (int j = 0; j < a.K; ++j) {
        if (id_s[j] != id) continue;
        if (j < k) return;
        sum += p_s[j];
    }
    put(id, sc * ex2_fast((zk - m) * f) - G * sum);
}
static_assert(kMaxEntries <= kWideThreads, "one entry per thread");

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

template <int THREADS, int ITEMS, int CS, bool STREAM>
cudaError_t launch_rows(const DistillArgs& g, int64_t ctas, int slice4, cudaStream_t s) {
    const size_t smem = STREAM ? (size_t)slice4 * sizeof(float4) : 0;
    if (STREAM) {
        const cudaError_t e = allow_smem<distill_kernel<THREADS, ITEMS, CS, STREAM>>((size_t)THREADS * ITEMS * sizeof(float4));
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CS;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CS > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, distill_kernel<THREADS, ITEMS, CS, STREAM>, g, slice4, g.N == 1 && g.loss_mean ? 1 : 0);
}

template <int CS>
cudaError_t launch_slices(const DistillArgs& g, int sms, cudaStream_t s) {
    const int slice4 = (int)((g.ld / 4 + CS - 1) / CS), most = sms / CS;
    // many rows per cluster: a loop over rows with the next one in flight; the narrower variants overlap CTAs instead
    if (slice4 > 512 * 12) {
        if (g.N > most) return launch_rows<512, kMostItems, CS, true>(g, (int64_t)most * CS, slice4, s);
        return launch_rows<512, kMostItems, CS, false>(g, g.N * CS, slice4, s);
    }
    if (slice4 > 512 * 4) return launch_rows<512, 12, CS, false>(g, g.N * CS, slice4, s);
    if (slice4 > 128 * 4) return launch_rows<512, 4, CS, false>(g, g.N * CS, slice4, s);
    return launch_rows<128, 4, CS, false>(g, g.N * CS, slice4, s);
}

}  // namespace

cudaError_t launch_softmax_distill(const DistillArgs& g, cudaStream_t s) {
    int dev = 0, sms = 148;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    const int64_t n4 = g.ld / 4, held = 512 * kMostItems;
    // as many CTAs per row as its columns need, more while SMs would be idle and a CTA keeps four values a thread
    int cs = 1;
    while (cs < 8 && (n4 > held * cs || (g.N * cs * 2 <= sms && n4 > 512 * cs))) cs *= 2;
    cudaError_t e;
    if (n4 > held * cs) {
        BT_KERNEL_LAUNCH((distill_wide_kernel), (unsigned)g.N, kWideThreads, 0, s, g);
        e = cudaGetLastError();
    } else {
        e = cs == 1 ? launch_slices<1>(g, sms, s) : cs == 2 ? launch_slices<2>(g, sms, s) : cs == 4 ? launch_slices<4>(g, sms, s) : launch_slices<8>(g, sms, s);
    }
    if (e != cudaSuccess) return e;
    BT_COUNT_LAUNCH();
    if (g.loss_mean && (g.N > 1 || n4 > held * cs)) {
        BT_KERNEL_LAUNCH((weighted_mean_kernel), 1, 1024, 0, s, (const float*)g.losses, g.aim, g.N, g.loss_mean);
        BT_COUNT_LAUNCH();
    }
    return cudaGetLastError();
}

}  // namespace bt
