// Distillation from a teacher's top logits, on the student's logits: losses and gradient in one kernel.
//
//     z' = z / tau, q = softmax(z'), p_k = softmax_k(t_k / tau) (or exp(t_k / tau - lse))
//     loss = tau^2 sum_k p_k (log p_k - log q_{i_k}),   dz_v = g tau (S q_v - sum_{k: i_k = v} p_k),   S = sum_k p_k
//
// The entries touch few columns: every thread stores its columns of g tau S q, and behind a barrier the threads that own an
// entry store the columns of the aim once more, from the logits that they have read before.
#include "head.cuh"

namespace bt {

namespace {

constexpr int kDistillThreads = 512;

struct Entries {
    int id[kMaxEntries];
    float p[kMaxEntries], z[kMaxEntries];
};

__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const DistillArgs g) {
    constexpr int T = kDistillThreads;
    __shared__ Entries en;
    __shared__ float smf[T / 32];
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
    const float norm = teacher_norm<T>(a, row, g.V, g.bad, smf, any);
    const float log_s = logf(s);
    float S = 0.f, loss = 0.f;
    for (int k = threadIdx.x; k < a.K; k += T) {
        int id;
        const float lp = entry_logit(a, row, k, g.V, nullptr, id) - norm, p = any ? expf(lp) : 0.f;
        en.id[k] = p != 0.f ? id : -1;
        en.p[k] = p;
        if (p != 0.f) {
            en.z[k] = z[id];
            S += p;
            loss += p * (lp + (log_s - (en.z[k] - m) * (1.0f / a.tau)));
        }
    }
    S = block_all<T>(S, smf, SumOp());
    loss = block_all<T>(loss, smf, SumOp());
    const float w = row_weight(a, row);
    if (threadIdx.x == 0) g.losses[row] = loss * (a.tau * a.tau);
    if (!g.dz && !g.dz_hi) return;
    const float G = a.inv_count * w * a.tau;
    const bool live = G != 0.f && S != 0.f;
    auto put = [&](int64_t v, float d) {
        if (g.dz) g.dz[row * g.ld + v] = d;
        if (g.dz_hi) split_tf32(d, g.dz_hi[row * g.ld + v], g.dz_lo[row * g.ld + v]);
    };
    const float sc = G * S / s;
    for (int64_t v = threadIdx.x; v < g.ld; v += T) put(v, live && v < g.V ? sc * ex2_fast((z[v] - m) * f) : 0.f);
    __syncthreads();
    if (!live) return;
    for (int k = threadIdx.x; k < a.K; k += T) {
        const int id = en.id[k];
        if (id < 0) continue;
        float p = 0.f;
        bool first = true;
        for (int j = 0; first && j < a.K; ++j) {
            if (en.id[j] != id) continue;
            if (j < k) first = false;
            else p += en.p[j];
        }
        if (first) put(id, sc * ex2_fast((en.z[k] - m) * f) - G * p);
    }
}

__global__ void __launch_bounds__(1024) weighted_mean_kernel(const float* __restrict__ losses, const LossAim a, int64_t N,
                                                             float* __restrict__ mean) {
    __shared__ double sm[32];
    pdl_wait();
    pdl_trigger();
    double t = 0.0;
    for (int64_t n = threadIdx.x; n < N; n += 1024) {
        const float w = row_weight(a, n);
        t += w != 0.f ? (double)losses[n] * (double)w : 0.0;
    }
    t = block_all<1024>(t, sm, SumOp());
    if (threadIdx.x == 0) *mean = (float)(t * (double)a.inv_count);
}

}  // namespace

cudaError_t launch_softmax_distill(const DistillArgs& g, cudaStream_t s) {
    BT_KERNEL_LAUNCH((distill_kernel), (unsigned)g.N, kDistillThreads, 0, s, g);
    BT_COUNT_LAUNCH();
    if (g.loss_mean) {
        BT_KERNEL_LAUNCH((weighted_mean_kernel), 1, 1024, 0, s, (const float*)g.losses, g.aim, g.N, g.loss_mean);
        BT_COUNT_LAUNCH();
    }
    return cudaGetLastError();
}

}  // namespace bt
