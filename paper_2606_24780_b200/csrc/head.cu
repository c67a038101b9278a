// Losses at the language-model head without the logits.
//
//     z_nv = x_n . W_v / tau,   lse_n = log sum_v exp z_nv,   q_nv = exp(z_nv - lse_n)
//     cross entropy (tau = 1):  loss_n = lse_n - z_{n, y_n}
//     distillation:             loss_n = tau^2 sum_k p_nk (log p_nk - z_{n, i_nk} + lse_n)
//     both:                     dz_nv = g_n (q_nv - a_nv),   dx = dz W,   dW = dz^T x
// where a_nv is the row's aim (1 at the target; the sum of p_nk / S_n over the entries with i_nk = v, S_n = sum_k p_nk) and
// g_n = inv_count w_n tau S_n.  The forward keeps one (maximum, sum) pair per row and strip of the vocabulary, joined
// by head_finish_kernel, which also forms the few scores that the loss needs by themselves; the backward forms z again.
//
// The kernels here are for few rows: the weights are read in full width by every SM and each value is used for
// up to eight rows from registers.
#include "head.cuh"

namespace bt {

namespace {

constexpr int kRows = 8;                    // rows of x that one launch carries
constexpr int kStrips = 592;                // CTAs over the vocabulary (4 per SM)
constexpr int kThreads = 256;
constexpr int kFinishThreads = 256;

struct RowParams {                          // backward, per row
    float L;                                // lse in units of log 2; +inf: the row has no part in the loss
    float g;                                // inv_count w tau S
    int target;                             // column whose aim is 1; below zero: none
};

struct Scratch {
    HeadHeader* head;
    float2* stats;                          // forward: [N][strips]
    RowParams* rows;                        // backward: [N]
    int* eid;                               // [N][K] columns of the aim, each once; below zero: none
    float* ep;                              // [N][K] its weights there
    float* u;                               // [V][kRows]
    float* dx_part;                         // [strips][kRows][C]
};

size_t fwd_layout(Scratch& s, uint8_t* base, int64_t N) {
    size_t at = kHeadHeader;
    s.head = (HeadHeader*)base;
    s.stats = (float2*)(base + at);
    return at + head_pad((size_t)N * kStrips * sizeof(float2));
}

size_t bwd_layout(Scratch& s, uint8_t* base, int64_t N, int C, int V, int K) {
    size_t at = kHeadHeader;
    s.head = (HeadHeader*)base;
    s.rows = (RowParams*)(base + at);
    at += head_pad((size_t)N * sizeof(RowParams));
    s.eid = (int*)(base + at);
    at += head_pad((size_t)N * K * 4);
    s.ep = (float*)(base + at);
    at += head_pad((size_t)N * K * 4);
    s.u = (float*)(base + at);
    at += head_pad((size_t)V * kRows * 4);
    s.dx_part = (float*)(base + at);
    return at + head_pad((size_t)kStrips * kRows * C * 4);
}

__device__ __forceinline__ float4 ld_value(const float* hi, const float* lo, int64_t i4) {
    const float4 a = ld4(hi, i4);
    return lo ? add4(a, ld4(lo, i4)) : a;
}
__device__ __forceinline__ float dot4(float4 a, float4 b, float acc) {
    return fmaf(a.w, b.w, fmaf(a.z, b.z, fmaf(a.y, b.y, fmaf(a.x, b.x, acc))));
}

// Dot products of RV consecutive rows of W with the NR rows of x in shared memory, by one warp.  Lane l returns the one
// of row l / (32 / (RV NR)) / NR of W and row (that) % NR of x; lanes that share a product hold it alike.
template <int NR, int RV>
__device__ __forceinline__ float warp_dots(const float4* xs, int C4, const float* w, const float* w_lo, int64_t v0, int V) {
    const int lane = threadIdx.x & 31;
    constexpr int R = RV * NR;
    float acc[R];
#pragma unroll
    for (int i = 0; i < R; ++i) acc[i] = 0.f;
    int64_t at[RV];
#pragma unroll
    for (int i = 0; i < RV; ++i) at[i] = (v0 + i < V ? v0 + i : V - 1) * C4;
#pragma unroll 2
    for (int c = lane; c < C4; c += 32) {
        float4 wv[RV];
#pragma unroll
        for (int i = 0; i < RV; ++i) wv[i] = ld_value(w, w_lo, at[i] + c);
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const float4 xv = xs[n * C4 + c];
#pragma unroll
            for (int i = 0; i < RV; ++i) acc[i * NR + n] = dot4(wv[i], xv, acc[i * NR + n]);
        }
    }
    // every step halves the products a lane carries and doubles the lanes summed
    int o = 16;
#pragma unroll
    for (int half = R / 2; half >= 1; half /= 2, o /= 2) {
        const bool up = lane & o;
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const float keep = up ? acc[i + half] : acc[i], give = up ? acc[i] : acc[i + half];
            acc[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
    float z = acc[0];
    for (; o >= 1; o /= 2) z += __shfl_xor_sync(0xffffffffu, z, o);
    return z;
}

__device__ __forceinline__ void rows_to_smem(float4* xs, const float* x, const float* x_lo, int64_t row0, int rows, int NR, int C4) {
    for (int i = threadIdx.x; i < NR * C4; i += kThreads) {
        const int n = i / C4;
        xs[i] = n < rows ? ld_value(x, x_lo, (row0 + n) * C4 + (i - n * C4)) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __syncthreads();
}

// Row statistics over a strip of the vocabulary, in units of log 2.
template <int NR, int RV>
__global__ void __launch_bounds__(kThreads) head_stats_rows_kernel(const HeadArgs g, int64_t row0, int rows, float2* stats,
                                                                   HeadHeader* head) {
    extern __shared__ float4 xs[];
    __shared__ float2 part[kThreads];
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && threadIdx.x == 0) *head = HeadHeader{0, 0u};
    const int C4 = g.C / 4, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    rows_to_smem(xs, g.x, g.x_lo, row0, rows, NR, C4);
    constexpr int R = RV * NR, kShare = 32 / R;
    const int idx = lane / kShare, vi = idx / NR;
    const float f = kLog2e / g.aim.tau;
    float m = -INFINITY, s = 0.f;
    for (int64_t v0 = ((int64_t)blockIdx.x * (kThreads / 32) + warp) * RV; v0 < g.V; v0 += (int64_t)gridDim.x * (kThreads / 32) * RV) {
        const float z = warp_dots<NR, RV>(xs, C4, g.w, g.w_lo, v0, g.V) * f;
        if (v0 + vi < g.V) {
            const float m1 = fmaxf(m, z);
            s = s * ex2_fast(m - m1) + ex2_fast(z - m1);
            m = m1;
        }
    }
    part[threadIdx.x] = make_float2(m, (lane & (kShare - 1)) ? 0.f : s);
    __syncthreads();
    if (threadIdx.x < rows) {
        m = -INFINITY, s = 0.f;
        for (int i = 0; i < kThreads; ++i)
            if ((((i & 31) / kShare) % NR) == threadIdx.x && part[i].y != 0.f) m = fmaxf(m, part[i].x);
        for (int i = 0; i < kThreads; ++i)
            if ((((i & 31) / kShare) % NR) == threadIdx.x && part[i].y != 0.f) s += part[i].y * ex2_fast(part[i].x - m);
        stats[(row0 + threadIdx.x) * gridDim.x + blockIdx.x] = make_float2(m, s);
    }
}

// One row per CTA: joins the partial statistics, forms the scores of the row's aim and the loss.
__global__ void __launch_bounds__(kFinishThreads) head_finish_kernel(const HeadArgs g, const float2* __restrict__ stats, int strips,
                                                                     HeadHeader* head) {
    __shared__ float smf[kFinishThreads / 32];
    __shared__ double smd[kFinishThreads / 32];
    pdl_wait();
    pdl_trigger();
    const int64_t row = blockIdx.x;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float2* st = stats + row * strips;
    float m = -INFINITY, s = 0.f;
    for (int i = threadIdx.x; i < strips; i += kFinishThreads)
        if (st[i].y != 0.f) m = fmaxf(m, st[i].x);          // a strip without columns has the sum zero
    m = block_all<kFinishThreads>(m, smf, MaxOp());
    for (int i = threadIdx.x; i < strips; i += kFinishThreads)
        if (st[i].y != 0.f) s += st[i].y * ex2_fast(st[i].x - m);
    s = block_all<kFinishThreads>(s, smf, SumOp());
    const float lse = (m + log2f(s)) * kLn2;

    const int C4 = g.C / 4;
    auto score = [&](int v) {                               // by a warp
        float z = 0.f;
        for (int c = lane; c < C4; c += 32)
            z = dot4(ld_value(g.x, g.x_lo, row * C4 + c), ld_value(g.w, g.w_lo, (int64_t)v * C4 + c), z);
        return warp_sum(z) * (1.0f / g.aim.tau);
    };
    float loss = 0.f;
    if (g.aim.targets) {
        int t = g.aim.targets[row];
        if (t >= 0) {
            if (t >= g.V) {
                if (g.bad && threadIdx.x == 0) atomicCAS(g.bad, 0, (int)row + 1);
                t = 0;
            }
            if (warp == 0) loss = lse - score(t);
        }
    } else {
        bool any;
        const float norm = teacher_norm<kFinishThreads>(g.aim, row, g.V, g.bad, smf, any);
        float t = 0.f;
        for (int k = warp; any && k < g.aim.K; k += kFinishThreads / 32) {
            int id;
            const float lp = entry_logit(g.aim, row, k, g.V, nullptr, id) - norm, p = expf(lp);
            if (p != 0.f) t += p * (lp + (lse - score(id)));    // NaN is not zero: such a row has no finite loss
        }
        loss = block_all<kFinishThreads>(lane == 0 ? t : 0.f, smf, SumOp()) * (g.aim.tau * g.aim.tau);
    }
    if (threadIdx.x == 0) {
        if (g.lse) g.lse[row] = lse;
        g.losses[row] = loss;
    }
    if (g.loss_mean) mean_by_last<kFinishThreads>(g.aim, g.losses, g.N, &head->rows_done, gridDim.x, g.loss_mean, smd);
}

// One row per CTA: what the backward needs to know of it.  Entries with the same id are joined into the first of them.
__global__ void __launch_bounds__(kFinishThreads) head_rows_kernel(const HeadArgs g, RowParams* rows, int* eid, float* ep,
                                                                   HeadHeader* head) {
    extern __shared__ int ids[];            // [K], then the weights [K]
    __shared__ float smf[kFinishThreads / 32];
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && threadIdx.x == 0) *head = HeadHeader{0, 0u};
    const int64_t row = blockIdx.x;
    const LossAim& a = g.aim;
    RowParams r;
    r.L = g.lse_in[row] * kLog2e;
    r.g = a.inv_count * row_weight(a, row) * a.tau;
    r.target = -1;
    bool live = r.g != 0.f;
    if (a.targets) {
        const int t = a.targets[row];
        live = live && t >= 0;
        r.target = t >= g.V ? 0 : t;
    } else {
        float* p = (float*)(ids + a.K);
        bool any;
        const float norm = teacher_norm<kFinishThreads>(a, row, g.V, nullptr, smf, any);
        float sum = 0.f;
        for (int k = threadIdx.x; k < a.K; k += kFinishThreads) {
            int id = -1;
            const float t = any ? entry_logit(a, row, k, g.V, nullptr, id) : -INFINITY;
            p[k] = any ? expf(t - norm) : 0.f;
            ids[k] = p[k] != 0.f ? id : -1;
            sum += p[k];
        }
        sum = block_all<kFinishThreads>(sum, smf, SumOp());
        live = live && sum != 0.f;
        r.g *= sum;
        for (int k = threadIdx.x; k < a.K; k += kFinishThreads) {
            const int id = ids[k];
            float w = 0.f;
            bool first = live && id >= 0;
            for (int j = 0; first && j < a.K; ++j) {
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
        r.g = 0.f;
        r.target = -1;
    }
    if (threadIdx.x == 0) rows[row] = r;
}

// u[v][n] = g_n (q_nv - [v = target]) for the rows of one launch.
template <int NR, int RV>
__global__ void __launch_bounds__(kThreads) head_grad_rows_kernel(const HeadArgs g, int64_t row0, int rows,
                                                                  const RowParams* __restrict__ params, float* __restrict__ u) {
    extern __shared__ float4 xs[];
    pdl_wait();
    pdl_trigger();
    const int C4 = g.C / 4, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    rows_to_smem(xs, g.x, g.x_lo, row0, rows, NR, C4);
    constexpr int kShare = 32 / (RV * NR);
    const int idx = lane / kShare, vi = idx / NR, n = idx % NR;
    const float f = kLog2e / g.aim.tau;
    const RowParams r = n < rows ? params[row0 + n] : RowParams{INFINITY, 0.f, -1};
    for (int64_t v0 = ((int64_t)blockIdx.x * (kThreads / 32) + warp) * RV; v0 < g.V; v0 += (int64_t)gridDim.x * (kThreads / 32) * RV) {
        const float z = warp_dots<NR, RV>(xs, C4, g.w, g.w_lo, v0, g.V) * f;
        const int64_t v = v0 + vi;
        if (v < g.V && (lane & (kShare - 1)) == 0)
            u[v * NR + n] = r.L == INFINITY ? 0.f : r.g * (ex2_fast(z - r.L) - (v == r.target ? 1.f : 0.f));
    }
}

// The teacher's part of u.
__global__ void __launch_bounds__(256) head_grad_entries_kernel(int64_t row0, int rows, int NR, int K, const RowParams* __restrict__ params,
                                                                const int* __restrict__ eid, const float* __restrict__ ep, float* u) {
    pdl_wait();
    pdl_trigger();
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * K) return;
    const int n = i / K, id = eid[row0 * K + i];
    if (id >= 0) u[(int64_t)id * NR + n] -= params[row0 + n].g * ep[row0 * K + i];
}

// dW_v = sum_n u_vn x_n and a strip's part of dx_n = sum_v u_vn W_v: a thread owns four columns and reads u of a row of
// W as all threads of its threadIdx.y do.
template <int NR>
__global__ void __launch_bounds__(kThreads) head_products_rows_kernel(const HeadArgs g, int64_t row0, int rows, const float* __restrict__ u,
                                                                  float* dx_part) {
    pdl_wait();
    pdl_trigger();
    const int C4 = g.C / 4, c = blockIdx.y * blockDim.x + threadIdx.x;
    if (c >= C4) return;
    float4 xv[NR], acc[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        xv[n] = n < rows ? ld_value(g.x, g.x_lo, (row0 + n) * C4 + c) : make_float4(0.f, 0.f, 0.f, 0.f);
        acc[n] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    const int lanes = gridDim.x * blockDim.y;
    for (int64_t v = blockIdx.x * blockDim.y + threadIdx.y; v < g.V; v += lanes) {
        const float4 wv = g.dx_hi || g.dx ? ld_value(g.w, g.w_lo, v * C4 + c) : make_float4(0.f, 0.f, 0.f, 0.f);
        float4 d = make_float4(0.f, 0.f, 0.f, 0.f);
        float uv[NR];
#pragma unroll
        for (int n = 0; n < NR; n += 4) {
            const float4 t = ld4(u, (v * NR + n) / 4);
            uv[n] = t.x; uv[n + 1] = t.y; uv[n + 2] = t.z; uv[n + 3] = t.w;
        }
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const float t = uv[n];
            acc[n] = make_float4(fmaf(t, wv.x, acc[n].x), fmaf(t, wv.y, acc[n].y), fmaf(t, wv.z, acc[n].z), fmaf(t, wv.w, acc[n].w));
            // a row without part in the loss may hold anything
            if (t != 0.f) d = make_float4(fmaf(t, xv[n].x, d.x), fmaf(t, xv[n].y, d.y), fmaf(t, xv[n].z, d.z), fmaf(t, xv[n].w, d.w));
        }
        if (g.dw) {
            float4* out = reinterpret_cast<float4*>(g.dw) + v * C4 + c;
            *out = row0 ? add4(*out, d) : d;
        }
    }
    if (g.dx || g.dx_hi) {
        float4* out = reinterpret_cast<float4*>(dx_part) + (int64_t)(blockIdx.x * blockDim.y + threadIdx.y) * NR * C4 + c;
#pragma unroll
        for (int n = 0; n < NR; ++n) out[n * C4] = acc[n];
    }
}

__global__ void __launch_bounds__(256) head_dx_rows_kernel(const HeadArgs g, int64_t row0, int rows, int NR, int parts,
                                                           const float* __restrict__ dx_part) {
    __shared__ float4 sm[8][32];
    pdl_wait();
    pdl_trigger();
    const int C4 = g.C / 4, lane = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int i = blockIdx.x * 32 + lane;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < rows * C4) {
#pragma unroll 4
        for (int k = y; k < parts; k += 8) t = add4(t, ld4(dx_part, (int64_t)k * NR * C4 + i));
    }
    sm[y][lane] = t;
    __syncthreads();
    if (y == 0 && i < rows * C4) {
        for (int k = 1; k < 8; ++k) t = add4(t, sm[k][lane]);
        store_raw_split(t, g.dx, g.dx_hi, g.dx_lo, row0 * C4 + i);
    }
}

constexpr size_t rows_smem(int NR, int C) { return (size_t)NR * C * sizeof(float); }

}  // namespace

size_t head_fwd_scratch_bytes(int64_t N, int C, int V, int K) {
    Scratch s;
    return fwd_layout(s, nullptr, N);
}

size_t head_bwd_scratch_bytes(int64_t N, int C, int V, int K, int piece) {
    Scratch s;
    return bwd_layout(s, nullptr, N, C, V, K);
}

cudaError_t launch_head_fwd(const HeadArgs& g, cudaStream_t s) {
    Scratch w;
    fwd_layout(w, g.scratch, g.N);
    const size_t smem = rows_smem(kRows, g.C);
    cudaError_t e = allow_smem<head_stats_rows_kernel<8, 4>>(rows_smem(kRows, 4096));
    if (e != cudaSuccess) return e;
    for (int64_t row0 = 0; row0 < g.N; row0 += kRows) {
        const int rows = (int)(g.N - row0 < kRows ? g.N - row0 : kRows);
        BT_KERNEL_LAUNCH((head_stats_rows_kernel<8, 4>), kStrips, kThreads, smem, s, g, row0, rows, w.stats, w.head);
        BT_COUNT_LAUNCH();
    }
    BT_KERNEL_LAUNCH((head_finish_kernel), (unsigned)g.N, kFinishThreads, 0, s, g, (const float2*)w.stats, kStrips, w.head);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

cudaError_t launch_head_bwd(const HeadArgs& g, cudaStream_t s) {
    Scratch w;
    const int K = g.aim.targets ? 0 : g.aim.K, C4 = g.C / 4;
    bwd_layout(w, g.scratch, g.N, g.C, g.V, K);
    cudaError_t e = allow_smem<head_grad_rows_kernel<8, 4>>(rows_smem(kRows, 4096));
    if (e != cudaSuccess) return e;
    BT_KERNEL_LAUNCH((head_rows_kernel), (unsigned)g.N, kFinishThreads, (size_t)K * 8, s, g, w.rows, w.eid, w.ep, w.head);
    BT_COUNT_LAUNCH();
    const int tx = C4 < kThreads ? C4 : kThreads, ry = kThreads / tx, strips = kStrips / ry;
    for (int64_t row0 = 0; row0 < g.N; row0 += kRows) {
        const int rows = (int)(g.N - row0 < kRows ? g.N - row0 : kRows);
        BT_KERNEL_LAUNCH((head_grad_rows_kernel<8, 4>), kStrips, kThreads, rows_smem(kRows, g.C), s, g, row0, rows,
                         (const RowParams*)w.rows, w.u);
        BT_COUNT_LAUNCH();
        if (K) {
            BT_KERNEL_LAUNCH((head_grad_entries_kernel), (rows * K + 255) / 256, 256, 0, s, row0, rows, kRows, K,
                             (const RowParams*)w.rows, (const int*)w.eid, (const float*)w.ep, w.u);
            BT_COUNT_LAUNCH();
        }
        BT_KERNEL_LAUNCH((head_products_rows_kernel<8>), dim3(strips, (C4 + tx - 1) / tx), dim3(tx, ry), 0, s, g, row0, rows, (const float*)w.u, w.dx_part);
        BT_COUNT_LAUNCH();
        if (g.dx || g.dx_hi) {
            BT_KERNEL_LAUNCH((head_dx_rows_kernel), (rows * C4 + 31) / 32, 256, 0, s, g, row0, rows, kRows, strips * ry,
                             (const float*)w.dx_part);
            BT_COUNT_LAUNCH();
        }
    }
    return cudaGetLastError();
}

}  // namespace bt
