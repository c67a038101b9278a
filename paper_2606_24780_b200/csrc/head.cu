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
// Up to eight rows go through the kernels here in plain FP32: the weights are read once in full width and each value is used
// for all rows from registers.  More rows go to the tensor cores (head_tc.cu) on pairs of FP16 numbers that
// head_pairs_kernel makes of x and W.
#include "head.cuh"

namespace bt {

namespace {

constexpr int kRows = 8;                    // rows of x that the plain kernels carry
constexpr int kParts = 592;                 // CTAs that look for the largest value
constexpr int kStrips = 296;                // CTAs over the vocabulary (2 per SM)
constexpr int kThreads = 256;
constexpr int kFinishThreads = 256;

// Powers of two of the FP16 pairs: W and y are held times 2^kw and 2^ky.
struct Scales {
    float dx, dw;                           // from accumulators of u W and u^T y to the results
};

struct Scratch {
    HeadHeader* head;
    float2* stats;                          // forward: [N][strips]
    RowParams* rows;                        // backward: [N]
    int* eid;                               // [N][K] columns of the aim, each once; below zero: none
    float* ep;                              // [N][K] its weights there
    // few rows
    float* u;                               // [V][kRows]
    float* dx_part;                         // [strips][kRows][C]
    // tensor cores
    Scales* scales;
    float *wpart, *ypart;                   // [kParts] largest values
    float* rowmax;                          // [N]
    float* rowf;                            // [N]
    __half *x16, *y16, *w16, *u16;          // pairs: [2][N][C], [2][N][C], [2][V][C], [2][N][ldu]
    float* partials;
};

bool few_rows(int64_t N) { return N <= kRows; }

// Columns of one piece of the vocabulary, a multiple of 256: pieces of about the same size, of at most `piece` columns or
// 512 MB of u.
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
    s.wpart = take<float>(base, at, kParts);
    s.rowf = take<float>(base, at, N);
    s.x16 = take<__half>(base, at, 2 * (size_t)N * C);
    s.w16 = take<__half>(base, at, 2 * (size_t)V * C);
}

size_t fwd_layout(Scratch& s, uint8_t* base, int64_t N, int C, int V) {
    size_t at = kHeadHeader;
    s = Scratch{};
    s.head = (HeadHeader*)base;
    s.stats = take<float2>(base, at, (size_t)N * (few_rows(N) ? kStrips : head_stats_strips(V)));
    if (!few_rows(N)) tc_layout(s, base, at, N, C, V);
    return at;
}

size_t bwd_layout(Scratch& s, uint8_t* base, int64_t N, int C, int V, int K, int piece) {
    size_t at = kHeadHeader;
    s = Scratch{};
    s.head = (HeadHeader*)base;
    s.rows = take<RowParams>(base, at, N);
    s.eid = take<int>(base, at, (size_t)N * K);
    s.ep = take<float>(base, at, (size_t)N * K);
    if (few_rows(N)) {
        s.u = take<float>(base, at, (size_t)V * kRows);
        s.dx_part = take<float>(base, at, (size_t)kStrips * kRows * C);
        return at;
    }
    tc_layout(s, base, at, N, C, V);
    s.ypart = take<float>(base, at, kParts);
    s.rowmax = take<float>(base, at, N);
    s.y16 = take<__half>(base, at, 2 * (size_t)N * C);
    s.u16 = take<__half>(base, at, 2 * (size_t)N * piece_columns(N, V, piece));
    s.partials = take<float>(base, at, head_partial_bytes() / sizeof(float));
    return at;
}

template <bool PLANES>
__device__ __forceinline__ float4 ld_w(const HeadArgs& g, int64_t i4) {
    return PLANES ? add4(ld4(g.w, i4), ld4(g.w_lo, i4)) : ld4(g.w, i4);
}
__device__ __forceinline__ float4 ld_value(const float* hi, const float* lo, int64_t i4) {
    const float4 a = ld4(hi, i4);
    return lo ? add4(a, ld4(lo, i4)) : a;
}
__device__ __forceinline__ float dot4(float4 a, float4 b, float acc) {
    return fmaf(a.w, b.w, fmaf(a.z, b.z, fmaf(a.y, b.y, fmaf(a.x, b.x, acc))));
}

// The rows of W that this warp of the grid takes, to within one as many as any other.
__device__ __forceinline__ void warp_share(int V, int64_t& v0, int64_t& v1) {
    const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), all = (int64_t)gridDim.x * (kThreads / 32);
    v0 = w * V / all;
    v1 = (w + 1) * V / all;
}

// Dot products of RV consecutive rows of W (fewer before v1) with the NR rows of x in shared memory, by one warp.  Lane l returns the one
// of row l / (32 / (RV NR)) / NR of W and row (that) % NR of x; lanes that share a product hold it alike.
template <int NR, int RV, bool PLANES>
__device__ __forceinline__ float warp_dots(const float4* xs, int C4, const HeadArgs& g, int64_t v0, int64_t v1) {
    const int lane = threadIdx.x & 31;
    constexpr int R = RV * NR;
    float acc[R];
#pragma unroll
    for (int i = 0; i < R; ++i) acc[i] = 0.f;
    int64_t at[RV];
#pragma unroll
    for (int i = 0; i < RV; ++i) at[i] = (v0 + i < v1 ? v0 + i : v1 - 1) * C4;
#pragma unroll 2
    for (int c = lane; c < C4; c += 32) {
        float4 wv[RV];
#pragma unroll
        for (int i = 0; i < RV; ++i) wv[i] = ld_w<PLANES>(g, at[i] + c);
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

__device__ __forceinline__ void rows_to_smem(float4* xs, const float* x, const float* x_lo, int rows, int NR, int C4) {
    for (int i = threadIdx.x; i < NR * C4; i += kThreads) {
        const int n = i / C4;
        xs[i] = n < rows ? ld_value(x, x_lo, i) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __syncthreads();
}

// Row statistics over a strip of the vocabulary, in units of log 2.
template <int NR, int RV, bool PLANES>
__global__ void __launch_bounds__(kThreads, 2) head_stats_rows_kernel(const HeadArgs g, int rows, float2* stats,
                                                                   HeadHeader* head) {
    extern __shared__ float4 xs[];
    __shared__ float2 part[kThreads];
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && threadIdx.x == 0) *head = HeadHeader{0, 0u};
    const int C4 = g.C / 4, lane = threadIdx.x & 31;
    rows_to_smem(xs, g.x, g.x_lo, rows, NR, C4);
    constexpr int R = RV * NR, kShare = 32 / R;
    const int idx = lane / kShare, vi = idx / NR;
    const float f = kLog2e / g.aim.tau;
    float m = -INFINITY, s = 0.f;
    int64_t v0, v1;
    warp_share(g.V, v0, v1);
    for (; v0 < v1; v0 += RV) {
        const float z = warp_dots<NR, RV, PLANES>(xs, C4, g, v0, v1) * f;
        if (v0 + vi < v1) {
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
        stats[threadIdx.x * gridDim.x + blockIdx.x] = make_float2(m, s);
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

// The same for targets, a row per warp: with 8,192 rows the CTA per row above takes 88 us, most of it barriers, this 9.
__global__ void __launch_bounds__(kFinishThreads) head_finish_target_kernel(const HeadArgs g, const float2* __restrict__ stats, int strips,
                                                                            HeadHeader* head) {
    __shared__ double smd[kFinishThreads / 32];
    pdl_wait();
    pdl_trigger();
    const int64_t row = blockIdx.x * (int64_t)(kFinishThreads / 32) + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (row < g.N) {
        int t = g.aim.targets[row];
        if (t >= g.V) {
            if (g.bad && lane == 0) atomicCAS(g.bad, 0, (int)row + 1);
            t = 0;
        }
        const float2* st = stats + row * strips;
        float m = -INFINITY, s = 0.f, z = 0.f;
#pragma unroll 4
        for (int i = lane; i < strips; i += 32) {
            const float2 p = st[i];
            if (p.y != 0.f) {
                const float m1 = fmaxf(m, p.x);
                s = s * ex2_fast(m - m1) + p.y * ex2_fast(p.x - m1);
                m = m1;
            }
        }
        const float top = warp_max(m);
        s = warp_sum(s != 0.f ? s * ex2_fast(m - top) : 0.f);       // a lane without strips has the sum zero
        const float lse = (top + log2f(s)) * kLn2;
        const int C4 = g.C / 4;
        if (t >= 0) {
#pragma unroll 4
            for (int c = lane; c < C4; c += 32)
                z = dot4(ld_value(g.x, g.x_lo, row * C4 + c), ld_value(g.w, g.w_lo, (int64_t)t * C4 + c), z);
            z = warp_sum(z);
        }
        if (lane == 0) {
            if (g.lse) g.lse[row] = lse;
            g.losses[row] = t >= 0 ? lse - z : 0.f;
        }
    }
    if (g.loss_mean) mean_by_last<kFinishThreads>(g.aim, g.losses, g.N, &head->rows_done, gridDim.x, g.loss_mean, smd);
}

// Planes: the hi plane stands for the value, whose largest it bounds within 2^-11 of itself.
__device__ __forceinline__ float max4(float m, float4 v) {
    return fmaxf(fmaxf(m, fmaxf(fabsf(v.x), fabsf(v.y))), fmaxf(fabsf(v.z), fabsf(v.w)));
}

// One row per CTA: what the backward needs to know of it.  Entries with the same id are joined into the first of them.
__global__ void __launch_bounds__(kFinishThreads) head_rows_kernel(const HeadArgs g, RowParams* rows, int* eid, float* ep,
                                                                   float* rowmax, HeadHeader* head) {
    extern __shared__ int ids[];            // [K], then the weights [K]
    __shared__ float smf[kFinishThreads / 32];
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && threadIdx.x == 0) *head = HeadHeader{0, 0u};
    const int64_t row = blockIdx.x;
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
        r.L_rest = 0.f;
        r.g = 0.f;
        r.target = -1;
    }
    if (threadIdx.x == 0) rows[row] = r;
    if (rowmax && live) {                   // the same for all threads
        float m = 0.f;
        for (int c = threadIdx.x; c < g.C / 4; c += kFinishThreads) m = max4(m, ld4(g.x, row * (g.C / 4) + c));
        m = block_all<kFinishThreads>(m, smf, MaxOp());
        if (threadIdx.x == 0) rowmax[row] = m;
    }
}

// u[v][n] = g_n (q_nv - [v = target]) for the rows of one launch.
template <int NR, int RV, bool PLANES>
__global__ void __launch_bounds__(kThreads, 2) head_grad_rows_kernel(const HeadArgs g, int rows,
                                                                  const RowParams* __restrict__ params, float* __restrict__ u) {
    extern __shared__ float4 xs[];
    pdl_wait();
    pdl_trigger();
    const int C4 = g.C / 4, lane = threadIdx.x & 31;
    rows_to_smem(xs, g.x, g.x_lo, rows, NR, C4);
    constexpr int kShare = 32 / (RV * NR);
    const int idx = lane / kShare, vi = idx / NR, n = idx % NR;
    const float f = kLog2e / g.aim.tau;
    const RowParams r = n < rows ? params[n] : RowParams{INFINITY, 0.f, 0.f, -1};
    int64_t v0, v1;
    warp_share(g.V, v0, v1);
    for (; v0 < v1; v0 += RV) {
        const float z = warp_dots<NR, RV, PLANES>(xs, C4, g, v0, v1);
        const int64_t v = v0 + vi;
        if (v < v1 && (lane & (kShare - 1)) == 0)
            u[v * NR + n] = r.L == INFINITY ? 0.f : r.g * (ex2_fast(fmaf(z, f, -r.L) - r.L_rest) - (v == r.target ? 1.f : 0.f));
    }
}

// The teacher's part of u.
__global__ void __launch_bounds__(256) head_grad_entries_kernel(int rows, int NR, int K, const RowParams* __restrict__ params,
                                                                const int* __restrict__ eid, const float* __restrict__ ep, float* u) {
    pdl_wait();
    pdl_trigger();
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * K) return;
    const int n = i / K, id = eid[i];
    if (id >= 0) u[(int64_t)id * NR + n] -= params[n].g * ep[i];
}

// dW_v = sum_n u_vn x_n and a strip's part of dx_n = sum_v u_vn W_v: a thread owns four columns and reads u of a row of
// W as all threads of its threadIdx.y do.
template <int NR, bool PLANES>
__global__ void __launch_bounds__(kThreads, 2) head_products_rows_kernel(const HeadArgs g, int rows, const float* __restrict__ u,
                                                                  float* dx_part) {
    pdl_wait();
    pdl_trigger();
    const int C4 = g.C / 4, c = blockIdx.y * blockDim.x + threadIdx.x;
    if (c >= C4) return;
    float4 xv[NR], acc[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        xv[n] = n < rows ? ld_value(g.x, g.x_lo, n * C4 + c) : make_float4(0.f, 0.f, 0.f, 0.f);
        acc[n] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    const int64_t lanes = (int64_t)gridDim.x * blockDim.y, at = (int64_t)blockIdx.x * blockDim.y + threadIdx.y, v1 = (at + 1) * g.V / lanes;
#pragma unroll 4
    for (int64_t v = at * g.V / lanes; v < v1; ++v) {
        const float4 wv = g.dx_hi || g.dx ? ld_w<PLANES>(g, v * C4 + c) : make_float4(0.f, 0.f, 0.f, 0.f);
        float4 d = make_float4(0.f, 0.f, 0.f, 0.f);
        float uv[NR];
        if (NR >= 4) {
#pragma unroll
            for (int n = 0; n < NR; n += 4) {
                const float4 t = ld4(u, (v * NR + n) / 4);
                uv[n] = t.x; uv[(n + 1) % NR] = t.y; uv[(n + 2) % NR] = t.z; uv[(n + 3) % NR] = t.w;
            }
        } else {
#pragma unroll
            for (int n = 0; n < NR; ++n) uv[n] = u[v * NR + n];
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
            *out = d;
        }
    }
    if (g.dx || g.dx_hi) {
        float4* out = reinterpret_cast<float4*>(dx_part) + (int64_t)(blockIdx.x * blockDim.y + threadIdx.y) * NR * C4 + c;
#pragma unroll
        for (int n = 0; n < NR; ++n) out[n * C4] = acc[n];
    }
}

__global__ void __launch_bounds__(256) head_dx_rows_kernel(const HeadArgs g, int rows, int NR, int parts,
                                                           const float* __restrict__ dx_part) {
    __shared__ float4 sm[8][32];
    pdl_wait();
    pdl_trigger();
    const int C4 = g.C / 4, lane = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int i = blockIdx.x * 32 + lane;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < rows * C4) {
#pragma unroll 8
        for (int k = y; k < parts; k += 8) t = add4(t, ld4(dx_part, (int64_t)k * NR * C4 + i));
    }
    sm[y][lane] = t;
    __syncthreads();
    if (y == 0 && i < rows * C4) {
        for (int k = 1; k < 8; ++k) t = add4(t, sm[k][lane]);
        store_raw_split(t, g.dx, g.dx_hi, g.dx_lo, i);
    }
}

// ---------------------------------------------------------------- FP16 pairs

// The k with 2^k m in [2^14, 2^15), where 2^k is an FP32 number.
__device__ __forceinline__ int pair_exponent(float m) {
    const int e = (int)((__float_as_uint(m) >> 23) & 255u) - 127;
    return min(14 - e, 126);                // zero and denormal numbers: e = -127
}
__device__ __forceinline__ float pow2(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// Largest absolute values of W, and of y_nc = g_n x_nc (backward), per CTA.
__global__ void __launch_bounds__(kThreads) head_max_kernel(const HeadArgs g, const RowParams* __restrict__ rows,
                                                            const float* __restrict__ rowmax, float* wpart, float* ypart, HeadHeader* head) {
    __shared__ float smf[kThreads / 32];
    pdl_wait();
    pdl_trigger();
    if (head && blockIdx.x == 0 && threadIdx.x == 0) *head = HeadHeader{0, 0u};
    const int64_t n4 = (int64_t)g.V * (g.C / 4), step = (int64_t)gridDim.x * kThreads;
    float m = 0.f;
#pragma unroll 8
    for (int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x; i < n4; i += step) m = max4(m, ld4(g.w, i));
    m = block_all<kThreads>(m, smf, MaxOp());
    if (threadIdx.x == 0) wpart[blockIdx.x] = m;
    if (!rows) return;
    m = 0.f;
    for (int64_t n = blockIdx.x * (int64_t)kThreads + threadIdx.x; n < g.N; n += step)
        if (rows[n].g != 0.f) m = fmaxf(m, fabsf(rows[n].g) * rowmax[n]);
    m = block_all<kThreads>(m, smf, MaxOp());
    if (threadIdx.x == 0) ypart[blockIdx.x] = m;
}

// Four values times s as pairs.
__device__ __forceinline__ void pairs4(float4 v, float s, uint2& hi, uint2& lo) {
    const float t[4] = {v.x * s, v.y * s, v.z * s, v.w * s};
    const __half2 a = __floats2half2_rn(t[0], t[1]), b = __floats2half2_rn(t[2], t[3]);
    const float2 fa = __half22float2(a), fb = __half22float2(b);
    const __half2 c = __floats2half2_rn(t[0] - fa.x, t[1] - fa.y), d = __floats2half2_rn(t[2] - fb.x, t[3] - fb.y);
    hi = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    lo = make_uint2(*reinterpret_cast<const uint32_t*>(&c), *reinterpret_cast<const uint32_t*>(&d));
}

// W and x, and y for the backward, as pairs: W and y at one power of two, the rows of x each at its own.
__global__ void __launch_bounds__(kThreads) head_pairs_kernel(const HeadArgs g, const RowParams* __restrict__ rows, const Scratch s) {
    __shared__ float smf[kThreads / 32];
    pdl_wait();
    pdl_trigger();
    float m = 0.f, my = 0.f;
    for (int i = threadIdx.x; i < kParts; i += kThreads) {
        m = fmaxf(m, s.wpart[i]);
        if (rows) my = fmaxf(my, s.ypart[i]);
    }
    const int kw = pair_exponent(block_all<kThreads>(m, smf, MaxOp())), ky = rows ? pair_exponent(block_all<kThreads>(my, smf, MaxOp())) : 0;
    if (rows && blockIdx.x == 0 && threadIdx.x == 0) *s.scales = Scales{ldexpf(1.0f, -15 - kw), ldexpf(1.0f, -15 - ky)};
    const int64_t n8 = (int64_t)g.V * g.C / 8, step = (int64_t)gridDim.x * kThreads;
    const float sw = pow2(kw);
#pragma unroll 4
    for (int64_t k = blockIdx.x * (int64_t)kThreads + threadIdx.x; k < n8; k += step) {
        const int64_t i = n8 - 1 - k;       // backwards: the end of W is what head_max_kernel has left in L2
        uint2 h0, l0, h1, l1;
        pairs4(ld_value(g.w, g.w_lo, 2 * i), sw, h0, l0);
        pairs4(ld_value(g.w, g.w_lo, 2 * i + 1), sw, h1, l1);
        reinterpret_cast<uint4*>(s.w16)[i] = make_uint4(h0.x, h0.y, h1.x, h1.y);
        reinterpret_cast<uint4*>(s.w16)[n8 + i] = make_uint4(l0.x, l0.y, l1.x, l1.y);
    }
    const int C4 = g.C / 4, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t nx = g.N * C4;
    for (int64_t row = blockIdx.x * (int64_t)(kThreads / 32) + warp; row < g.N; row += gridDim.x * (int64_t)(kThreads / 32)) {
        float mx = 0.f;
        for (int c = lane; c < C4; c += 32) mx = max4(mx, ld4(g.x, row * C4 + c));
        const int kx = pair_exponent(warp_max(mx));
        const float sx = pow2(kx), sy = pow2(ky), gr = rows ? rows[row].g : 0.f;
        for (int c = lane; c < C4; c += 32) {
            const float4 v = ld_value(g.x, g.x_lo, row * C4 + c);
            uint2 h, l;
            pairs4(v, sx, h, l);
            reinterpret_cast<uint2*>(s.x16)[row * C4 + c] = h;
            reinterpret_cast<uint2*>(s.x16)[nx + row * C4 + c] = l;
            if (!rows) continue;
            pairs4(make_float4(v.x * gr, v.y * gr, v.z * gr, v.w * gr), sy, h, l);
            if (gr == 0.f) h = l = make_uint2(0u, 0u);          // whatever the row holds
            reinterpret_cast<uint2*>(s.y16)[row * C4 + c] = h;
            reinterpret_cast<uint2*>(s.y16)[nx + row * C4 + c] = l;
        }
        // scores whose factor leaves this range are zero to FP32, or beyond it
        if (lane == 0) s.rowf[row] = ldexpf(kLog2e / g.aim.tau, max(-120, min(120, -kx - kw)));
    }
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

cudaError_t make_pairs(const HeadArgs& g, const Scratch& w, bool back, cudaStream_t s) {
    BT_KERNEL_LAUNCH((head_max_kernel), kParts, kThreads, 0, s, g, back ? w.rows : nullptr, w.rowmax, w.wpart, w.ypart, back ? nullptr : w.head);
    BT_COUNT_LAUNCH();
    BT_KERNEL_LAUNCH((head_pairs_kernel), 148 * 8, kThreads, 0, s, g, back ? w.rows : nullptr, w);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

HalfMat pair_matrix(const __half* p, int64_t rows, int64_t cols) { return HalfMat{p, rows * cols, rows, cols, cols}; }

cudaError_t backward_in_pieces(const HeadArgs& g, const Scratch& w, int K, cudaStream_t s) {
    cudaError_t e = make_pairs(g, w, true, s);
    if (e != cudaSuccess) return e;
    const HalfMat x = pair_matrix(w.x16, g.N, g.C), y = pair_matrix(w.y16, g.N, g.C);
    const int ldu = piece_columns(g.N, g.V, g.piece);
    float* dx = g.dx ? g.dx : g.dx_hi;      // sums over the pieces go where the result will be
    for (int v0 = 0; v0 < g.V; v0 += ldu) {
        const int cols = g.V - v0 < ldu ? g.V - v0 : ldu;
        const HalfMat wp{w.w16 + (int64_t)v0 * g.C, (int64_t)g.V * g.C, cols, g.C, g.C}, u{w.u16, g.N * ldu, g.N, cols, ldu};
        e = launch_head_grad(x, wp, v0, w.rowf, w.rows, w.u16, ldu, u.plane, &w.head->err, s);
        if (e == cudaSuccess && K) {
            BT_KERNEL_LAUNCH((head_pair_entries_kernel), grid_for(g.N * K, 148 * 8), 256, 0, s, g.N, K, (const int*)w.eid, (const float*)w.ep, v0,
                             cols, w.u16, (int64_t)ldu, u.plane);
            BT_COUNT_LAUNCH();
        }
        if (e == cudaSuccess && dx) e = launch_head_dx(u, wp, w.rows, &w.scales->dx, v0 > 0, dx, w.partials, &w.head->err, s);
        if (e == cudaSuccess && g.dw) e = launch_head_dw(u, y, &w.scales->dw, g.dw + (int64_t)v0 * g.C, w.partials, &w.head->err, s);
        if (e != cudaSuccess) return e;
    }
    if (g.dx_hi) {
        BT_KERNEL_LAUNCH((head_planes_kernel), grid_for(g.N * g.C / 4, 148 * 8), 256, 0, s, (const float*)dx, g.dx_hi, g.dx_lo, g.N * g.C / 4);
        BT_COUNT_LAUNCH();
    }
    return cudaGetLastError();
}

constexpr size_t rows_smem(int NR, int C) { return (size_t)NR * C * sizeof(float); }

}  // namespace

size_t head_fwd_scratch_bytes(int64_t N, int C, int V, int) {
    Scratch s;
    return fwd_layout(s, nullptr, N, C, V);
}

size_t head_bwd_scratch_bytes(int64_t N, int C, int V, int K, int piece) {
    if (N < 1) return kHeadHeader;
    Scratch s;
    return bwd_layout(s, nullptr, N, C, V, K, piece);
}

namespace {

// x of more than two rows takes four rows of W at a time, one and two take eight: 32 products or fewer per lane
template <int NR, bool PLANES>
cudaError_t few_fwd(const HeadArgs& g, const Scratch& w, cudaStream_t s) {
    constexpr int RV = NR > 2 ? 4 : 8;
    const cudaError_t e = allow_smem<head_stats_rows_kernel<NR, RV, PLANES>>(rows_smem(NR, 4096));
    if (e != cudaSuccess) return e;
    BT_KERNEL_LAUNCH((head_stats_rows_kernel<NR, RV, PLANES>), kStrips, kThreads, rows_smem(NR, g.C), s, g, (int)g.N, w.stats, w.head);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

template <int NR, bool PLANES>
cudaError_t few_bwd(const HeadArgs& g, const Scratch& w, int K, cudaStream_t s) {
    constexpr int RV = NR > 2 ? 4 : 8;
    const cudaError_t e = allow_smem<head_grad_rows_kernel<NR, RV, PLANES>>(rows_smem(NR, 4096));
    if (e != cudaSuccess) return e;
    const int rows = (int)g.N, C4 = g.C / 4, tx = C4 < kThreads ? C4 : kThreads, ry = kThreads / tx, strips = kStrips / ry < 1 ? 1 : kStrips / ry;
    BT_KERNEL_LAUNCH((head_grad_rows_kernel<NR, RV, PLANES>), kStrips, kThreads, rows_smem(NR, g.C), s, g, rows, (const RowParams*)w.rows, w.u);
    BT_COUNT_LAUNCH();
    if (K) {
        BT_KERNEL_LAUNCH((head_grad_entries_kernel), (rows * K + 255) / 256, 256, 0, s, rows, NR, K, (const RowParams*)w.rows, (const int*)w.eid,
                         (const float*)w.ep, w.u);
        BT_COUNT_LAUNCH();
    }
    BT_KERNEL_LAUNCH((head_products_rows_kernel<NR, PLANES>), dim3(strips, (C4 + tx - 1) / tx), dim3(tx, ry), 0, s, g, rows, (const float*)w.u, w.dx_part);
    BT_COUNT_LAUNCH();
    if (g.dx || g.dx_hi) {
        BT_KERNEL_LAUNCH((head_dx_rows_kernel), (rows * C4 + 31) / 32, 256, 0, s, g, rows, NR, strips * ry, (const float*)w.dx_part);
        BT_COUNT_LAUNCH();
    }
    return cudaGetLastError();
}

template <bool PLANES>
cudaError_t few_fwd_any(const HeadArgs& g, const Scratch& w, cudaStream_t s) {
    return g.N > 4 ? few_fwd<8, PLANES>(g, w, s) : g.N > 2 ? few_fwd<4, PLANES>(g, w, s) : g.N > 1 ? few_fwd<2, PLANES>(g, w, s) : few_fwd<1, PLANES>(g, w, s);
}
template <bool PLANES>
cudaError_t few_bwd_any(const HeadArgs& g, const Scratch& w, int K, cudaStream_t s) {
    return g.N > 4 ? few_bwd<8, PLANES>(g, w, K, s) : g.N > 2 ? few_bwd<4, PLANES>(g, w, K, s)
                   : g.N > 1 ? few_bwd<2, PLANES>(g, w, K, s) : few_bwd<1, PLANES>(g, w, K, s);
}

}  // namespace

cudaError_t launch_head_fwd(const HeadArgs& g, cudaStream_t s) {
    Scratch w;
    fwd_layout(w, g.scratch, g.N, g.C, g.V);
    cudaError_t e;
    int strips = kStrips;
    if (few_rows(g.N)) {
e = g.w_lo ? few_fwd_any<true>(g, w, s) : few_fwd_any<false>(g, w, s);
    } else {
        strips = head_stats_strips(g.V);
        e = make_pairs(g, w, false, s);
        if (e == cudaSuccess)
            e = launch_head_stats(pair_matrix(w.x16, g.N, g.C), pair_matrix(w.w16, g.V, g.C), w.rowf, w.stats, &w.head->err, s);
    }
    if (e != cudaSuccess) return e;
    if (g.aim.targets && !few_rows(g.N))
        BT_KERNEL_LAUNCH((head_finish_target_kernel), (unsigned)((g.N + kFinishThreads / 32 - 1) / (kFinishThreads / 32)), kFinishThreads, 0, s, g,
                         (const float2*)w.stats, strips, w.head);
    else
        BT_KERNEL_LAUNCH((head_finish_kernel), (unsigned)g.N, kFinishThreads, 0, s, g, (const float2*)w.stats, strips, w.head);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

cudaError_t launch_head_bwd(const HeadArgs& g, cudaStream_t s) {
    Scratch w;
    const int K = g.aim.targets ? 0 : g.aim.K;
    bwd_layout(w, g.scratch, g.N, g.C, g.V, K, g.piece);
    BT_KERNEL_LAUNCH((head_rows_kernel), (unsigned)g.N, kFinishThreads, (size_t)K * 8, s, g, w.rows, w.eid, w.ep, w.rowmax, w.head);
    BT_COUNT_LAUNCH();
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    if (!few_rows(g.N)) return backward_in_pieces(g, w, K, s);
    return g.w_lo ? few_bwd_any<true>(g, w, K, s) : few_bwd_any<false>(g, w, K, s);
}

}  // namespace bt
