// The head's losses for few rows of x: the weights are read once, and everything that a row of them gives is formed while
// it is in registers: its scores z, and in the backward its gradient dW_v = sum_n u_vn x_n and its part of dx_n = sum_v u_vn W_v.
//
// A group of threads owns a share of the vocabulary, a thread of it four columns (eight, from 2,048 on) of every row: x, the
// sums for dx and the current four rows of W are in registers.  The dot products are folded over a warp, sixteen of
// them in sixteen shuffles, and over the group through shared memory.  Rows come in by asynchronous copies, sixteen values of
// four ahead, into places that no other thread reads: what bounds the kernel is the copies' rate (HBM):
// 31 us for one row against 50,257 x 768 (5.0 TB/s).  The gradients of five rows against 50,257 x 1,024 take 100, reading and
// writing at 4.1 TB/s: two barriers per four rows of W, and registers for two CTAs to an SM.
#include "head.cuh"

namespace bt {

namespace {

// Rows of W at a time: up to 32 products.
__host__ __device__ constexpr int batch_rows(int nr, int cols) { return cols > 1 || nr > 4 ? 4 : 8; }

__device__ __forceinline__ void copy16(float4* dst, const float4* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
// Four values as two pairs: the SM multiplies and adds FP32 pairs in one instruction.
struct V4 {
    unsigned long long a, b;
};
__device__ __forceinline__ unsigned long long fma2(unsigned long long x, unsigned long long y, unsigned long long z) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
    return r;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long x, unsigned long long y) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ unsigned long long both(float v) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float sum_of(unsigned long long v) {
    float lo, hi;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
    return lo + hi;
}
__device__ __forceinline__ V4 ldv(const float4* p) {
    const ulonglong2 t = *reinterpret_cast<const ulonglong2*>(p);
    return V4{t.x, t.y};
}
__device__ __forceinline__ V4 addv(V4 x, V4 y) { return V4{add2(x.a, y.a), add2(x.b, y.b)}; }
__device__ __forceinline__ V4 fmav(unsigned long long t, V4 x, V4 acc) { return V4{fma2(t, x.a, acc.a), fma2(t, x.b, acc.b)}; }
__device__ __forceinline__ void stv(float4* p, V4 v) {
    asm volatile("st.global.cs.v2.b64 [%0], {%1, %2};" ::"l"(p), "l"(v.a), "l"(v.b) : "memory");
}

constexpr int kPrefetch = 64 * 1024;
// CTAs per SM: of up to 256 threads three for one or two rows of x, two for more; one of more threads.
__host__ __device__ constexpr int few_ctas(int nr, int threads) { return threads > 256 ? 1 : nr <= 2 ? 3 : 2; }

struct Few {
    int rows, G;                            // rows of x of this launch; threads of a group, a multiple of 32
    int64_t row0;
    float2* stats;                          // forward: [N][gridDim.x]
    float* zk;                              // forward: [N] scores of the targets, or [V][kFewRows] all of them for a teacher
    const RowParams* params;                // backward
    const float* aim;                       // backward: [V][kFewRows] weights of a teacher's entries (nullable)
    float* dx_part;                         // backward: [gridDim.x][kFewRows][C]
    HeadHeader* head;
};

template <int ROWS, int COLS, bool PLANES, bool BACK, int THREADS>
__global__ void __launch_bounds__(THREADS, few_ctas(ROWS, THREADS)) head_few_kernel(const HeadArgs g, const Few a) {
    // products are counted for a power of two of rows
    constexpr int NR = ROWS > 4 ? 8 : ROWS > 2 ? 4 : ROWS, kBatch = batch_rows(NR, COLS), kForms = PLANES ? 2 : 1, kDepth = 16 / (kBatch * kForms * COLS);
    constexpr int R = kBatch * NR, kFold = R > 16 ? 16 : R, kFoldRows = kFold / NR, kShare = 32 / kFold;
    extern __shared__ float4 slots[];       // [kDepth][kBatch][COLS][kForms][threads]: sixteen values of four per thread
    __shared__ float part[2][16][32];       // [parity][warp][product]
    __shared__ __align__(16) float us[16][32];
    __shared__ float2 ends[16][32];
    // backward: the share's first rows on their way into L2 while the kernel before looks at the rows (5 rows against 50,257 x
    // 1,024: 108.5 us to 104.5, L2 cold)
    if (BACK && threadIdx.x == 0) {
        const int64_t r0 = (int64_t)blockIdx.x * g.V / gridDim.x, r1 = (blockIdx.x + 1LL) * g.V / gridDim.x;
        const int64_t bytes = min((r1 - r0) * g.C * 4, (int64_t)kPrefetch);      // a multiple of 128
        for (int k = 0; k < (PLANES ? 2 : 1); ++k)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"((k ? g.w_lo : g.w) + r0 * g.C), "r"((uint32_t)bytes) : "memory");
    }
    pdl_wait();
    pdl_trigger();
    if (!BACK && a.row0 == 0 && blockIdx.x == 0 && threadIdx.x == 0) *a.head = HeadHeader{0, 0u};
    const int C4 = g.C / 4, lane = threadIdx.x & 31, wi = threadIdx.x >> 5, groups = blockDim.x / a.G, gi = threadIdx.x / a.G, t = threadIdx.x - gi * a.G;
    const int w0 = gi * (a.G / 32), w1 = w0 + a.G / 32;            // the group's warps
    const int64_t parts = (int64_t)gridDim.x * groups, at = (int64_t)blockIdx.x * groups + gi;
    const int64_t v_first = at * g.V / parts, v_end = (at + 1) * g.V / parts;
    const int batches = (int)(((g.V + parts - 1) / parts + kBatch - 1) / kBatch);       // of the largest share
    const float f = kLog2e / g.aim.tau;

    auto fetch = [&](int b) {
#pragma unroll
        for (int r = 0; r < kBatch; ++r) {
            const int64_t v = v_first + (int64_t)b * kBatch + r;
#pragma unroll
            for (int k = 0; k < COLS; ++k) {
                const int c = t + a.G * k;
                if (v >= v_end || c >= C4) continue;
                float4* dst = slots + (((b % kDepth) * kBatch + r) * COLS + k) * kForms * blockDim.x + threadIdx.x;
                copy16(dst, reinterpret_cast<const float4*>(g.w) + v * C4 + c);
                if (PLANES) copy16(dst + blockDim.x, reinterpret_cast<const float4*>(g.w_lo) + v * C4 + c);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (int b = 0; b < kDepth; ++b) fetch(b);

    V4 x[ROWS][COLS], dx[ROWS][COLS];
#pragma unroll
    for (int n = 0; n < ROWS; ++n)
#pragma unroll
        for (int k = 0; k < COLS; ++k) {
            const int c = t + a.G * k;
            x[n][k] = dx[n][k] = V4{0ull, 0ull};
            if (n >= a.rows || c >= C4) continue;
            if (BACK && a.params[a.row0 + n].L == INFINITY) continue;      // the row has no part in the loss, whatever it holds
            const int64_t i = (a.row0 + n) * C4 + c;
            x[n][k] = ldv(reinterpret_cast<const float4*>(g.x) + i);
            if (g.x_lo) x[n][k] = addv(x[n][k], ldv(reinterpret_cast<const float4*>(g.x_lo) + i));
        }
    const int my_n = t % NR;                // of the product that this thread sums up over the group (t < R)
    RowParams mine{INFINITY, 0.f, 0.f, -1};
    if (BACK && t < R && my_n < a.rows) mine = a.params[a.row0 + my_n];
    int target = -1;
    if (!BACK && g.aim.targets && t < R && my_n < a.rows) {
        target = g.aim.targets[a.row0 + my_n];
        if (target >= g.V) target = 0;
    }
    float m = -INFINITY, s = 0.f;

    for (int b = 0; b < batches; ++b) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
        const int64_t v0 = v_first + (int64_t)b * kBatch;
        V4 w[kBatch][COLS];
#pragma unroll
        for (int r = 0; r < kBatch; ++r)
#pragma unroll
            for (int k = 0; k < COLS; ++k) {
                w[r][k] = V4{0ull, 0ull};
                if (v0 + r >= v_end || t + a.G * k >= C4) continue;
                const float4* src = slots + (((b % kDepth) * kBatch + r) * COLS + k) * kForms * blockDim.x + threadIdx.x;
                w[r][k] = PLANES ? addv(ldv(src), ldv(src + blockDim.x)) : ldv(src);
            }
        fetch(b + kDepth);                  // into the places just read

        // sixteen products at a time: every step halves those that a lane carries and doubles the lanes summed, and lane l ends
        // with product l / kShare
#pragma unroll
        for (int r0 = 0; r0 < kBatch; r0 += kFoldRows) {
            float acc[kFold];
#pragma unroll
            for (int r = 0; r < kFoldRows; ++r)
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    unsigned long long p = 0ull;
                    if (n < ROWS) {
#pragma unroll
                        for (int k = 0; k < COLS; ++k) p = fma2(w[r0 + r][k].b, x[n % ROWS][k].b, fma2(w[r0 + r][k].a, x[n % ROWS][k].a, p));
                    }
                    acc[r * NR + n] = sum_of(p);
                }
            int o = 16;
#pragma unroll
            for (int half = kFold / 2; half >= 1; half /= 2, o /= 2) {
                const bool up = lane & o;
#pragma unroll
                for (int i = 0; i < half; ++i) {
                    const float keep = up ? acc[i + half] : acc[i], give = up ? acc[i] : acc[i + half];
                    acc[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                }
            }
            float z = acc[0];
#pragma unroll
            for (; o >= 1; o /= 2) z += __shfl_xor_sync(0xffffffffu, z, o);
            if ((lane & (kShare - 1)) == 0) part[b & 1][wi][r0 * NR + lane / kShare] = z;
        }
        __syncthreads();
        if (t < R) {
            float z = part[b & 1][w0][t];
            for (int k = w0 + 1; k < w1; ++k) z += part[b & 1][k][t];
            const int64_t v = v0 + t / NR;
            if (!BACK) {
                if (v < v_end) {
                    const float z2 = __fmul_rn(z, f), m1 = fmaxf(m, z2);       // rounded before the differences
                    s = s * ex2_fast(m - m1) + ex2_fast(z2 - m1);
                    m = m1;
                    if (v == target) a.zk[a.row0 + my_n] = z2;
                    if (!g.aim.targets && my_n < a.rows) a.zk[v * kFewRows + a.row0 + my_n] = z2;
                }
            } else {
                float u = 0.f;
                if (v < v_end && mine.L != INFINITY) {
                    const float aim = a.aim ? a.aim[v * kFewRows + my_n] : v == mine.target ? 1.f : 0.f;
                    u = mine.g * (ex2_fast(fmaf(z, f, -mine.L) - mine.L_rest) - aim);
                }
                us[gi][t] = u;
            }
        }
        if (!BACK) continue;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kBatch; ++r) {
            V4 d[COLS];
#pragma unroll
            for (int k = 0; k < COLS; ++k) d[k] = V4{0ull, 0ull};
#pragma unroll
            for (int n = 0; n < ROWS; ++n) {
                const unsigned long long u = both(us[gi][r * NR + n]);
#pragma unroll
                for (int k = 0; k < COLS; ++k) {
                    dx[n][k] = fmav(u, w[r][k], dx[n][k]);
                    d[k] = fmav(u, x[n][k], d[k]);
                }
            }
            if (g.dw && v0 + r < v_end) {
#pragma unroll
                for (int k = 0; k < COLS; ++k) {
                    const int c = t + a.G * k;
                    if (c >= C4) continue;
                    float4* out = reinterpret_cast<float4*>(g.dw) + (v0 + r) * C4 + c;
                    stv(out, d[k]);
                }
            }
        }
    }
    if (BACK) {
        if (!a.dx_part) return;
        // the groups' sums meet in the copies' place: [rows][COLS][threads]
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int n = 0; n < ROWS; ++n)
#pragma unroll
            for (int k = 0; k < COLS; ++k) *reinterpret_cast<ulonglong2*>(slots + (n * COLS + k) * blockDim.x + threadIdx.x) = make_ulonglong2(dx[n][k].a, dx[n][k].b);
        __syncthreads();
        if (gi > 0) return;
        for (int n = 0; n < a.rows; ++n)
#pragma unroll
            for (int k = 0; k < COLS; ++k) {
                const int c = t + a.G * k;
                if (c >= C4) continue;
                V4 d = ldv(slots + (n * COLS + k) * blockDim.x + t);
                for (int i = 1; i < groups; ++i) d = addv(d, ldv(slots + (n * COLS + k) * blockDim.x + i * a.G + t));
                stv(reinterpret_cast<float4*>(a.dx_part) + ((int64_t)blockIdx.x * kFewRows + n) * C4 + c, d);
            }
    } else {
        if (t < R) ends[gi][t] = make_float2(m, s);
        __syncthreads();
        if ((int)threadIdx.x < a.rows) {
            m = -INFINITY, s = 0.f;
            for (int k = 0; k < groups; ++k)
                for (int i = threadIdx.x; i < R; i += NR)
                    if (ends[k][i].y != 0.f) m = fmaxf(m, ends[k][i].x);
            for (int k = 0; k < groups; ++k)
                for (int i = threadIdx.x; i < R; i += NR)
                    if (ends[k][i].y != 0.f) s += ends[k][i].y * ex2_fast(ends[k][i].x - m);
            a.stats[(a.row0 + threadIdx.x) * gridDim.x + blockIdx.x] = make_float2(m, s);
        }
    }
}

// dx of the rows from the CTAs' parts, 32 columns of four per CTA.
__global__ void __launch_bounds__(256) head_few_dx_kernel(const HeadArgs g, int parts, const float* __restrict__ dx_part) {
    __shared__ float4 sm[8][32];
    pdl_wait();
    pdl_trigger();
    const int C4 = g.C / 4, lane = threadIdx.x & 31, y = threadIdx.x >> 5, i = blockIdx.x * 32 + lane, n = blockIdx.y;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < C4) {
#pragma unroll 8
        for (int k = y; k < parts; k += 8) t = add4(t, ld4(dx_part, ((int64_t)k * kFewRows + n) * C4 + i));
    }
    sm[y][lane] = t;
    __syncthreads();
    if (y == 0 && i < C4) {
        for (int k = 1; k < 8; ++k) t = add4(t, sm[k][lane]);
        store_raw_split(t, g.dx, g.dx_hi, g.dx_lo, (int64_t)n * C4 + i);
    }
}

// A teacher's entries as a dense table over the vocabulary, zero elsewhere.
__global__ void __launch_bounds__(256) head_few_aim_kernel(int rows, int K, const int* __restrict__ eid, const float* __restrict__ ep,
                                                           float* aim) {
    pdl_wait();
    pdl_trigger();
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * K) return;
    const int id = eid[i];
    if (id >= 0) aim[(int64_t)id * kFewRows + i / K] = ep[i];
}

struct Shape {
    int cols, G, groups;
};
Shape shape_of(int C) {
    Shape p;
    const int C4 = C / 4;
    p.cols = C4 > 512 ? 2 : 1;
    p.G = ((C4 + p.cols - 1) / p.cols + 31) / 32 * 32;
    p.groups = p.G >= 256 ? 1 : 256 / p.G;
    return p;
}
// CTAs: as many as fit the SMs, but eight rows of W to a group at least.
int ctas_of(const Shape& p, int V, int per_sm) {
    const int most = 148 * per_sm, want = V / (8 * p.groups);
    return want < 1 ? 1 : want < most ? want : most;
}

template <int ROWS, int COLS, bool PLANES, bool BACK, int THREADS>
cudaError_t launch(const HeadArgs& g, const Few& a, const Shape& p, int grid, cudaStream_t s) {
    constexpr size_t smem = (size_t)16 * THREADS * sizeof(float4);
    const cudaError_t e = allow_smem<head_few_kernel<ROWS, COLS, PLANES, BACK, THREADS>>(smem);
    if (e != cudaSuccess) return e;
    const int threads = p.G * p.groups;
    BT_KERNEL_LAUNCH((head_few_kernel<ROWS, COLS, PLANES, BACK, THREADS>), grid, threads, (size_t)16 * threads * sizeof(float4), s, g, a);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

template <bool PLANES, bool BACK>
cudaError_t launch_rows(const HeadArgs& g, const Few& a, const Shape& p, int grid, cudaStream_t s) {
    if (p.cols == 2) return a.rows > 2 ? launch<4, 2, PLANES, BACK, 512>(g, a, p, grid, s) : launch<2, 2, PLANES, BACK, 512>(g, a, p, grid, s);
    if (p.G > 256) return a.rows > 4 ? launch<8, 1, PLANES, BACK, 512>(g, a, p, grid, s) : launch<4, 1, PLANES, BACK, 512>(g, a, p, grid, s);
    return a.rows > 6 ? launch<8, 1, PLANES, BACK, 256>(g, a, p, grid, s) : a.rows > 4 ? launch<6, 1, PLANES, BACK, 256>(g, a, p, grid, s) : a.rows > 2 ? launch<4, 1, PLANES, BACK, 256>(g, a, p, grid, s)
         : a.rows > 1 ? launch<2, 1, PLANES, BACK, 256>(g, a, p, grid, s) : launch<1, 1, PLANES, BACK, 256>(g, a, p, grid, s);
}

// Rows of x that one launch carries: those that fit the registers.
int rows_at_once(const Shape& p) { return p.cols == 2 ? 4 : kFewRows; }
int grid_of(const Shape& p, int V, int64_t rows) {
    // the last launch of several may carry fewer rows, but writes as many parts
    const int n = (int)(rows < rows_at_once(p) ? rows : rows_at_once(p));
    return ctas_of(p, V, few_ctas(n, p.G * p.groups));
}

}  // namespace

int head_few_at_once(int C) { return rows_at_once(shape_of(C)); }
int head_few_strips(int64_t N, int C, int V) { return grid_of(shape_of(C), V, N); }
cudaError_t launch_head_few_stats(const HeadArgs& g, float2* stats, float* zk, HeadHeader* head, cudaStream_t s) {
    const Shape p = shape_of(g.C);
    const int grid = grid_of(p, g.V, g.N);
    for (int64_t row0 = 0; row0 < g.N; row0 += rows_at_once(p)) {
        Few a{};
        a.rows = (int)(g.N - row0 < rows_at_once(p) ? g.N - row0 : rows_at_once(p));
        a.G = p.G; a.row0 = row0; a.stats = stats; a.zk = zk; a.head = head;
        const cudaError_t e = g.w_lo ? launch_rows<true, false>(g, a, p, grid, s) : launch_rows<false, false>(g, a, p, grid, s);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t launch_head_few_grad(const HeadArgs& g, const RowParams* params, int K, const int* eid, const float* ep, float* aim, float* dx_part,
                                 cudaStream_t s) {
    const Shape p = shape_of(g.C);
    const int grid = grid_of(p, g.V, g.N);
    Few a{};
    a.rows = (int)g.N;
    a.G = p.G; a.params = params; a.aim = K ? aim : nullptr; a.dx_part = g.dx || g.dx_hi ? dx_part : nullptr;
    cudaError_t e;
    if (K) {
        e = cudaMemsetAsync(aim, 0, (size_t)g.V * kFewRows * sizeof(float), s);
        if (e != cudaSuccess) return e;
        BT_KERNEL_LAUNCH((head_few_aim_kernel), (a.rows * K + 255) / 256, 256, 0, s, a.rows, K, eid, ep, aim);
        BT_COUNT_LAUNCH();
    }
    e = g.w_lo ? launch_rows<true, true>(g, a, p, grid, s) : launch_rows<false, true>(g, a, p, grid, s);
    if (e != cudaSuccess || !a.dx_part) return e;
    BT_KERNEL_LAUNCH((head_few_dx_kernel), dim3((g.C / 4 + 31) / 32, a.rows), 256, 0, s, g, grid, (const float*)dx_part);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

}  // namespace bt
