// The losses at the language-model head: row arithmetic and scratch shared by their kernels.
#pragma once
#include <cuda_fp16.h>
#include <math.h>

#include "common.cuh"

namespace bt {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxEntries = 1024;           // of a teacher, per row

// Scratch starts with this header; the other regions begin on multiples of 256 bytes.
struct HeadHeader {
    int err;                                // device error word of the bounded waits
    unsigned rows_done;                     // rows whose loss is written: the CTA of the last one forms the mean
};
constexpr size_t kHeadHeader = 256;
inline size_t head_pad(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

struct __align__(16) RowParams {            // backward, per row
    float L, L_rest;                        // lse in units of log 2 and its rounding; +inf: the row has no part in the loss
    float g;                                // inv_count w tau S
    int target;                             // column whose aim is 1; below zero: none
};

// The tensor-core products (head_tc.cu).  An operand: FP16 pairs, lo plane at hi + plane, ld values between rows.
struct HalfMat {
    const __half* hi;
    int64_t plane, rows, cols, ld;
};
struct HeadStrips {
    int cols, count;                        // columns of a strip of the statistics, strips per row
};
HeadStrips head_stats_strips(int64_t N, int C, int V);
size_t head_partial_bytes();
// The scores that the losses need by themselves, in units of log 2: read off the sums that the statistics are made of.  A score formed
// anew, in another order or another precision, is off by what it is rounded by: with a loss of 1e-8 and a score of 30 that
// is all of the loss, in either direction.
struct HeadScores {
    const int* targets;                     // [N], zk [N]; null: a teacher's K entries,
    int K;                                  // zk [N][K], of which
    const int2* entries;                    // [N][K] holds (column, place in zk) by ascending column, and
    const uint32_t* spans;                  // [N][strips] those of each strip: from the lower half to the upper one
    float* zk;
};
// stats [N][strips] = (maximum, sum) of z in units of log 2 over strips of columns, by rowf [N] and colf [V] from
// accumulators there.
cudaError_t launch_head_stats(const HalfMat& x, const HalfMat& w, const float* rowf, const float* colf, const HeadScores& scores, float2* stats,
                              int* err, cudaStream_t s);
// u = 2^15 (q - [v = target]) as pairs for the columns v0 .. v0 + w.rows - 1, zero in rows without part in the loss.
cudaError_t launch_head_grad(const HalfMat& x, const HalfMat& w, int v0, const float* rowf, const RowParams* rows, __half* u, int64_t ldu,
                             int64_t u_plane, int* err, cudaStream_t s);
// dx = (+ dx) g_n scale u W;  dw = scale u^T y.
cudaError_t launch_head_dx(const HalfMat& u, const HalfMat& w, const RowParams* rows, const float* scale, bool onto, float* dx, float* partials,
                           int* err, cudaStream_t s);
cudaError_t launch_head_dw(const HalfMat& u, const HalfMat& y, const float* scale, float* dw, float* partials, int* err, cudaStream_t s);

// Few rows in plain FP32 (head_rows.cu): statistics [N][head_few_strips(N, C, V)], with zk [N] the targets' scores, or [V][kFewRows] all scores
// where there is a teacher; gradients with a table [V][kFewRows] and parts
// of dx [head_few_strips(N, C, V)][kFewRows][C] in scratch.
constexpr int kFewRows = 8;                 // of x in one pass over the weights
int head_few_at_once(int C);                // rows that one launch carries; the backward takes no more
int head_few_strips(int64_t N, int C, int V);
cudaError_t launch_head_few_stats(const HeadArgs& g, float2* stats, float* zk, HeadHeader* head, cudaStream_t s);
cudaError_t launch_head_few_grad(const HeadArgs& g, const RowParams* params, int K, const int* eid, const float* ep, float* aim, float* dx_part,
                                 cudaStream_t s);

// FP16 pairs: the k with 2^k m in [2^14, 2^15), where 2^k and 2^-k are FP32 numbers.
__device__ __forceinline__ int pair_exponent(float m) {
    const int e = (int)((__float_as_uint(m) >> 23) & 255u) - 127;
    return min(14 - e, 126);                // zero and denormal numbers: e = -127
}
__device__ __forceinline__ float pow2(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }
// Two values as FP16 pairs.
__device__ __forceinline__ void to_pairs(float a, float b, uint32_t& hi, uint32_t& lo) {
    const __half2 h = __floats2half2_rn(a, b);
    const float2 f = __half22float2(h);
    const __half2 l = __floats2half2_rn(a - f.x, b - f.y);
    hi = *reinterpret_cast<const uint32_t*>(&h);
    lo = *reinterpret_cast<const uint32_t*>(&l);
}

// The tensor core cuts its running sum to FP32 with every instruction, always toward zero.  A sum that grows to its final size
// over n instructions comes out short by some n / 2 times 2^-24 of it times the mean of the cut: measured, 0.54 for
// random operands, 0.6 for aligned ones, 1.2 where all products are positive.  n is 3 per 16 of the contraction index between
// two sums in registers; the products are made longer by 0.56.  That is right on the mean of random operands, and not for others: sums
// of products of one sign stay short by 1.0e-6 to 2.0e-6 of themselves after 72 instructions (3e-7 after 12), and a score of one product
// alone, of which nothing is cut, comes out 1.2e-6 (2e-7) too large.  lse has that error; a loss is formed beside the score itself.
inline float head_growth(double n) { return (float)(1.0 + 0.5 * 0.56 / (1 << 24) * n); }

// Statistics of up to 128 rows straight from W (head_direct.cu): [N][head_direct_strips(C, V)].  A teacher's entries are sorted into
// strips of their own, 32 columns each.
bool head_direct_fits(int64_t N);
int head_direct_strips(int C, int V);
inline HeadStrips head_direct_entry_strips(int V) { return HeadStrips{32, (V + 31) / 32}; }
cudaError_t launch_head_direct(const HeadArgs& h, const HalfMat& x, const float* rowf, const HeadScores& scores, float2* stats, int* err, cudaStream_t s);
// The same of u (as launch_head_grad, for `cols` columns from v0 on), and dx = (+ dx) g_n u W from those columns, as planes too with the last.
cudaError_t launch_head_direct_grad(const HeadArgs& h, const HalfMat& x, int v0, int cols, const float* rowf, const RowParams* rows, __half* u, int64_t ldu,
                                    int64_t u_plane, int* err, cudaStream_t s);
cudaError_t launch_head_direct_dx(const HeadArgs& h, const HalfMat& u, int v0, const RowParams* rows, bool onto, bool last, float* partials, int* err,
                                  cudaStream_t s);

// Column of entry k of a row, below zero where there is none.  An id behind the vocabulary counts as id 0 and is recorded.
__device__ __forceinline__ int entry_id(const LossAim& a, int64_t row, int k, int V, int* bad) {
    const int id = a.ids[row * a.K + k];
    if (id < V) return id;
    if (bad) atomicCAS(bad, 0, (int)row + 1);
    return 0;
}
// Its logit in units of the softened softmax, -inf where there is none (a weight of zero).
__device__ __forceinline__ float entry_logit(const LossAim& a, int64_t row, int k, int V, int* bad, int& id) {
    id = entry_id(a, row, k, V, bad);
    return id < 0 ? -INFINITY : a.logits[row * a.K + k] * (1.0f / a.tau);
}

// Whether a row has an id twice.  Up to 32 entries, one to a lane of the first warp, are matched there; more go through a table of at least
// two places per entry in shared memory (a power of two; emptied to -1, with a barrier, before the first call).  All pairs compared
// take 850 us more for 8,192 rows of 1,024 entries and 20 more for 8,000 of 64; 16 entries through the table 3 more for 8,000 rows.
__host__ __device__ inline int id_places(int K) {
    int n = 128;
    while (n < 2 * K) n *= 2;
    return K > 32 ? n : 0;
}
// By the threads k < K of the row's block, each for its entry (below zero: none); true for one of two at least.
__device__ __forceinline__ bool seen_before(int* table, int places, int K, int id) {
    if (places == 0) {
        const unsigned same = __match_any_sync(K < 32 ? (1u << K) - 1u : 0xffffffffu, id);
        return id >= 0 && __popc(same) > 1;
    }
    if (id < 0) return false;
    unsigned h = (unsigned)id * 2654435761u;           // mixed twice: ids in even steps would crowd
    h = (h ^ h >> 16) * 2654435761u >> 16;
    for (;; ++h) {                                      // ends: half of the places stay empty
        const int there = atomicCAS(table + (h & (places - 1)), -1, id);
        if (there == -1) return false;
        if (there == id) return true;
    }
}

__device__ __forceinline__ float row_weight(const LossAim& a, int64_t row) { return a.row_w ? a.row_w[row] : 1.0f; }

// Sum or maximum over the block (THREADS threads, a multiple of 32); every thread gets it.  `sm` holds THREADS / 32
// values and may be reused as soon as the call returns.
template <int THREADS, typename T, typename F>
__device__ __forceinline__ T block_all(T v, T* sm, F op) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
    __syncthreads();
    T r = sm[0];
#pragma unroll
    for (int w = 1; w < THREADS / 32; ++w) r = op(r, sm[w]);
    __syncthreads();
    return r;
}
struct SumOp {
    template <typename T>
    __device__ __forceinline__ T operator()(T a, T b) const { return a + b; }
};
struct MaxOp {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// The logarithm of a teacher's normaliser for one row, in two parts: a weight's logarithm is (t - top) - rest, where their sum would be
// rounded by 2^-24 of the largest logit.
struct TeacherNorm {
    float top, rest;
};
__device__ __forceinline__ float log_weight(float t, TeacherNorm n) { return (t - n.top) - n.rest; }
// `any`: the row has an entry.  All threads of the block call it.
template <int THREADS>
__device__ __forceinline__ TeacherNorm teacher_norm(const LossAim& a, int64_t row, int V, int* bad, float* sm, bool& any) {
    float m = -INFINITY;
    int id, have = 0;
    for (int k = threadIdx.x; k < a.K; k += THREADS) {
        const float t = entry_logit(a, row, k, V, bad, id);
        have |= t != -INFINITY;             // a logit that is not a number counts: the row then has no finite loss
        m = fmaxf(m, t);
    }
    any = __syncthreads_or(have) != 0;
    if (!any) return TeacherNorm{0.f, 0.f};
    if (a.lse) return TeacherNorm{a.lse[row], 0.f};
    m = block_all<THREADS>(m, sm, MaxOp());
    float s = 0.f;
    for (int k = threadIdx.x; k < a.K; k += THREADS) s += expf(entry_logit(a, row, k, V, nullptr, id) - m);
    return TeacherNorm{m, logf(block_all<THREADS>(s, sm, SumOp()))};
}

// The mean loss, by the block that finishes last: inv_count * sum_n w_n losses_n in a fixed order, in 64 bits.  Rows
// of weight zero are left out whatever their loss is.
template <int THREADS>
__device__ __forceinline__ void mean_by_last(const LossAim& a, const float* losses, int64_t N, unsigned* rows_done, unsigned blocks,
                                             float* mean, double* sm) {
    __shared__ bool last;
    __syncthreads();                        // the block's own loss is written
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(rows_done, 1u) == blocks - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double t = 0.0;
#pragma unroll 8
    for (int64_t n = threadIdx.x; n < N; n += THREADS) {
        const float w = row_weight(a, n);
        t += w != 0.f ? (double)__ldcg(losses + n) * (double)w : 0.0;
    }
    t = block_all<THREADS>(t, sm, SumOp());
    if (threadIdx.x == 0) *mean = (float)(t * (double)a.inv_count);
}

}  // namespace bt
