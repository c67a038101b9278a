// Key spans of a packed batch: which keys each query may read, as one range per row.
//
// A document is a maximal run of equal ids inside a sequence; ids below zero are padding, which reads
// nothing and is read by nobody.  With s and e the first and one-past-last position of the document of
// position i and p the end of its prefix (the run of marked positions it begins with, p = s without one),
// query i reads the keys [lo, hi) and key i is read by the queries [qlo, qhi):
//     lo = max(s, i - window + 1)   hi  = max(i + 1, p)
//     qlo = i < p ? s : i           qhi = min(e, i + window)
// The two are inverse to each other because lo and hi never fall along a document.  Kernels mask with
// the row ranges and skip whole tiles by the ranges of 64-row blocks (union over the block's non-empty
// rows), so that a packed batch costs what its documents cost.
//
// One CTA per sequence: a running maximum of the document starts from the left, running minima of the
// next start and of the next unmarked position from the right, then the formulas.  Latency-bound (a few
// block scans); it runs once per batch and serves every layer, forward and backward.
#include "common.cuh"

namespace bt {

namespace {

constexpr int kThreads = 1024, kItems = 4, kChunk = kThreads * kItems;

struct MaxOp { __device__ int operator()(int a, int b) const { return max(a, b); } };
struct MinOp { __device__ int operator()(int a, int b) const { return min(a, b); } };

// Exclusive scan of one value per thread over the block, in thread order; `carry` joins on the left, `total`
// is the whole block with it.
template <typename Op>
__device__ __forceinline__ int block_scan_exclusive(int v, int identity, int carry, int* sm, int& total) {
    const Op op;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc = op(inc, t);
    }
    __syncthreads();
    if (lane == 31) sm[warp] = inc;
    __syncthreads();
    if (warp == 0) {
        int w = sm[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w = op(w, t);
        }
        sm[lane] = w;
    }
    __syncthreads();
    const int before = warp ? sm[warp - 1] : identity;
    const int up = __shfl_up_sync(0xffffffffu, inc, 1);
    const int own = lane ? op(before, up) : before;
    total = op(carry, sm[31]);
    return op(carry, own);
}

// kspan / qspan double as temporaries of the CTA's own sequence: kspan.x = s, kspan.y = e, qspan.x = next
// unmarked position.
__global__ void __launch_bounds__(kThreads) attention_spans_kernel(const int32_t* __restrict__ doc,
                                                                   const int32_t* __restrict__ mark, int window, int T,
                                                                   int blocks, int2* kspan, int2* qspan, int2* kblock,
                                                                   int2* qblock) {
    __shared__ int sm[32];
    pdl_wait();
    pdl_trigger();
    const int64_t base = (int64_t)blockIdx.x * T;
    auto id = [&](int i) { return doc ? doc[base + i] : 0; };
    const int chunks = (T + kChunk - 1) / kChunk;

    int carry = 0;                                            // document starts, from the left
    for (int c = 0; c < chunks; ++c) {
        const int i0 = c * kChunk + (int)threadIdx.x * kItems;
        int st[kItems], run = 0;
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const int i = i0 + k;
            st[k] = (i < T && (i == 0 || id(i) != id(i - 1))) ? i : 0;
            run = max(run, st[k]);
        }
        int total;
        int before = block_scan_exclusive<MaxOp>(run, 0, carry, sm, total);
        carry = total;
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            before = max(before, st[k]);
            if (i0 + k < T) kspan[base + i0 + k].x = before;
        }
    }

    int carry_e = T, carry_u = T;                             // ends and unmarked positions, from the right
    for (int c = chunks - 1; c >= 0; --c) {
        const int r0 = (c + 1) * kChunk - 1 - (int)threadIdx.x * kItems;   // this thread's rightmost position
        int nx[kItems], un[kItems], run_e = T, run_u = T;
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const int i = r0 - k;
            // e of position i is the next start after i
            nx[k] = (i + 1 < T && id(i + 1) != id(i)) ? i + 1 : T;
            un[k] = (i < T && (mark == nullptr || mark[base + i] == 0)) ? i : T;
            run_e = min(run_e, nx[k]);
            run_u = min(run_u, un[k]);
        }
        int total;
        int e = block_scan_exclusive<MinOp>(run_e, T, carry_e, sm, total);
        carry_e = total;
        int u = block_scan_exclusive<MinOp>(run_u, T, carry_u, sm, total);
        carry_u = total;
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            e = min(e, nx[k]);
            u = min(u, un[k]);
            if (r0 - k < T) {
                kspan[base + r0 - k].y = e;
                qspan[base + r0 - k].x = u;
            }
        }
    }
    __syncthreads();

    // p of a document is the next unmarked position at its start: read by all of its rows before any
    // row's temporaries are overwritten
    for (int c = 0; c < chunks; ++c) {
        const int i0 = c * kChunk + (int)threadIdx.x * kItems;
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const int i = i0 + k;
            if (i < T) {
                const int2 se = kspan[base + i];
                qspan[base + i].y = min(se.y, qspan[base + se.x].x);
            }
        }
    }
    __syncthreads();

    for (int c = 0; c < chunks; ++c) {
        const int i0 = c * kChunk + (int)threadIdx.x * kItems;
        int2 ku = make_int2(0x7fffffff, -1), qu = ku;
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const int i = i0 + k;
            if (i >= T) continue;
            const int2 se = kspan[base + i];
            const int p = qspan[base + i].y;
            int2 ks = make_int2(i, i), qs = ks;
            if (id(i) >= 0) {
                const int back = window > 0 ? min(i - se.x, window - 1) : i - se.x;
                const int ahead = window > 0 ? min(se.y - i, window) : se.y - i;
                ks = make_int2(i - back, max(i + 1, p));
                qs = make_int2(i < p ? se.x : i, i + ahead);
                ku = make_int2(min(ku.x, ks.x), max(ku.y, ks.y));
                qu = make_int2(min(qu.x, qs.x), max(qu.y, qs.y));
            }
            kspan[base + i] = ks;
            qspan[base + i] = qs;
        }
        // 16 neighbouring threads hold one 64-row block
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
            ku.x = min(ku.x, __shfl_xor_sync(0xffffffffu, ku.x, o));
            ku.y = max(ku.y, __shfl_xor_sync(0xffffffffu, ku.y, o));
            qu.x = min(qu.x, __shfl_xor_sync(0xffffffffu, qu.x, o));
            qu.y = max(qu.y, __shfl_xor_sync(0xffffffffu, qu.y, o));
        }
        if ((threadIdx.x & 15) == 0 && i0 < T) {
            kblock[(int64_t)blockIdx.x * blocks + (i0 >> 6)] = ku.y < 0 ? make_int2(0, 0) : ku;
            qblock[(int64_t)blockIdx.x * blocks + (i0 >> 6)] = qu.y < 0 ? make_int2(0, 0) : qu;
        }
    }
}

}  // namespace

// Layout of the spans buffer: kspan [B*T], qspan [B*T], kblock [B * ceil(T / 64)], qblock (the same).
SpanView attention_span_view(const void* spans, int B, int T) {
    SpanView v{};
    if (!spans) return v;
    const int64_t n = (int64_t)B * T, nb = (int64_t)B * ((T + 63) / 64);
    v.k = static_cast<const int2*>(spans);
    v.q = v.k + n;
    v.kblock = v.q + n;
    v.qblock = v.kblock + nb;
    return v;
}
size_t attention_spans_bytes(int B, int T) {
    return (size_t)(2 * ((int64_t)B * T + (int64_t)B * ((T + 63) / 64))) * sizeof(int2);
}

cudaError_t launch_attention_spans(const int32_t* doc, const int32_t* mark, int window, int B, int T, void* spans,
                                   cudaStream_t s) {
    const SpanView v = attention_span_view(spans, B, T);
    BT_KERNEL_LAUNCH((attention_spans_kernel), B, kThreads, 0, s, doc, mark, window, T, (T + 63) / 64,
                     const_cast<int2*>(v.k), const_cast<int2*>(v.q), const_cast<int2*>(v.kblock),
                     const_cast<int2*>(v.qblock));
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

}  // namespace bt
