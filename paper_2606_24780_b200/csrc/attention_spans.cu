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
// All four come from the nearest events around i: the document start at or before it (s), the next one (e), the
// last unmarked position at or before it (i lies in the prefix when that is before s) and the next unmarked one
// (p = min(e, that), needed inside the prefix only).  One CTA takes 1,024 positions of a sequence: four scans in one
// pass over its threads, after a walk outwards over the neighbouring chunks until their events settle what
// reaches in.  Latency-bound; it runs once per batch and serves every layer, forward and backward.
// B 8, T 1,024: 8.0 us as one CTA per sequence with a pass per scan, 4.3 us so; one sequence of 8,192: 33 and 8.8 us.
#include "common.cuh"

namespace bt {

namespace {

constexpr int kThreads = 256, kItems = 4, kChunk = kThreads * kItems, kWarps = kThreads / 32;

// Nearest events: document starts and unmarked positions, the largest of what is to the left and the smallest of what is
// to the right (-1 and T: none).
struct Events {
    int start, mark, next_start, next_mark;
};
__device__ __forceinline__ Events join(const Events& a, const Events& b) {
    return {max(a.start, b.start), max(a.mark, b.mark), min(a.next_start, b.next_start), min(a.next_mark, b.next_mark)};
}

struct Ids {
    const int32_t *doc, *mark;     // of this sequence
    int T;
    __device__ __forceinline__ bool starts(int i) const { return i == 0 || (doc && doc[i] != doc[i - 1]); }
    __device__ __forceinline__ bool unmarked(int i) const { return mark == nullptr || mark[i] == 0; }
    // events of this thread's positions of chunk c
    __device__ __forceinline__ Events of(int c) const {
        Events ev{-1, -1, T, T};
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
            const int i = c * kChunk + (int)threadIdx.x * kItems + k;
            if (i >= T) break;
            if (starts(i)) ev = join(ev, {i, -1, i, T});
            if (unmarked(i)) ev = join(ev, {-1, i, T, i});
        }
        return ev;
    }
};

__device__ __forceinline__ Events reduce_block(Events ev, Events* sm) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        ev = join(ev, {__shfl_xor_sync(0xffffffffu, ev.start, o), __shfl_xor_sync(0xffffffffu, ev.mark, o),
                       __shfl_xor_sync(0xffffffffu, ev.next_start, o), __shfl_xor_sync(0xffffffffu, ev.next_mark, o)});
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = ev;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) ev = join(ev, sm[w]);
    return ev;
}

__global__ void __launch_bounds__(kThreads) attention_spans_kernel(const int32_t* __restrict__ doc,
                                                                   const int32_t* __restrict__ mark, int window, int T,
                                                                   int blocks, int2* kspan, int2* qspan, int2* kblock,
                                                                   int2* qblock) {
    __shared__ Events sm[kWarps];
    pdl_wait();
    pdl_trigger();
    const int64_t base = (int64_t)blockIdx.x * T;
    const Ids ids{doc ? doc + base : nullptr, mark ? mark + base : nullptr, T};
    const int chunk = blockIdx.y, chunks = gridDim.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int i0 = chunk * kChunk + (int)threadIdx.x * kItems;

    // what reaches in from the left and from the right
    Events in{-1, -1, T, T};
    const bool own_start = doc == nullptr || ids.starts(chunk * kChunk);
    if (!doc) in.start = 0;
    if (chunk > 0 && !(own_start && (doc || !mark)))
        for (int c = chunk - 1; c >= 0 && (in.start < 0 || (!doc && in.mark < 0)); --c) {
            const Events ev = reduce_block(ids.of(c), sm);
            in.start = max(in.start, ev.start);
            in.mark = max(in.mark, ev.mark);
        }
    if (doc || mark)
        for (int c = chunk + 1; c < chunks && in.next_start == T && (doc || in.next_mark == T); ++c) {
            const Events ev = reduce_block(ids.of(c), sm);
            in.next_start = min(in.next_start, ev.next_start);
            in.next_mark = min(in.next_mark, ev.next_mark);
        }

    // scans over the chunk: from the left inclusive of the own position, from the right exclusive for starts (e is the
    // next start after i) and inclusive for unmarked positions
    bool st[kItems], un[kItems], live[kItems];
    Events own{-1, -1, T, T};
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int i = i0 + k;
        st[k] = i < T && ids.starts(i);
        un[k] = i < T && ids.unmarked(i);
        live[k] = i < T && (doc == nullptr || ids.doc[i] >= 0);
        if (st[k]) own = join(own, {i, -1, i, T});
        if (un[k]) own = join(own, {-1, i, T, i});
    }
    Events left = own, right = own;          // inclusive over the warp: left uses the maxima, right the minima
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int a = __shfl_up_sync(0xffffffffu, left.start, o), b = __shfl_up_sync(0xffffffffu, left.mark, o);
        const int c = __shfl_down_sync(0xffffffffu, right.next_start, o), d = __shfl_down_sync(0xffffffffu, right.next_mark, o);
        if (lane >= o) {
            left.start = max(left.start, a);
            left.mark = max(left.mark, b);
        }
        if (lane + o < 32) {
            right.next_start = min(right.next_start, c);
            right.next_mark = min(right.next_mark, d);
        }
    }
    __syncthreads();
    if (lane == 31) {
        sm[warp].start = left.start;
        sm[warp].mark = left.mark;
    }
    if (lane == 0) {
        sm[warp].next_start = right.next_start;
        sm[warp].next_mark = right.next_mark;
    }
    __syncthreads();
    // exclusive of this thread
    Events ex{__shfl_up_sync(0xffffffffu, left.start, 1), __shfl_up_sync(0xffffffffu, left.mark, 1),
              __shfl_down_sync(0xffffffffu, right.next_start, 1), __shfl_down_sync(0xffffffffu, right.next_mark, 1)};
    if (lane == 0) ex.start = ex.mark = -1;
    if (lane == 31) ex.next_start = ex.next_mark = T;
    ex = join(ex, in);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) {
            ex.start = max(ex.start, sm[w].start);
            ex.mark = max(ex.mark, sm[w].mark);
        }
        if (w > warp) {
            ex.next_start = min(ex.next_start, sm[w].next_start);
            ex.next_mark = min(ex.next_mark, sm[w].next_mark);
        }
    }
    int e[kItems], u[kItems];
#pragma unroll
    for (int k = kItems - 1; k >= 0; --k) {
        e[k] = ex.next_start;
        if (st[k]) ex.next_start = i0 + k;
        if (un[k]) ex.next_mark = i0 + k;
        u[k] = ex.next_mark;
    }
    int2 ku = make_int2(0x7fffffff, -1), qu = ku;
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int i = i0 + k;
        if (st[k]) ex.start = i;
        if (un[k]) ex.mark = i;
        if (i >= T) continue;
        int2 ks = make_int2(i, i), qs = ks;
        if (live[k]) {
            const int s = ex.start;
            const bool prefix = ex.mark < s;                // nothing unmarked from s to i
            const int back = window > 0 ? min(i - s, window - 1) : i - s;
            const int ahead = window > 0 ? min(e[k] - i, window) : e[k] - i;
            ks = make_int2(i - back, prefix ? max(i + 1, min(e[k], u[k])) : i + 1);
            qs = make_int2(prefix ? s : i, i + ahead);
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
    BT_KERNEL_LAUNCH((attention_spans_kernel), dim3(B, (T + kChunk - 1) / kChunk), kThreads, 0, s, doc, mark, window, T, (T + 63) / 64,
                     const_cast<int2*>(v.k), const_cast<int2*>(v.q), const_cast<int2*>(v.kblock),
                     const_cast<int2*>(v.qblock));
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

}  // namespace bt
