// Attention with modified scores: which kernels run for which inputs.
#include "common.cuh"

namespace bt {

cudaError_t launch_attention_dvec(const float* o, const float* o_lo, const float* d_o, const float* d_o_lo, int B,
                                  int T, int C, int H, float* dvec, cudaStream_t s);
cudaError_t launch_attention_mod_fwd_simt(const AttnModArgs& g, cudaStream_t s);
cudaError_t launch_attention_mod_bwd_simt(const AttnModArgs& g, cudaStream_t s);

cudaError_t launch_attention_mod_fwd_tc(const AttnModArgs& g, cudaStream_t s);
cudaError_t launch_attention_mod_bwd_tc(const AttnModArgs& g, cudaStream_t s);
bool attention_mod_mma_supports(const AttnModArgs& g);
cudaError_t launch_attention_mod_fwd_mma(const AttnModArgs& g, cudaStream_t s);
cudaError_t launch_attention_mod_bwd_mma(const AttnModArgs& g, cudaStream_t s);
cudaError_t launch_attention_mod_fwd_tc128(const AttnModArgs& g, cudaStream_t s);
cudaError_t launch_attention_mod_bwd_tc128(const AttnModArgs& g, cudaStream_t s);

namespace {

// Which kernels.  The tcgen05 ones read planes; arrays given raw become planes in scratch, a pass over qkv (and dO) and a
// launch.  The warp-level ones start at once, but take three times as long per score.  16 heads of 32, cap:
//     T 128, batch 64    forward 59 us warp-level, 57 us tcgen05;   gradients 203, 168
//     T 2,000, batch 4   481, 195;   1,561, 532
// and of 16 columns, zeros in half of the tcgen05 tiles: T 256, batch 32    52, 52;   161, 166.  Hence T d > 4,096: at 4,096
// itself heads of 16 are 3 % better off on the warp-level kernels and heads of 32 up to a fifth worse, below it
// (T 64, heads of 32: forward 43, 64, gradients 138, 198) the former win.  Wider heads always: one raw sequence of 64, 12 heads of
// 64, took 10 us warp-level and 15 so forward, 46 and 24 backward.
bool on_tcgen05(const AttnModArgs& g) { return attn_mod_wants_planes(g.T, g.C / g.H) || !attention_mod_mma_supports(g); }

// Up to two arrays into planes in one launch; x.n4 and y.n4 float4 values (a launch costs as much as 3 MB of copying).
struct ToSplit {
    const float* from;
    float *hi, *lo;
    int64_t n4;
};
__global__ void __launch_bounds__(256) split_two_kernel(const ToSplit x, const ToSplit y) {
    pdl_wait();
    pdl_trigger();
    for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < x.n4 + y.n4; i += (int64_t)gridDim.x * blockDim.x) {
        const ToSplit& a = i < x.n4 ? x : y;
        const int64_t k = i < x.n4 ? i : i - x.n4;
        store_raw_split(ld4(a.from, k), nullptr, a.hi, a.lo, k);
    }
}

cudaError_t make_planes(AttnModArgs& g, cudaStream_t s) {
    const int64_t n = (int64_t)g.B * g.T * g.C;
    ToSplit x{}, y{};
    if (!g.qkv_lo) {
        x = ToSplit{g.qkv, g.planes, g.planes + 3 * n, 3 * n / 4};
        g.qkv = x.hi;
        g.qkv_lo = x.lo;
    }
    if (g.d_o && !g.d_o_lo) {
        y = ToSplit{g.d_o, g.planes + 6 * n, g.planes + 7 * n, n / 4};
        g.d_o = y.hi;
        g.d_o_lo = y.lo;
    }
    if (x.n4 + y.n4 == 0) return cudaSuccess;
    const int64_t blocks = (x.n4 + y.n4 + 255) / 256;
    BT_KERNEL_LAUNCH((split_two_kernel), (int)(blocks < 148 * 16 ? blocks : 148 * 16), 256, 0, s, x, y);
    BT_COUNT_LAUNCH();
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_mod_fwd(const AttnModArgs& args, bool simt, cudaStream_t s) {
    AttnModArgs g = args;
    if (!simt && on_tcgen05(g)) {
        const cudaError_t e = make_planes(g, s);
        if (e != cudaSuccess) return e;
        return g.C / g.H == 128 ? launch_attention_mod_fwd_tc128(g, s) : launch_attention_mod_fwd_tc(g, s);
    }
    if (!simt) return launch_attention_mod_fwd_mma(g, s);
    const cudaError_t e = cudaMemsetAsync(g.err, 0, sizeof(int), s);   // the other kernels clear it themselves
    return e != cudaSuccess ? e : launch_attention_mod_fwd_simt(g, s);
}

cudaError_t launch_attention_mod_bwd(const AttnModArgs& args, bool simt, cudaStream_t s) {
    AttnModArgs g = args;
    if (!simt && on_tcgen05(g)) {
        const cudaError_t e = make_planes(g, s);
        if (e != cudaSuccess) return e;
        return g.C / g.H == 128 ? launch_attention_mod_bwd_tc128(g, s) : launch_attention_mod_bwd_tc(g, s);
    }
    if (!simt) return launch_attention_mod_bwd_mma(g, s);
    cudaError_t e = cudaMemsetAsync(g.err, 0, sizeof(int), s);
    if (e == cudaSuccess) e = launch_attention_dvec(g.o, nullptr, g.d_o, g.d_o_lo, g.B, g.T, g.C, g.H, g.dvec, s);
    return e != cudaSuccess ? e : launch_attention_mod_bwd_simt(g, s);
}

}  // namespace bt
