// Attention with modified scores: which kernels run for which inputs.
#include "common.cuh"

namespace bt {

cudaError_t launch_attention_dvec(const float* o, const float* o_lo, const float* d_o, const float* d_o_lo, int B,
                                  int T, int C, int H, float* dvec, cudaStream_t s);
cudaError_t launch_attention_mod_fwd_simt(const AttnModArgs& g, cudaStream_t s);
cudaError_t launch_attention_mod_bwd_simt(const AttnModArgs& g, cudaStream_t s);

bool attention_mod_tc_supports(const AttnModArgs& g);
cudaError_t launch_attention_mod_fwd_tc(const AttnModArgs& g, cudaStream_t s);
cudaError_t launch_attention_mod_bwd_tc(const AttnModArgs& g, cudaStream_t s);
bool attention_mod_mma_supports(const AttnModArgs& g);
cudaError_t launch_attention_mod_fwd_mma(const AttnModArgs& g, cudaStream_t s);
cudaError_t launch_attention_mod_bwd_mma(const AttnModArgs& g, cudaStream_t s);
bool attention_mod_tc128_supports(const AttnModArgs& g);
cudaError_t launch_attention_mod_fwd_tc128(const AttnModArgs& g, cudaStream_t s);
cudaError_t launch_attention_mod_bwd_tc128(const AttnModArgs& g, cudaStream_t s);

namespace {

// Heads of 16 and 32 columns arrive as raw arrays.  Planes for the tcgen05 kernels are a pass over qkv (and dO) into
// scratch and a launch each; the warp-level kernels start at once, but take three times as long per score.  16 heads of 32, cap:
//     T 128, batch 64    forward 59 us warp-level, 57 us tcgen05;   gradients 203, 168
//     T 2,000, batch 4   481, 192;   1,561, 532
// and of 16 columns, zeros in half of the tcgen05 tiles: T 256, batch 32    52, 52;   161, 166.
bool narrow_tc(const AttnModArgs& g) { return g.planes && (attn_mod_wants_planes(g.T, g.C / g.H) || !attention_mod_mma_supports(g)); }

cudaError_t narrow_planes(AttnModArgs& g, cudaStream_t s) {
    const int64_t n = (int64_t)g.B * g.T * g.C;
    cudaError_t e = cudaSuccess;
    if (!g.qkv_lo) {
        e = launch_split(g.qkv, g.planes, g.planes + 3 * n, 3 * n, s);
        g.qkv = g.planes;
        g.qkv_lo = g.planes + 3 * n;
    }
    if (e == cudaSuccess && g.d_o && !g.d_o_lo) {
        float* p = g.planes + 6 * n;
        e = launch_split(g.d_o, p, p + n, n, s);
        g.d_o = p;
        g.d_o_lo = p + n;
    }
    return e;
}

}  // namespace

cudaError_t launch_attention_mod_fwd(const AttnModArgs& args, bool simt, cudaStream_t s) {
    AttnModArgs g = args;
    cudaError_t e;
    if (!simt && narrow_tc(g)) return (e = narrow_planes(g, s)) != cudaSuccess ? e : launch_attention_mod_fwd_tc(g, s);
    if (!simt && attention_mod_tc_supports(g)) return launch_attention_mod_fwd_tc(g, s);
    if (!simt && attention_mod_tc128_supports(g)) return launch_attention_mod_fwd_tc128(g, s);
    if (!simt && attention_mod_mma_supports(g)) return launch_attention_mod_fwd_mma(g, s);
    e = cudaMemsetAsync(g.err, 0, sizeof(int), s);   // the other kernels clear it themselves
    if (e != cudaSuccess) return e;
    return launch_attention_mod_fwd_simt(g, s);
}

cudaError_t launch_attention_mod_bwd(const AttnModArgs& args, bool simt, cudaStream_t s) {
    AttnModArgs g = args;
    cudaError_t e;
    if (!simt && narrow_tc(g)) return (e = narrow_planes(g, s)) != cudaSuccess ? e : launch_attention_mod_bwd_tc(g, s);
    if (!simt && attention_mod_tc_supports(g) && g.d_o_lo) return launch_attention_mod_bwd_tc(g, s);
    if (!simt && attention_mod_tc128_supports(g) && g.d_o_lo) return launch_attention_mod_bwd_tc128(g, s);
    if (!simt && attention_mod_mma_supports(g)) return launch_attention_mod_bwd_mma(g, s);
    e = cudaMemsetAsync(g.err, 0, sizeof(int), s);
    if (e == cudaSuccess) e = launch_attention_dvec(g.o, nullptr, g.d_o, g.d_o_lo, g.B, g.T, g.C, g.H, g.dvec, s);
    if (e != cudaSuccess) return e;
    return launch_attention_mod_bwd_simt(g, s);
}

}  // namespace bt
