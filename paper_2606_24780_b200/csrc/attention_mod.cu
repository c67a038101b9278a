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

cudaError_t launch_attention_mod_fwd(const AttnModArgs& g, bool simt, cudaStream_t s) {
    if (!simt && attention_mod_tc_supports(g)) return launch_attention_mod_fwd_tc(g, s);
    if (!simt && attention_mod_tc128_supports(g)) return launch_attention_mod_fwd_tc128(g, s);
    if (!simt && attention_mod_mma_supports(g)) return launch_attention_mod_fwd_mma(g, s);
    const cudaError_t e = cudaMemsetAsync(g.err, 0, sizeof(int), s);   // the other kernels clear it themselves
    if (e != cudaSuccess) return e;
    return launch_attention_mod_fwd_simt(g, s);
}

cudaError_t launch_attention_mod_bwd(const AttnModArgs& g, bool simt, cudaStream_t s) {
    if (!simt && attention_mod_tc_supports(g) && g.d_o_lo) return launch_attention_mod_bwd_tc(g, s);
    if (!simt && attention_mod_tc128_supports(g) && g.d_o_lo) return launch_attention_mod_bwd_tc128(g, s);
    if (!simt && attention_mod_mma_supports(g)) return launch_attention_mod_bwd_mma(g, s);
    cudaError_t e = cudaMemsetAsync(g.err, 0, sizeof(int), s);
    if (e == cudaSuccess) e = launch_attention_dvec(g.o, nullptr, g.d_o, g.d_o_lo, g.B, g.T, g.C, g.H, g.dvec, s);
    if (e != cudaSuccess) return e;
    return launch_attention_mod_bwd_simt(g, s);
}

}  // namespace bt
