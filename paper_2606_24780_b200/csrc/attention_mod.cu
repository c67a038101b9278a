// Attention with modified scores: which kernels run for which inputs.
#include "common.cuh"

namespace bt {

cudaError_t launch_attention_dvec(const float* o, const float* o_lo, const float* d_o, const float* d_o_lo, int B,
                                  int T, int C, int H, float* dvec, cudaStream_t s);
cudaError_t launch_attention_mod_fwd_simt(const AttnModArgs& g, cudaStream_t s);
cudaError_t launch_attention_mod_bwd_simt(const AttnModArgs& g, cudaStream_t s);

cudaError_t launch_attention_mod_fwd(const AttnModArgs& g, bool simt, cudaStream_t s) {
    (void)simt;
    return launch_attention_mod_fwd_simt(g, s);
}

cudaError_t launch_attention_mod_bwd(const AttnModArgs& g, bool simt, cudaStream_t s) {
    (void)simt;
    cudaError_t e = launch_attention_dvec(g.o, nullptr, g.d_o, g.d_o_lo, g.B, g.T, g.C, g.H, g.dvec, s);
    if (e != cudaSuccess) return e;
    return launch_attention_mod_bwd_simt(g, s);
}

}  // namespace bt
