// gs_xattn_simt_window.cu -- attention on CUDA cores through a window (a translation unit of its own for the build's sake).

#include "gs_xattn_simt.cuh"

namespace gs {

cudaError_t launch_xattn_simt_window(const XattnArgs& a, cudaStream_t s) { return forward_all<true>(a, s); }
cudaError_t launch_xattn_simt_window_backward(const XattnArgs& a, cudaStream_t s) { return backward_all<true>(a, s); }

}  // namespace gs
