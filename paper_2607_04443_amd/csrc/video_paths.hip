// gfx950 (MI355X, CDNA4): the video kernel over 8-bit pages and under token windows
// (video_core.hpp), one kernel per cache format.  The bf16 one is for windows alone.
// Bound, like the bf16 kernel, by the matrix pipe and by the instructions issued beside
// it.  920 rows, 40 heads: a window of 3680 tokens over bf16 pages 88 us (0.76 of the
// rate of a large matrix product over the pairs that are seen, pages at both edges
// being taken whole); 8 units of history 136 us (e4m3) and 156 us (int8), 127 us over
// bf16 pages by the kernel without windows; 32 units 540 us (int8).
#include <hip/hip_ext.h>

#include "video_core.hpp"
#include "ws_kernels.hpp"

namespace ws {
namespace {

__global__ WS_ONE_WAVE_PER_SIMD void window_attn_kernel(const AttnArgs a) {
  unit_attn<Path<kFmtBf16, true>, kQueriesAny>(a);
}
__global__ WS_ONE_WAVE_PER_SIMD void int8_attn_kernel(const AttnArgs a) {
  unit_attn<Path<kFmtInt8, true>, kQueriesAny>(a);
}
__global__ WS_ONE_WAVE_PER_SIMD void e4m3_attn_kernel(const AttnArgs a) {
  unit_attn<Path<kFmtE4m3, true>, kQueriesAny>(a);
}

}  // namespace

hipError_t launch_path_attention(const AttnArgs& a, hipStream_t stream, hipEvent_t start, hipEvent_t stop) {
  const dim3 grid(a.n_wg), block(kVideoWaves * 64);
  const auto kernel = a.format == kFmtBf16 ? window_attn_kernel : a.format == kFmtInt8 ? int8_attn_kernel : e4m3_attn_kernel;
  if (start || stop)
    hipExtLaunchKernelGGL(kernel, grid, block, 0, stream, start, stop, 0, a);
  else
    hipLaunchKernelGGL(kernel, grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace ws
