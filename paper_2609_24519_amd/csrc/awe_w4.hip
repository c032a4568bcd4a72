// Products with 4-bit weights in scaled groups (awe_gemm_w4):
//   Y[i,j] = sx[i] sum_g s[j,g] sum_{k in g} X[i,k] (u[j,k] - z[j,g]).
#include "quant_device.h"

namespace awe {
namespace {

// One wave per output: lanes stride over the reduction, a partial sum per lane, one tree at the end.
__global__ __launch_bounds__(256) void w4_plain_kernel(W4Launch g) {
  const int lane = threadIdx.x & 63;
  const int64_t o = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t i = o / g.N, j = o % g.N;
  if (i >= g.M) return;
  float sum = 0.f;
  for (int64_t k = lane; k < g.K; k += 64) {
    const int64_t grp = k / g.group;
    const int u = (g.w[j * g.ldw + k / 2] >> (4 * (k & 1))) & 15;
    const int z = g.zeros != nullptr ? g.zeros[j * g.ldz + grp] : 8;
    const float x = g.x_type == AWE_I8 ? (float)reinterpret_cast<const int8_t*>(g.x)[i * g.ldx + k]
                                       : load_real(g.x, i * g.ldx + k, g.x_type);
    sum += load_real(g.scales, j * g.lds + grp, g.s_type) * (x * (float)(u - z));
  }
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) store_real(g.y, i * g.ldy + j, g.y_type, g.x_scales != nullptr ? sum * g.x_scales[i] : sum);
}

}  // namespace

awe_status launch_w4(const W4Launch& g, hipStream_t stream) {
  const int64_t blocks = (g.M * g.N + 3) / 4;
  if (blocks > 0x7fffffffLL) {
    set_error("too many outputs");
    return AWE_ERR_UNSUPPORTED;
  }
  hipLaunchKernelGGL(w4_plain_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, g);
  return launched("w4 launch");
}

}  // namespace awe
