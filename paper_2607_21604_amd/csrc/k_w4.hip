// Products of a few rows with 4-bit weights.
#include <algorithm>

#include "gemm_dev.h"
#include "kernels.h"

namespace akvs {

// A wave per output and row: lanes take 8 weights each in turn. Simple; the weights are read once
// for each row.
__device__ __forceinline__ float w4_dot(const W4Args &a, int o, int r, int lane) {
  const uint8_t *w = a.w + (size_t)o * (a.n_in / 2);
  const _Float16 *meta = reinterpret_cast<const _Float16 *>(a.meta + (size_t)o * (a.n_in / 64));
  float s = 0.f;
  for (int k = lane * 8; k < a.n_in; k += 512) {
    float wv[8], xv[8];
    cache_load8(w, meta, AKVS_U4G64, 0, a.n_in, k, wv);
    if (a.x_dtype == AKVS_BF16) load8(reinterpret_cast<const bf16_t *>(a.x) + r * a.ldx + k, xv);
    else load8(reinterpret_cast<const float *>(a.x) + r * a.ldx + k, xv);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(wv[i], xv[i], s);
  }
  return wave_sum(s);
}

__global__ __launch_bounds__(256) void k_w4_simple(W4Args a) {
  const int lane = threadIdx.x & 63, wide = a.swiglu ? a.n_out / 2 : a.n_out;
  const int o = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (o >= wide) return;
  for (int r = 0; r < a.rows; ++r) {
    float y = w4_dot(a, o, r, lane);
    if (a.swiglu) y = silu(y) * w4_dot(a, o + wide, r, lane);
    if (lane != 0) continue;
    const size_t at = r * a.ldy + o;
    if (a.resid) y += a.resid[at];
    if (a.y_dtype == AKVS_BF16) store1(reinterpret_cast<bf16_t *>(a.y) + at, y);
    else reinterpret_cast<float *>(a.y)[at] = y;
  }
}

size_t w4_ws_floats(int rows, int n_out, int n_in) { return 0; }

hipError_t launch_w4(const W4Args &a, float *ws, hipStream_t st) {
  const int wide = a.swiglu ? a.n_out / 2 : a.n_out;
  if (a.rows == 0 || wide == 0) return hipSuccess;
  hipLaunchKernelGGL(k_w4_simple, dim3((wide + 3) / 4), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace akvs
