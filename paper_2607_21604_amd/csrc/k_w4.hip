// Products of a few rows with 4-bit weights.
//
// y = x W^T with W = scale c + zero per group of 64: for each group
//   sum x w = scale (sum x (16 + c) - 16 sum x) + zero sum x,
// where a nibble c put into the upper mantissa bits of a bf16 of 16 is 16 + c, exactly, so that the
// weights go to the matrix cores without a rounding, two in an instruction; -16 sum x comes from
// the matrix cores as well. x in bf16 is taken as it is, in fp32 as three bf16 that add up to it.
#include <algorithm>

#include "four_bit_dev.h"
#include "gemm_dev.h"
#include "kernels.h"

namespace akvs {

constexpr int W4_UNIT = 128;        // two groups: 64 bytes of a row of codes
constexpr int W4_RUN = 4 * W4_UNIT; // what a wave takes at a time

// Lane l, g = l / 16, loads 16 of a unit's 64 bytes of row l % 16, so that lanes 0..31 hold its first
// group and lanes 32..63 its second. Swapping halves leaves one group in each pair of words, and
// lane g with elements w4_first(g) .. + 15 of it.
__device__ __forceinline__ int w4_first(int g) { return ((g & 1) << 5) + ((g >> 1) << 4); }

// x as it is multiplied: the fragment of group elements w4_first(g) + 8 st .., row r.
template <int XP>
struct W4X;
template <>
struct W4X<1> {
  const bf16_t *x;
  __device__ bf16x8_t get(int, size_t at) const {
    return order8(*reinterpret_cast<const u32x4_t *>(x + at));
  }
};
template <>
struct W4X<3> {  // planes of [rows][n_in], already in the products' order
  const bf16_t *x;
  size_t plane;
  __device__ bf16x8_t get(int p, size_t at) const {
    return *reinterpret_cast<const bf16x8_t *>(x + p * plane + at);
  }
};

// fp32 rows as three bf16 parts (truncated, so that each difference is exact), every 8 elements in
// the order 0, 4, 1, 5, 2, 6, 3, 7.
__global__ __launch_bounds__(256) void k_w4_split(const float *__restrict__ x, long long ldx,
                                                  int rows, int n_in, bf16_t *__restrict__ out) {
  const int per = n_in / 8;
  const size_t id = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= (size_t)rows * per) return;
  const int r = (int)(id / per), e = (int)(id - (size_t)r * per) * 8;
  float v[8];
  load8(x + r * ldx + e, v);
#pragma unroll
  for (int p = 0; p < 3; ++p) {
    u32x4_t q;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = __float_as_uint(v[2 * i]), b = __float_as_uint(v[2 * i + 1]);
      q[i] = (a >> 16) | (b & 0xffff0000u);
      v[2 * i] -= __uint_as_float(a & 0xffff0000u);
      v[2 * i + 1] -= __uint_as_float(b & 0xffff0000u);
    }
    *reinterpret_cast<bf16x8_t *>(out + ((size_t)p * rows + r) * n_in + e) = order8(q);
  }
}

__device__ __forceinline__ void w4_put(const W4Args &a, int r, int o, float y) {
  const size_t at = r * a.ldy + o;
  if (a.resid) y += a.resid[at];
  if (a.y_dtype == AKVS_BF16) store1(reinterpret_cast<bf16_t *>(a.y) + at, y);
  else reinterpret_cast<float *>(a.y)[at] = y;
}

// Up to 16 rows. Block: 16 outputs, or NW = 2 of these tiles (with SWIGLU a gate's and an up's);
// its waves take runs of 512 elements in turn, codes a run ahead, and are summed in order through
// LDS. MFMA 16x16x32, rows of x as rows, outputs as columns: a lane holds 4 rows of one output,
// whose scale and zero it has itself.
template <int NW, int XP, bool SWIGLU>
__global__ __launch_bounds__(1024, 4) void k_w4_rows(W4Args a, W4X<XP> x, int ldx, int row0) {
  extern __shared__ float s_y[];  // [waves][NW][16][16 + 1]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int g = lane >> 4, lr = lane & 15;
  const int wide = SWIGLU ? a.n_out / 2 : a.n_out;
  const int o0 = blockIdx.x * 16 * (SWIGLU ? NW / 2 : NW);
  const int groups = a.n_in / 64, rows = min(a.rows - row0, 16);
  const uint8_t *w[NW];
  const uint32_t *meta[NW];
#pragma unroll
  for (int t = 0; t < NW; ++t) {  // (outputs past the last read its weights again)
    const int o = SWIGLU ? min(o0 + (t >> 1) * 16 + lr, wide - 1) + (t & 1) * wide
                         : min(o0 + t * 16 + lr, wide - 1);
    w[t] = a.w + (size_t)o * (a.n_in / 2);
    meta[t] = a.meta + (size_t)o * groups;
  }
  const size_t xrow = (size_t)(row0 + min(lr, rows - 1)) * ldx;
  f32x4_t y[NW];
#pragma unroll
  for (int t = 0; t < NW; ++t) y[t] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
  const CodeBits cb = bf16_bits();
  const bf16x8_t m16 = __builtin_bit_cast(
      bf16x8_t, (u32x4_t){0xc180c180u, 0xc180c180u, 0xc180c180u, 0xc180c180u});  // -16
  const int runs = (a.n_in + W4_RUN - 1) / W4_RUN, last_byte = a.n_in / 2 - 16;
  // codes of unit u of the run; meta of unit g of it, both groups
  auto codes = [&](int t, int run, int u) __attribute__((always_inline)) {
    return *reinterpret_cast<const u32x4_t *>(w[t] + min(run * (W4_RUN / 2) + u * 64 + g * 16, last_byte));
  };
  struct Meta {
    uint32_t a, b;
  };
  auto metas = [&](int t, int run) __attribute__((always_inline)) {
    const int gr = run * 8 + g * 2;
    return Meta{meta[t][min(gr, groups - 1)], meta[t][min(gr + 1, groups - 1)]};
  };
  if (wave < runs) {
    u32x4_t c[NW][4];
    Meta md[NW];
#pragma unroll
    for (int t = 0; t < NW; ++t) {
      md[t] = metas(t, wave);
#pragma unroll
      for (int u = 0; u < 4; ++u) c[t][u] = codes(t, wave, u);
    }
    for (int run = wave; run < runs; run += waves) {
      const int next = min(run + waves, runs - 1);
      uint32_t ma[NW][4], mb[NW][4];
#pragma unroll
      for (int t = 0; t < NW; ++t) {
        spread4(md[t].a, ma[t]);
        spread4(md[t].b, mb[t]);
        md[t] = metas(t, next);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int k = run * W4_RUN + u * W4_UNIT;
        if (k >= a.n_in) break;
        const bool both = k + 64 < a.n_in;
        bf16x8_t xf[XP][2][2];
#pragma unroll
        for (int p = 0; p < XP; ++p)
#pragma unroll
          for (int gr = 0; gr < 2; ++gr)
#pragma unroll
            for (int st = 0; st < 2; ++st)
              xf[p][gr][st] = x.get(p, xrow + k + (gr && both ? 64 : 0) + w4_first(g) + st * 8);
        f32x4_t off[2];
#pragma unroll
        for (int gr = 0; gr < 2; ++gr) {
          off[gr] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int p = 0; p < XP; ++p)
#pragma unroll
            for (int st = 0; st < 2; ++st)
              off[gr] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[p][gr][st], m16, off[gr], 0, 0, 0);
        }
#pragma unroll
        for (int t = 0; t < NW; ++t) {
          uint32_t cw[2][2] = {{c[t][u][0], c[t][u][1]}, {c[t][u][2], c[t][u][3]}};
          swap_halves(cw[0][0], cw[1][0]);
          swap_halves(cw[0][1], cw[1][1]);
          c[t][u] = codes(t, next, u);
#pragma unroll
          for (int gr = 0; gr < 2; ++gr) {
            if (gr && !both) break;
            f32x4_t s = off[gr];
#pragma unroll
            for (int st = 0; st < 2; ++st) {
              const bf16x8_t wf = codes8(cw[gr][st], cb);
#pragma unroll
              for (int p = 0; p < XP; ++p)
                s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[p][gr][st], wf, s, 0, 0, 0);
            }
            const uint32_t m = gr ? mb[t][u] : ma[t][u];
            const float scale = scale_of(m), zero = -0.0625f * zero_of(m);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[t][i] = fmaf(scale, s[i], fmaf(zero, off[gr][i], y[t][i]));
          }
        }
      }
    }
  }
  // y[t][i]: row 4 g + i of output lr of tile t
  constexpr int ST = 17;
#pragma unroll
  for (int t = 0; t < NW; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) s_y[((wave * NW + t) * 16 + 4 * g + i) * ST + lr] = y[t][i];
  __syncthreads();
  constexpr int TILES = SWIGLU ? NW / 2 : NW;
  for (int e = threadIdx.x; e < TILES * 256; e += blockDim.x) {
    const int t = e >> 8, r = (e >> 4) & 15, c = e & 15, o = o0 + t * 16 + c;
    if (r >= rows || o >= wide) continue;
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int h = 0; h < (SWIGLU ? 2 : 1); ++h) {
      const float *p = s_y + ((SWIGLU ? 2 * t + h : t) * 16 + r) * ST + c;
      for (int v = 0; v < waves; ++v) s[h] += p[v * NW * 16 * ST];
    }
    w4_put(a, row0 + r, o, SWIGLU ? silu(s[0]) * s[1] : s[0]);
  }
}

static size_t w4_planes(int rows, int n_in) { return 3 * (size_t)rows * n_in; }

size_t w4_ws_floats(int rows, int n_out, int n_in) { return (w4_planes(rows, n_in) + 1) / 2; }

template <int XP>
static hipError_t w4_rows(const W4Args &a, const W4X<XP> &x, long long ldx, hipStream_t st) {
  const int wide = a.swiglu ? a.n_out / 2 : a.n_out;
  const int runs = (a.n_in + W4_RUN - 1) / W4_RUN;
  const int waves = std::max(1, std::min(8, runs));
  for (int row0 = 0; row0 < a.rows; row0 += 16) {
    const int nw = a.swiglu ? 2 : 1;
    const dim3 g((wide + 15) / 16), b(64 * waves);
    const size_t lds = waves * nw * 16 * 17 * sizeof(float);
    if (a.swiglu)
      hipLaunchKernelGGL((k_w4_rows<2, XP, true>), g, b, lds, st, a, x, (int)ldx, row0);
    else
      hipLaunchKernelGGL((k_w4_rows<1, XP, false>), g, b, lds, st, a, x, (int)ldx, row0);
  }
  return hipGetLastError();
}

hipError_t launch_w4(const W4Args &a, float *ws, hipStream_t st) {
  if (a.rows == 0 || a.n_out == 0) return hipSuccess;
  if (a.x_dtype == AKVS_BF16)
    return w4_rows<1>(a, {reinterpret_cast<const bf16_t *>(a.x)}, a.ldx, st);
  bf16_t *planes = reinterpret_cast<bf16_t *>(ws);
  const size_t octets = (size_t)a.rows * (a.n_in / 8);
  hipLaunchKernelGGL(k_w4_split, dim3((unsigned)((octets + 255) / 256)), dim3(256), 0, st,
                     reinterpret_cast<const float *>(a.x), a.ldx, a.rows, a.n_in, planes);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return w4_rows<3>(a, {planes, (size_t)a.rows * a.n_in}, a.n_in, st);
}

}  // namespace akvs
