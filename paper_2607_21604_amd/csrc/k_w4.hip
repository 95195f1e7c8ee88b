// Products of a few rows with 4-bit weights.
//
// y = x W^T with W = scale c + zero per group of 64: for each group
//   sum x w = scale (sum x (16 + c) - 16 sum x) + zero sum x,
// where a nibble c put into the upper mantissa bits of a bf16 of 16 is 16 + c, exactly, so that the
// weights go to the matrix cores without a rounding, two in an instruction. A group's sum x is
// formed once, in fp32; sum zero sum x over the groups is a matrix product of its own, 1 / 64 as
// long. x in bf16 is taken as it is, in fp32 as three bf16 that add up to it.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "four_bit_dev.h"
#include "gemm_dev.h"
#include "kernels.h"
#include "quant_dev.h"

namespace akvs {

constexpr int W4_UNIT = 128;        // two groups: 64 bytes of a row of codes
constexpr int W4_RUN = 4 * W4_UNIT; // what a wave takes at a time

// Lane l, g = l / 16, loads 16 of a unit's 64 bytes of row l % 16, so that lanes 0..31 hold its first
// group and lanes 32..63 its second. Swapping halves leaves one group in each pair of words, and
// lane g with elements w4_first(g) .. + 15 of it.
__device__ __forceinline__ int w4_first(int g) { return ((g & 1) << 5) + ((g >> 1) << 4); }

// How a call is cut: a block has `slice` runs of the reduction (of blockIdx.y), its rows of x in LDS
// for `held` of them at a time, and waves / wk tiles of outputs, whose runs wk waves share.
struct W4Plan {
  int nw, waves, wk, slice, held, slices, rows;  // nw: tiles of a wave; rows: of x in the block
};

// Octets of x that a thread requests at a time on their way to LDS; parts: of an element.
constexpr int w4_batch(int parts) { return parts == 1 ? 8 : 4; }

__device__ __forceinline__ void w4_put(const W4Args &a, int r, int o, float y) {
  const size_t at = r * a.ldy + o;
  if (a.resid) y += a.resid[at];
  if (a.y_dtype == AKVS_BF16) store1(reinterpret_cast<bf16_t *>(a.y) + at, y);
  else reinterpret_cast<float *>(a.y)[at] = y;
}

// fp32 elements as XP = 3 bf16 parts (truncated, so that each difference is exact), bf16 as they are.
__device__ __forceinline__ u32x4_t w4_part(const bf16_t *, u32x4_t &x, float (&)[8]) { return x; }
__device__ __forceinline__ u32x4_t w4_part(const float *, u32x4_t &, float (&v)[8]) {
  u32x4_t q;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = __float_as_uint(v[2 * i]), b = __float_as_uint(v[2 * i + 1]);
    q[i] = (a >> 16) | (b & 0xffff0000u);
    v[2 * i] -= __uint_as_float(a & 0xffff0000u);
    v[2 * i + 1] -= __uint_as_float(b & 0xffff0000u);
  }
  return q;
}
__device__ __forceinline__ void w4_read(const bf16_t *p, u32x4_t &x, float (&)[8]) {
  x = *reinterpret_cast<const u32x4_t *>(p);
}
__device__ __forceinline__ void w4_read(const float *p, u32x4_t &, float (&v)[8]) { load8(p, v); }
__device__ __forceinline__ float octet_sum(const bf16_t *, const u32x4_t &x, const float (&)[8]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    s += __uint_as_float(x[i] << 16) + __uint_as_float(x[i] & 0xffff0000u);
  return s;
}
__device__ __forceinline__ float octet_sum(const float *, const u32x4_t &, const float (&v)[8]) {
  return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}

// A wave has 16 outputs, or NW tiles of them (with SWIGLU tiles of gate and up in turn), and NX
// tiles of 16 rows. MFMA 16x16x32, rows of x as rows, outputs as columns: a lane holds 4 rows of
// one output, whose scale and zero it has itself. x goes to LDS, every 8 elements in the order of
// the codes; codes are loaded a run ahead.
//   5 rows 5120 -> 55296 (gate and up): 39 us, 4.0 TB/s of codes and meta. Loads take 64 bytes of 16
//   rows; whole lines of 8 rows would stream 4 us faster, and lose as much on the lanes' exchange.
//   33 rows 27648 -> 5120: 32 us, and 5 for the sums of 18 slices: x of a block (101 KB) enters before
//   its first product. 64 rows 5120 -> 55296: 83 us, products and their x from LDS.
template <int NW, int NX, typename TX, bool SWIGLU>
__global__ __launch_bounds__(768, 3) void k_w4(W4Args a, W4Plan p, int row0, float *part) {
  constexpr int XP = std::is_same<TX, float>::value ? 3 : 1;
  constexpr bool UNITS_WHOLE = NX == 1 && NW == 1;
  extern __shared__ __attribute__((aligned(16))) char s_x[];  // [XP][rows][held], then sums
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, lr = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wk = wave % p.wk, wn = wave / p.wk;
  const int wide = SWIGLU ? a.n_out / 2 : a.n_out, groups = a.n_in / 64;
  constexpr int TILES = SWIGLU ? NW / 2 : NW;  // of the result
  const int o0 = (blockIdx.x * (p.waves / p.wk) + wn) * 16 * TILES;
  const int k0 = blockIdx.y * p.slice * W4_RUN, k1 = min(a.n_in, k0 + p.slice * W4_RUN);
  const int stride = p.held * W4_RUN * 2 + 16;  // bytes of a row of x
  const uint8_t *w[NW];
  const uint32_t *meta[NW];
#pragma unroll
  for (int t = 0; t < NW; ++t) {  // (outputs past the last read its weights again)
    const int o = SWIGLU ? min(o0 + (t >> 1) * 16 + lr, wide - 1) + (t & 1) * wide
                         : min(o0 + t * 16 + lr, wide - 1);
    w[t] = a.w + (size_t)o * (a.n_in / 2);
    meta[t] = a.meta + (size_t)o * groups;
  }
  const int last_byte = a.n_in / 2 - 16;
  // codes of unit u from element k on; meta of unit g, both groups
  auto codes = [&](int t, int k, int u) __attribute__((always_inline)) {
    return *reinterpret_cast<const u32x4_t *>(w[t] + min(k / 2 + u * 64 + g * 16, last_byte));
  };
  struct Meta {
    uint32_t a, b;
  };
  auto metas = [&](int t, int k) __attribute__((always_inline)) {
    const int gr = k / 64 + g * 2;
    return Meta{meta[t][min(gr, groups - 1)], meta[t][min(gr + 1, groups - 1)]};
  };
  const bool live = o0 < wide;  // (waves past the last output only load x)
  u32x4_t c[NW][4];
  Meta md[NW];
  int k = k0 + wk * W4_RUN;
  const int step = p.wk * W4_RUN;
  // -16 times the sums of x over groups, [group][16 NX rows]; rows past the last are the last one's
  constexpr int XR = 16 * NX;
  float *s_sum = reinterpret_cast<float *>(s_x + (size_t)XP * p.rows * stride);
  if (live && k < k1) {
#pragma unroll
    for (int t = 0; t < NW; ++t) {
      md[t] = metas(t, k);
#pragma unroll
      for (int u = 0; u < 4; ++u) c[t][u] = codes(t, k, u);
    }
  }
  // x from element kb to ke, its octets row by row, BATCH of a thread requested at a time
  auto stage = [&](int kb, int ke) __attribute__((always_inline)) {
    constexpr int BATCH = w4_batch(XP);
    const int per = (ke - kb) / 8, total = p.rows * per, threads = p.waves * 64;
    const int rows_on = threads / per, on = threads % per;  // of a thread's next octet
    int r = tid / per, e = tid % per;
    for (int i = tid; i < total; i += BATCH * threads) {
      u32x4_t x[BATCH];
      float v[BATCH][8];
      int at_r[BATCH], at_e[BATCH];
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        at_r[b] = r;
        at_e[b] = e;
        r += rows_on;
        e += on;
        if (e >= per) {
          e -= per;
          ++r;
        }
        if (i + b * threads < total)
          w4_read(reinterpret_cast<const TX *>(a.x) + (row0 + at_r[b]) * a.ldx + kb + at_e[b] * 8,
                  x[b], v[b]);
      }
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        if (i + b * threads >= total) break;  // (the same for the 8 lanes of a group)
        float sum = octet_sum(static_cast<const TX *>(nullptr), x[b], v[b]);
#pragma unroll
        for (int q = 0; q < XP; ++q)
          *reinterpret_cast<bf16x8_t *>(s_x + (q * p.rows + at_r[b]) * stride + at_e[b] * 16) =
              order8(w4_part(static_cast<const TX *>(nullptr), x[b], v[b]));
        sum = -16.f * oct_sum(sum);
        if ((lane & 7) == 0)
          for (int row = at_r[b]; row < (at_r[b] == p.rows - 1 ? XR : at_r[b] + 1); ++row)
            s_sum[at_e[b] / 8 * XR + row] = sum;
      }
    }
  };
  f32x4_t y[NW][NX];
#pragma unroll
  for (int t = 0; t < NW; ++t)
#pragma unroll
    for (int n = 0; n < NX; ++n) y[t][n] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
  const CodeBits cb = bf16_bits();
  const char *x0[NX];
#pragma unroll
  for (int n = 0; n < NX; ++n)
    x0[n] = s_x + min(n * 16 + lr, p.rows - 1) * stride + w4_first(g) * 2;
  // sum zero sum x over a run's eight groups: lane g has the zeros of two, in two bf16 parts (11
  // bits), and takes the sums in three; 2 x 2 places of its eight for each part of the sums
  auto zeros = [&](int k, int kb) __attribute__((always_inline)) {
    const int gr = (k - kb) / 64 + g * 2;
    const bool in0 = k + g * 128 < k1, in1 = k + g * 128 + 64 < k1;
    bf16x8_t zf[NW];
#pragma unroll
    for (int t = 0; t < NW; ++t) {
      const float za = in0 ? -0.0625f * zero_of(md[t].a) : 0.f;
      const float zb = in1 ? -0.0625f * zero_of(md[t].b) : 0.f;
      const uint32_t a = __float_as_uint(za), b = __float_as_uint(zb);
      const uint32_t hi = (a >> 16) | (b & 0xffff0000u);
      const uint32_t lo = (__float_as_uint(za - __uint_as_float(a & 0xffff0000u)) >> 16) |
                          (__float_as_uint(zb - __uint_as_float(b & 0xffff0000u)) & 0xffff0000u);
      zf[t] = __builtin_bit_cast(bf16x8_t, (u32x4_t){hi, lo, hi, lo});
    }
#pragma unroll
    for (int n = 0; n < NX; ++n) {
      float v[2] = {in0 ? s_sum[gr * XR + n * 16 + lr] : 0.f,
                    in1 ? s_sum[(gr + 1) * XR + n * 16 + lr] : 0.f};
      uint32_t q[3];
#pragma unroll
      for (int e = 0; e < 3; ++e) {
        const uint32_t a = __float_as_uint(v[0]), b = __float_as_uint(v[1]);
        q[e] = (a >> 16) | (b & 0xffff0000u);
        v[0] -= __uint_as_float(a & 0xffff0000u);
        v[1] -= __uint_as_float(b & 0xffff0000u);
      }
      const bf16x8_t x01 = __builtin_bit_cast(bf16x8_t, (u32x4_t){q[0], q[0], q[1], q[1]});
      const bf16x8_t x2 = __builtin_bit_cast(bf16x8_t, (u32x4_t){q[2], q[2], 0u, 0u});
#pragma unroll
      for (int t = 0; t < NW; ++t) {
        y[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x01, zf[t], y[t][n], 0, 0, 0);
        y[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x2, zf[t], y[t][n], 0, 0, 0);
      }
    }
  };
  for (int kb = k0; kb < k1; kb += p.held * W4_RUN) {
    const int ke = min(k1, kb + p.held * W4_RUN);
    if (kb > k0) __syncthreads();  // (x of the runs before is read)
    stage(kb, ke);
    __syncthreads();
    if (!live) continue;
    for (k = kb + wk * W4_RUN; k < ke; k += step) {
      // the next run of this wave, maybe of the next x; none: any
      const int then = k + step < ke ? k + step : ke + wk * W4_RUN;
      const int next = min(then, a.n_in - 1) / W4_RUN * W4_RUN;
      uint32_t ma[NW][4], mb[NW][4];
#pragma unroll
      for (int t = 0; t < NW; ++t) {
        spread4(md[t].a, ma[t]);
        spread4(md[t].b, mb[t]);
      }
      zeros(k, kb);
#pragma unroll
      for (int t = 0; t < NW; ++t) md[t] = metas(t, next);
      // (whole runs without a branch, so that LDS reads go ahead of the products)
      auto units = [&](auto whole) __attribute__((always_inline)) {
        constexpr bool WHOLE = decltype(whole)::value;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int ku = k + u * W4_UNIT;
          if (!WHOLE && ku >= k1) break;
          const bool both = WHOLE || ku + 64 < k1;
          uint32_t cw[NW][2][2];
#pragma unroll
          for (int t = 0; t < NW; ++t) {
            cw[t][0][0] = c[t][u][0];
            cw[t][0][1] = c[t][u][1];
            cw[t][1][0] = c[t][u][2];
            cw[t][1][1] = c[t][u][3];
            swap_halves(cw[t][0][0], cw[t][1][0]);
            swap_halves(cw[t][0][1], cw[t][1][1]);
          }
          // (the two halves of a line one right after the other: 5 rows 5120 -> 55296 from memory
          // 48 us a unit at a time, 42 in pairs)
          if ((u & 1) && then < k1) {
#pragma unroll
            for (int t = 0; t < NW; ++t) {
              c[t][u - 1] = codes(t, next, u - 1);
              c[t][u] = codes(t, next, u);
            }
          }
#pragma unroll
          for (int gr = 0; gr < 2; ++gr) {
            if (gr && !both) break;
            bf16x8_t wf[NW][2];
#pragma unroll
            for (int t = 0; t < NW; ++t)
#pragma unroll
              for (int st = 0; st < 2; ++st) wf[t][st] = codes8(cw[t][gr][st], cb);
#pragma unroll
            for (int n = 0; n < NX; ++n) {
              bf16x8_t xf[XP][2];
#pragma unroll
              for (int q = 0; q < XP; ++q)
#pragma unroll
                for (int st = 0; st < 2; ++st)
                  xf[q][st] = *reinterpret_cast<const bf16x8_t *>(
                      x0[n] + q * p.rows * stride + (ku - kb + gr * 64 + st * 8) * 2);
              const f32x4_t off = *reinterpret_cast<const f32x4_t *>(
                  s_sum + ((ku - kb) / 64 + gr) * XR + n * 16 + 4 * g);
#pragma unroll
              for (int t = 0; t < NW; ++t) {
                f32x4_t s = off;
#pragma unroll
                for (int q = 0; q < XP; ++q)
#pragma unroll
                  for (int st = 0; st < 2; ++st)
                    s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[q][st], wf[t][st], s, 0, 0, 0);
                const uint32_t m = gr ? mb[t][u] : ma[t][u];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[t][n][i] = fmaf(scale_of(m), s[i], y[t][n][i]);
              }
            }
          }
        }
      };
      if (UNITS_WHOLE && k + W4_RUN <= k1) units(std::true_type{});
      else units(std::false_type{});
    }
  }
  // y[t][n][i]: row 16 n + 4 g + i of output lr of tile t
  if (p.wk > 1) {  // the waves of a tile in order, through LDS
    constexpr int ST = 17, SIZE = NW * NX * 16 * ST;
    float *s_y = s_sum + p.held * (W4_RUN / 64) * XR;
    float *mine = s_y + wave * SIZE;
#pragma unroll
    for (int t = 0; t < NW; ++t)
#pragma unroll
      for (int n = 0; n < NX; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          mine[((t * NX + n) * 16 + 4 * g + i) * ST + lr] = y[t][n][i];
    __syncthreads();
    const float *first = s_y + wn * p.wk * SIZE;
    for (int e = wk * 64 + lane; e < TILES * NX * 256; e += p.wk * 64) {
      const int t = e / (NX * 256), r = e / 16 % (NX * 16), col = e & 15, o = o0 + t * 16 + col;
      if (r >= p.rows || o >= wide) continue;
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int h = 0; h < (SWIGLU ? 2 : 1); ++h) {
        const float *q = first + ((SWIGLU ? 2 * t + h : t) * NX * 16 + r) * ST + col;
        for (int v = 0; v < p.wk; ++v) s[h] += q[v * SIZE];
      }
      if (part) {
#pragma unroll
        for (int h = 0; h < (SWIGLU ? 2 : 1); ++h)
          part[((size_t)blockIdx.y * p.rows + r) * a.n_out + o + h * wide] = s[h];
      } else {
        w4_put(a, row0 + r, o, SWIGLU ? silu(s[0]) * s[1] : s[0]);
      }
    }
    return;
  }
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const int o = o0 + t * 16 + lr;
    if (o >= wide) continue;
#pragma unroll
    for (int n = 0; n < NX; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = n * 16 + 4 * g + i;
        if (r >= p.rows) continue;
        const float s = y[SWIGLU ? 2 * t : t][n][i], u = SWIGLU ? y[SWIGLU ? 2 * t + 1 : 0][n][i] : 0.f;
        if (part) {
          float *q = part + ((size_t)blockIdx.y * p.rows + r) * a.n_out + o;
          q[0] = s;
          if (SWIGLU) q[wide] = u;
        } else {
          w4_put(a, row0 + r, o, SWIGLU ? silu(s) * u : s);
        }
      }
  }
}

// The slices' sums in order, and what is made of them. Eight of them are requested at a time.
__device__ __forceinline__ float w4_slices(const float *p, size_t all, int slices) {
  float s = 0.f;
  for (int q0 = 0; q0 < slices; q0 += 8) {
    float x[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) x[q] = p[min(q0 + q, slices - 1) * all];
#pragma unroll
    for (int q = 0; q < 8; ++q) s += q0 + q < slices ? x[q] : 0.f;
  }
  return s;
}
__global__ __launch_bounds__(256) void k_w4_sum(W4Args a, int slices, int rows, int row0,
                                                const float *__restrict__ part) {
  const int wide = a.swiglu ? a.n_out / 2 : a.n_out;
  const size_t id = (size_t)blockIdx.x * 256 + threadIdx.x, all = (size_t)rows * a.n_out;
  if (id >= (size_t)rows * wide) return;
  const int r = (int)(id / wide), o = (int)(id - (size_t)r * wide);
  const float *p = part + (size_t)r * a.n_out + o;
  float s = w4_slices(p, all, slices);
  if (a.swiglu) s = silu(s) * w4_slices(p + wide, all, slices);
  w4_put(a, row0 + r, o, s);
}

// Rows in one read of the weights.
static int w4_most_rows(int parts) { return parts == 1 ? 64 : 32; }
// LDS of a block: x, its sums, and with shared tiles their parts.
static size_t w4_lds(const W4Plan &p, int parts) {
  const int nx = (p.rows + 15) / 16;
  return (size_t)parts * p.rows * (p.held * W4_RUN * 2 + 16) +
         p.held * (W4_RUN / 64) * 16 * nx * sizeof(float) +
         (p.wk > 1 ? p.waves * p.nw * nx * 16 * 17 * sizeof(float) : 0);
}

// The cut (slices of the reduction, runs whose x is held, waves of a block, waves that share a tile)
// whose estimated end is the earliest, in us: a block takes FIXED, STAGE and a TRIP to memory for every
// batch of the x that it takes in, then its waves' runs at the rate of a unit's instructions or of its
// share of the memory, whichever is slower, and 1 at least; whole rounds of resident blocks follow each
// other; slices take another launch. Few outputs are sliced, to fill the device; many are not, their
// blocks take x in turns: no partial sums.
//   1 row 3584 -> 4608: 4 of 8 waves a tile 6.9 us, 8 of 8 7.4, 4 of 4 7.4, 2 of 4 7.9, 1 of 4 10.1.
//   5 rows 5120 -> 55296 (SWIGLU): a wave a tile 41, two 41, blocks of 4 waves 43, 2 slices 46.
//   64 rows 5120 -> 55296 (SWIGLU): x of 2 runs in 5 turns 83, in 5 slices 101.
//   17 rows 5120 -> 7168: 4 slices in blocks of 8 waves 14, of 4 waves with two tiles each 20, 2
//   turns of 5 runs 25.
//   33 rows 27648 -> 5120: 18 slices in blocks of 12 waves (one round) 36, of 8 47, 27 slices 47, 54
//   58.
static W4Plan w4_make_plan(int rows, int n_out, int n_in, bool swiglu, int parts, int cus) {
  constexpr double FIXED = 2.5, STAGE = 1, TRIP = 1.2, CYCLES = 1300, BYTES = 5.2e6;
  constexpr size_t LDS = 160 << 10;
  W4Plan p, best;
  p.rows = std::min(rows, w4_most_rows(parts));
  const int nx = (p.rows + 15) / 16;
  const int runs = (n_in + W4_RUN - 1) / W4_RUN;
  const size_t run_lds = (size_t)parts * p.rows * W4_RUN * 2 + (W4_RUN / 64) * 16 * nx * sizeof(float);
  double least = 1e30;
  auto consider = [&](int slices) {
    p.slice = (runs + slices - 1) / slices;
    p.slices = (runs + p.slice - 1) / p.slice;
    for (int nw : {1, 2}) {
      if (swiglu ? nw == 1 : nw == 2 && nx == 1) continue;
      p.nw = nw;
      const long long tiles = (n_out + 16 * nw - 1) / (16 * nw);
      // resident waves of a SIMD (by registers), and cycles of a run's instructions
      const int occ = nx == 1 && (nw == 1 || parts == 1) ? 4 : 3;
      const double cycles = 4 * (4.0 * (8 + 31 * nw + 9 * nx * nw) + 16.0 * 4 * nx * nw * parts);
      for (int waves : {8, 4, 12})  // (8 where the estimate is the same)
        for (int wk : {1, 2, 4, 8}) {
          if (waves % wk || (wk > 1 && wk > p.slice)) continue;
          p.waves = waves;
          p.wk = wk;
          p.held = 0;
          const size_t rest = w4_lds(p, parts);  // beside the x and sums of held runs
          for (int share : {1, 2}) {             // blocks of a unit that LDS is for
            if (rest + run_lds > LDS / share) break;
            const int most = (int)std::min<size_t>(p.slice, (LDS / share - rest) / run_lds);
            const int times = (p.slice + most - 1) / most;
            p.held = (p.slice + times - 1) / times;
            if (p.held < wk) continue;  // (a wave has a run of every x)
            const size_t lds = rest + p.held * run_lds;
            const int each = std::max(1, (int)std::min<size_t>(LDS / lds, occ * 4 / waves));
            const long long blocks = (tiles * wk + waves - 1) / waves * p.slices;
            const double rounds = std::ceil((double)blocks / (cus * each));
            const double resident = std::min<double>(each, std::ceil((double)blocks / cus)) * waves;
            const double run = std::max(
                {1.0, cycles * std::max(1.0, resident / 4) / CYCLES,
                 resident * std::min<double>(cus, blocks) * nw * 16 * W4_RUN * 0.5625 / BYTES});
            // (x's octets, w4_batch of a thread requested at a time)
            const int threads = waves * 64 * w4_batch(parts);
            const double stage =
                STAGE + TRIP * ((p.rows * p.held * (W4_RUN / 8) + threads - 1) / threads);
            const double walk = (p.slice + wk - 1) / wk * run;
            const double t = rounds * (FIXED + times * stage + walk) + (wk > 1 ? 0.5 : 0) +
                             (p.slices > 1 ? 4 + 1e-6 * p.slices * p.rows * n_out : 0);
            if (t < least) {
              least = t;
              best = p;
            }
            if (times == 1) break;
          }
        }
    }
  };
  // the fewest slices, and from about as few as their x is held whole
  const int whole = (int)std::max<size_t>(1, LDS / run_lds);
  int slices = 1;
  for (int n = 0; n < 8 && slices <= runs; ++n) {
    if (n == 4) slices = std::max(slices, (runs + whole - 1) / whole);
    consider(slices);
    slices = p.slice > 1 ? (runs + p.slice - 2) / (p.slice - 1) : runs + 1;
  }
  return best;
}

// The same, kept per thread for the sizes that come again (1.5 us of a call's 8 otherwise).
static W4Plan w4_plan(int rows, int n_out, int n_in, bool swiglu, int parts) {
  struct Known {
    int rows, n_out, n_in, kind, cus;
    W4Plan plan;
  };
  thread_local Known known[64] = {};
  rows = std::min(rows, w4_most_rows(parts));  // (what the plan is of)
  const int kind = 2 * parts + swiglu, cus = gemm_cu_count();
  Known &k = known[(rows * 7u + n_out / 16 * 3u + n_in / 64 * 5u + kind) % 64];
  if (k.rows != rows || k.n_out != n_out || k.n_in != n_in || k.kind != kind || k.cus != cus)
    k = {rows, n_out, n_in, kind, cus, w4_make_plan(rows, n_out, n_in, swiglu, parts, cus)};
  return k.plan;
}

static size_t w4_part_floats(const W4Plan &p, int n_out) {
  return p.slices > 1 ? (size_t)p.slices * p.rows * n_out : 0;
}

size_t w4_ws_floats(int rows, int n_out, int n_in, bool swiglu, int x_dtype) {
  if (rows == 0 || n_out == 0) return 0;
  return w4_part_floats(w4_plan(rows, n_out, n_in, swiglu, x_dtype == AKVS_BF16 ? 1 : 3), n_out);
}

template <int NW, int NX, typename TX, bool SWIGLU>
static hipError_t w4_launch(const W4Args &a, const W4Plan &p, int row0, float *part,
                            hipStream_t st) {
  constexpr int XP = std::is_same<TX, float>::value ? 3 : 1;
  const int per = 16 * (SWIGLU ? NW / 2 : NW) * (p.waves / p.wk);
  const int wide = SWIGLU ? a.n_out / 2 : a.n_out;
  const dim3 g((wide + per - 1) / per, p.slices), b(64 * p.waves);
  const size_t lds = w4_lds(p, XP);
  hipLaunchKernelGGL((k_w4<NW, NX, TX, SWIGLU>), g, b, lds, st, a, p, row0, part);
  return hipGetLastError();
}

template <typename TX, bool SWIGLU>
static hipError_t w4_rows(const W4Args &a, const W4Plan &p, int row0, float *part, hipStream_t st) {
  const int nx = (p.rows + 15) / 16;
  if (nx == 1) return w4_launch<SWIGLU ? 2 : 1, 1, TX, SWIGLU>(a, p, row0, part, st);
  if constexpr (!SWIGLU) {
    if (p.nw == 1) {
      if constexpr (std::is_same<TX, bf16_t>::value) {
        if (nx == 3) return w4_launch<1, 3, TX, false>(a, p, row0, part, st);
        if (nx == 4) return w4_launch<1, 4, TX, false>(a, p, row0, part, st);
      }
      return w4_launch<1, 2, TX, false>(a, p, row0, part, st);
    }
  }
  if constexpr (std::is_same<TX, bf16_t>::value) {
    if (nx == 3) return w4_launch<2, 3, TX, SWIGLU>(a, p, row0, part, st);
    if (nx == 4) return w4_launch<2, 4, TX, SWIGLU>(a, p, row0, part, st);
  }
  return w4_launch<2, 2, TX, SWIGLU>(a, p, row0, part, st);
}

hipError_t launch_w4(const W4Args &a, float *ws, hipStream_t st) {
  if (a.rows == 0 || a.n_out == 0) return hipSuccess;
  const bool bf = a.x_dtype == AKVS_BF16;
  W4Plan p = w4_plan(a.rows, a.n_out, a.n_in, a.swiglu, bf ? 1 : 3);
  float *part = p.slices > 1 ? ws : nullptr;
  const int most = p.rows;
  for (int row0 = 0; row0 < a.rows; row0 += most) {
    p.rows = std::min(most, a.rows - row0);
    if (p.rows <= 16 && !a.swiglu) p.nw = 1;  // (the last rows of many)
    hipError_t e = bf ? (a.swiglu ? w4_rows<bf16_t, true>(a, p, row0, part, st)
                                  : w4_rows<bf16_t, false>(a, p, row0, part, st))
                      : (a.swiglu ? w4_rows<float, true>(a, p, row0, part, st)
                                  : w4_rows<float, false>(a, p, row0, part, st));
    if (e != hipSuccess) return e;
    if (!part) continue;
    const size_t n = (size_t)p.rows * (a.swiglu ? a.n_out / 2 : a.n_out);
    hipLaunchKernelGGL(k_w4_sum, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, a, p.slices,
                       p.rows, row0, part);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace akvs
