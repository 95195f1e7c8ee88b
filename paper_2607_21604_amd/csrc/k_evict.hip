// Eviction from caches by accumulated attention weight: selection of the kept keys, then the
// gather of their rows.
#include "kernels.h"

namespace akvs {

// Order of the weights as unsigned numbers: 1 for a NaN, then -inf .. +inf, -0 as +0. (0 is
// left for what is no key and 0xffffffff for keys that are kept without comparison: -inf maps to
// 0x007fffff, +inf to 0xff800000.)
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);  // (-0 + 0 = +0)
  const uint32_t k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  return w != w ? 1u : k;
}

// Block = one KV head of one sequence, NW waves; wave w has the keys [w * per, (w + 1) * per), R
// of a lane's at a time in registers (ONE: all of them, read once). The smallest kept candidate
// T is found a digit at a time (11, 11 and 10 bits): a histogram in LDS of the candidates that
// agree with T so far, its counts summed from the top by all threads, and the bin in which the
// count reaches what is wanted. Then each wave lists its kept keys in order; of the keys equal
// to T the first are kept. Short sequences are bound by a dozen barriers and the LDS round
// trips between them (6 us at 300 keys, 11 at 4516), long ones by the instructions per key on
// one compute unit; neither depends on how many heads there are up to 256.
constexpr int EV_BINS = 2048;
template <int NW, int R, bool ONE>
__global__ __launch_bounds__(NW * 64) void k_evict_select(const float *__restrict__ weights,
                                                          EvictArgs a, int hkv,
                                                          int32_t *__restrict__ keep,
                                                          float *__restrict__ w_out) {
  constexpr int T_ = NW * 64, PER_T = EV_BINS / T_;
  __shared__ int hist[EV_BINS];
  __shared__ __attribute__((aligned(16))) int s_wave[NW], s_gt[NW], s_eq[NW];
  __shared__ int s_pick[2];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int seq = blockIdx.x / hkv;
  const float *w = weights + (size_t)blockIdx.x * a.n_keys;
  keep += (size_t)blockIdx.x * a.n_keep;
  if (w_out) w_out += (size_t)blockIdx.x * a.dst_rows;
  const int n = a.lens ? min(max(a.lens[seq], 0), a.n_keys) : a.n_keys;
  const int kept = min(n, a.n_keep);
  const bool all = n <= a.n_keep;
  // candidates [c0, c1), of which `want` are kept; the keys beside them are kept, as is every key
  // where there are no more than may be
  const int want = a.n_keep - a.n_first - a.n_recent;
  const int c0 = all ? n : a.n_first, c1 = all ? n : n - a.n_recent;
  const int steps = (n + T_ - 1) / T_, b0 = wave * steps * 64, b1 = min(b0 + steps * 64, n);
  uint32_t key[R];
  auto read = [&](int s0) __attribute__((always_inline)) {
    float x[R];
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (s0 + i < steps) x[i] = w[min(b0 + (s0 + i) * 64 + lane, n - 1)];
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (s0 + i < steps) {
        const int j = b0 + (s0 + i) * 64 + lane;
        key[i] = j >= c0 && j < c1 ? weight_key(x[i]) : 0xffffffffu;
        if (j >= b1) key[i] = 0u;
      }
  };
  if (ONE) read(0);
  // f(key index, key) over this wave's keys (indices from b1 on: none)
  auto each = [&](auto &&f) __attribute__((always_inline)) {
    for (int s0 = 0; s0 < (ONE ? 1 : steps); s0 += R) {
      if (!ONE) read(s0);
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (s0 + i < steps) f(b0 + (s0 + i) * 64 + lane, key[i]);
    }
  };
  uint32_t T = 0xfffffffeu;  // (no candidate is kept)
  int eq_take = 0;
  if (!all && want > 0) {
    int left = want;  // how many of the candidates that agree with T are kept
    T = 0;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const int bits = pass == 2 ? 10 : 11;
#pragma unroll
      for (int i = 0; i < PER_T; ++i) hist[t + i * T_] = 0;
      __syncthreads();
      each([&](int, uint32_t u) {
        // (what is no candidate agrees with no T but the smallest)
        if (pass == 0 ? u - 1 < 0xfffffffeu : (u ^ T) < (1u << (shift + bits)) && u != 0)
          atomicAdd(&hist[(u >> shift) & ((1u << bits) - 1)], 1);
      });
      __syncthreads();
      // thread t has the bins below EV_BINS - t * PER_T, the highest first
      int h[PER_T], mine = 0;
#pragma unroll
      for (int i = 0; i < PER_T; ++i) {
        h[i] = hist[EV_BINS - 1 - (t * PER_T + i)];
        mine += h[i];
      }
      int upto = mine;  // the counts of this wave's threads up to this one
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(upto, o, 64);
        if (lane >= o) upto += x;
      }
      if (lane == 63) s_wave[wave] = upto;
      __syncthreads();
      int above = upto - mine, before[NW];
#pragma unroll
      for (int v = 0; v < NW; ++v) before[v] = s_wave[v];
#pragma unroll
      for (int v = 0; v < NW; ++v) above += v < wave ? before[v] : 0;
#pragma unroll
      for (int i = 0; i < PER_T; ++i) {
        if (above < left && above + h[i] >= left) {  // (one bin of one thread)
          s_pick[0] = EV_BINS - 1 - (t * PER_T + i);
          s_pick[1] = above;
        }
        above += h[i];
      }
      __syncthreads();
      T |= (uint32_t)s_pick[0] << shift;
      left -= s_pick[1];
    }
    eq_take = left;
  }
  int gt = 0, eq = 0;
  each([&](int, uint32_t u) {
    gt += u > T;
    eq += u == T;
  });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    gt += __shfl_xor(gt, o, 64);
    eq += __shfl_xor(eq, o, 64);
  }
  if (lane == 0) {
    s_gt[wave] = gt;
    s_eq[wave] = eq;
  }
  __syncthreads();
  int at = 0, eqs = 0;  // kept keys and keys equal to T before this wave's
  int gts[NW], es[NW];
#pragma unroll
  for (int v = 0; v < NW; ++v) {
    gts[v] = s_gt[v];
    es[v] = s_eq[v];
  }
#pragma unroll
  for (int v = 0; v < NW; ++v)
    if (v < wave) {
      at += gts[v] + min(es[v], max(eq_take - eqs, 0));
      eqs += es[v];
    }
  each([&](int j, uint32_t u) {
    unsigned long long m = __ballot(u > T);
    const unsigned long long e = __ballot(u == T);
    bool take = u > T;
    if (e) {  // (few steps have one)
      take |= u == T && eqs + (int)__popcll(e & ((1ull << lane) - 1)) < eq_take;
      m = __ballot(take);
      eqs += __popcll(e);
    }
    if (take) {
      const int i = at + (int)__popcll(m & ((1ull << lane) - 1));
      keep[i] = j;
      if (w_out) w_out[i] = w[j];
    }
    at += __popcll(m);
  });
  for (int i = kept + t; i < a.n_keep; i += T_) keep[i] = -1;
  if (w_out)
    for (int i = kept + t; i < a.dst_rows; i += T_) w_out[i] = 0.f;
}

// Rows of kept keys and their values: a thread moves 16 bytes of each of EV_U rows, all indices
// and then all loads requested at once (index, row and store are a chain of three round trips).
// Blocks (row group, sequence).
constexpr int EV_U = 4;
__global__ __launch_bounds__(256) void k_evict_gather(const u32x4_t *__restrict__ k,
                                                      const u32x4_t *__restrict__ v, EvictArgs a,
                                                      int hkv, int row16,
                                                      const int32_t *__restrict__ keep,
                                                      u32x4_t *__restrict__ k_out,
                                                      u32x4_t *__restrict__ v_out,
                                                      int32_t *lens_out) {
  const int seq = blockIdx.y;
  if (lens_out && blockIdx.x == 0 && threadIdx.x == 0) {
    const int n = a.lens ? min(max(a.lens[seq], 0), a.n_keys) : a.n_keys;
    lens_out[seq] = min(n, a.n_keep);
  }
  if (!k) return;
  const unsigned width = hkv * row16;  // 16-byte chunks of a token's row
  const unsigned id = blockIdx.x * 256 + threadIdx.x;
  const unsigned rows = (a.n_keep + EV_U - 1) / EV_U;  // this thread's rows are `rows` apart
  const unsigned i0 = id / width, ch = id - i0 * width;
  if (i0 >= rows) return;
  keep += ((size_t)seq * hkv + ch / row16) * a.n_keep;
  int j[EV_U];
#pragma unroll
  for (int u = 0; u < EV_U; ++u) {
    const unsigned i = i0 + u * rows;
    j[u] = i < (unsigned)a.n_keep ? keep[i] : -1;
    if (j[u] >= a.n_keys) j[u] = -1;
  }
  const size_t src = (size_t)seq * a.src_rows, dst = (size_t)seq * a.dst_rows;
  u32x4_t x[EV_U], y[EV_U];
#pragma unroll
  for (int u = 0; u < EV_U; ++u)
    if (j[u] >= 0) {
      x[u] = k[(src + j[u]) * width + ch];
      y[u] = v[(src + j[u]) * width + ch];
    }
#pragma unroll
  for (int u = 0; u < EV_U; ++u)
    if (j[u] >= 0) {
      k_out[(dst + i0 + u * rows) * width + ch] = x[u];
      v_out[(dst + i0 + u * rows) * width + ch] = y[u];
    }
}

// Few keys: eight waves (300 / 1500 keys 5.2 / 7.1 us, with four 5.7 / 8.5, with sixteen 6.4 / 7.9).
hipError_t launch_evict_select(const float *weights, const EvictArgs &a, int hkv, int32_t *keep,
                               float *w_out, hipStream_t s) {
  const dim3 g((unsigned)(a.n_seq * hkv));
#define AKVS_SELECT(NW_, R_, ONE_)                                                              \
  hipLaunchKernelGGL((k_evict_select<NW_, R_, ONE_>), g, dim3(NW_ * 64), 0, s, weights, a, hkv, \
                     keep, w_out)
  if (a.n_keys <= 2048) AKVS_SELECT(8, 4, true);
  else if (a.n_keys <= 8192) AKVS_SELECT(16, 8, true);
  else if (a.n_keys <= 32768) AKVS_SELECT(16, 32, true);
  else AKVS_SELECT(16, 32, false);
#undef AKVS_SELECT
  return hipGetLastError();
}

hipError_t launch_evict_gather(const void *k, const void *v, const EvictArgs &a, int hkv,
                               int row_bytes, const int32_t *keep, void *k_out, void *v_out,
                               int32_t *lens_out, hipStream_t s) {
  if (!k && !lens_out) return hipSuccess;
  const int row16 = row_bytes / 16;
  const long long threads = k ? (long long)((a.n_keep + EV_U - 1) / EV_U) * hkv * row16 : 1;
  hipLaunchKernelGGL(k_evict_gather, dim3((unsigned)((threads + 255) / 256), a.n_seq), dim3(256), 0,
                     s, reinterpret_cast<const u32x4_t *>(k), reinterpret_cast<const u32x4_t *>(v), a,
                     hkv, row16, keep, reinterpret_cast<u32x4_t *>(k_out),
                     reinterpret_cast<u32x4_t *>(v_out), lens_out);
  return hipGetLastError();
}

}  // namespace akvs
