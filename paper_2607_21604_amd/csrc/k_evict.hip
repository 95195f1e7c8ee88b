// Eviction from caches by accumulated attention weight: selection of the kept keys, then the
// gather of their rows.
#include "kernels.h"

namespace akvs {

// Order of the weights as unsigned numbers: a NaN smallest, then -inf .. +inf, -0 as +0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w);
  if (w != w) return 0u;
  if (u == 0x80000000u) return 0x80000000u;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Block = one KV head of one sequence. The kept weights' smallest key T is found eight bits at
// a time from a histogram of the candidates that agree with T so far; then wave w lists the
// kept keys of its 1/16 of the sequence in order. Of the keys equal to T the first are kept.
constexpr int EV_T = 1024, EV_W = EV_T / 64;
__global__ __launch_bounds__(EV_T) void k_evict_select(const float *__restrict__ weights,
                                                       EvictArgs a, int hkv,
                                                       int32_t *__restrict__ keep,
                                                       float *__restrict__ w_out) {
  __shared__ int hist[256];
  __shared__ int s_pick[2];
  __shared__ int s_gt[EV_W], s_eq[EV_W];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int seq = blockIdx.x / hkv;
  const float *w = weights + (size_t)blockIdx.x * a.n_keys;
  keep += (size_t)blockIdx.x * a.n_keep;
  if (w_out) w_out += (size_t)blockIdx.x * a.dst_rows;
  const int n = a.lens ? min(max(a.lens[seq], 0), a.n_keys) : a.n_keys;
  const int kept = min(n, a.n_keep);
  const bool all = n <= a.n_keep;
  // candidates [c0, c1): every key where all are kept, none of them then
  const int c0 = a.n_first, c1 = n - a.n_recent, want = a.n_keep - a.n_first - a.n_recent;
  uint32_t T = 0;
  int eq_take = 0;
  if (!all && want > 0) {
    int left = want;  // how many of the candidates that agree with T are kept
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (t < 256) hist[t] = 0;
      __syncthreads();
      for (int j = c0 + t; j < c1; j += EV_T) {
        const uint32_t u = weight_key(w[j]);
        if (shift == 24 || (u >> (shift + 8)) == (T >> (shift + 8)))
          atomicAdd(&hist[(u >> shift) & 255], 1);
      }
      __syncthreads();
      if (t == 0) {
        int above = 0, d = 255;
        while (d > 0 && above + hist[d] < left) above += hist[d--];
        s_pick[0] = d;
        s_pick[1] = above;
      }
      __syncthreads();
      T |= (uint32_t)s_pick[0] << shift;
      left -= s_pick[1];
      __syncthreads();
    }
    eq_take = left;
  }
  // [b0, b1): this wave's keys, in order
  const int per = ((n + EV_W - 1) / EV_W + 63) / 64 * 64;
  const int b0 = min(wave * per, n), b1 = min(b0 + per, n);
  auto sort_of = [&](int j) {  // 2: kept, 1: equal to T, 0: evicted
    if (j >= b1) return 0;
    if (all || j < c0 || j >= c1) return 2;
    if (want <= 0) return 0;
    const uint32_t u = weight_key(w[j]);
    return u > T ? 2 : u == T ? 1 : 0;
  };
  int gt = 0, eq = 0;
  for (int j0 = b0; j0 < b1; j0 += 64) {
    const int k = sort_of(j0 + lane);
    gt += __popcll(__ballot(k == 2));
    eq += __popcll(__ballot(k == 1));
  }
  if (lane == 0) {
    s_gt[wave] = gt;
    s_eq[wave] = eq;
  }
  __syncthreads();
  int at = 0, eqs = 0;  // kept keys and keys equal to T before this wave's
  for (int v = 0; v < wave; ++v) {
    at += s_gt[v] + min(s_eq[v], max(eq_take - eqs, 0));
    eqs += s_eq[v];
  }
  const unsigned long long below = (1ull << lane) - 1;
  for (int j0 = b0; j0 < b1; j0 += 64) {
    const int k = sort_of(j0 + lane);
    const unsigned long long e = __ballot(k == 1);
    const bool take = k == 2 || (k == 1 && eqs + __popcll(e & below) < eq_take);
    const unsigned long long m = __ballot(take);
    if (take) {
      const int i = at + __popcll(m & below);
      keep[i] = j0 + lane;
      if (w_out) w_out[i] = w[j0 + lane];
    }
    at += __popcll(m);
    eqs += __popcll(e);
  }
  for (int i = kept + t; i < a.n_keep; i += EV_T) keep[i] = -1;
  if (w_out)
    for (int i = kept + t; i < a.dst_rows; i += EV_T) w_out[i] = 0.f;
}

// A thread moves 16 bytes of a kept key's row and of its value's.
__global__ __launch_bounds__(256) void k_evict_gather(const char *__restrict__ k,
                                                      const char *__restrict__ v, EvictArgs a,
                                                      int hkv, int row16,
                                                      const int32_t *__restrict__ keep,
                                                      char *__restrict__ k_out,
                                                      char *__restrict__ v_out, int32_t *lens_out) {
  const long long gid = (long long)blockIdx.x * 256 + threadIdx.x;
  if (lens_out && gid < a.n_seq) {
    const int n = a.lens ? min(max(a.lens[gid], 0), a.n_keys) : a.n_keys;
    lens_out[gid] = min(n, a.n_keep);
  }
  if (!k) return;
  const long long row = gid / row16;  // (sequence, kept row, head)
  const int c = (int)(gid - row * row16);
  const long long si = row / hkv;
  const int h = (int)(row - si * hkv), seq = (int)(si / a.n_keep), i = (int)(si % a.n_keep);
  if (seq >= a.n_seq) return;
  const int j = keep[((size_t)seq * hkv + h) * a.n_keep + i];
  if (j < 0 || j >= a.n_keys) return;
  const size_t src = (((size_t)seq * a.src_rows + j) * hkv + h) * row16 + c;
  const size_t dst = (((size_t)seq * a.dst_rows + i) * hkv + h) * row16 + c;
  reinterpret_cast<uint4 *>(k_out)[dst] = reinterpret_cast<const uint4 *>(k)[src];
  reinterpret_cast<uint4 *>(v_out)[dst] = reinterpret_cast<const uint4 *>(v)[src];
}

hipError_t launch_evict_select(const float *weights, const EvictArgs &a, int hkv, int32_t *keep,
                               float *w_out, hipStream_t s) {
  hipLaunchKernelGGL(k_evict_select, dim3((unsigned)(a.n_seq * hkv)), dim3(EV_T), 0, s, weights, a,
                     hkv, keep, w_out);
  return hipGetLastError();
}

hipError_t launch_evict_gather(const void *k, const void *v, const EvictArgs &a, int hkv,
                               int row_bytes, const int32_t *keep, void *k_out, void *v_out,
                               int32_t *lens_out, hipStream_t s) {
  if (!k && !lens_out) return hipSuccess;
  const int row16 = row_bytes / 16;
  long long threads = k ? (long long)a.n_seq * a.n_keep * hkv * row16 : a.n_seq;
  if (lens_out && threads < a.n_seq) threads = a.n_seq;
  hipLaunchKernelGGL(k_evict_gather, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s,
                     reinterpret_cast<const char *>(k), reinterpret_cast<const char *>(v), a, hkv,
                     row16, keep, reinterpret_cast<char *>(k_out), reinterpret_cast<char *>(v_out),
                     lens_out);
  return hipGetLastError();
}

}  // namespace akvs
