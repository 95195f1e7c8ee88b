// Attention over sequences in pages of 4-bit codes.
#include <algorithm>
#include <cmath>

#include "kernels.h"
#include "pages_dev.h"

namespace akvs {

// The request that row r is of, or -1.
__device__ __forceinline__ int paged_request(const PagedBatch &s, int r) {
  if (!s.row_start) return r / s.rows_max;
  int lo = 0, hi = s.n_req;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (s.row_start[mid + 1] > r) hi = mid;
    else lo = mid + 1;
  }
  return lo < s.n_req ? lo : -1;
}

// A block per (row, query head): a thread per key forms its score, then threads take a dim each of
// a share of the keys. Simple; keys are read once per query head.
template <int HD>
__global__ __launch_bounds__(256) void k_paged_simple(PagedBatch s, PagePool p,
                                                      const bf16_t *__restrict__ Q, int hq, int hkv,
                                                      float scale_log2, bf16_t *out,
                                                      float *__restrict__ lse) {
  constexpr int SHARES = 256 / HD;
  __shared__ float s_q[HD], s_p[256], s_red[4], s_o[SHARES][HD];
  const int tid = threadIdx.x, head = blockIdx.x % hq, r = blockIdx.x / hq;
  const int h = head / (hq / hkv), mask = (1 << p.shift) - 1;
  const int b = paged_request(s, r);
  if (b < 0) return;
  int r0, r1, len;
  paged_rows(s, b, r0, r1);
  if (r < r0 || r >= r1) return;
  const int32_t *table = paged_keys(s, b, len);
  const int seen = max(len - r1 + r + 1, 0);
  if (tid < HD) s_q[tid] = load1(Q + ((size_t)r * hq + head) * HD + tid);
  const int d = tid % HD, share = tid / HD;
  float m = -INFINITY, l = 0.f, o = 0.f;
  __syncthreads();
  auto row_of = [&](int j, bool &there) {
    const int page = table[j >> p.shift];
    there = page >= 0 && page < p.n_pages;
    return (((size_t)(there ? page : 0) * hkv + h) << p.shift) + (j & mask);
  };
  for (int base = 0; base < seen; base += 256) {
    const int n = min(256, seen - base);
    float sc = -INFINITY;
    if (tid < n) {
      bool there;
      const size_t row = row_of(base + tid, there);
      sc = 0.f;
      for (int e = 0; e < HD && there; e += 8) {
        float x[8];
        cache_load8(p.k, reinterpret_cast<const _Float16 *>(p.k_meta), AKVS_U4G64, row, HD, e, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) sc = fmaf(x[i], s_q[e + i], sc);
      }
      sc *= scale_log2;
    }
    float mx = wave_max(sc);
    if ((tid & 63) == 0) s_red[tid >> 6] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
    const float m_new = fmaxf(m, mx), off = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = exp2f(m - off);
    s_p[tid] = tid < n ? exp2f(sc - off) : 0.f;
    m = m_new;
    __syncthreads();
    l *= alpha;
    o *= alpha;
    for (int j = 0; j < n; ++j) l += s_p[j];
    for (int j = share; j < n; j += SHARES) {
      bool there;
      const size_t row = row_of(base + j, there);
      if (there)
        o = fmaf(s_p[j], cache_load1(p.v, reinterpret_cast<const _Float16 *>(p.v_meta), AKVS_U4G64,
                                     row, HD, d), o);
    }
    __syncthreads();
  }
  s_o[share][d] = o;
  __syncthreads();
  const size_t item = (size_t)r * hq + head;
  if (tid < HD) {
    float x = s_o[0][tid];
#pragma unroll
    for (int q = 1; q < SHARES; ++q) x += s_o[q][tid];
    store1(out + item * HD + tid, l == 0.f ? 0.f : x / l);
  }
  if (lse && tid == 0)
    lse[item] =
        l == 0.f ? -INFINITY : (m == -INFINITY ? 0.f : m * 0.6931471805599453f) + logf(l);
}

size_t paged_part_floats(const PagedBatch &s, int hq, int hkv, int hd) { return 0; }

hipError_t launch_paged_attention(const PagedBatch &s, const PagePool &p, const void *q, int hq,
                                  int hkv, int hd, void *out, float *lse, float *part,
                                  hipStream_t st) {
  if (s.n_rows == 0) return hipSuccess;
  const dim3 g((unsigned)s.n_rows * hq), b(256);
  const float scale = 1.4426950408889634f / sqrtf((float)hd);
  const bf16_t *Q = reinterpret_cast<const bf16_t *>(q);
  bf16_t *O = reinterpret_cast<bf16_t *>(out);
  if (hd == 128)
    hipLaunchKernelGGL(k_paged_simple<128>, g, b, 0, st, s, p, Q, hq, hkv, scale, O, lse);
  else
    hipLaunchKernelGGL(k_paged_simple<64>, g, b, 0, st, s, p, Q, hq, hkv, scale, O, lse);
  return hipGetLastError();
}

}  // namespace akvs
