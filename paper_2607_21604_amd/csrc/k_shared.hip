// Attention of a batch over one shared context, and the weights that its keys received.
#include "kernels.h"

namespace akvs {

// Rows of request b: [r0, r1). Values of row_start are clamped into the buffers.
__device__ __forceinline__ void shared_rows(const SharedBatch &s, int b, int &r0, int &r1) {
  if (s.row_start) {
    r0 = min(max(s.row_start[b], 0), s.n_rows);
    r1 = min(max(s.row_start[b + 1], r0), s.n_rows);
  } else {
    r0 = b * s.rows_max;
    r1 = r0 + s.rows_max;
  }
}
__device__ __forceinline__ int shared_live(const SharedBatch &s) {
  return s.row_start ? min(max(s.row_start[s.n_req], 0), s.n_rows) : s.n_rows;
}

// A wave per (row, query head): a lane per key for the scores, a lane per dim (or two) for the
// values.
template <typename TS>
__global__ __launch_bounds__(64) void k_shared_attn(SharedBatch s, const TS *__restrict__ Q,
                                                    const TS *__restrict__ Kp,
                                                    const TS *__restrict__ Vp,
                                                    const TS *__restrict__ Ko,
                                                    const TS *__restrict__ Vo, int hq, int hkv,
                                                    int hd, float scale_log2,
                                                    TS *__restrict__ out, float *lse) {
  const int lane = threadIdx.x, r = blockIdx.x / hq, h = blockIdx.x % hq, kvh = h / (hq / hkv);
  if (r >= shared_live(s)) return;
  int b = 0;
  if (s.row_start) {
    int lo = 0, hi = s.n_req - 1;  // the last request that starts at or before r
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s.row_start[mid] <= r) lo = mid;
      else hi = mid - 1;
    }
    b = lo;
  } else {
    b = r / s.rows_max;
  }
  int r0, r1;
  shared_rows(s, b, r0, r1);
  const int own = s.own_rows ? min(max(s.own_len[b], 0), s.own_rows) : 0;
  const int seen = min(max(own - (r1 - r0) + (r - r0) + 1, 0), own);
  const TS *q = Q + ((size_t)r * hq + h) * hd;
  float m = -INFINITY, l = 0.f, o[2] = {0.f, 0.f};
  for (int part = 0; part < 2; ++part) {
    const int n = part ? seen : s.prefix_len;
    const size_t base = part ? (size_t)b * s.own_rows : 0;
    const TS *K = part ? Ko : Kp, *V = part ? Vo : Vp;
    for (int k0 = 0; k0 < n; k0 += 64) {
      const int k = min(k0 + lane, n - 1);
      float sc = 0.f;
      for (int d = 0; d < hd; d += 8) {
        float a[8], c[8];
        load8(q + d, a);
        load8(K + ((base + k) * hkv + kvh) * hd + d, c);
#pragma unroll
        for (int i = 0; i < 8; ++i) sc = fmaf(a[i], c[i], sc);
      }
      sc = k0 + lane < n ? sc * scale_log2 : -INFINITY;
      const float m_new = fmaxf(m, wave_max(sc)), off = m_new == -INFINITY ? 0.f : m_new;
      const float p = exp2f(sc - off), alpha = exp2f(m - off);
      m = m_new;
      l = l * alpha + wave_sum(p);
      o[0] *= alpha;
      o[1] *= alpha;
      for (int e = 0; e < 64 && k0 + e < n; ++e) {
        const float pe = __shfl(p, e, 64);
        const TS *v = V + ((base + k0 + e) * hkv + kvh) * hd;
        o[0] = fmaf(pe, load1(v + lane), o[0]);
        if (hd > 64) o[1] = fmaf(pe, load1(v + 64 + lane), o[1]);
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  TS *dst = out + ((size_t)r * hq + h) * hd;
  store1(dst + lane, o[0] * inv);
  if (hd > 64) store1(dst + 64 + lane, o[1] * inv);
  if (lse && lane == 0)
    lse[(size_t)r * hq + h] = l == 0.f ? -INFINITY : (m == -INFINITY ? 0.f : m) * 0.6931471805599453f + logf(l);
}

// A thread per key of one KV head; blocks past the prefix's serve a request's own keys.
template <typename TS>
__global__ __launch_bounds__(256) void k_attn_weights(SharedBatch s, const TS *__restrict__ Q,
                                                      const float *__restrict__ lse,
                                                      const TS *__restrict__ Kp,
                                                      const TS *__restrict__ Ko, int hq, int hkv,
                                                      int hd, float scale, int prefix_blocks,
                                                      int own_blocks, const float *wp_prev,
                                                      float *wp, const float *wo_prev,
                                                      float *wo) {
  const int kvh = blockIdx.y, G = hq / hkv;
  int blk = blockIdx.x, r0 = 0, r1, n, n_all, own = 0;
  const TS *K;
  const float *prev;
  float *w;
  const bool prefix = blk < prefix_blocks;
  if (prefix) {
    r1 = shared_live(s);
    n = n_all = s.prefix_len;
    K = Kp;
    prev = wp_prev ? wp_prev + (size_t)kvh * n : nullptr;
    w = wp + (size_t)kvh * n;
  } else {
    blk -= prefix_blocks;
    const int b = blk / own_blocks;
    blk -= b * own_blocks;
    shared_rows(s, b, r0, r1);
    n = own = min(max(s.own_len[b], 0), s.own_rows);
    n_all = s.own_rows;
    K = Ko + (size_t)b * s.own_rows * hkv * hd;
    const size_t o = ((size_t)b * hkv + kvh) * n_all;
    prev = wo_prev ? wo_prev + o : nullptr;
    w = wo + o;
  }
  const int j = blk * 256 + threadIdx.x;
  if (j >= n_all) return;
  float sum = 0.f;
  if (j < n) {
    const TS *k = K + ((size_t)j * hkv + kvh) * hd;
    for (int r = r0; r < r1; ++r) {
      if (!prefix && j > own - (r1 - r0) + (r - r0)) continue;
      for (int g = 0; g < G; ++g) {
        const int h = kvh * G + g;
        const float ls = lse[(size_t)r * hq + h];
        if (ls == -INFINITY) continue;
        const TS *q = Q + ((size_t)r * hq + h) * hd;
        float sc = 0.f;
        for (int d = 0; d < hd; d += 8) {
          float a[8], c[8];
          load8(q + d, a);
          load8(k + d, c);
#pragma unroll
          for (int i = 0; i < 8; ++i) sc = fmaf(a[i], c[i], sc);
        }
        sum += expf(sc * scale - ls);
      }
    }
  }
  w[j] = (prev ? prev[j] : 0.f) + sum;
}

template <typename TS>
static hipError_t shared_attention(const SharedBatch &s, const void *q, const void *kp,
                                   const void *vp, const void *ko, const void *vo, int hq,
                                   int hkv, int hd, void *out, float *lse, hipStream_t st) {
  auto p = [](const void *x) { return reinterpret_cast<const TS *>(x); };
  hipLaunchKernelGGL(k_shared_attn<TS>, dim3((unsigned)((size_t)s.n_rows * hq)), dim3(64), 0, st, s,
                     p(q), p(kp), p(vp), p(ko), p(vo), hq, hkv, hd,
                     1.4426950408889634f / sqrtf((float)hd), reinterpret_cast<TS *>(out), lse);
  return hipGetLastError();
}

hipError_t launch_shared_attention(const SharedBatch &s, const void *q, const void *kp,
                                   const void *vp, const void *ko, const void *vo, int hq,
                                   int hkv, int hd, int dtype, void *out, float *lse,
                                   hipStream_t st) {
  if (s.n_rows == 0) return hipSuccess;
  return dtype == AKVS_BF16
             ? shared_attention<bf16_t>(s, q, kp, vp, ko, vo, hq, hkv, hd, out, lse, st)
             : shared_attention<float>(s, q, kp, vp, ko, vo, hq, hkv, hd, out, lse, st);
}

template <typename TS>
static hipError_t attention_weights(const SharedBatch &s, const void *q, const float *lse,
                                    const void *kp, const void *ko, int hq, int hkv, int hd,
                                    const float *wp_prev, float *wp, const float *wo_prev,
                                    float *wo, hipStream_t st) {
  const int pb = wp ? (s.prefix_len + 255) / 256 : 0, ob = wo ? (s.own_rows + 255) / 256 : 0;
  const size_t blocks = pb + (size_t)s.n_req * ob;
  if (blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(k_attn_weights<TS>, dim3((unsigned)blocks, hkv), dim3(256), 0, st, s,
                     reinterpret_cast<const TS *>(q), lse, reinterpret_cast<const TS *>(kp),
                     reinterpret_cast<const TS *>(ko), hq, hkv, hd, 1.0f / sqrtf((float)hd), pb,
                     ob, wp_prev, wp, wo_prev, wo);
  return hipGetLastError();
}

hipError_t launch_attention_weights(const SharedBatch &s, const void *q, const float *lse,
                                    const void *kp, const void *ko, int hq, int hkv, int hd,
                                    int dtype, const float *wp_prev, float *wp,
                                    const float *wo_prev, float *wo, hipStream_t st) {
  return dtype == AKVS_BF16 ? attention_weights<bf16_t>(s, q, lse, kp, ko, hq, hkv, hd, wp_prev, wp,
                                                        wo_prev, wo, st)
                            : attention_weights<float>(s, q, lse, kp, ko, hq, hkv, hd, wp_prev, wp,
                                                       wo_prev, wo, st);
}

}  // namespace akvs
