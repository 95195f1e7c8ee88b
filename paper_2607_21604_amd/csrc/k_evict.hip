// Eviction from caches by accumulated attention weight: selection of the kept keys, then the
// gather of their rows.
#include <algorithm>
#include <type_traits>

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

// One sequence's keys: [0, n), of which the candidates [c0, c1) are compared and `want` of them
// kept; the keys beside them are kept, as is every key where there are no more than may be.
struct EvictSeq {
  int n, kept, c0, c1, want;
  bool all;
  __device__ __forceinline__ EvictSeq(const EvictArgs &a, int seq) {
    n = a.lens ? min(max(a.lens[seq], 0), a.n_keys) : a.n_keys;
    kept = min(n, a.n_keep);
    all = n <= a.n_keep;
    want = all ? 0 : a.n_keep - a.n_first - a.n_recent;
    c0 = all ? n : a.n_first;
    c1 = all ? n : n - a.n_recent;
  }
  // key j, or 0 past b1, as a number
  __device__ __forceinline__ uint32_t order(float w, int j, int b1) const {
    return j >= b1 ? 0u : j >= c0 && j < c1 ? weight_key(w) : 0xffffffffu;
  }
};
constexpr int EV_BINS = 2048;
constexpr uint32_t EV_NONE = 0xfffffffeu;  // T where no candidate is kept
constexpr int digit_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
constexpr int digit_bits(int pass) { return pass == 2 ? 10 : 11; }

// Counts key u, if it is a candidate that agrees with T so far, under its next digit. (What is no
// candidate agrees with no T but the smallest.)
template <int PASS>
__device__ __forceinline__ void count_digit(int *hist, uint32_t u, uint32_t T) {
  constexpr int shift = digit_shift(PASS), bits = digit_bits(PASS);
  if (PASS == 0 ? u - 1 < 0xfffffffeu : (u ^ T) < (1u << (shift + bits)) && u != 0)
    atomicAdd(&hist[(u >> shift) & ((1u << bits) - 1)], 1);
}

// The bin in which the count from the top reaches `left`, and the count above it. Thread t has
// the PER_T bins below EV_BINS - t * PER_T, the highest first. Two barriers.
template <int NW, int PER_T>
__device__ __forceinline__ void top_bin(const int (&h)[PER_T], int left, int *s_wave, int *s_pick) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  int mine = 0;
#pragma unroll
  for (int i = 0; i < PER_T; ++i) mine += h[i];
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
}

// Lists the block's kept keys in order: those above T and, of those equal to it, the first
// eq_take - eqs. `at`: where the first goes; each(f): f(key index, number) over a wave's keys.
template <int NW, typename Each>
__device__ __forceinline__ void list_kept(Each &&each, uint32_t T, int eq_take, int at, int eqs,
                                          int *s_gt, int *s_eq, const float *w, int32_t *keep,
                                          float *w_out) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
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
}

// Block = one KV head of one sequence, NW waves; wave w has the keys [w * per, (w + 1) * per), R
// of a lane's at a time in registers (ONE: all of them, read once). The smallest kept candidate
// T is found a digit at a time (11, 11 and 10 bits): a histogram in LDS of the candidates that
// agree with T so far, its counts summed from the top by all threads, and the bin in which the
// count reaches what is wanted. Then each wave lists its kept keys in order; of the keys equal
// to T the first are kept. Short sequences are bound by a dozen barriers and the LDS round
// trips between them (5.2 us at 300 keys, 7.1 at 1500, 11.5 at 4516), long ones by the
// instructions per key on one compute unit; neither depends on how many heads there are up to
// one a unit.
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
  const float *w = weights + (size_t)blockIdx.x * a.n_keys;
  keep += (size_t)blockIdx.x * a.n_keep;
  if (w_out) w_out += (size_t)blockIdx.x * a.dst_rows;
  const EvictSeq q(a, blockIdx.x / hkv);
  const int steps = (q.n + T_ - 1) / T_, b0 = wave * steps * 64, b1 = min(b0 + steps * 64, q.n);
  uint32_t key[R];
  auto read = [&](int s0) __attribute__((always_inline)) {
    float x[R];
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (s0 + i < steps) x[i] = w[min(b0 + (s0 + i) * 64 + lane, q.n - 1)];
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (s0 + i < steps) key[i] = q.order(x[i], b0 + (s0 + i) * 64 + lane, b1);
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
  uint32_t T = EV_NONE;
  int left = 0;  // how many of the candidates that agree with T are kept
  auto digit = [&](auto pass) __attribute__((always_inline)) {
    constexpr int PASS = decltype(pass)::value;
#pragma unroll
    for (int i = 0; i < PER_T; ++i) hist[t + i * T_] = 0;
    __syncthreads();
    each([&](int, uint32_t u) { count_digit<PASS>(hist, u, T); });
    __syncthreads();
    int h[PER_T];
#pragma unroll
    for (int i = 0; i < PER_T; ++i) h[i] = hist[EV_BINS - 1 - (t * PER_T + i)];
    top_bin<NW>(h, left, s_wave, s_pick);
    T |= (uint32_t)s_pick[0] << digit_shift(PASS);
    left -= s_pick[1];
  };
  if (q.want > 0) {
    T = 0;
    left = q.want;
    digit(std::integral_constant<int, 0>());
    digit(std::integral_constant<int, 1>());
    digit(std::integral_constant<int, 2>());
  }
  list_kept<NW>(each, T, left, 0, 0, s_gt, s_eq, w, keep, w_out);
  for (int i = q.kept + t; i < a.n_keep; i += T_) keep[i] = -1;
  if (w_out)
    for (int i = q.kept + t; i < a.dst_rows; i += T_) w_out[i] = 0.f;
}

// The same over several blocks a head, each with `per` keys, in four launches: STAGE 0 .. 2 count
// their digit (16 bits a bin) for all blocks to sum in the next launch, STAGE 3 lists. What the
// blocks before this one hold above T follows from the same histograms, so that no block waits
// for another and no counter is cleared. A block leaves (T, left, keys before it above T) to its
// own next stage. Blocks (chunk, head).
constexpr int EVL_NW = 16, EVL_R = 4;  // waves, keys of a lane at a time
struct EvictLong {
  int chunks, per;
  uint32_t *hist[2];  // [heads][chunks][EV_BINS / 2] pairs of counts, by turns
  int4 *state;        // [heads][chunks]
};
template <int STAGE>
__global__ __launch_bounds__(EVL_NW * 64) void k_evict_long(const float *__restrict__ weights,
                                                            EvictArgs a, EvictLong p, int hkv,
                                                            int32_t *__restrict__ keep,
                                                            float *__restrict__ w_out) {
  constexpr int T_ = EVL_NW * 64, PAIRS = EV_BINS / 2;
  static_assert(PAIRS == T_, "a thread has a pair of bins");
  __shared__ int hist[EV_BINS];
  __shared__ __attribute__((aligned(16))) int s_wave[EVL_NW], s_gt[EVL_NW], s_eq[EVL_NW];
  __shared__ int s_pick[3];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int chunk = blockIdx.x % p.chunks, head = blockIdx.x / p.chunks;
  const float *w = weights + (size_t)head * a.n_keys;
  const EvictSeq q(a, head / hkv);
  const int start = min(chunk * p.per, q.n), end = min(start + p.per, q.n);
  const int steps = (end - start + T_ - 1) / T_;
  const int b0 = start + wave * steps * 64, b1 = min(b0 + steps * 64, end);
  uint32_t T = STAGE == 3 && q.want <= 0 ? EV_NONE : 0u;
  int left = max(q.want, 0), before = 0, eqs = 0;
  if (STAGE < 3 && q.want <= 0) return;
  if (STAGE > 0 && q.want > 0) {
    if (STAGE > 1) {
      const int4 st = p.state[(size_t)head * p.chunks + chunk];
      T = (uint32_t)st.x;
      left = st.y;
      before = st.z;
    }
    // bins 2047 - 2 t and the one below: all blocks' counts, and those of the blocks before
    const uint32_t *h = p.hist[(STAGE - 1) & 1] + (size_t)head * p.chunks * PAIRS + PAIRS - 1 - t;
    int sum[2] = {0, 0}, bef[2] = {0, 0};
    for (int c0 = 0; c0 < p.chunks; c0 += 8) {
      uint32_t x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = h[(size_t)min(c0 + i, p.chunks - 1) * PAIRS];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (c0 + i >= p.chunks) x[i] = 0;
        sum[0] += x[i] >> 16;
        sum[1] += x[i] & 0xffffu;
        if (c0 + i >= chunk) x[i] = 0;
        bef[0] += x[i] >> 16;
        bef[1] += x[i] & 0xffffu;
      }
    }
    top_bin<EVL_NW>(sum, left, s_wave, s_pick);
    const int bin = s_pick[0], top = EV_BINS - 1 - 2 * t;
    int over = (top > bin ? bef[0] : 0) + (top - 1 > bin ? bef[1] : 0);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) over += __shfl_xor(over, o, 64);
    if (lane == 0) s_gt[wave] = over;
    if (bin == top) s_pick[2] = bef[0];
    if (bin == top - 1) s_pick[2] = bef[1];
    __syncthreads();
#pragma unroll
    for (int v = 0; v < EVL_NW; ++v) before += s_gt[v];
    eqs = s_pick[2];  // (of the last digit: keys equal to T)
    T |= (uint32_t)bin << digit_shift(STAGE - 1);
    left -= s_pick[1];
    if (STAGE < 3 && t == 0)
      p.state[(size_t)head * p.chunks + chunk] = make_int4((int)T, left, before, 0);
    __syncthreads();  // (s_gt is used again)
  }
  auto each = [&](auto &&f) __attribute__((always_inline)) {
    for (int s0 = 0; s0 < steps; s0 += EVL_R) {
      float x[EVL_R];
#pragma unroll
      for (int i = 0; i < EVL_R; ++i)
        if (s0 + i < steps) x[i] = w[min(b0 + (s0 + i) * 64 + lane, q.n - 1)];
#pragma unroll
      for (int i = 0; i < EVL_R; ++i)
        if (s0 + i < steps) {
          const int j = b0 + (s0 + i) * 64 + lane;
          f(j, q.order(x[i], j, b1));
        }
    }
  };
  if constexpr (STAGE < 3) {
    hist[t] = hist[t + T_] = 0;
    __syncthreads();
    each([&](int, uint32_t u) { count_digit<STAGE>(hist, u, T); });
    __syncthreads();
    p.hist[STAGE & 1][(size_t)(head * p.chunks + chunk) * PAIRS + t] =
        (uint32_t)hist[2 * t] | (uint32_t)hist[2 * t + 1] << 16;
  } else {
    keep += (size_t)head * a.n_keep;
    if (w_out) w_out += (size_t)head * a.dst_rows;
    // keys before this block that are kept without comparison, above T, and equal to it
    const int at = min(start, q.c0) + max(start - q.c1, 0) + before + min(eqs, left);
    list_kept<EVL_NW>(each, T, left, at, eqs, s_gt, s_eq, w, keep, w_out);
    for (int i = q.kept + chunk * T_ + t; i < a.n_keep; i += p.chunks * T_) keep[i] = -1;
    if (w_out)
      for (int i = q.kept + chunk * T_ + t; i < a.dst_rows; i += p.chunks * T_) w_out[i] = 0.f;
  }
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

// Sequences too long for a block's registers are split, up to a block a compute unit and 16 a
// head (each sums the counts of all of its head), where that leaves four a head at least: 8 / 32 /
// 64 heads of 34000 keys 24 / 27 / 31 us, of 120500 keys 29 / 43 / 80, in one block each 51 to 52
// and 126 to 130; 128 heads in two blocks each 49 and 131, in one 52 and 133. Shorter ones are as
// fast whole: 8 heads of 16384 / 26335 keys 17 / 21 us, split 21 / 21. A block has 4096 keys at
// least, what its lanes read at once, and fewer than 2^16, a bin's count.
static bool evict_splits(const EvictArgs &a, int hkv) {
  return a.n_keys > 32768 && (long long)a.n_seq * hkv * 4 <= gemm_cu_count();
}
static EvictLong evict_long(const EvictArgs &a, int hkv) {
  constexpr int UNIT = EVL_NW * 64 * EVL_R;
  EvictLong p{};
  const long long most = std::min(16, gemm_cu_count() / (a.n_seq * hkv)) * UNIT;
  p.per = (int)std::min((a.n_keys + most - 1) / most, 15LL) * UNIT;
  p.chunks = (a.n_keys + p.per - 1) / p.per;
  return p;
}
size_t evict_scratch_bytes(const EvictArgs &a, int hkv) {
  if (!evict_splits(a, hkv)) return 0;
  return (size_t)a.n_seq * hkv * evict_long(a, hkv).chunks * (2 * EV_BINS * 2 + sizeof(int4));
}

// Few keys: eight waves (300 / 1500 keys 5.2 / 7.1 us; four 5.7 / 8.5, sixteen 6.4 / 7.9).
hipError_t launch_evict_select(const float *weights, const EvictArgs &a, int hkv, int32_t *keep,
                               float *w_out, void *scratch, hipStream_t s) {
  const dim3 g((unsigned)(a.n_seq * hkv));
  if (scratch) {
    EvictLong p = evict_long(a, hkv);
    const size_t items = (size_t)g.x * p.chunks;
    p.state = reinterpret_cast<int4 *>(scratch);
    p.hist[0] = reinterpret_cast<uint32_t *>(p.state + items);
    p.hist[1] = p.hist[0] + items * (EV_BINS / 2);
#define AKVS_STAGE(STAGE_)                                                                        \
  hipLaunchKernelGGL((k_evict_long<STAGE_>), dim3((unsigned)items), dim3(EVL_NW * 64), 0, s,      \
                     weights, a, p, hkv, keep, w_out)
    AKVS_STAGE(0);
    AKVS_STAGE(1);
    AKVS_STAGE(2);
    AKVS_STAGE(3);
#undef AKVS_STAGE
    return hipGetLastError();
  }
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
