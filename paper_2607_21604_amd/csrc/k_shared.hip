// Attention of a batch over one shared context, and the weights that its keys received.
//
// Both treat the (row, query head) pairs that read one KV head as rows of one matrix: 16
// decoding requests of 5 heads per KV head are 80 rows against the shared keys, which are then
// read once, through LDS, for all of them. The prefix is cut into splits and a request's own
// keys into chunks; each is a work item of its own, all items run in one launch and leave
// (output, maximum, sum) partials that a second launch merges.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kernels.h"

namespace akvs {

// Rows of request b: [r0, r1), at most rows_max. Values of row_start are clamped into the
// buffers.
__device__ __forceinline__ void shared_rows(const SharedBatch &s, int b, int &r0, int &r1) {
  if (s.row_start) {
    r0 = min(max(s.row_start[b], 0), s.n_rows);
    r1 = min(max(s.row_start[b + 1], r0), min(s.n_rows, r0 + s.rows_max));
  } else {
    r0 = b * s.rows_max;
    r1 = r0 + s.rows_max;
  }
}
__device__ __forceinline__ int shared_live(const SharedBatch &s) {
  return s.row_start ? min(max(s.row_start[s.n_req], 0), s.n_rows) : s.n_rows;
}

// Work items of one call. Blocks [0, prefix_blocks): (split, pair tile, KV head), KV heads
// innermost, so that the blocks streaming one head's keys share an XCD's L2; then (request,
// chunk, pair tile, KV head) of the own keys.
struct SharedPlan {
  int p_pairs, p_tiles, splits, split_keys, prefix_blocks;  // pairs of a tile, tiles, ..
  int o_pairs, o_tiles, chunks, chunk_keys;
  int slots;  // partials per (row, head): splits + chunks
  bool whole;  // no prefix items: a request's items take the prefix's keys, then its own
};
constexpr int SH_TILE = 64;  // keys of an LDS tile

// The item that a block serves: `pairs` pairs from v0 of rows [r0, r1), keys [k0, k1). own = -1:
// the prefix's keys, which every row sees; else the request's own, rows from `base` of their
// tensors. A whole item numbers its keys so that tiles hold one kind: [0, first) are the
// prefix's, own key j is shift + j, shift the next multiple of a tile (else both are 0).
struct SharedItem {
  int kvh, r0, r1, v0, pairs, k0, k1, slot, own, first, shift;
  size_t base;
};
template <bool WHOLE>
__device__ __forceinline__ bool shared_item(const SharedBatch &s, const SharedPlan &p, int hkv,
                                            int G, SharedItem &it) {
  int id = blockIdx.x;
  const bool prefix = !WHOLE && id < p.prefix_blocks;
  if (!WHOLE && !prefix) id -= p.prefix_blocks;
  it.kvh = id % hkv;
  id /= hkv;
  it.first = it.shift = 0;
  if (prefix) {
    const int tile = id % p.p_tiles, split = id / p.p_tiles;
    it.pairs = p.p_pairs;
    it.v0 = tile * it.pairs;
    it.r0 = 0;
    it.r1 = shared_live(s);
    it.k0 = split * p.split_keys;
    it.k1 = min(s.prefix_len, it.k0 + p.split_keys);
    it.slot = split;
    it.own = -1;
    it.base = 0;
  } else {
    const int tile = id % p.o_tiles;
    id /= p.o_tiles;
    const int chunk = id % p.chunks, b = id / p.chunks;
    it.pairs = p.o_pairs;
    it.v0 = tile * it.pairs;
    shared_rows(s, b, it.r0, it.r1);
    it.own = min(max(s.own_len[b], 0), s.own_rows);
    it.k0 = chunk * p.chunk_keys;
    it.k1 = min(it.own, it.k0 + p.chunk_keys);
    it.slot = p.splits + chunk;
    it.base = (size_t)b * s.own_rows;
    if (WHOLE) {
      it.first = s.prefix_len;
      it.shift = (s.prefix_len + SH_TILE - 1) / SH_TILE * SH_TILE;
      it.k1 = it.own > 0 ? it.shift + it.own : it.first;
    }
  }
  return it.v0 < (it.r1 - it.r0) * G;
}
// The end of the keys that row r (of the item's rows) sees.
__device__ __forceinline__ int shared_seen(const SharedItem &it, int r) {
  const int own = it.own - (it.r1 - r) + 1;
  return it.own < 0 ? it.k1 : own > 0 ? min(it.shift + own, it.k1) : it.first;
}

__device__ __forceinline__ bool odd_bf16(uint32_t lo16) { return (lo16 & 0x7f80u) == 0x7f80u; }

// bf16. Block = 4 waves over a tile of 32 * groups pairs (groups 1, 2 or 4) and one key range.
// Keys stream through LDS in tiles of 64, loaded into registers a tile ahead; a wave takes 32
// pairs and 32 or 64 of the tile's keys: with 4 groups each wave has a group, with 2 two waves
// share a group's keys, with 1 two of the waves only load. Scores are formed transposed,
// S^T = K Q^T (MFMA 32x32x16): lane l holds 16 scores of pair l % 32, which is the operand
// layout of O^T = V^T P^T; V^T comes from row-major rows by the transposing LDS read. Softmax
// statistics and outputs are fp32; the probabilities are rounded to bf16 for the second
// product (the matrix cores' type), their sum is not.
// Few rows over a long prefix are bound by its bytes (5 rows over 130001 keys of 28/4 heads 61 us
// with the merge, 4.5 TB/s), over shorter ones by a block's latency, 7.5 us and 1.75 per tile.
// Many rows are bound by the softmax between the products, which two waves a SIMD hide in part
// (1328 rows over 16128 keys of 40/8 heads 498 us, 888 TFLOP/s).
template <int HD, bool WHOLE>
__global__ __launch_bounds__(256, 2) void k_shared_bf16(
    SharedBatch s, SharedPlan p, const bf16_t *__restrict__ Q, const bf16_t *__restrict__ Kp,
    const bf16_t *__restrict__ Vp, const bf16_t *__restrict__ Ko, const bf16_t *__restrict__ Vo,
    int hq, int hkv, float scale_log2, bf16_t *__restrict__ out, float *__restrict__ lse,
    _Float16 *__restrict__ part_o, float4 *__restrict__ part_ml) {
  constexpr int KS = HD / 16, DB = HD / 32, CPK = HD / 8;
  constexpr int KST = HD + 8, VST = HD + 32;       // row strides: fragment reads on all banks
  constexpr int NCH = SH_TILE * CPK / 256;         // 16-byte chunks of K (and V) per thread
  constexpr int KB = SH_TILE * KST, VB = SH_TILE * VST;
  __shared__ __attribute__((aligned(16))) bf16_t s_kv[2 * (KB + VB)];
  __shared__ int s_odd;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, hi = lane >> 5;
  const int G = hq / hkv;
  SharedItem it;
  if (!shared_item<WHOLE>(s, p, hkv, G, it)) return;
  const bf16_t *K = it.own < 0 ? Kp : Ko, *V = it.own < 0 ? Vp : Vo;
  // this wave's pairs and its share of a tile's two 32-key halves
  const int groups = it.pairs >> 5;
  const int group = groups == 4 ? wave : groups == 2 ? wave >> 1 : 0;
  const bool works = groups > 1 || wave < 2;
  const int st0 = groups == 4 ? 0 : wave & 1, st_step = groups == 4 ? 1 : 2;
  const int n_pairs = (it.r1 - it.r0) * G;
  const int v = it.v0 + group * 32 + (lane & 31);
  const bool valid = v < n_pairs;
  const int r = it.r0 + (valid ? v : it.v0) / G, head = it.kvh * G + (valid ? v : it.v0) % G;
  const int seen = valid ? shared_seen(it, r) : 0;
  // what the tile's last and first rows see: keys past the one are not read, keys up to the
  // other need no mask
  const int last = min(n_pairs, it.v0 + it.pairs) - 1;
  const int k1 = shared_seen(it, it.r0 + last / G), all_see = shared_seen(it, it.r0 + it.v0 / G);
  const size_t prow = ((size_t)it.slot * s.n_rows + r) * hq + head;
  const int nkt = k1 > it.k0 ? (k1 - it.k0 + SH_TILE - 1) / SH_TILE : 0;
  const bool writes = valid && (groups == 4 || (works && (wave & 1) == 0));
  if (nkt == 0 && p.slots > 1) {
    if (writes && hi == 0) part_ml[prow] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    return;
  }

  bf16x8_t qf[KS];
  {
    const bf16_t *q = Q + ((size_t)r * hq + head) * HD + hi * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8_t *>(q + ks * 16);
  }
  f32x16_t o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;  // (l_run: of this lane's half of the keys)

  // Chunk i of a thread is 16 bytes of key row tid / CPK + i * (256 / CPK) of a tile: a fixed
  // offset from the tile's first key, whose address is the same for all threads.
  u32x4_t kreg[NCH], vreg[NCH];
  const uint32_t row_bytes = hkv * HD * 2;
  const uint32_t off0 = tid / CPK * row_bytes + tid % CPK * 16;
  auto load = [&](int key0) __attribute__((always_inline)) {
    const bool pre = WHOLE && key0 < it.shift;
    const size_t at = pre ? key0 : it.base + key0 - it.shift;
    const size_t start = at * row_bytes + it.kvh * (HD * 2);
    const char *kt = reinterpret_cast<const char *>(pre ? Kp : K) + start;
    const char *vt = reinterpret_cast<const char *>(pre ? Vp : V) + start;
    const int end = (pre ? it.first : k1) - 1 - key0;  // the last key, which keys past it re-read
    if (end >= SH_TILE - 1) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const uint32_t off = off0 + i * (256 / CPK) * row_bytes;
        kreg[i] = *reinterpret_cast<const u32x4_t *>(kt + off);
        vreg[i] = *reinterpret_cast<const u32x4_t *>(vt + off);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const uint32_t off =
            min(tid / CPK + i * (256 / CPK), end) * row_bytes + tid % CPK * 16;
        kreg[i] = *reinterpret_cast<const u32x4_t *>(kt + off);
        vreg[i] = *reinterpret_cast<const u32x4_t *>(vt + off);
      }
    }
  };
  // Values that some pair of the tile must not see take part with probability 0, and 0 * inf is
  // NaN: where such a value is not finite, 0 goes to LDS, and the pairs that do see it get it
  // added at the end.
  auto store = [&](int key0, int buf) __attribute__((always_inline)) {
    bf16_t *ks = s_kv + buf * (KB + VB), *vs = ks + KB;
    const int all = WHOLE && key0 < it.shift ? it.first : all_see;
    const bool some_hidden = key0 + SH_TILE > all;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = tid + 256 * i, kr = c / CPK, e0 = (c % CPK) * 8;
      if (some_hidden && key0 + kr >= all) {
        bool odd = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t w = vreg[i][j];
          const bool a = odd_bf16(w), b = odd_bf16(w >> 16);
          odd |= a | b;
          vreg[i][j] = w & (a ? 0xffff0000u : 0xffffffffu) & (b ? 0xffffu : 0xffffffffu);
        }
        if (odd) s_odd = 1;
      }
      *reinterpret_cast<u32x4_t *>(ks + kr * KST + e0) = kreg[i];
      *reinterpret_cast<u32x4_t *>(vs + kr * VST + e0) = vreg[i];
    }
  };
  if (tid == 0) s_odd = 0;
  if (nkt) load(it.k0);
  __syncthreads();
  if (nkt) store(it.k0, 0);
  // vmcnt(0): with the query fragments known to be there, the loop's waits are for keys alone
  // (without it each product waited for the tile just requested: 16 rows over 16128 keys of 40/8
  // heads 26.5 us, 22.7 with it)
  __builtin_amdgcn_s_waitcnt(0x0f70);
  __syncthreads();
  for (int kt = 0; kt < nkt; ++kt) {
    const int key0 = it.k0 + kt * SH_TILE;
    const bool more = kt + 1 < nkt;
    if (more) load(key0 + SH_TILE);
    const bf16_t *ks_ = s_kv + (kt & 1) * (KB + VB), *vs_ = ks_ + KB;
    for (int st = works ? st0 : 2; st < 2; st += st_step) {
      const int sk0 = key0 + st * 32;
      if (sk0 >= k1) break;
      // S^T block: score i is key sk0 + (i / 4) * 8 + hi * 4 + i % 4 of this lane's pair
      f32x16_t sc;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 0.f;
      const bf16_t *krow = ks_ + (st * 32 + (lane & 31)) * KST + hi * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            *reinterpret_cast<const bf16x8_t *>(krow + ks * 16), qf[ks], sc, 0, 0, 0);
      // V^T operand of step t, dims db * 32 + lane % 32: its 8 slots are keys 16 t + 4 hi + 0..3
      // and the same + 8 of the block
      bf16x8_t vf[2][DB];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          typedef short v4s __attribute__((ext_vector_type(4)));
          const bf16_t *vb = vs_ + (st * 32 + 16 * t + 4 * hi + ((lane & 15) >> 2)) * VST +
                             db * 32 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
          const v4s x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) v4s *)(vb));
          const v4s x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) v4s *)(vb + 8 * VST));
          __builtin_memcpy(&vf[t][db], &x0, 8);
          __builtin_memcpy(reinterpret_cast<char *>(&vf[t][db]) + 8, &x1, 8);
        }
      const bool pre = WHOLE && key0 < it.shift;
      if (sk0 + 32 > (pre ? it.first : all_see)) {
        const int lim = (pre ? it.first : seen) - (sk0 + hi * 4);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if ((i >> 2) * 8 + (i & 3) >= lim) sc[i] = -INFINITY;
      }
      float mx = sc[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
      // the running maximum rises only when some score exceeds it by more than 2^8
      if (__ballot(mx * scale_log2 > m_run + 8.f)) {
        const float mp = fmaxf(mx, __shfl_xor(mx, 32, 64)) * scale_log2;
        const float m_new = fmaxf(m_run, mp);
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] *= alpha;
        l_run *= alpha;
        m_run = m_new;
      }
      const float m_off = m_run == -INFINITY ? 0.f : m_run;  // (no key yet: every p is 0)
      float pv[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        pv[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], scale_log2, -m_off));
        l_run += pv[i];
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        uint32_t pw[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) pw[j] = pack_bf2(pv[8 * t + 2 * j], pv[8 * t + 2 * j + 1]);
        bf16x8_t pb;
        __builtin_memcpy(&pb, pw, 16);
#pragma unroll
        for (int db = 0; db < DB; ++db)
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[t][db], pb, o[db], 0, 0, 0);
      }
    }
    if (more) store(key0 + SH_TILE, (kt + 1) & 1);
    __syncthreads();
  }
  float l = l_run + __shfl_xor(l_run, 32, 64);
  if (groups < 4) {  // the two waves of a group: the odd one hands over through LDS
    float *x = reinterpret_cast<float *>(s_kv) + group * (HD / 2 + 2) * 64 + lane;
    if (works && (wave & 1)) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[(db * 16 + i) * 64] = o[db][i];
      x[HD / 2 * 64] = m_run;
      x[(HD / 2 + 1) * 64] = l;
    }
    __syncthreads();
    if (!works || (wave & 1)) return;
    const float m2 = x[HD / 2 * 64], l2 = x[(HD / 2 + 1) * 64];
    const float mm = fmaxf(m_run, m2), off = mm == -INFINITY ? 0.f : mm;
    // a half without a key has m = -inf, l = 0 and o = 0; one of NaN scores l = NaN
    const float a = __builtin_amdgcn_exp2f(m_run - off), b = __builtin_amdgcn_exp2f(m2 - off);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = a * o[db][i] + b * x[(db * 16 + i) * 64];
    l = a * l + b * l2;
    m_run = mm;
  }
  if (!valid) return;
  if (s_odd) {  // values left out above that this pair sees
    for (int k = max(max(it.k0, it.shift), all_see); k < seen; ++k) {
      const bf16_t *vr = V + ((it.base + k - it.shift) * hkv + it.kvh) * HD + hi * 4;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const uint2 w = *reinterpret_cast<const uint2 *>(vr + db * 32 + q4 * 8);
          const uint32_t x[4] = {w.x & 0xffffu, w.x >> 16, w.y & 0xffffu, w.y >> 16};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (odd_bf16(x[j])) o[db][4 * q4 + j] += __uint_as_float(x[j] << 16);
        }
    }
  }
  // o[db][i] is dim db * 32 + (i / 4) * 8 + hi * 4 + i % 4 of the pair
  if (p.slots > 1) {
    float big = 0.f;  // the pair's largest finite value
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float x = fabsf(o[db][i]);
        big = x < INFINITY ? fmaxf(big, x) : big;
      }
    big = fmaxf(big, __shfl_xor(big, 32, 64));
    const int e = max(__builtin_amdgcn_frexp_expf(big), -100) - 15;
    const float down = ldexpf(1.f, -e);
    _Float16 *po = part_o + prow * HD + hi * 4;
    typedef _Float16 f16x4_t __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        f16x4_t x;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = (_Float16)(o[db][4 * q4 + j] * down);
        *reinterpret_cast<f16x4_t *>(po + db * 32 + q4 * 8) = x;
      }
    if (hi == 0) part_ml[prow] = make_float4(m_run, l, ldexpf(1.f, e), 0.f);
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  bf16_t *orow = out + ((size_t)r * hq + head) * HD + hi * 4;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4)
      store4(orow + db * 32 + q4 * 8, o[db][4 * q4] * inv, o[db][4 * q4 + 1] * inv,
             o[db][4 * q4 + 2] * inv, o[db][4 * q4 + 3] * inv);
  if (lse && hi == 0)
    lse[(size_t)r * hq + head] =
        l == 0.f ? -INFINITY : (m_run == -INFINITY ? 0.f : m_run * 0.6931471805599453f) + logf(l);
}

// out = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s over a pair's slots, M = max m_s. A slot
// holds (m, l, f) and its output over f: fp32 values with f = 1, or fp16 with f a power of two
// that brings the largest to [2^14, 2^15). fp16 carries 11 bits of a slot's large values, three
// more than the bf16 result keeps, at half the traffic of fp32. A slot whose keys the pair's tile
// does not reach holds f = 0: its output was not written and takes no part. Every other slot
// counts whatever its weight is, so that what is NaN in one (m = -inf, l = NaN where all scores
// are NaN) is NaN in the result, as where the keys are not split.
__device__ __forceinline__ void part_load8(const float *p, float (&x)[8]) { load8(p, x); }
__device__ __forceinline__ void part_load8(const _Float16 *p, float (&x)[8]) {
  typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
  const f16x8_t v = *reinterpret_cast<const f16x8_t *>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
}
__device__ __forceinline__ bool slot_counts(float4 ml) { return ml.z != 0.f; }
__device__ __forceinline__ float slot_factor(float4 ml, float M) {
  return M == -INFINITY ? 1.f : exp2f(ml.x - M);  // (no maximum: scores NaN, or no key seen)
}
__device__ __forceinline__ float merged_lse(float M, float l) {
  if (l == 0.f) return -INFINITY;
  return (M == -INFINITY ? 0.f : M * 0.6931471805599453f) + logf(l);
}

// Few slots: a thread has 8 dims of a pair and requests all slots at once.
constexpr int MERGE_FEW = 4;
template <typename TS, typename TP, int FEW>
__global__ __launch_bounds__(256) void k_shared_merge_few(SharedBatch s, int slots, int hq, int hd,
                                                          const TP *__restrict__ part_o,
                                                          const float4 *__restrict__ part_ml,
                                                          TS *__restrict__ out,
                                                          float *__restrict__ lse) {
  const int per = hd >> 3;
  const size_t id = (size_t)blockIdx.x * 256 + threadIdx.x, item = id / per;
  const int e0 = (int)(id - item * per) * 8;
  if (item >= (size_t)shared_live(s) * hq) return;
  const size_t stride = (size_t)s.n_rows * hq;
  float4 ml[FEW];
  float x[FEW][8];
#pragma unroll
  for (int u = 0; u < FEW; ++u)
    if (u < slots) {
      ml[u] = part_ml[u * stride + item];
      part_load8(part_o + (u * stride + item) * hd + e0, x[u]);
    }
  float M = -INFINITY, l = 0.f, a[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = 0.f;
#pragma unroll
  for (int u = 0; u < FEW; ++u)
    if (u < slots) M = fmaxf(M, ml[u].x);
#pragma unroll
  for (int u = 0; u < FEW; ++u)
    if (u < slots) {
      if (!slot_counts(ml[u])) continue;
      const float w = slot_factor(ml[u], M);
      l = fmaf(w, ml[u].y, l);
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = fmaf(w * ml[u].z, x[u][i], a[i]);
    }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] *= inv;
  store8(out + item * hd + e0, a);
  if (lse && e0 == 0) lse[item] = merged_lse(M, l);
}

// Blocks of a merge with a wave or a block per pair: a grid dimension has fewer than 2^32 threads.
static dim3 merge_grid(size_t blocks) {
  constexpr size_t WIDE = 1 << 20;
  return dim3((unsigned)std::min(blocks, WIDE), (unsigned)((blocks + WIDE - 1) / WIDE));
}
__device__ __forceinline__ size_t merge_block() {
  return (size_t)blockIdx.y * gridDim.x + blockIdx.x;
}

// Up to 32 slots: a wave per pair, its lanes a slot's (m, l, f) each, while HD / 8 lanes take the
// outputs of a slot and 64 / (HD / 8) slots are read at a time, the first MERGE_AHEAD of a lane
// requested with the statistics: one round trip to memory and no barrier. Attention of 235 rows
// over 1386 keys of 28/4 heads takes 27 us with it, 33 with a block per pair as below, 126 over
// 549 of 24/8 17 and 20; one row in 64 splits (28 pairs) 20.5 and 18.8.
constexpr int MERGE_WAVE = 32, MERGE_AHEAD = 4;
template <typename TS, typename TP, int HD>
__global__ __launch_bounds__(256) void k_shared_merge_wave(SharedBatch s, int slots, int hq,
                                                           const TP *__restrict__ part_o,
                                                           const float4 *__restrict__ part_ml,
                                                           TS *__restrict__ out,
                                                           float *__restrict__ lse) {
  constexpr int PER = HD / 8, TEAMS = 64 / PER;
  const int lane = threadIdx.x & 63, team = lane / PER, e0 = lane % PER * 8;
  const size_t item = merge_block() * 4 + (threadIdx.x >> 6), stride = (size_t)s.n_rows * hq;
  if (item >= (size_t)shared_live(s) * hq) return;
  const float4 ml =
      lane < slots ? part_ml[lane * stride + item] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
  float x[MERGE_AHEAD][8];
  auto request = [&](int u0) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < MERGE_AHEAD; ++q)
      part_load8(part_o + (min(u0 + q * TEAMS + team, slots - 1) * stride + item) * HD + e0, x[q]);
  };
  request(0);
  const float M = wave_max(ml.x), w = slot_factor(ml, M);
  const float l = wave_sum(slot_counts(ml) ? w * ml.y : 0.f);
  const float wf = slot_counts(ml) ? w * ml.z : -1.f;  // (-1: takes no part)
  float a[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = 0.f;
  for (int u0 = 0; u0 < slots; u0 += MERGE_AHEAD * TEAMS) {
    if (u0 > 0) request(u0);
#pragma unroll
    for (int q = 0; q < MERGE_AHEAD; ++q) {
      const int u = u0 + q * TEAMS + team;
      const float wq = __shfl(wf, u & 63, 64);
      if (u < slots && !(wq < 0.f)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = fmaf(wq, x[q][i], a[i]);
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int o = PER; o < 64; o <<= 1) a[i] += __shfl_xor(a[i], o, 64);
    a[i] *= inv;
  }
  if (team == 0) store8(out + item * HD + e0, a);
  if (lse && lane == 0) lse[item] = merged_lse(M, l);
}

// Many slots: block = one pair. Its threads have a slot's (m, l, f) each, for the maximum, the
// factors and their sum; then 256 / (hd / 8) teams of hd / 8 threads take the slots in turn, four
// outputs requested at a time, and are added in order through LDS.
static_assert(MERGE_SLOTS % 256 == 0, "a block takes 256 slots at a time");
template <typename TS, typename TP, int HD>
__global__ __launch_bounds__(256) void k_shared_merge(SharedBatch s, int slots, int hq,
                                                      const TP *__restrict__ part_o,
                                                      const float4 *__restrict__ part_ml,
                                                      TS *__restrict__ out,
                                                      float *__restrict__ lse) {
  constexpr int PER = HD / 8, TEAMS = 256 / PER;
  __shared__ float s_w[MERGE_SLOTS];
  __shared__ float s_a[TEAMS][HD];
  __shared__ float s_m[4], s_l[4];
  const int tid = threadIdx.x, wave = tid >> 6;
  const size_t item = merge_block(), stride = (size_t)s.n_rows * hq;
  if (item >= (size_t)shared_live(s) * hq) return;
  float4 ml[MERGE_SLOTS / 256];
  float M = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < MERGE_SLOTS / 256; ++i) {
    const int u = tid + 256 * i;
    if (256 * i < slots) {
      ml[i] = u < slots ? part_ml[u * stride + item] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
      M = fmaxf(M, ml[i].x);
    }
  }
  M = wave_max(M);
  if ((tid & 63) == 0) s_m[wave] = M;
  __syncthreads();
  M = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
#pragma unroll
  for (int i = 0; i < MERGE_SLOTS / 256; ++i) {
    const int u = tid + 256 * i;
    if (u < slots) {
      const bool counts = slot_counts(ml[i]);
      const float w = slot_factor(ml[i], M);
      if (counts) l = fmaf(w, ml[i].y, l);
      s_w[u] = counts ? w * ml[i].z : -1.f;  // (-1: takes no part)
    }
  }
  l = wave_sum(l);
  if ((tid & 63) == 0) s_l[wave] = l;
  __syncthreads();
  l = ((s_l[0] + s_l[1]) + s_l[2]) + s_l[3];
  const int e0 = (tid % PER) * 8, team = tid / PER;
  float a[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = 0.f;
  for (int u0 = team; u0 < slots; u0 += 4 * TEAMS) {
    float x[4][8], w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int u = u0 + q * TEAMS;
      w[q] = u < slots ? s_w[u] : -1.f;
      part_load8(part_o + (min(u, slots - 1) * stride + item) * HD + e0, x[q]);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (!(w[q] < 0.f)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = fmaf(w[q], x[q][i], a[i]);
      }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) s_a[team][e0 + i] = a[i];
  __syncthreads();
  if (tid < HD) {
    float o = s_a[0][tid];
#pragma unroll
    for (int q = 1; q < TEAMS; ++q) o += s_a[q][tid];
    store1(out + item * HD + tid, l == 0.f ? 0.f : o / l);
  }
  if (lse && tid == 0) lse[item] = merged_lse(M, l);
}

__device__ __forceinline__ bool odd_f32(float x) {
  return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u;
}

// fp32, on v_mfma_f32_16x16x4_f32. Block = 16 pairs; its waves take the 16-key tiles of the
// item's range in turn, each with its own maximum, sum and output, merged through LDS in wave
// order at the end, so that the loop has no barrier; keys and values come straight to
// registers, a tile ahead. Scores are formed transposed: lane l holds the scores of pair l % 16
// at keys 4 (l / 16) + 0..3 of the tile, the operand layout of O^T = V^T P^T as it is; row
// l % 16 of V^T block c stands for dim (l % 16) * C + c, so that a lane's values are contiguous.
// 85 rows over 2055 keys of 28/4 heads take 43 us: about 10 of a launch do not depend on the keys,
// and an MFMA takes 18 to 22 ns in the loop (15 in a row) with one or two waves a SIMD. Two pair
// tiles a wave, which halve the reads from L2, were slower (49 us).
template <int HD, bool WHOLE>
__global__ __launch_bounds__(256, 2) void k_shared_f32(
    SharedBatch s, SharedPlan p, const float *__restrict__ Q, const float *__restrict__ Kp,
    const float *__restrict__ Vp, const float *__restrict__ Ko, const float *__restrict__ Vo,
    int hq, int hkv, float scale_log2, float *__restrict__ out, float *__restrict__ lse,
    float *__restrict__ part_o, float4 *__restrict__ part_ml) {
  constexpr int C = HD / 16, NW = 4;
  __shared__ float s_o[NW][HD][17];
  __shared__ float s_m[NW][16], s_l[NW][16];
  __shared__ int s_odd;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lr = lane & 15, lg = lane >> 4, G = hq / hkv;
  SharedItem it;
  if (!shared_item<WHOLE>(s, p, hkv, G, it)) return;
  const float *K = it.own < 0 ? Kp : Ko, *V = it.own < 0 ? Vp : Vo;
  const int n_pairs = (it.r1 - it.r0) * G, v = it.v0 + lr;
  const bool valid = v < n_pairs;
  const int r = it.r0 + (valid ? v : it.v0) / G, head = it.kvh * G + (valid ? v : it.v0) % G;
  const int seen = valid ? shared_seen(it, r) : 0;
  const int last = min(n_pairs, it.v0 + 16) - 1;
  const int k1 = shared_seen(it, it.r0 + last / G), all_see = shared_seen(it, it.r0 + it.v0 / G);
  if (k1 <= it.k0 && p.slots > 1) {
    if (tid < 16 && valid)
      part_ml[((size_t)it.slot * s.n_rows + r) * hq + head] =
          make_float4(-INFINITY, 0.f, 0.f, 0.f);
    return;
  }
  if (tid == 0) s_odd = 0;
  __syncthreads();
  f32x4_t qf[C], o[C];
  {
    const float *q = Q + ((size_t)r * hq + head) * HD + lg * 4;
#pragma unroll
    for (int c = 0; c < C; ++c) qf[c] = *reinterpret_cast<const f32x4_t *>(q + 16 * c);
  }
  const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int c = 0; c < C; ++c) o[c] = zero;
  float m = -INFINITY, l = 0.f;  // of pair lr (l: this lane's quarter of the keys)
  struct Tile {
    f32x4_t k[C];
    float v[4][C];
  };
  // keys past the last one re-read it (where no own key is seen it is the prefix's: own rows
  // before `shift` do not exist)
  auto fetch = [&](Tile &t, int key0) __attribute__((always_inline)) {
    const bool pre = WHOLE && (key0 < it.shift || k1 == it.first);
    const float *kb = pre ? Kp : K, *vb = pre ? Vp : V;
    const int end = (pre ? it.first : k1) - 1;
    const size_t base = pre ? 0 : it.base - it.shift;  // (wraps; key + base does not)
    const float *k = kb + ((base + min(key0 + lr, end)) * hkv + it.kvh) * HD + lg * 4;
#pragma unroll
    for (int c = 0; c < C; ++c) t.k[c] = *reinterpret_cast<const f32x4_t *>(k + 16 * c);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float *x =
          vb + ((base + min(key0 + lg * 4 + e, end)) * hkv + it.kvh) * HD + lr * C;
#pragma unroll
      for (int c = 0; c < C; c += 4)
        *reinterpret_cast<f32x4_t *>(&t.v[e][c]) = *reinterpret_cast<const f32x4_t *>(x + c);
    }
  };
  auto attend = [&](Tile &t, int key0) __attribute__((always_inline)) {
    f32x4_t s0 = zero, s1 = zero;  // two chains of dependent MFMAs
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(t.k[c][e], qf[c][e], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(t.k[c][e + 1], qf[c][e + 1], s1, 0, 0, 0);
      }
    f32x4_t x = s0 + s1;
    const bool pre = WHOLE && key0 < it.shift;
    const int see = pre ? it.first : seen, all = pre ? it.first : all_see;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      x[e] = key0 + lg * 4 + e < see ? x[e] * scale_log2 : -INFINITY;
    if (key0 + 16 > all) {  // a hidden value that is not finite must not meet p = 0
      bool odd = false;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (key0 + lg * 4 + e >= all) {
#pragma unroll
          for (int c = 0; c < C; ++c)
            if (odd_f32(t.v[e][c])) {
              odd = true;
              t.v[e][c] = 0.f;
            }
        }
      if (odd) s_odd = 1;
    }
    float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_new = fmaxf(m, mx);
    const float off = m_new == -INFINITY ? 0.f : m_new;  // no key yet: every p is 0
    const float alpha = __builtin_amdgcn_exp2f(m - off);
    f32x4_t q;
#pragma unroll
    for (int e = 0; e < 4; ++e) q[e] = __builtin_amdgcn_exp2f(x[e] - off);
    l = l * alpha + ((q[0] + q[1]) + (q[2] + q[3]));
    m = m_new;
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] *= alpha;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int c = 0; c < C; ++c)
        o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.v[e][c], q[e], o[c], 0, 0, 0);
  };
  constexpr int STEP = NW * 16;
  int key0 = it.k0 + wave * 16;
  if (key0 < k1) {
    Tile t0, t1;
    fetch(t0, key0);
    while (true) {  // the next tile (the last key where there is none) is in flight meanwhile
      fetch(t1, key0 + STEP);
      attend(t0, key0);
      key0 += STEP;
      if (key0 >= k1) break;
      fetch(t0, key0 + STEP);
      attend(t1, key0);
      key0 += STEP;
      if (key0 >= k1) break;
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  // o[c][e] is dim (4 lg + e) C + c of pair lr
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e) s_o[wave][(4 * lg + e) * C + c][lr] = o[c][e];
  if (lg == 0) {
    s_m[wave][lr] = m;
    s_l[wave][lr] = l;
  }
  __syncthreads();
  for (int i = wave; i < 16 && it.v0 + i < n_pairs; i += NW) {  // a wave per pair, lanes on dims
    const int vi = it.v0 + i, ri = it.r0 + vi / G, hi = it.kvh * G + vi % G;
    float mm = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) mm = fmaxf(mm, s_m[w][i]);
    float so[HD / 64] = {}, sl = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      // a wave without a key of the pair has l = 0 (m = -inf is also what NaN scores leave, with
      // a sum of NaN)
      const float lw = s_l[w][i], a = __builtin_amdgcn_exp2f(s_m[w][i] - mm);
      if (lw == 0.f) continue;
      sl = fmaf(mm == -INFINITY ? 1.f : a, lw, sl);
#pragma unroll
      for (int c = 0; c < HD / 64; ++c) so[c] = fmaf(a, s_o[w][64 * c + lane][i], so[c]);
    }
    if (s_odd) {  // values left out above that this pair sees
      const int end = shared_seen(it, ri);
      for (int k = max(max(it.k0, it.shift), all_see); k < end; ++k) {
        const float *x = V + ((it.base + k - it.shift) * hkv + it.kvh) * HD + lane;
#pragma unroll
        for (int c = 0; c < HD / 64; ++c)
          if (odd_f32(x[64 * c])) so[c] += x[64 * c];
      }
    }
    const size_t row = (size_t)ri * hq + hi;
    if (p.slots > 1) {
      const size_t prow = (size_t)it.slot * s.n_rows * hq + row;
#pragma unroll
      for (int c = 0; c < HD / 64; ++c) part_o[prow * HD + 64 * c + lane] = so[c];
      if (lane == 0) part_ml[prow] = make_float4(mm, sl, 1.f, 0.f);
    } else {
      const float inv = sl == 0.f ? 0.f : 1.0f / sl;
#pragma unroll
      for (int c = 0; c < HD / 64; ++c) out[row * HD + 64 * c + lane] = so[c] * inv;
      if (lse && lane == 0)
        lse[row] =
            sl == 0.f ? -INFINITY : (mm == -INFINITY ? 0.f : mm * 0.6931471805599453f) + logf(sl);
    }
  }
}

// ---- the weights that keys received ----------------------------------------------------
// Scores again, S = Q K^T, on the matrix cores (bf16: 32x32x16, fp32: 16x16x4), with pairs as
// rows and keys as columns, so that a lane holds scores of one key: p = exp(s - lse) is summed
// over pairs inside the lane, and a key's sum never leaves its column. A wave keeps a tile of
// keys in registers; the pair tiles pass through LDS for the block's four waves, the next one
// in flight. (Each wave fetching the queries itself was bound by that: 32 rows of 256 bytes
// are 32 cache lines an instruction; 1171 rows over 4516 keys of 24/8 heads took 162 us, now 49.)
// Many rows are bound by the instructions of the exponentials and sums between the products and
// by whole blocks a unit, few by latency and the keys' bytes (16 rows over 16128 keys of 40/8 heads
// 10.7 us, 3.5 TB/s).
typedef __attribute__((ext_vector_type(4))) int i32x4_t;
template <typename TS>
struct WeightTile;
template <>
struct WeightTile<bf16_t> {  // 32 pairs x 32 keys; C value i of a lane: row pair(i)
  static constexpr int PAIRS = 32, KEYS = 32, NC = 16;
  typedef f32x16_t Acc;
  __device__ static int pair(int i, int sub) { return (i >> 2) * 8 + sub * 4 + (i & 3); }
  __device__ static Acc mma(u32x4_t q, u32x4_t k, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, q),
                                                   __builtin_bit_cast(bf16x8_t, k), c, 0, 0, 0);
  }
};
template <>
struct WeightTile<float> {  // 16 x 16
  static constexpr int PAIRS = 16, KEYS = 16, NC = 4;
  typedef f32x4_t Acc;
  __device__ static int pair(int i, int sub) { return sub * 4 + i; }
  __device__ static Acc mma(u32x4_t q, u32x4_t k, Acc c) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(q[e]), __uint_as_float(k[e]), c, 0,
                                               0, 0);
    return c;
  }
};

// Blocks [0, prefix_blocks): (part, key block, KV head), part: a share of the pair tiles, whose
// sums go to a buffer of their own where there are several; then (request, key block, part of
// the request's tiles, KV head) of the own keys.
struct WeightPlan {
  int nk, parts, part_pairs, key_blocks, prefix_blocks;
  int own_parts, own_pairs, own_blocks;  // own_blocks: of keys
};

// NK: key tiles of a wave. Two halve the LDS reads of a pair tile, which bound long walks.
template <typename TS, int HD, int NK>
__global__ __launch_bounds__(256, 2) void k_attn_weights(SharedBatch s, WeightPlan p,
                                                      const TS *__restrict__ Q,
                                                      const float *__restrict__ lse,
                                                      const TS *__restrict__ Kp,
                                                      const TS *__restrict__ Ko, int hq, int hkv,
                                                      float scale_log2, const float *wp_prev,
                                                      float *wp, const float *wo_prev,
                                                      float *wo) {
  typedef WeightTile<TS> W;
  constexpr int NSUB = 64 / W::KEYS;               // lanes that share a row or column
  constexpr int ROW = HD * sizeof(TS), CPR = ROW / 16, C = CPR / NSUB;
  constexpr int STRIDE = ROW + 16;                 // fragment reads on all banks
  constexpr int NCH = W::PAIRS * CPR / 256;        // 16-byte chunks of a tile per thread
  __shared__ __attribute__((aligned(16))) char s_q[2][W::PAIRS * STRIDE];
  __shared__ __attribute__((aligned(16))) float s_lse[2][W::PAIRS];
  __shared__ __attribute__((aligned(16))) int s_seen[2][W::PAIRS];
  __shared__ int s_masked[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, G = hq / hkv;
  const int li = lane % W::KEYS, sub = lane / W::KEYS;  // this lane's row / column, and its part
  int id = blockIdx.x, r0 = 0, r1, n, n_all, own = 0, kb, v0 = 0, n_pairs;
  const TS *K;
  const float *prev;
  float *w;
  const bool prefix = id < p.prefix_blocks;
  if (!prefix) id -= p.prefix_blocks;
  const int kvh = id % hkv;
  id /= hkv;
  if (prefix) {
    kb = id % p.key_blocks;
    const int part = id / p.key_blocks;
    r1 = shared_live(s);
    n = n_all = s.prefix_len;
    K = Kp;
    prev = wp_prev ? wp_prev + (size_t)kvh * n : nullptr;
    w = wp + ((size_t)part * hkv + kvh) * n;
    v0 = part * p.part_pairs;
    n_pairs = min(r1 * G, v0 + p.part_pairs);
  } else {
    const int part = id % p.own_parts;
    id /= p.own_parts;
    const int b = id / p.own_blocks;
    kb = id - b * p.own_blocks;
    shared_rows(s, b, r0, r1);
    n = own = min(max(s.own_len[b], 0), s.own_rows);
    n_all = s.own_rows;
    K = Ko + (size_t)b * s.own_rows * hkv * HD;
    const size_t o = ((size_t)b * hkv + kvh) * n_all;
    prev = wo_prev ? wo_prev + o : nullptr;
    w = wo + (size_t)part * s.n_req * hkv * n_all + o;
    v0 = part * p.own_pairs;
    n_pairs = min((r1 - r0) * G, v0 + p.own_pairs);
  }
  constexpr int KEYS = NK * W::KEYS;  // of a wave
  const int j0 = kb * 4 * KEYS, j = j0 + wave * KEYS + li;
  float sum[NK];
#pragma unroll
  for (int u = 0; u < NK; ++u) sum[u] = 0.f;
  if (j0 < n && v0 < n_pairs) {
    u32x4_t kf[NK][C];
#pragma unroll
    for (int u = 0; u < NK; ++u) {
      const char *k = reinterpret_cast<const char *>(
          K + ((size_t)min(j + u * W::KEYS, n - 1) * hkv + kvh) * HD);
#pragma unroll
      for (int c = 0; c < C; ++c)
        kf[u][c] = *reinterpret_cast<const u32x4_t *>(k + (c * NSUB + sub) * 16);
    }
    // This thread's chunks of a tile belong to pairs that are PAIRS apart from one tile to the
    // next: their places (in query heads) are carried along, without a division per tile. The
    // first threads have a pair's lse and how many keys it sees (0: no pair, or a row without
    // keys).
    const int dr = W::PAIRS / G, dg = W::PAIRS % G, last = (r1 - 1) * hq + kvh * G + G - 1;
    struct Pair {
      int g, at;  // head of the KV head's G, place in [n_rows][hq]
    };
    auto pair_at = [&](int v) { return Pair{v % G, (r0 + v / G) * hq + kvh * G + v % G}; };
    auto next = [&](Pair &x) __attribute__((always_inline)) {
      const bool wrap = x.g + dg >= G;
      x.g += wrap ? dg - G : dg;
      x.at += dr * hq + dg + (wrap ? hq - G : 0);
    };
    Pair mine[NCH], first = pair_at(v0 + tid % W::PAIRS);
#pragma unroll
    for (int i = 0; i < NCH; ++i) mine[i] = pair_at(v0 + (tid + 256 * i) / CPR);
    int row = r0 + (v0 + tid % W::PAIRS) / G;  // of `first`
    struct Tile {
      u32x4_t q[NCH];
      float ls;
      int seen;
    };
    auto load = [&](Tile &x) __attribute__((always_inline)) {  // (past the end: the last pair)
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const char *a = reinterpret_cast<const char *>(Q + (size_t)min(mine[i].at, last) * HD);
        x.q[i] = *reinterpret_cast<const u32x4_t *>(a + (tid + 256 * i) % CPR * 16);
        next(mine[i]);
      }
      x.ls = lse[min(first.at, last)];
      x.seen = row >= r1 ? 0 : prefix ? n : min(max(own - (r1 - row) + 1, 0), n);
      row += dr + (first.g + dg >= G);
      next(first);
    };
    auto store = [&](const Tile &x, int buf) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int c = tid + 256 * i;
        *reinterpret_cast<u32x4_t *>(&s_q[buf][c / CPR * STRIDE + c % CPR * 16]) = x.q[i];
      }
      if (tid < W::PAIRS) {
        const int seen = x.ls == -INFINITY ? 0 : x.seen;
        s_lse[buf][tid] = x.ls * 1.4426950408889634f;
        s_seen[buf][tid] = seen;
        const bool any = __ballot(seen < min(j0 + 4 * KEYS, n)) != 0;
        if (tid == 0) s_masked[buf] = any;
      }
    };
    auto weigh = [&](int buf) __attribute__((always_inline)) {
      typename W::Acc c[NK];
#pragma unroll
      for (int u = 0; u < NK; ++u)
#pragma unroll
        for (int i = 0; i < W::NC; ++i) c[u][i] = 0.f;
      const char *q = &s_q[buf][li * STRIDE + sub * 16];
#pragma unroll
      for (int e = 0; e < C; ++e) {
        const u32x4_t x = *reinterpret_cast<const u32x4_t *>(q + e * NSUB * 16);
#pragma unroll
        for (int u = 0; u < NK; ++u) c[u] = W::mma(x, kf[u][e], c[u]);
      }
      float x[NK][W::NC];
#pragma unroll
      for (int i = 0; i < W::NC / 4; ++i) {
        const f32x4_t off = *reinterpret_cast<const f32x4_t *>(&s_lse[buf][W::pair(4 * i, sub)]);
#pragma unroll
        for (int u = 0; u < NK; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x[u][4 * i + e] =
                __builtin_amdgcn_exp2f(fmaf(c[u][4 * i + e], scale_log2, -off[e]));
      }
      if (s_masked[buf]) {
#pragma unroll
        for (int i = 0; i < W::NC / 4; ++i) {
          const i32x4_t end = *reinterpret_cast<const i32x4_t *>(&s_seen[buf][W::pair(4 * i, sub)]);
#pragma unroll
          for (int u = 0; u < NK; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              x[u][4 * i + e] = j + u * W::KEYS < end[e] ? x[u][4 * i + e] : 0.f;
        }
      }
#pragma unroll
      for (int u = 0; u < NK; ++u) {
#pragma unroll
        for (int o = W::NC / 2; o > 0; o >>= 1)
#pragma unroll
          for (int i = 0; i < o; ++i) x[u][i] += x[u][i + o];
        sum[u] += x[u][0];
      }
    };
    // Loads run two tiles ahead, in registers, and are made whether or not there is a tile: a
    // block alone on its compute unit is else bound by their latency (16 rows over 16128 keys of
    // 40/8 heads 11.3 -> 10.9 us).
    Tile a, b;
    load(a);
    load(b);
    store(a, 0);
    __syncthreads();
    while (true) {
      load(a);
      weigh(0);
      v0 += W::PAIRS;
      if (v0 >= n_pairs) break;
      store(b, 1);
      __syncthreads();
      load(b);
      weigh(1);
      v0 += W::PAIRS;
      if (v0 >= n_pairs) break;
      store(a, 0);
      __syncthreads();
    }
  }
#pragma unroll
  for (int u = 0; u < NK; ++u) {
#pragma unroll
    for (int o = W::KEYS; o < 64; o <<= 1) sum[u] += __shfl_xor(sum[u], o, 64);
    const int k = j + u * W::KEYS;
    if (sub == 0 && k < n_all) w[k] = (prev ? prev[k] : 0.f) + (k < n ? sum[u] : 0.f);
  }
}

// w = prev + the parts' sums in order: n weights of the prefix, n_own of the own keys.
struct WeightSum {
  const float *part, *prev;
  float *w;
  int parts;
  size_t n;
};
// Blocks [0, blocks) are the prefix's, then the own keys'.
__device__ __forceinline__ void sum_parts(const WeightSum &x, size_t i) {
  if (i >= x.n) return;
  float sum = x.part[i];
  for (int q = 1; q < x.parts; ++q) sum += x.part[q * x.n + i];
  x.w[i] = (x.prev ? x.prev[i] : 0.f) + sum;
}
__global__ __launch_bounds__(256) void k_weight_parts(WeightSum shared, int blocks, WeightSum own) {
  const int id = blockIdx.x;
  if (id < blocks) sum_parts(shared, (size_t)id * 256 + threadIdx.x);
  else sum_parts(own, (size_t)(id - blocks) * 256 + threadIdx.x);
}

// Items of a call. bf16 tiles have 32, 64 or 128 pairs (see k_shared_bf16), fp32 ones 16; two
// blocks share a compute unit. Own keys go in chunks of two key tiles at least (their lengths
// are known on the device alone: most of the room for them may be empty). The prefix is cut
// into the number of splits whose estimated end is the earliest, in units of the time that a
// block alone on its unit takes for a key tile (1.75 us): such a block takes 4.3 + its tiles, one
// that shares its unit 7.5 + 1.7 times them. Blocks that fit the chip together end with the
// longest of them; else whole rounds of prefix blocks, the rest of them, and the own keys'
// blocks that had no place follow each other. Each split's partials cost a write and a read.
// Up to six tiles of prefix and own keys together, each request's blocks take both (whole) and
// there is nothing to merge: 16 requests over 60 / 190 / 320 / 450 keys and up to 64 own of 28/4
// heads 7.3 / 9.4 / 11.5 / 15.4 us whole, 10.1 / 12.8 / 13.0 / 11.9 in pieces (fp32, 4 heads of
// 64: 6.2 / 7.9 / 9.5 / 12.5 and 8.5 / 10.1 / 10.1 / 10.1).
//   16 rows over 4096 / 8192 / 16384 / 32768 / 65536 keys of 40/8 heads, this launch alone: 256
//   prefix blocks 11.1 / 14.6 / 21.0 / 34.9 / 62.7 us, 512 of them - / 19.6 / 23.3 / 37.1 / 60.8;
//   with 128 blocks of own keys and 16128 keys 256 prefix blocks are 4 us faster than 504 (own
//   blocks wait for a place). 1328 rows over 16128 (416 tiles of pairs): 516 us with one split,
//   491 with three, 511 with four. 85 fp32 rows over 2055 keys of 28/4 heads: 57 us with two, 43
//   with three, 49 with four.
static SharedPlan shared_plan(const SharedBatch &s, int hq, int hkv, int hd, int dtype) {
  constexpr double BYTES = 7e6;  // partials moved in a tile's time
  SharedPlan p{};
  const int G = hq / hkv, blocks = 2 * gemm_cu_count();
  const bool bf = dtype == AKVS_BF16;
  auto tile_pairs = [&](long long pairs) {
    return !bf ? 16 : pairs > 64 ? 128 : pairs > 32 ? 64 : 32;
  };
  auto tiles_of = [](long long n, int per) { return (int)((n + per - 1) / per); };
  const long long pp = (long long)s.n_rows * G, op = (long long)s.rows_max * G;
  p.p_pairs = tile_pairs(pp);
  p.p_tiles = tiles_of(pp, p.p_pairs);
  p.o_pairs = tile_pairs(op);
  p.o_tiles = tiles_of(op, p.o_pairs);
  auto cut = [&](long long n, int kt, int *pieces, int *piece_keys) {
    n = std::max(1LL, std::min<long long>(n, std::min(MERGE_SLOTS / 2, kt / 2)));
    const int per = kt ? (int)((kt + n - 1) / n) : 1;
    *piece_keys = per * SH_TILE;
    *pieces = (kt + per - 1) / per;
  };
  const long long o_items = s.own_rows ? (long long)s.n_req * p.o_tiles * hkv : 0;
  cut(o_items ? blocks / o_items : 1, tiles_of(s.own_rows, SH_TILE), &p.chunks, &p.chunk_keys);
  const int ot = tiles_of(s.own_rows, SH_TILE);
  p.whole = s.prefix_len > 0 && o_items > 0 && o_items <= blocks &&
            tiles_of(s.prefix_len, SH_TILE) + ot <= 6;
  if (p.whole) {
    p.chunks = p.slots = 1;
    return p;
  }
  const double o_blocks = (double)o_items * p.chunks;
  const long long items = (long long)p.p_tiles * hkv;
  const int kt = tiles_of(s.prefix_len, SH_TILE);
  const double move = (double)s.n_rows * hq * hd * 4 / BYTES;  // of one split's partials
  auto end = [&](long long n) {
    auto alone = [](double tiles) { return tiles + 4.3; };
    auto shared = [](double tiles) { return 1.7 * tiles + 7.5; };
    const double tiles = (double)kt / n, own = p.chunk_keys / SH_TILE;
    const long long count = items * n, all = count + (long long)o_blocks;
    double t;
    if (all <= blocks / 2) {
      t = std::max(alone(tiles), o_blocks > 0 ? alone(own) : 0);
    } else if (all <= blocks) {
      t = std::max(shared(tiles), o_blocks > 0 ? shared(own) : 0);
    } else {
      const long long rest = count % blocks;
      t = count / blocks * shared(tiles);
      if (rest) t += rest <= blocks / 2 && count > blocks ? alone(tiles) : shared(tiles);
      if (o_blocks > 0) t += shared(own) * std::max(1.0, o_blocks / blocks);
    }
    return t + move * n + (n + p.chunks > 1 ? 3 : 0);
  };
  long long best = 1;
  const long long most = std::max(1, std::min(MERGE_SLOTS / 2, kt / 2));
  auto consider = [&](double n) {
    const long long k = std::max(1LL, std::min((long long)n, most));
    if (end(k) < end(best)) best = k;
  };
  if (items && kt) {
    consider((blocks / 2 - o_blocks) / items);
    consider((blocks - o_blocks) / items);
    for (int rounds = 1; rounds <= 8; ++rounds) consider((double)rounds * blocks / items);
  }
  cut(best, kt, &p.splits, &p.split_keys);
  p.prefix_blocks = p.splits * p.p_tiles * hkv;
  p.slots = p.splits + p.chunks;
  return p;
}

size_t shared_part_floats(const SharedBatch &s, int hq, int hkv, int hd, int dtype) {
  if (s.n_rows == 0) return 0;
  const SharedPlan p = shared_plan(s, hq, hkv, hd, dtype);
  const size_t items = (size_t)p.slots * s.n_rows * hq;
  return p.slots > 1 ? items * (dtype == AKVS_BF16 ? hd / 2 : hd) + items * 4 : 0;
}

template <typename TS, typename TP, int HD>
static hipError_t shared_merge(const SharedBatch &s, int slots, int hq, const TP *po,
                               const float4 *ml, TS *out, float *lse, hipStream_t st, int eight = 0) {
  const size_t items = (size_t)s.n_rows * hq;
  const dim3 b(256);
  const dim3 gf((unsigned)((items * (HD / 8) + 255) / 256));
  if (slots > MERGE_FEW && slots <= eight) {
    hipLaunchKernelGGL((k_shared_merge_few<TS, TP, 8>), gf, b, 0, st, s, slots, hq, HD, po, ml, out,
                       lse);
    return hipGetLastError();
  }
  if (slots <= MERGE_FEW) {
    hipLaunchKernelGGL((k_shared_merge_few<TS, TP, MERGE_FEW>), gf, b, 0, st, s, slots, hq, HD, po, ml,
                       out, lse);
  } else if (slots <= MERGE_WAVE) {
    const dim3 gm = merge_grid((items + 3) / 4);
    hipLaunchKernelGGL((k_shared_merge_wave<TS, TP, HD>), gm, b, 0, st, s, slots, hq, po, ml, out, lse);
  } else {
    const dim3 gm = merge_grid(items);
    hipLaunchKernelGGL((k_shared_merge<TS, TP, HD>), gm, b, 0, st, s, slots, hq, po, ml, out, lse);
  }
  return hipGetLastError();
}

hipError_t launch_merge_slots(const SharedBatch &s, int slots, int hq, int hd, const void *po,
                              const void *ml, void *out, float *lse, hipStream_t st) {
  const float *o = reinterpret_cast<const float *>(po);
  const float4 *m = reinterpret_cast<const float4 *>(ml);
  bf16_t *O = reinterpret_cast<bf16_t *>(out);
  // (many pairs in up to 8 slots: 13200 in 6 take 8.8 us so, 9.5 with a wave each)
  const int eight = (size_t)s.n_rows * hq >= 4096 ? 8 : 0;
  return hd == 128 ? shared_merge<bf16_t, float, 128>(s, slots, hq, o, m, O, lse, st, eight)
                   : shared_merge<bf16_t, float, 64>(s, slots, hq, o, m, O, lse, st, eight);
}

template <typename TS, int HD>
static hipError_t shared_attention(const SharedBatch &s, const void *q, const void *kp,
                                   const void *vp, const void *ko, const void *vo, int hq,
                                   int hkv, int dtype, void *out, float *lse, float *part,
                                   hipStream_t st) {
  auto x = [](const void *a) { return reinterpret_cast<const TS *>(a); };
  TS *O = reinterpret_cast<TS *>(out);
  SharedPlan p = shared_plan(s, hq, hkv, HD, dtype);
  const size_t items = (size_t)s.n_rows * hq;
  typedef typename std::conditional<sizeof(TS) == 2, _Float16, float>::type TP;
  float4 *ml = reinterpret_cast<float4 *>(part);  // (m, l, f) of every slot, then the outputs
  TP *po = reinterpret_cast<TP *>(ml + p.slots * items);
  size_t blocks = p.prefix_blocks + (size_t)s.n_req * p.chunks * p.o_tiles * hkv;
  if (blocks == 0) {  // no key at all: one item without keys writes the rows' zeros
    p.splits = p.slots = 1;
    p.prefix_blocks = p.p_tiles * hkv;
    blocks = p.prefix_blocks;
  }
  const dim3 g((unsigned)blocks), b(256);
  const float scale = 1.4426950408889634f / sqrtf((float)HD);
#define AKVS_ATTEND(KERNEL_)                                                                      \
  hipLaunchKernelGGL(KERNEL_, g, b, 0, st, s, p, x(q), x(kp), x(vp), x(ko), x(vo), hq, hkv, scale, \
                     O, lse, po, ml)
  if constexpr (sizeof(TS) == 2) {
    if (p.whole) AKVS_ATTEND((k_shared_bf16<HD, true>));
    else AKVS_ATTEND((k_shared_bf16<HD, false>));
  } else {
    if (p.whole) AKVS_ATTEND((k_shared_f32<HD, true>));
    else AKVS_ATTEND((k_shared_f32<HD, false>));
  }
#undef AKVS_ATTEND
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.slots <= 1) return e;
  return shared_merge<TS, TP, HD>(s, p.slots, hq, po, ml, O, lse, st);
}

hipError_t launch_shared_attention(const SharedBatch &s, const void *q, const void *kp,
                                   const void *vp, const void *ko, const void *vo, int hq,
                                   int hkv, int hd, int dtype, void *out, float *lse, float *part,
                                   hipStream_t st) {
  if (s.n_rows == 0) return hipSuccess;
#define AKVS_SHARED(TS_, HD_) \
  shared_attention<TS_, HD_>(s, q, kp, vp, ko, vo, hq, hkv, dtype, out, lse, part, st)
  if (dtype == AKVS_BF16) return hd == 128 ? AKVS_SHARED(bf16_t, 128) : AKVS_SHARED(bf16_t, 64);
  return hd == 128 ? AKVS_SHARED(float, 128) : AKVS_SHARED(float, 64);
#undef AKVS_SHARED
}

// Two key tiles a wave share a pair tile's staging and LDS reads, but a block then has 256 keys and
// its unit three blocks of 166 registers: taken where the prefix makes two such blocks a unit by
// parts of eight tiles (1171 rows over 4516 keys of 24/8 heads: 57 us with two, 63 with one; 584
// over 16128 of 40/8 127 and 140; 189 over 506 of 40/8 23 and 18). The pairs go in parts while the
// keys alone do not fill the units, at least four tiles each. So do a request's over its own keys,
// eight tiles each, or its one block walks them all: 256 rows over 9000 keys and 256 own of
// 28/4 heads 73 us whole, 35 in parts as long as the prefix's, 33 by eight; 1835 rows of 8 requests
// over 2000 92, 55 and 49 (up to 16 blocks a unit: most of the room may be empty).
template <typename TS>
static WeightPlan weight_plan(const SharedBatch &s, int hq, int hkv, bool prefix, bool own) {
  typedef WeightTile<TS> W;
  WeightPlan p;
  const int cus = gemm_cu_count();
  auto tiles_of = [&](long long rows) {
    return (int)((rows * (hq / hkv) + W::PAIRS - 1) / W::PAIRS);
  };
  const int tiles = tiles_of(s.n_rows), own_tiles = tiles_of(s.rows_max);
  const long long wide = (s.prefix_len + 8 * W::KEYS - 1) / (8 * W::KEYS);
  p.nk = wide * hkv * (tiles / 8) >= 2 * cus ? 2 : 1;
  const int keys = 4 * W::KEYS * p.nk;
  p.key_blocks = (s.prefix_len + keys - 1) / keys;
  p.own_blocks = (s.own_rows + keys - 1) / keys;
  const long long blocks = std::max(1LL, (long long)p.key_blocks * hkv);
  long long parts = std::max(1LL, (p.nk == 2 ? 2LL : 4LL) * cus / blocks);
  parts = std::min<long long>(parts, std::max(1, tiles / 4));
  const int per = tiles ? (int)((tiles + parts - 1) / parts) : 1;
  p.parts = tiles ? (tiles + per - 1) / per : 1;
  p.part_pairs = per * W::PAIRS;
  const int walk = std::max(4, std::min(per, 8));
  const long long own_most = 16LL * cus / std::max(1LL, (long long)s.n_req * p.own_blocks * hkv);
  const int own_parts =
      (int)std::max(1LL, std::min<long long>((own_tiles + walk - 1) / walk, own_most));
  const int own_per = std::max(1, (own_tiles + own_parts - 1) / own_parts);
  p.own_parts = std::max(1, (own_tiles + own_per - 1) / own_per);
  p.own_pairs = own_per * W::PAIRS;
  p.prefix_blocks = prefix ? p.parts * p.key_blocks * hkv : 0;
  if (!own) p.own_blocks = 0;
  return p;
}

static size_t own_weights(const SharedBatch &s, int hkv) {
  return (size_t)s.n_req * hkv * s.own_rows;
}
// Floats of the prefix's parts, then of the own keys', where there are several.
static size_t prefix_part_floats(const SharedBatch &s, const WeightPlan &p, int hkv) {
  return p.parts > 1 ? (size_t)p.parts * hkv * s.prefix_len : 0;
}
size_t weight_part_floats(const SharedBatch &s, int hq, int hkv, int dtype) {
  const WeightPlan p = dtype == AKVS_BF16 ? weight_plan<bf16_t>(s, hq, hkv, true, true)
                                          : weight_plan<float>(s, hq, hkv, true, true);
  return prefix_part_floats(s, p, hkv) + (p.own_parts > 1 ? p.own_parts * own_weights(s, hkv) : 0);
}

static size_t weight_blocks(const SharedBatch &s, const WeightPlan &p, int hkv) {
  return p.prefix_blocks + (size_t)s.n_req * p.own_blocks * p.own_parts * hkv;
}
size_t weight_blocks(const SharedBatch &s, int hq, int hkv, int dtype, bool prefix, bool own) {
  const WeightPlan p = dtype == AKVS_BF16 ? weight_plan<bf16_t>(s, hq, hkv, prefix, own)
                                          : weight_plan<float>(s, hq, hkv, prefix, own);
  return weight_blocks(s, p, hkv);
}

template <typename TS>
static hipError_t attention_weights(const SharedBatch &s, const void *q, const float *lse,
                                    const void *kp, const void *ko, int hq, int hkv, int hd,
                                    const float *wp_prev, float *wp, const float *wo_prev,
                                    float *wo, float *part, hipStream_t st) {
  const WeightPlan p = weight_plan<TS>(s, hq, hkv, wp != nullptr, wo != nullptr);
  const size_t blocks = weight_blocks(s, p, hkv);
  if (blocks == 0) return hipSuccess;
  const bool split = p.parts > 1 && p.prefix_blocks > 0;
  const bool own_split = p.own_parts > 1 && p.own_blocks > 0;
  float *own_part = part + prefix_part_floats(s, p, hkv);
  const float scale = 1.4426950408889634f / sqrtf((float)hd);
  auto x = [](const void *a) { return reinterpret_cast<const TS *>(a); };
#define AKVS_WEIGHTS(HD_, NK_)                                                                 \
  hipLaunchKernelGGL((k_attn_weights<TS, HD_, NK_>), dim3((unsigned)blocks), dim3(256), 0, st, s,  \
                     p, x(q), lse, x(kp), x(ko), hq, hkv, scale, split ? nullptr : wp_prev,        \
                     split ? part : wp, own_split ? nullptr : wo_prev, own_split ? own_part : wo)
  if (hd == 128) {
    if (p.nk == 2) AKVS_WEIGHTS(128, 2); else AKVS_WEIGHTS(128, 1);
  } else {
    if (p.nk == 2) AKVS_WEIGHTS(64, 2); else AKVS_WEIGHTS(64, 1);
  }
#undef AKVS_WEIGHTS
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !(split || own_split)) return e;
  const WeightSum shared{part, wp_prev, wp, p.parts, split ? (size_t)hkv * s.prefix_len : 0};
  const WeightSum own{own_part, wo_prev, wo, p.own_parts, own_split ? own_weights(s, hkv) : 0};
  const int blocks_shared = (int)((shared.n + 255) / 256), blocks_own = (int)((own.n + 255) / 256);
  hipLaunchKernelGGL(k_weight_parts, dim3(blocks_shared + blocks_own), dim3(256), 0, st, shared,
                     blocks_shared, own);
  return hipGetLastError();
}

hipError_t launch_attention_weights(const SharedBatch &s, const void *q, const float *lse,
                                    const void *kp, const void *ko, int hq, int hkv, int hd,
                                    int dtype, const float *wp_prev, float *wp,
                                    const float *wo_prev, float *wo, float *part,
                                    hipStream_t st) {
  return dtype == AKVS_BF16 ? attention_weights<bf16_t>(s, q, lse, kp, ko, hq, hkv, hd, wp_prev, wp,
                                                        wo_prev, wo, part, st)
                            : attention_weights<float>(s, q, lse, kp, ko, hq, hkv, hd, wp_prev, wp,
                                                       wo_prev, wo, part, st);
}

}  // namespace akvs
