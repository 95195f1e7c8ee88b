// Attention over sequences in pages of 4-bit codes.
//
// The (row, query head) pairs of a request that read one KV head are the columns of a matrix, as in
// the attention over a shared context. Codes go to the matrix cores as they are, with (scale s,
// zero z) of a group of 64 elements outside the products,
//   q.k   = sum_groups s (sum q c) + z sum q
//   sum p v = sum (p s) (c - 8) + sum p (z + 8 s),
// so that scores hold no rounded operand, and the rounding of p s to fp16 meets what a value
// differs from its group's middle by. A nibble put into the mantissa of a constant is that constant
// plus the code, exactly, in one instruction for two; the constants' share is taken off by the
// matrix cores as well.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "four_bit_dev.h"
#include "kernels.h"
#include "pages_dev.h"

namespace akvs {

// Work items of a call: (pair tile, chunk of its keys, request, KV head), KV heads innermost. The
// device deals blocks out to its parts in turn, so the items that may be empty, the last tiles and
// chunks, are outermost: with them inside, a power of two of them leaves all of the empty ones to
// the same part (6 requests of up to 4 tiles: half of the device idle, 123 us against 101).
struct PagedPlan {
  int pairs, tiles, chunks, chunk_keys;  // pairs: of a tile; chunk_keys: at most
  int slots;                             // blocks of a head at a time; 0: chunk_keys is the cut
  bool many;                             // k_paged_many's
};
constexpr int PG_TILE = 64;  // keys a wave takes at a time
// Parts of the keys leave their outputs in fp32: parts may cancel, and fp16 (scaled by a power of two)
// keeps 11 bits of each. 13200 pairs in 6 parts are merged in 8.8 us, in fp16 in 6.4, after a launch
// that takes 92.6 and 94.7, fp16 having to find the largest value first.

// Sum (MAX: largest, of numbers >= 0) over a wave by DPP: rows of 16, then each row's last to the next.
template <bool MAX>
__device__ __forceinline__ float wave_all(float x) {
  auto step = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
    const float y = __int_as_float(__builtin_amdgcn_update_dpp(
        0, __float_as_int(x), decltype(ctrl)::value, decltype(rows)::value, 0xf, true));
    x = MAX ? fmaxf(x, y) : x + y;
  };
  using std::integral_constant;
  step(integral_constant<int, 0x111>(), integral_constant<int, 0xf>());  // row_shr 1, 2, 4, 8
  step(integral_constant<int, 0x112>(), integral_constant<int, 0xf>());
  step(integral_constant<int, 0x114>(), integral_constant<int, 0xf>());
  step(integral_constant<int, 0x118>(), integral_constant<int, 0xf>());
  step(integral_constant<int, 0x142>(), integral_constant<int, 0xa>());  // row_bcast 15, 31
  step(integral_constant<int, 0x143>(), integral_constant<int, 0xc>());
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// Request b's rows, keys and table, and the keys of a chunk. Where the plan leaves it open, that is
// the least for which the requests' own lengths, a lane each, make one round of blocks, tried at 1 to
// 7/4 of an even share and cut into no more than the plan's chunks; the same in all blocks of a call.
// It costs 0.6 to 1.5 us, and makes up for a max_len far above the lengths, as captured calls have it:
//   8 requests of 3000 to 4000 keys, 28/4 heads: 15.0 us for any max_len; by the plan's cut 14.6 for a
//   max_len of 4000, 16.7 for 16000, 33 for 64000. 6 questions of 39 to 92 rows over 3155 to 8115 keys,
//   40/8 heads: 100 us, 107 for a max_len of 131000; 102 and 307. (32 requests of 4500 to 8128 keys in
//   two chunks each are as fast either way: k_paged_few has the plan's cut below 8 chunks.)
__device__ __forceinline__ const int32_t *paged_request(const PagedBatch &s, const PagedPlan &plan,
                                                        int G, int b, int &r0, int &r1, int &len,
                                                        int &chunk_keys) {
  chunk_keys = plan.chunk_keys;
  if (plan.slots == 0) {
    paged_rows(s, b, r0, r1);
    return paged_keys(s, b, len);
  }
  const int lane = threadIdx.x & 63, mine = min(lane, s.n_req - 1);
  const int q = s.seq ? s.seq[mine] : mine;
  paged_rows(s, mine, r0, r1);
  paged_keys(s, mine, len);
  const float tiles = lane < s.n_req ? (float)(((r1 - r0) * G + plan.pairs - 1) / plan.pairs) : 0.f;
  const int kt = tiles > 0.f ? (len + PG_TILE - 1) / PG_TILE : 0;
  const float work = wave_all<false>(tiles * kt);
  const int most = (int)wave_all<true>((float)kt);
  const int unit = plan.many ? 1 : 4, least = (most + plan.chunks - 1) / plan.chunks;
  int c = plan.chunk_keys / PG_TILE;
  for (int f = 4; f <= 7; ++f) {
    int t = max(max((int)(work * f / (4 * plan.slots)) + 1, least), 2);
    t = (t + unit - 1) / unit * unit;
    if (t >= c) break;
    if (wave_all<false>(tiles * (float)((kt + t - 1) / t)) <= (float)plan.slots) {
      c = t;
      break;
    }
  }
  chunk_keys = max(c, least) * PG_TILE;
  r0 = __builtin_amdgcn_readlane(r0, b);
  r1 = __builtin_amdgcn_readlane(r1, b);
  len = __builtin_amdgcn_readlane(len, b);
  const int own = __builtin_amdgcn_readlane(q, b);
  return s.table + (own >= 0 && own < s.n_seq ? (size_t)own * s.max_pages : 0);
}

// Few pairs. Block = 4 waves over a tile of 16 / NB pairs and one chunk of keys; its waves take the
// chunk's tiles of 64 keys in turn, each with its own maximum, sum and output, merged through LDS at
// the end, so that the loop has no barrier. MFMA 16x16x32, lane l: g = l / 16.
//   Scores, S^T = K Q^T, 16 keys T = 0..3 of the tile at a time: the lane holds the scores of column
//   l % 16 at keys 16 T + 4 g .. + 3; the reduction takes elements 64 group + 16 g + 8 step .. + 7.
//   Outputs, O^T = V^T P^T: a step's reduction takes 16 keys of two T, V^T comes from rows in LDS by
//   the transposing read of 4-bit elements, 16 keys of a dim at once.
// Instructions on scores are what bounds it beside the bytes, so columns are not left empty where
// few pairs leave room (NB > 1): the columns are NB copies of the pairs, and copy T % NB belongs to
// the keys of T. Queries are 0 in the others' columns, so that NB products add into one accumulator,
// and so are a copy's probabilities in the others' places of the reduction.
// Loads of the next tile, and its pages' numbers (scalar: 16 consecutive keys lie in one page, with
// WIDE pages of 64 rows or more the tile) a tile earlier, are in flight meanwhile.
//   32 requests of 4700 to 16000 keys, 40/8 heads: 87 us, 4.8 TB/s of codes and meta. 32 of 4500 to
//   8100 keys whose first 4096 are the same, 28/4 heads: 27 us for 43 MB; a wave's tile takes 2.5 us
//   beside another wave's, instructions on codes (half) and scores.
template <int HD, int NB, bool WIDE>
__global__ __launch_bounds__(256, 2) void k_paged_few(
    PagedBatch s, PagePool p, PagedPlan plan, const bf16_t *__restrict__ Q, int hq, int hkv,
    float scale_log2, bf16_t *__restrict__ out, float *__restrict__ lse,
    float *__restrict__ part_o, float4 *__restrict__ part_ml) {
  constexpr int NG = HD / 64, DB = HD / 16;      // groups of a row, blocks of 16 dims
  constexpr int RB = HD / 2;                     // bytes of a row's codes
  constexpr int VST = RB + 16;                   // row stride in LDS: reads on all banks
  constexpr int VC = RB / 16;                    // 16-byte chunks of a row
  constexpr int NV = PG_TILE * RB / 1024;        // of these per lane
  constexpr int VROWS = 64 / VC;                 // rows that a load of the wave takes
  constexpr int COLS = 16 / NB, NS = 16 / NB;  // NS: a lane's scores of a tile
  constexpr int OST = HD + 4;
  constexpr int STAGE = PG_TILE * VST + 2 * NG * PG_TILE * 4;  // of a wave
  constexpr int MERGE = 16 * OST * 4;
  constexpr int WAVE_BYTES = (STAGE > MERGE ? STAGE : MERGE);
  __shared__ __attribute__((aligned(16))) char s_mem[4 * WAVE_BYTES];
  __shared__ float s_m[4][16], s_l[4][16];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, lr = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int copy = lr / COLS;  // (NB = 1: 0)
  const int G = hq / hkv;
  int id = blockIdx.x;
  const int h = id % hkv;
  id /= hkv;
  const int b = id % s.n_req;
  id /= s.n_req;
  const int chunk = id % plan.chunks, tile = id / plan.chunks;
  int r0, r1, len, chunk_keys;
  const int32_t *table = paged_request(s, plan, G, b, r0, r1, len, chunk_keys);
  const int n_pairs = (r1 - r0) * G, v0 = tile * COLS;
  if (v0 >= n_pairs) return;
  auto seen_by = [&](int r) { return max(len - r1 + r + 1, 0); };
  const int last = min(n_pairs, v0 + COLS) - 1;
  const int k0 = chunk * chunk_keys;
  const int k1 = min(k0 + chunk_keys, seen_by(r0 + last / G));
  const int all_see = min(seen_by(r0 + v0 / G), k1);
  const bool split = plan.chunks > 1;
  auto place = [&](int v, int &r, int &head) {
    r = r0 + v / G;
    head = h * G + v % G;
  };
  if (k1 <= k0) {
    const int i = tid / (HD / 8);  // a pair's dims in pieces of 8
    for (int v = v0 + i; v <= last; v += 256 / (HD / 8)) {
      int r, head;
      place(v, r, head);
      const size_t row = (size_t)r * hq + head;
      const int e = tid % (HD / 8);
      if (split) {
        if (e == 0)
          part_ml[(size_t)chunk * s.n_rows * hq + row] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
      } else {
        *reinterpret_cast<u32x4_t *>(out + row * HD + e * 8) = (u32x4_t){0, 0, 0, 0};
        if (lse && e == 0) lse[row] = -INFINITY;
      }
    }
    return;
  }

  // queries, and their sums over a group's elements
  bf16x8_t qf[NB][NG][2];
  float qs[NG];
  int seen;
  const int v = v0 + lr % COLS;
  int r, head;
  place(min(v, last), r, head);
  seen = v <= last ? min(seen_by(r), k1) : 0;
  const bf16_t *q = Q + ((size_t)r * hq + head) * HD + g * 16;
#pragma unroll
  for (int gr = 0; gr < NG; ++gr) {
    float sum = 0.f;
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      const u32x4_t x = *reinterpret_cast<const u32x4_t *>(q + gr * 64 + st * 8);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        sum += __uint_as_float(x[i] << 16) + __uint_as_float(x[i] & 0xffff0000u);
#pragma unroll
      for (int c = 0; c < NB; ++c)
        qf[c][gr][st] = order8(NB == 1 || copy == c ? x : (u32x4_t){0, 0, 0, 0});
    }
    sum += __shfl_xor(sum, 16, 64);
    qs[gr] = sum + __shfl_xor(sum, 32, 64);
  }
  // o: of p s 2^-e (1024 + c), share: what of it is not p s 2^-e (c - 8), in every element, until
  // settle() takes it off; zs, l_run: of this lane's keys
  f32x4_t o[DB], share[NG];
  float zs[NG], m_run, l_run;
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int gr = 0; gr < NG; ++gr) {
    share[gr] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    zs[gr] = 0.f;
  }
  m_run = -INFINITY;
  l_run = 0.f;
  // which half of a word of two bf16 (of two groups, or of two keys) goes to which half of the
  // reduction's places for two T, and which to none: selectors of v_perm_b32
  auto selector = [&](int st, int half) {
    const uint32_t from = half ? 0x0302u : 0x0100u;
    const int T = copy - 2 * st;  // of this lane's copy (NB = 4); NB = 2: T = copy
    if (NB == 4 && (T < 0 || T > 1)) return 0x0c0c0c0cu;
    return (NB == 4 ? T : copy) ? (from << 16) | 0x0c0cu : 0x0c0c0000u | from;
  };
  uint32_t sel[2][2];
#pragma unroll
  for (int st = 0; st < 2; ++st)
#pragma unroll
    for (int half = 0; half < 2; ++half) sel[st][half] = selector(st, half);

  const CodeBits cb = bf16_bits();
  const F16Bits fb = f16_bits();
  // p s is fp16 times 2^(P_BITS - e), 2^e being at least the largest scale so far: up to 2^15; what is
  // lost below fp16's smallest is 2^-32 of the largest (2^-28 at every other key)
  constexpr float P_BITS = 7.f;
  uint32_t top = 0;  // the largest scale's bits, and e
  int e_run = -40;
  char *mem = s_mem + wave * WAVE_BYTES;
  uint32_t *s_km = reinterpret_cast<uint32_t *>(mem + PG_TILE * VST), *s_vm = s_km + NG * PG_TILE;
  const int mask = (1 << p.shift) - 1, last_page = (k1 - 1) >> p.shift;
  struct Tile {
    i32x2_t k[4][NG];
    u32x4_t v[NV];
    uint32_t km[NG], vm[NG];
  };
  // (read through scalar registers: nothing writes the table meanwhile)
  typedef const __attribute__((address_space(4))) int32_t *entries_t;
  const entries_t entries = (entries_t)(uintptr_t)table;
  constexpr int NI = WIDE ? 1 : 4;  // pages of a tile at most
  struct Ids {
    int page[NI];
  };
  // the pages of the tile's 16 keys each, clamped into the sequence
  auto pages_at = [&](int key0) __attribute__((always_inline)) {
    Ids x;
#pragma unroll
    for (int T = 0; T < NI; ++T) x.page[T] = entries[min((key0 + 16 * T) >> p.shift, last_page)];
    return x;
  };
  auto load = [&](Tile &t, int key0, const Ids &ids) __attribute__((always_inline)) {
    size_t row[NI];  // of the pool's rows of all heads, where 16 keys begin (uniform)
    bool there[NI];
#pragma unroll
    for (int T = 0; T < NI; ++T) {
      there[T] = ids.page[T] >= 0 && ids.page[T] < p.n_pages;
      row[T] = (((size_t)(there[T] ? ids.page[T] : 0) * hkv + h) << p.shift) +
               ((key0 + 16 * T) & mask);
    }
#pragma unroll
    for (int T = 0; T < 4; ++T) {
      const uint8_t *k = WIDE ? p.k + row[0] * RB + T * 16 * RB : p.k + row[T * (NI - 1) / 3] * RB;
#pragma unroll
      for (int gr = 0; gr < NG; ++gr)
        t.k[T][gr] = *reinterpret_cast<const i32x2_t *>(k + lr * RB + g * 8 + gr * 32);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {  // (HD 64: the rows of two T in a load)
      if constexpr (WIDE) {
        t.v[j] = *reinterpret_cast<const u32x4_t *>(p.v + row[0] * RB + j * 1024 + lane * 16);
      } else if constexpr (VROWS == 16) {
        t.v[j] = *reinterpret_cast<const u32x4_t *>(p.v + row[j] * RB + lane * 16);
      } else {
        const uint8_t *v = p.v + (lane < 32 ? row[2 * j] : row[2 * j + 1]) * RB;
        t.v[j] = *reinterpret_cast<const u32x4_t *>(v + (lane & 31) * 16);
      }
    }
    // meta of key `lane`
    const uint32_t *km = p.k_meta, *vm = p.v_meta;
    bool live = key0 + lane < k1;
    if constexpr (WIDE) {
      km += row[0] * NG + lane * NG;
      vm += row[0] * NG + lane * NG;
      live = live && there[0];
    } else {
      const size_t a = g & 1 ? row[1] : row[0], c = g & 1 ? row[3] : row[2];
      const bool ta = g & 1 ? there[1] : there[0], tc = g & 1 ? there[3] : there[2];
      const size_t mine = ((g & 2 ? c : a) + lr) * NG;
      km += mine;
      vm += mine;
      live = live && (g & 2 ? tc : ta);
    }
#pragma unroll
    for (int gr = 0; gr < NG; ++gr) {
      const uint32_t a = km[gr], c = vm[gr];
      t.km[gr] = live ? a : 0u;
      t.vm[gr] = live ? c : 0u;
    }
  };
  // Values and meta to this wave's LDS (its reads of the tile before are done: in order). Row 16 g +
  // 4 T + i of the values is key 16 T + 4 g + i.
  auto stash = [&](const Tile &t) __attribute__((always_inline)) {
    uint32_t big = scale_bits(t.vm[0]);  // (infinities and NaN count as nothing)
    if constexpr (NG == 2) big = max(big, scale_bits(t.vm[1]));
    if (__ballot(big > top)) {
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) big = max(big, (uint32_t)__shfl_xor((int)big, d, 64));
      top = big;
      const int e = max((int)(big >> 10) - 14, -14);  // scale < 2^e
      const float down = ldexpf(1.f, e_run - max(e, e_run));
      e_run = max(e, e_run);
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= down;
#pragma unroll
      for (int gr = 0; gr < NG; ++gr) share[gr] *= down;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int key = j * VROWS + lane / VC;
      const int at = 16 * ((key >> 2) & 3) + 4 * (key >> 4) + (key & 3);
      *reinterpret_cast<u32x4_t *>(mem + at * VST + lane % VC * 16) = t.v[j];
    }
#pragma unroll
    for (int gr = 0; gr < NG; ++gr) {
      s_km[gr * PG_TILE + lane] = t.km[gr];
      s_vm[gr * PG_TILE + lane] = t.vm[gr];
    }
    __builtin_amdgcn_wave_barrier();
  };
  auto attend = [&](const Tile &t, int key0) __attribute__((always_inline)) {
    float sc[NS];
#pragma unroll
    for (int u = 0; u < 4 / NB; ++u) {
      f32x4_t c[NG];
#pragma unroll
      for (int gr = 0; gr < NG; ++gr) {
        const float off = -16.f * qs[gr];
        c[gr] = (f32x4_t){off, off, off, off};
      }
#pragma unroll
      for (int cp = 0; cp < NB; ++cp)
#pragma unroll
        for (int gr = 0; gr < NG; ++gr)
#pragma unroll
          for (int st = 0; st < 2; ++st) {
            const bf16x8_t kf = codes8((uint32_t)t.k[u * NB + cp][gr][st], cb);
            c[gr] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[cp][gr][st], c[gr], 0, 0, 0);
          }
#pragma unroll
      for (int gr = 0; gr < NG; ++gr) {
        const u32x4_t m = *reinterpret_cast<const u32x4_t *>(s_km + gr * PG_TILE +
                                                             16 * (u * NB + copy) + 4 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float &x = sc[4 * u + i];
          x = fmaf(zero_of(m[i]), qs[gr], gr == 0 ? 0.f : x);
          x = fmaf(scale_of(m[i]), c[gr][i], x);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    const bool masked = key0 + PG_TILE > all_see;
    f16x8_t pf[NG][2];
    const int lim = seen - (key0 + 16 * copy + 4 * g);  // score 4 u + i: key 16 NB u + i of it
    if (masked) {
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if ((i >> 2) * 16 * NB + (i & 3) >= lim) sc[i] = -INFINITY;
    }
    float mx = sc[0];
#pragma unroll
    for (int i = 1; i < NS; ++i) mx = fmaxf(mx, sc[i]);
    // the running maximum rises only when some score exceeds it by more than 2^8
    if (__ballot(mx * scale_log2 > m_run + 8.f)) {
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * scale_log2;
      const float m_new = fmaxf(m_run, mx);
      const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= alpha;
#pragma unroll
      for (int gr = 0; gr < NG; ++gr) {
        share[gr] *= alpha;
        zs[gr] *= alpha;
      }
      l_run *= alpha;
      m_run = m_new;
    }
    const float m_off =
        (m_run == -INFINITY ? 0.f : m_run) - P_BITS;  // (no key yet: every p is 0)
    float pv[NS], ps[NG][NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      pv[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], scale_log2, -m_off));
      l_run += pv[i];
    }
    // (odd places of the reduction have 16 times the code)
    const float down[2] = {ldexpf(1.f, -e_run), ldexpf(1.f, -e_run - 4)};
#pragma unroll
    for (int gr = 0; gr < NG; ++gr) {
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int u = 0; u < NS / 4; ++u) {
        u32x4_t m = *reinterpret_cast<const u32x4_t *>(s_vm + gr * PG_TILE + 16 * (u * NB + copy) +
                                                       4 * g);
        if (masked) {  // a hidden key's scale and zero may be anything: 0 times them is not taken
#pragma unroll
          for (int j = 0; j < 4; ++j) m[j] = 16 * NB * u + j < lim ? m[j] : 0u;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p_ = pv[4 * u + j];
          // (one mixed instruction each)
          ps[gr][4 * u + j] = fmaf(p_ * down[j & 1], scale_of(m[j]), 0.f);
          zs[gr] = fmaf(p_, zero_of(m[j]), zs[gr]);
          sum[j & 1] += ps[gr][4 * u + j];
        }
      }
      // 8 sum p s
      zs[gr] = fmaf(ldexpf(8.f, e_run), fmaf(16.f, sum[1], sum[0]), zs[gr]);
    }
    // a step's places: (key i of T = 2 st, key i of 2 st + 1), i = 0..3
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      u32x4_t x[NG];
      if constexpr (NB == 1) {
#pragma unroll
        for (int gr = 0; gr < NG; ++gr)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            x[gr][i] = pack_half2(ps[gr][8 * st + i], ps[gr][8 * st + 4 + i]);
      } else {
        const int u = NB == 4 ? 0 : st;
        if constexpr (NG == 2) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t w = pack_half2(ps[0][4 * u + i], ps[1][4 * u + i]);
            x[0][i] = __builtin_amdgcn_perm(0u, w, sel[st][0]);
            x[1][i] = __builtin_amdgcn_perm(0u, w, sel[st][1]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            const uint32_t w = pack_half2(ps[0][4 * u + i], ps[0][4 * u + i + 1]);
            x[0][i] = __builtin_amdgcn_perm(0u, w, sel[st][0]);
            x[0][i + 1] = __builtin_amdgcn_perm(0u, w, sel[st][1]);
          }
        }
      }
#pragma unroll
      for (int gr = 0; gr < NG; ++gr) pf[gr][st] = __builtin_bit_cast(f16x8_t, x[gr]);
    }
    __builtin_amdgcn_sched_barrier(0);
    // 1024 + 8 and, of a 16th, 1024 + 128
    const f16x8_t rest = __builtin_bit_cast(
        f16x8_t, (u32x4_t){0x64086408u, 0x64806480u, 0x64086408u, 0x64806480u});
#pragma unroll
    for (int gr = 0; gr < NG; ++gr)
#pragma unroll
      for (int st = 0; st < 2; ++st)
        share[gr] =
            __builtin_amdgcn_mfma_f32_16x16x32_f16(rest, pf[gr][st], share[gr], 0, 0, 0);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const i32x2_t w = __builtin_amdgcn_ds_read_tr4_b64_v2i32(
          (__attribute__((address_space(3))) i32x2_t *)(mem + lane * VST + db * 8));
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const f16x8_t vf = raw8((uint32_t)w[st], fb);
        o[db] =
            __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[db / 4][st], o[db], 0, 0, 0);
      }
      if (db & 1) __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_wave_barrier();
  };
  // The constants' part of o is a hundred times what is wanted, and rounds as such: left in to the
  // end, 65536 keys of even weights in a block came out wrong by 0.7 to 2.4 % (root mean square),
  // taken off every two tiles by 0.17 %, as the rounding to bf16 alone. It costs 1 % where
  // instructions bound (16 requests of 5 or 6 rows over 3000 to 9000 keys 61.1 us to 61.9).
  auto settle = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] -= share[db / 4];
#pragma unroll
    for (int gr = 0; gr < NG; ++gr) share[gr] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
  };
  constexpr int STEP = 4 * PG_TILE;
  int key0 = k0 + wave * PG_TILE;
  if (key0 < k1) {
    Tile t0, t1;
    load(t0, key0, pages_at(key0));
    Ids ids = pages_at(key0 + STEP);
    while (true) {  // (past the end: the last page again)
      stash(t0);
      load(t1, key0 + STEP, ids);
      ids = pages_at(key0 + 2 * STEP);
      __builtin_amdgcn_sched_barrier(0);
      attend(t0, key0);
      key0 += STEP;
      if (key0 >= k1) break;
      stash(t1);
      load(t0, key0 + STEP, ids);
      ids = pages_at(key0 + 2 * STEP);
      __builtin_amdgcn_sched_barrier(0);
      attend(t1, key0);
      settle();
      key0 += STEP;
      if (key0 >= k1) break;
    }
  }
  // the waves' and copies' parts through LDS: rows of a column's outputs
  __syncthreads();
  float *mine = reinterpret_cast<float *>(mem);
  float l = l_run;
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
#pragma unroll
  for (int gr = 0; gr < NG; ++gr) {
    float z = zs[gr];
    z += __shfl_xor(z, 16, 64);
    z += __shfl_xor(z, 32, 64);
    const float up = ldexpf(1.f, e_run), sh = share[gr][0];
#pragma unroll
    for (int db = 4 * gr; db < 4 * gr + 4; ++db) {
      f32x4_t x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = fmaf(o[db][i] - sh, up, z);
      *reinterpret_cast<f32x4_t *>(mine + lr * OST + db * 16 + 4 * g) = x;
    }
  }
  if (g == 0) {
    s_m[wave][lr] = m_run - P_BITS;
    s_l[wave][lr] = l;
  }
  __syncthreads();
  constexpr int PER = HD / 8;  // lanes of a pair
  const int e0 = tid % PER * 8;
  for (int i = tid / PER; v0 + i <= last; i += 256 / PER) {
    float mm = -INFINITY, l = 0.f, a[8];
#pragma unroll
    for (int w = 0; w < 4 * NB; ++w) mm = fmaxf(mm, s_m[w / NB][i + w % NB * COLS]);
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = 0.f;
#pragma unroll
    for (int w = 0; w < 4 * NB; ++w) {
      // a part without a key of the pair has l = 0 (m = -inf is also what NaN scores leave, with
      // a sum of NaN)
      const int c = i + w % NB * COLS;
      const float lw = s_l[w / NB][c];
      if (lw == 0.f) continue;
      const float f = mm == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(s_m[w / NB][c] - mm);
      l = fmaf(f, lw, l);
      const float *x = reinterpret_cast<const float *>(s_mem + w / NB * WAVE_BYTES) + c * OST + e0;
      float xv[8];
      load8(x, xv);
#pragma unroll
      for (int j = 0; j < 8; ++j) a[j] = fmaf(f, xv[j], a[j]);
    }
    int r, head;
    place(v0 + i, r, head);
    const size_t row = (size_t)r * hq + head;
    if (split) {
      const size_t prow = (size_t)chunk * s.n_rows * hq + row;
      store8(part_o + prow * HD + e0, a);
      if (e0 == 0) part_ml[prow] = make_float4(mm, l, 1.f, 0.f);
    } else {
      const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
      for (int j = 0; j < 8; ++j) a[j] *= inv;
      store8(out + row * HD + e0, a);
      if (lse && e0 == 0)
        lse[row] =
            l == 0.f ? -INFINITY : (mm == -INFINITY ? 0.f : mm * 0.6931471805599453f) + logf(l);
    }
  }
}

// Many pairs. Block = 4 waves over 32 * groups pairs (groups 1, 2 or 4) and one chunk of keys. Tiles
// of 64 keys are put into LDS as fp16, from codes loaded two tiles ahead: the keys' codes, exactly,
// whose scales and zeros the scores get after the products; the values themselves, rounded once (those
// that may lie outside fp16's range apart); a wave takes 32 pairs and 32 or 64 of the
// tile's keys: with 4 groups each wave has a group, with 2 two waves share a group's keys, with
// 1 two of the waves only load. Scores are formed transposed, S^T = K Q^T (MFMA 32x32x16): lane l
// holds 16 scores of pair l % 32, the operand layout of O^T = V^T P^T; V^T comes from row-major
// rows by the transposing LDS read. Queries are fp16 scaled by a power of two per pair, the
// probabilities fp16 times 2^7, so that what is lost below fp16's smallest is 2^-32 of the
// largest; statistics and outputs are fp32.
//   6 questions of 39 to 92 rows over 3155 to 8115 keys, 40/8 heads: 97 us, 345 TFLOP/s. The matrix
//   cores are busy 0.16 of that, the vector unit 0.32, LDS 0.21, at 1.1 waves a SIMD of the 2 that fit:
//   they wait for each other's steps, and the longest question's blocks for nobody.
template <int HD, bool WIDE>
__global__ __launch_bounds__(256, 2) void k_paged_many(PagedBatch s, PagePool p, PagedPlan plan,
                                                       const bf16_t *__restrict__ Q, int hq,
                                                       int hkv, float scale_log2,
                                                       bf16_t *__restrict__ out,
                                                       float *__restrict__ lse,
                                                       float *__restrict__ part_o,
                                                       float4 *__restrict__ part_ml) {
  constexpr int KS = HD / 16, DB = HD / 32, NG = HD / 64, RB = HD / 2;
  constexpr int WORDS = HD / 32;                   // of codes per thread: 4 threads a row
  constexpr int KST = HD + 8, VST = HD + 32;       // row strides: fragment reads on all banks
  constexpr int KB = PG_TILE * KST, VB = PG_TILE * VST;
  constexpr float P_BITS = 7.f;
  __shared__ __attribute__((aligned(16))) _Float16 s_kv[2 * (KB + VB)];
  __shared__ __attribute__((aligned(16))) uint32_t s_km[2][NG][PG_TILE];
  __shared__ int s_odd;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, hi = lane >> 5;
  const int G = hq / hkv;
  int id = blockIdx.x;
  const int h = id % hkv;
  id /= hkv;
  const int b = id % s.n_req;
  id /= s.n_req;
  const int chunk = id % plan.chunks, tile = id / plan.chunks;
  int r0, r1, len, chunk_keys;
  const int32_t *table = paged_request(s, plan, G, b, r0, r1, len, chunk_keys);
  const int n_pairs = (r1 - r0) * G, v0 = tile * plan.pairs;
  if (v0 >= n_pairs) return;
  auto seen_by = [&](int r) { return max(len - r1 + r + 1, 0); };
  const int last = min(n_pairs, v0 + plan.pairs) - 1;
  // this wave's pairs and its share of a tile's two 32-key halves
  const int groups = last - v0 >= 64 ? 4 : last - v0 >= 32 ? 2 : 1;
  const int group = groups == 4 ? wave : groups == 2 ? wave >> 1 : 0;
  const bool works = groups > 1 || wave < 2;
  const int st0 = groups == 4 ? 0 : wave & 1, st_step = groups == 4 ? 1 : 2;
  const int v = v0 + group * 32 + (lane & 31);
  const bool valid = v <= last;
  const int r = r0 + (valid ? v : v0) / G, head = h * G + (valid ? v : v0) % G;
  const int k0 = chunk * chunk_keys;
  const int k1 = min(k0 + chunk_keys, seen_by(r0 + last / G));
  const int all_see = seen_by(r0 + v0 / G), seen = valid ? min(seen_by(r), k1) : 0;
  const size_t prow = ((size_t)chunk * s.n_rows + r) * hq + head;
  const int nkt = k1 > k0 ? (k1 - k0 + PG_TILE - 1) / PG_TILE : 0;
  const bool writes = valid && (groups == 4 || (works && (wave & 1) == 0));
  if (nkt == 0 && plan.chunks > 1) {
    if (writes && hi == 0) part_ml[prow] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    return;
  }

  // A thread has a quarter of a row's codes, keys and values.
  const int krow = tid >> 2, kq = tid & 3;
  const F16Bits fb = f16_bits();
  typedef __attribute__((ext_vector_type(WORDS))) uint32_t words_t;
  struct Codes {
    words_t k, v;
    uint32_t km, vm;
  };
  const int last_page = (max(k1, 1) - 1) >> p.shift, mask = (1 << p.shift) - 1;
  // (WIDE: the tile lies in one page, whose number is read through scalar registers: nothing writes
  // the table meanwhile)
  typedef const __attribute__((address_space(4))) int32_t *entries_t;
  const entries_t entries = (entries_t)(uintptr_t)table;
  auto page_at = [&](int key0) {
    if constexpr (WIDE) return entries[min(key0 >> p.shift, last_page)];
    else return table[min((key0 + krow) >> p.shift, last_page)];
  };
  auto load = [&](Codes &c, int key0, int page) __attribute__((always_inline)) {
    const bool there = page >= 0 && page < p.n_pages, live = there && key0 + krow < k1;
    // rows of the pool's heads: where the tile begins (or this thread's row), and from there
    const size_t base = (((size_t)(there ? page : 0) * hkv + h) << p.shift) +
                        ((key0 + (WIDE ? 0 : krow)) & mask);
    const int row = WIDE ? krow : 0;
    c.k = *reinterpret_cast<const words_t *>(p.k + base * RB + row * RB + kq * (RB / 4));
    c.v = *reinterpret_cast<const words_t *>(p.v + base * RB + row * RB + kq * (RB / 4));
    const uint32_t km = (p.k_meta + base * NG)[row * NG + kq * NG / 4];
    const uint32_t vm = (p.v_meta + base * NG)[row * NG + kq * NG / 4];
    c.km = live ? km : 0u;
    c.vm = live ? vm : 0u;
  };
  Codes c;
  int page = 0;
  if (nkt) {
    load(c, k0, page_at(k0));
    page = page_at(k0 + PG_TILE);
  }

  // the pair's query, its largest element brought to [2^7, 2^8)
  f16x8_t qf[KS], qz;  // qz: the sum over group hi's elements in three fp16 parts, for its zeros
  float q_scale = scale_log2;
  {
    const bf16_t *q = Q + ((size_t)r * hq + head) * HD + hi * 8;
    float x[KS][8], big = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      load8(q + ks * 16, x[ks]);
#pragma unroll
      for (int i = 0; i < 8; ++i) big = fmaxf(big, fabsf(x[ks][i]));
    }
    big = fmaxf(big, __shfl_xor(big, 32, 64));
    int e = 0;
    if (big > 0.f && big < INFINITY) e = max(__builtin_amdgcn_frexp_expf(big), -100) - 8;
    const float down = ldexpf(1.f, -e);
    q_scale *= ldexpf(1.f, e);
    float sums[2] = {0.f, 0.f};
#pragma unroll
    for (int gr = 0; gr < NG; ++gr) {
#pragma unroll
      for (int ks = 4 * gr; ks < 4 * gr + 4; ++ks)
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[gr] += x[ks][i] * down;
      sums[gr] += __shfl_xor(sums[gr], 32, 64);
    }
    float rest = hi ? sums[1] : sums[0];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      qz[i] = i < 3 ? (_Float16)rest : (_Float16)0.f;
      rest -= (float)qz[i];
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)  // (in the order of exact8, as the keys are)
#pragma unroll
      for (int i = 0; i < 8; ++i) qf[ks][i] = (_Float16)(x[ks][(i & 1) * 4 + i / 2] * down);
  }
  f32x16_t o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;  // (l_run: of this lane's half of the keys)

  // Dims are in LDS in the order of values8, 0 4 1 5 2 6 3 7 of every 8, until the end.
  // Values that some pair of the tile must not see take part with probability 0, and 0 * inf is
  // NaN; and scale and zero may make a value past fp16's range, which only 32 bits hold. Where a
  // group's scale or zero lets that be, 0 goes to LDS, and the pairs that see it get it added at the
  // end. Pieces of the values are written in an order that differs by row, so that rows four apart
  // in a bank do not meet.
  auto store = [&](Codes &c, int key0, int buf) __attribute__((always_inline)) {
    _Float16 *ks = s_kv + buf * (KB + VB) + krow * KST + kq * (HD / 4);
    _Float16 *vs = s_kv + buf * (KB + VB) + KB + krow * VST + kq * (HD / 4);
    if (wide_values(c.vm)) {
      s_odd = 1;
      c.vm = 0;
    }
#pragma unroll
    for (int j = 0; j < WORDS; ++j)
      *reinterpret_cast<f16x8_t *>(ks + j * 8) = exact8(c.k[j], fb);
    if ((kq & (4 / NG - 1)) == 0) s_km[buf][kq * NG / 4][krow] = c.km;
    const f16x2_t m = __builtin_bit_cast(f16x2_t, c.vm), sc = {m[0], m[0]}, z = {m[1], m[1]};
    words_t w = c.v;
    const int turn = krow & (WORDS - 1);
#pragma unroll
    for (int bit = 1; bit < WORDS; bit <<= 1) {
      words_t u;
#pragma unroll
      for (int j = 0; j < WORDS; ++j) u[j] = turn & bit ? w[(j + bit) & (WORDS - 1)] : w[j];
      w = u;
    }
#pragma unroll
    for (int j = 0; j < WORDS; ++j)
      *reinterpret_cast<f16x8_t *>(vs + ((j + turn) & (WORDS - 1)) * 8) = values8(w[j], sc, z, fb);
  };
  if (tid == 0) s_odd = 0;
  __syncthreads();
  if (nkt) {
    store(c, k0, 0);
    load(c, k0 + PG_TILE, page);  // (past the end: its last page again)
    page = page_at(k0 + 2 * PG_TILE);
  }
  __syncthreads();
  for (int kt = 0; kt < nkt; ++kt) {
    const int key0 = k0 + kt * PG_TILE;
    const _Float16 *ks_ = s_kv + (kt & 1) * (KB + VB), *vs_ = ks_ + KB;
    __builtin_amdgcn_s_setprio(1);
    for (int st = works ? st0 : 2; st < 2; st += st_step) {
      const int sk0 = key0 + st * 32;
      if (sk0 >= k1) break;
      // S^T block: score i is key sk0 + (i / 4) * 8 + hi * 4 + i % 4 of this lane's pair
      f32x16_t acc[NG], sc;
      {  // zeros times the query's sums
        const uint32_t m = s_km[kt & 1][hi & (NG - 1)][st * 32 + (lane & 31)];
        const uint32_t z = (m >> 16) | (m & 0xffff0000u);
        f16x8_t zf = __builtin_bit_cast(f16x8_t, (u32x4_t){z, z & 0xffffu, 0u, 0u});
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.f;
        sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(zf, qz, sc, 0, 0, 0);
      }
      const _Float16 *kr = ks_ + (st * 32 + (lane & 31)) * KST + hi * 8;
#pragma unroll
      for (int gr = 0; gr < NG; ++gr) {
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[gr][i] = 0.f;
#pragma unroll
        for (int ks = 4 * gr; ks < 4 * gr + 4; ++ks)
          acc[gr] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
              *reinterpret_cast<const f16x8_t *>(kr + ks * 16), qf[ks], acc[gr], 0, 0, 0);
      }
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4)
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
          const u32x4_t m = *reinterpret_cast<const u32x4_t *>(
              &s_km[kt & 1][gr][st * 32 + i4 * 8 + hi * 4]);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            sc[4 * i4 + j] = fmaf(scale_of(m[j]), acc[gr][4 * i4 + j], sc[4 * i4 + j]);
        }
      // V^T operand of step t, dims db * 32 + lane % 32: its 8 slots are keys 16 t + 4 hi + 0..3
      // and the same + 8 of the block
      f16x8_t vf[2][DB];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          typedef short v4s __attribute__((ext_vector_type(4)));
          const _Float16 *vb = vs_ + (st * 32 + 16 * t + 4 * hi + ((lane & 15) >> 2)) * VST +
                               db * 32 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
          const v4s x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) v4s *)(vb));
          const v4s x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) v4s *)(vb + 8 * VST));
          __builtin_memcpy(&vf[t][db], &x0, 8);
          __builtin_memcpy(reinterpret_cast<char *>(&vf[t][db]) + 8, &x1, 8);
        }
      if (sk0 + 32 > min(all_see, k1)) {
        const int lim = seen - (sk0 + hi * 4);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if ((i >> 2) * 8 + (i & 3) >= lim) sc[i] = -INFINITY;
      }
      float mx = sc[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
      // the running maximum rises only when some score exceeds it by more than 2^8
      if (__ballot(mx * q_scale > m_run + 8.f)) {
        const float mp = fmaxf(mx, __shfl_xor(mx, 32, 64)) * q_scale;
        const float m_new = fmaxf(m_run, mp);
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] *= alpha;
        l_run *= alpha;
        m_run = m_new;
      }
      const float m_off = (m_run == -INFINITY ? 0.f : m_run) - P_BITS;  // (no key yet: every p is 0)
      float pv[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        pv[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], q_scale, -m_off));
        l_run += pv[i];
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f16x8_t pb;
#pragma unroll
        for (int j = 0; j < 8; ++j) pb[j] = (_Float16)pv[8 * t + j];
#pragma unroll
        for (int db = 0; db < DB; ++db)
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[t][db], pb, o[db], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    if (kt + 1 < nkt) {
      store(c, key0 + PG_TILE, (kt + 1) & 1);
      load(c, key0 + 2 * PG_TILE, page);
      page = page_at(key0 + 3 * PG_TILE);
    }
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
    const float fa = __builtin_amdgcn_exp2f(m_run - off), fb = __builtin_amdgcn_exp2f(m2 - off);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = fa * o[db][i] + fb * x[(db * 16 + i) * 64];
    l = fa * l + fb * l2;
    m_run = mm;
  }
  // o[db][i] becomes dim db * 32 + (i / 4) * 8 + hi * 4 + i % 4 of the pair (all lanes take part)
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      uint32_t x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = __float_as_uint(o[db][4 * q4 + j]);
      swap_halves(x[0], x[1]);
      swap_halves(x[2], x[3]);
      o[db][4 * q4] = __uint_as_float(x[0]);
      o[db][4 * q4 + 1] = __uint_as_float(x[2]);
      o[db][4 * q4 + 2] = __uint_as_float(x[1]);
      o[db][4 * q4 + 3] = __uint_as_float(x[3]);
    }
  if (!valid) return;
  if (s_odd) {  // values left out above that this pair sees: finite ones by their probability
    for (int k = k0; k < seen; ++k) {
      const int pg = table[k >> p.shift];
      if (pg < 0 || pg >= p.n_pages) continue;
      const size_t row = (((size_t)pg * hkv + h) << p.shift) + (k & mask);
      bool any = false;
      for (int gr = 0; gr < NG; ++gr) any |= wide_values(p.v_meta[row * NG + gr]);
      if (!any) continue;
      float s = 0.f;
      for (int gr = 0; gr < NG; ++gr) {
        const bf16_t *q = Q + ((size_t)r * hq + head) * HD + gr * 64;
        const uint8_t *kc = p.k + row * RB + gr * 32;
        float qc = 0.f, q1 = 0.f;
        for (int e = 0; e < 64; e += 8) {
          float x[8];
          load8(q + e, x);
          const uint32_t w = *reinterpret_cast<const uint32_t *>(kc + e / 2);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            qc = fmaf(x[j], (float)((w >> (4 * j)) & 15u), qc);
            q1 += x[j];
          }
        }
        const uint32_t mt = p.k_meta[row * NG + gr];
        s += fmaf(scale_of(mt), qc, zero_of(mt) * q1);
      }
      const float pk = __builtin_amdgcn_exp2f(
          fmaf(s, scale_log2, P_BITS - (m_run == -INFINITY ? 0.f : m_run)));
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const uint32_t mt = p.v_meta[row * NG + db / 2];
        if (!wide_values(mt)) continue;
        const float sv = scale_of(mt), zv = zero_of(mt);
        const float f = fabsf(sv) < INFINITY && fabsf(zv) < INFINITY ? pk : 1.f;
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const uint32_t w =
              *reinterpret_cast<const uint16_t *>(p.v + row * RB + db * 16 + q4 * 4 + hi * 2);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            o[db][4 * q4 + j] =
                fmaf(f, fmaf(sv, (float)((w >> (4 * j)) & 15u), zv), o[db][4 * q4 + j]);
        }
      }
    }
  }
  if (plan.chunks > 1) {
    float *po = part_o + prow * HD + hi * 4;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<float4 *>(po + db * 32 + q4 * 8) = make_float4(
            o[db][4 * q4], o[db][4 * q4 + 1], o[db][4 * q4 + 2], o[db][4 * q4 + 3]);
    if (hi == 0) part_ml[prow] = make_float4(m_run - P_BITS, l, 1.f, 0.f);
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
        l == 0.f ? -INFINITY
                 : ((m_run == -INFINITY ? 0.f : m_run) - P_BITS) * 0.6931471805599453f + logf(l);
}

// Pairs of a request and KV head: up to 48 are k_paged_few's, in tiles of up to 16 of which each reads
// the codes (the second from the caches), more k_paged_many's.
//   16 requests of 3000 to 9000 keys, 40/8 heads: 30 pairs 62 us in two tiles, 73 in one of 32 (256
//   registers, one block a unit), 81 by k_paged_many; 40 pairs 69 in three and 82; 60 pairs 92 in four
//   and 83.
// Up to 8 pairs are there twice, up to 4 of heads of 64 four times (at 128 the queries' copies leave
// no registers: 32 requests with 3 pairs each 54 us twice, 73 four times; heads of 64, 2 pairs, 57
// and 53).
// The keys are cut into the number of chunks whose estimated end is the earliest, taking every
// sequence to be as long as the longest: a block takes FIXED and WALK per tile that it walks (its
// waves walk a quarter each in k_paged_few), ALONE of that where it has its unit for itself; whole
// rounds of blocks, and what is left of them, follow each other.
//   32 requests of 4700 to 16000 keys of 40/8 heads: chunks of 8192 keys (one round) 92 us, of 4096
//   102, of 16384 99; 3 of 91000 to 122000 of 28/4: 2816 (one round) 40, 2560 (a little more) 50,
//   1536 45, 6144 46; 16 of 3000 to 19000 with 16 pairs of heads of 64: 3200 (3 blocks a unit) 38,
//   2432 (4) 32.
static PagedPlan paged_plan(const PagedBatch &s, int hq, int hkv, int hd) {
  PagedPlan p;
  const int G = hq / hkv;
  const long long pairs = (long long)s.rows_max * G;
  p.pairs = pairs <= 4 && hd == 64 ? 4 : pairs <= 8 ? 8 : pairs <= 48 ? 16 : pairs <= 64 ? 64 : 128;
  p.many = pairs > 48;
  p.tiles = (int)((pairs + p.pairs - 1) / p.pairs);
  // (MOVED: bytes of the partials in a us, most of them to and from the caches)
  const double FIXED = 7, WALK = p.many ? 3.3 : 2.55, ALONE = 0.6, MOVED = 1e7;
  const int kt = (s.limit + PG_TILE - 1) / PG_TILE, unit = p.many ? 1 : 4;
  // (k_paged_few, heads of 64: 3 blocks fit a unit, and some are empty)
  const long long slots = gemm_cu_count() * (hd == 128 ? 2LL : p.many ? 3LL : 4LL);
  // (tiles of a request that has fewer rows than another are empty)
  const double items =
      hkv * std::min((double)s.n_req * p.tiles, (double)s.n_rows * G / p.pairs + 0.5 * s.n_req);
  const double moved = (double)s.n_rows * hq * (8 * hd + 32) / MOVED;  // a chunk's partials
  auto end = [&](long long n) {
    const double walk = WALK * (double)(((kt + n - 1) / n + unit - 1) / unit);
    const double count = items * n, rounds = std::floor(count / slots), rest = count - rounds * slots;
    double t = rounds * (FIXED + walk);
    if (rest > 0) t += FIXED + walk * (rest <= slots / 2 ? ALONE : 1.0);
    return t + (n > 1 ? 4 + moved * n : 0);
  };
  const long long most = std::max(1, std::min(MERGE_SLOTS, (kt + 3) / 4));
  long long best = 1;
  auto consider = [&](double want) {
    const long long n = std::max(1LL, std::min((long long)want, most));
    if (end(n) < end(best)) best = n;
  };
  for (double rounds : {0.5, 1.0, 2.0, 3.0, 4.0}) consider(rounds * slots / std::max(1.0, items));
  const int per = kt ? (int)((kt + best - 1) / best) : 1;
  p.chunk_keys = (per + unit - 1) / unit * unit * PG_TILE;
  p.chunks = std::max(1, (s.limit + p.chunk_keys - 1) / p.chunk_keys);
  // the cut is made anew of the lengths, by k_paged_many in up to half as many chunks more
  p.slots = s.n_req <= 64 && (p.many ? p.chunks > 1 : p.chunks >= 8) ? (int)(slots / hkv) : 0;
  if (p.slots && p.many) p.chunks = (int)std::min(most, (p.chunks * 3LL + 1) / 2);
  return p;
}

size_t paged_part_floats(const PagedBatch &s, int hq, int hkv, int hd) {
  if (s.n_rows == 0) return 0;
  const PagedPlan p = paged_plan(s, hq, hkv, hd);
  const size_t items = (size_t)p.chunks * s.n_rows * hq;
  return p.chunks > 1 ? items * hd + items * 4 : 0;
}

long long paged_blocks(const PagedBatch &s, int hq, int hkv, int hd) {
  const PagedPlan p = paged_plan(s, hq, hkv, hd);
  return (long long)s.n_req * p.chunks * p.tiles * hkv;
}

hipError_t launch_paged_attention(const PagedBatch &s, const PagePool &p, const void *q, int hq,
                                  int hkv, int hd, void *out, float *lse, float *part,
                                  hipStream_t st) {
  if (s.n_rows == 0) return hipSuccess;
  const PagedPlan plan = paged_plan(s, hq, hkv, hd);
  const dim3 g((unsigned)((size_t)s.n_req * plan.chunks * plan.tiles * hkv)), b(256);
  const float scale = 1.4426950408889634f / sqrtf((float)hd);
  const bf16_t *Q = reinterpret_cast<const bf16_t *>(q);
  bf16_t *O = reinterpret_cast<bf16_t *>(out);
  float4 *ml = reinterpret_cast<float4 *>(part);  // (m, l, f) of every slot, then the outputs
  float *po = reinterpret_cast<float *>(ml + (size_t)plan.chunks * s.n_rows * hq);
#define AKVS_PAGED(...)                                                                          \
  hipLaunchKernelGGL((__VA_ARGS__), g, b, 0, st, s, p, plan, Q, hq, hkv, scale, O, lse, po, ml)
#define AKVS_PAGED_FEW(HD_, NB_)                            \
  if (p.shift >= 6) AKVS_PAGED(k_paged_few<HD_, NB_, true>); \
  else AKVS_PAGED(k_paged_few<HD_, NB_, false>)
#define AKVS_PAGED_HD(HD_)                                 \
  if (plan.many) {                                         \
    if (p.shift >= 6) AKVS_PAGED(k_paged_many<HD_, true>); \
    else AKVS_PAGED(k_paged_many<HD_, false>);             \
  } else if (plan.pairs == 16) {                           \
    AKVS_PAGED_FEW(HD_, 1);                                \
  } else if (plan.pairs == 8) {                            \
    AKVS_PAGED_FEW(HD_, 2);                                \
  }
  if (hd == 128) {
    AKVS_PAGED_HD(128)
  } else {
    AKVS_PAGED_HD(64) else {
      AKVS_PAGED_FEW(64, 4);
    }
  }
#undef AKVS_PAGED_FEW
#undef AKVS_PAGED_HD
#undef AKVS_PAGED
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.chunks <= 1) return e;
  const SharedBatch rows{s.n_req, s.n_rows, s.rows_max, 0, 0, s.row_start, nullptr};
  return launch_merge_slots(rows, plan.chunks, hq, hd, po, ml, out, lse, st);
}

}  // namespace akvs
