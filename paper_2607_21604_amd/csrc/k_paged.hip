// Attention over sequences in pages of 4-bit codes.
//
// The (row, query head) pairs of a request that read one KV head are the columns of a matrix, as in
// the attention over a shared context. Codes go to the matrix cores as they are: a nibble c put
// into the upper mantissa bits of a bf16 of 16 is 16 + c, exactly, in one instruction for two, and
// with (scale s, zero z) of a group of 64 elements outside the products
//   q.k   = sum_groups s (sum q (16 + c) - 16 sum q) + z sum q
//   sum p v = sum p s (16 + c) - 24 sum p s + sum p (z + 8 s)
// (p s rounded to bf16 in the first two sums, which together hold p s (c - 8), about as large as
// the values' deviations; the last one in fp32). Scores hold no rounded operand.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "four_bit_dev.h"
#include "kernels.h"
#include "pages_dev.h"

namespace akvs {

// Work items of a call: (request, chunk of its keys, pair tile, KV head), KV heads innermost.
struct PagedPlan {
  int tiles, chunks, chunk_keys;
};
constexpr int PG_TILE = 64;  // keys a wave takes at a time

// Block = 4 waves over NP tiles of 16 pairs and one chunk of keys; its waves take the chunk's
// tiles of 64 keys in turn, each with its own maximum, sum and output, merged through LDS at the
// end, so that the loop has no barrier. MFMA 16x16x32, lane l: g = l / 16.
//   Scores, S^T = K Q^T: row r of key tile T stands for key 16 (r / 4) + 4 T + r % 4, so that lane
//   l holds the scores of pair l % 16 at keys 16 g .. 16 g + 15; its reduction takes elements
//   64 group + 16 g + 8 step .. + 7.
//   Outputs, O^T = V^T P^T: the lane's keys are its part of the reduction; V^T comes from rows in
//   LDS by the transposing read of 4-bit elements, 16 keys of a dim at once.
// Loads of the next tile, and its pages' numbers a tile earlier, are in flight meanwhile; 16
// consecutive keys lie in one page.
template <int HD, int NP>
__global__ __launch_bounds__(256, 2) void k_paged_few(PagedBatch s, PagePool p, PagedPlan plan,
                                                      const bf16_t *__restrict__ Q, int hq, int hkv,
                                                      float scale_log2, bf16_t *__restrict__ out,
                                                      float *__restrict__ lse,
                                                      _Float16 *__restrict__ part_o,
                                                      float4 *__restrict__ part_ml) {
  constexpr int NG = HD / 64, DB = HD / 16;      // groups of a row, blocks of 16 dims
  constexpr int RB = HD / 2;                     // bytes of a row's codes
  constexpr int VST = RB + 16;                   // row stride in LDS: reads on all banks
  constexpr int NV = PG_TILE * RB / 1024;        // 16-byte chunks of V per lane
  constexpr int VKEYS = 1024 / RB;               // keys of one such load of the wave
  constexpr int MST = 16 * NG * 4 + 16;          // of the meta of 16 keys
  constexpr int OST = HD + 4;
  constexpr int STAGE = PG_TILE * VST + 8 * MST; // of a wave
  constexpr int MERGE = 16 * NP * OST * 4;
  constexpr int WAVE_BYTES = (STAGE > MERGE ? STAGE : MERGE);
  __shared__ __attribute__((aligned(16))) char s_mem[4 * WAVE_BYTES];
  __shared__ float s_m[4][16 * NP], s_l[4][16 * NP];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, lr = lane & 15;
  const int G = hq / hkv;
  int id = blockIdx.x;
  const int h = id % hkv;
  id /= hkv;
  const int tile = id % plan.tiles;
  id /= plan.tiles;
  const int chunk = id % plan.chunks, b = id / plan.chunks;
  int r0, r1, len;
  paged_rows(s, b, r0, r1);
  const int32_t *table = paged_keys(s, b, len);
  const int n_pairs = (r1 - r0) * G, v0 = tile * 16 * NP;
  if (v0 >= n_pairs) return;
  auto seen_by = [&](int r) { return max(len - r1 + r + 1, 0); };
  const int last = min(n_pairs, v0 + 16 * NP) - 1;
  const int k0 = chunk * plan.chunk_keys;
  const int k1 = min(k0 + plan.chunk_keys, seen_by(r0 + last / G));
  const int all_see = seen_by(r0 + v0 / G);
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
  bf16x8_t qf[NP][NG][2];
  float qs[NP][NG];
  int seen[NP];
#pragma unroll
  for (int np = 0; np < NP; ++np) {
    const int v = v0 + np * 16 + lr;
    int r, head;
    place(min(v, last), r, head);
    seen[np] = v <= last ? seen_by(r) : 0;
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
        qf[np][gr][st] = order8(x);
      }
      sum += __shfl_xor(sum, 16, 64);
      qs[np][gr] = sum + __shfl_xor(sum, 32, 64);
    }
  }
  f32x4_t o[NP][DB], ones[NP][NG];  // ones: the sums of the rounded p s, in every element
  float zs[NP][NG], m_run[NP], l_run[NP];  // (zs, l_run: of this lane's keys)
#pragma unroll
  for (int np = 0; np < NP; ++np) {
#pragma unroll
    for (int db = 0; db < DB; ++db) o[np][db] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int gr = 0; gr < NG; ++gr) {
      ones[np][gr] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
      zs[np][gr] = 0.f;
    }
    m_run[np] = -INFINITY;
    l_run[np] = 0.f;
  }

  char *mem = s_mem + wave * WAVE_BYTES;
  char *s_km = mem + PG_TILE * VST, *s_vm = s_km + 4 * MST;
  const int last_page = (k1 - 1) >> p.shift;
  struct Tile {
    i32x2_t k[4][NG];
    u32x4_t v[NV];
    uint32_t km[NG], vm[NG];
  };
  // the page of the 16 keys from key0 + 16 g on, clamped into the sequence
  auto page_at = [&](int key0) { return table[min((key0 + 16 * g) >> p.shift, last_page)]; };
  auto load = [&](Tile &t, int key0, int page) __attribute__((always_inline)) {
    const int mask = (1 << p.shift) - 1;
    const bool there = page >= 0 && page < p.n_pages;
    const int at = there ? page : 0;
    // rows of 16 keys of every group, in rows of the pool's heads
    const size_t mine = (((size_t)at * hkv + h) << p.shift) + ((key0 + 16 * g) & mask);
    {
      const bool live = there && key0 + lane < k1;
      const uint32_t *km = p.k_meta + (mine + lr) * NG, *vm = p.v_meta + (mine + lr) * NG;
#pragma unroll
      for (int gr = 0; gr < NG; ++gr) {
        t.km[gr] = live ? km[gr] : 0u;
        t.vm[gr] = live ? vm[gr] : 0u;
      }
    }
    {
      const int kg = lr >> 2;
      const int kp = __shfl(at, kg * 16, 64);
      const size_t row = (((size_t)kp * hkv + h) << p.shift) + ((key0 + 16 * kg) & mask) + (lr & 3);
      const uint8_t *k = p.k + row * RB + g * 8;
#pragma unroll
      for (int T = 0; T < 4; ++T)
#pragma unroll
        for (int gr = 0; gr < NG; ++gr)
          t.k[T][gr] = *reinterpret_cast<const i32x2_t *>(k + T * 4 * RB + gr * 32);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      // keys j VKEYS .. of the tile, lane's at lane / (RB / 16)
      const int key = j * VKEYS + lane / (RB / 16), vg = key >> 4;
      const int vp = __shfl(at, vg * 16, 64);
      const size_t row = (((size_t)vp * hkv + h) << p.shift) + ((key0 + key) & mask);
      t.v[j] = *reinterpret_cast<const u32x4_t *>(p.v + row * RB + lane % (RB / 16) * 16);
    }
  };
  // values and meta to this wave's LDS (its reads of the tile before are done: in order)
  auto stash = [&](const Tile &t) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      *reinterpret_cast<u32x4_t *>(mem + (j * VKEYS + lane / (RB / 16)) * VST +
                                   lane % (RB / 16) * 16) = t.v[j];
#pragma unroll
    for (int gr = 0; gr < NG; ++gr) {
      *reinterpret_cast<uint32_t *>(s_km + g * MST + (gr * 16 + lr) * 4) = t.km[gr];
      *reinterpret_cast<uint32_t *>(s_vm + g * MST + (gr * 16 + lr) * 4) = t.vm[gr];
    }
    __builtin_amdgcn_wave_barrier();
  };
  auto attend = [&](const Tile &t, int key0) __attribute__((always_inline)) {
    float sc[NP][16];
#pragma unroll
    for (int T = 0; T < 4; ++T) {
      u32x4_t km[NG];  // of keys 16 g + 4 T ..
#pragma unroll
      for (int gr = 0; gr < NG; ++gr)
        km[gr] = *reinterpret_cast<const u32x4_t *>(s_km + g * MST + (gr * 16 + 4 * T) * 4);
      bf16x8_t kf[NG][2];
#pragma unroll
      for (int gr = 0; gr < NG; ++gr)
#pragma unroll
        for (int st = 0; st < 2; ++st) kf[gr][st] = codes8((uint32_t)t.k[T][gr][st]);
#pragma unroll
      for (int np = 0; np < NP; ++np) {
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
          const float off = -16.f * qs[np][gr];
          f32x4_t c = {off, off, off, off};
#pragma unroll
          for (int st = 0; st < 2; ++st)
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[gr][st], qf[np][gr][st], c, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t m = km[gr][i];
            const float base = gr == 0 ? zero_of(m) * qs[np][gr]
                                       : fmaf(zero_of(m), qs[np][gr], sc[np][4 * T + i]);
            sc[np][4 * T + i] = fmaf(scale_of(m), c[i], base);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    const bool masked = key0 + PG_TILE > min(all_see, k1);
    bf16x8_t pf[NP][NG][2];
#pragma unroll
    for (int np = 0; np < NP; ++np) {
      const int lim = min(seen[np], k1) - (key0 + 16 * g);  // of this lane's 16 keys
      if (masked) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (i >= lim) sc[np][i] = -INFINITY;
      }
      float mx = sc[np][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[np][i]);
      // the running maximum rises only when some score exceeds it by more than 2^8
      if (__ballot(mx * scale_log2 > m_run[np] + 8.f)) {
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * scale_log2;
        const float m_new = fmaxf(m_run[np], mx);
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[np] - m_new);
#pragma unroll
        for (int db = 0; db < DB; ++db) o[np][db] *= alpha;
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
          ones[np][gr] *= alpha;
          zs[np][gr] *= alpha;
        }
        l_run[np] *= alpha;
        m_run[np] = m_new;
      }
      const float m_off = m_run[np] == -INFINITY ? 0.f : m_run[np];  // (no key yet: every p is 0)
      float pv[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        pv[i] = __builtin_amdgcn_exp2f(fmaf(sc[np][i], scale_log2, -m_off));
        l_run[np] += pv[i];
      }
#pragma unroll
      for (int gr = 0; gr < NG; ++gr) {
        float ps[16];
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          u32x4_t m = *reinterpret_cast<const u32x4_t *>(s_vm + g * MST + (gr * 16 + 4 * i4) * 4);
          if (masked) {  // a hidden key's scale and zero may be anything: 0 times them is not taken
#pragma unroll
            for (int j = 0; j < 4; ++j) m[j] = 4 * i4 + j < lim ? m[j] : 0u;
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float sv = scale_of(m[j]), p_ = pv[4 * i4 + j];
            ps[4 * i4 + j] = p_ * sv;
            zs[np][gr] = fmaf(p_, fmaf(8.f, sv, zero_of(m[j])), zs[np][gr]);
          }
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          u32x4_t x;
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = pack_bf2(ps[8 * st + i], ps[8 * st + 4 + i]);
          pf[np][gr][st] = __builtin_bit_cast(bf16x8_t, x);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    const bf16x8_t one = __builtin_bit_cast(
        bf16x8_t, (u32x4_t){0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
#pragma unroll
    for (int np = 0; np < NP; ++np)
#pragma unroll
      for (int gr = 0; gr < NG; ++gr)
#pragma unroll
        for (int st = 0; st < 2; ++st)
          ones[np][gr] =
              __builtin_amdgcn_mfma_f32_16x16x32_bf16(one, pf[np][gr][st], ones[np][gr], 0, 0, 0);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const i32x2_t w = __builtin_amdgcn_ds_read_tr4_b64_v2i32(
          (__attribute__((address_space(3))) i32x2_t *)(mem + lane * VST + db * 8));
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const bf16x8_t vf = codes8((uint32_t)w[st]);
#pragma unroll
        for (int np = 0; np < NP; ++np)
          o[np][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[np][db / 4][st], o[np][db], 0,
                                                              0, 0);
      }
      if (db & 1) __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_wave_barrier();
  };
  constexpr int STEP = 4 * PG_TILE;
  int key0 = k0 + wave * PG_TILE;
  if (key0 < k1) {
    Tile t0, t1;
    load(t0, key0, page_at(key0));
    int page = page_at(key0 + STEP);
    while (true) {
      const int next = page_at(key0 + 2 * STEP);
      stash(t0);
      load(t1, key0 + STEP, page);  // (past the end: its last page again)
      __builtin_amdgcn_sched_barrier(0);
      attend(t0, key0);
      key0 += STEP;
      if (key0 >= k1) break;
      page = page_at(key0 + 2 * STEP);
      stash(t1);
      load(t0, key0 + STEP, next);
      __builtin_amdgcn_sched_barrier(0);
      attend(t1, key0);
      key0 += STEP;
      if (key0 >= k1) break;
    }
  }
  // the waves' parts through LDS: rows of a pair's outputs
  __syncthreads();
  float *mine = reinterpret_cast<float *>(mem);
#pragma unroll
  for (int np = 0; np < NP; ++np) {
    float l = l_run[np];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
#pragma unroll
    for (int gr = 0; gr < NG; ++gr) {
      float z = zs[np][gr];
      z += __shfl_xor(z, 16, 64);
      z += __shfl_xor(z, 32, 64);
      z = fmaf(-24.f, ones[np][gr][0], z);
#pragma unroll
      for (int db = 4 * gr; db < 4 * gr + 4; ++db)
        *reinterpret_cast<f32x4_t *>(mine + (np * 16 + lr) * OST + db * 16 + 4 * g) =
            o[np][db] + (f32x4_t){z, z, z, z};
    }
    if (g == 0) {
      s_m[wave][np * 16 + lr] = m_run[np];
      s_l[wave][np * 16 + lr] = l;
    }
  }
  __syncthreads();
  constexpr int PER = HD / 8;  // lanes of a pair
  const int e0 = tid % PER * 8;
  for (int i = tid / PER; v0 + i <= last; i += 256 / PER) {
    float mm = -INFINITY, l = 0.f, a[8];
#pragma unroll
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, s_m[w][i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      // a wave without a key of the pair has l = 0 (m = -inf is also what NaN scores leave, with
      // a sum of NaN)
      const float lw = s_l[w][i];
      if (lw == 0.f) continue;
      const float f = mm == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(s_m[w][i] - mm);
      l = fmaf(f, lw, l);
      const float *x = reinterpret_cast<const float *>(s_mem + w * WAVE_BYTES) + i * OST + e0;
      float xv[8];
      load8(x, xv);
#pragma unroll
      for (int j = 0; j < 8; ++j) a[j] = fmaf(f, xv[j], a[j]);
    }
    int r, head;
    place(v0 + i, r, head);
    const size_t row = (size_t)r * hq + head;
    if (split) {  // fp16 scaled by a power of two, as the merge takes them
      float big = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = fabsf(a[j]);
        big = x < INFINITY ? fmaxf(big, x) : big;
      }
#pragma unroll
      for (int d = 1; d < PER; d <<= 1) big = fmaxf(big, __shfl_xor(big, d, 64));
      const int e = max(__builtin_amdgcn_frexp_expf(big), -100) - 15;
      const float down = ldexpf(1.f, -e);
      const size_t prow = (size_t)chunk * s.n_rows * hq + row;
      typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
      f16x8_t x;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = (_Float16)(a[j] * down);
      *reinterpret_cast<f16x8_t *>(part_o + prow * HD + e0) = x;
      if (e0 == 0) part_ml[prow] = make_float4(mm, l, ldexpf(1.f, e), 0.f);
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

static int pair_tiles(const PagedBatch &s, int G, int *np) {
  const long long pairs = (long long)s.rows_max * G;
  *np = pairs > 16 ? 2 : 1;
  return (int)((pairs + 16 * *np - 1) / (16 * *np));
}

static PagedPlan paged_plan(const PagedBatch &s, int hq, int hkv) {
  PagedPlan p;
  int np;
  p.tiles = pair_tiles(s, hq / hkv, &np);
  const long long items = (long long)s.n_req * p.tiles * hkv;
  const int kt = (s.limit + PG_TILE - 1) / PG_TILE;
  // chunks of whole rounds of the block's waves
  const long long want = std::max(1LL, 4LL * gemm_cu_count() / std::max(1LL, items));
  const long long most = std::max(1, std::min(MERGE_SLOTS, kt / 8));
  const int per = kt ? (int)((kt + std::min(want, most) - 1) / std::min(want, most)) : 1;
  p.chunk_keys = (per + 3) / 4 * 4 * PG_TILE;
  p.chunks = std::max(1, (s.limit + p.chunk_keys - 1) / p.chunk_keys);
  return p;
}

size_t paged_part_floats(const PagedBatch &s, int hq, int hkv, int hd) {
  if (s.n_rows == 0) return 0;
  const PagedPlan p = paged_plan(s, hq, hkv);
  const size_t items = (size_t)p.chunks * s.n_rows * hq;
  return p.chunks > 1 ? items * (hd / 2) + items * 4 : 0;
}

hipError_t launch_paged_attention(const PagedBatch &s, const PagePool &p, const void *q, int hq,
                                  int hkv, int hd, void *out, float *lse, float *part,
                                  hipStream_t st) {
  if (s.n_rows == 0) return hipSuccess;
  const PagedPlan plan = paged_plan(s, hq, hkv);
  int np;
  pair_tiles(s, hq / hkv, &np);
  const dim3 g((unsigned)((size_t)s.n_req * plan.chunks * plan.tiles * hkv)), b(256);
  const float scale = 1.4426950408889634f / sqrtf((float)hd);
  const bf16_t *Q = reinterpret_cast<const bf16_t *>(q);
  bf16_t *O = reinterpret_cast<bf16_t *>(out);
  float4 *ml = reinterpret_cast<float4 *>(part);  // (m, l, f) of every slot, then the outputs
  _Float16 *po = reinterpret_cast<_Float16 *>(ml + (size_t)plan.chunks * s.n_rows * hq);
#define AKVS_PAGED(HD_, NP_)                                                                      \
  hipLaunchKernelGGL((k_paged_few<HD_, NP_>), g, b, 0, st, s, p, plan, Q, hq, hkv, scale, O, lse, \
                     po, ml)
  if (hd == 128) {
    if (np == 2) AKVS_PAGED(128, 2); else AKVS_PAGED(128, 1);
  } else {
    if (np == 2) AKVS_PAGED(64, 2); else AKVS_PAGED(64, 1);
  }
#undef AKVS_PAGED
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.chunks <= 1) return e;
  const SharedBatch rows{s.n_req, s.n_rows, s.rows_max, 0, 0, s.row_start, nullptr};
  return launch_merge_slots(rows, plan.chunks, hq, hd, po, ml, out, lse, st);
}

}  // namespace akvs
