// Pages of 4-bit caches: rows in and out, and which page belongs to which sequence.
#include <algorithm>

#include "kernels.h"
#include "pages_dev.h"
#include "quant_dev.h"

namespace akvs {

// ---- rows in and out -------------------------------------------------------------------------
// Where a row of a batch lies: (page, row of the page); page -1: no key of its sequence, or none
// of the pool's pages; -2: no row of the batch.
struct Place {
  int page, at;
};

// A block's rows [R0, R0 + n): a thread per request finds those of its rows that are among them.
// One round trip for batches of up to 256 requests; of more, those before R0's are skipped by a
// binary search. Ends with a barrier.
__device__ __forceinline__ void paged_places(const PagedBatch &s, const PagePool &p, int R0, int n,
                                             Place *places) {
  const int tid = threadIdx.x, end = min(R0 + n, s.n_rows);
  // A request's table and keys: no keys where its sequence could not grow by these rows.
  auto keys_of = [&](int b, int &len) {
    const int32_t *table = paged_keys(s, b, len);
    if (s.grown) {
      const int q = s.seq ? s.seq[b] : b;
      if (q >= 0 && q < s.n_seq && s.grown[q] == 0) len = 0;
    }
    return table;
  };
  auto place = [&](const int32_t *table, int key, int len) {
    int page = -1;
    if (key >= 0 && key < len) page = table[key >> p.shift];
    if (page < 0 || page >= p.n_pages) page = -1;
    return Place{page, key & ((1 << p.shift) - 1)};
  };
  if (!s.row_start) {
    for (int i = tid; i < n; i += 256) {
      Place x{-2, 0};
      if (R0 + i < end) {
        const int b = (R0 + i) / s.rows_max;
        int len;
        const int32_t *table = keys_of(b, len);
        x = place(table, len - s.rows_max + (R0 + i - b * s.rows_max), len);
      }
      places[i] = x;
    }
    __syncthreads();
    return;
  }
  for (int i = tid; i < n; i += 256) places[i] = Place{-2, 0};
  __syncthreads();
  int b0 = 0;
  if (s.n_req > 256) {  // the first request that ends past R0
    int hi = s.n_req;
    while (b0 < hi) {
      const int mid = (b0 + hi) >> 1;
      if (s.row_start[mid + 1] > R0) hi = mid;
      else b0 = mid + 1;
    }
  }
  for (int base = b0; base < s.n_req; base += 256) {
    const int b = base + tid;
    if (b < s.n_req) {
      int r0, r1, len;
      paged_rows(s, b, r0, r1);
      if (r0 < end && r1 > R0) {
        const int32_t *table = keys_of(b, len);
        for (int r = max(r0, R0); r < min(r1, end); ++r)
          places[r - R0] = place(table, len - r1 + r, len);
      }
    }
    if (s.row_start[base] >= end) break;  // (the same for all threads)
  }
  __syncthreads();
}

// An item is an octet of a row's keys and values both; a block's rows make 1024 of them at most, a
// thread has those that are 256 apart. Few rows take blocks of one item a thread, whose loads are
// made before the row's place is known: 16 rows are bound by round trips to memory (request ->
// sequence -> length, table -> page), many rows by their bytes (16128 rows of 8 heads of 128: 28 us
// to store, 4.7 TB/s, 28 to load as fp32, 6.0 TB/s).
constexpr int PG_ITEMS = 4;  // of a thread, at most
static int rows_per_block(int n_rows, int items) {
  const int most = std::max(1, PG_ITEMS * 256 / items), least = std::max(1, 256 / items);
  return std::min(256, std::max(least, std::min(most, n_rows / (2 * gemm_cu_count()))));
}

template <int HD>
__global__ __launch_bounds__(256) void k_store_pages(PagedBatch s, PagePool p,
                                                     const bf16_t *__restrict__ K, long long ldk,
                                                     const bf16_t *__restrict__ V, long long ldv,
                                                     int hkv, int rows) {
  constexpr int OH = HD / 8;  // octets of a head
  __shared__ Place places[256];
  const int R0 = blockIdx.x * rows, octets = hkv * OH, n = min(rows, s.n_rows - R0) * octets;
  float k[8], v[8];
  auto read = [&](int o) {
    const int i = o / octets, e = o - i * octets;
    load8(K + (R0 + i) * ldk + e * 8, k);
    load8(V + (R0 + i) * ldv + e * 8, v);
  };
  if ((int)threadIdx.x < n) read(threadIdx.x);
  paged_places(s, p, R0, rows, places);
  for (int o = threadIdx.x; o < n; o += 256) {
    const int i = o / octets, e = o - i * octets, h = e / OH, c = e % OH;
    if (o >= 256) read(o);
    const Place at = places[i];
    if (at.page < 0) continue;  // (the same for the 8 lanes of a group)
    const size_t row = (((size_t)at.page * hkv + h) << p.shift) + at.at;
    uint32_t w, meta;
    u4_octet(k, w, meta);
    reinterpret_cast<uint32_t *>(p.k)[row * OH + c] = w;
    if ((c & 7) == 0) p.k_meta[row * (HD / 64) + c / 8] = meta;
    u4_octet(v, w, meta);
    reinterpret_cast<uint32_t *>(p.v)[row * OH + c] = w;
    if ((c & 7) == 0) p.v_meta[row * (HD / 64) + c / 8] = meta;
  }
}

template <int HD, typename TO>
__device__ __forceinline__ void load_octet(const uint8_t *codes, const uint32_t *meta, size_t row,
                                           int c, bool there, TO *out) {
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (there)
    cache_load8(codes, reinterpret_cast<const _Float16 *>(meta), AKVS_U4G64, row, HD, c * 8, x);
  store8(out, x);
}
template <int HD, typename TO>
__global__ __launch_bounds__(256) void k_load_pages(PagedBatch s, PagePool p, int hkv, int rows,
                                                    TO *__restrict__ K, TO *__restrict__ V) {
  constexpr int OH = HD / 8;
  __shared__ Place places[256];
  const int R0 = blockIdx.x * rows, octets = hkv * OH, n = min(rows, s.n_rows - R0) * octets;
  paged_places(s, p, R0, rows, places);
  for (int o = threadIdx.x; o < n; o += 256) {
    const int i = o / octets, e = o - i * octets, h = e / OH, c = e % OH;
    const Place at = places[i];
    if (at.page == -2) continue;
    const size_t row = (((size_t)max(at.page, 0) * hkv + h) << p.shift) + at.at;
    const size_t to = ((size_t)(R0 + i) * octets + e) * 8;
    if (K) load_octet<HD>(p.k, p.k_meta, row, c, at.page >= 0, K + to);
    if (V) load_octet<HD>(p.v, p.v_meta, row, c, at.page >= 0, V + to);
  }
}

hipError_t launch_store_pages(const PagedBatch &s, const PagePool &p, const void *k, long long ldk,
                              const void *v, long long ldv, int hkv, int hd, hipStream_t st) {
  if (s.n_rows == 0 || p.n_pages == 0) return hipSuccess;
  const int rows = rows_per_block(s.n_rows, hkv * hd / 8);
  const dim3 g((s.n_rows + rows - 1) / rows), b(256);
  auto x = [](const void *a) { return reinterpret_cast<const bf16_t *>(a); };
  if (hd == 128)
    hipLaunchKernelGGL(k_store_pages<128>, g, b, 0, st, s, p, x(k), ldk, x(v), ldv, hkv, rows);
  else
    hipLaunchKernelGGL(k_store_pages<64>, g, b, 0, st, s, p, x(k), ldk, x(v), ldv, hkv, rows);
  return hipGetLastError();
}

hipError_t launch_load_pages(const PagedBatch &s, const PagePool &p, int hkv, int hd, void *k,
                             void *v, int dtype, hipStream_t st) {
  if (s.n_rows == 0 || (!k && !v)) return hipSuccess;
  const int rows = rows_per_block(s.n_rows, hkv * hd / 8);
  const dim3 g((s.n_rows + rows - 1) / rows), b(256);
#define AKVS_LOAD(HD_, T_)                                                                     \
  hipLaunchKernelGGL((k_load_pages<HD_, T_>), g, b, 0, st, s, p, hkv, rows,                    \
                     reinterpret_cast<T_ *>(k), reinterpret_cast<T_ *>(v))
  if (dtype == AKVS_BF16) {
    if (hd == 128) AKVS_LOAD(128, bf16_t); else AKVS_LOAD(64, bf16_t);
  } else {
    if (hd == 128) AKVS_LOAD(128, float); else AKVS_LOAD(64, float);
  }
#undef AKVS_LOAD
  return hipGetLastError();
}

// ---- whose pages ---------------------------------------------------------------------------
// Integers only. Reference counts are changed by integer atomics, whose order does not matter;
// which page goes where follows from ranks (prefix sums), so that results do not depend on timing.

__device__ __forceinline__ int pages_of(const PageTable &t, int len) {
  return min((int)(((long long)max(len, 0) + (1 << t.shift) - 1) >> t.shift), t.max_pages);
}
__device__ __forceinline__ bool in_pool(const PageTable &t, int id) {
  return id >= 0 && id < t.n_pages;
}

// A block per pair.
__global__ __launch_bounds__(256) void k_fork_pages(PageTable t, int n, const int32_t *src,
                                                    const int32_t *dst) {
  const int i = blockIdx.x, a = src[i], b = dst[i];
  if (a < 0 || a >= t.n_seq || b < 0 || b >= t.n_seq) return;
  bool out = t.len[b] != 0;
  for (int j = threadIdx.x; j < n; j += 256) out |= src[j] == b || (j < i && dst[j] == b);
  if (__syncthreads_or(out)) return;
  const int len = t.len[a], used = pages_of(t, len);
  const int32_t *from = t.table + (size_t)a * t.max_pages;
  int32_t *to = t.table + (size_t)b * t.max_pages;
  for (int j = threadIdx.x; j < used; j += 256) {
    const int id = from[j];
    to[j] = id;
    if (in_pool(t, id)) atomicAdd(&t.ref[id], 1);
  }
  if (threadIdx.x == 0) {
    t.len[b] = max(len, 0);
    if (t.grown) t.grown[b] = 1;
  }
}

// A block per sequence.
__global__ __launch_bounds__(256) void k_free_pages(PageTable t, int n, const int32_t *seq) {
  const int i = blockIdx.x, a = seq[i];
  if (a < 0 || a >= t.n_seq) return;
  bool out = false;
  for (int j = threadIdx.x; j < i; j += 256) out |= seq[j] == a;
  if (__syncthreads_or(out)) return;
  const int used = pages_of(t, t.len[a]);
  int32_t *mine = t.table + (size_t)a * t.max_pages;
  for (int j = threadIdx.x; j < used; j += 256) {
    const int id = mine[j];
    mine[j] = -1;
    if (in_pool(t, id)) atomicSub(&t.ref[id], 1);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    t.len[a] = 0;
    if (t.grown) t.grown[a] = 1;
  }
}

// Pages are counted in segments of 1024, 4 a thread.
constexpr int SEG_PER = 4, SEG = SEG_PER * 256;
static int segments(const PageTable &t) { return (t.n_pages + SEG - 1) / SEG; }

__device__ __forceinline__ int wave_sum_int(int x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}
__device__ __forceinline__ int block_sum(int x) {  // of 256 threads
  __shared__ int s[4];
  x = wave_sum_int(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
  __syncthreads();
  return s[0] + s[1] + s[2] + s[3];
}
// Sum of the threads before this one; total: of all.
__device__ __forceinline__ int block_scan(int x, int &total) {
  __shared__ int s[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int y = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int z = __shfl_up(y, o, 64);
    if (lane >= o) y += z;
  }
  __syncthreads();
  if (lane == 63) s[wave] = y;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) before += s[w];
    total += s[w];
  }
  return before + y - x;
}

// Bit j: page (segment start + 4 thread + j) is in use; pages past the last are not counted in
// `there`.
struct SegBits {
  uint32_t used, there;
};
__device__ __forceinline__ SegBits seg_bits(const PageTable &t, int seg) {
  const int id0 = seg * SEG + threadIdx.x * SEG_PER;
  SegBits x{0, 0};
  if (id0 + SEG_PER <= t.n_pages) {
    const int4 v = *reinterpret_cast<const int4 *>(t.ref + id0);
    x.used = (uint32_t)(v.x > 0) | (uint32_t)(v.y > 0) << 1 | (uint32_t)(v.z > 0) << 2 |
             (uint32_t)(v.w > 0) << 3;
    x.there = 15u;
  } else {
    for (int j = 0; j < SEG_PER && id0 + j < t.n_pages; ++j) {
      x.used |= (uint32_t)(t.ref[id0 + j] > 0) << j;
      x.there |= 1u << j;
    }
  }
  return x;
}
// Sum of the counts of segments [0, n).
__device__ __forceinline__ int seg_before(const int32_t *count, int n) {
  int x = 0;
  for (int j = threadIdx.x; j < n; j += 256) x += count[j];
  return block_sum(x);
}

// The same from the pages themselves: of a few segments a launch less.
//   192 branches end, begin again and grow, three segments: 29.3 us with a launch for the counts, 26.3
//   without; 1500 pages move together in 3 layers: 50.6 and 49.0.
constexpr int FEW_SEGS = 8;
__device__ __forceinline__ uint32_t seg_pages(const PageTable &t, int seg, bool used) {
  const SegBits x = seg_bits(t, seg);
  return used ? x.used : x.there & ~x.used;
}
__device__ __forceinline__ int pages_before(const PageTable &t, int n, bool used) {
  int x = 0;
  for (int j = 0; j < n; ++j) x += __popc(seg_pages(t, j, used));
  return block_sum(x);
}

// Workspace of akvs_grow_pages (ints): claim [n_seq], ends [n], copies [n], need [n],
// count [segments], list [n_pages]; of akvs_compact_pages: count, rank [n_pages], refs [n_pages].
struct GrowWs {
  int32_t *claim, *ends, *copies, *need, *count, *list;
};
static size_t pad4(size_t n) { return (n + 3) & ~(size_t)3; }
static GrowWs grow_ws(const PageTable &t, int n, int32_t *ws) {
  GrowWs w;
  w.claim = ws;
  w.ends = w.claim + pad4(t.n_seq);
  w.copies = w.ends + pad4(n);
  w.need = w.copies + pad4(n);
  w.count = w.need + pad4(n);
  w.list = w.count + pad4(segments(t));
  return w;
}
size_t pages_ws_ints(const PageTable &t, int n) {
  const size_t pages = pad4(t.n_pages), seg = pad4(segments(t));
  return std::max(pad4(t.n_seq) + 3 * pad4(n) + seg + pages, seg + 2 * pages);
}

// Block 0: what each sequence needs (pages, and one of them for a copy: bit 30), -1 where it cannot
// be served, and the sums up to it. The other blocks count the free pages of a segment each, or, of
// few segments, list them.
__device__ __forceinline__ void grow_list(uint32_t bits, int seg, int rank, int need,
                                          int32_t *list) {
  const int id0 = seg * SEG + threadIdx.x * SEG_PER;
  while (bits && rank < need) {
    const int j = __ffs(bits) - 1;
    list[rank++] = id0 + j;
    bits &= bits - 1;
  }
}
constexpr int NEED_COPY = 1 << 30;
__global__ __launch_bounds__(256) void k_grow_need(PageTable t, int n, const int32_t *seq,
                                                   const int32_t *add, GrowWs w, bool list) {
  if (blockIdx.x > 0) {
    const int seg = blockIdx.x - 1;
    const uint32_t bits = seg_pages(t, seg, false);
    int c;
    const int rank = block_scan(__popc(bits), c);
    if (threadIdx.x == 0) w.count[seg] = c;
    if (list) grow_list(bits, seg, rank + pages_before(t, seg, false), t.n_pages, w.list);
    return;
  }
  for (int i = threadIdx.x; i < n; i += 256) {
    const int a = seq[i];
    if (a >= 0 && a < t.n_seq) w.claim[a] = 0x7fffffff;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += 256) {
    const int a = seq[i];
    if (a >= 0 && a < t.n_seq) atomicMin(&w.claim[a], i);
  }
  __syncthreads();
  int ends = 0, copies = 0;
  for (int base = 0; base < n; base += 256) {
    const int i = base + threadIdx.x;
    int need = 0, copy = 0;
    bool ok = false;
    if (i < n) {
      const int a = seq[i], more = add[i];
      // (claim: read past this block's own atomics)
      ok = a >= 0 && a < t.n_seq && more >= 0 &&
           __hip_atomic_load(&w.claim[a], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == i;
      if (ok) {
        const int rows = 1 << t.shift, old = max(t.len[a], 0);
        const long long want = ((long long)old + more + rows - 1) >> t.shift;
        ok = want <= t.max_pages && old + (long long)more <= 0x7fffffff;
        if (ok && more > 0) {
          const int have = (int)(((long long)old + rows - 1) >> t.shift);
          if (old & (rows - 1)) {
            const int last = t.table[(size_t)a * t.max_pages + (old >> t.shift)];
            copy = in_pool(t, last) && t.ref[last] > 1;
          }
          need = (int)want - have + copy;
        }
      }
    }
    int tn, tc;
    const int en = block_scan(need, tn), ec = block_scan(copy, tc);
    if (i < n) {
      w.ends[i] = ends + en + need;
      w.copies[i] = copies + ec + copy;
      w.need[i] = ok ? need | (copy ? NEED_COPY : 0) : -1;
    }
    ends += tn;
    copies += tc;
  }
}

// The free pages that are needed, in ascending order.
__global__ __launch_bounds__(256) void k_grow_pick(PageTable t, int n, GrowWs w) {
  const uint32_t bits = seg_pages(t, blockIdx.x, false);
  const int need = w.ends[n - 1], before = seg_before(w.count, blockIdx.x);
  if (before >= need) return;
  int total;
  const int rank = before + block_scan(__popc(bits), total);
  grow_list(bits, blockIdx.x, rank, need, w.list);
}

// A wave per sequence; the last block: the totals, and -1 past the last move. All that a wave needs is
// requested before the free pages are counted, which decides whether its sequence is served.
__global__ __launch_bounds__(256) void k_grow_assign(PageTable t, int n, int segs,
                                                     const int32_t *seq, const int32_t *add,
                                                     GrowWs w, int32_t *served, int32_t *move_src,
                                                     int32_t *move_dst, int32_t *counts) {
  auto serves = [&](int need, int ends, int free_pages) {
    return need >= 0 && ((need & ~NEED_COPY) == 0 || ends <= free_pages);
  };
  if (blockIdx.x == gridDim.x - 1) {
    __shared__ int s_moves[4], s_taken[4];
    int i = threadIdx.x, x = -1, e = 0, c = 0;
    auto read = [&]() {
      x = w.need[i];
      e = w.ends[i];
      c = w.copies[i];
    };
    if (i < n) read();
    const int free_pages = seg_before(w.count, segs);
    int moves = 0, taken = 0;
    while (i < n) {
      if (serves(x, e, free_pages) && (x & ~NEED_COPY)) {
        moves = max(moves, c);
        taken = max(taken, e);
      }
      i += 256;
      if (i < n) read();
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      moves = max(moves, __shfl_xor(moves, d, 64));
      taken = max(taken, __shfl_xor(taken, d, 64));
    }
    if ((threadIdx.x & 63) == 0) {
      s_moves[threadIdx.x >> 6] = moves;
      s_taken[threadIdx.x >> 6] = taken;
    }
    __syncthreads();
    moves = max(max(s_moves[0], s_moves[1]), max(s_moves[2], s_moves[3]));
    taken = max(max(s_taken[0], s_taken[1]), max(s_taken[2], s_taken[3]));
    for (int i = moves + threadIdx.x; i < n; i += 256) move_src[i] = move_dst[i] = -1;
    if (threadIdx.x == 0) {
      counts[0] = moves;
      counts[1] = taken;
    }
    return;
  }
  const int i = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  int x = -1, ends = 0, copies = 0, more = 0, old = 0, last = 0, first = 0;
  int32_t *mine = nullptr, *grown = nullptr;
  if (i < n) {
    const int a = seq[i];
    if (t.grown && a >= 0 && a < t.n_seq && w.claim[a] == i) grown = t.grown + a;
    x = w.need[i];
    ends = w.ends[i];
    copies = w.copies[i];
    more = add[i];
    if (x >= 0) {  // (a is a sequence)
      old = max(t.len[a], 0);
      mine = t.table + (size_t)a * t.max_pages;
      if (x & NEED_COPY) last = mine[old >> t.shift];
      const int need = x & ~NEED_COPY, at = ends - need + lane;
      if (lane < need && at < t.n_pages) first = w.list[at];
    }
  }
  const int free_pages = seg_before(w.count, segs);
  if (i >= n) return;
  const bool ok = serves(x, ends, free_pages);
  if (lane == 0) {
    served[i] = ok;
    if (grown) *grown = ok;
  }
  if (!ok) return;
  const int need = x & ~NEED_COPY, base = ends - need;
  const bool copy = x & NEED_COPY;
  const int have = (int)(((long long)old + (1 << t.shift) - 1) >> t.shift);
  const int start = copy ? old >> t.shift : have;
  if (copy && lane == 0) {
    const int m = copies - 1;
    move_src[m] = last;
    move_dst[m] = first;
    atomicSub(&t.ref[last], 1);
  }
  for (int j = lane; j < need; j += 64) {
    const int id = j < 64 ? first : w.list[base + j];
    mine[start + j] = id;
    t.ref[id] = 1;
  }
  if (lane == 0) t.len[seq[i]] = old + more;
}

__global__ __launch_bounds__(256) void k_compact_count(PageTable t, int32_t *count) {
  const int c = block_sum(__popc(seg_bits(t, blockIdx.x).used));
  if (threadIdx.x == 0) count[blockIdx.x] = c;
}

// Ranks: the pages in use from number N (of all in use) on move, the k-th to the k-th free number
// below N. rank [n_pages] of those that move, -1 of others from N on; refs [moves] theirs. count:
// NULL where there are few segments.
__global__ __launch_bounds__(256) void k_compact_rank(PageTable t, int segs, const int32_t *count,
                                                      int32_t *rank, int32_t *refs,
                                                      int32_t *move_src, int32_t *move_dst,
                                                      int32_t *counts) {
  auto used_before = [&](int n) {
    return count ? seg_before(count, n) : pages_before(t, n, true);
  };
  const int N = used_before(segs), sn = N / SEG;
  // pages in use below N: whole segments, and those of N's segment before it
  int below = used_before(min(sn, segs));
  if (sn < segs) {
    const int lim = N - (sn * SEG + (int)threadIdx.x * SEG_PER);
    const uint32_t mask = lim >= SEG_PER ? 15u : lim > 0 ? (1u << lim) - 1 : 0u;
    below += block_sum(__popc(seg_bits(t, sn).used & mask));
  }
  const int moves = N - below;
  const SegBits x = seg_bits(t, blockIdx.x);
  int total;
  int before = used_before(blockIdx.x);
  before += block_scan(__popc(x.used), total);
  const int id0 = blockIdx.x * SEG + threadIdx.x * SEG_PER;
  for (int j = 0; j < SEG_PER && id0 + j < t.n_pages; ++j) {
    const int id = id0 + j;
    const bool used = (x.used >> j) & 1;
    if (id < N) {
      if (!used) move_dst[id - before] = id;
    } else {
      const int k = before - below;
      rank[id] = used ? k : -1;
      if (used) {
        move_src[k] = id;
        refs[k] = t.ref[id];
      }
    }
    if (id >= moves) {
      move_src[id] = move_dst[id] = -1;
    }
    before += used;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    counts[0] = moves;
    counts[1] = N;
  }
}

// Entries and refs afterwards: blocks [0, entry_blocks) take 256 entries each, the others 256
// refs. Each value is read by the thread that writes it, so the outputs may be the inputs.
__global__ __launch_bounds__(256) void k_compact_write(PageTable t, int entry_blocks,
                                                       const int32_t *rank, const int32_t *refs,
                                                       const int32_t *move_dst,
                                                       const int32_t *counts, int32_t *table_out,
                                                       int32_t *ref_out) {
  const int N = counts[1];
  if (blockIdx.x < (unsigned)entry_blocks) {
    const size_t e = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= (size_t)t.n_seq * t.max_pages) return;
    const int s = (int)(e / t.max_pages), j = (int)(e - (size_t)s * t.max_pages);
    int id = t.table[e];
    if (id >= N && id < t.n_pages && j < pages_of(t, t.len[s]) && rank[id] >= 0)
      id = move_dst[rank[id]];
    table_out[e] = id;
    return;
  }
  const int id = (blockIdx.x - entry_blocks) * 256 + threadIdx.x;
  if (id >= t.n_pages) return;
  if (id >= N) {
    ref_out[id] = 0;
    return;
  }
  const int own = t.ref[id];
  if (own > 0) {
    ref_out[id] = own;
    return;
  }
  int lo = 0, hi = counts[0] - 1;  // its place among the targets
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (move_dst[mid] < id) lo = mid + 1;
    else hi = mid;
  }
  ref_out[id] = refs[lo];
}

// Pieces of 16 KB of (move, layer, codes and meta of keys and values), blocks in turn.
constexpr int MOVE_PIECE = 16384, MOVE_BLOCKS = 2048;
__global__ __launch_bounds__(256) void k_move_pages(PagePool p, int layers, int code_bytes,
                                                    int meta_bytes, const int32_t *src,
                                                    const int32_t *dst, int max_moves,
                                                    const int32_t *n_moves) {
  const int moves = n_moves ? min(max(*n_moves, 0), max_moves) : max_moves;
  const int cp = (code_bytes + MOVE_PIECE - 1) / MOVE_PIECE;
  const int mp = (meta_bytes + MOVE_PIECE - 1) / MOVE_PIECE;
  const int per = 2 * (cp + mp);
  const long long all = (long long)moves * layers * per;
  for (long long id = blockIdx.x; id < all; id += gridDim.x) {
    const long long ml = id / per;
    const int m = (int)(ml / layers), layer = (int)(ml - (long long)m * layers);
    int piece = (int)(id - ml * per);
    const int a = src[m], b = dst[m];
    if (a < 0 || a >= p.n_pages || b < 0 || b >= p.n_pages) continue;
    const bool meta = piece >= 2 * cp;
    if (meta) piece -= 2 * cp;
    const int pieces = meta ? mp : cp, bytes = meta ? meta_bytes : code_bytes;
    const bool v = piece >= pieces;
    if (v) piece -= pieces;
    char *base = meta ? reinterpret_cast<char *>(v ? p.v_meta : p.k_meta)
                      : reinterpret_cast<char *>(v ? p.v : p.k);
    base += (size_t)layer * p.n_pages * bytes;
    const char *from = base + (size_t)a * bytes;
    char *to = base + (size_t)b * bytes;
    const int end = min(bytes, (piece + 1) * MOVE_PIECE);
    u32x4_t x[MOVE_PIECE / 4096];
#pragma unroll
    for (int u = 0; u < MOVE_PIECE / 4096; ++u) {
      const int o = piece * MOVE_PIECE + u * 4096 + threadIdx.x * 16;
      if (o < end) x[u] = *reinterpret_cast<const u32x4_t *>(from + o);
    }
#pragma unroll
    for (int u = 0; u < MOVE_PIECE / 4096; ++u) {
      const int o = piece * MOVE_PIECE + u * 4096 + threadIdx.x * 16;
      if (o < end) *reinterpret_cast<u32x4_t *>(to + o) = x[u];
    }
  }
}

hipError_t launch_fork_pages(const PageTable &t, int n, const int32_t *src, const int32_t *dst,
                             hipStream_t st) {
  if (n == 0) return hipSuccess;
  hipLaunchKernelGGL(k_fork_pages, dim3(n), dim3(256), 0, st, t, n, src, dst);
  return hipGetLastError();
}

hipError_t launch_free_pages(const PageTable &t, int n, const int32_t *seq, hipStream_t st) {
  if (n == 0) return hipSuccess;
  hipLaunchKernelGGL(k_free_pages, dim3(n), dim3(256), 0, st, t, n, seq);
  return hipGetLastError();
}

hipError_t launch_grow_pages(const PageTable &t, int n, const int32_t *seq, const int32_t *add,
                             int32_t *served, int32_t *move_src, int32_t *move_dst,
                             int32_t *counts, int32_t *ws, hipStream_t st) {
  const int segs = segments(t);
  const GrowWs w = grow_ws(t, n, ws);
  const dim3 b(256);
  if (n > 0) {
    hipLaunchKernelGGL(k_grow_need, dim3(1 + segs), b, 0, st, t, n, seq, add, w, segs <= FEW_SEGS);
    if (segs > FEW_SEGS) hipLaunchKernelGGL(k_grow_pick, dim3(segs), b, 0, st, t, n, w);
  }
  hipLaunchKernelGGL(k_grow_assign, dim3((n + 3) / 4 + 1), b, 0, st, t, n, segs, seq, add, w,
                     served, move_src, move_dst, counts);
  return hipGetLastError();
}

hipError_t launch_compact_pages(const PageTable &t, int32_t *table_out, int32_t *ref_out,
                                int32_t *move_src, int32_t *move_dst, int32_t *counts, int32_t *ws,
                                hipStream_t st) {
  const int segs = segments(t);
  int32_t *count = ws, *rank = count + pad4(segs), *refs = rank + pad4(t.n_pages);
  const dim3 b(256);
  if (segs > FEW_SEGS) hipLaunchKernelGGL(k_compact_count, dim3(segs), b, 0, st, t, count);
  hipLaunchKernelGGL(k_compact_rank, dim3(std::max(segs, 1)), b, 0, st, t, segs,
                     segs > FEW_SEGS ? count : nullptr, rank, refs, move_src, move_dst, counts);
  const int entries = (int)(((size_t)t.n_seq * t.max_pages + 255) / 256);
  hipLaunchKernelGGL(k_compact_write, dim3(entries + (t.n_pages + 255) / 256), b, 0, st, t, entries,
                     rank, refs, move_dst, counts, table_out, ref_out);
  return hipGetLastError();
}

hipError_t launch_move_pages(const PagePool &p, int layers, int hkv, int hd, const int32_t *src,
                             const int32_t *dst, int max_moves, const int32_t *n_moves,
                             hipStream_t st) {
  if (max_moves == 0 || layers == 0 || p.n_pages == 0) return hipSuccess;
  const int codes = (hkv * hd / 2) << p.shift, meta = (hkv * hd / 64 * 4) << p.shift;
  const long long per = 2LL * ((codes + MOVE_PIECE - 1) / MOVE_PIECE +
                               (meta + MOVE_PIECE - 1) / MOVE_PIECE);
  const long long all = per * max_moves * layers;
  hipLaunchKernelGGL(k_move_pages, dim3((unsigned)std::min<long long>(all, MOVE_BLOCKS)), dim3(256),
                     0, st, p, layers, codes, meta, src, dst, max_moves, n_moves);
  return hipGetLastError();
}

}  // namespace akvs
