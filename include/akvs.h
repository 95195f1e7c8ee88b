/*
 * akvs.h - C ABI of the AgentKVShift reuse-prefill library for AMD MI355X (gfx950).
 *
 * The library computes the reuse prefill of "AgentKVShift: Efficient KV Cache Reuse
 * for Agentic Memory Systems": a query is prefilled on top of m memory units whose
 * per-layer K/V caches were computed once, each unit alone at position 0 (Sec. 3.1).
 * Cached keys are re-rotated to the unit's new offset, a small probe subset of each
 * unit plus the query is recomputed at every layer from the check layer on, each
 * unit's fresh-minus-reused offset is estimated on its probes, and every other token
 * is corrected by one weighted vector add (Sec. 3.3, Algorithm 1).
 *
 * Conventions shared by every entry point
 *  - Ownership: every tensor argument is a caller-owned DEVICE pointer, dense,
 *    row-major, 16-byte aligned, unless the argument says "host". Descriptor structs
 *    and chunk-length arrays are host memory read during the call only. The library
 *    never allocates, frees or keeps a pointer; scratch memory comes from a caller
 *    workspace sized by akvs_workspace_size / akvs_step_workspace_size (the one
 *    exception, akvs_decode_step_noalloc, uses a fixed device array of the library).
 *  - Streams: every call only enqueues work on `stream` and returns; buffers must stay
 *    alive until the stream has finished. akvs_chunk_meta and the query functions are
 *    host-only. Calls on different streams must not share output or workspace buffers.
 *  - Errors: an akvs_status is returned. Arguments are validated before anything is
 *    enqueued: an invalid call enqueues nothing and writes nothing. A HIP launch
 *    failure returns AKVS_EHIP. akvs_last_error() gives a message for the calling
 *    thread's last failure. No C++ exception crosses this interface.
 *  - Values held in device memory (token ids, positions, probe indices, chunk
 *    metadata) cannot be checked on the host. Kernels bound-check them and never
 *    read or write outside the buffers described here; an out-of-range value
 *    produces unspecified numbers in the affected rows, never a fault.
 *  - Determinism: no floating-point atomics; identical inputs on the same device give
 *    bitwise identical outputs.
 *  - dtypes: AKVS_F32 model = fp32 weights, activations and K/V; AKVS_BF16 model =
 *    bf16 weights and K/V, fp32 residual stream and accumulation. Quantised caches
 *    (AKVS_U4G64 / AKVS_U2G64 / AKVS_E4M3G64) are only valid as cache inputs of a bf16
 *    model.
 *
 * Layouts (L layers, D model width, Hq / Hkv heads, hd head dim, F FFN width,
 * kvw = Hkv*hd, T_c = sum of unit lengths, q = query length, T = T_c + q)
 *  - weights per layer [out][in]: w_qkv [(Hq+2Hkv)*hd][D] (q rows, then k, then v),
 *    w_o [D][Hq*hd], w_gate_up [2F][D] (gate rows first), w_down [D][F], norms [D];
 *    embed [V][D]; final_norm [D]. Weight dtype = model dtype.
 *  - unit caches k/v [L][T_c][Hkv][hd], units back to back in context order, token t
 *    of a unit stored as rotated at position t. Quantised: codes
 *    [L][T_c][Hkv][hd*bits/8] uint8 (low bits first: 4-bit element 2k is the low
 *    nibble of byte k, 2-bit element 4k is bits 0-1 of byte k) and meta
 *    [L][T_c][Hkv][hd/64][2] fp16 (scale, zero); x = scale*code + zero.
 *  - corrected / fresh caches [L][T][Hkv][hd], indexed by position.
 *  - rotary table [n_pos][hd/2][2] fp32 (cos, sin) of p * theta^(-2k/hd), rotate-half
 *    pairing of dimension k with k + hd/2.
 *  - pages of a 4-bit cache (one layer): codes [n_pages][Hkv][page_rows][hd/2] uint8 and meta
 *    [n_pages][Hkv][page_rows][hd/64][2] fp16 (scale, zero), the codes as in a quantised cache:
 *    a head's rows of a page are contiguous. Key j of a sequence is row j % page_rows of the
 *    page that entry j / page_rows of the sequence's table names.
 *  - 4-bit weights [out][in]: codes [out][in/2] uint8, meta [out][in/64][2] fp16 (what
 *    akvs_quantize_cache makes of rows of `in` elements).
 */
#ifndef AKVS_H
#define AKVS_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t akvs_status;
enum {
  AKVS_OK = 0,
  AKVS_EINVAL = 1,       /* null pointer, bad range, misaligned pointer          */
  AKVS_ESHAPE = 2,       /* inconsistent sizes                                   */
  AKVS_EDTYPE = 3,       /* dtype not valid for this argument / model            */
  AKVS_EUNSUPPORTED = 4, /* valid but not implemented (e.g. head_dim not 64/128) */
  AKVS_ENOSPACE = 5,     /* workspace too small                                  */
  AKVS_EHIP = 6          /* HIP runtime error while enqueueing                   */
};

enum { AKVS_F32 = 0, AKVS_BF16 = 1, AKVS_U4G64 = 2, AKVS_U2G64 = 3, AKVS_E4M3G64 = 4 };

/* akvs_reuse_cfg.flags */
enum {
  AKVS_F_NO_CORRECTION = 1u,       /* offsets forced to 0 (probes fresh, others as reused)   */
  AKVS_F_UNIT_WEIGHTS = 2u,        /* w = 1 instead of min(d, 1)                            */
  AKVS_F_FRESH_IF_RECOMPUTED = 4u, /* a token recomputed for either side takes fresh K and V */
  AKVS_F_NO_PREFIX_RECOMPUTE = 8u, /* stale reuse: no check layer; needs refresh_num == 0    */
  AKVS_F_GIVEN_PROBES = 16u,       /* probe sets come from the caller instead of top-b       */
  AKVS_F_PRE_ROPE_OFFSETS = 32u    /* key offsets taken before the rotary map: each probe's
                                      difference is rotated back by its position before the
                                      mean, the offset rotated to each corrected token's */
};

typedef struct akvs_model_cfg {
  int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, ffn_dim, vocab;
  float rope_theta, rms_eps;
  int32_t dtype; /* AKVS_F32 or AKVS_BF16 */
} akvs_model_cfg;

typedef struct akvs_layer_w {
  const void *attn_norm, *w_qkv, *w_o, *mlp_norm, *w_gate_up, *w_down;
} akvs_layer_w;

/* The retrieved units, the query and the method's parameters (Sec. 3.3, Alg. 1). */
typedef struct akvs_reuse_cfg {
  int32_t n_chunks;          /* m >= 1                                               */
  const int32_t *chunk_len;  /* host [m], every n_i >= 1                             */
  int32_t query_len;         /* q >= 1                                               */
  int32_t refresh_num, refresh_den; /* r = num/den in [0, 1]; b_i = ceil(num*n_i/den) */
  int32_t check_layer;       /* 0-based layer of the divergence check, < n_layers    */
  uint32_t flags;            /* AKVS_F_*                                             */
  int32_t refresh_v_num, refresh_v_den; /* value-side ratio (asymmetric K/V budgets);
                                           den 0: the key ratio for both sides       */
} akvs_reuse_cfg;

/* A unit cache: k, v in the cache layout above; k_meta / v_meta only when quantised. */
typedef struct akvs_cache {
  const void *k, *v;
  const void *k_meta, *v_meta;
  int32_t dtype; /* AKVS_F32 (f32 model), AKVS_BF16, AKVS_U4G64, AKVS_U2G64, AKVS_E4M3G64
                    (bf16 model) */
} akvs_cache;

/* Outputs of akvs_reuse_prefill. h_query, k_corr, v_corr are required; the others
 * may be NULL (then kept in the workspace only). */
typedef struct akvs_reuse_out {
  float *h_query;          /* [q][D] final-normed query rows                         */
  void *k_corr, *v_corr;   /* [L][T][Hkv][hd], model dtype                           */
  int32_t *probe_k, *probe_v; /* [sum b_i] global positions, per unit ascending (CSR) */
  float *d_k, *d_v;        /* [T_c] check-layer divergences                          */
  int32_t *rows;           /* [T] recomputed positions, ascending; first n_rows used  */
  int32_t *n_rows;         /* [1] number of recomputed rows M                        */
  int32_t kv_rows;         /* rows per layer of k_corr / v_corr: 0 means T; a larger
                              value leaves room for the tokens a decode step appends */
} akvs_reuse_out;

/* A batch of requests that go on from one shared context (akvs_shared_attention,
 * akvs_attention_weights). Rows are new tokens, packed request by request; every row sees all
 * keys of the shared prefix, and of its request's own keys those up to its own: the rows of a
 * request are its last ones, so row i of its n sees own keys 0 .. own_len - n + i. */
typedef struct akvs_shared_cfg {
  int32_t n_req;        /* B >= 1                                                            */
  int32_t n_rows;       /* rows that q, out and lse hold, >= 0                               */
  int32_t rows_max;     /* the most rows of one request, >= 1                                */
  int32_t prefix_len;   /* shared keys P, >= 0 (0: none)                                     */
  int32_t own_rows;     /* rows per request of k_own / v_own, >= 0 (0: none)                 */
  const int32_t *row_start; /* device [B + 1], from 0, ascending, <= n_rows: request b has rows
                               row_start[b] .. row_start[b + 1] - 1, at most rows_max of them.
                               NULL: every request has rows_max (n_rows = B * rows_max, or 0)  */
  const int32_t *own_len;   /* device [B]: own keys, 0 .. own_rows (NULL where own_rows = 0)  */
} akvs_shared_cfg;

/* What akvs_evict_cache keeps. A sequence is what has a cache of its own: a layer, a request. */
typedef struct akvs_evict_cfg {
  int32_t n_seq;        /* S >= 1                                                            */
  int32_t n_keys;       /* keys per sequence (of `weights`), >= 0                            */
  int32_t src_rows;     /* rows per sequence of k / v, >= n_keys (0: n_keys)                 */
  int32_t n_keep;       /* keys kept per sequence and KV head, >= 1                          */
  int32_t dst_rows;     /* rows per sequence of k_out / v_out, >= n_keep (0: n_keep)         */
  int32_t n_first, n_recent; /* always kept: the first and the last keys (n_first + n_recent
                                <= n_keep)                                                   */
  const int32_t *lens;  /* device [S]: keys of each sequence, 0 .. n_keys (NULL: n_keys)     */
} akvs_evict_cfg;

/* One layer's cache of 4-bit codes in pages (layout above). Layers of a model that follow each
 * other in memory are n_pages pages apart. */
typedef struct akvs_pages {
  uint8_t *k, *v;         /* codes                                                           */
  void *k_meta, *v_meta;  /* (scale, zero) of every 64 elements                              */
  int32_t n_pages;        /* >= 0 (0: none, pointers may be NULL)                            */
  int32_t page_rows;      /* keys of a page: 16, 32, 64, 128 or 256                          */
} akvs_pages;

/* The pages of S sequences, of all layers alike. A page may be named by several sequences: ref
 * counts them; a page with ref <= 0 is free. Entries that a sequence's length does not reach are
 * never read. */
typedef struct akvs_page_table {
  int32_t n_seq, max_pages;   /* S >= 1; entries of a sequence, >= 1                         */
  int32_t n_pages, page_rows; /* as in akvs_pages                                            */
  int32_t *table;             /* device [S][max_pages]                                       */
  int32_t *len;               /* device [S]: keys of each sequence                           */
  int32_t *ref;               /* device [n_pages]                                            */
  int32_t *grown;             /* device [S], or NULL: 0 for a sequence that the last
                                 akvs_grow_pages of it could not serve, 1 for others (ones
                                 at first); akvs_free_pages and akvs_fork_pages make it 1    */
} akvs_page_table;

/* A batch over sequences in pages (akvs_store_pages, akvs_load_pages, akvs_paged_attention). Rows
 * are packed request by request as in akvs_shared_cfg; a request's rows are the last keys of its
 * sequence: row i of its n is key len - n + i, and sees keys 0 .. len - n + i. */
typedef struct akvs_paged_cfg {
  int32_t n_req;        /* B >= 1                                                            */
  int32_t n_rows;       /* rows that q, out, .. hold, >= 0                                   */
  int32_t rows_max;     /* the most rows of one request, >= 1                                */
  int32_t n_seq;        /* sequences of `len` and `table`, >= 1                              */
  int32_t max_pages;    /* entries of a sequence in `table`, >= 1                            */
  int32_t max_len;      /* no sequence of the batch has more keys (longer ones count as this
                           long), 0 .. max_pages * page_rows: what calls are planned for     */
  const int32_t *row_start; /* device [B + 1] as in akvs_shared_cfg, or NULL                 */
  const int32_t *seq;   /* device [B]: the sequence of each request; NULL: b (B <= n_seq)    */
  const int32_t *len;   /* device [n_seq]: keys, the rows' own among them                    */
  const int32_t *table; /* device [n_seq][max_pages]                                         */
  const int32_t *grown; /* device [n_seq], or NULL: akvs_store_pages stores no rows of
                           sequences with 0 (akvs_page_table's); the others do not read it   */
} akvs_paged_cfg;

/* What akvs_w4_product makes of W x. */
enum {
  AKVS_W4_STORE = 0,  /* y = W x (+ resid)                                                   */
  AKVS_W4_SWIGLU = 1  /* y = silu(g) u, g the first half of W x, u the second                */
};

/* ---- library information ---------------------------------------------------- */
int32_t akvs_version(void);
const char *akvs_status_string(akvs_status s);
const char *akvs_last_error(void);

/* ---- host helpers -------------------------------------------------------------- */

/* Per-unit bookkeeping (Sec. 3.3: b = ceil(r n), exact integers). Host only.
 * meta_out (host, may be NULL): [2][m][4], table 0 for the keys and table 1 for the
 * values, row i = (start s_i, length n_i, budget b_i of that side, CSR offset of the
 * unit's probes of that side = b_0 + ... + b_{i-1}); the two tables differ only when the
 * value side has its own ratio. totals_out (host, may be NULL): [5] = (T_c, sum b_K,i,
 * row cap = sum min(n_i, b_K,i + b_V,i) + q, T, sum b_V,i). Device copies of meta_out
 * are the `chunk_meta` argument of the step entries below. */
akvs_status akvs_chunk_meta(const akvs_reuse_cfg *cfg, int32_t *meta_out, int32_t *totals_out);

/* Workspace bytes of akvs_reuse_prefill (cfg != NULL) or of akvs_full_prefill over
 * n_tokens tokens (cfg == NULL). Returns 0 for an invalid configuration. */
size_t akvs_workspace_size(const akvs_model_cfg *m, const akvs_reuse_cfg *cfg, int32_t n_tokens);
/* Workspace bytes of akvs_probe_qkv / akvs_probe_out_mlp over n_rows rows. */
size_t akvs_step_workspace_size(const akvs_model_cfg *m, int32_t n_rows);
/* Workspace bytes that let akvs_sparse_query_attention split the key range of n_rows rows
 * over n_keys keys (the launch configuration of the reuse prefill: the split partials and,
 * for few rows, a plan of the split made on the device from the positions); 0 when that
 * call would not split (fp32 models, or enough row tiles to fill the GPU). */
size_t akvs_attention_workspace_size(const akvs_model_cfg *m, int32_t n_rows, int32_t n_keys);

/* The kernels that akvs_probe_qkv and akvs_probe_out_mlp take for n_rows rows: out (host, [4]) =
 * codes of the w_qkv, w_o, w_gate_up and w_down products. Host only; lets tests and profiles
 * say which kernel ran. A code is one of the enum plus: the tile of the MFMA kernel
 * (0..3: 16 x 64, 32 x 64, 16 x 128, 32 x 128) for AKVS_G_F32_MFMA; 10 x tile + K slices for
 * AKVS_G_FEW; the tile for AKVS_G_8WAVE; the K slices for AKVS_G_8WAVE_SPLIT. */
enum {
  AKVS_G_F32_MFMA = 0, AKVS_G_F32_LDS = 10, AKVS_G_FEW = 100, AKVS_G_8WAVE = 200,
  AKVS_G_8WAVE_SPLIT = 300, AKVS_G_4WAVE = 400
};
akvs_status akvs_projection_kernels(const akvs_model_cfg *m, int32_t n_rows, int32_t *out);

/* ---- step entries ---------------------------------------------------------------- */

/* Rotary table for positions 0..n_pos-1 (Sec. 2: reused states are moved to their new
 * positions by adjusting their positional embedding; rotary embeddings, rotate-half form, are
 * this library's reading of the decoders of Sec. 4.1, and every re-rotation, probe QKV
 * projection and pre-RoPE offset reads this table):
 * table[p][k] = (cos, sin)(p * theta^(-2k/hd)), angles and their cos/sin in fp64, stored
 * rounded to fp32. table: [n_pos][hd/2][2], caller-owned device memory, 16-byte aligned;
 * n_pos = 0 writes nothing. Errors: EINVAL (n_pos < 0, hd odd or outside [2, 1024],
 * theta <= 0, null or misaligned table), EHIP. */
akvs_status akvs_rope_table(int32_t n_pos, int32_t head_dim, float rope_theta, float *table,
                            hipStream_t stream);

/* Re-encode cached keys at a new offset (Sec. 2, positional re-encoding of reused
 * states): k_dst[t] = Rot(pos_delta[t]) deq(k_src[t]), v_dst[t] = deq(v_src[t]).
 * src: n_tokens rows of [Hkv][hd] in the cache layout of src->dtype (one layer);
 * pos_delta: device [n_tokens], 0 <= delta < rope_rows; rope: akvs_rope_table output
 * with rope_rows rows. dst_dtype: AKVS_F32 (f32 cache) or AKVS_BF16. */
akvs_status akvs_rerotate_keys(const akvs_cache *src, int32_t n_tokens, int32_t n_kv_heads,
                               int32_t head_dim, const int32_t *pos_delta, const float *rope,
                               int32_t rope_rows, void *k_dst, void *v_dst, int32_t dst_dtype,
                               hipStream_t stream);

/* Check-layer divergence (Sec. 3.3 display equation): d_k[t] = || k_fresh[t] -
 * Rot(pos_delta[t]) deq(k_cached[t]) ||_2 over all Hkv*hd components, d_v likewise
 * without rotation; fp32 sums. fresh: [n_tokens][Hkv][hd] of fresh_dtype (F32/BF16);
 * cache: one layer as in akvs_rerotate_keys; pos_delta may be NULL (no rotation). */
akvs_status akvs_check_divergence(const void *k_fresh, const void *v_fresh, int32_t fresh_dtype,
                                  const akvs_cache *cache, int32_t n_tokens, int32_t n_kv_heads,
                                  int32_t head_dim, const int32_t *pos_delta, const float *rope,
                                  int32_t rope_rows, float *d_k, float *d_v, hipStream_t stream);

/* Probe selection (Sec. 3.3 "Probe selection"; Alg. 1): per unit i, S_K,i = the b_i
 * tokens of largest d_k (equal values: the earlier token first), S_V,i likewise;
 * weights w = min(d, 1) (1 with AKVS_F_UNIT_WEIGHTS). With AKVS_F_GIVEN_PROBES the
 * sets are read from probe_k / probe_v (as written below) instead. Writes
 *  probe_k [sum b_K,i], probe_v [sum b_V,i]: global positions, ascending within each
 *   unit, unit i at the CSR offset of its side's table (meta[0][i][3] / meta[1][i][3]);
 *  flags [T_c] uint8: bit0 = in S_K, bit1 = in S_V;  w_k, w_v [T_c] fp32;
 *  chunk_rows [m]: |S_K,i u S_V,i|;
 *  rows [row cap]: recomputed positions R = (u_i S_K,i u S_V,i) u query, ascending;
 *  n_rows [1]: |R|;  fresh_row [T]: index in R of each position, -1 if not recomputed.
 * chunk_meta: device copy of akvs_chunk_meta's meta_out. d_k, d_v must be finite. A
 * probe array may be NULL when its side's budgets are all 0. */
akvs_status akvs_select_probes(const float *d_k, const float *d_v, const akvs_reuse_cfg *cfg,
                               const int32_t *chunk_meta, int32_t *probe_k, int32_t *probe_v,
                               float *w_k, float *w_v, uint8_t *flags, int32_t *chunk_rows,
                               int32_t *rows, int32_t *n_rows, int32_t *fresh_row,
                               hipStream_t stream);

/* Probe-row projections (Alg. 1, recompute of the probe rows): x = RMSNorm(h[r]) *
 * attn_norm; [q|k|v] = x W_qkv^T; RoPE on q and k at positions[r]. h: [n_rows][D] fp32;
 * positions: device [n_rows] (each < rope_rows); q: [n_rows][Hq][hd], k_fresh / v_fresh:
 * [n_rows][Hkv][hd] in the model dtype. */
akvs_status akvs_probe_qkv(const float *h, int32_t n_rows, const int32_t *positions,
                           const akvs_model_cfg *m, const akvs_layer_w *lw, const float *rope,
                           int32_t rope_rows, void *q, void *k_fresh, void *v_fresh, void *ws,
                           size_t ws_bytes, hipStream_t stream);

/* Per-unit offsets of one layer (Sec. 3.3 "Mean estimation"; Alg. 1):
 * mu_k[i] = (1/b_i) sum_{j in S_K,i} (k_fresh[fresh_row[j]] - Rot(s_i) deq(k_cached[j])),
 * mu_v likewise without rotation; 0 when b_i = 0 or with AKVS_F_NO_CORRECTION. With
 * AKVS_F_PRE_ROPE_OFFSETS each key term is first rotated back by -j (the offset is then
 * a pre-RoPE vector). Probe terms are summed in ascending position order in fp32. k_fresh / v_fresh: [rows][Hkv][hd]
 * model dtype; cache: one layer; mu_k, mu_v: [m][Hkv][hd] fp32. */
akvs_status akvs_chunk_offset(const void *k_fresh, const void *v_fresh, const int32_t *fresh_row,
                              const akvs_cache *cache, const akvs_reuse_cfg *cfg,
                              const int32_t *chunk_meta, const int32_t *probe_k,
                              const int32_t *probe_v, const akvs_model_cfg *m, const float *rope,
                              int32_t rope_rows, float *mu_k, float *mu_v, hipStream_t stream);

/* Corrected cache of one layer (Alg. 1 inner loop; Sec. 3.3 "AgentKVShift correction").
 * For a unit token j of unit i: k_corr[j] = k_fresh[fresh_row[j]] if j in S_K,i (any
 * recomputed j with AKVS_F_FRESH_IF_RECOMPUTED), else Rot(s_i) deq(k_cached[j]) +
 * w_k[j] mu_k[i] (w_k[j] Rot(j) mu_k[i] with AKVS_F_PRE_ROPE_OFFSETS); v_corr likewise
 * with S_V and no rotation. Query positions T_c..T-1
 * take their fresh rows. k_corr, v_corr: [T][Hkv][hd] model dtype (one layer). */
akvs_status akvs_apply_correction(const akvs_cache *cache, const float *mu_k, const float *mu_v,
                                  const float *w_k, const float *w_v, const uint8_t *flags,
                                  const void *k_fresh, const void *v_fresh,
                                  const int32_t *fresh_row, const akvs_reuse_cfg *cfg,
                                  const int32_t *chunk_meta, const akvs_model_cfg *m,
                                  const float *rope, int32_t rope_rows, void *k_corr,
                                  void *v_corr, hipStream_t stream);

/* Attention of sparse query rows over a full key range (Alg. 1 recompute of the probe
 * rows against the whole corrected context): row r at position positions[r] attends
 * to keys 0..positions[r] (< n_keys) with scores q.k/sqrt(hd), fp32 softmax, query
 * head h reading KV head h/(Hq/Hkv). q: [n_rows][Hq][hd]; k, v: [n_keys][Hkv][hd];
 * out: [n_rows][Hq*hd]; all model dtype. positions must be ascending. ws (may be NULL)
 * of ws_bytes >= akvs_attention_workspace_size lets the call split the key range and
 * merge the parts, as the reuse prefill does; a non-NULL ws that is too small is
 * AKVS_ENOSPACE. (Few rows over many keys run with 8 parts a tile in a smaller ws, as the
 * reuse calls do in theirs.) */
akvs_status akvs_sparse_query_attention(const void *q, const int32_t *positions, int32_t n_rows,
                                        const void *k, const void *v, int32_t n_keys,
                                        const akvs_model_cfg *m, void *out, void *ws,
                                        size_t ws_bytes, hipStream_t stream);

/* Rest of the probe rows' layer (Algorithm 1, "recompute fresh KV for S_K u S_V at layer
 * l": the fresh K/V of the next layer need these rows' hidden states carried through this
 * layer's attention output and MLP; Sec. 3.3): h += attn_out W_o^T;
 * x = RMSNorm(h) * mlp_norm; h += (silu(x W_gate^T) * (x W_up^T)) W_down^T.
 * h: [n_rows][D] fp32 (updated in place); attn_out: [n_rows][Hq*hd] model dtype. */
akvs_status akvs_probe_out_mlp(float *h, int32_t n_rows, const void *attn_out,
                               const akvs_model_cfg *m, const akvs_layer_w *lw, void *ws,
                               size_t ws_bytes, hipStream_t stream);

/* Group-64 quantiser of a cache (Sec. 4.5 composition with KV quantisation). For each
 * group of 64 head-dim elements:
 *   bits 2 / 4 (AKVS_U2G64 / AKVS_U4G64, asymmetric integer codes): zero = fp16(min),
 *     scale = fp16((max-min) / (2^bits - 1)) computed in fp32,
 *     code = clamp(rne((x - zero) / scale), 0, 2^bits - 1) (0 when scale == 0);
 *   bits 8 (AKVS_E4M3G64, FP8 E4M3 codes): scale = fp16(max|x| / 448) computed in fp32,
 *     zero = 0, code = E4M3 of clamp(x / scale, -448, 448) rounded half to even (OCP FP8
 *     E4M3: bias 7, no infinity, 448 the largest finite value; 0 when scale == 0).
 * x: [n_rows][hd] of x_dtype (F32 or BF16), hd a multiple of 64; codes:
 * [n_rows][hd*bits/8]; meta: [n_rows][hd/64][2] fp16 (scale, zero). */
akvs_status akvs_quantize_cache(const void *x, int32_t x_dtype, int32_t n_rows, int32_t head_dim,
                                int32_t bits, uint8_t *codes, void *meta, hipStream_t stream);

/* ---- whole-procedure entries -------------------------------------------------------- */

/* Reuse prefill (Algorithm 1 over all layers). tokens: device [T] ids (units in order,
 * then the query), each in [0, vocab). lw: host array of n_layers layer weight sets.
 * Layers before check_layer are computed for every token; from check_layer on only
 * R = probes u query is recomputed and every unit token takes its corrected state.
 * With AKVS_F_GIVEN_PROBES, out->probe_k / out->probe_v must hold the sets on entry. */
akvs_status akvs_reuse_prefill(const int32_t *tokens, const void *embed, const akvs_layer_w *lw,
                               const void *final_norm, const akvs_model_cfg *m,
                               const akvs_reuse_cfg *cfg, const akvs_cache *cache,
                               const akvs_reuse_out *out, void *ws, size_t ws_bytes,
                               hipStream_t stream);

/* Batched reuse prefill (the paper's batch axis, Sec. 4.4 / Table 3: B requests served
 * together). Request b is exactly the call akvs_reuse_prefill(tokens[b], ..., &cfgs[b],
 * &caches[b], &outs[b]) — its own units, query, unit caches, outputs and probe sets —
 * but from the check layer on the recomputed rows of all requests form one row block,
 * so every projection GEMM reads its weights once per layer for the whole batch;
 * offsets, correction and attention stay per request. tokens, cfgs, caches and outs are
 * host arrays of `batch` entries (device pointers inside, as for akvs_reuse_prefill).
 * Every cfg must use the same check_layer and AKVS_F_NO_PREFIX_RECOMPUTE setting
 * (AKVS_EINVAL otherwise). ws: akvs_batch_workspace_size bytes. */
akvs_status akvs_reuse_prefill_batch(const int32_t *const *tokens, int32_t batch,
                                     const void *embed, const akvs_layer_w *lw,
                                     const void *final_norm, const akvs_model_cfg *m,
                                     const akvs_reuse_cfg *cfgs, const akvs_cache *caches,
                                     const akvs_reuse_out *outs, void *ws, size_t ws_bytes,
                                     hipStream_t stream);
/* Workspace bytes of akvs_reuse_prefill_batch (0 for an invalid configuration). */
size_t akvs_batch_workspace_size(const akvs_model_cfg *m, const akvs_reuse_cfg *cfgs,
                                 int32_t batch);

/* Full prefill (the no-reuse baseline; also the standalone caching of a unit with
 * pos0 = 0, Sec. 3.1). tokens: device [n] ids at positions pos0..pos0+n-1. h_out:
 * [n][D] fp32 final-normed hidden states (may be NULL); k_out, v_out: [L][n][Hkv][hd]
 * model dtype (post-RoPE keys). */
akvs_status akvs_full_prefill(const int32_t *tokens, int32_t n_tokens, int32_t pos0,
                              const void *embed, const akvs_layer_w *lw, const void *final_norm,
                              const akvs_model_cfg *m, float *h_out, void *k_out, void *v_out,
                              void *ws, size_t ws_bytes, hipStream_t stream);

/* ---- first decode step over the corrected caches -------------------------------------
 * The consumer of a reuse prefill: the next token is predicted from the last final-normed
 * query row, then generated tokens run through every layer attending to the corrected
 * keys and values (Sec. 3.1: the reused states serve the generation that follows). The
 * output embedding w_out is [vocab][D] in the model dtype; NULL means tied to the input
 * embedding (as in the 3B-class decoders the paper evaluates). Greedy pick: the largest
 * logit, equal values resolved to the lowest index, -1 if no logit is a number. */

/* Workspace of akvs_decode_step with n_past cached tokens (also enough for akvs_lm_head
 * when n_past >= 0). 0 for an invalid model. */
size_t akvs_decode_workspace_size(const akvs_model_cfg *m, int32_t n_past);

/* logits[r][:] = h[r] . w_out^T and tokens[r] = greedy pick, r < n_rows. h: device
 * [n_rows][D] fp32 final-normed rows (e.g. the last row of h_query); logits (device
 * [n_rows][vocab] fp32) or tokens (device [n_rows]) may be NULL, not both. */
akvs_status akvs_lm_head(const float *h, int32_t n_rows, const void *w_out,
                         const akvs_model_cfg *m, float *logits, int32_t *tokens, void *ws,
                         size_t ws_bytes, hipStream_t stream);

/* One decode step: token (device [1]) at position n_past. k_cache, v_cache: device
 * [L][cache_rows][Hkv][hd] model dtype, rows 0..n_past-1 valid (e.g. the k_corr / v_corr
 * of a reuse prefill written with kv_rows = cache_rows); the step writes the token's
 * post-RoPE key and value to row n_past of every layer. Outputs logits (device [vocab]
 * fp32, may be NULL) and next_token (device [1], may be NULL). Errors: EINVAL for
 * n_past < 0 or cache_rows <= n_past, null or misaligned pointers; ENOSPACE. */
akvs_status akvs_decode_step(const int32_t *token, int32_t n_past, const void *embed,
                             const akvs_layer_w *lw, const void *final_norm, const void *w_out,
                             const akvs_model_cfg *m, void *k_cache, void *v_cache,
                             int32_t cache_rows, float *logits, int32_t *next_token, void *ws,
                             size_t ws_bytes, hipStream_t stream);

/* ---- decode step without allocation ---------------------------------------------------
 * For callers that cannot allocate device memory or pass a workspace: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc. akvs_decode_step_noalloc
 * is akvs_decode_step (same arguments, same kernels, identical results) with the workspace
 * taken from a device array inside the library of AKVS_NOALLOC_SCRATCH_BYTES bytes, which
 * every device that runs it holds until the process ends. The call itself allocates nothing
 * and frees nothing; its first call on a device looks up that device's array address.
 * Errors: AKVS_ENOSPACE when akvs_decode_workspace_size(m, n_past) exceeds
 * AKVS_NOALLOC_SCRATCH_BYTES (the attention partials grow with n_past: about 200K past
 * tokens for the 32B-class shape); AKVS_EINVAL when `stream` belongs to a device other
 * than the calling thread's current one; otherwise as akvs_decode_step. All calls on one
 * device share that device's array: calls that overlap in time on one device (on different
 * streams, or from several threads without ordering) race on it and give unspecified
 * results. Calls ordered on one stream are safe; the array keeps the last call's contents,
 * none of which a later call reads before writing it. */
#define AKVS_NOALLOC_SCRATCH_BYTES ((size_t)32 << 20)
akvs_status akvs_decode_step_noalloc(const int32_t *token, int32_t n_past, const void *embed,
                                     const akvs_layer_w *lw, const void *final_norm,
                                     const void *w_out, const akvs_model_cfg *m, void *k_cache,
                                     void *v_cache, int32_t cache_rows, float *logits,
                                     int32_t *next_token, hipStream_t stream);

/* ---- a batch over one shared context -----------------------------------------------------
 * Serving steps of several requests that continue from the same corrected caches: the new
 * tokens' queries and keys are normalised per head and rotated, their keys and values join
 * their requests' own caches, every row attends to the shared prefix and to its request's own
 * keys, the weight that each cached key received is summed, and the keys of least weight are
 * evicted. One layer per call (akvs_evict_cache: any number of sequences). */

/* Per-head RMS norms of queries and keys with the rotary map, for decoders that normalise
 * both per head (Sec. 4.1 evaluates Qwen3): x = x rsqrt(mean(x^2) + rms_eps) * norm over hd,
 * then the rotation at positions[r]; one rounding, at the end. Values are copied.
 * q: [n_rows][Hq][hd], k, v: [n_rows][Hkv][hd], model dtype, row r at r * ldq / ldk / ldv
 * elements (a packed projection output, or dense tensors; each ld * element size a multiple
 * of 16 bytes); q_norm, k_norm: [hd] model dtype, NULL: that side is not normalised;
 * positions: device [n_rows], each < rope_rows; kv_rows: device [n_rows] row of k_out / v_out
 * that takes row r (one outside [0, n_kv_rows), e.g. -1, is written nowhere; rows must be
 * distinct), NULL: row r, n_kv_rows >= n_rows then. q_out: [n_rows][Hq][hd]; k_out, v_out:
 * [n_kv_rows][Hkv][hd]; rows that no token names stay as they were. q_out may be q where
 * ldq = Hq * hd (k_out k and v_out v likewise, without kv_rows); outputs overlap nothing else.
 * v and v_out may both be NULL, k_out and v_out where n_kv_rows is 0. Errors: EINVAL (negative
 * sizes, null or misaligned pointers, strides shorter than a row or not of 16 bytes,
 * n_kv_rows < n_rows without kv_rows, overlaps), ESHAPE (too large), EHIP. */
akvs_status akvs_qk_norm_rope(const void *q, int64_t ldq, const void *k, int64_t ldk,
                              const void *v, int64_t ldv, int32_t n_rows,
                              const int32_t *positions, const void *q_norm, const void *k_norm,
                              const akvs_model_cfg *m, const float *rope, int32_t rope_rows,
                              const int32_t *kv_rows, int32_t n_kv_rows, void *q_out,
                              void *k_out, void *v_out, hipStream_t stream);

/* Workspace bytes of akvs_shared_attention and akvs_attention_weights over this batch; 0 for
 * an invalid one, or where neither needs any. */
size_t akvs_shared_workspace_size(const akvs_model_cfg *m, const akvs_shared_cfg *c);

/* Attention of a batch's rows over the shared prefix and each request's own keys, scores
 * q.k/sqrt(hd), softmax over both together. Scores, maxima, sums and lse are fp32. bf16 models
 * round the probabilities p to bf16 for their product with the values, and, where the keys are
 * split, a split's outputs to fp16 scaled by a power of two per row and head: together up to
 * about (2^-8 + 2^-11) sum p |v| beside the rounding of out itself. fp32 models round neither.
 * The prefix is read once for 128 (row, query head) pairs of a KV head (fp32 models: 16),
 * whichever requests they are of; contexts of a few hundred keys once for each request.
 * q: [n_rows][Hq][hd]; k_prefix, v_prefix: [P][Hkv][hd] (e.g. one layer of a reuse prefill's
 * k_corr / v_corr); k_own, v_own: [B][own_rows][Hkv][hd]; out: [n_rows][Hq][hd]; all model
 * dtype. lse (device [n_rows][Hq] fp32, may be NULL): natural log of the row's sum of
 * exp(score). A row that sees no key, or whose scores are all -inf, gets out 0 and lse -inf. Keys
 * past a row's last one are never part of its result, whatever they hold; rows from
 * row_start[B] on stay as they were.
 * out may be q; out, lse and ws overlap nothing else.
 * Errors: EINVAL (sizes, pointers, overlaps) / ESHAPE / ENOSPACE, EHIP. */
akvs_status akvs_shared_attention(const void *q, const akvs_shared_cfg *c, const void *k_prefix,
                                  const void *v_prefix, const void *k_own, const void *v_own,
                                  const akvs_model_cfg *m, void *out, float *lse, void *ws,
                                  size_t ws_bytes, hipStream_t stream);

/* Attention weight that each key received from a batch's rows, summed over the rows that see
 * it and the Hq/Hkv query heads of its KV head, added to what it had:
 * w[j] = w_prev[j] + sum_r sum_h exp(q.k_j/sqrt(hd) - lse[r][h]), fp32 sums in a fixed order.
 * q, lse: as akvs_shared_attention took and left them; w_prefix, w_prefix_prev: device
 * [Hkv][P] fp32; w_own, w_own_prev: [B][Hkv][own_rows] fp32 (keys past own_len keep what they
 * had). A w_*_prev may be its w_* itself, or NULL (0); w_prefix, w_own and ws overlap nothing
 * else. w_prefix or w_own may be NULL: that side is not formed (both: where there are no keys).
 * A row with lse = -inf gives nothing. Errors as above. */
akvs_status akvs_attention_weights(const void *q, const float *lse, const akvs_shared_cfg *c,
                                   const void *k_prefix, const void *k_own,
                                   const akvs_model_cfg *m, const float *w_prefix_prev,
                                   float *w_prefix, const float *w_own_prev, float *w_own,
                                   void *ws, size_t ws_bytes, hipStream_t stream);

/* Workspace bytes of akvs_evict_cache; 0 if invalid. It is needed where `keep` is NULL; with
 * `keep` it may be NULL or smaller, and lets the call split long sequences over blocks (the
 * same result). */
size_t akvs_evict_workspace_size(const akvs_model_cfg *m, const akvs_evict_cfg *c);

/* Eviction by accumulated weight: per sequence of n keys and per KV head, the first n_first
 * and the last n_recent keys and of the others those of largest weight (equal ones: the lower
 * index; a NaN counts as the smallest) are kept, min(n, n_keep) in all, in their order; keys
 * and values move to rows 0.. of k_out / v_out as they are (keys keep their rotation).
 * k, v: [S][src_rows][Hkv][hd] model dtype; weights: [S][Hkv][n_keys] fp32; keep (device
 * [S][Hkv][n_keep], may be NULL): indices of the kept keys, -1 past the last; k_out, v_out:
 * [S][dst_rows][Hkv][hd], rows past the kept ones stay as they were; k, v, k_out, v_out may all
 * be NULL (selection alone), some where there are no rows to move (src_rows = n_keys = 0);
 * weights_out (device [S][Hkv][dst_rows] fp32, may be NULL): the kept keys' weights, then 0;
 * lens_out (device [S], may be NULL, may be lens): keys kept. Outputs and ws overlap nothing
 * else.
 * Errors: EINVAL (sizes, pointers, overlaps) / ESHAPE / ENOSPACE, EHIP. */
akvs_status akvs_evict_cache(const void *k, const void *v, const float *weights,
                             const akvs_evict_cfg *c, const akvs_model_cfg *m, int32_t *keep,
                             void *k_out, void *v_out, float *weights_out, int32_t *lens_out,
                             void *ws, size_t ws_bytes, hipStream_t stream);

/* ---- decoding from four bits ----------------------------------------------------------------
 * Caches of many sequences in pages of 4-bit codes (the format of akvs_quantize_cache with bits
 * 4), which sequences may share, and products with weights in the same format. bf16 models only
 * (AKVS_EDTYPE). A sequence index, length or page outside its range is as if the sequence were
 * empty, cut or the page missing: nothing is read or written for it. */

/* Quantises a batch's new keys and values into their pages, with the codes and meta that
 * akvs_quantize_cache gives them (values past fp16's range are outside the format). k, v:
 * [n_rows][Hkv][hd] model dtype, row r at r * ldk / ldv elements (each ld * 2 bytes a multiple of
 * 16); pages that rows go to are named by one sequence of the batch only. Rows past row_start[B],
 * rows that are no key of their sequence (more rows than keys) and rows of a sequence that could not
 * grow by them (grown) go nowhere: without `grown` they would be taken for its last keys of before. Errors: EINVAL
 * (sizes, pointers, strides, overlaps) / EDTYPE / EUNSUPPORTED (page_rows) / ESHAPE, EHIP. */
akvs_status akvs_store_pages(const void *k, int64_t ldk, const void *v, int64_t ldv,
                             const akvs_paged_cfg *c, const akvs_pages *p,
                             const akvs_model_cfg *m, hipStream_t stream);

/* The other way: what the pages hold for a batch's rows (any keys at the end of each sequence, all
 * of them with n = len). k_out, v_out: [n_rows][Hkv][hd] of dtype (F32: scale * code + zero
 * exactly rounded; BF16), either may be NULL. Rows that are no key of their sequence, or whose page
 * is missing, are 0; rows past row_start[B] stay as they were. Errors as above. */
akvs_status akvs_load_pages(const akvs_paged_cfg *c, const akvs_pages *p, const akvs_model_cfg *m,
                            void *k_out, void *v_out, int32_t dtype, hipStream_t stream);

/* Workspace bytes of akvs_paged_attention over this batch; 0 for an invalid one, or where it
 * needs none. */
size_t akvs_paged_workspace_size(const akvs_model_cfg *m, const akvs_paged_cfg *c);

/* Attention of a batch's rows over their sequences' pages, scores q.k/sqrt(hd), softmax. q, out:
 * [n_rows][Hq][hd] model dtype; lse (device [n_rows][Hq] fp32, may be NULL): natural log of the
 * row's sum of exp(score). A row that sees no key, or whose scores are all -inf, gets out 0 and
 * lse -inf. Keys past a row's last one, and what their places in a page hold, are never part of its
 * result; rows past row_start[B] stay as they were. A missing page's keys and values count as 0
 * (with n_pages = 0 there are no keys).
 * Scores are formed of q and the codes in fp32 (rows_max * Hq / Hkv above 48: of q scaled into fp16
 * by a power of two, which is exact for elements down to 2^-24 of the row's largest). Probabilities
 * are rounded to fp16, with a value's scale or beside the value rounded to fp16 (fp32 where scale and
 * zero lead past fp16's range); sums, of parts of the keys too, and statistics are fp32: 65536 keys of
 * even weights lose no more than the bf16 result's own rounding. A query with an infinity may give NaN
 * in its own row.
 * out may be q; out, lse and ws overlap nothing else. Errors as above, ENOSPACE. */
akvs_status akvs_paged_attention(const void *q, const akvs_paged_cfg *c, const akvs_pages *p,
                                 const akvs_model_cfg *m, void *out, float *lse, void *ws,
                                 size_t ws_bytes, hipStream_t stream);

/* Sequences dst[i] (device [n], empty ones) become what src[i] are: they share all their pages,
 * the last one too. A pair is left out where an index is out of range, dst[i] is not empty, is
 * named as dst by an earlier pair, or is a source of the call. Errors: EINVAL / ESHAPE /
 * EUNSUPPORTED (page_rows), EHIP. */
akvs_status akvs_fork_pages(const akvs_page_table *t, int32_t n, const int32_t *src,
                            const int32_t *dst, hipStream_t stream);

/* Sequences seq[i] (device [n]; one named twice is one) end: their pages' refs are lowered, their
 * entries are -1 and their lengths 0. Errors as above. */
akvs_status akvs_free_pages(const akvs_page_table *t, int32_t n, const int32_t *seq,
                            hipStream_t stream);

/* Workspace bytes of akvs_grow_pages over n sequences and of akvs_compact_pages (n = 0). 0 if
 * invalid. */
size_t akvs_pages_workspace_size(const akvs_page_table *t, int32_t n);

/* Room for add[i] >= 0 more keys in sequences seq[i] (device [n] both), whose lengths grow by
 * that: pages of the lowest free numbers, sequence by sequence in order. A last page that has room
 * and is shared (ref > 1 before the call) is replaced by a page of the sequence's own, its first
 * new one: that page's contents are to be copied, as listed in move_src / move_dst (device [n]
 * int32 each, in order, -1 past the last; akvs_move_pages). served (device [n]): 1, or 0 for a
 * sequence that stays as it was: an index out of range or named earlier, add[i] < 0, more than
 * max_pages pages, or no free pages left (one that needs any follows one that could not be served);
 * grown has the same of every sequence named, of its first entry.
 * counts (device [2]): copies listed, pages taken. Outputs and ws overlap nothing else. Errors as
 * above, ENOSPACE. */
akvs_status akvs_grow_pages(const akvs_page_table *t, int32_t n, const int32_t *seq,
                            const int32_t *add, int32_t *served, int32_t *move_src,
                            int32_t *move_dst, int32_t *counts, void *ws, size_t ws_bytes,
                            hipStream_t stream);

/* The pages in use (ref > 0) move to the lowest numbers: of N in use, those from number N on take
 * the free numbers below N, in ascending order both. move_src, move_dst (device [n_pages] each, -1
 * past the last): whose contents go where (akvs_move_pages, before the tables are used again);
 * table_out, ref_out: the tables afterwards, may be t's own; counts (device [2]): moves, N.
 * Outputs and ws overlap nothing else. Errors as above. */
akvs_status akvs_compact_pages(const akvs_page_table *t, int32_t *table_out, int32_t *ref_out,
                               int32_t *move_src, int32_t *move_dst, int32_t *counts, void *ws,
                               size_t ws_bytes, hipStream_t stream);

/* Copies pages src[i] to pages dst[i] (device), i < min(*n_moves, max_moves) (n_moves: device,
 * NULL: max_moves of them), in n_layers layers, p being the first. Indices out of range are left
 * out; no page is both a source and a target, nor a target twice. Errors as above. */
akvs_status akvs_move_pages(const akvs_pages *p, int32_t n_layers, const akvs_model_cfg *m,
                            const int32_t *src, const int32_t *dst, int32_t max_moves,
                            const int32_t *n_moves, hipStream_t stream);

/* Workspace bytes that any akvs_w4_product of these sizes needs at most; 0 if invalid, or where none
 * does. (Those whose reduction is not cut need none.) */
size_t akvs_w4_workspace_size(int32_t n_rows, int32_t n_out, int32_t n_in);

/* Products of rows with 4-bit weights: (W x)[r][o] = sum_i x[r][i] (scale code + zero)[o][i],
 * fp32 sums, weights not rounded. x: [n_rows][n_in] of x_dtype (F32 or BF16), row r at r * ldx
 * elements (ldx * element size a multiple of 16); w, w_meta: n_out rows of n_in, a multiple of 64;
 * y: [n_rows][n_out] ([n_out / 2] with AKVS_W4_SWIGLU, n_out even) of y_dtype, row r at r * ldy.
 * resid (fp32, strides as y, may be y; y_dtype F32 and AKVS_W4_STORE only) or NULL. The weights
 * are read once for 64 rows (x in F32: 32). A row of x that holds an infinity, or
 * elements above 2^116, may give NaN. y and ws overlap nothing else. Errors: EINVAL (sizes, strides,
 * mode, pointers, overlaps) / EDTYPE / ESHAPE / ENOSPACE, EHIP. */
akvs_status akvs_w4_product(const void *x, int64_t ldx, int32_t x_dtype, int32_t n_rows,
                            const uint8_t *w, const void *w_meta, int32_t n_out, int32_t n_in,
                            int32_t mode, const float *resid, void *y, int64_t ldy,
                            int32_t y_dtype, void *ws, size_t ws_bytes, hipStream_t stream);

/* ---- kernel timing -------------------------------------------------------------------
 * akvs_profile_enable(mask): for every kernel class whose bit (1 << class) is set in
 * mask, the library brackets each launch of that class with a pair of HIP events
 * recorded on the launch stream and accumulates the number of launches and the summed
 * event time (0 disables). akvs_profile_read waits for the recorded events, returns the
 * class totals and clears that class. Process-wide state, meant for a single
 * benchmarking thread. */
enum {
  AKVS_K_GEMM = 0, AKVS_K_ATTENTION = 1, AKVS_K_CORRECTION = 2, AKVS_K_OFFSET = 3,
  AKVS_K_DIVERGENCE = 4, AKVS_K_SELECT = 5, AKVS_K_NORM = 6, AKVS_K_OTHER = 7,
  AKVS_K_GEMV = 8, AKVS_K_NCLASSES = 9
};
akvs_status akvs_profile_enable(int32_t class_mask);
akvs_status akvs_profile_read(int32_t kernel_class, int64_t *launches, double *total_ms);

/* ---- counter calibration ----------------------------------------------------------------
 * akvs_mfma_busy_loop: not part of the method; the reference point for hardware counters
 * of matrix-core use and for the MFMA rate the chip sustains. Launches n_blocks blocks of
 * 256 threads in which every wave issues iters (rounded up to even) x 8 independent
 * 32x32x16 bf16 MFMAs on random operands that change from one MFMA to the next, and
 * nothing else (the matrix cores of every SIMD it occupies stay busy), then writes one
 * fp32 per thread to out (device
 * [n_blocks * 256], caller-owned, 16-byte aligned). Asynchronous on stream. Errors:
 * EINVAL for negative sizes, a null or misaligned out (with n_blocks > 0); EHIP. */
akvs_status akvs_mfma_busy_loop(int32_t n_blocks, int32_t iters, float *out, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* AKVS_H */
