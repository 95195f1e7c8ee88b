"""Device-memory plumbing around libakvs: allocate outputs and workspaces with torch,
marshal the descriptors, call the C entry points on the current stream.

Nothing here computes any part of the method; every step runs in the library.
"""
from __future__ import annotations

import operator
from typing import Optional, Sequence

import torch

from . import akvs


class Engine:
    """A decoder (weights on one device) and the calls of the library over it."""

    def __init__(self, shape, weights: dict, device="cuda"):
        self.shape = shape
        self.device = torch.device(device)
        self.weights = weights
        self.n_layers = len(weights["layers"])
        self.m = akvs.model_cfg(shape, n_layers=self.n_layers)
        self.layers = akvs.layer_array(weights)
        self.dtype = torch.float32 if self.m.dtype == akvs.AKVS_F32 else torch.bfloat16
        self._ws = None

    def workspace(self, nbytes: int) -> torch.Tensor:
        """The engine's workspace, grown when a call needs more. A grown workspace replaces
        the old tensor; a captured graph keeps its own reference to the tensor it was
        captured with (see ReuseGraph), so replays never run on freed memory."""
        if self._ws is None or self._ws.numel() < nbytes:
            self._ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
        return self._ws

    def full_prefill(self, tokens: torch.Tensor, pos0: int = 0, want_h: bool = True):
        n = int(tokens.numel())
        sh = self.shape
        L = self.n_layers
        k = torch.empty((L, n, sh.n_kv_heads, sh.head_dim), dtype=self.dtype, device=self.device)
        v = torch.empty_like(k)
        h = torch.empty((n, sh.d_model), dtype=torch.float32, device=self.device) if want_h else None
        ws = self.workspace(akvs.akvs_workspace_size(self.m, None, n))
        akvs.akvs_full_prefill(tokens, n, pos0, self.weights["embed"], self.layers,
                               self.weights["final_norm"], self.m, h, k, v, ws)
        return h, k, v

    def lm_head(self, h: torch.Tensor, w_out: Optional[torch.Tensor] = None):
        """Logits [n][vocab] fp32 and greedy tokens [n] of final-normed rows h [n][D]
        (w_out None: tied to the input embedding)."""
        n = int(h.shape[0])
        logits = torch.empty((n, self.shape.vocab), dtype=torch.float32, device=self.device)
        toks = torch.empty(n, dtype=torch.int32, device=self.device)
        ws = self.workspace(akvs.akvs_decode_workspace_size(self.m, 0))
        akvs.akvs_lm_head(h.contiguous(), n, w_out if w_out is not None else self.weights["embed"],
                          self.m, logits, toks, ws)
        return logits, toks

    def decode_step(self, token: torch.Tensor, n_past: int, k_cache: torch.Tensor,
                    v_cache: torch.Tensor, w_out: Optional[torch.Tensor] = None, logits=None,
                    next_token=None):
        """One decode step of `token` (device int32 [1]) at position n_past over caches
        [L][cache_rows][Hkv][hd] (rows < n_past valid; row n_past is written). Returns
        (logits [vocab] fp32, next token [1] int32)."""
        if logits is None:
            logits = torch.empty(self.shape.vocab, dtype=torch.float32, device=self.device)
        if next_token is None:
            next_token = torch.empty(1, dtype=torch.int32, device=self.device)
        ws = self.workspace(akvs.akvs_decode_workspace_size(self.m, n_past))
        akvs.akvs_decode_step(token, n_past, self.weights["embed"], self.layers,
                              self.weights["final_norm"], w_out, self.m, k_cache, v_cache,
                              int(k_cache.shape[1]), logits, next_token, ws)
        return logits, next_token

    def cache_units(self, tokens: torch.Tensor, chunk_lens: Sequence[int]):
        """Standalone per-unit caches: each unit prefilled alone at position 0, laid out
        [L][T_c][Hkv][hd] with the units back to back."""
        sh = self.shape
        tc = int(sum(chunk_lens))
        kc = torch.empty((self.n_layers, tc, sh.n_kv_heads, sh.head_dim), dtype=self.dtype,
                         device=self.device)
        vc = torch.empty_like(kc)
        s = 0
        for n in chunk_lens:
            _, k, v = self.full_prefill(tokens[s:s + n], 0, want_h=False)
            kc[:, s:s + n].copy_(k)
            vc[:, s:s + n].copy_(v)
            s += n
        return kc, vc

    # ---- a batch over one shared context ----------------------------------------------------

    def _need(self, name: str, x, shape, dtype=None):
        """A contiguous tensor of this shape (None: any size) and type on this engine's device."""
        dtype = self.dtype if dtype is None else dtype
        ok = x.dtype == dtype and x.dim() == len(shape) and x.is_contiguous() and all(
            a == b for a, b in zip(x.shape, shape) if b is not None)
        if not ok or x.device.type != self.device.type:
            raise ValueError(f"{name}: need a contiguous {dtype} tensor "
                             f"[{']['.join('n' if b is None else str(b) for b in shape)}] on "
                             f"{self.device.type}, got {x.dtype} {tuple(x.shape)} on {x.device.type}")
        self._here(name, x)
        return x

    def _here(self, name: str, x):
        """Calls run on the current device's current stream: tensors of another are refused."""
        if x.is_cuda and x.device.index != torch.cuda.current_device():
            raise ValueError(f"{name} is on {x.device}, the current device is "
                             f"cuda:{torch.cuda.current_device()}")

    def _scratch(self, nbytes: int):
        """Workspace of one call over a shared context, from torch's pool of the current stream
        (or of the graph under capture): calls on two streams and captured graphs share none."""
        if nbytes == 0:
            return None
        return torch.empty(nbytes, dtype=torch.uint8, device=self.device)

    def qk_norm_rope(self, q, k, v, positions, q_norm, k_norm, rope, k_cache=None, v_cache=None,
                     kv_rows=None, q_out=None):
        """Per-head norms and rotation of new tokens' queries [n][Hq*hd] and keys [n][Hkv*hd]
        (columns of a packed projection, or dense), their values copied: queries to q_out
        [n][Hq][hd], keys and values to the rows kv_rows (int32 [n]) of k_cache / v_cache
        [rows][Hkv][hd], or, without caches, to new tensors row by row. q_norm / k_norm [hd] or
        None; rope: akvs_rope_table output. Returns (q_out, k, v)."""
        sh, n = self.shape, int(q.shape[0])
        for name, x, heads in (("q", q, sh.n_q_heads), ("k", k, sh.n_kv_heads),
                               ("v", v, sh.n_kv_heads)):
            if x.dtype != self.dtype or x.device.type != self.device.type or x.shape[0] != n or (
                    n and x[0].numel() != heads * sh.head_dim):
                raise ValueError(f"{name}: need {n} {self.dtype} rows of {heads * sh.head_dim}")
            self._here(name, x)
        self._need("positions", positions, (n,), torch.int32)
        for name, x in (("q_norm", q_norm), ("k_norm", k_norm)):
            if x is not None:
                self._need(name, x, (sh.head_dim,))
        self._need("rope", rope, (None, sh.head_dim // 2, 2), torch.float32)
        if (k_cache is None) != (v_cache is None) or (k_cache is None and kv_rows is not None):
            raise ValueError("k_cache, v_cache and kv_rows go together")
        if k_cache is None:
            k_cache = torch.empty((n, sh.n_kv_heads, sh.head_dim), dtype=self.dtype,
                                  device=self.device)
            v_cache = torch.empty_like(k_cache)
        self._need("k_cache", k_cache, (None, sh.n_kv_heads, sh.head_dim))
        self._need("v_cache", v_cache, tuple(k_cache.shape))
        if kv_rows is not None:
            self._need("kv_rows", kv_rows, (n,), torch.int32)
        if q_out is None:
            q_out = torch.empty((n, sh.n_q_heads, sh.head_dim), dtype=self.dtype,
                                device=self.device)
        self._need("q_out", q_out, (n, sh.n_q_heads, sh.head_dim))
        akvs.akvs_qk_norm_rope(q, k, v, n, positions, q_norm, k_norm, self.m, rope,
                               int(rope.shape[0]), kv_rows, int(k_cache.shape[0]), q_out, k_cache,
                               v_cache)
        return q_out, k_cache, v_cache

    def _ints_of(self, values, keep=False):
        """An int32 tensor of Python ints for calls on the current stream, without a wait for the
        device: through pinned memory, which torch keeps until the copy is done (a captured copy would
        read it at every replay). keep: for later calls on any stream, after a wait for the copy."""
        cuda = self.device.type == "cuda"
        if cuda and torch.cuda.is_current_stream_capturing():
            raise ValueError("a call under capture takes device tensors, not lists")
        x = torch.tensor(values, dtype=torch.int32, pin_memory=cuda)
        return x.to(self.device, non_blocking=not keep) if cuda else x

    def _row_start(self, n, row_start, rows_max, keep=False):
        """A row_start that is no tensor is checked, gives rows_max and is copied to the device."""
        if row_start is not None and not torch.is_tensor(row_start):
            at = [operator.index(x) for x in row_start]
            rows = [b - a for a, b in zip(at, at[1:])]
            if not rows or at[0] != 0 or min(rows) < 0 or at[-1] > n:
                raise ValueError(f"row_start: need ascending rows from 0 to at most {n}")
            if rows_max is not None and max(rows) > rows_max:
                raise ValueError(f"row_start holds a request of {max(rows)} rows, rows_max is {rows_max}")
            rows_max = max(rows)
            row_start = self._ints_of(at, keep)
        return row_start, rows_max

    def _shared(self, q, k_prefix, k_own, own_len, row_start, rows_max):
        """The batch that these tensors describe."""
        sh, n = self.shape, int(q.shape[0])
        self._need("q", q, (n, sh.n_q_heads, sh.head_dim))
        self._need("k_prefix", k_prefix, (None, sh.n_kv_heads, sh.head_dim))
        cap = 0
        if k_own is not None:
            self._need("k_own", k_own, (None, None, sh.n_kv_heads, sh.head_dim))
            cap = int(k_own.shape[1])
        row_start, rows_max = self._row_start(n, row_start, rows_max)
        if row_start is not None:
            self._need("row_start", row_start, (None,), torch.int32)
            B = int(row_start.numel()) - 1
        elif k_own is not None:
            B = int(k_own.shape[0])
        else:
            B = 1
        if k_own is not None and int(k_own.shape[0]) != B:
            raise ValueError(f"k_own holds {int(k_own.shape[0])} requests, row_start {B}")
        if cap:
            if own_len is None:
                raise ValueError("k_own needs own_len")
            self._need("own_len", own_len, (B,), torch.int32)
        if rows_max is None:
            if row_start is None and n % max(B, 1):
                raise ValueError(f"{n} rows of {B} requests need row_start")
            rows_max = n if row_start is not None else n // max(B, 1)
        return akvs.shared_cfg(B, n, max(int(rows_max), 1), int(k_prefix.shape[0]), cap, row_start,
                               own_len if cap else None)

    def shared_attention(self, q, k_prefix, v_prefix, k_own=None, v_own=None, own_len=None,
                         row_start=None, rows_max=None, out=None, lse=None):
        """Attention of a batch's rows q [n][Hq][hd] over a shared prefix [P][Hkv][hd] (one layer)
        and each request's own keys [B][rows][Hkv][hd], the first own_len (int32 [B]) of them,
        which end with the rows' own. row_start (B + 1 of them): the requests' rows (None: equally
        many each), a sequence of ints, or (as under capture) an int32 tensor, then with rows_max,
        the most of one request: without it each request is planned for all rows (768 rows of 256
        requests over 2000 keys of 28/4 heads 107 us, 55 with it), and many requests of many rows
        are refused. Returns (out, lse)."""
        c = self._shared(q, k_prefix, k_own, own_len, row_start, rows_max)
        self._need("v_prefix", v_prefix, tuple(k_prefix.shape))
        if (k_own is None) != (v_own is None):
            raise ValueError("k_own and v_own go together")
        if v_own is not None:
            self._need("v_own", v_own, tuple(k_own.shape))
        if out is None:
            out = torch.empty_like(q)
        if lse is None:
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device=self.device)
        self._need("out", out, tuple(q.shape))
        self._need("lse", lse, tuple(q.shape[:2]), torch.float32)
        ws = self._scratch(akvs.akvs_shared_workspace_size(self.m, c))
        akvs.akvs_shared_attention(q, c, k_prefix, v_prefix, k_own, v_own, self.m, out, lse, ws)
        return out, lse

    def attention_weights(self, q, lse, k_prefix, k_own=None, own_len=None, row_start=None,
                          rows_max=None, w_prefix=None, w_own=None):
        """Adds the attention weights that the rows of a shared_attention call gave its keys to
        w_prefix [Hkv][P] and (with k_own) w_own [B][Hkv][rows], fp32, made from 0 where they are
        None; row_start and rows_max as there. Returns (w_prefix, w_own)."""
        c = self._shared(q, k_prefix, k_own, own_len, row_start, rows_max)
        self._need("lse", lse, tuple(q.shape[:2]), torch.float32)
        hkv = self.shape.n_kv_heads
        shapes = [(hkv, c.prefix_len), (c.n_req, hkv, c.own_rows) if k_own is not None else None]
        prev, w = [w_prefix, w_own], [w_prefix, w_own]
        for i, shape in enumerate(shapes):
            if w[i] is None and shape is not None:
                w[i] = torch.empty(shape, dtype=torch.float32, device=self.device)
            elif w[i] is not None:
                if shape is None:
                    raise ValueError("w_own needs k_own")
                self._need(("w_prefix", "w_own")[i], w[i], shape, torch.float32)
        ws = self._scratch(akvs.akvs_shared_workspace_size(self.m, c))
        akvs.akvs_attention_weights(q, lse, c, k_prefix, k_own, self.m, prev[0], w[0], prev[1],
                                    w[1], ws)
        return w[0], w[1]

    def evict_cache(self, k, v, weights, n_keep: int, n_first: int = 0, n_recent: int = 0,
                    lens=None, dst_rows: int = 0):
        """Caches [S][rows][Hkv][hd] cut to n_keep keys per sequence and KV head by weights
        [S][Hkv][n]: the first n_first, the last n_recent and those of largest weight. lens
        (int32 [S]): keys per sequence (None: n). The new caches have dst_rows (0: n_keep) rows,
        zero past the kept ones. Returns (keep, k, v, weights, lens)."""
        sh = self.shape
        self._need("weights", weights, (None, sh.n_kv_heads, None), torch.float32)
        S, n = int(weights.shape[0]), int(weights.shape[2])
        self._need("k", k, (S, None, sh.n_kv_heads, sh.head_dim))
        self._need("v", v, tuple(k.shape))
        if int(k.shape[1]) < n:
            raise ValueError(f"k holds {int(k.shape[1])} rows of {n} keys")
        if lens is not None:
            self._need("lens", lens, (S,), torch.int32)
        c = akvs.evict_cfg(S, n, n_keep, n_first, n_recent, int(k.shape[1]), dst_rows, lens)
        rows, dev = max(dst_rows, n_keep), self.device
        keep = torch.empty((S, sh.n_kv_heads, n_keep), dtype=torch.int32, device=dev)
        k_out = torch.empty((S, rows, sh.n_kv_heads, sh.head_dim), dtype=self.dtype, device=dev)
        v_out = torch.empty_like(k_out)
        filled = min(n, n_keep) if lens is None else 0  # (rows that every sequence fills)
        k_out[:, filled:].zero_()
        v_out[:, filled:].zero_()
        w_out = torch.empty((S, sh.n_kv_heads, rows), dtype=torch.float32, device=dev)
        lens_out = torch.empty(S, dtype=torch.int32, device=dev)
        ws = self._scratch(akvs.akvs_evict_workspace_size(self.m, c))
        akvs.akvs_evict_cache(k, v, weights, c, self.m, keep, k_out, v_out, w_out, lens_out, ws)
        return keep, k_out, v_out, w_out, lens_out

    def w4_product(self, x, codes, meta, swiglu: bool = False, resid=None, y=None, y_dtype=None):
        """x [rows][n_in] (rows may lie apart) times 4-bit weights (quantize_weight), to y
        [rows][n_out], or with swiglu silu(gate) * up [rows][n_out / 2] of weights whose first half
        of rows is the gate's; resid (fp32) is added, y may be resid. A y that is not given is
        made, of y_dtype (the engine's; fp32 with resid). Returns y."""
        self._need("codes", codes, (None, None), torch.uint8)
        n_out, n_in = int(codes.shape[0]), 2 * int(codes.shape[1])
        self._need("meta", meta, (n_out, n_in // 64, 2), torch.float16)
        if x.dim() != 2:
            raise ValueError("x: need [rows][n_in]")
        if resid is not None and (swiglu or (y_dtype if y is None else y.dtype) not in (
                None, torch.float32)):
            raise ValueError("resid goes with an fp32 y, without swiglu")
        if y is None:
            if y_dtype is None:
                y_dtype = torch.float32 if resid is not None else self.dtype
            y = torch.empty((x.shape[0], n_out // 2 if swiglu else n_out), dtype=y_dtype,
                            device=self.device)
        for name, t in (("x", x), ("y", y), ("resid", resid)):
            if t is not None:
                if t.device.type != self.device.type:
                    raise ValueError(f"{name} is on {t.device}, not on {self.device.type}")
                self._here(name, t)
        ws = self._scratch(akvs.akvs_w4_workspace_size(int(x.shape[0]), n_out, n_in))
        akvs.akvs_w4_product(x, codes, meta, y,
                             akvs.AKVS_W4_SWIGLU if swiglu else akvs.AKVS_W4_STORE, resid, ws)
        return y

    def reuse_prefill(self, tokens: torch.Tensor, chunk_lens: Sequence[int], query_len: int,
                      k_cache: torch.Tensor, v_cache: torch.Tensor, refresh=(1, 5),
                      check_layer: int = 1, flags: int = 0, k_meta=None, v_meta=None,
                      cache_dtype: Optional[int] = None, given_probes=None, outputs=None,
                      kv_rows: int = 0, refresh_v=None):
        """Run the reuse prefill. Returns a dict of device tensors (h_query, k_corr, v_corr,
        probe_k, probe_v, d_k, d_v, rows, n_rows). `outputs` may pass a previous result
        dict to reuse its buffers. kv_rows > T sizes k_corr / v_corr [L][kv_rows][Hkv][hd]
        (rows T.. left for decode steps). refresh_v: the value side's own ratio."""
        sh = self.shape
        cfg = akvs.reuse_cfg(chunk_lens, query_len, refresh, check_layer, flags, refresh_v)
        _, (tc, sum_b, row_cap, t_all, sum_bv) = akvs.akvs_chunk_meta(cfg)
        if outputs is None:
            dev = self.device
            outputs = {
                "h_query": torch.empty((query_len, sh.d_model), dtype=torch.float32, device=dev),
                "k_corr": torch.empty((self.n_layers, max(kv_rows, t_all), sh.n_kv_heads,
                                       sh.head_dim), dtype=self.dtype, device=dev),
                "probe_k": torch.empty(max(sum_b, 1), dtype=torch.int32, device=dev),
                "probe_v": torch.empty(max(sum_bv, 1), dtype=torch.int32, device=dev),
                "d_k": torch.empty(tc, dtype=torch.float32, device=dev),
                "d_v": torch.empty(tc, dtype=torch.float32, device=dev),
                "rows": torch.empty(t_all, dtype=torch.int32, device=dev),
                "n_rows": torch.empty(1, dtype=torch.int32, device=dev),
            }
            outputs["v_corr"] = torch.empty_like(outputs["k_corr"])
        if given_probes is not None:
            outputs["probe_k"][:sum_b].copy_(given_probes[0])
            outputs["probe_v"][:sum_bv].copy_(given_probes[1])
        o = outputs
        out = akvs.ReuseOut(*(akvs.ptr(o[k]) for k in ("h_query", "k_corr", "v_corr", "probe_k",
                                                       "probe_v", "d_k", "d_v", "rows", "n_rows")),
                            int(o["k_corr"].shape[1]))
        cache = akvs.cache_struct(k_cache, v_cache, k_meta, v_meta,
                                  cache_dtype if cache_dtype is not None else akvs.dtype_code(k_cache))
        ws = self.workspace(akvs.akvs_workspace_size(self.m, cfg))
        akvs.akvs_reuse_prefill(tokens, self.weights["embed"], self.layers,
                                self.weights["final_norm"], self.m, cfg, cache, out, ws)
        outputs["_sum_b"] = sum_b
        outputs["_sum_b_v"] = sum_bv
        return outputs


def _reuse_outputs(engine, query_len, tc, sum_b, t_all, sum_bv=None):
    sh, dev = engine.shape, engine.device
    out = {
        "h_query": torch.empty((query_len, sh.d_model), dtype=torch.float32, device=dev),
        "k_corr": torch.empty((engine.n_layers, t_all, sh.n_kv_heads, sh.head_dim),
                              dtype=engine.dtype, device=dev),
        "probe_k": torch.empty(max(sum_b, 1), dtype=torch.int32, device=dev),
        "probe_v": torch.empty(max(sum_b if sum_bv is None else sum_bv, 1), dtype=torch.int32,
                               device=dev),
        "d_k": torch.empty(tc, dtype=torch.float32, device=dev),
        "d_v": torch.empty(tc, dtype=torch.float32, device=dev),
        "rows": torch.empty(t_all, dtype=torch.int32, device=dev),
        "n_rows": torch.empty(1, dtype=torch.int32, device=dev),
    }
    out["v_corr"] = torch.empty_like(out["k_corr"])
    out["_sum_b"] = sum_b
    out["_sum_b_v"] = sum_b if sum_bv is None else sum_bv
    return out


def reuse_prefill_batch(engine: Engine, requests, refresh=(1, 5), check_layer: int = 1,
                        flags: int = 0, outputs=None):
    """Batched reuse prefill (akvs_reuse_prefill_batch). `requests`: list of dicts with
    tokens, chunk_lens, query_len, k_cache, v_cache (and optional k_meta, v_meta,
    cache_dtype). Returns one output dict per request (as Engine.reuse_prefill);
    `outputs` may pass a previous result list to reuse its buffers."""
    cfgs, caches, outs = [], [], []
    if outputs is None:
        outputs = []
        for r in requests:
            cfg = akvs.reuse_cfg(r["chunk_lens"], r["query_len"], refresh, check_layer, flags)
            _, (tc, sum_b, _, t_all, sum_bv) = akvs.akvs_chunk_meta(cfg)
            outputs.append(_reuse_outputs(engine, r["query_len"], tc, sum_b, t_all, sum_bv))
    for r, o in zip(requests, outputs):
        cfgs.append(akvs.reuse_cfg(r["chunk_lens"], r["query_len"], refresh, check_layer, flags))
        dt = r.get("cache_dtype")
        caches.append(akvs.cache_struct(r["k_cache"], r["v_cache"], r.get("k_meta"), r.get("v_meta"),
                                        dt if dt is not None else akvs.dtype_code(r["k_cache"])))
        outs.append(akvs.ReuseOut(*(akvs.ptr(o[k]) for k in ("h_query", "k_corr", "v_corr",
                                                            "probe_k", "probe_v", "d_k", "d_v",
                                                            "rows", "n_rows"))))
    ca, cc, co = akvs.batch_arrays(cfgs, caches, outs)
    ws = engine.workspace(akvs.akvs_batch_workspace_size(engine.m, ca, len(requests)))
    akvs.akvs_reuse_prefill_batch([r["tokens"] for r in requests], engine.weights["embed"],
                                  engine.layers, engine.weights["final_norm"], engine.m, ca, cc,
                                  co, ws)
    return outputs


def cache_dtype_for_bits(bits: int) -> int:
    """Cache dtype code of a group-64 format: 4 / 2-bit integer or 8-bit FP8 E4M3."""
    return {4: akvs.AKVS_U4G64, 2: akvs.AKVS_U2G64, 8: akvs.AKVS_E4M3G64}[bits]


def quantize_cache(x: torch.Tensor, bits: int):
    """Group-64 quantised copy of a cache [..][hd] (codes uint8, meta fp16 (scale, zero));
    bits 4 / 2: integer codes, 8: FP8 E4M3 codes."""
    hd = x.shape[-1]
    rows = x.numel() // hd
    codes = torch.empty(x.shape[:-1] + (hd * bits // 8,), dtype=torch.uint8, device=x.device)
    meta = torch.empty(x.shape[:-1] + (hd // 64, 2), dtype=torch.float16, device=x.device)
    akvs.akvs_quantize_cache(x.contiguous(), rows, hd, bits, codes, meta)
    return codes, meta


def quantize_weight(w: torch.Tensor):
    """4-bit copy of a weight [n_out][n_in] (n_in a multiple of 64) for Engine.w4_product:
    codes uint8 [n_out][n_in / 2], meta fp16 [n_out][n_in / 64][2] (scale, zero)."""
    if w.dim() != 2 or w.shape[1] % 64:
        raise ValueError(f"w: need [n_out][n_in], n_in a multiple of 64, got {tuple(w.shape)}")
    return quantize_cache(w, 4)


class PagedCache:
    """Keys and values of many sequences, in pages of 4-bit codes that sequences may share: pools
    of all the engine's layers and one table of pages (akvs_pages, akvs_page_table). Everything is
    allocated here, once: the methods that follow run on the current stream without a host
    synchronisation and can be captured, but for a batch of ints, which may be used on any stream and
    waits for their copy. Sequences (`seq`, `src`, `dst`) are given as ints, which are checked and
    copied to the device, or (as under capture) as an int32 tensor, whose entries out of range the
    device leaves out."""

    def __init__(self, engine: Engine, n_seq: int, max_len: int, n_pages: int, page_rows: int = 64):
        if min(n_seq, max_len) < 1 or n_pages < 0 or page_rows not in (16, 32, 64, 128, 256):
            raise ValueError("need n_seq, max_len >= 1, n_pages >= 0 and pages of 16 to 256 rows")
        sh, dev = engine.shape, engine.device
        self.engine, self.page_rows, self.n_seq = engine, page_rows, n_seq
        max_pages = -(-max_len // page_rows)
        self.max_len = max_pages * page_rows  # keys a sequence can have
        rows = (engine.n_layers, n_pages, sh.n_kv_heads, page_rows)
        self.k, self.v = (torch.zeros(rows + (sh.head_dim // 2,), dtype=torch.uint8, device=dev)
                          for _ in range(2))
        self.k_meta, self.v_meta = (torch.zeros(rows + (sh.head_dim // 64, 2), dtype=torch.float16,
                                                device=dev) for _ in range(2))
        self.table = torch.full((n_seq, max_pages), -1, dtype=torch.int32, device=dev)
        self.len = torch.zeros(n_seq, dtype=torch.int32, device=dev)
        self.ref = torch.zeros(n_pages, dtype=torch.int32, device=dev)
        self.grown = torch.ones(n_seq, dtype=torch.int32, device=dev)
        self.t = akvs.page_table(self.table, self.len, self.ref, page_rows, self.grown)
        self.layers = [akvs.pages(*x) for x in zip(self.k, self.v, self.k_meta, self.v_meta)]

    def _layer(self, layer):
        if not 0 <= layer < len(self.layers):
            raise ValueError(f"layer {layer} of {len(self.layers)}")
        self.engine._here("the cache", self.table)
        return self.layers[layer]

    def _seq(self, name, seq, keep=False):
        if not torch.is_tensor(seq):
            seq = [operator.index(x) for x in seq]
            if any(not 0 <= x < self.n_seq for x in seq):
                raise ValueError(f"{name}: need sequences of 0 to {self.n_seq - 1}")
            seq = self.engine._ints_of(seq, keep)
        self.engine._here("the cache", self.table)
        return self.engine._need(name, seq, (None,), torch.int32)

    def _ints(self, n):
        return torch.empty(n, dtype=torch.int32, device=self.engine.device)

    def batch(self, n_rows: int, seq=None, row_start=None, rows_max=None, max_len=None):
        """A batch of n_rows new or last rows of sequences seq (None: of all, in order), request
        by request; row_start and rows_max as in Engine.shared_attention. max_len: the most keys
        that a sequence of the batch has when it runs (None: what the cache has room for), which
        calls are planned for; longer sequences are cut to it. It stays valid while the sequences
        grow within it."""
        eng = self.engine
        if max_len is None:
            max_len = self.max_len
        if not 0 <= max_len <= self.max_len:
            raise ValueError(f"max_len {max_len} outside 0 to {self.max_len}")
        row_start, rows_max = eng._row_start(n_rows, row_start, rows_max, keep=True)
        if seq is not None:
            seq = self._seq("seq", seq, keep=True)
            B = int(seq.numel())
        else:
            B = self.n_seq if row_start is None else int(row_start.numel()) - 1
        if B < 1:
            raise ValueError("a batch of no request")
        if row_start is not None:
            eng._need("row_start", row_start, (B + 1,), torch.int32)
        elif n_rows % B:
            raise ValueError(f"{n_rows} rows of {B} requests need row_start")
        if rows_max is None:
            rows_max = n_rows if row_start is not None else n_rows // B
        return akvs.paged_cfg(B, n_rows, max(int(rows_max), 1), self.len, self.table, max_len,
                              row_start, seq, self.grown)

    def store(self, layer: int, k, v, batch):
        """New keys and values [rows][Hkv*hd] (columns of a packed projection, or dense
        [rows][Hkv][hd]) of a batch, whose sequences have grown by them (grow), into one layer's
        pages. A sequence that its last grow could not serve gets none of them: it stays as it was,
        also under capture. Sequences of the batch must not share the pages that the rows go to:
        pages that grow gave them are their own."""
        sh, eng = self.engine.shape, self.engine
        p = self._layer(layer)
        for name, x in (("k", k), ("v", v)):
            if x.dtype != eng.dtype or x.device.type != eng.device.type or (
                    int(x.shape[0]) != batch.n_rows or
                    (batch.n_rows and x[0].numel() != sh.n_kv_heads * sh.head_dim)):
                raise ValueError(f"{name}: need {batch.n_rows} {eng.dtype} rows of "
                                 f"{sh.n_kv_heads * sh.head_dim}")
            eng._here(name, x)
        akvs.akvs_store_pages(k, v, batch, p, eng.m)

    def load(self, layer: int, batch, dtype=None):
        """What one layer's pages hold for a batch's rows, the last keys of its sequences: (k, v)
        [rows][Hkv][hd] of dtype (the engine's; torch.float32: scale * code + zero). Rows of no
        request are 0."""
        sh, eng = self.engine.shape, self.engine
        p = self._layer(layer)
        k = torch.zeros((batch.n_rows, sh.n_kv_heads, sh.head_dim), dtype=dtype or eng.dtype,
                        device=eng.device)
        v = torch.zeros_like(k)
        akvs.akvs_load_pages(batch, p, eng.m, k, v)
        return k, v

    def attention(self, layer: int, q, batch, out=None, lse=None):
        """Attention of a batch's rows q [rows][Hq][hd] over their sequences' keys in one layer,
        each row up to its own key. out may be q. Returns (out, lse)."""
        sh, eng = self.engine.shape, self.engine
        p = self._layer(layer)
        eng._need("q", q, (batch.n_rows, sh.n_q_heads, sh.head_dim))
        if out is None:
            out = torch.empty_like(q)
        if lse is None:
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device=eng.device)
        eng._need("out", out, tuple(q.shape))
        eng._need("lse", lse, tuple(q.shape[:2]), torch.float32)
        ws = eng._scratch(akvs.akvs_paged_workspace_size(eng.m, batch))
        akvs.akvs_paged_attention(q, batch, p, eng.m, out, lse, ws)
        return out, lse

    def fork(self, src, dst):
        """Empty sequences dst become what src are: they share all pages, until one grows."""
        src, dst = self._seq("src", src), self._seq("dst", dst)
        if src.numel() != dst.numel():
            raise ValueError(f"{src.numel()} sources of {dst.numel()} sequences")
        akvs.akvs_fork_pages(self.t, src, dst)

    def free(self, seq):
        """Sequences end; pages that no other has are free."""
        akvs.akvs_free_pages(self.t, self._seq("seq", seq))

    def grow(self, seq, add):
        """Room for add keys more (an int for all, ints, or an int32 tensor) in every sequence of
        seq, with a copy, in all layers, of a last page that is shared. Returns served (int32 per
        sequence: 1, or 0 where there is no room and the sequence stays as it was, through the
        batch's store too, until another grow serves it)."""
        seq = self._seq("seq", seq)
        n, eng = int(seq.numel()), self.engine
        if not torch.is_tensor(add):
            each = hasattr(add, "__len__")
            add = [operator.index(x) for x in (add if each else [add])]
            if any(x < 0 for x in add):
                raise ValueError("add: need numbers >= 0")
            add = eng._ints_of(add) if each else torch.full((n,), add[0], dtype=torch.int32,
                                                             device=eng.device)
        eng._need("add", add, (n,), torch.int32)
        served, src, dst, counts = self._ints(n), self._ints(n), self._ints(n), self._ints(2)
        ws = eng._scratch(akvs.akvs_pages_workspace_size(self.t, n))
        akvs.akvs_grow_pages(self.t, seq, add, served, src, dst, counts, ws)
        akvs.akvs_move_pages(self.layers[0], len(self.layers), eng.m, src, dst, n, counts)
        return served

    def compact(self):
        """The pages in use move to the lowest numbers, in all layers. Returns counts (int32:
        pages moved, pages in use)."""
        eng, n = self.engine, int(self.ref.numel())
        eng._here("the cache", self.table)
        src, dst, counts = self._ints(n), self._ints(n), self._ints(2)
        ws = eng._scratch(akvs.akvs_pages_workspace_size(self.t, 0))
        akvs.akvs_compact_pages(self.t, self.table, self.ref, src, dst, counts, ws)
        akvs.akvs_move_pages(self.layers[0], len(self.layers), eng.m, src, dst, n, counts)
        return counts


class BatchGraph:
    """One batched reuse-prefill call (reuse_prefill_batch) captured in a HIP graph, as
    ReuseGraph does for a single request: an eager call sizes the workspace and allocates
    the outputs, the capture reruns it on the same buffers, replay() reruns every kernel."""

    def __init__(self, engine: Engine, requests, *args, **kw):
        kw.pop("outputs", None)
        self.out = reuse_prefill_batch(engine, requests, *args, **kw)
        torch.cuda.synchronize(engine.device)
        self.ws = engine._ws  # the captured kernels address this workspace: keep it alive
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            reuse_prefill_batch(engine, requests, *args, outputs=self.out, **kw)
        torch.cuda.synchronize(engine.device)
        assert engine._ws is self.ws

    def replay(self):
        self.graph.replay()
        return self.out


class ReuseGraph:
    """One reuse-prefill call captured in a HIP graph (torch.cuda.CUDAGraph).

    The call is made once eagerly (which sizes the workspace and allocates the outputs),
    then captured; replay() reruns every kernel on the same buffers, so new token ids or
    cache contents are written into the captured tensors in place. The library's calls
    are capture-safe: kernel launches only (host tables travel as kernel arguments), no
    allocation, copy, memset or synchronisation. Kernel timing (akvs_profile_enable) must
    be off while capturing."""

    def __init__(self, engine: Engine, *args, **kw):
        kw.pop("outputs", None)
        self.out = engine.reuse_prefill(*args, **kw)
        torch.cuda.synchronize(engine.device)
        self.ws = engine._ws  # the captured kernels address this workspace: keep it alive
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            engine.reuse_prefill(*args, outputs=self.out, **kw)
        torch.cuda.synchronize(engine.device)
        assert engine._ws is self.ws

    def replay(self):
        self.graph.replay()
        return self.out


class FullGraph:
    """akvs_full_prefill over fixed token buffers captured in a HIP graph (the baseline
    counterpart of ReuseGraph); the outputs live in the graph's memory pool."""

    def __init__(self, engine: Engine, tokens: torch.Tensor, pos0: int = 0, want_h: bool = True):
        engine.full_prefill(tokens, pos0, want_h)  # sizes the workspace
        torch.cuda.synchronize(engine.device)
        self.ws = engine._ws  # the captured kernels address this workspace: keep it alive
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.out = engine.full_prefill(tokens, pos0, want_h)
        torch.cuda.synchronize(engine.device)
        assert engine._ws is self.ws

    def replay(self):
        self.graph.replay()
        return self.out
