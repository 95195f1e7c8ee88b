"""Operators over a shared context: what they refuse, without a GPU."""
import ctypes

import pytest
import torch

from paper_2607_21604_amd import akvs
from tests.libutil import ensure_built

A = 4096  # an aligned address that nothing reads: every call here is refused


@pytest.fixture(scope="module")
def lib():
    return ensure_built()


def model(hq=24, hkv=8, hd=128, dtype=akvs.AKVS_BF16):
    return akvs.ModelCfg(1, 256, hq, hkv, hd, 256, 64, 1e4, 1e-6, dtype)


def shared(**kw):
    d = dict(n_req=4, n_rows=4, rows_max=1, prefix_len=100, own_rows=16, row_start=None, own_len=A)
    d.update(kw)
    return akvs.SharedCfg(*d.values())


SHARED = [
    (dict(n_req=0), akvs.AKVS_EINVAL), (dict(n_rows=-1), akvs.AKVS_EINVAL),
    (dict(rows_max=0), akvs.AKVS_EINVAL), (dict(prefix_len=-1), akvs.AKVS_EINVAL),
    (dict(own_rows=-1), akvs.AKVS_EINVAL), (dict(own_len=None), akvs.AKVS_EINVAL),
    (dict(n_rows=5), akvs.AKVS_ESHAPE), (dict(rows_max=2), akvs.AKVS_ESHAPE),
    (dict(prefix_len=1 << 28), akvs.AKVS_ESHAPE),
    (dict(n_req=1 << 10, n_rows=1 << 10, own_rows=1 << 22), akvs.AKVS_ESHAPE),
    (dict(n_rows=1 << 24, row_start=A), akvs.AKVS_ESHAPE),
    (dict(n_req=1 << 18, n_rows=1 << 20, rows_max=1 << 20, row_start=A), akvs.AKVS_ESHAPE),
    # launches of 2^32 threads or more
    (dict(n_req=1, n_rows=1 << 23, rows_max=1 << 23), akvs.AKVS_ESHAPE),
    (dict(n_req=1 << 16, n_rows=1 << 10, rows_max=1 << 10, row_start=A), akvs.AKVS_ESHAPE),
    (dict(n_req=1 << 18, n_rows=1 << 18, own_rows=1 << 12), akvs.AKVS_ESHAPE),
]


@pytest.mark.parametrize("kw,status", SHARED)
def test_invalid_batches(lib, kw, status):
    m, c = model(), shared(**kw)
    assert akvs.akvs_shared_workspace_size(m, c) == 0
    assert lib.akvs_shared_attention(A, ctypes.byref(c), A, A, A, A, ctypes.byref(m), A, A, A,
                                     1 << 40, None) == status
    assert lib.akvs_attention_weights(A, A, ctypes.byref(c), A, A, ctypes.byref(m), A, A, A, A, A,
                                      1 << 40, None) == status


def test_invalid_models(lib):
    c, e = shared(), akvs.evict_cfg(2, 100, 10)
    for m, status in ((model(hd=96), akvs.AKVS_EUNSUPPORTED), (model(hq=20), akvs.AKVS_ESHAPE),
                      (model(dtype=akvs.AKVS_U4G64), akvs.AKVS_EDTYPE)):
        r = ctypes.byref(m)
        assert lib.akvs_shared_attention(A, ctypes.byref(c), A, A, A, A, r, A, A, A, 1 << 40,
                                         None) == status
        assert lib.akvs_attention_weights(A, A, ctypes.byref(c), A, A, r, A, A, A, A, A, 1 << 40,
                                          None) == status
        assert lib.akvs_evict_cache(A, A, A, ctypes.byref(e), r, A, A, A, A, A, A, 1 << 40,
                                    None) == status
        assert lib.akvs_qk_norm_rope(A, 4096, A, 4096, A, 4096, 4, A, A, A, r, A, 10, None, 4, A, A,
                                     A, None) == status
        assert akvs.akvs_shared_workspace_size(m, c) == 0
        assert akvs.akvs_evict_workspace_size(m, e) == 0


def test_null_and_misaligned_pointers(lib):
    m, c = model(), shared()
    args = [A, ctypes.byref(c), A, A, A, A, ctypes.byref(m), A, A, A, 1 << 40, None]
    for i in (0, 1, 2, 3, 4, 5, 6, 7):
        bad = list(args)
        bad[i] = None
        assert lib.akvs_shared_attention(*bad) == akvs.AKVS_EINVAL, i
    for i in (0, 2, 3, 4, 5, 7, 8, 9):
        bad = list(args)
        bad[i] = A + 8
        assert lib.akvs_shared_attention(*bad) == akvs.AKVS_EINVAL, i
    args = [A, A, ctypes.byref(c), A, A, ctypes.byref(m), A, A, A, A, A, 1 << 40, None]
    for i in (0, 1, 2, 3, 4, 5):
        bad = list(args)
        bad[i] = None
        assert lib.akvs_attention_weights(*bad) == akvs.AKVS_EINVAL, i
    for i in (0, 1, 3, 4, 6, 7, 8, 9, 10):
        bad = list(args)
        bad[i] = A + 4
        assert lib.akvs_attention_weights(*bad) == akvs.AKVS_EINVAL, i
    bad = list(args)
    bad[7] = bad[9] = None
    assert lib.akvs_attention_weights(*bad) == akvs.AKVS_EINVAL


def test_rows_max_above_the_rows_is_the_rows(lib):
    """A batch that says more rows per request than there are asks for no more workspace.
    (A short context is taken whole and needs none; a long one is split.)"""
    m = model()
    for prefix in (100, 8000):
        a, b = (akvs.akvs_shared_workspace_size(m, shared(n_rows=6, row_start=A, rows_max=r,
                                                          prefix_len=prefix))
                for r in (6, 1 << 30))
        assert a == b
        assert (a > 0) == (prefix == 8000)


def test_norm_overlaps(lib):
    """Outputs over inputs other than their own, over each other, and in place where rows lie
    apart or move."""
    m, es = model(), 2
    q, k, v, qo, ko, vo, pos = (1 << 30, 2 << 30, 3 << 30, 4 << 30, 5 << 30, 6 << 30, 7 << 30)
    base = dict(q=q, ldq=24 * 128, k=k, ldk=8 * 128, v=v, ldv=8 * 128, rows=4, kv=None, n_kv=4,
                qo=qo, ko=ko, vo=vo)
    for kw in (dict(qo=k), dict(qo=k - 4 * 24 * 128 * es + 16), dict(ko=q), dict(ko=v), dict(vo=k),
               dict(ko=qo), dict(vo=ko), dict(ko=qo + 4 * 24 * 128 * es - 16),
               dict(qo=q + 24 * 128 * es), dict(qo=q, ldq=40 * 128), dict(ko=k, ldk=16 * 128),
               dict(ko=k, kv=pos), dict(vo=v, kv=pos), dict(ko=v - 8 * 128 * es, kv=pos, n_kv=2),
               dict(ko=v - 9 * 8 * 128 * es, kv=pos, n_kv=10)):
        d = dict(base)
        d.update(kw)
        assert lib.akvs_qk_norm_rope(
            d["q"], d["ldq"], d["k"], d["ldk"], d["v"], d["ldv"], d["rows"], pos, None, None,
            ctypes.byref(m), pos, 10, d["kv"], d["n_kv"], d["qo"], d["ko"], d["vo"],
            None) == akvs.AKVS_EINVAL, kw


def test_norms_of_too_many_rows(lib):
    for n in (1 << 23, (1 << 31) - 1):
        m = model()
        assert lib.akvs_qk_norm_rope(A, 4096, A, 4096, A, 4096, n, A, A, A, ctypes.byref(m), A, 10,
                                     None, n, A, A, A, None) == akvs.AKVS_ESHAPE


def test_workspace(lib):
    for kw in (dict(), dict(prefix_len=8000), dict(own_rows=3000), dict(n_req=64, n_rows=64)):
        m, c = model(), shared(**kw)
        need = akvs.akvs_shared_workspace_size(m, c)
        if need == 0:
            continue
        assert lib.akvs_shared_attention(A, ctypes.byref(c), A, A, A, A, ctypes.byref(m), A, A, A,
                                         need - 1, None) == akvs.AKVS_ENOSPACE
        assert lib.akvs_shared_attention(A, ctypes.byref(c), A, A, A, A, ctypes.byref(m), A, A, None,
                                         need, None) == akvs.AKVS_ENOSPACE


@pytest.mark.parametrize("kw,status", [
    (dict(n_seq=0), akvs.AKVS_EINVAL), (dict(n_keys=-1), akvs.AKVS_EINVAL),
    (dict(n_keep=0), akvs.AKVS_EINVAL), (dict(n_first=-1), akvs.AKVS_EINVAL),
    (dict(n_recent=-1), akvs.AKVS_EINVAL), (dict(n_first=6, n_recent=5), akvs.AKVS_EINVAL),
    (dict(src_rows=99), akvs.AKVS_ESHAPE), (dict(dst_rows=9), akvs.AKVS_ESHAPE),
    (dict(n_seq=1 << 17), akvs.AKVS_ESHAPE), (dict(n_keep=1 << 27, n_seq=1), akvs.AKVS_ESHAPE), (dict(n_first=1 << 30, n_recent=1 << 30), akvs.AKVS_EINVAL)])
def test_invalid_evictions(lib, kw, status):
    d = dict(n_seq=2, n_keys=100, src_rows=0, n_keep=10, dst_rows=0, n_first=0, n_recent=0, lens=None)
    d.update(kw)
    m, c = model(), akvs.EvictCfg(*d.values())
    assert akvs.akvs_evict_workspace_size(m, c) == 0
    assert lib.akvs_evict_cache(A, A, A, ctypes.byref(c), ctypes.byref(m), A, A, A, A, A, A, 1 << 40,
                                None) == status


def test_eviction_buffers(lib):
    """Missing and misaligned buffers, a short workspace, and outputs over inputs."""
    m, c = model(2, 2, 64), akvs.evict_cfg(2, 100, 10)
    row = 2 * 64 * 2
    k, v, ko, vo = 1 << 20, 2 << 20, 3 << 20, 4 << 20
    call = lambda *a: lib.akvs_evict_cache(*a[:3], ctypes.byref(c), ctypes.byref(m), *a[3:], None)  # noqa: E731
    ok = [k, v, 5 << 20, 6 << 20, ko, vo, 7 << 20, 8 << 20, A, 1 << 30]
    for i in (0, 1, 2, 4, 5):  # k, v, weights, k_out, v_out missing one by one
        bad = list(ok)
        bad[i] = None
        assert call(*bad) == akvs.AKVS_EINVAL, i
    for i in (0, 1, 2, 3, 4, 5, 6, 8):
        bad = list(ok)
        bad[i] += 4
        assert call(*bad) == akvs.AKVS_EINVAL, i
    need = akvs.akvs_evict_workspace_size(m, c)
    bad = list(ok)
    bad[3], bad[9] = None, need - 1
    assert call(*bad) == akvs.AKVS_ENOSPACE
    bad[8], bad[9] = None, need
    assert call(*bad) == akvs.AKVS_ENOSPACE
    for i, at in ((4, k), (4, v + 2 * 100 * row - 16), (5, k - 2 * 10 * row + 16), (5, ko), (6, 5 << 20)):
        bad = list(ok)
        bad[i] = at
        assert call(*bad) == akvs.AKVS_EINVAL, (i, at)
        assert b"overlap" in lib.akvs_last_error()


def test_norm_arguments(lib):
    m = model()
    ok = [A, 24 * 128, A, 8 * 128, A, 8 * 128, 4, A, A, A, ctypes.byref(m), A, 10, None, 4, A, A, A,
          None]
    for i in (0, 2, 4, 7, 10, 11, 15, 16, 17):
        bad = list(ok)
        bad[i] = None
        assert lib.akvs_qk_norm_rope(*bad) == akvs.AKVS_EINVAL, i
    for i in (0, 2, 4, 8, 9, 11, 15, 16, 17):
        bad = list(ok)
        bad[i] = A + 8
        assert lib.akvs_qk_norm_rope(*bad) == akvs.AKVS_EINVAL, i
    for i, x in ((1, 24 * 128 - 8), (3, 1016), (5, 0), (1, 24 * 128 + 4), (3, 1028), (6, -1), (12, 0),
                 (14, 3), (14, -1)):
        bad = list(ok)
        bad[i] = x
        assert lib.akvs_qk_norm_rope(*bad) == akvs.AKVS_EINVAL, (i, x)


def test_binding_refuses_wrong_tables_and_rows():
    with pytest.raises(ValueError):
        akvs.shared_cfg(4, 4, 1, 10, 8, None, torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        akvs.shared_cfg(4, 4, 1, 10, 8, torch.zeros(5, dtype=torch.int64), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        akvs.evict_cfg(4, 10, 5, lens=torch.zeros(2, dtype=torch.int32))
    x = torch.zeros(6, 8, 16)
    assert akvs.rows_ptr(x[:, 2:4])[1] == 128 and akvs.rows_ptr(x[:1, 2:4])[1] == 32
    with pytest.raises(ValueError):
        akvs.rows_ptr(x[:, :, :8])
    with pytest.raises(ValueError):
        akvs.rows_ptr(x.transpose(0, 1))


class _Shape:
    n_layers, d_model, n_q_heads, n_kv_heads, head_dim, ffn_dim, vocab = 1, 256, 6, 2, 64, 256, 64
    rope_theta, rms_eps, dtype = 1e4, 1e-6, "bf16"


@pytest.fixture(scope="module")
def engine(lib):
    from paper_2607_21604_amd.runtime import Engine
    w = {k: torch.zeros(8) for k in ("attn_norm", "w_qkv", "w_o", "mlp_norm", "w_gate_up", "w_down")}
    return Engine(_Shape, {"layers": [w]}, "cpu")


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32)


def test_engine_refuses_wrong_tensors(engine):
    """Shapes and types that the C entries cannot see are refused by the engine's methods."""
    q, kp, ko, ln = bf(3, 6, 64), bf(10, 2, 64), bf(3, 8, 2, 64), i32(1, 2, 3)
    for args in ((q.float(), kp, kp), (q, kp.float(), kp), (q, kp, bf(9, 2, 64)),
                 (q, kp, kp, ko, None, ln), (q, kp, kp, ko, bf(3, 7, 2, 64), ln),
                 (q, kp, kp, ko, ko), (q, kp, kp, ko, ko, i32(1, 2)),
                 (q, kp, kp, ko, ko, ln.long()), (q, kp, kp, ko, ko, ln, i32(0, 1, 3)),
                 (bf(4, 6, 64), kp, kp, ko, ko, ln), (q.transpose(1, 2), kp, kp)):
        with pytest.raises(ValueError):
            engine.shared_attention(*args)
    with pytest.raises(ValueError):
        engine.shared_attention(q, kp, kp, out=bf(2, 6, 64))
    lse = torch.zeros(3, 6)
    for kw in (dict(lse=lse.double()), dict(w_prefix=torch.zeros(2, 9)),
               dict(w_own=torch.zeros(3, 2, 8)), dict(k_own=ko, own_len=ln, w_own=torch.zeros(3, 2, 7))):
        a = dict(lse=lse)
        a.update(kw)
        with pytest.raises(ValueError):
            engine.attention_weights(q, a.pop("lse"), kp, **a)
    k, w = bf(2, 30, 2, 64), torch.zeros(2, 2, 30)
    for args in ((k.float(), k, w, 5), (k, bf(2, 29, 2, 64), w, 5), (k, k, w.double(), 5),
                 (k, k, torch.zeros(2, 3, 30), 5), (k, k, w, 5, 0, 0, i32(1)),
                 (bf(2, 20, 2, 64), bf(2, 20, 2, 64), w, 5)):
        with pytest.raises(ValueError):
            engine.evict_cache(*args)
    rope, pos = torch.zeros(5, 32, 2), i32(0, 1, 2)
    for args in ((q, bf(3, 128), bf(3, 127), pos, None, None, rope),
                 (q.float(), bf(3, 128), bf(3, 128), pos, None, None, rope),
                 (q, bf(3, 128), bf(2, 128), pos, None, None, rope),
                 (q, bf(3, 128), bf(3, 128), pos.long(), None, None, rope),
                 (q, bf(3, 128), bf(3, 128), pos, bf(63), None, rope),
                 (q, bf(3, 128), bf(3, 128), pos, None, None, rope, bf(9, 2, 64)),
                 (q, bf(3, 128), bf(3, 128), pos, None, None, rope, None, None, pos),
                 (q, bf(3, 128), bf(3, 128), pos, None, None, torch.zeros(5, 64, 2))):
        with pytest.raises(ValueError):
            engine.qk_norm_rope(*args)


MB = 1 << 20


def overlapping(lib, call, args, cases):
    """Every call with one buffer moved over another is refused and says so."""
    for name, at in cases:
        bad = dict(args)
        bad[name] = at
        assert call(bad) == akvs.AKVS_EINVAL, (name, at)
        assert b"overlaps" in lib.akvs_last_error(), (name, at)


@pytest.mark.parametrize("prefix,own", [(100, 16), (8000, 16), (8000, 0)])
def test_attention_overlaps(lib, prefix, own):
    """Outputs and the workspace over inputs, tables and each other; out over q is q itself or
    nothing of it."""
    m, rows = model(24, 8, 128), 4
    q, kv = rows * 24 * 128 * 2, 8 * 128 * 2
    a = {n: (16 + 64 * i) * MB for i, n in enumerate(
        ("q", "kp", "vp", "ko", "vo", "start", "len", "out", "lse", "ws"))}
    need = akvs.akvs_shared_workspace_size(m, shared(prefix_len=prefix, own_rows=own))

    def call(x):
        c = shared(prefix_len=prefix, own_rows=own, row_start=x["start"], own_len=x["len"])
        return lib.akvs_shared_attention(x["q"], ctypes.byref(c), x["kp"], x["vp"], x["ko"], x["vo"],
                                         ctypes.byref(m), x["out"], x["lse"], x["ws"], need, None)
    cases = [("out", a["q"] + 16), ("out", a["q"] - 16), ("out", a["kp"]),
             ("out", a["kp"] - q + 16), ("out", a["vp"] + prefix * kv - 16), ("out", a["start"]),
             ("out", a["len"]), ("lse", a["q"]), ("lse", a["out"]), ("lse", a["out"] + q - 16),
             ("lse", a["kp"]), ("lse", a["start"]), ("lse", a["len"] - rows * 24 * 4 + 16)]
    if own:
        cases += [("out", a["ko"] + 4 * own * kv - 16), ("lse", a["vo"])]
    if need:
        cases += [("ws", a["q"]), ("ws", a["out"] - need + 256), ("ws", a["lse"]), ("ws", a["vp"]),
                  ("out", a["ws"] + need - 16)]
    overlapping(lib, call, a, cases)


@pytest.mark.parametrize("prefix,own,rows", [(100, 16, 4), (8000, 16, 4), (300, 64, 256)])
def test_weights_overlaps(lib, prefix, own, rows):
    """Weights over inputs, tables, each other and each other's earlier ones; a side's earlier
    weights are its weights or nothing of them."""
    m = model(24, 8, 128)
    cfg = dict(prefix_len=prefix, own_rows=own, n_rows=rows, rows_max=rows // 4)
    wp, wo = 8 * prefix * 4, 4 * 8 * own * 4
    a = {n: (16 + 64 * i) * MB for i, n in enumerate(
        ("q", "lse", "kp", "ko", "start", "len", "wp0", "wo0", "wp", "wo", "ws"))}
    need = akvs.akvs_shared_workspace_size(m, shared(**cfg))

    def call(x):
        c = shared(row_start=x["start"], own_len=x["len"], **cfg)
        return lib.akvs_attention_weights(x["q"], x["lse"], ctypes.byref(c), x["kp"], x["ko"],
                                          ctypes.byref(m), x["wp0"], x["wp"], x["wo0"], x["wo"], x["ws"],
                                          need, None)
    cases = [("wp", a["wp0"] + 16), ("wp", a["wp0"] - 16), ("wo", a["wo0"] + 16), ("wp", a["wo0"]),
             ("wo", a["wp0"]), ("wo", a["wp"]), ("wo", a["wp"] + wp - 16), ("wp", a["wo"] + wo - 16),
             ("wp", a["q"]), ("wo", a["lse"]), ("wp", a["kp"]), ("wo", a["ko"]), ("wo", a["start"]),
             ("wp", a["len"] - wp + 16)]
    if need:
        cases += [("ws", a["q"]), ("ws", a["wp"] - need + 256), ("ws", a["wo0"]), ("wo", a["ws"])]
    overlapping(lib, call, a, cases)
    for side in ("wp", "wo"):  # a side that is not formed
        b = dict(a)
        b[side] = b[side + "0"] = None
        overlapping(lib, call, b, [({"wp": "wo", "wo": "wp"}[side], a["q"])])


@pytest.mark.parametrize("keys", [100, 40000])
def test_eviction_overlaps(lib, keys):
    """Each output and the workspace over inputs and each other; lens_out over lens is lens itself."""
    m, S, H, keep = model(2, 2, 64), 2, 2, 10
    e = akvs.evict_cfg(S, keys, keep)
    a = {n: (16 + 64 * i) * MB for i, n in enumerate(
        ("k", "v", "w", "lens", "keep", "ko", "vo", "wo", "lo", "ws"))}
    need = akvs.akvs_evict_workspace_size(m, e)

    def call(x):
        c = akvs.EvictCfg(S, keys, 0, keep, 0, 0, 0, x["lens"])
        return lib.akvs_evict_cache(x["k"], x["v"], x["w"], ctypes.byref(c), ctypes.byref(m), x["keep"],
                                    x["ko"], x["vo"], x["wo"], x["lo"], x["ws"], need, None)
    n_keep, n_w = S * H * keep * 4, S * H * keys * 4
    cases = [("keep", a["w"] + n_w - 16), ("keep", a["k"]), ("keep", a["ko"]), ("keep", a["wo"]),
             ("keep", a["lens"]), ("ko", a["keep"] + n_keep - 16), ("wo", a["w"]), ("wo", a["vo"]),
             ("wo", a["lens"]), ("lo", a["lens"] + 4), ("lo", a["w"]), ("lo", a["keep"]), ("lo", a["vo"]),
             ("ws", a["w"]), ("ws", a["keep"] - need + 256), ("ws", a["lens"]), ("vo", a["ws"])]
    overlapping(lib, call, a, cases)
    a["keep"] = None
    overlapping(lib, call, a, [("ws", a["k"]), ("ws", a["wo"] - need + 16)])


def test_norm_overlaps_of_tables(lib):
    """Outputs over positions, rows, gains and the rotary table."""
    m, n, hd = model(24, 8, 128), 4, 128
    a = {x: (16 + 64 * i) * MB for i, x in enumerate(
        ("q", "k", "v", "pos", "gq", "gk", "rope", "rows", "qo", "ko", "vo"))}

    def call(x):
        return lib.akvs_qk_norm_rope(x["q"], 24 * hd, x["k"], 8 * hd, x["v"], 8 * hd, n, x["pos"],
                                     x["gq"], x["gk"], ctypes.byref(m), x["rope"], 10, x["rows"], 9,
                                     x["qo"], x["ko"], x["vo"], None)
    overlapping(lib, call, a, [(o, a[i]) for o in ("qo", "ko", "vo") for i in
                               ("pos", "gq", "gk", "rope", "rows")] +
                [("qo", a["rope"] + 10 * hd * 4 - 16), ("vo", a["pos"] - 9 * 8 * hd * 2 + 16)])


def test_weights_of_too_long_a_prefix(lib):
    """Prefixes within the batch's limits whose keys alone are 2^32 threads."""
    for m, kw in ((model(8, 8, 64), dict(prefix_len=(1 << 28) - 1)),
                  (model(32, 32, 64, akvs.AKVS_F32), dict(prefix_len=1 << 25)),
                  (model(16, 16, 64), dict(prefix_len=(1 << 27) - 64, n_req=64, n_rows=64))):
        c = shared(**kw)
        assert akvs.akvs_shared_workspace_size(m, c) > 0
        assert lib.akvs_attention_weights(A, A, ctypes.byref(c), A, A, ctypes.byref(m), A, A, A, A, A,
                                          1 << 40, None) == akvs.AKVS_ESHAPE


def test_engine_takes_rows_from_the_host(engine):
    """row_start as a sequence: checked, copied, and planned for its longest request, so that a
    batch of many requests fits that does not with all rows for each."""
    kp, B = bf(8000, 2, 64), 4096
    q, ko, ln = bf(3 * B, 6, 64), bf(B, 4, 2, 64), torch.ones(B, dtype=torch.int32)
    st = [3 * i for i in range(B + 1)]
    c = engine._shared(q, kp, ko, ln, st, None)
    t = engine._shared(q, kp, ko, ln, i32(*st), 3)
    assert c.rows_max == t.rows_max == 3 and c.n_req == t.n_req == B and c.n_rows == t.n_rows
    assert c._keep[0].tolist() == st and c._keep[0].dtype == torch.int32
    need = akvs.akvs_shared_workspace_size(engine.m, c)
    assert need == akvs.akvs_shared_workspace_size(engine.m, t) > 0
    every = engine._shared(q, kp, ko, ln, i32(*st), None)
    assert every.rows_max == 3 * B and akvs.akvs_shared_workspace_size(engine.m, every) == 0
    q = bf(9, 6, 64)
    assert engine._shared(q, kp, None, None, (0, 0, 5, 5, 8), None).rows_max == 5
    assert engine._shared(q, kp, None, None, torch.tensor([0, 2, 9]).numpy(), 8).rows_max == 7
    assert engine._shared(q[:0], kp, None, None, [0, 0], None).rows_max == 1
    for bad, most in (([0, 5, 4], None), ([1, 5], None), ([0, 10], None), ([0], None), ([], None),
                      ([0, 4, 9], 4), ([0, -1, 9], None)):
        with pytest.raises(ValueError, match="row_start"):
            engine._shared(q, kp, None, None, bad, most)
    with pytest.raises(TypeError):
        engine._shared(q, kp, None, None, [0, 4.5], None)
