"""Operators that decode from four bits: what they refuse, without a GPU."""
import ctypes

import pytest
import torch

from paper_2607_21604_amd import akvs
from tests.libutil import ensure_built

A = 4096  # an aligned address that nothing reads: every call here is refused
FAR = [i << 40 for i in range(1, 16)]  # addresses of buffers that do not overlap
by = ctypes.byref


@pytest.fixture(scope="module")
def lib():
    return ensure_built()


def model(hq=24, hkv=8, hd=128, dtype=akvs.AKVS_BF16):
    return akvs.ModelCfg(1, 256, hq, hkv, hd, 256, 64, 1e4, 1e-6, dtype)


def cfg(**kw):
    d = dict(n_req=4, n_rows=4, rows_max=1, n_seq=6, max_pages=10, max_len=500, row_start=None,
             seq=FAR[10], len=FAR[11], table=FAR[12])
    d.update(kw)
    return akvs.PagedCfg(*d.values())


def pages(**kw):
    d = dict(k=FAR[0], v=FAR[1], k_meta=FAR[2], v_meta=FAR[3], n_pages=40, page_rows=64)
    d.update(kw)
    return akvs.Pages(*d.values())


def table(**kw):
    d = dict(n_seq=6, max_pages=10, n_pages=40, page_rows=64, table=FAR[0], len=FAR[1], ref=FAR[2])
    d.update(kw)
    return akvs.PageTable(*d.values())


def calls(lib, m, c, p):
    """(store, load, attention) with buffers of their own."""
    m, c, p = by(m), by(c), by(p)
    return (lambda: lib.akvs_store_pages(FAR[4], 1024, FAR[5], 1024, c, p, m, None),
            lambda: lib.akvs_load_pages(c, p, m, FAR[4], FAR[5], akvs.AKVS_F32, None),
            lambda: lib.akvs_paged_attention(FAR[4], c, p, m, FAR[5], FAR[6], FAR[7], 1 << 39, None))


BATCHES = [
    (dict(n_req=0), akvs.AKVS_EINVAL), (dict(n_req=(1 << 20) + 1), akvs.AKVS_EINVAL),
    (dict(n_rows=-1), akvs.AKVS_EINVAL), (dict(rows_max=0), akvs.AKVS_EINVAL),
    (dict(n_seq=0), akvs.AKVS_EINVAL), (dict(max_pages=0), akvs.AKVS_EINVAL),
    (dict(max_len=-1), akvs.AKVS_EINVAL), (dict(len=None), akvs.AKVS_EINVAL),
    (dict(table=None), akvs.AKVS_EINVAL), (dict(seq=None, n_req=7, n_rows=7), akvs.AKVS_ESHAPE),
    (dict(n_rows=5), akvs.AKVS_ESHAPE), (dict(rows_max=2), akvs.AKVS_ESHAPE),
    (dict(n_rows=1 << 24, row_start=A), akvs.AKVS_ESHAPE),
    (dict(n_seq=1 << 16, max_pages=1 << 15), akvs.AKVS_ESHAPE),
    (dict(max_len=1 << 28, max_pages=1 << 24), akvs.AKVS_ESHAPE),
    (dict(n_req=1 << 18, n_rows=1 << 20, rows_max=1 << 20, row_start=A, max_len=600),
     akvs.AKVS_ESHAPE),
]


@pytest.mark.parametrize("kw,status", BATCHES)
def test_invalid_batches(lib, kw, status):
    m, c = model(), cfg(**kw)
    assert akvs.akvs_paged_workspace_size(m, c) == 0
    for call in calls(lib, m, c, pages()):
        assert call() == status


def test_more_keys_than_pages(lib):
    for call in calls(lib, model(), cfg(max_len=641), pages()):
        assert call() == akvs.AKVS_ESHAPE


@pytest.mark.parametrize("kw,status", [
    (dict(page_rows=48), akvs.AKVS_EUNSUPPORTED), (dict(page_rows=8), akvs.AKVS_EUNSUPPORTED),
    (dict(page_rows=512), akvs.AKVS_EUNSUPPORTED), (dict(page_rows=0), akvs.AKVS_EUNSUPPORTED),
    (dict(n_pages=-1), akvs.AKVS_EINVAL), (dict(n_pages=1 << 28), akvs.AKVS_ESHAPE),
    (dict(k=None), akvs.AKVS_EINVAL), (dict(v=None), akvs.AKVS_EINVAL),
    (dict(k_meta=None), akvs.AKVS_EINVAL), (dict(v_meta=None), akvs.AKVS_EINVAL),
    (dict(k=FAR[0] + 8), akvs.AKVS_EINVAL), (dict(v_meta=FAR[3] + 4), akvs.AKVS_EINVAL),
])
def test_invalid_pages(lib, kw, status):
    p, m = pages(**kw), model()
    for call in calls(lib, m, cfg(), p):
        assert call() == status
    assert lib.akvs_move_pages(by(p), 2, by(m), FAR[4], FAR[5], 3, None, None) == status


@pytest.mark.parametrize("m,status", [
    (model(hd=96), akvs.AKVS_EUNSUPPORTED), (model(hq=20), akvs.AKVS_ESHAPE),
    (model(dtype=akvs.AKVS_U4G64), akvs.AKVS_EDTYPE), (model(dtype=akvs.AKVS_F32), akvs.AKVS_EDTYPE)])
def test_invalid_models(lib, m, status):
    for call in calls(lib, m, cfg(), pages()):
        assert call() == status
    assert lib.akvs_move_pages(by(pages()), 2, by(m), FAR[4], FAR[5], 3, None, None) == status
    assert akvs.akvs_paged_workspace_size(m, cfg()) == 0


def test_null_descriptors(lib):
    m, c, p, t = by(model()), by(cfg()), by(pages()), by(table())
    E = akvs.AKVS_EINVAL
    for mm, cc, pp in ((None, c, p), (m, None, p), (m, c, None)):
        assert lib.akvs_store_pages(FAR[4], 1024, FAR[5], 1024, cc, pp, mm, None) == E
        assert lib.akvs_load_pages(cc, pp, mm, FAR[4], FAR[5], akvs.AKVS_F32, None) == E
        assert lib.akvs_paged_attention(FAR[4], cc, pp, mm, FAR[5], FAR[6], FAR[7], 1 << 39,
                                        None) == E
    assert lib.akvs_fork_pages(None, 1, FAR[4], FAR[5], None) == E
    assert lib.akvs_free_pages(None, 1, FAR[4], None) == E
    assert lib.akvs_fork_pages(t, 1, None, FAR[5], None) == E
    assert lib.akvs_fork_pages(t, 1, FAR[4], None, None) == E
    assert lib.akvs_free_pages(t, 1, None, None) == E
    assert akvs.load().akvs_pages_workspace_size(None, 1) == 0


def test_store_arguments(lib):
    m, c, p = by(model()), by(cfg()), by(pages())
    ok = [FAR[4], 1024, FAR[5], 1024, c, p, m, None]
    for i, bad in ((0, None), (2, None), (0, FAR[4] + 2), (2, FAR[5] + 8), (1, 1023), (3, 1020),
                   (1, 1028), (0, FAR[1]), (2, FAR[2] + 16), (0, FAR[0] + (1 << 20) - 16)):
        args = list(ok)
        args[i] = bad
        assert lib.akvs_store_pages(*args) == akvs.AKVS_EINVAL, (i, bad)
    args = list(ok)
    args[1] = 1 << 31
    assert lib.akvs_store_pages(*args) == akvs.AKVS_ESHAPE


def test_load_arguments(lib):
    m, c, p = by(model()), by(cfg()), by(pages())
    ok = [c, p, m, FAR[4], FAR[5], akvs.AKVS_F32, None]
    for i, bad, status in ((5, akvs.AKVS_U4G64, akvs.AKVS_EDTYPE), (3, FAR[4] + 4, akvs.AKVS_EINVAL),
                           (4, FAR[4], akvs.AKVS_EINVAL), (3, FAR[0], akvs.AKVS_EINVAL),
                           (4, FAR[12], akvs.AKVS_EINVAL)):
        args = list(ok)
        args[i] = bad
        assert lib.akvs_load_pages(*args) == status, (i, bad)
    args = list(ok)
    args[3] = args[4] = None
    assert lib.akvs_load_pages(*args) == akvs.AKVS_EINVAL


@pytest.mark.parametrize("kw", [
    dict(n_req=1 << 16, n_rows=1 << 16, rows_max=1 << 16),  # 2^16 requests of up to 4096 tiles
    dict(n_req=1 << 20, n_rows=(1 << 24) // 28 - 1, rows_max=400, max_len=640),
])
def test_attention_of_too_many_blocks(lib, kw):
    c = cfg(row_start=FAR[13], **kw)
    assert lib.akvs_paged_attention(FAR[4], by(c), by(pages()), by(model()), FAR[5], FAR[6], FAR[7],
                                    1 << 39, None) == akvs.AKVS_ESHAPE


def test_attention_arguments(lib):
    m, c, p = by(model()), by(cfg()), by(pages())
    ok = [FAR[4], c, p, m, FAR[5], FAR[6], FAR[7], 1 << 39, None]
    for i, bad in ((0, None), (4, None), (0, FAR[4] + 8), (4, FAR[5] + 8), (5, FAR[6] + 4),
                   (6, FAR[7] + 8), (4, FAR[4] + 16), (5, FAR[5]), (4, FAR[3]), (5, FAR[11]),
                   (4, FAR[12])):
        args = list(ok)
        args[i] = bad
        assert lib.akvs_paged_attention(*args) == akvs.AKVS_EINVAL, (i, bad)
    need = akvs.akvs_paged_workspace_size(model(), cfg(max_pages=1 << 10, max_len=60000))
    if need:
        c = by(cfg(max_pages=1 << 10, max_len=60000))
        for ws, n in ((None, 0), (FAR[7], need - 1)):
            args = [FAR[4], c, p, m, FAR[5], FAR[6], ws, n, None]
            assert lib.akvs_paged_attention(*args) == akvs.AKVS_ENOSPACE


@pytest.mark.parametrize("kw,status", [
    (dict(n_seq=0), akvs.AKVS_EINVAL), (dict(max_pages=0), akvs.AKVS_EINVAL),
    (dict(n_pages=-1), akvs.AKVS_EINVAL), (dict(page_rows=20), akvs.AKVS_EUNSUPPORTED),
    (dict(n_pages=1 << 28), akvs.AKVS_ESHAPE), (dict(n_seq=1 << 24), akvs.AKVS_ESHAPE),
    (dict(n_seq=1 << 16, max_pages=1 << 15), akvs.AKVS_ESHAPE),
    (dict(max_pages=1 << 25), akvs.AKVS_ESHAPE), (dict(table=None), akvs.AKVS_EINVAL),
    (dict(len=None), akvs.AKVS_EINVAL), (dict(ref=None), akvs.AKVS_EINVAL),
    (dict(ref=FAR[2] + 4), akvs.AKVS_EINVAL), (dict(len=FAR[0]), akvs.AKVS_EINVAL),
    (dict(ref=FAR[1]), akvs.AKVS_EINVAL)])
def test_invalid_tables(lib, kw, status):
    t = by(table(**kw))
    overlap = "len" in kw and kw["len"] == FAR[0] or kw.get("ref") == FAR[1]
    assert (lib.akvs_pages_workspace_size(t, 2) == 0) != overlap
    assert lib.akvs_fork_pages(t, 2, FAR[4], FAR[5], None) == status
    assert lib.akvs_free_pages(t, 2, FAR[4], None) == status
    assert lib.akvs_grow_pages(t, 2, FAR[4], FAR[5], FAR[6], FAR[7], FAR[8], FAR[9], FAR[10],
                               1 << 39, None) == status
    if not overlap:
        assert lib.akvs_compact_pages(t, FAR[4], FAR[5], FAR[6], FAR[7], FAR[8], FAR[9], 1 << 39,
                                      None) == status


def test_table_arguments(lib):
    t, E, N = by(table()), akvs.AKVS_EINVAL, akvs.AKVS_ENOSPACE
    need = lib.akvs_pages_workspace_size(t, 2)
    assert need > 0 and lib.akvs_pages_workspace_size(t, -1) == 0
    assert lib.akvs_fork_pages(t, -1, FAR[4], FAR[5], None) == E
    assert lib.akvs_fork_pages(t, 2, FAR[0], FAR[5], None) == E      # src in the table
    assert lib.akvs_fork_pages(t, 2, FAR[4], FAR[1], None) == E      # dst in len
    assert lib.akvs_free_pages(t, 2, FAR[2], None) == E              # seq in ref
    grow = [t, 2, FAR[4], FAR[5], FAR[6], FAR[7], FAR[8], FAR[9], FAR[10], need, None]
    for i, bad, status in ((2, None, E), (3, None, E), (4, None, E), (5, None, E), (6, None, E),
                           (7, None, E), (8, None, N), (9, need - 1, N), (8, FAR[10] + 4, E),
                           (4, FAR[4], E), (5, FAR[6], E), (6, FAR[7] + 4, E), (7, FAR[2], E),
                           (8, FAR[0], E), (1, -1, E)):
        args = list(grow)
        args[i] = bad
        assert lib.akvs_grow_pages(*args) == status, (i, bad)
    comp = [t, FAR[4], FAR[5], FAR[6], FAR[7], FAR[8], FAR[9], need, None]
    for i, bad, status in ((1, None, E), (2, None, E), (3, None, E), (4, None, E), (5, None, E),
                           (6, None, N), (7, 16, N), (6, FAR[9] + 8, E), (1, FAR[0] + 16, E),
                           (1, FAR[2], E), (2, FAR[0], E), (3, FAR[4], E), (4, FAR[1], E)):
        args = list(comp)
        args[i] = bad
        assert lib.akvs_compact_pages(*args) == status, (i, bad)


def test_move_arguments(lib):
    m, p, E = by(model()), by(pages()), akvs.AKVS_EINVAL
    ok = [p, 2, m, FAR[4], FAR[5], 3, FAR[6], None]
    for i, bad, status in ((1, -1, E), (5, -1, E), (3, None, E), (4, None, E), (3, FAR[0], E),
                           (4, FAR[3], E), (6, FAR[1], E), (1, 1 << 16, akvs.AKVS_ESHAPE),
                           (5, 1 << 28, akvs.AKVS_ESHAPE), (0, None, E), (2, None, E)):
        args = list(ok)
        args[i] = bad
        assert lib.akvs_move_pages(*args) == status, (i, bad)
    # layers that reach the next buffer: 40 pages of 64 rows of 8 heads of 64 bytes a layer
    layer = 40 * 64 * 8 * 64
    near = pages(v=FAR[0] + 2 * layer)
    assert lib.akvs_move_pages(by(near), 3, m, FAR[4], FAR[5], 3, None, None) == E


def test_w4_arguments(lib):
    E, S, D = akvs.AKVS_EINVAL, akvs.AKVS_ESHAPE, akvs.AKVS_EDTYPE
    B, F = akvs.AKVS_BF16, akvs.AKVS_F32
    ok = dict(x=FAR[0], ldx=128, xt=B, rows=3, w=FAR[1], meta=FAR[2], n_out=10, n_in=128, mode=0,
              resid=None, y=FAR[3], ldy=10, yt=F, ws=FAR[4], n=1 << 39)
    for kw, status in (
            (dict(rows=-1), E), (dict(n_out=-1), E), (dict(n_in=0), E), (dict(n_in=96), E),
            (dict(rows=1 << 24), S), (dict(n_out=1 << 24), S), (dict(n_in=1 << 24, ldx=1 << 24), S),
            (dict(rows=1 << 16, n_out=1 << 16, ldy=1 << 16), S), (dict(xt=akvs.AKVS_U4G64), D),
            (dict(yt=akvs.AKVS_E4M3G64), D), (dict(mode=2), E), (dict(mode=-1), E),
            (dict(mode=1, n_out=11, ldy=11), E), (dict(mode=1, resid=FAR[5]), E),
            (dict(yt=B, resid=FAR[5]), E), (dict(x=None), E), (dict(w=None), E),
            (dict(meta=None), E), (dict(y=None), E), (dict(x=FAR[0] + 8), E),
            (dict(w=FAR[1] + 4), E), (dict(meta=FAR[2] + 4), E), (dict(y=FAR[3] + 4), E),
            (dict(resid=FAR[5] + 4), E), (dict(ldx=127), E), (dict(ldx=132), E), (dict(ldy=9), E),
            (dict(ldx=1 << 31), S), (dict(ldy=1 << 31), S), (dict(xt=F, ldx=130), E),
            (dict(y=FAR[0]), E), (dict(y=FAR[1] + 16), E), (dict(y=FAR[2]), E),
            (dict(resid=FAR[3] + 16), E), (dict(mode=1, y=FAR[0] + 3 * 256 - 16), E)):
        a = dict(ok)
        a.update(kw)
        assert lib.akvs_w4_product(*a.values(), None) == status, kw
    assert akvs.akvs_w4_workspace_size(-1, 10, 128) == 0
    assert akvs.akvs_w4_workspace_size(1, 10, 100) == 0


def test_calls_without_rows_or_pages_do_nothing(lib):
    """Valid calls that have nothing to do enqueue nothing (there is no GPU here)."""
    m, t = by(model()), by(table())
    assert lib.akvs_store_pages(None, 0, None, 0, by(cfg(n_rows=0)), by(pages()), m, None) == 0
    assert lib.akvs_load_pages(by(cfg(n_rows=0)), by(pages()), m, None, None, 0, None) == 0
    c = cfg(n_rows=0)
    need = akvs.akvs_paged_workspace_size(model(), c)
    assert need == 0
    assert lib.akvs_paged_attention(None, by(c), by(pages()), m, None, None, None, 0, None) == 0
    assert lib.akvs_fork_pages(t, 0, None, None, None) == 0
    assert lib.akvs_free_pages(t, 0, None, None) == 0
    assert lib.akvs_move_pages(by(pages()), 2, m, None, None, 0, None, None) == 0
    assert lib.akvs_move_pages(by(pages(k=None, v=None, k_meta=None, v_meta=None, n_pages=0)), 2, m,
                               FAR[4], FAR[5], 3, None, None) == 0
    assert lib.akvs_w4_product(None, 0, 0, 0, None, None, 5, 64, 0, None, None, 0, 0, None, 0,
                               None) == 0
    assert lib.akvs_w4_product(None, 0, 0, 3, None, None, 0, 64, 0, None, None, 0, 0, None, 0,
                               None) == 0


def test_wrappers_check_their_tensors(lib):
    u8, f16, i32 = torch.uint8, torch.float16, torch.int32
    k, meta = torch.zeros(3, 2, 16, 64, dtype=u8), torch.zeros(3, 2, 16, 2, 2, dtype=f16)
    p = akvs.pages(k, k.clone(), meta, meta.clone())
    assert (p.n_pages, p.page_rows) == (3, 16)
    with pytest.raises(ValueError, match="k_meta"):
        akvs.pages(k, k.clone(), k.clone(), meta)
    with pytest.raises(ValueError, match="v:"):
        akvs.pages(k, torch.zeros(3, 2, 32, 64, dtype=u8), meta, meta)
    tab, lens = torch.zeros(4, 5, dtype=i32), torch.zeros(4, dtype=i32)
    t = akvs.page_table(tab, lens, torch.zeros(3, dtype=i32), 16)
    assert (t.n_seq, t.max_pages, t.n_pages, t.page_rows) == (4, 5, 3, 16)
    for bad in (lens[:3], lens.long()):
        with pytest.raises(ValueError, match="int32"):
            akvs.page_table(tab, bad, torch.zeros(3, dtype=i32), 16)
        with pytest.raises(ValueError, match="int32"):
            akvs.paged_cfg(2, 2, 1, bad, tab, 16)
    with pytest.raises(ValueError, match="int32"):
        akvs.paged_cfg(2, 2, 1, lens, tab, 16, seq=lens[:1])
    x, w, wm = torch.zeros(2, 128), torch.zeros(6, 64, dtype=u8), torch.zeros(6, 2, 2, dtype=f16)
    for y, kw, text in ((torch.zeros(2, 5), {}, "do not fit"),
                        (torch.zeros(2, 6), dict(mode=akvs.AKVS_W4_SWIGLU), "do not fit"),
                        (torch.zeros(2, 6), dict(resid=torch.zeros(2, 8)[:, :6]), "resid"),
                        (torch.zeros(2, 6), dict(resid=torch.zeros(2, 6).bfloat16()), "resid")):
        with pytest.raises(ValueError, match=text):
            akvs.akvs_w4_product(x, w, wm, y, **kw)
    with pytest.raises(ValueError, match="weights"):
        akvs.akvs_w4_product(x, w, wm[:5], torch.zeros(2, 6))


def test_the_marks_of_sequences_without_room(lib):
    """`grown` lies apart from what a call writes, at an aligned address."""
    E, m = akvs.AKVS_EINVAL, by(model())
    for t in (table(grown=FAR[8] + 4), table(grown=FAR[0] + 16), table(grown=FAR[2] + 16),
              table(grown=FAR[4])):
        assert lib.akvs_fork_pages(by(t), 1, FAR[4], FAR[5], None) == E
        assert lib.akvs_free_pages(by(t), 1, FAR[4], None) == E
        assert lib.akvs_grow_pages(by(t), 1, FAR[4], FAR[5], FAR[6], FAR[7], FAR[9], FAR[10],
                                   FAR[11], 1 << 39, None) == E
    for x in (FAR[0], FAR[3] + 16):
        assert lib.akvs_store_pages(FAR[4], 1024, FAR[5], 1024, by(cfg(grown=x)), by(pages()), m,
                                    None) == E
    lens, tab = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 5, dtype=torch.int32)
    for bad in (lens[:3], lens.long()):
        with pytest.raises(ValueError, match="int32"):
            akvs.page_table(tab, lens, torch.zeros(3, dtype=torch.int32), 16, bad)
        with pytest.raises(ValueError, match="int32"):
            akvs.paged_cfg(2, 2, 1, lens, tab, 16, grown=bad)


def test_loading_checks_its_outputs(lib):
    """Both of one type and as many rows as the batch's: nothing is written past their ends."""
    m, F, B = model(), torch.float32, torch.bfloat16
    c = akvs.paged_cfg(2, 5, 3, torch.zeros(4, dtype=torch.int32),
                       torch.zeros(4, 5, dtype=torch.int32), 16,
                       row_start=torch.zeros(3, dtype=torch.int32))
    k = torch.zeros(3, 8, 16, 64, dtype=torch.uint8)
    meta = torch.zeros(3, 8, 16, 2, 2, dtype=torch.float16)
    p = akvs.pages(k, k.clone(), meta, meta.clone())
    rows = lambda n, dt, hd=128: torch.zeros(n, 8, hd, dtype=dt)
    for a, b in ((rows(5, F), rows(5, B)), (rows(5, B), rows(5, F)), (rows(4, F), rows(5, F)),
                 (rows(5, F), rows(4, F)), (None, rows(4, B)), (rows(5, B, 64), None),
                 (rows(5, F), rows(5, F, 64))):
        with pytest.raises(ValueError, match="out"):
            akvs.akvs_load_pages(c, p, m, a, b)


def test_pages_fit_the_model(lib):
    """Codes and meta of one width, the model's, and of its KV heads: no call reads past them."""
    u8, f16 = torch.uint8, torch.float16
    k, meta = torch.zeros(3, 8, 16, 64, dtype=u8), torch.zeros(3, 8, 16, 2, 2, dtype=f16)
    thin, one = torch.zeros(3, 8, 16, 32, dtype=u8), torch.zeros(3, 8, 16, 1, 2, dtype=f16)
    for args in ((k, thin, meta, meta), (k, k, one, meta), (k, k, meta, one), (k, k, meta, meta[..., 0]),
                 (thin, thin, meta, meta), (k[..., :48].contiguous(),) * 2 + (meta,) * 2,
                 (k[:, 0].contiguous(),) * 2 + (meta[:, 0].contiguous(),) * 2):
        with pytest.raises(ValueError):
            akvs.pages(*args)
    c = akvs.paged_cfg(2, 2, 1, torch.zeros(4, dtype=torch.int32),
                       torch.zeros(4, 5, dtype=torch.int32), 16)
    for args, m in (((thin, thin, one, one), model()), ((k, k, meta, meta), model(hd=64)),
                    ((k, k, meta, meta), model(hq=16, hkv=16)), ((k, k, meta, meta), model(hkv=4))):
        p = akvs.pages(*args)
        rows = torch.zeros(2, m.n_kv_heads, m.head_dim, dtype=torch.bfloat16)
        q = torch.zeros(2, m.n_q_heads, m.head_dim, dtype=torch.bfloat16)
        moves = torch.zeros(2, dtype=torch.int32)
        for call in (lambda: akvs.akvs_store_pages(rows, rows.clone(), c, p, m),
                     lambda: akvs.akvs_load_pages(c, p, m, rows, rows.clone()),
                     lambda: akvs.akvs_paged_attention(q, c, p, m, q.clone()),
                     lambda: akvs.akvs_move_pages(p, 1, m, moves, moves.clone(), 2)):
            with pytest.raises(ValueError, match="pages"):
                call()


def test_storing_and_attending_check_their_rows(lib):
    """As many rows as the batch's, of the model's type and width."""
    m, F, B = model(), torch.float32, torch.bfloat16
    c = akvs.paged_cfg(2, 5, 3, torch.zeros(4, dtype=torch.int32),
                       torch.zeros(4, 5, dtype=torch.int32), 16,
                       row_start=torch.zeros(3, dtype=torch.int32))
    k = torch.zeros(3, 8, 16, 64, dtype=torch.uint8)
    meta = torch.zeros(3, 8, 16, 2, 2, dtype=torch.float16)
    p = akvs.pages(k, k.clone(), meta, meta.clone())
    z = lambda *s, dt=B: torch.zeros(s, dtype=dt)
    ok = z(5, 8, 128)
    for x in (z(4, 8, 128), z(5, 8, 64), z(5, 8, 128, dt=F), z(5, 512)):
        for args in ((x, ok), (ok, x)):
            with pytest.raises(ValueError, match="^[kv]:"):
                akvs.akvs_store_pages(*args, c, p, m)
    q, out, lse = z(5, 24, 128), z(5, 24, 128), z(5, 24, dt=F)
    for bad, name in ((z(4, 24, 128), "q"), (z(5, 24, 128, dt=F), "q"), (z(4, 24, 128), "out"),
                      (z(5, 24, 128, dt=F), "out"), (z(4, 24, dt=F), "lse"), (z(5, 24), "lse")):
        a = dict(q=q, out=out, lse=lse)
        a[name] = bad
        with pytest.raises(ValueError, match=name + ":"):
            akvs.akvs_paged_attention(a["q"], c, p, m, a["out"], a["lse"])
