"""What the engine's 4-bit products and paged caches refuse, and the batches they describe."""
import pytest
import torch

from tests.libutil import ensure_built

BF, U8, F16 = torch.bfloat16, torch.uint8, torch.float16


class Shape:
    n_layers, d_model, n_q_heads, n_kv_heads, head_dim, ffn_dim, vocab = 2, 256, 8, 2, 64, 320, 64
    rope_theta, rms_eps, dtype = 1e4, 1e-6, "bf16"


def make_engine(device):
    from paper_2607_21604_amd.runtime import Engine
    w = {k: torch.zeros(8, device=device) for k in ("attn_norm", "w_qkv", "w_o", "mlp_norm",
                                                    "w_gate_up", "w_down")}
    return Engine(Shape, {"layers": [w, w]}, device)


@pytest.fixture(scope="module")
def engine():
    ensure_built()
    return make_engine("cpu")


@pytest.fixture()
def cache(engine):
    from paper_2607_21604_amd.runtime import PagedCache
    return PagedCache(engine, 5, 100, 12, 16)


def bf(*shape):
    return torch.zeros(shape, dtype=BF)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32)


@pytest.mark.parametrize("args", [(0, 10, 3), (1, 0, 3), (1, 10, -1), (1, 10, 3, 48), (1, 10, 3, 8)])
def test_sizes_of_a_cache(engine, args):
    from paper_2607_21604_amd.runtime import PagedCache
    with pytest.raises(ValueError):
        PagedCache(engine, *args)


def test_layout(cache):
    assert cache.max_len == 112 and tuple(cache.table.shape) == (5, 7)
    assert tuple(cache.k.shape) == (2, 12, 2, 16, 32)
    assert tuple(cache.v_meta.shape) == (2, 12, 2, 16, 1, 2)
    assert bool((cache.table == -1).all()) and not cache.len.any() and not cache.ref.any()
    a, b = cache.layers
    assert b.k == a.k + 12 * 2 * 16 * 32 and b.v_meta == a.v_meta + 12 * 2 * 16 * 4
    assert (a.n_pages, a.page_rows) == (12, 16)


def test_batches(cache):
    c = cache.batch(10)
    assert (c.n_req, c.n_rows, c.rows_max, c.n_seq, c.max_pages, c.max_len) == (5, 10, 2, 5, 7, 112)
    c = cache.batch(7, seq=[4, 0, 4], row_start=[0, 3, 3, 6], max_len=40)
    assert (c.n_req, c.n_rows, c.rows_max, c.max_len) == (3, 7, 3, 40)
    c = cache.batch(7, seq=i32(1, 2), row_start=i32(0, 3, 7))
    assert (c.n_req, c.rows_max) == (2, 7)
    for args in ((9,), (4, [0, 1, 2]), (4, [0, 5]), (4, [-1, 0]), (4, i32(0, 1).long()),
                 (4, [0, 1], [0, 2]), (4, [0, 1], [0, 3, 5]), (4, [0, 1], i32(0, 2)),
                 (4, [0, 1], [0, 1, 4], 2), (5, [0], None, None, 113),
                 (5, [0], None, None, -1), (0, []), (0, [], [0])):
        with pytest.raises(ValueError):
            cache.batch(*args)


def test_refusals_of_a_cache(cache):
    c = cache.batch(5)
    k, q = bf(5, 2, 64), bf(5, 8, 64)
    for args in ((2, k, k, c), (-1, k, k, c), (0, k.float(), k, c), (0, k, bf(4, 2, 64), c),
                 (0, k, bf(5, 1, 64), c)):
        with pytest.raises(ValueError):
            cache.store(*args)
    for args, kw in (((2, q, c), {}), ((0, q.float(), c), {}), ((0, bf(4, 8, 64), c), {}),
                     ((0, q, c), dict(out=bf(5, 8, 32))), ((0, q, c), dict(lse=torch.zeros(5, 7))),
                     ((0, q.transpose(0, 1).contiguous().transpose(0, 1), c), {})):
        with pytest.raises(ValueError):
            cache.attention(*args, **kw)
    with pytest.raises(ValueError):
        cache.load(2, c)
    for call in (lambda: cache.fork([0], [1, 2]), lambda: cache.fork([5], [0]),
                 lambda: cache.fork([0], [-1]), lambda: cache.free([5]),
                 lambda: cache.free(torch.zeros(2)), lambda: cache.grow([0, 5], 1),
                 lambda: cache.grow([0, 1], [1]), lambda: cache.grow([0, 1], -1),
                 lambda: cache.grow([0], i32(1, 2)), lambda: cache.grow([0, 1], [1, -1])):
        with pytest.raises(ValueError):
            call()


def test_refusals_of_a_product(engine):
    x, codes, meta = bf(3, 128), torch.zeros((6, 64), dtype=U8), torch.zeros((6, 2, 2), dtype=F16)
    for args, kw in (((x, codes.int(), meta), {}), ((x, codes, meta.float()), {}),
                     ((x, codes, meta[:5].contiguous()), {}), ((bf(3, 64), codes, meta), {}),
                     ((bf(128), codes, meta), {}), ((x, codes, meta), dict(y=bf(3, 7))),
                     ((x, codes, meta), dict(swiglu=True, y=bf(3, 6))),
                     ((x, codes, meta), dict(resid=bf(3, 6))),
                     ((x, codes, meta), dict(resid=torch.zeros(3, 5))),
                     ((x, codes, meta), dict(swiglu=True, resid=torch.zeros(3, 3))),
                     ((x, codes, meta), dict(resid=torch.zeros(3, 6), y_dtype=BF)),
                     ((x, codes, meta), dict(resid=torch.zeros(3, 6), y=bf(3, 6)))):
        with pytest.raises(ValueError):
            engine.w4_product(*args, **kw)


def test_weights_are_of_whole_groups():
    from paper_2607_21604_amd.runtime import quantize_weight
    for w in (torch.zeros(4, 96), torch.zeros(2, 2, 64)):
        with pytest.raises(ValueError):
            quantize_weight(w)
