"""Decoding from a paged 4-bit cache with 4-bit weights, the calls together as they are used: every
call against its definition in 64 bits, taken of what it was given, sequences that share pages
against a cache of their own, replays of a captured step against eager ones."""
import pytest
import torch

from paper_2607_21604_amd import akvs
from paper_2607_21604_amd.runtime import PagedCache, quantize_weight
from tests import four_bit_ref as ref
from tests.gpu_util import DEV
from tests.libutil import ensure_built
from tests.test_paged_cache import Shape, make_engine

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
HQ, HKV, HD, D, FF = Shape.n_q_heads, Shape.n_kv_heads, Shape.head_dim, Shape.d_model, Shape.ffn_dim


def randn(seed, *shape, std=1.0):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randn(shape, generator=g) * std


def rounded(bound, y, dt):
    return bound + (2.0 ** -8 if dt == BF else 2.0 ** -24) * (y.abs() + bound)


class Decoder:
    """Two layers of 4-bit weights (no norms but the heads') over a paged cache."""

    def __init__(self, n_seq, max_len, n_pages, page_rows):
        ensure_built()
        self.eng = make_engine(DEV)
        self.cache = PagedCache(self.eng, n_seq, max_len, n_pages, page_rows)
        sizes = [((HQ + 2 * HKV) * HD, D), (D, HQ * HD), (2 * FF, D), (D, FF)]
        self.w = [[quantize_weight(randn(9 * i + j, *s, std=s[1] ** -0.5).to(DEV))
                   for j, s in enumerate(sizes)] for i in range(2)]
        self.gains = [[(1 + 0.1 * randn(50 + 2 * i + j, HD)).to(DEV, BF) for j in range(2)]
                      for i in range(2)]
        self.rope = torch.empty((max_len, HD // 2, 2), dtype=F32, device=DEV)
        akvs.akvs_rope_table(max_len, HD, 1e4, self.rope)
        self.want = ref.Tables(self.cache.table.tolist(), [0] * n_seq, [0] * n_pages, page_rows)
        self.keys = [[[None] * n_seq for _ in range(2)] for _ in range(2)]  # [layer][k or v][seq]

    def step(self, x, pos, batch):
        """The rows' last hidden states, fp32; every call's input and output in self.seen."""
        eng, c, a, b = self.eng, self.cache, HQ * HD, (HQ + HKV) * HD
        self.seen = []
        for i in range(2):
            qkv_w, o_w, gu_w, down_w = self.w[i]
            qkv = eng.w4_product(x, *qkv_w, y_dtype=BF)
            q, k, v = eng.qk_norm_rope(qkv[:, :a], qkv[:, a:b], qkv[:, b:], pos, *self.gains[i],
                                       self.rope)
            c.store(i, k, v, batch)
            back = c.load(i, batch, F32)
            out, lse = c.attention(i, q, batch)
            mid = eng.w4_product(out.flatten(1), *o_w, resid=x)
            act = eng.w4_product(mid, *gu_w, swiglu=True)
            end = eng.w4_product(act, *down_w, resid=mid)
            self.seen.append(dict(x=x, qkv=qkv, q=q, k=k, v=v, back=back, out=out, lse=lse, mid=mid,
                                  act=act, end=end))
            x = end
        return x

    def check_tables(self):
        c = self.cache
        assert c.table.tolist() == self.want.table and c.len.tolist() == self.want.len
        assert c.ref.tolist() == self.want.ref

    def grow(self, seq, add):
        served = self.cache.grow(seq, add)
        add = [add] * len(seq) if isinstance(add, int) else list(add)
        want, _, _ = self.want.grow(list(seq), add)
        assert served.tolist() == want
        self.check_tables()
        return want

    def fork(self, src, dst):
        self.cache.fork(src, dst)
        self.want.fork(src, dst)
        for layer in self.keys:
            for x in layer:
                for a, b in zip(src, dst):
                    x[b] = x[a]
        self.check_tables()

    def check(self, seq, start):
        """What the last step saw, its rows being new keys of `seq`."""
        for i, s in enumerate(self.seen):
            s = {n: [y.cpu() for y in x] if isinstance(x, tuple) else x.cpu() for n, x in s.items()}
            qkv_w, o_w, gu_w, down_w = ([y.cpu() for y in x] for x in self.w[i])
            for name, x, w, r in (("qkv", s["x"], qkv_w, 0), ("mid", s["out"].flatten(1), o_w, s["x"]),
                                  ("end", s["act"], down_w, s["mid"])):
                y, tol = ref.product(x, *w)
                y = y + (r.double() if torch.is_tensor(r) else 0)
                assert bool(((s[name].double() - y).abs() <= rounded(tol, y, s[name].dtype)).all())
            y, tol = ref.product(s["mid"], *gu_w)
            (g, u), (tg, tu) = y.chunk(2, 1), tol.chunk(2, 1)
            z = g * torch.sigmoid(g)
            tol = 1.1 * tg * (u.abs() + tu) + tu * z.abs() + 2.0 ** -20 * (1 + g.abs()) * (z * u).abs()
            assert bool(((s["act"].double() - z * u).abs() <= rounded(tol, z * u, BF)).all())
            pools, longest = [], max(self.want.len)
            for j, (new, back) in enumerate(zip((s["k"], s["v"]), s["back"])):
                codes, meta = ref.quantise(new)
                got = back.double()
                exact = ref.values(codes, meta)
                assert bool(((got - exact).abs() <= 2.0 ** -24 * exact.abs()).all())
                pool = [torch.zeros((len(self.want.len), HKV, longest) + codes.shape[2:],
                                    dtype=codes.dtype),
                        torch.zeros((len(self.want.len), HKV, longest) + meta.shape[2:],
                                    dtype=meta.dtype)]
                for b, a in enumerate(seq):
                    mine = [z[start[b]:start[b + 1]] for z in (codes, meta)]
                    old = self.keys[i][j][a]
                    self.keys[i][j][a] = mine if old is None else [torch.cat(z) for z in zip(old, mine)]
                for a, z in enumerate(self.keys[i][j]):
                    if z is not None:
                        for dst, src in zip(pool, z):
                            dst[a, :, :src.shape[0]] = src.transpose(0, 1)
                pools.append(pool)
            r = ref.attention(s["q"], *pools, [[a] for a in range(len(self.want.len))],
                              self.want.len, start, seq)
            err = (s["out"].double() - r["out"]).abs()
            assert bool((err <= ref.out_bound(r, HD, longest)).all())
            err = (s["lse"].double() - r["lse"]).abs()
            assert bool((err <= ref.lse_bound(r, HD, longest)).all())

    def run(self, seq, counts, seed, check=True):
        """New tokens of sequences that have grown by them."""
        n = sum(counts)
        start = [0]
        for x in counts:
            start.append(start[-1] + x)
        pos = torch.tensor([self.want.len[a] - c + j for a, c in zip(seq, counts) for j in range(c)],
                           dtype=torch.int32, device=DEV)
        x = randn(seed, n, D).to(DEV)
        y = self.step(x, pos, self.cache.batch(n, seq, start))
        if check:
            self.check(seq, start)
        return y


@pytest.mark.parametrize("page_rows", [16, 64])
def test_prompts_branches_and_decoding(page_rows):
    d = Decoder(7, 160, 40, page_rows)
    assert d.grow([0, 3], [70, 16]) == [1, 1]
    d.run([0, 3], [70, 16], 1)
    d.fork([0, 0, 3], [1, 2, 4])
    for t in range(3):  # of the branches, then of all of them
        seq = [1, 4, 2] if t < 2 else [4, 0, 1, 2, 3]
        assert d.grow(seq, 1) == [1] * len(seq)
        d.run(seq, [1] * len(seq), 10 + t)
    d.cache.free([0, 4])
    d.want.free([0, 4])
    for layer in d.keys:
        for x in layer:
            x[0] = x[4] = None
    table, refs, moves, want = d.want.compact()
    assert d.cache.compact().tolist() == want
    d.want.table, d.want.ref = table, refs
    d.check_tables()
    assert d.grow([5, 2, 1], [40, 3, 9]) == [1, 1, 1]  # a new prompt beside old ones
    d.run([5, 2, 1], [40, 3, 9], 20)


def test_a_full_pool_and_a_full_sequence():
    d = Decoder(3, 48, 5, 16)
    assert d.grow([0, 1, 2], [48, 20, 1]) == [1, 1, 0]
    assert d.grow([0, 1], 1) == [0, 1]
    d.cache.free([0])
    d.want.free([0])
    assert d.grow([2], 33) == [1]
    d.run([2, 1], [33, 21], 3)


def test_branches_answer_as_sequences_of_their_own():
    """The same bits from shared pages as from pages of each sequence."""
    shared, own = Decoder(4, 128, 40, 16), Decoder(4, 128, 40, 16)
    shared.grow([0], 45)
    shared.run([0], [45], 1, check=False)
    shared.fork([0, 0, 0], [1, 2, 3])
    x = randn(1, 45, D)
    own.grow([0, 1, 2, 3], 45)
    pos = torch.arange(45, dtype=torch.int32, device=DEV)
    for a in range(4):
        own.step(x.to(DEV), pos, own.cache.batch(45, [a]))
    for t in range(4):
        for d in (shared, own):
            d.grow([3, 1, 2], 1)
        a, b = (d.run([3, 1, 2], [1, 1, 1], 30 + t, check=False) for d in (shared, own))
        assert torch.equal(a, b)


def test_a_captured_step():
    """Grow, two layers and a count of the rows' positions in one graph, replayed with eager work
    between: the bits of eager steps."""
    n, seq = 3, [2, 0, 1]
    eager, d = Decoder(3, 128, 30, 16), Decoder(3, 128, 30, 16)
    for e in (eager, d):
        e.grow([0, 1, 2], [20, 31, 5])
        e.run([0, 1, 2], [20, 31, 5], 4, check=False)
    ids = torch.tensor(seq, dtype=torch.int32, device=DEV)
    add = torch.ones(n, dtype=torch.int32, device=DEV)
    pos = torch.tensor([5, 20, 31], dtype=torch.int32, device=DEV)
    batch = d.cache.batch(n, ids)
    x = torch.zeros(n, D, device=DEV)
    keep = [t.clone() for t in (d.cache.table, d.cache.len, d.cache.ref)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        d.cache.grow(ids, add)
        y = d.step(x, pos, batch)
        pos.add_(1)
    for a, b in zip((d.cache.table, d.cache.len, d.cache.ref), keep):
        assert torch.equal(a, b)  # (captured, not run)
    for t in range(20):
        x.copy_(randn(60 + t, n, D))
        g.replay()
        torch.cuda.synchronize()
        eager.grow(seq, 1)
        want = eager.run(seq, [1] * n, 60 + t, check=False)
        assert torch.equal(y, want)
        assert torch.equal(d.cache.table, eager.cache.table)


def test_tokens_of_a_sequence_without_room_are_stored_nowhere():
    """What grow could not serve stays as it was through the step that follows, in its own pages and
    in those that others share, until a grow serves it; eager, then captured."""
    d = Decoder(5, 64, 6, 16)
    c, n = d.cache, HKV * HD
    assert d.grow([0, 3], [40, 20]) == [1, 1]
    d.run([0, 3], [40, 20], 1)
    d.fork([0, 0], [1, 2])  # 3 pages of three sequences, the last of them not full; one page is left
    pools = (c.k, c.v, c.k_meta, c.v_meta)
    k, v = (randn(i, 3, n).to(DEV, BF) for i in (5, 6))
    batch = c.batch(3, [1, 0, 3])
    seq = torch.tensor([1, 0, 3], dtype=torch.int32, device=DEV)
    add = torch.ones(3, dtype=torch.int32, device=DEV)

    def step():
        served = c.grow(seq, add)
        for i in range(2):
            c.store(i, k, v, batch)
        return served

    def check(before, served, want):
        assert served.tolist() == want
        d.check_tables()
        after = [x.clone() for x in pools]
        for x, y in zip(after, before):  # all but the rows that went in are as before
            for b, (a, ok) in enumerate(zip((1, 0, 3), want)):
                if ok:
                    j = d.want.len[a] - 1
                    page = d.want.table[a][j // 16]
                    assert not torch.equal(x[:, page, :, j % 16], y[:, page, :, j % 16])
                    if page in moved:
                        x[:, page] = y[:, page]
                    x[:, page, :, j % 16] = y[:, page, :, j % 16]
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))

    # the copy for sequence 1 takes the last page; 0, whose page 2 shares, gets none; 3 has room
    # (one that needs no page is served)
    before = [x.clone() for x in pools]
    got = step()
    want, moves, _ = d.want.grow([1, 0, 3], [1, 1, 1])
    moved = [b for _, b in moves]
    assert want == [1, 0, 1]
    check(before, got, want)
    before = [x.clone() for x in pools]
    got = step()
    want, moves, _ = d.want.grow([1, 0, 3], [1, 1, 1])
    moved = []
    assert want == [1, 0, 1] and not moves
    check(before, got, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for t in range(3):
        if t == 2:  # then there is room
            c.free([2])
            d.want.free([2])
        k.copy_(randn(20 + t, 3, n))
        before = [x.clone() for x in pools]
        g.replay()
        torch.cuda.synchronize()
        want, moves, _ = d.want.grow([1, 0, 3], [1, 1, 1])
        assert want == [1, int(t == 2), 1] and not moves
        check(before, got, want)


@pytest.mark.parametrize("ends", [[0], [0, 1]])
def test_a_sequence_without_room_begins_anew(ends):
    """One that never had room becomes a branch, ended before or not: its tokens are stored."""
    d = Decoder(3, 64, 2, 16)
    c = d.cache
    assert d.grow([0, 1], [17, 16]) == [1, 0]
    k, v = (randn(i, 1, HKV * HD).to(DEV, BF) for i in (5, 6))
    c.free(ends)
    d.want.free(ends)
    d.grow([2], 5)
    d.fork([2], [1])
    c.store(0, k, v, c.batch(1, [1]))  # (sequence 2 has the same page)
    back = c.load(0, c.batch(1, [2]), F32)
    for x, y in zip(back, (k, v)):
        want = ref.values(*ref.quantise(y.view(1, HKV, HD).cpu()))
        assert torch.equal(x.cpu(), want.float())


def test_calls_with_lists_do_not_wait_for_the_device():
    """Lists and numbers are copied without a wait."""
    d = Decoder(4, 64, 8, 16)
    x, c = randn(1, 3, HKV * HD).to(DEV, BF), d.cache
    batch = c.batch(3, [0, 1, 3], [0, 1, 2, 3])
    torch.cuda.synchronize()
    torch.cuda.set_sync_debug_mode("error")
    try:
        served = c.grow([0, 3], [20, 3])
        c.fork([0], [1])
        c.grow([0, 1, 3], 1)
        c.store(1, x, x, batch)
        c.free([3])
        c.free([])
        c.compact()
    finally:
        torch.cuda.set_sync_debug_mode("default")
    assert served.tolist() == [1, 1] and c.len.tolist() == [21, 21, 0, 0]


def test_a_batch_of_lists_is_used_on_another_stream():
    """Made while the current stream is busy, used at once on one that does not wait for it."""
    d, own = Decoder(4, 64, 8, 16), Decoder(4, 64, 8, 16)
    x = randn(1, 3, HKV * HD).to(DEV, BF)
    for e in (d, own):
        e.grow([0, 1, 3], 1)
        e.cache.store(1, x, x, e.cache.batch(3, [0, 1, 3]))
    big = torch.ones(1 << 28, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(4):
        for _ in range(30):
            big.mul_(1.0)
        batch = d.cache.batch(3, [3, 0, 1], [0, 1, 2, 3])
        with torch.cuda.stream(side):
            got = d.cache.load(1, batch, F32)
        side.synchronize()
        want = own.cache.load(1, own.cache.batch(3, [3, 0, 1]), F32)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_lists_are_refused_under_capture():
    """A replay would read a list's copy from memory that is another's by then."""
    c = Decoder(4, 64, 8, 16).cache
    ids = torch.tensor([0, 3], dtype=torch.int32, device=DEV)
    for call in (lambda: c.grow([0], 1), lambda: c.grow(ids, [1, 2]), lambda: c.free([1]),
                 lambda: c.batch(2, [0, 3]), lambda: c.batch(2, ids, [0, 1, 2])):
        g = torch.cuda.CUDAGraph()
        with pytest.raises(ValueError, match="capture"):
            with torch.cuda.graph(g):
                ids.add_(0)
                call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        served = c.grow(ids, 2)
    for t in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert served.tolist() == [1, 1] and c.len.tolist() == [2 + 2 * t, 0, 0, 2 + 2 * t]
