"""Plain 64-bit definitions of the operators that decode from four bits, a row and a head at a
time, the page tables' rules in Python, and the error bounds that their tests use."""
import math

import torch

import oracle

EPS = 2.0 ** -24  # half a step of fp32, relative


def quantise(x):
    """(packed codes, meta) of x [..][n] (CPU tensor), by the oracle."""
    codes, meta = oracle.quantize_g64(x.float().numpy(), 4)
    return torch.from_numpy(oracle.pack_codes(codes, 4)), torch.from_numpy(meta)


def parts(codes, meta):
    """(codes 0..15, scale, zero), 64-bit, [..][n] each."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).double()
    m = meta.double().repeat_interleave(64, dim=-2)
    return c, m[..., 0], m[..., 1]


def values(codes, meta):
    c, s, z = parts(codes, meta)
    return s * c + z


def place(table, page_rows, n_pages, j):
    """(page or -1, row) of key j of a sequence."""
    page = int(table[j // page_rows])
    return (page if 0 <= page < n_pages else -1), j % page_rows


def keys_of(pages, table, n):
    """Codes and meta (scale, zero) parts of keys 0..n-1, [n][Hkv][hd]; missing pages: 0."""
    codes, meta = pages
    out = []
    for j in range(n):
        page, at = place(table, codes.shape[2], codes.shape[0], j)
        if page < 0:
            out.append(tuple(torch.zeros(codes.shape[1], codes.shape[3] * 2, dtype=torch.float64)
                             for _ in range(3)))
        else:
            out.append(parts(codes[page, :, at], meta[page, :, at]))
    return [torch.stack(x) for x in zip(*out)]


def attention(q, k_pages, v_pages, table, lens, row_start, seq):
    """dict of out, lse and, per output, what its bound is made of (top: at least the largest scale of
    a value of the sequence). All tensors on the CPU."""
    n, hq, hd = q.shape
    hkv = k_pages[0].shape[1]
    G = hq // hkv
    q = q.double()
    r = {"out": torch.full((n, hq, hd), math.nan, dtype=torch.float64)}
    for x in ("mass", "coarse", "fine", "top"):
        r[x] = torch.zeros(n, hq, hd, dtype=torch.float64)
    r["lse"] = torch.full((n, hq), math.nan, dtype=torch.float64)
    r["reach"] = torch.zeros(n, hq, dtype=torch.float64)
    for b in range(len(row_start) - 1):
        r0, r1 = int(row_start[b]), int(row_start[b + 1])
        sq = int(seq[b])
        known = 0 <= sq < len(lens)
        ln = int(lens[sq]) if known else 0
        if r1 > r0 and ln:
            kc, ks, kz = keys_of(k_pages, table[sq], ln)
            vc, vs, vz = keys_of(v_pages, table[sq], ln)
        for i in range(r0, r1):
            seen = min(max(ln - r1 + i + 1, 0), ln)
            if seen == 0:
                r["out"][i], r["lse"][i] = 0.0, -math.inf
                continue
            up = lambda x: x[:seen].repeat_interleave(G, dim=1)
            s, z, c = up(ks), up(kz), up(kc)
            sc = (q[i][None] * (s * c + z)).sum(-1) / math.sqrt(hd)
            r["lse"][i] = torch.logsumexp(sc, 0)
            p = torch.exp(sc - r["lse"][i])[..., None]
            x = up(vs) * up(vc) + up(vz)
            r["out"][i] = (p * x).sum(0)
            r["mass"][i] = (p * x.abs()).sum(0)
            r["coarse"][i] = (p * up(vs).abs() * (up(vc) - 8).abs()).sum(0)
            r["fine"][i] = (p * (40 * up(vs).abs() + up(vz).abs())).sum(0)
            r["top"][i] = vs.nan_to_num(0, 0, 0).abs().max() + r["mass"][i].nan_to_num(0, 0, 0).max()
            r["reach"][i] = (q[i].abs()[None] * (60 * s.abs() + z.abs())).sum(-1).max(0).values \
                / math.sqrt(hd)
    return r


def attention_by_heads(q, k_pages, v_pages, table, lens, row_start, seq):
    """What attention() gives, a request's KV head at a time: for many rows or keys."""
    n, hq, hd = q.shape
    hkv = k_pages[0].shape[1]
    G = hq // hkv
    r = {"out": torch.full((n, hq, hd), math.nan, dtype=torch.float64)}
    for x in ("mass", "coarse", "fine", "top"):
        r[x] = torch.zeros(n, hq, hd, dtype=torch.float64)
    r["lse"] = torch.full((n, hq), math.nan, dtype=torch.float64)
    r["reach"] = torch.zeros(n, hq, dtype=torch.float64)
    for b in range(len(row_start) - 1):
        r0, r1, sq = int(row_start[b]), int(row_start[b + 1]), int(seq[b])
        ln = int(lens[sq]) if 0 <= sq < len(lens) else 0
        if r1 == r0:
            continue
        if ln == 0:
            r["out"][r0:r1], r["lse"][r0:r1] = 0.0, -math.inf
            continue
        at = [place(table[sq], k_pages[0].shape[2], k_pages[0].shape[0], j) for j in range(ln)]
        page, row = (torch.tensor(x) for x in zip(*at))
        there = (page >= 0)[:, None]
        seen = (torch.arange(ln - r1 + r0, ln) + 1).clamp(min=0)
        hidden = (torch.arange(ln)[None] >= seen[:, None]).repeat_interleave(G, 0)
        none = (seen == 0).repeat_interleave(G)
        for h in range(hkv):
            (kc, ks, kz), (vc, vs, vz) = (
                [torch.where(there, x, 0.0) for x in parts(p[0][page.clamp(min=0), h, row],
                                                           p[1][page.clamp(min=0), h, row])]
                for p in (k_pages, v_pages))
            rows, heads = slice(r0, r1), slice(h * G, (h + 1) * G)
            qh = q[rows, heads].double().reshape(-1, hd)
            sc = (qh @ (ks * kc + kz).T / math.sqrt(hd)).masked_fill(hidden, -math.inf)
            lse = torch.logsumexp(sc, 1)
            p = torch.exp(sc - torch.where(none, 0.0, lse)[:, None])
            reach = (qh.abs() @ (60 * ks.abs() + kz.abs()).T / math.sqrt(hd)).masked_fill(hidden, 0)
            mass = p @ (vs * vc + vz).abs()
            big = torch.where(none[:, None], 0.0, mass).max(-1, keepdim=True).values
            for name, x in (("out", p @ (vs * vc + vz)), ("lse", lse), ("mass", mass),
                            ("coarse", p @ (vs.abs() * (vc - 8).abs())),
                            ("fine", p @ (40 * vs.abs() + vz.abs())), ("reach", reach.max(1).values),
                            ("top", (vs.abs().max() + big).expand_as(mass))):
                r[name][rows, heads] = x.view(r[name][rows, heads].shape)
    return r


def score_bound(reach, hd):
    """Error of a score formed in 32 bits from codes: x = scale (c + 16) + (zero - 16 scale) with codes
    taken as 16 + c (or c), at most 64 products of q and up to 31, and 16 times q's sum, are added
    per group (66 roundings of up to 47 sum |q|), q's sum itself (64 roundings) is multiplied with 16
    scale and zero; scaling, the groups' sum and the logarithm's base are 8 more. reach = sum |q|
    (60 scale + |zero|): 66 * 47 + 64 * 16 + 8 * 31 = 4374 scale < 100 * 60, 72 |zero| < 100."""
    return 100 * EPS * reach


def out_bound(r, hd, keys):
    """|kernel - definition| of an output. Scores off by d change each probability by a factor
    within e^+-d, numerator and denominator both; exponentials 2^-22. fp16 rounds (2^-11 each) either
    p scale, which meets the code less 8 (coarse; the constant's share is taken of the rounded
    numbers), or p and the value (mass twice), then split keys' outputs. What lies below fp16's
    smallest is lost, 2^-25 of p scale 2^(7 - e) / 16 at worst with 2^e at most twice the largest
    scale, times a code of at most 8 from the middle: 2^-25 2^-7 16 8 2 = 2^-24 of the largest scale
    a key; 2^-32 of a value for p. Sums of `keys` terms in 32 bits add keys * 2^-24 of what is added:
    p scale (1024 + c) and its share (2100 scale: fine has 40, so 53 of it). The result is rounded
    to bf16."""
    d = 2 * (score_bound(r["reach"], hd)[..., None] + 2.0 ** -22)
    tol = d * r["mass"] + (keys + 24) * EPS * (53 * r["fine"] + r["mass"]) + 1e-30
    tol = tol + 2.0 ** -11 * (2 * r["coarse"] + 3 * r["mass"]) * (1 + d)
    tol = tol + keys * 2.0 ** -24 * r["top"]
    return tol + 2.0 ** -8 * (r["out"].abs() + tol)


def lse_bound(r, hd, keys):
    return score_bound(r["reach"], hd) + (keys + 16) * EPS + 2.0 ** -22 * (1 + r["lse"].abs())


def product(x, codes, meta):
    """(W x, its bound) in 64 bits, [rows][n_out]. The bound: x in up to three bf16 parts, 16 + c
    less 24 per group of 64 (3 * 66 roundings of up to 55 scale sum |x|), x's sum (66) with
    24 scale and zero + 8 scale, sums over the groups and parts of the reduction in any order."""
    x = x.double()
    c, s, z = parts(codes, meta)
    w = s * c + z
    groups = x.shape[1] // 64
    y = x @ w.T
    a = x.abs()
    big = a @ s.abs().T, a @ (z.abs() + 8 * s.abs()).T
    bound = EPS * ((3 * 66 * 55 + 66 * 24 + (groups + 24) * 8) * big[0] + (groups + 90) * big[1])
    return y, bound + 1e-30


# ---- page tables -----------------------------------------------------------------------------

class Tables:
    """The rules of the page operators, step by step."""

    def __init__(self, table, lens, ref, page_rows):
        self.table, self.len, self.ref = [list(r) for r in table], list(lens), list(ref)
        self.rows = page_rows

    def used(self, s):
        return min(-(-max(self.len[s], 0) // self.rows), len(self.table[0]))

    def count(self, page, d):
        if 0 <= page < len(self.ref):
            self.ref[page] += d

    def fork(self, src, dst):
        S, empty = len(self.len), [x == 0 for x in self.len]
        for i, (a, b) in enumerate(zip(src, dst)):
            if not (0 <= a < S and 0 <= b < S) or not empty[b] or b in src or b in dst[:i]:
                continue
            for j in range(self.used(a)):
                self.table[b][j] = self.table[a][j]
                self.count(self.table[a][j], 1)
            self.len[b] = max(self.len[a], 0)

    def free(self, seq):
        for i, a in enumerate(seq):
            if not 0 <= a < len(self.len) or a in seq[:i]:
                continue
            for j in range(self.used(a)):
                self.count(self.table[a][j], -1)
                self.table[a][j] = -1
            self.len[a] = 0

    def grow(self, seq, add):
        """(served, moves, counts)"""
        before = list(self.ref)
        free = [i for i, x in enumerate(before) if x <= 0]
        served, moves, taken, asked = [], [], 0, 0
        for i, (a, n) in enumerate(zip(seq, add)):
            ok = 0 <= a < len(self.len) and a not in seq[:i] and n >= 0
            if ok:
                old = max(self.len[a], 0)
                have, want = -(-old // self.rows), -(-(old + n) // self.rows)
                ok = want <= len(self.table[0])
            if not ok:
                served.append(0)
                continue
            copy = 0
            if n > 0 and old % self.rows:
                last = self.table[a][old // self.rows]
                copy = int(0 <= last < len(before) and before[last] > 1)
            need = want - have + copy if n > 0 else 0
            asked += need
            if need and asked > len(free):
                served.append(0)
                continue
            new = free[asked - need:asked]
            if need:
                taken = asked
            if copy:
                moves.append((last, new[0]))
                self.count(last, -1)
            for j, page in enumerate(new):
                self.table[a][(old // self.rows if copy else have) + j] = page
                self.ref[page] = 1
            self.len[a] = old + n
            served.append(1)
        return served, moves, [len(moves), taken]

    def compact(self):
        """(table, ref, moves, counts)"""
        n = sum(x > 0 for x in self.ref)
        src = [i for i, x in enumerate(self.ref) if x > 0 and i >= n]
        dst = [i for i, x in enumerate(self.ref) if x <= 0 and i < n]
        to = dict(zip(src, dst))
        table = [list(r) for r in self.table]
        for s in range(len(table)):
            for j in range(self.used(s)):
                table[s][j] = to.get(table[s][j], table[s][j])
        ref = [x if i < n else 0 for i, x in enumerate(self.ref)]
        for a, b in to.items():
            ref[b] = self.ref[a]
        return table, ref, list(to.items()), [len(src), n]
