"""Plain 64-bit definitions of the operators over a shared context, a row and a head at a time,
and the error bounds that their tests use."""
import math

import torch


def rows_of(row_start, b):
    return int(row_start[b]), int(row_start[b + 1])


def seen_by(n, own_len, i):
    """Own keys that row i of a request's n rows sees."""
    return min(max(own_len - n + i + 1, 0), own_len)


def attention(q, kp, vp, ko, vo, row_start, own_len):
    """(out, lse, mass, reach) in 64 bits: mass = sum_j p_j |v_j| (what rounded probabilities are
    off against), reach = the largest sum_d |q_d k_d| / sqrt(hd) of a key the row sees."""
    n, hq, hd = q.shape
    G = hq // kp.shape[1]
    q, kp, vp, ko, vo = (t.double().cpu() for t in (q, kp, vp, ko, vo))
    out = torch.full((n, hq, hd), math.nan, dtype=torch.float64)
    lse = torch.full((n, hq), math.nan, dtype=torch.float64)
    mass, reach = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(len(own_len)):
        r0, r1 = rows_of(row_start, b)
        for r in range(r0, r1):
            s = seen_by(r1 - r0, int(own_len[b]), r - r0)
            k = torch.cat((kp, ko[b, :s])).repeat_interleave(G, dim=1)
            v = torch.cat((vp, vo[b, :s])).repeat_interleave(G, dim=1)
            if k.shape[0] == 0:
                out[r], lse[r] = 0.0, -math.inf
                continue
            sc = (q[r][None] * k).sum(-1) / math.sqrt(hd)
            lse[r] = torch.logsumexp(sc, 0)
            p = torch.exp(sc - lse[r])
            out[r] = (p[..., None] * v).sum(0)
            mass[r] = (p[..., None] * v.abs()).sum(0)
            reach[r] = (q[r].abs()[None] * k.abs()).sum(-1).max(0).values / math.sqrt(hd)
    return out, lse, mass, reach


def weights(q, lse, kp, ko, row_start, own_len, own_rows):
    """Weight that each key received, [Hkv][P] and [B][Hkv][own_rows], and the same sums of
    (1 + reach + |lse|) (see weights_bound)."""
    hq, hd = q.shape[1:]
    hkv = kp.shape[1]
    G, B = hq // hkv, len(own_len)
    q, kp, ko, lse = (t.double().cpu() for t in (q, kp, ko, lse))
    wp = torch.zeros(2, hkv, kp.shape[0], dtype=torch.float64)
    wo = torch.zeros(2, B, hkv, own_rows, dtype=torch.float64)

    def give(w, r, k):  # k [n][Hkv][hd]
        kk = k.repeat_interleave(G, dim=1)
        p = torch.exp((q[r][None] * kk).sum(-1) / math.sqrt(hd) - lse[r])
        far = 1 + (q[r].abs()[None] * kk.abs()).sum(-1) / math.sqrt(hd) + lse[r].abs()
        w[0] += p.view(-1, hkv, G).sum(-1).T
        w[1] += (p * far).view(-1, hkv, G).sum(-1).T

    for b in range(B):
        r0, r1 = rows_of(row_start, b)
        for r in range(r0, r1):
            s = seen_by(r1 - r0, int(own_len[b]), r - r0)
            if math.isinf(float(lse[r, 0])):
                continue
            give(wp, r, kp)
            give(wo[:, b, :, :s], r, ko[b, :s])
    return wp[0], wo[0], wp[1], wo[1]


def score_bound(reach, hd):
    """Error of a score formed in 32 bits: hd products added in any order, then scaled, the
    running maximum subtracted and its logarithm's base changed (8 more roundings of values
    no larger than reach)."""
    return (hd + 8) * 2.0 ** -24 * reach


def out_bound(out, mass, reach, hd, keys, dtype):
    """|kernel - definition| of an output. Scores off by d change every probability by a factor
    within e^+-d, numerator and denominator both; sums of `keys` terms in 32 bits add
    keys * 2^-24 to each; exponentials 2^-22. In bf16 the probabilities (2^-8, relative)
    and the result are rounded as well."""
    d = 2 * (score_bound(reach, hd)[..., None] + (keys + 16) * 2.0 ** -24 + 2.0 ** -22)
    tol = d * mass + 1e-30
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * mass * (1 + d) + 2.0 ** -8 * (out.abs() + 2 * tol)
    return tol


def lse_bound(lse, reach, hd, keys):
    """As above for log-sum-exp: a score's error, the sum's relative one and two roundings of
    the result and its parts."""
    return score_bound(reach, hd) + (keys + 16) * 2.0 ** -24 + 2.0 ** -22 * (1 + lse.abs())


def weights_bound(w, far, hd, terms):
    """far: sums of p (1 + reach + |lse|): a weight's score is off by score_bound, its exponent's
    terms by a rounding each; `terms` are added in 32 bits."""
    return (hd + 16) * 2.0 ** -24 * far + (terms + 4) * 2.0 ** -24 * w + 1e-30


def norm_rope(x, gain, cos, sin, eps):
    """Per-head RMS norm and rotation of [n][H][hd] in 64 bits, and sum of the magnitudes that a
    result is the difference of."""
    x = x.double().cpu()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double().cpu()
    half = x.shape[-1] // 2
    lo, hi = x[..., :half], x[..., half:]
    c, s = cos[:, None].double().cpu(), sin[:, None].double().cpu()
    a = torch.cat((lo * c - hi * s, hi * c + lo * s), -1)
    m = torch.cat((lo.abs() * c.abs() + hi.abs() * s.abs(), hi.abs() * c.abs() + lo.abs() * s.abs()), -1)
    return a, m


def evict(w, n, keep, first, recent):
    """Kept indices of one head, ascending: forced ones, then the largest weights (equal ones in
    order, NaN last)."""
    if n <= keep:
        return list(range(n))
    mid = list(range(first, n - recent))
    mid.sort(key=lambda j: (math.isnan(w[j]), -w[j] if not math.isnan(w[j]) else 0.0, j))
    return sorted(list(range(first)) + mid[:keep - first - recent] + list(range(n - recent, n)))
