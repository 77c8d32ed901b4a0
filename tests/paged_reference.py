"""Plain 64-bit forms of the paged cache's operators, for the tests, and pools to run them on."""

import math

import torch

BF = torch.bfloat16
UNREAD = 0x7ffffff0          # a table entry that no call may look at (it would be recorded as an error)


class Pool:
    """A pool on the CPU whose pages of a batch lie anywhere: k and v bf16 [n_pages, h_kv, page, d], table int32 [batch, pages].
    rows[i] positions of sequence i are filled; everything else holds NaN."""

    def __init__(self, rows, h_kv, page, d, seed=0, cap=None, layout="heads", k_size=1.0, v_size=1.0):
        g = torch.Generator().manual_seed(seed)
        b, self.page, self.layout = len(rows), page, layout
        self.cap = cap if cap is not None else max(max(rows), 1)
        per = -(-self.cap // page)
        need = [-(-r // page) for r in rows]
        n_pages = sum(need) + 2
        order = torch.randperm(n_pages, generator=g).int()
        self.table = torch.full((b, per), UNREAD, dtype=torch.int32)
        shape = (n_pages, h_kv, page, d)
        self.k, self.v = torch.full(shape, math.nan, dtype=BF), torch.full(shape, math.nan, dtype=BF)
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = order[at:at + n]
            at += n
            for j in range(n):
                live = min(page, rows[i] - j * page)
                e = int(self.table[i, j])
                self.k[e, :, :live] = (torch.randn(h_kv, live, d, generator=g) * k_size).to(BF)
                self.v[e, :, :live] = (torch.randn(h_kv, live, d, generator=g) * v_size).to(BF)

    def cuda(self):
        """(K, V, table) on the GPU, K and V in the pool's layout."""
        def move(x):
            if self.layout == "rows":                      # [n_pages, page, h_kv, d] in memory
                return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
            return x.cuda()
        k, v = move(self.k), move(self.v)
        if self.layout == "both":                          # one tensor holds a page's K and V
            k, v = torch.stack([k, v], 1).unbind(1)
        return k, v, self.table.cuda()

    def unit(self, i, h, rows):
        """K and V rows (a tensor of positions) of one (sequence, KV head), 64 bits; positions of absent pages: NaN."""
        e = self.table[i][rows // self.page].long()
        there = (e >= 0) & (e < self.k.shape[0])
        out = []
        for x in (self.k, self.v):
            y = x[e.clamp(0, x.shape[0] - 1), h, rows % self.page].double()
            out.append(torch.where(there[:, None], y, torch.full_like(y, math.nan)))
        return out[0], out[1], there


def attend(q, k, v, visible):
    """q [r, d], k and v [n, d], visible bool [r, n]: o, lse and sum p |v| / sum p, fp64; a row that sees nothing: 0, -inf, 0.
    Rows that a query does not see have no part in its output, whatever they hold."""
    r, d = q.shape
    o, lse, spread = torch.zeros(r, d, dtype=torch.float64), torch.full((r,), -math.inf, dtype=torch.float64), torch.zeros(r, d, dtype=torch.float64)
    for i in range(r):
        at = visible[i].nonzero().squeeze(1)
        if len(at) == 0:
            continue
        x = (k[at] @ q[i].double()) / math.sqrt(d)
        m = x.max()
        p = torch.exp(x - m)
        o[i], spread[i] = p @ v[at] / p.sum(), p @ v[at].abs() / p.sum()
        lse[i] = m + torch.log(p.sum())
    return o, lse, spread


def check(o, lse, want_o, want_lse, spread, what=""):
    """o (bf16) and lse (fp32) of a call against the 64-bit ones; spread: sum p |v| / sum p.

    An output is rounded to bf16 once: 2^-8 of it at most.  Scores are fp32 sums of at most 128 exact products: with an
    error of 2^-23 of the largest term for each of 8 partial sums, 2^-20 of sum |q k| log2(e) / sqrt(d), which is about 10 for
    these tests' rows and 80 for the sharp ones: 2^-13.7 of a weight at most.  Weights are held in two bf16 terms
    (2^-17), exponentials and sums of them to 2^-21.  Together within 2^-12 of sum p |v|.  The log of the normaliser carries
    the same 2^-13.7 (7.6e-5) and a log."""
    o, lse = o.double().cpu(), lse.double().cpu()
    empty = want_lse == -math.inf
    assert (o[empty] == 0).all() and (lse[empty] == -math.inf).all(), f"{what}: a row that sees nothing"
    o, lse, want_o, want_lse, spread = (x[~empty] for x in (o, lse, want_o, want_lse, spread))
    if not len(o):
        return
    assert torch.isfinite(o).all(), f"{what}: not finite"
    tol = 2.0 ** -8 * want_o.abs() + 2.0 ** -12 * spread + 1e-37
    worst = ((o - want_o).abs() / tol).max().item()
    assert worst <= 1, f"{what}: {worst:.2f} times the tolerance"
    tol = 8e-5 + 1e-5 * want_lse.abs()
    worst = ((lse - want_lse).abs() / tol).max().item()
    assert worst <= 1, f"{what}: lse {worst:.2f} times the tolerance"


def rotate(x, pos, inv_freq, interleaved, scale=1.0):
    """Rows x [..., n, d] at positions pos [n], 64 bits: pairs of the first 2 len(inv_freq) elements turned by pos * inv_freq."""
    x = x.double().clone()
    r = 2 * len(inv_freq)
    angle = pos.double()[:, None] * inv_freq.double()
    c, s = torch.cos(angle) * scale, torch.sin(angle) * scale
    a, b = (x[..., 0:r:2].clone(), x[..., 1:r:2].clone()) if interleaved else (x[..., :r // 2].clone(), x[..., r // 2:r].clone())
    u, w = a * c - b * s, a * s + b * c
    if interleaved:
        x[..., 0:r:2], x[..., 1:r:2] = u, w
    else:
        x[..., :r // 2], x[..., r // 2:r] = u, w
    return x


def rotate_tolerance(x, want, inv_freq, interleaved, scale=1.0):
    """How far a rotated row may be off: a rounding to bf16 (2^-8 of it), and the fp32 steps before: an argument rounded to
    2^-24 of a half turn, a sine and a cosine to 2^-22, two products and a sum rounded to 2^-24: together within 2^-20 of
    the pair's magnitudes."""
    x = x.double().abs()
    r = 2 * len(inv_freq)
    both = torch.zeros_like(x)
    if interleaved:
        both[..., 0:r:2] = both[..., 1:r:2] = x[..., 0:r:2] + x[..., 1:r:2]
    else:
        both[..., :r // 2] = both[..., r // 2:r] = x[..., :r // 2] + x[..., r // 2:r]
    return 2.0 ** -8 * want.abs() + 2.0 ** -20 * abs(scale) * both + 1e-37
