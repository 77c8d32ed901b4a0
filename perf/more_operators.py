"""The paged KV cache: rows that join it with their position rotation, rows read back, and the attentions that read it.

The cache is a pool of pages, [n_pages, h_kv, page, head_dim] bf16 for K and for V, and a table [batch, pages] of
page numbers: position p of sequence b is row p % page of page table[b, p // page].  A negative entry stands for a page
that is not there (given back behind a window), whose positions are hidden.  Four kinds of case, each a call that a
serving loop makes:

  append  new tokens' queries, keys and values as a projection leaves them: queries and keys rotated to their
          positions, keys and values written into their pages.  A block of n tokens behind every sequence's context, or
          prompts of unequal lengths packed one behind the other.
  read    a context's rows as [batch, h_kv, rows, head_dim]: the keys for a selection of the drafter's view, or both.
  verify  n_q queries at positions T .. T + n_q - 1 over keys [0, T + i]; n_q = 1 decodes one token.
  draft   one drafter pass j over a sparse view: the kept positions and the drafted rows T .. T + j.

Sizes: contexts of 1K to 128K, pages of 16 to 256 rows, budgets 64 to 8192, blocks of 1 to 21 queries, GQA groups
1, 4 and 8, head_dim 64 and 128, pools with a page's heads or its rows outermost, bf16 and fp32 projections.
"""

from __future__ import annotations

import math

import torch

own = False          # True: run() calls the package's operators; False: their plain form

BF, F32 = torch.bfloat16, torch.float32
TINY, GQA4, GQA8, MHA = (8, 2, 64), (32, 8, 128), (32, 4, 128), (32, 32, 128)
ELEMENTS = 8 * 8 * 16384 * 128        # of K (and of V) in the largest cases
APPENDED = 4 * 8192 * 48 * 128        # of queries, keys and values together


def _case(kind, batch, heads, t_ctx, n, page, ragged=0.0, rows_outer=False, **kw):
    h_q, h_kv, d = heads
    return dict(kind=kind, batch=batch, h_q=h_q, h_kv=h_kv, d=d, t_ctx=t_ctx, n=n, page=page, ragged=ragged,
                rows_outer=rows_outer, **kw)


def listed():
    return [
        # the smallest append: one sequence's next token
        dict(_case("append", 1, TINY, 1023, 1, 16, dtype="bf16", packed=False, pairs=False), name="append_tiny"),
        # a serving batch's next tokens behind unequal contexts
        dict(_case("append", 64, GQA4, 1000, 1, 16, 0.9, dtype="bf16", packed=False, pairs=False), name="append_decode_b64"),
        # prompts of unequal lengths packed one behind the other, fp32 projections, neighbours paired
        dict(_case("append", 7, GQA8, 0, 2111, 32, 0.8, True, dtype="fp32", packed=True, pairs=True), name="append_prompts_b7"),
        # a batch of whole prompts
        dict(_case("append", 4, GQA4, 0, 8192, 16, dtype="bf16", packed=False, pairs=False), name="append_8k_b4"),
        # a few thousand rows of K and V, odd lengths
        dict(_case("read", 3, TINY, 5001, 5001, 16, 0.3, with_v=True), name="read_5001_b3"),
        # the keys of a whole context, for a selection of the drafter's view
        dict(_case("read", 8, GQA4, 16384, 16384, 64, with_v=False), name="read_keys_16k_b8"),
        # decoding, the smallest: one short sequence
        dict(_case("verify", 1, TINY, 1023, 1, 16, window=0), name="decode_1k_tiny"),
        # decoding a serving batch of unequal lengths, small pages
        dict(_case("verify", 32, GQA4, 8000, 1, 16, 0.8, window=0), name="decode_8k_b32_ragged"),
        # decoding one token behind a long document
        dict(_case("verify", 1, GQA4, 131071, 1, 64, 0.0, True, window=0), name="decode_128k_b1"),
        # the paper's longest draft, groups of 8 (168 query rows a KV head), unequal odd lengths
        dict(_case("verify", 5, GQA8, 9001, 21, 32, 0.5, window=0), name="verify_gamma20_ragged"),
        # the smallest drafter pass
        dict(_case("draft", 1, TINY, 1024, 2, 16, budget=256), name="draft_1k_tiny"),
        # the serving batch's drafter pass
        dict(_case("draft", 8, GQA4, 16384, 4, 16, budget=512), name="draft_16k_b8"),
    ]


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, odd ones among them."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["append", "append", "append", "read", "verify", "verify", "verify", "verify", "draft", "draft"])
    heads = rng.choice([TINY, GQA4, GQA4, GQA8, MHA])
    page, rows_outer = rng.choice([16, 16, 32, 64, 128, 256]), rng.random() < 0.3
    if kind == "append":
        per_token = (heads[0] + 2 * heads[1]) * heads[2]
        packed, dtype = rng.random() < 0.4, rng.choice(["bf16", "bf16", "fp32"])
        n = log(2, 4000) if packed else rng.choice([1, 1, 6, 21, log(1, 8192)])
        batch = log(1, max(1, min(64, APPENDED // per_token // n // (2 if dtype == "fp32" else 1))))
        t = 0 if n > 21 and rng.random() < 0.5 else log(1, max(1, min(16384, ELEMENTS // 2 // (heads[1] * heads[2] * batch))))
        return _case(kind, batch, heads, t, n, page, rng.choice([0.0, 0.5, 0.9]) if batch > 1 else 0.0, rows_outer,
                     dtype=dtype, packed=packed, pairs=rng.random() < 0.3)
    n = rng.choice([1, 1, 1, 4, 6, 6, 9, 13, 21]) if kind == "verify" else rng.randint(0, 19)
    rows = n * heads[0] // heads[1] if kind == "verify" else 1
    most = ELEMENTS // (heads[1] * heads[2]) * 24 // max(24, rows)
    t = log(1 if kind == "read" else 128, min({"read": 16384, "verify": 131072, "draft": 32768}[kind], most))
    batch = log(1, max(1, min(64, most // t)))
    c = _case(kind, batch, heads, t, n, page, rng.choice([0.0, 0.5, 0.9]) if batch > 1 else 0.0, rows_outer)
    if kind == "read":
        c.update(n=t, with_v=rng.random() < 0.5)
    if kind == "verify":
        c["window"] = log(64, t) if rng.random() < 0.2 else 0
    if kind == "draft":
        c["budget"] = min(log(64, 8192), t)
    return c


# ------------------------------------------------------------------------------------ shapes


def _spread(c, most, least):
    """A number for every sequence: most, or spread evenly over [(1 - ragged) most, most]."""
    b = c["batch"]
    if not c["ragged"]:
        return [most] * b
    return [max(least, most - int(i * c["ragged"] * most / (b - 1))) for i in range(b)]


def _lens(c):
    """Context length of every sequence."""
    return _spread(c, c["t_ctx"], 0 if c["kind"] == "append" else 1)


def _counts(c):
    """New tokens of every sequence (append)."""
    return _spread(c, c["n"], 1) if c["packed"] else [c["n"]] * c["batch"]


def _behind(c):
    """Rows behind a context."""
    return {"append": c["n"], "read": 0, "verify": c["n"], "draft": c["n"] + 1}[c["kind"]]


def _pages(c):
    return -(-(c["t_ctx"] + _behind(c)) // c["page"])


def _first_pages(c, t):
    """Pages [1, this) of a sequence are not there: behind the window, but for the first one."""
    return max(1, (t - c["window"]) // c["page"]) if c.get("window") else 1


def _keys(c, t):
    """Keys that the block's last query sees."""
    return t + c["n"] - (_first_pages(c, t) - 1) * c["page"]


def work(c):
    b, hq, hkv, d, n, kind = (c[k] for k in ("batch", "h_q", "h_kv", "d", "n", "kind"))
    if kind == "append":
        rows = sum(_counts(c)) * (hq + 2 * hkv)
        return dict(bytes=rows * d * (6 if c["dtype"] == "fp32" else 4), flops=rows * d * 3)
    lens = _lens(c)
    if kind == "read":
        rows = sum(min(n, t) for t in lens) * hkv * (2 if c["with_v"] else 1)
        return dict(bytes=rows * d * 4, flops=rows)
    qo = b * hq * (n if kind == "verify" else 1)
    keys = sum(_keys(c, t) if kind == "verify" else min(c["budget"], t) + n + 1 for t in lens) * hkv
    view = b * hkv * (c["budget"] + 1) * 4 if kind == "draft" else 0
    return dict(bytes=keys * 4 * d + qo * (4 * d + 4) + view, flops=4 * d * keys * hq // hkv * (n if kind == "verify" else 1))


# ------------------------------------------------------------------------------------ inputs


def _rows(g, shape, keys):
    """Rows as a model makes them: keys whose channels differ in size (a few are several times the others), values
    N(0, 1), now and then a row several times larger.  shape: [any, heads, any, head_dim]."""
    x = torch.randn(shape, generator=g, device="cuda")
    if keys:
        x *= torch.exp(0.4 * torch.randn(shape[1], 1, shape[3], generator=g, device="cuda"))
    else:
        x *= torch.where(torch.rand(shape[0], shape[1], shape[2], 1, generator=g, device="cuda") < 0.01, 6.0, 1.0)
    return x


class State:
    pass


def prepare(c, seed):
    g = torch.Generator("cuda").manual_seed(int(seed))
    s = State()
    s.case = c
    b, hq, hkv, d, t, n, kind, page = (c[k] for k in ("batch", "h_q", "h_kv", "d", "t_ctx", "n", "kind", "page"))
    lens, per = _lens(c), _pages(c)
    s.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    # a pool somewhat larger than the batch's pages, which lie anywhere in it; entries behind a sequence's rows are -1
    n_pages = b * per + per // 8 + 1
    order = torch.randperm(n_pages, generator=g, device="cuda")[:b * per].view(b, per).int()
    new = torch.tensor(_counts(c) if kind == "append" else [_behind(c)] * b, device="cuda")
    slot = torch.arange(per, device="cuda")
    used = slot * page < (s.lens + new).view(b, 1)
    if c.get("window"):
        gone = torch.tensor([_first_pages(c, x) for x in lens], device="cuda").view(b, 1)
        used &= (slot == 0) | (slot >= gone)
    s.table = torch.where(used, order, -1).int().contiguous()
    shape = (n_pages, hkv, page, d)
    s.k, s.v = _rows(g, shape, True).to(BF), _rows(g, shape, False).to(BF)
    if c["rows_outer"]:                   # [n_pages, page, h_kv, d] in memory
        s.k, s.v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (s.k, s.v))
    if kind == "append":
        s.dtype = F32 if c["dtype"] == "fp32" else BF
        total = sum(_counts(c)) if c["packed"] else b * n
        # the projection's output, [token, heads, d]
        qkv = torch.randn(total, hq + 2 * hkv, d, generator=g, device="cuda").to(s.dtype)
        s.starts = None
        if c["packed"]:
            ends = torch.tensor(_counts(c), device="cuda").cumsum(0)
            s.starts = torch.cat([ends.new_zeros(1), ends]).int()
            s.q_rows, s.k_rows, s.v_rows = qkv.transpose(0, 1).split([hq, hkv, hkv])
            s.q_out = torch.empty(hq, total, d, dtype=BF, device="cuda")
        else:
            s.q_rows, s.k_rows, s.v_rows = qkv.view(b, n, -1, d).transpose(1, 2).split([hq, hkv, hkv], dim=1)
            s.q_out = torch.empty(b, hq, n, d, dtype=BF, device="cuda")
        s.inv_freq = 500000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
    if kind == "read":
        s.out = [torch.zeros(b, hkv, n, d, dtype=BF, device="cuda") for _ in range(2 if c["with_v"] else 1)]
    if kind == "verify":
        s.q = torch.randn(b, hq, n, d, generator=g, device="cuda").to(BF)
    if kind == "draft":
        s.q = torch.randn(b, hq, d, generator=g, device="cuda").to(BF)
        # a view keeps the first positions, the last and, in between, some of the rest, ascending
        score = torch.rand(b, hkv, t, generator=g, device="cuda")
        pos = torch.arange(t, device="cuda")
        length = s.lens.view(b, 1, 1)
        score = torch.where((pos < 4) | (pos >= length - c["budget"] // 4), score + 1, score)
        score = torch.where(pos < length, score, -1.0)
        top, idx = score.topk(c["budget"], dim=-1)
        idx = torch.where(top >= 0, idx, 1 << 30).sort(-1).values
        s.idx = torch.where(idx < 1 << 30, idx, -1).int()
        s.count = (s.idx >= 0).sum(-1).int()
    if own:
        import paper_2606_00144_gb300 as bd

        s.bd = bd
        s.shape = bd.make_shape(b, hq, hkv, d, t, t + _behind(c), s.lens if c["ragged"] else None)
        s.cache = bd.PagedCache(s.k, s.v)
        if kind == "append":
            s.rope = bd.Rope(s.inv_freq, interleaved=c["pairs"])
        if kind in ("verify", "draft"):
            op = bd.BD_OP_PAGED_VERIFY if kind == "verify" else bd.BD_OP_PAGED_DRAFT
            s.ws = bd.Workspace(bd.bd_workspace_size(s.shape, op, c.get("budget", 0), n if kind == "verify" else n + 1))
            s.o = torch.empty_like(s.q)
            s.lse = torch.empty(s.q.shape[:-1], dtype=F32, device="cuda")
    return s


# ------------------------------------------------------------------------------------ the passes


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    bd, c, kind = s.bd, s.case, s.case["kind"]
    if kind == "append":
        bd.bd_paged_append(s.shape, s.q_rows, s.k_rows, s.v_rows, s.rope, s.cache, s.table, s.q_out, row_starts=s.starts)
        return {"q": s.q_out, "k": s.k, "v": s.v}
    if kind == "read":
        bd.bd_paged_read(s.shape, s.cache, s.table, s.out[0], s.out[1] if c["with_v"] else None, first_row=c["t_ctx"] - c["n"])
        return {"k": s.out[0], "v": s.out[1]} if c["with_v"] else {"k": s.out[0]}
    if kind == "verify":
        bd.bd_paged_verify_attn(s.shape, s.q, c["n"], s.cache, s.table, s.o, s.lse, s.ws)
    else:
        bd.bd_paged_draft_attn(s.shape, s.q, s.cache, s.table, s.idx, s.count, c["budget"], c["n"], s.o, s.lse, s.ws)
    return {"o": s.o, "lse": s.lse}


def _tokens(s):
    """Sequence and position of every new token, in the order of the rows."""
    c, dev = s.case, s.k.device
    if c["packed"]:
        counts = (s.starts[1:] - s.starts[:-1]).long()
        seq = torch.repeat_interleave(torch.arange(c["batch"], device=dev), counts, output_size=s.q_rows.shape[1])
        return seq, s.lens.long()[seq] + torch.arange(len(seq), device=dev) - s.starts.long()[seq]
    seq = torch.arange(c["batch"], device=dev).repeat_interleave(c["n"])
    return seq, s.lens.long()[seq] + torch.arange(c["n"], device=dev).repeat(c["batch"])


def _rotated(x, cos, sin, pairs):
    """x [..., tokens, d] by the tokens' cos and sin [tokens, d / 2]: elements (2 j, 2 j + 1) or (j, j + d / 2) together."""
    if pairs:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)


def _attend(q, k, v, hidden):
    """softmax(q k^T / sqrt(d)) v and its log-sum-exp over the keys that are not hidden."""
    x = q @ k.transpose(-1, -2) * q.shape[-1] ** -0.5
    x = x.masked_fill(hidden, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - m)
    l = p.sum(-1, keepdim=True)
    return (p @ v) / l, (m + torch.log(l)).squeeze(-1)


def _run_plain(s):
    c, kind = s.case, s.case["kind"]
    b, hq, hkv, d, n, page = (c[k] for k in ("batch", "h_q", "h_kv", "d", "n", "page"))
    dev = s.k.device
    if kind == "append":
        seq, pos = _tokens(s)
        angle = pos.double().unsqueeze(-1) * s.inv_freq
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
        # [heads, tokens, d]
        q, k, v = (x if c["packed"] else x.transpose(0, 1).flatten(1, 2) for x in (s.q_rows, s.k_rows, s.v_rows))
        q = _rotated(q.float(), cos, sin, c["pairs"]).to(BF)
        k = _rotated(k.float(), cos, sin, c["pairs"]).to(BF)
        at = s.table[seq, pos // page].long()
        s.k[at, :, pos % page] = k.transpose(0, 1)
        s.v[at, :, pos % page] = v.to(BF).transpose(0, 1)
        return {"q": q if c["packed"] else q.view(hq, b, n, d).transpose(0, 1), "k": s.k, "v": s.v}
    if kind == "read":
        pos = torch.arange(c["t_ctx"] - n, c["t_ctx"], device=dev)
        at = s.table[:, pos // page].long()                     # [b, n]
        there = (pos < s.lens.view(b, 1)).view(b, 1, n, 1)
        out = []
        for x in (s.k, s.v)[:len(s.out)]:
            rows = x[at.clamp(min=0), :, pos % page].transpose(1, 2)
            out.append(torch.where(there, rows, torch.zeros_like(rows)))
        return dict(zip("kv", out))
    if kind == "verify":
        per = s.table.shape[1]
        at = s.table.long().clamp(min=0)
        k, v = (x[at].transpose(1, 2).reshape(b, hkv, per * page, d).float() for x in (s.k, s.v))
        pos = torch.arange(per * page, device=dev)
        last = s.lens.view(b, 1, 1, 1) + torch.arange(n, device=dev).repeat(hq // hkv).view(1, 1, -1, 1)
        gone = (s.table < 0).repeat_interleave(page, 1).view(b, 1, 1, -1)
        o, lse = _attend(s.q.float().view(b, hkv, hq // hkv * n, d), k, v, (pos > last) | gone)
        return {"o": o.to(BF).view(b, hq, n, d), "lse": lse.view(b, hq, n)}
    kept = torch.where(torch.arange(c["budget"], device=dev) < s.count.unsqueeze(-1), s.idx.long(), 0)
    drafted = s.lens.long().view(b, 1, 1) + torch.arange(n + 1, device=dev)
    pos = torch.cat([kept, drafted.expand(b, hkv, n + 1)], -1)
    at = s.table.long().unsqueeze(1).expand(b, hkv, -1).gather(2, pos // page)
    head = torch.arange(hkv, device=dev).view(1, hkv, 1)
    k, v = s.k[at, head, pos % page].float(), s.v[at, head, pos % page].float()
    slot = torch.arange(c["budget"] + n + 1, device=dev)
    hidden = ((slot < c["budget"]) & (slot >= s.count.unsqueeze(-1))).unsqueeze(2)
    o, lse = _attend(s.q.float().view(b, hkv, hq // hkv, d), k, v, hidden)
    return {"o": o.to(BF).view(b, hq, d), "lse": lse.view(b, hq)}


# ------------------------------------------------------------------------------------ 64 bits


def _turned(x, seq_pos, inv_freq, pairs):
    """Rows [tokens, heads, d] in 64 bits, as complex numbers times e^(i angle)."""
    x = x.double()
    z = torch.complex(x[..., 0::2], x[..., 1::2]) if pairs else torch.complex(*x.split(x.shape[-1] // 2, -1))
    angle = torch.outer(seq_pos.double(), inv_freq).unsqueeze(1)
    z = z * torch.polar(torch.ones_like(angle), angle)
    return torch.view_as_real(z).flatten(-2) if pairs else torch.cat([z.real, z.imag], -1)


def exact(c, seed):
    s = prepare(c, seed)
    kind, b, hq, hkv, d, n, page = (c[k] for k in ("kind", "batch", "h_q", "h_kv", "d", "n", "page"))
    dev, G, lens = s.k.device, hq // hkv, _lens(c)
    if kind == "append":
        counts = _counts(c)
        k, v = s.k.double(), s.v.double()
        q = torch.empty(s.q_out.shape, dtype=torch.float64, device=dev)
        at = 0
        for i in range(b):
            pos = torch.arange(lens[i], lens[i] + counts[i], device=dev)
            rows = slice(at, at + counts[i])
            xq, xk, xv = ((x[:, rows] if c["packed"] else x[i]).transpose(0, 1) for x in (s.q_rows, s.k_rows, s.v_rows))
            (q[:, rows] if c["packed"] else q[i]).copy_(_turned(xq, pos, s.inv_freq, c["pairs"]).transpose(0, 1))
            xk = _turned(xk, pos, s.inv_freq, c["pairs"])
            for j in range(lens[i] // page, (lens[i] + counts[i] - 1) // page + 1):
                lo, hi = max(lens[i], j * page), min(lens[i] + counts[i], (j + 1) * page)
                to, src = slice(lo - j * page, hi - j * page), slice(lo - lens[i], hi - lens[i])
                k[s.table[i, j], :, to] = xk[src].transpose(0, 1)
                v[s.table[i, j], :, to] = xv[src].double().transpose(0, 1)
            at += counts[i]
        return {"q": q, "k": k, "v": v}

    def unit(pool, i, h, rows):
        """Rows of one (sequence, KV head) in 64 bits."""
        return pool[:, h][s.table[i].long()[rows // page], rows % page].double()

    if kind == "read":
        out = [torch.zeros(b, hkv, n, d, dtype=torch.float64, device=dev) for _ in s.out]
        first = c["t_ctx"] - n
        for x, pool in zip(out, (s.k, s.v)):
            for i in range(b):
                rows = torch.arange(first, lens[i], device=dev)
                for h in range(hkv):
                    x[i, h, :len(rows)] = unit(pool, i, h, rows)
        return dict(zip("kv", out))
    o = torch.empty(s.q.shape, dtype=torch.float64, device=dev)
    lse = torch.empty(s.q.shape[:-1], dtype=torch.float64, device=dev)
    for i in range(b):
        for h in range(hkv):
            heads = slice(h * G, (h + 1) * G)
            if kind == "verify":
                rows = torch.arange(lens[i] + n, device=dev)
                if c["window"]:
                    rows = rows[(rows < page) | (rows >= _first_pages(c, lens[i]) * page)]
                last = lens[i] + torch.arange(n, device=dev).repeat(G)
            else:
                kept = s.idx[i, h, :int(s.count[i, h])].long()
                rows = torch.cat([kept, lens[i] + torch.arange(n + 1, device=dev)])
                last = torch.full((G,), c["t_ctx"] + n + 1, device=dev)
            k, v = unit(s.k, i, h, rows), unit(s.v, i, h, rows)
            x = s.q[i, heads].double().reshape(-1, d) @ k.T / math.sqrt(d)
            x[rows.unsqueeze(0) > last.unsqueeze(1)] = -math.inf
            lse[i, heads] = torch.logsumexp(x, 1).view(lse[i, heads].shape)
            o[i, heads] = (torch.softmax(x, 1) @ v).view(o[i, heads].shape)
    return {"o": o, "lse": lse}
