"""The 4-bit KV cache: writing rows into it, reading them back, and the two attentions that read it.

A cache row of head_dim elements is held as head_dim 4-bit codes, two to a byte (element 2 j in the
low half of byte j), and one bf16 scale for every group of 32 elements:

    scale = bf16(max |x| / 7),   code = clamp(round(x / scale), -7, 7) + 8,   value = (code - 8) * scale

(the quotient in fp32, rounded half to even; a group that holds a NaN or an infinity has the scale
NaN; a scale of 0 gives codes of 8).  Four kinds of case, each a call that a decoding loop makes:

  append  a block's (or a prefill's) K and V rows written into the cache and read back: the values
          that the cache stands for, as a model that wants them exact would use them.
  read    rows read back: the keys for a re-selection, or both for a prefill over a cached prefix.
  verify  the verifier's block, n_q queries at positions T .. T + n_q - 1 over keys [0, T + i]
          (n_q = 1: ordinary decoding of one token).
  draft   one drafter pass j over a sparse view: the kept positions and the drafted rows T .. T + j.

Sizes: the contexts of the evaluation (1K to 16K) and of a 128K-context model, budgets 256 to 8192,
blocks of 1 to 21 queries, GQA groups 1, 4 and 8, head_dim 64 and 128, sequences of equal and of
unequal lengths, bf16 and fp32 rows.
"""

from __future__ import annotations

import math

import torch

own = False          # True: run() calls the package's operators; False: their plain form

GROUP = 32
BF, F32 = torch.bfloat16, torch.float32
TINY, GQA4, GQA8, MHA = (8, 2, 64), (32, 8, 128), (32, 4, 128), (32, 32, 128)
ELEMENTS = 8 * 8 * 16384 * 128        # of K (and of V) in the largest cases


def _case(kind, batch, heads, t_ctx, n, ragged=0.0, **kw):
    h_q, h_kv, d = heads
    return dict(kind=kind, batch=batch, h_q=h_q, h_kv=h_kv, d=d, t_ctx=t_ctx, n=n, ragged=ragged, **kw)


def listed():
    return [
        # the smallest append: one short sequence's verify block joins the cache
        dict(_case("append", 1, TINY, 1024, 6, dtype="bf16", by_token=False), name="append_tiny"),
        # a serving batch of unequal lengths; rows as a projection leaves them, [batch, row, head, d], in fp32
        dict(_case("append", 8, GQA4, 16380, 6, 0.6, dtype="fp32", by_token=True), name="append_ragged_b8"),
        # a whole prefill written at once
        dict(_case("append", 8, GQA4, 0, 16384, dtype="bf16", by_token=False), name="prefill_16k_b8"),
        # a few thousand rows of both tensors in fp32, odd length
        dict(_case("read", 3, TINY, 5001, 5001, dtype="fp32", with_v=True), name="read_5001_b3"),
        # the keys of a whole context, for a re-selection of the drafter's view
        dict(_case("read", 8, GQA4, 16384, 16384, dtype="bf16", with_v=False), name="read_keys_16k_b8"),
        # the smallest verify block
        dict(_case("verify", 1, TINY, 1024, 6), name="verify_1k_tiny"),
        # ordinary decoding, one token behind a long document
        dict(_case("verify", 1, GQA4, 131071, 1), name="decode_128k_b1"),
        # the serving batch's verify block
        dict(_case("verify", 8, GQA4, 16384, 6), name="verify_16k_b8"),
        # the paper's longest draft, groups of 8 (168 query rows a KV head), unequal odd lengths
        dict(_case("verify", 5, GQA8, 9001, 21, 0.5), name="verify_gamma20_ragged"),
        # the smallest drafter pass
        dict(_case("draft", 1, TINY, 1024, 2, budget=256), name="draft_1k_tiny"),
        # the serving batch's drafter pass
        dict(_case("draft", 8, GQA4, 16384, 4, budget=512), name="draft_16k_b8"),
        # long documents of unequal lengths, a quarter of each kept, deep in the paper's longest draft
        dict(_case("draft", 2, GQA8, 32768, 19, 0.3, budget=8192), name="draft_32k_b2"),
    ]


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, odd ones among them."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["append", "append", "read", "verify", "verify", "verify", "draft", "draft"])
    heads = rng.choice([TINY, GQA4, GQA4, GQA8, MHA])
    per_row = heads[1] * heads[2]
    n = rng.choice([1, 1, 2, 4, 6, 6, 9, 13, 21]) if kind == "verify" else rng.randint(0, 19)
    rows = n * heads[0] // heads[1] if kind == "verify" else 1
    t_hi = {"append": 16384, "read": 16384, "verify": 131072, "draft": 32768}[kind]
    most = ELEMENTS // per_row * 24 // max(24, rows)
    t = log(1 if kind in ("append", "read") else 128, min(t_hi, most))
    batch = log(1, max(1, min(16, most // t)))
    ragged = rng.choice([0.0, 0.0, 0.5, 0.9]) if batch > 1 and kind != "read" else 0.0
    c = _case(kind, batch, heads, t, n, ragged)
    if kind == "append":
        c.update(n=rng.choice([1, 6, 21, max(1, t // 2), t]), dtype=rng.choice(["bf16", "bf16", "fp32"]),
                 by_token=rng.random() < 0.5)
        if c["dtype"] == "fp32":
            c["n"] = max(1, min(c["n"], t // 2))
        c["t_ctx"] = rng.choice([0, t])
    if kind == "read":
        c.update(n=rng.choice([t, max(1, t // 3)]), dtype=rng.choice(["bf16", "bf16", "fp32"]),
                 with_v=rng.random() < 0.5)
    if kind == "draft":
        c["budget"] = min(log(64, 8192), t)
    return c


# ------------------------------------------------------------------------------------ shapes


def _lens(c):
    """Context length of every sequence: t_ctx, or spread evenly over [(1 - ragged) t_ctx, t_ctx]."""
    b, t = c["batch"], c["t_ctx"]
    if not c["ragged"]:
        return [t] * b
    return [max(0, t - int(i * c["ragged"] * t / (b - 1))) for i in range(b)]


def _t_cap(c):
    return c["t_ctx"] + {"append": c["n"], "read": 0, "verify": c["n"], "draft": c["n"] + 1}[c["kind"]]


def _count(c, t):
    return min(c["budget"], t)


def work(c):
    b, hq, hkv, d, n, k = c["batch"], c["h_q"], c["h_kv"], c["d"], c["n"], c["kind"]
    row = d // 2 + d // GROUP * 2                        # a cache row: codes and scales
    if k in ("append", "read"):
        esize = 4 if c["dtype"] == "fp32" else 2
        rows = b * hkv * n * (2 if k == "append" or c["with_v"] else 1)
        # append: the rows in, the cache rows out, the values out; read: cache rows in, values out
        return dict(bytes=rows * (row + d * esize * (2 if k == "append" else 1)),
                    flops=rows * d * (5 if k == "append" else 2))
    lens, qo = _lens(c), b * hq * (n if k == "verify" else 1)
    keys = sum(t + n if k == "verify" else _count(c, t) + n + 1 for t in lens) * hkv
    view = b * hkv * (c["budget"] + 1) * 4 if k == "draft" else 0
    return dict(bytes=keys * 2 * row + qo * (4 * d + 4) + view,
                flops=4 * d * keys * hq // hkv * (n if k == "verify" else 1))


# ------------------------------------------------------------------------------------ inputs


def _rows(g, shape, keys, dtype):
    """Rows as a model makes them: keys whose channels differ in size (a few are several times the
    others), values N(0, 1), now and then a row several times larger."""
    x = torch.randn(shape, generator=g, device="cuda")
    if keys:
        ch = torch.exp(0.4 * torch.randn(shape[1], 1, shape[3], generator=g, device="cuda"))
        x *= ch
    else:
        x *= torch.where(torch.rand(shape[0], shape[1], shape[2], 1, generator=g, device="cuda") < 0.01, 6.0, 1.0)
    return x.to(dtype)


def _quantise(x):
    """Codes (two to a byte) and bf16 scales of rows [..., d]."""
    x = x.float()
    x = x.unflatten(-1, (-1, GROUP))
    amax = x.abs().amax(-1, keepdim=True)
    scale = (amax / torch.full_like(amax, 7.0)).to(BF)
    scale = torch.where(torch.isfinite(amax), scale, torch.full_like(scale, math.nan))
    s = scale.float()
    code = torch.round(x / s).clamp(-7, 7)
    code = torch.where(s > 0, code, torch.zeros_like(code)).flatten(-2).to(torch.int32) + 8
    return (code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8), scale.squeeze(-1)


def _values(codes, scales):
    """The fp32 values that codes and scales stand for."""
    q = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() - 8.0
    return (q.unflatten(-1, (-1, GROUP)) * scales.float().unsqueeze(-1)).flatten(-2)


class State:
    pass


def prepare(c, seed):
    g = torch.Generator("cuda").manual_seed(int(seed))
    s = State()
    s.case = c
    b, hq, hkv, d, t, n, kind = (c[k] for k in ("batch", "h_q", "h_kv", "d", "t_ctx", "n", "kind"))
    cap = _t_cap(c)
    s.lens = torch.tensor(_lens(c), dtype=torch.int32, device="cuda")
    if kind == "append":
        s.dtype = F32 if c["dtype"] == "fp32" else BF
        shape = (b, hkv, n, d)
        s.k_rows, s.v_rows = _rows(g, shape, True, s.dtype), _rows(g, shape, False, s.dtype)
        if c["by_token"]:
            s.k_rows, s.v_rows = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (s.k_rows, s.v_rows))
        s.codes = [torch.zeros(b, hkv, cap, d // 2, dtype=torch.uint8, device="cuda") for _ in range(2)]
        s.scales = [torch.zeros(b, hkv, cap, d // GROUP, dtype=BF, device="cuda") for _ in range(2)]
        s.out = [torch.empty(shape, dtype=s.dtype, device="cuda") for _ in range(2)]
    else:
        s.codes, s.scales = zip(*[_quantise(_rows(g, (b, hkv, cap, d), keys, BF)) for keys in (True, False)])
    if kind == "read":
        s.dtype = F32 if c["dtype"] == "fp32" else BF
        s.out = [torch.empty(b, hkv, n, d, dtype=s.dtype, device="cuda") for _ in range(2 if c["with_v"] else 1)]
    if kind == "verify":
        s.q = torch.randn(b, hq, n, d, generator=g, device="cuda").to(BF)
    if kind == "draft":
        s.q = torch.randn(b, hq, d, generator=g, device="cuda").to(BF)
        # a view keeps the first positions, the last and, in between, some of the rest, ascending
        score = torch.rand(b, hkv, max(t, 1), generator=g, device="cuda")
        pos = torch.arange(max(t, 1), device="cuda")
        length = s.lens.view(b, 1, 1)
        score = torch.where((pos < 4) | (pos >= length - c["budget"] // 4), score + 1, score)
        score = torch.where(pos < length, score, -1.0)
        top, idx = score.topk(min(c["budget"], max(t, 1)), dim=-1)
        idx = torch.where(top >= 0, idx, cap).sort(-1).values
        s.idx = torch.full((b, hkv, c["budget"]), -1, dtype=torch.int32, device="cuda")
        s.idx[..., :idx.shape[-1]] = torch.where(idx < cap, idx, -1).int()
        s.count = (s.idx >= 0).sum(-1).int()
    if own:
        import paper_2606_00144_gb300 as bd

        s.bd = bd
        s.shape = bd.make_shape(b, hq, hkv, d, t, cap, s.lens if c["ragged"] else None)
        s.cache = bd.QuantCache(s.codes[0], s.scales[0], s.codes[1], s.scales[1])
        if kind in ("verify", "draft"):
            op = bd.BD_OP_QUANT_VERIFY if kind == "verify" else bd.BD_OP_QUANT_DRAFT
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
        bd.bd_quant_write(s.shape, s.k_rows, s.v_rows, s.cache)
        bd.bd_quant_read(s.shape, s.cache, s.out[0], s.out[1])   # the rows behind each sequence's length
        return {"k": s.out[0], "v": s.out[1]}
    if kind == "read":
        bd.bd_quant_read(s.shape, s.cache, s.out[0], s.out[1] if c["with_v"] else None, first_row=c["t_ctx"] - c["n"])
        return {"k": s.out[0], "v": s.out[1]} if c["with_v"] else {"k": s.out[0]}
    if kind == "verify":
        bd.bd_quant_verify_attn(s.shape, s.q, c["n"], s.cache, s.o, s.lse, s.ws)
    else:
        bd.bd_quant_draft_attn(s.shape, s.q, s.cache, s.idx, s.count, c["budget"], c["n"], s.o, s.lse, s.ws)
    return {"o": s.o, "lse": s.lse}


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
    b, hq, hkv, d, n = (c[k] for k in ("batch", "h_q", "h_kv", "d", "n"))
    dev = s.codes[0].device
    if kind == "append":
        at = s.lens.long().view(b, 1, 1, 1) + torch.arange(n, device=dev).view(1, 1, n, 1)
        at = at.expand(b, hkv, n, 1)
        (kc, ks), (vc, vs) = _quantise(s.k_rows), _quantise(s.v_rows)
        s.codes[0].scatter_(2, at.expand_as(kc), kc)
        s.codes[1].scatter_(2, at.expand_as(vc), vc)
        s.scales[0].scatter_(2, at.expand_as(ks), ks)
        s.scales[1].scatter_(2, at.expand_as(vs), vs)
        return {"k": _values(s.codes[0].gather(2, at.expand_as(kc)), s.scales[0].gather(2, at.expand_as(ks))).to(s.dtype),
                "v": _values(s.codes[1].gather(2, at.expand_as(vc)), s.scales[1].gather(2, at.expand_as(vs))).to(s.dtype)}
    if kind == "read":
        r = slice(c["t_ctx"] - n, c["t_ctx"])
        out = {"k": _values(s.codes[0][:, :, r], s.scales[0][:, :, r]).to(s.dtype)}
        if c["with_v"]:
            out["v"] = _values(s.codes[1][:, :, r], s.scales[1][:, :, r]).to(s.dtype)
        return out
    length = s.lens.view(b, 1, 1, 1)
    if kind == "verify":
        q = s.q.float().view(b, hkv, hq // hkv * n, d)
        pos = torch.arange(s.codes[0].shape[2], device=dev)
        last = length + torch.arange(n, device=dev).repeat(hq // hkv).view(1, 1, -1, 1)
        o, lse = _attend(q, _values(s.codes[0], s.scales[0]), _values(s.codes[1], s.scales[1]), pos > last)
        return {"o": o.to(BF).view(b, hq, n, d), "lse": lse.view(b, hq, n)}
    q = s.q.float().view(b, hkv, hq // hkv, d)
    kept = torch.where(torch.arange(c["budget"], device=dev) < s.count.unsqueeze(-1), s.idx.long(), 0)
    drafted = s.lens.long().view(b, 1, 1) + torch.arange(n + 1, device=dev)
    rows = torch.cat([kept, drafted.expand(b, hkv, n + 1)], -1).unsqueeze(-1)
    slot = torch.arange(c["budget"] + n + 1, device=dev)
    hidden = ((slot < c["budget"]) & (slot >= s.count.unsqueeze(-1))).unsqueeze(2)
    at_c, at_s = rows.expand(-1, -1, -1, d // 2), rows.expand(-1, -1, -1, d // GROUP)
    k = _values(s.codes[0].gather(2, at_c), s.scales[0].gather(2, at_s))
    v = _values(s.codes[1].gather(2, at_c), s.scales[1].gather(2, at_s))
    o, lse = _attend(q, k, v, hidden)
    return {"o": o.to(BF).view(b, hq, d), "lse": lse.view(b, hq)}


# ------------------------------------------------------------------------------------ 64 bits


def _stored(x):
    """What a row x is after quantising, in 64 bits: every element moved to the nearest multiple of
    its group's scale."""
    x = x.double()
    y = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    top = y.abs().max(-1, keepdim=True).values
    step = (top / 7).float().bfloat16().double()
    n = torch.where(step > 0, (y / step).float().double().round(), torch.zeros_like(y))
    return (n.clamp(-7, 7) * step).reshape(x.shape)


_TABLE = [[(byte & 15) - 8.0, (byte >> 4) - 8.0] for byte in range(256)]


def _unit_rows(codes, scales, rows):
    """Rows of one (sequence, KV head) in 64 bits."""
    table = torch.tensor(_TABLE, dtype=torch.float64, device=codes.device)
    x = table[codes[rows].long()].reshape(len(rows), -1)
    return x * scales[rows].double().repeat_interleave(GROUP, -1)


def exact(c, seed):
    s = prepare(c, seed)
    kind, b, hq, hkv, d, n = (c[k] for k in ("kind", "batch", "h_q", "h_kv", "d", "n"))
    if kind == "append":
        return {"k": _stored(s.k_rows), "v": _stored(s.v_rows)}
    dev, G, lens = s.codes[0].device, hq // hkv, _lens(c)
    if kind == "read":
        rows = torch.arange(c["t_ctx"] - n, c["t_ctx"], device=dev)
        both = [torch.stack([torch.stack([_unit_rows(codes[i, h], scales[i, h], rows) for h in range(hkv)])
                             for i in range(b)]) for codes, scales in zip(s.codes, s.scales)]
        return {"k": both[0], "v": both[1]} if c["with_v"] else {"k": both[0]}
    o = torch.empty(s.q.shape, dtype=torch.float64, device=dev)
    lse = torch.empty(s.q.shape[:-1], dtype=torch.float64, device=dev)
    for i in range(b):
        for h in range(hkv):
            heads = slice(h * G, (h + 1) * G)
            if kind == "verify":
                rows = torch.arange(lens[i] + n, device=dev)
                last = lens[i] + torch.arange(n, device=dev).repeat(G)
            else:
                kept = s.idx[i, h, :int(s.count[i, h])].long()
                rows = torch.cat([kept, lens[i] + torch.arange(n + 1, device=dev)])
                last = torch.full((G,), c["t_ctx"] + n + 1, device=dev)
            k, v = (_unit_rows(codes[i, h], scales[i, h], rows) for codes, scales in zip(s.codes, s.scales))
            x = s.q[i, heads].double().reshape(-1, d) @ k.T / math.sqrt(d)
            x[rows.unsqueeze(0) > last.unsqueeze(1)] = -math.inf
            lse[i, heads] = torch.logsumexp(x, 1).view(lse[i, heads].shape)
            o[i, heads] = (torch.softmax(x, 1) @ v).view(o[i, heads].shape)
    return {"o": o, "lse": lse}
