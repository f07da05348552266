"""Operators of a generator that keeps its keys and values in 4 bits, as cases that can be timed.

Chunk-wise video generation and the text models beside it run the same step for every layer: place this step's tokens in the pages of
a cache, norm and rotate queries and keys, write keys and values into the cache in 4 bits, and attend to all that is cached.

    tables   sol_attn_block_tables: pages, block tables, slots and positions from the requests' lengths
    norm     sol_attn_qk_norm_rope: RMS norm of each head of q and k and the position rotation
    append   sol_attn_cache_append and sol_attn_cache_read: keys and values into the cache, and back as the values that are held
    attend   sol_attn_cache_attention: softmax attention over the pages of each request

A page of the cache holds ``page`` tokens of every key/value head, in units of 16 tokens.  A unit of d channels is 18 d bytes: the codes
of the keys and of the values (e2m1, the lower channel in the lower four bits) and their scales (e4m3, one for 16 channels).  Keys' codes lie
[token][d / 2]; the rest as the lanes of a matrix product read it (token = 8 half + 2 t + e for values, 8 half + g for keys):

    values' codes   [half 2][g 8][t 4][e 2][d / 16]    channels g d / 8 ...
    keys' scales    [g 8][t 4][half 2][d / 64]         groups t d / 64 ...
    values' scales  [group d / 16][t 4][half 2][e 2]

Sizes: heads and token counts of this package's video and image workloads; requests, pages and lengths as servers have them.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
_MOST_FLOPS = 4.0 * 40 * 1560 * 32760 * 128        # of an attention that is drawn
_MOST_TOKENS = 1 << 19                             # cached tokens of an attention that is drawn, over all requests


def _tables(requests, old, new, page, name=None):
    return _named({"op": "tables", "requests": requests, "old": old, "new": new, "page": page}, name)


def _norm(batch, tokens, heads, kv_heads, d, kind, rot, interleaved, heads_first, far, name=None):
    return _named({"op": "norm", "batch": batch, "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "d": d, "type": kind, "rot": rot,
                   "interleaved": interleaved, "heads_first": heads_first, "far": far}, name)


def _append(tokens, kv_heads, d, kind, page, k_exp, v_exp, name=None):
    return _named({"op": "append", "tokens": tokens, "kv_heads": kv_heads, "d": d, "type": kind, "page": page, "k_exp": k_exp,
                   "v_exp": v_exp}, name)


def _attend(requests, queries, context, heads, kv_heads, d, kind, page, causal, even, name=None):
    return _named({"op": "attend", "requests": requests, "queries": queries, "context": context, "heads": heads, "kv_heads": kv_heads,
                   "d": d, "type": kind, "page": page, "causal": causal, "even": even}, name)


def _named(case, name):
    return {**case, "name": name} if name else case


def listed():
    return [
        # one decoding step of a full batch: most requests need no new page
        _tables(64, 8000, 1, 16, "tables_step"),
        # the prompts of a batch come in, behind prefixes that are cached already
        _tables(192, 2000, 2000, 64, "tables_prompts"),
        # one token of each of 32 requests, far into their sequences
        _norm(1, 32, 40, 8, 128, "bf16", 128, False, False, 131072, "norm_step"),
        # q and k of a whole 480p video, heads first as the fused kernels' default layout has it
        _norm(1, 32760, 40, 40, 128, "bf16", 128, True, True, 32760, "norm_video480"),
        # two prompts of text with small heads, half of the channels rotated, odd length
        _norm(2, 5077, 16, 4, 64, "fp16", 32, False, False, 8192, "norm_text"),
        # one token of each of 32 requests into the cache
        _append(32, 8, 128, "bf16", 16, 0, 0, "append_step"),
        # five latent frames of a 480p video into the cache
        _append(7800, 40, 128, "bf16", 64, 1, -2, "append_frames"),
        # the first words of one conversation: latency
        _attend(1, 1, 777, 16, 2, 64, "fp16", 16, True, True, "attend_one"),
        # a decoding step of a full batch of ragged requests
        _attend(64, 1, 15000, 40, 8, 128, "bf16", 64, True, False, "attend_step"),
        # a decoding step of one long document
        _attend(1, 1, 262143, 40, 8, 128, "bf16", 128, True, True, "attend_long"),
        # prompts come in behind cached prefixes, requests that decode among them
        _attend(6, 1000, 8000, 16, 4, 64, "fp16", 32, True, False, "attend_prompts"),
        # the next latent frame of a 480p video attends to all frames
        _attend(1, 1560, 32760, 40, 40, 128, "bf16", 64, False, True, "attend_frame"),
    ]


def _spread(rng, low, high):
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    op = rng.choice(["tables", "norm", "norm", "append", "attend", "attend", "attend"])
    kind, page, d = rng.choice(["bf16", "bf16", "fp16"]), rng.choice([16, 32, 64, 128]), rng.choice([64, 128, 128])
    if op == "tables":
        return _tables(_spread(rng, 1, 192), _spread(rng, 16, 8000), _spread(rng, 1, 2000), page)
    if op == "norm":
        heads, kv_heads = rng.choice([(40, 40), (40, 8), (24, 24), (16, 4), (16, 1), (2, 2)])
        tokens = _spread(rng, 1, 32760)
        batch = rng.choice([1, 1, 2, 3])
        rot = rng.choice([d, d, d // 2, 3 * d // 4])
        return _norm(batch, max(1, tokens // batch), heads, kv_heads, d, kind, rot, rng.random() < 0.5, rng.random() < 0.4,
                     32760 + rng.randrange(100000))
    if op == "append":
        return _append(_spread(rng, 1, 7800), rng.choice([1, 2, 4, 8, 24, 40]), d, kind, page, rng.choice([0, 0, 1, -3]), rng.choice([0, 0, -2, 2]))
    while True:
        heads, kv_heads = rng.choice([(40, 40), (40, 8), (24, 24), (24, 3), (16, 4), (16, 1), (2, 2)])
        requests = _spread(rng, 1, 64)
        context = _spread(rng, 1, 262143)
        queries = rng.choice([1, 1, 1, rng.randint(2, 8), _spread(rng, 8, 2000)])
        c = _attend(requests, min(queries, context), context, heads, kv_heads, d, kind, page, rng.random() < 0.7, rng.random() < 0.3)
        # scores of the plain form, padded, and the two limits of a pass
        if requests * context <= _MOST_TOKENS and work(c)["flops"] <= _MOST_FLOPS and work(c)["bytes"] < 6e8 and \
                float(requests) * heads * queries * context <= 2.1e9 and float(requests) * kv_heads * context * d <= 1.1e9:
            return c


# ---------------------------------------------------------------------------------------------------------------------------- inputs
def _lengths(c, seed):
    """(cached tokens behind this step, tokens of this step) of each request of an attention; the seed has a say in their order."""
    n = c["requests"]
    if c["even"]:
        return [c["context"]] * n, [c["queries"]] * n
    g = torch.Generator().manual_seed(17)
    share = torch.rand(n, generator=g).tolist()
    some = torch.rand(n, generator=g).tolist()
    kv = [max(1, round(c["context"] * (1 / 8 + 7 / 8 * s))) for s in share]
    kv[n // 2] = c["context"]
    new = [max(1, round(c["queries"] * s)) if s > 0.25 else 1 for s in some]   # a quarter of the requests decode
    new[n // 3] = c["queries"]
    kv[n // 3] = max(kv[n // 3], c["queries"])
    order = torch.randperm(n, generator=g.manual_seed(seed)).tolist()
    return [kv[b] for b in order], [min(new[b], kv[b]) for b in order]


def _codes(x, exp):
    """e2m1 codes (uint8) and e4m3 scales (float32) of x [..., d], and the values they stand for."""
    y = x.float() * 2.0 ** -exp
    y = y.reshape(*y.shape[:-1], -1, 16)
    amax = y.abs().amax(-1, keepdim=True)
    s = (amax / torch.full_like(amax, 6)).clamp(max=448).to(torch.float8_e4m3fn).float()    # (divided by a tensor: a product with 1 / 6 moves ties)
    a = torch.where(s > 0, y.abs() / s, 0)
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte() +
            (a > 5).byte())
    value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=x.device)[code.int()] * s * 2.0 ** exp
    value = torch.where(y < 0, -value, value).flatten(-2)
    return (code + 8 * (y < 0).byte()).flatten(-2), s.squeeze(-1), value


def _pages(k, v):
    """The bytes of pages whose keys and values are k, v [pages, heads, page, d]: uint8 [pages, heads, page / 16, 18 d]."""
    p, h, n, d = k.shape
    (kc, ks, _), (vc, vs, _) = _codes(k, 0), _codes(v, 0)
    kc, vc = ((x[..., 0::2] + 16 * x[..., 1::2]).reshape(p, h, n // 16, 16, d // 2) for x in (kc, vc))
    ks, vs = (x.to(torch.float8_e4m3fn).view(torch.uint8).reshape(p, h, n // 16, 16, d // 16) for x in (ks, vs))
    vc = vc.reshape(p, h, n // 16, 2, 4, 2, 8, d // 16).permute(0, 1, 2, 3, 6, 4, 5, 7)
    ks = ks.reshape(p, h, n // 16, 2, 8, 4, d // 64).permute(0, 1, 2, 4, 5, 3, 6)
    vs = vs.reshape(p, h, n // 16, 2, 4, 2, d // 16).permute(0, 1, 2, 6, 4, 3, 5)
    return torch.cat([x.reshape(p, h, n // 16, -1) for x in (kc, vc, ks, vs)], -1).contiguous()


def _cu(new, device="cuda"):
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    return torch.tensor(cu, dtype=torch.int32, device=device)


def prepare(case, seed):
    c, dev = case, "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    t = _TYPES.get(c.get("type"))

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device=dev) * scale

    s = {"case": c}
    if c["op"] == "tables":
        n, page = c["requests"], c["page"]
        cpu = torch.Generator().manual_seed(3)
        old = torch.randint(0, c["old"] + 1, (n,), generator=cpu)
        new = torch.randint(1, c["new"] + 1, (n,), generator=cpu)
        mix = torch.randperm(n, generator=cpu.manual_seed(seed))
        old, new = old[mix], new[mix]
        have, need = -(-old // page), -(-(old + new) // page)
        total, width = int(need.sum()), int(need.max()) + 2
        order = torch.randperm(total + 50, generator=cpu).int()
        table = torch.full((n, width), -1, dtype=torch.int32)
        at = 0
        for b, k in enumerate(have.tolist()):
            table[b, :k] = order[at:at + k]
            at += k
        free = order[at:]
        tokens = int(new.sum())
        s.update(old=old.int().to(dev), new=new.int().to(dev), table=table.to(dev), free=free.to(dev),
                 free_count=torch.tensor([len(free)], dtype=torch.int32, device=dev), page=page,
                 cu=torch.zeros(n + 1, dtype=torch.int32, device=dev), kv=torch.zeros(n, dtype=torch.int32, device=dev),
                 slots=torch.zeros(tokens, dtype=torch.int32, device=dev), positions=torch.zeros(tokens, dtype=torch.int32, device=dev),
                 result=torch.zeros(2, dtype=torch.int32, device=dev))
    elif c["op"] == "norm":
        B, n, d = c["batch"], c["tokens"], c["d"]

        def heads(h):
            x = normal(B, h, n, d) if c["heads_first"] else normal(B, n, h, d)
            return (x * torch.exp(normal(d, scale=0.5))).to(t)

        q, k = heads(c["heads"]), heads(c["kv_heads"])
        angle = torch.arange(c["far"], device=dev, dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(c["rot"] // 2, device=dev, dtype=torch.float64) * 2 / c["rot"])
        s.update(q=q, k=k, q_out=torch.empty_like(q), k_out=torch.empty_like(k), cos=angle.cos().float(), sin=angle.sin().float(),
                 positions=torch.randint(0, c["far"], (B, n), generator=g, device=dev, dtype=torch.int32),
                 q_weight=1 + normal(d, scale=0.1), k_weight=1 + normal(d, scale=0.1))
    elif c["op"] == "append":
        n, h, d, page = c["tokens"], c["kv_heads"], c["d"], c["page"]
        pages = -(-2 * n // page) + 3
        outlier = torch.exp(normal(d, scale=0.7))
        s.update(k=(normal(n, h, d) * outlier).to(t), v=normal(n, h, d, scale=0.5).to(t), pages=pages,
                 cache=torch.zeros(pages * h * page // 16 * 18 * d, dtype=torch.uint8, device=dev),
                 slots=torch.randperm(pages * page, generator=g, device=dev)[:n].sort()[0].int(),
                 k_out=torch.empty(n, h, d, dtype=t, device=dev), v_out=torch.empty(n, h, d, dtype=t, device=dev))
    else:
        kv, new = _lengths(c, seed)
        h, d, page = c["kv_heads"], c["d"], c["page"]
        counts = [-(-n // page) for n in kv]
        pages = sum(counts) + 2
        cpu = torch.Generator().manual_seed(seed + 5)
        order = torch.randperm(pages, generator=cpu).int()
        table = torch.zeros(len(kv), max(counts), dtype=torch.int32)
        at = 0
        for b, n in enumerate(counts):
            table[b, :n] = order[at:at + n]
            at += n
        cache = torch.cat([_pages(normal(m, h, page, d), normal(m, h, page, d))
                           for m in [min(1 + (1 << 26) // (h * page * d), pages - a) for a in range(0, pages, 1 + (1 << 26) // (h * page * d))]])
        q = normal(sum(new), c["heads"], d, scale=1.5).to(t)
        s.update(q=q, cu=_cu(new), kv=torch.tensor(kv, dtype=torch.int32, device=dev), table=table.to(dev), cache=cache.reshape(-1),
                 pages=pages, max_q=max(new), out=torch.empty_like(q), lse=torch.empty(sum(new), c["heads"], device=dev))
    return s


# ----------------------------------------------------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return _run_own(state)
    return {"tables": _plain_tables, "norm": _plain_norm, "append": _plain_append, "attend": _plain_attend}[state["case"]["op"]](state)


def _run_own(s):
    from paper_2607_24027_b200 import binding as sol
    c = s["case"]
    if c["op"] == "tables":
        sol.sol_attn_block_tables(s["old"], s["new"], s["free"], s["free_count"], s["table"], s["cu"], s["kv"], s["slots"], s["result"],
                                  s["page"], positions=s["positions"])
        return [s[x] for x in ("table", "cu", "kv", "slots", "positions", "result")]
    if c["op"] == "norm":
        sol.sol_attn_qk_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], s["cos"], s["sin"], positions=s["positions"],
                                  q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6, interleaved=c["interleaved"],
                                  layout=sol.SOL_LAYOUT_BHND if c["heads_first"] else sol.SOL_LAYOUT_BNHD)
        return [s["q_out"], s["k_out"]]
    if "handle" not in s:      # what a program keeps: the cache's description and the workspace
        s["handle"] = sol.Cache(s["cache"], s["pages"], c["page"], c["kv_heads"], c["d"], c.get("k_exp", 0), c.get("v_exp", 0))
        if c["op"] == "attend":
            s["workspace"] = sol.make_cache_workspace(s["max_q"], c["heads"], c["kv_heads"], c["d"])
    if c["op"] == "append":
        sol.sol_attn_cache_append(s["k"], s["v"], s["slots"], s["handle"])
        sol.sol_attn_cache_read(s["handle"], s["slots"], s["k_out"], s["v_out"])
        return [s["k_out"], s["v_out"]]
    sol.sol_attn_cache_attention(s["q"], s["cu"], s["kv"], s["table"], s["handle"], s["out"], s["max_q"], s["workspace"], lse=s["lse"],
                               causal=c["causal"])
    return [s["out"], s["lse"]]


def _plain_tables(s):
    page, old, new, table = s["page"], s["old"].long(), s["new"].long(), s["table"].long()
    kv = old + new
    cu = torch.cat([new.new_zeros(1), new.cumsum(0)])
    have, need = (old + page - 1) // page, (kv + page - 1) // page
    start = (need - have).cumsum(0) - (need - have)
    column = torch.arange(table.shape[1], device=table.device)
    rank = start[:, None] + column - have[:, None]
    count = s["free_count"].long()
    fresh = (column >= have[:, None]) & (column < need[:, None])
    page_id = torch.where(rank < count, s["free"].long()[(count - 1 - rank).clamp(0, s["free"].shape[0] - 1)], -1)
    table = torch.where(fresh, page_id, table)
    token = torch.arange(s["slots"].shape[0], device=table.device)
    b = torch.searchsorted(cu, token, right=True) - 1
    position = old[b] + token - cu[b]
    at = table[b, position // page]
    slots = torch.where(at >= 0, at * page + position % page, -1)
    taken = torch.minimum((need - have).sum(), count)
    return [x.int() for x in (table, cu, kv, slots, position, torch.cat([count - taken, (slots < 0).sum()[None]]))]


def _plain_norm(s):
    c, rot = s["case"], s["case"]["rot"]
    cos, sin = s["cos"][s["positions"].long()], s["sin"][s["positions"].long()]      # [B, n, rot / 2]
    cos, sin = (x[:, None] if c["heads_first"] else x[:, :, None] for x in (cos, sin))

    def one(x, w):
        y = x.float()
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * w
        r = y[..., :rot]
        if c["interleaved"]:
            a, b = r[..., 0::2], r[..., 1::2]
            r = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        else:
            a, b = r[..., :rot // 2], r[..., rot // 2:]
            r = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        return torch.cat([r, y[..., rot:]], -1).to(x.dtype)

    return [one(s["q"], s["q_weight"]), one(s["k"], s["k_weight"])]


def _plain_append(s):
    c = s["case"]
    return [_codes(s["k"], c["k_exp"])[2].to(s["k"].dtype), _codes(s["v"], c["v_exp"])[2].to(s["v"].dtype)]


def _plain_cached(s):
    """Keys and values of every request in order, float32 [requests, heads, columns of the table * page, d]."""
    c = s["case"]
    h, d, page = c["kv_heads"], c["d"], c["page"]
    raw = s["cache"].view(s["pages"], h, page // 16, 18 * d)[s["table"].long()]      # [requests, columns, heads, units, bytes]
    lead = raw.shape[:4]
    value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=raw.device)
    kc = raw[..., :8 * d].reshape(*lead, 16, d // 2)
    vc = raw[..., 8 * d:16 * d].reshape(*lead, 2, 8, 4, 2, d // 16).permute(0, 1, 2, 3, 4, 6, 7, 5, 8).reshape(*lead, 16, d // 2)
    ks = raw[..., 16 * d:17 * d].reshape(*lead, 8, 4, 2, d // 64).permute(0, 1, 2, 3, 6, 4, 5, 7).reshape(*lead, 16, d // 16, 1)
    vs = raw[..., 17 * d:].reshape(*lead, d // 16, 4, 2, 2).permute(0, 1, 2, 3, 6, 5, 7, 4).reshape(*lead, 16, d // 16, 1)

    def values(codes, scales):
        x = value[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()].reshape(*lead, 16, d // 16, 16)
        x = (x * scales.contiguous().view(torch.float8_e4m3fn).float()).reshape(*lead, 16, d)
        return x.permute(0, 2, 1, 3, 4, 5).reshape(lead[0], h, -1, d)

    return values(kc, ks), values(vc, vs)


def _plain_attend(s):
    c, q = s["case"], s["q"]
    n, h, group, d = s["max_q"], c["kv_heads"], c["heads"] // c["kv_heads"], c["d"]
    k, v = _plain_cached(s)
    cu, kv = s["cu"].long(), s["kv"].long()
    new = cu[1:] - cu[:-1]
    i = torch.arange(n, device=q.device)
    rows = (cu[:-1, None] + i).clamp(max=q.shape[0] - 1)                             # [requests, n]
    x = q[rows].float().reshape(-1, n, h, group, d).permute(0, 2, 3, 1, 4).reshape(-1, h, group * n, d)
    score = (x @ k.transpose(-1, -2)).mul_(d ** -0.5)
    sees = kv[:, None] - new[:, None] + i + 1 if c["causal"] else kv[:, None].expand(-1, n)
    hidden = torch.arange(k.shape[2], device=q.device) >= torch.minimum(sees, kv[:, None])[..., None]      # [requests, n, keys]
    score = score.view(-1, h, group, n, k.shape[2]).masked_fill_(hidden[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    weight = score.sub_(top).exp_()
    total = weight.sum(-1, keepdim=True)
    out = (weight.view(-1, h, group * n, k.shape[2]) @ v).view(-1, h, group, n, d) / total.clamp(min=1e-30)
    lse = (top + total.log()).squeeze(-1)
    token = torch.arange(q.shape[0], device=q.device)
    b = torch.searchsorted(cu, token, right=True) - 1
    at = token - cu[b]
    return [out.permute(0, 3, 1, 2, 4)[b, at].reshape(q.shape).to(q.dtype), lse.permute(0, 3, 1, 2)[b, at].reshape(q.shape[:2])]


# ------------------------------------------------------------------------------------------------------------------------- the work
def work(case):
    c = case
    if c["op"] == "tables":
        tokens, pages = c["requests"] * (1 + c["new"]) / 2, c["requests"] * (1 + c["new"]) / 2 / c["page"]
        return {"bytes": 8 * tokens + 8 * pages + 16 * c["requests"], "flops": 0}
    if c["op"] == "norm":
        tokens, rows = c["batch"] * c["tokens"], c["batch"] * c["tokens"] * (c["heads"] + c["kv_heads"])
        return {"bytes": 4 * rows * c["d"] + tokens * (4 * c["rot"] + 4), "flops": rows * (5 * c["d"] + 3 * c["rot"])}
    if c["op"] == "append":     # both calls: 16-bit values in, the cache written and read, 16-bit values out
        values = 2.0 * c["tokens"] * c["kv_heads"] * c["d"]
        return {"bytes": values * (2 + 9 / 16 + 9 / 16 + 2) + 8 * c["tokens"], "flops": 6 * values}
    kv, new = _lengths(c, 1)
    seen = sum(sum(range(a - n + 1, a + 1)) if c["causal"] else a * n for a, n in zip(kv, new))
    tokens = sum(new)
    return {"bytes": 18 / 16 * c["kv_heads"] * c["d"] * sum(kv) + tokens * c["heads"] * (4 * c["d"] + 4),
            "flops": 4.0 * c["heads"] * c["d"] * seen}


# ------------------------------------------------------------------------------------------------------------- the definition, 64 bits
def _nearest(x, table):
    """Index of the entry of the ascending `table` that is nearest to x >= 0; the even one of two."""
    middle = (table[1:] + table[:-1]) / 2
    low = torch.searchsorted(middle, x.contiguous())
    tie = (low < len(middle)) & (middle[low.clamp(max=len(middle) - 1)] == x)
    return torch.where(tie & (low % 2 == 1), low + 1, low)


# The numbers by their codes, from the host: a power on the GPU need not be exact.
_E4M3 = [(m if e == 0 else (8 + m) * 2.0 ** (e - 1)) * 2.0 ** -9 for e in range(16) for m in range(8)][:127]
_E2M1 = [(m if e == 0 else (2 + m) * 2.0 ** (e - 1)) / 2 for e in range(4) for m in range(2)]


def _number(table, code):
    return torch.tensor(table, dtype=torch.float64, device=code.device)[code]


def _exact_held(x, exp):
    scales, values = (torch.tensor(t, dtype=torch.float64, device=x.device) for t in (_E4M3, _E2M1))
    y = (x.double() / 2.0 ** exp).unflatten(-1, (-1, 16))
    s = scales[_nearest(y.abs().amax(-1, keepdim=True), 6 * scales)]
    return torch.where(s == 0, 0, y.sign() * values[_nearest(torch.where(s == 0, 0, y.abs() / s), values)] * s * 2.0 ** exp).flatten(-2)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    dev = "cuda"
    if c["op"] == "tables":
        old, new, table, free = (s[x].tolist() for x in ("old", "new", "table", "free"))
        page, cu, kv, slots, positions = c["page"], [0], [], [], []
        for b, (o, n) in enumerate(zip(old, new)):
            for p in range(o, o + n):
                if p % page == 0 or (p == o and o % page == 0):
                    table[b][p // page] = free.pop() if free else -1
                at = table[b][p // page]
                slots.append(at * page + p % page if at >= 0 else -1)
                positions.append(p)
            cu.append(cu[-1] + n)
            kv.append(o + n)
        answer = (table, cu, kv, slots, positions, [len(free), sum(x < 0 for x in slots)])
        return [torch.tensor(x, dtype=torch.int32, device=dev) for x in answer]
    if c["op"] == "norm":
        half = c["rot"] // 2
        first = torch.arange(half, device=dev) * (2 if c["interleaved"] else 1)
        second = first + (1 if c["interleaved"] else half)
        at = s["positions"].long()
        turn = torch.complex(s["cos"].double(), s["sin"].double())[at]
        turn = turn.unsqueeze(1) if c["heads_first"] else turn.unsqueeze(2)

        def one(x, w):
            y = x.double()
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / c["d"] + 1e-6) * w.double()
            z = torch.complex(y[..., first], y[..., second]) * turn
            y[..., first], y[..., second] = z.real, z.imag
            return y

        return [one(s["q"], s["q_weight"]), one(s["k"], s["k_weight"])]
    if c["op"] == "append":
        return [_exact_held(s["k"], c["k_exp"]), _exact_held(s["v"], c["v_exp"])]
    kv, cu = s["kv"].tolist(), s["cu"].tolist()
    h, group, d, page = c["kv_heads"], c["heads"] // c["kv_heads"], c["d"], c["page"]
    row, ch = torch.arange(page, device=dev)[:, None], torch.arange(d, device=dev)[None, :]
    unit, i = row // 16 * 18 * d, row % 16
    lane = ch // (d // 8) * 4 + i % 8 // 2
    key_at = unit + i * d // 2 + ch // 2
    value_at = unit + 8 * d + ((i // 8 * 32 + lane) * 2 + i % 2) * (d // 16) + ch % (d // 8) // 2
    key_scale = unit + 16 * d + (i % 8 * 8 + ch // (d // 4) * 2 + i // 8) * (d // 64) + ch % (d // 4) // 16
    value_scale = unit + 17 * d + ch // 16 * 16 + i % 8 // 2 * 4 + i // 8 * 2 + i % 2
    key_scale, value_scale = key_scale.expand(page, d), value_scale.expand(page, d)
    cache = s["cache"].view(s["pages"], h, -1)
    out, lse = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev), torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=dev)
    for b, n in enumerate(kv):
        m = cu[b + 1] - cu[b]
        pages = s["table"][b, :-(-n // page)].long()
        for head in range(h):
            bytes_ = cache[pages, head]

            def held(codes, scales):
                x = bytes_[:, codes].int() >> 4 * (ch & 1).int() & 15
                return (torch.where(x > 7, -1.0, 1.0) * _number(_E2M1, x & 7) * _number(_E4M3, bytes_[:, scales].int())).reshape(-1, d)[:n]

            k, v = held(key_at, key_scale), held(value_at, value_scale)
            for j in range(head * group, (head + 1) * group):
                z = s["q"][cu[b]:cu[b + 1], j].double() @ k.T / math.sqrt(d)
                if c["causal"]:
                    z = torch.where(torch.arange(n, device=dev)[None, :] > (n - m + torch.arange(m, device=dev))[:, None], -math.inf, z)
                lse[cu[b]:cu[b + 1], j] = torch.logsumexp(z, -1)
                out[cu[b]:cu[b + 1], j] = torch.softmax(z, -1) @ v
    return [out, lse]
