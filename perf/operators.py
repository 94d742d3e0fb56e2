"""Measured cases of the step's cache and logits operators: plain torch forms and the library's calls on the same inputs.

Four operators, in the order a speculate-and-verify step uses them:

  store    rotary positions for the queries and keys of a draft tree (position = prefix_len + depth of the slot) and the
           write of K and V into the paged cache, bf16 or 8 bits with a power-of-two scale per block of tokens and head
  attn     tree-masked attention over the 8-bit cache
  target   penalties, biases and grammar masks on the verified logits, and the token the target chooses after each slot
  commit   the accepted slots' rows become context inside the 8-bit cache

`own` selects the side: False computes the plain forms, True makes the calls a user makes of the library."""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2, "f32": torch.float32}
MOST = {"e4m3": 448.0, "e5m2": 57344.0}
SMALLEST_SCALE = 2.0 ** -100
D = 128


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # eight requests in plain decoding, a token each: the smallest call, where only latency counts
        dict(name="store decode", op="store", kv="e4m3", B=8, N=1, Hq=32, Hkv=8, page=16, block=16, ctx=4096, rot=128,
             interleaved=False, token_major=False),
        # the 256-request configuration's step: 8-slot trees
        dict(name="store high", op="store", kv="e4m3", B=256, N=8, Hq=32, Hkv=8, page=16, block=16, ctx=65536, rot=128,
             interleaved=False, token_major=False),
        # 64-slot trees and 64 query heads into a bf16 cache, half of each head rotated, pairs interleaved
        dict(name="store wide bf16", op="store", kv="bf16", B=128, N=64, Hq=64, Hkv=8, page=16, block=16, ctx=49152, rot=64,
             interleaved=True, token_major=False),
        # plain decoding of eight requests: one query token, 4096 keys
        dict(name="attn decode", op="attn", kv="e4m3", B=8, N=1, Hq=32, Hkv=8, page=16, block=16, lo=4096, hi=4096,
             token_major=False),
        # 8-slot trees over lognormal contexts around 12288 tokens, a quarter of the 256-request configuration
        dict(name="attn high", op="attn", kv="e4m3", B=64, N=8, Hq=32, Hkv=8, page=16, block=16, lo=4096, hi=32768,
             token_major=False),
        # 32 requests with 32-slot trees, 16K to 32K tokens: 128 query rows per kv head
        dict(name="attn low", op="attn", kv="e4m3", B=32, N=32, Hq=32, Hkv=8, page=16, block=16, lo=16384, hi=32768,
             token_major=False),
        # the end of a long-tailed batch: four requests up to 131072 tokens, e5m2, pages of 32 stored token by token
        dict(name="attn tail e5m2", op="attn", kv="e5m2", B=4, N=24, Hq=32, Hkv=8, page=32, block=32, lo=8192, hi=131072,
             token_major=True),
        # greedy choice with penalties and a grammar in plain decoding
        dict(name="target decode", op="target", dtype="bf16", B=8, N=1, V=32000, ctx=4096, bias=16, mask=True, out=False),
        # the 256-request configuration's step
        dict(name="target high", op="target", dtype="bf16", B=256, N=8, V=32000, ctx=32768, bias=16, mask=True, out=False),
        # 32-slot trees, a large odd vocabulary in 32 bits, the processed logits written back for a sampler
        dict(name="target low f32", op="target", dtype="f32", B=32, N=32, V=131071, ctx=32768, bias=64, mask=True, out=True),
        # the step of eight requests with 16-slot trees
        dict(name="commit tiny", op="commit", kv="e4m3", B=8, N=16, Hkv=8, page=16, block=16, ctx=4096, token_major=False),
        # the step of 256 requests with 32-slot trees
        dict(name="commit high e5m2", op="commit", kv="e5m2", B=256, N=32, Hkv=8, page=32, block=32, ctx=32768,
             token_major=True),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["store", "attn", "attn", "target", "commit"])
    page = rng.choice([8, 16, 32, 64, 128])
    block = rng.choice([b for b in (8, 16, 32, 64, 128) if b <= page])
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 4, 5, 8])
    N = _spread(rng, 1, 64)
    token_major = rng.random() < 0.5
    if op == "store":
        kv = rng.choice(["bf16", "e4m3", "e5m2"])
        B = _spread(rng, 1, max(1, min(256, 400000 // (N * Hkv * (G + 2)))))
        return dict(op=op, kv=kv, B=B, N=N, Hq=Hkv * G, Hkv=Hkv, page=page, block=block, ctx=_spread(rng, 64, 131072),
                    rot=2 * rng.randint(0, 64), interleaved=rng.random() < 0.5, token_major=token_major)
    if op == "commit":
        return dict(op=op, kv=rng.choice(["e4m3", "e5m2"]), B=_spread(rng, 1, 256), N=max(2, N // 2), Hkv=Hkv, page=page,
                    block=block, ctx=_spread(rng, 64, 32768), token_major=token_major)
    if op == "target":
        V = _spread(rng, 1000, 131071)
        B = _spread(rng, 1, max(1, min(256, 100000000 // (N * V))))
        return dict(op=op, dtype=rng.choice(["bf16", "f32"]), B=B, N=N, V=V, ctx=_spread(rng, 1, 16384),
                    bias=rng.randint(0, 64), mask=rng.random() < 0.7, out=rng.random() < 0.4)
    hi = _spread(rng, 64, 131072)
    B = _spread(rng, 1, max(1, min(64, 4000000 // (hi * Hkv))))
    N = max(1, min(N, 512 // G, 260000000 // (B * hi * Hkv * G)))
    return dict(op=op, kv=rng.choice(["e4m3", "e5m2"]), B=B, N=N, Hq=Hkv * G, Hkv=Hkv, page=page, block=block,
                lo=max(1, hi // rng.choice([1, 2, 16])), hi=hi, token_major=token_major)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ints(g, lo, hi, shape):
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)


def _tree(g, B, N):
    """Random draft trees: parent[j] < j, mostly recent slots; a few trees are shorter than N slots."""
    j = torch.arange(N, device="cuda")
    back = _ints(g, 1, 4, (B, N))
    parent = torch.clamp(j - back, min=0).to(torch.int32)
    parent[:, 0] = -1
    n = torch.where(torch.rand(B, generator=g, device="cuda") < 0.25, _ints(g, 1, N + 1, (B,)), torch.full_like(back[:, 0], N))
    parent = torch.where(j < n[:, None], parent, torch.full_like(parent, -1))
    return parent.contiguous(), n.to(torch.int32).contiguous()


def _pool(g, kv, pages, Hkv, page, block, token_major):
    """A cache with what earlier tokens left in it, and its scales (none for bf16)."""
    shape = (pages, page, Hkv, D) if token_major else (pages, Hkv, page, D)
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
    scale = None
    if kv != "bf16":
        x = (x * (MOST[kv] / 4)).clamp_(-MOST[kv], MOST[kv])
        s = torch.exp(0.25 * torch.randn((pages, Hkv, page // block), generator=g, device="cuda")) * 4 / MOST[kv]
        scale = s.contiguous()
    x = x.to(TYPES[kv])
    return (x.permute(0, 2, 1, 3) if token_major else x), scale


def _tail_pages(g, case):
    """Page tables whose leading pages are shared by all requests (a common prompt) and whose last ones are their own."""
    B, N, page = case["B"], case["N"], case["page"]
    prefix = _ints(g, 0, case["ctx"], (B,))
    per = (N - 1) // page + 3                                   # own pages: the one before the tree, the tree, one more
    shared = 16
    width = (case["ctx"] + N - 1) // page + 2
    first = torch.clamp(prefix // page - 1, min=0)
    col = torch.arange(width, device="cuda")[None, :]
    order = torch.randperm(B * per, generator=g, device="cuda").view(B, per) + shared
    own_at = (col - first[:, None]).clamp(0, per - 1)
    mine = torch.gather(order, 1, own_at.long())
    inside = (col >= first[:, None]) & (col < first[:, None] + per)
    table = torch.where(inside, mine, col % shared).to(torch.int32)
    return prefix, table.contiguous(), shared + B * per


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    op, B, N = case["op"], case["B"], case["N"]
    s["parent"], s["n"] = _tree(g, B, N)
    if op in ("store", "commit"):
        s["prefix"], s["table"], pages = _tail_pages(g, case)
        args = (g, case["kv"], pages, case["Hkv"], case["page"], case["block"], case["token_major"])
        s["k_pool"], s["k_scale"] = _pool(*args)
        s["v_pool"], s["v_scale"] = _pool(*args)
    if op == "store":
        Hq, Hkv = case["Hq"], case["Hkv"]
        # q, k and v as one projection leaves them: three parts of the same rows
        qkv = torch.randn((B, N, (Hq + 2 * Hkv) * D), generator=g, device="cuda").to(torch.bfloat16)
        qkv = qkv * torch.exp(0.7 * torch.randn((B, N, 1), generator=g, device="cuda")).to(torch.bfloat16)
        s["q"], s["k"], s["v"] = (x.unflatten(2, (-1, D)) for x in qkv.split([Hq * D, Hkv * D, Hkv * D], dim=2))
        half = case["rot"] // 2
        s["inv_freq"] = (1000000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / max(1, half))).float()
    if op == "attn":
        lo, hi, page = case["lo"], case["hi"], case["page"]
        u = torch.rand(B, generator=g, device="cuda")
        s["prefix"] = torch.round(lo * (hi / lo) ** u).to(torch.int32)
        width = (hi + N + page - 1) // page
        need = (s["prefix"] + N + page - 1) // page
        at = torch.cumsum(need, 0) - need
        pages = int(need.sum())
        order = torch.randperm(pages, generator=g, device="cuda")
        col = torch.arange(width, device="cuda")[None, :]
        own_at = (at[:, None] + col).clamp(max=pages - 1)
        s["table"] = torch.where(col < need[:, None], order[own_at.long()], 0).to(torch.int32).contiguous()
        args = (g, case["kv"], pages, case["Hkv"], page, case["block"], case["token_major"])
        s["k_pool"], s["k_scale"] = _pool(*args)
        s["v_pool"], s["v_scale"] = _pool(*args)
        s["q"] = torch.randn((B, N, case["Hq"], D), generator=g, device="cuda").to(torch.bfloat16)
        s["scale"] = 1.0 / math.sqrt(D)
    if op == "target":
        V = case["V"]
        dt = TYPES[case["dtype"]]
        s["logits"] = (3.0 * torch.randn((B, N, V), generator=g, device="cuda", dtype=dt)).to(dt)
        length = _ints(g, max(1, case["ctx"] // 2), case["ctx"] + 1, (B,)).long()
        s["ctx_off"] = torch.cat([length.new_zeros(1), torch.cumsum(length, 0)])
        total = int(s["ctx_off"][-1])
        zipf = torch.rand(total, generator=g, device="cuda") ** 3
        s["ctx"] = (zipf * V).to(torch.int32).clamp_(max=V - 1)
        s["prompt_len"] = (length // 3).to(torch.int32)
        s["ids"] = torch.where(s["parent"] >= 0, _ints(g, 0, V, (B, N)), torch.full_like(s["parent"], -1))
        s["ids"][:, 0] = s["ctx"][s["ctx_off"][1:] - 1]
        s["repetition"] = 1.0 + 0.3 * torch.rand(B, generator=g, device="cuda")
        s["presence"] = 0.5 * torch.rand(B, generator=g, device="cuda")
        s["frequency"] = 0.1 * torch.rand(B, generator=g, device="cuda")
        m = case["bias"]
        s["bias_off"] = torch.arange(B + 1, device="cuda", dtype=torch.int64) * m
        # distinct tokens per request
        s["bias_ids"] = ((_ints(g, 0, V, (B, 1)) + torch.arange(m, device="cuda", dtype=torch.int32) * (V // max(1, m))) % V).reshape(-1).to(torch.int32).contiguous()
        s["bias_val"] = 2.0 * torch.randn(B * m, generator=g, device="cuda")
        words = (V + 31) // 32
        s["mask"] = torch.randint(-2 ** 31, 2 ** 31, (B, N, words), generator=g, device="cuda", dtype=torch.int64).to(torch.int32) if case["mask"] else None
    if op == "commit":
        # a root path of each tree, of random length: what the acceptance leaves
        anc = _ancestors(s["parent"], s["n"])
        leaf = (torch.rand(B, generator=g, device="cuda") * s["n"]).long()
        on = anc[torch.arange(B, device="cuda"), leaf]                                      # [B, N], root included
        on[:, 0] = False
        slot = torch.arange(N, device="cuda", dtype=torch.int32).expand(B, N)
        s["path"] = torch.sort(torch.where(on, slot, torch.full_like(slot, 1 << 20)), dim=1).values
        s["alen"] = on.sum(1).to(torch.int32)
        s["path"] = torch.where(slot < s["alen"][:, None], s["path"], torch.full_like(slot, -1)).contiguous()
        s["ids"] = _ints(g, 0, 32000, (B, N))
        s["bonus"] = _ints(g, 0, 32000, (B,))
        s["tail0"], s["tail_len0"] = _ints(g, 0, 32000, (B, 32)), torch.full((B,), 32, dtype=torch.int32, device="cuda")
        s["tail"], s["tail_len"], s["prefix0"] = s["tail0"].clone(), s["tail_len0"].clone(), s["prefix"].clone()
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _ancestors(parent, n):
    """[B, N, N] bool: slot a is j or an ancestor of j (both below n)."""
    B, N = parent.shape
    up = torch.zeros((B, N, N), dtype=torch.float64, device=parent.device)
    up.scatter_(2, parent.clamp(min=0).long()[:, :, None], (parent >= 0).double()[:, :, None])
    eye = torch.eye(N, dtype=torch.float64, device=parent.device)
    live = torch.arange(N, device=parent.device) < n[:, None]
    return (torch.matrix_power(up + eye, 64) > 0) & live[:, :, None]


def _rotate(x, cos, sin, rot, interleaved):
    """x float32 [B, N, H, D]; cos, sin float32 [B, N, rot / 2]."""
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., : rot // 2], x[..., rot // 2: rot])
    c, s = cos[:, :, None, :], sin[:, :, None, :]
    y, z = a * c - b * s, b * c + a * s
    r = torch.stack([y, z], -1).flatten(-2) if interleaved else torch.cat([y, z], -1)
    return torch.cat([r, x[..., rot:]], -1)


def _pow2_scale(a, kv):
    """The smallest power of two s with a <= MOST * s (0 for a = 0)."""
    m, e = torch.frexp(a)
    e = e - (9 if kv == "e4m3" else 16) + (m > 0.875)
    return torch.where(a > 0, torch.ldexp(torch.ones_like(a), e).clamp(min=SMALLEST_SCALE), torch.zeros_like(a))


def _to8(x, kv):
    return x.clamp(-MOST[kv], MOST[kv]).to(TYPES[kv])


def _blocks(s, first, count):
    """The scale blocks number first // block .. of every request: first positions, page, row in the page, block in the page."""
    c = s["case"]
    pos0 = (first // c["block"])[:, None] * c["block"] + torch.arange(count, device="cuda")[None, :] * c["block"]
    col = (pos0 // c["page"]).clamp(max=s["table"].shape[1] - 1).long()
    return pos0, torch.gather(s["table"], 1, col).long(), pos0 % c["page"]


def _store_plain(s):
    c, B, N = s["case"], s["case"]["B"], s["case"]["N"]
    anc = _ancestors(s["parent"], s["n"])
    depth = (anc.sum(-1) - 1).clamp(min=0)
    angle = (s["prefix"].double()[:, None] + depth)[:, :, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    q = _rotate(s["q"].float(), cos, sin, c["rot"], c["interleaved"])
    k = _rotate(s["k"].float(), cos, sin, c["rot"], c["interleaved"])
    v = s["v"].float()
    slot = torch.arange(N, device="cuda")
    live = slot < s["n"][:, None]
    out = torch.where(live[:, :, None, None], q, torch.zeros_like(q)).to(torch.bfloat16)
    if c["kv"] == "bf16":
        pos = (s["prefix"][:, None] + slot)[live]
        page = torch.gather(s["table"], 1, (s["prefix"][:, None] + slot).long() // c["page"])[live].long()
        s["k_pool"][page, :, pos % c["page"]] = k[live].to(torch.bfloat16)
        s["v_pool"][page, :, pos % c["page"]] = v[live].to(torch.bfloat16)
        return out, s["k_pool"], s["v_pool"]
    _store_blocks(s, k, "k")
    _store_blocks(s, v, "v")
    return out, s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"]


def _store_blocks(s, x, which):
    c, kv, N, blk = s["case"], s["case"]["kv"], s["case"]["N"], s["case"]["block"]
    pool, scale = s[which + "_pool"], s[which + "_scale"]
    pos0, page, row0 = _blocks(s, s["prefix"], (N - 1) // blk + 2)
    used = pos0 < (s["prefix"] + s["n"])[:, None]
    r = torch.arange(blk, device="cuda")
    pos = pos0[:, :, None] + r                                                   # [B, nb, blk]
    slot = pos - s["prefix"][:, None, None]
    new = (slot >= 0) & (slot < s["n"][:, None, None])
    old = slot < 0
    b = torch.arange(x.shape[0], device="cuda")[:, None, None]
    rows = x[b, slot.clamp(0, N - 1).long()].permute(0, 1, 3, 2, 4)              # [B, nb, H, blk, D]
    rows = torch.where(new[:, :, None, :, None], rows, torch.zeros_like(rows))
    h = torch.arange(x.shape[2], device="cuda")[None, None, :]
    sb = (row0 // blk)[:, :, None]
    s_old = scale[page[:, :, None], h, sb]
    s_old = torch.where((pos0 < s["prefix"][:, None])[:, :, None], s_old, torch.zeros_like(s_old))
    s_new = torch.maximum(s_old, _pow2_scale(rows.abs().amax((-1, -2)), kv))
    s_new = torch.where(s_new > 0, s_new, torch.ones_like(s_new))
    at = (page[:, :, None, None], h[..., None], (row0[:, :, None] + r)[:, :, None, :])
    codes = pool.view(torch.uint8)[at].view(TYPES[kv])
    moved = _to8(codes.float() * (s_old / s_new)[..., None, None], kv).view(torch.uint8)
    grown = (s_new != s_old)[..., None] & old[:, :, None, :]
    fresh = _to8(rows / s_new[..., None, None], kv).view(torch.uint8)
    codes = torch.where(grown[..., None], moved, codes.view(torch.uint8))
    codes = torch.where(new[:, :, None, :, None], fresh, codes)
    at = tuple(t.expand(codes.shape[:-1])[used] for t in at)
    pool.view(torch.uint8)[at] = codes[used]
    scale[page[:, :, None].expand_as(s_new)[used], h.expand_as(s_new)[used], sb.expand_as(s_new)[used]] = s_new[used]


def _cached(s, which, width):
    """The cache of every request as float32 [B, Hkv, width * page, D], scales applied."""
    pool, scale, c = s[which + "_pool"], s[which + "_scale"], s["case"]
    pages = s["table"][:, :width].long()
    x = pool.view(torch.uint8)[pages].view(pool.dtype).float()                   # [B, w, H, page, D]
    x = x * scale[pages].repeat_interleave(c["block"], -1)[..., None]
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3)


def _attn_plain(s):
    c, B, N = s["case"], s["case"]["B"], s["case"]["N"]
    Hkv, G = c["Hkv"], c["Hq"] // c["Hkv"]
    width = s["table"].shape[1]
    k, v = _cached(s, "k", width), _cached(s, "v", width)
    pos = torch.arange(width * c["page"], device="cuda")
    col = pos - s["prefix"][:, None]                                             # [B, L]: slot of each position
    anc = _ancestors(s["parent"], s["n"])
    seen = torch.gather(anc, 2, col.clamp(0, N - 1).long()[:, None, :].expand(B, N, -1))
    seen = (col < 0)[:, None, :] | (seen & (col >= 0)[:, None, :] & (col < s["n"][:, None])[:, None, :])
    v = torch.where((col < s["n"][:, None])[:, None, :, None], v, torch.zeros_like(v))
    q = s["q"].float().unflatten(2, (Hkv, G)).permute(0, 2, 1, 3, 4).flatten(2, 3)     # [B, Hkv, N * G, D]
    z = q @ k.transpose(-1, -2) * s["scale"]
    z = z.masked_fill(~seen.repeat_interleave(G, 1)[:, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - top)
    den = p.sum(-1, keepdim=True)
    o = p @ v / den
    live = (torch.arange(N, device="cuda") < s["n"][:, None])[:, :, None]
    o = o.unflatten(2, (N, G)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    lse = (top + torch.log(den))[..., 0].unflatten(2, (N, G)).permute(0, 2, 1, 3).flatten(2, 3)
    return torch.where(live[..., None], o, torch.zeros_like(o)).to(torch.bfloat16), torch.where(live, lse, torch.zeros_like(lse))


def _target_plain(s):
    c, B, N, V = s["case"], s["case"]["B"], s["case"]["N"], s["case"]["V"]
    length = s["ctx_off"][1:] - s["ctx_off"][:-1]
    req = torch.repeat_interleave(torch.arange(B, device="cuda"), length)
    at = torch.arange(s["ctx"].numel(), device="cuda") - s["ctx_off"][req]
    flat = req * V + s["ctx"].long()
    seen = torch.zeros(B * V, device="cuda").index_fill_(0, flat, 1.0).view(B, 1, V)
    made = torch.zeros(B * V, device="cuda").scatter_add_(0, flat, (at >= s["prompt_len"][req]).float()).view(B, 1, V)
    anc = _ancestors(s["parent"], s["n"])
    anc[:, :, 0] = False                                                         # the root is the context's last token
    path = torch.zeros((B, N, V), device="cuda").scatter_add_(2, s["ids"].clamp(min=0).long()[:, None, :].expand(B, N, N), anc.float())
    made = made + path
    seen = (seen > 0) | (path > 0)
    x = s["logits"].float()
    rep = s["repetition"][:, None, None]
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = x - s["frequency"][:, None, None] * made
    x = x - torch.where(made > 0, s["presence"][:, None, None], 0.0)
    bias = torch.zeros((B, V), device="cuda")
    bias.scatter_(1, s["bias_ids"].view(B, -1).long(), s["bias_val"].view(B, -1))
    x = x + bias[:, None, :]
    if s["mask"] is not None:
        tok = torch.arange(V, device="cuda")
        x = x.masked_fill(((s["mask"][:, :, tok // 32] >> (tok % 32)) & 1) == 0, -math.inf)
    top, best = x.max(-1)
    first = torch.where(x == top[..., None], torch.arange(V, device="cuda"), V).amin(-1)     # ties go to the lowest index
    live = torch.arange(N, device="cuda") < s["n"][:, None]
    target = torch.where(live & (top > -math.inf), first, -1).to(torch.int32)
    if not c["out"]:
        return target
    return target, torch.where(live[:, :, None], x, torch.zeros_like(x)).to(s["logits"].dtype)


def _commit_plain(s):
    c, N, blk, page = s["case"], s["case"]["N"], s["case"]["block"], s["case"]["page"]
    p, k = s["prefix0"], s["alen"]
    pos0, pg, row0 = _blocks(s, p + 1, (N - 1) // blk + 2)
    used = pos0 <= (p + k)[:, None]
    r = torch.arange(blk, device="cuda")
    pos = pos0[:, :, None] + r
    d = pos - p[:, None, None] - 1                                               # index on the path
    shape = d.shape
    on_path = (d >= 0) & (d < k[:, None, None])
    step = torch.gather(s["path"], 1, d.clamp(0, N - 1).long().flatten(1)).view(shape)
    src = torch.where(on_path, p[:, None, None] + step, pos)
    live = pos <= (p + k)[:, None, None]
    col = (src // page).clamp(0, s["table"].shape[1] - 1).long()
    src_page = torch.gather(s["table"], 1, col.flatten(1)).view(shape).long()
    h = torch.arange(c["Hkv"], device="cuda")[None, None, :, None]
    sb = (row0 // blk)[:, :, None]
    new = {}
    _commit_rows(s, "k", src_page, src % page, h, live, new)
    _commit_rows(s, "v", src_page, src % page, h, live, new)
    rows = (row0[:, :, None] + r)[:, :, None, :]
    write = (used[:, :, None] & live)[:, :, None, :].expand(-1, -1, c["Hkv"], -1)
    at = tuple(t.expand(write.shape)[write] for t in (pg[:, :, None, None], h, rows))
    s["k_pool"].view(torch.uint8)[at] = new["k"][0][write]
    s["v_pool"].view(torch.uint8)[at] = new["v"][0][write]
    keep = (used & (k > 0)[:, None])[:, :, None].expand(-1, -1, c["Hkv"])
    at = tuple(t.expand(keep.shape)[keep] for t in (pg[:, :, None], h[..., 0], sb))
    s["k_scale"][at], s["v_scale"][at] = new["k"][1][keep], new["v"][1][keep]
    window = torch.cat([s["tail0"], torch.gather(s["ids"], 1, s["path"].clamp(min=0).long()), s["bonus"][:, None]], 1)
    P = s["tail0"].shape[1]
    take = torch.arange(P, device="cuda")[None, :] + (k + 1)[:, None]            # the window is full: its last P tokens
    take = torch.where(take >= (P + k)[:, None], P + N, take).long()             # the bonus stands behind all N path places
    s["tail"].copy_(torch.gather(window, 1, take))
    s["tail_len"].copy_(s["tail_len0"])
    s["prefix"].copy_(p + k + 1)
    return s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"], s["prefix"], s["tail"], s["tail_len"]


def _commit_rows(s, which, page, row, h, live, new):
    kv, blk = s["case"]["kv"], s["case"]["block"]
    pool, scale = s[which + "_pool"], s[which + "_scale"]
    codes = pool.view(torch.uint8)[page[:, :, None, :], h, row[:, :, None, :]]
    from_s = scale[page[:, :, None, :], h, (row // blk)[:, :, None, :]]
    s_new = torch.where(live[:, :, None, :], from_s, torch.zeros_like(from_s)).amax(-1)
    ratio = from_s / s_new[..., None]
    again = _to8(codes.view(TYPES[kv]).float() * ratio[..., None], kv).view(torch.uint8)
    new[which] = torch.where((ratio != 1)[..., None], again, codes), s_new


# ------------------------------------------------------------------------------------------------ the library's calls
def _own(s):
    from paper_2607_17299_b200 import binding as war
    c, op = s["case"], s["case"]["op"]
    if op == "store":
        if "q_out" not in s:
            s["q_out"] = torch.zeros((c["B"], c["N"], c["Hq"], D), dtype=torch.bfloat16, device="cuda")
        war.war_rope_store(s["q"], s["k"], s["v"], s["inv_freq"], s["table"], s["prefix"], s["n"], s["parent"], s["k_pool"],
                           s["v_pool"], s["k_scale"], s["v_scale"], s["q_out"], interleaved=c["interleaved"])
        pools = (s["q_out"], s["k_pool"], s["v_pool"])
        return pools if c["kv"] == "bf16" else pools + (s["k_scale"], s["v_scale"])
    if op == "attn":
        if "params" not in s:
            s["params"] = war.attn_quant_params(s["q"], s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"], s["table"], s["scale"])
            s["ws"] = war.new_quant_workspace(s["params"], "cuda")
            s["out"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros(s["q"].shape[:3], device="cuda")
        war.war_verify_attn_quant(s["q"], s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"], s["table"], s["prefix"], s["n"],
                                  s["parent"], s["params"], s["ws"], s["out"], s["lse"])
        return s["out"], s["lse"]
    if op == "target":
        if "target" not in s:
            s["target"] = torch.zeros((c["B"], c["N"]), dtype=torch.int32, device="cuda")
            s["out"] = torch.zeros_like(s["logits"]) if c["out"] else None
        war.war_target(s["logits"], s["n"], s["ids"], s["parent"], s["target"], d_ctx=s["ctx"], d_ctx_off=s["ctx_off"],
                       d_prompt_len=s["prompt_len"], d_repetition=s["repetition"], d_presence=s["presence"],
                       d_frequency=s["frequency"], d_bias_off=s["bias_off"], d_bias_ids=s["bias_ids"], d_bias_val=s["bias_val"],
                       d_mask=s["mask"], d_out=s["out"])
        return (s["target"], s["out"]) if c["out"] else s["target"]
    s["prefix"].copy_(s["prefix0"])
    s["tail"].copy_(s["tail0"])
    s["tail_len"].copy_(s["tail_len0"])
    war.war_commit_quant(s["ids"], s["alen"], s["path"], s["bonus"], s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"], s["table"],
                         s["prefix"], s["tail"], s["tail_len"])
    return s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"], s["prefix"], s["tail"], s["tail_len"]


def run(state):
    if own:
        return _own(state)
    return dict(store=_store_plain, attn=_attn_plain, target=_target_plain, commit=_commit_plain)[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    op, B, N = case["op"], case["B"], case["N"]
    if op == "store":
        rows, kv_bytes = B * N, 2 if case["kv"] == "bf16" else 1
        Hq, Hkv = case["Hq"], case["Hkv"]
        return {"bytes": rows * D * (4 * Hq + 4 * Hkv + 2 * kv_bytes * Hkv) + 4 * rows, "flops": rows * case["rot"] * 3 * (Hq + Hkv)}
    if op == "attn":
        lo, hi = case["lo"], case["hi"]
        mean = lo if hi == lo else (hi - lo) / math.log(hi / lo)              # the lengths are spread over their logarithm
        keys = B * (mean + N)
        per_key = case["Hkv"] * (2 * D + 8 / case["block"])
        return {"bytes": keys * per_key + 4 * keys / case["page"] + B * N * case["Hq"] * (4 * D + 4),
                "flops": 4 * keys * N * case["Hq"] * D}
    if op == "target":
        size = 2 if case["dtype"] == "bf16" else 4
        values = B * N * case["V"]
        return {"bytes": values * (size * (2 if case["out"] else 1) + (0.125 if case["mask"] else 0)) + B * case["ctx"] * 3 + 12 * B * N,
                "flops": 6 * values}
    moved = B * min(N - 1, 12) / 2                                            # path lengths; a row is read and written
    return {"bytes": moved * case["Hkv"] * 2 * 2 * D + B * (8 * N + 300), "flops": 0}


# ------------------------------------------------------------------------------------------------ 64 bits
def _chain(parent, j):
    up = []
    while j >= 0:
        up.append(j)
        j = parent[j]
    return up


def _round8(x, kv):
    """float64 values rounded to the 8-bit type's grid (ties to even), saturating."""
    bits, low = (3, -6) if kv == "e4m3" else (2, -14)
    e = torch.frexp(x)[1].double() - 1
    step = torch.exp2(torch.clamp(e, min=low) - bits)
    return torch.clamp(torch.round(x / step) * step, -MOST[kv], MOST[kv])


def _exact_store(s):
    c, N, kv, blk, page = s["case"], s["case"]["N"], s["case"]["kv"], s["case"]["block"], s["case"]["page"]
    q, rot = s["q"].double(), c["rot"]
    out = torch.zeros_like(q)
    pools = [s["k_pool"].double(), s["v_pool"].double()]
    scales = [None if t is None else t.double() for t in (s["k_scale"], s["v_scale"])]
    parent, n, prefix, table = (s[x].tolist() for x in ("parent", "n", "prefix", "table"))
    f = s["inv_freq"].double()
    idx = torch.arange(rot, device="cuda")
    first, second = (idx[0::2], idx[1::2]) if c["interleaved"] else (idx[: rot // 2], idx[rot // 2:])
    for b in range(c["B"]):
        m, p = n[b], prefix[b]
        at = torch.tensor([p + len(_chain(parent[b], j)) - 1 for j in range(m)], device="cuda", dtype=torch.float64)
        turn = torch.polar(torch.ones((m, rot // 2), device="cuda", dtype=torch.float64), at[:, None] * f)[:, None, :]
        rotated = []
        for x in (q[b, :m], s["k"][b, :m].double()):
            y = x.clone()
            w = torch.complex(x[..., first], x[..., second]) * turn
            y[..., first], y[..., second] = w.real, w.imag
            rotated.append(y)
        out[b, :m] = rotated[0]
        for which, rows in enumerate((rotated[1], s["v"][b, :m].double())):
            pool, scale = pools[which], scales[which]
            if kv == "bf16":
                where = torch.tensor([[table[b][(p + j) // page], (p + j) % page] for j in range(m)], device="cuda")
                pool[where[:, 0], :, where[:, 1]] = rows
                continue
            for start in range(p // blk * blk, p + m, blk):
                pg, r0 = table[b][start // page], start % page
                j0, j1 = max(0, start - p), min(m, start + blk - p)
                new = rows[j0:j1].transpose(0, 1)                                # [Hkv, rows, D]
                a = new.abs().amax((1, 2))
                part, power = torch.frexp(a / MOST[kv])                          # a power of two divides exactly: part 0.5
                need = torch.where(a > 0, torch.exp2(power.double() - (part == 0.5).double()), 0.0)
                had = scale[pg, :, r0 // blk] if start < p else torch.zeros_like(need)
                now = torch.maximum(had, need)
                now = torch.where(now > 0, now, 1.0)
                o = max(0, p - start)
                if o:
                    lived = pool[pg, :, r0:r0 + o]
                    pool[pg, :, r0:r0 + o] = torch.where((now != had)[:, None, None], _round8(lived * (had / now)[:, None, None], kv), lived)
                pool[pg, :, r0 + o:r0 + o + j1 - j0] = _round8(new / now[:, None, None], kv)
                scale[pg, :, r0 // blk] = now
    return (out, pools[0], pools[1]) if kv == "bf16" else (out, pools[0], pools[1], scales[0], scales[1])


def _exact_attn(s):
    c, N = s["case"], s["case"]["N"]
    Hkv, G = c["Hkv"], c["Hq"] // c["Hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:3], dtype=torch.float64, device="cuda")
    parent, n, prefix = s["parent"].tolist(), s["n"].tolist(), s["prefix"].tolist()
    for b in range(c["B"]):
        m, p = n[b], prefix[b]
        L = p + m
        pages = s["table"][b, : -(-L // c["page"])].long()
        see = torch.zeros((m, L), dtype=torch.bool)
        see[:, :p] = True
        for j in range(m):
            see[j, [p + a for a in _chain(parent[b], j)]] = True
        see = see.cuda()[:, None, :]
        for h in range(Hkv):
            K, V = ((pool[pages, h].double().reshape(len(pages), -1, c["block"], D) * sc[pages, h].double()[:, :, None, None]).reshape(-1, D)[:L]
                    for pool, sc in ((s["k_pool"], s["k_scale"]), (s["v_pool"], s["v_scale"])))
            z = torch.einsum("jgd,cd->jgc", s["q"][b, :m, h * G:(h + 1) * G].double(), K) * s["scale"]
            z = torch.where(see, z, -math.inf)
            lse[b, :m, h * G:(h + 1) * G] = torch.logsumexp(z, -1)
            out[b, :m, h * G:(h + 1) * G] = torch.softmax(z, -1) @ V
    return out, lse


def _exact_target(s):
    c, V = s["case"], s["case"]["V"]
    if not c["out"]:
        return None
    out = torch.zeros(s["logits"].shape, dtype=torch.float64, device="cuda")
    parent, n, off, ids, plen = (s[x].tolist() for x in ("parent", "n", "ctx_off", "ids", "prompt_len"))
    m = c["bias"]
    tok = torch.arange(V, device="cuda")
    for b in range(c["B"]):
        ctx = s["ctx"][off[b]:off[b + 1]].long()
        every, made = torch.bincount(ctx, minlength=V), torch.bincount(ctx[plen[b]:], minlength=V)
        for j in range(n[b]):
            path = torch.tensor([ids[b][a] for a in _chain(parent[b], j) if a > 0], dtype=torch.int64, device="cuda")
            more = torch.bincount(path, minlength=V)
            x = s["logits"][b, j].double()
            r = s["repetition"][b].double()
            x = torch.where(every + more > 0, torch.where(x > 0, x / r, x * r), x)
            x = x - s["frequency"][b].double() * (made + more) - s["presence"][b].double() * (made + more > 0)
            x[s["bias_ids"][b * m:(b + 1) * m].long()] += s["bias_val"][b * m:(b + 1) * m].double()
            if s["mask"] is not None:
                x[(torch.bitwise_right_shift(s["mask"][b, j][tok // 32], tok % 32) & 1) == 0] = -math.inf
            out[b, j] = x
    return None, out


def _exact_commit(s):
    c, kv, blk, page, Hkv = s["case"], s["case"]["kv"], s["case"]["block"], s["case"]["page"], s["case"]["Hkv"]
    table, prefix, alen, path = (s[x].tolist() for x in ("table", "prefix0", "alen", "path"))
    done = []
    for pool, scale in ((s["k_pool"], s["k_scale"]), (s["v_pool"], s["v_scale"])):
        values, sc = pool.double(), scale.double()
        new_v, new_s = values.clone(), sc.clone()
        for b in range(c["B"]):
            p, k = prefix[b], alen[b]
            come = {p + 1 + d: p + path[b][d] for d in range(k)}
            for start in range((p + 1) // blk * blk, p + k + 1, blk):
                if k == 0:
                    break
                lives = [(x, come.get(x, x)) for x in range(start, min(start + blk, p + k + 1))]
                frm = torch.tensor([[table[b][y // page], y % page] for _, y in lives], device="cuda")
                fs = sc[frm[:, 0], :, frm[:, 1] // blk]                           # [rows, Hkv]
                now = fs.amax(0)
                rows = values[frm[:, 0], :, frm[:, 1]]                            # [rows, Hkv, D]
                ratio = fs / now
                rows = torch.where((ratio != 1)[..., None], _round8(rows * ratio[..., None], kv), rows)
                pg, r0 = table[b][start // page], start % page
                new_v[pg, :, r0:r0 + len(lives)] = rows.transpose(0, 1)
                new_s[pg, :, r0 // blk] = now
        done.append((new_v, new_s))
    (k_new, ks), (v_new, vs) = done
    return k_new, v_new, ks, vs, None, None, None


def exact(case, seed):
    if case["op"] == "commit" and case["B"] * case["N"] > 20000:
        return None
    if case["op"] == "attn" and case["B"] * case["hi"] * case["N"] * case["Hq"] > 1.5e9:
        return None
    s = prepare(case, seed)
    return dict(store=_exact_store, attn=_exact_attn, target=_exact_target, commit=_exact_commit)[case["op"]](s)
