"""Measured cases of rollouts that share cache pages: plain torch forms and the library's calls on the same inputs.

Synchronous rollouts run every prompt several times, so groups of requests hold the same pages in front and their own behind.

  attn      tree-masked attention over such a batch, the shared part of a group computed once for all of its members
  fork      requests become copies of others: full pages shared, the partly filled last page copied
  turnover  finished requests give their pages back, the running ones get room for the next tree
  compact   used pages move to the front of the pool, so that its end can be given away
  groups    which requests share how much, read off the page tables

`own` selects the side: False computes the plain forms, True makes the calls a user makes of the library."""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
MOST = {"e4m3": 448.0, "e5m2": 57344.0}
D = 128
P = 32                                                                          # tail window


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # plain decoding of one prompt's eight rollouts, 4096 tokens of prompt: the smallest attention, only latency counts
        dict(name="attn decode", op="attn", kv="bf16", groups=1, members=8, alone=0, N=1, Hq=32, Hkv=8, page=16, block=16, slo=4096, shi=4096,
             plo=16, phi=256, token_major=False),
        # the 256-request configuration as 32 prompts with eight rollouts each, 8-slot trees
        dict(name="attn high", op="attn", kv="bf16", groups=32, members=8, alone=0, N=8, Hq=32, Hkv=8, page=16, block=16, slo=6144, shi=16384,
             plo=256, phi=4096, token_major=False),
        # 32-slot trees, 16K to 32K tokens of prompt, some requests alone: more query rows in a group than a tile has
        dict(name="attn low", op="attn", kv="bf16", groups=4, members=7, alone=4, N=32, Hq=32, Hkv=8, page=16, block=16, slo=16384, shi=32768,
             plo=128, phi=2048, token_major=False),
        # an 8-bit cache stored token by token, sixteen prompts with four rollouts each
        dict(name="attn e4m3", op="attn", kv="e4m3", groups=16, members=4, alone=3, N=8, Hq=32, Hkv=8, page=32, block=32, slo=8192, shi=32768,
             plo=256, phi=4096, token_major=True),
        # one prompt's prefill is done and seven more rollouts start from it
        dict(name="fork one prompt", op="fork", kv="bf16", prompts=1, members=8, Hkv=8, page=16, block=16, slo=4096, shi=4100, plo=0, phi=0,
             resample=False, token_major=False),
        # 32 groups of eight rollouts go on from members drawn anew: what a beam or a resampling step does to a cache
        dict(name="fork resample e4m3", op="fork", kv="e4m3", prompts=32, members=8, Hkv=8, page=32, block=32, slo=4096, shi=16384, plo=128,
             phi=2048, resample=True, token_major=True),
        # eight requests, trees of 8 slots
        dict(name="turnover small", op="turnover", prompts=2, members=4, N=8, page=16, slo=2048, shi=4096, plo=16, phi=512, spare=4096),
        # 1024 requests in a pool of about half a million pages, trees of 32 slots
        dict(name="turnover large", op="turnover", prompts=128, members=8, N=32, page=16, slo=4096, shi=16384, plo=256, phi=8192, spare=262144),
        # a small pool at the end of a rollout phase
        dict(name="compact small", op="compact", kv="bf16", prompts=8, members=2, Hkv=8, page=16, block=16, slo=512, shi=2048, plo=16, phi=512,
             spare=0.1, token_major=False),
        # a layer's pool of 3.5 GB, 8-bit codes of 64-token pages
        dict(name="compact large e5m2", op="compact", kv="e5m2", prompts=32, members=4, Hkv=8, page=64, block=32, slo=4096, shi=16384, plo=512,
             phi=8192, spare=0.1, token_major=False),
        # eight rollouts of one prompt
        dict(name="groups small", op="groups", prompts=1, members=8, page=16, system=16, slo=2048, shi=4096, plo=16, phi=512),
        # 512 requests of 64 prompts behind one system prompt
        dict(name="groups large", op="groups", prompts=64, members=8, page=16, system=64, slo=8192, shi=65536, plo=256, phi=8192),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "fork", "turnover", "compact", "groups"])
    page = rng.choice([8, 16, 32, 64, 128])
    block = rng.choice([b for b in (8, 16, 32, 64, 128) if b <= page])
    Hkv = rng.choice([1, 2, 4, 8])
    token_major = rng.random() < 0.5
    kv = rng.choice(["bf16", "bf16", "e4m3", "e5m2"])
    phi = _spread(rng, 1, 8192)
    plo = max(1, phi // rng.choice([1, 4, 16]))
    if op == "attn":
        G = rng.choice([1, 2, 4, 5, 8])
        shi = _spread(rng, 64, 65536)
        slo = max(1, shi // rng.choice([1, 2, 8]))
        members = _spread(rng, 2, 16)
        groups = _spread(rng, 1, max(1, min(32, 1500000 // (Hkv * (shi + members * phi)))))
        alone = rng.choice([0, 0, 1, 3])
        keys = groups * members * (shi + phi) + alone * (shi + phi)
        N = max(1, min(_spread(rng, 1, 64), 512 // G, 400000000 // (keys * Hkv * G)))
        return dict(op=op, kv=kv, groups=groups, members=members, alone=alone, N=N, Hq=Hkv * G, Hkv=Hkv, page=page, block=block, slo=slo,
                    shi=shi, plo=plo, phi=phi, token_major=token_major)
    shi = _spread(rng, 64, 32768)
    slo = max(1, shi // rng.choice([1, 2, 8]))
    members = _spread(rng, 2, 16)
    if op == "groups":
        return dict(op=op, prompts=_spread(rng, 1, 64), members=members, page=page, system=rng.choice([0, 1, 16]), slo=slo, shi=shi, plo=plo, phi=phi)
    if op == "turnover":
        prompts = _spread(rng, 1, max(1, min(128, 1024 // members)))
        return dict(op=op, prompts=prompts, members=members, N=_spread(rng, 1, 64), page=page, slo=slo, shi=shi, plo=plo, phi=phi,
                    spare=_spread(rng, 2048, 131072))
    prompts = _spread(rng, 1, max(1, min(64, 2000000 // (Hkv * (shi + members * phi)))))
    if op == "fork":
        resample = rng.random() < 0.5
        return dict(op=op, kv=kv, prompts=prompts, members=members, Hkv=Hkv, page=page, block=block, slo=slo, shi=shi, plo=plo if resample else 0,
                    phi=phi if resample else 0, resample=resample, token_major=token_major)
    return dict(op=op, kv=kv, prompts=prompts, members=members, Hkv=Hkv, page=page, block=block, slo=slo, shi=shi, plo=plo, phi=phi,
                spare=rng.choice([0.0, 0.2, 0.5]), token_major=token_major)


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
    parent = torch.clamp(j - _ints(g, 1, 4, (B, N)), min=0).to(torch.int32)
    parent[:, 0] = -1
    n = torch.where(torch.rand(B, generator=g, device="cuda") < 0.25, _ints(g, 1, N + 1, (B,)), torch.full_like(parent[:, 0], N))
    parent = torch.where(j < n[:, None], parent, torch.full_like(parent, -1))
    return parent.contiguous(), n.to(torch.int32).contiguous()


def _pool(g, c, pages):
    """One layer's cache with what earlier tokens left in it, and its scales (none for bf16)."""
    kv, Hkv, page = c["kv"], c["Hkv"], c["page"]
    shape = (pages, page, Hkv, D) if c["token_major"] else (pages, Hkv, page, D)
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
    scale = None
    if kv != "bf16":
        x = x.mul_(MOST[kv] / 4).clamp_(-MOST[kv], MOST[kv])
        scale = torch.exp(0.25 * torch.randn((pages, Hkv, page // c["block"]), generator=g, device="cuda")) * 4 / MOST[kv]
    x = x.to(TYPES[kv])
    return (x.permute(0, 2, 1, 3) if c["token_major"] else x), scale


def _pools(s, g, pages):
    s["k_pool"], s["k_scale"] = _pool(g, s["case"], pages)
    s["v_pool"], s["v_scale"] = _pool(g, s["case"], pages)


def _books(rnd, sizes, c, room, spare, system=0):
    """Page tables of groups with these numbers of members: the prompt's full pages are the group's, behind them each has its own.
    `room`: slots behind the prefix that have pages too.  Requests of all groups are mixed."""
    page = c["page"]
    order = list(range(sum(sizes)))
    rnd.shuffle(order)
    B, at, rows, groups = len(order), system, [None] * len(order), []
    prefix = np.zeros(B, np.int64)
    for size in sizes:
        idx = sorted(order.pop() for _ in range(size))
        shared = _spread(rnd, c["slo"], c["shi"]) // page if size > 1 or c["op"] != "attn" else 0
        common = np.concatenate([np.arange(system), np.arange(at, at + shared)])
        at += shared
        groups.append((idx, len(common) * page))
        for b in idx:
            mine = _spread(rnd, c["plo"], c["phi"]) if c["phi"] else 0
            prefix[b] = len(common) * page + mine if size > 1 or c["op"] != "attn" else _spread(rnd, c["slo"], c["shi"]) + mine
            own_pages = -(-(prefix[b] + room) // page) - len(common)
            rows[b] = np.concatenate([common, np.arange(at, at + own_pages)])
            at += own_pages
    # the pool is as large as the longest requests of such a case would need, and a part more
    longest = system * page + c["shi"] + c["phi"] + room
    most = system + len(sizes) * (c["shi"] // page) + B * ((c["phi"] + page + room) // page + 1) if c["op"] != "attn" else at
    pages = most + (int(most * spare) if isinstance(spare, float) else spare)
    place = np.random.RandomState(rnd.randrange(1 << 31)).permutation(pages)
    width = (longest + page) // page + 8
    table, held = np.full((B, width), -1, np.int32), np.array([len(r) for r in rows], np.int32)
    for b in range(B):
        table[b, :held[b]] = place[rows[b]]
    return table, held, prefix.astype(np.int32), groups, pages


def _sizes(rnd, groups, members):
    """Group sizes around `members`, their sum groups * members."""
    sizes = [members] * groups
    for _ in range(groups):
        a, b = rnd.randrange(groups), rnd.randrange(groups)
        if a != b and sizes[a] > 2 and sizes[b] < 2 * members:
            sizes[a], sizes[b] = sizes[a] - 1, sizes[b] + 1
    return sizes


def _state(s, table, held, prefix, pages, rnd):
    """The books of a pool as an engine keeps them, in one buffer, and a copy of it to start every pass from."""
    B, width = table.shape
    refs = np.bincount(table[table >= 0], minlength=pages).astype(np.int32)
    words = (pages + 31) // 32
    bits = np.zeros(words * 32, np.uint8)
    bits[:pages] = refs == 0
    free = np.packbits(bits, bitorder="little").view(np.int32)
    tail = np.array([[rnd.randrange(32000) for _ in range(P)] for _ in range(B)], np.int32)
    parts = dict(refs=refs, free=free, table=table, held=held, prefix=prefix, tail=tail, tail_len=np.full(B, P, np.int32))
    if "running" in s:
        parts["tail_len"][~s.pop("running")] = -1
    s["books0"] = torch.from_numpy(np.concatenate([x.reshape(-1) for x in parts.values()])).cuda()
    s["books"] = s["books0"].clone()
    at = 0
    for name, x in parts.items():
        s[name] = s["books"][at:at + x.size].view(x.shape)
        at += x.size


def prepare(case, seed):
    g, rnd = _gen(seed), random.Random(seed)
    s, c, op = dict(case=case), case, case["op"]
    if op == "attn":
        table, _, prefix, groups, pages = _books(rnd, _sizes(rnd, c["groups"], c["members"]) + [1] * c["alone"], c, c["N"], 0)
        B = len(prefix)
        leader, shared = np.arange(B, dtype=np.int32), np.zeros(B, np.int32)
        for idx, length in groups:
            if len(idx) > 1:
                leader[idx], shared[idx] = idx[0], length
        s["table"], s["prefix"], s["leader"], s["shared"] = (torch.from_numpy(x).cuda() for x in (np.maximum(table, 0), prefix, leader, shared))
        s["groups"], s["prefix_h"] = groups, prefix.tolist()                     # an engine knows them on the host as well
        s["parent"], s["n"] = _tree(g, B, c["N"])
        _pools(s, g, pages)
        s["q"] = torch.randn((B, c["N"], c["Hq"], D), generator=g, device="cuda").to(torch.bfloat16)
        s["scale"] = 1.0 / math.sqrt(D)
        return s
    sizes = [c["members"]] * c["prompts"]
    if op == "groups":
        table, held, prefix, _, pages = _books(rnd, sizes, c, 8, 64, system=c["system"])
        running = torch.rand(len(prefix), generator=g, device="cuda") < 0.9
        s["table"], s["prefix"] = torch.from_numpy(table).cuda(), torch.from_numpy(prefix).cuda()
        s["tail_len"] = torch.where(running, P, -1).to(torch.int32)
        s["min_shared"] = c["system"] * c["page"] + 1
        return s
    if op == "fork" and not c["resample"]:
        # every prompt is in one request, the other rows of its group are empty and not running
        one = dict(c, plo=1, phi=c["page"])
        table, held, prefix, _, pages = _books(rnd, [1] * c["prompts"], one, 0, c["prompts"] * c["members"])
        m, B = c["members"], c["prompts"] * c["members"]
        at = np.arange(c["prompts"]) * m + rnd.randrange(m)
        big, bh, bp = np.full((B, table.shape[1]), -1, np.int32), np.zeros(B, np.int32), np.zeros(B, np.int32)
        big[at], bh[at], bp[at] = table, held, prefix
        s["running"] = np.isin(np.arange(B), at)
        src = np.repeat(at, m).astype(np.int32)
        _state(s, big, bh, bp, pages, rnd)
    else:
        room = 0 if op == "turnover" else 8
        spare = c["prompts"] * c["members"] if op == "fork" else c["spare"]
        table, held, prefix, groups, pages = _books(rnd, sizes, c, room, spare)
        src = np.arange(len(prefix), dtype=np.int32)
        for idx, _ in groups:
            for b in idx:
                src[b] = rnd.choice(idx)
        _state(s, table, held, prefix, pages, rnd)
    if op == "fork":
        s["src"] = torch.from_numpy(src).cuda()
    if op == "turnover":
        s["done"] = (torch.rand(len(prefix), generator=g, device="cuda") < 0.25).to(torch.int32)
    if op in ("fork", "compact"):
        _pools(s, g, pages)
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


def _cached(s, which, pages):
    """The cache rows of these pages [..., w] as float32 [..., Hkv, w * page, D], scales applied."""
    pool, scale = s[which + "_pool"], s[which + "_scale"]
    pages = pages.long()
    x = pool[pages].float() if scale is None else pool.view(torch.uint8)[pages].view(pool.dtype).float()
    if scale is not None:
        x = x * scale[pages].repeat_interleave(s["case"]["block"], -1)[..., None]
    return x.transpose(-4, -3).flatten(-3, -2)


def _attn_plain(s):
    c, N, page = s["case"], s["case"]["N"], s["case"]["page"]
    Hkv, G = c["Hkv"], c["Hq"] // c["Hkv"]
    out = torch.zeros(s["q"].shape, device="cuda")
    lse = torch.zeros(s["q"].shape[:3], device="cuda")
    anc = _ancestors(s["parent"], s["n"])
    for idx, shared in s["groups"]:
        m, sp = len(idx), shared // page if len(idx) > 1 else 0
        width = max(-(-(s["prefix_h"][b] + N) // page) for b in idx)
        q = s["q"][idx].float().unflatten(2, (Hkv, G)).permute(2, 0, 1, 3, 4)                  # [Hkv, m, N, G, D]
        table = s["table"][idx]
        k, v = _cached(s, "k", table[0, :sp]), _cached(s, "v", table[0, :sp])                  # [Hkv, S, D]
        zs = (q.flatten(1, 3) @ k.transpose(-1, -2) * s["scale"]).unflatten(1, (m, N * G))     # [Hkv, m, N * G, S]
        ko, vo = (_cached(s, x, table[:, sp:width]).transpose(0, 1) for x in "kv")             # [Hkv, m, L, D]
        col = sp * page + torch.arange((width - sp) * page, device="cuda") - s["prefix"][idx][:, None]
        live = (col < s["n"][idx][:, None])
        seen = torch.gather(anc[idx], 2, col.clamp(0, N - 1).long()[:, None, :].expand(m, N, -1)) & live[:, None, :]
        seen = (seen | (col < 0)[:, None, :]).repeat_interleave(G, 1)                          # [m, N * G, L]
        zo = (q.flatten(2, 3) @ ko.transpose(-1, -2) * s["scale"]).masked_fill(~seen, -math.inf)
        vo = torch.where(live[:, :, None], vo, torch.zeros_like(vo))
        top = zo.amax(-1, keepdim=True)
        if sp:
            top = torch.maximum(top, zs.amax(-1, keepdim=True))
        ps, po = torch.exp(zs - top), torch.exp(zo - top)
        den = ps.sum(-1, keepdim=True) + po.sum(-1, keepdim=True)
        o = ((ps.flatten(1, 2) @ v).unflatten(1, (m, N * G)) + po @ vo) / den
        out[idx] = o.unflatten(2, (N, G)).permute(1, 2, 0, 3, 4).flatten(2, 3)
        lse[idx] = (top + torch.log(den))[..., 0].unflatten(2, (N, G)).permute(1, 2, 0, 3).flatten(2, 3)
    live = (torch.arange(N, device="cuda") < s["n"][:, None])[:, :, None]
    return torch.where(live[..., None], out, torch.zeros_like(out)).to(torch.bfloat16), torch.where(live, lse, torch.zeros_like(lse))


def _free_first(s):
    """The pages in the order in which they are given out: free ones from the lowest up."""
    return torch.sort((s["refs"] > 0).to(torch.int32), stable=True).indices.to(torch.int32)


def _count(s, rows):
    """How often every page is in the marked entries of the tables."""
    pages = s["refs"].numel()
    flat = torch.where(rows, s["table"], pages).flatten().long()
    return torch.zeros(pages + 1, dtype=torch.int32, device="cuda").scatter_add_(0, flat, torch.ones_like(flat, dtype=torch.int32))[:pages]


def _free_bits(s):
    bits = torch.zeros(s["free"].numel() * 32, dtype=torch.int64, device="cuda")
    bits[:s["refs"].numel()] = s["refs"] == 0
    word = (bits.view(-1, 32) << torch.arange(32, device="cuda")).sum(1)
    s["free"].copy_(torch.where(word >= 2 ** 31, word - 2 ** 32, word))


def _cols(s):
    return torch.arange(s["table"].shape[1], device="cuda", dtype=torch.int32)[None, :]


def _move_rows(s, frm, to, rows):
    page = s["case"]["page"]
    for which in "kv":
        pool, scale = s[which + "_pool"], s[which + "_scale"]
        pool = pool if scale is None else pool.view(torch.uint8)
        keep = (torch.arange(page, device="cuda") < rows[:, None])[:, None, :, None]
        pool[to] = torch.where(keep, pool[frm], pool[to])
        if scale is not None:
            first = torch.arange(0, page, s["case"]["block"], device="cuda")
            scale[to] = torch.where((first < rows[:, None])[:, None, :], scale[frm], scale[to])


def _fork_plain(s):
    page, B = s["case"]["page"], s["src"].numel()
    me = torch.arange(B, device="cuda")
    src = s["src"].clamp(min=0).long()
    take = (s["src"] >= 0) & (src != me) & (s["tail_len"][src] >= 0)
    full, rows = s["prefix"][src] // page, s["prefix"][src] % page
    last = torch.gather(s["table"][src], 1, full.clamp(max=s["table"].shape[1] - 1).long()[:, None])[:, 0].clamp(min=0)
    part = take & (rows > 0)
    first = torch.full((B,), B, device="cuda").scatter_reduce_(0, src, torch.where(take, me, B), "amin")
    hand = part & take[src] & (first[src] == me) & (s["refs"][last.long()] == 1)
    fresh = part & ~hand
    to = _free_first(s)[(torch.cumsum(fresh, 0) - 1).clamp(min=0)]
    col = _cols(s)
    mark = torch.where(hand, last, to)[:, None]
    new = torch.where(col < full[:, None], s["table"][src], torch.where((col == full[:, None]) & part[:, None], mark, -1))
    lost = _count(s, (col < s["held"][:, None]) & take[:, None])
    s["table"].copy_(torch.where(take[:, None], new, s["table"]))
    s["held"].copy_(torch.where(take, full + part, s["held"]))
    s["refs"].add_(_count(s, (col < s["held"][:, None]) & take[:, None]) - lost)
    _free_bits(s)
    for x in ("prefix", "tail", "tail_len"):
        s[x].copy_(s[x][torch.where(take, src, me)])
    _move_rows(s, last[fresh].long(), to[fresh].long(), rows[fresh])
    return torch.ones(1, dtype=torch.int32, device="cuda"), fresh.sum().to(torch.int32).view(1)


def _turnover_plain(s):
    col = _cols(s)
    done = s["done"] > 0
    gone = (col < s["held"][:, None]) & done[:, None]
    s["refs"].sub_(_count(s, gone))
    s["table"].masked_fill_(gone, -1)
    s["held"].masked_fill_(done, 0)
    s["tail_len"].masked_fill_(done, -1)
    want = (s["prefix"] + s["case"]["N"] + s["case"]["page"] - 1) // s["case"]["page"]
    need = torch.where(s["tail_len"] >= 0, (want - s["held"]).clamp(min=0), 0)
    upto = torch.cumsum(need, 0)
    granted = (s["tail_len"] >= 0) & ((need == 0) | (upto <= (s["refs"] == 0).sum()))
    new = granted[:, None] & (col >= s["held"][:, None]) & (col < (s["held"] + need)[:, None])
    k = (upto - need)[:, None] + col - s["held"][:, None]
    s["table"].copy_(torch.where(new, _free_first(s)[k.clamp(0, s["refs"].numel() - 1).long()], s["table"]))
    s["held"].add_(torch.where(granted, need, 0).to(torch.int32))
    s["refs"].add_(_count(s, new))
    _free_bits(s)
    return (granted.to(torch.int32),)


def _compact_plain(s):
    used = s["refs"] > 0
    count = used.sum()
    page = torch.arange(used.numel(), device="cuda")
    frm, to = torch.nonzero(used & (page >= count))[:, 0].flip(0), torch.nonzero(~used & (page < count))[:, 0]
    place = page.to(torch.int32)
    place[frm] = to.to(torch.int32)
    s["table"].copy_(torch.where(_cols(s) < s["held"][:, None], place[s["table"].clamp(min=0).long()], s["table"]))
    s["refs"][to] = s["refs"][frm]
    s["refs"][frm] = 0
    _free_bits(s)
    _move_rows(s, frm, to, torch.full_like(frm, s["case"]["page"]))
    return count.to(torch.int32).view(1), torch.tensor(frm.numel(), dtype=torch.int32, device="cuda").view(1)


def _groups_plain(s):
    page, table, B = s["case"]["page"], s["table"], s["table"].shape[0]
    me = torch.arange(B, device="cuda")
    at = (s["min_shared"] + page - 1) // page - 1
    full = torch.where(s["tail_len"] >= 0, s["prefix"] // page, 0)
    key = torch.where(full > at, table[:, at], -1 - me)                          # (a request without such a page is like no other)
    same = key[:, None] == key[None, :]
    leader = same.to(torch.uint8).argmax(1)
    agree = (table == table[leader]) & (_cols(s) < torch.minimum(full, full[leader])[:, None])
    common = torch.cumprod(agree.to(torch.int32), 1).sum(1)
    least = torch.full((B,), 1 << 30, device="cuda").scatter_reduce_(0, leader, common, "amin")[leader]
    group = (same.sum(1) > 1) & (least > at)
    return torch.where(group, leader, me).to(torch.int32), torch.where(group, least * page, 0).to(torch.int32)


# ------------------------------------------------------------------------------------------------ the library's calls
def _attn_own(s, war):
    cache = (s["k_pool"], s["v_pool"]) if s["k_scale"] is None else (s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"])
    quant = s["k_scale"] is not None
    if "params" not in s:
        make, room = (war.attn_quant_params, war.new_shared_quant_workspace) if quant else (war.attn_params, war.new_shared_workspace)
        s["params"] = make(s["q"], *cache, s["table"], s["scale"])
        s["ws"] = room(s["params"], "cuda")
        s["out"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros(s["q"].shape[:3], device="cuda")
    call = war.war_verify_attn_shared_quant if quant else war.war_verify_attn_shared
    call(s["q"], *cache, s["table"], s["prefix"], s["n"], s["parent"], s["leader"], s["shared"], s["params"], s["ws"], s["out"], s["lse"])
    return s["out"], s["lse"]


def _buffers(s, war):
    """The pool's books as the calls take them, and what they write beside."""
    if "pages" not in s:
        B = s["held"].numel()
        s["pages"] = war.Pages(s["refs"], s["free"], s["table"], s["held"])
        s["copies"] = torch.zeros((s["refs"].numel() if s["case"]["op"] == "compact" else B, 3), dtype=torch.int32, device="cuda")
        s["n_copies"], s["word"] = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
        s["granted"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    return s["pages"]


def _fork_own(s, war):
    war.war_pages_fork(_buffers(s, war), s["src"], s["case"]["page"], s["prefix"], s["tail"], s["tail_len"], s["copies"], s["n_copies"], s["word"])
    war.war_pages_copy(s["copies"], s["n_copies"], s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"])
    return s["word"], s["n_copies"]


def _turnover_own(s, war):
    pages = _buffers(s, war)
    war.war_pages_free(pages, s["done"], s["tail_len"])
    war.war_pages_grow(pages, s["case"]["N"], s["case"]["page"], s["prefix"], s["tail_len"], s["granted"])
    return (s["granted"],)


def _compact_own(s, war):
    pages = _buffers(s, war)
    if "ws" not in s:
        s["ws"] = war.new_compact_workspace(pages)
    war.war_pages_compact(pages, s["case"]["page"], s["ws"], s["copies"], s["n_copies"], s["word"])
    war.war_pages_copy(s["copies"], s["n_copies"], s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"])
    return s["word"], s["n_copies"]


def _groups_own(s, war):
    if "leader" not in s:
        s["leader"], s["shared"] = torch.zeros_like(s["prefix"]), torch.zeros_like(s["prefix"])
    war.war_prefix_groups(s["table"], s["prefix"], s["tail_len"], s["case"]["page"], s["min_shared"], s["leader"], s["shared"])
    return s["leader"], s["shared"]


def run(state):
    s, op = state, state["case"]["op"]
    if op in ("fork", "turnover", "compact"):
        s["books"].copy_(s["books0"])                                            # every pass starts from the same books
    if own:
        from paper_2607_17299_b200 import binding as war
        result = dict(attn=_attn_own, fork=_fork_own, turnover=_turnover_own, compact=_compact_own, groups=_groups_own)[op](s, war)
    else:
        result = dict(attn=_attn_plain, fork=_fork_plain, turnover=_turnover_plain, compact=_compact_plain, groups=_groups_plain)[op](s)
    if op in ("attn", "groups"):
        return result
    result = (s["books"],) + result
    if op != "turnover":
        result += (s["k_pool"], s["v_pool"])
        if s["k_scale"] is not None:
            result += (s["k_scale"], s["v_scale"])
    return result


# ------------------------------------------------------------------------------------------------ work
def _mean(lo, hi):
    """Mean of lengths that are spread over their logarithm."""
    return lo if hi <= lo else (hi - lo) / math.log(hi / lo)


def work(case):
    c, op = case, case["op"]
    shared, mine = _mean(c["slo"], c["shi"]), _mean(c["plo"], c["phi"]) if c["phi"] else 0
    if op == "attn":
        B = c["groups"] * c["members"] + c["alone"]
        per_key = c["Hkv"] * (4 * D if c["kv"] == "bf16" else 2 * D + 8 / c["block"]) + 4 / c["page"]
        keys = (c["groups"] + c["alone"]) * shared + B * (mine + c["N"])
        return {"bytes": keys * per_key + B * c["N"] * c["Hq"] * (4 * D + 4), "flops": 4 * B * (shared + mine + c["N"] / 2) * c["N"] * c["Hq"] * D}
    B = c["prompts"] * c["members"]
    pages = (c["prompts"] * shared + B * mine) / c["page"]
    entries = B * (shared + mine) / c["page"]
    if op == "groups":
        return {"bytes": 4 * (entries + B * c["system"]) + 16 * B, "flops": 0}
    row = 2 * c["Hkv"] * D * (2 if c["kv"] == "bf16" else 1) if op != "turnover" else 0      # K and V of a token
    if op == "fork":
        changed = (B - c["prompts"]) if not c["resample"] else B * (1 - 1 / c["members"])
        moved = changed * (1 if not c["resample"] else 0.6) * c["page"] / 2
        return {"bytes": 2 * moved * row + changed / B * entries * 16 + B * 400, "flops": 0}
    if op == "turnover":
        return {"bytes": 0.25 * entries * 12 + B * 24 + (pages + c["spare"]) / 8, "flops": 0}
    most = (c["prompts"] * c["shi"] + B * c["phi"]) / c["page"] * (1 + c["spare"])
    moved = pages * max(0.1, 1 - pages / most) * c["page"]
    return {"bytes": 2 * moved * row + 8 * entries, "flops": 0}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """Attention in 64 bits, request by request and head by head; the other operators move whole numbers and codes."""
    if case["op"] != "attn":
        return None
    c, N, page, Hkv, G = case, case["N"], case["page"], case["Hkv"], case["Hq"] // case["Hkv"]
    B = c["groups"] * c["members"] + c["alone"]
    if B * (c["shi"] + c["phi"]) * N * c["Hq"] > 4e9:
        return None
    s = prepare(case, seed)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:3], dtype=torch.float64, device="cuda")
    parent, n = s["parent"].tolist(), s["n"].tolist()
    for b in range(B):
        m, p = n[b], s["prefix_h"][b]
        see = torch.zeros((m, p + m), dtype=torch.bool)
        see[:, :p] = True
        for j in range(m):
            a = j
            while a >= 0:
                see[j, p + a] = True
                a = parent[b][a]
        see = see.cuda()[:, None, :]
        pages = s["table"][b, : -(-(p + m) // page)].long()
        for h in range(Hkv):
            K, V = (s[x + "_pool"][pages, h].double() if s[x + "_scale"] is None else
                    s[x + "_pool"].view(torch.uint8)[pages, h].view(TYPES[c["kv"]]).double()
                    * s[x + "_scale"][pages, h].double().repeat_interleave(c["block"], 1)[..., None] for x in "kv")
            z = torch.einsum("jgd,cd->jgc", s["q"][b, :m, h * G:(h + 1) * G].double(), K.reshape(-1, D)[:p + m]) * s["scale"]
            z = torch.where(see, z, -math.inf)
            lse[b, :m, h * G:(h + 1) * G] = torch.logsumexp(z, -1)
            out[b, :m, h * G:(h + 1) * G] = torch.softmax(z, -1) @ V.reshape(-1, D)[:p + m]
    return out, lse
