"""Operators for drafted and moved tokens of the paged 8-bit cache, as cases that can be timed and compared:
attention from a tree of drafted tokens, the walk along the accepted ones, and the move of cached tokens.

A tree of drafted tokens lies in a sequence's newest slots, parents before children; each sees the slots before the tree
and its own ancestors.  Of the tokens that the model picks after every node the walk finds the path that agrees.  Kept
tokens then move together, in all layers, each block of 16 slots under a scale of its own.  Shapes are those of the
library's other cases: 28 query / 4 KV heads of 128 (and 32/8, 16/2, 14/2 of 64), prompts of 448 x 448 to 3836 x 2156 pixels.

`own` false: elementary torch operations in 32 bits; true: the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 16            # tokens that share a scale
E4M3 = torch.float8_e4m3fn
VOCAB = 152064
MAX_CODES = 960 << 20                   # cached codes of the largest listed batch of trees
MAX_SCORES = 28 * 26 * 40 * 28007       # query x key x head of it, padded to its longest
MAX_MOVED = 28 * 4 * 128 * 2 * 4260     # codes that the largest listed move writes


def _pace():
    from paper_2608_27206_gb300 import pace
    return pace


def _dev():
    return torch.device("cuda")


# ----------------------------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------------------------
def _spread(n, lo, hi):
    """n odd and even lengths from lo to hi, spread over their logarithm, in no order."""
    got = [round(lo * (hi / lo) ** (i / (n - 1))) for i in range(n)]
    return ",".join(str(got[i * 29 % n]) for i in range(n))


def _times(x, n):
    return ",".join([str(x)] * n)


def listed():
    qwen = {"q_heads": 28, "kv_heads": 4, "dim": 128}
    return [
        # one short chat about a 448 x 448 image drafts 7 tokens: the smallest tree
        {"name": "tree_1_7", "kind": "tree", "lens": "411", "nodes": "7", "shape": "random", "page": 16, "window": 0, "sinks": 0, **qwen},
        # one unpruned 4K prompt with a usual tree of 26 tokens
        {"name": "tree_1_4k", "kind": "tree", "lens": "10851", "nodes": "26", "shape": "random", "page": 64, "window": 0, "sinks": 0, **qwen},
        # eight chats with 64 drafted tokens each, four children to a node
        {"name": "tree_8_64", "kind": "tree", "lens": _spread(8, 764, 9064), "nodes": _times(64, 8), "shape": "fours", "page": 32,
         "window": 0, "sinks": 0, "q_heads": 32, "kv_heads": 8, "dim": 128},
        # 40 long chats of many images with 26 tokens each: the largest cache
        {"name": "tree_40_long", "kind": "tree", "lens": _spread(40, 5001, 28007), "nodes": _times(26, 40), "shape": "random", "page": 64,
         "window": 0, "sinks": 0, **qwen},
        # a small model's windowed layer, trees of every size, one of a single token
        {"name": "tree_16_d64", "kind": "tree", "lens": _spread(16, 405, 6001), "nodes": "1,48,7,31,64,12,3,26,100,2,5,40,17,60,9,22",
         "shape": "forest", "page": 16, "window": 1024, "sinks": 4, "q_heads": 14, "kv_heads": 2, "dim": 64},
        # a wide search: 256 drafted tokens on one pruned 4K prompt
        {"name": "tree_1_256", "kind": "tree", "lens": "4516", "nodes": "256", "shape": "random", "page": 128, "window": 0, "sinks": 0, **qwen},
        # one chat's tree of 26: nothing but latency
        {"name": "accept_1", "kind": "accept", "nodes": "26", "shape": "random"},
        # the largest batch: 512 chats
        {"name": "accept_512", "kind": "accept", "nodes": _times(64, 512), "shape": "fours"},
        # eight answers are forked from one prompt: the tokens of its part-filled last page, in all layers
        {"name": "move_fork8", "kind": "move", "what": "fork", "lens": _times(407, 8), "nodes": _times(23, 8), "kept": _times(23, 8), "layers": 28,
         "page": 64, **qwen},
        # the accepted tokens of 64 chats' trees, in all layers, into the pages that the chats keep
        {"name": "move_drafts64", "kind": "move", "what": "drafts", "lens": _spread(64, 700, 1900), "nodes": _times(26, 64),
         "kept": ",".join(["3,1,5,2,4,2,7,1"] * 8), "layers": 28, "page": 32, **qwen},
        # a cached 4K prompt is pruned to 40 % of its visual tokens for one question, and stays whole for the next: all layers
        {"name": "move_prune_4k", "kind": "move", "what": "prune", "lens": "10589", "nodes": "10589", "kept": "4260", "layers": 28, "page": 64,
         **qwen},
        # the same in the layers below the one that scores the tokens, for a batch of ragged prompts of a small model
        {"name": "move_prune_d64", "kind": "move", "what": "prune", "lens": "1064,404,2700,1303,333,2016", "nodes": "1064,404,2693,1303,333,2000",
         "kept": "445,181,1096,540,152,817", "layers": 2, "page": 16, "q_heads": 14, "kv_heads": 2, "dim": 64},
    ]


HEADS = [(28, 4, 128), (28, 4, 128), (28, 4, 128), (32, 8, 128), (16, 2, 128), (14, 2, 64)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _csv(v):
    return ",".join(map(str, v))


def draw(rng):
    hq, hk, d = rng.choice(HEADS)
    base = {"page": rng.choice([16, 32, 64, 128, 256]), "q_heads": hq, "kv_heads": hk, "dim": d}
    kind = rng.choice(["tree", "tree", "tree", "accept", "move", "move"])
    shape = rng.choice(["random", "random", "fours", "chain", "forest"])
    if kind == "accept":
        nodes = [_log_int(rng, 1, 256) for _ in range(_log_int(rng, 1, 512))]
        while sum(nodes) > 512 * 64:
            nodes.pop()
        return {"kind": kind, "nodes": _csv(nodes), "shape": shape}
    if kind == "tree":
        n, most = _log_int(rng, 1, 40), _log_int(rng, 4, 256)
        nodes = [_log_int(rng, 1, most) for _ in range(n)]
        lens = [x + _log_int(rng, 1, 28000) for x in nodes]
        while len(lens) > 1 and (len(lens) * max(lens) * 2 * hk * d > MAX_CODES or len(lens) * max(nodes) * max(lens) * hq > MAX_SCORES):
            lens.pop()
            nodes.pop()
        window, sinks = rng.choice([(0, 0), (0, 0), (0, 0), (4096, 4), (1024, 4), (_log_int(rng, 16, 8000), rng.randrange(0, 65))])
        return {"kind": kind, "lens": _csv(lens), "nodes": _csv(nodes), "shape": shape, "window": window, "sinks": sinks, **base}
    what, layers = rng.choice(["fork", "drafts", "prune"]), rng.choice([1, 2, 14, 28])
    if what == "fork":
        length = _log_int(rng, 20, 6000)
        if length % base["page"] == 0:
            length += 5
        n = length % base["page"]
        nodes = [n] * _log_int(rng, 1, 32)
        lens, kept = [length] * len(nodes), list(nodes)
    elif what == "drafts":
        nodes = [_log_int(rng, 2, 100) for _ in range(_log_int(rng, 1, 96))]
        kept = [min(x, _log_int(rng, 1, 12)) for x in nodes]
        lens = [x + _log_int(rng, 1, 4000) for x in nodes]
    else:
        nodes = [_log_int(rng, 64, 10000) for _ in range(rng.choice([1, 1, 2, 4]))]
        kept = [max(1, round(x * rng.uniform(0.05, 0.95))) for x in nodes]
        lens = [x + rng.choice([0, 0, rng.randrange(40)]) for x in nodes]
    while len(nodes) > 1 and sum(kept) * layers * 2 * hk * d > MAX_MOVED:
        nodes.pop(), kept.pop(), lens.pop()
    while sum(kept) * layers * 2 * hk * d > MAX_MOVED or sum(lens) * layers * 2 * hk * d > 3 * MAX_MOVED:
        layers = max(1, layers // 2)
        if layers == 1:
            kept = [min(kept[0], MAX_MOVED // (2 * hk * d))]
            break
    return {"kind": kind, "what": what, "lens": _csv(lens), "nodes": _csv(nodes), "kept": _csv(kept), "layers": layers, **base}


# ----------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------
def _gen(seed, part=0):
    g = torch.Generator(device=_dev())
    g.manual_seed(1000003 * int(seed) + part)
    return g


def _numbers(text):
    return [int(x) for x in str(text).split(",")]


def _prefix(n):
    out = [0]
    for x in n:
        out.append(out[-1] + x)
    return out


def _device_ints(x):
    return torch.tensor(x, dtype=torch.int32, device=_dev())


def _seq_and_place(cu):
    """Of every row of a packed batch: its sequence, and its place there."""
    n = torch.tensor([b - a for a, b in zip(cu, cu[1:])], device=_dev())
    seq = torch.repeat_interleave(torch.arange(n.numel(), device=_dev()), n)
    return seq, torch.arange(cu[-1], device=_dev()) - torch.tensor(cu, device=_dev())[seq]


def _parents(g, cu, shape):
    """int32 [nodes]: each node's parent in its own tree, -1 for none; node 0 has none."""
    _, t = _seq_and_place(cu)
    u = torch.rand(t.numel(), generator=g, device=_dev(), dtype=torch.float64)
    if shape == "chain":
        p = t - 1
    elif shape == "fours":
        p = (t - 1) // 4
    else:
        p = (u * t).long().clamp(max=t - 1)
        if shape == "forest":       # some nodes that follow the context itself
            p = torch.where(torch.rand(t.numel(), generator=g, device=_dev()) < 0.15, torch.full_like(p, -1), p)
    return torch.where(t > 0, p, torch.full_like(p, -1)).to(torch.int32)


def _tokens(g, rows, heads, dim):
    """bf16 [rows, heads, dim]: N(0, 1) times one LogNormal(0, 0.5) factor per row."""
    x = torch.randn(rows, heads, dim, generator=g, device=_dev())
    return (x * torch.exp(0.5 * torch.randn(rows, 1, 1, generator=g, device=_dev()))).to(torch.bfloat16)


def _pow2(e):
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _scale_for(amax):
    """The smallest power of two s with amax <= 448 s, between 2^-64 and 2^120."""
    f, e = torch.frexp(amax)
    e = e - 9 + (f > 0.875)
    return _pow2(torch.where(amax > 0, e, torch.full_like(e, -64)).clamp(-64, 120))


def _pages(g, lens, page, spare=3):
    """Shuffled pages for sequences of `lens` slots: the table (-1 behind a sequence's last page) and their number."""
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + spare
    order = torch.randperm(n_pages, generator=g, device=_dev()).to(torch.int32)
    table = torch.full((len(lens), max(max(need), 1)), -1, dtype=torch.int32, device=_dev())
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, n_pages


def _codes(g, n_pages, heads, page, dim):
    """Codes and scales that stand for such tokens."""
    x = torch.randn(n_pages, heads, page, dim, generator=g, device=_dev())
    x *= torch.exp(0.5 * torch.randn(n_pages, 1, page, 1, generator=g, device=_dev()))
    x = x.view(n_pages, heads, page // BLOCK, BLOCK * dim)
    s = _scale_for(x.abs().amax(3))
    return (x / s[..., None]).to(E4M3).view(n_pages, heads, page, dim), s


def _forget(codes, scales, used):
    """NaN in every slot of a page behind its `used` first ones, and in scales of blocks without a used slot."""
    page = codes.shape[-2]
    free = torch.arange(page, device=_dev())[None, :] >= used[:, None]
    codes.view(torch.uint8).masked_fill_(free[:, None, :, None], 0x7F)
    scales.masked_fill_(free[:, None, ::BLOCK], math.nan)


def _used(table, lens, n_pages, page):
    """Slots of each page that hold a token."""
    used = torch.zeros(n_pages, dtype=torch.int64, device=_dev())
    count = (lens[:, None].long() - torch.arange(table.shape[1], device=_dev()) * page).clamp(0, page).reshape(-1)
    used[table.clamp(min=0).long().reshape(-1)[count > 0]] = count[count > 0]
    return used


def _prepare_tree(case, seed):
    hq, hk, d, page = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    lens, nodes, g = _numbers(case["lens"]), _numbers(case["nodes"]), _gen(seed, 1)
    s = {"case": dict(case), "nodes": nodes, "cu": _prefix(nodes), "max_len": max(lens), "lens": _device_ints(lens)}
    s["table"], n_pages = _pages(g, lens, page)
    s["k"], s["ks"] = _codes(g, n_pages, hk, page, d)
    s["v"], s["vs"] = _codes(g, n_pages, hk, page, d)
    used = _used(s["table"], s["lens"], n_pages, page)
    _forget(s["k"], s["ks"], used)
    _forget(s["v"], s["vs"], used)
    s["Q"] = _tokens(_gen(seed, 2), s["cu"][-1], hq, d)
    s["parents"] = _parents(_gen(seed, 3), s["cu"], case["shape"])
    s["out"] = torch.empty_like(s["Q"])
    if own:     # what a program that uses the library keeps: the cache's handle and the workspace
        P = _pace()
        s["cache"] = P.KvCache(s["k"], s["v"], s["ks"], s["vs"])
        n = P.pace_kv_tree_attention_workspace_size(s["cache"], s["cu"], hq, s["max_len"])
        s["ws"] = torch.empty(max(n, 16), dtype=torch.uint8, device=_dev())
    return s


def _prepare_accept(case, seed):
    nodes, g = _numbers(case["nodes"]), _gen(seed, 1)
    cu = _prefix(nodes)
    n = cu[-1]
    s = {"case": dict(case), "nodes": nodes, "cu": cu, "parents": _parents(g, cu, case["shape"])}
    seq, t = _seq_and_place(cu)
    s["tokens"] = torch.randint(0, VOCAB, (n,), generator=g, device=_dev()).to(torch.int32)
    # a token is picked after every node; for most of those with children it is one of theirs
    right = torch.full((n + 1,), -1, dtype=torch.int64, device=_dev())
    chosen = (s["parents"] >= 0) & (torch.rand(n, generator=g, device=_dev()) < 0.6)
    at = torch.where(chosen, s["parents"].long() + t.new_tensor(cu)[seq], torch.full_like(t, n))
    right.scatter_reduce_(0, at, torch.arange(n, device=_dev()), "amax")
    other = torch.randint(0, VOCAB, (n,), generator=g, device=_dev()).to(torch.int32)
    s["picked"] = torch.where(right[:n] >= 0, s["tokens"][right[:n].clamp(min=0)], other)
    s["rows"], s["counts"] = torch.empty(n, dtype=torch.int32, device=_dev()), torch.empty(len(nodes), dtype=torch.int32, device=_dev())
    s["next"] = torch.empty_like(s["counts"])
    return s


def _prepare_move(case, seed):
    hk, d, page, layers = case["kv_heads"], case["dim"], case["page"], case["layers"]
    lens, nodes, kept, g = _numbers(case["lens"]), _numbers(case["nodes"]), _numbers(case["kept"]), _gen(seed, 1)
    B = len(lens)
    s = {"case": dict(case), "nodes": nodes, "cu": _prefix(nodes), "lens": _device_ints(lens)}
    # From the page in that its newest tokens begin a sequence has pages of its own, and others where the kept ones go; what is
    # before them is shared (one image, many questions) and stays where it is.  Forked answers have the newest tokens' pages in common too.
    first = [(a - n) // page for a, n in zip(lens, nodes)]
    tail = [-(-a // page) - f for a, f in zip(lens, first)]
    dst_tail = [-(-(a - n + k) // page) - f for a, n, k, f in zip(lens, nodes, kept, first)]
    fork = case["what"] == "fork"
    src, n_src = _pages(g, [x * page for x in (tail[:1] if fork else tail)], page, 0)
    dst, n_dst = _pages(g, [x * page for x in dst_tail], page, 0)
    width = max(f + max(a, b) for f, a, b in zip(first, tail, dst_tail))
    common = 2
    s["table"] = torch.full((B, width), -1, dtype=torch.int32, device=_dev())
    for b in range(B):
        s["table"][b, :first[b]] = torch.arange(first[b], dtype=torch.int32, device=_dev()) % common
    s["dst"] = s["table"].clone()
    for b in range(B):
        f = first[b]
        s["table"][b, f:f + tail[b]] = common + src[0 if fork else b, :tail[b]]
        s["dst"][b, f:f + dst_tail[b]] = common + n_src + dst[b, :dst_tail[b]]
    n_pages = common + n_src + n_dst
    s["k"], s["v"] = (torch.empty((layers, n_pages, hk, page, d), dtype=E4M3, device=_dev()) for _ in "kv")
    s["ks"], s["vs"] = (torch.empty((layers, n_pages, hk, page // BLOCK), dtype=torch.float32, device=_dev()) for _ in "kv")
    before = torch.tensor([a - n for a, n in zip(lens, nodes)], device=_dev())
    used = torch.maximum(_used(s["table"], s["lens"], n_pages, page), _used(s["dst"], before, n_pages, page))
    for l in range(layers):
        for c, f in (("k", "ks"), ("v", "vs")):
            x, y = _codes(g, n_pages, hk, page, d)
            y *= _pow2(torch.randint(-2, 3, y.shape, generator=g, device=_dev()))      # (channels of a real model differ more than these)
            s[c][l], s[f][l] = x, y
            _forget(s[c][l], s[f][l], used)
    # what stays: the first of a tree's nodes and a path, a prompt's text and its best visual tokens, or everything
    seq, t = _seq_and_place(s["cu"])
    rank = torch.rand(t.numel(), generator=g, device=_dev())
    rank = torch.where((t < 20) & (torch.tensor(kept, device=_dev())[seq] > 20) | (t == 0), rank - 1, rank)
    rows, cu_rows = [], [0]
    for b in range(B):
        a, z = s["cu"][b], s["cu"][b + 1]
        rows.append(rank[a:z].argsort()[:kept[b]].sort().values + a)
        cu_rows.append(cu_rows[-1] + kept[b])
    s["cu_rows"], s["counts"] = cu_rows, None
    s["rows"] = None if fork else torch.cat(rows).to(torch.int32)
    if case["what"] == "drafts":        # as the walk leaves them: a list as long as the tree, and how many count
        s["rows"] = torch.full((s["cu"][-1],), -1, dtype=torch.int32, device=_dev())
        for b in range(B):
            s["rows"][s["cu"][b]:s["cu"][b] + kept[b]] = rows[b].to(torch.int32)
        s["cu_rows"], s["counts"] = s["cu"], _device_ints(kept)
    s["new_lens"] = torch.empty(B, dtype=torch.int32, device=_dev())
    if own:     # the handle of the layers
        P = _pace()
        s["cache"] = P.KvLayers([P.KvCache(s["k"][l], s["v"][l], s["ks"][l], s["vs"][l]) for l in range(layers)])
    return s


def prepare(case, seed):
    return {"tree": _prepare_tree, "accept": _prepare_accept, "move": _prepare_move}[case["kind"]](case, seed)


# ----------------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if not own:
        return {"tree": _plain_tree, "accept": _plain_accept, "move": _plain_move}[case["kind"]](s)
    P = _pace()
    if case["kind"] == "tree":
        return P.pace_kv_tree_attention(s["cache"], s["Q"], s["cu"], s["parents"], s["lens"], s["table"], s["max_len"], window=case["window"],
                                        sinks=case["sinks"], out=s["out"], ws=s["ws"])
    if case["kind"] == "accept":
        P.pace_draft_accept(s["tokens"], s["parents"], s["picked"], s["cu"], rows=s["rows"], counts=s["counts"], next_tokens=s["next"])
        return {"rows": s["rows"], "counts": s["counts"], "next": s["next"]}
    P.pace_kv_compact(s["cache"], s["cu"], s["lens"], s["table"], cu_rows=s["cu_rows"], rows=s["rows"], counts=s["counts"],
                      dst_table=s["dst"], new_lens=s["new_lens"])
    return _moved(s)


def _moved(s):
    """The whole cache, as the values that its codes have and the scales they are multiplied by, and the lengths."""
    return {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"], "lens": s["new_lens"]}


# ---- plain form: the tree --------------------------------------------------------------------
def _dense(codes, scales, table):
    """[B, heads, slots, D] in 32 bits: every sequence's pages, one after the other."""
    at = table.clamp(min=0).long()
    x = codes.view(torch.uint8)[at].view(E4M3).float()
    b, n, h, page, d = x.shape
    x = x.view(b, n, h, page // BLOCK, BLOCK, d).mul_(scales[at][..., None, None])
    return x.view(b, n, h, page, d).transpose(1, 2).reshape(b, h, n * page, d)


def _family(parents, nodes):
    """[B, T, T]: whether u is t or one of its ancestors.  The k-th square of "itself or its parent" reaches 2^k generations up."""
    B, T = parents.shape
    a = torch.eye(T, device=_dev()).repeat(B, 1, 1)
    a.scatter_(2, parents.clamp(min=0)[..., None], torch.maximum(a.gather(2, parents.clamp(min=0)[..., None]), (parents >= 0).float()[..., None]))
    for _ in range(max(1, (T - 1).bit_length())):
        a = (torch.matmul(a, a) > 0).float()
    return a > 0


def _plain_tree(s):
    case, B, most = s["case"], len(s["nodes"]), max(s["nodes"])
    hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
    nodes, cu = torch.tensor(s["nodes"], device=_dev()), torch.tensor(s["cu"][:-1], device=_dev())
    t = torch.arange(most, device=_dev())
    there = t[None, :] < nodes[:, None]                                 # [B, T]
    row = (cu[:, None] + t).clamp(max=s["cu"][-1] - 1)
    family = _family(torch.where(there, s["parents"][row].long(), -torch.ones_like(row)), nodes)
    depth = family.sum(2) - 1
    q = s["Q"][row].float()                                             # [B, T, Hq, D]
    k, v = _dense(s["k"], s["ks"], s["table"]), _dense(s["v"], s["vs"], s["table"])
    j = torch.arange(k.shape[2], device=_dev())
    base = (s["lens"].long() - nodes)[:, None]                          # [B, 1]
    node = (j - base).clamp(0, most - 1)                                # [B, slots]
    place = torch.where(j < base, j.expand_as(node), base + depth.gather(1, node))
    inside = (j >= base) & (j < base + nodes[:, None])
    see = (j < base)[:, None] | (family.gather(2, node[:, None].expand(-1, most, -1)) & inside[:, None])
    if case["window"] > 0:
        see &= (place[:, None] > (base + depth)[..., None] - case["window"]) | (place < case["sinks"])[:, None]
    see &= there[..., None]
    any_sees = see.any(1)[:, None, :, None]
    k, v = torch.where(any_sees, k, torch.zeros_like(k[:1, :1, :1, :1])), torch.where(any_sees, v, torch.zeros_like(v[:1, :1, :1, :1]))
    q = q.view(B, most, hk, hq // hk, d).permute(0, 2, 1, 3, 4).reshape(B, hk, -1, d)
    w = torch.matmul(q * d ** -0.5, k.transpose(2, 3)).view(B, hk, most, hq // hk, -1)
    w.masked_fill_(~see[:, None, :, None, :], -math.inf)
    top = w.amax(4, keepdim=True)
    w.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = w.sum(4).view(B, hk, -1, 1)
    o = torch.matmul(w.view(B, hk, -1, w.shape[4]), v) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.view(B, hk, most, hq // hk, d).permute(0, 2, 1, 3, 4).reshape(B, most, hq, d)
    return o[there].to(torch.bfloat16)


# ---- plain form: the walk --------------------------------------------------------------------
def _plain_accept(s):
    cu, n, B = torch.tensor(s["cu"], device=_dev()), s["cu"][-1], len(s["nodes"])
    seq, t = _seq_and_place(s["cu"])
    me = torch.arange(n, device=_dev())
    up = torch.where(s["parents"] >= 0, s["parents"].long() + cu[seq], torch.full_like(me, n))
    picked = torch.cat([s["picked"], s["picked"].new_full((1,), -1)])
    agrees = (up < n) & (s["tokens"] == picked[up])
    # of every node the first child that agrees (n: none); then whom 1, 2, 4, ... such steps from node 0 reach
    to = torch.full((n + 1,), n, dtype=torch.int64, device=_dev())
    to.scatter_reduce_(0, torch.where(agrees, up, torch.full_like(up, n)), torch.where(agrees, me, torch.full_like(me, n)), "amin")
    to[n] = n
    on = torch.cat([t == 0, torch.zeros(1, dtype=torch.bool, device=_dev())])
    for _ in range(max(1, (max(s["nodes"]) - 1).bit_length())):
        reached = torch.zeros(n + 1, dtype=torch.int64, device=_dev()).scatter_reduce_(0, to, on.long(), "amax")
        on = on | (reached > 0)
        on[n] = False
        to = to[to]
    on = on[:n]
    rank = torch.cumsum(on.long(), 0)
    before = torch.cat([rank.new_zeros(1), rank])[cu[seq]]
    place = torch.where(on, cu[seq] + rank - before - 1, torch.full_like(me, n))
    rows = torch.full((n + 1,), -1, dtype=torch.int64, device=_dev())
    rows[place] = torch.where(on, me, torch.full_like(me, -1))
    counts = torch.zeros(B, dtype=torch.int64, device=_dev()).scatter_add_(0, seq, on.long())
    last = torch.zeros(B, dtype=torch.int64, device=_dev()).scatter_reduce_(0, seq, torch.where(on, me, torch.zeros_like(me)), "amax")
    return {"rows": rows[:n].to(torch.int32), "counts": counts.to(torch.int32), "next": s["picked"][last]}


# ---- plain form: the move --------------------------------------------------------------------
def _plain_move(s):
    page = s["case"]["page"]
    nodes, lens = torch.tensor(s["nodes"], device=_dev()), s["lens"].long()
    base = lens - nodes
    seq, place = _seq_and_place(s["cu_rows"])
    count = s["counts"].long() if s["counts"] is not None else torch.bincount(seq, minlength=nodes.numel())
    live = place < count[seq]
    row = s["rows"].long() if s["rows"] is not None else torch.arange(place.numel(), device=_dev())
    src = base[seq] + row - torch.tensor(s["cu"], device=_dev())[seq]
    seq, place, src = seq[live], place[live], src[live]
    # the tokens that move, and those that are in the first block already
    lead = base % BLOCK
    early = torch.arange(BLOCK, device=_dev())
    has = (early < lead[:, None]) & (count > 0)[:, None]
    e_seq, e_at = has.nonzero(as_tuple=True)
    from_page = torch.cat([s["table"][seq, src // page], s["dst"][e_seq, (base[e_seq] - lead[e_seq]) // page]]).long()
    slot = torch.cat([base[seq] + place, base[e_seq] - lead[e_seq] + e_at])
    src = torch.cat([src, slot[seq.numel():]])
    to_page = s["dst"][torch.cat([seq, e_seq]), slot // page].long()
    layers, _, heads, _, dim = s["k"].shape
    per = page // BLOCK
    for codes, scales in ((s["k"], s["ks"]), (s["v"], s["vs"])):
        raw = codes.view(torch.uint8)
        x = raw[:, from_page, :, src % page].view(E4M3).float()                     # [tokens, layers, heads, D]
        x = x * scales[:, from_page, :, src % page // BLOCK][..., None]
        block = ((torch.arange(layers, device=_dev())[:, None] * codes.shape[1] + to_page[:, None, None]) * heads
                 + torch.arange(heads, device=_dev())) * per + (slot % page // BLOCK)[:, None, None]
        amax = torch.zeros(scales.numel(), device=_dev())
        amax.scatter_reduce_(0, block.reshape(-1), x.abs().amax(3).reshape(-1), "amax")
        now = _scale_for(amax)[block]
        scales.view(-1)[block.reshape(-1)] = now.reshape(-1)
        raw[:, to_page, :, slot % page] = (x / now[..., None]).to(E4M3).view(torch.uint8)
    s["new_lens"].copy_(base + count)
    return _moved(s)


# ----------------------------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------------------------
def _seen(length, nodes, window, sinks):
    """Query-key pairs of a sequence in its context (a node's own ancestors left out: few), and the slots that some node sees."""
    base = length - nodes
    keys = base if window <= 0 else min(base, window - 1 + min(sinks, max(0, base - window + 1)))
    return nodes * (keys + 1), keys + nodes


def work(case):
    nodes = _numbers(case["nodes"])
    if case["kind"] == "accept":
        return {"bytes": 16 * sum(nodes) + 8 * len(nodes), "flops": 0}
    hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "move":
        read = _numbers(case["kept"])[:1] if case["what"] == "fork" else _numbers(case["kept"])
        return {"bytes": case["layers"] * (sum(read) + sum(_numbers(case["kept"]))) * hk * (2 * d + 8 / BLOCK), "flops": 0}
    seen = [_seen(a, b, case["window"], case["sinks"]) for a, b in zip(_numbers(case["lens"]), nodes)]
    return {"bytes": (4 * hq * d + 4) * sum(nodes) + sum(x[1] for x in seen) * hk * (2 * d + 8 / BLOCK),
            "flops": 4 * d * hq * sum(x[0] for x in seen)}


# ----------------------------------------------------------------------------------------------
# the same in 64 bits
# ----------------------------------------------------------------------------------------------
def _inputs(case, seed):
    """The inputs alone, whatever `own` says."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def _exact_tree(case, seed):
    s = _inputs(case, seed)
    hk, g, d, page = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["dim"], case["page"]
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device=_dev())
    parents = s["parents"].tolist()
    for b, (L, n) in enumerate(zip(_numbers(case["lens"]), s["nodes"])):
        a, base = s["cu"][b], L - n
        hide = torch.zeros((n, L), dtype=torch.bool)
        depth, above = [], []
        for t in range(n):
            p = parents[a + t]
            depth.append(0 if p < 0 else depth[p] + 1)
            above.append([t] if p < 0 else above[p] + [t])
            hide[t, base:] = True
            hide[t, [base + u for u in above[t]]] = False
        if case["window"] > 0:
            at = torch.cat([torch.arange(base), base + torch.tensor(depth)])
            last = base + torch.tensor(depth)[:, None]
            hide |= (at <= last - case["window"]) & (at >= case["sinks"])
        hide = hide.to(_dev())
        pages = s["table"][b, :-(-L // page)].long()
        for h in range(hk):
            kv = []
            for c, f in ((s["k"], s["ks"]), (s["v"], s["vs"])):
                x = c.view(torch.uint8)[pages, h].view(E4M3).double().view(-1, BLOCK, d) * f[pages, h].double().view(-1, 1, 1)
                kv.append(x.view(-1, d)[:L])
            w = (s["Q"][a:a + n, h * g:(h + 1) * g].double().reshape(-1, d) @ kv[0].t() * d ** -0.5).view(n, g, L)
            w = torch.softmax(w.masked_fill(hide[:, None], -math.inf), 2)
            out[a:a + n, h * g:(h + 1) * g] = (w.view(-1, L) @ kv[1]).view(n, g, d)
    return out


def _pow2_64(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _e4m3_64(x):
    """The value with 4 significant bits, no finer than 2^-9, that is nearest to x; ties to even."""
    _, e = torch.frexp(x)
    step = _pow2_64((e - 1).clamp(min=-6) - 3)
    return (x / step).round() * step


def _exact_move(case, seed):
    s = _inputs(case, seed)
    page, out = case["page"], {}
    lists = [[] for _ in s["nodes"]]
    rows = list(range(s["cu"][-1])) if s["rows"] is None else s["rows"].tolist()
    for b, k in enumerate(_numbers(case["kept"])):
        lists[b] = [r - s["cu"][b] for r in rows[s["cu_rows"][b]:s["cu_rows"][b] + k]]
    lens = _numbers(case["lens"])
    for c, f in (("k", "ks"), ("v", "vs")):
        codes, scales = s[c].double(), s[f].double()
        was = codes.clone(), scales.clone()
        layers, _, heads, _, dim = codes.shape
        for b, kept in enumerate(lists):
            base = lens[b] - s["nodes"][b]
            lead = base % BLOCK
            at = torch.tensor(list(range(base - lead, base)) + [base + r for r in kept], device=_dev())
            from_page = torch.cat([s["dst"][b, at[:lead] // page], s["table"][b, at[lead:] // page]]).long()
            x = was[0][:, from_page, :, at % page] * was[1][:, from_page, :, at % page // BLOCK][..., None]      # [tokens, layers, heads, D]
            n = x.shape[0]
            pad = -n % BLOCK
            x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, 0, 0, pad)).view(-1, BLOCK, layers, heads, dim)
            fr, e = torch.frexp(x.abs().amax((1, 4)) / 448)      # the least e with amax / 448 <= 2^e
            e = torch.where(fr > 0.5, e, e - 1)
            sc = _pow2_64(torch.where(fr > 0, e, torch.full_like(e, -64)).clamp(-64, 120))      # [blocks, layers, heads]
            y = _e4m3_64(x / sc[:, None, :, :, None]).view(-1, layers, heads, dim)[:n]
            slot = torch.arange(n, device=_dev()) + base - lead
            codes[:, s["dst"][b, slot // page].long(), :, slot % page] = y
            scales[:, s["dst"][b, slot[::BLOCK] // page].long(), :, slot[::BLOCK] % page // BLOCK] = sc
        out[c], out[f] = codes, scales
    out["lens"] = torch.tensor([a - n + len(k) for a, n, k in zip(lens, s["nodes"], lists)], dtype=torch.int32, device=_dev())
    return out


def _exact_accept(case, seed):
    s = _inputs(case, seed)
    tokens, parents, picked = s["tokens"].tolist(), s["parents"].tolist(), s["picked"].tolist()
    rows, counts, after = [-1] * len(tokens), [], []
    for a, z in zip(s["cu"], s["cu"][1:]):
        path = [a]
        for t in range(a + 1, z):       # (children come after their parents)
            if parents[t] + a == path[-1] and parents[t] >= 0 and tokens[t] == picked[path[-1]]:
                path.append(t)
        rows[a:a + len(path)] = path
        counts.append(len(path))
        after.append(picked[path[-1]])
    return {"rows": _device_ints(rows), "counts": _device_ints(counts), "next": _device_ints(after)}


def exact(case, seed):
    return {"tree": _exact_tree, "accept": _exact_accept, "move": _exact_move}[case["kind"]](case, seed)
