"""A step of speculative decoding on grouped-query layers over the paged 8-bit cache, for timing and for comparing results.

Every request brings a tree of drafted tokens: node 0 is the last token of its text, every other node follows its parent, which stands
before it.  The nodes' K and V rows are in the cache already (its last tokens).  The calls around a model's layers are a kind of case each (`op`):
  masks     from the parents: which nodes each node follows, as a set of 64 bits, and its position in the text;
  attend    the nodes' queries over the kept tokens of the text (the first `sink` and the last `window`) and the nodes that they follow;
  verify    which drafted tokens stay, and the logarithm of each one's probability: from the target's logits, given random numbers and, where
            the drafts were drawn, their probabilities;
  keep      the rows of the nodes that stay move up in the caches of all layers, rounded again where a block's scale is another one;
  truncate  the requests lose the other nodes, and the pages that held nothing else go back on the pool's stack.

Pages hold 128 tokens in shuffled order.  Sink and window pairs and the lengths are those of `workloads/configs.py`; head counts, widths
and vocabularies are generic.
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 128
NODES = 64                      # most nodes of a tree
_MOST_CODES = 64 * 16384 * 8 * 128     # tokens x KV heads x head width of an `attend` pass: no case has more
_MOST_PRODUCTS = 64 * 64 * 8192 * 32 * 128  # queries x kept tokens x query heads x head width of one
_MOST_LOGITS = 1280 * 100003    # of a `verify` pass
_MOST_MOVED = 64 * 32 * 32 * 8 * 128   # nodes x layers x KV heads x head width of a `keep` pass
_MOST_REQUESTS = 1500


# ---------------------------------------------------------------------------------------------- cases

def _masks(batch, nodes, even, **kw):
    """even: every request brings `nodes` nodes; otherwise 1 to `nodes` of them."""
    return dict(kw, op="masks", batch=batch, nodes=nodes, even=even)


def _attend(batch, nodes, even, q_heads, kv_heads, head_dim, shortest, longest, sink, window, scale_tokens=64, out="bf16", **kw):
    """Lengths without the nodes."""
    return dict(kw, op="attend", batch=batch, nodes=nodes, even=even, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, shortest=shortest,
                longest=longest, sink=sink, window=window, scale_tokens=scale_tokens, out=out)


def _verify(batch, nodes, even, vocab, logits, drawn, greedy, **kw):
    """drawn: the drafts are a chain drawn from probabilities that are given; otherwise a tree of likely tokens.  greedy: one request in
    so many has temperature 0 (0: none)."""
    return dict(kw, op="verify", batch=batch, nodes=nodes, even=even, vocab=vocab, logits=logits, drawn=drawn, greedy=greedy)


def _keep(batch, nodes, even, layers, kv_heads, head_dim, scale_tokens, **kw):
    return dict(kw, op="keep", batch=batch, nodes=nodes, even=even, layers=layers, kv_heads=kv_heads, head_dim=head_dim, scale_tokens=scale_tokens)


def _truncate(batch, nodes, even, shortest, longest, **kw):
    return dict(kw, op="truncate", batch=batch, nodes=nodes, even=even, shortest=shortest, longest=longest)


def listed():
    return [
        # one chat with a small tree
        _masks(1, 8, True, name="masks_b1"),
        # a large offline batch with the largest trees
        _masks(1500, 64, False, name="masks_b1500"),
        # one chat with a small tree: launches and latency
        _attend(1, 8, True, 32, 8, 128, 300, 300, 0, 4096, name="attend_b1_short"),
        # a compressed layer (sink and window of the headline decode), wide heads, fp32 results
        _attend(48, 25, True, 16, 2, 256, 2048, 32768, 128, 2048, scale_tokens=128, out="fp32", name="attend_b48_window"),
        # an ordinary batch of ragged lengths and trees, nothing compressed
        _attend(64, 64, False, 32, 8, 128, 1000, 16000, 0, 20000, scale_tokens=32, name="attend_b64_ragged"),
        # one chat with a small tree
        _verify(1, 8, True, 32000, "bf16", False, 0, name="verify_b1_tree"),
        # chains of five drawn tokens, the probabilities that they were drawn from given
        _verify(64, 6, True, 131072, "bf16", True, 8, name="verify_b64_chain"),
        # larger trees; an odd vocabulary, logits in fp32
        _verify(32, 40, True, 100003, "fp32", False, 4, name="verify_b32_trees"),
        # one chat, a model of few layers
        _keep(1, 8, True, 4, 8, 128, 64, name="keep_b1"),
        # a batch with larger trees, a model of 32 layers
        _keep(64, 32, False, 32, 8, 128, 32, name="keep_b64"),
        _truncate(64, 8, True, 1024, 65536, name="truncate_b64"),
        _truncate(1500, 64, False, 1, 4096, name="truncate_b1500"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(["masks", "attend", "attend", "attend", "verify", "verify", "verify", "keep", "keep", "truncate"])
    nodes, even = _log_int(rng, 1, NODES), rng.random() < 0.5
    if op == "masks":
        return _masks(_log_int(rng, 1, _MOST_REQUESTS), nodes, even)
    if op == "truncate":
        longest = _log_int(rng, 1, 65536)
        return _truncate(_log_int(rng, 1, _MOST_REQUESTS), nodes, even, _log_int(rng, 1, longest), longest)
    if op == "attend":
        kv_heads = rng.choice([1, 2, 3, 4, 8, 8, 16])
        group = rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
        longest = _log_int(rng, 1, 65536)
        shortest = longest if rng.random() < 0.3 else _log_int(rng, 1, longest)
        sink, window = rng.choice([(0, longest + NODES), (0, longest + NODES), (128, 2048), (64, 512), (4, 1000), (4, 40), (128, 8192)])
        case = _attend(_log_int(rng, 1, 256), nodes, even, group * kv_heads, kv_heads, rng.choice([64, 128, 128, 256]), shortest, longest, sink, window,
                       scale_tokens=rng.choice([32, 64, 128]), out=rng.choice(["bf16", "bf16", "fp32"]))
    elif op == "verify":
        drawn = rng.random() < 0.5
        case = _verify(_log_int(rng, 1, 256), min(nodes, 16) if drawn else nodes, even, _log_int(rng, 200, 262144), rng.choice(["bf16", "bf16", "fp32"]), drawn,
                       rng.choice([0, 1, 2, 5]))
    else:
        case = _keep(_log_int(rng, 1, 256), max(nodes, 2), even, _log_int(rng, 1, 40), rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 128, 256]),
                     rng.choice([32, 64, 128]))
    while case["batch"] > 1:
        batch, nodes = case["batch"], case["nodes"]
        if op == "attend":
            # (what a pass reads, and what the padded plain form lays out)
            rows = min(case["longest"], case["sink"] + case["window"]) + nodes + 2 * PAGE
            if (batch * rows * case["kv_heads"] * case["head_dim"] <= _MOST_CODES and batch * case["longest"] * case["kv_heads"] * case["head_dim"] <= _MOST_CODES
                    and batch * nodes * rows * case["q_heads"] * case["head_dim"] <= _MOST_PRODUCTS):
                break
        elif op == "verify":
            if batch * nodes * case["vocab"] * (2 if case["drawn"] else 1) <= _MOST_LOGITS:
                break
        elif batch * max(nodes, 32) * case["layers"] * case["kv_heads"] * case["head_dim"] <= _MOST_MOVED:
            break
        case["batch"] = max(1, batch * 3 // 4)
    return case


def _plan(case):
    """Of each request: tokens of its text without the nodes, the nodes' parents, and which nodes stay (for `keep` and `truncate`, where that is
    an input).  A matter of the case and not of the seed: the work is the same for every seed."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    texts, trees, kept = [], [], []
    lo, hi = case.get("shortest", 1), case.get("longest", 1000)
    for _ in range(case["batch"]):
        n = case["nodes"] if case["even"] else _log_int(rng, 1, case["nodes"])
        texts.append(hi if lo == hi else _log_int(rng, lo, hi))
        chain = case.get("drawn", False)
        # (a node follows one of the nodes that came last, rarely an earlier one: deep and wide parts)
        tree = [-1] + [t - 1 if chain else rng.choice([t - 1, rng.randrange(max(0, t - 4), t), rng.randrange(t)]) for t in range(1, n)]
        trees.append(tree)
        t, path = rng.randrange(n), []
        while t >= 0:
            path.append(t)
            t = tree[t]
        kept.append(path[::-1])
    return texts, trees, kept


def _pages(n):
    return -(-n // PAGE)


# ---------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(counts):
    return _ints([0] + list(np.cumsum(counts)))


def _masks_of(tree):
    masks = []
    for t, parent in enumerate(tree):
        masks.append((masks[parent] if parent >= 0 else 0) | 1 << t)
    return masks


def _pool(lead, kv_heads, head_dim, scale_tokens, gen):
    """Pages as a program has them after it has served for a while: every slot holds codes of some token, each block its scale.  K rows have a
    few channels that stand out."""
    codes = [torch.empty(lead + (kv_heads, PAGE, head_dim), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
    scales = [torch.empty(lead + (kv_heads, PAGE // scale_tokens), dtype=torch.float32, device="cuda") for _ in range(2)]
    step = max(1, (1 << 28) // (kv_heads * PAGE * head_dim))
    for which, spread in ((0, 3.0), (1, 0.0)):
        flat, flat_scales = codes[which].view(-1, kv_heads, PAGE, head_dim), scales[which].view(-1, kv_heads, PAGE // scale_tokens)
        for a in range(0, flat.shape[0], step):
            some = min(step, flat.shape[0] - a)
            x = torch.randn((some, kv_heads, PAGE, head_dim), device="cuda", generator=gen)
            x *= 1 + spread * (torch.rand(head_dim, device="cuda", generator=gen) > 0.95)
            x = x.view(some, kv_heads, PAGE // scale_tokens, scale_tokens * head_dim)
            # blocks of other sizes beside each other, so that a row that changes blocks is rounded again
            x *= torch.exp2(torch.randint(-2, 3, x.shape[:3], device="cuda", generator=gen).float())[..., None]
            part, exponent = torch.frexp(x.abs().amax(-1))
            s = torch.ldexp(torch.ones_like(part), exponent - 9 + (part > 0.875).int())
            flat[a:a + some] = (x / s[..., None]).to(torch.float8_e4m3fn).view(some, kv_heads, PAGE, head_dim)
            flat_scales[a:a + some] = s
    return codes + scales


def _table(used, order):
    width = max(used)
    column = torch.arange(width, device="cuda")[None]
    table = torch.where(column < _ints(used)[:, None], order[(_starts(used)[:-1, None] + column).clamp(max=order.numel() - 1)], 0)
    return table.int().contiguous()


def prepare(case, seed):
    gen = _generator(seed)
    op, batch = case["op"], case["batch"]
    texts, trees, kept = _plan(case)
    news = [len(t) for t in trees]
    tokens = sum(news)
    lens = [a + b for a, b in zip(texts, news)]
    start = _starts(news)
    if op == "masks":
        # another seed: other texts
        L = _ints(lens) + torch.randint(0, 5000, (batch,), device="cuda", generator=gen).int()
        return dict(op=op, parents=_ints([p for t in trees for p in t]), seq_lens=L, q_start=start,
                    masks=torch.empty(tokens, dtype=torch.int64, device="cuda"), positions=torch.empty(tokens, dtype=torch.int32, device="cuda"))
    if op == "truncate":
        used = [_pages(n) for n in lens]
        order = torch.randperm(sum(used) + 100, device="cuda", generator=gen).int()
        stack = torch.full((order.numel(),), -1, dtype=torch.int32, device="cuda")
        stack[:100] = order[sum(used):]
        return dict(op=op, seq_lens=_ints(lens), dropped=_ints([n - len(k) for n, k in zip(news, kept)]), page_table=_table(used, order), free_pages=stack,
                    free_count=_ints([100]), seq_lens_out=torch.empty(batch, dtype=torch.int32, device="cuda"), free_count_out=_ints([0]))
    if op == "verify":
        return dict(_logits(case, trees, gen), op=op, q_start=start, batch=batch, most=max(news), path=torch.empty(tokens, dtype=torch.int32, device="cuda"),
                    out_tokens=torch.empty(tokens, dtype=torch.int32, device="cuda"), logprobs=torch.empty(tokens, device="cuda"), dropped=torch.empty(batch, dtype=torch.int32, device="cuda"))
    kv_heads, head_dim, scale_tokens = case["kv_heads"], case["head_dim"], case["scale_tokens"]
    if op == "keep":
        # (only the pages that nodes lie in are there)
        inside = [a % PAGE for a in texts]
        lens = [a + b for a, b in zip(inside, news)]
        used = [_pages(n) for n in lens]
        order = torch.randperm(sum(used), device="cuda", generator=gen).int()
        k, v, ks, vs = _pool((case["layers"], sum(used)), kv_heads, head_dim, scale_tokens, gen)
        path = [p for n, way in zip(news, kept) for p in way + [-1] * (n - len(way))]
        return dict(op=op, path=_ints(path), seq_lens=_ints(lens), q_start=start, page_table=_table(used, order), k_cache=k, v_cache=v, k_scales=ks, v_scales=vs)
    used = [_pages(n) for n in lens]
    order = torch.randperm(sum(used), device="cuda", generator=gen).int()
    k, v, ks, vs = _pool((sum(used),), kv_heads, head_dim, scale_tokens, gen)
    q = torch.randn((tokens, case["q_heads"], head_dim), device="cuda", generator=gen).bfloat16()
    masks = [m - (1 << 64) if m >> 63 else m for t in trees for m in _masks_of(t)]
    dtype = torch.float32 if case["out"] == "fp32" else torch.bfloat16
    return dict(op=op, q=q, k_cache=k, v_cache=v, k_scales=ks, v_scales=vs, page_table=_table(used, order), seq_lens=_ints(lens), q_start=start,
                masks=torch.tensor(masks, dtype=torch.int64, device="cuda"), most=max(news), sink=case["sink"], window=case["window"], softmax_scale=head_dim ** -0.5,
                out=torch.empty(q.shape, dtype=dtype, device="cuda"), lse=torch.empty(q.shape[:2], dtype=torch.float32, device="cuda"))


def _logits(case, trees, gen):
    """The target's logits: most tokens unlikely, some that stand out.  Drafts: drawn from a distribution near the target's, or the
    tokens that a model near it holds most likely, an own one for each child of a node."""
    vocab, tokens, batch = case["vocab"], sum(len(t) for t in trees), case["batch"]
    dtype = torch.bfloat16 if case["logits"] == "bf16" else torch.float32
    temperature = 0.5 + 0.75 * torch.rand(batch, device="cuda", generator=gen)
    if case["greedy"]:
        temperature[torch.arange(batch, device="cuda") % case["greedy"] == 0] = 0.0
    uniforms = torch.rand((tokens, 2), device="cuda", generator=gen)
    logits = torch.empty((tokens, vocab), dtype=dtype, device="cuda")
    probs = torch.empty((tokens, vocab), dtype=torch.float32, device="cuda") if case["drawn"] else None
    drafts = torch.zeros(tokens, dtype=torch.int64, device="cuda")
    request = [b for b, t in enumerate(trees) for _ in t]
    begin = np.cumsum([0] + [len(t) for t in trees])
    # of each node: its parent among all nodes, and how many of the parent's children come before it
    parent, before = [], []
    for b, tree in enumerate(trees):
        seen = {}
        for p in tree:
            parent.append(p + int(begin[b]) if p >= 0 else -1)
            before.append(seen.get(p, 0))
            seen[p] = before[-1] + 1
    widest = max(before) + 1
    child, of, rank = (torch.tensor(x, dtype=torch.int64, device="cuda") for x in ([i for i, p in enumerate(parent) if p >= 0],
                       [p for p in parent if p >= 0], [before[i] for i, p in enumerate(parent) if p >= 0]))
    step = max(1, (1 << 27) // vocab)
    for a in range(0, tokens, step):
        some = min(step, tokens - a)
        x = 2.0 * torch.randn((some, vocab), device="cuda", generator=gen)
        x.scatter_add_(1, torch.randint(0, vocab, (some, 6), device="cuda", generator=gen), 6.0 + 8.0 * torch.rand((some, 6), device="cuda", generator=gen))
        x = x.to(dtype)
        logits[a:a + some] = x
        near = x.float() + 0.7 * torch.randn((some, vocab), device="cuda", generator=gen)
        mine = (of >= a) & (of < a + some)
        if case["drawn"]:
            t = temperature[torch.tensor(request[a:a + some], device="cuda")].clamp(min=0.2)
            probs[a:a + some] = torch.softmax(near / t[:, None], -1)
            token = torch.multinomial(probs[a:a + some], 1, generator=gen)[:, 0]
            drafts[child[mine]] = token[of[mine] - a]
        else:
            drafts[child[mine]] = near.topk(min(widest, vocab), dim=-1).indices[of[mine] - a, rank[mine].clamp(max=vocab - 1)]
    return dict(logits=logits, draft_probs=probs, tokens=drafts.int(), parents=_ints([p for t in trees for p in t]), temperature=temperature, uniforms=uniforms)


# ---------------------------------------------------------------------------------------------- plain forms

def _requests(start, tokens):
    """Of each of the call's tokens: its request, and its number among the request's."""
    token = torch.arange(tokens, device=start.device)
    request = torch.searchsorted(start[1:].contiguous(), token, right=True)
    return request, token - start[request]


def _masks_plain(s):
    parents, start = s["parents"].long(), s["q_start"].long()
    request, mine = _requests(start, parents.numel())
    token = torch.arange(parents.numel(), device=parents.device)
    masks = torch.ones_like(parents) << mine
    # every pass doubles the way that the sets reach up
    up = torch.where(parents >= 0, start[request] + parents, token)
    for _ in range(6):
        masks, up = masks | masks[up], up[up]
    bits = (masks[:, None] >> torch.arange(NODES, device=parents.device)) & 1
    n = start[1:] - start[:-1]
    return {"masks": masks, "positions": ((s["seq_lens"] - n)[request] + bits.sum(1) - 1).int()}


def _attend_plain(s):
    q, table, L, start, sink, window, most = s["q"], s["page_table"].long(), s["seq_lens"].long(), s["q_start"].long(), s["sink"], s["window"], s["most"]
    batch, width = table.shape
    _, heads, _, dim = s["k_cache"].shape
    group = q.shape[1] // heads
    count = start[1:] - start[:-1]
    text = L - count
    # the pages that hold kept tokens of any of a request's queries
    first = ((text + 1 - window).clamp(min=0) // PAGE)[:, None]
    front = _pages(sink)
    column = torch.arange(min(width, front + _pages(window + most) + 1), device=q.device)[None]
    page = torch.where(column < front, column, torch.maximum(first, torch.full_like(first, front)) + column - front)
    place = (page[..., None] * PAGE + torch.arange(PAGE, device=q.device)).view(batch, 1, -1)     # [batch, 1, tokens]
    page = table.gather(1, page.clamp(max=width - 1))
    # queries padded to the largest number; the nodes that each follows, and their positions in the text
    t = torch.arange(most, device=q.device)[None]
    row = (start[:-1, None] + t).clamp(max=q.shape[0] - 1)
    node = torch.arange(NODES, device=q.device)
    follows = (((s["masks"][row][..., None] >> node) & 1) > 0) & (node < count[:, None, None])     # [batch, queries, nodes]
    depth = follows.long().cumsum(-1) - 1
    reach = (text[:, None] + follows.sum(-1))[..., None]                                           # tokens up to the query and with it
    at = text[:, None, None] + depth
    follows &= (at < sink) | (at >= reach - window)
    kept = (place < text[:, None, None]) & ((place < sink) | (place >= reach - window))            # [batch, queries, tokens]
    number = (place - text[:, None, None]).expand(-1, most, -1)
    kept |= (number >= 0) & (number < NODES) & follows.gather(2, number.clamp(0, NODES - 1))
    kept &= (t < count[:, None])[..., None]
    def laid_out(cache, scales):
        x = cache.view(torch.uint8)[page].view(cache.dtype).float() * scales[page].repeat_interleave(PAGE // scales.shape[2], 3)[..., None]
        return x.transpose(1, 2).reshape(batch, heads, -1, dim)                                   # [batch, heads, tokens, dim]
    x = q[row].float().view(batch, most, heads, group, dim).transpose(1, 2).reshape(batch, heads, most * group, dim)
    logits = torch.matmul(x, laid_out(s["k_cache"], s["k_scales"]).transpose(2, 3)) * s["softmax_scale"]
    mask = kept[:, None, :, None].expand(-1, -1, -1, group, -1).reshape(batch, 1, most * group, -1)
    logits = torch.where(mask, logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    weights = torch.exp(logits - torch.where(top.isinf(), 0.0, top))
    total = weights.sum(-1, keepdim=True)
    values = torch.where(kept.any(1)[:, None, :, None], laid_out(s["v_cache"], s["v_scales"]), 0.0)
    out = torch.matmul(weights, values) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total))[..., 0]
    # back to one row per query token
    request, mine = _requests(start, q.shape[0])
    out = out.view(batch, heads, most, group, dim)[request, :, mine].reshape(q.shape)
    lse = lse.view(batch, heads, most, group)[request, :, mine].reshape(q.shape[:2])
    return {"out": out.to(s["out"].dtype), "lse": lse}


def _verify_plain(s):
    # (in 64 bits: a sum that is off by a little makes another token of a random number next to a border)
    logits, tokens, parents, start = s["logits"].double(), s["tokens"].long(), s["parents"].long(), s["q_start"].long()
    nodes, vocab = logits.shape
    request, mine = _requests(start, nodes)
    T = s["temperature"].double()[request][:, None]
    greedy = ~(T > 0)[:, 0]
    top = logits.amax(1, keepdim=True)
    index = torch.arange(vocab, device=logits.device)
    best = torch.where(logits == top, index, vocab).amin(1)
    # (a request that takes the likeliest token: probabilities at temperature 1)
    scaled = (logits - top) / torch.where(T > 0, T, 1.0)
    del logits
    p = torch.exp(scaled)
    total = p.sum(1, keepdim=True)
    p /= total
    # children: the first of each node
    parent = torch.where(parents >= 0, start[request] + parents, nodes)
    node = torch.arange(nodes, device=p.device)
    child = torch.full((nodes + 1,), nodes, device=p.device).scatter_reduce(0, parent, node, "amin")[:nodes]
    accepted = torch.zeros(nodes, dtype=torch.bool, device=p.device)
    if s["draft_probs"] is not None:
        q = s["draft_probs"].double()
        has = (child < nodes) & ~greedy
        drafted = tokens[child.clamp(max=nodes - 1)]
        u = s["uniforms"][:, 0].double()
        accepted = has & (u * q.gather(1, drafted[:, None])[:, 0] < p.gather(1, drafted[:, None])[:, 0])
        rest = (p - q).clamp(min=0)
        del q
        p = torch.where((has & ~accepted & (rest.sum(1) > 0))[:, None], rest, p)
        del rest
    sums = p.cumsum(1)
    del p
    border = s["uniforms"][:, 1].double() * sums[:, -1]
    drawn = torch.searchsorted(sums, border[:, None], right=True)[:, 0].clamp(max=vocab - 1)
    del sums
    token = torch.where(greedy, best, drawn)
    # the first child that holds the token
    match = torch.where((parent < nodes) & (token[parent.clamp(max=nodes - 1)] == tokens), parent, nodes)
    following = torch.full((nodes + 1,), nodes, device=token.device).scatter_reduce(0, match, node, "amin")[:nodes]
    following = torch.where(accepted, child, following)
    token = torch.where(accepted, tokens[child.clamp(max=nodes - 1)], token)
    logprob = (scaled.gather(1, token[:, None]) - torch.log(total))[:, 0]
    # down the tree
    path, out = torch.full((nodes + 1,), -1, device=token.device), torch.full((nodes + 1,), -1, device=token.device)
    said = torch.zeros(nodes + 1, dtype=torch.float64, device=token.device)
    at, length = start[:-1].clone(), torch.zeros_like(start[:-1])
    for step in range(s["most"]):
        alive = at < nodes
        here = at.clamp(max=nodes - 1)
        slot = torch.where(alive, start[:-1] + step, nodes)
        path[slot], out[slot], said[slot] = here - start[:-1], token[here], logprob[here]
        length += alive
        at = torch.where(alive, following[here], nodes)
    return {"path": path[:nodes].int(), "out_tokens": out[:nodes].int(), "logprobs": said[:nodes].float(), "dropped": (start[1:] - start[:-1] - length).int()}


def _keep_one(cache, scales, page, place, to_page, to_place, base):
    """One cache of all layers: row `place` of page `page` goes to row `to_place` of `to_page`.  base: the first node's row counted from the
    page that the row goes to."""
    layers, pages, heads, _, dim = cache.shape
    blocks = scales.shape[3]
    each = PAGE // blocks
    flat = scales.transpose(2, 3).reshape(layers, pages * blocks, heads)
    block, to_block = page * blocks + place // each, to_page * blocks + to_place // each
    held = (base - to_place // each * each).clamp(0, each)                          # tokens of the text in the block that a row goes to
    largest = torch.zeros_like(flat).scatter_reduce(1, to_block[None, :, None].expand(layers, -1, heads), flat[:, block], "amax")
    touched = torch.zeros(pages * blocks, dtype=torch.long, device=cache.device).scatter_reduce(0, to_block, held + 1, "amax")[None, :, None]
    scale = torch.where(touched == 0, flat, torch.where(touched > 1, torch.maximum(flat, largest), largest))
    rows = cache.view(torch.uint8)[:, page, :, place].view(cache.dtype)             # [rows, layers, heads, dim]
    rows = rows.float() * _ratio(flat[:, block], scale[:, to_block]).transpose(0, 1)[..., None]
    # text tokens of a block whose scale has grown
    text = (torch.arange(each, device=cache.device) < touched.view(1, pages, 1, blocks, 1) - 1)[..., None]
    ratio = _ratio(flat, scale).reshape(layers, pages, blocks, heads).transpose(2, 3)[..., None, None]
    codes = cache.view(layers, pages, heads, blocks, each, dim)
    for i in range(layers):
        grown = torch.where(text[0] & (ratio[i] < 1), codes[i].float() * ratio[i], codes[i].float())
        cache[i] = grown.to(cache.dtype).reshape(cache.shape[1:])
    scales.copy_(scale.reshape(layers, pages, blocks, heads).transpose(2, 3))
    cache.view(torch.uint8)[:, to_page, :, to_place] = rows.to(cache.dtype).view(torch.uint8)


def _ratio(old, new):
    return torch.where(new > 0, old / torch.where(new > 0, new, 1.0), 1.0)


def _keep_plain(s):
    start, path, table = s["q_start"].long(), s["path"].long(), s["page_table"].long()
    request, mine = _requests(start, path.numel())
    text = (s["seq_lens"].long() - (start[1:] - start[:-1]))[request]
    stays = path >= 0
    # (rows that go nowhere: those that stay where they are take part, all others are a copy of the first)
    old, new = text + torch.where(stays, path, 0), text + torch.where(stays, mine, 0)
    page, to_page = table[request, old // PAGE], table[request, new // PAGE]
    for cache, scales in (("k_cache", "k_scales"), ("v_cache", "v_scales")):
        _keep_one(s[cache], s[scales], page, old % PAGE, to_page, new % PAGE, text - new // PAGE * PAGE)
    return {name: s[name] for name in ("k_cache", "v_cache", "k_scales", "v_scales")}


def _truncate_plain(s):
    L, table, stack, count = s["seq_lens"].long(), s["page_table"], s["free_pages"], s["free_count"].long()
    after = L - s["dropped"].long().clamp(min=0)
    after = after.clamp(min=0)
    had, has = (L + PAGE - 1) // PAGE, (after + PAGE - 1) // PAGE
    sums = torch.cumsum(had - has, 0)
    column = torch.arange(table.shape[1], device=table.device)[None]
    at = count + (sums - (had - has))[:, None] + column - has[:, None]
    back = (column >= has[:, None]) & (column < had[:, None])
    more = torch.cat([stack, stack[:1]])
    more[torch.where(back, at, stack.numel()).reshape(-1)] = table.reshape(-1)
    stack.copy_(more[:-1])
    return {"seq_lens": after.int(), "free_pages": stack, "free_count": (count + sums[-1]).int()}


# ---------------------------------------------------------------------------------------------- passes

def run(s):
    if not own:
        return {"masks": _masks_plain, "attend": _attend_plain, "verify": _verify_plain, "keep": _keep_plain, "truncate": _truncate_plain}[s["op"]](s)
    import paper_2511_22481_amd as oa
    if s["op"] == "masks":
        oa.omniattn_tree_masks(s["parents"], s["seq_lens"], s["q_start"], s["masks"], s["positions"])
        return {"masks": s["masks"], "positions": s["positions"]}
    if s["op"] == "verify":
        if "workspace" not in s:  # a serving loop keeps it
            size = oa.omniattn_tree_verify_workspace_bytes(num_tokens=s["logits"].shape[0], vocab=s["logits"].shape[1])
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        oa.omniattn_tree_verify(s["logits"], s["draft_probs"], s["tokens"], s["parents"], s["q_start"], s["temperature"], s["uniforms"], s["path"],
                                s["out_tokens"], s["logprobs"], s["dropped"], s["workspace"])
        return {"path": s["path"], "out_tokens": s["out_tokens"], "logprobs": s["logprobs"], "dropped": s["dropped"]}
    if s["op"] == "keep":
        oa.omniattn_gqa_keep(s["path"], s["seq_lens"], s["q_start"], s["page_table"], s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"])
        return {name: s[name] for name in ("k_cache", "v_cache", "k_scales", "v_scales")}
    if s["op"] == "truncate":
        oa.omniattn_table_truncate(s["seq_lens"], s["dropped"], s["page_table"], s["free_pages"], s["free_count"], s["seq_lens_out"], s["free_count_out"])
        return {"seq_lens": s["seq_lens_out"], "free_pages": s["free_pages"], "free_count": s["free_count_out"]}
    if "workspace" not in s:
        size = oa.omniattn_gqa_workspace_bytes(batch=s["seq_lens"].shape[0], num_queries=s["q"].shape[0], num_q_heads=s["q"].shape[1],
                                               num_kv_heads=s["k_cache"].shape[1], head_dim=s["q"].shape[2])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    oa.omniattn_gqa_tree(s["q"], s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"], s["page_table"], s["seq_lens"], s["q_start"], s["masks"],
                         s["out"], s["lse"], s["workspace"], sink=s["sink"], window=s["window"], softmax_scale=s["softmax_scale"])
    return {"out": s["out"], "lse": s["lse"]}


def _kept(case, text, positions):
    """Tokens that a node's query keeps: of the text, and of the nodes that it follows (their positions)."""
    reach = positions[-1] + 1
    low = max(reach - case["window"], case["sink"], 0)
    return min(text, case["sink"]) + max(0, text - low) + sum(p < case["sink"] or p >= reach - case["window"] for p in positions)


def work(case):
    texts, trees, kept = _plan(case)
    batch, tokens = case["batch"], sum(len(t) for t in trees)
    if case["op"] == "masks":
        return {"bytes": 4 * tokens + 4 * (2 * batch + 1) + 12 * tokens, "flops": 0}
    if case["op"] == "truncate":
        back = sum(_pages(a + len(t)) - _pages(a + len(k)) for a, t, k in zip(texts, trees, kept))
        return {"bytes": 4 * (3 * batch + 2 + 2 * back), "flops": 0}
    if case["op"] == "verify":
        # every node's logits (which of them count is not known before); of the drafts' probabilities those of the drafted tokens
        size = 2 if case["logits"] == "bf16" else 4
        return {"bytes": tokens * (case["vocab"] * size + 8 + 8 + 12) + batch * 12 + 4 + (4 * tokens if case["drawn"] else 0), "flops": 4 * tokens * case["vocab"]}
    heads, dim, each = case["kv_heads"], case["head_dim"], case["scale_tokens"]
    if case["op"] == "keep":
        moved, blocks = 0, 0
        for a, way in zip(texts, kept):
            a %= PAGE
            moved += sum(p != i for i, p in enumerate(way))
            blocks += len({(a + i) // each for i, p in enumerate(way) if p != i} | {(a + p) // each for i, p in enumerate(way) if p != i})
        return {"bytes": 2 * case["layers"] * heads * (2 * moved * dim + 8 * blocks) + 4 * (tokens + 2 * batch), "flops": 0}
    read, products = 0, 0
    for text, tree in zip(texts, trees):
        depth = [m.bit_count() for m in _masks_of(tree)]
        union = text + len(tree) - max(0, text + 1 - case["window"] - case["sink"])
        read += union * heads * 2 * dim + -(-union // each) * heads * 8 + 4 * _pages(union)
        products += sum(_kept(case, text, range(text, text + d)) for d in depth) * case["q_heads"] * dim * 4
    width = 4 if case["out"] == "fp32" else 2
    return {"bytes": read + tokens * (case["q_heads"] * (dim * (2 + width) + 4) + 8) + 4 * (2 * batch + 1), "flops": products}


# ---------------------------------------------------------------------------------------------- in 64 bits

def _e4m3(x):
    """Numbers (64 bits, within 448) rounded to the nearest that e4m3 holds, ties to even."""
    exponent = np.maximum(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -20))), -6)
    step = 2.0 ** (exponent - 3)
    return np.rint(x / step) * step


def _exact_verify(case, s, trees):
    path, out, logprobs, dropped, first = [], [], [], [], 0
    tokens, uniforms, temperature = s["tokens"].tolist(), s["uniforms"].double().cpu().numpy(), s["temperature"].double().tolist()
    for tree, T in zip(trees, temperature):
        way, said, chances, at = [], [], [], 0
        while at is not None:
            row = s["logits"][first + at].double().cpu().numpy()
            children = [c for c in range(len(tree)) if tree[c] == at]
            u0, u1 = uniforms[first + at]
            p = np.exp((row - row.max()) / (T or 1.0))
            total = p.sum()
            p /= total
            if T == 0:
                token = int(row.argmax())
            else:
                rest, token = p, None
                if case["drawn"] and children:
                    q = s["draft_probs"][first + at].double().cpu().numpy()
                    x = tokens[first + children[0]]
                    if u0 * q[x] < p[x]:
                        token = x
                    elif np.maximum(p - q, 0).sum() > 0:
                        rest = np.maximum(p - q, 0)
                if token is None:
                    sums = np.cumsum(rest)
                    token = int(np.searchsorted(sums, u1 * sums[-1], side="right"))
            way.append(at)
            said.append(token)
            chances.append((row[token] - row.max()) / (T or 1.0) - math.log(total))
            at = next((c for c in children if tokens[first + c] == token), None)
        n = len(tree)
        path += way + [-1] * (n - len(way))
        out += said + [-1] * (n - len(way))
        logprobs += chances + [0.0] * (n - len(way))
        dropped.append(n - len(way))
        first += n
    return {"path": torch.tensor(path, dtype=torch.int32), "out_tokens": torch.tensor(out, dtype=torch.int32),
            "logprobs": torch.tensor(logprobs, dtype=torch.float64), "dropped": torch.tensor(dropped, dtype=torch.int32)}


def _exact_keep(case, s, texts, trees, kept):
    result, table = {}, s["page_table"].tolist()
    each = case["scale_tokens"]
    for name in ("k", "v"):
        # (a slice of layers at a time would say no more: heads and layers are alike)
        codes = s[name + "_cache"].float().cpu().numpy().astype(np.float64)
        scales = s[name + "_scales"].cpu().numpy().astype(np.float64)
        for b, (text, way) in enumerate(zip(texts, kept)):
            text %= PAGE
            def slot(at):
                return table[b][at // PAGE], at % PAGE
            rows = [(codes[:, slot(text + p)[0], :, slot(text + p)[1]].copy(), scales[:, slot(text + p)[0], :, slot(text + p)[1] // each].copy()) for p in way]
            for block in sorted({(text + i) // each for i in range(len(way))}):
                page, low = slot(block * each)
                mine = [i for i in range(len(way)) if (text + i) // each == block]
                held = max(0, text - block * each)
                old = scales[:, page, :, low // each].copy()
                new = np.max([rows[i][1] for i in mine] + ([old] if held else []), axis=0)
                some = np.where(new > 0, new, 1)
                codes[:, page, :, low:low + held] = _e4m3(codes[:, page, :, low:low + held] * np.where(new > 0, old / some, 1)[..., None, None])
                for i in mine:
                    codes[:, page, :, slot(text + i)[1]] = _e4m3(rows[i][0] * np.where(new > 0, rows[i][1] / some, 1)[..., None])
                scales[:, page, :, low // each] = new
        result[name + "_cache"], result[name + "_scales"] = torch.from_numpy(codes), torch.from_numpy(scales)
    return {name: result[name] for name in ("k_cache", "v_cache", "k_scales", "v_scales")}


def exact(case, seed):
    if case["op"] in ("masks", "truncate"):
        return None  # whole numbers
    texts, trees, kept = _plan(case)
    if case["op"] == "keep":
        if sum(_pages(a % PAGE + len(t)) for a, t in zip(texts, trees)) * case["layers"] * case["kv_heads"] * case["head_dim"] * PAGE > 1 << 27:
            return None
        return _exact_keep(case, prepare(case, seed), texts, trees, kept)
    s = prepare(case, seed)
    if case["op"] == "verify":
        return _exact_verify(case, s, trees)
    heads, dim, each = case["kv_heads"], case["head_dim"], case["scale_tokens"]
    group = case["q_heads"] // heads
    outs, lses, at = [], [], 0
    for b, (text, tree) in enumerate(zip(texts, trees)):
        new = len(tree)
        pages = s["page_table"][b].long()
        mask = torch.zeros((new, text + new), dtype=torch.bool)
        for t, m in enumerate(_masks_of(tree)):
            follows = [a for a in range(new) if m >> a & 1]
            reach = text + len(follows)
            mask[t, max(0, reach - case["window"]):text] = True
            mask[t, :min(text, case["sink"])] = True
            for depth, a in enumerate(follows):
                mask[t, text + a] = text + depth < case["sink"] or text + depth >= reach - case["window"]
        mask = mask.cuda()
        some = mask.any(0).nonzero()[:, 0]
        def rows(cache, scales):
            page, off = pages[some // PAGE], some % PAGE
            return (cache.view(torch.uint8)[page, :, off].view(torch.float8_e4m3fn).double() * scales.double()[page, :, off // each][..., None]).transpose(0, 1)
        k, v = rows(s["k_cache"], s["k_scales"]), rows(s["v_cache"], s["v_scales"])        # [heads, kept, dim]
        x = s["q"][at:at + new].double().view(new, heads, group, dim).permute(1, 0, 2, 3).reshape(heads, new * group, dim)
        # (the softmax scale is an argument of 32 bits)
        logits = torch.bmm(x, k.transpose(1, 2).contiguous()) * float(np.float32(s["softmax_scale"]))
        logits = logits.masked_fill(~mask[:, some].repeat_interleave(group, 0)[None], -math.inf)
        lse = torch.logsumexp(logits, -1)
        out = torch.bmm(torch.exp(logits - lse[..., None]).nan_to_num(0.0), v.contiguous())
        outs.append(out.view(heads, new, group, dim).permute(1, 0, 2, 3).reshape(new, heads * group, dim))
        lses.append(lse.view(heads, new, group).permute(1, 0, 2).reshape(new, heads * group))
        at += new
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
