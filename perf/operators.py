"""Serving work on layers with grouped-query attention over a paged cache held in 8 bits, for timing and for
comparing results.

A decode or verification step of such a layer takes three calls, and each is a kind of case here (`op`):
  extend   the step's block table and slot map, on the GPU: every request grows by its new tokens, takes the
           pages that it needs from the pool's stack of free pages, and each new token learns its slot;
  append   the new tokens' K and V rows go to their slots as e4m3 codes.  A block of `scale_tokens` tokens of a
           KV head shares one scale, a power of two, which may grow with a block's later tokens;
  attend   the new tokens' queries against the cache through the table, causal, over the kept tokens (the
           first `sink` and the last `window`; a window no shorter than the request keeps all of them).

Pages hold 128 tokens in shuffled order.  Sink and window pairs and the lengths are those of `workloads/configs.py`
and of the layers that the pattern search leaves uncompressed; head counts and widths are the usual ones of
grouped-query layers.
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 128
_MOST_CODES = 64 * 32768 * 8 * 128   # kept tokens x KV heads x head width of an `attend` pass: no case has more
_MOST_TOKENS = 65536                 # new tokens of an `append` or `extend` pass


# ---------------------------------------------------------------------------------------------- cases

def _extend(batch, shortest, longest, new, busy, **kw):
    """busy: one request in so many brings a chunk of up to `new` tokens, the others one token (1: all bring chunks)."""
    return dict(kw, op="extend", batch=batch, shortest=shortest, longest=longest, new=new, busy=busy)


def _append(batch, new, busy, kv_heads, head_dim, scale_tokens, **kw):
    return dict(kw, op="append", batch=batch, new=new, busy=busy, kv_heads=kv_heads, head_dim=head_dim, scale_tokens=scale_tokens)


def _attend(batch, q_heads, kv_heads, head_dim, shortest, longest, sink, window, new=1, busy=1, scale_tokens=64, out="bf16", **kw):
    return dict(kw, op="attend", batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, shortest=shortest,
                longest=longest, sink=sink, window=window, new=new, busy=busy, scale_tokens=scale_tokens, out=out)


def listed():
    return [
        # a decode step's tables: every request brings one token, some of them open a page
        _extend(64, 1024, 65536, 1, 1, name="extend_b64_decode"),
        # decode steps with chunks of prompts among them
        _extend(256, 1, 32768, 512, 8, name="extend_b256_mixed"),
        # prompts of a large offline batch, all at once
        _extend(1500, 1, 4096, 64, 1, name="extend_b1500_prompts"),
        # one token of each of 64 requests
        _append(64, 1, 1, 8, 128, 64, name="append_b64_decode"),
        # chunks of prompts beside decoding requests; one head fewer than a power of two
        _append(133, 700, 16, 7, 128, 32, name="append_b133_mixed"),
        # prompts: as many tokens as a prefill step takes
        _append(32, 2048, 1, 8, 128, 128, name="append_b32_prompts"),
        # one short interactive request: launches and latency
        _attend(1, 32, 8, 128, 77, 77, 0, 128, name="attend_b1_short"),
        # one long document: its cache has to be split over the whole GPU
        _attend(1, 32, 8, 128, 131072, 131072, 0, 131072, name="attend_b1_128k"),
        # an ordinary batch of ragged lengths
        _attend(93, 28, 4, 128, 200, 20000, 0, 20000, scale_tokens=32, name="attend_b93_ragged"),
        # a compressed layer (sink and window of the headline decode), draft tokens to verify, wide heads, fp32 results
        _attend(64, 16, 2, 256, 2048, 32768, 128, 2048, new=5, scale_tokens=128, out="fp32", name="attend_b64_verify"),
        # many short chats on a layer without grouping, narrow heads
        _attend(256, 12, 12, 64, 1, 2000, 4, 1024, name="attend_b256_mha"),
        # an uncompressed layer of the headline batch
        _attend(64, 64, 8, 128, 32768, 32768, 0, 32768, name="attend_b64_32k"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(["extend", "append", "attend", "attend", "attend"])
    if op == "extend":
        case = _extend(_log_int(rng, 1, 1500), rng.choice([0, 1, 100]), _log_int(rng, 128, 65536), _log_int(rng, 1, 2048), rng.choice([1, 2, 8, 30]))
    elif op == "append":
        case = _append(_log_int(rng, 1, 256), _log_int(rng, 1, 2048), rng.choice([1, 1, 4, 16]), rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 128, 256]),
                       rng.choice([32, 64, 128]))
    else:
        kv_heads = rng.choice([1, 2, 3, 4, 8, 8, 16])
        group = rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
        longest = _log_int(rng, 16, 131072)
        shortest = longest if rng.random() < 0.3 else _log_int(rng, 1, longest)
        new = rng.choice([1, 1, 1, 2, 5, 16])
        sink, window = rng.choice([(0, longest), (0, longest), (128, 2048), (64, 512), (4, 1000), (128, 8192)])
        case = _attend(_log_int(rng, 1, 256), group * kv_heads, kv_heads, rng.choice([64, 128, 128, 256]), shortest, longest, sink, window, new=new,
                       busy=rng.choice([1, 3]), scale_tokens=rng.choice([32, 64, 128]), out=rng.choice(["bf16", "bf16", "fp32"]))
    while case["batch"] > 1:
        lens, news = _lengths(case)
        if op == "attend":
            # (what a pass reads, and what the padded plain form lays out)
            tokens = case["batch"] * min(case["longest"], case["sink"] + case["window"] + case["new"] + 2 * PAGE)
            if tokens * case["kv_heads"] * case["head_dim"] <= _MOST_CODES and sum(lens) * case["kv_heads"] * case["head_dim"] <= _MOST_CODES:
                break
        elif op == "append":
            if sum(news) * case["kv_heads"] * case["head_dim"] <= _MOST_TOKENS * 8 * 128:
                break
        elif sum(news) <= _MOST_TOKENS:
            break
        case["batch"] = max(1, case["batch"] * 3 // 4)
    return case


def _lengths(case):
    """Tokens of each request with its new ones, and how many of them are new.  A matter of the case and not of the seed: the
    work is the same for every seed."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    batch, new = case["batch"], case["new"]
    def chunk():
        if rng.randrange(case["busy"]):
            return 1
        if case["busy"] > 1 or case["op"] == "extend":
            return _log_int(rng, 1, new)
        return new if case["op"] == "attend" else rng.randint((new + 1) // 2, new)
    news = [chunk() for _ in range(batch)]
    if case["op"] == "append":
        lens = [rng.randrange(PAGE) + n for n in news]  # (only the pages that new tokens go to are there)
    else:
        lo, hi = case["shortest"], case["longest"]
        lens = [hi if lo == hi else round(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1)))) - 1 for _ in range(batch)]
        lens = [max(0, n) for n in lens] if case["op"] == "extend" else [max(1, n) for n in lens]
        if case["op"] == "extend":
            lens = [a + b for a, b in zip(lens, news)]
        else:
            news = [min(a, b) for a, b in zip(news, lens)]
    return lens, news


def _pages(n):
    return -(-n // PAGE)


def _kept(case, n):
    return min(n, case["sink"] + case["window"])


# ---------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(counts):
    return _ints([0] + list(np.cumsum(counts)))


def _rows(shape, gen, spread):
    """K or V rows: unit variance, some channels larger (K has a few that stand out), some tokens larger."""
    x = torch.randn(shape, device="cuda", generator=gen)
    x *= 1 + spread * (torch.rand(shape[-1], device="cuda", generator=gen) > 0.95)
    return x


def _pool(num_pages, kv_heads, head_dim, scale_tokens, gen):
    """Pages as a program has them after it has served for a while: every slot holds codes of some token, each block its scale."""
    codes = [torch.empty((num_pages, kv_heads, PAGE, head_dim), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
    scales = [torch.empty((num_pages, kv_heads, PAGE // scale_tokens), dtype=torch.float32, device="cuda") for _ in range(2)]
    step = max(1, (1 << 28) // (kv_heads * PAGE * head_dim))
    for which, spread in ((0, 3.0), (1, 0.0)):
        for a in range(0, num_pages, step):
            x = _rows((min(step, num_pages - a), kv_heads, PAGE // scale_tokens, scale_tokens * head_dim), gen, spread)
            s = _scale(x.abs().amax(-1))
            codes[which][a:a + step] = (x / s[..., None]).to(torch.float8_e4m3fn).view(x.shape[0], kv_heads, PAGE, head_dim)
            scales[which][a:a + step] = s
    return codes + scales


def prepare(case, seed):
    gen = _generator(seed)
    op, batch = case["op"], case["batch"]
    lens, news = _lengths(case)
    tokens = sum(news)
    if op == "extend":
        before = [a - b for a, b in zip(lens, news)]
        used, need = [_pages(n) for n in before], sum(_pages(a) - _pages(b) for a, b in zip(lens, before))
        order = torch.randperm(sum(used) + need + 100, device="cuda", generator=gen).int()
        width = max(_pages(n) for n in lens) + 1
        column = torch.arange(width, device="cuda")[None]
        first, many = _starts(used)[:-1, None], _ints(used)[:, None]
        table = torch.where(column < many, order[(first + column).clamp(max=order.numel() - 1)], -1).int()
        return dict(op=op, seq_lens=_ints(before), new_lens=_ints(news), free_pages=order[sum(used):].contiguous(), free_count=_ints([need + 100]),
                    page_table=table, seq_lens_out=torch.empty(batch, dtype=torch.int32, device="cuda"), free_count_out=_ints([0]),
                    q_start=torch.empty(batch + 1, dtype=torch.int32, device="cuda"), slot_map=torch.empty(tokens, dtype=torch.int32, device="cuda"))
    kv_heads, head_dim, scale_tokens = case["kv_heads"], case["head_dim"], case["scale_tokens"]
    used = [_pages(n) for n in lens]
    num_pages = sum(used)
    order = torch.randperm(num_pages, device="cuda", generator=gen).int()
    k, v, ks, vs = _pool(num_pages, kv_heads, head_dim, scale_tokens, gen)
    state = dict(op=op, k_cache=k, v_cache=v, k_scales=ks, v_scales=vs)
    start = _starts(news)
    if op == "append":
        token = torch.arange(tokens, device="cuda")
        request = torch.repeat_interleave(torch.arange(batch, device="cuda"), _ints(news), output_size=tokens)
        at = (_ints(lens) - _ints(news))[request] + token - start[request]
        slots = order[_starts(used)[request] + at // PAGE] * PAGE + at % PAGE
        # K and V as they leave a projection that computes queries, keys and values together
        fused = torch.empty((tokens, 3 * kv_heads, head_dim), dtype=torch.bfloat16, device="cuda")
        fused[:, kv_heads:2 * kv_heads] = _rows((tokens, kv_heads, head_dim), gen, 3.0)
        fused[:, 2 * kv_heads:] = _rows((tokens, kv_heads, head_dim), gen, 0.0)
        # some tokens stand out
        fused *= 1 + 7 * (torch.rand((tokens, 1, 1), device="cuda", generator=gen) > 0.98).bfloat16()
        return dict(state, k_new=fused[:, kv_heads:2 * kv_heads], v_new=fused[:, 2 * kv_heads:], slot_map=slots.int())
    q = torch.randn((tokens, case["q_heads"], head_dim), device="cuda", generator=gen).bfloat16()
    width = max(used)
    column = torch.arange(width, device="cuda")[None]
    table = torch.where(column < _ints(used)[:, None], order[(_starts(used)[:-1, None] + column).clamp(max=num_pages - 1)], 0).int()
    dtype = torch.float32 if case["out"] == "fp32" else torch.bfloat16
    return dict(state, q=q, page_table=table.contiguous(), seq_lens=_ints(lens), q_start=start, most_new=max(news), sink=case["sink"], window=case["window"],
                softmax_scale=head_dim ** -0.5, out=torch.empty(q.shape, dtype=dtype, device="cuda"),
                lse=torch.empty(q.shape[:2], dtype=torch.float32, device="cuda"))


# ---------------------------------------------------------------------------------------------- plain forms

def _scale(largest):
    """The smallest power of two by which a block whose largest magnitude this is fits e4m3 (448 = 7/8 of 2^9); 0 for a block of zeros."""
    part, exponent = torch.frexp(largest)
    exponent = (exponent - 9 + (part > 0.875).int()).clamp(min=-126)
    return torch.where(largest > 0, torch.ldexp(torch.ones_like(largest), exponent), 0.0)


def _extend_plain(s):
    L, n, table, most = s["seq_lens"].long(), s["new_lens"].long(), s["page_table"], s["slot_map"].numel()
    width, free, count = table.shape[1], s["free_pages"], s["free_count"].long()
    end = torch.cumsum(n.clamp(min=0), 0)
    start = end - n.clamp(min=0)
    had, has = (L + PAGE - 1) // PAGE, (L + n + PAGE - 1) // PAGE
    fine = (n >= 0) & (L >= 0) & (has <= width) & (end <= most)
    need = torch.where(fine, has - had, 0)
    sums = torch.cumsum(need, 0)
    fine &= (need == 0) | (sums <= count)
    need = torch.where(fine, need, 0)
    column = torch.arange(width, device=table.device)[None]
    at = count - 1 - (sums - need)[:, None] - (column - had[:, None])
    fresh = (column >= had[:, None]) & (column < (had + need)[:, None])
    table.copy_(torch.where(fresh, free[at.clamp(0, free.numel() - 1)], table))
    token = torch.arange(most, device=table.device)
    request = torch.searchsorted(end, token, right=True).clamp(max=L.numel() - 1)
    place = L[request] + token - start[request]
    page = table[request, (place // PAGE).clamp(0, width - 1)]
    slots = torch.where(fine[request] & (token < end[request]), page * PAGE + place % PAGE, -1)
    return {"page_table": table, "seq_lens": torch.where(fine, L + n, L).int(), "free_count": (count - need.sum()).int(),
            "q_start": torch.cat([start[:1], end]).int(), "slot_map": slots.int()}


def _append_one(new, slots, cache, scales):
    pages, heads, _, width = cache.shape
    blocks = scales.shape[2]
    each = PAGE // blocks
    x = new.float()
    size = x.abs()
    size = torch.where(size.isfinite(), size, 0.0).amax(-1)                      # [tokens, heads]
    slots = slots.long()
    block, offset = slots // each, slots % each
    largest = torch.zeros((pages * blocks, heads), device=x.device).scatter_reduce(0, block[:, None].expand(-1, heads), size, "amax")
    lowest = torch.full((pages * blocks,), each, device=x.device).scatter_reduce(0, block, offset, "amin")[:, None]
    old = scales.transpose(1, 2).reshape(pages * blocks, heads)
    scale = torch.where(lowest == 0, _scale(largest), torch.where(lowest < each, torch.maximum(old, _scale(largest)), old))
    # tokens that a block held before take the grown scale
    ratio = torch.where(scale > 0, old / scale, 1.0)
    ratio = ratio.reshape(pages, blocks, heads).transpose(1, 2)[:, :, :, None, None]
    held = torch.arange(each, device=x.device) < lowest.view(pages, 1, blocks, 1)
    codes = cache.view(pages, heads, blocks, each, width)
    moved = torch.where(held[..., None] & (ratio < 1), (codes.float() * ratio).to(cache.dtype).float(), codes.float()).to(cache.dtype)
    cache.copy_(moved.reshape(cache.shape))
    scales.copy_(scale.reshape(pages, blocks, heads).transpose(1, 2))
    # a block of zeros has scale 0 and zero codes; numbers that are not finite become NaN
    inverse = torch.where(scale > 0, 1 / scale, 0.0)[block][..., None]
    code = torch.where(x.isfinite(), x * inverse, math.nan).to(cache.dtype)
    cache.view(torch.uint8)[slots // PAGE, :, slots % PAGE] = code.view(torch.uint8)


def _append_plain(s):
    _append_one(s["k_new"], s["slot_map"], s["k_cache"], s["k_scales"])
    _append_one(s["v_new"], s["slot_map"], s["v_cache"], s["v_scales"])
    return {name: s[name] for name in ("k_cache", "v_cache", "k_scales", "v_scales")}


def _attend_plain(s):
    q, table, L, start, sink, window, most = s["q"], s["page_table"].long(), s["seq_lens"].long(), s["q_start"].long(), s["sink"], s["window"], s["most_new"]
    batch, width = table.shape
    _, heads, _, dim = s["k_cache"].shape
    group = q.shape[1] // heads
    count = start[1:] - start[:-1]
    # the pages that hold kept tokens of any of a request's queries
    first = ((L - count + 1 - window).clamp(min=0) // PAGE)[:, None]
    front = _pages(sink)
    column = torch.arange(min(width, front + _pages(window + most) + 1), device=q.device)[None]
    page = torch.where(column < front, column, torch.maximum(first, torch.full_like(first, front)) + column - front)
    place = (page[..., None] * PAGE + torch.arange(PAGE, device=q.device)).view(batch, 1, -1)     # [batch, 1, tokens]
    page = table.gather(1, page.clamp(max=width - 1))
    # queries padded to the largest number
    t = torch.arange(most, device=q.device)[None]
    row = (start[:-1, None] + t).clamp(max=q.shape[0] - 1)
    reach = torch.where(t < count[:, None], L[:, None] - count[:, None] + t + 1, 0)[..., None]   # tokens that a query sees
    kept = (place < reach) & ((place < sink) | (place >= reach - window))                        # [batch, queries, tokens]
    def laid_out(cache, scales):
        x = cache.view(torch.uint8)[page].view(cache.dtype).float() * scales[page].repeat_interleave(PAGE // scales.shape[2], 3)[..., None]
        return x.transpose(1, 2).reshape(batch, heads, -1, dim)                                   # [batch, heads, tokens, dim]
    x = q[row].float().view(batch, most, heads, group, dim).transpose(1, 2).reshape(batch, heads, most * group, dim)
    logits = torch.matmul(x, laid_out(s["k_cache"], s["k_scales"]).transpose(2, 3)) * s["softmax_scale"]
    kept = kept[:, None, :, None].expand(-1, -1, -1, group, -1).reshape(batch, 1, most * group, -1)
    logits = torch.where(kept, logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    weights = torch.exp(logits - torch.where(top.isinf(), 0.0, top))
    total = weights.sum(-1, keepdim=True)
    values = torch.where(kept.any(2)[..., None], laid_out(s["v_cache"], s["v_scales"]), 0.0)
    out = torch.matmul(weights, values) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total))[..., 0]
    # back to one row per query token
    token = torch.arange(q.shape[0], device=q.device)
    request = torch.searchsorted(start[1:], token, right=True)
    mine = token - start[request]
    out = out.view(batch, heads, most, group, dim)[request, :, mine].reshape(q.shape)
    lse = lse.view(batch, heads, most, group)[request, :, mine].reshape(q.shape[:2])
    return {"out": out.to(s["out"].dtype), "lse": lse}


# ---------------------------------------------------------------------------------------------- passes

def run(s):
    if not own:
        return {"extend": _extend_plain, "append": _append_plain, "attend": _attend_plain}[s["op"]](s)
    import paper_2511_22481_amd as oa
    if s["op"] == "extend":
        oa.omniattn_table_extend(s["seq_lens"], s["new_lens"], s["free_pages"], s["free_count"], s["page_table"], s["seq_lens_out"],
                                 s["free_count_out"], s["q_start"], s["slot_map"])
        return {"page_table": s["page_table"], "seq_lens": s["seq_lens_out"], "free_count": s["free_count_out"], "q_start": s["q_start"],
                "slot_map": s["slot_map"]}
    if s["op"] == "append":
        oa.omniattn_gqa_append(s["k_new"], s["v_new"], s["slot_map"], s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"])
        return {name: s[name] for name in ("k_cache", "v_cache", "k_scales", "v_scales")}
    if "workspace" not in s:  # a serving loop keeps it
        size = oa.omniattn_gqa_workspace_bytes(batch=s["seq_lens"].shape[0], num_queries=s["q"].shape[0], num_q_heads=s["q"].shape[1],
                                               num_kv_heads=s["k_cache"].shape[1], head_dim=s["q"].shape[2])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    oa.omniattn_gqa_decode(s["q"], s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"], s["page_table"], s["seq_lens"], s["q_start"],
                           s["out"], s["lse"], s["workspace"], sink=s["sink"], window=s["window"], softmax_scale=s["softmax_scale"])
    return {"out": s["out"], "lse": s["lse"]}


def work(case):
    lens, news = _lengths(case)
    batch, tokens = case["batch"], sum(news)
    if case["op"] == "extend":
        fresh = sum(_pages(a) - _pages(a - b) for a, b in zip(lens, news))
        # lengths in and out, first tokens, the pages taken and their entries, the pages that slots lie in, the slots
        touched = sum(_pages(a) - (a - b) // PAGE for a, b in zip(lens, news))
        return {"bytes": 4 * (4 * batch + 3 + fresh + touched + tokens), "flops": 0}
    heads, dim, each = case["kv_heads"], case["head_dim"], case["scale_tokens"]
    if case["op"] == "append":
        blocks = sum(-(-a // each) - (a - b) // each for a, b in zip(lens, news))
        return {"bytes": 2 * (tokens * heads * dim * 3 + blocks * heads * 8) + 4 * tokens, "flops": 2 * 2 * tokens * heads * dim}
    read, products = 0, 0
    for n, new in zip(lens, news):
        union = min(n, case["sink"] + case["window"] + (new - 1 if case["window"] else 0))
        read += union * heads * 2 * dim + -(-union // each) * heads * 8 + 4 * _pages(union)
        products += sum(_kept(case, n - t) for t in range(new)) * case["q_heads"] * dim * 4
    width = 4 if case["out"] == "fp32" else 2
    return {"bytes": read + tokens * case["q_heads"] * (dim * (2 + width) + 4) + 4 * (2 * batch + 1), "flops": products}


# ---------------------------------------------------------------------------------------------- in 64 bits

def _e4m3(x):
    """Numbers (64 bits, within 448) rounded to the nearest that e4m3 holds, ties to even."""
    exponent = np.maximum(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -20))), -6)
    step = 2.0 ** (exponent - 3)
    return np.rint(x / step) * step


def _exact_append(new, slots, codes, scales):
    codes, scales = codes.float().cpu().numpy().astype(np.float64), scales.cpu().numpy().astype(np.float64)
    new, slots = new.float().cpu().numpy().astype(np.float64), slots.cpu().numpy()
    each = PAGE // scales.shape[2]
    i = 0
    while i < len(slots):
        page, offset = divmod(int(slots[i]), PAGE)
        block, low = offset // each, offset % each
        many = 1
        while i + many < len(slots) and low + many < each and slots[i + many] == slots[i] + many:
            many += 1
        rows = new[i:i + many].transpose(1, 0, 2)
        biggest = np.abs(rows).max((1, 2))
        scale = np.where(biggest > 0, 2.0 ** np.maximum(np.ceil(np.log2(np.maximum(biggest, 1e-300) / 448)), -126), 0.0)
        if low:
            scale = np.maximum(scale, scales[page, :, block])
            held = codes[page, :, block * each:block * each + low]
            held *= scales[page, :, block, None, None]
            held[:] = _e4m3(held / np.where(scale > 0, scale, 1)[:, None, None])
        codes[page, :, offset:offset + many] = _e4m3(rows / np.where(scale > 0, scale, 1)[:, None, None])
        scales[page, :, block] = scale
        i += many
    return torch.from_numpy(codes), torch.from_numpy(scales)


def exact(case, seed):
    if case["op"] == "extend":
        return None  # whole numbers
    s = prepare(case, seed)
    if case["op"] == "append":
        if sum(_lengths(case)[1]) * case["kv_heads"] * case["head_dim"] > 1 << 26:
            return None
        k, ks = _exact_append(s["k_new"], s["slot_map"], s["k_cache"], s["k_scales"])
        v, vs = _exact_append(s["v_new"], s["slot_map"], s["v_cache"], s["v_scales"])
        return {"k_cache": k, "v_cache": v, "k_scales": ks, "v_scales": vs}
    lens, news = _lengths(case)
    heads, dim, each = case["kv_heads"], case["head_dim"], case["scale_tokens"]
    group = case["q_heads"] // heads
    outs, lses, at = [], [], 0
    for b, (n, new) in enumerate(zip(lens, news)):
        pages = s["page_table"][b, :_pages(n)].long()
        position = torch.arange(n, device="cuda")
        mask = torch.stack([(position < n - new + t + 1) & ((position < case["sink"]) | (position >= n - new + t + 1 - case["window"])) for t in range(new)])
        some = mask.any(0).nonzero()[:, 0]
        def rows(cache, scales):
            page, off = pages[some // PAGE], some % PAGE
            return (cache.view(torch.uint8)[page, :, off].view(torch.float8_e4m3fn).double() * scales.double()[page, :, off // each][..., None]).transpose(0, 1)
        k, v = rows(s["k_cache"], s["k_scales"]), rows(s["v_cache"], s["v_scales"])        # [heads, kept, dim]
        x = s["q"][at:at + new].double().view(new, heads, group, dim).permute(1, 0, 2, 3).reshape(heads, new * group, dim)
        # (the softmax scale is an argument of 32 bits)
        logits = torch.bmm(x, k.transpose(1, 2).contiguous()) * float(np.float32(s["softmax_scale"]))
        hidden = ~mask[:, some].repeat_interleave(group, 0)[None]
        logits = logits.masked_fill(hidden, -math.inf)
        lse = torch.logsumexp(logits, -1)
        out = torch.bmm(torch.exp(logits - lse[..., None]).nan_to_num(0.0), v)
        outs.append(out.view(heads, new, group, dim).permute(1, 0, 2, 3).reshape(new, heads * group, dim))
        lses.append(lse.view(heads, new, group).permute(1, 0, 2).reshape(new, heads * group))
        at += new
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
