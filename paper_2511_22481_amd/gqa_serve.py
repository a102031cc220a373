"""A server's steps over the grouped-query layers of a model: requests arrive with prompts, take pages from a pool as they grow,
attend to their caches in 8 bits, and give the pages back when they are done.  Steps with chunks of prompts are called
one by one; steps in which every request brings at most one token are captured once and replayed, since tables, slots and the division
of the work are made on the device.

    python -m paper_2511_22481_amd.gqa_serve [--requests 64] [--prompt 1000] [--answer 100] [--layers 8] [--heads 32]
                                             [--kv-heads 8] [--dim 128] [--sink 0] [--window 1000000] [--drafts 0]

Prints one line: requests, steps, tokens, the largest number of pages in use, and us per layer of a decode step.  (The model's other parts
are left out: queries, keys and values are random rows.)  With --drafts N a request's step brings a tree of its last token and N drafted ones,
of which those stay that the target's logits agree with (here a rule that the drafts guess right two times in three), and the line says how
many tokens a step gives.
"""
import argparse
import json

PAGE = 128
NODES = 64  # of a tree, at most


class Pool:
    """The layers' caches and the requests' tables, which all layers share."""

    def __init__(self, requests, layers, pages, kv_heads, head_dim, max_pages, scale_tokens=64, device="cuda"):
        import torch
        ints = dict(dtype=torch.int32, device=device)
        codes = (layers, pages, kv_heads, PAGE, head_dim)
        # (pages hold nothing that counts before it is written)
        self.k, self.v = (torch.empty(codes, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn) for _ in range(2))
        self.k_scales, self.v_scales = (torch.empty((layers, pages, kv_heads, PAGE // scale_tokens), device=device) for _ in range(2))
        self.lens = torch.zeros(requests, **ints)
        self.table = torch.zeros((requests, max_pages), **ints)
        self.free, self.free_count = torch.arange(pages, **ints), torch.full((1,), pages, **ints)
        self.q_start = torch.zeros(requests + 1, **ints)

    def extend(self, new_lens, slots):
        from . import omniattn_table_extend
        omniattn_table_extend(self.lens, new_lens, self.free, self.free_count, self.table, self.lens, self.free_count, self.q_start, slots)

    def attend(self, layer, qkv, slots, out, lse, workspace, sink, window):
        """qkv: the new tokens' rows [tokens, query heads + 2 KV heads, head width]."""
        from . import omniattn_gqa_append, omniattn_gqa_decode
        heads, q_heads = self.k.shape[2], out.shape[1]
        q, k, v = qkv[:, :q_heads], qkv[:, q_heads:q_heads + heads], qkv[:, q_heads + heads:]
        cache = self.k[layer], self.v[layer], self.k_scales[layer], self.v_scales[layer]
        omniattn_gqa_append(k, v, slots, *cache)
        omniattn_gqa_decode(q, *cache, self.table, self.lens, self.q_start, out, lse, workspace, sink=sink, window=window,
                            softmax_scale=out.shape[2] ** -0.5)

    def attend_tree(self, layer, qkv, slots, masks, out, lse, workspace, sink, window):
        """As attend, for the nodes of trees."""
        from . import omniattn_gqa_append, omniattn_gqa_tree
        heads, q_heads = self.k.shape[2], out.shape[1]
        q, k, v = qkv[:, :q_heads], qkv[:, q_heads:q_heads + heads], qkv[:, q_heads + heads:]
        cache = self.k[layer], self.v[layer], self.k_scales[layer], self.v_scales[layer]
        omniattn_gqa_append(k, v, slots, *cache)
        omniattn_gqa_tree(q, *cache, self.table, self.lens, self.q_start, masks, out, lse, workspace, sink=sink, window=window,
                          softmax_scale=out.shape[2] ** -0.5)

    def keep(self, path, dropped):
        """Of the trees that the last extend counted, the nodes on `path` stay, dropped[b] others go."""
        from . import omniattn_gqa_keep, omniattn_table_truncate
        omniattn_gqa_keep(path, self.lens, self.q_start, self.table, self.k, self.v, self.k_scales, self.v_scales)
        omniattn_table_truncate(self.lens, dropped, self.table, self.free, self.free_count, self.lens, self.free_count)

    def release(self, done):
        from . import omniattn_table_release
        omniattn_table_release(self.lens, done, self.table, self.free, self.free_count)


def serve(pool, prompts, answers, q_heads, sink, window, rows, chunk=512, graph=True, observe=None):
    """Request b brings prompts[b] tokens, `chunk` to a step at most, and then answers[b] more, one to a step.  rows(step, buffer) fills the new
    tokens' rows of all layers, [layers, tokens, query heads + 2 KV heads, head width]; observe(step, new_lens, out, lse) sees what the
    layers give.  A request for whose new tokens there are no pages keeps its length (pool.lens; its rows of out and lse mean nothing) and brings
    them again in the next step, when others may have given pages back.  RuntimeError if a step has pages for none.  Returns what happened."""
    import torch
    from . import omniattn_gqa_decode_workspace_bytes
    layers, pages, heads, _, dim = pool.k.shape
    batch, device = len(prompts), pool.k.device
    # (a request without a prompt begins with its answer, a token a step)
    most = max(batch, sum(max(min(p, chunk), min(a, 1)) for p, a in zip(prompts, answers)))
    qkv = torch.empty((layers, most, q_heads + 2 * heads, dim), dtype=torch.bfloat16, device=device)
    out = torch.empty((layers, most, q_heads, dim), dtype=torch.bfloat16, device=device)
    lse = torch.empty((layers, most, q_heads), device=device)
    slots = torch.empty(most, dtype=torch.int32, device=device)
    new_lens, done = (torch.zeros(batch, dtype=torch.int32, device=device) for _ in range(2))
    workspace = torch.empty(omniattn_gqa_decode_workspace_bytes(batch, most, q_heads, heads, dim), dtype=torch.uint8, device=device)

    def step(n):
        """A step of up to n new tokens."""
        pool.extend(new_lens, slots[:n])
        for i in range(layers):
            pool.attend(i, qkv[i, :n], slots[:n], out[i, :n], lse[i, :n], workspace, sink, window)

    wait, left, captured = list(prompts), list(answers), None
    held = pool.lens.tolist()
    steps = tokens = used = 0
    decode_us = []
    while any(wait) or any(left):
        news = [min(w, chunk) if w else min(a, 1) for w, a in zip(wait, left)]
        alone = not any(wait)
        n = batch if alone else sum(news)
        new_lens.copy_(torch.tensor(news, dtype=torch.int32))
        rows(steps, qkv[:, :n])
        if alone and graph and captured is None:
            # (a warm-up with nothing to do: the tables stay as they are)
            new_lens.zero_()
            step(n)
            torch.cuda.synchronize()
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured):
                step(n)
            new_lens.copy_(torch.tensor(news, dtype=torch.int32))
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        captured.replay() if alone and graph else step(n)
        end.record()
        end.synchronize()
        if alone:
            decode_us.append(begin.elapsed_time(end) * 1000 / layers)
        if observe:
            observe(steps, news, out, lse)
        # (extend takes a request's tokens as a whole or not at all)
        lens = pool.lens.tolist()
        news = [n if after == before + n else 0 for n, before, after in zip(news, held, lens)]
        if not any(news):
            raise RuntimeError(f"{int(pool.free_count)} free pages of {pages}, and none of the requests that are left can go on: lengths {lens}, still to come {[w + a for w, a in zip(wait, left)]}")
        steps += 1
        tokens += sum(news)
        used = max(used, pages - int(pool.free_count))
        gone = []
        for b, (w, a) in enumerate(zip(wait, left)):
            wait[b], left[b] = (w - news[b], a) if w else (w, a - news[b])
            gone.append(int(news[b] > 0 and wait[b] == 0 and left[b] == 0))
        if any(gone):
            done.copy_(torch.tensor(gone, dtype=torch.int32))
            pool.release(done)
        held = [0 if g else n for g, n in zip(gone, lens)]
    return {"requests": batch, "steps": steps, "tokens": tokens, "pages": used, "free_at_the_end": int(pool.free_count),
            "decode_us_per_layer": sorted(decode_us)[len(decode_us) // 2] if decode_us else None}


def speculate(pool, prompts, answers, q_heads, sink, window, rows, draft, logits, temperature=0.0, uniforms=None, chunk=512, out_dtype=None, observe=None):
    """Requests with the prompts' tokens (lists) get answers[b] tokens each, by trees of drafted tokens.

    rows(tokens, positions, buffer) fills the rows of all layers for tokens at positions of their texts, [layers, tokens, query heads + 2 KV heads,
    head width]; logits(out) gives the target's logits [tokens, vocabulary] from what the layers give, [layers, tokens, query heads, head
    width].  draft(texts) returns for every text (a list; None: nothing is wanted, no nodes) the tree that follows it: tokens and parents of 1 to 64 nodes
    (ValueError otherwise), the first one the text's last token, and the probabilities that the first children were drawn from (a tensor [nodes of all,
    vocabulary], or None).  uniforms(nodes) returns the random numbers [nodes, 2] (needed with a temperature).  observe(step, texts) sees the texts as they
    grow.

    The prompts (of requests with an answer) have to fit in the pool together; after that a request whose tree finds no pages waits, as in serve.  A request ends early where the
    target has no token (logits of -inf or NaN only); "cut_short" says how many have.  Returns what happened, and the texts."""
    import torch
    from . import omniattn_gqa_workspace_bytes, omniattn_tree_masks, omniattn_tree_verify, omniattn_tree_verify_workspace_bytes
    if temperature > 0 and uniforms is None:
        raise ValueError("random numbers are needed with a temperature")
    layers, pages, heads, _, dim = pool.k.shape
    batch, device = len(prompts), pool.k.device
    ints = dict(dtype=torch.int32, device=device)

    def on_gpu(values, **kw):
        return torch.tensor(values, **{**ints, **kw})
    texts, goal = [list(p) for p in prompts], [len(p) + a for p, a in zip(prompts, answers)]
    heat = torch.full((batch,), temperature, device=device)

    def extend(news):
        """True for the requests that the tokens fit."""
        before = pool.lens.clone()
        slots = torch.empty(sum(news), **ints)
        pool.extend(on_gpu(news), slots)
        return slots, pool.lens == before + on_gpu(news)

    def call(tokens, positions, slots, masks):
        n = slots.numel()
        qkv = torch.empty((layers, n, q_heads + 2 * heads, dim), dtype=torch.bfloat16, device=device)
        rows(tokens, positions, qkv)
        out = torch.empty((layers, n, q_heads, dim), dtype=torch.bfloat16 if out_dtype is None else out_dtype, device=device)
        lse = torch.empty((n, q_heads), device=device)
        workspace = torch.empty(omniattn_gqa_workspace_bytes(batch, n, q_heads, heads, dim), dtype=torch.uint8, device=device)
        for i in range(layers):
            if masks is None:
                pool.attend(i, qkv[i], slots, out[i], lse, workspace, sink, window)
            else:
                pool.attend_tree(i, qkv[i], slots, masks, out[i], lse, workspace, sink, window)
        return out

    # the prompts without their last tokens, which are the first trees' first nodes (of a request that wants no answer nothing is looked at: it has no pages)
    at, last = [0] * batch, [max(len(p) - 1, 0) if a > 0 else 0 for p, a in zip(prompts, answers)]
    while any(a < n for a, n in zip(at, last)):
        news = [min(chunk, n - a) for a, n in zip(at, last)]
        slots, fits = extend(news)
        if not bool((fits & (on_gpu(news) > 0)).any()):
            raise RuntimeError(f"{int(pool.free_count)} free pages of {pages} are too few for the prompts")
        call(on_gpu([t for p, a, n in zip(prompts, at, news) for t in p[a:a + n]]), on_gpu([i for a, n in zip(at, news) for i in range(a, a + n)]), slots, None)
        at = [a + n * f for a, n, f in zip(at, news, fits.tolist())]
    steps = given = used = short = 0
    while any(0 < len(t) < g for t, g in zip(texts, goal)):
        wanted = [t if 0 < len(t) < g else None for t, g in zip(texts, goal)]
        tokens, parents, probs = draft(wanted)
        if len(tokens) != batch or len(parents) != batch:
            raise ValueError(f"{len(tokens)} and {len(parents)} trees' tokens and parents for {batch} texts")
        for b, (text, tree, up) in enumerate(zip(wanted, tokens, parents)):
            # (of a larger tree verification keeps nothing, again and again)
            if len(tree) > NODES or len(up) != len(tree) or (text is not None and not len(tree)):
                raise ValueError(f"text {b}: a tree of {len(tree)} tokens and {len(up)} parents; as many of either wanted, 1 to {NODES}")
        news = [len(t) for t in tokens]
        slots, fits = extend(news)
        if not bool((fits & (on_gpu(news) > 0)).any()):
            raise RuntimeError(f"{int(pool.free_count)} free pages of {pages}, and no request's tree fits: lengths {pool.lens.tolist()}")
        used = max(used, pages - int(pool.free_count))
        total = sum(news)
        node, parent = on_gpu([t for x in tokens for t in x]), on_gpu([p for x in parents for p in x])
        masks, positions = torch.empty(total, dtype=torch.int64, device=device), torch.empty(total, **ints)
        omniattn_tree_masks(parent, pool.lens, pool.q_start, masks, positions)
        # (lengths of requests that wait do not count their nodes: these would stand that much too far in front)
        request = torch.repeat_interleave(torch.arange(batch, device=device), on_gpu(news), output_size=total)
        positions += (on_gpu(news) * ~fits)[request]
        target = logits(call(node, positions, slots, masks))
        path, following, dropped = torch.empty(total, **ints), torch.empty(total, **ints), torch.empty(batch, **ints)
        workspace = torch.empty(omniattn_tree_verify_workspace_bytes(total, target.shape[1]), dtype=torch.uint8, device=device)
        numbers = torch.zeros((total, 2), device=device) if uniforms is None else uniforms(total)
        omniattn_tree_verify(target, probs, node, parent, pool.q_start, heat, numbers, path, following, None, dropped, workspace)
        # (a request whose tree found no pages has no nodes in the cache: nothing of it moves or goes)
        path.masked_fill_(~fits[request], -1)
        dropped.masked_fill_(~fits, 0)
        pool.keep(path, dropped)
        following, gone, fit, start = following.tolist(), dropped.tolist(), fits.tolist(), [0]
        done = [0] * batch
        for b, n in enumerate(news):
            new = [t for t in following[start[-1]:start[-1] + n] if t >= 0] if fit[b] else []
            start.append(start[-1] + n)
            # (the path's last node has no token behind it: the cache holds what the text ends with already, and the next tree could not begin with it)
            ended = fit[b] and len(new) < n - gone[b]
            new = new[:goal[b] - len(texts[b])]
            texts[b] += new
            given += len(new)
            if ended and len(texts[b]) < goal[b]:
                goal[b] = len(texts[b])
                short += 1
            done[b] = int(n > 0 and len(texts[b]) >= goal[b])
        if observe:
            observe(steps, texts)
        steps += 1
        if any(done):
            pool.release(on_gpu(done))
    return {"requests": batch, "steps": steps, "tokens": given, "pages": used, "free_at_the_end": int(pool.free_count),
            "tokens_per_step": round(given / max(steps, 1), 2), "cut_short": short}, texts


def main():
    ap = argparse.ArgumentParser()
    for name, default in (("requests", 64), ("prompt", 1000), ("answer", 100), ("layers", 8), ("heads", 32), ("kv-heads", 8), ("dim", 128), ("sink", 0), ("window", 10 ** 6),
                          ("drafts", 0)):
        ap.add_argument("--" + name, type=int, default=default)
    args = ap.parse_args()
    import torch
    if not torch.cuda.is_available():
        raise SystemExit("needs a GPU: the library has no CPU path")
    gen = torch.Generator().manual_seed(1)
    prompts, answers = (torch.randint(1, 2 * n + 1, (args.requests,), generator=gen).tolist() for n in (args.prompt, args.answer))
    if not 0 <= args.drafts < NODES:
        ap.error(f"a tree has up to {NODES} nodes: at most {NODES - 1} drafts")
    each = [-(-(p + a + args.drafts) // PAGE) for p, a in zip(prompts, answers)]
    pool = Pool(args.requests, args.layers, sum(each), args.kv_heads, args.dim, max(each))
    if args.drafts:
        print(json.dumps(_guessed(pool, prompts, answers, args)))
    else:
        print(json.dumps(serve(pool, prompts, answers, args.heads, args.sink, args.window, lambda step, buffer: buffer.normal_())))


def _guessed(pool, prompts, answers, args, vocab=1000):
    """A rule in the target's place: behind token t follows 7 t + 1.  Every draft follows the node before it and is right two times in three."""
    import random
    import torch
    rng = random.Random(1)
    nodes = []

    def draft(texts):
        nodes.clear()
        tokens = [[] if t is None else [t[-1]] for t in texts]
        for tree in tokens:
            for _ in range(args.drafts if tree else 0):
                tree.append((7 * tree[-1] + (1 if rng.random() < 2 / 3 else 2)) % vocab)
            nodes.extend(tree)
        return tokens, [list(range(-1, len(t) - 1)) for t in tokens], None

    def logits(out):
        scores = torch.zeros((out.shape[1], vocab), dtype=torch.bfloat16, device=out.device)
        return scores.scatter_(1, torch.tensor([[(7 * t + 1) % vocab] for t in nodes], device=out.device), 20.0)
    texts = [[rng.randrange(vocab) for _ in range(p)] for p in prompts]
    return speculate(pool, texts, answers, args.heads, args.sink, args.window, lambda tokens, positions, buffer: buffer.normal_(), draft, logits)[0]


if __name__ == "__main__":
    main()
