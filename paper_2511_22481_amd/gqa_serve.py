"""A server's steps over the grouped-query layers of a model: requests arrive with prompts, take pages from a pool as they grow,
attend to their caches in 8 bits, and give the pages back when they are done.  Steps with chunks of prompts are called
one by one; steps in which every request brings at most one token are captured once and replayed, since tables, slots and the division
of the work are made on the device.

    python -m paper_2511_22481_amd.gqa_serve [--requests 64] [--prompt 1000] [--answer 100] [--layers 8] [--heads 32]
                                             [--kv-heads 8] [--dim 128] [--sink 0] [--window 1000000]

Prints one line: requests, steps, tokens, the largest number of pages in use, and us per layer of a decode step.  (The model's other parts
are left out: queries, keys and values are random rows.)
"""
import argparse
import json

PAGE = 128


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

    def release(self, done):
        from . import omniattn_table_release
        omniattn_table_release(self.lens, done, self.table, self.free, self.free_count)


def serve(pool, prompts, answers, q_heads, sink, window, rows, chunk=512, graph=True, observe=None):
    """Request b brings prompts[b] tokens, `chunk` to a step at most, and then answers[b] more, one to a step.  rows(step, buffer) fills the new
    tokens' rows of all layers, [layers, tokens, query heads + 2 KV heads, head width]; observe(step, new_lens, out, lse) sees what the
    layers give.  A request for whose new tokens there are no pages keeps its length (pool.lens; its rows of out and lse mean nothing) and brings
    them again in the next step, when others may have given pages back.  RuntimeError if a step has pages for none.  Returns what happened."""
    import torch
    from . import omniattn_gqa_workspace_bytes
    layers, pages, heads, _, dim = pool.k.shape
    batch, device = len(prompts), pool.k.device
    # (a request without a prompt begins with its answer, a token a step)
    most = max(batch, sum(max(min(p, chunk), min(a, 1)) for p, a in zip(prompts, answers)))
    qkv = torch.empty((layers, most, q_heads + 2 * heads, dim), dtype=torch.bfloat16, device=device)
    out = torch.empty((layers, most, q_heads, dim), dtype=torch.bfloat16, device=device)
    lse = torch.empty((layers, most, q_heads), device=device)
    slots = torch.empty(most, dtype=torch.int32, device=device)
    new_lens, done = (torch.zeros(batch, dtype=torch.int32, device=device) for _ in range(2))
    workspace = torch.empty(omniattn_gqa_workspace_bytes(batch, most, q_heads, heads, dim), dtype=torch.uint8, device=device)

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


def main():
    ap = argparse.ArgumentParser()
    for name, default in (("requests", 64), ("prompt", 1000), ("answer", 100), ("layers", 8), ("heads", 32), ("kv-heads", 8), ("dim", 128), ("sink", 0), ("window", 10 ** 6)):
        ap.add_argument("--" + name, type=int, default=default)
    args = ap.parse_args()
    import torch
    if not torch.cuda.is_available():
        raise SystemExit("needs a GPU: the library has no CPU path")
    gen = torch.Generator().manual_seed(1)
    prompts, answers = (torch.randint(1, 2 * n + 1, (args.requests,), generator=gen).tolist() for n in (args.prompt, args.answer))
    each = [-(-(p + a) // PAGE) for p, a in zip(prompts, answers)]
    pool = Pool(args.requests, args.layers, sum(each), args.kv_heads, args.dim, max(each))
    print(json.dumps(serve(pool, prompts, answers, args.heads, args.sink, args.window, lambda step, buffer: buffer.normal_())))


if __name__ == "__main__":
    main()
