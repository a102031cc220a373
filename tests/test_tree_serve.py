"""The calls around a tree of drafts together, as a server makes them: trees come, are attended to, verified, and leave the cache what a text
without drafts would have left there."""
import random

import pytest
import torch

import paper_2511_22481_amd as oa
from paper_2511_22481_amd.gqa_serve import PAGE, Pool, speculate

gpu = pytest.mark.gpu
LAYERS, Q_HEADS, HEADS, VOCAB, TABLE = 2, 6, 2, 40, 997


class Model:
    """Rows of a token at a position come from a table; the target's logits are a projection of what the layers give.  The largest number of every
    K and V row is 1.75, so that a block's scale is 2^-8 whatever lies in it, and codes do not depend on the way that led to them."""

    def __init__(self, dim, seed):
        g = torch.Generator().manual_seed(seed)
        x = torch.randn((LAYERS, TABLE, Q_HEADS + 2 * HEADS, dim), generator=g)
        kv = x[:, :, Q_HEADS:]
        kv *= 1.75 / kv.abs().amax(-1, keepdim=True)
        self.rows_of = x.bfloat16().cuda()
        self.head = torch.randn((LAYERS * Q_HEADS * dim, VOCAB), generator=g).cuda() * 3

    def index(self, tokens, positions):
        return (tokens.long() * 31 + positions.long() * 7) % TABLE

    def rows(self, tokens, positions, buffer):
        buffer.copy_(self.rows_of[:, self.index(tokens, positions)])

    def logits(self, out):
        return out.float().transpose(0, 1).reshape(out.shape[1], -1) @ self.head


def _plain(model, dim, prompts, answers, sink, window):
    """A token at a time, greedily, with the calls that know no trees.  Returns the texts and the smallest distance between the two largest logits."""
    batch = len(prompts)
    pool = Pool(batch, LAYERS, 40, HEADS, dim, 8, scale_tokens=32)
    texts, closest = [list(p) for p in prompts], float("inf")
    news = [len(p) for p in prompts]
    for _ in range(max(answers)):
        n = sum(news)
        slots = torch.empty(n, dtype=torch.int32, device="cuda")
        pool.extend(torch.tensor(news, dtype=torch.int32, device="cuda"), slots)
        tokens = torch.tensor([t for x, k in zip(texts, news) for t in x[len(x) - k:]], device="cuda")
        positions = torch.tensor([i for x, k in zip(texts, news) for i in range(len(x) - k, len(x))], device="cuda")
        qkv = torch.empty((LAYERS, n, Q_HEADS + 2 * HEADS, dim), dtype=torch.bfloat16, device="cuda")
        model.rows(tokens, positions, qkv)
        out, lse = torch.empty((LAYERS, n, Q_HEADS, dim), device="cuda"), torch.empty((n, Q_HEADS), device="cuda")
        ws = torch.empty(oa.omniattn_gqa_workspace_bytes(batch, n, Q_HEADS, HEADS, dim), dtype=torch.uint8, device="cuda")
        for i in range(LAYERS):
            pool.attend(i, qkv[i], slots, out[i], lse, ws, sink, window)
        best = model.logits(out).topk(2)
        last = torch.tensor(news).cumsum(0) - 1
        for b, r in enumerate(last.tolist()):
            if len(texts[b]) < len(prompts[b]) + answers[b]:
                closest = min(closest, (best.values[r, 0] - best.values[r, 1]).item())
                texts[b].append(best.indices[r, 0].item())
        news = [1] * batch
    return texts, closest


def _near(dim):
    """Logits nearer than this may change places between two ways of summing.  An output is a mean, weighted with relative errors of about 2^-23 (32-bit
    scores, exponentials and sums, weights of 22 bits), of values up to 1.75: off by 1.75 * 2^-23 = 2.1e-7 in the mean square at the most.  A difference of two
    logits adds LAYERS * Q_HEADS * dim of them, times the difference of two numbers of deviation 3, and each of the two ways has its own errors: a
    deviation of 2.1e-7 * 3 sqrt(2) * sqrt(2) * sqrt(LAYERS * Q_HEADS * dim), 5e-5 at width 128.  Five of them."""
    return 5 * 1.75 * 2.0 ** -23 * 6 * (LAYERS * Q_HEADS * dim) ** 0.5


def _trees(rng, nodes, knows, wide=3):
    """Drafts that know the answer now and then: knows(text) is the token behind it."""
    def draft(texts):
        all_tokens, all_parents = [], []
        for text in texts:
            if text is None:
                all_tokens.append([])
                all_parents.append([])
                continue
            tokens, parents, ways = [text[-1]], [-1], [list(text)]
            for t in range(1, rng.randint(1, nodes)):
                p = rng.choice([t - 1, max(0, t - rng.randint(1, wide))])
                token = knows(ways[p]) if rng.random() < 0.7 else rng.randrange(VOCAB)
                tokens.append(token)
                parents.append(p)
                ways.append(ways[p] + [token])
            all_tokens.append(tokens)
            all_parents.append(parents)
        return all_tokens, all_parents, None
    return draft


@gpu
@pytest.mark.parametrize("dim,sink,window", [(64, 0, 10 ** 6), (128, 4, 60), (256, 0, 90)])
def test_trees_give_the_text_that_single_tokens_give(dim, sink, window):
    model, rng = Model(dim, dim), random.Random(dim)
    prompts = [[rng.randrange(VOCAB) for _ in range(n)] for n in (1, 30, 100, 127, 200)]
    answers = [25, 40, 33, 20, 1]
    want, closest = _plain(model, dim, prompts, answers, sink, window)
    assert closest > _near(dim)
    start = [len(p) for p in prompts]

    def knows(text):
        for b, full in enumerate(want):
            if full[:len(text)] == text and len(text) < len(full):
                return full[len(text)]
        return 0
    pool = Pool(len(prompts), LAYERS, 40, HEADS, dim, 8, scale_tokens=32)
    held = pool.free_count.item()
    what, texts = speculate(pool, prompts, answers, Q_HEADS, sink, window, model.rows, _trees(rng, 12, knows), model.logits, out_dtype=torch.float32)
    assert texts == want
    assert what["tokens"] == sum(answers) and what["steps"] < max(answers) and what["free_at_the_end"] == held
    assert [len(t) for t in texts] == [s + a for s, a in zip(start, answers)]


@gpu
@pytest.mark.parametrize("temperature", [0.0, 0.8])
def test_the_cache_holds_what_the_texts_say(temperature):
    """After every step, the rows of every text without its last token, whatever was drafted: codes in their slots, scales, pages, lengths."""
    dim, rng, gen = 64, random.Random(5), torch.Generator(device="cuda").manual_seed(5)
    model = Model(dim, 5)
    prompts = [[rng.randrange(VOCAB) for _ in range(n)] for n in (3, 120, 64, 250)]
    pool = Pool(len(prompts), LAYERS, 30, HEADS, dim, 6, scale_tokens=32)
    seen = []

    def observe(step, texts):
        lens, table = pool.lens.tolist(), pool.table.tolist()
        assert lens == [len(t) - 1 for t in texts]
        in_use = [p for b, n in enumerate(lens) for p in table[b][:-(-n // PAGE)]]
        free = pool.free[:pool.free_count.item()].tolist()
        assert sorted(in_use + free) == list(range(30))
        for b, text in enumerate(texts):
            n = lens[b]
            at = torch.arange(n, device="cuda")
            slot = torch.tensor(table[b], device="cuda")[at // PAGE]
            want = model.rows_of[:, model.index(torch.tensor(text[:n], device="cuda"), at), Q_HEADS:].float()
            for cache, scales, rows in ((pool.k, pool.k_scales, want[:, :, :HEADS]), (pool.v, pool.v_scales, want[:, :, HEADS:])):
                assert (scales[:, slot, :, at % PAGE // 32] == 2.0 ** -8).all()
                codes = cache.view(torch.uint8)[:, slot, :, at % PAGE].view(torch.float8_e4m3fn)     # [tokens, layers, heads, dim]
                assert torch.equal(codes.float(), (rows * 256).to(torch.float8_e4m3fn).float().transpose(0, 1))
        seen.append(sum(lens))
    draft = _trees(rng, 20, lambda text: (text[-1] * 5 + len(text)) % VOCAB)
    # (logits that prefer what the drafts guess, so that paths of several nodes stay)
    nodes = []

    def wrapped(texts):
        tokens, parents, probs = draft(texts)
        nodes[:] = [(t, len(text) + depth) for text, tree, up in zip(texts, tokens, parents) for t, depth in zip(tree, _depths(up))]
        return tokens, parents, probs

    def logits(out):
        scores = model.logits(out) * 0.01
        likely = torch.tensor([[(t * 5 + n) % VOCAB] for t, n in nodes], device="cuda")
        return scores.scatter_add(1, likely, torch.full((len(nodes), 1), 4.0, device="cuda"))
    speculate(pool, prompts, [60] * 4, Q_HEADS, 0, 10 ** 6, model.rows, wrapped, logits, temperature=temperature,
              uniforms=lambda n: torch.rand((n, 2), device="cuda", generator=gen), observe=lambda step, texts: observe(step, texts) if all(len(t) < 60 + len(p) for t, p in zip(texts, prompts)) else None)
    assert len(seen) > 3 and seen[-1] - seen[0] > 2 * 4 * (len(seen) - 1)   # (more than two tokens a request and step)


def _depths(parents):
    depths = []
    for p in parents:
        depths.append(depths[p] + 1 if p >= 0 else 0)
    return depths


@gpu
def test_requests_that_find_no_pages_wait():
    model, rng = Model(64, 7), random.Random(7)
    prompts = [[rng.randrange(VOCAB) for _ in range(n)] for n in (120, 125, 100)]
    want, closest = _plain(model, 64, prompts, [30, 20, 10], 0, 10 ** 6)
    assert closest > _near(64)
    pool = Pool(3, LAYERS, 4, HEADS, 64, 3, scale_tokens=32)   # (three requests of two pages each, sooner or later)
    what, texts = speculate(pool, prompts, [30, 20, 10], Q_HEADS, 0, 10 ** 6, model.rows, _trees(rng, 6, lambda text: rng.randrange(VOCAB)), model.logits,
                            out_dtype=torch.float32)
    assert texts == want and what["free_at_the_end"] == 4 and what["pages"] <= 4
    with pytest.raises(RuntimeError):
        speculate(Pool(3, LAYERS, 2, HEADS, 64, 3), prompts, [30, 20, 10], Q_HEADS, 0, 10 ** 6, model.rows, _trees(rng, 6, lambda text: 0), model.logits)


def _state(seed, batch=5, nodes=9, dim=64, vocab=300):
    g = torch.Generator(device="cuda").manual_seed(seed)
    total = batch * nodes
    pool = Pool(batch, LAYERS, 30, HEADS, dim, 6, scale_tokens=32)
    for t in (pool.k, pool.v):
        t.view(torch.uint8).zero_()
    pool.k_scales.fill_(2.0 ** -8)
    pool.v_scales.fill_(2.0 ** -8)
    i = dict(dtype=torch.int32, device="cuda")
    return dict(pool=pool, news=torch.full((batch,), nodes, **i), slots=torch.zeros(total, **i), masks=torch.zeros(total, dtype=torch.int64, device="cuda"),
                positions=torch.zeros(total, **i), qkv=torch.zeros((LAYERS, total, Q_HEADS + 2 * HEADS, dim), dtype=torch.bfloat16, device="cuda"),
                out=torch.zeros((LAYERS, total, Q_HEADS, dim), dtype=torch.bfloat16, device="cuda"), lse=torch.zeros((total, Q_HEADS), device="cuda"),
                ws=torch.empty(oa.omniattn_gqa_workspace_bytes(batch, total, Q_HEADS, HEADS, dim), dtype=torch.uint8, device="cuda"),
                logits=torch.zeros((total, vocab), device="cuda"), probs=torch.zeros((total, vocab), device="cuda"), tokens=torch.zeros(total, **i), parents=torch.zeros(total, **i),
                heat=torch.tensor([0.0, 1.0, 0.7, 1.3, 1.0], device="cuda"), uniforms=torch.zeros((total, 2), device="cuda"), path=torch.zeros(total, **i), said=torch.zeros(total, **i),
                chance=torch.zeros(total, device="cuda"), dropped=torch.zeros(batch, **i),
                vws=torch.empty(oa.omniattn_tree_verify_workspace_bytes(total, vocab), dtype=torch.uint8, device="cuda")), g


def _step(s):
    pool = s["pool"]
    pool.extend(s["news"], s["slots"])
    oa.omniattn_tree_masks(s["parents"], pool.lens, pool.q_start, s["masks"], s["positions"])
    for i in range(LAYERS):
        pool.attend_tree(i, s["qkv"][i], s["slots"], s["masks"], s["out"][i], s["lse"], s["ws"], 4, 100)
    oa.omniattn_tree_verify(s["logits"], s["probs"], s["tokens"], s["parents"], pool.q_start, s["heat"], s["uniforms"], s["path"], s["said"], s["chance"], s["dropped"], s["vws"])
    pool.keep(s["path"], s["dropped"])


def _inputs(s, g, step, kind):
    batch, total, vocab = s["news"].numel(), s["tokens"].numel(), s["logits"].shape[1]
    nodes, rng = total // batch, random.Random(step)
    s["qkv"].copy_(torch.randn(s["qkv"].shape, device="cuda", generator=g))
    s["logits"].copy_(torch.randn(s["logits"].shape, device="cuda", generator=g) * 4)
    s["probs"].copy_(torch.softmax(s["logits"] + torch.randn(s["logits"].shape, device="cuda", generator=g), -1))
    s["uniforms"].copy_(torch.rand(s["uniforms"].shape, device="cuda", generator=g))
    parents = [p for _ in range(batch) for p in [-1] + [t - 1 if kind == "chain" else rng.randrange(t) for t in range(1, nodes)]]
    first = torch.tensor([b * nodes + max(p, 0) for b in range(batch) for p in parents[b * nodes:(b + 1) * nodes]], device="cuda")
    drawn = torch.multinomial(s["probs"], 1, generator=g)[:, 0]
    s["tokens"].copy_(drawn[first])
    s["parents"].copy_(torch.tensor(parents))


NAMES = ("slots", "masks", "positions", "out", "lse", "path", "said", "chance", "dropped")


@gpu
def test_a_captured_step_follows_the_growing_texts():
    """Two graphs of the same calls on two pools that share their workspaces, replayed in turn with eager steps on a third pool between them."""
    eager, g = _state(1)
    captured = [_state(1)[0] for _ in range(2)]
    for name in ("ws", "vws"):
        captured[1][name] = captured[0][name]
    graphs = []
    for s in captured:
        _inputs(s, torch.Generator(device="cuda").manual_seed(0), 0, "chain")
        pool = s["pool"]
        names = ("lens", "table", "free", "free_count", "q_start", "k_scales", "v_scales")
        first = {n: getattr(pool, n).clone() for n in names}
        _step(s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _step(s)
        for n, t in first.items():
            getattr(pool, n).copy_(t)
        for t in (pool.k, pool.v):
            t.view(torch.uint8).zero_()
        graphs.append(graph)
    torch.cuda.synchronize()
    for step in range(6):
        seed = 100 + step
        for s in (eager, *captured):
            _inputs(s, torch.Generator(device="cuda").manual_seed(seed), step, "chain" if step % 2 else "any")
        _step(eager)
        torch.cuda.synchronize()
        for graph, s in zip(graphs, captured):
            graph.replay()
            torch.cuda.synchronize()
            for name in NAMES:
                assert torch.equal(eager[name], s[name]), (step, name)
            for name in ("lens", "table", "free", "free_count", "k_scales", "v_scales"):
                assert torch.equal(getattr(eager["pool"], name), getattr(s["pool"], name)), (step, name)
            for name in ("k", "v"):
                assert torch.equal(getattr(eager["pool"], name).view(torch.uint8), getattr(s["pool"], name).view(torch.uint8)), (step, name)


@gpu
def test_calls_on_another_stream():
    here, g = _state(2)
    there, _ = _state(2)
    for s in (here, there):
        _inputs(s, torch.Generator(device="cuda").manual_seed(9), 1, "any")
    _step(here)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        _step(there)
    stream.synchronize()
    for name in NAMES:
        assert torch.equal(here[name], there[name]), name
    # and the stream as an argument
    again, _ = _state(2)
    masks = torch.zeros_like(again["masks"])
    again["pool"].lens.fill_(9)
    again["pool"].q_start.copy_(torch.arange(0, 46, 9))
    torch.cuda.synchronize()
    oa.omniattn_tree_masks(here["parents"], again["pool"].lens, again["pool"].q_start, masks, None, stream=stream)
    stream.synchronize()
    assert torch.equal(masks, here["masks"])


@gpu
def test_the_command_serves_drafts():
    import json
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(oa.__file__)))
    res = subprocess.run([sys.executable, "-m", "paper_2511_22481_amd.gqa_serve", "--requests", "6", "--prompt", "100", "--answer", "20", "--layers", "2", "--heads", "4", "--kv-heads", "2",
                          "--dim", "64", "--drafts", "5"], capture_output=True, text=True, cwd=root, timeout=100)
    assert res.returncode == 0, res.stderr[-2000:]
    what = json.loads(res.stdout)
    assert what["tokens"] >= 6 and what["tokens_per_step"] > 2 and what["steps"] > 0


def test_a_temperature_needs_random_numbers():
    with pytest.raises(ValueError):
        speculate(None, [[1]], [1], 1, 0, 1, None, None, None, temperature=0.5)


@gpu
def test_two_steps_at_once():
    """Two pools' steps on two streams, call by call in turn, each with workspaces of its own."""
    want, got = [], []
    for k in range(2):
        for states in (want, got):
            s, _ = _state(2)
            _inputs(s, torch.Generator(device="cuda").manual_seed(20 + k), k, "any")
            states.append(s)
    for s in want:
        _step(s)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in got]

    def in_turn(call):
        for stream, s in zip(streams, got):
            with torch.cuda.stream(stream):
                call(s)
    in_turn(lambda s: s["pool"].extend(s["news"], s["slots"]))
    in_turn(lambda s: oa.omniattn_tree_masks(s["parents"], s["pool"].lens, s["pool"].q_start, s["masks"], s["positions"]))
    for i in range(LAYERS):
        in_turn(lambda s: s["pool"].attend_tree(i, s["qkv"][i], s["slots"], s["masks"], s["out"][i], s["lse"], s["ws"], 4, 100))
    in_turn(lambda s: oa.omniattn_tree_verify(s["logits"], s["probs"], s["tokens"], s["parents"], s["pool"].q_start, s["heat"], s["uniforms"], s["path"], s["said"], s["chance"],
                                              s["dropped"], s["vws"]))
    in_turn(lambda s: s["pool"].keep(s["path"], s["dropped"]))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for name in NAMES:
            assert torch.equal(a[name], b[name]), name
        assert torch.equal(a["pool"].lens, b["pool"].lens) and torch.equal(a["pool"].k.view(torch.uint8), b["pool"].k.view(torch.uint8))


class Rule:
    """Behind token t follows 21 t + 7 (which comes by all tokens), with a logit that no other token comes near; behind the tokens of `dead` the target has nothing to say (`nothing` for
    every logit).  Drafts guess right two times in three."""

    def __init__(self, seed, dead=(), nothing=float("-inf")):
        self.rng, self.dead, self.nothing, self.nodes = random.Random(seed), set(dead), nothing, []

    def after(self, token):
        return (21 * token + 7) % VOCAB

    def text(self, prompt, answer):
        """What a prompt becomes."""
        out = list(prompt)
        while answer and out[-1] not in self.dead:
            out.append(self.after(out[-1]))
            answer -= 1
        return out

    def draft(self, texts):
        self.nodes.clear()
        trees = [[] if t is None else [t[-1]] for t in texts]
        for tree in trees:
            for _ in range(self.rng.randint(0, 9) if tree else 0):
                tree.append(self.after(tree[-1]) if self.rng.random() < 2 / 3 else self.rng.randrange(VOCAB))
            self.nodes.extend(tree)
        return trees, [list(range(-1, len(t) - 1)) for t in trees], None

    def logits(self, out):
        scores = torch.zeros((out.shape[1], VOCAB), device="cuda").scatter_(1, torch.tensor([[self.after(t)] for t in self.nodes], device="cuda"), 200.0)
        return torch.where(torch.tensor([t in self.dead for t in self.nodes], device="cuda")[:, None], self.nothing, scores)


def _rows(tokens, positions, buffer):
    buffer.normal_()


@gpu
@pytest.mark.parametrize("temperature,nothing", [(0.0, float("-inf")), (0.9, float("-inf")), (0.9, float("nan"))])
def test_a_request_ends_where_the_target_has_no_token(temperature, nothing):
    """Behind a prompt, or on the way.  The others go on, with as many tokens in the cache as their texts say, and all pages come back."""
    rule = Rule(3, dead=(11,), nothing=nothing)
    prompts = [[5, 3], [2, 11], [9, 17], [30], [1] * 130, [4]]
    answers = [20, 20, 25, 10, 9, 1]
    want = [rule.text(p, a) for p, a in zip(prompts, answers)]
    short = [len(w) < len(p) + a for w, p, a in zip(want, prompts, answers)]
    assert any(short) and not all(short) and any(s and len(w) > len(p) + 1 for s, w, p in zip(short, want, prompts))
    pool = Pool(len(prompts), LAYERS, 20, HEADS, 64, 3, scale_tokens=32)

    def observe(step, texts):
        for n, text, full in zip(pool.lens.tolist(), texts, want):
            assert text == full[:len(text)] and (n in (0, len(text) - 1) or text == full)
    what, texts = speculate(pool, prompts, answers, Q_HEADS, 0, 10 ** 6, _rows, rule.draft, rule.logits, temperature=temperature,
                            uniforms=lambda n: torch.rand((n, 2), device="cuda"), observe=observe)
    assert texts == want
    assert what["free_at_the_end"] == 20 and what["cut_short"] == sum(short) and what["tokens"] == sum(len(w) - len(p) for w, p in zip(want, prompts))


@gpu
def test_requests_without_an_answer_hold_no_pages():
    """Among others that would find too few pages if they did, and alone."""
    rule = Rule(4)
    prompts, answers = [[1] * 300, [2] * 100, [3] * 260, [], [4]], [0, 50, 0, 5, 0]
    pool = Pool(5, LAYERS, 2, HEADS, 64, 3, scale_tokens=32)
    what, texts = speculate(pool, prompts, answers, Q_HEADS, 0, 10 ** 6, _rows, rule.draft, rule.logits)
    assert texts == [rule.text(p, a) if p else [] for p, a in zip(prompts, answers)]
    assert what["free_at_the_end"] == 2 and pool.lens.tolist() == [0] * 5 and what["tokens"] == 50 and what["cut_short"] == 0
    pool = Pool(2, LAYERS, 4, HEADS, 64, 3, scale_tokens=32)
    what, texts = speculate(pool, [[1] * 140, [2] * 5], [0, 0], Q_HEADS, 0, 10 ** 6, _rows, rule.draft, rule.logits)
    assert texts == [[1] * 140, [2] * 5] and what["free_at_the_end"] == 4 and what["steps"] == 0


@pytest.mark.parametrize("tokens,parents", [([[1] * 65, [2]], [[-1] + [0] * 64, [-1]]), ([[1], []], [[-1], []]), ([[1, 3], [2]], [[-1], [-1]]), ([[1]], [[-1]])])
def test_trees_that_speculate_refuses(tokens, parents):
    """More nodes than a tree may have, none for a text that is to grow, tokens and parents of other numbers, a tree too few."""
    pool = Pool(2, LAYERS, 4, HEADS, 64, 2, device="cpu")
    with pytest.raises(ValueError):
        speculate(pool, [[1], [2]], [5, 5], Q_HEADS, 0, 10, _rows, lambda texts: (tokens, parents, None), None)


@gpu
def test_the_cache_where_scales_change():
    """Rows whose largest numbers lie up to 2^6 apart, drafted and kept or dropped: what a text's slots hold is its rows, as far as a block's scale allows, which
    may be one that a dropped node has left (append raises a block's scale, and nothing lowers it again as long as tokens of the text lie in the block).
    A row is rounded when it is appended, to 2^-4 of a number or to half a subnormal step, 2^-10 of the scale; after that scales only grow, at least twofold,
    and codes times a power of two are rounded again only where they become subnormal: together 2^-10 of the last scale times 1 + 1/2 + .. < 2."""
    dim, rng = 64, random.Random(8)
    model, rule = Model(dim, 8), Rule(8)
    g = torch.Generator().manual_seed(8)
    factor = 2.0 ** torch.randint(-3, 4, (LAYERS, TABLE, 2 * HEADS, 1), generator=g).float()
    model.rows_of[:, :, Q_HEADS:] *= factor.cuda().bfloat16()
    prompts = [[rng.randrange(VOCAB) for _ in range(n)] for n in (3, 120, 64, 250)]
    pool = Pool(len(prompts), LAYERS, 30, HEADS, dim, 6, scale_tokens=32)
    seen = {"blocks": 0, "raised": 0, "steps": 0}

    def least(rows):
        """The smallest power of two by which the largest magnitude is at most 448."""
        part, exponent = torch.frexp(rows.abs().amax((-1, -2)).double() / 448)
        return torch.ldexp(torch.ones_like(part), exponent - (part == 0.5).int())

    def observe(step, texts):
        lens, table = pool.lens.tolist(), pool.table.tolist()
        for b, text in enumerate(texts):
            n = lens[b]
            if n != len(text) - 1:
                continue      # (it has its answer)
            at = torch.arange(n, device="cuda")
            slot = torch.tensor(table[b], device="cuda")[at // PAGE]
            want = model.rows_of[:, model.index(torch.tensor(text[:n], device="cuda"), at), Q_HEADS:].double()
            for cache, scales, rows in ((pool.k, pool.k_scales, want[:, :, :HEADS]), (pool.v, pool.v_scales, want[:, :, HEADS:])):
                codes = cache.view(torch.uint8)[:, slot, :, at % PAGE].view(torch.float8_e4m3fn).double()      # [tokens, layers, heads, dim]
                scale = scales[:, slot, :, at % PAGE // 32].double()                                           # [tokens, layers, heads]
                rows = rows.transpose(0, 1)
                assert ((codes * scale[..., None] - rows).abs() <= 2.0 ** -4 * rows.abs() + 2.0 ** -9 * scale[..., None]).all()
                for first in range(0, n, 32):
                    here, need = scale[first], least(rows[first:first + 32].permute(1, 2, 0, 3))
                    assert (scale[first:first + 32] == here).all() and (here >= need).all() and (here <= 2.0 ** -8 * 2.0 ** 3).all()
                    seen["blocks"] += here.numel()
                    seen["raised"] += int((here > need).sum())
        seen["steps"] += 1
    trees = _trees(rng, 20, lambda text: rule.after(text[-1]))

    def draft(texts):
        tokens, parents, probs = trees(texts)
        rule.nodes[:] = [t for tree in tokens for t in tree]
        return tokens, parents, probs
    what, texts = speculate(pool, prompts, [60] * 4, Q_HEADS, 0, 10 ** 6, model.rows, draft, rule.logits, observe=observe)
    assert texts == [rule.text(p, 60) for p in prompts] and what["steps"] < 40
    assert 0 < seen["raised"] < seen["blocks"], seen


@gpu
def test_nodes_of_requests_that_wait_have_their_positions():
    """rows is asked for their rows too: at the positions that they will have, not in front of the text."""
    rule, expected, waited = Rule(9), [], []
    prompts, answers = [[3] * 100, [7], [9], [11] * 2], [20, 12, 15, 9]
    pool = Pool(4, LAYERS, 2, HEADS, 64, 2, scale_tokens=32)

    def draft(texts):
        trees = rule.draft(texts)
        expected[:] = [len(text) - 1 + depth for text, tree in zip(texts, trees[0]) for depth in range(len(tree))]
        waited.append(sum(t is not None for t in texts))
        return trees

    def rows(tokens, positions, buffer):
        if waited:    # (after the prompts)
            assert positions.tolist() == expected and tokens.tolist() == rule.nodes
        buffer.normal_()
    what, texts = speculate(pool, prompts, answers, Q_HEADS, 0, 10 ** 6, rows, draft, rule.logits)
    assert texts == [rule.text(p, a) for p, a in zip(prompts, answers)] and what["pages"] == 2 and what["free_at_the_end"] == 2 and waited[0] == 4
