"""Trees of drafted tokens on the GPU: masks, attention, verification, the rows that stay and the pages that go, against plain 64-bit
implementations (tests/tree_reference.py)."""
import ctypes
import random

import numpy as np
import pytest
import torch

import gqa_reference as gref
import tree_reference as ref
import paper_2511_22481_amd as oa

PAGE = 128
gpu = pytest.mark.gpu


def ints(values, device="cuda"):
    return torch.tensor(values, dtype=torch.int32, device=device)


def longs(masks):
    return torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64, device="cuda")


def starts(counts):
    return [0] + [int(x) for x in np.cumsum(counts)]


def tree_of(rng, n, kind="any"):
    """Parents: any tree, a chain, all children of the first node, or several roots."""
    if kind == "chain":
        return [t - 1 for t in range(n)]
    if kind == "star":
        return [-1] + [0] * (n - 1)
    if kind == "roots":
        return [rng.choice([-1, rng.randrange(t) if t else -1]) for t in range(n)]
    return [-1] + [rng.choice([t - 1, rng.randrange(t)]) for t in range(1, n)]


# ------------------------------------------------------------------------------------------------ masks

@gpu
@pytest.mark.parametrize("batch,most,kind", [(1, 1, "any"), (1, 64, "chain"), (3, 64, "any"), (5, 63, "star"), (65, 17, "roots"), (700, 64, "any"), (1, 0, "any"), (6, 70, "any")])
def test_masks(batch, most, kind):
    rng = random.Random(batch + most)
    news = [most if b == 0 else rng.randint(0, most) for b in range(batch)]
    lens = [n + rng.choice([0, 5, 1000, 2 ** 31 - 200]) for n in news]
    trees = [tree_of(rng, n, kind) if n else [] for n in news]
    if kind == "roots":  # parents that are no nodes before the child
        trees = [[rng.choice([p, p, t, t + 1, -7, 2 ** 31 - 1]) for t, p in enumerate(tree)] for tree in trees]
    start = starts(news)
    total = start[-1]
    got = torch.full((total + 3,), -9, dtype=torch.int64, device="cuda")
    at = torch.full((total + 3,), -9, dtype=torch.int32, device="cuda")
    parents = ints([p for t in trees for p in t] or [0])[:total]
    oa.omniattn_tree_masks(parents, ints(lens), ints(start), got[:total], at[:total])
    want = [ref.masks(t, L - len(t)) for t, L in zip(trees, lens)]
    assert [m & (1 << 64) - 1 for m in got[:total].tolist()] == [m for w in want for m in w[0]]
    assert at[:total].tolist() == [p for w in want for p in w[1]]
    assert got[total:].tolist() == [-9] * 3 and at[total:].tolist() == [-9] * 3
    got.fill_(-9)
    oa.omniattn_tree_masks(parents, ints(lens), ints(start), got[:total])
    assert [m & (1 << 64) - 1 for m in got[:total].tolist()] == [m for w in want for m in w[0]]


@gpu
def test_masks_of_one_node_each_and_rows_of_no_request():
    masks, at = torch.full((4,), -9, dtype=torch.int64, device="cuda"), ints([-9] * 4)
    oa.omniattn_tree_masks(ints([-1, 0, 5, -1]), ints([1, 7, 128, 0]), None, masks, at)
    assert masks.tolist() == [1] * 4 and at.tolist() == [0, 6, 127, -1]
    masks.fill_(-9)
    oa.omniattn_tree_masks(ints([-1, 0, 0, -1]), ints([9]), ints([1, 3]), masks)
    assert masks.tolist() == [-9, 1, 3, -9]


# ------------------------------------------------------------------------------------------------ attention

class Problem:
    """A cache with shuffled pages; everything that no query keeps is poisoned (codes NaN, scales of blocks without kept tokens NaN or infinite)."""

    def __init__(self, lens, sets, q_heads, kv_heads, dim, each, sink, window, seed=0, poison=True):
        g = torch.Generator()
        g.manual_seed(seed)
        self.lens, self.sink, self.window, self.scale = lens, sink, window, dim ** -0.5
        news = [len(s) for s in sets]
        self.q_start, self.sets = starts(news), [m for s in sets for m in s]
        used = [max(0, -(-n // PAGE)) for n in lens]
        pages, width = sum(used) + 3, max(1, max(used))
        order = torch.randperm(pages, generator=g).tolist()
        self.table = [[order.pop() if c < u else 0 for c in range(width)] for u in used]
        x = torch.randn((2, pages, kv_heads, PAGE, dim), generator=g)
        blocks = x.view(2, pages, kv_heads, PAGE // each, each, dim)
        self.scales = blocks.abs().amax((-1, -2)) / 448 * (1 + torch.rand(blocks.shape[:4], generator=g))     # (not only powers of two)
        self.codes = (blocks / self.scales[..., None, None]).view(x.shape).to(torch.float8_e4m3fn)
        self.q = torch.randn((self.q_start[-1], q_heads, dim), generator=g).bfloat16()
        kept = np.zeros((pages, PAGE), dtype=bool)
        for b, (L, n) in enumerate(zip(lens, news)):
            for t in range(n):
                for j in ref.kept(self.sets[self.q_start[b] + t], L, n, sink, window):
                    kept[self.table[b][j // PAGE], j % PAGE] = True
        if poison:
            gone = torch.from_numpy(~kept)
            raw = self.codes.view(torch.uint8)
            raw[:] = torch.where(gone[None, :, None, :, None], torch.tensor(0x7f, dtype=torch.uint8), raw)
            empty = gone.view(pages, PAGE // each, each).all(-1)
            bad = torch.tensor([float("nan"), float("inf")])[torch.randint(0, 2, self.scales.shape, generator=g)]
            self.scales = torch.where(empty[None, :, None, :], bad, self.scales)

    def wide_table(self):
        """The table with so many columns more that the call is none of the small ones, for which blocks of 16 rows are taken."""
        batch, kv_heads, columns = len(self.lens), self.codes.shape[2], len(self.table[0])
        tiles = -(-(-(-len(self.sets) // batch) * (self.q.shape[1] // kv_heads)) // 16)
        return [r + [0] * max(0, 16 * 256 // (batch * kv_heads * tiles) + 1 - columns) for r in self.table]

    def run(self, out_dtype=torch.bfloat16, q_start=True, fill=0xff, pad=0):
        (k, v), (ks, vs), q = self.codes.cuda(), self.scales.cuda(), self.q.cuda()
        if pad:
            wide = torch.full((q.shape[0], q.shape[1] + pad, q.shape[2]), float("nan"), dtype=q.dtype, device="cuda")
            wide[:, :q.shape[1]] = q
            q = wide[:, :q.shape[1]]
        out = torch.full(self.q.shape, float("nan"), dtype=out_dtype, device="cuda")
        lse = torch.full(self.q.shape[:2], float("nan"), device="cuda")
        size = oa.omniattn_gqa_workspace_bytes(len(self.lens), max(1, q.shape[0]), q.shape[1], k.shape[1], q.shape[2])
        ws = torch.full((size,), fill, dtype=torch.uint8, device="cuda")
        oa.omniattn_gqa_tree(q, k, v, ks, vs, ints(self.table), ints(self.lens), ints(self.q_start) if q_start else None, longs(self.sets), out, lse, ws,
                             sink=self.sink, window=self.window, softmax_scale=self.scale)
        torch.cuda.synchronize()
        return out, lse

    def check(self, out_dtype=torch.bfloat16, **kw):
        result, short = self._check(out_dtype, **kw), self.table
        self.table = self.wide_table()
        try:
            self._check(out_dtype, **kw)
        finally:
            self.table = short
        return result

    def _check(self, out_dtype, **kw):
        out, lse = self.run(out_dtype, **kw)
        fn = ref.attend_fp32 if out_dtype == torch.float32 else ref.attend_bf16
        k, v = gref.as_double(self.codes)
        ks, vs = gref.as_double(self.scales)
        want, want_lse, tol, lse_tol = fn(gref.as_double(self.q), k, v, ks, vs, self.table, self.lens, self.q_start, self.sets, self.sink, self.window, self.scale)
        got, got_lse = gref.as_double(out), gref.as_double(lse)
        assert np.array_equal(got_lse == -np.inf, want_lse == -np.inf)
        fine = np.isfinite(want_lse)
        assert (np.abs(got_lse[fine] - want_lse[fine]) <= lse_tol[fine]).all(), np.argwhere(~(np.abs(got_lse - want_lse) <= lse_tol))[:5]
        err = np.abs(got - want)
        assert (err <= tol).all(), (np.argwhere(~(err <= tol))[:5], np.nanmax(err / np.maximum(tol, 1e-300)))
        return out, lse


def sets_of(rng, news, kind="any"):
    if kind == "random":   # sets that are no tree's, some of them empty, some with bits of nodes that are not there
        return [[rng.choice([0, rng.getrandbits(64), rng.getrandbits(64) & rng.getrandbits(64) & rng.getrandbits(64), 1 << rng.randrange(64)]) for _ in range(n)] for n in news]
    return [ref.masks(tree_of(rng, n, kind) if n else [], 0)[0] for n in news]


# rows of a KV head (nodes x group) that take each kernel: one to four row tiles, and the wide ones
SHAPES = [(64, 1, 1), (64, 4, 2), (64, 7, 1), (64, 12, 12), (128, 4, 4), (128, 8, 2), (128, 14, 2), (256, 3, 1), (256, 16, 2)]


@gpu
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("nodes", [1, 3, 9, 40])
@pytest.mark.parametrize("dim,q_heads,kv_heads", SHAPES)
def test_trees(dim, q_heads, kv_heads, nodes, out_dtype):
    rng = random.Random(nodes + dim + q_heads)
    news = [nodes, max(1, nodes // 2), nodes, 0, 1]
    lens = [n + t for n, t in zip(news, (0, 127 - nodes // 2, 200, 40, 300))]
    for each, (sink, window) in zip((32, 64, 128), ((0, 10 ** 6), (4, 60), (130, 0))):
        Problem(lens, sets_of(rng, news), q_heads, kv_heads, dim, each, sink, window, seed=nodes).check(out_dtype)


@gpu
@pytest.mark.parametrize("sink,window", [(0, 0), (0, 1), (0, 2), (1, 0), (3, 5), (128, 128), (130, 7), (64, 64), (10 ** 6, 0), (100, 0), (126, 1), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("dim,group", [(64, 2), (128, 5), (256, 1), (128, 1)])
def test_kept_sets(sink, window, dim, group):
    """Windows shorter than a tree is deep, sinks that end among the nodes, texts of no token."""
    rng = random.Random(sink % 1000 + window % 1000 + dim)
    news = [20, 64, 7, 33, 1, 16]
    lens = [n + t for n, t in zip(news, (110, 90, 0, 124, 129, 500))]
    for kind in ("any", "chain", "star"):
        Problem(lens, sets_of(rng, news, kind), 2 * group, 2, dim, 32, sink, window, seed=window % 100).check()


@gpu
@pytest.mark.parametrize("sink,window", [(0, 10 ** 6), (4, 40), (0, 3)])
@pytest.mark.parametrize("dim,q_heads,kv_heads", [(64, 3, 3), (64, 32, 2), (128, 2, 2), (128, 6, 1), (128, 16, 1), (256, 2, 1), (256, 8, 1)])
def test_any_sets_empty_ones_among_them(dim, q_heads, kv_heads, sink, window):
    rng = random.Random(dim + q_heads + window % 100)
    news = [5, 64, 30, 1, 2]
    lens = [n + t for n, t in zip(news, (300, 100, 3, 0, 128))]
    Problem(lens, sets_of(rng, news, "random"), q_heads, kv_heads, dim, 64, sink, window, seed=3).check()


@gpu
@pytest.mark.parametrize("dim,q_heads,kv_heads", [(64, 2, 2), (128, 4, 1), (256, 2, 1)])
def test_more_nodes_than_bits_or_tokens(dim, q_heads, kv_heads):
    rng = random.Random(dim)
    news = [90, 130, 70, 64]
    lens = [300, 130, 20, 10]   # (the last two have fewer tokens than nodes)
    Problem(lens, sets_of(rng, news, "random"), q_heads, kv_heads, dim, 64, 2, 10 ** 6, seed=4).check()


@gpu
@pytest.mark.parametrize("group,nodes,dim", [(1, 1, 64), (1, 6, 64), (4, 4, 64), (3, 4, 128)])
def test_many_short_requests(group, nodes, dim):
    rng = random.Random(group)
    batch = 300 if dim == 64 else 150
    news = [rng.randint(1, nodes) for _ in range(batch)]
    lens = [n + rng.choice([0, 1, 31, 100, 128, 250]) for n in news]
    for sink, window in ((0, 10 ** 6), (2, 40)):
        Problem(lens, sets_of(rng, news), 4 * group, 4, dim, 32, sink, window, seed=group).check()


@gpu
@pytest.mark.parametrize("dim,q_heads,kv_heads,nodes", [(64, 2, 1, 5), (128, 4, 2, 3), (128, 8, 1, 12), (256, 2, 1, 4), (256, 4, 1, 10)])
def test_long_texts_are_split_and_joined(dim, q_heads, kv_heads, nodes):
    rng = random.Random(nodes)
    Problem([20000, 77, 5003], sets_of(rng, [nodes, 2, nodes]), q_heads, kv_heads, dim, 64, 0, 10 ** 6, seed=5, poison=False).check(torch.float32)


@gpu
@pytest.mark.parametrize("dim,group", [(64, 1), (64, 6), (128, 1), (128, 8), (256, 1), (256, 6)])
def test_nan_reaches_only_the_queries_that_see_it(dim, group):
    """A node's V or K row, and a token of the text at the edge of some windows."""
    rng = random.Random(6)
    tree = tree_of(rng, 12)
    sets = ref.masks(tree, 0)[0]
    L, window = 200 + 12, 150
    for slot, in_k in ((200 + 5, False), (200 + 5, True), (200, False), (200 + 1 - 150, False), (200 + 2 - 150, True)):
        p = Problem([L], [sets], 2 * group, 2, dim, 64, 0, window, seed=7, poison=False)
        clean, clean_lse = p.run()
        page = p.table[0][slot // PAGE]
        p.codes.view(torch.uint8)[0 if in_k else 1, page, 1, slot % PAGE, 3] = 0xff
        out, lse = p.run()
        for t, m in enumerate(sets):
            hit = slot in ref.kept(m, L, 12, 0, window)
            mine, others = slice(group, 2 * group), slice(0, group)
            assert torch.equal(out[t, others], clean[t, others])
            assert torch.isnan(lse[t, mine]).all() == (hit and in_k) and (in_k or torch.equal(lse, clean_lse))
            bad = torch.isnan(out[t, mine])
            if not hit:
                assert not bad.any() and torch.equal(out[t, mine], clean[t, mine])
            else:
                assert bad.all() if in_k else (bad[:, 3].all() and bad.sum() == group)


@gpu
@pytest.mark.parametrize("dim,group,nodes", [(64, 6, 12), (64, 2, 12), (128, 2, 12), (128, 4, 12), (128, 5, 12), (128, 8, 12), (128, 8, 40), (256, 2, 12), (256, 6, 12)])
def test_nan_in_calls_that_are_not_small(dim, group, nodes):
    """As above, by the kernels of large calls, texts cut into shares, and a token that every node keeps among them."""
    rng = random.Random(7)
    sets = [ref.masks(tree_of(rng, nodes), 0)[0] for _ in range(2)]
    text, window = 1500, 900
    p = Problem([text + nodes, 300 + nodes], sets, 2 * group, 2, dim, 64, 4, window, seed=7, poison=False)
    p.table = p.wide_table()
    clean, clean_lse = p.run()
    k = p.codes.clone()
    for slot, in_k in ((text + 5, False), (text + 5, True), (text, False), (text + 2 - window, True), (text + 3 - window, False), (1100, False), (1100, True), (2, False), (50, False)):
        p.codes = k.clone()
        p.codes.view(torch.uint8)[0 if in_k else 1, p.table[0][slot // PAGE], 1, slot % PAGE, 3] = 0xff
        out, lse = p.run()
        assert torch.equal(out[nodes:], clean[nodes:]) and torch.equal(lse[nodes:], clean_lse[nodes:])
        for t, m in enumerate(sets[0]):
            hit = slot in ref.kept(m, text + nodes, nodes, 4, window)
            mine, others = slice(group, 2 * group), slice(0, group)
            assert torch.equal(out[t, others], clean[t, others]) and torch.equal(lse[t, others], clean_lse[t, others])
            assert torch.isnan(lse[t, mine]).all() == (hit and in_k) and (in_k or torch.equal(lse, clean_lse))
            bad = torch.isnan(out[t, mine])
            if not hit:
                assert not bad.any() and torch.equal(out[t, mine], clean[t, mine])
            else:
                assert bad.all() if in_k else (bad[:, 3].all() and bad.sum() == group)


@gpu
@pytest.mark.parametrize("kind", ["any", "chain"])
@pytest.mark.parametrize("dim,group", [(64, 1), (64, 4), (128, 1), (128, 4), (256, 1)])
def test_a_block_of_zeros_before_one_of_very_large_values(dim, group, kind):
    """The text's values are 0 with scales of 0, those of the nodes in the second page have a scale of 2^60: the queries that see none of these give 0 or what
    the nodes of the first page hold."""
    text = 103
    p = Problem([text + 64], sets_of(random.Random(dim), [64], kind), 2 * group, 2, dim, 32, 0, 10 ** 6, seed=dim, poison=False)
    p.scales[1, p.table[0][0], :, :3], p.scales[1, p.table[0][1], :, 0] = 0.0, 2.0 ** 60
    out, lse = p.check(torch.float32)
    first = [t for t, m in enumerate(p.sets) if m >> 128 - text == 0]
    assert len(first) >= 25 and (out[first].abs() < 10).all()
    if kind == "chain":
        (k, v), (ks, vs) = p.codes.cuda(), p.scales.cuda()
        got = oa.gqa_decode(p.q.cuda(), k, v, ks, vs, ints(p.table), ints(p.lens), 0, 10 ** 6, p.scale, q_start=ints(p.q_start), out_dtype=torch.float32)[0]
        assert (got[first].abs() < 10).all() and torch.isfinite(got).all()


@gpu
@pytest.mark.parametrize("dim,q_heads", [(64, 40), (128, 24), (128, 70), (256, 33)])
def test_groups_of_more_rows_than_a_block_of_16(dim, q_heads):
    """A node's query heads over several blocks, in small calls and others."""
    rng = random.Random(dim + q_heads)
    news = [5, 1, 9]
    Problem([n + rng.randint(0, 700) for n in news], sets_of(rng, news), q_heads, 1, dim, 64, 4, 300, seed=q_heads).check(torch.float32)


@gpu
def test_strides_one_node_each_and_what_the_workspace_holds():
    p = Problem([129, 1, 300], [[1], [1], [0]], 8, 2, 128, 64, 0, 10 ** 6)
    out, lse = p.check(pad=3)
    assert (out[2] == 0).all() and (lse[2] == -np.inf).all()
    other = p.run(q_start=False, fill=0)
    assert torch.equal(out, other[0]) and torch.equal(lse, other[1])


@gpu
@pytest.mark.parametrize("dim,nodes,group", [(64, 1, 1), (64, 40, 4), (128, 3, 4), (128, 7, 4), (128, 20, 4), (128, 2, 40), (256, 30, 2)])
def test_calls_without_trees_ask_for_no_more_than_they_need(dim, nodes, group):
    """Rows of a block, their outputs and statistics in 32 bits, two blocks to a work group, and a word of 64 bits to a row of the call; blocks of a decode have 64
    rows at most (two work groups to a compute unit, or one where they have 64 rows of a width above 64; four of 16 rows, with four shares each, at width 64)."""
    batch, heads = 9, 2
    sizes = [f(batch, batch * nodes, heads * group, heads, dim) for f in (oa.omniattn_gqa_decode_workspace_bytes, oa.omniattn_gqa_workspace_bytes)]
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    slots = 2 * cus * (64 if dim > 64 else 256)
    assert sizes[0] <= sizes[1] and sizes[0] <= slots * (16 + 4 * dim) + 8 * batch * nodes * heads * group + 512
    p = Problem([n + 300 for n in [nodes] * batch], sets_of(random.Random(dim), [nodes] * batch, "chain"), heads * group, heads, dim, 64, 0, 10 ** 6, poison=False)
    (k, v), (ks, vs), q = p.codes.cuda(), p.scales.cuda(), p.q.cuda()
    args = q, k, v, ks, vs, ints(p.table), ints(p.lens)
    start = ints(p.q_start)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    held = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    want, want_lse = oa.gqa_decode(*args, 0, 10 ** 6, p.scale, q_start=start)
    # (torch rounds tensors to 512 bytes, and those above 10 MB to 2 MB: 17848832 bytes of workspace become 18874368)
    assert torch.cuda.max_memory_allocated() - held <= sizes[0] + 2 * q.numel() + 4 * want_lse.numel() + 2 * 512 + 2 ** 21
    out, lse = torch.empty_like(want), torch.empty_like(want_lse)
    ws = torch.full((sizes[0],), 0xff, dtype=torch.uint8, device="cuda")
    for n in (batch * nodes, batch):   # (fewer queries, too)
        oa.omniattn_gqa_decode(q[:n], k, v, ks, vs, ints(p.table), ints(p.lens), start if n == batch * nodes else None, out[:n], lse[:n], ws, sink=0, window=10 ** 6, softmax_scale=p.scale)
        if n == batch * nodes:
            assert torch.equal(out, want) and torch.equal(lse, want_lse)
    torch.cuda.synchronize()


@gpu
def test_a_workspace_without_trees_is_refused_where_a_tree_needs_more():
    p = Problem([20000] * 8, sets_of(random.Random(1), [16] * 8), 32, 8, 128, 64, 0, 10 ** 6, poison=False)
    (k, v), (ks, vs), q = p.codes.cuda(), p.scales.cuda(), p.q.cuda()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    ws = torch.empty(oa.omniattn_gqa_decode_workspace_bytes(8, 128, 32, 8, 128), dtype=torch.uint8, device="cuda")
    with pytest.raises(oa.OmniAttnError) as e:
        oa.omniattn_gqa_tree(q, k, v, ks, vs, ints(p.table), ints(p.lens), ints(p.q_start), longs(p.sets), out, lse, ws, sink=0, window=10 ** 6, softmax_scale=p.scale)
    assert e.value.code == -3


@gpu
def test_a_chain_is_what_decode_computes():
    p = Problem([150, 260, 700], sets_of(random.Random(1), [20, 3, 64], "chain"), 8, 2, 128, 64, 4, 100, poison=False)
    out, lse = p.check()
    (k, v), (ks, vs) = p.codes.cuda(), p.scales.cuda()
    chain, chain_lse = oa.gqa_decode(p.q.cuda(), k, v, ks, vs, ints(p.table), ints(p.lens), 4, 100, p.scale, q_start=ints(p.q_start))
    # (both are off by the same bounds; blocks may be cut elsewhere)
    assert (out.float() - chain.float()).abs().max() <= 2.0 ** -7 * chain.abs().max()
    assert torch.allclose(lse, chain_lse, rtol=0, atol=1e-4)
    wrapped = oa.gqa_tree(p.q.cuda(), k, v, ks, vs, ints(p.table), ints(p.lens), longs(p.sets), 4, 100, p.scale, q_start=ints(p.q_start))
    assert torch.equal(wrapped[0], out) and torch.equal(wrapped[1], lse)


@gpu
def test_rows_of_no_request_are_left_alone():
    p = Problem([200, 130], sets_of(random.Random(2), [6, 6]), 4, 2, 64, 64, 0, 10 ** 6)
    p.q_start = [2, 5, 9]
    p.lens = [200, 130]
    (k, v), (ks, vs) = torch.nan_to_num(p.codes.float()).to(torch.float8_e4m3fn).cuda(), torch.ones_like(p.scales).cuda()
    out, lse = torch.full(p.q.shape, 7.0, dtype=torch.bfloat16, device="cuda"), torch.full(p.q.shape[:2], 7.0, device="cuda")
    ws = torch.empty(oa.omniattn_gqa_workspace_bytes(2, 12, 4, 2, 64), dtype=torch.uint8, device="cuda")
    oa.omniattn_gqa_tree(p.q.cuda(), k, v, ks, vs, ints(p.table), ints(p.lens), ints(p.q_start), longs(p.sets), out, lse, ws, sink=0, window=10 ** 6, softmax_scale=p.scale)
    for rows in (slice(0, 2), slice(9, 12)):
        assert (out[rows] == 7).all() and (lse[rows] == 7).all()
    assert not (lse[2:9] == 7).any()


# ------------------------------------------------------------------------------------------------ verification

def _verify(logits, q, tokens, parents, start, T, uniforms, logprobs=True, fill=0xff):
    total, vocab = logits.shape
    path, out = (torch.full((total,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    chances = torch.full((total,), -9.0, device="cuda") if logprobs else None
    dropped = torch.full((len(T),), -9, dtype=torch.int32, device="cuda")
    ws = torch.full((max(1, oa.omniattn_tree_verify_workspace_bytes(total, vocab)),), fill, dtype=torch.uint8, device="cuda")
    oa.omniattn_tree_verify(logits, q, ints(tokens) if total else ints([0])[:0], ints(parents) if total else ints([0])[:0], None if start is None else ints(start),
                            torch.tensor(T, dtype=torch.float32, device="cuda"), uniforms, path, out, chances, dropped, ws)
    return path, out, chances, dropped


def _check_verify(logits, q, tokens, parents, start, T, uniforms):
    path, out, chances, dropped = _verify(logits, q, tokens, parents, start, T, uniforms)
    wide = gref.as_double(logits)
    drafts, u = None if q is None else gref.as_double(q), gref.as_double(uniforms)
    T = [float(np.float32(x)) for x in T]
    for b, t in enumerate(T):
        rows = slice(start[b], start[b + 1])
        n = start[b + 1] - start[b]
        way, said, chance = ref.verify(wide[rows], None if q is None else drafts[rows], tokens[rows], parents[rows], t, u[rows])
        rest = [-1] * (n - len(way))
        assert path[rows].tolist() == way + rest, b
        assert out[rows].tolist() == said + rest, b
        assert dropped[b].item() == n - len(way), b
        got = gref.as_double(chances[rows])
        want = np.array(chance + [0.0] * len(rest))
        # One rounding to fp32.  A weight is off by 5.6e-11 of itself; a part's sum takes two such factors and its place among the row's parts two
        # more (a lane's and the wave's), so that a row's sum, and the logarithm, is off by 4 * 5.6e-11 and a few 2^-53 of it.
        assert np.array_equal(np.isinf(got), np.isinf(want))
        fine = np.isfinite(want)
        assert (np.abs(got[fine] - want[fine]) <= 2.0 ** -24 * np.abs(want[fine]) + 2.3e-10).all()
    return path, out, chances, dropped


def _drafts(rng, gen, news, vocab, dtype, with_q, T, peak=4.0, kind="any"):
    """Logits, the drafts' probabilities, tokens that are often the target's, parents, uniforms (on the CPU)."""
    total = sum(news)
    logits = (torch.randn((total, vocab), generator=gen) * peak).to(dtype)
    parents = [p for n in news for p in (tree_of(rng, n, kind) if n else [])]
    q = torch.softmax((logits.float() + torch.randn((total, vocab), generator=gen)) / 0.8, -1) if with_q else None
    start = starts(news)
    tokens = [0] * total
    for b in range(len(news)):
        for i in range(start[b], start[b + 1]):
            p = parents[i]
            if 0 <= p < i - start[b]:
                row = start[b] + p
                likely = logits[row].float().topk(min(3, vocab)).indices.tolist()
                tokens[i] = int(torch.multinomial(q[row], 1, generator=gen)) if with_q and rng.random() < 0.8 else rng.choice(likely)
    return logits, q, tokens, parents, start, torch.rand((total, 2), generator=gen)


VOCABS = [1, 2, 7, 8, 9, 63, 511, 512, 513, 2047, 2048, 2049, 5000, 70001]


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("with_q", [False, True])
@pytest.mark.parametrize("vocab", VOCABS)
def test_verify(vocab, with_q, dtype):
    rng, gen = random.Random(vocab), torch.Generator().manual_seed(vocab)
    news = [1, 5, 16, 3, 0, 17, 2, 40, 64, 7] if vocab < 10000 else [5, 3, 1, 20]
    T = [rng.choice([0.0, 0.3, 1.0, 1.7]) for _ in news]
    logits, q, tokens, parents, start, u = _drafts(rng, gen, news, vocab, dtype, with_q, T)
    got = _check_verify(logits.cuda(), None if q is None else q.cuda(), tokens, parents, start, T, u.cuda())
    again = _verify(logits.cuda(), None if q is None else q.cuda(), tokens, parents, start, T, u.cuda(), fill=0)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@gpu
@pytest.mark.parametrize("dtype,offset,extra", [(torch.bfloat16, 1, 3), (torch.bfloat16, 0, 8), (torch.float32, 3, 1), (torch.bfloat16, 5, 0)])
def test_verify_rows_of_any_stride_and_alignment(dtype, offset, extra):
    """Rows that begin anywhere, with NaN around them."""
    rng, gen = random.Random(offset), torch.Generator().manual_seed(offset)
    news, vocab = [6, 1, 9], 3001
    T = [1.0, 0.7, 0.0]
    logits, q, tokens, parents, start, u = _drafts(rng, gen, news, vocab, dtype, True, T)
    stride = vocab + extra
    def laid_out(x):
        flat = torch.full((offset + stride * x.shape[0],), float("inf"), dtype=x.dtype, device="cuda")
        view = flat[offset:].view(x.shape[0], stride)[:, :vocab]
        view.copy_(x)
        return view
    _check_verify(laid_out(logits), laid_out(q), tokens, parents, start, T, u.cuda())


@gpu
@pytest.mark.parametrize("with_q", [False, True])
def test_verify_special_logits(with_q):
    """Ties, masked tokens, rows of nothing, infinities, NaN, tiny and huge temperatures, tokens outside the vocabulary."""
    rng, gen = random.Random(1), torch.Generator().manual_seed(1)
    vocab, inf, nan = 4099, float("inf"), float("nan")
    T = [0.0, 1.0, 1e-30, 1e30, inf, nan, -1.0, 1e-45, 1.0, 1.0, 0.0, 0.5]
    news = [4] * len(T)
    logits, q, tokens, parents, start, u = _drafts(rng, gen, news, vocab, torch.float32, with_q, T, kind="chain")
    logits[0, 100] = logits[0, 4000] = logits[0, 7] = 60.0                       # a tie: the first
    logits[4:8, ::2] = -inf                                                       # half of the tokens masked
    logits[20:24] = -inf                                                          # (a temperature of NaN: greedy) nothing left
    logits[24, 50] = nan
    logits[32:36] = -inf
    logits[36, 77] = logits[36, 2500] = inf
    logits[40:44] = nan
    logits[44] = 3.4e38
    logits[44, 9] = -3.4e38
    logits[1, :] = -inf
    logits[1, 4098] = -3e38
    tokens[9], tokens[13] = vocab, -5
    tokens[37] = 77
    _check_verify(logits.cuda(), None if q is None else q.cuda(), tokens, parents, start, T, u.cuda())


@gpu
def test_verify_drafts_that_equal_the_target_and_uniforms_at_the_ends():
    vocab, nodes = 1000, 6
    gen = torch.Generator().manual_seed(2)
    logits = torch.randn((nodes, vocab), generator=gen) * 3
    q = torch.softmax(logits.double(), -1).float()
    parents = [t - 1 for t in range(nodes)]
    tokens = [0] + [int(torch.multinomial(q[t], 1, generator=gen)) for t in range(nodes - 1)]
    for u0, u1 in ((0.0, 0.0), (1 - 2.0 ** -24, 1 - 2.0 ** -24), (0.5, 0.0), (0.0, 1 - 2.0 ** -24)):
        u = torch.tensor([[u0, u1]] * nodes)
        path = _check_verify(logits.cuda(), q.cuda(), tokens, parents, [0, nodes], [1.0], u.cuda())[0]
        if u0 < 0.9:
            assert path.tolist() == list(range(nodes))
        _check_verify(logits.cuda(), None, tokens, parents, [0, nodes], [1.0], u.cuda())
    # nothing is left of max(p - q, 0): p itself
    _check_verify(logits.cuda(), torch.full_like(q, 2.0).cuda(), tokens, parents, [0, nodes], [1.0], torch.full((nodes, 2), 0.9, device="cuda"))


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("drafts", ["none", "near", "above"])
@pytest.mark.parametrize("vocab,front,back", [(6000, 2048, 1500), (6001, 3000, 0), (4097, 0, 2048), (270000, 130 * 2048, 100)])
def test_verify_uniforms_at_the_ends_over_many_parts(vocab, front, back, dtype, drafts):
    """The first and the last token that has a probability, where whole parts of a row have none: behind masks of large negative numbers, or because a
    small temperature leaves nothing of them.  Few nodes to a request, and more than a work group has waves.  (Distances from a row's top are whole numbers where the
    temperature is small: over it none lies between 707, from where on the kernel takes a weight for 0, and 746, from where on exp in 64 bits is 0.)"""
    rng, gen = random.Random(vocab + front), torch.Generator().manual_seed(vocab + front)
    ends = (0.0, 1 - 2.0 ** -24)
    for nodes, kinds in ((3, [(T, mask, u1) for T in (1.0, 0.02, 0.005) for mask in (-1e9, -3e38, -float("inf")) for u1 in ends]),
                         (20, [(1.0, -1e9, 0.0), (0.02, -1e9, 0.0), (0.005, -40.0, 0.0), (0.005, -40.0, ends[1])])):
        if vocab > 10 ** 5:
            nodes, kinds = 9 if nodes == 20 else 2, rng.sample(kinds, 3)
        total = nodes * len(kinds)
        logits, parents, start = torch.empty((total, vocab)), [t - 1 for t in range(nodes)] * len(kinds), starts([nodes] * len(kinds))
        q = {"none": None, "near": torch.empty((total, vocab)), "above": torch.full((total, vocab), 2.0)}[drafts]
        u, tokens = torch.empty((total, 2)), [0] * total
        for b, (T, mask, u1) in enumerate(kinds):
            rows = slice(start[b], start[b + 1])
            logits[rows] = torch.randn((nodes, vocab), generator=gen) * 3 if T == 1.0 else -torch.randint(0, 40, (nodes, vocab), generator=gen).float()
            logits[rows, :front] = mask
            logits[rows, vocab - back:] = mask
            logits[rows, vocab - back - 1] = 0.0      # (a token next to the masked ones that has a probability at any temperature)
            u[rows, 0], u[rows, 1] = 0.9, u1
            exact = logits[rows].to(dtype).double()
            for i, row in enumerate(exact):
                t = float(np.float32(T))
                if drafts == "near":
                    q[start[b] + i] = torch.softmax((row + torch.randn(vocab, generator=gen).double()) / t, -1).float()
                if i + 1 < nodes:    # (the token that follows without drafts' probabilities: the walk goes on)
                    tokens[start[b] + i + 1] = ref.verify(gref.as_double(row[None]), None, [0], [-1], t, np.array([[0.9, u1]]))[1][0]
        path, out = _check_verify(logits.to(dtype).cuda(), None if q is None else q.cuda(), tokens, parents, start, [T for T, _, _ in kinds], u.cuda())[:2]
        assert (out.cpu()[torch.tensor(start[:-1])] >= 0).all()
        if drafts != "near":
            assert path.tolist() == list(range(nodes)) * len(kinds)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("drafts", ["none", "above", "half"])
@pytest.mark.parametrize("nodes,vocab", [(3, 8), (12, 64), (3, 5000), (20, 5001), (2, 300000)])
def test_verify_borders_between_tokens_of_the_same_logit(nodes, vocab, dtype, drafts):
    """2^a likeliest tokens, all others far away: weights of 1 and 0, so that sums, probabilities and borders at u1 = j / 2^a are exact in 64 bits, and the token is
    the one behind the border.  half: the drafts' probabilities are 2 / 2^a for half of these tokens, and u0 lies on the border to the first child's or a step of 32
    bits below it."""
    rng, gen = random.Random(vocab + nodes), torch.Generator().manual_seed(vocab + nodes)
    batch = 12 if vocab < 10 ** 5 else 3
    total = batch * nodes
    # (one temperature so small that nothing else is left, and logits near 0)
    T = [rng.choice([1.0, 0.7, 1.9, 0.001]) for _ in range(batch)]
    logits, u, tokens = torch.empty((total, vocab)), torch.empty((total, 2)), [0] * total
    q = {"none": None, "above": torch.full((total, vocab), 2.0), "half": torch.zeros((total, vocab))}[drafts]
    for i in range(total):
        many = 2 ** rng.randint(1, min(12, vocab.bit_length() - 1))
        top = rng.choice([0.0, 7.3, -11.6, 30.1])
        far = rng.choice([-float("inf"), -1e9]) if T[i // nodes] > 0.01 else top - 2.0 - 10 * torch.rand(vocab, generator=gen)
        logits[i] = far
        at = torch.randperm(vocab, generator=gen)[:many].sort().values
        logits[i, at] = top
        u[i] = torch.tensor([0.9, rng.randrange(many) / many])
        if drafts == "half":
            some = at[torch.randperm(many, generator=gen)[:many // 2]]
            q[i, some] = 2 / many
            u[i] = torch.tensor([rng.choice([0.5, 0.5 - 2.0 ** -24]), rng.randrange(many) / many])
            if (i + 1) % nodes:
                tokens[i + 1] = some[rng.randrange(len(some))].item()
        elif (i + 1) % nodes:    # (the walk goes on)
            tokens[i + 1] = at[int(u[i, 1] * many)].item()
    parents, start = [t - 1 for t in range(nodes)] * batch, starts([nodes] * batch)
    path = _check_verify(logits.to(dtype).cuda(), None if q is None else q.cuda(), tokens, parents, start, T, u.cuda())[0]
    if drafts != "half":
        assert path.tolist() == list(range(nodes)) * batch


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("batch,nodes,vocab", [(1, 6, 1000), (3, 20, 5000), (2, 64, 300000)])
def test_verify_refused_first_children_that_are_sampled_after_all(batch, nodes, vocab, dtype):
    """Drafts' probabilities above the target's everywhere: a first child is refused, nothing is left of max(p - q, 0), and p's sample is the same
    token.  Node 9 has a q that leaves something of p."""
    rng, gen = random.Random(vocab), torch.Generator().manual_seed(vocab)
    logits, q, tokens, parents, start, u = _drafts(rng, gen, [nodes] * batch, vocab, dtype, True, [1.0] * batch, kind="chain")
    for b in range(batch):
        for t in range(nodes - 1):
            row = start[b] + t
            logits[row, tokens[row + 1]] = 30.0
            if t % 4 != 3:
                q[row] = 2.0
                u[row, 0] = 0.75
            if t == 9:   # (refused, and another token in its place)
                q[row] = 0.0
                q[row, tokens[row + 1]] = 2.0
    path = _check_verify(logits.cuda(), q.cuda(), tokens, parents, start, [1.0] * batch, u.cuda())[0]
    assert (path.view(batch, nodes)[:, :10].amax(1) == min(nodes - 1, 9)).all()


@gpu
def test_verify_nodes_that_the_walk_does_not_reach_and_too_many_of_them():
    rng, gen = random.Random(3), torch.Generator().manual_seed(3)
    vocab, news = 50, [65, 4, 64, 100, 6]
    T = [1.0] * 5
    logits, _, tokens, parents, start, u = _drafts(rng, gen, news, vocab, torch.float32, False, T, kind="roots")
    path, out, chances, dropped = _check_verify(logits.cuda(), None, tokens, parents, start, T, u.cuda())
    assert dropped[0].item() == 65 and dropped[3].item() == 100
    # one node each without q_start; rows of no request
    T = [0.0, 1.0, 0.5]
    got = _verify(logits[:3].cuda(), None, tokens[:3], parents[:3], None, T, u[:3].cuda(), logprobs=False)
    assert got[0].tolist() == [0, 0, 0] and got[3].tolist() == [0, 0, 0]
    assert got[1].tolist() == _check_verify(logits[:3].cuda(), None, tokens[:3], parents[:3], [0, 1, 2, 3], T, u[:3].cuda())[1].tolist()
    got = _verify(logits[:9].cuda(), None, tokens[:9], parents[:9], [2, 5, 6], [1.0, 1.0], u[:9].cuda())
    for t in got[:3]:
        assert t[:2].tolist() == [-9] * 2 and t[6:].tolist() == [-9] * 3


@gpu
@pytest.mark.parametrize("with_q", [False, True])
@pytest.mark.parametrize("batch,most,vocab", [(150, 3, 40), (150, 30, 2100), (2, 9, 270000), (3, 40, 300001)])
def test_verify_many_requests_and_large_vocabularies(batch, most, vocab, with_q):
    """More requests than a wave looks at at once, more parts of a row than it does; few nodes to a request and many."""
    rng, gen = random.Random(batch + vocab), torch.Generator().manual_seed(vocab)
    news = [rng.randint(0, most) for _ in range(batch)]
    T = [rng.choice([0.0, 0.6, 1.0, 40.0]) for _ in news]      # (40: all of the parts have a share)
    logits, q, tokens, parents, start, u = _drafts(rng, gen, news, vocab, torch.bfloat16, with_q, T)
    _check_verify(logits.cuda(), None if q is None else q.cuda(), tokens, parents, start, T, u.cuda())


@gpu
def test_verify_of_nothing():
    got = _verify(torch.empty((0, 100), device="cuda"), None, [], [], [0, 0, 0], [1.0, 0.0], torch.empty((0, 2), device="cuda"))
    assert got[3].tolist() == [0, 0]


@gpu
@pytest.mark.parametrize("with_q", [False, True])
def test_verified_tokens_are_distributed_as_the_target(with_q):
    """200000 requests with the same two tokens to draft: the first new token has the target's distribution, whatever the drafts were."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    batch, vocab = 200000, 6
    row = torch.tensor([1.0, 0.2, -1.0, 2.0, 0.5, -3.0], device="cuda")
    p = torch.softmax(row.double() / 0.9, -1)
    q = torch.softmax(torch.tensor([2.0, 0.0, 0.0, -1.0, 1.0, 0.0], device="cuda"), -1)
    logits = row.expand(2 * batch, vocab).contiguous()
    drafts = torch.multinomial(q.expand(batch, vocab), 1, generator=gen)[:, 0].int()
    tokens = torch.stack([torch.zeros_like(drafts), drafts], 1).reshape(-1).contiguous()
    parents = ints([-1, 0]).repeat(batch)
    start = torch.arange(0, 2 * batch + 1, 2, device="cuda").int()
    u = torch.rand((2 * batch, 2), device="cuda", generator=gen)
    path, out = (torch.empty(2 * batch, dtype=torch.int32, device="cuda") for _ in range(2))
    dropped = torch.empty(batch, dtype=torch.int32, device="cuda")
    ws = torch.empty(oa.omniattn_tree_verify_workspace_bytes(2 * batch, vocab), dtype=torch.uint8, device="cuda")
    oa.omniattn_tree_verify(logits, q.expand(2 * batch, vocab).contiguous() if with_q else None, tokens, parents, start,
                            torch.full((batch,), 0.9, device="cuda"), u, path, out, None, dropped, ws)
    share = torch.bincount(out[::2].long(), minlength=vocab).double() / batch
    # five standard deviations of a share
    assert ((share - p).abs() <= 5 * (p * (1 - p) / batch).sqrt()).all(), (share.tolist(), p.tolist())
    taken = (dropped == 0).double().mean().item()
    want = torch.minimum(p, q.double()).sum().item() if with_q else (p * q.double()).sum().item()
    assert abs(taken - want) <= 5 * (want * (1 - want) / batch) ** 0.5


# ------------------------------------------------------------------------------------------------ rows that stay

def _cache(layers, pages, heads, dim, each, seed, special=False):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (2, layers, pages, heads, PAGE, dim), generator=g, dtype=torch.uint8)
    if not special:
        codes[(codes & 0x7f) == 0x7f] = 0x3a
    scales = 2.0 ** torch.randint(-4, 5, (2, layers, pages, heads, PAGE // each), generator=g).float()
    if special:
        scales *= 1 + (torch.rand(scales.shape, generator=g) < 0.3) * torch.rand(scales.shape, generator=g)
        scales[torch.rand(scales.shape, generator=g) < 0.2] = 0.0
    return codes.view(torch.float8_e4m3fn), scales


def _check_keep(path, lens, start, table, codes, scales, with_start=True, squeeze=False):
    k, v = codes.cuda()
    ks, vs = scales.cuda()
    if squeeze:
        k, v, ks, vs = k[0], v[0], ks[0], vs[0]
    oa.omniattn_gqa_keep(ints(path), ints(lens), ints(start) if with_start else None, ints(table), k, v, ks, vs)
    for got, got_scales, was, was_scales in ((k, ks, codes[0], scales[0]), (v, vs, codes[1], scales[1])):
        want, want_scales = gref.as_double(was), gref.as_double(was_scales)
        ref.keep(path, lens, start, table, want, want_scales)
        assert np.array_equal(gref.as_double(got).reshape(want.shape), want, equal_nan=True)
        assert np.array_equal(gref.as_double(got_scales).reshape(want_scales.shape), want_scales)


def _paths(rng, news, kind="any"):
    out = []
    for n in news:
        m = rng.randint(0, n)
        way = list(range(m)) if kind == "same" else sorted(rng.sample(range(n), m))
        if kind == "first" and n:
            way = [0] + [p for p in way if p > 0]
        out += way + [-1] * (n - len(way))
    return out


@gpu
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("each", [32, 64, 128])
@pytest.mark.parametrize("layers,heads,kind", [(1, 1, "any"), (3, 5, "first"), (2, 8, "same"), (2, 2, "special")])
def test_keep(dim, each, layers, heads, kind):
    rng = random.Random(dim + each + layers)
    news = [1, 64, 64, 0, 5, 40, 33, 2, 64, 17]
    lens = [n + t for n, t in zip(news, (0, 0, 100, 50, 126, 31, 64, 127, 95, rng.randint(0, 300)))]
    used = [-(-n // PAGE) for n in lens]
    order = random.Random(1).sample(range(sum(used) + 2), sum(used))
    table = [[order.pop() if c < u else 0 for c in range(max(used))] for u in used]
    codes, scales = _cache(layers, sum(used) + 2, heads, dim, each, dim, kind == "special")
    for seed in range(3):
        _check_keep(_paths(rng, news, kind), lens, starts(news), table, codes, scales, squeeze=layers == 1)


@gpu
def test_keep_paths_that_end_early_and_requests_that_are_left_alone():
    news = [6, 6, 6, 6, 70, 9, 5]
    path = [0, 2, 1, 3, 4, 5] + [1, 1, 2, 3, 4, 5] + [0, 3, 9, 4, 5, 5] + [-1, 2, 3, 4, 5, -1] + sorted(random.Random(1).sample(range(70), 30)) + [-1] * 40 + [2, 4, 6, 8] + [-1] * 5 \
        + [2 ** 31 - 1, 1, 2, 3, 4]
    lens = [20, 130, 129, 40, 200, 5, 77]   # (the last but one has fewer tokens than nodes)
    table = [[3 * b + c for c in range(3)] for b in range(7)]
    codes, scales = _cache(2, 22, 2, 64, 32, 1)
    _check_keep(path, lens, starts(news), table, codes, scales)
    # one node each
    _check_keep([0, 5, -1], [3, 128, 129], [0, 1, 2, 3], [r[:2] for r in table[:3]], codes, scales, with_start=False)


@gpu
@pytest.mark.parametrize("layers,heads,each", [(46, 2, 32), (31, 5, 64)])
def test_keep_of_more_layers_than_waves_at_once_is_that_of_each_layer(layers, heads, each):
    """A wave takes several layers then, the last one fewer."""
    batch, dim = 300, 64
    rng, g = random.Random(layers), torch.Generator(device="cuda").manual_seed(layers)
    news = [rng.choice([0, 1, 5, 31, 64]) for _ in range(batch)]
    lens = [n + rng.randint(0, 200) for n in news]
    used = [-(-n // PAGE) for n in lens]
    order = rng.sample(range(sum(used) + 2), sum(used))
    table = ints([[order.pop() if c < u else 0 for c in range(max(used))] for u in used])
    codes = torch.randint(0, 0x7f, (2, layers, sum(used) + 2, heads, PAGE, dim), generator=g, dtype=torch.uint8, device="cuda")
    scales = 2.0 ** torch.randint(-4, 5, (2, layers, sum(used) + 2, heads, PAGE // each), generator=g, device="cuda").float()
    path, args = ints(_paths(rng, news)), (ints(lens), ints(starts(news)), table)
    want, want_scales = codes.clone(), scales.clone()
    for i in range(layers):
        oa.omniattn_gqa_keep(path, *args, *(t[i].view(torch.float8_e4m3fn) for t in want), want_scales[0][i], want_scales[1][i])
    assert not torch.equal(want, codes)
    oa.omniattn_gqa_keep(path, *args, *(t.view(torch.float8_e4m3fn) for t in codes), scales[0], scales[1])
    assert torch.equal(codes, want) and torch.equal(scales, want_scales)


@gpu
def test_keep_of_many_layers_past_two_gigabytes():
    """Layers whose codes lie more than 2^32 bytes behind the first."""
    layers, pages, heads, dim = 70, 512, 8, 128
    k = torch.zeros((layers, pages, heads, PAGE, dim), dtype=torch.uint8, device="cuda")
    assert k.numel() > 2 ** 32
    scales = torch.ones((2, layers, pages, heads, 2), device="cuda")
    table = ints([[500, 511]])
    at = torch.arange(8, device="cuda", dtype=torch.uint8) + 0x30
    k[:, 500, :, 124:128] = at[None, None, :4, None]
    k[:, 511, :, :4] = at[None, None, 4:, None]
    k = k.view(torch.float8_e4m3fn)
    v = k.clone()
    oa.omniattn_gqa_keep(ints([0, 3, 6, -1, -1, -1, -1, -1]), ints([132]), ints([0, 8]), table, k, v, scales[0], scales[1])
    for t in (k.view(torch.uint8), v.view(torch.uint8)):
        assert (t[:, 500, :, 124:128] == at[[0, 3, 6, 3]][None, None, :, None]).all()
        assert (t[:, 511, :, :4] == at[None, None, 4:, None]).all()


# ------------------------------------------------------------------------------------------------ pages that go

@gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch,seed", [(1, 0), (64, 1), (65, 2), (1024, 3), (1500, 4), (2500, 5)])
def test_truncate(batch, seed, in_place):
    rng = random.Random(seed)
    lens = [rng.choice([0, 1, 128, 129, 256, 257, rng.randint(0, 700)]) for _ in range(batch)]
    dropped = [rng.choice([0, 0, 1, 2, 64, 128, 129, -3, L, L + 5, 2 ** 31 - 1, -2 ** 31]) for L in lens]
    table = [[10 * b + k for k in range(6)] for b in range(batch)]
    held = rng.sample(range(1 << 20, 1 << 21), 9)
    entries = 9 + 6 * batch
    for most in (entries, 9 + batch // 3):   # (the second stack is full before all pages are back: it takes no more)
        stack = held + [-7] * (most - 9)
        want = ref.truncate(lens, dropped, table, stack, 9, most)
        guard = ints(stack + [-8] * 4)
        L, c = ints(lens), ints([9])
        L_out, c_out = (L, c) if in_place else (torch.full_like(L, -9), torch.full_like(c, -9))
        wide = torch.full((batch, 8), -5, dtype=torch.int32, device="cuda")
        wide[:, :6] = ints(table)
        oa.omniattn_table_truncate(L, ints(dropped), wide[:, :6], guard[:most], c, L_out, c_out)
        assert L_out.tolist() == want[0] and guard.tolist() == want[1] + [-8] * 4 and c_out.tolist() == [want[2]]


@gpu
def test_truncate_of_nonsense_lengths():
    lens, dropped = [-5, 2 ** 31 - 1, 900, 0], [3, 2 ** 31 - 1, 100, 7]
    table = [[1, 2], [3, 4], [5, 6], [7, 8]]
    stack, c = ints([-7] * 8), ints([0])
    L = ints(lens)
    oa.omniattn_table_truncate(L, ints(dropped), ints(table), stack, c, L, c)
    # (lengths past the table: its pages)
    assert L.tolist() == [-5, 0, 800, 0] and c.tolist() == [2] and stack.tolist() == [3, 4] + [-7] * 6


# ------------------------------------------------------------------------------------------------ refusals

GOOD = 0x1000   # an address that is aligned and never read: the calls below are refused before


def _gqa(**kw):
    fields = dict(batch=2, num_queries=2, num_q_heads=4, num_kv_heads=2, head_dim=128, page_size=128, scale_tokens=64, max_pages_per_seq=4,
                  page_table_stride=4, num_pages=9, sink=0, window=100, softmax_scale=0.1, out_dtype=oa.BF16)
    fields.update(kw)
    return oa.Gqa(**fields)


def test_tree_masks_refuses_bad_arguments():
    lib = oa.load_library()
    good = [2, 5, GOOD, GOOD, GOOD, GOOD, GOOD, None]
    for at, value in ((0, 0), (0, -1), (1, -1), (2, None), (3, None), (4, None), (5, None), (5, GOOD + 4)):
        assert lib.omniattn_tree_masks(*(good[:at] + [value] + good[at + 1:])) == -1, (at, value)
    assert lib.omniattn_tree_masks(1 << 27, 5, *good[2:]) == -2
    assert lib.omniattn_tree_masks(2, 0, None, None, GOOD, None, None, None) == 0


@pytest.mark.parametrize("at,value", [(1, None), (1, GOOD + 2), (2, 511), (2, 504), (3, None), (3, GOOD + 8), (4, None), (5, None), (6, None), (7, None), (8, None),
                                      (9, None), (10, None), (10, GOOD + 4), (11, None), (11, GOOD + 4), (12, None)])
def test_tree_attention_refuses_bad_arguments(at, value):
    lib = oa.load_library()
    g = _gqa(num_queries=3)   # (so that a missing q_start is refused too)
    args = [ctypes.byref(g), GOOD, 512, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, 1 << 40, None]
    args[at] = value
    assert lib.omniattn_gqa_tree(*args) == -1
    assert lib.omniattn_gqa_tree(*([None] + args[1:])) == -1


@pytest.mark.parametrize("change,code", [(dict(batch=0), -1), (dict(window=-1), -1), (dict(head_dim=96), -2), (dict(scale_tokens=16), -2), (dict(softmax_scale=float("nan")), -1),
                                         (dict(page_table_stride=3), -1), (dict(num_queries=1 << 30), -2)])
def test_tree_attention_refuses_bad_problems(change, code):
    g = _gqa(**change)
    assert oa.load_library().omniattn_gqa_tree(ctypes.byref(g), GOOD, 512, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, 1 << 40, None) == code


@pytest.mark.parametrize("change,code", [(dict(batch=0), -1), (dict(num_tokens=-1), -1), (dict(vocab=0), -1), (dict(vocab=-5), -1), (dict(logits_dtype=oa.FP8_E4M3), -2),
                                         (dict(vocab=2 ** 31 - 1), -2), (dict(num_tokens=2 ** 31 - 1, vocab=2 ** 20), -2),
                                         (dict(num_tokens=2 ** 26), -2), (dict(num_tokens=2 ** 20, vocab=2 ** 17), -2), (dict(batch=2 ** 23), -2)])
def test_verify_refuses_bad_problems(change, code):
    lib = oa.load_library()
    v = oa.Verify(**dict(dict(batch=2, num_tokens=5, vocab=100, logits_dtype=oa.BF16), **change))
    assert lib.omniattn_tree_verify(ctypes.byref(v), GOOD, 2 ** 40, GOOD, 2 ** 40, *[GOOD] * 10, 1 << 60, None) == code
    assert lib.omniattn_tree_verify_workspace_bytes(ctypes.byref(v)) == 0


@pytest.mark.parametrize("at,value,code", [(0, None, -1), (1, None, -1), (2, 99, -1), (4, 99, -1), (5, None, -1), (6, None, -1), (7, None, -1), (8, None, -1), (9, None, -1), (10, None, -1),
                                           (11, None, -1), (13, None, -1), (14, None, -3), (14, GOOD + 16, -3), (15, 5 * 24 - 1, -3)])
def test_verify_refuses_bad_arguments(at, value, code):
    lib = oa.load_library()
    v = oa.Verify(batch=2, num_tokens=5, vocab=100, logits_dtype=oa.BF16)
    args = [ctypes.byref(v), GOOD, 100, GOOD, 100, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, 1 << 40, None]
    args[at] = value
    assert lib.omniattn_tree_verify(*args) == code


def test_keep_refuses_bad_arguments():
    lib = oa.load_library()
    g = _gqa(num_queries=3)
    good = [ctypes.byref(g), 4, *[GOOD] * 8, None]
    for at, value in ((0, None), (1, -1), (2, None), (3, None), (4, None), (5, None), (6, None), (6, GOOD + 8), (7, None), (7, GOOD + 4), (8, None), (9, None)):
        assert lib.omniattn_gqa_keep(*(good[:at] + [value] + good[at + 1:])) == -1, (at, value)
    for change, code in ((dict(batch=0), -1), (dict(head_dim=32), -2), (dict(scale_tokens=8), -2), (dict(page_table_stride=2), -1), (dict(num_pages=1 << 24), -2), (dict(batch=1 << 30), -2),
                         (dict(batch=1 << 23), -2)):
        h = _gqa(**dict(dict(num_queries=3), **change))
        assert lib.omniattn_gqa_keep(ctypes.byref(h), 4, *[GOOD] * 8, None) == code, change
    assert lib.omniattn_gqa_keep(ctypes.byref(g), 0, *[GOOD] * 8, None) == 0
    empty = _gqa(num_queries=0)
    assert lib.omniattn_gqa_keep(ctypes.byref(empty), 4, *[GOOD] * 8, None) == 0


def test_truncate_refuses_bad_arguments():
    lib = oa.load_library()
    t = oa.Table(batch=2, page_size=128, max_pages_per_seq=4, max_tokens=0, page_table_stride=4, num_pages=100)
    spread = [GOOD * (i + 1) for i in range(7)]
    for i in range(7):
        assert lib.omniattn_table_truncate(ctypes.byref(t), *(spread[:i] + [None] + spread[i + 1:]), None) == -1
    assert lib.omniattn_table_truncate(ctypes.byref(t), *(spread[:5] + [spread[0] + 4] + spread[6:]), None) == -1
    assert lib.omniattn_table_truncate(None, *spread, None) == -1
    for change, code in ((dict(batch=0), -1), (dict(page_size=64), -2), (dict(num_pages=0), -1), (dict(page_table_stride=3), -1)):
        fields = dict(dict(batch=2, page_size=128, max_pages_per_seq=4, max_tokens=0, page_table_stride=4, num_pages=100), **change)
        assert lib.omniattn_table_truncate(ctypes.byref(oa.Table(**fields)), *spread, None) == code


def _refused(call, *args, **kw):
    with pytest.raises(oa.OmniAttnError) as e:
        call(*args, **kw)
    assert e.value.code == -1


def test_the_binding_refuses_what_is_no_cuda_tensor():
    i = torch.zeros(4, dtype=torch.int32)
    f = torch.zeros(4)
    cache, scales = torch.zeros((2, 1, PAGE, 64), dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros((2, 1, 2))
    _refused(oa.omniattn_tree_masks, i, i, None, torch.zeros(4, dtype=torch.int64))
    _refused(oa.omniattn_table_truncate, i, i, i.view(4, 1), i, i[:1], i, i[:1])
    _refused(oa.omniattn_gqa_keep, i, i, None, i.view(4, 1), cache, cache, scales, scales)
    _refused(oa.omniattn_gqa_tree, torch.zeros((4, 1, 64), dtype=torch.bfloat16), cache, cache, scales, scales, i.view(4, 1), i, None, torch.zeros(4, dtype=torch.int64),
             torch.zeros((4, 1, 64)), torch.zeros((4, 1)), None, sink=0, window=1, softmax_scale=1.0)
    _refused(oa.omniattn_tree_verify, torch.zeros((4, 9)), None, i, i, None, f, torch.zeros((4, 2)), i, i, f, i, None)
    with pytest.raises(oa.OmniAttnError) as e:
        oa.gqa_tree(torch.zeros((4, 1, 64), dtype=torch.bfloat16), cache, cache, scales, scales, i.view(4, 1), i, torch.zeros(4, dtype=torch.int64), 0, 1, 1.0)
    assert e.value.code == -4


@gpu
def test_the_binding_refuses_wrong_tensors():
    def check(call, good, bad):
        call(*good)
        for at, value in bad:
            _refused(call, *(good[:at] + [value] + good[at + 1:]))
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
    f = lambda *shape: torch.zeros(shape, device="cuda")
    m = torch.zeros(4, dtype=torch.int64, device="cuda")
    check(oa.omniattn_tree_masks, [i(4), i(2) + 9, i(3), m, i(4)], [(0, i(4).long()), (1, i(4)), (2, i(2)), (3, m[:3]), (3, m.int()), (4, i(3)), (4, f(4))])
    ws = torch.empty(oa.omniattn_tree_verify_workspace_bytes(4, 9), dtype=torch.uint8, device="cuda")
    check(oa.omniattn_tree_verify, [f(4, 9), f(4, 9), i(4), i(4), i(3), f(2), f(4, 2), i(4), i(4), f(4), i(2), ws],
          [(0, f(4, 9).half()), (0, f(36)), (0, f(9, 4).t()), (1, f(4, 8)), (1, f(4, 9).bfloat16()), (2, i(3)), (3, i(5)), (4, i(4)), (5, f(3)), (6, f(4)), (7, i(3)), (8, f(4)), (9, i(4)),
           (9, f(3)), (10, i(3))])
    with pytest.raises(oa.OmniAttnError):
        oa.omniattn_tree_verify(f(4, 9), None, i(4), i(4), i(3), f(2), f(4, 2), i(4), i(4), f(4), i(2), ws[:100])
    cache, scales = torch.zeros((2, 3, 1, PAGE, 64), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), f(2, 3, 1, 2)
    check(oa.omniattn_gqa_keep, [i(4) - 1, i(2) + 9, i(3), i(2, 1), cache, cache.clone(), scales, scales.clone()],
          [(0, i(4).long()), (1, i(2).float()), (2, i(4)), (3, i(3, 1)), (4, cache[0]), (4, cache[:, :2]), (6, scales[0]), (6, f(2, 3, 1, 3)), (6, f(2, 3, 2, 2)), (6, f(1, 3, 1, 2)),
           (4, cache[None])])
    check(oa.omniattn_table_truncate, [i(2), i(2), i(2, 3), i(5), i(1), i(2), i(1)], [(0, f(2)), (1, i(3)), (2, i(3, 3)), (2, i(3, 2).t()), (3, f(5)), (4, i(2)), (5, i(3)), (6, i(2))])


def test_workspaces_of_verification():
    assert oa.omniattn_tree_verify_workspace_bytes(0, 100) == 0
    sizes = [oa.omniattn_tree_verify_workspace_bytes(n, 5000) for n in (1, 2, 50, 51)]
    assert sizes == sorted(sizes) and sizes[0] >= 3 * 24
    with pytest.raises(oa.OmniAttnError):
        oa.omniattn_tree_verify_workspace_bytes(5, 0)


# ------------------------------------------------------------------------------------------------ the kernel for many rows of width 128

MANY = 16 * 256   # steps of 32 rows and a page from which on it is taken, with 256 compute units


def _width(batch, kv_heads, rows):
    """Columns of a table that make a call large enough for it, whatever the lengths are."""
    return -(-MANY // (batch * kv_heads * -(-rows // 32)))


class Wide(Problem):
    """A table with as many columns as the rule asks for."""

    def run(self, *args, **kw):
        batch, tokens, (q_heads, kv_heads) = len(self.lens), len(self.sets), (self.q.shape[1], self.codes.shape[2])
        rows = -(-tokens // batch) * (q_heads // kv_heads)
        assert rows > 32
        short = self.table
        self.table = [r + [0] * max(0, _width(batch, kv_heads, rows) - len(r)) for r in short]
        try:
            return super().run(*args, **kw)
        finally:
            self.table = short


@gpu
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("sink,window", [(0, 10 ** 6), (4, 60), (130, 0), (0, 1), (3, 200)])
@pytest.mark.parametrize("group,kv_heads,news", [(1, 2, [64, 40, 33, 64]), (3, 1, [64, 1, 12, 0, 22]), (4, 2, [8, 9, 16, 17, 24, 25, 32, 33]), (16, 1, [3, 2, 64])])
def test_many_rows(group, kv_heads, news, sink, window, out_dtype):
    """Blocks of 32, 64, 96 and 128 rows, and several of them."""
    rng = random.Random(group + sink)
    lens = [n + rng.choice([0, 5, 100, 128 - n // 2, 300, 450]) for n in news]
    for each, kind in ((32, "any"), (128, "chain")):
        Wide(lens, sets_of(rng, news, kind), group * kv_heads, kv_heads, 128, each, sink, window, seed=group).check(out_dtype)


@gpu
@pytest.mark.parametrize("sink,window", [(0, 10 ** 6), (4, 40), (0, 3)])
def test_many_rows_any_sets(sink, window):
    rng = random.Random(window)
    news = [40, 64, 90, 1, 2, 64]
    lens = [n + t for n, t in zip(news, (300, 100, 30, 0, 128, -50))]
    Wide(lens, sets_of(rng, news, "random"), 4, 2, 128, 64, sink, window, seed=3).check()
    Wide(lens, sets_of(rng, news, "random"), 7, 1, 128, 32, sink, window, seed=4).check(torch.float32)


@gpu
@pytest.mark.parametrize("group,nodes", [(1, 40), (4, 12), (4, 40), (8, 64)])
def test_many_rows_long_texts_are_split_and_joined(group, nodes):
    rng = random.Random(nodes)
    Wide([9000, 77 + nodes, 5003, 64], sets_of(rng, [nodes, 2, nodes, 64]), group, 1, 128, 64, 0, 10 ** 6, seed=5, poison=False).check(torch.float32)


@gpu
@pytest.mark.parametrize("sink,window,group,each", [(0, 100, 8, 32), (4, 100, 8, 64), (0, 20, 13, 128), (7, 0, 8, 64)])
def test_many_rows_of_many_short_requests(sink, window, group, each):
    """Blocks of few pages, which are not cut."""
    rng = random.Random(window)
    news = [rng.choice([0, 1, 12, 25, 33, 40, 64, 70]) for _ in range(200)]
    lens = [n + rng.randint(0, 260) for n in news]
    pages = min(max(-(-n // PAGE) for n in lens), -(-sink // PAGE) + -(-window // PAGE) + 1)
    assert pages <= 3 and 200 * 2 * pages * -(-(-(-sum(news) // 200) * group) // 32) >= MANY
    Problem(lens, sets_of(rng, news), 2 * group, 2, 128, each, sink, window, seed=window)._check(torch.float32)


@gpu
def test_many_rows_of_negative_and_zero_softmax_scale():
    rng = random.Random(8)
    news = [20, 12, 33]
    p = Wide([n + 200 for n in news], sets_of(rng, news), 8, 2, 128, 64, 0, 150, seed=8)
    for p.scale in (-0.1, 0.0, -1e-30, 3.0):
        p.check(torch.float32)


@gpu
@pytest.mark.parametrize("group", [1, 8])
def test_many_rows_nan_reaches_only_the_queries_that_see_it(group):
    rng = random.Random(6)
    n = 40 if group == 1 else 12
    sets = ref.masks(tree_of(rng, n), 0)[0]
    L, window = 200 + n, 150
    for slot, in_k in ((200 + 5, False), (200 + 5, True), (200, False), (200 + 1 - 150, False), (200 + 2 - 150, True)):
        p = Wide([L], [sets], 2 * group, 2, 128, 64, 0, window, seed=7, poison=False)
        clean, clean_lse = p.run()
        p.codes.view(torch.uint8)[0 if in_k else 1, p.table[0][slot // PAGE], 1, slot % PAGE, 3] = 0xff
        out, lse = p.run()
        for t, m in enumerate(sets):
            hit = slot in ref.kept(m, L, n, 0, window)
            mine, others = slice(group, 2 * group), slice(0, group)
            assert torch.equal(out[t, others], clean[t, others])
            assert torch.isnan(lse[t, mine]).all() == (hit and in_k) and (in_k or torch.equal(lse, clean_lse))
            bad = torch.isnan(out[t, mine])
            if not hit:
                assert not bad.any() and torch.equal(out[t, mine], clean[t, mine])
            else:
                assert bad.all() if in_k else (bad[:, 3].all() and bad.sum() == group)


@gpu
def test_many_rows_bf16_results_are_the_fp32_results_rounded_and_the_same_every_time():
    rng = random.Random(9)
    news = [rng.randint(5, 40) for _ in range(60)]
    p = Wide([n + rng.randint(0, 900) for n in news], sets_of(rng, news), 8, 2, 128, 32, 4, 300, seed=9)
    out, lse = p.run(fill=0x7f)
    wide, wide_lse = p.run(torch.float32, pad=2)
    assert torch.equal(out, wide.bfloat16()) and torch.equal(lse, wide_lse)
    again = p.run(fill=0)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


# ------------------------------------------------------------------------------------------------ large caches, long texts

@gpu
@pytest.mark.parametrize("nodes", [2, 40])
def test_a_cache_of_more_than_four_gigabytes(nodes):
    """Pages at the end of a pool whose byte offsets pass 32 bits give what the same pages at its beginning give."""
    heads, dim, each = 8, 128, 64
    pages = 2 ** 32 // (heads * PAGE * dim) + 40
    k, v = (torch.zeros((pages, heads, PAGE, dim), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = torch.zeros((2, pages, heads, PAGE // each), device="cuda")
    p = (Wide if nodes > 32 else Problem)([300], sets_of(random.Random(1), [nodes]), 8, 8, dim, each, 0, 10 ** 6, seed=71, poison=False)
    want, want_lse = p.check(torch.float32)
    ws = torch.empty(oa.omniattn_gqa_workspace_bytes(1, nodes, 8, heads, dim), dtype=torch.uint8, device="cuda")
    for own in ([3, 1, 2], [pages - 1, pages - 30, pages - 2]):
        pick, was = torch.tensor(own, device="cuda"), torch.tensor(p.table[0], device="cuda")
        for cache, codes in ((k, p.codes[0]), (v, p.codes[1])):
            cache.view(torch.uint8)[pick] = codes.view(torch.uint8).cuda()[was]
        ks[pick], vs[pick] = p.scales[0].cuda()[was], p.scales[1].cuda()[was]
        out, lse = torch.empty_like(want), torch.empty_like(want_lse)
        table = ints([own + [0] * (max(3, _width(1, heads, nodes)) - 3 if nodes > 32 else 0)])
        oa.omniattn_gqa_tree(p.q.cuda(), k, v, ks, vs, table, ints([300]), None if nodes == 1 else ints([0, nodes]), longs(p.sets), out, lse, ws, sink=0, window=10 ** 6, softmax_scale=p.scale)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


@gpu
@pytest.mark.parametrize("sink,window", [(0, 2 ** 31 - 1), (2 ** 31 - 1, 0), (0, 2 ** 30 + 1000), (100, 2 ** 30 + 900), (0, 2 ** 30 - 100)])
@pytest.mark.parametrize("dim,q_heads", [(64, 1), (128, 1), (128, 11), (256, 3), (128, 40)])
def test_requests_of_more_than_2_30_tokens(dim, q_heads, sink, window):
    """The first page holds nearly all of the weight, one page of zero keys and values stands for all the others, the nodes' among them.  Logits are 40 and 0,
    so the 2^30 others are 2^30 exp(-40) / 128 = 4e-11 of the sum, and what the rounding of their own sum does is far below the tolerance: 128 weights
    and their sum (2^-22, 2^-24 each), logits of 40 (2^-20 for the products, the factor and exp2)."""
    length, nodes = 2 ** 30 + 1000, 3
    table = torch.zeros((1, -(-length // PAGE)), dtype=torch.int32, device="cuda")
    table[0, 0] = 1
    k, v = torch.zeros((2, 2, 1, PAGE, dim), dtype=torch.float32)
    k[1], v[1] = 1.0, (torch.arange(PAGE) % 5).float()[None, :, None]
    k, v = (t.to(torch.float8_e4m3fn).cuda() for t in (k, v))
    ones = torch.ones((2, 1, 2), device="cuda")
    q = torch.ones((nodes, q_heads, dim), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty((nodes, q_heads, dim), device="cuda"), torch.empty((nodes, q_heads), device="cuda")
    ws = torch.empty(oa.omniattn_gqa_workspace_bytes(1, nodes, q_heads, 1, dim), dtype=torch.uint8, device="cuda")
    oa.omniattn_gqa_tree(q, k, v, ones, ones, table, ints([length]), ints([0, nodes]), longs([1, 3, 5]), out, lse, ws, sink=sink, window=window, softmax_scale=40 / dim)
    for t, position in enumerate((length - nodes, length - nodes + 1, length - nodes + 1)):
        kept = [j for j in range(PAGE) if j < sink or j > position - window]
        if kept:
            want, want_lse = sum(j % 5 for j in kept) / len(kept), 40 + np.log(len(kept))
        else:
            want, want_lse = 0.0, np.log(window)
        assert np.abs(gref.as_double(lse[t]) - want_lse).max() <= 40 * 2.0 ** -20 + 128 * 2.0 ** -23 + (0 if kept else 1e-3)
        assert np.abs(gref.as_double(out[t]) - want).max() <= 4 * (40 * 2.0 ** -20 + 128 * 2.0 ** -22)
