"""Grouped-query layers over the paged 8-bit cache on the GPU: tables, append and attention against plain 64-bit
implementations (tests/gqa_reference.py)."""
import ctypes
import random

import numpy as np
import pytest
import torch

import gqa_reference as ref
import paper_2511_22481_amd as oa

PAGE = 128
gpu = pytest.mark.gpu


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def ints(values, device="cuda"):
    return torch.tensor(values, dtype=torch.int32, device=device)


# ------------------------------------------------------------------------------------------------ tables

def _tables(lens, news, width, free, count, max_tokens, in_place, extra_columns=0):
    """Runs extend on the GPU and the reference, compares everything."""
    batch = len(lens)
    rng = random.Random(len(lens) + count)
    table = [[rng.randrange(1 << 20) for _ in range(width)] for _ in range(batch)]
    want = ref.extend(lens, news, free, count, table, max_tokens)
    wide = torch.full((batch, width + extra_columns), -7, dtype=torch.int32, device="cuda")
    wide[:, :width] = ints(table)
    t = wide[:, :width]
    L, c = ints(lens), ints([count])
    L_out, c_out = (L, c) if in_place else (torch.full_like(L, -9), torch.full_like(c, -9))
    q_start = torch.full((batch + 1,), -9, dtype=torch.int32, device="cuda")
    slots = torch.full((max_tokens,), -9, dtype=torch.int32, device="cuda")
    oa.omniattn_table_extend(L, ints(news), ints(free), c, t, L_out, c_out, q_start, slots)
    assert t.tolist() == want[0]
    assert L_out.tolist() == want[1]
    assert c_out.tolist() == [want[2]]
    assert q_start.tolist() == want[3]
    assert slots.tolist() == want[4]
    assert extra_columns == 0 or bool((wide[:, width:] == -7).all())
    return want


@gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch,longest,new,seed", [
    (1, 0, 1, 0), (1, 300, 1, 1), (3, 130, 1, 2), (64, 5000, 1, 3), (64, 600, 200, 4), (65, 128, 2, 5), (1024, 500, 1, 6), (1025, 500, 1, 7),
    (1500, 300, 40, 8), (2500, 129, 3, 9), (7, 400, 3000, 10), (2, 0, 5000, 11)])
def test_extend(batch, longest, new, seed, in_place):
    rng = random.Random(seed)
    lens = [rng.choice([0, longest, rng.randint(0, longest), rng.randint(0, longest) // PAGE * PAGE]) for _ in range(batch)]
    news = [rng.choice([0, 1, new, rng.randint(0, new)]) for _ in range(batch)]
    width = max(1, max((a + b + PAGE - 1) // PAGE for a, b in zip(lens, news)))
    need = sum((a + b + PAGE - 1) // PAGE - (a + PAGE - 1) // PAGE for a, b in zip(lens, news))
    free = rng.sample(range(1 << 20), need + 5)
    _tables(lens, news, width, free, len(free), sum(news), in_place, extra_columns=seed % 3)
    # entries of slot_map behind the last token, a stack with nothing to spare, an empty one
    _tables(lens, news, width, free, need, sum(news) + 3000 * (seed % 2) + 1, in_place)
    _tables(lens, news, width, free, 0, sum(news), in_place)


@gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seed", range(6))
def test_extend_refuses_requests_that_do_not_fit(seed, in_place):
    """Rows of the table too short, negative lengths, tokens behind the slot map, a stack that runs out in the middle."""
    rng = random.Random(seed)
    batch = rng.choice([5, 70, 1300])
    lens = [rng.choice([-1, 0, 5, 127, 128, 500, 2 ** 31 - 1]) for _ in range(batch)]
    news = [rng.choice([-3, 0, 1, 1, 300, 700]) if seed % 2 else rng.choice([-1, 0, 1]) for _ in range(batch)]
    free = rng.sample(range(1 << 20), 400)
    total = sum(max(n, 0) for n in news)
    for count in (400, 17, 1):
        _tables(lens, news, 6, free, count, max(1, total - rng.randrange(1 + total // 2)), in_place)
    # the largest lengths: no sum wraps
    got = _tables([0, 1, 2], [2 ** 31 - 1, 1, 1], 6, free, 400, 10, in_place)[1] if seed == 0 and not in_place else None
    assert got is None or got == [0, 1, 2]


@gpu
@pytest.mark.parametrize("batch,seed", [(1, 0), (64, 1), (1500, 2)])
def test_release_gives_the_pages_back(batch, seed):
    rng = random.Random(seed)
    lens = [rng.choice([0, 1, 128, 129, rng.randint(0, 700)]) for _ in range(batch)]
    done = [rng.choice([0, 1, 7, -1, 0]) for _ in range(batch)]
    table = [[b * 10 + k for k in range(6)] for b in range(batch)]
    held = rng.sample(range(1 << 20, 1 << 21), 9)
    back = [table[b][k] for b in range(batch) if done[b] for k in range(-(-lens[b] // PAGE))]
    free = torch.full((9 + len(back) + 4,), -7, dtype=torch.int32, device="cuda")
    free[:9] = ints(held)
    L, c = ints(lens), ints([9])
    oa.omniattn_table_release(L, ints(done), ints(table), free, c)
    assert free.tolist() == held + back + [-7] * 4
    assert c.tolist() == [9 + len(back)]
    assert L.tolist() == [0 if d else n for n, d in zip(lens, done)]
    # released, then taken again: the last one back is the first one out
    if back:
        news = [1 if d else 0 for d in done]
        t = ints(table)
        q, s = torch.empty(batch + 1, dtype=torch.int32, device="cuda"), torch.empty(sum(news), dtype=torch.int32, device="cuda")
        need = sum(news)
        if need <= len(held) + len(back):
            oa.omniattn_table_extend(L, ints(news), free, c, t, L, c, q, s)
            stack = held + back
            assert [x // PAGE for x in s.tolist()] == stack[::-1][:need]


@gpu
def test_release_into_a_full_stack_stays_inside_it():
    free = ints([1, 2, 3, 4])
    L, c = ints([500, 300]), ints([2])
    guard = torch.full((8,), -7, dtype=torch.int32, device="cuda")
    guard[:4] = free
    oa.omniattn_table_release(L, ints([1, 1]), ints([[10, 11, 12, 13], [14, 15, 16, 17]]), guard[:4], c)
    assert guard.tolist() == [1, 2, 10, 11, -7, -7, -7, -7]
    assert c.tolist() == [4] and L.tolist() == [0, 0]


# ------------------------------------------------------------------------------------------------ append

def _cache(pages, heads, dim, each, seed):
    """Codes of every kind but NaN, scales that are powers of two."""
    g = _gen(seed)
    codes = torch.randint(0, 256, (2, pages, heads, PAGE, dim), generator=g, dtype=torch.uint8)
    codes[(codes & 0x7f) == 0x7f] = 0x3a
    scales = 2.0 ** torch.randint(-9, 3, (2, pages, heads, PAGE // each), generator=g).float()
    return codes.view(torch.float8_e4m3fn), scales


def _check_append(new, slots, codes, scales, got_codes, got_scales, what=""):
    want, want_scales = ref.as_double(codes), ref.as_double(scales)
    defined = ref.append(ref.as_double(new), slots, want, want_scales)
    got = ref.as_double(got_codes)
    assert np.array_equal(ref.as_double(got_scales), want_scales), what
    same = (got == want) | (np.isnan(got) & np.isnan(want)) | ~defined[..., None]
    assert same.all(), (what, np.argwhere(~same)[:5])


@gpu
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("each", [32, 64, 128])
@pytest.mark.parametrize("heads,runs,seed", [
    (1, [(0, 1)], 0),                                          # one token, first of its block
    (3, [(5, 1), (127, 1), (64, 1), (33, 1)], 1),              # single tokens inside blocks
    (2, [(0, 128)], 2),                                        # a whole page
    (2, [(1, 127), (100, 28), (31, 2), (63, 65)], 3),          # ragged runs over block borders
    (5, [(17, 300), (0, 1), (90, 38), (0, 129)], 4),           # over several pages, single ones between
])
def test_append(dim, each, heads, runs, seed):
    g = _gen(100 * seed + dim + each)
    pages = sum((a + n + PAGE - 1) // PAGE for a, n in runs) + 2
    order = torch.randperm(pages, generator=g).tolist()
    slots = []
    for a, n in runs:
        own = [order.pop() for _ in range((a + n + PAGE - 1) // PAGE)]
        slots += [own[i // PAGE] * PAGE + i % PAGE for i in range(a, a + n)]
    codes, scales = _cache(pages, heads, dim, each, seed)
    # rows of very different size: blocks' scales grow, stay, and become tiny; some rows are zeros
    new = torch.randn((2, len(slots), heads, dim), generator=g) * 2.0 ** torch.randint(-20, 8, (2, len(slots), heads, 1), generator=g).float()
    new[:, ::7] = 0
    new = new.bfloat16()
    k, v = codes.cuda()
    ks, vs = scales.cuda()
    gpu_new = new.cuda()
    for repeat in range(2):   # a second time on the same slots: nothing moves
        oa.omniattn_gqa_append(gpu_new[0], gpu_new[1], ints(slots), k, v, ks, vs)
        _check_append(new[0], slots, codes[0], scales[0], k, ks, f"k {repeat}")
        _check_append(new[1], slots, codes[1], scales[1], v, vs, f"v {repeat}")


@gpu
@pytest.mark.parametrize("dim,heads", [(64, 2), (128, 7), (256, 1)])
@pytest.mark.parametrize("each", [32, 128])
def test_append_single_tokens_beside_prompts(dim, heads, each):
    """A mixed step: hundreds of single tokens, pairs and threes, whole chunks between them, in the places of their blocks that the others leave."""
    rng = random.Random(dim + each)
    runs = [rng.choice([1] * 12 + [2, 3, 5, 9, 150]) for _ in range(400)]
    slots, pages = [], 0
    for n in runs:
        first = rng.choice([0, 1, 31, 32, 77, 126, 127])
        at = [pages * PAGE + first + i for i in range(n)]
        pages += (first + n + PAGE - 1) // PAGE
        slots += at
    codes, scales = _cache(pages, heads, dim, each, dim)
    new = torch.randn((2, len(slots), heads, dim), generator=_gen(dim)) * 2.0 ** torch.randint(-20, 8, (2, len(slots), heads, 1), generator=_gen(each)).float()
    new = new.bfloat16()
    k, v = codes.cuda()
    ks, vs = scales.cuda()
    on_gpu = new.cuda()
    oa.omniattn_gqa_append(on_gpu[0], on_gpu[1], ints(slots), k, v, ks, vs)
    _check_append(new[0], slots, codes[0], scales[0], k, ks)
    _check_append(new[1], slots, codes[1], scales[1], v, vs)


@gpu
def test_append_strided_rows_unknown_slots_and_special_numbers():
    """K and V as slices of one tensor, tokens without a slot among them, infinities, NaN, subnormal and the largest numbers."""
    g = _gen(5)
    heads, dim, each, pages = 3, 128, 32, 6
    slots = [0, 1, -1, 64, 40, 41, 42, -1, -1, 200, 201, 202, 203, 700, 3 * PAGE + 31, 3 * PAGE + 32, 6 * PAGE, 2 ** 31 - 1]
    fused = torch.randn((len(slots), 4 * heads, dim), generator=g)
    fused[4, :, 3] = float("inf")
    fused[5, :, 4] = float("nan")
    fused[6, :, 5] = -float("inf")
    fused[9] = 2.0 ** -130
    fused[10:13] = 0
    fused[13] = 3.3e38
    fused[14, :, :] = float("inf")
    fused = fused.bfloat16()
    codes, scales = _cache(pages, heads, dim, each, 6)
    k, v = codes.cuda()
    ks, vs = scales.cuda()
    on_gpu = fused.cuda()
    oa.omniattn_gqa_append(on_gpu[:, heads:2 * heads], on_gpu[:, 2 * heads:3 * heads], ints(slots), k, v, ks, vs)
    _check_append(fused[:, heads:2 * heads], slots, codes[0], scales[0], k, ks)
    _check_append(fused[:, 2 * heads:3 * heads], slots, codes[1], scales[1], v, vs)


@gpu
@pytest.mark.parametrize("each", [32, 128])
def test_append_token_by_token_is_near_one_call(each):
    """A block filled one token at a time, its scale growing on the way: every number within the rounding of the final scale (half a step,
    once for each time that the scale grew, and steps of subnormal codes are 2^-9 of the scale)."""
    g = _gen(9)
    rows = (torch.randn((2, PAGE, 2, 64), generator=g) * torch.linspace(0.01, 30, PAGE)[None, :, None, None]).bfloat16()
    k, v = torch.zeros((2, 1, 2, PAGE, 64), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    ks, vs = torch.full((2, 1, 2, PAGE // each), 77.0, device="cuda")
    on_gpu = rows.cuda()
    for i in range(PAGE):
        oa.omniattn_gqa_append(on_gpu[0, i:i + 1], on_gpu[1, i:i + 1], ints([i]), k, v, ks, vs)
    for got, s, x in ((k, ks, rows[0]), (v, vs, rows[1])):
        want = ref.as_double(x).transpose(1, 0, 2).reshape(2, PAGE // each, each, 64)
        scale = ref.as_double(s)[0][..., None, None]
        top = np.abs(want).max((2, 3), keepdims=True)
        assert np.array_equal(scale, 2.0 ** np.ceil(np.log2(top / 448)))
        value = ref.as_double(got)[0].reshape(want.shape) * scale
        # the scale grew at most 13 times (a factor of 3000 in the rows' size): each rounds subnormal codes once more
        assert (np.abs(value - want) <= np.abs(want) * 2.0 ** -4 + 13 * 2.0 ** -10 * scale).all()


# ------------------------------------------------------------------------------------------------ attention

class Problem:
    """A cache with shuffled pages, everything that no query keeps poisoned with NaN (codes and scales of blocks without kept tokens)."""

    def __init__(self, lens, news, q_heads, kv_heads, dim, each, sink, window, seed=0, spread=1.0, poison=True, extra_pages=3, q_stride=0):
        g = _gen(seed)
        self.lens, self.q_start, self.sink, self.window = lens, [0] + list(np.cumsum(news)), sink, window
        self.q_start = [int(x) for x in self.q_start]
        self.scale = dim ** -0.5
        used = [max(0, -(-n // PAGE)) for n in lens]
        pages, width = sum(used) + extra_pages, max(1, max(used, default=1))
        order = torch.randperm(pages, generator=g).tolist()
        self.table = [[order.pop() if c < u else 0 for c in range(width)] for u in used]
        self.codes, self.scales = _cache(pages, kv_heads, dim, each, seed)
        # values of order one whatever the block's scale
        x = torch.randn((2, pages, kv_heads, PAGE, dim), generator=g)
        self.scales *= torch.rand(self.scales.shape, generator=g) + 0.5       # (not only powers of two)
        blocks = x.view(2, pages, kv_heads, PAGE // each, each, dim)
        top = blocks.abs().amax((-1, -2), keepdim=True)
        self.scales = torch.where(torch.rand(self.scales.shape, generator=g) < 0.1, self.scales, top[..., 0, 0] / 448)
        self.codes = (blocks / self.scales[..., None, None]).clamp(-448, 448).view(x.shape).to(torch.float8_e4m3fn)
        tokens = self.q_start[-1]
        self.q = (torch.randn((tokens, q_heads, dim), generator=g) * spread).bfloat16()
        if poison:
            kept = np.zeros((pages, PAGE), dtype=bool)
            for b, L in enumerate(lens):
                n = news[b]
                for t in range(n):
                    reach = L - n + t + 1
                    for j in list(range(min(sink, max(reach, 0)))) + list(range(max(0, reach - window), max(reach, 0))):
                        kept[self.table[b][j // PAGE], j % PAGE] = True
            gone = torch.from_numpy(~kept)
            raw = self.codes.view(torch.uint8)
            raw[:] = torch.where(gone[None, :, None, :, None], torch.tensor(0x7f, dtype=torch.uint8), raw)
            empty = gone.view(pages, PAGE // each, each).all(-1)
            self.scales = torch.where(empty[None, :, None, :], torch.tensor(float("nan")), self.scales)
        self.q_pad = q_stride

    def run(self, out_dtype, q_start=True, workspace_fill=None):
        k, v = self.codes.cuda()
        ks, vs = self.scales.cuda()
        q = self.q.cuda()
        if self.q_pad:
            wide = torch.full((q.shape[0], q.shape[1] + self.q_pad, q.shape[2]), float("nan"), dtype=q.dtype, device="cuda")
            wide[:, :q.shape[1]] = q
            q = wide[:, :q.shape[1]]
        out = torch.full(self.q.shape, float("nan"), dtype=out_dtype, device="cuda")
        lse = torch.full(self.q.shape[:2], float("nan"), dtype=torch.float32, device="cuda")
        size = oa.omniattn_gqa_workspace_bytes(len(self.lens), max(1, q.shape[0]), q.shape[1], k.shape[1], q.shape[2])
        # (whatever a workspace holds at the start must not matter)
        ws = torch.full((size,), 0xff if workspace_fill is None else workspace_fill, dtype=torch.uint8, device="cuda")
        oa.omniattn_gqa_decode(q, k, v, ks, vs, ints(self.table), ints(self.lens), ints(self.q_start) if q_start else None, out, lse, ws,
                               sink=self.sink, window=self.window, softmax_scale=self.scale)
        torch.cuda.synchronize()
        return out, lse

    def check(self, out_dtype=torch.bfloat16, **kw):
        out, lse = self.run(out_dtype, **kw)
        fn = ref.attend_fp32 if out_dtype == torch.float32 else ref.attend_bf16
        k, v = ref.as_double(self.codes)
        ks, vs = ref.as_double(self.scales)
        want, want_lse, tol, lse_tol = fn(ref.as_double(self.q), k, v, ks, vs, self.table, self.lens, self.q_start, self.sink, self.window, self.scale)
        got, got_lse = ref.as_double(out), ref.as_double(lse)
        assert np.array_equal(np.isfinite(got_lse), np.isfinite(want_lse))
        assert np.array_equal(got_lse == -np.inf, want_lse == -np.inf)
        fine = np.isfinite(want_lse)
        assert (np.abs(got_lse[fine] - want_lse[fine]) <= lse_tol[fine]).all()
        err = np.abs(got - want)
        assert (err <= tol).all(), (np.argwhere(~(err <= tol))[:5], np.nanmax(err / np.maximum(tol, 1e-300)))
        return out, lse


LENGTHS = [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 700]


@gpu
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,q_heads,kv_heads,each", [(64, 4, 4, 32), (64, 6, 2, 64), (128, 8, 2, 32), (128, 5, 1, 128), (128, 14, 2, 64), (256, 3, 1, 64), (256, 16, 2, 128)])
def test_lengths_one_query(dim, q_heads, kv_heads, each, out_dtype):
    lens = LENGTHS + [0, 1500]
    p = Problem(lens, [1] * len(lens), q_heads, kv_heads, dim, each, 0, 4096, seed=dim + q_heads)
    p.lens[-2] = 0
    p.check(out_dtype)


@gpu
@pytest.mark.parametrize("sink,window", [(0, 0), (0, 1), (1, 0), (4, 100), (128, 128), (130, 300), (64, 5000), (5000, 0), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_kept_sets(sink, window, dim):
    lens = [1, 4, 100, 128, 400, 433, 900]
    p = Problem(lens, [1] * len(lens), 4, 2, dim, 32, min(sink, 10 ** 6), min(window, 10 ** 6), seed=sink % 1000 + window % 1000)
    p.sink, p.window = sink, window
    p.check()


@gpu
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("sink,window", [(0, 10 ** 6), (4, 100), (130, 20), (0, 1), (3, 0)])
@pytest.mark.parametrize("dim,q_heads,kv_heads", [(64, 7, 1), (128, 3, 3), (128, 16, 2), (256, 10, 2)])
def test_several_queries(dim, q_heads, kv_heads, sink, window, out_dtype):
    """Ragged numbers of new tokens, none and a whole prompt among them: causal, blocks of 16, 32 and 64 rows and what is left of them."""
    for most in (2, 5, 30):
        lens = [most, 129, 300, 31, 64 + most, 513, 5]
        news = [most, 2, 0, 1, most, min(most, 3), 5 if most >= 5 else 1]
        p = Problem(lens, news, q_heads, kv_heads, dim, 32, sink, window, seed=most + dim)
        p.check(out_dtype)


@gpu
@pytest.mark.parametrize("each", [32, 64, 128])
def test_a_chunk_longer_than_a_block_of_rows(each):
    """More query rows than one block takes: a prompt's second chunk."""
    Problem([300, 77], [90, 77], 4, 1, 128, each, 0, 10 ** 6, seed=each).check()
    Problem([300, 77], [90, 77], 4, 2, 64, each, 8, 50, seed=each).check(torch.float32)


@gpu
@pytest.mark.parametrize("batch,length,q_heads,kv_heads,dim", [(1, 40000, 8, 2, 128), (2, 9000, 3, 1, 64), (1, 20000, 2, 2, 256), (3, 5000, 16, 1, 128)])
def test_long_requests_are_split_and_joined(batch, length, q_heads, kv_heads, dim):
    lens = [length - 77 * b for b in range(batch)]
    p = Problem(lens, [1] * batch, q_heads, kv_heads, dim, 64, 0, 10 ** 6, seed=3, poison=False)
    p.check()
    p.check(torch.float32, workspace_fill=0)


@gpu
def test_many_requests_fill_every_work_group_several_times():
    rng = random.Random(4)
    lens = [rng.choice([0, 1, 50, 128, 200, 400]) for _ in range(700)]
    p = Problem(lens, [min(1, n) for n in lens], 2, 2, 64, 32, 0, 10 ** 6, seed=4, poison=False)
    p.check()
    lens = [rng.choice([1, 50, 128, 200, 400]) for _ in range(300)]
    Problem(lens, [min(n, rng.choice([1, 1, 3])) for n in lens], 4, 1, 128, 128, 16, 100, seed=5, poison=False).check()


@gpu
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group,most,sink,window", [(1, 1, 4, 150), (1, 3, 0, 10 ** 6), (3, 3, 2, 40), (16, 1, 0, 1), (1, 20, 130, 60)])
def test_many_short_requests_of_narrow_heads(group, most, sink, window, out_dtype):
    """2048 blocks and more, of one wave each: empty ones, parts of a page, blocks cut between waves, requests of more rows than a block."""
    rng = random.Random(group + most)
    lens = [rng.choice([0, 1, 31, 32, 33, 65, 128, 129, 200, 290]) for _ in range(256)]
    news = [min(n, rng.choice([0, 1, most]) if most > 1 else 1) for n in lens]
    Problem(lens, news, 8 * group, 8, 64, 32, sink, window, seed=group, extra_pages=0).check(out_dtype)


@gpu
@pytest.mark.parametrize("dim,q_heads,kv_heads,most", [(64, 3, 3, 1), (64, 8, 8, 1), (128, 8, 2, 1), (128, 4, 1, 8), (128, 8, 1, 12), (256, 2, 1, 1), (256, 8, 1, 5)])
@pytest.mark.parametrize("columns,sink,window", [(1, 0, 10 ** 6), (2, 0, 10 ** 6), (4, 0, 10 ** 6), (12, 4, 128), (12, 0, 200)])
def test_blocks_of_few_pages_are_not_cut(dim, q_heads, kv_heads, most, columns, sink, window):
    """Narrow tables and small windows: from one request to many more blocks than work groups, empty ones among them."""
    rng = random.Random(columns + dim)
    for batch in (1, 7, 300):
        lens = [min(rng.choice([0, 1, 127, 128, 129, 400, 1500]), columns * PAGE) for _ in range(batch)]
        news = [min(n, rng.randint(0, most) if most > 1 else 1) for n in lens]
        news[0] = min(lens[0], most)
        if sum(news) == 0:
            lens[0], news[0] = 100, most
        p = Problem(lens, news, q_heads, kv_heads, dim, 64, sink, window, seed=batch, poison=batch < 100, extra_pages=1)
        p.table = [row[:columns] + [0] * (columns - len(row)) for row in p.table]
        p.check(torch.float32 if columns == 2 else torch.bfloat16)


@gpu
@pytest.mark.parametrize("dim,q_heads,kv_heads", [(64, 32, 2), (128, 48, 2), (64, 120, 120)])
def test_prompts_of_many_rows(dim, q_heads, kv_heads):
    """More than 65536 rows, of which a few are in parts."""
    lens, news = [700, 0, 130, 690], [700, 0, 65, 690]
    assert sum(news) * q_heads > 65536 or q_heads == 32
    if q_heads == 32:
        lens, news = lens + [700], news + [700]
    Problem(lens, news, q_heads, kv_heads, dim, 64, 4, 200, seed=dim + q_heads, poison=False).check()


@gpu
@pytest.mark.parametrize("dim,q_heads,kv_heads", [(64, 2, 2), (128, 8, 2), (128, 5, 1), (256, 4, 1)])
def test_more_queries_than_tokens(dim, q_heads, kv_heads):
    """Requests whose new tokens found no pages: queries before the first token keep nothing."""
    Problem([0, 3, 200, 40, 0], [40, 20, 20, 41, 1], q_heads, kv_heads, dim, 64, 2, 30, seed=dim).check()
    Problem([0, 3], [1, 4], q_heads, kv_heads, dim, 64, 0, 10 ** 6, seed=dim).check(torch.float32)


@gpu
@pytest.mark.parametrize("dim,kv_heads", [(64, 8), (128, 8), (256, 16)])
def test_tables_for_very_long_requests(dim, kv_heads):
    """Columns for 2^29 tokens: units of work are counted in 64 bits.  The same blocks, the same bits as with a table of few columns."""
    lens = [random.Random(b).choice([0, 1, 100, 700, 1500]) for b in range(70)]
    p = Problem(lens, [min(1, n) for n in lens], kv_heads, kv_heads, dim, 64, 0, 10 ** 6, seed=dim, poison=False)
    want, want_lse = p.check()
    k, v = p.codes.cuda()
    ks, vs = p.scales.cuda()
    table = torch.zeros((70, 2 ** 22), dtype=torch.int32, device="cuda")
    table[:, :len(p.table[0])] = ints(p.table)
    out, lse = oa.gqa_decode(p.q.cuda(), k, v, ks, vs, table, ints(p.lens), 0, 2 ** 29, p.scale, q_start=ints(p.q_start))
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@gpu
@pytest.mark.parametrize("group,most,sink,window", [(1, 1, 0, 10 ** 6), (3, 5, 0, 10 ** 6), (2, 2, 100, 1500)])
def test_a_few_long_requests_among_many_short_ones(group, most, sink, window):
    """Waves that work alone through blocks of 64 quarters of pages and, with several queries, one more."""
    rng = random.Random(most)
    lens = [rng.choice([0, 1, 1, 5, 40]) for _ in range(256)]
    for b in (0, 7, 100, 101, 255):
        lens[b] = rng.choice([2048, 2047, 2017, 1900])
    lens[7] = 2048
    Problem(lens, [min(n, most) for n in lens], 8 * group, 8, 64, 128, sink, window, seed=most, poison=False).check()


@gpu
def test_nan_among_many_short_requests():
    lens, news = [150] * 256, [3] * 256
    clean = Problem(lens, news, 8, 8, 64, 64, 1, 30, seed=9, poison=False)
    p = Problem(lens, news, 8, 8, 64, 64, 1, 30, seed=9, poison=False)
    for b, at, head, column in ((3, 149, 0, 63), (3, 148, 7, 0), (100, 119, 4, 17), (255, 0, 5, 40), (200, 60, 2, 9)):
        p.codes[1].view(torch.uint8)[p.table[b][at // PAGE], head, at % PAGE, column] = 0x7f
    (want, want_lse), (out, lse) = clean.run(torch.float32), p.run(torch.float32)
    bad = torch.zeros(want.shape, dtype=torch.bool)
    bad[3 * 3 + 2, 0, 63] = True           # token 149: the last query's
    bad[3 * 3 + 1:3 * 3 + 3, 7, 0] = True  # token 148: the last two queries'
    bad[100 * 3:100 * 3 + 2, 4, 17] = True  # token 119 has left the last query's window
    bad[255 * 3:255 * 3 + 3, 5, 40] = True  # token 0 is a sink
    assert torch.equal(out.isnan().cpu(), bad) and torch.equal(lse, want_lse)
    assert torch.equal(out.cpu()[~bad], want.cpu()[~bad])


@gpu
def test_peaked_and_shifted_logits():
    """Large logits that grow along the request (the reference is raised again and again) and shrink (it never is)."""
    for sign in (1, -1):
        p = Problem([1000, 1000], [1, 1], 4, 1, 128, 32, 0, 10 ** 6, seed=8, poison=False, spread=6.0)
        ramp = torch.linspace(0, 30, 1000)
        for b in range(2):
            direction = p.q[b, 0].float() / p.q[b, 0].float().norm()
            for j in range(1000):
                page = p.table[b][j // PAGE]
                p.scales[0, page, :, (j % PAGE) // 32] = 0.05
                row = torch.randn(128, generator=_gen(j)) + sign * ramp[j] * direction * 0.2
                p.codes[0].view(torch.uint8)[page, 0, j % PAGE] = (row / 0.05).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        p.check(torch.float32)
        p.check()


@gpu
def test_value_scales_far_apart():
    """Neighbouring blocks' scales differ by 2^40, and zero: each block counts with its own."""
    p = Problem([500, 130], [1, 2], 4, 2, 128, 32, 0, 10 ** 6, seed=11, poison=False)
    g = _gen(12)
    p.scales[1] *= 2.0 ** torch.randint(-40, 1, p.scales[1].shape, generator=g).float()
    p.scales[1][torch.rand(p.scales[1].shape, generator=g) < 0.2] = 0
    p.scales[0][torch.rand(p.scales[0].shape, generator=g) < 0.2] = 0
    p.check(torch.float32)


@gpu
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_nan_reaches_only_the_queries_that_keep_it(dim):
    """A cached NaN in a K or a V row among several queries' tokens: queries before it are untouched, later ones that keep it are NaN."""
    base = Problem([200], [6], 4, 1, dim, 32, 2, 20, seed=dim, poison=False)
    clean, clean_lse = base.run(torch.float32)
    for at in (197, 194, 180, 1, 100):
        for which in (0, 1):
            p = Problem([200], [6], 4, 1, dim, 32, 2, 20, seed=dim, poison=False)
            p.codes[which].view(torch.uint8)[p.table[0][at // PAGE], 0, at % PAGE, 3] = 0xff if at % 2 else 0x7f
            out, lse = p.run(torch.float32)
            for t in range(6):
                reach = 195 + t
                keeps = at < reach and (at < 2 or at >= reach - 20)
                if not keeps:
                    assert torch.equal(out[t], clean[t]) and torch.equal(lse[t], clean_lse[t])
                elif which == 0:
                    assert bool(out[t].isnan().all()) and bool(lse[t].isnan().all())
                else:
                    assert bool(out[t, :, 3].isnan().all()) and torch.equal(lse[t], clean_lse[t])
                    rest = [c for c in range(dim) if c != 3]
                    assert torch.equal(out[t][:, rest], clean[t][:, rest])


@gpu
def test_nan_and_infinite_queries_stay_in_their_rows():
    p = Problem([300, 40], [2, 1], 4, 2, 128, 64, 0, 10 ** 6, seed=21)
    clean, clean_lse = p.run(torch.bfloat16)
    p.q[1, 2, 5] = float("nan")
    p.q[2, 0, 7] = float("inf")
    out, lse = p.run(torch.bfloat16)
    bad = torch.zeros((3, 4), dtype=torch.bool)
    bad[1, 2] = bad[2, 0] = True
    assert bool(out.cpu()[bad].isnan().all()) and bool(lse.cpu()[bad].isnan().all())
    assert torch.equal(out.cpu()[~bad], clean.cpu()[~bad]) and torch.equal(lse.cpu()[~bad], clean_lse.cpu()[~bad])


@gpu
def test_scales_of_the_softmax():
    for scale in (0.0, -0.3, 1e-30, 2.0):
        p = Problem([200, 77], [1, 3], 4, 2, 64, 32, 0, 10 ** 6, seed=31)
        p.scale = scale
        p.check(torch.float32)


@gpu
def test_strides_and_one_query_without_q_start():
    p = Problem([200, 1, 77, 500], [1] * 4, 4, 2, 128, 32, 4, 100, seed=41, q_stride=3)
    a, la = p.check()
    b, lb = p.run(torch.bfloat16, q_start=False)
    assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and torch.equal(la, lb)
    # a page table that is a part of a wider one
    k, v = p.codes.cuda()
    ks, vs = p.scales.cuda()
    wide = torch.full((4, 9), 2 ** 30, dtype=torch.int32, device="cuda")
    width = len(p.table[0])
    wide[:, 2:2 + width] = ints(p.table)
    out, lse = torch.empty_like(a), torch.empty_like(la)
    ws = torch.empty(oa.omniattn_gqa_workspace_bytes(4, 4, 4, 2, 128), dtype=torch.uint8, device="cuda")
    oa.omniattn_gqa_decode(p.q.cuda(), k, v, ks, vs, wide[:, 2:2 + width], ints(p.lens), None, out, lse, ws, sink=4, window=100, softmax_scale=p.scale)
    assert torch.equal(a.view(torch.int16), out.view(torch.int16)) and torch.equal(la, lse)


@gpu
def test_rows_of_no_request_are_left_alone():
    """More query rows than q_start covers (a captured step with room for more): the rest keeps its contents."""
    p = Problem([200, 300], [2, 1], 4, 2, 128, 64, 0, 10 ** 6, seed=51)
    want, want_lse = p.run(torch.bfloat16)
    p.q = torch.cat([p.q, torch.full((5, 4, 128), float("nan"), dtype=torch.bfloat16)])
    out, lse = p.run(torch.bfloat16)
    assert torch.equal(out[:3], want) and torch.equal(lse[:3], want_lse)
    assert bool(out[3:].isnan().all()) and bool(lse[3:].isnan().all())


@gpu
def test_same_inputs_same_bits():
    p = Problem([5000, 77, 900], [1, 4, 2], 8, 2, 128, 64, 0, 10 ** 6, seed=61, poison=False)
    a = [p.run(torch.float32, workspace_fill=f) for f in (0, 0xff, 0x7f)]
    for out, lse in a[1:]:
        assert torch.equal(out, a[0][0]) and torch.equal(lse, a[0][1])


@gpu
def test_a_cache_of_more_than_four_gigabytes():
    """Pages at the end of a pool whose byte offsets pass 32 bits, for append and attention."""
    heads, dim, each = 8, 128, 64
    pages = 2 ** 32 // (heads * PAGE * dim) + 40
    k = torch.zeros((pages, heads, PAGE, dim), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v = torch.zeros((pages, heads, PAGE, dim), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    ks, vs = torch.zeros((2, pages, heads, PAGE // each), device="cuda")
    g = _gen(71)
    small = Problem([300], [1], 16, 8, dim, each, 0, 10 ** 6, seed=71, poison=False)
    new = torch.randn((2, 300, heads, dim), generator=g).bfloat16()
    results = []
    for own in ([3, 1, 2], [pages - 1, pages - 30, pages - 2]):
        slots = ints([own[i // PAGE] * PAGE + i % PAGE for i in range(300)])
        oa.omniattn_gqa_append(new[0].cuda(), new[1].cuda(), slots, k, v, ks, vs)
        results.append(oa.gqa_decode(small.q.cuda(), k, v, ks, vs, ints([own]), ints([300]), 0, 1000, dim ** -0.5, out_dtype=torch.float32))
        pick = torch.tensor(own, device="cuda")
        small.codes = torch.stack([k.view(torch.uint8)[pick], v.view(torch.uint8)[pick]]).cpu().view(torch.float8_e4m3fn)
        small.scales = torch.stack([ks[pick], vs[pick]]).cpu()
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
    small.table, small.lens = [[0, 1, 2]], [300]
    out, lse = small.check(torch.float32)
    assert torch.equal(out, results[0][0])


@gpu
def test_other_streams():
    """Calls on a stream that is not the current one, ordered by the caller."""
    p = Problem([2000, 77], [1, 1], 8, 2, 128, 64, 0, 10 ** 6, seed=81, poison=False)
    want, want_lse = p.run(torch.bfloat16)
    k, v = p.codes.cuda()
    ks, vs = p.scales.cuda()
    q, table, lens, start = p.q.cuda(), ints(p.table), ints(p.lens), ints(p.q_start)
    out, lse = torch.zeros_like(want), torch.zeros_like(want_lse)
    ws = torch.empty(oa.omniattn_gqa_workspace_bytes(2, 2, 8, 2, 128), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    oa.omniattn_gqa_decode(q, k, v, ks, vs, table, lens, start, out, lse, ws, sink=0, window=10 ** 6, softmax_scale=p.scale, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@gpu
def test_a_captured_step_follows_the_growing_requests():
    """extend, append and decode in one graph, replayed while requests grow over page borders; eager work between the replays.  Every
    replay equals the eager calls."""
    batch, heads, q_heads, dim, each, pages, width = 5, 2, 6, 128, 64, 40, 6
    g = _gen(91)

    def fresh():
        k, v = torch.zeros((2, pages, heads, PAGE, dim), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        ks, vs = torch.zeros((2, pages, heads, PAGE // each), device="cuda")
        return dict(k=k, v=v, ks=ks, vs=vs, lens=ints([0] * batch), free=torch.arange(pages, dtype=torch.int32, device="cuda"), count=ints([pages]),
                    table=torch.zeros((batch, width), dtype=torch.int32, device="cuda"), start=torch.zeros(batch + 1, dtype=torch.int32, device="cuda"),
                    slots=torch.zeros(400, dtype=torch.int32, device="cuda"), new=torch.zeros((400, q_heads + 2 * heads, dim), dtype=torch.bfloat16, device="cuda"),
                    news=ints([1] * batch), out=torch.zeros((400, q_heads, dim), dtype=torch.bfloat16, device="cuda"),
                    lse=torch.zeros((400, q_heads), device="cuda"), ws=torch.empty(oa.omniattn_gqa_workspace_bytes(batch, 400, q_heads, heads, dim), dtype=torch.uint8, device="cuda"))

    def step(s):
        oa.omniattn_table_extend(s["lens"], s["news"], s["free"], s["count"], s["table"], s["lens"], s["count"], s["start"], s["slots"])
        q, k, v = s["new"][:, :q_heads], s["new"][:, q_heads:q_heads + heads], s["new"][:, q_heads + heads:]
        oa.omniattn_gqa_append(k, v, s["slots"], s["k"], s["v"], s["ks"], s["vs"])
        oa.omniattn_gqa_decode(q, s["k"], s["v"], s["ks"], s["vs"], s["table"], s["lens"], s["start"], s["out"], s["lse"], s["ws"], sink=4, window=150, softmax_scale=0.1)

    eager, replayed = fresh(), fresh()
    first = {n: t.clone() for n, t in replayed.items()}
    step(replayed)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(replayed)
    for n, t in first.items():
        replayed[n].copy_(t) if t.dtype != torch.float8_e4m3fn else replayed[n].view(torch.uint8).copy_(t.view(torch.uint8))
    for news in ([100, 1, 128, 57, 3], [1] * 5, [1, 1, 1, 30, 1], [50, 0, 1, 1, 200], [1] * 5, [0, 0, 0, 0, 1]):
        new = torch.randn((400, q_heads + 2 * heads, dim), generator=g).bfloat16()
        for s in (eager, replayed):
            s["news"].copy_(ints(news))
            s["new"].copy_(new)
        step(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        total = sum(news)
        assert eager["lens"].tolist() == replayed["lens"].tolist()
        for name in ("table", "slots", "start", "count"):
            assert torch.equal(eager[name], replayed[name]), name
        assert torch.equal(eager["out"][:total], replayed["out"][:total]) and torch.equal(eager["lse"][:total], replayed["lse"][:total])
        # and against the reference on the cache as it is
        k, v = ref.as_double(eager["k"]), ref.as_double(eager["v"])
        want, want_lse, tol, lse_tol = ref.attend_bf16(ref.as_double(new[:total, :q_heads]), k, v, ref.as_double(eager["ks"]), ref.as_double(eager["vs"]),
                                                       eager["table"].tolist(), eager["lens"].tolist(), eager["start"].tolist(), 4, 150, 0.1)
        assert (np.abs(ref.as_double(eager["out"][:total]) - want) <= tol).all()
        assert (np.abs(ref.as_double(eager["lse"][:total]) - want_lse) <= lse_tol).all()


# ------------------------------------------------------------------------------------------------ refusals

def _gqa(**kw):
    fields = dict(batch=2, num_queries=2, num_q_heads=4, num_kv_heads=2, head_dim=128, page_size=128, scale_tokens=64, max_pages_per_seq=4,
                  page_table_stride=4, num_pages=9, sink=0, window=100, softmax_scale=0.1, out_dtype=oa.BF16)
    fields.update(kw)
    return oa.Gqa(**fields)


GOOD = 0x1000   # an address that is aligned and never read: the calls below are refused before


@pytest.mark.parametrize("change,code", [
    (dict(batch=0), -1), (dict(num_q_heads=3), -1), (dict(num_kv_heads=0), -1), (dict(num_q_heads=0), -1), (dict(max_pages_per_seq=0), -1), (dict(num_pages=0), -1),
    (dict(num_queries=-1), -1), (dict(sink=-1), -1), (dict(window=-1), -1), (dict(page_table_stride=3), -1), (dict(softmax_scale=float("nan")), -1),
    (dict(softmax_scale=float("inf")), -1), (dict(page_size=64), -2), (dict(head_dim=96), -2), (dict(scale_tokens=16), -2), (dict(scale_tokens=0), -2),
    (dict(out_dtype=oa.FP8_E4M3), -2), (dict(num_pages=1 << 24), -2), (dict(num_queries=1 << 30), -2), (dict(max_pages_per_seq=1 << 24, page_table_stride=1 << 25), -2)])
def test_decode_refuses_bad_problems(change, code):
    lib = oa.load_library()
    g = _gqa(**change)
    rc = lib.omniattn_gqa_decode(ctypes.byref(g), GOOD, 512, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, 1 << 40, None)
    assert rc == code


@pytest.mark.parametrize("at,value", [(1, None), (1, GOOD + 2), (2, 511), (2, 504), (3, None), (3, GOOD + 8), (4, None), (4, GOOD + 1), (5, None), (6, None), (7, None), (8, None),
                                      (9, None), (10, None), (10, GOOD + 4), (11, None)])
def test_decode_refuses_bad_arguments(at, value):
    lib = oa.load_library()
    g = _gqa(num_queries=3)   # (so that a missing q_start is refused too: two requests, three queries)
    args = [ctypes.byref(g), GOOD, 512, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, 1 << 40, None]
    args[at] = value
    assert lib.omniattn_gqa_decode(*args) == -1
    assert lib.omniattn_gqa_decode(*([None] + args[1:])) == -1


@pytest.mark.parametrize("at,value,code", [
    (1, -1, -1), (2, None, -1), (2, GOOD + 2, -1), (3, 252, -1), (3, 248, -1), (4, None, -1), (5, 257, -1), (6, None, -1), (7, None, -1), (8, None, -1), (8, GOOD + 8, -1), (9, None, -1),
    (10, None, -1), (1, 2 ** 31 - 1, -2)])
def test_append_refuses_bad_arguments(at, value, code):
    lib = oa.load_library()
    g = _gqa()
    args = [ctypes.byref(g), 5, GOOD, 256, GOOD, 256, GOOD, GOOD, GOOD, GOOD, GOOD, None]
    args[at] = value
    assert lib.omniattn_gqa_append(*args) == code
    assert lib.omniattn_gqa_append(*([None] + args[1:])) == -1


def test_append_of_no_tokens_does_nothing():
    lib = oa.load_library()
    g = _gqa()
    assert lib.omniattn_gqa_append(ctypes.byref(g), 0, None, 256, None, 256, None, None, None, None, None, None) == 0


@pytest.mark.parametrize("change,code", [(dict(batch=0), -1), (dict(page_size=16), -2), (dict(max_pages_per_seq=0), -1), (dict(max_tokens=-1), -1), (dict(page_table_stride=3), -1),
                                         (dict(num_pages=0), -1), (dict(num_pages=1 << 24), -2)])
def test_tables_refuse_bad_problems(change, code):
    lib = oa.load_library()
    fields = dict(batch=2, page_size=128, max_pages_per_seq=4, max_tokens=10, page_table_stride=4, num_pages=100)
    fields.update(change)
    t = oa.Table(**fields)
    spread = [GOOD * (i + 1) for i in range(9)]
    assert lib.omniattn_table_extend(ctypes.byref(t), *spread, None) == code
    assert lib.omniattn_table_release(ctypes.byref(t), *spread[:5], None) == code


def test_tables_refuse_missing_and_overlapping_arrays():
    lib = oa.load_library()
    t = oa.Table(batch=2, page_size=128, max_pages_per_seq=4, max_tokens=10, page_table_stride=4, num_pages=100)
    spread = [GOOD * (i + 1) for i in range(9)]
    for i in range(9):
        assert lib.omniattn_table_extend(ctypes.byref(t), *(spread[:i] + [None] + spread[i + 1:]), None) == -1
    for i in range(5):
        assert lib.omniattn_table_release(ctypes.byref(t), *(spread[:5][:i] + [None] + spread[:5][i + 1:]), None) == -1
    # seq_lens_out one entry behind seq_lens
    assert lib.omniattn_table_extend(ctypes.byref(t), *(spread[:5] + [spread[0] + 4] + spread[6:]), None) == -1
    assert lib.omniattn_table_extend(None, *spread, None) == -1


def test_the_binding_refuses_what_is_no_cuda_tensor():
    """Before anything reaches the library: host tensors, other types and sizes, and things that are no tensors."""
    n = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    good = [n(3), n(3), n(9), n(1), n(3, 4), n(3), n(1), n(4), n(5)]
    for bad in [good] + [good[:i] + [x] + good[i + 1:] for i in range(9) for x in (None, 7, [1], torch.zeros(3), n(2, 2).t())]:
        with pytest.raises(oa.OmniAttnError) as e:
            oa.omniattn_table_extend(*bad)
        assert e.value.code == -1
        with pytest.raises(oa.OmniAttnError):
            oa.omniattn_table_release(bad[0], bad[1], bad[4], bad[2], bad[3])
    codes, scales = torch.zeros((2, 1, 128, 64), dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros((2, 1, 2))
    rows = torch.zeros((3, 1, 64), dtype=torch.bfloat16)
    for cache in ([codes, codes, scales, scales], [codes[:1], codes, scales, scales], [codes.view(torch.uint8), codes, scales, scales], [codes, codes, None, scales],
                  [codes, codes, scales[:, :, :0], scales[:, :, :0]]):
        with pytest.raises(oa.OmniAttnError):
            oa.omniattn_gqa_append(rows, rows, n(3), *cache)
        with pytest.raises(oa.OmniAttnError):
            oa.omniattn_gqa_decode(rows, *cache, n(3, 4), n(3), None, rows, torch.zeros((3, 1)), None, sink=0, window=1, softmax_scale=1.0)
    with pytest.raises(TypeError):
        oa.omniattn_table_extend(*good[:8])


@gpu
def test_the_binding_refuses_numbers_out_of_range():
    p = Problem([200], [1], 4, 2, 128, 64, 0, 1000, seed=1)
    k, v = p.codes.cuda()
    ks, vs = p.scales.cuda()
    out, lse = torch.empty((1, 4, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((1, 4), device="cuda")
    ws = torch.empty(oa.omniattn_gqa_workspace_bytes(1, 1, 4, 2, 128), dtype=torch.uint8, device="cuda")
    call = lambda **kw: oa.omniattn_gqa_decode(p.q.cuda(), k, v, ks, vs, ints(p.table), ints(p.lens), None, out, lse, ws, **{**dict(sink=0, window=1000, softmax_scale=0.1), **kw})
    call()
    for bad in (dict(sink=2 ** 31), dict(window=-1), dict(window=2 ** 70), dict(sink=-2 ** 40), dict(softmax_scale=float("nan"))):
        with pytest.raises(oa.OmniAttnError) as e:
            call(**bad)
        assert e.value.code == -1
    for bad in (dict(sink=1.5), dict(window=None), dict(softmax_scale="1")):
        with pytest.raises(TypeError):
            call(**bad)
    call(stream=torch.cuda.current_stream())
    torch.cuda.synchronize()


@gpu
def test_workspace_is_checked():
    p = Problem([200], [1], 4, 2, 128, 64, 0, 1000, seed=1)
    k, v = p.codes.cuda()
    ks, vs = p.scales.cuda()
    out, lse = torch.empty((1, 4, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((1, 4), device="cuda")
    size = oa.omniattn_gqa_workspace_bytes(1, 1, 4, 2, 128)
    for ws in (None, torch.empty(size - 1, dtype=torch.uint8, device="cuda"), torch.empty(size + 256, dtype=torch.uint8, device="cuda")[16:]):
        with pytest.raises(oa.OmniAttnError) as e:
            oa.omniattn_gqa_decode(p.q.cuda(), k, v, ks, vs, ints(p.table), ints(p.lens), None, out, lse, ws, sink=0, window=1000, softmax_scale=0.1)
        assert e.value.code == -3


@gpu
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("batch,q_heads,kv_heads", [(1, 1, 1), (200, 12, 12), (64, 32, 4), (300, 40, 2), (2048, 1, 1)])
def test_a_workspace_is_enough_for_fewer_queries(batch, q_heads, kv_heads, dim):
    sizes = [oa.omniattn_gqa_workspace_bytes(batch, n, q_heads, kv_heads, dim) for n in (1, batch, 3 * batch, 10 * batch, 17 * batch, 40 * batch, 100 * batch)]
    assert sizes == sorted(sizes)


@gpu
def test_a_server_keeps_one_workspace():
    """Prompts and single tokens in turn, with the workspace of the most tokens."""
    batch, heads, dim = 200, 12, 64
    ws = torch.full((oa.omniattn_gqa_workspace_bytes(batch, 10 * batch, heads, heads, dim),), 0xff, dtype=torch.uint8, device="cuda")
    for news in ([1] * batch, [10] * batch, [30] * 60 + [1] * 140):
        p = Problem([n + 20 for n in news], news, heads, heads, dim, 64, 4, 30, seed=len(news) + news[0], extra_pages=0)
        want, want_lse = p.run(torch.bfloat16)
        k, v = p.codes.cuda()
        ks, vs = p.scales.cuda()
        out, lse = torch.empty_like(want), torch.empty_like(want_lse)
        oa.omniattn_gqa_decode(p.q.cuda(), k, v, ks, vs, ints(p.table), ints(p.lens), ints(p.q_start), out, lse, ws, sink=4, window=30, softmax_scale=p.scale)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


@gpu
def test_the_binding_refuses_wrong_tensors():
    p = Problem([200], [1], 4, 2, 128, 64, 0, 1000, seed=1)
    k, v = p.codes.cuda()
    ks, vs = p.scales.cuda()
    q, table, lens = p.q.cuda(), ints(p.table), ints(p.lens)
    for bad in (dict(q=q.float()), dict(q=q[:, :, ::2]), dict(k=k.view(torch.uint8)), dict(v=v[:, :1]), dict(ks=ks.double()), dict(vs=vs[:, :, :1]), dict(table=table.long()),
                dict(table=table.t()[:1].t() if table.shape[1] > 1 else table.long()), dict(lens=lens.long()), dict(lens=lens.cpu())):
        a = dict(q=q, k=k, v=v, ks=ks, vs=vs, table=table, lens=lens)
        a.update(bad)
        if bad.get("table") is not None and bad["table"].dtype == torch.int32:
            continue
        with pytest.raises(oa.OmniAttnError):
            oa.gqa_decode(a["q"], a["k"], a["v"], a["ks"], a["vs"], a["table"], a["lens"], 0, 1000, 0.1)
    with pytest.raises(oa.OmniAttnError):
        oa.gqa_decode(p.q, k, v, ks, vs, table, lens, 0, 1000, 0.1)
    with pytest.raises(oa.OmniAttnError):
        oa.omniattn_gqa_append(q[:, :2], q[:, :2], ints([1, 2]), k, v, ks, vs)


@gpu
@pytest.mark.parametrize("dim,q_heads,kv_heads,batch,longest,most,window", [
    (64, 8, 2, 5, 3000, 1, 10 ** 6), (128, 8, 2, 5, 3000, 1, 10 ** 6), (256, 8, 2, 5, 3000, 1, 10 ** 6),      # blocks of 16 rows, cut and joined
    (64, 8, 2, 3, 900, 7, 10 ** 6), (128, 8, 2, 3, 900, 7, 10 ** 6),                                          # of 32
    (64, 16, 2, 3, 900, 9, 10 ** 6), (128, 16, 2, 3, 900, 9, 10 ** 6), (256, 16, 2, 3, 900, 9, 10 ** 6),      # of 64
    (64, 8, 8, 256, 300, 1, 10 ** 6),                                                                         # a wave to a block
    (128, 8, 2, 5, 3000, 1, 100)])                                                                            # not cut
def test_bf16_results_are_the_fp32_results_rounded(dim, q_heads, kv_heads, batch, longest, most, window):
    """Both come from the same sums in fp32, and only the last rounding differs: equal, not only near."""
    lens = [random.Random(b).randint(most, longest) for b in range(batch)]
    p = Problem(lens, [most] * batch, q_heads, kv_heads, dim, 64, 4, window, seed=dim + most, poison=False)
    (want, want_lse), (got, got_lse) = p.run(torch.float32), p.run(torch.bfloat16)
    assert torch.equal(got, want.bfloat16()) and torch.equal(got_lse, want_lse)


@gpu
@pytest.mark.parametrize("sink,window", [(0, 2 ** 31 - 1), (2 ** 31 - 1, 0), (0, 2 ** 30 + 1000), (100, 2 ** 30 + 900), (0, 2 ** 30 - 100)])
@pytest.mark.parametrize("dim,q_heads", [(64, 1), (128, 1), (128, 40)])
def test_requests_of_more_than_2_30_tokens(dim, q_heads, sink, window):
    """The first page holds nearly all of the weight, one page of zero keys and values stands for all the others.  Logits are 40 and 0, so the 2^30 others are
    2^30 exp(-40) / 128 = 4e-11 of the sum, and what the rounding of their own sum does is far below the tolerance: 128 weights and their sum (2^-22, 2^-24
    each), logits of 40 (2^-20 for the products, the factor and exp2)."""
    length = 2 ** 30 + 1000
    columns = -(-length // PAGE)
    table = torch.zeros((1, columns), dtype=torch.int32, device="cuda")
    table[0, 0] = 1
    k, v = torch.zeros((2, 2, 1, PAGE, dim), dtype=torch.float32)
    k[1], v[1] = 1.0, (torch.arange(PAGE) % 5).float()[None, :, None]
    k, v = (t.to(torch.float8_e4m3fn).cuda() for t in (k, v))
    ones = torch.ones((2, 1, 2), device="cuda")
    q = torch.ones((1, q_heads, dim), dtype=torch.bfloat16, device="cuda")
    out, lse = oa.gqa_decode(q, k, v, ones, ones, table, ints([length]), sink, window, 40 / dim, out_dtype=torch.float32)
    kept = [j for j in range(PAGE) if j < sink or j >= length - window]
    if kept:
        want, want_lse = sum(j % 5 for j in kept) / len(kept), 40 + np.log(len(kept))
    else:
        want, want_lse = 0.0, np.log(window)
    assert np.abs(ref.as_double(lse) - want_lse).max() <= 40 * 2.0 ** -20 + 128 * 2.0 ** -23 + (0 if kept else 1e-3)
    assert np.abs(ref.as_double(out) - want).max() <= 4 * (40 * 2.0 ** -20 + 128 * 2.0 ** -22)


@gpu
@pytest.mark.parametrize("batch,columns", [(1, 4), (3, 1), (1, 1)])
def test_tables_of_one_row_or_one_column_whatever_their_strides(batch, columns):
    """A stride that no element is reached by may be any number: a column seen as the only row, a row seen as the only column."""
    lens = [columns * PAGE - 9 - b for b in range(batch)]
    p = Problem(lens, [1] * batch, 4, 2, 128, 64, 0, 10 ** 6, seed=batch)
    (want, want_lse), (k, v), (ks, vs) = p.run(torch.bfloat16), p.codes.cuda(), p.scales.cuda()
    table = ints(p.table)
    odd = torch.full((columns, batch), 7, dtype=torch.int32, device="cuda").t().copy_(table)   # strides (1, batch)
    wide = torch.full((batch, 2 * columns), 7, dtype=torch.int32, device="cuda")[:, ::2]         # strides (2 columns, 2)
    tables = [odd] + ([wide.copy_(table)] if columns == 1 else [])
    assert all(t.shape == table.shape and torch.equal(t, table) for t in tables)
    for t in tables:
        out, lse = oa.gqa_decode(p.q.cuda(), k, v, ks, vs, t, ints(p.lens), 0, 10 ** 6, p.scale)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        before = [n - 1 for n in lens]
        free, count, q_start, slots = ints([50, 51, 52]), ints([3]), torch.empty(batch + 1, dtype=torch.int32, device="cuda"), torch.empty(batch, dtype=torch.int32, device="cuda")
        got = torch.empty(batch, dtype=torch.int32, device="cuda")
        oa.omniattn_table_extend(ints(before), ints([1] * batch), free, count, t, got, torch.empty_like(count), q_start, slots)
        assert got.tolist() == lens and slots.tolist() == [p.table[b][n // PAGE] * PAGE + n % PAGE for b, n in enumerate(before)]
        oa.omniattn_table_release(got, ints([1] * batch), t, torch.empty(batch * columns, dtype=torch.int32, device="cuda"), ints([0]))
        assert got.tolist() == [0] * batch


@gpu
def test_the_binding_refuses_wrong_tables():
    """int32 tables that would be read out of their rows: columns apart, too many or too few rows, rows that overlap, other numbers of dimensions."""
    p = Problem([200, 77], [1, 1], 4, 2, 128, 64, 0, 1000, seed=1)
    k, v = p.codes.cuda()
    ks, vs = p.scales.cuda()
    q, lens = p.q.cuda(), ints(p.lens)
    columns = len(p.table[0])
    assert columns == 2
    good = torch.full((4, 2 * columns), 1, dtype=torch.int32, device="cuda")
    good[:2, :columns] = ints(p.table)
    bad = [good[:2, ::2], good[:3, :columns], good[:1, :columns], good[0, :columns], good[:2, None, :columns], good[:columns, :2].t(), good[:1, :columns].expand(2, columns),
           torch.as_strided(good, (2, columns), (1, 1)), good[:2, :0]]
    for t in bad:
        with pytest.raises(oa.OmniAttnError) as e:
            oa.gqa_decode(q, k, v, ks, vs, t, lens, 0, 1000, 0.1)
        assert e.value.code == -1, t.shape
        n = torch.zeros(3, dtype=torch.int32, device="cuda")
        with pytest.raises(oa.OmniAttnError) as e:
            oa.omniattn_table_extend(lens, lens, ints([1]), ints([1]), t, lens, ints([1]), n, n)
        assert e.value.code == -1
        with pytest.raises(oa.OmniAttnError) as e:
            oa.omniattn_table_release(lens, lens, t, ints([1]), ints([1]))
        assert e.value.code == -1
    want = oa.gqa_decode(q, k, v, ks, vs, ints(p.table), lens, 0, 1000, 0.1)
    got = oa.gqa_decode(q, k, v, ks, vs, good[:2, :columns], lens, 0, 1000, 0.1)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and lens.tolist() == p.lens
