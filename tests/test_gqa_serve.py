"""The three calls of a grouped-query step together, as a server makes them: requests come, grow, finish and give their pages back."""
import numpy as np
import pytest
import torch

import gqa_reference as ref
from paper_2511_22481_amd.gqa_serve import PAGE, Pool, serve

gpu = pytest.mark.gpu
PROMPTS, ANSWERS = [300, 1, 40, 129, 256], [7, 9, 0, 3, 5]
Q_HEADS, HEADS, DIM, LAYERS, SINK, WINDOW = 6, 2, 64, 2, 4, 200


def _rows(step, buffer):
    """The same rows for the same step, whichever way it is called."""
    g = torch.Generator().manual_seed(step)
    full = torch.randn((LAYERS, 500, Q_HEADS + 2 * HEADS, DIM), generator=g).bfloat16()
    buffer.copy_(full[:, :buffer.shape[1]])


def _run(graph):
    pool = Pool(len(PROMPTS), LAYERS, 12, HEADS, DIM, 5)
    seen = []

    def observe(step, news, out, lse):
        n = sum(news)
        seen.append((news, out[:, :n].clone(), lse[:, :n].clone(), pool.lens.tolist(), pool.table.tolist(), pool.q_start.tolist(),
                     [t.cpu() for t in (pool.k, pool.v, pool.k_scales, pool.v_scales)]))
    return serve(pool, PROMPTS, ANSWERS, Q_HEADS, SINK, WINDOW, _rows, chunk=128, graph=graph, observe=observe), seen


@gpu
def test_steps_follow_the_reference_and_pages_come_back():
    what, seen = _run(graph=False)
    assert what["tokens"] == sum(PROMPTS) + sum(ANSWERS) and what["free_at_the_end"] == 12 and what["pages"] <= 12
    grown = [0] * len(PROMPTS)
    for step, (news, out, lse, lens, table, q_start, (k, v, ks, vs)) in enumerate(seen):
        grown = [g + n for g, n in zip(grown, news)]
        assert all(length == g for length, g, n in zip(lens, grown, news) if n)  # (finished requests have given theirs up)
        full = torch.empty((LAYERS, sum(news), Q_HEADS + 2 * HEADS, DIM), dtype=torch.bfloat16)
        _rows(step, full)
        for i in range(LAYERS):
            cache = [ref.as_double(t[i]) for t in (k, v, ks, vs)]
            want, want_lse, tol, lse_tol = ref.attend_bf16(ref.as_double(full[i, :, :Q_HEADS]), *cache, table, lens, q_start, SINK, WINDOW, DIM ** -0.5)
            assert (np.abs(ref.as_double(out[i]) - want) <= tol).all(), (step, i)
            assert (np.abs(ref.as_double(lse[i]) - want_lse) <= lse_tol).all(), (step, i)


@gpu
def test_replayed_steps_are_the_called_ones():
    called, replayed = _run(graph=False)[1], _run(graph=True)[1]
    assert len(called) == len(replayed)
    for step, (a, b) in enumerate(zip(called, replayed)):
        assert a[0] == b[0] and a[3:6] == b[3:6], step
        assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2]), step


def test_a_pool_has_room_for_every_scale():
    pool = Pool(3, 2, 4, 1, 64, 2, scale_tokens=32, device="cpu")
    assert pool.k.shape == (2, 4, 1, PAGE, 64) and pool.k_scales.shape == (2, 4, 1, 4) and pool.free.tolist() == [0, 1, 2, 3]


def _check_step(step, pool, news, granted, out, lse, before):
    """A step against the reference: lengths, and the results of the requests whose tokens are in the cache."""
    lens, table, q_start = pool.lens.tolist(), pool.table.tolist(), pool.q_start.tolist()
    assert lens == [a + n for a, n in zip(before, granted)], step
    assert q_start == [int(x) for x in np.cumsum([0] + news)], step
    full = torch.empty((LAYERS, sum(news), Q_HEADS + 2 * HEADS, DIM), dtype=torch.bfloat16)
    _rows(step, full)
    rows = np.repeat([n == g for n, g in zip(news, granted)], news)
    for i in range(LAYERS):
        cache = [ref.as_double(t[i]) for t in (pool.k, pool.v, pool.k_scales, pool.v_scales)]
        want, want_lse, tol, lse_tol = ref.attend_bf16(ref.as_double(full[i, :, :Q_HEADS]), *cache, table, lens, q_start, SINK, WINDOW, DIM ** -0.5)
        assert (np.abs(ref.as_double(out[i, :sum(news)]) - want) <= tol)[rows].all(), (step, i)
        assert (np.abs(ref.as_double(lse[i, :sum(news)]) - want_lse) <= lse_tol)[rows].all(), (step, i)


@gpu
@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("prompts,answers", [([128, 0], [0, 5]), ([300, 0, 0, 7], [2, 4, 1, 0]), ([0, 0, 0], [3, 1, 2])])
def test_requests_without_a_prompt(prompts, answers, graph):
    """Their first tokens come beside whole chunks of the others: the buffers have room for all of them."""
    pool = Pool(len(prompts), LAYERS, 8, HEADS, DIM, 3)
    grown = [0] * len(prompts)

    def observe(step, news, out, lse):
        before = [n if any(w) else 0 for n, w in zip(grown, left)]   # (finished requests have given theirs up)
        _check_step(step, pool, news, news, out, lse, before)
        for b, n in enumerate(news):
            grown[b] += n
            left[b] = [max(0, left[b][0] - n), left[b][1] - max(0, n - left[b][0])]
    left = [[p, a] for p, a in zip(prompts, answers)]
    what = serve(pool, prompts, answers, Q_HEADS, SINK, WINDOW, _rows, chunk=128, graph=graph, observe=observe)
    assert grown == [p + a for p, a in zip(prompts, answers)] and what["tokens"] == sum(grown) and what["free_at_the_end"] == 8


@gpu
@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("pages", [5, 6, 8])
def test_a_small_pool_makes_requests_wait(pages, graph):
    """Fewer pages than the requests have together at the end: those that are refused bring their tokens again, and every token is served once."""
    pool = Pool(len(PROMPTS), LAYERS, pages, HEADS, DIM, 5)
    left, grown, refused = [[p, a] for p, a in zip(PROMPTS, ANSWERS)], [0] * len(PROMPTS), 0

    def observe(step, news, out, lse):
        nonlocal refused
        before = [n if any(w) else 0 for n, w in zip(grown, left)]
        granted = [n if now == old + n else 0 for n, old, now in zip(news, before, pool.lens.tolist())]
        refused += sum(n > g for n, g in zip(news, granted))
        _check_step(step, pool, news, granted, out, lse, before)
        for b, n in enumerate(granted):
            assert n <= (min(left[b][0], 128) or min(left[b][1], 1))
            grown[b] += n
            left[b] = [left[b][0] - n, left[b][1]] if left[b][0] else [0, left[b][1] - n]
    what = serve(pool, PROMPTS, ANSWERS, Q_HEADS, SINK, WINDOW, _rows, chunk=128, graph=graph, observe=observe)
    assert refused > 0 and grown == [p + a for p, a in zip(PROMPTS, ANSWERS)]
    assert what["tokens"] == sum(grown) and what["free_at_the_end"] == pages and what["pages"] <= pages


@gpu
@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("pages,columns,prompts,answers", [(2, 5, [300], [7]), (3, 5, [256, 256, 256], [0, 0, 0]), (12, 2, [200, 400], [5, 0]), (1, 1, [128], [1])])
def test_requests_that_can_never_be_served_are_reported(pages, columns, prompts, answers, graph):
    """A prompt longer than the pool, requests that hold each other's pages, a table with too few columns: an error, not a count of tokens."""
    pool = Pool(len(prompts), LAYERS, pages, HEADS, DIM, columns)
    with pytest.raises(RuntimeError, match="still to come"):
        serve(pool, prompts, answers, Q_HEADS, SINK, WINDOW, lambda step, buffer: buffer.normal_(), chunk=128, graph=graph)
    assert int(pool.free_count) == pages - int(((pool.lens + PAGE - 1) // PAGE).sum())
