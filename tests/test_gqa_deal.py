"""How grouped-query attention deals out its work, on the host: the kernels' own code (csrc/gqa_deal.h) compiled for the CPU under the sanitizers,
for calls of any size (CPU only)."""
import os
import random
import subprocess

import pytest

from test_sanitizers import ENV, ROOT, SAN, _build

SHAPES = [(16, 2, 128), (32, 2, 128), (64, 2, 128), (16, 4, 32)]   # rows of a block, cost of its start, tokens of a unit


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("deal") / "deal")
    _build(["g++", "-std=c++17", *SAN, os.path.join(ROOT, "tests", "sanitize", "deal_driver.cpp"), "-o", exe])

    def run(calls):
        """calls: (rows, start, grain), KV heads, group, sink, window, uncut, shares, [(tokens, queries), ...]"""
        lines = [" ".join(map(str, [*shape, heads, group, sink, window, int(uncut), shares, len(requests), *(x for r in requests for x in r)]))
                 for shape, heads, group, sink, window, uncut, shares, requests in calls]
        res = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, env=ENV)
        assert res.returncode == 0, (res.stdout[-500:], res.stderr[-2000:])
        assert res.stdout.strip() == f"ok {len(calls)}"
    return run


def test_ordinary_calls(driver):
    rng = random.Random(1)
    calls = []
    for i in range(400):
        batch = rng.choice([1, 2, 7, 60])
        lens = [rng.choice([0, 1, 127, 128, 129, rng.randint(0, 6000)]) for _ in range(batch)]
        requests = [(n, rng.choice([0, 1, min(n, 5), min(n, rng.randint(0, 300)), 3])) for n in lens]
        calls.append((SHAPES[i % 4], rng.choice([1, 2, 7]), rng.choice([1, 3, 8, 16, 100]), *rng.choice([(0, 10 ** 6), (4, 100), (0, 0), (130, 700), (5000, 0)]), i % 3 == 0,
                      rng.choice([1, 2, 17, 256, 512, 4096]), requests))
    driver(calls)


@pytest.mark.parametrize("shape,heads,group,shares,requests", [
    (SHAPES[2], 32, 4, 256, [(2 ** 20, 2 ** 20)]),                          # 8.6e9 units, 2.7e8 a head
    (SHAPES[2], 8, 8, 256, [(1_200_000, 1_200_000)]),                       # 5.6e9
    (SHAPES[0], 64, 1, 512, [(500_000, 500_000)]),                          # 3.9e9: from 2^31 to 2^32
    (SHAPES[2], 2, 16, 256, [(2 ** 27, 2 ** 20)]),                          # 2.7e11 a head: more than 32 bits by itself
    (SHAPES[1], 8, 8, 512, [(700, 1)] * 100 + [(1_200_000, 1_200_000), (0, 0), (5, 5)] + [(900_000, 600_000)]),
    (SHAPES[2], 8, 8, 256, [(9, 1)] * 600 + [(1_300_000, 1_300_000)]),      # (more requests than threads)
])
def test_prompts_of_more_units_than_32_bits(driver, shape, heads, group, shares, requests):
    driver([(shape, heads, group, 0, 2 ** 30, False, shares, requests)])


@pytest.mark.parametrize("shape", SHAPES[:3])
def test_windows_and_requests_of_nearly_2_31_tokens(driver, shape):
    """The longest table and whatever keeps all of it; more queries than tokens beside it."""
    most = 2 ** 31 - 128
    for sink, window in ((0, most), (most, 0), (most, most), (5, most - 1), (2 ** 30, 2 ** 30)):
        driver([(shape, 2, 1, sink, window, False, 256, [(most, 64), (3, 70), (most - 77, 1), (0, 5)])])
