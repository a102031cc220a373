"""How tree attention deals out its work, on the host: the kernels' own code compiled for the CPU under the sanitizers (CPU only)."""
import os
import random
import subprocess

import pytest

from test_sanitizers import ENV, ROOT, SAN, _build


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("deal") / "tree_deal")
    _build(["g++", "-std=c++17", *SAN, os.path.join(ROOT, "tests", "sanitize", "tree_deal_driver.cpp"), "-o", exe])

    def run(calls):
        """calls: rows of a block, KV heads, group, sink, window, shares, [(tokens, nodes), ...]"""
        lines = [" ".join(map(str, [*head, len(requests), *(x for r in requests for x in r)])) for *head, requests in calls]
        res = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, env=ENV)
        assert res.returncode == 0, (res.stdout[-500:], res.stderr[-2000:])
        assert res.stdout.strip() == f"ok {len(calls)}"
    return run


def test_ordinary_calls(driver):
    rng = random.Random(1)
    calls = []
    for i in range(400):
        requests = [(rng.choice([0, 1, 64, 127, 128, 129, rng.randint(0, 3000)]), rng.choice([0, 1, 5, 16, 33, 64, 64, 70, 200])) for _ in range(rng.choice([1, 2, 7, 40]))]
        calls.append(((16, 64, 128)[i % 3], rng.choice([1, 2, 7]), rng.choice([1, 3, 4, 8, 16]), *rng.choice([(0, 10 ** 6), (4, 100), (0, 0), (130, 7), (0, 1), (5000, 0), (100, 0)]),
                      rng.choice([1, 2, 17, 512]), requests))
    driver(calls)


@pytest.mark.parametrize("rows", [16, 64, 128])
def test_windows_and_requests_of_nearly_2_31_tokens(driver, rows):
    most = 2 ** 31 - 128
    for sink, window in ((0, most), (most, 0), (most, most), (5, most - 1), (2 ** 30, 2 ** 30), (0, 1)):
        driver([(rows, 2, 1, sink, window, 256, [(most, 64), (3, 70), (most - 77, 1), (0, 5), (most, 1000)])])
