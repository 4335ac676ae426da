"""Which kernel attends over the 4-bit cache: the rule itself (plain C++), compiled and asked for the calls of the GPU tests."""
import os
import shutil
import subprocess

import pytest

from kv4_shapes import FOUR, ROWS, TWO

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_24174_amd", "csrc")
CXX = shutil.which("g++") or shutil.which("c++")
MAIN = """
#include "kv4_order.h"
#include <cstdio>
int main() {
    long batch, kv_heads, pairs, max_kv, fixed;
    while (std::scanf("%ld %ld %ld %ld %ld", &batch, &kv_heads, &pairs, &max_kv, &fixed) == 5) {
        const Kv4Order o = kv4_order(batch, (int)kv_heads, pairs, max_kv, fixed ? 4 : 64, fixed != 0);
        std::printf("%d %d %d\\n", o.kw, o.chunks, o.chunk_tiles);
    }
}
"""


@pytest.fixture(scope="module")
def order(tmp_path_factory):
    if not CXX:
        pytest.skip("no C++ compiler")
    at = tmp_path_factory.mktemp("order")
    (at / "main.cpp").write_text(MAIN)
    subprocess.run([CXX, "-std=c++20", "-O1", "-Wall", "-Werror", "-I", CSRC, str(at / "main.cpp"), "-o", str(at / "order")], check=True)

    def ask(calls, fixed=False):
        text = "\n".join(f"{b} {kvh} {rows * (h // kvh)} {kv} {int(fixed)}" for b, kvh, h, hd, rows, kv in calls)
        out = subprocess.run([str(at / "order")], input=text, capture_output=True, text=True, check=True).stdout.split("\n")
        return [tuple(map(int, line.split())) for line in out if line]
    return ask


def test_the_calls_of_the_gpu_tests(order):
    for cases in (ROWS, FOUR, TWO):
        got = order([call for call, _ in cases.values()])
        assert {name: o[:2] for name, o in zip(cases, got)} == {name: want for name, (_, want) in cases.items()}


def test_few_pairs_never_take_the_prompts_kernel(order):
    """Waves without pairs of their own would decode tiles for the one that has some."""
    calls = [(b, kvh, kvh * share, 64, rows, 700) for b in (1, 64, 255, 256, 512, 4096) for kvh in (1, 2, 8) for share in (1, 4, 7) for rows in (1, 5, 9, 16, 30)]
    for call, o in zip(calls, order(calls)):
        pairs = call[4] * call[2] // call[1]
        if pairs <= 16:
            assert o[0] in (4, 8), (call, o)
        elif pairs <= 64:
            assert o[0] == 2, (call, o)


def test_orders_cover_their_keys(order):
    """Every tile is in a chunk, no chunk is empty, there are at most 64; a fixed order depends on what a session holds fixed alone."""
    calls = [(b, kvh, kvh * 4, 128, rows, kv) for b in (1, 3, 64) for kvh in (1, 8) for rows in (1, 9, 600) for kv in (0, 1, 31, 33, 700, 4097, 131072)]
    for fixed in (False, True):
        for call, (kw, chunks, per) in zip(calls, order(calls, fixed)):
            tiles = (call[5] + 31) // 32
            assert 1 <= chunks <= (4 if fixed else 64) and kw in ((2,) if fixed else (1, 2, 4, 8))
            assert chunks == 1 or (chunks - 1) * per < tiles <= chunks * per
