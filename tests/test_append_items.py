"""How many items an append with tok_start has and which calls it refuses, by the library's own function compiled for the
host (no GPU needed)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2601_08670_gb300", "csrc")

MAIN = r"""
#include "kv_append.cuh"
#include <cstdio>
int main() {
  pced::AppendArgs a;
  int units, cluster;
  while (scanf("%d %d %d %d %d %d", &a.T, &a.c.S, &a.c.Hkv, &a.c.block_rows, &units, &cluster) == 6) {
    const long long items = pced::append_items(a, units, cluster);
    printf("%lld %d\n", items, items ? a.heads : 0);
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("no nvcc")
    d = tmp_path_factory.mktemp("items")
    (d / "main.cu").write_text(MAIN)
    subprocess.run([nvcc, "-std=c++17", "-gencode", "arch=compute_103a,code=sm_103a", "-I", CSRC, "-I",
                    os.path.join(ROOT, "include"), "-o", str(d / "main"), str(d / "main.cu")], check=True, timeout=300)
    return str(d / "main")


def items(program, *cases):
    text = "\n".join(" ".join(map(str, c)) for c in cases)
    out = subprocess.run([program], input=text, capture_output=True, text=True, check=True, timeout=60).stdout
    return [tuple(map(int, line.split())) for line in out.splitlines()]


def test_items_and_heads(program):
    # T, S, Hkv, block_rows, units, CTAs of an item
    got = items(program, (1056, 33, 4, 128, 16, 1), (1056, 33, 4, 128, 16, 8), (9, 9, 8, 64, 16, 1), (3, 3, 3, 16, 32, 1),
                (1, 1, 8, 16, 16, 1))
    assert got == [(74, 1), (74, 1), (18, 8), (6, 1), (2, 8)]


def test_a_grid_without_clusters_takes_eight_times_the_items(program):
    T, Hkv = 2 ** 31 - 1, 8  # 2^27 + 1 items of 16 rows, 2^30 + 8 CTAs
    assert items(program, (T, 1, Hkv, 16, 16, 1), (T, 1, Hkv, 16, 16, 8)) == [((T // 16) + 2, 1), (0, 0)]
    assert items(program, (T, 1, 16, 16, 16, 1)) == [(0, 0)]  # 2^31


def test_the_8_bit_append_asks_for_no_clusters():
    assert "append_items(a, APP_THREADS / (c.D / 16), 1)" in open(os.path.join(CSRC, "kv_append8.cu")).read()
