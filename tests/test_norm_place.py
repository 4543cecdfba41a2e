"""Which heads the lanes of the norm's kernels store (csrc/norm_place.h): every head of every token by exactly one group of lanes, as the outputs may be the inputs.  Host code."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = """
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "norm_place.h"
int main(int, char** v) {
  const int tokens = atoi(v[1]), heads = atoi(v[2]), dim = atoi(v[3]), grid = atoi(v[4]);       // grid 0: a workgroup for all its items, else steps of the whole grid
  const int blocks = swz::norm_blocks(heads), items = tokens * blocks, per = swz::kNormThreads / (dim / 8);
  const int workgroups = grid ? grid : swz::norm_workgroups(items, dim);
  std::vector<int> stores(tokens * heads);
  for (int w = 0; w < workgroups; ++w)
    for (int64_t first = (int64_t)w * per; first < items; first += grid ? (int64_t)grid * per : items)
      for (int mine = 0; mine < per; ++mine) {
        const swz::NormPlace p = swz::norm_place(first + mine, items, blocks);
        if (p.token < 0 || p.token >= tokens || p.head0 < 0 || p.head0 >= heads) return 1;
        for (int i = 0; i < swz::kNormHeads; ++i)
          if (swz::norm_stores(p, i, heads)) ++stores[p.token * heads + p.head0 + i];
      }
  for (int n : stores) printf("%d ", n);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("place")
    (d / "place.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2508_20258_amd", "csrc"), str(d / "place.cpp"), "-o", str(d / "place")], check=True)
    return str(d / "place")


@pytest.mark.parametrize("grid", [0, 1, 3])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tokens,heads", [(1, 1), (1, 8), (2, 3), (16, 4), (17, 4), (37, 8), (32, 16), (33, 5), (123, 32)])
def test_every_head_is_stored_once(program, tokens, heads, dim, grid):
    out = subprocess.run([program, str(tokens), str(heads), str(dim), str(grid)], check=True, capture_output=True, text=True).stdout
    assert list(map(int, out.split())) == [1] * (tokens * heads)
