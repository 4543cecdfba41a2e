"""The order of the attention launches (csrc/prompt_order.h): every (turn, key head, query head of it) once, each key head on few XCDs, turns spread over all.  Host code."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = """
#include <cstdio>
#include <cstdlib>
#include "prompt_order.h"
int main(int, char** v) {
  const int turns = atoi(v[1]), heads = atoi(v[2]), group = atoi(v[3]), xcd = atoi(v[4]), sets = swz::prompt_sets(heads, xcd);
  const int n = (int)swz::prompt_workgroups(turns, heads, group, xcd);
  for (int w = 0; w < n; ++w) {
    const swz::PromptPiece p = swz::prompt_piece(w, turns, heads, group, xcd, sets);
    printf("%d %d %d\\n", p.turn, p.k_head, p.member);
  }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("order")
    (d / "order.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2508_20258_amd", "csrc"), str(d / "order.cpp"), "-o", str(d / "order")], check=True)
    return str(d / "order")


@pytest.mark.parametrize("xcd", [1, 2, 3, 8])
@pytest.mark.parametrize("heads,group", [(1, 1), (1, 8), (2, 3), (3, 2), (4, 4), (8, 4), (12, 1), (16, 1)])
def test_every_piece_once(program, heads, group, xcd):
    for turns in (1, 2, 7, 33):
        out = subprocess.run([program, str(turns), str(heads), str(group), str(xcd)], check=True, capture_output=True, text=True).stdout
        pieces = [tuple(map(int, line.split())) for line in out.splitlines()]
        assert len(pieces) % xcd == 0 and len(pieces) < turns * heads * group + xcd * group
        real = [p for p in pieces if p[0] >= 0]
        assert sorted(real) == [(t, h, m) for t in range(turns) for h in range(heads) for m in range(group)]
        for x in range(xcd):
            mine = [p for p in pieces[x::xcd] if p[0] >= 0]
            assert [p[0] for p in mine] == sorted(p[0] for p in mine)                                     # turns in order
            if heads % xcd == 0:
                assert {p[1] for p in mine} == set(range(x * heads // xcd, (x + 1) * heads // xcd))       # whole key heads
            if xcd % heads == 0:
                assert len({p[1] for p in mine}) <= 1
