"""CPU: which form of linear attention a batch takes, from the library's own plan rules, for the batches that the GPU tests
run: a change of the estimate that moves one of them to another kernel shows here."""
import os
import shutil
import subprocess

import pytest

from tests.linear_forms import CUT, LONG, SHORT, SHORTER, TWO, WHOLE

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "linear_plan.h"
int main(int argc, char** argv) {   // CUs, heads, new tokens of each request
  std::vector<int32_t> c;
  for (int i = 3; i < argc; ++i) c.push_back(atoi(argv[i]));
  s2l_batch b = {};
  b.num_reqs = (int32_t)c.size();
  b.chunk_lens_host = c.data();
  const s2l::LinearPlan p = s2l::linear_plan(&b, atoi(argv[2]), atoi(argv[1]));
  printf("%d %d %d %d %d %d %d %zu\n", p.piece_tokens, p.unit_tokens, p.pieces, p.cut_reqs, p.ws_states, p.short_reqs, (int)p.narrow,
         s2l::linear_bytes(p, atoi(argv[2])));
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    gxx = os.environ.get("CXX") or shutil.which("g++")
    if not gxx:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("linear_plan")
    (d / "plan.cpp").write_text(PROGRAM)
    subprocess.run([gxx, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-Wall", "-Wno-unknown-pragmas", "-Werror", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2604_16395_amd", "csrc"), "-o", str(d / "plan"), str(d / "plan.cpp")], check=True)

    def run(C, hq, cus=256):
        out = subprocess.run([str(d / "plan"), str(cus), str(hq), *map(str, C)], check=True, capture_output=True, text=True).stdout
        names = ("piece_tokens", "unit_tokens", "pieces", "cut_reqs", "ws_states", "short_reqs", "narrow", "bytes")
        return dict(zip(names, map(int, out.split())))
    return run


def form(p):
    return CUT if p["cut_reqs"] else SHORT if not p["pieces"] else TWO if p["narrow"] else WHOLE


@pytest.mark.parametrize("name", LONG)
def test_the_long_batches_take_their_forms(plan, name):
    expected, C, hq, _, blocks, pieces = LONG[name]
    p = plan(C, hq)
    assert (form(p), -(-p["unit_tokens"] // 32), p["pieces"]) == (expected, blocks, pieces)


@pytest.mark.parametrize("name", SHORTER)
def test_the_other_batches_take_their_forms(plan, name):
    for expected, C, hq in SHORTER[name]:
        assert form(plan(C, hq)) == expected, (C, hq)


@pytest.mark.parametrize("seed", range(30))
def test_a_plan_covers_its_batch(plan, seed):
    """Pieces, states and bytes follow from the lengths and the length of a piece; two workgroups a head only without cuts."""
    import random
    rng = random.Random(seed)
    C = [rng.choice([rng.randint(0, 8), rng.randint(0, 300), rng.randint(0, 5000)]) for _ in range(rng.randint(1, 70))]
    hq = rng.choice([1, 2, 8, 32, 64])
    p = plan(C, hq, rng.choice([1, 64, 256]))
    assert p["piece_tokens"] % 32 == 0 and p["piece_tokens"] > 0
    long = [c for c in C if c > 5]
    pieces = [-(-c // p["piece_tokens"]) for c in long]
    assert p["short_reqs"] == len(C) - len(long) and p["pieces"] == sum(pieces)
    assert p["cut_reqs"] == sum(n > 1 for n in pieces) and p["ws_states"] == sum(n + 1 for n in pieces if n > 1)
    assert p["bytes"] == p["ws_states"] * hq * 128 * 128 * 4
    assert p["unit_tokens"] == max([min(c, p["piece_tokens"]) for c in long], default=0)
    assert not (p["narrow"] and p["cut_reqs"])
