"""How rotary positions and appends are dealt to blocks, asked of the built library by a small program (no GPU: nothing is launched)."""
import os
import subprocess

import pytest

from paper_2503_01840_b200 import binding as sb
from paper_2503_01840_b200 import build

ASK = r"""
#include <cstdio>
#include <cstdlib>
#include "kv_cache.cuh"
int main(int n, char **v) {                     // threes of tokens, heads, heads that a block rotates at a time
  for (int i = 1; i + 2 < n; i += 3) {
    const spec::RopePlan p = spec::rope_plan(atoi(v[i]), atoi(v[i + 1]), atoi(v[i + 2]));
    printf("%d %d\n", p.per_block, p.heads);
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("plans")
    src, exe = d / "ask.cu", d / "ask"
    src.write_text(ASK)
    lib = sb.library_path()
    sb.lib()
    subprocess.run([build.NVCC, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, str(src), lib, "-o", str(exe),
                    "-Xlinker", "-rpath", "-Xlinker", os.path.dirname(lib)], check=True, capture_output=True)

    def ask(cases):
        out = subprocess.run([str(exe), *(str(x) for c in cases for x in c)], check=True, capture_output=True, text=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return ask


def test_blocks_take_several_tokens_of_one_head_too(plans):
    (many, _), (some, _), (few, _), (one, _) = plans([(16384, 1, 32), (1000, 1, 32), (148, 1, 32), (1, 1, 8)])
    assert (many, some, few, one) == (16, 7, 1, 1)


def test_every_head_of_every_token_has_a_block_and_few_tokens_have_many(plans):
    cases = [(t, h, step) for t in (1, 2, 63, 148, 149, 1001, 16384, 200000) for h in (1, 2, 3, 5, 16, 40, 48, 120, 257, 4096) for step in (8, 16, 32, 64, 128)]
    for (t, h, step), (per_block, heads) in zip(cases, plans(cases)):
        assert 1 <= per_block <= 16 and 2 <= heads <= max(2, h)          # 2: quotients by the number of heads are taken by a 32-bit reciprocal
        assert per_block == 1 or -(-t // per_block) * per_block < t + per_block
        if t <= 148:
            assert per_block == 1
        # the last slot's number times the reciprocal's error stays below 2^32
        assert (per_block * heads + 256) * heads < 1 << 32
