"""How single-token attention takes a call apart, asked of the built library by a small program (no GPU: nothing is launched)."""
import os
import subprocess

import pytest

from paper_2503_01840_b200 import binding as sb
from paper_2503_01840_b200 import build

ASK = r"""
#include <cstdio>
#include <cstdlib>
#include "attn_decode.cuh"
int main(int n, char **v) {                     // fp32 queries, format, batch, heads, KV heads, head size, positions
  const spec::DecodePlan p = spec::decode_attn_plan(atoi(v[1]), atoi(v[2]), atoi(v[3]), atoi(v[4]), atoi(v[5]), atoi(v[6]), 148, atoll(v[7]));
  printf("%d %d %d %d %d", p.chunks, p.heads, p.columns, p.groups, p.warps);
}
"""
FORMATS = {"fp32": 0, "bf16": 1, "e4m3": 2, "int8": 3}


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plans")
    src, exe = d / "ask.cu", d / "ask"
    src.write_text(ASK)
    lib = sb.library_path()
    sb.lib()
    subprocess.run([build.NVCC, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, str(src), lib, "-o", str(exe),
                    "-Xlinker", "-rpath", "-Xlinker", os.path.dirname(lib)], check=True, capture_output=True)

    def ask(dtype, fmt, batch, H, G, hd, positions=1 << 31):
        out = subprocess.run([str(exe), *map(str, (int(dtype == "fp32"), FORMATS[fmt], batch, H, G, hd, positions))], check=True, capture_output=True).stdout
        return dict(zip(("chunks", "heads", "columns", "groups", "warps"), map(int, out.split())))
    return ask


@pytest.mark.parametrize("batch", [1, 10, 11, 16, 8192])
@pytest.mark.parametrize("dtype,fmt", [("bf16", "bf16"), ("bf16", "e4m3"), ("bf16", "int8"), ("fp32", "e4m3"), ("fp32", "int8")])
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("group", [1, 4, 8, 9, 13, 14, 15, 16, 17, 24, 32, 33])
def test_a_cache_is_walked_no_more_often_than_the_columns_ask_for(plan, dtype, fmt, batch, hd, group):
    """16 columns hold 16 query heads, or 8 in fp32; heads of 256, and fewer than 22 (sequence, KV head)s for 148 CTAs, have 8 columns."""
    p = plan(dtype, fmt, batch, 2 * group, 2, hd)
    held = (16 if hd < 256 and 2 * batch >= 22 else 8) // (2 if dtype == "fp32" else 1)
    assert p["chunks"] == -(-group // held) and p["heads"] == -(-group // p["chunks"])
    assert p["columns"] >= p["heads"] * (2 if dtype == "fp32" else 1) and p["groups"] > 0


@pytest.mark.parametrize("batch", [1, 8192])
@pytest.mark.parametrize("dtype,fmt,hd", [("fp32", "fp32", 128), ("fp32", "fp32", 256), ("bf16", "e4m3", 80), ("bf16", "bf16", 240)])
@pytest.mark.parametrize("group", [1, 3, 8, 9, 16])
def test_plain_fmas_give_up_heads_only_for_a_table_that_leaves_no_room(plan, dtype, fmt, hd, batch, group):
    """Eight warps of eight heads of 256 take 199680 bytes for queries and two partial states each, and 8193 numbers of the table 32784: more than 224 KB."""
    p = plan(dtype, fmt, batch, group, 1, hd)
    most = 4 if hd == 256 and batch == 8192 and group in (8, 16) else 8              # (nine heads go as five and four)
    assert p["groups"] == 0 and p["chunks"] == -(-group // most) and p["heads"] == -(-group // p["chunks"])
    table = (4 * (batch + 1) + 15) // 16 * 16
    state = p["heads"] * hd + (2 * p["heads"] + 3) // 4 * 4
    assert table + 4 * p["warps"] * (p["columns"] * hd + 64 + 2 * state) <= 224 * 1024


def test_a_narrow_table_of_few_sequences_is_walked_by_halves(plan):
    """256 KB of keys and values a CTA, by what the table holds: 32 segments of 128-byte rows in 148 CTAs have that at 4736 positions, of 256-byte rows at 2368."""
    for fmt, line in (("e4m3", 4736), ("bf16", 2368)):
        assert plan("bf16", fmt, 16, 32, 2, 128, line)["chunks"] == 1 and plan("bf16", fmt, 16, 32, 2, 128, line - 1)["chunks"] == 2
        assert plan("bf16", fmt, 16, 16, 2, 128, line - 1)["chunks"] == 1
        assert plan("bf16", fmt, 37, 32, 2, 128, 16)["chunks"] == 1      # 74 segments may stay whole
