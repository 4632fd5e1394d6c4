"""The order in which the XCDs take a grouped GEMM's tiles (csrc/tile_order.h): by the matrix's
features, whatever the tiles' shape, the tokens and the ranges of K."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_23635_amd", "csrc")


def test_lists_are_of_narrow_matrices(tmp_path):
    src = tmp_path / "order.cpp"
    src.write_text("""#include "tile_order.h"
static_assert(moe::one_list(256, false) && moe::one_list(2047, false) && !moe::one_list(2048, false), "bf16, large tiles");
static_assert(moe::one_list(256, true) && moe::one_list(7936, true) && !moe::one_list(8192, true), "small e4m3 tiles");
int main() {}
""")
    subprocess.run(["g++", "-std=c++17", "-fsyntax-only", "-I", CSRC, str(src)], check=True)


def test_the_kernels_ask_by_features():
    """Every call names the matrix's features themselves: not tiles times a tile's token rows, which is
    another number where a tile is not square, nor features times ranges of K."""
    with open(os.path.join(CSRC, "moe_prefill.hip")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    head = re.search(r"TilePos find_tile\(([^)]*)\)\s*\{(.*?)\n\}", text, re.S)
    assert [a.split()[-1] for a in head.group(1).split(",")][2] == "features"
    body = head.group(2)
    assert "one_list(features, small_e4m3)" in body and body.count("features") == 1
    calls = re.findall(r"= find_tile\(([^;]*)\);", text)
    assert len(calls) == 2 and all(c.split(",")[2].strip() == "M" for c in calls)
    assert len(re.findall(r"const int M = kMode == kGateUp \? 2 \* a\.f : a\.d\b", text)) == 2
