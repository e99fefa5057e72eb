"""How a product of 4-bit microscaled matrices is cut into tiles and parts (csrc/mx4_plan.hpp), compiled for the host: no GPU is
needed."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAIN = r"""
#include <cstdio>
#include "mx4_plan.hpp"
int main() {
  long long M, N, K, room;
  while (std::scanf("%lld %lld %lld %lld", &M, &N, &K, &room) == 4) {
    const halp::ProductPlan best = halp::product_plan(M, N, K, 256, halp::kMostCuts);
    const long long need = halp::plan_workspace(M, N, best);
    const halp::ProductPlan p = halp::product_plan_within(M, N, K, 256, need + room < 0 ? 0 : need + room);
    std::printf("%d %d %d %d %lld", best.tile, best.cuts, p.tile, p.cuts, need);
    for (int tile = 64; tile <= 256; tile *= 2) std::printf(" %.9g", halp::product_us(M, N, K, 256, {tile, 1}));
    std::printf("\n");
  }
}
"""
SIZES = [(1000, 784, 60000), (300, 784, 60000), (2000, 2000, 30000), (3000, 500, 10000), (1024, 1024, 16384), (600, 600, 20000),
         (128, 128, 60000), (300, 4096, 4096), (8192, 8192, 8192), (1, 1, 1), (70, 90, 9000), (1, 5, 0), (2 ** 20, 33, 1000)]


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("mx4_plan")
    (tmp / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_1803_03383_amd", "csrc"),
                    "-o", str(tmp / "main"), str(tmp / "main.cpp")], check=True)

    def run(room):
        text = "".join("%d %d %d %d\n" % (*s, room) for s in SIZES)
        out = subprocess.run([str(tmp / "main")], input=text, capture_output=True, text=True, check=True).stdout
        return [[float(v) for v in line.split()] for line in out.splitlines()]
    return run


def test_products_without_room_for_parts_take_the_tiles_that_are_best_uncut(plans):
    seen = 0
    for room in (-1, -2 ** 50):  # a byte less than it takes, and none
        for size, (tile, cuts, own, parts, need, *us) in zip(SIZES, plans(room)):
            if need > 0:
                assert parts == 1 and us[int(own).bit_length() - 7] == min(us), size
                seen += own != tile
            else:
                assert (own, parts) == (tile, cuts) and cuts == 1, size
    assert seen  # sizes whose tiles in parts are others than alone


def test_products_with_room_are_made_in_parts(plans):
    for size, (tile, cuts, own, parts, need, *_) in zip(SIZES, plans(0)):
        assert (own, parts) == (tile, cuts), size
        assert need == (4 * cuts * size[0] * -(-size[1] // 4) * 4 if cuts > 1 else 0), size
