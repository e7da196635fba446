"""How many CTAs share a tile of the 8-bit product (csrc/sqnn_fp8_plan.h, host code): never more clusters than run at once, whatever the runtime counts."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HARNESS = r"""
#include "sqnn_fp8_plan.h"
#include <cstdio>
using namespace sqnn;
int main()
{
    unsigned tiles, wanted, most, sms, per_sm, counts;
    while (std::scanf("%u %u %u %u %u %u", &tiles, &wanted, &most, &sms, &per_sm, &counts) == 6) {
        const auto runtime = [&](unsigned cluster) { return sms * counts / cluster; };
        std::printf("%u\n", split_for(tiles, wanted, most, [&](unsigned c) { return clusters_at_once(runtime(c), c, sms, per_sm); }));
    }
}
"""


@pytest.fixture(scope="module")
def splits(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src, exe = str(d / "plan.cpp"), str(d / "plan")
    with open(src, "w") as f:
        f.write(HARNESS)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-I", os.path.join(ROOT, "paper_1905_10138_b200", "csrc"), src, "-o", exe], check=True)

    def run(cases):
        text = "\n".join(" ".join(map(str, c)) for c in cases)
        return [int(v) for v in subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split()]
    return run


def test_all_clusters_run_at_once_whatever_the_runtime_counts(splits):
    sms = 148
    cases = [(tiles, wanted, 8, sms, per_sm, counts) for tiles in (1, 3, 8, 20, 32, 37, 47, 60, 75, 100, 148, 149, 200, 300) for wanted in (118, 148, 185, 1000)
             for per_sm in (1, 2, 3) for counts in (1, 2, 3)]
    for (tiles, wanted, most, _, per_sm, counts), split in zip(cases, splits(cases)):
        assert 1 <= split <= most
        if split > 1:
            assert tiles * split <= sms * max(per_sm, counts), (tiles, wanted, per_sm, counts, split)


def test_a_runtime_that_counts_all_gives_the_same_splits(splits):
    sms = 160                                                      # (no rounding: clusters of every size up to eight divide it, or nearly)
    for per_sm in (2, 3):
        for cluster_tiles in (10, 20, 32, 40, 64, 80):
            one, all_ = splits([(cluster_tiles, 1000, 5, sms, per_sm, 1), (cluster_tiles, 1000, 5, sms, per_sm, per_sm)])
            assert abs(one - all_) <= 1 and cluster_tiles * max(one, all_) <= sms * per_sm


def test_splits_of_known_sizes(splits):
    # 4096 x 9216: batch 1 (two CTAs an SM) and batch 64 (one); 6000 x 3000 batch 8; 1024 x 1024 batch 1, eight blocks of columns
    assert splits([(32, 185, 8, 148, 2, 1), (32, 118, 8, 148, 1, 1), (47, 185, 8, 148, 2, 1), (8, 185, 8, 148, 2, 1)]) == [6, 4, 4, 8]
