"""How tiles are dealt to the workers of attention over the paged caches: the kernel's own arithmetic, on the host, against whole numbers of any size.  With ranges that go with the square root of a unit's
tiles, the cost of all tiles times a worker's number comes near 2^32 on 148 multiprocessors and passes it from 150 on."""
import subprocess

import pytest

from paper_2605_23258_b200 import build

PROGRAM = r"""
#include "decode_q4.cuh"
#include <cstdio>
#include <cmath>
using vec::dq4::Deal;
int main() {
    long long sms, warps, cost, X;
    while (std::scanf("%lld %lld %lld %lld", &sms, &warps, &cost, &X) == 4) {
        // one unit: the longest ranges
        const int shortest = (int)cost * std::max((int)(.25f * std::sqrt((float)X / (float)cost) + .5f), 1);
        const Deal deal(X, (int)(sms * warps), shortest);
        std::printf("%d %d %d", shortest, deal.workers, deal.step > 0.);
        for (int w = 0; w <= deal.workers; ++w) std::printf(" %lld", (long long)deal.begin(w));
        std::printf("\n");
    }
}
"""


@pytest.fixture(scope="module")
def deal(tmp_path_factory):
    at = tmp_path_factory.mktemp("deal")
    (at / "deal.cu").write_text(PROGRAM)
    done = subprocess.run([build._nvcc(), *[f for f in build.NVCC_FLAGS if f != "-O3"], "-O1", str(at / "deal.cu"), "-o", str(at / "deal")], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert done.returncode == 0, done.stdout

    def run(cases):
        out = subprocess.run([str(at / "deal")], input="\n".join(" ".join(map(str, c)) for c in cases), stdout=subprocess.PIPE, text=True, check=True).stdout
        return [list(map(int, line.split())) for line in out.splitlines()]
    return run


@pytest.mark.parametrize("sms", [148, 160])
@pytest.mark.parametrize("warps,cost", [(16, 5), (12, 4), (8, 2)])
def test_ranges_are_whole_and_in_order(deal, sms, warps, cost):
    """From one tile to where the ranges become multiples of one fp64 number, and behind that: each begins where the one before ends, and is a tile at the least."""
    most = cost * (warps * sms) ** 2 // 16                                                      # about where there is work for all workers
    cases = [(sms, warps, cost, X) for X in [cost, 7 * cost, 1000 * cost, 100003, *(most * i // 24 for i in (1, 3, 7, 13, 18, 20, 22, 23, 24, 25, 26, 40))]]
    few = 0
    for (_, _, _, X), (shortest, workers, many, *begin) in zip(cases, deal(cases)):
        assert 1 <= workers <= sms * warps and begin[0] == 0 and begin[-1] == X and len(begin) == workers + 1
        assert all(b - a >= cost for a, b in zip(begin, begin[1:])), X
        if not many:
            few = max(few, X * workers)
            assert begin == [X * w // workers for w in range(workers + 1)], X
    if warps == 16:
        assert few > (2 ** 32 if sms == 160 else 0.9 * 2 ** 32)

