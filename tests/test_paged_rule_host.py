"""How attention over pages shares its rows out (csrc/paged_rule.h, compiled for the host): a cluster that finds no room is never chosen, and the choices
that were measured are made."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_04476_b200", "csrc")
MAIN = """
#include <cstdio>
#include "paged_rule.h"
int main() {
  int dh, n[PA_SIZES], room[PA_SIZES];
  long long runs, tiles, resident;
  while (std::scanf("%d %lld %lld %lld %d %d %d %d", &dh, &runs, &tiles, &resident, n, n + 1, n + 2, n + 3) == 8) {
    for (int i = 0; i < PA_SIZES; ++i) room[i] = cluster_ctas(n[i], 1 << i);
    std::printf("%d\\n", paged_join_ranks(dh, runs, tiles, resident, room));
  }
}
"""
CLUSTERS = {False: (296, 148, 71, 33), True: (148, 74, 33, 15)}       # clusters of each size that a B200 holds: 256 channels or fewer


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    cxx = os.environ.get("CXX", "g++")
    if not shutil.which(cxx):
        pytest.skip("no C++ compiler")
    at = tmp_path_factory.mktemp("rule")
    (at / "main.cpp").write_text(MAIN)
    subprocess.run([cxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-I" + CSRC, str(at / "main.cpp"), "-o", str(at / "rule")], check=True)

    def ask(calls):
        """Ranks for each (dh, runs, rows, clusters of each size that fit)."""
        unit = {32: 256, 64: 128, 128: 64, 256: 64}
        text = "".join(f"{dh} {runs} {-(-rows // unit[dh])} {148 if dh == 256 else 296} {' '.join(map(str, n))}\n" for dh, runs, rows, n in calls)
        out = subprocess.run([str(at / "rule")], input=text, capture_output=True, text=True, check=True).stdout
        return [int(x) for x in out.split()]
    return ask


def test_a_cluster_without_room_is_never_chosen(rule):
    sizes = [(dh, runs, rows) for dh in (32, 64, 128, 256) for runs in (1, 2, 5, 16, 33, 64, 150, 300, 4000, 400000) for rows in
             (1, 64, 500, 2048, 5001, 16384, 100000, 1 << 24)]
    for out in ((0,), (1,), (2,), (3,), (2, 3), (1, 2, 3), (0, 1, 2, 3)):
        calls = [(dh, runs, rows, [0 if i in out else n for i, n in enumerate(CLUSTERS[dh == 256])]) for dh, runs, rows in sizes]
        got = rule(calls)
        assert not set(got) & {1 << i for i in out}
        if len(out) == 4:
            assert set(got) == {0}
        else:
            assert len(set(got)) > 1                           # what fits is still made use of
    for n in (-1, -7):                                         # an answer that is no number of clusters
        assert set(rule([(dh, runs, rows, [n] * 4) for dh, runs, rows in sizes])) == {0}


# (rows, sequences): us with clusters of 8, the best smaller ones, and shared out, 8/2 heads x 128
MEASURED = {(1024, 1): (4.4, 5.5, 5.9), (8192, 1): (14, 25, 8.0), (2048, 16): (7.3, 8.3, 11.8), (512, 64): (17, 6.7, 11.1), (2048, 256): (120, 79, 90),
            (16384, 12): (35, 41, 39), (16384, 16): (43, 48, 49), (16384, 18): (61, 52, 53), (16384, 32): (83, 80, 85)}


def test_the_choice_is_the_faster_one_where_it_was_measured(rule):
    got = rule([(128, 2 * B, rows, CLUSTERS[False]) for rows, B in MEASURED])
    for ranks, (case, us) in zip(got, MEASURED.items()):
        assert us[{8: 0, 0: 2}.get(ranks, 1)] <= 1.03 * min(us), case
