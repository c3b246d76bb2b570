"""Which tile of queries a workgroup of attention over latent vectors has (csrc/latent_choice.h, compiled for the host): every tile once, whatever the numbers, and balanced
where a CU holds two workgroups."""
import random
import subprocess

import pytest

from paper_2305_17423_amd import build

PROGRAM = r"""
#include <cstdio>
#include "%s/latent_choice.h"
using namespace fise;
int main() {
    int heads, tiles, per_cu;
    while (std::scanf("%%d %%d %%d", &heads, &tiles, &per_cu) == 3) {
        for (int w = 0; w < heads * tiles; ++w) {
            const ExpandedPlace p = expanded_place(w, heads, tiles, per_cu);
            std::printf("%%d %%d ", p.head, p.tile);
        }
        for (int i = 0; i < tiles; ++i) std::printf("%%d %%d ", expanded_line_tile(i, tiles), expanded_line_place(expanded_line_tile(i, tiles), tiles));
        std::printf("\n");
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("order")
    (d / "order.cpp").write_text(PROGRAM % build.CSRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", str(d / "order"), str(d / "order.cpp")], check=True)

    def run(sizes):
        r = subprocess.run([str(d / "order")], input="\n".join(" ".join(map(str, s)) for s in sizes), check=True, capture_output=True, text=True)
        out = []
        for (heads, tiles, _), line in zip(sizes, r.stdout.splitlines()):
            v = list(map(int, line.split()))
            n = 2 * heads * tiles
            out.append((list(zip(v[:n:2], v[1:n:2])), list(zip(v[n::2], v[n + 1::2]))))
        assert len(out) == len(sizes)
        return out
    return run


def sizes():
    """(heads of all elements, tiles, workgroups a CU holds): as many tiles as the CUs hold workgroups, a few more, many."""
    rng = random.Random(7)
    s = [(16, 32, 2), (16, 33, 2), (16, 64, 2), (40, 16, 2), (171, 3, 2), (8, 64, 2), (512, 1, 2), (513, 1, 2), (3, 171, 2), (129, 4, 2), (640, 5, 2), (16, 16, 1), (33, 8, 1)]
    while len(s) < 300:
        per_cu, heads, tiles = rng.choice([1, 2, 2]), int(2 ** rng.uniform(0, 10)), int(2 ** rng.uniform(0, 9))
        if per_cu * 256 <= heads * tiles <= 6000:
            s.append((heads, tiles, per_cu))
    return s


def test_every_tile_has_a_workgroup(ask):
    for (heads, tiles, per_cu), (places, line) in zip(sizes(), ask(sizes())):
        assert sorted(places) == [(h, t) for h in range(heads) for t in range(tiles)], (heads, tiles, per_cu)
        assert sorted(t for t, _ in line) == list(range(tiles)) and [p for _, p in line] == list(range(tiles)), tiles


def test_an_xcd_has_whole_heads(ask):
    for (heads, tiles, per_cu), (places, _) in zip(sizes(), ask(sizes())):
        if heads % 8 == 0:
            for w, (h, _) in enumerate(places):
                assert h // (heads // 8) == w % 8, (heads, tiles)


def test_the_two_workgroups_of_a_cu_share_the_keys_evenly(ask):
    """The first two rounds of workgroups: tile numbers of a CU's two add up to the same, one more or one less, for any number of tiles."""
    for (heads, tiles, per_cu), (places, _) in zip(sizes(), ask(sizes())):
        if per_cu == 2:
            sums = [places[w][1] + places[w + 256][1] for w in range(256)]
            assert max(sums) - min(sums) <= 2 and abs(sum(sums) / 256 - min(sums)) <= 1, (heads, tiles)
        else:
            assert [t for _, t in places[:256]] == sorted((t for _, t in places[:256]), reverse=True) or heads % 8, (heads, tiles)


def test_gpu_cases_are_of_this_kind():
    import test_gpu_latent_order as gpu
    for B, M, n, H, d, dr, dv, r, lens in gpu.CASES:
        tiles, per_cu = -(-M // 128), 1 if d + dr > 192 or dv > 128 else 2
        assert tiles >= 4 and B * H * tiles >= per_cu * 256, (B, M, H)
