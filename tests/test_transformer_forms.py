"""Which form the cases of the GPU tests of 4-bit products and of attention over latent vectors run on, and what must hold for any size: the launchers' own rules
(csrc/w4_choice.h, csrc/latent_choice.h), compiled for the host.  A form that has lost its last case fails here."""
import random
import subprocess

import pytest

import test_gpu_latent as latent
import test_gpu_w4 as w4
from paper_2305_17423_amd import build

PROGRAM = r"""
#include <cstdio>
#include "%s/latent_choice.h"
#include "%s/w4_choice.h"
using namespace fise;
int main() {
    int what, v[9];
    while (std::scanf("%%d", &what) == 1) {
        for (int i = 0; i < (what ? 9 : 4); ++i) if (std::scanf("%%d", &v[i]) != 1) return 1;
        if (!what) {                                     // 0 M N K split: a product with 4-bit weights
            const W4Choice c = w4_choose(v[0], v[1], v[2], v[3] != 0);
            std::printf("%%d %%d %%d %%d %%d %%d %%d %%d %%d %%d %%d %%d\n", c.staged, c.pieces, c.slab, c.slabs, c.mt, c.kt, c.waves_k, c.chunks, c.tiles_n, c.groups_n, c.x_at, c.lds);
            continue;
        }
        const LatentShape s{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7], v[8] != 0};      // 1 B M n heads d dr dv r causal
        const AbsorbedLayout a = absorbed_layout(s);
        const ExpandedLayout e = expanded_layout(s);
        std::printf("%%d %%d %%d %%d %%d %%d %%d %%d %%d", latent_width(s.r), latent_shared(s.dr), absorbed_tiles(s), absorbed_workgroups(s), absorbed_tokens(s), expanded_tile(s), expanded_whole(s),
                    expanded_workgroups(s), latent_expands(s));
        std::printf(" %%zu %%zu %%zu %%zu %%zu %%lld %%zu %%zu %%zu %%zu %%zu\n", a.table, a.q, a.ml, a.part, a.total, e.n_pad, e.k, e.v, e.ml, e.part, e.total);
    }
}
"""
W4 = ("staged", "pieces", "slab", "slabs", "mt", "kt", "waves_k", "chunks", "tiles_n", "groups_n", "x_at", "lds")
LATENT = ("width", "shared", "tiles", "workgroups", "tokens", "tile", "whole", "expanded_workgroups", "expands", "table", "q", "ml", "part", "total", "n_pad", "xk", "xv", "xml", "xpart", "xtotal")


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("forms")
    (d / "forms.cpp").write_text(PROGRAM % (build.CSRC, build.CSRC))
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", str(d / "forms"), str(d / "forms.cpp")], check=True)

    def run(what, questions):
        r = subprocess.run([str(d / "forms")], input="\n".join(" ".join(str(int(v)) for v in (what, *q)) for q in questions), check=True, capture_output=True, text=True)
        out = [dict(zip((W4, LATENT)[what], map(int, line.split()))) for line in r.stdout.splitlines()]
        assert len(out) == len(questions)
        return out
    return run


def test_forms_of_4_bit_products(ask):
    cases = [(M, N, K, xt == "f32" or silu) for M, N, K, _, xt, _, silu, _ in w4.CASES]
    got = ask(0, cases)
    forms = {("staged" if c["staged"] else "resident", c["pieces"], c["mt"], c["kt"] if not c["staged"] else 0, c["chunks"] > 1) for c in got}
    # every number of tiles of rows and columns that a wave keeps, one round and several, whole x and its three parts
    assert {f[2:4] for f in forms if f[0] == "resident"} == {(1, 1), (1, 2), (1, 4), (2, 1), (2, 2), (4, 1)}
    assert {(f[1], f[4]) for f in forms if f[0] == "resident"} == {(1, False), (1, True), (3, False), (3, True)}
    assert {f[1:3] for f in forms if f[0] == "staged"} == {(1, 2), (1, 4), (3, 2), (3, 4)}
    assert {c["waves_k"] for c in got if c["staged"]} == {1, 2, 4}
    assert any(c["slabs"] > 1 for c in got) and any(c["tiles_n"] > 1 and not c["staged"] for c in got)


def test_any_4_bit_product_is_covered(ask):
    rng = random.Random(3)
    log = lambda top: int(2 ** rng.uniform(0, top))
    cases = [(log(10), log(17), 8 * log(12), rng.random() < 0.5) for _ in range(4000)] + [(m, n, k, s) for m in (1, 64, 4096) for n in (1, 1 << 20) for k in (8, 65536) for s in (False, True)]
    for (M, N, K, split), c in zip(cases, ask(0, cases)):
        tn, tk = -(-N // 16), -(-K // 128)
        assert c["slab"] * c["pieces"] <= 16 * c["mt"] <= 64 and c["slab"] * c["slabs"] >= M, (M, N, K)
        assert c["tiles_n"] * c["groups_n"] >= tn and c["lds"] <= 160 * 1024, (M, N, K)
        if c["staged"]:
            assert c["chunks"] * 4 >= tk and c["waves_k"] * c["tiles_n"] == 8, (M, N, K)
        else:
            assert c["kt"] * c["mt"] <= 4 and c["waves_k"] * 64 <= (512 if c["mt"] == 4 else 1024) and c["waves_k"] * c["kt"] * c["chunks"] >= tk, (M, N, K)
            assert c["x_at"] + (16 * (c["waves_k"] * 128 + 8) * 2 if split else 0) <= c["lds"] and c["tiles_n"] * c["waves_k"] * c["mt"] * 1024 <= c["lds"], (M, N, K)
            assert c["chunks"] == 1 or not split or c["x_at"] >= c["tiles_n"] * c["waves_k"] * c["mt"] * 1024, (M, N, K)      # x must not lie on parts that are still added to


def test_forms_of_latent_attention(ask):
    cases = [(*c, 0) for c in latent.CASES] + [(*c[:-1], causal) for c in latent.LENGTHS for causal in (0, 1)]
    got = ask(1, cases)
    assert {(c["width"], c["shared"]) for c in got} == {(w, s) for w in (128, 256, 384, 512) for s in (0, 64)}
    assert {c["tokens"] for c in got} == {1, 4, 16}
    assert {c["tile"] for c in got} == set(range(7)) and {c["tile"] for c in got if not c["whole"]} == set(range(7))
    assert len({c["tile"] for c in got if c["whole"]}) >= 2
    assert {c["expands"] for c in got} == {0, 1}


def test_which_form_is_taken(ask):
    wide = (16, 128, 64, 128, 512)
    cases = [(B, 1, n, *wide, 0) for B in (1, 32) for n in (2, 100, 32768)] + [(1, n, n, *wide, 1) for n in (512, 4096, 32768)]
    assert [c["expands"] for c in ask(1, cases)] == [0] * 6 + [1] * 3


def test_any_workspace_is_in_order(ask):
    rng = random.Random(4)
    log = lambda top: int(2 ** rng.uniform(0, top))
    cases = [(log(6), log(11), log(15), log(7), 8 * rng.randint(1, 20), 8 * rng.randint(0, 8), 8 * rng.randint(1, 20), 8 * rng.randint(1, 64), rng.random() < 0.5) for _ in range(3000)]
    for (B, M, n, H, d, dr, dv, r, causal), c in zip(cases, ask(1, cases)):
        tag = (B, M, n, H, d, dr, dv, r)
        for names in (("table", "q", "ml", "part", "total"), ("table", "xk", "xv", "xml", "xpart", "xtotal")):
            at = [c[k] for k in names]
            assert at == sorted(at) and all(x % 256 == 0 for x in at), tag
        groups, width = B * c["tiles"], c["width"] + c["shared"]
        assert c["tiles"] * 64 >= M * H and c["q"] >= 4 * (groups + 1) and c["ml"] - c["q"] >= B * M * H * width * 2, tag
        assert c["part"] - c["ml"] >= (groups + c["workgroups"]) * 64 * 8 and c["total"] - c["part"] >= (groups + c["workgroups"]) * 64 * c["width"] * 4, tag
        assert c["n_pad"] >= n and c["n_pad"] % 128 == 0 and c["xml"] - c["xv"] >= B * H * dv * c["n_pad"] * 2 and c["xv"] - c["xk"] >= B * H * (d + dr) * c["n_pad"] * 2, tag
        groups = B * H * -(-M // 128)
        slots = 0 if c["whole"] else groups + c["expanded_workgroups"]
        assert c["xpart"] - c["xml"] >= slots * 128 * 8 and c["xtotal"] - c["xpart"] >= slots * 128 * dv * 4, tag
        assert c["expanded_workgroups"] == groups if c["whole"] else c["expanded_workgroups"] <= 512, tag
