"""Which form the cases of the GPU tests of 8-bit products, routing and experts run on, and what must hold for any size: the launchers' own rules (csrc/fp8_choice.h, csrc/route_choice.h),
compiled for the host.  A form that has lost its last case fails here."""
import random
import subprocess

import pytest

import test_gpu_experts as experts
import test_gpu_fp8 as fp8
import test_gpu_route as route
from paper_2305_17423_amd import build

PROGRAM = r"""
#include <cstdio>
#include "%s/fp8_choice.h"
#include "%s/route_choice.h"
using namespace fise;
int main() {
    long long what, v[8];
    while (std::scanf("%%lld", &what) == 1) {
        for (int i = 0; i < 8; ++i) if (std::scanf("%%lld", &v[i]) != 1) return 1;
        if (what == 0) {                                 // M N K exact codes
            const Fp8Choice c = fp8_choose(v[0], v[1], v[2], v[3] != 0, v[4] != 0);
            const Fp8Space s = fp8_space(v[0], v[2]);
            std::printf("%%d %%d %%d %%lld %%lld %%d %%d %%lld %%lld %%lld\n", c.form, c.bm, c.bn, (long long)c.m_tiles, (long long)c.n_tiles, c.waves, (int)c.make_rows, (long long)s.stride, (long long)s.scale_off, (long long)s.bytes);
        } else if (what == 1) {                          // T K I N E k x_row_bytes y_bytes
            const ExpertChoice c = expert_choose(v[0], v[1], v[2], v[3], v[4], v[5], v[6], (int)v[7]);
            std::printf("%%d %%d %%lld %%d %%d %%lld %%lld %%lld %%lld %%lld %%lld %%lld %%lld %%lld %%lld\n", c.form, c.bm, (long long)c.m_tiles, c.waves_in, c.waves_out, (long long)c.x_stride, (long long)c.x_scale_off,
                        (long long)c.h_off, (long long)c.h_stride, (long long)c.h_scale_off, (long long)c.out_off, (long long)c.row_exp_off, (long long)c.table_off, (long long)c.place_off, (long long)c.bytes);
        } else {                                         // T E k groups lists
            const RouteChoice c = route_choose(v[0], (int)v[1], (int)v[2], (int)v[3], v[4] != 0);
            std::printf("%%d %%d %%d %%d %%d %%d %%lld %%lld %%lld\n", c.lanes, c.values, c.single, c.waves, c.wave_tokens, c.chunks, (long long)c.hist_off, (long long)c.total_off, (long long)c.bytes);
        }
    }
}
"""
FIELDS = (("form", "bm", "bn", "m_tiles", "n_tiles", "waves", "make_rows", "stride", "scale_off", "bytes"),
          ("form", "bm", "m_tiles", "waves_in", "waves_out", "x_stride", "x_scale_off", "h_off", "h_stride", "h_scale_off", "out_off", "row_exp_off", "table_off", "place_off", "bytes"),
          ("lanes", "values", "single", "waves", "wave_tokens", "chunks", "hist_off", "total_off", "bytes"))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("forms")
    (d / "f.cpp").write_text(PROGRAM % (build.CSRC, build.CSRC))
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", str(d / "f"), str(d / "f.cpp")], check=True)

    def run(what, cases):
        text = "".join(" ".join(str(int(v)) for v in (what, *c, *(0,) * (8 - len(c)))) + "\n" for c in cases)
        out = subprocess.run([str(d / "f")], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        return [dict(zip(FIELDS[what], map(int, line.split()))) for line in out]
    return run


def test_every_form_of_a_product_has_a_case(ask):
    got = ask(0, [(M, N, K, y == "f32", x == "e4m3") for M, N, K, x, y, _, _ in fp8.CASES])
    seen = {(c["form"], y == "f32") for c, (_, _, _, _, y, _, _) in zip(got, fp8.CASES)}
    assert seen >= {(0, False), (1, False), (1, True), (2, False), (2, True), (3, False), (3, True), (4, False), (4, True)}, seen
    few = {((M + 15) // 16, x if not c["make_rows"] else "made") for c, (M, _, _, x, _, _, _) in zip(got, fp8.CASES) if c["form"] == 3}
    assert {("f32"), ("bf16"), ("e4m3"), ("made")} <= {x for _, x in few} and {1, 2, 4} <= {n for n, _ in few}, few


def test_every_form_of_experts_has_a_case(ask):
    got = ask(1, [(T, K, I, N, E, k, K * (4 if x == "f32" else 2), 4 if y == "f32" else 2) for T, E, K, I, N, k, _, x, y, _ in experts.CASES])
    assert {(c["form"], c["bm"]) for c in got} >= {(0, 0), (1, 32), (1, 128), (1, 256)}, got


def test_every_form_of_routing_has_a_case(ask):
    got = ask(2, [(T, E, k, groups, 1) for T, E, k, _, _, _, groups, _, _, _ in route.CASES])
    assert {(c["lanes"], c["values"], c["single"]) for c in got} == {(16, 4, 0), (16, 4, 1), (16, 16, 0), (16, 16, 1), (64, 16, 0), (64, 16, 1)}


def test_what_holds_for_any_size(ask):
    rng = random.Random(11)
    size = lambda top: int(2 ** rng.uniform(0, top))
    products = [(size(20), size(20), 16 * size(16), rng.random() < 0.5, rng.random() < 0.5) for _ in range(3000)]
    for c, (M, N, K, exact, codes) in zip(ask(0, [tuple(int(v) for v in p) for p in products]), products):
        assert c["m_tiles"] * c["bm"] >= M > (c["m_tiles"] - 1) * c["bm"] and c["n_tiles"] * c["bn"] >= N
        assert not (exact and c["form"] == 0) and not (codes and c["make_rows"]) and (c["form"] == 3 or c["make_rows"] != codes)
        if c["form"] == 3:
            assert M <= 64 and 1 <= c["waves"] <= 16 and (codes or c["make_rows"] or M <= 16)
        assert c["stride"] >= K and c["stride"] % 128 == 0 and c["scale_off"] >= M * c["stride"] and c["bytes"] >= c["scale_off"] + 4 * M * (c["stride"] // 128)
    cases = []
    while len(cases) < 3000:
        T, K, I, N, E = size(18), 16 * size(12), 16 * size(12), 8 * size(13), size(10)
        k = min(size(6), 64)
        if T * k < 2 ** 24 and T * K < 2 ** 30:
            cases.append((T, K, I, N, E, k, K * rng.choice([2, 4]), rng.choice([2, 4])))
    for c, (T, K, I, N, E, k, row, y) in zip(ask(1, cases), cases):
        P = T * k
        if c["form"] == 0:
            assert T <= 4 and c["bytes"] >= 4 * P * I and 1 <= c["waves_in"] <= 16 and 1 <= c["waves_out"] <= 16 and 4 * P * I < 2 ** 30 and T * row < 2 ** 30
            continue
        counts = [0] * E
        for p in range(min(P, 2000)):
            counts[rng.randrange(E)] += 1
        assert sum(-(-n // c["bm"]) for n in counts) <= c["m_tiles"]
        offs = [c[n] for n in ("x_scale_off", "h_off", "h_scale_off", "out_off", "row_exp_off", "table_off", "place_off", "bytes")]
        need = [T * c["x_stride"], 4 * T * (c["x_stride"] // 128), P * c["h_stride"], 4 * P * (c["h_stride"] // 128), P * N * y, 0 if y == 4 else P * -(-N // 32), 8 * c["m_tiles"], 4 * P]
        for begin, end, n in zip([0] + offs, offs, need):
            assert end - begin >= n and begin % 256 == 0
    cases = [(size(22), E, min(size(6), E, 64), rng.choice([g for g in (1, 2, 4, 8, 16, 64) if E % g == 0]), 1) for E in (size(10) for _ in range(2000))]
    for c, (T, E, k, groups, _) in zip(ask(2, cases), cases):
        assert c["lanes"] * c["values"] >= E and c["lanes"] >= k and c["lanes"] >= groups
        assert c["chunks"] * c["waves"] * c["wave_tokens"] >= T and c["wave_tokens"] % (64 // c["lanes"]) == 0
        assert c["waves"] * c["wave_tokens"] * k < 65536                       # ranks have sixteen bits
        if c["single"]:
            assert c["chunks"] == 1 and c["bytes"] == 0 and T * k <= 4096
        else:
            assert c["hist_off"] >= 4 * T * k and c["total_off"] - c["hist_off"] >= 4 * E * c["chunks"] and c["bytes"] - c["total_off"] >= 4 * E
