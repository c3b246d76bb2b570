"""Which kernel instances the GPU tests of 8-bit products and of experts reach: number of pieces of sixteen rows, kind of x and type of y for products of few rows, form and types for the
others.  An instance that no case runs fails here."""
import itertools

import test_gpu_experts as experts
import test_gpu_experts_sums as expert_sums
import test_gpu_fp8 as fp8
import test_gpu_fp8_sums as sums
from test_experts_forms import ask  # noqa: F401


def test_products(ask):  # noqa: F811
    cases = [(M, N, K, x, y) for M, N, K, x, y, *_ in fp8.CASES] + sums.CASES
    got = ask(0, [(M, N, K, y == "f32", x == "e4m3") for M, N, K, x, y in cases])
    few, tiles = set(), set()
    for c, (M, _, _, x, y) in zip(got, cases):
        if c["form"] == 3:                                                     # pieces as the launcher rounds them up: 1, 2, 4
            few.add((1 if M <= 16 else 2 if M <= 32 else 4, "codes" if x == "e4m3" else "made" if c["make_rows"] else x, y))
        else:
            tiles.add((c["form"], y))
    assert few >= set(itertools.product((1, 2, 4), ("codes", "made"), ("bf16", "f32"))) | set(itertools.product((1,), ("bf16", "f32"), ("bf16", "f32"))), few
    assert tiles >= {(0, "bf16")} | set(itertools.product((1, 2, 4), ("bf16", "f32"))), tiles


def test_experts(ask):  # noqa: F811
    cases = experts.CASES + expert_sums.MORE
    got = ask(1, [(T, K, I, N, E, k, K * (4 if x == "f32" else 2), 4 if y == "f32" else 2) for T, E, K, I, N, k, _, x, y, _ in cases])
    seen = {(c["form"], c["bm"], y) for c, (*_, y, _) in zip(got, cases)}
    assert seen == {(0, 0, "bf16"), (0, 0, "f32"), (1, 32, "bf16"), (1, 32, "f32"), (1, 128, "bf16"), (1, 128, "f32"), (1, 256, "bf16")}, seen
    assert {(c["form"], x) for c, (*_, x, _, _) in zip(got, cases)} == set(itertools.product((0, 1), ("bf16", "f32")))
    # float results of as many pairs as bf16 ones take tiles of 256 rows for: exact ones all the same
    assert any(y == "f32" and T * k >= 512 * E and c["bm"] == 128 for c, (T, E, _, _, _, k, _, _, y, _) in zip(got, cases))
