"""GPU checks of the routing of tokens to experts against its definition in 64 bits: ids, offsets and order of the pairs equal, weights to float.

Tolerance of a weight, from arithmetic: a score is within 2^-22 of its value in float, k of them and their sum add k roundings and a division, the scale one: (k + 8) 2^-22 of it holds that."""
import math

import pytest
import torch

from helpers import DEV

pytestmark = pytest.mark.gpu
T_ = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def define(logits, bias, k, score, groups, top_groups, group_top, renorm, scale):
    """Row by row, in doubles."""
    T, E = logits.shape
    l = logits.double()
    ids, weights = torch.full((T, k), -1, dtype=torch.int32), torch.zeros((T, k), dtype=torch.float64)
    s = torch.softmax(l, 1) if score == "softmax" else torch.sigmoid(l)
    for t in range(T):
        row, alive = l[t], l[t] > -math.inf
        key = s[t].clone() if bias is None else s[t] + bias.double()
        if bias is None and (groups == 1 or group_top == 1):                   # the order of the scores is that of the logits
            key = row.clone()
        if bool(torch.isnan(row).any()) or (score == "softmax" and bool((row == math.inf).any())) or bool(torch.isnan(key[alive]).any()):
            weights[t] = math.nan
            continue
        key = [float(v) if a else -math.inf for v, a in zip(key, alive)]
        if groups > 1:
            size = E // groups
            sums = []
            for g in range(groups):
                best = [v for v in sorted(key[g * size:(g + 1) * size], reverse=True)[:group_top] if v > -math.inf]
                sums.append(sum(best) if best else -math.inf)
            kept = sorted(range(groups), key=lambda g: (-sums[g], g))[:top_groups]
            key = [v if e // size in kept else -math.inf for e, v in enumerate(key)]
        order = [e for e in sorted(range(E), key=lambda e: (-key[e], e))[:k] if key[e] > -math.inf]
        w = [float(s[t, e]) for e in order]
        total = sum(w)
        for j, e in enumerate(order):
            ids[t, j] = e
            weights[t, j] = scale * (w[j] / total if renorm and total > 0 else 0.0 if renorm else w[j])
    flat = ids.view(-1).tolist()
    lists = [[p for p, e in enumerate(flat) if e == x] for x in range(E)] if T * k * E < 3e6 else None
    if lists is None:
        lists = [[] for _ in range(E)]
        for p, e in enumerate(flat):
            if e >= 0:
                lists[e].append(p)
    offsets = [0]
    for v in lists:
        offsets.append(offsets[-1] + len(v))
    return ids, weights, torch.tensor(offsets, dtype=torch.int32), torch.tensor(sum(lists, []), dtype=torch.int32)


def run(fb, logits, bias, k, lists=True, **kw):
    T, E = logits.shape
    ids, w = torch.full((T, k), 99, dtype=torch.int32, device=DEV), torch.full((T, k), 99.0, device=DEV)
    o, s = (torch.full((n,), -7, dtype=torch.int32, device=DEV) for n in (E + 1, T * k))
    a = fb.route_args(logits.to(DEV), ids, w, o if lists else None, s if lists else None, bias=None if bias is None else bias.to(DEV), **kw)
    ws = torch.full((max(fb.fise_route_experts_workspace_bytes(a), 256),), 0x5A, dtype=torch.uint8, device=DEV)
    fb.fise_route_experts(a, ws)
    return ids.cpu(), w.cpu(), o.cpu(), s.cpu()


def check(fb, logits, bias, k, score="softmax", groups=1, top_groups=1, group_top=1, renormalize=True, scale=1.0):
    got = run(fb, logits, bias, k, score=score, groups=groups, top_groups=top_groups, group_top=group_top, renormalize=renormalize, scale=scale)
    ids, w, o, s = define(logits, bias, k, score, groups, top_groups, group_top, renormalize, scale)
    assert torch.equal(got[0], ids)
    assert torch.equal(torch.isnan(got[1]), torch.isnan(w))
    err = (got[1].double() - w).abs().nan_to_num()
    assert bool((err <= (k + 8) * 2.0 ** -22 * w.abs().nan_to_num() + 1e-40).all()), float(err.max())
    assert torch.equal(got[2], o)
    n = int(o[-1])
    assert torch.equal(got[3][:n], s) and bool((got[3][n:] == -7).all())       # behind the last pair: as it was
    few = run(fb, logits, bias, k, lists=False, score=score, groups=groups, top_groups=top_groups, group_top=group_top, renormalize=renormalize, scale=scale)
    assert torch.equal(few[0], got[0]) and torch.equal(few[1].view(torch.int32), got[1].view(torch.int32)) and bool((few[2] == -7).all())


# T, E, k, type, score, bias, groups, top_groups, group_top, renorm: one token, one expert, one place; all experts; widths of every form; one workgroup and several, with part of one
CASES = [(1, 16, 2, "bf16", "softmax", False, 1, 1, 1, True), (1, 1, 1, "f32", "sigmoid", True, 1, 1, 1, True), (3, 5, 5, "f32", "softmax", False, 1, 1, 1, False),
         (7, 64, 8, "f32", "sigmoid", True, 8, 4, 2, True), (33, 60, 4, "bf16", "softmax", True, 4, 2, 1, True), (64, 256, 8, "f32", "sigmoid", True, 8, 4, 2, True),
         (65, 256, 16, "bf16", "softmax", False, 1, 1, 1, True), (100, 255, 7, "f32", "softmax", True, 5, 3, 2, False), (256, 128, 6, "bf16", "sigmoid", False, 2, 1, 2, True),
         (257, 128, 6, "bf16", "sigmoid", False, 1, 1, 1, False), (300, 8, 2, "f32", "softmax", False, 1, 1, 1, True), (700, 160, 6, "f32", "softmax", False, 8, 3, 1, False),
         (20, 1024, 64, "f32", "softmax", False, 1, 1, 1, True), (200, 320, 10, "bf16", "sigmoid", True, 64, 32, 2, True), (90, 64, 33, "f32", "sigmoid", False, 32, 32, 1, True),
         (2500, 512, 3, "f32", "sigmoid", True, 16, 5, 2, True), (64, 64, 64, "f32", "softmax", True, 1, 1, 1, True), (5000, 64, 2, "bf16", "softmax", False, 1, 1, 1, True),
         (129, 4, 4, "bf16", "sigmoid", True, 2, 2, 2, True)]


@pytest.mark.parametrize("T,E,k,type,score,bias,groups,top_groups,group_top,renorm", CASES)
def test_random(fb, T, E, k, type, score, bias, groups, top_groups, group_top, renorm):
    g = torch.Generator().manual_seed(T * 31 + E)
    logits = (1.5 * torch.randn((T, E), generator=g) + 0.5 * torch.randn((E,), generator=g)).to(T_[type])
    b = 0.1 * torch.randn((E,), generator=g) if bias else None
    check(fb, logits, b, k, score, groups, top_groups, group_top, renorm, 2.5)


@pytest.mark.parametrize("score,bias,groups", [("softmax", False, 1), ("sigmoid", True, 1), ("softmax", True, 4), ("sigmoid", False, 4)])
@pytest.mark.parametrize("T", [40, 500])
def test_masked_and_broken_rows(fb, T, score, bias, groups):
    """Experts that are away, in some rows all of them or all but one; the type's lowest value; infinities and NaN, also in groups that do not take part; equal logits."""
    g = torch.Generator().manual_seed(T)
    E, k = 32, 6
    logits = torch.randn((T, E), generator=g).bfloat16().float()
    logits[torch.rand((T, E), generator=g) < 0.4] = -math.inf
    logits[0] = -math.inf
    logits[1, 1:] = -math.inf
    logits[2] = torch.finfo(torch.float32).min
    logits[3, 4] = math.nan
    logits[4, 31] = math.inf
    logits[5] = 0.25                                                            # ties: the lowest experts, in order
    logits[6, 8:] = torch.finfo(torch.float32).min
    logits[7, :16] = -math.inf
    logits[8, 5] = 88.0
    b = (torch.randint(-2, 3, (E,), generator=g).float() / 8) if bias else None
    if bias:
        b[3] = -math.inf                                                        # an expert that nobody gets
    check(fb, logits, b, k, score, groups, min(2, groups), 2, True, 1.0)
    if bias:
        b[9] = math.nan
        check(fb, logits, b, k, score, groups, min(2, groups), 2, False, 1.0)


def test_ties_of_scores_next_to_each_other(fb):
    """Logits one step of float apart, and a bias that nearly evens them out: the order is that of 64 bits."""
    g = torch.Generator().manual_seed(2)
    base = torch.randn((400, 1), generator=g)
    step = torch.randint(-2, 3, (400, 64), generator=g)
    logits = (base.view(torch.int32) + step.to(torch.int32)).view(torch.float32)
    check(fb, logits, None, 8, "sigmoid")
    check(fb, logits, None, 8, "softmax")
    check(fb, logits, torch.randint(-1, 2, (64,), generator=g).float() * 2.0 ** -25, 8, "sigmoid")


def test_many_tokens(fb):
    """More pairs than a few workgroups hold: the order of all of them, by a stable sort."""
    g = torch.Generator().manual_seed(4)
    T, E, k = 50001, 256, 8
    logits = torch.randn((T, E), generator=g)
    logits[torch.rand((T,), generator=g) < 0.01] = -math.inf
    ids, w, o, s = run(fb, logits, None, k)
    want = logits.sort(dim=1, descending=True, stable=True).indices[:, :k].to(torch.int32)         # (topk leaves the order of equal ones open)
    alive = logits[:, 0] > -math.inf
    assert torch.equal(ids[alive], want[alive]) and bool((ids[~alive] == -1).all()) and bool((w[~alive] == 0).all())
    flat = ids.view(-1).long()
    n = int((flat >= 0).sum())
    order = torch.where(flat < 0, E, flat).sort(stable=True).indices[:n]
    assert torch.equal(s[:n].long(), order) and torch.equal(o.long(), torch.cat((torch.zeros(1, dtype=torch.int64), torch.bincount(flat[flat >= 0], minlength=E).cumsum(0))))
    again = run(fb, logits, None, k)
    assert all(torch.equal(a, b) for a, b in zip((ids, o, s), (again[0], again[2], again[3])))


def test_rows_with_gaps_and_none(fb):
    logits = torch.randn((50, 40), device=DEV)
    ids, w = torch.zeros((50, 3), dtype=torch.int32, device=DEV), torch.zeros((50, 3), device=DEV)
    fb.fise_route_experts(fb.route_args(logits[:, 3:36], ids, w))
    assert torch.equal(ids.long(), logits[:, 3:36].sort(dim=1, descending=True, stable=True).indices[:, :3])
    o = torch.full((34,), 5, dtype=torch.int32, device=DEV)
    fb.fise_route_experts(fb.route_args(logits[:0, 3:36], ids[:0], w[:0], o, ids.view(-1)[:0]))
    assert bool((o == 5).all())


@pytest.mark.parametrize("type", ["bf16", "f32"])
def test_zeros_of_both_signs_and_negative_ties(fb, type):
    """Zeros of both signs are one number, negative logits tie like positive ones; keys that cancel in a group's sum."""
    g = torch.Generator().manual_seed(21)
    z = torch.where(torch.rand((60, 32), generator=g) < 0.5, 0.0, -0.0).to(T_[type])
    check(fb, z, None, 5)
    check(fb, -torch.randint(0, 4, (60, 32), generator=g).to(T_[type]), None, 7, "sigmoid")
    b = torch.cat((torch.full((16,), -1.0), torch.zeros(16)))[torch.randperm(32, generator=g)]
    check(fb, torch.randn((300, 32), generator=g).to(T_[type]), b, 4, "sigmoid", 8, 3, 2, True, 1.0)
    check(fb, torch.randn((300, 32), generator=g).to(T_[type]), b * 1e4, 4, "softmax", 8, 3, 2, False, 1.0)
