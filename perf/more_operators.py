"""Operators of transformer denoisers with experts, as timeable cases: rotary positions on several axes, products in 8-bit floating point with a
scale for each block of 128, routing of tokens to experts, and the experts' gated feed-forward with its weighted sum.

Widths are those of the SD-1.5-shaped UNet the benchmark runs (320 / 640 / 1280 channels, feed-forwards of 1280 - 5120, 64 x 64 tokens in tiles of 8 x 8)
and generic ones (powers of two, odd sizes).  Weights are e4m3 codes with one float scale for 128 x 128 of them, activations normal with a few large
channels, logits normal with experts that are liked more than others.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2, "e4m3": 1}
BLOCK, TOP = 128, 448.0                       # columns of a scale, largest value of e4m3


def listed():
    return [
        # the shared key part and 16 heads of one new token, far along a long sequence
        dict(name="rotary_token_16x64", kind="rotary", B=1, grid="1 1 1", M=1, tile=0, n=0, heads=16, d=64, start=0, axes="64", pairing="halves", shared=False,
             far=1000000, keys=1, type="bf16", inverse=False),
        # the active tokens of an edit: the rotated part of queries of 8 heads, and their shared key into the map of latent vectors
        dict(name="rotary_edit_768of4096", kind="rotary", B=2, grid="1 64 64", M=768, tile=8, n=12, heads=8, d=72, start=40, axes="16 16", pairing="adjacent",
             shared=False, far=0, keys=160, type="bf16", inverse=False),
        # queries and keys of every token of a short video, time, height and width
        dict(name="rotary_video_16x64x64", kind="rotary", B=1, grid="16 64 64", M=65536, tile=0, n=0, heads=16, d=128, start=0, axes="16 56 56", pairing="adjacent",
             shared=False, far=0, keys=0, type="bf16", inverse=False),
        # the first layer of a time embedding, one step of one image
        dict(name="fp8_time_embed_1x1280x320", kind="fp8", M=1, N=1280, K=320, x="f32", y="f32", residual=False),
        # feed-forward of the deepest level with the few tokens that a small mask leaves there, odd widths, added to what is there
        dict(name="fp8_tokens_54x1283x5136", kind="fp8", M=54, N=1283, K=5136, x="bf16", y="bf16", residual=True),
        # the first feed-forward product of the active tokens of an edit, rows in 8 bits already
        dict(name="fp8_edit_1536x10240x1280", kind="fp8", M=1536, N=10240, K=1280, x="e4m3", y="bf16", residual=False),
        # a wide layer of a large model, every token of a batch
        dict(name="fp8_dense_8192x8192x8192", kind="fp8", M=8192, N=8192, K=8192, x="bf16", y="bf16", residual=False),
        # one token among a few experts
        dict(name="route_token_1of16", kind="route", T=1, E=16, k=2, type="bf16", score="softmax", bias=False, groups=1, top_groups=1, group_top=1, renorm=True, masked=False),
        # every token of a batch of large latents among many experts, balanced by a bias, experts in groups
        dict(name="route_dense_65536of256", kind="route", T=65536, E=256, k=8, type="f32", score="sigmoid", bias=True, groups=8, top_groups=4, group_top=2, renorm=True, masked=False),
        # one token
        dict(name="experts_token_1x1280_2of16", kind="experts", T=1, K=1280, I=640, E=16, k=2, x="bf16", residual=True),
        # a batch of single tokens, more experts than they need
        dict(name="experts_tokens_64x2048_6of64", kind="experts", T=64, K=2048, I=1408, E=64, k=6, x="bf16", residual=True),
        # every token of a batch of large latents
        dict(name="experts_dense_16384x4096_8of64", kind="experts", T=16384, K=4096, I=1536, E=64, k=8, x="bf16", residual=True),
    ]


def _numbers(text):
    return [int(n) for n in text.split()]


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 4e12, w["flops"] / 2e15)


def draw(rng):
    def between(lo, hi):             # whole number, its logarithm uniform
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotary", "fp8", "fp8", "route", "experts", "experts"])
    top = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in ("rotary", "fp8", "route", "experts")}
    while True:
        if kind == "rotary":
            tile = rng.choice([0, 0, 1, 2, 4, 8])
            T, H, W = rng.choice([1, 1, between(2, 32)]), 8 * between(1, 16), 8 * between(1, 16)
            tokens = T * H * W
            n = between(1, tokens // tile ** 2) if tile else 0
            axes = rng.choice([[16, 56, 56], [32, 32], [16, 16], [20, 22, 22], [64], [24, 20, 20]])
            far = rng.choice([0, 0, 4096, 1000000]) if not tile else 0
            M = n * tile * tile if tile else between(1, 4096) if far else tokens
            rot, start = sum(axes), rng.choice([0, 0, 40, 128])
            case = dict(kind=kind, B=rng.choice([1, 2, 2, 4]), grid=f"{T} {H} {W}", M=M, tile=tile, n=n, heads=between(1, 32), d=rot + start, start=start,
                        axes=" ".join(map(str, axes)), pairing=rng.choice(["adjacent", "adjacent", "halves", "axis_halves"]), shared=rng.random() < 0.3, far=far,
                        keys=rng.choice([0, 1, rot + 128]), type=rng.choice(["bf16", "bf16", "f32"]), inverse=rng.random() < 0.25)
        elif kind == "fp8":
            x = rng.choice(["bf16", "bf16", "f32", "e4m3"])
            case = dict(kind=kind, M=between(1, 16384), N=between(64, 16384), K=16 * between(4, 640), x=x,
                        y=rng.choice(["bf16", "bf16", "f32"]), residual=rng.random() < 0.3)
        elif kind == "route":
            E = rng.choice([4, 8, 16, 32, 60, 64, 128, 160, 256])
            groups = rng.choice([1, 1] + [g for g in (2, 4, 8) if E % g == 0 and E // g >= 2])
            top_groups = rng.randint(max(1, groups // 2), groups)
            k = rng.choice([k for k in (1, 2, 4, 6, 8) if k <= top_groups * (E // groups)])
            case = dict(kind=kind, T=between(1, 65536), E=E, k=k, type=rng.choice(["bf16", "f32"]), score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5,
                        groups=groups, top_groups=top_groups, group_top=rng.choice([1, 2]), renorm=rng.random() < 0.7, masked=rng.random() < 0.3)
        else:
            E = rng.choice([4, 8, 16, 32, 64, 128, 256])
            case = dict(kind=kind, T=between(1, 16384), K=16 * between(8, 256), I=16 * between(4, 160), E=E, k=rng.choice([k for k in (1, 2, 4, 6, 8) if k <= E]),
                        x=rng.choice(["bf16", "bf16", "f32"]), residual=rng.random() < 0.7)
            if 3 * E * case["K"] * case["I"] > 1.3e9:
                continue
        if _cost(case) <= top[kind]:
            return case


# --------------------------------------------------------------------------- inputs
def _normal(g, shape, std=1.0, mean=0.0, type="f32"):
    return torch.empty(shape, device=DEV).normal_(mean, std, generator=g).to(TYPES[type])


def _rows_of(g, M, K, type):
    """Activations: a channel in a hundred is twenty times as large as the others."""
    loud = 1.0 + 19.0 * (torch.rand((K,), generator=g, device=DEV) < 0.01)
    return (torch.empty((M, K), device=DEV).normal_(0.0, 1.0, generator=g) * loud).to(TYPES[type])


def _weights(g, lead, N, K):
    """Codes [*lead, N, K] of e4m3 and the scale of each 128 x 128 of them, as a checkpoint keeps them: the largest magnitude of a block is 448 of its scales."""
    shape = (*lead, -(-N // BLOCK), -(-K // BLOCK))
    scale = (torch.rand(shape, generator=g, device=DEV) + 0.5).mul_(3.0 / (TOP * math.sqrt(K)))
    codes = torch.empty((*lead, N, K), dtype=torch.float8_e4m3fn, device=DEV)
    flat = codes.view(-1, N, K)
    for i in range(flat.shape[0]):
        flat[i] = torch.empty((N, K), device=DEV).normal_(0.0, TOP / 4.0, generator=g).clamp_(-TOP, TOP).to(torch.float8_e4m3fn)
    return codes, scale


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    if case["kind"] == "rotary":
        B, M, heads, d, rot, t = case["B"], case["M"], case["heads"], case["d"], sum(_numbers(case["axes"])), case["type"]
        s = dict(q=_normal(g, (B, M, heads, d), type=t), idx=None, pos=None)
        if case["tile"]:
            T, H, W = _numbers(case["grid"])
            tiles = T * (H // case["tile"]) * (W // case["tile"])
            s["idx"] = torch.randperm(tiles, generator=g, device=DEV)[:case["n"]].sort().values.to(torch.int32)
        if case["far"]:
            s["pos"] = torch.randint(case["far"] // 2, case["far"], (B, M, len(_numbers(case["axes"]))), generator=g, device=DEV).to(torch.int32)
        s["theta"] = [10000.0, 10000.0, 1000.0][:len(_numbers(case["axes"]))]
        if case["keys"] == 0:                                      # keys like the queries
            s["k"] = _normal(g, (B, M, heads, d), type=t)
        else:                                                      # one key of all heads
            s["k"] = _normal(g, (B, M, 1, rot), type=t)
        if case["keys"] > 1:                                       # that goes into the last channels of a map of latent vectors
            rows = math.prod(_numbers(case["grid"])) if not case["far"] else M
            s["map"] = _normal(g, (B, rows, case["keys"]), type=t)
        return s
    if case["kind"] == "fp8":
        M, N, K = case["M"], case["N"], case["K"]
        y = case["y"]
        s = dict(bias=_normal(g, (N,), 0.1, type=y), residual=_normal(g, (M, N), type=y) if case["residual"] else None)
        s["w"], s["w_scale"] = _weights(g, (), N, K)
        if case["x"] == "e4m3":
            s["x"] = torch.empty((M, K), device=DEV).normal_(0.0, TOP / 4.0, generator=g).clamp_(-TOP, TOP).to(torch.float8_e4m3fn)
            s["x_scale"] = torch.rand((-(-K // BLOCK), M), generator=g, device=DEV).add_(0.5).mul_(4.0 / TOP)
        else:
            s["x"], s["x_scale"] = _rows_of(g, M, K, case["x"]), None
        return s
    if case["kind"] == "route":
        T, E = case["T"], case["E"]
        liked = torch.empty((E,), device=DEV).normal_(0.0, 0.5, generator=g)
        logits = torch.empty((T, E), device=DEV).normal_(0.0, 1.5, generator=g).add_(liked).to(TYPES[case["type"]])
        if case["masked"]:                                         # experts that are away, and rows that have none
            logits[torch.rand((T, E), generator=g, device=DEV) < 0.2] = -math.inf
            logits[torch.rand((T,), generator=g, device=DEV) < 0.05] = -math.inf
        return dict(logits=logits, bias=_normal(g, (E,), 0.1) if case["bias"] else None)
    T, K, I, E, k = (case[n] for n in ("T", "K", "I", "E", "k"))
    liked = torch.empty((E,), device=DEV).normal_(0.0, 0.5, generator=g)
    picks = torch.empty((T, E), device=DEV).normal_(0.0, 1.0, generator=g).add_(liked).topk(k, 1)
    s = dict(ids=picks.indices.to(torch.int32), weights=torch.softmax(picks.values, 1), x=_rows_of(g, T, K, case["x"]),
             residual=_normal(g, (T, K), type="bf16") if case["residual"] else None)
    flat = s["ids"].view(-1).long()
    s["slots"] = flat.sort(stable=True).indices.to(torch.int32)
    s["offsets"] = torch.cat((flat.new_zeros(1), torch.bincount(flat, minlength=E).cumsum(0))).to(torch.int32)
    s["w_in"], s["w_in_scale"] = _weights(g, (E, 2), I, K)
    s["w_out"], s["w_out_scale"] = _weights(g, (E,), K, I)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    from paper_2305_17423_amd import binding as fb
    s["fb"] = fb
    if case["kind"] == "rotary":
        s["q_out"] = torch.empty_like(s["q"])
        out, key_map = torch.empty_like(s["k"]), False
        if "map" in s:
            rot = sum(_numbers(case["axes"]))
            out, key_map = s["map"][:, :, None, case["keys"] - rot:], not case["far"]
        s["k_out"] = out
        s["args"] = fb.rotary_args([fb.rotary_tensor(s["q"], s["q_out"], start=case["start"]),
                                    fb.rotary_tensor(s["k"], out, start=case["start"] if case["keys"] == 0 else 0, y_is_map=key_map)],
                                   axes=_numbers(case["axes"]), theta=s["theta"], pos=s["pos"], grid=_numbers(case["grid"]), tile_idx=s["idx"], n_active=case["n"], tile=case["tile"],
                                   pairing=case["pairing"], shared_frequencies=case["shared"], inverse=case["inverse"])
    elif case["kind"] == "fp8":
        s["y"] = torch.empty((case["M"], case["N"]), dtype=TYPES[case["y"]], device=DEV)
        s["args"] = fb.fp8_linear_args(s["x"], s["w"], s["w_scale"], s["y"], x_scale=s["x_scale"], bias=s["bias"], residual=s["residual"])
        s["ws"] = torch.empty(max(fb.fise_fp8_linear_workspace_bytes(s["args"]), 256), dtype=torch.uint8, device=DEV)
    elif case["kind"] == "route":
        T, E, k = case["T"], case["E"], case["k"]
        s["ids"], s["weights"] = torch.empty((T, k), dtype=torch.int32, device=DEV), torch.empty((T, k), device=DEV)
        s["offsets"], s["slots"] = torch.empty(E + 1, dtype=torch.int32, device=DEV), torch.full((T * k,), -1, dtype=torch.int32, device=DEV)
        s["args"] = fb.route_args(s["logits"], s["ids"], s["weights"], s["offsets"], s["slots"], score=case["score"], bias=s["bias"], groups=case["groups"],
                                  top_groups=case["top_groups"], group_top=case["group_top"], renormalize=case["renorm"], scale=1.5)
        s["ws"] = torch.empty(max(fb.fise_route_experts_workspace_bytes(s["args"]), 256), dtype=torch.uint8, device=DEV)
    else:
        s["y"] = torch.empty((case["T"], case["K"]), dtype=torch.bfloat16, device=DEV)
        s["args"] = fb.expert_mlp_args(s["x"], s["ids"], s["weights"], s["offsets"], s["slots"], s["w_in"], s["w_in_scale"], s["w_out"], s["w_out_scale"], s["y"],
                                       residual=s["residual"])
        s["ws"] = torch.empty(max(fb.fise_expert_mlp_workspace_bytes(s["args"]), 256), dtype=torch.uint8, device=DEV)
    return s


# --------------------------------------------------------------------------- one pass
def _tokens(idx, case):
    """Token numbers of the rows: those of the active tiles in list order, row-major inside a tile, or all."""
    T, H, W = _numbers(case["grid"])
    tile = case["tile"]
    if idx is None:
        return torch.arange(T * H * W, device=DEV)
    t, p = idx.long()[:, None], torch.arange(tile * tile, device=DEV)[None, :]
    per_row, per_map = W // tile, (H // tile) * (W // tile)
    y, x = t % per_map // per_row * tile + p // tile, t % per_row * tile + p % tile
    return ((t // per_map * H + y) * W + x).reshape(-1)


def _turned(x, angle, case, start):
    """x [B, M, heads, d] with its pairs turned by angle [B or 1, M, pairs] (64 bits), the other channels as they are."""
    axes, pairs = _numbers(case["axes"]), sum(_numbers(case["axes"])) // 2
    i = torch.arange(pairs, device=DEV)
    if case["pairing"] == "adjacent":
        a, b = 2 * i, 2 * i + 1
    elif case["pairing"] == "halves":
        a, b = i, i + pairs
    else:
        begin = torch.cat([torch.full((n // 2,), sum(axes[:j]), device=DEV) for j, n in enumerate(axes)])
        a = i + begin // 2
        b = a + torch.cat([torch.full((n // 2,), n // 2, device=DEV) for n in axes])
    c, s = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    if case["inverse"]:
        s = -s
    y = x.float()
    u, v = y[..., start + a], y[..., start + b]
    y = y.clone()
    y[..., start + a] = u * c - v * s
    y[..., start + b] = u * s + v * c
    return y.to(x.dtype)


def _plain_rotary(s, case):
    axes, far = _numbers(case["axes"]), case["far"]
    tokens = None if far else _tokens(s["idx"], case)
    T, H, W = _numbers(case["grid"])
    if far:
        pos = s["pos"].double()
    else:
        pos = torch.stack((tokens // (H * W), tokens // W % H, tokens % W)[3 - len(axes):], -1)[None].double() if len(axes) > 1 else tokens[None, :, None].double()
    total, parts, first = sum(axes), [], 0
    for j, n in enumerate(axes):
        e = torch.arange(n // 2, device=DEV, dtype=torch.float64)
        e = 2.0 * (e + first) / total if case["shared"] else 2.0 * e / n
        parts.append(pos[..., j:j + 1] * s["theta"][0 if case["shared"] else j] ** -e)
        first += n // 2
    angle = torch.cat(parts, -1)
    q = _turned(s["q"], angle, case, case["start"])
    k = _turned(s["k"], angle, case, case["start"] if case["keys"] == 0 else 0)
    if "map" not in s:
        return q, k
    if far:
        s["map"][..., case["keys"] - total:] = k[:, :, 0]
    else:
        s["map"][:, tokens, case["keys"] - total:] = k[:, :, 0]
    return q, s["map"]


def _eight(x):
    """Values that rows have in e4m3 with a scale, a power of two, for 128 columns: the smallest that leaves none above 448."""
    M, K = x.shape
    pad = -K % BLOCK
    v = torch.cat((x, x.new_zeros((M, pad))), 1).view(M, -1, BLOCK) if pad else x.view(M, -1, BLOCK)
    m, e = torch.frexp(v.abs().amax(-1, keepdim=True))                # = m 2^e with m in [0.5, 1), and 448 = 0.875 2^9
    e = torch.clamp(e - 9 + (m > 0.875).to(e.dtype), min=-126)
    q = torch.ldexp(v, -e).to(torch.float8_e4m3fn).float()
    return torch.ldexp(q, e).view(M, K + pad)[:, :K]


def _wide(codes, scale):
    """Weights from their codes [N, K] and scales."""
    N, K = codes.shape
    return codes.float() * scale.repeat_interleave(BLOCK, 0)[:N].repeat_interleave(BLOCK, 1)[:, :K]


def _plain_fp8(s, case):
    K = case["K"]
    if s["x_scale"] is None:
        x = _eight(s["x"].float())
    else:
        x = s["x"].float() * s["x_scale"].t().repeat_interleave(BLOCK, 1)[:, :K]
    y = x @ _wide(s["w"], s["w_scale"]).t() + s["bias"].float()
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(TYPES[case["y"]])


def _plain_route(s, case):
    T, E, k, G = case["T"], case["E"], case["k"], case["groups"]
    l = s["logits"].double()
    there = l > -math.inf
    if case["score"] == "softmax":
        top = l.amax(1, keepdim=True)
        p = torch.exp(l - torch.where(top > -math.inf, top, torch.zeros_like(top)))
        total = p.sum(1, keepdim=True)
        score = p / torch.where(total > 0, total, torch.ones_like(total))
    else:
        score = 1.0 / (1.0 + torch.exp(-l))
    key = (score if s["bias"] is None else score + s["bias"].double()).masked_fill(~there, -math.inf)
    if G > 1:
        best = key.view(T, G, E // G).sort(dim=-1, descending=True).values[..., :case["group_top"]]
        of_group = torch.where(best > -math.inf, best, torch.zeros_like(best)).sum(-1).masked_fill(best[..., 0] == -math.inf, -math.inf)
        chosen = of_group.sort(dim=-1, descending=True, stable=True).indices[:, :case["top_groups"]]
        keep = torch.zeros((T, G), dtype=torch.bool, device=DEV).scatter_(1, chosen, True)
        key = key.masked_fill(~keep.repeat_interleave(E // G, 1), -math.inf)
    order = key.sort(dim=1, descending=True, stable=True)
    ids, taken = order.indices[:, :k], order.values[:, :k] > -math.inf
    w = torch.where(taken, score.gather(1, ids), torch.zeros((), dtype=torch.float64, device=DEV))
    if case["renorm"]:
        total = w.sum(1, keepdim=True)
        w = w / torch.where(total > 0, total, torch.ones_like(total))
    ids = torch.where(taken, ids, torch.full_like(ids, -1))
    flat = torch.where(ids < 0, torch.full_like(ids, E), ids).reshape(-1)
    count = torch.zeros(E + 1, dtype=torch.int64, device=DEV).scatter_add_(0, flat, torch.ones_like(flat))
    offsets = torch.cat((count.new_zeros(1), count[:E].cumsum(0)))
    slots = flat.sort(stable=True).indices
    slots = torch.where(torch.arange(T * k, device=DEV) < offsets[E], slots, torch.full_like(slots, -1))
    return ids.to(torch.int32), (1.5 * w).float(), offsets.to(torch.int32), slots.to(torch.int32)


def _plain_experts(s, case):
    T, k = case["T"], case["k"]
    x = _eight(s["x"].float())
    y = torch.zeros((T, case["K"]), device=DEV) if s["residual"] is None else s["residual"].float()
    ends = s["offsets"].tolist()
    for e in range(case["E"]):
        if ends[e] == ends[e + 1]:
            continue
        pair = s["slots"][ends[e]:ends[e + 1]].long()
        rows = x[pair // k]
        gate, up = (rows @ _wide(s["w_in"][e, j], s["w_in_scale"][e, j]).t() for j in (0, 1))
        h = _eight(gate / (1.0 + torch.exp(-gate)) * up)
        y.index_add_(0, pair // k, s["weights"].view(-1)[pair][:, None] * (h @ _wide(s["w_out"][e], s["w_out_scale"][e]).t()))
    return y.to(torch.bfloat16)


def run(state):
    case = state["case"]
    if not own:
        return {"rotary": _plain_rotary, "fp8": _plain_fp8, "route": _plain_route, "experts": _plain_experts}[case["kind"]](state, case)
    fb = state["fb"]
    if case["kind"] == "rotary":
        fb.fise_rotary(state["args"])
        return state["q_out"], state["map"] if "map" in state else state["k_out"]
    if case["kind"] == "fp8":
        fb.fise_fp8_linear(state["args"], state["ws"])
        return state["y"]
    if case["kind"] == "route":
        fb.fise_route_experts(state["args"], state["ws"])
        return state["ids"], state["weights"], state["offsets"], state["slots"]
    fb.fise_expert_mlp(state["args"], state["ws"])
    return state["y"]


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["kind"] == "rotary":
        rows, e = case["B"] * case["M"], SIZE[case["type"]]
        keys = case["heads"] * case["d"] if case["keys"] == 0 else sum(_numbers(case["axes"]))
        return {"bytes": 2 * rows * (case["heads"] * case["d"] + keys) * e, "flops": 3 * rows * (case["heads"] * sum(_numbers(case["axes"])) + keys)}
    if case["kind"] == "fp8":
        M, N, K = case["M"], case["N"], case["K"]
        y, blocks = SIZE[case["y"]], -(-K // BLOCK)
        return {"bytes": N * K + 4 * -(-N // BLOCK) * blocks + M * K * SIZE[case["x"]] + (4 * M * blocks if case["x"] == "e4m3" else 0) + N * y
                + (2 if case["residual"] else 1) * M * N * y, "flops": 2 * M * N * K}
    if case["kind"] == "route":
        T, E, k = case["T"], case["E"], case["k"]
        return {"bytes": T * E * SIZE[case["type"]] + T * k * 12 + 4 * E, "flops": T * E * 8}
    T, K, I, E, k = (case[n] for n in ("T", "K", "I", "E", "k"))
    used = E * (1.0 - (1.0 - k / E) ** T)                             # experts that some token picks
    return {"bytes": used * (3 * K * I * (1.0 + 4.0 / BLOCK ** 2)) + T * K * (SIZE[case["x"]] + (4 if case["residual"] else 2)) + 12 * T * k, "flops": 6 * T * k * K * I}


# --------------------------------------------------------------------------- the definitions in 64 bits
def _exact_rows(x):
    """Rows in e4m3 times a power of two for 128 columns, and back: the nearest value, ties to the even code."""
    x = x.to(torch.float64)
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], BLOCK):
        v = x[:, c:c + BLOCK]
        largest = v.abs().amax(1, keepdim=True)
        e = torch.ceil(torch.log2(torch.clamp(largest, min=1e-300) / TOP))
        e = torch.where(largest > TOP * torch.exp2(e), e + 1, torch.where(largest <= TOP * torch.exp2(e - 1), e - 1, e)).clamp(min=-126.0)
        u = v / torch.exp2(e)
        step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3)
        out[:, c:c + BLOCK] = torch.round(u / step) * step * torch.exp2(e)
    return out


def _exact_product(x, codes, scale):
    """x (64 bits) times the weights: block by block of columns."""
    N, K = codes.shape
    y = torch.zeros((x.shape[0], N), dtype=torch.float64, device=DEV)
    for c in range(0, K, 1024):
        w = codes[:, c:c + 1024].to(torch.float64)
        for n in range(0, N, BLOCK):
            w[n:n + BLOCK] *= scale[n // BLOCK, c // BLOCK:(c + 1024) // BLOCK].to(torch.float64).repeat_interleave(BLOCK)[None, :w.shape[1]]
        y += x[:, c:c + 1024].contiguous() @ w.t().contiguous()
    return y


def exact(case, seed):
    s = _inputs(case, seed)
    f64 = torch.float64
    if case["kind"] == "rotary":
        T, H, W = _numbers(case["grid"])
        axes, half = _numbers(case["axes"]), sum(_numbers(case["axes"])) // 2
        grid = torch.arange(T * H * W, device=DEV).view(T, H, W)
        if case["tile"]:
            t = case["tile"]
            grid = grid.view(T, H // t, t, W // t, t).transpose(2, 3).reshape(-1, t * t)[s["idx"].long()]
        token = grid.reshape(-1)
        where = {1: [token], 2: [token % (H * W) // W, token % W], 3: [token // (H * W), token % (H * W) // W, token % W]}[len(axes)]

        def turned(x, start):
            y = x.to(f64)
            first, begin = 0, 0
            for j, n in enumerate(axes):
                place = s["pos"][..., j].to(f64) if case["far"] else where[j].to(f64)[None]
                for i in range(n // 2):
                    w = s["theta"][0] ** (-2.0 * (first + i) / (2 * half)) if case["shared"] else s["theta"][j] ** (-2.0 * i / n)
                    a, b = {"adjacent": (2 * (first + i), 2 * (first + i) + 1), "halves": (first + i, first + i + half),
                            "axis_halves": (begin + i, begin + i + n // 2)}[case["pairing"]]
                    z = torch.complex(x[..., start + a].to(f64), x[..., start + b].to(f64))
                    z = z * torch.polar(torch.ones_like(place), place * (-w if case["inverse"] else w))[:, :, None]
                    y[..., start + a], y[..., start + b] = z.real, z.imag
                first, begin = first + n // 2, begin + n
            return y
        q, k = turned(s["q"], case["start"]), turned(s["k"], case["start"] if case["keys"] == 0 else 0)
        if "map" not in s:
            return q, k
        rows = torch.arange(case["M"], device=DEV) if case["far"] else token
        out = s["map"].to(f64)
        out[:, rows, case["keys"] - 2 * half:] = k[:, :, 0]
        return q, out
    if case["kind"] == "fp8":
        if s["x_scale"] is None:
            x = _exact_rows(s["x"])
        else:
            x = s["x"].to(f64)
            for c in range(0, case["K"], BLOCK):
                x[:, c:c + BLOCK] *= s["x_scale"][c // BLOCK][:, None].to(f64)
        y = _exact_product(x, s["w"], s["w_scale"]) + s["bias"].to(f64)
        return y if s["residual"] is None else y + s["residual"].to(f64)
    if case["kind"] == "route":
        T, E, k, G = case["T"], case["E"], case["k"], case["groups"]
        l = s["logits"].to(f64)
        score = torch.nan_to_num(torch.softmax(l, 1), nan=0.0) if case["score"] == "softmax" else torch.sigmoid(l)
        key = score.clone() if s["bias"] is None else score + s["bias"].to(f64)
        key[torch.isneginf(l)] = -math.inf

        def first_of(values):                                         # the largest, the lowest index among equals
            best = values.amax(1)
            return best, (values == best[:, None]).to(torch.uint8).argmax(1)
        row = torch.arange(T, device=DEV)
        if G > 1:
            of_group = torch.full((T, G), -math.inf, dtype=f64, device=DEV)
            for j in range(G):
                members = key[:, j * (E // G):(j + 1) * (E // G)].clone()
                for i in range(case["group_top"]):
                    best, at = first_of(members)
                    of_group[:, j] = torch.where(best == -math.inf, of_group[:, j], best if i == 0 else of_group[:, j] + best)
                    members[row, at] = -math.inf
            allowed = torch.zeros((T, G), dtype=torch.bool, device=DEV)
            for i in range(case["top_groups"]):
                best, at = first_of(of_group)
                allowed[row, at] |= best > -math.inf
                of_group[row, at] = -math.inf
            key[~allowed.repeat_interleave(E // G, 1)] = -math.inf
        ids, weights = torch.full((T, k), -1, dtype=torch.int32, device=DEV), torch.zeros((T, k), dtype=f64, device=DEV)
        for j in range(k):
            best, at = first_of(key)
            some = best > -math.inf
            ids[:, j] = torch.where(some, at, -1).to(torch.int32)
            weights[:, j] = torch.where(some, score[row, at], 0.0)
            key[row, at] = -math.inf
        if case["renorm"]:
            weights = torch.nan_to_num(weights / weights.sum(1, keepdim=True), nan=0.0)
        flat = ids.view(-1)
        slots, offsets, filled = torch.full((T * k,), -1, dtype=torch.int32, device=DEV), [0], 0
        for e in range(E):
            mine = (flat == e).nonzero()[:, 0]
            slots[filled:filled + mine.numel()] = mine.to(torch.int32)
            filled += mine.numel()
            offsets.append(filled)
        return ids, 1.5 * weights, torch.tensor(offsets, dtype=torch.int32, device=DEV), slots
    T, K, I, E, k = (case[n] for n in ("T", "K", "I", "E", "k"))
    x, ids, weights = _exact_rows(s["x"]), s["ids"].long(), s["weights"].to(f64)
    y = torch.zeros((T, K), dtype=f64, device=DEV) if s["residual"] is None else s["residual"].to(f64)
    for e in range(E):
        token, j = (ids == e).nonzero(as_tuple=True)
        if token.numel() == 0:
            continue
        gate, up = (_exact_product(x[token], s["w_in"][e, i], s["w_in_scale"][e, i]) for i in (0, 1))
        h = _exact_rows(gate * torch.sigmoid(gate) * up)
        y[token] += weights[token, j][:, None] * _exact_product(h, s["w_out"][e], s["w_out_scale"][e])
    return y
