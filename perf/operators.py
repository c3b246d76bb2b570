"""Operators of transformer denoisers, as timeable cases: products of a few rows with 4-bit weights, norms around a block with its gate
and its modulation, and attention over a cache of latent vectors.

Widths are those of the SD-1.5-shaped UNet the benchmark runs (320 / 640 / 1280 channels, 8 heads, time projections 20160 x 1280) and
generic ones (powers of two, odd sizes).  Weights are random with 1 / sqrt(columns), activations normal, modulations small.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # the first layer of a time embedding, one step of one image
        dict(name="w4_time_embed_1x1280x320", kind="w4", M=1, N=1280, K=320, group=32, x="f32", y="f32", silu=False, residual=False),
        # the time projections of all ResNet blocks as one product, image and unconditioned image
        dict(name="w4_time_proj_2x20160x1280", kind="w4", M=2, N=20160, K=1280, group=64, x="f32", y="f32", silu=True, residual=False),
        # feed-forward of the deepest level with the few tokens that a small mask leaves there, odd widths, added to what is there
        dict(name="w4_tokens_27x1283x5120", kind="w4", M=27, N=1283, K=5120, group=128, x="bf16", y="bf16", silu=False, residual=True),
        # a wide layer of a large model for a batch of single tokens
        dict(name="w4_wide_16x28672x8192", kind="w4", M=16, N=28672, K=8192, group=128, x="bf16", y="bf16", silu=False, residual=False),
        # the norms around a block on the active tokens of the deepest level
        dict(name="norm_8x8_c1280_3of64", kind="norm", B=2, H=8, W=8, C=1280, tile=1, n=3, type="bf16", post="none", pre="layer", gate=True, mod=True),
        # the same on the finest level of a 512 x 512 image, 12 of 64 tiles
        dict(name="norm_64x64_c320_12of64", kind="norm", B=2, H=64, W=64, C=320, tile=8, n=12, type="bf16", post="rms", pre="layer", gate=True, mod=True),
        # every token of a batch of large latents, wide model, norms before and after the block
        dict(name="norm_dense_64x64_c4096", kind="norm", B=4, H=64, W=64, C=4096, tile=0, n=0, type="bf16", post="rms", pre="rms", gate=True, mod=False),
        # one token against a short cache
        dict(name="latent_token_1000keys", kind="latent", B=1, M=1, n=1000, heads=8, d=64, dr=0, dv=64, r=128, causal=False, ragged=False),
        # the active tokens of an edit (12 of 64 tiles of 8 x 8) against the whole latent map
        dict(name="latent_edit_768of4096", kind="latent", B=2, M=768, n=4096, heads=8, d=40, dr=32, dv=40, r=128, causal=False, ragged=False),
        # a batch of single tokens, caches of different lengths
        dict(name="latent_decode_16x8192", kind="latent", B=16, M=1, n=8192, heads=16, d=128, dr=64, dv=128, r=512, causal=False, ragged=True),
        # a large batch, two tokens each, long caches
        dict(name="latent_decode_32x32768", kind="latent", B=32, M=2, n=32768, heads=32, d=128, dr=64, dv=128, r=512, causal=True, ragged=True),
        # a long prompt attends to itself
        dict(name="latent_prompt_4096", kind="latent", B=1, M=4096, n=4096, heads=16, d=128, dr=64, dv=128, r=512, causal=True, ragged=False),
    ]


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 4e12, w["flops"] / 8e14)


def draw(rng):
    def between(lo, hi):             # whole number, its logarithm uniform
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["w4", "norm", "latent", "latent"])
    top = max(_cost(c) for c in listed())
    while True:
        if kind == "w4":
            x = rng.choice(["bf16", "bf16", "f32"])
            case = dict(kind=kind, M=between(1, 64), N=between(64, 28672), K=8 * between(8, 1024), group=rng.choice([32, 64, 128, 256]), x=x,
                        y=rng.choice([x, x, "f32"]), silu=rng.random() < 0.3, residual=rng.random() < 0.3)
        elif kind == "norm":
            tile = rng.choice([0, 1, 2, 4, 8])
            H, W = 8 * between(1, 12), 8 * between(1, 12)
            n = between(1, H * W // tile ** 2) if tile else 0
            case = dict(kind=kind, B=rng.choice([1, 2, 2, 4]), H=H, W=W, C=8 * between(8, 1024), tile=tile, n=n, type=rng.choice(["bf16", "bf16", "f32"]),
                        post=rng.choice(["none", "rms", "layer"]), pre=rng.choice(["none", "rms", "layer", "layer"]), gate=rng.random() < 0.8,
                        mod=rng.random() < 0.7)
        else:
            tokens = rng.choice(["one", "few", "many"])
            d = rng.choice([32, 40, 64, 80, 128, 160])
            n = between(16, 65536)
            case = dict(kind=kind, B=between(1, 32), M={"one": 1, "few": between(2, 8), "many": between(9, 4096)}[tokens], n=n,
                        heads=rng.choice([4, 8, 16, 32, 64]), d=d, dr=rng.choice([0, 32, 64]), dv=rng.choice([d, d, 64]),
                        r=rng.choice([64, 128, 256, 320, 512]), causal=rng.random() < 0.4, ragged=rng.random() < 0.5)
            if case["B"] * case["heads"] * case["M"] * n > 2 ** 28 or case["M"] > n:
                continue
        if _cost(case) <= top:
            return case


# --------------------------------------------------------------------------- inputs
def _normal(g, shape, std=1.0, mean=0.0, type="f32"):
    return torch.empty(shape, device=DEV).normal_(mean, std, generator=g).to(TYPES[type])


def _lengths(case, g):
    if not case["ragged"]:
        return None
    n = case["n"]
    return torch.randint(n // 4, n + 1, (case["B"],), generator=g, device=DEV).to(torch.int32)


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    if case["kind"] == "w4":
        M, N, K, group = case["M"], case["N"], case["K"], case["group"]
        G = -(-K // group)
        return dict(x=_normal(g, (M, K), type=case["x"]), codes=torch.randint(-8, 8, (N, K), generator=g, device=DEV, dtype=torch.int8),
                    scale=(torch.rand((N, G), generator=g, device=DEV) + 0.5).mul_(0.25 / math.sqrt(K)).to(torch.bfloat16),
                    bias=_normal(g, (N,), 0.1, type=case["y"]), residual=_normal(g, (M, N), type=case["y"]) if case["residual"] else None)
    if case["kind"] == "norm":
        B, H, W, C, tile, t = case["B"], case["H"], case["W"], case["C"], case["tile"], case["type"]
        rows = case["n"] * tile * tile if tile else H * W
        s = dict(x=_normal(g, (B, H, W, C), 1.5, type=t), h=_normal(g, (B, rows, C), 0.7, 0.1, t), r=_normal(g, (B, H, W, C), type=t), idx=None)
        if tile:
            tiles = (H // tile) * (W // tile)
            s["idx"] = torch.randperm(tiles, generator=g, device=DEV)[:case["n"]].sort().values.to(torch.int32)
        for side in ("post", "pre"):
            s[side + "_w"] = _normal(g, (C,), 0.1, 1.0, t) if case[side] != "none" else None
            s[side + "_b"] = _normal(g, (C,), 0.1, type=t) if case[side] == "layer" else None
        s["mod"] = _normal(g, (B, 3 * C), 0.3)                      # gate, scale and shift side by side, as one product leaves them
        return s
    B, M, n, heads, d, dr, dv, r = (case[k] for k in ("B", "M", "n", "heads", "d", "dr", "dv", "r"))
    return dict(q=_normal(g, (B, M, heads, d + dr), type="bf16"), cache=_normal(g, (B, n, r + dr), type="bf16"), kv_len=_lengths(case, g),
                w_uk=_normal(g, (heads, d, r), 1.0 / math.sqrt(r), type="bf16"), w_uv=_normal(g, (heads, dv, r), 1.0 / math.sqrt(r), type="bf16"))


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "norm":
        C, mod = case["C"], s["mod"]
        s["gate"] = mod[:, :C] if case["gate"] else None
        s["scale"], s["shift"] = (mod[:, C:2 * C], mod[:, 2 * C:]) if case["mod"] else (None, None)
    if not own:
        return s
    from paper_2305_17423_amd import binding as fb
    s["fb"] = fb
    if case["kind"] == "w4":
        N, K, group = case["N"], case["K"], case["group"]
        s["packed"] = torch.empty(fb.fise_w4_bytes(N, K, group), dtype=torch.uint8, device=DEV)
        wide = s["scale"].float().repeat_interleave(group, 1)[:, :K]
        fb.fise_w4_pack(s["codes"].float().mul_(wide), s["packed"], group, scale=s["scale"])
        s["y"] = torch.empty((case["M"], N), dtype=TYPES[case["y"]], device=DEV)
        s["args"] = fb.w4_linear_args(s["x"], s["packed"], group, s["y"], bias=s["bias"], residual=s["residual"], silu_in=case["silu"])
    elif case["kind"] == "norm":
        s["y"] = torch.empty_like(s["h"]) if case["pre"] != "none" or case["mod"] else None
        s["args"] = fb.gated_norm_args(s["x"], h=s["h"], post=case["post"], post_w=s["post_w"], post_b=s["post_b"], gate=s["gate"], res_scale=0.75,
                                       pre=case["pre"], pre_w=s["pre_w"], pre_b=s["pre_b"], mod_scale=s["scale"], mod_shift=s["shift"], eps=1e-5,
                                       tile_idx=s["idx"], n_active=case["n"], tile=case["tile"], r=s["r"], y=s["y"])
    else:
        s["out"] = torch.empty((case["B"], case["M"], case["heads"] * case["dv"]), dtype=torch.bfloat16, device=DEV)
        s["args"] = fb.latent_attention_args(s["q"], s["cache"], s["w_uk"], s["w_uv"], s["out"], scale=1.0 / math.sqrt(case["d"] + case["dr"]),
                                             kv_len=s["kv_len"], causal=case["causal"])
        s["ws"] = torch.empty(max(fb.fise_latent_attention_workspace_bytes(s["args"]), 256), dtype=torch.uint8, device=DEV)
    return s


# --------------------------------------------------------------------------- one pass
def _plain_w4(s, case):
    x = s["x"].float()
    if case["silu"]:
        x = x / (1.0 + torch.exp(-x))
    w = s["codes"].float() * s["scale"].float().repeat_interleave(case["group"], 1)[:, :case["K"]]
    y = x @ w.t() + s["bias"].float()
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(TYPES[case["y"]])


def _norm(v, kind, w, b, eps=1e-5):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    if kind != "none":
        v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + eps)
    if w is not None:
        v = v * w.to(v.dtype)
    return v if b is None else v + b.to(v.dtype)


def _rows(idx, case):
    """Token numbers of the active rows, tile by tile in list order, row-major inside a tile."""
    tile, W = case["tile"], case["W"]
    if idx is None:
        return torch.arange(case["H"] * W, device=DEV)
    t, p = idx.long()[:, None], torch.arange(tile * tile, device=DEV)[None, :]
    per = W // tile
    return ((t // per * tile + p // tile) * W + t % per * tile + p % tile).reshape(-1)


def _plain_norm(s, case):
    rows, C = _rows(s["idx"], case), case["C"]
    x = s["x"].view(case["B"], -1, C)[:, rows].float()
    h = _norm(s["h"].float(), case["post"], s["post_w"], s["post_b"])
    if s["gate"] is not None:
        h = s["gate"][:, None] * h
    r = 0.75 * x + h
    s["r"].view(case["B"], -1, C)[:, rows] = r.to(s["r"].dtype)
    if case["pre"] == "none" and not case["mod"]:
        return s["r"]
    y = _norm(r, case["pre"], s["pre_w"], s["pre_b"])
    if s["scale"] is not None:
        y = y * (1.0 + s["scale"][:, None]) + s["shift"][:, None]
    return s["r"], y.to(s["h"].dtype)


def _attend(q, c, lens, w_uk, w_uv, case, dtype):
    """Keys and values of every head from the latent vectors, one batch element at a time."""
    B, M, n, heads, d, r = (case[k] for k in ("B", "M", "n", "heads", "d", "r"))
    few = M * heads < n // 8                                          # few queries: meet the latent vectors themselves
    scale, out = 1.0 / math.sqrt(d + case["dr"]), []
    w_uk, w_uv, keys = w_uk.to(dtype), w_uv.to(dtype), torch.arange(n, device=DEV)
    for b in range(B):
        qb, cb = q[b].to(dtype).transpose(0, 1).contiguous(), c[b].to(dtype)           # [heads, M, d + dr], [n, r + dr]
        length = keys.new_tensor(n) if lens is None else lens[b].long()
        if few:
            full = torch.cat((torch.bmm(qb[..., :d].contiguous(), w_uk), qb[..., d:]), -1)
            s = (full.reshape(heads * M, -1) @ cb.t().contiguous()).view(heads, M, n)
        else:
            k = torch.matmul(cb[:, :r].contiguous(), w_uk.transpose(1, 2).contiguous())           # [heads, n, d]
            s = torch.bmm(qb[..., :d].contiguous(), k.transpose(1, 2).contiguous())
            if case["dr"]:
                s = s + torch.matmul(qb[..., d:].contiguous(), cb[:, r:].t().contiguous())
        seen = keys[None, :] < length
        if case["causal"]:
            seen = keys[None, :] < length - M + 1 + torch.arange(M, device=DEV)[:, None]
        s = (s * scale).masked_fill(~seen, -math.inf)
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
        total = p.sum(-1, keepdim=True)
        p = torch.where(total > 0, p / total, torch.zeros_like(p))
        if few:
            o = torch.bmm((p.reshape(heads * M, n) @ cb[:, :r].contiguous()).view(heads, M, r), w_uv.transpose(1, 2).contiguous())
        else:
            o = torch.bmm(p, torch.matmul(cb[:, :r].contiguous(), w_uv.transpose(1, 2).contiguous()))
        out.append(o.transpose(0, 1).reshape(M, -1))
    return torch.stack(out)


def run(state):
    case = state["case"]
    if not own:
        if case["kind"] == "w4":
            return _plain_w4(state, case)
        if case["kind"] == "norm":
            return _plain_norm(state, case)
        return _attend(state["q"], state["cache"], state["kv_len"], state["w_uk"], state["w_uv"], case, torch.float32).to(torch.bfloat16)
    fb = state["fb"]
    if case["kind"] == "w4":
        fb.fise_w4_linear(state["args"])
        return state["y"]
    if case["kind"] == "norm":
        fb.fise_masked_gated_norm(state["args"])
        return state["r"] if state["y"] is None else (state["r"], state["y"])
    fb.fise_latent_attention(state["args"], state["ws"])
    return state["out"]


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["kind"] == "w4":
        M, N, K = case["M"], case["N"], case["K"]
        y = SIZE[case["y"]]
        return {"bytes": N * K / 2 + 2 * N * -(-K // case["group"]) + M * K * SIZE[case["x"]] + N * y + (2 if case["residual"] else 1) * M * N * y,
                "flops": 2 * M * N * K}
    if case["kind"] == "norm":
        B, C, e = case["B"], case["C"], SIZE[case["type"]]
        rows = B * (case["n"] * case["tile"] ** 2 if case["tile"] else case["H"] * case["W"])
        moved = 4 if case["pre"] != "none" or case["mod"] else 3
        return {"bytes": rows * C * e * moved + B * C * 4 * (case["gate"] + 2 * case["mod"]), "flops": 16 * rows * C}
    B, M, n, heads, d, dr, dv, r = (case[k] for k in ("B", "M", "n", "heads", "d", "dr", "dv", "r"))
    keys = n * (0.625 if case["ragged"] else 1.0)                     # lengths are uniform between a quarter and the whole
    pairs = M * (keys - (M - 1) / 2 if case["causal"] else keys)      # (query, key) of a head
    absorbed = 2 * M * heads * r * (d + dv) + 2 * heads * pairs * (2 * r + dr)
    expanded = 2 * keys * heads * r * (d + dv) + 2 * heads * pairs * (d + dr + dv)
    return {"bytes": 2 * (B * keys * (r + dr) + B * M * heads * (d + dr + dv) + heads * r * (d + dv)), "flops": B * min(absorbed, expanded)}


# --------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    f64 = torch.float64
    if case["kind"] == "w4":
        x = s["x"].to(f64)
        if case["silu"]:
            x = x * torch.sigmoid(x)
        y = torch.empty((case["M"], case["N"]), dtype=f64, device=DEV)
        group = case["group"]
        for n0 in range(0, case["N"], 4096):
            acc = s["bias"][n0:n0 + 4096].to(f64).expand(case["M"], -1).clone()
            for k0 in range(0, case["K"], 1024):                      # (whole groups)
                codes, scale = s["codes"][n0:n0 + 4096, k0:k0 + 1024].to(f64), s["scale"][n0:n0 + 4096, k0 // group:(k0 + 1024) // group].to(f64)
                acc += (x[:, k0:k0 + 1024] @ (codes * scale.repeat_interleave(group, 1)[:, :codes.shape[1]]).t().contiguous())
            y[:, n0:n0 + 4096] = acc
        return y if s["residual"] is None else y + s["residual"].to(f64)
    if case["kind"] == "norm":
        B, H, W, C, tile = case["B"], case["H"], case["W"], case["C"], case["tile"]
        order = torch.arange(H * W, device=DEV).view(H, W)
        if tile:
            order = order.view(H // tile, tile, W // tile, tile).transpose(1, 2).reshape(-1, tile * tile)[s["idx"].long()]
        order = order.reshape(-1)

        def normed(v, kind, w, b):
            if kind == "none":
                return v
            centre = v.mean(-1, keepdim=True) if kind == "layer" else 0.0
            v = (v - centre) / torch.sqrt(((v - centre) ** 2).mean(-1, keepdim=True) + 1e-5) * w.to(f64)
            return v if b is None else v + b.to(f64)
        gate, scale, shift = (t[:, None].to(f64) for t in s["mod"].split(C, 1))
        r_map, ys = s["r"].to(f64).view(B, H * W, C), []
        for b in range(B):
            branch = normed(s["h"][b].to(f64), case["post"], s["post_w"], s["post_b"])
            r = 0.75 * s["x"][b].view(H * W, C)[order].to(f64) + (branch * gate[b] if case["gate"] else branch)
            r_map[b, order] = r
            y = normed(r, case["pre"], s["pre_w"], s["pre_b"])
            ys.append(y * (1.0 + scale[b]) + shift[b] if case["mod"] else y)
        r_map = r_map.view(B, H, W, C)
        return r_map if case["pre"] == "none" and not case["mod"] else (r_map, torch.stack(ys))
    B, M, n, heads, d, r = (case[k] for k in ("B", "M", "n", "heads", "d", "r"))
    if B * heads * M * n * (d + r) > 6e12:
        return None
    out = torch.zeros((B, M, heads, case["dv"]), dtype=f64, device=DEV)
    for b in range(B):
        length = n if s["kv_len"] is None else int(s["kv_len"][b])
        if length == 0:
            continue
        c, pe = s["cache"][b, :length, :r].to(f64), s["cache"][b, :length, r:].to(f64)
        q = s["q"][b].to(f64)
        for h in range(heads):
            logits = (q[:, h, :d] @ s["w_uk"][h].to(f64)) @ c.t() + q[:, h, d:] @ pe.t()
            logits = logits / math.sqrt(d + case["dr"])
            if case["causal"]:
                ahead = torch.arange(length, device=DEV)[None, :] > length - M + torch.arange(M, device=DEV)[:, None]
                logits[ahead] = -math.inf
            p = torch.nan_to_num(torch.softmax(logits, -1), nan=0.0)
            out[b, :, h] = (p @ c) @ s["w_uv"][h].to(f64).t()
    return out.view(B, M, -1)
