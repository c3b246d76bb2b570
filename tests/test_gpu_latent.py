"""GPU checks of attention over a cache of latent vectors, both forms, against 64-bit arithmetic.

Tolerances, from arithmetic: a rounding to bf16 is uniform in half a step, 1.65e-3 of the value in the mean square.  Between the inputs and an output lie those of
the queries behind W_uk or of the keys (which move a probability by that times its score, of standard deviation 1 here, at most 1.5), of the probabilities, of
the values (expanded form), and of the output.  All but the last are independent from key to key, so an output o = sum_j p_j v_j is off by a normal error of
sqrt(1.5^2 + 2) * 1.65e-3 = 3.4e-3 times sqrt(sum_j p_j^2 v_j^2), which the reference adds up, and by half a step of its own: held to 2e-2 times
that root (six standard deviations, for up to a million outputs) + 2^-8 |o|.  (Relative to the root mean square of all outputs this would be wrong: with few keys
a query's outputs are many times as large as with hundreds, and so is what they are off by.)
With many keys one error of the absorbed form is left that does not average out: what rounding takes from channel c of a query behind W_uk, 1.65e-3 |q~_c|, moves every
score by that times the key's channel, and the values have a share w_c of that same channel, of variance 1 here: an error of scale * 1.65e-3 sqrt(sum_c q~_c^2 w_c^2),
six times which is allowed besides (with 1030 keys of 64 channels, and that rounding as the only one, 64-bit arithmetic is off by 1.005 of the tolerance without it at
one of two million outputs).  Over all outputs the relative L2 error is at most
sqrt(1.5^2 + 3) * 1.65e-3 = 3.8e-3, held to 5e-3."""
import math

import pytest
import torch

from helpers import DEV, host, rel_l2

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
L2 = 5e-3
ABSORBED, EXPANDED = 1, 2


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def reference(q, c, wk, wv, lens, scale, causal, form=2):
    q, c, wk, wv = (t.double().cpu() for t in (q, c, wk, wv))
    B, M, H, _ = q.shape
    d, r = wk.shape[1:]
    out = torch.zeros((B, M, H, wv.shape[1]), dtype=torch.float64)
    spread = torch.zeros_like(out)
    for b in range(B):
        n = lens[b]
        if n == 0:
            continue
        k = torch.einsum("jr,hdr->hjd", c[b, :n, :r], wk)
        v = torch.einsum("jr,hvr->hjv", c[b, :n, :r], wv)
        s = torch.einsum("mhd,hjd->hmj", q[b, :, :, :d], k) + torch.einsum("mhd,jd->hmj", q[b, :, :, d:], c[b, :n, r:])
        s = s * scale
        if causal:
            s = s.masked_fill(torch.arange(n)[None, :] > n - M + torch.arange(M)[:, None], -math.inf)
        seen = s.amax(-1, keepdim=True) > -math.inf
        p = torch.where(seen, torch.softmax(s, -1), torch.zeros((), dtype=torch.float64))
        out[b] = torch.einsum("hmj,hjv->mhv", p, v)
        spread[b] = torch.einsum("hmj,hjv->mhv", p ** 2, v ** 2).sqrt()
        if form == ABSORBED:                                                    # (in units of 2e-2)
            spread[b] += 6 * 1.65e-3 / 2e-2 * scale * torch.einsum("mhr,hvr->mhv", torch.einsum("mhd,hdr->mhr", q[b, :, :, :d], wk) ** 2, wv ** 2).sqrt()
    return out.reshape(B, M, -1), spread.reshape(B, M, -1)


def inputs(g, B, M, n, H, d, dr, dv, r, extra=0, poison=None):
    rnd = lambda *s, k=1.0: (k * torch.randn(s, generator=g)).to(BF)
    q, c = rnd(B, M, H, d + dr), rnd(B, n + extra, r + dr)
    if poison is not None:
        for b, ln in enumerate(poison):
            c[b, ln:] = math.nan
    return q.to(DEV), c.to(DEV), rnd(H, d, r, k=1 / math.sqrt(r)).to(DEV), rnd(H, dv, r, k=1 / math.sqrt(r)).to(DEV)


def run(fb, q, c, wk, wv, form, scale, **kw):
    B, M, H, _ = q.shape
    out = torch.full((B, M, H * wv.shape[1]), float("nan"), dtype=BF, device=DEV)
    a = fb.latent_attention_args(q, c, wk, wv, out, scale, form=form, **kw)
    ws = torch.full((fb.fise_latent_attention_workspace_bytes(a),), 0xFF, dtype=torch.uint8, device=DEV)      # NaN, whatever it is read as
    fb.fise_latent_attention(a, ws)
    first = out.clone()
    out.fill_(float("nan"))
    fb.fise_latent_attention(a, ws)                                             # on what the first call left in the workspace
    assert torch.equal(first.view(torch.int16), out.view(torch.int16))          # (bits: NaN compares with nothing)
    return out


def check(got, want, rows=slice(None)):
    want, spread = (t[:, rows] for t in want)
    assert bool(got.isfinite().all())
    off = (got.double().cpu() - want).abs() / (2.0 ** -8 * want.abs() + 2e-2 * spread).clamp_min(1e-30)
    assert float(off.max()) <= 1 and rel_l2(host(got), want.numpy()) <= L2, (float(off.max()), rel_l2(host(got), want.numpy()))


# B, M, keys, heads, d, dr, dv, r: one token and one key, key counts around a block, rows around a tile of 64 and of 128 queries, every width the kernels are built
# for and widths between them, head dims that are no multiple of 16 or 32, more groups than workgroups and the other way round
CASES = [(1, 1, 1, 1, 8, 0, 8, 8), (1, 1, 1000, 8, 64, 0, 64, 128), (2, 1, 33, 16, 128, 64, 128, 512), (3, 5, 31, 13, 40, 32, 40, 128), (2, 17, 64, 4, 80, 0, 80, 320),
         (1, 65, 65, 1, 160, 64, 160, 512), (2, 9, 200, 8, 64, 8, 96, 256), (5, 2, 127, 32, 32, 64, 64, 384), (1, 300, 300, 2, 40, 32, 40, 136), (1, 4, 4100, 8, 128, 64, 128, 512),
         (2, 130, 257, 8, 160, 0, 64, 256), (1, 33, 95, 3, 24, 40, 56, 72), (4, 1, 2049, 64, 128, 64, 128, 512), (1, 200, 64, 16, 128, 64, 128, 512), (2, 768, 1024, 8, 40, 32, 40, 128),
         # a workgroup for every tile of the expanded form: heads in eights and not, several tiles
         (4, 3, 70, 128, 64, 32, 64, 128), (3, 2, 65, 171, 32, 0, 32, 64), (1, 1100, 130, 64, 128, 64, 128, 512), (1, 140, 200, 128, 160, 64, 160, 256),
         (2, 20, 300, 8, 64, 0, 64, 512), (1, 3, 1500, 24, 64, 0, 64, 440), (2, 130, 140, 6, 64, 64, 64, 128), (1, 150, 300, 5, 64, 40, 56, 264)]


@pytest.mark.parametrize("form", [ABSORBED, EXPANDED])
@pytest.mark.parametrize("B,M,n,H,d,dr,dv,r", CASES)
def test_all_keys(fb, B, M, n, H, d, dr, dv, r, form):
    g = torch.Generator().manual_seed(B + M + n + r)
    q, c, wk, wv = inputs(g, B, M, n, H, d, dr, dv, r)
    scale = 1 / math.sqrt(d + dr)
    check(run(fb, q, c, wk, wv, form, scale), reference(q, c, wk, wv, [n] * B, scale, False))


@pytest.mark.parametrize("M,H", [(1, 5), (2, 8), (1, 17), (4, 8), (3, 11)])
@pytest.mark.parametrize("r", [128, 256, 384, 512])
@pytest.mark.parametrize("dr", [0, 64])
def test_few_rows(fb, M, H, r, dr):
    """16 rows or fewer, 32 or fewer, more, at every width; causal, lengths that differ."""
    g = torch.Generator().manual_seed(M * H + r + dr)
    B, n, lens = 3, 333, [333, 40, 1]
    q, c, wk, wv = inputs(g, B, M, n, H, 64, dr, 64, r, poison=lens)
    want = reference(q, c, wk, wv, lens, 0.1, True, ABSORBED)
    check(run(fb, q, c, wk, wv, ABSORBED, 0.1, kv_len=torch.tensor(lens, dtype=torch.int32, device=DEV), causal=True), want)


# lengths of none, one, part and all of the keys, and outside of what there is; behind them NaN; with causal rows, more rows than keys leave rows empty
LENGTHS = [(4, 1, 300, 8, 64, 32, 64, 128, [0, 1, 300, 129]), (3, 7, 96, 16, 128, 64, 128, 512, [96, 5, 0]), (2, 150, 200, 4, 40, 0, 40, 128, [200, 77]), (2, 70, 33, 2, 80, 64, 80, 320, [33, 32]),
           (6, 3, 500, 30, 128, 64, 64, 256, [500, 0, 0, 64, 65, 3]), (1, 513, 700, 3, 64, 0, 64, 384, [640]), (4, 129, 300, 64, 32, 0, 32, 64, [300, 0, 64, 150]), (1, 1100, 1100, 64, 64, 32, 64, 128, [1100]),
           (2, 300, 150, 90, 40, 8, 40, 64, [150, 2]),
           # expanded: two halves of a part's keys, of the same and of different numbers of blocks, one of them empty
           (4, 70, 1500, 6, 64, 32, 64, 128, [1500, 70, 1001, 33]), (2, 200, 1300, 5, 128, 64, 128, 512, [1300, 1089]), (2, 140, 1100, 3, 96, 0, 96, 128, [1100, 0]),
           (2, 640, 1030, 52, 32, 0, 32, 64, [1030, 700])]


@pytest.mark.parametrize("form", [ABSORBED, EXPANDED])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,M,n,H,d,dr,dv,r,lens", LENGTHS)
def test_lengths_and_causal_rows(fb, B, M, n, H, d, dr, dv, r, lens, causal, form):
    g = torch.Generator().manual_seed(M + n)
    q, c, wk, wv = inputs(g, B, M, n, H, d, dr, dv, r, extra=40, poison=lens)
    scale = 1 / math.sqrt(d + dr)
    want = reference(q, c, wk, wv, lens, scale, causal, form)
    got = run(fb, q, c, wk, wv, form, scale, kv_len=torch.tensor(lens, dtype=torch.int32, device=DEV), n_keys=n, causal=causal)
    check(got, want)
    empty = (want[0] == 0).all(-1)
    assert bool((got.cpu()[empty] == 0).all())
    if max(lens) == n:                                                          # outside 0 .. n_keys: the nearest of those
        far = torch.tensor([2 ** 30 if ln == n else -7 if ln == 0 else ln for ln in lens], dtype=torch.int32, device=DEV)
        assert torch.equal(run(fb, q, c, wk, wv, form, scale, kv_len=far, n_keys=n, causal=causal), got)


@pytest.mark.parametrize("form", [ABSORBED, EXPANDED])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_a_key_that_a_query_does_not_see_has_no_effect(fb, form, value):
    g = torch.Generator().manual_seed(11)
    B, M, n, H, d, dr, dv, r = 1, 70, 100, 2, 64, 32, 64, 128
    q, c, wk, wv = inputs(g, B, M, n, H, d, dr, dv, r)
    want = reference(q, c, wk, wv, [n], 0.1, True)
    at = 60                                                                     # query m is token 30 + m: queries 0 .. 29 do not see it
    for col in (5, r + 3):
        bad = c.clone()
        bad[0, at, col] = value
        got = run(fb, q, bad, wk, wv, form, 0.1, causal=True)
        check(got[:, :at - (n - M)], want, slice(0, at - (n - M)))
        if math.isnan(value):
            assert bool(got[:, at - (n - M):].isnan().all())
    qn = q.clone()
    qn[0, 3, 1, 0] = math.nan
    got = run(fb, qn, c, wk, wv, form, 0.1, causal=True).view(M, H, dv)
    assert bool(got[3, 1].isnan().all())
    got[3, 1] = want[0].view(M, H, dv)[3, 1].to(got)
    check(got.view(1, M, -1), want)


@pytest.mark.parametrize("form", [ABSORBED, EXPANDED])
def test_scores_far_apart(fb, form):
    """One key outweighs the rest by hundreds: its value comes out, whichever block it is in."""
    g = torch.Generator().manual_seed(12)
    B, M, n, H, d, dr, dv, r = 1, 96, 96, 1, 64, 64, 64, 128
    q, c, wk, wv = inputs(g, B, M, n, H, d, dr, dv, r)
    c[..., r:], q[..., d:] = 0, 0
    pick = torch.randperm(n, generator=g)
    for m in range(M):                                                          # 64 channels: a key's number in plus and minus ones
        bits = torch.tensor([1.0 if int(pick[m]) >> (i % 7) & 1 else -1.0 for i in range(64)])
        key = torch.tensor([1.0 if m >> (i % 7) & 1 else -1.0 for i in range(64)])
        q[0, m, 0, d:], c[0, m, r:] = (8 * bits).to(BF).to(DEV), (8 * key).to(BF).to(DEV)
    want = reference(q, c, wk, wv, [n], 1.0, False)
    check(run(fb, q, c, wk, wv, form, 1.0), want)


def test_forms_agree_and_auto_is_one_of_them(fb):
    g = torch.Generator().manual_seed(13)
    for B, M, n, H in ((2, 1, 600, 16), (1, 600, 600, 16)):
        q, c, wk, wv = inputs(g, B, M, n, H, 128, 64, 128, 512)
        outs = [run(fb, q, c, wk, wv, f, 0.07) for f in (0, ABSORBED, EXPANDED)]
        assert torch.equal(outs[0], outs[1]) or torch.equal(outs[0], outs[2])
        assert rel_l2(host(outs[1]), host(outs[2])) <= 2 * L2


def test_two_captured_graphs_and_eager_calls(fb):
    """Two captured calls with a workspace each on two streams, replayed with eager calls between, while the lengths change."""
    g = torch.Generator().manual_seed(14)
    calls = []
    for B, M, n, H, form in ((3, 1, 700, 16, ABSORBED), (1, 200, 260, 4, EXPANDED)):
        q, c, wk, wv = inputs(g, B, M, n, H, 64, 32, 64, 256)
        lens = torch.full((B,), n, dtype=torch.int32, device=DEV)
        out = torch.zeros((B, M, H * 64), dtype=BF, device=DEV)
        a = fb.latent_attention_args(q, c, wk, wv, out, 0.1, kv_len=lens, causal=True, form=form)
        ws = torch.zeros(fb.fise_latent_attention_workspace_bytes(a), dtype=torch.uint8, device=DEV)
        st = torch.cuda.Stream()
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=st):
            fb.fise_latent_attention(a, ws, stream=st)
        calls.append((a, lens, out, gr, st, n, form))
    for rep in range(4):
        want = []
        for a, lens, out, gr, st, n, form in calls:
            lens.copy_(torch.randint(0, n + 1, lens.shape, generator=g).to(torch.int32))
            ws = torch.zeros(fb.fise_latent_attention_workspace_bytes(a), dtype=torch.uint8, device=DEV)
            fb.fise_latent_attention(a, ws)
            want.append(out.clone())
            out.fill_(float("nan"))
        torch.cuda.synchronize()
        for a, lens, out, gr, st, n, form in calls:
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        for (a, lens, out, *_), w in zip(calls, want):
            assert torch.equal(out, w), rep


@pytest.mark.parametrize("form", [ABSORBED, EXPANDED])
@pytest.mark.parametrize("M", [1, 200])
def test_no_keys_at_all(fb, form, M):
    q, c, wk, wv = inputs(torch.Generator().manual_seed(16), 2, M, 9, 3, 64, 32, 64, 128)
    assert bool((run(fb, q, c * math.nan, wk, wv, form, 0.1, n_keys=0) == 0).all())


@pytest.mark.parametrize("form", [ABSORBED, EXPANDED])
def test_offsets_past_32_bits(fb, form):
    """Caches of 4.8 GB an element, keys of 7 GB and values of 5 GB: all keys zeros but a few, the last ones among them, whose shared keys give them scores near ln(n), so
    that they and the zeros (score 0) each have a part.  Scores are exact; values and output are rounded as ever, and a lane's sum of n / 512 probabilities by 2^-24 each, 5e-4
    at most, which the tolerance for rounded keys that there are not has room for."""
    g = torch.Generator().manual_seed(17)
    B, M, n, H, d, dr, dv, r = 2, 3, 4200000, 2, 160, 64, 160, 512
    q, few, wk, wv = inputs(g, B, M, 8, H, d, dr, dv, r)
    at = torch.tensor([0, 77777, n // 2, 3728300, n - 130, n - 64, n - 2, n - 1], device=DEV)
    q.zero_()
    q[..., d] = 1
    few[..., r:] = torch.tensor([15, 15.5, 16, 14, 15.25, 14.5, 15.75, 16.5], device=DEV).to(BF)[None, :, None]
    cache = torch.zeros((B, n, r + dr), dtype=BF, device=DEV)
    cache[:, at] = few
    out = torch.full((B, M, H * dv), float("nan"), dtype=BF, device=DEV)
    a = fb.latent_attention_args(q, cache, wk, wv, out, 1.0, form=form)
    fb.fise_latent_attention(a, torch.empty((fb.fise_latent_attention_workspace_bytes(a),), dtype=torch.uint8, device=DEV))
    e = torch.exp(few[..., r].double().cpu())
    p = e / (e.sum(-1, keepdim=True) + n - at.numel())
    assert 0.5 < float(p.sum(-1).min()) and float(p.sum(-1).max()) < 0.95
    v = torch.einsum("bjr,hdr->bhjd", few[..., :r].double().cpu(), wv.double().cpu())
    want, spread = torch.einsum("bj,bhjd->bhd", p, v), torch.einsum("bj,bhjd->bhd", p ** 2, v ** 2).sqrt()
    check(out, tuple(t.reshape(B, 1, -1).expand(B, M, -1) for t in (want, spread)))
