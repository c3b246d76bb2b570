"""Attention over latent vectors with the form left to the library takes every size that one of the forms takes; no GPU needed (sizes are checked before anything is launched)."""
import ctypes
import random

import pytest

from paper_2305_17423_amd import binding as fb

A = 0x10000          # never dereferenced


def args(form, B, M, n, H, d=128, dr=64, dv=128, r=512, causal=0):
    a = fb.fise_latent_attention_args()
    for k, v in dict(q=A, cache=A, w_uk=A, w_uv=A, out=2 * A, B=B, M=M, n_keys=n, cache_tokens=n, heads=H, d=d, dr=dr, dv=dv, r=r, scale=0.1, dtype=1, causal=causal, form=form).items():
        setattr(a, k, v)
    return a


def taken(a):
    need = fb.fise_latent_attention_workspace_bytes(a)
    code = fb.lib().fise_latent_attention(ctypes.byref(a), None, 0, None)
    assert code == (-1 if need else -2), fb.fise_last_error()                  # a missing workspace, or a refused size
    return need


@pytest.mark.parametrize("size", [(1, 2000, 1 << 26, 16), (300, 300, 2, 65535), (1, 1 << 14, 1, 65535), (4, 512, 1 << 24, 16), (1, 1 << 19, 1 << 19, 16), (1, 4096, 4096, 16), (1, 1, 1000, 8)])
@pytest.mark.parametrize("causal", [0, 1])
def test_sizes_that_one_form_takes(size, causal):
    need = [taken(args(form, *size, causal=causal)) for form in (0, 1, 2)]
    assert need[0] in ([n for n in need[1:] if n] or [0])


def test_any_size():
    rng = random.Random(9)
    log = lambda top: int(2 ** rng.uniform(0, top))
    seen = set()
    for _ in range(4000):
        size = (log(12), log(20), log(26), log(16), 8 * rng.randint(1, 20), 8 * rng.randint(0, 8), 8 * rng.randint(1, 20), 8 * rng.randint(1, 64), rng.random() < 0.5)
        need = [taken(args(form, *size)) for form in (0, 1, 2)]
        assert need[0] in ([n for n in need[1:] if n] or [0]), size
        seen.add(tuple(map(bool, need)))
    assert seen == {(True, True, True), (False, False, False), (True, True, False), (True, False, True)}
