"""Attention over a paged cache at the ends of its number formats: weights far below the
largest one over long caches, values and scores near the largest numbers."""
import math

import pytest
import torch

from tests.paged_common import Batch, half_step

pytestmark = pytest.mark.gpu

# (new tokens per sequence or None for one each, in the form of single tokens): 16, 64 and 128 rows in a tile
FORMS = [None, 5, 48, 160]


def shared_sequences(n, count, new, **kw):
    """``count`` sequences of n positions, all in the same pages: enough units of work that none is
    cut along its keys."""
    b = Batch([n], [new] if new else None, page=256, **kw)
    b.lens, b.new = [n] * count, [new or 1] * count
    b.table = b.table.expand(count, -1).contiguous()
    b.len = b.len.expand(count).contiguous()
    b.begin = torch.arange(count + 1, dtype=torch.int32, device="cuda") * (new or 1)
    b.rows = b.n_tok = count * (new or 1)
    b.q = torch.zeros((b.rows, b.nq * b.d), dtype=b.dtype, device="cuda")
    b.out = torch.full_like(b.q, 7.0)
    b.lse = torch.full((b.rows, b.nq), 7.0, device="cuda")
    return b


@pytest.mark.parametrize("new", FORMS)
@pytest.mark.parametrize("act,f8,d", [("f16", False, 64), ("f16", False, 128), ("f16", True, 64), ("bf16", False, 64)])
def test_many_small_weights_beside_one_large(new, act, f8, d):
    """One key (an attention sink) scores 18 above 131071 others, whose weights of e^-18 (2^-25.97) of its own
    add up to 0.2%. Its value is 0, theirs is alike, so out is their share of the sum.

    The bound on out: the output's rounding, a rounding of each weight and of their sum (for one
    product per weight), exp2's 2^-15 and the sum's error as in lse below, all of the output itself, and
    2^-14 of the values for weights at the lower end of their type, an eighth of the half step of an output
    as large as a value: a weight off by 2^-32 of the largest one makes half of that with this many. On
    lse: the weights of up to 32 keys are added up before they join a running sum, which makes n / 32
    roundings of half a step of it, 2^-12."""
    n, count = 131072, 64
    b = shared_sequences(n, count, new, kv_heads=8, d=d, act=act, f8=f8, scales=False)
    k = torch.zeros((n, 8, d), device="cuda")
    k[0, :, 0] = 18.0
    value = torch.linspace(-2.0, 2.0, d, device="cuda").to(b.cache_dtype).float()
    v = value.expand(n, 8, d).clone()
    v[0] = 0.0
    b.fill(0, k, v)
    b.q.view(-1, d)[:, 0] = 1.0
    b.attend(scale=1.0)
    t = new or 1
    others = torch.arange(n - t, n, dtype=torch.float64, device="cuda")     # keys of token i beside the first
    total = math.exp(18.0) + others
    want = ((others / total)[:, None, None] * value.double()).expand(t, 8, d).reshape(1, t, 8 * d)
    got = b.out.double().view(count, t, 8 * d)
    u = half_step(b.dtype)
    tol = (3 * u + 2.0 ** -15 + 2.0 ** -12) * want.abs() + 2.0 ** -14 * 2.0
    assert bool(((got - want).abs() <= tol).all()), float((got - want).abs().max())
    lse = b.lse.double().view(count, t, 8)
    assert bool(((lse - total.log()[:, None]).abs() <= 2.0 ** -12 + 2.0 ** -18 + (d + 8) * 2.0 ** -24 * 18).all())


@pytest.mark.parametrize("new", FORMS)
@pytest.mark.parametrize("size", [3e38, 1e30, 1e-20])
def test_values_near_the_largest_numbers(new, size):
    """Values alike at every position give themselves, whatever the weights: also where sums of
    them are beyond fp32."""
    lens = [max(n, new or 1) for n in (1, 2, 40, 900, 20000)]
    b = Batch(lens, [new] * 5 if new else None, kv_heads=2, group=2, d=64, act="bf16", page=64)
    value = (torch.linspace(0.5, 1.0, 64, device="cuda") * size).bfloat16()
    value[1::2] *= -1
    for s, n in enumerate(b.lens):
        b.slots(b.v_pool)[b.at(s)] = value
    b.attend()
    got, want = b.out.double().view(-1, 64), value.double()
    # the output's rounding, one of each weight and of their sum, fp32 sums
    assert bool(((got - want).abs() <= (3 * half_step(b.dtype) + 2.0 ** -15) * want.abs()).all())
