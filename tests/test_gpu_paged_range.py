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


@pytest.mark.parametrize("new", FORMS)
@pytest.mark.parametrize("act,sigma", [("f16", 300.0), ("f16", 5000.0), ("f16", 20000.0), ("bf16", 1e6), ("bf16", 1e12)])
def test_scores_far_beyond_their_rounding(new, act, sigma):
    """Scores of 10^5 to 10^24, whose fp32 steps are larger than the weights' range: the weights are
    those of the rounded scores, finite, and one key that stands out by more than the scores' errors
    takes all. (``check`` derives the scores' error and asserts that all is finite where the definition is.)"""
    lens = [max(n, new or 1) for n in (1, 33, 700, 5000)]
    b = Batch(lens, [new] * 4 if new else None, kv_heads=2, group=2, d=128, act=act, page=32, sigma=0.0)
    g, most = torch.Generator(device="cuda").manual_seed(3), 60000.0 if act == "f16" else 1e30
    big = lambda *shape: torch.empty(shape, device="cuda").normal_(0, sigma, generator=g).clamp(-most, most)
    for s, n in enumerate(b.lens):
        b.slots(b.k_pool)[b.at(s)] = big(n, 2, 128).to(b.dtype)
    b.q[:b.rows] = big(b.rows, b.nq * 128).to(b.dtype)
    b.attend()
    b.check(rounded=True)
    # where the largest score stands out, its value (rounded, with its weight and the sum's rounding)
    row, clear = 0, 0
    for s, (n, t) in enumerate(zip(b.lens, b.new)):
        k, v = b.read(b.k_pool, s), b.read(b.v_pool, s)
        q = b.q[row:row + t].double().view(t, 2, 2, 128).permute(1, 2, 0, 3).reshape(2, 2 * t, 128)
        kt = k.permute(1, 2, 0).contiguous()
        x = torch.matmul(q, kt) / math.sqrt(128)
        hidden = torch.arange(n, device="cuda") > torch.arange(n - t, n, device="cuda").repeat(2)[:, None]
        e = 2 * 132 * 2.0 ** -24 * torch.matmul(q.abs(), kt.abs()).amax(-1) / math.sqrt(128) + 40
        best = x.masked_fill(hidden, -math.inf).topk(min(2, n), -1)
        alone = best.values[..., 0] - best.values[..., -1] > e if n > 1 else torch.ones_like(e, dtype=torch.bool)
        alone |= ~best.values[..., -1].isfinite()
        at = best.indices[..., 0]
        want = v.permute(1, 0, 2).gather(1, at[..., None].expand(-1, -1, 128))
        got = b.out[row:row + t].double().view(t, 2, 2, 128).permute(1, 2, 0, 3).reshape(2, 2 * t, 128)
        off = (got - want).abs() - 3 * half_step(b.dtype) * want.abs() - 2.0 ** -20
        assert bool((off[alone] <= 0).all()), (s, float(off[alone].max()))
        clear += int(alone.sum())
        row += t
    assert clear > b.rows  # of 4 heads: the test tests something
