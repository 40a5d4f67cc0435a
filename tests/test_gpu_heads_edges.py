"""vt_paged_append_heads and vt_rotate_heads where single bits and the range of fp32 matter."""
import math

import pytest
import torch

from paper_2607_07046_amd import voltron as vt
from tests.paged_common import F8, Batch
from tests.rows_common import p, stream

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("type", ["f16", "bf16"])

# quotients on both sides of every kind of step, past the largest number and below the smallest, both zeros
GRID = torch.cat([torch.tensor([m * 2.0 ** e for e in range(-14, 9) for m in (1.0, 1.0625, 1.1875, 1.3125, 1.9375)]),
                  torch.tensor([448.0, 456.0, 464.0, 465.0, 480.0, 1e4, 6e4, math.inf, math.nan, 0.0])])
GRID = torch.cat([GRID, -GRID])


def pools(b):
    """The bytes of both pools at the positions of the first sequence."""
    return [b.slots(t)[b.at(0)].contiguous().view(torch.uint8).cpu() for t in (b.k_pool, b.v_pool)]


def rows_of(b, scale):
    """The grid times each head's scale, over every place of 64 rows of 4 heads."""
    base = GRID[torch.arange(64 * 4 * b.d) % GRID.numel()].view(64, 4, b.d).cuda()
    return (base if scale is None else base * scale[:, None]).to(b.dtype).flatten(1)


def batch(type, d, f8, scales):
    b = Batch([64], [64], kv_heads=4, group=1, d=d, act=type, f8=f8, scales=False)
    if scales:
        b.k_scale = torch.tensor([0.75, 0.01171875, 3.0, 1e-3], device="cuda")
        b.v_scale = torch.tensor([1.0, 5.0, 0.375, 7.0], device="cuda")
    k, v = rows_of(b, b.k_scale), rows_of(b, b.v_scale)
    return b, k, v, b.io(q=None, q_rot=None, k=p(k), ld_k=4 * d, v=p(v), ld_v=4 * d)


@BOTH
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scales", [False, True])
def test_append_f8_bytes(type, d, scales):
    """What is stored is the rounded quotient byte for byte, the sign of zero included; NaN stays NaN."""
    b, k, v, io = batch(type, d, True, scales)
    vt.vt_paged_append_heads(b.kv(), io, None, None, stream())
    torch.cuda.synchronize()
    for x, scale, got in zip((k, v), (b.k_scale, b.v_scale), pools(b)):
        q = x.cpu().view(64, 4, d).float()
        q = q if scale is None else q / scale.cpu()[:, None]
        want = q.clamp(-448, 448).to(F8).view(torch.uint8)
        there = ~q.isnan()
        assert torch.equal(got[there], want[there])
        assert bool(got.view(F8).float()[~there].isnan().all())
        zeros = there & (q == 0)
        assert bool((got[zeros & q.signbit()] == 0x80).all()) and bool((got[zeros & ~q.signbit()] == 0).all())


@BOTH
@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("scales", [False, True])
def test_bytes_of_a_plain_append(type, f8, scales):
    """Without norms and rotation both appends store the same bytes, whatever the numbers."""
    stored = []
    for call in (lambda b, io: vt.vt_paged_append(b.kv(), io, 0.0, 0, stream()),
                 lambda b, io: vt.vt_paged_append_heads(b.kv(), io, None, None, stream())):
        b, _, _, io = batch(type, 64, f8, scales and f8)
        call(b, io)
        torch.cuda.synchronize()
        stored.append(pools(b))
    for one, other in zip(*stored):
        assert torch.equal(one, other)
