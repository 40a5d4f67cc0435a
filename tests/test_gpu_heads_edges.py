"""vt_paged_append_heads and vt_rotate_heads where single bits and the range of fp32 matter."""
import math

import pytest
import torch

from paper_2607_07046_amd import voltron as vt
from tests.paged_common import F8, Batch
from tests.rows_common import p, stream
from tests.test_gpu_rows import Heads, check_append, gains_of

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


# Sizes of the numbers and of the gains: products of a number with its gain beyond the range of fp32 although the
# normalised number's are far inside it; products that have no full precision in fp32; numbers past both borders of the
# fast statistics.
FAR = pytest.mark.parametrize("size,gain,eps", [(1e18, 1e21, 1e-5), (1e-14, 1e-30, 0.0), (1e-14, 1e30, 0.0),
                                                (1e18, 1e-30, 1e-5), (1.0, 1e37, 1e-6), (1.0, 1e-36, 1e-6), (1e25, 1e25, 1e-5),
                                                (1e-30, 1e-12, 0.0)])
TURNS = pytest.mark.parametrize("rope", [None, dict(base=10000.0), dict(base=10000.0, flags=1),
                                         dict(base=500000.0, dims=50, flags=1, amplitude=0.75)])


def scaled(t, by):
    """Numbers of |x| up to 1 times ``by``."""
    t.copy_((t.double().clamp(-1, 1) * by).to(t.dtype))


@FAR
@TURNS
@pytest.mark.parametrize("d", [64, 128])
def test_head_norms_with_far_gains(size, gain, eps, rope, d):
    """Whatever the sizes of numbers and gains, results that bf16 holds are right. Tolerances as everywhere; numbers
    below fp32's normal ones (2^-126) may count as zero."""
    x = Heads("bf16", 7, 5, 3, d, eps=eps, far=300)
    for t in (x.q, x.k):
        scaled(t, size)
    for t in (x.q_gain, x.k_gain):
        scaled(t, gain)
    x.call(rope)
    ref = {n: x.reference(n, rope, x.pos) for n in ("q", "k")}
    assert all(float(w.abs().max()) < 3e38 for w, _ in ref.values())
    x.check(rope, ref={n: (w, t + 2.0 ** -126) for n, (w, t) in ref.items()})


@pytest.mark.parametrize("size,gain,eps", [(1e18, 1e21, 1e-5), (1e-14, 1e30, 0.0)])
@pytest.mark.parametrize("flags", [0, 1])
def test_append_with_far_gains(size, gain, eps, flags):
    b = Batch([40, 17], [7, 17], kv_heads=3, group=2, d=128, act="bf16")
    gains = gains_of(b)
    for t in gains:
        scaled(t, gain)
    before = {n: b.slots(getattr(b, n + "_pool")).clone() for n in ("k", "v")}
    g = torch.Generator(device="cuda").manual_seed(1)
    qkv = torch.empty((b.n_tok, (b.nq + 6) * 128), dtype=b.dtype, device="cuda").normal_(generator=g)
    scaled(qkv, size)
    q, k, v = qkv[:, :b.nq * 128], qkv[:, b.nq * 128:-3 * 128], qkv[:, -3 * 128:]
    q_rot = torch.empty((b.n_tok, b.nq * 128), dtype=b.dtype, device="cuda")
    rope = dict(base=10000.0, flags=flags)
    io = b.io(q=p(q), ld_q=qkv.stride(0), k=p(k), ld_k=qkv.stride(0), v=p(v), ld_v=qkv.stride(0), q_rot=p(q_rot))
    vt.vt_paged_append_heads(b.kv(), io, vt.vt_head_norm(q_gain=p(gains[0]), k_gain=p(gains[1]), eps=eps), vt.vt_rope(**rope),
                             stream())
    torch.cuda.synchronize()
    check_append(b, rope, gains, eps, q, k, v, q_rot, before)
