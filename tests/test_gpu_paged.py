"""The paged cache on the device: append with rotation, attention of single
tokens and of chunks, against the definition in float64 (tests/paged_common.py
derives the bounds)."""
import math

import numpy as np
import pytest
import torch

from paper_2607_07046_amd import voltron as vt
from tests.paged_common import F8, F8_MAX, Batch, half_step

pytestmark = pytest.mark.gpu

EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 65, 127, 128, 129, 255, 257]


# ---- append ------------------------------------------------------------------
def rotated(x, pos, base, halves):
    d = x.shape[-1]
    if base == 0:
        return x
    i = torch.arange(d // 2, dtype=torch.float64, device="cuda")
    a = pos.double()[:, None] * base ** (-2.0 * i / d)
    c, s = a.cos()[:, None], a.sin()[:, None]
    lo, hi = (slice(0, d // 2), slice(d // 2, d)) if halves else (slice(0, d, 2), slice(1, d, 2))
    y = torch.empty_like(x)
    y[..., lo] = x[..., lo] * c - x[..., hi] * s
    y[..., hi] = x[..., lo] * s + x[..., hi] * c
    return y


def append(b, base=10000.0, flags=0, with_q=True, in_place=False, stream=None, ld_extra=0):
    """Appends new random rows; returns the inputs and the rotated queries."""
    g = torch.Generator(device="cuda").manual_seed(99)
    w, kw = b.nq * b.d, b.kv_heads * b.d
    ld = w + 2 * kw + ld_extra
    qkv = torch.full((b.n_tok, ld), math.nan, dtype=b.dtype, device="cuda")
    qkv[:b.rows] = torch.empty((b.rows, ld), device="cuda").normal_(generator=g).to(b.dtype)
    kept = qkv.clone()
    q_rot = qkv[:, :w] if in_place else torch.full((b.n_tok, w), 7.0, dtype=b.dtype, device="cuda")
    p = qkv.data_ptr()
    io = b.io(q=p if with_q else None, ld_q=ld, k=p + 2 * w, ld_k=ld, v=p + 2 * (w + kw), ld_v=ld,
              q_rot=q_rot.data_ptr(), ld_qr=ld if in_place else w)
    vt.vt_paged_append(b.kv(), io, base, flags, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return kept, q_rot


def check_append(b, base=10000.0, flags=0, skip=lambda s, p: False, **kw):
    before = [t.view(torch.uint8).clone() for t in (b.k_pool, b.v_pool)]
    qkv, q_rot = append(b, base, flags, **kw)
    w, kvw, d = b.nq * b.d, b.kv_heads * b.d, b.d
    part = lambda a, n: qkv[:b.rows, a:a + n].double().reshape(b.rows, -1, d)
    pos = torch.cat([torch.arange(n - t, n, device="cuda") for n, t in zip(b.lens, b.new)])
    seq = [s for s, t in enumerate(b.new) for _ in range(t)]
    # fp32 rotation: three roundings, and the hardware's sine and cosine, of the pair's length
    slack = 2.0 ** -18 if base else 0.0
    near = lambda got, want, norm, u, tiny: bool(((got - want).abs() <= u * want.abs() + slack * norm + tiny).all())
    live = pos >= 0
    if kw.get("with_q", True):
        q = part(0, w)
        got = q_rot[:b.rows].double().reshape(b.rows, -1, d)
        assert near(got[live], rotated(q, pos, base, flags)[live], q.abs().amax(), half_step(b.dtype), 2.0 ** -25)
        if not kw.get("in_place"):
            assert bool((got[~live] == 7.0).all()) and bool((q_rot[b.rows:] == 7.0).all())
    k, v = rotated(part(w, kvw), pos, base, flags), part(w + kvw, kvw)
    expect = [t.clone() for t in before]
    for pool, x, scale, was in ((b.k_pool, k, b.k_scale, expect[0]), (b.v_pool, v, b.v_scale, expect[1])):
        x = x if scale is None else x / scale.double()[:, None]
        mem = was.view(pool.dtype)
        for r in range(b.rows):
            s, p = seq[r], int(pos[r])
            if p < 0 or skip(s, p):
                continue
            page, slot = int(b.table[s, p // b.page]), p % b.page
            got = b.slots(pool)[page, slot]
            b.slots(mem)[page, slot] = got  # what was written is judged here, the rest below
            got = (got.view(F8).float() if b.f8 else got).double()
            want = x[r].clamp(-F8_MAX, F8_MAX) if b.f8 else x[r]
            if b.f8:
                assert near(got, want, F8_MAX * 0.01, half_step(F8), 2.0 ** -10), (r, s, p)
            elif pool is b.v_pool:
                assert torch.equal(got, want), (r, s, p)
            else:
                assert near(got, want, want.abs().amax(), half_step(b.dtype), 2.0 ** -25), (r, s, p)
    # no other byte of the pools has changed
    assert torch.equal(expect[0], b.k_pool.view(torch.uint8)) and torch.equal(expect[1], b.v_pool.view(torch.uint8))
    return q_rot


@pytest.mark.parametrize("act,f8", [("f16", False), ("bf16", False), ("f16", True), ("bf16", True)])
@pytest.mark.parametrize("d,order,page,flags", [(64, "head", 16, 0), (128, "slot", 1, 0), (128, "head", 64, 1),
                                                (64, "slot", 8, 1)])
def test_append_ragged(act, f8, d, order, page, flags):
    b = Batch([5, 1, 40, 17, 3], [3, 1, 9, 0, 3], kv_heads=3, group=2, d=d, page=page, order=order, act=act, f8=f8, pad=2)
    check_append(b, flags=flags, ld_extra=8)
    assert int(b.status) == 0


@pytest.mark.parametrize("heads,group", [(1, 1), (1, 17), (40, 1), (8, 16)])
def test_append_head_layouts(heads, group):
    check_append(Batch([33, 7], [5, 2], kv_heads=heads, group=group, d=128))
    check_append(Batch([33, 7], kv_heads=heads, group=group, d=64), in_place=True)


def test_append_one_token_each_with_idle_slots():
    b = Batch([5, 0, 1, 0, 129], kv_heads=2, group=4, d=128)
    check_append(b)
    assert int(b.status) == 0


def test_append_without_queries_or_rotation():
    check_append(Batch([20, 4], [7, 4]), with_q=False)
    check_append(Batch([20, 4], [7, 4]), base=0.0)


@pytest.mark.parametrize("flags", [0, 1])
@pytest.mark.parametrize("pos", [1000003, 2 ** 30 + 1])
def test_append_far_positions(pos, flags):
    """Angles of positions that a float does not hold; only the last page exists."""
    b = Batch([1], kv_heads=2, d=128, page=32768)
    b.lens = [pos + 1]
    b.max_pages = pos // b.page + 1
    b.table = torch.full((1, b.max_pages + 1), -1, dtype=torch.int32, device="cuda")
    b.table[0, pos // b.page] = 1
    b.len = torch.tensor(b.lens, dtype=torch.int32, device="cuda")
    check_append(b, base=500000.0, flags=flags)


@pytest.mark.parametrize("n", [1, 63, 64, 65, 300, 4097])
def test_append_many_sequences(n):
    """The search for a row's sequence, with empty sequences in between."""
    rng = np.random.default_rng(n)
    new = rng.integers(0, 3, n)
    if new.sum() == 0:
        new[0] = 1
    lens = new + rng.integers(0, 5, n)
    b = Batch(lens.tolist(), new.tolist(), kv_heads=1, d=64, page=4, pad=3)
    qkv, q_rot = append(b)
    at = torch.cat([torch.arange(l - t, l) for l, t in zip(lens, new)]).cuda()
    seq = torch.repeat_interleave(torch.arange(n), torch.from_numpy(new)).cuda()
    got = b.slots(b.v_pool)[b.table[seq, at // 4].long(), at % 4].flatten(1)
    assert torch.equal(got, qkv[:b.rows, 128:192])
    q = qkv[:b.rows, :64].double()[:, None]
    assert bool(((q_rot[:b.rows].double() - rotated(q, at, 10000.0, 0)[:, 0]).abs() <= 2.0 ** -11 * 6 + 1e-4).all())
    assert bool((q_rot[b.rows:] == 7.0).all())


def test_append_f8_extremes():
    """Saturation, ties to even, subnormals, NaN and infinities of the 8-bit format."""
    b = Batch([1], kv_heads=1, d=64, f8=True, scales=False)
    v = torch.zeros(64, dtype=torch.float16, device="cuda")
    vals = [448.0, 449.0, 1000.0, -60000.0, math.inf, -math.inf, math.nan, 0.0, -0.0, 2.0 ** -9, 2.0 ** -10, 2.0 ** -10 * 1.5,
            1.0625, 1.1875, 17.0, 19.0, 0.0146484375, 240.0, 464.0, -2.0 ** -9]
    v[:len(vals)] = torch.tensor(vals, dtype=torch.float16)
    qkv = torch.cat([torch.zeros(128, dtype=torch.float16, device="cuda"), v])[None].contiguous()
    p = qkv.data_ptr()
    io = b.io(k=p + 128, ld_k=192, v=p + 256, ld_v=192)
    vt.vt_paged_append(b.kv(), io, 0.0, 0, None)
    torch.cuda.synchronize()
    got = b.slots(b.v_pool)[int(b.table[0, 0]), 0, 0].view(F8).float()
    want = torch.where(v.isnan(), v.float(), v.float().clamp(-448, 448)).to(F8).float()
    assert torch.equal(got.nan_to_num(-1.0), want.nan_to_num(-1.0))
    assert torch.equal(got.signbit()[:6], want.signbit()[:6])


def test_append_bad_pages_are_reported_and_not_stored():
    b = Batch([40, 20, 5], [30, 2, 5], kv_heads=2, d=64, page=16)
    b.table[0, 1] = b.n_pages        # positions 16..31
    b.table[2, 0] = -1
    check_append(b, skip=lambda s, p: (s == 0 and 16 <= p < 32) or s == 2)
    assert int(b.status) == vt.VT_PAGED_BAD_PAGE


def test_append_past_the_table():
    b = Batch([40, 20], [30, 2], kv_heads=2, d=64, page=16)
    kv = b.kv(max_pages=2)
    before = b.k_pool.view(torch.uint8).clone()
    real, b.kv = b.kv, lambda **k: kv
    check_append(b, skip=lambda s, p: p >= 32)
    assert int(b.status) == vt.VT_PAGED_BAD_LEN and not torch.equal(before, b.k_pool.view(torch.uint8))


# ---- attention of single tokens --------------------------------------------------
@pytest.mark.parametrize("act,f8", [("f16", False), ("bf16", False), ("f16", True), ("bf16", True)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,order", [(16, "head"), (1, "slot"), (8, "head"), (256, "slot"), (32, "slot"), (2, "head")])
def test_decode_edges(act, f8, d, page, order):
    b = Batch(EDGES, kv_heads=2, group=4, d=d, page=page, order=order, act=act, f8=f8, extra=1)
    b.attend()
    b.check()
    assert int(b.status) == 0


@pytest.mark.parametrize("heads,group", [(1, 1), (3, 3), (8, 8), (2, 16), (2, 17), (1, 40), (40, 1), (1, 128)])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_head_layouts(heads, group, d):
    b = Batch([300, 77, 0, 1], kv_heads=heads, group=group, d=d)
    b.attend()
    b.check()


@pytest.mark.parametrize("window", [1, 2, 16, 33, 100, 1000, 2 ** 31 - 1])
@pytest.mark.parametrize("page", [4, 16, 128])
def test_decode_window(window, page):
    b = Batch(EDGES + [700], kv_heads=2, group=2, d=128, page=page, window=window)
    for s, n in enumerate(b.lens):   # pages that lie wholly before the window are gone
        b.table[s, :max(0, n - window) // page] = -5
    missing = {s: list(range(max(0, n - window) // page * page)) for s, n in enumerate(b.lens)}
    b.attend()
    # positions before the window are masked anyway
    for s, m in missing.items():
        b.table[s, :len(m) // page] = 0
    b.check()
    assert int(b.status) == 0


@pytest.mark.parametrize("lens", [[20001], [65537, 3], [9000, 1, 0, 17000], [4096] * 9])
@pytest.mark.parametrize("heads,group,d,f8", [(1, 1, 64, False), (2, 8, 128, False), (2, 5, 128, True)])
def test_decode_long(lens, heads, group, d, f8):
    """Caches whose length is split over many workgroups and joined."""
    b = Batch(lens, kv_heads=heads, group=group, d=d, page=64, f8=f8)
    b.attend()
    b.check()


def test_decode_pieces_fitted_to_rounds():
    """Cuts that give a few more pieces than run at once, which are made again with longer
    ones: of one sequence, of ragged ones, of more than a workgroup has threads."""
    rng = np.random.default_rng(5)
    for lens, heads, group in (([6500], 10, 1), (rng.integers(900, 4000, 12).tolist(), 8, 2),
                               (rng.integers(1, 300, 299).tolist() + [20000], 2, 1)):
        b = Batch(lens, kv_heads=heads, group=group, d=64, page=32)
        b.attend()
        b.check()


def test_decode_more_items_than_workgroups():
    rng = np.random.default_rng(3)
    b = Batch(rng.integers(0, 90, 700).tolist(), kv_heads=8, group=2, d=64)
    b.attend()
    b.check()


def test_decode_sharp_and_large_scores():
    """Maxima that come late, weights far apart, scores of hundreds."""
    for sigma in (0.0, 4.0, 12.0):
        b = Batch([1500, 31], kv_heads=2, group=3, d=128, sigma=sigma)
        b.attend()
        b.check()
    b = Batch([1500], kv_heads=1, group=1, d=64)   # keys that grow: every block raises the maximum
    k = b.q[0, :64].double() * torch.linspace(-3, 3, 1500, dtype=torch.float64, device="cuda")[:, None]
    b.fill(0, k[:, None], torch.randn(1500, 1, 64, device="cuda"))
    b.attend()
    b.check()


def test_decode_scale():
    b = Batch([333, 12], kv_heads=2, group=2, d=64)
    b.attend(scale=0.5)
    b.check(scale=0.5)


@pytest.mark.parametrize("page", [8, 16, 64])
def test_decode_bad_pages_are_masked_and_reported(page):
    b = Batch([200, 150, 64, 90], kv_heads=2, group=4, d=128, page=page)
    b.table[0, 0] = -1
    b.table[1, 70 // page] = b.n_pages
    for i in range(-(-64 // page)):
        b.table[2, i] = -7           # nothing left of this one
    first = 70 // page * page
    missing = {0: list(range(page)), 1: list(range(first, min(first + page, 150))), 2: list(range(64))}
    keep = b.table.clone()
    b.attend()
    b.table = torch.where((keep < 0) | (keep >= b.n_pages), 0, keep)  # for the definition's own reads
    b.check(missing=missing)
    assert int(b.status) == vt.VT_PAGED_BAD_PAGE


def test_decode_length_past_the_table():
    """The keys that the table can name are attended to, and the status says so."""
    b = Batch([100, 48], kv_heads=2, group=2, d=64, page=16)
    ws = b.workspace()
    vt.vt_paged_decode_attn(b.kv(max_pages=3), b.io(), 0.0, 0, ws.data_ptr(), ws.numel(), None)
    torch.cuda.synchronize()
    assert int(b.status) == vt.VT_PAGED_BAD_LEN
    b.check(missing={0: list(range(48, 100))})


def test_decode_without_lse_or_status_and_strided():
    b = Batch([70, 300, 5], kv_heads=2, group=4, d=64)
    w = b.nq * b.d
    wide = torch.full((3, w + 72), math.nan, dtype=b.dtype, device="cuda")
    wide[:, :w] = b.q
    out = torch.full((3, w + 40), 7.0, dtype=b.dtype, device="cuda")
    ws = b.workspace()
    vt.vt_paged_decode_attn(b.kv(status=None), b.io(q_rot=wide.data_ptr(), ld_qr=w + 72, out=out.data_ptr(),
                                                    ld_out=w + 40, lse=None), 0.0, 0, ws.data_ptr(), ws.numel(), None)
    b.attend()
    assert torch.equal(out[:, :w], b.out) and bool((out[:, w:] == 7.0).all())


# ---- chunks ------------------------------------------------------------------------
CHUNKS = [([1], [1]), ([17], [17]), ([40, 3, 0, 70, 1], [5, 3, 0, 70, 1]), ([300, 129, 128], [2, 129, 64]),
          ([1000, 33, 256], [300, 33, 1]), ([130] * 5, [129, 1, 2, 65, 130])]


@pytest.mark.parametrize("lens,new", CHUNKS)
@pytest.mark.parametrize("act,f8", [("f16", False), ("bf16", False), ("bf16", True)])
@pytest.mark.parametrize("group,d,page,order", [(1, 64, 16, "head"), (4, 128, 32, "slot"), (3, 128, 2, "head"),
                                                (8, 64, 128, "slot"), (1, 128, 16, "slot")])
def test_chunk_edges(lens, new, act, f8, group, d, page, order):
    b = Batch(lens, new, kv_heads=2, group=group, d=d, page=page, order=order, act=act, f8=f8, pad=2)
    b.attend()
    b.check(rounded=True)
    assert int(b.status) == 0


@pytest.mark.parametrize("window", [1, 7, 64, 100, 129, 5000])
@pytest.mark.parametrize("page", [1, 16, 64])
def test_chunk_window(window, page):
    b = Batch([700, 40, 300, 5], [400, 40, 3, 1], kv_heads=2, group=2, d=128, page=page, window=window)
    for s, (n, t) in enumerate(zip(b.lens, b.new)):
        b.table[s, :max(0, n - t - window + 1) // page] = -5
    b.attend()
    b.table.clamp_(min=0)
    b.check(rounded=True)
    assert int(b.status) == 0


@pytest.mark.parametrize("lens,new", [([9000], [5]), ([20000, 100], [130, 100]), ([5000, 5000, 17], [64, 700, 2]),
                                      ([2500], [2500])])
@pytest.mark.parametrize("heads,group,d,f8", [(1, 1, 64, False), (2, 4, 128, False), (1, 8, 128, True)])
def test_chunk_long(lens, new, heads, group, d, f8):
    b = Batch(lens, new, kv_heads=heads, group=group, d=d, page=64, f8=f8, act="bf16" if f8 else "f16")
    b.attend()
    b.check(rounded=True)


@pytest.mark.parametrize("lens,new,group", [([3000, 1200, 2000], [250, 256, 200], 4),
                                            ([3100, 1300, 2000, 900, 2300], [60, 64, 33, 41, 50], 1)])
def test_chunk_pieces_fitted_to_rounds(lens, new, group):
    b = Batch(lens, new, kv_heads=8, group=group, d=64, page=32)
    b.attend()
    b.check(rounded=True)


@pytest.mark.parametrize("heads,group", [(1, 16), (1, 17), (1, 130), (5, 1)])
def test_chunk_head_layouts(heads, group):
    b = Batch([70, 9], [33, 2], kv_heads=heads, group=group, d=128)
    b.attend()
    b.check(rounded=True)


def test_chunk_sequence_shorter_than_its_new_tokens():
    """Rows at negative positions see nothing."""
    b = Batch([2, 30], [2, 5], kv_heads=2, group=2, d=64, pad=0)
    b.len[0] = 1
    b.attend()
    assert bool((b.out[0] == 0).all()) and bool((b.lse[0] == -math.inf).all())
    v = b.read(b.v_pool, 0)[0]
    assert torch.equal(b.out[1].view(2, 2, 64).double(), v[:, None].expand(2, 2, 64))


@pytest.mark.parametrize("page", [8, 16, 64])
@pytest.mark.parametrize("new", [3, 200])
def test_chunk_bad_pages_are_masked_and_reported(page, new):
    b = Batch([250, 130], [new, 2], kv_heads=2, group=2, d=128, page=page)
    b.table[0, 1] = -1
    b.table[1, 0] = 2 ** 30
    b.attend()
    b.table = torch.where((b.table < 0) | (b.table >= b.n_pages), 0, b.table)
    b.check(rounded=True, missing={0: list(range(page, 2 * page)), 1: list(range(page))})
    assert int(b.status) == vt.VT_PAGED_BAD_PAGE


@pytest.mark.parametrize("value", [math.inf, math.nan])
@pytest.mark.parametrize("new", [1, 4, 40, 300])
@pytest.mark.parametrize("d,act", [(128, "f16"), (64, "bf16")])
def test_chunk_values_that_later_tokens_bring(value, new, d, act):
    """An infinite or NaN value (or key) of a chunk's last token leaves the rows before it alone."""
    b = Batch([320], [new], kv_heads=2, group=2, d=d, act=act)
    at = b.at(0, 319, 1)
    b.slots(b.v_pool)[at[0], at[1], 0, 5] = value
    b.slots(b.k_pool)[at[0], at[1], 1, 3] = math.nan
    b.attend()
    out = b.out.double().view(new, 2, 2, d)
    assert not bool(out[-1, 0, :, 5].isfinite().any()) and not bool(out[-1, 1].isfinite().any())
    ok = torch.ones_like(out, dtype=torch.bool)
    ok[-1, 0, :, 5] = False
    ok[-1, 1] = False
    assert bool(out[ok].isfinite().all())
    if new > 1:   # and exactly as the sequence without that token gives
        c = Batch([320], [new], kv_heads=2, group=2, d=d, act=act)
        c.attend()
        assert torch.equal(b.out[:-1], c.out[:-1])


@pytest.mark.parametrize("new", [1, 5, 40, 200])
@pytest.mark.parametrize("f8", [False, True])
def test_sequences_that_share_pages(new, f8):
    """A common beginning in pages that two sequences name."""
    b = Batch([700, 650, 300], [new, new, 1], kv_heads=2, group=2, d=128, page=16, f8=f8)
    b.table[1, :20] = b.table[0, :20]
    b.table[2, :3] = b.table[0, :3]
    b.attend()
    b.check(rounded=True)


@pytest.mark.parametrize("new", [1, 5, 40, 300])
@pytest.mark.parametrize("d,act", [(128, "f16"), (64, "bf16")])
def test_values_and_queries_that_are_not_finite(new, d, act):
    """A visible infinity stays in its element, a NaN query in its head's row."""
    b = Batch([900, 400], [new, new], kv_heads=2, group=2, d=d, act=act)
    at = b.at(0, 130, 1)
    b.slots(b.v_pool)[at[0], at[1], 1, 7] = math.inf
    b.q[new, d + 3] = math.nan
    b.attend()
    b.check(rounded=True)


def test_chunk_of_one_token_each_equals_decode():
    a = Batch([100, 0, 1, 4000], kv_heads=2, group=4, d=128)
    b = Batch([100, 0, 1, 4000], [1, 1, 1, 1], kv_heads=2, group=4, d=128)
    a.attend()
    b.attend()
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)
    b.out.fill_(7.0)
    b.ragged = False
    b.attend(chunk=True)
    assert torch.equal(a.out, b.out)


# ---- together ------------------------------------------------------------------------
def test_offsets_past_32_bits():
    """A pool of more than 4 GiB, its last page in use."""
    b = Batch([70, 33], [40, 1], kv_heads=1, group=2, d=128, page=32)
    stride = (1 << 31) + 512                        # elements: pages 4 GiB apart
    big = [torch.zeros(2 * stride + 32 * 128, dtype=torch.float16, device="cuda") for _ in range(2)]
    b.table[0, :3] = torch.tensor([2, 0, 1], dtype=torch.int32)
    b.table[1, :2] = torch.tensor([1, 2], dtype=torch.int32)
    for pool, mem in ((b.k_pool, big[0]), (b.v_pool, big[1])):
        pool[:3] = torch.randn(3, 1, 32, 128, device="cuda").half()
        for i in range(3):
            mem[i * stride:i * stride + 32 * 128] = pool[i].flatten()
    ws = b.workspace()
    kv = b.kv(k=big[0].data_ptr(), v=big[1].data_ptr(), page_stride=stride, n_pages=3)
    vt.vt_paged_chunk_attn(kv, b.io(), 0.0, 0, ws.data_ptr(), ws.numel(), None)
    torch.cuda.synchronize()
    b.check(rounded=True)
    assert int(b.status) == 0


@pytest.mark.parametrize("new", [1, 3, 200])
def test_windows_at_the_largest_positions(new):
    """Attention does not depend on where a window lies: the same one at the end of the range of
    positions, its other pages long gone, gives the same bits."""
    b = Batch([30000], [new], kv_heads=2, group=2, d=64, page=32768, window=100)
    b.attend()
    b.check(rounded=True)
    out, lse = b.out.clone(), b.lse.clone()
    far = 65534
    table = torch.full((1, far + 1), -1, dtype=torch.int32, device="cuda")
    table[0, far] = b.table[0, 0]
    b.table, b.max_pages = table, far + 1
    b.len += far * 32768
    ws = b.workspace()
    vt.vt_paged_chunk_attn(b.kv(ld_table=far + 1), b.io(), 0.0, 100, ws.data_ptr(), ws.numel(), None)
    torch.cuda.synchronize()
    assert torch.equal(out, b.out) and torch.equal(lse, b.lse) and int(b.status) == 0


def test_contiguous_cache_of_the_layer():
    """The cache that vt_layer_prefill_chunk fills, read as a paged one: slots of a head side by
    side, table 0, 1, 2, .. ; its last page is not whole."""
    from synth import get
    from tests.gpu_common import GpuShard
    wl = get("tiny")
    sh = GpuShard(wl, capacity=wl.ctx + 50, max_tokens=50, fill_ctx=True)
    sh.prefill(sh.li.x_chunk(50))
    n, H, d = sh.kv.len, sh.info.n_kv_heads, sh.dims.head_dim
    b = Batch([n], kv_heads=H, group=2, d=d, page=16)
    pages = -(-n // 16)
    table = torch.arange(pages, dtype=torch.int32, device="cuda")
    kv = b.kv(k=sh.kc.data_ptr(), v=sh.vc.data_ptr(), page_stride=16 * d, head_stride=sh.cap * d, slot_stride=d,
              n_pages=pages, table=table.data_ptr(), ld_table=pages, max_pages=pages)
    ws = b.workspace()
    vt.vt_paged_decode_attn(kv, b.io(), 0.0, 0, ws.data_ptr(), ws.numel(), None)
    torch.cuda.synchronize()
    b.fill(0, sh.kc[:, :n].transpose(0, 1), sh.vc[:, :n].transpose(0, 1))
    b.check()


def test_a_conversation_in_pages():
    """Prompts of different lengths in chunks, then tokens one by one, three sequences, through one
    captured graph per shape: append, then attention, against the whole sequences in float64."""
    H, G, d, P, steps = 2, 4, 128, 16, 6
    total = [37, 150, 5]
    b = Batch([n + steps for n in total], kv_heads=H, group=G, d=d, page=P, act="bf16", extra=1)
    g = torch.Generator(device="cuda").manual_seed(4)
    rows = {s: torch.empty((n, (H * G + 2 * H) * d), device="cuda").normal_(generator=g).bfloat16()
            for s, n in enumerate(b.lens)}
    b.k_pool.fill_(math.nan)
    b.v_pool.fill_(math.nan)
    status = b.status
    done = [0, 0, 0]
    ws = None

    def step(new):
        nonlocal ws
        s = Batch([1], kv_heads=H, group=G, d=d, page=P, act="bf16")
        s.__dict__.update(k_pool=b.k_pool, v_pool=b.v_pool, table=b.table, max_pages=b.max_pages, n_pages=b.n_pages,
                          status=status)
        s.lens, s.new = [a + t for a, t in zip(done, new)], list(new)
        s.ragged = new != [1, 1, 1]
        s.len = torch.tensor(s.lens, dtype=torch.int32, device="cuda")
        s.begin = torch.tensor([0] + list(new)).cumsum(0).to(torch.int32).cuda()
        s.rows = s.n_tok = sum(new)
        qkv = torch.cat([rows[i][done[i]:done[i] + t] for i, t in enumerate(new)])
        w = H * G * d
        s.q = torch.empty((s.rows, w), dtype=torch.bfloat16, device="cuda")
        s.out = torch.full_like(s.q, 7.0)
        s.lse = torch.full((s.rows, H * G), 7.0, device="cuda")
        ws = s.workspace() if ws is None else ws
        p, ld = qkv.data_ptr(), qkv.shape[1]
        io = s.io(q=p, ld_q=ld, k=p + 2 * w, ld_k=ld, v=p + 2 * (w + H * d), ld_v=ld)
        call = vt.vt_paged_chunk_attn if s.ragged else vt.vt_paged_decode_attn
        graph = torch.cuda.CUDAGraph()
        kv = s.kv()
        with torch.cuda.graph(graph):
            st = torch.cuda.current_stream().cuda_stream
            vt.vt_paged_append(kv, io, 10000.0, 0, st)
            call(kv, io, 0.0, 0, ws.data_ptr(), ws.numel(), st)
        for _ in range(2):   # a step done twice is the same step
            graph.replay()
            torch.cuda.synchronize()
            s.check(rounded=True)
        want = rotated(qkv[:, :w].double().view(-1, H * G, d), torch.cat(
            [torch.arange(a, a + t, device="cuda") for a, t in zip(done, new)]), 10000.0, 0)
        assert bool(((s.q.double().view_as(want) - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all())
        for i, t in enumerate(new):
            done[i] += t

    step([20, 70, 5])
    step([17, 3, 0])
    step([0, 77, 0])
    for _ in range(steps):
        step([1, 1, 1])
    assert done == b.lens and int(status) == 0
    # the cache holds the rotated keys and the values of every position
    for s, n in enumerate(b.lens):
        k = rows[s][:, H * G * d:(H * G + H) * d].double().view(n, H, d)
        want = rotated(k, torch.arange(n, device="cuda"), 10000.0, 0)
        assert bool(((b.read(b.k_pool, s) - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all())
        assert torch.equal(b.read(b.v_pool, s), rows[s][:, (H * G + H) * d:].double().view(n, H, d))


def test_graph_replays_follow_the_lengths():
    """One captured decode serves other lengths, tables and queries; with eager work in between."""
    b = Batch([700, 300, 64], kv_heads=2, group=4, d=128)
    ws = b.workspace()
    b.attend(ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.attend(ws, sync=False)
    full = list(b.lens)
    for lens in ([700, 300, 64], [1, 0, 64], [699, 17, 3], [0, 0, 0], full):
        b.lens = lens
        b.len.copy_(torch.tensor(lens, dtype=torch.int32))
        b.q.copy_(torch.randn_like(b.q))
        b.out.fill_(7.0)
        torch.randn(300, 300, device="cuda").sum()
        g.replay()
        torch.cuda.synchronize()
        assert not ws[:8192].any()
        b.check()
        again = b.out.clone()
        b.attend(ws)
        assert torch.equal(again, b.out)


def test_one_workspace_for_many_shapes():
    """A workspace of the largest need serves every smaller call in turn."""
    ws = Batch([1], kv_heads=1, group=16, d=128).workspace()
    for lens, new, group, d in (([9000, 50], None, 16, 128), ([3000], [100], 2, 64), ([30] * 40, None, 1, 64),
                                ([20000], None, 1, 128), ([800, 20], [500, 20], 8, 128)):
        b = Batch(lens, new, kv_heads=1, group=group, d=d, page=32)
        b.attend(ws)
        b.check(rounded=new is not None)


def test_partial_results_stay_in_the_workspace():
    """505 units, each a little too long for one piece: the most pieces that a split comes to."""
    b = Batch([5600] * 101, [128] * 101, kv_heads=5, group=1, d=64, page=64)
    n = b.workspace().numel()
    ws = torch.zeros(n + (1 << 20), dtype=torch.uint8, device="cuda")
    ws[n:] = 0xA5
    vt.vt_paged_chunk_attn(b.kv(), b.io(), 0.0, 0, ws.data_ptr(), n, None)
    torch.cuda.synchronize()
    assert bool((ws[n:] == 0xA5).all()) and not ws[:8192].any()
    b.check(rounded=True)


def test_two_streams_with_a_workspace_each():
    a = Batch([30000], kv_heads=2, group=4, d=128, page=64, seed=1)
    b = Batch([5000, 20], [300, 20], kv_heads=2, group=2, d=64, seed=2)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    wss = a.workspace(), b.workspace()
    torch.cuda.synchronize()
    for _ in range(3):
        for x, s, w in zip((a, b), streams, wss):
            with torch.cuda.stream(s):
                x.attend(w, sync=False)
    torch.cuda.synchronize()
    a.check()
    b.check(rounded=True)


def test_results_repeat_bit_for_bit():
    for b in (Batch([30001, 7], kv_heads=2, group=8, d=128, page=64), Batch([3000, 90], [200, 90], kv_heads=1, group=4, d=128)):
        ws = b.workspace()
        first = [t.clone() for t in b.attend(ws)]
        for _ in range(4):
            again = b.attend(ws)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("seed", range(12))
def test_random_batches(seed):
    rng = np.random.default_rng(1000 + seed)
    n = int(rng.integers(1, 12))
    new = np.maximum(0, np.exp(rng.uniform(-0.5, 5.5, n)).astype(int))
    lens = new + np.exp(rng.uniform(0, 7, n)).astype(int) - 1
    if new.sum() == 0:
        new[0], lens[0] = 1, max(1, lens[0])
    f8 = bool(rng.random() < 0.4)
    b = Batch(lens.tolist(), new.tolist(), kv_heads=int(rng.choice([1, 2, 3, 8])), group=int(rng.choice([1, 2, 5, 8, 16])),
              d=int(rng.choice([64, 128])), page=int(2 ** rng.integers(0, 9)), order=str(rng.choice(["head", "slot"])),
              act=str(rng.choice(["f16", "bf16"])), f8=f8, window=int(rng.choice([0, 0, 50, 400])), pad=int(rng.integers(0, 3)),
              seed=seed)
    b.attend()
    b.check(rounded=True)
    assert int(b.status) == 0
