"""vt_norm_rows, vt_rotate_heads and vt_paged_append_heads against float64, element by element."""
import math

import pytest
import torch

from paper_2607_07046_amd import voltron as vt
from tests.paged_common import F8, Batch
from tests.rows_common import ACT_TYPES, MARK, around, half_step, ld, least, marked, matrix, p, stream, untouched

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("type", ["f16", "bf16"])


# ---- norms of rows ------------------------------------------------------------
class Norm:
    def __init__(self, type, M, N, parts=0, with_h=True, eps=1e-5, sigma=1.0, seed=0, pad=8):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.dtype, self.type = ACT_TYPES[type]
        self.M, self.N, self.eps = M, N, eps
        make = lambda: matrix(g, M, N, self.dtype, pad, sigma)
        self.x, self.partial, self.peer = make(), make() if parts > 0 else None, make() if parts > 1 else None
        self.gain = torch.empty(N, device="cuda").normal_(1, 0.3, generator=g).to(self.dtype)
        self.h = marked(M, N, self.dtype, pad) if with_h else None
        self.y = marked(M, N, self.dtype, pad)

    def call(self, **change):
        f = dict(type=self.type, n_rows=self.M, hidden=self.N, eps=self.eps, x=p(self.x), ld_x=ld(self.x),
                 partial=p(self.partial), ld_partial=ld(self.partial), peer=p(self.peer), ld_peer=ld(self.peer),
                 gain=p(self.gain), h=p(self.h), ld_h=ld(self.h), y=p(self.y), ld_y=ld(self.y))
        f.update(change)
        vt.vt_norm_rows(vt.vt_norm_io(**f), stream())

    def reference(self):
        """h: two fp32 additions and a rounding. y, of h as the kernel wrote it or, where it did not, of the same
        sums rounded by torch: the mean of N squares is within (N + 2) 2^-24 of itself, its root within half of that,
        the quotient and three products add 4 2^-24."""
        h = self.x.float()
        for t in (self.partial, self.peer):
            h = h if t is None else h + t.float()
        want_h = self.x.double() + sum(t.double() for t in (self.partial, self.peer) if t is not None)
        h = h.to(self.dtype).double()
        eps = float(torch.tensor(self.eps, dtype=torch.float32))  # as the call takes it (1e-42 is 5e-4 off)
        y = h / (h.square().mean(-1, keepdim=True) + eps).sqrt() * self.gain.double()
        tol = (half_step(self.dtype) + (self.N / 2 + 6) * 2.0 ** -24) * y.abs() + least(self.dtype)
        size = self.x.double().abs() + sum(t.double().abs() for t in (self.partial, self.peer) if t is not None)
        return want_h, half_step(self.dtype) * want_h.abs() + 2.0 ** -23 * size + least(self.dtype), y, tol

    def check(self, ref=None):
        want_h, tol_h, y, tol = ref or self.reference()
        torch.cuda.synchronize()
        if self.h is not None:
            assert bool(((self.h.double() - want_h).abs() <= tol_h).all()) and untouched(self.h)
        off = (self.y.double() - y).abs() - tol
        assert bool((off <= 0).all()), f"worst {float(off.max())} over its tolerance"
        assert untouched(self.y)


@BOTH
@pytest.mark.parametrize("M,N", [(1, 1), (1, 7), (3, 8), (5, 100), (4, 511), (1, 512), (9, 513), (64, 1001), (65, 1024),
                                 (130, 2050), (64, 4096), (1, 8192), (63, 8192), (2, 9000), (3, 16383), (2, 16384),
                                 (1500, 40), (1100, 1376), (2049, 520), (1025, 5120), (1030, 8200), (1026, 16384)])
@pytest.mark.parametrize("parts", [0, 1, 2])
def test_norm(type, M, N, parts):
    x = Norm(type, M, N, parts, seed=M + N)
    x.call()
    x.check()


@BOTH
@pytest.mark.parametrize("M,N", [(3, 515), (200, 4096), (1200, 1000)])
def test_norm_without_h(type, M, N):
    for parts in (0, 2):
        x = Norm(type, M, N, parts, with_h=False, seed=2)
        x.call()
        x.check()


@BOTH
@pytest.mark.parametrize("M,N", [(5, 300), (70, 4096), (1300, 2056)])
@pytest.mark.parametrize("out,into", [("h", "x"), ("h", "partial"), ("h", "peer"), ("y", "x"), ("y", "peer")])
def test_norm_in_place(type, M, N, out, into):
    x = Norm(type, M, N, 2, seed=4)
    ref = x.reference()
    t = getattr(x, into)
    x.call(**{out: p(t), "ld_" + out: ld(t)})
    torch.cuda.synchronize()
    getattr(x, out).copy_(t)
    assert bool(around(t)[:, N:].isnan().all())
    x.check(ref)


@BOTH
@pytest.mark.parametrize("h,y", [("x", "partial"), ("partial", "x"), ("peer", "partial")])
@pytest.mark.parametrize("M,N", [(3, 40), (67, 900), (1100, 2050), (9, 16384)])
def test_norm_with_both_outputs_in_place(type, M, N, h, y):
    x = Norm(type, M, N, 2, seed=5)
    ref = x.reference()
    th, ty = getattr(x, h), getattr(x, y)
    x.call(h=p(th), ld_h=ld(th), y=p(ty), ld_y=ld(ty))
    torch.cuda.synchronize()
    x.h.copy_(th)
    x.y.copy_(ty)
    x.check(ref)


@pytest.mark.parametrize("N", [8, 500, 5000])
@pytest.mark.parametrize("size,eps", [(3e38, 1e-5), (1e25, 0.0), (1e-30, 0.0), (1e-20, 1e-5), (1e-38, 0.0), (1e-22, 1e-42)])
def test_norm_of_any_bf16_numbers(N, size, eps):
    """Squares outside of fp32's range, next to rows inside it."""
    x = Norm("bf16", 6, N, 0, eps=eps, seed=7)
    x.x[::2] = (x.x[::2].double().clamp(-1, 1) * size).to(torch.bfloat16)
    x.call()
    want_h, tol_h, y, tol = x.reference()
    x.check((want_h, tol_h, y, tol + 2.0 ** -126))  # (numbers below fp32's normal ones may count as zero)


@BOTH
def test_norm_of_zeros_infinities_and_nan(type):
    x = Norm(type, 6, 1000, 0)
    x.x[0] = 0
    x.x[1, 999] = math.inf
    x.x[2, 0] = math.nan
    clean = Norm(type, 6, 1000, 0)
    x.call()
    clean.call()
    torch.cuda.synchronize()
    assert bool((x.y[0] == 0).all())
    assert bool(x.y[1, 999].isnan()) and bool((x.y[1, :999] == 0).all())
    assert bool(x.y[2].isnan().all())
    assert torch.equal(x.y[3:], clean.y[3:])
    x = Norm(type, 1, 16, 0, eps=0.0)
    x.x.zero_()
    x.call()
    torch.cuda.synchronize()
    assert bool(x.y.isnan().all())


def test_norm_beyond_2_gib():
    M, wide = 70000, 16384
    buf = torch.empty((M, wide), dtype=torch.float16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    buf[:, :512].normal_(generator=g)
    x = Norm("f16", 300, 512, 0)
    x.call(n_rows=M, x=p(buf), ld_x=wide, h=buf[:, 4096:].data_ptr(), ld_h=wide, y=buf[:, 8192:].data_ptr(), ld_y=wide)
    for first in (0, M - 300):
        rows = slice(first, first + 300)
        x.x.copy_(buf[rows, :512])
        x.h.copy_(buf[rows, 4096:4608])
        x.y.copy_(buf[rows, 8192:8704])
        x.check()


# ---- heads --------------------------------------------------------------------
def speeds(rope, d):
    """Radians per position of each pair, one by one from the definition."""
    dims = rope.get("dims", 0) or d
    out = []
    for i in range(dims // 2):
        f = float(torch.tensor(rope["base"], dtype=torch.float32)) ** (-2.0 * i / dims)
        factor, low, high = rope.get("factor", 0.0) or 1.0, rope.get("low", 0.0), rope.get("high", 0.0)
        turns = rope.get("context", 0) * f / math.tau
        k = 0.0 if high == 0 or turns <= low else (1.0 if turns >= high else (turns - low) / (high - low))
        out.append(f * (k + (1 - k) / factor))
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def turned(x, gain, pos, rope, d, eps, dtype):
    """Heads [row][head][d] with their norm and rotation, and a bound. Norm: as for rows, d terms. Angles: in
    double, their cosine and sine from a float of up to half a revolution, 2^-25 of one off (2^-22 rad), evaluated within
    2^-22 by the hardware, times the amplitude: 2^-20 (|u| + |w|) in all, the products among it."""
    x = x.double()
    err = torch.zeros_like(x)
    if gain is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * gain.double()
        err = (d / 2 + 6) * 2.0 ** -24 * x.abs()
    if rope is not None and rope["base"]:
        n = (rope.get("dims", 0) or d) // 2
        amp = rope.get("amplitude", 0.0) or 1.0
        a = pos.double()[:, None, None] * speeds(rope, d)
        c, s = a.cos() * amp, a.sin() * amp
        i, j = (slice(0, n), slice(n, 2 * n)) if rope.get("flags") else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
        u, w, eu, ew = x[..., i].clone(), x[..., j].clone(), err[..., i].clone(), err[..., j].clone()
        e = amp * (2.0 ** -20 * (u.abs() + w.abs()) + eu + ew)
        x[..., i], x[..., j] = u * c - w * s, u * s + w * c
        err[..., i], err[..., j] = e, e
    return x, err + half_step(dtype) * (x.abs() + err) + least(dtype)


ROPES = [None, dict(base=0.0), dict(base=10000.0), dict(base=10000.0, flags=1), dict(base=500000.0, dims=32),
         dict(base=500000.0, dims=32, flags=1), dict(base=10000.0, dims=2), dict(base=10000.0, dims=2, flags=1),
         dict(base=10000.0, dims=50), dict(base=10000.0, dims=50, flags=1), dict(base=10000.0, dims=62, flags=1),
         dict(base=10000.0, factor=4.0), dict(base=10000.0, factor=4.0, flags=1, amplitude=1.25),
         dict(base=500000.0, factor=8.0, low=1.0, high=4.0, context=8192, flags=1),
         dict(base=10000.0, dims=24, factor=16.0, low=1.0, high=32.0, context=4096, amplitude=0.5),
         dict(base=1.0, flags=1)]


class Heads:
    def __init__(self, type, M, nq, nk, d, gains=True, far=5000, seed=0, sigma=1.0, eps=1e-6):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.dtype, self.type = ACT_TYPES[type]
        self.M, self.nq, self.nk, self.d, self.eps = M, nq, nk, d, eps
        self.q, self.k = matrix(g, M, nq * d, self.dtype, 16, sigma), matrix(g, M, nk * d, self.dtype, 8, sigma)
        self.q_out, self.k_out = marked(M, nq * d, self.dtype, 8), marked(M, nk * d, self.dtype, 24)
        gain = lambda: torch.empty(d, device="cuda").normal_(1, 0.3, generator=g).to(self.dtype)
        self.q_gain, self.k_gain = (gain(), gain()) if gains else (None, None)
        self.pos = torch.randint(0, far, (M,), dtype=torch.int32, device="cuda", generator=g)

    def call(self, rope=None, **change):
        f = dict(type=self.type, n_tok=self.M, head_dim=self.d, pos=p(self.pos), n_q_heads=self.nq, q=p(self.q),
                 ld_q=ld(self.q), q_out=p(self.q_out), ld_qo=ld(self.q_out), n_k_heads=self.nk, k=p(self.k),
                 ld_k=ld(self.k), k_out=p(self.k_out), ld_ko=ld(self.k_out))
        f.update(change)
        norm = None
        if self.q_gain is not None or self.k_gain is not None:
            norm = vt.vt_head_norm(q_gain=p(self.q_gain), k_gain=p(self.k_gain), eps=self.eps)
        vt.vt_rotate_heads(vt.vt_heads_io(**f), norm, None if rope is None else vt.vt_rope(**rope), stream())

    def check(self, rope, pos=None, ref=None):
        torch.cuda.synchronize()
        pos = self.pos if pos is None else pos
        for name in ("q", "k"):
            out = getattr(self, name + "_out")
            want, tol = ref[name] if ref else self.reference(name, rope, pos)
            off = (out.unflatten(1, (-1, self.d)).double() - want).abs() - tol
            assert bool((off <= 0).all()), f"{name}: worst {float(off.max())} over its tolerance"
            assert untouched(out)

    def reference(self, name, rope, pos):
        x = getattr(self, name).unflatten(1, (-1, self.d))
        return turned(x, getattr(self, name + "_gain"), pos, rope, self.d, self.eps, self.dtype)


@BOTH
@pytest.mark.parametrize("rope", ROPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gains", [False, True])
def test_rotate(type, rope, d, gains):
    x = Heads(type, 13, 5, 3, d, gains)
    x.call(rope)
    x.check(rope)


@BOTH
@pytest.mark.parametrize("M,nq,nk,d", [(1, 1, 1, 64), (1, 64, 8, 128), (2, 1, 0, 64), (3, 0, 1, 128), (511, 7, 1, 64),
                                       (512, 3, 3, 128), (700, 32, 32, 64), (1025, 40, 10, 128), (4, 1024, 1024, 64)])
@pytest.mark.parametrize("halves", [0, 1])
def test_rotate_shapes(type, M, nq, nk, d, halves):
    x = Heads(type, M, max(nq, 1), max(nk, 1), d, seed=M, far=200000)
    rope = dict(base=10000.0, dims=d - 16, flags=halves)
    x.call(rope, n_q_heads=nq, n_k_heads=nk, **({} if nq else dict(q=None, q_out=None)),
           **({} if nk else dict(k=None, k_out=None)))
    x.nq, x.nk = nq, nk
    for name, n in (("q", nq), ("k", nk)):
        if n == 0:
            torch.cuda.synchronize()
            assert bool((around(getattr(x, name + "_out")) == MARK).all())
            setattr(x, name + "_out", marked(M, d, x.dtype))  # stands for what is not computed
            getattr(x, name + "_out").copy_(x.reference(name, rope, x.pos)[0].flatten(1))
    x.check(rope)


@pytest.mark.parametrize("pos0", [0, 17, 1000000, 2 ** 31 - 1 - 599])
def test_rotate_rows_from_a_position(pos0):
    x = Heads("f16", 600, 2, 2, 64)
    rope = dict(base=10000.0, factor=2.0)
    x.call(rope, pos=None, pos0=pos0)
    x.check(rope, torch.arange(600, device="cuda") + pos0)


@BOTH
@pytest.mark.parametrize("rope", [ROPES[2], ROPES[9]])
def test_rotate_in_place(type, rope):
    x = Heads(type, 520, 9, 4, 128)
    ref = {n: x.reference(n, rope, x.pos) for n in ("q", "k")}
    x.call(rope, q_out=p(x.q), ld_qo=ld(x.q), k_out=p(x.k), ld_ko=ld(x.k))
    torch.cuda.synchronize()
    assert bool(around(x.q)[:, 9 * 128:].isnan().all()) and bool(around(x.k)[:, 4 * 128:].isnan().all())
    x.q_out.copy_(x.q)
    x.k_out.copy_(x.k)
    x.check(rope, ref=ref)


def test_rotate_skips_negative_positions():
    x = Heads("f16", 20, 3, 2, 64)
    x.pos[5:9] = -1
    x.pos[11] = -(2 ** 31)
    skipped = x.pos < 0
    x.call(ROPES[3])
    torch.cuda.synchronize()
    assert bool((x.q_out[skipped] == MARK).all()) and bool((x.k_out[skipped] == MARK).all())
    for t, n in ((x.q_out, "q"), (x.k_out, "k")):
        t[skipped] = x.reference(n, ROPES[3], x.pos)[0].flatten(1)[skipped].to(x.dtype)
    x.check(ROPES[3])


@pytest.mark.parametrize("which", ["q_gain", "k_gain"])
def test_norm_of_one_kind_of_heads(which):
    x = Heads("bf16", 9, 4, 2, 128)
    setattr(x, which, None)
    x.call(ROPES[3])
    x.check(ROPES[3])


@pytest.mark.parametrize("size,eps", [(3e38, 1e-5), (1e-30, 0.0), (1e-20, 1e-6)])
def test_head_norms_of_any_bf16_numbers(size, eps):
    """A head whose squares leave fp32's range beside heads whose squares do not."""
    x = Heads("bf16", 6, 4, 2, 64, eps=eps)
    for t in (x.q, x.k):
        v = t.unflatten(1, (-1, 64))
        v[:, ::2] = (v[:, ::2].double().clamp(-1, 1) * size).to(torch.bfloat16)
    x.call(ROPES[3])
    ref = {n: x.reference(n, ROPES[3], x.pos) for n in ("q", "k")}
    x.check(None, ref={n: (w, t + 2.0 ** -126) for n, (w, t) in ref.items()})


def test_odd_numbers_stay_in_their_head():
    """NaN and infinity in a head change that head only; without a norm, in numbers that do not turn, only themselves."""
    for gains in (False, True):
        x, clean = Heads("f16", 4, 4, 2, 128, gains), Heads("f16", 4, 4, 2, 128, gains)
        x.q[1, 2 * 128 + 100] = math.inf
        x.k[2, 5] = math.nan
        rope = dict(base=10000.0, dims=64, flags=1)
        x.call(rope)
        clean.call(rope)
        torch.cuda.synchronize()
        for name, at in (("q", (1, 2, 100)), ("k", (2, 0, 5))):
            a, b = (getattr(t, name + "_out").unflatten(1, (-1, 128)) for t in (x, clean))
            same = a == b
            hit = torch.zeros_like(same)
            if gains:
                hit[at[0], at[1]] = True
            else:
                hit[at] = True
                if at[2] < 64:
                    hit[at[0], at[1], at[2] + 32] = True
            assert bool(same[~hit].all())
            assert not bool(a[at].isfinite())


# ---- into a paged cache -------------------------------------------------------
def append_heads(b, rope, gains, eps=1e-6, seed=1, pad_rows=True, **change):
    """A step's rows through vt_paged_append_heads. Returns q, k and v as given and the rotated queries."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = (b.nq + 2 * b.kv_heads) * b.d
    qkv = torch.full((b.n_tok, wide), math.nan, dtype=b.dtype, device="cuda")
    qkv[:b.rows] = torch.empty((b.rows, wide), device="cuda").normal_(generator=g).to(b.dtype)
    cut = (0, b.nq * b.d, (b.nq + b.kv_heads) * b.d, wide)
    q, k, v = (qkv[:, cut[i]:cut[i + 1]] for i in range(3))
    q_rot = torch.full((b.n_tok, b.nq * b.d), MARK, dtype=b.dtype, device="cuda")
    f = dict(q=p(q), ld_q=wide, k=p(k), ld_k=wide, v=p(v), ld_v=wide, q_rot=p(q_rot))
    f.update(change)
    norm = None if gains is None else vt.vt_head_norm(q_gain=p(gains[0]), k_gain=p(gains[1]), eps=eps)
    vt.vt_paged_append_heads(b.kv(), b.io(**f), norm, None if rope is None else vt.vt_rope(**rope), stream())
    torch.cuda.synchronize()
    return q, k, v, q_rot


def check_append(b, rope, gains, eps, q, k, v, q_rot, before):
    heads = lambda t: t[:b.rows].unflatten(1, (-1, b.d))
    pos = torch.cat([torch.arange(n - t, n) for n, t in zip(b.lens, b.new)]).cuda()
    gq, gk = gains or (None, None)
    there = (pos >= 0).nonzero().flatten()
    want, tol = turned(heads(q)[there], gq, pos[there], rope, b.d, eps, b.dtype)
    assert bool(((heads(q_rot)[there].double() - want).abs() <= tol).all())
    skipped = torch.ones(b.n_tok, dtype=torch.bool, device="cuda")
    skipped[there] = False
    assert bool((q_rot[skipped] == MARK).all())
    wk, tk = turned(heads(k)[there], gk, pos[there], rope, b.d, eps, b.dtype)
    wv = heads(v)[there].double()
    row = 0
    at_k = []
    for s, (n, t) in enumerate(zip(b.lens, b.new)):
        lo = max(n - t, 0)
        if n > lo:
            at_k.append(b.at(s, lo, n - lo))
        row += t
    page, slot = (torch.cat([a[i] for a in at_k]) for i in range(2))
    for name, w, tol, scale in (("k", wk, tk, b.k_scale), ("v", wv, torch.zeros_like(wv), b.v_scale)):
        pool = b.slots(getattr(b, name + "_pool"))
        got = pool[page, slot]
        if b.f8:
            sc = 1.0 if scale is None else scale.double()[:, None]
            got = got.view(F8).double()
            w, tol = (w / sc).clamp(-448, 448), tol / sc
            tol = tol + 2.0 ** -4 * (w.abs() + tol) + 2.0 ** -10  # half a step; the smallest number is 2^-9
        assert bool(((got.double() - w).abs() <= tol).all()), name
        # no other number of the pool changed
        mask = torch.ones(pool.shape[:2], dtype=torch.bool, device="cuda")
        mask[page, slot] = False
        byte = lambda t: t.view(torch.uint8) if t.dtype == torch.uint8 else t.contiguous().view(torch.int16)
        assert torch.equal(byte(pool[mask]), byte(before[name][mask]))


def gains_of(b, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.empty(b.d, device="cuda").normal_(1, 0.3, generator=g).to(b.dtype) for _ in range(2)]


def run_append(b, rope, gains, eps=1e-6):
    before = {n: b.slots(getattr(b, n + "_pool")).clone() for n in ("k", "v")}
    check_append(b, rope, gains, eps, *append_heads(b, rope, gains, eps), before)
    assert int(b.status) == 0


@BOTH
@pytest.mark.parametrize("rope", ROPES)
@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_append(type, rope, f8, d):
    b = Batch([40, 0, 17, 5], [7, 1, 17, 1], kv_heads=3, group=2, d=d, page=16, act=type, f8=f8, pad=3)
    run_append(b, rope, gains_of(b))
    b = Batch([40, 0, 17, 5], kv_heads=3, group=2, d=d, page=16, order="slot", act=type, f8=f8)
    run_append(b, rope, None)


@BOTH
@pytest.mark.parametrize("page,order", [(1, "slot"), (8, "head"), (256, "slot")])
@pytest.mark.parametrize("heads,group", [(1, 1), (8, 8), (32, 1)])
def test_append_layouts(type, page, order, heads, group):
    b = Batch([300, 33, 1, 0, 64], [260, 1, 1, 2, 64], kv_heads=heads, group=group, d=128, page=page, order=order, act=type,
              pad=5, f8=heads == 8)
    run_append(b, dict(base=500000.0, dims=96, flags=1, factor=8.0, low=1.0, high=4.0, context=8192), gains_of(b))


def test_append_many_tokens():
    b = Batch([700, 150], [650, 149], kv_heads=4, group=2, d=64, page=32)
    run_append(b, ROPES[2], gains_of(b))


def test_append_beside_plain_append():
    """Without norms and on the plain rotation: what vt_paged_append stores. Values bit for bit; the products of a
    rotation may be fused otherwise, 2^-22 (|u| + |w|) apart with numbers below 8, so that a few results round the other way."""
    for flags in (0, 1):
        for f8 in (False, True):
            a, b = (Batch([90, 33], [50, 33], kv_heads=4, group=2, d=128, f8=f8, seed=5) for _ in range(2))
            q, k, v, q_rot = append_heads(a, dict(base=10000.0, flags=flags), None)
            wide = q.stride(0)
            other = torch.full_like(q_rot, MARK)
            vt.vt_paged_append(b.kv(), b.io(q=p(q), ld_q=wide, k=p(k), ld_k=wide, v=p(v), ld_v=wide, q_rot=p(other)),
                               10000.0, flags, stream())
            torch.cuda.synchronize()
            byte = lambda t: t.contiguous().view(torch.uint8)
            assert torch.equal(byte(a.v_pool), byte(b.v_pool))
            near = lambda x, y, step: bool((x.isnan() & y.isnan() | ((x - y).abs() <= step * y.abs() + 2.0 ** -18)).all())
            assert near(q_rot.double(), other.double(), 2.0 ** -10)
            assert float((q_rot != other).double().mean()) < 0.01
            assert near(a.k_pool.float().double(), b.k_pool.float().double(), 2.0 ** -3 if f8 else 2.0 ** -10)


@BOTH
def test_append_f8_quotients(type):
    """Quotients exactly between two 8-bit numbers go to the even one, whatever the scale's reciprocal; numbers past the
    largest saturate, infinities too; NaN stays; subnormal and zero quotients. Bit for bit the rounded true quotient."""
    b = Batch([64], [64], kv_heads=4, group=1, d=64, act=type, f8=True)
    b.k_scale = torch.tensor([0.75, 0.01171875, 3.0, 1e-3], device="cuda")
    b.v_scale = torch.tensor([1.0, 5.0, 0.375, 7.0], device="cuda")
    grid = torch.cat([torch.tensor([m * 2.0 ** e for e in range(-12, 9) for m in (1.0, 1.0625, 1.1875, 1.3125, 1.9375)]),
                      torch.tensor([448.0, 456.0, 464.0, 465.0, 480.0, 1e4, 6e4, math.inf, math.nan, 0.0, -0.0])])
    vals = torch.cat([grid, -grid])
    i = torch.arange(64 * 4 * 64) % vals.numel()
    base = vals[i].view(64, 4, 64).cuda()
    rows = lambda scale: (base * scale[:, None]).to(b.dtype).flatten(1)
    k, v = rows(b.k_scale), rows(b.v_scale)
    vt.vt_paged_append_heads(b.kv(), b.io(q=None, q_rot=None, k=p(k), ld_k=256, v=p(v), ld_v=256), None, None, stream())
    torch.cuda.synchronize()
    for x, scale, pool in ((k, b.k_scale, b.k_pool), (v, b.v_scale, b.v_pool)):
        q = (x.view(64, 4, 64).float() / scale[:, None])
        want = torch.where(q.isnan(), q, q.clamp(-448, 448)).to(F8)
        got = b.slots(pool)[b.at(0)].view(F8)
        assert torch.equal(got.float().nan_to_num(1e9), want.float().nan_to_num(1e9))
        assert torch.equal(got.view(torch.uint8) >> 7, want.view(torch.uint8) >> 7) or bool(want.isnan().any())


@pytest.mark.parametrize("at,value", [(3, math.inf), (40, math.nan), (90, math.inf), (127, math.nan)])
def test_append_f8_odd_numbers(at, value):
    """An infinite or NaN number of a key reaches what it turns with as in the formulas, and saturates or stays NaN."""
    b = Batch([20], [20], kv_heads=2, group=1, d=128, f8=True)
    rope = dict(base=10000.0, dims=80, flags=1)
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.empty((20, 256), device="cuda").normal_(generator=g).to(b.dtype) for _ in range(2))
    k[4, at], v[5, at] = value, value
    vt.vt_paged_append_heads(b.kv(), b.io(q=None, q_rot=None, k=p(k), ld_k=256, v=p(v), ld_v=256), None, vt.vt_rope(**rope), stream())
    torch.cuda.synchronize()
    want, _ = turned(k.unflatten(1, (2, 128)), None, torch.arange(20, device="cuda"), rope, 128, 0.0, b.dtype)
    got = b.slots(b.k_pool)[b.at(0)].view(F8).float()
    assert torch.equal(got.isnan(), want.isnan())
    assert bool((got[want.isinf()].abs() == 448).all()) and bool((got[want.isinf()] * want[want.isinf()] > 0).all())
    vq = b.slots(b.v_pool)[b.at(0)].view(F8).float()
    assert torch.equal(vq.isnan(), v.unflatten(1, (2, 128)).isnan())


def test_append_queries_in_place_and_without_queries():
    b = Batch([30, 20], [9, 20], kv_heads=2, group=3, d=64, pad=2)
    gains = gains_of(b)
    before = {n: b.slots(getattr(b, n + "_pool")).clone() for n in ("k", "v")}
    q, k, v, q_rot = append_heads(b, ROPES[3], gains, q=None)
    assert bool((q_rot == MARK).all())
    given = q.clone()
    wide = q.stride(0)
    norm = vt.vt_head_norm(q_gain=p(gains[0]), k_gain=p(gains[1]), eps=1e-6)
    vt.vt_paged_append_heads(b.kv(), b.io(q=p(q), ld_q=wide, k=p(k), ld_k=wide, v=p(v), ld_v=wide, q_rot=p(q), ld_qr=wide),
                             norm, vt.vt_rope(**ROPES[3]), stream())
    torch.cuda.synchronize()
    out = torch.full((b.n_tok, b.nq * b.d), MARK, dtype=b.dtype, device="cuda")
    out[:b.rows] = q[:b.rows]
    assert bool(q[b.rows:].isnan().all())
    check_append(b, ROPES[3], gains, 1e-6, given, k, v, out, before)


def test_append_bad_pages_and_lengths():
    b = Batch([40, 20, 17], [3, 2, 1], kv_heads=2, d=64, page=16)
    b.table[1, 1] = b.n_pages  # positions 18, 19 of the second
    before = {n: b.slots(getattr(b, n + "_pool")).clone() for n in ("k", "v")}
    q, k, v, q_rot = append_heads(b, ROPES[3], None)
    assert int(b.status) == vt.VT_PAGED_BAD_PAGE
    pos = torch.tensor([37, 38, 39, 18, 19, 16], device="cuda")
    want, tol = turned(q.unflatten(1, (-1, 64)), None, pos, ROPES[3], 64, 0, b.dtype)
    assert bool(((q_rot.unflatten(1, (-1, 64)).double() - want).abs() <= tol).all()), "queries are rotated all the same"
    mask = torch.ones(before["k"].shape[:2], dtype=torch.bool, device="cuda")
    for s, first, n in ((0, 37, 3), (2, 16, 1)):
        mask[b.at(s, first, n)] = False
    for n in ("k", "v"):
        now = b.slots(getattr(b, n + "_pool"))
        same = (now == before[n]) | (now.isnan() & before[n].isnan())
        assert bool(same[mask].all()) and not bool(same[~mask].all())
    b = Batch([40, 20], [1, 1], kv_heads=2, d=64, page=16)
    b.len[0] = b.max_pages * 16 + 1
    append_heads(b, None, None)
    assert int(b.status) == vt.VT_PAGED_BAD_LEN


def test_append_graph_with_other_lengths():
    """One captured step; between replays the lengths, pages and rows change."""
    b = Batch([33, 20, 5], kv_heads=2, group=2, d=128, page=16, extra=2)
    gains = gains_of(b)
    wide = (b.nq + 2 * b.kv_heads) * b.d
    qkv = torch.empty((3, wide), dtype=b.dtype, device="cuda")
    q_rot = torch.full((3, b.nq * b.d), MARK, dtype=b.dtype, device="cuda")
    q, k, v = qkv[:, :b.nq * b.d], qkv[:, b.nq * b.d:-b.kv_heads * b.d], qkv[:, -b.kv_heads * b.d:]
    kv, io = b.kv(), b.io(q=p(q), ld_q=wide, k=p(k), ld_k=wide, v=p(v), ld_v=wide, q_rot=p(q_rot))
    norm, rope = vt.vt_head_norm(q_gain=p(gains[0]), k_gain=p(gains[1]), eps=1e-6), ROPES[13]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vt.vt_paged_append_heads(kv, io, norm, vt.vt_rope(**rope), stream())
    for lens in ([34, 0, 6], [35, 21, 7], [36, 22, 8]):
        b.lens = lens
        b.len.copy_(torch.tensor(lens, dtype=torch.int32))
        qkv.normal_()
        q_rot.fill_(MARK)
        before = {n: b.slots(getattr(b, n + "_pool")).clone() for n in ("k", "v")}
        graph.replay()
        torch.cuda.synchronize()
        check_append(b, rope, gains, 1e-6, q, k, v, q_rot, before)
