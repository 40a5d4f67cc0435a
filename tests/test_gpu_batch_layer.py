"""A decoder layer's shard for a batch of sequences over a paged cache, put together from the row
operators and the paged attention: against the fp64 oracle's layer sequence by sequence, and, with
biases, head norms, partial rotation and another gate, against the same steps in float64."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2607_07046_amd import voltron as vt
from synth import get
from synth.gen import LayerInputs
from tests import common
from tests.gpu_common import h16
from tests.paged_common import Batch
from tests.rows_common import ACT_TYPES, ACTS, act64, half_step, p, stream
from tests.test_gpu_rows import turned

pytestmark = pytest.mark.gpu

# The parity bar of tests/common.py is derived for outputs behind two fp16 roundings of a vector (the normalised input,
# the attention output). Here five independent ones stand before the attention partial: the normalised input, the
# projections as written, the rotated queries and keys, the weights of the attention and its output. Errors add
# in squares: sqrt(5 / 2) times the bar.
MORE = math.sqrt(5 / 2)


class Layer:
    """One shard's weights and the buffers of up to ``rows`` rows of a step."""

    def __init__(self, w, b, rows, hidden, eps, rope, act="silu", head_norm=None):
        self.w, self.b, self.rows, self.hidden, self.eps, self.act = w, b, rows, hidden, eps, act
        self.rope, self.head_norm = vt.vt_rope(**rope), head_norm
        self.dtype, self.type = b.dtype, b.type
        buf = lambda n: torch.full((rows, -(-n // 8) * 8), math.nan, dtype=b.dtype, device="cuda")[:, :n]
        d, nq, nkv, cols = b.d, b.nq, b.kv_heads, w["wd"].shape[1]
        self.x, self.u, self.h, self.wn, self.p_attn, self.p_ffn, self.y = (buf(hidden) for _ in range(7))
        self.qkv, self.q_rot, self.o, self.m = buf((nq + 2 * nkv) * d), buf(nq * d), buf(nq * d), buf(cols)
        self.ws = torch.zeros(vt.vt_linear_workspace_size(self.linear(self.u, "wqkv", self.qkv)), dtype=torch.uint8,
                              device="cuda")
        self.attn_ws = b.workspace()

    def linear(self, x, name, y, act="none", residual=None, bias=None, up=None):
        w = self.w[name]
        f = dict(type=self.type, act=ACTS[act], n_rows=self.rows, n_in=w.shape[1], n_out=w.shape[0], x=p(x), ld_x=x.stride(0),
                 w=p(w), ld_w=w.stride(0), bias=p(self.w.get(bias)), y=p(y), ld_y=y.stride(0))
        if residual is not None:
            f.update(residual=p(residual), ld_res=residual.stride(0))
        if up:
            f.update(w_up=p(self.w[up]), ld_up=self.w[up].stride(0))
        return vt.vt_linear_io(**f)

    def norm(self, x, gain, y, partial=None, h=None):
        f = dict(type=self.type, n_rows=self.rows, hidden=self.hidden, eps=self.eps, x=p(x), ld_x=x.stride(0),
                 gain=p(self.w[gain]), y=p(y), ld_y=y.stride(0))
        if partial is not None:
            f.update(partial=p(partial), ld_partial=partial.stride(0), h=p(h), ld_h=h.stride(0))
        vt.vt_norm_rows(vt.vt_norm_io(**f), stream())

    def step(self):
        b, s = self.b, stream()
        d, nq, nkv, wide = b.d, b.nq, b.kv_heads, self.qkv.stride(0)
        run = lambda io, f=vt.vt_linear: f(io, self.ws.data_ptr(), self.ws.numel(), s)
        self.norm(self.x, "g_attn", self.u)
        run(self.linear(self.u, "wqkv", self.qkv, bias="b_qkv"))
        io = b.io(n_tok=self.rows, q=p(self.qkv), ld_q=wide, k=p(self.qkv[:, nq * d:]), ld_k=wide,
                  v=p(self.qkv[:, (nq + nkv) * d:]), ld_v=wide, q_rot=p(self.q_rot), ld_qr=self.q_rot.stride(0), out=p(self.o),
                  ld_out=self.o.stride(0), lse=None)
        vt.vt_paged_append_heads(b.kv(), io, self.head_norm, self.rope, s)
        attend = vt.vt_paged_chunk_attn if b.ragged else vt.vt_paged_decode_attn
        attend(b.kv(), io, 0.0, b.window, self.attn_ws.data_ptr(), self.attn_ws.numel(), s)
        run(self.linear(self.o, "wo", self.p_attn))
        self.norm(self.x, "g_ffn", self.wn, partial=self.p_attn, h=self.h)
        run(self.linear(self.wn, "wg", self.m, act=self.act, up="wu"), vt.vt_linear_gated)
        run(self.linear(self.m, "wd", self.p_ffn))
        run(self.linear(self.m, "wd", self.y, residual=self.h))


@pytest.mark.parametrize("key,lens,new", [
    ("tiny", [140, 57, 9, 200], [12, 1, 9, 130]), ("tiny", [17, 129, 1, 60, 33], None),
    ("7b", [300, 64, 77], [260, 1, 16]), ("7b", [1025, 1, 350, 18], None), ("70b_gqa", [40, 90], [3, 90])])
def test_layer_of_a_batch(key, lens, new):
    wl = get(key)
    d, li = wl.dims, LayerInputs(wl)
    r = oracle.shard_ranges(d.n_heads, d.n_kv_heads, d.ffn, wl.fracs, wl.fracs, wl.device)
    hd = d.head_dim
    q0, q1 = r.q_head_begin * hd, (r.q_head_begin + r.n_q_heads) * hd
    k0, k1 = r.kv_head_begin * hd, (r.kv_head_begin + r.n_kv_heads) * hd
    c0, c1 = r.col_begin, r.col_begin + r.n_cols
    ow = oracle.ShardWeights(g_attn=li.g_attn(), wq=li.rows("wq", q0, q1), wk=li.rows("wk", k0, k1),
                             wv=li.rows("wv", k0, k1), wo=li.cols("wo", q0, q1), g_ffn=li.g_ffn(),
                             wg=li.rows("wg", c0, c1), wu=li.rows("wu", c0, c1), wd=li.cols("wd", c0, c1))

    def padded(a):  # rows of a multiple of 8, NaN between
        t = h16(a)
        out = torch.full((t.shape[0], -(-t.shape[1] // 8) * 8), math.nan, dtype=t.dtype, device="cuda")[:, :t.shape[1]]
        return out.copy_(t)

    w = dict(wqkv=padded(np.concatenate([ow.wq, ow.wk, ow.wv])), wo=padded(ow.wo), wg=padded(ow.wg), wu=padded(ow.wu),
             wd=padded(ow.wd), g_attn=h16(ow.g_attn), g_ffn=h16(ow.g_ffn))
    b = Batch(lens, new, kv_heads=r.n_kv_heads, group=r.n_q_heads // r.n_kv_heads, d=hd, page=16, window=d.window)
    layer = Layer(w, b, b.rows, d.hidden, d.rms_eps, dict(base=d.rope_base))
    new = b.new
    k_ctx, v_ctx = li.kv_context_heads(r.kv_head_begin, r.kv_head_begin + r.n_kv_heads)  # [heads][positions][d]
    X = li.x_chunk(b.rows) if b.rows > 1 else li.x(0)[None]
    layer.x.copy_(h16(X))
    for s, (n, t) in enumerate(zip(lens, new)):  # each sequence's own stretch of the context
        ctx = n - t
        if ctx:
            at, c = b.at(s, 0, ctx), min(s, k_ctx.shape[1] - ctx)
            kt, vt_ = (h16(np.transpose(a[:, c:c + ctx], (1, 0, 2))) for a in (k_ctx, v_ctx))
            b.slots(b.k_pool)[at], b.slots(b.v_pool)[at] = kt, vt_
    layer.step()
    torch.cuda.synchronize()
    row = 0
    for s, (n, t) in enumerate(zip(lens, new)):
        ctx, rows = n - t, slice(row, row + t)
        row += t
        c = min(s, k_ctx.shape[1] - ctx)
        ref = oracle.prefill(ow, r.n_q_heads, r.n_kv_heads, hd, d.rms_eps, d.rope_base, X[rows], k_ctx[:, c:c + ctx],
                             v_ctx[:, c:c + ctx], ctx, window=d.window)
        ref["p_ffn"], ref["y"] = oracle.ffn_sublayer(ow, d.rms_eps, np.asarray(ref["h"], np.float16).astype(np.float64))
        for name in ("p_attn", "h", "p_ffn", "y"):
            got = getattr(layer, name)[rows].float().cpu().numpy().astype(np.float64)
            assert common.max_rel_err(got, ref[name]) <= MORE * common.REL_TOL, (name, s)
            assert common.norm_rel_err(got, ref[name]) <= MORE * common.NORM_TOL, (name, s)


def model64(layer, gains, rope, eps_head):
    """The step in float64 from layer.x and the cache before it, rounded where the device writes a result."""
    b, w, t = layer.b, layer.w, layer.dtype
    R = lambda a: a.to(t).double()
    D = lambda name: w[name].double()
    norm = lambda a, g: R(a / (a.square().mean(-1, keepdim=True) + layer.eps).sqrt() * D(g))
    x = layer.x.double()
    qkv = R(norm(x, "g_attn") @ D("wqkv").t() + D("b_qkv"))
    nq, nkv, d, G = b.nq, b.kv_heads, b.d, b.group
    heads = qkv.unflatten(1, (-1, d))
    pos = torch.cat([torch.arange(n - k, n) for n, k in zip(b.lens, b.new)]).cuda()
    q = R(turned(heads[:, :nq], gains[0], pos, rope, d, eps_head, t)[0])
    k = R(turned(heads[:, nq:nq + nkv], gains[1], pos, rope, d, eps_head, t)[0])
    v = heads[:, nq + nkv:]
    o = torch.zeros_like(q)
    row = 0
    for s, (n, m) in enumerate(zip(b.lens, b.new)):
        rows = slice(row, row + m)
        row += m
        ks, vs = b.read(b.k_pool, s).clone(), b.read(b.v_pool, s).clone()
        ks[n - m:], vs[n - m:] = k[rows], v[rows]
        for h in range(nq):
            sc = q[rows, h] @ ks[:, h // G].t() / math.sqrt(d)
            hidden = torch.arange(n, device="cuda")[None] > torch.arange(n - m, n, device="cuda")[:, None]
            o[rows, h] = torch.softmax(sc.masked_fill(hidden, -math.inf), -1) @ vs[:, h // G]
    o = R(o.flatten(1))
    p_attn = R(o @ D("wo").t())
    h = R(x + p_attn)
    wn = norm(h, "g_ffn")
    m = R(act64(wn @ D("wg").t(), layer.act) * (wn @ D("wu").t()))
    return dict(qkv=qkv, q_rot=q.flatten(1), o=o, p_attn=p_attn, h=h, wn=wn, m=m, y=R(h + m @ D("wd").t()))


def batch_layer(type, lens, new, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype, _ = ACT_TYPES[type]
    H, kv_heads, group, d, cols = 520, 2, 3, 64, 700
    b = Batch(lens, new, kv_heads=kv_heads, group=group, d=d, page=8, act=type, extra=3, seed=seed)
    rnd = lambda *s, sigma=1.0, mean=0.0: torch.empty(s, device="cuda").normal_(mean, sigma, generator=g).to(dtype)
    wq = (kv_heads * group + 2 * kv_heads) * d
    w = dict(wqkv=rnd(wq, H, sigma=H ** -0.5), b_qkv=rnd(wq, sigma=0.3), wo=rnd(H, b.nq * d, sigma=(b.nq * d) ** -0.5),
             wg=rnd(cols, H, sigma=H ** -0.5), wu=rnd(cols, H, sigma=H ** -0.5), g_attn=rnd(H, sigma=0.1, mean=1.0),
             g_ffn=rnd(H, sigma=0.1, mean=1.0))
    wd = torch.full((H, 704), math.nan, dtype=dtype, device="cuda")[:, :cols]
    w["wd"] = wd.copy_(rnd(H, cols, sigma=cols ** -0.5))
    gains = (rnd(d, sigma=0.1, mean=1.0), rnd(d, sigma=0.1, mean=1.0))
    rope = dict(base=500000.0, dims=48, flags=1, factor=4.0, low=1.0, high=4.0, context=64, amplitude=1.1)
    layer = Layer(w, b, b.rows, H, 1e-5, rope, "gelu_tanh", vt.vt_head_norm(q_gain=p(gains[0]), k_gain=p(gains[1]), eps=1e-6))
    layer.x.copy_(rnd(b.rows, H))
    return layer, gains, rope


def check(layer, want):
    """Each result against the model's. They are rounded at the same places; in front of a rounding they differ by far
    less than a step, so some of a step's results are a step apart, and what follows carries that on: after n roundings
    at most n half steps in the 2-norm (each moves a vector by less than a half step of it; products with these
    weights and norms keep relative errors, up to a factor of 2 for the gated product of two)."""
    torch.cuda.synchronize()
    for n, name in enumerate(("qkv", "q_rot", "o", "p_attn", "h", "wn", "m", "y"), 2):
        got = getattr(layer, name).double()
        off = float((got - want[name]).norm() / want[name].norm())
        assert off <= 2 * n * half_step(layer.dtype), (name, off)


@pytest.mark.parametrize("type", ["f16", "bf16"])
@pytest.mark.parametrize("lens,new", [([70, 5, 33], [70, 1, 8]), ([70, 5, 33, 9], None), ([300], [280]), ([1], None)])
def test_layer_with_everything(type, lens, new):
    layer, gains, rope = batch_layer(type, lens, new)
    want = model64(layer, gains, rope, 1e-6)
    layer.step()
    check(layer, want)


def test_captured_layer_over_several_steps():
    """One captured step for single tokens; lengths grow and inputs change between its replays."""
    layer, gains, rope = batch_layer("f16", [20, 7, 31], None)
    b = layer.b
    layer.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step()
    free = set(range(b.n_pages)) - {int(x) for s, n in enumerate(b.lens) for x in b.table[s, :-(-n // b.page)]}
    for _ in range(4):
        for s, n in enumerate(b.lens):
            if n % b.page == 0:
                b.table[s, n // b.page] = free.pop()
        b.lens = [n + 1 for n in b.lens]
        b.len += 1
        layer.x.normal_()
        for t in (layer.qkv, layer.o, layer.m, layer.y):
            t.fill_(math.nan)
        want = model64(layer, gains, rope, 1e-6)
        graph.replay()
        check(layer, want)
    assert int(b.status) == 0
