"""The paged key-value cache operators as measurable cases.

A server that runs a shard for several sequences keeps their keys and values in pages
of a pool. Three operators work on it: new tokens are rotated and appended
(``append``), one new token per sequence attends to its cache (``decode``), and
chunks of several new tokens per sequence attend causally to theirs (``chunk``).

``run`` makes the calls where ``own`` is true; else it computes the same from
elementary torch operations in float32 (angles in float64). ``exact`` is the
definition in float64, sequence by sequence.
"""
import math
import random

import torch

own = False

F16, BF16, F8 = torch.float16, torch.bfloat16, torch.float8_e4m3fn
TYPES = {"f16": F16, "bf16": BF16, "f8": F8}
E4M3_MAX = 448.0


def _case(kind, type, cache, kv_heads, group, head_dim, page, order, seqs, lens, tokens=1, spread=0.0, window=0,
          base=10000.0, halves=False, idle=0):
    """seqs sequences of up to ``lens`` positions with up to ``tokens`` new ones each; ``spread`` is the share by
    which lengths fall below that (0: all alike), ``idle`` the batch slots without a sequence."""
    return dict(kind=kind, type=type, cache=cache, kv_heads=kv_heads, group=group, head_dim=head_dim, page=page,
                order=order, seqs=seqs, lens=lens, tokens=tokens, spread=spread, window=window, base=base,
                halves=halves, idle=idle)


def listed():
    return [
        # One new token of one sequence on the small layer (8 heads of 64): launch latency.
        dict(name="append_one", **_case("append", "f16", "f16", 8, 1, 64, 16, "head", 1, 129)),
        # A decode step's tokens of 64 sequences on the 70B-shaped GQA layer (64 heads, 8 KV heads).
        dict(name="append_step_64", **_case("append", "f16", "f16", 8, 8, 128, 16, "head", 64, 4096, spread=0.9)),
        # Ragged prompts of the 7B-shaped layer going into an 8-bit cache, slots outside heads.
        dict(name="append_prompts_f8", **_case("append", "bf16", "f8", 32, 1, 128, 64, "slot", 11, 1537, tokens=1201,
                                               spread=0.7, base=500000.0, halves=True)),
        # A short context of one sequence on the small layer: launch latency.
        dict(name="decode_one", **_case("decode", "f16", "f16", 8, 1, 64, 16, "head", 1, 129)),
        # The ordinary serving step: 64 sequences around 4096 positions, GQA.
        dict(name="decode_64_gqa", **_case("decode", "f16", "f16", 8, 8, 128, 16, "head", 64, 4097, spread=0.5)),
        # A wide ragged batch on the 7B-shaped layer, three slots idle, slots outside heads.
        dict(name="decode_125_mha", **_case("decode", "bf16", "bf16", 32, 1, 128, 64, "slot", 125, 2053, spread=0.95,
                                            idle=3)),
        # One sequence with a very long 8-bit cache: the work has to be split over its length.
        dict(name="decode_long_f8", **_case("decode", "bf16", "f8", 8, 8, 128, 128, "head", 1, 131071)),
        # A few drafted tokens of 16 sequences to be verified at once.
        dict(name="chunk_draft_16", **_case("chunk", "f16", "f16", 8, 8, 128, 16, "head", 16, 4099, tokens=5,
                                            spread=0.6)),
        # A prompt's first 4096 tokens on the 7B-shaped layer.
        dict(name="chunk_prompt_4096", **_case("chunk", "f16", "f16", 32, 1, 128, 16, "head", 1, 4096, tokens=4096)),
        # Ragged prompts with odd lengths, GQA, sliding window of 1024.
        dict(name="chunk_ragged_swa", **_case("chunk", "bf16", "bf16", 8, 4, 128, 32, "slot", 7, 3333, tokens=1999,
                                              spread=0.8, window=1024)),
        # 512 further tokens of a long document in an 8-bit cache.
        dict(name="chunk_512_long_f8", **_case("chunk", "bf16", "f8", 8, 8, 128, 128, "head", 1, 33280, tokens=512)),
        # A short prompt on the small layer: launch latency.
        dict(name="chunk_short", **_case("chunk", "f16", "f16", 8, 1, 64, 16, "head", 1, 17, tokens=17)),
    ]


def _logint(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "decode", "decode", "chunk", "chunk"])
    type = rng.choice(["f16", "bf16"])
    heads = rng.choice([1, 2, 3, 4, 8, 10, 16, 32])
    c = _case(kind, type, rng.choice([type, type, "f8"]), heads, rng.choice([1, 1, 2, 4, 5, 8, 16]) if heads < 16 else 1,
              rng.choice([64, 128, 128]), rng.choice([1, 8, 16, 16, 32, 64, 128, 256]), rng.choice(["head", "slot"]),
              1, 1, spread=round(rng.uniform(0.0, 0.95), 2), window=0 if kind == "append" else rng.choice([0, 0, 0, 100, 1024]),
              base=rng.choice([10000.0, 500000.0]), halves=rng.random() < 0.5)
    if kind == "append":
        c.update(seqs=_logint(rng, 1, 128), tokens=_logint(rng, 1, 4096))
        c.update(lens=c["tokens"] + _logint(rng, 1, 8192))
    elif kind == "decode":
        c.update(seqs=_logint(rng, 1, 128), lens=_logint(rng, 1, 131072), idle=rng.choice([0, 0, 1, 5]))
    else:
        c.update(seqs=_logint(rng, 1, 24), tokens=_logint(rng, 2, 4096))
        c.update(lens=c["tokens"] + rng.choice([0, _logint(rng, 1, 65536)]))
    while _too_large(c):  # shorter and fewer until it costs no more than the largest listed case
        c["seqs"] = max(1, c["seqs"] * 3 // 4)
        c["tokens"] = max(1, c["tokens"] * 3 // 4)
        c["lens"] = max(c["tokens"], c["lens"] * 3 // 4)
    return c


def _too_large(c):
    w = work(c)
    most = max(c["lens"], 1) * c["seqs"] * c["kv_heads"] * c["head_dim"]
    scores = max(c["lens"], 1) * c["seqs"] * c["tokens"] * c["kv_heads"] * c["group"]
    if c["kind"] == "append":
        return w["bytes"] > 2.0e8 or most > 2 ** 28
    if c["kind"] == "decode":
        return w["bytes"] > 2.2e9 or most > 2 ** 30
    return w["flops"] > 1.37e11 or w["bytes"] > 2.2e9 or scores > 2 ** 29 or most > 2 ** 29


# ---- sizes ------------------------------------------------------------------
def _shapes(c):
    """Lengths with the new tokens, and the new tokens, of each batch slot."""
    rng = random.Random(c["seqs"] * 1000003 + c["lens"] * 101 + c["tokens"])
    lens, new = [], []
    for s in range(c["seqs"]):
        short = 1.0 - c["spread"] * rng.random() if s else 1.0  # the first has the full length
        n = max(1, int(c["tokens"] * short))
        new.append(n)
        lens.append(max(n, int(c["lens"] * (1.0 - c["spread"] * rng.random() if s else 1.0))))
    if c["kind"] == "decode":
        lens += [0] * c["idle"]
        new += [1] * c["idle"]
    return lens, new


def work(c):
    lens, new = _shapes(c)
    d, nkv, nq = c["head_dim"], c["kv_heads"], c["kv_heads"] * c["group"]
    kv = 1 if c["cache"] == "f8" else 2
    rows = sum(new)
    if c["kind"] == "append":
        return {"bytes": rows * d * (2 * nq * 2 + 2 * nkv * (2 + kv)), "flops": 6 * rows * d // 2 * (nq + nkv)}
    keys = pairs = 0
    for n, t in zip(lens, new):
        if n == 0:
            continue
        keys += min(n, c["window"] + t - 1) if c["window"] else n
        first, full = n - t, 0  # tokens at first..n-1
        if c["window"]:
            full = max(0, min(t, n - max(first, c["window"] - 1)))  # tokens that see a whole window
        pairs += full * c["window"] + sum(range(first + 1, first + 1 + t - full))
    return {"bytes": 2 * keys * nkv * d * kv + rows * nq * (2 * d * 2 + 4), "flops": 4 * d * nq * pairs}


# ---- inputs -----------------------------------------------------------------
def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    act, cache = TYPES[c["type"]], TYPES[c["cache"]]
    d, nkv, nq, P = c["head_dim"], c["kv_heads"], c["kv_heads"] * c["group"], c["page"]
    lens, new = _shapes(c)
    pages = [-(-n // P) for n in lens]
    spare = 3
    n_pages, most = sum(pages) + spare, max(max(pages), 1) + 2
    # pages in the order in which a pool hands them out after some use; entries past a sequence's end are stale
    free = torch.randperm(n_pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(lens), most), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(pages):
        table[s, :n] = free[at:at + n]
        at += n
    shape = (n_pages, nkv, P, d) if c["order"] == "head" else (n_pages, P, nkv, d)
    k = torch.empty(shape, dtype=act, device="cuda").normal_(generator=g)
    v = torch.empty(shape, dtype=act, device="cuda").normal_(generator=g)
    k_scale = v_scale = None
    if c["cache"] == "f8":  # the usual range of a head's values over the format's
        k_scale = torch.empty(nkv, device="cuda").uniform_(0.01, 0.02, generator=g)
        v_scale = torch.empty(nkv, device="cuda").uniform_(0.01, 0.02, generator=g)
        per = (1, nkv, 1, 1) if c["order"] == "head" else (1, 1, nkv, 1)
        k = (k.float() / k_scale.view(per)).clamp(-E4M3_MAX, E4M3_MAX).to(F8)
        v = (v.float() / v_scale.view(per)).clamp(-E4M3_MAX, E4M3_MAX).to(F8)
    rows = sum(new)
    begin = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    # rows as one QKV projection leaves them
    qkv = torch.empty((rows, (nq + 2 * nkv) * d), dtype=act, device="cuda").normal_(generator=g)
    st = dict(c=c, k=k, v=v, k_scale=k_scale, v_scale=v_scale, table=table, begin=begin, qkv=qkv, rows=rows, most=most,
              len=torch.tensor(lens, dtype=torch.int32, device="cuda"), longest=max(max(lens), 1), widest=max(new),
              seqs=len(lens), n_pages=n_pages, nq=nq)
    if c["kind"] == "append":
        st.update(q=qkv[:, :nq * d], new_k=qkv[:, nq * d:(nq + nkv) * d], new_v=qkv[:, (nq + nkv) * d:],
                  q_rot=torch.empty((rows, nq * d), dtype=act, device="cuda"))
    else:
        st.update(q=qkv[:, :nq * d], out=torch.empty((rows, nq * d), dtype=act, device="cuda"),
                  lse=torch.empty((rows, nq), dtype=torch.float32, device="cuda"))
    if own:
        st.update(_handles(st))
    return st


# ---- the framework's calls ----------------------------------------------------
def _handles(st):
    """The descriptors and the workspace that a program keeps beside its cache."""
    from paper_2607_07046_amd import voltron as vt
    c, d, P, nkv = st["c"], st["c"]["head_dim"], st["c"]["page"], st["c"]["kv_heads"]
    names = {"f16": vt.VT_T_F16, "bf16": vt.VT_T_BF16, "f8": vt.VT_T_F8E4M3}
    p = lambda t: None if t is None else t.data_ptr()
    head = c["order"] == "head"
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv = vt.vt_paged_kv(k=p(st["k"]), v=p(st["v"]), page_stride=nkv * P * d, head_stride=P * d if head else d,
                        slot_stride=d if head else nkv * d, n_pages=st["n_pages"], page_size=P, n_kv_heads=nkv,
                        head_dim=d, type=names[c["cache"]], k_scale=p(st["k_scale"]), v_scale=p(st["v_scale"]),
                        table=p(st["table"]), ld_table=st["most"], max_pages=st["most"], len=p(st["len"]),
                        n_seqs=st["seqs"], status=p(status))
    io = vt.vt_paged_io(type=names[c["type"]], n_tok=st["rows"], n_q_heads=st["nq"],
                        q_begin=None if c["tokens"] == 1 else p(st["begin"]))
    if c["kind"] == "append":
        io.q, io.ld_q, io.k, io.ld_k = p(st["q"]), st["qkv"].shape[1], p(st["new_k"]), st["qkv"].shape[1]
        io.v, io.ld_v, io.q_rot, io.ld_qr = p(st["new_v"]), st["qkv"].shape[1], p(st["q_rot"]), st["nq"] * d
        return dict(vt=vt, kv=kv, io=io, status=status)
    io.q_rot, io.ld_qr = p(st["q"]), st["qkv"].shape[1]
    io.out, io.ld_out, io.lse = p(st["out"]), st["nq"] * d, p(st["lse"])
    ws = torch.zeros(vt.vt_paged_workspace_size(kv, io), dtype=torch.uint8, device="cuda")
    return dict(vt=vt, kv=kv, io=io, status=status, ws=ws)


def _calls(st):
    vt, c = st["vt"], st["c"]
    stream = torch.cuda.current_stream().cuda_stream
    if c["kind"] == "append":
        vt.vt_paged_append(st["kv"], st["io"], c["base"], vt.VT_ROPE_HALVES if c["halves"] else 0, stream)
        return {"q_rot": st["q_rot"], "k": st["k"], "v": st["v"]}
    attend = vt.vt_paged_decode_attn if c["kind"] == "decode" else vt.vt_paged_chunk_attn
    attend(st["kv"], st["io"], 0.0, c["window"], st["ws"].data_ptr(), st["ws"].numel(), stream)
    return {"out": st["out"], "lse": st["lse"]}


# ---- the plain form -----------------------------------------------------------
def _slots(st, pool):
    """The pool as [page][slot][head][d]."""
    return pool.transpose(1, 2) if st["c"]["order"] == "head" else pool


def _where(st):
    """Sequence and position of every row."""
    r = torch.arange(st["rows"], dtype=torch.int32, device="cuda")
    s = torch.searchsorted(st["begin"][1:].contiguous(), r, right=True)
    return s, st["len"][s] - st["begin"][s + 1] + r


def _turn(x, pos, base, halves):
    d = x.shape[-1]
    i = torch.arange(d // 2, dtype=torch.float64, device="cuda")
    a = pos.double()[:, None] * base ** (-2.0 * i / d)
    cos, sin = a.cos().float()[:, None], a.sin().float()[:, None]
    x = x.float()
    if halves:
        u, w = x[..., :d // 2], x[..., d // 2:]
        return torch.cat((u * cos - w * sin, u * sin + w * cos), -1)
    u, w = x[..., 0::2], x[..., 1::2]
    return torch.stack((u * cos - w * sin, u * sin + w * cos), -1).flatten(-2)


def _stored(x, scale, to):
    if scale is None:
        return x.to(to)
    return (x / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(to)


def _plain_append(st):
    c, d = st["c"], st["c"]["head_dim"]
    s, pos = _where(st)
    q = _turn(st["q"].unflatten(1, (-1, d)), pos, c["base"], c["halves"])
    k = _turn(st["new_k"].unflatten(1, (-1, d)), pos, c["base"], c["halves"])
    v = st["new_v"].unflatten(1, (-1, d)).float()
    st["q_rot"].copy_(q.flatten(1))
    page, slot = st["table"][s, pos // c["page"]], pos % c["page"]
    byte = lambda t: t.view(torch.uint8) if t.dtype == F8 else t  # an indexed store has no 8-bit float form
    byte(_slots(st, st["k"]))[page, slot] = byte(_stored(k, st["k_scale"], st["k"].dtype))
    byte(_slots(st, st["v"]))[page, slot] = byte(_stored(v, st["v_scale"], st["v"].dtype))
    return {"q_rot": st["q_rot"], "k": st["k"], "v": st["v"]}


def _plain_attention(st):
    c, d, nkv, G, L = st["c"], st["c"]["head_dim"], st["c"]["kv_heads"], st["c"]["group"], st["longest"]
    B, W = st["seqs"], st["widest"]
    # every sequence's keys and values in order, padded to the longest: [head][sequence] products
    p = torch.arange(L, device="cuda")
    page = st["table"][:, p // c["page"]].clamp(min=0)
    def gather(pool, scale):
        pool = _slots(st, pool)
        pool = (pool.view(torch.uint8) if pool.dtype == F8 else pool)[page, p % c["page"]]
        pool = (pool.view(F8) if scale is not None else pool).float()
        return (pool if scale is None else pool * scale[:, None]).transpose(1, 2)
    keys = gather(st["k"], st["k_scale"]).reshape(B * nkv, L, d)
    values = gather(st["v"], st["v_scale"]).reshape(B * nkv, L, d)
    values = torch.where((p >= st["len"][:, None]).repeat_interleave(nkv, 0)[..., None], 0.0, values)
    # rows padded to the widest chunk
    t = torch.arange(W, device="cuda")
    count = st["begin"].diff()
    row = (st["begin"][:-1, None] + t).clamp(max=st["rows"] - 1)
    q = st["q"].unflatten(1, (nkv, G, d))[row].float().permute(0, 2, 1, 3, 4).reshape(B * nkv, W * G, d)
    scores = torch.bmm(q, keys.transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(d))
    pos = (st["len"] - count)[:, None] + t
    hidden = (p > pos[..., None]) | (t >= count[:, None])[..., None] | (p >= st["len"][:, None, None])
    if c["window"]:
        hidden |= p <= pos[..., None] - c["window"]
    scores = scores.view(B, nkv, W, G, L).masked_fill_(hidden[:, None, :, None], -math.inf).view(B * nkv, W * G, L)
    top = scores.amax(-1, keepdim=True)
    weights = scores.sub_(torch.where(top.isinf(), 0.0, top)).exp_()
    total = weights.sum(-1, keepdim=True)
    out = torch.bmm(weights, values) / torch.where(total == 0, 1.0, total)
    lse = (total.log() + top).squeeze(-1)
    # back to the rows in use
    there = t < count[:, None]
    out = out.view(B, nkv, W, G, d).transpose(1, 2)[there].flatten(1)
    st["out"].copy_(out)
    st["lse"].copy_(lse.view(B, nkv, W, G).transpose(1, 2)[there].flatten(1))
    return {"out": st["out"], "lse": st["lse"]}


def run(st):
    if own:
        return _calls(st)
    return _plain_append(st) if st["c"]["kind"] == "append" else _plain_attention(st)


# ---- the definition in 64 bits ------------------------------------------------
def exact(c, seed):
    st = prepare(c, seed)
    d, nkv, nq, P, G = c["head_dim"], c["kv_heads"], st["nq"], c["page"], c["group"]
    lens, new = _shapes(c)
    k, v = _slots(st, st["k"]), _slots(st, st["v"])
    heads = lambda name: st[name].reshape(st["rows"], -1, d).double()
    row = 0
    if c["kind"] == "append":
        k, v = k.double(), v.double()
        q, nk, nv = heads("q"), heads("new_k"), heads("new_v")
        out = torch.empty_like(q)
        f = torch.tensor([c["base"] ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64, device="cuda")
        first, second = (slice(0, d // 2), slice(d // 2, d)) if c["halves"] else (slice(0, d, 2), slice(1, d, 2))
        for s, (n, t) in enumerate(zip(lens, new)):
            pos = torch.arange(n - t, n, device="cuda")
            z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos[:, None] * f)[:, None]
            at = (st["table"][s, pos // P].long(), pos % P)
            for src, dst in ((q, out), (nk, None)):
                x = src[row:row + t]
                y = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * z
                r = torch.empty_like(x)
                r[..., first], r[..., second] = y.real, y.imag
                if dst is not None:
                    dst[row:row + t] = r
                elif st["k_scale"] is not None:
                    k[at] = (r / st["k_scale"].double()[:, None]).clamp(-E4M3_MAX, E4M3_MAX)
                else:
                    k[at] = r
            w = nv[row:row + t]
            v[at] = w if st["v_scale"] is None else (w / st["v_scale"].double()[:, None]).clamp(-E4M3_MAX, E4M3_MAX)
            row += t
        return {"q_rot": out.flatten(1), "k": k.transpose(1, 2) if c["order"] == "head" else k,
                "v": v.transpose(1, 2) if c["order"] == "head" else v}
    q = heads("q")
    out = torch.zeros_like(q)
    lse = torch.full((st["rows"], nq), -math.inf, dtype=torch.float64, device="cuda")
    one = torch.ones(nkv, dtype=torch.float64, device="cuda")
    ks, vs = (one if st[n] is None else st[n].double() for n in ("k_scale", "v_scale"))
    for s, (n, t) in enumerate(zip(lens, new)):
        if n:
            lo = max(0, n - t - c["window"] + 1) if c["window"] else 0
            used = st["table"][s, :-(-n // P)].long()
            for h in range(nkv):
                kh = k[used, :, h].double().reshape(-1, d)[lo:n] * ks[h]
                vh = v[used, :, h].double().reshape(-1, d)[lo:n] * vs[h]
                for b in range(0, t, 1024):
                    m = min(1024, t - b)
                    rows = slice(row + b, row + b + m)
                    pos = torch.arange(n - t + b, n - t + b + m, device="cuda")[:, None]
                    key = torch.arange(lo, n, device="cuda")[None]
                    seen = key <= pos
                    if c["window"]:
                        seen &= key > pos - c["window"]
                    qh = q[rows, h * G:(h + 1) * G].transpose(0, 1).reshape(G * m, d)
                    x = (qh @ kh.T / math.sqrt(d)).masked_fill(~seen.repeat(G, 1), -math.inf)
                    z = torch.logsumexp(x, -1)
                    lse[rows, h * G:(h + 1) * G] = z.reshape(G, m).T
                    out[rows, h * G:(h + 1) * G] = (torch.exp(x - z[:, None]) @ vh).reshape(G, m, d).transpose(0, 1)
        row += t
    return {"out": out.flatten(1), "lse": lse}
