"""A batch over a paged cache on the device, and the definition in float64.

Everything that a call must not use holds NaN: slots of pages past a
sequence's end, pages that nobody owns, padding rows; table entries past a
sequence's last page point nowhere.
"""
import math

import torch

from paper_2607_07046_amd import voltron as vt

ACT = {"f16": (torch.float16, vt.VT_T_F16), "bf16": (torch.bfloat16, vt.VT_T_BF16)}
F8 = torch.float8_e4m3fn
F8_MAX = 448.0


def half_step(dtype):
    """A rounding's largest relative error."""
    return torch.finfo(dtype).eps / 2


class Batch:
    """Sequences with lens[s] positions, the last new[s] of them this step's."""

    def __init__(self, lens, new=None, kv_heads=2, group=1, d=64, page=16, order="head", act="f16", f8=False, window=0,
                 pad=0, extra=0, seed=0, sigma=1.0, scales=True, ragged=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.new = list(lens), list(new) if new is not None else [1] * len(lens)
        self.ragged = new is not None if ragged is None else ragged
        self.kv_heads, self.group, self.d, self.page, self.window = kv_heads, group, d, page, window
        self.nq = kv_heads * group
        self.dtype, self.type = ACT[act]
        self.cache_dtype = F8 if f8 else self.dtype
        self.order, self.f8 = order, f8
        pages = [-(-n // page) for n in self.lens]
        self.n_pages = sum(pages) + 2
        self.max_pages = max(max(pages), 1) + extra
        free = torch.randperm(self.n_pages, device="cuda", generator=g).to(torch.int32)
        self.table = torch.full((len(lens), self.max_pages + 1), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
        at = 0
        for s, n in enumerate(pages):
            self.table[s, :n] = free[at:at + n]
            at += n
        shape = (self.n_pages, page, kv_heads, d)  # [page][slot][head], in memory as ``order`` says
        self.k_scale = torch.empty(kv_heads, device="cuda").uniform_(0.01, 0.02, generator=g) if f8 and scales else None
        self.v_scale = torch.empty(kv_heads, device="cuda").uniform_(0.01, 0.02, generator=g) if f8 and scales else None
        self.k_pool, self.v_pool = self._pool(shape), self._pool(shape)
        self.len = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.begin = torch.tensor([0] + self.new, dtype=torch.int64).cumsum(0).to(torch.int32).cuda()
        self.rows = sum(self.new)
        self.n_tok = self.rows + pad
        for s, n in enumerate(self.lens):
            if n:
                self.fill(s, torch.empty((n, kv_heads, d), device="cuda").normal_(0, sigma, generator=g),
                          torch.empty((n, kv_heads, d), device="cuda").normal_(0, 1, generator=g))
        self.q = torch.full((self.n_tok, self.nq * d), math.nan, dtype=self.dtype, device="cuda")
        self.q[:self.rows] = torch.empty((self.rows, self.nq * d), device="cuda").normal_(0, sigma, generator=g).to(
            self.dtype)
        self.out = torch.full_like(self.q, 7.0)
        self.lse = torch.full((self.n_tok, self.nq), 7.0, dtype=torch.float32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def _pool(self, shape):
        p, page, h, d = shape
        mem = (p, h, page, d) if self.order == "head" else shape
        t = torch.full(mem, math.nan, dtype=self.dtype, device="cuda").to(self.cache_dtype)
        return t

    def slots(self, pool):
        """[page][slot][head][d] of a pool; 8-bit numbers as bytes."""
        p = pool.view(torch.uint8) if self.f8 else pool
        return p.transpose(1, 2) if self.order == "head" else p

    def at(self, s, first=0, n=None):
        pos = torch.arange(first, self.lens[s] if n is None else first + n, device="cuda")
        return self.table[s, pos // self.page].long(), pos % self.page

    def stored(self, x, scale):
        if not self.f8:
            return x.to(self.dtype)
        x = x.float() if scale is None else x.float() / scale[:, None]
        return x.clamp(-F8_MAX, F8_MAX).to(F8).view(torch.uint8)

    def fill(self, s, k, v):
        self.slots(self.k_pool)[self.at(s)] = self.stored(k, self.k_scale)
        self.slots(self.v_pool)[self.at(s)] = self.stored(v, self.v_scale)

    def read(self, pool, s, scale=None):
        """A sequence's cached numbers in float64, [position][head][d]."""
        x = self.slots(pool)[self.at(s)]
        x = (x.view(F8).float() if self.f8 else x).double()
        return x if scale is None else x * scale.double()[:, None]

    # ---- the calls ------------------------------------------------------------
    def kv(self, **change):
        head, d, P, H = self.order == "head", self.d, self.page, self.kv_heads
        p = lambda t: None if t is None else t.data_ptr()
        f = dict(k=p(self.k_pool), v=p(self.v_pool), page_stride=H * P * d, head_stride=P * d if head else d,
                 slot_stride=d if head else H * d, n_pages=self.n_pages, page_size=P, n_kv_heads=H, head_dim=d,
                 type=vt.VT_T_F8E4M3 if self.f8 else self.type, k_scale=p(self.k_scale), v_scale=p(self.v_scale),
                 table=p(self.table), ld_table=self.max_pages + 1, max_pages=self.max_pages, len=p(self.len),
                 n_seqs=len(self.lens), status=p(self.status))
        f.update(change)
        return vt.vt_paged_kv(**f)

    def io(self, **change):
        w = self.nq * self.d
        f = dict(type=self.type, n_tok=self.n_tok, n_q_heads=self.nq,
                 q_begin=self.begin.data_ptr() if self.ragged else None, q_rot=self.q.data_ptr(), ld_qr=w,
                 out=self.out.data_ptr(), ld_out=w, lse=self.lse.data_ptr())
        f.update(change)
        return vt.vt_paged_io(**f)

    def workspace(self):
        return torch.zeros(vt.vt_paged_workspace_size(self.kv(), self.io()), dtype=torch.uint8, device="cuda")

    def attend(self, ws=None, scale=0.0, sync=True, chunk=None):
        ws = self.workspace() if ws is None else ws
        call = vt.vt_paged_chunk_attn if (self.ragged if chunk is None else chunk) else vt.vt_paged_decode_attn
        call(self.kv(), self.io(), scale, self.window, ws.data_ptr(), ws.numel(),
             torch.cuda.current_stream().cuda_stream)
        if sync:
            torch.cuda.synchronize()
            assert not ws[:8192].any(), "synchronisation words are not zero after the call"
        return self.out, self.lse

    # ---- the definition ---------------------------------------------------------
    def reference(self, scale=0.0, missing=None):
        """out, lse, and what a bound on their errors needs: the weighted mean of |v| and the
        largest sum of |q||k|. missing[s]: positions of sequence s whose page is bad."""
        scale = scale or 1.0 / math.sqrt(self.d)
        G, H, d = self.group, self.kv_heads, self.d
        out = torch.zeros((self.rows, self.nq, d), dtype=torch.float64, device="cuda")
        mean = torch.zeros_like(out)
        lse = torch.full((self.rows, self.nq), -math.inf, dtype=torch.float64, device="cuda")
        size = torch.zeros_like(lse)
        row = 0
        for s, (n, t) in enumerate(zip(self.lens, self.new)):
            rows = slice(row, row + t)
            row += t
            if n == 0 or t == 0:
                continue
            k, v = self.read(self.k_pool, s, self.k_scale), self.read(self.v_pool, s, self.v_scale)
            if missing and s in missing:
                k[missing[s]] = 0.0
                v[missing[s]] = 0.0
            q = self.q[rows].double().view(t, H, G, d).permute(1, 2, 0, 3)            # H G t d
            kt = k.permute(1, 2, 0).contiguous()[:, None]                               # H 1 d n
            x = torch.matmul(q, kt) * scale
            big = torch.matmul(q.abs(), kt.abs()) * scale
            pos = torch.arange(n - t, n, device="cuda")[:, None]
            key = torch.arange(n, device="cuda")[None]
            seen = key <= pos
            if self.window:
                seen &= key > pos - self.window
            if missing and s in missing:
                seen[:, missing[s]] = False
            x = x.masked_fill(~seen, -math.inf)
            z = torch.logsumexp(x, -1, keepdim=True)
            w = torch.where(z.isinf(), 0.0, torch.exp(x - torch.where(z.isinf(), 0.0, z)))
            # a value that a row does not see has no part in it, whatever it is
            vh = v.permute(1, 0, 2).contiguous()[:, None]
            vz = torch.where(vh.isfinite(), vh, 0.0)
            place = lambda y: y.permute(2, 0, 1, 3).reshape(t, self.nq, -1)
            out[rows] = place(torch.matmul(w, vz))
            if not bool(vh.isfinite().all()):
                odd = torch.matmul((w > 0).double(), (~vh.isfinite()).double()) > 0
                out[rows] = torch.where(place(odd), math.nan, out[rows])
            mean[rows] = place(torch.matmul(w, vz.abs()))
            lse[rows] = place(z).squeeze(-1)
            size[rows] = place(big.masked_fill(~seen, 0.0).amax(-1, keepdim=True)).squeeze(-1)
        return out.flatten(1), lse, mean.flatten(1), size

    def check(self, rounded=False, scale=0.0, missing=None):
        """out and lse against the definition. The bound, per element:
        - the output's own rounding, half a step of it;
        - scores: a dot product of d terms in fp32, each sum within d 2^-24 of its sum of |q k|, and
          the products with scale and log2 e: e = (d + 4) 2^-24 max sum|q k| scale. A weight is
          off by e of itself and so is the sum: 2 e of the weighted mean of |v|;
        - exp2, the sums of n weights and the products' accumulation in fp32, and weights rounded
          with their remainder (2^-17 for bf16): 2^-15 of that mean together; where weights are
          rounded once (``rounded``), a half step for each of them and one for their sum;
        - fp16 weights below 2^-14 of the largest: 2^-25 each in the product, n of them."""
        want, lse, mean, size = self.reference(scale, missing)
        u = half_step(self.dtype)
        e = (self.d + 4) * 2.0 ** -24 * size.repeat_interleave(self.d, 1)
        n = max(max(self.lens), 1)
        vmax = max([float(self.read(self.v_pool, s, self.v_scale).nan_to_num(0, 0, 0).abs().max()) for s, m in
                    enumerate(self.lens) if m] + [1e-9])
        tiny = (n * 2.0 ** -25 * vmax if rounded and self.dtype == torch.float16 else 0.0) + 2.0 ** -24
        tol = u * want.abs() + (2 * e + 2.0 ** -15 + (2 * u if rounded else 0.0)) * mean + tiny
        got = self.out[:self.rows].double()
        assert torch.equal(got.isfinite(), want.isfinite())
        off = torch.where(want.isfinite(), (got - want).abs() - tol, torch.tensor(-1.0, dtype=torch.float64, device="cuda"))
        assert bool((off <= 0).all()), (f"worst {float(off.max())} over its tolerance at "
                                        f"{divmod(int(off.argmax()), off.shape[1])}")
        ltol = (self.d + 4) * 2.0 ** -24 * size + 2.0 ** -18 + 2.0 ** -22 * torch.where(lse.isfinite(), lse.abs(), 0.0)
        gl = self.lse[:self.rows].double()
        assert torch.equal(gl.isfinite(), lse.isfinite())
        fin = lse.isfinite()
        assert bool(((gl - lse).abs()[fin] <= ltol[fin]).all()), float(((gl - lse).abs() - ltol)[fin].max())
        assert bool((gl[~fin & ~lse.isnan()] == -math.inf).all())
        # padding rows as they were
        assert bool((self.out[self.rows:] == 7.0).all()) and bool((self.lse[self.rows:] == 7.0).all())
