"""Refusals of the paged-cache entry points, none of which reaches the GPU, and
their workspace size; and the compiler's output around the loads into LDS."""
import math
import os
import re
import subprocess

import pytest

from paper_2607_07046_amd import build
from paper_2607_07046_amd import voltron as vt

P = 0x10000  # an aligned address that nothing reads


def kv(**change):
    f = dict(k=P, v=P, page_stride=2 * 16 * 64, head_stride=16 * 64, slot_stride=64, n_pages=8, page_size=16,
             n_kv_heads=2, head_dim=64, type=vt.VT_T_F16, table=P, ld_table=4, max_pages=4, len=P, n_seqs=3,
             status=P)
    f.update(change)
    return vt.vt_paged_kv(**f)


def io(**change):
    f = dict(type=vt.VT_T_F16, n_tok=3, n_q_heads=4, q=P, ld_q=256, k=P, ld_k=128, v=P, ld_v=128, q_rot=P, ld_qr=256,
             out=P, ld_out=256, lse=P)
    f.update(change)
    return vt.vt_paged_io(**f)


def append(k, i, base=10000.0, flags=0):
    vt.vt_paged_append(k, i, base, flags, None)


def decode(k, i, scale=0.0, window=0, ws=P, ws_bytes=1 << 30):
    vt.vt_paged_decode_attn(k, i, scale, window, ws, ws_bytes, None)


def chunk(k, i, scale=0.0, window=0, ws=P, ws_bytes=1 << 30):
    vt.vt_paged_chunk_attn(k, i, scale, window, ws, ws_bytes, None)


def refused(status, call, *args, **kw):
    with pytest.raises(vt.VoltronError) as e:
        call(*args, **kw)
    assert e.value.status == status and e.value.detail
    return e.value.detail


BOTH = [  # refused by append and attention alike
    (vt.VT_ERR_ARG, dict(k=None), {}),
    (vt.VT_ERR_ARG, dict(v=None), {}),
    (vt.VT_ERR_ARG, dict(table=None), {}),
    (vt.VT_ERR_ARG, dict(len=None), {}),
    (vt.VT_ERR_ALIGN, dict(k=P + 8), {}),
    (vt.VT_ERR_ALIGN, dict(v=P + 2), {}),
    (vt.VT_ERR_ALIGN, dict(table=P + 2), {}),
    (vt.VT_ERR_ALIGN, dict(len=P + 1), {}),
    (vt.VT_ERR_ALIGN, dict(status=P + 2), {}),
    (vt.VT_ERR_ALIGN, dict(type=vt.VT_T_F8E4M3, k_scale=P + 2), {}),
    (vt.VT_ERR_ALIGN, dict(slot_stride=68), {}),
    (vt.VT_ERR_ALIGN, dict(head_stride=16 * 64 + 4), {}),
    (vt.VT_ERR_ALIGN, dict(page_stride=2 * 16 * 64 + 1), {}),
    (vt.VT_ERR_ALIGN, dict(type=vt.VT_T_F8E4M3, slot_stride=72), {}),
    (vt.VT_ERR_ARG, dict(slot_stride=0), {}),
    (vt.VT_ERR_ARG, dict(slot_stride=-64), {}),
    (vt.VT_ERR_ARG, dict(slot_stride=56), {}),
    (vt.VT_ERR_ARG, dict(page_stride=-2048), {}),
    (vt.VT_ERR_ARG, dict(head_stride=0), {}),
    (vt.VT_ERR_UNSUPPORTED, dict(slot_stride=1 << 24), {}),
    (vt.VT_ERR_ARG, dict(page_stride=1 << 41), {}),
    (vt.VT_ERR_UNSUPPORTED, dict(page_stride=1 << 40, n_pages=65), {}),
    (vt.VT_ERR_UNSUPPORTED, dict(n_pages=2 ** 31 - 1, page_stride=1 << 16), {}),
    (vt.VT_ERR_ARG, dict(n_pages=0), {}),
    (vt.VT_ERR_ARG, dict(page_size=0), {}),
    (vt.VT_ERR_ARG, dict(page_size=24), {}),
    (vt.VT_ERR_ARG, dict(page_size=65536), {}),
    (vt.VT_ERR_ARG, dict(page_size=-16), {}),
    (vt.VT_ERR_ARG, dict(max_pages=0), {}),
    (vt.VT_ERR_ARG, dict(ld_table=3), {}),
    (vt.VT_ERR_ARG, dict(n_kv_heads=0), {}),
    (vt.VT_ERR_ARG, dict(n_kv_heads=3), {}),
    (vt.VT_ERR_ARG, dict(n_kv_heads=8), {}),
    (vt.VT_ERR_UNSUPPORTED, dict(head_dim=96), {}),
    (vt.VT_ERR_UNSUPPORTED, dict(head_dim=256), {}),
    (vt.VT_ERR_ARG, dict(type=vt.VT_T_BF16), {}),
    (vt.VT_ERR_ARG, dict(type=7), {}),
    (vt.VT_ERR_ARG, dict(n_seqs=0), {}),
    (vt.VT_ERR_ARG, dict(n_seqs=4), {}),
    (vt.VT_ERR_UNSUPPORTED, dict(n_seqs=70000), dict(q_begin=P)),
    (vt.VT_ERR_ARG, {}, dict(type=vt.VT_T_F8E4M3)),
    (vt.VT_ERR_ARG, {}, dict(type=-1)),
    (vt.VT_ERR_ARG, {}, dict(n_tok=0)),
    (vt.VT_ERR_ARG, {}, dict(n_tok=5)),
    (vt.VT_ERR_UNSUPPORTED, {}, dict(n_tok=(1 << 20) + 1, q_begin=P)),
    (vt.VT_ERR_ARG, {}, dict(n_q_heads=0)),
    (vt.VT_ERR_ARG, {}, dict(n_q_heads=5)),
    (vt.VT_ERR_UNSUPPORTED, {}, dict(n_q_heads=1026)),
    (vt.VT_ERR_ARG, {}, dict(q_rot=None)),
    (vt.VT_ERR_ALIGN, {}, dict(q_rot=P + 4)),
    (vt.VT_ERR_ALIGN, {}, dict(ld_qr=260)),
    (vt.VT_ERR_ARG, {}, dict(ld_qr=248)),
    (vt.VT_ERR_ARG, {}, dict(ld_qr=(1 << 32) + 8)),
]


@pytest.mark.parametrize("status,k,i", BOTH)
def test_refused_by_all(status, k, i):
    refused(status, append, kv(**k), io(**i))
    refused(status, chunk, kv(**k), io(**i))
    if not i.get("q_begin"):
        refused(status, decode, kv(**k), io(**i))


@pytest.mark.parametrize("status,i", [
    (vt.VT_ERR_ARG, dict(k=None)), (vt.VT_ERR_ARG, dict(v=None)), (vt.VT_ERR_ALIGN, dict(k=P + 2)),
    (vt.VT_ERR_ALIGN, dict(v=P + 8)), (vt.VT_ERR_ALIGN, dict(q=P + 2)), (vt.VT_ERR_ALIGN, dict(ld_k=132)),
    (vt.VT_ERR_ARG, dict(ld_v=120)), (vt.VT_ERR_ARG, dict(ld_q=128)), (vt.VT_ERR_ARG, dict(ld_q=264)),
    (vt.VT_ERR_ALIGN, dict(q_begin=P + 2))])
def test_append_refuses(status, i):
    refused(status, append, kv(), io(**i))


@pytest.mark.parametrize("base", [-1.0, math.inf, math.nan])
def test_append_refuses_base(base):
    refused(vt.VT_ERR_ARG, append, kv(), io(), base=base)


def test_append_refuses_flags():
    refused(vt.VT_ERR_ARG, append, kv(), io(), flags=2)


@pytest.mark.parametrize("call", [decode, chunk])
@pytest.mark.parametrize("status,i,a", [
    (vt.VT_ERR_ARG, dict(out=None), {}), (vt.VT_ERR_ALIGN, dict(out=P + 8), {}), (vt.VT_ERR_ARG, dict(ld_out=128), {}),
    (vt.VT_ERR_ALIGN, dict(lse=P + 2), {}), (vt.VT_ERR_ARG, {}, dict(scale=-0.5)), (vt.VT_ERR_ARG, {}, dict(scale=math.inf)),
    (vt.VT_ERR_ARG, {}, dict(scale=math.nan)), (vt.VT_ERR_ARG, {}, dict(window=-1)), (vt.VT_ERR_WORKSPACE, {}, dict(ws=None)),
    (vt.VT_ERR_ALIGN, {}, dict(ws=P + 4)), (vt.VT_ERR_WORKSPACE, {}, dict(ws_bytes=4096))])
def test_attention_refuses(call, status, i, a):
    refused(status, call, kv(), io(**i), **a)


def test_more_tiles_than_a_launch_has():
    refused(vt.VT_ERR_UNSUPPORTED, decode, kv(n_seqs=65536, n_kv_heads=256), io(n_tok=65536, n_q_heads=256, ld_qr=1 << 14,
                                                                              ld_out=1 << 14))


def test_decode_refuses_chunks():
    assert "q_begin" in refused(vt.VT_ERR_ARG, decode, kv(), io(q_begin=P))


def test_workspace_size():
    n = vt.vt_paged_workspace_size(kv(), io())
    assert n > 0
    refused(vt.VT_ERR_WORKSPACE, decode, kv(), io(), ws_bytes=n - 1)
    refused(vt.VT_ERR_UNSUPPORTED, vt.vt_paged_workspace_size, kv(head_dim=32), io())
    lib = vt.load_library()
    assert lib.vt_paged_workspace_size(None, None, None) == vt.VT_ERR_ARG
    assert lib.vt_paged_append(None, None, 0.0, 0, None) == vt.VT_ERR_ARG
    assert lib.vt_paged_decode_attn(None, None, 0.0, 0, None, 0, None) == vt.VT_ERR_ARG
    assert lib.vt_paged_chunk_attn(None, None, 0.0, 0, None, 0, None) == vt.VT_ERR_ARG


def test_direct_loads_keep_their_target(tmp_path):
    """A load into LDS takes its target from m0: in the compiler's output each one directly
    follows the write of m0 and the wait state that it needs, and nothing else uses m0."""
    source, out = os.path.join(build.CSRC, "paged_chunk.hip"), tmp_path / "paged_chunk.s"
    subprocess.run([build.HIPCC, *build.FLAGS, "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                    "--cuda-device-only", "-S", source, "-o", str(out)], check=True, capture_output=True)
    lines = [t for t in (line.split(";")[0].strip() for line in out.read_text().split("\n"))
             if t and not t.startswith(".") and not t.endswith(":")]
    loads = [i for i, t in enumerate(lines) if t.startswith("global_load_lds")]
    assert loads
    for i in loads:
        assert re.match(r"s_mov_b32 m0, s\d+$", lines[i - 2]) and lines[i - 1] == "s_nop 0", lines[i - 2:i + 1]
    assert sum(re.search(r"\bm0\b", t) is not None for t in lines) == len(loads)
