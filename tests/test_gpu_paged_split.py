"""Splits of a paged batch at their limits, on the device: the most pieces that a call comes to, chunks
of more sequences than a workgroup has threads, replays of a captured chunk."""
import numpy as np
import pytest
import torch

from paper_2607_07046_amd import voltron as vt
from tests.paged_common import Batch
from tests.paged_split import MOST, MOST_HEADS, PART, SYNC_BYTES, split, tile_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [16, 64, 128])
def test_most_pieces_stay_in_the_workspace(rows):
    """Nearly two pieces for each item aimed at: the last one's partial result is written, nothing
    behind the workspace is."""
    lens, new = MOST[rows]
    b = Batch(lens, None if rows == 16 else new, kv_heads=MOST_HEADS, d=64, page=64)
    n, guard = b.workspace().numel(), 1 << 20
    ws = torch.zeros(n + guard, dtype=torch.uint8, device="cuda")
    ws[n:] = 0xA5
    call = vt.vt_paged_decode_attn if rows == 16 else vt.vt_paged_chunk_attn
    call(b.kv(), b.io(), 0.0, 0, ws.data_ptr(), n, None)
    torch.cuda.synchronize()
    assert bool((ws[n:] == 0xA5).all()) and not ws[:SYNC_BYTES].any()
    pieces, size = split(lens, new, 1, MOST_HEADS, rows)[2], PART[rows](64)
    end = SYNC_BYTES + pieces * size
    assert bool(ws[end - size:end].any()) and not bool(ws[end:n].any())
    b.check(rounded=rows != 16)


@pytest.mark.parametrize("most,mean_rows,f8", [(3, 16, False), (80, 64, True), (200, 128, False)])
@pytest.mark.parametrize("window", [0, 150])
def test_chunks_of_many_sequences(most, mean_rows, f8, window):
    """More sequences than threads, some long, some without new tokens, in each size of tile."""
    rng = np.random.default_rng(most)
    new = rng.integers(0, most, 600)
    lens = new + rng.integers(0, 200, 600)
    lens[[5, 300, 599]] += [9000, 20000, 3000]
    assert tile_rows(new.tolist(), 1) == mean_rows
    b = Batch(lens.tolist(), new.tolist(), kv_heads=2, group=1, d=64, page=32, f8=f8, act="bf16" if f8 else "f16",
              window=window, pad=3)
    b.attend()
    b.check(rounded=True)
    assert int(b.status) == 0


@pytest.mark.parametrize("pad,rows", [(4, 16), (60, 64), (500, 128)])
def test_replays_of_a_chunk_follow_lengths_and_rows(pad, rows):
    """One captured call serves other lengths, rows and tables, idle slots and padding among them; with eager
    work in between. (The host chose the tile when it captured.)"""
    b = Batch([900, 40, 3000, 17], [40, 9, 7, 4], kv_heads=2, group=2, d=128, page=16, pad=pad)
    assert tile_rows([b.n_tok, 0, 0, 0], 2) == rows
    ws = b.workspace()
    b.attend(ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.attend(ws, sync=False)
    full = list(b.lens)
    for lens, new in ((full, [40, 9, 7, 4]), ([900, 0, 2999, 5], [1, 0, 58, 1]), ([0, 0, 0, 0], [0, 0, 0, 0]),
                      ([60, 40, 1000, 17], [60, 0, 0, 0]), (full, [1, 1, 1, 1])):
        b.lens, b.new, b.rows = lens, new, sum(new)
        b.len.copy_(torch.tensor(lens, dtype=torch.int32))
        b.begin.copy_(torch.tensor([0] + new).cumsum(0).to(torch.int32))
        b.q[:b.rows] = torch.randn((b.rows, b.q.shape[1]), device="cuda").to(b.dtype)
        torch.randn(300, 300, device="cuda").sum()
        for _ in range(2):
            b.out.fill_(7.0)
            b.lse.fill_(7.0)
            g.replay()
            torch.cuda.synchronize()
            assert not ws[:8192].any()
            b.check(rounded=True)
