"""The bounds that the split of a paged batch keeps, on the host: fewer than ``target`` units are cut,
into fewer than 2 * target pieces, which is what the workspace holds."""
import numpy as np
import pytest

from paper_2607_07046_amd import voltron as vt
from tests.paged_split import MOST, MOST_HEADS, PART, SYNC_BYTES, TILES, split, tile_rows


@pytest.mark.parametrize("rows", [16, 64, 128])
def test_pieces_stay_below_their_bound(rows):
    rng = np.random.default_rng(rows)
    _, target, _ = TILES[rows]
    for _ in range(3000):
        s, heads, group = int(np.exp(rng.uniform(0, 6.5))), int(rng.choice([1, 2, 5, 8, 32])), int(rng.choice([1, 4, 8]))
        new = np.exp(rng.uniform(0, rng.uniform(0.1, 7), s)).astype(int)
        lens = new + np.exp(rng.uniform(rng.uniform(0, 8), 11.5, s)).astype(int)
        items, units, pieces, _ = split(lens.tolist(), new.tolist(), group, heads, rows, int(rng.choice([0, 0, 500])))
        assert units < target and pieces < 2 * target


@pytest.mark.parametrize("rows", [16, 64, 128])
def test_most_pieces(rows):
    lens, new = MOST[rows]
    _, target, _ = TILES[rows]
    assert tile_rows(new, 1, rows != 16) == rows
    items, units, pieces, x = split(lens, new, 1, MOST_HEADS, rows)
    assert items > 4 * target and pieces == 2 * units and 2 * target * 0.97 < pieces < 2 * target


@pytest.mark.parametrize("d", [64, 128])
def test_workspace_holds_the_most_pieces(d):
    kv = vt.vt_paged_kv(head_dim=d, n_kv_heads=1, n_seqs=1, type=vt.VT_T_F16)
    io = vt.vt_paged_io(type=vt.VT_T_F16, n_tok=1, n_q_heads=1)
    n = vt.vt_paged_workspace_size(kv, io)
    for rows, (_, target, _) in TILES.items():
        assert 4 * target <= SYNC_BYTES and SYNC_BYTES + 2 * target * PART[rows](d) <= n
