"""What vt_linear and vt_linear_gated give a product to, asked of the library without a GPU, and the lists of sizes
that tests run on one."""
import ctypes

from paper_2607_07046_amd import voltron as vt
from tests.rows_common import stride_of

BASE = 1 << 20  # an address at a line; nothing is read
# rows and weight rows of the kernels' tiles, in the library's order: thin, mid (5), tile (columns of 256 and of 128)
TILES = ((16, 16), (16, 64), (32, 64), (64, 64), (64, 128), (128, 128), (256, 256))
TILE = 6


class Plan:
    """Of a projection whose matrices are laid out as tests.rows_common.Linear does."""

    def __init__(self, M, K, N, gated, pad=8, shift=0):
        up = stride_of(K, 24 if pad == 8 else pad)
        io = vt.vt_linear_io(type=vt.VT_T_F16, n_rows=M, n_in=K, n_out=N, x=BASE + 2 * shift, ld_x=stride_of(K, pad),
                             w=BASE + 2 * shift, ld_w=stride_of(K, pad), w_up=BASE if gated else None,
                             ld_up=up if gated else 0, y=BASE, ld_y=stride_of(N, pad))
        out = (ctypes.c_int32 * 6)()
        assert vt.load_library().vt_test_linear_plan(ctypes.byref(io), int(gated), out) == 6
        self.kernel, self.slices, self.steps, self.wide, self.columns, self.lines = out
        self.gated, self.end = gated, K % 64 != 0

    def form(self):
        """What the kernels' code tells apart: kernel, kind, slices, whole lines, an end of K inside a step, the
        columns' widths, and for tiles whose steps are unrolled by two whether there is one or an odd number."""
        widths = (self.wide > 0, self.columns > 0) if self.kernel == TILE else ()
        turns = (self.steps == 1, self.steps % 2) if 1 < self.kernel < TILE else ()
        return self.kernel, self.gated, self.slices > 1, bool(self.lines), self.end, widths, turns

    def epilogue(self):
        return self.kernel, self.gated, self.slices > 1


# rows, n_in, n_out, row padding: forms that no other list reaches (single rows in slices; whole lines of large weights,
# K a multiple of 64), and tiles of 64 rows and more in slices
FORMS = [(2, 4777, 195, 8), (11, 5324, 65, 8), (16, 9001, 40, 8), (1, 2502, 33, "lines"), (1, 3328, 89, 0),
         (13, 8192, 72, 8), (1, 1216, 14866, 8), (1, 4480, 1884, 8), (3, 384, 22429, 8), (21, 1408, 14094, 8),
         (19, 10432, 1065, 16), (17, 7424, 1452, 16), (18, 5672, 1610, 8), (21, 1408, 6088, 8), (19, 576, 16594, 8),
         (19, 1544, 5892, 64), (121, 9030, 691, 8), (895, 3879, 152, 8), (378, 5154, 1391, 8), (491, 4956, 583, 8),
         (599, 9512, 1096, 8), (643, 10390, 1154, "lines"), (280, 6950, 1703, 8)]
