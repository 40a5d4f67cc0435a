"""vt_linear and vt_linear_gated against float64, element by element."""
import math

import pytest
import torch

from paper_2607_07046_amd import voltron as vt
from tests.rows_common import ACTS, MARK, Linear, act64, around, p

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("type", ["f16", "bf16"])


@pytest.fixture(scope="module")
def ws():
    return Linear("f16", 1, 8, 8).workspace()


# rows, n_in, n_out: single rows and numbers, one less and one more than a tile, a step, a matrix instruction
SHAPES = [(1, 1, 1), (1, 7, 5), (1, 8, 16), (1, 64, 17), (1, 65, 16), (1, 512, 1536), (1, 4096, 333), (2, 63, 15),
          (3, 100, 257), (5, 515, 64), (15, 1100, 48), (16, 128, 16), (17, 127, 31), (31, 520, 130), (32, 96, 33),
          (33, 72, 100), (48, 1000, 77), (63, 65, 129), (64, 512, 512), (65, 640, 63), (100, 2048, 260),
          (127, 33, 128), (128, 256, 256), (129, 264, 255), (200, 777, 300), (255, 96, 257), (256, 512, 256),
          (257, 320, 520), (300, 1030, 700), (511, 136, 513), (513, 2050, 264), (1030, 520, 1000), (257, 5, 10), (300, 32, 257),
          (300, 64, 300), (300, 90, 300), (300, 128, 130), (300, 161, 270), (300, 192, 600), (300, 224, 300), (2400, 200, 2500)]


# for each tile of the kernels, whole and in slices of K, with ends of rows, features and K inside it
LARGE = [(20, 898, 75), (2279, 1322, 9), (754, 1846, 30), (1089, 2307, 21), (2885, 130, 140), (2794, 2496, 30),
         (3119, 2210, 17), (262, 37, 1836), (1577, 33, 673), (614, 3771, 769), (2575, 3719, 196), (663, 33, 3138),
         (781, 100, 2565), (337, 4092, 2839), (90, 8193, 4141), (80, 5742, 3326), (1378, 256, 3918), (2171, 230, 2423),
         (2337, 65, 2682), (3785, 33, 4161), (4115, 200, 3319), (3380, 1, 3699), (3869, 359, 3362), (2500, 448, 4008),
         (862, 256, 5974), (1249, 1, 4901), (1420, 1, 8586), (2774, 64, 4459), (3939, 75, 5250), (3887, 1, 3044),
         (2046, 64, 5268)]
# and for those of 32 rows and more: one stage of K, an even and an odd number, an end inside the last
TILES = [(1, 3551, 8980), (2, 4928, 8693), (17, 377, 1), (17, 384, 1), (17, 426, 1), (17, 832, 1), (17, 7168, 5161),
         (17, 7546, 8599), (17, 8606, 8925), (18, 326, 1), (18, 345, 1), (18, 386, 1), (18, 514, 1), (18, 6369, 4467),
         (18, 6592, 8446), (18, 6688, 4367), (19, 384, 1), (19, 393, 1), (19, 448, 1), (19, 6918, 4587),
         (19, 7424, 4757), (25, 321, 1), (33, 129, 8422), (34, 6339, 4540), (35, 130, 5545), (37, 67, 8684),
         (37, 128, 8879), (50, 64, 8341), (66, 139, 6083), (66, 3776, 5273), (66, 4274, 4180), (66, 4516, 8705),
         (66, 5763, 6497), (66, 6627, 2942), (70, 6714, 5486), (71, 170, 8523), (71, 4672, 4116), (72, 3456, 8925),
         (75, 3713, 4254), (113, 1, 8726), (130, 67, 6825), (131, 133, 7003), (138, 128, 6894), (203, 73, 4851),
         (222, 130, 8490), (225, 137, 4116), (228, 72, 8769), (240, 64, 8905), (301, 68, 6606), (322, 1, 6917),
         (322, 151, 5743), (452, 192, 4307), (491, 128, 4111), (518, 64, 8447), (584, 72, 1681), (585, 6592, 579),
         (693, 2624, 1), (711, 3520, 1), (721, 2564, 1), (723, 3648, 1), (747, 3110, 1), (769, 3053, 1),
         (771, 2887, 1), (813, 2564, 1), (828, 2624, 1), (850, 8, 5277), (933, 1, 8843), (988, 64, 8362),
         (1061, 2358, 1), (1132, 8, 918), (1180, 1756, 1), (1238, 1922, 1), (1349, 129, 705), (1368, 1, 6716),
         (1384, 7123, 1), (1887, 64, 8770), (1949, 9, 4141), (1957, 192, 531), (1964, 8, 1052), (2013, 8, 8954),
         (2019, 1, 8758), (2059, 4800, 1), (2101, 6144, 1), (2145, 4480, 1), (2415, 4166, 1), (2710, 1, 1705),
         (2721, 1, 707), (2749, 3264, 1), (2764, 2754, 1), (2803, 3460, 1), (2825, 2721, 1), (2967, 8, 3285),
         (3089, 3617, 1), (3146, 64, 1299), (3225, 2900, 1), (3266, 8, 267), (3295, 64, 291), (3383, 128, 265),
         (3431, 3015, 1), (3469, 1, 1154), (3557, 1, 257), (3781, 64, 2437), (4100, 64, 1), (4107, 1, 1),
         (4113, 64, 1), (4113, 64, 33), (4120, 150, 36), (4124, 8, 559), (4127, 64, 203), (4147, 80, 37),
         (4158, 192, 41), (4170, 69, 34), (4231, 1, 101), (4283, 9, 67), (4314, 8, 1), (4320, 1, 35),
         (4325, 8512, 66), (4327, 1, 1), (4340, 192, 217), (4366, 128, 66), (4433, 8, 106), (4451, 1, 68),
         (4467, 6021, 74), (4472, 192, 82), (4476, 8321, 66), (4489, 8643, 41), (4503, 8, 1), (4504, 128, 33),
         (4542, 8, 39), (4547, 64, 66), (4676, 71, 195), (4771, 67, 68), (4787, 8, 844), (4847, 5379, 77),
         (4872, 64, 387), (4965, 135, 66), (4978, 142, 69), (4983, 73, 69)]
SHAPES += LARGE + TILES


# rows between 128-byte lines, at them, and matrices that start between them
PLACES = pytest.mark.parametrize("pad,shift", [(8, 0), ("lines", 0), ("lines", 40), (16, 8)])


@BOTH
@PLACES
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_shapes(ws, type, M, K, N, pad, shift):
    x = Linear(type, M, K, N, pad=pad, shift=shift, seed=M + K + N)
    x.call(ws)
    x.check()


@BOTH
@PLACES
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_gated_shapes(ws, type, M, K, N, pad, shift):
    x = Linear(type, M, K, N, act="silu", gated=True, pad=pad, shift=shift, seed=M + K + N + 1)
    x.call(ws)
    x.check()


@BOTH
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M", [1, 40, 300])
def test_epilogue(ws, type, act, gated, M):
    x = Linear(type, M, 200, 140, act=act, bias=True, residual=True, gated=gated, seed=M, sigma=3.0)
    x.call(ws)
    x.check()


@BOTH
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,K,N", LARGE)
def test_epilogue_of_all_tiles(ws, type, act, gated, M, K, N):
    x = Linear(type, M, min(K, 4200), N, act=act, bias=True, residual=True, gated=gated, seed=M)
    x.call(ws)
    x.check()


@BOTH
@pytest.mark.parametrize("bias,residual", [(True, False), (False, True)])
@pytest.mark.parametrize("M,K,N", [(1, 72, 133), (70, 72, 133), (260, 72, 133), (1200, 70, 2565), (2400, 136, 4003)])
def test_bias_or_residual(ws, type, bias, residual, M, K, N):
    x = Linear(type, M, K, N, bias=bias, residual=residual, seed=3)
    x.call(ws)
    x.check()


@BOTH
@pytest.mark.parametrize("M,K,N", [(1, 16384, 64), (4, 8192, 100), (64, 8192, 48), (64, 16000, 260), (130, 8200, 70),
                                   (200, 9000, 256), (300, 4096, 500)])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("pad", [8, 32, "lines"])
def test_long_sums(ws, type, M, K, N, gated, pad):
    """Few tiles and a long K: slices of K over several workgroups."""
    x = Linear(type, M, K, N, act="silu" if gated else "none", gated=gated, residual=True, pad=pad, seed=K)
    x.call(ws)
    x.check()
    first = x.y.clone()
    for _ in range(3):
        x.y.fill_(MARK)
        x.call(ws)
        assert torch.equal(x.y, first), "equal calls, other bits"


@BOTH
def test_growing_sums(ws, type):
    x = Linear(type, 70, 8192, 96, positive=True, sigma=0.1)
    x.call(ws)
    x.check()


@BOTH
@pytest.mark.parametrize("M,K,N", [(1, 512, 96), (1, 9000, 40), (50, 512, 96), (260, 512, 300), (90, 8193, 4141),
                                   (1200, 70, 2565), (2400, 136, 4003)])
def test_residual_in_place(ws, type, M, K, N):
    x = Linear(type, M, K, N, act="gelu", residual=True, seed=9)
    before = x.residual.clone()
    x.call(ws, y=p(x.residual), ld_y=x.residual.stride(0))
    x.y.copy_(x.residual)
    x.check(before)
    assert bool(around(x.residual)[:, N:].isnan().all())


@BOTH
@pytest.mark.parametrize("M,N", [(3, 301), (60, 301), (257, 301), (600, 301), (1200, 2565), (2000, 4005)])
@pytest.mark.parametrize("gated", [False, True])
def test_rows_and_features_apart(ws, type, M, N, gated):
    """NaN and infinity in a row or a weight reach its own results and no others."""
    x = Linear(type, M, 330, N, gated=gated, act="silu" if gated else "none", seed=5)
    x.call(ws)
    clean = x.y.clone()
    x.x[1, 329] = math.nan
    x.w[N - 1, 7] = math.inf
    x.call(ws)
    rows = torch.arange(M, device="cuda") != 1
    assert torch.equal(x.y[rows][:, :N - 1], clean[rows][:, :N - 1])
    assert bool(x.y[1].isnan().all())
    assert bool((~x.y[:, N - 1].isfinite()).sum() >= M // 4)  # silu(-inf) * u is NaN, inf stays, and some x are 0
    assert bool((around(x.y)[:, N:] == MARK).all())


def test_overflow_of_f16(ws):
    x = Linear("f16", 20, 64, 40, sigma=60000.0)
    x.x.clamp_(-65504, 65504)
    x.w.mul_(100)
    x.call(ws)
    z, _ = x.sums(x.w, None)
    big = z.abs() > 66000
    assert bool((x.y[big].double() == torch.sign(z[big]) * math.inf).all()) and bool(x.y[z.abs() < 65000].isfinite().all())


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_activations_far_out(ws, act):
    """x w^T = z exactly, over what bf16 holds: the tails go to 0 and z, never to NaN."""
    z = torch.cat([torch.linspace(-30, 30, 601), torch.tensor([-3e38, -1e20, -300.0, 300.0, 1e20, 3e38])])
    x = Linear("bf16", z.numel(), 8, 8, act=act)
    x.x.zero_()
    x.w.zero_()
    x.x[:, 0] = z.cuda().to(torch.bfloat16)
    x.w[:, 0] = 1.0
    x.call(ws)
    exact = x.x[:, 0].double()
    want = torch.where(exact < -200, 0.0, torch.where(exact > 200, exact, 0.0))
    mid = exact.abs() <= 200
    want[mid] = act64(exact[mid], act)
    got = x.y[:, 0].double()
    # half a step, the activation's 2^-16, and for tails the exponent's 2^-23 z^2 / 2
    tol = (2.0 ** -8 + 2.0 ** -16 + 2.0 ** -23 * exact.clamp(-200, 200) ** 2) * want.abs() + 2.0 ** -126
    assert bool(((got - want).abs() <= tol).all())


def test_activations_of_infinities(ws):
    for act, at_inf in (("none", (math.inf, -math.inf)), ("relu", (math.inf, 0.0)), ("silu", (math.inf, math.nan)),
                        ("gelu", (math.inf, math.nan)), ("gelu_tanh", (math.inf, math.nan))):
        x = Linear("f16", 3, 8, 8, act=act, bias=True)
        x.x.zero_()
        x.bias[:] = torch.tensor([math.inf, -math.inf, math.nan, 0, 1, -1, 2, -2])
        x.call(ws)
        got = x.y[0].double().cpu()
        for i in range(2):
            assert math.isnan(got[i]) if math.isnan(at_inf[i]) else got[i] == at_inf[i], (act, i)
        assert got[2] == 0.0 if act == "relu" else math.isnan(got[2])
        assert bool(got[3:].isfinite().all())


# large weights, whose rows are loaded by lines, for each tile between single rows and prompts, whole and in slices of K
COLD = [(1, 1389, 12276), (1, 1538, 11308), (1, 618, 13746), (5, 1476, 5766), (11, 10155, 1669), (1, 6659, 2570), (3, 4632, 1831),
        (1, 11844, 731), (18, 1259, 13486), (31, 1283, 13507), (30, 1151, 7369), (9, 1223, 7833), (17, 9562, 1774), (17, 3523, 4835),
        (29, 8895, 953), (17, 13381, 646), (64, 4715, 16356), (41, 3960, 8319), (34, 4038, 4170), (77, 2951, 9826),
        (81, 3013, 4764), (200, 520, 16652)]


@BOTH
@pytest.mark.parametrize("pad", [0, 8, 24, 48])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,K,N", COLD)
def test_rows_of_large_weights_between_lines(ws, type, M, K, N, gated, pad):
    x = Linear(type, M, K, N, act="silu" if gated else "none", gated=gated, pad=pad, seed=M + K)
    x.call(ws)
    x.check()


@BOTH
@pytest.mark.parametrize("M", [3, 20, 70, 200])
@pytest.mark.parametrize("pad", [0, 8, 16, 24, 32, 40, 48, 56, 4096])
def test_strides(ws, type, M, pad):
    """Every place of a row in a line; rows far apart, as slices of one wide buffer."""
    x = Linear(type, M, 200, 72, pad=pad, residual=True)
    x.call(ws)
    x.check()


@BOTH
def test_widest_stride(ws, type):
    far = Linear(type, 2, 16, 9, pad=(1 << 22) - 16)
    assert far.x.stride(0) == 1 << 22
    far.call(ws)
    far.check()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,K,N", [(1, 70, 90), (40, 136, 90), (129, 200, 260), (2337, 65, 2682)])
def test_widest_strides_of_every_tile(ws, gated, M, K, N):
    """Rows and weights at the widest stride: a tile's offsets end just below 2^31."""
    wide = 1 << 22
    far = Linear("bf16", M, K, N, act="silu" if gated else "none", gated=gated, seed=M)
    for name in ("x", "w", "w_up") if gated else ("x", "w"):
        t = getattr(far, name)
        buf = torch.empty((t.shape[0], wide), dtype=t.dtype, device="cuda")
        buf[:, :K + 8] = math.nan
        buf[:, :K].copy_(t)
        setattr(far, name, buf[:, :K])
    far.call(ws)
    far.check()


@pytest.mark.parametrize("M,N", [(1, 20), (20, 9)])
def test_longest_rows(ws, M, N):
    x = Linear("f16", M, (1 << 22) - 3, N, pad=0, seed=N)
    x.call(ws)
    x.check()


def test_weights_beyond_2_gib(ws):
    x = Linear("bf16", 5, 8192, 8)
    N = 140000
    w = torch.empty((N, 8192), dtype=torch.bfloat16, device="cuda").normal_(0, 0.01)
    y = torch.full((5, N), MARK, dtype=torch.bfloat16, device="cuda")
    x.call(ws, w=p(w), ld_w=8192, n_out=N, y=p(y), ld_y=N)
    for first in (0, N // 2, N - 300):
        part = Linear("bf16", 5, 8192, 300)
        part.x.copy_(x.x)
        part.w = w[first:first + 300]
        part.y.copy_(y[:, first:first + 300])
        part.check()


def test_rows_beyond_2_gib(ws):
    """Outputs, inputs and the residual pass 32-bit offsets."""
    M, K, N = 70000, 64, 24
    g = torch.Generator(device="cuda").manual_seed(1)
    wide = torch.empty((M, 16384), dtype=torch.float16, device="cuda")
    wide[:, :64].normal_(generator=g)
    wide[:, 8192:8192 + N].normal_(generator=g)
    x = Linear("f16", 300, K, N, residual=True)
    x.call(ws, n_rows=M, x=p(wide), ld_x=16384, residual=wide[:, 8192:].data_ptr(), ld_res=16384,
           y=wide[:, 12288:].data_ptr(), ld_y=16384)
    for first in (0, 40000, M - 300):
        rows = slice(first, first + 300)
        x.x.copy_(wide[rows, :K])
        x.residual.copy_(wide[rows, 8192:8192 + N])
        x.y.copy_(wide[rows, 12288:12288 + N])
        x.check()


def test_two_streams():
    """Calls at once, each with its workspace."""
    a, b = Linear("f16", 8, 8192, 64, seed=1), Linear("bf16", 200, 4096, 300, gated=True, act="silu", seed=2)
    wa, wb = a.workspace(), b.workspace()
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        for x, w, s in ((a, wa, streams[0]), (b, wb, streams[1])):
            with torch.cuda.stream(s):
                x.call(w, sync=False)
    torch.cuda.synchronize()
    a.check()
    b.check()


def test_graph_replays(ws):
    """One captured step of several projections, replayed on new inputs."""
    xs = [Linear("f16", 1, 4096, 64, seed=1), Linear("f16", 70, 4096, 48, residual=True, seed=2),
          Linear("f16", 300, 512, 600, gated=True, act="silu", seed=3), Linear("f16", 90, 8193, 4141, seed=4),
          Linear("f16", 2171, 230, 2423, seed=5), Linear("f16", 2500, 448, 4008, bias=True, seed=6)]
    for x in xs:
        x.call(ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x in xs:
            x.call(ws, sync=False)
    for i in range(4):
        for x in xs:
            x.x.copy_(torch.randn(x.x.shape, device="cuda"))
            x.y.fill_(MARK)
        graph.replay()
        torch.cuda.synchronize()
        for x in xs:
            x.check()
        assert not ws[:16384].any()


def test_alternating_shapes_share_a_workspace(ws):
    xs = [Linear("bf16", m, k, n, seed=i, gated=i % 2 == 1) for i, (m, k, n) in
          enumerate([(1, 8192, 32), (64, 8192, 70), (200, 4096, 128), (2, 300, 4000), (260, 8192, 100)])]
    for x in xs + xs[::-1]:
        x.y.fill_(MARK)
        x.call(ws, sync=False)
    torch.cuda.synchronize()
    for x in xs:
        x.check()
