// Projections of a batch's rows: the host side of vt_linear and vt_linear_gated (the
// kernels are in linear_thin.hip, linear_mid.hip and linear_tile.hip).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <iterator>
#include <limits>

#include "linear.hpp"

using namespace vt;

namespace {

constexpr int kMaxRows = 1 << 20;
constexpr int64_t kMaxLd = int64_t(1) << 22;  // a tile's rows are addressed by 32-bit offsets

vt_status check_matrix(const void* p, int64_t ld, int64_t cols, int64_t most, const char* name) {
  if (!p) return fail(VT_ERR_ARG, "%s is NULL", name);
  if (!aligned16(p) || ld % 8) return fail(VT_ERR_ALIGN, "%s not 16-byte aligned or its ld not a multiple of 8", name);
  if (ld < cols) return fail(VT_ERR_ARG, "ld of %s (%lld) below %lld", name, static_cast<long long>(ld),
                             static_cast<long long>(cols));
  if (ld > most) return fail(VT_ERR_UNSUPPORTED, "ld of %s (%lld) above %lld", name, static_cast<long long>(ld),
                             static_cast<long long>(most));
  return VT_OK;
}

vt_status check_shape(const vt_linear_io* io) {
  if (!io) return fail(VT_ERR_ARG, "null io");
  if (io->type != VT_T_F16 && io->type != VT_T_BF16)
    return fail(VT_ERR_ARG, "type %d is neither VT_T_F16 nor VT_T_BF16", io->type);
  if (io->act < VT_ACT_NONE || io->act > VT_ACT_GELU_TANH) return fail(VT_ERR_ARG, "unknown activation %d", io->act);
  if (io->n_rows < 1 || io->n_in < 1 || io->n_out < 1)
    return fail(VT_ERR_ARG, "n_rows %d, n_in %d or n_out %d < 1", io->n_rows, io->n_in, io->n_out);
  if (io->n_rows > kMaxRows) return fail(VT_ERR_UNSUPPORTED, "more than %d rows", kMaxRows);
  return VT_OK;
}

// Which kernel takes a product, and in how many slices of K: the one with the shortest modelled time (us)
//   start + step * rounds * steps + tile * rounds + memory * MB + l2 * tile MB
//   + (slices > 1) (join + part * slices' MB + slice * slices):
// rounds of 256 workgroups (one per compute unit; those that fit beside each other overlap in ``step``), steps of 64 k of a
// slice, MB read and written once, MB that the tiles load. The constants are fitted to 4000 products of random sizes (1 to 8192
// rows, 64 to 16384 in, 16 to 32768 out, both kinds, every kernel and slice count): median error 5 to 7%, the
// choice 1.9% slower than the best of all measured on average, 8% in one of ten, 22% in one of a hundred.
// Without the kernel named the products are slower by (mean, worst): thin 0.9%, 1.3 times; 16 x 64 0.9%, 1.2; 32 rows 2.8%,
// 1.4; 64 x 64 2.4%, 1.4; 64 x 128 0.5%, 1.2; 128 x 128 1.5%, 1.5; 256 x 128 0.6%, 1.3; 256 x 256 0.9%, 1.4.
struct Cost {
  double start, step, tile, memory, l2, join, part, slice;
};
constexpr Cost kThinCost = {3.247, 0.0582, 0.202, 0.1123, 0.0, 1.217, 1.557, 0.094};
constexpr Cost kMidCost[] = {{3.087, 0.1322, 0.194, 0.0922, 0.0, 1.122, 0.578, 0.073},
                             {2.991, 0.0981, 0.464, 0.1073, 0.0110, 1.217, 0.381, 0.094},
                             {2.905, 0.1241, 0.999, 0.0640, 0.0182, 1.472, 0.279, 0.139},
                             {1.609, 0.1736, 2.757, 0.0826, 0.0171, 2.223, 0.234, 0.242},
                             {1.827, 0.2763, 3.842, 0.0316, 0.0261, 2.242, 0.163, 0.572}};
constexpr Cost kNarrowCost = {2.544, 0.5143, 5.432, 0.0584, 0.0253, 0, 0, 0};
constexpr Cost kWideCost = {3.319, 0.8613, 9.745, 0.0473, 0.0299, 0, 0, 0};
constexpr int kSlices[] = {1, 2, 3, 4, 6, 8, 12, 16};
constexpr int kThinRows = 16;  // beyond, the thin tile reads the weights more than once
constexpr int kUnits = 256;    // compute units
// Where rows do not start at 128-byte lines, the tiles of 64 rows and more of linear_mid.hip load whole lines: 10 to
// 30% faster with the weights in memory, 6% slower to 5% faster with weights still in the caches, 30% faster from 64
// MB on. The smaller tiles do for weights of this size (4 to 10% faster; below, no gain, and 15% slower in the
// caches).
constexpr int64_t kLinesFrom = int64_t(32) << 20;

enum Kernel { kUseThin, kUseMid, kUseTile };

struct Plan {
  Kernel kernel;
  int mid;     // of kMid
  int m_tiles, n_tiles, wide, splits, steps;
  bool lines;  // kUseMid: whole lines of rows that do not start at them
  double us;
};

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The last compute unit's end where ``many`` tiles of cost c start first and ``more`` of cost d fill up.
double ends_at(int64_t many, double c, int64_t more, double d) {
  const int64_t all = many / kUnits, odd = many % kUnits;  // odd units take one more of the first
  double end = static_cast<double>(all + (odd ? 1 : 0)) * c;
  for (int64_t n = up(more, kUnits);; ++n) {  // a unit takes up to n of the others
    const double t = std::max(end, all * c + n * d);
    const int64_t busy = odd ? static_cast<int64_t>((t - (all + 1) * c) / d) : 0;
    if ((kUnits - odd) * static_cast<int64_t>((t - all * c) / d + 1e-9) + odd * busy >= more) return t;
  }
}

Plan plan_of(int64_t M, int64_t N, int64_t K, bool gated) {
  Plan best{};
  best.us = std::numeric_limits<double>::infinity();
  const int64_t all = up(K, 64);
  const double mb = 2e-6 * (static_cast<double>(N) * K * (gated ? 2 : 1) + static_cast<double>(M) * (K + N));
  auto consider = [&](Kernel kernel, int mid, lin::Shape shape, const Cost& c) {
    const bool thin = kernel == kUseThin;
    const int64_t out = gated && !thin ? shape.features / 2 : shape.features;
    const int64_t wrows = gated && thin ? 2 * shape.features : shape.features;  // weight rows of a tile
    const int64_t mt = up(M, shape.rows), nt = up(N, out), tiles = mt * nt;
    int64_t last = 0;
    for (int want : kSlices) {
      if (want > 1 && (tiles > lin::kMaxTiles || tiles * want > 6 * kUnits || all < 2 * want)) break;
      const int64_t steps = up(all, want), splits = up(all, steps), work = tiles * splits;
      const int64_t part = splits > 1 ? 4 * work * shape.rows * wrows : 0;
      if (splits == last || part > static_cast<int64_t>(lin::kPartBytes)) continue;
      last = splits;
      const double rounds = static_cast<double>(up(work, kUnits));
      const double loads = 128e-6 * static_cast<double>(work) * steps * (shape.rows + wrows);
      const double us = c.start + rounds * (c.step * steps + c.tile) + c.memory * mb + c.l2 * loads +
                        (splits > 1 ? c.join + c.part * 1e-6 * part + c.slice * splits : 0.0);
      if (us < best.us)
        best = {kernel,  mid, static_cast<int>(mt), static_cast<int>(nt), 0, static_cast<int>(splits), static_cast<int>(steps), false, us};
    }
  };
  if (M <= kThinRows) consider(kUseThin, 0, lin::kThin, kThinCost);
  for (size_t i = 0; i < std::size(lin::kMid); ++i)
    if (lin::kMid[i].rows <= 64 || lin::kMid[i].rows < 4 * M)  // the others only multiply more rows that are not there
      consider(kUseMid, static_cast<int>(i), lin::kMid[i], kMidCost[i]);
  if (M > 64) {
    // Wide tiles, as many whole rounds of them as there are or some fewer, and narrow ones for the rest.
    const int64_t mt = up(M, lin::kWide.rows), wide = lin::kWide.features / (gated ? 2 : 1), narrow = wide / 2;
    const int64_t cols = up(N, wide);
    auto tile = [&](int64_t w) {
      const int64_t n = N > w * wide ? up(N - w * wide, narrow) : 0;
      const Cost& c = w ? kWideCost : kNarrowCost;
      const double loads = 128e-6 * static_cast<double>(all * mt) *
                           (w * (lin::kWide.rows + lin::kWide.features) + n * (lin::kNarrow.rows + lin::kNarrow.features));
      const double us = c.start + ends_at(w * mt, kWideCost.step * all + kWideCost.tile, n * mt,
                                          kNarrowCost.step * all + kNarrowCost.tile) +
                        c.memory * mb + c.l2 * loads;
      if (us < best.us)
        best = {kUseTile, 0, static_cast<int>(mt), static_cast<int>(n), static_cast<int>(w), 1, static_cast<int>(all), false, us};
    };
    tile(0);
    tile(cols);
    const int64_t rounds = cols * mt / kUnits;
    for (int64_t r = std::max<int64_t>(1, rounds - 2); r <= rounds; ++r) {
      const int64_t w = std::min(cols, r * kUnits / mt);
      if (w > 0 && w < cols) tile(w);
    }
  }
  return best;
}

Plan plan_of(const vt_linear_io& io, bool gated) {
  Plan p = plan_of(io.n_rows, io.n_out, io.n_in, gated);
  const auto line = [](const void* q) { return reinterpret_cast<uintptr_t>(q) % 128 == 0; };
  p.lines = p.kernel == kUseMid && (io.ld_x | io.ld_w | (gated ? io.ld_up : 0)) % 64 != 0 && line(io.x) && line(io.w) &&
            (!gated || line(io.w_up)) &&
            (lin::kMid[p.mid].rows >= 64 || static_cast<int64_t>(io.n_in) * io.n_out * (gated ? 4 : 2) >= kLinesFrom);
  return p;
}

vt_status project(const vt_linear_io* io, bool gated, void* ws, size_t ws_bytes, void* stream) {
  vt_status st = check_shape(io);
  if (st != VT_OK) return st;
  const int64_t K = io->n_in, N = io->n_out, far = int64_t(1) << 32;
  if ((st = check_matrix(io->x, io->ld_x, K, kMaxLd, "x")) != VT_OK) return st;
  if ((st = check_matrix(io->w, io->ld_w, K, kMaxLd, "w")) != VT_OK) return st;
  if ((st = check_matrix(io->y, io->ld_y, N, far, "y")) != VT_OK) return st;
  if (gated) {
    if ((st = check_matrix(io->w_up, io->ld_up, K, kMaxLd, "w_up")) != VT_OK) return st;
  } else if (io->w_up || io->bias_up) {
    return fail(VT_ERR_ARG, "w_up or bias_up without a gate: vt_linear_gated takes them");
  }
  if (io->residual) {
    if ((st = check_matrix(io->residual, io->ld_res, N, far, "residual")) != VT_OK) return st;
    if (io->residual == io->y && io->ld_res != io->ld_y) return fail(VT_ERR_ARG, "residual equals y at another ld");
  }
  if (!aligned16(io->bias) || !aligned16(io->bias_up)) return fail(VT_ERR_ALIGN, "bias not 16-byte aligned");
  if (io->y == io->x) return fail(VT_ERR_ARG, "y equals x");
  if (!ws || !aligned16(ws)) return fail(ws ? VT_ERR_ALIGN : VT_ERR_WORKSPACE, "workspace missing or misaligned");
  if (ws_bytes < lin::kSyncBytes + lin::kPartBytes)
    return fail(VT_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, lin::kSyncBytes + lin::kPartBytes);

  lin::Args a{};
  a.x = static_cast<const uint16_t*>(io->x);
  a.w[0] = static_cast<const uint16_t*>(io->w);
  a.w[1] = static_cast<const uint16_t*>(io->w_up);
  a.bias[0] = static_cast<const uint16_t*>(io->bias);
  a.bias[1] = static_cast<const uint16_t*>(io->bias_up);
  a.res = static_cast<const uint16_t*>(io->residual);
  a.y = static_cast<uint16_t*>(io->y);
  a.ld_x = io->ld_x;
  a.ld_w[0] = io->ld_w;
  a.ld_w[1] = io->ld_up;
  a.ld_r = io->ld_res;
  a.ld_y = io->ld_y;
  a.M = io->n_rows;
  a.N = io->n_out;
  a.K = io->n_in;
  a.act = io->act;
  const Plan p = plan_of(*io, gated);
  a.m_tiles = p.m_tiles;
  a.n_tiles = p.n_tiles;
  a.wide = p.wide;
  a.splits = p.splits;
  a.steps = p.steps;
  a.arrived = static_cast<uint32_t*>(ws);
  a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + lin::kSyncBytes);
  if (lin::grid_of(p.m_tiles, static_cast<int64_t>(p.n_tiles) * p.splits) + lin::grid_of(p.m_tiles, p.wide) >= (int64_t(1) << 22))
    return fail(VT_ERR_UNSUPPORTED, "%d x %d tiles: fewer rows or features per call", p.m_tiles, p.n_tiles + p.wide);
  const bool bf16 = io->type == VT_T_BF16;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e = p.kernel == kUseThin  ? lin::launch_thin(a, bf16, gated, s)
                       : p.kernel == kUseMid ? lin::launch_mid(a, p.mid, p.lines, bf16, gated, s)
                                             : lin::launch_tile(a, bf16, gated, s);
  return e == hipSuccess ? VT_OK : fail(VT_ERR_HIP, "projection launch: %s", hipGetErrorString(e));
}

}  // namespace

extern "C" vt_status vt_linear_workspace_size(const vt_linear_io* io, size_t* bytes) {
  clear_error();
  if (!bytes) return fail(VT_ERR_ARG, "null bytes");
  const vt_status st = check_shape(io);
  if (st != VT_OK) return st;
  *bytes = lin::kSyncBytes + lin::kPartBytes;
  return VT_OK;
}

extern "C" vt_status vt_linear(const vt_linear_io* io, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  return project(io, false, ws, ws_bytes, stream);
}

extern "C" vt_status vt_linear_gated(const vt_linear_io* io, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  return project(io, true, ws, ws_bytes, stream);
}

// For the tests: what a product is given to. out: the kernel (0 thin, 1 .. 5 of kMid, 6 tile), slices of K, k-steps of
// 64 of a slice, columns of 256-feature tiles, columns of the others, whole-line loads. Nothing is read through io's pointers.
extern "C" int vt_test_linear_plan(const vt_linear_io* io, int32_t gated, int32_t* out) {
  const Plan p = plan_of(*io, gated != 0);
  const int32_t all[] = {p.kernel == kUseThin ? 0 : (p.kernel == kUseMid ? 1 + p.mid : 1 + static_cast<int>(std::size(lin::kMid))),
                         p.splits, p.steps, p.wide, p.n_tiles, p.lines};
  std::copy(std::begin(all), std::end(all), out);
  return static_cast<int>(std::size(all));
}
