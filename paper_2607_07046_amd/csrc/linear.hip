// Projections of a batch's rows: the host side of vt_linear and vt_linear_gated (the
// kernels are in linear_thin.hip).
#include <hip/hip_runtime.h>

#include <algorithm>

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

struct Plan {
  bool tile;   // 256 x 256 tiles
  int mb, ob;  // else 16-row and 16-feature blocks of a tile
  int m_tiles, n_tiles, splits, steps;
};

Plan plan_of(int64_t M, int64_t N, int64_t K, bool gated) {
  Plan p{};
  if (M > 256) {
    p.tile = true;
    p.m_tiles = static_cast<int>((M + 255) / 256);
    p.n_tiles = static_cast<int>(gated ? (N + 127) / 128 : (N + 255) / 256);
    p.splits = 1;
    return p;
  }
  p.mb = M <= 16 ? 1 : (M <= 32 ? 2 : 4);
  p.ob = 1;
  p.m_tiles = static_cast<int>((M + 16 * p.mb - 1) / (16 * p.mb));
  p.n_tiles = static_cast<int>((N + 16 * p.ob - 1) / (16 * p.ob));
  const int64_t steps = (K + 63) / 64, tiles = static_cast<int64_t>(p.m_tiles) * p.n_tiles;
  int64_t splits = std::max<int64_t>(1, std::min<int64_t>(256 / tiles, steps / 16));
  const int64_t tile_bytes = 4 * 256 * static_cast<int64_t>(p.mb) * p.ob * (gated ? 2 : 1);
  splits = std::min<int64_t>(splits, std::max<int64_t>(1, static_cast<int64_t>(lin::kPartBytes) / (tile_bytes * tiles)));
  if (tiles > lin::kMaxTiles) splits = 1;
  p.steps = static_cast<int>((steps + splits - 1) / splits);
  p.splits = static_cast<int>((steps + p.steps - 1) / p.steps);
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
  const Plan p = plan_of(a.M, a.N, a.K, gated);
  a.m_tiles = p.m_tiles;
  a.n_tiles = p.n_tiles;
  a.splits = p.splits;
  a.steps = p.steps;
  a.arrived = static_cast<uint32_t*>(ws);
  a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + lin::kSyncBytes);
  if ((static_cast<int64_t>(p.n_tiles) * p.splits + 7) / 8 * 8 * p.m_tiles >= (int64_t(1) << 23))  // 2^32 threads
    return fail(VT_ERR_UNSUPPORTED, "%d x %d tiles: fewer rows or features per call", p.m_tiles, p.n_tiles);
  const bool bf16 = io->type == VT_T_BF16;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e = p.tile ? lin::launch_tile(a, bf16, gated, s) : lin::launch_thin(a, bf16, gated, p.mb, p.ob, s);
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
