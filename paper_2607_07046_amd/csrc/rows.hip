// Row-wise operators of a batch: norms of the rows.
#include <hip/hip_runtime.h>

#include <cmath>

#include "internal.hpp"
#include "linear.hpp"
#include "paged_append.hpp"

namespace vt {
namespace rows {

using pg::BFloat;
using pg::Half;

struct NormArgs {
  const uint16_t *x, *partial, *peer, *gain;
  uint16_t *h, *y;
  int64_t ld_x, ld_partial, ld_peer, ld_h, ld_y;
  int32_t M, N;
  float eps;
};

template <class T>
__device__ __forceinline__ void unpack(const u32x4 w, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) T::unpack2(w[e], v[2 * e], v[2 * e + 1]);
}

template <class T>
__device__ __forceinline__ u32x4 packed(const float (&v)[8]) {
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = T::pack2(v[2 * e], v[2 * e + 1]);
  return w;
}

// Sum over the workgroup's waves that share a row (TR threads of it), in a fixed order.
template <int TR, int NT, class S>
__device__ __forceinline__ S row_sum(S v, S* red) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  if (TR == kWave) return v;
  constexpr int W = TR / kWave;
  const int wave = threadIdx.x / kWave;
  if (threadIdx.x % kWave == 0) red[wave] = v;
  __syncthreads();
  S s = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) s += red[wave / W * W + i];
  __syncthreads();
  return s;
}

// h = x + partial + peer, y = h / sqrt(mean(h^2) + eps) * gain. TR threads take a row and hold it in registers, V
// groups of 8 numbers each, so every number is read and written once: memory bounds it. Measured: 8192 rows of 5120
// with a partial sum, bf16, 67 to 69 us, 4.9 to 5.0 TB/s; 64 rows of 8192 with a partial and the peers' sum 4.3 us in
// a captured graph.
constexpr int threads(int tr) { return tr <= 128 ? 256 : tr; }

template <class T, int TR, int V>
__global__ void __launch_bounds__(threads(TR)) norm_kernel(NormArgs a) {
  constexpr int NT = threads(TR), RPB = NT / TR;
  __shared__ double red[NT / kWave];
  const int t = threadIdx.x % TR;
  const int row = blockIdx.x * RPB + threadIdx.x / TR;
  const bool there = row < a.M;
  const int64_t r = there ? row : a.M - 1;  // (whole workgroups meet at the barriers)
  u32x4 wx[V], wp[V], wq[V], wg[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (i * TR + t) * 8;
    if (c >= a.N) continue;
    wx[i] = load16(a.x + r * a.ld_x + c);
    if (a.partial) wp[i] = load16(a.partial + r * a.ld_partial + c);
    if (a.peer) wq[i] = load16(a.peer + r * a.ld_peer + c);
    if (c + 8 <= a.N) {
      wg[i] = load16(a.gain + c);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        wg[i][e] = (c + 2 * e < a.N ? a.gain[c + 2 * e] : 0u) |
                   (c + 2 * e + 1 < a.N ? static_cast<uint32_t>(a.gain[c + 2 * e + 1]) << 16 : 0u);
    }
  }
  float h[V][8];
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (i * TR + t) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[i][e] = 0.f;
    if (c >= a.N) continue;
    unpack<T>(wx[i], h[i]);
    if (a.partial) {
      float v[8];
      unpack<T>(wp[i], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] += v[e];
    }
    if (a.peer) {
      float v[8];
      unpack<T>(wq[i], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] += v[e];
    }
    const bool whole = c + 8 <= a.N;
    u32x4 w = packed<T>(h[i]);
    unpack<T>(w, h[i]);  // the norm is of the numbers as written
    if (!whole) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e >= a.N) h[i][e] = 0.f;  // padding, whatever it holds
    }
    if (a.h && there) {
      uint16_t* p = a.h + r * a.ld_h + c;
      if (whole) *reinterpret_cast<u32x4*>(p) = w;
      else lin::store_first<8>(p, w, a.N % 8);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(h[i][e], h[i][e], ss);
  }
  ss = row_sum<TR, NT>(ss, reinterpret_cast<float*>(red));
  const float mean = ss / static_cast<float>(a.N) + a.eps;
  double wide = 0.0;
  // Squares of bf16 numbers leave the range of fp32 at 2^64 and 2^-63: such a row's statistics, and
  // its products, are taken in double.
  const bool out = !(mean > 1e-30f && mean < 1e37f);
  if (TR == kWave ? out : __syncthreads_or(out)) {
    double s2 = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) s2 += static_cast<double>(h[i][e]) * h[i][e];
    s2 = row_sum<TR, NT>(s2, red);
    wide = 1.0 / sqrt(s2 / a.N + a.eps);
  }
  if (!there) return;
  const float inv = 1.0f / sqrtf(mean);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (i * TR + t) * 8;
    if (c >= a.N) continue;
    float g[8];
    unpack<T>(wg[i], g);
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = out ? static_cast<float>(h[i][e] * wide * g[e]) : h[i][e] * inv * g[e];
    const u32x4 w = packed<T>(y);
    uint16_t* p = a.y + r * a.ld_y + c;
    if (c + 8 <= a.N) *reinterpret_cast<u32x4*>(p) = w;
    else lin::store_first<8>(p, w, a.N % 8);
  }
}

}  // namespace rows
}  // namespace vt

using namespace vt;

namespace {

constexpr int kMaxRows = 1 << 20, kMaxHidden = 16384;

// The fewest threads, in whole waves, that hold a row: idle ones cost (8192 rows of 2049 numbers on 512 threads 39
// us, on 320 35; of 5120 on 1024 71, on 640 69).
template <class T, int V, int TR, int... MORE>
void launch_norm(const rows::NormArgs& a, hipStream_t s) {
  if constexpr (sizeof...(MORE) > 0)
    if (a.N > TR * V * 8) return launch_norm<T, V, MORE...>(a, s);
  constexpr int NT = rows::threads(TR), RPB = NT / TR;
  hipLaunchKernelGGL((rows::norm_kernel<T, TR, V>), dim3((a.M + RPB - 1) / RPB), dim3(NT), 0, s, a);
}

template <class T>
void launch_norm(const rows::NormArgs& a, hipStream_t s) {
  if (a.N <= 8192) return launch_norm<T, 1, 64, 128, 192, 256, 320, 384, 448, 512, 640, 768, 896, 1024>(a, s);
  launch_norm<T, 2, 640, 768, 896, 1024>(a, s);
}

}  // namespace

extern "C" vt_status vt_norm_rows(const vt_norm_io* io, void* stream) {
  clear_error();
  if (!io) return fail(VT_ERR_ARG, "null io");
  if (io->type != VT_T_F16 && io->type != VT_T_BF16)
    return fail(VT_ERR_ARG, "type %d is neither VT_T_F16 nor VT_T_BF16", io->type);
  if (io->n_rows < 1 || io->hidden < 1) return fail(VT_ERR_ARG, "n_rows %d or hidden %d < 1", io->n_rows, io->hidden);
  if (io->n_rows > kMaxRows || io->hidden > kMaxHidden)
    return fail(VT_ERR_UNSUPPORTED, "more than %d rows or hidden above %d", kMaxRows, kMaxHidden);
  if (!(io->eps >= 0.f) || !std::isfinite(io->eps)) return fail(VT_ERR_ARG, "eps must be finite and >= 0");
  const struct {
    const void* p;
    int64_t ld;
    bool needed;
    const char* name;
  } ms[] = {{io->x, io->ld_x, true, "x"},
            {io->partial, io->ld_partial, false, "partial"},
            {io->peer, io->ld_peer, false, "peer"},
            {io->h, io->ld_h, false, "h"},
            {io->y, io->ld_y, true, "y"}};
  for (const auto& m : ms) {
    if (!m.p) {
      if (m.needed) return fail(VT_ERR_ARG, "%s is NULL", m.name);
      continue;
    }
    const vt_status st = pg::check_rows(m.p, m.ld, io->hidden, m.name);
    if (st != VT_OK) return st;
  }
  if (!io->gain) return fail(VT_ERR_ARG, "gain is NULL");
  if (!aligned16(io->gain)) return fail(VT_ERR_ALIGN, "gain not 16-byte aligned");
  // an output may take an input's place, row by row
  for (int o = 3; o < 5; ++o)
    for (int i = 0; i < 4; ++i)
      if (i != o && ms[o].p && ms[o].p == ms[i].p && (i == 3 || ms[o].ld != ms[i].ld))
        return fail(VT_ERR_ARG, "%s equals %s%s", ms[o].name, ms[i].name, i == 3 ? "" : " at another ld");
  rows::NormArgs a{};
  a.x = static_cast<const uint16_t*>(io->x);
  a.partial = static_cast<const uint16_t*>(io->partial);
  a.peer = static_cast<const uint16_t*>(io->peer);
  a.gain = static_cast<const uint16_t*>(io->gain);
  a.h = static_cast<uint16_t*>(io->h);
  a.y = static_cast<uint16_t*>(io->y);
  a.ld_x = io->ld_x;
  a.ld_partial = io->ld_partial;
  a.ld_peer = io->ld_peer;
  a.ld_h = io->ld_h;
  a.ld_y = io->ld_y;
  a.M = io->n_rows;
  a.N = io->hidden;
  a.eps = io->eps;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (io->type == VT_T_F16) launch_norm<pg::Half>(a, s);
  else launch_norm<pg::BFloat>(a, s);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? VT_OK : fail(VT_ERR_HIP, "norm launch: %s", hipGetErrorString(e));
}
