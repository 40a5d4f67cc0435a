// Shared by the kernels of vt_linear and vt_linear_gated: arguments and epilogue.
#pragma once

#include <atomic>
#include <type_traits>

#include "device.hpp"
#include "internal.hpp"
#include "paged.hpp"

namespace vt {
namespace lin {

using pg::BFloat;
using pg::Half;

constexpr float kLog2e = 1.4426950408889634f;

// y = act(x W^T + bias) + residual, gated: act(x W^T + bias) * (x W_up^T + bias_up) + residual.
struct Args {
  const uint16_t* x;
  const uint16_t* w[2];
  const uint16_t* bias[2];
  const uint16_t* res;
  uint16_t* y;
  int64_t ld_x, ld_w[2], ld_r, ld_y;
  int32_t M, N, K, act;
  int32_t m_tiles, n_tiles;
  int32_t wide;           // tile kernel: columns of 256 weight rows before the n_tiles of 128
  int32_t splits, steps;  // slices of K, and the k-steps of each
  float* part;            // the slices' sums
  uint32_t* arrived;      // per tile: slices done, zero between calls
};

// The workspace: arrival counters, then the slices' sums.
constexpr int kMaxTiles = 4096;  // of a split product
constexpr size_t kSyncBytes = kMaxTiles * sizeof(uint32_t);
constexpr size_t kPartBytes = size_t(64) << 20;

// This workgroup's tile: row of tiles and column (of the weights, and of its slices). Workgroups go round the XCDs one by
// one; each XCD gets one run of the tiles in the order of blocks of 2048 rows, column by column in them, so
// that the tiles running there at once share rows and weights in its L2. False: a workgroup too many.
constexpr int kXcds = 8;
__host__ __device__ inline int64_t grid_of(int64_t m_tiles, int64_t cols) { return (m_tiles * cols + kXcds - 1) / kXcds * kXcds; }
__device__ __forceinline__ bool my_tile(int id, int m_tiles, int cols, int tile_rows, int& m, int& col) {
  const int all = m_tiles * cols, run = (all + kXcds - 1) / kXcds;
  const int at = id % kXcds * run + id / kXcds;
  if (at >= all) return false;
  const int high = min(m_tiles, max(1, 2048 / tile_rows)), blk = at / (high * cols);
  const int rows = min(high, m_tiles - blk * high), in = at - blk * high * cols;
  col = in / rows;
  m = blk * high + in % rows;
  return true;
}

// Where an XCD starts in the n (>= 1) k-tiles of its slice; it goes on to the end and then from the beginning. Row
// strides are multiples of large powers of two as a rule, and the same columns of all rows lie in few of memory's
// channels: were all workgroups at the same columns, they would wait for those. One row of 8192 through 8192 features
// 35 -> 28 us, 64 through the gate and up projections of 7168 65 -> 50 (weights in memory); products of more than 512
// rows up to 5%.
__device__ __forceinline__ int first_of(int id, int n) { return id % kXcds * n / kXcds; }

// The activation functions in fp32. Half a step of the results' type is 2^-12 at least; exp2 and
// the reciprocal are the hardware's, a few 2^-24 off.
//
// 1 / (1 + exp(-z)), from numbers 2^-12 times as large: the hardware's reciprocal of one above 2^126 is 0, and z times
// the sigmoid is a number that bf16 holds down to z = -92. (The exponent of a z near 0 rounds 2^-21 off.)
__device__ __forceinline__ float sigmoid(float z) {
  constexpr float small = 0x1p-12f;
  return small * __builtin_amdgcn_rcpf(small + __builtin_amdgcn_exp2f(fmaf(-kLog2e, z, -12.f)));
}

// z Phi(z) with Phi(z) = erfc(-z / sqrt 2) / 2. erfc(x) = exp(-x^2) t Q(t), t = 1 / (1 + 0.54 x): the
// coefficients of Q are a fit to the scaled function over x >= 0 of least largest relative error (3.1e-6), so
// the left tail keeps its relative precision, which 1 + erf loses.
__device__ __forceinline__ float gelu(float z) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.54f * 0.70710678f, fabsf(z), 1.f));
  float q = 0.097615257f;
  q = fmaf(q, t, -0.31480265f);
  q = fmaf(q, t, 0.21606381f);
  q = fmaf(q, t, 0.12524414f);
  q = fmaf(q, t, 0.26698509f);
  q = fmaf(q, t, 0.30422452f);
  q = fmaf(q, t, 0.30467153f);
  const float h = 0.5f * t * q * __builtin_amdgcn_exp2f(-0.5f * kLog2e * z * z);
  return z * (z > 0.f ? 1.f - h : h);
}

// W values through the activation (uniform).
template <int W>
__device__ __forceinline__ void activate(float (&z)[W], int act) {
  switch (act) {
    case VT_ACT_RELU:
#pragma unroll
      for (int e = 0; e < W; ++e) z[e] = z[e] > 0.f ? z[e] : 0.f;
      break;
    case VT_ACT_SILU:
#pragma unroll
      for (int e = 0; e < W; ++e) z[e] *= sigmoid(z[e]);
      break;
    case VT_ACT_GELU:
#pragma unroll
      for (int e = 0; e < W; ++e) z[e] = gelu(z[e]);
      break;
    case VT_ACT_GELU_TANH:  // (1 + tanh u) / 2 = sigmoid(2 u)
#pragma unroll
      for (int e = 0; e < W; ++e)
        z[e] *= sigmoid(1.5957691216057308f * z[e] * fmaf(0.044715f * z[e], z[e], 1.f));
      break;
    default: break;
  }
}

// f(integral_constant 0), .., f(integral_constant N - 1)
template <int N, int I = 0, class F>
__device__ __forceinline__ void each(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    each<N, I + 1>(f);
  }
}

template <class T>
__device__ __forceinline__ float one(const uint16_t* p) {
  float a, b;
  T::unpack2(*p, a, b);
  return a;
}

// The first numbers of a group of W (4 or 8), fewer than W and as many in every lane: in pieces of 4, 2 and 1, whose
// places are the same for all lanes.
template <int W, class V>
__device__ __forceinline__ void store_first(uint16_t* y, V v, int count) {
  int at = 0;
  uint32_t lo = v[0], hi = v[1];
  if (W == 8 && (count & 4)) {
    *reinterpret_cast<pg::u32x2*>(y) = pg::u32x2{lo, hi};
    at = 4;
    lo = v[W / 2 - 2];
    hi = v[W / 2 - 1];
  }
  if (count & 2) {
    *reinterpret_cast<uint32_t*>(y + at) = lo;
    at += 2;
    lo = hi;
  }
  if (count & 1) y[at] = static_cast<uint16_t>(lo);
}

// W (4 or 8) consecutive features n.. of row m, from the product's sums to y. Whole groups by wide accesses; of the
// group that reaches past N the bias is read by single numbers, the residual as it is (rows may be read up to a
// multiple of 8) and nothing past N is written. (Both paths end in the same vector: stores to z and u on either side
// of the branch were merged into one at a variable index, in scratch memory.)
template <class T, bool GATED, int W>
__device__ __forceinline__ void finish(const Args& a, int m, int n, float (&z)[W], float (&u)[W]) {
  typedef unsigned int vec __attribute__((ext_vector_type(W / 2)));
  const bool whole = n + W <= a.N;
  auto add = [&](const uint16_t* p, bool all, float (&to)[W]) {
    vec v;
    if (all) {
      v = *reinterpret_cast<const vec*>(p);
    } else {
      each<W / 2>([&](auto E) {
        constexpr int e = decltype(E)::value;
        v[e] = (n + 2 * e < a.N ? p[2 * e] : 0u) | (n + 2 * e + 1 < a.N ? static_cast<uint32_t>(p[2 * e + 1]) << 16 : 0u);
      });
    }
    each<W / 2>([&](auto E) {
      constexpr int e = decltype(E)::value;
      float lo, hi;
      T::unpack2(v[e], lo, hi);
      to[2 * e] += lo;
      to[2 * e + 1] += hi;
    });
  };
  if (a.bias[0]) add(a.bias[0] + n, whole, z);
  activate(z, a.act);
  if (GATED) {
    if (a.bias[1]) add(a.bias[1] + n, whole, u);
#pragma unroll
    for (int e = 0; e < W; ++e) z[e] *= u[e];
  }
  if (a.res) add(a.res + m * a.ld_r + n, true, z);
  uint16_t* y = a.y + m * a.ld_y + n;
  vec v;
  each<W / 2>([&](auto E) {
    constexpr int e = decltype(E)::value;
    v[e] = T::pack2(z[2 * e], z[2 * e + 1]);
  });
  if (whole) {
    *reinterpret_cast<vec*>(y) = v;
  } else {
    store_first<W>(y, v, a.N % W);
  }
}

// The 8 numbers of w with those at index >= v set to zero.
__device__ __forceinline__ u32x4 keep_first(u32x4 w, int v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = v >= 2 * i + 2 ? w[i] : (v == 2 * i + 1 ? (w[i] & 0xFFFFu) : 0u);
  return w;
}

// 16 bytes at a lane's offset plus a uniform one. Only the lane's is range-checked: it is kOOB where
// nothing is to be read.
__device__ __forceinline__ u32x4 load_at(rsrc_t r, uint32_t lane_off, uint32_t off) {
  return __builtin_amdgcn_raw_buffer_load_b128(r, lane_off, off, 0);
}

// The kernels' tiles: rows, and features (of a gated product half as many, but on the thin tile).
struct Shape {
  int rows, features;
};
constexpr Shape kThin = {16, 16};
constexpr Shape kMid[] = {{16, 64}, {32, 64}, {64, 64}, {64, 128}, {128, 128}};
constexpr Shape kNarrow = {256, 128}, kWide = {256, 256};

// Dynamic LDS above 64 KiB has to be asked for, kernel by kernel, once per device.
class LdsOnce {
  std::atomic<bool> done_[64] = {};

 public:
  template <class F>
  hipError_t operator()(F&& all) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess || (dev < 64 && done_[dev].load(std::memory_order_acquire))) return e;
    all([&](const void* kernel, int bytes) {
      const hipError_t r = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
      if (r != hipSuccess) e = r;
    });
    if (e == hipSuccess && dev < 64) done_[dev].store(true, std::memory_order_release);
    return e;
  }
};

hipError_t launch_thin(const Args& a, bool bf16, bool gated, hipStream_t s);
// ``which``: of kMid. ``shift``: whole lines of rows that do not start at them (of matrices that do).
hipError_t launch_mid(const Args& a, int which, bool shift, bool bf16, bool gated, hipStream_t s);
hipError_t launch_tile(const Args& a, bool bf16, bool gated, hipStream_t s);

}  // namespace lin
}  // namespace vt
