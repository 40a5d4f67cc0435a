// Products of few rows with a large weight matrix: vt_linear and vt_linear_gated while their time is that
// of reading the weights.
//
// A workgroup takes a tile of 16 rows and 16 features; its waves share out the k-steps of
// its slice of K (64 k each, in turn, so that together they read whole pieces of a weight row), and each
// multiplies weights and activations straight from memory: both operands of a 16 x 16 x 32 matrix
// instruction are 16 bytes per lane of consecutive k, and nothing is used by two waves, so LDS would
// only stand in between. The waves' sums meet in LDS, in wave order; slices of K over several workgroups meet
// in the workspace, added in slice order by whichever arrives last, which waits for nobody.
//
// What bounds it: reading the weights, and for small ones the chain launch -> loads -> join. Measured in captured
// graphs: one row of 512 through 1536 features 3.7 to 4.3 us; one row of 4096 through the gate and up projections of
// 3302 features (54 MB) 11.7 to 12.4 us, 4.4 to 4.6 TB/s, where a copy of 4 GiB reaches 4.7.
#include "linear.hpp"

namespace vt {
namespace lin {

constexpr int NW = 8, HW = NW / 2;  // waves
constexpr int HS = 2, KS = 32 * HS;  // matrix instructions' k-steps, and k, of a step
constexpr int DEPTH = 2;             // steps in flight

template <class T, bool GATED>
__global__ void __launch_bounds__(NW* kWave) thin_kernel(Args a) {
  constexpr int FB = GATED ? 2 : 1, TN = kThin.features, TM = kThin.rows, LD = 16 * FB + 4;  // FB: weight matrices
  static_assert(TN == 16 && TM == 16, "one fragment of each");
  __shared__ __attribute__((aligned(16))) float red[HW * TM * LD];
  __shared__ uint32_t ticket;
  int m_tile, unit;
  if (!my_tile(blockIdx.x, a.m_tiles, a.n_tiles * a.splits, TM, m_tile, unit)) return;
  const int n_tile = unit % a.n_tiles, split = unit / a.n_tiles;
  const int m0 = m_tile * TM, n0 = n_tile * TN;
  const int t = threadIdx.x, lane = t % kWave, wave = __builtin_amdgcn_readfirstlane(t / kWave);
  const int q = lane / 16, r = lane % 16;

  const int rows_w = min(TN, a.N - n0), rows_x = min(TM, a.M - m0);
  const rsrc_t rx = make_rsrc(a.x + m0 * a.ld_x, static_cast<uint32_t>(rows_x * a.ld_x * 2));
  auto weights = [&](int i) { return make_rsrc(a.w[i] + n0 * a.ld_w[i], static_cast<uint32_t>(rows_w * a.ld_w[i] * 2)); };
  const rsrc_t rw0 = weights(0), rw1 = GATED ? weights(1) : rw0;
  uint32_t ow[FB];
#pragma unroll
  for (int f = 0; f < FB; ++f) ow[f] = r < rows_w ? static_cast<uint32_t>(r * a.ld_w[f] * 2) + q * 16 : kOOB;
  const uint32_t ox = r < rows_x ? static_cast<uint32_t>(r * a.ld_x * 2) + q * 16 : kOOB;

  f32x4 acc[FB];
#pragma unroll
  for (int f = 0; f < FB; ++f) acc[f] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 wf[DEPTH][FB][HS], xf[DEPTH][HS];
  const int full = a.K / KS, s0 = split * a.steps;
  const int s1 = min(s0 + a.steps, full), count = max(s1 - s0, 0), first = count ? first_of(blockIdx.x, count) : 0;
  // step i of this wave; past the slice's end nothing is read and zeros are multiplied
  auto load = [&](int i, u32x4 (&w)[FB][HS], u32x4 (&x)[HS]) {
    const int j = wave + i * NW, s = j + first < count ? j + first : j + first - count;
    const uint32_t gone = j < count ? 0u : kOOB, at = j < count ? static_cast<uint32_t>((s0 + s) * KS * 2) : 0u;
#pragma unroll
    for (int h = 0; h < HS; ++h) {
#pragma unroll
      for (int f = 0; f < FB; ++f) w[f][h] = load_at(f ? rw1 : rw0, ow[f] | gone, at + h * 64);
      x[h] = load_at(rx, ox | gone, at + h * 64);
    }
  };
  auto multiply = [&](const u32x4 (&w)[FB][HS], const u32x4 (&x)[HS]) {
#pragma unroll
    for (int h = 0; h < HS; ++h)
#pragma unroll
      for (int f = 0; f < FB; ++f) acc[f] = T::mfma16(w[f][h], x[h], acc[f]);
  };
  const int mine = s0 + wave < s1 ? (s1 - s0 - wave + NW - 1) / NW : 0;
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) load(d, wf[d], xf[d]);
  for (int i = 0; i < mine; i += DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      multiply(wf[d], xf[d]);
      load(i + DEPTH + d, wf[d], xf[d]);
    }
  }
  // the step that reaches past K: the numbers behind it are padding and may be anything
  if (a.K % KS != 0 && full >= s0 && full < s0 + a.steps && wave == (full - s0) % NW) {
#pragma unroll
    for (int h = 0; h < HS; ++h) {
      const int k = full * KS + h * 32 + q * 8;
      const uint32_t gone = k < a.K ? 0u : kOOB;
#pragma unroll
      for (int f = 0; f < FB; ++f)
        wf[0][f][h] = keep_first(load_at(f ? rw1 : rw0, ow[f] | gone, full * KS * 2 + h * 64), a.K - k);
      xf[0][h] = keep_first(load_at(rx, ox | gone, full * KS * 2 + h * 64), a.K - k);
    }
    multiply(wf[0], xf[0]);
  }

  // accumulator i of f: feature 4 q + i, row r
  auto place = [&](int w, int f) { return reinterpret_cast<f32x4*>(red + (w * TM + r) * LD + 16 * f + 4 * q); };
  if (wave >= HW) {
#pragma unroll
    for (int f = 0; f < FB; ++f) *place(wave - HW, f) = acc[f];
  }
  __syncthreads();
  if (wave < HW) {
#pragma unroll
    for (int f = 0; f < FB; ++f) {
      f32x4* p = place(wave, f);
      *p = acc[f] + *p;
    }
  }
  __syncthreads();
  auto sum4 = [&](int m, int n) __attribute__((always_inline)) {
    f32x4 s = *reinterpret_cast<const f32x4*>(red + m * LD + n);
#pragma unroll
    for (int w = 1; w < HW; ++w) s += *reinterpret_cast<const f32x4*>(red + (w * TM + m) * LD + n);
    return s;
  };
  auto out4 = [&](int m, int n, f32x4 z4, f32x4 u4) __attribute__((always_inline)) {
    float z[4] = {z4.x, z4.y, z4.z, z4.w}, u[4] = {u4.x, u4.y, u4.z, u4.w};
    finish<T, GATED, 4>(a, m0 + m, n0 + n, z, u);
  };
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  constexpr int UNITS = TM * TN / 4;
  if (a.splits == 1) {
    for (int i = t; i < UNITS; i += NW * kWave) {
      const int m = i / (TN / 4), n = i % (TN / 4) * 4;
      if (m >= rows_x || n >= rows_w) continue;
      out4(m, n, sum4(m, n), GATED ? sum4(m, TN + n) : zero);
    }
    return;
  }
  // slices: store this one's sums, then count it; whoever counts last adds all of them
  constexpr int TILE = TM * 16 * FB;
  const int tiles = a.m_tiles * a.n_tiles, tile = m_tile * a.n_tiles + n_tile;
  auto slice = [&](int sp) {
    return make_rsrc(a.part + (static_cast<int64_t>(sp) * tiles + tile) * TILE, static_cast<uint32_t>(TILE * 4));
  };
  {
    const rsrc_t p = slice(split);
    for (int i = t; i < TILE / 4; i += NW * kWave) {
      const int m = i / (FB * 4), n = i % (FB * 4) * 4;
      if (m >= rows_x) break;
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, sum4(m, n)), p, i * 16, 0, kCoherent);
    }
  }
  mem_done();
  __syncthreads();
  if (t == 0) ticket = __hip_atomic_fetch_add(a.arrived + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (ticket != static_cast<uint32_t>(a.splits - 1)) return;
  if (t == 0) sync_store(a.arrived + tile, 0u);
  for (int i = t; i < UNITS; i += NW * kWave) {
    const int m = i / (TN / 4), n = i % (TN / 4) * 4;
    if (m >= rows_x || n >= rows_w) continue;
    f32x4 z4 = zero, u4 = zero;
    const uint32_t at = static_cast<uint32_t>(m * FB * 16 + n) * 4;
#pragma unroll 4
    for (int sp = 0; sp < a.splits; ++sp) {
      const rsrc_t p = slice(sp);
      z4 += __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(p, at, 0, kCoherent));
      if (GATED) u4 += __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(p, at + TN * 4, 0, kCoherent));
    }
    out4(m, n, z4, u4);
  }
}

hipError_t launch_thin(const Args& a, bool bf16, bool gated, hipStream_t s) {
  void (*const kernels[])(Args) = {thin_kernel<Half, false>, thin_kernel<Half, true>, thin_kernel<BFloat, false>,
                                   thin_kernel<BFloat, true>};
  hipLaunchKernelGGL(kernels[2 * bf16 + gated], dim3(static_cast<uint32_t>(grid_of(a.m_tiles, a.n_tiles * a.splits))),
                     dim3(NW * kWave), 0, s, a);
  return hipGetLastError();
}

}  // namespace lin
}  // namespace vt
