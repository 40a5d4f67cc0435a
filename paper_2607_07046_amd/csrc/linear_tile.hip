// Products of many rows: vt_linear and vt_linear_gated on tiles of 256 rows x 256 features.
//
// Four waves, one per SIMD, of 128 x 128 each (accumulators in all 256 AGPRs). Both operands go from memory
// straight into LDS, 16 bytes a lane and 1 KiB an instruction, through a ring of ST stages of 32 k; a wave
// multiplies one stage while it reads the next one's fragments and sends its share of the loads of one
// further on, so that nothing stands between two products for longer than the first of them takes. The loads are
// issued in inline asm and waited for by their count: with the compiler's own form every read of LDS
// waits for all of them.
//
// LDS holds blocks of 16 rows x 32 k, chunk c (16 bytes) of row r at unit 4 r + (c ^ (r / 2 % 4) ^ (r / 8)): the
// rows that one fragment read takes together are in different banks. A gated product's weight
// blocks are four of the gate and four of the up projection in turn, 64 features of both for each wave, so a
// feature's two sums are in the same lane.
//
// The product's first operand is the weights: a lane's four accumulators are then four consecutive features of a
// row, one 16-byte store each on the way through LDS to the epilogue, in which 16 lanes take a row's
// features 8 at a time. That loop stays rolled (its instructions come from memory, once per workgroup).
//
// Rows past the matrices' ends are read from their last row (the sums are never stored). A last k-tile that
// reaches past K goes through registers, masked, and is multiplied first.
#include <mutex>
#include <type_traits>
#include <vector>

#include "linear.hpp"

namespace vt {
namespace lin {

constexpr int TM = 256, TN = 256, TT = 256, TK = 32, ST = 5;
constexpr int XB = TM * TK * 2, STAGE = XB + TN * TK * 2;  // bytes of a stage's rows, and of a stage
constexpr int TILE_LDS = ST * STAGE;
static_assert(TILE_LDS <= 160 * 1024, "one workgroup per compute unit");
constexpr int ER = 64, ELD = 132;  // rows in the epilogue's piece of LDS, their floats
static_assert(4 * ER * ELD * 4 <= TILE_LDS, "the epilogue's LDS");
constexpr int WALK_M = 8;  // row tiles of a block of an XCD's walk

// 16 bytes per lane from r[voff + soff] to LDS at m0 + 16 * lane. m0 is set in the block of the load, with
// the wait state between, or by put() ahead of it where a product is issued in between; the clobbers
// keep the compiler's own writes of m0 out.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int OFF>
__device__ __forceinline__ void put(uint32_t base) {
  asm volatile("s_add_u32 m0, %0, %1"
               :
               : "s"(__builtin_amdgcn_readfirstlane(base)), "n"(OFF)
               : "m0", "scc", "memory");
}
__device__ __forceinline__ void fetch(u32x4 r, uint32_t voff, uint32_t soff) {
  asm volatile("buffer_load_dwordx4 %0, %1, %2 offen lds"
               :
               : "v"(voff), "s"(r), "s"(__builtin_amdgcn_readfirstlane(soff))
               : "memory");
}
template <int OFF>
__device__ __forceinline__ void put_fetch(uint32_t base, u32x4 r, uint32_t voff, uint32_t soff) {
  asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, %4 offen lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(base)), "n"(OFF), "v"(voff), "s"(r),
                 "s"(__builtin_amdgcn_readfirstlane(soff))
               : "m0", "scc", "memory");
}
#pragma clang diagnostic pop

__device__ __forceinline__ u32x4 rsrc_words(const void* base, uint32_t bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  return u32x4{static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(p))),
               static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(p >> 32))) & 0xFFFFu,
               static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(bytes))), 0x00020000u};
}

template <int N, int I = 0, class F>
__device__ __forceinline__ void each(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    each<N, I + 1>(f);
  }
}

template <class T, bool GATED>
__global__ void __launch_bounds__(TT, 1) tile_kernel(Args a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  constexpr int NO = GATED ? TN / 2 : TN;  // features of a tile
  // An XCD takes every eighth column of tiles, in blocks of WALK_M rows of them: the tiles that run there
  // at once share rows and weights in its L2.
  const int id = blockIdx.x, groups = (a.n_tiles + 7) / 8, j = id / 8;
  const int bm = min(a.m_tiles, WALK_M), blk = j / (bm * groups);
  const int rows = min(bm, a.m_tiles - blk * bm), rr = j - blk * bm * groups;
  const int n_tile = rr / rows * 8 + id % 8, m_tile = blk * bm + rr % rows;
  if (n_tile >= a.n_tiles) return;
  const int m0 = m_tile * TM, n0 = n_tile * NO;
  const int t = threadIdx.x, lane = t % kWave, wave = __builtin_amdgcn_readfirstlane(t / kWave);
  const int KT = (a.K + TK - 1) / TK, full = a.K / TK;
  const bool tail = full != KT;

  const uint32_t lbase =
      static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds));
  // This wave loads blocks 4 w .. 4 w + 3 of the rows and of the weights; lane l's row and chunk of a
  // block are what LDS unit l holds.
  const int brow = lane / 4, bchunk = (lane % 4) ^ (brow >> 1 & 3) ^ (brow >> 3);
  const int which = GATED ? wave % 2 : 0, wrow = GATED ? wave / 2 * 64 : wave * 64;
  const int rows_x = min(TM, a.M - m0), rows_w = min(NO, a.N - n0);
  u32x4 rx = rsrc_words(a.x + m0 * a.ld_x, static_cast<uint32_t>(rows_x * a.ld_x * 2));
  u32x4 rw = rsrc_words(a.w[which] + n0 * a.ld_w[which], static_cast<uint32_t>(rows_w * a.ld_w[which] * 2));
  uint32_t xo[4], wo[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    xo[u] = static_cast<uint32_t>(min(wave * 64 + u * 16 + brow, rows_x - 1) * a.ld_x * 2) + bchunk * 16;
    wo[u] = static_cast<uint32_t>(min(wrow + u * 16 + brow, rows_w - 1) * a.ld_w[which] * 2) + bchunk * 16;
  }
  // A k-tile's loads of this wave: 0..3 rows, 4..7 weights. Past the last k-tile they go on with empty
  // ranges from offset 0 (no memory traffic, stages that nobody reads), so the counts stay.
  uint32_t koff = 0;
  int left = full;
  const uint32_t place0 = lbase + wave * 4096;
  auto target = [](auto i) {
    constexpr int v = decltype(i)::value;
    return std::integral_constant<int, (v < 4 ? v * 1024 : XB + (v - 4) * 1024)>{};
  };
  auto with = [&](auto I, auto&& f) {
    constexpr int i = decltype(I)::value;
    if constexpr (i < 4) f(rx, xo[i], koff);
    else f(rw, wo[i - 4], koff);
  };
  auto none_left = [&]() {
    rx.z = 0;
    rw.z = 0;
    koff = 0;
  };
  auto advance = [&]() {
    koff += TK * 2;
    if (--left <= 0) none_left();
  };
  auto stage_tail = [&]() {  // the k-tile that reaches past K, with zeros there, to stage 0
    const uint64_t px = (static_cast<uint64_t>(rx.y) << 32) | rx.x, pw = (static_cast<uint64_t>(rw.y) << 32) | rw.x;
    const rsrc_t bx = make_rsrc(reinterpret_cast<const void*>(px), rx.z);
    const rsrc_t bw = make_rsrc(reinterpret_cast<const void*>(pw), rw.z);
    const int k = full * TK + bchunk * 8;
    const uint32_t gone = k < a.K ? 0u : kOOB;
    char* to = lds + wave * 4096 + lane * 16;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const u32x4 vx = keep_first(load_at(bx, xo[u] | gone, full * TK * 2), a.K - k);
      const u32x4 vw = keep_first(load_at(bw, wo[u] | gone, full * TK * 2), a.K - k);
      *reinterpret_cast<u32x4*>(to + u * 1024) = vx;
      *reinterpret_cast<u32x4*>(to + XB + u * 1024) = vw;
    }
  };

  const int wm = wave / 2, wn = wave % 2;
  f32x4 acc[8][8];  // [features][rows]
#pragma unroll
  for (int f = 0; f < 8; ++f)
#pragma unroll
    for (int b = 0; b < 8; ++b) acc[f][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  // fragments of 16 rows x 32 k: lane l has row l % 16, chunk l / 16
  const int fr = lane % 16, fu = (fr * 4 + ((lane / 16) ^ (fr >> 1 & 3) ^ (fr >> 3))) * 16;
  const int xaddr = wm * 8192 + fu, waddr = XB + wn * 8192 + fu;
  u32x4 xf[2][8], wf[2][8];
  auto read1 = [&](int i, uint32_t stage, int set) {
    const char* S = lds + stage;
    if (i < 8) xf[set][i] = *reinterpret_cast<const u32x4*>(S + xaddr + i * 1024);
    else wf[set][i - 8] = *reinterpret_cast<const u32x4*>(S + waddr + (i - 8) * 1024);
  };
  auto multiply = [&](auto SET, uint32_t stage, uint32_t into) {
    constexpr int set = decltype(SET)::value;
    each<64>([&](auto I) {
      constexpr int i = decltype(I)::value, f = i / 8, b = i % 8;
      acc[f][b] = T::mfma16(wf[set][f], xf[set][b], acc[f][b]);
      if constexpr (i < 32 && i % 2 == 0) read1(i / 2, stage, 1 - set);
      if constexpr (i >= 32 && i % 4 == 0)
        put<decltype(target(std::integral_constant<int, (i - 32) / 4>{}))::value>(place0 + into);
      if constexpr (i >= 32 && i % 4 == 2) with(std::integral_constant<int, (i - 32) / 4>{}, fetch);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // The k-tile past K first, then 0, 1, ..; k-tile q of that order is in stage q % ST. While q is multiplied, q and
  // q + 1 are there and up to q + ST - 1 on the way: a wave waits for all but its newest ST - 3 k-tiles' loads.
  auto landed = [&]() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(8 * (ST - 3)) : "memory"); };
  const int shift = tail ? 1 : 0;
  if (tail) stage_tail();
  if (left <= 0) none_left();
  each<ST - 1>([&](auto Q) {
    constexpr int q = decltype(Q)::value;
    if (q >= shift) {
      each<8>([&](auto i) {
        with(i, [&](u32x4 r, uint32_t voff, uint32_t soff) {
          put_fetch<decltype(target(i))::value>(place0 + q * STAGE, r, voff, soff);
        });
      });
      advance();
    }
  });
  landed();
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) read1(i, 0, 0);
  __builtin_amdgcn_sched_barrier(0);
  uint32_t cur = 0, into = (ST - 1) * STAGE;
  auto step = [&](auto SET) {
    const uint32_t next = cur + STAGE == ST * STAGE ? 0 : cur + STAGE;
    multiply(SET, next, into);  // everyone is done with k-tile q - 1, whose stage takes q + ST - 1
    advance();
    landed();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    into = cur;
    cur = next;
  };
  // the accumulators are the AGPR half of the registers: without this the compiler moves some out in the loop
  auto pin = [&]() {
#pragma unroll
    for (int f = 0; f < 8; ++f)
#pragma unroll
      for (int b = 0; b < 8; ++b) asm volatile("" : "+a"(acc[f][b]));
  };
  pin();
  for (int q = 0; q < KT; q += 2) {
    step(std::integral_constant<int, 0>{});
    if (q + 1 < KT) step(std::integral_constant<int, 1>{});
  }
  pin();
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();

  // ---- epilogue, each wave for itself: ER rows at a time through its piece of LDS
  constexpr int LPR = GATED ? 8 : 16, RPP = kWave / LPR, PB = 4;  // lanes of a row, rows of a pass, passes in flight
  float* tl = reinterpret_cast<float*>(lds) + wave * ER * ELD;
  const int fc = lane % LPR * 8, n = n0 + wn * (GATED ? 64 : 128) + fc;
  const bool there = n < a.N, whole = n + 8 <= a.N;
  auto lds_sync = [&]() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  float bz[8] = {}, bu[8] = {};
  auto take = [&](const uint16_t* p, float (&to)[8]) {
    if (!p || !there) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) to[e] = n + e < a.N ? one<T>(p + n + e) : 0.f;
  };
  take(a.bias[0], bz);
  if (GATED) take(a.bias[1], bu);
  auto half = [&](auto HALF) {
    constexpr int hf = decltype(HALF)::value;
    const int ms = m0 + wm * 128 + hf * ER;
    if (ms >= a.M) return;
    lds_sync();
#pragma unroll
    for (int f = 0; f < 8; ++f)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        *reinterpret_cast<f32x4*>(tl + (16 * b + lane % 16) * ELD + 16 * f + 4 * (lane / 16)) = acc[f][4 * hf + b];
    lds_sync();
    u32x4 cur_r[PB], nxt_r[PB];
    auto ahead = [&](int r0, u32x4 (&to)[PB]) {
      if (!a.res || !whole) return;
#pragma unroll
      for (int p = 0; p < PB; ++p) {
        const int m = min(ms + r0 + p * RPP + lane / LPR, a.M - 1);
        to[p] = load16(a.res + m * a.ld_r + n);
      }
    };
    ahead(0, cur_r);
#pragma unroll 1
    for (int r0 = 0; r0 < ER; r0 += PB * RPP) {
      ahead(r0 + PB * RPP, nxt_r);
#pragma unroll
      for (int p = 0; p < PB; ++p) {
        const int mm = r0 + p * RPP + lane / LPR, m = ms + mm;
        if (m < a.M && there) {
          float z[8], u[8];
          auto row8 = [&](int at, float (&v)[8], const float (&b)[8]) {
            const f32x4 lo = *reinterpret_cast<const f32x4*>(tl + mm * ELD + at);
            const f32x4 hi = *reinterpret_cast<const f32x4*>(tl + mm * ELD + at + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              v[e] = lo[e] + b[e];
              v[4 + e] = hi[e] + b[4 + e];
            }
          };
          row8(fc, z, bz);
          activate(z, a.act);
          if (GATED) {
            row8(64 + fc, u, bu);
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] *= u[e];
          }
          uint16_t* y = a.y + m * a.ld_y + n;
          if (whole) {
            if (a.res) {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float lo, hi;
                T::unpack2(cur_r[p][e], lo, hi);
                z[2 * e] += lo;
                z[2 * e + 1] += hi;
              }
            }
            u32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = T::pack2(z[2 * e], z[2 * e + 1]);
            *reinterpret_cast<u32x4*>(y) = v;
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (n + e < a.N)
                y[e] = static_cast<uint16_t>(T::pack2(z[e] + (a.res ? one<T>(a.res + m * a.ld_r + n + e) : 0.f), 0.f));
          }
        }
      }
#pragma unroll
      for (int p = 0; p < PB; ++p) cur_r[p] = nxt_r[p];
    }
  };
  half(std::integral_constant<int, 0>{});
  half(std::integral_constant<int, 1>{});
}

// The kernels' dynamic LDS raised to what they use, once per device.
hipError_t launch_tile(const Args& a, bool bf16, bool gated, hipStream_t s) {
  static std::mutex mu;
  static std::vector<char> ready;
  void (*const kernels[])(Args) = {tile_kernel<Half, false>, tile_kernel<Half, true>, tile_kernel<BFloat, false>,
                                   tile_kernel<BFloat, true>};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  {
    std::lock_guard<std::mutex> lk(mu);
    if (static_cast<int>(ready.size()) <= dev) ready.resize(dev + 1);
    if (!ready[dev]) {
      for (auto* k : kernels) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, TILE_LDS);
        if (e != hipSuccess) return e;
      }
      ready[dev] = 1;
    }
  }
  hipLaunchKernelGGL(kernels[2 * bf16 + gated], dim3((a.n_tiles + 7) / 8 * 8 * a.m_tiles), dim3(TT), TILE_LDS, s, a);
  return hipGetLastError();
}

}  // namespace lin
}  // namespace vt
