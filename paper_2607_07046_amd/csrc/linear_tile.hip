// Products of many rows: vt_linear and vt_linear_gated on tiles of 256 rows x 256 features.
//
// Four waves, one per SIMD, of 128 x 128 each (accumulators in all 256 AGPRs). Both operands go from memory
// straight into LDS, 16 bytes a lane and 1 KiB an instruction, through a ring of ST stages of 32 k; a wave
// multiplies one stage while it reads the next one's fragments and sends its share of the loads of one
// further on, so that nothing stands between two products for longer than the first of them takes. A gated
// product's weight blocks are four of the gate and four of the up projection in turn, 64 features of both for each wave, so a
// feature's two sums are in the same lane.
//
// The product's first operand is the weights: a lane's four accumulators are then four consecutive features of a
// row, one 16-byte store each on the way through LDS to the epilogue, in which 16 lanes take a row's
// features 8 at a time. That loop stays rolled (its instructions come from memory, once per workgroup).
//
// Rows past the matrices' ends are read from their last row (the sums are never stored). A last k-tile that
// reaches past K goes through registers, masked, and is multiplied first.
#include <mutex>
#include <vector>

#include "linear_lds.hpp"

namespace vt {
namespace lin {

constexpr int TK = 32, TT = 256;
constexpr int WALK_M = 8;  // row tiles of a block of an XCD's walk

// Stages of the ring: as many as one workgroup (the large tiles) or two (128 x 128) have room for.
constexpr int stages(int mb, int nb) { return mb * nb == 64 ? 5 : (mb * nb == 32 ? 6 : 5); }
constexpr int stage_bytes(int mb, int nb) { return 2 * (mb + nb) * 1024; }
constexpr int tile_lds(int mb, int nb) { return stages(mb, nb) * stage_bytes(mb, nb); }

// MB, NB: 16-row blocks of rows and of weights of a wave.
template <class T, bool GATED, int MB, int NB, bool SPLIT>
__global__ void __launch_bounds__(TT, MB* NB == 16 ? 2 : 1) tile_kernel(Args a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  constexpr int ST = stages(MB, NB), STAGE = stage_bytes(MB, NB), XB = 2 * MB * 1024;
  constexpr int TM = 32 * MB, TN = 32 * NB, NO = GATED ? TN / 2 : TN;  // rows, weight rows, features of a tile
  constexpr int P = MB * NB, R = MB + NB, LX = MB / 2, LPS = R / 2;    // products, reads, loads of a wave per k-tile
  // An XCD takes every eighth column of tiles, in blocks of WALK_M rows of them: the tiles that run there
  // at once share rows and weights in its L2.
  const int cols = SPLIT ? a.n_tiles * a.splits : a.n_tiles;
  const int id = blockIdx.x, groups = (cols + 7) / 8, j = id / 8;
  const int bm = min(a.m_tiles, WALK_M), blk = j / (bm * groups);
  const int rows = min(bm, a.m_tiles - blk * bm), rr = j - blk * bm * groups;
  const int col = rr / rows * 8 + id % 8, m_tile = blk * bm + rr % rows;
  if (col >= cols) return;
  const int n_tile = SPLIT ? col % a.n_tiles : col, split = SPLIT ? col / a.n_tiles : 0;
  const int m0 = m_tile * TM, n0 = n_tile * NO;
  const int t = threadIdx.x, lane = t % kWave, wave = __builtin_amdgcn_readfirstlane(t / kWave);
  const int full = a.K / TK, kt0 = SPLIT ? split * a.steps : 0, kt1 = SPLIT ? min(kt0 + a.steps, full) : full;
  const bool tail = full * TK < a.K && (!SPLIT || (full >= kt0 && full < kt0 + a.steps));
  const int KT = max(kt1 - kt0, 0) + (tail ? 1 : 0);

  const uint32_t lbase = lds_address(lds);
  // This wave loads a quarter of the rows' blocks and of the weights'; lane l's row and chunk of a
  // block are what LDS unit l holds.
  const int brow = block_row(lane), bchunk = block_chunk(lane);
  const int which = GATED ? wave % 2 : 0, wrow = (GATED ? wave / 2 : wave) * NB * 8;
  const int rows_x = min(TM, a.M - m0), rows_w = min(NO, a.N - n0);
  u32x4 rx = rsrc_words(a.x + m0 * a.ld_x, static_cast<uint32_t>(rows_x * a.ld_x * 2));
  u32x4 rw = rsrc_words(a.w[which] + n0 * a.ld_w[which], static_cast<uint32_t>(rows_w * a.ld_w[which] * 2));
  uint32_t xo[LX], wo[NB / 2];
#pragma unroll
  for (int u = 0; u < LX; ++u)
    xo[u] = static_cast<uint32_t>(min(wave * MB * 8 + u * 16 + brow, rows_x - 1) * a.ld_x * 2) + bchunk * 16;
#pragma unroll
  for (int u = 0; u < NB / 2; ++u)
    wo[u] = static_cast<uint32_t>(min(wrow + u * 16 + brow, rows_w - 1) * a.ld_w[which] * 2) + bchunk * 16;
  // A k-tile's loads of this wave, the rows' first. Past the last k-tile they go on with empty
  // ranges from offset 0 (no memory traffic, stages that nobody reads), so the counts stay.
  uint32_t koff = kt0 * (TK * 2);
  int left = kt1 - kt0;
  const uint32_t placex = lbase + wave * LX * 1024, placew = lbase + XB + wave * (NB / 2) * 1024;
  auto place = [&](int i) { return i < LX ? placex : placew; };
  auto target = [](auto i) {
    constexpr int v = decltype(i)::value;
    return std::integral_constant<int, (v < LX ? v : v - LX) * 1024>{};
  };
  auto with = [&](auto I, auto&& f) {
    constexpr int i = decltype(I)::value;
    if constexpr (i < LX) f(rx, xo[i], koff);
    else f(rw, wo[i - LX], koff);
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
    const rsrc_t bx = rsrc_of(rx), bw = rsrc_of(rw);
    const int k = full * TK + bchunk * 8;
    const uint32_t gone = k < a.K ? 0u : kOOB;
#pragma unroll
    for (int u = 0; u < LX; ++u)
      *reinterpret_cast<u32x4*>(lds + (wave * LX + u) * 1024 + lane * 16) =
          keep_first(load_at(bx, xo[u] | gone, full * TK * 2), a.K - k);
#pragma unroll
    for (int u = 0; u < NB / 2; ++u)
      *reinterpret_cast<u32x4*>(lds + XB + (wave * (NB / 2) + u) * 1024 + lane * 16) =
          keep_first(load_at(bw, wo[u] | gone, full * TK * 2), a.K - k);
  };

  const int wm = wave / 2, wn = wave % 2;
  f32x4 acc[NB][MB];
#pragma unroll
  for (int f = 0; f < NB; ++f)
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[f][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int xaddr = wm * MB * 1024 + fragment_at(lane), waddr = XB + wn * NB * 1024 + fragment_at(lane);
  u32x4 xf[2][MB], wf[2][NB];
  auto read1 = [&](int i, uint32_t stage, int set) {
    const char* S = lds + stage;
    if (i < MB) xf[set][i] = *reinterpret_cast<const u32x4*>(S + xaddr + i * 1024);
    else wf[set][i - MB] = *reinterpret_cast<const u32x4*>(S + waddr + (i - MB) * 1024);
  };
  // The products of a k-tile. In the shadow of their first half the other register set is read (the next
  // k-tile, from ``stage``), in that of their second half the loads of a later one go out to ``into``.
  auto multiply = [&](auto SET, uint32_t stage, uint32_t into) {
    constexpr int set = decltype(SET)::value, H = P / 2;
    each<P>([&](auto I) {
      constexpr int i = decltype(I)::value, f = i / MB, b = i % MB;
      acc[f][b] = T::mfma16(wf[set][f], xf[set][b], acc[f][b]);
      if constexpr (i < H) {
        constexpr int r = (i * R + H - 1) / H;  // read r goes after product r H / R
        if constexpr (r < R && r * H / R == i) read1(r, stage, 1 - set);
      } else {
        each<LPS>([&](auto L) {
          constexpr int l = decltype(L)::value, at = H + l * H / LPS, gap = H / LPS / 2 > 0 ? H / LPS / 2 : 1;
          if constexpr (at == i) put<decltype(target(L))::value>(place(l) + into);
          if constexpr (at + gap == i) with(L, fetch);
        });
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // The k-tile past K first, then kt0, ..; k-tile q of that order is in stage q % ST. While q is multiplied, q and
  // q + 1 are there and up to q + ST - 1 on the way: a wave waits for all but its newest ST - 3 k-tiles' loads.
  auto landed = [&]() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LPS * (ST - 3)) : "memory"); };
  if (tail) stage_tail();
  if (left <= 0) none_left();
  each<ST - 1>([&](auto Q) {
    constexpr int q = decltype(Q)::value;
    if (q > 0 || !tail) {
      each<LPS>([&](auto i) {
        with(i, [&](u32x4 r, uint32_t voff, uint32_t soff) {
          put_fetch<decltype(target(i))::value>(place(decltype(i)::value) + q * STAGE, r, voff, soff);
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
  for (int i = 0; i < R; ++i) read1(i, 0, 0);
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
  // the accumulators are in AGPRs: without this the compiler moves some out in the loop
  auto pin = [&]() {
#pragma unroll
    for (int f = 0; f < NB; ++f)
#pragma unroll
      for (int b = 0; b < MB; ++b) asm volatile("" : "+a"(acc[f][b]));
  };
  pin();
  for (int q = 0; q < KT; q += 2) {
    step(std::integral_constant<int, 0>{});
    if (q + 1 < KT) step(std::integral_constant<int, 1>{});
  }
  pin();
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();

  if constexpr (SPLIT) {
    if (!join<NB, MB, 4>(a, acc, lds, m_tile * a.n_tiles + n_tile, split, wave, lane)) return;
    __syncthreads();
  }

  // ---- epilogue, each wave for itself: ER rows at a time through its piece of LDS
  constexpr int ER = 64, ELD = 16 * NB + 4;
  static_assert(4 * ER * ELD * 4 <= tile_lds(MB, NB) && MB % 4 == 0, "the epilogue's LDS");
  constexpr int LPR = GATED ? NB : 2 * NB, RPP = kWave / LPR, PB = 4;  // lanes of a row, rows of a pass, passes in flight
  float* tl = reinterpret_cast<float*>(lds) + wave * ER * ELD;
  const int fc = lane % LPR * 8, n = n0 + wn * (GATED ? NB * 8 : NB * 16) + fc;
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
  each<MB / 4>([&](auto HALF) {
    constexpr int hf = decltype(HALF)::value;
    const int ms = m0 + wm * MB * 16 + hf * ER;
    if (ms >= a.M) return;
    lds_sync();
#pragma unroll
    for (int f = 0; f < NB; ++f)
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
            row8(NB * 8 + fc, u, bu);
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
  });
}

// The kernels' dynamic LDS raised to what they use, once per device.
hipError_t launch_tile(const Args& a, bool bf16, bool gated, hipStream_t s) {
  static std::mutex mu;
  static std::vector<char> ready;
  void (*const kernels[])(Args) = {tile_kernel<Half, false, 8, 8, false>, tile_kernel<Half, true, 8, 8, false>,
                                   tile_kernel<BFloat, false, 8, 8, false>, tile_kernel<BFloat, true, 8, 8, false>};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  {
    std::lock_guard<std::mutex> lk(mu);
    if (static_cast<int>(ready.size()) <= dev) ready.resize(dev + 1);
    if (!ready[dev]) {
      for (auto* k : kernels) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, tile_lds(8, 8));
        if (e != hipSuccess) return e;
      }
      ready[dev] = 1;
    }
  }
  hipLaunchKernelGGL(kernels[2 * bf16 + gated], dim3((a.n_tiles + 7) / 8 * 8 * a.m_tiles), dim3(TT), tile_lds(8, 8), s, a);
  return hipGetLastError();
}

}  // namespace lin
}  // namespace vt
