// Products of many rows: vt_linear and vt_linear_gated on tiles of 256 rows x 256 or 128 weight rows.
//
// Four waves, one per SIMD, of 128 x 128 each (accumulators in all 256 AGPRs) or 128 x 64. Both operands go from
// memory straight into LDS, 16 bytes a lane and 1 KiB an instruction, in k-tiles of 64 through a ring of five
// half-tiles; a wave multiplies one k-step of 32 while it reads the next one's fragments and sends its share of the
// loads of a k-tile further on, so that nothing stands between two products for longer than the first of them takes.
// A gated product's weight blocks are half a wave's of the gate and half of the up projection in turn, for the same
// features, so a feature's two sums are in the same lane.
//
// The product's first operand is the weights: a lane's four accumulators are then four consecutive features of a
// row, one 16-byte store each on the way through LDS to the epilogue, in which 16 lanes take a row's
// features 8 at a time. That loop stays rolled (its instructions come from memory, once per workgroup).
//
// Rows past the matrices' ends are read from their last row (the sums are never stored). A last k-tile that
// reaches past K goes through registers, masked, and is multiplied first.
//
// What bounds it: the matrix units, 1450 to 1480 TFLOP/s at 8192 x 8192 x 8192 in bf16 (743 to 757 us); then the
// rounds of compute units that do not come out even, and the epilogue, which nothing overlaps and which is most of the
// time where K is short (4096 rows of 64 through 4096 features 17 us for 35 MB). 4096 rows of 5120 through 13824
// features with bias and GELU in fp16 468 to 494 us, 460 without the activation; of 4096 through a gate and an up
// projection of 11008 features each 524 to 540 us in bf16, 1370 to 1410 TFLOP/s.
#include "linear_lds.hpp"

namespace vt {
namespace lin {

constexpr int TK = 64, TT = 256;
constexpr int ST = 5;      // slots of half a k-tile
constexpr int ER = 64;     // rows of a wave in the epilogue's LDS

constexpr int slot_bytes(int mb, int nb) { return 2 * (mb + nb) * 1024; }
constexpr int tile_lds(int mb, int nb) {
  const int ring = ST * slot_bytes(mb, nb), epilogue = 4 * ER * (16 * nb + 4) * 4;
  return ring > epilogue ? ring : epilogue;
}

// The tile of row m_tile and of the features from n0. MB, NB: 16-row blocks of rows and of weights of a wave.
template <class T, bool GATED, int MB, int NB>
__device__ __forceinline__ void tile(const Args& a, char* lds, int m_tile, int n0) {
  constexpr int SLOT = slot_bytes(MB, NB), XB = 2 * MB * 1024;
  constexpr int TM = 32 * MB, TN = 32 * NB, NO = GATED ? TN / 2 : TN;  // rows, weight rows, features of a tile
  constexpr int P = MB * NB, R = MB + NB, LX = MB / 2, LPS = R / 2;    // products, reads, loads of a wave per half
  const int m0 = m_tile * TM;
  const int t = threadIdx.x, lane = t % kWave, wave = __builtin_amdgcn_readfirstlane(t / kWave);
  const int full = a.K / TK;
  const bool tail = full * TK < a.K;

  const uint32_t lbase = lds_address(lds);
  // A slot holds the first or the last 8 rows of every 16-row block, 64 k wide; this wave loads a quarter of its
  // row blocks and of its weight blocks.
  const int brow = block_row(lane);
  const int which = GATED ? wave % 2 : 0, wrow = (GATED ? wave / 2 : wave) * NB * 8;
  const int rows_x = min(TM, a.M - m0), rows_w = min(NO, a.N - n0);
  u32x4 rx = rsrc_words(a.x + m0 * a.ld_x, static_cast<uint32_t>(rows_x * a.ld_x * 2));
  u32x4 rw = rsrc_words(a.w[which] + n0 * a.ld_w[which], static_cast<uint32_t>(rows_w * a.ld_w[which] * 2));
  uint32_t xo[2][LX], wo[2][NB / 2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int u = 0; u < LX; ++u)
      xo[h][u] = static_cast<uint32_t>(min(wave * MB * 8 + u * 16 + h * 8 + brow, rows_x - 1) * a.ld_x * 2) +
                 block_chunk(lane, h) * 16;
#pragma unroll
    for (int u = 0; u < NB / 2; ++u)
      wo[h][u] = static_cast<uint32_t>(min(wrow + u * 16 + h * 8 + brow, rows_w - 1) * a.ld_w[which] * 2) +
                 block_chunk(lane, h) * 16;
  }
  // A half's loads of this wave, the rows' first. Past the last k-tile they go on with empty
  // ranges from offset 0 (no memory traffic, slots that nobody reads), so the counts stay.
  uint32_t koff = full ? first_of(blockIdx.x, full) * (TK * 2) : 0;
  int left = full;
  const uint32_t placex = lbase + wave * LX * 1024, placew = lbase + XB + wave * (NB / 2) * 1024;
  auto place = [&](int i) { return i < LX ? placex : placew; };
  auto target = [](auto i) {
    constexpr int v = decltype(i)::value;
    return std::integral_constant<int, (v < LX ? v : v - LX) * 1024>{};
  };
  auto with = [&](auto H, auto I, auto&& f) {
    constexpr int h = decltype(H)::value, i = decltype(I)::value;
    if constexpr (i < LX) f(rx, xo[h][i], koff);
    else f(rw, wo[h][i - LX], koff);
  };
  auto none_left = [&]() {
    rx.z = 0;
    rw.z = 0;
    koff = 0;
  };
  auto advance = [&]() {  // after both halves of a k-tile
    koff += TK * 2;
    if (koff == static_cast<uint32_t>(full) * (TK * 2)) koff = 0;
    if (--left <= 0) none_left();
  };
  auto stage_tail = [&]() {  // the k-tile that reaches past K, with zeros there, to the first two slots
    const rsrc_t bx = rsrc_of(rx), bw = rsrc_of(rw);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = full * TK + block_chunk(lane, h) * 8;
      const uint32_t gone = k < a.K ? 0u : kOOB;
#pragma unroll
      for (int u = 0; u < LX; ++u)
        *reinterpret_cast<u32x4*>(lds + h * SLOT + (wave * LX + u) * 1024 + lane * 16) =
            keep_first(load_at(bx, xo[h][u] | gone, full * TK * 2), a.K - k);
#pragma unroll
      for (int u = 0; u < NB / 2; ++u)
        *reinterpret_cast<u32x4*>(lds + h * SLOT + XB + (wave * (NB / 2) + u) * 1024 + lane * 16) =
            keep_first(load_at(bw, wo[h][u] | gone, full * TK * 2), a.K - k);
    }
  };

  const int wm = wave / 2, wn = wave % 2;
  f32x4 acc[NB][MB];
#pragma unroll
  for (int f = 0; f < NB; ++f)
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[f][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int fa = fragment_at(lane), xaddr = wm * MB * 1024, waddr = XB + wn * NB * 1024;
  const bool second = lane % 16 >= 8;  // this lane's row is in a k-tile's second slot
  u32x4 xf[2][MB], wf[2][NB];
  auto read1 = [&](int i, const char* S, int set) {
    if (i < MB) xf[set][i] = *reinterpret_cast<const u32x4*>(S + xaddr + i * 1024);
    else wf[set][i - MB] = *reinterpret_cast<const u32x4*>(S + waddr + (i - MB) * 1024);
  };
  // The products of a k-step (HALF: of the k-tile's two). In the shadow of their first half the other register set is
  // read (the next k-step, from S). This wave's loads of half HALF of a later k-tile go out to ``into`` beside
  // them, as early as there is room between two products.
  auto multiply = [&](auto HALF, const char* S, uint32_t into) {
    constexpr int set = decltype(HALF)::value, H = P / 2;
    each<P>([&](auto I) {
      constexpr int i = decltype(I)::value, f = i / MB, b = i % MB;
      acc[f][b] = T::mfma16(wf[set][f], xf[set][b], acc[f][b]);
      if constexpr (i < H) {
        constexpr int r = (i * R + H - 1) / H;  // read r goes after product r H / R
        if constexpr (r < R && r * H / R == i) read1(r, S, 1 - set);
      }
      each<LPS>([&](auto L) {
        constexpr int l = decltype(L)::value, at = ((2 * l + 1) * H / (2 * LPS)) | 1;
        if constexpr (at == i) put<decltype(target(L))::value>(place(l) + into);
        if constexpr (at + 1 == i) with(HALF, L, fetch);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // The k-tile past K first, then 0, 1, ..; k-tile q of that order is in slots 2 q and 2 q + 1 (mod ST). Its second
  // k-step's fragments are read beside its first products; then its slots are free. Beside its first products
  // half 0 of k-tile q + 2 goes out, to the fifth slot, beside its second ones half 1, to its own first slot. The next
  // k-tile has to be there before the second products: all but the newest half.
  const int KT = full + (tail ? 1 : 0);
  if (tail) stage_tail();
  if (left <= 0) none_left();
  each<2>([&](auto Q) {
    constexpr int q = decltype(Q)::value;
    if (q > 0 || !tail) {
      each<2>([&](auto h) {
        each<LPS>([&](auto i) {
          with(h, i, [&](u32x4 r, uint32_t voff, uint32_t soff) {
            put_fetch<decltype(target(i))::value>(place(decltype(i)::value) + (2 * q + decltype(h)::value) * SLOT, r,
                                                  voff, soff);
          });
        });
      });
      advance();
    }
  });
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * LPS) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  auto up = [&](uint32_t x) { return x + SLOT == ST * SLOT ? 0u : x + SLOT; };
  uint32_t cur = 0;  // the k-tile's first slot
  auto at = [&](uint32_t first) { return lds + (second ? up(first) : first); };
#pragma unroll
  for (int i = 0; i < R; ++i) read1(i, at(0) + fa, 0);
  __builtin_amdgcn_sched_barrier(0);
  auto step = [&]() {
    const uint32_t next = up(up(cur));
    multiply(std::integral_constant<int, 0>{}, at(cur) + (fa ^ 64), up(up(next)));
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LPS) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    multiply(std::integral_constant<int, 1>{}, at(next) + fa, cur);
    advance();
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
  for (int q = 0; q < KT; ++q) step();
  pin();
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();

  // ---- epilogue, each wave for itself: ER rows at a time through its piece of LDS
  constexpr int ELD = 16 * NB + 4;
  static_assert(MB % 4 == 0 && NB % 4 == 0, "");
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
      if (!a.res || !there) return;
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
          if (whole) *reinterpret_cast<u32x4*>(y) = v;
          else store_first<8>(y, v, a.N % 8);
        }
      }
#pragma unroll
      for (int p = 0; p < PB; ++p) cur_r[p] = nxt_r[p];
    }
  });
}

// Columns of wide tiles, then of narrow ones, which fill the last round of the compute units.
template <class T, bool GATED>
__global__ void __launch_bounds__(TT, 1) tile_kernel(Args a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  constexpr int WIDE = kWide.features / (GATED ? 2 : 1), NARROW = kNarrow.features / (GATED ? 2 : 1);
  const int id = blockIdx.x, wide = static_cast<int>(grid_of(a.m_tiles, a.wide));
  int m, col;
  if (id < wide) {
    if (my_tile(id, a.m_tiles, a.wide, kWide.rows, m, col)) tile<T, GATED, 8, 8>(a, lds, m, col * WIDE);
  } else {
    if (my_tile(id - wide, a.m_tiles, a.n_tiles, kNarrow.rows, m, col))
      tile<T, GATED, 8, 4>(a, lds, m, a.wide * WIDE + col * NARROW);
  }
}

hipError_t launch_tile(const Args& a, bool bf16, bool gated, hipStream_t s) {
  static LdsOnce once;
  void (*const kernels[])(Args) = {tile_kernel<Half, false>, tile_kernel<Half, true>, tile_kernel<BFloat, false>,
                                   tile_kernel<BFloat, true>};
  constexpr int lds = tile_lds(8, 8) > tile_lds(8, 4) ? tile_lds(8, 8) : tile_lds(8, 4);
  static_assert(lds <= 160 * 1024, "one workgroup per compute unit");
  const hipError_t e = once([&](auto&& raise) {
    for (auto* f : kernels) raise(reinterpret_cast<const void*>(f), lds);
  });
  if (e != hipSuccess) return e;
  const int64_t grid = grid_of(a.m_tiles, a.wide) + grid_of(a.m_tiles, a.n_tiles);
  hipLaunchKernelGGL(kernels[2 * bf16 + gated], dim3(static_cast<uint32_t>(grid)), dim3(TT), lds, s, a);
  return hipGetLastError();
}

}  // namespace lin
}  // namespace vt
