// Products of a batch's or a short prompt's rows: vt_linear and vt_linear_gated on tiles between those of
// linear_thin.hip and linear_tile.hip.
//
// WR x WC places of 16 MBW rows x 16 NBW weight rows each. Both operands come straight into LDS through a
// ring of ST stages of 64 k, up to ST - 1 of them on the way, each number once per tile; the
// waves wait for a stage by the count of their own loads and meet once per stage.
//
// On tiles of 32 rows and more two waves share a place and take one of a stage's two k-steps each (KW = 2): a place
// can then be twice as high, and LDS, which bounds these tiles, is read two thirds as much (128 x 128: 64 KiB of a
// stage, not 96). The next stage's fragments are read, and loads sent out, between single products. The two waves'
// sums meet in LDS at the end, half of the rows for each. A stage takes 0.098 us at 32 x 64, 0.125 at 64 x 64, 0.175
// at 64 x 128 and 0.278 at 128 x 128, where one wave per place that read, then multiplied took 0.148, 0.190, 0.259
// and 0.414.
//
// The product's first operand is the weights: a lane's accumulators are consecutive features of a row. The weight
// rows of two blocks are dealt to them four by four in turn, so a lane has 8 consecutive features,
// 16 bytes of the result, and the epilogue works from the registers. Slices of K over several workgroups
// meet in the workspace, in register order, added in slice order by whichever arrives last, which waits for
// nobody.
//
// Rows past the matrices' ends are read from their last row (the sums are never stored). The stage that reaches
// past K goes through registers, masked, and is multiplied first.
//
// Where rows do not start at 128-byte lines, 128 bytes of a row are in two lines, and each line is asked for twice,
// half of it a time, which memory serves at half its rate. SHIFT loads whole lines: a stage holds a line of each row,
// from the one of the row's start on, whose last chunks are the row's next ones. They lie where a row's chunks always
// do, so reads meet no bank conflict, and a lane takes its chunk from a stage or from the next one. Since 8 rows are
// whole lines, which of them depends on the row within the fragment alone: a lane's place in LDS is its own, and goes
// round the ring. It keeps one more stage and K's order; the stage past K comes last, its fragments masked. The matrices
// themselves have to start at lines, else there would be reads before them. (Measured, bf16: 64 rows of 4104 numbers
// through 14336 features 39 -> 28 us, as at 4096; with the weights in memory 640 rows of 3920 through 11678 118 ->
// 84; what the choice costs elsewhere is in linear.hip. With chunks where they lie in their lines, conflicts in LDS
// cost half of that again.)
//
// What bounds it: up to about 64 rows reading the weights, above it LDS (at 128 x 128 the products of a stage take
// 512 cycles, the fragments' reads 512 and the loads' writes 256; it takes about 650). Measured in bf16: 64 rows of
// 8192 through the gate and up projections of 7168 features 47 to 49 us, 4.8 to 5.0 TB/s; rows of 4096 through 4096
// features: 256 rows 16 us (540 TFLOP/s), 512 22 (780), 1024 33 (1040); 777 rows of 3302 through 4096 with a residual
// 28 to 32. Tried at 128 x 128 and not kept: a quarter of the products ahead of the meeting point, no faster; the large
// tile's schedule for four waves; three stages of 64 x 128, so that two workgroups fit, 1% slower.
#include "linear_lds.hpp"

namespace vt {
namespace lin {

template <class T, bool GATED, int WR, int WC, int KW, int MBW, int NBW, int ST, bool SHIFT>
__global__ void __launch_bounds__(WR* WC* KW* kWave) mid_kernel(Args a) {
  constexpr int NW = WR * WC * KW, XB = WR * MBW, WB = WC * NBW;  // waves; 16-row blocks of rows and of weights
  constexpr int U = 2 * (XB + WB), LPS = U / NW;              // units (8 rows x 64 k) of a stage, loads of a wave
  constexpr int NBO = GATED ? NBW / 2 : NBW;                 // 16-feature blocks of a wave
  constexpr int TM = 16 * XB, TN = 16 * WC * NBO, TK = 64, STAGE = U * 1024, PW = NBO % 2 ? 4 : 8;
  constexpr int HS = 2 / KW, MBO = MBW / KW;                  // k-steps of a stage, row blocks of the result, of a wave
  static_assert(U % NW == 0 && (!GATED || NBW % 2 == 0) && KW <= 2 && MBW % KW == 0, "");
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int m_tile, unit;
  if (!my_tile(blockIdx.x, a.m_tiles, a.n_tiles * a.splits, TM, m_tile, unit)) return;
  const int n_tile = unit % a.n_tiles, split = unit / a.n_tiles;
  const int m0 = m_tile * TM, n0 = n_tile * TN;
  const int t = threadIdx.x, lane = t % kWave, wave = __builtin_amdgcn_readfirstlane(t / kWave);
  const int full = a.K / TK, kt0 = split * a.steps, kt1 = min(kt0 + a.steps, full);
  const bool tail = full * TK < a.K && full >= kt0 && full < kt0 + a.steps;
  const int KT = max(kt1 - kt0, 0) + (tail ? 1 : 0);

  // This wave loads units wave, wave + NW, .. of a stage: unit v is half v % 2 of block v / 2, the rows' first.
  const int rows_x = min(TM, a.M - m0), rows_w = min(TN, a.N - n0);
  // up to the last 8 numbers of the last row: a line that SHIFT loads may go on past them
  auto matrix = [&](const uint16_t* p, int64_t ld, int first, int rows) {
    return rsrc_words(p + first * ld, static_cast<uint32_t>(((rows - 1) * ld + (a.K + 7) / 8 * 8) * 2));
  };
  const u32x4 rx = matrix(a.x, a.ld_x, m0, rows_x), rw0 = matrix(a.w[0], a.ld_w[0], n0, rows_w);
  const u32x4 rw1 = GATED ? matrix(a.w[1], a.ld_w[1], n0, rows_w) : rw0;
  // chunks (8 numbers) by which a row starts into its line
  auto into_line = [](int64_t row, int64_t ld) { return SHIFT ? static_cast<int>(row * ld / 8) % 8 : 0; };
  u32x4 rs[LPS];
  uint32_t off[LPS];
#pragma unroll
  for (int i = 0; i < LPS; ++i) {
    const int v = wave + NW * i, b = v / 2, half = v % 2, brow = 8 * half + block_row(lane);
    int64_t ld = a.ld_x;
    int row;
    rs[i] = rx;
    if (b < XB) {
      row = min(16 * b + brow, rows_x - 1);
    } else {
      const int wb = b - XB, fb = wb % NBW, fo = fb % NBO;
      const bool up = GATED && fb >= NBO;
      const int in = PW == 8 ? 32 * (fo / 2) + 8 * (brow / 4) + 4 * (fo % 2) + brow % 4 : 16 * fo + brow;
      row = min(wb / NBW * NBO * 16 + in, rows_w - 1);
      ld = up ? a.ld_w[1] : a.ld_w[0];
      rs[i] = up ? rw1 : rw0;
    }
    const int skip = into_line(row, ld);
    off[i] = static_cast<uint32_t>(row * ld * 2) - skip * 16 + (block_chunk(lane, half) + skip) % 8 * 16;
  }
  const uint32_t place0 = lds_address(lds) + wave * 1024;
  int next = kt0 + (SHIFT || kt1 <= kt0 ? 0 : first_of(blockIdx.x, kt1 - kt0)), left = SHIFT ? KT + 1 : kt1 - kt0;
  if (SHIFT) {  // lines may go on past the matrix: the offsets whose range is checked are the lanes' whole ones
#pragma unroll
    for (int i = 0; i < LPS; ++i) off[i] += static_cast<uint32_t>(kt0) * (TK * 2);
  }
  // Past the last stage the loads go on with empty ranges (no memory traffic, stages that nobody multiplies), so the
  // counts stay.
  auto load1 = [&](auto I, uint32_t stage) {
    constexpr int i = decltype(I)::value;
    const bool more = left > 0;
    u32x4 r = rs[i];
    r.z = more ? r.z : 0u;
    put_fetch<i * NW * 1024>(place0 + stage, r, off[i], more && !SHIFT ? static_cast<uint32_t>(next) * (TK * 2) : 0u);
    if (SHIFT) off[i] += TK * 2;
  };
  auto advance = [&]() {
    if (++next == kt1 && !SHIFT) next = kt0;
    --left;
  };
  auto load = [&](uint32_t stage) {
    each<LPS>([&](auto I) { load1(I, stage); });
    advance();
  };

  const int kw = wave / (WR * WC), wr = wave / WC % WR, wc = wave % WC;
  f32x4 acc[NBW][MBW];
#pragma unroll
  for (int f = 0; f < NBW; ++f)
#pragma unroll
    for (int b = 0; b < MBW; ++b) acc[f][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (tail && !SHIFT) {  // to stage 0, with zeros past K
#pragma unroll
    for (int i = 0; i < LPS; ++i) {
      const int u = wave + NW * i, k = full * TK + block_chunk(lane, u % 2) * 8;
      const u32x4 v = load_at(rsrc_of(rs[i]), off[i] | (k < a.K ? 0u : kOOB), full * (TK * 2));
      *reinterpret_cast<u32x4*>(lds + u * 1024 + lane * 16) = keep_first(v, a.K - k);
    }
  }
  each<(KW == 2 ? ST : ST - 1)>([&](auto Q) {
    constexpr int q = decltype(Q)::value;
    if (q > 0 || !tail || SHIFT) load(q * STAGE);
  });
  // Where this lane's parts of the fragments are (in the block of their first row, with SHIFT in the ring): of rows,
  // and of the gate's and the up projection's even and odd blocks, for both k-steps.
  uint32_t fx[HS], fw[GATED ? 2 : 1][2][HS];
  auto spot = [&](int row, int64_t ld, int h) {
    const int ks = kw * HS + h, chunk = 4 * ks + lane / 16;
    return static_cast<uint32_t>(lane % 16 / 8 * 1024 + (fragment_at(lane) ^ (ks * 64)) + (chunk + into_line(row, ld)) / 8 * STAGE);
  };
#pragma unroll
  for (int h = 0; h < HS; ++h) {
    const int r = lane % 16;
    fx[h] = spot(r, a.ld_x, h);
#pragma unroll
    for (int m = 0; m < (GATED ? 2 : 1); ++m)
#pragma unroll
      for (int odd = 0; odd < 2; ++odd) fw[m][odd][h] = spot(PW == 8 ? 4 * odd + r % 4 : r, a.ld_w[m], h);
  }
  uint32_t cur = 0;
  auto up = [](uint32_t x) { return x + STAGE == ST * STAGE ? 0u : x + STAGE; };
  auto turn = [](uint32_t& x) { x = min(x + STAGE, x + STAGE - ST * STAGE); };  // (below 0 is large)
  u32x4 xf[2][MBW], wf[2][NBW];
  // fragment i of k-step h of the stage at ``from``
  auto read1 = [&](int i, int set, int h, uint32_t from) {
    const char* at = lds + (SHIFT ? 0u : from);
    if (i < MBW) {
      xf[set][i] = *reinterpret_cast<const u32x4*>(at + fx[h] + (wr * MBW + i) * 2048);
    } else {
      const int f = i - MBW;
      wf[set][f] = *reinterpret_cast<const u32x4*>(at + fw[f / NBO][f % NBO % 2][h] + (XB + wc * NBW + f) * 2048);
    }
  };
  auto turn_all = [&](int h) {
    if (!SHIFT) return;
    turn(fx[h]);
#pragma unroll
    for (int m = 0; m < (GATED ? 2 : 1); ++m) {
      turn(fw[m][0][h]);
      if (NBO > 1) turn(fw[m][1][h]);
    }
  };
  auto read = [&](auto SET, int h, uint32_t from) {
#pragma unroll
    for (int i = 0; i < MBW + NBW; ++i) read1(i, decltype(SET)::value, h, from);
    turn_all(h);
  };
  auto mask = [&](auto SET, int h) {
    constexpr int set = decltype(SET)::value;
    const int keep = a.K - (full * TK + (kw * HS + h) * 32 + lane / 16 * 8);
#pragma unroll
    for (int b = 0; b < MBW; ++b) xf[set][b] = keep_first(xf[set][b], keep);
#pragma unroll
    for (int f = 0; f < NBW; ++f) wf[set][f] = keep_first(wf[set][f], keep);
  };
  auto multiply = [&](auto SET) {
    constexpr int set = decltype(SET)::value;
#pragma unroll
    for (int f = 0; f < NBW; ++f)
#pragma unroll
      for (int b = 0; b < MBW; ++b) acc[f][b] = T::mfma16(wf[set][f], xf[set][b], acc[f][b]);
  };
  auto meet = [&](auto N) {  // all but the newest N stages' loads of this wave have arrived, and its fragments
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LPS * decltype(N)::value) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  using S0 = std::integral_constant<int, 0>;
  using S1 = std::integral_constant<int, 1>;
  const int plain = SHIFT && tail ? KT - 1 : KT;
  if constexpr (KW == 2) {
    constexpr int P = MBW * NBW;
    static_assert(MBW + NBW <= P && LPS <= P, "room beside the products");
    constexpr bool ROOM = 2 * LPS <= P;
    // A stage is one k-step of this wave. The next one's fragments are read beside its products, so its own are in
    // registers when the waves meet, and the stage is free for the loads.
    meet(std::integral_constant<int, SHIFT ? ST - 2 : ST - 1>{});
    read(S0{}, 0, 0);
    auto step = [&](auto SET) {
      meet(std::integral_constant<int, SHIFT ? ST - 3 : ST - 2>{});
      const uint32_t next_stage = up(cur);
      each<P>([&](auto I) {  // a product, and what goes out beside it
        constexpr int i = decltype(I)::value, set = decltype(SET)::value, f = i / MBW, b = i % MBW;
        acc[f][b] = T::mfma16(wf[set][f], xf[set][b], acc[f][b]);
        if constexpr (i == 0) __builtin_amdgcn_sched_barrier(0);  // (else it is made to wait for the first read)
        if constexpr (i < MBW + NBW) read1(i, 1 - set, 0, next_stage);
        if constexpr (ROOM ? i % 2 == 1 && i / 2 < LPS : i >= P - LPS)
          load1(std::integral_constant<int, ROOM ? i / 2 : i - (P - LPS)>{}, cur);
        __builtin_amdgcn_sched_barrier(0);
      });
      turn_all(0);
      advance();
      cur = next_stage;
    };
    int q = 0;
    for (; q + 1 < plain; q += 2) {
      step(S0{});
      step(S1{});
    }
    if (q < plain) step(S0{});
    if (SHIFT && tail) {
      if (q < plain) {
        mask(S1{}, 0);
        multiply(S1{});
      } else {
        mask(S0{}, 0);
        multiply(S0{});
      }
    }
  } else {
    uint32_t into = (ST - 1) * STAGE;
    auto step = [&](auto MASK) {
      meet(std::integral_constant<int, SHIFT ? ST - 3 : ST - 2>{});
      load(into);
      read(S0{}, 0, cur);
      read(S1{}, HS - 1, cur);
      if constexpr (decltype(MASK)::value) {
        mask(S0{}, 0);
        mask(S1{}, HS - 1);
      }
      multiply(S0{});
      multiply(S1{});
      into = cur;
      cur = up(cur);
    };
    for (int q = 0; q < plain; ++q) step(std::false_type{});
    if (SHIFT && tail) step(std::true_type{});
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load is on its way into LDS when a wave ends

  // The result's blocks of this wave: with KW waves on a tile's place each takes a share of the rows, from all.
  f32x4 out[NBW][MBO];
  if constexpr (KW == 2) {
    __syncthreads();  // the ring is free
    auto give = [&](int b0) {
#pragma unroll
      for (int f = 0; f < NBW; ++f)
#pragma unroll
        for (int b = 0; b < MBO; ++b)
          *reinterpret_cast<f32x4*>(lds + (wave * NBW * MBO + f * MBO + b) * 1024 + lane * 16) = acc[f][b0 + b];
    };
    if (kw == 0) give(MBO);
    else give(0);
    __syncthreads();
    const int other = kw ? wave - WR * WC : wave + WR * WC;
    auto take = [&](int b0) {
#pragma unroll
      for (int f = 0; f < NBW; ++f)
#pragma unroll
        for (int b = 0; b < MBO; ++b)
          out[f][b] = acc[f][b0 + b] + *reinterpret_cast<f32x4*>(lds + (other * NBW * MBO + f * MBO + b) * 1024 + lane * 16);
    };
    if (kw == 0) take(0);
    else take(MBO);
  } else {
#pragma unroll
    for (int f = 0; f < NBW; ++f)
#pragma unroll
      for (int b = 0; b < MBO; ++b) out[f][b] = acc[f][b];
  }
  if (a.splits > 1 && !join<NBW, MBO, NW>(a, out, lds, m_tile * a.n_tiles + n_tile, split, wave, lane)) return;

#pragma unroll
  for (int b = 0; b < MBO; ++b) {
    const int m = m0 + (wr * MBW + kw * MBO + b) * 16 + lane % 16;
    if (m >= a.M) continue;
#pragma unroll
    for (int f = 0; f < NBO; f += PW / 4) {
      const int n = n0 + (wc * NBO + f) * 16 + lane / 16 * PW;
      if (n >= a.N) continue;
      float z[PW], u[PW];
#pragma unroll
      for (int e = 0; e < PW; ++e) {
        z[e] = out[f + e / 4][b][e % 4];
        u[e] = GATED ? out[NBO + f + e / 4][b][e % 4] : 0.f;
      }
      finish<T, GATED, PW>(a, m, n, z, u);
    }
  }
}

namespace {

struct Kernel {
  void (*run[4])(Args);  // fp16, fp16 gated, bf16, bf16 gated
  int threads, lds;
};

template <int WR, int WC, int KW, int MBW, int NBW, int ST, bool SHIFT>
constexpr Kernel kernel() {
  return {{mid_kernel<Half, false, WR, WC, KW, MBW, NBW, ST, SHIFT>, mid_kernel<Half, true, WR, WC, KW, MBW, NBW, ST, SHIFT>,
           mid_kernel<BFloat, false, WR, WC, KW, MBW, NBW, ST, SHIFT>, mid_kernel<BFloat, true, WR, WC, KW, MBW, NBW, ST, SHIFT>},
          WR * WC * KW * kWave,
          ST * 2 * (WR * MBW + WC * NBW) * 1024};
}

// in the order of kMid, rows at lines and not
const Kernel kKernels[][2] = {{kernel<1, 2, 1, 1, 2, 5, false>(), kernel<1, 2, 1, 1, 2, 6, true>()},
                              {kernel<1, 2, 2, 2, 2, 4, false>(), kernel<1, 2, 2, 2, 2, 5, true>()},
                              {kernel<2, 2, 2, 2, 2, 4, false>(), kernel<2, 2, 2, 2, 2, 5, true>()},
                              {kernel<2, 2, 2, 2, 4, 4, false>(), kernel<2, 2, 2, 2, 4, 5, true>()},
                              {kernel<2, 2, 2, 4, 4, 4, false>(), kernel<2, 2, 2, 4, 4, 5, true>()}};

}  // namespace

hipError_t launch_mid(const Args& a, int which, bool shift, bool bf16, bool gated, hipStream_t s) {
  static LdsOnce once;
  const hipError_t e = once([](auto&& raise) {
    for (const auto& pair : kKernels)
      for (const Kernel& k : pair)
        for (auto* f : k.run) raise(reinterpret_cast<const void*>(f), k.lds);
  });
  if (e != hipSuccess) return e;
  const Kernel& k = kKernels[which][shift];
  hipLaunchKernelGGL(k.run[2 * bf16 + gated], dim3(static_cast<uint32_t>(grid_of(a.m_tiles, a.n_tiles * a.splits))),
                     dim3(k.threads), k.lds, s, a);
  return hipGetLastError();
}

}  // namespace lin
}  // namespace vt
