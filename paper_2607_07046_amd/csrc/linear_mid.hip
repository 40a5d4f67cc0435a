// Products of a batch's or a short prompt's rows: vt_linear and vt_linear_gated on tiles between those of
// linear_thin.hip and linear_tile.hip.
//
// WR x WC waves of 16 MBW rows x 16 NBW weight rows each. Both operands come straight into LDS through a
// ring of ST stages of 64 k, up to ST - 1 of them on the way, each number once per tile; the
// waves wait for a stage by the count of their own loads and meet once per stage. Two workgroups
// share a compute unit, so one multiplies while the other waits.
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
// What bounds it: up to about 64 rows reading the weights, above it LDS (at 128 x 128 its reads and the loads' writes take
// 768 cycles of a stage, the products 512). Measured in bf16: 64 rows of 8192 through the gate and up projections of
// 7168 features 48 to 55 us, 4.3 to 4.9 TB/s; rows of 4096 through 4096 features: 256 rows 18 us (474 TFLOP/s),
// 512 25 (676), 1024 40 (853); 777 rows of 3302 to 4096 with a residual 39 to 43, 30 at 3328. Rows that do not start at
// 128-byte lines cost that: half of each line is fetched again for the next stage. Tried for them and not kept, since
// each lost more elsewhere: whole lines into LDS and fragments from two stages (64 rows through 14336 features 32
// us, not 39, but 20 to 60% slower wherever the weights were in the caches), and two stages' loads together (777 rows 38,
// not 42, other sizes 2 to 15% slower). 64 x 64 per wave on the large tile's schedule: 0 to 8% faster than 128 x 128 here.
#include "linear_lds.hpp"

namespace vt {
namespace lin {

template <class T, bool GATED, int WR, int WC, int MBW, int NBW, int ST>
__global__ void __launch_bounds__(WR* WC* kWave) mid_kernel(Args a) {
  constexpr int NW = WR * WC, XB = WR * MBW, WB = WC * NBW;  // waves; 16-row blocks of rows and of weights
  constexpr int U = 2 * (XB + WB), LPS = U / NW;              // units (8 rows x 64 k) of a stage, loads of a wave
  constexpr int NBO = GATED ? NBW / 2 : NBW;                 // 16-feature blocks of a wave
  constexpr int TM = 16 * XB, TN = 16 * WC * NBO, TK = 64, STAGE = U * 1024, PW = NBO % 2 ? 4 : 8;
  static_assert(U % NW == 0 && (!GATED || NBW % 2 == 0), "");
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
  const u32x4 rx = rsrc_words(a.x + m0 * a.ld_x, static_cast<uint32_t>(rows_x * a.ld_x * 2));
  const u32x4 rw0 = rsrc_words(a.w[0] + n0 * a.ld_w[0], static_cast<uint32_t>(rows_w * a.ld_w[0] * 2));
  const u32x4 rw1 = GATED ? rsrc_words(a.w[1] + n0 * a.ld_w[1], static_cast<uint32_t>(rows_w * a.ld_w[1] * 2)) : rw0;
  u32x4 rs[LPS];
  uint32_t off[LPS];
#pragma unroll
  for (int i = 0; i < LPS; ++i) {
    const int v = wave + NW * i, b = v / 2, half = v % 2, brow = 8 * half + block_row(lane);
    if (b < XB) {
      rs[i] = rx;
      off[i] = static_cast<uint32_t>(min(16 * b + brow, rows_x - 1) * a.ld_x * 2);
    } else {
      const int wb = b - XB, fb = wb % NBW, fo = fb % NBO;
      const bool up = GATED && fb >= NBO;
      const int in = PW == 8 ? 32 * (fo / 2) + 8 * (brow / 4) + 4 * (fo % 2) + brow % 4 : 16 * fo + brow;
      const int row = min(wb / NBW * NBO * 16 + in, rows_w - 1);
      rs[i] = up ? rw1 : rw0;
      off[i] = static_cast<uint32_t>(row * (up ? a.ld_w[1] : a.ld_w[0]) * 2);
    }
    off[i] += block_chunk(lane, half) * 16;
  }
  const uint32_t place0 = lds_address(lds) + wave * 1024;
  int next = kt0, left = kt1 - kt0;
  // Past the last stage the loads go on with empty ranges from offset 0 (no memory traffic, stages that nobody
  // reads), so the counts stay.
  auto load = [&](uint32_t stage) {
    const bool more = left > 0;
    const uint32_t at = more ? static_cast<uint32_t>(next) * (TK * 2) : 0u;
    each<LPS>([&](auto I) {
      constexpr int i = decltype(I)::value;
      u32x4 r = rs[i];
      r.z = more ? r.z : 0u;
      put_fetch<i * NW * 1024>(place0 + stage, r, off[i], at);
    });
    ++next;
    --left;
  };

  const int wr = wave / WC, wc = wave % WC, fa = lane % 16 / 8 * 1024 + fragment_at(lane);
  f32x4 acc[NBW][MBW];
#pragma unroll
  for (int f = 0; f < NBW; ++f)
#pragma unroll
    for (int b = 0; b < MBW; ++b) acc[f][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (tail) {  // to stage 0, with zeros past K
#pragma unroll
    for (int i = 0; i < LPS; ++i) {
      const int u = wave + NW * i, k = full * TK + block_chunk(lane, u % 2) * 8;
      const u32x4 v = load_at(rsrc_of(rs[i]), off[i] | (k < a.K ? 0u : kOOB), full * (TK * 2));
      *reinterpret_cast<u32x4*>(lds + u * 1024 + lane * 16) = keep_first(v, a.K - k);
    }
  }
  each<ST - 1>([&](auto Q) {
    constexpr int q = decltype(Q)::value;
    if (q > 0 || !tail) load(q * STAGE);
  });
  uint32_t cur = 0, into = (ST - 1) * STAGE;
  for (int q = 0; q < KT; ++q) {
    // all but the newest ST - 2 stages' loads of this wave, and its reads of the stage before
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LPS * (ST - 2)) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    load(into);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char* S = lds + cur + (fa ^ (h * 64));
      u32x4 xf[MBW], wf[NBW];
#pragma unroll
      for (int b = 0; b < MBW; ++b) xf[b] = *reinterpret_cast<const u32x4*>(S + (wr * MBW + b) * 2048);
#pragma unroll
      for (int f = 0; f < NBW; ++f) wf[f] = *reinterpret_cast<const u32x4*>(S + (XB + wc * NBW + f) * 2048);
#pragma unroll
      for (int f = 0; f < NBW; ++f)
#pragma unroll
        for (int b = 0; b < MBW; ++b) acc[f][b] = T::mfma16(wf[f], xf[b], acc[f][b]);
    }
    into = cur;
    cur = cur + STAGE == ST * STAGE ? 0 : cur + STAGE;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load is on its way into LDS when a wave ends

  if (a.splits > 1 && !join<NBW, MBW, NW>(a, acc, lds, m_tile * a.n_tiles + n_tile, split, wave, lane)) return;

#pragma unroll
  for (int b = 0; b < MBW; ++b) {
    const int m = m0 + (wr * MBW + b) * 16 + lane % 16;
    if (m >= a.M) continue;
#pragma unroll
    for (int f = 0; f < NBO; f += PW / 4) {
      const int n = n0 + (wc * NBO + f) * 16 + lane / 16 * PW;
      if (n >= a.N) continue;
      float z[PW], u[PW];
#pragma unroll
      for (int e = 0; e < PW; ++e) {
        z[e] = acc[f + e / 4][b][e % 4];
        u[e] = GATED ? acc[NBO + f + e / 4][b][e % 4] : 0.f;
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

template <int WR, int WC, int MBW, int NBW, int ST>
constexpr Kernel kernel() {
  return {{mid_kernel<Half, false, WR, WC, MBW, NBW, ST>, mid_kernel<Half, true, WR, WC, MBW, NBW, ST>,
           mid_kernel<BFloat, false, WR, WC, MBW, NBW, ST>, mid_kernel<BFloat, true, WR, WC, MBW, NBW, ST>},
          WR * WC * kWave,
          ST * 2 * (WR * MBW + WC * NBW) * 1024};
}

// in the order of kMid
const Kernel kKernels[] = {kernel<1, 2, 1, 2, 5>(), kernel<2, 2, 1, 2, 4>(), kernel<4, 2, 1, 2, 4>(),
                           kernel<4, 2, 1, 4, 4>(), kernel<4, 2, 2, 4, 4>()};

}  // namespace

hipError_t launch_mid(const Args& a, int which, bool bf16, bool gated, hipStream_t s) {
  static LdsOnce once;
  const hipError_t e = once([](auto&& raise) {
    for (const Kernel& k : kKernels)
      for (auto* f : k.run) raise(reinterpret_cast<const void*>(f), k.lds);
  });
  if (e != hipSuccess) return e;
  const Kernel& k = kKernels[which];
  hipLaunchKernelGGL(k.run[2 * bf16 + gated], dim3(static_cast<uint32_t>(grid_of(a.m_tiles, a.n_tiles * a.splits))),
                     dim3(k.threads), k.lds, s, a);
  return hipGetLastError();
}

}  // namespace lin
}  // namespace vt
