// Attention of few query rows over a paged cache: single tokens and short chunks.
//
// A tile is 16 rows of one KV head: the query heads that share it, for one token
// or several. Both products run on the matrix cores in the orientation that moves no
// data between lanes. For 32 keys p of a head,
//   S^T = K Q^T   (two 16 x 16 tiles: lane l has row l % 16, keys 4 (l / 16) + r)
//   O^T = V^T P^T (A and B operands of one lane are 8 numbers of its 16th column or
//                  row, along the summed index)
// and the summed index of the second product may be in any order: taking 4 (l / 16) + r
// of the first tile, then of the second, a lane's own weights are its B operand. V's
// operand is 8 keys of one element per lane; a lane loads 8 consecutive elements of
// each of its 8 keys (16 lanes have a row, 256 bytes) and turns its 8 x 8 numbers in
// registers, so neither K nor V passes through LDS.
//
// The weights are exp2(s - ref), ref a row's reference that follows its maximum seldom (kLag,
// kTop). A weight enters the product as its rounding and the rounding of the remainder (two
// products; the matrix cores have the time): the output's error is then that of its own
// rounding, and for fp16 up to 2^-32 of the largest value per key that the wave takes.
//
// What bounds it: every key and value is read once per tile, from HBM. A wave loads
// the next 32 keys and values (16 KiB) while it works on these. Measured: 64 sequences of
// 2061-4097 positions, 64 query heads on 8 KV heads of 128, fp16: 151-153 us for 818 MB, 5.4 TB/s (HBM
// reads by the counters 819 MB, matrix cores busy 5%); 125 ragged ones of up to 2053, 32 heads, bf16: 418-430
// us for 2.29 GB, 5.3-5.5 TB/s; one of 131071, 8-bit: 55-57 us for 268 MB, 4.7-4.9 TB/s. A 4 GiB device
// copy moves 4.7-4.9 TB/s. For short ones the chain lengths -> split -> page -> keys -> join
// bounds it: one sequence of 129 positions 5.9 us in a captured graph, of 4096 11.1.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "paged.hpp"

namespace vt {
namespace pg {

constexpr int RT = 256, RW = RT / kWave;  // threads and waves
constexpr int ROWS = 16, TK = 32;         // rows of a tile, keys of a wave's step
constexpr int RB = TK * RW;               // keys of a block

using RowPlan = Plan<ROWS, RB, RT>;

__device__ __forceinline__ void store_coherent(rsrc_t r, uint32_t off, f32x4 v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, off, 0, kCoherent);
}

__device__ __forceinline__ f32x4 load_coherent(rsrc_t r, uint32_t off) {
  return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, kCoherent));
}

// A partial result in the workspace: [ROWS][D] outputs, then a reference and a sum per row.
template <int D>
struct Part {
  static constexpr uint32_t kBytes = ROWS * (D + 2) * 4;
  static_assert(kBytes <= part_bytes(ROWS, D), "");
  static __device__ __forceinline__ uint32_t out(int row, int e) { return (row * D + e) * 4; }
  static __device__ __forceinline__ uint32_t stats(int row) { return (ROWS * D + 2 * row) * 4; }
};

// One wave's 32 keys and values as they were loaded, and which of them are not there.
template <bool F8, int D>
struct Tile {
  static constexpr int KV = D / 32 * (F8 ? 2 : 4);  // words of a lane's part of a key
  static constexpr int VV = D / 32 / (F8 ? 2 : 1);  // words of a lane's part of a value: D / 16 numbers
  uint32_t k[2][KV];
  uint32_t v[8][VV];
  uint32_t bad;  // bit 4 t + r: key 16 t + 4 (l / 16) + r is on a bad page
};

template <int N>
__device__ __forceinline__ void load_words(uint32_t* to, const char* p) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(p + i * 64);
#pragma unroll
      for (int e = 0; e < 4; ++e) to[4 * i + e] = w[e];
    }
  } else if constexpr (N == 2) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(p);
    to[0] = w[0];
    to[1] = w[1];
  } else {
    to[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// Pages of a wave's 32 keys. BIG (page_size >= 16): one per 16 keys, the same for all
// lanes; else one for each of a lane's keys.
template <bool BIG>
struct Pages {
  int32_t k[2];
  int32_t v[BIG ? 1 : 8];
};

template <class T, bool F8, int D, bool BIG>
__global__ void __launch_bounds__(RT, 2) attn_rows_kernel(AttnArgs a) {
  constexpr int NK = D / 32, NM = D / 16;  // steps of the first product, tiles of the second
  constexpr int MLD = D + 4;               // a row of the merge buffer
  __shared__ __attribute__((aligned(16))) float merge[RW][ROWS * MLD];
  __shared__ float merge_ref[RW][ROWS], merge_sum[RW][ROWS];
  __shared__ int lds[32];
  static_assert(kItemWords <= 32 && 10 * RT <= RW * ROWS * MLD, "");
  const int lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (blockIdx.x == 0 && a.p.status)
    for (int s = threadIdx.x; s < a.p.n_seqs; s += RT)
      if (a.p.len[s] > a.p.capacity) sync_or(a.p.status, VT_PAGED_BAD_LEN);

  Item it;
  if (!next_item<RowPlan>(a, blockIdx.x, it, lds)) return;
  const Seq& q = it.q;
  // this lane's row: query head it.head * group + j of token tok
  const int rows = q.nt * a.group;
  const int row = min(it.tile * ROWS + n, rows - 1), tok = row / a.group, j = row - tok * a.group;
  const bool there = it.tile * ROWS + n < rows;
  const int pos = q.pos0 + tok;  // its keys: klo <= p < khi
  const int khi = min(pos + 1, q.keys), klo = a.window > 0 ? max(pos, 0) - (a.window - 1) : 0;
  // keys that every row sees lie in full_lo .. full_hi - 1, those of any row below any_hi
  int full_hi = khi, full_lo = klo, any_hi = khi, any_lo = klo;
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    full_hi = min(full_hi, __shfl_xor(full_hi, o, kWave));
    full_lo = max(full_lo, __shfl_xor(full_lo, o, kWave));
    any_hi = max(any_hi, __shfl_xor(any_hi, o, kWave));
    any_lo = min(any_lo, __shfl_xor(any_lo, o, kWave));
  }
  full_hi = __builtin_amdgcn_readfirstlane(full_hi);
  full_lo = __builtin_amdgcn_readfirstlane(full_lo);
  any_hi = __builtin_amdgcn_readfirstlane(any_hi);
  any_lo = __builtin_amdgcn_readfirstlane(max(any_lo, 0));

  // the piece's blocks; this wave takes 32 keys of each
  const int b0 = it.block0 + static_cast<int>(static_cast<int64_t>(it.blocks) * it.piece / it.pieces);
  const int b1 = it.block0 + static_cast<int>(static_cast<int64_t>(it.blocks) * (it.piece + 1) / it.pieces);
  const int first = b0 * RB + wave * TK;
  int steps = b1 - b0;
  // past the tile's last key (never below the first: that is block 0's)
  if (steps > 0) steps = max(0, min(steps, (any_hi - first + RB - 1) / RB));
  const int skip = any_lo >= first + TK ? (any_lo - first - TK) / RB + 1 : 0;  // before its first key
  const char* kb = a.p.k + it.head * a.p.head;
  const char* vb = a.p.v + it.head * a.p.head;
  const ConstInt* tab = constant(a.p.table + it.s * a.p.ld_table);
  const uint32_t slot = static_cast<uint32_t>(a.p.slot);
  const int last = q.keys - 1;  // no position past it is read or looked up

  u32x4 qf[NK];
  {
    const uint16_t* qp = a.q + (q.b + tok) * a.ld_q + (static_cast<int64_t>(it.head) * a.group + j) * D;
#pragma unroll
    for (int s = 0; s < NK; ++s)
      // elements as the lane's key words hold them: an 8-bit load of 16 numbers feeds two steps
      qf[s] = load16(qp + (F8 ? (s / 2) * 64 + g * 16 + (s % 2) * 8 : s * 32 + g * 8));
  }
  const float ks = F8 && a.p.k_scale ? a.p.k_scale[it.head] : 1.f;
  const float sc = a.scale2 * ks;

  f32x4 o[NM];
#pragma unroll
  for (int m = 0; m < NM; ++m) o[m] = f32x4{0.f, 0.f, 0.f, 0.f};
  float ref = -INFINITY, sum = 0.f;

  auto start = [&](int i) { return first + min(i, steps - 1) * RB; };
  auto look = [&](int i, Pages<BIG>& pg) {
    const int p0 = start(i);
#pragma unroll
    for (int t = 0; t < 2; ++t)
      pg.k[t] = tab[min(p0 + 16 * t + (BIG ? 0 : n), last) >> a.p.shift];
    if constexpr (!BIG)
#pragma unroll
      for (int e = 0; e < 8; ++e) pg.v[e] = tab[min(p0 + 16 * (e / 4) + 4 * g + e % 4, last) >> a.p.shift];
  };
  auto load = [&](int i, const Pages<BIG>& pg, Tile<F8, D>& x) {
    const int p0 = start(i);
    x.bad = 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int key = min(p0 + 16 * t, last);  // of the tile's first row
      const bool ok = pg.k[t] >= 0 && pg.k[t] < a.p.n_pages;
      const int64_t page = static_cast<int64_t>(ok ? pg.k[t] : 0) * a.p.page;
      if constexpr (BIG) {
        const int64_t base = page + static_cast<int64_t>(key & a.p.mask) * a.p.slot;
        const int most = last - key;  // rows past the last position read that one again
        load_words<Tile<F8, D>::KV>(x.k[t], kb + base + static_cast<uint32_t>(min(n, most)) * slot + g * 16);
#pragma unroll
        for (int r = 0; r < 4; ++r)
          load_words<Tile<F8, D>::VV>(x.v[4 * t + r], vb + base + static_cast<uint32_t>(min(4 * g + r, most)) * slot +
                                                          n * Tile<F8, D>::VV * 4);
        if (!ok) x.bad |= 0xFu << (4 * t);
      } else {
        const int mine = min(p0 + 16 * t + n, last);
        load_words<Tile<F8, D>::KV>(x.k[t], kb + page + static_cast<int64_t>(mine & a.p.mask) * a.p.slot + g * 16);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int e = 4 * t + r, vk = min(p0 + 16 * t + 4 * g + r, last);
          const bool vok = pg.v[e] >= 0 && pg.v[e] < a.p.n_pages;
          load_words<Tile<F8, D>::VV>(x.v[e], vb + static_cast<int64_t>(vok ? pg.v[e] : 0) * a.p.page +
                                                  static_cast<int64_t>(vk & a.p.mask) * a.p.slot +
                                                  n * Tile<F8, D>::VV * 4);
          if (!vok) x.bad |= 1u << e;
        }
      }
    }
  };
  auto work = [&](int i, Tile<F8, D>& x) {
#pragma clang fp contract(off)  // weights are those of the rounded scores, as the reference is
    const int p0 = start(i);
    f32x4 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NK; ++c) {
        u32x4 kf;
        if constexpr (F8) {
          const uint32_t w0 = x.k[t][2 * c], w1 = x.k[t][2 * c + 1];
          kf = u32x4{T::template from_f8<false>(w0), T::template from_f8<true>(w0), T::template from_f8<false>(w1),
                     T::template from_f8<true>(w1)};
        } else {
          kf = u32x4{x.k[t][4 * c], x.k[t][4 * c + 1], x.k[t][4 * c + 2], x.k[t][4 * c + 3]};
        }
        s[t] = T::mfma16(kf, qf[c], s[t]);
      }
    }
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = s[e / 4][e % 4] * sc;
    const bool bad = BIG ? x.bad != 0 : __builtin_amdgcn_ballot_w64(x.bad != 0) != 0;
    const bool edge = bad || p0 < full_lo || p0 + TK > full_hi;
    // this lane's 8 keys, the pairs of V's words below
    auto key = [&](int e) { return p0 + 16 * (e / 4) + 4 * g + e % 4; };
    if (edge) {
      if (bad && a.p.status) {
        bool seen = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) seen |= (x.bad >> e & 1) && there && key(e) >= klo && key(e) < khi;
        if (seen) sync_or(a.p.status, VT_PAGED_BAD_PAGE);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (key(e) < klo || key(e) >= khi || (x.bad >> e & 1)) y[e] = -INFINITY;
        // values that no row sees stay out of the product even if they are infinite
        if (key(e) < any_lo || key(e) >= any_hi || (x.bad >> e & 1))
#pragma unroll
          for (int w = 0; w < Tile<F8, D>::VV; ++w) x.v[e][w] = 0;
      }
    }
    float top = y[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, y[e]);
    if (__builtin_amdgcn_ballot_w64(top - ref > T::kTop + kLag) != 0) {
      top = fmaxf(top, __shfl_xor(top, 16, kWave));
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      const float next = fmaxf(top - T::kTop, ref);
      const float alpha = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref - next);
      ref = next;
      sum *= alpha;
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[m][r] *= alpha;
    }
    const float base = ref == -INFINITY ? 0.f : ref;
    float all = 0.f;  // of this step: small weights together before they join a sum that may be large
    u32x4 hi, lo;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float pa = __builtin_amdgcn_exp2f(y[2 * w] - base), pb = __builtin_amdgcn_exp2f(y[2 * w + 1] - base);
      all += pa + pb;
      hi[w] = T::pack2(pa, pb);
      float ra, rb;
      T::unpack2(hi[w], ra, rb);
      lo[w] = T::pack2(pa - ra, pb - rb);
    }
    sum += all;
    // V's operands: element m of the lane's 8 keys. Words w of keys 2 i, 2 i + 1 hold
    // elements 2 w, 2 w + 1 (8-bit: 4 w .. 4 w + 3)
    u32x4 vf[NM];
#pragma unroll
    for (int i2 = 0; i2 < 4; ++i2)
#pragma unroll
      for (int w = 0; w < Tile<F8, D>::VV; ++w) {
        const uint32_t va = x.v[2 * i2][w], vb2 = x.v[2 * i2 + 1][w];
        if constexpr (F8) {
          const uint32_t e01 = __builtin_amdgcn_perm(vb2, va, 0x05010400), e23 = __builtin_amdgcn_perm(vb2, va, 0x07030602);
          vf[4 * w][i2] = T::template from_f8<false>(e01);
          vf[4 * w + 1][i2] = T::template from_f8<true>(e01);
          vf[4 * w + 2][i2] = T::template from_f8<false>(e23);
          vf[4 * w + 3][i2] = T::template from_f8<true>(e23);
        } else {
          vf[2 * w][i2] = __builtin_amdgcn_perm(vb2, va, 0x05040100);
          vf[2 * w + 1][i2] = __builtin_amdgcn_perm(vb2, va, 0x07060302);
        }
      }
    if (edge) {
      bool odd = false;
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int w = 0; w < 4; ++w) odd |= odd2<T>(vf[m][w]);
      if (__builtin_amdgcn_ballot_w64(odd) != 0) {
        // an infinite or NaN value that some rows see and others do not: a product for
        // each row with what that row does not see set to zero
#pragma unroll
        for (int m = 0; m < NM; ++m) {
          f32x4 keep = o[m];
#pragma unroll 1
          for (int c = 0; c < ROWS; ++c) {
            const int lo_c = __builtin_amdgcn_readlane(klo, c), hi_c = __builtin_amdgcn_readlane(khi, c);
            u32x4 z = vf[m];
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (key(e) < lo_c || key(e) >= hi_c) z[e / 2] &= e % 2 ? 0x0000FFFFu : 0xFFFF0000u;
            const f32x4 r = T::mfma16(z, lo, T::mfma16(z, hi, o[m]));
            if (n == c) keep = r;
          }
          o[m] = keep;
        }
        return;
      }
    }
#pragma unroll
    for (int m = 0; m < NM; ++m) o[m] = T::mfma16(vf[m], hi, o[m]);
#pragma unroll
    for (int m = 0; m < NM; ++m) o[m] = T::mfma16(vf[m], lo, o[m]);
  };

  if (skip < steps) {
    Tile<F8, D> xa, xb;
    Pages<BIG> pa, pb;
    look(skip, pa);
    look(skip + 1, pb);
    load(skip, pa, xa);
    for (int c = skip; c < steps; c += 2) {
      look(c + 2, pa);
      load(c + 1, pb, xb);
      work(c, xa);
      if (c + 1 >= steps) break;
      look(c + 3, pb);
      load(c + 2, pa, xa);
      work(c + 1, xb);
    }
  }
  sum += __shfl_xor(sum, 16, kWave);
  sum += __shfl_xor(sum, 32, kWave);

  // the waves' results together: lane's element m of tile m is D / 16 (4 g + r) + m
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int m = 0; m < NM; m += 4)
      *reinterpret_cast<f32x4*>(&merge[wave][n * MLD + (4 * g + r) * NM + m]) =
          f32x4{o[m][r], o[m + 1][r], o[m + 2][r], o[m + 3][r]};
  if (g == 0) {
    merge_ref[wave][n] = ref;
    merge_sum[wave][n] = sum;
  }
  __syncthreads();
  constexpr int CPR = D / 8;  // threads of a row, 8 elements each
  const int here = min(ROWS, rows - it.tile * ROWS);  // rows of this tile
  int mr = threadIdx.x / CPR, me = threadIdx.x % CPR * 8;
  bool writes = mr < here;
  float acc[8], top = -INFINITY, total = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  if (writes) {
#pragma unroll
    for (int w = 0; w < RW; ++w) top = fmaxf(top, merge_ref[w][mr]);
#pragma unroll
    for (int w = 0; w < RW; ++w) {
      const float r = merge_ref[w][mr], f = r == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(r - top);
      total += f * merge_sum[w][mr];
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += f * merge[w][mr * MLD + me + e];
    }
  }
  bool finish = true;
  if (it.pieces > 1) {
    const rsrc_t ru = make_rsrc(reinterpret_cast<char*>(a.part) + static_cast<int64_t>(it.slot) * Part<D>::kBytes,
                                it.pieces * Part<D>::kBytes);
    const uint32_t mine = it.piece * Part<D>::kBytes;
    if (writes) {
      store_coherent(ru, mine + Part<D>::out(mr, me), f32x4{acc[0], acc[1], acc[2], acc[3]});
      store_coherent(ru, mine + Part<D>::out(mr, me + 4), f32x4{acc[4], acc[5], acc[6], acc[7]});
      if (me == 0)
        __builtin_amdgcn_raw_buffer_store_b64(
            u32x2{__builtin_bit_cast(uint32_t, top), __builtin_bit_cast(uint32_t, total)}, ru, mine + Part<D>::stats(mr), 0,
            kCoherent);
    }
    mem_done();
    __syncthreads();
    if (threadIdx.x == 0)
      lds[0] = __hip_atomic_fetch_add(a.arrived + it.unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
               static_cast<uint32_t>(it.pieces - 1);
    __syncthreads();
    // the last piece to arrive joins them all, in their order: the result does not
    // depend on which one that is
    finish = lds[0] != 0;
    if (finish) {
      if (threadIdx.x == 0) sync_store(a.arrived + it.unit, 0u);
      // The threads of a row are CPR; what there are more of them than the tile's rows take
      // (n times) share the pieces, each adding up every n-th one, eight of them (their
      // references, sums and outputs) on their way at once.
      int rp = 1;
      while (rp < here) rp *= 2;
      const int n = RT / (CPR * rp), first_piece = threadIdx.x / (CPR * rp);
      mr = threadIdx.x / CPR % rp;
      top = -INFINITY;
      total = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = 0.f;
      if (mr < here)
        for (int c0 = first_piece; c0 < it.pieces; c0 += 8 * n) {
          float r[8], t[8];
          f32x4 u[8], v[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {  // pieces past the last one are out of the range: zeros
            const uint32_t at = (c0 + k * n) * Part<D>::kBytes;
            buf_ld_shared2(ru, at + Part<D>::stats(mr), r[k], t[k]);
            u[k] = load_coherent(ru, at + Part<D>::out(mr, me));
            v[k] = load_coherent(ru, at + Part<D>::out(mr, me + 4));
          }
          float next = top;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            if (c0 + k * n >= it.pieces) r[k] = -INFINITY;
            next = fmaxf(next, r[k]);
          }
          const float base = next == -INFINITY ? 0.f : next, f0 = __builtin_amdgcn_exp2f(top - base);
          total *= f0;
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] *= f0;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float f = __builtin_amdgcn_exp2f(r[k] - base);
            total += f * t[k];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              acc[e] += f * u[k][e];
              acc[4 + e] += f * v[k][e];
            }
          }
          top = next;
        }
      writes = mr < here && first_piece == 0;
      if (n > 1) {
        float* own = &merge[0][0] + threadIdx.x * 10;
#pragma unroll
        for (int e = 0; e < 8; ++e) own[e] = acc[e];
        own[8] = top;
        own[9] = total;
        __syncthreads();
        if (writes) {
          for (int w = 1; w < n; ++w) top = fmaxf(top, own[w * CPR * rp * 10 + 8]);
          const float base = top == -INFINITY ? 0.f : top;
          total = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] = 0.f;
          for (int w = 0; w < n; ++w) {
            const float* x = own + w * CPR * rp * 10;
            const float f = __builtin_amdgcn_exp2f(x[8] - base);
            total += f * x[9];
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] += f * x[e];
          }
        }
      }
    }
  }
  const int out_row = it.tile * ROWS + mr;
  if (finish && writes) {
    const int tk = out_row / a.group, hd = it.head * a.group + out_row - tk * a.group;
    const float vs = F8 && a.p.v_scale ? a.p.v_scale[it.head] : 1.f;
    const float inv = total == 0.f ? 0.f : vs / total;
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = T::pack2(acc[2 * e] * inv, acc[2 * e + 1] * inv);
    *reinterpret_cast<u32x4*>(a.out + (q.b + tk) * a.ld_out + static_cast<int64_t>(hd) * D + me) = w;
    if (a.lse && me == 0)
      a.lse[static_cast<int64_t>(q.b + tk) * a.n_q + hd] =
          total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
  }
}

hipError_t launch_rows(const AttnArgs& a, int type, bool f8, int head_dim, hipStream_t s) {
  const bool big = a.p.mask + 1 >= 16;
  auto pick = [&](auto X) -> void (*)(AttnArgs) {
    using T = decltype(X);
    if (head_dim == 128) {
      if (f8) return big ? attn_rows_kernel<T, true, 128, true> : attn_rows_kernel<T, true, 128, false>;
      return big ? attn_rows_kernel<T, false, 128, true> : attn_rows_kernel<T, false, 128, false>;
    }
    if (f8) return big ? attn_rows_kernel<T, true, 64, true> : attn_rows_kernel<T, true, 64, false>;
    return big ? attn_rows_kernel<T, false, 64, true> : attn_rows_kernel<T, false, 64, false>;
  };
  auto* kernel = type == VT_T_F16 ? pick(Half{}) : pick(BFloat{});
  static_assert(ROWS == 16 && RB == 128, "grid_of counts these");
  hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(grid_of(a, ROWS))), dim3(RT), 0, s, a);
  return hipGetLastError();
}

}  // namespace pg
}  // namespace vt
