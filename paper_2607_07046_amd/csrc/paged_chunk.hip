// Attention of many query rows over a paged cache: chunks of prompts.
//
// A workgroup of four waves takes a tile of rows of one KV head (a row is one query
// head of one token, the heads that share the KV head side by side), a wave 32 rows.
// Keys and values come in stages of 64 into LDS, once for all rows of the tile: 16-bit
// caches straight from memory, 8-bit ones through registers, where they are widened. Both
// products run as
//   S^T = K Q^T, O^T = V^T P^T on 32 x 32 x 16 matrix instructions:
// a lane has one row (l % 32) of every result, so the softmax needs other lanes only for
// a new maximum, and its weights are the second product's operand as they stand, if
// the key rows of the first are taken in the order with bits 2 and 3 swapped.
//
// LDS rows hold D numbers in 16-byte chunks, chunk c of row r at c ^ (r % CPR) for K,
// whose fragments take one chunk of 32 rows, and at c ^ 2 (r % (CPR / 2)) for V, whose
// transposing reads take two chunks of four rows.
//
// Weights are exp2(s - ref), ref a row's reference that follows the maximum seldom (kLag, kTop);
// they enter the product rounded once, as much as the output itself is (for fp16 also off by up to
// 2^-32 of the largest value per key).
//
// What bounds it: no one pipe. A stage is 1024 cycles of matrix instructions for a wave and about as many
// of vector ones (exponentials, packing), and a SIMD has two waves; for a prompt of 4096 tokens the two
// take about 5300 cycles for their stages, more than both pipes' work in a row. A's scores
// and B's product stand alone in their wave, the two waves keep no phase, and a third of the LDS's busy cycles
// are bank conflicts. Measured (LDS conflicts / active, matrix cores busy): that prompt, 32 heads, fp16, 173-187 us,
// 735-795 TFLOP/s (0.32, 36%); ragged prompts of up to 1999 with a window of 1024, group 4, 163-172 us (0.32, 30%); 512
// tokens per head behind 32768 positions with 8-bit numbers 572-600 us, 925-970 (0.39, 40%); a prompt of
// 8192, 32 query heads on 8, bf16, 558-569 us, 967-985 (the library's products of 8192^3 of such numbers 1280-1380).
// The clock falls from 2.5 to 2.0-2.1 GHz.
// Whole blocks of keys take an inner loop without masks, in which one block's weights stand between another's
// products; with the masks inside 617 and 196 us for prompts of 8192 and 4096 tokens. At head size 128 the 8-bit
// kernels keep 17-40 registers, and the 16-bit ones with pages below 16 positions 12-19, in scratch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "paged.hpp"

namespace vt {
namespace pg {

constexpr int CW = 4, CTH = CW * kWave;  // waves, threads
constexpr int KS = 64;                   // keys of a stage

typedef short v4h16 __attribute__((ext_vector_type(4)));

// In each group of 16 lanes, lane j reads 4 numbers of key j / 4 and lane i receives
// number i of the four keys.
__device__ __forceinline__ u32x2 lds_read_tr(const char* p) {
  return __builtin_bit_cast(
      u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                 (__attribute__((address_space(3))) v4h16*)(reinterpret_cast<uintptr_t>(
                     (const __attribute__((address_space(3))) char*)(p)))));
}

// 16 bytes per lane from base + voff into LDS at ``to`` + 16 * lane. The target goes
// through m0, which the block names as changed. (The warning is that m0 is not
// saved: it is reserved, so nothing is kept in it.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma_rows(uint32_t to, const char* base, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(to), "v"(voff), "s"(base)
               : "m0", "memory");
}
__device__ __forceinline__ void dma_lanes(uint32_t to, const char* p) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(to), "v"(p)
               : "m0", "memory");
}
#pragma clang diagnostic pop

__device__ __forceinline__ int swap_bits23(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

// A block's scores to weights in eight steps, to stand between products: step i forms the
// exponentials of numbers 2 i and 2 i + 1 and packs and adds up those of the step before.
template <class T>
struct Weights {
  const f32x16& s;
  const float sc, base;
  float e0, e1;
  __device__ __forceinline__ Weights(const f32x16& s, float sc, float base) : s(s), sc(sc), base(base) {}
  __device__ __forceinline__ void step(int i, u32x4 (&pf)[2], float& sum, float& top) {
    float x0 = fmaf(s[2 * i], sc, -base), x1 = fmaf(s[2 * i + 1], sc, -base);
    top = fmaxf(top, fmaxf(s[2 * i], s[2 * i + 1]));
    if (i > 0) put(i - 1, pf, sum);
    e0 = __builtin_amdgcn_exp2f(x0);
    e1 = __builtin_amdgcn_exp2f(x1);
    asm volatile("" : "+v"(e0), "+v"(e1), "+v"(top), "+v"(sum));  // (here, not where they are used)
  }
  __device__ __forceinline__ void end(u32x4 (&pf)[2], float& sum) { put(7, pf, sum); }

 private:
  __device__ __forceinline__ void put(int i, u32x4 (&pf)[2], float& sum) {
    sum += e0 + e1;
    pf[i / 4][i % 4] = T::pack2(e0, e1);
  }
};

// KG groups of waves share the rows and take every KG-th block of 32 keys.
template <int D, int KG>
struct Chunk {
  static constexpr int RGW = CW / KG;           // waves side by side over the rows
  static constexpr int ROWS = RGW * 32;
  static constexpr int STAGE = KS * D * 2 * 2;  // bytes of a stage: K, then V
  static constexpr int LDS = 2 * STAGE;
  // a partial result of a wave: [register quad][lane][4], then a reference and a sum per lane
  static constexpr int QUADS = D / 8;
  static constexpr uint32_t PART = RGW * kWave * (QUADS * 16 + 8);
  static_assert(PART <= part_bytes(ROWS, D) && KS == 64, "");
};

template <class T, bool F8, int D, bool BIG, int KG>
__global__ void __launch_bounds__(CTH, 2) attn_chunk_kernel(AttnArgs a) {
  using C = Chunk<D, KG>;
  using P = Plan<C::ROWS, KS, CTH>;
  constexpr int NK = D / 16, NM = D / 32, CPR = D / 8;
  constexpr int KV = KS * D * 2;  // bytes of a stage's K
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ int lds[32];
  __shared__ uint32_t absent[2][KS / 32];  // of a stage's keys: bit i of word b, key 32 b + i is on a bad page
  const int lane = threadIdx.x % kWave, ql = lane % 32, hf = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wr = wave % C::RGW, kg = wave / C::RGW;
  const uint32_t lbase =
      static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)smem));
  if (blockIdx.x == 0 && a.p.status)
    for (int s = threadIdx.x; s < a.p.n_seqs; s += CTH)
      if (a.p.len[s] > a.p.capacity) sync_or(a.p.status, VT_PAGED_BAD_LEN);

  Item it;
  if (!next_item<P>(a, blockIdx.x, it, lds)) return;
  const Seq& q = it.q;
  const int rows = q.nt * a.group;
  const int r0 = it.tile * C::ROWS + wr * 32 + ql, row = min(r0, rows - 1);
  const bool there = r0 < rows;
  const int tok = row / a.group, head = it.head * a.group + row - tok * a.group;
  const int pos = q.pos0 + tok;  // its keys: klo <= p < khi
  const int khi = min(pos + 1, q.keys), klo = a.window > 0 ? max(pos, 0) - (a.window - 1) : 0;
  // keys that every row of the wave sees lie in full_lo .. full_hi - 1, those of any row in any_lo ..
  // any_hi - 1
  int full_hi = khi, any_hi = khi, full_lo = klo, any_lo = klo;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    full_hi = min(full_hi, __shfl_xor(full_hi, o, kWave));
    any_hi = max(any_hi, __shfl_xor(any_hi, o, kWave));
    full_lo = max(full_lo, __shfl_xor(full_lo, o, kWave));
    any_lo = min(any_lo, __shfl_xor(any_lo, o, kWave));
  }
  full_hi = __builtin_amdgcn_readfirstlane(full_hi);
  any_hi = __builtin_amdgcn_readfirstlane(any_hi);
  full_lo = __builtin_amdgcn_readfirstlane(full_lo);
  any_lo = __builtin_amdgcn_readfirstlane(max(any_lo, 0));

  // the tile's own key blocks (its last row sees the most, its first one the earliest),
  // and this piece of them
  const int tpos0 = q.pos0 + it.tile * C::ROWS / a.group;
  const int tpos1 = q.pos0 + (min((it.tile + 1) * C::ROWS, rows) - 1) / a.group;
  const int thi = max(0, min(tpos1 + 1, q.keys)), tlo = a.window > 0 ? max(0, max(tpos0, 0) - (a.window - 1)) : 0;
  const int tb0 = tlo / KS, tbn = max(0, (thi + KS - 1) / KS - tb0);
  const int b0 = tb0 + static_cast<int>(static_cast<int64_t>(tbn) * it.piece / it.pieces);
  const int stages = tb0 + static_cast<int>(static_cast<int64_t>(tbn) * (it.piece + 1) / it.pieces) - b0;
  const char* kb = a.p.k + it.head * a.p.head;
  const char* vb = a.p.v + it.head * a.p.head;
  const uint32_t slot = static_cast<uint32_t>(a.p.slot);
  const int last = q.keys - 1;  // no position past it is read or looked up
  const int32_t* tabv = a.p.table + it.s * a.p.ld_table;
  ConstInt* tab = constant(tabv);

  u32x4 qf[NK];
  {
    const uint16_t* qp = a.q + (q.b + tok) * a.ld_q + static_cast<int64_t>(head) * D;
#pragma unroll
    for (int c = 0; c < NK; ++c) qf[c] = load16(qp + c * 16 + 8 * hf);
  }
  const float sc = a.scale2 * (F8 && a.p.k_scale ? a.p.k_scale[it.head] : 1.f);

  f32x16 o[NM];
  float ref = -INFINITY, sum = 0.f;
#pragma unroll
  for (int m = 0; m < NM; ++m) o[m] = f32x16{};

  // ---- stages into LDS -------------------------------------------------------
  // A wave loads 16 rows of K and of V, LPW loads of RPL rows each: 16 rows together, or (8-bit,
  // D 128) two times 8. Their page numbers are looked up a stage ahead. With pages of 16
  // and more (BIG) rows that are loaded together are on one page: one address for the wave,
  // and offsets of its lanes that are the same in every stage.
  constexpr int LPW = F8 ? D / 64 : D / 32, RPL = F8 ? 1024 / D : 512 / D;
  constexpr int LPR = kWave / RPL;                       // lanes of a row
  constexpr int UPG = F8 ? 1 : LPW, GR = LPW / UPG;      // loads of a group of rows, groups
  const int lrow = lane / LPR, lcol = lane % LPR;
  auto first_row = [&](int g) { return F8 ? g * (CW * RPL) + wave * RPL : wave * 16; };
  // byte offset of the lane's chunk of row u * RPL + lrow of a group, as LDS takes them: in the order
  // of the places, swizzled
  auto chunk_k = [&](int u) { return F8 ? lcol * 16 : (lcol ^ ((u * RPL + lrow) % CPR)) * 16; };
  auto chunk_v = [&](int u) { return F8 ? lcol * 16 : (lcol ^ (2 * ((u * RPL + lrow) % (CPR / 2)))) * 16; };
  constexpr bool AHEAD = F8;  // offsets kept from stage to stage: one register; for 16 bits they are eight and not there
  uint32_t koff[UPG], voff[UPG];
#pragma unroll
  for (int u = 0; u < UPG; ++u) {
    koff[u] = (u * RPL + lrow) * slot + chunk_k(u);
    voff[u] = (u * RPL + lrow) * slot + chunk_v(u);
  }
  int ids[BIG ? GR : LPW];
  u32x4 kreg[F8 ? LPW : 1], vreg[F8 ? LPW : 1];
  auto look = [&](int st) {
    const int p0 = (b0 + min(st, stages - 1)) * KS;
    if constexpr (BIG) {
#pragma unroll
      for (int g = 0; g < GR; ++g) ids[g] = tab[min(p0 + first_row(g), last) >> a.p.shift];
    } else {
#pragma unroll
      for (int u = 0; u < LPW; ++u)
        ids[u] = tabv[min(p0 + first_row(u / UPG) + u % UPG * RPL + lrow, last) >> a.p.shift];
    }
  };
  auto fetch = [&](int st) {
    const int p0 = (b0 + st) * KS, par = st & 1;
#pragma unroll
    for (int g = 0; g < GR; ++g) {
      const int r0 = first_row(g);
      const uint32_t to = __builtin_amdgcn_readfirstlane(lbase + par * C::STAGE + r0 * D * 2);
      uint32_t gone = 0;  // the group's rows on bad pages
      // one load of K and V: from lane addresses, or a wave's and a lane's offsets
      auto get = [&](int u, const char* kp, const char* vp, uint32_t ko, uint32_t vo) {
        if constexpr (F8) {
          kreg[g] = *reinterpret_cast<const u32x4*>(kp + ko);
          vreg[g] = *reinterpret_cast<const u32x4*>(vp + vo);
        } else if constexpr (BIG) {
          dma_rows(to + u * 1024, kp, ko);
          dma_rows(to + u * 1024 + KV, vp, vo);
        } else {
          dma_lanes(to + u * 1024, kp + ko);
          dma_lanes(to + u * 1024 + KV, vp + vo);
        }
      };
      if constexpr (BIG) {
        const bool ok = static_cast<uint32_t>(ids[g]) < static_cast<uint32_t>(a.p.n_pages);
        gone = ok ? 0u : (1u << (UPG * RPL)) - 1;
        const int key = min(p0 + r0, last);
        const uint64_t at = static_cast<uint64_t>(ok ? static_cast<uint32_t>(ids[g]) : 0u) * static_cast<uint64_t>(a.p.page) +
                            static_cast<uint64_t>(static_cast<uint32_t>(key & a.p.mask)) * slot;
        if (AHEAD && __builtin_expect(p0 + r0 + UPG * RPL - 1 <= last, 1)) {
#pragma unroll
          for (int u = 0; u < UPG; ++u) get(u, kb + at, vb + at, koff[u], voff[u]);
        } else {  // rows past the last position read that one again
#pragma unroll
          for (int u = 0; u < UPG; ++u) {
            const uint32_t row = static_cast<uint32_t>(min(u * RPL + lrow, last - key)) * slot;
            get(u, kb + at, vb + at, row + chunk_k(u), row + chunk_v(u));
          }
        }
      } else {
#pragma unroll
        for (int u = 0; u < UPG; ++u) {
          const int id = ids[g * UPG + u];
          const bool ok = id >= 0 && id < a.p.n_pages;
          const uint64_t m = __builtin_amdgcn_ballot_w64(!ok);
          if (m)
#pragma unroll
            for (int i = 0; i < RPL; ++i) gone |= static_cast<uint32_t>(m >> (i * LPR) & 1) << (u * RPL + i);
          const int64_t at = static_cast<int64_t>(ok ? id : 0) * a.p.page +
                             static_cast<int64_t>(min(p0 + r0 + u * RPL + lrow, last) & a.p.mask) * a.p.slot;
          get(u, kb + at, vb + at, chunk_k(u), chunk_v(u));
        }
      }
      // (every lane stores it: a branch that lanes take apart would cost the stages' loop its plain flow)
      char* flag = reinterpret_cast<char*>(absent[par]) + r0 / 8;
      if (UPG * RPL == 8) *reinterpret_cast<uint8_t*>(flag) = static_cast<uint8_t>(gone);
      else *reinterpret_cast<uint16_t*>(flag) = static_cast<uint16_t>(gone);
    }
  };
  // 8-bit: what fetch loaded, widened into its stage
  auto widen = [&](int st) {
    if constexpr (F8) {
      char* S = smem + (st & 1) * C::STAGE;
#pragma unroll
      for (int u = 0; u < GR; ++u) {
        const int r = first_row(u) + lrow;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          u32x4 w, x;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            w[2 * e] = T::template from_f8<false>(kreg[u][2 * h + e]);
            w[2 * e + 1] = T::template from_f8<true>(kreg[u][2 * h + e]);
            x[2 * e] = T::template from_f8<false>(vreg[u][2 * h + e]);
            x[2 * e + 1] = T::template from_f8<true>(vreg[u][2 * h + e]);
          }
          const int c = 2 * lcol + h;
          *reinterpret_cast<u32x4*>(S + r * D * 2 + (c ^ (r % CPR)) * 16) = w;
          *reinterpret_cast<u32x4*>(S + KV + r * D * 2 + (c ^ (2 * (r % (CPR / 2)))) * 16) = x;
        }
      }
    }
  };

  // ---- one block of 32 keys ------------------------------------------------------
  const int grp = lane / 16, jl = lane % 16;
  const int vkey = 8 * (grp / 2) + jl / 4, vdim = 2 * (grp % 2) + (jl % 4) / 2;
  const int kr = swap_bits23(ql);
  // A lane's parts of a block at S: chunk c of its key, and element 32 m + l % 32 of keys
  // 16 b + 8 hf .. + 7.
  // The swizzles are exclusive ors, so the chunks of a lane's key differ from its first one's
  // address in the bits of 32 c, and those of its values in the bits of 64 m (and, where h moves
  // their row by 4, of 128 h): a register for each of these, the rest in the instructions.
  const uint32_t kbase = kr * D * 2 + (hf ^ (kr % CPR)) * 16;
  const uint32_t vbase = vkey * D * 2 + (vdim ^ (2 * (vkey % (CPR / 2)))) * 16 + (jl % 2) * 8;
  uint32_t kat[NK], vat[NM];
#pragma unroll
  for (int c = 0; c < NK; ++c) kat[c] = kbase ^ (32 * c);
#pragma unroll
  for (int m = 0; m < NM; ++m) vat[m] = vbase ^ (64 * m);
#pragma unroll
  for (int c = 0; c < NK; ++c) asm volatile("" : "+v"(kat[c]));
#pragma unroll
  for (int m = 0; m < NM; ++m) asm volatile("" : "+v"(vat[m]));
  auto kfrag = [&](const char* S, int c) { return *reinterpret_cast<const u32x4*>(S + kat[c]); };
  auto vfrag = [&](const char* S, int m, int b) {
    u32x4 f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32x2 x = lds_read_tr(S + KV + (16 * b + 4 * h) * D * 2 + vat[D == 128 ? m ^ (2 * h) : m]);
      f[2 * h] = x[0];
      f[2 * h + 1] = x[1];
    }
    return f;
  };
  // the largest of a lane's scores
  auto largest = [&](const f32x16& s) {
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    return top;
  };
  // a new reference for the rows: the largest score so far
  auto refer = [&](float top) {
    top = fmaxf(top, __shfl_xor(top, 32, kWave));
    const float next = fmaxf(top - T::kTop, ref);
    const float alpha = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref - next);
    ref = next;
    sum *= alpha;
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[m][i] *= alpha;
  };
  // scores (times sc the weights' exponents) to weights, the second product's operand, and their sum (a
  // block's together before they join a sum that may be large)
  auto weigh = [&](const f32x16& s, float sc, u32x4 (&pf)[2], float& sum) {
    const float base = ref == -INFINITY ? 0.f : ref;
    float all = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const float pa = __builtin_amdgcn_exp2f(fmaf(s[2 * w], sc, -base));
      const float pb = __builtin_amdgcn_exp2f(fmaf(s[2 * w + 1], sc, -base));
      all += pa + pb;
      pf[w / 4][w % 4] = T::pack2(pa, pb);
    }
    sum += all;
  };
  // Bits of keys lo .. hi - 1 of the block of 32 from key p0 on.
  auto span = [](int p0, int lo, int hi) {
    const int l = min(max(lo - p0, 0), 32), h = min(max(hi - p0, 0), 32);
    return static_cast<uint32_t>(((uint64_t(1) << h) - 1) & ~((uint64_t(1) << l) - 1));
  };
  // The lane's 16 of a block's 32 bits: accumulator 8 b + e is key 16 b + 8 hf + e.
  auto own16 = [&](uint32_t w) { return (w >> (8 * hf) & 0xFFu) | (w >> (8 + 8 * hf) & 0xFF00u); };
  // One block by itself, from key p0 on, with a new reference: one that some rows of the wave
  // do not see whole, or whose scores ask for it; gone: its keys on bad pages.
  auto single = [&](const char* S, int p0, uint32_t gone) {
    const bool whole = p0 >= full_lo && p0 + 32 <= full_hi && gone == 0;
    f32x16 s = f32x16{};
    {
      u32x4 kf[NK];
#pragma unroll
      for (int c = 0; c < NK; ++c) kf[c] = kfrag(S, c);
      __builtin_amdgcn_sched_barrier(0);  // all of them on their way before the first product
#pragma unroll
      for (int c = 0; c < NK; ++c) s = T::mfma32(kf[c], qf[c], s);
    }
    u32x4 pf[2];
    uint32_t used = 0xFFFFu;  // of the lane's keys
    if (!whole) {
      const uint32_t mine = span(p0, klo, khi), sees = own16(mine & ~gone);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!(sees >> i & 1)) s[i] = -INFINITY;
      if (__builtin_amdgcn_ballot_w64(there && (mine & gone)) != 0 && a.p.status)
        sync_or(a.p.status, VT_PAGED_BAD_PAGE);
      used = own16(span(p0, any_lo, any_hi) & ~gone);
    }
    {
      // rounded before the reference is taken from them: where a score's step is larger than the
      // weights' range, the reference's rounding must be the weights'
#pragma clang fp contract(off)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = s[i] * sc;
    }
    refer(largest(s));
    weigh(s, 1.f, pf, sum);
    // values that no row of the wave sees stay out of the product even if they are
    // infinite
    auto seen = [&](int m, int b, uint32_t keys) {  // a fragment's values of these of the lane's keys
      u32x4 z = vfrag(S, m, b);
#pragma unroll
      for (int w = 0; w < 4; ++w)
        z[w] &= (keys >> (8 * b + 2 * w) & 1 ? 0xFFFFu : 0u) | (keys >> (8 * b + 2 * w + 1) & 1 ? 0xFFFF0000u : 0u);
      return z;
    };
    if (!whole) {
      uint32_t odd = 0;  // a zero half among the exponents' complements: an infinity or a NaN
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        u32x4 z[NM];
#pragma unroll
        for (int m = 0; m < NM; ++m) z[m] = seen(m, b, used);
#pragma unroll
        for (int m = 0; m < NM; ++m)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t c = ~z[m][w] & T::kExp;
            odd |= (c - 0x00010001u) & ~c & 0x80008000u;
          }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (__builtin_amdgcn_ballot_w64(odd != 0) != 0) {
        // where some rows see an infinite or NaN value and others do not, each row gets a
        // product of its own, with what it does not see set to zero
#pragma unroll
        for (int m = 0; m < NM; ++m) {
          f32x16 keep = o[m];
#pragma unroll 1
          for (int c = 0; c < 32; ++c) {
            const uint32_t row =
                own16(span(p0, __builtin_amdgcn_readlane(klo, c), __builtin_amdgcn_readlane(khi, c)) & ~gone);
            f32x16 r = o[m];
#pragma unroll
            for (int b = 0; b < 2; ++b) r = T::mfma32(seen(m, b, row), pf[b], r);
            if (ql == c) keep = r;
          }
          o[m] = keep;
        }
        return;
      }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      u32x4 z[NM];
#pragma unroll
      for (int m = 0; m < NM; ++m) z[m] = seen(m, b, used);
#pragma unroll
      for (int m = 0; m < NM; ++m) o[m] = T::mfma32(z[m], pf[b], o[m]);
    }
  };

  if (stages > 0) {
    // the query loads are waited for here, not among the stages' loads
#pragma unroll
    for (int c = 0; c < NK; ++c) asm volatile("" : "+v"(qf[c]));
    look(0);
    fetch(0);
    look(1);
    // Stage st: what was loaded has landed, everywhere after the barrier, and the stage
    // before is done with; the next one sets out for its place.
    int begun = -1;
    auto begin = [&](int st) {
      if (st == begun) return;
      begun = st;
      widen(st);
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (st + 1 < stages) fetch(st + 1);
      look(st + 2);
    };
    // Blocks t of 32 keys: two of a stage, or (KG 2) the wave's own one. An inner loop for
    // blocks that the wave's rows see whole, left at any other one and at one that
    // raises a reference, which goes the general way: with these cases inside it the outputs
    // moved between registers at every block.
    constexpr int BPS = 2 / KG;
    const int blocks = stages * BPS;
    auto stage_of = [&](int t) { return KG == 2 ? t : t >> 1; };
    auto sub_of = [&](int t) { return KG == 2 ? kg : t & 1; };
    auto first_key = [&](int t) { return (b0 + stage_of(t)) * KS + sub_of(t) * 32; };
    auto place = [&](int t) { return smem + (stage_of(t) & 1) * C::STAGE + sub_of(t) * 32 * D * 2; };
    int t = 0;
    while (t < blocks) {
      // A stage's two blocks A and B overlap: B's scores with A's weights, A's product with B's
      // weights. Weights against a reference that turns out too low are dropped before
      // they are used.
      if constexpr (KG == 1) {
        for (; t + 2 <= blocks; t += 2) {
          const int k0 = (b0 + (t >> 1)) * KS;
          if ((t & 1) != 0 || k0 < full_lo || k0 + KS > full_hi) break;
          begin(t >> 1);
          const int gone = absent[t >> 1 & 1][0] | absent[t >> 1 & 1][1];
          if (__builtin_amdgcn_readfirstlane(gone) != 0) break;
          const char* A = place(t);
          const char* B = A + 32 * D * 2;
          u32x4 kf[NK], vf[NM][2], pa[2], pb[2];
          f32x16 sa = f32x16{}, sb = f32x16{};
          const float base = ref == -INFINITY ? 0.f : ref;
#pragma unroll
          for (int c = 0; c < NK; ++c) kf[c] = kfrag(A, c);
#pragma unroll
          for (int c = 0; c < NK; ++c) {
            sa = T::mfma32(kf[c], qf[c], sa);
            kf[c] = kfrag(B, c);
            asm volatile("" : "+v"(sa));
          }
#pragma unroll
          for (int m = 0; m < NM; ++m)
#pragma unroll
            for (int b = 0; b < 2; ++b) vf[m][b] = vfrag(A, m, b);
          float suma = 0.f, sumb = 0.f, topa = -INFINITY, topb = -INFINITY;
          Weights<T> wa(sa, sc, base), wb(sb, sc, base);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int c = i * NK / 8; c < (i + 1) * NK / 8; ++c) sb = T::mfma32(kf[c], qf[c], sb);
            wa.step(i, pa, suma, topa);
            asm volatile("" : "+v"(sb));
            __builtin_amdgcn_sched_barrier(0);
          }
          wa.end(pa, suma);
          const bool raise_a = __builtin_amdgcn_ballot_w64(fmaf(topa, sc, -ref) > T::kTop + kLag) != 0;
          asm volatile("" : "+v"(pa[0]), "+v"(pa[1]), "+v"(suma));
          if (raise_a) break;
          sum += suma;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int j = i * NM / 4; j < (i + 1) * NM / 4; ++j) {
              const int m = j % NM, b = j / NM;
              o[m] = T::mfma32(vf[m][b], pa[b], o[m]);
              vf[m][b] = vfrag(B, m, b);
            }
            wb.step(i, pb, sumb, topb);
            __builtin_amdgcn_sched_barrier(0);
          }
          wb.end(pb, sumb);
          const bool raise_b = __builtin_amdgcn_ballot_w64(fmaf(topb, sc, -ref) > T::kTop + kLag) != 0;
          asm volatile("" : "+v"(pb[0]), "+v"(pb[1]), "+v"(sumb));
          if (raise_b) {
            ++t;  // A is done
            break;
          }
          sum += sumb;
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int m = 0; m < NM; ++m) o[m] = T::mfma32(vf[m][b], pb[b], o[m]);
        }
      } else {
        for (; t < blocks; ++t) {
          const int k0 = first_key(t);
          if (k0 < full_lo || k0 + 32 > full_hi) break;
          begin(stage_of(t));
          if (__builtin_amdgcn_readfirstlane(absent[stage_of(t) & 1][sub_of(t)]) != 0) break;
          const char* B = place(t);
          // all fragments are on their way before the first is used: V's arrive behind the scores
          u32x4 kf[NK], vf[NM][2], pf[2];
#pragma unroll
          for (int c = 0; c < NK; ++c) kf[c] = kfrag(B, c);
#pragma unroll
          for (int m = 0; m < NM; ++m)
#pragma unroll
            for (int b = 0; b < 2; ++b) vf[m][b] = vfrag(B, m, b);
          __builtin_amdgcn_sched_barrier(0);
          f32x16 s = f32x16{};
#pragma unroll
          for (int c = 0; c < NK; ++c) s = T::mfma32(kf[c], qf[c], s);
          if (__builtin_amdgcn_ballot_w64(fmaf(largest(s), sc, -ref) > T::kTop + kLag) != 0) break;
          weigh(s, sc, pf, sum);
#pragma unroll
          for (int m = 0; m < NM; ++m)
#pragma unroll
            for (int b = 0; b < 2; ++b) o[m] = T::mfma32(vf[m][b], pf[b], o[m]);
        }
      }
      if (t >= blocks) break;
      begin(stage_of(t));
      const int k0 = first_key(t);
      const uint32_t gone = __builtin_amdgcn_readfirstlane(absent[stage_of(t) & 1][sub_of(t)]);
      if (k0 < any_hi && k0 + 32 > any_lo) single(place(t), k0, gone);  // some row of the wave sees some of it
      ++t;
    }
  }
  sum += __shfl_xor(sum, 32, kWave);

  // the second half of the waves' results, left in LDS in register order, into the first's
  auto merge = [&]() {
    if constexpr (KG == 1) return;
    __syncthreads();
    float* part = reinterpret_cast<float*>(smem) + wr * (D / 2 + 2) * kWave + lane;
    if (kg == 1) {
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) part[(m * 16 + i) * kWave] = o[m][i];
      part[(D / 2) * kWave] = ref;
      part[(D / 2 + 1) * kWave] = sum;
    }
    __syncthreads();
    if (kg == 0) {
      const float r1 = part[(D / 2) * kWave], top = fmaxf(ref, r1), base = top == -INFINITY ? 0.f : top;
      const float f0 = __builtin_amdgcn_exp2f(ref - base), f1 = __builtin_amdgcn_exp2f(r1 - base);
      sum = sum * f0 + part[(D / 2 + 1) * kWave] * f1;
      ref = top;
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[m][i] = o[m][i] * f0 + part[(m * 16 + i) * kWave] * f1;
    }
  };
  merge();

  if (it.pieces > 1) {
    const rsrc_t ru = make_rsrc(reinterpret_cast<char*>(a.part) + static_cast<int64_t>(it.slot) * C::PART,
                                it.pieces * C::PART);
    // of this lane: quad i at 1 KiB steps, then (reference, sum)
    const uint32_t at = wr * (C::QUADS * 16 + 8) * kWave;
    auto quad = [&](int i) { return at + i * 16 * kWave + lane * 16; };
    const uint32_t stats = at + C::QUADS * 16 * kWave + lane * 8;
    if (kg == 0) {
      const uint32_t mine = it.piece * C::PART;
#pragma unroll
      for (int i = 0; i < C::QUADS; ++i) {
        const f32x4 x = {o[i / 4][i % 4 * 4], o[i / 4][i % 4 * 4 + 1], o[i / 4][i % 4 * 4 + 2], o[i / 4][i % 4 * 4 + 3]};
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), ru, mine + quad(i), 0, kCoherent);
      }
      __builtin_amdgcn_raw_buffer_store_b64(
          u32x2{__builtin_bit_cast(uint32_t, ref), __builtin_bit_cast(uint32_t, sum)}, ru, mine + stats, 0, kCoherent);
    }
    mem_done();
    __syncthreads();
    if (threadIdx.x == 0)
      lds[0] = __hip_atomic_fetch_add(a.arrived + it.unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
               static_cast<uint32_t>(it.pieces - 1);
    __syncthreads();
    // the last piece to arrive joins them all, in their order
    if (lds[0] == 0) return;
    if (threadIdx.x == 0) sync_store(a.arrived + it.unit, 0u);
    // two pieces' numbers on their way at once, the groups of waves taking turns
    ref = -INFINITY;
    sum = 0.f;
#pragma unroll
    for (int m = 0; m < NM; ++m) o[m] = f32x16{};
    for (int c = 2 * kg; c < it.pieces; c += 2 * KG) {
      float r[2], t[2];
      u32x4 x[2][C::QUADS];
#pragma unroll
      for (int k = 0; k < 2; ++k) {  // a piece past the last one is out of the range: zeros
        buf_ld_shared2(ru, (c + k) * C::PART + stats, r[k], t[k]);
#pragma unroll
        for (int i = 0; i < C::QUADS; ++i)
          x[k][i] = __builtin_amdgcn_raw_buffer_load_b128(ru, (c + k) * C::PART + quad(i), 0, kCoherent);
      }
      if (c + 1 >= it.pieces) r[1] = -INFINITY;
      const float top = fmaxf(ref, fmaxf(r[0], r[1])), base = top == -INFINITY ? 0.f : top;
      const float f = __builtin_amdgcn_exp2f(ref - base), f0 = __builtin_amdgcn_exp2f(r[0] - base),
                  f1 = __builtin_amdgcn_exp2f(r[1] - base);
      ref = top;
      sum = sum * f + t[0] * f0 + t[1] * f1;
#pragma unroll
      for (int i = 0; i < C::QUADS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[i / 4][i % 4 * 4 + e] = o[i / 4][i % 4 * 4 + e] * f + f0 * __builtin_bit_cast(f32x4, x[0][i])[e] +
                                    f1 * __builtin_bit_cast(f32x4, x[1][i])[e];
    }
    merge();
  }
  if (kg != 0 || !there) return;
  const float vs = F8 && a.p.v_scale ? a.p.v_scale[it.head] : 1.f;
  const float inv = sum == 0.f ? 0.f : vs / sum;
  uint16_t* op = a.out + (q.b + tok) * a.ld_out + static_cast<int64_t>(head) * D + 4 * hf;
  // accumulator i of tile m is element 32 m + 8 (i / 4) + 4 hf + i % 4
#pragma unroll
  for (int m = 0; m < NM; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<u32x2*>(op + 32 * m + 8 * i) = u32x2{T::pack2(o[m][4 * i] * inv, o[m][4 * i + 1] * inv),
                                                             T::pack2(o[m][4 * i + 2] * inv, o[m][4 * i + 3] * inv)};
  if (a.lse && hf == 0)
    a.lse[static_cast<int64_t>(q.b + tok) * a.n_q + head] =
        sum == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

hipError_t launch_chunk(const AttnArgs& a, int type, bool f8, int head_dim, int tile, hipStream_t s) {
  const bool big = a.p.mask + 1 >= 16;
  int shared = 0;
  auto pick = [&](auto X, auto F, auto B, auto DD) -> void (*)(AttnArgs) {
    using T = decltype(X);
    constexpr int D = decltype(DD)::value;
    constexpr bool f = decltype(F)::value, b = decltype(B)::value;
    if (tile == 64) {
      shared = std::max<int>(Chunk<D, 2>::LDS, Chunk<D, 2>::RGW * (D / 2 + 2) * kWave * 4);
      return attn_chunk_kernel<T, f, D, b, 2>;
    }
    shared = Chunk<D, 1>::LDS;
    return attn_chunk_kernel<T, f, D, b, 1>;
  };
  auto pick3 = [&](auto X, auto F, auto B) {
    return head_dim == 128 ? pick(X, F, B, std::integral_constant<int, 128>{})
                           : pick(X, F, B, std::integral_constant<int, 64>{});
  };
  auto pick2 = [&](auto X, auto F) {
    return big ? pick3(X, F, std::true_type{}) : pick3(X, F, std::false_type{});
  };
  auto pick1 = [&](auto X) { return f8 ? pick2(X, std::true_type{}) : pick2(X, std::false_type{}); };
  auto* kernel = type == VT_T_F16 ? pick1(Half{}) : pick1(BFloat{});
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, shared);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(grid_of(a, tile))), dim3(CTH), shared, s, a);
  return hipGetLastError();
}

}  // namespace pg
}  // namespace vt
