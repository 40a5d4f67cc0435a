// Shared by the paged-cache kernels: number formats, arguments, the split of a
// batch's attention into work items, and where a position's page is.
#pragma once

#include "device.hpp"
#include "internal.hpp"

namespace vt {
namespace pg {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr float kF8Max = 448.f;

// The activations' 16-bit type. pack2 rounds to nearest even.
struct Half {
  static __device__ __forceinline__ uint32_t pack2(float a, float b) {
    return __builtin_bit_cast(uint32_t, f16x2{static_cast<_Float16>(a), static_cast<_Float16>(b)});
  }
  static __device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b) { vt::unpack2(w, a, b); }
  // two 8-bit numbers of a word's low or high half, exactly
  template <bool HI>
  static __device__ __forceinline__ uint32_t from_f8(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, HI));
  }
  static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                  0);
  }
  static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                  0);
  }
  static constexpr uint32_t kExp = 0x7C007C00u;  // the exponent bits of both halves of a word
};

struct BFloat {
  static __device__ __forceinline__ uint32_t pack2(float a, float b) {
    return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
  }
  static __device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b) {
    a = __builtin_bit_cast(float, w << 16);
    b = __builtin_bit_cast(float, w & 0xFFFF0000u);
  }
  template <bool HI>
  static __device__ __forceinline__ uint32_t from_f8(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, HI));
  }
  static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
  }
  static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
  }
  static constexpr uint32_t kExp = 0x7F807F80u;
};

// Whether either half of a word is an infinity or NaN of type T.
template <class T>
__device__ __forceinline__ bool odd2(uint32_t w) {
  constexpr uint32_t lo = T::kExp & 0xFFFFu, hi = T::kExp & 0xFFFF0000u;
  return (w & lo) == lo || (w & hi) == hi;
}

// The pool and its sequences as the kernels take them; strides in bytes.
struct Pool {
  char* k;
  char* v;
  int64_t page, head, slot;
  const int32_t* table;
  int64_t ld_table;
  const int32_t* len;
  uint32_t* status;
  const float* k_scale;
  const float* v_scale;
  int32_t n_pages, shift, mask;  // page_size = 1 << shift = mask + 1
  int32_t capacity;              // positions a table row can name (at most 2^31 - 1)
  int32_t n_kv, n_seqs;
};

struct AttnArgs {
  Pool p;
  const uint16_t* q;
  int64_t ld_q;
  uint16_t* out;
  int64_t ld_out;
  float* lse;
  const int32_t* q_begin;
  int32_t n_tok, n_q, group, window;
  float scale2;  // softmax scale times log2 e
  uint32_t* arrived;  // one counter per split unit, zero between calls
  float* part;        // partial results of split units
  int32_t target;     // work items to aim at
  int32_t min_blocks; // key blocks of an item below which splitting stops
};

// Memory that nothing writes while a kernel runs: loads at addresses that all lanes
// share go through the scalar cache.
typedef const __attribute__((address_space(4))) int32_t ConstInt;
__device__ __forceinline__ ConstInt* constant(const int32_t* p) {
  return reinterpret_cast<ConstInt*>(reinterpret_cast<uintptr_t>(p));
}

// Sequence s of the batch: its rows b.., its new tokens nt, the position pos0 of
// the first of them (negative where the sequence is shorter than its new tokens) and
// the number of its keys.
struct Seq {
  int32_t b, nt, pos0, keys;
};

__device__ __forceinline__ Seq sequence(const AttnArgs& a, int s) {
  Seq q;
  int e;
  if (a.q_begin) {
    q.b = min(max(a.q_begin[s], 0), a.n_tok);
    e = min(max(a.q_begin[s + 1], q.b), a.n_tok);
  } else {
    q.b = s;
    e = s + 1;
  }
  q.nt = e - q.b;
  const int n = max(a.p.len[s], 0);
  q.pos0 = n - q.nt;
  q.keys = min(n, a.p.capacity);
  return q;
}

// One work item: a tile of a sequence's rows for one KV head, and a piece of its keys.
struct Item {
  int32_t s, tile, head, piece, pieces;
  int32_t block0, blocks;  // the tile's key blocks, of which this piece takes a share
  int32_t unit, slot;      // of a split unit: its counter and its first partial result
};

// Sums of three counts over the threads before this one (the block's totals in tot).
template <int NT>
__device__ __forceinline__ void scan3(int (&v)[3], int (&tot)[3], int* lds) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int own[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) own[i] = v[i];
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1)
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const int x = __shfl_up(v[i], o, kWave);
      if (lane >= o) v[i] += x;
    }
  if (lane == kWave - 1)
#pragma unroll
    for (int i = 0; i < 3; ++i) lds[wave * 3 + i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    int before = 0;
    tot[i] = 0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) {
      const int x = lds[w * 3 + i];
      if (w < wave) before += x;
      tot[i] += x;
    }
    v[i] += before - own[i];
  }
  __syncthreads();
}

// A sequence's share of the work on tiles of ROWS rows and key blocks of KEYS keys.
template <int ROWS, int KEYS>
struct Share {
  int32_t tiles, block0, blocks;
  __device__ __forceinline__ Share(const AttnArgs& a, const Seq& q) {
    const int64_t rows = static_cast<int64_t>(q.nt) * a.group;
    tiles = static_cast<int32_t>((rows + ROWS - 1) / ROWS);
    const int lo = a.window > 0 ? max(0, min(max(q.pos0, 0) - (a.window - 1), q.keys)) : 0;
    block0 = lo / KEYS;
    blocks = (q.keys - block0 * KEYS + KEYS - 1) / KEYS;
  }
};

// The split of the batch. Every workgroup computes it from the lengths alone, so
// nothing depends on what the host knows of them: with N key blocks in all (over
// tiles and heads), units longer than X = max(min_blocks, N / target) blocks are cut
// into pieces of about equal size. Fewer than ``target`` units are cut, into fewer than
// 2 * target pieces in all, whatever the lengths: that sizes counters and partials.
template <int ROWS, int KEYS, int NT>
struct Plan {
  int32_t per;     // sequences per thread
  int32_t most;    // X
  int32_t base[3]; // items, cut units and pieces of them before this thread's sequences
  int32_t total;   // items in all

  __device__ __forceinline__ int pieces(int blocks) const { return max(1, (blocks + most - 1) / most); }

  __device__ void make(const AttnArgs& a, int* lds) {
    per = (a.p.n_seqs + NT - 1) / NT;
    const int s0 = threadIdx.x * per, s1 = min(s0 + per, a.p.n_seqs);
    // units are counted in floating point: exact up to 2^24, and a cut near enough beyond
    float n = 0.f;
    for (int s = s0; s < s1; ++s) {
      const Seq q = sequence(a, s);
      const Share<ROWS, KEYS> h(a, q);
      n += static_cast<float>(h.tiles) * static_cast<float>(h.blocks) * a.p.n_kv;
    }
    n = block_sum<NT>(n, reinterpret_cast<float*>(lds));
    // rounding of n is covered by the factor: X must not fall below N / target
    most = max(a.min_blocks, static_cast<int32_t>(ceilf(fminf(n * 1.0001f / static_cast<float>(a.target), 1e9f))));
    int v[3] = {0, 0, 0}, tot[3];
    for (int s = s0; s < s1; ++s) {
      const Seq q = sequence(a, s);
      const Share<ROWS, KEYS> h(a, q);
      const int units = h.tiles * a.p.n_kv, pc = pieces(h.blocks);
      v[0] += units * pc;
      v[1] += pc > 1 ? units : 0;
      v[2] += pc > 1 ? units * pc : 0;
    }
    scan3<NT>(v, tot, lds);
#pragma unroll
    for (int i = 0; i < 3; ++i) base[i] = v[i];
    total = tot[0];
  }

  // Item i, found by the thread whose sequences hold it and handed to all through
  // lds (9 words).
  __device__ Item find(const AttnArgs& a, int i, int* lds) const {
    const int s0 = threadIdx.x * per, s1 = min(s0 + per, a.p.n_seqs);
    int at = base[0], unit = base[1], slot = base[2];
    __syncthreads();
    for (int s = s0; s < s1 && at <= i; ++s) {
      const Seq q = sequence(a, s);
      const Share<ROWS, KEYS> h(a, q);
      const int units = h.tiles * a.p.n_kv, pc = pieces(h.blocks), n = units * pc;
      if (i < at + n) {
        // heads fastest: with a multiple of 8 of them, one head's items share an XCD;
        // then pieces, then tiles, those with the most keys first
        int r = i - at;
        const int head = r % a.p.n_kv;
        r /= a.p.n_kv;
        const int piece = r % pc, tile = h.tiles - 1 - r / pc, u = tile * a.p.n_kv + head;
        lds[0] = s;
        lds[1] = tile;
        lds[2] = head;
        lds[3] = piece;
        lds[4] = pc;
        lds[5] = h.block0;
        lds[6] = h.blocks;
        lds[7] = unit + u;
        lds[8] = slot + u * pc;
      }
      at += n;
      if (pc > 1) {
        unit += units;
        slot += n;
      }
    }
    __syncthreads();
    Item t;
    int* o = reinterpret_cast<int*>(&t);
#pragma unroll
    for (int w = 0; w < 9; ++w) o[w] = __builtin_amdgcn_readfirstlane(lds[w]);
    return t;
  }
};

// ---- host side, in paged.hip -------------------------------------------------
constexpr int kTarget = 512;          // work items aimed at; fewer units than that are cut, and have counters
constexpr size_t kSyncBytes = 8192;   // the counters, at the start of the workspace
static_assert(kTarget * 4 <= kSyncBytes, "");

hipError_t launch_chunk(const AttnArgs& a, int type, bool f8, int head_dim, int tile, hipStream_t s);
hipError_t launch_rows(const AttnArgs& a, int type, bool f8, int head_dim, hipStream_t s);

}  // namespace pg
}  // namespace vt
