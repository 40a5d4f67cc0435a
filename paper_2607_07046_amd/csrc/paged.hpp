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

// Weights of a softmax are exp2(score - ref), ref a row's reference, 2^kTop below its maximum when it is
// set and following that when it rises by more than kLag: weights end at 2^(kTop + kLag), so sums and
// outputs are hardly ever rescaled. What is compared with kTop + kLag is a weight's own exponent as the weight
// takes it: beside scores whose steps are larger than kLag no other rounding bounds it.
constexpr float kLag = 8.f;

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
  // Weights up to 2^15, as large as fp16 has: those below the smallest one's half, 2^-25, are zero in a product
  // and all are off by as much, which of the largest one is then 2^-32 or less. With the maximum at 1 it was
  // 2^-25, and 131072 keys at 2^-26 of one large one, 0.2% of the sum, were not in the output at all.
  static constexpr float kTop = 7.f;
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
  // Weights up to 2^-32: fewer than 2^31 of them with values up to 2^128 add up to less than 2^127, so sums of
  // finite values are finite (with weights around 1 values of 3e38 gave infinity). Weights down to 2^-126
  // are still 2^-86 of the maximum's.
  static constexpr float kTop = -40.f;
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
  int32_t capacity;              // positions a table row can name, at most kMaxPositions
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
  Seq q;
  int32_t s, tile, head, piece, pieces;
  int32_t block0, blocks;  // the sequence's key blocks
  int32_t unit, slot;      // of a cut unit: its counter and its first partial result
};
constexpr int kItemWords = sizeof(Item) / 4;

// Inclusive sum over the lanes of a wave up to each lane: shifts within rows of 16,
// then the rows' last lanes broadcast into those behind.
template <int CTRL, int ROW_MASK = 0xF>
__device__ __forceinline__ int dpp_i(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROW_MASK, 0xF, false);
}
__device__ __forceinline__ int wave_scan(int v) {
  v += dpp_i<0x111>(v);        // row_shr:1
  v += dpp_i<0x112>(v);        // row_shr:2
  v += dpp_i<0x114>(v);        // row_shr:4
  v += dpp_i<0x118>(v);        // row_shr:8
  v += dpp_i<0x142, 0xA>(v);   // row_bcast:15 into rows 1 and 3
  v += dpp_i<0x143, 0xC>(v);   // row_bcast:31 into rows 2 and 3
  return v;
}

// Sums of three counts over the threads before this one (the block's totals in tot).
template <int NT>
__device__ __forceinline__ void scan3(int (&v)[3], int (&tot)[3], int* lds) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int own[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    own[i] = v[i];
    v[i] = wave_scan(v[i]);
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
// 2 * target pieces in all, whatever the lengths: that sizes counters and partials. (X may
// become longer, see fit.)
// Up to NT sequences a thread keeps its own one's length from the only load of it. More of them
// are walked two to four times by every workgroup, work that grows with sequences times items: a
// decode step of 64 positions and 8 KV heads takes 101-118 ns a sequence for 128 to 512 of them, 138
// for 1024, 280 for 4096, 1115 for 16384, 4613 for 65536; of 256 positions 200-223 up to 1024, 350 for 4096.
template <int ROWS, int KEYS, int NT>
struct Plan {
  int32_t per;     // sequences per thread
  int32_t most;    // X, longest piece in blocks
  int32_t base[3]; // items, cut units and pieces of them before this thread's sequences
  int32_t total;   // items in all
  Seq mine;        // this thread's sequence, if it has one only

  // The pieces of a unit are joined by one workgroup, in time that grows with their number.
  // A 16-row tile's partial results are small: 128 of them come in a few round trips. Those of
  // the larger tiles are as large as what one or two stages load: about as many pieces as a
  // piece has blocks, or (64 rows) twice that (32 rows over 32768 positions 43.3 -> 41.7 us with twice
  // as many, 128 rows 57.2 -> 70).
  static __device__ __forceinline__ int most_pieces(int blocks) {
    const float root = sqrtf(static_cast<float>(blocks));
    return ROWS == 16 ? 128 : max(1, static_cast<int>(ROWS == 64 ? 2.f * root : root));
  }
  __device__ __forceinline__ int pieces(int blocks) const {
    return min(most_pieces(blocks), max(1, (blocks + most - 1) / most));
  }

  __device__ __forceinline__ Seq seq(const AttnArgs& a, int s) const { return per == 1 ? mine : sequence(a, s); }

  __device__ __forceinline__ void cut(const AttnArgs& a, float n) {
    // n may be rounded: the factor keeps X from falling below N / target
    most = max(a.min_blocks, static_cast<int32_t>(ceilf(fminf(n * 1.0001f / static_cast<float>(a.target), 1e9f))));
  }

  // ``target`` items run at once, so X times the rounds of them is about the time: X times 5/4, 3/2 or
  // 2 is taken where its pieces fit into so many fewer rounds (16 sequences of 2056-4099 positions,
  // 8 heads of one or two tiles 59.5 -> 54 us, 12 ragged ones 45.2 -> 37.8, three chunks of 256 tokens
  // 136 -> 117). The counts are estimates (quotients are rounded); of at most 4 * target items
  // at X, and fewer at more, two counts' sums fit into a word. The cut stays the lengths' alone.
  __device__ __forceinline__ int longer(int i) const {  // less than 2^31: X is at most 10^9
    return i == 0 ? most : (i == 1 ? most + most / 4 : (i == 2 ? most + most / 2 : 2 * most));
  }
  struct Tries {
    float items[4];
  };
  __device__ __forceinline__ void count(const AttnArgs& a, const Share<ROWS, KEYS>& h, Tries& t) const {
    const float n = static_cast<float>(h.tiles * a.p.n_kv), b = static_cast<float>(h.blocks);
    const float top = static_cast<float>(most_pieces(h.blocks));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = ceilf(b * __builtin_amdgcn_rcpf(static_cast<float>(longer(i))) - 1e-3f);
      t.items[i] += n * fminf(top, fmaxf(p, 1.f));
    }
  }
  __device__ __forceinline__ void fit(const AttnArgs& a, const Tries& t) {
    float least = 0.f;
    int best = most;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = longer(i);
      const float time = ceilf(t.items[i] / static_cast<float>(a.target)) * static_cast<float>(x);
      if (i == 0 || time < least) {
        least = time;
        best = x;
      }
    }
    most = __builtin_amdgcn_readfirstlane(best);
  }

  // Whether pieces may fit better: some units are cut, into more items than run at once, and not
  // into so many that one round more or less makes no difference.
  __device__ __forceinline__ bool uneven(const AttnArgs& a, int items, int cut_pieces) const {
    return cut_pieces > 0 && items > a.target && items <= 4 * a.target;
  }

  // The items, cut units and pieces of them before this thread's sequences; the counts of all.
  __device__ __forceinline__ void count_all(const AttnArgs& a, int s0, int s1, int (&tot)[3], int* lds) {
#pragma unroll
    for (int i = 0; i < 3; ++i) base[i] = 0;
    for (int s = s0; s < s1; ++s) {
      const Share<ROWS, KEYS> h(a, seq(a, s));
      const int units = h.tiles * a.p.n_kv, pc = pieces(h.blocks);
      base[0] += units * pc;
      base[1] += pc > 1 ? units : 0;
      base[2] += pc > 1 ? units * pc : 0;
    }
    scan3<NT>(base, tot, lds);
  }

  __device__ __forceinline__ void make(const AttnArgs& a, int* lds) {
    per = (a.p.n_seqs + NT - 1) / NT;
    if (a.p.n_seqs == 1) {  // every thread has it, and nothing is to be summed up
      mine = sequence(a, 0);
      const Share<ROWS, KEYS> h(a, mine);
      cut(a, static_cast<float>(h.tiles) * static_cast<float>(h.blocks) * a.p.n_kv);
      base[0] = base[1] = base[2] = 0;
      const int units = h.tiles * a.p.n_kv;
      total = units * pieces(h.blocks);
      if (uneven(a, total, total - units)) {
        Tries t{};
        count(a, h, t);
        fit(a, t);
        total = units * pieces(h.blocks);
      }
      return;
    }
    const int s0 = threadIdx.x * per, s1 = min(s0 + per, a.p.n_seqs);
    if (per == 1 && s0 < s1) mine = sequence(a, s0);
    float n = 0.f;
    for (int s = s0; s < s1; ++s) {
      const Share<ROWS, KEYS> h(a, seq(a, s));
      n += static_cast<float>(h.tiles) * static_cast<float>(h.blocks) * a.p.n_kv;
    }
    cut(a, block_sum<NT>(n, reinterpret_cast<float*>(lds)));
    int tot[3];
    count_all(a, s0, s1, tot, lds);
    if (uneven(a, tot[0], tot[2])) {
      Tries t{};
      for (int s = s0; s < s1; ++s) count(a, Share<ROWS, KEYS>(a, seq(a, s)), t);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int sum = wave_scan(static_cast<int>(t.items[2 * i]) | static_cast<int>(t.items[2 * i + 1]) << 16);
        if (threadIdx.x % kWave == kWave - 1) lds[threadIdx.x / kWave * 2 + i] = sum;
      }
      __syncthreads();
      t = Tries{};
#pragma unroll
      for (int w = 0; w < NT / kWave * 2; ++w) {
        t.items[w % 2 * 2] += static_cast<float>(lds[w] & 0xFFFF);
        t.items[w % 2 * 2 + 1] += static_cast<float>(static_cast<uint32_t>(lds[w]) >> 16);
      }
      __syncthreads();
      fit(a, t);
      count_all(a, s0, s1, tot, lds);
    }
    total = tot[0];
  }

  // Item r of sequence s, whose cut units and their pieces start at unit and slot.
  __device__ __forceinline__ Item item(const AttnArgs& a, const Seq& q, int s, int r, int unit, int slot) const {
    const Share<ROWS, KEYS> h(a, q);
    // heads fastest: with a multiple of 8 of them, one head's items share an XCD; then
    // pieces, then tiles, those with the most keys first
    Item t;
    t.q = q;
    t.s = s;
    t.pieces = pieces(h.blocks);
    t.head = r % a.p.n_kv;
    r /= a.p.n_kv;
    t.piece = r % t.pieces;
    t.tile = h.tiles - 1 - r / t.pieces;
    t.block0 = h.block0;
    t.blocks = h.blocks;
    const int u = t.tile * a.p.n_kv + t.head;
    t.unit = unit + u;
    t.slot = slot + u * t.pieces;
    return t;
  }

  // Item i, found by the thread whose sequences hold it and handed to all through
  // lds (kItemWords words).
  __device__ __forceinline__ Item find(const AttnArgs& a, int i, int* lds) const {
    Item t;
    if (a.p.n_seqs == 1) {
      t = item(a, mine, 0, i, 0, 0);
    } else {
      const int s0 = threadIdx.x * per, s1 = min(s0 + per, a.p.n_seqs);
      int at = base[0], unit = base[1], slot = base[2];
      __syncthreads();
      for (int s = s0; s < s1 && at <= i; ++s) {
        const Seq q = seq(a, s);
        const Share<ROWS, KEYS> h(a, q);
        const int units = h.tiles * a.p.n_kv, pc = pieces(h.blocks), n = units * pc;
        if (i < at + n) {
          t = item(a, q, s, i - at, unit, slot);
          const int* w = reinterpret_cast<const int*>(&t);
#pragma unroll
          for (int k = 0; k < kItemWords; ++k) lds[k] = w[k];
        }
        at += n;
        if (pc > 1) {
          unit += units;
          slot += n;
        }
      }
      __syncthreads();
      int* w = reinterpret_cast<int*>(&t);
#pragma unroll
      for (int k = 0; k < kItemWords; ++k) w[k] = lds[k];
    }
    int* w = reinterpret_cast<int*>(&t);
#pragma unroll
    for (int k = 0; k < kItemWords; ++k) w[k] = __builtin_amdgcn_readfirstlane(w[k]);
    return t;
  }
};

// Item i; false if there is none.
template <class PLAN>
__device__ __forceinline__ bool next_item(const AttnArgs& a, int i, Item& t, int* lds) {
  PLAN plan;
  plan.make(a, lds);
  if (i >= plan.total) return false;
  t = plan.find(a, i, lds);
  return true;
}

// ---- host side, in paged.hip -------------------------------------------------
// Positions of a sequence: the end of the block behind the last one is still an int.
constexpr int32_t kMaxPositions = INT32_MAX - 4095;

// Most bytes of one partial result: its rows' outputs, and a reference and a sum for each of the
// two lanes that hold a row.
constexpr size_t part_bytes(int rows, int head_dim) { return static_cast<size_t>(rows) * (head_dim + 4) * 4; }

// Workgroups that cover a batch's items, one each, on tiles of ``rows`` rows: a cut into pieces of
// X or more blocks adds at most N / X <= target to the units. The rest ends at once.
inline int64_t grid_of(const AttnArgs& a, int rows) {
  const int64_t tiles = a.q_begin ? static_cast<int64_t>(a.n_tok) * a.group / rows + a.p.n_seqs
                                  : static_cast<int64_t>(a.p.n_seqs) * ((a.group + rows - 1) / rows);
  const int keys = rows == 16 ? 128 : 64;  // of a block
  const int64_t units = tiles * a.p.n_kv, blocks = (static_cast<int64_t>(a.p.capacity) + keys - 1) / keys;
  return units * blocks < units + a.target ? units * blocks : units + a.target;
}

// Work items aimed at by the largest tiles, two workgroups of which a compute unit holds.
// The smaller tiles aim at half of that, one per compute unit: their pieces wait for
// memory, and longer ones have less to start, to end and to join (one sequence of 131071
// positions with 8-bit numbers: 61 us with 512, 57 with 256; 64 of 8 tokens 136 and 110;
// 512 rows per head over 33280 positions on the largest tiles 583 and 737).
constexpr int kTarget = 512;
constexpr size_t kSyncBytes = 8192;   // the counters, at the start of the workspace
static_assert(kTarget * 4 <= kSyncBytes, "");

hipError_t launch_chunk(const AttnArgs& a, int type, bool f8, int head_dim, int tile, hipStream_t s);
hipError_t launch_rows(const AttnArgs& a, int type, bool f8, int head_dim, hipStream_t s);

}  // namespace pg
}  // namespace vt
