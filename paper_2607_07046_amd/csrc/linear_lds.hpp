// Loads from memory straight into LDS, and the layout that the projections' kernels give them there.
//
// LDS holds blocks of 8 rows x 64 k (1 KiB): one instruction of a wave, whose 8 lanes of a row read a whole
// 128-byte line (with 16 rows x 32 k every line was fetched twice, a product of 8192 x 8192 x 8192 took 843 us, where
// it takes 743 to 757). Chunk c (16 bytes) of row r of a fragment of 16 rows is at unit 8 (r % 8) + (c ^ (r / 2)) of block
// r / 8: the 16 lanes that a fragment's read serves together (0-3, 12-15, 20-23, 24-27 and the like)
// find it in different banks.
#pragma once

#include "linear.hpp"

namespace vt {
namespace lin {

// Row of its block and chunk that lane l's 16 bytes hold; ``half``: which block of a fragment's two it is.
__device__ __forceinline__ int block_row(int lane) { return lane / 8; }
__device__ __forceinline__ int block_chunk(int lane, int half) { return (lane % 8) ^ (4 * half + lane / 16); }
// Where lane l's part of a fragment (row l % 16, chunk l / 16 of the block's k-step) is in the block of its row;
// the other k-step of 32 is at that address ^ 64.
__device__ __forceinline__ int fragment_at(int lane) {
  const int r = lane % 16;
  return (r % 8 * 8 + ((lane / 16) ^ (r / 2))) * 16;
}

// 16 bytes per lane from r[voff + soff] to LDS at m0 + 16 * lane, in inline asm and waited for by their count: with
// the compiler's own form every read of LDS waits for all of them. m0 is set in the block of the load, with
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

// The same descriptor as make_rsrc, as four scalar words.
__device__ __forceinline__ u32x4 rsrc_words(const void* base, uint32_t bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  return u32x4{static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(p))),
               static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(p >> 32))) & 0xFFFFu,
               static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(bytes))), 0x00020000u};
}
__device__ __forceinline__ rsrc_t rsrc_of(u32x4 w) {
  return make_rsrc(reinterpret_cast<const void*>((static_cast<uint64_t>(w.y) << 32) | w.x), w.z);
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)p));
}

// A slice's sums to the workspace, in register order; whichever workgroup of the tile counts itself last adds all
// slices, in slice order, and is the one that returns true. Nobody waits for another. ``lds``: 4 bytes that
// nobody else uses until the call returns.
template <int NB, int MB, int NW>
__device__ __forceinline__ bool join(const Args& a, f32x4 (&acc)[NB][MB], char* lds, int tile, int split, int wave,
                                     int lane) {
  constexpr int TILE = NW * NB * MB * 256;  // floats
  // slices in flight together, as far as the registers go
  constexpr int JS = NB * MB <= 4 ? 8 : (NB * MB <= 8 ? 4 : (NB * MB <= 16 ? 2 : 1));
  const int tiles = a.m_tiles * a.n_tiles;
  const uint32_t mine = (wave * NB * MB * 64 + lane) * 16;
  auto slice = [&](int sp) {
    return make_rsrc(a.part + (static_cast<int64_t>(sp) * tiles + tile) * TILE, static_cast<uint32_t>(TILE * 4));
  };
  {
    const rsrc_t p = slice(split);
#pragma unroll
    for (int f = 0; f < NB; ++f)
#pragma unroll
      for (int b = 0; b < MB; ++b)
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[f][b]), p, mine + (f * MB + b) * 1024, 0,
                                               kCoherent);
  }
  mem_done();
  __syncthreads();
  uint32_t* ticket = reinterpret_cast<uint32_t*>(lds);
  if (threadIdx.x == 0)
    *ticket = __hip_atomic_fetch_add(a.arrived + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (*ticket != static_cast<uint32_t>(a.splits - 1)) return false;
  if (threadIdx.x == 0) sync_store(a.arrived + tile, 0u);
#pragma unroll
  for (int f = 0; f < NB; ++f)
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[f][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int sp = 0; sp < a.splits; sp += JS) {
    f32x4 v[JS][NB][MB];
#pragma unroll
    for (int i = 0; i < JS; ++i) {
      const rsrc_t s = slice(min(sp + i, a.splits - 1));
      const uint32_t at = sp + i < a.splits ? mine : kOOB;  // past the last slice: zeros
#pragma unroll
      for (int f = 0; f < NB; ++f)
#pragma unroll
        for (int b = 0; b < MB; ++b)
          v[i][f][b] = __builtin_bit_cast(
              f32x4, __builtin_amdgcn_raw_buffer_load_b128(s, at + (f * MB + b) * 1024, 0, kCoherent));
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < JS; ++i)
#pragma unroll
      for (int f = 0; f < NB; ++f)
#pragma unroll
        for (int b = 0; b < MB; ++b) acc[f][b] += v[i][f][b];
  }
  return true;
}

}  // namespace lin
}  // namespace vt
