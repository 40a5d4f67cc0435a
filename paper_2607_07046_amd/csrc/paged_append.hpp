// Shared by the kernels that store rows in a paged cache (paged.hip, heads.hip): frequencies, a row's
// place, the 8-bit format, and the checks of their entry points.
#pragma once

#include "paged.hpp"

namespace vt {
namespace pg {

// Frequencies of the rotated pairs in revolutions per position, in double: at
// position 10^6 a float's angle would be off by 0.06 rad.
struct Freq {
  double rev[64];
};

// The sequence whose rows end after row r: the number of ends q_begin[1..] that are
// <= r, found by all lanes of a wave 64 probes at a time (two round trips up to
// 4096 sequences).
__device__ __forceinline__ int sequence_of(const int32_t* q_begin, int n, int r) {
  const int lane = threadIdx.x % kWave;
  int lo = 0;
  while (n > kWave) {
    const int step = (n + kWave - 1) / kWave, i = (lane + 1) * step - 1;
    const bool below = i < n && q_begin[lo + i + 1] <= r;
    const int whole = __builtin_popcountll(__builtin_amdgcn_ballot_w64(below));
    lo += whole * step;
    n = min(step, n - whole * step);
  }
  const bool below = lane < n && q_begin[lo + lane + 1] <= r;
  return lo + __builtin_popcountll(__builtin_amdgcn_ballot_w64(below));
}

// Eight numbers as e4m3: value / scale rounded to nearest even, saturating; NaN stays.
__device__ __forceinline__ u32x2 to_f8(const float (&x)[8], float scale) {
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float t = x[e] / scale;
    y[e] = t > kF8Max ? kF8Max : (t < -kF8Max ? -kF8Max : t);
  }
  u32x2 r;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    int t = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w], y[4 * w + 1], 0, false);
    r[w] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2], y[4 * w + 3], t, true);
  }
  return r;
}

// Where row r of an append goes: its position and the byte offset of its slot; ``bad`` where the table or
// the pool has none for it (reported in the status word by the thread that ``report``s). False: the row
// is padding or of an idle slot and is skipped.
__device__ __forceinline__ bool place_row(const Pool& p, const int32_t* q_begin, int r, bool report, int64_t& pos,
                                          int64_t& at, bool& bad) {
  int s = r;
  if (q_begin) {
    s = __builtin_amdgcn_readfirstlane(sequence_of(q_begin, p.n_seqs, r));
    if (s >= p.n_seqs) return false;  // behind the last sequence
    pos = static_cast<int64_t>(p.len[s]) - q_begin[s + 1] + r;
  } else {
    pos = static_cast<int64_t>(p.len[s]) - 1;
  }
  if (pos < 0 || pos > INT32_MAX) return false;
  uint32_t what = pos >= p.capacity ? VT_PAGED_BAD_LEN : 0u;
  int page = 0;
  if (!what) {
    page = p.table[s * p.ld_table + (pos >> p.shift)];
    if (page < 0 || page >= p.n_pages) what = VT_PAGED_BAD_PAGE;
  }
  bad = what != 0;
  if (bad && p.status && report) sync_or(p.status, what);
  at = static_cast<int64_t>(bad ? 0 : page) * p.page + (pos & p.mask) * p.slot;
  return true;
}

inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Checks of the entry points on a paged cache: descriptors, the pool, and a matrix of rows.
vt_status check_paged(const vt_paged_kv* kv, const vt_paged_io* io);
vt_status check_pool(const vt_paged_kv& kv, const vt_paged_io& io);
vt_status check_rows(const void* p, int64_t ld, int64_t n, const char* name);
Pool pool_of(const vt_paged_kv& kv);

}  // namespace pg
}  // namespace vt
