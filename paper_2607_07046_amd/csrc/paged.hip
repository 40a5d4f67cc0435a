// Paged KV cache: append with position rotation, and the host side of all its
// entry points (the attention kernels are in paged_attn.hip and paged_chunk.hip).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "paged.hpp"

namespace vt {
namespace pg {

constexpr int CT = 256;  // threads per workgroup

// Frequencies of the rotated pairs in revolutions per position, in double: at
// position 10^6 a float's angle would be off by 0.06 rad.
struct Freq {
  double rev[64];
};

struct AppendArgs {
  Pool p;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* q_rot;
  int64_t ld_q, ld_k, ld_v, ld_qr;
  const int32_t* q_begin;
  int32_t n_tok, n_q;
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

// A workgroup takes one token: a thread turns the same 8 elements (with HALVES two
// groups of 8, half a head apart) of several heads, so their cosines and sines are
// computed once; its heads are the token's keys, values and queries in turn. Reads
// and writes every byte once: bound by memory for many tokens, by the chain row ->
// sequence -> length -> page -> store for few. Measured: 11 ragged prompts, 10310 tokens of 32 heads of
// 128, bf16 into 8-bit: 82 us for 422 MB, 5.1 TB/s; one token of 8 heads 1.9 us in a captured
// graph, of 64 sequences 2.4; called eagerly 6.9, the host's part of a launch.
template <class T, bool F8, bool HALVES, int D>
__global__ void __launch_bounds__(CT) append_kernel(AppendArgs a, Freq f) {
  constexpr int U = HALVES ? 2 : 1, CPR = D / 8 / U, HL = CT / CPR, NP = 4 * U;
  const int c = threadIdx.x % CPR, hl = threadIdx.x / CPR;
  const int r = blockIdx.x, nkv = a.p.n_kv, rows = 2 * nkv + (a.q ? a.n_q : 0);
  const int first = blockIdx.y * HL + hl, step = gridDim.y * HL;
  int s = r;
  int64_t pos;
  if (a.q_begin) {
    s = __builtin_amdgcn_readfirstlane(sequence_of(a.q_begin, a.p.n_seqs, r));
    if (s >= a.p.n_seqs) return;  // behind the last sequence
    pos = static_cast<int64_t>(a.p.len[s]) - a.q_begin[s + 1] + r;
  } else {
    pos = static_cast<int64_t>(a.p.len[s]) - 1;
  }
  if (pos < 0 || pos > INT32_MAX) return;
  uint32_t bad = pos >= a.p.capacity ? VT_PAGED_BAD_LEN : 0u;
  int page = 0;
  if (!bad) {
    page = a.p.table[s * a.p.ld_table + (pos >> a.p.shift)];
    if (page < 0 || page >= a.p.n_pages) bad = VT_PAGED_BAD_PAGE;
  }
  if (bad && a.p.status && threadIdx.x == 0 && blockIdx.y == 0) sync_or(a.p.status, bad);
  const int64_t at = static_cast<int64_t>(bad ? 0 : page) * a.p.page + (pos & a.p.mask) * a.p.slot;

  float cs[NP], sn[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    double rev = static_cast<double>(pos) * f.rev[c * NP + i];
    rev -= rint(rev);
    cs[i] = __builtin_amdgcn_cosf(static_cast<float>(rev));
    sn[i] = __builtin_amdgcn_sinf(static_cast<float>(rev));
  }
  const bool turned = f.rev[0] != 0.0;
  for (int h = first; h < rows; h += step) {
    const bool is_q = h >= 2 * nkv, is_v = !is_q && h >= nkv;
    const int j = is_q ? h - 2 * nkv : (is_v ? h - nkv : h);
    const uint16_t* src = (is_q ? a.q + r * a.ld_q : (is_v ? a.v + r * a.ld_v : a.k + r * a.ld_k)) + j * D + c * 8;
    float x[U][8];
    u32x4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      raw[u] = load16(src + u * (D / 2));
#pragma unroll
      for (int w = 0; w < 4; ++w) T::unpack2(raw[u][w], x[u][2 * w], x[u][2 * w + 1]);
    }
    const bool turn = turned && !is_v;
    if (turn) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        float& xa = HALVES ? x[0][i] : x[0][2 * i];
        float& xb = HALVES ? x[U - 1][i] : x[0][2 * i + 1];
        const float ya = xa * cs[i] - xb * sn[i], yb = xa * sn[i] + xb * cs[i];
        xa = ya;
        xb = yb;
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int w = 0; w < 4; ++w) raw[u][w] = T::pack2(x[u][2 * w], x[u][2 * w + 1]);
    }
    if (is_q) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        *reinterpret_cast<u32x4*>(a.q_rot + r * a.ld_qr + j * D + c * 8 + u * (D / 2)) = raw[u];
    } else if (!bad) {
      char* dst = (is_v ? a.p.v : a.p.k) + at + j * a.p.head;
      if (F8) {
        const float* sc = is_v ? a.p.v_scale : a.p.k_scale;
        const float scale = sc ? sc[j] : 1.f;
#pragma unroll
        for (int u = 0; u < U; ++u) *reinterpret_cast<u32x2*>(dst + c * 8 + u * (D / 2)) = to_f8(x[u], scale);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u) *reinterpret_cast<u32x4*>(dst + 2 * (c * 8 + u * (D / 2))) = raw[u];
      }
    }
  }
}

}  // namespace pg
}  // namespace vt

using namespace vt;

namespace {

constexpr int kMaxHeads = 1024, kMaxTokens = 1 << 20, kMaxSeqs = 1 << 16;

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

vt_status check_paged(const vt_paged_kv* kv, const vt_paged_io* io) {
  if (!kv || !io) return fail(VT_ERR_ARG, "null cache or io");
  if (io->type != VT_T_F16 && io->type != VT_T_BF16)
    return fail(VT_ERR_ARG, "activation type %d is neither VT_T_F16 nor VT_T_BF16", io->type);
  if (kv->type != io->type && kv->type != VT_T_F8E4M3)
    return fail(VT_ERR_ARG, "cache type %d: the activations' type (%d) or VT_T_F8E4M3", kv->type, io->type);
  if (kv->head_dim != 64 && kv->head_dim != 128)
    return fail(VT_ERR_UNSUPPORTED, "head_dim %d: only 64 and 128 are supported", kv->head_dim);
  if (kv->n_kv_heads < 1 || io->n_q_heads < kv->n_kv_heads || io->n_q_heads % kv->n_kv_heads)
    return fail(VT_ERR_ARG, "n_q_heads %d is not a positive multiple of n_kv_heads %d", io->n_q_heads,
                kv->n_kv_heads);
  if (io->n_q_heads > kMaxHeads) return fail(VT_ERR_UNSUPPORTED, "more than %d query heads", kMaxHeads);
  if (kv->n_seqs < 1 || io->n_tok < 1) return fail(VT_ERR_ARG, "n_seqs %d or n_tok %d < 1", kv->n_seqs, io->n_tok);
  if (kv->n_seqs > kMaxSeqs || io->n_tok > kMaxTokens)
    return fail(VT_ERR_UNSUPPORTED, "more than %d sequences or %d tokens", kMaxSeqs, kMaxTokens);
  if (!io->q_begin && io->n_tok != kv->n_seqs)
    return fail(VT_ERR_ARG, "without q_begin n_tok (%d) must be n_seqs (%d)", io->n_tok, kv->n_seqs);
  return VT_OK;
}

vt_status check_pool(const vt_paged_kv& kv, const vt_paged_io& io) {
  const int64_t elem = kv.type == VT_T_F8E4M3 ? 1 : 2, d = kv.head_dim;
  if (!kv.k || !kv.v) return fail(VT_ERR_ARG, "null pool");
  if (!aligned16(kv.k) || !aligned16(kv.v)) return fail(VT_ERR_ALIGN, "pool not 16-byte aligned");
  if (kv.page_size < 1 || kv.page_size > 32768 || (kv.page_size & (kv.page_size - 1)))
    return fail(VT_ERR_ARG, "page_size %d is not a power of two in 1..32768", kv.page_size);
  if (kv.n_pages < 1) return fail(VT_ERR_ARG, "n_pages %d < 1", kv.n_pages);
  const struct {
    int64_t v;
    bool used;
    const char* name;
  } st[] = {{kv.page_stride, kv.n_pages > 1, "page_stride"},
            {kv.head_stride, kv.n_kv_heads > 1, "head_stride"},
            {kv.slot_stride, true, "slot_stride"}};
  for (const auto& x : st) {
    if (x.v < (x.used ? d : 0) || x.v > (int64_t(1) << 40))
      return fail(VT_ERR_ARG, "%s %lld is below head_dim or above 2^40", x.name, static_cast<long long>(x.v));
    if (x.v * elem % 16) return fail(VT_ERR_ALIGN, "%s is not a multiple of 16 bytes", x.name);
  }
  if ((static_cast<int64_t>(kv.n_pages) - 1) > (int64_t(1) << 46) / std::max<int64_t>(kv.page_stride * elem, 1))
    return fail(VT_ERR_UNSUPPORTED, "pages span more than 2^46 bytes");
  // a tile's rows are addressed by 32-bit offsets
  if (kv.slot_stride * elem > (int64_t(1) << 24))
    return fail(VT_ERR_UNSUPPORTED, "slot_stride of more than 2^24 bytes");
  if (!kv.table || !kv.len) return fail(VT_ERR_ARG, "null table or len");
  if (kv.max_pages < 1 || kv.ld_table < kv.max_pages)
    return fail(VT_ERR_ARG, "max_pages %d < 1 or ld_table %lld below it", kv.max_pages,
                static_cast<long long>(kv.ld_table));
  if (!aligned4(kv.table) || !aligned4(kv.len) || !aligned4(kv.k_scale) || !aligned4(kv.v_scale) ||
      !aligned4(kv.status) || !aligned4(io.q_begin))
    return fail(VT_ERR_ALIGN, "table, len, scale, status or q_begin not 4-byte aligned");
  return VT_OK;
}

vt_status check_rows(const void* p, int64_t ld, int64_t n, const char* name) {
  if (!p) return fail(VT_ERR_ARG, "%s is NULL", name);
  if (!aligned16(p) || ld % 8) return fail(VT_ERR_ALIGN, "%s not 16-byte aligned or its ld not a multiple of 8", name);
  if (ld < n || ld > (int64_t(1) << 32))
    return fail(VT_ERR_ARG, "ld of %s (%lld) below %lld or above 2^32", name, static_cast<long long>(ld),
                static_cast<long long>(n));
  return VT_OK;
}

pg::Pool pool_of(const vt_paged_kv& kv) {
  const int64_t elem = kv.type == VT_T_F8E4M3 ? 1 : 2;
  int shift = 0;
  while ((1 << shift) < kv.page_size) ++shift;
  pg::Pool p{};
  p.k = static_cast<char*>(kv.k);
  p.v = static_cast<char*>(kv.v);
  p.page = kv.page_stride * elem;
  p.head = kv.head_stride * elem;
  p.slot = kv.slot_stride * elem;
  p.table = kv.table;
  p.ld_table = kv.ld_table;
  p.len = kv.len;
  p.status = kv.status;
  const bool f8 = kv.type == VT_T_F8E4M3;
  p.k_scale = f8 ? kv.k_scale : nullptr;
  p.v_scale = f8 ? kv.v_scale : nullptr;
  p.n_pages = kv.n_pages;
  p.shift = shift;
  p.mask = kv.page_size - 1;
  p.capacity = static_cast<int32_t>(
      std::min<int64_t>(static_cast<int64_t>(kv.max_pages) * kv.page_size, pg::kMaxPositions));
  p.n_kv = kv.n_kv_heads;
  p.n_seqs = kv.n_seqs;
  return p;
}

// Rows of an attention tile, by the mean rows of a sequence (what else the host could
// know of a batch is on the device): 16 (attn_rows_kernel), 64 or 128 (attn_chunk_kernel).
// All take every batch; keys and values pass once per tile and a tile's rows cost the
// same whether they are there or not. Measured with 16 / 64 / 128 (us), rows per sequence:
// 16 sequences of 4096 positions, 8 heads: 16 rows 54 / 60 / 70, 32 rows 61 / 63 / 71, 64 rows 97 /
// 63 / 72, 128 rows 168 / 87 / 75; with 8-bit caches 29 / 53 / 61, 36 / 53 / 59, 58 / 53 / 61, 110 / 87 / 64;
// one of 32768: 32 rows 32 / 41 / 54, 64 rows 49 / 42 / 55, 128 rows 83 / 50 / 56 (a single long one
// is the exception: the host does not know lengths).
// The mean misjudges batches of unlike sequences: 255 single tokens over 1024 positions and a prompt of
// 4096 (8 heads, mean 17) take 348 us together, 181 + 66 in two calls; 64 over 4096 and a prompt of 2048
// (group 8, mean 260) 306 and 191 + 104, with an 8-bit cache 256 and 101 + 108. So does a wide group of a single token
// (no q_begin: 16 rows, whose product keeps its remainder): 16 sequences of 4096 positions, 8 heads, group 64
// 84 us and 51 as chunks of one token, group 128 159 and 71.
int tile_rows(const vt_paged_kv& kv, const vt_paged_io& io) {
  if (!io.q_begin) return 16;
  const double rows = static_cast<double>(io.n_tok) * (io.n_q_heads / kv.n_kv_heads) / kv.n_seqs;
  return rows <= 32 ? 16 : (rows <= 64 ? 64 : 128);
}

// Fewer than 2 * kTarget pieces of the largest tile: the same for every batch.
size_t workspace_bytes(const vt_paged_kv& kv) {
  return pg::kSyncBytes + 2 * static_cast<size_t>(pg::kTarget) * pg::part_bytes(128, kv.head_dim);
}

vt_status attend(const vt_paged_kv* kv, const vt_paged_io* io, float scale, int32_t window, void* ws, size_t ws_bytes,
                 void* stream) {
  vt_status st = check_paged(kv, io);
  if (st == VT_OK) st = check_pool(*kv, *io);
  if (st != VT_OK) return st;
  const int64_t width = static_cast<int64_t>(io->n_q_heads) * kv->head_dim;
  if ((st = check_rows(io->q_rot, io->ld_qr, width, "q_rot")) != VT_OK) return st;
  if ((st = check_rows(io->out, io->ld_out, width, "out")) != VT_OK) return st;
  if (!aligned4(io->lse)) return fail(VT_ERR_ALIGN, "lse not 4-byte aligned");
  if (!(scale >= 0.f) || !std::isfinite(scale)) return fail(VT_ERR_ARG, "scale must be finite and >= 0");
  if (window < 0) return fail(VT_ERR_ARG, "window %d < 0", window);
  if (!ws || !aligned16(ws)) return fail(ws ? VT_ERR_ALIGN : VT_ERR_WORKSPACE, "workspace missing or misaligned");
  if (ws_bytes < workspace_bytes(*kv))
    return fail(VT_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, workspace_bytes(*kv));
  pg::AttnArgs a{};
  a.p = pool_of(*kv);
  a.q = static_cast<const uint16_t*>(io->q_rot);
  a.ld_q = io->ld_qr;
  a.out = static_cast<uint16_t*>(io->out);
  a.ld_out = io->ld_out;
  a.lse = io->lse;
  a.q_begin = io->q_begin;
  a.n_tok = io->n_tok;
  a.n_q = io->n_q_heads;
  a.group = io->n_q_heads / kv->n_kv_heads;
  a.window = window;
  a.scale2 = static_cast<float>((scale > 0.f ? scale : 1.0 / std::sqrt(static_cast<double>(kv->head_dim))) *
                                1.4426950408889634);
  a.arrived = static_cast<uint32_t*>(ws);
  a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + pg::kSyncBytes);
  const bool f8 = kv->type == VT_T_F8E4M3;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int tile = tile_rows(*kv, *io);
  a.target = tile == 128 ? pg::kTarget : pg::kTarget / 2;
  a.min_blocks = tile == 16 ? 2 : 4;
  const int64_t grid = pg::grid_of(a, tile);
  if (grid >= (int64_t(1) << 24))  // 2^32 threads
    return fail(VT_ERR_UNSUPPORTED, "%lld tiles of rows: fewer tokens, heads or sequences per call",
                static_cast<long long>(grid));
  hipError_t e = tile == 16 ? pg::launch_rows(a, io->type, f8, kv->head_dim, s)
                            : pg::launch_chunk(a, io->type, f8, kv->head_dim, tile, s);
  return e == hipSuccess ? VT_OK : fail(VT_ERR_HIP, "attention launch: %s", hipGetErrorString(e));
}

}  // namespace

extern "C" vt_status vt_paged_append(const vt_paged_kv* kv, const vt_paged_io* io, float rope_base, uint32_t flags,
                                     void* stream) {
  clear_error();
  vt_status st = check_paged(kv, io);
  if (st == VT_OK) st = check_pool(*kv, *io);
  if (st != VT_OK) return st;
  const int64_t d = kv->head_dim, qw = io->n_q_heads * d, kw = kv->n_kv_heads * d;
  if ((st = check_rows(io->k, io->ld_k, kw, "k")) != VT_OK) return st;
  if ((st = check_rows(io->v, io->ld_v, kw, "v")) != VT_OK) return st;
  if (io->q) {
    if ((st = check_rows(io->q, io->ld_q, qw, "q")) != VT_OK) return st;
    if ((st = check_rows(io->q_rot, io->ld_qr, qw, "q_rot")) != VT_OK) return st;
    if (io->q == io->q_rot && io->ld_q != io->ld_qr) return fail(VT_ERR_ARG, "q_rot equals q at another ld");
  }
  if (flags & ~VT_ROPE_HALVES) return fail(VT_ERR_ARG, "unknown flag bits 0x%x", flags);
  if (!(rope_base >= 0.f) || !std::isfinite(rope_base))
    return fail(VT_ERR_ARG, "rope_base must be finite and >= 0");
  pg::AppendArgs a{};
  a.p = pool_of(*kv);
  a.q = static_cast<const uint16_t*>(io->q);
  a.k = static_cast<const uint16_t*>(io->k);
  a.v = static_cast<const uint16_t*>(io->v);
  a.q_rot = static_cast<uint16_t*>(io->q_rot);
  a.ld_q = io->ld_q;
  a.ld_k = io->ld_k;
  a.ld_v = io->ld_v;
  a.ld_qr = io->ld_qr;
  a.q_begin = io->q_begin;
  a.n_tok = io->n_tok;
  a.n_q = io->n_q_heads;
  pg::Freq f{};
  if (rope_base > 0.f) {
    // powers by products with 64 bits of mantissa: off by 2^-57 at most, in the time of one pow
    const long double step = std::pow(static_cast<long double>(rope_base), -2.0L / static_cast<long double>(d));
    long double rev = 0.159154943091895335768883763372514362L;  // 1 / (2 pi)
    for (int i = 0; i < d / 2; ++i, rev *= step) f.rev[i] = static_cast<double>(rev);
  }
  // heads of a token over several workgroups only while there are few tokens
  const int halves = flags & VT_ROPE_HALVES ? 1 : 0, hl = pg::CT / (static_cast<int>(d) / 8 >> halves);
  const int rows = 2 * kv->n_kv_heads + (io->q ? io->n_q_heads : 0), parts = (rows + hl - 1) / hl;
  const dim3 grid(io->n_tok, io->n_tok >= 512 ? 1 : parts);
  const bool f8 = kv->type == VT_T_F8E4M3;
  auto pick = [&](auto T) -> void (*)(pg::AppendArgs, pg::Freq) {
    using X = decltype(T);
    if (d == 128) {
      if (f8) return halves ? pg::append_kernel<X, true, true, 128> : pg::append_kernel<X, true, false, 128>;
      return halves ? pg::append_kernel<X, false, true, 128> : pg::append_kernel<X, false, false, 128>;
    }
    if (f8) return halves ? pg::append_kernel<X, true, true, 64> : pg::append_kernel<X, true, false, 64>;
    return halves ? pg::append_kernel<X, false, true, 64> : pg::append_kernel<X, false, false, 64>;
  };
  auto* kernel = io->type == VT_T_F16 ? pick(pg::Half{}) : pick(pg::BFloat{});
  hipLaunchKernelGGL(kernel, grid, dim3(pg::CT), 0, static_cast<hipStream_t>(stream), a, f);
  hipError_t e = hipGetLastError();
  return e == hipSuccess ? VT_OK : fail(VT_ERR_HIP, "append launch: %s", hipGetErrorString(e));
}

extern "C" vt_status vt_paged_workspace_size(const vt_paged_kv* kv, const vt_paged_io* io, size_t* bytes) {
  clear_error();
  if (!bytes) return fail(VT_ERR_ARG, "null bytes");
  vt_status st = check_paged(kv, io);
  if (st != VT_OK) return st;
  *bytes = workspace_bytes(*kv);
  return VT_OK;
}

extern "C" vt_status vt_paged_decode_attn(const vt_paged_kv* kv, const vt_paged_io* io, float scale, int32_t window,
                                          void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  if (io && io->q_begin) return fail(VT_ERR_ARG, "q_begin must be NULL: one token per sequence");
  return attend(kv, io, scale, window, ws, ws_bytes, stream);
}

extern "C" vt_status vt_paged_chunk_attn(const vt_paged_kv* kv, const vt_paged_io* io, float scale, int32_t window,
                                         void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  return attend(kv, io, scale, window, ws, ws_bytes, stream);
}
