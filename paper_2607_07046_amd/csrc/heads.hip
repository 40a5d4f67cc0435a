// Queries and keys of a batch's rows: norms per head and position rotation, into a paged cache
// (vt_paged_append_heads) or into rows (vt_rotate_heads).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "paged.hpp"

namespace vt {
namespace pg {

constexpr int HT = 256;  // threads per workgroup

struct HeadsArgs {
  Pool p;                // paged only; n_kv key heads either way
  const int32_t* q_begin;
  const int32_t* pos;    // rows only, nullable: pos0 + row
  int64_t pos0;
  const uint16_t *q, *k, *v;
  uint16_t *q_out, *k_out;
  int64_t ld_q, ld_k, ld_v, ld_qo, ld_ko;
  const uint16_t *q_gain, *k_gain;  // nullable: not normalised
  float eps, amplitude;
  int32_t n_q, half;     // query heads (0: none); pairs that turn
};

// A workgroup takes one row: 8 (head size 64) or 16 lanes a head, 8 numbers each, so a lane's part of the rotation is the
// same for all heads that it gets and its angles are computed once. The head's sum of squares is
// a sum over its lanes; with HALVES the number that a number turns with is in another lane and comes
// through the wave's own piece of LDS (9 floats a lane, so that neither side has bank conflicts), wherever
// the turned part of a head ends. Every number is read and written once; a lane's next heads are in flight
// while one is computed.
template <class T, bool PAGED, bool F8, bool HALVES, int D>
__global__ void __launch_bounds__(HT) heads_kernel(HeadsArgs a, Freq f) {
  constexpr int CPR = D / 8, HL = HT / CPR, B = 4;
  __shared__ float swap[HALVES ? HT * 9 : 1];
  const int c = threadIdx.x % CPR, hl = threadIdx.x / CPR;
  const int r = blockIdx.x, nkv = a.p.n_kv, nk = PAGED ? 2 * nkv : nkv, heads = nk + a.n_q;
  const int first = blockIdx.y * HL + hl, step = gridDim.y * HL;
  int64_t pos = 0, at = 0;
  bool bad = false;
  if (PAGED) {
    if (!place_row(a.p, a.q_begin, r, threadIdx.x == 0 && blockIdx.y == 0, pos, at, bad)) return;
  } else {
    pos = a.pos ? static_cast<int64_t>(a.pos[r]) : a.pos0 + r;
    if (pos < 0) return;
  }
  u32x4 gq = {0u, 0u, 0u, 0u}, gk = gq;
  if (a.q_gain) gq = load16(a.q_gain + c * 8);
  if (a.k_gain) gk = load16(a.k_gain + c * 8);
  // what number e turns by, and with HALVES where its partner is
  constexpr int NP = HALVES ? 8 : 4;
  float cs[NP], sn[NP];
  int partner[HALVES ? 8 : 1];
  const int lane0 = threadIdx.x - c;
#pragma unroll
  for (int e = 0; e < NP; ++e) {
    const int i = HALVES ? c * 8 + e : c * 4 + e;  // a number of the head, or a pair
    const int pair = HALVES && i >= a.half ? i - a.half : i;
    cs[e] = 1.f;
    sn[e] = 0.f;
    if (HALVES) partner[e] = 0;
    if (pair < a.half) {
      double rev = static_cast<double>(pos) * f.rev[pair];
      rev -= rint(rev);
      cs[e] = __builtin_amdgcn_cosf(static_cast<float>(rev)) * a.amplitude;
      sn[e] = __builtin_amdgcn_sinf(static_cast<float>(rev)) * a.amplitude;
      if (HALVES) {
        const int o = i < a.half ? i + a.half : i - a.half;
        partner[e] = (lane0 + o / 8) * 9 + o % 8;
        if (i < a.half) sn[e] = -sn[e];  // u cos - w sin, w cos + u sin
      }
    }
  }
  const int turned = a.half * 2 - c * 8;  // numbers of this lane below it turn

  auto source = [&](int h) {
    if (h >= nk) return a.q + r * a.ld_q + (h - nk) * D + c * 8;
    if (PAGED && h >= nkv) return a.v + r * a.ld_v + (h - nkv) * D + c * 8;
    return a.k + r * a.ld_k + h * D + c * 8;
  };
  auto process = [&](int h, u32x4 raw) {
    const bool is_q = h >= nk, is_v = PAGED && !is_q && h >= nkv;
    const int j = is_q ? h - nk : (is_v ? h - nkv : h);
    float x[8];
#pragma unroll
    for (int w = 0; w < 4; ++w) T::unpack2(raw[w], x[2 * w], x[2 * w + 1]);
    if (!is_v) {
      if (is_q ? a.q_gain : a.k_gain) {
        float ss = 0.f, g[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
        ss = group_sum(ss, CPR);
        const u32x4 gw = is_q ? gq : gk;
#pragma unroll
        for (int w = 0; w < 4; ++w) T::unpack2(gw[w], g[2 * w], g[2 * w + 1]);
        const float mean = ss * (1.f / D) + a.eps;
        if (mean > 1e-30f && mean < 1e37f) {
          const float inv = 1.f / sqrtf(mean);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * g[e];
        } else {  // squares of bf16 numbers that leave fp32's range
          double s2 = 0.0;
#pragma unroll
          for (int e = 0; e < 8; ++e) s2 += static_cast<double>(x[e]) * x[e];
#pragma unroll
          for (int o = CPR / 2; o > 0; o >>= 1) s2 += __shfl_xor(s2, o, kWave);
          const double inv = 1.0 / sqrt(s2 / D + a.eps);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = static_cast<float>(x[e] * inv * g[e]);
        }
      }
      if (HALVES) {
        float* mine = swap + threadIdx.x * 9;
#pragma unroll
        for (int e = 0; e < 8; ++e) mine[e] = x[e];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = swap[partner[e]];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < turned ? x[e] * cs[e] + o[e] * sn[e] : x[e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float u = x[2 * e], w = x[2 * e + 1];
          if (2 * e < turned) {
            x[2 * e] = u * cs[e] - w * sn[e];
            x[2 * e + 1] = u * sn[e] + w * cs[e];
          }
        }
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) raw[w] = T::pack2(x[2 * w], x[2 * w + 1]);
    }
    if (is_q) {
      *reinterpret_cast<u32x4*>(a.q_out + r * a.ld_qo + j * D + c * 8) = raw;
    } else if (!PAGED) {
      *reinterpret_cast<u32x4*>(a.k_out + r * a.ld_ko + j * D + c * 8) = raw;
    } else if (!bad) {
      char* dst = (is_v ? a.p.v : a.p.k) + at + j * a.p.head;
      if (F8) {
        const float* sc = is_v ? a.p.v_scale : a.p.k_scale;
        *reinterpret_cast<u32x2*>(dst + c * 8) = to_f8(x, sc ? sc[j] : 1.f);
      } else {
        *reinterpret_cast<u32x4*>(dst + 16 * c) = raw;
      }
    }
  };
  for (int h = first; h < heads; h += B * step) {
    u32x4 raw[B];
#pragma unroll
    for (int b = 0; b < B; ++b)
      if (h + b * step < heads) raw[b] = load16(source(h + b * step));
#pragma unroll
    for (int b = 0; b < B; ++b)
      if (h + b * step < heads) process(h + b * step, raw[b]);
  }
}

namespace {

constexpr int kMaxHeads = 1024, kMaxTokens = 1 << 20;

// Revolutions per position of a head's pairs; their number in ``half``.
vt_status frequencies(const vt_rope* rope, int head_dim, Freq* f, int* half, float* amplitude) {
  *half = 0;
  *amplitude = 1.f;
  if (!rope) return VT_OK;
  const int dims = rope->dims ? rope->dims : head_dim;
  if (dims < 0 || dims % 2 || dims > head_dim)
    return fail(VT_ERR_ARG, "rope dims %d: even, up to head_dim %d", rope->dims, head_dim);
  if (rope->flags & ~VT_ROPE_HALVES) return fail(VT_ERR_ARG, "unknown rope flag bits 0x%x", rope->flags);
  if (!(rope->base >= 0.f) || !std::isfinite(rope->base)) return fail(VT_ERR_ARG, "rope base must be finite and >= 0");
  if (!std::isfinite(rope->factor) || !(rope->factor == 0.f || rope->factor >= 1.f))
    return fail(VT_ERR_ARG, "rope factor must be 0 or finite and >= 1");
  if (!(rope->low >= 0.f) || !std::isfinite(rope->low) || !(rope->high >= 0.f) || !std::isfinite(rope->high))
    return fail(VT_ERR_ARG, "rope low and high must be finite and >= 0");
  if ((rope->low > 0.f || rope->high > 0.f) && (rope->high <= rope->low || rope->context < 1))
    return fail(VT_ERR_ARG, "rope high must be above low, and context >= 1 with them");
  if (!(rope->amplitude >= 0.f) || !std::isfinite(rope->amplitude))
    return fail(VT_ERR_ARG, "rope amplitude must be finite and >= 0");
  if (rope->amplitude > 0.f) *amplitude = rope->amplitude;
  if (rope->base == 0.f) return VT_OK;
  *half = dims / 2;
  // powers by products with 64 bits of mantissa, off by 2^-57 at most
  const long double step = std::pow(static_cast<long double>(rope->base), -2.0L / static_cast<long double>(dims));
  const long double factor = rope->factor > 1.f ? rope->factor : 1.f;
  long double rev = 0.159154943091895335768883763372514362L;  // 1 / (2 pi)
  for (int i = 0; i < dims / 2; ++i, rev *= step) {
    long double keep = 0.0L;
    if (rope->high > 0.f)
      keep = std::min(1.0L, std::max(0.0L, (rev * rope->context - rope->low) /
                                               (static_cast<long double>(rope->high) - rope->low)));
    f->rev[i] = static_cast<double>(rev * (keep + (1.0L - keep) / factor));
  }
  return VT_OK;
}

vt_status check_norm(const vt_head_norm* norm) {
  if (!norm) return VT_OK;
  if (!aligned16(norm->q_gain) || !aligned16(norm->k_gain)) return fail(VT_ERR_ALIGN, "gains not 16-byte aligned");
  if (!(norm->eps >= 0.f) || !std::isfinite(norm->eps)) return fail(VT_ERR_ARG, "eps must be finite and >= 0");
  return VT_OK;
}

void take_norm(HeadsArgs& a, const vt_head_norm* norm) {
  if (!norm) return;
  a.q_gain = static_cast<const uint16_t*>(norm->q_gain);
  a.k_gain = static_cast<const uint16_t*>(norm->k_gain);
  a.eps = norm->eps;
}

template <class T, bool PAGED, bool F8>
auto pick(int d, bool halves) -> void (*)(HeadsArgs, Freq) {
  if (d == 128) return halves ? heads_kernel<T, PAGED, F8, true, 128> : heads_kernel<T, PAGED, F8, false, 128>;
  return halves ? heads_kernel<T, PAGED, F8, true, 64> : heads_kernel<T, PAGED, F8, false, 64>;
}

vt_status launch(void (*kernel)(HeadsArgs, Freq), const HeadsArgs& a, const Freq& f, int d, int n_tok, int heads,
                 void* stream) {
  // heads of a row over several workgroups only while there are few rows
  const int hl = HT / (d / 8), parts = (heads + hl - 1) / hl;
  hipLaunchKernelGGL(kernel, dim3(n_tok, n_tok >= 512 ? 1 : parts), dim3(HT), 0, static_cast<hipStream_t>(stream), a, f);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? VT_OK : fail(VT_ERR_HIP, "heads launch: %s", hipGetErrorString(e));
}

}  // namespace
}  // namespace pg
}  // namespace vt

using namespace vt;
using namespace vt::pg;

extern "C" vt_status vt_paged_append_heads(const vt_paged_kv* kv, const vt_paged_io* io, const vt_head_norm* norm,
                                           const vt_rope* rope, void* stream) {
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
  if ((st = check_norm(norm)) != VT_OK) return st;
  HeadsArgs a{};
  Freq f{};
  if ((st = frequencies(rope, kv->head_dim, &f, &a.half, &a.amplitude)) != VT_OK) return st;
  take_norm(a, norm);
  a.p = pool_of(*kv);
  a.q_begin = io->q_begin;
  a.q = static_cast<const uint16_t*>(io->q);
  a.k = static_cast<const uint16_t*>(io->k);
  a.v = static_cast<const uint16_t*>(io->v);
  a.q_out = static_cast<uint16_t*>(io->q_rot);
  a.ld_q = io->ld_q;
  a.ld_k = io->ld_k;
  a.ld_v = io->ld_v;
  a.ld_qo = io->ld_qr;
  a.n_q = io->q ? io->n_q_heads : 0;
  const bool f8 = kv->type == VT_T_F8E4M3, halves = rope && (rope->flags & VT_ROPE_HALVES);
  auto* kernel = io->type == VT_T_F16
                     ? (f8 ? pick<Half, true, true>(kv->head_dim, halves) : pick<Half, true, false>(kv->head_dim, halves))
                     : (f8 ? pick<BFloat, true, true>(kv->head_dim, halves) : pick<BFloat, true, false>(kv->head_dim, halves));
  return launch(kernel, a, f, kv->head_dim, io->n_tok, 2 * kv->n_kv_heads + a.n_q, stream);
}

extern "C" vt_status vt_rotate_heads(const vt_heads_io* io, const vt_head_norm* norm, const vt_rope* rope,
                                     void* stream) {
  clear_error();
  if (!io) return fail(VT_ERR_ARG, "null io");
  if (io->type != VT_T_F16 && io->type != VT_T_BF16)
    return fail(VT_ERR_ARG, "type %d is neither VT_T_F16 nor VT_T_BF16", io->type);
  if (io->head_dim != 64 && io->head_dim != 128)
    return fail(VT_ERR_UNSUPPORTED, "head_dim %d: only 64 and 128 are supported", io->head_dim);
  if (io->n_tok < 1) return fail(VT_ERR_ARG, "n_tok %d < 1", io->n_tok);
  if (io->n_tok > kMaxTokens) return fail(VT_ERR_UNSUPPORTED, "more than %d tokens", kMaxTokens);
  if (io->n_q_heads < 0 || io->n_k_heads < 0 || io->n_q_heads + static_cast<int64_t>(io->n_k_heads) < 1)
    return fail(VT_ERR_ARG, "n_q_heads %d and n_k_heads %d: none negative, not both 0", io->n_q_heads, io->n_k_heads);
  if (io->n_q_heads > kMaxHeads || io->n_k_heads > kMaxHeads)
    return fail(VT_ERR_UNSUPPORTED, "more than %d heads", kMaxHeads);
  if (!aligned4(io->pos)) return fail(VT_ERR_ALIGN, "pos not 4-byte aligned");
  if (!io->pos && (io->pos0 < 0 || static_cast<int64_t>(io->pos0) + io->n_tok - 1 > INT32_MAX))
    return fail(VT_ERR_ARG, "positions %d.. are negative or pass 2^31 - 1", io->pos0);
  const struct {
    int n;
    const void *in, *out;
    int64_t ld_in, ld_out;
    const char *in_name, *out_name;
  } parts[] = {{io->n_q_heads, io->q, io->q_out, io->ld_q, io->ld_qo, "q", "q_out"},
               {io->n_k_heads, io->k, io->k_out, io->ld_k, io->ld_ko, "k", "k_out"}};
  vt_status st;
  for (const auto& x : parts) {
    if (x.n == 0) continue;
    const int64_t w = static_cast<int64_t>(x.n) * io->head_dim;
    if ((st = check_rows(x.in, x.ld_in, w, x.in_name)) != VT_OK) return st;
    if ((st = check_rows(x.out, x.ld_out, w, x.out_name)) != VT_OK) return st;
    if (x.in == x.out && x.ld_in != x.ld_out) return fail(VT_ERR_ARG, "%s equals %s at another ld", x.out_name, x.in_name);
  }
  if ((st = check_norm(norm)) != VT_OK) return st;
  HeadsArgs a{};
  Freq f{};
  if ((st = frequencies(rope, io->head_dim, &f, &a.half, &a.amplitude)) != VT_OK) return st;
  take_norm(a, norm);
  a.pos = io->pos;
  a.pos0 = io->pos0;
  a.q = static_cast<const uint16_t*>(io->q);
  a.k = static_cast<const uint16_t*>(io->k);
  a.q_out = static_cast<uint16_t*>(io->q_out);
  a.k_out = static_cast<uint16_t*>(io->k_out);
  a.ld_q = io->ld_q;
  a.ld_k = io->ld_k;
  a.ld_qo = io->ld_qo;
  a.ld_ko = io->ld_ko;
  a.n_q = io->n_q_heads;
  a.p.n_kv = io->n_k_heads;
  const bool halves = rope && (rope->flags & VT_ROPE_HALVES);
  auto* kernel = io->type == VT_T_F16 ? pick<Half, false, false>(io->head_dim, halves)
                                      : pick<BFloat, false, false>(io->head_dim, halves);
  return launch(kernel, a, f, io->head_dim, io->n_tok, io->n_k_heads + io->n_q_heads, stream);
}
