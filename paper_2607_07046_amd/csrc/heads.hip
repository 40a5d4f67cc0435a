// Queries and keys of a batch's rows: norms per head and position rotation, into a paged cache
// (vt_paged_append_heads) or into rows (vt_rotate_heads).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "paged_append.hpp"

namespace vt {
namespace pg {

constexpr int HT = 256, HW = HT / kWave;  // threads and waves per workgroup

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

// Eight numbers as e4m3: number / scale, rounded to nearest even, saturating; NaN stays. The quotient is the product
// with the reciprocal and one correction, which leaves a division's result (an exact quotient that lies between
// two e4m3 numbers must not move) but for the sign of a zero: the remainder of -0 is +0, and so would be its quotient.
__device__ __forceinline__ u32x2 scaled_to_f8(const float (&x)[8], float scale, float rcp) {
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float q = x[e] * rcp, d = fmaf(fmaf(-q, scale, x[e]), rcp, q);
    y[e] = copysignf(fabsf(q) > kF8Max ? kF8Max : d, q);
  }
  u32x2 r;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    int t = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w], y[4 * w + 1], 0, false);
    r[w] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2], y[4 * w + 3], t, true);
  }
  return r;
}

// A workgroup takes one row, or for few rows a part of its heads; a wave's turn is 512 numbers of them, 8 per lane.
//   y_i = (inv x_i) g_i cos_i +- (inv x_j) g_j sin_i = (inv x_i) A_i + (inv x_j) B_i,  j the number that i turns with:
// A and B are the same for all of a row's query heads and for all of its key heads and are made once, in LDS.
// With HALVES x_j is in another lane: the head's 16-bit numbers go through LDS, in one 16-byte read where the
// halves are multiples of 8. Keys, values and queries start at whole turns of a wave, so what is done is the
// same for all of its lanes. Every number is read and written once; the next turns' loads are in flight
// while one is computed.
// What bounds it: memory for many rows, the chain row -> sequence -> length -> page -> store for few. Measured: ragged
// prompts, 10310 rows of 96 heads of 128, bf16 into 8-bit, half of each head turning: 91 to 94 us for 422 MB, 4.6 TB/s
// (a wave per row 96 to 164, the slower the more of them were at work; with A, B and the angles in each
// lane's registers 139); 4096 rows of 64 heads without a cache 30 us, 4.5 TB/s; 64 rows of 80 heads 3.6 to
// 4.0 us, one row 2.5 to 3.0 (all in captured graphs).
template <class T, bool PAGED, bool F8, bool HALVES, int D>
__global__ void __launch_bounds__(HT, 6) heads_kernel(HeadsArgs a, Freq f) {
  constexpr int CPR = D / 8, HL = kWave / CPR, B = 2;  // lanes of a head, heads of a turn, turns in flight
  constexpr int CS = 20;  // floats of a lane's A and B in LDS: 16 lanes in different banks
  enum Kind { K, V, Q };
  __shared__ __attribute__((aligned(16))) uint16_t swap[HALVES ? HT * 8 : 8];
  __shared__ float2 angle[D / 2];  // cosine and sine of each pair, times the amplitude
  __shared__ __attribute__((aligned(16))) float coef[2][CPR * CS];  // A and B of keys and queries
  const int c = threadIdx.x % CPR, hl = threadIdx.x % kWave / CPR;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = blockIdx.x, nkv = a.p.n_kv;
  const int tk = (nkv + HL - 1) / HL, tv = PAGED ? 2 * tk : tk, turns = tv + (a.n_q + HL - 1) / HL;
  const int first = blockIdx.y * HW + wave, step = gridDim.y * HW;
  const uint16_t* const row[] = {a.k + r * a.ld_k, PAGED ? a.v + r * a.ld_v : nullptr, a.q + r * a.ld_q};
  u32x4 raw[B];
  auto fetch = [&](int t0) {
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const int t = t0 + b * step;
      const Kind k = t < tk ? K : (t < tv ? V : Q);
      const int j = (t - (k == K ? 0 : (k == V ? tk : tv))) * HL + hl;
      if (t < turns && j < (k == Q ? a.n_q : nkv)) raw[b] = load16((k == K ? row[0] : (k == V ? row[1] : row[2])) + j * D + c * 8);
    }
  };
  // where no row can be padding, the first heads are on their way before the row's place is known
  const bool early = !PAGED || !a.q_begin;
  if (early) fetch(first);
  int64_t pos = 0, at = 0;
  bool bad = false;
  if (PAGED) {
    if (!place_row(a.p, a.q_begin, r, threadIdx.x == 0 && blockIdx.y == 0, pos, at, bad)) return;
  } else {
    pos = a.pos ? static_cast<int64_t>(a.pos[r]) : a.pos0 + r;
    if (pos < 0) return;
  }
  if (!early) fetch(first);

  auto lds_sync = [&]() {  // keeps the compiler to the order of the wave's LDS accesses
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  if (static_cast<int>(threadIdx.x) < a.half) {
    double rev = static_cast<double>(pos) * f.rev[threadIdx.x];
    rev -= rint(rev);
    angle[threadIdx.x] = make_float2(__builtin_amdgcn_cosf(static_cast<float>(rev)) * a.amplitude,
                                     __builtin_amdgcn_sinf(static_cast<float>(rev)) * a.amplitude);
  }
  // the number that number i of a head turns with
  auto partner = [&](int i) { return i >= 2 * a.half ? i : (HALVES ? (i < a.half ? i + a.half : i - a.half) : i ^ 1); };
  const bool aligned = a.half % 8 == 0, all = a.half * 2 == D;
  const int turned = a.half * 2 - c * 8;  // numbers of this lane below it turn
  uint16_t* const head = swap + (HALVES ? (threadIdx.x - c) * 8 : 0);
  auto unpack = [&](const u32x4 w, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) T::unpack2(w[e], v[2 * e], v[2 * e + 1]);
  };
  // the numbers that this lane's numbers turn with
  auto partners = [&](const u32x4 w, float (&o)[8]) {
    if (HALVES) {
      lds_sync();
      *reinterpret_cast<u32x4*>(head + c * 8) = w;
      lds_sync();
      u32x4 p;
      if (aligned) {
        p = *reinterpret_cast<const u32x4*>(head + partner(c * 8));
      } else {
        int i = c * 8;
        asm volatile("" : "+v"(i));  // the places are worked out here, not kept in registers over the loop
#pragma unroll
        for (int e = 0; e < 4; ++e)
          p[e] = head[partner(i + 2 * e)] | static_cast<uint32_t>(head[partner(i + 2 * e + 1)]) << 16;
      }
      unpack(p, o);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) T::unpack2(w[e], o[2 * e + 1], o[2 * e]);
    }
  };
  // A and B: thread t has number t % D of the keys' or the queries'
  __syncthreads();
  if (threadIdx.x < 2 * D) {
    const int k = threadIdx.x / D, i = threadIdx.x % D;
    const uint16_t* gain = k ? a.q_gain : a.k_gain;
    float co = 1.f, si = 0.f;
    if (i < 2 * a.half) {
      const float2 z = angle[HALVES ? (i < a.half ? i : i - a.half) : i / 2];
      co = z.x;
      si = (HALVES ? i < a.half : i % 2 == 0) ? -z.y : z.y;  // u cos - w sin, w cos + u sin
    }
    float g = 1.f, gp = 1.f, unused;
    if (gain) {
      T::unpack2(gain[i], g, unused);
      T::unpack2(gain[partner(i)], gp, unused);
    }
    coef[k][i / 8 * CS + i % 8] = g * co;
    coef[k][i / 8 * CS + 8 + i % 8] = gp * si;
  }
  __syncthreads();

  auto process = [&](auto KIND, int j, u32x4 w) {
    constexpr Kind kind = static_cast<Kind>(decltype(KIND)::value);
    float x[8];
    unpack(w, x);
    if (kind != V) {
      float o[8];
      partners(w, o);
      if (kind == Q ? a.q_gain != nullptr : a.k_gain != nullptr) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
        const float mean = group_sum(ss, CPR) * (1.f / D) + a.eps;
        // Numbers are normalised before they meet A and B: the product of a large one with a large gain, or of two small
        // ones, would leave fp32's range where the result does not.
        if (mean > 1e-30f && mean < 1e37f) {
          const float inv = __builtin_amdgcn_rsqf(mean);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] *= inv;
            o[e] *= inv;
          }
        } else {
          // Squares of bf16 numbers leave fp32's range at 2^64 and 2^-63: such a head's statistics and its first
          // products are taken in double.
          double s2 = 0.0;
#pragma unroll
          for (int e = 0; e < 8; ++e) s2 += static_cast<double>(x[e]) * x[e];
#pragma unroll
          for (int q = CPR / 2; q > 0; q >>= 1) s2 += __shfl_xor(s2, q, kWave);
          const double wide = 1.0 / sqrt(s2 / D + a.eps);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] = static_cast<float>(x[e] * wide);
            o[e] = static_cast<float>(o[e] * wide);
          }
        }
      }
      const f32x4* ab = reinterpret_cast<const f32x4*>(coef[kind == Q] + c * CS);
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        const f32x4 ca = ab[v], cb = ab[2 + v];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int e = 4 * v + q;
          const float own = x[e] * ca[q], both = fmaf(o[e], cb[q], own);
          x[e] = all || e < turned ? both : own;  // (infinity times a zero B would be NaN)
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = T::pack2(x[2 * e], x[2 * e + 1]);
    }
    if (kind == Q) {
      *reinterpret_cast<u32x4*>(a.q_out + r * a.ld_qo + j * D + c * 8) = w;
    } else if (!PAGED) {
      *reinterpret_cast<u32x4*>(a.k_out + r * a.ld_ko + j * D + c * 8) = w;
    } else if (!bad) {
      char* dst = (kind == V ? a.p.v : a.p.k) + at + j * a.p.head;
      if (F8) {
        const float* sc = kind == V ? a.p.v_scale : a.p.k_scale;
        const float scale = sc ? sc[j] : 1.f, rcp = __builtin_amdgcn_rcpf(scale);
        const bool normal = scale > 1e-37f && scale < 1e37f;  // and so is its reciprocal
        *reinterpret_cast<u32x2*>(dst + c * 8) = normal ? scaled_to_f8(x, scale, rcp) : to_f8(x, scale);
      } else {
        *reinterpret_cast<u32x4*>(dst + 16 * c) = w;
      }
    }
  };
  for (int t0 = first; t0 < turns; t0 += B * step) {
    u32x4 now[B];
#pragma unroll
    for (int b = 0; b < B; ++b) now[b] = raw[b];
    fetch(t0 + B * step);
#pragma unroll 1
    for (int b = 0; b < B; ++b) {  // rolled: one copy of the code
      const int t = t0 + b * step;
      if (t >= turns) break;
      const u32x4 w = now[0];
#pragma unroll
      for (int i = 0; i + 1 < B; ++i) now[i] = now[i + 1];
      if (t < tk) {
        const int j = t * HL + hl;
        if (j < nkv) process(std::integral_constant<int, K>{}, j, w);
      } else if (PAGED && t < tv) {
        const int j = (t - tk) * HL + hl;
        if (j < nkv) process(std::integral_constant<int, V>{}, j, w);
      } else {
        const int j = (t - tv) * HL + hl;
        if (j < a.n_q) process(std::integral_constant<int, Q>{}, j, w);
      }
    }
  }
}

namespace {

constexpr int kMaxHeads = 1024, kMaxTokens = 1 << 20;
constexpr int kGroups = 1024;  // workgroups to aim at: four on each compute unit

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

vt_status launch(void (*kernel)(HeadsArgs, Freq), const HeadsArgs& a, const Freq& f, int d, int n_tok, bool paged,
                 void* stream) {
  // a row's turns over several workgroups only while there are few rows
  const int hl = kWave * 8 / d, tk = (a.p.n_kv + hl - 1) / hl, turns = (paged ? 2 * tk : tk) + (a.n_q + hl - 1) / hl;
  const int parts = std::max(1, std::min((turns + HW - 1) / HW, kGroups / n_tok));
  hipLaunchKernelGGL(kernel, dim3(n_tok, parts), dim3(HT), 0, static_cast<hipStream_t>(stream), a, f);
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
  return launch(kernel, a, f, kv->head_dim, io->n_tok, true, stream);
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
  return launch(kernel, a, f, io->head_dim, io->n_tok, false, stream);
}
