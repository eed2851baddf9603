// Token log-probabilities of rows of logits and their backward.
//
// Forward, per row with z = scale x: one pass over the logits with the running
// maximum m of x, S = sum 2^u and, for the entropy, T = sum 2^u u, where
// u = (x - m) scale log2e (the difference first: exact near the maximum, and
// no overflow at the lowest values of the type).  Then
//   lse = scale m + ln S,  logp = u_y ln2 - ln S,  H = ln S - ln2 T / S.
// Backward: dx = scale (a (1[v = y] - p) - b p (log p + H)), element by element.
#include <math.h>

#include "../../include/bgpo.h"
#include "../../include/bgpo_policy.h"
#include "common.hpp"
#include "spans.hpp"

namespace bgpo {

// 16 bytes of a row at any alignment the element type allows (global memory
// takes unaligned accesses; a row of odd length starts off 16 bytes).
typedef uint32_t raw16 __attribute__((ext_vector_type(4), aligned(2), may_alias));

template <typename T>
struct Elem;
template <>
struct Elem<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ float one(uint16_t v) { return bf16_to_f32(v); }
  static __device__ __forceinline__ uint16_t round(float v) { return f32_to_bf16(v); }
  static __device__ __forceinline__ void unpack(const raw16& r, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(r[i] << 16);
      f[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ raw16 pack(const float (&f)[8]) {
    raw16 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    return r;
  }
};
template <>
struct Elem<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float one(float v) { return v; }
  static __device__ __forceinline__ float round(float v) { return v; }
  static __device__ __forceinline__ void unpack(const raw16& r, float (&f)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(r[i]);
  }
  static __device__ __forceinline__ raw16 pack(const float (&f)[4]) {
    raw16 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(f[i]);
    return r;
  }
};

// Statistics of a set of logits: maximum, S and T against it.
struct RowStats {
  float m, s, t;
};

// 2^-16384 = 0 and 0 * -16384 = 0: stands for the exponent of a logit of -inf
// where it is multiplied (0 * -inf is NaN).
constexpr float kNoExponent = -16384.f;

// the reference that exponents are taken against: 0 where nothing finite is
// known yet (-inf - -inf is NaN)
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }

template <bool ENT>
__device__ __forceinline__ void rescale(RowStats& a, float m, float ref, float c) {
  const float u = (a.m - ref) * c, f = __builtin_amdgcn_exp2f(u);
  if (ENT) a.t = f * (a.t + fmaxf(u, kNoExponent) * a.s);
  a.s *= f;
  a.m = m;
}

template <bool ENT>
__device__ __forceinline__ void join(RowStats& a, RowStats b, float c) {
  const float m = fmaxf(a.m, b.m), ref = reference(m);
  rescale<ENT>(a, m, ref, c);
  rescale<ENT>(b, m, ref, c);
  a.s += b.s;
  if (ENT) a.t += b.t;
}

template <bool ENT, int N>
__device__ __forceinline__ void add(RowStats& a, const float (&x)[N], float c) {
  float m = a.m;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
  const float ref = reference(m);
  rescale<ENT>(a, m, ref, c);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float u = (x[i] - ref) * c, e = __builtin_amdgcn_exp2f(u);
    a.s += e;
    if (ENT) a.t = fmaf(e, fmaxf(u, kNoExponent), a.t);
  }
}

template <bool ENT>
__device__ __forceinline__ RowStats join_wave(RowStats a, float c) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    RowStats b;
    b.m = __shfl_xor(a.m, off, 64);
    b.s = __shfl_xor(a.s, off, 64);
    b.t = ENT ? __shfl_xor(a.t, off, 64) : 0.f;
    join<ENT>(a, b, c);
  }
  return a;
}

struct LogitRows {
  const void* x;
  const int32_t* targets;
  const uint8_t* mask;
  int64_t rows, ld;
  int V;
  float scale;
  __device__ bool masked(int64_t r, int y) const { return y < 0 || (mask && !mask[r]); }
};

// the row's outputs from its statistics
template <typename T, bool ENT>
__device__ void finish_row(const LogitRows& p, int64_t r, int y, const RowStats& a, float* logp,
                           float* entropy, float* lse) {
  const float ls = a.s > 0.f ? logf(a.s) : NAN;
  float xy = NAN;
  if (y < p.V) xy = Elem<T>::one(static_cast<const T*>(p.x)[r * p.ld + y]);
  logp[r] = fmaf(xy - reference(a.m), p.scale, -ls);
  if (lse) lse[r] = fmaf(p.scale, reference(a.m), ls);
  if (ENT) entropy[r] = ls - kLn2 * (a.t / a.s);
}

// One workgroup per row.
template <typename T, bool ENT>
__global__ __launch_bounds__(256) void k_logits_logp(LogitRows p, float* __restrict__ logp,
                                                     float* __restrict__ entropy,
                                                     float* __restrict__ lse) {
  constexpr int N = Elem<T>::N;
  __shared__ RowStats red[4];
  const int64_t r = line_index();
  if (r >= p.rows) return;
  const int y = p.targets[r], tid = threadIdx.x;
  if (p.masked(r, y)) {
    if (tid == 0) {
      logp[r] = 0.f;
      if (lse) lse[r] = 0.f;
      if (ENT) entropy[r] = 0.f;
    }
    return;
  }
  const T* x = static_cast<const T*>(p.x) + r * p.ld;
  const float c = p.scale * kLog2e;
  RowStats a{-INFINITY, 0.f, 0.f};
  for (int i = tid * N; i + N <= p.V; i += 256 * N) {
    float f[N];
    Elem<T>::unpack(*reinterpret_cast<const raw16*>(x + i), f);
    add<ENT>(a, f, c);
  }
  const int i = p.V / N * N + tid;
  if (i < p.V) {
    const float f[1] = {Elem<T>::one(x[i])};
    add<ENT>(a, f, c);
  }
  a = join_wave<ENT>(a, c);
  if ((tid & 63) == 0) red[tid >> 6] = a;
  __syncthreads();
  if (tid) return;
  for (int w = 1; w < 4; ++w) join<ENT>(a, red[w], c);
  finish_row<T, ENT>(p, r, y, a, logp, entropy, lse);
}

// One workgroup per row.  May run in place: every element is read and written
// by one thread.
template <typename T>
__global__ __launch_bounds__(256) void k_logits_logp_bwd(LogitRows p, const float* __restrict__ lse,
                                                         const float* __restrict__ entropy,
                                                         const float* __restrict__ dlogp,
                                                         const float* __restrict__ dentropy,
                                                         T* dlogits, int64_t ld_out) {
  constexpr int N = Elem<T>::N;
  const int64_t r = line_index();
  if (r >= p.rows) return;
  const int y = p.targets[r], tid = threadIdx.x;
  const T* x = static_cast<const T*>(p.x) + r * p.ld;
  T* o = dlogits + r * ld_out;
  float a = 0.f, b = 0.f, l = 0.f, h = 0.f;
  const bool masked = p.masked(r, y);
  if (!masked) {
    a = dlogp[r];
    b = dentropy ? dentropy[r] : 0.f;
    l = lse[r];
    if (y >= p.V) l = NAN;
    h = dentropy ? entropy[r] : 0.f;
  }
  const bool none = masked || (a == 0.f && b == 0.f);
  a *= p.scale;
  b *= p.scale;
  auto grad = [&](float v, int i) -> float {
    const float t = fmaf(v, p.scale, -l), q = __builtin_amdgcn_exp2f(t * kLog2e);
    float g = -q * a;
    if (dentropy) g = fmaf(-q * b, fmaxf(t, kNoExponent) + h, g);
    return i == y ? g + a : g;
  };
  for (int i = tid * N; i + N <= p.V; i += 256 * N) {
    float f[N];
    if (none) {
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] = 0.f;
    } else {
      Elem<T>::unpack(*reinterpret_cast<const raw16*>(x + i), f);
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] = grad(f[e], i + e);
    }
    *reinterpret_cast<raw16*>(o + i) = Elem<T>::pack(f);
  }
  const int i = p.V / N * N + tid;
  if (i < p.V) o[i] = Elem<T>::round(none ? 0.f : grad(Elem<T>::one(x[i]), i));
}

static int check_logits(const bgpo_logits* p) {
  if (!p || p->rows < 0 || p->V < 1 || p->reserved || !(p->scale > 0.f) || !isfinite(p->scale) ||
      (p->in_dtype != BGPO_BF16 && p->in_dtype != BGPO_F32))
    return BGPO_ERR_INVALID_ARG;
  if (p->rows >= int64_t(1) << 31 || p->V > 1 << 24) return BGPO_ERR_UNSUPPORTED;
  if (bad_stride(p, p->ld, p->rows, p->V)) return BGPO_ERR_INVALID_ARG;
  return BGPO_OK;
}

static LogitRows logit_rows(const bgpo_logits* p, const void* x, const int32_t* targets,
                            const uint8_t* mask) {
  return LogitRows{x, targets, mask, p->rows, p->rows > 1 ? p->ld : 0, p->V, p->scale};
}

}  // namespace bgpo

using namespace bgpo;

extern "C" {

int bgpo_logits_workspace_size(const bgpo_logits* prob, size_t* bytes) {
  const int st = check_logits(prob);
  if (st != BGPO_OK) return st;
  if (!bytes) return BGPO_ERR_INVALID_ARG;
  *bytes = 0;
  return BGPO_OK;
}

int bgpo_logits_logp(const bgpo_logits* prob, const void* logits, const int32_t* targets,
                     const uint8_t* row_mask, float* logp, float* entropy, float* lse,
                     void* workspace, size_t ws_bytes, void* stream) {
  const int st = check_logits(prob);
  if (st != BGPO_OK) return st;
  if (prob->rows == 0) return BGPO_OK;
  if (!logits || !targets || !logp) return BGPO_ERR_INVALID_ARG;
  const bool f32 = prob->in_dtype == BGPO_F32;
  const int64_t n = prob->rows, e = f32 ? 4 : 2;
  const Array in[] = {{logits, n, prob->ld, prob->V, e}, vec(targets, n, 4), vec(row_mask, n, 1)};
  const Array out[] = {vec(logp, n, 4), vec(entropy, n, 4), vec(lse, n, 4)};
  if (misaligned(logits, e) || misaligned(targets, 4) || misaligned(logp, 4) || misaligned(entropy, 4) ||
      misaligned(lse, 4) || any_overlap(out, in))
    return BGPO_ERR_INVALID_ARG;
  const LogitRows p = logit_rows(prob, logits, targets, row_mask);
  const auto kernel = f32 ? (entropy ? k_logits_logp<float, true> : k_logits_logp<float, false>)
                          : (entropy ? k_logits_logp<uint16_t, true> : k_logits_logp<uint16_t, false>);
  kernel<<<line_grid(n), 256, 0, (hipStream_t)stream>>>(p, logp, entropy, lse);
  return hipGetLastError() == hipSuccess ? BGPO_OK : BGPO_ERR_HIP;
}

int bgpo_logits_logp_bwd(const bgpo_logits* prob, const void* logits, const int32_t* targets,
                         const uint8_t* row_mask, const float* lse, const float* entropy,
                         const float* dlogp, const float* dentropy, void* dlogits, int64_t ld_out,
                         void* stream) {
  const int st = check_logits(prob);
  if (st != BGPO_OK) return st;
  if (prob->rows == 0) return BGPO_OK;
  if (!logits || !targets || !lse || !dlogp || !dlogits || (dentropy && !entropy))
    return BGPO_ERR_INVALID_ARG;
  const bool f32 = prob->in_dtype == BGPO_F32;
  const int64_t n = prob->rows, e = f32 ? 4 : 2;
  if (bad_stride(dlogits, ld_out, n, prob->V)) return BGPO_ERR_INVALID_ARG;
  const bool in_place = dlogits == logits && (n == 1 || ld_out == prob->ld);
  const Array in[] = {{in_place ? nullptr : logits, n, prob->ld, prob->V, e}, vec(targets, n, 4),
                      vec(row_mask, n, 1), vec(lse, n, 4), vec(dentropy ? entropy : nullptr, n, 4),
                      vec(dlogp, n, 4), vec(dentropy, n, 4)};
  const Array out[] = {{dlogits, n, ld_out, prob->V, e}};
  if (misaligned(logits, e) || misaligned(dlogits, e) || misaligned(targets, 4) || misaligned(lse, 4) ||
      misaligned(entropy, 4) || misaligned(dlogp, 4) || misaligned(dentropy, 4) ||
      any_overlap(out, in))
    return BGPO_ERR_INVALID_ARG;
  const LogitRows p = logit_rows(prob, logits, targets, row_mask);
  const int64_t ldo = n > 1 ? ld_out : 0;
  hipStream_t s = (hipStream_t)stream;
  if (f32)
    k_logits_logp_bwd<float><<<line_grid(n), 256, 0, s>>>(p, lse, entropy, dlogp, dentropy,
                                                          static_cast<float*>(dlogits), ldo);
  else
    k_logits_logp_bwd<uint16_t><<<line_grid(n), 256, 0, s>>>(p, lse, entropy, dlogp, dentropy,
                                                             static_cast<uint16_t*>(dlogits), ldo);
  return hipGetLastError() == hipSuccess ? BGPO_OK : BGPO_ERR_HIP;
}

}  // extern "C"
