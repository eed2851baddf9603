// Policy and preference losses on log-probabilities, with their gradients.
//
// All of the arithmetic is in float64 (differences of log-probabilities, their
// exponentials, the comparison with the clip's borders, every sum): the kernels
// read 13 bytes per fp32 position and write 4, and the float64 work of a
// position takes less time than that.  Sums run in a fixed order.
#include <math.h>

#include <algorithm>

#include "../../include/bgpo.h"
#include "../../include/bgpo_policy.h"
#include "common.hpp"
#include "internal.hpp"
#include "spans.hpp"

namespace bgpo {

constexpr int kThreads = 256;
constexpr int kMaxWgs = 2048;       // workgroups of a pass, and rows of its partial sums

// Sum over the workgroup in a fixed order, returned to every thread; `red`
// holds NV values per wave and is free again after the call's last barrier.
template <int NV>
__device__ __forceinline__ void wg_sum(double (&v)[NV], double (*red)[NV]) {
  const int wave = threadIdx.x >> 6, n_waves = blockDim.x >> 6;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v[i] += __shfl_xor(v[i], off, 64);
    if ((threadIdx.x & 63) == 0) red[wave][i] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    v[i] = 0.0;
    for (int w = 0; w < n_waves; ++w) v[i] += red[w][i];
  }
  __syncthreads();
}

// ---------------------------------------------------------------- policy loss

struct PolicyArgs {
  const void *logp, *old, *ref;
  const float* adv;
  const uint8_t* mask;
  void* dlogp;
  double* stats;
  int32_t* flags;
  int64_t ld_logp, ld_old, ld_ref, ld_mask, ld_dlogp, ld_adv;
  int B, L, ratio, reduce, kl;
  double lo, hi, dual, kl_coef, loss_scale;
  double2* rows;      // [B] unmasked positions and sum of d of each response
  double* counts;     // [kMaxWgs] positions per workgroup of the first pass
  double* part;       // [kMaxWgs][kPolicySums]
  int count_wgs;      // workgroups of the first pass (0: it did not run)
};

// objective, KL, log ratio, positions, cut positions
constexpr int kPolicySums = 5;

// min(r A, clamp(r) A) with the second clip, and whether the gradient of r is
// cut off (the clamped term is strictly the one taken)
struct Clipped {
  double f;
  bool cut;
};
__device__ __forceinline__ Clipped clipped(double r, double A, const PolicyArgs& p) {
  const double free = r * A, held = fmin(fmax(r, p.lo), p.hi) * A;
  Clipped c{free, held < free};
  if (c.cut) c.f = held;
  if (p.dual > 0.0 && A < 0.0 && p.dual * A > c.f) c = Clipped{p.dual * A, true};
  return c;
}

// the KL estimator and its derivative w.r.t. logp at q = ref - logp
__device__ __forceinline__ void kl_term(int kind, double q, double* kl, double* dkl) {
  if (kind == BGPO_KL_K1) {
    *kl = -q;
    *dkl = 1.0;
  } else if (kind == BGPO_KL_K2) {
    *kl = 0.5 * q * q;
    *dkl = -q;
  } else {
    const double e = expm1(q);
    *kl = e - q;
    *dkl = -e;
  }
}

// First pass: unmasked positions and sum of d of each response, one workgroup
// per response.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_policy_rows(PolicyArgs p) {
  __shared__ double red[kThreads / 64][2];
  double count = 0.0;
  for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
    double v[2] = {0.0, 0.0};
    for (int i = threadIdx.x; i < p.L; i += kThreads)
      if (p.mask[b * p.ld_mask + i]) {
        v[0] += 1.0;
        if (p.ratio == BGPO_RATIO_SEQUENCE && p.old)
          v[1] += (double)static_cast<const T*>(p.logp)[b * p.ld_logp + i] -
                  (double)static_cast<const T*>(p.old)[b * p.ld_old + i];
      }
    wg_sum<2>(v, red);
    if (threadIdx.x == 0) p.rows[b] = make_double2(v[0], v[1]);
    count += v[0];
  }
  if (threadIdx.x == 0) p.counts[blockIdx.x] = count;
}

// Second pass: loss and gradient, one workgroup per response.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_policy_loss(PolicyArgs p) {
  __shared__ double red[kThreads / 64][kPolicySums];
  double sums[kPolicySums] = {0.0, 0.0, 0.0, 0.0, 0.0};
  double w = p.loss_scale;
  if (p.reduce == BGPO_REDUCE_TOKENS) {
    double n[1] = {0.0};
    for (int i = threadIdx.x; i < p.count_wgs; i += kThreads) n[0] += p.counts[i];
    wg_sum<1>(n, reinterpret_cast<double(*)[1]>(red));
    w = n[0] > 0.0 ? p.loss_scale / n[0] : 0.0;
  }
  bool bad = false;
  for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
    const double n = p.count_wgs ? p.rows[b].x : 1.0;
    if (p.reduce == BGPO_REDUCE_RESPONSES) w = n > 0.0 ? p.loss_scale / n : 0.0;
    // one ratio for the response: its objective at every position, and the
    // gradient of its n weights by d of one position
    Clipped row{0.0, false};
    double drow = 0.0;
    if (p.ratio == BGPO_RATIO_SEQUENCE && n > 0.0) {
      const double A = p.adv[b], r = exp(p.rows[b].y / n);
      row = clipped(r, A, p);
      drow = row.cut ? 0.0 : -w * r * A;      // n w / n
    }
    for (int i = threadIdx.x; i < p.L; i += kThreads) {
      double g = 0.0;
      if (p.mask[b * p.ld_mask + i]) {
        const double lp = static_cast<const T*>(p.logp)[b * p.ld_logp + i];
        const double d = p.old ? lp - (double)static_cast<const T*>(p.old)[b * p.ld_old + i] : 0.0;
        Clipped c = row;
        g = drow;
        if (p.ratio == BGPO_RATIO_TOKEN) {
          const double A = p.ld_adv ? p.adv[b * p.ld_adv + i] : p.adv[b], r = exp(d);
          c = clipped(r, A, p);
          g = c.cut ? 0.0 : -w * r * A;
        }
        if (p.ref) {
          double kl, dkl;
          kl_term(p.kl, (double)static_cast<const T*>(p.ref)[b * p.ld_ref + i] - lp, &kl, &dkl);
          sums[1] += w * kl;
          if (p.kl_coef != 0.0) g += p.kl_coef * w * dkl;
        }
        sums[0] -= w * c.f;
        sums[2] += w * d;
        sums[3] += 1.0;
        sums[4] += c.cut ? 1.0 : 0.0;
      }
      if (p.dlogp) {
        const T o = (T)g;
        bad = bad || !isfinite(o);
        static_cast<T*>(p.dlogp)[b * p.ld_dlogp + i] = o;
      }
    }
  }
  if (bad && p.flags) atomicOr(p.flags, kFlagNonfinite);
  wg_sum<kPolicySums>(sums, red);
  if (threadIdx.x < kPolicySums) p.part[blockIdx.x * kPolicySums + threadIdx.x] = sums[threadIdx.x];
}

__device__ void write_policy_stats(const PolicyArgs& p, const double (&s)[kPolicySums]) {
  const double loss = p.kl_coef != 0.0 ? s[0] + p.kl_coef * s[1] : s[0];
  p.stats[BGPO_POLICY_LOSS] = loss;
  p.stats[BGPO_POLICY_OBJECTIVE] = s[0];
  p.stats[BGPO_POLICY_KL] = s[1];
  p.stats[BGPO_POLICY_LOG_RATIO] = s[2];
  p.stats[BGPO_POLICY_TOKENS] = s[3];
  p.stats[BGPO_POLICY_CUT] = s[4];
  if (!isfinite(loss) && p.flags) atomicOr(p.flags, kFlagNonfinite);
}

__global__ __launch_bounds__(kThreads) void k_policy_stats(PolicyArgs p, int wgs) {
  __shared__ double red[kThreads / 64][kPolicySums];
  double s[kPolicySums] = {0.0, 0.0, 0.0, 0.0, 0.0};
  for (int i = threadIdx.x; i < wgs; i += kThreads)
#pragma unroll
    for (int c = 0; c < kPolicySums; ++c) s[c] += p.part[i * kPolicySums + c];
  wg_sum<kPolicySums>(s, red);
  if (threadIdx.x == 0) write_policy_stats(p, s);
}

static int check_policy(const bgpo_policy* p) {
  if (!p || p->B < 1 || p->L < 1 || (p->dtype != BGPO_F32 && p->dtype != BGPO_F64) ||
      p->ratio < BGPO_RATIO_TOKEN || p->ratio > BGPO_RATIO_SEQUENCE || p->reduce < BGPO_REDUCE_TOKENS ||
      p->reduce > BGPO_REDUCE_SUM || p->kl < BGPO_KL_K1 || p->kl > BGPO_KL_K3 ||
      !(p->clip_low >= 0.0 && p->clip_low <= 1.0) || !(p->clip_high >= 0.0) ||
      !(p->clip_dual == 0.0 || (p->clip_dual > 1.0 && isfinite(p->clip_dual))) ||
      !isfinite(p->kl_coef) || !isfinite(p->loss_scale) || p->ld_adv < 0 ||
      (p->ld_adv && p->ratio != BGPO_RATIO_TOKEN))
    return BGPO_ERR_INVALID_ARG;
  if ((int64_t)p->B * p->L > int64_t(1) << 40) return BGPO_ERR_UNSUPPORTED;
  return BGPO_OK;
}

static size_t policy_bytes(const bgpo_policy* p) {
  return (size_t)p->B * sizeof(double2) + kMaxWgs * (kPolicySums + 1) * sizeof(double);
}

template <typename T>
static int run_policy(PolicyArgs p, hipStream_t s) {
  const unsigned wgs = (unsigned)std::min<int64_t>(p.B, kMaxWgs);
  if (p.reduce != BGPO_REDUCE_SUM || p.ratio == BGPO_RATIO_SEQUENCE) {
    p.count_wgs = (int)wgs;
    k_policy_rows<T><<<wgs, kThreads, 0, s>>>(p);
    if (hipGetLastError() != hipSuccess) return BGPO_ERR_HIP;
  }
  k_policy_loss<T><<<wgs, kThreads, 0, s>>>(p);
  if (hipGetLastError() != hipSuccess) return BGPO_ERR_HIP;
  k_policy_stats<<<1, kThreads, 0, s>>>(p, (int)wgs);
  return hipGetLastError() == hipSuccess ? BGPO_OK : BGPO_ERR_HIP;
}

// ---------------------------------------------------------------- preference loss

// one side of the pairs
struct PrefSide {
  const void *theta, *ref;
  const uint8_t* mask;
  void* grad;
  float* adv;
  int64_t ld, ld_ref, ld_mask, ld_grad;
};

struct PrefArgs {
  PrefSide side[2];   // the preferred responses, the others
  double* margins;
  double* stats;
  int32_t* flags;
  int64_t adv_stride;
  int P, L, kind, mean;
  double beta, margin, smoothing, loss_scale;
  double2* part;      // [kMaxWgs] loss and count of m > 0
  double* msum;       // [kMaxWgs] sum of m
};

// log(1 + e^v) without overflow
__device__ __forceinline__ double softplus(double v) { return fmax(v, 0.0) + log1p(exp(-fabs(v))); }

// loss of a margin and its derivative
__device__ __forceinline__ void pref_term(const PrefArgs& p, double m, double* loss, double* dm) {
  if (p.kind == BGPO_PREF_SIGMOID) {
    const double e = p.smoothing;
    *loss = (1.0 - e) * softplus(-m) + (e != 0.0 ? e * softplus(m) : 0.0);
    *dm = -(1.0 - e) / (1.0 + exp(m)) + (e != 0.0 ? e / (1.0 + exp(-m)) : 0.0);
  } else if (p.kind == BGPO_PREF_HINGE) {
    *loss = m < 1.0 ? 1.0 - m : m >= 1.0 ? 0.0 : m;   // (NaN stays)
    *dm = m < 1.0 ? -1.0 : m >= 1.0 ? 0.0 : m;
  } else {
    const double v = (m - 0.5) / p.beta;
    *loss = v * v;
    *dm = 2.0 * v / p.beta;
  }
}

// One workgroup per pair: the scores of both responses, the margin's loss, and
// the gradient, which is one number per response.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_preference(PrefArgs p) {
  __shared__ double red[kThreads / 64][4];
  double loss_sum = 0.0, right = 0.0, m_sum = 0.0;
  bool bad = false;
  for (int q = blockIdx.x; q < p.P; q += gridDim.x) {
    double v[4] = {0.0, 0.0, 0.0, 0.0};     // score and positions of either side
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const PrefSide& s = p.side[k];
      for (int i = threadIdx.x; i < p.L; i += kThreads)
        if (!s.mask || s.mask[q * s.ld_mask + i]) {
          double x = static_cast<const T*>(s.theta)[q * s.ld + i];
          if (s.ref) x -= (double)static_cast<const T*>(s.ref)[q * s.ld_ref + i];
          v[2 * k] += x;
          v[2 * k + 1] += 1.0;
        }
    }
    wg_sum<4>(v, red);
    const double nw = p.mean ? fmax(v[1], 1.0) : 1.0, nl = p.mean ? fmax(v[3], 1.0) : 1.0;
    const double m = p.beta * (v[0] / nw - v[2] / nl) - p.margin;
    double loss, dm;
    pref_term(p, m, &loss, &dm);
    const double g = p.loss_scale * p.beta * dm;     // d loss / d s(win) = -d loss / d s(lose)
    loss_sum += p.loss_scale * loss;
    right += m > 0.0 ? 1.0 : 0.0;
    m_sum += m;
    bad = bad || !isfinite(g);
    if (threadIdx.x == 0) {
      if (p.margins) p.margins[q] = m;
      if (p.side[0].adv) {
        p.side[0].adv[q * p.adv_stride] = (float)-g;
        p.side[1].adv[q * p.adv_stride] = (float)g;
      }
    }
    if (p.side[0].grad) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const PrefSide& s = p.side[k];
        const T o = (T)(k ? -g / nl : g / nw);
        for (int i = threadIdx.x; i < p.L; i += kThreads)
          static_cast<T*>(s.grad)[q * s.ld_grad + i] = !s.mask || s.mask[q * s.ld_mask + i] ? o : (T)0;
      }
    }
  }
  if (bad && p.flags && threadIdx.x == 0) atomicOr(p.flags, kFlagNonfinite);
  if (threadIdx.x == 0) {
    p.part[blockIdx.x] = make_double2(loss_sum, right);
    p.msum[blockIdx.x] = m_sum;
  }
}

__global__ __launch_bounds__(kThreads) void k_preference_stats(PrefArgs p, int wgs) {
  __shared__ double red[kThreads / 64][3];
  double s[3] = {0.0, 0.0, 0.0};
  for (int i = threadIdx.x; i < wgs; i += kThreads) {
    s[0] += p.part[i].x;
    s[1] += p.part[i].y;
    s[2] += p.msum[i];
  }
  wg_sum<3>(s, red);
  if (threadIdx.x < 3) p.stats[threadIdx.x] = s[threadIdx.x];
  if (threadIdx.x == 0 && !isfinite(s[0]) && p.flags) atomicOr(p.flags, kFlagNonfinite);
}

static int check_preference(const bgpo_preference* p) {
  if (!p || p->P < 1 || p->L < 1 || (p->dtype != BGPO_F32 && p->dtype != BGPO_F64) ||
      p->kind < BGPO_PREF_SIGMOID || p->kind > BGPO_PREF_SQUARED || (p->mean != 0 && p->mean != 1) ||
      p->reserved || !(p->beta > 0.0) || !isfinite(p->beta) || !isfinite(p->margin) ||
      !isfinite(p->loss_scale) || !(p->label_smoothing >= 0.0 && p->label_smoothing < 1.0) ||
      (p->label_smoothing != 0.0 && p->kind != BGPO_PREF_SIGMOID))
    return BGPO_ERR_INVALID_ARG;
  if ((int64_t)p->P * p->L > int64_t(1) << 39) return BGPO_ERR_UNSUPPORTED;
  return BGPO_OK;
}

static size_t preference_bytes() { return kMaxWgs * 3 * sizeof(double); }

template <typename T>
static int run_preference(const PrefArgs& p, hipStream_t s) {
  const unsigned wgs = (unsigned)std::min<int64_t>(p.P, kMaxWgs);
  k_preference<T><<<wgs, kThreads, 0, s>>>(p);
  if (hipGetLastError() != hipSuccess) return BGPO_ERR_HIP;
  k_preference_stats<<<1, kThreads, 0, s>>>(p, (int)wgs);
  return hipGetLastError() == hipSuccess ? BGPO_OK : BGPO_ERR_HIP;
}

}  // namespace bgpo

using namespace bgpo;

extern "C" {

int bgpo_policy_workspace_size(const bgpo_policy* prob, size_t* bytes) {
  const int st = check_policy(prob);
  if (st != BGPO_OK) return st;
  if (!bytes) return BGPO_ERR_INVALID_ARG;
  *bytes = policy_bytes(prob);
  return BGPO_OK;
}

int bgpo_policy_loss(const bgpo_policy* prob, const void* logp, const void* logp_old,
                     const void* logp_ref, const float* adv, const uint8_t* resp_mask, void* dlogp,
                     double* stats, int32_t* status_flags, void* workspace, size_t ws_bytes,
                     void* stream) {
  const int st = check_policy(prob);
  if (st != BGPO_OK) return st;
  if (!logp || !adv || !resp_mask || !stats || (!logp_ref && prob->kl_coef != 0.0))
    return BGPO_ERR_INVALID_ARG;
  const int64_t B = prob->B, L = prob->L, e = prob->dtype == BGPO_F64 ? 8 : 4;
  if (bad_stride(logp, prob->ld_logp, B, L) || bad_stride(logp_old, prob->ld_old, B, L) ||
      bad_stride(logp_ref, prob->ld_ref, B, L) || bad_stride(resp_mask, prob->ld_mask, B, L) ||
      bad_stride(dlogp, prob->ld_dlogp, B, L) || (prob->ld_adv && bad_stride(adv, prob->ld_adv, B, L)))
    return BGPO_ERR_INVALID_ARG;
  if (misaligned(logp, e) || misaligned(logp_old, e) || misaligned(logp_ref, e) || misaligned(adv, 4) ||
      misaligned(dlogp, e) || misaligned(stats, 8) || misaligned(status_flags, 4))
    return BGPO_ERR_INVALID_ARG;
  const Array in[] = {{logp, B, prob->ld_logp, L, e}, {logp_old, B, prob->ld_old, L, e},
                      {logp_ref, B, prob->ld_ref, L, e}, {resp_mask, B, prob->ld_mask, L, 1},
                      prob->ld_adv ? Array{adv, B, prob->ld_adv, L, 4} : vec(adv, B, 4)};
  const Array out[] = {{dlogp, B, prob->ld_dlogp, L, e}, vec(stats, BGPO_POLICY_STATS, 8), vec(status_flags, 1, 4)};
  if (any_overlap(out, in)) return BGPO_ERR_INVALID_ARG;
  if (!workspace || ws_bytes < policy_bytes(prob) || misaligned(workspace, 256)) return BGPO_ERR_WORKSPACE;
  PolicyArgs p{logp, logp_old, logp_ref, adv, resp_mask, dlogp, stats, status_flags,
               prob->ld_logp, prob->ld_old, prob->ld_ref, prob->ld_mask, prob->ld_dlogp, prob->ld_adv,
               prob->B, prob->L, prob->ratio, prob->reduce, prob->kl,
               1.0 - prob->clip_low, 1.0 + prob->clip_high, prob->clip_dual, prob->kl_coef, prob->loss_scale};
  p.rows = static_cast<double2*>(workspace);
  p.counts = reinterpret_cast<double*>(p.rows + B);
  p.part = p.counts + kMaxWgs;
  p.count_wgs = 0;
  hipStream_t s = (hipStream_t)stream;
  return e == 8 ? run_policy<double>(p, s) : run_policy<float>(p, s);
}

int bgpo_preference_workspace_size(const bgpo_preference* prob, size_t* bytes) {
  const int st = check_preference(prob);
  if (st != BGPO_OK) return st;
  if (!bytes) return BGPO_ERR_INVALID_ARG;
  *bytes = preference_bytes();
  return BGPO_OK;
}

int bgpo_preference_loss(const bgpo_preference* prob, const void* win, const void* lose,
                         const void* win_ref, const void* lose_ref, const uint8_t* win_mask,
                         const uint8_t* lose_mask, void* dwin, void* dlose, double* margins,
                         float* adv_win, float* adv_lose, double* stats, int32_t* status_flags,
                         void* workspace, size_t ws_bytes, void* stream) {
  const int st = check_preference(prob);
  if (st != BGPO_OK) return st;
  if (!win || !lose || !stats || !win_ref != !lose_ref || !win_mask != !lose_mask || !dwin != !dlose ||
      !adv_win != !adv_lose || (adv_win && prob->P > 1 && (prob->adv_stride < 1 || prob->adv_stride > int64_t(1) << 24)))
    return BGPO_ERR_INVALID_ARG;
  const int64_t P = prob->P, L = prob->L, e = prob->dtype == BGPO_F64 ? 8 : 4;
  if (bad_stride(win, prob->ld_win, P, L) || bad_stride(lose, prob->ld_lose, P, L) ||
      bad_stride(win_ref, prob->ld_win_ref, P, L) || bad_stride(lose_ref, prob->ld_lose_ref, P, L) ||
      bad_stride(win_mask, prob->ld_win_mask, P, L) || bad_stride(lose_mask, prob->ld_lose_mask, P, L) ||
      bad_stride(dwin, prob->ld_dwin, P, L) || bad_stride(dlose, prob->ld_dlose, P, L))
    return BGPO_ERR_INVALID_ARG;
  if (misaligned(win, e) || misaligned(lose, e) || misaligned(win_ref, e) || misaligned(lose_ref, e) ||
      misaligned(dwin, e) || misaligned(dlose, e) || misaligned(margins, 8) || misaligned(adv_win, 4) ||
      misaligned(adv_lose, 4) || misaligned(stats, 8) || misaligned(status_flags, 4))
    return BGPO_ERR_INVALID_ARG;
  const int64_t as = P > 1 ? prob->adv_stride : 1;
  const Array in[] = {{win, P, prob->ld_win, L, e}, {lose, P, prob->ld_lose, L, e},
                      {win_ref, P, prob->ld_win_ref, L, e}, {lose_ref, P, prob->ld_lose_ref, L, e},
                      {win_mask, P, prob->ld_win_mask, L, 1}, {lose_mask, P, prob->ld_lose_mask, L, 1}};
  const Array out[] = {{dwin, P, prob->ld_dwin, L, e}, {dlose, P, prob->ld_dlose, L, e}, {adv_win, P, as, 1, 4},
                       {adv_lose, P, as, 1, 4}, vec(margins, P, 8), vec(stats, BGPO_PREF_STATS, 8),
                       vec(status_flags, 1, 4)};
  if (any_overlap(out, in)) return BGPO_ERR_INVALID_ARG;
  if (!workspace || ws_bytes < preference_bytes() || misaligned(workspace, 256)) return BGPO_ERR_WORKSPACE;
  PrefArgs p{{{win, win_ref, win_mask, dwin, adv_win, prob->ld_win, prob->ld_win_ref, prob->ld_win_mask, prob->ld_dwin},
              {lose, lose_ref, lose_mask, dlose, adv_lose, prob->ld_lose, prob->ld_lose_ref, prob->ld_lose_mask,
               prob->ld_dlose}},
             margins, stats, status_flags, as, prob->P, prob->L, prob->kind, prob->mean,
             prob->beta, prob->margin, prob->label_smoothing, prob->loss_scale};
  p.part = static_cast<double2*>(workspace);
  p.msum = reinterpret_cast<double*>(p.part + kMaxWgs);
  hipStream_t s = (hipStream_t)stream;
  return e == 8 ? run_preference<double>(p, s) : run_preference<float>(p, s);
}

}  // extern "C"
