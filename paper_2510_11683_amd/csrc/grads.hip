// Norm of a list of gradients, and their scaling to a largest norm.
//
// The list travels in the kernels' arguments, kTable entries to a launch.  Its
// tensors are cut into chunks of kChunk elements, numbered through the launch;
// a workgroup finds its chunk's tensor by bisection.
#include <math.h>

#include <algorithm>
#include <memory>
#include <new>

#include "../../include/bgpo.h"
#include "../../include/bgpo_grads.h"
#include "common.hpp"
#include "internal.hpp"
#include "spans.hpp"

namespace bgpo {

constexpr int kTable = 112;                // entries of a launch (3.7 KB of arguments)
constexpr int64_t kChunk = 16384;
constexpr int kNormWgs = 2048;             // workgroups of a norm pass, one partial each
constexpr int kMaxClipWgs = 1 << 22;

// 16 bytes at the alignment of the element type
typedef uint32_t raw16 __attribute__((ext_vector_type(4), aligned(2), may_alias));
typedef uint32_t raw8 __attribute__((ext_vector_type(2), aligned(2), may_alias));

struct Table {
  const void* src[kTable];
  void* dst[kTable];
  int64_t n[kTable];
  uint32_t first[kTable];                  // number of its first chunk
  uint8_t src_f32[kTable], dst_f32[kTable];
  uint32_t chunks;
  int count;
};

// the entry that holds chunk c
__device__ __forceinline__ int find_entry(const Table& t, uint32_t c) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= c) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Running norm of one thread: the sum of squares in float64, or the largest
// magnitude as bits (of a sign-less float they order like its value, infinity
// and then NaN above all).
template <bool MAX>
struct Norm {
  double sum = 0.0;
  uint32_t top = 0;
  __device__ __forceinline__ void add(float v) {
    if (MAX) top = max(top, __float_as_uint(v) & 0x7FFFFFFFu);
    else sum = fma((double)v, (double)v, sum);
  }
  __device__ __forceinline__ void add16(const raw16& r, bool f32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (f32) {
        add(__uint_as_float(r[i]));
      } else {
        add(__uint_as_float(r[i] << 16));
        add(__uint_as_float(r[i] & 0xFFFF0000u));
      }
    }
  }
  __device__ double value() const { return MAX ? (double)__uint_as_float(top) : sum; }
  // b joins a
  static __device__ double join(double a, double b) {
    if (!MAX) return a + b;
    return a != a || a > b ? a : b;        // (a NaN stays, from either)
  }
};

// Partial norms: workgroup k takes chunks k, k + grid, ..; the launches of a
// longer list go on from the partials before.
template <bool MAX>
__global__ __launch_bounds__(256) void k_grad_norm(Table t, bool first, double* __restrict__ part) {
  __shared__ double red[4];
  Norm<MAX> a;
  for (uint32_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const int e = find_entry(t, c);
    const int64_t at = (int64_t)(c - t.first[e]) * kChunk;
    const int n = (int)min(kChunk, t.n[e] - at);
    if (t.src_f32[e]) {
      const float* x = static_cast<const float*>(t.src[e]) + at;
      for (int i = threadIdx.x * 4; i + 4 <= n; i += 1024) a.add16(*reinterpret_cast<const raw16*>(x + i), true);
      const int i = (n & ~3) + threadIdx.x;
      if (i < n) a.add(x[i]);
    } else {
      const bf16_t* x = static_cast<const bf16_t*>(t.src[e]) + at;
      for (int i = threadIdx.x * 8; i + 8 <= n; i += 2048) a.add16(*reinterpret_cast<const raw16*>(x + i), false);
      const int i = (n & ~7) + threadIdx.x;
      if (i < n) a.add(bf16_to_f32(x[i]));
    }
  }
  double v = a.value();
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = Norm<MAX>::join(v, __shfl_xor(v, off, 64));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x) return;
  v = first ? 0.0 : part[blockIdx.x];
  for (int w = 0; w < 4; ++w) v = Norm<MAX>::join(v, red[w]);
  part[blockIdx.x] = v;
}

template <bool MAX>
__global__ __launch_bounds__(256) void k_grad_norm_final(const double* __restrict__ part, int wgs,
                                                         double* __restrict__ norm, int32_t* flags) {
  __shared__ double red[4];
  double v = 0.0;
  for (int i = threadIdx.x; i < wgs; i += 256) v = Norm<MAX>::join(v, part[i]);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = Norm<MAX>::join(v, __shfl_xor(v, off, 64));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x) return;
  v = red[0];
  for (int w = 1; w < 4; ++w) v = Norm<MAX>::join(v, red[w]);
  if (!MAX) v = sqrt(v);
  norm[0] = v;
  if (flags && !isfinite(v)) atomicOr(flags, kFlagNonfinite);
}

// One chunk after the other: dst = src * f, f = max_norm / norm where the norm
// is larger (and finite), else 1.  An entry that is its own output is left
// alone where f is 1.
__global__ __launch_bounds__(256) void k_grad_clip(Table t, double max_norm, const double* __restrict__ norm) {
  const double v = norm[0];
  const float f = isfinite(v) && v > max_norm ? (float)(max_norm / v) : 1.f;
  for (uint32_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const int e = find_entry(t, c);
    if (f == 1.f && t.src[e] == t.dst[e]) continue;
    const int64_t at = (int64_t)(c - t.first[e]) * kChunk;
    const int n = (int)min(kChunk, t.n[e] - at);
    const bool sf = t.src_f32[e], df = t.dst_f32[e];
    const float* xf = static_cast<const float*>(t.src[e]) + at;
    const bf16_t* xb = static_cast<const bf16_t*>(t.src[e]) + at;
    float* of = static_cast<float*>(t.dst[e]) + at;
    bf16_t* ob = static_cast<bf16_t*>(t.dst[e]) + at;
    for (int i = threadIdx.x * 4; i + 4 <= n; i += 1024) {
      float x[4];
      if (sf) {
        const raw16 r = *reinterpret_cast<const raw16*>(xf + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(r[k]) * f;
      } else {
        const raw8 r = *reinterpret_cast<const raw8*>(xb + i);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          x[2 * k] = __uint_as_float(r[k] << 16) * f;
          x[2 * k + 1] = __uint_as_float(r[k] & 0xFFFF0000u) * f;
        }
      }
      if (df) {
        raw16 r;
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = __float_as_uint(x[k]);
        *reinterpret_cast<raw16*>(of + i) = r;
      } else {
        raw8 r;
        r[0] = pack_bf16x2(x[0], x[1]);
        r[1] = pack_bf16x2(x[2], x[3]);
        *reinterpret_cast<raw8*>(ob + i) = r;
      }
    }
    const int i = (n & ~3) + threadIdx.x;
    if (i < n) {
      const float x = (sf ? xf[i] : bf16_to_f32(xb[i])) * f;
      if (df) of[i] = x;
      else ob[i] = f32_to_bf16(x);
    }
  }
}

static int64_t elem_bytes(const bgpo_tensor& t) { return t.dtype == BGPO_F32 ? 4 : 2; }

static int check_list(const bgpo_tensor* t, int32_t count) {
  if (count < 0 || (count && !t)) return BGPO_ERR_INVALID_ARG;
  for (int i = 0; i < count; ++i) {
    if (t[i].n < 0 || (t[i].n && !t[i].data) || (t[i].dtype != BGPO_BF16 && t[i].dtype != BGPO_F32) ||
        t[i].reserved || misaligned(t[i].data, elem_bytes(t[i])))
      return BGPO_ERR_INVALID_ARG;
    if (t[i].n > int64_t(1) << 38) return BGPO_ERR_UNSUPPORTED;
  }
  return BGPO_OK;
}

// Whether an output shares bytes with another entry of either list (an entry
// that is its own output counts once).
static int check_outputs(const bgpo_tensor* g, const bgpo_tensor* out, int32_t count) {
  struct Interval {
    uintptr_t lo, hi;
    bool out;
  };
  std::unique_ptr<Interval[]> v(new (std::nothrow) Interval[2 * (size_t)count + 1]);
  if (!v) return BGPO_ERR_HIP;
  int n = 0;
  auto add = [&](const bgpo_tensor& t, bool o) {
    if (t.n) v[n++] = Interval{(uintptr_t)t.data, (uintptr_t)t.data + (uintptr_t)(t.n * elem_bytes(t)), o};
  };
  for (int i = 0; i < count; ++i) {
    add(out[i], true);
    if (out[i].data != g[i].data || out[i].dtype != g[i].dtype) add(g[i], false);
  }
  const auto before = [](const Interval& a, const Interval& b) { return a.lo < b.lo; };
  if (!std::is_sorted(v.get(), v.get() + n, before)) std::sort(v.get(), v.get() + n, before);
  uintptr_t end = 0, out_end = 0;          // of all the intervals so far, and of the outputs
  for (int i = 0; i < n; ++i) {
    if (v[i].lo < out_end || (v[i].out && v[i].lo < end)) return BGPO_ERR_INVALID_ARG;
    end = std::max(end, v[i].hi);
    if (v[i].out) out_end = std::max(out_end, v[i].hi);
  }
  return BGPO_OK;
}

// Fills the table from entry `at` on; the entry it stops at.
static int fill_table(const bgpo_tensor* g, const bgpo_tensor* out, int32_t count, int at, Table* t) {
  t->count = 0;
  t->chunks = 0;
  for (; at < count && t->count < kTable; ++at) {
    if (!g[at].n) continue;
    const int k = t->count++;
    t->src[k] = g[at].data;
    t->dst[k] = out ? out[at].data : nullptr;
    t->n[k] = g[at].n;
    t->src_f32[k] = g[at].dtype == BGPO_F32;
    t->dst_f32[k] = out && out[at].dtype == BGPO_F32;
    t->first[k] = t->chunks;
    t->chunks += (uint32_t)((g[at].n + kChunk - 1) / kChunk);
  }
  return at;
}

template <bool MAX>
static int run_norm(const bgpo_tensor* g, int32_t count, double* norm, int32_t* flags, double* part,
                    hipStream_t s) {
  // the workgroups that the largest launch needs take part in every one
  Table t;
  uint32_t most = 0;
  for (int at = 0; at < count;) {
    at = fill_table(g, nullptr, count, at, &t);
    most = std::max(most, t.chunks);
  }
  const int wgs = (int)std::min<uint32_t>(most, kNormWgs);
  bool first = true;
  for (int at = 0; wgs && at < count;) {
    at = fill_table(g, nullptr, count, at, &t);
    if (!t.count) break;
    k_grad_norm<MAX><<<(unsigned)wgs, 256, 0, s>>>(t, first, part);
    if (hipGetLastError() != hipSuccess) return BGPO_ERR_HIP;
    first = false;
  }
  k_grad_norm_final<MAX><<<1, 256, 0, s>>>(part, wgs, norm, flags);
  return hipGetLastError() == hipSuccess ? BGPO_OK : BGPO_ERR_HIP;
}

}  // namespace bgpo

using namespace bgpo;

extern "C" {

size_t bgpo_grad_workspace_size(void) { return kNormWgs * sizeof(double); }

int bgpo_grad_norm(const bgpo_tensor* grads, int32_t count, int32_t norm_type, double* norm,
                   int32_t* status_flags, void* workspace, size_t ws_bytes, void* stream) {
  const int st = check_list(grads, count);
  if (st != BGPO_OK) return st;
  if (!norm || (norm_type != BGPO_NORM_L2 && norm_type != BGPO_NORM_MAX) || misaligned(norm, 8) ||
      misaligned(status_flags, 4))
    return BGPO_ERR_INVALID_ARG;
  if (!workspace || misaligned(workspace, 8) || ws_bytes < bgpo_grad_workspace_size())
    return BGPO_ERR_WORKSPACE;
  double* part = static_cast<double*>(workspace);
  hipStream_t s = (hipStream_t)stream;
  return norm_type == BGPO_NORM_MAX ? run_norm<true>(grads, count, norm, status_flags, part, s)
                                    : run_norm<false>(grads, count, norm, status_flags, part, s);
}

int bgpo_grad_clip(const bgpo_tensor* grads, const bgpo_tensor* out, int32_t count, double max_norm,
                   const double* norm, void* stream) {
  int st = check_list(grads, count);
  if (st == BGPO_OK && out) st = check_list(out, count);
  if (st != BGPO_OK) return st;
  if (!norm || misaligned(norm, 8) || !(max_norm >= 0.0) || !isfinite(max_norm)) return BGPO_ERR_INVALID_ARG;
  if (!out) out = grads;
  for (int i = 0; i < count; ++i)
    if (out[i].n != grads[i].n) return BGPO_ERR_INVALID_ARG;
  st = check_outputs(grads, out, count);
  if (st != BGPO_OK) return st;
  Table t;
  for (int at = 0; at < count;) {
    at = fill_table(grads, out, count, at, &t);
    if (!t.count) break;
    k_grad_clip<<<std::min<uint32_t>(t.chunks, kMaxClipWgs), 256, 0, (hipStream_t)stream>>>(t, max_norm, norm);
    if (hipGetLastError() != hipSuccess) return BGPO_ERR_HIP;
  }
  return BGPO_OK;
}

}  // extern "C"
