// Log probabilities of given tokens under rows of logits, the rows' entropies and best alternatives, and the gradient.
// With c the scale, m the row's largest logit, s = sum_j e^(c (z_j - m)) and q_j = c (z_j - m) - ln s (the log probability):
//   logprob = q_token,  entropy = ln s - c sum_j (z_j - m) e^(c (z_j - m)) / s,
//   dz_j = c (dlogprob (delta_j - p_j) - dentropy p_j (q_j + entropy)),  p_j = e^q_j.
// Logits are compared and subtracted before they are scaled: a row that holds its type's lowest value everywhere is then as
// good as any other, where c z would overflow.  All sums are fp32.
#include <hip/hip_runtime.h>

#include <cmath>

#include "device_utils.h"
#include "karma.h"
#include "kernels.h"

namespace karma {
namespace {

constexpr int LP_THREADS = 256;

template <typename T>
__device__ __forceinline__ float load1(const T* p);
template <>
__device__ __forceinline__ float load1<bf16_t>(const bf16_t* p) { return bf2f(*p); }
template <>
__device__ __forceinline__ float load1<float>(const float* p) { return *p; }
__device__ __forceinline__ void store1(bf16_t* p, float v) { *p = f2bf(v); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }

// largest, sum and first moment of a part of a row; empty: {-inf, 0, 0}
struct RowPart { float m, s, t; };
__device__ __forceinline__ RowPart join(const RowPart& a, const RowPart& b, float scale) {
  RowPart r;
  r.m = fmaxf(a.m, b.m);
  if (r.m == -INFINITY) return RowPart{r.m, a.s + b.s, a.t + b.t};   // nothing allowed so far (or NaN alone, which the sums carry)
  // a part whose largest is -inf has sums of zero; its difference must not make -inf * 0
  const float da = fmaxf(a.m - r.m, -1e30f), db = fmaxf(b.m - r.m, -1e30f);
  const float ea = expf(da * scale), eb = expf(db * scale);
  r.s = a.s * ea + b.s * eb;
  r.t = (a.t + (ea ? da * a.s : 0.f)) * ea + (b.t + (eb ? db * b.s : 0.f)) * eb;
  return r;
}

template <typename T>
__global__ __launch_bounds__(LP_THREADS) void logprob_fwd_kernel(LogprobFwd a) {
  __shared__ RowPart part[LP_THREADS];
  __shared__ float best_v[LP_THREADS];
  __shared__ int best_i[LP_THREADS];
  const int tid = threadIdx.x;
  const size_t r = blockIdx.x;
  const T* z = (const T*)a.logits + r * a.ld;
  RowPart p{-INFINITY, 0.f, 0.f};
  for (unsigned j = tid; j < a.cols; j += LP_THREADS) {
    const float v = load1(z + j);
    if (v > p.m) {
      const float d = fmaxf(p.m - v, -1e30f), e = expf(d * a.scale);
      p.t = (p.t + (e ? d * p.s : 0.f)) * e;
      p.s *= e;
      p.m = v;
    }
    const float d = v == -INFINITY ? -INFINITY : v - p.m, e = expf(d * a.scale);
    p.s += e;
    p.t += e == 0.f ? 0.f : d * e;
  }
  part[tid] = p;
  __syncthreads();
  for (int k = LP_THREADS / 2; k > 0; k >>= 1) {
    if (tid < k) part[tid] = join(part[tid], part[tid + k], a.scale);
    __syncthreads();
  }
  p = part[0];
  const float ls = p.m == -INFINITY && p.s == 0.f ? 0.f : logf(p.s);
  auto log_p = [&](float v) { return v == -INFINITY && p.s == p.s ? v : (v - p.m) * a.scale - ls; };
  if (tid == 0) {
    if (a.stats) { a.stats[2 * r] = p.m; a.stats[2 * r + 1] = ls; }
    if (a.entropy) a.entropy[r] = p.m == -INFINITY && p.s == 0.f ? 0.f : ls - a.scale * p.t / p.s;
    if (a.logprob) {
      const int t = a.tokens[r];
      a.logprob[r] = t >= 0 && (unsigned)t < a.cols ? log_p(load1(z + t)) : 0.f;
    }
  }
  // the k best, one after the other: the best among those behind the last one taken
  float lv = INFINITY;
  int li = -1;
  for (unsigned k = 0; k < a.top; ++k) {
    float bv = -INFINITY;
    int bi = INT32_MAX;
    for (unsigned j = tid; j < a.cols; j += LP_THREADS) {
      const float v = load1(z + j);
      if ((v < lv || (v == lv && (int)j > li)) && (v > bv || (v == bv && (int)j < bi))) { bv = v; bi = (int)j; }
    }
    best_v[tid] = bv;
    best_i[tid] = bi;
    __syncthreads();
    for (int n = LP_THREADS / 2; n > 0; n >>= 1) {
      if (tid < n && (best_v[tid + n] > best_v[tid] || (best_v[tid + n] == best_v[tid] && best_i[tid + n] < best_i[tid]))) {
        best_v[tid] = best_v[tid + n];
        best_i[tid] = best_i[tid + n];
      }
      __syncthreads();
    }
    lv = best_v[0];
    li = best_i[0];
    __syncthreads();
    if (tid == 0) {
      const bool any = li != INT32_MAX;
      a.top_id[r * a.top + k] = any ? li : -1;
      a.top_logprob[r * a.top + k] = any ? log_p(lv) : NAN;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(LP_THREADS) void logprob_bwd_kernel(LogprobBwd a) {
  const size_t r = blockIdx.x;
  const T* z = (const T*)a.logits + r * a.ld;
  T* d = (T*)a.dlogits + r * a.ld_d;
  const float m = a.stats[2 * r], ls = a.stats[2 * r + 1];
  const int token = a.tokens ? a.tokens[r] : -1;
  const float dl = a.dlogprob && token >= 0 && (unsigned)token < a.cols ? a.dlogprob[r] : 0.f;
  const float de = a.dentropy ? a.dentropy[r] : 0.f, ent = a.dentropy ? a.entropy[r] : 0.f;
  for (unsigned j = threadIdx.x; j < a.cols; j += LP_THREADS) {
    float v = 0.f;
    if (m != -INFINITY || ls != 0.f) {
      const float q = (load1(z + j) - m) * a.scale - ls, p = expf(q);
      v = -dl * p - (p == 0.f ? 0.f : de * p * (q + ent));
      if ((int)j == token) v += dl;
    }
    store1(d + j, v * a.scale);
  }
}

bool aligned_to(const void* p, size_t n) { return (uintptr_t)p % n == 0; }
bool good_rows(uint32_t rows, uint32_t cols, uint64_t ld) {
  return cols && cols <= INT32_MAX && rows <= INT32_MAX && ld >= cols && ld <= INT64_MAX / 8 / ((uint64_t)rows + 1);
}

}  // namespace

size_t token_logprob_ws_bytes(uint32_t, uint32_t, uint32_t) { return 0; }

int token_logprob_fwd(LogprobFwd a, bool bf16, hipStream_t s) {
  if (!a.ld) a.ld = a.cols;
  if (!good_rows(a.rows, a.cols, a.ld) || !(a.scale > 0.f) || !std::isfinite(a.scale)) return KARMA_E_INVAL;
  if (a.top > KARMA_TOP_MAX || a.top > a.cols || (a.top && (!a.top_logprob || !a.top_id))) return KARMA_E_INVAL;
  if ((a.logprob && !a.tokens) || (!a.logprob && !a.entropy && !a.stats && !a.top)) return KARMA_E_INVAL;
  if (!a.rows) return KARMA_OK;
  if (!a.logits || !aligned_to(a.logits, bf16 ? 2 : 4)) return KARMA_E_INVAL;
  if (a.ws_bytes < token_logprob_ws_bytes(a.rows, a.cols, a.top)) return KARMA_E_OOM;
  if (bf16) hipLaunchKernelGGL(logprob_fwd_kernel<bf16_t>, dim3(a.rows), dim3(LP_THREADS), 0, s, a);
  else hipLaunchKernelGGL(logprob_fwd_kernel<float>, dim3(a.rows), dim3(LP_THREADS), 0, s, a);
  return hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

int token_logprob_bwd(LogprobBwd a, bool bf16, hipStream_t s) {
  if (!a.ld) a.ld = a.cols;
  if (!a.ld_d) a.ld_d = a.cols;
  if (!good_rows(a.rows, a.cols, a.ld) || !good_rows(a.rows, a.cols, a.ld_d) || !(a.scale > 0.f) || !std::isfinite(a.scale)) return KARMA_E_INVAL;
  if ((a.dlogprob && !a.tokens) || (a.dentropy && !a.entropy) || (!a.dlogprob && !a.dentropy)) return KARMA_E_INVAL;
  if (!a.rows) return KARMA_OK;
  if (!a.logits || !a.stats || !a.dlogits || !aligned_to(a.logits, bf16 ? 2 : 4) || !aligned_to(a.dlogits, bf16 ? 2 : 4)) return KARMA_E_INVAL;
  if (bf16) hipLaunchKernelGGL(logprob_bwd_kernel<bf16_t>, dim3(a.rows), dim3(LP_THREADS), 0, s, a);
  else hipLaunchKernelGGL(logprob_bwd_kernel<float>, dim3(a.rows), dim3(LP_THREADS), 0, s, a);
  return hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

}  // namespace karma

using namespace karma;

extern "C" uint64_t karma_k_token_logprob_ws_bytes(uint32_t rows, uint32_t cols, uint32_t top) { return token_logprob_ws_bytes(rows, cols, top); }

#define KARMA_LOGPROB_ENTRIES(SUFFIX, T, BF16)                                                                                               \
  extern "C" int karma_k_token_logprob_fwd_##SUFFIX(const T* logits, uint64_t ld, const int32_t* tokens, float* logprob, float* entropy,     \
                                                    float* stats, float* top_logprob, int32_t* top_id, uint32_t rows, uint32_t cols,         \
                                                    uint32_t top, float scale, void* ws, uint64_t ws_bytes, void* stream) {                  \
    return token_logprob_fwd(LogprobFwd{logits, ld, tokens, logprob, entropy, stats, top_logprob, top_id, rows, cols, top, scale, ws,        \
                                        ws ? ws_bytes : 0}, BF16, (hipStream_t)stream);                                                      \
  }                                                                                                                                          \
  extern "C" int karma_k_token_logprob_bwd_##SUFFIX(const T* logits, uint64_t ld, const int32_t* tokens, const float* stats,                 \
                                                    const float* entropy, const float* dlogprob, const float* dentropy, T* dlogits,          \
                                                    uint64_t ld_d, uint32_t rows, uint32_t cols, float scale, void* stream) {                \
    return token_logprob_bwd(LogprobBwd{logits, ld, tokens, stats, entropy, dlogprob, dentropy, dlogits, ld_d, rows, cols, scale}, BF16,     \
                             (hipStream_t)stream);                                                                                           \
  }
KARMA_LOGPROB_ENTRIES(bf16, void, true)
KARMA_LOGPROB_ENTRIES(f32, float, false)
