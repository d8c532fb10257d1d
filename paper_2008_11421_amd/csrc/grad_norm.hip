// The global norm of many gradients and their clipping:
//   norm = s sqrt(sum over all tensors of sum_i g_i^2),  factor = s min(1, max_norm / norm),  out = factor g.
// Squares and their sums are fp64: the square of a bf16 or fp32 number is exact there and neither overflows nor vanishes, and 217 M
// of them lose nothing that counts.  Every workgroup leaves the sum of its elements in the workspace; those sums are added up in a
// fixed order by one workgroup, so that results are the same from call to call.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_utils.h"
#include "karma.h"
#include "kernels.h"

namespace karma {
namespace {

constexpr int GN_THREADS = 256;
constexpr unsigned GN_GRID = (1u << 24) - 1;        // workgroups of 256 lanes in a launch, which has less than 2^32
// Elements of a workgroup (norm).
constexpr unsigned GN_SPAN = 16384, GN_SPAN_FEW = 4096;
constexpr uint64_t GN_FEW = 16u << 20;
constexpr unsigned GC_SPAN = 4096;                  // (clipping)
static_assert(KARMA_GRAD_VALUES_MAX / GC_SPAN + 1 <= GN_GRID, "a tensor fits a launch");

struct NormTensor {
  const void* grad;
  size_t n;             // the highest bit: bf16
};
struct NormSet {        // the tensors of one launch, as kernel arguments
  static constexpr int MOST = 200;
  NormTensor t[MOST];
  unsigned first[MOST + 1];     // tensor k has workgroups [first[k], first[k + 1])
  int n;
};
struct ClipTensor {
  const void* grad; void* out;
  size_t n;             // the highest bits: bf16, out in bf16
};
struct ClipSet {
  static constexpr int MOST = 144;
  ClipTensor t[MOST];
  unsigned first[MOST + 1];
  int n;
};
struct EachSet {        // tensor k has the partial sums [first[k], first[k + 1])
  static constexpr int MOST = 960;
  unsigned first[MOST + 1];
  int n;
};
static_assert(sizeof(NormSet) + 16 <= 4096 && sizeof(ClipSet) + 16 <= 4096 && sizeof(EachSet) + 64 <= 4096, "kernel arguments");
constexpr size_t BIT_BF16 = (size_t)1 << 63, BIT_OUT = (size_t)1 << 62, BITS = BIT_BF16 | BIT_OUT;

template <typename Set>
__device__ __forceinline__ int tensor_of(const Set& u, unsigned block) {
  int lo = 0, hi = u.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (block >= u.first[mid]) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m, 64);
  return v;
}
// the sum over a workgroup of WAVES wavefronts, in every lane of the first
template <int WAVES>
__device__ __forceinline__ double block_sum64(double v) {
  __shared__ double part[WAVES];
  v = wave_sum64(v);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
  __syncthreads();
  v = threadIdx.x % 64 < WAVES ? part[threadIdx.x % 64] : 0.0;
  return wave_sum64(v);
}

// Vectors of 16 bytes lie on 16-byte boundaries of memory wherever the tensor begins: vector j has the elements j N - skip .. + N,
// those before the first and behind the last one are left out and their vector is read element by element.
template <typename T>
struct Vec16;
template <>
struct Vec16<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const u32x4& v, float* f) { unpack8(v, f); }
  static __device__ __forceinline__ float one(const bf16_t* p) { return bf2f(*p); }
};
template <>
struct Vec16<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const u32x4& v, float* f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(v[e]);
  }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
};

template <typename T>
__device__ __forceinline__ double squares(const T* g, size_t n, size_t at, unsigned span) {
  constexpr int N = Vec16<T>::N, BATCH = 4;
  const unsigned skip = (unsigned)((uintptr_t)g % 16 / sizeof(T));
  double sum = 0.0, sum2 = 0.0;
  const T* base = g - skip;
  for (unsigned v = threadIdx.x * N; v < span; v += GN_THREADS * N * BATCH) {
    u32x4 raw[BATCH];
    bool whole[BATCH];
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const size_t i = at + v + b * (GN_THREADS * N);
      whole[b] = v + b * (GN_THREADS * N) < span && i >= skip && i + N <= n + skip;
      raw[b] = whole[b] ? *(const u32x4*)(base + i) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const size_t i = at + v + b * (GN_THREADS * N);
      float f[N];
      Vec16<T>::unpack(raw[b], f);
      if (!whole[b] && v + b * (GN_THREADS * N) < span) {
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = i + e >= skip && i + e < n + skip ? Vec16<T>::one(base + i + e) : 0.f;
      }
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        sum = fma((double)f[e], (double)f[e], sum);
        sum2 = fma((double)f[e + 1], (double)f[e + 1], sum2);
      }
    }
  }
  return sum + sum2;
}

// partial[workgroup] = the sum of squares of `span` elements of one tensor
__global__ __launch_bounds__(GN_THREADS) void grad_squares_kernel(NormSet u, unsigned span, double* partial) {
  const int k = tensor_of(u, blockIdx.x);
  const size_t n = u.t[k].n & ~BITS, at = (size_t)(blockIdx.x - u.first[k]) * span;
  double s = u.t[k].n & BIT_BF16 ? squares((const bf16_t*)u.t[k].grad, n, at, span) : squares((const float*)u.t[k].grad, n, at, span);
  s = block_sum64<GN_THREADS / 64>(s);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

struct NormOut {
  float* norm; float* factor; float* each;      // each may be null, factor too
  float max_norm, scale;
};
// Workgroup 0 of the first launch: all partial sums.  The others: a wavefront for every tensor's own.
constexpr int FIN_THREADS = 1024;
__global__ __launch_bounds__(FIN_THREADS) void grad_finish_kernel(EachSet u, const double* partial, unsigned total, NormOut o, int with_total) {
  if (with_total && blockIdx.x == 0) {
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (unsigned i = threadIdx.x; i < total; i += 4 * FIN_THREADS)
#pragma unroll
      for (int b = 0; b < 4; ++b) s[b] += i + b * FIN_THREADS < total ? partial[i + b * FIN_THREADS] : 0.0;
    const double sum = block_sum64<FIN_THREADS / 64>((s[0] + s[1]) + (s[2] + s[3]));
    if (threadIdx.x == 0) {
      const double norm = (double)o.scale * sqrt(sum);
      if (o.norm) *o.norm = (float)norm;
      // (a norm that is not a number gives a factor that is none; an infinite one gives 0)
      if (o.factor) *o.factor = (float)((double)o.scale * (norm <= (double)o.max_norm ? 1.0 : (double)o.max_norm / norm));
    }
    return;
  }
  const int k = ((int)blockIdx.x - with_total) * (FIN_THREADS / 64) + threadIdx.x / 64;
  if (k >= u.n) return;
  double s = 0.0;
  for (unsigned i = u.first[k] + threadIdx.x % 64; i < u.first[k + 1]; i += 64) s += partial[i];
  s = wave_sum64(s);
  if (threadIdx.x % 64 == 0) o.each[k] = (float)((double)o.scale * sqrt(s));
}

template <typename T, typename O>
__device__ __forceinline__ void clip_span(const T* g, O* out, size_t n, size_t at, float factor) {
  constexpr int N = Vec16<T>::N, BATCH = GC_SPAN / (GN_THREADS * N);
  const unsigned skip = (unsigned)((uintptr_t)g % 16 / sizeof(T));
  const T* base = g - skip;
  O* to = out - skip;
  constexpr size_t OUT_BYTES = N * sizeof(O) < 16 ? N * sizeof(O) : 16;
  const bool fits = (uintptr_t)to % OUT_BYTES == 0;
  u32x4 raw[BATCH];
#pragma unroll
  for (int b = 0; b < BATCH; ++b) {
    const size_t i = at + (threadIdx.x + b * GN_THREADS) * N;
    raw[b] = i >= skip && i + N <= n + skip ? *(const u32x4*)(base + i) : u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int b = 0; b < BATCH; ++b) {
    const size_t i = at + (threadIdx.x + b * GN_THREADS) * N;
    if (i >= n + skip) continue;
    const bool whole = i >= skip && i + N <= n + skip;
    float f[N];
    Vec16<T>::unpack(raw[b], f);
    if (!whole) {
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] = i + e >= skip && i + e < n + skip ? Vec16<T>::one(base + i + e) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] *= factor;
    if (whole && fits) {
      if constexpr (sizeof(O) == 2) {
        if constexpr (N == 8) *(u32x4*)(to + i) = pack8(f);
        else *(u32x2*)(to + i) = u32x2{pack2(f[0], f[1]), pack2(f[2], f[3])};
      } else {
#pragma unroll
        for (int e = 0; e < N; e += 4)
          *(u32x4*)(to + i + e) = u32x4{__float_as_uint(f[e]), __float_as_uint(f[e + 1]), __float_as_uint(f[e + 2]), __float_as_uint(f[e + 3])};
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (i + e >= skip && i + e < n + skip) {
          if constexpr (sizeof(O) == 2) to[i + e] = f2bf(f[e]);
          else to[i + e] = f[e];
        }
    }
  }
}

__global__ __launch_bounds__(GN_THREADS) void grad_clip_kernel(ClipSet u, const float* factor) {
  const int k = tensor_of(u, blockIdx.x);
  const size_t bits = u.t[k].n, n = bits & ~BITS, at = (size_t)(blockIdx.x - u.first[k]) * GC_SPAN;
  const void* g = u.t[k].grad;
  void* out = u.t[k].out;
  const float f = *factor;
  const bool gbf = bits & BIT_BF16, obf = bits & BIT_OUT;
  if (f == 1.f && g == out && gbf == obf) return;      // nothing changes
  if (gbf) {
    if (obf) clip_span((const bf16_t*)g, (bf16_t*)out, n, at, f);
    else clip_span((const bf16_t*)g, (float*)out, n, at, f);
  } else {
    if (obf) clip_span((const float*)g, (bf16_t*)out, n, at, f);
    else clip_span((const float*)g, (float*)out, n, at, f);
  }
}

bool aligned_to(const void* p, size_t n) { return (uintptr_t)p % n == 0; }
size_t grad_size(const karma_grad_tensor& t) { return t.flags & KARMA_GRAD_BF16 ? 2 : 4; }
bool good_grads(const karma_grad_tensor* tensors, uint32_t n) {
  if (n > KARMA_GRAD_TENSORS_MAX) return false;
  uint64_t all = 0;
  for (uint32_t k = 0; k < n; ++k) {
    const karma_grad_tensor& t = tensors[k];
    if ((t.flags & ~3u) || t.n > KARMA_GRAD_VALUES_MAX) return false;
    if (t.n && (!t.grad || !aligned_to(t.grad, grad_size(t)))) return false;
    all += t.n;
    if (all > KARMA_GRAD_VALUES_MAX) return false;
  }
  return true;
}
// vectors begin up to one vector before the tensor
uint64_t spans(const karma_grad_tensor& t, unsigned span) {
  return t.n ? (t.n + (uintptr_t)t.grad % 16 / grad_size(t) + span - 1) / span : 0;
}
unsigned norm_span(const karma_grad_tensor* tensors, uint32_t n) {
  uint64_t all = 0;
  for (uint32_t k = 0; k < n; ++k) all += tensors[k].n;
  return all > GN_FEW ? GN_SPAN : GN_SPAN_FEW;
}

}  // namespace

size_t grad_norm_ws_bytes(const karma_grad_tensor* tensors, uint32_t n) {
  if (!good_grads(tensors, n)) return 0;
  const unsigned span = norm_span(tensors, n);
  uint64_t blocks = 0;
  for (uint32_t k = 0; k < n; ++k) blocks += spans(tensors[k], span);
  return std::max<uint64_t>(blocks, 1) * sizeof(double);
}

int grad_norm(const karma_grad_tensor* tensors, uint32_t n, float max_norm, float scale, float* norm, float* each, float* factor, void* ws,
              size_t ws_bytes, hipStream_t s) {
  if (!good_grads(tensors, n) || !(max_norm > 0.f) || !(scale > 0.f && scale <= 3.4028234e38f)) return KARMA_E_INVAL;
  if ((!norm && !factor && !each) || !aligned_to(norm, 4) || !aligned_to(factor, 4) || !aligned_to(each, 4)) return KARMA_E_INVAL;
  if (!ws || ws_bytes < grad_norm_ws_bytes(tensors, n)) return KARMA_E_OOM;
  if (!aligned_to(ws, 16)) return KARMA_E_INVAL;
  double* partial = (double*)ws;
  const unsigned span = norm_span(tensors, n);
  uint64_t total = 0;
  for (uint32_t k = 0; k < n;) {
    NormSet u;
    u.n = 0;
    u.first[0] = 0;
    uint64_t blocks = 0;
    for (; k < n && u.n < NormSet::MOST; ++k) {
      const uint64_t more = spans(tensors[k], span);
      if (!more) continue;
      if (blocks + more > GN_GRID) break;
      u.t[u.n] = NormTensor{tensors[k].grad, tensors[k].n | (tensors[k].flags & KARMA_GRAD_BF16 ? BIT_BF16 : 0)};
      blocks += more;
      u.first[++u.n] = (unsigned)blocks;
    }
    if (!u.n) continue;
    hipLaunchKernelGGL(grad_squares_kernel, dim3((unsigned)blocks), dim3(GN_THREADS), 0, s, u, span, partial + total);
    total += blocks;
  }
  NormOut o{norm, factor, each, max_norm, scale};
  uint64_t before = 0;
  bool first = norm || factor;
  uint32_t k = 0;
  do {
    EachSet u;
    u.n = 0;
    u.first[0] = (unsigned)before;
    if (each)
      for (; k < n && u.n < EachSet::MOST; ++k) {
        before += spans(tensors[k], span);
        u.first[++u.n] = (unsigned)before;
      }
    const unsigned grid = (first ? 1 : 0) + (u.n + FIN_THREADS / 64 - 1) / (FIN_THREADS / 64);
    if (grid) hipLaunchKernelGGL(grad_finish_kernel, dim3(grid), dim3(FIN_THREADS), 0, s, u, partial, (unsigned)total, o, first ? 1 : 0);
    o.each = each ? o.each + u.n : nullptr;
    first = false;
  } while (each && k < n);
  return hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

int grad_clip(const karma_grad_tensor* tensors, uint32_t n, const float* factor, hipStream_t s) {
  if (!good_grads(tensors, n) || !factor || !aligned_to(factor, 4)) return KARMA_E_INVAL;
  for (uint32_t k = 0; k < n; ++k)
    if (tensors[k].n && (!tensors[k].out || !aligned_to(tensors[k].out, tensors[k].flags & KARMA_GRAD_OUT_BF16 ? 2 : 4))) return KARMA_E_INVAL;
  bool launched = false;
  for (uint32_t k = 0; k < n;) {
    ClipSet u;
    u.n = 0;
    u.first[0] = 0;
    uint64_t blocks = 0;
    for (; k < n && u.n < ClipSet::MOST; ++k) {
      const karma_grad_tensor& t = tensors[k];
      const uint64_t more = spans(t, GC_SPAN);
      if (!more) continue;
      if (blocks + more > GN_GRID) break;
      u.t[u.n] = ClipTensor{t.grad, t.out, t.n | (t.flags & KARMA_GRAD_BF16 ? BIT_BF16 : 0) | (t.flags & KARMA_GRAD_OUT_BF16 ? BIT_OUT : 0)};
      blocks += more;
      u.first[++u.n] = (unsigned)blocks;
    }
    if (!u.n) continue;
    hipLaunchKernelGGL(grad_clip_kernel, dim3((unsigned)blocks), dim3(GN_THREADS), 0, s, u, factor);
    launched = true;
  }
  return !launched || hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

}  // namespace karma

using namespace karma;

extern "C" uint64_t karma_k_grad_norm_ws_bytes(const karma_grad_tensor* tensors, uint32_t n) {
  return n && !tensors ? 0 : grad_norm_ws_bytes(tensors, n);
}
extern "C" int karma_k_grad_norm(const karma_grad_tensor* tensors, uint32_t n, float max_norm, float grad_scale, float* norm, float* tensor_norms,
                                 float* factor, void* ws, uint64_t ws_bytes, void* stream) {
  if (n && !tensors) return KARMA_E_INVAL;
  return grad_norm(tensors, n, max_norm, grad_scale, norm, tensor_norms, factor, ws, ws_bytes, (hipStream_t)stream);
}
extern "C" int karma_k_grad_clip(const karma_grad_tensor* tensors, uint32_t n, const float* factor, void* stream) {
  if (n && !tensors) return KARMA_E_INVAL;
  return grad_clip(tensors, n, factor, (hipStream_t)stream);
}
