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
constexpr unsigned GC_SPAN = 4096;                  // elements of a workgroup (clipping)

// The tensors of one launch travel as kernel arguments, 4 KB in all: addresses of 48 bits with what is known of them above, the elements of a
// tensor's last workgroup, and the workgroups before it.
constexpr uint64_t BIT_BF16 = 1ull << 63, ADDRESS = (1ull << 48) - 1;
struct NormSet {
  static constexpr int MOST = 288;
  uint64_t grad[MOST];
  unsigned first[MOST + 1];     // tensor k has workgroups [first[k], first[k + 1])
  unsigned short last[MOST];    // elements of its last one, less one
  int n;
};
struct ClipSet {
  static constexpr int MOST = 184;
  uint64_t grad[MOST], out[MOST];
  unsigned first[MOST + 1];
  unsigned short last[MOST];
  int n;
};
struct EachSet {        // tensor k has the partial sums [first[k], first[k + 1])
  static constexpr int MOST = 960;
  unsigned first[MOST + 1];
  int n;
};
// (a tensor has up to two spans more than its values fill; the norm's spans are as long or longer)
static_assert(KARMA_GRAD_VALUES_MAX / GC_SPAN + 2 * NormSet::MOST <= GN_GRID && ClipSet::MOST <= NormSet::MOST, "the tensors of a launch fit it");
static_assert(sizeof(NormSet) + 16 <= 4096 && sizeof(ClipSet) + 16 <= 4096 && sizeof(EachSet) + 64 <= 4096, "kernel arguments");

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

// The elements [skip, n) of a span behind `base`, which lies on a 16-byte boundary.
template <typename T>
__device__ __forceinline__ double squares(const T* base, unsigned skip, unsigned n) {
  constexpr int N = Vec16<T>::N, BATCH = 4;
  double sum = 0.0, sum2 = 0.0;
  for (unsigned v = threadIdx.x * N; v < n; v += GN_THREADS * N * BATCH) {
    u32x4 raw[BATCH];
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const unsigned i = v + b * (GN_THREADS * N);
      raw[b] = i >= skip && i + N <= n ? *(const u32x4*)(base + i) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const unsigned i = v + b * (GN_THREADS * N);
      float f[N];
      Vec16<T>::unpack(raw[b], f);
      if (i < n && (i < skip || i + N > n)) {
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = i + e >= skip && i + e < n ? Vec16<T>::one(base + i + e) : 0.f;
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
// Workgroup `block` of tensor k: its elements [skip, n) behind *base.
template <typename T, typename Set>
__device__ __forceinline__ const T* span_of(const Set& u, int k, unsigned block, unsigned span, unsigned& skip, unsigned& n) {
  const T* g = (const T*)(uintptr_t)(u.grad[k] & ADDRESS);
  const unsigned before = (unsigned)((uintptr_t)g % 16 / sizeof(T)), at = block - u.first[k];
  skip = at ? 0 : before;
  n = block + 1 == u.first[k + 1] ? u.last[k] + 1u : span;
  return g - before + (size_t)at * span;
}

// Reads every value once, with a conversion and a product-and-sum of 64 bits for each: bound by memory (217 M values in bf16 72 us, 6.0 TB/s) and, in
// lists of many tensors, by launches of 288 tensors that drain one after the other (609 tensors of 63 M values 44 us).  A search of the workgroup's
// tensor by all lanes at once instead of step by step made no difference.
// partial[workgroup] = the sum of squares of `span` elements of one tensor
__global__ __launch_bounds__(GN_THREADS) void grad_squares_kernel(NormSet u, unsigned span, double* partial) {
  const int k = tensor_of(u, blockIdx.x);
  unsigned skip, n;
  double s;
  if (u.grad[k] & BIT_BF16) {
    const bf16_t* g = span_of<bf16_t>(u, k, blockIdx.x, span, skip, n);
    s = squares(g, skip, n);
  } else {
    const float* g = span_of<float>(u, k, blockIdx.x, span, skip, n);
    s = squares(g, skip, n);
  }
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

// Reads and writes every value once: 5.0 to 5.3 TB/s (609 tensors of 63 M values in bf16 50 us in four launches, 15.8 M from fp32 to bf16 17.7 us).
// Workgroups in falling order, which find more of what the norm has read last in the cache, took as long.
template <typename T, typename O>
__device__ __forceinline__ void clip_span(const ClipSet& u, int k, unsigned block, float factor) {
  constexpr int N = Vec16<T>::N, BATCH = GC_SPAN / (GN_THREADS * N);
  unsigned skip, n;
  const T* base = span_of<T>(u, k, block, GC_SPAN, skip, n);
  O* to = (O*)(uintptr_t)(u.out[k] & ADDRESS) + (base - (const T*)(uintptr_t)(u.grad[k] & ADDRESS));
  constexpr size_t OUT_BYTES = N * sizeof(O) < 16 ? N * sizeof(O) : 16;
  const bool fits = (uintptr_t)to % OUT_BYTES == 0;
  u32x4 raw[BATCH];
#pragma unroll
  for (int b = 0; b < BATCH; ++b) {
    const unsigned i = (threadIdx.x + b * GN_THREADS) * N;
    raw[b] = i >= skip && i + N <= n ? *(const u32x4*)(base + i) : u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int b = 0; b < BATCH; ++b) {
    const unsigned i = (threadIdx.x + b * GN_THREADS) * N;
    if (i >= n) continue;
    const bool whole = i >= skip && i + N <= n;
    float f[N];
    Vec16<T>::unpack(raw[b], f);
    if (!whole) {
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] = i + e >= skip && i + e < n ? Vec16<T>::one(base + i + e) : 0.f;
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
        if (i + e >= skip && i + e < n) {
          if constexpr (sizeof(O) == 2) to[i + e] = f2bf(f[e]);
          else to[i + e] = f[e];
        }
    }
  }
}

__global__ __launch_bounds__(GN_THREADS) void grad_clip_kernel(ClipSet u, const float* factor) {
  const unsigned block = blockIdx.x;
  const int k = tensor_of(u, block);
  const float f = *factor;
  const bool gbf = u.grad[k] & BIT_BF16, obf = u.out[k] & BIT_BF16;
  if (f == 1.f && u.grad[k] == u.out[k]) return;      // nothing changes
  if (gbf) {
    if (obf) clip_span<bf16_t, bf16_t>(u, k, block, f);
    else clip_span<bf16_t, float>(u, k, block, f);
  } else {
    if (obf) clip_span<float, bf16_t>(u, k, block, f);
    else clip_span<float, float>(u, k, block, f);
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
    if (t.n && (!t.grad || !aligned_to(t.grad, grad_size(t)) || (uintptr_t)t.grad > ADDRESS)) return false;
    all += t.n;
    if (all > KARMA_GRAD_VALUES_MAX) return false;
  }
  return true;
}
// vectors begin up to one vector before the tensor
uint64_t extent(const karma_grad_tensor& t) { return t.n ? t.n + (uintptr_t)t.grad % 16 / grad_size(t) : 0; }
uint64_t spans(const karma_grad_tensor& t, unsigned span) { return (extent(t) + span - 1) / span; }
uint64_t address(const void* p, bool bf16) { return ((uint64_t)(uintptr_t)p & ADDRESS) | (bf16 ? BIT_BF16 : 0); }
// Elements of a workgroup: few where workgroups are few (16 tensors of 0.5 M values in all 4.2 us in the kernel), more in long lists, for
// fewer sums to add up (one of 217 M in workgroups of 16384 / 32768: 76.6 / 78.7 us; 609 tensors of 63 M, clipped, of 8192 / 16384 / 32768: 99 / 100 / 101).
unsigned norm_span(const karma_grad_tensor* tensors, uint32_t n) {
  uint64_t all = 0;
  for (uint32_t k = 0; k < n; ++k) all += tensors[k].n;
  return all <= 16u << 20 ? 4096 : 16384;
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
      u.grad[u.n] = address(tensors[k].grad, tensors[k].flags & KARMA_GRAD_BF16);
      u.last[u.n] = (unsigned short)((extent(tensors[k]) - 1) % span);
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
  bool launched = total > 0;
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
    launched |= grid > 0;
    o.each = each ? o.each + u.n : nullptr;
    first = false;
  } while (each && k < n);
  return !launched || hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

int grad_clip(const karma_grad_tensor* tensors, uint32_t n, const float* factor, hipStream_t s) {
  if (!good_grads(tensors, n) || !factor || !aligned_to(factor, 4)) return KARMA_E_INVAL;
  for (uint32_t k = 0; k < n; ++k) {
    const karma_grad_tensor& t = tensors[k];
    const size_t out_size = t.flags & KARMA_GRAD_OUT_BF16 ? 2 : 4;
    if (t.n && (!t.out || (uintptr_t)t.out > ADDRESS || !aligned_to(t.out, out_size))) return KARMA_E_INVAL;
    // in place: a lane reads what it writes, and no other one does, if both have one size
    if (t.n && t.out == t.grad && out_size != grad_size(t)) return KARMA_E_INVAL;
  }
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
      u.grad[u.n] = address(t.grad, t.flags & KARMA_GRAD_BF16);
      u.out[u.n] = address(t.out, t.flags & KARMA_GRAD_OUT_BF16);
      u.last[u.n] = (unsigned short)((extent(t) - 1) % GC_SPAN);
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
