// Gated linear recurrence over packed sequences, forward and backward:
//   b_t = 1 / (1 + e^f_t)  (one minus the gate's sigmoid),  h_t = h_{t-1} + b_t (x_t - h_{t-1}).
// Gradients, from the last token to the first, with g the gradient of the state behind the token:
//   D_t = dh_t + g,  dx_t = b_t D_t,  df_t = D_t (h_{t-1} - x_t) (b_t - b_t^2),  g = D_t - b_t D_t.
// The weight b of the new value is computed, not the decay 1 - b: where a state lives for thousands of tokens b is small,
// and 1 - b rounded to 32 bits would lose it.  States and carries are fp32.
#include <hip/hip_runtime.h>

#include "device_utils.h"
#include "karma.h"
#include "kernels.h"

namespace karma {
namespace {

template <typename T>
__device__ __forceinline__ float load1(const T* p);
template <>
__device__ __forceinline__ float load1<bf16_t>(const bf16_t* p) { return bf2f(*p); }
template <>
__device__ __forceinline__ float load1<float>(const float* p) { return *p; }
__device__ __forceinline__ void store1(bf16_t* p, float v) { *p = f2bf(v); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }

__device__ __forceinline__ float share_of(float f) { return 1.f / (1.f + __expf(f)); }

struct ScanSpan { long first, last; };   // tokens [first, last) of a sequence
__device__ __forceinline__ ScanSpan span_of(const int* starts, long tokens, unsigned sequences, unsigned j) {
  if (!starts) { const long n = tokens / sequences; return ScanSpan{j * n, (j + 1) * n}; }
  // whatever the starts say, no token outside the tensors is touched
  const long a = starts[j], e = starts[j + 1];
  return ScanSpan{a < 0 ? 0 : a > tokens ? tokens : a, e < 0 ? 0 : e > tokens ? tokens : e};
}

template <typename T>
__global__ __launch_bounds__(64) void scan_fwd_kernel(ScanFwd a) {
  const unsigned cols = (a.s.channels + 63) / 64, j = blockIdx.x / cols, c = blockIdx.x % cols * 64 + threadIdx.x;
  if (c >= a.s.channels) return;
  const ScanSpan p = span_of(a.starts, a.s.tokens, a.s.sequences, j);
  float h = a.h0 ? a.h0[(size_t)j * a.s.channels + c] : 0.f;
  for (long t = p.first; t < p.last; ++t) {
    if (a.marks && t % KARMA_SCAN_MARK == 0) a.marks[(size_t)(t / KARMA_SCAN_MARK) * a.s.channels + c] = h;
    const float b = share_of(load1((const T*)a.gate + t * a.s.ld_gate + c)), x = load1((const T*)a.x + t * a.s.ld_x + c);
    h = fmaf(b, x - h, h);
    store1((T*)a.h + t * a.s.ld_h + c, h);
  }
  if (a.h_last) a.h_last[(size_t)j * a.s.channels + c] = h;
}

template <typename T>
__global__ __launch_bounds__(64) void scan_bwd_kernel(ScanBwd a) {
  __shared__ float before[KARMA_SCAN_MARK][64];
  const unsigned cols = (a.s.channels + 63) / 64, j = blockIdx.x / cols, c = blockIdx.x % cols * 64 + threadIdx.x;
  if (c >= a.s.channels) return;
  const ScanSpan p = span_of(a.starts, a.s.tokens, a.s.sequences, j);
  const size_t at = (size_t)j * a.s.channels + c;
  float g = a.dh_last ? a.dh_last[at] : 0.f;
  for (long end = p.last; end > p.first;) {
    const long mark = (end - 1) / KARMA_SCAN_MARK * KARMA_SCAN_MARK, begin = mark > p.first ? mark : p.first;
    float h = mark > p.first ? a.marks[(size_t)(mark / KARMA_SCAN_MARK) * a.s.channels + c] : a.h0 ? a.h0[at] : 0.f;
    for (long t = begin; t < end; ++t) {
      before[t - begin][threadIdx.x] = h;
      const float b = share_of(load1((const T*)a.gate + t * a.s.ld_gate + c)), x = load1((const T*)a.x + t * a.s.ld_x + c);
      h = fmaf(b, x - h, h);
    }
    for (long t = end - 1; t >= begin; --t) {
      const float b = share_of(load1((const T*)a.gate + t * a.s.ld_gate + c)), x = load1((const T*)a.x + t * a.s.ld_x + c);
      const float D = load1((const T*)a.dh + t * a.s.ld_h + c) + g;
      store1((T*)a.dx + t * a.s.ld_dx + c, b * D);
      store1((T*)a.dgate + t * a.s.ld_dgate + c, D * (before[t - begin][threadIdx.x] - x) * fmaf(-b, b, b));
      g = fmaf(-b, D, D);
    }
    end = begin;
  }
  if (a.dh0) a.dh0[at] = g;
}

// Sizes and strides as a call may give them; a stride of 0 becomes the number of channels.
int check_scan(karma_scan_shape& s, const void* starts) {
  if (!s.channels || !s.sequences || s.tokens > INT32_MAX || s.channels > INT32_MAX || s.sequences >= INT32_MAX) return KARMA_E_INVAL;
  if (!starts && s.tokens % s.sequences) return KARMA_E_INVAL;
  for (uint64_t* ld : {&s.ld_gate, &s.ld_x, &s.ld_h, &s.ld_dgate, &s.ld_dx}) {
    if (!*ld) *ld = s.channels;
    if (*ld < s.channels || *ld > INT64_MAX / 8 / (s.tokens + 1)) return KARMA_E_INVAL;
  }
  if ((uint64_t)((s.channels + 63) / 64) * s.sequences > INT32_MAX) return KARMA_E_INVAL;
  return KARMA_OK;
}
bool aligned_to(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

}  // namespace

size_t gated_scan_ws_bytes(const karma_scan_shape&) { return 0; }

int gated_scan_fwd(ScanFwd a, bool bf16, hipStream_t s) {
  const size_t e = bf16 ? 2 : 4;
  if (int st = check_scan(a.s, a.starts)) return st;
  if (a.s.tokens && (!a.gate || !a.x || !a.h)) return KARMA_E_INVAL;
  if (!aligned_to(a.gate, e) || !aligned_to(a.x, e) || !aligned_to(a.h, e)) return KARMA_E_INVAL;
  if (a.ws_bytes < gated_scan_ws_bytes(a.s)) return KARMA_E_OOM;
  const dim3 grid((a.s.channels + 63) / 64 * a.s.sequences);
  if (bf16) hipLaunchKernelGGL(scan_fwd_kernel<bf16_t>, grid, dim3(64), 0, s, a);
  else hipLaunchKernelGGL(scan_fwd_kernel<float>, grid, dim3(64), 0, s, a);
  return hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

int gated_scan_bwd(ScanBwd a, bool bf16, hipStream_t s) {
  const size_t e = bf16 ? 2 : 4;
  if (int st = check_scan(a.s, a.starts)) return st;
  if (a.s.tokens && (!a.gate || !a.x || !a.marks || !a.dh || !a.dgate || !a.dx)) return KARMA_E_INVAL;
  if (!aligned_to(a.gate, e) || !aligned_to(a.x, e) || !aligned_to(a.dh, e) || !aligned_to(a.dgate, e) || !aligned_to(a.dx, e)) return KARMA_E_INVAL;
  if (a.ws_bytes < gated_scan_ws_bytes(a.s)) return KARMA_E_OOM;
  const dim3 grid((a.s.channels + 63) / 64 * a.s.sequences);
  if (bf16) hipLaunchKernelGGL(scan_bwd_kernel<bf16_t>, grid, dim3(64), 0, s, a);
  else hipLaunchKernelGGL(scan_bwd_kernel<float>, grid, dim3(64), 0, s, a);
  return hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

}  // namespace karma

using namespace karma;

static int scan_fwd_entry(const void* gate, const void* x, const float* h0, const int32_t* starts, void* h, float* h_last, float* marks,
                          const karma_scan_shape* shape, void* ws, uint64_t ws_bytes, bool bf16, void* stream) {
  if (!shape) return KARMA_E_INVAL;
  return gated_scan_fwd(ScanFwd{gate, x, h0, starts, h, h_last, marks, *shape, ws, ws ? ws_bytes : 0}, bf16, (hipStream_t)stream);
}
static int scan_bwd_entry(const void* gate, const void* x, const float* h0, const int32_t* starts, const float* marks, const void* dh,
                          const float* dh_last, void* dgate, void* dx, float* dh0, const karma_scan_shape* shape, void* ws, uint64_t ws_bytes,
                          bool bf16, void* stream) {
  if (!shape) return KARMA_E_INVAL;
  return gated_scan_bwd(ScanBwd{gate, x, h0, starts, marks, dh, dh_last, dgate, dx, dh0, *shape, ws, ws ? ws_bytes : 0}, bf16,
                        (hipStream_t)stream);
}

extern "C" uint64_t karma_k_gated_scan_ws_bytes(const karma_scan_shape* shape) { return shape ? gated_scan_ws_bytes(*shape) : 0; }
extern "C" int karma_k_gated_scan_fwd_bf16(const void* gate, const void* x, const float* h0, const int32_t* starts, void* h, float* h_last,
                                           float* marks, const karma_scan_shape* shape, void* ws, uint64_t ws_bytes, void* stream) {
  return scan_fwd_entry(gate, x, h0, starts, h, h_last, marks, shape, ws, ws_bytes, true, stream);
}
extern "C" int karma_k_gated_scan_fwd_f32(const float* gate, const float* x, const float* h0, const int32_t* starts, float* h, float* h_last,
                                          float* marks, const karma_scan_shape* shape, void* ws, uint64_t ws_bytes, void* stream) {
  return scan_fwd_entry(gate, x, h0, starts, h, h_last, marks, shape, ws, ws_bytes, false, stream);
}
extern "C" int karma_k_gated_scan_bwd_bf16(const void* gate, const void* x, const float* h0, const int32_t* starts, const float* marks,
                                           const void* dh, const float* dh_last, void* dgate, void* dx, float* dh0,
                                           const karma_scan_shape* shape, void* ws, uint64_t ws_bytes, void* stream) {
  return scan_bwd_entry(gate, x, h0, starts, marks, dh, dh_last, dgate, dx, dh0, shape, ws, ws_bytes, true, stream);
}
extern "C" int karma_k_gated_scan_bwd_f32(const float* gate, const float* x, const float* h0, const int32_t* starts, const float* marks,
                                          const float* dh, const float* dh_last, float* dgate, float* dx, float* dh0,
                                          const karma_scan_shape* shape, void* ws, uint64_t ws_bytes, void* stream) {
  return scan_bwd_entry(gate, x, h0, starts, marks, dh, dh_last, dgate, dx, dh0, shape, ws, ws_bytes, false, stream);
}
