// Draws a token from every row of logits: temperature, top-k, top-p, min-p, one uniform number a row.
// With m the row's largest logit, token j weighs w_j = rint(2^40 e^((z_j - m) / T)).  Whole numbers: their sums are exact and the
// same in whatever order lanes, wavefronts and passes take them, so which token stays and which is drawn hangs on no order.
// Tokens are ordered by falling logit, equal ones by rising index; what top-k and top-p leave is a beginning of that order, "all before
// the pair (logit, index)", and min-p cuts its end off by weight.  The pair is found without sorting: the row is counted (or weighed)
// into 2048 bins of equal width in (m - z) / T, the bin that the border falls into is cut again by the bits of its logits, until a bin is a single
// value; of its tokens, which weigh the same, the first ones by index stay.
// A workgroup has a row and goes over it several times: the first time from memory, then from the L2.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_utils.h"
#include "karma.h"
#include "kernels.h"

namespace karma {
namespace {

typedef unsigned long long u64;
constexpr unsigned SP_GRID = 1u << 20;
constexpr int BINS = 2048, LAST = BINS - 1;
constexpr double ONE = 1099511627776.0;     // 2^40
// bins reach down to weights of 2^-42 of the largest: what falls into the last one weighs nothing
constexpr float REACH = 42.f * 0.69314718f;

// A row in 16-byte vectors on 16-byte boundaries: vector v has the columns v N - skip .. + N.
template <typename T>
struct RowVec;
template <>
struct RowVec<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const u32x4& v, float* f) { unpack8(v, f); }
  static __device__ __forceinline__ float one(const bf16_t* p) { return bf2f(*p); }
  // the order of logits as whole numbers
  static __device__ __forceinline__ unsigned key(float z) {
    const unsigned u = __float_as_uint(z + 0.f);
    return ((int)u < 0 ? ~u : u | 0x80000000u) >> 16;
  }
  static __device__ __forceinline__ float value(unsigned key) {
    const unsigned u = key << 16;
    return __uint_as_float((int)u < 0 ? u & 0x7fffffffu : ~u & 0xffff0000u);
  }
};
template <>
struct RowVec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const u32x4& v, float* f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(v[e]);
  }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
  static __device__ __forceinline__ unsigned key(float z) {
    const unsigned u = __float_as_uint(z + 0.f);
    return (int)u < 0 ? ~u : u | 0x80000000u;
  }
  static __device__ __forceinline__ float value(unsigned key) { return __uint_as_float((int)key < 0 ? key & 0x7fffffffu : ~key); }
};

// rint(2^40 2^y), y <= 0: 2^f on [-1/2, 1/2] as 1 + f q(f), q through the Chebyshev nodes, off by 2^-50 of itself; 2^0 is 1
__device__ __forceinline__ double weight_of(double y) {
  y = fmax(y, -64.0);
  const double n = rint(y), f = y - n;
  double q = 0x1.e5e9f548e5726p-28;
  q = fma(q, f, 0x1.b6571de2f2351p-24);
  q = fma(q, f, 0x1.62bfe46117445p-20);
  q = fma(q, f, 0x1.ffcb76789860fp-17);
  q = fma(q, f, 0x1.4309130378460p-13);
  q = fma(q, f, 0x1.5d87fe908f88ap-10);
  q = fma(q, f, 0x1.3b2ab6fba385fp-7);
  q = fma(q, f, 0x1.c6b08d7044119p-5);
  q = fma(q, f, 0x1.ebfbdff82c590p-3);
  q = fma(q, f, 0x1.62e42fefa39f7p-1);
  return rint(ldexp(fma(q, f, 1.0), (int)n + 40));
}

__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) v += (u64)__shfl_xor((long long)v, m, 64);
  return v;
}
__device__ __forceinline__ u64 wave_scan_u64(u64 v) {      // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const u64 o = (u64)__shfl_up((long long)v, m, 64);
    if (lane >= m) v += o;
  }
  return v;
}

template <int THREADS>
struct SampleShared {
  u64 mass[BINS];
  u64 total[THREADS / 64];
  u64 found_before;
  unsigned count[BINS];
  unsigned lo[THREADS / 64], hi[THREADS / 64];
  float top[THREADS / 64];
  unsigned found, found_in;
  int bad;
};

// The tokens that stay: those of a key above `key`, and of `key` itself those with an index up to `last`.
struct Border {
  unsigned key;
  unsigned last;
  __device__ __forceinline__ bool stays(unsigned k, unsigned index) const { return k > key || (k == key && index <= last); }
};

template <typename T, int THREADS>
struct Sampler {
  static constexpr int N = RowVec<T>::N, WAVES = THREADS / 64, BATCH = 4, TILE = 64 * N;
  typedef RowVec<T> R;
  const T* row;
  unsigned cols, skip;
  unsigned begin, end;      // tiles of this wavefront
  SampleShared<THREADS>& sh;
  int lane, wave;
  float m, s;               // largest logit; bins per logit
  double c;                 // log2 e / temperature

  __device__ __forceinline__ Sampler(SampleShared<THREADS>& shared) : sh(shared) {}

  __device__ __forceinline__ void read(unsigned tile, float* z) const {
    const unsigned at = tile * TILE + lane * N;      // column + skip
    if (at >= skip && at + N <= cols + skip) {
      R::unpack(*(const u32x4*)(row + at - skip), z);
      return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = at + e >= skip && at + e < cols + skip ? R::one(row + at + e - skip) : -INFINITY;
  }
  // f(z, column of the first) for the tiles of this wavefront, in order
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    unsigned t = begin;
    for (; t + BATCH <= end; t += BATCH) {
      float z[BATCH][N];
#pragma unroll
      for (int b = 0; b < BATCH; ++b) read(t + b, z[b]);
#pragma unroll
      for (int b = 0; b < BATCH; ++b) f(z[b], (t + b) * TILE + lane * N - skip);
    }
    for (; t < end; ++t) {
      float z[N];
      read(t, z);
      f(z, t * TILE + lane * N - skip);
    }
  }
  __device__ __forceinline__ int bin(float z) const { return (int)fminf((m - z) * s, (float)LAST); }
  __device__ __forceinline__ double weight(float z) const { return weight_of(((double)z - (double)m) * c); }

  __device__ __forceinline__ u64 block_sum(u64 v) const {
    v = wave_sum_u64(v);
    __syncthreads();
    if (lane == 0) sh.total[wave] = v;
    __syncthreads();
    u64 all = 0;
    for (int w = 0; w < WAVES; ++w) all += sh.total[w];
    return all;
  }
  __device__ __forceinline__ void clear_bins() const {
    __syncthreads();
    for (int i = threadIdx.x; i < BINS; i += THREADS) { sh.mass[i] = 0; sh.count[i] = 0; }
    __syncthreads();
  }
  // The first bin up to which there are `need` (at least 1) in all, and what lies before it: true if there is one.
  __device__ __forceinline__ bool find(bool by_mass, u64 need, unsigned& which, u64& before) const {
    constexpr int PER = BINS / THREADS;
    u64 own[PER], sum = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      own[i] = by_mass ? sh.mass[threadIdx.x * PER + i] : sh.count[threadIdx.x * PER + i];
      sum += own[i];
    }
    const u64 upto = wave_scan_u64(sum);
    if (lane == 63) sh.total[wave] = upto;
    if (threadIdx.x == 0) sh.found = BINS;
    __syncthreads();
    u64 at = upto - sum;
    for (int w = 0; w < wave; ++w) at += sh.total[w];
    if (at < need && at + sum >= need) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        if (at < need && at + own[i] >= need) { sh.found = threadIdx.x * PER + i; sh.found_before = at; }
        at += own[i];
      }
    }
    __syncthreads();
    which = sh.found;
    before = sh.found_before;
    return which < BINS;
  }

  // The column at which sum over columns of f (whole numbers) first exceeds `target`
  template <class F>
  __device__ __forceinline__ unsigned locate(F f, u64 target) const {
    u64 mine = 0;
    each([&](const float* z, unsigned col) {
#pragma unroll
      for (int e = 0; e < N; ++e) mine += f(z[e], col + e);
    });
    mine = wave_sum_u64(mine);
    __syncthreads();
    if (lane == 0) sh.total[wave] = mine;
    __syncthreads();
    return walk(f, target);
  }
  // ... where the sums of the wavefronts are in sh.total already
  template <class F>
  __device__ __forceinline__ unsigned walk(F f, u64 target) const {
    u64 at = 0;
    for (int w = 0; w < wave; ++w) at += sh.total[w];
    if (at <= target && target < at + sh.total[wave]) {
      for (unsigned t = begin; t < end; ++t) {
        float z[N];
        read(t, z);
        const unsigned col = t * TILE + lane * N - skip;
        u64 own[N], sum = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) { own[e] = f(z[e], col + e); sum += own[e]; }
        const u64 upto = wave_scan_u64(sum);
        const u64 all = (u64)__shfl((long long)upto, 63, 64);
        if (target < at + all) {
          u64 to = at + upto - sum;
          if (to <= target && target < to + sum) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
              if (to <= target && target < to + own[e]) sh.found_in = col + e;
              to += own[e];
            }
          }
          break;
        }
        at += all;
      }
    }
    __syncthreads();
    const unsigned r = sh.found_in;
    __syncthreads();
    return r;
  }

  // The border behind the token at which count (or mass) reaches `need`; `in` says which tokens count.  The bins of the row are in place.
  template <class In>
  __device__ __forceinline__ bool border(bool by_mass, u64 need, In in, Border& out) const {
    unsigned b;
    u64 before;
    if (!find(by_mass, need, b, before) || b == LAST) return false;
    need -= before;
    // the keys of the bin
    unsigned lo = 0xffffffffu, hi = 0;
    each([&](const float* z, unsigned col) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (bin(z[e]) == (int)b && in(z[e], col + e)) {
          const unsigned k = R::key(z[e]);
          lo = min(lo, k);
          hi = max(hi, k);
        }
    });
    for (int x = 1; x < 64; x *= 2) {
      lo = min(lo, (unsigned)__shfl_xor((int)lo, x, 64));
      hi = max(hi, (unsigned)__shfl_xor((int)hi, x, 64));
    }
    __syncthreads();
    if (lane == 0) { sh.lo[wave] = lo; sh.hi[wave] = hi; }
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) { lo = min(lo, sh.lo[w]); hi = max(hi, sh.hi[w]); }
    for (;;) {
      const unsigned range = hi - lo, shift = range < BINS ? 0 : 32 - __clz(range) - 11;
      clear_bins();
      each([&](const float* z, unsigned col) {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (bin(z[e]) == (int)b && in(z[e], col + e)) {
            const unsigned k = R::key(z[e]);
            if (k >= lo && k <= hi) {
              const unsigned at = (hi - k) >> shift;
              atomicAdd(&sh.count[at], 1u);
              if (by_mass) atomicAdd(&sh.mass[at], (u64)weight(z[e]));
            }
          }
      });
      unsigned at;
      if (!find(by_mass, need, at, before)) return false;      // (cannot be)
      need -= before;
      const unsigned top = hi - (at << shift);
      if (!shift) {
        out.key = top;
        // `need` of the bin's tokens, which weigh the same
        const unsigned all = sh.count[at];
        const u64 each_one = by_mass ? sh.mass[at] / all : 1, some = (need + each_one - 1) / each_one;
        __syncthreads();
        out.last = 0xffffffffu;
        if (some < all) out.last = locate([&](float z, unsigned col) { return (u64)(R::key(z) == top && in(z, col)); }, some - 1);
        return true;
      }
      hi = top;
      lo = max(lo, top - ((1u << shift) - 1));
    }
  }
};

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void sample_kernel(SampleArgs a) {
  __shared__ SampleShared<THREADS> sh;
  typedef Sampler<T, THREADS> S;
  typedef RowVec<T> R;
  S p(sh);
  const size_t r = blockIdx.x;
  p.row = (const T*)a.logits + r * a.ld;
  p.cols = a.cols;
  p.skip = (unsigned)((uintptr_t)p.row % 16 / sizeof(T));
  p.lane = threadIdx.x & 63;
  p.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned tiles = (p.cols + p.skip + S::TILE - 1) / S::TILE, per = (tiles + S::WAVES - 1) / S::WAVES;
  p.begin = min(p.wave * per, tiles);
  p.end = min(p.begin + per, tiles);
  const karma_sample_rule rule = a.rules[a.n_rules == 1 ? 0 : r];

  // the largest logit, and whether the row has an answer
  float m = -INFINITY;
  bool bad = false;
  p.each([&](const float* z, unsigned) {
#pragma unroll
    for (int e = 0; e < S::N; ++e) {
      m = fmaxf(m, z[e]);
      bad |= !(z[e] < INFINITY);
    }
  });
  m = wave_max(m);
  if (threadIdx.x == 0) sh.bad = 0;
  __syncthreads();
  if (p.lane == 0) sh.top[p.wave] = m;
  if (bad) sh.bad = 1;
  __syncthreads();
  for (int w = 0; w < S::WAVES; ++w) m = fmaxf(m, sh.top[w]);
  bad = sh.bad || m == -INFINITY || !(rule.temperature >= 0.f && rule.temperature < INFINITY) || rule.top_p != rule.top_p || rule.min_p != rule.min_p;
  if (bad) {
    if (threadIdx.x == 0) {
      if (a.token) a.token[r] = -1;
      if (a.logprob) a.logprob[r] = __uint_as_float(0x7fc00000u);
      if (a.kept) a.kept[r] = 0;
    }
    return;
  }
  p.m = m;
  if (rule.temperature == 0.f || rule.top_k == 1 || rule.top_p <= 0.f) {
    const unsigned token = p.locate([&](float z, unsigned) { return (u64)(z == m); }, 0);
    if (threadIdx.x == 0) {
      if (a.token) a.token[r] = (int)token;
      if (a.logprob) a.logprob[r] = 0.f;
      if (a.kept) a.kept[r] = 1;
    }
    return;
  }
  p.c = 1.4426950408889634074 / (double)rule.temperature;
  p.s = fminf((float)LAST / (REACH * rule.temperature), 1e30f);

  Border border{0, 0xffffffffu};
  if (rule.top_k && rule.top_k < a.cols) {
    p.clear_bins();
    p.each([&](const float* z, unsigned) {
#pragma unroll
      for (int e = 0; e < S::N; ++e) {
        const int b = p.bin(z[e]);
        if (b < LAST) atomicAdd(&sh.count[b], 1u);
      }
    });
    // (none where all tokens that weigh anything stay)
    p.border(false, rule.top_k, [&](float, unsigned) { return true; }, border);
  }
  if (rule.top_p < 1.f) {
    p.clear_bins();
    const Border k = border;
    double mine = 0.0;
    p.each([&](const float* z, unsigned col) {
#pragma unroll
      for (int e = 0; e < S::N; ++e) {
        const int b = p.bin(z[e]);
        if (b < LAST && k.stays(R::key(z[e]), col + e)) {
          const double w = p.weight(z[e]);
          mine += w;
          atomicAdd(&sh.mass[b], (u64)w);
        }
      }
    });
    const u64 all = p.block_sum((u64)mine);
    const u64 need = max((u64)ceil((double)rule.top_p * (double)all), (u64)1);
    p.border(true, need, [&](float z, unsigned col) { return k.stays(R::key(z), col); }, border);
    if (border.key == k.key) border.last = min(border.last, k.last);
  }
  const double least = rule.min_p > 0.f ? fmin((double)rule.min_p, 1.0) * ONE : 0.0;
  auto drawn = [&](float z, unsigned col) {
    if (!border.stays(R::key(z), col)) return (u64)0;
    const double w = p.weight(z);
    return w >= least ? (u64)w : 0;
  };
  u64 mine = 0;
  unsigned count = 0;
  p.each([&](const float* z, unsigned col) {
#pragma unroll
    for (int e = 0; e < S::N; ++e) {
      const u64 w = drawn(z[e], col + e);
      mine += w;
      count += w != 0;
    }
  });
  const u64 kept = p.block_sum(count), all = p.block_sum(mine);      // (sh.total holds the wavefronts' shares of `all`)
  const double u = a.uniform[r];
  const u64 target = min((u64)floor((u > 0.0 ? fmin(u, 1.0) : 0.0) * (double)all), all - 1);
  const unsigned token = p.walk(drawn, target);
  if (threadIdx.x == 0) {
    if (a.token) a.token[r] = (int)token;
    if (a.kept) a.kept[r] = (int)kept;
    if (a.logprob) {
      const float z = R::one(p.row + token);
      a.logprob[r] = (float)(((double)z - (double)m) / (double)rule.temperature - log((double)all / ONE));
    }
  }
}

bool aligned_to(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

}  // namespace

size_t sample_ws_bytes(uint32_t, uint32_t) { return 0; }

int sample_rows(SampleArgs a, bool bf16, hipStream_t s) {
  if (!a.ld) a.ld = a.cols;
  if (!a.cols || a.cols > KARMA_SAMPLE_COLS_MAX || a.rows >= SP_GRID || a.ld < a.cols || a.ld > INT64_MAX / 8 / ((uint64_t)a.rows + 1)) return KARMA_E_INVAL;
  if (a.n_rules != 1 && a.n_rules != a.rows) return KARMA_E_INVAL;
  if (!a.token && !a.logprob && !a.kept) return KARMA_E_INVAL;
  for (const void* p : {(const void*)a.rules, (const void*)a.uniform, (const void*)a.token, (const void*)a.logprob, (const void*)a.kept})
    if (!aligned_to(p, 4)) return KARMA_E_INVAL;
  if (!a.rows) return KARMA_OK;
  if (!a.logits || !a.rules || !a.uniform || !aligned_to(a.logits, bf16 ? 2 : 4)) return KARMA_E_INVAL;
  if (bf16) hipLaunchKernelGGL((sample_kernel<bf16_t, 1024>), dim3(a.rows), dim3(1024), 0, s, a);
  else hipLaunchKernelGGL((sample_kernel<float, 1024>), dim3(a.rows), dim3(1024), 0, s, a);
  return hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

}  // namespace karma

using namespace karma;

extern "C" uint64_t karma_k_sample_ws_bytes(uint32_t rows, uint32_t cols) { return sample_ws_bytes(rows, cols); }

#define KARMA_SAMPLE_ENTRY(SUFFIX, T, BF16)                                                                                                  \
  extern "C" int karma_k_sample_##SUFFIX(const T* logits, uint64_t ld, const karma_sample_rule* rules, uint32_t n_rules, const float* uniform, \
                                         int32_t* token, float* logprob, int32_t* kept, uint32_t rows, uint32_t cols, void* ws,              \
                                         uint64_t ws_bytes, void* stream) {                                                                  \
    return sample_rows(SampleArgs{logits, ld, rules, n_rules, uniform, token, logprob, kept, rows, cols, ws, ws ? ws_bytes : 0}, BF16,       \
                       (hipStream_t)stream);                                                                                                 \
  }
KARMA_SAMPLE_ENTRY(bf16, void, true)
KARMA_SAMPLE_ENTRY(f32, float, false)
