// Log probabilities of given tokens under rows of logits, the rows' entropies and best alternatives, and the gradient.
// With c the scale, m the row's largest logit, s = sum_j e^(c (z_j - m)) and q_j = c (z_j - m) - ln s (the log probability):
//   logprob = q_token,  entropy = ln s - c sum_j (z_j - m) e^(c (z_j - m)) / s,
//   dz_j = c (dlogprob (delta_j - p_j) - dentropy p_j (q_j + entropy)),  p_j = e^q_j.
// Logits are compared and subtracted before they are scaled: a row that holds its type's lowest value everywhere is then as
// good as any other, where c z would overflow.  All sums are fp32.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_utils.h"
#include "karma.h"
#include "kernels.h"

namespace karma {
namespace {

// ---- rows in 16-byte vectors --------------------------------------------------------------------------------
template <typename T>
struct Vec;
template <>
struct Vec<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void store(bf16_t* p, const float* f) { *(u32x4*)p = pack8(f); }
  static __device__ __forceinline__ float one(const bf16_t* p) { return bf2f(*p); }
  static __device__ __forceinline__ void put(bf16_t* p, float v) { *p = f2bf(v); }
  static __device__ __forceinline__ void unpack(const u32x4& v, float* f) { unpack8(v, f); }
};
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void store(float* p, const float* f) {
    *(u32x4*)p = u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
  static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
  static __device__ __forceinline__ void unpack(const u32x4& v, float* f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(v[e]);
  }
};
// Rows may begin anywhere (a vocabulary of odd size): `head` elements before the first 16-byte boundary and `tail` behind the
// last are taken one by one.
template <typename T>
struct Row {
  const T* at;
  unsigned head, vectors, tail;
  __device__ __forceinline__ Row(const T* z, unsigned cols) : at(z) {
    head = min((unsigned)((16 - (uintptr_t)z % 16) % 16 / sizeof(T)), cols);
    vectors = (cols - head) / Vec<T>::N;
    tail = cols - head - vectors * Vec<T>::N;
  }
};

// ---- maximum, sum and first moment of what has been seen --------------------------------------------------------
// m: the largest; s = sum of 2^(c2 (z - m)), t = sum of (z - m) 2^(c2 (z - m)).  Nothing seen: m the lowest finite value and s = 0,
// which no logit that is allowed leaves (the largest adds 1).  NaN comes through the exponential into s.
struct Running { float m, s, t; };
__device__ __forceinline__ Running nothing_seen() { return Running{-3.402823466e38f, 0.f, 0.f}; }
__device__ __forceinline__ void raise(Running& r, float m, float c2) {
  const float d = fmaxf(r.m - m, -1e30f), k = __builtin_amdgcn_exp2f(d * c2);   // (bounded: -inf times an s of 0)
  r.t = (r.t + d * r.s) * k;
  r.s *= k;
  r.m = m;
}
template <int N>
__device__ __forceinline__ float max_of(const float (&f)[N]) {
  float m = f[0];
#pragma unroll
  for (int e = 1; e < N; ++e) m = fmaxf(m, f[e]);
  return m;
}
template <int N>
__device__ __forceinline__ void take(Running& r, const float (&f)[N], float most, float c2) {
  if (most > r.m) raise(r, most, c2);
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float d = f[e] - r.m, x = __builtin_amdgcn_exp2f(d * c2);
    r.s += x;
    r.t = fmaf(x, fmaxf(d, -1e30f), r.t);   // (bounded: -inf times a probability of 0)
  }
}
__device__ __forceinline__ Running join(Running a, Running b, float c2) {
  const float m = fmaxf(a.m, b.m);
  raise(a, m, c2);
  raise(b, m, c2);
  return Running{m, a.s + b.s, a.t + b.t};
}
// The wavefront's: every lane's sums to the largest maximum at once, then added.
__device__ __forceinline__ Running wave_join(Running r, float c2) {
  raise(r, wave_max(r.m), c2);
  return Running{r.m, wave_sum(r.s), wave_sum(r.t)};
}

// ---- the best alternatives -------------------------------------------------------------------------------------
// Elements are kept as 64-bit keys: the value's bits in an order of whole numbers, then the inverted index, so that equal values are
// in ascending order; all keys differ.  0: none.  A wavefront collects in LDS, without order, what is not below its floor; most
// vectors fall to one comparison of their largest element.  When its room is full, wave_select throws out what is not among the best.
__device__ __forceinline__ uint64_t order_key(float v, unsigned i) {
  unsigned u = __float_as_uint(v);
  if (u == 0x80000000u) u = 0;      // -0 equals 0
  u = u & 0x80000000u ? ~u : u | 0x80000000u;
  return (uint64_t)u << 32 | (0xffffffffu - i);
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const unsigned u = (unsigned)(k >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_index(uint64_t k) { return (int)(0xffffffffu - (unsigned)k); }
constexpr int LP_THREADS = 256, LP_WAVES = LP_THREADS / 64;
constexpr int LP_KEEP = 128, LP_ROOM = LP_KEEP + 64;    // keys that wave_select may leave, and keys of a wavefront

// What a wavefront writes to LDS its other lanes read: in order within the wavefront, so the compiler alone has to be told.
__device__ __forceinline__ void wave_lds_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }
__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0));
}

// The largest number of 16 bits (and 16 zeros) that at least `top` of the wavefront's numbers reach: counted bit by bit.
template <int M>
__device__ __forceinline__ unsigned reached_by(const unsigned (&u)[M], int top) {
  unsigned at = 0;
#pragma unroll
  for (unsigned bit = 0x80000000u; bit >= 0x10000u; bit >>= 1) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) n += __popcll(__ballot(u[i] >= (at | bit)));
    if (n >= top) at |= bit;
  }
  return at;
}
// The places of keys among n keys in LDS: how many of those are larger.  (A comparison of 64 bits takes four times as long as one of
// 32: for few keys only.)
template <int M>
__device__ __forceinline__ void places(const uint64_t* keys, int n, const uint64_t (&k)[M], int (&place)[M]) {
#pragma unroll
  for (int i = 0; i < M; ++i) place[i] = 0;
  for (int j = 0; j < n; ++j) {
    const uint64_t o = keys[j];
#pragma unroll
    for (int i = 0; i < M; ++i) place[i] += o > k[i];
  }
}
// Places of keys that lie one a lane, among the n lanes that have one: from their registers, without a trip to LDS a key.
__device__ __forceinline__ int places_of_lanes(uint64_t k, int n) {
  int place = 0;
  for (int j = 0; j < n; ++j) {
    const uint64_t o = (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(k >> 32), j) << 32 | (unsigned)__builtin_amdgcn_readlane((int)k, j);
    place += o > k;
  }
  return place;
}
// One wavefront, n keys in its registers (key i of lane l being number 64 i + l): leaves the best of them in LDS from `keys` on and returns
// how many, at most LP_KEEP; with sorted, `top` of them (or all) in order.  least: a key that those that are not among the best do not
// reach.
template <int M>
__device__ __forceinline__ int wave_select(const uint64_t (&k)[M], int n, uint64_t* keys, int top, bool sorted, uint64_t& least) {
  const int lane = threadIdx.x & 63;
  wave_lds_fence();     // the keys may come from where the best go
  unsigned u[M];
#pragma unroll
  for (int i = 0; i < M; ++i) u[i] = (unsigned)(k[i] >> 32);
  if (sorted && n <= 32) {      // (counting first takes as long as 30 places do)
    const int place = places_of_lanes(k[0], n);
    if (k[0] && place < top) keys[place] = k[0];
    wave_lds_fence();
    return min(n, top);
  }
  const unsigned at = n > top ? reached_by<M>(u, top) : 1u;     // (1: all but the empty ones)
  least = n > top ? (uint64_t)at << 32 : 0;
  int left = 0;
#pragma unroll
  for (int i = 0; i < M; ++i) left += __popcll(__ballot(u[i] >= at));
  if (left > LP_KEEP) {     // too many alike in 16 bits: all places
#pragma unroll
    for (int i = 0; i < M; ++i) keys[i * 64 + lane] = k[i];
    wave_lds_fence();
    int place[M];
    places<M>(keys, n, k, place);
    wave_lds_fence();
#pragma unroll
    for (int i = 0; i < M; ++i)
      if (k[i] && place[i] < top) keys[place[i]] = k[i];
    wave_lds_fence();
    least = keys[top - 1];
    return top;
  }
  left = 0;
#pragma unroll
  for (int i = 0; i < M; ++i) {
    const uint64_t mask = __ballot(u[i] >= at);
    if (u[i] >= at) keys[left + lanes_below(mask)] = k[i];
    left += __popcll(mask);
  }
  wave_lds_fence();
  if (!sorted) return left;
  uint64_t f[2];
  int place[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) f[i] = lane + i * 64 < left ? keys[lane + i * 64] : 0;
  if (left > 64) {
    places<2>(keys, left, f, place);
  } else {
    place[0] = places_of_lanes(f[0], left);
    place[1] = top;
  }
  wave_lds_fence();
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (f[i] && place[i] < top) keys[place[i]] = f[i];
  wave_lds_fence();
  return min(left, top);
}
// the same for keys that lie one behind the other in LDS, from `keys` on
template <int M>
__device__ __forceinline__ int wave_select_lds(uint64_t* keys, int n, int top, bool sorted, uint64_t& least) {
  const int lane = threadIdx.x & 63;
  wave_lds_fence();
  uint64_t k[M];
#pragma unroll
  for (int i = 0; i < M; ++i) k[i] = lane + i * 64 < n ? keys[lane + i * 64] : 0;
  return wave_select<M>(k, n, keys, top, sorted, least);
}

struct Best {
  uint64_t* keys;     // LP_ROOM of LDS
  int count, top;     // the same in all lanes, as the following
  float floor;        // values below it are not among the best,
  unsigned before;    // nor are those equal to it from this column on
  __device__ __forceinline__ Best(uint64_t* keys_, int top_) : keys(keys_), count(0), top(top_), floor(-INFINITY), before(0xffffffffu) {}
  __device__ __forceinline__ void settle() {
    uint64_t least;
    count = wave_select_lds<LP_ROOM / 64>(keys, count, top, false, least);
    if (!least) return;
    const float v = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(key_value(least))));
    // (a floor by 16 bits alone has low bits of 0, as no column has; it may lie among the patterns below -inf, of NaN)
    const unsigned low = __builtin_amdgcn_readfirstlane((unsigned)least);
    if (v > floor || (v == floor && low)) {
      floor = v;
      before = low ? 0xffffffffu - low : 0xffffffffu;
    }
  }
  // the elements of a vector, the e-th of a lane being column base + e
  template <int N>
  __device__ __forceinline__ void look(const float (&f)[N], float most, unsigned base) {
    if (!__ballot(most >= floor)) return;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (!__ballot(f[e] >= floor)) continue;       // NaN is none
      bool in = f[e] > floor || (f[e] == floor && base + e < before);
      uint64_t mask = __ballot(in);
      if (count + __popcll(mask) > LP_ROOM) {
        settle();
        in = f[e] > floor || (f[e] == floor && base + e < before);
        mask = __ballot(in);
      }
      if (in) keys[count + lanes_below(mask)] = order_key(f[e], base + e);
      count += __popcll(mask);
    }
  }
  // The largest element that each lane has seen: 64 different ones, so `n` elements reach the n-th largest of them.
  static __device__ __forceinline__ float reached(float seen, int n) {
    const unsigned b = __float_as_uint(seen), u[1] = {b & 0x80000000u ? ~b : b | 0x80000000u};
    const unsigned at = reached_by<1>(u, n);
    const float v = __uint_as_float(at & 0x80000000u ? at & 0x7fffffffu : ~at);
    return v == v ? v : -INFINITY;     // (as above)
  }
  __device__ __forceinline__ void raise_to(float v) {
    if (v > floor) { floor = v; before = 0xffffffffu; }
  }
};

// ---- forward -------------------------------------------------------------------------------------------------
constexpr uint32_t LP_PLACES = 7 * 256;   // workgroups that run at once
constexpr int LP_BATCH = 4;     // vectors that a lane has under way

struct LogprobPart { float m, s, t, unused; };

// The token's logit, asked for at the beginning of a row: two trips to memory one after the other.
struct Named { bool any; float z; };
template <typename T>
__device__ __forceinline__ Named named_logit(const LogprobFwd& a, size_t r) {
  const int t = a.logprob ? a.tokens[r] : -1;
  const bool any = t >= 0 && (unsigned)t < a.cols;
  return Named{any, any ? Vec<T>::one((const T*)a.logits + r * a.ld + t) : 0.f};
}

__device__ __forceinline__ void finish_row(const LogprobFwd& a, size_t r, Running w, uint64_t key, const Named& named) {
  const int lane = threadIdx.x & 63;
  const bool empty = w.s == 0.f;
  if (empty) { w.m = -INFINITY; w.s = 1.f; w.t = 0.f; }
  const float ls = logf(w.s);
  auto log_p = [&](float v) { return empty ? -INFINITY : (v - w.m) * a.scale - ls; };
  if (lane == 0) {
    if (a.stats) { a.stats[2 * r] = w.m; a.stats[2 * r + 1] = ls; }
    if (a.entropy) a.entropy[r] = ls - a.scale * w.t / w.s;
    if (a.logprob) a.logprob[r] = named.any ? log_p(named.z) : 0.f;
  }
  if (lane < (int)a.top) {
    a.top_id[r * a.top + lane] = key ? key_index(key) : -1;
    a.top_logprob[r * a.top + lane] = key ? log_p(key_value(key)) : NAN;
  }
}

// W wavefronts share a part of a row (`parts` parts a row, W = 1: the whole row), lanes side by side on vectors.  One pass: every
// vector goes into the running sums and past the list of alternatives.  Bound by memory: 4096 x 32000 in bf16 55 us a call, 4.7
// TB/s (eight vectors under way instead of four: 62); with 5 alternatives 63, with 20 68, with 64 85, which is the work on keys (inserting
// them one by one into a list in registers took 72, 94 and 127; comparing all candidates with each other 87 with 5).
template <typename T, int W, bool TOP>
__global__ __launch_bounds__(LP_THREADS) void logprob_fwd_kernel(LogprobFwd a, unsigned parts, LogprobPart* sums, uint64_t* lists) {
  constexpr int N = Vec<T>::N;
  __shared__ Running wave_sums[LP_WAVES];
  __shared__ uint64_t keys[TOP ? LP_WAVES * LP_ROOM : 1];
  __shared__ int counts[LP_WAVES];
  __shared__ float floors[LP_WAVES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned unit = blockIdx.x * (LP_WAVES / W) + wave / W;    // a row's part
  const unsigned r = unit / parts, part = unit % parts, w = wave % W;
  const float c2 = a.scale * 1.44269504f;
  Running run = nothing_seen();
  Best best(keys + (TOP ? wave * LP_ROOM : 0), (int)a.top);
  Named named{false, 0.f};
  if (r < a.rows) {
    if (parts == 1 && w == 0) named = named_logit<T>(a, r);
    const Row<T> row((const T*)a.logits + (size_t)r * a.ld, a.cols);
    // (parts are as even as they can be: each of those that share a row has a vector for every lane)
    const unsigned per = row.vectors / parts, rest = row.vectors % parts, v0 = part * per + min(part, rest), v1 = v0 + per + (part < rest);
    const T* body = row.at + row.head;
    bool first = true;
    float seen = -INFINITY;
    for (unsigned v = v0 + w * 64; v < v1; v += LP_BATCH * W * 64) {
      u32x4 raw[LP_BATCH];
      float f[N], most[LP_BATCH];
#pragma unroll
      for (int k = 0; k < LP_BATCH; ++k) {
        const unsigned i = v + k * W * 64 + lane;
        if (i < v1) raw[k] = *(const u32x4*)(body + (size_t)i * N);
      }
#pragma unroll
      for (int k = 0; k < LP_BATCH; ++k) {
        most[k] = -INFINITY;
        if (v + k * W * 64 + lane < v1) {
          Vec<T>::unpack(raw[k], f);
          most[k] = max_of(f);
          take(run, f, most[k], c2);
        }
      }
      if (TOP) {
        // Wavefronts that share a row have a share of the best each: all of those reach the smallest of their floors.  After the first
        // batch nobody waits: an older floor of another costs time alone.
#pragma unroll
        for (int k = 0; k < LP_BATCH; ++k) seen = fmaxf(seen, most[k]);
        float reach = Best::reached(seen, ((int)a.top + W - 1) / W);
        if (W > 1) {
          volatile float* theirs = floors;
          theirs[wave] = reach;
          if (first) __syncthreads();
          for (int k = 0; k < W; ++k) reach = fminf(reach, theirs[k]);
          reach = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(reach)));
        }
        first = false;
        best.raise_to(reach);
#pragma unroll
        for (int k = 0; k < LP_BATCH; ++k) {
          const unsigned i = v + k * W * 64 + lane;
          if (i < v1) Vec<T>::unpack(raw[k], f);
          else
#pragma unroll
            for (int e = 0; e < N; ++e) f[e] = NAN;
          best.look(f, most[k], row.head + i * N);
        }
      }
    }
    // what lies before the first boundary and behind the last, with the first and the last part
    if (w == 0) {
      const unsigned ends = (part == 0 ? row.head : 0) + (part == parts - 1 ? row.tail : 0);
      if (ends) {
        const unsigned i = part == 0 && (unsigned)lane < row.head ? lane : a.cols - row.tail + (lane - (part == 0 ? row.head : 0));
        float f[1] = {NAN};
        if ((unsigned)lane < ends) {
          f[0] = Vec<T>::one(row.at + i);
          take(run, f, f[0], c2);
        }
        if (TOP) best.look(f, f[0], i);
      }
    }
  }
  run = wave_join(run, c2);
  uint64_t key = 0, least;
  if (W > 1) {
    if (TOP && best.count > LP_KEEP) best.settle();
    if (lane == 0) { wave_sums[wave] = run; counts[wave] = best.count; }
    __syncthreads();
    if (w) return;      // the first wavefront has the rest
#pragma unroll
    for (int k = 1; k < W; ++k) run = join(run, wave_sums[wave + k], c2);
    if (TOP) {
      // number i of all keys, the wavefronts' one behind the other
      int ends[W];
      ends[0] = best.count;
#pragma unroll
      for (int k = 1; k < W; ++k) ends[k] = ends[k - 1] + counts[wave + k];
      auto gather = [&](int i) {
        int at = i;
#pragma unroll
        for (int k = 1; k < W; ++k) at = i >= ends[k - 1] ? k * LP_ROOM + i - ends[k - 1] : at;
        return i < ends[W - 1] ? best.keys[at] : 0;
      };
      int n = ends[W - 1];
      if (n <= 128) {
        uint64_t k[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) k[i] = gather(lane + i * 64);
        n = wave_select<2>(k, n, best.keys, a.top, true, least);
      } else {
        uint64_t k[W * LP_KEEP / 64];
#pragma unroll
        for (int i = 0; i < W * LP_KEEP / 64; ++i) k[i] = gather(lane + i * 64);
        n = wave_select<W * LP_KEEP / 64>(k, n, best.keys, a.top, true, least);
      }
      if (lane < n) key = best.keys[lane];
    }
  } else if (TOP) {
    const int n = wave_select_lds<LP_ROOM / 64>(best.keys, best.count, a.top, true, least);
    if (lane < n) key = best.keys[lane];
  }
  if (r >= a.rows) return;
  if (parts == 1) { finish_row(a, r, run, key, named); return; }
  if (lane == 0) sums[unit] = LogprobPart{run.m, run.s, run.t, 0.f};
  if (TOP && lane < (int)a.top) lists[(size_t)unit * a.top + lane] = key;
}

// A workgroup joins a row's parts.  Of their lists only what reaches the largest of the lists' last keys can be among the best; where
// there is more than the room, it is settled in between.
template <typename T>
__global__ __launch_bounds__(LP_THREADS) void logprob_join_kernel(LogprobFwd a, unsigned parts, const LogprobPart* sums, const uint64_t* lists) {
  __shared__ uint64_t keys[2 * LP_THREADS];
  __shared__ int count;
  const int lane = threadIdx.x & 63, tid = threadIdx.x;
  const size_t r = blockIdx.x;
  const float c2 = a.scale * 1.44269504f;
  uint64_t key = 0, least;
  Running run = nothing_seen();
  const Named named = named_logit<T>(a, r);
  if (a.top) {
    const uint64_t* mine = lists + r * parts * a.top;
    const unsigned n = parts * a.top;
    uint64_t next = tid < (int)n ? mine[tid] : 0;
    // every wavefront finds the floor for itself
    uint64_t floor = 0;
    for (unsigned k = lane; k < parts; k += 64) floor = max(floor, mine[k * a.top + a.top - 1]);
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) floor = max(floor, (uint64_t)__shfl_xor((unsigned long long)floor, k));
    if (tid == 0) count = 0;
    for (unsigned v = 0; v < n; v += LP_THREADS) {
      const uint64_t k = next;
      const bool last = v + LP_THREADS >= n;
      next = v + LP_THREADS + tid < n ? mine[v + LP_THREADS + tid] : 0;
      __syncthreads();
      if (k && k >= floor) keys[atomicAdd(&count, 1)] = k;      // in any order: what is chosen does not depend on it
      __syncthreads();
      const int have = count;
      if (have <= LP_THREADS && !last) continue;
      if (tid < 64) {
        const int left = have <= 128 ? wave_select_lds<2>(keys, have, a.top, last, least) : wave_select_lds<2 * LP_THREADS / 64>(keys, have, a.top, last, least);
        if (lane == 0) count = left;
        if (last && lane < left) key = keys[lane];
      }
    }
  }
  if (tid < 64)
    for (unsigned k = lane; k < parts; k += 64) {
      const LogprobPart p = sums[r * parts + k];
      run = join(run, Running{p.m, p.s, p.t}, c2);
    }
  if (tid >= 64) return;
  run = wave_join(run, c2);
  finish_row(a, r, run, key, named);
}

// ---- backward ------------------------------------------------------------------------------------------------
// A wavefront has LP_BATCH vectors of each lane of one row; `units` wavefronts a row.  Bound by memory: 4096 x 51200 in bf16 144 us
// a call, 5.8 TB/s.
template <typename T>
__global__ __launch_bounds__(LP_THREADS) void logprob_bwd_kernel(LogprobBwd a, unsigned units) {
  constexpr int N = Vec<T>::N, SPAN = 64 * LP_BATCH;
  const int lane = threadIdx.x & 63;
  const unsigned unit = blockIdx.x * LP_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = unit % units;
  const size_t r = unit / units;
  if (r >= a.rows) return;
  const Row<T> row((const T*)a.logits + r * a.ld, a.cols);
  T* d = (T*)a.dlogits + r * a.ld_d;
  const float m = a.stats[2 * r], ls = a.stats[2 * r + 1];
  const int token = a.tokens ? a.tokens[r] : -1;
  const float dl = a.dlogprob && token >= 0 && (unsigned)token < a.cols ? a.dlogprob[r] * a.scale : 0.f;
  const float de = a.dentropy ? a.dentropy[r] * a.scale : 0.f, ent = a.dentropy ? a.entropy[r] : 0.f;
  const bool empty = m == -INFINITY && ls == 0.f;
  const float c2 = a.scale * 1.44269504f, ls2 = ls * 1.44269504f;
  auto grad = [&](float z, unsigned j) {
    const float q2 = fmaf(z - m, c2, -ls2), p = __builtin_amdgcn_exp2f(q2);
    // p = 0: nothing, whatever it is multiplied with (q2 of -inf or -1e20, a de that has overflowed).  NaN is not 0.  Elsewhere q2 is above
    // -150, and p comes before de: the product of the two is of the order of one.
    float v = p == 0.f ? 0.f : -p * dl - p * fmaf(q2, 0.693147181f, ent) * de;
    if ((int)j == token) v += dl;
    return empty ? 0.f : v;
  };
  const bool same = ((uintptr_t)row.at - (uintptr_t)d) % 16 == 0;      // both come in vectors at the same places
  const T* zb = row.at + row.head;
  T* db = d + row.head;
  const unsigned v0 = part * SPAN;
  u32x4 raw[LP_BATCH];
#pragma unroll
  for (int k = 0; k < LP_BATCH; ++k) {
    const unsigned i = v0 + k * 64 + lane;
    if (i < row.vectors) raw[k] = *(const u32x4*)(zb + (size_t)i * N);
  }
#pragma unroll
  for (int k = 0; k < LP_BATCH; ++k) {
    const unsigned i = v0 + k * 64 + lane;
    if (i >= row.vectors) break;
    float f[N];
    Vec<T>::unpack(raw[k], f);
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = grad(f[e], row.head + i * N + e);
    if (same) Vec<T>::store(db + (size_t)i * N, f);
    else
#pragma unroll
      for (int e = 0; e < N; ++e) Vec<T>::put(db + (size_t)i * N + e, f[e]);
  }
  if (part == 0) {
    const unsigned ends = row.head + row.tail;
    if ((unsigned)lane < ends) {
      const unsigned j = (unsigned)lane < row.head ? lane : a.cols - ends + lane;
      Vec<T>::put(d + j, grad(Vec<T>::one(row.at + j), j));
    }
  }
}

// Wavefronts for a row: one where four would not have a vector for every lane, and for rows of up to 512 vectors where there are many
// (16000 x 4000 in bf16: 29.5 us instead of 33.0, with 5 alternatives 41 instead of 57; 4097 x 8000: 25.7 and 25.0).  Parts of a row: as
// many as there is room for at once (seven workgroups on each of 256 compute units), none smaller than two vectors a lane, and none
// of rows that four vectors a lane hold twice: their join takes longer than it saves (with 20 alternatives, 1 x 5028 in one part / in
// parts of one vector a lane 7.2 / 11.0 us in the kernels, 8 x 16000 11.4 / 12.2; in parts of two / of one 1 x 160000 16.9 / 20.5, 64 x 51200
// 15.8 / 18.0, 8 x 51200 14.6 / 13.6).
struct LogprobCut { unsigned waves, parts; };
LogprobCut cut_rows(uint32_t rows, uint32_t cols, bool bf16) {
  const uint32_t vectors = cols / (bf16 ? 8 : 4);
  const uint32_t parts = vectors < 2 * LP_BATCH * LP_THREADS ? 1 : std::min(LP_PLACES / std::max(rows, 1u), vectors / (2 * LP_THREADS));
  if (parts <= 1) return LogprobCut{vectors <= (rows >= 4096 ? 512u : (unsigned)LP_THREADS) ? 1u : (unsigned)LP_WAVES, 1};
  return LogprobCut{(unsigned)LP_WAVES, parts};
}
constexpr uint32_t LP_GRID = (1u << 24) - 1;        // workgroups of 256 lanes in a launch, which has less than 2^32
size_t up16(size_t b) { return (b + 15) / 16 * 16; }

bool aligned_to(const void* p, size_t n) { return (uintptr_t)p % n == 0; }
bool good_rows(uint32_t rows, uint32_t cols, uint64_t ld) {
  return cols && cols <= INT32_MAX && rows <= LP_GRID && ld >= cols && ld <= INT64_MAX / 8 / ((uint64_t)rows + 1);
}

}  // namespace

// (the larger of the two types': fp32 rows have twice the vectors)
size_t token_logprob_ws_bytes(uint32_t rows, uint32_t cols, uint32_t top) {
  const uint64_t parts = cut_rows(rows, cols, false).parts;
  return parts > 1 ? up16(rows * parts * sizeof(LogprobPart)) + rows * parts * top * sizeof(uint64_t) : 0;
}

int token_logprob_fwd(LogprobFwd a, bool bf16, hipStream_t s) {
  if (!a.ld) a.ld = a.cols;
  if (!good_rows(a.rows, a.cols, a.ld) || !(a.scale >= 1e-20f && a.scale <= 1e20f)) return KARMA_E_INVAL;
  if (a.top > KARMA_TOP_MAX || a.top > a.cols || (a.top && (!a.top_logprob || !a.top_id))) return KARMA_E_INVAL;
  if ((a.logprob && !a.tokens) || (!a.logprob && !a.entropy && !a.stats && !a.top)) return KARMA_E_INVAL;
  for (const void* p : {(const void*)a.tokens, (const void*)a.logprob, (const void*)a.entropy, (const void*)a.stats, (const void*)a.top_logprob, (const void*)a.top_id})
    if (!aligned_to(p, 4)) return KARMA_E_INVAL;
  if (!a.rows) return KARMA_OK;
  if (!a.logits || !aligned_to(a.logits, bf16 ? 2 : 4)) return KARMA_E_INVAL;
  if (a.ws_bytes < token_logprob_ws_bytes(a.rows, a.cols, a.top)) return KARMA_E_OOM;
  if (!aligned_to(a.ws, 16)) return KARMA_E_INVAL;
  const LogprobCut cut = cut_rows(a.rows, a.cols, bf16);
  LogprobPart* sums = (LogprobPart*)a.ws;
  uint64_t* lists = (uint64_t*)((char*)a.ws + up16((size_t)a.rows * cut.parts * sizeof(LogprobPart)));
  const unsigned grid = (unsigned)(((uint64_t)a.rows * cut.parts + LP_WAVES / cut.waves - 1) / (LP_WAVES / cut.waves));
#define KARMA_LOGPROB_LAUNCH(T, W, TOP) hipLaunchKernelGGL((logprob_fwd_kernel<T, W, TOP>), dim3(grid), dim3(LP_THREADS), 0, s, a, cut.parts, sums, lists)
  if (bf16) {
    if (cut.waves == 1) { if (a.top) KARMA_LOGPROB_LAUNCH(bf16_t, 1, true); else KARMA_LOGPROB_LAUNCH(bf16_t, 1, false); }
    else { if (a.top) KARMA_LOGPROB_LAUNCH(bf16_t, LP_WAVES, true); else KARMA_LOGPROB_LAUNCH(bf16_t, LP_WAVES, false); }
    if (cut.parts > 1) hipLaunchKernelGGL(logprob_join_kernel<bf16_t>, dim3(a.rows), dim3(LP_THREADS), 0, s, a, cut.parts, sums, lists);
  } else {
    if (cut.waves == 1) { if (a.top) KARMA_LOGPROB_LAUNCH(float, 1, true); else KARMA_LOGPROB_LAUNCH(float, 1, false); }
    else { if (a.top) KARMA_LOGPROB_LAUNCH(float, LP_WAVES, true); else KARMA_LOGPROB_LAUNCH(float, LP_WAVES, false); }
    if (cut.parts > 1) hipLaunchKernelGGL(logprob_join_kernel<float>, dim3(a.rows), dim3(LP_THREADS), 0, s, a, cut.parts, sums, lists);
  }
#undef KARMA_LOGPROB_LAUNCH
  return hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

int token_logprob_bwd(LogprobBwd a, bool bf16, hipStream_t s) {
  if (!a.ld) a.ld = a.cols;
  if (!a.ld_d) a.ld_d = a.cols;
  if (!good_rows(a.rows, a.cols, a.ld) || !good_rows(a.rows, a.cols, a.ld_d) || !(a.scale >= 1e-20f && a.scale <= 1e20f)) return KARMA_E_INVAL;
  if ((a.dlogprob && !a.tokens) || (a.dentropy && !a.entropy) || (!a.dlogprob && !a.dentropy)) return KARMA_E_INVAL;
  for (const void* p : {(const void*)a.tokens, (const void*)a.stats, (const void*)a.entropy, (const void*)a.dlogprob, (const void*)a.dentropy})
    if (!aligned_to(p, 4)) return KARMA_E_INVAL;
  if (!a.rows) return KARMA_OK;
  if (!a.logits || !a.stats || !a.dlogits || !aligned_to(a.logits, bf16 ? 2 : 4) || !aligned_to(a.dlogits, bf16 ? 2 : 4)) return KARMA_E_INVAL;
  const unsigned vectors = a.cols / (bf16 ? 8 : 4), units = std::max(1u, (vectors + 64 * LP_BATCH - 1) / (64 * LP_BATCH));
  if ((uint64_t)a.rows * units > (uint64_t)LP_GRID * LP_WAVES) return KARMA_E_INVAL;
  const unsigned grid = (a.rows * units + LP_WAVES - 1) / LP_WAVES;
  if (bf16) hipLaunchKernelGGL(logprob_bwd_kernel<bf16_t>, dim3(grid), dim3(LP_THREADS), 0, s, a, units);
  else hipLaunchKernelGGL(logprob_bwd_kernel<float>, dim3(grid), dim3(LP_THREADS), 0, s, a, units);
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
