// Draws a token from every row of logits: temperature, top-k, top-p, min-p, one uniform number a row.
// With m the row's largest logit, token j weighs w_j = rint(2^40 e^((z_j - m) / T)).  Whole numbers: their sums are exact and the
// same in whatever order lanes, wavefronts and passes take them, so which token stays and which is drawn hangs on no order.
// Tokens are ordered by falling logit, equal ones by rising index; what top-k, top-p and min-p leave is a beginning of that order: all tokens
// above a logit, the border, and the first `ties` of those that equal it.  The border is found by counting and weighing the row, without sorting,
// and the draw by sums over runs of columns: of the wavefronts, of tiles, of lanes.
// A workgroup has a row and goes over it a few times: the first time from memory, then from the L2 where the rows under way fit it (4096 x 32000 in
// bf16, three rows of 64 KB on a compute unit, reads 464 MB for 250 MB of logits; 301 x 50021 in fp32 117 MB for 57).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_utils.h"
#include "karma.h"
#include "kernels.h"

namespace karma {
namespace {

typedef unsigned long long u64;
constexpr unsigned SP_GRID = 1u << 20;
static_assert(KARMA_SAMPLE_COLS_MAX < 1u << 23, "a row's weights of up to 2^40 add up to less than 2^63");
constexpr int BINS = 2048, LAST = BINS - 1;
constexpr double ONE = 1099511627776.0;     // 2^40
// bins reach down to weights of 2^-42 of the largest: what falls into the last one weighs nothing
constexpr float REACH = 42.f * 0.69314718f;
// (a small temperature divides into infinity; a large one leaves more than 2e-37)
__device__ __forceinline__ float bins_per_logit(float temperature) { return fminf((float)LAST / REACH / temperature, 1e30f); }

// A row in 16-byte vectors on 16-byte boundaries: vector v has the columns v N - skip .. + N.
template <typename T>
struct RowVec;
template <>
struct RowVec<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const u32x4& v, float* f) { unpack8(v, f); }
  static __device__ __forceinline__ float nth(const u32x4& v, int e) {
    const unsigned d = e & 4 ? (e & 2 ? v[3] : v[2]) : e & 2 ? v[1] : v[0];
    return __uint_as_float(e & 1 ? d & 0xffff0000u : d << 16);
  }
  static __device__ __forceinline__ u32x4 nothing() { return u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}; }
  static __device__ __forceinline__ void put(u32x4& v, unsigned at, bf16_t x) {
#pragma unroll
    for (unsigned i = 0; i < 4; ++i) v[i] = at / 2 != i ? v[i] : at % 2 ? (v[i] & 0xffff) | (unsigned)x << 16 : (v[i] & 0xffff0000u) | x;
  }
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
  static __device__ __forceinline__ float nth(const u32x4& v, int e) { return __uint_as_float(e & 2 ? (e & 1 ? v[3] : v[2]) : e & 1 ? v[1] : v[0]); }
  static __device__ __forceinline__ u32x4 nothing() { return u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u}; }
  static __device__ __forceinline__ void put(u32x4& v, unsigned at, float x) {
#pragma unroll
    for (unsigned i = 0; i < 4; ++i) v[i] = at == i ? __float_as_uint(x) : v[i];
  }
  static __device__ __forceinline__ unsigned key(float z) {
    const unsigned u = __float_as_uint(z + 0.f);
    return (int)u < 0 ? ~u : u | 0x80000000u;
  }
  static __device__ __forceinline__ float value(unsigned key) { return __uint_as_float((int)key < 0 ? key & 0x7fffffffu : ~key); }
};

// rint(2^40 2^(d c)) as a whole number, d <= 0: 2^f on [-1/2, 1/2] as 1 + f q(f), q through the Chebyshev nodes, off by 2^-50 of itself; d = 0 gives 2^40.
// Rounding to whole numbers is done by adding 1.5 2^52 and 2^52, which leaves the number in the lower bits, and the power of two goes into the
// exponent's bits: 64-bit additions and products run at the rate of 32-bit ones, conversions take several operations.
// The coefficients are kept in scalar registers: from literals each product-and-sum is preceded by a move (4096 x 32000 with
// top_p 168 -> 157 us).
struct Exp2 {
  double q[10];
  __device__ __forceinline__ Exp2()
      : q{0x1.62e42fefa39f7p-1, 0x1.ebfbdff82c590p-3, 0x1.c6b08d7044119p-5, 0x1.3b2ab6fba385fp-7, 0x1.5d87fe908f88ap-10, 0x1.4309130378460p-13,
          0x1.ffcb76789860fp-17, 0x1.62bfe46117445p-20, 0x1.b6571de2f2351p-24, 0x1.e5e9f548e5726p-28} {
#pragma unroll
    for (int i = 0; i < 10; ++i) asm volatile("" : "+s"(q[i]));
  }
};
__device__ __forceinline__ u64 weight_of(const Exp2& k, double d, double c) {
  constexpr double WHOLE = 0x1.8p52, POSITIVE = 0x1p52;
  const double y = fmax(fma(d, c, 40.0), -24.0), t = y + WHOLE, f = y - (t - WHOLE);
  double q = k.q[9];
#pragma unroll
  for (int i = 8; i >= 0; --i) q = fma(q, f, k.q[i]);
  q = fma(q, f, 1.0);
  const double w = __hiloint2double(__double2hiint(q) + (__double2loint(t) << 20), __double2loint(q));
  const double sum = w + POSITIVE;
  return (u64)((unsigned)__double2hiint(sum) & 0xfffffu) << 32 | (unsigned)__double2loint(sum);
}

// 64-bit sums over a wavefront by data-parallel-primitive moves (six reads through the LDS crossbar, twice over, take 700 cycles)
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ u64 dpp_u64(u64 v) {
  const int lo = __builtin_amdgcn_update_dpp(0, (int)(unsigned)v, CTRL, ROW_MASK, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(unsigned)(v >> 32), CTRL, ROW_MASK, 0xf, false);
  return (u64)(unsigned)hi << 32 | (unsigned)lo;
}
__device__ __forceinline__ u64 row_scan_u64(u64 v) {      // inclusive, of each 16 lanes
  v += dpp_u64<0x111, 0xf>(v);    // row_shr 1, 2, 4, 8
  v += dpp_u64<0x112, 0xf>(v);
  v += dpp_u64<0x114, 0xf>(v);
  v += dpp_u64<0x118, 0xf>(v);
  return v;
}
__device__ __forceinline__ u64 wave_scan_u64(u64 v) {      // inclusive
  v = row_scan_u64(v);
  v += dpp_u64<0x142, 0xa>(v);    // row_bcast:15 into rows 1 and 3
  v += dpp_u64<0x143, 0xc>(v);    // row_bcast:31 into rows 2 and 3
  return v;
}
__device__ __forceinline__ u64 read_lane_u64(u64 v, int lane) {
  return (u64)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)v, lane);
}
__device__ __forceinline__ u64 wave_sum_u64(u64 v) { return read_lane_u64(wave_scan_u64(v), 63); }

struct Bins {
  u64 mass[BINS];
  unsigned count[BINS];
};

// What stays of a row: the tokens of a logit above `logit`, and of its own the first `ties`, which weigh `weight` each.
struct Border {
  float logit;
  unsigned ties;
  u64 weight;
};
// Where a sum over columns in rising order first exceeds `target`, if of the ties only the first `ties` count.
struct Search {
  u64 target;
  unsigned ties;
};

// What a workgroup's wavefronts tell each other.
struct SampleShared {
  u64 total[16], before;
  unsigned number[16];
  Search left;
  int run;
  float top[16];
  unsigned found, token;
  float logit;
  int bad;
};
// A row and how a workgroup goes over it: a wavefront has a run of tiles of 64 vectors, so that its sums are those of a run of columns.
template <typename T, int THREADS>
struct Sampler {
  static constexpr int N = RowVec<T>::N, WAVES = THREADS / 64, TILE = 64 * N;
  // vectors under way: where a logit is a few operations, and where it is a weight
  static constexpr int LIGHT = THREADS == 1024 ? 8 : 4, HEAVY = 16 / N;
  typedef RowVec<T> R;
  const T* row;
  unsigned cols, skip, tiles, per;
  SampleShared& sh;
  int lane, wave;
  float m;                  // the largest logit
  double c;                 // log2 e / temperature
  Exp2 exp2;

  __device__ __forceinline__ Sampler(SampleShared& shared, const SampleArgs& a) : sh(shared) {
    row = (const T*)a.logits + (size_t)blockIdx.x * a.ld;
    cols = a.cols;
    skip = (unsigned)((uintptr_t)row % 16 / sizeof(T));
    tiles = (cols + skip + TILE - 1) / TILE;
    per = (tiles + WAVES - 1) / WAVES;
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  }
  // the vectors of the tiles t .. t + B - 1, of those before `end`; columns outside the row are -inf.  All loads are under way at once; where the
  // row begins or ends within a tile, its vectors that the row fills only in part are seen to afterwards.
  template <int B>
  __device__ __forceinline__ void read(u32x4 (&v)[B], unsigned t, unsigned end) const {
    const unsigned past = min(t + B, end);
    if ((t || !skip) && past * TILE <= cols + skip) {
      const T* from = row + (size_t)t * TILE - skip;
#pragma unroll
      for (int b = 0; b < B; ++b)
        if (t + b < past) v[b] = ((const u32x4*)from)[b * 64 + lane];
      return;
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const unsigned at = (t + b) * TILE + lane * N;      // column + skip
      v[b] = R::nothing();
      if (t + b < past && at >= skip && at + N <= cols + skip) v[b] = *(const u32x4*)(row + at - skip);
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const unsigned at = (t + b) * TILE + lane * N, to = min(at + N, cols + skip);
      if (t + b < past && (at < skip || at + N > cols + skip))
#pragma unroll 1
        for (unsigned i = max(at, skip); i < to; ++i) R::put(v[b], i - at, row[i - skip]);
    }
  }
  // f(vector, tile) for the tiles of this wavefront, BATCH of them under way
  template <int BATCH, class F>
  __device__ __forceinline__ void each_vector(F f) const {
    const unsigned begin = min(wave * per, tiles), end = min(begin + per, tiles);
    for (unsigned t = begin; t < end; t += BATCH) {
      u32x4 v[BATCH];
      read(v, t, end);
#pragma unroll
      for (int b = 0; b < BATCH; ++b)
        if (t + b < end) f(v[b], t + b);
    }
  }
  template <int BATCH = HEAVY, class F>
  __device__ __forceinline__ void each(F f) const {
    each_vector<BATCH>([&](const u32x4& v, unsigned) {
      float z[N];
      R::unpack(v, z);
#pragma unroll
      for (int e = 0; e < N; ++e) f(z[e]);
    });
  }
  __device__ __forceinline__ u64 weight(float z) const { return weight_of(exp2, (double)z - (double)m, c); }

  // sums over the wavefronts, which are in sh.total: those before this one, and all
  __device__ __forceinline__ u64 totals(u64& all) const {
    const u64 v = row_scan_u64(lane < WAVES ? sh.total[lane] : 0);
    all = read_lane_u64(v, 15);
    return wave ? read_lane_u64(v, wave - 1) : 0;
  }
  __device__ __forceinline__ u64 block_sum(u64 v) const {
    v = wave_sum_u64(v);
    __syncthreads();
    if (lane == 0) sh.total[wave] = v;
    __syncthreads();
    u64 all;
    totals(all);
    return all;
  }
  // what the threads before this one have in all
  __device__ __forceinline__ u64 block_before(u64 v, u64& all) const {
    const u64 upto = wave_scan_u64(v);
    __syncthreads();
    if (lane == 63) sh.total[wave] = upto;
    __syncthreads();
    return totals(all) + upto - v;
  }

  // Of the lanes (of the first 16, or all), which hold sums of consecutive runs of columns (the ties' number apart), the one in which the
  // search ends, and what is left to search there; -1 and what is left behind them all if it is none.
  template <bool ROW>
  __device__ __forceinline__ int pick(Search& s, u64 sum, unsigned number, u64 tie_weight) const {
    const unsigned upto = (unsigned)(ROW ? row_scan_u64(number) : wave_scan_u64(number)), before = upto - number;
    const u64 own = sum + tie_weight * min(number, s.ties > before ? s.ties - before : 0), all = ROW ? row_scan_u64(own) : wave_scan_u64(own);
    const u64 past = __ballot(all > s.target && (!ROW || lane < 16));
    const int k = past ? __ffsll((unsigned long long)past) - 1 : ROW ? 15 : 63;
    const unsigned ties = (unsigned)__builtin_amdgcn_readlane((int)(past ? before : upto), k);
    s.target -= read_lane_u64(past ? all - own : all, k);
    s.ties -= min(s.ties, ties);
    return past ? k : -1;
  }
  // This thread's sum over its columns without ties, and their number: left for all wavefronts to see.
  __device__ __forceinline__ void leave(u64 sum, unsigned number) const {
    sum = wave_sum_u64(sum);
    const unsigned n = (unsigned)wave_sum_u64(number);
    __syncthreads();
    if (lane == 0) { sh.total[wave] = sum; sh.number[wave] = n; }
    __syncthreads();
  }
  // the first wavefront's pick among all wavefronts' sums
  __device__ __forceinline__ int pick_wave(Search& s, u64 tie_weight) const {
    if (wave == 0) {
      const int k = pick<true>(s, lane < WAVES ? sh.total[lane] : 0, lane < WAVES ? sh.number[lane] : 0, tie_weight);
      if (lane == 0) { sh.run = k; sh.left = s; }
    }
    __syncthreads();
    s = sh.left;
    return sh.run;
  }
  // The search's end, in sh.token and sh.logit: among the wavefronts' runs, as `leave` left them, then among the run's tiles, a wavefront
  // each, and among its lanes.  f(logit, weight): whether it is a tie; its weight otherwise.
  template <class F>
  __device__ __forceinline__ void search(Search s, u64 tie_weight, F f) const {
    const unsigned begin = min((unsigned)max(pick_wave(s, tie_weight), 0) * per, tiles), end = min(begin + per, tiles);
    for (unsigned t = begin; t < end; t += WAVES) {
      float z[N];
      u64 own[N], sum = 0;
      unsigned is = 0;
      if (t + wave < end) {
        u32x4 v[1];
        read(v, t + wave, end);
        R::unpack(v[0], z);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          own[e] = 0;
          if (f(z[e], own[e])) is |= 1u << e;
          else sum += own[e];
        }
        // 512 logits weigh 2^49 at most: their ties are counted above that, in the same sum
        const u64 both = wave_sum_u64(sum + ((u64)__popc(is) << 50));
        if (lane == 0) { sh.total[wave] = both & ((1ull << 50) - 1); sh.number[wave] = (unsigned)(both >> 50); }
      } else if (lane == 0) {
        sh.total[wave] = 0;
        sh.number[wave] = 0;
      }
      __syncthreads();
      const int tile = pick_wave(s, tie_weight);
      if (tile < 0) continue;
      if (tile == wave) {
        const int k = pick<false>(s, sum, __popc(is), tie_weight);
        if (lane == k) {
          u64 upto = 0;
          unsigned ties = s.ties;
          int at = -1;
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const bool tie = is >> e & 1;
            upto += tie ? (ties ? tie_weight : 0) : own[e];
            if (tie && ties) --ties;
            if (at < 0 && upto > s.target) { at = e; sh.logit = z[e]; }
          }
          sh.token = (t + wave) * TILE + lane * N - skip + max(at, 0);
        }
      }
      break;
    }
    __syncthreads();
  }

  // the largest logit, and this thread's; false if the row has no answer
  __device__ __forceinline__ bool largest(float& own) {
    own = -INFINITY;
    bool bad = false;
    each<LIGHT>([&](float z) {
      own = fmaxf(own, z);
      bad |= !(z < INFINITY);
    });
    m = wave_max(own);
    __syncthreads();
    if (threadIdx.x == 0) sh.bad = 0;
    __syncthreads();
    if (lane == 0) sh.top[wave] = m;
    if (bad) sh.bad = 1;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, sh.top[w]);
    return !sh.bad && m > -INFINITY;
  }
};

__device__ __forceinline__ u64 top_p_need(float top_p, u64 all) { return max((u64)ceil((double)top_p * (double)all), (u64)1); }
__device__ __forceinline__ u64 draw_target(float uniform, u64 all) {
  const double u = uniform;
  return min((u64)floor((u > 0.0 ? fmin(u, 1.0) : 0.0) * (double)all), all - 1);
}
__device__ __forceinline__ void answer(const SampleArgs& a, int token, float logprob, int kept) {
  if (threadIdx.x) return;
  if (a.token) a.token[blockIdx.x] = token;
  if (a.logprob) a.logprob[blockIdx.x] = logprob;
  if (a.kept) a.kept[blockIdx.x] = kept;
}
__device__ __forceinline__ void no_answer(const SampleArgs& a) { answer(a, -1, __uint_as_float(0x7fc00000u), 0); }
template <class S>
__device__ __forceinline__ void drawn_answer(const SampleArgs& a, const S& p, float temperature, u64 all, unsigned kept) {
  if (threadIdx.x) return;
  answer(a, (int)p.sh.token, (float)(((double)p.sh.logit - (double)p.m) / (double)temperature - log((double)all / ONE)), (int)kept);
}

// ------------------------------------------------------------------------------------- by bins of the logits
// The row is counted and weighed into 2048 bins of equal width in (m - z) / T; the bin that a border falls into is cut again by the bits of
// its logits, until a bin is a single value.
template <typename T, int THREADS>
struct BinSampler : Sampler<T, THREADS> {
  typedef Sampler<T, THREADS> S;
  typedef RowVec<T> R;
  Bins &coarse, &fine;
  // bins per logit, of differences that are taken `h` times, and h m.  A difference that 32 bits do not hold weighs nothing up to a temperature of
  // 1.1e37 (it is more than 29 of those); beyond, halves of the logits are subtracted, whose difference is held.
  float s, h, hm;
  __device__ __forceinline__ BinSampler(const S& base, Bins* b) : S(base), coarse(b[0]), fine(b[1]) {}
  __device__ __forceinline__ void scale(float temperature) {
    h = temperature > 1e37f ? 0.5f : 1.f;
    hm = h * this->m;
    s = bins_per_logit(temperature) / h;
  }
  __device__ __forceinline__ int bin(float z) const { return (int)fminf(fmaf(-z, h, hm) * s, (float)LAST); }

  __device__ __forceinline__ void clear(Bins& b) const {
    __syncthreads();
    for (int i = threadIdx.x; i < BINS; i += THREADS) { b.mass[i] = 0; b.count[i] = 0; }
    __syncthreads();
  }
  // The first bin up to which there are `need` (at least 1) in all, and what lies before it: true if there is one.
  __device__ __forceinline__ bool find(const Bins& b, bool by_mass, u64 need, unsigned& which, u64& before) const {
    constexpr int PER = BINS / THREADS;
    u64 own[PER], sum = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      own[i] = by_mass ? b.mass[threadIdx.x * PER + i] : b.count[threadIdx.x * PER + i];
      sum += own[i];
    }
    if (threadIdx.x == 0) this->sh.found = BINS;
    u64 all, at = this->block_before(sum, all);
    if (at < need && at + sum >= need) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        if (at < need && at + own[i] >= need) { this->sh.found = threadIdx.x * PER + i; this->sh.before = at; }
        at += own[i];
      }
    }
    __syncthreads();
    which = this->sh.found;
    before = this->sh.before;
    return which < BINS;
  }
  // what the bins before `which` weigh
  __device__ __forceinline__ u64 mass_before(const Bins& b, unsigned which) const {
    u64 v = 0;
    for (unsigned i = threadIdx.x; i < which; i += THREADS) v += b.mass[i];
    return this->block_sum(v);
  }

  // The border within a bin: its logits, between `least` and `most`, are put into a list, and a thread adds up what is above one of them.  False if
  // there are more than the list holds.  (1 x 128000 in fp32 with top_p 121 -> 96 us.)
  struct Members {
    static constexpr unsigned MOST = 512;      // (a thread for each)
    float logit[MOST];
    u64 weight[MOST], mass[MOST];
    unsigned above[MOST], equal[MOST], n;
    Border border;
    u64 stays;
  };
  static_assert(sizeof(Members) <= sizeof(Bins), "room");
  __device__ __forceinline__ bool among(unsigned b, float least, float most, bool by_mass, bool weigh, u64 need, Border& out, u64& stays) const {
    Members& l = *(Members*)&fine;
    const unsigned tid = threadIdx.x;
    __syncthreads();
    if (tid == 0) l.n = 0;
    __syncthreads();
    this->template each<S::LIGHT>([&](float z) {
      if (z <= most && z >= least && bin(z) == (int)b) {
        const unsigned i = atomicAdd(&l.n, 1u);
        if (i < Members::MOST) l.logit[i] = z;
      }
    });
    __syncthreads();
    const unsigned n = l.n;
    if (!n || n > Members::MOST) return false;
    if (tid < Members::MOST) {
      l.weight[tid] = tid < n ? this->weight(l.logit[tid]) : 0;
      l.mass[tid] = 0; l.above[tid] = 0; l.equal[tid] = 0;
    }
    __syncthreads();
    const unsigned group = n <= 64 ? 64 : n <= 128 ? 128 : n <= 256 ? 256 : 512, me = tid % group;
    const float z = l.logit[min(me, n - 1)];
    unsigned above = 0, equal = 0;
    u64 mass = 0;
#pragma unroll 4
    for (unsigned j = tid / group; j < n; j += THREADS / group) {
      const float other = l.logit[j];
      const u64 w = l.weight[j];
      above += other > z;
      mass += other > z ? w : 0;
      equal += other == z;
    }
    if (me < n) {
      if (above) { atomicAdd(&l.above[me], above); atomicAdd(&l.mass[me], mass); }
      if (equal) atomicAdd(&l.equal[me], equal);
    }
    __syncthreads();
    if (tid < n) {
      // (the threads of equal logits write the same)
      const u64 w = l.weight[tid], before = by_mass ? l.mass[tid] : l.above[tid], own = by_mass ? w * l.equal[tid] : l.equal[tid];
      if (before < need && before + own >= need) {
        const unsigned ties = (unsigned)(by_mass ? (need - before + w - 1) / w : need - before);
        l.border = Border{z, ties, w};
        l.stays = l.mass[tid] + ties * w;
      }
    }
    __syncthreads();
    out = l.border;
    if (weigh) stays += l.stays;
    __syncthreads();
    return true;
  }

  // The border behind the token at which count (or mass) reaches `need`, and what stays up to it weighs (0 without `weigh`): false if all that
  // weighs anything stays.
  __device__ __forceinline__ bool border(bool by_mass, bool weigh, u64 need, Border& out, u64& stays) const {
    unsigned b;
    u64 before;
    if (!find(coarse, by_mass, need, b, before) || b == LAST) return false;
    stays = weigh ? (by_mass ? before : mass_before(coarse, b)) : 0;
    need -= before;
    // the keys of the bin, and some beside them: roundings move a logit by less than `slack`
    // (infinite where the bin reaches beyond the largest number)
    const float near = (float)b / (s * h), far = (float)(b + 1) / (s * h), slack = (fabsf(this->m) + far) * 0x1p-20f;
    const float most = fminf(fmaxf(this->m - near, -3.4028234e38f) + slack, this->m), least = fmaxf(this->m - far - slack, -3.4028234e38f);
    if (among(b, least, most, by_mass, weigh, need, out, stays)) return true;
    unsigned hi = R::key(most), lo = R::key(least);
    for (;;) {
      const unsigned range = hi - lo, shift = range < BINS ? 0 : 32 - __clz(range) - 11;
      clear(fine);
      this->each([&](float z) {
        const unsigned k = R::key(z);
        if (k >= lo && k <= hi && bin(z) == (int)b) {
          const unsigned at = (hi - k) >> shift;
          atomicAdd(&fine.count[at], 1u);
          if (weigh) atomicAdd(&fine.mass[at], this->weight(z));
        }
      });
      unsigned at;
      if (!find(fine, by_mass, need, at, before)) return false;      // (cannot be)
      need -= before;
      if (weigh) stays += by_mass ? before : mass_before(fine, at);
      const unsigned top = hi - (at << shift);
      if (!shift) {
        // `need` of the bin's tokens, which weigh the same
        out.logit = R::value(top);
        out.weight = this->weight(out.logit);
        out.ties = (unsigned)(by_mass ? (need + out.weight - 1) / out.weight : need);
        stays += out.ties * out.weight;
        __syncthreads();
        return true;
      }
      hi = top;
      lo = max(lo, top - ((1u << shift) - 1));
    }
  }
};

template <typename T, int THREADS>
__device__ __forceinline__ void sample_by_bins(const SampleArgs& a, const karma_sample_rule& rule, float uniform, u64 least, const Sampler<T, THREADS>& base,
                                               Bins* bins) {
  BinSampler<T, THREADS> p(base, bins);
  float own;
  if (!p.largest(own)) return no_answer(a);
  p.scale(rule.temperature);
  const bool by_count = rule.top_k && rule.top_k < a.cols, by_mass = rule.top_p < 1.f;
  Border border{-INFINITY, 0, 0};
  if (by_count || by_mass) {
    p.clear(p.coarse);
    u64 mine = 0;
    p.each([&](float z) {
      const int b = p.bin(z);
      if (b < LAST) {
        if (by_count) atomicAdd(&p.coarse.count[b], 1u);
        if (by_mass) {
          const u64 w = p.weight(z);
          mine += w;
          atomicAdd(&p.coarse.mass[b], w);
        }
      }
    });
    u64 all = by_mass ? p.block_sum(mine) : 0, stays;
    if (by_count && p.border(false, by_mass, rule.top_k, border, stays)) all = stays;
    if (by_mass) p.border(true, true, top_p_need(rule.top_p, all), border, stays);
  }
  // (the border's weight may be below min-p's: then none of its tokens stays)
  if (border.weight < least) border.ties = 0;
  auto drawn = [&](float z, u64& w) {
    if (z == border.logit) return true;
    if (z > border.logit) {
      const u64 v = p.weight(z);
      w = v >= least ? v : 0;
    }
    return false;
  };
  u64 mine = 0;
  unsigned count = 0, ties = 0;
  if (border.logit == -INFINITY && !least) {      // all stays
    p.each([&](float z) {
      const u64 w = p.weight(z);
      mine += w;
      count += w != 0;
    });
  } else {
    // what min-p leaves out needs no weight: by logits first, with room for what the cut's roundings move it by
    const float cut = least > 1 ? p.m + (float)((double)(log2f((float)(least - 1)) - 40.02f) / p.c) - fabsf(p.m) * 0x1p-20f : -INFINITY;
    p.each([&](float z) {
      if (z > border.logit && z >= cut) {
        const u64 w = p.weight(z);
        if (w >= least) { mine += w; count += w != 0; }
      }
      ties += z == border.logit;
    });
  }
  unsigned kept = (unsigned)p.block_sum(count) + (border.weight ? border.ties : 0);
  p.leave(mine, ties);
  u64 all;
  p.totals(all);
  all += border.ties * border.weight;
  p.search(Search{draw_target(uniform, all), border.ties}, border.weight, drawn);
  drawn_answer(a, p, rule.temperature, all, kept);
}

// ------------------------------------------------------------------------------------- by a list of the likeliest tokens
// With a small top_k: there are at least top_k logits from the threads' top_k-th largest maximum on.  Those, few more than top_k, are put
// into a list, and all else is sums over pairs of its tokens.  (64 x 51200 in fp32 with top_p 0.95: 20.6 us at top_k 128, 39 by bins
// at 129.)
// Up to a top_k where the other way is as fast (us by the list / the other way: bf16 512 x 8000 at top_k 96 15.3 / 17.5, at 128 23.4 / 17.3, 2048 x 16000
// at 96 51 / 54, at 128 78 / 54; fp32 at 128 24.5 / 25.1 and 89 / 122).
constexpr unsigned LIST_MOST = 256;
template <typename T>
constexpr unsigned LIST_TOP_K = sizeof(T) == 2 ? 96 : 128;
struct List {
  float logit[LIST_MOST];
  unsigned column[LIST_MOST], rank[LIST_MOST];
  u64 weight[LIST_MOST], before[LIST_MOST], drawn_before[LIST_MOST];
  unsigned count[BINS], n;
  float floor[16];
};
// false: the row has to go another way
template <typename T, int THREADS>
__device__ __forceinline__ bool sample_by_list(const SampleArgs& a, const karma_sample_rule& rule, float uniform, u64 least, Sampler<T, THREADS>& p, List& l) {
  constexpr int N = RowVec<T>::N, WAVES = THREADS / 64;
  const int tid = threadIdx.x;
  for (int i = tid; i < BINS; i += THREADS) l.count[i] = 0;
  if (tid == 0) { l.n = 0; p.sh.found = BINS; }
  float own;
  if (!p.largest(own)) {
    no_answer(a);
    return true;
  }
  // the bin of the top_k-th largest of the threads' maxima, and the smallest maximum that is not behind it
  const float s = bins_per_logit(rule.temperature);
  const int bin = (int)fminf((p.m - own) * s, (float)LAST);
  if (bin < LAST) atomicAdd(&l.count[bin], 1u);
  __syncthreads();
  constexpr int PER = BINS / THREADS;
  unsigned upto = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) upto += l.count[tid * PER + i];
  u64 all, at = p.block_before(upto, all);
  if (at < rule.top_k && at + upto >= rule.top_k) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const unsigned n = l.count[tid * PER + i];
      if (at < rule.top_k && at + n >= rule.top_k) p.sh.found = tid * PER + i;
      at += n;
    }
  }
  __syncthreads();
  if (p.sh.found == BINS) return false;
  float floor = -wave_max(bin <= (int)p.sh.found ? -own : -INFINITY);
  if (p.lane == 0) l.floor[p.wave] = floor;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) floor = fminf(floor, l.floor[w]);
  p.template each_vector<Sampler<T, THREADS>::LIGHT>([&](const u32x4& v, unsigned tile) {
    float z[N];
    RowVec<T>::unpack(v, z);
    float most = z[0];
#pragma unroll
    for (int e = 1; e < N; ++e) most = fmaxf(most, z[e]);
    if (most < floor) return;
    unsigned in = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) in |= z[e] >= floor ? 1u << e : 0;
    for (; in; in &= in - 1) {
      const int e = __ffs((int)in) - 1;
      const unsigned i = atomicAdd(&l.n, 1u);
      if (i < LIST_MOST) { l.logit[i] = RowVec<T>::nth(v, e); l.column[i] = tile * (64 * N) + p.lane * N - p.skip + e; }
    }
  });
  __syncthreads();
  const unsigned n = l.n;
  if (n > LIST_MOST) return false;
  const bool mine = tid < (int)n;
  const u64 weight = mine ? p.weight(l.logit[tid]) : 0;
  if (tid < (int)LIST_MOST) { l.weight[tid] = weight; l.rank[tid] = 0; l.before[tid] = 0; l.drawn_before[tid] = 0; }
  __syncthreads();
  // pairs: a token of the list for every thread of a group, and the groups share the others
  const unsigned group = n <= 64 ? 64 : n <= 128 ? 128 : 256, me = tid % group;
  const float z = l.logit[min(me, n - 1)];
  const unsigned column = l.column[min(me, n - 1)];
  unsigned rank = 0;
  u64 before = 0;
#pragma unroll 4
  for (unsigned j = tid / group; j < n; j += THREADS / group) {
    const float other = l.logit[j];
    const unsigned c = l.column[j];
    const u64 w = l.weight[j];
    const bool first = other > z || (other == z && c < column);
    rank += first;
    before += first ? w : 0;
  }
  if (me < n && rank) { atomicAdd(&l.rank[me], rank); atomicAdd(&l.before[me], before); }
  __syncthreads();
  // (a token's own thread from here on)
  rank = mine ? l.rank[tid] : n;
  before = mine ? l.before[tid] : 0;
  bool stays = rank < rule.top_k;
  if (rule.top_p < 1.f) {
    const u64 need = top_p_need(rule.top_p, p.block_sum(stays ? weight : 0));
    stays = stays && before < need;
  }
  stays = stays && weight && weight >= least;
  // 256 tokens weigh 2^48 at most: their number above that, in the same sum
  const u64 sums = p.block_sum(stays ? weight + (1ull << 52) : 0), total = sums & ((1ull << 52) - 1), target = draw_target(uniform, total);
  if (tid < (int)LIST_MOST) l.weight[tid] = stays ? weight : 0;
  __syncthreads();
  before = 0;
#pragma unroll 4
  for (unsigned j = tid / group; j < n; j += THREADS / group) {
    const unsigned c = l.column[j];
    const u64 w = l.weight[j];
    before += c < column ? w : 0;
  }
  if (me < n && before) atomicAdd(&l.drawn_before[me], before);
  __syncthreads();
  if (stays && l.drawn_before[tid] <= target && target < l.drawn_before[tid] + weight) {
    p.sh.token = l.column[tid];
    p.sh.logit = l.logit[tid];
  }
  __syncthreads();
  drawn_answer(a, p, rule.temperature, total, (unsigned)(sums >> 52));
  return true;
}

// ------------------------------------------------------------------------------------- by counters of bf16 logits
typedef short short2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ short2_t as_short2(unsigned v) { return __builtin_bit_cast(short2_t, v); }
__device__ __forceinline__ short2_t max2(short2_t a, short2_t b) { return __builtin_elementwise_max(a, b); }
// From 2^-14 to 2^18 there are 4096 bf16 numbers, and as many negative ones: the row is counted by its bits, and everything but the draw itself
// follows from the counters, with one weight for every value that occurs.  Ranks rise as logits fall: the positive ones, a group of 64 for 0
// alone, the negative ones.  The few numbers next to 0 are kept one by one; what lies below -2^18 is left out (masked logits) where it weighs
// nothing.  A row that has other numbers, many next to 0, or its border among those goes by bins.  (1024 x 16000 with top_p 0.95: 39 us; fp32 rows, by
// bins, 60.)
constexpr unsigned CT_LOW = 0x3880, CT_SIDE = 4096;
constexpr unsigned ZERO_GROUP = CT_SIDE / 64, CT_GROUPS = 2 * ZERO_GROUP + 1, RANK_ZERO = CT_SIDE, RANK_NEGATIVE = CT_SIDE + 64, CT_RANKS = RANK_NEGATIVE + CT_SIDE;
constexpr unsigned CT_TINY = 64;
constexpr float CT_FAR = 262144.f;
struct Counted {
  unsigned counter[2 * CT_SIDE];      // by bits: positive, negative
  unsigned zeros, tiny;
  unsigned short tiny_bits[CT_TINY];
  u64 mass[CT_GROUPS];
  unsigned count[CT_GROUPS];
  unsigned short list[CT_SIDE / 2];   // vectors of four counters of which one is not 0
  unsigned vectors;
  // the group that a border falls into and what lies before it; the border found, what stays up to it, and the weight of its rank
  u64 mass_before, stays, border_weight;
  unsigned group, count_before, border, ties, count_stays, first;
  int other, left_out;

  __device__ __forceinline__ unsigned of(unsigned rank) const {
    return rank < CT_SIDE ? counter[CT_SIDE - 1 - rank] : rank >= RANK_NEGATIVE ? counter[rank - RANK_NEGATIVE + CT_SIDE] : rank == RANK_ZERO ? zeros : 0;
  }
};
__device__ __forceinline__ float rank_value(unsigned rank) {
  const unsigned bits = rank < CT_SIDE ? CT_LOW + CT_SIDE - 1 - rank : rank >= RANK_NEGATIVE ? 0x8000 + CT_LOW + rank - RANK_NEGATIVE : 0;
  return __uint_as_float(bits << 16);
}
// (numbers that have no rank: one behind all)
__device__ __forceinline__ unsigned rank_of(unsigned u) {
  const unsigned i = (u & 0x7fff) - CT_LOW;
  if (i < CT_SIDE) return u & 0x8000 ? RANK_NEGATIVE + i : CT_SIDE - 1 - i;
  return u & 0x7fff ? CT_RANKS : RANK_ZERO;
}
__device__ __forceinline__ bool next_to_zero(unsigned u) { return (u & 0x7fff) - 1 < CT_LOW - 1; }
// the room of all ways, which later holds the weights by rank; with 49 KB three rows have room on a compute unit
constexpr size_t SAMPLE_ROOM = sizeof(Counted) > 2 * sizeof(Bins) ? sizeof(Counted) : 2 * sizeof(Bins);
constexpr unsigned CT_TABLE = SAMPLE_ROOM / sizeof(double);

// false: the row has to go by bins
template <int THREADS>
__device__ __forceinline__ bool sample_by_counters(const SampleArgs& a, const karma_sample_rule& rule, float uniform, u64 least, Sampler<bf16_t, THREADS>& p,
                                                   Counted& ct) {
  constexpr int AHEAD = THREADS == 1024 ? 8 : 4;
  const int lane = p.lane, wave = p.wave, tid = threadIdx.x;
  // ---- count the row; its first vectors are under way while the counters are cleared
  u32x4 ahead[AHEAD];
  const unsigned begin = min(wave * p.per, p.tiles), end = min(begin + p.per, p.tiles);
  p.read(ahead, begin, end);
  for (int i = tid; i < (int)CT_SIDE / 2; i += THREADS) ((u32x4*)ct.counter)[i] = u32x4{0, 0, 0, 0};
  for (int i = tid; i < (int)CT_GROUPS; i += THREADS) { ct.count[i] = 0; ct.mass[i] = 0; }
  if (tid == 0) {
    ct.zeros = 0; ct.tiny = 0; ct.vectors = 0; ct.other = 0; ct.left_out = 0; ct.first = CT_GROUPS; ct.group = CT_GROUPS; ct.border = CT_RANKS - 1; ct.ties = 0xffffffffu;
    ct.border_weight = 0;
  }
  __syncthreads();
  auto for_vectors = [&](auto f) {
#pragma unroll
    for (int b = 0; b < AHEAD; ++b)
      if (begin + b < end) f(ahead[b]);
    for (unsigned t = begin + AHEAD; t < end; t += AHEAD) {
      u32x4 v[AHEAD];
      p.read(v, t, end);
#pragma unroll
      for (int b = 0; b < AHEAD; ++b)
        if (t + b < end) f(v[b]);
    }
  };
  // f for each of a vector's logits for which `is` holds, in a loop that is not unrolled: few have any
  auto for_some = [&](const u32x4& v, auto is, auto f) {
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
      const unsigned d = i & 4 ? (i & 2 ? v[3] : v[2]) : i & 2 ? v[1] : v[0], u = i & 1 ? d >> 16 : d & 0xffff;
      if (is(u)) f(u);
    }
  };
  auto has_rank = [](unsigned u) { return (u & 0x7fff) - CT_LOW < CT_SIDE; };
  auto count = [&](const u32x4& v) {
    bool others = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned u = i % 2 ? v[i / 2] >> 16 : v[i / 2] & 0xffff, at = (u & 0x7fff) - CT_LOW;
      if (at < CT_SIDE) atomicAdd(&ct.counter[at + __umul24(u >> 15, CT_SIDE)], 1u);
      others |= at >= CT_SIDE;
    }
    if (!others) return;
    // most of them are masked, -inf or far below
    constexpr unsigned FAR = 0x8000 + CT_LOW + CT_SIDE, FARS = 0xff80 - FAR;
    bool left_out = false;
    others = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned u = i % 2 ? v[i / 2] >> 16 : v[i / 2] & 0xffff;
      left_out |= u - FAR < FARS;
      others |= !has_rank(u) && u - FAR > FARS;
    }
    if (left_out) ct.left_out = 1;
    if (!others) return;
    for_some(v, [&](unsigned u) { return !has_rank(u) && u - FAR > FARS; },
             [&](unsigned u) {
               if (!(u & 0x7fff)) atomicAdd(&ct.zeros, 1u);
               else if (next_to_zero(u)) {
                 const unsigned i = atomicAdd(&ct.tiny, 1u);
                 if (i < CT_TINY) ct.tiny_bits[i] = (unsigned short)u;
                 else ct.other = 1;
               } else ct.other = 1;
             });
  };
  auto largest_of = [](const u32x4& v) {
    // as whole numbers of 16 bits positive logits are ordered and negative ones lie below them
    const short2_t x = max2(max2(as_short2(v[0]), as_short2(v[1])), max2(as_short2(v[2]), as_short2(v[3])));
    return max(x[0], x[1]);
  };
  for_vectors(count);
  __syncthreads();
  if (ct.other) return false;
  // ---- the counters that are not 0 are put into a list by fours; 64 of them are a group
  for (int at = tid; at < (int)CT_SIDE / 2; at += THREADS) {
    const u32x4 v = ((const u32x4*)ct.counter)[at];
    const unsigned n = (v[0] + v[1]) + (v[2] + v[3]);
    const u64 some = __ballot(n != 0);
    if (!some) continue;
    unsigned place = 0;
    if (lane == 0) place = atomicAdd(&ct.vectors, (unsigned)__popcll(some));
    place = __builtin_amdgcn_readfirstlane(place) + __popcll(some & ((1ull << lane) - 1));
    if (n) {
      ct.list[place] = (unsigned short)at;
      atomicAdd(&ct.count[at < (int)CT_SIDE / 4 ? ZERO_GROUP - 1 - at / 16 : at / 16 + 1], n);
    }
  }
  if (tid == 0) ct.count[ZERO_GROUP] = ct.zeros + ct.tiny;
  __syncthreads();
  // ---- the largest logit
  const unsigned own_count = tid < (int)CT_GROUPS ? ct.count[tid] : 0, tiny = ct.tiny, vectors = ct.vectors;
  u64 row_count;
  const unsigned count_before = (unsigned)p.block_before(own_count, row_count);
  if (!row_count) return false;
  if (own_count && !count_before) ct.first = tid;
  __syncthreads();
  if (tiny && ct.first == ZERO_GROUP) return false;
  const unsigned first = ct.first * 64 + __ffsll((unsigned long long)__ballot(ct.of(ct.first * 64 + lane) != 0)) - 1;
  p.m = rank_value(first);
  if (ct.left_out && !(p.m + CT_FAR > REACH * rule.temperature)) return false;

  // f(group, four ranks of it, their counts); 0 and the numbers next to it are another matter
  auto sweep = [&](auto f) {
    for (unsigned i = tid; i < vectors; i += THREADS) {
      const unsigned at = ct.list[i];
      const u32x4 v = ((const u32x4*)ct.counter)[at];
      const bool high = at < CT_SIDE / 4;
      unsigned n[4], r[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        n[j] = v[j];
        r[j] = high ? CT_SIDE - 1 - (at * 4 + j) : RANK_NEGATIVE - CT_SIDE + at * 4 + j;
      }
      f(high ? ZERO_GROUP - 1 - at / 16 : at / 16 + 1, r, n);
    }
  };
  // (ranks before the first one have no tokens)
  auto rank_weight = [&](unsigned rank) { return p.weight(fminf(rank_value(rank), p.m)); };
  sweep([&](unsigned g, const unsigned* r, const unsigned* n) {
    u64 w = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) w += n[j] * rank_weight(r[j]);
    atomicAdd(&ct.mass[g], w);
  });
  if (ct.count[ZERO_GROUP] && wave == 0) {
    u64 w = lane == 0 ? ct.zeros * rank_weight(RANK_ZERO) : 0;
    if (lane < (int)tiny) w += p.weight(bf2f(ct.tiny_bits[lane]));
    w = wave_sum_u64(w);
    if (lane == 0) ct.mass[ZERO_GROUP] = w;
  }
  __syncthreads();
  const u64 own_mass = tid < (int)CT_GROUPS ? ct.mass[tid] : 0;
  u64 all;
  const u64 mass_before = p.block_before(own_mass, all);

  // ---- the tokens that stay: all of the ranks before `border`, and `ties` of its own.  One wavefront looks into the group.
  auto into_group = [&](u64 need, bool by_mass) {
    if (wave) return;
    const unsigned g = ct.group, n = ct.of(g * 64 + lane);
    const u64 w = n ? rank_weight(g * 64 + lane) : 0;
    const u64 mass = ct.mass_before + wave_scan_u64(n * w), number = ct.count_before + wave_scan_u64(n);
    const int at = __ffsll((unsigned long long)__ballot((by_mass ? mass : number) >= need)) - 1;
    if (lane != at) return;
    // as many of the rank's tokens, which weigh the same, as reach it
    const unsigned some = by_mass ? (unsigned)((need - (mass - n * w) + w - 1) / w) : (unsigned)(need - (number - n));
    ct.border = g * 64 + at;
    ct.ties = some;
    ct.border_weight = w;
    ct.stays = mass - (n - some) * w;
    ct.count_stays = (unsigned)number - (n - some);
  };
  auto from_here = [&]() { ct.group = tid; ct.mass_before = mass_before; ct.count_before = count_before; };
  if (rule.top_k && rule.top_k < row_count) {
    if (count_before < rule.top_k && count_before + own_count >= rule.top_k) from_here();
    __syncthreads();
    if (tiny && ct.group == ZERO_GROUP) return false;
    into_group(rule.top_k, false);
    __syncthreads();
    all = ct.stays;
  }
  if (rule.top_p < 1.f) {
    const u64 need = top_p_need(rule.top_p, all);
    if (mass_before < need && mass_before + own_mass >= need) from_here();
    __syncthreads();
    if (tiny && ct.group == ZERO_GROUP) return false;
    into_group(need, true);
  }
  __syncthreads();
  const unsigned border = ct.border;
  unsigned ties = ct.ties, kept = ct.count_stays;
  if (ct.border_weight && !least) all = ct.stays;
  else {
    u64 sum = 0;
    unsigned number = 0;
    auto add = [&](unsigned some, u64 w) {
      if (w >= least && w) { sum += some * w; number += some; }
    };
    sweep([&](unsigned g, const unsigned* r, const unsigned* n) {
      if (g > border / 64) return;
#pragma unroll
      for (int j = 0; j < 4; ++j) add(r[j] < border ? n[j] : r[j] == border ? min(n[j], ties) : 0, rank_weight(r[j]));
    });
    if (border >= RANK_ZERO) {
      if (tid == 0) add(border > RANK_ZERO ? ct.zeros : min(ct.zeros, ties), rank_weight(RANK_ZERO));
      if (tid < (int)tiny) add(1, p.weight(bf2f(ct.tiny_bits[tid])));
    }
    kept = (unsigned)p.block_sum(number);
    all = p.block_sum(sum);
  }
  const Search s{draw_target(uniform, all), ties};
  const u64 limit = p.weight(rank_value(border)), tie_weight = limit >= least ? limit : 0;
  const unsigned span = border - first;
  const float z_border = rank_value(border);
  auto weigh = [&](float z) {
    const u64 w = p.weight(z);
    return w >= least ? w : 0;
  };
  if (span + 2 <= CT_TABLE) {
    // The weights of the ranks that stay, where the counters were; a mark for the border's; and a 0 behind them that all others read: a read
    // without a branch can be under way with the next ones.  64 logits of a lane weigh 2^46 at most, and their marks lie above that.
    constexpr double MARK = 0x1p47;
    double* table = (double*)&ct;
    __syncthreads();
    for (unsigned i = tid; i <= span + 1; i += THREADS) table[i] = i < span ? (double)weigh(rank_value(first + i)) : i == span ? MARK : 0.0;
    __syncthreads();
    u64 sum = 0;
    unsigned number = 0;
    // `none`: whether none of a vector's logits stays, at six operations for eight of them
    auto pass = [&](auto none, auto add) {
      for (unsigned t = begin; t < end; t += AHEAD) {
        u32x4 v[AHEAD];
        p.read(v, t, end);
        double mine = 0.0;
#pragma unroll
        for (int b = 0; b < AHEAD; ++b)
          if (t + b < end && !__all(none(v[b]))) {
#pragma unroll
            for (int i = 0; i < 4; ++i) mine += add(v[b][i] & 0xffff) + add(v[b][i] >> 16);
          }
        const double marks = floor(mine * (1 / MARK));
        number += (unsigned)marks;
        sum += (u64)(mine - marks * MARK);
      }
    };
    const unsigned top = __float_as_uint(p.m) >> 16;
    // (the rank by one subtraction where all that stays has one sign)
    if (border < RANK_ZERO || first > RANK_ZERO) {
      const unsigned from = border < RANK_ZERO ? top : 0 - top, sign = border < RANK_ZERO ? 0xffffffffu : 0;      // top - u, or u - top
      const unsigned add = from - sign;
      const short least_bits = border < RANK_ZERO ? (short)(__float_as_uint(z_border) >> 16) : (short)-32768;
      pass([&](const u32x4& v) { return largest_of(v) < least_bits; }, [&](unsigned u) { return table[min((u ^ sign) + add, span + 1)]; });
      p.leave(sum, number);
      p.search(s, tie_weight, [&](float z, u64& w) {
        const unsigned i = min(((__float_as_uint(z) >> 16) ^ sign) + add, span + 1);
        w = (u64)table[i];
        return i == span;
      });
    } else {
      auto of = [&](unsigned u) { return table[min(rank_of(u) - first, span + 1)]; };
      auto stays = [&](unsigned u) { return next_to_zero(u) && __uint_as_float(u << 16) > z_border; };
      pass([&](const u32x4& v) {
             if (tiny) for_some(v, stays, [&](unsigned u) { sum += weigh(__uint_as_float(u << 16)); });
             return false;
           }, of);
      p.leave(sum, number);
      p.search(s, tie_weight, [&](float z, u64& w) {
        const unsigned u = __float_as_uint(z) >> 16;
        w = tiny && stays(u) ? weigh(z) : (u64)of(u);
        return z == z_border;
      });
    }
  } else {
    u64 mine = 0;
    unsigned number = 0;
    p.each([&](float z) {
      if (z > z_border) mine += weigh(z);
      number += z == z_border;
    });
    p.leave(mine, number);
    p.search(s, tie_weight, [&](float z, u64& w) {
      w = z > z_border ? weigh(z) : 0;
      return z == z_border;
    });
  }
  drawn_answer(a, p, rule.temperature, all, kept);
  return true;
}

// A row's way by its rule.  What bounds it: vector operations, of which a compute unit does one of 64 lanes a cycle, and the steps between barriers, some
// 500 to 2000 cycles each.  8 x 51200 in bf16 with top_k 50 and top_p 0.9: 13 us in the kernel, of which the two passes over the row take 6; 4096 x 32000 with
// top_p 0.95: 147 us, at 1.8 TB/s of logits.  Some 64 of them do not depend on the columns (4096 x 500 takes 73, x 2000 69, x 8000 87): clearing and
// walking the counters, weights of the values that occur, a table of them, some twenty barriers, 6600 vector operations a row by counter; the rest is 20 vector
// operations, an LDS atomic and an LDS read a logit, of which the operations alone take 67.  301 x 50021 in fp32 without limits: 40 us, two
// passes of which the second takes 20 operations of 64 bits a logit.
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == 512 ? 6 : 4) void sample_kernel(SampleArgs a) {
  constexpr bool COUNTED = sizeof(T) == 2;
  __shared__ SampleShared sh;
  __shared__ __attribute__((aligned(16))) unsigned char room[SAMPLE_ROOM];
  Sampler<T, THREADS> p(sh, a);
  const karma_sample_rule rule = a.rules[a.n_rules == 1 ? 0 : blockIdx.x];
  const float uniform = a.uniform[blockIdx.x];
  if (!(rule.temperature >= 0.f && rule.temperature < INFINITY) || rule.top_p != rule.top_p || rule.min_p != rule.min_p) return no_answer(a);
  if (rule.temperature == 0.f || rule.top_k == 1 || rule.top_p <= 0.f) {
    // one token stays: the first of the largest
    float own;
    if (!p.largest(own)) return no_answer(a);
    unsigned ties = 0;
    p.template each<Sampler<T, THREADS>::LIGHT>([&](float z) { ties += z == p.m; });
    p.leave(0, ties);
    p.search(Search{0, 1}, 1, [&](float z, u64&) { return z == p.m; });
    return answer(a, (int)sh.token, 0.f, 1);
  }
  p.c = 1.4426950408889634074 / (double)rule.temperature;
  const u64 least = rule.min_p > 0.f ? (u64)ceil(fmin((double)rule.min_p, 1.0) * ONE) : 0;
  static_assert(sizeof(List) <= SAMPLE_ROOM, "room");
  if (rule.top_k && rule.top_k <= LIST_TOP_K<T> && rule.top_k < a.cols) {
    if (sample_by_list<T, THREADS>(a, rule, uniform, least, p, *(List*)room)) return;
    __syncthreads();
  }
  if constexpr (COUNTED) {
    if ((rule.top_k && rule.top_k < a.cols) || rule.top_p < 1.f) {
      if (sample_by_counters<THREADS>(a, rule, uniform, least, p, *(Counted*)room)) return;
      __syncthreads();
    }
  }
  sample_by_bins<T, THREADS>(a, rule, uniform, least, p, (Bins*)room);
}

bool aligned_to(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

}  // namespace

// Threads of a row: more of them shorten a long row's way, where every row has a compute unit to itself (with top_p 0.95, us at 512 / 1024 threads: 1 x 128000 in
// bf16 34 / 27, in fp32 119 / 96; 256 x 51200 38 / 31 and 64 / 58; 256 x 12000 19.5 / 19.5 and 20.8 / 20.9, 64 x 8000 14.5 / 16.4 and 17.5 / 18.5); otherwise three rows of
// 512 threads on a compute unit are better than one of 1024 (300 x 51200 44 / 47 and 84 / 99, 1024 x 16000 39 / 67 and 60 / 87, 4096 x 2000 70 / 186 and 74 / 197).
static int sample_threads(uint32_t rows, uint32_t cols) { return rows <= 256 && cols > 12288 ? 1024 : 512; }

int sample_rows(SampleArgs a, bool bf16, hipStream_t s) {
  if (!a.ld) a.ld = a.cols;
  if (!a.cols || a.cols > KARMA_SAMPLE_COLS_MAX || a.rows >= SP_GRID || a.ld < a.cols || a.ld > INT64_MAX / 8 / ((uint64_t)a.rows + 1)) return KARMA_E_INVAL;
  if (a.n_rules != 1 && a.n_rules != a.rows) return KARMA_E_INVAL;
  if (!a.token && !a.logprob && !a.kept) return KARMA_E_INVAL;
  for (const void* p : {(const void*)a.rules, (const void*)a.uniform, (const void*)a.token, (const void*)a.logprob, (const void*)a.kept})
    if (!aligned_to(p, 4)) return KARMA_E_INVAL;
  if (!a.rows) return KARMA_OK;
  if (!a.logits || !a.rules || !a.uniform || !aligned_to(a.logits, bf16 ? 2 : 4)) return KARMA_E_INVAL;
#define KARMA_SAMPLE_LAUNCH(T, THREADS) hipLaunchKernelGGL((sample_kernel<T, THREADS>), dim3(a.rows), dim3(THREADS), 0, s, a)
  const int threads = sample_threads(a.rows, a.cols);
  if (bf16) { if (threads == 512) KARMA_SAMPLE_LAUNCH(bf16_t, 512); else KARMA_SAMPLE_LAUNCH(bf16_t, 1024); }
  else { if (threads == 512) KARMA_SAMPLE_LAUNCH(float, 512); else KARMA_SAMPLE_LAUNCH(float, 1024); }
#undef KARMA_SAMPLE_LAUNCH
  return hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

}  // namespace karma

using namespace karma;

// (none is needed: a row is one workgroup's)
extern "C" uint64_t karma_k_sample_ws_bytes(uint32_t, uint32_t) { return 0; }

#define KARMA_SAMPLE_ENTRY(SUFFIX, T, BF16)                                                                                                  \
  extern "C" int karma_k_sample_##SUFFIX(const T* logits, uint64_t ld, const karma_sample_rule* rules, uint32_t n_rules, const float* uniform, \
                                         int32_t* token, float* logprob, int32_t* kept, uint32_t rows, uint32_t cols, void*, uint64_t,       \
                                         void* stream) {                                                                                     \
    return sample_rows(SampleArgs{logits, ld, rules, n_rules, uniform, token, logprob, kept, rows, cols}, BF16, (hipStream_t)stream);        \
  }
KARMA_SAMPLE_ENTRY(bf16, void, true)
KARMA_SAMPLE_ENTRY(f32, float, false)
