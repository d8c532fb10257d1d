// Queries and keys on their way to attention: every head's vector x of d columns is normalised,
//   r = 1 / sqrt(mean(x^2) + eps),  n = r x gamma,
// and pairs (a, b) of its first `rot` columns are turned by the token's position times the pair's frequency,
//   (a, b) -> (a cos - b sin, b cos + a sin),
// a pair being columns i and i + rot / 2, or 2 i and 2 i + 1.  Backward: the gradient g of n is the output's, turned back;
//   dgamma = sum over tokens and heads of g r x,  dx = r g gamma - x r^3 mean(g gamma x).
// Everything is fp32 between one load and one store, but for the joins of dgamma's sums.  Angles are fp64 until they are reduced to a part
// of a turn, at most half of one, which is rounded to fp32 for sine and cosine: at a position of 100000 fp32 has lost 17 of the angle's 24 bits.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_utils.h"
#include "karma.h"
#include "kernels.h"

namespace karma {
namespace {

constexpr int QK_WAVES = 4, QK_BWD_WAVES = 8;


// V elements between memory and fp32, one access
template <typename T, int V>
struct Piece;
template <>
struct Piece<bf16_t, 8> { u32x4 v; };
template <>
struct Piece<bf16_t, 4> { u32x2 v; };
template <>
struct Piece<bf16_t, 2> { unsigned v; };
template <>
struct Piece<bf16_t, 1> { bf16_t v; };
template <>
struct Piece<float, 4> { u32x4 v; };
template <>
struct Piece<float, 2> { u32x2 v; };
template <>
struct Piece<float, 1> { float v; };

template <typename T, int V>
__device__ __forceinline__ Piece<T, V> load_piece(const T* p) { return *(const Piece<T, V>*)p; }
template <typename T, int V>
__device__ __forceinline__ Piece<T, V> no_piece() { return Piece<T, V>{}; }
__device__ __forceinline__ void to_f32(const Piece<bf16_t, 8>& p, float* f) { unpack8(p.v, f); }
__device__ __forceinline__ void to_f32(const Piece<bf16_t, 4>& p, float* f) {
#pragma unroll
  for (int i = 0; i < 2; ++i) { f[2 * i] = __uint_as_float(p.v[i] << 16); f[2 * i + 1] = __uint_as_float(p.v[i] & 0xffff0000u); }
}
__device__ __forceinline__ void to_f32(const Piece<bf16_t, 2>& p, float* f) { f[0] = __uint_as_float(p.v << 16); f[1] = __uint_as_float(p.v & 0xffff0000u); }
__device__ __forceinline__ void to_f32(const Piece<bf16_t, 1>& p, float* f) { f[0] = bf2f(p.v); }
template <int V>
__device__ __forceinline__ void to_f32(const Piece<float, V>& p, float* f) { __builtin_memcpy(f, &p, V * sizeof(float)); }
__device__ __forceinline__ void store_piece(bf16_t* p, const float* f, std::integral_constant<int, 8>) { *(u32x4*)p = pack8(f); }
__device__ __forceinline__ void store_piece(bf16_t* p, const float* f, std::integral_constant<int, 4>) { *(u32x2*)p = u32x2{pack2(f[0], f[1]), pack2(f[2], f[3])}; }
__device__ __forceinline__ void store_piece(bf16_t* p, const float* f, std::integral_constant<int, 2>) { *(unsigned*)p = pack2(f[0], f[1]); }
__device__ __forceinline__ void store_piece(bf16_t* p, const float* f, std::integral_constant<int, 1>) { *p = (bf16_t)pack2(f[0], 0.f); }
template <int V>
__device__ __forceinline__ void store_piece(float* p, const float* f, std::integral_constant<int, V>) {
  Piece<float, V> q;
  __builtin_memcpy(&q, f, V * sizeof(float));
  *(Piece<float, V>*)p = q;
}

struct QkArgs {
  const void* x[3];             // queries, keys, values (or what becomes of them backward: dyv)
  const void* dy[2];            // backward
  void* out[3];                 // y; backward dx
  const void* gamma[2];         // or null: ones
  float* partial;               // backward: a row [2][d] of sums for dgamma from every workgroup, or null
  const int* positions;         // or null: token % seq
  const double* freq;
  size_t ld_x[3], ld_dy[2], ld_out[3];
  unsigned tokens, seq;
  int heads[3], d, rot, norm;
  float eps;
  int lanes;                    // a head has `lanes` lanes, a power of two
  int parts;                    // a token's heads are divided over `parts` wavefronts
};

// sum over groups of `lanes` neighbouring lanes, left in every one of them
__device__ __forceinline__ float group_sum(float v, int lanes) {
  if (lanes >= 2) v += dpp_from<0xB1, 0xf>(0.f, v);     // quad_perm [1,0,3,2]
  if (lanes >= 4) v += dpp_from<0x4E, 0xf>(0.f, v);     // quad_perm [2,3,0,1]
  if (lanes >= 8) v += dpp_from<0x141, 0xf>(0.f, v);    // row_half_mirror
  if (lanes >= 16) v += dpp_from<0x140, 0xf>(0.f, v);   // row_mirror
  if (lanes >= 32) v += __shfl_xor(v, 16, 64);
  if (lanes >= 64) v += __shfl_xor(v, 32, 64);
  return v;
}

// What a lane has of every head: NU units of 2 V columns, V of them (lo) and V others (hi) that they turn with.  Unit u of the
// turned columns is u V .. and rot / 2 + u V .., or (PAIRS) 2 u V .. + 2 V, of which the second half may not turn; the columns behind
// `rot` are cut into runs of 2 V.
// Cosines and sines of a token's pairs are computed once by a wavefront, a pair a lane, and handed on through LDS.
typedef float PairTurn[KARMA_QK_D_MAX / 2][2];
template <int V, int NU, bool PAIRS>
struct Units {
  int lo[NU], hi[NU], unit[NU];
  bool there[NU], turns[NU], turns_hi[NU];
  float c[NU][V], s[NU][V];
  __device__ __forceinline__ void place(const QkArgs& a, int lane) {
    const int units = a.d / (2 * V);
#pragma unroll
    for (int k = 0; k < NU; ++k) {
      const int u = lane % a.lanes + k * a.lanes;
      there[k] = u < units;
      turns[k] = 2 * u * V < a.rot;
      turns_hi[k] = PAIRS && V > 1 ? (2 * u + 1) * V < a.rot : turns[k];
      unit[k] = turns[k] ? u : 0;
      const bool pairs = PAIRS || !turns[k];
      lo[k] = pairs ? 2 * u * V : u * V;
      hi[k] = pairs ? 2 * u * V + V : a.rot / 2 + u * V;
      if (!there[k]) lo[k] = hi[k] = 0;
    }
  }
  __device__ __forceinline__ void angles(const QkArgs& a, int lane, int token, PairTurn& pairs) {
    if (!a.rot) return;
    const double at = a.positions ? (double)a.positions[token] : (double)((unsigned)token % a.seq);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // (the last token's have been read)
    __builtin_amdgcn_wave_barrier();
    for (int i = lane; i < a.rot / 2; i += 64) {
      const double turn = at * a.freq[i] * 0.15915494309189533577;
      float s1, c1;
      sincospif(2.f * (float)(turn - rint(turn)), &s1, &c1);
      pairs[i][0] = c1;
      pairs[i][1] = s1;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < NU; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        c[k][e] = pairs[unit[k] * V + e][0];
        s[k][e] = pairs[unit[k] * V + e][1];
      }
  }
  // in place; dir -1: back.  (Columns that do not turn are left alone, not turned by 0: the other one may be infinite.)
  __device__ __forceinline__ void turn(int k, float* x, float* y, float dir) const {
    if constexpr (PAIRS && V > 1) {
      float f[2 * V];
#pragma unroll
      for (int e = 0; e < V; ++e) { f[e] = x[e]; f[V + e] = y[e]; }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float p = f[2 * e], q = f[2 * e + 1], t = dir * s[k][e];
        const bool on = e < V / 2 ? turns[k] : turns_hi[k];
        f[2 * e] = on ? fmaf(p, c[k][e], -q * t) : p;
        f[2 * e + 1] = on ? fmaf(q, c[k][e], p * t) : q;
      }
#pragma unroll
      for (int e = 0; e < V; ++e) { x[e] = f[e]; y[e] = f[V + e]; }
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float p = x[e], q = y[e], t = dir * s[k][e];
        x[e] = turns[k] ? fmaf(p, c[k][e], -q * t) : p;
        y[e] = turns[k] ? fmaf(q, c[k][e], p * t) : q;
      }
    }
  }
};

// Values: moved unchanged.  Iterations `first`, `first + step`, ... of 64 / lanes heads each.
template <typename T, int V, int NU, class U>
__device__ __forceinline__ void move_values(const QkArgs& a, const U& un, size_t token, int lane, int first, int step) {
  const int per = 64 / a.lanes, n = (a.heads[2] + per - 1) / per;
  const T* x = (const T*)a.x[2] + token * a.ld_x[2];
  T* y = (T*)a.out[2] + token * a.ld_out[2];
  for (int it = first; it < n; it += step) {
    const int head = it * per + lane / a.lanes;
    if (head >= a.heads[2]) continue;
#pragma unroll
    for (int k = 0; k < NU; ++k)
      if (un.there[k]) {
        const size_t at = (size_t)head * a.d;
        const Piece<T, V> p = load_piece<T, V>(x + at + un.lo[k]), q = load_piece<T, V>(x + at + un.hi[k]);
        *(Piece<T, V>*)(y + at + un.lo[k]) = p;
        *(Piece<T, V>*)(y + at + un.hi[k]) = q;
      }
  }
}

template <typename T, int V, int NU>
struct Gamma {
  Piece<T, V> lo[NU], hi[NU];
  template <class U>
  __device__ __forceinline__ void load(const void* g, const U& un) {
    if (!g) return;
#pragma unroll
    for (int k = 0; k < NU; ++k) {
      lo[k] = load_piece<T, V>((const T*)g + un.lo[k]);
      hi[k] = load_piece<T, V>((const T*)g + un.hi[k]);
    }
  }
};
template <typename T, int V>
__device__ __forceinline__ void to_gamma(bool given, const Piece<T, V>& p, float* f) {
  to_f32(p, f);
  if (!given)
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = 1.f;
}

// A wavefront has a token, or one part of its heads: 64 / lanes heads side by side, BATCH such groups under way, the first ones while the
// angles are computed.  Reads and writes every element once, some 30 operations each: bound by memory (8192 tokens of 84 heads of 152, values moved along,
// 93 us, 4.5 TB/s; 16384 parts at least: with 4096 it took 101) or, for few tokens, by one trip to memory for the position and the vectors and the angle's
// arithmetic (64 tokens of 48 heads of 128: 4.4 us).  A lane has both columns of its pairs, so that nothing is exchanged but the sum of squares.
// Stores that pass the cache by took longer (99 us: a line is written by two wavefronts).
template <typename T, int V, int NU, bool PAIRS>
__global__ __launch_bounds__(64 * QK_WAVES) void qk_fwd_kernel(QkArgs a) {
  constexpr int BATCH = NU * V * sizeof(T) >= 16 ? 2 : 4;
  __shared__ PairTurn pairs[QK_WAVES];
  const int lane = threadIdx.x & 63, per = 64 / a.lanes, sub = lane / a.lanes, wv = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const unsigned wave = blockIdx.x * QK_WAVES + wv;
  const unsigned token = wave / a.parts;
  if (token >= a.tokens) return;
  const int first = wave % a.parts;
  Units<V, NU, PAIRS> un;
  un.place(a, lane);
  const int nq = (a.heads[0] + per - 1) / per, n = nq + (a.heads[1] + per - 1) / per;
  const float inv_d = 1.f / (float)a.d;
  Piece<T, V> lo[BATCH][NU], hi[BATCH][NU];
  auto fetch = [&](int at) {
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int it = at + b * a.parts, seg = it < nq ? 0 : 1, head = (seg ? it - nq : it) * per + sub;
      const T* x = (const T*)a.x[seg] + (size_t)token * a.ld_x[seg] + (size_t)head * a.d;
#pragma unroll
      for (int k = 0; k < NU; ++k) {
        const bool in = it < n && head < a.heads[seg] && un.there[k];
        lo[b][k] = in ? load_piece<T, V>(x + un.lo[k]) : no_piece<T, V>();
        hi[b][k] = in ? load_piece<T, V>(x + un.hi[k]) : no_piece<T, V>();
      }
    }
  };
  Gamma<T, V, NU> gamma[2];
  fetch(first);
  gamma[0].load(a.gamma[0], un);
  gamma[1].load(a.gamma[1], un);
  un.angles(a, lane, token, pairs[wv]);
  int it = first;
  while (it < n) {
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int i = it + b * a.parts;
      if (i >= n) break;
      const int seg = i < nq ? 0 : 1, head = (seg ? i - nq : i) * per + sub;
      T* y = (T*)a.out[seg] + (size_t)token * a.ld_out[seg] + (size_t)head * a.d;
      float p[NU][V], q[NU][V], sum = 0.f;
#pragma unroll
      for (int k = 0; k < NU; ++k) {
        to_f32(lo[b][k], p[k]);
        to_f32(hi[b][k], q[k]);
#pragma unroll
        for (int e = 0; e < V; ++e) sum = fmaf(p[k][e], p[k][e], fmaf(q[k][e], q[k][e], sum));
      }
      const float r = a.norm ? 1.f / sqrtf(fmaf(group_sum(sum, a.lanes), inv_d, a.eps)) : 1.f;
#pragma unroll
      for (int k = 0; k < NU; ++k) {
        float gl[V], gh[V];
        to_gamma(a.gamma[seg] != nullptr, seg ? gamma[1].lo[k] : gamma[0].lo[k], gl);
        to_gamma(a.gamma[seg] != nullptr, seg ? gamma[1].hi[k] : gamma[0].hi[k], gh);
#pragma unroll
        for (int e = 0; e < V; ++e) { p[k][e] *= r * gl[e]; q[k][e] *= r * gh[e]; }
        un.turn(k, p[k], q[k], 1.f);
        if (head < a.heads[seg] && un.there[k]) {
          store_piece(y + un.lo[k], p[k], std::integral_constant<int, V>());
          store_piece(y + un.hi[k], q[k], std::integral_constant<int, V>());
        }
      }
    }
    it += BATCH * a.parts;
    if (it < n) fetch(it);
  }
  // the parts' turns go on through queries, keys and values
  move_values<T, V, NU>(a, un, token, lane, (it - n) % a.parts, a.parts);
}

// A workgroup's wavefronts have a token each, or a part of its heads, and then the next ones; first the queries of all, then the keys, as one sum for
// dgamma takes half the registers of two.  Bound by memory: 16384 tokens of 40 heads of 128 read 320 MB and write 160 in 99 to 101 us, 5.1 TB/s.
template <typename T, int V, int NU, bool PAIRS>
__global__ __launch_bounds__(64 * QK_BWD_WAVES) void qk_bwd_kernel(QkArgs a) {
  __shared__ PairTurn pairs[QK_BWD_WAVES];
  __shared__ float sums[QK_BWD_WAVES][2 * KARMA_QK_D_MAX];
  const int lane = threadIdx.x & 63, per = 64 / a.lanes, sub = lane / a.lanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Units<V, NU, PAIRS> un;
  un.place(a, lane);
  const float inv_d = 1.f / (float)a.d;
  const unsigned waves = gridDim.x * QK_BWD_WAVES, all = a.tokens * (unsigned)a.parts;
  int before = 0;       // groups of heads of the segments before
#pragma unroll 1
  for (int seg = 0; seg < 2; ++seg) {
    const int heads = a.heads[seg], n = (heads + per - 1) / per;
    float sum_lo[NU][V], sum_hi[NU][V];
#pragma unroll
    for (int k = 0; k < NU; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) sum_lo[k][e] = sum_hi[k][e] = 0.f;
    Gamma<T, V, NU> gamma;
    gamma.load(a.gamma[seg], un);
    const bool given = a.gamma[seg] != nullptr;
    for (unsigned w = blockIdx.x * QK_BWD_WAVES + wave; w < all; w += waves) {
      const unsigned token = w / a.parts;
      // the parts' turns go on through queries, keys and values
      int it = (int)((w + (unsigned)a.parts * ((unsigned)before / a.parts + 1) - (unsigned)before) % a.parts);
      if (it >= n) continue;
      const T* x = (const T*)a.x[seg] + (size_t)token * a.ld_x[seg];
      const T* dy = (const T*)a.dy[seg] + (size_t)token * a.ld_dy[seg];
      T* dx = (T*)a.out[seg] + (size_t)token * a.ld_out[seg];
      Piece<T, V> xl[NU], xh[NU], gl[NU], gh[NU];
      auto fetch = [&](int i) {
        const int head = i * per + sub;
        const size_t at = (size_t)head * a.d;
#pragma unroll
        for (int k = 0; k < NU; ++k) {
          const bool in = head < heads && un.there[k];
          gl[k] = in ? load_piece<T, V>(dy + at + un.lo[k]) : no_piece<T, V>();
          gh[k] = in ? load_piece<T, V>(dy + at + un.hi[k]) : no_piece<T, V>();
          xl[k] = in && a.norm ? load_piece<T, V>(x + at + un.lo[k]) : no_piece<T, V>();
          xh[k] = in && a.norm ? load_piece<T, V>(x + at + un.hi[k]) : no_piece<T, V>();
        }
      };
      fetch(it);
      un.angles(a, lane, token, pairs[wave]);
      while (it < n) {
        const int head = it * per + sub;
        const size_t at = (size_t)head * a.d;
        float p[NU][V], q[NU][V], f[NU][V], g[NU][V], sq = 0.f, dot = 0.f;
#pragma unroll
        for (int k = 0; k < NU; ++k) {
          to_f32(xl[k], p[k]);
          to_f32(xh[k], q[k]);
          to_f32(gl[k], f[k]);
          to_f32(gh[k], g[k]);
        }
        // the next group's vectors are on their way while this one is worked on
        it += a.parts;
        if (it < n) fetch(it);
#pragma unroll
        for (int k = 0; k < NU; ++k) {
          float ml[V], mh[V];
          to_gamma(given, gamma.lo[k], ml);
          to_gamma(given, gamma.hi[k], mh);
          un.turn(k, f[k], g[k], -1.f);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            sq = fmaf(p[k][e], p[k][e], fmaf(q[k][e], q[k][e], sq));
            dot = fmaf(f[k][e] * ml[e], p[k][e], fmaf(g[k][e] * mh[e], q[k][e], dot));
          }
        }
        float r = 1.f, back = 0.f;
        if (a.norm) {
          r = 1.f / sqrtf(fmaf(group_sum(sq, a.lanes), inv_d, a.eps));
          back = group_sum(dot, a.lanes) * inv_d * r * r;       // times r x
        }
#pragma unroll
        for (int k = 0; k < NU; ++k) {
          float ml[V], mh[V];
          to_gamma(given, gamma.lo[k], ml);
          to_gamma(given, gamma.hi[k], mh);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float u = r * p[k][e], v = r * q[k][e];
            sum_lo[k][e] = fmaf(f[k][e], u, sum_lo[k][e]);
            sum_hi[k][e] = fmaf(g[k][e], v, sum_hi[k][e]);
            f[k][e] = fmaf(f[k][e] * ml[e], r, -u * back);
            g[k][e] = fmaf(g[k][e] * mh[e], r, -v * back);
          }
          if (head < heads && un.there[k]) {
            store_piece(dx + at + un.lo[k], f[k], std::integral_constant<int, V>());
            store_piece(dx + at + un.hi[k], g[k], std::integral_constant<int, V>());
          }
        }
      }
    }
    before += n;
    if (!a.partial) continue;
    // the groups of lanes that have the same columns
#pragma unroll
    for (int k = 0; k < NU; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float l = sum_lo[k][e], h = sum_hi[k][e];
        for (int m = a.lanes; m < 64; m *= 2) {
          l += __shfl_xor(l, m, 64);
          h += __shfl_xor(h, m, 64);
        }
        if (sub == 0 && un.there[k]) {
          sums[wave][seg * a.d + un.lo[k] + e] = l;
          sums[wave][seg * a.d + un.hi[k] + e] = h;
        }
      }
  }
  for (unsigned w = blockIdx.x * QK_BWD_WAVES + wave; w < all && a.heads[2]; w += waves)
    move_values<T, V, NU>(a, un, w / a.parts, lane, (int)((w + (unsigned)a.parts * ((unsigned)before / a.parts + 1) - (unsigned)before) % a.parts), a.parts);
  if (!a.partial) return;
  // the wavefronts, in a fixed order and in 64 bits
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.d; i += 64 * QK_BWD_WAVES) {
    double v = 0.0;
#pragma unroll
    for (int w = 0; w < QK_BWD_WAVES; ++w) v += sums[w][i];
    a.partial[(size_t)blockIdx.x * 2 * a.d + i] = (float)v;
  }
}

// dgamma from the workgroups' rows: 16 columns a workgroup, 64 groups of rows (512 rows of 256 columns 4.6 us: a launch and two trips to memory).
// Wavefronts and rows are joined in 64 bits, a row is rounded to 32: dgamma of 2331 tokens of 7 heads of 72 is off by 0.8e-7 of itself, joined in 32 bits by
// 1.9e-7, in the same time (19.0 us forward and backward); with lanes joined and rows kept in 64 bits too it took 20.3.  A lane adds up its own terms and
// a wavefront its lanes' in 32 bits: 16384 tokens of 32 heads of 128 are off by 1.4e-7 (2.1e-7 with all joins in 32).
constexpr int DG_COLS = 16, DG_ROWS = 64;
__global__ __launch_bounds__(DG_COLS * DG_ROWS) void qk_dgamma_kernel(const float* partial, int rows, int d, float* dgamma_q, float* dgamma_k) {
  __shared__ double part[DG_ROWS][DG_COLS + 1];
  const int c = threadIdx.x % DG_COLS, g = threadIdx.x / DG_COLS, col = blockIdx.x * DG_COLS + c;
  double v = 0.0;
  if (col < 2 * d) {
#pragma unroll 8
    for (int r = g; r < rows; r += DG_ROWS) v += partial[(size_t)r * 2 * d + col];
  }
  part[g][c] = v;
  __syncthreads();
  if (threadIdx.x < DG_COLS && col < 2 * d) {
    double sum = 0.0;
#pragma unroll
    for (int r = 0; r < DG_ROWS; ++r) sum += part[r][threadIdx.x];
    float* out = col < d ? dgamma_q : dgamma_k;
    if (out) out[col < d ? col : col - d] = (float)sum;
  }
}

bool aligned_to(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

// Workgroups of the backward pass: a row of sums for dgamma each.
constexpr unsigned QK_BWD_GROUPS = 512, QK_PLACES = 16384;
unsigned bwd_groups(uint64_t waves) { return (unsigned)std::min<uint64_t>(QK_BWD_GROUPS, (waves + QK_BWD_WAVES - 1) / QK_BWD_WAVES); }

bool good_shape(const karma_qk_shape& s) {
  if (s.tokens > KARMA_QK_TOKENS_MAX || s.seq > KARMA_QK_TOKENS_MAX || (s.flags & ~3u)) return false;
  if (!s.d || s.d > KARMA_QK_D_MAX || s.d % 2 || s.rot > s.d || s.rot % 2 || (!s.rot && !(s.flags & KARMA_QK_NORM))) return false;
  if (s.heads_q + (uint64_t)s.heads_k == 0 || s.heads_q > KARMA_QK_HEADS_MAX || s.heads_k > KARMA_QK_HEADS_MAX || s.heads_v > KARMA_QK_HEADS_MAX) return false;
  if ((s.flags & KARMA_QK_NORM) && !(s.eps > 0.f && s.eps <= 3.4028234e38f)) return false;
  const uint64_t most = INT64_MAX / 8 / (s.tokens + 1);
  const uint64_t ld[3][3] = {{s.ld_q, s.ld_yq, s.ld_dq}, {s.ld_k, s.ld_yk, s.ld_dk}, {s.ld_v, s.ld_yv, s.ld_dv}};
  const uint64_t heads[3] = {s.heads_q, s.heads_k, s.heads_v};
  for (int k = 0; k < 3; ++k)
    for (uint64_t l : ld[k])
      if (heads[k] && l && (l < heads[k] * s.d || l > most)) return false;
  return true;
}

// How many elements an access has (all pointers, strides and the cut of a head's columns allow it), and how the lanes are dealt.
struct QkCut { int v, nu; };
// Backward a lane has eight columns at most: with sixteen it takes 154 registers (16384 tokens x 40 heads x 128: 132 us, with eight 99).
QkCut cut(const QkArgs& a, bool bf16, bool pairs, bool backward) {
  const size_t e = bf16 ? 2 : 4;
  int v = bf16 && !backward ? 8 : 4;
  auto whole = [&](int v) {
    if (pairs ? a.rot % v || a.d % (2 * v) : a.rot % (2 * v) || (a.d - a.rot) % (2 * v)) return false;
    for (int k = 0; k < 3; ++k) {
      if (!a.heads[k]) continue;
      const bool value = k == 2;
      if ((value || !backward || a.norm) && (!aligned_to(a.x[k], v * e) || a.ld_x[k] % v)) return false;
      if (!aligned_to(a.out[k], v * e) || a.ld_out[k] % v) return false;
      if (!value && backward && (!aligned_to(a.dy[k], v * e) || a.ld_dy[k] % v)) return false;
      if (!value && !aligned_to(a.gamma[k], v * e)) return false;
    }
    return true;
  };
  while (v > 1 && !whole(v)) v /= 2;
  return QkCut{v, a.d / (2 * v) > 64 ? 2 : 1};
}

template <bool BWD, typename T, int V, int NU, bool PAIRS>
void launch_one(const QkArgs& a, unsigned grid, hipStream_t s) {
  if constexpr (BWD) hipLaunchKernelGGL((qk_bwd_kernel<T, V, NU, PAIRS>), dim3(grid), dim3(64 * QK_BWD_WAVES), 0, s, a);
  else hipLaunchKernelGGL((qk_fwd_kernel<T, V, NU, PAIRS>), dim3(grid), dim3(64 * QK_WAVES), 0, s, a);
}
template <bool BWD, bool PAIRS>
void launch_cut(const QkArgs& a, QkCut c, bool bf16, unsigned grid, hipStream_t s) {
  if (bf16) {
    if (c.v == 8) {
      if constexpr (!BWD) launch_one<BWD, bf16_t, 8, 1, PAIRS>(a, grid, s);
    } else if (c.v == 4) launch_one<BWD, bf16_t, 4, 1, PAIRS>(a, grid, s);
    else if (c.v == 2) launch_one<BWD, bf16_t, 2, 1, PAIRS>(a, grid, s);
    else if (c.nu == 1) launch_one<BWD, bf16_t, 1, 1, PAIRS>(a, grid, s);
    else launch_one<BWD, bf16_t, 1, 2, PAIRS>(a, grid, s);
  } else {
    if (c.v == 4) launch_one<BWD, float, 4, 1, PAIRS>(a, grid, s);
    else if (c.v == 2) launch_one<BWD, float, 2, 1, PAIRS>(a, grid, s);
    else if (c.nu == 1) launch_one<BWD, float, 1, 1, PAIRS>(a, grid, s);
    else launch_one<BWD, float, 1, 2, PAIRS>(a, grid, s);
  }
}
// lanes of a head and wavefronts of a token
void deal(QkArgs& a, QkCut c) {
  const int units = a.d / (2 * c.v);
  a.lanes = 1;
  while (a.lanes * c.nu < units) a.lanes *= 2;
  const int per = 64 / a.lanes;
  // (values do not count: whether they are moved changes the order of sums only where they allow narrower accesses than queries and keys do)
  const int rounds = (a.heads[0] + per - 1) / per + (a.heads[1] + per - 1) / per;
  a.parts = (int)std::min<uint64_t>(rounds, std::max<uint64_t>(1, QK_PLACES / std::max(a.tokens, 1u)));
}

}  // namespace

size_t qk_rotary_ws_bytes(const karma_qk_shape& s) {
  if (!good_shape(s)) return 0;
  return s.flags & KARMA_QK_NORM ? (size_t)bwd_groups(std::max<uint64_t>(s.tokens, 1) * QK_PLACES) * 2 * s.d * sizeof(float) : 0;
}

// x, dy and out come with strides of 0 where rows lie one behind the other
static int qk_args(QkArgs& a, const karma_qk_shape& s, bool bf16, bool backward) {
  const size_t e = bf16 ? 2 : 4;
  a.tokens = (unsigned)s.tokens;
  a.seq = (unsigned)(s.seq ? s.seq : std::max<uint64_t>(s.tokens, 1));
  a.heads[0] = (int)s.heads_q; a.heads[1] = (int)s.heads_k; a.heads[2] = (int)s.heads_v;
  a.d = (int)s.d; a.rot = (int)s.rot; a.norm = s.flags & KARMA_QK_NORM ? 1 : 0; a.eps = s.eps;
  for (int k = 0; k < 3; ++k) {
    const size_t row = (size_t)a.heads[k] * s.d;
    if (!a.ld_x[k]) a.ld_x[k] = row;
    if (!a.ld_out[k]) a.ld_out[k] = row;
    if (k < 2 && !a.ld_dy[k]) a.ld_dy[k] = row;
    if (!a.heads[k] || !s.tokens) continue;
    const bool reads_x = k == 2 || !backward || a.norm;
    if (reads_x && (!a.x[k] || !aligned_to(a.x[k], e))) return KARMA_E_INVAL;
    if (!a.out[k] || !aligned_to(a.out[k], e)) return KARMA_E_INVAL;
    if (k < 2 && backward && (!a.dy[k] || !aligned_to(a.dy[k], e))) return KARMA_E_INVAL;
    // in place: a wavefront reads what it writes, and no other one does
    if (reads_x && a.out[k] == a.x[k] && a.ld_out[k] != a.ld_x[k]) return KARMA_E_INVAL;
    if (k < 2 && backward && a.out[k] == a.dy[k] && a.ld_out[k] != a.ld_dy[k]) return KARMA_E_INVAL;
  }
  for (int k = 0; k < 2; ++k) {
    if (a.gamma[k] && (!a.norm || !aligned_to(a.gamma[k], e))) return KARMA_E_INVAL;
    if (!a.heads[k]) a.gamma[k] = nullptr;      // (the kernels read what is given, in pieces whose size the kinds with heads allow)
  }
  if (s.rot && s.tokens && (!a.freq || !aligned_to(a.freq, 8))) return KARMA_E_INVAL;
  if (!aligned_to(a.positions, 4)) return KARMA_E_INVAL;
  // values that are in their place stay there
  if (a.x[2] == a.out[2]) a.heads[2] = 0;
  return KARMA_OK;
}

int qk_rotary_fwd(const void* const* x, const void* const* gamma, const int* positions, const double* freq, void* const* y, const karma_qk_shape& s,
                  bool bf16, hipStream_t stream) {
  if (!good_shape(s)) return KARMA_E_INVAL;
  QkArgs a{{x[0], x[1], x[2]}, {nullptr, nullptr}, {y[0], y[1], y[2]}, {gamma[0], gamma[1]}, nullptr, positions, freq,
           {s.ld_q, s.ld_k, s.ld_v}, {1, 1}, {s.ld_yq, s.ld_yk, s.ld_yv}};
  const int st = qk_args(a, s, bf16, false);
  if (st != KARMA_OK || !s.tokens) return st;
  const QkCut c = cut(a, bf16, s.flags & KARMA_QK_PAIRS, false);
  deal(a, c);
  const unsigned grid = (unsigned)(((uint64_t)a.tokens * a.parts + QK_WAVES - 1) / QK_WAVES);
  if (s.flags & KARMA_QK_PAIRS) launch_cut<false, true>(a, c, bf16, grid, stream);
  else launch_cut<false, false>(a, c, bf16, grid, stream);
  return hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

int qk_rotary_bwd(const void* const* dy, const void* const* x, const void* const* gamma, const int* positions, const double* freq, void* const* dx,
                  float* const* dgamma, const karma_qk_shape& s, void* ws, size_t ws_bytes, bool bf16, hipStream_t stream) {
  if (!good_shape(s)) return KARMA_E_INVAL;
  QkArgs a{{x[0], x[1], dy[2]}, {dy[0], dy[1]}, {dx[0], dx[1], dx[2]}, {gamma[0], gamma[1]}, nullptr, positions, freq,
           {s.ld_q, s.ld_k, s.ld_yv}, {s.ld_yq, s.ld_yk}, {s.ld_dq, s.ld_dk, s.ld_dv}};
  const int st = qk_args(a, s, bf16, true);
  if (st != KARMA_OK) return st;
  const bool sums = dgamma[0] || dgamma[1];
  if (sums && (!a.norm || !aligned_to(dgamma[0], 4) || !aligned_to(dgamma[1], 4))) return KARMA_E_INVAL;
  const QkCut c = cut(a, bf16, s.flags & KARMA_QK_PAIRS, true);
  deal(a, c);
  const unsigned grid = s.tokens ? bwd_groups((uint64_t)a.tokens * a.parts) : 0;
  if (sums) {
    if (!ws || ws_bytes < qk_rotary_ws_bytes(s)) return KARMA_E_OOM;
    if (!aligned_to(ws, 16)) return KARMA_E_INVAL;
    a.partial = (float*)ws;
  }
  if (grid) {
    if (s.flags & KARMA_QK_PAIRS) launch_cut<true, true>(a, c, bf16, grid, stream);
    else launch_cut<true, false>(a, c, bf16, grid, stream);
  }
  if (sums)
    hipLaunchKernelGGL(qk_dgamma_kernel, dim3((2 * a.d + DG_COLS - 1) / DG_COLS), dim3(DG_COLS * DG_ROWS), 0, stream, (const float*)a.partial, (int)grid, a.d,
                       dgamma[0], dgamma[1]);
  return (!grid && !sums) || hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

}  // namespace karma

using namespace karma;

extern "C" uint64_t karma_k_qk_rotary_ws_bytes(const karma_qk_shape* shape) { return shape ? qk_rotary_ws_bytes(*shape) : 0; }

#define KARMA_QK_ENTRIES(SUFFIX, T, BF16)                                                                                                      \
  extern "C" int karma_k_qk_rotary_fwd_##SUFFIX(const T* q, const T* k, const T* v, const T* gamma_q, const T* gamma_k, const int32_t* positions, \
                                                const double* freq, T* yq, T* yk, T* yv, const karma_qk_shape* shape, void* stream) {          \
    if (!shape) return KARMA_E_INVAL;                                                                                                          \
    const void *x[] = {q, k, v}, *gamma[] = {gamma_q, gamma_k};                                                                                \
    void* y[] = {yq, yk, yv};                                                                                                                  \
    return qk_rotary_fwd(x, gamma, positions, freq, y, *shape, BF16, (hipStream_t)stream);                                                     \
  }                                                                                                                                            \
  extern "C" int karma_k_qk_rotary_bwd_##SUFFIX(const T* dyq, const T* dyk, const T* dyv, const T* q, const T* k, const T* gamma_q,            \
                                                const T* gamma_k, const int32_t* positions, const double* freq, T* dq, T* dk, T* dv,           \
                                                float* dgamma_q, float* dgamma_k, const karma_qk_shape* shape, void* ws, uint64_t ws_bytes,    \
                                                void* stream) {                                                                                \
    if (!shape) return KARMA_E_INVAL;                                                                                                          \
    const void *dy[] = {dyq, dyk, dyv}, *x[] = {q, k}, *gamma[] = {gamma_q, gamma_k};                                                          \
    void* dx[] = {dq, dk, dv};                                                                                                                 \
    float* dgamma[] = {dgamma_q, dgamma_k};                                                                                                    \
    return qk_rotary_bwd(dy, x, gamma, positions, freq, dx, dgamma, *shape, ws, ws_bytes, BF16, (hipStream_t)stream);                          \
  }
KARMA_QK_ENTRIES(bf16, void, true)
KARMA_QK_ENTRIES(f32, float, false)
