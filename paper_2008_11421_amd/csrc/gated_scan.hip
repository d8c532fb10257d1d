// Gated linear recurrence over packed sequences, forward and backward:
//   b_t = 1 / (1 + e^f_t)  (one minus the gate's sigmoid),  h_t = h_{t-1} + b_t (x_t - h_{t-1}).
// Gradients, from the last token to the first, with g the gradient of the state behind the token:
//   D_t = dh_t + g,  dx_t = b_t D_t,  df_t = D_t (h_{t-1} - x_t) (b_t - b_t^2),  g = D_t - b_t D_t.
// Of b and a = 1 - b the smaller one is computed, and the other never: rounded to 32 bits it would lose what the smaller one says, how
// long a state lives where b is small, what is left of it where a is.  States and carries are fp32.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_utils.h"
#include "karma.h"
#include "kernels.h"

namespace karma {
namespace {

// ---- a lane's channels -----------------------------------------------------------------------------------------
// V neighbouring channels of one token, raw as loaded: bf16 pairs where everything is on 4-byte boundaries, else one value.
template <typename T, int V>
struct Lane;
template <>
struct Lane<bf16_t, 2> {
  typedef unsigned Raw;
  static __device__ __forceinline__ void get(Raw r, float (&v)[2]) { v[0] = __uint_as_float(r << 16); v[1] = __uint_as_float(r & 0xffff0000u); }
  static __device__ __forceinline__ Raw put(const float (&v)[2]) { return pack2(v[0], v[1]); }
};
template <>
struct Lane<bf16_t, 1> {
  typedef bf16_t Raw;
  static __device__ __forceinline__ void get(Raw r, float (&v)[1]) { v[0] = bf2f(r); }
  static __device__ __forceinline__ Raw put(const float (&v)[1]) { return f2bf(v[0]); }
};
template <>
struct Lane<float, 1> {
  typedef float Raw;
  static __device__ __forceinline__ void get(Raw r, float (&v)[1]) { v[0] = r; }
  static __device__ __forceinline__ Raw put(const float (&v)[1]) { return v[0]; }
};

// The smaller share s = e^-|f| / (1 + e^-|f|) with the gate's sign: s = b where f is positive, -s = a = 1 - b where it is negative (a sign
// of 0 too: both gates of infinity have s = 0).  Then h + b (x - h) is h + s (x - h) or x + s (x - h), and a product with a or b that is
// not s itself is the factor without its share s.
__device__ __forceinline__ float share_of(float f) {
  const float E = __builtin_amdgcn_exp2f(fabsf(f) * -1.44269504f);
  return copysignf(E * __builtin_amdgcn_rcpf(1.f + E), f);
}
// The choice by the sign: a mask of it and a merge of bits, in assembly, as the compiler would make a comparison of them (three places
// more: nothing may read it in the two behind it) and keep all those for a part's later runs, 64 pairs of scalar registers.
__device__ __forceinline__ float by_sign(float s, float positive, float negative) {
  float r;
  asm("v_ashrrev_i32 %0, 31, %1\n\tv_bfi_b32 %0, %0, %3, %2" : "=&v"(r) : "v"(s), "v"(positive), "v"(negative));
  return r;
}
__device__ __forceinline__ float where_positive(float s, float v) {
  float r;
  asm("v_ashrrev_i32 %0, 31, %1\n\tv_bfi_b32 %0, %0, 0, %2" : "=&v"(r) : "v"(s), "v"(v));
  return r;
}
__device__ __forceinline__ float step_of(float s, float x, float h) { return fmaf(s, x - h, by_sign(s, h, x)); }
__device__ __forceinline__ float kept(float s, float v) { return fmaf(-s, v, where_positive(s, v)); }      // a v
// a step of the state h and of the decay A of all steps so far
__device__ __forceinline__ void effect_of(float s, float x, float& h, float& A) {
  float base, rest;
  asm("v_ashrrev_i32 %0, 31, %2\n\tv_bfi_b32 %1, %0, 0, %5\n\tv_bfi_b32 %0, %0, %4, %3"
      : "=&v"(base), "=&v"(rest) : "v"(s), "v"(h), "v"(x), "v"(A));
  h = fmaf(s, x - h, base);
  A = fmaf(-s, A, rest);
}

// The compiler is not to keep what it made of a value that is used again later: the unpacked inputs of two runs through a part, and the
// addresses of all its rows, would take twice the registers (240 instead of 120 in the forward kernel).
template <typename R>
__device__ __forceinline__ R as_new(R r) {
  asm volatile("" : "+v"(r));
  return r;
}
__device__ __forceinline__ int as_new_scalar(int i) {
  asm volatile("" : "+s"(i));
  return i;
}

// ---- sequences -------------------------------------------------------------------------------------------------
struct Spans {
  const int* starts;
  int tokens, sequences, each;      // each: their length where starts is null
  // tokens [first, last) of sequence j; whatever the starts say, no token outside the tensors is touched
  __device__ __forceinline__ int at(int j) const {
    if (!starts) return j * each;
    const int t = starts[j];
    return t < 0 ? 0 : t > tokens ? tokens : t;
  }
  // the last sequence that begins at or before token t (-1: none)
  __device__ __forceinline__ int find(int t) const {
    if (!starts) return t / each;
    int lo = 0, hi = sequences + 1;     // entries below lo are <= t, those from hi on are not
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (at(mid) <= t) lo = mid + 1;
      else hi = mid;
    }
    return lo - 1;
  }
  // from sequence j on to the one that token t begins, or back to the one that token t ends: most often its neighbour, else searched for
  // (any number of sequences without tokens may lie between)
  __device__ __forceinline__ int next(int j, int t) const {
    if (j + 1 < sequences && at(j + 1) <= t) ++j;
    return j + 1 < sequences && at(j + 1) <= t ? find(t) : j;
  }
  __device__ __forceinline__ int previous(int j, int t) const {
    if (j > 0 && at(j) > t) --j;
    return j > 0 && at(j) > t ? find(t) : j;
  }
  __device__ __forceinline__ size_t row(int j, int channels) const { return (size_t)(j < 0 ? 0 : j >= sequences ? sequences - 1 : j) * channels; }
};

// The tokens of a wavefront, t0 .. t0 + L - 1, L <= 32
struct Part {
  unsigned begins;      // tokens that begin a sequence,
  unsigned ends;        // that end one,
  unsigned inside;      // that belong to one
  int seq;              // the last sequence that begins at or before t0
};
// A run of tokens of one sequence: the one that begins with the lowest token left.
__device__ __forceinline__ unsigned first_run(const Part& q, unsigned left) {
  const unsigned later = q.begins & left & (left - 1);      // (the lowest token left, if it begins one, begins this run)
  return later ? left & ((later & -later) - 1) : left;
}
// word: 8 bytes of LDS of the wavefront's own
template <int L>
__device__ __forceinline__ Part part_of(const Spans& p, int t0, unsigned long long* word) {
  const int lane = threadIdx.x & 63;
  unsigned long long bounds = 0;     // bit i: a boundary before token t0 + i, 0 <= i <= L
  Part r;
  r.seq = __builtin_amdgcn_readfirstlane(p.find(t0));
  const int first = __builtin_amdgcn_readfirstlane(p.at(0)), last = __builtin_amdgcn_readfirstlane(p.at(p.sequences));
  if (!p.starts) {
    for (long t = (long)r.seq * p.each; t <= t0 + L && t <= last; t += p.each)
      if (t >= t0) bounds |= 1ull << (t - t0);
  } else {
    if (lane == 0) *word = 0;
    for (int k = r.seq < 0 ? 0 : r.seq; k <= p.sequences; k += 64) {
      const int t = k + lane <= p.sequences ? p.at(k + lane) : INT32_MAX;
      if (t >= t0 && t - t0 <= L) atomicOr(word, 1ull << (t - t0));
      if (__ballot(t - t0 <= L) != ~0ull) break;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    bounds = *word;
    bounds = (unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(bounds >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)bounds);
  }
  const unsigned all = L == 32 ? ~0u : (1u << L) - 1;
  const int lo = first - t0, hi = last - t0;
  r.inside = lo >= L || hi <= 0 ? 0 : (lo > 0 ? all << lo : all) & (hi < L ? (1u << hi) - 1 : all) & all;
  r.begins = (unsigned)bounds & r.inside;
  r.ends = (unsigned)(bounds >> 1) & r.inside;
  return r;
}

// ---- the chain of workgroups ------------------------------------------------------------------------------------
// A chunk of KARMA_SCAN_MARK tokens and some channels belongs to a workgroup.  What it does to the state that comes in is
// out = A in + H; it publishes both at once (8 bytes a channel; A below 0: out = H, a sequence began in it).  Chunks in their order of
// work are in groups of as many as a workgroup has wavefronts: a workgroup looks at all effects of its group before its own at once, a
// wavefront at each, and at the state that the group begins with, which the group before's last workgroup publishes, and runs through
// them in their order: the same sums in the same order every time, and a trip to memory a group, not a chunk.
// Workgroups take their chunks by counters, in the order of work, and wait only for what comes before theirs: for workgroups that have
// begun, whose effects wait for nobody and whose states wait for earlier ones.  So every wait ends, whatever else is on the device and
// however many workgroups find room at once.  A word of all ones is not there yet.  Where a word does not come for a second or so (a
// workspace that another call is using), the states become NaN.
struct Chain {
  unsigned* tickets;            // one for every block of channels, CHAIN_APART numbers from one to the next
  unsigned long long* effect;   // [place in the order of work][block of channels][channel of a lane][lane]
  unsigned* state;              // [group][as above]; the first group begins with zeros
  int chunks, blocks, width;    // blocks of channels, channels of all blocks; chunks == 1: no chain
  int sharing;                  // blocks that share a counter: all or one
};
constexpr int CHAIN_APART = 32;         // 128 bytes: counters of their own cache lines
constexpr int CHAIN_LIMIT = 1 << 20;    // looks at a word, a microsecond or so each
constexpr int CHAIN_GROUP = 8;          // chunks of the smallest groups

template <int V>
__device__ __forceinline__ void publish(const Chain& c, int place, int first, const float (&A)[V], const float (&H)[V], bool cut) {
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const unsigned long long w = (unsigned long long)__float_as_uint(H[e]) << 32 | __float_as_uint(cut ? -1.f : A[e]);
    __hip_atomic_store(c.effect + (size_t)place * c.width + first + e * 64, w == ~0ull ? 0x7fc000007fc00000ull : w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}
// V words from `at` on, 64 apart; those that did not come are all ones, a NaN
template <int V, typename W>
__device__ __forceinline__ void await(const W* at, W (&w)[V]) {
  for (int n = 0; n < CHAIN_LIMIT; ++n) {
    bool missing = false;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      w[e] = __hip_atomic_load(at + e * 64, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      missing |= w[e] == (W)~(W)0;
    }
    if (!__ballot(missing)) break;
    __builtin_amdgcn_s_sleep(1);
  }
}
// what comes before a chunk in its group, in LDS
template <int V, int W>
struct Before {
  float A[W - 1][64 * V], H[W - 1][64 * V], state[64 * V];
};
// Wavefront w's part of it.
template <int V, int W>
__device__ __forceinline__ void look_back(const Chain& c, int place, int first, int w, Before<V, W>& b) {
  const int lane = threadIdx.x & 63, group = place / W;
  if (w < place % W) {
    unsigned long long word[V];
    await<V>(c.effect + (size_t)(group * W + w) * c.width + first, word);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      b.A[w][e * 64 + lane] = __uint_as_float((unsigned)word[e]);
      b.H[w][e * 64 + lane] = __uint_as_float((unsigned)(word[e] >> 32));
    }
  } else if (w == W - 1) {
    unsigned word[V] = {};
    if (group) await<V>(c.state + (size_t)group * c.width + first, word);
#pragma unroll
    for (int e = 0; e < V; ++e) b.state[e * 64 + lane] = __uint_as_float(word[e]);
  }
}
// The state that comes in, when all wavefronts have looked.
template <int V, int W>
__device__ __forceinline__ void run_through(int place, const Before<V, W>& b, float (&in)[V]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int e = 0; e < V; ++e) in[e] = b.state[e * 64 + lane];
  for (int k = 0; k < place % W; ++k)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float A = b.A[k][e * 64 + lane], H = b.H[k][e * 64 + lane];
      in[e] = A < 0.f ? H : fmaf(A, in[e], H);
    }
}
// The last workgroup of a group: the state that the next group begins with.
template <int V, int W>
__device__ __forceinline__ void hand_on(const Chain& c, int place, int first, const float (&out)[V]) {
  if (place % W != W - 1 || place + 1 >= c.chunks) return;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const unsigned u = __float_as_uint(out[e]);
    __hip_atomic_store(c.state + (size_t)(place / W + 1) * c.width + first + e * 64, u == ~0u ? 0x7fc00000u : u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}
// all words behind the counters, widths being multiples of 128
__global__ __launch_bounds__(256) void chain_clear_kernel(Chain c, size_t pieces) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i < (size_t)c.blocks) c.tickets[i * CHAIN_APART] = 0;
  if (i < pieces) ((u32x4*)c.effect)[i] = u32x4{~0u, ~0u, ~0u, ~0u};
}

// The work of this workgroup: a block of channels, and a chunk by its place in the order of work; false: none.
__device__ __forceinline__ bool take_work(const Chain& c, int& place, int& block) {
  __shared__ unsigned ticket;
  const unsigned own = blockIdx.x % c.blocks, first = c.sharing > 1 ? 0 : own;
  place = 0;
  block = own;
  if (c.chunks == 1) return true;
  if (threadIdx.x == 0) ticket = atomicAdd(c.tickets + (size_t)first * CHAIN_APART, 1u);
  __syncthreads();
  const unsigned unit = __builtin_amdgcn_readfirstlane((int)ticket);
  if (unit >= (unsigned)c.sharing * c.chunks) return false;     // (the counter is another call's too)
  place = unit / c.sharing;
  block = first + unit % c.sharing;
  return true;
}

// ---- forward ----------------------------------------------------------------------------------------------------
// W wavefronts have the chunk's tokens one part behind the other, L each, a lane V channels, everything in registers: one pass over
// memory, which bounds long calls (6 bytes an element in bf16 against some 27 issue slots of vector operations, of which the exponential and
// the reciprocal take eight).  Each wavefront runs through its part once for A and H, and, when the state before it is known, again for
// the states.  121 registers: two workgroups on a compute unit, so that one loads while the other waits.  One channel a lane takes 67 us
// instead of 58 for packed prompts.
template <typename T, int V, int L, int W>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(4))) void scan_fwd_kernel(ScanFwd a, Spans p, Chain chain) {
  typedef Lane<T, V> Ln;
  static_assert(L * W == KARMA_SCAN_MARK && W >= CHAIN_GROUP, "a chunk is what lies between two marks; room for the groups' states");
  __shared__ float effects[W][2][64 * V];
  __shared__ Before<V, W> before;
  __shared__ unsigned long long words[W];
  __shared__ int cuts[W];       // 1: a sequence begins in the part, 2: with its first token
  int chunk, block;
  if (!take_work(chain, chunk, block)) return;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), C = (int)a.s.channels;
  const int channel = block * 64 * V + lane * V, c = channel < C ? channel : C - V;     // (lanes without a channel repeat the last one)
  const bool mine = channel < C;
  const int t0 = chunk * KARMA_SCAN_MARK + w * L;
  typename Ln::Raw rf[L], rx[L];
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const size_t t = min(t0 + i, p.tokens - 1);
    rf[i] = *(const typename Ln::Raw*)((const T*)a.gate + t * a.s.ld_gate + c);
    rx[i] = *(const typename Ln::Raw*)((const T*)a.x + t * a.s.ld_x + c);
  }
  const Part q = part_of<L>(p, t0, words + w);
  const unsigned all = L == 32 ? ~0u : (1u << (L & 31)) - 1;
  const bool plain = q.inside == all && !q.begins && !q.ends;
  const int latest = 31 - __builtin_clz(q.begins | 1);      // the last token that begins a sequence, if one does
  auto initial = [&](int j, float (&v)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = a.h0 ? a.h0[p.row(j, C) + c + e] : 0.f;
  };
  // the state that the last sequence to begin here begins with: asked for while the inputs are under way, and kept, as by the second run
  // h_last may lie over it
  float s[L][V], A[V], h[V], begun[V] = {};
  if (q.begins) initial(p.next(q.seq, t0 + latest), begun);
#pragma unroll
  for (int e = 0; e < V; ++e) { A[e] = 1.f; h[e] = 0.f; }
#pragma unroll
  for (int i = 0; i < L; ++i) {
    Ln::get(rf[i], s[i]);
#pragma unroll
    for (int e = 0; e < V; ++e) s[i][e] = share_of(s[i][e]);
  }
  if (plain) {
#pragma unroll
    for (int i = 0; i < L; ++i) {
      float x[V];
      Ln::get(as_new(rx[i]), x);
#pragma unroll
      for (int e = 0; e < V; ++e) effect_of(s[i][e], x[e], h[e], A[e]);
    }
  } else {
    // (what lies before the last beginning has no effect behind the part)
    const unsigned run = q.inside & ~0u << latest;
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = begun[e];
#pragma unroll
    for (int i = 0; i < L; ++i) {
      if (!(run >> i & 1)) continue;
      float x[V];
      Ln::get(as_new(rx[i]), x);
#pragma unroll
      for (int e = 0; e < V; ++e) effect_of(s[i][e], x[e], h[e], A[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e) { effects[w][0][lane * V + e] = A[e]; effects[w][1][lane * V + e] = h[e]; }
  if (lane == 0) cuts[w] = (q.begins ? 1 : 0) | (q.begins & 1 ? 2 : 0);
  __syncthreads();
  // what the wavefronts before this one do together; the first wavefront has the whole chunk's
  float PA[V], PH[V];
  bool cut = false;
#pragma unroll
  for (int e = 0; e < V; ++e) { PA[e] = 1.f; PH[e] = 0.f; }
  for (int k = 0; k < (w == 0 ? W : w); ++k) {
    const bool fresh = cuts[k] & 1;
    cut |= fresh;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float Ak = effects[k][0][lane * V + e], Hk = effects[k][1][lane * V + e];
      PH[e] = fresh ? Hk : fmaf(Ak, PH[e], Hk);
      PA[e] *= Ak;
    }
  }
  float in[V] = {};
  const int words_at = block * 64 * V + lane;
  if (chain.chunks > 1) {
    const bool wants = !(cuts[0] & 2);
    if (w == 0) publish<V>(chain, chunk, words_at, PA, PH, cut);
    if (wants) look_back<V, W>(chain, chunk, words_at, w, before);
    __syncthreads();
    if (wants) run_through<V, W>(chunk, before, in);
  }
#pragma unroll
  for (int e = 0; e < V; ++e) h[e] = cut ? PH[e] : fmaf(PA[e], in[e], PH[e]);
  if (w == 0) {
    if (chain.chunks > 1) hand_on<V, W>(chain, chunk, words_at, h);
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = in[e];
  }
  if (w == 0 && a.marks && mine) {
#pragma unroll
    for (int e = 0; e < V; ++e) a.marks[(size_t)chunk * C + c + e] = h[e];
  }
  auto store = [&](int i) {
    if (mine) *(typename Ln::Raw*)((T*)a.h + (size_t)as_new_scalar(t0 + i) * a.s.ld_h + c) = Ln::put(h);
  };
  if (plain) {
#pragma unroll
    for (int i = 0; i < L; ++i) {
      float x[V];
      Ln::get(as_new(rx[i]), x);
#pragma unroll
      for (int e = 0; e < V; ++e) h[e] = step_of(s[i][e], x[e], h[e]);
      store(i);
    }
  } else {
    int j = q.seq;
    for (unsigned left = q.inside; left;) {
      const unsigned run = first_run(q, left);
      left &= ~run;
      if (q.begins & run) {
        j = p.next(j, t0 + __builtin_ctz(run));
        if (q.begins & left) {
          initial(j, h);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) h[e] = begun[e];
        }
      }
#pragma unroll
      for (int i = 0; i < L; ++i) {
        if (!(run >> i & 1)) continue;
        float x[V];
        Ln::get(as_new(rx[i]), x);
#pragma unroll
        for (int e = 0; e < V; ++e) h[e] = step_of(s[i][e], x[e], h[e]);
        store(i);
      }
      if ((q.ends & run) && a.h_last && mine) {
#pragma unroll
        for (int e = 0; e < V; ++e) a.h_last[p.row(j, C) + c + e] = h[e];
      }
    }
  }
  // sequences without tokens keep their states: each chunk has a share of all sequences
  if (a.h_last && p.starts && mine) {
    const long share = ((long)p.sequences + chain.chunks - 1) / chain.chunks;
    for (long k = chunk * share + w; k < min((long)p.sequences, (chunk + 1) * share); k += W)
      if (p.at((int)k) >= p.at((int)k + 1)) {
#pragma unroll
        for (int e = 0; e < V; ++e) a.h_last[k * C + c + e] = a.h0 ? a.h0[k * C + c + e] : 0.f;
      }
  }
}

// Short sequences (single tokens among them): a wavefront has a whole one.  Here its tokens t0 .. t0 + n - 1, 1 <= n <= L, of which only
// the first can have a mark before it; the last one is read again in place of those behind it.
template <typename T, int V, int L>
__device__ __forceinline__ void short_part(const ScanFwd& a, int t0, int n, unsigned c, float (&h)[V]) {
  typedef typename Lane<T, V>::Raw Raw;
  const T *gate = (const T*)a.gate + (size_t)t0 * a.s.ld_gate, *x = (const T*)a.x + (size_t)t0 * a.s.ld_x;
  T* out = (T*)a.h + (size_t)t0 * a.s.ld_h;
  Raw rf[L], rx[L];
#pragma unroll
  for (int i = 0; i < L; ++i) {
    rf[i] = *(const Raw*)(gate + c);
    rx[i] = *(const Raw*)(x + c);
    if (i + 1 < n) { gate += a.s.ld_gate; x += a.s.ld_x; }
  }
  if (a.marks && t0 % KARMA_SCAN_MARK == 0) {
#pragma unroll
    for (int e = 0; e < V; ++e) a.marks[(size_t)(t0 / KARMA_SCAN_MARK) * a.s.channels + c + e] = h[e];
  }
  float s[L][V];
#pragma unroll
  for (int i = 0; i < L; ++i) {
    Lane<T, V>::get(rf[i], s[i]);
#pragma unroll
    for (int e = 0; e < V; ++e) s[i][e] = share_of(s[i][e]);
  }
  auto step = [&](int i) {
    float in[V];
    Lane<T, V>::get(rx[i], in);
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = step_of(s[i][e], in[e], h[e]);
    *(Raw*)(out + c) = Lane<T, V>::put(h);
    out += a.s.ld_h;
  };
  if (n == L) {
#pragma unroll
    for (int i = 0; i < L; ++i) step(i);
  } else {
#pragma unroll
    for (int i = 0; i < L - 1; ++i)
      if (i < n) step(i);
  }
}
template <typename T, int V>
__global__ __launch_bounds__(256) void scan_fwd_short_kernel(ScanFwd a, Spans p, int blocks, int units) {
  const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (unit >= units) return;
  const int j = unit / blocks, C = (int)a.s.channels, c = (unit % blocks) * 64 * V + (threadIdx.x & 63) * V;
  if (c >= C) return;
  const int first = __builtin_amdgcn_readfirstlane(p.at(j)), last = __builtin_amdgcn_readfirstlane(p.at(j + 1));
  float h[V];
#pragma unroll
  for (int e = 0; e < V; ++e) h[e] = a.h0 ? a.h0[(size_t)j * C + c + e] : 0.f;
  for (int t = first; t < last;) {
    const int n = min(last - t, (int)KARMA_SCAN_MARK - t % (int)KARMA_SCAN_MARK);
    if (n >= 16) short_part<T, V, 16>(a, t, 16, c, h);      // (a copy for what most calls of many tokens take: no test a token)
    else if (n > 4) short_part<T, V, 16>(a, t, n, c, h);
    else short_part<T, V, 4>(a, t, n, c, h);
    t += min(n, 16);
  }
  if (a.h_last) {
#pragma unroll
    for (int e = 0; e < V; ++e) a.h_last[(size_t)j * C + c + e] = h[e];
  }
}

// ---- backward ---------------------------------------------------------------------------------------------------
// As forward, with the chain from the last chunk to the first: the gradient g of the state behind a part goes in, that of the state
// before it comes out, out = A g + R.  The states are run through again from the chunk's mark: 10 bytes an element in bf16 where reading
// h would make 12, and exact.  Three inputs, the shares and the gaps leave room for 16 tokens a wavefront, so the chunk takes 16
// wavefronts; 90 registers, 94 with states (STATES), so that wavefronts of the next chunk begin while the last of this one end: with 32 x
// 1024 tokens of 1024 channels 92 us a call, 94 with room for 128 registers; with states 101, 103.  One channel a lane: 117 and 136.
template <typename T, int V, int L, int W, bool STATES>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(5))) void scan_bwd_kernel(ScanBwd a, Spans p, Chain chain) {
  typedef Lane<T, V> Ln;
  static_assert(L * W == KARMA_SCAN_MARK && W >= CHAIN_GROUP, "a chunk is what lies between two marks; room for the groups' states");
  __shared__ float effects[W][3][64 * V];
  __shared__ Before<V, W> before;
  __shared__ float marks[64 * V];
  __shared__ unsigned long long words[W];
  __shared__ int cuts[W];       // 1: a sequence begins in the part, 2: one ends in it, 4: with its last token
  int place, block;
  if (!take_work(chain, place, block)) return;
  const int chunk = chain.chunks - 1 - place;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), C = (int)a.s.channels;
  const int channel = block * 64 * V + lane * V, c = channel < C ? channel : C - V;
  const bool mine = channel < C;
  const int t0 = chunk * KARMA_SCAN_MARK + w * L;
  typename Ln::Raw rf[L], rx[L], rd[L];
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const size_t t = min(t0 + i, p.tokens - 1);
    rf[i] = *(const typename Ln::Raw*)((const T*)a.gate + t * a.s.ld_gate + c);
    rx[i] = *(const typename Ln::Raw*)((const T*)a.x + t * a.s.ld_x + c);
    rd[i] = *(const typename Ln::Raw*)((const T*)a.dh + t * a.s.ld_h + c);
  }
  if (w == 0) {
#pragma unroll
    for (int e = 0; e < V; ++e) marks[lane * V + e] = a.marks[(size_t)chunk * C + c + e];
  }
  const Part q = part_of<L>(p, t0, words + w);
  float s[L][V], A[V], h[V], g[V];
#pragma unroll
  for (int e = 0; e < V; ++e) { A[e] = 1.f; h[e] = 0.f; g[e] = 0.f; }
#pragma unroll
  for (int i = 0; i < L; ++i) {
    Ln::get(rf[i], s[i]);
#pragma unroll
    for (int e = 0; e < V; ++e) s[i][e] = q.inside >> i & 1 ? share_of(s[i][e]) : 0.f;
  }
  auto initial = [&](int j, float (&v)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = STATES && a.h0 ? a.h0[p.row(j, C) + c + e] : 0.f;
  };
  auto final_gradient = [&](int j, float (&v)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = STATES && a.dh_last ? a.dh_last[p.row(j, C) + c + e] : 0.f;
  };
  auto step = [&](int i) {
    float x[V];
    Ln::get(as_new(rx[i]), x);
#pragma unroll
    for (int e = 0; e < V; ++e) effect_of(s[i][e], x[e], h[e], A[e]);
  };
  auto back = [&](int i) {
    float d[V];
    Ln::get(as_new(rd[i]), d);
#pragma unroll
    for (int e = 0; e < V; ++e) g[e] = kept(s[i][e], d[e] + g[e]);
  };
  // (what lies before the last beginning has no effect on later states, what lies behind the first end none on earlier gradients)
  const int latest = 31 - __builtin_clz(q.begins | 1), earliest = __builtin_ctz(q.ends | 1u << (L - 1));
  int j = q.seq;
  if (STATES && q.begins) j = p.next(j, t0 + latest);
  const int last_seq = j;     // of the part's last token
#pragma unroll
  for (int i = 0; i < L; ++i) {
    if (i == latest && q.begins) initial(j, h);
    step(i);
  }
  if (STATES && q.ends) j = p.previous(j, t0 + earliest);
#pragma unroll
  for (int i = L - 1; i >= 0; --i) {
    if (i == earliest && q.ends) final_gradient(j, g);
    back(i);
  }
#pragma unroll
  for (int e = 0; e < V; ++e) {
    effects[w][0][lane * V + e] = A[e];
    effects[w][1][lane * V + e] = h[e];
    effects[w][2][lane * V + e] = g[e];
  }
  if (lane == 0) cuts[w] = (q.begins ? 1 : 0) | (q.ends ? 2 : 0) | (q.ends >> (L - 1) & 1 ? 4 : 0);
  __syncthreads();
#pragma unroll
  for (int e = 0; e < V; ++e) h[e] = marks[lane * V + e];
  for (int k = 0; k < w; ++k) {
    const bool fresh = cuts[k] & 1;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float Hk = effects[k][1][lane * V + e];
      h[e] = fresh ? Hk : fmaf(effects[k][0][lane * V + e], h[e], Hk);
    }
  }
  // what the wavefronts behind this one do together; the last wavefront has the whole chunk's
  float PA[V], PR[V];
  bool cut = false;
#pragma unroll
  for (int e = 0; e < V; ++e) { PA[e] = 1.f; PR[e] = 0.f; }
  for (int k = W - 1; k > (w == W - 1 ? -1 : w); --k) {
    const bool fresh = cuts[k] & 2;
    cut |= fresh;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float Ak = effects[k][0][lane * V + e], Rk = effects[k][2][lane * V + e];
      PR[e] = fresh ? Rk : fmaf(Ak, PR[e], Rk);
      PA[e] *= Ak;
    }
  }
  float in[V] = {};
  const int words_at = block * 64 * V + lane;
  if (chain.chunks > 1) {
    const bool wants = !(cuts[W - 1] & 4);
    if (w == W - 1) publish<V>(chain, place, words_at, PA, PR, cut);
    if (wants) look_back<V, W>(chain, place, words_at, w, before);
    __syncthreads();
    if (wants) run_through<V, W>(place, before, in);
  }
#pragma unroll
  for (int e = 0; e < V; ++e) g[e] = cut ? PR[e] : fmaf(PA[e], in[e], PR[e]);
  if (w == W - 1) {
    if (chain.chunks > 1) hand_on<V, W>(chain, place, words_at, g);
#pragma unroll
    for (int e = 0; e < V; ++e) g[e] = in[e];
  }
  float gap[L][V];      // h_{t-1} - x_t
  auto part_from = [&](int i) {
    float x[V];
    Ln::get(as_new(rx[i]), x);
#pragma unroll
    for (int e = 0; e < V; ++e) { gap[i][e] = as_new(h[e] - x[e]); h[e] = fmaf(-s[i][e], gap[i][e], by_sign(s[i][e], h[e], x[e])); }
  };
  auto finish = [&](int i) {
    float d[V], dx[V], df[V];
    Ln::get(as_new(rd[i]), d);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float D = d[e] + g[e];
      const float own = as_new(s[i][e]), rest = where_positive(own, D);     // (as above: the product that follows)
      dx[e] = fmaf(own, D, D - rest);      // b D
      df[e] = D * gap[i][e] * fmaf(-own, own, fabsf(own));
      g[e] = fmaf(-own, D, rest);          // a D
    }
    if (!mine || !(q.inside >> i & 1)) return;
    const size_t t = as_new_scalar(t0 + i);
    *(typename Ln::Raw*)((T*)a.dx + t * a.s.ld_dx + c) = Ln::put(dx);
    *(typename Ln::Raw*)((T*)a.dgate + t * a.s.ld_dgate + c) = Ln::put(df);
  };
  j = q.seq;
#pragma unroll
  for (int i = 0; i < L; ++i) {
    if (q.begins >> i & 1) {
      if (STATES) j = p.next(j, t0 + i);
      initial(j, h);
    }
    part_from(i);
  }
  j = last_seq;
#pragma unroll
  for (int i = L - 1; i >= 0; --i) {
    if (q.ends >> i & 1) {
      if (STATES) j = p.previous(j, t0 + i);
      final_gradient(j, g);
    }
    finish(i);
    if (STATES && (q.begins >> i & 1) && a.dh0 && mine) {
      j = p.previous(j, t0 + i);
#pragma unroll
      for (int e = 0; e < V; ++e) a.dh0[p.row(j, C) + c + e] = g[e];
    }
  }
  if (STATES && a.dh0 && p.starts && mine) {
    const long share = ((long)p.sequences + chain.chunks - 1) / chain.chunks;
    for (long k = chunk * share + w; k < min((long)p.sequences, (chunk + 1) * share); k += W)
      if (p.at((int)k) >= p.at((int)k + 1)) {
#pragma unroll
        for (int e = 0; e < V; ++e) a.dh0[k * C + c + e] = a.dh_last ? a.dh_last[k * C + c + e] : 0.f;
      }
  }
}

__global__ void copy_or_zero_kernel(const float* x, float* y, size_t n) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) y[i] = x ? x[i] : 0.f;
}

// Whether wavefronts take whole sequences (`units` of them), at 0.11 us a token where they are few.  Sequences of one length, 1024 channels
// in bf16, us a call by whole sequences / in chunks: 4096 x 1 token 13.8 / 38.9; in a single chunk 1 x 96 11.3 / 12.1, 1 x 128 14.7 / 12.1;
// 16 x 128 15.0 / 16.3, 16 x 160 18.5 / 18.1; with 512 units (8 a sequence here) 64 x 192 23.0 / 27.0, 64 x 256 29.4 / 26.8; with 1024
// 128 x 256 34.5 / 49.3, 128 x 512 86 / 103.  Of packed ones nobody here knows the longest: up to 512 tokens more than sequences, of which it
// can have 513 at most.  64 x 8 5.3 / 19.9, 63 x 1 and one of 300 32.3 / 37.1, of 512 53.4 / 36.8, of 1900 189 / 37.3.
bool whole_sequences(const karma_scan_shape& s, bool packed, uint64_t units) {
  if (packed) return s.tokens <= s.sequences + 512ull && s.tokens <= 128ull * s.sequences;
  const uint64_t most = units >= 1024 ? 512 : units >= 512 ? 192 : s.tokens > KARMA_SCAN_MARK ? 128 : 96;
  return s.tokens <= most * s.sequences;
}

// chunks of a call; channels of all blocks whatever a lane has
uint64_t scan_chunks(uint64_t tokens) { return std::max<uint64_t>(1, (tokens + KARMA_SCAN_MARK - 1) / KARMA_SCAN_MARK); }
uint64_t scan_width(uint32_t channels) { return ((uint64_t)channels + 127) / 128 * 128; }

// Sizes and strides as a call may give them; a stride of 0 becomes the number of channels.
int check_scan(karma_scan_shape& s, const void* starts) {
  if (!s.channels || !s.sequences || s.tokens > INT32_MAX - 1024 || s.channels > INT32_MAX || s.sequences >= INT32_MAX) return KARMA_E_INVAL;
  if (!starts && s.tokens % s.sequences) return KARMA_E_INVAL;
  for (uint64_t* ld : {&s.ld_gate, &s.ld_x, &s.ld_h, &s.ld_dgate, &s.ld_dx}) {
    if (!*ld) *ld = s.channels;
    if (*ld < s.channels || *ld > INT64_MAX / 8 / (s.tokens + 1)) return KARMA_E_INVAL;
  }
  // a launch has less than 2^32 lanes: 64 for a sequence's block of channels, 1024 for a chunk's
  const uint64_t blocks = ((uint64_t)s.channels + 63) / 64;
  if (blocks * s.sequences > (1u << 26) - 4 || blocks * (scan_chunks(s.tokens) + 1) >= 1u << 22) return KARMA_E_INVAL;
  return KARMA_OK;
}
bool aligned_to(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

}  // namespace

// the counters of blocks of 64 channels, which are the more
static size_t chain_head(uint64_t width) { return width / 64 * CHAIN_APART * sizeof(unsigned); }
// effects, and states of the smallest groups
static size_t chain_words(uint64_t chunks, uint64_t width) { return (chunks * 8 + (chunks + CHAIN_GROUP - 1) / CHAIN_GROUP * 4) * width; }

size_t gated_scan_ws_bytes(const karma_scan_shape& given) {
  karma_scan_shape shape = given;
  const int any = 0;      // (whether all sequences have one length does not matter here)
  if (check_scan(shape, &any)) return 0;
  const uint64_t chunks = scan_chunks(shape.tokens), width = scan_width(shape.channels);
  return chunks > 1 ? chain_head(width) + chain_words(chunks, width) : 0;
}

static Spans spans_of(const karma_scan_shape& s, const int* starts) {
  return Spans{starts, (int)s.tokens, (int)s.sequences, starts ? 0 : (int)(s.tokens / s.sequences)};
}
// V channels a lane; the chain is cleared by a kernel ahead (a call that is captured has kernels alone).  One counter for all blocks of
// channels, or one each?  512 workgroups that begin at once wait some microseconds for one counter; from then on workgroups
// gain by not loading all at the same time, which one counter sees to.  So forward from 2048 workgroups on, four times what runs at
// once (one / each, us a call: 65536 x 2048 163 / 181, 32768 x 2048 95 / 97, 16384 x 2048 60 / 56, packed prompts 60 / 58; fp32
// 65536 x 2048 297 / 326, 32768 x 1024 90 / 92, 65536 x 256 64 / 59), and backward always (32 x 1024 x 1024 92 / 94, 32768 x 2048 164 / 171).
static Chain chain_of(const karma_scan_shape& s, int V, bool forward, void* ws, hipStream_t stream) {
  const uint64_t chunks = scan_chunks(s.tokens), width = scan_width(s.channels), blocks = ((uint64_t)s.channels + 64 * V - 1) / (64 * V);
  unsigned long long* effect = (unsigned long long*)((char*)ws + chain_head(width));
  const Chain c{(unsigned*)ws, effect, (unsigned*)(effect + chunks * width), (int)chunks, (int)blocks, (int)width,
                forward && blocks * chunks < 2048 ? 1 : (int)blocks};
  const size_t pieces = chain_words(chunks, width) / 16;
  if (chunks > 1) hipLaunchKernelGGL(chain_clear_kernel, dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, stream, c, pieces);
  return c;
}
static unsigned chain_grid(const Chain& c) { return (unsigned)c.blocks * (unsigned)c.chunks; }

int gated_scan_fwd(ScanFwd a, bool bf16, hipStream_t s) {
  const size_t e = bf16 ? 2 : 4;
  if (int st = check_scan(a.s, a.starts)) return st;
  if (a.s.tokens && (!a.gate || !a.x || !a.h)) return KARMA_E_INVAL;
  if (!aligned_to(a.gate, e) || !aligned_to(a.x, e) || !aligned_to(a.h, e) || !aligned_to(a.ws, 16)) return KARMA_E_INVAL;
  if (!aligned_to(a.h0, 4) || !aligned_to(a.starts, 4) || !aligned_to(a.h_last, 4) || !aligned_to(a.marks, 4)) return KARMA_E_INVAL;
  if (a.ws_bytes < gated_scan_ws_bytes(a.s)) return KARMA_E_OOM;
  const bool pairs = bf16 && a.s.channels % 2 == 0 && (a.s.ld_gate | a.s.ld_x | a.s.ld_h) % 2 == 0 && aligned_to(a.gate, 4) && aligned_to(a.x, 4) &&
                     aligned_to(a.h, 4);
  const Spans p = spans_of(a.s, a.starts);
  const int blocks = (int)((a.s.channels + (pairs ? 127 : 63)) / (pairs ? 128 : 64)), units = blocks * (int)a.s.sequences;
  if (whole_sequences(a.s, a.starts != nullptr, units)) {
    const dim3 grid((units + 3) / 4);
    if (pairs) hipLaunchKernelGGL((scan_fwd_short_kernel<bf16_t, 2>), grid, dim3(256), 0, s, a, p, blocks, units);
    else if (bf16) hipLaunchKernelGGL((scan_fwd_short_kernel<bf16_t, 1>), grid, dim3(256), 0, s, a, p, blocks, units);
    else hipLaunchKernelGGL((scan_fwd_short_kernel<float, 1>), grid, dim3(256), 0, s, a, p, blocks, units);
  } else {
    const Chain c = chain_of(a.s, pairs ? 2 : 1, true, a.ws, s);
    const dim3 grid(chain_grid(c));
    if (pairs) hipLaunchKernelGGL((scan_fwd_kernel<bf16_t, 2, 32, 8>), grid, dim3(512), 0, s, a, p, c);
    else if (bf16) hipLaunchKernelGGL((scan_fwd_kernel<bf16_t, 1, 32, 8>), grid, dim3(512), 0, s, a, p, c);
    else hipLaunchKernelGGL((scan_fwd_kernel<float, 1, 32, 8>), grid, dim3(512), 0, s, a, p, c);
  }
  return hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
}

int gated_scan_bwd(ScanBwd a, bool bf16, hipStream_t s) {
  const size_t e = bf16 ? 2 : 4;
  if (int st = check_scan(a.s, a.starts)) return st;
  if (a.s.tokens && (!a.gate || !a.x || !a.marks || !a.dh || !a.dgate || !a.dx)) return KARMA_E_INVAL;
  if (!aligned_to(a.gate, e) || !aligned_to(a.x, e) || !aligned_to(a.dh, e) || !aligned_to(a.dgate, e) || !aligned_to(a.dx, e) ||
      !aligned_to(a.ws, 16)) return KARMA_E_INVAL;
  if (!aligned_to(a.h0, 4) || !aligned_to(a.starts, 4) || !aligned_to(a.marks, 4) || !aligned_to(a.dh_last, 4) || !aligned_to(a.dh0, 4)) return KARMA_E_INVAL;
  if (a.ws_bytes < gated_scan_ws_bytes(a.s)) return KARMA_E_OOM;
  if (!a.s.tokens) {      // the gradient of a state that no token changed
    if (!a.dh0) return KARMA_OK;
    const size_t n = (size_t)a.s.sequences * a.s.channels;
    hipLaunchKernelGGL(copy_or_zero_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a.dh_last, a.dh0, n);
    return hipGetLastError() == hipSuccess ? KARMA_OK : KARMA_E_HIP;
  }
  const bool pairs = bf16 && a.s.channels % 2 == 0 && (a.s.ld_gate | a.s.ld_x | a.s.ld_h | a.s.ld_dgate | a.s.ld_dx) % 2 == 0 &&
                     aligned_to(a.gate, 4) && aligned_to(a.x, 4) && aligned_to(a.dh, 4) && aligned_to(a.dgate, 4) && aligned_to(a.dx, 4);
  const Spans p = spans_of(a.s, a.starts);
  const Chain c = chain_of(a.s, pairs ? 2 : 1, false, a.ws, s);
  const dim3 grid(chain_grid(c));
#define KARMA_SCAN_BWD(T, V)                                                                                           \
  do {                                                                                                                 \
    if (states) hipLaunchKernelGGL((scan_bwd_kernel<T, V, 16, 16, true>), grid, dim3(1024), 0, s, a, p, c);            \
    else hipLaunchKernelGGL((scan_bwd_kernel<T, V, 16, 16, false>), grid, dim3(1024), 0, s, a, p, c);                  \
  } while (0)
  const bool states = a.h0 || a.dh_last || a.dh0;
  if (pairs) KARMA_SCAN_BWD(bf16_t, 2);
  else if (bf16) KARMA_SCAN_BWD(bf16_t, 1);
  else KARMA_SCAN_BWD(float, 1);
#undef KARMA_SCAN_BWD
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
