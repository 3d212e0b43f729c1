// Log probabilities of given tokens, the entropy of their rows, and the likeliest
// alternatives, from one read of each logit row.
//
// With c = log2(e) / T, a maximum M of the logits z, S = sum 2^(c (z - M)) and
// W = sum 2^(c (z - M)) (z - M):
//   ln p(x) = ln 2 (c (z_x - M) - log2 S),   H = ln 2 (log2 S - c W / S).
// (The difference comes first, so rows of the type's lowest value overflow nothing.)
// A thread walks the 16-byte pieces of its row (or of its part of it) that lie a
// workgroup's width apart, and keeps its own maximum, sums, the piece where its
// maximum first stood, and its maximum in each of eight segments of the walk.  Of all
// threads the n with the largest (maximum, then earliest piece) hold the n largest
// logits between them: were one elsewhere, its thread's maximum would be among the n.
// A bound that those n reach (and some more threads: it comes from a bisection by
// ballots over one wave's registers, which ends where it lets through enough and not
// many more) names the segments of theirs that have to be read again, and of those
// only values that reach it count, mostly little more than n, which are ranked by
// counting.  (A piece is alone in its cache line for its thread: without the segments,
// 33 threads' walks for n = 20 are as much traffic as the row.)
//
// Few rows are cut into parts, each with a list of its n largest; the workgroup that
// finishes a row's last part joins them.  What it reads of the others was written
// through device-scope stores that had completed before the row's ticket was drawn.

#include "ent_internal.h"

#include <math.h>

#include <algorithm>

namespace ent {
namespace {

constexpr int kLpThreads = 256;
constexpr int kLpTop = ENT_MAX_TOP_LOGPROBS;
constexpr int kLpCand = 1024;         // candidates that are ranked at once (a wave alone: a quarter)
constexpr int kLpParts = 64;          // parts of a row, at most
constexpr int kLpWho = 64;            // threads that can reach the bound
constexpr int kLpSegs = 8;            // segments of a thread's walk
static_assert(kLpTop * kLpTop <= kLpCand, "keys of a row's n lists");
static_assert(kLpTop + kLpTop / 4 + 2 <= kLpWho, "threads over the bound");
static_assert(kLpParts == 64 && 2 * kLpParts <= kLpThreads, "a wave of lanes for the parts, and another");
typedef unsigned long long u64;

struct LpArgs {
  const void* logits;
  long long ld;
  int T, V, n_top, parts;
  const int* tokens;      // nullable
  const float* temp;      // nullable
  float t_cal;
  float* logprob;         // nullable
  float* entropy;         // nullable
  int* top_ids;
  float* top_lp;
  float* sums;            // [T * parts, 3]  (max, S, W) of parts
  u64* keys;              // [T * parts, n_top]  their largest logits, descending
  unsigned* tickets;      // [T]  finished parts, 0 between launches
  unsigned* flags;
};

// A logit and its index as one number: larger logit first, then lower index; 0 is none.
__device__ __forceinline__ unsigned lp_order(float x) {
  const unsigned u = __float_as_uint(x + 0.f);       // -0 as 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float lp_value(unsigned o) {
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ u64 lp_key(float x, int i) {
  return static_cast<u64>(lp_order(x)) << 32 | ~static_cast<unsigned>(i);
}

// A row's 16-byte pieces: piece p holds the elements [p N - shift, p N - shift + N)
// that lie in [0, V), so that pieces are aligned whatever the row's start.
template <typename T, bool STREAM>
struct Row {
  static constexpr int N = 16 / sizeof(T);
  static constexpr int kDrop = 32 - 8 * static_cast<int>(sizeof(T));
  const T* base;     // the row's first element
  int shift, V;
  __device__ __forceinline__ Row(const T* b, int v) : base(b), shift(static_cast<int>((reinterpret_cast<uintptr_t>(b) & 15) / sizeof(T))), V(v) {}
  __device__ __forceinline__ int pieces() const { return (V + shift + N - 1) / N; }
  static __device__ __forceinline__ float value(float x) { return x; }
  static __device__ __forceinline__ float value(uint16_t x) { return bf16_to_f32(x); }
  static __device__ __forceinline__ void widen(uint4 v, float (&x)[N]) {
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (N == 4) {
        x[i] = __uint_as_float(w[i]);
      } else {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ bool whole(int p) const { return p * N >= shift && (p + 1) * N - shift <= V; }
  __device__ __forceinline__ uint4 raw(int p) const {
    return load16<STREAM>(base + (static_cast<long long>(p) * N - shift));
  }
  // Any piece; elements outside the row read as -inf.
  __device__ __forceinline__ uint4 piece(int p) const {
    if (whole(p)) return raw(p);
    unsigned w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      constexpr int E = N / 4;                             // elements of a word
      w[j] = 0u;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = p * N + j * E + e - shift;
        unsigned bits = N == 4 ? 0xff800000u : 0xff80u;
        if (i >= 0 && i < V) {
          if constexpr (N == 4) bits = __float_as_uint(base[i]);
          else bits = base[i];
        }
        w[j] |= bits << (32 / E * e);
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void load(int p, float (&x)[N]) const { widen(piece(p), x); }
  static __device__ __forceinline__ uint4 nothing() {
    const unsigned w = N == 4 ? 0xff800000u : 0xff80ff80u;
    return make_uint4(w, w, w, w);
  }
};

// Sums relative to a maximum m of the logits (m = -inf: s = w = 0).
struct LpSums {
  float m, s, w;
};
// The scale c, and a difference from where on 2^(c d) is 0 (finite: 0 times it is 0).
struct LpScale {
  float c, low;
  __device__ __forceinline__ LpScale(const LpArgs& a, int row)
      : c(__fdiv_rn(kLog2e, (a.temp ? a.temp[row] : 1.f) * a.t_cal)), low(fmaxf(__fdividef(-200.f, c), -1e38f)) {}
};
__device__ __forceinline__ LpSums lp_to(const LpSums& a, float m, const LpScale& sc) {
  if (a.m == -INFINITY) return LpSums{m, a.s, a.w};          // 0, or the NaN of a row that has one
  const float d = a.m - m, f = __builtin_amdgcn_exp2f(d * sc.c);
  return LpSums{m, a.s * f, f * (a.w + a.s * fmaxf(d, sc.low))};
}
// The row's entropy and token; m and l (= log2 S) are what its other outputs are made of.
__device__ __forceinline__ void lp_outputs(const LpArgs& a, int row, const LpSums& t, float c, int tok, float z,
                                           float& m, float& l) {
  // Neither NaN nor +inf, and something besides -inf.
  const bool ok = t.s > 0.f && t.s < INFINITY && t.m < INFINITY;
  m = ok ? t.m : NAN;
  l = ok ? log2f(t.s) : NAN;
  if (a.entropy) a.entropy[row] = (l - c * (t.w / t.s)) * kLn2;
  if (a.logprob) a.logprob[row] = tok < a.V ? ((z - m) * c - l) * kLn2 : NAN;
  if (tok >= a.V) raise_flag(a.flags, ENT_DEV_BAD_TOKEN);
}
__device__ __forceinline__ void lp_write_top(const LpArgs& a, int row, int i, u64 key, float c, float m, float l) {
  const long long o = static_cast<long long>(row) * a.n_top + i;
  const float x = lp_value(static_cast<unsigned>(key >> 32));
  a.top_ids[o] = l == l ? static_cast<int>(~static_cast<unsigned>(key)) : -1;
  a.top_lp[o] = ((x - m) * c - l) * kLn2;
}

// Values that another workgroup of the launch reads.
template <typename V>
__device__ __forceinline__ void lp_share(V* p, V v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename V>
__device__ __forceinline__ V lp_shared(const V* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int NT>
struct LpShared {
  static constexpr int kCand = NT == kLpThreads ? kLpCand : kLpCand / 4;
  u64 key[NT];               // per thread: its largest logit (of its maxima, first piece)
  union {
    float seg[kLpSegs][NT];         // ... in each segment, until `again` is made of it
    u64 cand[kCand];
  };
  float red[3 * NT / 64];
  int again[kLpWho * kLpSegs];      // (segment, thread) that are read again
  u64 edge;
  int count, agains, last;
  float ml[2];
};

// A bound that at least n of a wave's keys (K a lane, distinct but for 0, which is none)
// reach, and at most `most` >= n of them: by bisection, first over the upper words, then,
// where too many share the n-th's, over the lower words of those.  All keys but 0 where
// they are no more than `most`, and anything where they are fewer than n.  DROP: bits of
// the upper words that no two logits differ in alone (16 for bf16).
template <int DROP, int K>
__device__ __forceinline__ u64 lp_bound(const u64 (&key)[K], int n, int most) {
  unsigned hi[K], top = 0u, least = 0xffffffffu;
  int there = 0;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    hi[k] = static_cast<unsigned>(key[k] >> 32) >> DROP;
    top = max(top, hi[k]);
    if (key[k] != 0ull) least = min(least, hi[k]);
    there += static_cast<int>(__popcll(__ballot(key[k] != 0ull)));
  }
  if (there <= most) return there < n ? 1ull : static_cast<u64>(wave_min_u(least)) << (32 + DROP);
  auto count = [&](unsigned from) {
    int c = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) c += static_cast<int>(__popcll(__ballot(hi[k] >= from)));
    return c;
  };
  // All keys but 0 reach `lo`, which grows while n do; fewer than n reach `end`.  Where
  // no lane is empty, each lane's largest reaches the least of them.
  unsigned lo = max(wave_min_u(top), 1u), end = wave_max_u(top) + 1u;
  lo = __builtin_amdgcn_readfirstlane(lo);
  end = __builtin_amdgcn_readfirstlane(end);
  int c = count(lo);
  while (c > most && end - lo > 1u) {
    const unsigned mid = lo + (end - lo) / 2u;
    const int m = count(mid);
    if (m >= n) {
      lo = mid;
      c = m;
    } else {
      end = mid;
    }
  }
  if (c <= most) return static_cast<u64>(lo) << (32 + DROP);
  // Too many at lo itself: the largest lower words among them.
  const int need = n - count(lo + 1u);
  auto ties = [&](unsigned from) {
    int t = 0;
#pragma unroll
    for (int k = 0; k < K; ++k)
      t += static_cast<int>(__popcll(__ballot(hi[k] == lo && static_cast<unsigned>(key[k]) >= from)));
    return t;
  };
  unsigned first = 0xffffffffu, last = 0u, same = 0u;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (hi[k] == lo) {
      same = static_cast<unsigned>(key[k] >> 32);
      first = min(first, static_cast<unsigned>(key[k]));
      last = max(last, static_cast<unsigned>(key[k]));
    }
  }
  unsigned low = wave_min_u(first), past = wave_max_u(last);   // at least `need` reach low
  low = __builtin_amdgcn_readfirstlane(low);
  past = __builtin_amdgcn_readfirstlane(past);
  same = wave_max_u(same);                     // the upper word that they share
  if (ties(past) >= need) return static_cast<u64>(same) << 32 | past;
  while (past - low > 1u) {
    const unsigned mid = low + (past - low) / 2u;
    if (ties(mid) >= need) low = mid;
    else past = mid;
  }
  return static_cast<u64>(same) << 32 | low;
}

// The n largest of sh.cand[0 .. cand) by counting: f(rank, key).
template <int NT, typename F>
__device__ __forceinline__ void lp_rank(const LpShared<NT>& sh, int cand, int n, F f) {
  for (int i = threadIdx.x; i < cand; i += NT) {
    const u64 mine = sh.cand[i];
    int rank = 0;
    for (int k = 0; k < cand; ++k) rank += sh.cand[k] > mine ? 1 : 0;
    if (rank < n) f(rank, mine);
  }
}

// The n largest logits of pieces [p0, p1), `per` pieces of a thread in a segment, given
// the threads' largest in sh.key and sh.seg.
template <typename R, int NT>
__device__ __forceinline__ void lp_largest(const LpArgs& a, LpShared<NT>& sh, const R& r, int p0, int p1, int per,
                                           int row, float c) {
  constexpr int N = R::N;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, n = a.n_top;
  const bool whole = a.parts == 1;
  auto put = [&](int rank, u64 key) {
    if (whole) lp_write_top(a, row, rank, key, c, sh.ml[0], sh.ml[1]);
    else lp_share(a.keys + static_cast<long long>(blockIdx.x) * n + rank, key);
  };
  // Threads whose largest logits are among the n largest of the threads', and some more.
  if (wave == 0) {
    u64 key[NT / 64];
#pragma unroll
    for (int k = 0; k < NT / 64; ++k) key[k] = sh.key[k * 64 + lane];
    const u64 e = lp_bound<R::kDrop>(key, n, n + n / 4 + 2);
    if (lane == 0) sh.edge = e;
  }
  __syncthreads();
  const u64 edge = sh.edge;
  const unsigned eo = static_cast<unsigned>(edge >> 32);
  const int ep = static_cast<unsigned>(edge) == 0u || eo == 0u ? 0x7fffffff : static_cast<int>(~static_cast<unsigned>(edge));
  if (sh.key[t] >= edge) {
#pragma unroll
    for (int g = 0; g < kLpSegs; ++g)
      if (p0 + t + g * per * NT < p1 && lp_order(sh.seg[g][t]) >= eo) sh.again[atomicAdd(&sh.agains, 1)] = g * NT + t;
  }
  __syncthreads();
  const int units = sh.agains * per;
  // Whether element (x, i) of piece p can be among the n largest.
  auto counts = [&](float x, int i, int p) {
    const unsigned o = lp_order(x);
    return i >= 0 && i < a.V && x == x && (o > eo || (o == eo && p <= ep));
  };
  for (int u = t; u < units; u += NT) {
    const int w = sh.again[u / per], p = p0 + w % NT + (w / NT * per + u % per) * NT;
    if (p < p1) {
      float x[N];
      r.load(p, x);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int i = p * N + j - r.shift;
        if (counts(x[j], i, p)) {
          const int at = atomicAdd(&sh.count, 1);
          if (at < sh.kCand) sh.cand[at] = lp_key(x[j], i);
        }
      }
    }
  }
  __syncthreads();
  const int cand = sh.count;
  if (cand <= sh.kCand) {
    lp_rank(sh, cand, n, put);
    // A part shorter than n, or a row with NaN.
    for (int i = cand + t; i < n; i += NT) put(i, 0ull);
    return;
  }
  // Rows whose largest logits crowd a few threads: one after the other, each the
  // largest key below the last.
  u64 last = ~0ull;
  for (int k = 0; k < n; ++k) {
    u64 best = 0ull;
    for (int p = p0 + t; p < p1; p += NT) {
      float x[N];
      r.load(p, x);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int i = p * N + j - r.shift;
        if (i >= 0 && i < a.V) {
          const u64 key = lp_key(x[j], i);
          if (key < last && key > best) best = key;
        }
      }
    }
    __syncthreads();
    sh.key[t] = best;
    __syncthreads();
    best = 0ull;
    for (int i = 0; i < NT; ++i) best = sh.key[i] > best ? sh.key[i] : best;
    if (t == 0) put(k, best);
    last = best;
  }
}

// A row's outputs from its parts' sums and descending lists, by one workgroup.  A bound
// that n keys reach: the n-th largest of the lists' first keys, or, of fewer lists, the
// least of their q-th, where q entries of each are n.
template <int DROP>
__device__ __forceinline__ void lp_join(const LpArgs& a, LpShared<kLpThreads>& sh, int row, const LpScale& sc, int tok,
                                        float z) {
  constexpr int NT = kLpThreads, K = kLpParts * kLpTop / NT;
  const int t = threadIdx.x, n = a.n_top, total = a.parts * n;
  const long long first = static_cast<long long>(row) * a.parts;
  const u64* keys = a.keys + first * n;
  u64 mine[K];
#pragma unroll
  for (int k = 0; k < K; ++k) mine[k] = t + k * NT < total ? lp_shared(keys + t + k * NT) : 0ull;
  if (t < 64) {
    // The bound, while the next wave forms the row's sums.
    if (t == 0) sh.count = 0;
    if (n > 0) {
      const int q = (n + a.parts - 1) / a.parts;
      u64 head = 0ull, e;                  // of the list, or its q-th key
      if (t < a.parts) head = lp_shared(keys + static_cast<long long>(t) * n + q - 1);
      if (q == 1) {
        const u64 one[1] = {head};
        e = lp_bound<DROP>(one, n, min(n + 3, kLpCand / n));    // lists whose keys all fit
      } else {
        const u64 least = t < a.parts ? head : ~0ull;
        e = static_cast<u64>(wave_min_u(static_cast<unsigned>(least >> 32))) << 32;    // all keys of this logit
      }
      if (t == 0) sh.edge = e;
    }
  } else if (t < 128) {
    const int i = t - 64;
    LpSums g{-INFINITY, 0.f, 0.f};
    if (i < a.parts) {
      const float* o = a.sums + 3 * (first + i);
      g = LpSums{lp_shared(o), lp_shared(o + 1), lp_shared(o + 2)};
    }
    g = lp_to(g, wave_max(g.m), sc);
    g.s = wave_sum(g.s);
    g.w = wave_sum(g.w);
    if (i == 0) lp_outputs(a, row, g, sc.c, tok, z, sh.ml[0], sh.ml[1]);
  }
  if (n == 0) return;
  __syncthreads();
  const u64 edge = sh.edge;
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (mine[k] != 0ull && mine[k] >= edge) {
      const int at = atomicAdd(&sh.count, 1);
      if (at < kLpCand) sh.cand[at] = mine[k];
    }
  __syncthreads();
  const int cand = min(sh.count, kLpCand);
  auto put = [&](int rank, u64 key) { lp_write_top(a, row, rank, key, sc.c, sh.ml[0], sh.ml[1]); };
  lp_rank(sh, cand, n, put);
  for (int i = cand + t; i < n; i += NT) put(i, 0ull);         // a row with NaN
}

// NT: threads of a workgroup; 64 take whole rows only.
template <typename T, bool STREAM, int NT>
__global__ __launch_bounds__(NT) void logprobs_kernel(LpArgs a) {
  using R = Row<T, STREAM>;
  constexpr int N = R::N;
  constexpr int U = STREAM ? 8 : 4;        // pieces of a thread in flight
  __shared__ LpShared<NT> sh;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const int tok = a.tokens ? a.tokens[row] : 0;
  if (tok < 0) return;
  const LpScale sc(a, row);
  const T* base = static_cast<const T*>(a.logits) + static_cast<long long>(row) * a.ld;
  const R r(base, a.V);
  const int np = r.pieces();
  const int p0 = static_cast<int>(static_cast<long long>(np) * part / a.parts);
  const int p1 = static_cast<int>(static_cast<long long>(np) * (part + 1) / a.parts);
  const float z = a.logprob && tok < a.V ? R::value(base[tok]) : 0.f;

  float mx = -INFINITY, s = 0.f, w = 0.f;
  int mp = p0 + t;                         // first piece that holds mx
  auto take = [&](uint4 v, int p) {
    float x[N];
    R::widen(v, x);
    float b = x[0];
#pragma unroll
    for (int j = 1; j < N; ++j) b = fmaxf(b, x[j]);
    if (b > mx) {
      const LpSums q = lp_to(LpSums{mx, s, w}, b, sc);
      s = q.s;
      w = q.w;
      mx = b;
      mp = p;
    }
    const float from = mx == -INFINITY ? 0.f : mx;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float d = x[j] - from;
      const float e = __builtin_amdgcn_exp2f(d * sc.c);
      s += e;
      w = fmaf(e, fmaxf(d, sc.low), w);      // e is 0 there; NaN stays in s
    }
    return b;
  };
  // The walk, in segments of `rounds` steps.
  const int rounds = (p1 - p0 + U * NT * kLpSegs - 1) / (U * NT * kLpSegs);
  const int in0 = r.shift ? 1 : 0, in1 = min(p1, (a.V + r.shift) / N);      // whole pieces of the part
  for (int g = 0, p = p0 + t; p - t < p1; ++g) {
    float top = -INFINITY;
    for (int k = 0; k < rounds; ++k, p += U * NT) {
      uint4 x[U];
      // Steps inside the row without a test per piece.
      if (p - t >= in0 && p - t + U * NT <= in1) {
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = r.raw(p + u * NT);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = p + u * NT < p1 ? r.piece(p + u * NT) : R::nothing();
      }
#pragma unroll
      for (int u = 0; u < U; ++u) top = fmaxf(top, take(x[u], p + u * NT));
    }
    sh.seg[g][t] = top;
  }

  // Sums of the workgroup.
  LpSums g{mx, s, w};
  {
    const float m = wave_max(g.m);
    g = lp_to(g, m, sc);
    g.s = wave_sum(g.s);
    g.w = wave_sum(g.w);
    if (lane == 0) {
      sh.red[3 * wave] = g.m;
      sh.red[3 * wave + 1] = g.s;
      sh.red[3 * wave + 2] = g.w;
    }
    sh.key[t] = p0 + t < p1 ? lp_key(mx, mp) : 0ull;
    if (t == 0) sh.count = sh.agains = 0;
    __syncthreads();
    float mm = sh.red[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) mm = fmaxf(mm, sh.red[3 * i]);
    float ss = 0.f, sw = 0.f;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) {
      const LpSums q = lp_to(LpSums{sh.red[3 * i], sh.red[3 * i + 1], sh.red[3 * i + 2]}, mm, sc);
      ss += q.s;
      sw += q.w;
    }
    g = LpSums{mm, ss, sw};
  }
  const bool whole = a.parts == 1;
  if (t == NT - 64) {                      // of the last wave: the first goes on with the bound
    if (whole) {
      lp_outputs(a, row, g, sc.c, tok, z, sh.ml[0], sh.ml[1]);
    } else {
      float* o = a.sums + 3 * blockIdx.x;
      lp_share(o, g.m);
      lp_share(o + 1, g.s);
      lp_share(o + 2, g.w);
    }
  }
  const int n = a.n_top;
  if (n > 0) lp_largest(a, sh, r, p0, p1, rounds * U, row, sc.c);
  if (whole) return;

  if constexpr (NT == kLpThreads) {
    // The row's last part joins them all.
    __builtin_amdgcn_s_waitcnt(0);         // this wave's device-scope stores have completed
    __syncthreads();
    if (t == 0)
      sh.last = __hip_atomic_fetch_add(a.tickets + row, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                static_cast<unsigned>(a.parts) - 1u;
    __syncthreads();
    if (!sh.last) return;
    if (t == 0) a.tickets[row] = 0u;
    lp_join<R::kDrop>(a, sh, row, sc, tok, z);
  }
}

}  // namespace

hipError_t launch_token_logprobs(const ent_ctx* c, int T, const void* logits, int logits_dtype,
                                 long long ld, const int* tokens, const float* temp, float* logprob,
                                 float* entropy, int n_top, int* top_ids, float* top_logprobs,
                                 hipStream_t s) {
  LpArgs a{};
  a.logits = logits;
  a.ld = ld;
  a.T = T;
  a.V = c->cfg.vocab;
  a.n_top = n_top;
  a.tokens = tokens;
  a.temp = temp;
  a.t_cal = c->cfg.t_cal;
  a.logprob = logprob;
  a.entropy = entropy;
  a.top_ids = top_ids;
  a.top_lp = top_logprobs;
  a.sums = c->lp_sums;
  a.keys = c->lp_keys;
  a.tickets = c->lp_tickets;
  a.flags = c->dev_flags;
  const bool bf16 = logits_dtype == ENT_BF16;
  // Parts of a row.  A workgroup a CU, of 16 KB at least; where that leaves a part more
  // than 32 KB, two a CU, and where it is then more than 16384 logits, up to four.  Us with
  // 128 / 256 / 512 / 1024 workgroups (n_top 5, 128256 logits): 4 rows of floats 9.6 / 10.7,
  // 16 rows 12.0 / 11.9 / 14.4, 32 rows 15.8 / 12.7 / 13.3, 64 rows 22.2 / 16.6 / 15.0 / 17.6,
  // 128 rows - / 22.9 / 19.0 / 19.4 (of 32000 - / 12.2 / 11.3), 256 rows - / 38 / 27.6 / 28.9; 16
  // rows of bf16 11.3 / 11.8 / 14.8, 64 rows 17.8 / 13.4 / 13.1 / 15.6 (n_top 20: 18.4 / 14.3 /
  // 14.3 / 17.8), 128 rows - / 18.8 / 16.7 / 16.5, 256 rows - / 24.5 / 22.7 / 21.9.  More rows than
  // CUs in two parts / whole: 400 of floats 47.3 / 45.9, 512 51.6 / 47.4; of bf16, n_top 0, 26.8 /
  // 27.6 and 27.3 / 30.0.
  const long long bytes = static_cast<long long>(a.V) * (bf16 ? 2 : 4);
  const int part16 = static_cast<int>((bytes + 16383) / 16384);
  const int longest = (a.V + 16383) / 16384, one = c->num_cu / T, two = 2 * c->num_cu / T;
  a.parts = std::max(std::min(one, part16), std::min((part16 + 1) / 2, std::max(two, longest)));
  a.parts = std::max(1, std::min({kLpParts, kLpSlots / T, a.parts}));
  // Logits that fill the last-level cache are read without a place in the caches, and with 8
  // pieces of a thread in flight.  Us streamed / not (128256 logits, n_top 5): of floats
  // 1 GB 166 / 186, 263 MB 51.4 / 53.6, 230 MB 48.9 / 49.0, 205 MB 47.4 / 47.1,
  // 130 MB 30.4 / 28.4; of bf16 500 MB 91.0 / 99.6, 230 MB 50.4 / 51.8, 205 MB 49.0 / 50.4, 130 MB
  // 35.4 / 32.3.
  const bool stream = bytes * T > kStreamBytes;
  // Short rows, and many of some length, to a wave each instead of to four: what a row
  // costs besides its reads is then four times as cheap, and rows are enough to fill the
  // GPU.  Us (n_top 5): 20000 rows of 1000 floats 26.4 against 66.5, of 8000 bf16 78
  // against 127, 5000 of 8000 floats 35.0 against 38.9, but 1000 of them 14.2 against 11.3
  // and 5000 of 16000 floats 66.9 against 62.5.
  const bool alone = a.parts == 1 && (bytes <= 4 << 10 || (bytes <= 32 << 10 && T >= 8 * c->num_cu));
  auto kern = bf16 ? (alone    ? logprobs_kernel<uint16_t, false, 64>
                      : stream ? logprobs_kernel<uint16_t, true, kLpThreads>
                               : logprobs_kernel<uint16_t, false, kLpThreads>)
                   : (alone    ? logprobs_kernel<float, false, 64>
                      : stream ? logprobs_kernel<float, true, kLpThreads>
                               : logprobs_kernel<float, false, kLpThreads>);
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(T) * a.parts), dim3(alone ? 64 : kLpThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace ent
