// Log probabilities of given tokens, the entropy of their rows, and the likeliest
// alternatives, from one read of each logit row.
//
// With c = log2(e) / T, a maximum M of the logits z, S = sum 2^(c (z - M)) and
// W = sum 2^(c (z - M)) (z - M):
//   ln p(x) = ln 2 (c (z_x - M) - log2 S),   H = ln 2 (log2 S - c W / S).
// (The difference comes first, so rows of the type's lowest value overflow nothing.)
// A thread walks the 16-byte pieces of its row (or of its part of it) that lie a
// workgroup's width apart, and keeps its own maximum, sums, and the piece where its
// maximum first stood.  Of all threads the n with the largest (maximum, then
// earliest piece) hold the n largest logits between them: were one elsewhere, its
// thread's maximum would be among the n.  Only their pieces are read again, and of
// those only values at or above the n-th such maximum count, mostly little more
// than n, which are ranked by counting.
//
// Few rows are cut into parts; a second launch joins their sums and lists.

#include "ent_internal.h"

#include <math.h>

#include <algorithm>

namespace ent {
namespace {

constexpr int kLpThreads = 256;
constexpr int kLpTop = ENT_MAX_TOP_LOGPROBS;
constexpr int kLpCand = 1024;         // candidates that are ranked at once
constexpr int kLpUnroll = 4;
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
  float4* sums;           // [T * parts]  (max, S, W) of parts
  u64* keys;              // [T * parts, n_top]  their largest logits, descending
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
template <typename T>
struct Row {
  static constexpr int N = 16 / sizeof(T);
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
    return *reinterpret_cast<const uint4*>(base + (static_cast<long long>(p) * N - shift));
  }
  // Any piece; elements outside the row read as -inf.
  __device__ __forceinline__ void load(int p, float (&x)[N]) const {
    if (whole(p)) {
      widen(raw(p), x);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int i = p * N + j - shift;
        x[j] = i >= 0 && i < V ? value(base[i]) : -INFINITY;
      }
    }
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

template <typename T>
__global__ __launch_bounds__(kLpThreads) void logprobs_kernel(LpArgs a) {
  constexpr int N = Row<T>::N, NT = kLpThreads, U = kLpUnroll;
  __shared__ u64 s_key[NT];
  __shared__ u64 s_cand[kLpCand];
  __shared__ float s_red[3 * NT / 64];
  __shared__ int s_who[kLpTop];
  __shared__ u64 s_edge;
  __shared__ int s_count;
  __shared__ float s_ml[2];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const int tok = a.tokens ? a.tokens[row] : 0;
  if (tok < 0) return;
  const LpScale sc(a, row);
  const T* base = static_cast<const T*>(a.logits) + static_cast<long long>(row) * a.ld;
  const Row<T> r(base, a.V);
  const int np = r.pieces();
  const int p0 = static_cast<int>(static_cast<long long>(np) * part / a.parts);
  const int p1 = static_cast<int>(static_cast<long long>(np) * (part + 1) / a.parts);
  const float z = a.logprob && tok < a.V ? Row<T>::value(base[tok]) : 0.f;

  float mx = -INFINITY, s = 0.f, w = 0.f;
  int mp = p0 + t;                         // first piece that holds mx
  auto take = [&](const float (&x)[N], int p) {
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
  };
  for (int p = p0 + t; p < p1; p += U * NT) {
    float x[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p + u * NT < p1) r.load(p + u * NT, x[u]);
      else {
#pragma unroll
        for (int j = 0; j < N; ++j) x[u][j] = -INFINITY;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) take(x[u], p + u * NT);
  }

  // Sums of the workgroup.
  LpSums g{mx, s, w};
  {
    const float m = wave_max(g.m);
    g = lp_to(g, m, sc);
    g.s = wave_sum(g.s);
    g.w = wave_sum(g.w);
    if (lane == 0) {
      s_red[3 * wave] = g.m;
      s_red[3 * wave + 1] = g.s;
      s_red[3 * wave + 2] = g.w;
    }
    s_key[t] = p0 + t < p1 ? lp_key(mx, mp) : 0ull;
    if (t == 0) {
      s_count = 0;
      s_edge = 0ull;
    }
    __syncthreads();
    float mm = s_red[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) mm = fmaxf(mm, s_red[3 * i]);
    float ss = 0.f, sw = 0.f;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) {
      const LpSums q = lp_to(LpSums{s_red[3 * i], s_red[3 * i + 1], s_red[3 * i + 2]}, mm, sc);
      ss += q.s;
      sw += q.w;
    }
    g = LpSums{mm, ss, sw};
  }
  const bool whole = a.parts == 1;
  if (t == 0) {
    if (whole) lp_outputs(a, row, g, sc.c, tok, z, s_ml[0], s_ml[1]);
    else a.sums[blockIdx.x] = make_float4(g.m, g.s, g.w, 0.f);
  }
  const int n = a.n_top;
  if (n == 0) return;

  // The n threads with the largest keys, and the n-th key.
  {
    const u64 mine = s_key[t];
    int rank = 0;
    for (int i = 0; i < NT; ++i) rank += s_key[i] > mine ? 1 : 0;
    if (mine != 0ull && rank < n) {
      s_who[rank] = t;
      if (rank == n - 1) s_edge = mine;
    }
  }
  const int who = min(n, min(NT, max(p1 - p0, 0)));
  __syncthreads();
  const u64 edge = s_edge;
  const float ev = lp_value(static_cast<unsigned>(edge >> 32));
  const int ep = static_cast<int>(~static_cast<unsigned>(edge));
  // Whether element (x, i) of piece p can be among the n largest.
  auto counts = [&](float x, int i, int p) {
    return i >= 0 && i < a.V && (edge == 0ull || x > ev || (x == ev && p <= ep));
  };
  for (int k = wave; k < who; k += NT / 64) {
    const int first = p0 + s_who[k];
    for (int p = first + lane * NT; p < p1; p += 64 * NT) {
      float x[N];
      r.load(p, x);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int i = p * N + j - r.shift;
        if (counts(x[j], i, p)) {
          const int at = atomicAdd(&s_count, 1);
          if (at < kLpCand) s_cand[at] = lp_key(x[j], i);
        }
      }
    }
  }
  __syncthreads();
  const int cand = s_count;
  auto put = [&](int rank, u64 key) {
    if (whole) lp_write_top(a, row, rank, key, sc.c, s_ml[0], s_ml[1]);
    else a.keys[static_cast<long long>(blockIdx.x) * n + rank] = key;
  };
  if (cand <= kLpCand) {
    for (int i = t; i < cand; i += NT) {
      const u64 mine = s_cand[i];
      int rank = 0;
      for (int k = 0; k < cand; ++k) rank += s_cand[k] > mine ? 1 : 0;
      if (rank < n) put(rank, mine);
    }
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
    s_key[t] = best;
    __syncthreads();
    best = 0ull;
    for (int i = 0; i < NT; ++i) best = s_key[i] > best ? s_key[i] : best;
    if (t == 0) put(k, best);
    last = best;
  }
}

// One wave a row: the parts' sums, and the n largest of their descending lists.
__global__ __launch_bounds__(64) void logprobs_join_kernel(LpArgs a, int logits_bf16) {
  __shared__ u64 s_key[64 * kLpTop];
  const int row = blockIdx.x, lane = threadIdx.x, n = a.n_top;
  const int tok = a.tokens ? a.tokens[row] : 0;
  if (tok < 0) return;
  const LpScale sc(a, row);
  const long long at = static_cast<long long>(row) * a.ld + tok;
  float z = 0.f;
  if (a.logprob && tok < a.V)
    z = logits_bf16 ? bf16_to_f32(static_cast<const uint16_t*>(a.logits)[at]) : static_cast<const float*>(a.logits)[at];
  const long long first = static_cast<long long>(row) * a.parts;
  LpSums g{-INFINITY, 0.f, 0.f};
  if (lane < a.parts) {
    const float4 v = a.sums[first + lane];
    g = LpSums{v.x, v.y, v.z};
  }
  for (int i = lane; i < a.parts * n; i += 64) s_key[i] = a.keys[first * n + i];
  g = lp_to(g, wave_max(g.m), sc);
  g.s = wave_sum(g.s);
  g.w = wave_sum(g.w);
  float m = 0.f, l = 0.f;
  if (lane == 0) lp_outputs(a, row, g, sc.c, tok, z, m, l);
  m = lane_at(m, 0);
  l = lane_at(l, 0);
  __syncthreads();
  int next = 0;
  for (int k = 0; k < n; ++k) {
    const u64 head = lane < a.parts && next < n ? s_key[lane * n + next] : 0ull;
    const unsigned hi = static_cast<unsigned>(head >> 32), lo = static_cast<unsigned>(head);
    const unsigned top = wave_max_u(hi);
    const unsigned low = wave_max_u(hi == top ? lo : 0u);
    const u64 best = static_cast<u64>(top) << 32 | low;
    if (head == best) ++next;              // keys differ, but for 0
    if (lane == 0) lp_write_top(a, row, k, best, sc.c, m, l);
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
  a.flags = c->dev_flags;
  const bool bf16 = logits_dtype == ENT_BF16;
  const int tile = kLpThreads * (bf16 ? 8 : 4);          // logits of a workgroup's step
  a.parts = std::max(1, std::min({kLpSlots / T, 64, (a.V + tile - 1) / tile}));
  auto kern = bf16 ? logprobs_kernel<uint16_t> : logprobs_kernel<float>;
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(T) * a.parts), dim3(kLpThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  hipLaunchKernelGGL(logprobs_join_kernel, dim3(T), dim3(64), 0, s, a, bf16 ? 1 : 0);
  return hipGetLastError();
}

}  // namespace ent
