// Root-mean-square norm of every query and key head and the rotation of its
// pairs by the token's position, in one pass over packed rows.
//
// A wave takes a part of a token's heads, 64 pieces of 16 bytes a step: 8, 16 or
// 32 lanes hold a head (sum of squares by cross-lane adds), so a lane holds the
// same dims of every head that it sees and forms its cosines and sines once.  With
// gains g and pairs (a, b) of inverse root r,
//   a' = r (x_a g_a cos - x_b g_b sin),  b' = r (x_b g_b cos + x_a g_a sin).
// Pairs (i, i + rot / 2) lie a whole number of lanes apart; where that is half a head they
// meet by lane moves, else by shuffles, and the two lanes form half of the angles each.
//
// Bound by memory, each row read and written once: 51624 rows of 64 + 8 heads of 128
// (bf16, 1.90 GB) 329 us = 5.8 TB/s, over a large copy's 4.7.  On the way there: four
// waves a row, each with all of its angles and a shuffle per value, 956 us.
// Few rows are a chain of round trips (starts, length, then sines): 128 rows 5.1 us with
// frequencies and gains loaded before the position is known, 6.8 with them after.

#include "ent_internal.h"

#include <math.h>

#include <algorithm>

namespace ent {
namespace {

constexpr int kRotThreads = 256;
// Waves that few rows are cut into.  64 + 8 heads of 128 in bf16, us with 2048 / 4096 /
// 8192 / 16384: 512 rows 7.6 / 7.8 / 9.7 / 10.0, 1024 rows 11.6 / 11.1 / 12.1 / 15.6, 2048
// rows 18.2 / 15.3 / 17.0 / 18.6, 4096 rows 34.5 / 34.8 / 35.2 / 32.6.
constexpr int kRotWaves = 4096;
// Steps of a wave from which on rows past the caches are streamed.
constexpr int kRotStreamSteps = 4;

struct RotArgs {
  const void* src[2];     // queries, keys
  void* dst[2];
  long long ld_src[2], ld_dst[2];
  const float* gain[2];   // nullable
  int heads[2];
  const float* freq;
  float eps;
  int rot, adjacent;
  const int* starts;      // nullable
  const int* ctx;         // nullable
  int B, T, room;         // room: largest ctx_lens
  int parts;              // waves of a row
  unsigned* flags;
};

// The largest b in [0, n) with s[b] <= x, one x of a whole wave; some b in range
// where s is not ascending.
__device__ __forceinline__ int find_request(const int* s, int n, int x) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 1) {
    const int w = (n + 63) / 64;
    const int below = __popcll(__ballot(lane * w < n && s[lo + min(lane * w, n - 1)] <= x));
    const int k = max(below - 1, 0);       // 0 too where s does not begin at or below x
    lo += k * w;
    n = min(w, n - k * w);
  }
  return lo;
}

// 16 bytes of a row as N floats.
template <typename T>
struct Piece {
  static constexpr int N = 16 / sizeof(T);
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
  static __device__ __forceinline__ uint4 narrow(const float (&x)[N]) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (N == 4) {
        w[i] = __float_as_uint(x[i]);
      } else {
        bf16x2 b;
        b[0] = static_cast<__bf16>(x[2 * i]);
        b[1] = static_cast<__bf16>(x[2 * i + 1]);
        w[i] = __builtin_bit_cast(unsigned, b);
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// Which lane holds a lane's pairs' other dims: itself (adjacent pairs), the lane half a
// head away (all dims turn in pairs of halves), or some other.
enum { kAdjacent, kHalves, kAnyHalves };

template <typename T, int D, int PAIRS, bool STREAM>
__global__ __launch_bounds__(kRotThreads) void rotate_kernel(RotArgs a) {
  using P = Piece<T>;
  constexpr int N = P::N;
  constexpr int L = D / N;                 // lanes of a head
  constexpr int H = 64 / L;                // heads of a wave's step
  constexpr int U = STREAM ? 6 : 3;        // steps whose loads are in flight together
  const int lane = threadIdx.x & 63, l = lane % L;
  const unsigned w = blockIdx.x * (kRotThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned parts = a.parts;
  const int row = static_cast<int>(w / parts), part = static_cast<int>(w - row * parts);
  if (row >= a.T) return;
  const int sq = (a.heads[0] + H - 1) / H, steps = sq + (a.heads[1] + H - 1) / H;
  const int s0 = part * steps / static_cast<int>(parts), s1 = (part + 1) * steps / static_cast<int>(parts);
  const int dim0 = l * N;
  const T* const src0 = static_cast<const T*>(a.src[0]) + row * a.ld_src[0];
  const T* const src1 = static_cast<const T*>(a.src[1]) + row * a.ld_src[1];
  // This lane's place in step s; past the last head, the last head again.
  auto place = [&](int s, bool& keys, bool& ok) {
    keys = s >= sq;
    const int h = (keys ? s - sq : s) * H + lane / L, heads = a.heads[keys ? 1 : 0];
    ok = h < heads;
    return min(h, heads - 1) * D + dim0;
  };
  auto fetch = [&](int s) {
    bool keys, ok;
    const int at = place(s, keys, ok);
    return load16<STREAM>((keys ? src1 : src0) + at);
  };
  uint4 raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) raw[u] = fetch(min(s0 + u, s1 - 1));
  // The lane's gains and frequencies are on their way before its position is known.
  const int half = a.rot / 2;
  const bool turns = PAIRS == kHalves || dim0 < a.rot;     // rot is a multiple of 16: all dims of a lane or none
  const bool second = PAIRS != kAdjacent && dim0 >= half;
  constexpr int F = N / 2;                 // angles that a lane forms, of its own pairs or half of its and its mate's
  const int f0 = PAIRS == kAdjacent ? dim0 / 2 : dim0 - (second ? half - F : 0);
  float freq[F];
#pragma unroll
  for (int j = 0; j < F; ++j) freq[j] = turns ? a.freq[f0 + j] : 0.f;
  float g[N];
  bool norm;
  auto gains = [&](int which) {
    const float* gain = a.gain[which];
    norm = gain != nullptr;
#pragma unroll
    for (int j = 0; j < N; ++j) g[j] = norm ? gain[dim0 + j] : 1.f;
  };
  int kind = s0 >= sq ? 1 : 0;             // whose gains g holds
  gains(kind);
  long long pos;
  {
    int b = row;
    long long at = 0;
    if (a.starts) {
      b = find_request(a.starts, a.B, row);
      const int first = a.starts[b];
      if (row < first || row >= a.starts[b + 1]) return;
      at = static_cast<long long>(row) - first;
    }
    const int n = a.ctx ? a.ctx[b] : 0;
    if (n < 0 || n > a.room) {
      if (part == 0 && lane == 0) raise_flag(a.flags, ENT_DEV_BAD_CTXLEN);
      return;
    }
    pos = n + at;
  }
  auto angle = [&](int j, float& c, float& s) {
    // In half turns, reduced to [-1, 1] in 64 bits.
    const double t = static_cast<double>(pos) * (static_cast<double>(freq[j]) * 0.31830988618379067154);
    sincospif(static_cast<float>(t - 2.0 * rint(0.5 * t)), &s, &c);
  };
  // The value of the lane that holds the pairs' other dims.
  const int mate = PAIRS != kAnyHalves || !turns ? lane : second ? lane - half / N : lane + half / N;
  auto other = [&](float v) {
    if constexpr (PAIRS == kHalves) return __uint_as_float(xor_lane<L / 2>(__float_as_uint(v)));
    else return __shfl(v, mate);
  };
  float cs[N], sn[N];                      // dims that do not turn: frequency 0
#pragma unroll
  for (int j = 0; j < F; ++j) {
    float c, s;
    angle(j, c, s);
    if constexpr (PAIRS == kAdjacent) {
      cs[2 * j] = cs[2 * j + 1] = c;
      sn[2 * j] = -s;
      sn[2 * j + 1] = s;
    } else {
      const float oc = other(c), os = other(s);
      cs[j] = second ? oc : c;
      cs[j + F] = second ? c : oc;
      sn[j] = second ? os : -s;
      sn[j + F] = second ? s : -os;
    }
  }
  T* const dst0 = static_cast<T*>(a.dst[0]) + row * a.ld_dst[0];
  T* const dst1 = static_cast<T*>(a.dst[1]) + row * a.ld_dst[1];
  for (int s = s0; s < s1; s += U) {
    uint4 now[U];
#pragma unroll
    for (int u = 0; u < U; ++u) now[u] = raw[u];
    if (s + U < s1) {
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u] = fetch(min(s + U + u, s1 - 1));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s + u >= s1) break;
      bool keys, ok;
      const int at = place(s + u, keys, ok);
      if (kind != (keys ? 1 : 0)) gains(kind = keys ? 1 : 0);
      float x[N], y[N];
      P::widen(now[u], x);
      float r = 1.f;
      if (norm) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) ss = fmaf(x[j], x[j], ss);
        ss = xor_add<1>(ss);
        ss = xor_add<2>(ss);
        ss = xor_add<4>(ss);
        if constexpr (L >= 16) ss = xor_add<8>(ss);
        if constexpr (L >= 32) ss = xor_add<16>(ss);
        r = rsqrtf(fmaf(ss, 1.f / D, a.eps));
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] *= g[j];
      }
#pragma unroll
      for (int j = 0; j < N; ++j) {
        float m;                           // the pair's other
        if constexpr (PAIRS == kAdjacent) m = x[j ^ 1];
        else m = other(x[j]);
        y[j] = r * (turns ? fmaf(x[j], cs[j], m * sn[j]) : x[j]);
      }
      if (ok) store16<STREAM>((keys ? dst1 : dst0) + at, P::narrow(y));
    }
  }
}

template <typename T, int D, bool STREAM>
auto rotate_pairs(int pairs) {
  return pairs == kAdjacent ? rotate_kernel<T, D, kAdjacent, STREAM>
         : pairs == kHalves ? rotate_kernel<T, D, kHalves, STREAM> : rotate_kernel<T, D, kAnyHalves, STREAM>;
}
template <typename T, int D>
auto rotate_for(int pairs, bool stream) {
  return stream ? rotate_pairs<T, D, true>(pairs) : rotate_pairs<T, D, false>(pairs);
}

}  // namespace

hipError_t launch_qk_norm_rope(const ent_ctx* c, int B, int T, const ent_qk_params& p, const void* q,
                               long long ldq, const void* k, long long ldk, const int* starts,
                               const int* ctx_lens, void* q_out, long long ldqo, void* k_out,
                               long long ldko, hipStream_t s) {
  const ent_config& f = c->cfg;
  RotArgs a{};
  a.src[0] = q; a.src[1] = k;
  a.dst[0] = q_out; a.dst[1] = k_out;
  a.ld_src[0] = ldq; a.ld_src[1] = ldk;
  a.ld_dst[0] = ldqo; a.ld_dst[1] = ldko;
  a.gain[0] = p.q_gain; a.gain[1] = p.k_gain;
  a.heads[0] = f.num_q_heads; a.heads[1] = f.num_kv_heads;
  a.freq = p.inv_freq;
  a.eps = p.eps;
  a.rot = p.rot_dim;
  a.adjacent = p.adjacent != 0;
  a.starts = starts;
  a.ctx = ctx_lens;
  a.B = B;
  a.T = T;
  a.room = f.max_blocks_per_seq * kBlock;
  a.flags = c->dev_flags;
  const bool bf16 = f.kv_dtype == ENT_BF16;
  // Waves of a row: where rows are few, as many as it has steps.
  const int per = 64 * (bf16 ? 8 : 4) / f.head_dim;
  const int steps = (f.num_q_heads + per - 1) / per + (f.num_kv_heads + per - 1) / per;
  a.parts = std::max(1, std::min(steps, kRotWaves / T));
  const long long waves = static_cast<long long>(T) * a.parts;
  const dim3 grid(static_cast<unsigned>((waves + kRotThreads / 64 - 1) / (kRotThreads / 64)));
  const int pairs = a.adjacent ? kAdjacent : a.rot == f.head_dim ? kHalves : kAnyHalves;
  // Rows that leave the last-level cache little room for anything else take no places in the
  // caches: 51624 rows of 64 + 8 heads of 128 in bf16 (1.9 GB) 329 us against 369 (loads alone
  // 368, stores alone 349, both with three steps in flight instead of six 334).  Fewer are soon
  // read by what follows.  Us streamed / not, MB read and written: 64 + 8 heads of 128 123:
  // 28.4 / 28.3, 147: 31.0 / 32.7, 184: 36.7 / 42.7; 16 + 8 of 128 123: 26.3 / 22.7, 147: 29.7 /
  // 30.3, 180: 35.3 / 39.9; of floats, 32 + 8 of 64, 123: 22.9 / 24.5, 180: 35.0 / 44.0.  Rows of
  // few steps load some pieces twice for want of six: 16 + 4 heads of 64 (3 steps) 184: 48.4 /
  // 45.2, 400: 101 / 88; 8 + 8 of 128 (4) 180: 38.0 / 40.5, 300: 59.6 / 61.3, 1000: 188 / 186.
  const long long bytes = 2ll * T * (f.num_q_heads + f.num_kv_heads) * f.head_dim * (bf16 ? 2 : 4);
  const bool stream = bytes > kStreamCopyBytes && steps / a.parts >= kRotStreamSteps;
  auto kern = bf16 ? (f.head_dim == 64 ? rotate_for<uint16_t, 64>(pairs, stream) : rotate_for<uint16_t, 128>(pairs, stream))
                   : (f.head_dim == 64 ? rotate_for<float, 64>(pairs, stream) : rotate_for<float, 128>(pairs, stream));
  hipLaunchKernelGGL(kern, grid, dim3(kRotThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace ent
