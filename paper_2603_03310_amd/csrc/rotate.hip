// Root-mean-square norm of every query and key head and the rotation of its
// pairs by the token's position, in one pass over packed rows.
//
// A wave takes a part of a token's heads, 64 pieces of 16 bytes a step: 8, 16 or
// 32 lanes hold a head (sum of squares by cross-lane adds), so a lane holds the
// same dims of every head that it sees and forms its cosines and sines once.  With
// gains g and pairs (a, b) of inverse root r,
//   a' = r (x_a g_a cos - x_b g_b sin),  b' = r (x_b g_b cos + x_a g_a sin):
// out_i = r (x_i A_i + x_p B_i) with A_i = g_i cos, B_i = -+ g_p sin per lane.
// Pairs (i, i + rot / 2) lie rot / 2 dims apart, a whole number of lanes.

#include "ent_internal.h"

#include <math.h>

#include <algorithm>

namespace ent {
namespace {

constexpr int kRotThreads = 256;

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

template <typename T>
struct Piece;
template <>
struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void load(const float* p, float (&x)[4]) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
  }
  static __device__ __forceinline__ void store(float* p, const float (&x)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  }
};
template <>
struct Piece<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void load(const uint16_t* p, float (&x)[8]) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void store(uint16_t* p, const float (&x)[8]) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bf16x2 b;
      b[0] = static_cast<__bf16>(x[2 * i]);
      b[1] = static_cast<__bf16>(x[2 * i + 1]);
      w[i] = __builtin_bit_cast(unsigned, b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

template <typename T, int D>
__global__ __launch_bounds__(kRotThreads) void rotate_kernel(RotArgs a) {
  using P = Piece<T>;
  constexpr int N = P::N;
  constexpr int L = D / N;                 // lanes of a head
  constexpr int H = 64 / L;                // heads of a wave's step
  const int lane = threadIdx.x & 63, l = lane % L;
  const long long w = static_cast<long long>(blockIdx.x) * (kRotThreads / 64) + (threadIdx.x >> 6);
  const int row = static_cast<int>(w / a.parts), part = static_cast<int>(w % a.parts);
  if (row >= a.T) return;
  long long pos;
  {
    int b = row;
    long long at = 0;
    if (a.starts) {
      b = find_request(a.starts, a.B, row);
      const int s0 = a.starts[b];
      if (row < s0 || row >= a.starts[b + 1]) return;
      at = static_cast<long long>(row) - s0;
    }
    const int n = a.ctx ? a.ctx[b] : 0;
    if (n < 0 || n > a.room) {
      if (part == 0 && lane == 0) raise_flag(a.flags, ENT_DEV_BAD_CTXLEN);
      return;
    }
    pos = n + at;
  }
  float cs[N], sn[N];
  const int half = a.rot / 2;
  const int dim0 = l * N;
  const bool turns = dim0 < a.rot;         // rot is a multiple of 16: all dims of a lane or none
  const bool second = !a.adjacent && dim0 >= half;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    cs[j] = 1.f;
    sn[j] = 0.f;
    if (turns) {
      const int i = a.adjacent ? (dim0 + j) / 2 : dim0 + j - (second ? half : 0);
      // In half turns, reduced to [-1, 1] in 64 bits.
      const double t = static_cast<double>(pos) * (static_cast<double>(a.freq[i]) * 0.31830988618379067154);
      float s, c;
      sincospif(static_cast<float>(t - 2.0 * rint(0.5 * t)), &s, &c);
      cs[j] = c;
      const bool up = a.adjacent ? (j & 1) : second;
      sn[j] = up ? s : -s;
    }
  }
  const int mate = a.adjacent || !turns ? lane : (second ? lane - half / N : lane + half / N);
  for (int which = 0; which < 2; ++which) {
    const T* src = static_cast<const T*>(a.src[which]) + static_cast<long long>(row) * a.ld_src[which];
    T* dst = static_cast<T*>(a.dst[which]) + static_cast<long long>(row) * a.ld_dst[which];
    const float* g = a.gain[which];
    float A[N], B[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int d = dim0 + j;
      const int p = a.adjacent ? (d ^ 1) : turns ? (second ? d - half : d + half) : d;
      A[j] = cs[j] * (g ? g[d] : 1.f);
      B[j] = sn[j] * (g ? g[p] : 1.f);
    }
    const int heads = a.heads[which];
    for (int h0 = part * H; h0 < heads; h0 += a.parts * H) {
      const int h = h0 + lane / L;
      const bool ok = h < heads;
      const int off = min(h, heads - 1) * D + dim0;
      float x[N], y[N];
      P::load(src + off, x);
      float r = 1.f;
      if (g) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) ss = fmaf(x[j], x[j], ss);
        ss = xor_add<1>(ss);
        ss = xor_add<2>(ss);
        ss = xor_add<4>(ss);
        if constexpr (L >= 16) ss = xor_add<8>(ss);
        if constexpr (L >= 32) ss = xor_add<16>(ss);
        r = rsqrtf(fmaf(ss, 1.f / D, a.eps));
      }
      if (!turns) {
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = r * (x[j] * A[j]);
      }
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float m = a.adjacent ? x[j ^ 1] : __shfl(x[j], mate);
        if (turns) y[j] = r * fmaf(x[j], A[j], m * B[j]);
      }
      if (ok) P::store(dst + off, y);
    }
  }
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
  a.parts = 4;
  const long long waves = static_cast<long long>(T) * a.parts;
  const dim3 grid(static_cast<unsigned>((waves + kRotThreads / 64 - 1) / (kRotThreads / 64)));
  const bool bf16 = f.kv_dtype == ENT_BF16;
  auto kern = bf16 ? (f.head_dim == 64 ? rotate_kernel<uint16_t, 64> : rotate_kernel<uint16_t, 128>)
                   : (f.head_dim == 64 ? rotate_kernel<float, 64> : rotate_kernel<float, 128>);
  hipLaunchKernelGGL(kern, grid, dim3(kRotThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace ent
