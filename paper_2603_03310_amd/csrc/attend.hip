// Causal attention over packed prompts (ent_prompt_attention).
//
//   o_t = sum_u p_tu v_u,  p_t. = softmax over u of scale <q_t, k_u>,
//   u in [first token of t's request, t]
//
// A workgroup takes one KV head and a stretch of packed tokens with all G query
// heads of the group: row r is token t0 + r / G, head g G + r % G.  So a K and
// V tile serves G heads, and few rows of a tile lie across the diagonal.  A
// stretch may hold several requests, or parts of them: each row has its own
// range of keys [lo, t], and tiles that all rows see whole need no mask.  There
// is no padding of short requests, and nothing to plan on the host.
//
// One pass over the keys with a running maximum and sum (fp32), on MFMA with
// the scores transposed, S^T = K Q^T: a lane then has 16 scores of one row per
// 32 x 32 block, so the row's statistics are in-lane but for one exchange
// between the wave's halves, and P^T comes out of the S^T accumulators in the
// layout that O^T += V^T P^T wants as its right operand (the order of keys within
// a block is free, and V's rows are taken in the accumulators' order).
#include "ent_internal.h"

#include <math.h>

#include <algorithm>

namespace ent {
namespace {

constexpr int kAttThreads = 256;
constexpr int kAttWaves = kAttThreads / 64;

typedef __bf16 bf16x8_t __attribute__((__vector_size__(8 * sizeof(__bf16))));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((__vector_size__(16 * sizeof(float))));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

struct AttArgs {
  const void* q;
  long long ldq;
  const void* k;
  long long ldk;
  const void* v;
  long long ldv;
  const int* starts;   // [B + 1]
  void* out;
  long long ldo;
  float* lse;          // nullable [T, H_q]
  int B, T, Hkv, G, lg;   // lg = log2 G
  int tiles;           // stretches of tokens
  float c;             // |scale| log2(e), > 0
  unsigned keep, flip; // queries are (q & keep) ^ flip: the scale's sign, or 0 where it is 0
};

// Where the rows' requests begin.  base: the largest start at or before the
// stretch's first token; bits: tokens of the stretch that begin a request.
template <int TOK>
struct AttRanges {
  int base, end;
  int bad_lo, bad_hi;    // keys whose values were set aside (att_set_aside)
  unsigned bits[(TOK + 31) / 32];
};

// Reads the starts (any values: all are taken as inside [0, T], so no row's
// range leaves the packed rows).  False where the stretch holds no token.
template <int TOK>
__device__ __forceinline__ bool att_ranges(const AttArgs& a, int t0, int ntok, AttRanges<TOK>& s) {
  const int t = threadIdx.x;
  constexpr int W = (TOK + 31) / 32;
  if (t < W) s.bits[t] = 0;
  if (t == W) s.base = 0;
  if (t == W + 1) {
    s.bad_lo = 0x7fffffff;
    s.bad_hi = -1;
  }
  if (t == W + 2) s.end = min(max(a.starts[a.B], 0), a.T);
  __syncthreads();
  int base = 0;
  for (int i = t; i < a.B; i += kAttThreads) {
    const int x = a.starts[i];
    if (x <= t0) base = max(base, x);
    else if (x < t0 + ntok) atomicOr(&s.bits[(x - t0) >> 5], 1u << ((x - t0) & 31));
  }
  base = static_cast<int>(wave_max_u(static_cast<unsigned>(base)));
  if ((t & 63) == 0 && base > 0) atomicMax(&s.base, base);
  __syncthreads();
  return t0 < s.end;
}
// First token of the request that token t0 + i belongs to.
template <int TOK>
__device__ __forceinline__ int att_lo(const AttRanges<TOK>& s, int t0, int i) {
  int w = i >> 5;
  unsigned m = s.bits[w] & (0xffffffffu >> (31 - (i & 31)));
  while (m == 0 && w > 0) m = s.bits[--w];
  return m ? t0 + 32 * w + 31 - __builtin_clz(m) : s.base;
}

// A weight of 0 does not keep an infinity or a NaN out of a product.  In tiles
// that some row sees in part (its own tail, or another request's tokens),
// values that are not finite are therefore taken as 0 and their keys noted;
// after the last tile the rows that do see such a key add its values.  (Where a
// tile is seen whole they go through the product; adding them once more to what
// they made infinite or NaN there changes nothing.)
__device__ __forceinline__ bool att_set_aside(uint4& w, bool bf16) {
  unsigned u[4] = {w.x, w.y, w.z, w.w};
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (bf16) {
      const bool lo = (u[i] & 0x7f80u) == 0x7f80u, hi = (u[i] & 0x7f800000u) == 0x7f800000u;
      any |= lo || hi;
      u[i] &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0x0000ffffu : 0xffffffffu);
    } else if ((u[i] & 0x7f800000u) == 0x7f800000u) {
      any = true;
      u[i] = 0;
    }
  }
  w = make_uint4(u[0], u[1], u[2], u[3]);
  return any;
}
__device__ __forceinline__ float att_not_finite(float x) {
  return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? x : 0.f;
}

// ---------------------------------------------------------------------------
// bf16.  Four waves of 32 NB rows each; keys in tiles of 64, in LDS twice (the
// next tile is loaded to registers behind the arithmetic on this one).
// ---------------------------------------------------------------------------
template <int D, int NB>
__global__ __launch_bounds__(kAttThreads, NB == 2 ? 1 : 2) void attend_bf16_kernel(AttArgs a) {
  constexpr int BM = kAttWaves * 32 * NB;   // rows
  constexpr int BN = 64;                    // keys of a tile
  constexpr int KS = D / 16;                // QK steps
  constexpr int DB = D / 32;                // blocks of 32 output dims
  // Row pitches: K's rows are read 16 B at a time, 16 rows in turn (4 banks
  // apart); V's 64 B of four rows at a time (16 banks apart).
  constexpr int PK = D + 8, PV = D + 32;
  constexpr int CH = D / 8;                 // 16 B pieces of a row
  constexpr int RP = kAttThreads / CH;      // rows loaded at once
  constexpr int NL = BN / RP;
  __shared__ __attribute__((aligned(16))) uint16_t s_k[2][BN * PK];
  __shared__ __attribute__((aligned(16))) uint16_t s_v[2][BN * PV];
  __shared__ AttRanges<BM> s_r;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int r32 = lane & 31, h = lane >> 5;
  const int g = blockIdx.x % a.Hkv;
  const int tile = a.tiles - 1 - static_cast<int>(blockIdx.x / a.Hkv);   // longest first
  const int ntok = BM >> a.lg;
  const int t0 = tile * ntok;
  if (!att_ranges(a, t0, ntok, s_r)) return;
  const int end = s_r.end;
  const int last = min(t0 + ntok, end) - 1;               // last token of the stretch
  const int kv0 = att_lo(s_r, t0, 0), lo_last = att_lo(s_r, t0, last - t0);
  const int nt = (last - kv0) / BN + 1;

  // This lane's rows.
  int tok[NB], lo[NB];
  bool row_ok[NB];
  bf16x8_t qf[NB][KS];
  const uint16_t* q = static_cast<const uint16_t*>(a.q);
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = wave * 32 * NB + nb * 32 + r32;
    tok[nb] = t0 + (r >> a.lg);
    row_ok[nb] = tok[nb] <= last;
    const int tk = min(tok[nb], last);
    lo[nb] = att_lo(s_r, t0, tk - t0);
    tok[nb] = tk;
    const uint16_t* p = q + tk * a.ldq + (g * a.G + (r & (a.G - 1))) * D + 8 * h;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      uint4 w = *reinterpret_cast<const uint4*>(p + 16 * ks);
      w = make_uint4((w.x & a.keep) ^ a.flip, (w.y & a.keep) ^ a.flip, (w.z & a.keep) ^ a.flip,
                     (w.w & a.keep) ^ a.flip);
      qf[nb][ks] = __builtin_bit_cast(bf16x8_t, w);
    }
  }
  // Keys that some row of this wave sees: [w_lo, w_hi].
  const int w_first = min(t0 + ((wave * 32 * NB) >> a.lg), last);
  const int w_hi = min(t0 + ((wave * 32 * NB + 32 * NB - 1) >> a.lg), last);
  const int w_lo = att_lo(s_r, t0, w_first - t0);
  const bool w_any = t0 + ((wave * 32 * NB) >> a.lg) <= last;

  const uint16_t* kp = static_cast<const uint16_t*>(a.k) + g * D;
  const uint16_t* vp = static_cast<const uint16_t*>(a.v) + g * D;
  const int lr = t / CH, lc = t % CH * 8;
  uint4 kr[NL], vr[NL];
  auto load = [&](int j) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int u = kv0 + j * BN + lr + i * RP;
      kr[i] = vr[i] = make_uint4(0u, 0u, 0u, 0u);
      if (u <= last) {
        kr[i] = *reinterpret_cast<const uint4*>(kp + u * a.ldk + lc);
        vr[i] = *reinterpret_cast<const uint4*>(vp + u * a.ldv + lc);
      }
    }
  };
  // Tiles that some row of the stretch does not see whole.
  auto part = [&](int j) { return kv0 + j * BN < lo_last || kv0 + j * BN + BN - 1 > t0; };
  auto stash = [&](int j) {
    const int buf = j & 1;
    if (part(j)) {
#pragma unroll
      for (int i = 0; i < NL; ++i)
        if (att_set_aside(vr[i], true)) {
          atomicMin(&s_r.bad_lo, kv0 + j * BN + lr + i * RP);
          atomicMax(&s_r.bad_hi, kv0 + j * BN + lr + i * RP);
        }
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      *reinterpret_cast<uint4*>(&s_k[buf][(lr + i * RP) * PK + lc]) = kr[i];
      *reinterpret_cast<uint4*>(&s_v[buf][(lr + i * RP) * PV + lc]) = vr[i];
    }
  };

  f32x16_t o[NB][DB];
  float m[NB], l[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m[nb] = -INFINITY;
    l[nb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[nb][db][i] = 0.f;
  }

  load(0);
  stash(0);
  __syncthreads();
  for (int j = 0; j < nt; ++j) {
    const int buf = j & 1;
    if (j + 1 < nt) load(j + 1);
    const int k0 = kv0 + j * BN;
    if (w_any && k0 <= w_hi && k0 + BN > w_lo) {
      f32x16_t s[NB][2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[nb][kb][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const bf16x8_t kf = *reinterpret_cast<const bf16x8_t*>(
              &s_k[buf][(32 * kb + r32) * PK + 16 * ks + 8 * h]);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            s[nb][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[nb][ks], s[nb][kb], 0, 0, 0);
        }
      }
      if (part(j)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int u = k0 + 32 * kb + 8 * (i / 4) + 4 * h + i % 4;
              if (u < lo[nb] || u > tok[nb]) s[nb][kb][i] = -INFINITY;
            }
      }
      bf16x8_t pf[NB][4];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float mx = s[nb][0][0];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[nb][kb][i]);
        mx = xor_max<32>(mx);
        // The reference moves only where some row's scores pass it by 2^8:
        // weights up to 256 are as exact as those up to 1.
        if (__any((mx - m[nb]) * a.c > 8.f)) {
          const float mn = fmaxf(m[nb], mx);
          const float alpha = mn == m[nb] ? 1.f : __builtin_amdgcn_exp2f((m[nb] - mn) * a.c);
          l[nb] *= alpha;
#pragma unroll
          for (int db = 0; db < DB; ++db) o[nb][db] *= alpha;
          m[nb] = mn;
        }
        const float mc = m[nb] == -INFINITY ? 0.f : m[nb] * a.c;
        float sum = 0.f;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float p = __builtin_amdgcn_exp2f(fmaf(s[nb][kb][i], a.c, -mc));
            s[nb][kb][i] = p;
            sum += p;
          }
        l[nb] += sum;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          // Weights to bf16 (2^-9 of each at most, and independent of each
          // other); the sum keeps them whole.
          unsigned w[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const f32x2_t pe = {s[nb][x / 2][8 * (x % 2) + 2 * y], s[nb][x / 2][8 * (x % 2) + 2 * y + 1]};
            w[y] = __builtin_bit_cast(unsigned, __builtin_convertvector(pe, bf16x2_t));
          }
          pf[nb][x] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
        }
      }
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          // V^T: lane (dim, half): keys 16 x + 4 h + 0..3 and + 8.
          const int row = 16 * x + 4 * h + ((lane & 15) >> 2);
          const int col = 32 * db + (lane & 16) + 4 * (lane & 3);
          typedef s16x4_t __attribute__((address_space(3)))* lds_t;
          const s16x4_t v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(&s_v[buf][row * PV + col]));
          const s16x4_t v1 =
              __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(&s_v[buf][(row + 8) * PV + col]));
          const uint2 w0 = __builtin_bit_cast(uint2, v0), w1 = __builtin_bit_cast(uint2, v1);
          const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, make_uint4(w0.x, w0.y, w1.x, w1.y));
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            o[nb][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[nb][x], o[nb][db], 0, 0, 0);
        }
    }
    if (j + 1 < nt) stash(j + 1);
    __syncthreads();
  }

  for (int u = s_r.bad_lo; u <= s_r.bad_hi; ++u) {
    const uint16_t* x = vp + u * a.ldv + 4 * h;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
      if (lo[nb] <= u && u <= tok[nb]) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            o[nb][db][i] += att_not_finite(bf16_to_f32(x[32 * db + 8 * (i / 4) + i % 4]));
      }
  }

  uint16_t* out = static_cast<uint16_t*>(a.out);
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const float lt = xor_add<32>(l[nb]);
    const int r = wave * 32 * NB + nb * 32 + r32;
    const int hq = g * a.G + (r & (a.G - 1));
    if (!row_ok[nb]) continue;
    const float inv = 1.f / lt;
    uint16_t* p = out + tok[nb] * a.ldo + hq * D + 4 * h;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        unsigned w[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const f32x2_t pe = {o[nb][db][4 * x + 2 * y] * inv, o[nb][db][4 * x + 2 * y + 1] * inv};
          w[y] = __builtin_bit_cast(unsigned, __builtin_convertvector(pe, bf16x2_t));
        }
        *reinterpret_cast<uint2*>(p + 32 * db + 8 * x) = make_uint2(w[0], w[1]);
      }
    if (a.lse && h == 0)
      a.lse[static_cast<long long>(tok[nb]) * (a.Hkv * a.G) + hq] = (m[nb] * a.c + log2f(lt)) * kLn2;
  }
}

// ---------------------------------------------------------------------------
// fp32, on the fp32 MFMA (32 x 32 x 2): the same form with one block of 32 rows
// a wave and tiles of 32 keys.  P^T needs no packing: an accumulator register
// holds the two keys of one step.
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(kAttThreads) void attend_f32_kernel(AttArgs a) {
  constexpr int BM = kAttWaves * 32, BN = 32;
  constexpr int KJ = D / 8;                 // groups of four QK steps
  constexpr int DB = D / 32;
  constexpr int PK = D + 4, PV = D + 8;     // V's rows four apart: 32 banks apart
  constexpr int CH = D / 4, RP = kAttThreads / CH, NL = BN / RP;
  __shared__ __attribute__((aligned(16))) float s_k[2][BN * PK];
  __shared__ __attribute__((aligned(16))) float s_v[2][BN * PV];
  __shared__ AttRanges<BM> s_r;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int r32 = lane & 31, h = lane >> 5;
  const int g = blockIdx.x % a.Hkv;
  const int tile = a.tiles - 1 - static_cast<int>(blockIdx.x / a.Hkv);
  const int ntok = BM >> a.lg;
  const int t0 = tile * ntok;
  if (!att_ranges(a, t0, ntok, s_r)) return;
  const int last = min(t0 + ntok, s_r.end) - 1;
  const int kv0 = att_lo(s_r, t0, 0), lo_last = att_lo(s_r, t0, last - t0);
  const int nt = (last - kv0) / BN + 1;
  const int r = wave * 32 + r32;
  const bool row_ok = t0 + (r >> a.lg) <= last;
  const int tok = min(t0 + (r >> a.lg), last);
  const int lo = att_lo(s_r, t0, tok - t0);
  const int hq = g * a.G + (r & (a.G - 1));
  f32x4_t qf[KJ];
  const float sign = a.keep ? (a.flip ? -1.f : 1.f) : 0.f;
  const float* qp = static_cast<const float*>(a.q) + tok * a.ldq + hq * D + 4 * h;
#pragma unroll
  for (int x = 0; x < KJ; ++x) qf[x] = *reinterpret_cast<const f32x4_t*>(qp + 8 * x) * sign;
  const int w_first = t0 + ((wave * 32) >> a.lg);
  const int w_hi = min(t0 + ((wave * 32 + 31) >> a.lg), last);
  const int w_lo = att_lo(s_r, t0, min(w_first, last) - t0);
  const float* kp = static_cast<const float*>(a.k) + g * D;
  const float* vp = static_cast<const float*>(a.v) + g * D;
  const int lr = t / CH, lc = t % CH * 4;
  f32x4_t kr[NL], vr[NL];
  auto load = [&](int j) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int u = kv0 + j * BN + lr + i * RP;
      kr[i] = vr[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (u <= last) {
        kr[i] = *reinterpret_cast<const f32x4_t*>(kp + u * a.ldk + lc);
        vr[i] = *reinterpret_cast<const f32x4_t*>(vp + u * a.ldv + lc);
      }
    }
  };
  auto part = [&](int j) { return kv0 + j * BN < lo_last || kv0 + j * BN + BN - 1 > t0; };
  auto stash = [&](int j) {
    const int buf = j & 1;
    if (part(j)) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        uint4 x = __builtin_bit_cast(uint4, vr[i]);
        if (att_set_aside(x, false)) {
          atomicMin(&s_r.bad_lo, kv0 + j * BN + lr + i * RP);
          atomicMax(&s_r.bad_hi, kv0 + j * BN + lr + i * RP);
          vr[i] = __builtin_bit_cast(f32x4_t, x);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      *reinterpret_cast<f32x4_t*>(&s_k[buf][(lr + i * RP) * PK + lc]) = kr[i];
      *reinterpret_cast<f32x4_t*>(&s_v[buf][(lr + i * RP) * PV + lc]) = vr[i];
    }
  };
  f32x16_t o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  float m = -INFINITY, l = 0.f;
  load(0);
  stash(0);
  __syncthreads();
  for (int j = 0; j < nt; ++j) {
    const int buf = j & 1;
    if (j + 1 < nt) load(j + 1);
    const int k0 = kv0 + j * BN;
    if (w_first <= last && k0 <= w_hi && k0 + BN > w_lo) {
      f32x16_t s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int x = 0; x < KJ; ++x) {
        const f32x4_t kf = *reinterpret_cast<const f32x4_t*>(&s_k[buf][r32 * PK + 8 * x + 4 * h]);
#pragma unroll
        for (int y = 0; y < 4; ++y)
          s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[y], qf[x][y], s, 0, 0, 0);
      }
      if (part(j)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int u = k0 + 8 * (i / 4) + 4 * h + i % 4;
          if (u < lo || u > tok) s[i] = -INFINITY;
        }
      }
      float mx = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
      mx = xor_max<32>(mx);
      if (__any(mx > m)) {
        const float mn = fmaxf(m, mx);
        const float alpha = mn == m ? 1.f : exp2f((m - mn) * a.c);
        l *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] *= alpha;
        m = mn;
      }
      const float mm = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = exp2f((s[i] - mm) * a.c);
        l += s[i];
      }
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int db = 0; db < DB; ++db)
          o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(
              s_v[buf][(8 * (i / 4) + 4 * h + i % 4) * PV + 32 * db + r32], s[i], o[db], 0, 0, 0);
    }
    if (j + 1 < nt) stash(j + 1);
    __syncthreads();
  }
  for (int u = s_r.bad_lo; u <= s_r.bad_hi; ++u) {
    const float* x = vp + u * a.ldv + 4 * h;
    if (lo <= u && u <= tok) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] += att_not_finite(x[32 * db + 8 * (i / 4) + i % 4]);
    }
  }
  const float lt = xor_add<32>(l);
  if (!row_ok) return;
  const float inv = 1.f / lt;
  float* p = static_cast<float*>(a.out) + tok * a.ldo + hq * D + 4 * h;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 4; ++x)
      *reinterpret_cast<float4*>(p + 32 * db + 8 * x) =
          make_float4(o[db][4 * x] * inv, o[db][4 * x + 1] * inv, o[db][4 * x + 2] * inv, o[db][4 * x + 3] * inv);
  if (a.lse && h == 0)
    a.lse[static_cast<long long>(tok) * (a.Hkv * a.G) + hq] = (m * a.c + log2f(lt)) * kLn2;
}

template <typename K>
hipError_t att_launch(K kernel, int bm, AttArgs& a, hipStream_t s) {
  const int ntok = bm / a.G;
  a.tiles = (a.T + ntok - 1) / ntok;
  hipLaunchKernelGGL(kernel, dim3(a.tiles * a.Hkv), dim3(kAttThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prompt_attention(const ent_ctx* c, int B, int T, const void* q, long long ldq,
                                   const void* k, long long ldk, const void* v, long long ldv,
                                   const int* starts, void* out, long long ldo, float* lse,
                                   hipStream_t s) {
  AttArgs a{};
  a.q = q;
  a.ldq = ldq;
  a.k = k;
  a.ldk = ldk;
  a.v = v;
  a.ldv = ldv;
  a.starts = starts;
  a.out = out;
  a.ldo = ldo;
  a.lse = lse;
  a.B = B;
  a.T = T;
  a.Hkv = c->cfg.num_kv_heads;
  a.G = c->group;
  a.lg = __builtin_ctz(c->group);
  a.c = fabsf(c->cfg.scale) * kLog2e;
  const bool bf16 = c->cfg.kv_dtype == ENT_BF16;
  a.flip = c->cfg.scale < 0.f ? 0x80008000u : 0u;
  a.keep = c->cfg.scale == 0.f ? 0u : 0xffffffffu;
  if (a.c == 0.f) a.c = 1.f;
  if (!bf16)
    return c->cfg.head_dim == 128 ? att_launch(attend_f32_kernel<128>, kAttWaves * 32, a, s)
                                  : att_launch(attend_f32_kernel<64>, kAttWaves * 32, a, s);
  const bool big = static_cast<long long>(T) * a.G * a.Hkv >= 256ll * 2 * c->num_cu;
  if (c->cfg.head_dim == 128)
    return big ? att_launch(attend_bf16_kernel<128, 2>, 256, a, s)
               : att_launch(attend_bf16_kernel<128, 1>, 128, a, s);
  return big ? att_launch(attend_bf16_kernel<64, 2>, 256, a, s)
             : att_launch(attend_bf16_kernel<64, 1>, 128, a, s);
}

}  // namespace ent
