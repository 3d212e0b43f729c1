// Causal attention over packed prompts (ent_prompt_attention).
//
//   o_t = sum_u p_tu v_u,  p_t. = softmax over u of scale <q_t, k_u>,
//   u in [first token of t's request, t]
//
// A workgroup takes one KV head and a stretch of one request's tokens with all
// G query heads of the group: row r is token t0 + r / G, head g G + r % G.  So a K
// and V tile serves G heads, and few keys of a stretch lie across the diagonal.
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
#include <type_traits>

namespace ent {
namespace {

constexpr int kAttF32Threads = 256;

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
  int lg_ntok;         // log2 of a stretch's tokens
  float c;             // |scale| log2(e), > 0
  unsigned keep, flip; // queries are (q & keep) ^ flip: the scale's sign, or 0 where it is 0
};

// A workgroup's stretch: tokens [t0, last] of the request that begins at `start`.
// Requests are cut into stretches of ntok tokens from their first; the
// stretches are taken longest rows first, over all requests (a stretch's work
// grows with its place k in the request, so by falling k), which the host
// cannot order as it does not know the lengths.  Stretch number i is found from
// the starts alone: with L_b stretches in request b, sum_b max(0, L_b - k) of
// them have a place of k or more.  Every wave finds it for itself, lanes
// over requests.  Starts of any value are taken as inside [0, T].
struct AttStretch {
  int start, t0, last;
};

__device__ __forceinline__ bool att_stretch(const AttArgs& a, int i, int lg_ntok, int* s_starts,
                                            AttStretch& st) {
  const int lane = threadIdx.x & 63;
  for (int b = threadIdx.x; b <= a.B; b += blockDim.x) s_starts[b] = min(max(a.starts[b], 0), a.T);
  __syncthreads();
  const int ntok = 1 << lg_ntok;
  auto count = [&](int b) {
    return b < a.B ? (max(s_starts[b + 1] - s_starts[b], 0) + ntok - 1) >> lg_ntok : 0;
  };
  int most = 0;
  for (int b = lane; b < a.B; b += 64) most = max(most, count(b));
  most = static_cast<int>(wave_max_u(static_cast<unsigned>(most)));
  // Stretches of place k or more.
  auto from = [&](int k) {
    unsigned n = 0;
    for (int b = lane; b < a.B; b += 64) n += max(count(b) - k, 0);
    return static_cast<int>(wave_sum_u(n));
  };
  int lo = 0, hi = most, above = 0;         // place lo holds i or a later one; above = from(hi) <= i
  if (a.B == 1) {
    if (i >= most) return false;
    lo = most - 1 - i;
    above = i;
  } else {
    if (i >= from(0)) return false;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1, n = from(mid);
      if (n > i) {
        lo = mid;
      } else {
        hi = mid;
        above = n;
      }
    }
  }
  // The request: of those with more than lo stretches, number i - above.
  int want = i - above, b0 = 0;
  for (;; b0 += 64) {
    if (b0 >= a.B) return false;            // starts so far from ascending that the sums passed 32 bits
    const unsigned long long has = __ballot(count(b0 + lane) > lo);
    const int n = __popcll(has);
    if (want < n) {
      const int before = __popcll(has & ((1ull << lane) - 1));
      const unsigned long long it = __ballot(((has >> lane) & 1) && before == want);
      b0 += __builtin_ctzll(it);
      break;
    }
    want -= n;
  }
  st.start = __builtin_amdgcn_readfirstlane(s_starts[b0]);
  st.t0 = __builtin_amdgcn_readfirstlane(st.start + (lo << lg_ntok));
  st.last = __builtin_amdgcn_readfirstlane(min(st.t0 + ntok, s_starts[b0 + 1]) - 1);
  return true;
}

// A weight of 0 does not keep an infinity or a NaN out of a product.  In tiles
// that some row sees in part,
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
// Whether any of eight bf16 values is not finite.
__device__ __forceinline__ bool att_any_not_finite_bf16(uint4 w) {
  typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
  auto mag = [](unsigned x) { return __builtin_bit_cast(u16x2_t, x & 0x7fff7fffu); };
  const u16x2_t m = __builtin_elementwise_max(__builtin_elementwise_max(mag(w.x), mag(w.y)),
                                              __builtin_elementwise_max(mag(w.z), mag(w.w)));
  return m.x >= 0x7f80 || m.y >= 0x7f80;
}
__device__ __forceinline__ float att_not_finite(float x) {
  return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? x : 0.f;
}

// The key groups' partial results of each row group, into those of group 0.  The
// tiles are dead, behind a barrier.
template <int D, int RG, int KG, typename S>
__device__ __forceinline__ void att_merge(S& sh, int kg, int rg, float c, float& m, float& l,
                                          f32x16_t (&o)[D / 32]) {
  if (KG == 1) return;
  const int lane = threadIdx.x & 63;
  if (kg > 0) {
    const int x = (kg - 1) * RG + rg;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        sh.o[x][4 * db + i][lane] = f32x4_t{o[db][4 * i], o[db][4 * i + 1], o[db][4 * i + 2], o[db][4 * i + 3]};
    sh.ml[x][0][lane] = m;
    sh.ml[x][1][lane] = l;
  }
  __syncthreads();
  if (kg > 0) return;
#pragma unroll
  for (int y = 1; y < KG; ++y) {
    const int x = (y - 1) * RG + rg;
    const float mx = sh.ml[x][0][lane], lx = sh.ml[x][1][lane];
    const float mn = fmaxf(m, mx);
    const float f0 = m == mn ? 1.f : exp2f((m - mn) * c);
    const float f1 = mx == mn ? 1.f : exp2f((mx - mn) * c);
    m = mn;
    l = l * f0 + lx * f1;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4_t p = sh.o[x][4 * db + i][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[db][4 * i + e] = o[db][4 * i + e] * f0 + p[e] * f1;
      }
  }
}

// ---------------------------------------------------------------------------
// bf16.  RG groups of 32 rows times KG groups of keys, eight waves: wave (rg, kg)
// takes its rows through every KG-th part of the keys, and the KG partial results
// of a row are merged at the end.
//
// Per 32 rows and 64 keys a wave has 32 products of 32 cycles each at the matrix
// cores and about 1000 cycles of vector work (exponentials above all), so either
// is hidden only behind the other's in another wave: see `half`.  What it took,
// for 32768 tokens, 32 / 8 heads of 128: four waves of 64 rows each 12.1 ms, eight
// of 32 rows 8.4; the halves half a turn apart and operands read ahead 7.9; tiles
// straight to LDS instead of through registers, spread over the products, 7.3 =
// 1208 TFLOP/s, where a 16384^3 library product reaches 1381 and the clock falls
// to about 1.9 GHz for either.
// ---------------------------------------------------------------------------
// Waves a SIMD: for D = 64 two workgroups fit a CU.
constexpr int att_waves(int D, int KG) { return D == 64 && KG == 1 ? 4 : 2; }

template <int D, int RG, int KG, int BN>
struct AttBf16 {
  static constexpr int BT = KG * BN;
  union {
    struct {
      __attribute__((aligned(256))) uint16_t k[2][BT * D];
      __attribute__((aligned(256))) uint16_t v[2][BT * D];
      // The queries lie from k[1] on until the first turn; this is what they pass the tiles by.
      uint16_t over[RG * 32 > 3 * BT ? (RG * 32 - 3 * BT) * D : 8];
    };
    // Partial outputs of the key groups but the first, a column per lane.
    f32x4_t o[KG > 1 ? RG * (KG - 1) : 1][D / 8][64];
  };
  float ml[KG > 1 ? RG * (KG - 1) : 1][2][64];
  int bad_lo, bad_hi;                     // keys whose values were set aside
};

template <int D, int RG, int KG, int BN>
__global__ __launch_bounds__(RG * KG * 64, att_waves(D, KG)) void attend_bf16_kernel(AttArgs a) {
  using S = AttBf16<D, RG, KG, BN>;
  constexpr int BM = RG * 32;               // rows
  constexpr int BT = S::BT;                 // keys of a tile
  constexpr int KB = BN / 32;               // blocks of 32 keys of a wave
  constexpr int KS = D / 16;                // QK steps
  constexpr int DB = D / 32;                // blocks of 32 output dims
  constexpr int CH = D / 8;                 // 16 B pieces of a row
  constexpr int WV = RG * KG, RW = 64 / CH; // waves; rows of one load
  constexpr int NL = BT / (WV * RW);        // loads of a wave and tile
  __shared__ S sh;
  extern __shared__ int s_starts[];
  const int t = threadIdx.x, lane = t & 63;
  const int wv = __builtin_amdgcn_readfirstlane(t >> 6), rg = wv % RG, kg = wv / RG;
  const int r32 = lane & 31, h = lane >> 5;
  const int g = blockIdx.x % a.Hkv;
  AttStretch st;
  if (!att_stretch(a, blockIdx.x / a.Hkv, a.lg_ntok, s_starts, st)) return;
  const int t0 = st.t0, last = st.last, kv0 = st.start;
  const int nt = (last - kv0) / BT + 1;
  if (t == 0) {
    sh.bad_lo = 0x7fffffff;
    sh.bad_hi = -1;
  }

  const uint16_t* kp = static_cast<const uint16_t*>(a.k) + g * D;
  const uint16_t* vp = static_cast<const uint16_t*>(a.v) + g * D;
  // Tiles go straight to LDS, 16 B a lane, a wave's 64 lanes in a row; piece c of
  // row r lies at c ^ f(r), which spreads the reads below over all banks and is
  // had by what each lane loads.
  const int l_row = wv * RW + lane / CH, l_pos = lane % CH;
  const int k_src = (l_pos ^ (D == 128 ? l_row & 15 : (l_row >> 1) & 7)) * 8;
  // Load i's row is i WV RW on, which f sees in one bit at most.
  static_assert((WV * RW) % (D == 128 ? 8 : 16) == 0, "f of a load's rows");
  auto k_src_of = [&](int i) { return D == 128 && (i * WV * RW & 8) ? k_src ^ 64 : k_src; };
  const int v_src = (l_pos ^ (D == 128 ? (l_row & 3) << 2 : (l_row & 2) << 1)) * 8;
  typedef __attribute__((address_space(3))) char* lds_char;
  auto lds_at = [](const void* p) {
    return static_cast<unsigned>(reinterpret_cast<uintptr_t>((lds_char)(p)));
  };
  // Load i of tile j into the buffer at LDS address `at` (in asm: behind the
  // builtin the compiler waits for all of them before every read of LDS.  It
  // writes no register but m0, which the compiler sets anew wherever it uses it,
  // and `landed` and a barrier stand before its data's use).
  auto load = [&](const uint16_t* p, long long ld, int src, int j, unsigned at, int i) {
    const int u0 = min(kv0 + j * BT, last), over = last - u0;
    const uint16_t* base = p + u0 * ld;
    // Past the last token that token's row again (no row sees it there).
    const unsigned off = 2u * (min(l_row + i * WV * RW, over) * static_cast<unsigned>(ld) + src);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "s"(at + (wv + i * WV) * RW * D * 2), "v"(off), "s"(base));
  };
  constexpr unsigned SZ = BT * D * 2;          // tile x lies in buffer x % 2
  const unsigned k_lds = lds_at(sh.k[0]), v_lds = lds_at(sh.v[0]);
  // Keys [u, u + n) that some row of the stretch does not see whole.
  auto part = [&](int u, int n) { return u + n - 1 > t0; };
  // Waits for this wave's loads; in V tile j, if a part tile, sets aside what it
  // loaded itself.
  auto landed = [&](int j) {
    const unsigned b = j & 1 ? SZ : 0;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (part(kv0 + j * BT, BT)) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        uint4* x = reinterpret_cast<uint4*>(&sh.v[0][b / 2 + (wv + i * WV) * RW * D + lane * 8]);
        uint4 w = *x;
        if (att_any_not_finite_bf16(w)) {
          att_set_aside(w, true);
          *x = w;
          atomicMin(&sh.bad_lo, kv0 + j * BT + l_row + i * WV * RW);
          atomicMax(&sh.bad_hi, kv0 + j * BT + l_row + i * WV * RW);
        }
      }
    }
  };
#pragma unroll
  for (int i = 0; i < NL; ++i) load(kp, a.ldk, k_src_of(i), 0, k_lds, i);
  // The queries too, in whole rows, laid out as K's tiles: a lane's own pieces of its row
  // straight from memory are 16 B here and there: one of 16 tokens 9.7 us so, 8.3 in rows.
  constexpr int NQ = BM / (WV * RW);
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const int row = l_row + i * WV * RW;
    const uint16_t* p = static_cast<const uint16_t*>(a.q) +
                        min(t0 + (row >> a.lg), last) * a.ldq + (g * a.G + (row & (a.G - 1))) * D + k_src_of(i);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :: "s"(k_lds + SZ + (wv + i * WV) * RW * D * 2), "v"(p));
  }

  // This lane's row.
  const int r = rg * 32 + r32;
  const bool row_ok = t0 + (r >> a.lg) <= last;
  const int tok = min(t0 + (r >> a.lg), last);
  const int hq = g * a.G + (r & (a.G - 1));
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  bf16x8_t qf[KS];
  {
    const int sw = D == 128 ? r & 15 : (r >> 1) & 7;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      uint4 w = *reinterpret_cast<const uint4*>(&sh.k[1][r * D + ((2 * ks + h) ^ sw) * 8]);
      w = make_uint4((w.x & a.keep) ^ a.flip, (w.y & a.keep) ^ a.flip, (w.z & a.keep) ^ a.flip,
                     (w.w & a.keep) ^ a.flip);
      qf[ks] = __builtin_bit_cast(bf16x8_t, w);
    }
  }
  typedef f32x16_t Scores[KB];
  f32x16_t o[DB];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;

  const int k_row = kg * BN + r32;
  const unsigned k_at = k_row * D * 2 + ((h ^ (D == 128 ? k_row & 15 : (k_row >> 1) & 7)) << 4);
  auto mask = [&](Scores& s, int j) {
    const int k0 = kv0 + j * BT + kg * BN;
    if (!part(k0, BN)) return;
    const int hi = tok - k0 - 4 * h;        // the last key seen, from the lane's first
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (32 * kb + 8 * (i / 4) + i % 4 > hi) s[kb][i] = -INFINITY;
  };
  auto top = [&](const Scores& s) {
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kb][i]);
    return xor_max<32>(mx);
  };
  // The reference moves only where some row's scores pass it by 2^8: weights
  // up to 256 are as exact as those up to 1.
  auto move = [&](float mx) {
    if (__any((mx - m) * a.c > 8.f)) {
      const float mn = fmaxf(m, mx);
      const float alpha = mn == m ? 1.f : __builtin_amdgcn_exp2f((m - mn) * a.c);
      l *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= alpha;
      m = mn;
    }
  };
  bf16x8_t pf[2 * KB];
  auto weigh = [&](Scores& s, auto between) {
    const float mc = m == -INFINITY ? 0.f : m * a.c;
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 2 * KB; ++x) {
      // Weights to bf16 (half a step each, independent of each other); the sum
      // keeps them whole.  Outputs are then 1.25 to 1.3 times as far from the exact
      // ones as their own rounding to bf16 makes them (2500 tokens, 32 / 8 heads of
      // 128: 0.00209 of their norm, the rounding alone 0.00161).  A second bf16 part
      // leaves the rounding alone, for half as many products again: 87 us instead
      // of 67 there, 535 instead of 419 for 24 packed requests, 10.2 ms instead of
      // 7.45 for 32768 tokens.
      unsigned w[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        f32x2_t p;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          p[z] = __builtin_amdgcn_exp2f(fmaf(s[x / 2][8 * (x % 2) + 2 * y + z], a.c, -mc));
          sum[z] += p[z];
        }
        w[y] = __builtin_bit_cast(unsigned, __builtin_convertvector(p, bf16x2_t));
      }
      pf[x] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
      between(x);
    }
    l += sum[0] + sum[1];
  };
  const int v_row = kg * BN + 4 * h + ((lane & 15) >> 2);
  const unsigned v_at = v_row * D * 2 +
                        (((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^
                          (D == 128 ? (v_row & 3) << 2 : (v_row & 2) << 1)) << 4) + ((lane & 1) << 3);
  // A turn at the matrix cores: O += P V of the tile in buffer bv, then S = K Q^T
  // of the tile in buffer bk.  Operands are read PF products ahead of their use;
  // the barriers hold the order (the scheduler's own fetches them as late as
  // registers allow, and every product then waits for LDS).
  constexpr int NV = 2 * KB * DB, NK = KS * KB, PF = 4;
  auto matrix = [&](auto do_pv, auto do_qk, unsigned bv, Scores& s, unsigned bk, auto between) {
    constexpr int I0 = decltype(do_pv)::value ? 0 : NV, I1 = decltype(do_qk)::value ? NV + NK : NV;
    const unsigned av = v_at + v_lds + bv, ak = k_at + k_lds + bk;
    typedef s16x4_t __attribute__((address_space(3)))* lds_t;
    typedef __attribute__((address_space(3))) const bf16x8_t* lds_frag;
    bf16x8_t f[PF];
    auto read = [&](int i) -> bf16x8_t {
      if (i < NV) {
        // V^T: lane (dim, half): keys 16 x + 4 h + 0..3 and + 8.
        const unsigned p = (av ^ (64 * (i % DB))) + 32 * D * (i / DB);
        const s16x4_t v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(uintptr_t)p);
        const s16x4_t v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(uintptr_t)(p + 16 * D));
        const uint2 w0 = __builtin_bit_cast(uint2, v0), w1 = __builtin_bit_cast(uint2, v1);
        return __builtin_bit_cast(bf16x8_t, make_uint4(w0.x, w0.y, w1.x, w1.y));
      }
      return *((lds_frag)(uintptr_t)((ak ^ (32 * ((i - NV) / KB))) + 64 * D * ((i - NV) % KB)));
    };
    if (decltype(do_qk)::value) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
    }
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = I0; i < I0 + PF; ++i) f[i % PF] = read(i);
#pragma unroll
    for (int i = I0; i < I1; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      if (i < NV)
        o[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % PF], pf[i / DB], o[i % DB], 0, 0, 0);
      else
        s[(i - NV) % KB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % PF], qf[(i - NV) / KB],
                                                                  s[(i - NV) % KB], 0, 0, 0);
      if (i + PF < I1) f[i % PF] = read(i + PF);
      if (i < NV && i % DB == DB - 1) between(i / DB);
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(0);
  };
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  auto nothing = [](int) {};

  // Two halves of the workgroup, a wave of each on every SIMD, run half a turn
  // apart: while one is at the matrix cores (O += P V of its last tile, S of its
  // next), the other forms weights.
  auto turn = [] {
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
  };
  Scores s;
  // Piece x of what turns 2 j and 2 j + 1 bring: K(j + 1) and V(j).  What they
  // replace, K(j - 1) and V(j - 2), was last read in turn 2 j - 1.
  auto fetch = [&](int j, int x) {
    if (x < NL) load(kp, a.ldk, k_src_of(x), j + 1, k_lds + (j & 1 ? 0 : SZ), x);
    else load(vp, a.ldv, v_src, j, v_lds + (j & 1 ? SZ : 0), x - NL);
  };
  // ... spread over the 2 KB parts of what the half does in turn 2 j.
  auto spread = [&](int j, int part) {
#pragma unroll
    for (int i = 0; i < 2 * NL; ++i)
      if (i * KB / NL == part) fetch(j, i);
  };
  auto half = [&](auto late_t) {
    constexpr bool late = decltype(late_t)::value;
    auto weights = [&](int j) {
      mask(s, j);
      move(top(s));
      weigh(s, [&](int x) { if (late) spread(j + 1, x); });
    };
#pragma unroll
    for (int x = 0; x < 2 * NL; ++x) fetch(0, x);
    if (late) turn();
    matrix(no, yes, 0, s, 0, nothing);
    if (late) landed(0);
    turn();
    weights(0);
    if (!late) landed(0);
    turn();
    for (int j = 1; j < nt; ++j) {
      matrix(yes, yes, j & 1 ? 0 : SZ, s, j & 1 ? SZ : 0, [&](int x) { if (!late) spread(j, x); });
      if (late) landed(j);
      turn();
      weights(j);
      if (!late) landed(j);
      turn();
    }
    matrix(yes, no, nt & 1 ? 0 : SZ, s, 0, nothing);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (!late) turn();
  };
  turn();                                 // all have their queries
  if (wv >= WV / 2) half(yes); else half(no);
  __syncthreads();

  att_merge<D, RG, KG>(sh, kg, rg, a.c, m, l, o);
  if (kg > 0) return;
  for (int u = sh.bad_lo; u <= sh.bad_hi; ++u) {
    const uint16_t* x = vp + u * a.ldv + 4 * h;
    if (u <= tok) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          o[db][i] += att_not_finite(bf16_to_f32(x[32 * db + 8 * (i / 4) + i % 4]));
    }
  }

  const float lt = xor_add<32>(l);
  const float inv = 1.f / lt;
  // The wave's halves exchange dims, so that each stores eight in a row.
  uint16_t* p = static_cast<uint16_t*>(a.out) + tok * a.ldo + hq * D + 8 * h;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 4; x += 2) {
      unsigned w[2][2];
#pragma unroll
      for (int z = 0; z < 2; ++z)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const f32x2_t pe = {o[db][4 * (x + z) + 2 * y] * inv, o[db][4 * (x + z) + 2 * y + 1] * inv};
          w[z][y] = __builtin_bit_cast(unsigned, __builtin_convertvector(pe, bf16x2_t));
        }
      const auto s0 = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
      const auto s1 = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
      if (row_ok) *reinterpret_cast<uint4*>(p + 32 * db + 8 * x) = make_uint4(s0[0], s1[0], s0[1], s1[1]);
    }
  if (!row_ok) return;
  if (a.lse && h == 0)
    a.lse[static_cast<long long>(tok) * (a.Hkv * a.G) + hq] = (m * a.c + log2f(lt)) * kLn2;
}

// ---------------------------------------------------------------------------
// fp32, on the fp32 MFMA (32 x 32 x 2): the same form, four waves as RG row and KG
// key groups, a block of 32 keys a wave.  P^T needs no packing: an accumulator
// register holds the two keys of one step.  The matrix cores bound it (16 times
// the cycles of bf16 a product), so nothing is staggered.
// ---------------------------------------------------------------------------
template <int D, int RG, int KG>
struct AttF32 {
  static constexpr int BT = 32 * KG;
  static constexpr int PK = D + 4, PV = D + 8;              // V's rows four apart: 32 banks apart
  // Two buffers where two workgroups still fit a CU's LDS; else one, and a barrier more a
  // tile.  us at one workgroup of two buffers and two of one (8 / 8 heads of 64): four
  // requests of 2000 tokens 288, 219; of 176 to 464 tokens 22.7, 23.6.  At 128 dims a
  // workgroup has a CU to itself for its registers (304 to 416 a lane), so <128, 2, 2>
  // could have two buffers; they gain nothing (32 / 8 heads, two and one: one request of
  // 1000 tokens 106.2, 105.0, of 2000 381.5, 378.8; four of 300 60.4, 59.9), and
  // <128, 1, 4> has no LDS for them.
  static constexpr int NBUF = 2 * BT * (PK + PV) * 4 <= 76000 ? 2 : 1;
  union {
    struct {
      __attribute__((aligned(16))) float k[NBUF][BT * PK];
      __attribute__((aligned(16))) float v[NBUF][BT * PV];
    };
    f32x4_t o[KG > 1 ? RG * (KG - 1) : 1][D / 8][64];
  };
  float ml[KG > 1 ? RG * (KG - 1) : 1][2][64];
  int bad_lo, bad_hi;
};

template <int D, int RG, int KG>
__global__ __launch_bounds__(kAttF32Threads) void attend_f32_kernel(AttArgs a) {
  using S = AttF32<D, RG, KG>;
  constexpr int BM = RG * 32, BT = S::BT, PK = S::PK, PV = S::PV, NBUF = S::NBUF;
  constexpr int KJ = D / 8;                 // groups of four QK steps
  constexpr int DB = D / 32;
  constexpr int CH = D / 4, RP = kAttF32Threads / CH, NL = BT / RP;
  static_assert(RG * KG * 64 == kAttF32Threads, "four waves");
  __shared__ S sh;
  extern __shared__ int s_starts[];
  const int t = threadIdx.x, lane = t & 63;
  const int rg = (t >> 6) % RG, kg = (t >> 6) / RG;
  const int r32 = lane & 31, h = lane >> 5;
  const int g = blockIdx.x % a.Hkv;
  AttStretch st;
  if (!att_stretch(a, blockIdx.x / a.Hkv, a.lg_ntok, s_starts, st)) return;
  const int t0 = st.t0, last = st.last, kv0 = st.start;
  const int nt = (last - kv0) / BT + 1;
  if (t == 0) {
    sh.bad_lo = 0x7fffffff;
    sh.bad_hi = -1;
  }
  __syncthreads();
  const int r = rg * 32 + r32;
  const bool row_ok = t0 + (r >> a.lg) <= last;
  const int tok = min(t0 + (r >> a.lg), last);
  const int hq = g * a.G + (r & (a.G - 1));
  const float sign = a.keep ? (a.flip ? -1.f : 1.f) : 0.f;
  const float* qp = static_cast<const float*>(a.q) + tok * a.ldq + hq * D + 4 * h;
  f32x4_t qf[KJ];
#pragma unroll
  for (int x = 0; x < KJ; ++x) qf[x] = *reinterpret_cast<const f32x4_t*>(qp + 8 * x) * sign;
  const int w_hi = min(t0 + ((rg * 32 + 31) >> a.lg), last);   // the last key that this wave's rows see
  const float* kp = static_cast<const float*>(a.k) + g * D;
  const float* vp = static_cast<const float*>(a.v) + g * D;
  const int lr = t / CH, lc = t % CH * 4;
  f32x4_t kr[NL], vr[NL];
  auto load = [&](int j) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int u = kv0 + j * BT + lr + i * RP;
      kr[i] = vr[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (u <= last) {
        kr[i] = *reinterpret_cast<const f32x4_t*>(kp + u * a.ldk + lc);
        vr[i] = *reinterpret_cast<const f32x4_t*>(vp + u * a.ldv + lc);
      }
    }
  };
  auto part = [&](int u, int n) { return u + n - 1 > t0; };
  auto stash = [&](int j) {
    const int buf = NBUF == 2 ? j & 1 : 0;
    if (part(kv0 + j * BT, BT)) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        uint4 x = __builtin_bit_cast(uint4, vr[i]);
        if (att_set_aside(x, false)) {
          atomicMin(&sh.bad_lo, kv0 + j * BT + lr + i * RP);
          atomicMax(&sh.bad_hi, kv0 + j * BT + lr + i * RP);
          vr[i] = __builtin_bit_cast(f32x4_t, x);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      *reinterpret_cast<f32x4_t*>(&sh.k[buf][(lr + i * RP) * PK + lc]) = kr[i];
      *reinterpret_cast<f32x4_t*>(&sh.v[buf][(lr + i * RP) * PV + lc]) = vr[i];
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
    const int buf = NBUF == 2 ? j & 1 : 0;
    if (j + 1 < nt) load(j + 1);
    const int k0 = kv0 + j * BT + kg * 32;
    if (k0 <= w_hi) {
      f32x16_t s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int x = 0; x < KJ; ++x) {
        const f32x4_t kf =
            *reinterpret_cast<const f32x4_t*>(&sh.k[buf][(kg * 32 + r32) * PK + 8 * x + 4 * h]);
#pragma unroll
        for (int y = 0; y < 4; ++y)
          s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[y], qf[x][y], s, 0, 0, 0);
      }
      if (part(k0, 32)) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (8 * (i / 4) + i % 4 > tok - k0 - 4 * h) s[i] = -INFINITY;
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
              sh.v[buf][(kg * 32 + 8 * (i / 4) + 4 * h + i % 4) * PV + 32 * db + r32], s[i], o[db], 0, 0, 0);
    }
    if (NBUF == 1) __syncthreads();
    if (j + 1 < nt) stash(j + 1);
    __syncthreads();
  }
  att_merge<D, RG, KG>(sh, kg, rg, a.c, m, l, o);
  if (kg > 0) return;
  for (int u = sh.bad_lo; u <= sh.bad_hi; ++u) {
    const float* x = vp + u * a.ldv + 4 * h;
    if (u <= tok) {
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
hipError_t att_launch(K kernel, int rows, int threads, AttArgs& a, hipStream_t s) {
  const int ntok = rows / a.G;
  a.lg_ntok = __builtin_ctz(ntok);
  const int n = (a.T + ntok - 1) / ntok + std::min(a.B, a.T);   // stretches, at most
  hipLaunchKernelGGL(kernel, dim3(n * a.Hkv), dim3(threads), (a.B + 1) * sizeof(int), s, a);
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
  // The keys are split over waves where the rows alone do not fill the CUs: a workgroup
  // takes a half or a quarter of the rows while that leaves each CU one at most, and a
  // half also where requests of 1024 tokens and more would leave CUs idle behind the
  // longest rows.  us with 256, 128 and 64 rows a workgroup: one request of 512 tokens
  // (32 / 8 heads of 128) 18.1, 13.5, 12.5; four of 300 15.3, 20.1, 30.0; one of 2500
  // 65.8, 69.0, 91.9; 3000 and 500 tokens (16 / 1 heads of 64) 55.0, 35.7, 38.4.
  const long long rows = static_cast<long long>(T) * a.G * a.Hkv;
  const long long cus = c->num_cu;
  if (!bf16) {
    // Fewer rows a workgroup here, since each takes longer.  us with 128, 64 and 32 rows a
    // workgroup: eight requests of 2048 tokens (32 / 8 heads of 128) 2720, 3090, -; one of
    // 1000 163, 106, 140; four of 2000 (8 / 8 heads of 64) 240, 201, 219; one of 2000 -,
    // 107, 76; 300, 500 and 700 (16 / 4) 69, 46, 39.
    const int rg = rows >= 256 * cus ? 4 : rows >= 96 * cus ? 2 : 1;
    if (c->cfg.head_dim == 128)
      return rg == 4   ? att_launch(attend_f32_kernel<128, 4, 1>, 128, kAttF32Threads, a, s)
             : rg == 2 ? att_launch(attend_f32_kernel<128, 2, 2>, 64, kAttF32Threads, a, s)
                       : att_launch(attend_f32_kernel<128, 1, 4>, 32, kAttF32Threads, a, s);
    return rg == 4   ? att_launch(attend_f32_kernel<64, 4, 1>, 128, kAttF32Threads, a, s)
           : rg == 2 ? att_launch(attend_f32_kernel<64, 2, 2>, 64, kAttF32Threads, a, s)
                     : att_launch(attend_f32_kernel<64, 1, 4>, 32, kAttF32Threads, a, s);
  }
  // Short requests (96 tokens on average, padding with them) take what a workgroup costs
  // beside its tiles, which several small ones on a CU hide for each other.  us with the
  // rule below and with two waves of 32 rows: one request of 16 tokens (32 / 8 heads of
  // 128) 8.4, 5.6; 200 of 1 53, 13; 4096 of 1 2180, 810; 512 of 64 214, 205; 300 of 96
  // 205, 180; 200 of 128 158, 171; 100 of 40 (8 / 8 heads of 64) 15.6, 7.3; but one of
  // 8000 among 200 of 10 524, 587.
  if (T <= 96ll * B)
    return c->cfg.head_dim == 128 ? att_launch(attend_bf16_kernel<128, 2, 1, 32>, 64, 128, a, s)
                                  : att_launch(attend_bf16_kernel<64, 2, 1, 32>, 64, 128, a, s);
  const int split = rows <= 64 * cus ? 4
                    : rows <= 128 * cus || (rows < 256 * cus && T >= 1024ll * B) ? 2 : 1;
  if (c->cfg.head_dim == 128)
    return split == 4   ? att_launch(attend_bf16_kernel<128, 2, 4, 32>, 64, 512, a, s)
           : split == 2 ? att_launch(attend_bf16_kernel<128, 4, 2, 64>, 128, 512, a, s)
                        : att_launch(attend_bf16_kernel<128, 8, 1, 64>, 256, 512, a, s);
  return split == 4   ? att_launch(attend_bf16_kernel<64, 2, 4, 32>, 64, 512, a, s)
         : split == 2 ? att_launch(attend_bf16_kernel<64, 4, 2, 64>, 128, 512, a, s)
                      : att_launch(attend_bf16_kernel<64, 8, 1, 64>, 256, 512, a, s);
}

}  // namespace ent
