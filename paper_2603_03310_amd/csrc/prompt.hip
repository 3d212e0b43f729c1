// Prompts into the paged cache: the plan of a batch of requests (block tables,
// packed starts, slot map), the store of packed keys and values at a slot map
// with the blocks' mean keys, and the store and the one-token append of an
// 8-bit cache.

#include "quant_dev.h"

#include <algorithm>

namespace ent {
namespace {

// ---------------------------------------------------------------------------
// The plan.  Request b holds ctx_b tokens in have_b = ceil(ctx_b / 16) blocks
// and gets n_b more, in ceil((ctx_b + n_b) / 16) - have_b blocks of the free
// list.  Both prefix sums (tokens, blocks) over the batch are formed by every
// workgroup for itself, from 8 B a request (at most 32 KB, in L2 after the
// first), so one launch does the whole plan: each workgroup then fills its part
// of the slot map and of the new table entries, the first also writes starts
// and lengths, and the one that finishes last moves the free list's head,
// which all have read by then.
//
// Requests are admitted in order while tokens and blocks last; the inclusive
// sums only grow, so "both fit" holds for a prefix of the batch and needs no
// second pass.
// ---------------------------------------------------------------------------
constexpr int kPlanThreads = 256;
constexpr int kPlanTokens = 2048;      // slots per workgroup

struct PlanArgs {
  const int* n_new;
  const int* ctx;
  int* tables;
  const int* ids;
  int n_ids;
  int* range;             // free list: [head, end)
  int B, MAXB, P, max_tokens;
  int* starts;
  long long* slots;
  int* new_lens;          // nullable
  unsigned* ticket;       // 0 between launches
  unsigned* flags;
};

// Sums of one value per thread before this thread's, and of all (two at once).
__device__ __forceinline__ void plan_scan(int& a, int& b, int& ta, int& tb, int* s_red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int kW = kPlanThreads / 64;
  const int ia = static_cast<int>(wave_scan_u(static_cast<unsigned>(a)));
  const int ib = static_cast<int>(wave_scan_u(static_cast<unsigned>(b)));
  if (lane == 63) {
    s_red[wave] = ia;
    s_red[kW + wave] = ib;
  }
  __syncthreads();
  int oa = ia - a, ob = ib - b;
  ta = tb = 0;
#pragma unroll
  for (int w = 0; w < kW; ++w) {
    if (w < wave) {
      oa += s_red[w];
      ob += s_red[kW + w];
    }
    ta += s_red[w];
    tb += s_red[kW + w];
  }
  a = oa;
  b = ob;
}

// The largest b in [0, B) with s[b] <= x (s ascending, s[0] <= x).
__device__ __forceinline__ int plan_find(const int* s, int B, int x) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs a) {
  extern __shared__ int s_mem[];
  __shared__ int s_red[2 * kPlanThreads / 64];
  int* s_tok = s_mem;                // [B + 1] packed start of each request
  int* s_blk = s_tok + a.B + 1;      // [B + 1] new blocks before it
  int* s_ctx = s_blk + a.B + 1;      // [B]
  const int t = threadIdx.x;
  const int per = (a.B + kPlanThreads - 1) / kPlanThreads;
  int head = a.range[0];
  const int end = a.range[1];
  const bool ring_ok = head >= 0 && head <= end && end <= a.n_ids;
  const int avail = ring_ok ? end - head : 0;
  if (!ring_ok) head = 0;
  unsigned bad = ring_ok ? 0u : ENT_DEV_BAD_TABLE;
  // n and ctx of a request; a bad one gets nothing.
  auto request = [&](int b, int& n, int& ctx, unsigned& f) {
    n = a.n_new[b];
    ctx = a.ctx[b];
    const int room = a.MAXB * kBlock;
    if (n < 0 || ctx < 0 || ctx > room) {
      f |= ENT_DEV_BAD_CTXLEN;
      n = 0;
    } else if (n > room - ctx) {
      f |= ENT_DEV_CACHE_FULL;
      n = 0;
    }
    ctx = min(max(ctx, 0), room);
  };
  int tok = 0, blk = 0;
  for (int i = 0; i < per; ++i) {
    const int b = t * per + i;
    if (b < a.B) {
      int n, ctx;
      request(b, n, ctx, bad);
      tok += n;
      blk += (ctx + n + kBlock - 1) / kBlock - (ctx + kBlock - 1) / kBlock;
    }
  }
  int all_tok, all_blk;
  plan_scan(tok, blk, all_tok, all_blk, s_red);
  // This thread's requests in turn; what does not fit counts nothing, and
  // neither does anything behind it.
  int last_tok = 0, last_blk = 0;    // sums of the admitted ones of this thread's
  for (int i = 0; i < per; ++i) {
    const int b = t * per + i;
    if (b < a.B) {
      int n, ctx;
      unsigned f = 0;
      request(b, n, ctx, f);
      const int need = (ctx + n + kBlock - 1) / kBlock - (ctx + kBlock - 1) / kBlock;
      s_tok[b] = tok;
      s_blk[b] = blk;
      s_ctx[b] = ctx;
      tok += n;
      blk += need;
      if (tok <= a.max_tokens && blk <= avail) {
        last_tok = tok;
        last_blk = blk;
      }
    }
  }
  // Totals of the admitted prefix: the largest sums that fit.
  last_tok = static_cast<int>(wave_max_u(static_cast<unsigned>(last_tok)));
  last_blk = static_cast<int>(wave_max_u(static_cast<unsigned>(last_blk)));
  __syncthreads();                   // s_red is read no more
  if ((t & 63) == 0) {
    s_red[t >> 6] = last_tok;
    s_red[kPlanThreads / 64 + (t >> 6)] = last_blk;
  }
  __syncthreads();
  int total = 0, taken = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    total = max(total, s_red[w]);
    taken = max(taken, s_red[kPlanThreads / 64 + w]);
  }
  if (all_tok > total || all_blk > taken) bad |= ENT_DEV_CACHE_FULL;
  for (int b = t; b < a.B; b += kPlanThreads) {
    s_tok[b] = min(s_tok[b], total);
    s_blk[b] = min(s_blk[b], taken);
  }
  if (t == 0) {
    s_tok[a.B] = total;
    s_blk[a.B] = taken;
  }
  __syncthreads();

  // A free id by its place in the list, -1 (flagged) where it is no block.
  auto free_id = [&](int i) {
    const int p = a.ids[head + i];
    if (p >= 0 && p < a.P) return p;
    bad |= ENT_DEV_BAD_TABLE;
    return -1;
  };
  // Slots of this workgroup's tokens, two consecutive ones a thread and step.
  const int t0 = blockIdx.x * kPlanTokens;
  const int t1 = min(a.max_tokens, t0 + kPlanTokens);
  auto slot_of = [&](int x) -> long long {
    if (x >= total) return -1;
    const int b = plan_find(s_tok, a.B, x);
    const int pos = s_ctx[b] + x - s_tok[b];
    const int j = pos / kBlock, have = (s_ctx[b] + kBlock - 1) / kBlock;
    int p;
    if (j < have) {
      p = a.tables[static_cast<long long>(b) * a.MAXB + j];
      if (p < 0 || p >= a.P) {
        bad |= ENT_DEV_BAD_TABLE;
        p = -1;
      }
    } else {
      p = free_id(s_blk[b] + j - have);
    }
    return p < 0 ? -1 : static_cast<long long>(p) * kBlock + pos % kBlock;
  };
  for (int x = t0 + t; x < t1; x += kPlanThreads) a.slots[x] = slot_of(x);
  // New table entries, dealt to all workgroups.
  for (int e = blockIdx.x * kPlanThreads + t; e < taken; e += gridDim.x * kPlanThreads) {
    const int b = plan_find(s_blk, a.B, e);
    const int j = (s_ctx[b] + kBlock - 1) / kBlock + e - s_blk[b];
    a.tables[static_cast<long long>(b) * a.MAXB + j] = free_id(e);
  }
  if (blockIdx.x == 0) {
    for (int b = t; b <= a.B; b += kPlanThreads) {
      a.starts[b] = s_tok[b];
      if (a.new_lens && b < a.B) a.new_lens[b] = a.ctx[b] + s_tok[b + 1] - s_tok[b];
    }
  }
  if (bad) raise_flag(a.flags, bad);
  __syncthreads();
  if (t == 0 && ring_ok && atomicInc(a.ticket, gridDim.x - 1) == gridDim.x - 1)
    a.range[0] = head + taken;
}

// ---------------------------------------------------------------------------
// Stores.  The slot map gives each packed token its place (block 16 + row).  A
// run is a maximal stretch of consecutive tokens in consecutive rows of one
// block; the workgroups of one group of 16 packed tokens handle the runs that
// begin there (one, where the map is a plan's and the requests are longer than
// a block), for their KV heads, so a tile is written by one workgroup.
// Memory-bound: every thread has its 16 B of K and of V in flight before
// anything waits; V goes through LDS to its dim-major form.
// ---------------------------------------------------------------------------
constexpr int kStoreThreads = 256;

struct StoreArgs {
  const void* k;
  long long ldk;
  const void* v;
  long long ldv;
  const long long* slots;
  int T;
  void* kc;
  void* vc;
  float* ks;              // scales (8-bit caches)
  float* vs;
  float* ksum;            // nullable
  int Hkv, P;
  unsigned* flags;
};

// The runs that begin at packed tokens [16 x, 16 x + 16): calls
// f(first token, block, first row, rows) for each.  Every wave finds them for
// itself: lane i holds the slot of token 16 x - 1 + i.
template <typename F>
__device__ __forceinline__ void each_run(const StoreArgs& a, int x, F f) {
  const int lane = threadIdx.x & 63;
  const long long tk = static_cast<long long>(x) * kBlock - 1 + lane;
  const long long lim = static_cast<long long>(a.P) * kBlock;
  long long sl = -1;
  if (tk >= 0 && tk < a.T && lane <= 2 * kBlock) {
    sl = a.slots[tk];
    if (sl < -1 || sl >= lim) {
      if (threadIdx.x < 64) raise_flag(a.flags, ENT_DEV_BAD_TABLE);
      sl = -1;
    }
  }
  const int lo = static_cast<int>(sl), hi = static_cast<int>(sl >> 32);
  const long long before = (static_cast<long long>(__shfl_up(hi, 1)) << 32) |
                           static_cast<unsigned>(__shfl_up(lo, 1));
  const bool cont = lane > 0 && sl >= 0 && sl == before + 1 && (sl & (kBlock - 1)) != 0;
  const unsigned long long conts = __ballot(cont);
  unsigned long long starts = __ballot(sl >= 0 && !cont) & (0xffffull << 1);   // lanes 1 .. 16
  while (starts) {
    const int i = __builtin_ctzll(starts);
    starts &= starts - 1;
    const int rows = 1 + static_cast<int>(__builtin_ctzll(~(conts >> (i + 1))));
    const long long s = (static_cast<long long>(lane_at(hi, i)) << 32) |
                        static_cast<unsigned>(lane_at(lo, i));
    f(x * kBlock - 1 + i, static_cast<int>(s / kBlock), static_cast<int>(s % kBlock), rows);
  }
}

template <typename T>
__device__ __forceinline__ float elem_f32(T x);
template <>
__device__ __forceinline__ float elem_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ float elem_f32<uint16_t>(uint16_t x) { return bf16_to_f32(x); }

// Caches of the inputs' type.
template <typename T, int D>
__global__ __launch_bounds__(kStoreThreads) void store_kernel(StoreArgs a) {
  constexpr int VE = 16 / sizeof(T);                 // elements of a 16 B piece
  constexpr int I = kBlock * D / VE;                 // pieces of a tile
  constexpr int HW = I < kStoreThreads ? kStoreThreads / I : 1;   // heads of a workgroup
  constexpr int NI = HW * I / kStoreThreads;
  constexpr int PITCH = D + VE;
  __shared__ __attribute__((aligned(16))) T s_k[HW * kBlock * PITCH], s_v[HW * kBlock * PITCH];
  const T* k = static_cast<const T*>(a.k);
  const T* v = static_cast<const T*>(a.v);
  T* kc = static_cast<T*>(a.kc);
  T* vc = static_cast<T*>(a.vc);
  const int g0 = blockIdx.y * HW;
  each_run(a, blockIdx.x, [&](int tok, int p, int row0, int rows) {
    const int row1 = row0 + rows;
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NI; ++n) {
      const int it = threadIdx.x + n * kStoreThreads;
      const int hh = it / I, r = it % I, row = r / (D / VE), c = r % (D / VE) * VE;
      const int g = g0 + hh;
      if (g < a.Hkv && row < row1) {
        const long long tile = (static_cast<long long>(p) * a.Hkv + g) * kBlock * D;
        T* const lk = s_k + (hh * kBlock + row) * PITCH + c;
        T* const lv = s_v + (hh * kBlock + row) * PITCH + c;
        if (row >= row0) {
          const long long src = tok + row - row0;
          const uint4 kx = *reinterpret_cast<const uint4*>(k + src * a.ldk + g * D + c);
          const uint4 vx = *reinterpret_cast<const uint4*>(v + src * a.ldv + g * D + c);
          *reinterpret_cast<uint4*>(lk) = kx;
          *reinterpret_cast<uint4*>(lv) = vx;
          *reinterpret_cast<uint4*>(kc + tile + row * D + c) = kx;
        } else if (a.ksum) {
          // An earlier row of the block, for its mean key.
          *reinterpret_cast<uint4*>(lk) = *reinterpret_cast<const uint4*>(kc + tile + row * D + c);
        }
      }
    }
    __syncthreads();
    if (rows == kBlock) {
#pragma unroll
      for (int n = 0; n < NI; ++n) {
        const int it = threadIdx.x + n * kStoreThreads;
        const int hh = it / I, r = it % I, d = r / (kBlock / VE), s = r % (kBlock / VE) * VE;
        if (g0 + hh < a.Hkv) {
          const long long tile = (static_cast<long long>(p) * a.Hkv + g0 + hh) * kBlock * D;
          T x[VE];
#pragma unroll
          for (int i = 0; i < VE; ++i) x[i] = s_v[(hh * kBlock + s + i) * PITCH + d];
          uint4 w;
          __builtin_memcpy(&w, x, 16);
          *reinterpret_cast<uint4*>(vc + tile + d * kBlock + s) = w;
        }
      }
    } else {
      // Part of a block: the other rows stay as they are.
      for (int e = threadIdx.x; e < HW * D * kBlock; e += kStoreThreads) {
        const int hh = e / (D * kBlock), d = e / kBlock % D, s = e % kBlock;
        if (g0 + hh < a.Hkv && s >= row0 && s < row1)
          vc[(static_cast<long long>(p) * a.Hkv + g0 + hh) * kBlock * D + d * kBlock + s] =
              s_v[(hh * kBlock + s) * PITCH + d];
      }
    }
    if (a.ksum) {
      for (int e = threadIdx.x; e < HW * D; e += kStoreThreads) {
        const int hh = e / D, d = e % D;
        if (g0 + hh < a.Hkv) {
          // In row order, as ent_block_summary adds.
          float sum = 0.f;
          for (int s = 0; s < row1; ++s) sum += elem_f32<T>(s_k[(hh * kBlock + s) * PITCH + d]);
          a.ksum[(static_cast<long long>(p) * a.Hkv + g0 + hh) * D + d] =
              __fdiv_rn(sum, static_cast<float>(row1));
        }
      }
    }
  });
}

// One run of an 8-bit cache's block for HW heads (bf16 inputs): the tile's new
// scale from the new rows' largest magnitude and, where the block had rows, its
// old scale; codes; V transposed through LDS; old codes rounded again where the
// scale grew; the mean of the keys that the cache then holds (a sum of 16 codes
// is exact in 32 bits, so its order is free).  Thread (row, 8 dims).
template <int D>
struct Store8 {
  static constexpr int I = kBlock * D / 8;                            // threads of a tile
  static constexpr int HW = kStoreThreads / I;
  static constexpr int WT = I / 64;                                   // waves of a tile
  static constexpr int PITCH = D + 16;
  __attribute__((aligned(16))) unsigned char k[HW * kBlock * PITCH];
  __attribute__((aligned(16))) unsigned char v[HW * kBlock * PITCH];
  float top[2][kStoreThreads / 64];
};

__device__ __forceinline__ void load_bf16_row(const uint16_t* p, float (&x)[8]) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(u[i] << 16);
    x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}

template <int D>
__device__ __forceinline__ void store8_run(const StoreArgs& a, Store8<D>& sh, int g0,
                                           const uint16_t* k, const uint16_t* v, int p, int row0,
                                           int rows) {
  using S = Store8<D>;
  const int t = threadIdx.x, hh = t / S::I, r = t % S::I, row = r / (D / 8), c = r % (D / 8) * 8;
  const int g = g0 + hh, row1 = row0 + rows;
  const bool head = g < a.Hkv, fresh = head && row >= row0 && row < row1, old = head && row < row0;
  const long long tg = static_cast<long long>(p) * a.Hkv + g;
  unsigned char* kc = static_cast<unsigned char*>(a.kc) + tg * kBlock * D;
  unsigned char* vc = static_cast<unsigned char*>(a.vc) + tg * kBlock * D;
  float kx[8], vx[8];
  uint2 kold = make_uint2(0u, 0u), vold = kold;
  float ks0 = 0.f, vs0 = 0.f;
  if (fresh) {
    load_bf16_row(k + (row - row0) * a.ldk + g * D + c, kx);
    load_bf16_row(v + (row - row0) * a.ldv + g * D + c, vx);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) kx[i] = vx[i] = 0.f;
  }
  if (head && row0 > 0) {
    ks0 = a.ks[tg];
    vs0 = a.vs[tg];
    if (old) kold = *reinterpret_cast<const uint2*>(kc + row * D + c);
  }
  float kt = 0.f, vt = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    kt = fmaxf(kt, q8_mag(kx[i]));
    vt = fmaxf(vt, q8_mag(vx[i]));
  }
  kt = wave_max(kt);
  vt = wave_max(vt);
  __syncthreads();                    // the last run's LDS is read no more
  if ((t & 63) == 0) {
    sh.top[0][t >> 6] = kt;
    sh.top[1][t >> 6] = vt;
  }
  __syncthreads();
  kt = vt = 0.f;
#pragma unroll
  for (int w = 0; w < S::WT; ++w) {
    kt = fmaxf(kt, sh.top[0][hh * S::WT + w]);
    vt = fmaxf(vt, sh.top[1][hh * S::WT + w]);
  }
  const float kn = q8_scale(kt), vn = q8_scale(vt);
  const float ks = row0 > 0 && ks0 > kn ? ks0 : kn, vs = row0 > 0 && vs0 > vn ? vs0 : vn;
  const bool kgrow = row0 > 0 && ks > ks0, vgrow = row0 > 0 && vs > vs0;
  // The reciprocal is exact but for a kept scale of the caller's own making
  // that is no power of two.
  auto codes = [](const float (&x)[8], float s) {
    const float inv = __fdiv_rn(1.f, s);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i] * inv;
    return make_uint2(q8_pack4(y[0], y[1], y[2], y[3]), q8_pack4(y[4], y[5], y[6], y[7]));
  };
  auto again = [](uint2 w, float f) {
    float y[8];
    q8_unpack4(w.x, y);
    q8_unpack4(w.y, y + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] *= f;
    return make_uint2(q8_pack4(y[0], y[1], y[2], y[3]), q8_pack4(y[4], y[5], y[6], y[7]));
  };
  unsigned char* const lk = sh.k + (hh * kBlock + row) * S::PITCH + c;
  if (fresh) {
    const uint2 kw = codes(kx, ks);
    *reinterpret_cast<uint2*>(kc + row * D + c) = kw;
    *reinterpret_cast<uint2*>(lk) = kw;
    *reinterpret_cast<uint2*>(sh.v + (hh * kBlock + row) * S::PITCH + c) = codes(vx, vs);
  } else if (old) {
    if (kgrow) {
      kold = again(kold, ks0 / ks);
      *reinterpret_cast<uint2*>(kc + row * D + c) = kold;
    }
    *reinterpret_cast<uint2*>(lk) = kold;
  }
  if (head && r == 0) {
    a.ks[tg] = ks;
    a.vs[tg] = vs;
  }
  __syncthreads();
  // V: a thread has 8 rows of one dim.
  const int d = r / 2, s0 = r % 2 * 8;
  if (head && s0 < row1) {
    unsigned char* const at = vc + d * kBlock + s0;
    if (vgrow && s0 < row0) vold = again(*reinterpret_cast<const uint2*>(at), vs0 / vs);
    unsigned char x[8];
    __builtin_memcpy(x, &vold, 8);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (s0 + i >= row0 && s0 + i < row1) x[i] = sh.v[(hh * kBlock + s0 + i) * S::PITCH + d];
    if (s0 >= row0 && s0 + 8 <= row1) {
      uint2 w;
      __builtin_memcpy(&w, x, 8);
      *reinterpret_cast<uint2*>(at) = w;
    } else {
      const int first = vgrow ? 0 : row0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (s0 + i >= first && s0 + i < row1) at[i] = x[i];
    }
  }
  if (a.ksum && head) {
    for (int e = r; e < D; e += S::I) {
      float sum = 0.f;
#pragma unroll
      for (int s = 0; s < kBlock; ++s) {
        const q8_f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8(sh.k[(hh * kBlock + s) * S::PITCH + e], false);
        if (s < row1) sum += x.x;
      }
      a.ksum[tg * D + e] = __fdiv_rn(sum, static_cast<float>(row1)) * ks;
    }
  }
}

template <int D>
__global__ __launch_bounds__(kStoreThreads) void store_q8_kernel(StoreArgs a) {
  __shared__ Store8<D> sh;
  each_run(a, blockIdx.x, [&](int tok, int p, int row0, int rows) {
    store8_run<D>(a, sh, blockIdx.y * Store8<D>::HW,
                  static_cast<const uint16_t*>(a.k) + tok * a.ldk,
                  static_cast<const uint16_t*>(a.v) + tok * a.ldv, p, row0, rows);
  });
}

// One token per sequence: a run of one row in block N / 16.  The workgroup of
// a sequence that finishes last (a counter per sequence, 0 between launches)
// sets its length, which the others have read by then.
template <int D>
__global__ __launch_bounds__(kStoreThreads) void append_q8_kernel(StoreArgs a, const int* tables,
                                                                  int* ctx_lens, int MAXB,
                                                                  unsigned* tickets) {
  __shared__ Store8<D> sh;
  const int b = blockIdx.x;
  const int N = ctx_lens[b];
  int p = -1;
  if (N < 0 || N >= MAXB * kBlock) {
    if (threadIdx.x == 0) raise_flag(a.flags, N < 0 ? ENT_DEV_BAD_CTXLEN : ENT_DEV_CACHE_FULL);
  } else {
    p = tables[static_cast<long long>(b) * MAXB + N / kBlock];
    if (p < 0 || p >= a.P) {
      if (threadIdx.x == 0) raise_flag(a.flags, ENT_DEV_BAD_TABLE);
      p = -1;
    }
  }
  if (p < 0) return;                  // every workgroup of the sequence, so no ticket is drawn
  store8_run<D>(a, sh, blockIdx.y * Store8<D>::HW, static_cast<const uint16_t*>(a.k) + b * a.ldk,
                static_cast<const uint16_t*>(a.v) + b * a.ldv, p, N % kBlock, 1);
  if (threadIdx.x == 0 && atomicInc(tickets + b, gridDim.y - 1) == gridDim.y - 1) ctx_lens[b] = N + 1;
}

StoreArgs store_args(const ent_ctx* c, const void* k, long long ldk, const void* v, long long ldv,
                     void* k_cache, void* v_cache, float* ksum) {
  StoreArgs a{};
  a.k = k;
  a.ldk = ldk;
  a.v = v;
  a.ldv = ldv;
  a.kc = k_cache;
  a.vc = v_cache;
  a.ksum = ksum;
  a.Hkv = c->cfg.num_kv_heads;
  a.P = c->cfg.num_pool_blocks;
  a.flags = c->dev_flags;
  return a;
}

template <int HW>
dim3 store_grid(const ent_ctx* c, int n) {
  return dim3(n, (c->cfg.num_kv_heads + HW - 1) / HW);
}

}  // namespace

hipError_t launch_prompt_plan(const ent_ctx* c, int B, const int* n_new, const int* ctx_lens,
                              int* tables, const int* free_ids, int n_ids, int* free_range,
                              int max_tokens, int* starts, long long* slots, int* new_lens,
                              hipStream_t s) {
  const PlanArgs a{n_new, ctx_lens, tables, free_ids, n_ids, free_range, B,
                   c->cfg.max_blocks_per_seq, c->cfg.num_pool_blocks, max_tokens, starts, slots,
                   new_lens, c->tickets, c->dev_flags};
  const int grid = std::max(1, (max_tokens + kPlanTokens - 1) / kPlanTokens);
  const size_t lds = static_cast<size_t>(3 * B + 2) * sizeof(int);
  hipLaunchKernelGGL(plan_kernel, dim3(grid), dim3(kPlanThreads), lds, s, a);
  return hipGetLastError();
}

hipError_t launch_prompt_store(const ent_ctx* c, int T, const void* k, long long ldk, const void* v,
                               long long ldv, const long long* slots, void* k_cache, void* v_cache,
                               float* ksum, hipStream_t s) {
  StoreArgs a = store_args(c, k, ldk, v, ldv, k_cache, v_cache, ksum);
  a.slots = slots;
  a.T = T;
  const int n = (T + kBlock - 1) / kBlock;
  const bool bf16 = c->cfg.kv_dtype == ENT_BF16;
  if (c->cfg.head_dim == 128) {
    if (bf16) hipLaunchKernelGGL((store_kernel<uint16_t, 128>), store_grid<1>(c, n), dim3(kStoreThreads), 0, s, a);
    else hipLaunchKernelGGL((store_kernel<float, 128>), store_grid<1>(c, n), dim3(kStoreThreads), 0, s, a);
  } else {
    if (bf16) hipLaunchKernelGGL((store_kernel<uint16_t, 64>), store_grid<2>(c, n), dim3(kStoreThreads), 0, s, a);
    else hipLaunchKernelGGL((store_kernel<float, 64>), store_grid<1>(c, n), dim3(kStoreThreads), 0, s, a);
  }
  return hipGetLastError();
}

hipError_t launch_prompt_store_q8(const ent_ctx* c, int T, const void* k, long long ldk,
                                  const void* v, long long ldv, const long long* slots,
                                  void* k_cache, void* v_cache, float* k_scale, float* v_scale,
                                  float* ksum, hipStream_t s) {
  StoreArgs a = store_args(c, k, ldk, v, ldv, k_cache, v_cache, ksum);
  a.slots = slots;
  a.T = T;
  a.ks = k_scale;
  a.vs = v_scale;
  const int n = (T + kBlock - 1) / kBlock;
  if (c->cfg.head_dim == 128)
    hipLaunchKernelGGL(store_q8_kernel<128>, store_grid<Store8<128>::HW>(c, n), dim3(kStoreThreads), 0, s, a);
  else
    hipLaunchKernelGGL(store_q8_kernel<64>, store_grid<Store8<64>::HW>(c, n), dim3(kStoreThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_kv_append_q8(const ent_ctx* c, int B, const void* k_new, const void* v_new,
                               const int* tables, int* ctx_lens, void* k_cache, void* v_cache,
                               float* k_scale, float* v_scale, float* ksum, hipStream_t s) {
  const long long ld = static_cast<long long>(c->cfg.num_kv_heads) * c->cfg.head_dim;
  StoreArgs a = store_args(c, k_new, ld, v_new, ld, k_cache, v_cache, ksum);
  a.ks = k_scale;
  a.vs = v_scale;
  const int MAXB = c->cfg.max_blocks_per_seq;
  if (c->cfg.head_dim == 128)
    hipLaunchKernelGGL(append_q8_kernel<128>, store_grid<Store8<128>::HW>(c, B), dim3(kStoreThreads), 0,
                       s, a, tables, ctx_lens, MAXB, c->tickets);
  else
    hipLaunchKernelGGL(append_q8_kernel<64>, store_grid<Store8<64>::HW>(c, B), dim3(kStoreThreads), 0,
                       s, a, tables, ctx_lens, MAXB, c->tickets);
  return hipGetLastError();
}

}  // namespace ent
