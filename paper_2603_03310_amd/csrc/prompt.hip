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
// and lengths, and the one that is the last to have read the free list's range
// moves its head.  Who is last is counted in two steps, each counter in a cache
// line of its own, and the count is taken before the slots and looked at after
// them: counting costs about 10 ns a workgroup and line (1.34M tokens of 256
// requests: 14.4 us with 656 workgroups and one counter, 21.1 with 1312, 21.5
// with their sixteen counters side by side, 9.0 with a line each, 8.4 so).
//
// Otherwise a chain of loads, sums and searches bounds it, mostly a launch's own
// few us: 64 requests that get a token each 4.3 us (5.6 with the counters for a
// single workgroup too and the free ids loaded where they are written).
//
// Requests are admitted in order while tokens and blocks last; the inclusive
// sums only grow, so "both fit" holds for a prefix of the batch and needs no
// second pass.
// ---------------------------------------------------------------------------
constexpr int kPlanThreads = 256;
constexpr int kPlanCounters = 16;      // counters of finished workgroups, and one over them
constexpr int kCounterPitch = 32;      // a cache line each
static_assert((kPlanCounters + 1) * kCounterPitch <= kMinTickets, "counters");

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
  unsigned* tickets;      // kPlanCounters + 1 of them, 0 between launches
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

// The largest b in [from, to) with s[b] <= x (s ascending, s[from] <= x).
__device__ __forceinline__ int plan_find(const int* s, int to, int x, int from) {
  int lo = from, hi = to;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// The same for one x of a whole wave: 64 places a step.
__device__ __forceinline__ int plan_find_uniform(const int* s, int to, int x) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = to;
  while (n > 1) {
    const int w = (n + 63) / 64;
    const int k = __popcll(__ballot(lane * w < n && s[lo + min(lane * w, n - 1)] <= x)) - 1;
    lo += k * w;
    n = min(w, n - k * w);
  }
  return lo;
}

// kPairs: pairs of slots of a thread.
template <int kPairs>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs a) {
  constexpr int kPlanTokens = 2 * kPairs * kPlanThreads;     // slots of a workgroup
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
  const int avail = ring_ok ? end - head : -1;         // -1: nobody is served, also who needs no block
  if (!ring_ok) head = 0;
  unsigned bad = ring_ok ? 0u : ENT_DEV_BAD_TABLE;
  // The block of this thread's first new table entry, on its way during the sums.
  const int e0 = blockIdx.x * kPlanThreads + t;
  const int id0 = e0 < avail ? a.ids[head + e0] : -1;
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
      s_tok[b] = n;
      s_ctx[b] = ctx;
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
      const int n = s_tok[b], ctx = s_ctx[b];          // its own of the loop before
      const int need = (ctx + n + kBlock - 1) / kBlock - (ctx + kBlock - 1) / kBlock;
      s_tok[b] = tok;
      s_blk[b] = blk;
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
  // Every workgroup finds the same here; the first raises it (an atomic of each, where
  // the free list ran out: 65.9 us instead of 6.8 with 656 workgroups).
  if (blockIdx.x != 0) bad = 0;
  for (int b = t; b < a.B; b += kPlanThreads) {
    s_tok[b] = min(s_tok[b], total);
    s_blk[b] = min(s_blk[b], taken);
  }
  if (t == 0) {
    s_tok[a.B] = total;
    s_blk[a.B] = taken;
  }
  __syncthreads();

  // This workgroup has read the free list's range (its threads' `avail`, before the
  // first barrier).  A counter of one workgroup is not needed.
  const unsigned n_wg = gridDim.x, c = blockIdx.x % kPlanCounters;
  const unsigned mine = (n_wg - c + kPlanCounters - 1) / kPlanCounters;       // workgroups of this counter
  const unsigned used = n_wg < kPlanCounters ? n_wg : kPlanCounters;
  bool last = t == 0 && ring_ok;
  unsigned ticket = mine - 1;
  if (last && mine > 1) ticket = atomicInc(a.tickets + c * kCounterPitch, mine - 1);

  const bool pairs = (reinterpret_cast<uintptr_t>(a.slots) & 15) == 0;
  // Slots of this workgroup's tokens, two consecutive ones a thread and step.  The
  // requests that the tokens lie in are found within those of its first and last,
  // mostly one or two; the block ids of all steps are then on their way together.
  const int t0 = blockIdx.x * kPlanTokens;
  const int t1 = min(total, t0 + kPlanTokens);           // tokens from here on are padding
  const bool one = gridDim.x == 1;                       // all of them
  const int r0 = t0 < t1 && !one ? plan_find_uniform(s_tok, a.B, t0) : 0;
  const int r1 = t0 < t1 && !one ? plan_find_uniform(s_tok, a.B, t1 - 1) + 1 : a.B;
  int page[2 * kPairs], row[2 * kPairs];
#pragma unroll
  for (int i = 0; i < 2 * kPairs; ++i) {
    const int x = t0 + 2 * (t + i / 2 * kPlanThreads) + i % 2;
    page[i] = row[i] = -1;
    if (x < t1) {
      const int b = plan_find(s_tok, r1, x, r0);
      const int pos = s_ctx[b] + x - s_tok[b];
      const int j = pos / kBlock, have = (s_ctx[b] + kBlock - 1) / kBlock;
      row[i] = pos % kBlock;
      page[i] = j < have ? a.tables[static_cast<long long>(b) * a.MAXB + j]
                         : a.ids[head + s_blk[b] + j - have];
    }
  }
#pragma unroll
  for (int i = 0; i < 2 * kPairs; i += 2) {
    const int x = t0 + 2 * (t + i / 2 * kPlanThreads);
    long long sl[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const bool ok = page[i + e] >= 0 && page[i + e] < a.P;
      if (row[i + e] >= 0 && !ok) bad |= ENT_DEV_BAD_TABLE;
      sl[e] = ok ? static_cast<long long>(page[i + e]) * kBlock + row[i + e] : -1;
    }
    if (x + 1 < a.max_tokens && pairs) {
      *reinterpret_cast<longlong2*>(a.slots + x) = make_longlong2(sl[0], sl[1]);
    } else {
      if (x < a.max_tokens) a.slots[x] = sl[0];
      if (x + 1 < a.max_tokens) a.slots[x + 1] = sl[1];
    }
  }
  // New table entries, dealt to all workgroups.
  for (int e = e0; e < taken; e += gridDim.x * kPlanThreads) {
    const int b = plan_find(s_blk, a.B, e, 0);
    const int j = (s_ctx[b] + kBlock - 1) / kBlock + e - s_blk[b];
    const int p = e == e0 ? id0 : a.ids[head + e];
    const bool ok = p >= 0 && p < a.P;
    if (!ok) bad |= ENT_DEV_BAD_TABLE;
    a.tables[static_cast<long long>(b) * a.MAXB + j] = ok ? p : -1;
  }
  if (blockIdx.x == 0) {
    for (int b = t; b <= a.B; b += kPlanThreads) {
      a.starts[b] = s_tok[b];
      if (a.new_lens && b < a.B) a.new_lens[b] = a.ctx[b] + s_tok[b + 1] - s_tok[b];
    }
  }
  if (bad) raise_flag(a.flags, bad);
  last = last && ticket == mine - 1;
  if (last && used > 1)
    last = atomicInc(a.tickets + kPlanCounters * kCounterPitch, used - 1) == used - 1;
  if (last) a.range[0] = head + taken;
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
//
// 16 elements a thread are few bytes for the work on them, so it is vector
// instructions that bound it, before memory: magnitudes are compared as bf16 bits,
// two at once, K's and V's maxima in one register; only a thread that holds
// something not finite clamps; V is transposed by bytes of words.  51624 tokens of
// 8 heads of 128: 94 us with float magnitudes, clamps throughout and single bytes,
// 75 us so (331 MB, 87% of a large copy's rate).  Four tiles in turn a
// workgroup with all loads issued at once: 113 against the 94.
template <int D>
struct Store8 {
  static constexpr int I = kBlock * D / 8;                            // threads of a tile
  static constexpr int HW = kStoreThreads / I;                        // tiles of a workgroup
  static constexpr int WT = I / 64;                                   // waves of a tile
  static constexpr int PITCH = D + 16;
  __attribute__((aligned(16))) unsigned char k[HW * kBlock * PITCH];
  __attribute__((aligned(16))) unsigned char v[HW * kBlock * PITCH];
  unsigned top[kStoreThreads / 64];
};

typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2_t pair16(unsigned x) { return __builtin_bit_cast(u16x2_t, x); }
__device__ __forceinline__ unsigned pair32(u16x2_t x) { return __builtin_bit_cast(unsigned, x); }
struct OpMaxPair {
  __device__ __forceinline__ unsigned operator()(unsigned x, unsigned y) const {
    return pair32(__builtin_elementwise_max(pair16(x), pair16(y)));
  }
};
// Largest magnitude bits of eight bf16 values (0x7f80 and more: not finite).
__device__ __forceinline__ unsigned top16(uint4 w) {
  const unsigned m = 0x7fff7fffu;
  OpMaxPair mx;
  const u16x2_t x = pair16(mx(mx(w.x & m, w.y & m), mx(w.z & m, w.w & m)));
  return max(static_cast<unsigned>(x.x), static_cast<unsigned>(x.y));
}
__device__ __forceinline__ void widen8(uint4 w, float (&x)[8]) {
  const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(u[i] << 16);
    x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}
// ... of those that are finite.
__device__ __forceinline__ unsigned top16_finite(uint4 w) {
  float x[8], t = 0.f;
  widen8(w, x);
#pragma unroll
  for (int i = 0; i < 8; ++i) t = fmaxf(t, q8_mag(x[i]));
  return __float_as_uint(t) >> 16;
}
// Eight codes of x / s (inv = 1 / s: exact but for a kept scale of the caller's own
// making that is no power of two).  Finite values stay under 464, which rounds to
// 448, as the scale covers them.
__device__ __forceinline__ uint2 codes8(uint4 w, float inv, bool clamp) {
  float y[8];
  widen8(w, y);
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] *= inv;
  if (clamp) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = q8_clamp(y[i]);
  }
  return make_uint2(q8_pack4(y[0], y[1], y[2], y[3]), q8_pack4(y[4], y[5], y[6], y[7]));
}
// Eight codes times f <= 1, rounded again.
__device__ __forceinline__ uint2 recode8(uint2 w, float f) {
  float y[8];
  q8_unpack4(w.x, y);
  q8_unpack4(w.y, y + 4);
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] *= f;
  return make_uint2(q8_pack4(y[0], y[1], y[2], y[3]), q8_pack4(y[4], y[5], y[6], y[7]));
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
  uint4 kx = make_uint4(0u, 0u, 0u, 0u), vx = kx;
  uint2 kold = make_uint2(0u, 0u);
  float ks0 = 0.f, vs0 = 0.f;
  if (fresh) {
    kx = *reinterpret_cast<const uint4*>(k + (row - row0) * a.ldk + g * D + c);
    vx = *reinterpret_cast<const uint4*>(v + (row - row0) * a.ldv + g * D + c);
  }
  if (head && row0 > 0) {
    ks0 = a.ks[tg];
    vs0 = a.vs[tg];
    if (old) kold = *reinterpret_cast<const uint2*>(kc + row * D + c);
  }
  unsigned kt = top16(kx), vt = top16(vx);
  const bool kbad = kt >= 0x7f80u, vbad = vt >= 0x7f80u;
  if (kbad) kt = top16_finite(kx);
  if (vbad) vt = top16_finite(vx);
  const unsigned both = wave_reduce(kt << 16 | vt, OpMaxPair());
  __syncthreads();                    // the last run's LDS is read no more
  if ((t & 63) == 0) sh.top[t >> 6] = both;
  __syncthreads();
  unsigned top = 0;
#pragma unroll
  for (int w = 0; w < S::WT; ++w) top = OpMaxPair()(top, sh.top[hh * S::WT + w]);
  const float kn = q8_scale(__uint_as_float(top & 0xffff0000u)), vn = q8_scale(__uint_as_float(top << 16));
  const float ks = row0 > 0 && ks0 > kn ? ks0 : kn, vs = row0 > 0 && vs0 > vn ? vs0 : vn;
  const bool kgrow = row0 > 0 && ks > ks0, vgrow = row0 > 0 && vs > vs0;
  unsigned char* const lk = sh.k + (hh * kBlock + row) * S::PITCH + c;
  if (fresh) {
    const uint2 kw = codes8(kx, __fdiv_rn(1.f, ks), kbad);
    *reinterpret_cast<uint2*>(kc + row * D + c) = kw;
    *reinterpret_cast<uint2*>(lk) = kw;
    *reinterpret_cast<uint2*>(sh.v + (hh * kBlock + row) * S::PITCH + c) =
        codes8(vx, __fdiv_rn(1.f, vs), vbad);
  } else if (old) {
    if (kgrow) {
      kold = recode8(kold, ks0 / ks);
      *reinterpret_cast<uint2*>(kc + row * D + c) = kold;
    }
    *reinterpret_cast<uint2*>(lk) = kold;
  }
  if (head && r == 0) {
    a.ks[tg] = ks;
    a.vs[tg] = vs;
  }
  __syncthreads();
  if (rows == kBlock) {
    // A whole block's V: a thread turns 8 rows of 4 dims.
    for (int e = r; e < D / 2; e += S::I) {
      const int d = e / 2 * 4, s0 = e % 2 * 8;
      unsigned w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        w[i] = *reinterpret_cast<const unsigned*>(sh.v + (hh * kBlock + s0 + i) * S::PITCH + d);
      uint2 o[4];
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        // Bytes 0 and 1, then 2 and 3, of pairs of rows; then dims.
        const unsigned a0 = __builtin_amdgcn_perm(w[4 * z + 1], w[4 * z], 0x05010400u);
        const unsigned a1 = __builtin_amdgcn_perm(w[4 * z + 1], w[4 * z], 0x07030602u);
        const unsigned b0 = __builtin_amdgcn_perm(w[4 * z + 3], w[4 * z + 2], 0x05010400u);
        const unsigned b1 = __builtin_amdgcn_perm(w[4 * z + 3], w[4 * z + 2], 0x07030602u);
        const unsigned q[4] = {__builtin_amdgcn_perm(b0, a0, 0x05040100u), __builtin_amdgcn_perm(b0, a0, 0x07060302u),
                               __builtin_amdgcn_perm(b1, a1, 0x05040100u), __builtin_amdgcn_perm(b1, a1, 0x07060302u)};
#pragma unroll
        for (int y = 0; y < 4; ++y) (z ? o[y].y : o[y].x) = q[y];
      }
      if (head) {
#pragma unroll
        for (int y = 0; y < 4; ++y) *reinterpret_cast<uint2*>(vc + (d + y) * kBlock + s0) = o[y];
      }
    }
  } else if (head) {
    // Part of one: a thread has 8 rows of one dim; the others stay as they are,
    // but for earlier ones that a larger scale rounds again.
    const int d = r / 2, s0 = r % 2 * 8;
    if (s0 < row1) {
      unsigned char* const at = vc + d * kBlock + s0;
      uint2 vold = make_uint2(0u, 0u);
      if (vgrow && s0 < row0) vold = recode8(*reinterpret_cast<const uint2*>(at), vs0 / vs);
      unsigned char x[8];
      __builtin_memcpy(x, &vold, 8);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (s0 + i >= row0 && s0 + i < row1) x[i] = sh.v[(hh * kBlock + s0 + i) * S::PITCH + d];
      const int first = vgrow ? 0 : row0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (s0 + i >= first && s0 + i < row1) at[i] = x[i];
    }
  }
  if (a.ksum && head) {
    // Four dims a thread, from the tile's last threads on (the first turn V).
    for (int e = S::I - 1 - r; e < D / 4; e += S::I) {
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < kBlock; ++s) {
        float x[4];
        q8_unpack4(*reinterpret_cast<const unsigned*>(sh.k + (hh * kBlock + s) * S::PITCH + 4 * e), x);
        if (s < row1) {
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i] += x[i];
        }
      }
      const float n = static_cast<float>(row1);
      *reinterpret_cast<float4*>(a.ksum + tg * D + 4 * e) =
          make_float4(__fdiv_rn(sum[0], n) * ks, __fdiv_rn(sum[1], n) * ks, __fdiv_rn(sum[2], n) * ks,
                      __fdiv_rn(sum[3], n) * ks);
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
  const size_t lds = static_cast<size_t>(3 * B + 2) * sizeof(int);
  // Two slots a thread while that makes four workgroups a CU at most, else four, since
  // every workgroup forms the sums again.  us with two and with four: one request of 2500
  // tokens 3.5, 3.9; 64 of 64 4.4, 5.4; 1000 of 300 7.4, 7.6; 256 of 5200 10.1, 8.1.
  if (max_tokens <= 4 * c->num_cu * 2 * kPlanThreads) {
    const int grid = std::max(1, (max_tokens + 2 * kPlanThreads - 1) / (2 * kPlanThreads));
    hipLaunchKernelGGL(plan_kernel<1>, dim3(grid), dim3(kPlanThreads), lds, s, a);
  } else {
    const int grid = (max_tokens + 4 * kPlanThreads - 1) / (4 * kPlanThreads);
    hipLaunchKernelGGL(plan_kernel<2>, dim3(grid), dim3(kPlanThreads), lds, s, a);
  }
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
    hipLaunchKernelGGL(store_q8_kernel<128>, (store_grid<Store8<128>::HW>(c, n)), dim3(kStoreThreads), 0, s, a);
  else
    hipLaunchKernelGGL(store_q8_kernel<64>, (store_grid<Store8<64>::HW>(c, n)), dim3(kStoreThreads), 0, s, a);
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
    hipLaunchKernelGGL(append_q8_kernel<128>, (store_grid<Store8<128>::HW>(c, B)), dim3(kStoreThreads), 0,
                       s, a, tables, ctx_lens, MAXB, c->tickets);
  else
    hipLaunchKernelGGL(append_q8_kernel<64>, (store_grid<Store8<64>::HW>(c, B)), dim3(kStoreThreads), 0,
                       s, a, tables, ctx_lens, MAXB, c->tickets);
  return hipGetLastError();
}

}  // namespace ent
