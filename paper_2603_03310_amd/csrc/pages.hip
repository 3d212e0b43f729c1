// Blocks of the paged cache shared by several sequences (fork), handed back to the
// free list (release), and moved to the pool's lower end (compact).
//
// shared[p] counts the holders of block p besides the first.  A fork adds one to
// every full block of its parent and copies the last, begun one, if any; a release
// takes one from every block of its sequences, and those that had none left over are
// free.  Sets of blocks are bitmaps of the pool, so what comes out of them is in
// ascending order whatever order the atomics came in.  Their words lie 64 bytes apart:
// atomics on one cache line come one after the other, and side by side a line would
// hold 1024 blocks.

#include "ent_internal.h"

#include <algorithm>

namespace ent {
namespace {

constexpr int kPageThreads = 256;
constexpr int kPlanThreads = 1024;
// Bits of a word, on average, from which on a wave writes them together.  Always so: 9.2
// us instead of 6.6 where 321 words have 509; from 32 on: 160 us instead of 158 for the
// lists of 5120 moves over 320 words.
constexpr int kDense = 8;
constexpr int kBitPitch = kPageBitBytes / 8;     // 64-bit words from one word of a bitmap to the next

// Where a block's contents lie: caches of tile_bytes a block, mean keys, scales.
struct PageStore {
  char* k;
  char* v;
  float* ks;            // scales (8-bit caches), else null
  float* vs;
  float* ksum;          // nullable
  long long tile_bytes; // of one block, all heads: a multiple of 16
  int sum_floats;       // H_kv d, a multiple of 4
  int Hkv;
};

__device__ __forceinline__ const uint4* at16(const void* p, long long byte) {
  return reinterpret_cast<const uint4*>(static_cast<const char*>(p) + byte);
}
__device__ __forceinline__ uint4* at16(void* p, long long byte) {
  return reinterpret_cast<uint4*>(static_cast<char*>(p) + byte);
}

// The copy of `units` 16-byte pieces by threads t of nt: U of a thread in flight while each
// has as many left (with 8 and 256 threads, blocks of 32 KB and their multiples), then one
// after the other, each a round trip.
template <int U, bool STREAM>
__device__ __forceinline__ void copy_units(const uint4* __restrict__ s, uint4* __restrict__ d, int units, int t,
                                           int nt) {
  int i = t;
  for (; i + (U - 1) * nt < units; i += U * nt) {
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = load16<STREAM>(s + i + u * nt);
#pragma unroll
    for (int u = 0; u < U; ++u) store16<STREAM>(d + i + u * nt, x[u]);
  }
  for (; i < units; i += nt) store16<STREAM>(d + i, load16<STREAM>(s + i));
}

// Block `from`'s contents to block `to` by threads t of nt: two pieces of keys and two of
// values in flight a thread.
__device__ __forceinline__ void copy_block(const PageStore& st, int from, int to, int t, int nt) {
  const uint4* sk = at16(static_cast<const void*>(st.k), from * st.tile_bytes);
  const uint4* sv = at16(static_cast<const void*>(st.v), from * st.tile_bytes);
  uint4 *dk = at16(st.k, to * st.tile_bytes), *dv = at16(st.v, to * st.tile_bytes);
  const int units = static_cast<int>(st.tile_bytes / 16);
  int i = t;
  for (; i + nt < units; i += 2 * nt) {
    const uint4 x = sk[i], y = sv[i], x1 = sk[i + nt], y1 = sv[i + nt];
    dk[i] = x;
    dv[i] = y;
    dk[i + nt] = x1;
    dv[i + nt] = y1;
  }
  for (; i < units; i += nt) {
    const uint4 x = sk[i], y = sv[i];
    dk[i] = x;
    dv[i] = y;
  }
  if (st.ksum)
    copy_units<1, false>(at16(static_cast<const void*>(st.ksum), 4ll * from * st.sum_floats),
                         at16(st.ksum, 4ll * to * st.sum_floats), st.sum_floats / 4, t, nt);
  if (st.ks) {
    for (int i = t; i < st.Hkv; i += nt) {
      st.ks[static_cast<long long>(to) * st.Hkv + i] = st.ks[static_cast<long long>(from) * st.Hkv + i];
      st.vs[static_cast<long long>(to) * st.Hkv + i] = st.vs[static_cast<long long>(from) * st.Hkv + i];
    }
  }
}

// Counting a launch's workgroups: the one whose count is the last does what has to wait
// for all.  In two steps, each counter in a cache line of its own (a count on one line
// takes about 10 ns); counters are 0 between launches.  One thread of each workgroup.
constexpr int kCounters = 16;
constexpr int kCounterPitch = 32;
static_assert((kCounters + 1) * kCounterPitch <= kMinTickets, "counters");
__device__ __forceinline__ bool count_out(unsigned* tickets) {
  const unsigned n_wg = gridDim.x, c = blockIdx.x % kCounters;
  const unsigned mine = (n_wg - c + kCounters - 1) / kCounters;      // workgroups of this counter
  const unsigned used = n_wg < kCounters ? n_wg : kCounters;
  if (mine > 1 && atomicInc(tickets + c * kCounterPitch, mine - 1) != mine - 1) return false;
  return used == 1 || atomicInc(tickets + kCounters * kCounterPitch, used - 1) == used - 1;
}

// Sum of v over the threads before this one, and of all; the whole workgroup calls it.
template <int NT>
__device__ __forceinline__ int scan_before(int v, int& all, int* red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int incl = static_cast<int>(wave_scan_u(static_cast<unsigned>(v)));
  if (lane == 63) red[wave] = incl;
  __syncthreads();
  int out = incl - v;
  all = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    if (w < wave) out += red[w];
    all += red[w];
  }
  __syncthreads();
  return out;
}

// Bitmaps of blocks: a 64-bit word per 64 of them.
typedef unsigned long long u64;
__device__ __forceinline__ int popc(u64 b) { return static_cast<int>(__popcll(b)); }
__device__ __forceinline__ bool set_bit(u64* bits, int p) {
  const u64 bit = 1ull << (p % 64);
  return (atomicOr(&bits[static_cast<long long>(p / 64) * kBitPitch], bit) & bit) != 0;
}
__device__ __forceinline__ u64 look_word(const u64* bits, int w, int words) {
  return w < words ? __hip_atomic_load(bits + static_cast<long long>(w) * kBitPitch, __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT)
                   : 0ull;
}
// ... and cleared for the next call.
__device__ __forceinline__ u64 take_word(u64* bits, int w, int words) {
  const u64 b = look_word(bits, w, words);
  if (b) bits[static_cast<long long>(w) * kBitPitch] = 0ull;
  return b;
}
// The bits of b below this lane's, and this lane's (b the same in every lane).
__device__ __forceinline__ int bits_below(u64 b) {
  return static_cast<int>(__builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(b >> 32),
                                                    __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(b), 0u)));
}
__device__ __forceinline__ bool bit_here(u64 b) { return __builtin_amdgcn_inverse_ballot_w64(b); }
// A workgroup's words (word t of thread t, `n` of them), each with a value: f(word, value,
// t) by all lanes of a wave, lane l for bit l, with consecutive words dealt to the waves and
// eight of them together (one after the other, a word is a chain of some 25 instructions:
// 120 ns).  s_b, s_v: a place per thread.
template <int NT, typename F>
__device__ __forceinline__ void each_word(u64 b, int v, int n, u64* s_b, int* s_v, F f) {
  constexpr int W = NT / 64, Q = 8;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  s_b[t] = b;
  s_v[t] = v;
  __syncthreads();
  const u64 mb = s_b[lane * W + wave];
  const int mv = s_v[lane * W + wave];
  for (int i = 0; i < 64 && i * W + wave < n; i += Q) {
    u64 w[Q], any = 0ull;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      w[q] = static_cast<u64>(static_cast<unsigned>(lane_at(static_cast<int>(mb >> 32), i + q))) << 32 |
             static_cast<unsigned>(lane_at(static_cast<int>(mb), i + q));
      any |= w[q];
    }
    if (any == 0ull) continue;
#pragma unroll
    for (int q = 0; q < Q; ++q) f(w[q], lane_at(mv, i + q), (i + q) * W + wave);
  }
  __syncthreads();
}

// Writes the ids of a workgroup's words (word t of thread t, of ids from id0 on; at most n
// words with bits), the first of a thread's at `at` and so on; those before place 0 are
// left out.  Where a word has few bits, each thread writes its own.  zero (nullable):
// becomes 0 at each of the ids.
template <int NT>
__device__ __forceinline__ void list_bits(u64 b, int at, int id0, int n, bool dense, int* out, u64* s_b, int* s_v,
                                          int* zero) {
  if (dense) {
    each_word<NT>(b, at, n, s_b, s_v, [&](u64 w, int first, int i) {
      const int place = first + bits_below(w), id = id0 + i * 64 + static_cast<int>(threadIdx.x & 63);
      if (bit_here(w)) {
        if (place >= 0) out[place] = id;
        if (zero) zero[id] = 0;
      }
    });
  } else {
    for (; b; b &= b - 1, ++at) {
      const int id = id0 + static_cast<int>(threadIdx.x) * 64 + __builtin_ctzll(b);
      if (at >= 0) out[at] = id;
      if (zero) zero[id] = 0;
    }
  }
}

struct Tables {
  int* tables;
  int* ctx;
  int R, MAXB, P;
  unsigned* flags;
};

// ---------------------------------------------------------------------------
// Fork.  Who is served, and with which new blocks, follows from all forks' rows and
// lengths: up to kForkOne forks every workgroup finds it for itself (a fork a thread),
// and the last to have done so moves the free list; more of them have one workgroup
// find it in a launch of its own (24 / 96 / 255 forks: 6.2 / 5.8 / 8.2 us in one launch,
// 8.6 / 8.4 / 11.3 in two).  A fork's workgroups are of two sorts, those that fill its row
// and count holders, and those that copy the begun block.  Bound by its chain of round
// trips (rows, lengths, the list, then the entry and the block): 96 forks of 4096 to 16001
// tokens (60240 counts, 96 blocks) 7.7 us.
// ---------------------------------------------------------------------------
constexpr int kForkOne = kPageThreads;

struct ForkArgs {
  Tables tb;
  int N;
  const int* src;
  const int* dst;
  int* shared;
  const int* ids;
  int n_ids;
  int* range;
  int4* rec;            // [N] (source row or -1, destination row, tokens, new block or -1)
  unsigned* tickets;
  int row_parts, parts; // workgroups of a fork that fill its row, and all of them
  PageStore st;
};

// What every fork does: emit(i, record).  Returns the free list's new lower end (its
// old one where the range is bad).  mem: R + (R + 31) / 32 ints.  ONE: N <= NT.
template <int NT, bool ONE, typename F>
__device__ __forceinline__ int fork_plan(const ForkArgs& a, int* mem, unsigned& bad, F emit) {
  __shared__ int s_red[NT / 64];
  __shared__ int s_cut;
  int* s_first = mem;                                            // [R] first fork to a row
  unsigned* s_from = reinterpret_cast<unsigned*>(mem + a.tb.R);  // bits of rows that are forked
  const int t = threadIdx.x;
  const int head = a.range[0], end = a.range[1];
  const bool ring_ok = head >= 0 && head <= end && end <= a.n_ids;
  const int avail = ring_ok ? end - head : 0;
  for (int i = t; i < a.tb.R; i += NT) s_first[i] = 0x7fffffff;
  for (int i = t; i < (a.tb.R + 31) / 32; i += NT) s_from[i] = 0u;
  if (t == 0) s_cut = ring_ok ? 0x7fffffff : 0;
  __syncthreads();
  auto row_ok = [&](int r) { return r >= 0 && r < a.tb.R; };
  const int per = ONE ? 1 : (a.N + NT - 1) / NT;       // consecutive forks of a thread
  for (int k = 0; k < per; ++k) {
    const int i = t * per + k;
    if (i < a.N) {
      const int s = a.src[i], d = a.dst[i];
      if (row_ok(d)) atomicMin(&s_first[d], i);
      if (row_ok(s)) atomicOr(&s_from[s / 32], 1u << (s % 32));
    }
  }
  __syncthreads();
  // Fork i's tokens, or -1 where it is passed over.
  bad |= ring_ok ? 0u : ENT_DEV_BAD_TABLE;
  auto tokens = [&](int i, int& s, int& d) {
    s = a.src[i];
    d = a.dst[i];
    const int n = row_ok(s) ? a.tb.ctx[s] : 0;
    if (!row_ok(s) || !row_ok(d) || s_first[d] != i || (s_from[d / 32] >> (d % 32) & 1u)) {
      bad |= ENT_DEV_BAD_ROW;
      return -1;
    }
    if (n < 0 || n > a.tb.MAXB * kBlock) {
      bad |= ENT_DEV_BAD_CTXLEN;
      return -1;
    }
    return n;
  };
  int need = 0, s = 0, d = 0, n = -1;        // of the thread's last fork, its only one if per is 1
  for (int k = 0; k < per; ++k) {
    const int i = t * per + k;
    if (i < a.N) {
      n = tokens(i, s, d);
      need += n > 0 && n % kBlock != 0;
    }
  }
  int all;
  const int before = scan_before<NT>(need, all, s_red);
  need = before;
  for (int k = 0; k < per; ++k) {
    const int i = t * per + k;
    if (i < a.N) {
      if (per > 1) n = tokens(i, s, d);
      if (n > 0 && n % kBlock != 0 && ++need > avail) {
        atomicMin(&s_cut, i);
        break;
      }
    }
  }
  __syncthreads();
  const int cut = s_cut;
  if (ring_ok && cut < a.N) bad |= ENT_DEV_CACHE_FULL;
  need = before;
  for (int k = 0; k < per; ++k) {
    const int i = t * per + k;
    if (i < a.N) {
      if (per > 1) n = tokens(i, s, d);
      const bool go = n >= 0 && i < cut, block = go && n % kBlock != 0;
      emit(i, make_int4(go ? s : -1, d, n, block ? head + need : -1));
      need += block;
    }
  }
  return ring_ok ? head + min(all, avail) : head;
}

__global__ __launch_bounds__(kPlanThreads) void fork_plan_kernel(ForkArgs a) {
  extern __shared__ int s_mem[];
  unsigned bad = 0;
  const int head = fork_plan<kPlanThreads, false>(a, s_mem, bad, [&](int i, int4 r) { a.rec[i] = r; });
  if (threadIdx.x == 0) a.range[0] = head;
  if (bad) raise_flag(a.tb.flags, bad);
}

// ONE: every workgroup plans for itself; else the records are there.
template <bool ONE>
__global__ __launch_bounds__(kPageThreads) void fork_kernel(ForkArgs a) {
  extern __shared__ int s_mem[];
  const int fork = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  int4 r;
  int head = 0;
  bool last = false;
  unsigned bad = 0;
  if constexpr (ONE) {
    __shared__ int4 s_rec;
    head = fork_plan<kPageThreads, true>(a, s_mem, bad, [&](int i, int4 x) { if (i == fork) s_rec = x; });
    // Every workgroup finds the same; the first raises it.
    if (blockIdx.x != 0) bad = 0;
    __syncthreads();                        // the free list's range has been read
    r = s_rec;
    if (threadIdx.x == 0) last = count_out(a.tickets);
  } else {
    r = a.rec[fork];
  }
  if (r.x >= 0) {
    const int* from = a.tb.tables + static_cast<long long>(r.x) * a.tb.MAXB;
    int* to = a.tb.tables + static_cast<long long>(r.y) * a.tb.MAXB;
    const int full = r.z / kBlock;
    if (part < a.row_parts) {
      for (int j = part * kPageThreads + threadIdx.x; j < full; j += a.row_parts * kPageThreads) {
        const int p = from[j];
        to[j] = p;
        if (p >= 0 && p < a.tb.P) atomicAdd(&a.shared[p], 1);
        else bad |= ENT_DEV_BAD_TABLE;
      }
      // No fork reads a row that another writes.
      if (part == 0 && threadIdx.x == 0) a.tb.ctx[r.y] = r.z;
    } else if (r.w >= 0) {
      const int p = from[full], id = a.ids[r.w];
      const bool ok = id >= 0 && id < a.tb.P, there = p >= 0 && p < a.tb.P;
      const int t = (part - a.row_parts) * kPageThreads + threadIdx.x;
      if (!ok || !there) bad |= ENT_DEV_BAD_TABLE;
      if (t == 0) to[full] = ok ? id : -1;
      if (ok && there) copy_block(a.st, p, id, t, (a.parts - a.row_parts) * kPageThreads);
    }
  }
  if (bad) raise_flag(a.tb.flags, bad);
  if (last) a.range[0] = head;
}

// ---------------------------------------------------------------------------
// Release.  Every workgroup takes a holder from some of its sequence's blocks; a block
// that had none left over goes into a bitmap.  The last workgroup lists the bitmap, clears
// it and sets the counts of its blocks back to 0 (given back by who found none left, at
// once: one atomic more in the chain, 7.3 and 14.2 us; the count read before it is taken
// from: 6.2 and 21.3).  Bound by the chain of round trips (row, length, entry, count, bit,
// workgroup count, bitmap: one sequence of 8144 tokens 6.6 us) and by the last workgroup's
// instructions (112 sequences of 73368 entries, 13128 blocks that become free: 13.3 us;
// with the list in a launch of one workgroup and a thread per word 24).
// ---------------------------------------------------------------------------
struct ReleaseArgs {
  Tables tb;
  int N;
  const int* rows;
  int* shared;          // nullable
  int* ids;
  int n_ids;
  int* range;
  u64* bits;            // a word per 64 blocks, kBitPitch apart, zero between calls
  unsigned* tickets;
  int parts;            // workgroups of a sequence
};

__global__ __launch_bounds__(kPlanThreads) void release_kernel(ReleaseArgs a) {
  __shared__ u64 s_b[kPlanThreads];
  __shared__ int s_v[kPlanThreads], s_red[kPlanThreads / 64];
  __shared__ int s_last;
  constexpr int NT = kPlanThreads;
  const int t = threadIdx.x, i = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const int row = a.rows[i], head = a.range[0], end = a.range[1];
  if (head < 0 || head > end || end > a.n_ids) {       // for every workgroup: none is counted
    if (blockIdx.x == 0 && t == 0) raise_flag(a.tb.flags, ENT_DEV_BAD_TABLE);
    return;
  }
  unsigned bad = 0;
  auto length = [&](int r) { return r >= 0 && r < a.tb.R ? a.tb.ctx[r] : -1; };
  auto length_ok = [&](int n) { return n >= 0 && n <= a.tb.MAXB * kBlock; };
  const int n = length(row);
  bool twice = false;
  for (int k = t; k < i; k += NT) twice |= a.rows[k] == row;
  if (__syncthreads_or(twice) || row < 0 || row >= a.tb.R) {
    bad = ENT_DEV_BAD_ROW;
  } else if (!length_ok(n)) {
    bad = ENT_DEV_BAD_CTXLEN;
  } else {
    const int nb = (n + kBlock - 1) / kBlock;
    const int* tab = a.tb.tables + static_cast<long long>(row) * a.tb.MAXB;
    for (int j = part * NT + t; j < nb; j += a.parts * NT) {
      const int p = tab[j];
      if (p < 0 || p >= a.tb.P) {
        bad |= ENT_DEV_BAD_TABLE;
      } else if (a.shared) {
        const int others = atomicSub(&a.shared[p], 1);
        if (others <= 0) (void)set_bit(a.bits, p);
        if (others < 0) bad |= ENT_DEV_BAD_TABLE;      // listed more often than held
      } else if (set_bit(a.bits, p)) {
        bad |= ENT_DEV_BAD_TABLE;
      }
    }
  }
  if (bad) raise_flag(a.tb.flags, bad);
  __builtin_amdgcn_s_waitcnt(0);            // this wave's bits are set
  __syncthreads();
  if (t == 0) s_last = count_out(a.tickets);
  __syncthreads();
  if (!s_last) return;

  const int words = (a.tb.P + 63) / 64;
  u64 x = take_word(a.bits, t, words);
  for (int k = t; k < a.N; k += NT) {
    const int r = a.rows[k];
    if (length_ok(length(r))) a.tb.ctx[r] = 0;
  }
  int total = popc(x), all;
  for (int w = NT + t; w < words; w += NT) total += popc(look_word(a.bits, w, words));
  int k = scan_before<NT>(total, total, s_red);
  int at = head - total;                    // place of the first; those below 0 find no room
  for (int w0 = 0; w0 < words; w0 += NT) {
    if (w0 > 0) x = take_word(a.bits, w0 + t, words);
    if (words > NT) k = scan_before<NT>(popc(x), all, s_red);
    list_bits<NT>(x, at + k, w0 * 64, words - w0, total >= kDense * words, a.ids, s_b, s_v, a.shared);
    if (words > NT) at += all;
  }
  if (t == 0) {
    a.range[0] = max(head - total, 0);
    if (total > head) raise_flag(a.tb.flags, ENT_DEV_CACHE_FULL);
  }
}

// ---------------------------------------------------------------------------
// Compact.  Blocks in use as a bitmap; the last workgroup to mark some forms its prefix
// sums, their number U, and who moves where (the i-th used block from U on to the i-th
// free place below U).  A second launch moves contents and rewrites tables and the free
// list.  Places that are written (below U, free) and read (from U on) do not meet, so moves
// are in any order.  Share counts are formed anew (sequences may have gone without a
// release): -1 for every block in the first launch, and in the second one more for each
// entry at its block's new place, and 0 for the free (10.4 us with 53 moves as without;
// 1004 sequences, 251 holders a block, 237 us, 190 without).  Bound by the copies: 5120
// moved blocks of 64 KB and their mean keys (713 MB) in 127 us of 137 = 5.6 TB/s, over a
// large copy's 4.7; the first launch's 11 are the chain of round trips and 5 for the lists
// of moves.  (One workgroup for a block, keys before values, four pieces a thread: 196 us
// in all; through the caches 157.)
// ---------------------------------------------------------------------------
struct CompactArgs {
  Tables tb;
  int* shared;          // nullable
  int* ids;
  int n_ids;
  int* range;
  int* n_used;          // nullable
  u64* bits;
  u64* words;           // [(P + 63) / 64]  the bitmap again
  int* sums;            // [(P + 63) / 64]  used blocks before the word
  int* from;            // [used] moves
  int* to;
  int* info;            // U, used blocks below U
  unsigned* tickets;
  int parts;            // workgroups of a row of the tables
  int row_wgs;          // of all rows
  PageStore st;
};

__global__ __launch_bounds__(kPlanThreads) void mark_kernel(CompactArgs a) {
  __shared__ u64 s_b[kPlanThreads];
  __shared__ int s_v[kPlanThreads], s_red[kPlanThreads / 64];
  __shared__ int s_below, s_last;
  constexpr int NT = kPlanThreads;
  const int t = threadIdx.x, row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const int n = row < a.tb.R ? a.tb.ctx[row] : 0;      // without sequences: one workgroup that marks nothing
  unsigned bad = 0;
  if (n < 0 || n > a.tb.MAXB * kBlock) {
    bad = ENT_DEV_BAD_CTXLEN;
  } else {
    const int nb = (n + kBlock - 1) / kBlock;
    const int* tab = a.tb.tables + static_cast<long long>(row) * a.tb.MAXB;
    for (int j = part * NT + t; j < nb; j += a.parts * NT) {
      const int p = tab[j];
      if (p >= 0 && p < a.tb.P) set_bit(a.bits, p);
      else bad |= ENT_DEV_BAD_TABLE;
    }
  }
  if (bad) raise_flag(a.tb.flags, bad);
  __builtin_amdgcn_s_waitcnt(0);            // this wave's bits are set
  __syncthreads();
  if (t == 0) s_last = count_out(a.tickets);
  __syncthreads();
  // Nobody waits for these in this launch.
  if (a.shared)
    for (int p = blockIdx.x * NT + t; p < a.tb.P; p += gridDim.x * NT) a.shared[p] = -1;
  if (!s_last) return;

  const int words = (a.tb.P + 63) / 64;
  int U = 0, k = 0, all;
  u64 x = 0;
  for (int w0 = 0; w0 < words; w0 += NT) {
    const int w = w0 + t;
    x = take_word(a.bits, w, words);
    k = U + scan_before<NT>(popc(x), all, s_red);
    if (w < words) {
      a.words[w] = x;
      a.sums[w] = k;
    }
    U += all;
  }
  // A thread meets its own words again (in registers where there is one step).
  if (t == 0) s_below = U;                  // where U is the whole pool, in whole words
  __syncthreads();
  const int last = U / 64;                  // the word that U lies in
  if (last < words && last % NT == t) {
    const bool here = words <= NT;
    s_below = (here ? k : a.sums[last]) + popc((here ? x : a.words[last]) & ((1ull << (U % 64)) - 1ull));
  }
  __syncthreads();
  const int below = s_below;
  for (int w0 = 0; w0 < words; w0 += NT) {
    const int w = w0 + t, base = w * 64;
    if (words > NT) {
      x = w < words ? a.words[w] : 0ull;
      k = w < words ? a.sums[w] : 0;
    }
    // Bits of ids below U.
    const u64 low = w >= words || base >= U ? 0ull : base + 64 <= U ? ~0ull : (1ull << (U - base)) - 1ull;
    const bool dense = U - below >= kDense * words;
    list_bits<NT>(~x & low, base - k, w0 * 64, words - w0, dense, a.to, s_b, s_v, nullptr);
    list_bits<NT>(x & ~low, k + popc(x & low) - below, w0 * 64, words - w0, dense, a.from, s_b, s_v, nullptr);
  }
  if (t == 0) {
    a.info[0] = U;
    a.info[1] = below;
    a.range[0] = a.n_ids - (a.tb.P - U);
    a.range[1] = a.n_ids;
    if (a.n_used) *a.n_used = U;
  }
}

// Half a move by a workgroup: the keys and what belongs to them, or the values.
template <bool STREAM>
__device__ __forceinline__ void move_half(const PageStore& st, int from, int to, bool keys) {
  const int t = threadIdx.x;
  char* const base = keys ? st.k : st.v;
  copy_units<8, STREAM>(at16(static_cast<const void*>(base), from * st.tile_bytes), at16(base, to * st.tile_bytes),
                        static_cast<int>(st.tile_bytes / 16), t, kPageThreads);
  if (keys && st.ksum)
    copy_units<1, STREAM>(at16(static_cast<const void*>(st.ksum), 4ll * from * st.sum_floats),
                          at16(st.ksum, 4ll * to * st.sum_floats), st.sum_floats / 4, t, kPageThreads);
  if (st.ks) {
    float* sc = keys ? st.ks : st.vs;
    for (int i = t; i < st.Hkv; i += kPageThreads)
      sc[static_cast<long long>(to) * st.Hkv + i] = sc[static_cast<long long>(from) * st.Hkv + i];
  }
}

// Workgroups [0, row_wgs) take rows of the tables and the free list, the others blocks.
__global__ __launch_bounds__(kPageThreads) void compact_kernel(CompactArgs a) {
  const int U = a.info[0], below = a.info[1], moves = U - below;
  const int t = threadIdx.x;
  if (blockIdx.x >= static_cast<unsigned>(a.row_wgs)) {
    // By what is moved, not by the pool: few blocks of a large one are soon read again.  Us
    // with / without places in the caches, MB read and written: blocks of 64 KB 27: 13.2 /
    // 15.5, 67: 21.0 / 24.3, 134: 34.1 / 37.7, 174: 47.8 / 45.6, 268: 69.7 / 63.2, 671: 152 /
    // 143; of 8-bit codes 134: 39.1 / 41.0, 168: 49.9 / 47.0; of 4 heads of 64 134: 39.4 / 40.3,
    // 168: 48.5 / 46.3; of floats 134: 32.7 / 36.9, 174: 46.8 / 45.7.
    const bool stream = 4 * a.st.tile_bytes * moves > kStreamCopyBytes;
    for (int m = blockIdx.x - a.row_wgs; m < 2 * moves; m += gridDim.x - a.row_wgs) {
      const int from = a.from[m >> 1], to = a.to[m >> 1];
      if (stream) move_half<true>(a.st, from, to, (m & 1) == 0);
      else move_half<false>(a.st, from, to, (m & 1) == 0);
    }
    return;
  }
  const int first = a.n_ids - (a.tb.P - U);
  for (int i = blockIdx.x * kPageThreads + t; i < a.tb.P - U; i += a.row_wgs * kPageThreads) {
    a.ids[first + i] = U + i;
    if (a.shared) a.shared[U + i] = 0;
  }
  if (moves == 0 && !a.shared) return;
  const int row = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const int n = row < a.tb.R ? a.tb.ctx[row] : 0;
  if (n < 0 || n > a.tb.MAXB * kBlock) return;
  const int nb = (n + kBlock - 1) / kBlock;
  int* tab = a.tb.tables + static_cast<long long>(row) * a.tb.MAXB;
  for (int j = part * kPageThreads + t; j < nb; j += a.parts * kPageThreads) {
    int p = tab[j];
    if (p < 0 || p >= a.tb.P) continue;
    if (p >= U)
      tab[j] = p = a.to[a.sums[p / 64] + popc(a.words[p / 64] & ((1ull << (p % 64)) - 1ull)) - below];
    if (a.shared) atomicAdd(&a.shared[p], 1);
  }
}

PageStore page_store(const ent_ctx* c, void* k, void* v, float* ks, float* vs, float* ksum) {
  const ent_config& f = c->cfg;
  PageStore st{};
  st.k = static_cast<char*>(k);
  st.v = static_cast<char*>(v);
  st.ks = ks;
  st.vs = vs;
  st.ksum = ksum;
  const int elem = ks ? 1 : f.kv_dtype == ENT_BF16 ? 2 : 4;
  st.tile_bytes = static_cast<long long>(f.num_kv_heads) * f.head_dim * kBlock * elem;
  st.sum_floats = f.num_kv_heads * f.head_dim;
  st.Hkv = f.num_kv_heads;
  return st;
}

Tables page_tables(const ent_ctx* c, int R, const int* tables, int* ctx) {
  return Tables{const_cast<int*>(tables), ctx, R, c->cfg.max_blocks_per_seq, c->cfg.num_pool_blocks, c->dev_flags};
}

// Workgroups of NT threads that share a row's entries: about a thousand in all.
int row_parts(const ent_ctx* c, int rows, int nt) {
  return std::max(1, std::min(1024 / rows, (c->cfg.max_blocks_per_seq + nt - 1) / nt));
}

}  // namespace

hipError_t launch_cache_fork(const ent_ctx* c, int N, int R, const int* src, const int* dst,
                             int* tables, int* ctx_lens, int* shared, const int* free_ids, int n_ids,
                             int* free_range, void* k_cache, void* v_cache, float* k_scale,
                             float* v_scale, float* ksum, hipStream_t s) {
  ForkArgs a{page_tables(c, R, tables, ctx_lens), N, src, dst, shared, free_ids, n_ids, free_range,
             c->fork_rec, c->tickets, 1, 2, page_store(c, k_cache, v_cache, k_scale, v_scale, ksum)};
  // Workgroups of a fork: of 256 to 1024 entries each for its row, of 8 KB at least for its
  // block, about a thousand in all.
  const int most = std::max(1, 512 / N);
  a.row_parts = std::min(most, (c->cfg.max_blocks_per_seq + kPageThreads - 1) / kPageThreads);
  a.parts = a.row_parts + static_cast<int>(std::min<long long>(most, (2 * a.st.tile_bytes + 8191) / 8192));
  const size_t lds = (static_cast<size_t>(R) + (R + 31) / 32) * sizeof(int);
  if (N <= kForkOne) {
    hipLaunchKernelGGL(fork_kernel<true>, dim3(N * a.parts), dim3(kPageThreads), lds, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(fork_plan_kernel, dim3(1), dim3(kPlanThreads), lds, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(fork_kernel<false>, dim3(N * a.parts), dim3(kPageThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_cache_release(const ent_ctx* c, int N, int R, const int* rows, const int* tables,
                                int* ctx_lens, int* shared, int* free_ids, int n_ids,
                                int* free_range, hipStream_t s) {
  ReleaseArgs a{page_tables(c, R, tables, ctx_lens), N, rows, shared, free_ids, n_ids, free_range,
                c->page_bits, c->tickets, row_parts(c, N, kPlanThreads)};
  hipLaunchKernelGGL(release_kernel, dim3(N * a.parts), dim3(kPlanThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_cache_compact(const ent_ctx* c, int R, int* tables, const int* ctx_lens, int* shared,
                                int* free_ids, int n_ids, int* free_range, void* k_cache,
                                void* v_cache, float* k_scale, float* v_scale, float* ksum,
                                int* n_used, hipStream_t s) {
  const int rows = std::max(R, 1);
  CompactArgs a{page_tables(c, R, tables, const_cast<int*>(ctx_lens)), shared, free_ids, n_ids, free_range,
                n_used, c->page_bits, c->page_words, c->page_sums, c->kept_phys,
                reinterpret_cast<int*>(c->iscores), c->page_info, c->tickets,
                row_parts(c, rows, kPlanThreads), 0, page_store(c, k_cache, v_cache, k_scale, v_scale, ksum)};
  hipLaunchKernelGGL(mark_kernel, dim3(rows * a.parts), dim3(kPlanThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.parts = row_parts(c, rows, kPageThreads);
  a.row_wgs = rows * a.parts;
  // A workgroup for each half of a move, as far as the pool could have as many, up to 32 a CU
  // (5120 moves, us with 3 / 5 / 8 / 16 / 32 a CU: 142.5 / 143.9 / 145.5 / 140.7 / 137.4).
  const long long halves = std::min<long long>(c->cfg.num_pool_blocks, 2ll * R * c->cfg.max_blocks_per_seq);
  const int copiers = static_cast<int>(std::min<long long>(std::max(halves, 1ll), 32ll * c->num_cu));
  hipLaunchKernelGGL(compact_kernel, dim3(a.row_wgs + copiers), dim3(kPageThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace ent
