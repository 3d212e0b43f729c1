// Blocks of the paged cache shared by several sequences (fork), handed back to the
// free list (release), and moved to the pool's lower end (compact).
//
// shared[p] counts the holders of block p besides the first.  A fork adds one to
// every full block of its parent and copies the last, begun one, if any; a release
// takes one from every block of its sequences, and those that had none left over are
// free.  Sets of blocks are bitmaps of the pool, so what comes out of them is in
// ascending order whatever order the atomics came in.

#include "ent_internal.h"

#include <algorithm>

namespace ent {
namespace {

constexpr int kPageThreads = 256;
constexpr int kPlanThreads = 1024;

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

// Block `from`'s contents to block `to` by threads t of nt: U pieces of keys and U of
// values in flight a thread.
template <int U>
__device__ __forceinline__ void copy_block(const PageStore& st, int from, int to, int t, int nt) {
  const uint4 *sk = at16(static_cast<const void*>(st.k), from * st.tile_bytes), *sv = at16(static_cast<const void*>(st.v), from * st.tile_bytes);
  uint4 *dk = at16(st.k, to * st.tile_bytes), *dv = at16(st.v, to * st.tile_bytes);
  const int units = static_cast<int>(st.tile_bytes / 16);
  for (int i = t; i < units; i += U * nt) {
    uint4 x[U], y[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * nt < units) {
        x[u] = sk[i + u * nt];
        y[u] = sv[i + u * nt];
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * nt < units) {
        dk[i + u * nt] = x[u];
        dv[i + u * nt] = y[u];
      }
  }
  if (st.ksum) {
    const uint4* s = at16(static_cast<const void*>(st.ksum), 4ll * from * st.sum_floats);
    uint4* d = at16(st.ksum, 4ll * to * st.sum_floats);
    for (int i = t; i < st.sum_floats / 4; i += nt) d[i] = s[i];
  }
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
// find it in a launch of its own.  A fork's workgroups are of two sorts, those that fill
// its row and count holders, and those that copy the begun block.
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
// old one where the range is bad).  mem: R + (R + 31) / 32 ints.
template <int NT, typename F>
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
  const int per = (a.N + NT - 1) / NT;       // consecutive forks of a thread
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
  const int head = fork_plan<kPlanThreads>(a, s_mem, bad, [&](int i, int4 r) { a.rec[i] = r; });
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
    head = fork_plan<kPageThreads>(a, s_mem, bad, [&](int i, int4 x) { if (i == fork) s_rec = x; });
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
      if (ok && there) copy_block<2>(a.st, p, id, t, (a.parts - a.row_parts) * kPageThreads);
    }
  }
  if (bad) raise_flag(a.tb.flags, bad);
  if (last) a.range[0] = head;
}

// ---------------------------------------------------------------------------
// Release.  A first launch takes a holder from every block and marks those that
// had none left; one workgroup then lists the marked ones.
// ---------------------------------------------------------------------------
struct ReleaseArgs {
  Tables tb;
  int N;
  const int* rows;
  int* shared;          // nullable
  int* ids;
  int n_ids;
  int* range;
  unsigned* bits;       // [(P + 31) / 32], zero between calls
};

__device__ __forceinline__ bool range_ok(const int* range, int n_ids, int& head) {
  head = range[0];
  const int end = range[1];
  return head >= 0 && head <= end && end <= n_ids;
}

__global__ __launch_bounds__(kPageThreads) void release_kernel(ReleaseArgs a) {
  const int i = blockIdx.x;
  const bool first = blockIdx.y == 0 && threadIdx.x == 0;
  int head;
  if (!range_ok(a.range, a.n_ids, head)) {
    if (first && i == 0) raise_flag(a.tb.flags, ENT_DEV_BAD_TABLE);
    return;
  }
  const int row = a.rows[i];
  bool twice = false;
  for (int k = threadIdx.x; k < i; k += kPageThreads) twice |= a.rows[k] == row;
  if (__syncthreads_or(twice) || row < 0 || row >= a.tb.R) {
    if (first) raise_flag(a.tb.flags, ENT_DEV_BAD_ROW);
    return;
  }
  const int n = a.tb.ctx[row];
  if (n < 0 || n > a.tb.MAXB * kBlock) {
    if (first) raise_flag(a.tb.flags, ENT_DEV_BAD_CTXLEN);
    return;
  }
  const int nb = (n + kBlock - 1) / kBlock;
  const int* tab = a.tb.tables + static_cast<long long>(row) * a.tb.MAXB;
  unsigned bad = 0;
  for (int j = blockIdx.y * kPageThreads + threadIdx.x; j < nb; j += gridDim.y * kPageThreads) {
    const int p = tab[j];
    if (p < 0 || p >= a.tb.P) {
      bad |= ENT_DEV_BAD_TABLE;
      continue;
    }
    const unsigned bit = 1u << (p % 32);
    if (a.shared) {
      const int old = atomicSub(&a.shared[p], 1);
      if (old <= 0) atomicOr(&a.bits[p / 32], bit);
      if (old < 0) bad |= ENT_DEV_BAD_TABLE;
    } else if (atomicOr(&a.bits[p / 32], bit) & bit) {
      bad |= ENT_DEV_BAD_TABLE;
    }
  }
  if (bad) raise_flag(a.tb.flags, bad);
}

__global__ __launch_bounds__(kPlanThreads) void release_list_kernel(ReleaseArgs a) {
  __shared__ int s_red[kPlanThreads / 64];
  const int t = threadIdx.x;
  int head;
  if (!range_ok(a.range, a.n_ids, head)) return;
  const int words = (a.tb.P + 31) / 32;
  int total = 0, all;
  for (int w0 = 0; w0 < words; w0 += kPlanThreads) {
    int n = 0;
    if (w0 + t < words) n = __popc(a.bits[w0 + t]);
    (void)scan_before<kPlanThreads>(n, all, s_red);
    total += all;
  }
  int at = head - total;                 // place of the first; those below 0 find no room
  for (int w0 = 0; w0 < words; w0 += kPlanThreads) {
    unsigned b = 0;
    if (w0 + t < words) b = a.bits[w0 + t];
    int k = at + scan_before<kPlanThreads>(__popc(b), all, s_red);
    if (b) a.bits[w0 + t] = 0u;
    while (b) {
      const int p = (w0 + t) * 32 + __builtin_ctz(b);
      b &= b - 1;
      if (k >= 0) a.ids[k] = p;
      ++k;
      if (a.shared) a.shared[p] = 0;
    }
    at += all;
  }
  for (int i = t; i < a.N; i += kPlanThreads) {
    const int row = a.rows[i];
    if (row >= 0 && row < a.tb.R) {
      const int n = a.tb.ctx[row];
      if (n >= 0 && n <= a.tb.MAXB * kBlock) a.tb.ctx[row] = 0;
    }
  }
  if (t == 0) {
    a.range[0] = max(head - total, 0);
    if (total > head) raise_flag(a.tb.flags, ENT_DEV_CACHE_FULL);
  }
}

// ---------------------------------------------------------------------------
// Compact.  Blocks in use as a bitmap; one workgroup forms its prefix sums, their
// number U, and who moves where (the i-th used block from U on to the i-th free
// place below U); then contents, counts, tables and the free list.  Places that are
// written (below U, free) and read (from U on) do not meet, so moves are in any order.
// ---------------------------------------------------------------------------
struct CompactArgs {
  Tables tb;
  int* shared;          // nullable
  int* ids;
  int n_ids;
  int* range;
  int* n_used;          // nullable
  unsigned* bits;
  int2* sums;           // [(P + 31) / 32] (used blocks before the word, the word)
  int* from;            // [used] moves
  int* to;
  int* info;            // U, used blocks below U
  PageStore st;
};

__global__ __launch_bounds__(kPageThreads) void mark_kernel(CompactArgs a) {
  const int row = blockIdx.x;
  const int n = a.tb.ctx[row];
  if (n < 0 || n > a.tb.MAXB * kBlock) {
    if (blockIdx.y == 0 && threadIdx.x == 0) raise_flag(a.tb.flags, ENT_DEV_BAD_CTXLEN);
    return;
  }
  const int nb = (n + kBlock - 1) / kBlock;
  const int* tab = a.tb.tables + static_cast<long long>(row) * a.tb.MAXB;
  bool bad = false;
  for (int j = blockIdx.y * kPageThreads + threadIdx.x; j < nb; j += gridDim.y * kPageThreads) {
    const int p = tab[j];
    if (p >= 0 && p < a.tb.P) atomicOr(&a.bits[p / 32], 1u << (p % 32));
    else bad = true;
  }
  if (bad) raise_flag(a.tb.flags, ENT_DEV_BAD_TABLE);
}

__global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(CompactArgs a) {
  __shared__ int s_red[kPlanThreads / 64];
  __shared__ int s_below;
  const int t = threadIdx.x;
  const int words = (a.tb.P + 31) / 32;
  int U = 0, all;
  for (int w0 = 0; w0 < words; w0 += kPlanThreads) {
    unsigned b = 0;
    if (w0 + t < words) b = a.bits[w0 + t];
    const int k = U + scan_before<kPlanThreads>(__popc(b), all, s_red);
    if (w0 + t < words) {
      a.sums[w0 + t] = make_int2(k, static_cast<int>(b));
      a.bits[w0 + t] = 0u;
    }
    U += all;
  }
  if (t == 0) s_below = U;               // where U is the whole pool
  __syncthreads();
  // Each thread reads back what it wrote itself.
  for (int w = t; w < words; w += kPlanThreads) {
    const int2 v = a.sums[w];
    if (w == U / 32) s_below = v.x + __popc(static_cast<unsigned>(v.y) & ((1u << (U % 32)) - 1u));
  }
  __syncthreads();
  const int below = s_below;
  for (int w = t; w < words; w += kPlanThreads) {
    const int2 v = a.sums[w];
    const int base = w * 32;
    unsigned used = static_cast<unsigned>(v.y), free = ~used;
    // Bits of ids below U.
    const unsigned low = base + 32 <= U ? ~0u : base >= U ? 0u : (1u << (U - base)) - 1u;
    int hole = base - v.x;               // free ids before the word
    for (unsigned m = free & low; m; m &= m - 1) a.to[hole++] = base + __builtin_ctz(m);
    int k = v.x + __popc(used & low) - below;
    for (unsigned m = used & ~low; m; m &= m - 1) a.from[k++] = base + __builtin_ctz(m);
  }
  if (t == 0) {
    a.info[0] = U;
    a.info[1] = below;
    a.range[0] = a.n_ids - (a.tb.P - U);
    a.range[1] = a.n_ids;
    if (a.n_used) *a.n_used = U;
  }
}

__global__ __launch_bounds__(kPageThreads) void compact_kernel(CompactArgs a) {
  const int U = a.info[0], below = a.info[1], moves = U - below;
  const int t = threadIdx.x;
  const long long all = static_cast<long long>(gridDim.x) * kPageThreads;
  const long long me = static_cast<long long>(blockIdx.x) * kPageThreads + t;
  for (int m = blockIdx.x; m < moves; m += gridDim.x) {
    const int from = a.from[m], to = a.to[m];
    copy_block<4>(a.st, from, to, t, kPageThreads);
    if (a.shared && t == 0) {
      a.shared[to] = a.shared[from];
      a.shared[from] = 0;
    }
  }
  // Tables: entries from U on follow their blocks.
  if (moves > 0) {
    const long long entries = static_cast<long long>(a.tb.R) * a.tb.MAXB;
    for (long long e = me; e < entries; e += all) {
      const int row = static_cast<int>(e / a.tb.MAXB), j = static_cast<int>(e % a.tb.MAXB);
      const int n = a.tb.ctx[row];
      if (n < 0 || n > a.tb.MAXB * kBlock || j >= (n + kBlock - 1) / kBlock) continue;
      const int p = a.tb.tables[e];
      if (p < U || p >= a.tb.P) continue;
      const int2 v = a.sums[p / 32];
      a.tb.tables[e] = a.to[v.x + __popc(static_cast<unsigned>(v.y) & ((1u << (p % 32)) - 1u)) - below];
    }
  }
  const int first = a.n_ids - (a.tb.P - U);
  for (long long i = me; i < a.tb.P - U; i += all) a.ids[first + i] = U + static_cast<int>(i);
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

// Workgroups that share a row's entries: about a thousand in all, 256 entries each at least.
unsigned row_parts(const ent_ctx* c, int rows) {
  const int most = (c->cfg.max_blocks_per_seq + kPageThreads - 1) / kPageThreads;
  return static_cast<unsigned>(std::max(1, std::min(most, 1024 / std::max(rows, 1))));
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
                c->page_bits};
  hipLaunchKernelGGL(release_kernel, dim3(N, row_parts(c, N)), dim3(kPageThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(release_list_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_cache_compact(const ent_ctx* c, int R, int* tables, const int* ctx_lens, int* shared,
                                int* free_ids, int n_ids, int* free_range, void* k_cache,
                                void* v_cache, float* k_scale, float* v_scale, float* ksum,
                                int* n_used, hipStream_t s) {
  CompactArgs a{page_tables(c, R, tables, const_cast<int*>(ctx_lens)), shared, free_ids, n_ids, free_range,
                n_used, c->page_bits, c->page_sums, c->kept_phys, reinterpret_cast<int*>(c->iscores),
                c->page_info, page_store(c, k_cache, v_cache, k_scale, v_scale, ksum)};
  hipLaunchKernelGGL(mark_kernel, dim3(R, row_parts(c, R)), dim3(kPageThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(compact_kernel, dim3(4 * c->num_cu), dim3(kPageThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace ent
