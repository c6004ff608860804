// The pages behind the sequences of a paged cache: rows of the block table share blocks, a count per block says how many rows
// hold it.  Rows forked, reordered, cut back and dropped; grown; the held blocks moved to the front of the pool; blocks copied.
//
// All decisions follow from the tables alone, in row and block order (the lowest free block first), so a call gives the same
// tables every time: the only atomics are integer additions to counts, whose order does not matter.
#include "cluster.cuh"
#include "serve_ops.h"

namespace adept {
namespace {

constexpr int PG_THREADS = 1024, PG_CTAS = 8;   // of the one cluster that grows rows, compacts, or forks (smaller tables: one CTA is no faster)

__device__ __forceinline__ bool held(const Pages& p, int e) { return e >= 0 && e < p.n_blocks; }
__device__ __forceinline__ int blocks_of(const Pages& p, int n) { return n / p.block_tokens + (n % p.block_tokens != 0); }

// Exclusive sum over the CTA's 1024 threads, the total in *total.
template <typename T>
__device__ __forceinline__ T cta_scan(T v, T* red, T* total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  T inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T u = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += u;
  }
  __syncthreads();   // red may still be read
  if (lane == 31) red[w] = inc;
  __syncthreads();
  const T mine = red[lane];   // every warp sums the warps' totals for itself: one barrier less
  T x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T u = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += u;
  }
  *total = __shfl_sync(0xffffffffu, x, 31);
  return inc - v + __shfl_sync(0xffffffffu, x - mine, w);
}
// Whether each of counts i .. i + 3 (below n) is that of a free block, as bits.
__device__ __forceinline__ unsigned free_bits(const int* ref, int i, int n) {
  if (i + 4 <= n) {
    const int4 f = *reinterpret_cast<const int4*>(ref + i);
    return (f.x == 0) | (f.y == 0) << 1 | (f.z == 0) << 2 | (f.w == 0) << 3;
  }
  unsigned m = 0;
  for (int k = 0; i + k < n; ++k) m |= (unsigned)(ref[i + k] == 0) << k;
  return m;
}

// ---------------------------------------------------------------------------------------------
// Fork: row b becomes the first length[b] positions of what row source[b] held before the call.
// ---------------------------------------------------------------------------------------------
struct ForkRow {
  int src, nb;   // row to take from (-1: none), blocks
};
__device__ __forceinline__ ForkRow fork_row(const Pages& p, const int* source, const int* length, int b) {
  const int s = source[b], n = length[b];
  if (s < 0 || (n <= 0 && s < p.n_seq)) return ForkRow{-1, 0};
  if (s >= p.n_seq || n > p.max_blocks * p.block_tokens) {   // out of range: the row stays as it is
    p.flag(ERRW_POS);
    return ForkRow{b, p.max_blocks};
  }
  return ForkRow{s, blocks_of(p, n)};
}

// What entry c of row b, whose block is `old`, becomes.
__device__ __forceinline__ int fork_source(const Pages& p, const ForkRow& f, int b, int c, int old) {
  return c >= f.nb ? -1 : f.src == b ? old : p.table[(size_t)f.src * p.max_blocks + c];
}
// The count of an entry that a row takes from another (1: no block), read before any count changes.
__device__ __forceinline__ int fork_count(const Pages& p, int e) { return held(p, e) ? p.ref[e] : e == -1; }
// Such an entry: -1 where it is no block, or one that is counted as free.
__device__ __forceinline__ int fork_taken(const Pages& p, int e, int count) {
  if (count > 0) return e;
  p.flag(ERRW_POS);
  return -1;
}
// The counts of entries that change from blocks `old` to `neu`, blocks or -1 (all on their way before the first is looked at).
template <int N>
__device__ __forceinline__ void fork_counts(const Pages& p, const int (&old)[N], const int (&neu)[N]) {
  int was[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    was[k] = 1;
    if (old[k] == neu[k]) continue;
    if (neu[k] >= 0) atomicAdd(p.ref + neu[k], 1);
    if (held(p, old[k])) was[k] = atomicSub(p.ref + old[k], 1);
    else if (old[k] != -1) p.flag(ERRW_POS);
  }
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (was[k] <= 0) {   // counted as free, or for fewer rows than hold it
      atomicAdd(p.ref + old[k], 1);
      p.flag(ERRW_POS);
    }
}
// Larger tables: a CTA for FORK_CHUNK entries of a row.  The first launch only reads: rows that come from others go into `stage`; the
// second changes counts and table (256 rows of 2048 entries, cut back, and grown by adept_kv_reserve: 12.4 us, by chunks of 256 14.7, of 1024
// 12.2, but 4096 rows of 512 cut back 10.0, by chunks of 1024 10.4, of 256 18.4).
constexpr int FORK_THREADS = 256, FORK_CHUNK = 512;
__global__ void __launch_bounds__(FORK_THREADS) kv_fork_read_kernel(Pages p, const int* source, const int* length, int* stage) {
  PDL_ENTRY();
  const int b = (int)blockIdx.x;
  const ForkRow f = fork_row(p, source, length, b);
  if (f.src == b) return;
  const size_t row = (size_t)b * p.max_blocks;
  constexpr int EACH = FORK_CHUNK / FORK_THREADS;
  for (int c0 = (int)blockIdx.y * FORK_CHUNK; c0 < p.max_blocks; c0 += (int)gridDim.y * FORK_CHUNK) {
    int neu[EACH], n[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int c = c0 + k * FORK_THREADS + threadIdx.x;
      neu[k] = c < p.max_blocks ? fork_source(p, f, b, c, -1) : -1;
    }
#pragma unroll
    for (int k = 0; k < EACH; ++k) n[k] = fork_count(p, neu[k]);
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int c = c0 + k * FORK_THREADS + threadIdx.x;
      if (c < p.max_blocks) stage[row + c] = fork_taken(p, neu[k], n[k]);
    }
  }
}
__global__ void __launch_bounds__(FORK_THREADS) kv_fork_write_kernel(Pages p, const int* source, const int* length, const int* stage) {
  PDL_ENTRY();
  const int b = (int)blockIdx.x;
  const ForkRow f = fork_row(p, source, length, b);
  const size_t row = (size_t)b * p.max_blocks;
  constexpr int EACH = FORK_CHUNK / FORK_THREADS;
  for (int c0 = (int)blockIdx.y * FORK_CHUNK; c0 < p.max_blocks; c0 += (int)gridDim.y * FORK_CHUNK) {
    int old[EACH], neu[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int c = c0 + k * FORK_THREADS + threadIdx.x;
      const bool in = c < p.max_blocks && !(f.src == b && c < f.nb);
      old[k] = in ? p.table[row + c] : -1;
      neu[k] = in && f.src != b ? stage[row + c] : -1;
    }
#pragma unroll
    for (int k = 0; k < EACH; ++k)
      if (old[k] != neu[k]) p.table[row + c0 + k * FORK_THREADS + threadIdx.x] = neu[k];
    fork_counts(p, old, neu);
  }
}

// Tables of up to an entry a thread of one cluster: those hold them between reading and writing (4096 entries, all rows moved, 3.3 us; two entries a
// thread, of 16384, 4.8 where the two launches take 4.0).
__global__ void __launch_bounds__(PG_THREADS) kv_fork_kernel(Pages p, const int* source, const int* length) {
  PDL_ENTRY();
  const int i = (int)blockIdx.x * PG_THREADS + threadIdx.x;
  int old[1] = {-1}, neu[1] = {-1}, n = 1;   // n: the count of a block that is taken from another row, else 1
  if (i < p.n_seq * p.max_blocks) {
    const int b = i / p.max_blocks, c = i - b * p.max_blocks;
    const ForkRow f = fork_row(p, source, length, b);
    old[0] = p.table[i];
    neu[0] = fork_source(p, f, b, c, old[0]);
    if (f.src != b) n = fork_count(p, neu[0]);
  }
  cluster_barrier();   // table and counts have been read
  neu[0] = fork_taken(p, neu[0], n);
  if (old[0] != neu[0]) p.table[i] = neu[0];
  fork_counts(p, old, neu);
}

// ---------------------------------------------------------------------------------------------
// Growth.  One cluster.  Every CTA looks at every row (a thread each; rows that ask for more than NARROW entries: a warp of one of the
// CTAs, which tells the others) and at its part of the counts; then each knows which rows are served, and gives the free blocks of
// its part to the entries that they fall to.  Bound by latency: four loads one behind the other, two barriers.
// ---------------------------------------------------------------------------------------------
constexpr int NARROW = 4, WORDS = 8;
constexpr unsigned ASKS = 1, KEEPS = 2, SHARED = 4, COPIES = 8, WIDE = 16, PART = 32;   // row flags: grows; keeps the shared block that it writes;
                            // writes a shared block in part; gets a copy of that; more than NARROW entries; its first holds positions that stay
constexpr int RELEASED = -0x7fffffff - 1;   // count of a block that its last holder has left, while free blocks are still being looked for
constexpr unsigned MANY = 1u << 30;   // sums of blocks stop here (more than there are)

struct ReserveCall {
  const int *length, *want;
  int *got, *src, *dst;
  unsigned* mask;   // [n_seq][mask_words]: of wide rows, entries that get a new block, from the row's first on that is written
  int mask_words, hash;   // hash: slots of the table of shared blocks (a power of two)
};

// Row b's entries that it will write: [j0, j1); none where it does not grow.
struct GrowRow {
  int n, want, j0, j1;
  bool asks, part;   // part: its first block holds positions that stay
};
__device__ __forceinline__ GrowRow grow_row(const Pages& p, const ReserveCall& a, int b) {
  GrowRow r;
  r.n = a.length[b];
  r.want = a.want[b];
  r.asks = r.want > r.n;
  if (r.n < 0 || r.want > p.max_blocks * p.block_tokens) {
    if (r.asks) p.flag(ERRW_POS);
    r.asks = false;
  }
  r.j0 = r.asks ? r.n / p.block_tokens : 0;
  r.j1 = r.asks ? blocks_of(p, r.want) : 0;
  r.part = r.asks && r.n != r.j0 * p.block_tokens;
  return r;
}
__device__ __forceinline__ unsigned shared_slot(const ReserveCall& a, int e) { return ((unsigned)e * 2654435761u >> 7) & (unsigned)(a.hash - 1); }
// Whether entry *at = e needs a new block, where f is its block's count (0: no block).  A block that is counted as free may be given to
// any row: the entry becomes -1.  (Every CTA that looks at it comes to the same, whether it still finds the block or not.)
__device__ __forceinline__ bool needs(const Pages& p, int* at, int e, int f) {
  if (!held(p, e)) {
    if (e != -1) p.flag(ERRW_POS);
    return true;
  }
  if (f <= 0) {
    p.flag(ERRW_POS);
    *at = -1;
    return true;
  }
  return f > 1;
}

__global__ void __launch_bounds__(PG_THREADS) kv_reserve_kernel(Pages p, ReserveCall a) {
  extern __shared__ __align__(16) unsigned char smem[];
  unsigned* pre = reinterpret_cast<unsigned*>(smem);   // [n_seq] blocks asked for by the rows up to this one
  unsigned *demand = pre + p.n_seq, *word = demand + p.n_seq, *flags = word + p.n_seq;   // [n_seq] blocks; a narrow row's entries; flags
  int *first = reinterpret_cast<int*>(flags + p.n_seq), *width = first + p.n_seq;        // [n_seq] its entries: first .. first + width - 1
  int *key = width + p.n_seq, *cnt = key + a.hash, *last = cnt + a.hash;   // shared blocks that rows write in part
  __shared__ int red[32];
  __shared__ unsigned redu[32], s_taken, s_free[PG_CTAS];
  __shared__ int s_freed, s_any;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = cluster_rank();
  if (tid == 0) s_freed = s_any = 0;
  cluster_arrive();
  for (int i = tid; i < a.hash; i += PG_THREADS) {
    key[i] = -1;
    cnt[i] = 0;
    last[i] = -1;
  }
  if (tid == 0) s_taken = 0;
  PDL_ENTRY();
  // free blocks of the CTA's part of the counts: the first 4096 are looked at once
  const int seg = ((p.n_blocks + PG_CTAS - 1) / PG_CTAS + 3) & ~3, i0 = min(p.n_blocks, rank * seg), i1 = min(p.n_blocks, i0 + seg);
  const unsigned bits0 = free_bits(p.ref, i0 + 4 * tid, i1);
  __syncthreads();   // (the hash)
  for (int b = tid; b < p.n_seq; b += PG_THREADS) {
    const GrowRow r = grow_row(p, a, b);
    int e[NARROW], f[NARROW];
#pragma unroll
    for (int k = 0; k < NARROW; ++k) e[k] = r.j0 + k < r.j1 ? p.table[(size_t)b * p.max_blocks + r.j0 + k] : -1;
#pragma unroll
    for (int k = 0; k < NARROW; ++k) f[k] = held(p, e[k]) ? p.ref[e[k]] : 0;
    unsigned w = 0, fl = r.asks ? ASKS : 0;
#pragma unroll
    for (int k = 0; k < NARROW; ++k)
      if (r.j0 + k < r.j1 && needs(p, p.table + (size_t)b * p.max_blocks + r.j0 + k, e[k], f[k])) w |= 1u << k;
    if (r.j1 - r.j0 > NARROW) fl |= WIDE;
    if (r.part && f[0] > 1) {
      // how many rows ask for the block, and the last of them
      fl |= SHARED;
      unsigned h = shared_slot(a, e[0]);
      for (;;) {   // (at most n_seq keys in a table of twice as many: ends)
        const int was = atomicCAS(key + h, -1, e[0]);
        if (was == -1 || was == e[0]) break;
        h = (h + 1) & (a.hash - 1);
      }
      atomicAdd(cnt + h, 1);
      atomicMax(last + h, b);
    }
    if (r.part) fl |= PART;
    word[b] = w;
    flags[b] = fl;
    first[b] = r.j0;
    width[b] = r.j1 - r.j0;
    if (!(fl & WIDE)) demand[b] = __popc(w);
  }
  int n_free = __popc(bits0), total = 0;
  for (int i = i0 + 4 * (PG_THREADS + tid); i < i1; i += 4 * PG_THREADS) n_free += __popc(free_bits(p.ref, i, i1));
  const int at0 = cta_scan(n_free, red, &total);   // (and the CTA's barrier; the free blocks before mine where a look is enough)
  for (int b = tid; b < p.n_seq; b += PG_THREADS) {
    const unsigned fl = flags[b];
    if (!(fl & SHARED)) continue;
    const GrowRow r = grow_row(p, a, b);
    const int e = p.table[(size_t)b * p.max_blocks + r.j0];
    unsigned h = shared_slot(a, e);
    while (key[h] != e && key[h] != -1) h = (h + 1) & (a.hash - 1);
    if (key[h] == e && cnt[h] == p.ref[e] && last[h] == b) {
      flags[b] = fl | KEEPS;
      word[b] &= ~1u;
      if (!(fl & WIDE)) demand[b] -= 1;
    } else {
      flags[b] = fl | COPIES;
    }
  }
  cluster_wait();   // the others' shared memory is there
  __syncthreads();
  // wide rows, of the CTA's share of them
  for (int b = rank + PG_CTAS * warp; b < p.n_seq; b += PG_CTAS * (PG_THREADS / 32)) {
    if (!(flags[b] & WIDE)) continue;
    const GrowRow r = grow_row(p, a, b);
    int* row = p.table + (size_t)b * p.max_blocks;
    unsigned n = 0;
    for (int j = r.j0; j < r.j1; j += 32 * WORDS) {   // (a long prompt's row: WORDS words' loads under way together)
      int e[WORDS], f[WORDS];
#pragma unroll
      for (int k = 0; k < WORDS; ++k) {
        const int c = j + 32 * k + lane;
        e[k] = c < r.j1 ? row[c] : -1;
      }
#pragma unroll
      for (int k = 0; k < WORDS; ++k) f[k] = held(p, e[k]) ? p.ref[e[k]] : 0;
#pragma unroll
      for (int k = 0; k < WORDS; ++k) {
        const int c = j + 32 * k + lane;
        const unsigned m = __ballot_sync(0xffffffffu, c == r.j0 ? word[b] & 1 : c < r.j1 && needs(p, row + c, e[k], f[k]));
        if (lane == 0 && j + 32 * k < r.j1) a.mask[(size_t)b * a.mask_words + (j - r.j0) / 32 + k] = m;
        n += __popc(m);
      }
    }
    if (lane < PG_CTAS) cluster_store(reinterpret_cast<int*>(demand + b), lane, (int)n);
  }
  if (tid < PG_CTAS) cluster_store(reinterpret_cast<int*>(s_free + rank), tid, total);
  cluster_barrier();

  // sums over the rows, in row order
  unsigned mine_free = 0, all_free = 0, asked = 0;
#pragma unroll
  for (int r = 0; r < PG_CTAS; ++r) {
    if (r < rank) mine_free += s_free[r];
    all_free += s_free[r];
  }
  for (int c0 = 0; c0 < p.n_seq; c0 += PG_THREADS) {
    const int b = c0 + tid, here = min(p.n_seq - c0, PG_THREADS);
    unsigned v = b < p.n_seq ? min(demand[b], MANY) : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned u = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v = min(v + u, MANY);
    }
    if (lane == 31) redu[warp] = v;
    __syncthreads();
    unsigned before = asked;
    for (int w = 0; w * 32 < here; ++w) {   // (as few warps as hold rows)
      if (w == warp) v = min(v + before, MANY);
      before = min(before + redu[w], MANY);
    }
    asked = before;
    if (b < p.n_seq) {
      pre[b] = v;
      // (the sums do not fall: the rows that are served are those up to the last that fits, and rows that ask for nothing)
      if (v <= all_free) atomicMax(&s_taken, v);
    }
    __syncthreads();
  }
  const unsigned taken = s_taken;
  const bool looked_at = seg <= 4 * PG_THREADS;   // every count was read before the first changes (the same in all CTAs)
  // The first `taken` free blocks, in ascending order, to the entries that ask, in order.  (With a thread's four entries looked up before the
  // first is written, 64 prompts of 16000 positions took 19 us instead of 27, but 4 rows that grow by 9, as most calls', 0.4 more.)
  auto give = [&](unsigned k, int id) {
    int b = 0;
    for (int hi = p.n_seq; b < hi;) {   // the first row with a larger sum
      const int mid = (b + hi) / 2;
      if (pre[mid] > k)
        hi = mid;
      else
        b = mid + 1;
    }
    // (not the row's lengths again: d_got may be written over them by another CTA)
    unsigned q = k - (pre[b] - demand[b]);
    int c = first[b];
    if (demand[b] == (unsigned)width[b]) {
      c += (int)q;   // all of them
    } else if (!(flags[b] & WIDE)) {
      unsigned w = word[b];
      for (; q; --q) w &= w - 1;
      c += __ffs(w) - 1;
    } else {
      const unsigned* m = a.mask + (size_t)b * a.mask_words;
      unsigned w = *m;
      for (int n = __popc(w); q >= (unsigned)n; n = __popc(w)) {
        q -= n;
        c += 32;
        w = *++m;
      }
      for (; q; --q) w &= w - 1;
      c += __ffs(w) - 1;
    }
    int* at = p.table + (size_t)b * p.max_blocks + c;
    const int e = *at;
    *at = id;
    p.ref[id] = 1;
    if (!held(p, e)) return;
    if (looked_at) {
      atomicSub(p.ref + e, 1);
    } else {   // counts are still to be read: a block that becomes free here is none of the free ones
      int* ref = p.ref + e;
      for (int was = *(volatile int*)ref, seen; was != RELEASED; was = seen) {
        seen = atomicCAS(ref, was, was == 1 ? RELEASED : was - 1);
        if (seen != was) continue;
        if (was == 1) s_freed = 1;
        break;
      }
    }
    if (c == first[b] && (flags[b] & PART)) {
      a.src[b] = e;
      a.dst[b] = id;
    }
  };
  unsigned base = mine_free;
  for (int i = i0; i < i1 && base < taken; i += 4 * PG_THREADS) {
    const unsigned bits = i == i0 ? bits0 : free_bits(p.ref, i + 4 * tid, i1);
    unsigned k = base + (i1 - i0 <= 4 * PG_THREADS ? at0 : cta_scan(__popc(bits), red, &total));
    for (unsigned m = bits; m && k < taken; m &= m - 1, ++k) give(k, i + 4 * tid + __ffs(m) - 1);
    base += total;
  }
  if (!looked_at) {
    __syncthreads();
    if (tid < PG_CTAS && s_freed) cluster_store(&s_any, tid, 1);
    cluster_barrier();
    if (s_any)
      for (int i = i0 + tid; i < i1; i += PG_THREADS)
        if (p.ref[i] == RELEASED) p.ref[i] = 0;
  }
  if (rank == 0) {
    for (int b = tid; b < p.n_seq; b += PG_THREADS) {
      const unsigned fl = flags[b];
      const bool served = (fl & ASKS) && (pre[b] <= all_free || (demand[b] == 0 && !(fl & KEEPS)));
      a.got[b] = served ? a.want[b] : a.length[b];
      if (!served || !(fl & COPIES)) a.src[b] = a.dst[b] = -1;   // (else written with the block)
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Compaction: with U blocks in use, the k-th of those in use past the first U ids goes to the k-th free one below U.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ unsigned used_bits(const int* ref, int i, int n) {
  if (i + 4 <= n) {
    const int4 f = *reinterpret_cast<const int4*>(ref + i);
    return (f.x > 0) | (f.y > 0) << 1 | (f.z > 0) << 2 | (f.w > 0) << 3;
  }
  unsigned m = 0;
  for (int k = 0; i + k < n; ++k) m |= (unsigned)(ref[i + k] > 0) << k;
  return m;
}
__global__ void __launch_bounds__(PG_THREADS) kv_compact_kernel(Pages p, int* used, int* src, int* dst, int* remap) {
  PDL_ENTRY();
  __shared__ int red[32], s_used[PG_CTAS], s_low;
  const int tid = threadIdx.x, rank = cluster_rank(), ctas = PG_CTAS;
  const int seg = ((p.n_blocks + ctas - 1) / ctas + 3) & ~3, i0 = min(p.n_blocks, rank * seg), i1 = min(p.n_blocks, i0 + seg);
  int n = 0, total = 0;
  for (int i = i0 + 4 * tid; i < i1; i += 4 * PG_THREADS) n += __popc(used_bits(p.ref, i, i1));
  cta_scan(n, red, &total);
  cluster_barrier();   // the others' shared memory is there
  if (tid < ctas) cluster_store(s_used + rank, tid, total);
  cluster_barrier();
  int U = 0, before = 0;
  for (int r = 0; r < ctas; ++r) {
    if (r < rank) before += s_used[r];
    U += s_used[r];
  }
  if (rank == 0 && tid == 0) *used = U;
  // blocks in use below U: counted by the CTA that holds id U (ids end at U where all are in use)
  if (U == p.n_blocks ? rank == 0 : (U >= i0 && U < i1)) {
    n = 0;
    for (int i = i0 + 4 * tid; i < min(i1, U); i += 4 * PG_THREADS) n += __popc(used_bits(p.ref, i, min(i1, U)));
    cta_scan(n, red, &total);
    if (tid < ctas) cluster_store(&s_low, tid, U == p.n_blocks ? U : before + total);
  }
  cluster_barrier();
  const int low = s_low, moves = U - low;
  for (int i = i0; i < i1; i += 4 * PG_THREADS) {
    const unsigned u = used_bits(p.ref, i + 4 * tid, i1);
    int at = before + cta_scan(__popc(u), red, &total);   // in use before the id
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int id = i + 4 * tid + j;
      if (id >= i1) break;
      if (u >> j & 1) {
        if (id >= U) src[at - low] = id;
        ++at;
      } else if (id < U) {
        dst[id - at] = id;
      }
      if (moves) remap[id] = id < U && (u >> j & 1) ? id : -1;
    }
    before += total;
  }
  const int all = ctas * PG_THREADS, me = rank * PG_THREADS + tid;
  for (int k = moves + me; k < p.n_blocks / 2; k += all) src[k] = dst[k] = -1;
  cluster_barrier();
  for (int k = me; k < moves; k += all) {
    const int s = src[k], d = dst[k];
    p.ref[d] = p.ref[s];
    p.ref[s] = 0;
    remap[s] = d;
  }
  cluster_barrier();
  // What an entry is now: remap, where it was counted as held.  (Without moves ids below U are those in use.)
  const size_t entries = (size_t)p.n_seq * p.max_blocks;
  constexpr int EACH = 4;   // (an entry and its look-up are two loads one behind the other: 4 at a time)
  for (size_t i0 = me; i0 < entries; i0 += (size_t)EACH * all) {
    int e[EACH], to[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) e[k] = i0 + (size_t)k * all < entries ? p.table[i0 + (size_t)k * all] : -1;
#pragma unroll
    for (int k = 0; k < EACH; ++k) to[k] = e[k] == -1 || (!moves && e[k] >= 0 && e[k] < U) ? e[k] : moves && held(p, e[k]) ? remap[e[k]] : -1;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      if (to[k] == e[k]) continue;
      if (to[k] == -1) p.flag(ERRW_POS);   // no block, or one that is counted as free: left as it is, unless a block has come there
      if (to[k] >= 0 || (e[k] >= 0 && e[k] < U)) p.table[i0 + (size_t)k * all] = to[k];
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Blocks copied in every layer.  Bound by HBM (a block that several pairs copy is read from L2 but once).  The CTAs take pieces of 32 KB in
// turn, of the pairs that name a block: where most do not (a row that writes into no shared block), those cost a look at their
// numbers.
// ---------------------------------------------------------------------------------------------
constexpr int CP_THREADS = 256, CP_LOADS = 8, CP_PIECE = CP_THREADS * CP_LOADS, CP_PAIRS = 1024;   // 16-byte loads; pairs looked at together

__global__ void __launch_bounds__(CP_THREADS) kv_copy_kernel(const __grid_constant__ CopyLayers c, int n_pairs, const int* src, const int* dst) {
  PDL_ENTRY();
  __shared__ int2 live[CP_PAIRS];
  __shared__ int s_warp[CP_THREADS / 32];
  constexpr int EACH = CP_PAIRS / CP_THREADS;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const unsigned vecs = (unsigned)(c.block_bytes / 16), pieces = (vecs + CP_PIECE - 1) / CP_PIECE, arrays = 2u * c.n_layers;
  for (int i0 = 0; i0 < n_pairs; i0 += CP_PAIRS) {
    // the pairs that name a block, in order (the same in every CTA)
    int2 mine[EACH];
    int n = 0;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int i = i0 + tid * EACH + k;
      mine[k] = i < n_pairs ? make_int2(src[i], dst[i]) : make_int2(-1, -1);
      bool ok = mine[k].x >= 0 && mine[k].y >= 0 && mine[k].x != mine[k].y;
      if (ok && (mine[k].x >= c.n_blocks || mine[k].y >= c.n_blocks)) {
        ok = false;
        if (c.err) atomicOr(c.err, (unsigned)ERRW_POS);
      }
      if (!ok) mine[k].x = -1;
      n += ok;
    }
    int at = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, at, o);
      if (lane >= o) at += u;
    }
    __syncthreads();   // the last pairs' list has been used
    if (lane == 31) s_warp[warp] = at;
    __syncthreads();
    at -= n;
    int total = 0;
#pragma unroll
    for (int w = 0; w < CP_THREADS / 32; ++w) {
      if (w < warp) at += s_warp[w];
      total += s_warp[w];
    }
#pragma unroll
    for (int k = 0; k < EACH; ++k)
      if (mine[k].x >= 0) live[at++] = mine[k];
    __syncthreads();
    const unsigned long long items = (unsigned long long)total * arrays * pieces;
    for (unsigned long long it = blockIdx.x; it < items; it += gridDim.x) {
      const unsigned long long q = it / pieces;
      const unsigned piece = (unsigned)(it - q * pieces), pr = (unsigned)(q / arrays), ar = (unsigned)(q - (unsigned long long)pr * arrays);
      const int2 p = live[pr];
      char* pool = (char*)(ar & 1 ? c.v[ar >> 1] : c.k[ar >> 1]);
      const uint4* from = reinterpret_cast<const uint4*>(pool + p.x * c.block_bytes);
      uint4* to = reinterpret_cast<uint4*>(pool + p.y * c.block_bytes);
      uint4 w[CP_LOADS];
      const unsigned v0 = piece * CP_PIECE + tid;
#pragma unroll
      for (int k = 0; k < CP_LOADS; ++k)
        if (v0 + k * CP_THREADS < vecs) w[k] = from[v0 + k * CP_THREADS];
#pragma unroll
      for (int k = 0; k < CP_LOADS; ++k)
        if (v0 + k * CP_THREADS < vecs) __stcs(to + v0 + k * CP_THREADS, w[k]);
      if (piece == 0 && c.exp_bytes) {
        uint8_t* ex = ar & 1 ? c.v_exp[ar >> 1] : c.k_exp[ar >> 1];
        const uint8_t* ef = ex + (size_t)p.x * c.exp_bytes;
        uint8_t* et = ex + (size_t)p.y * c.exp_bytes;
        if ((c.exp_bytes & 15) == 0) {
          for (int j = tid; j < c.exp_bytes / 16; j += CP_THREADS) reinterpret_cast<uint4*>(et)[j] = reinterpret_cast<const uint4*>(ef)[j];
        } else {
          for (int j = tid; j < c.exp_bytes; j += CP_THREADS) et[j] = ef[j];
        }
      }
    }
  }
}

int sm_count() {
  static const int sms = [] {
    int dev = 0, n = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    return n > 0 ? n : 1;
  }();
  return sms;
}
int mask_words(const Pages& p) { return p.max_blocks / 32 + 1; }

}  // namespace

size_t pages_workspace(const Pages& p) {
  const size_t fork = (size_t)p.n_seq * p.max_blocks, grow = (size_t)p.n_seq * mask_words(p), move = p.n_blocks;
  const size_t most = fork > grow ? fork : grow;
  return (most > move ? most : move) * sizeof(int);
}

cudaError_t launch_kv_fork(cudaStream_t st, const Pages& p, const int* source, const int* length, int* ws) {
  const long long entries = (long long)p.n_seq * p.max_blocks;
  if (entries <= PG_CTAS * PG_THREADS) return launch_cluster(kv_fork_kernel, dim3(PG_CTAS), PG_CTAS, PG_THREADS, 0, st, p, source, length);
  const int chunks = cdiv(p.max_blocks, FORK_CHUNK);
  const dim3 g((unsigned)p.n_seq, (unsigned)(chunks < 65535 ? chunks : 65535));
  cudaError_t e = launch_k(kv_fork_read_kernel, g, dim3(FORK_THREADS), 0, st, p, source, length, ws);
  if (e == cudaSuccess) e = launch_k(kv_fork_write_kernel, g, dim3(FORK_THREADS), 0, st, p, source, length, (const int*)ws);
  return e;
}

cudaError_t launch_kv_reserve(cudaStream_t st, const Pages& p, const int* length, const int* want, int* got, int* src, int* dst,
                              int* ws) {
  ReserveCall a{length, want, got, src, dst, reinterpret_cast<unsigned*>(ws), mask_words(p), 32};
  while (a.hash < 2 * p.n_seq) a.hash *= 2;
  const size_t smem = (size_t)p.n_seq * 24 + (size_t)a.hash * 12;
  struct Tag;
  cudaError_t e = smem_once<Tag>(kv_reserve_kernel, PG_MAX_SEQ * 24 + 2 * PG_MAX_SEQ * 12);
  if (e != cudaSuccess) return e;
  return launch_cluster(kv_reserve_kernel, dim3(PG_CTAS), PG_CTAS, PG_THREADS, smem, st, p, a);
}

cudaError_t launch_kv_compact(cudaStream_t st, const Pages& p, int* used, int* src, int* dst, int* ws) {
  return launch_cluster(kv_compact_kernel, dim3(PG_CTAS), PG_CTAS, PG_THREADS, 0, st, p, used, src, dst, ws);
}

cudaError_t launch_kv_copy_blocks(cudaStream_t st, const CopyLayers& c, int n_pairs, const int* src, const int* dst) {
  // Four CTAs an SM where there is little (128 pairs of blocks of 16 KB in 8 layers, with the calls that name them: 20.2 us, by a CTA a piece 22.2), up to 32, which end and start beside
  // each other, where there is much (2 GB: 321 us, by four 345).
  const long long vecs = c.block_bytes / 16, items = n_pairs * 2ll * c.n_layers * ((vecs + CP_PIECE - 1) / CP_PIECE), sms = sm_count();
  const long long want = items / 4 < 4 * sms ? 4 * sms : items / 4 < 32 * sms ? items / 4 : 32 * sms;
  return launch_k(kv_copy_kernel, dim3((unsigned)(items < want ? items : want)), dim3(CP_THREADS), 0, st, c, n_pairs, src, dst);
}

}  // namespace adept
