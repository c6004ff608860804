// The pages behind the sequences of a paged cache: rows of the block table share blocks, a count per block says how many rows
// hold it.  Rows forked, reordered, cut back and dropped; grown; the held blocks moved to the front of the pool; blocks copied.
//
// All decisions follow from the tables alone, in row and block order (the lowest free block first), so a call gives the same
// tables every time: the only atomics are integer additions to counts, whose order does not matter.
#include "cluster.cuh"
#include "serve_ops.h"

namespace adept {
namespace {

constexpr int PG_THREADS = 1024, PG_CTAS = 8;   // of the one cluster that grows rows or compacts

__device__ __forceinline__ bool held(const Pages& p, int e) { return e >= 0 && e < p.n_blocks; }
__device__ __forceinline__ int blocks_of(const Pages& p, int n) { return n / p.block_tokens + (n % p.block_tokens != 0); }

// Exclusive sum over the CTA's threads (all of them; 1024), the total in *total.
__device__ __forceinline__ int cta_scan(int v, int* red, int* total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += u;
  }
  __syncthreads();   // red may still be read
  if (lane == 31) red[w] = inc;
  __syncthreads();
  if (w == 0) {
    int x = red[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += u;
    }
    red[lane] = x;
  }
  __syncthreads();
  *total = red[31];
  return inc - v + (w ? red[w - 1] : 0);
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

// Counts of the blocks that rows lose and gain, and rows that come from others into `stage`; the table is only read.
__global__ void __launch_bounds__(256) kv_fork_count_kernel(Pages p, const int* source, const int* length, int* stage) {
  PDL_ENTRY();
  const int b = (int)blockIdx.x;
  const ForkRow f = fork_row(p, source, length, b);
  const size_t row = (size_t)b * p.max_blocks;
  for (int c = (f.src == b ? f.nb : 0) + (int)(blockIdx.y * 256 + threadIdx.x); c < p.max_blocks; c += (int)gridDim.y * 256) {
    const int old = p.table[row + c];
    int neu = c < f.nb ? p.table[(size_t)f.src * p.max_blocks + c] : -1;
    if (neu != -1 && !held(p, neu)) {
      p.flag(ERRW_POS);
      neu = -1;
    }
    if (f.src != b) stage[row + c] = neu;
    if (old == neu) continue;
    if (neu >= 0) atomicAdd(p.ref + neu, 1);
    if (old != -1 && (!held(p, old) || atomicSub(p.ref + old, 1) <= 0)) p.flag(ERRW_POS);   // (a count below its holders)
  }
}
__global__ void __launch_bounds__(256) kv_fork_write_kernel(Pages p, const int* source, const int* length, const int* stage) {
  PDL_ENTRY();
  const int b = (int)blockIdx.x;
  const ForkRow f = fork_row(p, source, length, b);
  const size_t row = (size_t)b * p.max_blocks;
  for (int c = (f.src == b ? f.nb : 0) + (int)(blockIdx.y * 256 + threadIdx.x); c < p.max_blocks; c += (int)gridDim.y * 256)
    p.table[row + c] = f.src == b ? -1 : stage[row + c];
}

// ---------------------------------------------------------------------------------------------
// Growth.  One cluster: each CTA a share of the counts and of the rows.
// ---------------------------------------------------------------------------------------------
constexpr unsigned ASKS = 1, KEEPS = 2;   // row flags: grows; keeps the shared block that it writes

struct ReserveCall {
  const int *length, *want;
  int *got, *src, *dst;
  int* list;        // free blocks, ascending, as many as are taken
  unsigned* mask;   // [n_seq][mask_words]: entries that get a new block, from the row's first on that is written
  int mask_words, hash;   // hash: slots of the table of shared blocks (a power of two)
};

// Row b's entries that it will write: [j0, j1); none where it does not grow.
struct GrowRow {
  int n, want, j0, j1;
  bool asks;
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
  return r;
}

__global__ void __launch_bounds__(PG_THREADS) kv_reserve_kernel(Pages p, ReserveCall a) {
  PDL_ENTRY();
  extern __shared__ __align__(16) unsigned char smem[];
  long long* pre = reinterpret_cast<long long*>(smem);                  // [n_seq] blocks asked for by the rows up to this one
  int* demand = reinterpret_cast<int*>(pre + p.n_seq);                  // [n_seq]
  int* flags = demand + p.n_seq;                                        // [n_seq]
  int *key = flags + p.n_seq, *cnt = key + a.hash, *last = cnt + a.hash;   // shared blocks that rows want to write
  __shared__ int red[32], s_free[PG_CTAS];
  __shared__ long long red64[32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = cluster_rank();

  // blocks that are written in part while several rows hold them: how many rows ask for each, and the last of those
  for (int i = tid; i < a.hash; i += PG_THREADS) {
    key[i] = -1;
    cnt[i] = 0;
    last[i] = -1;
  }
  cluster_barrier();   // (also: the others' shared memory is there)
  for (int b = tid; b < p.n_seq; b += PG_THREADS) {
    const GrowRow r = grow_row(p, a, b);
    if (!r.asks || r.n % p.block_tokens == 0) continue;
    const int e = p.table[(size_t)b * p.max_blocks + r.j0];
    if (!held(p, e) || p.ref[e] <= 1) continue;
    int h = (int)(((unsigned)e * 2654435761u) >> 7) & (a.hash - 1);
    for (;;) {   // (at most n_seq keys in a table of twice as many: ends)
      const int was = atomicCAS(key + h, -1, e);
      if (was == -1 || was == e) break;
      h = (h + 1) & (a.hash - 1);
    }
    atomicAdd(cnt + h, 1);
    atomicMax(last + h, b);
  }
  __syncthreads();

  // what each row asks for: the CTA's rows, a warp each
  const int rows = (p.n_seq + PG_CTAS - 1) / PG_CTAS, b0 = min(p.n_seq, rank * rows), b1 = min(p.n_seq, b0 + rows);
  for (int b = b0 + warp; b < b1; b += PG_THREADS / 32) {
    const GrowRow r = grow_row(p, a, b);
    int n = 0, fl = r.asks ? (int)ASKS : 0;
    for (int j = r.j0; j < r.j1; j += 32) {
      const int c = j + lane;
      bool need = false, keep = false;
      if (c < r.j1) {
        const int e = p.table[(size_t)b * p.max_blocks + c];
        if (!held(p, e)) {
          need = true;
          if (e != -1) p.flag(ERRW_POS);
        } else {
          const int f = p.ref[e];
          if (f <= 0) p.flag(ERRW_POS);   // (held, but counted as free)
          need = f > 1;
          if (need && c == r.j0 && r.n % p.block_tokens) {
            int h = (int)(((unsigned)e * 2654435761u) >> 7) & (a.hash - 1);
            while (key[h] != e && key[h] != -1) h = (h + 1) & (a.hash - 1);
            keep = key[h] == e && cnt[h] == f && last[h] == b;
            need = !keep;
          }
        }
      }
      const unsigned m = __ballot_sync(0xffffffffu, need);
      if (__any_sync(0xffffffffu, keep)) fl |= (int)KEEPS;
      if (lane == 0) a.mask[(size_t)b * a.mask_words + (j - r.j0) / 32] = m;
      n += __popc(m);
    }
    if (lane < PG_CTAS) {
      cluster_store(demand + b, lane, n);
      cluster_store(flags + b, lane, fl);
    }
  }
  // free blocks of the CTA's part of the counts
  const int seg = ((p.n_blocks + PG_CTAS - 1) / PG_CTAS + 3) & ~3, i0 = min(p.n_blocks, rank * seg), i1 = min(p.n_blocks, i0 + seg);
  int n_free = 0;
  for (int i = i0 + tid; i < i1; i += PG_THREADS) n_free += p.ref[i] == 0;
  int total = 0;
  cta_scan(n_free, red, &total);
  if (tid < PG_CTAS) cluster_store(s_free + rank, tid, total);
  cluster_barrier();

  // sums over the rows, in row order
  long long asked = 0, taken = 0, mine_free = 0, all_free = 0;
  for (int r = 0; r < PG_CTAS; ++r) {
    if (r < rank) mine_free += s_free[r];
    all_free += s_free[r];
  }
  for (int c0 = 0; c0 < p.n_seq; c0 += PG_THREADS) {
    const int b = c0 + tid;
    long long v = b < p.n_seq ? demand[b] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += u;
    }
    __syncthreads();
    if (lane == 31) red64[warp] = v;
    __syncthreads();
    for (int w = 0; w < warp; ++w) v += red64[w];
    v += asked;
    if (b < p.n_seq) pre[b] = v;
    for (int w = 0; w < PG_THREADS / 32; ++w) asked += red64[w];
  }
  __syncthreads();
  // (the sums do not fall: the rows that are served are those up to the last that fits, and rows that ask for nothing)
  for (int lo = 0, hi = p.n_seq; lo < hi;) {
    const int mid = (lo + hi) / 2;
    if (pre[mid] <= all_free) {
      taken = pre[mid];
      lo = mid + 1;
    } else {
      hi = mid;
    }
  }
  // the first `taken` free blocks, in ascending order
  long long base = mine_free;
  for (int i = i0; i < i1 && base < taken; i += PG_THREADS) {
    const int id = i + tid;
    const bool f = id < i1 && p.ref[id] == 0;
    const int at = cta_scan(f ? 1 : 0, red, &total);
    if (f && base + at < taken) a.list[base + at] = id;
    base += total;
  }
  cluster_barrier();

  for (int b = b0 + warp; b < b1; b += PG_THREADS / 32) {
    const GrowRow r = grow_row(p, a, b);
    const bool served = r.asks && (pre[b] <= all_free || (demand[b] == 0 && !(flags[b] & KEEPS)));
    int src = -1, dst = -1;
    long long k = pre[b] - demand[b];
    if (served && demand[b]) {
      for (int j = r.j0; j < r.j1; j += 32) {
        const unsigned m = a.mask[(size_t)b * a.mask_words + (j - r.j0) / 32];
        if (m >> lane & 1) {
          const int c = j + lane, id = a.list[k + __popc(m & ((1u << lane) - 1))];
          int* at = p.table + (size_t)b * p.max_blocks + c;
          const int e = *at;
          *at = id;
          p.ref[id] = 1;
          if (held(p, e)) {
            atomicSub(p.ref + e, 1);
            if (c == r.j0 && r.n % p.block_tokens) {
              src = e;
              dst = id;
            }
          }
        }
        k += __popc(m);
      }
    }
    if (lane == 0) {   // (the entry that is written in part is the row's first: lane 0's)
      a.got[b] = served ? r.want : r.n;
      a.src[b] = src;
      a.dst[b] = dst;
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Compaction: with U blocks in use, the k-th of those in use past the first U ids goes to the k-th free one below U.
// ---------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(PG_THREADS) kv_compact_kernel(Pages p, int* used, int* src, int* dst, int* remap) {
  PDL_ENTRY();
  __shared__ int red[32], s_used[PG_CTAS], s_low;
  const int tid = threadIdx.x, rank = cluster_rank();
  const int seg = (p.n_blocks + PG_CTAS - 1) / PG_CTAS, i0 = min(p.n_blocks, rank * seg), i1 = min(p.n_blocks, i0 + seg);
  int n = 0, total = 0;
  for (int i = i0 + tid; i < i1; i += PG_THREADS) n += p.ref[i] > 0;
  cta_scan(n, red, &total);
  cluster_barrier();   // the others' shared memory is there
  if (tid < PG_CTAS) cluster_store(s_used + rank, tid, total);
  cluster_barrier();
  int U = 0, before = 0;
  for (int r = 0; r < PG_CTAS; ++r) {
    if (r < rank) before += s_used[r];
    U += s_used[r];
  }
  if (rank == 0 && tid == 0) *used = U;
  // blocks in use below U: counted by the CTA that holds id U (ids end at U where all are in use)
  if (U == p.n_blocks ? rank == 0 : (U >= i0 && U < i1)) {
    n = 0;
    for (int i = i0 + tid; i < min(i1, U); i += PG_THREADS) n += p.ref[i] > 0;
    cta_scan(n, red, &total);
    if (tid < PG_CTAS) cluster_store(&s_low, tid, U == p.n_blocks ? U : before + total);
  }
  cluster_barrier();
  const int low = s_low, moves = U - low;
  for (int i = i0; i < i1; i += PG_THREADS) {
    const int id = i + tid;
    const bool u = id < i1 && p.ref[id] > 0;
    const int at = before + cta_scan(u ? 1 : 0, red, &total);   // in use before id
    if (id < i1 && id < U && !u) dst[id - at] = id;
    if (id < i1 && id >= U) {
      if (u) src[at - low] = id;
      remap[id] = -1;
    }
    before += total;
  }
  const int all = PG_CTAS * PG_THREADS, me = rank * PG_THREADS + tid;
  for (int k = moves + me; k < p.n_blocks / 2; k += all) src[k] = dst[k] = -1;
  cluster_barrier();
  for (int k = me; k < moves; k += all) {
    const int s = src[k], d = dst[k];
    p.ref[d] = p.ref[s];
    p.ref[s] = 0;
    remap[s] = d;
  }
  cluster_barrier();
  const size_t entries = (size_t)p.n_seq * p.max_blocks;
  for (size_t i = me; i < entries; i += all) {
    const int e = p.table[i];
    if (e < U && e >= -1) continue;
    const int to = held(p, e) ? remap[e] : -1;
    if (to >= 0)
      p.table[i] = to;
    else
      p.flag(ERRW_POS);   // (out of range, or a block that is counted as free)
  }
}

// ---------------------------------------------------------------------------------------------
// Blocks copied in every layer.
// ---------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256) kv_copy_kernel(const __grid_constant__ CopyLayers c, int n_pairs, const int* src, const int* dst) {
  PDL_ENTRY();
  const int l = (int)blockIdx.z >> 1, is_v = (int)blockIdx.z & 1;
  char* pool = (char*)(is_v ? c.v[l] : c.k[l]);
  uint8_t* ex = is_v ? c.v_exp[l] : c.k_exp[l];
  for (int i = (int)blockIdx.y; i < n_pairs; i += (int)gridDim.y) {
    const int s = src[i], d = dst[i];
    if (s < 0 || d < 0 || s == d) continue;
    if (s >= c.n_blocks || d >= c.n_blocks) {
      c.err ? (void)atomicOr(c.err, (unsigned)ERRW_POS) : (void)0;
      continue;
    }
    const uint4* from = reinterpret_cast<const uint4*>(pool + s * c.block_bytes);
    uint4* to = reinterpret_cast<uint4*>(pool + d * c.block_bytes);
    for (long long j = blockIdx.x * 256 + threadIdx.x; j < c.block_bytes / 16; j += gridDim.x * 256) to[j] = from[j];
    for (long long j = blockIdx.x * 256 + threadIdx.x; j < c.exp_bytes; j += gridDim.x * 256)
      ex[(size_t)d * c.exp_bytes + j] = ex[(size_t)s * c.exp_bytes + j];
  }
}

int mask_words(const Pages& p) { return p.max_blocks / 32 + 1; }

}  // namespace

size_t pages_workspace(const Pages& p) {
  const size_t fork = (size_t)p.n_seq * p.max_blocks, grow = (size_t)p.n_blocks + (size_t)p.n_seq * mask_words(p);
  return (fork > grow ? fork : grow) * sizeof(int);
}

cudaError_t launch_kv_fork(cudaStream_t st, const Pages& p, const int* source, const int* length, int* ws) {
  int cy = cdiv(p.max_blocks, 256);
  if (cy > 64) cy = 64;
  cudaError_t e = launch_k(kv_fork_count_kernel, dim3((unsigned)p.n_seq, (unsigned)cy), dim3(256), 0, st, p, source, length, ws);
  if (e == cudaSuccess)
    e = launch_k(kv_fork_write_kernel, dim3((unsigned)p.n_seq, (unsigned)cy), dim3(256), 0, st, p, source, length, (const int*)ws);
  return e;
}

cudaError_t launch_kv_reserve(cudaStream_t st, const Pages& p, const int* length, const int* want, int* got, int* src, int* dst,
                              int* ws) {
  ReserveCall a{length, want, got, src, dst, ws, reinterpret_cast<unsigned*>(ws + p.n_blocks), mask_words(p), 32};
  while (a.hash < 2 * p.n_seq) a.hash *= 2;
  const size_t smem = (size_t)p.n_seq * 16 + (size_t)a.hash * 12;
  struct Tag;
  cudaError_t e = smem_once<Tag>(kv_reserve_kernel, PG_MAX_SEQ * 16 + 2 * PG_MAX_SEQ * 12);
  if (e != cudaSuccess) return e;
  return launch_cluster(kv_reserve_kernel, dim3(PG_CTAS), PG_CTAS, PG_THREADS, smem, st, p, a);
}

cudaError_t launch_kv_compact(cudaStream_t st, const Pages& p, int* used, int* src, int* dst, int* ws) {
  return launch_cluster(kv_compact_kernel, dim3(PG_CTAS), PG_CTAS, PG_THREADS, 0, st, p, used, src, dst, ws);
}

cudaError_t launch_kv_copy_blocks(cudaStream_t st, const CopyLayers& c, int n_pairs, const int* src, const int* dst) {
  const long long pieces = (c.block_bytes / 16 + 255) / 256;
  const dim3 g((unsigned)(pieces < 8 ? pieces : 8), (unsigned)(n_pairs < 65535 ? n_pairs : 65535), (unsigned)(2 * c.n_layers));
  return launch_k(kv_copy_kernel, g, dim3(256), 0, st, c, n_pairs, src, dst);
}

}  // namespace adept
