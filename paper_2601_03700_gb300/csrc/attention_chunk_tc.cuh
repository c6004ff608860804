// Attention of a chunk of new tokens over a paged K/V cache on the tcgen05 tensor cores (what it computes:
// attention_chunk.cu), for the calls whose sequences bring more rows than a warp-level tile.
//
// Tile: two sub-tiles of 128 rows (row = token x query head of one KV head's group, all of one sequence) x key tiles of 128.
// Per key tile and sub-tile S = Q K^T (M 128, N 128, K d_h) and O += P V (P from tensor memory, V as stored, MN-major).
// The two sub-tiles alternate: while the softmax of one runs, the tensor core works on the other.  Tensor memory (512
// columns): S of sub-tile 0 and 1 (128 each), O of 0 and 1 (128 each); P (bf16, 64 columns) takes the place of its S.
//
// Warps:   0..3, 4..7   softmax of sub-tile 0 and 1, a thread per row (its TMEM lane): 128 scores in registers, running
//                       maximum (raised only by more than 2^8), exp2, sum, P to tensor memory; at the end O / l
//          8            issues the matrix instructions:  PV_0(j) S_0(j+1) PV_1(j) S_1(j+1)  (in issue order on the tensor
//                       core, so S_0(j+1) may overwrite P_0(j), and a completed S(j+1) means a completed PV(j))
//          9, 10, 11    fetch K blocks, V blocks and Q by TMA; 10 mends the V tiles at the causal edge
//
// The causal edge: from the first row's position on, a key tile holds keys that not every row attends, or none does.  Scores are
// masked there.  V entries that nobody attends become zero; a NaN or infinite one is replaced by zero and its key noted per
// column (the least one), and a row that attends that key gets NaN in that column at the end: 0 * NaN reaches nobody else.
//
// Work: every (tile, KV head) is a row of key tiles; all of them in a row are cut into equal runs, one per CTA (one CTA per SM),
// so the GPU is evenly loaded whatever the mix of lengths.  A run holds whole tiles and at most two parts of tiles, whose
// (maximum, sum, weighted V) go to the workspace and are joined in order by a second launch.
// 8-bit entries: a launch of its own first turns the positions of this kernel's sequences into bf16 (exactly: code * 2^e) in the
// workspace, once for all the tiles that read them.  Turned by warps of this kernel, tile by tile, they came at 9000 cycles
// a key tile (2048 of matrix instructions): a mixed batch took 121 us.
//
// P is rounded to bf16, as the matrix instructions take it; the sums l take the weights as they are, in fp32.
//
// Measured: 2048 tokens on 16384, 32 heads of 128 on 8, 373 us: 1.57 PFLOP/s, the tensor core 0.69 of the cycles busy, waiting
// for the softmax (a key tile of both sub-tiles takes 3085 cycles, its products 2048).  Short calls pay some 20 us beside their
// key tiles: launch and set-up 4, the first S 4, parts out and joined 8 (256 tokens on 4096, 32 heads: 34 us, 10 of them key
// tiles at that rate).
// Every wait is bounded; a CTA that gives up sets the error word, drains its copies and matrix instructions and leaves.
//
// The device side: the walk over the tiles and the kernels (launched from attention_chunk_tc.cu).
#pragma once
#include "kv_paged.h"
#include "tc_ptx.cuh"

#include <cuda_fp16.h>

namespace adept {
namespace {

constexpr int CT_BM = 128, CT_BN = 128, CT_ROWS = 2 * CT_BM;
constexpr float CT_RAISE = 8.f;
constexpr long long CT_DRAIN_CYCLES = 4000000000LL;

template <int DH>
struct CtShape {
  static constexpr int THREADS = 12 * 32;   // (three whole warpgroups, for setmaxnreg)
  static constexpr int HALVES = DH / 64;
  static constexpr int Q_BYTES = HALVES * CT_BM * 128;             // one sub-tile: [half][row][128 B]
  static constexpr int KV_BYTES = HALVES * CT_BN * 128;            // one K or V stage: [half][key][128 B]
  static constexpr int OFF_K = 2 * Q_BYTES, OFF_V = OFF_K + 2 * KV_BYTES, OFF_ST = OFF_V + 2 * KV_BYTES;
  static constexpr int TOTAL = OFF_ST + 8 * 2048;                  // 32 rows x 64 bytes of output per softmax warp
};

struct CtParams {
  ChunkCall a;
  CUtensorMap kmap, vmap;   // K and V as [n_blocks * n_kv_heads * 16][d_h], box {64, 16}
  CUtensorMap qmap;         // Q as [n_rows][n_heads][d_h], box {64, heads of a group, ts}
  int ts;                   // tokens of a sub-tile
  int runs;                 // CTAs
  int wide;                 // > 0: the maps are of widened entries, `wide` blocks per sequence in order (0: as the pool's)
  unsigned* no_err;         // where time-outs go without an error word (the workspace's last word)
};

// ---- the key tiles of all tiles in a row ----

// (Units fit 31 bits: the launcher refuses calls beyond, ct_total sequences that share rows.)
// sum over i in [0, n) of floor((a i + b) / m); the sum, and a n + b, below 2^32
__device__ unsigned floor_sum(unsigned n, unsigned m, unsigned a, unsigned b) {
  unsigned r = 0;
  while (n > 0) {
    r += (n & 1 ? (n - 1) / 2 * n : n / 2 * (n - 1)) * (a / m) + n * (b / m);
    a %= m;
    b %= m;
    const unsigned y = a * n + b, x = m;
    n = y / m;
    b = y % m;
    m = a;
    a = x;
    if (m == 0) break;
  }
  return r;
}
// Units of token tile t: its key tiles (with given positions, those of the whole sequence), and CT_TILE for what every tile costs
// (its queries' way in, its output's way out: two to three key tiles' time.  Without that, 37 tokens on nothing beside 512 on 1531
// put six tiles of one unit on the first SM: 49 us, 32 with it).
constexpr int CT_TILE = 2;
__device__ __forceinline__ int ct_units(bool given, int c, int len, int tq, int t) {
  return CT_TILE + max(0, (given ? len + CT_BN - 1 : len - c + min((t + 1) * tq, c) + CT_BN - 1) / CT_BN);
}
__device__ int ct_seq_units(bool given, int c, int len, int tq) {
  const int tiles = (c + tq - 1) / tq;
  if (tiles == 0) return 0;
  if (given) return tiles * ct_units(true, c, len, tq, 0);
  const int last = ct_units(false, c, len, tq, tiles - 1);
  if (tiles == 1) return last;
  if (len - c + tq < 1) {   // (first tiles without keys: one by one)
    int r = 0;
    for (int t = 0; t < tiles; ++t) r += ct_units(false, c, len, tq, t);
    return r;
  }
  return last + (tiles - 1) * CT_TILE + (int)floor_sum((unsigned)tiles - 1, CT_BN, (unsigned)tq, (unsigned)(len - c + tq + CT_BN - 1));
}

struct CtTile {
  int seq, q0, c, len, tile, kvh;
  int u0, units;   // first unit of the tile; its units
};
// Inclusive sum over the lanes.
__device__ __forceinline__ int warp_scan(int v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  return v;
}
// All units, taken together by a converged warp.  More than 31 bits hold, which takes row ranges that overlap: no work, flagged.
__device__ int ct_total(const ChunkCall& a, int tq) {
  long long tot = 0;
  for (int b = threadIdx.x & 31; b < a.c.n_seq; b += 32) {
    int q0, c, len;
    chunk_seq(a, b, q0, c, len);
    tot += ct_seq_units(a.row_pos, c, len, tq) * a.c.n_kv_heads;
  }
  const long long hi = __reduce_add_sync(0xffffffffu, (unsigned)(tot >> 24));
  tot = (hi << 24) + __reduce_add_sync(0xffffffffu, (unsigned)tot & 0xffffffu);
  if (tot >> 31) {
    a.c.flag(ERRW_POS);
    return 0;
  }
  return (int)tot;
}
// The tile that unit u lies in.
__device__ void ct_find(const ChunkCall& a, int tq, int u, CtTile& x) {
  const int lane = threadIdx.x & 31;
  int before = 0;
  for (int b0 = 0; b0 < a.c.n_seq; b0 += 32) {
    int q0 = 0, c = 0, len = 0;
    if (b0 + lane < a.c.n_seq) chunk_seq(a, b0 + lane, q0, c, len);
    const int mine = ct_seq_units(a.row_pos, c, len, tq) * a.c.n_kv_heads, inc = a.c.n_seq > 1 ? warp_scan(mine) : mine;
    const unsigned who = __ballot_sync(0xffffffffu, lane < a.c.n_seq - b0 && u < before + inc);
    if (!who) {
      before += __shfl_sync(0xffffffffu, inc, 31);
      continue;
    }
    const int src = __ffs(who) - 1;
    before += __shfl_sync(0xffffffffu, inc - mine, src);
    x.seq = b0 + src;
    x.q0 = __shfl_sync(0xffffffffu, q0, src);
    x.c = __shfl_sync(0xffffffffu, c, src);
    x.len = __shfl_sync(0xffffffffu, len, src);
    const int tiles = (x.c + tq - 1) / tq;
    for (int t0 = 0; t0 < tiles; t0 += 32) {
      const int t = t0 + lane, n = t < tiles ? ct_units(a.row_pos, x.c, x.len, tq, t) * a.c.n_kv_heads : 0, in2 = warp_scan(n);
      const unsigned w2 = __ballot_sync(0xffffffffu, u < before + in2);
      if (!w2) {
        before += __shfl_sync(0xffffffffu, in2, 31);
        continue;
      }
      const int s2 = __ffs(w2) - 1;
      before += __shfl_sync(0xffffffffu, in2 - n, s2);
      x.tile = t0 + s2;
      x.units = ct_units(a.row_pos, x.c, x.len, tq, x.tile);
      x.kvh = (u - before) / x.units;
      x.u0 = before + x.kvh * x.units;
      return;
    }
    return;
  }
}
// The tile behind x.
__device__ __forceinline__ void ct_next(const ChunkCall& a, int tq, CtTile& x) {
  x.u0 += x.units;
  if (++x.kvh < a.c.n_kv_heads) return;
  x.kvh = 0;
  if (++x.tile * tq >= x.c) {
    x.tile = 0;
    x.c = 0;
    while (x.c == 0 && ++x.seq < a.c.n_seq) chunk_seq(a, x.seq, x.q0, x.c, x.len);
  }
  x.units = ct_units(a.row_pos, x.c, x.len, tq, x.tile);
}
// Run i of `runs` (fewer where there are few units): equal shares, the first ones a unit longer; a run that would begin within the
// first units of a tile, before any of its key tiles is through, begins with the tile (ct_snap).
constexpr int CT_MIN_RUN = CT_TILE + 1;
__device__ __forceinline__ int ct_snap(int u, const CtTile& x) { return u - x.u0 <= CT_TILE ? x.u0 : u; }
__device__ __forceinline__ int ct_runs(int total, int runs) { return min(runs, (total + CT_MIN_RUN - 1) / CT_MIN_RUN); }
__device__ __forceinline__ int ct_start(int total, int runs, int i) { return total / runs * i + min(i, total % runs); }

// Workspace: a note per run on the tile it begins inside of; per slot (two a run) 256 (m, l) pairs; and per slot 256 rows of
// weighted V, four columns of all rows after the other (a warp of rows writes whole lines).
struct CtNote {
  int u0;             // first unit of the tile, -1: the run begins with a tile, or is empty
  int row0, kvh, n_tok;   // the tile's first row of Q, KV head, tokens
};   // (16 bytes, as what follows is read)
struct CtWs {
  CtNote* note;
  float* ml;
  float* o;
  __device__ CtWs(const CtParams& p)
      : note((CtNote*)p.a.part), ml(p.a.part + (size_t)p.runs * (sizeof(CtNote) / 4)), o(ml + (size_t)p.runs * 2 * CT_ROWS * 2) {}
  __device__ __forceinline__ float2* ml_at(int slot, int r) const {
    return reinterpret_cast<float2*>(ml) + (size_t)slot * CT_ROWS + r;
  }
  __device__ __forceinline__ float4* o_at(int slot, int dh, int d4, int r) const {
    return reinterpret_cast<float4*>(o) + ((size_t)slot * (dh / 4) + d4) * CT_ROWS + r;
  }
};
constexpr size_t ct_ws_floats(int runs, int dh) {
  return (size_t)runs * (sizeof(CtNote) / 4) + (size_t)runs * 2 * CT_ROWS * (dh + 2);
}

// Non-finite bf16 of a pair: 0xffff in its half; and whether there is one (a carry out of an exponent of all ones).
__device__ __forceinline__ uint32_t ct_bad2(uint32_t x) { return __vcmpeq2(x & 0x7f807f80u, 0x7f807f80u); }
__device__ __forceinline__ uint32_t ct_any_bad2(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }

// Two fp32 at once.
__device__ __forceinline__ uint64_t f2_pack(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void f2_unpack(uint64_t x, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x));
}
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// A CTA's part of one tile: key tiles j_lo .. j_hi.
struct CtSeg {
  CtTile x;
  int j_lo, j_hi, t0, n_tok;
  int lim_lo, k_end;   // keys of the tile's first and of its last token (nobody attends beyond)
  int nt0, nt1, n_it;  // key tiles with keys: per sub-tile, of the segment
  bool whole;          // the whole tile
  const int* table;
  __device__ __forceinline__ void set(const ChunkCall& a, int ts, const CtTile& tile, int u, int u_end) {
    x = tile;
    j_lo = max(u - x.u0 - CT_TILE, 0);
    j_hi = min(x.units, u_end - x.u0) - CT_TILE;
    whole = u == x.u0 && u_end - x.u0 >= x.units;
    t0 = x.tile * 2 * ts;
    n_tok = min(2 * ts, x.c - t0);
    lim_lo = keys(a, 0);
    k_end = keys(a, n_tok - 1);
    const int k_end0 = min(keys(a, min(ts, n_tok) - 1), k_end);   // (given positions might not ascend: nothing behind k_end is touched)
    nt0 = max(min(j_hi, (k_end0 + CT_BN - 1) / CT_BN) - j_lo, 0);
    nt1 = n_tok > ts ? max(min(j_hi, (k_end + CT_BN - 1) / CT_BN) - j_lo, 0) : 0;
    n_it = max(nt0, nt1);
    table = a.c.table + (size_t)x.seq * a.c.max_blocks;
  }
  // keys that token `tok` of the tile attends
  __device__ __forceinline__ int keys(const ChunkCall& a, int tok) const { return chunk_lim(a, x.q0, x.c, x.len, t0 + tok); }
  __device__ __forceinline__ int nt(int sub) const { return sub ? nt1 : nt0; }
  // key tile j (from the segment's first) holds keys that are not everybody's
  __device__ __forceinline__ bool edge(int j) const { return (j_lo + j + 1) * CT_BN > lim_lo || (j_lo + j + 1) * CT_BN > k_end; }
  // the row of key block b (from the sequence's first) in the pools seen as rows of d_h, -1: nobody's, -2: not there
  __device__ __forceinline__ int row_of(const KvPaged& c, int wide, int b) const {
    if (b * 16 >= k_end) return -1;
    const int blk = table[b];
    if (blk < 0 || blk >= c.n_blocks) return -2;
    return ((wide ? x.seq * wide + b : blk) * c.n_kv_heads + x.kvh) * 16;
  }
};

__device__ __forceinline__ void tma_load_q(const CUtensorMap* tm, uint64_t* bar, void* dst, int col, int head, int row) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          smem_u32(dst)),
      "l"((uint64_t)tm), "r"(col), "r"(head), "r"(row), "r"(smem_u32(bar)));
}

// The segments of a CTA follow each other without a stop: every role walks the tiles by itself, and meets the others at
// barriers only: Q full / free, a K or V stage full / free, S, P (two halves), O.  (With a stop of all warps, a
// look-up and Q's loads by all threads at each of a run's two or three segments, a call of ten key tiles a CTA took 70000
// cycles, 27000 of them on key tiles.)
template <int DH>
__global__ void __launch_bounds__(CtShape<DH>::THREADS, 1) chunk_tc_kernel(const __grid_constant__ CtParams p) {
  using L = CtShape<DH>;
  extern __shared__ __align__(1024) uint8_t ct_raw[];
  __shared__ __align__(8) uint64_t q_full, q_free, k_full[2], v_full[2], k_empty[2], v_empty[2], s_full[2], p_half[2], p_full[2],
      o_full[2], v_fix[2], drain;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  __shared__ int s_gone[4];      // blocks of a key tile that are not there, by tile % 4
  // Least key with a non-finite V entry, per column (causal edge), and whether there is one: for each sub-tile, by its segments with
  // keys % 4.  Each sub-tile has slots of its own because one without keys in a segment meets no barrier there: a slot that both
  // read could be needed again while the other still reads.
  __shared__ int s_pk[2][4][DH];
  __shared__ int s_poisoned[2][4];
  __shared__ int s_tok[CT_ROWS], s_off[CT_ROWS];   // token of a row in the tile (-1: none), its head's first column in the group
  __shared__ CtTile s_tile;
  __shared__ int s_u0, s_u1;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long wlim = wait_limit();
  volatile int* abort_flag = &s_abort;
  uint8_t* sm = ct_raw + ((1024 - (smem_u32(ct_raw) & 1023)) & 1023);
  uint8_t *sQ = sm, *sK = sm + L::OFF_K, *sV = sm + L::OFF_V;
  const ChunkCall& a = p.a;
  unsigned* err = a.c.err ? a.c.err : p.no_err;

  if (tid == 0) {
    mbar_init(&q_full, 1);
    mbar_init(&q_free, 1);
    for (int s = 0; s < 2; ++s) {
      mbar_init(&k_full[s], 1);
      mbar_init(&v_full[s], 1);
      mbar_init(&k_empty[s], 1);
      mbar_init(&v_empty[s], 1);
      mbar_init(&s_full[s], 1);
      mbar_init(&p_half[s], 4);
      mbar_init(&p_full[s], 4);
      mbar_init(&o_full[s], 1);
      mbar_init(&v_fix[s], 1);
    }
    mbar_init(&drain, 1);
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  const int group = a.n_heads / a.c.n_kv_heads, ts = p.ts, tq = 2 * ts, run = (int)blockIdx.x;
  if (tid >= 352 && tid < 355) {   // the maps' first use is a fetch of its own
    const CUtensorMap* map = tid == 352 ? &p.kmap : tid == 353 ? &p.vmap : &p.qmap;
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)map) : "memory");
  }
  if (warp == 8) {
    tmem_alloc(&s_tmem, 512);
    tmem_relinquish();
  }
  if (warp < 8) {   // (a row per thread)
    const int rr = tid & 127, tk = rr / group;
    s_tok[tid] = tk < ts ? (tid >> 7) * ts + tk : -1;
    s_off[tid] = rr % group * DH;
  }
  if (!a.late) pdl_wait();
  if (warp == 9 || warp == 10) {   // where the run begins, where it ends
    const int tot = ct_total(a, tq), runs = ct_runs(tot, p.runs), i = min(run + warp - 9, runs);
    CtTile x{};
    int u0 = tot;
    if (i < runs) {
      const int at = ct_start(tot, runs, i);
      ct_find(a, tq, at, x);
      u0 = ct_snap(at, x);
    }
    if (lane == 0) {
      if (warp == 9) {
        s_u0 = u0;
        s_tile = x;
      } else {
        s_u1 = u0;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_launch_dependents();   // after the tensor memory is held
  const uint32_t tmem = s_tmem;
  const int u_end = s_u1;
  int u = s_u0;
  CtTile x = s_tile;
  if (tid == 0) {   // the join's note: what tile this run begins inside of
    const int t0 = x.tile * tq;
    CtWs(p).note[run] = CtNote{u < u_end && u > x.u0 ? x.u0 : -1, x.q0 + t0, x.kvh, min(tq, x.c - t0)};
  }
  CtSeg g{};
  bool ok = true;

  // 384 x 168 registers at launch: 256 x 208 + 128 x 88
  if (warp < 8) {
    // ---- softmax of a row per thread
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int sub = warp >> 2, r = tid & 127, tok = s_tok[tid];
    const uint32_t base = tmem + ((uint32_t)((warp & 3) * 32) << 16), s_col = base + (uint32_t)(sub * 128),
                   o_col = base + 256u + (uint32_t)(sub * 128);
    const float sc = a.scale_log2;
    const CtWs ws(p);
    uint8_t* stage = sm + L::OFF_ST + warp * 2048;
    int ns = 0, no = 0, kt = 0;   // S tiles, outputs, key tiles so far
    int seg = -1;   // the sub-tile's segments with keys so far
    while (u < u_end) {
      g.set(a, ts, x, u, u_end);
      const bool mine = tok >= 0 && tok < g.n_tok;
      const int lim = mine ? min(g.keys(a, tok), g.k_end) : 0;
      const int sub_lo = sub * ts < g.n_tok ? g.keys(a, sub * ts) : 0;   // keys of the sub-tile's first token
      const int n_my = g.nt(sub);
      seg += n_my > 0;
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < n_my; ++j) {
        if (!(ok = mbar_wait_warp(&s_full[sub], (uint32_t)(ns & 1), abort_flag, err, wlim))) break;
        ++ns;
        tc_fence_after();
        float s[CT_BN];
        tmem_ld128(s_col, s);
        const int k0 = (g.j_lo + j) * CT_BN, gone = s_gone[(kt + j) & 3];
        if (k0 + CT_BN > sub_lo || gone) {
          const int nk_r = lim - k0;
#pragma unroll
          for (int e = 0; e < CT_BN; ++e)
            if (e >= nk_r || (gone >> (e >> 4) & 1)) s[e] = -INFINITY;
        }
        float mx[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) mx[e] = max3(s[e], s[e + 8], s[e + 16]);
#pragma unroll
        for (int e = 24; e < CT_BN - 8; e += 16)
#pragma unroll
          for (int q = 0; q < 8; ++q) mx[q] = max3(mx[q], s[e + q], s[e + 8 + q]);
#pragma unroll
        for (int q = 0; q < 8; ++q) mx[q] = fmaxf(mx[q], s[CT_BN - 8 + q]);
        const float tmax = fmaxf(max3(max3(mx[0], mx[1], mx[2]), mx[3], mx[4]), max3(mx[5], mx[6], mx[7])) * sc;
        float m_new = m;
        if (tmax > m && (m == -INFINITY || tmax - m > CT_RAISE)) m_new = tmax;
        const float f = (m == -INFINITY || m_new == m) ? 1.f : ex2_approx(m - m_new);
        if (__any_sync(0xffffffffu, f != 1.f)) {   // (S of this tile is complete, so O of the one before it is)
#pragma unroll 1
          for (int c = 0; c < DH / 32; ++c) {
            float v[32];
            tmem_ld32(o_col + (uint32_t)(c * 32), v);
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] *= f;
            tmem_st32(o_col + (uint32_t)(c * 32), v);
          }
          l *= f;
        }
        m = m_new;
        const float ref = m == -INFINITY ? 0.f : m;
        const uint64_t sc2 = f2_pack(sc, sc), ref2 = f2_pack(-ref, -ref);
        uint64_t sum[4] = {0, 0, 0, 0};
        // P in two halves: O += P V of the first half's keys runs beside the second half's exponentials
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t pk[32];
#pragma unroll
          for (int e = 0; e < 64; e += 2) {
            float p0, p1;
            f2_unpack(f2_fma(f2_pack(s[h * 64 + e], s[h * 64 + e + 1]), sc2, ref2), p0, p1);
            p0 = ex2_approx(p0);
            p1 = ex2_approx(p1);
            sum[(e >> 1) & 3] = f2_add(sum[(e >> 1) & 3], f2_pack(p0, p1));
            const __nv_bfloat162 pr = __floats2bfloat162_rn(p0, p1);
            pk[e >> 1] = *reinterpret_cast<const uint32_t*>(&pr);
          }
          tmem_st32u(s_col + (uint32_t)(h * 32), pk);
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(h ? &p_full[sub] : &p_half[sub]);
        }
        float l0, l1;
        f2_unpack(f2_add(f2_add(sum[0], sum[1]), f2_add(sum[2], sum[3])), l0, l1);
        l += l0 + l1;
      }
      if (!ok) break;
      kt += g.n_it;   // (the segment's key tiles: what s_gone goes by)
      // O / l, or the part
      float v[DH];
      if (n_my > 0) {   // (the same for the whole warp)
        if (!(ok = mbar_wait_warp(&o_full[sub], (uint32_t)(no & 1), abort_flag, err, wlim))) break;
        ++no;
        tc_fence_after();
        if constexpr (DH == 128) tmem_ld128(o_col, v);
        else tmem_ld64(o_col, v);
      } else {
#pragma unroll
        for (int e = 0; e < DH; ++e) v[e] = 0.f;
      }
      if (n_my > 0 && s_poisoned[sub][seg & 3]) {
#pragma unroll
        for (int e = 0; e < DH; ++e)
          if (s_pk[sub][seg & 3][e] < lim) v[e] = NAN;
      }
      if (sub == 0 || g.n_tok > ts) {
        if (g.whole) {
          // through the warp's stage, 32 columns at a time, so that whole sectors are written
          const float inv = l == 0.f ? 0.f : 1.f / l;
          bf16* out = (bf16*)a.out + (size_t)(g.x.q0 + g.t0) * a.ld_out + (size_t)g.x.kvh * group * DH;
#pragma unroll
          for (int c = 0; c < DH / 32; ++c) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t w[4];
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const __nv_bfloat162 pr = __floats2bfloat162_rn(v[c * 32 + 8 * e + 2 * q] * inv, v[c * 32 + 8 * e + 2 * q + 1] * inv);
                w[q] = *reinterpret_cast<const uint32_t*>(&pr);
              }
              *reinterpret_cast<uint4*>(stage + lane * 64 + ((e ^ ((lane >> 1) & 3)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
            }
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int rr = k * 8 + (lane >> 2), pc = lane & 3, row = warp * 32 + rr, tk = s_tok[row];
              if (tk >= 0 && tk < g.n_tok)
                *reinterpret_cast<uint4*>(out + tk * a.ld_out + s_off[row] + c * 32 + pc * 8) =
                    *reinterpret_cast<const uint4*>(stage + rr * 64 + ((pc ^ ((rr >> 1) & 3)) << 4));
            }
            __syncwarp();
          }
        } else if (mine) {
          const int slot = run * 2 + (u == g.x.u0 ? 1 : 0);
          *ws.ml_at(slot, sub * 128 + r) = make_float2(m, l);
#pragma unroll
          for (int e = 0; e < DH / 4; ++e)
            *ws.o_at(slot, DH, e, sub * 128 + r) = make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
        }
      }
      ct_next(a, tq, x);
      u = x.u0;
    }
  } else if (warp == 8) {
    // ---- matrix instructions: one thread (a warp that meets at every wait took 3900 cycles a key tile to issue what the tensor
    // core does in 2048), descriptors made once and moved by their address field
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    constexpr uint32_t IDESC_S = umma_idesc(CT_BN, false), IDESC_O = umma_idesc(DH, true);
    const uint64_t dq = sdesc_sw128(smem_u32(sQ)), dk = sdesc_sw128(smem_u32(sK)), dv = sdesc_mn_sw128(smem_u32(sV), CT_BN * 128);
    if (elect_one()) {
      int nq = 0, nk = 0, nv = 0, np[2] = {0, 0}, nf[2] = {0, 0};   // Q, K, V, P so far, mended V per stage
      auto wait = [&](uint64_t* bar, int phase) { return ok = mbar_wait(bar, (uint32_t)(phase & 1), abort_flag, err, wlim); };
      while (u < u_end && ok) {
        g.set(a, ts, x, u, u_end);
        if (g.n_it > 0 && !wait(&q_full, nq++)) break;
        for (int j = -1; j < g.n_it; ++j) {
          const int kn = nk, vn = nv, ks = kn & 1, vs = vn & 1;
          if (j + 1 < g.n_it) {
            if (!wait(&k_full[ks], kn >> 1)) break;
            ++nk;
          }
          if (j >= 0) {
            if (!wait(&v_full[vs], vn >> 1)) break;
            if ((g.edge(j) || s_gone[vn & 3]) && !wait(&v_fix[vs], nf[vs]++)) break;
            ++nv;
          }
          const uint64_t dks = dk + (uint64_t)(ks * (L::KV_BYTES >> 4)), dvs = dv + (uint64_t)(vs * (L::KV_BYTES >> 4));
#pragma unroll
          for (int sub = 0; sub < 2; ++sub) {
            if (j >= 0 && j < g.nt(sub)) {
              const uint32_t pa = tmem + (uint32_t)(sub * 128), oa = tmem + 256u + (uint32_t)(sub * 128);
              if (!wait(&p_half[sub], np[sub])) break;
              // (a P of this segment: its warps have read O of the segment before)
              tc_fence_after();
#pragma unroll
              for (int kk = 0; kk < 4; ++kk)
                umma_bf16_ts(oa, pa + (uint32_t)(kk * 8), dvs + (uint64_t)(kk * (16 * 128 >> 4)), IDESC_O, (j > 0 || kk > 0) ? 1u : 0u);
              if (!wait(&p_full[sub], np[sub])) break;
              tc_fence_after();
#pragma unroll
              for (int kk = 4; kk < 8; ++kk)
                umma_bf16_ts(oa, pa + (uint32_t)(kk * 8), dvs + (uint64_t)(kk * (16 * 128 >> 4)), IDESC_O, 1u);
              ++np[sub];
              if (j == g.nt(sub) - 1) umma_commit(&o_full[sub]);
            }
            if (j + 1 < g.nt(sub)) {
              tc_fence_after();
#pragma unroll
              for (int kk = 0; kk < DH / 16; ++kk) {
                const uint64_t at = (uint64_t)(((kk >> 2) * CT_BM * 128 + (kk & 3) * 32) >> 4);
                umma_bf16(tmem + (uint32_t)(sub * 128), dq + (uint64_t)(sub * (L::Q_BYTES >> 4)) + at, dks + at, IDESC_S, kk > 0 ? 1u : 0u);
              }
              umma_commit(&s_full[sub]);
            }
          }
          if (!ok) break;
          if (j + 1 < g.n_it) umma_commit(&k_empty[ks]);
          if (j + 1 == g.n_it - 1) umma_commit(&q_free);   // the segment's last S
          if (j >= 0) umma_commit(&v_empty[vs]);
        }
        ct_next(a, tq, x);
        u = x.u0;
      }
      // every matrix instruction has completed before tensor memory is given back
      umma_commit(&drain);
      const long long c0 = clock64();
      while (!mbar_try_wait(&drain, 0) && clock64() - c0 < CT_DRAIN_CYCLES) {
      }
    }
    __syncwarp();
  } else if (warp == 11) {
    // ---- TMA producer of Q: a segment's, once S of the one before it is through
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    int nq = 0;
    while (u < u_end) {
      g.set(a, ts, x, u, u_end);
      if (g.n_it > 0) {
        if (nq > 0 && !mbar_wait_warp(&q_free, (uint32_t)((nq - 1) & 1), abort_flag, err, wlim)) break;
        if (elect_one()) {
          const int subs = g.n_tok > ts ? 2 : 1;
          mbar_expect_tx(&q_full, (uint32_t)(subs * L::HALVES * ts * group * 128));
          for (int b = 0; b < subs; ++b)
            for (int hf = 0; hf < L::HALVES; ++hf)
              tma_load_q(&p.qmap, &q_full, sQ + b * L::Q_BYTES + hf * CT_BM * 128, hf * 64, g.x.kvh * group, g.x.q0 + g.t0 + b * ts);
        }
        __syncwarp();
        ++nq;
      }
      ct_next(a, tq, x);
      u = x.u0;
    }
    if (lane == 0) {   // (landed before the CTA ends)
      const long long c0 = clock64();
      while (nq > 0 && !mbar_try_wait(&q_full, (uint32_t)((nq - 1) & 1)) && clock64() - c0 < CT_DRAIN_CYCLES) {
      }
    }
    __syncwarp();
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    // ---- TMA producers: K (warp 9), V (warp 10, which also mends the V tiles at the edge)
    const bool kw = warp == 9;
    uint64_t *full = kw ? k_full : v_full, *empty = kw ? k_empty : v_empty;
    const CUtensorMap* map = kw ? &p.kmap : &p.vmap;
    uint8_t* dst0 = kw ? sK : sV;
    int cnt = 0;   // tiles sent so far
    // V tile j (the vi-th, blocks `gone` of it not there): entries nobody attends to zero, non-finite ones noted
    int seg0 = -1, seg1 = -1;   // segments with keys so far, of either sub-tile
    // The segment's notes for a sub-tile begin (warp-converged): no key in any column yet.
    auto note = [&](int sub, int slot) {
      if (s_poisoned[sub][slot]) return;
      __syncwarp();
      for (int e = lane; e < DH; e += 32) s_pk[sub][slot][e] = 0x7fffffff;
      s_poisoned[sub][slot] = 1;
      __syncwarp();
    };
    auto mend = [&](int j, int vi, int gone) {
      const int s = vi & 1;
      if (!mbar_wait_warp(&v_full[s], (uint32_t)((vi >> 1) & 1), abort_flag, err, wlim)) return false;
      uint8_t* v = sV + s * L::KV_BYTES;
      const int k0 = (g.j_lo + j) * CT_BN, n_key = min(g.k_end - k0, CT_BN);
      auto piece = [&](int hf, int key, int c) { return reinterpret_cast<uint4*>(v + hf * CT_BN * 128 + key * 128 + (c << 4)); };
      // (first to zero: what was not fetched may hold anything)
      for (int i = n_key * 8 + lane; i < CT_BN * 8; i += 32)
        for (int hf = 0; hf < L::HALVES; ++hf) *piece(hf, i >> 3, i & 7) = make_uint4(0, 0, 0, 0);
      if (gone)
        for (int i = lane; i < CT_BN * 8; i += 32)
          if (gone >> (i >> 7) & 1)
            for (int hf = 0; hf < L::HALVES; ++hf) *piece(hf, i >> 3, i & 7) = make_uint4(0, 0, 0, 0);
      __syncwarp();
#pragma unroll 1
      for (int i0 = 0; i0 < n_key * 8; i0 += 128) {   // 16 keys: a fetched block, or zeros
        auto at = [&](int q) { return piece(q >> 2, (i0 >> 3) + (q & 3) * 4 + (lane >> 3), lane & 7); };
        uint32_t any = 0;
#pragma unroll
        for (int q = 0; q < 4 * L::HALVES; ++q) {
          const uint4 y = *at(q);
          any |= ct_any_bad2(y.x) | ct_any_bad2(y.y) | ct_any_bad2(y.z) | ct_any_bad2(y.w);
        }
        if (__any_sync(0xffffffffu, any != 0)) {
          const bool of0 = j < g.nt0, of1 = j < g.nt1;   // (a sub-tile through with its key tiles may be reading its notes)
          if (of0) note(0, seg0 & 3);
          if (of1) note(1, seg1 & 3);
#pragma unroll 1
          for (int q = 0; q < 4 * L::HALVES; ++q) {
            const uint4 y = *at(q);
            const int key = (i0 >> 3) + (q & 3) * 4 + (lane >> 3), col = (q >> 2) * 64 + (((lane & 7) ^ (key & 7)) << 3);
            const uint32_t b[4] = {ct_bad2(y.x), ct_bad2(y.y), ct_bad2(y.z), ct_bad2(y.w)};
            *at(q) = make_uint4(y.x & ~b[0], y.y & ~b[1], y.z & ~b[2], y.w & ~b[3]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (b[e >> 1] >> ((e & 1) * 16) & 1) {
                if (of0) atomicMin(&s_pk[0][seg0 & 3][col + e], k0 + key);
                if (of1) atomicMin(&s_pk[1][seg1 & 3][col + e], k0 + key);
              }
          }
        }
      }
      fence_async_shared();
      __syncwarp();
      if (lane == 0) mbar_arrive(&v_fix[s]);
      return true;
    };
    while (u < u_end && ok) {
      g.set(a, ts, x, u, u_end);
      seg0 += g.nt0 > 0;
      seg1 += g.nt1 > 0;
      int gone = 0, gone_prev = 0;
      for (int j = 0; j <= g.n_it && ok; ++j) {
        gone_prev = gone;
        if (!kw && j > 0 && (g.edge(j - 1) || gone_prev) && !(ok = mend(j - 1, cnt - 1, gone_prev))) break;
        if (j == g.n_it) break;
        const int s = cnt & 1, row = lane < 8 ? g.row_of(a.c, p.wide, (g.j_lo + j) * 8 + lane) : -1;
        const unsigned on = __ballot_sync(0xffffffffu, row >= 0);
        gone = (int)__ballot_sync(0xffffffffu, row == -2);
        if (gone && lane == 0) a.c.flag(ERRW_POS);
        int rows8[8];
#pragma unroll
        for (int b = 0; b < 8; ++b) rows8[b] = __shfl_sync(0xffffffffu, row, b);
        if (cnt >= 2 && !(ok = mbar_wait_warp(&empty[s], (uint32_t)(((cnt >> 1) - 1) & 1), abort_flag, err, wlim))) break;
        // No notes of the segment yet, in the place of those of the sub-tile's four segments before (k).  V of two tiles ago is through, so
        // the sub-tile has handed over a P of its segment k + 2, behind its reading of the notes of k and k + 1.
        if (!kw && j == 0) {
          if (lane == 0 && g.nt0 > 0) s_poisoned[0][seg0 & 3] = 0;
          if (lane == 0 && g.nt1 > 0) s_poisoned[1][seg1 & 3] = 0;
          __syncwarp();
        }
        if (elect_one()) {
          if (kw) s_gone[cnt & 3] = gone;   // (tile cnt - 4 is through: its K stage has been freed twice over)
          // (blocks that are not fetched leave the stage's old contents: masked in S, mended in V)
          mbar_expect_tx(&full[s], (uint32_t)(__popc(on) * 16 * 128 * L::HALVES));
          for (int b = 0; b < 8; ++b)
            if (on >> b & 1)
              for (int hf = 0; hf < L::HALVES; ++hf)
                tma_load_2d(map, &full[s], dst0 + s * L::KV_BYTES + hf * CT_BN * 128 + b * 16 * 128, hf * 64, rows8[b]);
        }
        __syncwarp();
        ++cnt;
      }
      ct_next(a, tq, x);
      u = x.u0;
    }
    // every copy sent has landed before the CTA ends
    if (lane == 0) {
      for (int t = max(0, cnt - 2); t < cnt; ++t) {
        const long long c0 = clock64();
        while (!mbar_try_wait(&full[t & 1], (uint32_t)((t >> 1) & 1)) && clock64() - c0 < CT_DRAIN_CYCLES) {
        }
      }
    }
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 8) tmem_dealloc(tmem, 512);
  if (a.late) pdl_wait();
}

// Entries of 8 bits as bf16.  Work: the blocks of positions of this launch's sequences, K and V apart, all heads of one at a time;
// CTA i of n takes the i-th of n equal runs of them (the lengths are known on the device only).  A block goes to its place in
// the pool, or (wide > 0) to block b of `wide` of its sequence; one that several sequences share is written more than once there,
// with the same values.
constexpr int CW_THREADS = 256;
template <int DH>
__global__ void __launch_bounds__(CW_THREADS) chunk_widen_kernel(const __grid_constant__ ChunkCall a, int wide, bf16* k_out,
                                                                 bf16* v_out) {
  PDL_ENTRY();
  __shared__ int s_seq, s_blk, s_len;
  __shared__ long long s_u0, s_u1;
  const int lane = threadIdx.x & 31;
  if (threadIdx.x < 32) {
    long long tot = 0;
    for (int b = lane; b < a.c.n_seq; b += 32) {
      int q0, c, len;
      chunk_seq(a, b, q0, c, len);
      tot += (len + 15) / 16;
    }
    tot = __reduce_add_sync(0xffffffffu, (unsigned)(tot & 0xffffff)) + ((long long)__reduce_add_sync(0xffffffffu, (unsigned)(tot >> 24)) << 24);
    const long long u0 = 2 * tot * blockIdx.x / gridDim.x, u1 = 2 * tot * (blockIdx.x + 1) / gridDim.x;
    long long before = 0;
    for (int b0 = 0; b0 < a.c.n_seq && u0 < u1; b0 += 32) {   // the sequence that block u0 / 2 is of
      int q0 = 0, c = 0, len = 0;
      if (b0 + lane < a.c.n_seq) chunk_seq(a, b0 + lane, q0, c, len);
      const int mine = (len + 15) / 16;
      long long inc = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += v;
      }
      const unsigned who = __ballot_sync(0xffffffffu, u0 / 2 < before + inc);
      if (who) {
        if (lane == __ffs(who) - 1) {
          s_seq = b0 + lane;
          s_blk = (int)(u0 / 2 - before - (inc - mine));
          s_len = len;
        }
        break;
      }
      before += __shfl_sync(0xffffffffu, inc, 31);
    }
    if (lane == 0) {
      s_u0 = u0;
      s_u1 = u1;
    }
  }
  __syncthreads();
  int seq = s_seq, b = s_blk, len = s_len;
  const int n = a.c.n_kv_heads * 16 * (DH / 16);
  for (long long u = s_u0; u < s_u1; ++u) {
    const int blk = a.c.table[(size_t)seq * a.c.max_blocks + b], is_v = (int)(u & 1);
    if (blk >= 0 && blk < a.c.n_blocks) {
      const size_t from = (size_t)blk * a.c.n_kv_heads * 16, to = (wide ? (size_t)seq * wide + b : (size_t)blk) * a.c.n_kv_heads * 16;
      const uint8_t* codes = (const uint8_t*)(is_v ? a.c.v : a.c.k) + from * DH;
      const uint8_t* exps = (is_v ? a.c.v_exp : a.c.k_exp) + from;
      bf16* out = (is_v ? v_out : k_out) + to * DH;
#pragma unroll 4
      for (int i = threadIdx.x; i < n; i += CW_THREADS) {
        const uint4 w = reinterpret_cast<const uint4*>(codes)[i];
        const int e = exps[i / (DH / 16)];
        const float s = exp_scale(e);
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
        uint32_t y[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const uint32_t h = e4m3x2_f16x2(x[q >> 1] >> (q & 1 ? 16 : 0));
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
          const __nv_bfloat162 r = __floats2bfloat162_rn(f.x * s, f.y * s);
          y[q] = *reinterpret_cast<const uint32_t*>(&r);
        }
        reinterpret_cast<uint4*>(out)[2 * i] = make_uint4(y[0], y[1], y[2], y[3]);
        reinterpret_cast<uint4*>(out)[2 * i + 1] = make_uint4(y[4], y[5], y[6], y[7]);
      }
    }
    if (is_v && ++b * 16 >= len) {
      b = 0;
      len = 0;
      while (len == 0 && ++seq < a.c.n_seq) {
        int q0, c;
        chunk_seq(a, seq, q0, c, len);
      }
    }
  }
}

// Join of the tiles that runs share: CTA (i, y) takes the tile that run i + 1 is the first to begin inside of, a sixteenth of its
// rows in use (20 rows of 32 heads on 8 over 4096 keys 16.7 us, by eighths and by 32nds 17.7; 256 of 32 heads 34.4, 36.4 and 35.6;
// 512 on 1531, 32 heads on 8, 31.5, 30.9 and 33.1).  Parts: run i's (the tile's beginning), run i + 1's, ... in order.
constexpr int CJ_SPLIT = 16;
template <int DH>
__global__ void __launch_bounds__(256) chunk_tc_join_kernel(const __grid_constant__ CtParams p) {
  PDL_ENTRY();
  const CtWs ws(p);
  const int run = (int)blockIdx.x + 1, tid = threadIdx.x;
  const CtNote n = ws.note[run];
  if (n.u0 < 0 || ws.note[run - 1].u0 == n.u0) return;
  int n_part = 2;
  while (run + n_part - 1 < p.runs && ws.note[run + n_part - 1].u0 == n.u0) ++n_part;
  const ChunkCall& a = p.a;
  const int group = a.n_heads / a.c.n_kv_heads;
  // a warp takes 8 rows x 4 pieces of 4 columns: whole lines of the parts, whole sectors of the output
  const int lane = tid & 31, rl = lane & 7, dl = lane >> 3;
  const int used = p.ts * group, live = n.n_tok * group, n8 = (live + 7) / 8;   // rows of a sub-tile, of the tile, its eights
  for (int w = (int)blockIdx.y * 8 + (tid >> 5); w < n8 * (DH / 16); w += CJ_SPLIT * 8) {
    const int i = w % n8 * 8 + rl, d4 = w / n8 * 4 + dl;   // (a piece of a row's columns, all eights after the other)
    if (i >= live) continue;
    const int sub = i >= used, rr = i - sub * used, r = sub * CT_BM + rr, tok = sub * p.ts + rr / group;
    float M = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < n_part; k0 += 4) {
      float2 ml[4];
      float4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        ml[k] = make_float2(-INFINITY, 0.f);
        v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (k0 + k < n_part) {
          const int slot = (run - 1 + k0 + k) * 2 + (k0 + k == 0);
          ml[k] = __ldcg(ws.ml_at(slot, r));
          v[k] = __ldcg(ws.o_at(slot, DH, d4, r));
        }
      }
      float mn = M;
#pragma unroll
      for (int k = 0; k < 4; ++k) mn = fmaxf(mn, ml[k].x);
      const float ref = mn == -INFINITY ? 0.f : mn, f = ex2_approx(M - ref);
      M = mn;
      l *= f;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] *= f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float x = ex2_approx(ml[k].x - ref);
        l += x * ml[k].y;
        o[0] += x * v[k].x;
        o[1] += x * v[k].y;
        o[2] += x * v[k].z;
        o[3] += x * v[k].w;
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const __nv_bfloat162 y0 = __floats2bfloat162_rn(o[0] * inv, o[1] * inv), y1 = __floats2bfloat162_rn(o[2] * inv, o[3] * inv);
    *reinterpret_cast<uint2*>((bf16*)a.out + (size_t)(n.row0 + tok) * a.ld_out + (size_t)(n.kvh * group + rr % group) * DH + d4 * 4) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&y0), *reinterpret_cast<const uint32_t*>(&y1));
  }
}

}  // namespace
}  // namespace adept
