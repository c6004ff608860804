// A paged K/V cache given by its pointers (adept_kv_cache), and the launchers of the kernels that
// write it (kv_store.cu) and attend over it (attention_chunk.cu, attention_chunk_tc.cu).
#pragma once
#include "common.cuh"

#include <atomic>

namespace adept {

enum KvType : int { KV_F32 = 0, KV_BF16 = 1, KV_E4M3 = 2 };

// K and V as [n_blocks][n_kv_heads][block_tokens][head_dim].  KV_E4M3: one byte per element and, in k_exp / v_exp
// [n_blocks][n_kv_heads][block_tokens], the exponent e (+ 127) of each (position, head): value = code * 2^e.
struct KvPaged {
  void* k;
  void* v;
  uint8_t* k_exp;
  uint8_t* v_exp;
  const int* table;   // [n_seq][max_blocks]
  unsigned* err;      // error word (NULL: none)
  int type, n_blocks, n_kv_heads, head_dim, block_tokens, n_seq, max_blocks;
  __device__ __forceinline__ void flag(unsigned bits) const {
    if (err) atomicOr(err, bits);
  }
};

// Rows of K and V into the cache at (seq[r], pos[r]); seq[r] < 0: the row is left out.  src_bf16: element type of the
// rows (else fp32); ld in elements.
cudaError_t launch_kv_append(cudaStream_t st, const KvPaged& c, int n_rows, int src_bf16, const void* k, long long ld_k,
                             const void* v, long long ld_v, const int* seq, const int* pos);
// The entries at (seq[r], pos[r]) back as rows (a row with seq[r] < 0 is not written); seq NULL: position pos0 + r of seq0.
cudaError_t launch_kv_gather(cudaStream_t st, const KvPaged& c, int n_rows, int dst_bf16, void* k, long long ld_k, void* v,
                             long long ld_v, const int* seq, const int* pos, int seq0 = 0, int pos0 = 0);
// bf16 entries that a pass left in a staging cache (layers src_layer0 ..) into the 8-bit cache c (of the first of n_layers
// layers): rows [0, n_rows[y]) of layer y (NULL: max_rows), row r token row_tok[r] (NULL: r) at (tok_seq, tok_pos).
cudaError_t launch_kv_requant(cudaStream_t st, const KVCacheView& src, int src_layer0, const KvPaged& c, int n_layers,
                              const int* n_rows, int max_rows, const int* row_tok, const int* tok_seq, const int* tok_pos);

// One attention call: the new tokens of n_seq sequences (rows q_start[b] .. q_start[b + 1]) at the last of sequence b's
// kv_len[b] cached positions, or at those that row_pos gives, each attending its own position and those before it.
struct ChunkCall {
  KvPaged c;
  const void* q;      // [n_rows][ld_q], head h at column h * head_dim (bf16; fp32 for an fp32 cache)
  void* out;          // [n_rows][ld_out], the same type
  long long ld_q, ld_out;
  const int* q_start;
  const int* kv_len;
  const int* row_pos;   // position per row, ascending within a sequence (NULL: the last ones)
  int n_rows, n_heads, max_q, max_kv;
  int c_lo, c_hi;     // the launch's sequences: those with c_lo to c_hi new tokens
  int late;           // the launch needs nothing of the one before it: it waits for that at its end, for those behind it
  float scale_log2;   // log2(e) / sqrt(head_dim)
  float* part;        // workspace
};
// Bytes of `part` that a call of these bounds needs; no call of fewer sequences or smaller bounds on the same pool needs more.
size_t chunk_workspace(const KvPaged& c, int n_heads, int max_q, int max_kv);
cudaError_t launch_chunk_attention(cudaStream_t st, const ChunkCall& a, int* launches);
// The tcgen05 kernel (attention_chunk_tc.cu): what it takes (rows on 16 bytes and an sm_100-family GPU besides), its workspace,
// its launches.
bool chunk_tc_takes(const KvPaged& c, int n_heads);
size_t chunk_tc_workspace(const KvPaged& c, int max_kv);
// Whether a call's (tile, KV head, key tile) triples fit 31 bits (hours of work otherwise).
bool chunk_tc_fits(const KvPaged& c, int n_heads, int n_rows, int max_q, int max_kv);
// (the widening of 8-bit entries to bf16 in the workspace, which goes first, is a launch of its own)
cudaError_t launch_chunk_widen(cudaStream_t st, const ChunkCall& a, int* launches);
cudaError_t launch_chunk_tc(cudaStream_t st, const ChunkCall& a, int* launches);
cudaError_t set_wait_limit_ct(long long cycles);
cudaError_t set_wait_limit_cf(long long cycles);

// ---------------------------------------------------------------------------------------------
// Work split.  A tile is up to tq new tokens of one sequence (all query heads of a group of one KV head); its keys are
// taken in units of `unit`.  A call with fewer tiles than the GPU holds CTAs (`target`) splits each sequence's keys into equal
// runs so that at most `target` items exist; an item of a split tile leaves a partial (maximum, sum, weighted V) in slot
// `item` of the workspace, joined in split order by a second launch.  The split follows from the device's lengths, so a
// captured launch stays balanced when they change.
// ---------------------------------------------------------------------------------------------
struct SplitPlan {
  int tq, groups, unit, target;   // tokens per tile; head groups; keys per unit; items aimed at
};
struct SplitItem {
  int seq, q0, c, len;        // sequence, its first row, new tokens, cached positions
  int tile, group;            // token tile, head group
  int split, n_split;         // this item's run of keys, and how many
  int units, u0, u1;          // the sequence's units of keys; this item's
  int slot0;                  // slot of the tile's first split
};

// Lengths of sequence b, or no work (c = 0) where they are out of bounds or not this launch's.
__device__ __forceinline__ void chunk_seq(const ChunkCall& a, int b, int& q0, int& c, int& len) {
  q0 = __ldcg(a.q_start + b);   // (past L1: a join reads them before its dependency wait)
  c = __ldcg(a.q_start + b + 1) - q0;
  len = __ldcg(a.kv_len + b);
  const int cap = min(a.max_kv, a.c.max_blocks * a.c.block_tokens);
  if (q0 < 0 || c < 0 || c > a.max_q || q0 > a.n_rows - c || len < 0 || len > cap) {
    a.c.flag(ERRW_POS);
    c = 0;
  }
  if (c < a.c_lo || c > a.c_hi) c = 0;
  if (c == 0) len = 0;
}

// Keys that new token j of a sequence attends.
__device__ __forceinline__ int chunk_lim(const ChunkCall& a, int q0, int c, int len, int j) {
  return a.row_pos ? min(max(a.row_pos[q0 + j], -1), len - 1) + 1 : max(len - c + j + 1, 0);
}

// Item `id` of the plan (joined: tile `id`, its splits taken together), looked up by one converged warp; false: none.  32-bit
// sums by one instruction each: in 64 bits, with shuffles, the look-up took 4000 cycles of a call of 15000.
__device__ __forceinline__ bool split_find(const ChunkCall& a, const SplitPlan& p, int id, bool joined, SplitItem& it) {
  const int lane = threadIdx.x & 31, n_seq = a.c.n_seq;
  unsigned base = 0, tot = 0;
  bool huge = false;   // more units than the sum holds: no split
  int q0 = 0, c = 0, len = 0;
  for (int b0 = 0; b0 < n_seq; b0 += 32) {
    const int b = b0 + lane;
    q0 = c = len = 0;
    if (b < n_seq) chunk_seq(a, b, q0, c, len);
    const unsigned t = (unsigned)((c + p.tq - 1) / p.tq) * p.groups;
    const unsigned long long w = (unsigned long long)t * ((len + p.unit - 1) / p.unit);
    base += t;
    huge |= w + tot >= 1u << 26;
    tot += (unsigned)w;
  }
  base = __reduce_add_sync(0xffffffffu, min(base, 1u << 26));
  tot = __reduce_add_sync(0xffffffffu, tot);
  huge = __any_sync(0xffffffffu, huge) != 0;
  // run length S: sum over tiles of ceil(units / S) <= tot / S + base <= target
  unsigned S = 1u << 30;
  const unsigned target = (unsigned)p.target;
  if (base < target && !huge) S = max(1u, (tot + (target - base) - 1) / (target - base));
  int before = 0, slots = 0;   // of the sequences before these 32
  for (int b0 = 0; b0 < n_seq; b0 += 32) {
    const int b = b0 + lane;
    if (n_seq > 32) {
      q0 = c = len = 0;
      if (b < n_seq) chunk_seq(a, b, q0, c, len);
    }
    const int tiles = (c + p.tq - 1) / p.tq, units = (len + p.unit - 1) / p.unit;
    const int ns = max((int)(((unsigned)units + S - 1) / S), 1);
    const int n_it = tiles * p.groups * ns, mine = joined ? tiles * p.groups : n_it;
    int inc = mine, sl = n_it;
    if (n_seq > 1) {
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, inc, o), w = __shfl_up_sync(0xffffffffu, sl, o);
        if (lane >= o) {
          inc += u;
          sl += w;
        }
      }
    }
    const int lo = before + inc - mine;
    const unsigned who = __ballot_sync(0xffffffffu, id >= lo && id < lo + mine);
    if (who) {
      const int src = __ffs(who) - 1;
      const int s0 = __shfl_sync(0xffffffffu, slots + sl - n_it, src);
      int r = id - __shfl_sync(0xffffffffu, lo, src);
      it.seq = b0 + src;
      it.q0 = __shfl_sync(0xffffffffu, q0, src);
      it.c = __shfl_sync(0xffffffffu, c, src);
      it.len = __shfl_sync(0xffffffffu, len, src);
      it.n_split = __shfl_sync(0xffffffffu, ns, src);
      const int un = __shfl_sync(0xffffffffu, units, src), nt = __shfl_sync(0xffffffffu, tiles, src);
      it.units = un;
      it.split = 0;
      if (!joined) {
        const int k = r / it.n_split;
        it.split = r - k * it.n_split;
        r = k;
      }
      // the last tiles (the longest) come first, all head groups of one together
      const int back = r / p.groups;
      it.group = r - back * p.groups;
      it.tile = nt - 1 - back;
      it.slot0 = s0 + r * it.n_split;
      const int per = (un + it.n_split - 1) / it.n_split;
      it.u0 = min(un, it.split * per);
      it.u1 = min(un, it.u0 + per);
      return true;
    }
    before += __shfl_sync(0xffffffffu, inc, n_seq > 1 ? 31 : 0);
    slots += __shfl_sync(0xffffffffu, sl, n_seq > 1 ? 31 : 0);
  }
  return false;
}
// Two e4m3 codes (low 16 bits) as two fp16: exact, NaN stays NaN.  (One instruction; through the toolkit's half2 type the few-row
// kernel took 62.6 us where it took 55.5.)
__device__ __forceinline__ uint32_t e4m3x2_f16x2(uint32_t codes) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)codes));
  return h;
}
// The scale of an exponent byte, 2^(b - 127) (b = 0: the subnormal 2^-127).
__device__ __forceinline__ float exp_scale(int b) { return __uint_as_float(max((unsigned)b << 23, 0x400000u)); }

// Sets a kernel's dynamic shared memory, once per device (Tag: a type of the kernel's own).
template <typename Tag, typename K>
inline cudaError_t smem_once(K* kernel, int bytes) {
  static std::atomic<unsigned long long> done{0};   // bit per device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
  if (bit && (done.load() & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit);
  return e;
}

// Items there can be at most: the target, or one per tile where there are more tiles.
static inline long long split_items(const SplitPlan& p, int n_seq, int n_rows, int max_q) {
  const long long by_seq = (long long)n_seq * (((long long)max_q + p.tq - 1) / p.tq);   // (max_q may be any bound)
  const long long by_rows = n_rows / p.tq + (long long)n_seq;
  const long long tiles = (by_seq < by_rows ? by_seq : by_rows) * p.groups;
  return tiles > p.target ? tiles : p.target;
}

}  // namespace adept
