// Attention of a chunk of new tokens over a paged K/V cache: sequence b brings c_b >= 0 new tokens, the last of its kv_len_b
// cached positions (or given ones of them); the token at position p attends positions 0..p.
//
//   out = sum_k exp(s_k - m) v_k / sum_k exp(s_k - m),   s_k = q . k_k / sqrt(head_dim),   m = max s_k
//
// in one pass over the keys with the running maximum and sum (fp32, exponentials in base 2).  A row that no key gives any weight
// (a chunk longer than kv_len, no block there, all scores -infinity) gives zeros: its sum is zero, as no other row's is (the
// score that last raised the maximum has weight 1, a NaN score gives a sum of NaN).  What lies behind a token's position is never
// used: neither scores nor V entries of masked positions enter a sum, so NaN or infinities there do not spread.  Keys in blocks
// that the table does not hold (negative, out of range) are left out and flagged.
//
// The split of the work, and the join of split tiles, are in kv_paged.h.
#define ADEPT_TU_ID 14
#include "gemm_tc.h"
#include "kv_paged.h"
#include "tc_ptx.cuh"

#include <cuda_fp8.h>

#include <algorithm>

namespace adept {
namespace {

// ---------------------------------------------------------------------------------------------
// Any type, head size, alignment and block size: CUDA-core kernel.  CTA = up to CG_ROWS new tokens of one query head x a
// run of keys, 128 keys at a time: a thread per key for the scores, a warp per token for the softmax, for the weighted sum a
// thread per four dimensions of every KG-th key.  Such calls are short and bound by latency, one load behind the other, so
// all loads are of four elements, several under way: fp32, 22 rows of 4 heads of 64 over up to 101 keys in 8.2 us (17.8 with
// one element a load, two key groups); 512 rows of 12 heads over 2560 keys in 369 us (9.8 TFLOP/s, each tile of 4 rows reading
// K and V from L2 again).
// ---------------------------------------------------------------------------------------------
constexpr int CG_ROWS = 4, CG_KEYS = 128;

// Elements i .. i + 3 of K or V as fp32; e4m3 codes without their exponent.
template <int KT>
__device__ __forceinline__ float4 kv_four(const void* p, size_t i) {
  if constexpr (KT == KV_F32) {
    return *reinterpret_cast<const float4*>((const float*)p + i);
  } else if constexpr (KT == KV_BF16) {
    const uint2 w = *reinterpret_cast<const uint2*>((const bf16*)p + i);
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                       __uint_as_float(w.y & 0xffff0000u));
  } else {
    const uint32_t w = *reinterpret_cast<const uint32_t*>((const uint8_t*)p + i), h0 = e4m3x2_f16x2(w), h1 = e4m3x2_f16x2(w >> 16);
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&h0)), y = __half22float2(*reinterpret_cast<const __half2*>(&h1));
    return make_float4(x.x, x.y, y.x, y.y);
  }
}
// Part buffers of slot s: `rows` rows of (m, l) at part, of DH sums behind all the (m, l).
struct PartView {
  float* ml;
  float* o;
  __device__ PartView(const ChunkCall& a, const SplitPlan& p, int rows, int dh, int slot)
      : ml(a.part + (size_t)slot * rows * 2), o(a.part + (size_t)p.target * rows * 2 + (size_t)slot * rows * dh) {}
};

template <int DH, int KT, typename T>
__global__ void __launch_bounds__(CG_KEYS) chunk_any_kernel(const __grid_constant__ ChunkCall a, const __grid_constant__ SplitPlan p) {
  __shared__ SplitItem s_it;
  __shared__ int s_have;
  constexpr int QD = DH / 4, KG = CG_KEYS / QD;   // fours of dimensions; key groups of the weighted sum
  __shared__ __align__(16) float s_q[CG_ROWS][DH];
  __shared__ float s_p[CG_ROWS][CG_KEYS];
  __shared__ long long s_e[CG_KEYS];
  __shared__ float s_vs[CG_KEYS], s_corr[CG_ROWS];
  __shared__ __align__(16) float s_red[KG][CG_ROWS][DH];
  PDL_ENTRY();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (warp == 0) {
    SplitItem it;
    const bool have = split_find(a, p, (int)blockIdx.x, false, it);
    if (lane == 0) {
      s_it = it;
      s_have = have;
    }
  }
  __syncthreads();
  if (!s_have) return;
  const SplitItem it = s_it;
  const int h = it.group, kvh = h / (a.n_heads / a.c.n_kv_heads), bt = a.c.block_tokens;
  const int j0 = it.tile * CG_ROWS, n = min(CG_ROWS, it.c - j0);
  int lim[CG_ROWS];   // keys that each row attends
#pragma unroll
  for (int r = 0; r < CG_ROWS; ++r) lim[r] = r < n ? chunk_lim(a, it.q0, it.c, it.len, j0 + r) : 0;
  for (int i = tid; i < n * DH; i += CG_KEYS)
    s_q[i / DH][i % DH] = to_f<T>(((const T*)a.q)[(size_t)(it.q0 + j0 + i / DH) * a.ld_q + (size_t)h * DH + i % DH]);
  const int k_end = min(it.u1 * CG_KEYS, max(max(lim[0], lim[1]), max(lim[2], lim[3])));
  const int d = tid % QD * 4, kg = tid / QD;
  float acc[CG_ROWS][4], m = -INFINITY, l = 0.f;   // (m, l of row `warp`)
#pragma unroll
  for (int r = 0; r < CG_ROWS; ++r) acc[r][0] = acc[r][1] = acc[r][2] = acc[r][3] = 0.f;
  for (int k0 = it.u0 * CG_KEYS; k0 < k_end; k0 += CG_KEYS) {
    const int key = k0 + tid;
    long long e = -1;
    float ks = 1.f;
    if (key < k_end) {
      const int blk = a.c.table[(size_t)it.seq * a.c.max_blocks + key / bt];
      if (blk >= 0 && blk < a.c.n_blocks)
        e = ((long long)blk * a.c.n_kv_heads + kvh) * bt + key % bt;
      else
        a.c.flag(ERRW_POS);
    }
    if (KT == KV_E4M3) {
      if (e >= 0) ks = exp_scale(a.c.k_exp[e]);
      s_vs[tid] = e >= 0 ? exp_scale(a.c.v_exp[e]) : 0.f;
    }
    s_e[tid] = e;
    __syncthreads();   // (and s_q; s_p and s_corr of the previous round are read)
    float dot[CG_ROWS];
#pragma unroll
    for (int r = 0; r < CG_ROWS; ++r) dot[r] = 0.f;
    if (e >= 0) {
#pragma unroll 8
      for (int i = 0; i < DH; i += 4) {
        const float4 x = kv_four<KT>(a.c.k, (size_t)e * DH + i);
#pragma unroll
        for (int r = 0; r < CG_ROWS; ++r) {
          const float4 q = *reinterpret_cast<const float4*>(&s_q[r][i]);
          dot[r] = fmaf(x.w, q.w, fmaf(x.z, q.z, fmaf(x.y, q.y, fmaf(x.x, q.x, dot[r]))));
        }
      }
    }
#pragma unroll
    for (int r = 0; r < CG_ROWS; ++r)
      s_p[r][tid] = e >= 0 && key < lim[r] ? dot[r] * ks * a.scale_log2 : -INFINITY;
    __syncthreads();
    {
      float v[CG_KEYS / 32], mx = m;
#pragma unroll
      for (int i = 0; i < CG_KEYS / 32; ++i) {
        v[i] = s_p[warp][i * 32 + lane];
        mx = fmaxf(mx, v[i]);
      }
      mx = warp_max(mx);
      const float ref = mx == -INFINITY ? 0.f : mx, corr = exp2f(m - ref);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < CG_KEYS / 32; ++i) {
        const float w = exp2f(v[i] - ref);
        s_p[warp][i * 32 + lane] = w;
        sum += w;
      }
      l = l * corr + warp_sum(sum);
      m = mx;
      if (lane == 0) s_corr[warp] = corr;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < CG_ROWS; ++r)
#pragma unroll
      for (int x = 0; x < 4; ++x) acc[r][x] *= s_corr[r];
    const int nk = min(CG_KEYS, k_end - k0);
    for (int k1 = kg; k1 < nk; k1 += 4 * KG) {
      float4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = k1 + j * KG;
        const long long ev = k < nk ? s_e[k] : -1;
        v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (ev >= 0) v[j] = kv_four<KT>(a.c.v, (size_t)ev * DH + d);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = k1 + j * KG;
        if (k >= nk) break;
#pragma unroll
        for (int r = 0; r < CG_ROWS; ++r) {
          if (k0 + k >= lim[r]) continue;   // (0 times what a masked entry holds might be NaN)
          const float w = s_p[r][k], vs = KT == KV_E4M3 ? s_vs[k] : 1.f;   // (no entry: 0 times 0)
          acc[r][0] = fmaf(w, v[j].x * vs, acc[r][0]);
          acc[r][1] = fmaf(w, v[j].y * vs, acc[r][1]);
          acc[r][2] = fmaf(w, v[j].z * vs, acc[r][2]);
          acc[r][3] = fmaf(w, v[j].w * vs, acc[r][3]);
        }
      }
    }
    __syncthreads();
  }
  const PartView pv(a, p, CG_ROWS, DH, it.slot0 + it.split);
  if (lane == 0) s_corr[warp] = l;
  if (it.n_split > 1 && lane == 0 && warp < n) {
    pv.ml[warp * 2] = m;
    pv.ml[warp * 2 + 1] = l;
  }
#pragma unroll
  for (int r = 0; r < CG_ROWS; ++r)
    *reinterpret_cast<float4*>(&s_red[kg][r][d]) = make_float4(acc[r][0], acc[r][1], acc[r][2], acc[r][3]);
  __syncthreads();
  for (int i = tid; i < n * DH; i += CG_KEYS) {
    const int r = i / DH, x = i % DH;
    float o = 0.f;
#pragma unroll
    for (int g = 0; g < KG; ++g) o += s_red[g][r][x];
    if (it.n_split > 1)
      pv.o[r * DH + x] = o;
    else
      ((T*)a.out)[(size_t)(it.q0 + j0 + r) * a.ld_out + (size_t)h * DH + x] =
          from_f<T>(s_corr[r] == 0.f ? 0.f : o / s_corr[r]);
  }
}

// ---------------------------------------------------------------------------------------------
// bf16 queries over bf16 or e4m3 entries in blocks of 16 positions: warp-level matrix instructions (m16n8k16), for the calls
// that are a stream of K and V (steps, checks of a few tokens).  CTA = a tile of ROWS rows (token x query head of the KV
// head's group) x a run of keys, CF_WARPS warps taking blocks in turn, each with a softmax and sums of its own, merged in
// warp order at the end.
//
// A head's 16 positions of a block are one contiguous piece of the pool: each warp keeps STAGES of them (K, V, exponents)
// under way by bulk copies into a ring of its own, so no warp waits for another, and no register holds what is under way.
// From the ring the words go straight into fragments: the order of the head's dimensions inside q.k is free, so a thread's
// B fragments of S = Q K^T are whole 16-byte pieces of its key's row (Q is loaded in the same order), and the columns of O are
// dealt out so that a thread's B fragments of O = P V are 16-byte pieces of four keys' rows, pairs of keys packed by byte
// permutes.  (V lies in four groups 32 bytes apart: in one piece the rows that neighbours read lay under each other, 4 wavefronts
// where one is enough.)
// e4m3: K as fp16, one conversion for two codes (bf16 takes four instructions), with Q as fp16 too, each row moved by a power
// of two so that its largest element lies in [2^14, 2^15): exact down to 2^-28 of it.  V as bf16, since P has to keep bf16's
// range (a position of little weight may hold a V of any size).  K's exponent scales S, V's scales P.
//
// A tile's keys are split over CTAs even where they are few (12 heads of 64, 333 keys: 7.2 us split and joined, 7.7 by 12 CTAs;
// 1000 keys 7.6 and 14.5), in one of two ways.  Where a cluster of up to 8 CTAs a tile is enough (cs > 1), its CTAs take
// equal shares and join through distributed shared memory, in one launch.  Else each tile gets as many as balance the GPU
// (split_find), whose partials a second launch joins.
//
// ROWS = 8: where no tile has more than 8 rows the keys are the 16 rows of the matrix instructions and the queries their 8
// columns (S^T = K Q^T, O^T = V^T P^T), which halves them and the softmax; the same words of K and V in the same registers, P's
// fragments turned round in between.  Against 16 rows: 8 bits, a token of 32 heads of 128 over 30011 keys 45.6 us for 53.2, 16
// sequences of a token, 32 heads on 8, 21.0 for 24.2; bf16, a token of 32 heads over 2000 keys 11.3 for 12.1, 8 sequences over up to
// 4000 56.9 for 57.8.
//
// P is rounded to bf16 (2^-8 relative at most) because the matrix instruction takes 16 bits of it and of V; the sums l take the
// weights as they are, in fp32.  Against 64 bits an output is off by 2.3e-3 of its size (rms) where the rounding of the output alone
// gives 1.7e-3.
//
// Measured: that token over 30011 keys, 8 bits (248 MB) 45.6 us, 5.4 TB/s, bound by instruction issue and latency (12 warps an SM,
// each waiting on its own conversions and reads); 8 sequences over up to 4000 keys in bf16 (295 MB) 56.9 us, 5.2 TB/s; 4 to 5
// tokens of 4 sequences over 8.4 thousand keys, bf16 (139 MB), 30.9 us, 8 of them launches and the join.
// ---------------------------------------------------------------------------------------------
constexpr int CF_WARPS = 4, CF_ROWS = 16;
constexpr float CF_RAISE = 8.f;   // the running maximum is raised once a score exceeds it by 2^8: weights stay below 256
constexpr long long CF_DRAIN_CYCLES = 4000000000LL;

template <int BYTES>
struct Words {
  uint32_t w[BYTES / 4];
};
template <int BYTES>
__device__ __forceinline__ Words<BYTES> lds(const void* p) {
  Words<BYTES> r;
  if constexpr (BYTES == 16) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    r.w[0] = x.x; r.w[1] = x.y; r.w[2] = x.z; r.w[3] = x.w;
  } else if constexpr (BYTES == 8) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    r.w[0] = x.x; r.w[1] = x.y;
  } else {
    r.w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
  return r;
}
template <bool F16>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (F16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The transpose of an 8 x 8 matrix of 16-bit elements over the warp (lane: row lane / 4, columns 2 (lane % 4) and the next).
__device__ __forceinline__ uint32_t turn8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&x);
}
// Two e4m3 codes (low 16 bits) as two bf16: exact, NaN stays NaN.
__device__ __forceinline__ uint32_t e4m3x2_bf16x2(uint32_t codes) {
  const uint32_t h = e4m3x2_f16x2(codes);
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  return pack_bf16(f.x, f.y);
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The value at `p` in the shared memory of the cluster's CTA `rank`.
__device__ __forceinline__ uint32_t cluster_addr(const void* p, int rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ float ld_cluster(const float* p, int rank) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_addr(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ float4 ld_cluster4(const float* p, int rank) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(cluster_addr(p, rank)) : "memory");
  return v;
}
// A bounded wait of the whole warp for a stage; false: it did not land in time, or another warp gave up.
__device__ __forceinline__ bool cf_wait(uint64_t* bar, unsigned parity, volatile int* abort_flag, unsigned* err, long long lim) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity)) {
    if (*abort_flag) return false;
    if (clock64() - t0 > lim) {
      if (err) atomicOr(err, ERRW_TIMEOUT);
      return false;
    }
  }
  return true;
}
// Words of four keys' rows (0, 1 and 8, 9 of a fragment) to B fragments: f(column of the word, b0, b1), all bf16.
template <int KT, typename F>
__device__ __forceinline__ void cf_pairs(uint32_t k0, uint32_t k1, uint32_t k2, uint32_t k3, F f) {
  if constexpr (KT == KV_BF16) {
    f(0, __byte_perm(k0, k1, 0x5410), __byte_perm(k2, k3, 0x5410));
    f(1, __byte_perm(k0, k1, 0x7632), __byte_perm(k2, k3, 0x7632));
  } else {
    const uint32_t x0 = __byte_perm(k0, k1, 0x5140), x1 = __byte_perm(k2, k3, 0x5140);
    const uint32_t y0 = __byte_perm(k0, k1, 0x7362), y1 = __byte_perm(k2, k3, 0x7362);
    f(0, e4m3x2_bf16x2(x0 & 0xffffu), e4m3x2_bf16x2(x1 & 0xffffu));
    f(1, e4m3x2_bf16x2(x0 >> 16), e4m3x2_bf16x2(x1 >> 16));
    f(2, e4m3x2_bf16x2(y0 & 0xffffu), e4m3x2_bf16x2(y1 & 0xffffu));
    f(3, e4m3x2_bf16x2(y0 >> 16), e4m3x2_bf16x2(y1 >> 16));
  }
}

template <int DH, int KT, int ROWS>
struct FewShape {
  static constexpr int ES = KT == KV_BF16 ? 2 : 1;
  static constexpr int NB = KT == KV_BF16 ? 1 : 2;         // blocks of 16 keys per warp and round
  static constexpr int STAGES = 2 * NB;                    // blocks in a warp's ring
  static constexpr int UNIT = CF_WARPS * NB * 16;
  static constexpr int KVEC = DH * ES / 4 < 16 ? DH * ES / 4 : 16, KN = DH * ES / 4 / KVEC, KE = KVEC / ES;   // K pieces of a thread
  static constexpr int VVEC = DH * ES / 8 < 16 ? DH * ES / 8 : 16, VN = DH * ES / 8 / VVEC, VE = VVEC / ES;   // V pieces
  static constexpr int BLOCK = 16 * DH * ES;               // bytes of a block of one head
  // V in groups of 4 keys, 32 bytes apart: the four keys' rows that neighbours read lie under different banks
  static constexpr int GROUP = BLOCK / 4 + 32, EXPS = BLOCK + 4 * GROUP;
  static constexpr int BYTES = 2 * BLOCK + (KT == KV_E4M3 ? 32 : 0);   // of a stage: K, V, exponents
  static constexpr int STAGE = EXPS + (KT == KV_E4M3 ? 32 : 0);
  static constexpr int RING = CF_WARPS * STAGES * STAGE, MERGE = CF_WARPS * ROWS * (DH + 4) * 4;
  static constexpr int SMEM = RING > MERGE ? RING : MERGE;
};

template <int DH, int KT, int ROWS>
__global__ void __launch_bounds__(CF_WARPS * 32, 3) chunk_few_kernel(const __grid_constant__ ChunkCall a,
                                                                     const __grid_constant__ SplitPlan p, int per_tok, int sub,
                                                                     int cs) {
  using F = FewShape<DH, KT, ROWS>;
  constexpr bool W8 = ROWS == 8;
  constexpr int KS = DH / 16, NS = F::NB * (W8 ? 1 : 2), NO = DH / (W8 ? 16 : 8);   // k-steps; fragments of S in a round, of O
  auto rh = [](int e) { return W8 ? e & 1 : e >> 1; };   // which of the thread's two rows element e of a fragment is of
  constexpr bool F16 = KT == KV_E4M3;   // S in fp16
  __shared__ SplitItem s_it;
  __shared__ int s_have, s_abort;
  __shared__ float s_m[CF_WARPS][ROWS], s_l[CF_WARPS][ROWS];
  __shared__ float s_cm[ROWS], s_cl[ROWS];   // of the CTA, for its cluster
  __shared__ __align__(8) uint64_t s_full[CF_WARPS][F::STAGES];
  extern __shared__ __align__(128) uint8_t s_dyn[];   // the rings; then [warp][row][DH + 4] floats
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  if (tid < CF_WARPS * F::STAGES) {
    mbar_init(&s_full[tid / F::STAGES][tid % F::STAGES], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid == 0) s_abort = 0;
  const long long wlim = wait_limit();
  KT_BEGIN();
  if (!a.late) pdl_wait();
  KT_WAITED();
  pdl_launch_dependents();
  const int rank = cs > 1 ? (int)blockIdx.x % cs : 0;
  if (warp == 0) {
    SplitItem it;
    const bool have = split_find(a, p, (int)blockIdx.x / cs, cs > 1, it);
    if (cs > 1 && have) {
      const int per = (it.units + cs - 1) / cs;
      it.split = rank;
      it.n_split = cs;
      it.u0 = min(it.units, rank * per);
      it.u1 = min(it.units, it.u0 + per);
    }
    if (lane == 0) {
      s_it = it;
      s_have = have;
    }
  }
  __syncthreads();
  if (!s_have) {   // (all CTAs of a cluster)
    if (a.late) pdl_wait();
    return;
  }
  const SplitItem it = s_it;
  const int group = a.n_heads / a.c.n_kv_heads, kvh = it.group / sub, g0 = it.group % sub * per_tok;
  const int j0 = it.tile * p.tq, n = min(p.tq, it.c - j0);
  const int n_row = n * per_tok;   // rows of the tile in use (those with g0 + r % per_tok >= group hold nothing)
  auto keys_of = [&](int j) { return chunk_lim(a, it.q0, it.c, it.len, j0 + j); };
  const int lim_lo = keys_of(0), lim_hi = keys_of(n - 1);                     // keys of the tile's first and last token
  const int k_end = min(min(it.u1 * F::UNIT, it.len), lim_hi);                // keys that anyone attends
  const int b_end = (k_end + 15) >> 4;
  const int* table = a.c.table + (size_t)it.seq * a.c.max_blocks;
  unsigned* err = a.c.err;

  // ---- the warp's ring: its blocks in order, NB of them a round
  constexpr int STEP = CF_WARPS * F::NB;
  const int first = it.u0 * (F::UNIT / 16) + warp * F::NB;
  uint8_t* ring = s_dyn + warp * F::STAGES * F::STAGE;
  // table entries of the warp's next 32 blocks, a lane each (block i of the warp: first + i / NB * STEP + i % NB)
  int tab = -1, sent = 0, landed = 0;
  unsigned there = 0;   // bit i % 32: block i is there (what is sent and not yet used: at most STAGES)
  auto send = [&]() {   // block `sent` of the warp into its stage
    const int i = sent;
    if (i % 32 == 0) {
      const int b = first + (i + lane) / F::NB * STEP + (i + lane) % F::NB;
      tab = -1;
      if (b < b_end) {
        tab = table[b];
        if (tab < 0 || tab >= a.c.n_blocks) {
          a.c.flag(ERRW_POS);
          tab = -1;
        }
      }
    }
    const int blk = __shfl_sync(0xffffffffu, tab, i % 32);
    there = blk >= 0 ? there | 1u << (i % 32) : there & ~(1u << (i % 32));
    if (blk >= 0 && elect_one()) {
      uint8_t* st = ring + i % F::STAGES * F::STAGE;
      uint64_t* bar = &s_full[warp][i % F::STAGES];
      const size_t e = ((size_t)blk * a.c.n_kv_heads + kvh) * 16;
      mbar_expect_tx(bar, F::BYTES);
      bulk_load(st, (const uint8_t*)a.c.k + e * (DH * F::ES), F::BLOCK, bar);
#pragma unroll
      for (int q = 0; q < 4; ++q)
        bulk_load(st + F::BLOCK + q * F::GROUP, (const uint8_t*)a.c.v + e * (DH * F::ES) + q * (F::BLOCK / 4), F::BLOCK / 4, bar);
      if constexpr (KT == KV_E4M3) {
        bulk_load(st + F::EXPS, a.c.k_exp + e, 16, bar);
        bulk_load(st + F::EXPS + 16, a.c.v_exp + e, 16, bar);
      }
    }
    __syncwarp();
    ++sent;
  };
  // ---- Q fragments of rows g (and g + 8); the keys that this thread's two rows of S attend: g and g + 8, or 2 t and 2 t + 1
  uint32_t qf[KS][W8 ? 2 : 4];
  int lim[2];
  float rs[2];   // what a row's S is multiplied by
#pragma unroll
  for (int r2 = 0; r2 < 2; ++r2) {
    const int r = W8 ? 2 * t + r2 : g + 8 * r2;
    lim[r2] = r < n_row && g0 + r % per_tok < group ? keys_of(r / per_tok) : 0;
    rs[r2] = a.scale_log2;
  }
#pragma unroll
  for (int r2 = 0; r2 < ROWS / 8; ++r2) {
    const int r = g + 8 * r2, j = r / per_tok, gq = g0 + r % per_tok;
    const bool on = r < n_row && gq < group;
    const bf16* q = (const bf16*)a.q + (size_t)(it.q0 + j0 + j) * a.ld_q + (size_t)(kvh * group + gq) * DH;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      constexpr int SP = F::KE / 4;   // k-steps of a piece
      const int dim = (s / SP * 4 + t) * F::KE + s % SP * 4;
      uint2 x = make_uint2(0, 0);
      if (on) x = *reinterpret_cast<const uint2*>(q + dim);
      qf[s][r2] = x.x;
      qf[s][ROWS / 8 + r2] = x.y;
    }
  }
  // blocks of this warp (whole rounds; those past b_end are not there)
  const int n_blk = first < b_end ? (b_end - first + STEP - 1) / STEP * F::NB : 0;
  for (int i = 0; i < F::STAGES && i < n_blk; ++i) send();

  if constexpr (F16) {
#pragma unroll
    for (int r2 = 0; r2 < ROWS / 8; ++r2) {
      unsigned top = 0;   // exponent field of the row's largest finite element
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t w = qf[s][r2 + ROWS / 8 * h];
          const unsigned lo = (w >> 7) & 0xffu, hi = (w >> 23) & 0xffu;
          top = max(top, max(lo == 255u ? 0u : lo, hi == 255u ? 0u : hi));
        }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int e = max((int)top, 15);                                      // (rows below 2^-112 keep fewer bits)
      const float up = __uint_as_float((unsigned)(127 + 14 + 127 - e) << 23);   // 2^(14 - (e - 127))
      rs[r2] = a.scale_log2 * __uint_as_float((unsigned)(e - 14) << 23);   // 2^((e - 127) - 14)
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t& w = qf[s][r2 + ROWS / 8 * h];
          const __half2 y = __floats2half2_rn(__uint_as_float(w << 16) * up, __uint_as_float(w & 0xffff0000u) * up);
          w = *reinterpret_cast<const uint32_t*>(&y);
        }
    }
    if constexpr (W8) {   // from the lanes that hold rows 2 t and 2 t + 1 of Q
      const float of_g = rs[0];
      rs[0] = __shfl_sync(0xffffffffu, of_g, 8 * t);
      rs[1] = __shfl_sync(0xffffffffu, of_g, 8 * t + 4);
    }
  }

  // Which key of a block is which index of the matrix instructions is free, too: 4 q .. 4 q + 3 are 2 q, 2 q + 1, 8 + 2 q and
  // 9 + 2 q, so that a thread's V rows are one group
  const int key_g = 4 * (g >> 1) + (g & 1);   // index g; key_g + 2: index 8 + g
  float o[NO][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int j = 0; j < NO; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;

  bool ok = true;
  unsigned cf_phase = 0;   // bit s: parity of stage s's next copy
  for (int i0 = 0; i0 < n_blk; i0 += F::NB) {
    const int b = first + i0 / F::NB * STEP;
    bool here[F::NB], edge = false;   // edge: some key of the round is not everyone's
    const uint8_t* st[F::NB];
#pragma unroll
    for (int i = 0; i < F::NB; ++i) {
      const int x = i0 + i, sg = x % F::STAGES;
      here[i] = there >> (x % 32) & 1;
      edge |= !here[i];
      st[i] = ring + sg * F::STAGE;
      if (here[i] && ok && (ok = cf_wait(&s_full[warp][sg], cf_phase >> sg & 1u, &s_abort, err, wlim))) cf_phase ^= 1u << sg;
      landed += ok;
    }
    if (!__all_sync(0xffffffffu, ok)) {
      ok = false;
      break;
    }
    edge |= (b + F::NB) * 16 > lim_lo || (b + F::NB) * 16 > k_end;
    // S = Q K^T (W8: its transpose, K Q^T)
    float s[NS][4];
#pragma unroll
    for (int i = 0; i < F::NB; ++i) {
      Words<F::KVEC> k[2][F::KN];   // of keys key_g and key_g + 2
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int c = 0; c < F::KN; ++c) k[nt][c] = lds<F::KVEC>(st[i] + (key_g + 2 * nt) * (DH * F::ES) + (c * 4 + t) * F::KVEC);
#pragma unroll
      for (int nt = 0; nt < (W8 ? 1 : 2); ++nt) {
        float(&d)[4] = s[W8 ? i : 2 * i + nt];
        d[0] = d[1] = d[2] = d[3] = 0.f;
#pragma unroll
        for (int c = 0; c < F::KN; ++c)
#pragma unroll
          for (int w = 0; w < F::KE / 4; ++w) {
            const int ks = c * (F::KE / 4) + w;
            auto lo = [&](int n) { return KT == KV_BF16 ? k[n][c].w[2 * w] : e4m3x2_f16x2(k[n][c].w[w] & 0xffffu); };
            auto hi = [&](int n) { return KT == KV_BF16 ? k[n][c].w[2 * w + 1] : e4m3x2_f16x2(k[n][c].w[w] >> 16); };
            if constexpr (W8) {
              const uint32_t kf[4] = {lo(0), lo(1), hi(0), hi(1)};
              mma16816<F16>(d, kf, qf[ks][0], qf[ks][1]);
            } else {
              mma16816<F16>(d, qf[ks], lo(nt), hi(nt));
            }
          }
        if constexpr (KT == KV_E4M3 && W8) {
          const float e0 = exp_scale(st[i][F::EXPS + key_g]), e1 = exp_scale(st[i][F::EXPS + key_g + 2]);
          d[0] *= e0 * rs[0]; d[1] *= e0 * rs[1]; d[2] *= e1 * rs[0]; d[3] *= e1 * rs[1];
        } else if constexpr (KT == KV_E4M3) {
          const uint32_t e = *reinterpret_cast<const uint16_t*>(st[i] + F::EXPS + 4 * t + 2 * nt);
          const float e0 = exp_scale(e & 0xff), e1 = exp_scale(e >> 8);
          d[0] *= e0 * rs[0]; d[1] *= e1 * rs[0]; d[2] *= e0 * rs[1]; d[3] *= e1 * rs[1];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) d[e] *= rs[0];
        }
      }
    }
    unsigned att = ~0u;   // bit (fragment, element): the row attends the key
    if (edge) {
      att = 0;
#pragma unroll
      for (int x = 0; x < NS; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = b * 16 + (W8 ? x * 16 + key_g + 2 * (e >> 1) : (x >> 1) * 16 + 4 * t + 2 * (x & 1) + (e & 1));
          const bool on = here[W8 ? x : x / 2] && key < min(lim[rh(e)], k_end);
          att |= (unsigned)on << (x * 4 + e);
          if (!on) s[x][e] = -INFINITY;
        }
    }
    // softmax of the two rows
    float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int x = 0; x < NS; ++x) {
      mx[0] = fmaxf(mx[0], fmaxf(s[x][0], s[x][W8 ? 2 : 1]));
      mx[1] = fmaxf(mx[1], fmaxf(s[x][W8 ? 1 : 2], s[x][3]));
    }
    float ref[2];
    bool raise = false;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
#pragma unroll
      for (int w = W8 ? 4 : 1; w <= (W8 ? 16 : 2); w *= 2) mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], w));
      raise |= mx[r] > m[r] + CF_RAISE || (m[r] == -INFINITY && mx[r] > m[r]);
    }
    if (__any_sync(0xffffffffu, raise)) {
      float f[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float mn = fmaxf(m[r], mx[r]);
        f[r] = mn == -INFINITY ? 1.f : ex2_approx(m[r] - mn);
        m[r] = mn;
        l[r] *= f[r];
      }
#pragma unroll
      for (int j = 0; j < NO; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] *= f[rh(e)];
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) ref[r] = m[r] == -INFINITY ? 0.f : m[r];
#pragma unroll
    for (int x = 0; x < NS; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[x][e] = ex2_approx(s[x][e] - ref[rh(e)]);
        l[rh(e)] += s[x][e];
      }
    // O += P V (W8: its transpose, V^T P^T, whose fragments of P^T are those of S's transpose turned round)
#pragma unroll
    for (int i = 0; i < F::NB; ++i) {
      constexpr int NP = W8 ? 2 : 4;
      uint32_t pf[NP];
      float ve[4] = {1.f, 1.f, 1.f, 1.f};   // V's scales: of keys 4 t to 4 t + 3 (W8: of key_g, key_g + 2)
      if constexpr (KT == KV_E4M3) {
        const uint8_t* vp = st[i] + F::EXPS + 16;
        if constexpr (W8) {
          ve[0] = exp_scale(vp[key_g]);
          ve[1] = exp_scale(vp[key_g + 2]);
        } else {
          const uint32_t x = *reinterpret_cast<const uint32_t*>(vp + 4 * t);
#pragma unroll
          for (int e = 0; e < 4; ++e) ve[e] = exp_scale(x >> (8 * e) & 0xff);
        }
      }
      // fragment e of P: elements 2 e and 2 e + 1 of the block's S
#pragma unroll
      for (int e = 0; e < NP; ++e) {
        const float(&x)[4] = s[W8 ? i : 2 * i + (e >> 1)];
        const int at = (e & 1) * 2;
        pf[e] = pack_bf16(x[at] * ve[W8 ? e : (e >> 1) * 2], x[at + 1] * ve[W8 ? e : (e >> 1) * 2 + 1]);
      }
      const uint8_t* vb = st[i] + F::BLOCK + t * F::GROUP + g * F::VVEC;
      auto row = [&](int k, int c) { return lds<F::VVEC>(vb + k * (DH * F::ES) + c * 8 * F::VVEC); };   // key 4 t + k
      uint32_t h0 = 0, h1 = 0;   // W8: the fragment of V before, the upper half of the matrix instruction's
      if (!edge) {
        if constexpr (W8) {
          pf[0] = turn8x8(pf[0]);
          pf[1] = turn8x8(pf[1]);
        }
#pragma unroll
        for (int c = 0; c < F::VN; ++c) {
          const Words<F::VVEC> v0 = row(0, c), v1 = row(1, c), v2 = row(2, c), v3 = row(3, c);
#pragma unroll
          for (int w = 0; w < F::VVEC / 4; ++w) {
            cf_pairs<KT>(v0.w[w], v1.w[w], v2.w[w], v3.w[w], [&](int e, uint32_t b0, uint32_t b1) {
              const int j = c * F::VE + w * (4 / F::ES) + e;
              if constexpr (W8) {
                if (j & 1) {
                  const uint32_t vf[4] = {h0, b0, h1, b1};
                  mma16816<false>(o[j / 2], vf, pf[0], pf[1]);
                }
                h0 = b0;
                h1 = b1;
              } else {
                mma16816<false>(o[j], pf, b0, b1);
              }
            });
          }
        }
        continue;
      }
      // V of keys that nobody here attends counts as zero; a NaN or infinite one that only some rows attend must not reach
      // the others through 0 * NaN: it counts as zero, and is put into the sums of its rows as NaN
      uint32_t ones[NP];
#pragma unroll
      for (int e = 0; e < NP; ++e) {
        const unsigned bits = att >> ((W8 ? i : 2 * i + (e >> 1)) * 4 + (e & 1) * 2);
        ones[e] = (bits & 1u ? 0x3f80u : 0u) | (bits & 2u ? 0x3f800000u : 0u);
        pf[e] &= (bits & 1u ? 0xffffu : 0u) | (bits & 2u ? 0xffff0000u : 0u);   // (an exponent of no entry may be anything)
        if constexpr (W8) {
          ones[e] = turn8x8(ones[e]);
          pf[e] = turn8x8(pf[e]);
        }
      }
#pragma unroll
      for (int c = 0; c < F::VN; ++c) {
        Words<F::VVEC> v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[k] = row(k, c);
          if (!here[i] || (b + i) * 16 + 4 * t + k >= k_end)
#pragma unroll
            for (int w = 0; w < F::VVEC / 4; ++w) v[k].w[w] = 0;
        }
#pragma unroll
        for (int w = 0; w < F::VVEC / 4; ++w)
          cf_pairs<KT>(v[0].w[w], v[1].w[w], v[2].w[w], v[3].w[w], [&](int e, uint32_t b0, uint32_t b1) {
            const int j = c * F::VE + w * (4 / F::ES) + e;
            if (W8 && !(j & 1)) {
              h0 = b0;
              h1 = b1;
              return;
            }
            float(&d)[4] = o[W8 ? j / 2 : j];
            const uint32_t n0 = __vcmpeq2(b0 & 0x7f807f80u, 0x7f807f80u), n1 = __vcmpeq2(b1 & 0x7f807f80u, 0x7f807f80u);
            float cnt[4] = {0.f, 0.f, 0.f, 0.f};
            bool bad;
            if constexpr (W8) {
              const uint32_t n2 = __vcmpeq2(h0 & 0x7f807f80u, 0x7f807f80u), n3 = __vcmpeq2(h1 & 0x7f807f80u, 0x7f807f80u);
              const uint32_t vf[4] = {h0 & ~n2, b0 & ~n0, h1 & ~n3, b1 & ~n1};
              mma16816<false>(d, vf, pf[0], pf[1]);
              bad = __any_sync(0xffffffffu, (n0 | n1 | n2 | n3) != 0);
              const uint32_t nf[4] = {n2 & 0x3f803f80u, n0 & 0x3f803f80u, n3 & 0x3f803f80u, n1 & 0x3f803f80u};
              if (bad) mma16816<false>(cnt, nf, ones[0], ones[1]);
            } else {
              mma16816<false>(d, pf, b0 & ~n0, b1 & ~n1);
              bad = __any_sync(0xffffffffu, (n0 | n1) != 0);
              if (bad) mma16816<false>(cnt, ones, n0 & 0x3f803f80u, n1 & 0x3f803f80u);
            }
            if (bad) {
#pragma unroll
              for (int x = 0; x < 4; ++x)
                if (cnt[x] > 0.f) d[x] = NAN;
            }
          });
      }
    }
    __syncwarp();   // everybody has read the round's stages
#pragma unroll
    for (int i = 0; i < F::NB; ++i)
      if (sent < n_blk) send();
  }
  if (!ok) {   // a copy did not land in time: what is sent lands before the CTA leaves
    s_abort = 1;
    if (lane == 0)
      for (int i = landed; i < sent; ++i) {
        const long long c0 = clock64();
        while ((there >> (i % 32) & 1) && !mbar_try_wait(&s_full[warp][i % F::STAGES], cf_phase >> (i % F::STAGES) & 1u) &&
               clock64() - c0 < CF_DRAIN_CYCLES) {
        }
      }
    __syncwarp();
  }
  __syncthreads();   // the rings' place is free

  // merge of the warps, in warp order
  float* s_o = reinterpret_cast<float*>(s_dyn);
#pragma unroll
  for (int r = 0; r < 2; ++r) {
#pragma unroll
    for (int w = W8 ? 4 : 1; w <= (W8 ? 16 : 2); w *= 2) l[r] += __shfl_xor_sync(0xffffffffu, l[r], w);
    if ((W8 ? g : t) == 0) {
      s_m[warp][W8 ? 2 * t + r : g + 8 * r] = m[r];
      s_l[warp][W8 ? 2 * t + r : g + 8 * r] = l[r];
    }
  }
  constexpr int LD = DH + 4;
#pragma unroll
  for (int jj = 0; jj < NO; ++jj) {
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int j = W8 ? 2 * jj + (x >> 1) : jj, c = j / F::VE, e = j % F::VE;
      const int r = W8 ? 2 * t + (x & 1) : g + 8 * (x >> 1), at = W8 ? g : 2 * t + (x & 1);
      if (r < n_row) s_o[(warp * ROWS + r) * LD + (c * 8 + at) * F::VE + e] = o[jj][x];
    }
  }
  __syncthreads();
  const PartView pv(a, p, CF_ROWS, DH, it.slot0 + it.split);
  for (int i = tid; i < n_row * (DH / 4); i += CF_WARPS * 32) {
    const int r = i / (DH / 4), d = i % (DH / 4) * 4, j = r / per_tok, gq = g0 + r % per_tok;
    if (gq >= group) continue;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < CF_WARPS; ++w) M = fmaxf(M, s_m[w][r]);
    const float mref = M == -INFINITY ? 0.f : M;
    float L = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < CF_WARPS; ++w) {
      const float f = ex2_approx(s_m[w][r] - mref);
      const float4 v = *reinterpret_cast<const float4*>(&s_o[(w * ROWS + r) * LD + d]);
      L += f * s_l[w][r];
      x[0] += f * v.x;
      x[1] += f * v.y;
      x[2] += f * v.z;
      x[3] += f * v.w;
    }
    if (cs > 1) {   // into the place of the first warp's sums, which this thread alone has read
      *reinterpret_cast<float4*>(&s_o[r * LD + d]) = make_float4(x[0], x[1], x[2], x[3]);
      if (d == 0) {
        s_cm[r] = M;
        s_cl[r] = L;
      }
    } else if (it.n_split > 1) {
      *reinterpret_cast<float4*>(pv.o + r * DH + d) = make_float4(x[0], x[1], x[2], x[3]);
      if (d == 0) *reinterpret_cast<float2*>(pv.ml + r * 2) = make_float2(M, L);
    } else {
      const float inv = L == 0.f ? 0.f : 1.f / L;
      uint2 y = make_uint2(pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv));
      *reinterpret_cast<uint2*>((bf16*)a.out + (size_t)(it.q0 + j0 + j) * a.ld_out + (size_t)(kvh * group + gq) * DH + d) = y;
    }
  }
  if (cs > 1) {
    // join over the cluster, in rank order: each CTA a share of the elements, all ranks' loads under way together
    cluster_sync();
    for (int i = tid + rank * (CF_WARPS * 32); i < n_row * (DH / 4); i += CF_WARPS * 32 * cs) {
      const int r = i / (DH / 4), d = i % (DH / 4) * 4, j = r / per_tok, gq = g0 + r % per_tok;
      if (gq >= group) continue;
      float m8[8], l8[8];
      float4 x8[8];
      float M = -INFINITY;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        m8[c] = -INFINITY;
        l8[c] = 0.f;
        x8[c] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < cs) {
          m8[c] = ld_cluster(&s_cm[r], c);
          l8[c] = ld_cluster(&s_cl[r], c);
          x8[c] = ld_cluster4(&s_o[r * LD + d], c);
        }
        M = fmaxf(M, m8[c]);
      }
      const float mref = M == -INFINITY ? 0.f : M;
      float L = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const float f = ex2_approx(m8[c] - mref);
        L += f * l8[c];
        x[0] += f * x8[c].x;
        x[1] += f * x8[c].y;
        x[2] += f * x8[c].z;
        x[3] += f * x8[c].w;
      }
      const float inv = L == 0.f ? 0.f : 1.f / L;
      *reinterpret_cast<uint2*>((bf16*)a.out + (size_t)(it.q0 + j0 + j) * a.ld_out + (size_t)(kvh * group + gq) * DH + d) =
          make_uint2(pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv));
    }
    cluster_sync();   // (a CTA's shared memory stays until all have read it)
  }
  if (a.late) pdl_wait();
}

// ---------------------------------------------------------------------------------------------
// Join of split tiles: CTA (i, y) = part y of tile i's elements; per element the splits' partials, taken in turn by as many groups
// of threads as the part leaves room for, the groups joined in order at the end.
//   M = max m_i,  out = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i
// Four partials' loads are under way at a time: with one at a time a join of 14 took 9 us, most of it memory latency.
// ---------------------------------------------------------------------------------------------
constexpr int CJ_THREADS = 256;
constexpr unsigned CJ_PARTS = 16;
struct JoinAcc {
  float m, l, o[4];
  __device__ __forceinline__ void add(const float (&mi)[4], const float (&li)[4], const float4 (&oi)[4]) {
    const float mn = fmaxf(fmaxf(fmaxf(mi[0], mi[1]), fmaxf(mi[2], mi[3])), m), ref = mn == -INFINITY ? 0.f : mn;
    const float f = ex2_approx(m - ref);   // (nothing yet, or a split without keys: 2^-inf = 0)
    m = mn;
    l *= f;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float w = ex2_approx(mi[k] - ref);
      l += w * li[k];
      o[0] += w * oi[k].x;
      o[1] += w * oi[k].y;
      o[2] += w * oi[k].z;
      o[3] += w * oi[k].w;
    }
  }
};
template <int DH, typename T>
__global__ void __launch_bounds__(CJ_THREADS) chunk_join_kernel(const __grid_constant__ ChunkCall a,
                                                                const __grid_constant__ SplitPlan p, int rows, int per_tok, int sub) {
  // rows: of a tile; per_tok: query heads of a tile's token; sub: tiles' head groups per KV head
  __shared__ SplitItem s_it;
  __shared__ int s_have;
  __shared__ float s_acc[6][CJ_THREADS];
  // The look-up runs beside the partials' kernel: it reads the lengths only, which that kernel, or the one before it, has
  // waited for before it let its follower start.
  const int tid = threadIdx.x;
  if (tid < 32) {
    SplitItem it;
    const bool have = split_find(a, p, (int)blockIdx.x, true, it);
    if (tid == 0) {
      s_it = it;
      s_have = have;
    }
  }
  KT_BEGIN();
  pdl_wait();
  KT_WAITED();
  pdl_launch_dependents();
  __syncthreads();
  if (!s_have || s_it.n_split <= 1) return;
  const SplitItem it = s_it;
  const int group = a.n_heads / a.c.n_kv_heads;
  const int j0 = it.tile * p.tq, n = min(p.tq, it.c - j0);
  const PartView pv(a, p, rows, DH, it.slot0);
  const int all = n * per_tok * (DH / 4), part = (all + (int)gridDim.y - 1) / (int)gridDim.y;   // elements of four columns
  const int i0 = (int)blockIdx.y * part, live = min(part, all - i0);
  if (live <= 0) return;
  const int groups = max(1, min(CJ_THREADS / live, (it.n_split + 3) / 4));
  const int gr = live < CJ_THREADS ? tid / live : 0;
  for (int i = live < CJ_THREADS ? tid % live : tid; i < live; i += CJ_THREADS) {
    const int r = (i0 + i) / (DH / 4), d = (i0 + i) % (DH / 4) * 4, j = r / per_tok, g = it.group % sub * per_tok + r % per_tok;
    JoinAcc x{-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    if (gr < groups) {
      for (int s0 = gr * 4; s0 < it.n_split; s0 += groups * 4) {
        float m[4], l[4];
        float4 o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          m[k] = -INFINITY;
          l[k] = 0.f;
          o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (s0 + k < it.n_split) {
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(pv.ml + ((size_t)(s0 + k) * rows + r) * 2));
            m[k] = ml.x;
            l[k] = ml.y;
            o[k] = __ldcg(reinterpret_cast<const float4*>(pv.o + ((size_t)(s0 + k) * rows + r) * DH + d));
          }
        }
        x.add(m, l, o);
      }
    }
    if (groups > 1) {   // (live < CJ_THREADS: every thread is here once)
      s_acc[0][tid] = x.m;
      s_acc[1][tid] = x.l;
#pragma unroll
      for (int e = 0; e < 4; ++e) s_acc[2 + e][tid] = x.o[e];
      __syncthreads();
      if (gr > 0) return;
      for (int k0 = 1; k0 < groups; k0 += 4) {
        float m[4], l[4];
        float4 o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int at = (k0 + k) * live + i;
          const bool on = k0 + k < groups;
          m[k] = on ? s_acc[0][at] : -INFINITY;
          l[k] = on ? s_acc[1][at] : 0.f;
          o[k] = on ? make_float4(s_acc[2][at], s_acc[3][at], s_acc[4][at], s_acc[5][at]) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        x.add(m, l, o);
      }
    }
    if (gr > 0 || g >= group) continue;
    const int h = it.group / sub * group + g;
    T* dst = (T*)a.out + (size_t)(it.q0 + j0 + j) * a.ld_out + (size_t)h * DH + d;
#pragma unroll
    for (int e = 0; e < 4; ++e) dst[e] = from_f<T>(x.l == 0.f ? 0.f : x.o[e] / x.l);
  }
}

int chunk_sms() {
  static const int sms = [] {
    int dev = 0, n = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    return std::max(1, n);
  }();
  return sms;
}

// How the CUDA-core and the few-row kernel run a call: plan, rows of a tile, query heads of a tile's token, head groups per KV head.
struct ChunkHow {
  bool few;
  SplitPlan p;
  int rows, per_tok, sub;
  bool may_split;
};
ChunkHow chunk_how(const KvPaged& c, int n_heads, int max_kv, bool aligned) {
  const int group = n_heads / c.n_kv_heads;
  ChunkHow w;
  w.few = c.type != KV_F32 && c.block_tokens == 16 && aligned;
  if (w.few) {
    w.rows = CF_ROWS;
    w.per_tok = std::min(group, CF_ROWS);
    w.sub = cdiv(group, w.per_tok);
    w.p = SplitPlan{CF_ROWS / w.per_tok, c.n_kv_heads * w.sub, CF_WARPS * 16 * (c.type == KV_BF16 ? 1 : 2), chunk_sms() * 3};
  } else {
    w.rows = CG_ROWS;
    w.per_tok = 1;
    w.sub = group;
    w.p = SplitPlan{CG_ROWS, n_heads, CG_KEYS, chunk_sms() * 4};
  }
  w.may_split = max_kv > w.p.unit;
  return w;
}
size_t how_bytes(const ChunkHow& w, const KvPaged& c) {
  return w.may_split ? (size_t)w.p.target * w.rows * (c.head_dim + 2) * sizeof(float) : 0;
}
// The most new tokens of a sequence that the few-row kernel takes.  It reads K and V again for each tile of 16 rows, which costs by
// the tiles of all sequences and heads; the tcgen05 kernel reads them once, but costs some 10 us more whatever the call, and
// 8-bit entries have to be widened for it.  Few-row and tcgen05 kernel in us, over 4096 keys, tokens x heads on KV heads x d_h:
//   bf16   8 x 32/8 x 128   14.3 15.1     16 x 32/8 x 128   16.9 16.1     32 x 32/32 x 128  25.2 24.0     16 x 32/32 x 128  22.5 23.6
//          48 x 12/12 x 64  14.0 14.1     96 x 12/12 x 64   18.3 14.8     96 x 4/2 x 128    15.4 18.8     16 x (8 x 32/8 x 128)   80 58
//   8-bit  16 x 32/8 x 128  20.5 25.5     48 x 32/8 x 128   33.3 30.3     64 x 32/32 x 128  40.3 54.3     96 x 32/32 x 128  55.1 59.4
//          96 x 12/12 x 64  19.7 23.1     128 x 12/12 x 64  23.6 23.5     16 x (8 x 32/8 x 128)   90 150  16 x (32 x 32/8 x 128)  225 157
// (Of these the rule takes the slower kernel at 96 x 32/32 x 128 over 8 bits, by 8 %.)
// Where sequences of both kinds meet: over bf16 entries all go to the tcgen05 kernel (its tiles are mostly empty for few
// tokens, but it reads K and V at the rate of the memory all the same), 8-bit ones are shared out (use_both).  7 sequences of a
// token over 2000 keys beside one of 256 over 1000, 32 heads on 8: bf16 30.8 us, shared out 41.7; 8-bit 54.6 and 43.3.
int few_tokens(const KvPaged& c, int n_heads) {
  const long long tiles = 24ll * 128 / ((long long)c.n_seq * c.n_kv_heads * c.head_dim) + (c.type == KV_E4M3 ? 4 : 0);
  return (int)std::max(1ll, tiles) * std::max(1, CF_ROWS / (n_heads / c.n_kv_heads));
}
// (no positions at all: the rows' zeros are the few-row kernel's, as there is nothing to widen or to map)
bool use_tc(const KvPaged& c, int n_heads, int max_q, int max_kv) {
  return max_kv > 0 && max_q > few_tokens(c, n_heads) && chunk_tc_takes(c, n_heads);
}
bool use_both(const KvPaged& c) { return c.type == KV_E4M3 && c.n_seq > 1; }

template <int DH, int KT, int ROWS>
struct FewTag {};

template <int DH, int KT, int ROWS>
cudaError_t few_t(cudaStream_t st, const ChunkCall& a, const ChunkHow& w, dim3 grid, int cs) {
  constexpr int smem = FewShape<DH, KT, ROWS>::SMEM;
  const cudaError_t e = smem_once<FewTag<DH, KT, ROWS>>(chunk_few_kernel<DH, KT, ROWS>, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(CF_WARPS * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  int n = 0;
  if (g_pdl) {
    at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cs > 1) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = (unsigned)cs;
    at[n].val.clusterDim.y = at[n].val.clusterDim.z = 1;
    ++n;
  }
  cfg.attrs = at;
  cfg.numAttrs = (unsigned)n;
  return cudaLaunchKernelEx(&cfg, chunk_few_kernel<DH, KT, ROWS>, a, w.p, w.per_tok, w.sub, cs);
}

template <int DH, int KT, typename T>
cudaError_t chunk_t(cudaStream_t st, const ChunkCall& a, const ChunkHow& w, int* launches) {
  const int max_c = std::min(a.max_q, a.c_hi);
  SplitPlan one = w.p;
  one.target = 0;
  const long long tiles = split_items(one, a.c.n_seq, a.n_rows, max_c);   // at most
  const dim3 grid((unsigned)split_items(w.p, a.c.n_seq, a.n_rows, max_c));
  cudaError_t e = cudaErrorInvalidValue;
  ++*launches;
  if (!w.few) {
    e = launch_k(chunk_any_kernel<DH, KT, T>, grid, dim3(CG_KEYS), 0, st, a, w.p);
  } else if constexpr (KT != KV_F32) {
    // A cluster per tile: the largest of 8, 4, 2 CTAs whose clusters find room at once, where that leaves a CTA a few rounds
    // (4 at heads of 128, 2 at 64, 1 at 32).  bf16, one call of a token each in a captured graph, cluster and split: 12 heads of 64,
    // 500 keys 5.5 and 7.4 us, 1000 keys 6.2 and 7.6, 2000 keys 7.6 and 7.7; 32 heads of 128 on 8, 500 keys 6.7 and 7.9,
    // 2000 keys 8.7 and 8.9, 4000 keys 12.0 and 10.1, 3 sequences of up to 4000 12.7 and 10.7.  (8 bits, 4000 keys: 11.7 and
    // 10.5, where the rule, by rounds of twice the keys, still takes the cluster.)  Clusters that had no room at once: 8 sequences
    // of 500 keys 14.6 and 10.5, 8 of up to 4000 keys and 32 heads 69 and 57.
    const long long units = cdiv(a.max_kv, w.p.unit);
    int cs = 8;
    while (cs > 1 && tiles * cs > w.p.target) cs >>= 1;
    const bool clusters = cs > 1 && w.may_split && units * 32 <= DH * cs;
    const dim3 g = clusters ? dim3((unsigned)(tiles * cs)) : grid;
    if (!clusters) cs = 1;
    const bool eight = (long long)max_c * (a.n_heads / a.c.n_kv_heads) <= 8;   // no tile has more rows
    e = eight ? few_t<DH, KT, 8>(st, a, w, g, cs) : few_t<DH, KT, 16>(st, a, w, g, cs);
    if (clusters) return e;
  }
  if (e == cudaSuccess && w.may_split) {
    ++*launches;
    // (more tiles than the target: none is split)
    const unsigned x = (unsigned)std::min<long long>(tiles, w.p.target), y = std::min(CJ_PARTS, std::max(1u, w.p.target / x));
    e = launch_k(chunk_join_kernel<DH, T>, dim3(x, y), dim3(CJ_THREADS), 0, st, a, w.p, w.rows, w.per_tok, w.sub);
  }
  return e;
}

cudaError_t chunk_simple(cudaStream_t st, const ChunkCall& a, bool aligned, int* launches) {
  const ChunkHow w = chunk_how(a.c, a.n_heads, a.max_kv, aligned);
#define CH_DH(D)                                                                   \
  case D:                                                                          \
    if (a.c.type == KV_F32) return chunk_t<D, KV_F32, float>(st, a, w, launches);  \
    if (a.c.type == KV_BF16) return chunk_t<D, KV_BF16, bf16>(st, a, w, launches); \
    return chunk_t<D, KV_E4M3, bf16>(st, a, w, launches);
  switch (a.c.head_dim) {
    CH_DH(32)
    CH_DH(64)
    CH_DH(128)
  }
#undef CH_DH
  return cudaErrorInvalidValue;
}

size_t round256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

// (whatever kernel the rows' alignment and the GPU pick.  Grows with n_seq, max_q and max_kv: few_tokens falls with n_seq, all
// else rises or stays.)
size_t chunk_workspace(const KvPaged& c, int n_heads, int max_q, int max_kv) {
  const size_t any = how_bytes(chunk_how(c, n_heads, max_kv, false), c), few = how_bytes(chunk_how(c, n_heads, max_kv, true), c);
  size_t tc = few;
  if (use_tc(c, n_heads, max_q, max_kv)) tc = (use_both(c) ? round256(few) : 0) + chunk_tc_workspace(c, max_kv);
  return std::max(any, tc);
}

cudaError_t launch_chunk_attention(cudaStream_t st, const ChunkCall& a0, int* launches) {
  ChunkCall a = a0;
  a.c_lo = 1;
  a.c_hi = a.max_q;
  a.late = 0;
  *launches = 0;
  const bool aligned = (((uintptr_t)a.q | (uintptr_t)a.out) & 15) == 0 && a.ld_q % 8 == 0 && a.ld_out % 8 == 0;
  if (!aligned || !use_tc(a.c, a.n_heads, a.max_q, a.max_kv) || !tc_gemm_supported()) return chunk_simple(st, a, aligned, launches);
  if (a.c.type != KV_E4M3) return launch_chunk_tc(st, a, launches);
  ChunkCall t = a;   // the tcgen05 kernel's share
  if (use_both(a.c)) {
    a.c_hi = few_tokens(a.c, a.n_heads);
    t.c_lo = a.c_hi + 1;
    t.part = (float*)((char*)a.part + round256(how_bytes(chunk_how(a.c, a.n_heads, a.max_kv, true), a.c)));
  }
  cudaError_t e = launch_chunk_widen(st, t, launches);
  // The few-row kernel needs nothing of the widening: it fills the SMs as that leaves them (late).  Its join waits for both,
  // then lets the tcgen05 kernel start, which so needs not wait for the join in turn.
  if (use_both(a.c) && e == cudaSuccess) {
    a.late = 1;
    e = chunk_simple(st, a, aligned, launches);
    t.late = *launches == 3;   // (there is a join)
  }
  return e == cudaSuccess ? launch_chunk_tc(st, t, launches) : e;
}

ADEPT_WAIT_LIMIT_SETTER(cf)

}  // namespace adept
