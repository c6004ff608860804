// Attention of a chunk of new tokens over a paged K/V cache: sequence b brings c_b >= 0 new tokens, the last of its kv_len_b
// cached positions; the token at position p attends positions 0..p.
//
//   out = sum_k exp(s_k - m) v_k / sum_k exp(s_k - m),   s_k = q . k_k / sqrt(head_dim),   m = max s_k
//
// in one pass over the keys with the running maximum and sum (fp32, exponentials in base 2).  A token without keys (a chunk
// longer than kv_len) gives zeros.  What lies behind a token's position is never used: neither scores nor V entries of
// masked positions enter a sum, so NaN or infinities there do not spread.  Keys in blocks that the table does not hold
// (negative, out of range) are left out and flagged.
//
// The split of the work, and the join of split tiles, are in kv_paged.h.
#include "kv_paged.h"

#include <cuda_fp8.h>

#include <algorithm>

namespace adept {
namespace {

// ---------------------------------------------------------------------------------------------
// Any type, head size, alignment and block size: CUDA-core kernel.  CTA = up to CG_ROWS new tokens of one query head x a
// run of keys, 128 keys at a time: a thread per key for the scores, a warp per token for the softmax, a thread per
// dimension for the weighted sum.
// ---------------------------------------------------------------------------------------------
constexpr int CG_ROWS = 4, CG_KEYS = 128;

// Element i of entry `e` of K or V as fp32; e4m3 codes without their exponent.
template <int KT>
__device__ __forceinline__ float kv_elem(const void* p, size_t i) {
  if constexpr (KT == KV_F32) return ((const float*)p)[i];
  else if constexpr (KT == KV_BF16) return __bfloat162float(((const bf16*)p)[i]);
  else return __half2float(__half(__nv_cvt_fp8_to_halfraw(((const uint8_t*)p)[i], __NV_E4M3)));
}
__device__ __forceinline__ float exp_scale(int b) {   // 2^(b - 127)
  return b ? __uint_as_float((unsigned)b << 23) : __uint_as_float(0x400000u);
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
  __shared__ float s_q[CG_ROWS][DH];
  __shared__ float s_p[CG_ROWS][CG_KEYS];
  __shared__ long long s_e[CG_KEYS];
  __shared__ float s_vs[CG_KEYS], s_corr[CG_ROWS];
  __shared__ float s_red[CG_KEYS];
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
  const int past = it.len - it.c;   // row j's position is past + j
  for (int i = tid; i < n * DH; i += CG_KEYS)
    s_q[i / DH][i % DH] = to_f<T>(((const T*)a.q)[(size_t)(it.q0 + j0 + i / DH) * a.ld_q + (size_t)h * DH + i % DH]);
  const int k_end = min(it.u1 * CG_KEYS, min(it.len, past + j0 + n));
  constexpr int KG = CG_KEYS / DH > 0 ? CG_KEYS / DH : 1;   // key groups of the weighted sum
  const int d = tid % DH, kg = tid / DH;
  float acc[CG_ROWS], m = -INFINITY, l = 0.f;   // (m, l of row `warp`)
#pragma unroll
  for (int r = 0; r < CG_ROWS; ++r) acc[r] = 0.f;
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
    if (KT == KV_E4M3 && e >= 0) {
      ks = exp_scale(a.c.k_exp[e]);
      s_vs[tid] = exp_scale(a.c.v_exp[e]);
    }
    s_e[tid] = e;
    __syncthreads();   // (and s_q; s_p and s_corr of the previous round are read)
    float dot[CG_ROWS];
#pragma unroll
    for (int r = 0; r < CG_ROWS; ++r) dot[r] = 0.f;
    if (e >= 0) {
      for (int i = 0; i < DH; ++i) {
        const float x = kv_elem<KT>(a.c.k, (size_t)e * DH + i);
#pragma unroll
        for (int r = 0; r < CG_ROWS; ++r) dot[r] = fmaf(x, s_q[r][i], dot[r]);
      }
    }
#pragma unroll
    for (int r = 0; r < CG_ROWS; ++r)
      s_p[r][tid] = e >= 0 && r < n && key <= past + j0 + r ? dot[r] * ks * a.scale_log2 : -INFINITY;
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
    for (int r = 0; r < CG_ROWS; ++r) acc[r] *= s_corr[r];
    const int nk = min(CG_KEYS, k_end - k0);
    for (int k = kg; k < nk; k += KG) {
      const long long ev = s_e[k];
      if (ev < 0) continue;
      float x = kv_elem<KT>(a.c.v, (size_t)ev * DH + d);
      if (KT == KV_E4M3) x *= s_vs[k];
#pragma unroll
      for (int r = 0; r < CG_ROWS; ++r)
        if (k0 + k <= past + j0 + r) acc[r] = fmaf(s_p[r][k], x, acc[r]);
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
  for (int r = 0; r < CG_ROWS; ++r) {
    s_red[tid] = acc[r];
    __syncthreads();
    float o = 0.f;
    if (tid < DH)
      for (int g = 0; g < KG; ++g) o += s_red[g * DH + tid];
    if (tid < DH && r < n) {
      const float sum = s_corr[r];
      if (it.n_split > 1)
        pv.o[r * DH + tid] = o;
      else
        ((T*)a.out)[(size_t)(it.q0 + j0 + r) * a.ld_out + (size_t)h * DH + tid] =
            from_f<T>(past + j0 + r < 0 ? 0.f : o / sum);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------
// Join of split tiles: CTA = one tile; per row the splits' partials in split order.
//   M = max m_i,  out = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i
// ---------------------------------------------------------------------------------------------
template <int DH, typename T>
__global__ void __launch_bounds__(128) chunk_join_kernel(const __grid_constant__ ChunkCall a, const __grid_constant__ SplitPlan p,
                                                         int rows, int per_tok, int sub) {
  // rows: of a tile; per_tok: query heads of a tile's token; sub: tiles' head groups per KV head
  __shared__ SplitItem s_it;
  __shared__ int s_have;
  PDL_ENTRY();
  const int tid = threadIdx.x;
  if (tid < 32) {
    SplitItem it;
    const bool have = split_find(a, p, (int)blockIdx.x, true, it);
    if (tid == 0) {
      s_it = it;
      s_have = have;
    }
  }
  __syncthreads();
  if (!s_have || s_it.n_split <= 1) return;
  const SplitItem it = s_it;
  const int group = a.n_heads / a.c.n_kv_heads;
  const int past = it.len - it.c, j0 = it.tile * p.tq, n = min(p.tq, it.c - j0);
  const PartView pv(a, p, rows, DH, it.slot0);
  for (int i = tid; i < n * per_tok * (DH / 4); i += 128) {
    const int r = i / (DH / 4), d = i % (DH / 4) * 4, j = r / per_tok, g = it.group % sub * per_tok + r % per_tok;
    if (g >= group) continue;
    const int h = it.group / sub * group + g;
    float M = -INFINITY;
    for (int s = 0; s < it.n_split; ++s) M = fmaxf(M, __ldcg(pv.ml + ((size_t)s * rows + r) * 2));
    float L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    const float ref = M == -INFINITY ? 0.f : M;
    for (int s = 0; s < it.n_split; ++s) {
      const float2 ml = __ldcg(reinterpret_cast<const float2*>(pv.ml + ((size_t)s * rows + r) * 2));
      const float4 x = __ldcg(reinterpret_cast<const float4*>(pv.o + ((size_t)s * rows + r) * DH + d));
      const float w = exp2f(ml.x - ref);   // (a split without keys: 2^-inf = 0)
      L += w * ml.y;
      o[0] += w * x.x;
      o[1] += w * x.y;
      o[2] += w * x.z;
      o[3] += w * x.w;
    }
    T* dst = (T*)a.out + (size_t)(it.q0 + j0 + j) * a.ld_out + (size_t)h * DH + d;
#pragma unroll
    for (int e = 0; e < 4; ++e) dst[e] = from_f<T>(past + j0 + j < 0 ? 0.f : o[e] / L);
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

// How a call is run: its plan, rows of a tile and query heads of a tile's token.
struct ChunkHow {
  SplitPlan p;
  int rows, per_tok, sub;
  bool may_split;
};
ChunkHow chunk_how(const KvPaged& c, int n_heads, int n_rows, int max_q, int max_kv) {
  ChunkHow w;
  w.rows = CG_ROWS;
  w.per_tok = 1;
  w.sub = n_heads / c.n_kv_heads;
  w.p = SplitPlan{CG_ROWS, n_heads, CG_KEYS, chunk_sms() * 4};
  (void)n_rows;
  (void)max_q;
  w.may_split = max_kv > w.p.unit;
  return w;
}

}  // namespace

size_t chunk_workspace(const KvPaged& c, int n_heads, int n_rows, int max_q, int max_kv) {
  const ChunkHow w = chunk_how(c, n_heads, n_rows, max_q, max_kv);
  return w.may_split ? (size_t)w.p.target * w.rows * (c.head_dim + 2) * sizeof(float) : 0;
}

template <int DH, int KT, typename T>
static cudaError_t chunk_t(cudaStream_t st, const ChunkCall& a, const ChunkHow& w, int* launches) {
  const long long items = split_items(w.p, a.c.n_seq, a.n_rows, a.max_q);
  *launches = 1;
  cudaError_t e = launch_k(chunk_any_kernel<DH, KT, T>, dim3((unsigned)items), dim3(CG_KEYS), 0, st, a, w.p);
  if (e == cudaSuccess && w.may_split) {
    *launches = 2;
    e = launch_k(chunk_join_kernel<DH, T>, dim3((unsigned)w.p.target), dim3(128), 0, st, a, w.p, w.rows, w.per_tok, w.sub);
  }
  return e;
}

cudaError_t launch_chunk_attention(cudaStream_t st, const ChunkCall& a, int* launches) {
  const ChunkHow w = chunk_how(a.c, a.n_heads, a.n_rows, a.max_q, a.max_kv);
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

}  // namespace adept
