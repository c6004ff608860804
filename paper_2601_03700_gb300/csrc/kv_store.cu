// Rows of K and V into a paged cache, quantised as they are written, and entries of the cache back into rows.
//
// 8-bit form: for each (position, KV head), a = max |x| over the finite elements, a = 1.f 2^E; e = E - 8, one more where
// 1.f > 1.75 (so that a 2^-e <= 448, the largest e4m3), at least -126, 0 for a = 0.  Stored: e + 127 and e4m3(x 2^-e), round to
// nearest even.  The multiplication by a power of two is exact, so an element is rounded once, and reading back to bf16
// or fp32 is exact (4 significant bits).  A scale of 24 bits would gain nothing: e4m3's relative step does not depend on the
// scale.  NaN stays NaN; e4m3 has no infinity, an infinite element is stored as NaN.
//
// Bound by HBM: each element is read once and written once.  A thread holds 16 elements of a vector (head_dim elements of K or of
// V of one position), two vectors at a time with every load issued before the first is used.  A CTA takes whole rows, or a
// part of one where there are few.  What hides the look-ups (row -> position -> block -> entry, one load behind the other) is
// many small CTAs at different stages of that: 3 x 30011 rows of 32 heads of 128 from 8 bits to bf16 (738 MB) took 143 us with
// 256 threads of four vectors, 137 with 256 of two, 125 with 128 of two (5.9 TB/s), 127 with 128 of one, 123 with 64 of two (which
// writes 2048 rows in 41 us where 128 threads take 37).
#include "kv_paged.h"

#include <cuda_fp8.h>

#include <type_traits>

namespace adept {
namespace {

constexpr int KS_THREADS = 128, KS_ITEMS = 2, KS_EL = 16;

// 16 elements as they lie in memory (VEC: by 16 bytes), and as fp32.
template <typename T>
struct Piece {
  uint32_t w[KS_EL * sizeof(T) / 4];
  __device__ __forceinline__ void f32(float (&x)[KS_EL]) const {
#pragma unroll
    for (int i = 0; i < KS_EL; ++i) {
      if constexpr (sizeof(T) == 2)
        x[i] = __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
      else
        x[i] = __uint_as_float(w[i]);
    }
  }
  __device__ __forceinline__ void from(const float (&x)[KS_EL]) {
#pragma unroll
    for (int i = 0; i < KS_EL; ++i) {
      if constexpr (sizeof(T) == 2) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[i & ~1], x[i | 1]);
        w[i >> 1] = *reinterpret_cast<const uint32_t*>(&h);
      } else {
        w[i] = __float_as_uint(x[i]);
      }
    }
  }
  template <bool VEC>
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(w) / 16; ++i) {
        const uint4 v = reinterpret_cast<const uint4*>(p)[i];
        w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
      }
    } else {
      float x[KS_EL];
#pragma unroll
      for (int i = 0; i < KS_EL; ++i) x[i] = to_f<T>(p[i]);
      from(x);
    }
  }
  template <bool VEC>
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(w) / 16; ++i)
        reinterpret_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    } else {
      float x[KS_EL];
      f32(x);
#pragma unroll
      for (int i = 0; i < KS_EL; ++i) p[i] = from_f<T>(x[i]);
    }
  }
};

// Entry (position, head 0) of row r, as an index of [block][head][slot], or -1.
__device__ __forceinline__ long long entry0(const KvPaged& c, int seq, int pos) {
  if (seq < 0) return -1;   // a row that is left out
  int blk = -1;
  if (seq < c.n_seq && pos >= 0 && pos < c.max_blocks * c.block_tokens)
    blk = c.table[(size_t)seq * c.max_blocks + pos / c.block_tokens];
  if (blk < 0 || blk >= c.n_blocks) {
    c.flag(ERRW_POS);
    return -1;
  }
  return (long long)blk * c.n_kv_heads * c.block_tokens + pos % c.block_tokens;
}

// Item i of a CTA's rows: row, K or V, head, 16 elements of the head.
template <int DH>
struct Item {
  int r, is_v, h, sub;
  __device__ __forceinline__ Item(int i, int hk, int per_row) {
    r = (int)(((float)i + 0.5f) * (1.f / (float)per_row));   // (i < 2^21: exact)
    const int w = i - r * per_row, vec = w / (DH / KS_EL);
    sub = w % (DH / KS_EL);
    is_v = vec >= hk;
    h = vec - (is_v ? hk : 0);
  }
};

// 16 elements of a vector that TPV neighbouring threads hold, into entry `e` of K or V (-1: nowhere).
template <int DH>
__device__ __forceinline__ void store_e4m3(const KvPaged& c, bool is_v, long long e, int sub, const float (&y)[KS_EL]) {
  float a = 0.f;
#pragma unroll
  for (int j = 0; j < KS_EL; ++j) {
    const float b = fabsf(y[j]);
    a = fmaxf(a, b == INFINITY ? 0.f : b);   // (fmaxf leaves NaN out)
  }
#pragma unroll
  for (int o = DH / KS_EL / 2; o; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
  const unsigned bits = __float_as_uint(a);
  int ex = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  ex = a == 0.f ? 0 : max(ex, -126);
  const float s = __uint_as_float((unsigned)(127 - ex) << 23);
  uint32_t out[KS_EL / 4];
#pragma unroll
  for (int j = 0; j < KS_EL / 2; ++j) {
    float y0 = y[2 * j] * s, y1 = y[2 * j + 1] * s;
    if (fabsf(y[2 * j]) == INFINITY) y0 = NAN;
    if (fabsf(y[2 * j + 1]) == INFINITY) y1 = NAN;
    const uint32_t two = __nv_cvt_float2_to_fp8x2(make_float2(y0, y1), __NV_SATFINITE, __NV_E4M3);
    if (j & 1)
      out[j >> 1] |= two << 16;
    else
      out[j >> 1] = two;
  }
  if (e >= 0) {
    *reinterpret_cast<uint4*>((uint8_t*)(is_v ? c.v : c.k) + (size_t)e * DH + sub * KS_EL) = make_uint4(out[0], out[1], out[2], out[3]);
    if (sub == 0) (is_v ? c.v_exp : c.k_exp)[e] = (uint8_t)(ex + 127);
  }
}

template <int DH, typename T, int KT, bool VEC>
__global__ void __launch_bounds__(KS_THREADS) kv_append_kernel(KvPaged c, int n_rows, int rows_cta, const T* k, long long ld_k,
                                                               const T* v, long long ld_v, const int* seq, const int* pos) {
  PDL_ENTRY();
  constexpr int TPV = DH / KS_EL;   // threads of a vector: neighbours
  const int hk = c.n_kv_heads, per_row = 2 * hk * TPV, row0 = (int)blockIdx.x * rows_cta;
  const int total = min(rows_cta, n_rows - row0) * per_row;
  constexpr int PASS = KS_THREADS * KS_ITEMS;
  for (int i0 = (int)blockIdx.z * PASS; i0 < total; i0 += (int)gridDim.z * PASS) {
    Piece<T> x[KS_ITEMS];
    long long e[KS_ITEMS];   // the vector's entry, -1: not written
#pragma unroll
    for (int q = 0; q < KS_ITEMS; ++q) {
      const int i = i0 + q * KS_THREADS + threadIdx.x;
      const Item<DH> it(min(i, total - 1), hk, per_row);
      const long long r = row0 + it.r;
      x[q].template load<VEC>((it.is_v ? v + r * ld_v : k + r * ld_k) + (size_t)it.h * DH + it.sub * KS_EL);
      e[q] = i < total ? entry0(c, seq[r], pos[r]) : -1;
      if (e[q] >= 0) e[q] += (long long)it.h * c.block_tokens;
    }
#pragma unroll
    for (int q = 0; q < KS_ITEMS; ++q) {
      const Item<DH> it(min(i0 + q * KS_THREADS + (int)threadIdx.x, total - 1), hk, per_row);
      float y[KS_EL];
      x[q].f32(y);
      if constexpr (KT == KV_E4M3) {
        store_e4m3<DH>(c, it.is_v, e[q], it.sub, y);
      } else if (e[q] >= 0) {
        using C = typename std::conditional<KT == KV_BF16, bf16, float>::type;
        Piece<C> z;
        z.from(y);
        z.template store<true>((C*)(it.is_v ? c.v : c.k) + (size_t)e[q] * DH + it.sub * KS_EL);
      }
    }
  }
}

// bf16 entries of a staging cache into an 8-bit one: rows [0, n_rows[y]) of layer y (n_rows NULL: max_rows), row r token
// row_tok[r] (NULL: r) at (tok_seq, tok_pos).  Layer y of the source is src_layer0 + y.
template <int DH>
__global__ void __launch_bounds__(KS_THREADS) kv_requant_kernel(KVCacheView src, int src_layer0, KvPaged c, const int* n_rows,
                                                                int max_rows, int rows_cta, const int* row_tok,
                                                                const int* tok_seq, const int* tok_pos) {
  PDL_ENTRY();
  constexpr int TPV = DH / KS_EL;
  const int y = (int)blockIdx.y, n = n_rows ? min(n_rows[y], max_rows) : max_rows;
  const int hk = c.n_kv_heads, per_row = 2 * hk * TPV, row0 = (int)blockIdx.x * rows_cta;
  const int total = min(rows_cta, n - row0) * per_row;
  const long long layer = (long long)y * c.n_blocks * hk * c.block_tokens;   // entries
  for (int i0 = (int)blockIdx.z * KS_THREADS; i0 < total; i0 += (int)gridDim.z * KS_THREADS) {
    const int i = i0 + (int)threadIdx.x;
    const Item<DH> it(min(i, total - 1), hk, per_row);
    const int tok = row_tok ? row_tok[row0 + it.r] : row0 + it.r, seq = tok_seq[tok], pos = tok_pos[tok];
    const long long from = src.checked_base(src_layer0 + y, seq, pos);
    const long long e0 = i < total && from >= 0 ? entry0(c, seq, pos) : -1;
    float x[KS_EL];
#pragma unroll
    for (int j = 0; j < KS_EL; ++j) x[j] = 0.f;
    if (e0 >= 0) {
      Piece<bf16> w;
      w.template load<true>((const bf16*)(it.is_v ? src.v : src.k) + from + (size_t)it.h * src.head_stride() + it.sub * KS_EL);
      w.f32(x);
    }
    store_e4m3<DH>(c, it.is_v, e0 < 0 ? -1 : layer + e0 + (long long)it.h * c.block_tokens, it.sub, x);
  }
}

template <int DH, typename T, int KT, bool VEC>
__global__ void __launch_bounds__(KS_THREADS) kv_gather_kernel(KvPaged c, int n_rows, int rows_cta, T* k, long long ld_k, T* v,
                                                               long long ld_v, const int* seq, const int* pos, int seq0, int pos0) {
  PDL_ENTRY();
  constexpr int TPV = DH / KS_EL;
  const int hk = c.n_kv_heads, per_row = 2 * hk * TPV, row0 = (int)blockIdx.x * rows_cta;
  const int total = min(rows_cta, n_rows - row0) * per_row;
  using C = typename std::conditional<KT == KV_F32, float, bf16>::type;
  constexpr int PASS = KS_THREADS * KS_ITEMS;
  for (int i0 = (int)blockIdx.z * PASS; i0 < total; i0 += (int)gridDim.z * PASS) {
    Piece<C> x[KS_ITEMS];   // (e4m3: 16 codes in the first four words)
    int ex[KS_ITEMS];
    bool on[KS_ITEMS];
#pragma unroll
    for (int q = 0; q < KS_ITEMS; ++q) {
      const int i = i0 + q * KS_THREADS + threadIdx.x;
      const Item<DH> it(min(i, total - 1), hk, per_row);
      const long long r = row0 + it.r;
      const long long e0 = i >= total ? -1 : seq ? entry0(c, seq[r], pos[r]) : entry0(c, seq0, pos0 + (int)r);
      on[q] = e0 >= 0;
      if (!on[q]) continue;
      const size_t e = (size_t)(e0 + (long long)it.h * c.block_tokens), at = e * DH + it.sub * KS_EL;
      const void* pool = it.is_v ? c.v : c.k;
      if constexpr (KT == KV_E4M3) {
        const uint4 w = *reinterpret_cast<const uint4*>((const uint8_t*)pool + at);
        x[q].w[0] = w.x; x[q].w[1] = w.y; x[q].w[2] = w.z; x[q].w[3] = w.w;
        ex[q] = (it.is_v ? c.v_exp : c.k_exp)[e];
      } else {
        x[q].template load<true>((const C*)pool + at);
      }
    }
#pragma unroll
    for (int q = 0; q < KS_ITEMS; ++q) {
      if (!on[q]) continue;
      const Item<DH> it(i0 + q * KS_THREADS + (int)threadIdx.x, hk, per_row);
      const long long r = row0 + it.r;
      float y[KS_EL];
      if constexpr (KT == KV_E4M3) {
        const float s = exp_scale(ex[q]);
#pragma unroll
        for (int j = 0; j < KS_EL / 2; ++j) {
          const uint32_t h = e4m3x2_f16x2(x[q].w[j >> 1] >> (j & 1 ? 16 : 0));
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
          y[2 * j] = f.x * s;
          y[2 * j + 1] = f.y * s;
        }
      } else {
        x[q].f32(y);
      }
      Piece<T> z;
      z.from(y);
      z.template store<VEC>((it.is_v ? v + r * ld_v : k + r * ld_k) + (size_t)it.h * DH + it.sub * KS_EL);
    }
  }
}

// Rows of a CTA: one pass of all its threads, at least one row, where there are rows enough for two CTAs an SM.  Where there are
// not, the passes of a row that is longer than one get a CTA each (z): 8 rows of 32 heads of 128 written and read back took 5.5 us
// by 16 CTAs, 8.2 by 8; 30000 rows 285 us by a CTA a row, 304 by two.
int ks_rows(const KvPaged& c, int n_rows, int pass, int* z) {
  static const int sms = [] {
    int dev = 0, n = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    return n > 0 ? n : 1;
  }();
  const int per_row = 2 * c.n_kv_heads * (c.head_dim / KS_EL), full = pass / per_row;
  const int spread = n_rows / (2 * sms);
  const int r = full < spread ? full : spread;
  *z = spread < 1 ? cdiv(per_row, pass) : 1;
  return r > 1 ? r : 1;
}

bool rows_aligned(const void* k, long long ld_k, const void* v, long long ld_v, int esz) {
  return (((uintptr_t)k | (uintptr_t)v) & 15) == 0 && (ld_k * esz) % 16 == 0 && (ld_v * esz) % 16 == 0;
}

template <int DH, typename T, int KT>
cudaError_t append_t(cudaStream_t st, const KvPaged& c, int n, const void* k, long long ld_k, const void* v, long long ld_v,
                     const int* seq, const int* pos) {
  auto kern = rows_aligned(k, ld_k, v, ld_v, (int)sizeof(T)) ? kv_append_kernel<DH, T, KT, true> : kv_append_kernel<DH, T, KT, false>;
  int z;
  const int rows = ks_rows(c, n, KS_THREADS * KS_ITEMS, &z);
  return launch_k(kern, dim3((unsigned)cdiv(n, rows), 1, (unsigned)z), dim3(KS_THREADS), 0, st, c, n, rows, (const T*)k, ld_k, (const T*)v, ld_v, seq, pos);
}
template <int DH, typename T, int KT>
cudaError_t gather_t(cudaStream_t st, const KvPaged& c, int n, void* k, long long ld_k, void* v, long long ld_v, const int* seq,
                     const int* pos, int seq0, int pos0) {
  auto kern = rows_aligned(k, ld_k, v, ld_v, (int)sizeof(T)) ? kv_gather_kernel<DH, T, KT, true> : kv_gather_kernel<DH, T, KT, false>;
  int z;
  const int rows = ks_rows(c, n, KS_THREADS * KS_ITEMS, &z);
  return launch_k(kern, dim3((unsigned)cdiv(n, rows), 1, (unsigned)z), dim3(KS_THREADS), 0, st, c, n, rows, (T*)k, ld_k, (T*)v, ld_v, seq, pos, seq0, pos0);
}

#define KS_DISPATCH(F, BF, ...)                                                                   \
  switch (c.head_dim * 8 + c.type * 2 + (BF ? 1 : 0)) {                                           \
    case 32 * 8 + KV_F32 * 2: return F<32, float, KV_F32>(__VA_ARGS__);                           \
    case 32 * 8 + KV_F32 * 2 + 1: return F<32, bf16, KV_F32>(__VA_ARGS__);                        \
    case 32 * 8 + KV_BF16 * 2: return F<32, float, KV_BF16>(__VA_ARGS__);                         \
    case 32 * 8 + KV_BF16 * 2 + 1: return F<32, bf16, KV_BF16>(__VA_ARGS__);                      \
    case 32 * 8 + KV_E4M3 * 2: return F<32, float, KV_E4M3>(__VA_ARGS__);                         \
    case 32 * 8 + KV_E4M3 * 2 + 1: return F<32, bf16, KV_E4M3>(__VA_ARGS__);                      \
    case 64 * 8 + KV_F32 * 2: return F<64, float, KV_F32>(__VA_ARGS__);                           \
    case 64 * 8 + KV_F32 * 2 + 1: return F<64, bf16, KV_F32>(__VA_ARGS__);                        \
    case 64 * 8 + KV_BF16 * 2: return F<64, float, KV_BF16>(__VA_ARGS__);                         \
    case 64 * 8 + KV_BF16 * 2 + 1: return F<64, bf16, KV_BF16>(__VA_ARGS__);                      \
    case 64 * 8 + KV_E4M3 * 2: return F<64, float, KV_E4M3>(__VA_ARGS__);                         \
    case 64 * 8 + KV_E4M3 * 2 + 1: return F<64, bf16, KV_E4M3>(__VA_ARGS__);                      \
    case 128 * 8 + KV_F32 * 2: return F<128, float, KV_F32>(__VA_ARGS__);                         \
    case 128 * 8 + KV_F32 * 2 + 1: return F<128, bf16, KV_F32>(__VA_ARGS__);                      \
    case 128 * 8 + KV_BF16 * 2: return F<128, float, KV_BF16>(__VA_ARGS__);                       \
    case 128 * 8 + KV_BF16 * 2 + 1: return F<128, bf16, KV_BF16>(__VA_ARGS__);                    \
    case 128 * 8 + KV_E4M3 * 2: return F<128, float, KV_E4M3>(__VA_ARGS__);                       \
    case 128 * 8 + KV_E4M3 * 2 + 1: return F<128, bf16, KV_E4M3>(__VA_ARGS__);                    \
  }                                                                                               \
  return cudaErrorInvalidValue

}  // namespace

cudaError_t launch_kv_append(cudaStream_t st, const KvPaged& c, int n_rows, int src_bf16, const void* k, long long ld_k,
                             const void* v, long long ld_v, const int* seq, const int* pos) {
  KS_DISPATCH(append_t, src_bf16, st, c, n_rows, k, ld_k, v, ld_v, seq, pos);
}

cudaError_t launch_kv_gather(cudaStream_t st, const KvPaged& c, int n_rows, int dst_bf16, void* k, long long ld_k, void* v,
                             long long ld_v, const int* seq, const int* pos, int seq0, int pos0) {
  KS_DISPATCH(gather_t, dst_bf16, st, c, n_rows, k, ld_k, v, ld_v, seq, pos, seq0, pos0);
}

cudaError_t launch_kv_requant(cudaStream_t st, const KVCacheView& src, int src_layer0, const KvPaged& c, int n_layers,
                              const int* n_rows, int max_rows, const int* row_tok, const int* tok_seq, const int* tok_pos) {
  auto kern = c.head_dim == 128 ? kv_requant_kernel<128> : c.head_dim == 64 ? kv_requant_kernel<64> : kv_requant_kernel<32>;
  int z;
  const int rows = ks_rows(c, max_rows, KS_THREADS, &z);
  return launch_k(kern, dim3((unsigned)cdiv(max_rows, rows), (unsigned)n_layers, (unsigned)z), dim3(KS_THREADS), 0, st, src, src_layer0, c, n_rows,
                  max_rows, rows, row_tok, tok_seq, tok_pos);
}

}  // namespace adept
