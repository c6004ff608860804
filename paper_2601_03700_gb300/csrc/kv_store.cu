// Rows of K and V into a paged cache, quantised as they are written, and entries of the cache back into rows.
//
// 8-bit form: for each (position, KV head), a = max |x| over the finite elements, a = 1.f 2^E; e = E - 8, one more where
// 1.f > 1.75 (so that a 2^-e <= 448, the largest e4m3), at least -126, 0 for a = 0.  Stored: e + 127 and e4m3(x 2^-e), round to
// nearest even.  The multiplication by a power of two is exact, so an element is rounded once, and reading back to bf16
// or fp32 is exact (4 significant bits).  A scale of 24 bits would gain nothing: e4m3's relative step does not depend on the
// scale.  NaN stays NaN; e4m3 has no infinity, an infinite element is stored as NaN.
//
// Bound by HBM: each element is read once and written once.  A vector (head_dim elements of K or of V) is held by
// head_dim / 8 threads, 8 elements each.
#include "kv_paged.h"

#include <cuda_fp8.h>

namespace adept {
namespace {

constexpr int KS_THREADS = 256;

template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (VEC && sizeof(T) == 2) {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  } else if constexpr (VEC) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_f<T>(p[i]);
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (VEC && sizeof(T) == 2) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
  } else if constexpr (VEC) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = from_f<T>(x[i]);
  }
}

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

// Thread group of TPV = head_dim / 8 threads per vector; a vector index is (row, K or V, head).
template <int DH, typename T, int KT, bool VEC>
__global__ void __launch_bounds__(KS_THREADS) kv_append_kernel(KvPaged c, int n_rows, const T* k, long long ld_k, const T* v,
                                                               long long ld_v, const int* seq, const int* pos) {
  PDL_ENTRY();
  constexpr int TPV = DH / 8;
  const int sub = threadIdx.x % TPV, hk = c.n_kv_heads;
  const long long n_vec = (long long)n_rows * 2 * hk;
  const long long step = (long long)gridDim.x * (KS_THREADS / TPV);
  // (whole warps leave the loop together: the vectors of a warp are padded up to it)
  const long long n_pad = (n_vec + 32 / TPV - 1) / (32 / TPV) * (32 / TPV);
  for (long long i = (long long)blockIdx.x * (KS_THREADS / TPV) + threadIdx.x / TPV; i < n_pad; i += step) {
    const bool in = i < n_vec;
    const long long ii = in ? i : n_vec - 1;
    const long long r = ii / (2 * hk);
    const int w = (int)(ii - r * (2 * hk)), is_v = w >= hk, h = is_v ? w - hk : w;
    float x[8];
    load8<T, VEC>((is_v ? v + r * ld_v : k + r * ld_k) + (size_t)h * DH + sub * 8, x);
    const long long e0 = in ? entry0(c, seq[r], pos[r]) : -1;
    const size_t e = (size_t)(e0 + (long long)h * c.block_tokens);
    if constexpr (KT == KV_E4M3) {
      float a = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float b = fabsf(x[j]);
        a = fmaxf(a, b == INFINITY ? 0.f : b);   // (fmaxf leaves NaN out)
      }
#pragma unroll
      for (int o = TPV / 2; o; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
      const unsigned bits = __float_as_uint(a);
      int ex = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
      ex = a == 0.f ? 0 : max(ex, -126);
      const float s = __uint_as_float((unsigned)(127 - ex) << 23);
      uint32_t out[2];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float y0 = x[2 * j] * s, y1 = x[2 * j + 1] * s;
        if (fabsf(x[2 * j]) == INFINITY) y0 = NAN;
        if (fabsf(x[2 * j + 1]) == INFINITY) y1 = NAN;
        const uint32_t two = __nv_cvt_float2_to_fp8x2(make_float2(y0, y1), __NV_SATFINITE, __NV_E4M3);
        if (j & 1)
          out[j >> 1] |= two << 16;
        else
          out[j >> 1] = two;
      }
      if (e0 >= 0) {
        *reinterpret_cast<uint2*>((uint8_t*)(is_v ? c.v : c.k) + e * DH + sub * 8) = make_uint2(out[0], out[1]);
        if (sub == 0) (is_v ? c.v_exp : c.k_exp)[e] = (uint8_t)(ex + 127);
      }
    } else if (e0 >= 0) {
      if constexpr (KT == KV_BF16)
        store8<bf16, true>((bf16*)(is_v ? c.v : c.k) + e * DH + sub * 8, x);
      else
        store8<float, true>((float*)(is_v ? c.v : c.k) + e * DH + sub * 8, x);
    }
  }
}

template <int DH, typename T, int KT, bool VEC>
__global__ void __launch_bounds__(KS_THREADS) kv_gather_kernel(KvPaged c, int n_rows, T* k, long long ld_k, T* v,
                                                               long long ld_v, const int* seq, const int* pos) {
  PDL_ENTRY();
  constexpr int TPV = DH / 8;
  const int sub = threadIdx.x % TPV, hk = c.n_kv_heads;
  const long long n_vec = (long long)n_rows * 2 * hk;
  const long long step = (long long)gridDim.x * (KS_THREADS / TPV);
  for (long long i = (long long)blockIdx.x * (KS_THREADS / TPV) + threadIdx.x / TPV; i < n_vec; i += step) {
    const long long r = i / (2 * hk);
    const int w = (int)(i - r * (2 * hk)), is_v = w >= hk, h = is_v ? w - hk : w;
    const long long e0 = entry0(c, seq[r], pos[r]);
    if (e0 < 0) continue;
    const size_t e = (size_t)(e0 + (long long)h * c.block_tokens);
    float x[8];
    if constexpr (KT == KV_E4M3) {
      const uint2 codes = *reinterpret_cast<const uint2*>((const uint8_t*)(is_v ? c.v : c.k) + e * DH + sub * 8);
      // 2^e with e down to -127 (a byte of 0 is the subnormal 2^-127)
      const int b = (is_v ? c.v_exp : c.k_exp)[e];
      const float s = b ? __uint_as_float((unsigned)b << 23) : __uint_as_float(0x400000u);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t word = j < 2 ? codes.x : codes.y;
        const __half2_raw hr = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(word >> (j & 1 ? 16 : 0)), __NV_E4M3);
        const float2 f = __half22float2(__half2(hr));
        x[2 * j] = f.x * s;
        x[2 * j + 1] = f.y * s;
      }
    } else if constexpr (KT == KV_BF16) {
      load8<bf16, true>((const bf16*)(is_v ? c.v : c.k) + e * DH + sub * 8, x);
    } else {
      load8<float, true>((const float*)(is_v ? c.v : c.k) + e * DH + sub * 8, x);
    }
    store8<T, VEC>((is_v ? v + r * ld_v : k + r * ld_k) + (size_t)h * DH + sub * 8, x);
  }
}

int ks_grid(const KvPaged& c, int n_rows) {
  static const int sms = [] {
    int dev = 0, n = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    return n > 0 ? n : 1;
  }();
  const long long per = KS_THREADS / (c.head_dim / 8), n = ((long long)n_rows * 2 * c.n_kv_heads + per - 1) / per;
  const long long most = (long long)sms * 8;
  return (int)(n < most ? n : most);
}

bool rows_aligned(const void* k, long long ld_k, const void* v, long long ld_v, int esz) {
  return (((uintptr_t)k | (uintptr_t)v) & 15) == 0 && (ld_k * esz) % 16 == 0 && (ld_v * esz) % 16 == 0;
}

template <int DH, typename T, int KT>
cudaError_t append_t(cudaStream_t st, const KvPaged& c, int n, const void* k, long long ld_k, const void* v, long long ld_v,
                     const int* seq, const int* pos) {
  auto kern = rows_aligned(k, ld_k, v, ld_v, (int)sizeof(T)) ? kv_append_kernel<DH, T, KT, true> : kv_append_kernel<DH, T, KT, false>;
  return launch_k(kern, dim3(ks_grid(c, n)), dim3(KS_THREADS), 0, st, c, n, (const T*)k, ld_k, (const T*)v, ld_v, seq, pos);
}
template <int DH, typename T, int KT>
cudaError_t gather_t(cudaStream_t st, const KvPaged& c, int n, void* k, long long ld_k, void* v, long long ld_v, const int* seq,
                     const int* pos) {
  auto kern = rows_aligned(k, ld_k, v, ld_v, (int)sizeof(T)) ? kv_gather_kernel<DH, T, KT, true> : kv_gather_kernel<DH, T, KT, false>;
  return launch_k(kern, dim3(ks_grid(c, n)), dim3(KS_THREADS), 0, st, c, n, (T*)k, ld_k, (T*)v, ld_v, seq, pos);
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
                             long long ld_v, const int* seq, const int* pos) {
  KS_DISPATCH(gather_t, dst_bf16, st, c, n_rows, k, ld_k, v, ld_v, seq, pos);
}

}  // namespace adept
