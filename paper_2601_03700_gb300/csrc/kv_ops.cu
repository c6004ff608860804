// C ABI of the operators on a caller-owned paged K/V cache (adept_kv_cache): checks of the arguments, then one or two
// launches on the caller's stream.  They hold no state and allocate nothing.
#include "adept.h"
#include "common.cuh"
#include "kernels.h"
#include "kv_paged.h"
#include "model_view.h"

#include <cmath>
#include <cstdarg>
#include <cstdio>

using namespace adept;

namespace {

adept_status bad(adept_status s, const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  global_set_error(buf);
  return s;
}

adept_status view_of(const adept_kv_cache* c, KvPaged* v) {
  if (!c) return bad(ADEPT_ERR_INVALID_ARG, "NULL cache");
  if (c->kv_type < ADEPT_KV_F32 || c->kv_type > ADEPT_KV_E4M3) return bad(ADEPT_ERR_INVALID_ARG, "kv_type %d unknown", c->kv_type);
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128)
    return bad(ADEPT_ERR_INVALID_ARG, "head_dim %d unsupported (32, 64 or 128)", c->head_dim);
  if (c->n_blocks < 1 || c->n_kv_heads < 1 || c->block_tokens < 1 || c->n_seq < 1 || c->max_blocks_per_seq < 1)
    return bad(ADEPT_ERR_INVALID_ARG, "non-positive cache size");
  if ((long long)c->max_blocks_per_seq * c->block_tokens > (1ll << 30) || (long long)c->n_kv_heads * c->head_dim > (1 << 20))
    return bad(ADEPT_ERR_INVALID_ARG, "cache too large (2^30 positions a sequence, 2^20 elements a position)");
  if (!c->d_k || !c->d_v || !c->d_block_table) return bad(ADEPT_ERR_INVALID_ARG, "NULL cache pointer");
  if (((uintptr_t)c->d_block_table | (uintptr_t)c->d_err) & 3) return bad(ADEPT_ERR_INVALID_ARG, "misaligned block table or error word");
  if (((uintptr_t)c->d_k | (uintptr_t)c->d_v) & 15) return bad(ADEPT_ERR_INVALID_ARG, "K and V must start on 16 bytes");
  if (c->kv_type == ADEPT_KV_E4M3 && (!c->d_k_exp || !c->d_v_exp))
    return bad(ADEPT_ERR_INVALID_ARG, "an e4m3 cache needs its exponents");
  if (c->kv_type == ADEPT_KV_E4M3 && (((uintptr_t)c->d_k_exp | (uintptr_t)c->d_v_exp) & 15))
    return bad(ADEPT_ERR_INVALID_ARG, "the exponents must start on 16 bytes");
  *v = KvPaged{c->d_k, c->d_v, c->d_k_exp, c->d_v_exp, c->d_block_table, c->d_err, c->kv_type, c->n_blocks, c->n_kv_heads,
               c->head_dim, c->block_tokens, c->n_seq, c->max_blocks_per_seq};
  return ADEPT_OK;
}

adept_status rows_ok(const KvPaged& v, int n_rows, int dtype, const void* k, int64_t ld_k, const void* vv, int64_t ld_v,
                     const int32_t* seq, const int32_t* pos) {
  if (n_rows < 0) return bad(ADEPT_ERR_INVALID_ARG, "n_rows %d < 0", n_rows);
  if (dtype != ADEPT_DTYPE_F32 && dtype != ADEPT_DTYPE_BF16) return bad(ADEPT_ERR_INVALID_ARG, "dtype %d unknown", dtype);
  if (n_rows == 0) return ADEPT_OK;
  if (!k || !vv || !seq || !pos) return bad(ADEPT_ERR_INVALID_ARG, "NULL device pointer");
  const int64_t w = (int64_t)v.n_kv_heads * v.head_dim;
  if (ld_k < w || ld_v < w) return bad(ADEPT_ERR_INVALID_ARG, "row stride below the %lld elements of a row", (long long)w);
  const uintptr_t m = dtype == ADEPT_DTYPE_BF16 ? 1 : 3;
  if (((uintptr_t)k | (uintptr_t)vv) & m) return bad(ADEPT_ERR_INVALID_ARG, "misaligned rows");
  if (((uintptr_t)seq | (uintptr_t)pos) & 3) return bad(ADEPT_ERR_INVALID_ARG, "misaligned sequences or positions");
  return ADEPT_OK;
}

adept_status launched(cudaError_t e) {
  if (e == cudaSuccess) return ADEPT_OK;
  cudaGetLastError();
  return bad(ADEPT_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}

adept_status call_ok(const KvPaged& v, int n_heads, int n_rows, int max_q, int max_kv) {
  if (n_heads < 1 || n_heads % v.n_kv_heads || n_heads > (1 << 15))
    return bad(ADEPT_ERR_INVALID_ARG, "n_heads %d is no multiple of n_kv_heads %d, or above 2^15", n_heads, v.n_kv_heads);
  if (n_rows < 0 || max_q < 0 || max_kv < 0) return bad(ADEPT_ERR_INVALID_ARG, "negative size");
  if (max_kv > v.max_blocks * v.block_tokens)
    return bad(ADEPT_ERR_INVALID_ARG, "max_kv_len %d above the %d positions of a sequence", max_kv, v.max_blocks * v.block_tokens);
  if ((long long)n_rows * n_heads > (1ll << 30) || (long long)v.n_seq * n_heads >= (1ll << 30))
    return bad(ADEPT_ERR_CAPACITY, "n_rows * n_heads above 2^30, or n_seq * n_heads");
  if (n_heads / v.n_kv_heads <= 128 && !chunk_tc_fits(v, n_heads, n_rows, max_q, max_kv))
    return bad(ADEPT_ERR_CAPACITY, "a call of more than 2^31 tiles");
  return ADEPT_OK;
}

}  // namespace

extern "C" {

adept_status adept_kv_append(const adept_kv_cache* c, int n_rows, int dtype, const void* d_k, int64_t ld_k, const void* d_v,
                             int64_t ld_v, const int32_t* d_seq, const int32_t* d_pos, void* stream) {
  KvPaged v;
  adept_status s = view_of(c, &v);
  if (s == ADEPT_OK) s = rows_ok(v, n_rows, dtype, d_k, ld_k, d_v, ld_v, d_seq, d_pos);
  if (s != ADEPT_OK || n_rows == 0) return s;
  PdlScope pdl(true);
  return launched(launch_kv_append((cudaStream_t)stream, v, n_rows, dtype == ADEPT_DTYPE_BF16, d_k, ld_k, d_v, ld_v, d_seq, d_pos));
}

adept_status adept_kv_gather(const adept_kv_cache* c, int n_rows, int dtype, void* d_k, int64_t ld_k, void* d_v, int64_t ld_v,
                             const int32_t* d_seq, const int32_t* d_pos, void* stream) {
  KvPaged v;
  adept_status s = view_of(c, &v);
  if (s == ADEPT_OK) s = rows_ok(v, n_rows, dtype, d_k, ld_k, d_v, ld_v, d_seq, d_pos);
  if (s != ADEPT_OK || n_rows == 0) return s;
  PdlScope pdl(true);
  return launched(launch_kv_gather((cudaStream_t)stream, v, n_rows, dtype == ADEPT_DTYPE_BF16, d_k, ld_k, d_v, ld_v, d_seq, d_pos));
}

int64_t adept_chunk_attention_workspace(const adept_kv_cache* c, int n_heads, int n_rows, int max_q_len, int max_kv_len) {
  KvPaged v;
  if (view_of(c, &v) != ADEPT_OK || call_ok(v, n_heads, n_rows, max_q_len, max_kv_len) != ADEPT_OK) return -1;
  return (int64_t)chunk_workspace(v, n_heads, max_q_len, max_kv_len);
}

adept_status adept_chunk_attention(const adept_kv_cache* c, int n_heads, int n_rows, const void* d_q, int64_t ld_q,
                                   const int32_t* d_q_start, const int32_t* d_kv_len, const int32_t* d_row_pos,
                                   int max_q_len, int max_kv_len, void* d_out, int64_t ld_out, void* d_ws, int64_t ws_bytes, void* stream) {
  ChunkCall a{};
  adept_status s = view_of(c, &a.c);
  if (s == ADEPT_OK) s = call_ok(a.c, n_heads, n_rows, max_q_len, max_kv_len);
  if (s != ADEPT_OK) return s;
  if (n_rows == 0 || max_q_len == 0) return ADEPT_OK;
  if (!d_q || !d_out || !d_q_start || !d_kv_len) return bad(ADEPT_ERR_INVALID_ARG, "NULL device pointer");
  const int64_t w = (int64_t)n_heads * a.c.head_dim;
  if (ld_q < w || ld_out < w) return bad(ADEPT_ERR_INVALID_ARG, "row stride below the %lld elements of a row", (long long)w);
  const uintptr_t m = a.c.type == KV_F32 ? 3 : 1;
  if (((uintptr_t)d_q | (uintptr_t)d_out) & m) return bad(ADEPT_ERR_INVALID_ARG, "misaligned rows");
  if (((uintptr_t)d_q_start | (uintptr_t)d_kv_len | (uintptr_t)d_row_pos) & 3)
    return bad(ADEPT_ERR_INVALID_ARG, "misaligned lengths or positions");
  const int64_t need = (int64_t)chunk_workspace(a.c, n_heads, max_q_len, max_kv_len);
  if (need > 0 && (!d_ws || ws_bytes < need || ((uintptr_t)d_ws & 15)))
    return bad(ADEPT_ERR_INVALID_ARG, "workspace of %lld bytes, on 16 bytes, needed (adept_chunk_attention_workspace)", (long long)need);
  a.q = d_q;
  a.out = d_out;
  a.ld_q = ld_q;
  a.ld_out = ld_out;
  a.q_start = d_q_start;
  a.kv_len = d_kv_len;
  a.row_pos = d_row_pos;
  a.n_rows = n_rows;
  a.n_heads = n_heads;
  a.max_q = max_q_len;
  a.max_kv = max_kv_len;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)a.c.head_dim);
  a.part = (float*)d_ws;
  PdlScope pdl(true);
  int launches = 0;
  return launched(launch_chunk_attention((cudaStream_t)stream, a, &launches));
}

adept_status adept_kv_check(const adept_kv_cache* c, void* stream) {
  KvPaged v;
  const adept_status s = view_of(c, &v);
  if (s != ADEPT_OK) return s;
  if (!v.err) return bad(ADEPT_ERR_INVALID_ARG, "the cache has no error word");
  cudaStream_t st = (cudaStream_t)stream;
  cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
  cudaError_t e = cudaStreamIsCapturing(st, &cap);
  if (e == cudaSuccess && cap != cudaStreamCaptureStatusNone)
    return bad(ADEPT_ERR_INVALID_ARG, "a check waits for its stream, which cannot be captured into a graph");
  unsigned w = 0;
  if (e == cudaSuccess) e = take_error_word(st, v.err, &w);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return bad(ADEPT_ERR_CUDA, "reading the error word: %s", cudaGetErrorString(e));
  }
  if (w & ERRW_TIMEOUT) return bad(ADEPT_ERR_TIMEOUT, "a device-side wait timed out (word 0x%x)", w);
  if (w) return bad(ADEPT_ERR_DEVICE_INPUT, "device-side input check failed (word 0x%x)", w);
  return ADEPT_OK;
}

}  // extern "C"
