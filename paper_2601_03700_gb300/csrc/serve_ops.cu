// C ABI of the pages behind a paged K/V cache and of the verification of drafted tokens: checks of the arguments, then one or two
// launches on the caller's stream.  The calls hold no state and allocate nothing.
#include "serve_ops.h"
#include "kernels.h"
#include "op_status.h"

using namespace adept;

namespace {

adept_status pages_of(const adept_kv_pages* p, Pages* v) {
  if (!p) return bad(ADEPT_ERR_INVALID_ARG, "NULL pages");
  if (p->n_blocks < 1 || p->block_tokens < 1 || p->n_seq < 1 || p->max_blocks_per_seq < 1)
    return bad(ADEPT_ERR_INVALID_ARG, "non-positive size of the pages");
  if ((long long)p->max_blocks_per_seq * p->block_tokens > (1ll << 30))
    return bad(ADEPT_ERR_INVALID_ARG, "rows too long (2^30 positions)");
  if (p->n_blocks > (1 << 30)) return bad(ADEPT_ERR_INVALID_ARG, "n_blocks %d above 2^30", p->n_blocks);
  if (!p->d_block_table || !p->d_ref) return bad(ADEPT_ERR_INVALID_ARG, "NULL block table or counts");
  if (((uintptr_t)p->d_block_table | (uintptr_t)p->d_err) & 3) return bad(ADEPT_ERR_INVALID_ARG, "misaligned block table or error word");
  if ((uintptr_t)p->d_ref & 15) return bad(ADEPT_ERR_INVALID_ARG, "the counts must start on 16 bytes");
  *v = Pages{p->d_block_table, p->d_ref, p->d_err, p->n_blocks, p->block_tokens, p->n_seq, p->max_blocks_per_seq};
  return ADEPT_OK;
}

adept_status pages_ws(const Pages& p, const void* ws, int64_t bytes) {
  const int64_t need = (int64_t)pages_workspace(p);
  if (!ws || bytes < need || ((uintptr_t)ws & 15))
    return bad(ADEPT_ERR_INVALID_ARG, "workspace of %lld bytes, on 16 bytes, needed (adept_kv_pages_workspace)", (long long)need);
  return ADEPT_OK;
}

}  // namespace

extern "C" {

int64_t adept_kv_pages_workspace(const adept_kv_pages* p) {
  Pages v;
  return pages_of(p, &v) == ADEPT_OK ? (int64_t)pages_workspace(v) : -1;
}

adept_status adept_kv_fork(const adept_kv_pages* p, const int32_t* d_source, const int32_t* d_length, void* d_ws, int64_t ws_bytes,
                           void* stream) {
  Pages v;
  adept_status s = pages_of(p, &v);
  if (s == ADEPT_OK) s = pages_ws(v, d_ws, ws_bytes);
  if (s != ADEPT_OK) return s;
  if (!d_source || !d_length) return bad(ADEPT_ERR_INVALID_ARG, "NULL device pointer");
  if (((uintptr_t)d_source | (uintptr_t)d_length) & 3) return bad(ADEPT_ERR_INVALID_ARG, "misaligned rows or lengths");
  PdlScope pdl(true);
  return launched(launch_kv_fork((cudaStream_t)stream, v, d_source, d_length, (int*)d_ws));
}

adept_status adept_kv_reserve(const adept_kv_pages* p, const int32_t* d_length, const int32_t* d_new_length, int32_t* d_got,
                              int32_t* d_copy_src, int32_t* d_copy_dst, void* d_ws, int64_t ws_bytes, void* stream) {
  Pages v;
  adept_status s = pages_of(p, &v);
  if (s == ADEPT_OK) s = pages_ws(v, d_ws, ws_bytes);
  if (s != ADEPT_OK) return s;
  if (v.n_seq > PG_MAX_SEQ) return bad(ADEPT_ERR_CAPACITY, "%d rows: adept_kv_reserve takes up to %d", v.n_seq, PG_MAX_SEQ);
  if (!d_length || !d_new_length || !d_got || !d_copy_src || !d_copy_dst) return bad(ADEPT_ERR_INVALID_ARG, "NULL device pointer");
  if (((uintptr_t)d_length | (uintptr_t)d_new_length | (uintptr_t)d_got | (uintptr_t)d_copy_src | (uintptr_t)d_copy_dst) & 3)
    return bad(ADEPT_ERR_INVALID_ARG, "misaligned lengths or blocks");
  PdlScope pdl(true);
  return launched(launch_kv_reserve((cudaStream_t)stream, v, d_length, d_new_length, d_got, d_copy_src, d_copy_dst, (int*)d_ws));
}

adept_status adept_kv_compact(const adept_kv_pages* p, int32_t* d_used, int32_t* d_copy_src, int32_t* d_copy_dst, void* d_ws,
                              int64_t ws_bytes, void* stream) {
  Pages v;
  adept_status s = pages_of(p, &v);
  if (s == ADEPT_OK) s = pages_ws(v, d_ws, ws_bytes);
  if (s != ADEPT_OK) return s;
  if (!d_used || (v.n_blocks > 1 && (!d_copy_src || !d_copy_dst))) return bad(ADEPT_ERR_INVALID_ARG, "NULL device pointer");
  if (((uintptr_t)d_used | (uintptr_t)d_copy_src | (uintptr_t)d_copy_dst) & 3) return bad(ADEPT_ERR_INVALID_ARG, "misaligned count or blocks");
  PdlScope pdl(true);
  return launched(launch_kv_compact((cudaStream_t)stream, v, d_used, d_copy_src, d_copy_dst, (int*)d_ws));
}

adept_status adept_kv_copy_blocks(const adept_kv_cache* caches, int n_caches, int n_pairs, const int32_t* d_src, const int32_t* d_dst,
                                  void* stream) {
  if (!caches || n_caches < 1) return bad(ADEPT_ERR_INVALID_ARG, "no cache");
  if (n_pairs < 0) return bad(ADEPT_ERR_INVALID_ARG, "n_pairs %d < 0", n_pairs);
  KvPaged first;
  for (int i = 0; i < n_caches; ++i) {   // all before anything is enqueued
    KvPaged v;
    const adept_status s = view_of(caches + i, &v);
    if (s != ADEPT_OK) return s;
    if (i == 0) first = v;
    if (v.type != first.type || v.n_blocks != first.n_blocks || v.n_kv_heads != first.n_kv_heads || v.head_dim != first.head_dim ||
        v.block_tokens != first.block_tokens)
      return bad(ADEPT_ERR_INVALID_ARG, "cache %d has blocks of another kind or number than the first", i);
  }
  if (n_pairs == 0) return ADEPT_OK;
  if (!d_src || !d_dst) return bad(ADEPT_ERR_INVALID_ARG, "NULL device pointer");
  if (((uintptr_t)d_src | (uintptr_t)d_dst) & 3) return bad(ADEPT_ERR_INVALID_ARG, "misaligned blocks");
  PdlScope pdl(true);
  for (int i0 = 0; i0 < n_caches; i0 += CP_LAYERS) {
    CopyLayers c{};
    c.n_layers = n_caches - i0 < CP_LAYERS ? n_caches - i0 : CP_LAYERS;
    for (int i = 0; i < c.n_layers; ++i) {
      const adept_kv_cache& k = caches[i0 + i];
      c.k[i] = k.d_k;
      c.v[i] = k.d_v;
      c.k_exp[i] = k.d_k_exp;
      c.v_exp[i] = k.d_v_exp;
    }
    const long long entries = (long long)first.n_kv_heads * first.block_tokens;
    c.err = first.err;
    c.n_blocks = first.n_blocks;
    c.block_bytes = entries * first.head_dim * (first.type == KV_F32 ? 4 : first.type == KV_BF16 ? 2 : 1);
    c.exp_bytes = first.type == KV_E4M3 ? entries : 0;
    const adept_status s = launched(launch_kv_copy_blocks((cudaStream_t)stream, c, n_pairs, d_src, d_dst));
    if (s != ADEPT_OK) return s;
  }
  return ADEPT_OK;
}

int64_t adept_verify_workspace(int n_rows) {
  if (n_rows < 0 || n_rows > (1 << 24)) {
    bad(ADEPT_ERR_INVALID_ARG, "n_rows %d outside 0 .. 2^24", n_rows);
    return -1;
  }
  return (int64_t)verify_workspace(n_rows);
}

adept_status adept_verify_drafts(int n_seq, int n_rows, int vocab, int target_dtype, const void* d_target, int64_t ld_target,
                                 int draft_dtype, const void* d_draft, int64_t ld_draft, const int32_t* d_tokens,
                                 const int32_t* d_start, const float* d_temperature, const float* d_u, int32_t* d_accepted,
                                 int32_t* d_next, float* d_logprob, uint32_t* d_err, void* d_ws, int64_t ws_bytes, void* stream) {
  if (n_seq < 0 || n_rows < 0) return bad(ADEPT_ERR_INVALID_ARG, "negative size");
  if (vocab < 1 || vocab > (1 << 20)) return bad(ADEPT_ERR_INVALID_ARG, "vocab %d outside 1 .. 2^20", vocab);
  // (every row looks for its sequence among all)
  if (n_rows > (1 << 24) || n_seq > (1 << 16)) return bad(ADEPT_ERR_CAPACITY, "more than 2^24 rows or 2^16 sequences");
  for (const int dt : {target_dtype, draft_dtype})
    if (dt != ADEPT_DTYPE_F32 && dt != ADEPT_DTYPE_BF16) return bad(ADEPT_ERR_INVALID_ARG, "dtype %d unknown", dt);
  if (n_seq == 0) return ADEPT_OK;
  if (!d_start || !d_accepted || !d_next) return bad(ADEPT_ERR_INVALID_ARG, "NULL device pointer");
  if (n_rows > 0) {
    if (!d_target || !d_tokens || !d_u) return bad(ADEPT_ERR_INVALID_ARG, "NULL device pointer");
    if (ld_target < vocab || (d_draft && ld_draft < vocab)) return bad(ADEPT_ERR_INVALID_ARG, "row stride below the vocabulary");
    if (((uintptr_t)d_target & (target_dtype == ADEPT_DTYPE_BF16 ? 1 : 3)) || ((uintptr_t)d_draft & (draft_dtype == ADEPT_DTYPE_BF16 ? 1 : 3)))
      return bad(ADEPT_ERR_INVALID_ARG, "misaligned logits");
    const int64_t need = (int64_t)verify_workspace(n_rows);
    if (!d_ws || ws_bytes < need || ((uintptr_t)d_ws & 15))
      return bad(ADEPT_ERR_INVALID_ARG, "workspace of %lld bytes, on 16 bytes, needed (adept_verify_workspace)", (long long)need);
  }
  if (((uintptr_t)d_tokens | (uintptr_t)d_start | (uintptr_t)d_temperature | (uintptr_t)d_u | (uintptr_t)d_accepted |
       (uintptr_t)d_next | (uintptr_t)d_logprob | (uintptr_t)d_err) & 3)
    return bad(ADEPT_ERR_INVALID_ARG, "misaligned tokens, numbers or results");
  VerifyCall a{n_seq, n_rows, vocab, target_dtype == ADEPT_DTYPE_BF16, draft_dtype == ADEPT_DTYPE_BF16, d_target, d_draft, ld_target,
               ld_draft, d_tokens, d_start, d_temperature, d_u, d_accepted, d_next, d_logprob, d_err, d_ws};
  PdlScope pdl(true);
  return launched(launch_verify((cudaStream_t)stream, a));
}

adept_status adept_error_check(uint32_t* d_err, void* stream) {
  if (!d_err || ((uintptr_t)d_err & 3)) return bad(ADEPT_ERR_INVALID_ARG, "NULL or misaligned error word");
  cudaStream_t st = (cudaStream_t)stream;
  cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
  cudaError_t e = cudaStreamIsCapturing(st, &cap);
  if (e == cudaSuccess && cap != cudaStreamCaptureStatusNone)
    return bad(ADEPT_ERR_INVALID_ARG, "a check waits for its stream, which cannot be captured into a graph");
  unsigned w = 0;
  if (e == cudaSuccess) e = take_error_word(st, d_err, &w);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return bad(ADEPT_ERR_CUDA, "reading the error word: %s", cudaGetErrorString(e));
  }
  if (w & ERRW_TIMEOUT) return bad(ADEPT_ERR_TIMEOUT, "a device-side wait timed out (word 0x%x)", w);
  if (w) return bad(ADEPT_ERR_DEVICE_INPUT, "device-side input check failed (word 0x%x)", w);
  return ADEPT_OK;
}

}  // extern "C"
