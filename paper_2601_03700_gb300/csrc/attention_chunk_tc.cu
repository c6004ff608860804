// Launches of the tcgen05 chunk attention (attention_chunk_tc.cuh): what it takes, its workspace, its launches.
#define ADEPT_TU_ID 13
#include "attention_chunk_tc.cuh"
#include "gemm_tc.h"

#include <algorithm>
#include <cstring>

namespace adept {
namespace {

int ct_sms() {
  static const int sms = [] {
    int dev = 0, n = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    return std::max(1, n);
  }();
  return sms;
}

// Workspace: the parts, a word for time-outs, the widened K and V.
size_t ct_parts_bytes(int dh) { return (ct_ws_floats(ct_sms(), dh) * 4 + 16 + 255) / 256 * 256; }
// Widened entries lie as their blocks lie in the pool, or, where the call's sequences can hold fewer blocks than the pool has, in
// order of (sequence, block): blocks per sequence then, else 0.  Never more than the pool, so that every size here grows with
// n_seq and max_kv (a model takes its workspace once, for the largest of both).
int ct_wide(const KvPaged& c, int max_kv) {
  const long long per = cdiv(max_kv, 16);
  return (long long)c.n_seq * per < c.n_blocks ? (int)per : 0;
}
size_t ct_wide_blocks(const KvPaged& c, int max_kv) {
  const int per = ct_wide(c, max_kv);
  return per ? (size_t)c.n_seq * per : (size_t)c.n_blocks;
}
size_t ct_wide_bytes(const KvPaged& c, int max_kv) {   // of K, or of V
  return c.type == KV_E4M3 ? ct_wide_blocks(c, max_kv) * c.n_kv_heads * 16 * c.head_dim * 2 : 0;
}

void* wide_k(const ChunkCall& a) { return (char*)a.part + ct_parts_bytes(a.c.head_dim); }
void* wide_v(const ChunkCall& a) { return (char*)wide_k(a) + ct_wide_bytes(a.c, a.max_kv); }

template <int DH>
cudaError_t launch_t(cudaStream_t st, CtParams& p, int* launches) {
  constexpr int smem = CtShape<DH>::TOTAL + 1024;
  const KvPaged& c = p.a.c;
  cudaError_t e = smem_once<CtShape<DH>>(chunk_tc_kernel<DH>, smem);
  if (e != cudaSuccess) return e;
  void *k = c.k, *v = c.v;
  uint64_t rows = (uint64_t)c.n_blocks * c.n_kv_heads * 16;
  if (c.type == KV_E4M3) {
    p.wide = ct_wide(c, p.a.max_kv);
    rows = (uint64_t)ct_wide_blocks(c, p.a.max_kv) * c.n_kv_heads * 16;
    k = wide_k(p.a);
    v = wide_v(p.a);
  }
  const uint64_t kv_dims[2] = {DH, rows}, kv_strides[1] = {DH * 2};
  const uint64_t q_dims[3] = {DH, (uint64_t)p.a.n_heads, (uint64_t)p.a.n_rows}, q_strides[2] = {DH * 2, (uint64_t)p.a.ld_q * 2};
  const uint32_t kv_box[2] = {64, 16}, q_box[3] = {64, (uint32_t)(p.a.n_heads / c.n_kv_heads), (uint32_t)p.ts};
  if (!tc_encode_plain(&p.kmap, k, 2, kv_dims, kv_strides, kv_box) || !tc_encode_plain(&p.vmap, v, 2, kv_dims, kv_strides, kv_box) ||
      !tc_encode_plain(&p.qmap, p.a.q, 3, q_dims, q_strides, q_box))
    return cudaErrorInvalidValue;
  e = launch_k(chunk_tc_kernel<DH>, dim3(p.runs), dim3(CtShape<DH>::THREADS), smem, st, p);
  if (e != cudaSuccess) return e;
  *launches += 2;
  return launch_k(chunk_tc_join_kernel<DH>, dim3(std::max(1, p.runs - 1), CJ_SPLIT), dim3(256), 0, st, p);
}

}  // namespace

bool chunk_tc_takes(const KvPaged& c, int n_heads) {
  return c.type != KV_F32 && c.block_tokens == 16 && (c.head_dim == 64 || c.head_dim == 128) &&
         n_heads / c.n_kv_heads <= CT_BM && (long long)c.n_blocks * c.n_kv_heads * 16 < (1ll << 31);
}

size_t chunk_tc_workspace(const KvPaged& c, int max_kv) { return ct_parts_bytes(c.head_dim) + 2 * ct_wide_bytes(c, max_kv); }

bool chunk_tc_fits(const KvPaged& c, int n_heads, int n_rows, int max_q, int max_kv) {
  const long long tq = 2 * (CT_BM / (n_heads / c.n_kv_heads));
  const long long tiles = std::min(c.n_seq * ((max_q + tq - 1) / tq), n_rows / tq + c.n_seq);
  return tiles * c.n_kv_heads * (CT_TILE + cdiv(max_kv, CT_BN)) < (1ll << 31);
}

cudaError_t launch_chunk_widen(cudaStream_t st, const ChunkCall& a, int* launches) {
  const int wide = ct_wide(a.c, a.max_kv);
  const dim3 grid((unsigned)std::min<long long>(ct_sms() * 8, 2ll * cdiv(a.max_kv, 16) * a.c.n_seq));
  ++*launches;
  return launch_k(a.c.head_dim == 128 ? chunk_widen_kernel<128> : chunk_widen_kernel<64>, grid, dim3(CW_THREADS), 0, st, a, wide,
                  (bf16*)wide_k(a), (bf16*)wide_v(a));
}

cudaError_t launch_chunk_tc(cudaStream_t st, const ChunkCall& a, int* launches) {
  CtParams p;
  memset(&p, 0, sizeof p);
  p.a = a;
  p.ts = CT_BM / (a.n_heads / a.c.n_kv_heads);
  p.runs = ct_sms();
  p.no_err = (unsigned*)(a.part + ct_ws_floats(p.runs, a.c.head_dim));
  return a.c.head_dim == 128 ? launch_t<128>(st, p, launches) : launch_t<64>(st, p, launches);
}

ADEPT_WAIT_LIMIT_SETTER(ct)

}  // namespace adept
