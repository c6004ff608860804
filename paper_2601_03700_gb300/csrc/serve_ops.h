// Operators around a paged K/V cache that serving needs (serve_ops.cu holds their C ABI): the pages behind the sequences
// (kv_pages.cu) and the verification of drafted tokens (verify.cu).
#pragma once
#include "common.cuh"
#include "kv_paged.h"

namespace adept {

// A block table that its owner's calls change, and per block the number of rows that hold it (0: free).
struct Pages {
  int* table;      // [n_seq][max_blocks], -1: no block
  int* ref;        // [n_blocks]
  unsigned* err;   // error word (NULL: none)
  int n_blocks, block_tokens, n_seq, max_blocks;
  __device__ __forceinline__ void flag(unsigned bits) const {
    if (err) atomicOr(err, bits);
  }
};
constexpr int PG_MAX_SEQ = 4096;   // rows of a call of launch_kv_reserve

size_t pages_workspace(const Pages& p);   // bytes of ws that any of the three calls needs
cudaError_t launch_kv_fork(cudaStream_t st, const Pages& p, const int* source, const int* length, int* ws);
cudaError_t launch_kv_reserve(cudaStream_t st, const Pages& p, const int* length, const int* want, int* got, int* src, int* dst,
                              int* ws);
cudaError_t launch_kv_compact(cudaStream_t st, const Pages& p, int* used, int* src, int* dst, int* ws);

// Blocks src[i] to dst[i] of every layer's K and V (and exponents), all layers of one geometry.
constexpr int CP_LAYERS = 32;   // of one launch
struct CopyLayers {
  void* k[CP_LAYERS];
  void* v[CP_LAYERS];
  uint8_t* k_exp[CP_LAYERS];
  uint8_t* v_exp[CP_LAYERS];
  unsigned* err;
  int n_layers, n_blocks, exp_bytes;   // exp_bytes: of a block's exponents (0: none)
  long long block_bytes;               // of a block's K
};
cudaError_t launch_kv_copy_blocks(cudaStream_t st, const CopyLayers& c, int n_pairs, const int* src, const int* dst);

// One verification call: sequence b's rows start[b] .. start[b + 1] - 1 of the target's logits; row r's distribution follows
// token tokens[r], and tokens[r + 1] is the draft that it is held against (none behind the sequence's last row).
struct VerifyCall {
  int n_seq, n_rows, vocab;
  int t_bf16, d_bf16;
  const void* target;   // [n_rows][ld_t]
  const void* draft;    // [n_rows][ld_d] or NULL: drafts are certain
  long long ld_t, ld_d;
  const int* tokens;    // [n_rows]
  const int* start;     // [n_seq + 1]
  const float* temp;    // [n_seq] or NULL: 1
  const float* u;       // [n_rows]
  int* accepted;        // [n_seq]
  int* next;            // [n_seq]
  float* logprob;       // [n_rows] or NULL
  unsigned* err;
  void* ws;
  __device__ __forceinline__ void flag(unsigned bits) const {
    if (err) atomicOr(err, bits);
  }
};
size_t verify_workspace(int n_rows);   // bytes of ws; no smaller call needs more
cudaError_t launch_verify(cudaStream_t st, const VerifyCall& a);

}  // namespace adept
