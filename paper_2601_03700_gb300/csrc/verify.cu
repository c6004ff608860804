// Drafted tokens against the target's logits.
//
// Row r of a sequence holds the target's logits behind token tokens[r]; p_r = softmax(l_r / T), q_r the draft's.  Draft x =
// tokens[r + 1] holds where log u_r + log q_r(x) < log p_r(x); at the first row whose draft does not, the next token is drawn from
// max(p_r - q_r, 0), at the last row from p_r.
//
// Two launches.  The first streams every row once, each in parts of a CTA, and leaves per part the maximum, the sum of exp((l - max) / T), the
// maximum's first index (greedy sequences) and the draft's logit: HBM-bound, 437 MB at 6.2 TB/s (64 chunks of 8 drafts over 131072
// tokens, fp32 and bf16).  The second, a cluster per sequence, decides.  Sums of 32 bits decide a draft unless the two sides are closer
// than their errors (close_of); those, and the drawing, go by weights of two 32-bit parts each (2^-37 relative at most): with a vocabulary of
// V tokens the cumulative sum has V steps, and an error of 2^-24 would move the drawn token with odds of V 2^-23.  It reads one row of
// the target and one of the draft a sequence, most of it from L2, and is bound by the weights' arithmetic (about 40 operations a
// weight) where there are many sequences, by the chain loads -> sums -> barrier -> sums where there are few.  One launch, in which a
// cluster takes its rows' statistics as well, was no faster: one chunk of 4 drafts over 50257 tokens 15.8 us where two took 14.7.
#include "cluster.cuh"
#include "serve_ops.h"

#include <float.h>

namespace adept {
namespace {

constexpr int VS_THREADS = 128, VS_LOADS = 4, VS_PARTS = 8;   // statistics: 16-byte loads of a thread under way (twice), CTAs of a row at most
constexpr float VS_HUGE = 1e6f;
constexpr int VD_THREADS = 512, VD_CTAS = 16;    // decision: threads of a CTA, CTAs of a sequence at most
constexpr int VD_MANY = 32;                      // tokens a thread from which on it takes four at a time, else two
constexpr int VD_LEAST = 20;                     // max(p - q, 0) sums to less than 2^-this: the token is drawn from p
constexpr int VD_FINE = 14;                      // to less than 2^-this (or p without the draft): summed token by token
constexpr float VD_NEAR = 3.814697265625e-06f;   // 2^-18: p and q nearer than this may be taken for either above the other
constexpr float VD_SURE = 5.820766091346741e-11f;   // 2^-34: what that may make of the sum, else those tokens are looked at again
constexpr int VD_NEARS = 64;                     // as many as a CTA remembers; with more, the sum is taken token by token
constexpr long long VD_NOTHING = 1 << 14;        // of the sums' 2^-58: what rounding leaves of nothing
constexpr int VD_TAB = 64;

// Difference of the logarithms of a test's two sides below which 32-bit sums do not decide it.  A sum's error: a thread's
// chain of additions and rescalings, one for each of its 16-byte pieces, 2^-22 each; the exponents, rounded in three places 2^-24 of up to
// log2 V + 2 units on average; 20 more for the joins.  Two sums, and three logarithms of 2^-23 of up to log V or log 2^-24.
__device__ __forceinline__ float close_of(int vocab, int parts) {
  return 2 * 2.384185791015625e-07f * (vocab / (4 * VS_THREADS * parts) + 1 + 22 + 20 + 12);
}

struct Stat {
  float m, z;   // maximum; sum of exp((l - m) / T)
  int at;       // first index of the maximum (greedy sequences)
  float l;      // the row's first part: the logit of the token that is held against it
};

__device__ __forceinline__ bool temp_ok(float t) { return t == 0.f || (t >= 9.765625e-4f && t <= 1024.f); }

// Sequence b's rows, false: out of range (or none).
struct SeqRows {
  int s, e;
  bool ok;
};
__device__ __forceinline__ SeqRows seq_rows(const VerifyCall& a, int b) {
  SeqRows r;
  r.s = a.start[b];
  r.e = a.start[b + 1];
  r.ok = r.s >= 0 && r.e >= r.s && r.e <= a.n_rows;
  return r;
}

// 16 bytes of logits.
template <typename T>
struct Vec {
  static constexpr int N = 16 / (int)sizeof(T);
  static __device__ __forceinline__ uint4 none() {   // -infinity
    const uint32_t w = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    return make_uint4(w, w, w, w);
  }
  static __device__ __forceinline__ float at(const uint4& v, int i) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
  }
};

// Maximum so far and z = sum of 2^(l c - M) with M = m c as fp32 has it: one fused operation, one exponential and one addition an
// element.  What M's rounding makes of z (off) is a factor that all its terms have.  Where |m c| is large M is m c itself.
struct Running {
  float m = -INFINITY, z = 0.f;
  int at = -1;   // where the maximum was first met (what add was given; joined: any of them)
  static __device__ __forceinline__ float off(float m, float c) {
    const float M = __fmul_rn(m, c);
    return fabsf(M) < VS_HUGE ? __fmaf_rn(m, c, -M) : 0.f;
  }
  __device__ __forceinline__ void raise(float to, float c) {
    if (m != -INFINITY) z *= ex2_approx((m - to) * c - off(m, c) + off(to, c));   // (else z is 0, or NaN)
    m = to;
  }
  __device__ __forceinline__ void join(float om, float oz, float c) {
    if (om > m) raise(om, c);
    z += om == -INFINITY ? oz : oz * ex2_approx((om - m) * c - off(om, c) + off(m, c));
  }
  template <typename T, int L>   // L 16-byte pieces
  __device__ __forceinline__ void add(const uint4 (&w)[L], int i0, float c) {
    using V = Vec<T>;
    float g = -INFINITY;
#pragma unroll
    for (int i = 0; i < L; ++i)
#pragma unroll
      for (int k = 0; k < V::N; ++k) g = fmaxf(g, V::at(w[i], k));
    if (g > m) {
      raise(g, c);
      at = i0;
    }
    float s = 0.f;
    const float M = __fmul_rn(m, c);
    if (fabsf(M) < VS_HUGE) {
#pragma unroll
      for (int i = 0; i < L; ++i)
#pragma unroll
        for (int k = 0; k < V::N; ++k) s += ex2_approx(__fmaf_rn(V::at(w[i], k), c, -M));
    } else {   // (or nothing above -infinity was there yet)
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int i = 0; i < L; ++i)
#pragma unroll
        for (int k = 0; k < V::N; ++k) s += ex2_approx((V::at(w[i], k) - ref) * c);
    }
    z += s;
  }
};

// Statistics of part blockIdx.x % parts of row blockIdx.x / parts, the target's (blockIdx.y = 0) or the draft's, for the first sequence that
// names the row: *owner.
template <typename T>
__device__ __forceinline__ void row_stats(const VerifyCall& a, const T* x, bool draft, int r, int part, int parts, Stat* out, int* owner) {
  using V = Vec<T>;
  __shared__ int s_seq, s_at;
  __shared__ float s_m[VS_THREADS / 32], s_z[VS_THREADS / 32];
  const int tid = threadIdx.x, lane = tid & 31, n = a.vocab;
  // elements before the first 16-byte boundary, 16-byte pieces, the rest
  const int head = min(n, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T));
  const int nv = (n - head) / V::N, v0 = (int)((long long)nv * part / parts), v1 = (int)((long long)nv * (part + 1) / parts);
  const uint4* body = reinterpret_cast<const uint4*>(x + head);
  auto load = [&](int v, uint4 (&w)[VS_LOADS]) {
#pragma unroll
    for (int i = 0; i < VS_LOADS; ++i) w[i] = v + i * VS_THREADS < v1 ? __ldcs(body + v + i * VS_THREADS) : V::none();
  };
  // the first loads are under way while the row's sequence is looked up
  int v = v0 + tid;
  uint4 w[VS_LOADS];
  load(v, w);
  uint4 ends[1] = {V::none()};   // what lies beside the 16-byte pieces: an element each
  const int past = head + nv * V::N + tid - 32;
  const bool first = part == 0 && tid < head, last = part == parts - 1 && tid >= 32 && past < n;
  int end_at = first ? tid : past;
  if (first || last) ends[0].x = sizeof(T) == 4 ? *reinterpret_cast<const uint32_t*>(x + end_at) : 0xff800000u | *reinterpret_cast<const uint16_t*>(x + end_at);
  int id = -1;   // the token that the row's distribution is held against
  if (tid == 0) {
    s_seq = 0x7fffffff;
    if (part == 0 && r + 1 < a.n_rows) id = a.tokens[r + 1];
  }
  __syncthreads();
  for (int b = tid; b < a.n_seq; b += VS_THREADS) {
    const SeqRows q = seq_rows(a, b);
    if (q.ok && q.s <= r && r < q.e) atomicMin(&s_seq, b);
  }
  const float held = id >= 0 && id < n ? to_f<T>(x[id]) : -INFINITY;
  __syncthreads();
  if (!draft && part == 0 && tid == 0) *owner = s_seq;
  if (s_seq == 0x7fffffff) return;   // nobody's row
  const float t = a.temp ? a.temp[s_seq] : 1.f;
  if (!temp_ok(t)) return;
  if (draft && (t == 0.f || r == a.start[s_seq + 1] - 1)) return;   // a draft row that nothing is held against
  const float c = 1.44269504088896f / (t == 0.f ? 1.f : t);   // (a greedy sequence has the probabilities of T = 1)
  Running run;
  if (first) run.add<T>(ends, -2, c);
  while (v < v1) {   // the next loads under way before these are used
    uint4 next[VS_LOADS];
    const int u = v + VS_LOADS * VS_THREADS;
    load(u, next);
    run.add<T>(w, v, c);
#pragma unroll
    for (int i = 0; i < VS_LOADS; ++i) w[i] = next[i];
    v = u;
  }
  if (last) run.add<T>(ends, -2, c);
  const float mine = run.m;
  auto warp_join = [&](int o0) {
    for (int o = o0; o; o >>= 1) run.join(__shfl_xor_sync(0xffffffffu, run.m, o), __shfl_xor_sync(0xffffffffu, run.z, o), c);
  };
  const int where = run.at;
  warp_join(16);
  if (lane == 0) {
    s_m[tid >> 5] = run.m;
    s_z[tid >> 5] = run.z;
  }
  if (tid == 0) s_at = 0x7fffffff;
  __syncthreads();
  run.m = s_m[lane % (VS_THREADS / 32)];
  run.z = s_z[lane % (VS_THREADS / 32)];
  warp_join(VS_THREADS / 64);
  if (t == 0.f) {   // (uniform) the first index of the maximum: the threads that met it look at those pieces again
    if (mine == run.m) {
      if (where == -2) {
        atomicMin(&s_at, end_at);
      } else if (where >= 0) {
        load(where, w);
#pragma unroll
        for (int i = VS_LOADS - 1; i >= 0; --i)
#pragma unroll
          for (int k = V::N - 1; k >= 0; --k)
            if (V::at(w[i], k) == mine) end_at = head + (where + i * VS_THREADS) * V::N + k;
        atomicMin(&s_at, end_at);
      }
    }
    __syncthreads();
  }
  if (tid == 0) *out = Stat{run.m, run.z * ex2_approx(-Running::off(run.m, c)), s_at, held};
}

template <typename TT, typename TD>
__global__ void __launch_bounds__(VS_THREADS, 8) verify_stats_kernel(VerifyCall a, int parts, Stat* stats, int* owner) {
  PDL_ENTRY();
  const int r = (int)blockIdx.x / parts, part = (int)blockIdx.x % parts;
  Stat* out = stats + ((size_t)blockIdx.y * a.n_rows + r) * parts + part;
  if (blockIdx.y == 0)
    row_stats(a, (const TT*)a.target + r * a.ld_t, false, r, part, parts, out, owner + r);
  else
    row_stats(a, (const TD*)a.draft + r * a.ld_d, true, r, part, parts, out, nullptr);
}

// ---------------------------------------------------------------------------------------------
// Numbers of two 32-bit parts, h + l with |l| at most half a step of h: about 2^-46 relative.  64-bit arithmetic runs at
// two operations a cycle and SM here: with the sums and the joins in it a call of one chunk of 4 drafts over 50257 tokens took 54 us,
// without it 25.
// ---------------------------------------------------------------------------------------------
struct Two {
  float h, l;
};
__device__ __forceinline__ Two norm2(float h, float l) {   // |l| <= |h|, or h = 0
  const float s = __fadd_rn(h, l);
  return Two{s, __fsub_rn(l, __fsub_rn(s, h))};
}
// a + b = s + e (Knuth)
__device__ __forceinline__ Two sum_of(float a, float b) {
  const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
  return Two{s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Two operator+(Two a, Two b) {
  const Two s = sum_of(a.h, b.h);
  return norm2(s.h, __fadd_rn(s.l, __fadd_rn(a.l, b.l)));
}
__device__ __forceinline__ Two operator*(Two a, Two b) {
  const float p = __fmul_rn(a.h, b.h);
  return norm2(p, __fmaf_rn(a.h, b.h, -p) + __fmaf_rn(a.h, b.l, a.l * b.h));
}
__device__ __forceinline__ Two operator/(Two a, Two b) {   // (one step of division by the first part, then of the remainder)
  const float q = __fdiv_rn(a.h, b.h);
  const float p = __fmul_rn(q, b.h), e = __fmaf_rn(q, b.h, -p);
  const float r = __fsub_rn(a.h, p) - e + __fmaf_rn(-q, b.l, a.l);
  return norm2(q, __fdiv_rn(r, b.h));
}

// Sums over threads in whole numbers, so that any order gives the same: of 2^-58 times the power of two in the row's sum of weights,
// as the 32-bit sums have it.
__device__ __forceinline__ float unit_of(float z) { return __uint_as_float((312u << 23) - (__float_as_uint(z) & 0x7f800000u)); }   // in one
__device__ __forceinline__ long long whole(Two v, float unit) { return max(__float2ll_rn(v.h * unit) + __float2ll_rn(v.l * unit), 0ll); }
__device__ __forceinline__ long long warp_sum(long long v) {   // 0 <= v < 2^61, the sum below 2^62
  constexpr unsigned M = (1u << 27) - 1;
  const unsigned a = __reduce_add_sync(0xffffffffu, (unsigned)v & M), b = __reduce_add_sync(0xffffffffu, (unsigned)(v >> 27) & M),
                 c = __reduce_add_sync(0xffffffffu, (unsigned)(v >> 54));
  return (long long)a + ((long long)b << 27) + ((long long)c << 54);
}
__device__ __forceinline__ Two two_of(long long v) {
  const float h = __ll2float_rn(v);
  return Two{h, __ll2float_rn(v - __float2ll_rn(h))};
}
// a / b to 2^-44: one step of division by the first part, then of the remainder
__device__ __forceinline__ Two quotient(Two a, Two b) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(b.h));
  const float q = a.h * r;
  return norm2(q, r * (__fmaf_rn(-q, b.h, a.h) + __fmaf_rn(-q, b.l, a.l)));
}

// 2^(k / 64) in two parts; a CTA's copy.
struct VdTab {
  float h[VD_TAB], l[VD_TAB];
};
__device__ const float2 VD_POW[VD_TAB] = {
    {0x1.0000000000000p+0f, 0x0.0p+0f}, {0x1.02c9a40000000p+0f, -0x1.887fa00000000p-28f},
    {0x1.059b0e0000000p+0f, -0x1.9d4f520000000p-25f}, {0x1.0874520000000p+0f, -0x1.e2990e0000000p-26f},
    {0x1.0b55860000000p+0f, 0x1.9f31220000000p-25f}, {0x1.0e3ec40000000p+0f, -0x1.a585cc0000000p-25f},
    {0x1.11301e0000000p+0f, -0x1.fdb4960000000p-25f}, {0x1.1429aa0000000p+0f, 0x1.d525bc0000000p-25f},
    {0x1.172b840000000p+0f, -0x1.c157420000000p-27f}, {0x1.1a35be0000000p+0f, 0x1.6df96e0000000p-25f},
    {0x1.1d48740000000p+0f, -0x1.d2e8ca0000000p-25f}, {0x1.2063b80000000p+0f, 0x1.0c519a0000000p-25f},
    {0x1.2387a60000000p+0f, 0x1.ceac480000000p-25f}, {0x1.26b4560000000p+0f, 0x1.789f380000000p-26f},
    {0x1.29e9e00000000p+0f, -0x1.5c04240000000p-25f}, {0x1.2d285a0000000p+0f, 0x1.b900c20000000p-26f},
    {0x1.306fe00000000p+0f, 0x1.4636e20000000p-25f}, {0x1.33c08c0000000p+0f, -0x1.b37d200000000p-25f},
    {0x1.371a740000000p+0f, -0x1.18aac60000000p-25f}, {0x1.3a7db40000000p+0f, -0x1.634c020000000p-25f},
    {0x1.3dea640000000p+0f, 0x1.8246840000000p-25f}, {0x1.4160a20000000p+0f, 0x1.f72e2a0000000p-28f},
    {0x1.44e0860000000p+0f, 0x1.8624b40000000p-30f}, {0x1.486a2c0000000p+0f, -0x1.47d8660000000p-25f},
    {0x1.4bfdae0000000p+0f, -0x1.593abc0000000p-25f}, {0x1.4f9b280000000p+0f, -0x1.2c5a6c0000000p-25f},
    {0x1.5342b60000000p+0f, -0x1.2c56100000000p-25f}, {0x1.56f4740000000p+0f, -0x1.295b040000000p-25f},
    {0x1.5ab07e0000000p+0f, -0x1.5bd5ec0000000p-27f}, {0x1.5e76f20000000p+0f, -0x1.4a5bd60000000p-25f},
    {0x1.6247ec0000000p+0f, -0x1.f8b5500000000p-25f}, {0x1.6623880000000p+0f, 0x1.2a91120000000p-27f},
    {0x1.6a09e60000000p+0f, 0x1.9fcef40000000p-26f}, {0x1.6dfb240000000p+0f, -0x1.cd72e80000000p-27f},
    {0x1.71f75e0000000p+0f, 0x1.1d8bee0000000p-25f}, {0x1.75feb60000000p+0f, -0x1.37b3060000000p-25f},
    {0x1.7a11480000000p+0f, -0x1.829fd00000000p-25f}, {0x1.7e2f340000000p+0f, -0x1.2616340000000p-25f},
    {0x1.82589a0000000p+0f, -0x1.accc7c0000000p-26f}, {0x1.868d9a0000000p+0f, -0x1.2edb440000000p-26f},
    {0x1.8ace540000000p+0f, 0x1.15506e0000000p-27f}, {0x1.8f1aea0000000p+0f, -0x1.baa2320000000p-26f},
    {0x1.93737c0000000p+0f, -0x1.e647440000000p-25f}, {0x1.97d82a0000000p+0f, -0x1.0d8d840000000p-31f},
    {0x1.9c49180000000p+0f, 0x1.51f8480000000p-27f}, {0x1.a0c6680000000p+0f, -0x1.2886a60000000p-26f},
    {0x1.a5503c0000000p+0f, -0x1.b83b540000000p-25f}, {0x1.a9e6b60000000p+0f, -0x1.50c0480000000p-25f},
    {0x1.ae89fa0000000p+0f, -0x1.a94b140000000p-26f}, {0x1.b33a2c0000000p+0f, -0x1.ec3a820000000p-26f},
    {0x1.b7f7700000000p+0f, -0x1.a094380000000p-25f}, {0x1.bcc1ea0000000p+0f, -0x1.f687c60000000p-25f},
    {0x1.c199be0000000p+0f, -0x1.3d56b20000000p-27f}, {0x1.c67f120000000p+0f, 0x1.cafa2a0000000p-25f},
    {0x1.cb720e0000000p+0f, -0x1.8837cc0000000p-27f}, {0x1.d072d40000000p+0f, 0x1.40f1300000000p-25f},
    {0x1.d5818e0000000p+0f, -0x1.822dbc0000000p-27f}, {0x1.da9e600000000p+0f, 0x1.ed99420000000p-27f},
    {0x1.dfc9740000000p+0f, -0x1.908c940000000p-25f}, {0x1.e502ee0000000p+0f, 0x1.e2cffe0000000p-26f},
    {0x1.ea4afa0000000p+0f, 0x1.52486c0000000p-27f}, {0x1.efa1be0000000p+0f, 0x1.cc2b440000000p-25f},
    {0x1.f507660000000p+0f, -0x1.246eb00000000p-26f}, {0x1.fa7c180000000p+0f, 0x1.9e90d80000000p-28f},
};

// l - m in two parts (exact while neither overflows)
__device__ __forceinline__ Two minus(float l, float m) { return sum_of(l, -m); }

// What a row's weights exp((l - m) / T) are taken with.
struct Scale {
  float t, low;   // T (1 for a greedy sequence, which has those probabilities); -80 T
  Two inv;        // 1 / T
};
__device__ __forceinline__ Scale scale_of(float t) {
  if (t == 0.f || t == 1.f) return Scale{1.f, -80.f, Two{1.f, 0.f}};
  return Scale{t, -80.f * t, Two{1.f, 0.f} / Two{t, 0.f}};
}

// Two numbers each, whose operations are one instruction.
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair(float a, float b) {
  Pair r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 both(Pair a) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a));
  return r;
}
__device__ __forceinline__ Pair same(float a) { return pair(a, a); }
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ Pair sub2(Pair a, Pair b) { return fma2(b, same(-1.f), a); }
struct TwoPair {
  Pair h, l;
  __device__ __forceinline__ Two first() const { return Two{both(h).x, both(l).x}; }
  __device__ __forceinline__ Two second() const { return Two{both(h).y, both(l).y}; }
};
__device__ __forceinline__ TwoPair sum_of(Pair a, Pair b) {
  const Pair s = add2(a, b), t = sub2(s, a);
  return TwoPair{s, add2(sub2(a, sub2(s, t)), sub2(b, t))};
}
struct SumPair {   // two sums
  Pair h = 0, l = 0;
  __device__ __forceinline__ void add(const TwoPair& x) {
    const TwoPair s = sum_of(h, x.h);
    l = add2(l, add2(s.l, x.l));
    h = s.h;
  }
  __device__ __forceinline__ Two value() const {
    const TwoPair t{h, l};
    const Two a = t.first(), b = t.second();
    return norm2(a.h, a.l) + norm2(b.h, b.l);
  }
};

// exp(x), x = (l - m) / T = j log(2) / 64 + r + rl, |r| <= log(2) / 128, for two l: 2^(j / 64) by its exponent and the table, and four
// terms of the series of exp(r + rl), whose first is kept in two parts.  The others are below 2^-16: rounding them costs 2^-40 a step, 2^-37 +
// 2^-45 |x| in all at most (2^-37.7 the largest of 2.8 million, at temperatures from 2^-10 to 100).  rl, what x's rounding leaves, is
// up to 2^-22 at x = -7: in the first term alone it left weights 2^-26 off.  Both r and j's product with the first part of log(2) / 64
// are multiples of 2^-31, so that r comes out exactly but for the second parts.
// The first part of the result is the nearest to it: which of p and q is above the other goes by those, and sums of many second parts would
// round them off.  Below exp(-80), -infinity too, it is exp(-80) = 2^-115: no sum sees 2^20 of those, and none is drawn.
__device__ __forceinline__ TwoPair weights(float l0, float l1, float m, const Scale& c, const VdTab& tab) {
  const TwoPair d = sum_of(pair(l0, l1), same(-m));
  float2 h = both(d.h), l = both(d.l);
  l.x = h.x > c.low ? l.x : 0.f;
  l.y = h.y > c.low ? l.y : 0.f;
  Pair xh = pair(fmaxf(h.x, c.low), fmaxf(h.y, c.low)), xl = pair(l.x, l.y);
  if (c.t != 1.f) {
    const Pair p = mul2(xh, same(c.inv.h));
    xl = add2(fma2(xh, same(c.inv.h), mul2(p, same(-1.f))), fma2(xh, same(c.inv.l), mul2(xl, same(c.inv.h))));
    xh = p;
  }
  constexpr float LN_H = 0.010830424726009369f, LN_L = -2.976022206446771e-11f;   // log(2) / 64 in two parts
  const Pair jm = fma2(xh, same(92.33248261689366f), same(12582912.f));   // 1.5 2^23: the nearest whole number in the last bits
  const Pair jf = add2(jm, same(-12582912.f));
  const Pair r = fma2(jf, same(-LN_H), xh), rl = fma2(jf, same(-LN_L), xl);
  const float2 jb = both(jm);
  const int j0 = __float_as_int(jb.x), j1 = __float_as_int(jb.y);
  const Pair th = pair(tab.h[j0 & (VD_TAB - 1)], tab.h[j1 & (VD_TAB - 1)]), tl = pair(tab.l[j0 & (VD_TAB - 1)], tab.l[j1 & (VD_TAB - 1)]);
  const Pair v = add2(r, rl), y = fma2(mul2(v, v), fma2(v, fma2(v, same(1.f / 24.f), same(1.f / 6.f)), same(0.5f)), rl);   // exp(r + rl) = 1 + r + y
  const Pair ph = mul2(th, r), pl = fma2(th, r, mul2(ph, same(-1.f)));
  const Pair s = add2(th, ph), e = sub2(ph, sub2(s, th));
  const Pair lo = add2(e, add2(pl, fma2(th, y, fma2(tl, r, tl))));
  // 2^floor(j / 64): the whole number's bits above the table's, moved to the exponent (what lies above leaves the word)
  const Pair sc = pair(__int_as_float(((j0 & ~(VD_TAB - 1)) << 17) + 0x3f800000), __int_as_float(((j1 & ~(VD_TAB - 1)) << 17) + 0x3f800000));
  const Pair w = add2(s, lo);   // (lo is up to 2^-15 of s)
  return TwoPair{mul2(w, sc), mul2(sub2(lo, sub2(w, s)), sc)};
}

// The row that is looked at closely.
template <typename TT, typename TD, int LOADS>
struct Row {
  const TT* p;
  const TD* q;        // NULL: no draft distribution
  float mp, mq;
  Scale c;
  Two rho;            // sum of p's weights / sum of q's
  int certain;        // the draft that has all of q (-1: none)
  int plain;          // w = p
  // Tokens k0, k0 + 32, .. below k1, LOADS at a time: f(first of them, p's logits, q's), -infinity past the end.  The next ones' loads are
  // under way meanwhile.  Two at a time where a thread has few (one chunk over 50257 tokens, 6 a thread: 14.5 us, by four 15.0), four where it has
  // many (64 chunks over 131072, 128 a thread: 119 us, by two 128).
  template <typename F>
  __device__ __forceinline__ void each(int k0, int k1, F f) const {
    auto load = [&](int k, float (&x)[LOADS], float (&y)[LOADS]) {
#pragma unroll
      for (int j = 0; j < LOADS; ++j) {
        const int i = k + 32 * j;
        x[j] = i < k1 ? to_f<TT>(p[i]) : -INFINITY;
        y[j] = q && i < k1 ? to_f<TD>(q[i]) : -INFINITY;
      }
    };
    float x[LOADS], y[LOADS];
    if (k0 < k1) load(k0, x, y);
    for (int k = k0; k < k1; k += 32 * LOADS) {
      float u[LOADS], v[LOADS];
      load(k + 32 * LOADS, u, v);
      f(k, x, y);
#pragma unroll
      for (int j = 0; j < LOADS; ++j) {
        x[j] = u[j];
        y[j] = v[j];
      }
    }
  }
  // p - q of two tokens from the logits, times the sum of p's weights
  __device__ __forceinline__ TwoPair gap(float x0, float x1, float y0, float y1, const VdTab& tab) const {
    const TwoPair a = weights(x0, x1, mp, c, tab), b = weights(y0, y1, mq, c, tab);
    const Pair ph = mul2(same(-rho.h), b.h), pl = add2(fma2(same(-rho.h), b.h, mul2(ph, same(-1.f))), fma2(same(-rho.h), b.l, mul2(same(-rho.l), b.h)));
    const TwoPair d = sum_of(a.h, ph);
    const Pair e = add2(d.l, add2(a.l, pl)), s = add2(d.h, e);
    return TwoPair{s, sub2(e, sub2(s, d.h))};
  }
  // what tokens i and i + 32 are drawn with: max(p - q, 0)
  __device__ __forceinline__ TwoPair residual(int i, float x0, float x1, float y0, float y1, const VdTab& tab) const {
    if (plain) return weights(x0, x1, mp, c, tab);
    const TwoPair d = q ? gap(x0, x1, y0, y1, tab) : weights(x0, x1, mp, c, tab);
    float2 h = both(d.h), l = both(d.l);
    if (q ? !(h.x > 0.f) : i == certain) h.x = l.x = 0.f;
    if (q ? !(h.y > 0.f) : i + 32 == certain) h.y = l.y = 0.f;
    return TwoPair{pair(h.x, h.y), pair(l.x, l.y)};
  }
};

// The warp's sum of tokens k0 .. k1 - 1's residuals.
template <typename TT, typename TD, int LOADS>
__device__ __forceinline__ long long residual_sum(const Row<TT, TD, LOADS>& row, int k0, int k1, float unit, const VdTab& tab) {
  SumPair sw;
  row.each(k0 + (threadIdx.x & 31), k1, [&](int k, const float (&x)[LOADS], const float (&y)[LOADS]) {
#pragma unroll
    for (int j = 0; j < LOADS; j += 2) sw.add(row.residual(k + 32 * j, x[j], x[j + 1], y[j], y[j + 1], tab));
  });
  return warp_sum(whole(sw.value(), unit));
}
// (for what seldom runs, out of the kernel's way)
template <typename TT, typename TD, int LOADS>
__device__ __noinline__ long long residual_sum_seldom(Row<TT, TD, LOADS> row, int k0, int k1, float unit, const VdTab& tab) {
  return residual_sum(row, k0, k1, unit, tab);
}
// The token among k0 .. k1 - 1 with which the sum, `sum` before them, passes `at`; else the last with a weight (what rounding leaves), or -1.
template <typename TT, typename TD, int LOADS>
__device__ __forceinline__ int walk(const Row<TT, TD, LOADS>& row, int k0, int k1, long long sum, long long at, float unit, const VdTab& tab) {
  const int lane = threadIdx.x & 31;
  int token = -1;
  for (; k0 < k1; k0 += 32) {
    const int k = k0 + lane;
    const bool in = k < k1;
    const Two v = row.residual(k, in ? to_f<TT>(row.p[k]) : -INFINITY, -INFINITY, in && row.q ? to_f<TD>(row.q[k]) : -INFINITY, -INFINITY, tab).first();
    const long long w = in ? whole(v, unit) : 0;
    long long inc = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += u;
    }
    const unsigned over = __ballot_sync(0xffffffffu, w > 0 && sum + inc > at), some = __ballot_sync(0xffffffffu, w > 0);
    if (over) return k0 + __ffs(over) - 1;
    if (some) token = k0 + 31 - __clz(some);
    sum += __shfl_sync(0xffffffffu, inc, 31);
  }
  return token;
}
// A token whose p is next to its q: what the sum of p's above q, less q's there, has to be mended by (0: it was on its side).
template <typename TT, typename TD, int LOADS>
__device__ __noinline__ long long mend(Row<TT, TD, LOADS> row, int k, float rho32, float unit, const VdTab& tab) {
  const float x = to_f<TT>(row.p[k]), y = to_f<TD>(row.q[k]);
  const bool above = __fmaf_rn(both(weights(y, y, row.mq, row.c, tab).h).x, -rho32, both(weights(x, x, row.mp, row.c, tab).h).x) > 0.f;
  const Two d = row.gap(x, x, y, y, tab).first();
  return above == (d.h > 0.f) ? 0 : whole(d.h > 0.f ? d : Two{-d.h, -d.l}, unit);
}

template <typename TT, typename TD, int LOADS>
__global__ void __launch_bounds__(VD_THREADS) verify_decide_kernel(VerifyCall a, int parts, const Stat* stats, const int* owner) {
  constexpr int WARPS = VD_THREADS / 32;
  static_assert(WARPS >= 5 && WARPS <= 32 && VD_CTAS <= 32, "sums and run_of by a warp");
  __shared__ VdTab tab;
  __shared__ int s_first;
  __shared__ float4 s_row;   // maximum and sum of the row in question, the target's and the draft's
  // sums of the ranks and of this CTA's warps: p's weights, q's, those of p where p is above q, those of q there, those of q next to p; what
  // is drawn from
  enum { OF_P, OF_Q, P_ABOVE, Q_ABOVE, Q_NEAR, DRAWN, MENDED, SUMS };
  __shared__ int s_near[VD_NEARS], s_nears;   // tokens with p next to q, and how many there are
  __shared__ unsigned long long s_mend;
  __shared__ long long s_at;   // the draw's number in the sum of what is drawn from
  __shared__ int s_how;
  __shared__ Two s_rho;
  __shared__ long long s_part[SUMS][VD_CTAS], s_warp[SUMS][WARPS], s_piece[WARPS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = cluster_rank(), ctas = cluster_size(), b = (int)blockIdx.x / ctas;
  if (tid == 0) {
    s_mend = 0;
    s_nears = 0;
  }
  if (tid < VD_TAB) {
    tab.h[tid] = VD_POW[tid].x;
    tab.l[tid] = VD_POW[tid].y;
  }
  PDL_ENTRY();
  const SeqRows q = seq_rows(a, b);
  const float t = a.temp ? a.temp[b] : 1.f;
  cluster_barrier();   // (also: the others' shared memory is there)
  const int n = q.ok ? q.e - q.s : 0;
  const bool greedy = t == 0.f, soft = a.draft != nullptr && !greedy;
  auto give = [&](int acc, int nxt) {
    if (rank == 0 && tid == 0) {
      a.accepted[b] = acc;
      a.next[b] = nxt;
    }
  };
  if (n == 0 || !temp_ok(t)) {   // (uniform over the cluster)
    const bool idle = q.ok && n == 0;
    if (!idle && rank == 0 && tid == 0) a.flag(q.ok ? ERRW_VALUE : ERRW_POS);
    give(idle ? 0 : -1, -1);
    return;
  }
  const Scale sc = scale_of(t);
  const float close = sc.t * close_of(a.vocab, parts);
  // maximum and sum of a row from its parts', all loads together
  auto stat = [&](int which, int r) {
    const Stat* s = stats + ((size_t)which * a.n_rows + r) * parts;
    float2 x[VS_PARTS];
#pragma unroll
    for (int k = 0; k < VS_PARTS; ++k) x[k] = k < parts ? *reinterpret_cast<const float2*>(s + k) : make_float2(-INFINITY, 0.f);
    float m = x[0].x, z = 0.f;
#pragma unroll
    for (int k = 1; k < VS_PARTS; ++k) m = fmaxf(m, x[k].x);
    const float c = 1.44269504088896f * sc.inv.h;
#pragma unroll
    for (int k = 0; k < VS_PARTS; ++k)
      if (k < parts) z += x[k].x == m || x[k].x == -INFINITY ? x[k].y : x[k].y * ex2_approx((x[k].x - m) * c);
    return make_float2(m, z);
  };
  auto drafted_at = [&](int which, int r) { return stats[((size_t)which * a.n_rows + r) * parts].l; };   // the draft's logit in a row
  auto best = [&](int r) {   // the first index of a target row's maximum
    const Stat* s = stats + (size_t)r * parts;
    float m[VS_PARTS];
    int at[VS_PARTS];
#pragma unroll
    for (int k = 0; k < VS_PARTS; ++k) {
      m[k] = k < parts ? s[k].m : -INFINITY;
      at[k] = k < parts ? s[k].at : 0;
    }
#pragma unroll
    for (int k = 1; k < VS_PARTS; ++k)
      if (m[k] > m[0]) {
        m[0] = m[k];
        at[0] = at[k];
      }
    return at[0];
  };
  // log of exp((l - m) / T) / z
  auto log_share = [&](float l, float m, float z) {
    const Two d = minus(l, m);
    if (!(d.h * sc.inv.h >= -FLT_MAX)) return -INFINITY;
    const Two x = d * sc.inv + Two{-logf(z), 0.f};
    return x.h + x.l;
  };

  // how a row stands by its 32-bit sums; the last row, behind which there is no draft, stops
  enum { HOLDS = 0, STOPS = 1, CLOSE = 2, BAD = 3 };
  auto stands = [&](int i, float4& row) {
    const int r = q.s + i;
    const bool last = i == n - 1, drafted = soft && !last;
    const float2 p = stat(0, r), d = drafted ? stat(1, r) : make_float2(0.f, 1.f);
    const int x = last ? 0 : a.tokens[r + 1], whose = owner[r];
    const float u = greedy ? 0.f : a.u[r], lp = drafted_at(0, r), lq = drafted ? drafted_at(1, r) : 0.f;
    row = make_float4(p.x, p.y, d.x, d.y);
    if (whose != b || !(p.y > 0.f)) return (int)BAD;   // another sequence's row too; nothing above -infinity, a NaN, +infinity
    if (last) return (int)STOPS;
    if (x < 0 || x >= a.vocab) return (int)BAD;
    if (greedy) return best(r) == x ? (int)HOLDS : (int)STOPS;
    if (!(u >= 0.f && u < 1.f) || !(d.y > 0.f)) return (int)BAD;
    // T times the difference of the logarithms: what holds has it below 0
    const Two dp = minus(lp, p.x), dq = drafted ? minus(lq, d.x) : Two{0.f, 0.f};
    if (dp.h == -INFINITY) return (int)STOPS;
    if (u == 0.f || dq.h == -INFINITY) return (int)HOLDS;
    const float logs = logf(p.y) + logf(u) - logf(d.y);
    const float by = (dq + Two{-dp.h, -dp.l} + Two{sc.t * logs, 0.f}).h;
    return fabsf(by) < close ? (int)CLOSE : by < 0.f ? (int)HOLDS : (int)STOPS;
  };
  // the first row from `from` on that does not hold, and how it stands; s_row
  auto first_from = [&](int from, int& i, int& code) {
    __syncthreads();
    if (tid == 0) s_first = 0x7fffffff;
    __syncthreads();
    int mine = 0;
    float4 row;
    for (int k = from + tid; k < n && !mine; k += VD_THREADS) {
      const int c = stands(k, row);
      if (c != HOLDS) mine = k * 4 + c;
    }
    if (mine) atomicMin(&s_first, mine);
    __syncthreads();
    const int first = s_first;
    if (mine == first) s_row = row;
    __syncthreads();
    i = first >> 2;
    code = first & 3;
  };
  Row<TT, TD, LOADS> row;
  row.c = sc;
  const int share = (a.vocab + ctas - 1) / ctas, v0 = min(a.vocab, rank * share), v1 = min(a.vocab, v0 + share);
  const int each = ((share + WARPS - 1) / WARPS + 31) & ~31, w0 = min(v1, v0 + warp * each), w1 = min(v1, w0 + each);
  // the CTA's sum of its warps' numbers v to place `part` of every CTA of the cluster, by one warp
  auto exchange = [&](const long long* v, long long* part) {
    const long long s = warp_sum(lane < WARPS ? v[lane] : 0);
    if (lane < ctas) cluster_store(&part[rank], lane, s);
  };
  auto total = [&](const long long* part) { return warp_sum(lane < ctas ? part[lane] : 0); };
  float unit = 0.f, unit_q = 0.f;
  float rho32 = 0.f;   // Zp / Zq by the 32-bit sums
  long long zp = 0, zq = 0;
  auto look = [&](int r) {   // precise sums of row r: the warps' in s_warp, the ranks' in s_part
    const float4 st = s_row;
    row.p = (const TT*)a.target + r * a.ld_t;
    row.q = soft && r < q.e - 1 ? (const TD*)a.draft + r * a.ld_d : nullptr;
    row.mp = st.x;
    row.mq = st.z;
    unit = unit_of(st.y);
    unit_q = unit_of(st.w);
    SumPair sp;
    if (row.q) {
      SumPair sq, above_p, above_q;
      float near = 0.f;
      rho32 = __fdividef(st.y, st.w);
      row.each(w0 + lane, w1, [&](int k, const float (&x)[LOADS], const float (&y)[LOADS]) {
        bool by[LOADS], any = false;
        float qh[LOADS];
#pragma unroll
        for (int j = 0; j < LOADS; j += 2) {
          const TwoPair p = weights(x[j], x[j + 1], row.mp, row.c, tab), d = weights(y[j], y[j + 1], row.mq, row.c, tab);
          sp.add(p);
          sq.add(d);
          // (less 10^-36: masked tokens, and those past the end, are next to nothing)
          const float2 g = both(fma2(d.h, same(-rho32), p.h)), lim = both(fma2(p.h, same(VD_NEAR), same(-1e-36f))), dh = both(d.h);
          const Pair in = pair(g.x > 0.f ? 1.f : 0.f, g.y > 0.f ? 1.f : 0.f);
          above_p.add(TwoPair{mul2(p.h, in), mul2(p.l, in)});
          above_q.add(TwoPair{mul2(d.h, in), mul2(d.l, in)});
          by[j] = fabsf(g.x) < lim.x;
          by[j + 1] = fabsf(g.y) < lim.y;
          any |= by[j] || by[j + 1];
          qh[j] = dh.x;
          qh[j + 1] = dh.y;
        }
        if (any) {
#pragma unroll
          for (int j = 0; j < LOADS; ++j)
            if (by[j]) {
              near += qh[j];
              const int at = atomicAdd(&s_nears, 1);
              if (at < VD_NEARS) s_near[at] = k + 32 * j;
            }
        }
      });
      const long long of_q = warp_sum(whole(sq.value(), unit_q)), p_above = warp_sum(whole(above_p.value(), unit)),
                      q_above = warp_sum(whole(above_q.value(), unit_q)), q_near = warp_sum(whole(Two{near, 0.f}, unit_q));
      if (lane == 0) {
        s_warp[OF_Q][warp] = of_q;
        s_warp[P_ABOVE][warp] = p_above;
        s_warp[Q_ABOVE][warp] = q_above;
        s_warp[Q_NEAR][warp] = q_near;
      }
    } else {
      row.each(w0 + lane, w1, [&](int, const float (&x)[LOADS], const float (&)[LOADS]) {
#pragma unroll
        for (int j = 0; j < LOADS; j += 2) sp.add(weights(x[j], x[j + 1], row.mp, row.c, tab));
      });
    }
    const long long of_p = warp_sum(whole(sp.value(), unit));
    if (lane == 0) s_warp[OF_P][warp] = of_p;
    __syncthreads();
    if (row.q && warp == Q_NEAR && s_nears > VD_NEARS) {   // (a sum that says so)
      if (lane == 0) s_warp[Q_NEAR][0] = 1ll << 58;
      __syncwarp();
    }
    if (warp < (row.q ? DRAWN : OF_Q)) exchange(s_warp[warp], s_part[warp]);
    cluster_barrier();
    zp = total(s_part[OF_P]);
    if (row.q) zq = total(s_part[OF_Q]);
  };
  // The row that stops.  (A loop, so that both steps, most of the kernel's code, are there once: instructions come from L2, and
  // with two copies of each 16 chunks took 19.1 us where they take 18.4.)
  int i = -1, code = BAD;
  const bool draws = greedy || (a.u[q.e - 1] >= 0.f && a.u[q.e - 1] < 1.f);
  while (draws) {
    first_from(i + 1, i, code);
    if (code == BAD || greedy) break;
    const int r = q.s + i;
    look(r);
    if (code == STOPS) break;
    // a draft that is too close: decided by the precise sums, in 64 bits
    if (tid == 0) {
      const double dp = (double)drafted_at(0, r) - row.mp, dq = row.q ? (double)drafted_at(1, r) - row.mq : 0.0;
      const double logs = log((double)a.u[r]) + log((double)zp / unit) - (row.q ? log((double)zq / unit_q) : 0.0);
      s_first = dq - dp + (double)t * logs < 0.0;
    }
    __syncthreads();
    if (!s_first) break;
    cluster_barrier();   // (the sums of that row have been read: s_part is free, and the next row's list is empty)
    if (tid == 0) s_nears = 0;
  }
  if (code == BAD) {
    if (rank == 0 && tid == 0) a.flag(ERRW_VALUE);
    give(-1, -1);
    return;
  }
  const int r = q.s + i;
  if (a.logprob && rank == ctas - 1) {   // (not the CTA that gives the result)
    for (int k = q.s + tid; k < r; k += VD_THREADS) {
      const float2 p = stat(0, k);
      a.logprob[k] = log_share(drafted_at(0, k), p.x, p.y);
    }
  }
  if (greedy) {
    if (rank == 0 && tid == 0) {
      give(i, best(r));
      if (a.logprob) a.logprob[r] = -logf(s_row.y);
    }
    return;
  }
  row.certain = soft || r == q.e - 1 ? -1 : a.tokens[r + 1];
  row.plain = r == q.e - 1;
  // What is drawn from: its sum, the ranks' and this CTA's warps'.  One warp settles it (conversions of 64 bits run at a few a cycle and SM).
  enum { PLAIN = 0, RESIDUAL = 1, WRONG_SIDES = 2, BY_TOKEN = 3 };
  auto settle = [&](long long all) {   // by all lanes of the warp: the sum and the draw's number in it
    const bool fall_back = !row.plain && all < zp >> VD_LEAST;
    const long long sum = fall_back ? zp : all;
    // u in the middle of its 2^-24, times the sum
    s_at = (long long)__umul64hi(__float2ull_rz(a.u[q.e - 1] * 18446744073709551616.f) + (1ull << 39), (unsigned long long)sum);
    return row.plain || fall_back ? PLAIN : RESIDUAL;
  };
  if (row.plain) {
    if (warp == 0) s_how = settle(zp);
  } else {
    // sum of max(p - q, 0) = that of p where p is above q, less that of q there.  "Above" went by the 32-bit sums' quotient: a token whose p
    // and q are nearer than that is off may be on the wrong side, which changes the sum by that much of its q
    if (warp == 0 && row.q) {
      const Two rho = quotient(two_of(zp), two_of(zq));   // in p's units over q's
      const float by = __int_as_float(0x3f800000 + __float_as_int(unit_q) - __float_as_int(unit));
      const float off = fabsf(rho32 - rho.h * by) / (rho.h * by) + 2.384185791015625e-07f;   // (and the comparison's roundings)
      auto rest = [&](long long above_p, long long above_q) {
        const Two x = rho * two_of(above_q);
        const long long v = above_p - __float2ll_rn(x.h) - __float2ll_rn(x.l);
        return v < VD_NOTHING ? 0ll : v;
      };
      if (lane < WARPS) s_warp[DRAWN][lane] = rest(s_warp[P_ABOVE][lane], s_warp[Q_ABOVE][lane]);
      const long long part = lane < ctas ? rest(s_part[P_ABOVE][lane], s_part[Q_ABOVE][lane]) : 0;
      if (lane < ctas) s_part[DRAWN][lane] = part;
      const long long all = warp_sum(part), q_near = total(s_part[Q_NEAR]);
      s_rho = Two{rho.h * by, rho.l * by};
      if (all < zp >> VD_FINE || off > VD_NEAR || q_near >= 1ll << 58)
        s_how = BY_TOKEN;
      else if (off * rho.h * __ll2float_rn(q_near) > VD_SURE * __ll2float_rn(all))
        s_how = WRONG_SIDES;
      else
        s_how = settle(all);
    }
    if (warp == 0 && !row.q) {   // all of p but the draft (p's sums are rounded to 2^-45 or so: where little is left, the others are summed by themselves)
      const int x = row.certain, at_rank = x / share, at_warp = (x - at_rank * share) / each;
      const long long wx = whole(weights(drafted_at(0, r), -INFINITY, row.mp, row.c, tab).first(), unit);
      auto rest = [&](long long v, bool has) { return has ? (v - wx < VD_NOTHING ? 0ll : v - wx) : v; };
      if (lane < WARPS) s_warp[DRAWN][lane] = rest(s_warp[OF_P][lane], rank == at_rank && lane == at_warp);
      const long long part = lane < ctas ? rest(s_part[OF_P][lane], lane == at_rank) : 0;
      if (lane < ctas) s_part[DRAWN][lane] = part;
      const long long all = warp_sum(part);
      s_how = all < zp >> VD_FINE ? (int)BY_TOKEN : settle(all);
    }
    __syncthreads();
    if (row.q) row.rho = s_rho;
    const int how = s_how;
    if (how >= WRONG_SIDES) {   // (uniform over the cluster)
      if (how == BY_TOKEN) {
        const long long vw = residual_sum_seldom(row, w0, w1, unit, tab);
        if (lane == 0) s_warp[DRAWN][warp] = vw;
        cluster_barrier();   // (and every CTA has read its s_part)
        if (warp == 0) exchange(s_warp[DRAWN], s_part[DRAWN]);
      } else {
        if (tid < s_nears) {
          const int k = s_near[tid];
          const unsigned long long more = (unsigned long long)mend(row, k, rho32, unit, tab);
          if (more) {
            atomicAdd(reinterpret_cast<unsigned long long*>(&s_warp[DRAWN][(k - v0) / each]), more);
            atomicAdd(&s_mend, more);
          }
        }
        __syncthreads();
        if (tid < ctas) cluster_store(&s_part[MENDED][rank], tid, (long long)s_mend);
      }
      cluster_barrier();
      if (warp == 0) {
        if (how == WRONG_SIDES && lane < ctas) s_part[DRAWN][lane] += s_part[MENDED][lane];
        __syncwarp();
        s_how = settle(total(s_part[DRAWN]));
      }
    }
  }
  __syncthreads();
  row.plain = s_how == PLAIN;
  const long long at = s_at;
  const long long *by_rank = s_part[row.plain ? OF_P : DRAWN], *by_warp = s_warp[row.plain ? OF_P : DRAWN];
  // the run in which the sum passes `at`: the last of those that hold something and begin at or below it (by a warp)
  long long before = 0;
  auto run_of = [&](const long long* v, int n_runs) {
    const long long x = lane < n_runs ? v[lane] : 0;
    long long inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += u;
    }
    const long long from = before + inc - x;
    const unsigned ok = __ballot_sync(0xffffffffu, x > 0 && from <= at);
    const int k = ok ? 31 - __clz(ok) : 0;
    before = __shfl_sync(0xffffffffu, from, k);
    return k;
  };
  if (rank != run_of(by_rank, ctas)) return;
  // this CTA's run, of it a warp's, which all warps look at in shares
  const int ow = run_of(by_warp, WARPS);
  const int r0 = min(v1, v0 + ow * each), r1 = min(v1, r0 + each), piece = ((each + WARPS - 1) / WARPS + 31) & ~31;
  const int p0 = min(r1, r0 + warp * piece), p1 = min(r1, p0 + piece);
  const long long vw = residual_sum(row, p0, p1, unit, tab);
  if (lane == 0) s_piece[warp] = vw;
  __syncthreads();
  if (warp != run_of(s_piece, WARPS)) return;
  int token = -1;
  for (int again = 0; again < 2 && token < 0; ++again)   // (again: a run of tokens with p next to q, on the wrong sides; odds of 2^-34)
    token = walk(row, again ? 0 : p0, again ? a.vocab : p1, again ? 0 : before, at, unit, tab);
  if (lane == 0) {
    a.accepted[b] = i;
    a.next[b] = token;
    if (a.logprob) a.logprob[r] = log_share(to_f<TT>(row.p[max(token, 0)]), row.mp, __ll2float_rn(zp) / unit);
  }
}

int verify_sms() {
  static const int sms = [] {
    int dev = 0, n = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    return n > 0 ? n : 1;
  }();
  return sms;
}

// CTAs of a row: as many as give the GPU four CTAs an SM, while each has two rounds of its threads.
int verify_parts(int n_rows, int vocab) {
  int parts = 1;
  while (parts < VS_PARTS && (long long)n_rows * parts < 4 * verify_sms() && vocab / (2 * parts) >= VS_THREADS * 8) parts *= 2;
  return parts;
}

// CTAs of a sequence: the most (of an SM each) whose clusters find room for all sequences at once, or nearly: 64 sequences of 131072 tokens took
// 119 us by 2 CTAs each, 126 by 4; one sequence of 50257 tokens 14.5 by 16 CTAs, 16.2 by 8; eight of 32000, of whose clusters of 16 seven find
// room, 18.6 by 16, 17.6 by 8; sixteen chunks of which one waits (some of them greedy, and done at once) 18.5 by 8, 21.2 by 4.
// at_once(c): how many clusters of c find room.
template <typename F>
int verify_ctas(int n_seq, F at_once) {
  for (int ctas = VD_CTAS; ctas > 1; ctas /= 2) {
    const int n = at_once(ctas);
    if (n > 0 && n_seq <= n + n / 8) return ctas;
  }
  return 1;
}

template <typename TT, typename TD>
cudaError_t verify_t(cudaStream_t st, const VerifyCall& a) {
  const int parts = a.n_rows > 0 ? verify_parts(a.n_rows, a.vocab) : 1;
  Stat* stats = (Stat*)a.ws;
  int* owner = (int*)(stats + (size_t)2 * VS_PARTS * a.n_rows);   // [n_rows] the sequence that a row's statistics are for
  if (a.n_rows > 0) {
    const cudaError_t e = launch_k(verify_stats_kernel<TT, TD>, dim3((unsigned)(a.n_rows * parts), a.draft ? 2 : 1), dim3(VS_THREADS), 0, st, a, parts, stats, owner);
    if (e != cudaSuccess) return e;
  }
  struct Tag;
  struct Tag4;
  auto two = verify_decide_kernel<TT, TD, 2>, four = verify_decide_kernel<TT, TD, 4>;
  cudaError_t e = cluster16_once<Tag>(two);
  if (e == cudaSuccess) e = cluster16_once<Tag4>(four);
  if (e != cudaSuccess) return e;
  auto is_four = [&](int ctas) { return a.vocab / ctas >= VD_MANY * VD_THREADS; };
  const int ctas = verify_ctas(a.n_seq, [&](int c) { return is_four(c) ? clusters_at_once<Tag4>(four, c, VD_THREADS) : clusters_at_once<Tag>(two, c, VD_THREADS); });
  return launch_cluster(is_four(ctas) ? four : two, dim3((unsigned)(a.n_seq * ctas)), ctas, VD_THREADS, 0, st, a, parts, (const Stat*)stats, (const int*)owner);
}

}  // namespace

size_t verify_workspace(int n_rows) { return (size_t)n_rows * (2 * VS_PARTS * sizeof(Stat) + sizeof(int)); }

cudaError_t launch_verify(cudaStream_t st, const VerifyCall& a) {
  if (a.t_bf16) return a.d_bf16 ? verify_t<bf16, bf16>(st, a) : verify_t<bf16, float>(st, a);
  return a.d_bf16 ? verify_t<float, bf16>(st, a) : verify_t<float, float>(st, a);
}

}  // namespace adept

// Host-side check of the rule (no device work): at_once[i] clusters of 2^i CTAs find room.
extern "C" __attribute__((visibility("default"))) int adept_debug_verify_ctas(int n_seq, const int* at_once) {
  return adept::verify_ctas(n_seq, [&](int c) {
    int i = 0;
    while (1 << i < c) ++i;
    return at_once[i];
  });
}
