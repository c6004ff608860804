// Drafted tokens against the target's logits.
//
// Row r of a sequence holds the target's logits behind token tokens[r]; p_r = softmax(l_r / T), q_r the draft's.  Draft x =
// tokens[r + 1] holds where log u_r + log q_r(x) < log p_r(x); at the first row whose draft does not, the next token is drawn from
// max(p_r - q_r, 0), at the last row from p_r.
//
// Two launches.  The first streams every row once (HBM-bound) and leaves its maximum, the sum of exp((l - max) / T) and the
// first index of the maximum.  The second, a cluster per sequence, decides.  Sums of 32 bits decide a draft unless the two
// sides are closer than their errors (close_of); those, and the drawing, go by weights of two 32-bit parts each (2^-40 relative):
// with a vocabulary of V tokens the cumulative sum has V steps, and an error of 2^-24 would move the drawn token with odds of V 2^-23.
#include "cluster.cuh"
#include "serve_ops.h"

#include <float.h>

namespace adept {
namespace {

constexpr int VS_THREADS = 256;                  // rows' statistics
constexpr int VD_THREADS = 512, VD_CTAS = 8;     // decision: threads of a CTA, CTAs of a sequence's cluster
constexpr double VD_LEAST = 9.5367431640625e-07; // 2^-20: residual mass below which the token is drawn from p
constexpr int VD_TAB = 64;

// Relative difference of the two sides of a test below which 32-bit sums do not decide it.  A sum's error: a thread's chain of
// additions and rescalings, one for each of its 16-byte pieces, 2^-22 each; the exponentials' argument, rounded in three places
// 2^-24 of up to log2 V + 2 units on average; 20 more for the joins.  Two sums.
__device__ __forceinline__ double close_of(int vocab, int n_split) {
  return 2 * 2.384185791015625e-07 * (vocab / (4 * VS_THREADS * n_split) + 1 + 22 + 20);
}

struct Stat {
  float m, z;   // maximum; sum of exp((l - m) / T)
  int at;       // first index of the maximum
  int pad;
};

// 1 / T in units of log 2; a greedy sequence (T = 0) has the probabilities of T = 1.
__device__ __forceinline__ bool temp_ok(float t) { return t == 0.f || (t >= 9.765625e-4f && t <= 1024.f); }
__device__ __forceinline__ double log2_scale(float t) { return 1.4426950408889634 / (t == 0.f ? 1.0 : (double)t); }

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

template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(const float* p, float (&x)[4]) {
    const float4 v = __ldcs(reinterpret_cast<const float4*>(p));
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
  }
};
template <>
struct Vec<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(const bf16* p, float (&x)[8]) {
    const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
  }
};

// The maximum starts at the type's lowest value, not at -infinity: rows that begin with masked tokens need no special case
// (lowest - lowest = 0, -infinity - lowest = -infinity).
struct Running {
  float m = -FLT_MAX, z = 0.f;
  int at = 0x7fffffff;
  __device__ __forceinline__ void join(float om, float oz, int oat, float c) {
    if (om > m || (om == m && oat < at)) at = oat;
    const float nm = fmaxf(m, om);
    z = z * ex2_approx((m - nm) * c) + oz * ex2_approx((om - nm) * c);
    m = nm;
  }
  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N], int i0, float c) {
    float g = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) g = fmaxf(g, x[i]);
    if (g > m) {
      z *= ex2_approx((m - g) * c);
      m = g;
      at = 0x7fffffff;
    }
    if (at == 0x7fffffff) {
#pragma unroll
      for (int i = N - 1; i >= 0; --i)
        if (x[i] == m) at = i0 + i;
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s += ex2_approx((x[i] - m) * c);
    z += s;
  }
};

template <typename T>
__device__ void row_stats(const T* x, int V, float c, int split, int n_split, Stat* out) {
  constexpr int N = Vec<T>::N;
  __shared__ float s_m[VS_THREADS / 32], s_z[VS_THREADS / 32];
  __shared__ int s_at[VS_THREADS / 32];
  const int tid = threadIdx.x;
  // elements before the first 16-byte boundary, 16-byte pieces, the rest
  const int head = min(V, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T));
  const int nv = (V - head) / N, v0 = (int)((long long)nv * split / n_split), v1 = (int)((long long)nv * (split + 1) / n_split);
  Running r;
  if (split == 0 && tid < head) {
    const float y[1] = {to_f<T>(x[tid])};
    r.add(y, tid, c);
  }
  for (int v = v0 + tid; v < v1; v += VS_THREADS) {
    float y[N];
    Vec<T>::get(x + head + (size_t)v * N, y);
    r.add(y, head + v * N, c);
  }
  const int tail = head + nv * N + tid;
  if (split == n_split - 1 && tail < V) {
    const float y[1] = {to_f<T>(x[tail])};
    r.add(y, tail, c);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1)
    r.join(__shfl_xor_sync(0xffffffffu, r.m, o), __shfl_xor_sync(0xffffffffu, r.z, o), __shfl_xor_sync(0xffffffffu, r.at, o), c);
  if ((tid & 31) == 0) {
    s_m[tid >> 5] = r.m;
    s_z[tid >> 5] = r.z;
    s_at[tid >> 5] = r.at;
  }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < VS_THREADS / 32; ++w) r.join(s_m[w], s_z[w], s_at[w], c);
    *out = Stat{r.m, r.z, r.at, 0};
  }
}

// Statistics of part blockIdx.x % n_split of row blockIdx.x / n_split: the target's (blockIdx.y = 0) or the draft's.
template <typename TT, typename TD>
__global__ void __launch_bounds__(VS_THREADS) verify_stats_kernel(VerifyCall a, int n_split, Stat* stats) {
  PDL_ENTRY();
  __shared__ int s_seq;
  const int r = (int)(blockIdx.x / n_split), split = (int)(blockIdx.x % n_split), tid = threadIdx.x;
  if (tid == 0) s_seq = 0x7fffffff;
  __syncthreads();
  for (int b = tid; b < a.n_seq; b += VS_THREADS) {
    const SeqRows q = seq_rows(a, b);
    if (q.ok && q.s <= r && r < q.e) atomicMin(&s_seq, b);
  }
  __syncthreads();
  if (s_seq == 0x7fffffff) return;   // nobody's row
  const float t = a.temp ? a.temp[s_seq] : 1.f;
  if (!temp_ok(t)) return;
  if (blockIdx.y && (t == 0.f || r == a.start[s_seq + 1] - 1)) return;   // a draft row that nothing is held against
  Stat* out = stats + ((size_t)blockIdx.y * a.n_rows + r) * n_split + split;
  const float c = (float)log2_scale(t);
  if (blockIdx.y == 0)
    row_stats((const TT*)a.target + r * a.ld_t, a.vocab, c, split, n_split, out);
  else
    row_stats((const TD*)a.draft + r * a.ld_d, a.vocab, c, split, n_split, out);
}

// ---------------------------------------------------------------------------------------------
// Weights of two 32-bit parts.
// ---------------------------------------------------------------------------------------------
struct Two {
  float h, l;
};
__device__ __forceinline__ Two two_of(double x) {
  const float h = (float)x;
  return Two{h, (float)(x - (double)h)};
}
// Sum of two-part numbers, each thread's own (Knuth's two-sum; the low parts add up beside it).
struct Sum2 {
  float h = 0.f, l = 0.f;
  __device__ __forceinline__ void add(Two x) {
    const float s = __fadd_rn(h, x.h), t = __fsub_rn(s, h);
    l = __fadd_rn(l, __fadd_rn(__fadd_rn(__fsub_rn(h, __fsub_rn(s, t)), __fsub_rn(x.h, t)), x.l));
    h = s;
  }
  __device__ __forceinline__ double value() const { return (double)h + (double)l; }
};

// exp((l - m) / T) = 2^t, t = (l - m) c with c = log2(e) / T: t = n + k / 64 + r, |r| <= 1/128; 2^(k/64) from a table, 2^r from four
// terms of its series, whose first is kept in two parts (the others are below 2^-16, and rounding them costs 2^-40).  0 below
// 2^-64: what is left out of a sum of 2^20 weights is below 2^-44.
__device__ __forceinline__ Two weight(float l, float m, Two c, const float2* tab) {
  const float d = __fsub_rn(l, m), b = __fsub_rn(d, l);
  const float dl = __fsub_rn(__fsub_rn(l, __fsub_rn(d, b)), __fadd_rn(m, b));   // l - m = d + dl
  const float th = __fmul_rn(d, c.h);
  if (!(th > -64.f)) return Two{0.f, 0.f};
  const float tl = __fmaf_rn(d, c.h, -th) + __fmaf_rn(d, c.l, dl * c.h);
  const float j = rintf(th * VD_TAB);
  const float r = __fmaf_rn(j, -1.f / VD_TAB, th);   // exact
  const int ji = (int)j;
  const float2 T = tab[ji & (VD_TAB - 1)];
  constexpr float LN2_H = 0.693147182464599609375f, LN2_L = -1.90465429995776804e-09f;   // log 2 in two parts
  const float sh = __fmul_rn(r, LN2_H);
  const float sl = __fmaf_rn(r, LN2_H, -sh) + __fmaf_rn(r, LN2_L, tl * LN2_H);
  const float y = sl + sh * sh * __fmaf_rn(sh, __fmaf_rn(sh, 1.f / 24.f, 1.f / 6.f), 0.5f);   // 2^r = 1 + sh + y
  const float ph = __fmul_rn(T.x, sh), pl = __fmaf_rn(T.x, sh, -ph);
  const float s = __fadd_rn(T.x, ph), e = __fsub_rn(ph, __fsub_rn(s, T.x));
  const float lo = e + (pl + __fmaf_rn(T.x, y, __fmaf_rn(T.y, sh, T.y)));
  const float sc = __uint_as_float((unsigned)(127 + (ji >> 6)) << 23);   // 2^n, n >= -65
  const float h = __fadd_rn(s, lo);
  return Two{h * sc, __fsub_rn(lo, __fsub_rn(h, s)) * sc};
}

// What the cluster's threads share of the row that is looked at closely.
template <typename TT, typename TD>
struct Row {
  const TT* p;
  const TD* q;        // NULL: no draft distribution, or none to take away
  float mp, mq;
  Two c, rho;         // scale; sum of p's weights / sum of q's
  int certain;        // the draft that has all of q (-1: none)
  int plain;          // w = p
  __device__ __forceinline__ Two at_p(int i, const float2* tab) const { return weight(to_f<TT>(p[i]), mp, c, tab); }
  // max(p_i - q_i, 0), times the sum of p's weights
  __device__ __forceinline__ Two residual(int i, const float2* tab) const {
    const Two a = at_p(i, tab);
    if (plain) return a;
    if (!q) return i == certain ? Two{0.f, 0.f} : a;
    const Two b = weight(to_f<TD>(q[i]), mq, c, tab);
    const float ph = __fmul_rn(rho.h, b.h), pl = __fmaf_rn(rho.h, b.h, -ph) + __fmaf_rn(rho.h, b.l, rho.l * b.h);
    const float s = __fsub_rn(a.h, ph), t = __fsub_rn(s, a.h);
    const float e = __fsub_rn(__fsub_rn(a.h, __fsub_rn(s, t)), __fadd_rn(ph, t));   // a.h - ph = s + e
    const float lo = e + __fsub_rn(a.l, pl), h = __fadd_rn(s, lo);
    if (!(h > 0.f)) return Two{0.f, 0.f};
    return Two{h, __fsub_rn(lo, __fsub_rn(h, s))};
  }
};

__device__ __forceinline__ double warp_sum2(double v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <typename TT, typename TD>
__global__ void __launch_bounds__(VD_THREADS) verify_decide_kernel(VerifyCall a, int n_split, const Stat* stats) {
  PDL_ENTRY();
  constexpr int WARPS = VD_THREADS / 32;
  __shared__ float2 tab[VD_TAB];
  __shared__ int s_first;
  __shared__ double s_part[3][VD_CTAS], s_warp[3][WARPS];
  __shared__ float s_mp, s_mq, s_z[2];
  __shared__ int s_at;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = cluster_rank(), b = (int)blockIdx.x / VD_CTAS;
  if (tid < VD_TAB) {
    const Two t = two_of(exp2((double)tid / VD_TAB));
    tab[tid] = make_float2(t.h, t.l);
  }
  cluster_barrier();   // (also: the others' shared memory is there)
  const SeqRows q = seq_rows(a, b);
  const float t = a.temp ? a.temp[b] : 1.f;
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
  const float cf = (float)log2_scale(t);
  auto joined = [&](int which, int r) {
    Running x;
    const Stat* s = stats + ((size_t)which * a.n_rows + r) * n_split;
    for (int i = 0; i < n_split; ++i) x.join(s[i].m, s[i].z, s[i].at, cf);
    return x;
  };
  const double inv_t = greedy ? 1.0 : 1.0 / (double)t;
  const double close = close_of(a.vocab, n_split);

  // how a row stands by its 32-bit sums; the last row, behind which there is no draft, stops
  enum { HOLDS = 0, STOPS = 1, CLOSE = 2, BAD = 3 };
  auto judge = [&](int i) {
    const int r = q.s + i;
    const Running p = joined(0, r);
    if (!(p.z > 0.f)) return (int)BAD;   // nothing above -infinity, a NaN, +infinity
    if (i == n - 1) return (int)STOPS;
    const int x = a.tokens[r + 1];
    if (x < 0 || x >= a.vocab) return (int)BAD;
    if (greedy) return p.at == x ? (int)HOLDS : (int)STOPS;
    const float u = a.u[r];
    if (!(u >= 0.f && u < 1.f)) return (int)BAD;
    double lq = 0.0;
    if (soft) {
      const Running d = joined(1, r);
      if (!(d.z > 0.f)) return (int)BAD;
      lq = ((double)to_f<TD>(((const TD*)a.draft)[r * a.ld_d + x]) - d.m) * inv_t - log((double)d.z);
    }
    const double lp = ((double)to_f<TT>(((const TT*)a.target)[r * a.ld_t + x]) - p.m) * inv_t - log((double)p.z);
    const double left = log((double)u) + lq;
    if (left > -INFINITY && lp > -INFINITY && fabs(left - lp) < close) return (int)CLOSE;
    return left < lp ? (int)HOLDS : (int)STOPS;
  };
  // the first row from `from` on that does not hold, and how it stands
  auto first_from = [&](int from, int& i, int& code) {
    __syncthreads();
    if (tid == 0) s_first = 0x7fffffff;
    __syncthreads();
    for (int k = from + tid; k < n; k += VD_THREADS) {
      const int c = judge(k);
      if (c != HOLDS) atomicMin(&s_first, k * 4 + c);
    }
    __syncthreads();
    i = s_first >> 2;
    code = s_first & 3;
  };
  int i, code;
  first_from(0, i, code);

  Row<TT, TD> row;
  row.c = two_of(log2_scale(t));
  const int share = (a.vocab + VD_CTAS - 1) / VD_CTAS, v0 = min(a.vocab, rank * share), v1 = min(a.vocab, v0 + share);
  const int each = ((share + WARPS - 1) / WARPS + 31) & ~31, w0 = min(v1, v0 + warp * each), w1 = min(v1, w0 + each);
  // sums over the vocabulary of up to two values a token, in every CTA; the warps' own in s_warp
  auto sums = [&](auto value, double& x, double& y) {
    Sum2 sx, sy;
    for (int k = w0 + lane; k < w1; k += 32) value(k, sx, sy);
    const double wx = warp_sum2(sx.value()), wy = warp_sum2(sy.value());
    __syncthreads();
    if (lane == 0) {
      s_warp[0][warp] = wx;
      s_warp[1][warp] = wy;
    }
    __syncthreads();
    if (tid < 2 * VD_CTAS) {
      const int which = tid / VD_CTAS, to = tid % VD_CTAS;
      double s = 0;
      for (int w = 0; w < WARPS; ++w) s += s_warp[which][w];
      cluster_store(&s_part[which][rank], to, s);
    }
    cluster_barrier();
    x = y = 0;
    for (int k = 0; k < VD_CTAS; ++k) {
      x += s_part[0][k];
      y += s_part[1][k];
    }
    cluster_barrier();   // (s_part is free again)
  };
  double zp = 0, zq = 0;
  auto look = [&](int r) {   // maxima and precise sums of row r
    if (tid == 0) {
      const Running p = joined(0, r);
      s_mp = p.m;
      s_at = p.at;
      s_z[0] = p.z;
      if (soft && r < q.e - 1) s_mq = joined(1, r).m;
    }
    __syncthreads();
    row.p = (const TT*)a.target + r * a.ld_t;
    row.q = soft && r < q.e - 1 ? (const TD*)a.draft + r * a.ld_d : nullptr;
    row.mp = s_mp;
    row.mq = s_mq;
    if (greedy) return;
    sums([&](int k, Sum2& x, Sum2& y) {
      x.add(row.at_p(k, tab));
      if (row.q) y.add(weight(to_f<TD>(row.q[k]), row.mq, row.c, tab));
    }, zp, zq);
  };
  // drafts that are too close: decided by the precise sums
  while (code == CLOSE) {
    const int r = q.s + i, x = a.tokens[r + 1];
    look(r);
    const double lp = ((double)to_f<TT>(row.p[x]) - row.mp) * inv_t - log(zp);
    const double lq = row.q ? ((double)to_f<TD>(row.q[x]) - row.mq) * inv_t - log(zq) : 0.0;
    if (!(log((double)a.u[r]) + lq < lp)) {
      code = STOPS;
      break;
    }
    first_from(i + 1, i, code);
  }
  const float u_draw = a.u[q.e - 1];
  if (code == BAD || (!greedy && !(u_draw >= 0.f && u_draw < 1.f))) {
    if (rank == 0 && tid == 0) a.flag(ERRW_VALUE);
    give(-1, -1);
    return;
  }
  const int r = q.s + i;
  look(r);
  int nxt = s_at;
  if (!greedy) {
    row.certain = a.draft || r == q.e - 1 ? -1 : a.tokens[r + 1];
    row.plain = r == q.e - 1;
    row.rho = two_of(row.q ? zp / zq : 0.0);
    double all_w = zp, all_p = zp;
    sums([&](int k, Sum2& x, Sum2& y) {
      x.add(row.residual(k, tab));
      y.add(row.at_p(k, tab));
    }, all_w, all_p);
    const bool fall_back = !(all_w >= VD_LEAST * zp);
    if (fall_back) {
      row.plain = 1;
      all_w = all_p;
    }
    const int which = fall_back ? 1 : 0;
    const double at = ((double)u_draw + 2.98023223876953125e-08) * all_w;   // u in the middle of its 2^-24
    // the warp in whose run the sum passes `at`: the last run that begins at or below it and holds something
    __syncthreads();
    double mine = 0;
    for (int w = 0; w < WARPS; ++w) mine += s_warp[which][w];
    // (the parts were overwritten by no one since the sums: every CTA holds its own runs; the ranks' are exchanged again)
    if (tid < VD_CTAS) cluster_store(&s_part[2][rank], tid, mine);
    cluster_barrier();
    double before = 0;
    int owner = 0;
    double owner_before = 0, sum = 0;
    for (int k = 0; k < VD_CTAS; ++k) {
      if (s_part[2][k] > 0 && sum <= at) {
        owner = k;
        owner_before = sum;
      }
      sum += s_part[2][k];
    }
    before = owner_before;
    if (rank == owner) {
      int ow = 0;
      double ob = before, s = before;
      for (int w = 0; w < WARPS; ++w) {
        if (s_warp[which][w] > 0 && s <= at) {
          ow = w;
          ob = s;
        }
        s += s_warp[which][w];
      }
      if (warp == ow) {
        int best = -1;   // the last token with a weight so far: what rounding leaves
        double run = ob;
        for (int k0 = w0; k0 < w1; k0 += 32) {
          const int k = k0 + lane;
          double w = 0;
          if (k < w1) {
            const Two x = row.residual(k, tab);
            w = (double)x.h + (double)x.l;
          }
          double inc = w;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const double v = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += v;
          }
          const unsigned over = __ballot_sync(0xffffffffu, w > 0 && run + inc > at), some = __ballot_sync(0xffffffffu, w > 0);
          if (over) {
            best = k0 + __ffs(over) - 1;
            break;
          }
          if (some) best = k0 + 31 - __clz(some);
          run += __shfl_sync(0xffffffffu, inc, 31);
        }
        if (lane == 0 && best >= 0) {   // (the run holds something)
          a.accepted[b] = i;
          a.next[b] = best;
          if (a.logprob) a.logprob[r] = (float)(((double)to_f<TT>(row.p[best]) - row.mp) * inv_t - log(zp));
        }
      }
    }
  } else {
    give(i, nxt);
    if (a.logprob && rank == 0 && tid == 0) a.logprob[r] = (float)-log((double)s_z[0]);
  }
  if (a.logprob && rank == 0) {
    for (int k = tid; k < i; k += VD_THREADS) {
      const Running p = joined(0, q.s + k);
      const int x = a.tokens[q.s + k + 1];
      a.logprob[q.s + k] = (float)(((double)to_f<TT>(((const TT*)a.target)[(q.s + k) * a.ld_t + x]) - p.m) * inv_t - log((double)p.z));
    }
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

// Parts of a row: enough CTAs to fill the GPU, each with a few rounds of its threads.
int verify_target() { return 4 * verify_sms(); }
int verify_splits(int n_rows, int vocab) {
  const int want = cdiv(verify_target(), n_rows), most = vocab / (VS_THREADS * 8) + 1;
  return want < most ? want : most;
}

template <typename TT, typename TD>
cudaError_t verify_t(cudaStream_t st, const VerifyCall& a) {
  const int s = a.n_rows > 0 ? verify_splits(a.n_rows, a.vocab) : 1;
  Stat* stats = (Stat*)a.ws;
  if (a.n_rows > 0) {
    const cudaError_t e = launch_k(verify_stats_kernel<TT, TD>, dim3((unsigned)(a.n_rows * s), a.draft ? 2 : 1), dim3(VS_THREADS), 0, st, a, s, stats);
    if (e != cudaSuccess) return e;
  }
  return launch_cluster(verify_decide_kernel<TT, TD>, a.n_seq * VD_CTAS, VD_CTAS, VD_THREADS, 0, st, a, s, (const Stat*)stats);
}

}  // namespace

// (n_rows times the parts of a row is at most this; a smaller call needs no more)
size_t verify_workspace(int n_rows) { return (size_t)2 * (verify_target() + (size_t)n_rows) * sizeof(Stat); }

cudaError_t launch_verify(cudaStream_t st, const VerifyCall& a) {
  if (a.t_bf16) return a.d_bf16 ? verify_t<bf16, bf16>(st, a) : verify_t<bf16, float>(st, a);
  return a.d_bf16 ? verify_t<float, bf16>(st, a) : verify_t<float, float>(st, a);
}

}  // namespace adept
