// Softmax attention with capped, biased and masked scores: what all its kernels share.
//
//   s_ij = scale q_i . k_j;   with a cap c: s = c tanh(s / c);   with slopes: s -= slope_h |p_i - j|
//   A_ij = exp(s_ij - lse_i) over the pairs that the masks leave, lse_i = log sum_j exp(s_ij);   O_i = sum_j A_ij v_j
//   delta_i = dO_i . O_i;  ds_ij = A_ij (dO_i . v_j - delta_i) (1 - tanh^2) scale;
//   dV_j = sum_i A_ij dO_i;  dQ_i = sum_j ds_ij k_j;  dK_j = sum_i ds_ij q_i     (sums over the query heads of a key head)
// Query i stands at key position p_i = i + len - nq, len = kv_len of its batch element (or nk).  A pair is allowed if
//   j < len,  and with `causal`: j <= p_i or j < prefix,  and with documents: doc_q[i] == doc_k[j] >= 0.
// A row that the masks leave empty has O = 0, lse = -inf and no gradient.
// Scores live in base 2: x = s log2(e), so that an exponential is one ex2.
#pragma once
#include "ln_common.cuh"

namespace ln {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct SmView { void* p; long long b, h, t; };          // [B, H, n, d], strides of batch, head, token in elements, channels adjacent

struct SmArgs {
  SmView q, k, v, o, dout, dq, dk, dv;
  float* lse;                                           // [B, Hq, nq]
  float* delta;                                         // [B, Hq, nq] (backward, workspace)
  int B, Hq, Hk, group /* Hq / Hk */, nq, nk, d;
  float scale, cap;                                     // cap 0: none
  int causal;
  const int* prefix; const int* kv_len;                 // [B] or NULL
  const float* slopes;                                  // [Hq] or NULL
  const int* doc_q; const int* doc_k;                   // [B, nq], [B, nk] or both NULL
  const int4* rq; const int4* rk;                       // per 64 tokens: smallest and largest document (min > max: none), padding?
  int tq, tk;                                           // ceil(nq / 64), ceil(nk / 64)
  int* dev_status;
};

// What a batch element's masks come down to.
struct SmMask {
  int len, off, pre, causal;
  __device__ __forceinline__ SmMask(const SmArgs& a, int b) {
    len = a.kv_len ? min(max(a.kv_len[b], 0), a.nk) : a.nk;
    off = len - a.nq;
    causal = a.causal;
    pre = a.causal && a.prefix ? min(max(a.prefix[b], 0), len) : 0;
  }
  // keys that query i may see are [0, limit(i)); limit grows with i
  __device__ __forceinline__ int limit(int i) const { return causal ? max(min(i + off + 1, len), pre) : len; }
  // queries that may see key j (< len) are [first(j), nq)
  __device__ __forceinline__ int first(int j) const { return causal && j >= pre ? j - off : 0; }
};

// Documents of the 64-token tiles [t0, t1) as one entry.
__device__ __forceinline__ int4 sm_docs(const int4* r, int t0, int t1) {
  int4 m = r[t0];
  for (int t = t0 + 1; t < t1; ++t) {
    const int4 e = r[t];
    m.x = min(m.x, e.x); m.y = max(m.y, e.y); m.z |= e.z;
  }
  return m;
}
__device__ __forceinline__ bool sm_meet(const int4& a, const int4& b) { return a.x <= a.y && b.x <= b.y && a.x <= b.y && b.x <= a.y; }

// Smallest and largest document id of every 64 tokens; negative ids are padding.  Grid (tiles, B), one warp.
__global__ void __launch_bounds__(32) k_sm_docs(const int* __restrict__ dq, const int* __restrict__ dk, int nq, int nk, int tq, int tk,
                                               int4* __restrict__ rq, int4* __restrict__ rk) {
  pdl_wait();
  const bool key = (int)blockIdx.x >= tq;
  const int t = key ? blockIdx.x - tq : blockIdx.x, b = blockIdx.y, n = key ? nk : nq;
  const int* d = (key ? dk : dq) + (long long)b * n;
  int lo = 0x7fffffff, hi = -1, pad = 0;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = t * 64 + u * 32 + threadIdx.x;
    if (i >= n) continue;
    const int id = d[i];
    if (id < 0) { pad = 1; continue; }
    lo = min(lo, id); hi = max(hi, id);
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  pad = __reduce_or_sync(0xffffffffu, pad);
  if (threadIdx.x == 0) (key ? rk : rq)[(long long)b * (key ? tk : tq) + t] = make_int4(lo, hi, pad, 0);
}

// The moving 64-token tiles [lo, hi) that the stationary rows [s0, s0 + S) of a CTA can meet: keys for stationary queries
// (KEYS false), queries for stationary keys (KEYS true).  Called by all threads; sh: 2 ints of shared memory.
template <int S, bool KEYS>
__device__ __forceinline__ int2 sm_range(const SmArgs& a, const SmMask& m, int b, int s0, int* sh) {
  int lo = 0, hi = 0;
  if (KEYS) {
    if (s0 < m.len) { lo = max(m.first(s0), 0) / 64; hi = a.tq; }
  } else {
    hi = (max(m.limit(min(s0 + S, a.nq) - 1), 0) + 63) / 64;
  }
  if (!a.rq) return make_int2(lo, max(lo, hi));
  const int4* rs = (KEYS ? a.rk + (long long)b * a.tk : a.rq + (long long)b * a.tq);
  const int4* rm = (KEYS ? a.rq + (long long)b * a.tq : a.rk + (long long)b * a.tk);
  const int4 mine = sm_docs(rs, s0 / 64, min((s0 + S) / 64, KEYS ? a.tk : a.tq));
  __syncthreads();
  if (threadIdx.x == 0) { sh[0] = 0x7fffffff; sh[1] = 0; }
  __syncthreads();
  int first = 0x7fffffff, last = 0;
  for (int t = lo + threadIdx.x; t < hi; t += blockDim.x)
    if (sm_meet(mine, rm[t])) { first = min(first, t); last = t + 1; }
  if (last) { atomicMin(sh, first); atomicMax(sh + 1, last); }      // integer extremes: the order does not matter
  __syncthreads();
  lo = sh[0]; hi = sh[1];
  __syncthreads();
  return hi ? make_int2(lo, hi) : make_int2(0, 0);
}

// Whether the masks leave every pair of queries [i0, i1) and keys [j0, j1) (all in range).
__device__ __forceinline__ bool sm_whole(const SmArgs& a, const SmMask& m, int b, int i0, int i1, int j0, int j1) {
  if (i1 > a.nq || j1 > m.limit(i0)) return false;
  if (!a.rq) return true;
  const int4 x = sm_docs(a.rq + (long long)b * a.tq, i0 / 64, (i1 + 63) / 64), y = sm_docs(a.rk + (long long)b * a.tk, j0 / 64, (j1 + 63) / 64);
  return x.x == x.y && y.x == y.y && x.x == y.x && !x.z && !y.z;
}

}  // namespace ln
