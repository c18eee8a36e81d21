// Softmax attention on the CUDA cores, forward and backward, for fp32 storage (products with 24-bit operands).
// One CTA = 64 stationary rows; the moving rows stream through shared memory in tiles of 64.  256 threads, thread (ty, tx) of
// 16 x 16 owns rows 4 ty .. 4 ty + 3 and moving rows tx + 16 q of a 64 x 64 score tile, and D / 16 channels of its four
// accumulator rows.  Bound by the FP32 pipe: 4 d operations a pair forward, 14 d backward (the query pass and the key
// pass each form the scores again, so that no sum depends on the order of atomics).  32 heads of 784 tokens, causal, 64 channels:
// 122, 161 and 217 us, 30 % of the pipe: a 4 x 4 register tile reads shared memory once for every five multiply-adds.
#pragma once
#include "ln_softmax.cuh"

namespace ln {

constexpr int SS = 64, SSG = SS + 4;                       // tile edge; pitch of a score tile in shared memory
template <int D> __host__ __device__ constexpr size_t sm_fwd_smem() { return sizeof(float) * (size_t)(3 * SS * (D + 4) + SS * SSG); }
template <int D, bool KEYS> __host__ __device__ constexpr size_t sm_bwd_smem() { return sizeof(float) * (size_t)(4 * SS * (D + 4) + (KEYS ? 2 : 1) * SS * SSG + 2 * SS); }

// 64 rows of a [n, d] slab (row r0 first) into a tile with pitch D + 4; rows at or behind n and rows of padding are zero
// whatever they hold.
template <int D>
__device__ __forceinline__ void sm_tile(float* dst, const float* src, long long stride, int r0, int n, const int* doc) {
  for (int idx = threadIdx.x; idx < SS * (D / 4); idx += 256) {
    const int r = idx / (D / 4), c = idx % (D / 4) * 4, i = r0 + r;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < n && !(doc && doc[i] < 0)) v = ld4(src + (long long)i * stride + c);
    *reinterpret_cast<float4*>(dst + r * (D + 4) + c) = v;
  }
}

// s[k][q] = sum_c A[4 ty + k][c] B[tx + 16 q][c]; even and odd channels in the halves of a packed multiply-add, which takes one
// issue slot for both
template <int D>
__device__ __forceinline__ void sm_dots(const float* A, const float* B, int ty, int tx, float (&s)[4][4]) {
  f32x2 p[4][4];
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int q = 0; q < 4; ++q) p[k][q] = pack2(0.f, 0.f);
#pragma unroll 4
  for (int c = 0; c < D; c += 4) {
    ulonglong2 a[4], b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) a[k] = *reinterpret_cast<const ulonglong2*>(A + (ty * 4 + k) * (D + 4) + c);
#pragma unroll
    for (int q = 0; q < 4; ++q) b[q] = *reinterpret_cast<const ulonglong2*>(B + (tx + 16 * q) * (D + 4) + c);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int q = 0; q < 4; ++q) p[k][q] = fma2(a[k].y, b[q].y, fma2(a[k].x, b[q].x, p[k][q]));
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float lo, hi;
      unpack2(p[k][q], lo, hi);
      s[k][q] = lo + hi;
    }
}

// acc[k][.] += sum_j G[4 ty + k][j] B[j][channels of tx, in pairs]
template <int D>
__device__ __forceinline__ void sm_add(const float* G, const float* B, int ty, int tx, f32x2 (&acc)[4][D / 32]) {
#pragma unroll 2
  for (int j = 0; j < SS; j += 4) {
    float g[4][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 t = *reinterpret_cast<const float4*>(G + (ty * 4 + k) * SSG + j);
      g[k][0] = t.x; g[k][1] = t.y; g[k][2] = t.z; g[k][3] = t.w;
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      f32x2 v[D / 32];
      ld_col_pairs<D>(B + (j + s) * (D + 4), tx, v);
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int q = 0; q < D / 32; ++q) acc[k][q] = fma2(pack2(g[k][s], g[k][s]), v[q], acc[k][q]);
    }
  }
}

// Score of a pair in base 2, and 1 - tanh^2 of the cap (1 without).
__device__ __forceinline__ float sm_score(float dot, const SmArgs& a, float slope2, float dist, float& bend) {
  float x = dot * a.scale;
  bend = 1.f;
  if (a.cap > 0.f) {
    const float t = tanhf(x / a.cap);
    x = t * a.cap;
    bend = 1.f - t * t;
  }
  return fmaf(x, kLog2e, -slope2 * fabsf(dist));
}

template <int D>
__global__ void __launch_bounds__(256, D == 128 ? 1 : 2) k_softmax_fwd(const __grid_constant__ SmArgs a) {
  pdl_wait();
  extern __shared__ __align__(16) float sm_smem[];
  float *Qs = sm_smem, *Ks = Qs + SS * (D + 4), *Vs = Ks + SS * (D + 4), *Ps = Vs + SS * (D + 4);
  __shared__ int sh[2];
  const int b = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq, hk = h / a.group;
  const int i0 = ((int)gridDim.y - 1 - (int)blockIdx.y) * SS, tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;   // long causal rows first
  const float* Q = static_cast<const float*>(a.q.p) + b * a.q.b + h * a.q.h;
  const float* K = static_cast<const float*>(a.k.p) + b * a.k.b + hk * a.k.h;
  const float* V = static_cast<const float*>(a.v.p) + b * a.v.b + hk * a.v.h;
  const SmMask m(a, b);
  const int* dq = a.doc_q ? a.doc_q + (long long)b * a.nq : nullptr;
  const int* dk = a.doc_k ? a.doc_k + (long long)b * a.nk : nullptr;
  const float slope2 = a.slopes ? a.slopes[h] * kLog2e : 0.f;
  const int2 range = sm_range<SS, false>(a, m, b, i0, sh);
  sm_tile<D>(Qs, Q, a.q.t, i0, a.nq, nullptr);
  f32x2 acc[4][D / 32];
  float mx[4], sum[4];
  int lim[4], doc[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = i0 + ty * 4 + k;
    mx[k] = -INFINITY; sum[k] = 0.f;
    lim[k] = i < a.nq ? m.limit(i) : 0;
    doc[k] = dq && i < a.nq ? dq[i] : 0;
    if (doc[k] < 0) lim[k] = 0;
#pragma unroll
    for (int q = 0; q < D / 32; ++q) acc[k][q] = pack2(0.f, 0.f);
  }
  for (int t = range.x; t < range.y; ++t) {
    const int j0 = t * SS;
    __syncthreads();
    sm_tile<D>(Ks, K, a.k.t, j0, m.len, dk);
    sm_tile<D>(Vs, V, a.v.t, j0, m.len, dk);
    __syncthreads();
    float s[4][4] = {};
    sm_dots<D>(Qs, Ks, ty, tx, s);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float away = (float)(i0 + ty * 4 + k + m.off - j0 - tx);        // position of the query less that of key j0 + tx
      float top = -INFINITY;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int j = j0 + tx + 16 * q;
        float bend;
        const float x = sm_score(s[k][q], a, slope2, away - (float)(16 * q), bend);
        s[k][q] = j < lim[k] && (!dk || dk[j] == doc[k]) ? x : -INFINITY;
        top = fmaxf(top, s[k][q]);
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const float now = fmaxf(mx[k], top), ref = now == -INFINITY ? 0.f : now;
      const float old = ex2(mx[k] - ref);
      mx[k] = now;
      sum[k] *= old;
#pragma unroll
      for (int q = 0; q < D / 32; ++q) acc[k][q] = mul2(acc[k][q], pack2(old, old));
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float e = ex2(s[k][q] - ref);
        sum[k] += e;
        Ps[(ty * 4 + k) * SSG + tx + 16 * q] = e;
      }
    }
    __syncthreads();
    sm_add<D>(Ps, Vs, ty, tx, acc);
  }
  float* O = static_cast<float*>(a.o.p) + b * a.o.b + h * a.o.h;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], o);
    const int i = i0 + ty * 4 + k;
    if (i >= a.nq) continue;
    const float inv = sum[k] > 0.f ? 1.f / sum[k] : (sum[k] == 0.f ? 0.f : sum[k]);     // NaN stays
#pragma unroll
    for (int q = 0; q < D / 32; ++q) {
      float u, v;
      unpack2(mul2(acc[k][q], pack2(inv, inv)), u, v);
      O[i * a.o.t + ColMap<D>::col(tx, 2 * q)] = u;
      O[i * a.o.t + ColMap<D>::col(tx, 2 * q + 1)] = v;
    }
    if (tx == 0) a.lse[(long long)blockIdx.x * a.nq + i] = sum[k] == 0.f ? -INFINITY : mx[k] * kLn2 + logf(sum[k]);
  }
}

// KEYS false: stationary queries (X1 = Q, X2 = dO), moving keys (Y1 = K, Y2 = V): dQ, and delta for the other pass.
// KEYS true: stationary keys (X1 = K, X2 = V), moving queries (Y1 = Q, Y2 = dO) of every query head of the group: dK, dV.
template <int D, bool KEYS>
__global__ void __launch_bounds__(256, D == 128 ? 1 : 2) k_softmax_bwd(const __grid_constant__ SmArgs a) {
  pdl_wait();
  extern __shared__ __align__(16) float sm_smem[];
  constexpr int TF = SS * (D + 4);
  float *X1 = sm_smem, *X2 = X1 + TF, *Y1 = X2 + TF, *Y2 = Y1 + TF, *S = Y2 + TF, *P = S + SS * SSG, *L = S + (KEYS ? 2 : 1) * SS * SSG, *Dl = L + SS;
  __shared__ int sh[2];
  const int H = KEYS ? a.Hk : a.Hq, b = blockIdx.x / H, hs = blockIdx.x % H;
  const int tile = KEYS ? blockIdx.y : gridDim.y - 1 - blockIdx.y, s0 = tile * SS;      // long causal rows first
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const SmMask m(a, b);
  const int* dq = a.doc_q ? a.doc_q + (long long)b * a.nq : nullptr;
  const int* dk = a.doc_k ? a.doc_k + (long long)b * a.nk : nullptr;
  const int2 range = sm_range<SS, KEYS>(a, m, b, s0, sh);
  auto slab = [&](const SmView& v, int h) { return static_cast<const float*>(v.p) + b * v.b + h * v.h; };
  if (KEYS) {
    sm_tile<D>(X1, slab(a.k, hs), a.k.t, s0, m.len, dk);
    sm_tile<D>(X2, slab(a.v, hs), a.v.t, s0, m.len, dk);
  } else {
    sm_tile<D>(X1, slab(a.q, hs), a.q.t, s0, a.nq, dq);
    sm_tile<D>(X2, slab(a.dout, hs), a.dout.t, s0, a.nq, dq);
    // delta: row r = tid / 4, a quarter of the channels each
    const int r = tid >> 2, i = s0 + r;
    float v = 0.f;
    if (i < a.nq && !(dq && dq[i] < 0)) {
      const float* o = slab(a.o, hs) + (long long)i * a.o.t;
      const float* g = slab(a.dout, hs) + (long long)i * a.dout.t;
      for (int c = (tid & 3) * (D / 4); c < ((tid & 3) + 1) * (D / 4); c += 4) {
        const float4 x = ld4(o + c), y = ld4(g + c);
        v += x.x * y.x + x.y * y.y + x.z * y.z + x.w * y.w;
      }
    }
    v += __shfl_xor_sync(0xffffffffu, v, 1);
    v += __shfl_xor_sync(0xffffffffu, v, 2);
    if ((tid & 3) == 0) {
      Dl[r] = v;
      L[r] = i < a.nq ? a.lse[(long long)blockIdx.x * a.nq + i] * kLog2e : 0.f;
      if (i < a.nq) a.delta[(long long)blockIdx.x * a.nq + i] = v;
    }
  }
  f32x2 a1[4][D / 32], a2[4][D / 32];
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int q = 0; q < D / 32; ++q) a1[k][q] = a2[k][q] = pack2(0.f, 0.f);
  for (int h = KEYS ? hs * a.group : hs; h < (KEYS ? (hs + 1) * a.group : hs + 1); ++h) {
    const int hk = h / a.group;
    const float slope2 = a.slopes ? a.slopes[h] * kLog2e : 0.f;
    for (int t = range.x; t < range.y; ++t) {
      const int m0 = t * SS;
      __syncthreads();
      if (KEYS) {
        sm_tile<D>(Y1, slab(a.q, h), a.q.t, m0, a.nq, dq);
        sm_tile<D>(Y2, slab(a.dout, h), a.dout.t, m0, a.nq, dq);
        if (tid < SS) {
          const long long at = ((long long)b * a.Hq + h) * a.nq + m0 + tid;
          L[tid] = m0 + tid < a.nq ? a.lse[at] * kLog2e : 0.f;
          Dl[tid] = m0 + tid < a.nq ? a.delta[at] : 0.f;
        }
      } else {
        sm_tile<D>(Y1, slab(a.k, hk), a.k.t, m0, m.len, dk);
        sm_tile<D>(Y2, slab(a.v, hk), a.v.t, m0, m.len, dk);
      }
      __syncthreads();
      float s[4][4] = {}, g[4][4] = {};
      sm_dots<D>(X1, Y1, ty, tx, s);
      sm_dots<D>(X2, Y2, ty, tx, g);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        // position of the query less that of the key, moving row tx
        const float away = (float)(KEYS ? m0 + tx + m.off - (s0 + ty * 4 + k) : s0 + ty * 4 + k + m.off - (m0 + tx));
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int rs = ty * 4 + k, rm = tx + 16 * q, i = KEYS ? m0 + rm : s0 + rs, j = KEYS ? s0 + rs : m0 + rm, ri = KEYS ? rm : rs;
          const bool ok = i < a.nq && j < m.limit(i) && (!dk || (dq[i] >= 0 && dq[i] == dk[j]));
          float bend;
          const float x = sm_score(s[k][q], a, slope2, away + (KEYS ? (float)(16 * q) : -(float)(16 * q)), bend);
          const float p = ok ? ex2(x - L[ri]) : 0.f;
          const float ds = ok ? p * (g[k][q] - Dl[ri]) * bend * a.scale : 0.f;
          S[rs * SSG + rm] = ds;
          if (KEYS) P[rs * SSG + rm] = p;
        }
      }
      __syncthreads();
      sm_add<D>(S, Y1, ty, tx, a2);
      if (KEYS) sm_add<D>(P, Y2, ty, tx, a1);
    }
  }
  const SmView& o2 = KEYS ? a.dk : a.dq;
  float* g2 = static_cast<float*>(o2.p) + b * o2.b + hs * o2.h;
  float* g1 = KEYS ? static_cast<float*>(a.dv.p) + b * a.dv.b + hs * a.dv.h : nullptr;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = s0 + ty * 4 + k;
    if (i >= (KEYS ? a.nk : a.nq)) continue;
#pragma unroll
    for (int q = 0; q < D / 32; ++q) {
      float u, v;
      unpack2(a2[k][q], u, v);
      g2[i * o2.t + ColMap<D>::col(tx, 2 * q)] = u;
      g2[i * o2.t + ColMap<D>::col(tx, 2 * q + 1)] = v;
      if (KEYS) {
        unpack2(a1[k][q], u, v);
        g1[i * a.dv.t + ColMap<D>::col(tx, 2 * q)] = u;
        g1[i * a.dv.t + ColMap<D>::col(tx, 2 * q + 1)] = v;
      }
    }
  }
}

}  // namespace ln
