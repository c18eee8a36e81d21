// Rotary positions on queries and keys, alone or behind an RMS norm of every head, and their adjoints.
//
//   y = rope(w),  w = x (rope alone)  or  w_c = g_c x_c rstd,  rstd = (mean_c x_c^2 + eps)^(-1/2)
//   rope turns the channel pairs of the first r channels, (2i, 2i+1) or (i, i + r/2), by the angle t_i = 2 pi pos turns_i:
//     (u, v) = f (a cos t - b sin t, a sin t + b cos t);    the other channels are copied
//   adjoint: q = rope^T(dy) (angle -t);  dg_c = sum q_c x_c rstd;  p = q g;  dx = rstd p - x rstd^3 mean_c(p_c x_c)
//
// Bound by memory traffic: every tensor is read or written once, in 16-byte pieces.  A row (token, head) belongs to
// LPR = d * sizeof(T) / 16 adjacent lanes, one piece each, so that the sums over a head are a few shuffles and the partner of
// the half layout is r/2 channels = a whole number of lanes away.  A lane group keeps its token and walks the heads of Q and K:
// sine and cosine are formed once per (token, pair) and lane, and stay in registers.
//
// Angles: the table holds turns per position as a 64-bit binary fraction, so pos * turns modulo 2^64 is the fraction of a turn
// with an error below pos * 2^-64 whatever the position (a 32-bit product would be off by 0.06 rad at a million).  What is
// rounded to 32 bits is the remainder within half a turn.
#pragma once
#include "ln_common.cuh"

namespace ln {

struct QkTensor {                     // one of Q, K: x [B, H, n, d] in, y out, dy the gradient of y (backward); strides in elements
  const void* x; const void* dy; void* y;
  long long xs[3], ds[3], ys[3];      // batch, head, token
  const float* g;                     // [d] gain or NULL = ones
  int H;
};
struct QkArgs {
  QkTensor t[2];
  const int* pos; long long pos_b, pos_n;       // position of (b, token) at pos[b pos_b + token pos_n]; NULL: start + token
  int start, tokens /* B n */, n, r, heads /* of both tensors */, hpg /* heads per lane group */, chunks /* ceil(heads / hpg) */;
  const unsigned long long* turns;              // [r / 2]
  float factor, sign, eps;
  float* dgpart;                                // [CTA][2][d] partial gain gradients (backward with gains)
};

template <typename T> struct Piece;             // 16 bytes of a row
template <> struct Piece<float> {
  static constexpr int E = 4;
  static __device__ __forceinline__ void open(const uint4& w, float (&v)[4]) {
    v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ uint4 close(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
};
template <> struct Piece<bf16> {
  static constexpr int E = 8;
  static __device__ __forceinline__ void open(const uint4& w, float (&v)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(u[e] << 16); v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u); }
  }
  static __device__ __forceinline__ uint4 close(const float (&v)[8]) {     // the one rounding to the storage type
    uint32_t u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
      u[e] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
};

enum { QK_ROPE = 0, QK_NORM = 1, QK_NORM_BWD = 2 };

// Sine and cosine of 2 pi part / 2^32.  The nearest quarter turn comes off in integers, exactly; the rest, within an eighth of a turn,
// goes through the Taylor series to degree 9 and 8 (remainders below 2e-9 and 3e-8), two roundings more: about 2^-23.  Against sincospif:
// 8 x 50176 tokens of four heads with 64 channels 104.6 -> 99.1 us, of ten heads with 128 channels 70.7 -> 69.4, with the norm 94.8 -> 92.4.
__device__ __forceinline__ void turn_sincos(uint32_t part, float& sn, float& cs) {
  const uint32_t quarter = part + (1u << 29);                              // its top two bits: the nearest quarter turn
  const float x = (float)((int)(part - (quarter & 0xc0000000u))) * 1.4629180792671596e-9f;     // 2 pi 2^-32
  const float z = x * x;
  float s = fmaf(z, 2.7557319e-6f, -1.9841270e-4f), c = fmaf(z, 2.4801587e-5f, -1.3888889e-3f);
  s = fmaf(s, z, 8.3333333e-3f);
  c = fmaf(c, z, 4.1666667e-2f);
  s = fmaf(s, z, -1.6666667e-1f);
  c = fmaf(c, z, -0.5f);
  s = fmaf(s * z, x, x);
  c = fmaf(c, z, 1.f);
  const bool odd = quarter & 0x40000000u;
  const uint32_t s_sign = quarter & 0x80000000u, c_sign = (quarter + 0x40000000u) & 0x80000000u;
  sn = __uint_as_float(__float_as_uint(odd ? c : s) ^ s_sign);
  cs = __uint_as_float(__float_as_uint(odd ? s : c) ^ c_sign);
}

// LPR lanes per row; INTER: interleaved layout.  256 threads.  U heads of a lane group are in flight at a time, with four CTAs an SM
// (two for the backward pass, whose sums over rows stay in registers).  16 x 4096 tokens of 16 heads with 128 channels, us, floor 82
// at the copy rate: rotation 100 (eight in flight and three CTAs 122, two and five CTAs 120); with the norm, 10 heads, floor 51: 92
// (four in flight 120), backward, floor 77: 130 (three CTAs 181).  fp32, 10 heads, floors 102, 102 and 154:
// 107, 135 and 219.
template <typename T, int LPR, bool INTER, int MODE>
__global__ void __launch_bounds__(256, MODE == QK_NORM_BWD ? 2 : 4) k_qk_rope(const __grid_constant__ QkArgs a) {
  pdl_wait();
  constexpr int E = Piece<T>::E, D = LPR * E, TPW = 32 / LPR, U = MODE == QK_ROPE ? 4 : 2;
  const int lane = threadIdx.x & 31, lr = lane % LPR, c0 = lr * E;
  const int warp = blockIdx.x * 8 + (threadIdx.x >> 5), warps = gridDim.x * 8;
  const bool turned = c0 < a.r;
  // the lane that holds the partners of the half layout, and the sign of their share
  const int hop = a.r / 2 / E;
  const int partner = !turned ? lane : (c0 < a.r / 2 ? lane + hop : lane - hop);
  const float psign = c0 < a.r / 2 ? -a.sign : a.sign;
  const unsigned long long* turns = a.turns + (!turned ? 0 : INTER ? c0 / 2 : (c0 < a.r / 2 ? c0 : c0 - a.r / 2));
  __shared__ __align__(16) float s_gain[2][D];
  const int pc0 = partner % LPR * E;
  if (MODE != QK_ROPE) {
    for (int e = threadIdx.x; e < 2 * D; e += 256) s_gain[e / D][e % D] = a.t[e / D].g ? a.t[e / D].g[e % D] : 1.f;
    __syncthreads();
  }
  float dg[2][E];
#pragma unroll
  for (int e = 0; e < E; ++e) dg[0][e] = dg[1][e] = 0.f;

  const int units = (a.tokens + TPW - 1) / TPW * a.chunks;
  for (int unit = warp; unit < units; unit += warps) {
    const int f = unit / a.chunks * TPW + lane / LPR;
    const bool live = f < a.tokens;
    const int b = live ? f / a.n : 0, tok = live ? f % a.n : 0;
    float co[INTER ? E / 2 : E], si[INTER ? E / 2 : E];
    {
      const long long p = a.pos ? a.pos[b * a.pos_b + tok * a.pos_n] : (long long)a.start + tok;
      if (turned)
#pragma unroll
        for (int e = 0; e < (INTER ? E / 2 : E); ++e) {
          turn_sincos((uint32_t)(((unsigned long long)p * __ldg(turns + e)) >> 32), si[e], co[e]);
          co[e] *= a.factor;
          si[e] *= a.factor * (INTER ? a.sign : psign);
        }
    }
    // w (this lane's channels) and, in the half layout, the partners' pw -> turned; other channels keep even an infinity
    auto turn = [&](float (&w)[E], const float (&pw)[E]) {
      if (!turned) return;
      if (INTER) {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          const float x = w[2 * e], y = w[2 * e + 1];
          w[2 * e] = fmaf(x, co[e], -y * si[e]);
          w[2 * e + 1] = fmaf(x, si[e], y * co[e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = fmaf(w[e], co[e], pw[e] * si[e]);
      }
    };
    auto across = [&](const uint4& v) {
      return make_uint4(__shfl_sync(0xffffffffu, v.x, partner), __shfl_sync(0xffffffffu, v.y, partner),
                        __shfl_sync(0xffffffffu, v.z, partner), __shfl_sync(0xffffffffu, v.w, partner));
    };
    auto row_sum = [&](float s) {
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      return s;
    };
    const int h0 = unit % a.chunks * a.hpg, h1 = min(a.heads, h0 + a.hpg), hq = a.t[0].H;
    if (MODE != QK_NORM_BWD) {
      // heads of Q and of K alike, U of them in flight
      const T *x[2], *xe;
      T *y[2], *ye;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        x[s] = static_cast<const T*>(a.t[s].x) + b * a.t[s].xs[0] + tok * a.t[s].xs[2] + c0;
        y[s] = static_cast<T*>(a.t[s].y) + b * a.t[s].ys[0] + tok * a.t[s].ys[2] + c0;
      }
      for (int h = h0; h < h1; h += U) {
        uint4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int k = h + u;
          xe = k < hq ? x[0] + k * a.t[0].xs[1] : x[1] + (k - hq) * a.t[1].xs[1];
          v[u] = make_uint4(0u, 0u, 0u, 0u);
          if (live && k < h1) v[u] = *reinterpret_cast<const uint4*>(xe);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int k = h + u;
          if (k >= h1) break;                                   // the same for the whole warp
          float w[E], pw[E];
          Piece<T>::open(v[u], w);
          if (!INTER) Piece<T>::open(across(v[u]), pw);
          if (MODE == QK_NORM) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) ss = fmaf(w[e], w[e], ss);
            const float rstd = rsqrtf(row_sum(ss) * (1.f / D) + a.eps);
            const float* g = &s_gain[k < hq ? 0 : 1][0];
#pragma unroll
            for (int e = 0; e < E; e += 4) {
              const float4 t = *reinterpret_cast<const float4*>(g + c0 + e);
              w[e] *= t.x * rstd; w[e + 1] *= t.y * rstd; w[e + 2] *= t.z * rstd; w[e + 3] *= t.w * rstd;
              if (!INTER) {
                const float4 q = *reinterpret_cast<const float4*>(g + pc0 + e);
                pw[e] *= q.x * rstd; pw[e + 1] *= q.y * rstd; pw[e + 2] *= q.z * rstd; pw[e + 3] *= q.w * rstd;
              }
            }
          }
          turn(w, pw);
          ye = k < hq ? y[0] + k * a.t[0].ys[1] : y[1] + (k - hq) * a.t[1].ys[1];
          if (live) *reinterpret_cast<uint4*>(ye) = Piece<T>::close(w);
        }
      }
      continue;
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const QkTensor& t = a.t[s];
      const int first = s ? hq : 0;
      const int g0 = max(h0 - first, 0), g1 = min(h1 - first, t.H);
      if (g0 >= g1) continue;                                   // the same for the whole warp
      const T* x = static_cast<const T*>(t.x) + b * t.xs[0] + tok * t.xs[2] + c0;
      const T* dy = static_cast<const T*>(t.dy) + b * t.ds[0] + tok * t.ds[2] + c0;
      T* y = static_cast<T*>(t.y) + b * t.ys[0] + tok * t.ys[2] + c0;
      for (int h = g0; h < g1; h += U) {
        uint4 xv[U], dv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          xv[u] = dv[u] = make_uint4(0u, 0u, 0u, 0u);
          if (live && h + u < g1) {
            xv[u] = *reinterpret_cast<const uint4*>(x + (h + u) * t.xs[1]);
            dv[u] = *reinterpret_cast<const uint4*>(dy + (h + u) * t.ds[1]);
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (h + u >= g1) break;                               // the same for the whole warp
          float w[E], q[E], pq[E], g[E];
          Piece<T>::open(xv[u], w);
          Piece<T>::open(dv[u], q);
          if (!INTER) Piece<T>::open(across(dv[u]), pq);
          turn(q, pq);
#pragma unroll
          for (int e = 0; e < E; e += 4) {
            const float4 v = *reinterpret_cast<const float4*>(&s_gain[s][c0 + e]);
            g[e] = q[e] * v.x; g[e + 1] = q[e + 1] * v.y; g[e + 2] = q[e + 2] * v.z; g[e + 3] = q[e + 3] * v.w;
          }
          float ss = 0.f, px = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) { ss = fmaf(w[e], w[e], ss); px = fmaf(g[e], w[e], px); }
          ss = row_sum(ss); px = row_sum(px);
          const float rstd = live ? rsqrtf(ss * (1.f / D) + a.eps) : 0.f;   // no row: nothing for dg
          const float k = px * (1.f / D) * rstd * rstd * rstd;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            dg[s][e] = fmaf(q[e], w[e] * rstd, dg[s][e]);
            w[e] = fmaf(g[e], rstd, -w[e] * k);
          }
          if (live) *reinterpret_cast<uint4*>(y + (h + u) * t.ys[1]) = Piece<T>::close(w);
        }
      }
    }
  }
  if (MODE == QK_NORM_BWD && a.dgpart) {
    // the CTA's rows, added in a fixed order: lane groups of a warp by shuffles, warps through shared memory
    __shared__ float red[8][2][D];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float v = dg[s][e];
#pragma unroll
        for (int o = LPR; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane < LPR) red[threadIdx.x >> 5][s][c0 + e] = v;
      }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += 256) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) v += red[w][i / D][i % D];
      a.dgpart[(long long)blockIdx.x * 2 * D + i] = v;
    }
  }
}

// dg[s][c] = sum over the CTAs of part[cta][s][c], in double and in a fixed order.  One CTA per 32 of the 2 d sums: warp w adds the
// CTAs w, w + 32, ..., four loads in flight, and the warps are added in order.
__global__ void __launch_bounds__(1024) k_gain_sum(const float* __restrict__ part, int ctas, int d, float* __restrict__ dgq, float* __restrict__ dgk) {
  pdl_wait();
  __shared__ double red[32][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
  double s = 0.0;
#pragma unroll 4
  for (int p = w; p < ctas; p += 32) s += (double)part[(long long)p * 2 * d + i];
  red[w][lane] = s;
  __syncthreads();
  if (w) return;
#pragma unroll
  for (int k = 1; k < 32; ++k) s += red[k][lane];
  float* o = i < d ? dgq : dgk;
  if (o) o[i % d] = (float)s;
}

}  // namespace ln
