// Softmax attention on the 5th-generation tensor cores (tcgen05 + TMEM), bf16 storage, forward.
//
// One CTA = two tiles of 128 queries of one head; the keys stream through shared memory in tiles of 128, copied by TMA.
//   S_t = Q_t K^T          (128 x 128, K = d)   both operands in shared memory, result in TMEM
//   A_t = exp2(x - ref)    a thread owns a row: no shuffles; rounded to bf16 and written over S_t in TMEM
//   O_t (+)= A_t V         (128 x d, K = 128)   left operand in TMEM, accumulator in TMEM
// Warps 0-3 and 4-7 form the exponentials of tile 0 and 1, warp 8 copies, warp 9 issues the products.  While one tile's
// exponentials are formed the tensor core works for the other tile.
// The reference of a row's exponentials is a maximum that is only renewed when the true one has grown by more than 8 (base 2):
// the accumulator is then rescaled in TMEM, which is rare; A stays below 2^8, whose rounding to bf16 is the same half step, and
// row sums are kept in 32 bits.  A enters the product rounded to bf16 (2^-8 of its value), as Q, K and V are.
// Bound: 4 * 128 * 128 * d operations on the tensor core against 128 * 128 exponentials (16 a clock and SM; 2 more special
// functions with a cap): at d = 128 both take 1024 clocks a tile, at d = 64 the exponentials are the longer part.
#pragma once
#include "ln_softmax.cuh"
#include "ln_tile_umma.cuh"

namespace ln {

// score of a pair in base 2 from the product, the distance's share taken off; CAP: x = cap log2(e) tanh(dot scale / cap), with
// tanh(y) = 1 - 2 / (exp(2 y) + 1): off by 2^-22 of the cap, where an approximate tanh would be off by 2^-11 of it
struct SmScore { float mul, cap2, slope2; };
__device__ __forceinline__ SmScore sm_score_of(const SmArgs& a, int h) {
  SmScore s;
  s.mul = a.cap > 0.f ? 2.f * kLog2e * a.scale / a.cap : a.scale * kLog2e;
  s.cap2 = a.cap * kLog2e;
  s.slope2 = a.slopes ? a.slopes[h] * kLog2e : 0.f;
  return s;
}
__device__ __forceinline__ float rcp_fast(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
// r = 1 / (exp(2 y) + 1); tanh(y) = 1 - 2 r, 1 - tanh(y)^2 = 4 r (1 - r)
__device__ __forceinline__ float sm_cap_r(float dot, const SmScore& s) { return rcp_fast(ex2(dot * s.mul) + 1.f); }

constexpr int SU_THREADS = 320;
template <int D> struct SuFwd {
  static constexpr int kTile = 128 * D * 2;                       // bytes of a 128-row tile
  static constexpr int kStages = D == 64 ? 4 : 2;
  static constexpr size_t kSmem = 1024 + (size_t)kTile * (2 + 2 * kStages);
};

// Rows r of a tile with keep(r) false become zeros (a whole warp; a row stays within its 128 bytes under the swizzle).
template <int D, typename F> __device__ __forceinline__ void tile_clear(char* tile, int rows, F keep) {
  for (int r = threadIdx.x & 31; r < rows; r += 32)
    if (!keep(r))
#pragma unroll
      for (int blk = 0; blk < D / 64; ++blk)
#pragma unroll
        for (int p = 0; p < 8; ++p) *reinterpret_cast<uint4*>(tile + (blk * rows + r) * 128 + p * 16) = make_uint4(0u, 0u, 0u, 0u);
  umma::fence_smem_to_mma();
  __syncwarp();
}

// x[0..31] of a row, keys j0 + c0 ..: -infinity where the masks leave nothing (lim: the row's limit minus j0 + c0)
__device__ __forceinline__ void sm_mask32(float* x, int lim, const int* dk, int doc, int j, int nk) {
#pragma unroll
  for (int e = 0; e < 32; ++e)
    if (e >= lim) x[e] = -INFINITY;
  if (dk) {
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      const int id = j + e < nk ? __ldg(dk + j + e) : -1;          // the same address for the whole warp
      if (id != doc) x[e] = -INFINITY;
    }
  }
}

// A bounded wait whose outcome is the same in every lane.
__device__ __forceinline__ bool warp_wait(unsigned long long* bar, uint32_t parity) { return __all_sync(0xffffffffu, umma::mbar_wait(bar, parity)); }

template <int D, bool CAP, bool BIAS>
__global__ void __launch_bounds__(SU_THREADS, 1) k_softmax_fwd_umma(const __grid_constant__ SmArgs a, const __grid_constant__ TileMap mq,
                                                                  const __grid_constant__ TileMap mk, const __grid_constant__ TileMap mv) {
  pdl_wait();
  constexpr int NS = SuFwd<D>::kStages, TB = SuFwd<D>::kTile;
  extern __shared__ __align__(16) char su_smem[];
  char* base = su_smem + ((1024u - (umma::s32(su_smem) & 1023u)) & 1023u);
  char *sQ = base, *sK = base + 2 * TB, *sV = sK + NS * TB;
  __shared__ unsigned long long q_full, k_full[NS], k_free[NS], v_full[NS], v_free[NS], v_raw, s_full[2], p_ready[2], o_full[2], spare;
  __shared__ uint32_t tmem_slot;
  __shared__ int sh[2];
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int bh = blockIdx.x, b = bh / a.Hq, h = bh % a.Hq, hk = h / a.group;
  const int i0 = ((int)gridDim.y - 1 - (int)blockIdx.y) * 256;                 // long causal rows first
  const SmMask m(a, b);
  const int2 range = sm_range<256, false>(a, m, b, i0, sh);
  const int nt = (range.y - range.x + 1) / 2, k0 = range.x * 64;             // key tiles of 128 from k0
  if (tid == 0) {
    umma::mbar_init(&q_full, 1); umma::mbar_init(&v_raw, 1); umma::mbar_init(&spare, 1);
    for (int s = 0; s < NS; ++s) {
      umma::mbar_init(&k_full[s], 1); umma::mbar_init(&k_free[s], 1); umma::mbar_init(&v_full[s], 1); umma::mbar_init(&v_free[s], 1);
    }
    for (int t = 0; t < 2; ++t) { umma::mbar_init(&s_full[t], 1); umma::mbar_init(&p_ready[t], 4); umma::mbar_init(&o_full[t], 1); }
  }
  if (warp == 9) umma::tmem_alloc(&tmem_slot, 512);
  umma::fence_before_sync();
  __syncthreads();
  umma::fence_after_sync();
  const uint32_t tm = tmem_slot;
  const int* dk = a.doc_k ? a.doc_k + (long long)b * a.nk : nullptr;
  bool ok = true;

  if (warp == 8) {                                                           // copies
    const bool one = umma::elect_one();
    const int qh = h * mq.head, qb = b * mq.batch, kh = hk * mk.head, kb = b * mk.batch, vh = hk * mv.head, vb = b * mv.batch;
    if (nt > 0 && one) {
      umma::mbar_expect_tx(&q_full, 2 * TB);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int blk = 0; blk < D / 64; ++blk)
          umma::tile_load(umma::s32(sQ) + t * TB + blk * 16384, &mq.map, blk * 64, i0 + t * 128, qh, qb, &q_full);
    }
    int raw = 0, j = 0;
    for (; j < nt && ok; ++j) {
      const int s = j % NS, j0 = k0 + j * 128;
      const uint32_t again = (uint32_t)(j / NS - 1) & 1;
      if (j >= NS) ok = warp_wait(&k_free[s], again);
      if (one && ok) {
        umma::mbar_expect_tx(&k_full[s], TB);
#pragma unroll
        for (int blk = 0; blk < D / 64; ++blk)
          umma::tile_load(umma::s32(sK) + s * TB + blk * 16384, &mk.map, blk * 64, j0, kh, kb, &k_full[s]);
      }
      if (j >= NS && ok) ok = warp_wait(&v_free[s], again);
      if (!ok) break;
      // a value row that no query uses may hold an infinity: rows behind the filled length, and padding, become zeros
      bool clear = j0 + 128 > m.len && m.len < a.nk;
      if (a.rk) clear |= sm_docs(a.rk + (long long)b * a.tk, j0 / 64, min(j0 / 64 + 2, a.tk)).z != 0;
      unsigned long long* bar = clear ? &v_raw : &v_full[s];
      if (one) {
        umma::mbar_expect_tx(bar, TB);
#pragma unroll
        for (int blk = 0; blk < D / 64; ++blk)
          umma::tile_load(umma::s32(sV) + s * TB + blk * 16384, &mv.map, blk * 64, j0, vh, vb, bar);
      }
      if (clear) {
        ok = warp_wait(&v_raw, raw++ & 1);
        tile_clear<D>(sV + s * TB, 128, [&](int r) { const int key = j0 + r; return key >= a.nk || (key < m.len && !(dk && dk[key] < 0)); });
        if (one) umma::mbar_arrive(&v_full[s]);
      }
    }
    if (!ok)                                                                 // no copy is in flight when the CTA ends
      for (int s = 0; s < NS; ++s) {
        const int last = (j - 1 - s) / NS;                                   // uses of stage s so far, less one
        if (j > s) { umma::mbar_wait(&k_full[s], last & 1); umma::mbar_wait(&v_full[s], last & 1); }
        if (j % NS == s && j < nt) umma::mbar_wait(&k_full[s], (j / NS) & 1, 1 << 12);
      }
  } else if (warp == 9) {                                                    // products
    if (umma::elect_one() && nt > 0) {
      const uint32_t id_s = umma::instr_desc(128, false, false), id_o = umma::instr_desc(D, false, true);
      const int steps = a.d / 16;
      const uint32_t qa = umma::s32(sQ), ka = umma::s32(sK), va = umma::s32(sV);
      auto scores = [&](int t, int s) {
        for (int ks = 0; ks < steps; ++ks)
          umma::mma(tm + t * 128, umma::rows_desc(qa + t * TB, 128, ks), umma::rows_desc(ka + s * TB, 128, ks), id_s, ks > 0);
        umma::commit(&s_full[t]);
      };
      ok = umma::mbar_wait(&q_full, 0) && umma::mbar_wait(&k_full[0], 0);
      umma::fence_after_sync();
      if (ok) { scores(0, 0); scores(1, 0); if (NS < nt) umma::commit(&k_free[0]); }
      for (int j = 0; j < nt && ok; ++j) {
        const int s = j % NS, s1 = (j + 1) % NS;
        ok = umma::mbar_wait(&v_full[s], (j / NS) & 1);
        if (ok && j + 1 < nt) ok = umma::mbar_wait(&k_full[s1], ((j + 1) / NS) & 1);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          ok = ok && umma::mbar_wait(&p_ready[t], j & 1);
          if (!ok) break;
          umma::fence_after_sync();
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            umma::mma_ta(tm + 256 + t * D, tm + t * 128 + ks * 8, umma::cols_desc(va + s * TB, 128, ks), id_o, j > 0 || ks > 0);
          if (j + 1 < nt) scores(t, s1);
          else umma::commit(&o_full[t]);
        }
        // only where the copying warp waits for it: no arrival is under way when the CTA ends
        if (ok && j + NS < nt) umma::commit(&v_free[s]);
        if (ok && j + 1 + NS < nt) umma::commit(&k_free[s1]);
      }
      if (!ok) { umma::commit(&spare); umma::mbar_wait(&spare, 0); }          // no product is in flight when the CTA ends
    }
  } else {                                                                   // exponentials
    const int t = warp >> 2, lane = tid & 31, row = (warp & 3) * 32 + lane, i = i0 + t * 128 + row;
    const uint32_t quarter = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tm + quarter + t * 128, to = tm + quarter + 256 + t * D;
    const int doc = a.doc_q && i < a.nq ? a.doc_q[(long long)b * a.nq + i] : 0;
    const int lim = i < a.nq && doc >= 0 ? m.limit(i) : 0;
    const SmScore sc = sm_score_of(a, h);
    float ref = -INFINITY, sum = 0.f;
    for (int j = 0; j < nt; ++j) {
      const int j0 = k0 + j * 128;
      const bool whole = sm_whole(a, m, b, i0 + t * 128, i0 + t * 128 + 128, j0, j0 + 128);
      ok = warp_wait(&s_full[t], j & 1);
      if (!ok) break;
      umma::fence_after_sync();
      float x[128];
#pragma unroll
      for (int c = 0; c < 4; ++c) umma::tmem_ld32_async(ts + c * 32, x + c * 32);
      umma::tmem_ld_wait();
#pragma unroll
      for (int c = 0; c < 4; ++c) umma::tie32(x + c * 32);
      if (CAP) {
#pragma unroll
        for (int e = 0; e < 128; ++e) x[e] = fmaf(-2.f * sc.cap2, sm_cap_r(x[e], sc), sc.cap2);
      }
      if (BIAS) {
        const float p = (float)(i + m.off - j0);
#pragma unroll
        for (int e = 0; e < 128; ++e) x[e] = fmaf(-sc.slope2, fabsf(p - (float)e), CAP ? x[e] : x[e] * sc.mul);
      }
      if (!whole) {
#pragma unroll
        for (int c = 0; c < 4; ++c) sm_mask32(x + c * 32, lim - j0 - c * 32, dk, doc, j0 + c * 32, a.nk);
      }
      float top[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
      for (int e = 4; e < 128; ++e) top[e & 3] = fmaxf(top[e & 3], x[e]);
      float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
      if (!(CAP || BIAS)) mx *= sc.mul;                                      // scale > 0: the largest product is the largest score
      const bool grown = mx > ref + 8.f;                                     // also the first finite maximum of a row
      if (__any_sync(0xffffffffu, grown)) {
        const float now = grown ? mx : ref;
        const float f = grown ? (ref == -INFINITY ? 0.f : ex2(ref - now)) : 1.f;
        ref = now;
        sum *= f;
        if (j > 0) {                                                         // every product into O is complete (s_full follows them)
#pragma unroll
          for (int c = 0; c < D; c += 32) {
            float o[32];
            uint32_t w[32];
            umma::tmem_ld32_async(to + c, o);
            umma::tmem_ld_wait();
            umma::tie32(o);
#pragma unroll
            for (int e = 0; e < 32; ++e) w[e] = __float_as_uint(o[e] * f);
            umma::tmem_st32(to + c, w);
          }
        }
      }
      const float shift = ref == -INFINITY ? 0.f : -ref;
      float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t w[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          const int u = c * 64 + 2 * e;
          const float p0 = ex2(CAP || BIAS ? x[u] + shift : fmaf(x[u], sc.mul, shift));
          const float p1 = ex2(CAP || BIAS ? x[u + 1] + shift : fmaf(x[u + 1], sc.mul, shift));
          part[(2 * e) & 3] += p0; part[(2 * e + 1) & 3] += p1;
          w[e] = umma::pack_bf16(p0, p1);
        }
        umma::tmem_st32(ts + c * 32, w);
      }
      sum += (part[0] + part[1]) + (part[2] + part[3]);
      umma::tmem_st_wait();
      umma::fence_before_sync();
      __syncwarp();
      if (lane == 0) umma::mbar_arrive(&p_ready[t]);
    }
    if (nt > 0) {
      ok = ok && warp_wait(&o_full[t], 0);
      umma::fence_after_sync();
    }
    if (ok) {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      // a warp's 32 rows go through its part of the query tile (no product reads it any more), 16-byte pieces swizzled by row
      char* stage = sQ + t * TB + (warp & 3) * 32 * D * 2;
      constexpr int PR = D / 8;                                              // pieces a row
#pragma unroll
      for (int c = 0; c < D; c += 32) {
        float o[32];
        if (nt > 0) {
          umma::tmem_ld32_async(to + c, o);
          umma::tmem_ld_wait();
          umma::tie32(o);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            w[e] = nt > 0 ? umma::pack_bf16(o[8 * q + 2 * e] * inv, o[8 * q + 2 * e + 1] * inv) : 0u;
          *reinterpret_cast<uint4*>(stage + (lane * PR + ((c / 8 + q) ^ (lane & 7))) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
      __syncwarp();
      bf16* O = static_cast<bf16*>(a.o.p) + b * a.o.b + h * a.o.h;
      const int first = i0 + t * 128 + (warp & 3) * 32, pieces = a.d / 8;
      for (int e = lane; e < 32 * pieces; e += 32) {
        const int r = e / pieces, p = e % pieces;
        if (first + r < a.nq)
          *reinterpret_cast<uint4*>(O + (first + r) * a.o.t + p * 8) = *reinterpret_cast<const uint4*>(stage + (r * PR + (p ^ (r & 7))) * 16);
      }
      if (i < a.nq) a.lse[(long long)bh * a.nq + i] = sum == 0.f ? -INFINITY : (ref + __log2f(sum)) * kLn2;
    }
  }
  __syncwarp();
  umma::fence_before_sync();
  __syncthreads();
  if (warp == 9) umma::tmem_dealloc(tm, 512);
  umma::report_timeout(ok, a.dev_status, bh);
}

}  // namespace ln
