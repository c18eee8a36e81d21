// Softmax attention on the 5th-generation tensor cores (tcgen05 + TMEM), bf16 storage, forward.
//
// One CTA = T tiles of 128 queries of one head; the keys stream through shared memory in tiles of 128, copied by TMA.
//   S_t = Q_t K^T          (128 x 128, K = d)   both operands in shared memory, result in TMEM
//   A_t = exp2(x - ref)    a thread owns a row: no shuffles; rounded to bf16 and written over S_t in TMEM
//   O_t (+)= A_t V         (128 x d, K = 128)   left operand in TMEM, accumulator in TMEM
// Warps 4 t .. 4 t + 3 form the exponentials of tile t, one warp copies, one warp a tile issues the products (a wait costs some 200
// clocks beside the products' operand reads, and with one warp for both tiles each waited for the other's).  While one tile's
// exponentials are formed the tensor core works for the other one: of the same CTA (T = 2: each key tile is copied once for both)
// or of the other CTA on the SM (T = 1, with 64 channels, and for short rows, where starting and ending a CTA is most of it: 384
// heads of 197 tokens 39 -> 31 us).
// With 64 channels TMEM has room for A beside S: S of the next key tile is formed as soon as this one's is in registers.
// The reference of a row's exponentials is a maximum that is only renewed when the true one has grown by more than 8 (base 2):
// the accumulator is then rescaled in TMEM, which is rare; A stays below 2^8, whose rounding to bf16 is the same half step, and
// row sums are kept in 32 bits.  A enters the product rounded to bf16 (2^-8 of its value), as Q, K and V are.
// Key tiles come last first: with a distance bias the nearest keys then set the reference at once.
// Bound: 4 * 128 * 128 * d operations on the tensor core (1024 clocks a tile at d = 128) against 128 * 128 exponentials at 16 a
// clock and SM (1024 clocks; with a cap 1.25 more special functions each, see sm_cap4).  32 heads of 4096 tokens without masks: 128
// channels 269 to 300 us (0.92 to 1.02 PFLOP/s, a tile every 2100 clocks), with a cap of 20 579, with a bias 395 to 420; 64 channels 205, 406
// and 246.
#pragma once
#include "ln_softmax.cuh"
#include "ln_tile_umma.cuh"

namespace ln {

__device__ __forceinline__ float min_nan(float x, float y) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y)); return r; }
// Scores in base 2 from products (dot), through a value x: score = mid + down x.  Without a cap x is the product itself.  With one the
// score is cap log2(e) tanh(y), y = dot scale / cap, and tanh(y) = 1 - 2 r, x = r = 1 / (exp(2 y) + 1): off by 2^-22 of the cap (an approximate
// tanh would be off by 2^-11 of it), and 1 - tanh(y)^2 = 4 r (1 - r).  2^-22 of a cap above 128 is more than 2^-15 of a score of one and grows with
// the cap: there x is the score itself with its sign changed, from the product where y is small (see sm_cap4_wide).
// A branch on it in the kernels of smaller caps cost those 8 % (128 channels forward 581 -> 628 us), so wide caps have kernels of their own: 32
// heads of 4096 tokens, 128 channels, forward 823 us where smaller caps take 592, both backward passes 1314 and 1096.
constexpr float kWideCap = 128.f;
enum { CAP_NONE = 0, CAP_USUAL = 1, CAP_WIDE = 2 };
__host__ __device__ __forceinline__ int cap_kind(float cap) { return cap > kWideCap ? CAP_WIDE : cap > 0.f ? CAP_USUAL : CAP_NONE; }
struct SmScore { float mul, lin, cap2, slope2, down, mid; int kind; };
__device__ __forceinline__ SmScore sm_score_of(const SmArgs& a, int h) {
  SmScore s;
  s.kind = cap_kind(a.cap);
  s.lin = a.scale * kLog2e;
  s.mul = s.kind ? fminf(2.f * kLog2e * a.scale / a.cap, 3.4028235e38f) : s.lin;     // finite: a product of zero has to stay zero
  s.cap2 = a.cap * kLog2e;
  s.slope2 = a.slopes ? a.slopes[h] * kLog2e : 0.f;
  s.down = s.kind == CAP_USUAL ? -2.f * s.cap2 : s.kind ? -1.f : s.mul;
  s.mid = s.kind == CAP_USUAL ? s.cap2 : 0.f;
  return s;
}
__device__ __forceinline__ float rcp_fast(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
// dot products -> r, four at a time with one reciprocal: 1 / u = v / (u v).  exp(2 y) is held at 2^30 (r = 2^-30 there, tanh = 1 to
// 2^-29), so that a product of four stays in range.  One NaN makes all four NaN: they are scores of one row, and masked products are cleared before.
__device__ __forceinline__ void sm_cap4(float (&x)[4], float mul) {
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = min_nan(x[k] * mul, 30.f);
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = ex2(x[k]) + 1.f;
  const float u = x[0] * x[1], v = x[2] * x[3], r = rcp_fast(u * v), ru = r * v, rv = r * u;
  const float r0 = ru * x[1], r1 = ru * x[0], r2 = rv * x[3], r3 = rv * x[2];
  x[0] = r0; x[1] = r1; x[2] = r2; x[3] = r3;
}

// dot products -> scores with their sign changed, for wide caps.  Below |y| = 1/2 the score is the uncapped one times tanh(y) / y, its Taylor
// series to y^14 (remainder 1e-8): a few half steps of the score whatever the cap.  Beyond, cap (1 - 2 r) is as good.  A whole warp: the
// second form only where some lane needs it (its branch also keeps the compiler from spreading 32 of these over the registers: 728
// bytes of stack without).
__device__ __forceinline__ void sm_cap4_wide(float (&x)[4], const SmScore& s) {
  const float half = s.mul * (0.5f * kLn2);
  float n[4];
  bool near = true;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float y = x[k] * half, u = y * y;
    float p = fmaf(u, -1.4558344e-3f, 3.5921280e-3f);
    p = fmaf(p, u, -8.8632355e-3f);
    p = fmaf(p, u, 2.1869488e-2f);
    p = fmaf(p, u, -5.3968254e-2f);
    p = fmaf(p, u, 1.3333333e-1f);
    p = fmaf(p, u, -3.3333333e-1f);
    p = fmaf(p, u, 1.f);
    n[k] = -(x[k] * s.lin) * p;
    near = near && fabsf(y) < 0.5f;
  }
  if (!__all_sync(0xffffffffu, near)) {
    float r[4] = {x[0], x[1], x[2], x[3]};
    sm_cap4(r, s.mul);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (!(fabsf(x[k] * half) < 0.5f)) n[k] = fmaf(2.f * r[k], s.cap2, -s.cap2);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = n[k];
}

template <int D, int T> struct SuFwd {
  static constexpr int kTile = 128 * D * 2;                       // bytes of a 128-row tile
  static constexpr int kStages = T == 1 && D == 128 ? 1 : 2;
  static constexpr int kThreads = T * 160 + 32, kCtas = T == 1 ? 2 : 1;
  static constexpr int kTmem = T == 1 ? 256 : 512;
  static constexpr size_t kSmem = 1024 + (size_t)kTile * (T + 2 * kStages);
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

// A bounded wait whose outcome is the same in every lane.
__device__ __forceinline__ bool warp_wait(unsigned long long* bar, uint32_t parity) { return __all_sync(0xffffffffu, umma::mbar_wait(bar, parity)); }

// The 32 moving tokens from j that the masks leave a row, as bits: [from, to), and those of its document.  A whole warp, a row a lane:
// a lane fetches one token's document, and a turn of the loop serves all the tokens and rows of one document.
__device__ __forceinline__ uint32_t sm_left(int from, int to, const int* dm, int doc, int j, int n) {
  from = max(from - j, 0); to = min(max(to - j, 0), 32);
  uint32_t left = (to == 32 ? 0xffffffffu : (1u << to) - 1u) & (from < 32 ? 0xffffffffu << from : 0u);
  if (dm) {
    const int at = j + (int)(threadIdx.x & 31), id = at < n ? dm[at] : -1;
    uint32_t todo = 0xffffffffu, mine = 0;
    while (todo) {
      const int d = __shfl_sync(0xffffffffu, id, __ffs(todo) - 1);
      const uint32_t same = __ballot_sync(0xffffffffu, id == d);
      if (doc == d) mine = same;
      todo &= ~same;
    }
    left &= mine;
  }
  return left;
}

// Keys are split over CTAs (blockIdx.z) where the query tiles alone do not fill the GPU: a CTA takes `chunk` of its key tiles.
struct SmSplit { int chunk, splits; float* o; float2* ml; };       // parts: [row][split][d], maximum (base 2) and sum

template <int D, int T, int CAP, bool BIAS>
__global__ void __launch_bounds__(SuFwd<D, T>::kThreads, SuFwd<D, T>::kCtas)
k_softmax_fwd_umma(const __grid_constant__ SmArgs a, const __grid_constant__ TileMap mq, const __grid_constant__ TileMap mk,
                   const __grid_constant__ TileMap mv, const __grid_constant__ SmSplit sp) {
  pdl_wait();
  constexpr int NS = SuFwd<D, T>::kStages, TB = SuFwd<D, T>::kTile, COPY = 4 * T, MMA = 4 * T + 1, TMEM = SuFwd<D, T>::kTmem;
  constexpr bool EARLY = D == 64;                                              // A beside S, not over it
  constexpr int TP = EARLY ? T * 128 : 0, PC = EARLY ? 64 : 128, TO = TP + T * (EARLY ? 64 : 128);     // columns of A and O; of A a tile
  extern __shared__ __align__(16) char su_smem[];
  char* base = su_smem + ((1024u - (umma::s32(su_smem) & 1023u)) & 1023u);
  char *sQ = base, *sK = base + T * TB, *sV = sK + NS * TB;
  __shared__ unsigned long long q_full, k_full[NS], k_free[NS], v_full[NS], v_free[NS], v_raw, s_full[T], s_read[T], p_ready[T], o_full[T], spare[T];
  __shared__ uint32_t tmem_slot;
  __shared__ int sh[2];
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int bh = blockIdx.x, b = bh / a.Hq, h = bh % a.Hq, hk = h / a.group;
  const int i0 = ((int)gridDim.y - 1 - (int)blockIdx.y) * (T * 128);           // long causal rows first
  const SmMask m(a, b);
  const int2 range = sm_range<T * 128, false>(a, m, b, i0, sh);
  // key tiles of 128 from k0, the last one first
  const int all = (range.y - range.x + 1) / 2, z0 = sp.splits > 1 ? (int)blockIdx.z * sp.chunk : 0;
  const int nt = sp.splits > 1 ? min(max(all - z0, 0), sp.chunk) : all, k0 = range.x * 64 + z0 * 128;
  const bool alone = sp.splits == 1 || all <= sp.chunk;                        // this CTA has all keys of its rows
  if (sp.splits > 1 && blockIdx.z && nt == 0) {                                // nothing for this split: a part of nothing
    if (!alone)
      for (int r = tid; r < T * 128 && i0 + r < a.nq; r += SuFwd<D, T>::kThreads)
        sp.ml[((long long)bh * a.nq + i0 + r) * sp.splits + blockIdx.z] = make_float2(-INFINITY, 0.f);
    return;
  }
  if (tid == 0) {
    umma::mbar_init(&q_full, 1); umma::mbar_init(&v_raw, 1);
    for (int s = 0; s < NS; ++s) {
      umma::mbar_init(&k_full[s], 1); umma::mbar_init(&k_free[s], T); umma::mbar_init(&v_full[s], 1); umma::mbar_init(&v_free[s], T);
    }
    for (int t = 0; t < T; ++t) {
      umma::mbar_init(&s_full[t], 1); umma::mbar_init(&s_read[t], 4); umma::mbar_init(&p_ready[t], 4); umma::mbar_init(&o_full[t], 1); umma::mbar_init(&spare[t], 1);
    }
  }
  if (warp == MMA) umma::tmem_alloc(&tmem_slot, TMEM);
  umma::fence_before_sync();
  __syncthreads();
  umma::fence_after_sync();
  const uint32_t tm = tmem_slot;
  const int* dk = a.doc_k ? a.doc_k + (long long)b * a.nk : nullptr;
  bool ok = true;

  if (warp == COPY) {                                                        // copies
    const bool one = umma::elect_one();
    const int qh = h * mq.head, qb = b * mq.batch, kh = hk * mk.head, kb = b * mk.batch, vh = hk * mv.head, vb = b * mv.batch;
    if (nt > 0 && one) {
      umma::mbar_expect_tx(&q_full, T * TB);
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int blk = 0; blk < D / 64; ++blk)
          umma::tile_load(umma::s32(sQ) + t * TB + blk * 16384, &mq.map, blk * 64, i0 + t * 128, qh, qb, &q_full);
    }
    int raw = 0, ks = 0, vs = 0;                                             // copies begun: rows to be cleared first, K and V tiles
    for (int j = 0; j < nt && ok; ++j) {
      const int s = j % NS, j0 = k0 + (nt - 1 - j) * 128;
      const uint32_t again = (uint32_t)(j / NS - 1) & 1;
      if (j >= NS) ok = warp_wait(&k_free[s], again);
      if (one && ok) {
        umma::mbar_expect_tx(&k_full[s], TB);
#pragma unroll
        for (int blk = 0; blk < D / 64; ++blk)
          umma::tile_load(umma::s32(sK) + s * TB + blk * 16384, &mk.map, blk * 64, j0, kh, kb, &k_full[s]);
      }
      if (ok) ++ks;
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
      ++vs;
      if (clear) {
        ok = warp_wait(&v_raw, raw++ & 1);
        tile_clear<D>(sV + s * TB, 128, [&](int r) { const int key = j0 + r; return key >= a.nk || (key < m.len && !(dk && dk[key] < 0)); });
        if (one) umma::mbar_arrive(&v_full[s]);
      }
    }
    // no copy is in flight when the CTA ends, whichever wait of whichever warp ran out
    if (nt > 0) umma::mbar_wait(&q_full, 0);
    if (raw > 0) umma::mbar_wait(&v_raw, (uint32_t)(raw - 1) & 1);
    for (int s = 0; s < NS; ++s) {
      if (ks > s) umma::mbar_wait(&k_full[s], (uint32_t)((ks - 1 - s) / NS) & 1);
      if (vs > s) umma::mbar_wait(&v_full[s], (uint32_t)((vs - 1 - s) / NS) & 1);
    }
  } else if (warp >= MMA) {                                                  // products of tile t
    if (umma::elect_one() && nt > 0) {
      const int t = warp - MMA;
      const uint32_t id_s = umma::instr_desc(128, false, false), id_o = umma::instr_desc(D, false, true);
      const uint64_t qd = umma::rows_desc(umma::s32(sQ) + t * TB), kd = umma::rows_desc(umma::s32(sK)), vd = umma::cols_desc(umma::s32(sV), 128);
      const uint32_t ts = tm + t * 128, tp = tm + TP + t * PC, to = tm + TO + t * D;
      auto scores = [&](int j) {                                             // d = 32: the upper channels are zeros
        const int s = j % NS;
        ok = ok && umma::mbar_wait(&k_full[s], (j / NS) & 1);
        if (!ok) return;
        umma::fence_after_sync();
        const uint64_t k0 = kd + (uint64_t)(s * (TB >> 4));
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) umma::mma(ts, qd + umma::rows_step(128, ks), k0 + umma::rows_step(128, ks), id_s, ks > 0);
        umma::commit(&s_full[t]);
        if (j + NS < nt) umma::commit(&k_free[s]);                           // only where the copying warp waits for it: no arrival is
      };                                                                     // under way when the CTA ends
      ok = umma::mbar_wait(&q_full, 0);
      scores(0);
      for (int j = 0; j < nt && ok; ++j) {
        const int s = j % NS;
        if (EARLY && j + 1 < nt) {
          ok = umma::mbar_wait(&s_read[t], j & 1);
          scores(j + 1);
        }
        ok = ok && umma::mbar_wait(&v_full[s], (j / NS) & 1) && umma::mbar_wait(&p_ready[t], j & 1);
        if (!ok) break;
        umma::fence_after_sync();
        const uint64_t v0 = vd + (uint64_t)(s * (TB >> 4));
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) umma::mma_ta(to, tp + ks * 8, v0 + umma::cols_step(ks), id_o, j > 0 || ks > 0);
        if (EARLY || j + 1 == nt) umma::commit(&o_full[t]);
        if (j + NS < nt) umma::commit(&v_free[s]);
        if (!EARLY && j + 1 < nt) scores(j + 1);
      }
      umma::commit(&spare[t]);                                               // nor a product
      umma::mbar_wait(&spare[t], 0);
    }
  } else {                                                                   // exponentials
    const int t = warp >> 2, lane = tid & 31, row = (warp & 3) * 32 + lane, i = i0 + t * 128 + row;
    const uint32_t quarter = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tm + quarter + t * 128, tp = tm + quarter + TP + t * PC, to = tm + quarter + TO + t * D;
    const int doc = a.doc_q && i < a.nq ? a.doc_q[(long long)b * a.nq + i] : 0;
    const int lim = i < a.nq && doc >= 0 ? m.limit(i) : 0;
    const SmScore sc = sm_score_of(a, h);
    float ref = -INFINITY, sum = 0.f;
    for (int j = 0; j < nt; ++j) {
      const int j0 = k0 + (nt - 1 - j) * 128;
      const bool whole = sm_whole(a, m, b, i0 + t * 128, i0 + t * 128 + 128, j0, j0 + 128);
      uint32_t left[4];
      if (!whole)
#pragma unroll
        for (int c = 0; c < 4; ++c) left[c] = sm_left(0, lim, dk, doc, j0 + c * 32, a.nk);
      ok = warp_wait(&s_full[t], j & 1);
      if (!ok) break;
      umma::fence_after_sync();
      float x[128];
#pragma unroll
      for (int c = 0; c < 4; ++c) umma::tmem_ld32_async(ts + c * 32, x + c * 32);
      umma::tmem_ld_wait();
#pragma unroll
      for (int c = 0; c < 4; ++c) umma::tie32(x + c * 32);
      if (EARLY) {
        umma::fence_before_sync();
        __syncwarp();
        if (lane == 0) umma::mbar_arrive(&s_read[t]);
      }
      // x: products, what stands for a capped score (SmScore), or scores with a bias; the score in base 2 is x ka + kb
      const float down = CAP == CAP_USUAL ? -2.f * sc.cap2 : CAP ? -1.f : sc.mul, mid = CAP == CAP_USUAL ? sc.cap2 : 0.f;
      const float ka = BIAS ? 1.f : down, kb = BIAS ? 0.f : mid;
      if (CAP) {
        if (!whole)
#pragma unroll
          for (int e = 0; e < 128; ++e)
            if (!((left[e >> 5] >> (e & 31)) & 1u)) x[e] = 0.f;
#pragma unroll
        for (int e = 0; e < 128; e += 4) {
          float q[4] = {x[e], x[e + 1], x[e + 2], x[e + 3]};
          if (CAP == CAP_WIDE) sm_cap4_wide(q, sc); else sm_cap4(q, sc.mul);
#pragma unroll
          for (int k = 0; k < 4; ++k) x[e + k] = q[k];
        }
      }
      if (BIAS) {
        const float p = (float)(i + m.off - j0);
#pragma unroll
        for (int e = 0; e < 128; ++e) {
          const float far = sc.slope2 * fabsf(p - (float)e);
          x[e] = fmaf(down, x[e], CAP == CAP_USUAL ? mid - far : -far);
        }
      }
      constexpr bool DOWN = CAP != CAP_NONE && !BIAS;                                    // the largest score has the smallest x
      if (!whole)
#pragma unroll
        for (int e = 0; e < 128; ++e)
          if (!((left[e >> 5] >> (e & 31)) & 1u)) x[e] = DOWN ? INFINITY : -INFINITY;
      auto further = [](float u, float v) { return DOWN ? fminf(u, v) : fmaxf(u, v); };
      float top[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
      for (int e = 4; e + 8 <= 124 + 4; e += 8)
#pragma unroll
        for (int k = 0; k < 4; ++k) top[k] = further(further(top[k], x[e + 2 * k]), x[e + 2 * k + 1]);
#pragma unroll
      for (int k = 0; k < 4; ++k) top[k] = further(top[k], x[124 + k]);
      const float mx = fmaf(further(further(top[0], top[1]), further(top[2], top[3])), ka, kb);
      if (EARLY && j > 0) {                                                  // A may be written, O be scaled: the product before is done
        ok = warp_wait(&o_full[t], (j - 1) & 1);
        if (!ok) break;
        umma::fence_after_sync();
      }
      const bool grown = mx > ref + 8.f;                                     // also the first finite maximum of a row
      if (__any_sync(0xffffffffu, grown)) {
        const float now = grown ? mx : ref;
        const float f = grown ? (ref == -INFINITY ? 0.f : ex2(ref - now)) : 1.f;
        ref = now;
        sum *= f;
        if (j > 0) {                                                         // every product into O is complete (else s_full follows them)
#pragma unroll
          for (int c = 0; c < D; c += 16) {
            float o[16];
            uint32_t w[16];
            umma::tmem_ld16_async(to + c, o);
            umma::tmem_ld_wait();
            umma::tie16(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(o[e] * f);
            umma::tmem_st16(to + c, w);
          }
        }
      }
      const float shift = kb + (ref == -INFINITY ? 0.f : -ref);
      f32x2 part[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};
      // exponentials, rounded and packed over the scores
      const f32x2 ka2 = pack2(ka, ka), kb2 = pack2(shift, shift);
#pragma unroll
      for (int c = 0; c < 128; c += 32) {
        uint32_t w[16];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const f32x2 v = pack2(x[c + e], x[c + e + 1]);
          float p0, p1;
          unpack2(BIAS ? add2(v, kb2) : fma2(v, ka2, kb2), p0, p1);
          p0 = ex2(p0); p1 = ex2(p1);
          part[(e >> 1) & 1] = add2(part[(e >> 1) & 1], pack2(p0, p1));
          w[e / 2] = umma::pack_bf16(p0, p1);
        }
        umma::tmem_st16(tp + c / 2, w);
      }
      {
        float u0, u1;
        unpack2(add2(part[0], part[1]), u0, u1);
        sum += u0 + u1;
      }
      umma::tmem_st_wait();
      umma::fence_before_sync();
      __syncwarp();
      if (lane == 0) umma::mbar_arrive(&p_ready[t]);
    }
    if (nt > 0) {
      ok = ok && warp_wait(&o_full[t], EARLY ? (nt - 1) & 1 : 0);
      umma::fence_after_sync();
    }
    if (ok && !alone) {                                                      // a part: 32-bit accumulators as they are
      float* po = sp.o + (((long long)bh * a.nq + i) * sp.splits + blockIdx.z) * a.d;
#pragma unroll
      for (int c = 0; c < D; c += 32) {                                      // every lane loads (the instruction is the warp's), rows in range store
        float o[32];
        umma::tmem_ld32_async(to + c, o);
        umma::tmem_ld_wait();
        umma::tie32(o);
        if (i < a.nq && c < a.d)
#pragma unroll
          for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(po + c + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
      }
      if (i < a.nq) sp.ml[((long long)bh * a.nq + i) * sp.splits + blockIdx.z] = make_float2(ref, sum);
    } else if (ok) {
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
      if (i < a.nq) {
        a.lse[(long long)bh * a.nq + i] = sum == 0.f ? -INFINITY : (ref + __log2f(sum)) * kLn2;
        // one part, whole: the join passes over the row
        if (sp.splits > 1) sp.ml[((long long)bh * a.nq + i) * sp.splits] = make_float2(0.f, -1.f);
      }
    }
  }
  __syncwarp();
  umma::fence_before_sync();
  __syncthreads();
  if (warp == MMA) umma::tmem_dealloc(tm, TMEM);
  umma::report_timeout(ok, a.dev_status, bh);
}

}  // namespace ln
