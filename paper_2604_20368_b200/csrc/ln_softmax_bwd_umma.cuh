// Softmax attention on the 5th-generation tensor cores (tcgen05 + TMEM), bf16 storage, backward.
//
// One CTA = 128 stationary rows X of one head; the moving rows Y stream through shared memory in tiles of 64, copied by TMA.
//   queries stationary (KEYS false):  X1 = Q, X2 = dO;  Y1 = K, Y2 = V;   dQ += ds Y1, M += A Y1
//   keys stationary    (KEYS true):   X1 = K, X2 = V;   Y1 = Q, Y2 = dO of every query head of the group;  dK += ds Y1, dV += A Y2
// Per tile: S = X1 Y1^T and dP = X2 Y2^T (128 x 64, K = d, operands in shared memory), then A = exp2(x - lse) and
// ds = A (dP - delta) (1 - tanh^2), both rounded to bf16 and written over S and dP in TMEM, from where they are the left operands
// of the products into the accumulators (128 x d in TMEM).  A thread owns a row of a group of four warps.  With 128 channels S and dP
// have two buffers (NB = 2): one group forms the exponentials of the even tiles, one those of the odd ones, and while one waits for
// the tensor core the other has work.  With 64 channels a CTA has one buffer and one group, and two CTAs share an SM, which
// hides the start and the end of a CTA too.  One warp copies, one issues the products.  `scale` is applied once, to the accumulators.
// delta from the stored O is off by O's rounding, up to 2^-8 sum|dO||O|, more than anything else where a row's softmax is
// peaked.  The sum of a row's ds says by how much (it is zero for the right delta): the query pass adds it up in 32 bits, takes it
// times M = A K off dQ, and hands the corrected delta to the key pass (dQ and dK of 4096 tokens with scores of 3 standard deviations:
// 2.7e-3 -> 2.4e-3 of their norm, of 16 tokens 4.0e-3 -> 2.4e-3, where their own rounding is 1.7e-3).
// Two passes form S and dP twice (4 products a pair each, M among them, instead of 5 in all): no atomics, and every sum has one order.
// Bound by the tensor core's operand reads: with 64 columns a product reads 128 + 64 rows of shared memory for 128 x 64 results.
// 32 heads of 4096 tokens without masks: 128 channels query pass 478 us, key pass 459 (1.20 PFLOP/s); 64 channels 293 and 332; with a cap of 20
// 566 and 588, 478 and 482.
#pragma once
#include "ln_softmax_umma.cuh"

namespace ln {

template <int D> struct SuBwd {
  static constexpr int kX = 128 * D * 2, kY = 64 * D * 2;         // bytes of a stationary and of a moving tile
  static constexpr int kBuffers = D == 64 ? 1 : 2, kStages = D == 64 ? 3 : 4;
  static constexpr int kThreads = kBuffers * 128 + 64, kCtas = D == 64 ? 2 : 1, kTmem = D == 64 ? 256 : 512;
  static constexpr size_t kSmem = 1024 + 2 * (size_t)kX + 2 * (size_t)kY * kStages;
};

template <int D, int CAP, bool BIAS, bool KEYS>
__global__ void __launch_bounds__(SuBwd<D>::kThreads, SuBwd<D>::kCtas)
k_softmax_bwd_umma(const __grid_constant__ SmArgs a, const __grid_constant__ TileMap mx1, const __grid_constant__ TileMap mx2,
                   const __grid_constant__ TileMap my1, const __grid_constant__ TileMap my2) {
  pdl_wait();
  constexpr int NS = SuBwd<D>::kStages, XB = SuBwd<D>::kX, YB = SuBwd<D>::kY, NB = SuBwd<D>::kBuffers, COPY = 4 * NB, MMA = 4 * NB + 1;
  extern __shared__ __align__(16) char su_smem[];
  char* base = su_smem + ((1024u - (umma::s32(su_smem) & 1023u)) & 1023u);
  char *sX = base, *sY = base + 2 * XB;                                      // X1, X2; per stage Y1, Y2
  __shared__ unsigned long long x_full, y_full[NS], y_free[NS], y_raw, l_full[NS], s_full[NB], p_ready[NB], acc_full, spare;
  __shared__ uint32_t tmem_slot;
  __shared__ __align__(16) float sL[KEYS ? NS : 1][64], sD[KEYS ? NS : 1][64];     // -lse (base 2) and -delta of the moving queries
  __shared__ float sRow[KEYS ? 1 : NB][128];                                 // a group's part of a row's delta, then of its sum of ds
  __shared__ int sh[2];
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int H = KEYS ? a.Hk : a.Hq, b = blockIdx.x / H, hs = blockIdx.x % H;
  const int s0 = (KEYS ? (int)blockIdx.y : (int)gridDim.y - 1 - (int)blockIdx.y) * 128;     // the longest causal rows first
  const SmMask m(a, b);
  const int2 range = sm_range<128, KEYS>(a, m, b, s0, sh);
  const int nt = range.y - range.x, total = KEYS ? nt * a.group : nt;
  if (tid == 0) {
    umma::mbar_init(&x_full, 1); umma::mbar_init(&y_raw, 1); umma::mbar_init(&acc_full, 1); umma::mbar_init(&spare, 1);
    for (int s = 0; s < NS; ++s) { umma::mbar_init(&y_full[s], 1); umma::mbar_init(&y_free[s], 1); umma::mbar_init(&l_full[s], 1); }
    for (int t = 0; t < NB; ++t) { umma::mbar_init(&s_full[t], 1); umma::mbar_init(&p_ready[t], 4); }
  }
  if (warp == MMA) umma::tmem_alloc(&tmem_slot, SuBwd<D>::kTmem);
  umma::fence_before_sync();
  __syncthreads();
  umma::fence_after_sync();
  const uint32_t tm = tmem_slot;                                             // S, dP (64 columns each) of every buffer; accumulators
  constexpr int ACC2 = NB * 128, ACC1 = NB * 128 + D;                        // ds Y1;  A Y2 (keys stationary) or A Y1
  const int* dq = a.doc_q ? a.doc_q + (long long)b * a.nq : nullptr;
  const int* dk = a.doc_k ? a.doc_k + (long long)b * a.nk : nullptr;
  const int first_head = KEYS ? hs * a.group : hs;                           // query head of the first moving tile
  bool ok = true;

  if (warp == COPY) {                                                           // copies
    const bool one = umma::elect_one();
    if (total > 0 && one) {
      umma::mbar_expect_tx(&x_full, 2 * XB);
#pragma unroll
      for (int blk = 0; blk < D / 64; ++blk) {
        umma::tile_load(umma::s32(sX) + blk * 16384, &mx1.map, blk * 64, s0, hs * mx1.head, b * mx1.batch, &x_full);
        umma::tile_load(umma::s32(sX) + XB + blk * 16384, &mx2.map, blk * 64, s0, hs * mx2.head, b * mx2.batch, &x_full);
      }
    }
    int raw = 0, n = 0;                                                      // copies begun: rows to be cleared first, all tiles
    for (; n < total; ++n) {
      const int s = n % NS, m0 = (range.x + n % nt) * 64, hq = first_head + n / nt, hy = KEYS ? hq : hs / a.group;
      if (n >= NS) ok = warp_wait(&y_free[s], (uint32_t)(n / NS - 1) & 1);
      if (!ok) break;
      // moving rows that no pair uses may hold an infinity (see the forward kernel)
      bool clear = !KEYS && m0 + 64 > m.len && m.len < a.nk;
      if (a.rq) clear |= (KEYS ? a.rq[(long long)b * a.tq + m0 / 64] : a.rk[(long long)b * a.tk + m0 / 64]).z != 0;
      unsigned long long* bar = clear ? &y_raw : &y_full[s];
      char* y = sY + s * 2 * YB;
      if (one) {
        umma::mbar_expect_tx(bar, 2 * YB);
#pragma unroll
        for (int blk = 0; blk < D / 64; ++blk) {
          umma::tile_load(umma::s32(y) + blk * 8192, &my1.map, blk * 64, m0, hy * my1.head, b * my1.batch, bar);
          umma::tile_load(umma::s32(y) + YB + blk * 8192, &my2.map, blk * 64, m0, hy * my2.head, b * my2.batch, bar);
        }
      }
      if (KEYS) {
        const long long at = ((long long)b * a.Hq + hq) * a.nq + m0;
#pragma unroll
        for (int u = 0; u < 64; u += 32) {
          const bool in = m0 + u + lane < a.nq;
          sL[s][u + lane] = in ? -a.lse[at + u + lane] * kLog2e : 0.f;
          sD[s][u + lane] = in ? -a.delta[at + u + lane] : 0.f;
        }
        __syncwarp();
        if (one) umma::mbar_arrive(&l_full[s]);
      }
      if (clear) {
        ok = warp_wait(&y_raw, raw++ & 1);
        auto keep = [&](int r) {
          const int row = m0 + r;
          return KEYS ? row >= a.nq || dq[row] >= 0 : row >= a.nk || (row < m.len && !(dk && dk[row] < 0));
        };
        tile_clear<D>(y, 64, keep);
        if (KEYS) tile_clear<D>(y + YB, 64, keep);
        if (one) umma::mbar_arrive(&y_full[s]);
        if (!ok) { ++n; break; }
      }
    }
    // no copy is in flight when the CTA ends, whichever wait of whichever warp ran out
    if (total > 0) umma::mbar_wait(&x_full, 0);
    if (raw > 0) umma::mbar_wait(&y_raw, (uint32_t)(raw - 1) & 1);
    for (int s = 0; s < NS; ++s)
      if (n > s) umma::mbar_wait(&y_full[s], (uint32_t)((n - 1 - s) / NS) & 1);
  } else if (warp == MMA) {                                                    // products
    if (umma::elect_one() && total > 0) {
      const uint32_t id_s = umma::instr_desc(64, false, false), id_a = umma::instr_desc(D, false, true);
      const uint64_t x1 = umma::rows_desc(umma::s32(sX)), x2 = x1 + (XB >> 4), yr = umma::rows_desc(umma::s32(sY)), yc = umma::cols_desc(umma::s32(sY), 64);
      auto arrived = [&](int n) { ok = ok && umma::mbar_wait(&y_full[n % NS], (uint32_t)(n / NS) & 1); };
      auto scores = [&](int n) {                                             // S and dP of tile n (d = 32: the upper channels are zeros)
        const int s = n % NS, buf = n % NB;
        const uint64_t y1 = yr + (uint64_t)(s * (2 * YB >> 4)), y2 = y1 + (YB >> 4);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) umma::mma(tm + buf * 128, x1 + umma::rows_step(128, ks), y1 + umma::rows_step(64, ks), id_s, ks > 0);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) umma::mma(tm + buf * 128 + 64, x2 + umma::rows_step(128, ks), y2 + umma::rows_step(64, ks), id_s, ks > 0);
        umma::commit(&s_full[buf]);
      };
      ok = umma::mbar_wait(&x_full, 0);
      arrived(0);
      umma::fence_after_sync();
      if (ok) scores(0);
      if (NB > 1 && total > 1) {
        arrived(1);
        if (ok) scores(1);
      }
      for (int n = 0; n < total && ok; ++n) {
        const int s = n % NS, buf = n % NB;
        const uint64_t y1 = yc + (uint64_t)(s * (2 * YB >> 4)), y2 = y1 + (YB >> 4);
        // a wait costs some 200 clocks beside the products' operand reads, so the one for tile n + NB comes while this tile's
        // exponentials are still being formed
        if (n + NB < total) arrived(n + NB);
        ok = ok && umma::mbar_wait(&p_ready[buf], (uint32_t)(n / NB) & 1);
        if (!ok) break;
        umma::fence_after_sync();
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {                                     // 64 columns became 32 packed ones at the front of their place
          const uint32_t at = tm + buf * 128 + ks * 8;
          umma::mma_ta(tm + ACC1, at, (KEYS ? y2 : y1) + umma::cols_step(ks), id_a, n > 0 || ks > 0);
          umma::mma_ta(tm + ACC2, at + 64, y1 + umma::cols_step(ks), id_a, n > 0 || ks > 0);
        }
        if (n + NS < total) umma::commit(&y_free[s]);                        // only where the copying warp waits for it
        if (n + NB < total) scores(n + NB);
      }
      if (ok) umma::commit(&acc_full);
      umma::commit(&spare);                                                  // no product is in flight when the CTA ends
      umma::mbar_wait(&spare, 0);
    }
  } else {                                                                   // exponentials
    const int group = warp >> 2, row = (warp & 3) * 32 + lane, r = s0 + row;
    const uint32_t quarter = (uint32_t)((warp & 3) * 32) << 16;
    int doc, lo, hi;                                                         // moving tokens [lo, hi) are left by the masks but the documents'
    float rowL = 0.f, rowD = 0.f;
    if (KEYS) {
      doc = dk && r < a.nk ? dk[r] : 0;
      lo = m.first(r); hi = r < m.len && doc >= 0 ? a.nq : 0;
    } else {
      doc = dq && r < a.nq ? dq[r] : 0;
      lo = 0; hi = r < a.nq && doc >= 0 ? m.limit(r) : 0;
      // delta: a thread of every group a row, its share of the channels each
      const long long at = (long long)blockIdx.x * a.nq + r;
      float v = 0.f;
      if (r < a.nq) {
        const bf16* o = static_cast<const bf16*>(a.o.p) + b * a.o.b + hs * a.o.h + r * a.o.t + group * (a.d / NB);
        const bf16* g = static_cast<const bf16*>(a.dout.p) + b * a.dout.b + hs * a.dout.h + r * a.dout.t + group * (a.d / NB);
#pragma unroll 4
        for (int c = 0; c < a.d / NB; c += 8) {
          const uint4 x = *reinterpret_cast<const uint4*>(o + c), y = *reinterpret_cast<const uint4*>(g + c);
          const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v = fmaf(__uint_as_float(xs[e] << 16), __uint_as_float(ys[e] << 16), v);
            v = fmaf(__uint_as_float(xs[e] & 0xffff0000u), __uint_as_float(ys[e] & 0xffff0000u), v);
          }
        }
        rowL = a.lse[at] * kLog2e;
      }
      rowD = v;
      if (NB > 1) {
        sRow[group][row] = v;
        asm volatile("bar.sync 1, 256;" ::: "memory");
        rowD = sRow[0][row] + sRow[NB - 1][row];
        asm volatile("bar.sync 1, 256;" ::: "memory");                       // read by both before it takes the sums of ds
      }
    }
    f32x2 rest2 = pack2(0.f, 0.f);                                           // sum of this row's ds before the cap's factor
    const int* dm = KEYS ? dq : dk;
    const int nm = KEYS ? a.nq : a.nk, buf = group;
    SmScore sc = sm_score_of(a, first_head);
    const float down = CAP == CAP_USUAL ? -2.f * sc.cap2 : CAP ? -1.f : sc.mul;
    const f32x2 ka = pack2(down, down), kb = pack2(sc.cap2, sc.cap2);
    const f32x2 rowL2 = pack2(-rowL, -rowL), rowD2 = pack2(-rowD, -rowD);
    const uint32_t ts = tm + quarter + buf * 128;
    int tile = range.x + group, head = first_head;                            // of moving tile n
    uint32_t turn = 0;                                                       // how often this group has waited for its buffer
    for (int n = group; n < total; n += NB, ++turn) {
      while (tile >= range.x + nt) {                                         // the next query head of the group
        tile -= nt; ++head;
        if (BIAS) sc.slope2 = a.slopes[head] * kLog2e;
      }
      const int s = n % NS, m0 = tile * 64;
      tile += NB;
      const bool whole = KEYS ? s0 + 128 <= a.nk && sm_whole(a, m, b, m0, m0 + 64, s0, s0 + 128) : sm_whole(a, m, b, s0, s0 + 128, m0, m0 + 64);
      ok = (!KEYS || warp_wait(&l_full[s], (uint32_t)(n / NS) & 1)) && warp_wait(&s_full[buf], turn & 1);
      if (!ok) break;
      umma::fence_after_sync();
      // 32 columns at a time; what the masks leave out is 0 in A and ds, whatever the products are
      auto columns = [&](int c0, auto masked) {
        constexpr bool MASKED = decltype(masked)::value;
        float x[32], g[32];
        umma::tmem_ld32_async(ts + c0, x);
        umma::tmem_ld32_async(ts + 64 + c0, g);
        const uint32_t left = MASKED ? sm_left(lo, hi, dm, doc, m0 + c0, nm) : 0xffffffffu;
        const float away = (float)(KEYS ? m0 + c0 + m.off - r : r + m.off - m0 - c0);   // position of the query less the key's, column 0
        umma::tmem_ld_wait();
        umma::tie32(x);
        umma::tie32(g);
        uint32_t wp[16], wd[16];
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          f32x2 L[2] = {rowL2, rowL2}, Dl[2] = {rowD2, rowD2}, bend[2];
          if (KEYS) {
            const ulonglong2 u = *reinterpret_cast<const ulonglong2*>(&sL[s][c0 + e]), v = *reinterpret_cast<const ulonglong2*>(&sD[s][c0 + e]);
            L[0] = u.x; L[1] = u.y; Dl[0] = v.x; Dl[1] = v.y;
          }
          float q[4] = {x[e], x[e + 1], x[e + 2], x[e + 3]};
          if (CAP) {
            if (MASKED)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (!((left >> (e + k)) & 1u)) q[k] = 0.f;
            if (CAP == CAP_WIDE) sm_cap4_wide(q, sc); else sm_cap4(q, sc.mul);
          }
          float p[4], d[4];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const f32x2 v = pack2(q[2 * k], q[2 * k + 1]);
            if (CAP == CAP_WIDE) {                                           // v is a score over the cap, tanh, but for its sign
              const f32x2 t = mul2(v, pack2(1.f / sc.cap2, 1.f / sc.cap2));
              bend[k] = fma2(mul2(t, pack2(-1.f, -1.f)), t, pack2(1.f, 1.f));
            } else if (CAP) bend[k] = mul2(v, fma2(v, pack2(-4.f, -4.f), pack2(4.f, 4.f)));
            unpack2(fma2(v, ka, CAP == CAP_USUAL ? add2(kb, L[k]) : L[k]), p[2 * k], p[2 * k + 1]);
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (BIAS) p[k] = fmaf(-sc.slope2, fabsf(away + (KEYS ? (float)(e + k) : -(float)(e + k))), p[k]);
            if (MASKED && !((left >> (e + k)) & 1u)) p[k] = -INFINITY;
            p[k] = ex2(p[k]);
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            f32x2 v = mul2(pack2(p[2 * k], p[2 * k + 1]), add2(pack2(g[e + 2 * k], g[e + 2 * k + 1]), Dl[k]));
            unpack2(v, d[2 * k], d[2 * k + 1]);
          }
          if (MASKED)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (!((left >> (e + k)) & 1u)) d[k] = 0.f;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            f32x2 v = pack2(d[2 * k], d[2 * k + 1]);
            if (!KEYS) rest2 = add2(rest2, v);
            if (CAP) {
              v = mul2(v, bend[k]);
              unpack2(v, d[2 * k], d[2 * k + 1]);
              if (!KEYS) unpack2(mul2(pack2(p[2 * k], p[2 * k + 1]), bend[k]), p[2 * k], p[2 * k + 1]);
            }
          }
          { wp[e / 2] = umma::pack_bf16(p[0], p[1]); wp[e / 2 + 1] = umma::pack_bf16(p[2], p[3]); }
          wd[e / 2] = umma::pack_bf16(d[0], d[1]); wd[e / 2 + 1] = umma::pack_bf16(d[2], d[3]);
        }
        umma::tmem_st16(ts + c0 / 2, wp);
        umma::tmem_st16(ts + 64 + c0 / 2, wd);
      };
      if (whole) {
#pragma unroll 1
        for (int c0 = 0; c0 < 64; c0 += 32) columns(c0, std::false_type());
      } else {
#pragma unroll 1
        for (int c0 = 0; c0 < 64; c0 += 32) columns(c0, std::true_type());
      }
      umma::tmem_st_wait();
      umma::fence_before_sync();
      __syncwarp();
      if (lane == 0) umma::mbar_arrive(&p_ready[buf]);
    }
    if (total > 0) {
      ok = ok && warp_wait(&acc_full, 0);
      umma::fence_after_sync();
    }
    float rest = 0.f;
    if (!KEYS) {
      float u;
      unpack2(rest2, rest, u);
      rest += u;
      if (NB > 1) {
        sRow[group][row] = rest;
        asm volatile("bar.sync 1, 256;" ::: "memory");
        rest = sRow[0][row] + sRow[NB - 1][row];
      }
      if (group == 0 && r < a.nq) a.delta[(long long)blockIdx.x * a.nq + r] = rowD + rest;
    }
    if (ok) {
      // rows of this warp, its group's share of the channels, through its part of the stationary tiles (no product reads them any more)
      constexpr int HC = D / NB, PR = HC / 8;
      const int rows = (KEYS ? a.nk : a.nq) - s0 - (warp & 3) * 32, pieces = min(max(a.d - group * HC, 0), HC) / 8;
#pragma unroll
      for (int out = 0; out < (KEYS ? 2 : 1); ++out) {
        char* stage = sX + out * XB + (warp * 32 * HC) * 2;
        const float mul = out ? 1.f : a.scale;
#pragma unroll
        for (int c = 0; c < HC; c += 32) {
          float o[32], w1[32];
          if (total > 0) {
            umma::tmem_ld32_async(tm + quarter + (out ? ACC1 : ACC2) + group * HC + c, o);
            if (!KEYS) umma::tmem_ld32_async(tm + quarter + ACC1 + group * HC + c, w1);
            umma::tmem_ld_wait();
            umma::tie32(o);
            if (!KEYS) {
              umma::tie32(w1);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = fmaf(-rest, w1[e], o[e]);
            }
          }
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = total > 0 ? umma::pack_bf16(o[8 * q + 2 * e] * mul, o[8 * q + 2 * e + 1] * mul) : 0u;
            *reinterpret_cast<uint4*>(stage + (lane * PR + ((c / 8 + q) ^ (lane & 7))) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
        __syncwarp();
        const SmView& v = out ? a.dv : (KEYS ? a.dk : a.dq);
        bf16* G = static_cast<bf16*>(v.p) + b * v.b + hs * v.h + group * HC;
        const long long first = s0 + (warp & 3) * 32;
        for (int e = lane; e < 32 * pieces; e += 32) {
          const int rr = e / pieces, p = e % pieces;
          if (rr < rows)
            *reinterpret_cast<uint4*>(G + (first + rr) * v.t + p * 8) = *reinterpret_cast<const uint4*>(stage + (rr * PR + (p ^ (rr & 7))) * 16);
        }
      }
    }
  }
  __syncwarp();
  umma::fence_before_sync();
  __syncthreads();
  if (warp == MMA) umma::tmem_dealloc(tm, SuBwd<D>::kTmem);
  umma::report_timeout(ok, a.dev_status, KEYS ? b * a.Hq + first_head : (int)blockIdx.x);
}

}  // namespace ln
