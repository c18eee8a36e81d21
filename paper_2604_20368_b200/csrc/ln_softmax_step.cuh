// Softmax attention of a few queries (a serving step): the rows of a key head are its group's query heads times nq <= 16 queries,
// and a long cache is read once for all of them.
//
// Bound by memory traffic: the keys and values of a head, once.  The keys are split over CTAs, over the four warps of a CTA in
// turns of 16 keys, and every warp keeps maximum, sum and accumulator of its own; warps are joined through shared memory, CTAs
// by k_softmax_join.  bf16 rows become the operands of mma.sync as they are (m16n8k16, fp32 accumulate; 16 rows are all a serving step
// has, a tcgen05 tile would be 128): both products sum over an axis whose order is free, so a lane's 16-byte piece of a row IS its
// share of an operand, and no lane needs what another one fetched.
//   S = Q K^T   B = K^T: lane (g, c) = (lane / 4, lane % 4) holds channels 32 l + 8 c .. of key g, which stand for k-steps 2 l, 2 l + 1
//   O = A V     B = V:   lane (g, c) holds channels 8 g .. (and 64 + 8 g .., or 4 g ..) of keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9; column
//               tile j is channel 8 g + j (then 64 + 8 g + j - 8, or 4 g + j): eight lanes read 128 bytes in a row
#pragma once
#include "ln_mma.cuh"
#include "ln_softmax_umma.cuh"

namespace ln {

constexpr int ST_ROWS = 16, ST_WARPS = 4;

struct StepPlan { int chunk, splits; };              // keys a CTA, CTAs a key head
struct StepPart { float* o; float2* ml; };           // [row][split][d] partial outputs, maximum (base 2) and sum of every partial

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { uint32_t r; asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(sel)); return r; }

// Score in base 2 from the product for fp32 storage, with the cap through the accurate tanh (bf16 storage: sm_cap4).
__device__ __forceinline__ float step_score(float dot, const SmArgs& a, float slope2, int dist) {
  float x = dot * a.scale;
  if (a.cap > 0.f) x = a.cap * tanhf(x / a.cap);
  return fmaf(x, kLog2e, -slope2 * (float)abs(dist));
}

// A lane's pieces of the next turns are on their way through shared memory, which serves as a longer register file: a lane reads only
// what it copied itself, lane by lane, so no barrier is involved and no bank is hit twice.  Two turns of the eight warps of two CTAs are 128 KB in
// flight on an SM with 128 channels; with one turn in registers the same kernel waited half its time (16 caches of up to 50176
// keys, 8 query heads on 2: 184 -> 133 us, 617 MB).
constexpr int ST_STAGES = 3;
template <int D> __host__ __device__ constexpr int step_pieces() { return 2 * (D / 32) + 4 * (D == 128 ? 2 : 1); }      // 16 bytes each (d = 32: values 8)
template <int D> __host__ __device__ constexpr size_t step_smem() { return (size_t)ST_STAGES * ST_WARPS * step_pieces<D>() * 512; }

// 16 or 8 bytes global -> shared; zeros (and nothing read) if not `in`
template <int N> __device__ __forceinline__ void step_copy(void* dst, const void* src, bool in) {
  const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
  if (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(in ? 16 : 0) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(d), "l"(src), "r"(in ? 8 : 0) : "memory");
}

// A CTA's accumulators: the result itself if it is the only split, else its part.  s_m, s_l [warp][pitch_r]; s_o [part][row][pitch_o],
// NPART parts to be added.
template <typename T, int D, int NPART>
__device__ __forceinline__ void step_write(const SmArgs& a, const StepPlan& pl, const StepPart& part, int b, int hk, int split, int rows, const float* s_m,
                                           const float* s_l, int pitch_r, const float* s_o, int pitch_w, int pitch_o) {
  for (int e = threadIdx.x; e < rows * D; e += ST_WARPS * 32) {
    const int r = e / D, ch = e % D, h = hk * a.group + r / a.nq, i = r % a.nq;
    const long long row = ((long long)b * a.Hq + h) * a.nq + i;
    float t = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < ST_WARPS; ++w) t = fmaxf(t, s_m[w * pitch_r + r]);
#pragma unroll
    for (int w = 0; w < ST_WARPS; ++w) {
      const float mw = s_m[w * pitch_r + r], lw = s_l[w * pitch_r + r];
      l += mw == -INFINITY ? lw : lw * ex2(mw - t);                          // a sum of nothing is zero, NaN stays
    }
    float o = s_o[r * pitch_o + ch];
#pragma unroll
    for (int w = 1; w < NPART; ++w) o += s_o[w * pitch_w + r * pitch_o + ch];
    if (pl.splits == 1) {
      static_cast<T*>(a.o.p)[b * a.o.b + h * a.o.h + i * a.o.t + ch] = from_f<T>(l == 0.f ? 0.f : o / l);
      if (ch == 0) a.lse[row] = l == 0.f ? -INFINITY : t * kLn2 + logf(l);
    } else {
      part.o[(row * pl.splits + split) * D + ch] = o;
      if (ch == 0) part.ml[row * pl.splits + split] = make_float2(t, l);
    }
  }
}

template <int D>
__global__ void __launch_bounds__(ST_WARPS * 32, 2) k_softmax_step(const __grid_constant__ SmArgs a, StepPlan pl, StepPart part) {
  pdl_wait();
  constexpr int KL = D / 32, VW = D / 16, NT = D / 8;      // 16-byte pieces of a key row a lane, words of a value row a lane, column tiles
  const int split = blockIdx.x, hk = blockIdx.y % a.Hk, b = blockIdx.y / a.Hk;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
  const SmMask m(a, b);
  const int rows = a.group * a.nq;
  const int k0 = split * pl.chunk, k1 = min(min(k0 + pl.chunk, m.len), m.limit(a.nq - 1));
  const bf16* K = static_cast<const bf16*>(a.k.p) + b * a.k.b + hk * a.k.h;
  const bf16* V = static_cast<const bf16*>(a.v.p) + b * a.v.b + hk * a.v.h;
  const int* dk = a.doc_k ? a.doc_k + (long long)b * a.nk : nullptr;
  // rows g and g + 8 of this lane: query head, query, limit, document, slope
  int lim[2], doc[2], pos[2];
  float slope2[2];
  uint32_t qa[2][KL * 4];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int r = g + 8 * s, hq = hk * a.group + r / a.nq, i = r % a.nq;
    const bool in = r < rows;
    doc[s] = in && a.doc_q ? a.doc_q[(long long)b * a.nq + i] : 0;
    lim[s] = in && doc[s] >= 0 ? m.limit(i) : 0;
    pos[s] = i + m.off;
    slope2[s] = in && a.slopes ? a.slopes[hq] * kLog2e : 0.f;
#pragma unroll
    for (int l = 0; l < KL; ++l) {
      uint4 v = make_uint4(0u, 0u, 0u, 0u);                // padding is zeros whatever it holds
      if (in && doc[s] >= 0) v = *reinterpret_cast<const uint4*>(static_cast<const bf16*>(a.q.p) + b * a.q.b + hq * a.q.h + i * a.q.t + l * 32 + c * 8);
      qa[s][4 * l] = v.x; qa[s][4 * l + 1] = v.y; qa[s][4 * l + 2] = v.z; qa[s][4 * l + 3] = v.w;
    }
  }
  const SmScore sc = sm_score_of(a, hk * a.group);
  const float ka = sc.down, kb = sc.mid;
  const int sure = dk ? 0 : min(k1, m.limit(0));           // every row sees the keys before it (rows that do not exist go nowhere)
  float acc[NT][4], mx[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
  for (int j = 0; j < NT; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;

  extern __shared__ __align__(16) char st_smem[];
  constexpr int NP = step_pieces<D>();
  char* mine = st_smem + (size_t)warp * ST_STAGES * NP * 512 + lane * 16;    // [stage][piece][lane]
  // the 16 keys from j0: lane group g has keys j0 + g and j0 + 8 + g, and values of j0 + 2 c, + 1, + 8, + 9.  Absent ones are zeros
  // whatever they hold: a value is multiplied by its zero, and a cap's reciprocal is shared by four scores of a row.
  auto fetch = [&](int j0, int stage) {
    char* to = mine + stage * NP * 512;
    if (j0 < k1) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int j = j0 + 8 * t + g;
        const bool in = j < k1 && !(dk && dk[j] < 0);
        const bf16* row = K + (in ? (long long)j * a.k.t : 0) + c * 8;
#pragma unroll
        for (int l = 0; l < KL; ++l) step_copy<16>(to + (t * KL + l) * 512, row + l * 32, in);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int j = j0 + 2 * c + (u & 1) + 8 * (u >> 1);
        const bool in = j < k1 && !(dk && dk[j] < 0);
        const bf16* row = V + (in ? (long long)j * a.v.t : 0) + g * (D == 32 ? 4 : 8);
        char* at = to + (2 * KL + u * (D == 128 ? 2 : 1)) * 512;
        if (D == 32) step_copy<8>(at, row, in);
        else
#pragma unroll
          for (int q = 0; q < VW / 4; ++q) step_copy<16>(at + q * 512, row + q * 64, in);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int j0 = k0 + warp * 16, stage = 0;
#pragma unroll
  for (int s = 0; s < ST_STAGES - 1; ++s) fetch(j0 + s * ST_WARPS * 16, s);
  for (; j0 < k1; j0 += ST_WARPS * 16) {
    asm volatile("cp.async.wait_group %0;" ::"n"(ST_STAGES - 2) : "memory");
    const char* from = mine + stage * NP * 512;
    fetch(j0 + (ST_STAGES - 1) * ST_WARPS * 16, (stage + ST_STAGES - 1) % ST_STAGES);
    stage = (stage + 1) % ST_STAGES;
    float s[2][4] = {};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int l = 0; l < KL; ++l) {
        const uint4 kv = *reinterpret_cast<const uint4*>(from + (t * KL + l) * 512);
        const uint32_t A0[4] = {qa[0][4 * l], qa[1][4 * l], qa[0][4 * l + 1], qa[1][4 * l + 1]};
        const uint32_t A1[4] = {qa[0][4 * l + 2], qa[1][4 * l + 2], qa[0][4 * l + 3], qa[1][4 * l + 3]};
        mma_bf16(s[t], A0, kv.x, kv.y);
        mma_bf16(s[t], A1, kv.z, kv.w);
      }
    // scores in base 2: lane (g, c) has keys j0 + 8 t + 2 c + e for rows g and g + 8; a reciprocal of the cap serves one row's four,
    // so that a NaN stays in its row
    if (sc.kind != CAP_NONE) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float q[4] = {s[0][2 * r], s[0][2 * r + 1], s[1][2 * r], s[1][2 * r + 1]};
        if (sc.kind == CAP_WIDE) sm_cap4_wide(q, sc); else sm_cap4(q, sc.mul);
        s[0][2 * r] = q[0]; s[0][2 * r + 1] = q[1]; s[1][2 * r] = q[2]; s[1][2 * r + 1] = q[3];
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[t][e] = fmaf(s[t][e], ka, kb);
    if (a.slopes) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[t][e] = fmaf(-slope2[e >> 1], (float)abs(pos[e >> 1] - (j0 + 8 * t + 2 * c + (e & 1))), s[t][e]);
    }
    if (j0 + 16 > sure) {                                  // some row sees some of these keys not
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = j0 + 8 * t + 2 * c + (e & 1), r = e >> 1;
          if (!(j < lim[r] && j < k1 && (!dk || dk[j] == doc[r]))) s[t][e] = -INFINITY;
        }
    }
    float ref[2], old[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float top = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float now = fmaxf(mx[r], top);
      ref[r] = now == -INFINITY ? 0.f : now;
      old[r] = ex2(mx[r] - ref[r]);
      mx[r] = now;
      sum[r] *= old[r];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float p = ex2(s[t][2 * r + e] - ref[r]);
          s[t][2 * r + e] = p;
          sum[r] += p;
        }
    }
    if (__any_sync(0xffffffffu, old[0] != 1.f || old[1] != 1.f)) {
#pragma unroll
      for (int j = 0; j < NT; ++j) { acc[j][0] *= old[0]; acc[j][1] *= old[0]; acc[j][2] *= old[1]; acc[j][3] *= old[1]; }
    }
    const __nv_bfloat162 p0 = __floats2bfloat162_rn(s[0][0], s[0][1]), p1 = __floats2bfloat162_rn(s[0][2], s[0][3]);
    const __nv_bfloat162 p2 = __floats2bfloat162_rn(s[1][0], s[1][1]), p3 = __floats2bfloat162_rn(s[1][2], s[1][3]);
    const uint32_t A[4] = {*reinterpret_cast<const uint32_t*>(&p0), *reinterpret_cast<const uint32_t*>(&p1), *reinterpret_cast<const uint32_t*>(&p2),
                           *reinterpret_cast<const uint32_t*>(&p3)};
    uint32_t vb[4][VW];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const char* at = from + (2 * KL + u * (D == 128 ? 2 : 1)) * 512;
      if (D == 32) {
        const uint2 v = *reinterpret_cast<const uint2*>(at);
        vb[u][0] = v.x; vb[u][1] = v.y;
      } else {
#pragma unroll
        for (int q = 0; q < VW / 4; ++q) {
          const uint4 v = *reinterpret_cast<const uint4*>(at + q * 512);
          vb[u][4 * q] = v.x; vb[u][4 * q + 1] = v.y; vb[u][4 * q + 2] = v.z; vb[u][4 * q + 3] = v.w;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const uint32_t sel = j & 1 ? 0x7632u : 0x5410u;
      mma_bf16(acc[j], A, prmt(vb[0][j >> 1], vb[1][j >> 1], sel), prmt(vb[2][j >> 1], vb[3][j >> 1], sel));
    }
  }
  // join the warps: every warp leaves its maxima, sums and scaled accumulators, in the memory of the copies
  __shared__ float s_m[ST_WARPS][ST_ROWS], s_l[ST_WARPS][ST_ROWS];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], 1);
    sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], 2);
    if (c == 0) { s_m[warp][g + 8 * r] = mx[r]; s_l[warp][g + 8 * r] = sum[r]; }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();
  float* s_o = reinterpret_cast<float*>(st_smem);          // [warp][row][D + 4]
  float f[2];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < ST_WARPS; ++w) top = fmaxf(top, s_m[w][g + 8 * r]);
    f[r] = mx[r] == -INFINITY ? 0.f : ex2(mx[r] - top);
  }
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e)                            // column n = 2 c + (e & 1) of tile j: channel 8 n + j (j < 8), 64 + 8 n + j - 8; 4 n + j
      s_o[(warp * ST_ROWS + g + 8 * (e >> 1)) * (D + 4) + (j >> 3) * 64 + (2 * c + (e & 1)) * (D == 32 ? 4 : 8) + (j & 7)] = acc[j][e] * f[e >> 1];
  __syncthreads();
  step_write<bf16, D, ST_WARPS>(a, pl, part, b, hk, split, rows, &s_m[0][0], &s_l[0][0], ST_ROWS, s_o, ST_ROWS * (D + 4), D + 4);
}

// The same for fp32 storage on the CUDA cores (products with 24-bit operands), for up to RB rows.  A warp takes 32 keys a turn: lane
// (g, c) has channels 16 l + 4 c .. of key g of a group of eight, four groups one after the other; a dot product is the four lanes'
// shares added.  The exponentials go through shared memory, and every lane owns D / 32 channels of the accumulators.
template <int D, int RB>
__global__ void __launch_bounds__(ST_WARPS * 32) k_softmax_step_f32(const __grid_constant__ SmArgs a, StepPlan pl, StepPart part) {
  pdl_wait();
  constexpr int KL = D / 16, CD = D / 32;
  const int split = blockIdx.x, hk = blockIdx.y % a.Hk, b = blockIdx.y / a.Hk;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
  const SmMask m(a, b);
  const int rows = a.group * a.nq;
  const int k0 = split * pl.chunk, k1 = min(min(k0 + pl.chunk, m.len), m.limit(a.nq - 1));
  const float* K = static_cast<const float*>(a.k.p) + b * a.k.b + hk * a.k.h;
  const float* V = static_cast<const float*>(a.v.p) + b * a.v.b + hk * a.v.h;
  const int* dk = a.doc_k ? a.doc_k + (long long)b * a.nk : nullptr;
  __shared__ __align__(16) float s_q[RB][D], s_p[ST_WARPS][32][RB], s_o[RB][D];
  __shared__ int s_lim[RB], s_doc[RB], s_pos[RB];
  __shared__ float s_slope[RB], s_m[ST_WARPS][RB], s_l[ST_WARPS][RB];
  for (int e = tid; e < RB * D; e += ST_WARPS * 32) {
    const int r = e / D, ch = e % D;
    s_q[r][ch] = r < rows ? static_cast<const float*>(a.q.p)[b * a.q.b + (hk * a.group + r / a.nq) * a.q.h + (r % a.nq) * a.q.t + ch] : 0.f;
  }
  if (tid < RB) {
    const int i = tid % a.nq, doc = tid < rows && a.doc_q ? a.doc_q[(long long)b * a.nq + i] : 0;
    s_doc[tid] = doc;
    s_lim[tid] = tid < rows && doc >= 0 ? m.limit(i) : 0;
    s_pos[tid] = i + m.off;
    s_slope[tid] = tid < rows && a.slopes ? a.slopes[hk * a.group + tid / a.nq] * kLog2e : 0.f;
  }
  __syncthreads();
  float acc[RB][CD], mx[RB], sum[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    mx[r] = -INFINITY; sum[r] = 0.f;
#pragma unroll
    for (int q = 0; q < CD; ++q) acc[r][q] = 0.f;
  }
  for (int j0 = k0 + warp * 32; j0 < k1; j0 += ST_WARPS * 32) {
    float s[RB][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int j = j0 + 8 * t + g;
      float4 k[KL];
#pragma unroll
      for (int l = 0; l < KL; ++l) {
        k[l] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (j < k1) k[l] = __ldg(reinterpret_cast<const float4*>(K + (long long)j * a.k.t + l * 16 + c * 4));
      }
      const int doc = dk && j < k1 ? dk[j] : 0;
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        float d = 0.f;
#pragma unroll
        for (int l = 0; l < KL; ++l) {
          const float4 q = *reinterpret_cast<const float4*>(&s_q[r][l * 16 + c * 4]);
          d = fmaf(q.x, k[l].x, d); d = fmaf(q.y, k[l].y, d); d = fmaf(q.z, k[l].z, d); d = fmaf(q.w, k[l].w, d);
        }
        d += __shfl_xor_sync(0xffffffffu, d, 1);
        d += __shfl_xor_sync(0xffffffffu, d, 2);
        const float x = step_score(d, a, s_slope[r], s_pos[r] - j);
        s[r][t] = j < k1 && j < s_lim[r] && (!dk || doc == s_doc[r]) ? x : -INFINITY;
      }
    }
    __syncwarp();
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      float top = fmaxf(fmaxf(s[r][0], s[r][1]), fmaxf(s[r][2], s[r][3]));
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const float now = fmaxf(mx[r], top), ref = now == -INFINITY ? 0.f : now, old = ex2(mx[r] - ref);
      mx[r] = now;
      sum[r] *= old;
#pragma unroll
      for (int q = 0; q < CD; ++q) acc[r][q] *= old;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float p = ex2(s[r][t] - ref);
        sum[r] += p;
        if (c == (r & 3)) s_p[warp][8 * t + g][r] = p;
      }
    }
    __syncwarp();
    const int n = min(32, k1 - j0);
#pragma unroll 4
    for (int j = 0; j < n; ++j) {
      float v[CD];
      const bool in = !(dk && dk[j0 + j] < 0);             // absent keys are zeros whatever they hold
#pragma unroll
      for (int q = 0; q < CD; ++q) v[q] = in ? __ldg(V + (long long)(j0 + j) * a.v.t + q * 32 + lane) : 0.f;
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        const float p = s_p[warp][j][r];
#pragma unroll
        for (int q = 0; q < CD; ++q) acc[r][q] = fmaf(p, v[q], acc[r][q]);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < RB; ++r) {
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], o);
    if (lane == 0) { s_m[warp][r] = mx[r]; s_l[warp][r] = sum[r]; }
  }
  __syncthreads();
  for (int w = 0; w < ST_WARPS; ++w) {
    if (w == warp)
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        float t = -INFINITY;
#pragma unroll
        for (int k = 0; k < ST_WARPS; ++k) t = fmaxf(t, s_m[k][r]);
        const float f = mx[r] == -INFINITY ? 0.f : ex2(mx[r] - t);
#pragma unroll
        for (int q = 0; q < CD; ++q) s_o[r][q * 32 + lane] = (w ? s_o[r][q * 32 + lane] : 0.f) + acc[r][q] * f;
      }
    __syncthreads();
  }
  step_write<float, D, 1>(a, pl, part, b, hk, split, rows, &s_m[0][0], &s_l[0][0], RB, &s_o[0][0], 0, D);
}

// Partial results of a row -> its output and lse.  W warps per row take the parts in turns and are added in order: four where
// rows are few and parts many (a step: 18 parts of 128 rows 17 -> 11 us, of which 5 are the measurement), one where it is the other way round.
template <typename T, int W>
__global__ void __launch_bounds__(128) k_softmax_join(const __grid_constant__ SmArgs a, int splits, StepPart part) {
  pdl_wait();
  constexpr int R = 4 / W;                                 // rows a CTA
  const int lane = threadIdx.x & 31, w = (threadIdx.x >> 5) % W;
  const long long row = (long long)blockIdx.x * R + (threadIdx.x >> 5) / W;
  const bool in = row < (long long)a.B * a.Hq * a.nq;
  if (W == 1 && !in) return;                               // W = 4: one row a CTA, always in range
  const float2* ml = part.ml + row * splits;
  if (ml[0].y < 0.f) return;                               // a row that one CTA had whole is written already
  float top = -INFINITY;
  for (int s = lane; s < splits; s += 32) top = fmaxf(top, ml[s].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  float l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = w; s < splits; s += W) {
    const float2 m = ml[s];
    const float f = m.x == -INFINITY ? 0.f : ex2(m.x - top);
    l += m.x == -INFINITY ? m.y : m.y * f;                 // NaN stays
    const float* o = part.o + (row * splits + s) * a.d;
    if (f != 0.f)                                          // a part of nothing holds nothing
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q * 32 < a.d) acc[q] = fmaf(f, o[q * 32 + lane], acc[q]);
  }
  if (W > 1) {
    __shared__ float s_acc[W][4][32], s_l[W];
#pragma unroll
    for (int q = 0; q < 4; ++q) s_acc[w][q][lane] = acc[q];
    if (lane == 0) s_l[w] = l;
    __syncthreads();
    if (w) return;
#pragma unroll
    for (int k = 1; k < W; ++k) {
      l += s_l[k];
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[q] += s_acc[k][q][lane];
    }
  }
  const int i = (int)(row % a.nq), h = (int)(row / a.nq % a.Hq), b = (int)(row / a.nq / a.Hq);
  T* O = static_cast<T*>(a.o.p) + b * a.o.b + h * a.o.h + i * a.o.t;
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (q * 32 < a.d) O[q * 32 + lane] = from_f<T>(acc[q] * inv);
  if (lane == 0) a.lse[row] = l == 0.f ? -INFINITY : top * kLn2 + logf(l);
}

}  // namespace ln
