// C ABI of the query / key preparation and of softmax attention: host-side validation, buffer layout and launches.
#include <cudaTypedefs.h>
#include <math.h>
#include <stdint.h>
#include <algorithm>

#include "../../include/laplace_nystrom.h"
#include "ln_host.cuh"
#include "ln_rope.cuh"
#include "ln_softmax_simt.cuh"
#include "ln_softmax_step.cuh"
#include "ln_softmax_bwd_umma.cuh"
#include "ln_softmax_umma.cuh"

using namespace ln;
using namespace ln::host;

namespace {

constexpr long long kMostTokens = 1ll << 30, kMostRows = (1ll << 31) - 64, kMostTiled = 65535ll * 64;

// Strides of the three outer axes as the kernels use them (an axis of length one has none); false if the view cannot be read
// in 16-byte pieces, or if it is an output whose rows overlap.
bool open_view(const ln_view* v, long long B, long long H, long long n, int d, int dtype, bool output, long long (&s)[3]) {
  if (!v || !v->data || !aligned16(v->data)) return false;
  const int per = dtype == LN_F32 ? 4 : 8;
  const long long ext[3] = {B, H, n}, given[3] = {v->batch, v->head, v->token};
  for (int i = 0; i < 3; ++i) {
    s[i] = ext[i] == 1 ? 0 : given[i];
    if (s[i] < 0 || s[i] % per || s[i] > (1ll << 38)) return false;
  }
  if (!output) return true;
  int order[3] = {0, 1, 2};                         // by stride
  for (int i = 0; i < 2; ++i)
    for (int k = 0; k < 2 - i; ++k)
      if (s[order[k]] > s[order[k + 1]]) { const int t = order[k]; order[k] = order[k + 1]; order[k + 1] = t; }
  long long span = d;                               // elements that the axes so far cover
  for (int i = 0; i < 3; ++i) {
    const int o = order[i];
    if (ext[o] == 1) continue;
    if (s[o] < span) return false;
    span = s[o] * (ext[o] - 1) + span;
  }
  return true;
}

// ------------------------------------------------------------------------------------------ rotary positions, norms
int check_rope(const ln_rope* p, int B, int n, int Hq, int Hk) {
  if (!p || B <= 0 || n <= 0 || Hq <= 0 || Hk < 0 || p->d <= 0 || p->r < 0 || p->r > p->d) return LN_ERR_ARG;
  if (p->dtype != LN_F32 && p->dtype != LN_BF16) return LN_ERR_ARG;
  if ((p->r > 0) != (p->turns != nullptr) || !isfinite(p->factor)) return LN_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(p->turns) & 7u || reinterpret_cast<uintptr_t>(p->pos) & 3u) return LN_ERR_ARG;
  if ((p->d != 32 && p->d != 64 && p->d != 128) || p->r % 16) return LN_ERR_UNSUPPORTED;
  if (n > kMostTokens || (long long)B * n > kMostRows / ((long long)Hq + Hk)) return LN_ERR_UNSUPPORTED;
  return LN_OK;
}

// Heads per lane group and CTAs.  Every lane group forms the sines of its token once for all its heads, so a group walks as
// many heads as leave the GPU full: as many warps as are resident, at the four CTAs an SM that the kernel is built for, two in the backward
// pass.  64 x 197 tokens, 6 + 6 heads x 64: rotation 10.6 us, with the norm 14.0, backward 19.1; with groups for six CTAs an SM in all three
// 12.8, 16.2 and 23.4, and no shape faster.
struct QkPlan { int hpg, chunks, ctas; };
QkPlan plan_qk(const ln_rope* p, int B, int n, int heads, bool bwd) {
  const int lpr = p->d / (p->dtype == LN_F32 ? 4 : 8), tpw = 32 / lpr;
  const long long groups = ((long long)B * n + tpw - 1) / tpw, slots = 8ll * (bwd ? 2 : 4) * sm_count();       // warps resident
  int hpg = heads;
  while (hpg > 1 && groups * ((heads + hpg - 1) / hpg) < slots) hpg = (hpg + 1) / 2;
  QkPlan q;
  q.hpg = hpg; q.chunks = (heads + hpg - 1) / hpg;
  const long long want = (groups * q.chunks + 7) / 8, most = bwd ? 4ll * sm_count() : 24ll * sm_count();
  q.ctas = (int)(want < most ? want : most);
  return q;
}

int run_qk(const ln_rope* p, int mode, float sign, int B, int n, int Hq, int Hk, float eps, const float* gq, const float* gk,
           const ln_view* Q, const ln_view* K, const ln_view* dQr, const ln_view* dKr, const ln_view* Qo, const ln_view* Ko,
           float* dgq, float* dgk, float* part, cudaStream_t st) {
  QkArgs a = {};
  const ln_view *in[2] = {Q, K}, *up[2] = {dQr, dKr}, *out[2] = {Qo, Ko};
  const float* g[2] = {gq, gk};
  const int H[2] = {Hq, Hk};
  for (int s = 0; s < 2; ++s) {
    QkTensor& t = a.t[s];
    t.H = H[s]; t.g = g[s];
    if (!H[s]) continue;
    if (!open_view(in[s], B, H[s], n, p->d, p->dtype, false, t.xs) || !open_view(out[s], B, H[s], n, p->d, p->dtype, true, t.ys)) return LN_ERR_ARG;
    if (mode == QK_NORM_BWD && !open_view(up[s], B, H[s], n, p->d, p->dtype, false, t.ds)) return LN_ERR_ARG;
    t.x = in[s]->data; t.y = out[s]->data; t.dy = mode == QK_NORM_BWD ? up[s]->data : nullptr;
  }
  const QkPlan q = plan_qk(p, B, n, Hq + Hk, mode == QK_NORM_BWD);
  a.pos = p->pos; a.pos_b = p->pos_batch; a.pos_n = p->pos_token; a.start = p->start;
  a.tokens = B * n; a.n = n; a.r = p->r; a.heads = Hq + Hk; a.hpg = q.hpg; a.chunks = q.chunks;
  a.turns = reinterpret_cast<const unsigned long long*>(p->turns);
  a.factor = p->factor; a.sign = sign; a.eps = eps; a.dgpart = part;
  auto go = [&](auto type, auto lpr, auto inter) {
    using T = decltype(type);
    constexpr int L = decltype(lpr)::value;
    constexpr bool I = decltype(inter)::value;
    if (mode == QK_ROPE) LN_LAUNCH("k_rope_qk", st, enqueue(k_qk_rope<T, L, I, QK_ROPE>, q.ctas, 256, 0, st, a));
    else if (mode == QK_NORM) LN_LAUNCH("k_qk_norm_rope", st, enqueue(k_qk_rope<T, L, I, QK_NORM>, q.ctas, 256, 0, st, a));
    else LN_LAUNCH("k_qk_norm_rope_bwd", st, enqueue(k_qk_rope<T, L, I, QK_NORM_BWD>, q.ctas, 256, 0, st, a));
  };
  auto lanes = [&](auto type, auto inter) {
    constexpr int E = Piece<decltype(type)>::E;
    if (p->d == 32) go(type, std::integral_constant<int, 32 / E>(), inter);
    else if (p->d == 64) go(type, std::integral_constant<int, 64 / E>(), inter);
    else go(type, std::integral_constant<int, 128 / E>(), inter);
  };
  auto layout = [&](auto type) { if (p->interleaved) lanes(type, std::true_type()); else lanes(type, std::false_type()); };
  if (p->dtype == LN_F32) layout(float()); else layout(bf16());
  if (part) LN_LAUNCH("k_gain_sum", st, enqueue(k_gain_sum, 2 * p->d / 32, 1024, 0, st, part, q.ctas, p->d, dgq, dgk));
  return launch_ok();
}

// ------------------------------------------------------------------------------------------ softmax attention
int check_softmax(const ln_softmax* p, bool bwd) {
  if (!p || p->B <= 0 || p->Hq <= 0 || p->Hk <= 0 || p->nq <= 0 || p->nk <= 0 || p->d <= 0 || p->Hq % p->Hk) return LN_ERR_ARG;
  if (p->dtype != LN_F32 && p->dtype != LN_BF16) return LN_ERR_ARG;
  if (!(p->scale > 0.f) || !isfinite(p->scale) || !(p->cap >= 0.f) || !isfinite(p->cap) || (p->causal != 0 && p->causal != 1)) return LN_ERR_ARG;
  if ((p->prefix && !p->causal) || (p->doc_q != nullptr) != (p->doc_k != nullptr)) return LN_ERR_ARG;
  const void* words[] = {p->prefix, p->kv_len, p->slopes, p->doc_q, p->doc_k};
  for (const void* w : words)
    if (reinterpret_cast<uintptr_t>(w) & 3u) return LN_ERR_ARG;
  if ((p->d != 32 && p->d != 64 && p->d != 128) || (long long)p->B * p->Hq > 65535 || p->nq > kMostTiled || p->nk > (bwd ? kMostTiled : kMostTokens)) return LN_ERR_UNSUPPORTED;
  return LN_OK;
}

// A serving step: the rows that share a key head fit one 16-row tile.  Its keys are split over CTAs, eight for every SM in all (two are
// resident; sequences of a batch have different lengths; four or six: a tenth slower, twelve: more to join) and 256 keys at least.
bool is_step(const ln_softmax* p) { return (long long)(p->Hq / p->Hk) * p->nq <= ST_ROWS; }
StepPlan plan_step(const ln_softmax* p) {
  const long long heads = (long long)p->B * p->Hk, want = (8ll * sm_count() + heads - 1) / heads;
  long long chunk = (p->nk + want - 1) / want;
  chunk = (chunk + 127) / 128 * 128;
  if (chunk < 256) chunk = 256;
  StepPlan s;
  s.chunk = (int)chunk; s.splits = (int)cdiv(p->nk, chunk);
  return s;
}

// tcgen05 forward: query tiles a CTA (T), and the split of the keys over CTAs where the query tiles alone do not fill the GPU.
// One tile and two CTAs an SM: always with up to 64 channels (32 heads x 4096 tokens 205 us, two tiles 205; with a cap 406 and 447, with
// a bias 246 and 295), and for short rows; with 128 channels and long rows two tiles, which copy each key tile once for both.
struct SplitPlan { int tiles, chunk, splits; };
SplitPlan plan_split(const ln_softmax* p) {
  SplitPlan s;
  s.tiles = p->d <= 64 || p->nq <= 128 || p->nk <= 512 ? 1 : 2;
  const long long slots = (s.tiles == 1 ? 2ll : 1ll) * sm_count();           // CTAs resident
  const long long heads = (long long)p->B * p->Hq, blocks = cdiv(p->nq, 128 * s.tiles), keys = cdiv(p->nk, 128);
  s.chunk = (int)keys; s.splits = 1;
  if (blocks * heads >= 2 * slots) return s;
  // key tiles of all CTAs together; causal rows see half of the last nq keys
  long long total = blocks * keys;
  if (p->causal && !p->prefix) total -= blocks * (std::min(p->nq, p->nk) / 128) / 2;
  long long chunk = (total * heads + 3 * slots - 1) / (3 * slots);
  if (chunk < 8) chunk = 8;
  if (chunk >= keys) return s;
  s.chunk = (int)chunk; s.splits = (int)((keys + chunk - 1) / chunk);
  return s;
}

// Workspace: the documents of every 64 tokens, (backward) delta, (forward, a step) the splits' partial results.
struct SmWork { int4 *rq, *rk; float* delta; StepPart part; size_t bytes; };
SmWork carve_softmax(const ln_softmax* p, bool bwd, void* base) {
  Carver c(base);
  SmWork w = {};
  if (!bwd && is_step(p)) {
    const StepPlan s = plan_step(p);
    const size_t rows = (size_t)p->B * p->Hq * p->nq * s.splits;
    if (s.splits > 1) {
      w.part.o = c.take(rows * p->d);
      w.part.ml = reinterpret_cast<float2*>(c.take(rows * 2));
    }
    w.bytes = c.off;
    return w;
  }
  if (p->doc_q) {
    w.rq = reinterpret_cast<int4*>(c.take((size_t)p->B * cdiv(p->nq, 64) * 4));
    w.rk = reinterpret_cast<int4*>(c.take((size_t)p->B * cdiv(p->nk, 64) * 4));
  }
  if (bwd) w.delta = c.take((size_t)p->B * p->Hq * p->nq);
  if (!bwd && p->dtype == LN_BF16) {
    const SplitPlan s = plan_split(p);
    const size_t rows = (size_t)p->B * p->Hq * p->nq * s.splits;
    if (s.splits > 1) {
      w.part.o = c.take(rows * p->d);
      w.part.ml = reinterpret_cast<float2*>(c.take(rows * 2));
    }
  }
  w.bytes = c.off;
  return w;
}

SmArgs softmax_args(const ln_softmax* p, const SmWork& w, int32_t* dev_status) {
  SmArgs a = {};
  a.B = p->B; a.Hq = p->Hq; a.Hk = p->Hk; a.group = p->Hq / p->Hk; a.nq = p->nq; a.nk = p->nk; a.d = p->d;
  a.scale = p->scale; a.cap = p->cap; a.causal = p->causal; a.prefix = p->prefix; a.kv_len = p->kv_len; a.slopes = p->slopes;
  a.doc_q = p->doc_q; a.doc_k = p->doc_k; a.rq = w.rq; a.rk = w.rk; a.tq = (int)cdiv(p->nq, 64); a.tk = (int)cdiv(p->nk, 64);
  a.delta = w.delta; a.dev_status = dev_status;
  return a;
}

bool open_sm(const ln_softmax* p, const ln_view* v, bool keys, bool output, SmView* o) {
  long long s[3];
  if (!open_view(v, p->B, keys ? p->Hk : p->Hq, keys ? p->nk : p->nq, p->d, p->dtype, output, s)) return false;
  o->p = v->data; o->b = s[0]; o->h = s[1]; o->t = s[2];
  return s[2] || (keys ? p->nk : p->nq) == 1;       // a broadcast token axis has no tensor map
}

void softmax_docs(const SmArgs& a, const SmWork& w, cudaStream_t st) {
  if (a.doc_q) LN_LAUNCH("k_sm_docs", st, enqueue(k_sm_docs, dim3(a.tq + a.tk, a.B), 32, 0, st, a.doc_q, a.doc_k, a.nq, a.nk, a.tq, a.tk, w.rq, w.rk));
}

template <typename T> void softmax_join(const SmArgs& a, int splits, const StepPart& part, cudaStream_t st) {
  const long long rows = (long long)a.B * a.Hq * a.nq;
  if (rows <= 16ll * sm_count()) LN_LAUNCH("k_softmax_join", st, enqueue(k_softmax_join<T, 4>, dim3((unsigned)rows), 128, 0, st, a, splits, part));
  else LN_LAUNCH("k_softmax_join", st, enqueue(k_softmax_join<T, 1>, dim3(cdiv(rows, 4)), 128, 0, st, a, splits, part));
}

void softmax_step(const ln_softmax* p, const SmArgs& a, const SmWork& w, cudaStream_t st) {
  const StepPlan s = plan_step(p);
  const dim3 grid(s.splits, a.B * a.Hk);
  auto go = [&](auto kern, size_t smem = 0) {
    if (smem) want_smem(kern, smem);
    LN_LAUNCH("k_softmax_step", st, enqueue(kern, grid, ST_WARPS * 32, smem, st, a, s, w.part));
  };
  auto f32 = [&](auto d) {
    constexpr int D = decltype(d)::value;
    const int rows = a.group * a.nq;
    if (rows == 1) go(k_softmax_step_f32<D, 1>); else if (rows <= 4) go(k_softmax_step_f32<D, 4>); else go(k_softmax_step_f32<D, ST_ROWS>);
  };
  if (p->dtype == LN_BF16) { if (p->d == 32) go(k_softmax_step<32>, step_smem<32>()); else if (p->d == 64) go(k_softmax_step<64>, step_smem<64>()); else go(k_softmax_step<128>, step_smem<128>()); }
  else if (p->d == 32) f32(std::integral_constant<int, 32>());
  else if (p->d == 64) f32(std::integral_constant<int, 64>());
  else f32(std::integral_constant<int, 128>());
  if (s.splits == 1) return;
  if (p->dtype == LN_BF16) softmax_join<bf16>(a, s.splits, w.part, st); else softmax_join<float>(a, s.splits, w.part, st);
}

template <int D> void softmax_fwd_simt(const SmArgs& a, cudaStream_t st) {
  want_smem(k_softmax_fwd<D>, sm_fwd_smem<D>());
  LN_LAUNCH("k_softmax_fwd", st, enqueue(k_softmax_fwd<D>, dim3(a.B * a.Hq, cdiv(a.nq, SS)), 256, sm_fwd_smem<D>(), st, a));
}
template <int D> void softmax_bwd_simt(const SmArgs& a, cudaStream_t st) {
  want_smem(k_softmax_bwd<D, false>, sm_bwd_smem<D, false>());
  LN_LAUNCH("k_softmax_bwd_q", st, enqueue(k_softmax_bwd<D, false>, dim3(a.B * a.Hq, cdiv(a.nq, SS)), 256, sm_bwd_smem<D, false>(), st, a));
  want_smem(k_softmax_bwd<D, true>, sm_bwd_smem<D, true>());
  LN_LAUNCH("k_softmax_bwd_kv", st, enqueue(k_softmax_bwd<D, true>, dim3(a.B * a.Hk, cdiv(a.nk, SS)), 256, sm_bwd_smem<D, true>(), st, a));
}

// The driver's encoder of tensor maps, by name (the library is not linked against the driver).
PFN_cuTensorMapEncodeTiled_v12000 map_encoder() {
  static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) p = nullptr;
    cudaGetLastError();
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  }();
  return fn;
}

// Tensor map of a bf16 [B, H, n, d] view for blocks of `rows` rows x 64 channels; channels behind d and rows behind n arrive as zeros.
bool tile_map(const SmView& v, int B, int H, int n, int d, int rows, TileMap* m) {
  const auto encode = map_encoder();
  if (!encode) return false;
  m->head = v.h != 0; m->batch = v.b != 0;
  const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)n, (cuuint64_t)(m->head ? H : 1), (cuuint64_t)(m->batch ? B : 1)};
  // a stride of zero: an axis of length one, or one that the map leaves out
  const cuuint64_t strides[3] = {(cuuint64_t)(v.t ? 2 * v.t : 16), (cuuint64_t)(v.h ? 2 * v.h : 16), (cuuint64_t)(v.b ? 2 * v.b : 16)};
  const cuuint32_t box[4] = {64, (cuuint32_t)rows, 1, 1}, step[4] = {1, 1, 1, 1};
  return encode(&m->map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, v.p, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// f(kind of the cap), a constant
template <typename F> void by_cap(float cap, const F& f) {
  const int kind = cap_kind(cap);
  if (kind == CAP_WIDE) f(std::integral_constant<int, CAP_WIDE>());
  else if (kind == CAP_USUAL) f(std::integral_constant<int, CAP_USUAL>());
  else f(std::integral_constant<int, CAP_NONE>());
}

template <int D, int T> int softmax_fwd_umma(const SmArgs& a, const SplitPlan& pl, const StepPart& part, cudaStream_t st) {
  TileMap q, k, v;
  if (!tile_map(a.q, a.B, a.Hq, a.nq, a.d, 128, &q) || !tile_map(a.k, a.B, a.Hk, a.nk, a.d, 128, &k) || !tile_map(a.v, a.B, a.Hk, a.nk, a.d, 128, &v)) return LN_ERR_CUDA;
  const SmSplit sp = {pl.chunk, pl.splits, part.o, part.ml};
  auto go = [&](auto kern) {
    want_smem(kern, SuFwd<D, T>::kSmem);
    LN_LAUNCH("k_softmax_fwd", st, enqueue(kern, dim3(a.B * a.Hq, cdiv(a.nq, T * 128), pl.splits), SuFwd<D, T>::kThreads, SuFwd<D, T>::kSmem, st, a, q, k, v, sp));
  };
  auto bias = [&](auto cap) {
    constexpr int C = decltype(cap)::value;
    if (a.slopes) go(k_softmax_fwd_umma<D, T, C, true>); else go(k_softmax_fwd_umma<D, T, C, false>);
  };
  by_cap(a.cap, bias);
  if (pl.splits > 1) softmax_join<bf16>(a, pl.splits, part, st);
  return LN_OK;
}

template <int D> int softmax_bwd_umma(const SmArgs& a, cudaStream_t st) {
  TileMap sq, sdo, sk, sv, mq, mdo, mk, mv;                                  // stationary tiles of 128 rows, moving ones of 64
  if (!tile_map(a.q, a.B, a.Hq, a.nq, a.d, 128, &sq) || !tile_map(a.dout, a.B, a.Hq, a.nq, a.d, 128, &sdo) || !tile_map(a.k, a.B, a.Hk, a.nk, a.d, 128, &sk) ||
      !tile_map(a.v, a.B, a.Hk, a.nk, a.d, 128, &sv) || !tile_map(a.q, a.B, a.Hq, a.nq, a.d, 64, &mq) || !tile_map(a.dout, a.B, a.Hq, a.nq, a.d, 64, &mdo) ||
      !tile_map(a.k, a.B, a.Hk, a.nk, a.d, 64, &mk) || !tile_map(a.v, a.B, a.Hk, a.nk, a.d, 64, &mv)) return LN_ERR_CUDA;
  auto go = [&](auto q, auto kv) {
    want_smem(q, SuBwd<D>::kSmem);
    LN_LAUNCH("k_softmax_bwd_q", st, enqueue(q, dim3(a.B * a.Hq, cdiv(a.nq, 128)), SuBwd<D>::kThreads, SuBwd<D>::kSmem, st, a, sq, sdo, mk, mv));
    want_smem(kv, SuBwd<D>::kSmem);
    LN_LAUNCH("k_softmax_bwd_kv", st, enqueue(kv, dim3(a.B * a.Hk, cdiv(a.nk, 128)), SuBwd<D>::kThreads, SuBwd<D>::kSmem, st, a, sk, sv, mq, mdo));
  };
  auto bias = [&](auto cap) {
    constexpr int C = decltype(cap)::value;
    if (a.slopes) go(k_softmax_bwd_umma<D, C, true, false>, k_softmax_bwd_umma<D, C, true, true>);
    else go(k_softmax_bwd_umma<D, C, false, false>, k_softmax_bwd_umma<D, C, false, true>);
  };
  by_cap(a.cap, bias);
  return LN_OK;
}

}  // namespace

extern "C" {

int rope_fwd(const ln_rope* p, int32_t B, int32_t n, int32_t Hq, int32_t Hk, const ln_view* Q, const ln_view* K, const ln_view* Qr,
             const ln_view* Kr, void* stream) {
  const int rc = check_rope(p, B, n, Hq, Hk);
  if (rc != LN_OK) return rc;
  return run_qk(p, QK_ROPE, 1.f, B, n, Hq, Hk, 0.f, nullptr, nullptr, Q, K, nullptr, nullptr, Qr, Kr, nullptr, nullptr, nullptr, static_cast<cudaStream_t>(stream));
}

int rope_bwd(const ln_rope* p, int32_t B, int32_t n, int32_t Hq, int32_t Hk, const ln_view* dQr, const ln_view* dKr, const ln_view* dQ,
             const ln_view* dK, void* stream) {
  const int rc = check_rope(p, B, n, Hq, Hk);
  if (rc != LN_OK) return rc;
  return run_qk(p, QK_ROPE, -1.f, B, n, Hq, Hk, 0.f, nullptr, nullptr, dQr, dKr, nullptr, nullptr, dQ, dK, nullptr, nullptr, nullptr, static_cast<cudaStream_t>(stream));
}

int qk_norm_rope_fwd(const ln_rope* p, int32_t B, int32_t n, int32_t Hq, int32_t Hk, float eps, const float* gq, const float* gk,
                     const ln_view* Q, const ln_view* K, const ln_view* Qr, const ln_view* Kr, void* stream) {
  const int rc = check_rope(p, B, n, Hq, Hk);
  if (rc != LN_OK) return rc;
  if (!(eps >= 0.f) || !isfinite(eps) || !aligned16(gq) || !aligned16(gk)) return LN_ERR_ARG;
  return run_qk(p, QK_NORM, 1.f, B, n, Hq, Hk, eps, gq, gk, Q, K, nullptr, nullptr, Qr, Kr, nullptr, nullptr, nullptr, static_cast<cudaStream_t>(stream));
}

size_t qk_norm_rope_bwd_workspace_bytes(const ln_rope* p, int32_t B, int32_t n, int32_t Hq, int32_t Hk) {
  if (check_rope(p, B, n, Hq, Hk) != LN_OK) return 0;
  return align_up((size_t)plan_qk(p, B, n, Hq + Hk, true).ctas * 2 * p->d * sizeof(float), 256);
}

int qk_norm_rope_bwd(const ln_rope* p, int32_t B, int32_t n, int32_t Hq, int32_t Hk, float eps, const float* gq, const float* gk,
                     const ln_view* Q, const ln_view* K, const ln_view* dQr, const ln_view* dKr, const ln_view* dQ, const ln_view* dK,
                     float* dgq, float* dgk, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_rope(p, B, n, Hq, Hk);
  if (rc != LN_OK) return rc;
  if (!(eps >= 0.f) || !isfinite(eps) || !aligned16(gq) || !aligned16(gk) || !aligned16(dgq) || !aligned16(dgk)) return LN_ERR_ARG;
  const bool gains = dgq || dgk;
  if (gains && (!ws || !aligned16(ws))) return LN_ERR_ARG;
  if (gains && ws_bytes < qk_norm_rope_bwd_workspace_bytes(p, B, n, Hq, Hk)) return LN_ERR_WORKSPACE;
  return run_qk(p, QK_NORM_BWD, -1.f, B, n, Hq, Hk, eps, gq, gk, Q, K, dQr, dKr, dQ, dK, dgq, dgk, gains ? static_cast<float*>(ws) : nullptr,
                static_cast<cudaStream_t>(stream));
}

size_t softmax_attention_workspace_bytes(const ln_softmax* p, int32_t backward) {
  if (check_softmax(p, backward != 0) != LN_OK) return 0;
  const size_t n = carve_softmax(p, backward != 0, nullptr).bytes;
  return n ? n : 256;                               // never 0 for a valid problem
}

int softmax_attention_fwd(const ln_softmax* p, const ln_view* Q, const ln_view* K, const ln_view* V, const ln_view* O, float* lse, void* ws,
                          size_t ws_bytes, int32_t* dev_status, void* stream) {
  const int rc = check_softmax(p, false);
  if (rc != LN_OK) return rc;
  const SmWork w = carve_softmax(p, false, ws);
  SmArgs a = softmax_args(p, w, dev_status);
  if (!open_sm(p, Q, false, false, &a.q) || !open_sm(p, K, true, false, &a.k) || !open_sm(p, V, true, false, &a.v) || !open_sm(p, O, false, true, &a.o)) return LN_ERR_ARG;
  if (!lse || !aligned16(lse) || !ws || !aligned16(ws)) return LN_ERR_ARG;
  if (ws_bytes < w.bytes) return LN_ERR_WORKSPACE;
  a.lse = lse;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dev_status) cudaMemsetAsync(dev_status, 0, sizeof(int32_t) * (size_t)p->B * p->Hq, st);
  if (is_step(p)) { softmax_step(p, a, w, st); return launch_ok(); }
  softmax_docs(a, w, st);
  int made = LN_OK;
  if (p->dtype == LN_BF16) {
    const SplitPlan pl = plan_split(p);
    if (p->d <= 64) made = softmax_fwd_umma<64, 1>(a, pl, w.part, st);
    else made = pl.tiles == 1 ? softmax_fwd_umma<128, 1>(a, pl, w.part, st) : softmax_fwd_umma<128, 2>(a, pl, w.part, st);
  }
  else if (p->d == 32) softmax_fwd_simt<32>(a, st);
  else if (p->d == 64) softmax_fwd_simt<64>(a, st);
  else softmax_fwd_simt<128>(a, st);
  const int launched = launch_ok();
  return made != LN_OK ? made : launched;
}

int softmax_attention_bwd(const ln_softmax* p, const ln_view* Q, const ln_view* K, const ln_view* V, const ln_view* O, const float* lse,
                          const ln_view* dO, const ln_view* dQ, const ln_view* dK, const ln_view* dV, void* ws, size_t ws_bytes, int32_t* dev_status,
                          void* stream) {
  const int rc = check_softmax(p, true);
  if (rc != LN_OK) return rc;
  const SmWork w = carve_softmax(p, true, ws);
  SmArgs a = softmax_args(p, w, dev_status);
  if (!open_sm(p, Q, false, false, &a.q) || !open_sm(p, K, true, false, &a.k) || !open_sm(p, V, true, false, &a.v) || !open_sm(p, O, false, false, &a.o) ||
      !open_sm(p, dO, false, false, &a.dout) || !open_sm(p, dQ, false, true, &a.dq) || !open_sm(p, dK, true, true, &a.dk) || !open_sm(p, dV, true, true, &a.dv)) return LN_ERR_ARG;
  if (!lse || !aligned16(lse) || !ws || !aligned16(ws)) return LN_ERR_ARG;
  if (ws_bytes < w.bytes) return LN_ERR_WORKSPACE;
  a.lse = const_cast<float*>(lse);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dev_status) cudaMemsetAsync(dev_status, 0, sizeof(int32_t) * (size_t)p->B * p->Hq, st);
  softmax_docs(a, w, st);
  int made = LN_OK;
  if (p->dtype == LN_BF16) made = p->d == 128 ? softmax_bwd_umma<128>(a, st) : softmax_bwd_umma<64>(a, st);
  else if (p->d == 32) softmax_bwd_simt<32>(a, st);
  else if (p->d == 64) softmax_bwd_simt<64>(a, st);
  else softmax_bwd_simt<128>(a, st);
  const int launched = launch_ok();
  return made != LN_OK ? made : launched;
}

}  // extern "C"
