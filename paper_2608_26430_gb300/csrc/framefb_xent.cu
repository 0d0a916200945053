// Entry points of the linear head's cross entropy: checks, workspace layout,
// tensor maps, launches (kernels in framefb_xent.cuh).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <initializer_list>

#include "framefb.h"
#include "framefb_dense.h"
#include "framefb_xent.cuh"
#include "framefb_xent.h"

namespace {

namespace fx = ffb::xent;

constexpr int64_t kMaxDim = int64_t{1} << 30;       // tokens, features, vocabulary: TMA coordinates are 32-bit
constexpr int kFewSmem = 100 * 1024;                // H of few tokens: two blocks on an SM
constexpr int64_t kPieceBytes = int64_t{256} << 20; // P of one piece of the vocabulary

inline int64_t rup(int64_t x, int64_t a) { return (x + a - 1) / a * a; }
inline bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 0;
  return sms;
}

// How a call is cut, and where its workspace regions start (bytes).
struct Plan {
  int64_t npad, ldc;         // token rows up to whole tiles; row length of the gathered H
  int64_t vp;                // vocabulary columns of a piece (a multiple of kBN)
  int32_t parts;             // bf16 parts of P
  int32_t bn;                // forward: columns of a tile
  bool join;                 // tiles may be cut into slices
  int64_t head, idx, tgt, hc, tlogit, rowloss, part, coef, lse, P, acc, slots, bytes;
};

// Sizes within TMA's coordinates, and tile counts within 31 bits.
bool sizes_ok(int64_t N, int32_t d, int32_t V) {
  if (N < 0 || N > kMaxDim || d < 1 || d > kMaxDim || V < 1 || V > kMaxDim) return false;
  const int64_t mt = N / fx::kHalf + 1, vt = V / fx::kHalf + 1, dt = d / fx::kBN + 1;
  return mt * vt <= INT32_MAX && vt * dt + mt * dt <= INT32_MAX;
}

// Columns of a launch's tiles (kb: K blocks of its shortest sums): 256; 128
// where 256 would leave pairs without a tile (64 tokens of 768 x 1000, dH and
// dW: 34.6 -> 26.0 us); 512, whose epilogues nothing hides and whose last
// round costs more, where a pair has 16 tiles of long sums (2048 tokens of
// 4096 x 120011, dH and dW: 3.92 -> 3.80 ms; 8192 of 4096 x 32000, forward:
// 1.18 -> 1.13 ms).
int tile_columns(int64_t mt, int64_t cols, int64_t kb, int pairs) {
  if (mt * ((cols + fx::kBN - 1) / fx::kBN) < pairs) return fx::kBN / 2;
  return kb >= 32 && mt * ((cols + fx::kMaxBN - 1) / fx::kMaxBN) >= 16 * pairs ? fx::kMaxBN : fx::kBN;
}

Plan plan_of(int64_t N, int32_t d, int32_t V, int32_t ops, int pairs) {
  Plan p{};
  p.npad = std::max<int64_t>(rup(N, fx::kBM), fx::kBM);
  p.ldc = rup(d, 64);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t o = at;
    at = rup(at + bytes, 1024);
    return o;
  };
  p.head = take(sizeof(fx::Head));
  p.idx = take(p.npad * 4);
  p.tgt = take(p.npad * 4);
  p.hc = take(N * p.ldc * 2);
  if (ops & FRAMEFB_XENT_FORWARD) {
    p.tlogit = take(p.npad * 4);
    p.rowloss = take(p.npad * 4);
    p.bn = tile_columns(p.npad / fx::kBM, V, (d + fx::kBK - 1) / fx::kBK, pairs);
    p.part = take(std::max<int64_t>(p.npad * ((V + p.bn / 2 - 1) / (p.bn / 2)),
                                    int64_t{4} * pairs * fx::kFewTokens) * 8);
  }
  if (ops & (FRAMEFB_XENT_DH | FRAMEFB_XENT_DW)) {
    p.coef = take(p.npad * 4);
    p.lse = take(p.npad * 4);
    p.parts = N <= fx::kHalf ? 2 : 1;
    // pieces of equal size whose P takes at most kPieceBytes (at least one column tile)
    const int64_t most = std::max<int64_t>(kPieceBytes / (2 * p.parts * p.npad) / fx::kMaxBN * fx::kMaxBN, fx::kMaxBN);
    const int64_t pieces = (V + most - 1) / most;
    p.vp = rup((V + pieces - 1) / pieces, fx::kMaxBN);
    p.P = take(p.npad * p.parts * p.vp * 2);
    const int64_t slot = 2 * fx::slot_floats(fx::kMaxBN) * 4;  // of a pair
    if ((ops & FRAMEFB_XENT_DH) && V > p.vp) p.acc = take(p.npad / fx::kBM * ((d + fx::kMaxBN - 1) / fx::kMaxBN) * slot);
    // K long enough for slices (dH: over the piece, dW: over the tokens): at most one a pair each
    const bool sh = (ops & FRAMEFB_XENT_DH) && p.vp / fx::kBK * p.parts >= 2 * fx::kMinSlice;
    const bool sw = (ops & FRAMEFB_XENT_DW) && (N + fx::kBK - 1) / fx::kBK * p.parts >= 2 * fx::kMinSlice;
    p.join = sh || sw;
    if (p.join) p.slots = take((sh + sw) * pairs * slot);
  }
  p.bytes = at;
  return p;
}

// Tensor map of a row-major bf16 [rows][cols] array in 64 x 64 boxes.
bool encode(CUtensorMap* map, const void* base, int64_t cols, int64_t rows, int64_t ld) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld) * 2};
  const cuuint32_t box[2] = {64, 64};
  return ffb_host::encode_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

bool rows_ok(const void* p, int64_t ld, int32_t d) {
  return p && aligned16(p) && ld >= d && ld % 8 == 0 && ld <= (int64_t{1} << 38);
}

// CTA pairs of the contraction kernel that the current device runs at once
// (0 when a query fails).  Asked once per device, with the kernels' shared
// memory limits set at the same time.
int resident_pairs() {
  static std::atomic<int> known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  int n = known[dev].load(std::memory_order_acquire);
  if (n > 0) return n;
  for (const auto f : {fx::xent_gemm_kernel<fx::STATS, fx::kBN>, fx::xent_gemm_kernel<fx::STATS, fx::kBN / 2>,
                       fx::xent_gemm_kernel<fx::STATS, fx::kMaxBN>, fx::xent_gemm_kernel<fx::PROB, fx::kBN>,
                       fx::xent_gemm_kernel<fx::PROB, fx::kBN / 2>, fx::xent_gemm_kernel<fx::PROB, fx::kMaxBN>,
                       fx::xent_gemm_kernel<fx::GRADS, fx::kBN>, fx::xent_gemm_kernel<fx::GRADS, fx::kBN / 2>,
                       fx::xent_gemm_kernel<fx::GRADS, fx::kMaxBN>})
    if (cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, fx::kSmem) != cudaSuccess) return 0;
  for (const auto f : {fx::xent_few_kernel<1>, fx::xent_few_kernel<2>, fx::xent_few_kernel<4>})
    if (cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem) != cudaSuccess) return 0;
  cudaLaunchAttribute cluster{};
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = 2;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(2 * static_cast<unsigned>(std::max(1, sm_count())));
  cfg.blockDim = dim3(fx::kThreads);
  cfg.dynamicSmemBytes = fx::kSmem;
  cfg.attrs = &cluster;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&n, fx::xent_gemm_kernel<fx::STATS, fx::kBN>, &cfg) != cudaSuccess) return 0;
  known[dev].store(n, std::memory_order_release);
  return n;
}

// `chained`: the kernel may start while the call's previous one ends
// (programmatic dependent launch; it waits by itself).
framefb_status launch(const void* f, int64_t blocks, int threads, size_t smem, void** kargs, bool chained,
                      cudaStream_t st) {
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks));
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = chained ? 1 : 0;
  return cudaLaunchKernelExC(&cfg, f, kargs) == cudaSuccess ? FRAMEFB_OK : FRAMEFB_ECUDA;
}

template <typename Args>
framefb_status launch(void (*f)(Args), int64_t blocks, int threads, size_t smem, const Args& args, bool chained,
                      cudaStream_t st) {
  void* kargs[] = {const_cast<Args*>(&args)};
  return launch(reinterpret_cast<const void*>(f), blocks, threads, smem, kargs, chained, st);
}

// One persistent pair of CTAs per pair of SMs (as many as the device runs at
// once: the pairs take fixed shares of the tiles).
template <int MODE, int BN>
framefb_status launch_gemm(int64_t tiles, int pairs, const fx::GemmArgs& g, cudaStream_t st) {
  return launch(fx::xent_gemm_kernel<MODE, BN>, 2 * std::min<int64_t>(tiles, pairs), fx::kThreads, fx::kSmem, g, true, st);
}

// The logits of `cols` columns (STATS, PROB) in tiles of bn columns.
template <int MODE>
framefb_status launch_logits(int64_t mt, int64_t cols, int bn, int pairs, const fx::GemmArgs& g, cudaStream_t st) {
  const int64_t tiles = mt * ((cols + bn - 1) / bn);
  return bn > fx::kBN    ? launch_gemm<MODE, fx::kMaxBN>(tiles, pairs, g, st)
         : bn == fx::kBN ? launch_gemm<MODE, fx::kBN>(tiles, pairs, g, st)
                         : launch_gemm<MODE, fx::kBN / 2>(tiles, pairs, g, st);
}

#define FFB_TRY(x)                           \
  do {                                       \
    const framefb_status st_ = (x);          \
    if (st_ != FRAMEFB_OK) return st_;       \
  } while (0)

// dH and dW of a piece, and the sums of the tiles that are cut into slices
// (`join`: there may be some).  More CTAs than tiles may be asked for.
template <int BN>
framefb_status launch_grads(int64_t mt, bool join, int pairs, const fx::GemmArgs& g, cudaStream_t st) {
  const int64_t vt = g.vp / fx::kBM, nt = (g.d + BN - 1) / BN;
  const int64_t tiles = join ? pairs : ((g.dh ? mt : 0) + (g.dw ? vt : 0)) * nt;
  const int32_t used = static_cast<int32_t>(std::min<int64_t>(tiles, pairs));
  FFB_TRY((launch_gemm<fx::GRADS, BN>(tiles, pairs, g, st)));
  if (!join) return FRAMEFB_OK;
  fx::GemmArgs a = g;
  int32_t n = used;
  void* kargs[] = {&a, &n};
  return launch(reinterpret_cast<const void*>(fx::xent_join_kernel<BN>), 2 * pairs, fx::kJoinThreads, 0, kargs, true, st);
}

// The checks that both directions share.
framefb_status check(const framefb_xent* x, framefb_dtype dtype) {
  if (!x || (dtype != FRAMEFB_BF16 && dtype != FRAMEFB_F32) || !sizes_ok(x->N, x->d, x->V)) return FRAMEFB_EINVAL;
  if (dtype != FRAMEFB_BF16) return FRAMEFB_EUNSUPPORTED;
  if (reinterpret_cast<uintptr_t>(x->target) % 8) return FRAMEFB_EINVAL;
  if (x->N > 0 && (!rows_ok(x->H, x->ldh, x->d) || !rows_ok(x->W, x->ldw, x->d) || !x->target || !x->lse))
    return FRAMEFB_EINVAL;
  return FRAMEFB_OK;
}

// fp32 vectors (NULL passes), in the direction that looks at them.
bool aligned4(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (reinterpret_cast<uintptr_t>(p) % 4) return false;
  return true;
}

framefb_status check_ws(const Plan& p, const void* ws, size_t ws_bytes) {
  if (!ws || ws_bytes < static_cast<size_t>(p.bytes)) return FRAMEFB_EWORKSPACE;
  return reinterpret_cast<uintptr_t>(ws) % 256 ? FRAMEFB_EINVAL : FRAMEFB_OK;
}

// The arguments of xent_prep_kernel that both directions share.
fx::PrepArgs prep_args(const framefb_xent* x, const Plan& p, char* w) {
  fx::PrepArgs a{};
  a.N = x->N;
  a.chunk = (x->N + fx::kPrepBlocks - 1) / fx::kPrepBlocks;
  a.ignore = x->ignore_index;
  a.V = x->V;
  a.d = x->d;
  a.target = x->target;
  a.H = static_cast<const __nv_bfloat16*>(x->H);
  a.ldh = x->ldh;
  a.ldc = p.ldc;
  a.head = reinterpret_cast<fx::Head*>(w + p.head);
  a.idx = reinterpret_cast<int32_t*>(w + p.idx);
  a.tgt = reinterpret_cast<int32_t*>(w + p.tgt);
  a.Hc = reinterpret_cast<__nv_bfloat16*>(w + p.hc);
  return a;
}

framefb_status launch_prep(const fx::PrepArgs& a, cudaStream_t st) {
  return launch(fx::xent_prep_kernel, (a.N + a.chunk - 1) / a.chunk, fx::kPrepThreads, 0, a, false, st);
}

// The forward pass of few tokens: one launch streams W, one joins its blocks.
int64_t few_smem(int nt, int32_t d) { return (int64_t{d} + 7) / 8 * 2 * nt * static_cast<int64_t>(sizeof(float4)); }

int few_nt(int64_t N) { return N <= 1 ? 1 : N <= 2 ? 2 : 4; }

bool few(int64_t N, int32_t d) { return N <= fx::kFewTokens && few_smem(few_nt(N), d) <= kFewSmem; }

framefb_status launch_few(fx::FewArgs& a, int pairs, cudaStream_t st) {
  const int nt = few_nt(a.N);
  const auto f = nt == 1 ? fx::xent_few_kernel<1> : nt == 2 ? fx::xent_few_kernel<2> : fx::xent_few_kernel<4>;
  const int64_t per = fx::kFewThreads / 32 * fx::kFewRows;
  a.blocks = static_cast<int32_t>(std::min<int64_t>((a.V + per - 1) / per, std::min(fx::few_blocks(nt) * sm_count(), 4 * pairs)));
  if (a.blocks <= 0) return FRAMEFB_ECUDA;
  FFB_TRY(launch(f, a.blocks, fx::kFewThreads, few_smem(nt, a.d), a, false, st));
  return launch(fx::xent_few_loss_kernel, 1, 32 * fx::kFewTokens, 0, a, true, st);
}

}  // namespace

extern "C" size_t framefb_xent_workspace_size(int64_t N, int32_t d, int32_t V, int32_t ops) {
  const int pairs = resident_pairs();
  if (!sizes_ok(N, d, V) || N == 0 || pairs <= 0) return 0;
  return static_cast<size_t>(plan_of(N, d, V, ops, pairs).bytes);
}

extern "C" framefb_status framefb_xent_forward(const framefb_xent* x, framefb_dtype dtype, void* ws, size_t ws_bytes,
                                               void* stream) {
  FFB_TRY(check(x, dtype));
  if (!aligned4({x->loss, x->lse, x->loss_mean})) return FRAMEFB_EINVAL;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (x->N == 0) {
    if (x->loss_mean && cudaMemsetAsync(x->loss_mean, 0, sizeof(float), st) != cudaSuccess) return FRAMEFB_ECUDA;
    return FRAMEFB_OK;
  }
  if (!x->loss) return FRAMEFB_EINVAL;
  const int pairs = resident_pairs();
  if (pairs <= 0) return FRAMEFB_ECUDA;
  const Plan p = plan_of(x->N, x->d, x->V, FRAMEFB_XENT_FORWARD, pairs);
  FFB_TRY(check_ws(p, ws, ws_bytes));
  char* w = static_cast<char*>(ws);

  if (few(x->N, x->d)) {
    fx::FewArgs f{};
    f.N = static_cast<int32_t>(x->N);
    f.d = x->d;
    f.V = x->V;
    f.ignore = x->ignore_index;
    f.target = x->target;
    f.H = static_cast<const __nv_bfloat16*>(x->H);
    f.ldh = x->ldh;
    f.W = static_cast<const __nv_bfloat16*>(x->W);
    f.ldw = x->ldw;
    f.part = reinterpret_cast<float2*>(w + p.part);
    f.tlogit = reinterpret_cast<float*>(w + p.tlogit);
    f.loss = x->loss;
    f.lse = x->lse;
    f.mean = x->loss_mean;
    return launch_few(f, pairs, st);
  }

  fx::PrepArgs a = prep_args(x, p, w);
  a.loss = x->loss;
  a.lse_out = x->lse;
  a.tlogit = reinterpret_cast<float*>(w + p.tlogit);

  fx::GemmArgs g{};
  if (!encode(&g.a[0], a.Hc, x->d, x->N, p.ldc) || !encode(&g.h, x->H, x->d, x->N, x->ldh) ||
      !encode(&g.b[0], x->W, x->d, x->V, x->ldw))
    return FRAMEFB_ECUDA;
  g.N = static_cast<int32_t>(x->N);
  g.head = a.head;
  g.d = x->d;
  g.V = x->V;
  g.vcols = x->V;
  g.tgt = a.tgt;
  g.npad = p.npad;
  g.part = reinterpret_cast<float2*>(w + p.part);
  g.tlogit = a.tlogit;

  fx::LossArgs l{};
  l.head = a.head;
  l.idx = a.idx;
  l.part = g.part;
  l.tlogit = a.tlogit;
  l.rowloss = reinterpret_cast<float*>(w + p.rowloss);
  l.npad = p.npad;
  l.tiles = (x->V + p.bn / 2 - 1) / (p.bn / 2);
  l.loss = x->loss;
  l.lse = x->lse;
  l.mean = x->loss_mean;

  FFB_TRY(launch_prep(a, st));
  FFB_TRY(launch_logits<fx::STATS>(p.npad / fx::kBM, x->V, p.bn, pairs, g, st));
  return launch(fx::xent_loss_kernel, (x->N + fx::kLossRows - 1) / fx::kLossRows, fx::kLossThreads, 0, l, true, st);
}

extern "C" framefb_status framefb_xent_backward(const framefb_xent* x, framefb_dtype dtype, void* ws, size_t ws_bytes,
                                                void* stream) {
  FFB_TRY(check(x, dtype));
  if (!aligned4({x->lse, x->dloss})) return FRAMEFB_EINVAL;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!std::isfinite(x->scale) || (x->dH && !rows_ok(x->dH, x->lddh, x->d)) || (x->dW && !rows_ok(x->dW, x->lddw, x->d)))
    return FRAMEFB_EINVAL;
  if (x->N == 0) {  // no tokens: dW is 0
    if (x->dW && cudaMemset2DAsync(x->dW, static_cast<size_t>(x->lddw) * 2, 0, static_cast<size_t>(x->d) * 2,
                                   static_cast<size_t>(x->V), st) != cudaSuccess)
      return FRAMEFB_ECUDA;
    return FRAMEFB_OK;
  }
  const int32_t ops = (x->dH ? FRAMEFB_XENT_DH : 0) | (x->dW ? FRAMEFB_XENT_DW : 0);
  if (!ops) return FRAMEFB_OK;
  const int pairs = resident_pairs();
  if (pairs <= 0) return FRAMEFB_ECUDA;
  const Plan p = plan_of(x->N, x->d, x->V, ops, pairs);
  FFB_TRY(check_ws(p, ws, ws_bytes));
  char* w = static_cast<char*>(ws);

  fx::PrepArgs a = prep_args(x, p, w);
  a.scale = x->scale;
  a.lse_in = x->lse;
  a.dloss = x->dloss;
  a.dH = static_cast<__nv_bfloat16*>(x->dH);
  a.lddh = x->lddh;
  a.coef = reinterpret_cast<float*>(w + p.coef);
  a.lse = reinterpret_cast<float*>(w + p.lse);

  fx::GemmArgs g{};
  g.N = static_cast<int32_t>(x->N);
  g.head = a.head;
  g.d = x->d;
  g.V = x->V;
  g.dh = x->dH != nullptr;
  g.dw = x->dW != nullptr;
  const auto on32 = [](const void* q, int64_t ld) { return !q || (reinterpret_cast<uintptr_t>(q) % 32 == 0 && ld % 16 == 0); };
  g.sectors = on32(x->dH, x->lddh) && on32(x->dW, x->lddw);
  g.idx = a.idx;
  g.tgt = a.tgt;
  g.coef = a.coef;
  g.lse = a.lse;
  g.npad = p.npad;
  g.P = reinterpret_cast<__nv_bfloat16*>(w + p.P);
  g.ldp = p.parts * p.vp;
  g.parts = p.parts;
  g.vp = static_cast<int32_t>(p.vp);
  g.acc = reinterpret_cast<float*>(w + p.acc);
  g.slots = reinterpret_cast<float*>(w + p.slots);
  g.dH = a.dH;
  g.lddh = x->lddh;
  g.dW = static_cast<__nv_bfloat16*>(x->dW);
  g.lddw = x->lddw;
  CUtensorMap hc, wm, pm;
  if (!encode(&hc, a.Hc, x->d, x->N, p.ldc) || !encode(&g.h, x->H, x->d, x->N, x->ldh) || !encode(&wm, x->W, x->d, x->V, x->ldw) ||
      !encode(&pm, g.P, g.ldp, p.npad, g.ldp))
    return FRAMEFB_ECUDA;

  FFB_TRY(launch_prep(a, st));
  const int64_t mt = p.npad / fx::kBM, vt = p.vp / fx::kBM;  // all pieces are cut alike
  const int64_t kd = (x->d + fx::kBK - 1) / fx::kBK, kw = g.dw ? (x->N + fx::kBK - 1) / fx::kBK : INT32_MAX;
  const int bnl = tile_columns(mt, p.vp, kd, pairs);
  const int bn = tile_columns((g.dh ? mt : 0) + (g.dw ? vt : 0), x->d, std::min(kw, p.vp / fx::kBK), pairs);
  for (int64_t v0 = 0; v0 < x->V; v0 += p.vp) {
    g.v0 = static_cast<int32_t>(v0);
    g.vcols = static_cast<int32_t>(std::min<int64_t>(p.vp, x->V - v0));
    g.first = v0 == 0;
    g.last = v0 + p.vp >= x->V;
    g.a[0] = hc;
    g.b[0] = wm;
    FFB_TRY(launch_logits<fx::PROB>(mt, g.vcols, bnl, pairs, g, st));
    g.a[0] = g.a[1] = pm;
    g.b[1] = hc;
    FFB_TRY(bn > fx::kBN    ? launch_grads<fx::kMaxBN>(mt, p.join, pairs, g, st)
            : bn == fx::kBN ? launch_grads<fx::kBN>(mt, p.join, pairs, g, st)
                            : launch_grads<fx::kBN / 2>(mt, p.join, pairs, g, st));
  }
  return FRAMEFB_OK;
}

namespace ffb_host {

framefb_status xent_wait_timeouts(uint32_t* count) {
  if (cudaMemcpyFromSymbol(count, fx::g_xent_timeouts, sizeof(uint32_t)) != cudaSuccess) return FRAMEFB_ECUDA;
  return FRAMEFB_OK;
}

}  // namespace ffb_host
