// Entry points of dropout and layer norm: checks, launch shapes, launches
// (kernels in framefb_norm.cuh).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "framefb.h"
#include "framefb_norm.cuh"
#include "framefb_smem.h"

namespace {

namespace fn = ffb::norm;

constexpr int32_t kMaxNormDim = 16384;  // 1024 threads x 16 columns in registers

int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 0;
  return sms;
}

// Drop parameters -> kernel form; false for p outside [0, 1) or rows that the
// generator's 32-bit row counter cannot number.
bool drop_of(const framefb_dropout_params* p, int64_t N, ffb::DropK& k) {
  k = ffb::DropK{};
  k.scale = 1.f;
  if (!p) return true;
  const double q = p->p;
  if (!(q >= 0.0 && q < 1.0)) return false;
  if (N > (int64_t{1} << 32)) return false;
  ffb::set_keys(k, p->seed);
  k.o0 = static_cast<uint32_t>(p->offset);
  k.o1 = static_cast<uint32_t>(p->offset >> 32);
  k.thr = static_cast<uint32_t>(std::floor(q * 4294967296.0));
  k.scale = static_cast<float>(1.0 / (1.0 - q));
  return true;
}

// One array of rows: non-null, aligned to its element, ld >= d; `vec` is
// cleared when its rows do not all start on 16 bytes.
struct Rows {
  const void* p;
  int64_t ld;
};

bool check_rows(std::initializer_list<Rows> rows, int64_t N, int32_t d, int esz, bool& vec) {
  for (const Rows& r : rows) {
    if (!r.p) continue;
    if (r.ld < d || reinterpret_cast<uintptr_t>(r.p) % esz) return false;
    if (r.ld > INT64_MAX / esz / std::max<int64_t>(N, 1)) return false;  // the array's bytes fit 63 bits
    vec = vec && reinterpret_cast<uintptr_t>(r.p) % 16 == 0 && (r.ld * esz) % 16 == 0;
  }
  return true;
}

bool check_f32(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (reinterpret_cast<uintptr_t>(p) % 4) return false;
  return true;
}

// Launch shape of the norm kernels: threads per row, vectors per thread,
// groups (rows at work) per block.  The vectors per thread (forward: at most
// 32 columns, gradient, which keeps column sums too: 24 bf16 or 16 fp32) that
// leave the fewest lanes of the row's last warp empty, more of them where it
// is even.  Up to two rows an SM: one vector a thread where that takes at most
// 512 threads, which has a row done soonest (one row of 4096 with a residual:
// 4.6 -> 3.1 us).  Blocks have about 512 threads (384 with over 16 columns a
// thread: more registers).
struct Shape {
  int threads, nv, groups;
  bool wide() const { return threads > 512; }
};

Shape shape_of(int64_t N, int32_t d, int E, int sms, bool full, bool grad) {
  const int nvec = full ? d / E : (d + 127) / 128 * 32, most = !full ? 4 : grad ? (E == 8 ? 3 : 4) : 32 / E;
  Shape s{0, 0, 0};
  double best = 0;
  for (int nv = 1; nv <= most; ++nv) {
    if ((!full && nv != 1 && nv != most) || (nv > 4 && nv != most)) continue;  // the kernels there are
    const int threads = ((nvec + nv - 1) / nv + 31) / 32 * 32;
    const bool wide_ok = nv == 16 / E;  // the only variant of over 512 threads
    if (threads > 1024 || (threads > 512 && !wide_ok) || (threads > 384 && nv * E > 16)) continue;
    const bool few = N <= 2 * sms && nv == 1;
    const double score = few ? 2 : static_cast<double>(nvec) / (nv * threads) * (1 + 0.1 * nv);
    if (score > best) {
      best = score;
      s.threads = threads;
      s.nv = nv;
    }
  }
  // few rows: fewer groups to a block, so that every SM gets some
  const int64_t per_sm = (N + sms - 1) / sms, block = s.nv * E > 16 ? 384 : 512;
  const int64_t room = s.threads == 32 ? fn::kMaxGroups : fn::kMaxGroups - 1;
  s.groups = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({block / s.threads, room, per_sm})));
  return s;
}

using KernelFn = const void*;

template <typename T, bool FULL, bool DROP, bool RES>
KernelFn norm_fn(const Shape& s) {
  constexpr int W = 16 / fn::Deal<T, FULL>::E;
  if (s.wide()) return reinterpret_cast<KernelFn>(fn::norm_kernel<T, FULL, DROP, RES, W, 1024, 1>);
  if (s.nv == 1) return reinterpret_cast<KernelFn>(fn::norm_kernel<T, FULL, DROP, RES, 1, 512, 2>);
  if (s.nv == W) return reinterpret_cast<KernelFn>(fn::norm_kernel<T, FULL, DROP, RES, W, 512, 2>);
  if constexpr (FULL) {
    if constexpr (W == 4) {
      if (s.nv == 2) return reinterpret_cast<KernelFn>(fn::norm_kernel<T, FULL, DROP, RES, 2, 512, 2>);
      if (s.nv == 3) return reinterpret_cast<KernelFn>(fn::norm_kernel<T, FULL, DROP, RES, 3, 512, 2>);
      return reinterpret_cast<KernelFn>(fn::norm_kernel<T, FULL, DROP, RES, 8, 384, 2>);
    } else {
      if (s.nv == 3) return reinterpret_cast<KernelFn>(fn::norm_kernel<T, FULL, DROP, RES, 3, 384, 2>);
      return reinterpret_cast<KernelFn>(fn::norm_kernel<T, FULL, DROP, RES, 4, 384, 2>);
    }
  }
  return nullptr;
}

template <typename T, bool FULL, bool DROP>
KernelFn norm_grad_fn(const Shape& s) {
  constexpr int W = 16 / fn::Deal<T, FULL>::E;
  if (s.wide()) return reinterpret_cast<KernelFn>(fn::norm_grad_kernel<T, FULL, DROP, W, 1024, true>);
  if (s.nv == 1) return reinterpret_cast<KernelFn>(fn::norm_grad_kernel<T, FULL, DROP, 1, 512, false>);
  if (s.nv == W) return reinterpret_cast<KernelFn>(fn::norm_grad_kernel<T, FULL, DROP, W, 512, false>);
  if constexpr (FULL) {
    if constexpr (W == 4) {
      if (s.nv == 2) return reinterpret_cast<KernelFn>(fn::norm_grad_kernel<T, FULL, DROP, 2, 512, false>);
      return reinterpret_cast<KernelFn>(fn::norm_grad_kernel<T, FULL, DROP, 3, 512, false>);
    } else {
      return reinterpret_cast<KernelFn>(fn::norm_grad_kernel<T, FULL, DROP, 3, 384, false>);
    }
  }
  return nullptr;
}

template <typename T>
KernelFn pick_norm(bool full, bool drop, bool res, const Shape& s) {
  if (!full) return norm_fn<T, false, false, false>(s);
  if (drop) return res ? norm_fn<T, true, true, true>(s) : norm_fn<T, true, true, false>(s);
  return res ? norm_fn<T, true, false, true>(s) : norm_fn<T, true, false, false>(s);
}

template <typename T>
KernelFn pick_grad(bool full, bool drop, const Shape& s) {
  if (!full) return norm_grad_fn<T, false, false>(s);
  return drop ? norm_grad_fn<T, true, true>(s) : norm_grad_fn<T, true, false>(s);
}

// Bytes of the 16-byte pieces that cover a row wherever it starts.
int32_t piece_bytes(int32_t d, int esz) { return static_cast<int32_t>((static_cast<int64_t>(d) * esz + 30) / 16 * 16); }

// Rows of the ring: what fits beside `params` bytes, up to 4 (1: the row at work only).
constexpr size_t kSmemPerSm = 210 * 1024;
// The same of each of two forward blocks on an SM: 105 KB, or 101 beside the
// 12 KB that rows off 16 bytes have as static shared memory (with 105 only one
// block fitted and the other half of the grid waited for it).
constexpr size_t kSmUsable = 228 * 1024, kReserved = 1024;  // of an SM; per block
constexpr size_t room_of_two(bool full) { return (full ? 105 : 101) * 1024; }
static_assert(2 * (room_of_two(true) + fn::norm_static(true, 512) + kReserved) <= kSmUsable &&
                  2 * (room_of_two(false) + fn::norm_static(false, 512) + kReserved) <= kSmUsable,
              "two blocks fit an SM");
int stages_of(size_t room, size_t params, size_t stage) {
  if (stage == 0) return 0;
  return static_cast<int>(std::min<size_t>(fn::kMaxStages, std::max<size_t>(1, (room - params) / stage)));
}

// Runs of 32 vectors in a row: norm_colsum_kernel's blocks along it.
int64_t slabs_of(int32_t d, int E, bool full) { return full ? (d / E + 31) / 32 : (d + 127) / 128; }

// Blocks of the gradient: one per SM, as each leaves 8 d bytes of column sums.
int64_t grad_blocks(int64_t N, const Shape& s, int sms) {
  return std::min<int64_t>((N + s.groups - 1) / s.groups, sms);
}

// Rows of column sums that the gradient leaves: one per block, or (wide rows)
// as many as give norm_colsum_kernel four blocks an SM.
int64_t sum_rows(int64_t N, int32_t d, int E, bool full, const Shape& s, int sms) {
  if (!s.wide()) return grad_blocks(N, s, sms);
  return std::min<int64_t>((N + fn::kSumWarps - 1) / fn::kSumWarps, (4 * sms + slabs_of(d, E, full) - 1) / slabs_of(d, E, full));
}

bool dtype_ok(framefb_dtype dt) { return dt == FRAMEFB_F32 || dt == FRAMEFB_BF16; }

// `chained`: the kernel may start while the one before it ends (programmatic
// dependent launch; it waits by itself).
framefb_status launch(KernelFn f, dim3 blocks, int threads, size_t smem, void* args, bool chained, void* stream) {
  void* kargs[] = {args};
  if (smem > 24 * 1024) {  // with the kernels' static 24 KB over what needs no opt-in
    const framefb_status st = ffb_host::allow_smem(f, smem);
    if (st != FRAMEFB_OK) return st;
  }
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = blocks;
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cfg.attrs = &attr;
  cfg.numAttrs = chained ? 1 : 0;
  return cudaLaunchKernelExC(&cfg, f, kargs) == cudaSuccess ? FRAMEFB_OK : FRAMEFB_ECUDA;
}

dim3 grid(int64_t x, int64_t y = 1) { return dim3(static_cast<unsigned>(x), static_cast<unsigned>(y)); }

}  // namespace

extern "C" framefb_status framefb_dropout(const void* X, int64_t ldx, const void* R, int64_t ldr, void* Y, int64_t ldy,
                                          int64_t N, int32_t d, framefb_dtype dtype,
                                          const framefb_dropout_params* drop, void* stream) {
  fn::DropArgs a{};
  if (!dtype_ok(dtype) || N < 0 || d < 1 || !drop || !drop_of(drop, N, a.k)) return FRAMEFB_EINVAL;
  if (N == 0) return FRAMEFB_OK;
  const int esz = dtype == FRAMEFB_F32 ? 4 : 2, E = 16 / esz;
  bool vec = true;
  if (!X || !Y || !check_rows({{X, ldx}, {R, ldr}, {Y, ldy}}, N, d, esz, vec)) return FRAMEFB_EINVAL;
  a.X = X;
  a.R = R;
  a.Y = Y;
  a.ldx = ldx;
  a.ldr = ldr;
  a.ldy = ldy;
  a.d = d;
  const bool full = vec && d % E == 0;
  const int64_t vpr = full ? d / E : (static_cast<int64_t>(d) + 127) / 128 * 32;  // as Deal
  a.vpr = static_cast<int32_t>(vpr);
  a.total = N * a.vpr;
  a.drow = fn::kDropThreads / a.vpr;
  a.dvec = fn::kDropThreads % a.vpr;
  const int64_t per = fn::kDropThreads * fn::kDropUnroll;
  const int64_t blocks = (a.total + per - 1) / per;
  if (blocks > INT32_MAX) return FRAMEFB_EINVAL;
  KernelFn f = dtype == FRAMEFB_F32 ? (full ? reinterpret_cast<KernelFn>(fn::dropout_kernel<float, true>)
                                            : reinterpret_cast<KernelFn>(fn::dropout_kernel<float, false>))
                                    : (full ? reinterpret_cast<KernelFn>(fn::dropout_kernel<__nv_bfloat16, true>)
                                            : reinterpret_cast<KernelFn>(fn::dropout_kernel<__nv_bfloat16, false>));
  return launch(f, grid(blocks), fn::kDropThreads, 0, &a, false, stream);
}

extern "C" framefb_status framefb_layernorm_forward(const framefb_norm* n, framefb_dtype dtype, void* stream) {
  fn::NormArgs a{};
  if (!n || !dtype_ok(dtype) || n->N < 0 || n->d < 1 || !(n->eps >= 0.f) || !std::isfinite(n->eps) ||
      !drop_of(n->drop, n->N, a.k))
    return FRAMEFB_EINVAL;
  if (n->d > kMaxNormDim) return FRAMEFB_EUNSUPPORTED;
  if (n->N == 0) return FRAMEFB_OK;
  const int esz = dtype == FRAMEFB_F32 ? 4 : 2;
  bool vec = true;
  if (!n->X || !n->Y ||
      !check_rows({{n->X, n->ldx}, {n->R, n->ldr}, {n->Z, n->ldz}, {n->Y, n->ldy}}, n->N, n->d, esz, vec) ||
      !check_f32({n->gamma, n->beta, n->mean, n->rstd}))
    return FRAMEFB_EINVAL;
  const int sms = sm_count();
  if (sms <= 0) return FRAMEFB_ECUDA;
  a.N = n->N;
  a.d = n->d;
  a.eps = n->eps;
  a.inv_d = 1.f / static_cast<float>(n->d);
  a.X = n->X;
  a.R = n->R;
  a.Z = n->Z;
  a.Y = n->Y;
  a.ldx = n->ldx;
  a.ldr = n->ldr;
  a.ldz = n->ldz;
  a.ldy = n->ldy;
  a.gamma = n->gamma;
  a.beta = n->beta;
  a.mean = n->mean;
  a.rstd = n->rstd;
  const bool full = vec && n->d % (16 / esz) == 0, drop = a.k.thr != 0, res = n->R != nullptr;
  const int E = full ? 16 / esz : 4;
  const Shape s = shape_of(n->N, n->d, E, sms, full, false);
  a.groups = s.groups;
  KernelFn f = dtype == FRAMEFB_F32 ? pick_norm<float>(full, drop, res, s) : pick_norm<__nv_bfloat16>(full, drop, res, s);
  const size_t params = s.nv > 1 ? static_cast<size_t>(8) * s.nv * s.threads * E : 0;  // gamma, beta
  // the ring: vectors of every thread, or the pieces of whole rows; as in the kernel
  const bool ring = full && !(s.wide() && dtype == FRAMEFB_F32 && res);
  a.stage_bytes = piece_bytes(n->d, esz);
  const size_t stage = ring                ? static_cast<size_t>(16) * (res ? 2 : 1) * s.nv * s.threads * s.groups
                       : !full && !s.wide() ? static_cast<size_t>(a.stage_bytes) * (res ? 2 : 1) * s.groups
                                            : 0;
  // two blocks on an SM where their parameters and two rows of the ring fit
  const int per_sm = !s.wide() && params + 2 * stage <= room_of_two(full) ? 2 : 1;
  a.stages = stages_of(per_sm == 2 ? room_of_two(full) : kSmemPerSm, params, stage);
  const int64_t blocks = std::min<int64_t>((n->N + s.groups - 1) / s.groups, static_cast<int64_t>(sms) * per_sm);
  return launch(f, grid(blocks), s.threads * s.groups, params + a.stages * stage, &a, false, stream);
}

extern "C" size_t framefb_layernorm_workspace_size(int64_t N, int32_t d) {
  const int sms = sm_count();
  if (N <= 0 || d < 1 || d > kMaxNormDim || sms <= 0) return 0;
  int64_t rows = sum_rows(N, d, 4, false, shape_of(N, d, 4, sms, false, true), sms);
  for (const int E : {4, 8})
    if (d % E == 0) rows = std::max(rows, sum_rows(N, d, E, true, shape_of(N, d, E, sms, true, true), sms));
  return static_cast<size_t>(rows) * 2 * static_cast<size_t>(d) * sizeof(float);
}

extern "C" framefb_status framefb_layernorm_backward(const framefb_norm* n, framefb_dtype dtype, void* ws,
                                                     size_t ws_bytes, void* stream) {
  fn::NormGradArgs a{};
  if (!n || !dtype_ok(dtype) || n->N < 0 || n->d < 1 || !drop_of(n->drop, n->N, a.k)) return FRAMEFB_EINVAL;
  if (n->d > kMaxNormDim) return FRAMEFB_EUNSUPPORTED;
  if (!check_f32({n->gamma, n->mean, n->rstd, n->dgamma, n->dbeta})) return FRAMEFB_EINVAL;
  const int esz = dtype == FRAMEFB_F32 ? 4 : 2;
  const bool sums = n->dgamma || n->dbeta;
  bool vec = true;
  if (n->N > 0 && (!n->dY || !n->Z || !n->mean || !n->rstd ||
                   !check_rows({{n->dY, n->lddy}, {n->Z, n->ldz}, {n->dZin, n->lddzin}, {n->dZ, n->lddz}, {n->dX, n->lddx}},
                               n->N, n->d, esz, vec)))
    return FRAMEFB_EINVAL;
  const int sms = sm_count();
  if (sms <= 0) return FRAMEFB_ECUDA;
  const size_t need = sums ? framefb_layernorm_workspace_size(n->N, n->d) : 0;
  if (need > 0 && (!ws || ws_bytes < need)) return FRAMEFB_EWORKSPACE;
  if (need > 0 && reinterpret_cast<uintptr_t>(ws) % 256) return FRAMEFB_EINVAL;
  const bool full = vec && n->d % (16 / esz) == 0;
  const int E = full ? 16 / esz : 4;
  const Shape s = shape_of(n->N, n->d, E, sms, full, true);
  const int64_t blocks = n->N > 0 ? grad_blocks(n->N, s, sms) : 0;
  const int64_t rows = n->N > 0 ? sum_rows(n->N, n->d, E, full, s, sms) : 0;
  if (blocks > 0) {
    a.N = n->N;
    a.d = n->d;
    a.inv_d = 1.f / static_cast<float>(n->d);
    a.dY = n->dY;
    a.Z = n->Z;
    a.dZin = n->dZin;
    a.dZ = n->dZ;
    a.dX = n->dX;
    a.lddy = n->lddy;
    a.ldz = n->ldz;
    a.lddzin = n->lddzin;
    a.lddz = n->lddz;
    a.lddx = n->lddx;
    a.gamma = n->gamma;
    a.mean = n->mean;
    a.rstd = n->rstd;
    a.part = sums ? static_cast<float*>(ws) : nullptr;
    a.groups = s.groups;
    const bool drop = a.dX && a.k.thr != 0;
    KernelFn f = dtype == FRAMEFB_F32 ? pick_grad<float>(full, drop, s) : pick_grad<__nv_bfloat16>(full, drop, s);
    // gamma, then the ring and in its place the column sums of the groups
    const size_t row = static_cast<size_t>(4) * s.nv * s.threads * E, params = s.nv > 1 ? row : 0;
    const bool ring = full && !(s.wide() && dtype == FRAMEFB_F32);  // as in the kernel
    a.stage_bytes = piece_bytes(n->d, esz);
    const size_t stage = ring                ? static_cast<size_t>(n->dZin ? 48 : 32) * s.nv * s.threads * s.groups
                         : !full && !s.wide() ? static_cast<size_t>(a.stage_bytes) * (n->dZin ? 3 : 2) * s.groups
                                              : 0;
    a.stages = stages_of(kSmemPerSm, params, stage);
    const size_t smem = params + std::max(a.stages * stage, s.wide() ? 0 : 2 * row * s.groups);
    if (s.wide() && sums) {  // before the gradient, whose outputs may lie over its inputs
      KernelFn g = dtype == FRAMEFB_F32 ? (full ? reinterpret_cast<KernelFn>(fn::norm_colsum_kernel<float, true>)
                                                : reinterpret_cast<KernelFn>(fn::norm_colsum_kernel<float, false>))
                                        : (full ? reinterpret_cast<KernelFn>(fn::norm_colsum_kernel<__nv_bfloat16, true>)
                                                : reinterpret_cast<KernelFn>(fn::norm_colsum_kernel<__nv_bfloat16, false>));
      const framefb_status st = launch(g, grid(slabs_of(n->d, E, full), rows), 32 * fn::kSumWarps, 0, &a, false, stream);
      if (st != FRAMEFB_OK) return st;
    }
    const framefb_status st = launch(f, grid(blocks), s.threads * s.groups, smem, &a, false, stream);
    if (st != FRAMEFB_OK) return st;
  }
  if (!sums) return FRAMEFB_OK;
  fn::NormColsArgs c{};
  c.part = static_cast<const float*>(ws);
  c.dgamma = n->dgamma;
  c.dbeta = n->dbeta;
  c.blocks = static_cast<int32_t>(rows);  // no rows: the sums are 0
  c.d = n->d;
  return launch(reinterpret_cast<KernelFn>(fn::norm_cols_kernel), grid((2 * static_cast<int64_t>(n->d) + 31) / 32),
                32 * fn::kColRows, 0, &c, rows > 0, stream);
}
