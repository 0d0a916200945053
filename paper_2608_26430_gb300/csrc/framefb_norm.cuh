// Dropout and layer norm of libframefb (bf16 or fp32 rows, fp32 arithmetic).
//
//   dropout            Y = [R +] drop(X)
//   layer norm         Z = [R +] drop(X);  mu = mean(Z), rstd = (var(Z) + eps)^-1/2
//                      Y = (Z - mu) rstd gamma + beta
//   its gradient       xh = (Z - mu) rstd, a = dY gamma
//                      dZ = rstd (a - mean(a) - xh mean(a xh)) [+ dZin];  dX = drop(dZ)
//                      dgamma = sum_t dY xh,  dbeta = sum_t dY
//
// All three read every input once and write every output once, but for the
// column sums of wide rows, which are a second reading of dY and Z.
// Included by framefb_norm.cu only.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "framefb_dropout.cuh"
#include "framefb_ptx.cuh"

namespace ffb {
namespace norm {

// How a row of d columns is dealt out in vectors of E columns; thread t of a
// group has vectors t, t + T, ...
//   FULL   every row starts on 16 bytes and d is a multiple of E: a vector is
//          16 bytes in one access.
//   not    E = 4 columns, 32 apart: a warp's vectors are 128 columns, and each
//          of its accesses is 32 neighbours, whatever the alignment.  (Four or
//          eight neighbours a thread, one access each, take four times the
//          passes through L1: 8191 x 4095 bf16 dropout 86 us.)
template <typename T, bool FULL>
struct Deal {
  static constexpr int E = FULL ? 16 / static_cast<int>(sizeof(T)) : 4;
  static constexpr int STEP = FULL ? 1 : 32;  // columns from one element of a vector to the next
  __device__ __forceinline__ static int col(int v) { return FULL ? v * E : (v >> 5) * 128 + (v & 31); }
  // Elements of vector v that are inside the row: the first cnt of them.
  __device__ __forceinline__ static int cnt(int c, int d) {
    return max(0, min(E, FULL ? d - c : (d - c + 31) >> 5));
  }
};

// A vector as it stands in memory, zeros for what is past the row (FULL: all
// of it or nothing; otherwise one element per word).
template <typename T, bool FULL>
__device__ __forceinline__ uint4 load_raw(const T* row, int col, int cnt) {
  if constexpr (FULL) {
    return cnt ? *reinterpret_cast<const uint4*>(row + col) : make_uint4(0, 0, 0, 0);
  } else {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < cnt) {
        if constexpr (sizeof(T) == 4)
          w[e] = reinterpret_cast<const uint32_t*>(row + col)[32 * e];
        else
          w[e] = reinterpret_cast<const uint16_t*>(row + col)[32 * e];
      }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// As fp32 pairs.
template <typename T, bool FULL, int P>
__device__ __forceinline__ void unpack(const uint4& u, float2 (&f)[P]) {
  if constexpr (sizeof(T) == 4) {
    f[0] = make_float2(__uint_as_float(u.x), __uint_as_float(u.y));
    f[1] = make_float2(__uint_as_float(u.z), __uint_as_float(u.w));
  } else if constexpr (FULL) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
  } else {
    f[0] = make_float2(__uint_as_float(u.x << 16), __uint_as_float(u.y << 16));
    f[1] = make_float2(__uint_as_float(u.z << 16), __uint_as_float(u.w << 16));
  }
}

template <typename T, bool FULL, int P>
__device__ __forceinline__ void store_vec(T* row, int col, int cnt, const float2 (&f)[P]) {
  if constexpr (FULL) {
    if (!cnt) return;
    uint4 u;
    if constexpr (P == 2)
      u = make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
    else
      u = make_uint4(pack_bf16(f[0].x, f[0].y), pack_bf16(f[1].x, f[1].y), pack_bf16(f[2].x, f[2].y), pack_bf16(f[3].x, f[3].y));
    *reinterpret_cast<uint4*>(row + col) = u;
  } else {
    const float g[4] = {f[0].x, f[0].y, f[1].x, f[1].y};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < cnt) {
        if constexpr (sizeof(T) == 4)
          row[col + 32 * e] = g[e];
        else
          row[col + 32 * e] = __float2bfloat16_rn(g[e]);
      }
  }
}

__device__ __forceinline__ float keep(uint32_t w, float x, const DropK& k) { return w >= k.thr ? x * k.scale : 0.f; }

// Dropout of one vector.  FULL: the vector's own counters.  Otherwise the
// warp's lanes draw the 128 columns' words, four neighbours each, and pass
// them on through `mix` (this warp's 128 words; all of its lanes are here).
template <bool FULL, int P>
__device__ __forceinline__ void drop_vec(float2 (&x)[P], const DropK& k, uint32_t row, int col, uint4* mix) {
  if constexpr (FULL) {
#pragma unroll
    for (int b = 0; b < P / 2; ++b) {
      const uint4 w = philox4x32((static_cast<uint32_t>(col) >> 2) + b, row, k);
      x[2 * b] = make_float2(keep(w.x, x[2 * b].x, k), keep(w.y, x[2 * b].y, k));
      x[2 * b + 1] = make_float2(keep(w.z, x[2 * b + 1].x, k), keep(w.w, x[2 * b + 1].y, k));
    }
  } else {
    const int lane = threadIdx.x & 31;
    mix[lane] = philox4x32(((static_cast<uint32_t>(col) & ~127u) >> 2) + lane, row, k);
    __syncwarp();
    const uint32_t* w = reinterpret_cast<const uint32_t*>(mix) + lane;
    x[0] = make_float2(keep(w[0], x[0].x, k), keep(w[32], x[0].y, k));
    x[1] = make_float2(keep(w[64], x[1].x, k), keep(w[96], x[1].y, k));
    __syncwarp();
  }
}

// ---------------------------------------------------------------------------
// Dropout: one vector of a row per thread and step, kDropUnroll of them in
// flight (four, with fewer warps on an SM: 35 us instead of 32 below).  Bound
// by HBM, 2 (3 with R) passes over the array, where an element has 4 bytes:
// 8192 x 4096 fp32 with R 57 us, 7.0 TB/s.  bf16 has half the bytes to the same
// instructions: of some 187 per 8 columns the generator's rounds are 80 (20 wide
// multiplications and 20 xors per 4 columns), addresses, selections, scaling
// and packing the rest.  No pipe is full (integer multipliers 65 % busy, ALUs
// 52 %, 2.6 instructions a cycle): 8192 x 4096 32 us, 4.2 TB/s.
// ---------------------------------------------------------------------------
constexpr int kDropThreads = 256;
constexpr int kDropUnroll = 2;

struct DropArgs {
  const void* X;
  const void* R;
  void* Y;
  int64_t ldx, ldr, ldy;
  int64_t total;        // vectors: N * vpr
  int32_t d, vpr;       // columns and vectors per row (not FULL: whole warps of them)
  int32_t drow, dvec;   // kDropThreads vectors on: so many rows and vectors
  DropK k;
};

template <typename T, bool FULL>
__global__ void __launch_bounds__(kDropThreads, 6) dropout_kernel(const DropArgs a) {
  using D = Deal<T, FULL>;
  constexpr int P = D::E / 2;
  __shared__ uint4 mix[FULL ? 1 : kDropThreads / 32][32];
  const int64_t i0 = static_cast<int64_t>(blockIdx.x) * (kDropThreads * kDropUnroll) + threadIdx.x;
  int64_t row[kDropUnroll];
  int col[kDropUnroll], cnt[kDropUnroll];
  // one division a thread, a 32-bit one where the count allows
  int64_t r0 = a.total <= INT32_MAX ? static_cast<int64_t>(static_cast<uint32_t>(i0) / static_cast<uint32_t>(a.vpr)) : i0 / a.vpr;
  int32_t v = static_cast<int32_t>(i0 - r0 * a.vpr);
  uint4 x[kDropUnroll], r[kDropUnroll];
#pragma unroll
  for (int u = 0; u < kDropUnroll; ++u) {
    row[u] = r0;
    col[u] = D::col(v);
    cnt[u] = i0 + u * kDropThreads < a.total ? D::cnt(col[u], a.d) : 0;
    x[u] = load_raw<T, FULL>(static_cast<const T*>(a.X) + row[u] * a.ldx, col[u], cnt[u]);
    if (a.R) r[u] = load_raw<T, FULL>(static_cast<const T*>(a.R) + row[u] * a.ldr, col[u], cnt[u]);
    r0 += a.drow;
    v += a.dvec;
    if (v >= a.vpr) {
      v -= a.vpr;
      ++r0;
    }
  }
#pragma unroll
  for (int u = 0; u < kDropUnroll; ++u) {
    float2 f[P];
    unpack<T, FULL>(x[u], f);
    if (a.k.thr) drop_vec<FULL>(f, a.k, static_cast<uint32_t>(row[u]), col[u], mix[FULL ? 0 : threadIdx.x >> 5]);
    if (a.R) {
      float2 g[P];
      unpack<T, FULL>(r[u], g);
#pragma unroll
      for (int e = 0; e < P; ++e) f[e] = make_float2(f[e].x + g[e].x, f[e].y + g[e].y);
    }
    store_vec<T, FULL>(static_cast<T*>(a.Y) + row[u] * a.ldy, col[u], cnt[u], f);
  }
}

// ---------------------------------------------------------------------------
// Layer norm.  A block is `groups` groups of T = blockDim.x / groups threads
// (whole warps); a group takes one row at a time and its threads hold vectors
// t, t + T, ... (NV of them) of the row in registers, so a row is read once
// and its mean and the sum of squared deviations from that mean are fp32 sums
// over registers, one after the other (no cancellation).  Groups wait for
// nobody else (a named barrier each).  The rows a group takes next are on
// their way while it works on one: without that, loads, reductions and stores
// take turns (16384 x 4096 bf16 gradient: 245 us instead of 90).  Whole vectors come
// through a ring in shared memory of `stages` rows per group, by asynchronous
// copies that each thread issues and waits for itself (what it copies only it
// reads, so the ring needs no barrier); other rows as the 16-byte pieces that
// cover them, with a barrier of the group per row (5000 x 6001 bf16 gradient
// one row ahead in registers: 219 us instead of 66).  A warp's shuffles,
// barrier and square root cost some 200 instructions a row, as many as the
// arithmetic of 40 columns a lane, so a thread takes 16 to 32 columns where
// the row allows it (16384 x 4096 bf16 forward with 8: 89 us instead of 46).
// gamma and beta wait in shared memory, as float4 planes that a warp reads
// without conflicts (one vector a thread: in registers).
// Bound by HBM: forward 46 us, 5.8 TB/s at 16384 x 4096 bf16; gradient with
// dZin 90 us, 6.0 TB/s; 8000 x 2047 fp32 gradient 41 us, 4.8 TB/s.  Short
// calls are launch and latency: 3.1 us for one row of 4096.
// ---------------------------------------------------------------------------
struct NormArgs {
  int64_t N;
  int32_t d;
  float eps, inv_d;
  const void* X;
  const void* R;
  void* Z;
  void* Y;
  int64_t ldx, ldr, ldz, ldy;
  const float* gamma;
  const float* beta;
  float* mean;
  float* rstd;
  int32_t groups, stages, stage_bytes;
  DropK k;
};

struct NormGradArgs {
  int64_t N;
  int32_t d;
  float inv_d;
  const void* dY;
  const void* Z;
  const void* dZin;
  void* dZ;
  void* dX;
  int64_t lddy, ldz, lddzin, lddz, lddx;
  const float* gamma;
  const float* mean;
  const float* rstd;
  float* part;  // [blocks][2][d] column sums (dgamma, dbeta), or NULL
  int32_t groups, stages, stage_bytes;
  DropK k;
};

// A thread's place: its group, its warps' partners in sums over the group.
struct Place {
  int T, group, tid, half;  // half: half the smallest power of two >= warps of the group
  __device__ __forceinline__ explicit Place(int groups) {
    T = blockDim.x / groups;
    group = threadIdx.x / T;
    tid = threadIdx.x - group * T;
    half = 1;
    while (2 * half < T >> 5) half <<= 1;
  }
};

// Sums of K values over a group of T threads; every thread gets them.  `sh`
// holds 32 * K floats; calls that share it are separated by a barrier of the
// group.
template <int K>
__device__ __forceinline__ void group_sum(float (&v)[K], float* sh, const Place& p) {
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  if (p.T == 32) return;
  const int nw = p.T >> 5, lane = p.tid & 31, from = lane & (2 * p.half - 1);
  if (lane == 0) {
#pragma unroll
    for (int k = 0; k < K; ++k) sh[k * 32 + (p.tid >> 5)] = v[k];
  }
  asm volatile("bar.sync %0, %1;" ::"r"(p.group + 1), "r"(p.T) : "memory");
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = from < nw ? sh[k * 32 + from] : 0.f;
  for (int o = p.half; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
}

// gamma or beta in shared memory, filled by the whole block for nvec vectors:
// FULL, E / 4 planes of one float4 per vector, otherwise column by column.
template <typename T, bool FULL>
__device__ __forceinline__ void fill_param(float4* plane, const float* p, int nvec, int d, float none) {
  constexpr int E = Deal<T, FULL>::E;
  for (int q = threadIdx.x; q < nvec * (E / 4); q += blockDim.x) {
    const int c = FULL ? q % nvec * E + q / nvec * 4 : 4 * q;
    float f[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = p && c + e < d ? __ldg(p + c + e) : none;
    plane[q] = make_float4(f[0], f[1], f[2], f[3]);
  }
}

template <typename T, bool FULL, int P>
__device__ __forceinline__ void read_param(const float4* plane, int nvec, int v, float2 (&f)[P]) {
  if constexpr (FULL) {
#pragma unroll
    for (int q = 0; q < P / 2; ++q) {
      const float4 x = plane[q * nvec + v];
      f[2 * q] = make_float2(x.x, x.y);
      f[2 * q + 1] = make_float2(x.z, x.w);
    }
  } else {
    const float* x = reinterpret_cast<const float*>(plane) + Deal<T, FULL>::col(v);
    f[0] = make_float2(x[0], x[32]);
    f[1] = make_float2(x[64], x[96]);
  }
}

// The same straight from memory (kernels of one vector a thread, which keep
// it in registers: few rows, where filling shared memory would cost more than
// the rows).
template <typename T, bool FULL, int P>
__device__ __forceinline__ void load_param(const float* p, int col, int cnt, float none, float2 (&f)[P]) {
  float g[2 * P];
  if (FULL && p && cnt && reinterpret_cast<uintptr_t>(p) % 16 == 0) {
#pragma unroll
    for (int q = 0; q < P / 2; ++q) {
      const float4 x = __ldg(reinterpret_cast<const float4*>(p + col) + q);
      g[4 * q] = x.x;
      g[4 * q + 1] = x.y;
      g[4 * q + 2] = x.z;
      g[4 * q + 3] = x.w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 2 * P; ++e) g[e] = p && e < cnt ? __ldg(p + col + e * Deal<T, FULL>::STEP) : none;
  }
#pragma unroll
  for (int e = 0; e < P; ++e) f[e] = make_float2(g[2 * e], g[2 * e + 1]);
}

// Two fp32 lanes in one instruction (each rounded as its scalar form).
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 o;
  asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n add.rn.f32x2 z, x, y;\n mov.b64 {%0, %1}, z;\n}"
      : "=f"(o.x), "=f"(o.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return o;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 o;
  asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mul.rn.f32x2 z, x, y;\n mov.b64 {%0, %1}, z;\n}"
      : "=f"(o.x), "=f"(o.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return o;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 o;
  asm("{\n .reg .b64 x, y, z, w;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mov.b64 z, {%6, %7};\n"
      " fma.rn.f32x2 w, x, y, z;\n mov.b64 {%0, %1}, w;\n}"
      : "=f"(o.x), "=f"(o.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return o;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// 1 / sqrt(v): the approximation with one Newton step.
__device__ __forceinline__ float inv_sqrt(float v) {
  const float r = rsqrtf(v);
  return r > 0.f && r < INFINITY ? r * fmaf(-0.5f * v * r, r, 1.5f) : r;
}

constexpr int kMaxGroups = 16;  // named barriers 1 to 15; a group of one warp needs none

// Rows on their way: A arrays (the call uses `used` of them) of NV vectors a
// thread.  RING: `stages` rows deep in shared memory; otherwise the row at
// work in registers.
template <typename T, bool RING, int A, int NV>
struct Rows {
  uint4 reg[RING ? 1 : A][RING ? 1 : NV];
  uint4* ring;     // this thread's slot of (stage 0, array 0, vector 0)
  int32_t pitch;   // threads of the block: from one slot to the next
  int32_t stages, at, used;

  __device__ __forceinline__ uint4* slot(int stage, int arr, int i) { return ring + ((stage * used + arr) * NV + i) * pitch; }

  // Start the row of array `arr` at `row`, which the thread's columns may lie past.
  template <bool FULL>
  __device__ __forceinline__ void start(int stage, int arr, const T* row, const int (&col)[NV], const int (&cnt)[NV]) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if constexpr (RING) {
        if (cnt[i])
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(slot(stage, arr, i))), "l"(row + col[i])
                       : "memory");
      } else {
        reg[arr][i] = load_raw<T, FULL>(row, col[i], cnt[i]);
      }
    }
  }
  __device__ __forceinline__ uint4 get(int arr, int i) {
    if constexpr (RING) return *slot(at, arr, i);
    return reg[arr][i];
  }
  // One row's copies are a group of their own (also when there was no row left to start).
  __device__ __forceinline__ void commit() {
    if constexpr (RING) asm volatile("cp.async.commit_group;" ::: "memory");
  }
  // The oldest row has landed once at most stages - 1 younger ones are pending.
  __device__ __forceinline__ void wait() {
    if constexpr (RING) {
      switch (stages) {
        case 1: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
        case 2: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
        case 3: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
        default: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
      }
    }
  }
  __device__ __forceinline__ int last_stage() const { return at == 0 ? stages - 1 : at - 1; }
  __device__ __forceinline__ void advance() {
    if constexpr (RING) at = at + 1 == stages ? 0 : at + 1;
  }
};

// Rows that do not start on 16 bytes, on their way: a ring of `stages` rows of
// A arrays in shared memory that a group's threads fill and read together.  A
// row comes as the 16-byte pieces that cover it (its neighbours' bytes at both
// ends are read along and not used); pieces that reach past the array's own
// first or last element go element by element.
template <typename T, int A, int NV>
struct Staged {
  uint8_t* base;   // the group's ring
  int32_t bytes;   // of one array's row: its pieces
  int32_t stages, at, used, T_, tid, group;
  uint32_t phase[A];  // of the row at work: where it starts in its first piece

  __device__ __forceinline__ uint8_t* buf(int stage, int arr) { return base + (stage * used + arr) * bytes; }

  __device__ __forceinline__ void start(int stage, int arr, const T* row, const T* lo, const T* hi, int d) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(row), end = a + static_cast<uintptr_t>(d) * sizeof(T);
    const uintptr_t first = a & ~static_cast<uintptr_t>(15);
    const uint32_t dst = smem_u32(buf(stage, arr));
    for (uint32_t o = tid * 16u; first + o < end; o += T_ * 16u) {
      const uintptr_t g = first + o;
      if (g >= reinterpret_cast<uintptr_t>(lo) && g + 16 <= reinterpret_cast<uintptr_t>(hi)) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + o), "l"(g) : "memory");
      } else {
        for (uintptr_t e = max(g, a); e < min(g + 16, end); e += sizeof(T))
          *reinterpret_cast<T*>(buf(stage, arr) + (e - first)) = *reinterpret_cast<const T*>(e);
      }
    }
  }
  __device__ __forceinline__ void sync() {
    if (T_ == 32)
      __syncwarp();
    else
      asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(T_) : "memory");
  }
  __device__ __forceinline__ uint4 get(int arr, int col, int cnt) {
    const uint8_t* p = buf(at, arr) + phase[arr] + static_cast<uint32_t>(col) * sizeof(T);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < cnt) {
        if constexpr (sizeof(T) == 4)
          w[e] = *reinterpret_cast<const uint32_t*>(p + 128 * e);
        else
          w[e] = *reinterpret_cast<const uint16_t*>(p + 64 * e);
      }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  // Row `row` is here and the row before it is done with: `fetch` may start the next one in its place.
  template <typename F>
  __device__ __forceinline__ void turn(F&& fetch) {
    if (stages == 1) {
      sync();
      fetch(0);
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      sync();
      return;
    }
    switch (stages) {
      case 2: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
      case 3: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
      default: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
    }
    sync();
    fetch(at == 0 ? stages - 1 : at - 1);
  }
  __device__ __forceinline__ void advance() { at = at + 1 == stages ? 0 : at + 1; }
};

template <typename T>
__device__ __forceinline__ uint32_t phase_of(const void* base, int64_t row, int64_t ld) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(base) + row * ld * sizeof(T)) & 15u;
}

constexpr int kMaxStages = 4;

// Static shared memory of norm_kernel: the sums' exchange and the masks passed on.
constexpr size_t norm_static(bool full, int maxt) { return kMaxGroups * 2 * 32 * 4 + (full ? 1 : maxt / 32) * 512; }

// Forward.  DROP, RES: whether the call drops and adds (FULL; otherwise both are looked up).
template <typename T, bool FULL, bool DROP, bool RES, int NV, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) norm_kernel(const NormArgs a) {
  using D = Deal<T, FULL>;
  constexpr int E = D::E, P2 = E / 2;
  constexpr int A = FULL && !RES ? 1 : 2;  // X, R
  // wide fp32 rows with a residual: gamma, beta and one row of the ring are more than an SM's shared memory
  constexpr bool RING = FULL && !(MAXT > 512 && sizeof(T) == 4 && RES);
  extern __shared__ float4 dyn[];          // gamma, beta, ring
  __shared__ float sh[kMaxGroups][2][32];
  __shared__ uint4 mix[FULL ? 1 : MAXT / 32][32];
  static_assert(sizeof(sh) + sizeof(mix) == norm_static(FULL, MAXT), "what the launch shapes count with");
  const Place p(a.groups);
  const int nvec = NV * p.T;
  int col[NV], cnt[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    col[i] = D::col(p.tid + i * p.T);
    cnt[i] = D::cnt(col[i], a.d);
  }
  const bool res = FULL ? RES : a.R != nullptr;
  const bool drop = FULL ? DROP : a.k.thr != 0;
  const int64_t step = static_cast<int64_t>(gridDim.x) * a.groups;
  int64_t row = static_cast<int64_t>(blockIdx.x) * a.groups + p.group;
  constexpr bool STAGED = !FULL && MAXT <= 512;
  Rows<T, RING, A, NV> in;
  Staged<T, A, NV> st;
  in.ring = reinterpret_cast<uint4*>(NV > 1 ? dyn + 2 * nvec * (E / 4) : dyn) + threadIdx.x;
  in.pitch = blockDim.x;
  in.stages = a.stages;
  in.at = 0;
  in.used = A;
  if constexpr (STAGED) {
    st.used = res ? 2 : 1;
    st.bytes = a.stage_bytes;
    st.stages = a.stages;
    st.base = reinterpret_cast<uint8_t*>(NV > 1 ? dyn + 2 * nvec * (E / 4) : dyn) + p.group * (a.stages * st.used * st.bytes);
    st.at = 0;
    st.T_ = p.T;
    st.tid = p.tid;
    st.group = p.group;
  }
  // rows move on by `step`: pointers are added up, not multiplied out
  const T* xr = static_cast<const T*>(a.X) + row * a.ldx;
  const T* rr = static_cast<const T*>(a.R) + row * a.ldr;
  const int64_t dxr = step * a.ldx, drr = step * a.ldr;
  int64_t next = row;
  auto fetch = [&](int stage) {
    if (next < a.N) {
      if constexpr (STAGED) {
        st.start(stage, 0, xr, static_cast<const T*>(a.X), static_cast<const T*>(a.X) + ((a.N - 1) * a.ldx + a.d), a.d);
        if (res)
          st.start(stage, 1, rr, static_cast<const T*>(a.R), static_cast<const T*>(a.R) + ((a.N - 1) * a.ldr + a.d), a.d);
      } else {
        in.template start<FULL>(stage, 0, xr, col, cnt);
        if (A == 2 && res) in.template start<FULL>(stage, A - 1, rr, col, cnt);
      }
    }
    if constexpr (STAGED)
      asm volatile("cp.async.commit_group;" ::: "memory");
    else
      in.commit();
    next += step;
    xr += dxr;
    rr += drr;
  };
  const int ahead = RING || STAGED ? a.stages - 1 : 0;
  if constexpr (RING) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (!cnt[i])
        for (int s = 0; s < a.stages * A; ++s) *in.slot(0, s, i) = make_uint4(0, 0, 0, 0);  // columns past the row
  }
  for (int s = 0; s < ahead; ++s) fetch(s);
  float2 g1[P2], b1[P2];
  if constexpr (NV == 1) {
    load_param<T, FULL>(a.gamma, col[0], cnt[0], 1.f, g1);
    load_param<T, FULL>(a.beta, col[0], cnt[0], 0.f, b1);
  } else {
    fill_param<T, FULL>(dyn, a.gamma, nvec, a.d, 1.f);
    fill_param<T, FULL>(dyn + nvec * (E / 4), a.beta, nvec, a.d, 0.f);
    __syncthreads();
  }
  T* yr = static_cast<T*>(a.Y) + row * a.ldy;
  T* zr = static_cast<T*>(a.Z) + row * a.ldz;
  for (; row < a.N; row += step, yr += step * a.ldy, zr += step * a.ldz) {
    if constexpr (STAGED) {
      st.turn(fetch);
      st.phase[0] = phase_of<T>(a.X, row, a.ldx);
      if (A == 2 && res) st.phase[A - 1] = phase_of<T>(a.R, row, a.ldr);
    } else {
      fetch(in.last_stage());
      in.wait();
    }
    auto get = [&](int arr, int i) {
      if constexpr (STAGED) return st.get(arr, col[i], cnt[i]);
      return in.get(arr, i);
    };
    float2 z[NV][P2], s2 = both(0.f), q2 = both(0.f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      unpack<T, FULL>(get(0, i), z[i]);
      if (drop) drop_vec<FULL>(z[i], a.k, static_cast<uint32_t>(row), col[i], mix[FULL ? 0 : threadIdx.x >> 5]);
      if (A == 2 && res) {
        float2 t[P2];
        unpack<T, FULL>(get(A - 1, i), t);
#pragma unroll
        for (int e = 0; e < P2; ++e) z[i][e] = add2(z[i][e], t[e]);
      }
#pragma unroll
      for (int e = 0; e < P2; ++e) s2 = add2(s2, z[i][e]);
    }
    if constexpr (STAGED)
      st.advance();
    else
      in.advance();
    float s[1] = {s2.x + s2.y};
    group_sum(s, sh[p.group][0], p);
    const float mean = s[0] / static_cast<float>(a.d);  // a division: a constant row whose sum is exact has that constant as its mean
    if (a.Z) {
#pragma unroll
      for (int i = 0; i < NV; ++i) store_vec<T, FULL>(zr, col[i], cnt[i], z[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int e = 0; e < P2; ++e) z[i][e] = add2(z[i][e], both(-mean));
      if (FULL ? cnt[i] > 0 : cnt[i] == E) {
#pragma unroll
        for (int e = 0; e < P2; ++e) q2 = fma2(z[i][e], z[i][e], q2);
      } else if (!FULL) {
#pragma unroll
        for (int e = 0; e < P2; ++e) {
          if (2 * e < cnt[i]) q2.x = fmaf(z[i][e].x, z[i][e].x, q2.x);
          if (2 * e + 1 < cnt[i]) q2.y = fmaf(z[i][e].y, z[i][e].y, q2.y);
        }
      }
    }
    float q[1] = {q2.x + q2.y};
    group_sum(q, sh[p.group][1], p);
    const float rstd = inv_sqrt(fmaf(q[0], a.inv_d, a.eps));
    if (p.tid == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float2 g[P2], b[P2];
      if constexpr (NV > 1) {
        read_param<T, FULL>(dyn, nvec, p.tid + i * p.T, g);
        read_param<T, FULL>(dyn + nvec * (E / 4), nvec, p.tid + i * p.T, b);
      }
#pragma unroll
      for (int e = 0; e < P2; ++e) b[e] = fma2(mul2(z[i][e], both(rstd)), NV > 1 ? g[e] : g1[e], NV > 1 ? b[e] : b1[e]);
      store_vec<T, FULL>(yr, col[i], cnt[i], b);
    }
  }
}

// The gradient.  A group keeps the column sums of its rows in registers; the
// block adds its groups' sums in shared memory and writes one pair of rows,
// which norm_cols_kernel adds over the blocks.  (WIDE, over 512 threads a
// row, has no registers left for them: norm_colsum_kernel reads dY and Z
// too, before this kernel, which may write over them.)  Every order is fixed, so dgamma and dbeta do not depend on
// timing.
// xh = (Z - mean) rstd on rows far from zero: Z rstd - mean rstd in one fused
// step has the rounding of mean * rstd in it (2e-4 of xh at a mean of 4096
// deviations).  So either the mean goes first, as in the forward pass, one
// instruction more; or (CARRY) that product's rounding error lo, which is
// exact by a second fused step and the same for the whole row, is added to the
// row's sums and to dgamma's terms.  CARRY where the first form costs more:
// with dropout, whose 24-column variant then spills (12608 x 768 bf16 with dZin
// 25.9 us instead of 29.8), and wide rows off 16 bytes (3600 x 9001 fp32 289
// us instead of 322); aligned wide rows the other way (2048 x 14336 bf16 74.7
// us, 78.8 with CARRY).
template <typename T, bool FULL, bool DROP, int NV, int MAXT, bool WIDE>
__global__ void __launch_bounds__(MAXT, 1) norm_grad_kernel(const NormGradArgs a) {
  using D = Deal<T, FULL>;
  constexpr int E = D::E, Q = E / 4, P2 = E / 2;
  constexpr int NA = WIDE ? 1 : NV;  // vectors whose sums are in registers (WIDE: none)
  constexpr bool CARRY = FULL ? DROP && !WIDE : WIDE;
  constexpr bool RING = FULL && !(WIDE && sizeof(T) == 4);  // wide fp32: gamma and a row of the ring are too much
  // gamma (NV > 1); then the ring, and after it in the same place the groups' sums [2][groups][d]
  extern __shared__ float4 dyn[];
  __shared__ float sh[kMaxGroups][2][64];
  __shared__ uint4 mix[FULL ? 1 : MAXT / 32][32];
  const Place p(a.groups);
  const int nvec = NV * p.T;
  float4* sums = NV > 1 ? dyn + nvec * Q : dyn;
  int col[NV], cnt[NV];
  float2 dg[NA][P2], db[NA][P2];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    col[i] = D::col(p.tid + i * p.T);
    cnt[i] = D::cnt(col[i], a.d);
    if constexpr (!WIDE) {
#pragma unroll
      for (int e = 0; e < P2; ++e) dg[i][e] = db[i][e] = both(0.f);
    }
  }
  const bool drop = FULL ? DROP : a.k.thr != 0;
  const int64_t step = static_cast<int64_t>(gridDim.x) * a.groups;
  int64_t row = static_cast<int64_t>(blockIdx.x) * a.groups + p.group;
  constexpr bool STAGED = !FULL && !WIDE;
  Rows<T, RING, 3, NV> in;  // dY, Z, dZin
  Staged<T, 3, NV> st;
  in.ring = reinterpret_cast<uint4*>(sums) + threadIdx.x;
  in.pitch = blockDim.x;
  in.stages = a.stages;
  in.at = 0;
  in.used = a.dZin ? 3 : 2;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if constexpr (STAGED) {
    st.used = in.used;
    st.bytes = a.stage_bytes;
    st.stages = a.stages;
    st.base = reinterpret_cast<uint8_t*>(sums) + p.group * (a.stages * st.used * st.bytes);
    st.at = 0;
    st.T_ = p.T;
    st.tid = p.tid;
    st.group = p.group;
  }
  int64_t next = row;
  auto fetch = [&](int stage) {
    const int64_t at = next;
    next += step;
    if constexpr (STAGED) {
      if (at < a.N) {
        auto start = [&](int arr, const void* q, int64_t ld) {
          const T* b = static_cast<const T*>(q);
          st.start(stage, arr, b + at * ld, b, b + ((a.N - 1) * ld + a.d), a.d);
        };
        start(0, a.dY, a.lddy);
        start(1, a.Z, a.ldz);
        if (a.dZin) start(2, a.dZin, a.lddzin);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      return;
    }
    if (at < a.N) {
      in.template start<FULL>(stage, 0, static_cast<const T*>(a.dY) + at * a.lddy, col, cnt);
      in.template start<FULL>(stage, 1, static_cast<const T*>(a.Z) + at * a.ldz, col, cnt);
      if (a.dZin) in.template start<FULL>(stage, 2, static_cast<const T*>(a.dZin) + at * a.lddzin, col, cnt);
    }
    in.commit();
  };
  const int ahead = RING || STAGED ? a.stages - 1 : 0;
  if constexpr (RING) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (!cnt[i])
        for (int s = 0; s < in.used * a.stages; ++s) *in.slot(0, s, i) = make_uint4(0, 0, 0, 0);  // columns past the row
  }
  for (int s = 0; s < ahead; ++s) fetch(s);
  float mu1 = 0.f, rs1 = 0.f;  // of the next row
  if (row < a.N) {
    mu1 = __ldg(a.mean + row);
    rs1 = __ldg(a.rstd + row);
  }
  float2 g1[P2];
  if constexpr (NV == 1) {
    load_param<T, FULL>(a.gamma, col[0], cnt[0], 1.f, g1);
  } else {
    fill_param<T, FULL>(dyn, a.gamma, nvec, a.d, 1.f);
    __syncthreads();
  }
  int buf = 0;
  for (; row < a.N; row += step) {
    if constexpr (STAGED) {
      st.turn(fetch);
      st.phase[0] = phase_of<T>(a.dY, row, a.lddy);
      st.phase[1] = phase_of<T>(a.Z, row, a.ldz);
      if (a.dZin) st.phase[2] = phase_of<T>(a.dZin, row, a.lddzin);
    } else {
      fetch(in.last_stage());
    }
    auto get = [&](int arr, int i) {
      if constexpr (STAGED) return st.get(arr, col[i], cnt[i]);
      return in.get(arr, i);
    };
    const float rstd = rs1, mu = mu1, shift = -mu1 * rs1, lo = CARRY ? fmaf(-mu1, rs1, -shift) : 0.f;
    if (row + step < a.N) {
      mu1 = __ldg(a.mean + row + step);
      rs1 = __ldg(a.rstd + row + step);
    }
    if constexpr (!STAGED) in.wait();
    float2 ag[NV][P2], xh[NV][P2], s1 = both(0.f), s2 = both(0.f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float2 dy[P2], g[P2];
      unpack<T, FULL>(get(0, i), dy);
      unpack<T, FULL>(get(1, i), xh[i]);
      if constexpr (NV > 1) read_param<T, FULL>(dyn, nvec, p.tid + i * p.T, g);
#pragma unroll
      for (int e = 0; e < P2; ++e) {
        // past the row's end dy = 0: xh there adds to no sum and is not stored
        xh[i][e] = CARRY ? fma2(xh[i][e], both(rstd), both(shift)) : mul2(add2(xh[i][e], both(-mu)), both(rstd));
        ag[i][e] = mul2(dy[e], NV > 1 ? g[e] : g1[e]);
        s1 = add2(s1, ag[i][e]);
        s2 = fma2(ag[i][e], xh[i][e], s2);
        if constexpr (!WIDE) {
          db[i][e] = add2(db[i][e], dy[e]);
          dg[i][e] = fma2(dy[e], CARRY ? add2(xh[i][e], both(lo)) : xh[i][e], dg[i][e]);
        }
      }
    }
    float s[2] = {s1.x + s1.y, s2.x + s2.y};
    group_sum(s, sh[p.group][buf], p);
    buf ^= 1;
    // dz = rstd (a - mean(a)) - xh c2, with c2 = rstd mean(a xh); xh + lo in place of xh where it is carried
    const float c2 = (CARRY ? fmaf(lo, s[0], s[1]) : s[1]) * a.inv_d * rstd;
    const float c1 = CARRY ? fmaf(lo, c2, s[0] * a.inv_d * rstd) : s[0] * a.inv_d * rstd;
    T* dzr = static_cast<T*>(a.dZ) + row * a.lddz;
    T* dxr = static_cast<T*>(a.dX) + row * a.lddx;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float2 dz[P2];
#pragma unroll
      for (int e = 0; e < P2; ++e) dz[e] = fma2(xh[i][e], both(-c2), fma2(ag[i][e], both(rstd), both(-c1)));
      if (a.dZin) {
        float2 u[P2];
        unpack<T, FULL>(get(2, i), u);
#pragma unroll
        for (int e = 0; e < P2; ++e) dz[e] = add2(dz[e], u[e]);
      }
      if (a.dZ) store_vec<T, FULL>(dzr, col[i], cnt[i], dz);
      if (a.dX) {
        if (drop) drop_vec<FULL>(dz, a.k, static_cast<uint32_t>(row), col[i], mix[FULL ? 0 : threadIdx.x >> 5]);
        store_vec<T, FULL>(dxr, col[i], cnt[i], dz);
      }
    }
    if constexpr (STAGED)
      st.advance();
    else
      in.advance();
  }
  if constexpr (!WIDE) {
    if (!a.part) return;
    float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * a.d;
    // float4 planes again: [dg, db][group][plane][vector]
    if constexpr (RING || STAGED) asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int v = p.tid + i * p.T;
        sums[(p.group * Q + q) * nvec + v] = make_float4(dg[i][2 * q].x, dg[i][2 * q].y, dg[i][2 * q + 1].x, dg[i][2 * q + 1].y);
        sums[((a.groups + p.group) * Q + q) * nvec + v] =
            make_float4(db[i][2 * q].x, db[i][2 * q].y, db[i][2 * q + 1].x, db[i][2 * q + 1].y);
      }
    __syncthreads();
    for (int u = threadIdx.x; u < 2 * Q * nvec; u += blockDim.x) {
      const int which = u / (Q * nvec), x = u - which * Q * nvec, c = D::col(x % nvec) + x / nvec * 4;
      float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int g = 0; g < a.groups; ++g) {
        const float4 f = sums[(which * a.groups + g) * Q * nvec + x];
        t = make_float4(t.x + f.x, t.y + f.y, t.z + f.z, t.w + f.w);
      }
      const float f[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e * D::STEP < a.d) part[static_cast<int64_t>(which) * a.d + c + e * D::STEP] = f[e];
    }
  }
}

// Column sums of wide rows: a warp takes 32 vectors of every kSumWarps-th row
// of the block's rows, the block joins its warps and writes one pair of rows
// (its 32 vectors of them).  Grid: vectors of a row / 32, runs of rows.  fp32
// off 16 bytes: held to 48 registers, with which five blocks are on an SM and
// the grid of about four takes one round (with 50, four: 3600 x 9001 gradient
// 308 us instead of 289).
// Bound by HBM, a second reading of dY and Z: 2048 x 14336 bf16 gradient with
// this pass 74 us, with the sums in shared memory beside the rows 109 us.
constexpr int kSumWarps = 8;
template <typename T, bool FULL>
__global__ void __launch_bounds__(32 * kSumWarps, FULL || sizeof(T) == 2 ? 0 : 5) norm_colsum_kernel(const NormGradArgs a) {
  using D = Deal<T, FULL>;
  constexpr int E = D::E, P2 = E / 2;
  __shared__ float2 sh[kSumWarps][2 * P2][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = D::col(blockIdx.x * 32 + lane), cnt = D::cnt(col, a.d);
  const int64_t r0 = a.N * blockIdx.y / gridDim.y, r1 = a.N * (blockIdx.y + 1) / gridDim.y;
  float2 dg[P2], db[P2];
#pragma unroll
  for (int e = 0; e < P2; ++e) dg[e] = db[e] = both(0.f);
#pragma unroll 4
  for (int64_t r = r0 + warp; r < r1; r += kSumWarps) {
    const float rstd = __ldg(a.rstd + r), mu = __ldg(a.mean + r);
    float2 dy[P2], z[P2];
    unpack<T, FULL>(load_raw<T, FULL>(static_cast<const T*>(a.dY) + r * a.lddy, col, cnt), dy);
    unpack<T, FULL>(load_raw<T, FULL>(static_cast<const T*>(a.Z) + r * a.ldz, col, cnt), z);
#pragma unroll
    for (int e = 0; e < P2; ++e) {
      db[e] = add2(db[e], dy[e]);
      dg[e] = fma2(dy[e], mul2(add2(z[e], both(-mu)), both(rstd)), dg[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < P2; ++e) {
    sh[warp][e][lane] = dg[e];
    sh[warp][P2 + e][lane] = db[e];
  }
  __syncthreads();
  float* part = a.part + static_cast<int64_t>(blockIdx.y) * 2 * a.d;
  for (int k = warp; k < 2 * P2; k += kSumWarps) {  // pair k of [dg, db]
    float2 t = sh[0][k][lane];
#pragma unroll
    for (int w = 1; w < kSumWarps; ++w) t = add2(t, sh[w][k][lane]);
    const int which = k / P2, e = k % P2 * 2;
    float* o = part + static_cast<int64_t>(which) * a.d + col;
    if (e < cnt) o[e * D::STEP] = t.x;
    if (e + 1 < cnt) o[(e + 1) * D::STEP] = t.y;
  }
}

// out[c] = sum over the blocks of their column sums, c < 2 d (dgamma, dbeta):
// 32 columns per CTA, kColRows threads per column, joined in a fixed order.
// Latency: 2 to 3 us after the gradient (152 rows of sums from L2).
constexpr int kColRows = 16;
struct NormColsArgs {
  const float* part;
  float* dgamma;
  float* dbeta;
  int32_t blocks, d;
};

__global__ void __launch_bounds__(32 * kColRows) norm_cols_kernel(const NormColsArgs a) {
  __shared__ float sh[kColRows][32];
  const int lane = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + lane;
  const int64_t w = 2 * static_cast<int64_t>(a.d);
  float s = 0.f;
  asm volatile("griddepcontrol.wait;" ::: "memory");  // launched while the kernel before it ends
  if (c < w) {
#pragma unroll 8
    for (int b = r; b < a.blocks; b += kColRows) s += a.part[b * w + c];
  }
  sh[r][lane] = s;
  __syncthreads();
  if (r == 0 && c < w) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < kColRows; ++i) s += sh[i][lane];
    if (c < a.d) {
      if (a.dgamma) a.dgamma[c] = s;
    } else if (a.dbeta) {
      a.dbeta[c - a.d] = s;
    }
  }
}

}  // namespace norm
}  // namespace ffb
