// Residual norm: the step between two blocks of a model on its residual stream.
//
//   u  = x rstd_post (o + w_post),  rstd_post = 1 / sqrt(mean(x^2) + eps)   (no w_post: u = x)
//   r' = alpha r + g u                                                      (no r: r' = g u)
//   y  = r' rstd_pre (o + w_pre),   rstd_pre  = 1 / sqrt(mean(r'^2) + eps)
//
// and backward, from dy and dr' (the later blocks' gradient of r'),
//   q  = dy (o + w_pre), n = r' rstd_pre
//   D  = dr' + rstd_pre (q - n mean(q n))          dw_pre  = sum_t dy n
//   dr = alpha D;  du = g D;  dg = D u             dw_post = sum_t du m,  m = x rstd_post
//   dx = rstd_post (p - m mean(p m)),  p = du (o + w_post)
// The backward needs one round of row sums: with t = dr' + rstd_pre q and gu = g u
// (a token's gate left out of g here),
//   A = sum q n,  B = sum gu t,  C = sum gu rstd_pre n,  sum gu D = B - (A / H) C
// and the last is what mean(p m) and a token's dg are made of.
//
// All arithmetic and all sums are fp32, each output is rounded once; y is formed from
// the unrounded r'.  The weights' gradients are summed over a block's rows in
// registers, then over the blocks in a fixed order, so the results are the same bits
// in every run.
//
// HBM bounds both directions where a row's chain (its sums are shuffles, a barrier and
// loads that wait for one another, 500 to 1000 clocks) is hidden by other rows of the SM;
// the backward of long rows has registers for one row at a time only.  Measured (bf16,
// both norms, channel gate): forward 32768 x 2048 with an fp32 stream 141 us, 5.7 TB/s;
// 16001 x 5120 113 us, 5.8; backward 190 us, 6.4, and 188 us, 5.2.  Steps: rows read
// twice from memory and the parameters with them 574 us (16001 x 5120 backward); rows
// held in registers and prefetched into them 184, but 289 against 190 with fp32 streams;
// parameters in shared memory and rows read there twice, several side by side 254.
#pragma once

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <cuda_runtime.h>

#include "molt_internal.cuh"
#include "ptx.cuh"
#include "vec.cuh"

namespace molt {

struct NormArgs {
  int64_t T;
  int H;
  int64_t x_ld, r_ld, dy_ld;       // elements between rows of x, r and dy
  const void *x, *r;               // r: the residual (forward: or nullptr) or r' (backward)
  const void *w_post, *gate, *w_pre;
  float *rstd_post, *rstd_pre;     // written by the forward (or nullptr), read by the backward
  void *y, *r_out;                 // forward (each or nullptr)
  const void *dy, *dr;             // backward; dr or nullptr
  void *dx, *dr_out, *dgate;       // dgate: [T] or [T, H]; dr_out or nullptr
  int stages, stage_bytes;         // persistent kernels: rows in flight, bytes of a row's stage
  int at_r, at_dy, at_dr, at_gate; // and where its parts lie in it
  unsigned* err;
  float* part;                     // [blocks, 3, H] sums of dw_post, the channel gate's gradient, dw_pre
  float alpha, eps, offset;
  int gate_kind;                   // MOLT_GATE_*
  int param_f32;                   // w_post, w_pre and a channel gate are fp32, else of x's type
};

constexpr int kNormMaxThreads = 512;              // of a row
constexpr int kNormMaxH = kNormMaxThreads * 32;   // longer rows take the kernels that loop over columns

// Barrier between the threads of a row: a warp (of a block of several rows), or the block.
// (Named barriers for rows of several warps side by side cost twice the time of a row:
// 65536 rows of 1024 elements backwards 273 and 135 us.)
__device__ __forceinline__ void row_barrier() {
  if (blockDim.x == 32)
    __syncwarp();
  else
    __syncthreads();
}

// Sums over a row's threads, kN (1 to 4) values at a time.  One warp a row: by shuffles.
// Several: the warps' sums pass through shared memory with one barrier (two buffers in
// turn, so that a row's sums are read before they are overwritten).  Four values cost
// hardly more shuffles than one: in the first two steps the lanes share the values out,
// a quarter of the warp to each.  All threads get the same bits.
template <int kN, int kMaxThreads>
struct RowSum {
  static constexpr int kWarps = kMaxThreads / 32;   // of a row, at most
  float4* buf;   // the row's part of a turn's buffer, a word to each of the block's warps
  int turn = 0;
  __device__ explicit RowSum(float4 (*b)[32]) : buf(b[0] + threadIdx.y * (blockDim.x >> 5)) {}
  // the warp's sum of value `lane / 8` (kN = 1: of the one value)
  static __device__ __forceinline__ float share(const float (&v)[kN]) {
    const int lane = threadIdx.x & 31;
    float s = v[0];
    if constexpr (kN > 1) {
      float w[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kN; ++k) w[k] = v[k];
      const bool up = lane & 16, odd = lane & 8;
      // lanes below 16 go on with values 0 and 1, the others with 2 and 3
      const float a = (up ? w[2] : w[0]) + __shfl_xor_sync(0xffffffffu, up ? w[0] : w[2], 16);
      const float b = (up ? w[3] : w[1]) + __shfl_xor_sync(0xffffffffu, up ? w[1] : w[3], 16);
      s = (odd ? b : a) + __shfl_xor_sync(0xffffffffu, odd ? a : b, 8);
    } else {
      s += __shfl_xor_sync(0xffffffffu, s, 16);
      s += __shfl_xor_sync(0xffffffffu, s, 8);
    }
    s += __shfl_xor_sync(0xffffffffu, s, 4);
    s += __shfl_xor_sync(0xffffffffu, s, 2);
    s += __shfl_xor_sync(0xffffffffu, s, 1);
    return s;
  }
  __device__ __forceinline__ void operator()(float (&v)[kN]) {
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    const float s = share(v);
    if (warps == 1) {
#pragma unroll
      for (int k = 0; k < kN; ++k) v[k] = __shfl_sync(0xffffffffu, s, 8 * k);
      return;
    }
    if (lane % 8 == 0) reinterpret_cast<float*>(buf + 32 * turn + (threadIdx.x >> 5))[lane / 8] = s;
    row_barrier();
    // lane l: warps l % 8, l % 8 + 8, ...
    constexpr int kReads = (kWarps + 7) / 8;
    float4 q[kReads];
#pragma unroll
    for (int i = 0; i < kReads; ++i) q[i] = buf[32 * turn + min(lane % 8 + 8 * i, warps - 1)];
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      v[k] = 0.f;
#pragma unroll
      for (int i = 0; i < kReads; ++i) {
        const float p = k == 0 ? q[i].x : k == 1 ? q[i].y : k == 2 ? q[i].z : q[i].w;
        v[k] += lane % 8 + 8 * i < warps ? p : 0.f;
      }
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
#pragma unroll
      for (int k = 0; k < kN; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    }
    turn ^= 1;
  }
};

// kV elements of a parameter vector, as fp32
template <int kV, class X>
__device__ __forceinline__ void load_param(const void* p, int f32, int c, float (&v)[kV]) {
  if (f32)
    load_vec<kV>(static_cast<const float*>(p) + c, v);
  else
    load_vec<kV>(static_cast<const X*>(p) + c, v);
}

// Forward.  blockDim.x threads hold a row in registers, E elements each as E / kV
// vectors of kV; blockDim.y rows to a block (more than one only where a row is one warp's).
template <class X, class R, int E>
__global__ void __launch_bounds__(kNormMaxThreads) norm_fwd_kernel(const NormArgs a) {
  constexpr int kV = 8, N = E / kV;
  __shared__ float4 buf[2][32];
  RowSum<1, kNormMaxThreads> row_sum(buf);
  const int H = a.H, G = blockDim.x;
  const float inv_H = 1.f / static_cast<float>(H);
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y; t < a.T;
       t += static_cast<int64_t>(gridDim.x) * blockDim.y) {
    const X* x = static_cast<const X*>(a.x) + t * a.x_ld;
    const R* r = a.r ? static_cast<const R*>(a.r) + t * a.r_ld : nullptr;
    float u[N][kV], rv[N][kV];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * G + threadIdx.x) * kV;
#pragma unroll
      for (int j = 0; j < kV; ++j) u[i][j] = 0.f;
      if (c < H) load_vec<kV>(x + c, u[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * G + threadIdx.x) * kV;
#pragma unroll
      for (int j = 0; j < kV; ++j) rv[i][j] = 0.f;
      if (r && c < H) load_vec<kV>(r + c, rv[i]);
    }
    if (a.w_post) {
      float ss[1] = {0.f};
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < kV; ++j) ss[0] = fmaf(u[i][j], u[i][j], ss[0]);
      row_sum(ss);
      const float rstd = rsqrtf(fmaf(ss[0], inv_H, a.eps));
      if (a.rstd_post && threadIdx.x == 0) a.rstd_post[t] = rstd;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int c = (i * G + threadIdx.x) * kV;
        if (c >= H) continue;
        float w[kV];
        load_param<kV, X>(a.w_post, a.param_f32, c, w);
#pragma unroll
        for (int j = 0; j < kV; ++j) u[i][j] *= rstd * (a.offset + w[j]);
      }
    }
    const float gt = a.gate_kind == MOLT_GATE_TOKEN ? static_cast<const float*>(a.gate)[t] : 1.f;
    float ss[1] = {0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * G + threadIdx.x) * kV;
      if (c >= H) continue;
      if (a.gate_kind == MOLT_GATE_CHANNEL || a.gate_kind == MOLT_GATE_FULL) {
        float g[kV];
        if (a.gate_kind == MOLT_GATE_CHANNEL)
          load_param<kV, X>(a.gate, a.param_f32, c, g);
        else
          load_vec<kV>(static_cast<const X*>(a.gate) + t * H + c, g);
#pragma unroll
        for (int j = 0; j < kV; ++j) u[i][j] *= g[j];
      }
#pragma unroll
      for (int j = 0; j < kV; ++j) {
        u[i][j] = fmaf(a.alpha, rv[i][j], gt * u[i][j]);
        ss[0] = fmaf(u[i][j], u[i][j], ss[0]);
      }
      if (a.r_out) store_vec<kV>(static_cast<R*>(a.r_out) + t * H + c, u[i]);
    }
    if (!a.w_pre) continue;
    row_sum(ss);
    const float rstd = rsqrtf(fmaf(ss[0], inv_H, a.eps));
    if (a.rstd_pre && threadIdx.x == 0) a.rstd_pre[t] = rstd;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * G + threadIdx.x) * kV;
      if (c >= H) continue;
      float w[kV];
      load_param<kV, X>(a.w_pre, a.param_f32, c, w);
#pragma unroll
      for (int j = 0; j < kV; ++j) u[i][j] *= rstd * (a.offset + w[j]);
      store_vec<kV>(static_cast<X*>(a.y) + t * H + c, u[i]);
    }
  }
}

// ---------------------------------------------------------------------------
// Persistent forms: a block works on one row at a time, on four where a row is one warp's;
// as many blocks as the SM holds.  Rows come by bulk copies into shared memory, the next
// while the present one is worked on (more stages gained nothing), one lane to each
// matrix; the parameters stay in registers.  A bulk copy moves whole 16-byte words: a row
// that begins inside a word brings the words it touches and is read at its offset; words
// that reach outside the matrix (its first and last row) are filled in element by element.
//   kV = 8: rows of whole vectors; a thread holds E / 8 vectors of 8 elements.
//   kV = 2: rows of whole pairs; a thread holds E / 2 pairs, blockDim.x pairs apart.
//   kV = 1: any row; a thread holds elements blockDim.x apart.
// Multiplications and additions are done two at a time (f32x2: a tenth fewer instructions).
// ---------------------------------------------------------------------------
constexpr int kRingStages = 2;
constexpr int kRingRows = 4;     // of a block, where a row is one warp's

// The rows of one matrix on their way through the ring; every lane of a row's first warp
// has one, lane i the i-th matrix's (bytes 0: none).
struct Stream {
  const uint8_t* next;      // the next row to copy
  int64_t step;             // bytes from there to the one after
  const uint8_t *lo, *hi;   // the matrix's first byte and its end
  int bytes;                // of a row
  int at;                   // offset in a stage
};

template <class T>
__device__ __forceinline__ void set_stream(Stream& s, int lane, int which, const void* base, int64_t ld, int64_t row,
                                           int64_t rows_step, int64_t T_rows, int H, int at) {
  if (lane != which || base == nullptr) return;
  const T* p = static_cast<const T*>(base);
  s.next = reinterpret_cast<const uint8_t*>(p + row * ld);
  s.step = rows_step * ld * static_cast<int64_t>(sizeof(T));
  s.lo = reinterpret_cast<const uint8_t*>(p);
  s.hi = reinterpret_cast<const uint8_t*>(p + (T_rows - 1) * ld + H);
  s.bytes = H * static_cast<int>(sizeof(T));
  s.at = at;
}

// Copies the next row of every stream into `stage`, complete when `bar` flips; by a whole warp.
template <int kV>
__device__ __forceinline__ void ring_fetch(Stream& s, uint8_t* stage, uint32_t bar) {
  const uint8_t *src = s.next, *end = src + s.bytes;
  uint8_t* dst = stage + s.at;
  int n = s.bytes;
  if constexpr (kV != 8) {
    const uint8_t* w0 = reinterpret_cast<const uint8_t*>(reinterpret_cast<uintptr_t>(src) & ~uintptr_t(15));
    const uint8_t* w1 = reinterpret_cast<const uint8_t*>((reinterpret_cast<uintptr_t>(end) + 15) & ~uintptr_t(15));
    __syncwarp();   // a row of one warp: all lanes have read what the stage held
    if (n > 0) {
      // words that reach outside the matrix: their bytes inside it, two at a time (elements
      // are of two or four bytes), ordered before the copies that will fill the stage again
      auto edge = [&](const uint8_t* w) {
        for (int b = 0; b < 16; b += 2)
          if (w + b >= s.lo && w + b < s.hi)
            *reinterpret_cast<uint16_t*>(dst + (w - w0) + b) = *reinterpret_cast<const uint16_t*>(w + b);
        fence_proxy_async_smem();
      };
      const uint8_t* first = w0;
      if (first < s.lo) {
        edge(first);
        first += 16;
      }
      if (w1 > s.hi && w1 > first) {
        w1 -= 16;
        edge(w1);
      }
      dst += first - w0;
      src = first;
      n = static_cast<int>(w1 - first);
    }
  }
  const int total = __reduce_add_sync(0xffffffffu, n);
  __syncwarp();   // the elements filled in come before the arrival
  if ((threadIdx.x & 31) == 0) mbar_arrive_expect_tx(bar, static_cast<uint32_t>(total));
  __syncwarp();
  if (n > 0)
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                     static_cast<uint32_t>(__cvta_generic_to_shared(dst))),
                 "l"(src), "r"(n), "r"(bar)
                 : "memory");
  s.next += s.step;
}

// Where a row lies in its stage.
template <class T, int kV>
__device__ __forceinline__ const T* staged_row(const uint8_t* stage, int at, const T* base, int64_t first_element) {
  if constexpr (kV == 8) return reinterpret_cast<const T*>(stage + at);
  return reinterpret_cast<const T*>(stage + at + (reinterpret_cast<uintptr_t>(base + first_element) & 15));
}

// The full barriers of the rows' stages; give_up: a wait ran out (the row's elements are
// then whatever the stage held, the device status says so, and further waits are short).
struct RingBars {
  uint32_t bar0;
  bool give_up = false;
  __device__ __forceinline__ void wait(int slot, uint32_t parity, unsigned* err) {
    const uint32_t bar = bar0 + 8 * slot;
    if (mbar_try_wait(bar, parity)) return;
    const uint64_t t0 = globaltimer_ns(), limit = give_up ? kWaitTimeoutNs >> 12 : kWaitTimeoutNs;
    for (uint32_t i = 1; i < kWaitMaxPolls; ++i) {
      if (mbar_try_wait(bar, parity)) return;
      if ((i & 31u) == 0u && globaltimer_ns() - t0 > limit) break;
    }
    give_up = true;
    atomicOr(err, kDevErrTimeout);
  }
};

// A thread's share of a row: E elements as pairs.
template <int kV, int E>
struct Share {
  static constexpr int kPairs = E / 2;
  int H;
  // of the vector that element e begins
  __device__ __forceinline__ int col(int e) const {
    return (e / kV * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * kV;
  }
  __device__ __forceinline__ bool has(int e) const { return col(e) < H; }
  // elements past the row's end read as 0
  template <class T>
  __device__ __forceinline__ void load(const T* row, F2 (&v)[kPairs]) const {
    if constexpr (kV == 8) {
#pragma unroll
      for (int e = 0; e < E; e += 8) {
        if (has(e)) {
          load_pairs(row + col(e), v + e / 2);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[e / 2 + j] = f2(0.f);
        }
      }
    } else if constexpr (kV == 2) {
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        float p[2] = {0.f, 0.f};
        if (has(e)) load_vec<2>(row + col(e), p);
        v[e / 2] = f2(p[0], p[1]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; e += 2)
        v[e / 2] = f2(has(e) ? to_float(row[col(e)]) : 0.f, has(e + 1) ? to_float(row[col(e + 1)]) : 0.f);
    }
  }
  template <class T>
  __device__ __forceinline__ void store(T* row, const F2 (&v)[kPairs]) const {
    if constexpr (kV == 8) {
#pragma unroll
      for (int e = 0; e < E; e += 8)
        if (has(e)) store_pairs(row + col(e), v + e / 2);
    } else if constexpr (kV == 2) {
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float p[2] = {v[e / 2].x(), v[e / 2].y()};
        if (has(e)) store_vec<2>(row + col(e), p);
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        if (has(e)) from_float(v[e / 2].x(), row[col(e)]);
        if (has(e + 1)) from_float(v[e / 2].y(), row[col(e + 1)]);
      }
    }
  }
};

// A parameter plus `add`, or `otherwise`.
template <class X, int kV, int E>
__device__ __forceinline__ void param(const void* p, int f32, float add, float otherwise, const Share<kV, E>& sh, F2 (&v)[E / 2]) {
  if (p == nullptr) {
#pragma unroll
    for (int j = 0; j < E / 2; ++j) v[j] = f2(otherwise);
    return;
  }
  if (f32)
    sh.load(static_cast<const float*>(p), v);
  else
    sh.load(static_cast<const X*>(p), v);
#pragma unroll
  for (int j = 0; j < E / 2; ++j) v[j] = add2(v[j], f2(add));
}

// The stages of a row's matrices, and the rows on their way.
template <int kV>
struct Ring {
  uint8_t* rows;     // this row's stages
  RingBars full;
  Stream s{};
  int slot = 0;
  uint32_t parity = 0;
  __device__ __forceinline__ Ring(const NormArgs& a, uint8_t* smem, uint64_t (*bars)[kRingStages])
      : rows(smem + static_cast<size_t>(threadIdx.y) * a.stages * a.stage_bytes), full{smem_u32(&bars[threadIdx.y][0])} {
    if (threadIdx.x == 0) {
      for (int i = 0; i < a.stages; ++i) mbar_init(full.bar0 + 8 * i, 1);
      fence_mbar_init();
    }
    __syncthreads();
  }
  // (by the row's first warp, once its matrices are set)
  __device__ __forceinline__ void begin(const NormArgs& a, int t, int step) {
    for (int i = 0; i < a.stages; ++i)
      if (static_cast<int64_t>(t) + static_cast<int64_t>(i) * step < a.T) ring_fetch<kV>(s, rows + i * a.stage_bytes, full.bar0 + 8 * i);
  }
  __device__ __forceinline__ uint8_t* wait(const NormArgs& a) {
    full.wait(slot, parity, a.err);
    return rows + slot * a.stage_bytes;
  }
  // the present stage has been read by all of the row's threads, which have met since
  __device__ __forceinline__ void refill(const NormArgs& a, int t, int step) {
    if (threadIdx.x < 32 && static_cast<int64_t>(t) + static_cast<int64_t>(a.stages) * step < a.T)
      ring_fetch<kV>(s, rows + slot * a.stage_bytes, full.bar0 + 8 * slot);
    if (++slot == a.stages) {
      slot = 0;
      parity ^= 1u;
    }
  }
};

template <class X, class R, int kV, int E, int kThreads, int kBlocks, bool kFull>
__global__ void __launch_bounds__(kThreads, kBlocks) norm_fwd_rows_kernel(const NormArgs a) {
  constexpr int P = E / 2;
  __shared__ float4 buf[2][32];
  __shared__ __align__(8) uint64_t bars[kRingRows][kRingStages];
  extern __shared__ __align__(16) uint8_t smem[];
  RowSum<1, kThreads> row_sum(buf);
  const Share<kV, E> sh{a.H};
  const int H = a.H;
  const float inv_H = 1.f / static_cast<float>(H);
  const bool token = a.gate_kind == MOLT_GATE_TOKEN, one_warp = blockDim.x == 32;
  const int step = gridDim.x * blockDim.y, T = static_cast<int>(a.T);
  int t = blockIdx.x * blockDim.y + threadIdx.y;
  Ring<kV> ring(a, smem, bars);
  if (threadIdx.x < 32) {
    set_stream<X>(ring.s, threadIdx.x, 0, a.x, a.x_ld, t, step, a.T, H, 0);
    set_stream<R>(ring.s, threadIdx.x, 1, a.r, a.r_ld, t, step, a.T, H, a.at_r);
    if constexpr (kFull) set_stream<X>(ring.s, threadIdx.x, 2, a.gate, H, t, step, a.T, H, a.at_gate);
    ring.begin(a, t, step);
  }
  float gt_next = token && t < T ? static_cast<const float*>(a.gate)[t] : 1.f;
  F2 wg[P], wpr[P];   // (o + w_post) times a channel gate, o + w_pre
  {
    F2 c[P];
    param<X, kV, E>(a.w_post, a.param_f32, a.offset, 1.f, sh, wg);
    param<X, kV, E>(a.gate_kind == MOLT_GATE_CHANNEL ? a.gate : nullptr, a.param_f32, 0.f, 1.f, sh, c);
    param<X, kV, E>(a.w_pre, a.param_f32, a.offset, 0.f, sh, wpr);
#pragma unroll
    for (int j = 0; j < P; ++j) wg[j] = mul2(wg[j], c[j]);
  }
  for (; t < T; t += step) {
    const uint8_t* stage = ring.wait(a);
    const int64_t row0 = static_cast<int64_t>(t) * H;
    F2 u[P], v[P];
    sh.load(staged_row<X, kV>(stage, 0, static_cast<const X*>(a.x), t * a.x_ld), u);
    if (a.r) sh.load(staged_row<R, kV>(stage, a.at_r, static_cast<const R*>(a.r), t * a.r_ld), v);
    F2 q = f2(0.f);
    if (a.w_post) {
#pragma unroll
      for (int j = 0; j < P; ++j) q = fma2(u[j], u[j], q);
    }
    if constexpr (kFull) {
      F2 c[P];
      sh.load(staged_row<X, kV>(stage, a.at_gate, static_cast<const X*>(a.gate), row0), c);
#pragma unroll
      for (int j = 0; j < P; ++j) u[j] = mul2(u[j], c[j]);
    }
    float scale = gt_next;
    if (token && t + step < T) gt_next = static_cast<const float*>(a.gate)[t + step];
    if (a.w_post) {
      float ss[1] = {q.x() + q.y()};
      row_sum(ss);
      const float rstd = rsqrtf(fmaf(ss[0], inv_H, a.eps));
      if (a.rstd_post && threadIdx.x == 0) a.rstd_post[t] = rstd;
      scale *= rstd;
    }
    // The stage is free once all threads have the row in registers.  A row of one warp
    // hands it back here, longer ones after the row's stores, which then are not behind
    // the next row's loads (65536 x 1024 97 and 87 us; 65536 x 256 29 and 39).
    if (one_warp) ring.refill(a, t, step);
    q = f2(0.f);
#pragma unroll
    for (int j = 0; j < P; ++j) {
      u[j] = mul2(mul2(u[j], f2(scale)), wg[j]);
      if (a.r) u[j] = fma2(f2(a.alpha), v[j], u[j]);
      q = fma2(u[j], u[j], q);
    }
    if (!a.w_pre) {
      if (a.r_out) sh.store(static_cast<R*>(a.r_out) + row0, u);
      if (!one_warp) {
        row_barrier();
        ring.refill(a, t, step);
      }
      continue;
    }
    float ss[1] = {q.x() + q.y()};
    row_sum(ss);
    if (a.r_out) sh.store(static_cast<R*>(a.r_out) + row0, u);
    const float rstd = rsqrtf(fmaf(ss[0], inv_H, a.eps));
    if (a.rstd_pre && threadIdx.x == 0) a.rstd_pre[t] = rstd;
#pragma unroll
    for (int j = 0; j < P; ++j) u[j] = mul2(mul2(u[j], f2(rstd)), wpr[j]);
    sh.store(static_cast<X*>(a.y) + row0, u);
    if (!one_warp) ring.refill(a, t, step);
  }
}

template <class X, class R, int kV, int E, int kThreads, int kBlocks, bool kFull>
__global__ void __launch_bounds__(kThreads, kBlocks) norm_bwd_rows_kernel(const NormArgs a) {
  constexpr int P = E / 2;
  __shared__ float4 buf[2][32];
  __shared__ __align__(8) uint64_t bars[kRingRows][kRingStages];
  extern __shared__ __align__(16) uint8_t smem[];
  RowSum<3, kThreads> row_sum(buf);
  const Share<kV, E> sh{a.H};
  const int H = a.H;
  const float inv_H = 1.f / static_cast<float>(H);
  const bool token = a.gate_kind == MOLT_GATE_TOKEN, channel = a.gate_kind == MOLT_GATE_CHANNEL;
  const int step = gridDim.x * blockDim.y, T = static_cast<int>(a.T);
  int t = blockIdx.x * blockDim.y + threadIdx.y;
  Ring<kV> ring(a, smem, bars);
  if (threadIdx.x < 32) {
    set_stream<X>(ring.s, threadIdx.x, 0, a.x, a.x_ld, t, step, a.T, H, 0);
    set_stream<R>(ring.s, threadIdx.x, 1, a.w_pre ? a.r : nullptr, a.r_ld, t, step, a.T, H, a.at_r);
    set_stream<X>(ring.s, threadIdx.x, 2, a.w_pre ? a.dy : nullptr, a.dy_ld, t, step, a.T, H, a.at_dy);
    set_stream<R>(ring.s, threadIdx.x, 3, a.dr, H, t, step, a.T, H, a.at_dr);
    if constexpr (kFull) set_stream<X>(ring.s, threadIdx.x, 4, a.gate, H, t, step, a.T, H, a.at_gate);
    ring.begin(a, t, step);
  }
  // a row's statistics and token gate, loaded a row ahead
  float n_pre = 0.f, n_post = 1.f, n_gate = 1.f;
  auto stats_of = [&](int row) {
    if (row >= T) return;
    if (a.w_pre) n_pre = a.rstd_pre[row];
    if (a.w_post) n_post = a.rstd_post[row];
    if (token) n_gate = static_cast<const float*>(a.gate)[row];
  };
  stats_of(t);
  F2 wg[P], wpr[P];   // (o + w_post) times a channel gate, o + w_pre
  {
    F2 c[P];
    param<X, kV, E>(a.w_post, a.param_f32, a.offset, 1.f, sh, wg);
    param<X, kV, E>(channel ? a.gate : nullptr, a.param_f32, 0.f, 1.f, sh, c);
    param<X, kV, E>(a.w_pre, a.param_f32, a.offset, 0.f, sh, wpr);
#pragma unroll
    for (int j = 0; j < P; ++j) wg[j] = mul2(wg[j], c[j]);
  }
  // sums over rows: of D m (times a token's or an element's gate; a channel's is the same
  // in every row and multiplies the sum), and of dy n
  F2 sum_dm[P], sum_pre[P];
#pragma unroll
  for (int j = 0; j < P; ++j) sum_dm[j] = sum_pre[j] = f2(0.f);
  for (; t < T; t += step) {
    const float pre = n_pre, post = n_post, gate = n_gate;
    if (T - t > step) stats_of(t + step);
    const uint8_t* stage = ring.wait(a);
    const int64_t row0 = static_cast<int64_t>(t) * H;
    F2 tt[P], n[P], m[P], c[kFull ? P : 1];   // t = dr' + rstd_pre dy (o + w_pre), r', x, an element's gate
    F2 q0 = f2(0.f), q1 = f2(0.f), q2 = f2(0.f);
    sh.load(staged_row<X, kV>(stage, 0, static_cast<const X*>(a.x), t * a.x_ld), m);
    if (a.dr) {
      sh.load(staged_row<R, kV>(stage, a.at_dr, static_cast<const R*>(a.dr), row0), tt);
    } else {
#pragma unroll
      for (int j = 0; j < P; ++j) tt[j] = f2(0.f);
    }
    if constexpr (kFull) sh.load(staged_row<X, kV>(stage, a.at_gate, static_cast<const X*>(a.gate), row0), c);
    if (a.w_pre) {
      F2 d[P];
      sh.load(staged_row<R, kV>(stage, a.at_r, static_cast<const R*>(a.r), t * a.r_ld), n);
      sh.load(staged_row<X, kV>(stage, a.at_dy, static_cast<const X*>(a.dy), t * a.dy_ld), d);
#pragma unroll
      for (int j = 0; j < P; ++j) {
        d[j] = mul2(d[j], f2(pre));
        const F2 p = mul2(d[j], wpr[j]);
        tt[j] = add2(tt[j], p);
        q0 = fma2(p, n[j], q0);
        sum_pre[j] = fma2(d[j], n[j], sum_pre[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < P; ++j) n[j] = f2(0.f);
    }
#pragma unroll
    for (int j = 0; j < P; ++j) {
      F2 xg = mul2(m[j], wg[j]);
      if constexpr (kFull) xg = mul2(xg, c[j]);
      q1 = fma2(xg, tt[j], q1);
      q2 = fma2(xg, n[j], q2);
    }
    float sums[3] = {q0.x() + q0.y(), q1.x() + q1.y(), q2.x() + q2.y()};
    row_sum(sums);
    ring.refill(a, t, step);
    const float c_n = pre * pre * (sums[0] * inv_H);               // D = t - c_n r'
    const float gu_D = post * fmaf(-c_n, sums[2], sums[1]);        // sum of g u D, without a token's gate
    const float c_d = post * gate;                                 // dx = c_d g D (o + w_post) - c_x x
    const float c_x = post * post * (gate * gu_D * inv_H);
    if (token && threadIdx.x == 0) static_cast<float*>(a.dgate)[t] = gu_D;
    F2 o[P];
#pragma unroll
    for (int j = 0; j < P; ++j) {
      tt[j] = fma2(f2(-c_n), n[j], tt[j]);                         // D
      o[j] = mul2(f2(a.alpha), tt[j]);
    }
    if (a.dr_out) sh.store(static_cast<R*>(a.dr_out) + row0, o);
    if constexpr (kFull) {
#pragma unroll
      for (int j = 0; j < P; ++j) {
        o[j] = mul2(tt[j], mul2(mul2(m[j], f2(post)), wg[j]));
        tt[j] = mul2(tt[j], c[j]);
      }
      sh.store(static_cast<X*>(a.dgate) + row0, o);
    }
#pragma unroll
    for (int j = 0; j < P; ++j) {
      tt[j] = mul2(tt[j], f2(c_d));
      sum_dm[j] = fma2(tt[j], m[j], sum_dm[j]);
      o[j] = mul2(tt[j], wg[j]);
      if (a.w_post) o[j] = fma2(f2(-c_x), m[j], o[j]);
    }
    sh.store(static_cast<X*>(a.dx) + row0, o);
  }
  // the block's sums: dw_post = g sum_dm, a channel gate's gradient (o + w_post) sum_dm
  float* ysum = reinterpret_cast<float*>(smem);   // [blockDim.y, H] where a block has several rows
  auto put = [&](int which, const void* factor, float add, const F2 (&v)[P]) {
    float* out = a.part + (static_cast<int64_t>(blockIdx.x) * 3 + which) * H;
    F2 f[P];
    param<X, kV, E>(factor, a.param_f32, add, 1.f, sh, f);
#pragma unroll
    for (int j = 0; j < P; ++j) f[j] = mul2(f[j], v[j]);
    if (blockDim.y == 1) {   // (a row of the parts is on a boundary of kV elements)
      sh.store(out, f);
      return;
    }
    __syncthreads();   // the rows are done with, or the sums before are out
    sh.store(ysum + threadIdx.y * H, f);
    __syncthreads();
    for (int i = threadIdx.y * blockDim.x + threadIdx.x; i < H; i += blockDim.x * blockDim.y) {
      float sum = 0.f;
      for (int y = 0; y < static_cast<int>(blockDim.y); ++y) sum += ysum[y * H + i];
      out[i] = sum;
    }
  };
  if (a.w_post) put(0, channel ? a.gate : nullptr, 0.f, sum_dm);
  if (channel) put(1, a.w_post, a.offset, sum_dm);
  if (a.w_pre) put(2, nullptr, 0.f, sum_pre);
}

// Rows of more than kNormMaxH elements, or of any length: threads walk the columns and
// read the row again for every step of it (from L2).
template <class X, class R>
__global__ void __launch_bounds__(kNormMaxThreads) norm_fwd_long_kernel(const NormArgs a) {
  __shared__ float4 buf[2][32];
  RowSum<1, kNormMaxThreads> row_sum(buf);
  const int H = a.H;
  const float inv_H = 1.f / static_cast<float>(H);
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const X* x = static_cast<const X*>(a.x) + t * a.x_ld;
    const R* r = a.r ? static_cast<const R*>(a.r) + t * a.r_ld : nullptr;
    float rstd_post = 1.f;
    if (a.w_post) {
      float ss[1] = {0.f};
      for (int c = threadIdx.x; c < H; c += blockDim.x) {
        const float v = to_float(x[c]);
        ss[0] = fmaf(v, v, ss[0]);
      }
      row_sum(ss);
      rstd_post = rsqrtf(fmaf(ss[0], inv_H, a.eps));
      if (a.rstd_post && threadIdx.x == 0) a.rstd_post[t] = rstd_post;
    }
    const float gt = a.gate_kind == MOLT_GATE_TOKEN ? static_cast<const float*>(a.gate)[t] : 1.f;
    auto stream = [&](int c) -> float {
      float u = to_float(x[c]), w[1];
      if (a.w_post) {
        load_param<1, X>(a.w_post, a.param_f32, c, w);
        u *= rstd_post * (a.offset + w[0]);
      }
      if (a.gate_kind == MOLT_GATE_CHANNEL) {
        load_param<1, X>(a.gate, a.param_f32, c, w);
        u *= w[0];
      } else if (a.gate_kind == MOLT_GATE_FULL) {
        u *= to_float(static_cast<const X*>(a.gate)[t * H + c]);
      }
      return fmaf(a.alpha, r ? to_float(r[c]) : 0.f, gt * u);
    };
    float rstd = 0.f;
    if (a.w_pre) {
      float ss[1] = {0.f};
      for (int c = threadIdx.x; c < H; c += blockDim.x) {
        const float v = stream(c);
        ss[0] = fmaf(v, v, ss[0]);
      }
      row_sum(ss);
      rstd = rsqrtf(fmaf(ss[0], inv_H, a.eps));
      if (a.rstd_pre && threadIdx.x == 0) a.rstd_pre[t] = rstd;
    }
    for (int c = threadIdx.x; c < H; c += blockDim.x) {
      const float v = stream(c);
      if (a.w_pre) {
        float w[1];
        load_param<1, X>(a.w_pre, a.param_f32, c, w);
        from_float(v * (rstd * (a.offset + w[0])), static_cast<X*>(a.y)[t * H + c]);
      }
      if (a.r_out) from_float(v, static_cast<R*>(a.r_out)[t * H + c]);
    }
  }
}

template <class X, class R>
__global__ void __launch_bounds__(kNormMaxThreads) norm_bwd_long_kernel(const NormArgs a) {
  __shared__ float4 buf[2][32];
  RowSum<3, kNormMaxThreads> row_sum(buf);
  const int H = a.H;
  const float inv_H = 1.f / static_cast<float>(H);
  float* part = a.part + static_cast<int64_t>(blockIdx.x) * 3 * H;
  bool first = true;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x, first = false) {
    const X* x = static_cast<const X*>(a.x) + t * a.x_ld;
    const R* r = static_cast<const R*>(a.r) + t * a.r_ld;
    const X* dy = static_cast<const X*>(a.dy) + t * a.dy_ld;
    const R* dr = a.dr ? static_cast<const R*>(a.dr) + t * H : nullptr;
    const float rstd_pre = a.w_pre ? a.rstd_pre[t] : 0.f, rstd_post = a.w_post ? a.rstd_post[t] : 1.f;
    const float gt = a.gate_kind == MOLT_GATE_TOKEN ? static_cast<const float*>(a.gate)[t] : 1.f;
    float n, q, m, dyc, drc, wpo, g;
    auto read = [&](int c) {
      float w[1];
      n = q = dyc = 0.f;
      wpo = g = 1.f;
      if (a.w_pre) {
        load_param<1, X>(a.w_pre, a.param_f32, c, w);
        n = to_float(r[c]) * rstd_pre;
        dyc = to_float(dy[c]);
        q = dyc * (a.offset + w[0]);
      }
      drc = dr ? to_float(dr[c]) : 0.f;
      m = to_float(x[c]) * rstd_post;
      if (a.w_post) {
        load_param<1, X>(a.w_post, a.param_f32, c, w);
        wpo = a.offset + w[0];
      }
      if (a.gate_kind == MOLT_GATE_CHANNEL) {
        load_param<1, X>(a.gate, a.param_f32, c, w);
        g = w[0];
      } else if (a.gate_kind == MOLT_GATE_FULL) {
        g = to_float(static_cast<const X*>(a.gate)[t * H + c]);
      }
    };
    float s[3] = {0.f, 0.f, 0.f};
    for (int c = threadIdx.x; c < H; c += blockDim.x) {
      read(c);
      const float gu = g * m * wpo;
      s[0] = fmaf(q, n, s[0]);
      s[1] = fmaf(gu, fmaf(rstd_pre, q, drc), s[1]);
      s[2] = fmaf(gu, rstd_pre * n, s[2]);
    }
    row_sum(s);
    const float mean_qn = s[0] * inv_H;
    const float gu_D = s[1] - mean_qn * s[2];
    const float mean_pm = gt * gu_D * inv_H;
    if (a.gate_kind == MOLT_GATE_TOKEN && threadIdx.x == 0) static_cast<float*>(a.dgate)[t] = gu_D;
    for (int c = threadIdx.x; c < H; c += blockDim.x) {
      read(c);
      const float D = fmaf(rstd_pre, q - n * mean_qn, drc);
      const float Du = D * (m * wpo), du = gt * g * D;
      // a thread keeps to its columns, so the block's sums need no ordering among threads
      auto add = [&](int which, float v) { part[which * H + c] = (first ? 0.f : part[which * H + c]) + v; };
      if (a.w_post) add(0, du * m);
      if (a.gate_kind == MOLT_GATE_CHANNEL) add(1, Du);
      if (a.w_pre) add(2, dyc * n);
      from_float(a.w_post ? rstd_post * (du * wpo - m * mean_pm) : du, static_cast<X*>(a.dx)[t * H + c]);
      if (a.dr_out) from_float(a.alpha * D, static_cast<R*>(a.dr_out)[t * H + c]);
      if (a.gate_kind == MOLT_GATE_FULL) from_float(Du, static_cast<X*>(a.dgate)[t * H + c]);
    }
  }
}

// how a row of H elements is laid out: threads to a row, rows to a block, elements to
// a thread (0: the kernels that loop over columns) and to a vector
struct NormShape {
  int threads, rows, elems, vec;
  bool persistent;
  size_t smem;
};

constexpr int kRingSmem = 216 * 1024;   // dynamic shared memory of the persistent kernels on an SM, at most
constexpr int kMaxBlocksPerSM = 8;

// Of a kernel on a device: allowed the shared memory above, and its registers to a warp.
struct KernelInfo {
  std::atomic<int> regs[64] = {};
  template <class K>
  cudaError_t get(K* kernel, int* warp_regs) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    int r = regs[dev & 63].load(std::memory_order_acquire);
    if (r == 0) {
      cudaFuncAttributes at{};
      e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingSmem);
      if (e == cudaSuccess) e = cudaFuncGetAttributes(&at, kernel);
      if (e != cudaSuccess) return e;
      r = (at.numRegs * 32 + 255) / 256 * 256;
      regs[dev & 63].store(r, std::memory_order_release);
    }
    *warp_regs = r;
    return cudaSuccess;
  }
};

template <class X, class R>
cudaError_t launch_norm_rows(const NormArgs& a, const NormShape& s, int n_sm, int* grid, bool bwd, cudaStream_t stream) {
  using Kernel = void (*)(const NormArgs);
  // by the elements and threads of a row: 8 and up to 640, 16 and up to 192, 320 and 512
  // (rows_shape gives 16 elements to 193 to 320 threads in the forward of vectors and pairs only)
#define MOLT_FWD(V, E, THREADS, BLOCKS) \
  norm_fwd_rows_kernel<X, R, V, E, THREADS, BLOCKS, false>, norm_fwd_rows_kernel<X, R, V, E, THREADS, BLOCKS, true>
#define MOLT_BWD(V, E, THREADS, BLOCKS) \
  norm_bwd_rows_kernel<X, R, V, E, THREADS, BLOCKS, false>, norm_bwd_rows_kernel<X, R, V, E, THREADS, BLOCKS, true>
#define MOLT_NONE nullptr, nullptr
#define MOLT_ROWS(V, FWD_320)                           \
  {{MOLT_FWD(V, 8, 640, 1), MOLT_BWD(V, 8, 640, 1)},    \
   {MOLT_FWD(V, 16, 192, 1), MOLT_BWD(V, 16, 128, 3)},  \
   {FWD_320, MOLT_NONE},                                \
   {MOLT_FWD(V, 16, 512, 1), MOLT_BWD(V, 16, 512, 1)}}
  static constexpr Kernel kernels[3][4][4] = {MOLT_ROWS(1, MOLT_NONE), MOLT_ROWS(2, MOLT_FWD(2, 16, 320, 2)),
                                              MOLT_ROWS(8, MOLT_FWD(8, 16, 320, 2))};
#undef MOLT_ROWS
#undef MOLT_NONE
#undef MOLT_BWD
#undef MOLT_FWD
  static KernelInfo info[3][4][4];
  const int vec = s.vec == 8 ? 2 : s.vec == 2 ? 1 : 0, size = s.elems == 8 ? 0 : s.threads <= 192 ? 1 : s.threads <= 320 ? 2 : 3;
  const int which = (bwd ? 2 : 0) + (a.gate_kind == MOLT_GATE_FULL ? 1 : 0);
  const Kernel k = kernels[vec][size][which];
  if (k == nullptr) return cudaErrorInvalidValue;   // a shape that rows_shape does not give
  int warp_regs;
  const cudaError_t e = info[vec][size][which].get(k, &warp_regs);
  if (e != cudaSuccess) return e;
  // one wave of blocks: as many as registers and shared memory hold
  const int warps = s.threads / 32 * s.rows;
  const int per_sm = std::max(1, std::min({kMaxBlocksPerSM, 65536 / (warps * warp_regs), kRingSmem / static_cast<int>(s.smem + 2048)}));
  *grid = static_cast<int>(std::min<int64_t>((a.T + s.rows - 1) / s.rows, static_cast<int64_t>(n_sm) * per_sm));
  k<<<*grid, dim3(s.threads, s.rows), s.smem, stream>>>(a);
  return cudaGetLastError();
}

// grid: the blocks launched
template <class X, class R>
cudaError_t launch_norm_typed(const NormArgs& a, const NormShape& s, int n_sm, int* grid, bool bwd, cudaStream_t stream) {
  if (s.persistent) return launch_norm_rows<X, R>(a, s, n_sm, grid, bwd, stream);
  if (bwd) {
    *grid = static_cast<int>(std::min<int64_t>(a.T, 2 * static_cast<int64_t>(n_sm)));
    norm_bwd_long_kernel<X, R><<<*grid, s.threads, 0, stream>>>(a);
    return cudaGetLastError();
  }
  *grid = static_cast<int>((a.T + s.rows - 1) / s.rows);
  auto* k = s.elems == 0    ? norm_fwd_long_kernel<X, R>
            : s.elems == 8  ? norm_fwd_kernel<X, R, 8>
            : s.elems == 16 ? norm_fwd_kernel<X, R, 16>
                            : norm_fwd_kernel<X, R, 32>;
  k<<<*grid, dim3(s.threads, s.rows), 0, stream>>>(a);
  return cudaGetLastError();
}

// one translation unit per type of x (norm_*.cu)
cudaError_t launch_norm_bf16(const NormArgs& a, const NormShape& s, int n_sm, int* grid, bool r_f32, bool bwd, cudaStream_t stream);
cudaError_t launch_norm_fp16(const NormArgs& a, const NormShape& s, int n_sm, int* grid, bool r_f32, bool bwd, cudaStream_t stream);
cudaError_t launch_norm_fp32(const NormArgs& a, const NormShape& s, int n_sm, int* grid, bool bwd, cudaStream_t stream);

}  // namespace molt
