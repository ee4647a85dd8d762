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
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "molt_internal.cuh"
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
  float* part;                     // [blocks, 3, H] sums of dw_post, the channel gate's gradient, dw_pre
  float alpha, eps, offset;
  int gate_kind;                   // MOLT_GATE_*
  int param_f32;                   // w_post, w_pre and a channel gate are fp32, else of x's type
};

constexpr int kNormMaxThreads = 512;
constexpr int kNormMaxH = kNormMaxThreads * 32;   // longer rows take the kernels that loop over columns

// Sums over a row's threads, kN values at a time: a warp by shuffles, several warps
// through shared memory with one barrier (two buffers in turn, so that a row's sums
// are read before they are overwritten).
template <int kN>
struct RowSum {
  float (*buf)[kN][16];
  int turn = 0;
  __device__ explicit RowSum(float (*b)[kN][16]) : buf(b) {}
  __device__ __forceinline__ void operator()(float (&v)[kN]) {
#pragma unroll
    for (int k = 0; k < kN; ++k) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    }
    const int warps = blockDim.x >> 5;
    if (warps == 1) return;   // one warp a row
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int k = 0; k < kN; ++k) buf[turn][k][threadIdx.x >> 5] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      float s = 0.f;
      for (int w = 0; w < warps; ++w) s += buf[turn][k][w];
      v[k] = s;
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
template <class X, class R, int kV, int E>
__global__ void __launch_bounds__(kNormMaxThreads) norm_fwd_kernel(const NormArgs a) {
  constexpr int N = E / kV;
  __shared__ float buf[2][1][16];
  RowSum<1> row_sum(buf);
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

// One element's terms in the backward, from what a row keeps.
struct NormElem {
  float n, t, gu, m;   // r' rstd_pre, dr' + rstd_pre q, g u (without a token's gate), x rstd_post (or x)
};

// Backward.  As the forward's layout; a row's elements are read twice (the second
// time they are in L1 or L2), so that registers hold the sums over the rows.
template <class X, class R, int kV, int E>
__global__ void __launch_bounds__(kNormMaxThreads) norm_bwd_kernel(const NormArgs a) {
  constexpr int N = E / kV;
  __shared__ float buf[2][3][16];
  extern __shared__ __align__(16) float ysum[];   // [blockDim.y, H] where a block has several rows
  RowSum<3> row_sum(buf);
  const int H = a.H, G = blockDim.x;
  const float inv_H = 1.f / static_cast<float>(H);
  const bool channel = a.gate_kind == MOLT_GATE_CHANNEL;
  float dw_post[N][kV] = {}, dg[N][kV] = {}, dw_pre[N][kV] = {};
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y; t < a.T;
       t += static_cast<int64_t>(gridDim.x) * blockDim.y) {
    const X* x = static_cast<const X*>(a.x) + t * a.x_ld;
    const R* r = static_cast<const R*>(a.r) + t * a.r_ld;
    const X* dy = static_cast<const X*>(a.dy) + t * a.dy_ld;
    const R* dr = a.dr ? static_cast<const R*>(a.dr) + t * H : nullptr;
    const X* gate = static_cast<const X*>(a.gate) + t * H;   // where it is [T, H]
    const float rstd_pre = a.w_pre ? a.rstd_pre[t] : 0.f, rstd_post = a.w_post ? a.rstd_post[t] : 1.f;
    const float gt = a.gate_kind == MOLT_GATE_TOKEN ? static_cast<const float*>(a.gate)[t] : 1.f;
    float xv[kV], rv[kV], dyv[kV], drv[kV], wpo[kV], wpr[kV], gv[kV];
    auto read = [&](int c) {
      load_vec<kV>(x + c, xv);
#pragma unroll
      for (int j = 0; j < kV; ++j) {
        rv[j] = dyv[j] = drv[j] = wpr[j] = 0.f;
        wpo[j] = gv[j] = 1.f;
      }
      if (a.w_pre) {
        load_vec<kV>(r + c, rv);
        load_vec<kV>(dy + c, dyv);
        load_param<kV, X>(a.w_pre, a.param_f32, c, wpr);
#pragma unroll
        for (int j = 0; j < kV; ++j) wpr[j] += a.offset;
      }
      if (dr) load_vec<kV>(dr + c, drv);
      if (a.w_post) {
        load_param<kV, X>(a.w_post, a.param_f32, c, wpo);
#pragma unroll
        for (int j = 0; j < kV; ++j) wpo[j] += a.offset;
      }
      if (channel)
        load_param<kV, X>(a.gate, a.param_f32, c, gv);
      else if (a.gate_kind == MOLT_GATE_FULL)
        load_vec<kV>(gate + c, gv);
    };
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * G + threadIdx.x) * kV;
      if (c >= H) continue;
      read(c);
#pragma unroll
      for (int j = 0; j < kV; ++j) {
        const float n = rv[j] * rstd_pre, q = dyv[j] * wpr[j];
        const float gu = gv[j] * (xv[j] * rstd_post) * wpo[j];
        s[0] = fmaf(q, n, s[0]);
        s[1] = fmaf(gu, fmaf(rstd_pre, q, drv[j]), s[1]);
        s[2] = fmaf(gu, rstd_pre * n, s[2]);
      }
    }
    row_sum(s);
    const float mean_qn = s[0] * inv_H;
    const float gu_D = s[1] - mean_qn * s[2];     // sum of g u D, without a token's gate
    const float mean_pm = gt * gu_D * inv_H;
    if (a.gate_kind == MOLT_GATE_TOKEN && threadIdx.x == 0) static_cast<float*>(a.dgate)[t] = gu_D;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (i * G + threadIdx.x) * kV;
      if (c >= H) continue;
      read(c);
      float dx[kV], dro[kV], dgo[kV];
#pragma unroll
      for (int j = 0; j < kV; ++j) {
        const float n = rv[j] * rstd_pre, q = dyv[j] * wpr[j], m = xv[j] * rstd_post;
        const float D = fmaf(rstd_pre, q - n * mean_qn, drv[j]);
        const float Du = D * (m * wpo[j]), du = gt * gv[j] * D;
        dw_pre[i][j] = fmaf(dyv[j], n, dw_pre[i][j]);
        dw_post[i][j] = fmaf(du, m, dw_post[i][j]);
        if (channel) dg[i][j] += Du;
        dgo[j] = Du;
        dro[j] = a.alpha * D;
        dx[j] = a.w_post ? rstd_post * (du * wpo[j] - m * mean_pm) : du;
      }
      store_vec<kV>(static_cast<X*>(a.dx) + t * H + c, dx);
      if (a.dr_out) store_vec<kV>(static_cast<R*>(a.dr_out) + t * H + c, dro);
      if (a.gate_kind == MOLT_GATE_FULL) store_vec<kV>(static_cast<X*>(a.dgate) + t * H + c, dgo);
    }
  }
  // the block's sums: its rows' warps one after the other
  auto put = [&](int which, const float (&v)[N][kV]) {
    float* out = a.part + (static_cast<int64_t>(blockIdx.x) * 3 + which) * H;
    if (blockDim.y > 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int c = (i * G + threadIdx.x) * kV;
        if (c < H) store_vec<kV>(ysum + threadIdx.y * H + c, v[i]);
      }
      __syncthreads();
      for (int c = threadIdx.y * G + threadIdx.x; c < H; c += G * blockDim.y) {
        float sum = 0.f;
        for (int y = 0; y < static_cast<int>(blockDim.y); ++y) sum += ysum[y * H + c];
        out[c] = sum;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int c = (i * G + threadIdx.x) * kV;
        if (c < H) store_vec<kV>(out + c, v[i]);
      }
    }
  };
  if (a.w_post) put(0, dw_post);
  if (channel) put(1, dg);
  if (a.w_pre) put(2, dw_pre);
}

// Rows of more than kNormMaxH elements, or of any length: threads walk the columns and
// read the row again for every step of it (from L2).
template <class X, class R>
__global__ void __launch_bounds__(kNormMaxThreads) norm_fwd_long_kernel(const NormArgs a) {
  __shared__ float buf[2][1][16];
  RowSum<1> row_sum(buf);
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
  __shared__ float buf[2][3][16];
  RowSum<3> row_sum(buf);
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
// a thread (0: the kernels that loop over columns)
struct NormShape {
  int threads, rows, elems, vec;
};

template <class X, class R>
cudaError_t launch_norm_fwd_typed(const NormArgs& a, const NormShape& s, int grid, cudaStream_t stream) {
  const dim3 block(s.threads, s.rows);
  void (*k)(const NormArgs) = nullptr;
  if (s.elems == 0)
    k = norm_fwd_long_kernel<X, R>;
  else if (s.vec == 8)
    k = s.elems == 8 ? norm_fwd_kernel<X, R, 8, 8> : s.elems == 16 ? norm_fwd_kernel<X, R, 8, 16> : norm_fwd_kernel<X, R, 8, 32>;
  else
    k = s.elems == 8 ? norm_fwd_kernel<X, R, 1, 8> : s.elems == 16 ? norm_fwd_kernel<X, R, 1, 16> : norm_fwd_kernel<X, R, 1, 32>;
  k<<<grid, block, 0, stream>>>(a);
  return cudaGetLastError();
}

template <class X, class R>
cudaError_t launch_norm_bwd_typed(const NormArgs& a, const NormShape& s, int grid, cudaStream_t stream) {
  const dim3 block(s.threads, s.rows);
  void (*k)(const NormArgs) = nullptr;
  if (s.elems == 0)
    k = norm_bwd_long_kernel<X, R>;
  else if (s.vec == 8)
    k = s.elems == 8 ? norm_bwd_kernel<X, R, 8, 8> : s.elems == 16 ? norm_bwd_kernel<X, R, 8, 16> : norm_bwd_kernel<X, R, 8, 32>;
  else
    k = s.elems == 8 ? norm_bwd_kernel<X, R, 1, 8> : s.elems == 16 ? norm_bwd_kernel<X, R, 1, 16> : norm_bwd_kernel<X, R, 1, 32>;
  const size_t smem = s.rows > 1 ? static_cast<size_t>(s.rows) * a.H * sizeof(float) : 0;
  k<<<grid, block, smem, stream>>>(a);
  return cudaGetLastError();
}

// one translation unit per type of x (norm_*.cu)
cudaError_t launch_norm_bf16(const NormArgs& a, const NormShape& s, int grid, bool r_f32, bool bwd, cudaStream_t stream);
cudaError_t launch_norm_fp16(const NormArgs& a, const NormShape& s, int grid, bool r_f32, bool bwd, cudaStream_t stream);
cudaError_t launch_norm_fp32(const NormArgs& a, const NormShape& s, int grid, bool bwd, cudaStream_t stream);

}  // namespace molt
