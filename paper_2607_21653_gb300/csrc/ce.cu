// Softmax cross entropy over the LM head: the row kernels around the forward and the
// backward over chunks, which it shares with the policy loss.
//
//   l_t  = lse_t - (1 - e) z_t,x - e mean_v z_tv + c lse_t^2     (label smoothing e, z term c)
//   L    = sum_t w_t l_t / D,  D = denom, or the number of active rows
//   dL/dz_tv = (w_t / D) [ (1 + 2 c lse_t) p_tv - e / V - (1 - e) [v = x_t] ]
//
// lse, z_x and the sum of z come from the forward's epilogue on tiles of logits on chip,
// dL/dz from the backward's (kGradScaled), which forms the tiles again, or from H = 640 on
// reads what the forward's epilogue kept of them in 16 bits (kKeepTile).
//
// Two things make it more exact than its products.  The tensor cores add in fp32 but cut
// off what does not fit, 256 times at H = 4096: the target's logit, which often is by far
// the largest, comes out 1e-6 too small.  So its logit is formed again in fp32, here
// where the rows are packed, and replaces the product's in the row's sum and in the
// gradient: the target's entry of dL/dz is finished where the rows are merged, from what
// the row's other columns sum to, and the backward's tiles take it as it is (see finish_row).
// And the gradient is rounded to bf16 without the factor 1 / D: a target that the model
// does not expect then is -1, which bf16 holds exactly, where -1 / D would be off by up to
// 0.4 % for all of them alike; the factor multiplies the products' sums.  (Relative errors
// of logp and of dW before: 1.6e-6 and up to 2.9e-3.)
#include <climits>
#include <cstdint>
#include <cuda_runtime.h>

#include "merge.cuh"
#include "molt_internal.cuh"
#include "pack.cuh"
#include "ptx.cuh"

namespace molt {
namespace {

// values of x[0, n) other than `ignore`, by the whole block
__device__ __forceinline__ int count_targets(const int32_t* __restrict__ x, int n, int ignore) {
  const int head = min(n, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / 4);
  const int nvec = (n - head) / 4;
  const int4* v = reinterpret_cast<const int4*>(x + head);
  int c = 0;
  if (static_cast<int>(threadIdx.x) < head) c += x[threadIdx.x] != ignore;
#pragma unroll 4
  for (int i = threadIdx.x; i < nvec; i += kPackThreads) {
    const int4 q = v[i];
    c += (q.x != ignore) + (q.y != ignore) + (q.z != ignore) + (q.w != ignore);
  }
  for (int i = head + 4 * nvec + threadIdx.x; i < n; i += kPackThreads) c += x[i] != ignore;
  return block_sum(c);
}

// Copies a row's vectors i0, i0 + step, ... and sums h w over them, by a warp, in fp32
// throughout.
__device__ __forceinline__ float copy_dot(const uint16_t* __restrict__ h, const uint16_t* __restrict__ w, uint16_t* __restrict__ to,
                                          int H, int i0, int step) {
  const uint4 *a = reinterpret_cast<const uint4*>(h), *b = reinterpret_cast<const uint4*>(w);
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = i0; i < H / 8; i += step) {
    const uint4 x = __ldg(a + i), y = __ldg(b + i);
    reinterpret_cast<uint4*>(to)[i] = x;
    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[j] = fmaf(__uint_as_float(xs[j] << 16), __uint_as_float(ys[j] << 16), s[j]);
      s[j] = fmaf(__uint_as_float(xs[j] & 0xffff0000u), __uint_as_float(ys[j] & 0xffff0000u), s[j]);
    }
  }
  return warp_sum((s[0] + s[1]) + (s[2] + s[3]));
}

// The rows whose target is not ignored, packed (see pack_rows): maps, hidden rows,
// targets, weights and the targets' logits; zero hidden rows up to a whole K block of the
// dW product; also the call's zeroing.
__global__ void __launch_bounds__(kPackThreads) ce_pack_kernel(
    const int32_t* __restrict__ targets, const float* __restrict__ weight, int ignore, bool any_ignored, int T, int H, int V,
    const uint16_t* __restrict__ hidden, const uint16_t* __restrict__ W, int32_t* __restrict__ row_map,
    int32_t* __restrict__ pos, int32_t* __restrict__ counts, uint16_t* __restrict__ h_p, int32_t* __restrict__ tok_p,
    float* __restrict__ w_p, float* __restrict__ z_p, float* __restrict__ logp_out, float* __restrict__ lse_out,
    uint32_t* __restrict__ ctl, int ctl_words) {
  for (int i = blockIdx.x * kPackThreads + threadIdx.x; i < ctl_words; i += gridDim.x * kPackThreads) ctl[i] = 0u;
  const int share = (T + gridDim.x - 1) / gridDim.x;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * share;
  if (first >= T) return;
  const int t0 = static_cast<int>(first), t1 = min(T, t0 + share);
  const int before = any_ignored ? count_targets(targets, t0, ignore) : t0;
  const int total = pack_rows(
      t0, t1, before, H, nullptr, nullptr, [&](int t) { return !any_ignored || targets[t] != ignore; },
      [&](int t, bool live, int k) {
        pos[t] = live ? k : -1;
        if (live) {
          row_map[k] = t;
          tok_p[k] = targets[t];
          if (weight) w_p[k] = weight[t];
        } else {
          if (logp_out) logp_out[t] = 0.f;
          if (lse_out) lse_out[t] = 0.f;
        }
      });
  __syncthreads();
  // Copies and dots in one pass (with rows copied first 4 us more at T = 12974, H = 2560): a
  // warp to a row, or where the block has fewer rows than warps, several (T = 100, H = 4096
  // 2 us less).
  constexpr int kWarps = kPackThreads / 32;
  __shared__ float part[kWarps];
  const int cnt = total - before, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int per_row = cnt <= 1 ? 8 : cnt == 2 ? 4 : cnt <= 4 ? 2 : 1, of_row = warp % per_row;
  for (int i = warp / per_row; i < cnt; i += kWarps / per_row) {
    const int k = before + i, x = tok_p[k];
    const uint16_t* src = hidden + static_cast<int64_t>(row_map[k]) * H;
    // a target outside [0, V): the merge leaves the row out
    const float z = copy_dot(src, x >= 0 && x < V ? W + static_cast<int64_t>(x) * H : src, h_p + static_cast<int64_t>(k) * H, H,
                             of_row * 32 + lane, per_row * 32);
    if (lane == 0) {
      if (per_row == 1)
        z_p[k] = z;
      else
        part[warp] = z;   // the only row of the warp
    }
  }
  if (per_row > 1) {
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < cnt) {
      float z = 0.f;
      for (int i = 0; i < per_row; ++i) z += part[threadIdx.x * per_row + i];
      z_p[before + threadIdx.x] = z;
    }
  }
  if (t1 != T) return;
  if (threadIdx.x == 0) {
    counts[0] = total;
    counts[3] = total;
    counts[4] = 0;
    counts[5] = 0;
  }
  const int64_t v0 = static_cast<int64_t>(total) * (H / 8), v1 = (static_cast<int64_t>(total) + kBK - 1) / kBK * kBK * (H / 8);
#pragma unroll 4
  for (int64_t v = v0 + threadIdx.x; v < v1; v += kPackThreads) reinterpret_cast<uint4*>(h_p)[v] = make_uint4(0, 0, 0, 0);
}

// A sum as two floats, good to about 48 bits.  FP64 runs at a 64th of the rate here: an
// addition takes a warp 60 clocks, and the merge kernel's sums in it took half of its time
// (16200 clocks at T = 512, of which the last block's 7400).
struct Sum2 {
  float h = 0.f, l = 0.f;
  __device__ __forceinline__ void add(float bh, float bl) {
    const float s = h + bh, b = s - h;
    float e = (h - (s - b)) + (bh - b) + (l + bl);
    if (!(fabsf(s) < INFINITY)) e = 0.f;   // infinities stay what they are
    h = s + e;
    l = e - (h - s);
    if (!(fabsf(h) < INFINITY)) l = 0.f;
  }
  __device__ __forceinline__ void add(Sum2 o) { add(o.h, o.l); }
  // a product, whole
  static __device__ __forceinline__ Sum2 product(float a, float b) {
    Sum2 p;
    p.h = a * b;
    p.l = fabsf(p.h) < INFINITY ? fmaf(a, b, -p.h) : 0.f;
    return p;
  }
  __device__ __forceinline__ void warp_sum() {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float oh = __shfl_xor_sync(0xffffffffu, h, o), ol = __shfl_xor_sync(0xffffffffu, l, o);
      add(oh, ol);
    }
  }
  __device__ __forceinline__ double value() const { return static_cast<double>(h) + static_cast<double>(l); }
};

constexpr int kCeSums = 3;   // w l, -logp, lse^2
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A row's splits merged by kGroups threads: thread (r, g) = (t % kRows, t / kRows) takes
// every kGroups-th, eight loads at a time.  Valid in group 0; every thread calls it.
template <int kRows, int kGroups, bool kSumZ>
__device__ __forceinline__ RowStats merge_row(const float4* __restrict__ part, int64_t stride, int n_parts, int k, bool act) {
  __shared__ float4 sh[kGroups][kRows];
  const int r = threadIdx.x % kRows, g = threadIdx.x / kRows;
  RowStats st{-INFINITY, 0.f, 0.f};
  auto add = [&](float m, float s, float q) {
    if (s == 0.f) return;   // no columns.  A NaN passes
    const float M = fmaxf(st.M, m);
    const float f0 = st.S == 0.f ? 0.f : ex2_approx((st.M - M) * kLog2e), f1 = ex2_approx((m - M) * kLog2e);
    st.S = st.S * f0 + s * f1;
    if (kSumZ) st.Q += q;
    st.M = M;
  };
  for (int s0 = g; act && s0 < n_parts; s0 += 8 * kGroups) {
    float4 p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int s = s0 + i * kGroups;
      p[i] = s < n_parts ? part[s * stride + k] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // The forward's exponentials are 2^(z log2e - mL) with mL = m log2e rounded to fp32: all
      // of them 2^rho too large, rho up to 1e-6 at m = 20, which is a loss of 1e-6 too much or
      // too little.  s takes 2^-rho = 1 - a + a^2 / 2 (rho is small wherever logits mean
      // anything).
      const float rho = fmaf(p[i].x, kLog2e, -__fmul_rn(p[i].x, kLog2e));
      const float a = kLn2 * fminf(fmaxf(rho, -0.01f), 0.01f);
      add(p[i].x, fmaf(p[i].y, a * fmaf(0.5f, a, -1.f), p[i].y), p[i].z);
    }
  }
  // groups in pairs, halves of the rest at a time
#pragma unroll
  for (int half = kGroups / 2; half > 0; half /= 2) {
    if (g >= half && g < 2 * half) sh[g][r] = make_float4(st.M, st.S, st.Q, 0.f);
    __syncthreads();
    if (g < half) {
      const float4 o = sh[g + half][r];
      add(o.x, o.y, o.z);
    }
  }
  return st;
}

// A row's lse and log p of its target, whose logit is z where the products had z_mma:
// with R the others' sum over e^z, log p = -log(1 + R), without lse's rounding (2^-20 at
// z = 20, which is all of the loss of a row that the model predicts that well) and without a
// difference of logits.  What R is off by is the sum's rounding and that of the
// exponentials, a few 2^-24.
struct RowEnd {
  float lse, logp;
};
__device__ __forceinline__ RowEnd finish_row(const RowStats& st, float z, float z_mma) {
  float rest = st.S - ex2_approx((z_mma - st.M) * kLog2e);
  if (rest < 0.f) rest = 0.f;   // (rounding.  A NaN passes)
  if (z > st.M - 1.f) {
    const float l = log1pf(rest * ex2_approx((st.M - z) * kLog2e));
    return {z + l, -l};
  }
  const float d = z - st.M, l = logf(rest + ex2_approx(d * kLog2e));
  return {st.M + l, d - l};
}

// One block per kRows packed rows: the rows' lse, losses and backward values, and their
// partial sums; the block that is done last adds all of them in a fixed order.
template <int kRows, int kGroups, bool kSmooth>
__global__ void __launch_bounds__(kRows* kGroups) ce_merge_kernel(
    CeArgs a, int T, int Tcap, int V, int n_parts, int32_t* __restrict__ counts, const int32_t* __restrict__ row_map,
    const int32_t* __restrict__ tok_p, const float* __restrict__ w_p, const float4* __restrict__ part,
    const float* __restrict__ zx, const float* __restrict__ z_p, float* __restrict__ lse_o, float* __restrict__ target_o,
    float* __restrict__ cp_o, float* __restrict__ cu_o, float2* __restrict__ red, float* __restrict__ scale_out,
    float* __restrict__ loss_out, float* __restrict__ logp_out, float* __restrict__ lse_out,
    molt_ce_stats* __restrict__ stats, unsigned* err) {
  static_assert(kRows <= 32, "a row's lane in the first warp");
  const int k = blockIdx.x * kRows + threadIdx.x % kRows;
  // the row's other values beside the count and the splits (a row past the count: any value)
  const bool lead = threadIdx.x < kRows && k < Tcap;
  const int n = counts[0];
  const int x = lead ? tok_p[k] : 0, t = lead ? row_map[min(k, T - 1)] : 0;
  const float z_mma = lead ? zx[k] : 0.f, z_row = lead ? z_p[k] : 0.f, w_row = lead && w_p ? w_p[k] : 1.f;
  const int n_blocks = max(1, (n + kRows - 1) / kRows);
  if (static_cast<int>(blockIdx.x) >= n_blocks) return;
  const bool act = k < n;
  const RowStats st = merge_row<kRows, kGroups, kSmooth>(part, Tcap, n_parts, k, act);
  __shared__ bool last;
  if (threadIdx.x < 32) {
    Sum2 s[kCeSums];
    if (act && threadIdx.x < kRows) {
      const bool in = x >= 0 && x < V;   // else no loss and no gradient
      if (!in) atomicOr(err, kDevErrTokenRange);
      // (no target: the sum as it is)
      const RowEnd end = in ? finish_row(st, z_row, z_mma) : RowEnd{st.M + logf(st.S), 0.f};
      const float lse = end.lse, logp = end.logp;
      const float w = in ? w_row : 0.f;
      float l = -logp, minus = expm1f(logp);   // minus: p - 1
      if constexpr (kSmooth) {
        // off: the mean over the vocabulary of -log p
        const float off = a.smoothing != 0.f ? lse - st.Q / static_cast<float>(V) : l;
        l = fmaf(a.z_loss * lse, lse, fmaf(a.smoothing, off - l, l));
        const float e_V = a.smoothing / static_cast<float>(V), zl = 2.f * a.z_loss;
        minus += fmaf(zl * lse, 1.f + minus, a.smoothing - e_V);
        cp_o[k] = w * fmaf(zl, lse, 1.f);
        cu_o[k] = w * e_V;
      } else {
        cp_o[k] = w;
        cu_o[k] = 0.f;
      }
      target_o[k] = w * minus;
      lse_o[k] = lse;
      if (logp_out) logp_out[t] = logp;
      if (lse_out) lse_out[t] = lse;
      if (in) {
        s[0] = Sum2::product(w, l);
        s[1].h = -logp;
        s[2] = Sum2::product(lse, lse);
      }
    }
#pragma unroll
    for (int i = 0; i < kCeSums; ++i) s[i].warp_sum();
    if (threadIdx.x == 0) {
#pragma unroll
      for (int i = 0; i < kCeSums; ++i) red[static_cast<int64_t>(blockIdx.x) * kRedSlots + i] = make_float2(s[i].h, s[i].l);
      __threadfence();
      last = atomicAdd(counts + 5, 1) == n_blocks - 1;
    }
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  constexpr int kWarps = kRows * kGroups / 32;
  __shared__ float2 tot[kWarps][kCeSums];
  Sum2 s[kCeSums];
  for (int b = threadIdx.x; b < n_blocks; b += kRows * kGroups) {
#pragma unroll
    for (int i = 0; i < kCeSums; ++i) {
      const float2 v = __ldcg(red + static_cast<int64_t>(b) * kRedSlots + i);
      s[i].add(v.x, v.y);
    }
  }
  // (warps without a block have nothing to add)
  const int warps = min(kWarps, (n_blocks + 31) / 32);
  if (static_cast<int>(threadIdx.x) / 32 < warps) {
#pragma unroll
    for (int i = 0; i < kCeSums; ++i) {
      s[i].warp_sum();
      if (threadIdx.x % 32 == 0) tot[threadIdx.x / 32][i] = make_float2(s[i].h, s[i].l);
    }
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int g = 1; g < warps; ++g) {
#pragma unroll
    for (int i = 0; i < kCeSums; ++i) s[i].add(tot[g][i].x, tot[g][i].y);
  }
  const double D = a.denom > 0.0 ? a.denom : static_cast<double>(n);
  if (!(D > 0.0)) atomicOr(err, kDevErrZeroDenom);
  const double inv_D = D > 0.0 ? 1.0 / D : 0.0, loss = D > 0.0 ? s[0].value() * inv_D : 0.0;
  *loss_out = static_cast<float>(loss);
  *scale_out = static_cast<float>(inv_D);
  if (stats) {
    stats->denom = D;
    stats->loss = loss;
    stats->sum_nll = s[1].value();
    stats->sum_lse_sq = s[2].value();
    stats->n_active = n;
  }
}

__global__ void __launch_bounds__(256) cast_bf16_kernel(const float* __restrict__ src, int64_t n8, uint16_t* __restrict__ dst) {
  for (int64_t i = blockIdx.x * static_cast<int64_t>(256) + threadIdx.x; i < n8; i += static_cast<int64_t>(gridDim.x) * 256) {
    const float4 a = reinterpret_cast<const float4*>(src)[2 * i], b = reinterpret_cast<const float4*>(src)[2 * i + 1];
    reinterpret_cast<uint4*>(dst)[i] =
        make_uint4(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w), pack_bf16x2(b.x, b.y), pack_bf16x2(b.z, b.w));
  }
}

}  // namespace

cudaError_t launch_ce_pack(const CeArgs& a, int T, int H, int V, const uint16_t* hidden, const uint16_t* W, const Workspace& ws,
                           float* logp_out, float* lse_out, int64_t ctl_words, int n_sm, cudaStream_t s) {
  // an ignore_index that no int32 can have ignores nothing
  const bool any = a.ignore_index >= INT32_MIN && a.ignore_index <= INT32_MAX;
  ce_pack_kernel<<<n_sm * 8, kPackThreads, 0, s>>>(a.targets, a.weight, any ? static_cast<int>(a.ignore_index) : 0, any, T, H, V,
                                                   hidden, W, ws.row_map, ws.pos_of_row, ws.counts, ws.h_p, ws.tok_p, ws.b_p,
                                                   ws.adv_p, logp_out, lse_out, ws.ctl, static_cast<int>(ctl_words));
  return cudaGetLastError();
}

cudaError_t launch_ce_merge(const CeArgs& a, bool smooth, int T, int Tcap, int V, int n_parts, const Workspace& ws, float* loss_out,
                            float* logp_out, float* lse_out, molt_ce_stats* stats, unsigned* err, cudaStream_t s) {
  // few rows have many splits each: eight rows and 64 groups of threads to a block (T =
  // 100 with 594 splits: 32 rows to a block, the splits read twice, took 24 us)
  const bool few = n_parts > 64;
  auto* k = few ? (smooth ? &ce_merge_kernel<8, 64, true> : &ce_merge_kernel<8, 64, false>)
                : (smooth ? &ce_merge_kernel<32, 8, true> : &ce_merge_kernel<32, 8, false>);
  const int rows = few ? 8 : 32;
  k<<<(T + rows - 1) / rows, few ? 512 : 256, 0, s>>>(a, T, Tcap, V, n_parts, ws.counts, ws.row_map, ws.tok_p,
                                                      a.weight ? ws.b_p : nullptr, ws.part, ws.zx, ws.adv_p, ws.lse, ws.coef,
                                                      ws.ecoef, ws.mu, reinterpret_cast<float2*>(ws.red), ws.scale, loss_out, logp_out, lse_out, stats, err);
  return cudaGetLastError();
}

cudaError_t launch_cast_bf16(const float* src, int64_t n, uint16_t* dst, int n_sm, cudaStream_t s) {
  cast_bf16_kernel<<<n_sm * 8, 256, 0, s>>>(src, n / 8, dst);
  return cudaGetLastError();
}

}  // namespace molt
