// Softmax cross entropy over the LM head: the row kernels around the forward and the
// backward over chunks, which it shares with the policy loss.
//
//   l_t  = lse_t - (1 - e) z_t,x - e mean_v z_tv + c lse_t^2     (label smoothing e, z term c)
//   L    = sum_t w_t l_t / D,  D = denom, or the number of active rows
//   dL/dz_tv = (w_t / D) [ (1 + 2 c lse_t) p_tv - e / V - (1 - e) [v = x_t] ]
//
// The logits exist only as tiles on chip: lse, z_x and the sum of z come from the
// forward's epilogue, dL/dz from the backward's, where with e = c = 0 it is the policy
// loss's coef (p - [target]) and else kGradSmooth's.
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

// The rows whose target is not ignored, packed (see pack_rows): maps, hidden rows,
// targets and weights; zero hidden rows up to a whole K block of the dW product; also
// the call's zeroing.
__global__ void __launch_bounds__(kPackThreads) ce_pack_kernel(
    const int32_t* __restrict__ targets, const float* __restrict__ weight, int ignore, bool any_ignored, int T, int H,
    const uint16_t* __restrict__ hidden, int32_t* __restrict__ row_map, int32_t* __restrict__ pos,
    int32_t* __restrict__ counts, uint16_t* __restrict__ h_p, int32_t* __restrict__ tok_p, float* __restrict__ w_p,
    float* __restrict__ logp_out, float* __restrict__ lse_out, uint32_t* __restrict__ ctl, int ctl_words) {
  for (int i = blockIdx.x * kPackThreads + threadIdx.x; i < ctl_words; i += gridDim.x * kPackThreads) ctl[i] = 0u;
  const int share = (T + gridDim.x - 1) / gridDim.x;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * share;
  if (first >= T) return;
  const int t0 = static_cast<int>(first), t1 = min(T, t0 + share);
  const int before = any_ignored ? count_targets(targets, t0, ignore) : t0;
  const int total = pack_rows(
      t0, t1, before, H, hidden, h_p, [&](int t) { return !any_ignored || targets[t] != ignore; },
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

constexpr int kCeSums = 3;   // w l, -logp, lse^2

// One block per kRedRows packed rows: the row's lse, loss and backward values, and the
// rows' partial sums; the block that is done last adds all of them in a fixed order.
template <int kGroups, bool kSmooth>
__global__ void __launch_bounds__(kRedRows * kGroups) ce_merge_kernel(
    CeArgs a, int Tcap, int V, int n_parts, int32_t* __restrict__ counts, const int32_t* __restrict__ row_map,
    const int32_t* __restrict__ tok_p, const float* __restrict__ w_p, const float4* __restrict__ part,
    const float* __restrict__ zx, float* __restrict__ lse_o, float* __restrict__ coef_o, float* __restrict__ cp_o,
    float* __restrict__ cu_o, double* __restrict__ red, float* __restrict__ loss_out, float* __restrict__ logp_out,
    float* __restrict__ lse_out, molt_ce_stats* __restrict__ stats, unsigned* err) {
  const int n = counts[0];
  const int n_blocks = max(1, (n + kRedRows - 1) / kRedRows);
  if (static_cast<int>(blockIdx.x) >= n_blocks) return;
  const int k = blockIdx.x * kRedRows + threadIdx.x % kRedRows;
  const bool act = k < n;
  const RowStats st = merge_row_parts<kGroups, kSmooth>(part, Tcap, n_parts, k, act);
  const double D = a.denom > 0.0 ? a.denom : static_cast<double>(n);
  __shared__ bool last;
  if (threadIdx.x < kRedRows) {
    double s[kCeSums] = {0.0, 0.0, 0.0};
    if (act) {
      const float lse = st.M + logf(st.S);
      const int x = tok_p[k];
      const bool in = x >= 0 && x < V;   // else no loss and no gradient
      if (!in) atomicOr(err, kDevErrTokenRange);
      const float logp = in ? zx[k] - lse : 0.f;
      const float w = in ? (w_p ? w_p[k] : 1.f) : 0.f;
      float l = -logp;
      const float c = D > 0.0 ? static_cast<float>(static_cast<double>(w) / D) : 0.f;
      if constexpr (kSmooth) {
        // off: the mean over the vocabulary of -log p
        const float off = a.smoothing != 0.f ? lse - st.Q / static_cast<float>(V) : l;
        l = fmaf(a.z_loss * lse, lse, fmaf(a.smoothing, off - l, l));
        coef_o[k] = c * (1.f - a.smoothing);
        cp_o[k] = c * fmaf(2.f * a.z_loss, lse, 1.f);
        cu_o[k] = c * (a.smoothing / static_cast<float>(V));
      } else {
        coef_o[k] = c;
      }
      lse_o[k] = lse;
      const int t = row_map[k];
      if (logp_out) logp_out[t] = logp;
      if (lse_out) lse_out[t] = lse;
      if (in) {
        s[0] = static_cast<double>(w) * static_cast<double>(l);
        s[1] = -static_cast<double>(logp);
        s[2] = static_cast<double>(lse) * static_cast<double>(lse);
      }
    }
#pragma unroll
    for (int i = 0; i < kCeSums; ++i) s[i] = warp_sum<double>(s[i]);
    if (threadIdx.x == 0) {
#pragma unroll
      for (int i = 0; i < kCeSums; ++i) red[static_cast<int64_t>(blockIdx.x) * kRedSlots + i] = s[i];
      __threadfence();
      last = atomicAdd(counts + 5, 1) == n_blocks - 1;
    }
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  __shared__ double tot[kGroups][kCeSums];
  double s[kCeSums] = {0.0, 0.0, 0.0};
  for (int b = threadIdx.x; b < n_blocks; b += kRedRows * kGroups) {
#pragma unroll
    for (int i = 0; i < kCeSums; ++i) s[i] += __ldcg(red + static_cast<int64_t>(b) * kRedSlots + i);
  }
#pragma unroll
  for (int i = 0; i < kCeSums; ++i) s[i] = warp_sum<double>(s[i]);
  if (threadIdx.x % 32 == 0) {
#pragma unroll
    for (int i = 0; i < kCeSums; ++i) tot[threadIdx.x / 32][i] = s[i];
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int g = 1; g < kGroups; ++g) {
#pragma unroll
    for (int i = 0; i < kCeSums; ++i) s[i] += tot[g][i];
  }
  if (!(D > 0.0)) atomicOr(err, kDevErrZeroDenom);
  const double loss = D > 0.0 ? s[0] / D : 0.0;
  *loss_out = static_cast<float>(loss);
  if (stats) {
    stats->denom = D;
    stats->loss = loss;
    stats->sum_nll = s[1];
    stats->sum_lse_sq = s[2];
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

cudaError_t launch_ce_pack(const CeArgs& a, int T, int H, const uint16_t* hidden, const Workspace& ws, float* logp_out,
                           float* lse_out, int64_t ctl_words, int n_sm, cudaStream_t s) {
  // an ignore_index that no int32 can have ignores nothing
  const bool any = a.ignore_index >= INT32_MIN && a.ignore_index <= INT32_MAX;
  ce_pack_kernel<<<n_sm * 8, kPackThreads, 0, s>>>(a.targets, a.weight, any ? static_cast<int>(a.ignore_index) : 0, any, T, H,
                                                   hidden, ws.row_map, ws.pos_of_row, ws.counts, ws.h_p, ws.tok_p, ws.b_p,
                                                   logp_out, lse_out, ws.ctl, static_cast<int>(ctl_words));
  return cudaGetLastError();
}

cudaError_t launch_ce_merge(const CeArgs& a, bool smooth, int Tcap, int V, int n_parts, const Workspace& ws, float* loss_out,
                            float* logp_out, float* lse_out, molt_ce_stats* stats, unsigned* err, cudaStream_t s) {
  const int groups = merge_groups(n_parts);
  auto* k = groups == kMergeGroupsMany
                ? (smooth ? &ce_merge_kernel<kMergeGroupsMany, true> : &ce_merge_kernel<kMergeGroupsMany, false>)
                : (smooth ? &ce_merge_kernel<kMergeGroupsFew, true> : &ce_merge_kernel<kMergeGroupsFew, false>);
  k<<<Tcap / kRedRows, kRedRows * groups, 0, s>>>(a, Tcap, V, n_parts, ws.counts, ws.row_map, ws.tok_p,
                                                  a.weight ? ws.b_p : nullptr, ws.part, ws.zx, ws.lse, ws.coef, ws.ecoef, ws.mu,
                                                  ws.red, loss_out, logp_out, lse_out, stats, err);
  return cudaGetLastError();
}

cudaError_t launch_cast_bf16(const float* src, int64_t n, uint16_t* dst, int n_sm, cudaStream_t s) {
  cast_bf16_kernel<<<n_sm * 8, 256, 0, s>>>(src, n / 8, dst);
  return cudaGetLastError();
}

}  // namespace molt
