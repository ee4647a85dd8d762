// Gated feed-forward block for a few tokens (decoding): h = act(x Wg^T) (x Wu^T), y = h Wd^T
// with at most 16 rows in x.
//
// 2 T flops to a weight of two bytes: the weights' way from HBM bounds it, so they are
// streamed once from global memory into registers, 16 bytes to a lane and row, with no stage
// between.  Both operands of a product may have their K in any order as long as it is the
// same one, so a lane's eight neighbouring elements of a row serve as its parts of two
// m16n8k16 fragments: lane 4 g + c has k = 8 c .. 8 c + 7 of a step of 32 of rows g and g + 8
// (weights: the 16 rows of the product) and of row g of x (its 8 columns).  tcgen05 would
// need the weights in shared memory and 128 rows to a tile, to win nothing: the tensor cores
// are idle nine tenths of the time either way.  In the first product the 16 rows are eight of
// Wg and the same eight of Wu, so that a lane ends with g and u of the same elements.
//
// A block's warps share its 16 rows and divide K; their sums are added in order.  The second product's
// launch may begin while the first one's last blocks run: its first weights are on their way
// before it waits for h.
// T = 1, H = 4096, F = 10944, bf16: 45 us, 5.9 TB/s of 6.8 (51 where the second launch begins after
// the first).
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <type_traits>

#include "ffn.cuh"
#include "ffn_act.cuh"
#include "molt_internal.cuh"
#include "ptx.cuh"
#include "vec.cuh"

namespace molt {
namespace {

constexpr int kUnroll = 4;     // steps of 32 in flight: 4 KB of weights to a warp

__device__ __forceinline__ uint4 load_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1, const __nv_bfloat16*) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1, const __half*) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// kTiles: eight tokens each.  kGlu: the first product, w0 and w1 are Wg and Wu; else w0 is Wd.
template <class T, int kTiles, bool kGlu, int kWarps>
__global__ void __launch_bounds__(32 * kWarps, (!kGlu && kWarps == 16 ? 2 : 0)) ffn_rows_kernel(const FfnRows a) {
  __shared__ float4 part[kWarps - 1][kTiles][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
  const int r0 = blockIdx.x * (kGlu ? 8 : 16);
  const T* const x = static_cast<const T*>(a.x);
  // rows g and g + 8 of the product (n is a multiple of 8: the second eight may be missing)
  const int ra = r0 + g, rb = kGlu ? r0 + g : min(r0 + 8 + g, a.n - 1);
  const T* const wa = static_cast<const T*>(a.w0) + static_cast<int64_t>(ra) * a.w0_ld;
  const T* const wb = kGlu ? static_cast<const T*>(a.w1) + static_cast<int64_t>(rb) * a.w1_ld
                           : static_cast<const T*>(a.w0) + static_cast<int64_t>(rb) * a.w0_ld;
  float acc[kTiles][4] = {};
  if constexpr (kGlu) asm volatile("griddepcontrol.launch_dependents;");
  bool waiting = !kGlu;
  auto wait_for_x = [&]() {   // x of the second product is what the launch before has written
    if (!waiting) return;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    waiting = false;
  };
  auto load_x = [](const T* p) {   // (so not as read-only data)
    const uint4* const q = reinterpret_cast<const uint4*>(p);
    return kGlu ? __ldg(q) : __ldcg(q);
  };
  // this warp's steps of 32
  const int steps = (a.k + 31) / 32, s0 = steps * warp / kWarps, s1 = steps * (warp + 1) / kWarps;
  const uint4 none = make_uint4(0, 0, 0, 0);
  auto work = [&](int s, auto checked) {
    uint4 wa4[kUnroll], wb4[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      const int k = (s + i) * 32 + c * 8;
      const bool in = !decltype(checked)::value || (s + i < s1 && k < a.k);
      wa4[i] = in ? load_stream(wa + k) : none;
      wb4[i] = in ? load_stream(wb + k) : none;
    }
    wait_for_x();
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      const int k = (s + i) * 32 + c * 8;
      const bool in = !decltype(checked)::value || (s + i < s1 && k < a.k);
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const int row = t * 8 + g;
        const uint4 xv = in && row < a.t ? load_x(x + static_cast<int64_t>(row) * a.x_ld + k) : none;
        mma16816(acc[t], wa4[i].x, wb4[i].x, wa4[i].y, wb4[i].y, xv.x, xv.y, x);
        mma16816(acc[t], wa4[i].z, wb4[i].z, wa4[i].w, wb4[i].w, xv.z, xv.w, x);
      }
    }
  };
  int s = s0;
  // whole steps only: the last may reach past k
  for (; s + kUnroll <= s1 && (s + kUnroll) * 32 <= a.k; s += kUnroll) work(s, std::false_type{});
  for (; s < s1; s += kUnroll) work(s, std::true_type{});
  wait_for_x();
  if (warp > 0) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) part[warp - 1][t][lane] = make_float4(acc[t][0], acc[t][1], acc[t][2], acc[t][3]);
  }
  __syncthreads();
  if (warp > 0) return;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
#pragma unroll
    for (int w = 0; w < kWarps - 1; ++w) {
      const float4 p = part[w][t][lane];
      acc[t][0] += p.x;
      acc[t][1] += p.y;
      acc[t][2] += p.z;
      acc[t][3] += p.w;
    }
    // elements (row g, tokens 2 c and 2 c + 1), then row g + 8
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int token = t * 8 + 2 * c + j;
      if (token >= a.t) continue;
      const int64_t at = static_cast<int64_t>(token) * a.n + r0 + g;
      if constexpr (kGlu) {
        with_activation(a.act, [&](auto act) {
          float unused;
          from_float(ffn_activate<decltype(act)::value, false>(acc[t][j], unused) * acc[t][2 + j], static_cast<T*>(a.out[0])[at]);
        });
        if (a.out[1] != nullptr) {
          from_float(acc[t][j], static_cast<T*>(a.out[1])[at]);
          from_float(acc[t][2 + j], static_cast<T*>(a.out[2])[at]);
        }
      } else {
        from_float(acc[t][j], static_cast<T*>(a.out[0])[at]);
        if (r0 + 8 + g < a.n) from_float(acc[t][2 + j], static_cast<T*>(a.out[0])[at + 8]);
      }
    }
  }
}

// Eight warps to a block, or sixteen where the SMs would otherwise hold fewer than sixteen
// each (the second product at H = 4096, F = 10944: 256 blocks, 27 us with eight).
template <class T, int kTiles, bool kGlu>
cudaError_t launch(const FfnRows& r, int n_sm, cudaStream_t s) {
  const int blocks = kGlu ? r.n / 8 : (r.n + 15) / 16;
  const bool many = blocks >= 2 * n_sm;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(many ? 256 : 512);
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = kGlu ? 0 : 1;
  return cudaLaunchKernelEx(&cfg, many ? ffn_rows_kernel<T, kTiles, kGlu, 8> : ffn_rows_kernel<T, kTiles, kGlu, 16>, r);
}
template <class T, int kTiles>
cudaError_t launch(const FfnRows& r, bool glu, int n_sm, cudaStream_t s) {
  return glu ? launch<T, kTiles, true>(r, n_sm, s) : launch<T, kTiles, false>(r, n_sm, s);
}

}  // namespace

cudaError_t launch_ffn_rows(const FfnRows& r, bool glu, bool fp16, cudaStream_t s) {
  const int n_sm = device_sm_count();
  if (r.t <= 8)
    return fp16 ? launch<__half, 1>(r, glu, n_sm, s) : launch<__nv_bfloat16, 1>(r, glu, n_sm, s);
  return fp16 ? launch<__half, 2>(r, glu, n_sm, s) : launch<__nv_bfloat16, 2>(r, glu, n_sm, s);
}

}  // namespace molt
