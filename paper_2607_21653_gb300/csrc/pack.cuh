// Packing of the rows that a call works on, shared by the row kernels.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

namespace molt {

// sums over a warp in a fixed tree
template <typename T>
__device__ __forceinline__ T warp_sum(T v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Order-preserving packing.  A grid of kPackThreads-thread blocks splits the rows
// evenly; each block counts the live rows before its own (a vectorised scan of the
// flags up to there, a few us at most: they sit in L2), so the count, the maps and
// the copies are one launch.  Before, one block compacted and a second kernel
// copied: 4 us more on the smallest call, 13 of 46 at T = 32768.
constexpr int kPackThreads = 256;

__device__ __forceinline__ int block_sum(int v) {
  __shared__ int ws[kPackThreads / 32];
  v = __reduce_add_sync(0xffffffffu, v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) ws[threadIdx.x >> 5] = v;
  __syncthreads();
  int t = 0;
#pragma unroll
  for (int i = 0; i < kPackThreads / 32; ++i) t += ws[i];
  return t;
}

// nonzero bytes of m[0, n), by the whole block
__device__ __forceinline__ int count_bytes(const uint8_t* __restrict__ m, int n) {
  const int head = min(n, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(m) & 15)) & 15));
  const int nvec = (n - head) / 16;
  const uint4* v = reinterpret_cast<const uint4*>(m + head);
  auto word = [](uint32_t w) { return __popc((((w & 0x7f7f7f7fu) + 0x7f7f7f7fu) | w) & 0x80808080u); };
  int c = 0;
  for (int i = threadIdx.x; i < head; i += kPackThreads) c += m[i] ? 1 : 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < nvec; i += kPackThreads) {
    const uint4 x = v[i];
    c += word(x.x) + word(x.y) + word(x.z) + word(x.w);
  }
  for (int i = head + 16 * nvec + threadIdx.x; i < n; i += kPackThreads) c += m[i] ? 1 : 0;
  return block_sum(c);
}

// The block's share of rows [0, n), 256 at a time: row(k, live, j) for every row k
// (j its index among the live ones, `before` of which precede the share), then the
// live rows' hidden rows copied from src row k to dst row j (src nullptr: none).
// Returns the number of live rows up to the end of the share.
template <class Live, class Row>
__device__ __forceinline__ int pack_rows(int k0, int k1, int before, int H, const uint16_t* __restrict__ src,
                                         uint16_t* __restrict__ dst, Live live_of_row, Row row) {
  __shared__ int wsum[kPackThreads / 32];
  __shared__ int list[kPackThreads];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int vpr = H / 8;   // 16-byte vectors per row
  for (int base = k0; base < k1; base += kPackThreads) {
    const int k = base + threadIdx.x;
    const bool live = k < k1 && live_of_row(k);
    const unsigned m = __ballot_sync(0xffffffffu, live);
    __syncthreads();
    if (lane == 0) wsum[w] = __popc(m);
    __syncthreads();
    int pre = 0, cnt = 0;
#pragma unroll
    for (int i = 0; i < kPackThreads / 32; ++i) {
      pre += i < w ? wsum[i] : 0;
      cnt += wsum[i];
    }
    const int j = pre + __popc(m & ((1u << lane) - 1u));
    if (live) list[j] = k;
    if (k < k1) row(k, live, before + j);
    __syncthreads();
    if (src != nullptr) {
#pragma unroll 4
      for (int i = threadIdx.x; i < cnt * vpr; i += kPackThreads) {
        const int q = i / vpr, v = i - q * vpr;
        reinterpret_cast<uint4*>(dst + static_cast<int64_t>(before + q) * H)[v] =
            reinterpret_cast<const uint4*>(src + static_cast<int64_t>(list[q]) * H)[v];
      }
    }
    before += cnt;
  }
  return before;
}

}  // namespace molt
