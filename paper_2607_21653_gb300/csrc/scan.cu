// Gated linear recurrence over packed sequences, forward, backward and one step.
//
//   sigmoid form   h_t = a_t h_{t-1} + (1 - a_t) v_t,  a_t = 1 / (1 + e^-f_t)
//   log form       h_t = a_t h_{t-1} + v_t,            a_t = e^f_t
//   backward, D_t the gradient of h_t:   D_t = dy_t + E_{t+1},   E_t = a_t D_t
//     sigmoid   df_t = D_t (h_{t-1} - v_t) a_t (1 - a_t),  dv_t = D_t (1 - a_t)
//     log       df_t = D_t h_{t-1} a_t,                    dv_t = D_t
// E past a sequence's last row is the gradient of its final state, E of its first row that
// of its initial one.
//
// What a row does to h is an affine map (a, b), and maps compose, so rows can be taken
// together: a tile is 128 rows by 64 channels, a warp has 16 rows of it, a lane two channels.
// Every warp composes its rows' maps; the maps of a tile's warps, and of the tiles of a
// cluster, are folded in order; and then every warp goes through its rows again from the
// state that it now knows.  The backward's E is the same from the other end; h it forms
// again from the states that the forward kept at every 128th row.  A row that begins a
// sequence cuts: what comes before is not multiplied by zero but left out, so that an
// infinite or NaN state stays in its sequence.
//
// Everything is held as m = a - 1: with a as a float near 1 the memory 1 / (1 - a) of a
// channel would be off by 2^-24 / (1 - a); h + m (h - v) and h + m h + v need no a at all.
//
// Layout: a strip of channels belongs to a cluster of up to eight blocks, which take a
// tile each, exchange their maps through one another's shared memory (512 bytes to each
// peer) and go on together, so that the inputs are read once and a super step of 1024 rows
// costs one exchange.  Of two further warps one brings the tiles ahead (TMA, and from
// cu_seqlens which rows begin and end a sequence), the other folds the maps.  Few strips and many rows are cut into segments besides: a first
// launch folds each segment's map, the second starts from what precedes its own.
#include <algorithm>
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>
#include <initializer_list>

#include "molt_internal.cuh"
#include "ptx.cuh"
#include "vec.cuh"

namespace molt {
namespace {

constexpr int kTile = 128;               // rows of a tile, and between kept states
constexpr int kWarps = 8, kRows = kTile / kWarps;
constexpr int kThreads = 32 * (kWarps + 2);
constexpr int kStrip = 64;               // channels of a block
constexpr int kMaxCluster = 8;           // 4 where tiles do not come by TMA (shared memory for two blocks to an SM)
constexpr int kFormSigmoid = 0, kFormLog = 1;
constexpr float kLog2e = 1.4426950408889634f;

struct ScanArgs {
  const void *gate, *value, *dy;
  int64_t gate_ld, value_ld, dy_ld;
  const float* h0;         // [B, H] or nullptr
  const float* dfinal;     // [B, H] or nullptr
  const int32_t* cu;       // [B + 1] or nullptr: B sequences of L rows
  int64_t T;
  int H, L;
  int64_t B;
  void* y;                 // forward
  int fill;                // rows outside of every sequence get zeros
  float* final_state;      // [B, H] or nullptr
  float* states;           // [tiles, H], written by the forward (or nullptr), read by the backward
  void *dgate, *dvalue;    // backward
  float* dinit;            // [B, H] or nullptr
  int tiles, seg_tiles;    // tiles in all, and of a segment
  float4* seg_maps;        // [segments, strips, 32]: (A, b) of two channels, A < 0: cut
  unsigned* err;
};
struct ScanMaps {
  CUtensorMap gate, value, dy;   // boxes of 64 channels by 128 rows
  CUtensorMap out0, out1;        // y, or dgate and dvalue: boxes of 64 channels by 16 rows
};

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ F2 zero2() { return f2(0.f, 0.f); }
__device__ __forceinline__ F2 sub2(F2 a, F2 b) { return fma2(b, f2(-1.f), a); }

// m = a - 1 of two gates.  sigmoid: -1 / (1 + e^f), no digits lost on either side.  log: e^f - 1,
// by its series where the difference would lose digits (the first term left out is
// 0.35^7 / 8! of the first, 1.6e-8)
template <int kForm>
__device__ __forceinline__ F2 decay(F2 f) {
  if constexpr (kForm == kFormSigmoid) {
    const F2 x = mul2(f, f2(kLog2e));
    return f2(rcp_approx(-1.f - ex2_approx(x.x())), rcp_approx(-1.f - ex2_approx(x.y())));
  } else {
    F2 p = f2(1.f / 5040.f);
    p = fma2(p, f, f2(1.f / 720.f));
    p = fma2(p, f, f2(1.f / 120.f));
    p = fma2(p, f, f2(1.f / 24.f));
    p = fma2(p, f, f2(1.f / 6.f));
    p = fma2(p, f, f2(0.5f));
    p = fma2(p, f, f2(1.f));
    p = mul2(p, f);
    const F2 x = mul2(f, f2(kLog2e));
    return f2(fabsf(f.x()) < 0.35f ? p.x() : ex2_approx(x.x()) - 1.f, fabsf(f.y()) < 0.35f ? p.y() : ex2_approx(x.y()) - 1.f);
  }
}
// h_t from h_{t-1}
template <int kForm>
__device__ __forceinline__ F2 step(F2 h, F2 m, F2 v) {
  if constexpr (kForm == kFormSigmoid) return fma2(m, sub2(h, v), h);
  return add2(fma2(m, h, h), v);
}

// two neighbouring channels of a row, of which `left` exist; kPair: both or none, aligned
template <bool kPair, class T>
__device__ __forceinline__ F2 load2(const T* p, int left) {
  float v[2] = {0.f, 0.f};
  if constexpr (kPair) {
    if (left > 1) load_vec<2>(p, v);
  } else {
    if (left > 0) v[0] = to_float(p[0]);
    if (left > 1) v[1] = to_float(p[1]);
  }
  return f2(v[0], v[1]);
}
template <bool kPair, class T>
__device__ __forceinline__ void store2(T* p, F2 x, int left) {
  if constexpr (kPair) {
    const float v[2] = {x.x(), x.y()};
    if (left > 1) store_vec<2>(p, v);
  } else {
    if (left > 0) from_float(x.x(), p[0]);
    if (left > 1) from_float(x.y(), p[1]);
  }
}

// Which rows of a tile begin or end a sequence (a bit each), and which one (of those rows);
// lo and hi: the tile's rows that are in any.
struct TileRows {
  uint32_t starts[kTile / 32], ends[kTile / 32];
  int seq[kTile];
  int lo, hi;
};

// Fills `t` for the rows from row0 on; by one warp.  Returns the first bound that is not below
// row0; `at` is what it returned for the tile before in the walk (at first 0, backwards
// B + 1).
template <bool kBwd>
__device__ __forceinline__ int64_t mark_rows(const ScanArgs& a, int64_t row0, TileRows& t, int64_t at, int lane) {
  const int n = static_cast<int>(a.T - row0 < kTile ? a.T - row0 : kTile);
  if (lane < kTile / 32) t.starts[lane] = t.ends[lane] = 0u;
  __syncwarp();
  if (a.cu == nullptr) {
    if (lane == 0) {
      t.lo = 0;
      t.hi = n;
    }
    int64_t b = row0 / a.L;
    int64_t v = b * a.L - row0;   // where sequence b begins
    for (b += lane, v += int64_t(lane) * a.L; v < n; b += 32, v += int64_t(32) * a.L) {
      if (v >= 0) {
        t.seq[v] = static_cast<int>(b);
        atomicOr(&t.starts[v >> 5], 1u << (v & 31));
      }
      const int64_t e = v + a.L - 1;
      if (e < n) {
        t.seq[e] = static_cast<int>(b);
        atomicOr(&t.ends[e >> 5], 1u << (e & 31));
      }
    }
    __syncwarp();
    return 0;
  }
  if (lane == 0) {
    const int64_t first = a.cu[0] - row0, last = a.cu[a.B] - row0;
    t.lo = static_cast<int>(first < 0 ? 0 : first > n ? n : first);
    t.hi = static_cast<int>(last < 0 ? 0 : last > n ? n : last);
  }
  // the first bound that is not below row0: among the 32 next to the last one's, or by 32
  // probes at a time
  int64_t lo, hi;
  if constexpr (!kBwd) {
    const int64_t b = at + lane;
    const int n_below = __popc(__ballot_sync(0xffffffffu, b <= a.B && a.cu[b] < row0));
    lo = at + n_below;
    hi = n_below == 32 ? a.B + 1 : lo;
  } else {
    const int64_t b = at - 1 - lane;
    const int n_above = __popc(__ballot_sync(0xffffffffu, b >= 0 && a.cu[b] >= row0));
    hi = at - n_above;
    lo = n_above == 32 ? 0 : hi;
  }
  while (lo < hi) {
    const int64_t stride = (hi - lo + 31) / 32, b = lo + lane * stride;
    const unsigned below = __ballot_sync(0xffffffffu, b < hi && a.cu[b] < row0);
    const int k = __popc(below);   // probes below row0: a prefix of them
    const int64_t base = lo;
    if (k == 0) break;
    lo = base + (k - 1) * stride + 1;
    hi = min(hi, base + k * stride);
  }
  const int64_t found = lo;
  // bounds in [row0, row0 + n]: each ends the sequence before it and begins the one after
  for (int64_t b0 = found;; b0 += 32) {
    const int64_t b = b0 + lane;
    const int64_t v = b <= a.B ? a.cu[b] - row0 : int64_t(n) + 1;
    const bool in = v >= 0 && v <= n;
    if (in && v < n && b < a.B && a.cu[b + 1] - row0 > v) {
      t.seq[v] = static_cast<int>(b);
      atomicOr(&t.starts[v >> 5], 1u << (v & 31));
    }
    if (in && v > 0 && b > 0 && a.cu[b - 1] - row0 < v) {
      t.seq[v - 1] = static_cast<int>(b - 1);
      atomicOr(&t.ends[(v - 1) >> 5], 1u << ((v - 1) & 31));
    }
    if (!__all_sync(0xffffffffu, in)) break;
  }
  __syncwarp();
  return found;
}

// Sequences without rows keep their state: out = in (0 where there is none).
__device__ __forceinline__ void pass_empty(const ScanArgs& a, const float* in, float* out, int c0, int block, int blocks) {
  if (out == nullptr || (a.cu == nullptr && a.L > 0)) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int64_t b = int64_t(block) * kWarps + warp; b < a.B; b += int64_t(blocks) * kWarps) {
    if (a.cu != nullptr && a.cu[b + 1] > a.cu[b]) continue;
    for (int c = c0 + lane; c < min(c0 + kStrip, a.H); c += 32) out[b * a.H + c] = in ? in[b * a.H + c] : 0.f;
  }
}
// cu_seqlens that descend or leave the rows are reported.
__device__ __forceinline__ void check_bounds(const ScanArgs& a, int block, int blocks) {
  if (a.cu == nullptr) return;
  bool bad = false;
  for (int64_t b = int64_t(block) * (kWarps * 32) + threadIdx.x; b <= a.B; b += int64_t(blocks) * (kWarps * 32))
    bad |= a.cu[b] < 0 || a.cu[b] > a.T || (b > 0 && a.cu[b] < a.cu[b - 1]);
  if (bad) atomicOr(a.err, kDevErrUnsortedGroups);
}

// An affine map of two channels' states, h -> A h + b, with a cut in A's sign (A of a map
// that has none is not negative).
struct Map {
  F2 A, b;
};
__device__ __forceinline__ float4 pack(Map m, bool cut) {
  return make_float4(cut ? -1.f : m.A.x(), cut ? -1.f : m.A.y(), m.b.x(), m.b.y());
}
// m applied to h
__device__ __forceinline__ F2 apply(const float4& m, F2 h) {
  return f2(m.x < 0.f ? m.z : fmaf(m.x, h.x(), m.z), m.y < 0.f ? m.w : fmaf(m.y, h.y(), m.w));
}
// first m, then n
__device__ __forceinline__ float4 compose(const float4& m, const float4& n) {
  const F2 b = apply(n, f2(m.z, m.w));
  const bool cut = n.x < 0.f || m.x < 0.f || n.y < 0.f || m.y < 0.f;   // in both channels at once
  return make_float4(cut ? -1.f : m.x * n.x, cut ? -1.f : m.y * n.y, b.x(), b.y());
}

// What the warps of a block and the blocks of a cluster tell one another in a step.  warps:
// the map of each warp's rows, then that of all the warps before it.  Two slots for the
// peers, so that one a step ahead does not write what is still read.
template <int kCluster>
struct Exchange {
  float4 warps[kWarps][32];
  float4 tile[32];
  float4 peers[2][kCluster - 1][32];
};

// the eight warps with rows, and the one that folds
__device__ __forceinline__ void maps_sync() { asm volatile("bar.sync 1, %0;" ::"n"((kWarps + 1) * 32) : "memory"); }

// A stage is the tile's rows of each tensor.  As many as leave room for two blocks to an SM (one
// of fp32).  Rows that do not come by TMA begin inside a word and may need one more.
template <class T, bool kFast>
constexpr int kPitch = kStrip * static_cast<int>(sizeof(T)) + (kFast || sizeof(T) == 4 ? 0 : 4);
template <class T, int kTensors, bool kFast>
constexpr int kStageBytesOf = kTensors * kTile * kPitch<T, kFast>;
template <int kTensors>
constexpr int kStagesOf = kTensors == 2 ? 3 : 2;

__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A row's channels c0 .. c0 + n - 1 to shared memory, by words, from any address; first, last:
// no element lies before or behind them that may be read along.
template <class T>
__device__ __forceinline__ void copy_row(uint32_t dst, const T* row, int n, bool first, bool last, int lane) {
  if constexpr (sizeof(T) == 4) {
    if (lane < n) cp_async4(dst + 4 * lane, row + lane);
    if (lane + 32 < n) cp_async4(dst + 4 * (lane + 32), row + lane + 32);
  } else {
    const int off = static_cast<int>(reinterpret_cast<uintptr_t>(row) >> 1 & 1);
    auto word = [&](int l) {
      const int e = 2 * l - off;   // its first element
      if (e >= n) return;
      if ((e < 0 && first) || (e + 1 >= n && last)) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
          if (e + j >= 0 && e + j < n)
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(dst + 4 * l + 2 * j), "h"(reinterpret_cast<const uint16_t*>(row)[e + j])
                         : "memory");
        return;
      }
      cp_async4(dst + 4 * l, row + e);
    };
    word(lane);
    if (off && lane == 0) word(32);
  }
}

// kBwd: rows from the last one backwards.  kMapOnly: a segment's map alone.  kFast: tiles by TMA
// and pairs of channels; else elements one by one from any address.
template <class T, int kForm, bool kBwd, bool kMapOnly, bool kFast>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) scan_kernel(const __grid_constant__ ScanMaps maps,
                                                                              const ScanArgs a) {
  // tensors of a tile: gate, value (the backward's map needs none), dy
  constexpr bool kValue = !(kBwd && kMapOnly);
  constexpr int kTensors = kBwd && !kMapOnly ? 3 : 2, kV = 1, kD = kValue ? 2 : 1;
  constexpr int kStages = kStagesOf<kTensors>;
  constexpr int kRowBytes = kPitch<T, kFast>;
  constexpr int kStageBytes = kStageBytesOf<T, kTensors, kFast>, kTensorBytes = kStageBytes / kTensors;
  extern __shared__ __align__(128) uint8_t smem_raw[];
  __shared__ __align__(16) Exchange<kFast ? kMaxCluster : kMaxCluster / 2> ex;
  __shared__ float4 h_maps[kBwd && !kMapOnly ? kWarps : 1][32];   // then, in x and y, h before each warp's rows
  __shared__ TileRows rows_sh[kStages];
  __shared__ __align__(8) uint64_t full_bar[kStages], empty_bar[kStages], peer_bar[2];
  __shared__ int abort_sh;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  volatile int* abort_flag = &abort_sh;
  uint32_t size;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(size));
  const int S = static_cast<int>(size), rank = static_cast<int>(cluster_ctarank());
  const int strip = blockIdx.x / S, strips = gridDim.x / S;
  const int c0 = strip * kStrip, c = c0 + 2 * lane, left = a.H - c;
  const int seg = blockIdx.y, seg0 = seg * a.seg_tiles, seg_n = min(a.seg_tiles, a.tiles - seg0);
  const int n_steps = (seg_n + S - 1) / S;
  // the tile of step k, or -1
  auto tile_of = [&](int k) -> int {
    const int i = k * S + rank;
    return i >= seg_n ? -1 : kBwd ? seg0 + seg_n - 1 - i : seg0 + i;
  };

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&full_bar[s]), kFast ? 2 : 1);
      mbar_init(smem_u32(&empty_bar[s]), kWarps);
    }
    for (int s = 0; s < 2; ++s) mbar_init(smem_u32(&peer_bar[s]), 1);
    abort_sh = 0;
    fence_mbar_init();
  }
  const float4 identity = make_float4(1.f, 1.f, 0.f, 0.f);
  __syncthreads();
  cluster_sync_all();   // every block's barriers exist before a peer's message

  if (warp == kWarps) {
    // tiles, and their rows' bounds, ahead of the others
    int64_t at = kBwd ? a.B + 1 : 0;
    int issued = 0;
    for (int k = 0; k < n_steps; ++k) {
      const int tile = tile_of(k), st = k % kStages;
      if (tile < 0) break;
      if (!mbar_wait(smem_u32(&empty_bar[st]), ((k / kStages) & 1u) ^ 1u, abort_flag, a.err)) break;
      if (kFast && lane == 0) {
        const uint32_t bar = smem_u32(&full_bar[st]), dst = smem_u32(smem_raw) + st * kStageBytes;
        mbar_arrive_expect_tx(bar, kStageBytes);
        tma_load_2d(dst, &maps.gate, bar, c0, tile * kTile);
        if constexpr (kValue) tma_load_2d(dst + kV * kTensorBytes, &maps.value, bar, c0, tile * kTile);
        if constexpr (kBwd) tma_load_2d(dst + kD * kTensorBytes, &maps.dy, bar, c0, tile * kTile);
      }
      ++issued;
      at = mark_rows<kBwd>(a, int64_t(tile) * kTile, rows_sh[st], at, lane);
      if (lane == 0) mbar_arrive(smem_u32(&full_bar[st]));
    }
    // copies land in this block's memory: wait for the last ones before it may exit
    if (lane == 0)
      for (int k = max(0, issued - kStages); k < issued; ++k)
        mbar_wait_drain(smem_u32(&full_bar[k % kStages]), (k / kStages) & 1u, a.err);
  } else if (warp == kWarps + 1) {
    // a step's maps: the tile's, for all blocks of the cluster, and what precedes each warp's rows
    for (int k = 0; k < n_steps; ++k) {
      const int tile = tile_of(k), slot = k & 1;
      F2 h = zero2();   // backward: the state before the tile
      if constexpr (kBwd && !kMapOnly)
        if (tile >= 0) h = load2<kFast>(a.states + int64_t(tile) * a.H + c, left);
      maps_sync();
      float4 before[kWarps], t = identity;
#pragma unroll
      for (int j = 0; j < kWarps; ++j) before[j] = ex.warps[kBwd ? kWarps - 1 - j : j][lane];
#pragma unroll
      for (int j = 0; j < kWarps; ++j) {
        const float4 own = before[j];
        before[j] = t;
        t = compose(t, own);
      }
      const uint32_t bar = smem_u32(&peer_bar[slot]);
      const int4 bits = make_int4(__float_as_int(t.x), __float_as_int(t.y), __float_as_int(t.z), __float_as_int(t.w));
      for (int p = 0; p < S; ++p)
        if (p != rank)
          st_async_v4(mapa_shared(smem_u32(&ex.peers[slot][rank < p ? rank : rank - 1][lane]), p), mapa_shared(bar, p), bits);
      ex.tile[lane] = t;
#pragma unroll
      for (int j = 0; j < kWarps; ++j) ex.warps[kBwd ? kWarps - 1 - j : j][lane] = before[j];
      if constexpr (kBwd && !kMapOnly) {
#pragma unroll
        for (int j = 0; j < kWarps; ++j) before[j] = h_maps[j][lane];
#pragma unroll
        for (int j = 0; j < kWarps; ++j) {
          *reinterpret_cast<float2*>(&h_maps[j][lane]) = make_float2(h.x(), h.y());
          h = apply(before[j], h);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive_expect_tx(bar, (S - 1) * 512);
    }
  } else {
    if (!kMapOnly && seg == 0) {
      pass_empty(a, kBwd ? a.dfinal : a.h0, kBwd ? a.dinit : a.final_state, c0, rank, S);
      if (strip == 0) check_bounds(a, rank, S);
    }
    const int r0 = warp * kRows;
    const auto of_seq = [&](const float* p, int b) { return p ? load2<kFast>(p + int64_t(b) * a.H + c, left) : zero2(); };
    // the state before the segment (E after it)
    F2 carry = zero2();
    float4 total = identity;
    if constexpr (!kMapOnly) {
      for (int s = kBwd ? static_cast<int>(gridDim.y) - 1 : 0; s != seg; s += kBwd ? -1 : 1)
        carry = apply(a.seg_maps[(int64_t(s) * strips + strip) * 32 + lane], carry);
    }
    // rows that do not come by TMA: every warp copies its own, all stages but one ahead
    const void* const tensor_of[3] = {a.gate, kValue ? a.value : a.dy, a.dy};
    const int64_t ld_of[3] = {a.gate_ld, kValue ? a.value_ld : a.dy_ld, a.dy_ld};
    uint32_t odd_base = 0, odd_ld = 0;   // whether a tensor's rows begin inside a word: at row 0, and for odd rows besides
    auto load_rows = [&](int k) {
      const int t = k < n_steps ? tile_of(k) : -1;
      if (t >= 0) {
#pragma unroll
        for (int j = 0; j < kTensors; ++j) {
          const uint32_t dst = smem_u32(smem_raw) + (k % kStages) * kStageBytes + j * kTensorBytes + r0 * kRowBytes;
#pragma unroll 4
          for (int i = 0; i < kRows; ++i) {
            const int64_t r = int64_t(t) * kTile + r0 + i;
            if (r >= a.T) break;
            copy_row(dst + i * kRowBytes, static_cast<const T*>(tensor_of[j]) + r * ld_of[j] + c0, min(kStrip, a.H - c0),
                     r == 0 && c0 == 0, r == a.T - 1 && c0 + kStrip >= a.H, lane);
          }
        }
      }
      cp_async_commit();
    };
    if constexpr (!kFast) {
#pragma unroll
      for (int j = 0; j < kTensors; ++j) {
        odd_base |= static_cast<uint32_t>(reinterpret_cast<uintptr_t>(tensor_of[j]) >> 1 & 1) << j;   // (c0 is even)
        odd_ld |= static_cast<uint32_t>(ld_of[j] & 1) << j;
      }
#pragma unroll
      for (int k = 0; k < kStages - 1; ++k) load_rows(k);
    }
    bool alive = true;   // no wait has run out; else the loop goes on without work, for the barriers' sake
    // a stage whose rows are still read by this warp's copies: given back in the next step
    int held = -1;
    auto give_back = [&]() {
      if (held < 0) return;
      if (lane == 0) {
        bulk_wait_group_read<0>();
        mbar_arrive(smem_u32(&empty_bar[held]));
      }
      held = -1;
    };
    for (int k = 0; k < n_steps; ++k) {
      const int st = k % kStages, slot = k & 1;
      int tile = alive ? tile_of(k) : -1;
      const TileRows& rows = rows_sh[st];
      if (tile >= 0) {
        if (!mbar_wait(smem_u32(&full_bar[st]), (k / kStages) & 1u, abort_flag, a.err)) {
          alive = false;
          tile = -1;
        }
      }
      const int64_t row = int64_t(tile) * kTile + r0;   // the warp's first
      uint32_t starts = 0, ends = 0, valid = 0;         // a bit for each of its rows; valid: in a sequence
      if (tile >= 0) {
        starts = rows.starts[r0 >> 5] >> (r0 & 31) & 0xffffu;
        ends = rows.ends[r0 >> 5] >> (r0 & 31) & 0xffffu;
        const int lo = min(max(rows.lo - r0, 0), kRows), hi = min(max(rows.hi - r0, 0), kRows);
        valid = (1u << hi) - 1u & ~((1u << lo) - 1u);
        if constexpr (!kFast) {
          load_rows(k + kStages - 1);
          cp_async_wait<kStages - 1>();
          __syncwarp();
        }
      }
      const bool simple = valid == (1u << kRows) - 1u && (starts | ends) == 0;
      auto inside = [&](int i) -> bool { return valid >> i & 1u; };
      uint8_t* const stage8 = smem_raw + st * kStageBytes + r0 * kRowBytes;
      T* const stage = reinterpret_cast<T*>(stage8) + 2 * lane;
      auto get = [&](int tensor, int i) -> F2 {
        if constexpr (kFast || sizeof(T) == 4) {
          return load2<true>(reinterpret_cast<const T*>(reinterpret_cast<const uint8_t*>(stage) + tensor * kTensorBytes +
                                                        i * kRowBytes), 2);
        } else {
          const uint32_t* const w = reinterpret_cast<const uint32_t*>(stage8 + tensor * kTensorBytes + i * kRowBytes) + lane;
          const bool odd = (odd_base >> tensor ^ (odd_ld >> tensor & static_cast<uint32_t>(row + i))) & 1u;
          const uint32_t w0 = w[0], w1 = w[1];
          float lo, hi;
          unpack2(odd ? __byte_perm(w0, w1, 0x5432) : w0, static_cast<const T*>(nullptr), lo, hi);
          return f2(lo, hi);
        }
      };

      // ---- the maps of the warp's rows
      F2 m[kRows];
      float4 mine = identity, mine_h = identity;
      if (tile >= 0) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) m[i] = decay<kForm>(get(0, i));
        F2 A = f2(1.f), x = zero2(), z = zero2();   // x: the walk's, z: h in a backward walk
        bool cut = false, cut_z = false;
        if (simple) {
#pragma unroll
          for (int i = 0; i < kRows; ++i) {
            A = fma2(m[i], A, A);
            if constexpr (!kBwd) x = step<kForm>(x, m[i], get(kV, i));
            if constexpr (kBwd && !kMapOnly) z = step<kForm>(z, m[i], get(kV, i));
          }
          if constexpr (kBwd) {
#pragma unroll
            for (int i = kRows - 1; i >= 0; --i) {
              x = add2(x, get(kD, i));
              x = fma2(m[i], x, x);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < kRows; ++i) {
            if (!inside(i)) continue;
            A = fma2(m[i], A, A);
            if constexpr (!kBwd || !kMapOnly) {
              F2& w = kBwd ? z : x;
              if (starts >> i & 1u) {
                w = of_seq(a.h0, rows.seq[r0 + i]);
                (kBwd ? cut_z : cut) = true;
              }
              w = step<kForm>(w, m[i], get(kV, i));
            }
          }
          if constexpr (kBwd) {
#pragma unroll
            for (int i = kRows - 1; i >= 0; --i) {
              if (!inside(i)) continue;
              if (ends >> i & 1u) {
                x = of_seq(a.dfinal, rows.seq[r0 + i]);
                cut = true;
              }
              x = add2(x, get(kD, i));
              x = fma2(m[i], x, x);
            }
          }
        }
        mine = pack(Map{A, x}, cut);
        if constexpr (kBwd && !kMapOnly) mine_h = pack(Map{A, z}, cut_z);
      }
      ex.warps[warp][lane] = mine;
      if constexpr (kBwd && !kMapOnly) h_maps[warp][lane] = mine_h;
      maps_sync();
      give_back();
      if (!mbar_wait(smem_u32(&peer_bar[slot]), (k >> 1) & 1u, abort_flag, a.err)) {
        alive = false;
        tile = -1;
      }
      // ---- what enters the warp's rows, and the step after
      F2 in = carry;
      for (int p = 0; p < S; ++p) {
        const float4 of_tile = p == rank ? ex.tile[lane] : ex.peers[slot][p < rank ? p : p - 1][lane];
        if constexpr (kMapOnly) {
          if (warp == 0) total = compose(total, of_tile);
        } else {
          if (p == rank) {
            in = apply(ex.warps[warp][lane], carry);
            if (!kBwd && tile >= 0 && a.states && warp == 0) store2<kFast>(a.states + int64_t(tile) * a.H + c, carry, left);
          }
          carry = apply(of_tile, carry);
        }
      }

      // ---- the rows again
      if (tile < 0) continue;
      // results of a warp whose rows are all in sequences go out as a box, from where its gates
      // (and dy) have been
      bool boxed = false;
      if constexpr (!kBwd && !kMapOnly) {
        T* y = static_cast<T*>(a.y) + row * a.H + c;
        if (simple) {
          boxed = kFast;
#pragma unroll
          for (int i = 0; i < kRows; ++i) {
            in = step<kForm>(in, m[i], get(kV, i));
            if constexpr (kFast)
              store2<true>(stage + i * kStrip, in, 2);
            else
              store2<false>(y + int64_t(i) * a.H, in, left);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kRows; ++i) {
            if (!inside(i)) {
              if (a.fill && row + i < a.T) store2<kFast>(y + int64_t(i) * a.H, zero2(), left);
              continue;
            }
            if (starts >> i & 1u) in = of_seq(a.h0, rows.seq[r0 + i]);
            in = step<kForm>(in, m[i], get(kV, i));
            store2<kFast>(y + int64_t(i) * a.H, in, left);
            if ((ends >> i & 1u) && a.final_state) store2<kFast>(a.final_state + int64_t(rows.seq[r0 + i]) * a.H + c, in, left);
          }
        }
      } else if constexpr (!kMapOnly) {
        T* dg = static_cast<T*>(a.dgate) + row * a.H + c;
        T* dv = static_cast<T*>(a.dvalue) + row * a.H + c;
        const float2 before = *reinterpret_cast<const float2*>(&h_maps[warp][lane]);
        F2 h = f2(before.x, before.y);
        // dgate and dvalue of a row from D and E, h of the row before and its value
        auto grads = [&](int i, F2 D, F2 E, F2 hp, F2& df, F2& dval) {
          if constexpr (kForm == kFormSigmoid) {
            const F2 w = mul2(m[i], f2(-1.f));
            df = mul2(mul2(E, w), sub2(hp, get(kV, i)));
            dval = mul2(D, w);
          } else {
            df = mul2(E, hp);
            dval = D;
          }
        };
        F2 hp[kRows], df, dval;   // hp: h of the row before
        if (simple) {
          boxed = kFast;
#pragma unroll
          for (int i = 0; i < kRows; ++i) {
            hp[i] = h;
            h = step<kForm>(h, m[i], get(kV, i));
          }
#pragma unroll
          for (int i = kRows - 1; i >= 0; --i) {
            const F2 D = add2(get(kD, i), in);
            in = fma2(m[i], D, D);   // E
            grads(i, D, in, hp[i], df, dval);
            if constexpr (kFast) {
              store2<true>(stage + i * kStrip, df, 2);
              store2<true>(stage + kD * (kTile * kStrip) + i * kStrip, dval, 2);
            } else {
              store2<false>(dg + int64_t(i) * a.H, df, left);
              store2<false>(dv + int64_t(i) * a.H, dval, left);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < kRows; ++i) {
            if (!inside(i)) continue;
            if (starts >> i & 1u) h = of_seq(a.h0, rows.seq[r0 + i]);
            hp[i] = h;
            h = step<kForm>(h, m[i], get(kV, i));
          }
#pragma unroll
          for (int i = kRows - 1; i >= 0; --i) {
            if (!inside(i)) {
              if (row + i < a.T) {
                store2<kFast>(dg + int64_t(i) * a.H, zero2(), left);
                store2<kFast>(dv + int64_t(i) * a.H, zero2(), left);
              }
              continue;
            }
            if (ends >> i & 1u) in = of_seq(a.dfinal, rows.seq[r0 + i]);
            const F2 D = add2(get(kD, i), in);
            in = fma2(m[i], D, D);
            grads(i, D, in, hp[i], df, dval);
            store2<kFast>(dg + int64_t(i) * a.H, df, left);
            store2<kFast>(dv + int64_t(i) * a.H, dval, left);
            if ((starts >> i & 1u) && a.dinit) store2<kFast>(a.dinit + int64_t(rows.seq[r0 + i]) * a.H + c, in, left);
          }
        }
      }
      if (boxed) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          const uint32_t box = smem_u32(smem_raw) + st * kStageBytes + r0 * kStrip * static_cast<int>(sizeof(T));
          tma_store_2d(&maps.out0, box, c0, static_cast<int>(row));
          if constexpr (kBwd && !kMapOnly) tma_store_2d(&maps.out1, box + kD * kTensorBytes, c0, static_cast<int>(row));
          bulk_commit_group();
        }
        held = st;
      } else {
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&empty_bar[st]));
      }
    }
    give_back();
    if (lane == 0) bulk_wait_group<0>();
    if constexpr (!kFast) cp_async_wait<0>();
    if (kMapOnly && warp == 0 && rank == 0) a.seg_maps[(int64_t(seg) * strips + strip) * 32 + lane] = total;
  }
  __syncthreads();
  cluster_sync_all();   // no block leaves while a peer may still write to it
}

template <class T, int kForm>
__global__ void __launch_bounds__(256) scan_step_kernel(const T* gate, const T* value, const float* state, int64_t B, int H,
                                                        int64_t gate_ld, int64_t value_ld, T* y, float* state_out) {
  const int64_t n = B * H;
  for (int64_t i = blockIdx.x * int64_t(256) + threadIdx.x; i < n; i += gridDim.x * int64_t(256)) {
    const int64_t b = i / H;
    const int c = static_cast<int>(i - b * H);
    const F2 h = step<kForm>(f2(state[i]), decay<kForm>(f2(to_float(gate[b * gate_ld + c]))),
                             f2(to_float(value[b * value_ld + c])));
    state_out[i] = h.x();
    from_float(h.x(), y[i]);
  }
}

molt_status fail(molt_status s, const char* msg) {
  set_last_error(msg);
  return s;
}
molt_status cuda_fail(cudaError_t e, const char* what) {
  set_last_error(std::string(what) + ": " + cudaGetErrorString(e));
  return MOLT_ERR_CUDA;
}

molt_status check_desc(const molt_scan_desc* d, bool packed) {
  if (!d) return fail(MOLT_ERR_INVALID_ARG, "desc is NULL");
  if (d->T < 0 || d->H < 1 || d->B < 0) return fail(MOLT_ERR_INVALID_ARG, "sizes must satisfy T >= 0, H >= 1, B >= 0");
  if (d->dtype != MOLT_BF16 && d->dtype != MOLT_FP16 && d->dtype != MOLT_FP32)
    return fail(MOLT_ERR_INVALID_ARG, "unknown element type");
  if (d->form != MOLT_SCAN_SIGMOID && d->form != MOLT_SCAN_LOG) return fail(MOLT_ERR_INVALID_ARG, "unknown form of the recurrence");
  if (d->T > 2147483647 - 2 * kTile || d->H > 65536 || d->B > 2147483647 - 64)
    return fail(MOLT_ERR_UNSUPPORTED_SHAPE, "T and B must be below 2^31 - 256 and H at most 65536");
  if (!packed && (d->B == 0 ? d->T != 0 : d->T % d->B != 0))
    return fail(MOLT_ERR_INVALID_ARG, "without cu_seqlens T must be a multiple of B");
  for (const int64_t ld : {d->gate_stride, d->value_stride, d->dy_stride})
    if (ld != 0 && ld < d->H) return fail(MOLT_ERR_INVALID_ARG, "a row stride is 0 (rows side by side) or at least H");
  return MOLT_OK;
}

struct Operand {
  const void* p;
  int dtype;
};
molt_status check_elements(std::initializer_list<Operand> ops) {
  for (const Operand& o : ops)
    if (o.p && reinterpret_cast<uintptr_t>(o.p) % static_cast<size_t>(dtype_bytes(o.dtype)) != 0)
      return fail(MOLT_ERR_INVALID_ARG, "a pointer is not aligned to its element type");
  return MOLT_OK;
}

ScanArgs base_args(const molt_scan_desc* d, const int32_t* cu) {
  ScanArgs a{};
  a.T = d->T;
  a.H = static_cast<int>(d->H);
  a.B = d->B;
  a.cu = cu;
  a.L = cu == nullptr && d->B > 0 ? static_cast<int>(d->T / d->B) : 0;
  a.gate_ld = d->gate_stride ? d->gate_stride : d->H;
  a.value_ld = d->value_stride ? d->value_stride : d->H;
  a.dy_ld = d->dy_stride ? d->dy_stride : d->H;
  return a;
}

// Tiles can come by TMA and vectors be read two channels at a time.
bool fast_of(const ScanArgs& a, int dtype) {
  const size_t e = static_cast<size_t>(dtype_bytes(dtype));
  const auto at = [](const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; };
  for (const void* p : {a.gate, a.value, a.dy, static_cast<const void*>(a.y), static_cast<const void*>(a.dgate),
                        static_cast<const void*>(a.dvalue)})
    if (!at(p, 16)) return false;
  for (const float* p : {a.h0, a.dfinal, static_cast<const float*>(a.final_state), static_cast<const float*>(a.states),
                         static_cast<const float*>(a.dinit)})
    if (!at(p, 8)) return false;
  return a.H * e % 16 == 0 && a.gate_ld * e % 16 == 0 && a.value_ld * e % 16 == 0 && a.dy_ld * e % 16 == 0;
}

constexpr int kMaxSegments = 32;
int64_t strips_of(const molt_scan_desc* d) { return (d->H + kStrip - 1) / kStrip; }
size_t seg_bytes(const molt_scan_desc* d) { return static_cast<size_t>(kMaxSegments) * strips_of(d) * 32 * sizeof(float4) + 256; }

struct ScanPlan {
  int cluster, segments;
};
ScanPlan plan_of(const molt_scan_desc* d, int tiles, int n_sm, bool fast) {
  const int64_t strips = strips_of(d), slots = int64_t(n_sm) * (d->dtype == MOLT_FP32 ? 1 : 2);
  ScanPlan p;
  p.cluster = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({fast ? kMaxCluster : kMaxCluster / 2, slots / strips, tiles})));
  const int64_t room = slots / (strips * p.cluster), steps = (tiles + p.cluster - 1) / p.cluster;
  p.segments = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({kMaxSegments, room, steps / 8})));
  return p;
}

template <class T, int kForm, bool kBwd, bool kMapOnly, bool kFast>
cudaError_t launch_kernel(const ScanMaps& m, const ScanArgs& a, int strips, int cluster, int segments, cudaStream_t s) {
  constexpr int kTensors = kBwd && !kMapOnly ? 3 : 2;
  constexpr int smem = kStagesOf<kTensors> * kStageBytesOf<T, kTensors, kFast>;
  const auto k = &scan_kernel<T, kForm, kBwd, kMapOnly, kFast>;
  if (const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem); e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(strips * cluster, segments);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = cluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k, m, a);
}
template <class T, int kForm, bool kFast>
cudaError_t launch_form(const ScanMaps& m, const ScanArgs& a, bool bwd, bool map_only, int strips, int cluster, int segments,
                        cudaStream_t s) {
  if (bwd)
    return map_only ? launch_kernel<T, kForm, true, true, kFast>(m, a, strips, cluster, segments, s)
                    : launch_kernel<T, kForm, true, false, kFast>(m, a, strips, cluster, segments, s);
  return map_only ? launch_kernel<T, kForm, false, true, kFast>(m, a, strips, cluster, segments, s)
                  : launch_kernel<T, kForm, false, false, kFast>(m, a, strips, cluster, segments, s);
}
template <class T>
cudaError_t launch_type(const ScanMaps& m, const ScanArgs& a, int form, bool fast, bool bwd, bool map_only, int strips, int cluster,
                        int segments, cudaStream_t s) {
  const auto k = form == kFormSigmoid ? (fast ? launch_form<T, kFormSigmoid, true> : launch_form<T, kFormSigmoid, false>)
                                      : (fast ? launch_form<T, kFormLog, true> : launch_form<T, kFormLog, false>);
  return k(m, a, bwd, map_only, strips, cluster, segments, s);
}

molt_status launch(const molt_scan_desc* d, ScanArgs& a, bool bwd, void* workspace, size_t workspace_bytes, cudaStream_t s) {
  molt_status st;
  a.err = device_status_word(&st);
  if (!a.err) return st;
  const int strips = static_cast<int>(strips_of(d));
  a.tiles = static_cast<int>((a.T + kTile - 1) / kTile);
  const bool fast = a.tiles > 0 && fast_of(a, d->dtype);
  const ScanPlan plan = plan_of(d, a.tiles, device_sm_count(), fast);
  a.seg_tiles = (a.tiles + plan.segments - 1) / plan.segments;
  const int segments = a.tiles > 0 ? (a.tiles + a.seg_tiles - 1) / a.seg_tiles : 1;
  Scratch sc;
  if (segments > 1) {
    if (const molt_status e = get_scratch(sc, workspace, workspace_bytes, seg_bytes(d), s); e != MOLT_OK) return e;
    a.seg_maps = static_cast<float4*>(sc.aligned());
  }
  ScanMaps m{};
  if (fast) {
    const int e = dtype_bytes(d->dtype);
    const auto encode = [&](CUtensorMap* t, const void* p, int64_t ld, int rows = kTile) {
      return encode_tmap_plain(t, e == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, e, p, a.T, a.H, ld,
                               kStrip, rows);
    };
    if (const molt_status q = encode(&m.gate, a.gate, a.gate_ld); q != MOLT_OK) return q;
    if (const molt_status q = encode(&m.value, a.value, a.value_ld); q != MOLT_OK) return q;
    if (bwd)
      if (const molt_status q = encode(&m.dy, a.dy, a.dy_ld); q != MOLT_OK) return q;
    if (const molt_status q = encode(&m.out0, bwd ? a.dgate : a.y, a.H, kRows); q != MOLT_OK) return q;
    if (bwd)
      if (const molt_status q = encode(&m.out1, a.dvalue, a.H, kRows); q != MOLT_OK) return q;
  }
  for (int pass = segments > 1 ? 0 : 1; pass < 2; ++pass) {
    const bool map_only = pass == 0;
    const cudaError_t e =
        d->dtype == MOLT_FP32   ? launch_type<float>(m, a, d->form, fast, bwd, map_only, strips, plan.cluster, segments, s)
        : d->dtype == MOLT_FP16 ? launch_type<__half>(m, a, d->form, fast, bwd, map_only, strips, plan.cluster, segments, s)
                                : launch_type<__nv_bfloat16>(m, a, d->form, fast, bwd, map_only, strips, plan.cluster, segments, s);
    if (e != cudaSuccess) return cuda_fail(e, "gated scan");
    note_launches(1);
  }
  return MOLT_OK;
}

template <class T, int kForm>
void launch_step(const molt_scan_desc* d, const void* gate, const void* value, const float* state, void* y, float* out,
                 int grid, cudaStream_t s) {
  scan_step_kernel<T, kForm><<<grid, 256, 0, s>>>(
      static_cast<const T*>(gate), static_cast<const T*>(value), state, d->B, static_cast<int>(d->H),
      d->gate_stride ? d->gate_stride : d->H, d->value_stride ? d->value_stride : d->H, static_cast<T*>(y), out);
}

}  // namespace
}  // namespace molt

using namespace molt;

extern "C" {

size_t molt_gated_scan_workspace_bytes(const molt_scan_desc* desc) {
  return check_desc(desc, true) == MOLT_OK ? seg_bytes(desc) : 0;
}

molt_status molt_gated_scan_fwd(const molt_scan_desc* desc, const void* gate, const void* value, const float* initial_state,
                                const int32_t* cu_seqlens, void* y, float* final_state, float* states, void* workspace,
                                size_t workspace_bytes, cudaStream_t stream) {
  if (const molt_status st = check_desc(desc, cu_seqlens != nullptr); st != MOLT_OK) return st;
  if (desc->T > 0 && (!gate || !value || !y)) return fail(MOLT_ERR_INVALID_ARG, "null pointer");
  if (const molt_status st = check_elements({{gate, desc->dtype},
                                             {value, desc->dtype},
                                             {y, desc->dtype},
                                             {initial_state, MOLT_FP32},
                                             {cu_seqlens, MOLT_FP32},
                                             {final_state, MOLT_FP32},
                                             {states, MOLT_FP32}});
      st != MOLT_OK)
    return st;
  if (desc->T == 0 && (desc->B == 0 || !final_state)) return MOLT_OK;
  if (workspace && workspace_bytes < seg_bytes(desc)) return fail(MOLT_ERR_WORKSPACE, "workspace too small");
  ScanArgs a = base_args(desc, cu_seqlens);
  a.gate = gate;
  a.value = value;
  a.h0 = initial_state;
  a.y = y;
  a.final_state = final_state;
  a.states = states;
  a.fill = desc->fill_outside != 0;
  return launch(desc, a, false, workspace, workspace_bytes, stream);
}

molt_status molt_gated_scan_bwd(const molt_scan_desc* desc, const void* dy, const void* gate, const void* value,
                                const float* states, const float* initial_state, const int32_t* cu_seqlens,
                                const float* dfinal_state, void* dgate, void* dvalue, float* dinitial_state,
                                void* workspace, size_t workspace_bytes, cudaStream_t stream) {
  if (const molt_status st = check_desc(desc, cu_seqlens != nullptr); st != MOLT_OK) return st;
  if (desc->T > 0 && (!dy || !gate || !value || !states || !dgate || !dvalue)) return fail(MOLT_ERR_INVALID_ARG, "null pointer");
  if (const molt_status st = check_elements({{dy, desc->dtype},
                                             {gate, desc->dtype},
                                             {value, desc->dtype},
                                             {dgate, desc->dtype},
                                             {dvalue, desc->dtype},
                                             {states, MOLT_FP32},
                                             {initial_state, MOLT_FP32},
                                             {cu_seqlens, MOLT_FP32},
                                             {dfinal_state, MOLT_FP32},
                                             {dinitial_state, MOLT_FP32}});
      st != MOLT_OK)
    return st;
  if (desc->T == 0 && (desc->B == 0 || !dinitial_state)) return MOLT_OK;
  if (workspace && workspace_bytes < seg_bytes(desc)) return fail(MOLT_ERR_WORKSPACE, "workspace too small");
  ScanArgs a = base_args(desc, cu_seqlens);
  a.dy = dy;
  a.gate = gate;
  a.value = value;
  a.states = const_cast<float*>(states);
  a.h0 = initial_state;
  a.dfinal = dfinal_state;
  a.dgate = dgate;
  a.dvalue = dvalue;
  a.dinit = dinitial_state;
  return launch(desc, a, true, workspace, workspace_bytes, stream);
}

molt_status molt_gated_scan_step(const molt_scan_desc* desc, const void* gate, const void* value, const float* state,
                                 void* y, float* state_out, cudaStream_t stream) {
  if (const molt_status st = check_desc(desc, true); st != MOLT_OK) return st;
  if (desc->B != desc->T) return fail(MOLT_ERR_INVALID_ARG, "a step takes one row of each sequence: T = B");
  if (desc->B == 0) return MOLT_OK;
  if (!gate || !value || !state || !y || !state_out) return fail(MOLT_ERR_INVALID_ARG, "null pointer");
  if (const molt_status st = check_elements({{gate, desc->dtype},
                                             {value, desc->dtype},
                                             {y, desc->dtype},
                                             {state, MOLT_FP32},
                                             {state_out, MOLT_FP32}});
      st != MOLT_OK)
    return st;
  const int64_t blocks = (desc->B * desc->H + 255) / 256;
  const int grid = static_cast<int>(std::min<int64_t>(blocks, 16 * int64_t(device_sm_count())));
  const bool sig = desc->form == MOLT_SCAN_SIGMOID;
  const auto k = desc->dtype == MOLT_FP32   ? (sig ? launch_step<float, kFormSigmoid> : launch_step<float, kFormLog>)
                 : desc->dtype == MOLT_FP16 ? (sig ? launch_step<__half, kFormSigmoid> : launch_step<__half, kFormLog>)
                                            : (sig ? launch_step<__nv_bfloat16, kFormSigmoid> : launch_step<__nv_bfloat16, kFormLog>);
  k(desc, gate, value, state, y, state_out, grid, stream);
  if (const cudaError_t e = cudaGetLastError(); e != cudaSuccess) return cuda_fail(e, "gated scan step");
  note_launches(1);
  return MOLT_OK;
}

}  // extern "C"
