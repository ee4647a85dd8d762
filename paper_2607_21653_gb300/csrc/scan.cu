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
// Every warp composes its rows' maps, adds its predecessors' in order, and then goes
// through its rows again from the state that it now knows; the tile's own map carries the
// state on.  A row that begins a sequence cuts: what comes before is not multiplied
// by zero but left out, so that an infinite or NaN state stays in its sequence.
//
// Everything is held as 1 - a: with a as a float near 1 the memory 1 / (1 - a) of a channel
// would be off by 2^-24 / (1 - a), and h - (1 - a) (h - v) needs no a at all.
#include <algorithm>
#include <cstdint>
#include <cuda_runtime.h>

#include "molt_internal.cuh"
#include "ptx.cuh"
#include "vec.cuh"

namespace molt {
namespace {

constexpr int kTile = 128;               // rows of a tile, and between kept states
constexpr int kWarps = 8, kRows = kTile / kWarps;
constexpr int kStrip = 64;               // channels of a block
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
  unsigned* err;
};

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 1 - a of a gate's value
template <int kForm>
__device__ __forceinline__ float one_minus_a(float f) {
  if constexpr (kForm == kFormSigmoid) {
    const float e = ex2_approx(-kLog2e * fabsf(f)), r = rcp_approx(1.f + e);
    return f >= 0.f ? e * r : f < 0.f ? r : f;
  } else {
    // -(e^f - 1): by its series where the difference would lose digits (the first
    // term left out is 0.35^7 / 8! of the first, 1.6e-8)
    float p = 1.f / 5040.f;
    p = fmaf(p, f, 1.f / 720.f);
    p = fmaf(p, f, 1.f / 120.f);
    p = fmaf(p, f, 1.f / 24.f);
    p = fmaf(p, f, 1.f / 6.f);
    p = fmaf(p, f, 0.5f);
    p = fmaf(p, f, 1.f);
    return fabsf(f) < 0.35f ? -f * p : 1.f - ex2_approx(kLog2e * f);
  }
}
// h_t from h_{t-1}
template <int kForm>
__device__ __forceinline__ float step(float h, float na, float v) {
  if constexpr (kForm == kFormSigmoid) return fmaf(na, v - h, h);
  return fmaf(-na, h, h) + v;
}

// two neighbouring channels of a row, of which `left` exist
template <bool kPair, class T>
__device__ __forceinline__ float2 load2(const T* p, int left) {
  float v[2] = {0.f, 0.f};
  if constexpr (kPair) {
    if (left > 1) load_vec<2>(p, v);
  } else {
    if (left > 0) v[0] = to_float(p[0]);
    if (left > 1) v[1] = to_float(p[1]);
  }
  return make_float2(v[0], v[1]);
}
template <bool kPair, class T>
__device__ __forceinline__ void store2(T* p, float a, float b, int left) {
  if constexpr (kPair) {
    const float v[2] = {a, b};
    if (left > 1) store_vec<2>(p, v);
  } else {
    if (left > 0) from_float(a, p[0]);
    if (left > 1) from_float(b, p[1]);
  }
}

// Which rows of a tile begin or end a sequence, and which one: -1 for none.  lo and hi: the
// tile's rows that are in any.
struct TileRows {
  int start[kTile], end[kTile];
  int lo, hi;
};

// first b in [0, B] with cu[b] >= row (B + 1: none)
__device__ __forceinline__ int64_t first_bound(const int32_t* cu, int64_t B, int64_t row) {
  int64_t a = 0, z = B + 1;
  while (a < z) {
    const int64_t m = (a + z) / 2;
    if (cu[m] >= row)
      z = m;
    else
      a = m + 1;
  }
  return a;
}

// Fills `t` for the rows from row0 on; by one warp.
__device__ __forceinline__ void mark_rows(const ScanArgs& a, int64_t row0, TileRows& t, int lane) {
  const int n = static_cast<int>(a.T - row0 < kTile ? a.T - row0 : kTile);
#pragma unroll
  for (int i = lane; i < kTile; i += 32) t.start[i] = t.end[i] = -1;
  __syncwarp();
  if (a.cu == nullptr) {
    if (lane == 0) {
      t.lo = 0;
      t.hi = n;
    }
    for (int i = lane; i < n; i += 32) {
      const int64_t r = row0 + i, b = r / a.L;
      const int64_t in = r - b * a.L;
      if (in == 0) t.start[i] = static_cast<int>(b);
      if (in == a.L - 1) t.end[i] = static_cast<int>(b);
    }
    return;
  }
  if (lane == 0) {
    const int64_t first = a.cu[0] - row0, last = a.cu[a.B] - row0;
    t.lo = static_cast<int>(first < 0 ? 0 : first > n ? n : first);
    t.hi = static_cast<int>(last < 0 ? 0 : last > n ? n : last);
  }
  // bounds in [row0, row0 + n]: each ends the sequence before it and begins the one after
  for (int64_t b0 = first_bound(a.cu, a.B, row0);; b0 += 32) {
    const int64_t b = b0 + lane;
    const int64_t v = b <= a.B ? a.cu[b] - row0 : int64_t(n) + 1;
    const bool in = v >= 0 && v <= n;
    if (in && v < n && b < a.B && a.cu[b + 1] - row0 > v) t.start[v] = static_cast<int>(b);
    if (in && v > 0 && b > 0 && a.cu[b - 1] - row0 < v) t.end[v - 1] = static_cast<int>(b - 1);
    if (!__all_sync(0xffffffffu, in)) break;
  }
}

// Sequences without rows keep their state: out = in (0 where there is none).  By one block.
__device__ __forceinline__ void pass_empty(const ScanArgs& a, const float* in, float* out, int c0, int block, int blocks) {
  if (out == nullptr || (a.cu == nullptr && a.L > 0)) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int64_t b = int64_t(block) * kWarps + warp; b < a.B; b += int64_t(blocks) * kWarps) {
    bool empty = a.cu == nullptr && a.L == 0;
    if (a.cu != nullptr) {
      const int32_t lo = a.cu[b], hi = a.cu[b + 1];
      empty = hi <= lo;
      if ((hi < lo || lo < 0 || hi > a.T) && lane == 0 && c0 == 0) atomicOr(a.err, kDevErrUnsortedGroups);
    }
    if (!empty) continue;
    for (int c = c0 + lane; c < min(c0 + kStrip, a.H); c += 32) out[b * a.H + c] = in ? in[b * a.H + c] : 0.f;
  }
}

template <class T, int kForm, bool kPair>
__global__ void __launch_bounds__(kWarps * 32) scan_fwd_kernel(const ScanArgs a) {
  __shared__ TileRows rows;
  __shared__ float2 map_a[kWarps][32], map_b[kWarps][32];
  __shared__ int cut[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c0 = blockIdx.x * kStrip, c = c0 + 2 * lane, left = a.H - c;
  const T* gate = static_cast<const T*>(a.gate);
  const T* value = static_cast<const T*>(a.value);
  T* y = static_cast<T*>(a.y);
  float2 carry = make_float2(0.f, 0.f);
  const auto initial = [&](int b) {
    return a.h0 ? load2<kPair>(a.h0 + int64_t(b) * a.H + c, left) : make_float2(0.f, 0.f);
  };
  pass_empty(a, a.h0, a.final_state, c0, 0, 1);
  for (int64_t row0 = 0; row0 < a.T; row0 += kTile) {
    if (warp == 0) mark_rows(a, row0, rows, lane);
    if (a.states && warp == kWarps - 1)
      store2<kPair>(a.states + row0 / kTile * a.H + c, carry.x, carry.y, left);
    const int r = warp * kRows;
    const int n = static_cast<int>(min(int64_t(kRows), a.T - row0 - r));   // may be negative
    float2 na[kRows], v[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      na[i] = v[i] = make_float2(0.f, 0.f);
      if (i < n) {
        na[i] = load2<kPair>(gate + (row0 + r + i) * a.gate_ld + c, left);
        v[i] = load2<kPair>(value + (row0 + r + i) * a.value_ld + c, left);
      }
    }
    __syncthreads();   // rows
    float2 A = make_float2(1.f, 1.f), h = make_float2(0.f, 0.f);
    bool has_cut = false;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      na[i].x = one_minus_a<kForm>(na[i].x);
      na[i].y = one_minus_a<kForm>(na[i].y);
      if (r + i < rows.lo || r + i >= rows.hi) continue;
      const int b = rows.start[r + i];
      if (b >= 0) {
        h = initial(b);
        has_cut = true;
      }
      h.x = step<kForm>(h.x, na[i].x, v[i].x);
      h.y = step<kForm>(h.y, na[i].y, v[i].y);
      A.x = fmaf(-na[i].x, A.x, A.x);
      A.y = fmaf(-na[i].y, A.y, A.y);
    }
    map_a[warp][lane] = A;
    map_b[warp][lane] = h;
    if (lane == 0) cut[warp] = has_cut;
    __syncthreads();
    float2 in = carry;   // the state that enters this warp's rows
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w == warp) in = carry;
      const float2 pa = map_a[w][lane], pb = map_b[w][lane];
      carry.x = cut[w] ? pb.x : fmaf(pa.x, carry.x, pb.x);
      carry.y = cut[w] ? pb.y : fmaf(pa.y, carry.y, pb.y);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (r + i < rows.lo || r + i >= rows.hi) {
        if (a.fill && i < n) store2<kPair>(y + (row0 + r + i) * a.H + c, 0.f, 0.f, left);
        continue;
      }
      const int b = rows.start[r + i], e = rows.end[r + i];
      if (b >= 0) in = initial(b);
      in.x = step<kForm>(in.x, na[i].x, v[i].x);
      in.y = step<kForm>(in.y, na[i].y, v[i].y);
      store2<kPair>(y + (row0 + r + i) * a.H + c, in.x, in.y, left);
      if (e >= 0 && a.final_state) store2<kPair>(a.final_state + int64_t(e) * a.H + c, in.x, in.y, left);
    }
    __syncthreads();   // rows and maps are free
  }
}

template <class T, int kForm, bool kPair>
__global__ void __launch_bounds__(kWarps * 32) scan_bwd_kernel(const ScanArgs a) {
  __shared__ TileRows rows;
  __shared__ float2 map_a[kWarps][32], map_b[kWarps][32], map_e[kWarps][32];
  __shared__ int cut_h[kWarps], cut_e[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c0 = blockIdx.x * kStrip, c = c0 + 2 * lane, left = a.H - c;
  const T* gate = static_cast<const T*>(a.gate);
  const T* value = static_cast<const T*>(a.value);
  const T* dy = static_cast<const T*>(a.dy);
  T* dgate = static_cast<T*>(a.dgate);
  T* dvalue = static_cast<T*>(a.dvalue);
  float2 back = make_float2(0.f, 0.f);   // E of the row after the tile
  const auto of_seq = [&](const float* p, int b) {
    return p ? load2<kPair>(p + int64_t(b) * a.H + c, left) : make_float2(0.f, 0.f);
  };
  pass_empty(a, a.dfinal, a.dinit, c0, 0, 1);
  const int64_t tiles = (a.T + kTile - 1) / kTile;
  for (int64_t tile = tiles - 1; tile >= 0; --tile) {
    const int64_t row0 = tile * kTile;
    if (warp == 0) mark_rows(a, row0, rows, lane);
    const int r = warp * kRows;
    const int n = static_cast<int>(min(int64_t(kRows), a.T - row0 - r));   // may be negative
    float2 na[kRows], v[kRows], d[kRows], hp[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      na[i] = v[i] = d[i] = make_float2(0.f, 0.f);
      if (i < n) {
        na[i] = load2<kPair>(gate + (row0 + r + i) * a.gate_ld + c, left);
        v[i] = load2<kPair>(value + (row0 + r + i) * a.value_ld + c, left);
        d[i] = load2<kPair>(dy + (row0 + r + i) * a.dy_ld + c, left);
      }
    }
    __syncthreads();   // rows
    float2 A = make_float2(1.f, 1.f), h = make_float2(0.f, 0.f), E = make_float2(0.f, 0.f);
    bool ch = false, ce = false;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      na[i].x = one_minus_a<kForm>(na[i].x);
      na[i].y = one_minus_a<kForm>(na[i].y);
      if (r + i < rows.lo || r + i >= rows.hi) continue;
      const int b = rows.start[r + i];
      if (b >= 0) {
        h = of_seq(a.h0, b);
        ch = true;
      }
      h.x = step<kForm>(h.x, na[i].x, v[i].x);
      h.y = step<kForm>(h.y, na[i].y, v[i].y);
      A.x = fmaf(-na[i].x, A.x, A.x);
      A.y = fmaf(-na[i].y, A.y, A.y);
    }
#pragma unroll
    for (int i = kRows - 1; i >= 0; --i) {
      if (r + i < rows.lo || r + i >= rows.hi) continue;
      const int e = rows.end[r + i];
      if (e >= 0) {
        E = of_seq(a.dfinal, e);
        ce = true;
      }
      E.x += d[i].x;
      E.y += d[i].y;
      E.x = fmaf(-na[i].x, E.x, E.x);
      E.y = fmaf(-na[i].y, E.y, E.y);
    }
    map_a[warp][lane] = A;
    map_b[warp][lane] = h;
    map_e[warp][lane] = E;
    if (lane == 0) {
      cut_h[warp] = ch;
      cut_e[warp] = ce;
    }
    __syncthreads();
    float2 in = load2<kPair>(a.states + tile * a.H + c, left);
    for (int w = 0; w < warp; ++w) {
      const float2 pa = map_a[w][lane], pb = map_b[w][lane];
      in.x = cut_h[w] ? pb.x : fmaf(pa.x, in.x, pb.x);
      in.y = cut_h[w] ? pb.y : fmaf(pa.y, in.y, pb.y);
    }
    float2 out = back;
#pragma unroll
    for (int w = kWarps - 1; w >= 0; --w) {
      if (w == warp) out = back;
      const float2 pa = map_a[w][lane], pe = map_e[w][lane];
      back.x = cut_e[w] ? pe.x : fmaf(pa.x, back.x, pe.x);
      back.y = cut_e[w] ? pe.y : fmaf(pa.y, back.y, pe.y);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (r + i < rows.lo || r + i >= rows.hi) continue;
      const int b = rows.start[r + i];
      if (b >= 0) in = of_seq(a.h0, b);
      hp[i] = in;
      in.x = step<kForm>(in.x, na[i].x, v[i].x);
      in.y = step<kForm>(in.y, na[i].y, v[i].y);
    }
#pragma unroll
    for (int i = kRows - 1; i >= 0; --i) {
      if (r + i < rows.lo || r + i >= rows.hi) {
        if (i < n) {
          store2<kPair>(dgate + (row0 + r + i) * a.H + c, 0.f, 0.f, left);
          store2<kPair>(dvalue + (row0 + r + i) * a.H + c, 0.f, 0.f, left);
        }
        continue;
      }
      const int b = rows.start[r + i], e = rows.end[r + i];
      if (e >= 0) out = of_seq(a.dfinal, e);
      const float2 D = make_float2(d[i].x + out.x, d[i].y + out.y);
      out.x = fmaf(-na[i].x, D.x, D.x);   // E
      out.y = fmaf(-na[i].y, D.y, D.y);
      float2 df, dv = D;
      if constexpr (kForm == kFormSigmoid) {
        dv = make_float2(D.x * na[i].x, D.y * na[i].y);
        df = make_float2(out.x * na[i].x * (hp[i].x - v[i].x), out.y * na[i].y * (hp[i].y - v[i].y));
      } else {
        df = make_float2(out.x * hp[i].x, out.y * hp[i].y);
      }
      store2<kPair>(dgate + (row0 + r + i) * a.H + c, df.x, df.y, left);
      store2<kPair>(dvalue + (row0 + r + i) * a.H + c, dv.x, dv.y, left);
      if (b >= 0 && a.dinit) store2<kPair>(a.dinit + int64_t(b) * a.H + c, out.x, out.y, left);
    }
    __syncthreads();   // rows and maps are free
  }
}

template <class T, int kForm>
__global__ void __launch_bounds__(256) scan_step_kernel(const T* gate, const T* value, const float* state, int64_t B, int H,
                                                        int64_t gate_ld, int64_t value_ld, T* y, float* state_out) {
  const int64_t n = B * H;
  for (int64_t i = blockIdx.x * int64_t(256) + threadIdx.x; i < n; i += gridDim.x * int64_t(256)) {
    const int64_t b = i / H;
    const int c = static_cast<int>(i - b * H);
    const float h = step<kForm>(state[i], one_minus_a<kForm>(to_float(gate[b * gate_ld + c])),
                                to_float(value[b * value_ld + c]));
    state_out[i] = h;
    from_float(h, y[i]);
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

// rows and vectors can be read two channels at a time
bool pairs_of(const ScanArgs& a, int dtype) {
  const size_t n = 2 * static_cast<size_t>(dtype_bytes(dtype));
  const auto at = [](const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; };
  for (const void* p : {a.gate, a.value, a.dy, static_cast<const void*>(a.y), static_cast<const void*>(a.dgate),
                        static_cast<const void*>(a.dvalue)})
    if (!at(p, n)) return false;
  for (const void* p : {static_cast<const void*>(a.h0), static_cast<const void*>(a.dfinal),
                        static_cast<const void*>(a.final_state), static_cast<const void*>(a.states),
                        static_cast<const void*>(a.dinit)})
    if (!at(p, 8)) return false;
  return a.H % 2 == 0 && a.gate_ld % 2 == 0 && a.value_ld % 2 == 0 && a.dy_ld % 2 == 0;
}

template <class T, int kForm>
cudaError_t launch_scan(const ScanArgs& a, bool bwd, bool pair, cudaStream_t s) {
  const int grid = (a.H + kStrip - 1) / kStrip;
  if (bwd)
    (pair ? scan_bwd_kernel<T, kForm, true> : scan_bwd_kernel<T, kForm, false>)<<<grid, kWarps * 32, 0, s>>>(a);
  else
    (pair ? scan_fwd_kernel<T, kForm, true> : scan_fwd_kernel<T, kForm, false>)<<<grid, kWarps * 32, 0, s>>>(a);
  return cudaGetLastError();
}
template <class T>
cudaError_t launch_scan(const ScanArgs& a, int form, bool bwd, bool pair, cudaStream_t s) {
  return form == kFormSigmoid ? launch_scan<T, kFormSigmoid>(a, bwd, pair, s) : launch_scan<T, kFormLog>(a, bwd, pair, s);
}

molt_status launch(const molt_scan_desc* d, ScanArgs& a, bool bwd, cudaStream_t s) {
  molt_status st;
  a.err = device_status_word(&st);
  if (!a.err) return st;
  const bool pair = pairs_of(a, d->dtype);
  const cudaError_t e = d->dtype == MOLT_FP32   ? launch_scan<float>(a, d->form, bwd, pair, s)
                        : d->dtype == MOLT_FP16 ? launch_scan<__half>(a, d->form, bwd, pair, s)
                                                : launch_scan<__nv_bfloat16>(a, d->form, bwd, pair, s);
  if (e != cudaSuccess) return cuda_fail(e, "gated scan");
  note_launches(1);
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

molt_status molt_gated_scan_fwd(const molt_scan_desc* desc, const void* gate, const void* value, const float* initial_state,
                                const int32_t* cu_seqlens, void* y, float* final_state, float* states,
                                cudaStream_t stream) {
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
  ScanArgs a = base_args(desc, cu_seqlens);
  a.gate = gate;
  a.value = value;
  a.h0 = initial_state;
  a.y = y;
  a.final_state = final_state;
  a.states = states;
  a.fill = desc->fill_outside != 0;
  return launch(desc, a, false, stream);
}

molt_status molt_gated_scan_bwd(const molt_scan_desc* desc, const void* dy, const void* gate, const void* value,
                                const float* states, const float* initial_state, const int32_t* cu_seqlens,
                                const float* dfinal_state, void* dgate, void* dvalue, float* dinitial_state,
                                cudaStream_t stream) {
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
  return launch(desc, a, true, stream);
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
