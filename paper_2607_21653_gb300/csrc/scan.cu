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
// together: a tile is 128 rows (64 of the forward in fp32) by 64 channels, a warp has 16 (8)
// rows of it, a lane two channels.  Every warp composes its rows' maps; the maps of a tile's
// warps, and of the tiles of a cluster, are folded in order; and then every warp goes through
// its rows again from the state that it now knows.  The backward's E is the same from the other end; h it forms
// again from the states that the forward kept at every 128th row.  A row that begins a
// sequence cuts: what comes before is not multiplied by zero but left out, so that an
// infinite or NaN state stays in its sequence.
//
// A row is held as m = a - 1: with a as a float near 1 the memory 1 / (1 - a) of a
// channel would be off by 2^-24 / (1 - a); h + m (h - v) and h + m h + v need no a at all.  But of
// a near 0, which 1 + m has to 2^-24 of 1, h_t, E_t and dgate are multiples: such a row is held as a
// itself, h_t = v + a (h - v) and a h + v, with a bit that says so: in fp32 where a is below 1/2 (log: 0.7), in
// 16 bits where it is below 2^-7.  Above that 1 + m is off by 2^-15 of a at most, a sixteenth of an fp16
// result's rounding, and a warp's rows of which none is below take no selects.
//
// Layout: a strip of channels belongs to a cluster of up to eight blocks, which take a
// tile each, exchange their maps through one another's shared memory (512 bytes to each
// peer) and go on together, so that the inputs are read once and a super step of 1024 rows
// costs one exchange.  Of two further warps one brings the tiles ahead (TMA, and from
// cu_seqlens which rows begin and end a sequence), the other folds the maps.  Few strips and
// many rows are cut into segments besides: a first launch folds each segment's map, the second
// starts from what precedes its own.  Rows that TMA cannot take (an odd number of bytes, any
// address) are copied in the 16-byte words that hold them, in strips of 56 (fp32: 60) channels.
//
// Bound by a step's chain (maps, exchange, results), with memory and what the SM issues close
// behind: bf16, 65536 x 4096 in four sequences 305 us forward (238 for its bytes at 6.8 TB/s),
// 32768 x 2048 in one 147 us backward (99).  Also
// tried: tiles of 64 rows with three blocks to an SM (482 us for the first), the same a step ahead
// of the exchange (384), 128 rows a step ahead with m formed twice (362: the exponentials), one
// block of 16 warps a step ahead (399; narrow ones gain, 32768 x 1024 72 us for 89, but not so much).
#include <algorithm>
#include <atomic>
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>
#include <initializer_list>
#include <type_traits>

#include "molt_internal.cuh"
#include "ptx.cuh"
#include "vec.cuh"

namespace molt {
namespace {

constexpr int kStateRows = 128;          // rows between kept states
constexpr int kWarps = 8;
constexpr int kHalf = 8;                 // rows that a warp brings into registers at a time
// Halves of a warp's rows: two, or one of the forward in fp32, whose tiles have twice the
// bytes.  The backward's tile is the rows between two kept states.
template <class T, bool kBwd>
constexpr int kHalves = kBwd || sizeof(T) == 2 ? 2 : 1;
template <class T, bool kBwd>
constexpr int kTile = kWarps * kHalves<T, kBwd> * kHalf;
static_assert(kTile<float, true> == kStateRows && kStateRows % kTile<float, false> == 0);
constexpr int kThreads = 32 * (kWarps + 2);
// Channels of a block: 64, or as many as fill a row of the same bytes from any place in a 16-byte
// word.
template <class T, bool kFast>
constexpr int kStrip = kFast ? 64 : sizeof(T) == 2 ? 56 : 60;
constexpr int kMaxCluster = 8;
constexpr int kFormSigmoid = 0, kFormLog = 1;
constexpr float kLog2e = 1.4426950408889634f;
// Gates below it are held as a and not as a - 1.
template <class T, int kForm>
constexpr float kLowGate = sizeof(T) == 2 ? -4.875f : kForm == kFormSigmoid ? 0.f : -0.35f;

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
  CUtensorMap gate, value, dy;   // boxes of 64 channels by a tile's rows
  CUtensorMap out0, out1;        // y, or dgate and dvalue: boxes of 64 channels by a warp's rows
};

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ F2 zero2() { return f2(0.f, 0.f); }
__device__ __forceinline__ F2 sub2(F2 a, F2 b) { return fma2(b, f2(-1.f), a); }

// m = a - 1 of two gates, and a.  sigmoid: -1 / (1 + e^f), no digits lost on either side.  log: e^f - 1,
// by its series where the difference would lose digits (the first term left out is
// 0.35^7 / 8! of the first, 1.6e-8)
template <int kForm>
__device__ __forceinline__ F2 decay(F2 f, F2& a) {
  const F2 x = mul2(f, f2(kLog2e)), e = f2(ex2_approx(x.x()), ex2_approx(x.y()));
  if constexpr (kForm == kFormSigmoid) {
    const F2 m = f2(rcp_approx(-1.f - e.x()), rcp_approx(-1.f - e.y()));
    a = mul2(e, mul2(m, f2(-1.f)));
    return m;
  } else {
    a = e;
    F2 p = f2(1.f / 5040.f);
    p = fma2(p, f, f2(1.f / 720.f));
    p = fma2(p, f, f2(1.f / 120.f));
    p = fma2(p, f, f2(1.f / 24.f));
    p = fma2(p, f, f2(1.f / 6.f));
    p = fma2(p, f, f2(0.5f));
    p = fma2(p, f, f2(1.f));
    p = mul2(p, f);
    return f2(fabsf(f.x()) < 0.35f ? p.x() : e.x() - 1.f, fabsf(f.y()) < 0.35f ? p.y() : e.y() - 1.f);
  }
}
// Channels with a bit (of two) have x, the others y.
__device__ __forceinline__ F2 pick2(uint32_t bits, F2 x, F2 y) {
  return f2(bits & 1u ? x.x() : y.x(), bits & 2u ? x.y() : y.y());
}
// m of two gates, but a itself of those that are below `from`, which have their bit in `low`
template <int kForm>
__device__ __forceinline__ F2 coefficient(F2 f, float from, uint32_t& low) {
  F2 a;
  const F2 m = decay<kForm>(f, a);
  low = (f.x() < from ? 1u : 0u) | (f.y() < from ? 2u : 0u);
  return pick2(low, a, m);
}
// c A, c = m (bit 0 of a channel) or a (bit 1): a A
template <bool kSelect>
__device__ __forceinline__ F2 decayed(F2 A, F2 c, uint32_t low) {
  return fma2(c, A, kSelect ? pick2(low, zero2(), A) : A);
}
// h_t from h_{t-1}: h + m (h - v) = v + a (h - v);  (h + m h) + v = a h + v
template <int kForm, bool kSelect>
__device__ __forceinline__ F2 step(F2 h, F2 c, F2 v, uint32_t low) {
  if constexpr (kForm == kFormSigmoid) return fma2(c, sub2(h, v), kSelect ? pick2(low, v, h) : h);
  return add2(decayed<kSelect>(h, c, low), v);
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
// The same of fp32 if `on`, else zeros, by predicate: several loads go out together.
template <bool kPair>
__device__ __forceinline__ F2 load2_if(bool on, const float* p, int left) {
  float x = 0.f, y = 0.f;
  if constexpr (kPair) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %3, 0;\n\t@q ld.global.v2.f32 {%0, %1}, [%2];\n}"
                 : "+f"(x), "+f"(y)
                 : "l"(p), "r"(int(on && left > 1)));
  } else {
    asm volatile("{\n\t.reg .pred q, r;\n\tsetp.ne.b32 q, %3, 0;\n\tsetp.ne.b32 r, %4, 0;\n\t@q ld.global.f32 %0, [%2];\n\t@r ld.global.f32 %1, [%2+4];\n}"
                 : "+f"(x), "+f"(y)
                 : "l"(p), "r"(int(on && left > 0)), "r"(int(on && left > 1)));
  }
  return f2(x, y);
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

__device__ __forceinline__ void store32_if(bool on, void* p, uint32_t v) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q st.global.b32 [%0], %1;\n}" ::"l"(p), "r"(v), "r"(int(on)) : "memory");
}
__device__ __forceinline__ void store16_if(bool on, void* p, uint32_t v) {
  asm volatile("{\n\t.reg .pred q;\n\t.reg .b16 h, g;\n\tsetp.ne.b32 q, %2, 0;\n\tmov.b32 {h, g}, %1;\n\t@q st.global.b16 [%0], h;\n}" ::"l"(p),
               "r"(v), "r"(int(on))
               : "memory");
}
// A row's results, two to a lane, n channels from p on: as words, of neighbours' halves where the row
// begins inside one.  Predicates and no branches: those took longer than the rest of a row.
template <class T>
__device__ __forceinline__ void store_row(T* p, F2 x, int n, int lane) {
  const int left = n - 2 * lane;
  if constexpr (sizeof(T) == 4) {
    store32_if(left > 0, p + 2 * lane, __float_as_uint(x.x()));
    store32_if(left > 1, p + 2 * lane + 1, __float_as_uint(x.y()));
  } else {
    const bool off = reinterpret_cast<uintptr_t>(p) & 2;
    const uint32_t own = pack2(x.x(), x.y(), p), next = __shfl_down_sync(0xffffffffu, own, 1);
    T* const q = p + 2 * lane + (off ? 1 : 0);
    const int rest = left - (off ? 1 : 0);   // channels from q on
    const uint32_t w = off ? __byte_perm(own, next, 0x5432) : own;
    store16_if(off && lane == 0 && n > 0, p, own);
    store32_if(rest > 1, q, w);
    store16_if(rest == 1, q, w);
  }
}

// Which rows of a tile begin or end a sequence (a bit each), and which one (of those rows);
// lo and hi: the tile's rows that are in any.
template <int kN>
struct TileRows {
  uint32_t starts[kN / 32], ends[kN / 32];
  int seq[kN];
  int lo, hi;
};

// The states of sequence b in the strip of channels from c0 on, which will be wanted soon (32768 x 2048
// in 1024 sequences with initial states 183 -> 168 us; 136 with the loads by predicate).
__device__ __forceinline__ void fetch_states(const float* p, const ScanArgs& a, int64_t b, int c0) {
  if (p == nullptr) return;
  p += b * a.H + c0;
  asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
  if (c0 + 63 < a.H) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + 32));
}

// Fills `t` for the rows from row0 on; by one warp.  Returns the first bound that is not below
// row0; `at` is what it returned for the tile before in the walk (at first 0, backwards
// B + 1).
template <int kN, bool kBwd>
__device__ __forceinline__ int64_t mark_rows(const ScanArgs& a, int64_t row0, TileRows<kN>& t, int64_t at, int c0, int lane) {
  const int n = static_cast<int>(a.T - row0 < kN ? a.T - row0 : kN);
  if (lane < kN / 32) t.starts[lane] = t.ends[lane] = 0u;
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
        fetch_states(a.h0, a, b, c0);
      }
      const int64_t e = v + a.L - 1;
      if (e < n) {
        t.seq[e] = static_cast<int>(b);
        atomicOr(&t.ends[e >> 5], 1u << (e & 31));
        if (kBwd) fetch_states(a.dfinal, a, b, c0);
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
      fetch_states(a.h0, a, b, c0);
    }
    if (in && v > 0 && b > 0 && a.cu[b - 1] - row0 < v) {
      t.seq[v - 1] = static_cast<int>(b - 1);
      atomicOr(&t.ends[(v - 1) >> 5], 1u << ((v - 1) & 31));
      if (kBwd) fetch_states(a.dfinal, a, b - 1, c0);
    }
    if (!__all_sync(0xffffffffu, in)) break;
  }
  __syncwarp();
  return found;
}

// Sequences without rows keep their state: out = in (0 where there is none).
__device__ __forceinline__ void pass_empty(const ScanArgs& a, const float* in, float* out, int c0, int wide, int block, int blocks) {
  if (out == nullptr || (a.cu == nullptr && a.L > 0)) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int64_t b = int64_t(block) * kWarps + warp; b < a.B; b += int64_t(blocks) * kWarps) {
    if (a.cu != nullptr && a.cu[b + 1] > a.cu[b]) continue;
    for (int c = c0 + lane; c < min(c0 + wide, a.H); c += 32) out[b * a.H + c] = in ? in[b * a.H + c] : 0.f;
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

// An affine map of two channels' states, h -> A h + b, with a cut in the signs of both A (which are
// otherwise not below 0).
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
  const bool cut = (n.x < 0.f && n.y < 0.f) || (m.x < 0.f && m.y < 0.f);
  return make_float4(cut ? -1.f : m.x * n.x, cut ? -1.f : m.y * n.y, b.x(), b.y());
}

// What the warps of a block and the blocks of a cluster tell one another in a step.  warps:
// the map of each warp's rows, then in x and y what enters them.  tiles: the maps of all
// blocks' tiles, two slots, so that a peer a step ahead does not write what is still read.
struct Exchange {
  float4 warps[kWarps][32];
  float4 tiles[2][kMaxCluster][32];
};

// the eight warps with rows, and the one that folds
__device__ __forceinline__ void maps_sync() { asm volatile("bar.sync 1, %0;" ::"n"((kWarps + 1) * 32) : "memory"); }
// the latter's answer: the warps that wait for it at a barrier issue nothing meanwhile (polling an
// mbarrier they took a third of the SM's instructions)
__device__ __forceinline__ void folded() { asm volatile("bar.arrive 2, %0;" ::"n"((kWarps + 1) * 32) : "memory"); }
__device__ __forceinline__ void wait_folded() { asm volatile("bar.sync 2, %0;" ::"n"((kWarps + 1) * 32) : "memory"); }

// A stage is the tile's rows of each tensor, 64 channels' bytes each.  As many as leave room for
// two blocks to an SM (fp32 backward: one).
template <class T>
constexpr int kPitch = 64 * static_cast<int>(sizeof(T));
template <bool kBwd, bool kMapOnly>
constexpr int kStagesOf = kBwd && !kMapOnly ? 2 : 3;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// kRows rows' channels, n of them from `row` on, to shared memory in the 16-byte words that hold them,
// several rows at a time.  (20000 x 1031 forward 124 us; in words of four bytes, as many copies again
// three times, 150.)
template <class T, int kRows>
__device__ __forceinline__ void copy_rows(uint32_t dst, const T* row, int64_t ld, int n, int lane) {
  constexpr int kWords = kPitch<T> / 16, kAtOnce = 32 / kWords;
  const int word = lane % kWords, sub = lane / kWords;
  uintptr_t p = reinterpret_cast<uintptr_t>(row + sub * ld);
  dst += sub * kPitch<T> + word * 16;
#pragma unroll
  for (int i = 0; i < kRows / kAtOnce; ++i) {
    const int off = static_cast<int>(p & 15);
    if (word * 16 < off + n * static_cast<int>(sizeof(T)))
      cp_async16(dst + i * kAtOnce * kPitch<T>, reinterpret_cast<const void*>(p - off + word * 16));
    p += static_cast<uintptr_t>(kAtOnce * ld * static_cast<int64_t>(sizeof(T)));
  }
}
// The same for the first or last rows of the tensor, a number of them that need not be kRows, element by
// element: nothing beside them is read.
template <class T>
__device__ __forceinline__ void copy_edge_rows(uint8_t* dst, const T* row, int64_t ld, int rows, int n, int lane) {
  for (int i = 0; i < rows; ++i, row += ld, dst += kPitch<T>) {
    T* const at = reinterpret_cast<T*>(dst + (reinterpret_cast<uintptr_t>(row) & 15));
    for (int k = lane; k < n; k += 32) at[k] = row[k];
  }
}

// Two values of a row as they are in memory.
template <class T>
struct Raw {
  uint32_t w;
  __device__ __forceinline__ F2 f() const {
    float lo, hi;
    unpack2(w, static_cast<const T*>(nullptr), lo, hi);
    return f2(lo, hi);
  }
};
template <>
struct Raw<float> {
  F2 w;
  __device__ __forceinline__ F2 f() const { return w; }
};

// Bits of kLowGate in 16 bits.  Two numbers of one sign compare as their bits do, and one below 0 has more
// than any above: a maximum finds the gates furthest below 0.
template <class T>
constexpr uint32_t kLowBits = std::is_same<T, __half>::value ? 0xc4e0u : 0xc09cu;

template <class T, bool kBwd>
constexpr int kBlocksPerSM = kBwd && sizeof(T) == 4 ? 1 : 2;

// kBwd: rows from the last one backwards.  kMapOnly: a segment's map alone.  kFast: tiles by TMA
// and pairs of channels; else words and elements one by one from any address.
template <class T, int kForm, bool kBwd, bool kMapOnly, bool kFast>
__global__ void __launch_bounds__(kThreads, (kBlocksPerSM<T, kBwd>)) scan_kernel(const __grid_constant__ ScanMaps maps,
                                                                               const ScanArgs a) {
  // tensors of a tile: gate, value (the backward's map needs none), dy
  constexpr bool kGrads = kBwd && !kMapOnly, kValue = !kBwd || !kMapOnly;
  constexpr int kTensors = kGrads ? 3 : 2, kV = 1, kD = kValue ? 2 : 1;
  constexpr int kStages = kStagesOf<kBwd, kMapOnly>, kN = kTile<T, kBwd>, kParts = kHalves<T, kBwd>, kRows = kParts * kHalf;
  constexpr uint32_t kAll = (1u << kHalf) - 1u;
  constexpr bool kSelect = sizeof(T) == 4;   // rows held as a are as common as others
  constexpr int kRowBytes = kPitch<T>, kS = kStrip<T, kFast>;
  constexpr int kTensorBytes = kN * kRowBytes, kStageBytes = kTensors * kTensorBytes;
  extern __shared__ __align__(128) uint8_t smem_raw[];
  __shared__ __align__(16) Exchange ex;
  __shared__ float2 h_maps[kGrads ? kWarps : 1][32];   // b of the maps of h, then h before each warp's rows
  __shared__ TileRows<kN> rows_sh[kStages];
  __shared__ __align__(8) uint64_t full_bar[kStages], empty_bar[kStages], peer_bar[2];
  __shared__ int abort_sh;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  volatile int* abort_flag = &abort_sh;
  uint32_t size;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(size));
  const int S = static_cast<int>(size), rank = static_cast<int>(cluster_ctarank());
  const int strip = blockIdx.x / S, strips = gridDim.x / S;
  const int c0 = strip * kS, c = c0 + 2 * lane, wide = min(kS, a.H - c0), left = wide - 2 * lane;
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
        tma_load_2d(dst, &maps.gate, bar, c0, tile * kN);
        if constexpr (kValue) tma_load_2d(dst + kV * kTensorBytes, &maps.value, bar, c0, tile * kN);
        if constexpr (kBwd) tma_load_2d(dst + kD * kTensorBytes, &maps.dy, bar, c0, tile * kN);
      }
      ++issued;
      at = mark_rows<kN, kBwd>(a, int64_t(tile) * kN, rows_sh[st], at, c0, lane);
      if (lane == 0) mbar_arrive(smem_u32(&full_bar[st]));
    }
    // copies land in this block's memory: wait for the last ones before it may exit
    if (lane == 0)
      for (int k = max(0, issued - kStages); k < issued; ++k)
        mbar_wait_drain(smem_u32(&full_bar[k % kStages]), (k / kStages) & 1u, a.err);
  } else if (warp == kWarps + 1) {
    // folds a step's maps: the tile's, for all blocks of the cluster, and what enters each warp's rows
    F2 carry = zero2();           // the state before the step (E after it)
    float4 total = identity;
    if constexpr (!kMapOnly) {
      for (int s = kBwd ? static_cast<int>(gridDim.y) - 1 : 0; s != seg; s += kBwd ? -1 : 1)
        carry = apply(a.seg_maps[(int64_t(s) * strips + strip) * 32 + lane], carry);
    }
    for (int k = 0; k < n_steps; ++k) {
      const int tile = tile_of(k), slot = k & 1;
      const uint32_t bar = smem_u32(&peer_bar[slot]);
      if (S > 1 && lane == 0) mbar_arrive_expect_tx(bar, (S - 1) * 512);
      F2 h = zero2();   // backward: the state before the tile
      if constexpr (kGrads)
        if (tile >= 0) h = load2<kFast>(a.states + int64_t(tile) * a.H + c, left);
      maps_sync();
      float4 m[kWarps], pair[4], quad[2];   // in the order of the walk
      float4(*const warps)[32] = ex.warps;
#pragma unroll
      for (int j = 0; j < kWarps; ++j) m[j] = warps[kBwd ? kWarps - 1 - j : j][lane];
      float4 of_h[kGrads ? kWarps : 1];
      if constexpr (kGrads) {
#pragma unroll
        for (int j = 0; j < kWarps; ++j) {
          const float2 b = h_maps[kWarps - 1 - j][lane];
          const bool cut = __float_as_int(m[j].x) < 0, cut_h = __float_as_int(m[j].y) < 0;
          const float x = fabsf(m[j].x), y = fabsf(m[j].y);
          of_h[j] = make_float4(cut_h ? -1.f : x, cut_h ? -1.f : y, b.x, b.y);
          m[j].x = cut ? -1.f : x;
          m[j].y = cut ? -1.f : y;
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) pair[j] = compose(m[2 * j], m[2 * j + 1]);
#pragma unroll
      for (int j = 0; j < 2; ++j) quad[j] = compose(pair[2 * j], pair[2 * j + 1]);
      const float4 own = compose(quad[0], quad[1]);
      // one copy to each peer, all at once (a lane's 16 bytes to each in turn took 190 clocks a peer)
      ex.tiles[slot][rank][lane] = own;
      if (S > 1) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane < S && lane != rank) {
          const uint32_t at = smem_u32(&ex.tiles[slot][rank][0]);
          bulk_copy_cluster(mapa_shared(at, lane), at, 512, mapa_shared(bar, lane));
        }
      }
      if constexpr (kGrads) {   // while the peers' are on their way
#pragma unroll
        for (int j = kWarps - 1; j >= 0; --j) {
          h_maps[kWarps - 1 - j][lane] = make_float2(h.x(), h.y());
          h = apply(of_h[j], h);
        }
      }
      // (a wait that runs out raises the block's flag; what follows is then of no use, but ends)
      if (S > 1) mbar_wait(bar, (k >> 1) & 1u, abort_flag, a.err);
      constexpr int kTiles = kMaxCluster;
      float4 t[kTiles];
#pragma unroll
      for (int p = 0; p < kTiles; ++p) t[p] = ex.tiles[slot][p][lane];   // (of no use from S on)
      F2 here = carry;
      float4 upto = identity;
#pragma unroll
      for (int p = 0; p < kTiles; ++p) {
        if constexpr (kMapOnly) {
          if (p < S) upto = compose(upto, t[p]);
        } else {
          here.v = p == rank ? carry.v : here.v;
          const F2 next = apply(t[p], carry);
          carry.v = p < S ? next.v : carry.v;
        }
      }
      if constexpr (kMapOnly) {
        total = compose(total, upto);
        folded();
        continue;
      }
      auto put = [&](int j, F2 x) {
        *reinterpret_cast<float2*>(&warps[kBwd ? kWarps - 1 - j : j][lane]) = make_float2(x.x(), x.y());
      };
      const F2 two = apply(pair[0], here), four = apply(quad[0], here), six = apply(pair[2], four);
      put(0, here);
      put(1, apply(m[0], here));
      put(2, two);
      put(3, apply(m[2], two));
      put(4, four);
      put(5, apply(m[4], four));
      put(6, six);
      put(7, apply(m[6], six));
      folded();
      if (!kBwd && a.states && tile >= 0 && tile % (kStateRows / kN) == 0)
        store2<kFast>(a.states + int64_t(tile / (kStateRows / kN)) * a.H + c, here, left);
    }
    if (kMapOnly && rank == 0) a.seg_maps[(int64_t(seg) * strips + strip) * 32 + lane] = total;
  } else {
    if (!kMapOnly && seg == 0) {
      pass_empty(a, kBwd ? a.dfinal : a.h0, kBwd ? a.dinit : a.final_state, c0, kS, rank, S);
      if (strip == 0) check_bounds(a, rank, S);
    }
    const int r0 = warp * kRows;
    // rows that do not come by TMA: every warp copies its own, all stages but one ahead
    const void* const tensor_of[3] = {a.gate, kValue ? a.value : a.dy, a.dy};
    const int64_t ld_of[3] = {a.gate_ld, kValue ? a.value_ld : a.dy_ld, a.dy_ld};
    auto load_rows = [&](int k) {
      const int t = k < n_steps ? tile_of(k) : -1;
      if (t >= 0) {
#pragma unroll
        for (int j = 0; j < kTensors; ++j) {
          uint8_t* const dst = smem_raw + (k % kStages) * kStageBytes + j * kTensorBytes + r0 * kRowBytes;
          const int64_t r = int64_t(t) * kN + r0;
          const T* const src = static_cast<const T*>(tensor_of[j]) + r * ld_of[j] + c0;
          if (r > 0 && r + kRows < a.T)
            copy_rows<T, kRows>(smem_u32(dst), src, ld_of[j], wide, lane);
          else if (r < a.T)
            copy_edge_rows<T>(dst, src, ld_of[j], static_cast<int>(min(int64_t(kRows), a.T - r)), wide, lane);
        }
      }
      cp_async_commit();
    };
    if constexpr (!kFast) {
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
    // a half's rows: m, and the tensors' values.  The forward keeps m of both halves from the maps to
    // the results (its exponentials and reciprocals take as long as half of its bytes), the
    // backward that of the last.
    constexpr int kKept = kBwd ? 1 : kParts;
    F2 kept[kKept][kHalf];
    uint32_t low[kKept];   // two bits to a row: channels held as a
    uint32_t most = 0;     // of a warp's rows: see load_gates
    bool some = false;     // any held as a among the warp's channels (fp32: not asked)
    Raw<T> v[kHalf], d[kHalf];
    for (int k = 0; k < n_steps; ++k) {
      const int st = k % kStages;
      int tile = alive ? tile_of(k) : -1;
      const TileRows<kN>& rows = rows_sh[st];
      if (tile >= 0) {
        if (!mbar_wait(smem_u32(&full_bar[st]), (k / kStages) & 1u, abort_flag, a.err)) {
          alive = false;
          tile = -1;
        }
      }
      const int64_t row = int64_t(tile) * kN + r0;   // the warp's first
      // a bit for each of its rows: begins, ends a sequence; valid: is in one
      uint32_t starts = 0, ends = 0, valid = 0;
      if (tile >= 0) {
        starts = rows.starts[r0 >> 5] >> (r0 & 31) & ((1u << kRows) - 1u);
        ends = rows.ends[r0 >> 5] >> (r0 & 31) & ((1u << kRows) - 1u);
        const int lo = min(max(rows.lo - r0, 0), kRows), hi = min(max(rows.hi - r0, 0), kRows);
        valid = ((1u << hi) - 1u) & ~((1u << lo) - 1u);
        if constexpr (!kFast) {
          load_rows(k + kStages - 1);
          cp_async_wait<kStages - 1>();
          __syncwarp();
        }
      }
      uint8_t* const stage = smem_raw + st * kStageBytes + r0 * kRowBytes;
      // where a tensor's rows begin in their first 16-byte words: of the warp's first row, and from row to row
      uint32_t off[kTensors], off_step[kTensors];
      if constexpr (!kFast) {
#pragma unroll
        for (int j = 0; j < kTensors; ++j) {
          off_step[j] = static_cast<uint32_t>(ld_of[j]) * static_cast<uint32_t>(sizeof(T));
          off[j] = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(tensor_of[j])) + static_cast<uint32_t>(row) * off_step[j] +
                   static_cast<uint32_t>(c0) * static_cast<uint32_t>(sizeof(T));
        }
      }
      // `anew`: from memory whatever has been read before, so that nothing is kept in registers for it
      auto read = [&](int tensor, int i, auto anew) -> Raw<T> {
        using Word = std::conditional_t<decltype(anew)::value, const volatile uint32_t, const uint32_t>;
        const uint8_t* const p = stage + tensor * kTensorBytes + i * kRowBytes;
        Raw<T> r;
        if constexpr (kFast) {
          if constexpr (sizeof(T) == 4)
            r.w.v = *reinterpret_cast<const unsigned long long*>(p + 8 * lane);
          else
            r.w = *reinterpret_cast<Word*>(p + 4 * lane);
        } else {
          const uint32_t o = (off[tensor] + i * off_step[tensor]) & 15u;
          if constexpr (sizeof(T) == 4) {
            const float* const q = reinterpret_cast<const float*>(p + o) + 2 * lane;
            r.w = f2(q[0], q[1]);
          } else {
            Word* const q = reinterpret_cast<Word*>(p + (o & 12u)) + lane;
            r.w = __byte_perm(q[0], q[1], o & 2u ? 0x5432 : 0x3210);
          }
        }
        return r;
      };
      auto get = [&](int tensor, int i) -> Raw<T> { return read(tensor, i, std::false_type{}); };

      constexpr std::true_type kYes{};
      constexpr std::false_type kNo{};
      // a half's bits of `starts` and so on; plain: all of its rows are in one sequence and go on after it
      auto half_of = [&](uint32_t rows_bits, int q) -> uint32_t { return rows_bits >> (q * kHalf) & kAll; };
      auto plain = [&](int q) -> bool { return half_of(valid, q) == kAll && (half_of(starts, q) | half_of(ends, q)) == 0; };
      auto load_values = [&](int q, auto anew) {
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
          if constexpr (kValue) v[i] = read(kV, q * kHalf + i, anew);
          if constexpr (kBwd) d[i] = read(kD, q * kHalf + i, anew);
        }
      };
      // m of the half's rows; `most` becomes at least the bits of each channel's gate that is furthest below 0
      auto load_gates = [&](F2 (&m)[kHalf], int q, auto asked, uint32_t& most) {
        uint32_t w[kHalf] = {};
        F2 unused;
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
          const Raw<T> f = get(0, q * kHalf + i);
          if constexpr (!kSelect) w[i] = f.w;
          m[i] = decay<kForm>(f.f(), unused);
        }
        if constexpr (!kSelect && decltype(asked)::value) {
          most = __vimax3_u16x2(most, w[0], w[1]);
#pragma unroll
          for (int i = 2; i < kHalf; i += 2) most = __vimax3_u16x2(most, w[i], w[i + 1]);
        }
      };
      // the same with a for the gates below, which have their bits in `low`
      auto load_coefficients = [&](F2 (&m)[kHalf], uint32_t& low, int q) {
        low = 0;
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
          uint32_t bits;
          m[i] = coefficient<kForm>(read(0, q * kHalf + i, std::bool_constant<!kSelect>{}).f(), kLowGate<T, kForm>, bits);
          low |= bits << (2 * i);
        }
      };
      // rows outside of every sequence change nothing (no h behind the last one is used)
      auto leave_out = [&](F2 (&m)[kHalf], uint32_t& low, int q) {
        const uint32_t in = half_of(valid, q);
        if (in == kAll) return;
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
          if (in >> i & 1u) continue;
          m[i] = zero2();
          v[i] = d[i] = Raw<T>{};
          low &= ~(3u << (2 * i));
        }
      };
      // what the rows of these bits start from
      auto start_half = [&](const float* p, uint32_t bits, int q, F2 (&x)[kHalf]) {
        if (p == nullptr || bits == 0) {
#pragma unroll
          for (int i = 0; i < kHalf; ++i) x[i] = zero2();
          return;
        }
        int seq[kHalf];   // (of rows without a bit: whatever stands there, and not read by)
#pragma unroll
        for (int i = 0; i < kHalf; ++i) seq[i] = rows.seq[r0 + q * kHalf + i];
#pragma unroll
        for (int i = 0; i < kHalf; ++i) x[i] = load2_if<kFast>(bits >> i & 1u, p + (int64_t(seq[i]) * a.H + c), left);
      };
      auto pick = [](uint32_t bits, int i, F2 x, F2 y) -> F2 { return F2{bits >> i & 1u ? x.v : y.v}; };
      // the half's map of h (A, x), and in a backward walk of E (A, x) and of h (A, z); kCut: rows that begin or
      // end sequences may be among them, kSel: rows held as a
      auto map_half = [&](auto cuts, auto select, const F2 (&m)[kHalf], uint32_t low, int q, float4& of_walk, float4& of_h) {
        constexpr bool kCut = decltype(cuts)::value, kSel = decltype(select)::value;
        const uint32_t s = kCut ? half_of(starts, q) : 0u, e = kCut ? half_of(ends, q) : 0u;
        F2 A = f2(1.f), x = zero2(), z = zero2(), from[kHalf];
        if constexpr (kCut && kValue) start_half(a.h0, s, q, from);
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
          A = decayed<kSel>(A, m[i], low >> (2 * i));
          if constexpr (kValue) z = step<kForm, kSel>(kCut ? pick(s, i, from[i], z) : z, m[i], v[i].f(), low >> (2 * i));
        }
        if constexpr (kBwd) {
          if constexpr (kCut) start_half(a.dfinal, e, q, from);
#pragma unroll
          for (int i = kHalf - 1; i >= 0; --i)
            x = decayed<kSel>(add2(kCut ? pick(e, i, from[i], x) : x, d[i].f()), m[i], low >> (2 * i));
        }
        of_h = pack(Map{A, z}, s != 0);
        of_walk = kBwd ? pack(Map{A, x}, e != 0) : of_h;
      };
      auto take_half = [&](auto select, F2 (&m)[kHalf], uint32_t& low, int q, float4& of_walk, float4& of_h) {
        if constexpr (decltype(select)::value) {
          load_coefficients(m, low, q);
        } else {
          load_gates(m, q, kYes, most);
          low = 0;
        }
        load_values(q, std::bool_constant<!kSelect && decltype(select)::value>{});
        if (plain(q) && decltype(select)::value == kSelect) {
          map_half(kNo, select, m, low, q, of_walk, of_h);
        } else {
          leave_out(m, low, q);
          map_half(kYes, select, m, low, q, of_walk, of_h);
        }
      };

      // ---- the maps of the warp's rows
      float4 mine = identity, mine_h = identity, first_h = identity;   // first_h: the first half's
      if (tile >= 0) {
        auto take = [&](auto select) {
          [[maybe_unused]] float4 w, h;
          take_half(select, kept[0], low[0], 0, mine, mine_h);
          if constexpr (kParts == 2) {
            first_h = mine_h;
            take_half(select, kept[kKept - 1], low[kKept - 1], 1, w, h);
            mine = kBwd ? compose(w, mine) : compose(mine, w);
            if constexpr (kGrads) mine_h = compose(mine_h, h);
          }
        };
        most = 0;
        take(std::bool_constant<kSelect>{});
        // Gates below kLowGate, which are seldom in 16 bits, are found beside the rest, and all is done again
        // (65536 x 4096 forward 305 us; 359 with a branch behind the gates of every half, 400 with the
        // selects always.  Of inputs that have one in every tile 649, backward 1440 for 535; to look for them
        // first where the tile before had some, 559 and 1310, took 4 % of all others)
        if constexpr (!kSelect) {
          // (a channel that there is not may be what an earlier kernel has left in shared memory)
          some = __any_sync(0xffffffffu, ((kFast || left > 0) && (most << 16) > (kLowBits<T> << 16)) ||
                                             ((kFast || left > 1) && most > (kLowBits<T> << 16 | 0xffffu)));
          if (some) take(kYes);
        }
      }
      if constexpr (!kGrads) ex.warps[warp][lane] = mine;
      if constexpr (kGrads) {
        // the maps of E and of h have one A but for their cuts, which go in its signs
        const bool cut = mine.x < 0.f && mine.y < 0.f, cut_h = mine_h.x < 0.f && mine_h.y < 0.f;
        const float2 A = cut ? make_float2(mine_h.x, mine_h.y) : make_float2(mine.x, mine.y);   // (of no use if both are cut)
        ex.warps[warp][lane] = make_float4(copysignf(A.x, cut ? -1.f : 1.f), copysignf(A.y, cut_h ? -1.f : 1.f), mine.z, mine.w);
        h_maps[warp][lane] = make_float2(mine_h.z, mine_h.w);
      }
      give_back();
      maps_sync();
      if constexpr (kMapOnly) {
        if (tile >= 0 && lane == 0) mbar_arrive(smem_u32(&empty_bar[st]));   // (behind the sync)
      }
      // what enters the warp's rows (or: the maps have been read)
      wait_folded();
      if (kMapOnly || tile < 0) continue;
      const float2 entering = *reinterpret_cast<const float2*>(&ex.warps[warp][lane]);
      F2 in = f2(entering.x, entering.y);

      // ---- the rows again.  Where all of the warp's are in sequences their results go out as a box,
      // from where the gates (and dy) have been
      const bool boxed = kFast && valid == (1u << kRows) - 1u && !(kBwd && some);
      auto store_out = [&](T* p, F2 x) {
        if constexpr (kFast)
          store2<true>(p + 2 * lane, x, left);
        else
          store_row(p, x, wide, lane);
      };
      auto to_box = [&](int tensor, int i, F2 x) {
        store2<true>(reinterpret_cast<T*>(stage + tensor * kTensorBytes + i * kRowBytes) + 2 * lane, x, 2);
      };
      // a half whose rows are all in sequences: no branch at every row (65536 x 4096 forward 359 us with one, where it took 310)
      auto out_whole = [&](T* base, int tensor, int i, F2 x) {
        if constexpr (kFast)
          to_box(tensor, i, x);
        else
          store_out(base + (row + i) * a.H + c0, x);
      };
      if constexpr (!kBwd) {
        T* const y = static_cast<T*>(a.y);
#pragma unroll
        for (int q = 0; q < kParts; ++q) {
          if (kParts > 1) load_values(q, kNo);
          if (plain(q) && (!kFast || boxed) && !some) {
#pragma unroll
            for (int i = 0; i < kHalf; ++i) {
              in = step<kForm, kSelect>(in, kept[q][i], v[i].f(), low[q] >> (2 * i));
              out_whole(y, 0, q * kHalf + i, in);
            }
            continue;
          }
          const uint32_t s = half_of(starts, q), e = half_of(ends, q), is = half_of(valid, q);
          if (kParts > 1) leave_out(kept[q], low[q], q);
          F2 h[kHalf];   // first what rows start from, then h
          start_half(a.h0, s, q, h);
          auto walk = [&](auto select) {
#pragma unroll
            for (int i = 0; i < kHalf; ++i)
              h[i] = in = step<kForm, decltype(select)::value>(pick(s, i, h[i], in), kept[q][i], v[i].f(), low[q] >> (2 * i));
          };
          if (some)
            walk(kYes);
          else
            walk(std::bool_constant<kSelect>{});
          if (boxed) {
#pragma unroll
            for (int i = 0; i < kHalf; ++i) to_box(0, q * kHalf + i, h[i]);
          } else {
#pragma unroll
            for (int i = 0; i < kHalf; ++i)
              if (is >> i & 1u)
                store_out(y + (row + q * kHalf + i) * a.H + c0, h[i]);
              else if (a.fill && row + q * kHalf + i < a.T)
                store_out(y + (row + q * kHalf + i) * a.H + c0, zero2());
          }
          if (e != 0 && a.final_state) {
#pragma unroll
            for (int i = 0; i < kHalf; ++i)
              if (e >> i & 1u) store2<kFast>(a.final_state + int64_t(rows.seq[r0 + q * kHalf + i]) * a.H + c, h[i], left);
          }
        }
      } else {
        T* const dg = static_cast<T*>(a.dgate);
        T* const dv = static_cast<T*>(a.dvalue);
        const float2 before = h_maps[warp][lane];
        const F2 h_in = f2(before.x, before.y);
        // dgate and dvalue of a row from D and E and h of the row before
        auto grads = [&](auto select, int i, F2 D, F2 E, F2 hp, F2& df, F2& dval) {
          if constexpr (kForm == kFormSigmoid) {
            const F2 c = kept[0][i], w = decltype(select)::value ? sub2(pick2(low[0] >> (2 * i), f2(1.f), zero2()), c) : mul2(c, f2(-1.f));
            dval = mul2(D, w);
            df = mul2(mul2(E, w), sub2(hp, v[i].f()));
          } else {
            dval = D;
            df = mul2(E, hp);
          }
        };
#pragma unroll 1
        for (int q = kParts - 1; q >= 0; --q) {
          const F2(&m)[kHalf] = kept[0];
          F2 h = q > 0 ? apply(first_h, h_in) : h_in, hp[kHalf], df, dval;   // hp: h of the row before
          const bool again = q < kParts - 1;   // the last one's rows are still there
          if (plain(q) && (!kFast || boxed) && !some) {
            if (again) {
              if constexpr (kSelect)
                load_coefficients(kept[0], low[0], q);
              else
                load_gates(kept[0], q, kNo, most);
              load_values(q, kNo);
            }
#pragma unroll
            for (int i = 0; i < kHalf; ++i) {
              hp[i] = h;
              h = step<kForm, kSelect>(h, m[i], v[i].f(), low[0] >> (2 * i));
            }
#pragma unroll
            for (int i = kHalf - 1; i >= 0; --i) {
              const F2 D = add2(d[i].f(), in);
              in = decayed<kSelect>(D, m[i], low[0] >> (2 * i));   // E
              grads(std::bool_constant<kSelect>{}, i, D, in, hp[i], df, dval);
              out_whole(dg, 0, q * kHalf + i, df);
              out_whole(dv, kD, q * kHalf + i, dval);
            }
            continue;
          }
          const uint32_t s = half_of(starts, q), e = half_of(ends, q), is = half_of(valid, q);
          F2 from[kHalf];
          auto walk = [&](auto select, auto box) {
            constexpr bool kSel = decltype(select)::value;
            if (again) {
              if constexpr (kSel)
                load_coefficients(kept[0], low[0], q);
              else
                load_gates(kept[0], q, kNo, most);
              load_values(q, kNo);
              leave_out(kept[0], low[0], q);
            }
            start_half(a.h0, s, q, from);
#pragma unroll
            for (int i = 0; i < kHalf; ++i) {
              hp[i] = h = pick(s, i, from[i], h);
              h = step<kForm, kSel>(h, m[i], v[i].f(), low[0] >> (2 * i));
            }
            start_half(a.dfinal, e, q, from);
#pragma unroll
            for (int i = kHalf - 1; i >= 0; --i) {
              const F2 D = add2(d[i].f(), pick(e, i, from[i], in));
              in = decayed<kSel>(D, m[i], low[0] >> (2 * i));
              grads(select, i, D, in, hp[i], df, dval);
              from[i] = in;
              if constexpr (decltype(box)::value) {
                to_box(0, q * kHalf + i, df);
                to_box(kD, q * kHalf + i, dval);
              } else if (row + q * kHalf + i < a.T) {
                const bool in_one = is >> i & 1u;
                store_out(dg + (row + q * kHalf + i) * a.H + c0, in_one ? df : zero2());
                store_out(dv + (row + q * kHalf + i) * a.H + c0, in_one ? dval : zero2());
              }
            }
          };
          if (kFast ? !boxed : some)
            walk(kYes, kNo);   // (with no bit in low the same)
          else
            walk(std::bool_constant<kSelect>{}, std::bool_constant<kFast>{});
          if (s != 0 && a.dinit) {
#pragma unroll
            for (int i = 0; i < kHalf; ++i)
              if (s >> i & 1u) store2<kFast>(a.dinit + int64_t(rows.seq[r0 + q * kHalf + i]) * a.H + c, from[i], left);
          }
        }
      }
      if (boxed) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          const uint32_t box = smem_u32(stage);
          tma_store_2d(&maps.out0, box, c0, static_cast<int>(row));
          if constexpr (kGrads) tma_store_2d(&maps.out1, box + kD * kTensorBytes, c0, static_cast<int>(row));
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
  }
  __syncthreads();
  cluster_sync_all();   // no block leaves while a peer may still write to it
}

// One row of each sequence: kVec channels to a thread, `chunks` blocks to a row.
template <class T, int kForm, int kVec>
__global__ void __launch_bounds__(256) scan_step_kernel(const T* gate, const T* value, const float* state, int64_t B, int H,
                                                        int64_t gate_ld, int64_t value_ld, int chunks, T* y, float* state_out) {
  for (int64_t i = blockIdx.x; i < B * chunks; i += gridDim.x) {
    const int64_t b = i / chunks;
    const int c = (static_cast<int>(i - b * chunks) * 256 + static_cast<int>(threadIdx.x)) * kVec;
    if (c >= H) continue;
    float f[kVec], v[kVec], h[kVec];
    load_vec<kVec>(gate + b * gate_ld + c, f);
    load_vec<kVec>(value + b * value_ld + c, v);
    load_vec<kVec>(state + b * H + c, h);
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      uint32_t low;
      const F2 k = coefficient<kForm>(f2(f[j]), kLowGate<float, kForm>, low);
      h[j] = step<kForm, true>(f2(h[j]), k, f2(v[j]), low).x();
    }
    store_vec<kVec>(state_out + b * H + c, h);
    store_vec<kVec>(y + b * H + c, h);
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
  if (d->T > 2147483647 - 2 * kStateRows || d->H > 65536 || d->B > 2147483647 - 64)
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
int64_t strips_of(const molt_scan_desc* d, bool fast) {
  const int wide = d->dtype == MOLT_FP32 ? (fast ? kStrip<float, true> : kStrip<float, false>)
                                         : (fast ? kStrip<__half, true> : kStrip<__half, false>);
  return (d->H + wide - 1) / wide;
}
size_t seg_bytes(const molt_scan_desc* d) {
  return static_cast<size_t>(kMaxSegments) * strips_of(d, false) * 32 * sizeof(float4) + 256;
}

constexpr int kDevices = 16;

// One instance of the kernel.
struct ScanKernel {
  void (*fn)(const ScanMaps, const ScanArgs);
  int smem;
  // by device and a cluster's blocks: how many clusters run at once (0: not yet asked)
  std::atomic<int> clusters[kDevices][kMaxCluster + 1];
};
template <class T, int kForm, bool kBwd, bool kMapOnly, bool kFast>
ScanKernel* kernel_of() {
  constexpr int kTensors = kBwd && !kMapOnly ? 3 : 2;
  static ScanKernel k{&scan_kernel<T, kForm, kBwd, kMapOnly, kFast>,
                      kStagesOf<kBwd, kMapOnly> * kTile<T, kBwd> * kTensors * kPitch<T> + (kFast ? 0 : 128), {}};
  return &k;
}
template <class T, int kForm>
ScanKernel* kernel_of(bool bwd, bool map_only, bool fast) {
  if (fast)
    return bwd ? (map_only ? kernel_of<T, kForm, true, true, true>() : kernel_of<T, kForm, true, false, true>())
               : (map_only ? kernel_of<T, kForm, false, true, true>() : kernel_of<T, kForm, false, false, true>());
  return bwd ? (map_only ? kernel_of<T, kForm, true, true, false>() : kernel_of<T, kForm, true, false, false>())
             : (map_only ? kernel_of<T, kForm, false, true, false>() : kernel_of<T, kForm, false, false, false>());
}
template <class T>
ScanKernel* kernel_of(int form, bool bwd, bool map_only, bool fast) {
  return form == kFormSigmoid ? kernel_of<T, kFormSigmoid>(bwd, map_only, fast) : kernel_of<T, kFormLog>(bwd, map_only, fast);
}
ScanKernel* kernel_of(int dtype, int form, bool bwd, bool map_only, bool fast) {
  return dtype == MOLT_FP32   ? kernel_of<float>(form, bwd, map_only, fast)
         : dtype == MOLT_FP16 ? kernel_of<__half>(form, bwd, map_only, fast)
                              : kernel_of<__nv_bfloat16>(form, bwd, map_only, fast);
}

struct ScanLaunch {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr{};
  ScanLaunch(const ScanKernel* k, int strips, int cluster, int segments, cudaStream_t s) {
    cfg.gridDim = dim3(strips * cluster, segments);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = static_cast<size_t>(k->smem);
    cfg.stream = s;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = cluster;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
  }
};

// Clusters of so many blocks that run at once.  Blocks that the SMs hold are not all of use: a
// cluster's are in one GPC (clusters of 7 in three rounds of blocks to an SM: 448 of 456 blocks
// asked for, and two waves).
cudaError_t clusters_at_once(ScanKernel* k, int cluster, int& n) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  std::atomic<int>* const known = dev < kDevices ? &k->clusters[dev][cluster] : nullptr;
  n = known ? known->load(std::memory_order_relaxed) : 0;
  if (n > 0) return cudaSuccess;
  e = cudaFuncSetAttribute(k->fn, cudaFuncAttributeMaxDynamicSharedMemorySize, k->smem);
  if (e != cudaSuccess) return e;
  ScanLaunch l(k, 1, cluster, 1, nullptr);
  l.cfg.attrs = &l.attr;
  e = cudaOccupancyMaxActiveClusters(&n, k->fn, &l.cfg);
  if (e != cudaSuccess) return e;
  n = std::max(n, 1);
  if (known) known->store(n, std::memory_order_relaxed);
  return cudaSuccess;
}

struct ScanPlan {
  int cluster, segments;
};
// The largest clusters with which all strips run at once; the rows in segments where there is
// room for several times the strips, and each has eight steps or more.
cudaError_t plan_of(ScanKernel* k, int64_t strips, int tiles, ScanPlan& p) {
  p.cluster = p.segments = 1;
  int n = 0;
  for (int s = kMaxCluster; s >= 1; --s) {
    if (s > tiles && s > 1) continue;
    if (const cudaError_t e = clusters_at_once(k, s, n); e != cudaSuccess) return e;
    p.cluster = s;
    if (n >= strips) break;
  }
  const int64_t steps = (tiles + p.cluster - 1) / p.cluster;
  p.segments = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({kMaxSegments, n / strips, steps / 8})));
  return cudaSuccess;
}

molt_status launch(const molt_scan_desc* d, ScanArgs& a, bool bwd, void* workspace, size_t workspace_bytes, cudaStream_t s) {
  molt_status st;
  a.err = device_status_word(&st);
  if (!a.err) return st;
  const int tile = d->dtype == MOLT_FP32 ? (bwd ? kTile<float, true> : kTile<float, false>)
                                         : (bwd ? kTile<__half, true> : kTile<__half, false>);
  a.tiles = static_cast<int>((a.T + tile - 1) / tile);
  const bool fast = a.tiles > 0 && fast_of(a, d->dtype);
  const int strips = static_cast<int>(strips_of(d, fast));
  ScanPlan plan;
  if (const cudaError_t e = plan_of(kernel_of(d->dtype, d->form, bwd, false, fast), strips, a.tiles, plan); e != cudaSuccess)
    return cuda_fail(e, "gated scan");
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
    const auto encode = [&](CUtensorMap* t, const void* p, int64_t ld, int rows) {
      return encode_tmap_plain(t, e == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, e, p, a.T, a.H, ld,
                               kStrip<float, true>, rows);
    };
    if (const molt_status q = encode(&m.gate, a.gate, a.gate_ld, tile); q != MOLT_OK) return q;
    if (const molt_status q = encode(&m.value, a.value, a.value_ld, tile); q != MOLT_OK) return q;
    if (bwd)
      if (const molt_status q = encode(&m.dy, a.dy, a.dy_ld, tile); q != MOLT_OK) return q;
    if (const molt_status q = encode(&m.out0, bwd ? a.dgate : a.y, a.H, tile / kWarps); q != MOLT_OK) return q;
    if (bwd)
      if (const molt_status q = encode(&m.out1, a.dvalue, a.H, tile / kWarps); q != MOLT_OK) return q;
  }
  for (int pass = segments > 1 ? 0 : 1; pass < 2; ++pass) {
    ScanKernel* const k = kernel_of(d->dtype, d->form, bwd, pass == 0, fast);
    int n;   // (asked once: sets the kernel's shared memory)
    cudaError_t e = clusters_at_once(k, plan.cluster, n);
    if (e == cudaSuccess) {
      ScanLaunch l(k, strips, plan.cluster, segments, s);
      l.cfg.attrs = &l.attr;
      e = cudaLaunchKernelEx(&l.cfg, k->fn, m, a);
    }
    if (e != cudaSuccess) return cuda_fail(e, "gated scan");
    note_launches(1);
  }
  return MOLT_OK;
}

template <class T, int kForm>
void launch_step(const molt_scan_desc* d, const void* gate, const void* value, const float* state, void* y, float* out,
                 cudaStream_t s) {
  const int H = static_cast<int>(d->H);
  const int64_t g_ld = d->gate_stride ? d->gate_stride : H, v_ld = d->value_stride ? d->value_stride : H;
  const auto at = [](const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; };
  const bool vec = H % 4 == 0 && g_ld % 4 == 0 && v_ld % 4 == 0 && at(gate, 4 * sizeof(T)) && at(value, 4 * sizeof(T)) &&
                   at(y, 4 * sizeof(T)) && at(state, 16) && at(out, 16);
  const int chunks = (H + 256 * (vec ? 4 : 1) - 1) / (256 * (vec ? 4 : 1));
  const int grid = static_cast<int>(std::min<int64_t>(d->B * chunks, 16 * int64_t(device_sm_count())));
  const auto k = vec ? scan_step_kernel<T, kForm, 4> : scan_step_kernel<T, kForm, 1>;
  k<<<grid, 256, 0, s>>>(static_cast<const T*>(gate), static_cast<const T*>(value), state, d->B, H, g_ld, v_ld, chunks,
                         static_cast<T*>(y), out);
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
  if (const int64_t T = desc->T, H = desc->H, B = desc->B, e = dtype_bytes(desc->dtype);
      !spans_apart({{y, T, H, e}, {final_state, B, H, 4}, {states, (T + kStateRows - 1) / kStateRows, H, 4}},
                   {{gate, T, H, e, desc->gate_stride}, {value, T, H, e, desc->value_stride}, {initial_state, B, H, 4},
                    {cu_seqlens, B + 1, 1, 4}}))
    return fail(MOLT_ERR_INVALID_ARG, "outputs may not share memory with one another or with inputs");
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
  if (const int64_t T = desc->T, H = desc->H, B = desc->B, e = dtype_bytes(desc->dtype);
      !spans_apart({{dgate, T, H, e}, {dvalue, T, H, e}, {dinitial_state, B, H, 4}},
                   {{dy, T, H, e, desc->dy_stride}, {gate, T, H, e, desc->gate_stride}, {value, T, H, e, desc->value_stride},
                    {states, (T + kStateRows - 1) / kStateRows, H, 4}, {initial_state, B, H, 4}, {dfinal_state, B, H, 4},
                    {cu_seqlens, B + 1, 1, 4}}))
    return fail(MOLT_ERR_INVALID_ARG, "outputs may not share memory with one another or with inputs");
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
  const int64_t H = desc->H, B = desc->B;
  const int e = dtype_bytes(desc->dtype);
  // the state may be updated in place: each element by the thread that has read it
  if (!spans_apart({{y, B, H, e}, {state_out, B, H, 4}}, {{gate, B, H, e, desc->gate_stride}, {value, B, H, e, desc->value_stride}}) ||
      !spans_apart({{y, B, H, e}, {state_out == state ? nullptr : state_out, B, H, 4}}, {{state, B, H, 4}}))
    return fail(MOLT_ERR_INVALID_ARG, "outputs may not share memory with one another or with inputs (but state_out may be state)");
  const bool sig = desc->form == MOLT_SCAN_SIGMOID;
  const auto k = desc->dtype == MOLT_FP32   ? (sig ? launch_step<float, kFormSigmoid> : launch_step<float, kFormLog>)
                 : desc->dtype == MOLT_FP16 ? (sig ? launch_step<__half, kFormSigmoid> : launch_step<__half, kFormLog>)
                                            : (sig ? launch_step<__nv_bfloat16, kFormSigmoid> : launch_step<__nv_bfloat16, kFormLog>);
  k(desc, gate, value, state, y, state_out, stream);
  if (const cudaError_t status = cudaGetLastError(); status != cudaSuccess) return cuda_fail(status, "gated scan step");
  note_launches(1);
  return MOLT_OK;
}

}  // extern "C"
