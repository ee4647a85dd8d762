// Token embedding with scaling, and its gradient by sorted tokens.
//
//   out_t = s E[x_t]          dE_v = s sum_{t: x_t = v} dout_t
//
// Forward: a gather, bound by HBM (each row of E that occurs and out once): T = 65536,
// H = 4096, bf16, V = 151936: 121 us, 6.1 TB/s.
//
// Gradient: the positions are sorted by token (stably, so equal tokens stay in token
// order), cut into units of equally many sorted positions, and every unit adds up its
// runs of equal tokens in fp32.  A run inside a unit is written at once; a run that
// crosses units leaves one fp32 part in each, which a last kernel adds in order.  So a
// token that fills a tenth of the batch is spread over as many units as it needs, no
// atomics are used and the results are the same bits in every run.  Rows of tokens that
// do not occur are zeroed by blocks of the same launch, mixed with the units, so that
// dE is written exactly once.  At those sizes (20526 different tokens, 1.78 GB): 336 us, of
// which 286 this launch at 6.2 TB/s, 34 the sort and 10 the crossing runs.  (Zeroing rows
// beside the sort's launches instead gained nothing: what it took there it saved here.)
//
// Sorting: chunks of kSortChunk positions by counting, then every element finds its
// place among up to kMergeLists sorted chunks by binary search.
#include <algorithm>
#include <cstdint>
#include <cuda_runtime.h>

#include "../../include/molt.h"
#include "molt_internal.cuh"
#include "ptx.cuh"
#include "vec.cuh"

namespace molt {
namespace {

// ------------------------------------------------------------------- forward
struct EmbedArgs {
  const void* E;
  const int32_t* tok;
  int64_t T;
  int V, H;
  float scale;
  void* out;
  unsigned* err;
};

// blockDim.x threads to a row, blockDim.y groups of kRows rows to a block
template <class X, class O, int kV, int kRows>
__global__ void __launch_bounds__(256) embed_kernel(const EmbedArgs a) {
  const int64_t t0 = (static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y) * kRows;
  int tok[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    tok[k] = t0 + k < a.T ? a.tok[t0 + k] : 0;
    if (tok[k] < 0 || tok[k] >= a.V) {
      if (threadIdx.x == 0) atomicOr(a.err, kDevErrTokenRange);
      tok[k] = -1;
    }
  }
  const X* E = static_cast<const X*>(a.E);
  O* out = static_cast<O*>(a.out);
  for (int c = threadIdx.x * kV; c < a.H; c += blockDim.x * kV) {
    float v[kRows][kV];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
#pragma unroll
      for (int j = 0; j < kV; ++j) v[k][j] = 0.f;
      if (tok[k] >= 0) load_vec<kV>(E + static_cast<int64_t>(tok[k]) * a.H + c, v[k]);
    }
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
#pragma unroll
      for (int j = 0; j < kV; ++j) v[k][j] = tok[k] >= 0 ? v[k][j] * a.scale : 0.f;
      if (t0 + k < a.T) store_vec<kV>(out + (t0 + k) * a.H + c, v[k]);
    }
  }
}

// n elements from p set to zero by a warp, on any alignment
template <class O>
__device__ __forceinline__ void zero_span(O* p, int n) {
  const int lane = threadIdx.x & 31;
  const int head = min(n, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / static_cast<int>(sizeof(O)));
  constexpr int kPer = 16 / sizeof(O);
  const int body = (n - head) / kPer;
  const O zero = static_cast<O>(0.f);
  if (lane < head) p[lane] = zero;
  uint4* v = reinterpret_cast<uint4*>(p + head);
#pragma unroll 4
  for (int i = lane; i < body; i += 32) v[i] = make_uint4(0, 0, 0, 0);
  const int done = head + body * kPer;
  if (lane < n - done) p[done + lane] = zero;
}

// ------------------------------------------------------------------- sorting
// Chunks of positions are sorted by counting: an element's place is the number of
// elements of its chunk that are smaller, every pair compared: few steps that wait for
// one another.  4 us for 5003 positions and 8 for 65536, where radix passes of a block
// took 24 and 35 (chunks of 4096, which save a round of merging, 42).
constexpr int kSortElems = 128, kSortSplit = 4, kSortThreads = kSortElems * kSortSplit;
constexpr int kSortBits = 9, kSortChunk = 1 << kSortBits;

// Tokens that give no gradient (outside [0, V), or the padding token) get the key V and
// so come last.  Word: token << kSortBits | place in the chunk (64 bits where V needs
// them).  A block places kSortElems elements of a chunk, kSortSplit threads to an element,
// each comparing it with a part of the chunk.
template <class Word>
__global__ void __launch_bounds__(kSortThreads) sort_chunks_kernel(const int32_t* __restrict__ tok, int T, int V, int padding,
                                                                   uint32_t* __restrict__ keys_out,
                                                                   uint32_t* __restrict__ pos_out, int* __restrict__ n_cross,
                                                                   unsigned* err) {
  constexpr int kPer = 16 / sizeof(Word);
  __shared__ __align__(16) Word sh[kSortChunk];
  __shared__ int part_rank[kSortSplit][kSortElems];
  if (blockIdx.x == 0 && threadIdx.x == 0) *n_cross = 0;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kSortElems, base = first >> kSortBits << kSortBits;
  const int n = static_cast<int>(min(static_cast<int64_t>(kSortChunk), T - base));
  bool bad = false;
  static_assert(kSortThreads == kSortChunk);
  {
    const int i = threadIdx.x;
    Word w = ~Word(0);   // past the end: larger than every element
    if (i < n) {
      const int x = tok[base + i];
      const bool in = x >= 0 && x < V;
      bad |= !in;
      w = static_cast<Word>(in && x != padding ? x : V) << kSortBits | static_cast<Word>(i);
    }
    sh[i] = w;
  }
  if (bad && first == base) atomicOr(err, kDevErrTokenRange);
  __syncthreads();
  const int elem = threadIdx.x % kSortElems, split = threadIdx.x / kSortElems;
  const int i = static_cast<int>(first - base) + elem;
  const Word mine = sh[i];
  int count[4] = {0, 0, 0, 0};   // chains of their own: one alone waits for each addition
  const int share = ((n + kSortSplit - 1) / kSortSplit + 7) / 8 * 8;
  const int j1 = min((n + 7) / 8 * 8, (split + 1) * share);
#pragma unroll 4
  for (int j = split * share; j < j1; j += 8) {
    Word w[8];
#pragma unroll
    for (int q = 0; q < 8 / kPer; ++q)
      *reinterpret_cast<uint4*>(w + q * kPer) = *reinterpret_cast<const uint4*>(sh + j + q * kPer);
#pragma unroll
    for (int q = 0; q < 8; ++q) count[q % 4] += w[q] < mine ? 1 : 0;
  }
  part_rank[split][elem] = (count[0] + count[1]) + (count[2] + count[3]);
  __syncthreads();
  if (split != 0 || i >= n) return;
  int rank = 0;
#pragma unroll
  for (int q = 0; q < kSortSplit; ++q) rank += part_rank[q][elem];
  keys_out[base + rank] = static_cast<uint32_t>(mine >> kSortBits);
  pos_out[base + rank] = static_cast<uint32_t>(base + i);
}

// One step of a warp's search among sorted keys for the first that is not before `key`
// (kept in [lo, hi)): 32 probes at a time, so that 2^15 keys take three loads one after
// the other.  upper: keys equal to it are before it too.
struct WarpSearch {
  int lo, hi, p;
  uint32_t v;
  __device__ __forceinline__ void load(const uint32_t* __restrict__ keys) {
    const int lane = threadIdx.x & 31, span = hi - lo;
    p = span <= 32 ? lo + lane : lo + static_cast<int>(static_cast<int64_t>(lane + 1) * span / 33);
    if (p < hi) v = keys[p];
  }
  __device__ __forceinline__ void narrow(uint32_t key, bool upper) {
    const int c = __popc(__ballot_sync(0xffffffffu, p < hi && (v < key || (upper && v == key))));   // the first c are before
    const int p_last = __shfl_sync(0xffffffffu, p, max(c - 1, 0)), p_next = __shfl_sync(0xffffffffu, p, min(c, 31));
    if (c < 32) hi = min(hi, p_next);
    if (c > 0) lo = p_last + 1;
  }
};
__device__ __forceinline__ int warp_lower_bound(const uint32_t* __restrict__ keys, int n, uint32_t key) {
  WarpSearch s{0, n, 0, 0u};
  while (s.lo < s.hi) {
    s.load(keys);
    s.narrow(key, false);
  }
  return s.lo;
}

// Groups of up to kMergeLists sorted lists of `len` elements become one: an element's
// place is its own index plus, for every other list, the number of elements before it
// there (equal keys of earlier lists come first, as their positions do).  A block places
// kMergeElems neighbours of one list.  They fall into one window of each other list: a
// warp to a list finds the window's ends (both at once), the windows pass through shared
// memory kWindow elements of every list at a time, and kMergeSplit threads to an element
// search them there.  What counts is how few steps follow one another, and that the
// searches spread over all SMs: 4.5 us at T = 5003 and 13 a round at 65536, where a search
// in global memory for every element and list took 43 and blocks of 512 elements 11 and 19.
constexpr int kMergeLists = 16, kMergeElems = 64, kMergeThreads = 32 * kMergeLists, kWindow = 256;
constexpr int kMergeSplit = kMergeThreads / kMergeElems;   // threads to an element, each searches some of the lists
static_assert(kSortChunk % kMergeElems == 0 && kMergeLists % kMergeSplit == 0);

__global__ void __launch_bounds__(kMergeThreads) merge_lists_kernel(const uint32_t* __restrict__ keys,
                                                                    const uint32_t* __restrict__ pos, int T, int64_t len,
                                                                    int lists, uint32_t* __restrict__ keys_out,
                                                                    uint32_t* __restrict__ pos_out) {
  __shared__ uint32_t win[kMergeLists][kWindow];
  __shared__ int w_lo[kMergeLists], w_n[kMergeLists];
  __shared__ int before[kMergeSplit][kMergeElems];
  const int lane = threadIdx.x & 31, l = threadIdx.x >> 5;   // the warp's list
  const int64_t e0 = static_cast<int64_t>(blockIdx.x) * kMergeElems;   // lists begin at multiples of it
  const int elem = threadIdx.x % kMergeElems, split = threadIdx.x / kMergeElems;
  const int64_t e = e0 + elem;
  const int64_t list = e0 / len, group0 = list / kMergeLists * kMergeLists * len;
  const int mine = static_cast<int>(list % kMergeLists);
  const uint32_t k_first = keys[e0], k_last = keys[min(e0 + kMergeElems, static_cast<int64_t>(T)) - 1];
  const uint32_t k = e < T ? keys[e] : k_last;
  const uint32_t p = split == 0 && e < T ? pos[e] : 0u;
  const uint32_t* my_keys = keys + group0 + l * len;
  WarpSearch first{0, 0, 0, 0u}, last{0, 0, 0, 0u};
  {
    const int64_t l0 = group0 + l * len;
    first.hi = last.hi = l >= lists || l == mine || l0 >= T ? 0 : static_cast<int>(min(len, T - l0));
    while (first.lo < first.hi || last.lo < last.hi) {
      first.load(my_keys);
      last.load(my_keys);
      first.narrow(k_first, l < mine);   // equal keys of an earlier list come before
      last.narrow(k_last, l < mine);
    }
    if (lane == 0) {
      w_lo[l] = first.lo;
      w_n[l] = last.lo - first.lo;
    }
  }
  __syncthreads();
  int widest = 0;
#pragma unroll
  for (int i = 0; i < kMergeLists; ++i) widest = max(widest, w_n[i]);
  int n_before = 0;
  for (int w0 = 0; w0 < widest; w0 += kWindow) {
    const int n = min(kWindow, w_n[l] - w0);
#pragma unroll
    for (int i = 0; i < kWindow / 32; ++i)
      if (i * 32 + lane < n) win[l][i * 32 + lane] = my_keys[first.lo + w0 + i * 32 + lane];
    __syncthreads();
    constexpr int kEach = kMergeLists / kMergeSplit;
    int c[kEach] = {};   // of a list's m elements, those before this one
#pragma unroll 1
    for (int step = kWindow; step > 0; step >>= 1) {
#pragma unroll
      for (int q = 0; q < kEach; ++q) {
        const int i = split * kEach + q;
        const int m = min(kWindow, w_n[i] - w0);
        const uint32_t v = win[i][min(c[q] + step, kWindow) - 1];
        if ((v < k || (i < mine && v == k)) && c[q] + step <= m) c[q] += step;
      }
    }
#pragma unroll
    for (int q = 0; q < kEach; ++q) n_before += c[q];
    __syncthreads();
  }
  before[split][elem] = n_before;
  __syncthreads();
  if (split != 0 || e >= T) return;
  int64_t to = e - mine * len;
#pragma unroll
  for (int i = 0; i < kMergeLists; ++i) to += w_lo[i];
#pragma unroll
  for (int i = 0; i < kMergeSplit; ++i) to += before[i][elem];
  keys_out[to] = k;
  pos_out[to] = p;
}

// ------------------------------------------------------------------ gradient
struct EmbedGradArgs {
  const void* dout;
  const uint32_t *keys, *pos;   // sorted
  int T, V, H;
  int unit;                     // sorted positions to a unit
  int n_units, n_slabs, slab;   // slab: columns that a group of threads holds
  int sum_blocks, zero_blocks;
  bool add;                     // dE is added to
  int zero_rows;                // rows that one warp zeroes, at most 32
  float scale;
  void* dE;
  float* part;                  // [n_units, 2, H]: sums of a run from the unit before / into the unit after
  int* n_cross;                 // runs that cross units:
  int4* cross;                  // first unit, token, units
};

template <class O, int kV>
__device__ __forceinline__ void put_row(O* p, const float (&v)[kV], float scale, bool add) {
  float o[kV];
#pragma unroll
  for (int j = 0; j < kV; ++j) o[j] = scale * v[j];
  if constexpr (sizeof(O) == 4) {
    if (add) {
      float old[kV];
      load_vec<kV>(p, old);
#pragma unroll
      for (int j = 0; j < kV; ++j) o[j] += old[j];
    }
  }
  store_vec<kV>(p, o);
}

// The rows from v0 on of tokens that do not occur, zeroed by one warp.
template <class O>
__device__ __forceinline__ void zero_rows(const EmbedGradArgs& a, int64_t v0) {
  if (v0 >= a.V) return;
  const int lane = threadIdx.x & 31;
  const int rows = static_cast<int>(min(static_cast<int64_t>(a.zero_rows), a.V - v0));
  const uint32_t first = static_cast<uint32_t>(v0), end = first + rows;
  unsigned occur = 0;   // bit i: row v0 + i
  int i = warp_lower_bound(a.keys, a.T, first);
  while (i < a.T) {
    const uint32_t k = i + lane < a.T ? a.keys[i + lane] : 0xffffffffu;
    occur |= __reduce_or_sync(0xffffffffu, k < end ? 1u << (k - first) : 0u);
    const uint32_t last = __shfl_sync(0xffffffffu, k, 31);
    if (last >= end) break;
    // on to the next token: a frequent one fills many more keys
    const int next = i + 32;
    i = next < a.T && a.keys[next] == last ? max(next, warp_lower_bound(a.keys, a.T, last + 1)) : next;
  }
  // neighbours together: short rows of any length then are few unaligned ends
  for (unsigned m = ~occur & (rows == 32 ? 0xffffffffu : (1u << rows) - 1u); m != 0;) {
    const int at = __ffs(m) - 1, n = __ffs(~(m >> at)) - 1;   // n < 0: all 32
    const int len = n < 0 ? 32 : n;
    zero_span(static_cast<O*>(a.dE) + (v0 + at) * a.H, len * a.H);
    m = at + len >= 32 ? 0u : m & (0xffffffffu << (at + len));
  }
}

// kV elements as they are in memory, so that a batch of rows in flight takes few registers
template <class X, int kV>
struct Raw {
  static constexpr int kWords = kV * sizeof(X) / 4;
  alignas(16) uint32_t w[kWords];
  __device__ __forceinline__ void load(const X* p) {
    if constexpr (kWords == 1) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else if constexpr (kWords == 2) {
      *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(p);
    } else {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) reinterpret_cast<uint4*>(w)[i] = reinterpret_cast<const uint4*>(p)[i];
    }
  }
  __device__ __forceinline__ void get(float (&v)[kV]) const { load_vec<kV>(reinterpret_cast<const X*>(w), v); }
};
template <class X>
struct Raw<X, 1> {
  X x;
  __device__ __forceinline__ void load(const X* p) { x = *p; }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = to_float(x); }
};

// blockDim.x threads hold a slab of columns, 8 each; blockDim.y units to a block.
// sum_blocks of the blocks add up units, the others zero the rows of tokens that do not
// occur; the two kinds are mixed evenly over the grid.
template <class X, class O, int kV>
__global__ void __launch_bounds__(256) embed_grad_kernel(const EmbedGradArgs a) {
  constexpr int N = 8 / kV;
  constexpr int kBatch = sizeof(X) == 4 ? 4 : 8;
  const int64_t all = static_cast<int64_t>(a.sum_blocks) + a.zero_blocks;
  const int sum_before = static_cast<int>(static_cast<int64_t>(blockIdx.x) * a.sum_blocks / all);
  const bool sums = static_cast<int64_t>(blockIdx.x + 1) * a.sum_blocks / all > sum_before;
  O* dE = static_cast<O*>(a.dE);
  if (!sums) {
    const int warps = blockDim.x * blockDim.y / 32, warp = (threadIdx.y * blockDim.x + threadIdx.x) / 32;
    zero_rows<O>(a, (static_cast<int64_t>(blockIdx.x - sum_before) * warps + warp) * a.zero_rows);
    return;
  }
  const int u = (sum_before / a.n_slabs) * blockDim.y + threadIdx.y;
  if (u >= a.n_units) return;
  const int slab = sum_before % a.n_slabs, col0 = slab * a.slab;
  const int i0 = u * a.unit, i1 = min(a.T, i0 + a.unit);
  const bool add = a.add;
  auto column = [&](int n) { return col0 + (n * blockDim.x + threadIdx.x) * kV; };
  float acc[N][kV];
  auto flush = [&](uint32_t key, bool from_before, bool into_after) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int c = column(n);
      if (c < a.H) {
        if (from_before || into_after)
          store_vec<kV>(a.part + (static_cast<int64_t>(u) * 2 + (from_before ? 0 : 1)) * a.H + c, acc[n]);
        else
          put_row<O, kV>(dE + static_cast<int64_t>(key) * a.H + c, acc[n], a.scale, add);
      }
#pragma unroll
      for (int j = 0; j < kV; ++j) acc[n][j] = 0.f;
    }
  };
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int j = 0; j < kV; ++j) acc[n][j] = 0.f;
  uint32_t run = a.keys[i0];
  if (run >= static_cast<uint32_t>(a.V)) return;   // no gradient from here on
  bool from_before = i0 > 0 && a.keys[i0 - 1] == run;
  for (int i = i0; i < i1; i += kBatch) {
    uint32_t key[kBatch];
    Raw<X, kV> raw[kBatch][N];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      key[b] = i + b < i1 ? a.keys[i + b] : 0xffffffffu;
      const X* row = static_cast<const X*>(a.dout);
      if (key[b] < static_cast<uint32_t>(a.V)) row += static_cast<int64_t>(a.pos[i + b]) * a.H;
#pragma unroll
      for (int n = 0; n < N; ++n)
        if (key[b] < static_cast<uint32_t>(a.V) && column(n) < a.H) raw[b][n].load(row + column(n));
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (i + b >= i1) break;
      if (key[b] != run) {
        flush(run, from_before, false);
        run = key[b];
        from_before = false;
        if (run >= static_cast<uint32_t>(a.V)) return;
      }
#pragma unroll
      for (int n = 0; n < N; ++n) {
        if (column(n) >= a.H) continue;
        float v[kV];
        raw[b][n].get(v);
#pragma unroll
        for (int j = 0; j < kV; ++j) acc[n][j] += v[j];
      }
    }
  }
  const bool into_after = i1 < a.T && a.keys[i1] == run;
  flush(run, from_before, into_after);
  if (into_after && !from_before && slab == 0 && threadIdx.x < 32) {
    // units of the run: parts are (u, 1), (u + 1, 0), ... while a unit begins with the token
    int n_parts = 1;
    for (;;) {
      const int v = u + n_parts + threadIdx.x;
      const unsigned same = __ballot_sync(0xffffffffu, v < a.n_units && a.keys[static_cast<int64_t>(v) * a.unit] == run);
      n_parts += same == 0xffffffffu ? 32 : __ffs(~same) - 1;
      if (same != 0xffffffffu) break;
    }
    if (threadIdx.x == 0) a.cross[atomicAdd(a.n_cross, 1)] = make_int4(u, static_cast<int>(run), n_parts, 0);
  }
}

// The runs that cross units, 128 columns of a run at a time: a warp adds up the parts in
// order, four columns to a lane.  A run of many parts is split over the block's warps,
// warp w taking every kJoinWarps-th part, and their sums are added in order; a token
// that fills a twentieth of the batch would else be 20 us of one warp's loads.  (Which
// block takes which run does not matter to the sums.)
constexpr int kJoinWarps = 8, kJoinCols = 128, kJoinMany = 16;

template <class O>
__global__ void __launch_bounds__(32 * kJoinWarps) embed_join_kernel(const EmbedGradArgs a) {
  __shared__ float4 sh[kJoinWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool add = a.add, vec = a.H % 4 == 0;
  const int n_cross = *a.n_cross;
  const int c = blockIdx.x * kJoinCols + lane * 4;
  // columns c to c + 3 of every step-th part of a run from the k0-th on
  auto sum = [&](const int4& run, int k0, int step) {
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* p = a.part + static_cast<int64_t>(run.x) * 2 * a.H + c;
    auto load = [&](int k) {
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (k >= run.z) return v;
      const float* q = p + (static_cast<int64_t>(k) * 2 + (k == 0 ? 1 : 0)) * a.H;
      if (vec) {
        if (c < a.H) v = *reinterpret_cast<const float4*>(q);
      } else {
        if (c < a.H) v.x = q[0];
        if (c + 1 < a.H) v.y = q[1];
        if (c + 2 < a.H) v.z = q[2];
        if (c + 3 < a.H) v.w = q[3];
      }
      return v;
    };
#pragma unroll 1
    for (int k = k0; k < run.z; k += 4 * step) {
      const float4 v[4] = {load(k), load(k + step), load(k + 2 * step), load(k + 3 * step)};
#pragma unroll
      for (int i = 0; i < 4; ++i) s.x += v[i].x, s.y += v[i].y, s.z += v[i].z, s.w += v[i].w;
    }
    return s;
  };
  auto put = [&](const int4& run, const float4& s) {
    O* row = static_cast<O*>(a.dE) + static_cast<int64_t>(run.y) * a.H + c;
    const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float one[1] = {v[j]};
      if (c + j < a.H) put_row<O, 1>(row + j, one, a.scale, add);
    }
  };
  for (int r0 = blockIdx.y * kJoinWarps; r0 < n_cross; r0 += gridDim.y * kJoinWarps) {
    const int4 mine = r0 + warp < n_cross ? a.cross[r0 + warp] : make_int4(0, 0, 0, 0);
    if (mine.z > 0 && mine.z <= kJoinMany) put(mine, sum(mine, 0, 1));
    if (!__syncthreads_or(mine.z > kJoinMany)) continue;
    for (int i = r0; i < min(n_cross, r0 + kJoinWarps); ++i) {
      const int4 run = a.cross[i];
      if (run.z <= kJoinMany) continue;
      sh[warp][lane] = sum(run, warp, kJoinWarps);
      __syncthreads();
      if (warp == 0) {
        float4 s = sh[0][lane];
#pragma unroll
        for (int y = 1; y < kJoinWarps; ++y) {
          const float4 v = sh[y][lane];
          s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
        }
        put(run, s);
      }
      __syncthreads();
    }
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

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

constexpr int64_t kMaxCount = (int64_t(1) << 31) - (int64_t(1) << 17);   // 32-bit indices, also past a last block's end

molt_status check(int64_t T, int64_t H, int64_t V, int narrow, int wide, float scale) {
  if (T < 0 || H < 1 || V < 1) return fail(MOLT_ERR_INVALID_ARG, "sizes must satisfy T >= 0, H >= 1, V >= 1");
  if (T > kMaxCount || V > kMaxCount || H > 65536)
    return fail(MOLT_ERR_UNSUPPORTED_SHAPE, "T and V must be at most 2^31 - 2^17 and H at most 65536");
  if (narrow < MOLT_BF16 || narrow > MOLT_FP32 || (wide != narrow && wide != MOLT_FP32))
    return fail(MOLT_ERR_INVALID_ARG, "types are bf16, fp16 or fp32, the output's the input's or fp32");
  if (!(scale >= -1e30f && scale <= 1e30f)) return fail(MOLT_ERR_INVALID_ARG, "scale must be finite");
  return MOLT_OK;
}

// Elements to a load or store of rows of H side by side: as many as divide H, up to 8,
// and the two bases are aligned to.  (us, where only multiples of eight were read in
// vectors and now: T = 30000, H = 1566 forward 49 and 37; gradient, absent rows then also
// zeroed one by one, T = 26064, H = 4554, V = 49523 246 and 193.)
int vec_of(int64_t H, const void* p, int p_dtype, const void* q, int q_dtype) {
  for (int v = 8; v > 1; v /= 2)
    if (H % v == 0 && aligned(p, std::min(16, v * dtype_bytes(p_dtype))) && aligned(q, std::min(16, v * dtype_bytes(q_dtype))))
      return v;
  return 1;
}

// f(X, O): the types as values of their own
template <class F>
cudaError_t with_types(int x, int o, F f) {
  if (x == MOLT_FP32) return f(float{}, float{});
  if (x == MOLT_FP16) return o == MOLT_FP32 ? f(__half{}, float{}) : f(__half{}, __half{});
  return o == MOLT_FP32 ? f(__nv_bfloat16{}, float{}) : f(__nv_bfloat16{}, __nv_bfloat16{});
}

// threads that hold `n` vectors of a row between them, at most 256, in whole warps and
// as evenly as the row divides
struct Group {
  int threads, slabs, per_block;
};
Group group_of(int64_t n_vec) {
  Group g;
  g.slabs = static_cast<int>((n_vec + 255) / 256);
  g.threads = static_cast<int>(((n_vec + g.slabs - 1) / g.slabs + 31) / 32 * 32);
  g.per_block = 256 / g.threads;
  return g;
}

// Sorted positions to a unit: enough units to fill the GPU several times, few enough
// that the parts of crossing runs stay a small share of the rows read.
int unit_of(int64_t T) {
  int u = 8;
  while (u < 64 && T / u > 1024) u *= 2;
  return u;
}

struct GradLayout {
  size_t keys[2], pos[2], cross, part, total;
};
GradLayout grad_layout(int64_t T, int64_t H) {
  GradLayout L{};
  size_t o = 0;
  auto take = [&o](size_t bytes) {
    const size_t r = o;
    o += (bytes + 255) & ~size_t(255);
    return r;
  };
  for (int i = 0; i < 2; ++i) {
    L.keys[i] = take(static_cast<size_t>(T) * 4);
    L.pos[i] = take(static_cast<size_t>(T) * 4);
  }
  // no fewer units for a larger T: units double in size where their number would fall
  const int64_t units = std::min<int64_t>((T + 7) / 8, std::max<int64_t>(1025, (T + 63) / 64));
  L.cross = take(static_cast<size_t>(units + 1) * 16);
  L.part = take(static_cast<size_t>(units) * 2 * H * sizeof(float));
  L.total = o + 256;
  return L;
}

}  // namespace
}  // namespace molt

using namespace molt;

extern "C" {

molt_status molt_token_embedding(const void* E, int E_dtype, const int32_t* tokens, int64_t T, int64_t H, int64_t V,
                                 float scale, void* out, int out_dtype, cudaStream_t stream) {
  if (const molt_status st = check(T, H, V, E_dtype, out_dtype, scale); st != MOLT_OK) return st;
  if (T == 0) return MOLT_OK;
  if (!E || !tokens || !out) return fail(MOLT_ERR_INVALID_ARG, "null pointer");
  if (!aligned(E, dtype_bytes(E_dtype)) || !aligned(out, dtype_bytes(out_dtype)) || !aligned(tokens, 4))
    return fail(MOLT_ERR_INVALID_ARG, "a pointer is not aligned to its element type");
  molt_status st;
  EmbedArgs a{E, tokens, T, static_cast<int>(V), static_cast<int>(H), scale, out, device_status_word(&st)};
  if (!a.err) return st;
  const int vec = vec_of(H, E, E_dtype, out, out_dtype);
  const Group g = group_of(H / vec);
  // four rows to a thread keep enough loads in flight; where that leaves SMs idle, one
  const int rows = T >= 4 * int64_t(device_sm_count()) * g.per_block ? 4 : 1;
  const int grid = static_cast<int>((T + rows * g.per_block - 1) / (rows * g.per_block));
  const dim3 block(g.threads, g.per_block);
  const cudaError_t e = with_types(E_dtype, out_dtype, [&](auto x, auto o) {
    using X = decltype(x);
    using O = decltype(o);
    auto* k = vec == 8   ? (rows == 4 ? embed_kernel<X, O, 8, 4> : embed_kernel<X, O, 8, 1>)
              : vec == 4 ? (rows == 4 ? embed_kernel<X, O, 4, 4> : embed_kernel<X, O, 4, 1>)
              : vec == 2 ? (rows == 4 ? embed_kernel<X, O, 2, 4> : embed_kernel<X, O, 2, 1>)
                         : (rows == 4 ? embed_kernel<X, O, 1, 4> : embed_kernel<X, O, 1, 1>);
    k<<<grid, block, 0, stream>>>(a);
    return cudaGetLastError();
  });
  if (e != cudaSuccess) return cuda_fail(e, "token embedding");
  note_launches(1);
  return MOLT_OK;
}

size_t molt_token_embedding_bwd_workspace_bytes(int64_t T, int64_t H, int64_t V) {
  if (check(T, H, V, MOLT_FP32, MOLT_FP32, 1.f) != MOLT_OK) return 0;
  return grad_layout(T, H).total;
}

molt_status molt_token_embedding_bwd(const void* dout, int dout_dtype, const int32_t* tokens, int64_t T, int64_t H,
                                     int64_t V, float scale, int64_t padding_idx, void* dE, int dE_dtype, int accumulate,
                                     void* workspace, size_t workspace_bytes, cudaStream_t stream) {
  if (const molt_status st = check(T, H, V, dout_dtype, dE_dtype, scale); st != MOLT_OK) return st;
  if (!dE || (T > 0 && (!dout || !tokens))) return fail(MOLT_ERR_INVALID_ARG, "null pointer");
  if (!aligned(dE, dtype_bytes(dE_dtype)) || !aligned(dout, dtype_bytes(dout_dtype)) || !aligned(tokens, 4))
    return fail(MOLT_ERR_INVALID_ARG, "a pointer is not aligned to its element type");
  if (accumulate && dE_dtype != MOLT_FP32) return fail(MOLT_ERR_INVALID_ARG, "only an fp32 gradient can be added to");
  if (padding_idx >= V) return fail(MOLT_ERR_INVALID_ARG, "padding_idx must be below V (negative: none)");
  if (T == 0) {
    if (accumulate) return MOLT_OK;
    const cudaError_t e = cudaMemsetAsync(dE, 0, static_cast<size_t>(V) * H * dtype_bytes(dE_dtype), stream);
    return e == cudaSuccess ? MOLT_OK : cuda_fail(e, "memset dE");
  }
  molt_status st;
  unsigned* err = device_status_word(&st);
  if (!err) return st;
  const GradLayout L = grad_layout(T, H);
  Scratch sc;
  if (st = get_scratch(sc, workspace, workspace_bytes, L.total, stream); st != MOLT_OK) return st;
  uint8_t* p = static_cast<uint8_t*>(sc.aligned());
  uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(p + L.keys[0]), reinterpret_cast<uint32_t*>(p + L.keys[1])};
  uint32_t* pos[2] = {reinterpret_cast<uint32_t*>(p + L.pos[0]), reinterpret_cast<uint32_t*>(p + L.pos[1])};
  int* n_cross = reinterpret_cast<int*>(p + L.cross);
  const int n = static_cast<int>(T);

  const int padding = static_cast<int>(padding_idx < 0 ? -1 : padding_idx);
  const int sort_blocks = (n + kSortElems - 1) / kSortElems;
  const int merge_blocks = (n + kMergeElems - 1) / kMergeElems;
  auto* sort = V < (int64_t(1) << (32 - kSortBits)) ? sort_chunks_kernel<uint32_t> : sort_chunks_kernel<uint64_t>;
  sort<<<sort_blocks, kSortThreads, 0, stream>>>(tokens, n, static_cast<int>(V), padding, keys[0], pos[0], n_cross, err);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return cuda_fail(e, "token sort");
  note_launches(1);
  int at = 0;
  for (int64_t len = kSortChunk; len < T; len *= kMergeLists) {
    const int lists = static_cast<int>(std::min<int64_t>(kMergeLists, (T + len - 1) / len));
    merge_lists_kernel<<<merge_blocks, kMergeThreads, 0, stream>>>(keys[at], pos[at], n, len, lists, keys[1 - at],
                                                                   pos[1 - at]);
    if (e = cudaGetLastError(); e != cudaSuccess) return cuda_fail(e, "token merge");
    note_launches(1);
    at = 1 - at;
  }

  const int vec = vec_of(H, dout, dout_dtype, dE, dE_dtype);
  const Group g = group_of((H + 7) / 8);
  EmbedGradArgs a{};
  a.dout = dout;
  a.keys = keys[at];
  a.pos = pos[at];
  a.T = n;
  a.V = static_cast<int>(V);
  a.H = static_cast<int>(H);
  a.unit = unit_of(T);
  a.n_units = (n + a.unit - 1) / a.unit;
  a.n_slabs = g.slabs;
  a.slab = g.threads * 8;
  a.sum_blocks = (a.n_units + g.per_block - 1) / g.per_block * g.slabs;
  // at most 64 KB of dE to a zeroing warp, and 64 warps or more to an SM
  a.zero_rows = static_cast<int>(std::max<int64_t>(
      1, std::min({int64_t(32), 65536 / (H * dtype_bytes(dE_dtype)), V / (64 * int64_t(device_sm_count()))})));
  const int64_t block_rows = static_cast<int64_t>(a.zero_rows) * (g.threads * g.per_block / 32);
  a.zero_blocks = accumulate ? 0 : static_cast<int>((V + block_rows - 1) / block_rows);
  a.add = accumulate != 0;
  a.scale = scale;
  a.dE = dE;
  a.part = reinterpret_cast<float*>(p + L.part);
  a.n_cross = n_cross;
  a.cross = reinterpret_cast<int4*>(n_cross) + 1;
  e = with_types(dout_dtype, dE_dtype, [&](auto x, auto o) {
    using X = decltype(x);
    using O = decltype(o);
    auto* k = vec == 8   ? embed_grad_kernel<X, O, 8>
              : vec == 4 ? embed_grad_kernel<X, O, 4>
              : vec == 2 ? embed_grad_kernel<X, O, 2>
                         : embed_grad_kernel<X, O, 1>;
    k<<<a.sum_blocks + a.zero_blocks, dim3(g.threads, g.per_block), 0, stream>>>(a);
    return cudaGetLastError();
  });
  if (e != cudaSuccess) return cuda_fail(e, "embedding gradient");
  note_launches(1);
  if (a.n_units == 1) return MOLT_OK;
  e = with_types(dE_dtype, dE_dtype, [&](auto o, auto) {
    const int cols = (a.H + kJoinCols - 1) / kJoinCols;
    // one wave of blocks
    const int runs = std::min((a.n_units + kJoinWarps - 2) / kJoinWarps, std::max(1, 8 * device_sm_count() / cols));
    embed_join_kernel<decltype(o)><<<dim3(cols, runs), 32 * kJoinWarps, 0, stream>>>(a);
    return cudaGetLastError();
  });
  if (e != cudaSuccess) return cuda_fail(e, "embedding gradient join");
  note_launches(1);
  return MOLT_OK;
}

}  // extern "C"
