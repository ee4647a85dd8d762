// Token embedding with scaling, and its gradient by sorted tokens.
//
//   out_t = s E[x_t]          dE_v = s sum_{t: x_t = v} dout_t
//
// Forward: a gather, bound by HBM (each row of E that occurs and out once).
//
// Gradient: the positions are sorted by token (stably, so equal tokens stay in token
// order), cut into units of equally many sorted positions, and every unit adds up its
// runs of equal tokens in fp32.  A run inside a unit is written at once; a run that
// crosses units leaves one fp32 part in each, which a last kernel adds in order.  So a
// token that fills a tenth of the batch is spread over as many units as it needs, no
// atomics are used and the results are the same bits in every run.  Rows of tokens that
// do not occur are zeroed by blocks of the same launch, mixed with the units, so that
// dE is written exactly once.
//
// Sorting: chunks of kSortChunk positions by one block each (stable LSD radix in
// shared memory), then every element finds its place among up to kMergeLists sorted
// chunks by binary search.
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

// ------------------------------------------------------------------- sorting
constexpr int kSortThreads = 1024, kSortItems = 8, kSortChunk = kSortThreads * kSortItems;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMergeLists = 16;

// One block: the chunk's positions sorted by token.  Tokens that give no gradient
// (outside [0, V), or the padding token) get the key V and so come last.  `present`
// (nullptr: not wanted) is zeroed by all blocks, and with one block also marked.
// A pass ranks by `width` bits: a warp ranks its 256 consecutive items 32 at a time
// (matching lanes, then a running count per digit), the block scans the counts by
// digit and warp, and the items move to their places.
__global__ void __launch_bounds__(kSortThreads) sort_chunks_kernel(const int32_t* __restrict__ tok, int T, int V, int padding,
                                                                   int passes, int width, uint32_t* __restrict__ keys_out,
                                                                   uint32_t* __restrict__ pos_out,
                                                                   uint8_t* __restrict__ present, unsigned* err) {
  extern __shared__ __align__(16) uint8_t smem[];
  uint32_t* sh_key = reinterpret_cast<uint32_t*>(smem);                       // [kSortChunk]
  uint16_t* sh_pos = reinterpret_cast<uint16_t*>(sh_key + kSortChunk);        // [kSortChunk]
  uint32_t* count = reinterpret_cast<uint32_t*>(sh_pos + kSortChunk);         // [bins][kSortWarps]
  __shared__ uint32_t warp_tot[kSortWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int bins = 1 << width;
  const int64_t base = static_cast<int64_t>(blockIdx.x) * kSortChunk;
  const int n = static_cast<int>(min(static_cast<int64_t>(kSortChunk), T - base));
  if (present != nullptr) {   // a buffer of whole 16-byte words
    const int words = (V + 16) / 16;
    for (int i = blockIdx.x * kSortThreads + threadIdx.x; i < words; i += gridDim.x * kSortThreads)
      reinterpret_cast<uint4*>(present)[i] = make_uint4(0, 0, 0, 0);
  }
  // item r of this thread is item (warp * 256 + r * 32 + lane) of the chunk
  uint32_t key[kSortItems], pos[kSortItems];
  bool bad = false;
#pragma unroll
  for (int r = 0; r < kSortItems; ++r) {
    const int i = warp * (32 * kSortItems) + r * 32 + lane;
    key[r] = 0xffffffffu;   // past the end: after every token
    pos[r] = i;
    if (i < n) {
      const int x = tok[base + i];
      const bool in = x >= 0 && x < V;
      bad |= !in;
      key[r] = in && x != padding ? x : V;
    }
  }
  if (bad) atomicOr(err, kDevErrTokenRange);
  const uint32_t mask = bins - 1, below = (1u << lane) - 1u;
  const int used_warps = (n + 32 * kSortItems - 1) / (32 * kSortItems);
  for (int p = 0; p < passes; ++p) {
    const int shift = p * width;
    for (int i = threadIdx.x; i < bins * kSortWarps; i += kSortThreads) count[i] = 0;
    __syncthreads();
    uint32_t rank[kSortItems];
    if (warp < used_warps) {
#pragma unroll
      for (int r = 0; r < kSortItems; ++r) {
        const uint32_t d = (key[r] >> shift) & mask;
        const unsigned same = __match_any_sync(0xffffffffu, d);
        uint32_t* c = count + d * kSortWarps + warp;
        const uint32_t before = *c;
        __syncwarp();
        rank[r] = before + __popc(same & below);
        if ((same & below) == 0) *c = before + __popc(same);
        __syncwarp();
      }
    }
    __syncthreads();
    // exclusive scan of the counts in order of (digit, warp)
    const int per = (bins * kSortWarps + kSortThreads - 1) / kSortThreads;   // 1 to 8, consecutive
    uint32_t own = 0;
    const int i0 = threadIdx.x * per;
    for (int i = 0; i < per; ++i)
      if (i0 + i < bins * kSortWarps) own += count[i0 + i];
    uint32_t incl = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) warp_tot[warp] = incl;
    __syncthreads();
    if (warp == 0) {
      const uint32_t v = warp_tot[lane];
      uint32_t s = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += u;
      }
      warp_tot[lane] = s - v;
    }
    __syncthreads();
    uint32_t run = warp_tot[warp] + incl - own;
    for (int i = 0; i < per; ++i)
      if (i0 + i < bins * kSortWarps) {
        const uint32_t c = count[i0 + i];
        count[i0 + i] = run;
        run += c;
      }
    __syncthreads();
    if (warp < used_warps) {
#pragma unroll
      for (int r = 0; r < kSortItems; ++r) {
        const uint32_t at = count[((key[r] >> shift) & mask) * kSortWarps + warp] + rank[r];
        sh_key[at] = key[r];
        sh_pos[at] = static_cast<uint16_t>(pos[r]);
      }
    }
    __syncthreads();
    if (warp < used_warps) {
#pragma unroll
      for (int r = 0; r < kSortItems; ++r) {
        const int i = warp * (32 * kSortItems) + r * 32 + lane;
        key[r] = sh_key[i];
        pos[r] = sh_pos[i];
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kSortItems; ++r) {
    const int i = warp * (32 * kSortItems) + r * 32 + lane;
    if (i < n) {
      keys_out[base + i] = key[r];
      pos_out[base + i] = static_cast<uint32_t>(base) + pos[r];
      if (present != nullptr && gridDim.x == 1) present[key[r]] = 1;
    }
  }
}

// Groups of up to kMergeLists sorted lists of `len` elements become one: an element's
// place is its own index plus, for every other list, the number of elements before it
// there (equal keys of earlier lists come first, as their positions do).  Warp y of a
// block searches list y of the group for 32 elements.
__global__ void __launch_bounds__(32 * kMergeLists) merge_lists_kernel(const uint32_t* __restrict__ keys,
                                                                       const uint32_t* __restrict__ pos, int T, int64_t len,
                                                                       uint32_t* __restrict__ keys_out,
                                                                       uint32_t* __restrict__ pos_out,
                                                                       uint8_t* __restrict__ present) {
  __shared__ int found[kMergeLists][32];
  const int64_t e = static_cast<int64_t>(blockIdx.x) * 32 + threadIdx.x;   // lists begin at multiples of 32
  const int64_t list = e / len, group0 = list / kMergeLists * kMergeLists * len;
  const int64_t mine = (list % kMergeLists);
  const bool in = e < T;
  const uint32_t k = in ? keys[e] : 0u;
  const int64_t l0 = group0 + threadIdx.y * len, l1 = min(static_cast<int64_t>(T), l0 + len);
  int n = 0;
  if (in && l0 < l1) {
    if (threadIdx.y == mine) {
      n = static_cast<int>(e - l0);
    } else {
      const bool earlier = threadIdx.y < mine;   // then equal keys count too
      int lo = 0, hi = static_cast<int>(l1 - l0);
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        const uint32_t v = keys[l0 + mid];
        if (v < k || (earlier && v == k))
          lo = mid + 1;
        else
          hi = mid;
      }
      n = lo;
    }
  }
  found[threadIdx.y][threadIdx.x] = n;
  __syncthreads();
  if (threadIdx.y != 0 || !in) return;
  int64_t at = group0;
  for (int y = 0; y < static_cast<int>(blockDim.y); ++y) at += found[y][threadIdx.x];
  keys_out[at] = k;
  pos_out[at] = pos[e];
  if (present != nullptr) present[k] = 1;
}

// ------------------------------------------------------------------ gradient
struct EmbedGradArgs {
  const void* dout;
  const uint32_t *keys, *pos;   // sorted
  const uint8_t* present;       // [V + 1], or nullptr: dE is added to
  int T, V, H;
  int unit;                     // sorted positions to a unit
  int n_units, n_slabs, slab;   // slab: columns that a group of threads holds
  int sum_blocks, zero_blocks, zero_rows;
  float scale;
  void* dE;
  float* part;                  // [n_units, 2, H]: sums of a run from the unit before / into the unit after
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

// n elements from p set to zero by `threads` threads, on any alignment
template <class O>
__device__ __forceinline__ void zero_span(O* p, int n, int thread, int threads) {
  const int head = min(n, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / static_cast<int>(sizeof(O)));
  constexpr int kPer = 16 / sizeof(O);
  const int body = (n - head) / kPer;
  O zero;
  from_float(0.f, zero);
  if (thread < head) p[thread] = zero;
  uint4* v = reinterpret_cast<uint4*>(p + head);
  for (int i = thread; i < body; i += threads) v[i] = make_uint4(0, 0, 0, 0);
  const int done = head + body * kPer;
  if (thread < n - done) p[done + thread] = zero;
}

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
    const int v0 = (blockIdx.x - sum_before) * a.zero_rows, v1 = min(a.V, v0 + a.zero_rows);
    for (int v = v0 + threadIdx.y; v < v1; v += blockDim.y)
      if (!a.present[v]) zero_span(dE + static_cast<int64_t>(v) * a.H, a.H, threadIdx.x, blockDim.x);
    return;
  }
  const int u = (sum_before / a.n_slabs) * blockDim.y + threadIdx.y;
  if (u >= a.n_units) return;
  const int col0 = (sum_before % a.n_slabs) * a.slab;
  const int i0 = u * a.unit, i1 = min(a.T, i0 + a.unit);
  const bool add = a.present == nullptr;
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
    float v[kBatch][N][kV];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      key[b] = i + b < i1 ? a.keys[i + b] : 0xffffffffu;
      const X* row = static_cast<const X*>(a.dout);
      if (key[b] < static_cast<uint32_t>(a.V)) row += static_cast<int64_t>(a.pos[i + b]) * a.H;
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int c = column(n);
#pragma unroll
        for (int j = 0; j < kV; ++j) v[b][n][j] = 0.f;
        if (key[b] < static_cast<uint32_t>(a.V) && c < a.H) load_vec<kV>(row + c, v[b][n]);
      }
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (i + b < i1 && key[b] != run) {
        flush(run, from_before, false);
        run = key[b];
        from_before = false;
        if (run >= static_cast<uint32_t>(a.V)) return;
      }
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int j = 0; j < kV; ++j) acc[n][j] += v[b][n][j];
    }
  }
  flush(run, from_before, i1 < a.T && a.keys[i1] == run);
}

constexpr int kJoinGroups = 8;

// The runs that cross units: the block of the unit where a run begins adds the units'
// parts, group y of threads every kJoinGroups-th of them, then the groups in order.
template <class O>
__global__ void __launch_bounds__(32 * kJoinGroups) embed_join_kernel(const EmbedGradArgs a) {
  __shared__ float sh[kJoinGroups][32];
  const int u = blockIdx.x;
  const int i0 = u * a.unit, i1 = min(a.T, i0 + a.unit);
  if (i1 >= a.T) return;
  const uint32_t key = a.keys[i1 - 1];
  if (key >= static_cast<uint32_t>(a.V) || a.keys[i1] != key) return;   // the unit's last run ends with it
  if (i0 > 0 && a.keys[i0] == key && a.keys[i0 - 1] == key) return;     // or began earlier
  // units of the run: parts are (u, 1), (u + 1, 0), ... while a unit begins with the key
  int lo = u + 1, hi = a.n_units - 1;   // last unit that begins with it
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.keys[mid * a.unit] == key)
      lo = mid;
    else
      hi = mid - 1;
  }
  const int n_parts = lo - u + 1;
  O* row = static_cast<O*>(a.dE) + static_cast<int64_t>(key) * a.H;
  for (int c0 = blockIdx.y * 32; c0 < a.H; c0 += gridDim.y * 32) {
    const int c = c0 + threadIdx.x;
    float s = 0.f;
    if (c < a.H) {
#pragma unroll 4
      for (int k = threadIdx.y; k < n_parts; k += kJoinGroups)
        s += a.part[(static_cast<int64_t>(u + k) * 2 + (k == 0 ? 1 : 0)) * a.H + c];
    }
    sh[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y == 0 && c < a.H) {
      float v[1] = {0.f};
#pragma unroll
      for (int y = 0; y < kJoinGroups; ++y) v[0] += sh[y][threadIdx.x];
      put_row<O, 1>(row + c, v, a.scale, a.present == nullptr);
    }
    __syncthreads();
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
  size_t keys[2], pos[2], present, part, total;
};
GradLayout grad_layout(int64_t T, int64_t H, int64_t V) {
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
  L.present = take(static_cast<size_t>(V) + 16);
  // no fewer units for a larger T: units double in size where their number would fall
  const int64_t units = std::min<int64_t>((T + 7) / 8, std::max<int64_t>(1025, (T + 63) / 64));
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
  const bool vec = H % 8 == 0 && aligned(E, 16) && aligned(out, 16);
  const Group g = group_of(vec ? H / 8 : H);
  // four rows to a thread keep enough loads in flight; where that leaves SMs idle, one
  const int rows = T >= 4 * int64_t(device_sm_count()) * g.per_block ? 4 : 1;
  const int grid = static_cast<int>((T + rows * g.per_block - 1) / (rows * g.per_block));
  const dim3 block(g.threads, g.per_block);
  const cudaError_t e = with_types(E_dtype, out_dtype, [&](auto x, auto o) {
    using X = decltype(x);
    using O = decltype(o);
    auto* k = vec ? (rows == 4 ? embed_kernel<X, O, 8, 4> : embed_kernel<X, O, 8, 1>)
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
  return grad_layout(T, H, V).total;
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
  const GradLayout L = grad_layout(T, H, V);
  Scratch sc;
  if (st = get_scratch(sc, workspace, workspace_bytes, L.total, stream); st != MOLT_OK) return st;
  uint8_t* p = static_cast<uint8_t*>(sc.aligned());
  uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(p + L.keys[0]), reinterpret_cast<uint32_t*>(p + L.keys[1])};
  uint32_t* pos[2] = {reinterpret_cast<uint32_t*>(p + L.pos[0]), reinterpret_cast<uint32_t*>(p + L.pos[1])};
  uint8_t* present = accumulate ? nullptr : p + L.present;
  const int n = static_cast<int>(T);

  // keys are 0 to V; a pass takes up to 8 of their bits
  int bits = 1;
  while ((V >> bits) != 0) ++bits;
  const int passes = (bits + 7) / 8, width = (bits + passes - 1) / passes;
  const size_t smem = kSortChunk * 6 + (size_t(1) << width) * kSortWarps * 4;
  cudaError_t e = cudaFuncSetAttribute(sort_chunks_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       kSortChunk * 6 + 256 * kSortWarps * 4);
  if (e != cudaSuccess) return cuda_fail(e, "token sort");
  sort_chunks_kernel<<<(n + kSortChunk - 1) / kSortChunk, kSortThreads, smem, stream>>>(
      tokens, n, static_cast<int>(V), static_cast<int>(padding_idx < 0 ? -1 : padding_idx), passes, width, keys[0], pos[0],
      present, err);
  if (e = cudaGetLastError(); e != cudaSuccess) return cuda_fail(e, "token sort");
  note_launches(1);
  int at = 0;
  for (int64_t len = kSortChunk; len < T; len *= kMergeLists) {
    const bool last = len * kMergeLists >= T;
    const int lists = static_cast<int>(std::min<int64_t>(kMergeLists, (T + len - 1) / len));
    merge_lists_kernel<<<(n + 31) / 32, dim3(32, lists), 0, stream>>>(keys[at], pos[at], n, len, keys[1 - at], pos[1 - at],
                                                                      last ? present : nullptr);
    if (e = cudaGetLastError(); e != cudaSuccess) return cuda_fail(e, "token merge");
    note_launches(1);
    at = 1 - at;
  }

  const bool vec = H % 8 == 0 && aligned(dout, 16) && aligned(dE, 16);
  const Group g = group_of((H + 7) / 8);
  EmbedGradArgs a{};
  a.dout = dout;
  a.keys = keys[at];
  a.pos = pos[at];
  a.present = present;
  a.T = n;
  a.V = static_cast<int>(V);
  a.H = static_cast<int>(H);
  a.unit = unit_of(T);
  a.n_units = (n + a.unit - 1) / a.unit;
  a.n_slabs = g.slabs;
  a.slab = g.threads * 8;
  a.sum_blocks = (a.n_units + g.per_block - 1) / g.per_block * g.slabs;
  // about 64 KB of dE to a zeroing block
  a.zero_rows = static_cast<int>(std::max<int64_t>(1, 65536 / (H * dtype_bytes(dE_dtype))));
  a.zero_blocks = accumulate ? 0 : static_cast<int>((V + a.zero_rows - 1) / a.zero_rows);
  a.scale = scale;
  a.dE = dE;
  a.part = reinterpret_cast<float*>(p + L.part);
  e = with_types(dout_dtype, dE_dtype, [&](auto x, auto o) {
    using X = decltype(x);
    using O = decltype(o);
    auto* k = vec ? embed_grad_kernel<X, O, 8> : embed_grad_kernel<X, O, 1>;
    k<<<a.sum_blocks + a.zero_blocks, dim3(g.threads, g.per_block), 0, stream>>>(a);
    return cudaGetLastError();
  });
  if (e != cudaSuccess) return cuda_fail(e, "embedding gradient");
  note_launches(1);
  if (a.n_units == 1) return MOLT_OK;
  e = with_types(dE_dtype, dE_dtype, [&](auto o, auto) {
    embed_join_kernel<decltype(o)><<<dim3(a.n_units, std::min(8, (a.H + 31) / 32)), dim3(32, kJoinGroups), 0, stream>>>(a);
    return cudaGetLastError();
  });
  if (e != cudaSuccess) return cuda_fail(e, "embedding gradient join");
  note_launches(1);
  return MOLT_OK;
}

}  // extern "C"
