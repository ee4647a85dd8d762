// Dropout whose mask is a function of (seed, offset, row, column) and never stored:
//
//   out = res_scale residual + keep x / (1 - q),   q = round(2^16 p) / 2^16
//
// keep(row, column): 16 bits of Philox4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", SC 2011) are not below 2^16 q.  The
// counter's words are (column / 8, row, offset low, offset high), the key is the seed; one
// call of the generator serves eight columns, column 8 g + j taking half j % 2 (low first)
// of word j / 2.  The backward is the same map on the gradient.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cuda_runtime.h>
#include <initializer_list>

#include "molt_internal.cuh"
#include "vec.cuh"

namespace molt {
namespace {

constexpr int kThreads = 256;

struct DropArgs {
  const void *x, *residual;
  void* out;
  int64_t T, x_ld, r_ld;
  int H, groups;            // groups of eight columns of a row
  int rows;                 // rows of a tile
  uint32_t magic;           // i / groups = (i magic) >> 32 inside a tile
  uint32_t bound;           // keep: 16 bits, in a word's upper half, are not below it
  uint32_t row0;
  float scale, res_scale;
  uint64_t offset;
  uint2 keys[10];           // the rounds' keys of a seed on the host
  const uint64_t* words;    // seed and offset on the device, or nullptr
};

__host__ __device__ inline void round_keys(uint64_t seed, uint2 (&keys)[10]) {
  uint32_t x = static_cast<uint32_t>(seed), y = static_cast<uint32_t>(seed >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    keys[i].x = x;
    keys[i].y = y;
    x += 0x9E3779B9u;
    y += 0xBB67AE85u;
  }
}
// 128 bits of the generator.  The rounds' keys stand in the launch's parameters (or, of a seed on
// the device, in registers), where an instruction takes them as they are.
__device__ __forceinline__ uint4 philox(uint4 c, const uint2 (&k)[10]) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p0 = uint64_t(0xD2511F53u) * c.x, p1 = uint64_t(0xCD9E8D57u) * c.z;
    c = make_uint4(static_cast<uint32_t>(p1 >> 32) ^ c.y ^ k[i].x, static_cast<uint32_t>(p1),
                   static_cast<uint32_t>(p0 >> 32) ^ c.w ^ k[i].y, static_cast<uint32_t>(p0));
  }
  return c;
}

// 16 bytes, asked for where the statement stands; kApart: of a tensor that the call does not write
// (16001 x 5120 bf16: 62 us as read-only data, else 69).
template <bool kApart>
__device__ __forceinline__ uint4 load_now(const void* p) {
  uint4 v;
  if constexpr (kApart)
    asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  else
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// Eight elements as they are in memory.
template <class T, bool kApart>
struct Raw8 {
  uint4 q[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) q[i] = load_now<kApart>(reinterpret_cast<const uint4*>(p) + i);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const { load_vec<8>(reinterpret_cast<const T*>(q), v); }
};

// A thread's next group is on its way while it works on one (32768 x 4096 into an fp32 stream 240 us
// without, 212 with two groups at once, 205 so; 16001 x 5120 bf16 64, 73 and 62).
template <class Tin, class Tout, bool kVec, bool kRes, bool kWords, bool kApart>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const __grid_constant__ DropArgs a) {
  const Tin* x = static_cast<const Tin*>(a.x);
  const Tout* res = static_cast<const Tout*>(a.residual);
  Tout* out = static_cast<Tout*>(a.out);
  uint2 own_keys[10];
  uint64_t offset = a.offset;
  if constexpr (kWords) {
    round_keys(a.words[0], own_keys);
    offset = a.words[1];
  }
  struct Group {
    int64_t t;
    int c;
  };
  for (int64_t t0 = int64_t(blockIdx.x) * a.rows; t0 < a.T; t0 += int64_t(gridDim.x) * a.rows) {
    const int n = static_cast<int>(min(int64_t(a.rows), a.T - t0)) * a.groups;
    auto group = [&](int i) -> Group {
      const int r = a.groups == 1 ? i : static_cast<int>(__umulhi(static_cast<uint32_t>(i), a.magic));
      return {t0 + r, (i - r * a.groups) * 8};
    };
    auto random = [&](const Group& g) -> uint4 {
      const uint4 c = make_uint4(static_cast<uint32_t>(g.c) / 8u, a.row0 + static_cast<uint32_t>(g.t), static_cast<uint32_t>(offset),
                                 static_cast<uint32_t>(offset >> 32));
      if constexpr (kWords)
        return philox(c, own_keys);
      else
        return philox(c, a.keys);
    };
    auto kept = [&](const uint4& w, int j) -> bool {
      const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
      return (j & 1 ? ws[j / 2] & 0xffff0000u : ws[j / 2] << 16) >= a.bound;
    };
    auto work = [&](const Group& g, float (&v)[8], float (&o)[8]) {
      const uint4 w = random(g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // a dropped value is left out, not multiplied by zero
        const float d = kept(w, j) ? v[j] * a.scale : 0.f;
        o[j] = kRes ? fmaf(a.res_scale, o[j], d) : d;
      }
    };
    if constexpr (kVec) {
      Raw8<Tin, kApart> xr, x_next;
      Raw8<Tout, kApart> rr, r_next;
      int i = threadIdx.x;
      Group g = group(i);
      if (i < n) {
        xr.load(x + g.t * a.x_ld + g.c);
        if constexpr (kRes) rr.load(res + g.t * a.r_ld + g.c);
      }
      while (i < n) {
        const int next = i + kThreads;
        const Group h = group(next);
        if (next < n) {
          x_next.load(x + h.t * a.x_ld + h.c);
          if constexpr (kRes) r_next.load(res + h.t * a.r_ld + h.c);
        }
        float v[8], o[8];
        xr.get(v);
        if constexpr (kRes) rr.get(o);
        work(g, v, o);
        store_vec<8>(out + g.t * a.H + g.c, o);
        i = next;
        g = h;
        xr = x_next;
        rr = r_next;
      }
    } else {
      // a warp's 32 groups element by element, neighbours in neighbouring lanes: lane l of pass j has
      // element l % 8 of the group of lane 4 j + l / 8, which sends it what is known of the group
      // (20000 x 1031 bf16 43 us, 60 where every thread has the elements of its own group)
      const int lane = threadIdx.x & 31, k = lane % 8;
      const Tin* const x_tile = x + t0 * a.x_ld;
      const Tout* const res_tile = res + (kRes ? t0 * a.r_ld : 0);
      Tout* const out_tile = out + t0 * a.H;
      for (int i0 = threadIdx.x - lane; i0 < n; i0 += kThreads) {
        const Group g = group(i0 + lane);
        const uint32_t row = static_cast<uint32_t>(g.t - t0);
        const uint32_t count = i0 + lane < n ? min(8, a.H - g.c) : 0;
        const uint32_t x_at = row * static_cast<uint32_t>(a.x_ld) + g.c, r_at = row * static_cast<uint32_t>(a.r_ld) + g.c;
        const uint32_t out_at = row * static_cast<uint32_t>(a.H) + g.c;
        float v[8], r[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int from = 4 * j + lane / 8;
          const bool in = k < __shfl_sync(0xffffffffu, count, from);
          const uint32_t at = __shfl_sync(0xffffffffu, x_at, from) + k;
          v[j] = in ? to_float(x_tile[at]) : 0.f;
          if constexpr (kRes) {
            const uint32_t at_r = __shfl_sync(0xffffffffu, r_at, from) + k;
            r[j] = in ? to_float(res_tile[at_r]) : 0.f;
          }
        }
        const uint4 w = random(g);
        uint32_t flags = 0;   // kept, and behind the eight: there
#pragma unroll
        for (int j = 0; j < 8; ++j) flags |= (kept(w, j) ? 1u << j : 0u) | (j < count ? 256u << j : 0u);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int from = 4 * j + lane / 8;
          const uint32_t f = __shfl_sync(0xffffffffu, flags, from) >> k, at = __shfl_sync(0xffffffffu, out_at, from) + k;
          const float d = f & 1u ? v[j] * a.scale : 0.f;
          if (f & 256u) from_float(kRes ? fmaf(a.res_scale, r[j], d) : d, out_tile[at]);
        }
      }
    }
  }
}

molt_status fail(molt_status s, const char* msg) {
  set_last_error(msg);
  return s;
}

template <class Tin, class Tout, bool kVec, bool kRes>
void launch(const DropArgs& a, int grid, cudaStream_t s) {
  const bool apart = kVec && a.out != a.x && a.out != a.residual;
  const auto k = a.words ? (apart ? dropout_kernel<Tin, Tout, kVec, kRes, true, kVec> : dropout_kernel<Tin, Tout, kVec, kRes, true, false>)
                         : (apart ? dropout_kernel<Tin, Tout, kVec, kRes, false, kVec> : dropout_kernel<Tin, Tout, kVec, kRes, false, false>);
  k<<<grid, kThreads, 0, s>>>(a);
}
template <class Tin, class Tout>
void launch(const DropArgs& a, bool vec, int grid, cudaStream_t s) {
  if (vec)
    a.residual ? launch<Tin, Tout, true, true>(a, grid, s) : launch<Tin, Tout, true, false>(a, grid, s);
  else
    a.residual ? launch<Tin, Tout, false, true>(a, grid, s) : launch<Tin, Tout, false, false>(a, grid, s);
}

bool known_type(int dt) { return dt == MOLT_BF16 || dt == MOLT_FP16 || dt == MOLT_FP32; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace
}  // namespace molt

using namespace molt;

extern "C" molt_status molt_dropout(const molt_dropout_desc* d, const void* x, const void* residual,
                                    const uint64_t* seed_offset, void* out, cudaStream_t stream) {
  if (!d) return fail(MOLT_ERR_INVALID_ARG, "desc is NULL");
  if (d->T < 0 || d->H < 1) return fail(MOLT_ERR_INVALID_ARG, "sizes must satisfy T >= 0, H >= 1");
  if (d->H > 65536 || d->T > (int64_t(1) << 32) || d->first_row < 0 || d->first_row > (int64_t(1) << 32) - d->T)
    return fail(MOLT_ERR_UNSUPPORTED_SHAPE, "H must be at most 65536 and the rows lie in [0, 2^32)");
  if (!known_type(d->dtype) || !known_type(d->out_dtype)) return fail(MOLT_ERR_INVALID_ARG, "unknown element type");
  if (d->dtype != d->out_dtype && d->dtype != MOLT_FP32 && d->out_dtype != MOLT_FP32)
    return fail(MOLT_ERR_INVALID_ARG, "x and out are of one type, or one of them is fp32");
  if (!(d->p >= 0.0 && d->p <= 1.0)) return fail(MOLT_ERR_INVALID_ARG, "p must be in [0, 1]");
  if (!(d->res_scale >= -1e30f && d->res_scale <= 1e30f)) return fail(MOLT_ERR_INVALID_ARG, "res_scale must be finite");
  for (const int64_t ld : {d->x_stride, d->residual_stride})
    if (ld != 0 && ld < d->H) return fail(MOLT_ERR_INVALID_ARG, "a row stride is 0 (rows side by side) or at least H");
  if (d->T == 0) return MOLT_OK;
  if (!x || !out) return fail(MOLT_ERR_INVALID_ARG, "null pointer");
  const size_t ib = static_cast<size_t>(dtype_bytes(d->dtype)), ob = static_cast<size_t>(dtype_bytes(d->out_dtype));
  if (!aligned(x, ib) || !aligned(residual, ob) || !aligned(out, ob) || !aligned(seed_offset, 8))
    return fail(MOLT_ERR_INVALID_ARG, "a pointer is not aligned to its element type");
  const int64_t x_ld = d->x_stride ? d->x_stride : d->H, r_ld = d->residual_stride ? d->residual_stride : d->H;
  // written where it is read, element by element, by the thread that has read it
  if ((x == out && (ib != ob || (x_ld != d->H && d->T > 1))) || (residual == out && r_ld != d->H && d->T > 1))
    return fail(MOLT_ERR_INVALID_ARG, "a tensor is updated in place where its rows lie side by side and its type stays");
  if (const int eb = static_cast<int>(ib); !spans_apart({{out, d->T, d->H, static_cast<int>(ob)}},
                                                        {{x == out ? nullptr : x, d->T, d->H, eb, x_ld},
                                                         {residual == out ? nullptr : residual, d->T, d->H, static_cast<int>(ob), r_ld}}))
    return fail(MOLT_ERR_INVALID_ARG, "out is x, the residual or memory of its own");
  DropArgs a{};
  a.x = x;
  a.residual = residual;
  a.out = out;
  a.T = d->T;
  a.H = static_cast<int>(d->H);
  a.x_ld = x_ld;
  a.r_ld = r_ld;
  a.groups = (a.H + 7) / 8;
  // up to 16 groups to a thread, fewer where there would be too few blocks; i < 2^13 and groups
  // <= 2^13, so that the magic division is exact (i groups < 2^32)
  const int64_t most = 8 * int64_t(device_sm_count());
  a.rows = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(16 * kThreads / a.groups, (d->T + most - 1) / most)));
  a.rows = std::max(a.rows, std::min(1024, kThreads / a.groups));
  // places in a tile have 32 bits
  a.rows = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(a.rows, INT32_MAX / std::max(x_ld, r_ld) - 1)));
  a.magic = a.groups == 1 ? 0 : static_cast<uint32_t>(((uint64_t(1) << 32) + a.groups - 1) / a.groups);
  const uint32_t threshold = static_cast<uint32_t>(std::floor(d->p * 65536.0 + 0.5));
  a.bound = threshold < 65536 ? threshold << 16 : 0xffffffffu;   // (no 16 bits in an upper half reach that)
  a.scale = threshold < 65536 ? static_cast<float>(65536.0 / (65536.0 - threshold)) : 0.f;
  a.res_scale = d->res_scale;
  a.row0 = static_cast<uint32_t>(d->first_row);
  round_keys(d->seed, a.keys);
  a.offset = d->offset;
  a.words = seed_offset;
  const bool vec = a.H % 8 == 0 && aligned(x, 16) && aligned(out, 16) && aligned(residual, 16) && x_ld * ib % 16 == 0 &&
                   r_ld * ob % 16 == 0;
  const int64_t tiles = (d->T + a.rows - 1) / a.rows;
  const int grid = static_cast<int>(tiles < most ? tiles : most);
  using Launch = void (*)(const DropArgs&, bool, int, cudaStream_t);
  const bool i32 = d->dtype == MOLT_FP32, o32 = d->out_dtype == MOLT_FP32;
  const bool half = (i32 ? d->out_dtype : d->dtype) == MOLT_FP16;
  const Launch k = i32 && o32 ? &launch<float, float>
                   : i32      ? (half ? &launch<float, __half> : &launch<float, __nv_bfloat16>)
                   : o32      ? (half ? &launch<__half, float> : &launch<__nv_bfloat16, float>)
                              : (half ? &launch<__half, __half> : &launch<__nv_bfloat16, __nv_bfloat16>);
  k(a, vec, grid, stream);
  if (const cudaError_t e = cudaGetLastError(); e != cudaSuccess) {
    set_last_error(std::string("dropout: ") + cudaGetErrorString(e));
    return MOLT_ERR_CUDA;
  }
  note_launches(1);
  return MOLT_OK;
}
