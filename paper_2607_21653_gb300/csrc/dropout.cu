// Dropout whose mask is a function of (seed, offset, row, column) and never stored:
//
//   out = res_scale residual + keep x / (1 - q),   q = round(2^16 p) / 2^16
//
// keep(row, column): 16 bits of Philox4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", SC 2011) are not below 2^16 q.  The
// counter's words are (column / 8, row, offset low, offset high), the key is the seed; one
// call of the generator serves eight columns, column 8 g + j taking half j % 2 (low first)
// of word j / 2.  The backward is the same map on the gradient.
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
  uint32_t threshold, row0;
  float scale, res_scale;
  uint64_t seed, offset;
  const uint64_t* words;    // seed and offset on the device, or nullptr
};

// 128 bits of the generator
__device__ __forceinline__ uint4 philox(uint4 c, uint2 k) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p0 = uint64_t(0xD2511F53u) * c.x, p1 = uint64_t(0xCD9E8D57u) * c.z;
    c = make_uint4(static_cast<uint32_t>(p1 >> 32) ^ c.y ^ k.x, static_cast<uint32_t>(p1),
                   static_cast<uint32_t>(p0 >> 32) ^ c.w ^ k.y, static_cast<uint32_t>(p0));
    k.x += 0x9E3779B9u;
    k.y += 0xBB67AE85u;
  }
  return c;
}

template <class Tin, class Tout, bool kVec>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const DropArgs a) {
  const Tin* x = static_cast<const Tin*>(a.x);
  const Tout* res = static_cast<const Tout*>(a.residual);
  Tout* out = static_cast<Tout*>(a.out);
  const uint64_t seed = a.words ? a.words[0] : a.seed, offset = a.words ? a.words[1] : a.offset;
  const uint2 key = make_uint2(static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32));
  for (int64_t t0 = int64_t(blockIdx.x) * a.rows; t0 < a.T; t0 += int64_t(gridDim.x) * a.rows) {
    const int n = static_cast<int>(min(int64_t(a.rows), a.T - t0)) * a.groups;
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const int r = a.groups == 1 ? i : static_cast<int>(__umulhi(static_cast<uint32_t>(i), a.magic));
      const int g = i - r * a.groups, c = g * 8;
      const int64_t t = t0 + r;
      float v[8], o[8];
      const int left = min(8, a.H - c);
      if constexpr (kVec) {
        load_vec<8>(x + t * a.x_ld + c, v);
        if (res) load_vec<8>(res + t * a.r_ld + c, o);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[j] = j < left ? to_float(x[t * a.x_ld + c + j]) : 0.f;
          o[j] = res && j < left ? to_float(res[t * a.r_ld + c + j]) : 0.f;
        }
      }
      const uint4 w = philox(make_uint4(static_cast<uint32_t>(g), a.row0 + static_cast<uint32_t>(t),
                                        static_cast<uint32_t>(offset), static_cast<uint32_t>(offset >> 32)), key);
      const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t bits = j & 1 ? ws[j / 2] >> 16 : ws[j / 2] & 0xffffu;
        // a dropped value is left out, not multiplied by zero
        const float d = bits >= a.threshold ? v[j] * a.scale : 0.f;
        o[j] = res ? fmaf(a.res_scale, o[j], d) : d;
      }
      if constexpr (kVec) {
        store_vec<8>(out + t * a.H + c, o);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < left) from_float(o[j], out[t * a.H + c + j]);
      }
    }
  }
}

molt_status fail(molt_status s, const char* msg) {
  set_last_error(msg);
  return s;
}

template <class Tin, class Tout>
void launch(const DropArgs& a, bool vec, int grid, cudaStream_t s) {
  if (vec)
    dropout_kernel<Tin, Tout, true><<<grid, kThreads, 0, s>>>(a);
  else
    dropout_kernel<Tin, Tout, false><<<grid, kThreads, 0, s>>>(a);
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
  if (d->H > 65536 || d->T > (int64_t(1) << 32) || d->first_row < 0 || d->first_row + d->T > (int64_t(1) << 32))
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
  DropArgs a{};
  a.x = x;
  a.residual = residual;
  a.out = out;
  a.T = d->T;
  a.H = static_cast<int>(d->H);
  a.x_ld = x_ld;
  a.r_ld = r_ld;
  a.groups = (a.H + 7) / 8;
  // about eight groups to a thread; i < 2^14 and groups <= 2^13, so that the magic
  // division is exact (i groups < 2^32)
  a.rows = 8 * kThreads / a.groups > 1 ? 8 * kThreads / a.groups : 1;
  a.magic = a.groups == 1 ? 0 : static_cast<uint32_t>(((uint64_t(1) << 32) + a.groups - 1) / a.groups);
  a.threshold = static_cast<uint32_t>(std::floor(d->p * 65536.0 + 0.5));
  a.scale = a.threshold < 65536 ? static_cast<float>(65536.0 / (65536.0 - a.threshold)) : 0.f;
  a.res_scale = d->res_scale;
  a.row0 = static_cast<uint32_t>(d->first_row);
  a.seed = d->seed;
  a.offset = d->offset;
  a.words = seed_offset;
  const bool vec = a.H % 8 == 0 && aligned(x, 16) && aligned(out, 16) && aligned(residual, 16) && x_ld * ib % 16 == 0 &&
                   r_ld * ob % 16 == 0;
  const int64_t tiles = (d->T + a.rows - 1) / a.rows, most = 8 * int64_t(device_sm_count());
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
