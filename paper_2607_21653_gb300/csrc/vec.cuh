// Element types of the row operators (residual norm, embedding) and their loads and
// stores, all through fp32 registers.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

namespace molt {

// element types (values of molt_dtype)
constexpr int kBF16 = 0, kFP16 = 1, kFP32 = 2;
inline int dtype_bytes(int dt) { return dt == kFP32 ? 4 : 2; }

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ void from_float(float v, float& o) { o = v; }
__device__ __forceinline__ void from_float(float v, __nv_bfloat16& o) { o = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_float(float v, __half& o) { o = __float2half_rn(v); }

__device__ __forceinline__ void unpack2(uint32_t w, const __nv_bfloat16*, float& a, float& b) {
  a = __uint_as_float(w << 16);
  b = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack2(uint32_t w, const __half*, float& a, float& b) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
  a = f.x;
  b = f.y;
}
__device__ __forceinline__ uint32_t pack2(float a, float b, const __nv_bfloat16*) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, const __half*) {
  const __half2 p = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// kV = 1, 2, 4 or 8 consecutive elements, aligned to their size (at most 16 bytes)
template <int kV, class T>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[kV]) {
  if constexpr (kV == 1) {
    v[0] = to_float(*p);
  } else if constexpr (kV == 2 && sizeof(T) == 4) {
    const float2 a = *reinterpret_cast<const float2*>(p);
    v[0] = a.x, v[1] = a.y;
  } else if constexpr (kV == 4 && sizeof(T) == 4) {
    const float4 a = *reinterpret_cast<const float4*>(p);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
  } else if constexpr (kV == 2) {
    unpack2(*reinterpret_cast<const uint32_t*>(p), p, v[0], v[1]);
  } else if constexpr (kV == 4) {
    const uint2 a = *reinterpret_cast<const uint2*>(p);
    unpack2(a.x, p, v[0], v[1]);
    unpack2(a.y, p, v[2], v[3]);
  } else if constexpr (sizeof(T) == 4) {
    static_assert(kV == 8);
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
    static_assert(kV == 8);
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    unpack2(a.x, p, v[0], v[1]);
    unpack2(a.y, p, v[2], v[3]);
    unpack2(a.z, p, v[4], v[5]);
    unpack2(a.w, p, v[6], v[7]);
  }
}
template <int kV, class T>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[kV]) {
  if constexpr (kV == 1) {
    from_float(v[0], *p);
  } else if constexpr (kV == 2 && sizeof(T) == 4) {
    *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
  } else if constexpr (kV == 4 && sizeof(T) == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else if constexpr (kV == 2) {
    *reinterpret_cast<uint32_t*>(p) = pack2(v[0], v[1], p);
  } else if constexpr (kV == 4) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack2(v[0], v[1], p), pack2(v[2], v[3], p));
  } else if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    *reinterpret_cast<uint4*>(p) =
        make_uint4(pack2(v[0], v[1], p), pack2(v[2], v[3], p), pack2(v[4], v[5], p), pack2(v[6], v[7], p));
  }
}

// ------------------------------------------------- pairs of fp32
// One instruction for both.  Kept as one 64-bit value: as two floats, packed for every
// operation, the copies cost more than the pairs save.
struct F2 {
  unsigned long long v;
  __device__ __forceinline__ float x() const { return __uint_as_float(static_cast<uint32_t>(v)); }
  __device__ __forceinline__ float y() const { return __uint_as_float(static_cast<uint32_t>(v >> 32)); }
};
__device__ __forceinline__ F2 f2(float x, float y) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ F2 f2(float x) { return f2(x, x); }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
// 8 consecutive elements as pairs, 16-byte aligned
template <class T>
__device__ __forceinline__ void load_pairs(const T* p, F2* v) {
  if constexpr (sizeof(T) == 4) {
    const ulonglong2 a = reinterpret_cast<const ulonglong2*>(p)[0], b = reinterpret_cast<const ulonglong2*>(p)[1];
    v[0].v = a.x, v[1].v = a.y, v[2].v = b.x, v[3].v = b.y;
  } else {
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float lo, hi;
      unpack2(w[j], p, lo, hi);
      v[j] = f2(lo, hi);
    }
  }
}
template <class T>
__device__ __forceinline__ void store_pairs(T* p, const F2* v) {
  if constexpr (sizeof(T) == 4) {
    reinterpret_cast<ulonglong2*>(p)[0] = make_ulonglong2(v[0].v, v[1].v);
    reinterpret_cast<ulonglong2*>(p)[1] = make_ulonglong2(v[2].v, v[3].v);
  } else {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2(v[0].x(), v[0].y(), p), pack2(v[1].x(), v[1].y(), p),
                                              pack2(v[2].x(), v[2].y(), p), pack2(v[3].x(), v[3].y(), p));
  }
}

}  // namespace molt
