// C ABI of the residual norm (include/molt.h): argument checks, the layout of a row
// over threads, and the sum of the blocks' parts of the weights' gradients.
#include <algorithm>
#include <cstdint>
#include <cuda_runtime.h>
#include <initializer_list>

#include "molt_internal.cuh"
#include "norm_kernels.cuh"

namespace molt {
namespace {

constexpr int kSumCols = 32, kSumWarps = 32;

// out[c] (+)= sum over blocks of part[block][which][c], blocks in a fixed order: warp w
// takes every 32nd, eight loads at a time, then the warps' sums are added in order.
__global__ void __launch_bounds__(kSumCols * kSumWarps) norm_part_sum_kernel(const float* __restrict__ part, int blocks, int H,
                                                                             float* o0, float* o1, float* o2, int accumulate) {
  __shared__ float sh[kSumWarps][kSumCols];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int which = blockIdx.y;
  float* out = which == 0 ? o0 : which == 1 ? o1 : o2;
  if (out == nullptr) return;
  const int c = blockIdx.x * kSumCols + lane;
  float s = 0.f;
  if (c < H) {
    for (int b0 = warp; b0 < blocks; b0 += 8 * kSumWarps) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int b = b0 + i * kSumWarps;
        v[i] = b < blocks ? part[(static_cast<int64_t>(b) * 3 + which) * H + c] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];
    }
  }
  sh[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || c >= H) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < kSumWarps; ++w) s += sh[w][lane];
  out[c] = accumulate ? out[c] + s : s;
}

molt_status fail(molt_status s, const char* msg) {
  set_last_error(msg);
  return s;
}
molt_status cuda_fail(cudaError_t e, const char* what) {
  set_last_error(std::string(what) + ": " + cudaGetErrorString(e));
  return MOLT_ERR_CUDA;
}

bool known_type(int dt) { return dt == MOLT_BF16 || dt == MOLT_FP16 || dt == MOLT_FP32; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Rows are counted in 32 bits and the persistent kernels go on by a grid's rows, at most
// kMaxBlocksPerSM * kRingRows to an SM, past the last one: 2^17 are those of 4096 SMs.
constexpr int64_t kMaxRows = (int64_t(1) << 31) - (int64_t(1) << 17);
static_assert(kMaxBlocksPerSM * kRingRows * 4096 <= 1 << 17);

molt_status check_desc(const molt_norm_desc* d) {
  if (!d) return fail(MOLT_ERR_INVALID_ARG, "desc is NULL");
  if (d->T < 0 || d->H < 1) return fail(MOLT_ERR_INVALID_ARG, "sizes must satisfy T >= 0, H >= 1");
  if (d->T > kMaxRows || d->H > 65536)
    return fail(MOLT_ERR_UNSUPPORTED_SHAPE, "T must be at most 2^31 - 2^17 and H at most 65536");
  if (!known_type(d->dtype) || !known_type(d->residual_dtype) || !known_type(d->param_dtype))
    return fail(MOLT_ERR_INVALID_ARG, "unknown element type");
  if (d->residual_dtype != d->dtype && d->residual_dtype != MOLT_FP32)
    return fail(MOLT_ERR_INVALID_ARG, "the residual stream is of x's type or fp32");
  if (d->param_dtype != d->dtype && d->param_dtype != MOLT_FP32)
    return fail(MOLT_ERR_INVALID_ARG, "the weights are of x's type or fp32");
  if (d->gate_kind < MOLT_GATE_NONE || d->gate_kind > MOLT_GATE_FULL) return fail(MOLT_ERR_INVALID_ARG, "unknown gate kind");
  if (!(d->eps >= 0.f && d->eps <= 1e30f)) return fail(MOLT_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (!(d->res_scale >= -1e30f && d->res_scale <= 1e30f) || !(d->weight_offset >= -1e30f && d->weight_offset <= 1e30f))
    return fail(MOLT_ERR_INVALID_ARG, "res_scale and weight_offset must be finite");
  for (const int64_t ld : {d->x_stride, d->residual_stride, d->dy_stride})
    if (ld != 0 && ld < d->H) return fail(MOLT_ERR_INVALID_ARG, "a row stride is 0 (rows side by side) or at least H");
  return MOLT_OK;
}

// every pointer that is given, aligned to its element
struct Operand {
  const void* p;
  int dtype;
};
molt_status check_elements(std::initializer_list<Operand> ops) {
  for (const Operand& o : ops)
    if (o.p && !aligned(o.p, static_cast<size_t>(dtype_bytes(o.dtype))))
      return fail(MOLT_ERR_INVALID_ARG, "a pointer is not aligned to its element type");
  return MOLT_OK;
}

NormArgs base_args(const molt_norm_desc* d) {
  NormArgs a{};
  a.T = d->T;
  a.H = static_cast<int>(d->H);
  a.x_ld = d->x_stride ? d->x_stride : d->H;
  a.r_ld = d->residual_stride ? d->residual_stride : d->H;
  a.dy_ld = d->dy_stride ? d->dy_stride : d->H;
  a.alpha = d->res_scale;
  a.eps = d->eps;
  a.offset = d->weight_offset;
  a.gate_kind = d->gate_kind;
  a.param_f32 = d->param_dtype == MOLT_FP32;
  return a;
}

// Elements that rows can be read at a time: eight, where the rows' length is in whole
// vectors and every row and parameter on a 16-byte boundary; two, where they are in whole
// pairs (20000 x 1566 with an fp32 stream, one and two at a time: forward 137 and 76 us,
// backward 188 and 178); or one.
int vector_of(const molt_norm_desc* d, const NormArgs& a, std::initializer_list<const void*> ptrs) {
  const int b = dtype_bytes(d->dtype), rb = dtype_bytes(d->residual_dtype);
  const auto based = [&](int bytes) {
    for (const void* p : ptrs)
      if (!aligned(p, bytes)) return false;
    return true;
  };
  if (a.H % 8 == 0 && a.x_ld * b % 16 == 0 && a.r_ld * rb % 16 == 0 && a.dy_ld * b % 16 == 0 && based(16)) return 8;
  // (bases for pairs of the widest type among them)
  const bool wide = b == 4 || rb == 4 || dtype_bytes(d->param_dtype) == 4;
  return a.H % 2 == 0 && a.x_ld % 2 == 0 && a.r_ld % 2 == 0 && a.dy_ld % 2 == 0 && based(wide ? 8 : 4) ? 2 : 1;
}

// Rows in registers, a block to each (or to four short ones): for the few rows of a
// decoding step, and for vectors of more elements than the persistent kernels hold.
NormShape row_shape(int H, int vec) {
  NormShape s{};
  s.vec = vec;
  s.elems = vec != 8 ? 0 : H <= 8 * kNormMaxThreads ? 8 : H <= 16 * kNormMaxThreads ? 16 : H <= kNormMaxH ? 32 : 0;
  s.threads = s.elems == 0 ? kNormMaxThreads : ((H + s.elems - 1) / s.elems + 31) / 32 * 32;
  s.rows = s.threads == 32 ? 4 : 1;
  return s;
}

int64_t max_blocks(int n_sm) { return kMaxBlocksPerSM * static_cast<int64_t>(n_sm); }

// The persistent form of a call (in s and a), or false for rows that 16 elements to a
// thread do not hold or shared memory does not.  A row's stage holds, side by side, what
// is read of it.
bool rows_shape(const molt_norm_desc* d, bool bwd, NormArgs& a, NormShape& s) {
  if (a.H > 16 * kNormMaxThreads) return false;
  // a row that begins inside a 16-byte word touches one more
  const auto bytes = [&](int dt) { return a.H * dtype_bytes(dt) / 16 * 16 + (s.vec == 8 ? 0 : 32); };
  const int xb = bytes(d->dtype), rb = bytes(d->residual_dtype);
  int at = xb;
  auto take = [&at](bool wanted, int n) {
    const int r = at;
    if (wanted) at += n;
    return r;
  };
  a.at_r = take(bwd ? a.w_pre != nullptr : a.r != nullptr, rb);
  a.at_dy = take(bwd && a.w_pre != nullptr, xb);
  a.at_dr = take(bwd && a.dr != nullptr, rb);
  a.at_gate = take(a.gate_kind == MOLT_GATE_FULL, xb);
  a.stage_bytes = at;
  // 16 elements to a thread where that makes a row one warp's, in the forward for longer
  // rows too (32768 x 2048 with an fp32 stream: 8 elements 151 us, 16 142; 16001 x 5120 148
  // and 114), not in the backward, whose sums then take too many registers (191 and 213, 189
  // and 309), nor where elements come one by one (20000 x 2049 forward 122 and 126, but
  // 20000 x 1563 136 and 87: a rule by the length has not been looked for)
  const int most8 = !bwd && s.vec > 1 ? 256 : 8 * 640;
  const int elems = a.H <= 256 || (a.H > 512 && a.H <= most8) ? 8 : 16;
  s.elems = elems;
  s.threads = ((a.H + elems - 1) / elems + 31) / 32 * 32;
  s.rows = s.threads == 32 ? kRingRows : 1;
  a.stages = std::min(kRingStages, kRingSmem / (s.rows * a.stage_bytes));
  s.persistent = a.stages >= 1;
  if (!s.persistent) return false;
  s.smem = static_cast<size_t>(s.rows) * a.stages * a.stage_bytes;
  if (bwd && s.rows > 1) s.smem = std::max(s.smem, static_cast<size_t>(s.rows) * a.H * sizeof(float));
  return true;
}

cudaError_t launch(const molt_norm_desc* d, const NormArgs& a, const NormShape& s, int* grid, bool bwd, cudaStream_t stream) {
  const int n_sm = device_sm_count();
  const bool r_f32 = d->residual_dtype == MOLT_FP32;
  if (d->dtype == MOLT_FP32) return launch_norm_fp32(a, s, n_sm, grid, bwd, stream);
  return d->dtype == MOLT_FP16 ? launch_norm_fp16(a, s, n_sm, grid, r_f32, bwd, stream)
                               : launch_norm_bf16(a, s, n_sm, grid, r_f32, bwd, stream);
}

}  // namespace
}  // namespace molt

using namespace molt;

extern "C" {

molt_status molt_residual_norm_fwd(const molt_norm_desc* desc, const void* x, const void* residual, const void* w_post,
                                   const void* gate, const void* w_pre, void* y, void* residual_out, float* rstd_post,
                                   float* rstd_pre, cudaStream_t stream) {
  if (const molt_status st = check_desc(desc); st != MOLT_OK) return st;
  if (desc->T == 0) return MOLT_OK;
  if (!x || (desc->gate_kind != MOLT_GATE_NONE && !gate)) return fail(MOLT_ERR_INVALID_ARG, "null pointer");
  if ((w_pre == nullptr) != (y == nullptr)) return fail(MOLT_ERR_INVALID_ARG, "w_pre and y come together");
  if (!y && !residual_out) return fail(MOLT_ERR_INVALID_ARG, "neither y nor residual_out is wanted");
  if (residual && residual == residual_out && desc->T > 1 && desc->residual_stride != 0 && desc->residual_stride != desc->H)
    return fail(MOLT_ERR_INVALID_ARG, "a residual is updated in place where its rows lie side by side");
  const int gate_type = desc->gate_kind == MOLT_GATE_TOKEN     ? MOLT_FP32
                        : desc->gate_kind == MOLT_GATE_CHANNEL ? desc->param_dtype
                                                               : desc->dtype;
  if (const molt_status st = check_elements({{x, desc->dtype},
                                             {residual, desc->residual_dtype},
                                             {w_post, desc->param_dtype},
                                             {gate, gate_type},
                                             {w_pre, desc->param_dtype},
                                             {y, desc->dtype},
                                             {residual_out, desc->residual_dtype},
                                             {rstd_post, MOLT_FP32},
                                             {rstd_pre, MOLT_FP32}});
      st != MOLT_OK)
    return st;
  NormArgs a = base_args(desc);
  a.x = x;
  a.r = residual;
  a.w_post = w_post;
  a.gate = gate;
  a.w_pre = w_pre;
  a.y = y;
  a.r_out = residual_out;
  a.rstd_post = rstd_post;
  a.rstd_pre = rstd_pre;
  molt_status st;
  a.err = device_status_word(&st);
  if (!a.err) return st;
  NormShape s = row_shape(a.H, vector_of(desc, a, {x, residual, w_post, w_pre, y, residual_out,
                                                 desc->gate_kind == MOLT_GATE_TOKEN ? nullptr : gate}));
  // rows that the SMs hold at once gain nothing from copies ahead
  const NormShape few = s;
  if ((s.vec != 8 || a.T > 16 * int64_t(device_sm_count())) && !rows_shape(desc, false, a, s)) s = few;
  int grid;
  if (const cudaError_t e = launch(desc, a, s, &grid, false, stream); e != cudaSuccess) return cuda_fail(e, "residual norm");
  note_launches(1);
  return MOLT_OK;
}

size_t molt_residual_norm_bwd_workspace_bytes(const molt_norm_desc* desc) {
  if (check_desc(desc) != MOLT_OK) return 0;
  return static_cast<size_t>(std::min<int64_t>(desc->T, max_blocks(device_sm_count()))) * 3 * desc->H * sizeof(float) + 256;
}

molt_status molt_residual_norm_bwd(const molt_norm_desc* desc, const void* dy, const void* dresidual, const void* x,
                                   const void* residual, const float* rstd_post, const float* rstd_pre, const void* w_post,
                                   const void* gate, const void* w_pre, void* dx, void* dresidual_out, float* dw_post,
                                   void* dgate, float* dw_pre, int accumulate, void* workspace, size_t workspace_bytes,
                                   cudaStream_t stream) {
  if (const molt_status st = check_desc(desc); st != MOLT_OK) return st;
  const bool channel = desc->gate_kind == MOLT_GATE_CHANNEL;
  if ((w_post && !dw_post) || (w_pre && !dw_pre) || (desc->gate_kind != MOLT_GATE_NONE && desc->T > 0 && !dgate) ||
      (channel && !dgate))
    return fail(MOLT_ERR_INVALID_ARG, "every weight and gate needs its gradient's buffer");
  if (desc->T > 0) {
    if (!x || !dx || (desc->gate_kind != MOLT_GATE_NONE && !gate)) return fail(MOLT_ERR_INVALID_ARG, "null pointer");
    if (w_pre && (!dy || !residual || !rstd_pre))
      return fail(MOLT_ERR_INVALID_ARG, "w_pre needs dy, the residual stream and rstd_pre");
    if (!w_pre && !dresidual) return fail(MOLT_ERR_INVALID_ARG, "without w_pre the gradient comes from dresidual");
    if (w_post && !rstd_post) return fail(MOLT_ERR_INVALID_ARG, "w_post needs rstd_post");
  }
  const int gate_type = desc->gate_kind == MOLT_GATE_TOKEN ? MOLT_FP32 : channel ? desc->param_dtype : desc->dtype;
  const int dgate_type = desc->gate_kind == MOLT_GATE_FULL ? desc->dtype : MOLT_FP32;
  if (const molt_status st = check_elements({{dy, desc->dtype},
                                             {dresidual, desc->residual_dtype},
                                             {x, desc->dtype},
                                             {residual, desc->residual_dtype},
                                             {rstd_post, MOLT_FP32},
                                             {rstd_pre, MOLT_FP32},
                                             {w_post, desc->param_dtype},
                                             {gate, gate_type},
                                             {w_pre, desc->param_dtype},
                                             {dx, desc->dtype},
                                             {dresidual_out, desc->residual_dtype},
                                             {dw_post, MOLT_FP32},
                                             {dgate, dgate_type},
                                             {dw_pre, MOLT_FP32}});
      st != MOLT_OK)
    return st;
  float* sums[3] = {w_post ? dw_post : nullptr, channel ? static_cast<float*>(dgate) : nullptr, w_pre ? dw_pre : nullptr};
  if (desc->T == 0) {
    for (float* o : sums)
      if (o && !accumulate)
        if (const cudaError_t e = cudaMemsetAsync(o, 0, static_cast<size_t>(desc->H) * sizeof(float), stream); e != cudaSuccess)
          return cuda_fail(e, "memset");
    return MOLT_OK;
  }
  Scratch sc;
  if (const molt_status st = get_scratch(sc, workspace, workspace_bytes, molt_residual_norm_bwd_workspace_bytes(desc), stream);
      st != MOLT_OK)
    return st;
  NormArgs a = base_args(desc);
  a.dy = dy;
  a.dr = dresidual;
  a.x = x;
  a.r = residual;
  a.rstd_post = const_cast<float*>(rstd_post);
  a.rstd_pre = const_cast<float*>(rstd_pre);
  a.w_post = w_post;
  a.gate = gate;
  a.w_pre = w_pre;
  a.dx = dx;
  a.dr_out = dresidual_out;
  a.dgate = dgate;
  a.part = static_cast<float*>(sc.aligned());
  molt_status st;
  a.err = device_status_word(&st);
  if (!a.err) return st;
  NormShape s =
      row_shape(a.H, vector_of(desc, a, {dy, dresidual, x, residual, w_post, w_pre, dx, dresidual_out,
                                       desc->gate_kind == MOLT_GATE_TOKEN ? nullptr : gate,
                                       desc->gate_kind == MOLT_GATE_FULL ? dgate : nullptr}));
  if (!rows_shape(desc, true, a, s)) s = NormShape{kNormMaxThreads, 1, 0, 1, false, 0};
  int grid;
  if (const cudaError_t e = launch(desc, a, s, &grid, true, stream); e != cudaSuccess)
    return cuda_fail(e, "residual norm backward");
  note_launches(1);
  if (!sums[0] && !sums[1] && !sums[2]) return MOLT_OK;
  norm_part_sum_kernel<<<dim3((a.H + kSumCols - 1) / kSumCols, 3), kSumCols * kSumWarps, 0, stream>>>(
      a.part, grid, a.H, sums[0], sums[1], sums[2], accumulate ? 1 : 0);
  if (const cudaError_t e = cudaGetLastError(); e != cudaSuccess) return cuda_fail(e, "residual norm weight gradients");
  note_launches(1);
  return MOLT_OK;
}

}  // extern "C"
