// C ABI of the gated feed-forward block (include/molt.h): argument checks, tensor maps,
// how the products of a call are cut into units, and the launches.
#include <algorithm>
#include <cstdint>
#include <cuda_runtime.h>
#include <initializer_list>

#include "ffn.cuh"
#include "molt_internal.cuh"
#include "vec.cuh"

namespace molt {
namespace {

constexpr int64_t kMaxRows = int64_t(1) << 24, kMaxCols = int64_t(1) << 17;
constexpr int64_t kUnitBytes = 256 * 256 * sizeof(float);   // a part
constexpr int kMinUnit = 4;                                 // K blocks

molt_status fail(molt_status s, const char* msg) {
  set_last_error(msg);
  return s;
}
molt_status cuda_fail(cudaError_t e, const char* what) {
  set_last_error(std::string(what) + ": " + cudaGetErrorString(e));
  return MOLT_ERR_CUDA;
}
#define FFN_TRY(call)                    \
  do {                                   \
    const molt_status s_ = (call);       \
    if (s_ != MOLT_OK) return s_;        \
  } while (0)

size_t up256(size_t n) { return (n + 255) & ~size_t(255); }
int64_t tiles(int64_t n, int64_t of) { return (n + of - 1) / of; }

molt_status check_desc(const molt_ffn_desc* d) {
  if (!d) return fail(MOLT_ERR_INVALID_ARG, "desc is NULL");
  if (d->T < 0 || d->H < 1 || d->F < 1) return fail(MOLT_ERR_INVALID_ARG, "sizes must satisfy T >= 0, H >= 1, F >= 1");
  if (d->dtype != MOLT_BF16 && d->dtype != MOLT_FP16) return fail(MOLT_ERR_INVALID_ARG, "the block is computed on bf16 or fp16");
  if (d->activation < MOLT_ACT_SILU || d->activation > MOLT_ACT_RELU) return fail(MOLT_ERR_INVALID_ARG, "unknown activation");
  if (d->T > kMaxRows || d->H > kMaxCols || d->F > kMaxCols)
    return fail(MOLT_ERR_UNSUPPORTED_SHAPE, "T must be at most 2^24, H and F at most 2^17");
  if (d->H % 8 != 0 || d->F % 8 != 0) return fail(MOLT_ERR_UNSUPPORTED_SHAPE, "H and F must be multiples of 8");
  const int64_t least[5] = {d->H, d->H, d->H, d->F, d->H};
  const int64_t ld[5] = {d->x_stride, d->w_gate_stride, d->w_up_stride, d->w_down_stride, d->dy_stride};
  for (int i = 0; i < 5; ++i) {
    if (ld[i] != 0 && ld[i] < least[i])
      return fail(MOLT_ERR_INVALID_ARG, "a row stride is 0 (rows side by side) or at least the row's length");
    if (ld[i] % 8 != 0 || ld[i] > (int64_t(1) << 31)) return fail(MOLT_ERR_UNSUPPORTED_SHAPE, "row strides must be multiples of 8, at most 2^31");
  }
  return MOLT_OK;
}

molt_status check16(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (reinterpret_cast<uintptr_t>(p) % 16 != 0) return fail(MOLT_ERR_INVALID_ARG, "pointers must be 16-byte aligned");
  return MOLT_OK;
}

// What there is of a product, for the planning: tiles and K blocks.
struct Shape {
  int64_t n_m, n_n, nk;
};
Shape glu_shape(const molt_ffn_desc* d) { return {tiles(d->T, 256), tiles(d->F, 128), tiles(d->H, kBK)}; }
Shape down_shape(const molt_ffn_desc* d) { return {tiles(d->T, 256), tiles(d->H, 256), tiles(d->F, kBK)}; }
Shape dh_shape(const molt_ffn_desc* d) { return {tiles(d->T, 256), tiles(d->F, 256), tiles(d->H, kBK)}; }
Shape dx_shape(const molt_ffn_desc* d) { return {tiles(d->T, 256), tiles(d->H, 256), 2 * tiles(d->F, kBK)}; }
Shape dw_shape(int64_t rows, int64_t cols, int64_t T) { return {tiles(rows, 256), tiles(cols, 256), tiles(T, kBK)}; }

// Most units that a launch with split products has.
int64_t max_units(int pairs) { return 4 * static_cast<int64_t>(pairs); }

// Bytes that parts may take, which do not fall as T grows: a workspace for the largest
// batch serves every smaller one.
size_t part_bytes(std::initializer_list<Shape> shapes, int pairs) {
  int64_t n = 0;
  for (const Shape& s : shapes) n += s.n_m * s.n_n * std::max<int64_t>(1, s.nk / kMinUnit);
  return static_cast<size_t>(std::min(n, max_units(pairs)) * kUnitBytes);
}

// Times in K blocks of a tile, of which one takes about 0.28 us: a unit's begin and end, what
// a further launch takes, and a megabyte of parts, written and read.  (A launch by its cost where it
// waits for the one before to end; begun ahead of that, four of them took 35 us for 41.)
constexpr double kPerUnit = 1.5, kPerLaunch = 10.0, kPerMb = 2.0 / 6.8 / 0.28;

// Units of at least kMinUnit K blocks; `splits` wanted, and got.
void cut(int nk, int wanted, int& splits, int& unit) {
  const int s = std::max(1, std::min(wanted, nk / kMinUnit));
  unit = (nk + s - 1) / s;
  splits = (nk + unit - 1) / unit;
}
double parts_cost(const FfnProblem& p, int64_t units) {
  // (rows past the last one are not stored)
  const double rows = std::min(256.0, static_cast<double>(p.m) / p.n_m);
  return kPerLaunch + kPerMb * static_cast<double>(units) * rows * 256 * 4 / 1e6;
}

// One product: as many tiles as fill the pairs whole times, and the others with their K cut so
// that they take less than a round (T = 64, H = 4096, F = 10944: 86 tiles on 76 pairs took 54 us
// in two rounds).
int plan_one(FfnProblem* p, int pairs) {
  const int tiles = p->n_m * p->n_n, head = tiles / pairs * pairs, tail = tiles - head, nk = p->nk;
  int splits = 1, unit = nk;
  double best = nk + kPerUnit;
  for (int s = 2; s <= 32 && tail > 0; ++s) {
    int got, k;
    cut(nk, s, got, k);
    const int64_t units = int64_t(tail) * got;
    if (got < s || units > max_units(pairs)) continue;
    const double cost = static_cast<double>((units + pairs - 1) / pairs) * (k + kPerUnit) + parts_cost(*p, units);
    if (cost < best) {
      best = cost;
      splits = got;
      unit = k;
    }
  }
  p->tile0 = 0;
  p->splits = 1;
  p->unit_k = nk;
  p->n_tiles = tiles;
  if (splits == 1) return 1;
  FfnProblem* t = p;
  if (head > 0) {
    p->n_tiles = head;
    t = p + 1;
    *t = *p;
  }
  t->tile0 = head;
  t->n_tiles = tail;
  t->splits = splits;
  t->unit_k = unit;
  return head > 0 ? 2 : 1;
}

// Several products: units of one length at most, of a few lengths the one for which the pairs'
// share and the longest unit that may come last take least.
void plan_several(FfnProblem* p, int n, int pairs) {
  int64_t work = 0;
  for (int i = 0; i < n; ++i) work += int64_t(p[i].n_m) * p[i].n_n * p[i].nk;
  const int64_t share = std::max<int64_t>(1, (work + pairs - 1) / pairs);
  double best = -1;
  int64_t best_len = 0;
  for (int div = 0; div <= 8; ++div) {
    const int64_t len = div == 0 ? int64_t(1) << 30 : std::max<int64_t>(kMinUnit, share / div);
    double sum = 0, extra = 0;
    int longest = 0;
    int64_t split_units = 0;
    for (int i = 0; i < n; ++i) {
      int splits, unit;
      cut(p[i].nk, static_cast<int>((p[i].nk + len - 1) / len), splits, unit);
      const int64_t units = int64_t(p[i].n_m) * p[i].n_n * splits;
      sum += static_cast<double>(units) * (unit + kPerUnit);
      longest = std::max(longest, unit);
      if (splits > 1) {
        split_units += units;
        extra += parts_cost(p[i], units);
      }
    }
    if (split_units > max_units(pairs)) continue;
    const double cost = std::max(sum / pairs + longest * (pairs - 1.0) / pairs / 2, longest + kPerUnit) + extra;
    if (best < 0 || cost < best) {
      best = cost;
      best_len = len;
    }
  }
  for (int i = 0; i < n; ++i) {
    cut(p[i].nk, static_cast<int>((p[i].nk + best_len - 1) / best_len), p[i].splits, p[i].unit_k);
    p[i].tile0 = 0;
    p[i].n_tiles = p[i].n_m * p[i].n_n;
  }
}

constexpr CUtensorMapDataType k16 = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;   // bits are copied: both 16-bit types
constexpr CUtensorMapDataType k32 = CU_TENSOR_MAP_DATA_TYPE_FLOAT32;

// a matrix as an operand: K-major boxes of 128 rows, MN-major ones of 64
molt_status operand(CUtensorMap* m, const void* p, int64_t rows, int64_t cols, int64_t ld, bool mn) {
  return encode_tmap_rows(m, k16, 2, p, rows, cols, ld, kBK, mn ? 64 : 128);
}
molt_status out16(CUtensorMap* m, const void* p, int64_t rows, int64_t cols) {
  return encode_tmap_rows(m, k16, 2, p, rows, cols, 0, 64, 32);
}
molt_status out32(CUtensorMap* m, const void* p, int64_t rows, int64_t cols) {
  return encode_tmap_rows(m, k32, 4, p, rows, cols, 0, 32, 32);
}

// One product of a call, its outputs as pointers until it is known whether K is cut.
struct Product {
  FfnProblem p{};
  void* out[3] = {};
  void sizes(int64_t m, int64_t n, const Shape& s) {
    p.m = static_cast<int>(m);
    p.n = static_cast<int>(n);
    p.n_m = static_cast<int>(s.n_m);
    p.n_n = static_cast<int>(s.n_n);
    p.nk0 = p.nk = static_cast<int>(s.nk);
  }
};

// Plans, launches and, where K is cut, sums the parts of up to four products.
molt_status run(Product* q, int n, int act, bool fp16, void* parts, size_t parts_bytes, unsigned* err, cudaStream_t s) {
  const int n_sm = device_sm_count(), pairs = ffn_pairs(n_sm);
  FfnBatch b{};
  b.act = act;
  b.err = err;
  const Product* of[kFfnProblems];
  if (n == 1) {
    b.p[0] = q[0].p;
    b.n = plan_one(b.p, pairs);
    of[0] = of[1] = q;
  } else {
    for (int i = 0; i < n; ++i) {
      b.p[i] = q[i].p;
      of[i] = &q[i];
    }
    b.n = n;
    plan_several(b.p, n, pairs);
  }
  size_t at = 0;
  int first = 0;
  for (int i = 0; i < b.n; ++i) {
    FfnProblem& p = b.p[i];
    p.first = first;
    first += p.n_tiles * p.splits;
    if (p.splits > 1) {
      const int64_t rows = int64_t(p.splits) * p.n_tiles * 256;
      if (at + rows * 1024 > parts_bytes) return fail(MOLT_ERR_WORKSPACE, "parts of a split product do not fit");
      p.epi = kEpiPart;
      FFN_TRY(out32(&p.out[0], static_cast<char*>(parts) + at, rows, 256));
      at += rows * 1024;
      continue;
    }
    const int outs = p.epi == kEpiDglu || (p.epi == kEpiGlu && p.keep) ? 3 : p.epi == kEpiGlu32 ? 2 : 1;
    for (int k = 0; k < outs; ++k)
      FFN_TRY(p.epi == kEpiStore32 || p.epi == kEpiGlu32 ? out32(&p.out[k], of[i]->out[k], p.m, p.n)
                                                         : out16(&p.out[k], of[i]->out[k], p.m, p.n));
  }
  b.total = first;
  if (const cudaError_t e = launch_ffn_gemm(b, fp16, n_sm, s); e != cudaSuccess) return cuda_fail(e, "feed-forward products");
  note_launches(1);
  at = 0;
  for (int i = 0; i < b.n; ++i) {
    const FfnProblem& p = b.p[i];
    if (p.splits == 1) continue;
    FfnReduce r{};
    r.part = reinterpret_cast<const float*>(static_cast<char*>(parts) + at);
    r.splits = p.splits;
    r.tile0 = p.tile0;
    r.n_tiles = p.n_tiles;
    r.n_m = p.n_m;
    r.n_n = p.n_n;
    r.m = p.m;
    r.n = p.n;
    r.epi = of[i]->p.epi;
    r.act = act;
    r.add = p.add;
    r.keep = p.keep;
    r.wide = p.wide;
    r.gate = p.gate;
    r.up = p.up;
    for (int k = 0; k < 3; ++k) r.out[k] = of[i]->out[k];
    if (const cudaError_t e = launch_ffn_reduce(r, fp16, s); e != cudaSuccess) return cuda_fail(e, "feed-forward parts");
    note_launches(1);
    at += static_cast<size_t>(p.splits) * p.n_tiles * kUnitBytes;
  }
  return MOLT_OK;
}

int64_t ld_or(int64_t ld, int64_t n) { return ld ? ld : n; }

// the first product: g and u
molt_status glu_product(Product& q, const molt_ffn_desc* d, const void* x, const void* w_gate, const void* w_up) {
  q.sizes(d->T, d->F, glu_shape(d));
  q.p.glu = 1;
  FFN_TRY(operand(&q.p.a[0], x, d->T, d->H, ld_or(d->x_stride, d->H), false));
  FFN_TRY(operand(&q.p.b[0], w_gate, d->F, d->H, ld_or(d->w_gate_stride, d->H), false));
  return operand(&q.p.b[1], w_up, d->F, d->H, ld_or(d->w_up_stride, d->H), false);
}

size_t hidden_bytes(const molt_ffn_desc* d) { return up256(static_cast<size_t>(d->T) * d->F * 2); }

size_t parts_fwd(const molt_ffn_desc* d, int pairs) {
  return std::max(part_bytes({glu_shape(d)}, pairs), part_bytes({down_shape(d)}, pairs));
}
size_t parts_bwd(const molt_ffn_desc* d, int pairs) {
  const Shape dwg = dw_shape(d->F, d->H, d->T), dwd = dw_shape(d->H, d->F, d->T);
  return std::max({part_bytes({glu_shape(d)}, pairs), part_bytes({dh_shape(d)}, pairs),
                   part_bytes({dx_shape(d), dwg, dwg, dwd}, pairs)});
}

}  // namespace
}  // namespace molt

using namespace molt;

extern "C" {

size_t molt_gated_ffn_fwd_workspace_bytes(const molt_ffn_desc* desc) {
  if (check_desc(desc) != MOLT_OK) return 0;
  return hidden_bytes(desc) + parts_fwd(desc, ffn_pairs(device_sm_count())) + 256;
}

molt_status molt_gated_ffn_fwd(const molt_ffn_desc* desc, const void* x, const void* w_gate, const void* w_up,
                               const void* w_down, void* y, void* gate_out, void* up_out, void* workspace,
                               size_t workspace_bytes, cudaStream_t stream) {
  FFN_TRY(check_desc(desc));
  if ((gate_out == nullptr) != (up_out == nullptr)) return fail(MOLT_ERR_INVALID_ARG, "gate_out and up_out come together");
  if (desc->T == 0) return MOLT_OK;
  if (!x || !w_gate || !w_up || !w_down || !y) return fail(MOLT_ERR_INVALID_ARG, "null pointer");
  FFN_TRY(check16({x, w_gate, w_up, w_down, y, gate_out, up_out}));
  if (const int64_t T = desc->T, H = desc->H, F = desc->F;
      !spans_apart({{y, T, H, 2}, {gate_out, T, F, 2}, {up_out, T, F, 2}},
                   {{x, T, H, 2, desc->x_stride}, {w_gate, F, H, 2, desc->w_gate_stride}, {w_up, F, H, 2, desc->w_up_stride},
                    {w_down, H, F, 2, desc->w_down_stride}}))
    return fail(MOLT_ERR_INVALID_ARG, "outputs may not share memory with one another or with inputs");
  Scratch sc;
  FFN_TRY(get_scratch(sc, workspace, workspace_bytes, molt_gated_ffn_fwd_workspace_bytes(desc), stream));
  molt_status st;
  unsigned* err = device_status_word(&st);
  if (!err) return st;
  const bool fp16 = desc->dtype == MOLT_FP16;
  char* h = static_cast<char*>(sc.aligned());
  if (desc->T <= kFfnFewRows) {
    FfnRows r{x, w_gate, w_up, ld_or(desc->x_stride, desc->H), ld_or(desc->w_gate_stride, desc->H),
              ld_or(desc->w_up_stride, desc->H), {h, gate_out, up_out}, static_cast<int>(desc->T), static_cast<int>(desc->F),
              static_cast<int>(desc->H), desc->activation};
    cudaError_t e = launch_ffn_rows(r, true, fp16, stream);
    if (e != cudaSuccess) return cuda_fail(e, "feed-forward rows");
    note_launches(1);
    r = FfnRows{h, w_down, nullptr, desc->F, ld_or(desc->w_down_stride, desc->F), 0, {y, nullptr, nullptr},
                static_cast<int>(desc->T), static_cast<int>(desc->H), static_cast<int>(desc->F), desc->activation};
    e = launch_ffn_rows(r, false, fp16, stream);
    if (e != cudaSuccess) return cuda_fail(e, "feed-forward rows");
    note_launches(1);
    return MOLT_OK;
  }
  void* parts = h + hidden_bytes(desc);
  const size_t parts_bytes = parts_fwd(desc, ffn_pairs(device_sm_count()));
  Product q;
  FFN_TRY(glu_product(q, desc, x, w_gate, w_up));
  q.p.epi = kEpiGlu;
  q.p.keep = gate_out != nullptr;
  q.out[0] = h;
  q.out[1] = gate_out;
  q.out[2] = up_out;
  FFN_TRY(run(&q, 1, desc->activation, fp16, parts, parts_bytes, err, stream));
  Product down;
  down.sizes(desc->T, desc->H, down_shape(desc));
  down.p.epi = kEpiStore16;
  down.out[0] = y;
  FFN_TRY(operand(&down.p.a[0], h, desc->T, desc->F, desc->F, false));
  FFN_TRY(operand(&down.p.b[0], w_down, desc->H, desc->F, ld_or(desc->w_down_stride, desc->F), false));
  return run(&down, 1, desc->activation, fp16, parts, parts_bytes, err, stream);
}

size_t molt_gated_ffn_bwd_workspace_bytes(const molt_ffn_desc* desc, int kept) {
  if (check_desc(desc) != MOLT_OK) return 0;
  return (kept ? 3 : 7) * hidden_bytes(desc) + parts_bwd(desc, ffn_pairs(device_sm_count())) + 256;
}

molt_status molt_gated_ffn_bwd(const molt_ffn_desc* desc, const void* dy, const void* x, const void* w_gate,
                               const void* w_up, const void* w_down, const void* gate, const void* up, void* dx,
                               void* dw_gate, void* dw_up, void* dw_down, int dw_dtype, int accumulate, void* workspace,
                               size_t workspace_bytes, cudaStream_t stream) {
  FFN_TRY(check_desc(desc));
  if ((gate == nullptr) != (up == nullptr)) return fail(MOLT_ERR_INVALID_ARG, "gate and up come together");
  if (dw_dtype != desc->dtype && dw_dtype != MOLT_FP32)
    return fail(MOLT_ERR_INVALID_ARG, "the weights' gradients are of the block's type or fp32");
  if (accumulate && dw_dtype != MOLT_FP32) return fail(MOLT_ERR_INVALID_ARG, "gradients are added in fp32 only");
  if (!dw_gate || !dw_up || !dw_down) return fail(MOLT_ERR_INVALID_ARG, "null pointer");
  FFN_TRY(check16({dw_gate, dw_up, dw_down}));
  const int64_t T = desc->T, H = desc->H, F = desc->F;
  const int db = dtype_bytes(dw_dtype);
  if (!spans_apart({{dx, T, H, 2}, {dw_gate, F, H, db}, {dw_up, F, H, db}, {dw_down, H, F, db}},
                   {{dy, T, H, 2, desc->dy_stride}, {x, T, H, 2, desc->x_stride}, {w_gate, F, H, 2, desc->w_gate_stride},
                    {w_up, F, H, 2, desc->w_up_stride}, {w_down, H, F, 2, desc->w_down_stride}, {gate, T, F, 2}, {up, T, F, 2}}))
    return fail(MOLT_ERR_INVALID_ARG, "outputs may not share memory with one another or with inputs");
  if (T == 0) {
    const size_t n = static_cast<size_t>(H) * F * dtype_bytes(dw_dtype);
    for (void* p : {dw_gate, dw_up, dw_down})
      if (!accumulate)
        if (const cudaError_t e = cudaMemsetAsync(p, 0, n, stream); e != cudaSuccess) return cuda_fail(e, "memset");
    return MOLT_OK;
  }
  if (!dy || !x || !w_gate || !w_up || !w_down || !dx) return fail(MOLT_ERR_INVALID_ARG, "null pointer");
  FFN_TRY(check16({dy, x, w_gate, w_up, w_down, gate, up, dx}));
  const bool kept = gate != nullptr;
  Scratch sc;
  FFN_TRY(get_scratch(sc, workspace, workspace_bytes, molt_gated_ffn_bwd_workspace_bytes(desc, kept), stream));
  molt_status st;
  unsigned* err = device_status_word(&st);
  if (!err) return st;
  const bool fp16 = desc->dtype == MOLT_FP16;
  const size_t hb = hidden_bytes(desc);
  char* w = static_cast<char*>(sc.aligned());
  void *dg = w, *du = w + hb, *h = w + 2 * hb;
  w += 3 * hb;
  if (!kept) w += 4 * hb;
  void* parts = w;
  const size_t parts_bytes = parts_bwd(desc, ffn_pairs(device_sm_count()));
  if (!kept) {
    // g and u again, in fp32: rounded they would add as much to the gradients as dg and du
    // themselves, and at T = 8192, H = 4096, F = 10944 half the bytes would save 0.1 ms of 4
    void* g32 = static_cast<char*>(sc.aligned()) + 3 * hb;
    void* u32 = static_cast<char*>(g32) + 2 * hb;
    Product q;
    FFN_TRY(glu_product(q, desc, x, w_gate, w_up));
    q.p.epi = kEpiGlu32;
    q.out[0] = g32;
    q.out[1] = u32;
    FFN_TRY(run(&q, 1, desc->activation, fp16, parts, parts_bytes, err, stream));
    gate = g32;
    up = u32;
  }
  Product q;
  q.sizes(T, F, dh_shape(desc));
  q.p.epi = kEpiDglu;
  q.p.gate = gate;
  q.p.up = up;
  q.p.wide = !kept;
  q.p.b_mn = 1;
  q.out[0] = dg;
  q.out[1] = du;
  q.out[2] = h;
  FFN_TRY(operand(&q.p.a[0], dy, T, H, ld_or(desc->dy_stride, H), false));
  FFN_TRY(operand(&q.p.b[0], w_down, H, F, ld_or(desc->w_down_stride, F), true));
  FFN_TRY(run(&q, 1, desc->activation, fp16, parts, parts_bytes, err, stream));

  Product g[4];
  g[0].sizes(T, H, dx_shape(desc));
  g[0].p.nk0 = g[0].p.nk / 2;
  g[0].p.epi = kEpiStore16;
  g[0].p.b_mn = 1;
  g[0].out[0] = dx;
  FFN_TRY(operand(&g[0].p.a[0], dg, T, F, F, false));
  FFN_TRY(operand(&g[0].p.a[1], du, T, F, F, false));
  FFN_TRY(operand(&g[0].p.b[0], w_gate, F, H, ld_or(desc->w_gate_stride, H), true));
  FFN_TRY(operand(&g[0].p.b[1], w_up, F, H, ld_or(desc->w_up_stride, H), true));
  for (int i = 1; i < 4; ++i) {
    const int64_t rows = i == 3 ? H : F, cols = i == 3 ? F : H;
    g[i].sizes(rows, cols, dw_shape(rows, cols, T));
    g[i].p.epi = dw_dtype == MOLT_FP32 ? kEpiStore32 : kEpiStore16;
    g[i].p.add = accumulate != 0;
    g[i].p.a_mn = g[i].p.b_mn = 1;
    g[i].out[0] = i == 1 ? dw_gate : i == 2 ? dw_up : dw_down;
    if (i == 3) {
      FFN_TRY(operand(&g[i].p.a[0], dy, T, H, ld_or(desc->dy_stride, H), true));
      FFN_TRY(operand(&g[i].p.b[0], h, T, F, F, true));
    } else {
      FFN_TRY(operand(&g[i].p.a[0], i == 1 ? dg : du, T, F, F, true));
      FFN_TRY(operand(&g[i].p.b[0], x, T, H, ld_or(desc->x_stride, H), true));
    }
  }
  return run(g, 4, desc->activation, fp16, parts, parts_bytes, err, stream);
}

}  // extern "C"
