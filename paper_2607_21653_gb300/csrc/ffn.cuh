// Gated feed-forward block: what the C-ABI layer (ffn.cu) hands to its kernels.
#pragma once

#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

namespace molt {

// activations (values of MOLT_ACT_*)
constexpr int kActSilu = 0, kActGelu = 1, kActRelu = 2;

// What becomes of a unit's accumulator.
enum FfnEpilogue : int {
  kEpiStore16 = 0,   // rounded, stored through out[0]
  kEpiStore32 = 1,   // stored through out[0] in fp32 (add: reduce-added to it)
  kEpiGlu = 2,       // gate | up columns: h = act(g) u through out[0]; keep: g, u through out[1], out[2]
  kEpiGlu32 = 3,     // g and u in fp32 through out[0], out[1]
  kEpiDglu = 4,      // dh: dg, du and h through out[0], out[1], out[2], from gate and up
  kEpiPart = 5       // fp32 part of a split K through out[0]
};

// One product C[m,n] = sum_k A[m,k] B[n,k] in tiles of 256 x 256 (kEpiGlu*: 256 rows by 128
// columns of g and the same of u).  K is a series of blocks of 64, the first nk0 from a[0]
// and b[0], the others from a[1] and b[1]; it is cut into `splits` units of unit_k blocks.  The
// tiles are numbered along columns, kFfnRaster rows of tiles at a time; a problem has n_tiles
// of them from tile0 on.
constexpr int kFfnRaster = 8;
struct FfnProblem {
  CUtensorMap a[2], b[2], out[3];
  const void* gate;     // kEpiDglu: [m, n], of the operands' type or fp32 (wide)
  const void* up;
  int m, n;
  int n_m, n_n;         // the product's tiles
  int tile0, n_tiles;
  int nk0, nk;
  int splits, unit_k;
  int first;            // the first of its units in the launch
  int a_mn, b_mn;       // operand is MN-major (its rows run along K)
  int epi;              // FfnEpilogue
  int glu;              // b[0] and b[1] are W_gate and W_up, brought by one CTA of the pair each
  int add;              // kEpiStore32
  int keep;             // kEpiGlu
  int wide;             // kEpiDglu: gate and up are fp32
};
constexpr int kFfnProblems = 5;   // four products, one of them in two parts
struct FfnBatch {
  FfnProblem p[kFfnProblems];
  int n;                // problems
  int total;            // units
  int act;
  unsigned* err;
};

// Sums of a split K: out = sum_s part[s], as the problem's epilogue.
struct FfnReduce {
  const float* part;    // [splits][n_tiles][256][256]
  int splits, tile0, n_tiles, n_m, n_n;
  int m, n;
  int epi;              // the unsplit problem's
  int act, add, keep, wide;
  const void* gate;
  const void* up;
  void* out[3];
};

// A product for a few rows: out[t, n] = x[t, k] w[n, k]^T; the first one of the block has w0 =
// Wg and w1 = Wu and gives h (out[0]) and, unless nullptr, g and u.  Up to 16 rows: the whole block at
// H = 4096, F = 10944 takes 46 us of one row, 48 of 8, 58 of 9 and 61 of 16, where the tiles' kernel has 68 of
// 17 and of 32; at H = 896, F = 2392 17 of 16 rows and 22 of 17 (past 16 the rows' loads fill the registers
// that the weights' should have).
constexpr int kFfnFewRows = 16;
struct FfnRows {
  const void *x, *w0, *w1;
  int64_t x_ld, w0_ld, w1_ld;
  void* out[3];
  int t, n, k;
  int act;
};
cudaError_t launch_ffn_rows(const FfnRows& r, bool glu, bool fp16, cudaStream_t s);

int ffn_pairs(int n_sm);   // CTA pairs of a launch
cudaError_t launch_ffn_gemm(const FfnBatch& b, bool fp16, int n_sm, cudaStream_t s);
cudaError_t launch_ffn_reduce(const FfnReduce& r, bool fp16, cudaStream_t s);

}  // namespace molt
