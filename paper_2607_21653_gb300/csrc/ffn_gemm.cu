// Products of the gated feed-forward block, forward and backward, with what follows
// them:
//   forward    g = x Wg^T, u = x Wu^T, h = act(g) u;   y = h Wd^T
//   backward   dh = dy Wd, dg = dh u act'(g), du = dh act(g), h again
//              dx = dg Wg + du Wu;   dWg = dg^T x, dWu = du^T x, dWd = dy^T h
//
// All of them are tiles of 256 x 256 on CTA pairs (tcgen05 cta_group::2), 64 of K at a
// time through five stages of shared memory, fp32 accumulators in TMEM, two of them so
// that a tile's epilogue runs under the next one's products.  What makes the block one
// kernel per direction's elementwise part is the choice of columns: a tile of the first
// product has 128 columns of g and the same 128 of u side by side, one CTA of the pair
// bringing W_gate's rows and the other W_up's, so that a thread of the epilogue finds g
// and u of one element in its own lane; and a tile of dh is turned into dg, du and h
// where it leaves TMEM.  g, u and dh are never in memory unless the caller keeps g and u.
//
// A launch takes up to four problems (dx and the three weight gradients are one), whose
// units are dealt to the pairs in order: dx, which has 2 F of K, then the gradients, which have T
// (up to T = 2 F the end is ragged by a short unit).  Where there are fewer tiles than pairs K is cut into
// units whose fp32 parts launch_ffn_reduce adds in order (no atomics: the same bits in
// every run).
//
// Between the products h, dg and du are rounded to the operands' type, which the tensor cores take two of: a
// second rounding of the size of the result's (errors against 64 bits 1.4 times those of one; h
// as two 16-bit parts would be a third more operations forward and twice as many backward).  In fp16 what
// passes 65504 there is infinite, as in a model whose layers are all in fp16.
//
// Bound by the tensor cores, in long calls at the power cap: bf16, H = 4096, F = 10944, 16384 rows
// forward with g and u kept 2.46 to 2.8 ms over boxes (1.72 PFLOP/s are 2.56); 4096 rows, the product of g and
// u with its epilogue at 1.81 PFLOP/s, dx and dW at 1.94, dh 1.40: there the epilogue reads g and u,
// as many bytes again as it writes, and the products wait for it.
//
// Roles per CTA (352 threads): warps 0 and 10 TMA producers of the A and the B
// operand, warp 1 MMA issuer (even CTA) and TMEM owner, warps 2-9 epilogue, two
// per TMEM lane quarter.  All waits are bounded (ptx.cuh).
#include <cstdint>
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <type_traits>

#include "ffn.cuh"
#include "ffn_act.cuh"
#include "molt_internal.cuh"
#include "ptx.cuh"
#include "vec.cuh"

namespace molt {
namespace {

constexpr int kStages = 5;
constexpr int kHalf = 128 * kBK * 2;              // one operand's half of a stage, 16 KB
constexpr int kStageBytes = 2 * kHalf;            // 32 KB per CTA
constexpr int kOffBox = kStages * kStageBytes;    // 160 KB
constexpr int kBoxBytes = 4096;                   // 32 rows x 128 bytes
constexpr int kBoxes = 2;                         // of an epilogue warp
constexpr int kEpiWarps = 8;
constexpr int kWarpB = 2 + kEpiWarps;
constexpr int kThreads = 32 * (kWarpB + 1);
constexpr int kSmemBytes = 1024 + kOffBox + kEpiWarps * kBoxes * kBoxBytes;

// row and column of a tile
__device__ __forceinline__ void tile_at(int tile, int n_m, int n_n, int& tm, int& tn) {
  const int per = kFfnRaster * n_n, group = tile / per, in = tile - group * per;
  const int rows = min(kFfnRaster, n_m - group * kFfnRaster);
  tn = in / rows;
  tm = group * kFfnRaster + in - tn * rows;
}

struct Unit {
  const FfnProblem* p;
  int tm, tn;
  int part;        // of a split K: its place among the parts
  int k0, nk;      // first K block, K blocks
  int mma_n;       // columns of the products: 256, or 128 where the last tile has no more
};

__device__ __forceinline__ Unit unit_at(const FfnBatch& b, int i) {
  int k = 0;
  while (k + 1 < b.n && i >= b.p[k + 1].first) ++k;
  const FfnProblem& p = b.p[k];
  Unit u;
  u.p = &p;
  i -= p.first;
  const int tile = i / p.splits, split = i - tile * p.splits;
  tile_at(p.tile0 + tile, p.n_m, p.n_n, u.tm, u.tn);
  u.part = split * p.n_tiles + tile;
  u.k0 = split * p.unit_k;
  u.nk = min(p.unit_k, p.nk - u.k0);
  const int left = p.glu ? 2 * (p.n - u.tn * 128) : p.n - u.tn * 256;
  u.mma_n = left > 128 ? 256 : 128;
  return u;
}

// The launches of a call may begin while the one before still ends; none touches memory before that
// one is done, and so all before it are (1031 rows, H = 896, F = 2392: 35 us forward for 41, 64 backward
// for 70; 16384 rows of H = 4096 2.52 ms for 2.58).
__device__ __forceinline__ void in_turn() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
}

template <class T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    ffn_gemm_kernel(const __grid_constant__ FfnBatch b) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[kStages];    // even CTA: both CTAs' bytes land here
  __shared__ __align__(8) uint64_t empty_bar[kStages];   // both CTAs
  __shared__ __align__(8) uint64_t accf_bar[2];          // both CTAs: accumulator full
  __shared__ __align__(8) uint64_t acce_bar[2];          // even CTA: one arrival per epilogue warp of the pair
  __shared__ __align__(8) uint64_t done_bar;
  __shared__ uint32_t tmem_base_sh;
  __shared__ int abort_sh;

  const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;
  volatile int* abort_flag = &abort_sh;
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&full_bar[s]), 1);
      mbar_init(smem_u32(&empty_bar[s]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&accf_bar[i]), 1);
      mbar_init(smem_u32(&acce_bar[i]), 2 * kEpiWarps);
    }
    mbar_init(smem_u32(&done_bar), 1);
    abort_sh = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(&tmem_base_sh), 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();   // every CTA's barriers exist before any remote arrival
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_sh;
  in_turn();

  if (warp == 0 || warp == kWarpB) {
    if (lane == 0) {
      const bool is_a = warp == 0;
      const uint32_t full_lead0 = mapa_shared(smem_u32(&full_bar[0]), 0);
      uint32_t st = 0, ph = 0, n_it = 0;
      bool ok = true;
      for (int i = pair; ok && i < b.total; i += pairs) {
        const Unit u = unit_at(b, i);
        const FfnProblem& p = *u.p;
        const bool mn = is_a ? p.a_mn : p.b_mn;
        // first row (column) of C that this CTA brings
        const int c0 = is_a       ? u.tm * 256 + static_cast<int>(rank) * 128
                       : p.glu    ? u.tn * 128
                                  : u.tn * 256 + static_cast<int>(rank) * (u.mma_n / 2);
        const CUtensorMap* maps = is_a ? p.a : p.b;
        for (int kb = u.k0; kb < u.k0 + u.nk; ++kb) {
          if (!(ok = mbar_wait(smem_u32(&empty_bar[st]), ph ^ 1u, abort_flag, b.err))) break;
          const uint32_t dst = smem0 + st * kStageBytes + (is_a ? 0 : kHalf), fb = full_lead0 + st * 8;
          if (leader && is_a) mbar_arrive_expect_tx(smem_u32(&full_bar[st]), 2 * kStageBytes);
          ++n_it;
          const bool second = kb >= p.nk0;
          const int k = (second ? kb - p.nk0 : kb) * kBK;
          const CUtensorMap* m = maps + (p.glu && !is_a ? rank : second ? 1u : 0u);
          if (mn) {
            tma_load_2d_pair(dst, m, fb, c0, k);
            tma_load_2d_pair(dst + kHalf / 2, m, fb, c0 + 64, k);
          } else {
            tma_load_2d_pair(dst, m, fb, k, c0);
          }
          if (++st == kStages) {
            st = 0;
            ph ^= 1u;
          }
        }
      }
      if (leader && is_a) {
        // every copy into both CTAs completes on these barriers: wait for the
        // last issued stages before the pair may exit
        const uint32_t first = n_it > (uint32_t)kStages ? n_it - kStages : 0u;
        for (uint32_t j = first; j < n_it; ++j)
          mbar_wait_drain(smem_u32(&full_bar[j % kStages]), (j / kStages) & 1u, b.err);
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && leader) {
      uint32_t st = 0, ph = 0, ai = 0;
      bool ok = true;
      for (int i = pair; ok && i < b.total; i += pairs) {
        const Unit u = unit_at(b, i);
        const bool a_mn = u.p->a_mn, b_mn = u.p->b_mn;
        constexpr uint32_t kBf16Formats = (1u << 7) | (1u << 10);
        const uint32_t idesc = idesc_bf16_f32(256, u.mma_n, a_mn, b_mn) &
                               (std::is_same<T, __half>::value ? ~kBf16Formats : ~0u);
        // K-major operands advance 32 bytes per K = 16, MN-major ones 16 rows of 128
        const uint32_t a_step = a_mn ? 128u : 2u, b_step = b_mn ? 128u : 2u;
        const uint64_t ad0 = sdesc_sw128(smem0, a_mn ? 8192u : 16u, 1024);
        const uint64_t bd0 = sdesc_sw128(smem0 + kHalf, b_mn ? 8192u : 16u, 1024);
        const uint32_t buf = ai & 1u;
        if (!(ok = mbar_wait(smem_u32(&acce_bar[buf]), ((ai >> 1) & 1u) ^ 1u, abort_flag, b.err))) break;
        tc_fence_after();
        const uint32_t d = tmem_base + buf * 256;
        auto issue = [&](uint32_t stage, uint32_t accumulate) {
          umma4_bf16_pair(d, ad0 + stage * (kStageBytes >> 4), bd0 + stage * (kStageBytes >> 4), a_step, b_step,
                          idesc, accumulate);
          umma_commit_pair_mc(smem_u32(&empty_bar[stage]), 3);
        };
        // two stages per turn, as in the LM head's backward
        for (int kb = 0; kb < u.nk; kb += 2) {
          const bool two = kb + 1 < u.nk;
          const uint32_t st0 = st;
          if (!(ok = mbar_wait(smem_u32(&full_bar[st]), ph, abort_flag, b.err))) break;
          if (++st == kStages) {
            st = 0;
            ph ^= 1u;
          }
          if (two && !(ok = mbar_wait(smem_u32(&full_bar[st]), ph, abort_flag, b.err))) break;
          tc_fence_after();
          issue(st0, kb != 0 ? 1u : 0u);
          if (two) {
            issue(st, 1u);
            if (++st == kStages) {
              st = 0;
              ph ^= 1u;
            }
          }
        }
        if (!ok) break;
        umma_commit_pair_mc(smem_u32(&accf_bar[buf]), 3);
        ++ai;
      }
      umma_commit_pair_mc(smem_u32(&done_bar), 1);
      mbar_wait_drain(smem_u32(&done_bar), 0, b.err);
    }
  } else {
    const int q = warp & 3;
    const int hf = (warp - 2) >> 2;
    const uint32_t lane_off = static_cast<uint32_t>(q * 32) << 16;
    const uint32_t box0 = smem0 + kOffBox + (warp - 2) * kBoxes * kBoxBytes, box1 = box0 + kBoxBytes;
    const uint32_t acce_lead0 = mapa_shared(smem_u32(&acce_bar[0]), 0);
    const T* tag = nullptr;
    uint32_t ai = 0;   // accumulators read
    // until this warp's boxes have been read out
    auto boxes_free = [&]() {
      if (lane == 0) bulk_wait_group_read<0>();
      __syncwarp();
    };
    // eight values, 16 bytes, of the lane's row: the 128-byte swizzle
    auto put = [&](uint32_t box, int i, uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3) {
      st_shared_v4(box + lane * 128 + static_cast<uint32_t>(i ^ (lane & 7)) * 16, w0, w1, w2, w3);
    };
    for (int i = pair; i < b.total; i += pairs) {
      const Unit u = unit_at(b, i);
      const FfnProblem& p = *u.p;
      const uint32_t buf = ai & 1u;
      const int r0 = u.tm * 256 + static_cast<int>(rank) * 128 + q * 32;   // this warp's first row of C
      const bool rows_in = r0 < p.m;
      // kEpiDglu: g and u of 64 columns (fp32: 32) of the lane's row, as they are in memory.  The
      // first ones come while the products run, the others while boxes go out, but not ahead
      // of a fence, which would wait for them.  Not as read-only data: the launch before, which may
      // have written them, can end after this one has begun
      const int row = r0 + lane, col0 = u.tn * 256 + hf * 128;
      uint4 gq[8], uq[8];
      auto load_gu = [&](int c) {   // c: in 32 columns
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int f = col0 + c * 32 + j * (p.wide ? 4 : 8);
          if (row < p.m && f < p.n) {
            const int64_t at = (static_cast<int64_t>(row) * p.n + f) * (p.wide ? 4 : 2);
            gq[j] = __ldcg(reinterpret_cast<const uint4*>(static_cast<const char*>(p.gate) + at));
            uq[j] = __ldcg(reinterpret_cast<const uint4*>(static_cast<const char*>(p.up) + at));
          } else {
            gq[j] = uq[j] = make_uint4(0, 0, 0, 0);
          }
        }
      };
      if (p.epi == kEpiDglu && col0 < p.n) load_gu(0);
      if (!mbar_wait(smem_u32(&accf_bar[buf]), (ai >> 1) & 1u, abort_flag, b.err)) break;
      tc_fence_after();
      const uint32_t acc = tmem_base + lane_off + buf * 256;
      // accumulator read out: one arrival per warp hands it back
      auto release_acc = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_relaxed(acce_lead0 + buf * 8);
      };
      // a box of 32 rows stored (or added) at column col
      auto store_box = [&](const CUtensorMap* m, uint32_t box, int col, int row, bool add) {
        if (lane == 0 && rows_in) {
          if (add)
            tma_reduce_add_2d(m, box, col, row);
          else
            tma_store_2d(m, box, col, row);
        }
        if (lane == 0) bulk_commit_group();
      };
      auto stored = [&]() {   // the boxes' generic writes before the copies that read them
        fence_proxy_async_smem();
        __syncwarp();
      };
      if (p.epi == kEpiStore32 || p.epi == kEpiPart || p.epi == kEpiGlu32) {
        // 32 fp32 columns to a box.  Parts: whole tiles, one below the other
        const bool part = p.epi == kEpiPart;
        const int wide = part ? 256 : p.glu ? u.mma_n : min(256, p.n - u.tn * 256);
#pragma unroll 1
        for (int s = 0; s < 4; ++s) {
          const int col = hf * 128 + s * 32;
          if (col >= wide || col >= u.mma_n) break;
          float v[32];
          tmem_ld32(acc + col, v);
          const uint32_t box = s & 1 ? box1 : box0;
          if (!(s & 1)) boxes_free();
#pragma unroll
          for (int j = 0; j < 8; ++j)
            put(box, j, __float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]), __float_as_uint(v[4 * j + 2]),
                __float_as_uint(v[4 * j + 3]));
          stored();
          if (part) {
            store_box(&p.out[0], box, col, u.part * 256 + static_cast<int>(rank) * 128 + q * 32, false);
          } else if (p.glu) {
            const int half = u.mma_n / 2, c = col < half ? col : col - half;
            if (u.tn * 128 + c < p.n) store_box(&p.out[col < half ? 0 : 1], box, u.tn * 128 + c, r0, false);
          } else {
            store_box(&p.out[0], box, u.tn * 256 + col, r0, p.add != 0);
          }
        }
        release_acc();
      } else if (p.epi == kEpiStore16) {
        const int wide = min(256, p.n - u.tn * 256);
#pragma unroll 1
        for (int s = 0; s < 2; ++s) {
          const int col = hf * 128 + s * 64;
          if (col >= wide) break;
          const uint32_t box = s ? box1 : box0;
          if (s == 0) boxes_free();
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float v[32];
            tmem_ld32(acc + col + h * 32, v);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              put(box, h * 4 + j, pack2(v[8 * j], v[8 * j + 1], tag), pack2(v[8 * j + 2], v[8 * j + 3], tag),
                  pack2(v[8 * j + 4], v[8 * j + 5], tag), pack2(v[8 * j + 6], v[8 * j + 7], tag));
          }
          stored();
          store_box(&p.out[0], box, u.tn * 256 + col, r0, false);
        }
        release_acc();
      } else if (p.epi == kEpiGlu) {
        const int half = u.mma_n / 2;             // columns of g, then as many of u
        const int c0 = hf * 64, f0 = u.tn * 128 + c0;
        if (c0 < half && f0 < p.n) {
          boxes_free();
#pragma unroll 1
          for (int h = 0; h < 2; ++h) {
            float g[32], up[32], unused;
            tmem_ld32(acc + c0 + h * 32, g);
            tmem_ld32(acc + half + c0 + h * 32, up);
            with_activation(b.act, [&](auto act) {
#pragma unroll
              for (int j = 0; j < 32; ++j) up[j] *= ffn_activate<decltype(act)::value, false>(g[j], unused);
            });
#pragma unroll
            for (int j = 0; j < 4; ++j)
              put(box0, h * 4 + j, pack2(up[8 * j], up[8 * j + 1], tag), pack2(up[8 * j + 2], up[8 * j + 3], tag),
                  pack2(up[8 * j + 4], up[8 * j + 5], tag), pack2(up[8 * j + 6], up[8 * j + 7], tag));
          }
          stored();
          store_box(&p.out[0], box0, f0, r0, false);
          if (p.keep) {
#pragma unroll 1
            for (int o = 0; o < 2; ++o) {
              const uint32_t box = o == 0 ? box1 : box0;
              if (o == 1) boxes_free();
#pragma unroll 1
              for (int h = 0; h < 2; ++h) {
                float v[32];
                tmem_ld32(acc + o * half + c0 + h * 32, v);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  put(box, h * 4 + j, pack2(v[8 * j], v[8 * j + 1], tag), pack2(v[8 * j + 2], v[8 * j + 3], tag),
                      pack2(v[8 * j + 4], v[8 * j + 5], tag), pack2(v[8 * j + 6], v[8 * j + 7], tag));
              }
              stored();
              store_box(&p.out[1 + o], box, f0, r0, false);
            }
          }
        }
        release_acc();
      } else {   // kEpiDglu
#pragma unroll 1
        for (int s = 0; s < 2; ++s) {
          const int col = hf * 128 + s * 64, f0 = u.tn * 256 + col;
          if (f0 >= p.n) break;
          uint32_t hw[32];
          boxes_free();
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float dh[32];
            tmem_ld32(acc + col + h * 32, dh);
            uint32_t dg[16], du[16];
            auto gradients = [&](auto act, auto wide) {
#pragma unroll
              for (int e = 0; e < 32; e += 2) {
                float g0, g1, u0, u1;
                if constexpr (decltype(wide)::value) {
                  const uint4 a = gq[e / 4], c = uq[e / 4];
                  g0 = __uint_as_float(e & 2 ? a.z : a.x), g1 = __uint_as_float(e & 2 ? a.w : a.y);
                  u0 = __uint_as_float(e & 2 ? c.z : c.x), u1 = __uint_as_float(e & 2 ? c.w : c.y);
                } else {
                  const uint4 a = gq[h * 4 + e / 8], c = uq[h * 4 + e / 8];
                  const int k = e / 2 % 4;
                  unpack2(k == 0 ? a.x : k == 1 ? a.y : k == 2 ? a.z : a.w, tag, g0, g1);
                  unpack2(k == 0 ? c.x : k == 1 ? c.y : k == 2 ? c.z : c.w, tag, u0, u1);
                }
                float d0, d1;
                const float a0 = ffn_activate<decltype(act)::value, true>(g0, d0);
                const float a1 = ffn_activate<decltype(act)::value, true>(g1, d1);
                dg[e / 2] = pack2(dh[e] * u0 * d0, dh[e + 1] * u1 * d1, tag);
                du[e / 2] = pack2(dh[e] * a0, dh[e + 1] * a1, tag);
                hw[h * 16 + e / 2] = pack2(a0 * u0, a1 * u1, tag);
              }
            };
            with_activation(b.act, [&](auto act) {
              if (p.wide)
                gradients(act, std::true_type{});
              else
                gradients(act, std::false_type{});
            });
            if (p.wide && h == 0) load_gu(s * 2 + 1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              put(box0, h * 4 + j, dg[4 * j], dg[4 * j + 1], dg[4 * j + 2], dg[4 * j + 3]);
              put(box1, h * 4 + j, du[4 * j], du[4 * j + 1], du[4 * j + 2], du[4 * j + 3]);
            }
          }
          if (s == 1 || f0 + 64 >= p.n) release_acc();
          stored();
          store_box(&p.out[0], box0, f0, r0, false);
          store_box(&p.out[1], box1, f0, r0, false);
          if (s == 0 && f0 + 64 < p.n) load_gu(2);
          boxes_free();
#pragma unroll
          for (int j = 0; j < 8; ++j) put(box0, j, hw[4 * j], hw[4 * j + 1], hw[4 * j + 2], hw[4 * j + 3]);
          stored();
          store_box(&p.out[2], box0, f0, r0, false);
        }
        if (u.tn * 256 + hf * 128 >= p.n) release_acc();   // no columns for this warp
      }
      ++ai;
    }
    if (lane == 0) bulk_wait_group<0>();
    __syncwarp();
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync_all();   // no CTA leaves while the other may still touch its memory
  tc_fence_after();
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc_pair(tmem_base, 512);
  }
}

// Sums of the parts of a split K, in order: kReduceRows rows of a tile to a block, four columns
// to a thread, eight parts' loads at a time.
constexpr int kReduceRows = 4;
template <class T>
__global__ void __launch_bounds__(256) ffn_reduce_kernel(const FfnReduce r) {
  constexpr int kBlocks = 256 / kReduceRows;
  in_turn();
  const int tile = blockIdx.x / kBlocks;
  int tm, tn;
  tile_at(r.tile0 + tile, r.n_m, r.n_n, tm, tn);
  const bool glu = r.epi == kEpiGlu || r.epi == kEpiGlu32;
  // the columns of g and u in a tile of parts: 128 each, 64 in a last tile of no more
  const int wide = glu ? 128 : 256, quads = wide / 4;
  const int half = glu && r.n - tn * 128 <= 64 ? 64 : 128;
  const int64_t split_stride = static_cast<int64_t>(r.n_tiles) * 65536;
  for (int i = threadIdx.x; i < kReduceRows * quads; i += 256) {
    const int y = (blockIdx.x % kBlocks) * kReduceRows + i / quads, x = i % quads * 4;
    const int row = tm * 256 + y, c = tn * wide + x;
    if (row >= r.m || c >= r.n) continue;
    const int64_t at = static_cast<int64_t>(row) * r.n + c;
    const float* p = r.part + (static_cast<int64_t>(tile) * 256 + y) * 256 + x;
    auto sum = [&](int off, float (&v)[4]) {
      load_vec<4>(p + off, v);
      for (int s0 = 1; s0 < r.splits; s0 += 8) {
        float w[8][4];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (s0 + i < r.splits) load_vec<4>(p + off + (s0 + i) * split_stride, w[i]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (s0 + i < r.splits) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += w[i][e];
          }
        }
      }
    };
    float v[4];
    sum(0, v);
    auto put = [&](int o, const float (&x)[4]) { store_vec<4>(static_cast<T*>(r.out[o]) + at, x); };
    if (r.epi == kEpiStore16) {
      put(0, v);
    } else if (r.epi == kEpiStore32) {
      float* o = static_cast<float*>(r.out[0]) + at;
      if (r.add) {
        float w[4];
        load_vec<4>(o, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += w[e];
      }
      store_vec<4>(o, v);
    } else if (glu) {
      float up[4], h[4], unused;
      sum(half, up);
      if (r.epi == kEpiGlu32) {
        store_vec<4>(static_cast<float*>(r.out[0]) + at, v);
        store_vec<4>(static_cast<float*>(r.out[1]) + at, up);
        continue;
      }
      with_activation(r.act, [&](auto act) {
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = ffn_activate<decltype(act)::value, false>(v[e], unused) * up[e];
      });
      put(0, h);
      if (r.keep) {
        put(1, v);
        put(2, up);
      }
    } else {   // kEpiDglu
      float g[4], up[4], dg[4], du[4], h[4];
      if (r.wide) {
        load_vec<4>(static_cast<const float*>(r.gate) + at, g);
        load_vec<4>(static_cast<const float*>(r.up) + at, up);
      } else {
        load_vec<4>(static_cast<const T*>(r.gate) + at, g);
        load_vec<4>(static_cast<const T*>(r.up) + at, up);
      }
      with_activation(r.act, [&](auto act) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float d;
          const float a = ffn_activate<decltype(act)::value, true>(g[e], d);
          dg[e] = v[e] * up[e] * d;
          du[e] = v[e] * a;
          h[e] = a * up[e];
        }
      });
      put(0, dg);
      put(1, du);
      put(2, h);
    }
  }
}

}  // namespace

int ffn_pairs(int n_sm) { return n_sm / 2 > 0 ? n_sm / 2 : 1; }

template <class Arg>
static cudaError_t launch_early(void (*k)(const Arg), int grid, int threads, int smem, cudaStream_t s, const Arg& arg) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = static_cast<size_t>(smem);
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k, arg);
}

cudaError_t launch_ffn_gemm(const FfnBatch& b, bool fp16, int n_sm, cudaStream_t s) {
  const auto k = fp16 ? &ffn_gemm_kernel<__half> : &ffn_gemm_kernel<__nv_bfloat16>;
  const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
  if (e != cudaSuccess) return e;
  const int pairs = b.total < ffn_pairs(n_sm) ? b.total : ffn_pairs(n_sm);
  return launch_early(k, 2 * pairs, kThreads, kSmemBytes, s, b);
}

cudaError_t launch_ffn_reduce(const FfnReduce& r, bool fp16, cudaStream_t s) {
  const int grid = r.n_tiles * (256 / kReduceRows);
  return launch_early(fp16 ? &ffn_reduce_kernel<__half> : &ffn_reduce_kernel<__nv_bfloat16>, grid, 256, 0, s, r);
}

}  // namespace molt
