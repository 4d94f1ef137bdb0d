// Cross entropy against a vocabulary and its gradient on the tensor cores, in bf16 and in fp32.
//
// One matrix product with four operand layouts and ends (C is never the logits):
//   statistics   hidden W^T, per token and tile of 256 words the maximum and the sum of
//                exponentials (and the target's logit); a small kernel joins them
//   gradient     hidden W^T again, and g = (exp(logit - lse) - [word = target]) dloss,
//                rounded to bf16 for the products that follow, for one piece of the words
//   dhidden      g W, added up over the pieces in fp32
//   dweight      g^T hidden
// In fp32 every operand x is the sum of three bf16 numbers, x0 = bf16(x), x1 = bf16(x - x0), x2 =
// bf16(x - x0 - x1), which hold its 24 bits; a product is the sum of the six products of parts
// whose indices add up to at most 2 (what is left out is below 2^-24 of the whole), the smallest
// first, in the same fp32 accumulator. Six passes over K at the tensor cores' rate are about four
// times as fast as fp32 multiply-adds.
// 8 N H V operations for a forward and a backward pass, of which 6 are the least
// possible: the logits of N tokens and V words in fp32 would be kept otherwise.
//
// A pair of CTAs (one cluster) computes 256 x 256 of C, each CTA 128 rows of it:
// tcgen05.mma with cta_group::2, M = N = 256, K = 16, issued by the even CTA, both
// operands split between the two CTAs' shared memory, so that an SM loads 32 KB per 64
// columns of K where one CTA alone would load 48 KB for its 128 x 256 (the SMs' share of
// L2 bandwidth is about what the former needs). Warps are specialised: warp 8 loads
// tiles by TMA into a ring of six, warp 9 issues the products, warps 0-7 (half a row of C
// per thread) work on the result of one tile while the next is computed: two
// accumulators of 256 columns fill the tensor memory. Clusters walk over the tiles with a
// fixed stride, down groups of rows, so that both operands of the tiles in flight are in L2.
//
// The tensor cores' accumulator drops the bits below its last one at every step of 16 terms, which
// shrinks a sum by about 2^-25 per step: over 4096 terms log-sums came out 1.3e-6 too small, where
// rounded fp32 sums are 4e-8 off. Where the result is fp32 the row warps therefore take the
// sums out of tensor memory every 1024 terms (256 in fp32 products) and add them up rounded;
// what is rounded to bf16 afterwards is left in one accumulator.
//
// Bound by the tensor cores where tokens are many: 8192 x 4096 x 32000 forward 1.02 ms, 2.1 PFLOP/s, backward
// 3.32 ms, 1.94 PFLOP/s of its three products; 6001 x 8192 x 32003 1.75 and 5.35 ms. By the weights'
// bytes where they are few: 256 x 4096 x 32000 59 us for the statistics (262 MB, 4.5 TB/s), 51, 62 and 89
// for gradient, dhidden and dweight. fp32: 137 TFLOP/s of the product it stands for, 25 with fp32 multiply-adds.
// Results leave through a stage in shared memory: with a row per lane, 16 bytes each, dweight took 139 us
// of the latter and 8192 tokens 4.46 ms instead of 4.34.
#include <math.h>

#include "dmc_retrofit.cuh"
#include "dmc_tensor.cuh"

namespace dmc {

namespace {

constexpr int kM = 256;        // rows of C per cluster
constexpr int kK = 64;         // columns of a step
constexpr int kStages = 6;
constexpr int kHalf = 128 * kK * 2;  // bytes of a CTA's half of an operand's tile (of B at most)
constexpr int kProductThreads = 320;
constexpr int kStageRow = 80;  // bytes of a row of a result's stage: 64 and 16 of padding

struct ProductShared {
  unsigned char a[kStages][kHalf], b[kStages][kHalf];
  unsigned char stage[8][32 * kStageRow];
  uint64_t full[kStages], empty[kStages];
  uint64_t done[2], taken[2];  // an accumulator is complete; its rows have been read (both CTAs)
  uint32_t tmem;
  int abort;
};
constexpr int kProductSmem = sizeof(ProductShared) + 1024;
static_assert(kProductSmem <= 227 * 1024, "one CTA's shared memory");

enum class End { kStats, kGrad, kHidden, kWeight };

struct ProductArgs {
  LossArgs a;
  int rows, cols, depth;  // C is rows x cols, depth its sums' terms
  int passes;             // over depth: products of the operands' parts
  int group;              // row tiles of a group
  int v0;                 // first word of the piece
  bool first, last;       // of the pieces
  int shares;             // of a gradient's sums, see sum_shares
  CUtensorMap ma, mb;
};

// ---------------------------------------------------------------- cluster PTX

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
  return r;
}
// the address of the even CTA's copy of a shared variable
__device__ __forceinline__ uint32_t in_leader(uint32_t addr) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// TMA load into this CTA's shared memory that completes on a barrier of the cluster
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int part) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4, "
      "%5}], [%2];" ::"r"(dst),
      "l"(map), "r"(bar), "r"(x), "r"(y), "r"(part)
      : "memory");
}
// the operands' parts in pass i of six (of one: parts 0): (2, 0), (0, 2), (1, 1), (1, 0), (0, 1), (0, 0)
__device__ __forceinline__ int part_a(int passes, int i) { return passes == 1 ? 0 : (0x201100 >> (4 * (5 - i))) & 15; }
__device__ __forceinline__ int part_b(int passes, int i) { return passes == 1 ? 0 : (0x021010 >> (4 * (5 - i))) & 15; }
__device__ __forceinline__ void mma_pair(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, bool acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a), "l"(b), "r"(idesc), "r"(acc ? 1 : 0)
      : "memory");
}
// the products issued so far complete: arrives at the barrier of both CTAs
__device__ __forceinline__ void commit_pair(uint32_t bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
      "h"((uint16_t)3)
      : "memory");
}

struct Tile {
  int m, n;  // first row and column of C
};
template <int kN>
__device__ __forceinline__ Tile tile_of(const ProductArgs& p, int u) {
  const int tm = (p.rows + kM - 1) / kM, tn = (p.cols + kN - 1) / kN;
  const int per = p.group * tn, g = u / per, r = u % per;
  const int in = min(p.group, tm - g * p.group);
  Tile t;
  t.m = (g * p.group + r % in) * kM;
  t.n = r / in * kN;
  return t;
}

constexpr float kLog2e = 1.4426950408889634f;

template <End kEnd, bool kF32, int kN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kProductThreads, 1)
loss_product_kernel(const __grid_constant__ ProductArgs p) {
  constexpr int kHalfN = kN / 2;          // columns of a row thread
  constexpr int kHalfB = kHalf * kN / 256;  // bytes of a CTA's half of B's tile
  constexpr int kFinish = kF32 ? 16 : 32;   // columns that go to memory at a time
  constexpr bool kOften = kF32 || kEnd == End::kStats;  // sums leave tensor memory every few steps, see above
  // operands whose rows run along the sums' terms are MN-major
  constexpr bool kAmn = kEnd == End::kWeight, kBmn = kEnd == End::kHidden || kEnd == End::kWeight;
  extern __shared__ unsigned char smem_raw[];
  ProductShared& sh = *reinterpret_cast<ProductShared*>(smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
  const LossArgs& a = p.a;
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const uint32_t rank = cluster_rank();
  const int clusters = gridDim.x / 2, cluster = blockIdx.x / 2;
  const int tiles = ((p.rows + kM - 1) / kM) * ((p.cols + kN - 1) / kN);
  constexpr bool kShares = kEnd == End::kHidden || kEnd == End::kWeight;
  const int shares = kShares ? p.shares : 1, units = tiles * shares;  // work: a share of a tile's sums
  const int depth = (p.depth + kK - 1) / kK;                          // steps of a pass
  // the steps of a pass that are unit u's
  auto first_step = [&](int u) -> int { return kShares ? (int)((long long)depth * (u / tiles) / shares) : 0; };
  auto last_step = [&](int u) -> int { return kShares ? (int)((long long)depth * (u / tiles + 1) / shares) : depth; };
  // one past the last step that goes into the accumulator begun at step k of a unit's steps (of fp32's
  // passes the last one alone has large terms)
  auto chunk_end = [&](int steps, int k) -> int {
    const int all = steps * p.passes;
    if (kF32) return k < 5 * steps ? 5 * steps : min(all, k + 4);
    return kOften ? min(all, k + 16) : all;
  };
  volatile int* s_abort = &sh.abort;
  auto wait = [&](uint64_t* bar, uint32_t ph) -> bool { return warp_wait(smem_u32(bar), ph, s_abort, a.error); };

  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(smem_u32(&sh.full[i]), 1);
      mbar_init(smem_u32(&sh.empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sh.done[i]), 1);
      mbar_init(smem_u32(&sh.taken[i]), 16);  // the eight row warps of both CTAs
    }
    fence_mbar_init();
    sh.abort = 0;
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(512));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // both CTAs' barriers stand before either signals the other's
  tc_fence_after();
  const uint32_t tmem = tc_uniform(sh.tmem);

  if (warp == 8) {
    // ---------------------------------------------------------------- loads
    uint32_t n = 0;
    bool ok = true;
    for (int u = cluster; u < units && ok; u += clusters) {
      const Tile t = tile_of<kN>(p, kShares ? u % tiles : u);
      const int m = t.m + (int)rank * 128, c = t.n + (int)rank * kHalfN;  // this CTA's half
      const int begin = first_step(u), end = last_step(u);
      int k = begin, pass = 0, pa = part_a(p.passes, 0), pb = part_b(p.passes, 0);
#pragma unroll 1
      for (int x = 0; x < (end - begin) * p.passes; ++x, ++n) {
        const int s = n % kStages;
        ok = wait(&sh.empty[s], ((n / kStages) & 1) ^ 1);
        if (!ok) break;
        if (tc_elect()) {
          if (rank == 0) mbar_arrive_expect_tx(smem_u32(&sh.full[s]), 2 * (kHalf + kHalfB));
          const uint32_t bar = in_leader(smem_u32(&sh.full[s]));
          const uint32_t da = smem_u32(sh.a[s]), db = smem_u32(sh.b[s]);
          if (kAmn) {
            tma_load_pair(da, &p.ma, bar, m, k * kK, pa);
            tma_load_pair(da + kHalf / 2, &p.ma, bar, m + 64, k * kK, pa);
          } else {
            tma_load_pair(da, &p.ma, bar, k * kK, m, pa);
          }
          if (kBmn) {
            tma_load_pair(db, &p.mb, bar, c, k * kK, pb);
            if (kN == 256) tma_load_pair(db + kHalfB / 2, &p.mb, bar, c + 64, k * kK, pb);
          } else {
            tma_load_pair(db, &p.mb, bar, k * kK, c, pb);
          }
        }
        __syncwarp();
        if (++k == end) {
          k = begin;
          ++pass;
          pa = part_a(p.passes, pass);
          pb = part_b(p.passes, pass);
        }
      }
    }
    // the last tiles have been read (so every copy has landed, and every signal has come)
    for (uint32_t i = n > kStages ? n - kStages : 0; i < n; ++i)
      mbar_wait(smem_u32(&sh.empty[i % kStages]), (i / kStages) & 1, a.error);
  } else if (warp == 9) {
    // ---------------------------------------------------------------- products
    if (rank == 0) {
      constexpr uint32_t idesc = tc_idesc(kM, kN, kAmn, kBmn);
      // K-major: rows of 128 bytes, eight of them every 1024; MN-major: 64 elements of a
      // row per 128 bytes, the next 64 half a tile on
      const uint64_t da = tc_desc(smem_u32(sh.a[0]), kAmn ? kHalf / 2 : 16, 1024);
      const uint64_t db = tc_desc(smem_u32(sh.b[0]), kBmn ? kHalfB / 2 : 16, 1024);
      uint32_t n = 0, sums = 0;  // steps, accumulators begun
      bool ok = true;
      for (int u = cluster; u < units && ok; u += clusters) {
        const int steps = last_step(u) - first_step(u);
#pragma unroll 1
        for (int k0 = 0, end; k0 < steps * p.passes && ok; k0 = end, ++sums) {
          const uint32_t acc = sums & 1;
          end = chunk_end(steps, k0);
          ok = wait(&sh.taken[acc], ((sums >> 1) & 1) ^ 1);
          if (!ok) break;
          tc_fence_after();
#pragma unroll 1
          for (int k = k0; k < end; ++k, ++n) {
            const int s = n % kStages;
            ok = wait(&sh.full[s], (n / kStages) & 1);
            if (!ok) break;
            if (tc_elect()) {
              tc_fence_after();
#pragma unroll
              for (int kk = 0; kk < kK / 16; ++kk)
                mma_pair(tmem + acc * kN, da + (s * kHalf + kk * (kAmn ? 2048 : 32)) / 16,
                         db + (s * kHalf + kk * (kBmn ? 2048 : 32)) / 16, idesc, k > k0 || kk > 0);
              commit_pair(smem_u32(&sh.empty[s]));
              if (k == end - 1) commit_pair(smem_u32(&sh.done[acc]));
            }
            __syncwarp();
          }
        }
      }
      // the other CTA's signals have come
      for (uint32_t i = sums > 2 ? sums - 2 : 0; i < sums; ++i)
        mbar_wait(smem_u32(&sh.taken[i & 1]), (i >> 1) & 1, a.error);
    }
  } else {
    // ---------------------------------------------------------------- rows
    const int half = warp >> 2;  // of the tile's columns
    const uint32_t t_row = tmem + ((uint32_t)((warp & 3) * 32) << 16) + half * kHalfN;
    uint32_t sums = 0;
    bool ok = true;
    for (int u = cluster; u < units && ok; u += clusters) {
      const Tile t = tile_of<kN>(p, kShares ? u % tiles : u);
      const int row = t.m + (int)rank * 128 + (warp & 3) * 32 + lane, col = t.n + half * kHalfN;
      const int row0 = row - lane;  // of the warp
      const bool in = row < p.rows;
      // what the row needs beside C is on its way while the product runs
      int target = -1;
      float lse = 0.f, d = 0.f;
      if (kEnd == End::kStats || kEnd == End::kGrad) {
        if (in) target = a.targets[row];
        if (target >= a.V) target = -1;
      }
      if (kEnd == End::kGrad && in) {
        lse = a.lse[row] * kLog2e;
        d = target >= 0 ? a.dloss[row] : 0.f;
      }
      const int left = p.cols - col;  // columns that count (may be over 128 or below 1)
      const int word0 = p.v0 + col;
      // 64 bytes of each of the warp's rows, the first row's at `dst`, through the warp's stage, so that
      // a store has four neighbouring lanes per row; `bytes` of them (may be over 64) count
      auto put = [&](const uint4 (&x)[4], char* dst, long long stride, long long bytes) {
        unsigned char* stage = sh.stage[warp];
        __syncwarp();  // the stage has been read
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(stage + lane * kStageRow + i * 16) = x[i];
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = k * 8 + (lane >> 2), at = (lane & 3) * 16;
          const uint4 v = *reinterpret_cast<const uint4*>(stage + r * kStageRow + at);
          if (row0 + r < p.rows && at < bytes) *reinterpret_cast<uint4*>(dst + r * stride + at) = v;
        }
      };
      auto put_f32 = [&](const float* f, float* dst, long long stride, int columns) {
#pragma unroll
        for (int c = 0; c < kFinish; c += 16) {
          uint4 x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            x[i] = make_uint4(__float_as_uint(f[c + 4 * i]), __float_as_uint(f[c + 4 * i + 1]),
                              __float_as_uint(f[c + 4 * i + 2]), __float_as_uint(f[c + 4 * i + 3]));
          put(x, reinterpret_cast<char*>(dst + c), stride * 4, (columns - c) * 4ll);
        }
      };
      auto put_bf16 = [&](const float* f, void* dst, long long stride, int columns) {
        uint4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = Chunk<__nv_bfloat16>::pack(f + 8 * i);
        put(x, static_cast<char*>(dst), stride * 2, columns * 2ll);
      };
      // the end of the columns c .. c + kFinish - 1, by the whole warp
      auto finish = [&](int c, float* f) {
        if (c >= left) return;
        if (kEnd == End::kGrad) {
#pragma unroll
          for (int i = 0; i < kFinish; ++i) {
            const float pr = ex2f(fmaf(f[i], kLog2e, -lse));
            // an ignored position's gradient is zero whatever its logits are
            f[i] = target >= 0 ? (target == word0 + c + i ? pr - 1.f : pr) * d : 0.f;
          }
          // (the piece's rows are multiples of 16 bytes)
          if constexpr (!kF32) {
            put_bf16(f, static_cast<__nv_bfloat16*>(a.grad) + (long long)row0 * a.piece + col + c, a.piece, left - c);
          } else {
            char* g = static_cast<char*>(a.grad) + ((long long)row * a.piece + col + c) * 2;
#pragma unroll
            for (int part = 0; part < 3; ++part) {
              uint32_t w[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                w[i] = Chunk<__nv_bfloat16>::pack2(f[2 * i], f[2 * i + 1]);
                float lo, hi;  // what is left for the next part
                Chunk<__nv_bfloat16>::unpack2(w[i], lo, hi);
                f[2 * i] -= lo;
                f[2 * i + 1] -= hi;
              }
              uint4* dst = reinterpret_cast<uint4*>(g + (long long)part * a.N * a.piece * 2);
              if (in) dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
              if (in && c + 8 < left) dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
            }
          }
        }
        if (kEnd == End::kHidden || kEnd == End::kWeight) {
          if (shares > 1) {
            put_f32(f, a.sums + ((long long)(u / tiles) * p.rows + row0) * a.H + col + c, a.H, left - c);
            return;
          }
          const long long at = (long long)(kEnd == End::kWeight ? p.v0 + row0 : row0) * a.H + col + c;
          // in fp32 the pieces are added up where the result goes
          float* sum = kF32 ? static_cast<float*>(kEnd == End::kWeight ? a.dweight : a.dhidden) : a.dh;
          if (kEnd == End::kHidden && !p.first && in) {
            const float* before = sum + at + (long long)lane * a.H;
#pragma unroll
            for (int i = 0; i < kFinish; i += 4)
              if (c + i < left) {
                const float4 o = *reinterpret_cast<const float4*>(before + i);
                f[i] += o.x;
                f[i + 1] += o.y;
                f[i + 2] += o.z;
                f[i + 3] += o.w;
              }
          }
          if constexpr (!kF32) {
            if (kEnd == End::kWeight || p.last) {
              put_bf16(f, static_cast<__nv_bfloat16*>(kEnd == End::kWeight ? a.dweight : a.dhidden) + at, a.H, left - c);
              return;
            }
          }
          put_f32(f, sum + at, a.H, left - c);
        }
      };
      auto release = [&](uint32_t acc) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_cluster(in_leader(smem_u32(&sh.taken[acc])));
      };
      if constexpr (!kOften) {
        const uint32_t acc = sums & 1;
        if (!(ok = wait(&sh.done[acc], (sums >> 1) & 1))) break;
        tc_fence_after();
#pragma unroll 1
        for (int c = 0; c < kHalfN; c += 32) {
          float f[32];
          tc_ld32(t_row + acc * kN + c, f);
          tc_wait_ld();
          finish(c, f);
        }
        release(acc);
        ++sums;
      } else {
        const int steps = last_step(u) - first_step(u);
        float f[kHalfN];
#pragma unroll 1
        for (int k0 = 0; k0 < steps * p.passes; k0 = chunk_end(steps, k0), ++sums) {
          const uint32_t acc = sums & 1;
          if (!(ok = wait(&sh.done[acc], (sums >> 1) & 1))) break;
          tc_fence_after();
          if (k0 == 0) {
#pragma unroll
            for (int c = 0; c < kHalfN; c += 32) tc_ld32(t_row + acc * kN + c, f + c);
            tc_wait_ld();
          } else {
#pragma unroll
            for (int c = 0; c < kHalfN; c += 16) {
              float g[16];
              tc_ld16(t_row + acc * kN + c, g);
              tc_wait_ld();
#pragma unroll
              for (int i = 0; i < 16; ++i) f[c + i] += g[i];
            }
          }
          release(acc);
        }
        if (!ok) break;
        if (kEnd == End::kStats) {
          const bool mine = target >= word0 && target < word0 + kHalfN;
          float hit = 0.f;
          if (__any_sync(0xffffffffu, mine)) {
#pragma unroll
            for (int i = 0; i < kHalfN; ++i)
              if (target == word0 + i) hit = f[i];
          }
          if (left < kHalfN) {
#pragma unroll
            for (int i = 0; i < kHalfN; ++i) f[i] = i < left ? f[i] : -INFINITY;
          }
          float m4[4] = {f[0], f[1], f[2], f[3]};
#pragma unroll
          for (int i = 4; i < kHalfN; ++i) m4[i & 3] = fmaxf(m4[i & 3], f[i]);
          const float m = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
          const float ref = m == -INFINITY ? 0.f : m;
          float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < kHalfN; ++i) s4[i & 3] += ex2f((f[i] - ref) * kLog2e);
          if (in && left > 0) {
            a.part_m[(long long)(word0 / kHalfN) * a.N + row] = m;
            a.part_l[(long long)(word0 / kHalfN) * a.N + row] = (s4[0] + s4[1]) + (s4[2] + s4[3]);
            if (mine && target < p.v0 + p.cols) a.target_logit[row] = hit;
          }
        } else {
#pragma unroll
          for (int c = 0; c < kHalfN; c += 16) finish(c, f + c);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // neither CTA's shared or tensor memory is in use by the other
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
  }
}

// x in fp32, rows of H, as three bf16 numbers that add up to it: parts[3][rows][stride], four
// elements per thread, of one matrix or of two. Bound by HBM.
struct ToParts {
  const float* x;
  long long rows;
  char* parts;
};
__global__ void __launch_bounds__(256) loss_parts_kernel(const ToParts first, const ToParts second, int H, int stride) {
  const int per = H / 4;
  long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const bool one = i < first.rows * per;
  if (!one) i -= first.rows * per;
  const ToParts& m = one ? first : second;
  if (i >= m.rows * per) return;
  const long long r = i / per;
  const int c = (int)(i % per) * 4;
  const float4 v = *reinterpret_cast<const float4*>(m.x + r * H + c);
  float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int part = 0; part < 3; ++part) {
    uint32_t u[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      u[k] = Chunk<__nv_bfloat16>::pack2(f[2 * k], f[2 * k + 1]);
      float lo, hi;
      Chunk<__nv_bfloat16>::unpack2(u[k], lo, hi);
      f[2 * k] -= lo;
      f[2 * k + 1] -= hi;
    }
    *reinterpret_cast<uint2*>(m.parts + ((part * m.rows + r) * stride + c) * 2) = make_uint2(u[0], u[1]);
  }
}
// the parts of `words` rows of the weights, and with the first of them those of the hidden states
cudaError_t to_parts(const LossArgs& a, int v0, int words, cudaStream_t stream) {
  const ToParts weight = {static_cast<const float*>(a.weight) + (long long)v0 * a.H, words, static_cast<char*>(a.weight_parts)};
  const ToParts hidden = {static_cast<const float*>(a.hidden), v0 == 0 ? a.N : 0, static_cast<char*>(a.hidden_parts)};
  const long long n = (weight.rows + hidden.rows) * (a.H / 4);
  loss_parts_kernel<<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(weight, hidden, a.H, loss_stride(a.H));
  return cudaGetLastError();
}

// The shares' sums of a gradient, in their order, and dhidden of the pieces before: to `sum` in
// fp32 or to `out` in bf16. Bound by the L2 cache, where the sums still are.
__global__ void __launch_bounds__(256) loss_sums_kernel(const float* sums, int shares, long long n, float* sum, bool add,
                                                        __nv_bfloat16* out) {
  const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= n) return;
  float4 x = add ? *reinterpret_cast<const float4*>(sum + i) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = 0; s < shares; ++s) {
    const float4 y = *reinterpret_cast<const float4*>(sums + s * n + i);
    x.x += y.x;
    x.y += y.y;
    x.z += y.z;
    x.w += y.w;
  }
  if (out)
    *reinterpret_cast<uint2*>(out + i) =
        make_uint2(Chunk<__nv_bfloat16>::pack2(x.x, x.y), Chunk<__nv_bfloat16>::pack2(x.z, x.w));
  else
    *reinterpret_cast<float4*>(sum + i) = x;
}

// An operand: a matrix of `rows` x `cols` in bf16, or its three parts, rows `stride` elements
// apart, in boxes of `box` rows x 64 columns; what lies outside reads as zero.
cudaError_t matrix_map(CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint64_t stride, uint32_t box,
                       int parts) {
  const TensorMapEncode encode = tensor_map_encode();
  if (!encode) return cudaErrorNotSupported;
  const cuuint64_t dims[3] = {cols, rows, (cuuint64_t)parts}, strides[2] = {stride * 2, stride * 2 * rows};
  const cuuint32_t boxes[3] = {64, box, 1}, unit[3] = {1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, boxes, unit,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// Columns of a tile: 256, or 128 where tiles of 256 would be too few for half of the pairs of
// SMs: twice as many clusters, each with half the work per step (257 x 256 x 1009 in fp32, forward and
// backward, 135 us with 256, 80 with 128).
inline int tile_columns(int rows, int cols, int sms) {
  const long long tiles = (long long)ceil_div(rows, kM) * ceil_div(cols, 256);
  return tiles * 4 <= sms ? 128 : 256;
}

// Shares of a gradient's sums: as many as there are pairs of SMs for each tile, if their steps
// are eight at least. 8 x 1024 x 100000 forward and backward 512 us whole, 257 in shares; 100 x 2048 x 32000
// in fp32 1289 and 862; 257 x 256 x 1009 in fp32 62 and 49; 8192 x 256 x 1000 74 and 54.
inline int sum_shares(long long tiles, int steps, int passes, int pairs) {
  const long long most = min(steps, steps * passes / 8), n = min((long long)pairs, kSumTiles) / tiles;
  return (int)(n < 2 || most < 2 ? 1 : n < most ? n : most);
}

template <End kEnd, bool kF32, int kN>
cudaError_t launch_product(ProductArgs& p, int sms, cudaStream_t stream) {
  constexpr bool kShares = kEnd == End::kHidden || kEnd == End::kWeight;
  cudaError_t e = allow_shared<loss_product_kernel<kEnd, kF32, kN>>(kProductSmem);
  if (e != cudaSuccess) return e;
  const long long tm = ceil_div(p.rows, kM), tn = ceil_div(p.cols, kN);
  p.passes = kF32 ? 6 : 1;
  // row tiles whose operand takes about a third of L2
  const long long group = (40ll << 20) / ((long long)kM * p.depth * (kF32 ? 6 : 2));
  p.group = (int)(group < 1 ? 1 : group > tm ? tm : group);
  const int pairs = sms / 2;
  p.shares = kShares ? sum_shares(tm * tn, ceil_div(p.depth, kK), p.passes, pairs) : 1;
  const long long units = tm * tn * p.shares;
  loss_product_kernel<kEnd, kF32, kN><<<2 * (unsigned)(units < pairs ? units : pairs), kProductThreads, kProductSmem, stream>>>(p);
  e = cudaGetLastError();
  if (e != cudaSuccess || p.shares == 1) return e;
  const LossArgs& a = p.a;
  const long long n = (long long)p.rows * a.H, at = kEnd == End::kWeight ? (long long)p.v0 * a.H : 0;
  void* result = kEnd == End::kWeight ? a.dweight : a.dhidden;
  float* sum = kF32 ? static_cast<float*>(result) + at : a.dh;
  __nv_bfloat16* out = !kF32 && (kEnd == End::kWeight || p.last) ? static_cast<__nv_bfloat16*>(result) + at : nullptr;
  loss_sums_kernel<<<(unsigned)((n / 4 + 255) / 256), 256, 0, stream>>>(a.sums, p.shares, n, sum, kEnd == End::kHidden && !p.first,
                                                                        out);
  return cudaGetLastError();
}

// C = A B, with the boxes of rows of B's map for its layout
template <End kEnd, bool kF32>
cudaError_t product(ProductArgs& p, const void* a, uint64_t a_rows, uint64_t a_cols, uint64_t a_stride, const void* b,
                    uint64_t b_rows, uint64_t b_cols, uint64_t b_stride, int columns, int sms, cudaStream_t stream) {
  constexpr bool kAmn = kEnd == End::kWeight, kBmn = kEnd == End::kHidden || kEnd == End::kWeight;
  const int parts = kF32 ? 3 : 1;
  cudaError_t e = matrix_map(&p.ma, a, a_rows, a_cols, a_stride, kAmn ? 64 : 128, parts);
  if (e == cudaSuccess) e = matrix_map(&p.mb, b, b_rows, b_cols, b_stride, kBmn ? 64 : columns / 2, parts);
  if (e != cudaSuccess) return e;
  return columns == 128 ? launch_product<kEnd, kF32, 128>(p, sms, stream) : launch_product<kEnd, kF32, 256>(p, sms, stream);
}

template <bool kF32>
cudaError_t forward(const LossArgs& a, int* share, cudaStream_t stream) {
  const int stride = kF32 ? loss_stride(a.H) : a.H;
  int sms = 0;
  cudaError_t e = sm_count(&sms);
  const int columns = tile_columns(a.N, a.V, sms);
  *share = columns / 2;
  // fp32: by pieces, as the weights' parts are made; bf16: all words at once
  const int piece = kF32 ? a.piece : a.V;
  for (int v0 = 0; v0 < a.V && e == cudaSuccess; v0 += piece) {
    const int words = min(piece, a.V - v0);
    const char* w = static_cast<const char*>(a.weight) + (long long)v0 * a.H * (kF32 ? 4 : 2);
    if (kF32) e = to_parts(a, v0, words, stream);
    ProductArgs p = {};
    p.a = a;
    p.v0 = v0;
    p.rows = a.N;
    p.cols = words;
    p.depth = a.H;
    if (e == cudaSuccess)
      e = product<End::kStats, kF32>(p, kF32 ? a.hidden_parts : a.hidden, a.N, a.H, stride, kF32 ? a.weight_parts : w, words,
                                     a.H, stride, columns, sms, stream);
  }
  return e;
}

template <bool kF32>
cudaError_t backward(const LossArgs& a, cudaStream_t stream) {
  const int stride = kF32 ? loss_stride(a.H) : a.H;
  int sms = 0;
  cudaError_t e = sm_count(&sms);
  const void* hidden = kF32 ? a.hidden_parts : a.hidden;
  for (int v0 = 0; v0 < a.V && e == cudaSuccess; v0 += a.piece) {
    ProductArgs p = {};
    p.a = a;
    p.v0 = v0;
    p.first = v0 == 0;
    p.last = a.V - v0 <= a.piece;
    const int words = p.last ? a.V - v0 : a.piece;
    const char* w = static_cast<const char*>(a.weight) + (long long)v0 * a.H * (kF32 ? 4 : 2);
    if (kF32) {
      e = to_parts(a, v0, words, stream);
      w = static_cast<const char*>(a.weight_parts);
    }
    p.rows = a.N;
    p.cols = words;
    p.depth = a.H;
    if (e == cudaSuccess)
      e = product<End::kGrad, kF32>(p, hidden, a.N, a.H, stride, w, words, a.H, stride, tile_columns(a.N, words, sms), sms,
                                    stream);
    p.cols = a.H;
    p.depth = words;
    if (e == cudaSuccess)
      e = product<End::kHidden, kF32>(p, a.grad, a.N, words, a.piece, w, words, a.H, stride, tile_columns(a.N, a.H, sms), sms,
                                      stream);
    p.rows = words;
    p.depth = a.N;
    if (e == cudaSuccess)
      e = product<End::kWeight, kF32>(p, a.grad, a.N, words, a.piece, hidden, a.N, a.H, stride, tile_columns(words, a.H, sms),
                                      sms, stream);
  }
  return e;
}

}  // namespace

// share: words of each of the shares whose maxima and sums are left in part_m, part_l
cudaError_t loss_forward(const LossArgs& a, bool bf16, int* share, cudaStream_t stream) {
  return bf16 ? forward<false>(a, share, stream) : forward<true>(a, share, stream);
}
cudaError_t loss_backward(const LossArgs& a, bool bf16, cudaStream_t stream) {
  return bf16 ? backward<false>(a, stream) : backward<true>(a, stream);
}

}  // namespace dmc
