// Cross entropy against a vocabulary and its gradient in bf16, on the tensor cores.
//
// One matrix product with four operand layouts and ends (C is never the logits):
//   statistics   hidden W^T, per token and tile of 256 words the maximum and the sum of
//                exponentials (and the target's logit); a small kernel joins them
//   gradient     hidden W^T again, and g = (exp(logit - lse) - [word = target]) dloss,
//                rounded to bf16 for the products that follow, for one piece of the words
//   dhidden      g W, added up over the pieces in fp32
//   dweight      g^T hidden
// 8 N H V operations for a forward and a backward pass, of which 6 are the least
// possible: the logits of N tokens and V words in fp32 would be kept otherwise.
//
// A pair of CTAs (one cluster) computes 256 x 256 of C, each CTA 128 rows of it:
// tcgen05.mma with cta_group::2, M = N = 256, K = 16, issued by the even CTA, both
// operands split between the two CTAs' shared memory, so that an SM loads 32 KB per 64
// columns of K where one CTA alone would load 48 KB for its 128 x 256 (the SMs' share of
// L2 bandwidth is about what the former needs). Warps are specialised: warp 4 loads
// tiles by TMA into a ring of six, warp 5 issues the products, warps 0-3 (a row of C
// per thread) work on the result of one tile while the next is computed: two
// accumulators of 256 columns fill the tensor memory. Clusters walk over the tiles with a
// fixed stride, down groups of rows, so that both operands of the tiles in flight are in L2.
#include <math.h>

#include "dmc_retrofit.cuh"
#include "dmc_tensor.cuh"

namespace dmc {

namespace {

constexpr int kM = 256;        // rows of C per cluster
constexpr int kN = kLossTile;  // columns of C
constexpr int kK = 64;         // columns of a step
constexpr int kStages = 6;
constexpr int kHalf = 128 * kK * 2;  // bytes of a CTA's half of an operand's tile
constexpr int kProductThreads = 192;

struct ProductShared {
  unsigned char a[kStages][kHalf], b[kStages][kHalf];
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
  int group;              // row tiles of a group
  int v0;                 // first word of the piece
  bool first, last;       // of the pieces
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
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4}], "
      "[%2];" ::"r"(dst),
      "l"(map), "r"(bar), "r"(x), "r"(y)
      : "memory");
}
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

template <End kEnd>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kProductThreads, 1)
loss_product_kernel(const __grid_constant__ ProductArgs p) {
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
  const int steps = (p.depth + kK - 1) / kK;
  volatile int* s_abort = &sh.abort;
  auto wait = [&](uint64_t* bar, uint32_t ph) -> bool { return warp_wait(smem_u32(bar), ph, s_abort, a.error); };

  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(smem_u32(&sh.full[i]), 1);
      mbar_init(smem_u32(&sh.empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sh.done[i]), 1);
      mbar_init(smem_u32(&sh.taken[i]), 8);  // the four row warps of both CTAs
    }
    fence_mbar_init();
    sh.abort = 0;
  }
  if (warp == 5) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(512));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // both CTAs' barriers stand before either signals the other's
  tc_fence_after();
  const uint32_t tmem = tc_uniform(sh.tmem);

  if (warp == 4) {
    // ---------------------------------------------------------------- loads
    uint32_t n = 0;
    bool ok = true;
    for (int u = cluster; u < tiles && ok; u += clusters) {
      const Tile t = tile_of(p, u);
      const int m = t.m + (int)rank * 128, c = t.n + (int)rank * 128;  // this CTA's half
#pragma unroll 1
      for (int k = 0; k < steps; ++k, ++n) {
        const int s = n % kStages;
        ok = wait(&sh.empty[s], ((n / kStages) & 1) ^ 1);
        if (!ok) break;
        if (tc_elect()) {
          if (rank == 0) mbar_arrive_expect_tx(smem_u32(&sh.full[s]), 4 * kHalf);
          const uint32_t bar = in_leader(smem_u32(&sh.full[s]));
          const uint32_t da = smem_u32(sh.a[s]), db = smem_u32(sh.b[s]);
          if (kAmn) {
            tma_load_pair(da, &p.ma, bar, m, k * kK);
            tma_load_pair(da + kHalf / 2, &p.ma, bar, m + 64, k * kK);
          } else {
            tma_load_pair(da, &p.ma, bar, k * kK, m);
          }
          if (kBmn) {
            tma_load_pair(db, &p.mb, bar, c, k * kK);
            tma_load_pair(db + kHalf / 2, &p.mb, bar, c + 64, k * kK);
          } else {
            tma_load_pair(db, &p.mb, bar, k * kK, c);
          }
        }
        __syncwarp();
      }
    }
    // the last tiles have been read (so every copy has landed, and every signal has come)
    for (uint32_t i = n > kStages ? n - kStages : 0; i < n; ++i)
      mbar_wait(smem_u32(&sh.empty[i % kStages]), (i / kStages) & 1, a.error);
  } else if (warp == 5) {
    // ---------------------------------------------------------------- products
    if (rank == 0) {
      constexpr uint32_t idesc = tc_idesc(kM, kN, kAmn, kBmn);
      // K-major: rows of 128 bytes, eight of them every 1024; MN-major: 64 elements of a
      // row per 128 bytes, the next 64 half a tile on
      const uint64_t da = tc_desc(smem_u32(sh.a[0]), kAmn ? kHalf / 2 : 16, 1024);
      const uint64_t db = tc_desc(smem_u32(sh.b[0]), kBmn ? kHalf / 2 : 16, 1024);
      uint32_t n = 0, tile = 0;
      bool ok = true;
      for (int u = cluster; u < tiles && ok; u += clusters, ++tile) {
        const uint32_t acc = tile & 1;
        ok = wait(&sh.taken[acc], ((tile >> 1) & 1) ^ 1);
        if (!ok) break;
        tc_fence_after();
#pragma unroll 1
        for (int k = 0; k < steps; ++k, ++n) {
          const int s = n % kStages;
          ok = wait(&sh.full[s], (n / kStages) & 1);
          if (!ok) break;
          if (tc_elect()) {
            tc_fence_after();
#pragma unroll
            for (int kk = 0; kk < kK / 16; ++kk)
              mma_pair(tmem + acc * kN, da + (s * kHalf + kk * (kAmn ? 2048 : 32)) / 16,
                       db + (s * kHalf + kk * (kBmn ? 2048 : 32)) / 16, idesc, k > 0 || kk > 0);
            commit_pair(smem_u32(&sh.empty[s]));
            if (k == steps - 1) commit_pair(smem_u32(&sh.done[acc]));
          }
          __syncwarp();
        }
      }
      // the other CTA's signals have come
      for (uint32_t i = tile > 2 ? tile - 2 : 0; i < tile; ++i)
        mbar_wait(smem_u32(&sh.taken[i & 1]), (i >> 1) & 1, a.error);
    }
  } else {
    // ---------------------------------------------------------------- rows
    const uint32_t t_row = tmem + ((uint32_t)(warp * 32) << 16);
    uint32_t tile = 0;
    for (int u = cluster; u < tiles; u += clusters, ++tile) {
      const Tile t = tile_of(p, u);
      const uint32_t acc = tile & 1;
      const int row = t.m + (int)rank * 128 + tid;
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
      if (!wait(&sh.done[acc], (tile >> 1) & 1)) break;
      tc_fence_after();
      float mx = -INFINITY, sum = 0.f, hit = 0.f;
      const int word0 = (kEnd == End::kGrad ? p.v0 : 0) + t.n;
      const bool mine = target >= word0 && target < word0 + kN;
      const bool any = (kEnd == End::kStats || kEnd == End::kGrad) && __any_sync(0xffffffffu, mine);
#pragma unroll 1
      for (int c = 0; c < kN; c += 32) {
        if (t.n + c >= p.cols) break;
        float f[32];
        tc_ld32(t_row + acc * kN + c, f);
        tc_wait_ld();
        const int left = p.cols - (t.n + c);  // columns that count
        if (kEnd == End::kStats) {
          if (any)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (target == word0 + c + i) hit = f[i];
          if (left < 32)
#pragma unroll
            for (int i = 0; i < 32; ++i) f[i] = i < left ? f[i] : -INFINITY;
          float m4[4] = {f[0], f[1], f[2], f[3]};
#pragma unroll
          for (int i = 4; i < 32; ++i) m4[i & 3] = fmaxf(m4[i & 3], f[i]);
          const float m = fmaxf(mx, fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])));
          const float ref = m == -INFINITY ? 0.f : m * kLog2e;
          sum *= ex2f(mx * kLog2e - ref);
          mx = m;
          float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 32; ++i) s4[i & 3] += ex2f(fmaf(f[i], kLog2e, -ref));
          sum += (s4[0] + s4[1]) + (s4[2] + s4[3]);
        }
        if (kEnd == End::kGrad) {
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float pr = ex2f(fmaf(f[i], kLog2e, -lse));
            // an ignored position's gradient is zero whatever its logits are
            f[i] = target >= 0 ? ((any && target == word0 + c + i) ? pr - 1.f : pr) * d : 0.f;
          }
          if (in) {
            char* g = static_cast<char*>(a.grad) + ((long long)row * a.piece + t.n + c) * 2;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (8 * i < left)  // (the piece's rows are multiples of 16 bytes)
                reinterpret_cast<uint4*>(g)[i] = Chunk<__nv_bfloat16>::pack(f + 8 * i);
          }
        }
        if (kEnd == End::kHidden || kEnd == End::kWeight) {
          const long long at = (long long)(kEnd == End::kWeight ? p.v0 + row : row) * a.H + t.n + c;
          if (in) {
            if (kEnd == End::kHidden && !p.first) {
#pragma unroll
              for (int i = 0; i < 8; ++i)
                if (4 * i < left) {
                  const float4 o = *reinterpret_cast<const float4*>(a.dh + at + 4 * i);
                  f[4 * i] += o.x;
                  f[4 * i + 1] += o.y;
                  f[4 * i + 2] += o.z;
                  f[4 * i + 3] += o.w;
                }
            }
            if (kEnd == End::kWeight || p.last) {
              uint4* out = reinterpret_cast<uint4*>(static_cast<char*>(kEnd == End::kWeight ? a.dweight : a.dhidden) + at * 2);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (8 * i < left) out[i] = Chunk<__nv_bfloat16>::pack(f + 8 * i);
            } else {
#pragma unroll
              for (int i = 0; i < 8; ++i)
                if (4 * i < left)
                  *reinterpret_cast<float4*>(a.dh + at + 4 * i) = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_cluster(in_leader(smem_u32(&sh.taken[acc])));
      if (kEnd == End::kStats && in) {
        a.part_m[(long long)(t.n / kN) * a.N + row] = mx;
        a.part_l[(long long)(t.n / kN) * a.N + row] = sum;
        if (mine) a.target_logit[row] = hit;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // neither CTA's shared or tensor memory is in use by the other
  if (warp == 5) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
  }
}

// A matrix of `rows` x `cols` in bf16, rows `stride` bytes apart, in boxes of `box` rows x
// 64 columns; what lies outside reads as zero.
cudaError_t matrix_map(CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint64_t stride, uint32_t box) {
  const TensorMapEncode encode = tensor_map_encode();
  if (!encode) return cudaErrorNotSupported;
  const cuuint64_t dims[2] = {cols, rows}, strides[1] = {stride};
  const cuuint32_t boxes[2] = {64, box}, unit[2] = {1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, boxes, unit,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <End kEnd>
cudaError_t launch_product(ProductArgs& p, cudaStream_t stream) {
  auto* kernel = loss_product_kernel<kEnd>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kProductSmem);
  if (e != cudaSuccess) return e;
  int dev = 0, sms = 0;
  e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  const long long tm = (p.rows + kM - 1) / kM, tn = (p.cols + kN - 1) / kN;
  // row tiles whose operand takes about a third of L2
  const long long group = (40ll << 20) / ((long long)kM * p.depth * 2);
  p.group = (int)(group < 1 ? 1 : group > tm ? tm : group);
  const long long tiles = tm * tn;
  const int pairs = sms / 2;
  kernel<<<2 * (unsigned)(tiles < pairs ? tiles : pairs), kProductThreads, kProductSmem, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t loss_forward_bf16(const LossArgs& a, int* shares, cudaStream_t stream) {
  ProductArgs p = {};
  p.a = a;
  p.rows = a.N;
  p.cols = a.V;
  p.depth = a.H;
  *shares = ceil_div(a.V, kN);
  cudaError_t e = matrix_map(&p.ma, a.hidden, a.N, a.H, (uint64_t)a.H * 2, 128);
  if (e == cudaSuccess) e = matrix_map(&p.mb, a.weight, a.V, a.H, (uint64_t)a.H * 2, 128);
  return e == cudaSuccess ? launch_product<End::kStats>(p, stream) : e;
}

cudaError_t loss_backward_bf16(const LossArgs& a, cudaStream_t stream) {
  const uint64_t row = (uint64_t)a.H * 2, grow = (uint64_t)a.piece * 2;
  for (int v0 = 0; v0 < a.V; v0 += a.piece) {
    ProductArgs p = {};
    p.a = a;
    p.v0 = v0;
    p.first = v0 == 0;
    p.last = a.V - v0 <= a.piece;
    const int words = p.last ? a.V - v0 : a.piece;
    const char* w = static_cast<const char*>(a.weight) + v0 * row;
    p.rows = a.N;
    p.cols = words;
    p.depth = a.H;
    cudaError_t e = matrix_map(&p.ma, a.hidden, a.N, a.H, row, 128);
    if (e == cudaSuccess) e = matrix_map(&p.mb, w, words, a.H, row, 128);
    if (e == cudaSuccess) e = launch_product<End::kGrad>(p, stream);
    p.cols = a.H;
    p.depth = words;
    if (e == cudaSuccess) e = matrix_map(&p.ma, a.grad, a.N, words, grow, 128);
    if (e == cudaSuccess) e = matrix_map(&p.mb, w, words, a.H, row, 64);
    if (e == cudaSuccess) e = launch_product<End::kHidden>(p, stream);
    p.rows = words;
    p.depth = a.N;
    if (e == cudaSuccess) e = matrix_map(&p.ma, a.grad, a.N, words, grow, 64);
    if (e == cudaSuccess) e = matrix_map(&p.mb, a.hidden, a.N, a.H, row, 64);
    if (e == cudaSuccess) e = launch_product<End::kWeight>(p, stream);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace dmc
