// What the tensor-core attention kernels of the retrofitting calls share: tiles of 128
// rows, their loads, work items from a counter, rows of an epilogue.
#pragma once

#include <limits.h>
#include <math.h>

#include "dmc_retrofit.cuh"
#include "dmc_tensor.cuh"

namespace dmc {

constexpr int kR = 128;           // rows of a tile
constexpr int kAttnThreads = 384; // 12 warps: 0-7 rows, 8 products, 9 loads; the others complete a warpgroup
constexpr int kStageRow = 80;     // bytes of a row of an epilogue stage: 64 and 16 of padding
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Work items are taken from a counter: index 0 .. gridDim - 1 without one, then in the
// order in which CTAs come for more. Warp 9 takes an item ahead of the others and hands
// it to them. The last CTA resets the counter for the next launch.
struct WorkRing {
  int index[2];
  uint64_t full[2], empty[2];
};
__device__ __forceinline__ void work_init(WorkRing& w) {
  for (int i = 0; i < 2; ++i) {
    mbar_init(smem_u32(&w.full[i]), 1);
    mbar_init(smem_u32(&w.empty[i]), 9);  // the row warps and the product warp
  }
}
__device__ __forceinline__ void work_done(int* counter) {
  __threadfence();
  if (atomicAdd(&counter[1], 1) == (int)gridDim.x - 1) {
    counter[0] = 0;
    counter[1] = 0;
    __threadfence();
  }
}

template <int D>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int head, int tok) {
#pragma unroll
  for (int c = 0; c < D / 64; ++c) tma_load(dst + c * (kR * 128), map, bar, c * 64, head, tok);
}

// Rows of the epilogue: 32 columns of each lane's row (values f) to global memory through the
// warp's stage; row r of the warp at dst + r * stride bytes, rows at and after `rows` left out.
__device__ __forceinline__ void write_rows(unsigned char* stage, const float* f, char* dst, long long stride, int rows) {
  const int lane = threadIdx.x & 31;
  __syncwarp();  // the stage has been read
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<uint4*>(stage + lane * kStageRow + i * 16) = Chunk<__nv_bfloat16>::pack(f + i * 8);
  __syncwarp();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = k * 8 + (lane >> 2);
    const uint4 v = *reinterpret_cast<const uint4*>(stage + r * kStageRow + (lane & 3) * 16);
    if (r < rows) *reinterpret_cast<uint4*>(dst + r * stride + (lane & 3) * 16) = v;
  }
}

// Rows [r0, 128) of a tile set to zero, by a warp: weights are zero there, but what lies
// beyond a sequence's end need not be a number.
template <int D>
__device__ __forceinline__ void zero_rows(unsigned char* tile, int r0) {
  constexpr int kPieces = D / 8;  // of 16 bytes per row
#pragma unroll 1
  for (int x = threadIdx.x & 31; x < (kR - r0) * kPieces; x += 32) {
    const int r = r0 + x / kPieces, j = x % kPieces;
    *reinterpret_cast<uint4*>(tile + (j >> 3) * (kR * 128) + r * 128 + (j & 7) * 16) = make_uint4(0, 0, 0, 0);
  }
  fence_async_smem();
  __syncwarp();
}

// [token][head][D] in bf16, boxes of 128 tokens x 64 columns of one head; zero beyond the last token
inline cudaError_t heads_map(CUtensorMap* map, const void* base, int D, int heads, int tokens) {
  const TensorMapEncode encode = tensor_map_encode();
  if (!encode) return cudaErrorNotSupported;
  const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)tokens};
  const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)D * 2 * heads};
  const cuuint32_t box[3] = {64, 1, kR}, unit[3] = {1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, unit,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

inline cudaError_t sm_count(int* sms) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  return e == cudaSuccess ? cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) : e;
}

}  // namespace dmc
