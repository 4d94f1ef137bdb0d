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

// A piece of a sequence's tokens and a head.
struct Work {
  int t0, t1;  // the sequence's tokens
  int seq, at; // the sequence, the piece's index in it
  int head;    // below 0: no more work
};

// Pieces by cost: the k-th of all, when those of the highest index (kFromEnd: of the most
// pieces from it on) come first, whatever sequence they belong to, so that the last ones
// to be handed out are the cheapest. With f(L) = sum over sequences of max(0, pieces - L), the
// number of pieces with L others before (after) them, L is the largest with f(L) > k. For
// up to 128 sequences, by a whole warp (four sequences per lane). More are taken in their
// order (ordered_work), where one sequence matters less and the search over L would take longer
// than a short item. False: there are no more.
constexpr int kRankedSeqs = 128;
struct RankedSeqs {
  int t0[kRankedSeqs / 32], t1[kRankedSeqs / 32];  // the lane's sequences, empty where there is none
};
__device__ __forceinline__ void ranked_seqs(const Seqs& q, RankedSeqs& r) {
#pragma unroll
  for (int i = 0; i < kRankedSeqs / 32; ++i) {
    const int s = i * 32 + (threadIdx.x & 31);
    r.t0[i] = r.t1[i] = 0;
    if (q.num > kRankedSeqs || s >= q.num) continue;
    r.t0[i] = q.cu[s];
    r.t1[i] = q.cu[s + 1];
    if (!seq_ok(q, r.t0[i], r.t1[i])) r.t1[i] = r.t0[i];
  }
}
__device__ __forceinline__ bool ranked_work(const RankedSeqs& q, int piece, bool from_end, int k, Work& w) {
  const int lane = threadIdx.x & 31;
  int n[kRankedSeqs / 32], most = 0;
#pragma unroll
  for (int i = 0; i < kRankedSeqs / 32; ++i) {
    n[i] = (q.t1[i] - q.t0[i] + piece - 1) / piece;
    most = max(most, n[i]);
  }
  auto f = [&](int L) {
    int x = 0;
#pragma unroll
    for (int i = 0; i < kRankedSeqs / 32; ++i) x += max(0, n[i] - L);
    return __reduce_add_sync(0xffffffffu, x);
  };
  if (k >= f(0)) return false;
  int lo = 0, hi = __reduce_max_sync(0xffffffffu, most);  // f(lo) > k >= f(hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (f(mid) > k) lo = mid; else hi = mid;
  }
  int left = k - f(lo + 1);  // the left-th sequence of more than lo pieces
#pragma unroll
  for (int i = 0; i < kRankedSeqs / 32; ++i) {
    const unsigned int b = __ballot_sync(0xffffffffu, n[i] > lo);
    const unsigned int hit = __ballot_sync(0xffffffffu, n[i] > lo && __popc(b & ((1u << lane) - 1)) == left);
    if (hit) {
      const int from = __ffs(hit) - 1;
      w.seq = i * 32 + from;
      w.t0 = __shfl_sync(0xffffffffu, q.t0[i], from);
      w.t1 = __shfl_sync(0xffffffffu, q.t1[i], from);
    }
    left -= __popc(b);
  }
  w.at = from_end ? (w.t1 - w.t0 + piece - 1) / piece - 1 - lo : lo;
  return true;
}

__device__ __forceinline__ bool ordered_work(const Seqs& q, int piece, bool from_end, int k, Work& w) {
  const int lane = threadIdx.x & 31;
  for (int base = 0; base < q.num; base += 32) {
    const int s = base + lane;
    int n = 0, t0 = 0, t1 = 0;
    if (s < q.num) {
      t0 = q.cu[s];
      t1 = q.cu[s + 1];
      if (seq_ok(q, t0, t1)) n = (t1 - t0 + piece - 1) / piece;
    }
    const int all = __reduce_add_sync(0xffffffffu, n);
    if (k >= all) {
      k -= all;
      continue;
    }
    int upto = n;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, upto, off);
      if (lane >= off) upto += o;
    }
    const int hit = __ffs(__ballot_sync(0xffffffffu, k < upto)) - 1;
    const int i = k - __shfl_sync(0xffffffffu, upto - n, hit);
    w.seq = base + hit;
    w.t0 = __shfl_sync(0xffffffffu, t0, hit);
    w.t1 = __shfl_sync(0xffffffffu, t1, hit);
    w.at = from_end ? i : __shfl_sync(0xffffffffu, n, hit) - 1 - i;  // the most expensive first
    return true;
  }
  return false;
}

// Work is numbered by piece, heads fastest: items of one length run side by side. (Groups of heads whose
// K and V fit in L2, one group after another, are slower: four sequences of 2048 tokens, 32 heads, forward
// 134 -> 151 us; 8192 tokens of 64 / 8 heads, backward 2.74 -> 3.34 ms.) The numbers 0 .. gridDim - 1 go to the CTAs, then
// each takes the next from a counter. Warp 9 does so, one piece of work ahead of the other
// warps, and hands it to them. The last CTA resets the counter for the next launch.
struct WorkRing {
  Work work[2];
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

// Warp 9's side.
struct WorkSource {
  int number;  // the next work's, in the first lane (elsewhere it would be waited for)
  int turn;    // the next place in the ring
  RankedSeqs seqs;
};
__device__ __forceinline__ WorkSource work_source(const Seqs& q) {
  WorkSource src;
  src.number = blockIdx.x;
  src.turn = 0;
  ranked_seqs(q, src.seqs);
  return src;
}
// The next work, handed to the other warps too (head < 0: there is none, or a wait gave up).
template <typename Wait>
__device__ __forceinline__ Work take_work(WorkRing& ring, WorkSource& src, const Seqs& q, int piece, bool from_end, int heads,
                                          int most, int* counter, const Wait& wait) {
  Work w;
  w.t0 = w.t1 = w.seq = w.at = 0;
  w.head = -1;
  const int number = __shfl_sync(0xffffffffu, src.number, 0);
  if (number < most) {
    if ((threadIdx.x & 31) == 0) src.number = (int)gridDim.x + atomicAdd(counter, 1);
    const int k = number / heads;
    const bool there = q.num <= kRankedSeqs ? ranked_work(src.seqs, piece, from_end, k, w) : ordered_work(q, piece, from_end, k, w);
    if (there) w.head = number % heads;
  }
  const int sl = src.turn & 1;
  if (!wait(&ring.empty[sl], ((src.turn >> 1) & 1) ^ 1)) {
    w.head = -1;
    return w;
  }
  if ((threadIdx.x & 31) == 0) ring.work[sl] = w;
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&ring.full[sl]));
  ++src.turn;
  return w;
}
// The other warps' side (head < 0: no more work, or a wait gave up).
template <typename Wait>
__device__ __forceinline__ Work next_work(WorkRing& ring, int& turn, const Wait& wait) {
  const int sl = turn & 1;
  Work w;
  w.t0 = w.t1 = w.seq = w.at = 0;
  w.head = -1;
  if (!wait(&ring.full[sl], (turn >> 1) & 1)) return w;
  w.t0 = tc_uniform(ring.work[sl].t0);
  w.t1 = tc_uniform(ring.work[sl].t1);
  w.seq = tc_uniform(ring.work[sl].seq);
  w.at = tc_uniform(ring.work[sl].at);
  w.head = tc_uniform(ring.work[sl].head);
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&ring.empty[sl]));
  ++turn;
  return w;
}

template <int D>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int head, int tok) {
#pragma unroll
  for (int c = 0; c < D / 64; ++c) tma_load(dst + c * (kR * 128), map, bar, c * 64, head, tok);
}

// Rows of the epilogue: 64 bytes of each lane's row to global memory through the warp's
// stage; row r of the warp at dst + r * stride bytes, rows at and after `rows` left out.
__device__ __forceinline__ void write_rows(unsigned char* stage, const uint4 (&x)[4], char* dst, long long stride, int rows) {
  const int lane = threadIdx.x & 31;
  __syncwarp();  // the stage has been read
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(stage + lane * kStageRow + i * 16) = x[i];
  __syncwarp();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = k * 8 + (lane >> 2);
    const uint4 v = *reinterpret_cast<const uint4*>(stage + r * kStageRow + (lane & 3) * 16);
    if (r < rows) *reinterpret_cast<uint4*>(dst + r * stride + (lane & 3) * 16) = v;
  }
}
// 32 values of each row, as bf16
__device__ __forceinline__ void write_rows(unsigned char* stage, const float* f, char* dst, long long stride, int rows) {
  uint4 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = Chunk<__nv_bfloat16>::pack(f + i * 8);
  write_rows(stage, x, dst, stride, rows);
}

// Rows [r0, 128) of a tile set to zero, by a warp: weights are zero there, but what lies
// beyond a sequence's end need not be a number.
template <int D>
__device__ __forceinline__ void zero_rows(unsigned char* tile, int r0) {
  constexpr int kPieces = D / 8, kRows = 32 / kPieces;  // 16-byte pieces of a row, rows at a time
  const int j = threadIdx.x % kPieces;
  unsigned char* at = tile + (j >> 3) * (kR * 128) + (j & 7) * 16;
#pragma unroll 4
  for (int r = r0 + (threadIdx.x & 31) / kPieces; r < kR; r += kRows)
    *reinterpret_cast<uint4*>(at + r * 128) = make_uint4(0, 0, 0, 0);
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

}  // namespace dmc
