// What the retrofitting kernels share: the view of a call's packed sequences and
// of the handle's scratch.
#pragma once

#include <atomic>

#include "dmc_internal.cuh"

namespace dmc {

// What a launch asks of the runtime once per device and process: the number of SMs, and leave
// for a kernel to use so much shared memory.
constexpr int kMostDevices = 64;
inline cudaError_t this_device(int* dev) {
  const cudaError_t e = cudaGetDevice(dev);
  return e == cudaSuccess && *dev >= kMostDevices ? cudaErrorInvalidDevice : e;
}
inline cudaError_t sm_count(int* sms) {
  static std::atomic<int> known[kMostDevices];
  int dev = 0;
  cudaError_t e = this_device(&dev);
  if (e != cudaSuccess) return e;
  *sms = known[dev].load(std::memory_order_relaxed);
  if (*sms > 0) return cudaSuccess;
  e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess) known[dev].store(*sms, std::memory_order_relaxed);
  return e;
}
template <auto* kernel>
cudaError_t allow_shared(int bytes) {
  static std::atomic<bool> allowed[kMostDevices];
  int dev = 0;
  cudaError_t e = this_device(&dev);
  if (e != cudaSuccess || allowed[dev].load(std::memory_order_relaxed)) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) allowed[dev].store(true, std::memory_order_relaxed);
  return e;
}

constexpr int kStateChunk = 32;   // tokens per block of the states' kernels: one per lane

// A call's sequences. Work is split into pieces of `piece` tokens of one sequence;
// sequence s has the piece numbers from cu[s] / piece + s on: as many as it needs
// fit below the next one's, whatever the lengths, so the number of pieces follows
// from the call's arguments alone and a piece finds its sequence by a search of cu.
struct Seqs {
  const int* cu;
  int num, total, longest;
};
inline long long pieces(int total, int num_seqs, int piece) { return (long long)total / piece + num_seqs; }

struct Piece {
  int t0, t1;  // the sequence's tokens
  int at;      // the piece's index in it
  int seq;
  bool ok;     // there is such a piece
};

// Whether a sequence's bounds make sense; nothing outside [0, total) is ever touched.
__device__ __forceinline__ bool seq_ok(const Seqs& q, int t0, int t1) {
  return t0 >= 0 && t0 <= t1 && t1 <= q.total && t1 - t0 <= q.longest;
}

// By a whole warp: 32 sequences are looked at in one step.
__device__ __forceinline__ Piece find_piece(const Seqs& q, int piece, int index) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = q.num;  // the last sequence whose first piece is not after `index` is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32;
    const int s = lo + lane * step;
    const bool before = s < lo + n && q.cu[s] / piece + s <= index;
    const unsigned int b = __ballot_sync(0xffffffffu, before);
    const int k = b ? 31 - __clz(b) : 0;  // lane 0's sequence is not after it
    n = min(step, n - k * step);
    lo += k * step;
  }
  Piece p;
  p.seq = lo;
  p.t0 = q.cu[lo];
  p.t1 = q.cu[lo + 1];
  p.at = index - (p.t0 / piece + lo);
  p.ok = seq_ok(q, p.t0, p.t1) && p.at >= 0 && p.at < (p.t1 - p.t0 + piece - 1) / piece;
  return p;
}

// By one block of a call: faulty cu_seqlens set their bit. Whether this thread has found any.
__device__ __forceinline__ bool check_seqs(const Seqs& q, unsigned int* error) {
  bool bad = false;
  for (int s = threadIdx.x; s < q.num; s += blockDim.x) bad |= !seq_ok(q, q.cu[s], q.cu[s + 1]);
  if (threadIdx.x == 0) bad |= q.cu[0] != 0 || q.cu[q.num] != q.total;
  if (bad) atomicOr(error, DMC_FAULT_BAD_SEQLENS);
  return bad;
}

// A pair of neighbouring elements in fp32.
template <typename T> struct Pair;
template <> struct Pair<float> {
  using Raw = float2;
  static __device__ __forceinline__ float2 to_f(Raw r) { return r; }
  static __device__ __forceinline__ Raw from_f(float2 f) { return f; }
};
template <> struct Pair<__nv_bfloat16> {
  using Raw = uint32_t;
  static __device__ __forceinline__ float2 to_f(Raw r) {
    float2 f;
    Chunk<__nv_bfloat16>::unpack2(r, f.x, f.y);
    return f;
  }
  static __device__ __forceinline__ Raw from_f(float2 f) { return Chunk<__nv_bfloat16>::pack2(f.x, f.y); }
};

// Four bytes to shared memory, asynchronously; zero unless `valid` (src is a valid address anyway).
__device__ __forceinline__ void cp_async4_zfill(uint32_t dst, const void* src, bool valid) {
  const uint32_t n = valid ? 4u : 0u;
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}

struct StatesArgs {
  Seqs seqs;
  int Hq, Hkv, G;
  const void* q;
  long long q_tok, q_head;
  const void *k, *v;
  const float* noise;
  float offset, temperature;
  float* saved;         // [piece][Hkv][2 D + 4]: sums of k, of v, z before the piece's first token
  unsigned int* error;
  // forward
  void *kt, *vt;
  float *alpha, *bias;
  // backward
  const void *dkt, *dvt, *dbias;
  const float* dalpha;
  void* dq;
  long long dq_tok, dq_head;
  void *dk, *dv;
  // scratch
  uint64_t *sums, *carry;  // [piece][Hkv][2][D + 2]: a piece's own sums; what comes into it (with their launch)
  unsigned int* turns;     // come, gone, number of the launch, of the launch that has to stop
};

struct AttnArgs {
  Seqs seqs;
  int Hq, Hkv, G;
  const void *q, *k, *v;
  const float* bias;
  void* out;
  float* lse;           // [Hq][total]
  const void* dout;
  void *dq, *dk, *dv, *dbias;
  float* rows;          // scratch, per query: see attn_rows_kernel ([Hq][total] deltas for fp32)
  float* sums;          // scratch: sums of shares of a group's queries, see attn_shares
  int shares;
  int* counter;         // work items handed out, CTAs done: zero between launches
  unsigned int* error;
};

// Shares into which the kernels of dK and dV split each group's queries: one, unless the tiles of
// its KV heads (`items`) are fewer than two per SM of this GPU, when the longest item, not the sum
// of all, sets the time; then shares of whole heads. Items of more than one share never exceed
// 4 * 152, so their sums' scratch is bounded. Backward pass in bf16 whole and in shares, us: 600 tokens of
// 64 / 8 heads 113 and 68; 1000 of 40 / 8 113 and 81; 2048 of 32 / 8 177 and 161; 4096 of 64 / 8 932 and
// 769; where it gains least, two sequences of 1024 of 32 / 8, 109 and 111.
constexpr int kSplitItems = 2 * 152;
inline int attn_shares(long long items, int G) {
  if (items >= kSplitItems) return 1;
  const int n = (int)((kSplitItems + items - 1) / items), heads = (G + n - 1) / n;
  return (G + heads - 1) / heads;  // no more than the longest share asks for
}
// Numbers of the shares' sums: 2 D + 1 per row of 128 of each of their items
inline size_t attn_sums(int max_tokens, int Hkv, int G, int D) {
  const size_t all = (size_t)max_tokens * Hkv * G, most = 2 * kSplitItems * 128;
  return G == 1 ? 0 : (all < most ? all : most) * (2 * D + 1);
}

// The shares' sums, to be added up by attn_join_kernel: [share][KV head][token][D] of dV, then of
// dK, then [share][KV head][token] of dbias.
__device__ __forceinline__ float* share_rows(const AttnArgs& a, int D, bool dk, int share, int hk, int token) {
  return a.sums + ((((long long)(dk ? a.shares : 0) + share) * a.Hkv + hk) * a.seqs.total + token) * D;
}
__device__ __forceinline__ float* share_dbias(const AttnArgs& a, int D, int share, int hk) {
  return a.sums + (2ll * a.shares * D * a.Hkv + (long long)share * a.Hkv + hk) * a.seqs.total;
}

struct LossArgs {
  int N, H, V;
  const void *hidden, *weight;
  const int* targets;
  float *loss, *lse;
  const float* dloss;
  void *dhidden, *dweight;
  int piece;            // words of one piece of the backward pass (fp32: of both)
  // scratch
  void* grad;           // [N][piece] in bf16 (fp32: three parts): gradient of a piece's logits
  void *hidden_parts, *weight_parts;  // fp32: [3][N][stride], [3][piece][stride]
  float* dh;            // bf16: [N][H]: dhidden of the pieces so far
  float* sums;          // shares of a gradient's sums: [share][rows][H]
  float *part_m, *part_l;  // [shares][N]: maximum and sum of half a tile of the vocabulary
  float* target_logit;  // [N]
  unsigned int* error;
};

// Words of the largest tile of the vocabulary; a token's maximum and sum are kept for each half of one
constexpr int kLossTile = 256;
// Tiles of 256 x 256 of shares of a gradient's sums: one per pair of SMs of this GPU
constexpr long long kSumTiles = 152 / 2;
// Row length of an fp32 matrix's bf16 parts: rows of multiples of 16 bytes
inline int loss_stride(int H) { return (H + 7) / 8 * 8; }

}  // namespace dmc
