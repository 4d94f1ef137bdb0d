// The position rotation alone, of queries and keys in one launch (training, and prompts whose attention reads rotated
// rows). Its gradient is the same with the opposite turn.
//
// Every row is read and written once: bound by HBM. A thread takes 16 bytes of the first and 16 of the second half of a
// row, which hold whole pairs in both ways of pairing; the block's tokens' turns are computed once, into shared memory,
// for all of their heads.
#include "dmc_rotary.cuh"

namespace dmc {

namespace {

constexpr int kRotateThreads = 256;
constexpr int kRotateTokens = 4;  // most tokens of a block

struct RotateArgs {
  int tokens, per;  // per block
  int heads[2];
  const char* x[2];
  char* y[2];
  long long x_stride[2], y_stride[2];  // bytes between tokens
  const int* at;  // a token's position, or with cu that of its sequence's first token
  const int* cu;
  int seqs;
  const unsigned long long* turns;
  bool pairs, back;
};

__device__ __forceinline__ long long position(const RotateArgs& a, int t) {
  if (a.cu == nullptr) return a.at[t];
  int lo = 0, hi = a.seqs - 1;  // the last sequence that begins at t or before
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.cu[mid] <= t) lo = mid; else hi = mid - 1;
  }
  return (long long)a.at[lo] + (t - a.cu[lo]);
}

template <typename T, int D>
__global__ void __launch_bounds__(kRotateThreads) dmc_rotate_kernel(const RotateArgs a) {
  using CK = Chunk<T>;
  constexpr int E = CK::N, ROW = D * (int)sizeof(T), P = ROW / 32;  // threads per row
  __shared__ __align__(16) float2 cs[kRotateTokens][D / 2];
  const int t0 = blockIdx.x * a.per, n = min(a.per, a.tokens - t0);
  for (int i = threadIdx.x; i < n * (D / 2); i += kRotateThreads) {
    const int pair = i % (D / 2);
    float2 c = turn_of(turns_of_pair(a.turns, pair), position(a, t0 + i / (D / 2)));
    if (a.back) c.y = -c.y;
    cs[i / (D / 2)][pair] = c;
  }
  __syncthreads();
  const int p = threadIdx.x % P, all = a.heads[0] + a.heads[1];
  constexpr int kStep = kRotateThreads / P, U = 2;  // rows of the block at a time, of a thread in flight
  const int rows = n * all, first = blockIdx.y * kStep + threadIdx.x / P, step = gridDim.y * kStep;
  for (int r0 = first; r0 < rows; r0 += U * step) {
    uint4 lo[U], hi[U];
    char* to[U];
    int token[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * step;
      if (r >= rows) break;
      const int h = r % all, which = h >= a.heads[0];
      token[u] = r / all;
      const size_t off = (size_t)(h - (which ? a.heads[0] : 0)) * ROW + p * 16;
      const char* from = a.x[which] + (size_t)(t0 + token[u]) * a.x_stride[which] + off;
      to[u] = a.y[which] + (size_t)(t0 + token[u]) * a.y_stride[which] + off;
      lo[u] = *reinterpret_cast<const uint4*>(from);
      hi[u] = *reinterpret_cast<const uint4*>(from + ROW / 2);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (r0 + u * step >= rows) break;
      float x[E], y[E];
      CK::unpack(lo[u], x);
      CK::unpack(hi[u], y);
      const float2* c = cs[token[u]];
      const float x0 = x[0], x1 = a.pairs ? x[1] : y[0];  // the gate's pair, where p is 0
      if (a.pairs) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
          turn(c[p * (E / 2) + i], x[2 * i], x[2 * i + 1]);
          turn(c[D / 4 + p * (E / 2) + i], y[2 * i], y[2 * i + 1]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) turn(c[p * E + i], x[i], y[i]);
      }
      if (p == 0) {  // (turned by zero, a gate that is infinite would make its partner NaN)
        x[0] = x0;
        if (a.pairs) x[1] = x1; else y[0] = x1;
      }
      *reinterpret_cast<uint4*>(to[u]) = CK::pack(x);
      *reinterpret_cast<uint4*>(to[u] + ROW / 2) = CK::pack(y);
    }
  }
}

}  // namespace

static cudaError_t launch_rotate(RotateArgs& a, int esize, int D, cudaStream_t stream) {
  // few tokens: their heads are spread over blocks, too
  const int rows_at_once = kRotateThreads / (D * esize / 32);
  a.per = a.tokens >= 1024 ? kRotateTokens : 1;
  const dim3 grid(ceil_div(a.tokens, a.per), a.tokens >= 1024 ? 1 : ceil_div(a.heads[0] + a.heads[1], rows_at_once));
  if (esize == 4 && D == 64) dmc_rotate_kernel<float, 64><<<grid, kRotateThreads, 0, stream>>>(a);
  else if (esize == 4 && D == 128) dmc_rotate_kernel<float, 128><<<grid, kRotateThreads, 0, stream>>>(a);
  else if (esize == 2 && D == 64) dmc_rotate_kernel<__nv_bfloat16, 64><<<grid, kRotateThreads, 0, stream>>>(a);
  else if (esize == 2 && D == 128) dmc_rotate_kernel<__nv_bfloat16, 128><<<grid, kRotateThreads, 0, stream>>>(a);
  else return cudaErrorInvalidValue;
  return cudaGetLastError();
}

// The queries of a prompt, whose sequences begin at the positions `at`.
cudaError_t rotate_prompt_launch(const Layout& L, int num_seqs, int total_tokens, const void* q, void* q_out, const int* cu,
                                 const int* at, const unsigned long long* turns, bool pairs, cudaStream_t stream) {
  RotateArgs a = {};
  a.tokens = total_tokens;
  a.heads[0] = L.Hq;
  a.x[0] = static_cast<const char*>(q);
  a.y[0] = static_cast<char*>(q_out);
  a.x_stride[0] = a.y_stride[0] = (long long)L.Hq * L.row_bytes;
  a.at = at;
  a.cu = cu;
  a.seqs = num_seqs;
  a.turns = turns;
  a.pairs = pairs;
  return launch_rotate(a, L.esize, L.D, stream);
}

}  // namespace dmc

extern "C" dmc_status dmc_rotate(int32_t dtype, int32_t head_dim, int32_t num_tokens, const int32_t* positions_dev,
                                 const uint64_t* turns_dev, int32_t interleaved, int32_t inverse, int32_t num_q_heads,
                                 const void* q_dev, int64_t q_token_stride, void* q_out_dev, int64_t q_out_token_stride,
                                 int32_t num_k_heads, const void* k_dev, int64_t k_token_stride, void* k_out_dev,
                                 int64_t k_out_token_stride, cudaStream_t stream) {
  if ((dtype != DMC_F32 && dtype != DMC_BF16) || (head_dim != 64 && head_dim != 128) || num_tokens < 0 ||
      num_q_heads < 0 || num_k_heads < 0 || num_q_heads > 65536 || num_k_heads > 65536)
    return DMC_ERR_INVALID_ARG;
  if (num_tokens == 0 || num_q_heads + num_k_heads == 0) return DMC_OK;
  const int esize = dtype == DMC_F32 ? 4 : 2;
  if (!positions_dev || !turns_dev || (reinterpret_cast<uintptr_t>(positions_dev) & 3u) ||
      (reinterpret_cast<uintptr_t>(turns_dev) & 7u))
    return DMC_ERR_INVALID_ARG;
  dmc::RotateArgs a = {};
  a.tokens = num_tokens;
  a.heads[0] = num_q_heads;
  a.heads[1] = num_k_heads;
  a.x[0] = static_cast<const char*>(q_dev);
  a.x[1] = static_cast<const char*>(k_dev);
  a.y[0] = static_cast<char*>(q_out_dev);
  a.y[1] = static_cast<char*>(k_out_dev);
  const int64_t in[2] = {q_token_stride, k_token_stride}, out[2] = {q_out_token_stride, k_out_token_stride};
  for (int i = 0; i < 2; ++i) {
    if (a.heads[i] == 0) continue;
    const int64_t row = (int64_t)a.heads[i] * head_dim, most = (int64_t)1 << 40;
    const uintptr_t bits = reinterpret_cast<uintptr_t>(a.x[i]) | reinterpret_cast<uintptr_t>(a.y[i]);
    if (!a.x[i] || !a.y[i] || (bits & 15u) || in[i] < row || out[i] < row || in[i] > most || out[i] > most ||
        (in[i] * esize & 15) || (out[i] * esize & 15) || (a.x[i] == a.y[i] && in[i] != out[i]))
      return DMC_ERR_INVALID_ARG;
    a.x_stride[i] = in[i] * esize;
    a.y_stride[i] = out[i] * esize;
  }
  a.at = positions_dev;
  a.turns = reinterpret_cast<const unsigned long long*>(turns_dev);
  a.pairs = interleaved != 0;
  a.back = inverse != 0;
  return dmc::launch_rotate(a, esize, head_dim, stream) == cudaSuccess ? DMC_OK : DMC_ERR_CUDA;
}
