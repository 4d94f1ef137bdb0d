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
constexpr int kRowsInFlight = 4;  // of a thread

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
  bool prompt;     // the launch between the plan and the scan of a prompt that is appended
  float* weights;  // or null: omega of every token and KV head, where the scan looks for it
  int group;       // queries per KV head
};

// The sequence of token t, and its place there; false if it is of none (before the first or behind the last).
__device__ __forceinline__ bool sequence(const RotateArgs& a, int t, int& s, int& at) {
  int lo = 0, hi = a.seqs - 1;  // the last sequence that begins at t or before
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.cu[mid] <= t) lo = mid; else hi = mid - 1;
  }
  s = lo;
  at = t - a.cu[lo];
  return at >= 0 && t < a.cu[lo + 1];
}

// Turns of two pairs at a time, (cos, cos, sin, sin); thread p of a row needs places i * P + p (i = 0 .. E / 2 - 1: one
// 128-byte line of shared memory for a row's threads at a time).
template <typename T, int D>
__global__ void __launch_bounds__(kRotateThreads, 3) dmc_rotate_kernel(const RotateArgs a) {
  using CK = Chunk<T>;
  constexpr int E = CK::N, ROW = D * (int)sizeof(T), P = ROW / 32;  // threads per row
  __shared__ __align__(16) float4 cs[kRotateTokens][D / 4];
  __shared__ int s_seq[kRotateTokens], s_place[kRotateTokens];  // a token's sequence (-1: of none), and its place there
  if (a.prompt) griddep_launch_dependents();
  const int t0 = blockIdx.x * a.per, n = min(a.per, a.tokens - t0);
  const int p = threadIdx.x % P, all = a.heads[0] + a.heads[1];
  constexpr int kStep = kRotateThreads / P, U = kRowsInFlight;
  const int rows = n * all, step = gridDim.y * kStep;
  bool ready = false;
  int r = blockIdx.y * kStep + threadIdx.x / P;  // the thread's next row: head h of the block's token t
  int t = r / all, h = r % all;
  for (int r0 = blockIdx.y * kStep; r0 < rows; r0 += U * step) {
    uint4 lo[U], hi[U];
    char* to[U];
    int token[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      to[u] = nullptr;
      if (r < rows) {
        const bool key = h >= a.heads[0];  // (chosen field by field: the arguments stay where they are)
        const size_t off = (size_t)(h - (key ? a.heads[0] : 0)) * ROW + p * 16;
        const char* from = (key ? a.x[1] : a.x[0]) + (size_t)(t0 + t) * (key ? a.x_stride[1] : a.x_stride[0]) + off;
        to[u] = (key ? a.y[1] : a.y[0]) + (size_t)(t0 + t) * (key ? a.y_stride[1] : a.y_stride[0]) + off;
        token[u] = t;
        lo[u] = *reinterpret_cast<const uint4*>(from);
        hi[u] = *reinterpret_cast<const uint4*>(from + ROW / 2);
      }
      r += step;
      h += step;
      while (h >= all) {
        h -= all;
        ++t;
      }
    }
    if (!ready) {  // the tokens' turns (and omegas), while the first rows are on their way
      for (int i = threadIdx.x; i < n * (D / 2); i += kRotateThreads) {
        const int pair = i % (D / 2), q = pair / 2, tt = i / (D / 2);
        long long pos;
        if (a.cu == nullptr) {
          pos = a.at[t0 + tt];
        } else {
          int s, at;
          const bool any = sequence(a, t0 + tt, s, at);
          pos = (long long)a.at[s] + at;
          if (pair == 0) {
            s_seq[tt] = any ? s : -1;
            s_place[tt] = at;
          }
        }
        float2 c = turn_of(turns_of_pair(a.turns, pair), pos);
        if (a.back) c.y = -c.y;
        // (paired as neighbours, a thread's pairs are E / 4 twos of either half of the row)
        constexpr int C = E / 4;
        const int half = a.pairs && q >= D / 8, qq = q - half * (D / 8), per = a.pairs ? C : 2 * C;
        float* to4 = reinterpret_cast<float*>(&cs[tt][(half * C + qq % per) * P + qq / per]) + (pair & 1);
        to4[0] = c.x;
        to4[2] = c.y;
      }
      __syncthreads();
      ready = true;
      if (a.weights != nullptr && blockIdx.y == 0) {
        // omega = sigmoid(mean of the group's q[0]), of rows that are on their way in any case (in place, too: a gate is
        // only ever written as it is)
        const int H = a.heads[0] / a.group;
        for (int i = threadIdx.x; i < n * H; i += kRotateThreads) {
          const int tt = i / H, hk = i % H, s = s_seq[tt], at = s_place[tt];
          if (s < 0) continue;
          const char* q0 = a.x[0] + (size_t)(t0 + tt) * a.x_stride[0] + (size_t)hk * a.group * ROW;
          float g = 0.f;
          for (int x = 0; x < a.group; ++x) g += Elt<T>::to_f(*reinterpret_cast<const T*>(q0 + (size_t)x * ROW));
          a.weights[((size_t)prompt_chunk(t0 + tt - at, at / kPrefillChunk, s) * H + hk) * kPrefillChunk +
                    at % kPrefillChunk] = sigmoidf_(g / (float)a.group);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (to[u] == nullptr || (a.cu != nullptr && s_seq[token[u]] < 0)) continue;
      float x[E], y[E];
      CK::unpack(lo[u], x);
      CK::unpack(hi[u], y);
      const float x0 = x[0], x1 = a.pairs ? x[1] : y[0];  // the gate's pair, where p is 0
#pragma unroll
      for (int i = 0; i < E / 2; ++i) {
        const float4 w = cs[token[u]][i * P + p];
        const float2 c = make_float2(w.x, w.y), s = make_float2(w.z, w.w), m = make_float2(-w.z, -w.w);
        float2 f, g;  // the two pairs' first and second dims
        if (a.pairs) {
          float* v = i < E / 4 ? x + 4 * i : y + 4 * (i - E / 4);
          f = make_float2(v[0], v[2]);
          g = make_float2(v[1], v[3]);
          const float2 fn = fma2(g, m, mul2(f, c)), gn = fma2(f, s, mul2(g, c));
          v[0] = fn.x; v[2] = fn.y; v[1] = gn.x; v[3] = gn.y;
        } else {
          f = make_float2(x[2 * i], x[2 * i + 1]);
          g = make_float2(y[2 * i], y[2 * i + 1]);
          const float2 fn = fma2(g, m, mul2(f, c)), gn = fma2(f, s, mul2(g, c));
          x[2 * i] = fn.x; x[2 * i + 1] = fn.y; y[2 * i] = gn.x; y[2 * i + 1] = gn.y;
        }
      }
      if (p == 0) {  // (turned by zero, a gate that is infinite would make its partner NaN)
        x[0] = x0;
        if (a.pairs) x[1] = x1; else y[0] = x1;
      }
      *reinterpret_cast<uint4*>(to[u]) = CK::pack(x);
      *reinterpret_cast<uint4*>(to[u] + ROW / 2) = CK::pack(y);
    }
  }
  if (a.prompt) griddep_wait();  // the scan after this waits for the plan before it, too
}

}  // namespace

static cudaError_t launch_rotate(RotateArgs& a, int esize, int D, cudaStream_t stream) {
  // A block takes about as many rows as its threads have in flight: several tokens of few heads, or one token's heads
  // in parts (the turns of a token are then computed for each part). 8192 tokens of 32 + 32 heads of 128 in bf16 take
  // 41.4 us so (6.5 TB/s); 456 blocks, as many as run at once, of 18 tokens and with the next rows on their way while some
  // are worked, 45.9. Few rows in all go one to a thread's place instead, for latency: us of 512, 2048, 6144, 12,288 and
  // 32,768 rows so / with several in flight: 32 + 32 heads of 128 in bf16 2.3 / 3.0, 2.5 / 3.3, 2.8 / 3.4, 3.1 / 3.4,
  // 6.8 / 5.5; 64 + 8 2.5 / 2.8, 2.6 / 3.0, 2.8 / 3.0, 3.9 / 3.4, 7.2 / 5.2; 8 + 8 in fp32 2.5 / 3.2, 2.6 / 3.3, 3.0 / 3.3,
  // 4.9 / 4.6, 10.2 / 8.6.
  const int at_once = kRotateThreads / (D * esize / 32), all = a.heads[0] + a.heads[1];
  const bool few = (long long)a.tokens * all < 8192;
  a.per = few ? 1 : max(1, min(kRotateTokens, at_once * kRowsInFlight / all));
  const int blocks = ceil_div(a.tokens, a.per);
  const int parts = max(1, ceil_div(all, few ? at_once : at_once * kRowsInFlight));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks, parts);
  cfg.blockDim = dim3(kRotateThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.prompt ? 1 : 0;
  cudaError_t e = cudaErrorInvalidValue;
  if (esize == 4 && D == 64) e = cudaLaunchKernelEx(&cfg, dmc_rotate_kernel<float, 64>, a);
  if (esize == 4 && D == 128) e = cudaLaunchKernelEx(&cfg, dmc_rotate_kernel<float, 128>, a);
  if (esize == 2 && D == 64) e = cudaLaunchKernelEx(&cfg, dmc_rotate_kernel<__nv_bfloat16, 64>, a);
  if (esize == 2 && D == 128) e = cudaLaunchKernelEx(&cfg, dmc_rotate_kernel<__nv_bfloat16, 128>, a);
  return e != cudaSuccess ? e : cudaGetLastError();
}

// The queries of a prompt that is appended, whose sequences begin at the positions `at`: launched between the plan and
// the scan, beside the first of which it runs. weights: as in RotateArgs.
cudaError_t rotate_prompt_launch(const Layout& L, int num_seqs, int total_tokens, const void* q, void* q_out, const int* cu,
                                 const int* at, const unsigned long long* turns, bool pairs, float* weights,
                                 cudaStream_t stream) {
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
  a.prompt = true;
  a.weights = weights;
  a.group = L.G;
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
