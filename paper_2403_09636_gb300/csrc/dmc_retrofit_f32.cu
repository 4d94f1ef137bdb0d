// Attention of packed sequences in fp32 on the CUDA cores, with its gradients: every product
// and sum in fp32.
//
// All products are built from tiles of 64 x 64 in shared memory, a block of 16 x 16
// threads with 4 rows x 4 (or D / 16) columns each; rows are padded by 16 bytes, so
// that the 16-byte reads of 8 neighbouring rows fall into different banks.
#include <math.h>

#include "dmc_retrofit.cuh"

namespace dmc {

namespace {

constexpr int kT = 64;          // rows of a tile
constexpr int kThreads = 256;
constexpr int kW = kT + 4;      // row of a tile of weights

// rows [r0, r1) of a matrix of D columns into a tile, zero from r1 on
template <int D>
__device__ __forceinline__ void load_rows(float* tile, const float* src, long long stride, int rows) {
  for (int i = threadIdx.x; i < kT * (D / 2); i += kThreads) {
    const int r = i / (D / 2), c = i % (D / 2) * 2;
    float2 f = make_float2(0.f, 0.f);
    if (r < rows) f = *reinterpret_cast<const float2*>(src + r * stride + c);
    *reinterpret_cast<float2*>(tile + r * (D + 4) + c) = f;
  }
}

// acc[i][j] += X[ty + 16 i] . Y[tx + 16 j]
template <int D>
__device__ __forceinline__ void dot_tile(float (&acc)[4][4], const float* X, const float* Y) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll 2
  for (int c = 0; c < D; c += 4) {
    float4 x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float4*>(X + (ty + 16 * i) * (D + 4) + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = *reinterpret_cast<const float4*>(Y + (tx + 16 * i) * (D + 4) + c);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[i][j] = fmaf(x[i].x, y[j].x, acc[i][j]);
        acc[i][j] = fmaf(x[i].y, y[j].y, acc[i][j]);
        acc[i][j] = fmaf(x[i].z, y[j].z, acc[i][j]);
        acc[i][j] = fmaf(x[i].w, y[j].w, acc[i][j]);
      }
  }
}

// acc[i][4 c ..] += sum over r < 64 of W[ty + 16 i][r] Y[r][4 tx + 64 c ..]
template <int D>
__device__ __forceinline__ void sum_tile(float4 (&acc)[4][D / 64], const float* W, const float* Y) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll 2
  for (int r = 0; r < kT; r += 4) {
    float4 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const float4*>(W + (ty + 16 * i) * kW + r);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const float4 y = *reinterpret_cast<const float4*>(Y + (r + k) * (D + 4) + 4 * tx + 64 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = k == 0 ? w[i].x : k == 1 ? w[i].y : k == 2 ? w[i].z : w[i].w;
          acc[i][c].x = fmaf(x, y.x, acc[i][c].x);
          acc[i][c].y = fmaf(x, y.y, acc[i][c].y);
          acc[i][c].z = fmaf(x, y.z, acc[i][c].z);
          acc[i][c].w = fmaf(x, y.w, acc[i][c].w);
        }
      }
  }
}

__device__ __forceinline__ void store4(float* dst, float4 f) { *reinterpret_cast<float4*>(dst) = f; }

__device__ __forceinline__ float4 times(float4 a, float s) { return make_float4(a.x * s, a.y * s, a.z * s, a.w * s); }

// over the 16 threads of a row
__device__ __forceinline__ float row_max(float x) {
#pragma unroll
  for (int off = 8; off >= 1; off >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
  return x;
}
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int off = 8; off >= 1; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
  return x;
}

// ---------------------------------------------------------------- attention

// Whether query i sees row j
__device__ __forceinline__ bool sees(int i, int j, float bias) { return j == i || (j < i && bias != -INFINITY); }

template <int D>
__global__ void __launch_bounds__(kThreads) attn_kernel(const AttnArgs a) {
  extern __shared__ float smem[];
  float *Q = smem, *K = Q + kT * (D + 4), *V = K + kT * (D + 4), *W = V + kT * (D + 4);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, h = blockIdx.y, hk = h / a.G;
  if (blockIdx.x == 0 && h == 0) check_seqs(a.seqs, a.error);
  Piece p = find_piece(a.seqs, kT, blockIdx.x);
  if (!p.ok) return;
  p.at = (p.t1 - p.t0 + kT - 1) / kT - 1 - p.at;  // the longest rows first
  const int i0 = p.t0 + p.at * kT, rows = min(kT, p.t1 - i0);
  const float scale = 1.f / sqrtf((float)D);
  const long long qs = (long long)a.Hq * D, ks = (long long)a.Hkv * D;
  load_rows<D>(Q, static_cast<const float*>(a.q) + (long long)i0 * qs + (long long)h * D, qs, rows);
  float4 acc[4][D / 64] = {};
  float m[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = -INFINITY, l[i] = 0.f;
  for (int j0 = p.t0; j0 <= i0; j0 += kT) {
    const int keys = min(kT, p.t1 - j0);
    __syncthreads();
    load_rows<D>(K, static_cast<const float*>(a.k) + (long long)j0 * ks + (long long)hk * D, ks, keys);
    load_rows<D>(V, static_cast<const float*>(a.v) + (long long)j0 * ks + (long long)hk * D, ks, keys);
    __syncthreads();
    float s[4][4] = {};
    dot_tile<D>(s, Q, K);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int tok = j0 + tx + 16 * j;
      const float b = a.bias && tok < p.t1 ? a.bias[(long long)hk * a.seqs.total + tok] : 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int q = i0 + ty + 16 * i;
        s[i][j] = sees(q, tok, b) ? fmaf(s[i][j], scale, tok < q ? b : 0.f) : -INFINITY;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float mt = row_max(fmaxf(fmaxf(s[i][0], s[i][1]), fmaxf(s[i][2], s[i][3])));
      const float mn = fmaxf(m[i], mt), ref = mn == -INFINITY ? 0.f : mn;
      const float corr = expf(m[i] - ref);
      m[i] = mn;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float w = expf(s[i][j] - ref);
        sum += w;
        W[(ty + 16 * i) * kW + tx + 16 * j] = w;
      }
      l[i] = fmaf(l[i], corr, row_sum(sum));
#pragma unroll
      for (int c = 0; c < D / 64; ++c) acc[i][c] = times(acc[i][c], corr);
    }
    __syncthreads();
    sum_tile<D>(acc, W, V);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = ty + 16 * i;
    if (r >= rows) continue;
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
      store4(static_cast<float*>(a.out) + (long long)(i0 + r) * qs + (long long)h * D + 4 * tx + 64 * c,
             times(acc[i][c], 1.f / l[i]));
    if (tx == 0) a.lse[(long long)h * a.seqs.total + i0 + r] = m[i] + logf(l[i]);
  }
}

// The rows of Q's gradient: dQ_i = scale sum over j of dS_ij k_j, with
// dS = P (dO V^T - delta), delta_i = dO_i . out_i
template <int D>
__global__ void __launch_bounds__(kThreads) attn_dq_kernel(const AttnArgs a) {
  extern __shared__ float smem[];
  float *Q = smem, *O = Q + kT * (D + 4), *K = O + kT * (D + 4), *V = K + kT * (D + 4), *W = V + kT * (D + 4);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, h = blockIdx.y, hk = h / a.G;
  Piece p = find_piece(a.seqs, kT, blockIdx.x);
  if (!p.ok) return;
  p.at = (p.t1 - p.t0 + kT - 1) / kT - 1 - p.at;
  const int i0 = p.t0 + p.at * kT, rows = min(kT, p.t1 - i0);
  const float scale = 1.f / sqrtf((float)D);
  const long long qs = (long long)a.Hq * D, ks = (long long)a.Hkv * D;
  load_rows<D>(Q, static_cast<const float*>(a.q) + (long long)i0 * qs + (long long)h * D, qs, rows);
  load_rows<D>(O, static_cast<const float*>(a.dout) + (long long)i0 * qs + (long long)h * D, qs, rows);
  float lse[4], delta[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long long at = (long long)h * a.seqs.total + i0 + ty + 16 * i;
    const bool in = ty + 16 * i < rows;
    lse[i] = in ? a.lse[at] : 0.f;
    delta[i] = in ? a.rows[at] : 0.f;
  }
  float4 acc[4][D / 64] = {};
  for (int j0 = p.t0; j0 <= i0; j0 += kT) {
    const int keys = min(kT, p.t1 - j0);
    __syncthreads();
    load_rows<D>(K, static_cast<const float*>(a.k) + (long long)j0 * ks + (long long)hk * D, ks, keys);
    load_rows<D>(V, static_cast<const float*>(a.v) + (long long)j0 * ks + (long long)hk * D, ks, keys);
    __syncthreads();
    float s[4][4] = {}, dp[4][4] = {};
    dot_tile<D>(s, Q, K);
    dot_tile<D>(dp, O, V);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int tok = j0 + tx + 16 * j;
      const float b = a.bias && tok < p.t1 ? a.bias[(long long)hk * a.seqs.total + tok] : 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int q = i0 + ty + 16 * i;
        const float w = expf(fmaf(s[i][j], scale, tok < q ? b : 0.f) - lse[i]);
        W[(ty + 16 * i) * kW + tx + 16 * j] = sees(q, tok, b) ? w * (dp[i][j] - delta[i]) : 0.f;
      }
    }
    __syncthreads();
    sum_tile<D>(acc, W, K);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (ty + 16 * i < rows)
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
        store4(static_cast<float*>(a.dq) + (long long)(i0 + ty + 16 * i) * qs + (long long)h * D + 4 * tx + 64 * c,
               times(acc[i][c], scale));
}

// The rows of K's and V's gradients and of the bias's, summed over the queries of the
// group: dV_j = sum of P_ij dO_i, dK_j = scale sum of dS_ij q_i, dbias_j = sum over i > j of dS_ij
template <int D>
__global__ void __launch_bounds__(kThreads) attn_dkv_kernel(const AttnArgs a) {
  extern __shared__ float smem[];
  float *K = smem, *V = K + kT * (D + 4), *Q = V + kT * (D + 4), *O = Q + kT * (D + 4), *W = O + kT * (D + 4);
  float *S = W + kT * kW, *L = S + kT * kW, *E = L + kT;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, hk = blockIdx.y;
  const Piece p = find_piece(a.seqs, kT, blockIdx.x);
  if (!p.ok) return;
  const int j0 = p.t0 + p.at * kT, keys = min(kT, p.t1 - j0);
  const float scale = 1.f / sqrtf((float)D);
  const long long qs = (long long)a.Hq * D, ks = (long long)a.Hkv * D;
  load_rows<D>(K, static_cast<const float*>(a.k) + (long long)j0 * ks + (long long)hk * D, ks, keys);
  load_rows<D>(V, static_cast<const float*>(a.v) + (long long)j0 * ks + (long long)hk * D, ks, keys);
  float bias[4], db[4] = {};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = ty + 16 * j;
    bias[j] = a.bias && r < keys ? a.bias[(long long)hk * a.seqs.total + j0 + r] : 0.f;
  }
  float4 dk[4][D / 64] = {}, dv[4][D / 64] = {};
  for (int g = 0; g < a.G; ++g) {
    const int h = hk * a.G + g;
    for (int i0 = j0; i0 < p.t1; i0 += kT) {
      const int rows = min(kT, p.t1 - i0);
      __syncthreads();
      load_rows<D>(Q, static_cast<const float*>(a.q) + (long long)i0 * qs + (long long)h * D, qs, rows);
      load_rows<D>(O, static_cast<const float*>(a.dout) + (long long)i0 * qs + (long long)h * D, qs, rows);
      if (threadIdx.x < kT) {
        const long long at = (long long)h * a.seqs.total + i0 + threadIdx.x;
        const bool in = (int)threadIdx.x < rows;
        L[threadIdx.x] = in ? a.lse[at] : 0.f;
        E[threadIdx.x] = in ? a.rows[at] : 0.f;
      }
      __syncthreads();
      float s[4][4] = {}, dp[4][4] = {};
      dot_tile<D>(s, K, Q);
      dot_tile<D>(dp, V, O);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int tok = j0 + ty + 16 * j, r = tx + 16 * i, q = i0 + r;
          const bool seen = r < rows && sees(q, tok, bias[j]);
          const float w = seen ? expf(fmaf(s[j][i], scale, tok < q ? bias[j] : 0.f) - L[r]) : 0.f;
          const float ds = seen ? w * (dp[j][i] - E[r]) : 0.f;
          W[(ty + 16 * j) * kW + r] = w;
          S[(ty + 16 * j) * kW + r] = ds;
          if (tok < q) db[j] += ds;
        }
      __syncthreads();
      sum_tile<D>(dv, W, O);
      sum_tile<D>(dk, S, Q);
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = ty + 16 * j;
    const float b = row_sum(db[j]);
    if (r >= keys) continue;
    const long long at = (long long)(j0 + r) * ks + (long long)hk * D;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      store4(static_cast<float*>(a.dk) + at + 4 * tx + 64 * c, times(dk[j][c], scale));
      store4(static_cast<float*>(a.dv) + at + 4 * tx + 64 * c, dv[j][c]);
    }
    if (tx == 0 && a.dbias) static_cast<float*>(a.dbias)[(long long)hk * a.seqs.total + j0 + r] = b;
  }
}

// delta_i = dO_i . out_i, a warp per (token, head)
template <int D>
__global__ void __launch_bounds__(256) attn_delta_kernel(const AttnArgs a) {
  const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (blockIdx.x == 0) check_seqs(a.seqs, a.error);
  if (w >= (long long)a.seqs.total * a.Hq) return;
  float d = 0.f;
#pragma unroll
  for (int c = 2 * lane; c < D; c += 64) {
    const float2 x = *reinterpret_cast<const float2*>(static_cast<const float*>(a.out) + w * D + c);
    const float2 y = *reinterpret_cast<const float2*>(static_cast<const float*>(a.dout) + w * D + c);
    d = fmaf(x.x, y.x, fmaf(x.y, y.y, d));
  }
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) d += __shfl_xor_sync(0xffffffffu, d, off);
  if (lane == 0) a.rows[(w % a.Hq) * a.seqs.total + w / a.Hq] = d;
}

template <typename K>
cudaError_t allow(K* kernel, size_t bytes) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <int D>
cudaError_t attn_f(const AttnArgs& a, cudaStream_t stream) {
  constexpr size_t bytes = (3 * kT * (D + 4) + kT * kW) * 4;
  cudaError_t e = allow(attn_kernel<D>, bytes);
  if (e != cudaSuccess) return e;
  attn_kernel<D><<<dim3((unsigned)pieces(a.seqs.total, a.seqs.num, kT), a.Hq), kThreads, bytes, stream>>>(a);
  return cudaGetLastError();
}

template <int D>
cudaError_t attn_b(const AttnArgs& a, cudaStream_t stream) {
  constexpr size_t dq = (4 * kT * (D + 4) + kT * kW) * 4, dkv = (4 * kT * (D + 4) + 2 * kT * kW + 2 * kT) * 4;
  cudaError_t e = allow(attn_dq_kernel<D>, dq);
  if (e == cudaSuccess) e = allow(attn_dkv_kernel<D>, dkv);
  if (e != cudaSuccess) return e;
  const unsigned n = (unsigned)pieces(a.seqs.total, a.seqs.num, kT);
  attn_delta_kernel<D><<<(unsigned)(((long long)a.seqs.total * a.Hq + 7) / 8), 256, 0, stream>>>(a);
  attn_dkv_kernel<D><<<dim3(n, a.Hkv), kThreads, dkv, stream>>>(a);
  attn_dq_kernel<D><<<dim3(n, a.Hq), kThreads, dq, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t attn_forward_f32(const AttnArgs& a, int D, cudaStream_t stream) {
  return D == 128 ? attn_f<128>(a, stream) : attn_f<64>(a, stream);
}
cudaError_t attn_backward_f32(const AttnArgs& a, int D, cudaStream_t stream) {
  return D == 128 ? attn_b<128>(a, stream) : attn_b<64>(a, stream);
}

}  // namespace dmc
