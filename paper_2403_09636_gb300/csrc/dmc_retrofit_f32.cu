// Attention of packed sequences in fp32 on the CUDA cores, with its gradients, every product and
// sum in fp32: for calls of few rows, and the choice between these kernels and those of
// dmc_retrofit_parts.cu.
//
// All products are built from tiles of 32 rows in shared memory, by a block of 16 columns of
// threads; a thread takes every 16th column (two of them) and every 8th row (four). Rows are
// padded by 16 bytes, so that the 16-byte reads of 8 neighbouring rows fall into different banks.
// Multiply-adds come in pairs (fma.rn.f32x2), two neighbouring terms of a sum or two
// neighbouring columns, which leaves issue slots for the reads.
// Where SMs are left without a block, a block's steps one after another set the time: so small
// tiles, the next step's on their way meanwhile, dQ in one launch with dK and dV, and
// those in shares of a group's heads (attn_shares); products unrolled as a whole, whose reads then run
// ahead. 256 tokens of 4 heads of 64: forward 21 us, backward 31 (25 and 35 unrolled by 4 and 2; 26 and 63 in
// two launches without tiles ahead); 500 tokens of 32 / 8 heads of 128: backward 290 (280 by 4 and 2, 532 with
// whole groups). 256 threads per block were no faster (24 and 38, 731).
#include <math.h>

#include "dmc_retrofit.cuh"

namespace dmc {
cudaError_t attn_join(const AttnArgs& a, bool bf16, int D, cudaStream_t stream);
cudaError_t attn_forward_parts(const AttnArgs& a, int D, cudaStream_t stream);
cudaError_t attn_backward_parts(const AttnArgs& a, int D, cudaStream_t stream);

namespace {

constexpr int kT = 32;                  // rows of a tile
constexpr int kThreads = 128;
constexpr int kI = kT * 16 / kThreads;  // rows of a thread
constexpr int kJ = kT / 16;             // columns of a thread
constexpr int kTy = kThreads / 16;
constexpr int kW = kT + 4;              // row of a tile of weights

// `rows` rows of D columns, asynchronously, into a tile; zero from there on
template <int D>
__device__ __forceinline__ void load_rows(float* tile, const float* src, long long stride, int rows) {
#pragma unroll
  for (int i = threadIdx.x; i < kT * (D / 4); i += kThreads) {
    const int r = i / (D / 4), c = i % (D / 4) * 4;
    cp_async16_zfill(smem_u32(tile + r * (D + 4) + c), src + (r < rows ? r * stride : 0) + c, r < rows);
  }
}

// acc[i][j] += X[ty + kTy i] . Y[tx + 16 j], even and odd terms apart
template <int D>
__device__ __forceinline__ void dot_tile(float2 (&acc)[kI][kJ], const float* X, const float* Y) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int c = 0; c < D; c += 4) {
    float4 x[kI], y[kJ];
#pragma unroll
    for (int i = 0; i < kI; ++i) x[i] = *reinterpret_cast<const float4*>(X + (ty + kTy * i) * (D + 4) + c);
#pragma unroll
    for (int j = 0; j < kJ; ++j) y[j] = *reinterpret_cast<const float4*>(Y + (tx + 16 * j) * (D + 4) + c);
#pragma unroll
    for (int i = 0; i < kI; ++i)
#pragma unroll
      for (int j = 0; j < kJ; ++j) {
        acc[i][j] = fma2(make_float2(x[i].x, x[i].y), make_float2(y[j].x, y[j].y), acc[i][j]);
        acc[i][j] = fma2(make_float2(x[i].z, x[i].w), make_float2(y[j].z, y[j].w), acc[i][j]);
      }
  }
}

// acc[i][2 c], acc[i][2 c + 1] (columns 4 tx + 64 c ..) += sum over r < kT of W[ty + kTy i][r] Y[r][.]
template <int D>
__device__ __forceinline__ void sum_tile(float2 (&acc)[kI][D / 32], const float* W, const float* Y) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int r = 0; r < kT; r += 4) {
    float4 w[kI];
#pragma unroll
    for (int i = 0; i < kI; ++i) w[i] = *reinterpret_cast<const float4*>(W + (ty + kTy * i) * kW + r);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const float4 y = *reinterpret_cast<const float4*>(Y + (r + k) * (D + 4) + 4 * tx + 64 * c);
#pragma unroll
        for (int i = 0; i < kI; ++i) {
          const float x = k == 0 ? w[i].x : k == 1 ? w[i].y : k == 2 ? w[i].z : w[i].w;
          acc[i][2 * c] = fma2(make_float2(x, x), make_float2(y.x, y.y), acc[i][2 * c]);
          acc[i][2 * c + 1] = fma2(make_float2(x, x), make_float2(y.z, y.w), acc[i][2 * c + 1]);
        }
      }
  }
}

template <int D>
__device__ __forceinline__ void store_row(float* dst, const float2 (&f)[D / 32], float scale) {
  const int tx = threadIdx.x & 15;
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
    *reinterpret_cast<float4*>(dst + 4 * tx + 64 * c) =
        make_float4(f[2 * c].x * scale, f[2 * c].y * scale, f[2 * c + 1].x * scale, f[2 * c + 1].y * scale);
}

template <int I, int J>
__device__ __forceinline__ void clear(float2 (&x)[I][J]) {
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int j = 0; j < J; ++j) x[i][j] = make_float2(0.f, 0.f);
}

__device__ __forceinline__ float sum2(float2 x) { return x.x + x.y; }

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

// Tiles of step n, by `load(n)`: those of the next step are asked for here, once all threads
// are through with the step before.
template <typename Load>
__device__ __forceinline__ void stage_tiles(int n, int steps, const Load& load) {
  __syncthreads();  // the step before has read its tiles
  if (n == 0) {
    load(0);
    cp_async_commit();
  }
  if (n + 1 < steps) {
    load(n + 1);
    cp_async_commit();
    cp_async_wait<1>();
  } else {
    cp_async_wait<0>();
  }
  __syncthreads();
}

// Whether query i sees row j
__device__ __forceinline__ bool sees(int i, int j, float bias) { return j == i || (j < i && bias != -INFINITY); }

// of `own` tiles of the block's rows, two staged ones and two numbers of their rows, and weights
template <int D>
constexpr size_t tiles_bytes(int own, int weights) {
  return ((size_t)(own + 4) * kT * (D + 4) + (size_t)weights * kT * kW + 4 * kT) * 4;
}

// Weights take K's place once the scores are there.
template <int D>
__global__ void __launch_bounds__(kThreads, 2) attn_kernel(const AttnArgs a) {
  extern __shared__ float smem[];
  constexpr int kTile = kT * (D + 4);
  float* Q = smem;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, h = blockIdx.y, hk = h / a.G;
  if (blockIdx.x == 0 && h == 0) check_seqs(a.seqs, a.error);
  Piece p = find_piece(a.seqs, kT, blockIdx.x);
  if (!p.ok) return;
  p.at = (p.t1 - p.t0 + kT - 1) / kT - 1 - p.at;  // the longest rows first
  const int i0 = p.t0 + p.at * kT, rows = min(kT, p.t1 - i0);
  const float scale = 1.f / sqrtf((float)D);
  const long long qs = (long long)a.Hq * D, ks = (long long)a.Hkv * D;
  const float *k = static_cast<const float*>(a.k) + (long long)hk * D, *v = static_cast<const float*>(a.v) + (long long)hk * D;
  load_rows<D>(Q, static_cast<const float*>(a.q) + (long long)i0 * qs + (long long)h * D, qs, rows);
  float2 acc[kI][D / 32];
  clear(acc);
  float m[kI], l[kI];
#pragma unroll
  for (int i = 0; i < kI; ++i) m[i] = -INFINITY, l[i] = 0.f;
  const int steps = p.at + 1;
  auto load = [&](int n) {
    float* K = smem + (1 + (n & 1) * 2) * kTile;
    const int j0 = p.t0 + n * kT, keys = min(kT, p.t1 - j0);
    load_rows<D>(K, k + j0 * ks, ks, keys);
    load_rows<D>(K + kTile, v + j0 * ks, ks, keys);
  };
  float next_b[kJ];
  auto load_bias = [&](int n) {
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      const int tok = p.t0 + n * kT + tx + 16 * j;
      next_b[j] = a.bias && tok < p.t1 ? a.bias[(long long)hk * a.seqs.total + tok] : 0.f;
    }
  };
  load_bias(0);
  for (int n = 0; n < steps; ++n) {
    const int j0 = p.t0 + n * kT;
    float *K = smem + (1 + (n & 1) * 2) * kTile, *V = K + kTile, *W = K;
    float b[kJ];
#pragma unroll
    for (int j = 0; j < kJ; ++j) b[j] = next_b[j];
    stage_tiles(n, steps, load);
    load_bias(n + 1);
    float2 s2[kI][kJ];
    clear(s2);
    dot_tile<D>(s2, Q, K);
    __syncthreads();  // K has been read
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      const int q = i0 + ty + kTy * i;
      float s[kJ], mt = -INFINITY;
#pragma unroll
      for (int j = 0; j < kJ; ++j) {
        const int tok = j0 + tx + 16 * j;
        s[j] = sees(q, tok, b[j]) ? fmaf(sum2(s2[i][j]), scale, tok < q ? b[j] : 0.f) : -INFINITY;
        mt = fmaxf(mt, s[j]);
      }
      const float mn = fmaxf(m[i], row_max(mt)), ref = mn == -INFINITY ? 0.f : mn;
      const float corr = expf(m[i] - ref);
      m[i] = mn;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < kJ; ++j) {
        const float w = expf(s[j] - ref);
        sum += w;
        W[(ty + kTy * i) * kW + tx + 16 * j] = w;
      }
      l[i] = fmaf(l[i], corr, row_sum(sum));
#pragma unroll
      for (int c = 0; c < D / 32; ++c) acc[i][c] = mul2(acc[i][c], make_float2(corr, corr));
    }
    __syncthreads();
    sum_tile<D>(acc, W, V);
  }
#pragma unroll
  for (int i = 0; i < kI; ++i) {
    const int r = ty + kTy * i;
    if (r >= rows) continue;
    store_row<D>(static_cast<float*>(a.out) + (long long)(i0 + r) * qs + (long long)h * D, acc[i], 1.f / l[i]);
    if (tx == 0) a.lse[(long long)h * a.seqs.total + i0 + r] = m[i] + logf(l[i]);
  }
}

// The rows of Q's gradient: dQ_i = scale sum over j of dS_ij k_j, with
// dS = P (dO V^T - delta), delta_i = dO_i . out_i. Weights take V's place.
template <int D>
__device__ __forceinline__ void dq_rows(const AttnArgs& a, int h, float* smem) {
  constexpr int kTile = kT * (D + 4);
  float *Q = smem, *O = Q + kTile;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, hk = h / a.G;
  Piece p = find_piece(a.seqs, kT, blockIdx.x);
  if (!p.ok) return;
  p.at = (p.t1 - p.t0 + kT - 1) / kT - 1 - p.at;
  const int i0 = p.t0 + p.at * kT, rows = min(kT, p.t1 - i0);
  const float scale = 1.f / sqrtf((float)D);
  const long long qs = (long long)a.Hq * D, ks = (long long)a.Hkv * D, at = (long long)i0 * qs + (long long)h * D;
  const float *k = static_cast<const float*>(a.k) + (long long)hk * D, *v = static_cast<const float*>(a.v) + (long long)hk * D;
  load_rows<D>(Q, static_cast<const float*>(a.q) + at, qs, rows);
  load_rows<D>(O, static_cast<const float*>(a.dout) + at, qs, rows);
  float lse[kI], delta[kI];
#pragma unroll
  for (int i = 0; i < kI; ++i) {
    const long long n = (long long)h * a.seqs.total + i0 + ty + kTy * i;
    const bool in = ty + kTy * i < rows;
    lse[i] = in ? a.lse[n] : 0.f;
    delta[i] = in ? a.rows[n] : 0.f;
  }
  float2 acc[kI][D / 32];
  clear(acc);
  const int steps = p.at + 1;
  auto load = [&](int n) {
    float* K = smem + (2 + (n & 1) * 2) * kTile;
    const int j0 = p.t0 + n * kT, keys = min(kT, p.t1 - j0);
    load_rows<D>(K, k + j0 * ks, ks, keys);
    load_rows<D>(K + kTile, v + j0 * ks, ks, keys);
  };
  float next_b[kJ];
  auto load_bias = [&](int n) {
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      const int tok = p.t0 + n * kT + tx + 16 * j;
      next_b[j] = a.bias && tok < p.t1 ? a.bias[(long long)hk * a.seqs.total + tok] : 0.f;
    }
  };
  load_bias(0);
  for (int n = 0; n < steps; ++n) {
    const int j0 = p.t0 + n * kT;
    float *K = smem + (2 + (n & 1) * 2) * kTile, *V = K + kTile, *W = V;
    float b[kJ];
#pragma unroll
    for (int j = 0; j < kJ; ++j) b[j] = next_b[j];
    stage_tiles(n, steps, load);
    load_bias(n + 1);
    float2 s[kI][kJ], dp[kI][kJ];
    clear(s);
    clear(dp);
    dot_tile<D>(s, Q, K);
    dot_tile<D>(dp, O, V);
    __syncthreads();  // V has been read
#pragma unroll
    for (int i = 0; i < kI; ++i)
#pragma unroll
      for (int j = 0; j < kJ; ++j) {
        const int q = i0 + ty + kTy * i, tok = j0 + tx + 16 * j;
        const float w = expf(fmaf(sum2(s[i][j]), scale, tok < q ? b[j] : 0.f) - lse[i]);
        W[(ty + kTy * i) * kW + tx + 16 * j] = sees(q, tok, b[j]) ? w * (sum2(dp[i][j]) - delta[i]) : 0.f;
      }
    __syncthreads();
    sum_tile<D>(acc, W, K);
  }
#pragma unroll
  for (int i = 0; i < kI; ++i)
    if (ty + kTy * i < rows)
      store_row<D>(static_cast<float*>(a.dq) + at + (long long)(ty + kTy * i) * qs, acc[i], scale);
}

// The rows of K's and V's gradients and of the bias's, summed over the queries of the
// group: dV_j = sum of P_ij dO_i, dK_j = scale sum of dS_ij q_i, dbias_j = sum over i > j of dS_ij
template <int D>
__device__ __forceinline__ void dkv_rows(const AttnArgs& a, int hk, int share, float* smem) {
  constexpr int kTile = kT * (D + 4);
  float *K = smem, *V = K + kTile, *W = K + 6 * kTile;
  float *X = W + kT * kW, *numbers = X + kT * kW;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const Piece p = find_piece(a.seqs, kT, blockIdx.x);
  if (!p.ok) return;
  const int j0 = p.t0 + p.at * kT, keys = min(kT, p.t1 - j0);
  const float scale = 1.f / sqrtf((float)D);
  const long long qs = (long long)a.Hq * D, ks = (long long)a.Hkv * D, at = (long long)j0 * ks + (long long)hk * D;
  load_rows<D>(K, static_cast<const float*>(a.k) + at, ks, keys);
  load_rows<D>(V, static_cast<const float*>(a.v) + at, ks, keys);
  float bias[kI], db[kI];
#pragma unroll
  for (int j = 0; j < kI; ++j) {
    const int r = ty + kTy * j;
    bias[j] = a.bias && r < keys ? a.bias[(long long)hk * a.seqs.total + j0 + r] : 0.f;
    db[j] = 0.f;
  }
  float2 dk[kI][D / 32], dv[kI][D / 32];
  clear(dk);
  clear(dv);
  const int h0 = hk * a.G + share * a.G / a.shares, h1 = hk * a.G + (share + 1) * a.G / a.shares;
  const int tiles = (p.t1 - j0 + kT - 1) / kT, steps = (h1 - h0) * tiles;
  auto load = [&](int n) {
    float *Q = smem + (2 + (n & 1) * 2) * kTile, *L = numbers + (n & 1) * 2 * kT;
    const int h = h0 + n / tiles, i0 = j0 + n % tiles * kT, rows = min(kT, p.t1 - i0);
    const long long q0 = (long long)i0 * qs + (long long)h * D;
    load_rows<D>(Q, static_cast<const float*>(a.q) + q0, qs, rows);
    load_rows<D>(Q + kTile, static_cast<const float*>(a.dout) + q0, qs, rows);
    if (threadIdx.x < kT) {
      const bool in = (int)threadIdx.x < rows;
      const long long at = (long long)h * a.seqs.total + i0 + (in ? threadIdx.x : 0);
      cp_async4_zfill(smem_u32(L + threadIdx.x), a.lse + at, in);
      cp_async4_zfill(smem_u32(L + kT + threadIdx.x), a.rows + at, in);
    }
  };
  for (int n = 0; n < steps; ++n) {
    const float *Q = smem + (2 + (n & 1) * 2) * kTile, *O = Q + kTile;
    const float *L = numbers + (n & 1) * 2 * kT, *E = L + kT;
    const int i0 = j0 + n % tiles * kT, rows = min(kT, p.t1 - i0);
    stage_tiles(n, steps, load);
    float2 s[kI][kJ], dp[kI][kJ];
    clear(s);
    clear(dp);
    dot_tile<D>(s, K, Q);
    dot_tile<D>(dp, V, O);
#pragma unroll
    for (int j = 0; j < kI; ++j)
#pragma unroll
      for (int i = 0; i < kJ; ++i) {
        const int tok = j0 + ty + kTy * j, r = tx + 16 * i, q = i0 + r;
        const bool seen = r < rows && sees(q, tok, bias[j]);
        const float w = seen ? expf(fmaf(sum2(s[j][i]), scale, tok < q ? bias[j] : 0.f) - L[r]) : 0.f;
        const float ds = seen ? w * (sum2(dp[j][i]) - E[r]) : 0.f;
        W[(ty + kTy * j) * kW + r] = w;
        X[(ty + kTy * j) * kW + r] = ds;
        if (tok < q) db[j] += ds;
      }
    __syncthreads();
    sum_tile<D>(dv, W, O);
    sum_tile<D>(dk, X, Q);
  }
#pragma unroll
  for (int j = 0; j < kI; ++j) {
    const int r = ty + kTy * j;
    const float b = row_sum(db[j]);
    if (r >= keys) continue;
    const bool whole = a.shares == 1;
    store_row<D>(whole ? static_cast<float*>(a.dk) + at + r * ks : share_rows(a, D, true, share, hk, j0 + r), dk[j], scale);
    store_row<D>(whole ? static_cast<float*>(a.dv) + at + r * ks : share_rows(a, D, false, share, hk, j0 + r), dv[j], 1.f);
    if (tx == 0 && a.dbias)
      (whole ? static_cast<float*>(a.dbias) + (long long)hk * a.seqs.total : share_dbias(a, D, share, hk))[j0 + r] = b;
  }
}

// Both, beside one another, where each leaves SMs without a block: KV heads first, in shares of their groups
template <int D>
__global__ void __launch_bounds__(kThreads) attn_grads_kernel(const AttnArgs a) {
  extern __shared__ float smem[];
  const int y = blockIdx.y, kv = a.Hkv * a.shares;
  if (y < kv)
    dkv_rows<D>(a, y % a.Hkv, y / a.Hkv, smem);
  else
    dq_rows<D>(a, y - kv, smem);
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

template <auto* kernel>
cudaError_t launch(const AttnArgs& a, int heads, size_t bytes, cudaStream_t stream) {
  const cudaError_t e = allow_shared<kernel>((int)bytes);
  if (e != cudaSuccess) return e;
  kernel<<<dim3((unsigned)pieces(a.seqs.total, a.seqs.num, kT), heads), kThreads, bytes, stream>>>(a);
  return cudaGetLastError();
}

template <int D>
cudaError_t forward(const AttnArgs& a, cudaStream_t stream) {
  return launch<attn_kernel<D>>(a, a.Hq, tiles_bytes<D>(1, 0), stream);
}

template <int D>
cudaError_t backward(AttnArgs a, cudaStream_t stream) {
  a.shares = attn_shares(pieces(a.seqs.total, a.seqs.num, kT) * a.Hkv, a.G);
  const cudaError_t e = launch<attn_grads_kernel<D>>(a, a.Hkv * a.shares + a.Hq, tiles_bytes<D>(2, 2), stream);
  return e == cudaSuccess && a.shares > 1 ? attn_join(a, false, D, stream) : e;
}

cudaError_t deltas(const AttnArgs& a, int D, cudaStream_t stream) {
  const unsigned int blocks = (unsigned)(((long long)a.seqs.total * a.Hq + 7) / 8);
  if (D == 128)
    attn_delta_kernel<128><<<blocks, 256, 0, stream>>>(a);
  else
    attn_delta_kernel<64><<<blocks, 256, 0, stream>>>(a);
  return cudaGetLastError();
}

// Tiles of 64 rows of `heads` heads: what the tensor cores' kernels would have to share out
long long tiles64(const AttnArgs& a, int heads) { return pieces(a.seqs.total, a.seqs.num, 64) * heads; }

}  // namespace

// On the tensor cores from half a tile of 64 queries per SM on, us here and there: 132 tiles (one sequence of
// 2048 tokens, 4 heads of 64) 192 and 170, 256 (500 tokens, 32 / 8 heads of 128) 120 and 84; 20 are left here.
cudaError_t attn_forward_f32(const AttnArgs& a, int D, cudaStream_t stream) {
  int sms = 0;
  const cudaError_t e = sm_count(&sms);
  if (e != cudaSuccess) return e;
  if (tiles64(a, a.Hq) * 2 >= sms) return attn_forward_parts(a, D, stream);
  return D == 128 ? forward<128>(a, stream) : forward<64>(a, stream);
}
// From five tiles of KV heads per four SMs on: 160 tiles (300 tokens, 32 heads of 128) 131 and 143, 192 (1500
// tokens, 40 / 8 heads of 64) 1285 and 1067, 272 (two sequences of 1024, 8 heads of 128) 523 and 451.
cudaError_t attn_backward_f32(const AttnArgs& args, int D, cudaStream_t stream) {
  AttnArgs a = args;
  if (!a.bias) a.dbias = nullptr;
  int sms = 0;
  cudaError_t e = sm_count(&sms);
  if (e == cudaSuccess) e = deltas(a, D, stream);
  if (e != cudaSuccess) return e;
  if (tiles64(a, a.Hkv) * 4 >= 5 * sms) return attn_backward_parts(a, D, stream);
  return D == 128 ? backward<128>(a, stream) : backward<64>(a, stream);
}

}  // namespace dmc
