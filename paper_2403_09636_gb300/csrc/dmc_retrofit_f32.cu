// Attention of packed sequences in fp32 on the CUDA cores, with its gradients: every product
// and sum in fp32.
//
// All products are built from tiles of kT rows in shared memory, by a block of 16 columns of
// threads; a thread takes every 16th (kT / 16 of them) and every (threads / 16)-th row. Rows are
// padded by 16 bytes, so that the 16-byte reads of 8 neighbouring rows fall into different banks.
// Multiply-adds come in pairs (fma.rn.f32x2), two neighbouring terms of a sum or two
// neighbouring columns, which leaves issue slots for the reads: 12 reads of 16 bytes per 32 pairs.
// Bound by multiply-adds and the reads that feed them: 33 to 39 TFLOP/s with heads of 128 (10 sequences
// of 1148 tokens of 32 / 8 heads: forward 2.77 ms, backward 10.1 ms), 28 with heads of 64.
// Tiles of 64 rows, 256 threads; 32 rows and 128 threads where tiles of 64 would be fewer than two
// blocks per SM, so that a block's steps one after another set the time: twice as many blocks, whose steps take less
// than half as long, the next step's tiles on their way meanwhile, dQ in one launch with dK and dV, and
// those in shares of a group's heads (attn_shares). 256 tokens of 4 heads of 64: forward 25 us, backward 35 (63 in two
// launches without tiles ahead); 500 tokens of 32 / 8 heads of 128: 117 and 278 (532 with whole groups).
// 256 threads for tiles of 32 rows take 24 and 38, 138 and 731.
#include <math.h>

#include "dmc_retrofit.cuh"

namespace dmc {
cudaError_t attn_join(const AttnArgs& a, bool bf16, int D, cudaStream_t stream);

namespace {

template <int kRows>
struct Shape {
  static constexpr int kT = kRows;                     // rows of a tile
  static constexpr int kThreads = kRows == 64 ? 256 : 128;
  static constexpr int kI = kT * 16 / kThreads;        // rows of a thread
  static constexpr int kJ = kT / 16;                   // columns of a thread
  static constexpr int kTy = kThreads / 16;
  static constexpr int kW = kT + 4;                    // row of a tile of weights
  static constexpr int kStages = kRows == 64 ? 1 : 2;  // tiles of the sequence's other rows kept at once
};

// `rows` rows of D columns, asynchronously, into a tile; zero from there on
template <int D, class S>
__device__ __forceinline__ void load_rows(float* tile, const float* src, long long stride, int rows) {
#pragma unroll
  for (int i = threadIdx.x; i < S::kT * (D / 4); i += S::kThreads) {
    const int r = i / (D / 4), c = i % (D / 4) * 4;
    cp_async16_zfill(smem_u32(tile + r * (D + 4) + c), src + (r < rows ? r * stride : 0) + c, r < rows);
  }
}

// acc[i][j] += X[ty + kTy i] . Y[tx + 16 j], even and odd terms apart
template <int D, class S>
__device__ __forceinline__ void dot_tile(float2 (&acc)[S::kI][S::kJ], const float* X, const float* Y) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll 4
  for (int c = 0; c < D; c += 4) {
    float4 x[S::kI], y[S::kJ];
#pragma unroll
    for (int i = 0; i < S::kI; ++i) x[i] = *reinterpret_cast<const float4*>(X + (ty + S::kTy * i) * (D + 4) + c);
#pragma unroll
    for (int j = 0; j < S::kJ; ++j) y[j] = *reinterpret_cast<const float4*>(Y + (tx + 16 * j) * (D + 4) + c);
#pragma unroll
    for (int i = 0; i < S::kI; ++i)
#pragma unroll
      for (int j = 0; j < S::kJ; ++j) {
        acc[i][j] = fma2(make_float2(x[i].x, x[i].y), make_float2(y[j].x, y[j].y), acc[i][j]);
        acc[i][j] = fma2(make_float2(x[i].z, x[i].w), make_float2(y[j].z, y[j].w), acc[i][j]);
      }
  }
}

// acc[i][2 c], acc[i][2 c + 1] (columns 4 tx + 64 c ..) += sum over r < kT of W[ty + kTy i][r] Y[r][.]
template <int D, class S>
__device__ __forceinline__ void sum_tile(float2 (&acc)[S::kI][D / 32], const float* W, const float* Y) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll 2
  for (int r = 0; r < S::kT; r += 4) {
    float4 w[S::kI];
#pragma unroll
    for (int i = 0; i < S::kI; ++i) w[i] = *reinterpret_cast<const float4*>(W + (ty + S::kTy * i) * S::kW + r);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const float4 y = *reinterpret_cast<const float4*>(Y + (r + k) * (D + 4) + 4 * tx + 64 * c);
#pragma unroll
        for (int i = 0; i < S::kI; ++i) {
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

// Tiles of step n, by `load(n)`. With two stages those of the next step are asked for
// here, once all threads are through with the step before; with one they come when they are needed.
template <class S, typename Load>
__device__ __forceinline__ void stage_tiles(int n, int steps, const Load& load) {
  __syncthreads();  // the step before has read its tiles
  if (S::kStages == 1 || n == 0) {
    load(n);
    cp_async_commit();
  }
  if (S::kStages == 2 && n + 1 < steps) {
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
template <int D, int kRows>
constexpr size_t tiles_bytes(int own, int weights) {
  constexpr int stages = Shape<kRows>::kStages;
  return ((size_t)(own + 2 * stages) * kRows * (D + 4) + (size_t)weights * kRows * (kRows + 4) + 2 * stages * kRows) * 4;
}

// Weights take K's place once the scores are there.
template <int D, int kRows>
__global__ void __launch_bounds__(Shape<kRows>::kThreads, 2) attn_kernel(const AttnArgs a) {
  using S = Shape<kRows>;
  extern __shared__ float smem[];
  constexpr int kTile = S::kT * (D + 4);
  float* Q = smem;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, h = blockIdx.y, hk = h / a.G;
  if (blockIdx.x == 0 && h == 0) check_seqs(a.seqs, a.error);
  Piece p = find_piece(a.seqs, S::kT, blockIdx.x);
  if (!p.ok) return;
  p.at = (p.t1 - p.t0 + S::kT - 1) / S::kT - 1 - p.at;  // the longest rows first
  const int i0 = p.t0 + p.at * S::kT, rows = min(S::kT, p.t1 - i0);
  const float scale = 1.f / sqrtf((float)D);
  const long long qs = (long long)a.Hq * D, ks = (long long)a.Hkv * D;
  const float *k = static_cast<const float*>(a.k) + (long long)hk * D, *v = static_cast<const float*>(a.v) + (long long)hk * D;
  load_rows<D, S>(Q, static_cast<const float*>(a.q) + (long long)i0 * qs + (long long)h * D, qs, rows);
  float2 acc[S::kI][D / 32];
  clear(acc);
  float m[S::kI], l[S::kI];
#pragma unroll
  for (int i = 0; i < S::kI; ++i) m[i] = -INFINITY, l[i] = 0.f;
  const int steps = p.at + 1;
  auto load = [&](int n) {
    float* K = smem + (1 + n % S::kStages * 2) * kTile;
    const int j0 = p.t0 + n * S::kT, keys = min(S::kT, p.t1 - j0);
    load_rows<D, S>(K, k + j0 * ks, ks, keys);
    load_rows<D, S>(K + kTile, v + j0 * ks, ks, keys);
  };
  float next_b[S::kJ];
  auto load_bias = [&](int n) {
#pragma unroll
    for (int j = 0; j < S::kJ; ++j) {
      const int tok = p.t0 + n * S::kT + tx + 16 * j;
      next_b[j] = a.bias && tok < p.t1 ? a.bias[(long long)hk * a.seqs.total + tok] : 0.f;
    }
  };
  load_bias(0);
  for (int n = 0; n < steps; ++n) {
    const int j0 = p.t0 + n * S::kT;
    float *K = smem + (1 + n % S::kStages * 2) * kTile, *V = K + kTile, *W = K;
    float b[S::kJ];
#pragma unroll
    for (int j = 0; j < S::kJ; ++j) b[j] = next_b[j];
    stage_tiles<S>(n, steps, load);
    load_bias(n + 1);
    float2 s2[S::kI][S::kJ];
    clear(s2);
    dot_tile<D, S>(s2, Q, K);
    __syncthreads();  // K has been read
#pragma unroll
    for (int i = 0; i < S::kI; ++i) {
      const int q = i0 + ty + S::kTy * i;
      float s[S::kJ], mt = -INFINITY;
#pragma unroll
      for (int j = 0; j < S::kJ; ++j) {
        const int tok = j0 + tx + 16 * j;
        s[j] = sees(q, tok, b[j]) ? fmaf(sum2(s2[i][j]), scale, tok < q ? b[j] : 0.f) : -INFINITY;
        mt = fmaxf(mt, s[j]);
      }
      const float mn = fmaxf(m[i], row_max(mt)), ref = mn == -INFINITY ? 0.f : mn;
      const float corr = expf(m[i] - ref);
      m[i] = mn;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < S::kJ; ++j) {
        const float w = expf(s[j] - ref);
        sum += w;
        W[(ty + S::kTy * i) * S::kW + tx + 16 * j] = w;
      }
      l[i] = fmaf(l[i], corr, row_sum(sum));
#pragma unroll
      for (int c = 0; c < D / 32; ++c) acc[i][c] = mul2(acc[i][c], make_float2(corr, corr));
    }
    __syncthreads();
    sum_tile<D, S>(acc, W, V);
  }
#pragma unroll
  for (int i = 0; i < S::kI; ++i) {
    const int r = ty + S::kTy * i;
    if (r >= rows) continue;
    store_row<D>(static_cast<float*>(a.out) + (long long)(i0 + r) * qs + (long long)h * D, acc[i], 1.f / l[i]);
    if (tx == 0) a.lse[(long long)h * a.seqs.total + i0 + r] = m[i] + logf(l[i]);
  }
}

// The rows of Q's gradient: dQ_i = scale sum over j of dS_ij k_j, with
// dS = P (dO V^T - delta), delta_i = dO_i . out_i. Weights take V's place.
template <int D, int kRows>
__device__ __forceinline__ void dq_rows(const AttnArgs& a, int h, float* smem) {
  using S = Shape<kRows>;
  constexpr int kTile = S::kT * (D + 4);
  float *Q = smem, *O = Q + kTile;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, hk = h / a.G;
  Piece p = find_piece(a.seqs, S::kT, blockIdx.x);
  if (!p.ok) return;
  p.at = (p.t1 - p.t0 + S::kT - 1) / S::kT - 1 - p.at;
  const int i0 = p.t0 + p.at * S::kT, rows = min(S::kT, p.t1 - i0);
  const float scale = 1.f / sqrtf((float)D);
  const long long qs = (long long)a.Hq * D, ks = (long long)a.Hkv * D, at = (long long)i0 * qs + (long long)h * D;
  const float *k = static_cast<const float*>(a.k) + (long long)hk * D, *v = static_cast<const float*>(a.v) + (long long)hk * D;
  load_rows<D, S>(Q, static_cast<const float*>(a.q) + at, qs, rows);
  load_rows<D, S>(O, static_cast<const float*>(a.dout) + at, qs, rows);
  float lse[S::kI], delta[S::kI];
#pragma unroll
  for (int i = 0; i < S::kI; ++i) {
    const long long n = (long long)h * a.seqs.total + i0 + ty + S::kTy * i;
    const bool in = ty + S::kTy * i < rows;
    lse[i] = in ? a.lse[n] : 0.f;
    delta[i] = in ? a.rows[n] : 0.f;
  }
  float2 acc[S::kI][D / 32];
  clear(acc);
  const int steps = p.at + 1;
  auto load = [&](int n) {
    float* K = smem + (2 + n % S::kStages * 2) * kTile;
    const int j0 = p.t0 + n * S::kT, keys = min(S::kT, p.t1 - j0);
    load_rows<D, S>(K, k + j0 * ks, ks, keys);
    load_rows<D, S>(K + kTile, v + j0 * ks, ks, keys);
  };
  float next_b[S::kJ];
  auto load_bias = [&](int n) {
#pragma unroll
    for (int j = 0; j < S::kJ; ++j) {
      const int tok = p.t0 + n * S::kT + tx + 16 * j;
      next_b[j] = a.bias && tok < p.t1 ? a.bias[(long long)hk * a.seqs.total + tok] : 0.f;
    }
  };
  load_bias(0);
  for (int n = 0; n < steps; ++n) {
    const int j0 = p.t0 + n * S::kT;
    float *K = smem + (2 + n % S::kStages * 2) * kTile, *V = K + kTile, *W = V;
    float b[S::kJ];
#pragma unroll
    for (int j = 0; j < S::kJ; ++j) b[j] = next_b[j];
    stage_tiles<S>(n, steps, load);
    load_bias(n + 1);
    float2 s[S::kI][S::kJ], dp[S::kI][S::kJ];
    clear(s);
    clear(dp);
    dot_tile<D, S>(s, Q, K);
    dot_tile<D, S>(dp, O, V);
    __syncthreads();  // V has been read
#pragma unroll
    for (int i = 0; i < S::kI; ++i)
#pragma unroll
      for (int j = 0; j < S::kJ; ++j) {
        const int q = i0 + ty + S::kTy * i, tok = j0 + tx + 16 * j;
        const float w = expf(fmaf(sum2(s[i][j]), scale, tok < q ? b[j] : 0.f) - lse[i]);
        W[(ty + S::kTy * i) * S::kW + tx + 16 * j] = sees(q, tok, b[j]) ? w * (sum2(dp[i][j]) - delta[i]) : 0.f;
      }
    __syncthreads();
    sum_tile<D, S>(acc, W, K);
  }
#pragma unroll
  for (int i = 0; i < S::kI; ++i)
    if (ty + S::kTy * i < rows)
      store_row<D>(static_cast<float*>(a.dq) + at + (long long)(ty + S::kTy * i) * qs, acc[i], scale);
}

// The rows of K's and V's gradients and of the bias's, summed over the queries of the
// group: dV_j = sum of P_ij dO_i, dK_j = scale sum of dS_ij q_i, dbias_j = sum over i > j of dS_ij
template <int D, int kRows>
__device__ __forceinline__ void dkv_rows(const AttnArgs& a, int hk, int share, float* smem) {
  using S = Shape<kRows>;
  constexpr int kTile = S::kT * (D + 4);
  float *K = smem, *V = K + kTile, *W = K + (2 + 2 * S::kStages) * kTile;
  float *X = W + S::kT * S::kW, *numbers = X + S::kT * S::kW;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const Piece p = find_piece(a.seqs, S::kT, blockIdx.x);
  if (!p.ok) return;
  const int j0 = p.t0 + p.at * S::kT, keys = min(S::kT, p.t1 - j0);
  const float scale = 1.f / sqrtf((float)D);
  const long long qs = (long long)a.Hq * D, ks = (long long)a.Hkv * D, at = (long long)j0 * ks + (long long)hk * D;
  load_rows<D, S>(K, static_cast<const float*>(a.k) + at, ks, keys);
  load_rows<D, S>(V, static_cast<const float*>(a.v) + at, ks, keys);
  float bias[S::kI], db[S::kI];
#pragma unroll
  for (int j = 0; j < S::kI; ++j) {
    const int r = ty + S::kTy * j;
    bias[j] = a.bias && r < keys ? a.bias[(long long)hk * a.seqs.total + j0 + r] : 0.f;
    db[j] = 0.f;
  }
  float2 dk[S::kI][D / 32], dv[S::kI][D / 32];
  clear(dk);
  clear(dv);
  const int h0 = hk * a.G + share * a.G / a.shares, h1 = hk * a.G + (share + 1) * a.G / a.shares;
  const int tiles = (p.t1 - j0 + S::kT - 1) / S::kT, steps = (h1 - h0) * tiles;
  auto load = [&](int n) {
    float *Q = smem + (2 + n % S::kStages * 2) * kTile, *L = numbers + n % S::kStages * 2 * S::kT;
    const int h = h0 + n / tiles, i0 = j0 + n % tiles * S::kT, rows = min(S::kT, p.t1 - i0);
    const long long q0 = (long long)i0 * qs + (long long)h * D;
    load_rows<D, S>(Q, static_cast<const float*>(a.q) + q0, qs, rows);
    load_rows<D, S>(Q + kTile, static_cast<const float*>(a.dout) + q0, qs, rows);
    if (threadIdx.x < S::kT) {
      const bool in = (int)threadIdx.x < rows;
      const long long at = (long long)h * a.seqs.total + i0 + (in ? threadIdx.x : 0);
      cp_async4_zfill(smem_u32(L + threadIdx.x), a.lse + at, in);
      cp_async4_zfill(smem_u32(L + S::kT + threadIdx.x), a.rows + at, in);
    }
  };
  for (int n = 0; n < steps; ++n) {
    const float *Q = smem + (2 + n % S::kStages * 2) * kTile, *O = Q + kTile;
    const float *L = numbers + n % S::kStages * 2 * S::kT, *E = L + S::kT;
    const int i0 = j0 + n % tiles * S::kT, rows = min(S::kT, p.t1 - i0);
    stage_tiles<S>(n, steps, load);
    float2 s[S::kI][S::kJ], dp[S::kI][S::kJ];
    clear(s);
    clear(dp);
    dot_tile<D, S>(s, K, Q);
    dot_tile<D, S>(dp, V, O);
#pragma unroll
    for (int j = 0; j < S::kI; ++j)
#pragma unroll
      for (int i = 0; i < S::kJ; ++i) {
        const int tok = j0 + ty + S::kTy * j, r = tx + 16 * i, q = i0 + r;
        const bool seen = r < rows && sees(q, tok, bias[j]);
        const float w = seen ? expf(fmaf(sum2(s[j][i]), scale, tok < q ? bias[j] : 0.f) - L[r]) : 0.f;
        const float ds = seen ? w * (sum2(dp[j][i]) - E[r]) : 0.f;
        W[(ty + S::kTy * j) * S::kW + r] = w;
        X[(ty + S::kTy * j) * S::kW + r] = ds;
        if (tok < q) db[j] += ds;
      }
    __syncthreads();
    sum_tile<D, S>(dv, W, O);
    sum_tile<D, S>(dk, X, Q);
  }
#pragma unroll
  for (int j = 0; j < S::kI; ++j) {
    const int r = ty + S::kTy * j;
    const float b = row_sum(db[j]);
    if (r >= keys) continue;
    const bool whole = a.shares == 1;
    store_row<D>(whole ? static_cast<float*>(a.dk) + at + r * ks : share_rows(a, D, true, share, hk, j0 + r), dk[j], scale);
    store_row<D>(whole ? static_cast<float*>(a.dv) + at + r * ks : share_rows(a, D, false, share, hk, j0 + r), dv[j], 1.f);
    if (tx == 0 && a.dbias)
      (whole ? static_cast<float*>(a.dbias) + (long long)hk * a.seqs.total : share_dbias(a, D, share, hk))[j0 + r] = b;
  }
}

template <int D, int kRows>
__global__ void __launch_bounds__(Shape<kRows>::kThreads) attn_dq_kernel(const AttnArgs a) {
  extern __shared__ float smem[];
  dq_rows<D, kRows>(a, blockIdx.y, smem);
}
template <int D, int kRows>
__global__ void __launch_bounds__(Shape<kRows>::kThreads) attn_dkv_kernel(const AttnArgs a) {
  extern __shared__ float smem[];
  dkv_rows<D, kRows>(a, blockIdx.y, 0, smem);
}
// Both, beside one another, where each leaves SMs without a block: KV heads first, in shares of their groups
template <int D, int kRows>
__global__ void __launch_bounds__(Shape<kRows>::kThreads) attn_grads_kernel(const AttnArgs a) {
  extern __shared__ float smem[];
  const int y = blockIdx.y, kv = a.Hkv * a.shares;
  if (y < kv)
    dkv_rows<D, kRows>(a, y % a.Hkv, y / a.Hkv, smem);
  else
    dq_rows<D, kRows>(a, y - kv, smem);
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
cudaError_t launch(const AttnArgs& a, int heads, int rows, int threads, size_t bytes, cudaStream_t stream) {
  const cudaError_t e = allow_shared<kernel>((int)bytes);
  if (e != cudaSuccess) return e;
  kernel<<<dim3((unsigned)pieces(a.seqs.total, a.seqs.num, rows), heads), threads, bytes, stream>>>(a);
  return cudaGetLastError();
}

template <int D, int kRows>
cudaError_t forward(const AttnArgs& a, cudaStream_t stream) {
  return launch<attn_kernel<D, kRows>>(a, a.Hq, kRows, Shape<kRows>::kThreads, tiles_bytes<D, kRows>(1, 0), stream);
}

template <int D, int kRows>
cudaError_t backward(AttnArgs a, cudaStream_t stream) {
  constexpr int threads = Shape<kRows>::kThreads;
  if (!a.bias) a.dbias = nullptr;
  attn_delta_kernel<D><<<(unsigned)(((long long)a.seqs.total * a.Hq + 7) / 8), 256, 0, stream>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  a.shares = 1;
  if (kRows == 32) {
    a.shares = attn_shares(pieces(a.seqs.total, a.seqs.num, 32) * a.Hkv, a.G);
    e = launch<attn_grads_kernel<D, 32>>(a, a.Hkv * a.shares + a.Hq, 32, threads, tiles_bytes<D, 32>(2, 2), stream);
    return e == cudaSuccess && a.shares > 1 ? attn_join(a, false, D, stream) : e;
  }
  e = launch<attn_dkv_kernel<D, 64>>(a, a.Hkv, 64, threads, tiles_bytes<D, 64>(2, 2), stream);
  return e == cudaSuccess ? launch<attn_dq_kernel<D, 64>>(a, a.Hq, 64, threads, tiles_bytes<D, 64>(2, 0), stream) : e;
}

// Whether tiles of 64 rows would be fewer than two blocks per SM
bool small(const AttnArgs& a, int heads) {
  int sms = 0;
  return sm_count(&sms) == cudaSuccess && pieces(a.seqs.total, a.seqs.num, 64) * heads < 2 * sms;
}

}  // namespace

cudaError_t attn_forward_f32(const AttnArgs& a, int D, cudaStream_t stream) {
  if (small(a, a.Hq)) return D == 128 ? forward<128, 32>(a, stream) : forward<64, 32>(a, stream);
  return D == 128 ? forward<128, 64>(a, stream) : forward<64, 64>(a, stream);
}
cudaError_t attn_backward_f32(const AttnArgs& a, int D, cudaStream_t stream) {
  if (small(a, a.Hkv)) return D == 128 ? backward<128, 32>(a, stream) : backward<64, 32>(a, stream);
  return D == 128 ? backward<128, 64>(a, stream) : backward<64, 64>(a, stream);
}

}  // namespace dmc
