// Attention of packed sequences in fp32 on the tensor cores, with its gradients, for calls that
// fill the GPU (dmc_retrofit_f32.cu has the others).
//
// Every fp32 operand x is the sum of three bf16 numbers, x0 = bf16(x), x1 = bf16(x - x0), x2 = bf16(x - x0 -
// x1), which hold its 24 bits; a product is the sum of the six products of parts whose indices
// add up to at most 2 (what is left out is below 2^-24 of the whole). The five small ones have an
// accumulator of their own: the tensor cores drop the bits below an accumulator's last one at every
// step of 16 terms, so that few steps may go into the large one, D / 16 for a score and 4 or less for a sum over
// rows, which is added to the row's sum in fp32 afterwards.
//
// (tcgen05 would multiply faster. The forward pass, and heads of 64, would fit its tiles; the gradients of heads of
// 128 would not, three parts of K, V, Q and dO of 128 rows being 384 KB. It has not been written.)
// Tiles of 64 rows lie in shared memory as their three parts, split once when they are loaded;
// warps multiply 16 rows with mma.sync.m16n8k16, whose operands' layout lets a tile of weights become the
// left operand of the next product without leaving the registers. Rows are padded by 16 bytes: the
// eight rows of a matrix read fall into different banks. 8 warps, one block per SM (209 KB).
// Bound by the tensor cores' rate for these instructions (597 TFLOP/s, a sixth of which is 99 of fp32 products; busy
// for half of the time) and, between barriers that all warps pass, by the exponentials and the splitting:
// 10 sequences of 1148 tokens, 32 / 8 heads of 128, forward 2.03 ms (53 TFLOP/s), backward 7.09 ms (53); fp32
// multiply-adds in tiles of 64 took 2.77 and 10.1 (39, 37). 8 of 700 tokens, 16 / 8 heads of 64, 217 and 681
// us; 291 and 1069 so. The tests of a pair's mask only where queries and rows meet: 2.38 ms forward without.
#include <math.h>

#include "dmc_retrofit.cuh"

namespace dmc {

namespace {

constexpr int kT = 64;         // rows of a tile
constexpr int kThreads = 256;

template <int D>
struct Tile {
  static constexpr int kRow = D * 2 + 16;        // bytes
  static constexpr int kPart = kT * kRow;
  static constexpr int kBytes = 3 * kPart;
  static constexpr int kPer = kT * (D / 4) / kThreads;  // 16-byte pieces of a thread
};

// Rows of a tile, thread t's share of them when kN threads load 64 kN / 256 rows; zero from `rows` on
template <int D, int kN>
__device__ __forceinline__ void fetch(float4 (&x)[Tile<D>::kPer], int t, const float* src, long long stride, int rows) {
#pragma unroll
  for (int i = 0; i < Tile<D>::kPer; ++i) {
    const int at = t + i * kN, r = at / (D / 4), c = at % (D / 4) * 4;
    x[i] = r < rows ? *reinterpret_cast<const float4*>(src + r * stride + c) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
}
// two numbers' parts
__device__ __forceinline__ void split2(float x, float y, uint32_t (&w)[3]) {
#pragma unroll
  for (int p = 0; p < 3; ++p) {
    w[p] = Chunk<__nv_bfloat16>::pack2(x, y);
    float a, b;
    Chunk<__nv_bfloat16>::unpack2(w[p], a, b);
    x -= a;
    y -= b;
  }
}
template <int D, int kN>
__device__ __forceinline__ void keep(unsigned char* tile, int t, const float4 (&x)[Tile<D>::kPer]) {
#pragma unroll
  for (int i = 0; i < Tile<D>::kPer; ++i) {
    const int at = t + i * kN, r = at / (D / 4), c = at % (D / 4) * 4;
    uint32_t u[3], v[3];
    split2(x[i].x, x[i].y, u);
    split2(x[i].z, x[i].w, v);
#pragma unroll
    for (int p = 0; p < 3; ++p)
      *reinterpret_cast<uint2*>(tile + p * Tile<D>::kPart + r * Tile<D>::kRow + c * 2) = make_uint2(u[p], v[p]);
  }
}
template <int D, int kN>
__device__ __forceinline__ void load(unsigned char* tile, int t, const float* src, long long stride, int rows) {
  float4 x[Tile<D>::kPer];
  fetch<D, kN>(x, t, src, stride, rows);
  keep<D, kN>(tile, t, x);
}

// A barrier of one half of the block's warps
__device__ __forceinline__ void half_sync(int half) { asm volatile("bar.sync %0, 128;" ::"r"(1 + half) : "memory"); }

__device__ __forceinline__ void matrices(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void matrices_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void multiply(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the products of 16 rows' parts with part p of kN tiles of 8 columns (b[pair of tiles]: matrices' order)
template <int p, int kN>
__device__ __forceinline__ void multiply_part(float (&big)[kN][4], float (&small)[kN][4], const uint32_t (&a)[3][4],
                                              const uint32_t (&b)[kN / 2][4]) {
#pragma unroll
  for (int i = 2 - p; i >= 0; --i)
#pragma unroll
    for (int t = 0; t < kN; ++t)
      multiply(i + p > 0 ? small[t] : big[t], a[i], b[t / 2][t % 2 * 2], b[t / 2][t % 2 * 2 + 1]);
}

// s (16 rows x 8 kN columns) = X Y^T over D, of the tiles' rows at x and y
template <int D, int kN>
__device__ __forceinline__ void scores(float (&s)[kN][4], uint32_t x, uint32_t y) {
  constexpr int kRow = Tile<D>::kRow, kPart = Tile<D>::kPart;
  const int lane = threadIdx.x & 31;
  x += (lane & 15) * kRow + (lane >> 4) * 16;
  y += ((lane & 7) + (lane >> 4) * 8) * kRow + (lane >> 3 & 1) * 16;
  float small[kN][4];
#pragma unroll
  for (int t = 0; t < kN; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[t][e] = small[t][e] = 0.f;
#pragma unroll 2
  for (int k = 0; k < D / 16; ++k, x += 32, y += 32) {
    uint32_t a[3][4], b[3][kN / 2][4];
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      matrices(a[p], x + p * kPart);
#pragma unroll
      for (int h = 0; h < kN / 2; ++h) matrices(b[p][h], y + p * kPart + h * 16 * kRow);
    }
    multiply_part<2>(s, small, a, b[2]);
    multiply_part<1>(s, small, a, b[1]);
    multiply_part<0>(s, small, a, b[0]);
  }
#pragma unroll
  for (int t = 0; t < kN; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[t][e] += small[t][e];
}

// 16 x 16 weights, in the layout of two tiles of results, as a left operand
__device__ __forceinline__ void operand(uint32_t (&w)[3][4], const float (&l)[4], const float (&r)[4]) {
  uint32_t u[4][3];
  split2(l[0], l[1], u[0]);
  split2(l[2], l[3], u[1]);
  split2(r[0], r[1], u[2]);
  split2(r[2], r[3], u[3]);
#pragma unroll
  for (int p = 0; p < 3; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) w[p][i] = u[i][p];
}

// acc (16 rows x D) += W Y, W 16 x 16 kK weights, Y the tile's rows at y; kN tiles of 8 columns at a time
template <int D, int kK, int kN>
__device__ __forceinline__ void sums(float (&acc)[D / 8][4], const uint32_t (&w)[kK][3][4], uint32_t y) {
  constexpr int kRow = Tile<D>::kRow, kPart = Tile<D>::kPart;
  const int lane = threadIdx.x & 31;
  y += (lane & 15) * kRow + (lane >> 4) * 16;
#pragma unroll
  for (int t = 0; t < D / 8; t += kN) {
    float big[kN][4], small[kN][4];
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) big[i][e] = small[i][e] = 0.f;
#pragma unroll
    for (int k = 0; k < kK; ++k) {
      uint32_t b[3][kN / 2][4];
#pragma unroll
      for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int h = 0; h < kN / 2; ++h) matrices_trans(b[p][h], y + p * kPart + k * 16 * kRow + (t + 2 * h) * 16);
      multiply_part<2>(big, small, w[k], b[2]);
      multiply_part<1>(big, small, w[k], b[1]);
      multiply_part<0>(big, small, w[k], b[0]);
    }
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[t + i][e] += big[i][e] + small[i][e];
  }
}

template <int N>
__device__ __forceinline__ void clear(float (&x)[N][4]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[i][e] = 0.f;
}

// over the four lanes of a row
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
  return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
}
__device__ __forceinline__ float row_sum(float x) {
  x += __shfl_xor_sync(0xffffffffu, x, 1);
  return x + __shfl_xor_sync(0xffffffffu, x, 2);
}

// Whether query i sees row j
__device__ __forceinline__ bool sees(int i, int j, float bias) { return j == i || (j < i && bias != -INFINITY); }

// The rows of a warp's 16 x D sums that are this lane's (lane / 4 and 8 more), `rows` of the warp's count
template <int D>
__device__ __forceinline__ void store(float* dst, long long stride, int rows, const float (&x)[D / 8][4], float scale0,
                                      float scale1) {
  const int lane = threadIdx.x & 31, r = lane >> 2, c = (lane & 3) * 2;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (r + 8 * h >= rows) continue;
    const float scale = h ? scale1 : scale0;
#pragma unroll
    for (int t = 0; t < D / 8; ++t)
      *reinterpret_cast<float2*>(dst + (r + 8 * h) * stride + t * 8 + c) =
          make_float2(x[t][2 * h] * scale, x[t][2 * h + 1] * scale);
  }
}

// The sums of two warps with the same rows: the second's through shared memory (of 16 rows, D + 4 apart)
template <int D>
__device__ __forceinline__ void leave(float* at, const float (&x)[D / 8][4]) {
  store<D>(at, D + 4, 16, x, 1.f, 1.f);
}
template <int D>
__device__ __forceinline__ void gather(const float* at, float (&x)[D / 8][4]) {
  const int lane = threadIdx.x & 31, r = lane >> 2, c = (lane & 3) * 2;
#pragma unroll
  for (int t = 0; t < D / 8; ++t)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float2 y = *reinterpret_cast<const float2*>(at + (r + 8 * h) * (D + 4) + t * 8 + c);
      x[t][2 * h] += y.x;
      x[t][2 * h + 1] += y.y;
    }
}

// A block: 128 queries of a head, 16 per warp. K's next tile is fetched while S is computed and V's while
// O is, into registers, and kept when all warps are through with the present one. (Half of the warps half a
// step behind the others, so that exponentials run beside products, was 4 % slower: two more barriers.)
template <int D>
__global__ void __launch_bounds__(kThreads, 1) parts_forward_kernel(const AttnArgs a) {
  extern __shared__ unsigned char smem[];
  unsigned char *Q = smem, *K = Q + 2 * Tile<D>::kBytes, *V = K + Tile<D>::kBytes;
  float* biases = reinterpret_cast<float*>(V + Tile<D>::kBytes);  // [2][64]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, h = blockIdx.y, hk = h / a.G;
  if (blockIdx.x == 0 && h == 0) check_seqs(a.seqs, a.error);
  Piece p = find_piece(a.seqs, 2 * kT, blockIdx.x);
  if (!p.ok) return;
  p.at = (p.t1 - p.t0 + 2 * kT - 1) / (2 * kT) - 1 - p.at;  // the longest rows first
  const int i0 = p.t0 + p.at * 2 * kT, last = min(i0 + 2 * kT, p.t1) - 1;
  const int steps = (last - p.t0) / kT + 1;
  const float scale = 1.f / sqrtf((float)D);
  const long long qs = (long long)a.Hq * D, ks = (long long)a.Hkv * D;
  const float *q = static_cast<const float*>(a.q) + (long long)i0 * qs + (long long)h * D;
  const float *k = static_cast<const float*>(a.k) + (long long)hk * D, *v = static_cast<const float*>(a.v) + (long long)hk * D;
  const float* bias = a.bias ? a.bias + (long long)hk * a.seqs.total : nullptr;
  load<D, kThreads>(Q, tid, q, qs, p.t1 - i0);
  if (p.t1 - i0 > kT) load<D, kThreads>(Q + Tile<D>::kBytes, tid, q + kT * qs, qs, p.t1 - i0 - kT);
  load<D, kThreads>(K, tid, k + p.t0 * ks, ks, p.t1 - p.t0);
  load<D, kThreads>(V, tid, v + p.t0 * ks, ks, p.t1 - p.t0);
  if (tid < kT) biases[tid] = bias && p.t0 + tid < p.t1 ? bias[p.t0 + tid] : 0.f;
  __syncthreads();
  const uint32_t sq = smem_u32(Q) + (warp >> 2) * Tile<D>::kBytes + (warp & 3) * 16 * Tile<D>::kRow;
  const uint32_t sk = smem_u32(K), sv = smem_u32(V);
  const int row0 = i0 + warp * 16, mine = row0 + (lane >> 2), c0 = (lane & 3) * 2;
  float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  clear(o);
#pragma unroll 1
  for (int n = 0; n < steps; ++n) {
    const int j0 = p.t0 + n * kT;
    const bool more = n + 1 < steps, use = j0 <= row0 + 15 && row0 < p.t1;
    const float* b = biases + (n & 1) * kT;
    float4 next[Tile<D>::kPer];
    float next_b = 0.f;
    if (more) {
      fetch<D, kThreads>(next, tid, k + (long long)(j0 + kT) * ks, ks, p.t1 - j0 - kT);
      if (bias && tid < kT && j0 + kT + tid < p.t1) next_b = bias[j0 + kT + tid];
    }
    float s[8][4];
    if (use) scores<D, 8>(s, sq, sk);
    __syncthreads();  // K has been read
    if (more) {
      keep<D, kThreads>(K, tid, next);
      if (tid < kT) biases[((n + 1) & 1) * kT + tid] = next_b;
      fetch<D, kThreads>(next, tid, v + (long long)(j0 + kT) * ks, ks, p.t1 - j0 - kT);
    }
    if (use) {
      if (j0 + kT <= row0) {  // rows before all of the warp's queries
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const float2 y = *reinterpret_cast<const float2*>(b + t * 8 + c0);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float z = e & 1 ? y.y : y.x;
            s[t][e] = z == -INFINITY ? z : fmaf(s[t][e], scale, z);
          }
        }
      } else {
#pragma unroll
        for (int t = 0; t < 8; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = mine + 8 * (e >> 1), c = t * 8 + c0 + (e & 1), j = j0 + c;
            s[t][e] = sees(i, j, b[c]) ? fmaf(s[t][e], scale, j < i ? b[c] : 0.f) : -INFINITY;
          }
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float mt = -INFINITY;
#pragma unroll
        for (int t = 0; t < 8; ++t) mt = fmaxf(mt, fmaxf(s[t][2 * r], s[t][2 * r + 1]));
        const float mn = fmaxf(m[r], row_max(mt)), ref = mn == -INFINITY ? 0.f : mn, corr = expf(m[r] - ref);
        m[r] = mn;
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < 8; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            s[t][2 * r + e] = expf(s[t][2 * r + e] - ref);
            sum += s[t][2 * r + e];
          }
        l[r] = fmaf(l[r], corr, row_sum(sum));
#pragma unroll
        for (int t = 0; t < D / 8; ++t) {
          o[t][2 * r] *= corr;
          o[t][2 * r + 1] *= corr;
        }
      }
      uint32_t w[4][3][4];
#pragma unroll
      for (int x = 0; x < 4; ++x) operand(w[x], s[2 * x], s[2 * x + 1]);
      sums<D, 4, 4>(o, w, sv);
    }
    __syncthreads();  // V has been read
    if (more) {
      keep<D, kThreads>(V, tid, next);
      __syncthreads();
    }
  }
  store<D>(static_cast<float*>(a.out) + (long long)row0 * qs + (long long)h * D, qs, p.t1 - row0, o, 1.f / l[0], 1.f / l[1]);
  if ((lane & 3) == 0) {
#pragma unroll
    for (int r = 0; r < 2; ++r)
      if (mine + 8 * r < p.t1) a.lse[(long long)h * a.seqs.total + mine + 8 * r] = m[r] + logf(l[r]);
  }
}

// dQ of 64 queries of a head (see dmc_retrofit_f32.cu for the formulas): a warp has 16 of them and half of
// the rows of a tile of K and V. The halves load their own rows and go their own ways, the second
// from where the first has its first products, so that one's exponentials run beside the other's products
// (10 x 1148 tokens, backward 7.62 ms with barriers of the whole block, 7.09 so).
template <int D>
__global__ void __launch_bounds__(kThreads, 1) parts_dq_kernel(const AttnArgs a) {
  extern __shared__ unsigned char smem[];
  unsigned char *Q = smem, *O = Q + Tile<D>::kBytes, *K = O + Tile<D>::kBytes, *V = K + Tile<D>::kBytes;
  float* biases = reinterpret_cast<float*>(V + Tile<D>::kBytes);  // [2][64]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, h = blockIdx.y, hk = h / a.G;
  Piece p = find_piece(a.seqs, kT, blockIdx.x);
  if (!p.ok) return;
  p.at = (p.t1 - p.t0 + kT - 1) / kT - 1 - p.at;
  const int i0 = p.t0 + p.at * kT, steps = p.at + 1;
  const float scale = 1.f / sqrtf((float)D);
  const long long qs = (long long)a.Hq * D, ks = (long long)a.Hkv * D, at = (long long)i0 * qs + (long long)h * D;
  const float *k = static_cast<const float*>(a.k) + (long long)hk * D, *v = static_cast<const float*>(a.v) + (long long)hk * D;
  const float* bias = a.bias ? a.bias + (long long)hk * a.seqs.total : nullptr;
  load<D, kThreads>(Q, tid, static_cast<const float*>(a.q) + at, qs, p.t1 - i0);
  load<D, kThreads>(O, tid, static_cast<const float*>(a.dout) + at, qs, p.t1 - i0);
  load<D, kThreads>(K, tid, k + p.t0 * ks, ks, p.t1 - p.t0);
  load<D, kThreads>(V, tid, v + p.t0 * ks, ks, p.t1 - p.t0);
  if (tid < kT) biases[tid] = bias && p.t0 + tid < p.t1 ? bias[p.t0 + tid] : 0.f;
  const int group = warp & 3, half = warp >> 2;
  const int row0 = i0 + group * 16, mine = row0 + (lane >> 2), c0 = half * 32 + (lane & 3) * 2;
  float lse[2], delta[2];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const bool in = mine + 8 * r < p.t1;
    const long long x = (long long)h * a.seqs.total + mine + 8 * r;
    lse[r] = in ? a.lse[x] : 0.f;
    delta[r] = in ? a.rows[x] : 0.f;
  }
  __syncthreads();
  const uint32_t own = group * 16 * Tile<D>::kRow, other = half * 32 * Tile<D>::kRow;
  const uint32_t sq = smem_u32(Q) + own, so = smem_u32(O) + own, sk = smem_u32(K) + other, sv = smem_u32(V) + other;
  float dq[D / 8][4];
  clear(dq);
  const int t = tid & 127;  // of the half
  if (half) asm volatile("bar.sync 3, 256;" ::: "memory");
#pragma unroll 1
  for (int n = 0; n < steps; ++n) {
    const int j0 = p.t0 + n * kT, j1 = j0 + kT + half * 32;  // the next tile's first row of this half
    const bool more = n + 1 < steps;
    const float* b = biases + (n & 1) * kT;
    float4 next[Tile<D>::kPer];
    float next_b = 0.f;
    if (more) {
      fetch<D, 128>(next, t, v + (long long)j1 * ks, ks, p.t1 - j1);
      if (bias && t < 32 && j1 + t < p.t1) next_b = bias[j1 + t];
    }
    float dp[4][4], s[4][4];
    scores<D, 4>(dp, so, sv);
    half_sync(half);  // V has been read
    if (more) {
      keep<D, 128>(V + half * 32 * Tile<D>::kRow, t, next);
      if (t < 32) biases[((n + 1) & 1) * kT + half * 32 + t] = next_b;
      fetch<D, 128>(next, t, k + (long long)j1 * ks, ks, p.t1 - j1);
    }
    scores<D, 4>(s, sq, sk);
    if (n == 0 && !half) asm volatile("bar.arrive 3, 256;" ::: "memory");
    if (j0 + kT <= i0) {  // rows before all of the queries
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float2 y = *reinterpret_cast<const float2*>(b + t * 8 + c0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float z = e & 1 ? y.y : y.x;
          const float x = expf(fmaf(s[t][e], scale, z) - lse[e >> 1]);
          s[t][e] = z == -INFINITY ? 0.f : x * (dp[t][e] - delta[e >> 1]);
        }
      }
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = e >> 1, i = mine + 8 * r, c = t * 8 + c0 + (e & 1), j = j0 + c;
          const float x = expf(fmaf(s[t][e], scale, j < i ? b[c] : 0.f) - lse[r]);
          s[t][e] = sees(i, j, b[c]) ? x * (dp[t][e] - delta[r]) : 0.f;
        }
    }
    uint32_t w[2][3][4];
#pragma unroll
    for (int x = 0; x < 2; ++x) operand(w[x], s[2 * x], s[2 * x + 1]);
    sums<D, 2, 4>(dq, w, sk);
    half_sync(half);  // K has been read
    if (more) {
      keep<D, 128>(K + half * 32 * Tile<D>::kRow, t, next);
      half_sync(half);
    }
  }
  __syncthreads();
  float* through = reinterpret_cast<float*>(K) + group * 16 * (D + 4);
  if (half) leave<D>(through, dq);
  __syncthreads();
  if (half) return;
  gather<D>(through, dq);
  store<D>(static_cast<float*>(a.dq) + at + (long long)group * 16 * qs, qs, p.t1 - row0, dq, scale, scale);
}

// dK, dV and dbias of 64 rows of a KV head: a warp has 16 of them and half of the queries of a tile, everything
// transposed, so that the weights' rows are rows of K. The halves are apart as in dQ's kernel.
template <int D>
__global__ void __launch_bounds__(kThreads, 1) parts_dkv_kernel(const AttnArgs a) {
  extern __shared__ unsigned char smem[];
  unsigned char *K = smem, *V = K + Tile<D>::kBytes, *Q = V + Tile<D>::kBytes, *O = Q + Tile<D>::kBytes;
  float *L = reinterpret_cast<float*>(O + Tile<D>::kBytes), *E = L + kT;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, hk = blockIdx.y;
  const Piece p = find_piece(a.seqs, kT, blockIdx.x);
  if (!p.ok) return;
  const int j0 = p.t0 + p.at * kT;
  const float scale = 1.f / sqrtf((float)D);
  const long long qs = (long long)a.Hq * D, ks = (long long)a.Hkv * D, at = (long long)j0 * ks + (long long)hk * D;
  load<D, kThreads>(K, tid, static_cast<const float*>(a.k) + at, ks, p.t1 - j0);
  load<D, kThreads>(V, tid, static_cast<const float*>(a.v) + at, ks, p.t1 - j0);
  const int group = warp & 3, half = warp >> 2;
  const int row0 = j0 + group * 16, mine = row0 + (lane >> 2), c0 = half * 32 + (lane & 3) * 2;
  float b[2], db[2] = {0.f, 0.f};
#pragma unroll
  for (int r = 0; r < 2; ++r)
    b[r] = a.bias && mine + 8 * r < p.t1 ? a.bias[(long long)hk * a.seqs.total + mine + 8 * r] : 0.f;
  const uint32_t own = group * 16 * Tile<D>::kRow, other = half * 32 * Tile<D>::kRow;
  const uint32_t sk = smem_u32(K) + own, sv = smem_u32(V) + own, sq = smem_u32(Q) + other, so = smem_u32(O) + other;
  float dk[D / 8][4], dv[D / 8][4];
  clear(dk);
  clear(dv);
  const int tiles = (p.t1 - j0 + kT - 1) / kT, t = tid & 127;  // t: of the half
  __syncthreads();
  if (half) asm volatile("bar.sync 3, 256;" ::: "memory");
#pragma unroll 1
  for (int n = 0; n < a.G * tiles; ++n) {
    const int h = hk * a.G + n / tiles, i0 = j0 + n % tiles * kT, rows = min(kT, p.t1 - i0);
    const int r0 = half * 32;  // this half's first query of the tile
    const long long q0 = (long long)(i0 + r0) * qs + (long long)h * D;
    half_sync(half);  // the tiles before have been read
    load<D, 128>(Q + r0 * Tile<D>::kRow, t, static_cast<const float*>(a.q) + q0, qs, rows - r0);
    load<D, 128>(O + r0 * Tile<D>::kRow, t, static_cast<const float*>(a.dout) + q0, qs, rows - r0);
    if (t < 32) {
      const long long x = (long long)h * a.seqs.total + i0 + r0 + t;
      L[r0 + t] = r0 + t < rows ? a.lse[x] : 0.f;
      E[r0 + t] = r0 + t < rows ? a.rows[x] : 0.f;
    }
    half_sync(half);
    float s[4][4], dp[4][4];
    scores<D, 4>(s, sk, sq);
    scores<D, 4>(dp, sv, so);
    if (n == 0 && !half) asm volatile("bar.arrive 3, 256;" ::: "memory");
    if (i0 >= j0 + kT && rows == kT) {  // queries after all of the rows
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float2 l = *reinterpret_cast<const float2*>(L + t * 8 + c0), y = *reinterpret_cast<const float2*>(E + t * 8 + c0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float z = b[e >> 1];
          const float x = z == -INFINITY ? 0.f : expf(fmaf(s[t][e], scale, z) - (e & 1 ? l.y : l.x));
          const float ds = z == -INFINITY ? 0.f : x * (dp[t][e] - (e & 1 ? y.y : y.x));
          s[t][e] = x;
          dp[t][e] = ds;
          db[e >> 1] += ds;
        }
      }
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = e >> 1, j = mine + 8 * r, c = t * 8 + c0 + (e & 1), i = i0 + c;
          const bool seen = c < rows && sees(i, j, b[r]);
          const float x = seen ? expf(fmaf(s[t][e], scale, j < i ? b[r] : 0.f) - L[c]) : 0.f;
          const float ds = seen ? x * (dp[t][e] - E[c]) : 0.f;
          s[t][e] = x;
          dp[t][e] = ds;
          if (j < i) db[r] += ds;
        }
    }
    uint32_t w[2][3][4];
#pragma unroll
    for (int x = 0; x < 2; ++x) operand(w[x], s[2 * x], s[2 * x + 1]);
    sums<D, 2, 2>(dv, w, so);
#pragma unroll
    for (int x = 0; x < 2; ++x) operand(w[x], dp[2 * x], dp[2 * x + 1]);
    sums<D, 2, 2>(dk, w, sq);
  }
  __syncthreads();
  float* through = reinterpret_cast<float*>(Q) + group * 16 * (D + 4);
  float* other_db = reinterpret_cast<float*>(O + Tile<D>::kBytes);
#pragma unroll
  for (int r = 0; r < 2; ++r) db[r] = row_sum(db[r]);
  if (half) {
    leave<D>(through, dk);
    leave<D>(through + kT * (D + 4), dv);
    if ((lane & 3) == 0) {
      other_db[group * 16 + (lane >> 2)] = db[0];
      other_db[group * 16 + (lane >> 2) + 8] = db[1];
    }
  }
  __syncthreads();
  if (half) return;
  gather<D>(through, dk);
  gather<D>(through + kT * (D + 4), dv);
  const long long dst = at + (long long)group * 16 * ks;
  store<D>(static_cast<float*>(a.dk) + dst, ks, p.t1 - row0, dk, scale, scale);
  store<D>(static_cast<float*>(a.dv) + dst, ks, p.t1 - row0, dv, 1.f, 1.f);
  if (a.dbias && (lane & 3) == 0) {
#pragma unroll
    for (int r = 0; r < 2; ++r)
      if (mine + 8 * r < p.t1)
        static_cast<float*>(a.dbias)[(long long)hk * a.seqs.total + mine + 8 * r] =
            db[r] + other_db[group * 16 + (lane >> 2) + 8 * r];
  }
}

template <auto* kernel>
cudaError_t launch(const AttnArgs& a, int heads, int rows, int bytes, cudaStream_t stream) {
  const cudaError_t e = allow_shared<kernel>(bytes);
  if (e != cudaSuccess) return e;
  kernel<<<dim3((unsigned)pieces(a.seqs.total, a.seqs.num, rows), heads), kThreads, bytes, stream>>>(a);
  return cudaGetLastError();
}

template <int D>
constexpr int smem_bytes() {
  constexpr int bytes = 4 * Tile<D>::kBytes + 2 * kT * 4;
  static_assert(bytes <= 227 * 1024, "one block's shared memory");
  static_assert(2 * kT * (D + 4) * 4 <= 2 * Tile<D>::kBytes, "the second half's sums in the place of two tiles");
  return bytes;
}

}  // namespace

cudaError_t attn_forward_parts(const AttnArgs& a, int D, cudaStream_t stream) {
  return D == 128 ? launch<parts_forward_kernel<128>>(a, a.Hq, 2 * kT, smem_bytes<128>(), stream)
                  : launch<parts_forward_kernel<64>>(a, a.Hq, 2 * kT, smem_bytes<64>(), stream);
}
// (a.rows holds delta)
cudaError_t attn_backward_parts(const AttnArgs& a, int D, cudaStream_t stream) {
  const cudaError_t e = D == 128 ? launch<parts_dkv_kernel<128>>(a, a.Hkv, kT, smem_bytes<128>(), stream)
                                 : launch<parts_dkv_kernel<64>>(a, a.Hkv, kT, smem_bytes<64>(), stream);
  if (e != cudaSuccess) return e;
  return D == 128 ? launch<parts_dq_kernel<128>>(a, a.Hq, kT, smem_bytes<128>(), stream)
                  : launch<parts_dq_kernel<64>>(a, a.Hq, kT, smem_bytes<64>(), stream);
}

}  // namespace dmc
