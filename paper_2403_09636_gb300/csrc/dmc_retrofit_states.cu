// The relaxed compression's states and their gradient (Sec. 3.2, Eq.
// partial-accumulation with alpha in [0, 1]).
//
// With the unnormalised sums A_t = z_t k~_t (v alike, 2 D of them per token and
// head) the recurrence is linear:
//   A_t = alpha_t A_{t-1} + omega_t k_t,  z_t = alpha_t z_{t-1} + omega_t,  k~_t = A_t / z_t,
// and so is its gradient, from the last token to the first, with u_t = dk~_t / z_t
// and w_t = -(dk~_t . k~_t + dv~_t . v~_t) / z_t:
//   L_t = u_t + alpha_{t+1} L_{t+1},  Z_t = w_t + alpha_{t+1} Z_{t+1}
//   dk_t = omega_t L_t,  domega_t = L_t . k_t + Z_t,  dalpha_t = L_t . A_{t-1} + Z_t z_{t-1}
// (dots over k and v together). The sums are rebuilt from k, v and the sums at the
// chunk's start, which the forward pass saves in fp32: from the rounded states the
// difference that dalpha stands for would be lost where z is much larger than omega.
//
// A sequence is cut into chunks of 32 tokens, a warp per chunk, head and tensor (k or v): a token
// per lane for the gates, D / 32 neighbouring elements per lane for the rows, which each lane
// copies for itself to shared memory, once. A warp publishes the chunk's own sums and the
// product of its alphas, takes what comes in from the chunks before (after) it, and writes. What
// comes in follows the chain
//   in_{c+1} = own_c + prod_c in_c
// over its neighbours back to where the product of the alphas between falls below 2^-126 (nearly
// binary decisions: two or three chunks) or to the nearest of every 16th chunk, whose own `in`
// is waited for (dmc_chain.h). Where the chain begins follows from the data alone, so results do not depend on
// how far others have come. Chunks are taken from a counter, so that those a warp waits for have
// started; they publish before they wait. Every published number carries the number of the launch
// in the same 8 bytes: no fence or flag stands between it and its reader (a fence waited for
// the warp's loads and stores, 4 us of the 18 that a chunk took), and nothing has to be cleared
// between launches or replays of a graph.
//
// Bound by latency: a chunk is one chain of passes, scans and the wait for what comes in, and shared memory (9.5 KB
// per warp, 38.7 KB per two in the backward pass) leaves few warps per SM (30 and 15 % of the most) to fill the gaps: issue
// slots are 39 and 36 % busy, DRAM 48 and 33 %. Four sequences of 2048 tokens, 32 heads of 128, bf16: forward 70 us (272 MB,
// 3.9 TB/s), backward 156 us (407 MB, 2.6 TB/s: both dots of every token on top). Slower: warps that stay and take one chunk after another
// (backward 164; with chunks taken ahead, whose neighbours wait for one that has not begun, 217),
// rows read a second time from L2 instead of kept in shared memory (168 to 188).
#include <type_traits>

#include "dmc_chain.h"
#include "dmc_retrofit.cuh"

namespace dmc {

namespace {

constexpr int kC = kStateChunk;
constexpr int kPad = 4;  // z, the product of the chunk's alphas, and two unused

__host__ __device__ constexpr int sums_row(int D) { return 2 * D + kPad; }

// A token's gates, one token per lane; beyond the chunk's end the identity of the recurrence.
struct Gate {
  float alpha, rest, omega;  // rest: 1 - alpha; omega in units of 1 / kUnit
  float log_rest, slope;     // slope: of log(omega)
};

// Only ratios of the weights omega count, so they are kept larger by a power of two: sums of sigmoids
// far below the smallest fp32 number keep their bits, and those of others have the bits they have without. A
// mean of q[0] below kLeast counts as that, with 2^28 between the largest 1 / z and fp32's range.
constexpr float kUnit = 1152921504606846976.f;  // 2^60
constexpr float kLeast = -110.9f;               // omega kUnit = 2^-100

template <typename T>
__device__ __forceinline__ float element(const void* p, long long i) {
  return Elt<T>::to_f(static_cast<const T*>(p)[i]);
}

struct GateIn {
  float k, noise, q;
};
template <typename T, int D>
__device__ __forceinline__ GateIn gate_in(const StatesArgs& a, int h, int tok, bool in) {
  GateIn g = {0.f, 0.f, 0.f};
  if (!in) return g;
  g.k = element<T>(a.k, ((long long)tok * a.Hkv + h) * D);
  if (a.noise) g.noise = a.noise[(long long)h * a.seqs.total + tok];
#pragma unroll 8
  for (int j = 0; j < a.G; ++j) g.q += element<T>(a.q, (long long)tok * a.q_tok + (long long)(h * a.G + j) * a.q_head);
  return g;
}
// kUnit e^m for a mean m of the group's q[0] far below zero, as a product of numbers in range. The mean is taken again
// with what its sum and quotient round off: half a unit in the last place of -100 is 4e-6 of the weight.
template <typename T>
__device__ __noinline__ float small_omega(const StatesArgs& a, int h, int tok) {
  float sum = 0.f, rest = 0.f;
  for (int j = 0; j < a.G; ++j) {
    const float x = element<T>(a.q, (long long)tok * a.q_tok + (long long)(h * a.G + j) * a.q_head);
    const float to = sum + x, of_x = to - sum;
    rest += (sum - (to - of_x)) + (x - of_x);
    sum = to;
  }
  const float m = sum / (float)a.G;
  if (m < kLeast) return 7.88860905e-31f;  // 2^-100
  rest = (fmaf(-m, (float)a.G, sum) + rest) / (float)a.G;
  const float root = expf(0.5f * m);
  return root * kUnit * root * (1.f + rest);
}
template <typename T>
__device__ __forceinline__ Gate gate_of(const StatesArgs& a, GateIn v, int h, int tok, bool in, bool first) {
  Gate g;
  g.alpha = 1.f;
  g.rest = g.omega = g.log_rest = g.slope = 0.f;
  if (!in) return g;
  const float x = (v.k - a.offset + v.noise) / a.temperature;
  const float m = v.q / (float)a.G;
  if (m < -80.f) {
    g.omega = small_omega<T>(a, h, tok);
    g.slope = m < kLeast ? 0.f : 1.f;
  } else {
    const float e = expf(-m);
    g.omega = kUnit / (1.f + e);
    // 1 - omega, from the exponential where the difference would have lost its bits
    g.slope = m > 0.f ? e * (g.omega * (1.f / kUnit)) : 1.f - g.omega * (1.f / kUnit);
  }
  // both sides from the exponential that does not overflow
  const float e = expf(-fabsf(x)), big = 1.f / (1.f + e), small = e / (1.f + e);
  g.alpha = x >= 0.f ? big : small;
  g.rest = x >= 0.f ? small : big;
  if (x != x) g.alpha = g.rest = x;
  g.log_rest = -(fmaxf(x, 0.f) + log1pf(e));
  if (first) {
    g.alpha = 0.f;
    g.rest = 1.f;
  }
  return g;
}

// z of the 32 tokens, given z before the first; one token per lane.
__device__ __forceinline__ float scan_z(float alpha, float omega, float before) {
  const int lane = threadIdx.x & 31;
  float a = alpha, z = omega;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const float oa = __shfl_up_sync(0xffffffffu, a, off), oz = __shfl_up_sync(0xffffffffu, z, off);
    if (lane >= off) {
      z = fmaf(a, oz, z);
      a *= oa;
    }
  }
  return fmaf(a, before, z);
}

// ---- a lane's elements of a row

template <typename T, int D>
struct Row {
  static constexpr int kE = D / 32, kP = kE / 2;  // elements and pairs per lane
  static constexpr int kBytes = kE * (int)sizeof(T);
  using Word = typename std::conditional<kBytes == 4, uint32_t, typename std::conditional<kBytes == 8, uint2, uint4>::type>::type;

  static __device__ __forceinline__ void zero(T* at) { *reinterpret_cast<Word*>(at) = Word{}; }
  static __device__ __forceinline__ void read(const T* at, float2 (&f)[kP]) {
    const Word u = *reinterpret_cast<const Word*>(at);
    const typename Pair<T>::Raw* r = reinterpret_cast<const typename Pair<T>::Raw*>(&u);
#pragma unroll
    for (int i = 0; i < kP; ++i) f[i] = Pair<T>::to_f(r[i]);
  }
  static __device__ __forceinline__ void write(T* at, const float2 (&f)[kP]) {
    Word u;
    typename Pair<T>::Raw* r = reinterpret_cast<typename Pair<T>::Raw*>(&u);
#pragma unroll
    for (int i = 0; i < kP; ++i) r[i] = Pair<T>::from_f(f[i]);
    *reinterpret_cast<Word*>(at) = u;
  }
};

__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// n rows of D elements, `stride` elements apart, by a warp: a row per lane, completing on `bar`
template <typename T, int D>
__device__ __forceinline__ void load_chunk(T* to, const T* from, long long stride, int n, uint32_t bar) {
  const int lane = threadIdx.x & 31;
  if (lane < n)
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                     smem_u32(to + lane * D)),
                 "l"(from + lane * stride), "n"(D * (int)sizeof(T)), "r"(bar)
                 : "memory");
}

// A token's numbers for the passes over its elements, each twice: the two halves of a paired
// operation
struct Coef {
  float4 alpha_omega;  // alpha, alpha, omega, omega
  float4 rz_other;     // 1 / z, 1 / z; backward: the product of the alphas up to the token over z, twice
};
__device__ __forceinline__ float2 lo2(float4 f) { return make_float2(f.x, f.y); }
__device__ __forceinline__ float2 hi2(float4 f) { return make_float2(f.z, f.w); }

// ---- the order of warps

// words of StatesArgs::turns, each in a line of its own (everybody adds to the first two)
constexpr int kCome = 0, kGone = 32, kLaunch = 64, kStop = 96;  // kStop: the launch whose waits have to end

struct Turn {
  int index;         // in the order in which they come
  unsigned int tag;  // the launch
};
// one thread
__device__ __forceinline__ Turn take_turn(const StatesArgs& a) {
  Turn t;
  t.index = (int)atomicAdd(&a.turns[kCome], 1u);
  t.tag = *reinterpret_cast<volatile unsigned int*>(&a.turns[kLaunch]) + 1;
  return t;
}
// One thread, when its block has read all it needs from others; the last one prepares the next launch.
__device__ __forceinline__ void leave(const StatesArgs& a, const Turn& t) {
  if (atomicAdd(&a.turns[kGone], 1u) != gridDim.x - 1) return;
  a.turns[kCome] = a.turns[kGone] = 0;
  a.turns[kLaunch] = t.tag;
}

// Faulty cu_seqlens, where a chunk may have no neighbour, end this launch's waits (the fault bits stay from call
// to call and say nothing about it). One block.
__device__ __forceinline__ void check_seqs(const StatesArgs& a, unsigned int tag) {
  if (check_seqs(a.seqs, a.error)) *reinterpret_cast<volatile unsigned int*>(&a.turns[kStop]) = tag;
}

// ---- published numbers: {value, launch}

__device__ __forceinline__ uint64_t tagged(float x, unsigned int tag) { return (uint64_t)tag << 32 | __float_as_uint(x); }

template <int kE>
__device__ __forceinline__ void publish(uint64_t* row, const float2* f, unsigned int tag) {
  uint64_t* at = row + (threadIdx.x & 31) * kE;
#pragma unroll
  for (int i = 0; i < kE / 2; ++i)
    asm volatile("st.relaxed.gpu.global.v2.b64 [%0], {%1, %2};" ::"l"(at + 2 * i), "l"(tagged(f[i].x, tag)),
                 "l"(tagged(f[i].y, tag))
                 : "memory");
}
// z and the product of the chunk's alphas, by one lane
template <int D>
__device__ __forceinline__ void publish_zp(uint64_t* row, float z, float prod, unsigned int tag) {
  asm volatile("st.relaxed.gpu.global.v2.b64 [%0], {%1, %2};" ::"l"(row + D), "l"(tagged(z, tag)), "l"(tagged(prod, tag))
               : "memory");
}
__device__ __forceinline__ bool look_two(const uint64_t* at, float2& f, unsigned int tag) {
  uint64_t u, v;
  asm volatile("ld.relaxed.gpu.global.v2.b64 {%0, %1}, [%2];" : "=l"(u), "=l"(v) : "l"(at) : "memory");
  f = make_float2(__uint_as_float((unsigned int)u), __uint_as_float((unsigned int)v));
  return (unsigned int)(u >> 32) == tag && (unsigned int)(v >> 32) == tag;
}
// A row's z and product; the lane's elements of a row; whether they were there.
template <int D>
__device__ __forceinline__ bool look_zp(const uint64_t* row, float2& zp, unsigned int tag) {
  return look_two(row + D, zp, tag);
}
template <int D>
__device__ __forceinline__ bool look(const uint64_t* row, float2 (&f)[D / 64], unsigned int tag) {
  bool there = true;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) there &= look_two(row + (threadIdx.x & 31) * (D / 32) + 2 * i, f[i], tag);
  return there;
}
// After tries that found nothing, by a whole warp: whether to give up, since this has taken too long or
// another wait of the launch has (or its cu_seqlens do not fit).
__device__ __forceinline__ bool give_up(uint64_t& since, const StatesArgs& a, unsigned int tag) {
  __nanosleep(500);
  volatile unsigned int* stop = &a.turns[kStop];
  bool over = *stop == tag;
  const uint64_t t = globaltimer_ns();
  if (since == 0) since = t;
  if (t - since > kWaitLimitNs) {
    atomicOr(a.error, DMC_FAULT_WAIT_TIMEOUT);
    *stop = tag;
    over = true;
  }
  return __any_sync(0xffffffffu, over);
}
template <int D>
__device__ __forceinline__ void await(const StatesArgs& a, const uint64_t* row, float2 (&f)[D / 64], unsigned int tag) {
  uint64_t since = 0;
  for (int tries = 0; !__all_sync(0xffffffffu, look<D>(row, f, tag)); ++tries)
    if (tries >= 64 && give_up(since, a, tag)) return;
}

// What comes into a chunk from its n > 0 neighbours on one side, `step` apart: the lane's sums x,
// and z (Z). own, in: this chunk's rows.
template <int D>
__device__ __forceinline__ float come_in(const StatesArgs& a, const uint64_t* own, const uint64_t* in, int n, long long step,
                                         unsigned int tag, float2 (&x)[D / 64]) {
  constexpr int kP = D / 64;
  const int lane = threadIdx.x & 31, d = chain_reach(n);
  // a neighbour per lane: its z and the product of its alphas
  float2 zp = make_float2(0.f, 1.f);
  uint64_t since = 0;
  for (int tries = 0;; ++tries) {
    const bool there = lane >= d || look_zp<D>(own + (lane + 1) * step, zp, tag);
    if (__all_sync(0xffffffffu, there)) break;
    if (tries >= 64 && give_up(since, a, tag)) break;
  }
  float upto = zp.y;  // the product of the nearest lane + 1
#pragma unroll
  for (int off = 1; off < kAnchor; off <<= 1) {
    const float o = __shfl_up_sync(0xffffffffu, upto, off);
    if (lane >= off) upto *= o;
  }
  const unsigned int end = __ballot_sync(0xffffffffu, lane < d && chain_ends(zp.y, upto));
  const int far = end ? __ffs(end) : d;
  float z = 0.f;
#pragma unroll
  for (int i = 0; i < kP; ++i) x[i] = both(0.f);
  if (!end && d < n) {
    float2 zi;
    await<D>(a, in + d * step, x, tag);
    for (int tries = 0; !__all_sync(0xffffffffu, look_zp<D>(in + d * step, zi, tag)); ++tries)
      if (tries >= 64 && give_up(since, a, tag)) break;
    z = zi.x;
  }
  float2 o[kP], next[kP];
  bool there = look<D>(own + far * step, o, tag);
#pragma unroll 1
  for (int i = far; i > 0; --i) {
    bool soon = true;
    if (i > 1) soon = look<D>(own + (i - 1) * step, next, tag);
    if (!__all_sync(0xffffffffu, there)) await<D>(a, own + i * step, o, tag);
    const float zo = __shfl_sync(0xffffffffu, zp.x, i - 1), prod = __shfl_sync(0xffffffffu, zp.y, i - 1);
#pragma unroll
    for (int k = 0; k < kP; ++k) {
      x[k] = fma2(both(prod), x[k], o[k]);
      o[k] = next[k];
    }
    z = fmaf(prod, z, zo);
    there = soon;
  }
  return z;
}

template <int D>
__device__ __forceinline__ long long row_of(const StatesArgs& a, int chunk, int h, int which) {
  return (((long long)chunk * a.Hkv + h) * 2 + which) * (D + 2);
}

template <typename T, int D>
__global__ void __launch_bounds__(32) states_kernel(const StatesArgs a) {
  using R = Row<T, D>;
  __shared__ __align__(128) T rows[kC * D];
  __shared__ Coef coef[kC];
  __shared__ float2 weight[kC];  // omega times the product of the alphas after it, twice
  __shared__ uint64_t loaded;
  const int lane = threadIdx.x;
  Turn turn;
  if (lane == 0) {
    mbar_init(smem_u32(&loaded), 1);
    fence_mbar_init();
    turn = take_turn(a);
  }
  turn.index = __shfl_sync(0xffffffffu, turn.index, 0);
  turn.tag = __shfl_sync(0xffffffffu, turn.tag, 0);
  const int which = turn.index & 1, h = (turn.index >> 1) % a.Hkv, chunk = (turn.index >> 1) / a.Hkv;  // which: 0 k, 1 v
  if (turn.index == 0) check_seqs(a, turn.tag);
  const Piece p = find_piece(a.seqs, kC, chunk);
  if (!p.ok) {
    if (lane == 0) leave(a, turn);
    return;
  }
  const int tok0 = p.t0 + p.at * kC, n = min(kC, p.t1 - tok0), tok = tok0 + lane;
  const bool in_chunk = lane < n, goes_on = tok0 + kC < p.t1;
  const GateIn gi = gate_in<T, D>(a, h, tok, in_chunk);
  const long long step = (long long)a.Hkv * D, at = ((long long)tok0 * a.Hkv + h) * D;
  T* mine = rows + lane * R::kE;
  if (lane == 0) mbar_arrive_expect_tx(smem_u32(&loaded), n * D * sizeof(T));
  __syncwarp();
  load_chunk<T, D>(rows, static_cast<const T*>(which ? a.v : a.k) + at, step, n, smem_u32(&loaded));
  const Gate g = gate_of<T>(a, gi, h, tok, in_chunk, tok == p.t0);
  const long long row = row_of<D>(a, chunk, h, which), row_step = row_of<D>(a, 1, 0, 0);
  float after = g.alpha;  // product of the alphas from the token on
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const float o = __shfl_down_sync(0xffffffffu, after, off);
    if (lane + off < 32) after *= o;
  }
  const float prod = __shfl_sync(0xffffffffu, after, 0);
  if (goes_on) {
    const float rest = __shfl_down_sync(0xffffffffu, after, 1);
    const float w = g.omega * (lane == 31 ? 1.f : rest);
    weight[lane] = both(w);
    float z = w;
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) z += __shfl_xor_sync(0xffffffffu, z, off);
    if (lane == 0) publish_zp<D>(a.sums + row, z, prod, turn.tag);
  }
  mbar_wait(smem_u32(&loaded), 0, a.error);  // (if it gives up, the fault bit is set and the results mean nothing)
  if (which == 0 && in_chunk) rows[lane * D] = Elt<T>::from_f(0.f);  // k's first component is the gate
  __syncwarp();
  float2 sum[R::kP];
#pragma unroll
  for (int i = 0; i < R::kP; ++i) sum[i] = both(0.f);
  if (goes_on) {
#pragma unroll 8
    for (int t = 0; t < kC; ++t) {
      float2 x[R::kP];
      R::read(mine + t * D, x);
      const float2 w = weight[t];
#pragma unroll
      for (int i = 0; i < R::kP; ++i) sum[i] = fma2(w, x[i], sum[i]);
    }
    publish<R::kE>(a.sums + row, sum, turn.tag);
  }
  float zin = 0.f;
#pragma unroll
  for (int i = 0; i < R::kP; ++i) sum[i] = both(0.f);
  if (p.at > 0) {
    zin = come_in<D>(a, a.sums + row, a.carry + row, p.at, -row_step, turn.tag, sum);
    if (goes_on && asked_for(p.at, prod)) {
      publish<R::kE>(a.carry + row, sum, turn.tag);
      if (lane == 0) publish_zp<D>(a.carry + row, zin, 0.f, turn.tag);
    }
    float* saved = a.saved + ((long long)chunk * a.Hkv + h) * sums_row(D);
#pragma unroll
    for (int i = 0; i < R::kP; ++i) *reinterpret_cast<float2*>(saved + which * D + lane * R::kE + 2 * i) = sum[i];
    if (which == 0 && lane == 0) saved[2 * D] = zin;
  }
  if (lane == 0) leave(a, turn);
  const float rz = 1.f / scan_z(g.alpha, g.omega, zin);
  coef[lane].alpha_omega = make_float4(g.alpha, g.alpha, g.omega, g.omega);
  coef[lane].rz_other = make_float4(rz, rz, 0.f, 0.f);
  __syncwarp();
  T* dst = static_cast<T*>(which ? a.vt : a.kt) + at + lane * R::kE;
#pragma unroll 8
  for (int t = 0; t < n; ++t) {
    float2 x[R::kP], y[R::kP];
    R::read(mine + t * D, x);
    const float4 ao = coef[t].alpha_omega;
    const float2 z = *reinterpret_cast<const float2*>(&coef[t].rz_other);
#pragma unroll
    for (int i = 0; i < R::kP; ++i) {
      sum[i] = fma2(lo2(ao), sum[i], mul2(hi2(ao), x[i]));
      y[i] = mul2(z, sum[i]);
    }
    R::write(dst + t * step, y);
  }
  if (in_chunk && which == 0) {
    const long long i = (long long)h * a.seqs.total + tok;
    a.alpha[i] = g.alpha;
    if (tok > p.t0) a.bias[i - 1] = g.log_rest;
    if (tok == p.t1 - 1) a.bias[i] = 0.f;
  }
}

// Chunks from the last to the first, a block of a warp for k and a warp for v per chunk and
// head. A chunk passes on the sum over t of (its alphas up to t) u_t, and w_t alike. Dots over all
// elements go through shared memory: 16 partial sums per token, then a token per lane.
constexpr int kOfZeta = 0, kOfOmega = 1, kOfSum = 2;  // rows of `other`
template <typename T, int D>
struct BackShared {
  T rows[2][kC * D], grads[2][kC * D];
  Coef coef[2][kC];
  float dots[2][kC][17];
  float other[3][kC];         // v's shares of the dots, a row each: what one warp reads the other does not write again
  uint64_t loaded[2];
  Turn turn;
};

template <typename T, int D>
__global__ void __launch_bounds__(64) states_backward_kernel(const StatesArgs a) {
  using R = Row<T, D>;
  constexpr int kH = kC / 2;  // tokens whose sums are held at a time
  extern __shared__ __align__(16) char raw[];
  BackShared<T, D>& sh = *reinterpret_cast<BackShared<T, D>*>(raw);
  const int lane = threadIdx.x & 31, which = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&sh.loaded[i]), 1);
    fence_mbar_init();
    sh.turn = take_turn(a);
  }
  __syncthreads();
  const Turn turn = sh.turn;
  const int chunks = gridDim.x / a.Hkv, h = turn.index % a.Hkv, chunk = chunks - 1 - turn.index / a.Hkv;
  if (turn.index == 0) check_seqs(a, turn.tag);
  const Piece p = find_piece(a.seqs, kC, chunk);
  if (!p.ok) {
    if (threadIdx.x == 0) leave(a, turn);
    return;
  }
  const int tok0 = p.t0 + p.at * kC, n = min(kC, p.t1 - tok0), tok = tok0 + lane;
  const int after = (p.t1 - p.t0 + kC - 1) / kC - 1 - p.at;  // chunks after this one
  const bool in_chunk = lane < n;
  const GateIn gi = gate_in<T, D>(a, h, tok, in_chunk);
  const long long step = (long long)a.Hkv * D, at = ((long long)tok0 * a.Hkv + h) * D;
  T *mine = sh.rows[which] + lane * R::kE, *grads = sh.grads[which] + lane * R::kE;
  const uint32_t bar = smem_u32(&sh.loaded[which]);
  if (lane == 0) mbar_arrive_expect_tx(bar, 2 * n * D * sizeof(T));
  __syncwarp();
  load_chunk<T, D>(sh.rows[which], static_cast<const T*>(which ? a.v : a.k) + at, step, n, bar);
  load_chunk<T, D>(sh.grads[which], static_cast<const T*>(which ? a.dvt : a.dkt) + at, step, n, bar);
  // tokens from n on: zeros, and alpha 1, so that they change nothing
  for (int t = n; t < kC; ++t) {
    R::zero(mine + t * D);
    R::zero(grads + t * D);
  }
  const float* saved = a.saved + ((long long)chunk * a.Hkv + h) * sums_row(D);
  float2 sum0[R::kP], middle[R::kP];  // the sums before the chunk, before its second half
#pragma unroll
  for (int i = 0; i < R::kP; ++i) sum0[i] = both(0.f);
  float zbefore0 = 0.f, dbias = 0.f, dalpha = 0.f;
  if (p.at > 0) {
#pragma unroll
    for (int i = 0; i < R::kP; ++i) sum0[i] = *reinterpret_cast<const float2*>(saved + which * D + lane * R::kE + 2 * i);
    zbefore0 = saved[2 * D];
  }
  if (which == 0 && in_chunk && tok > p.t0) {
    const long long i = (long long)h * a.seqs.total + tok;
    dbias = element<T>(a.dbias, i - 1);
    if (a.dalpha) dalpha = a.dalpha[i];
  }
  const Gate g = gate_of<T>(a, gi, h, tok, in_chunk, tok == p.t0);
  const float z = scan_z(g.alpha, g.omega, zbefore0), rz = 1.f / z;
  float prod = g.alpha;  // of the alphas up to the token
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const float o = __shfl_up_sync(0xffffffffu, prod, off);
    if (lane >= off) prod *= o;
  }
  const float prod_all = __shfl_sync(0xffffffffu, prod, 31);
  const Coef* coef = sh.coef[which];
  sh.coef[which][lane].alpha_omega = make_float4(g.alpha, g.alpha, g.omega, g.omega);
  sh.coef[which][lane].rz_other = make_float4(rz, rz, prod * rz, prod * rz);
  // two dots, the 16 partial sums of one in row t, those of the other in row t + 16
  auto put = [&](int t, float2 c, float2 d) {
    const float x = c.x + c.y, y = d.x + d.y;
    const bool up = lane & 16;
    const float sum = (up ? y : x) + __shfl_xor_sync(0xffffffffu, up ? x : y, 16);
    sh.dots[which][t + (lane & 16)][lane & 15] = sum;
  };
  auto take = [&]() {  // the dot of the lane's row
    __syncwarp();
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) x += sh.dots[which][lane][i];
    __syncwarp();
    return x;
  };
  mbar_wait(bar, 0, a.error);  // (if it gives up, the fault bit is set and the results mean nothing)
  if (which == 0) {  // k's first component is the gate
    sh.rows[0][lane * D] = Elt<T>::from_f(0.f);
    sh.grads[0][lane * D] = Elt<T>::from_f(0.f);
  }
  __syncwarp();
  const long long row = row_of<D>(a, chunk, h, which), row_step = row_of<D>(a, 1, 0, 0);
  // forward over the chunk: the sums, g . A, and what the chunk passes on
  {
    float2 sum[R::kP], pass[R::kP];
#pragma unroll
    for (int i = 0; i < R::kP; ++i) {
      sum[i] = sum0[i];
      pass[i] = both(0.f);
    }
#pragma unroll 8
    for (int t = 0; t < kC; ++t) {
      float2 x[R::kP], gr[R::kP], d = both(0.f);
      R::read(mine + t * D, x);
      R::read(grads + t * D, gr);
      const float4 ao = coef[t].alpha_omega;
      const float2 w = hi2(coef[t].rz_other);
      if (t == kH)
#pragma unroll
        for (int i = 0; i < R::kP; ++i) middle[i] = sum[i];
#pragma unroll
      for (int i = 0; i < R::kP; ++i) {
        sum[i] = fma2(lo2(ao), sum[i], mul2(hi2(ao), x[i]));
        d = fma2(gr[i], sum[i], d);
        pass[i] = fma2(w, gr[i], pass[i]);
      }
      const float one = d.x + d.y;  // 16 partial sums, written by both halves of the warp
      sh.dots[which][t][lane & 15] = one + __shfl_xor_sync(0xffffffffu, one, 16);
    }
    if (p.at > 0) publish<R::kE>(a.sums + row, pass, turn.tag);
  }
  float zeta = take();
  if (which) sh.other[kOfZeta][lane] = zeta;
  __syncthreads();
  zeta = in_chunk ? -(zeta + sh.other[kOfZeta][lane]) * rz * rz : 0.f;  // (of use to the first warp)
  if (p.at > 0) {
    float s = zeta * prod;
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    if (lane == 0) publish_zp<D>(a.sums + row, which ? 0.f : s, prod_all, turn.tag);
  }
  float2 in[R::kP];  // alpha L of the next token
  float zin = 0.f;
#pragma unroll
  for (int i = 0; i < R::kP; ++i) in[i] = both(0.f);
  if (after > 0) {
    zin = come_in<D>(a, a.sums + row, a.carry + row, after, row_step, turn.tag, in);
    if (p.at > 0 && asked_for(after, prod_all)) {
      publish<R::kE>(a.carry + row, in, turn.tag);
      if (lane == 0) publish_zp<D>(a.carry + row, zin, 0.f, turn.tag);
    }
  }
  // from the last token to the first, half a chunk at a time: L, and its dots with the
  // values and with the sums before
  T* dst = static_cast<T*>(which ? a.dv : a.dk) + at + lane * R::kE;
  float domega = 0.f, dsum = 0.f;
#pragma unroll 1
  for (int half = 1; half >= 0; --half) {
    const int t0 = half * kH;
    float2 A[kH][R::kP], sum[R::kP];  // the sums before token t0 + j
#pragma unroll
    for (int i = 0; i < R::kP; ++i) sum[i] = half ? middle[i] : sum0[i];
#pragma unroll
    for (int j = 0; j < kH; ++j) {
      float2 x[R::kP];
      R::read(mine + (t0 + j) * D, x);
      const float4 ao = coef[t0 + j].alpha_omega;
#pragma unroll
      for (int i = 0; i < R::kP; ++i) {
        A[j][i] = sum[i];
        sum[i] = fma2(lo2(ao), sum[i], mul2(hi2(ao), x[i]));
      }
    }
#pragma unroll
    for (int j = kH - 1; j >= 0; --j) {
      const int t = t0 + j;
      float2 x[R::kP], gr[R::kP], dx = both(0.f), da = both(0.f), out[R::kP];
      R::read(mine + t * D, x);
      R::read(grads + t * D, gr);
      const float4 ao = coef[t].alpha_omega;
      const float2 z2 = lo2(coef[t].rz_other);
#pragma unroll
      for (int i = 0; i < R::kP; ++i) {
        const float2 l = fma2(gr[i], z2, in[i]);
        dx = fma2(l, x[i], dx);
        da = fma2(l, A[j][i], da);
        out[i] = mul2(hi2(ao), l);
        in[i] = mul2(lo2(ao), l);
      }
      put(j, dx, da);
      if (t < n) R::write(dst + t * step, out);  // (the first component of dk comes below)
    }
    // lanes 0-15: with the values, 16-31: with the sums; to the lanes of their tokens
    const float d = take();
    const float lo = __shfl_sync(0xffffffffu, d, lane & 15), hi = __shfl_sync(0xffffffffu, d, 16 + (lane & 15));
    if (lane >> 4 == half) {
      domega = lo;
      dsum = hi;
    }
  }
  if (which) {
    sh.other[kOfOmega][lane] = domega;
    sh.other[kOfSum][lane] = dsum;
  }
  __syncthreads();
  if (which) return;
  if (lane == 0) leave(a, turn);
  // Z_t = w_t + alpha_{t+1} Z_{t+1}; what comes in has its alpha already, and lanes from n on
  // are the identity (alpha 1, w 0)
  float next = __shfl_down_sync(0xffffffffu, g.alpha, 1);
  if (lane == 31) {
    next = 0.f;
    zeta += zin;
  }
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const float on = __shfl_down_sync(0xffffffffu, next, off), oz = __shfl_down_sync(0xffffffffu, zeta, off);
    if (lane + off < 32) {
      zeta = fmaf(next, oz, zeta);
      next *= on;
    }
  }
  float zbefore = __shfl_up_sync(0xffffffffu, z, 1);
  if (lane == 0) zbefore = zbefore0;
  if (in_chunk) {
    domega += sh.other[kOfOmega][lane] + zeta;
    dalpha += dsum + sh.other[kOfSum][lane] + zeta * zbefore;
    float dx = 0.f;
    if (tok > p.t0) dx = (dalpha * g.alpha * g.rest - dbias * g.alpha) / a.temperature;
    // over what lane 0 has written there
    static_cast<T*>(a.dk)[((long long)tok * a.Hkv + h) * D] = Elt<T>::from_f(dx);
    const T dq = Elt<T>::from_f(domega * g.omega * g.slope / (float)a.G);
    for (int j = 0; j < a.G; ++j)
      static_cast<T*>(a.dq)[(long long)tok * a.dq_tok + (long long)(h * a.G + j) * a.dq_head] = dq;
  }
}

template <typename T, int D>
cudaError_t forward(const StatesArgs& a, cudaStream_t stream) {
  states_kernel<T, D><<<(unsigned)(pieces(a.seqs.total, a.seqs.num, kC) * a.Hkv * 2), 32, 0, stream>>>(a);
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t backward(const StatesArgs& a, cudaStream_t stream) {
  constexpr int bytes = sizeof(BackShared<T, D>);
  const cudaError_t e = allow_shared<states_backward_kernel<T, D>>(bytes);
  if (e != cudaSuccess) return e;
  states_backward_kernel<T, D><<<(unsigned)(pieces(a.seqs.total, a.seqs.num, kC) * a.Hkv), 64, bytes, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t states_forward(const StatesArgs& a, bool bf16, int D, cudaStream_t stream) {
  if (bf16) return D == 128 ? forward<__nv_bfloat16, 128>(a, stream) : forward<__nv_bfloat16, 64>(a, stream);
  return D == 128 ? forward<float, 128>(a, stream) : forward<float, 64>(a, stream);
}
cudaError_t states_backward(const StatesArgs& a, bool bf16, int D, cudaStream_t stream) {
  if (bf16) return D == 128 ? backward<__nv_bfloat16, 128>(a, stream) : backward<__nv_bfloat16, 64>(a, stream);
  return D == 128 ? backward<float, 128>(a, stream) : backward<float, 64>(a, stream);
}

}  // namespace dmc
