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
// A sequence is cut into chunks of 32 tokens, a block per chunk and head with two
// neighbouring elements of k or v per thread, which reads its tokens once: it publishes the
// chunk's own sums and the product of its alphas, takes what comes in from the chunks before
// (after) it, and writes. What comes in follows the chain
//   in_{c+1} = own_c + prod_c in_c
// from the nearest chunk whose own `in` is known or whose product is 0: decisions that are
// nearly binary make the product of 32 alphas underflow, so that mostly one chunk is looked
// at. The chain is always evaluated in this order, so results do not depend on how far others
// have come. Blocks take their chunks from a counter, so that those a block waits for
// have started; they publish before they wait. Flags carry the launch's number, kept in
// device memory, so that nothing has to be cleared between launches (or replays of a graph).
#include "dmc_retrofit.cuh"

namespace dmc {

namespace {

constexpr int kC = kStateChunk;
constexpr int kPad = 4;  // z, the product of the chunk's alphas, and two unused

__host__ __device__ constexpr int sums_row(int D) { return 2 * D + kPad; }

// A token's gates, one token per lane; beyond the chunk's end the identity of the recurrence.
struct Gate {
  float alpha, rest, omega;  // rest: 1 - alpha
  float log_rest;
};

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
__device__ __forceinline__ Gate gate_of(const StatesArgs& a, GateIn v, bool in, bool first) {
  Gate g;
  g.alpha = 1.f;
  g.rest = g.omega = g.log_rest = 0.f;
  if (!in) return g;
  const float x = (v.k - a.offset + v.noise) / a.temperature;
  g.omega = 1.f / (1.f + expf(-v.q / (float)a.G));
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

// Of 32 values per lane: lane t gets the sum of all lanes' v[t].
__device__ __forceinline__ float transposed_sum(float* v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) {
    const bool up = lane & off;
#pragma unroll
    for (int i = 0; i < off; ++i) {
      const float send = up ? v[i] : v[i + off], keep = up ? v[i + off] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, off);
    }
  }
  return v[0];
}

template <int D>
struct StatesShared {
  float alpha[kC], omega[kC], rz[kC];
  float prod[kC];       // product of the alphas up to the token
  float dot[3][D / 32][kC];
  float e1[kC];         // second element of dk
  float zin;            // z (Z) that comes in
  int index, far;
  bool known;
  unsigned int launch;
};

// A chunk's rows of two tensors in shared memory: [tensor][token][D]
template <typename T, int D>
__device__ __forceinline__ void load_chunk(char* to, const void* k, const void* v, long long row, long long stride, int n) {
  constexpr int kRow = D * sizeof(T), kPieces = kRow / 16;
  for (int i = threadIdx.x; i < 2 * n * kPieces; i += D) {
    const int c = i % kPieces, t = i / kPieces % n, w = i / (kPieces * n);
    cp_async16(smem_u32(to) + (w * kC + t) * kRow + c * 16,
               static_cast<const char*>(w ? v : k) + (row + t * stride) * sizeof(T) + c * 16);
  }
}

// ---- the order of blocks

// words of StatesArgs::turns, each in a line of its own (all blocks add to the first two)
constexpr int kCome = 0, kGone = 32, kLaunch = 64;

// The block's chunk and head, in the order in which blocks come.
template <int D>
__device__ __forceinline__ int take_turn(const StatesArgs& a, StatesShared<D>& sh) {
  if (threadIdx.x == 0) {
    sh.index = (int)atomicAdd(&a.turns[kCome], 1u);
    sh.launch = *reinterpret_cast<volatile unsigned int*>(&a.turns[kLaunch]);
  }
  __syncthreads();
  return sh.index;
}
// Thread 0, when the block needs no other any more: how many have come so far before it.
__device__ __forceinline__ unsigned int gone(const StatesArgs& a) { return atomicAdd(&a.turns[kGone], 1u); }
// The last block prepares the next launch.
__device__ __forceinline__ void leave(const StatesArgs& a, unsigned int before, unsigned int launch) {
  if (before != gridDim.x - 1) return;
  a.turns[kCome] = a.turns[kGone] = 0;
  a.turns[kLaunch] = launch + 1;
}

constexpr unsigned int kOwn = 1, kIn = 2;  // published: the chunk's own sums; what comes into it, too

// By the whole block, after its values have been written.
__device__ __forceinline__ void publish(unsigned int* flag, unsigned int launch, unsigned int what) {
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(flag), "r"(launch << 2 | what) : "memory");
  }
}
// What a chunk has published, once there is something. 0: waited too long, or a fault has been
// found (a wait that gave up, or cu_seqlens that do not fit, where a chunk may have no neighbour).
__device__ __forceinline__ unsigned int published(const unsigned int* flag, unsigned int launch, unsigned int* error) {
  uint64_t since = 0;
  for (int tries = 0;; ++tries) {
    unsigned int f;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(f) : "l"(flag) : "memory");
    if (f >> 2 == (launch & 0x3fffffffu) && (f & 3)) return f & 3;
    if (tries < 64) continue;
    __nanosleep(500);
    if (*reinterpret_cast<volatile unsigned int*>(error)) return 0;
    const uint64_t t = globaltimer_ns();
    if (since == 0) since = t;
    if (t - since > kWaitLimitNs) {
      atomicOr(error, DMC_FAULT_WAIT_TIMEOUT);
      return 0;
    }
  }
}

// What comes into a chunk from its neighbours `dir` (-1: before it, 1: after it), of which
// there are `n`: the thread's pair of sums, and z (Z) in `zin`. own, in: the neighbours' rows.
template <int D>
__device__ __forceinline__ float2 come_in(const StatesArgs& a, StatesShared<D>& sh, const float* own, const float* in,
                                          int chunk, int h, int n, int dir, unsigned int launch, float& zin) {
  const int tid = threadIdx.x;
  const long long stride = (long long)a.Hkv * sums_row(D);
  own += ((long long)chunk * a.Hkv + h) * sums_row(D);
  in += ((long long)chunk * a.Hkv + h) * sums_row(D);
  if (tid == 0) {  // how many chunks to look at, and whether what came into the last is known
    int far = 0;
    unsigned int f = kOwn;
    while (far < n && f == kOwn) {
      ++far;
      f = published(a.flags + (long long)(chunk + dir * far) * a.Hkv + h, launch, a.error);
      if (__ldcg(own + dir * far * stride + 2 * D + 1) == 0.f) f = 0;
    }
    sh.far = far;
    sh.known = f == kIn;
  }
  __syncthreads();
  int far = sh.far;
  const bool known = sh.known;
  const float* row = own + dir * far * stride;
  float2 x = make_float2(0.f, 0.f), o = __ldcg(reinterpret_cast<const float2*>(row) + tid);
  float2 zp = __ldcg(reinterpret_cast<const float2*>(row + 2 * D));  // z, product
  zin = 0.f;
  if (known) {
    x = __ldcg(reinterpret_cast<const float2*>(in + dir * far * stride) + tid);
    zin = __ldcg(in + dir * far * stride + 2 * D);
  }
  while (true) {
    x.x = fmaf(zp.y, x.x, o.x);
    x.y = fmaf(zp.y, x.y, o.y);
    zin = fmaf(zp.y, zin, zp.x);
    if (--far == 0) return x;
    row = own + dir * far * stride;
    o = __ldcg(reinterpret_cast<const float2*>(row) + tid);
    zp = __ldcg(reinterpret_cast<const float2*>(row + 2 * D));
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(D) states_kernel(const StatesArgs a) {
  using P = Pair<T>;
  using Raw = typename P::Raw;
  __shared__ StatesShared<D> sh;
  __shared__ __align__(16) T rows[2 * kC * D];
  const int tid = threadIdx.x, lane = tid & 31;
  const int index = take_turn(a, sh), h = index % a.Hkv, chunk = index / a.Hkv;
  const unsigned int launch = sh.launch;
  if (index == 0) check_seqs(a.seqs, a.error);
  const Piece p = find_piece(a.seqs, kC, chunk);
  if (!p.ok) {
    if (tid == 0) leave(a, gone(a), launch);
    return;
  }
  const int tok0 = p.t0 + p.at * kC, n = min(kC, p.t1 - tok0);
  const bool in = lane < n, goes_on = tok0 + kC < p.t1;
  GateIn gi;
  if (tid < 32) gi = gate_in<T, D>(a, h, tok0 + lane, in);
  const long long row0 = ((long long)tok0 * a.Hkv + h) * D, step = (long long)a.Hkv * D;
  load_chunk<T, D>(reinterpret_cast<char*>(rows), a.k, a.v, row0, step, n);
  cp_async_commit();
  float* own = a.sums + ((long long)chunk * a.Hkv + h) * sums_row(D);
  Gate g;
  float prod = 1.f;
  if (tid < 32) {
    g = gate_of(a, gi, in, tok0 + lane == p.t0);
    sh.alpha[lane] = g.alpha;
    sh.omega[lane] = g.omega;
    const float z = scan_z(g.alpha, g.omega, 0.f);
    prod = g.alpha;
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) prod *= __shfl_xor_sync(0xffffffffu, prod, off);
    if (lane == 31) *reinterpret_cast<float2*>(own + 2 * D) = make_float2(z, prod);
    if (lane == 0) sh.prod[0] = prod;
  }
  cp_async_wait<0>();
  __syncthreads();
  const int which = tid / (D / 2), e = tid % (D / 2) * 2;
  const bool gate_pair = which == 0 && e == 0;
  auto value = [&](int t) {
    float2 x = P::to_f(*reinterpret_cast<const Raw*>(rows + (which * kC + t) * D + e));
    if (gate_pair) x.x = 0.f;
    return x;
  };
  unsigned int* flag = a.flags + (long long)chunk * a.Hkv + h;
  if (goes_on) {
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll 8
    for (int t = 0; t < kC; ++t) {
      const float2 x = value(t);
      const float al = sh.alpha[t], om = sh.omega[t];
      sum.x = fmaf(al, sum.x, om * x.x);
      sum.y = fmaf(al, sum.y, om * x.y);
    }
    reinterpret_cast<float2*>(own)[tid] = sum;
    publish(flag, launch, kOwn);
  }
  float2 sum = make_float2(0.f, 0.f);
  if (p.at > 0) {
    float zin;
    sum = come_in<D>(a, sh, a.sums, a.saved, chunk, h, p.at, -1, launch, zin);
    float* saved = a.saved + ((long long)chunk * a.Hkv + h) * sums_row(D);
    reinterpret_cast<float2*>(saved)[tid] = sum;
    if (tid == 0) {
      saved[2 * D] = zin;
      sh.zin = zin;
    }
    // (with a product of 0 nobody asks for what came in)
    if (goes_on && sh.prod[0] != 0.f)
      publish(flag, launch, kIn);
    else
      __syncthreads();
  }
  if (tid < 32) sh.rz[lane] = 1.f / scan_z(g.alpha, g.omega, p.at > 0 ? sh.zin : 0.f);
  __syncthreads();
  unsigned int before = 0;
  if (tid == 0) before = gone(a);
  T* dst = static_cast<T*>(which ? a.vt : a.kt) + row0 + e;
#pragma unroll 8
  for (int t = 0; t < n; ++t) {
    const float2 x = value(t);
    const float al = sh.alpha[t], om = sh.omega[t], rz = sh.rz[t];
    sum.x = fmaf(al, sum.x, om * x.x);
    sum.y = fmaf(al, sum.y, om * x.y);
    *reinterpret_cast<Raw*>(dst + t * step) = P::from_f(make_float2(sum.x * rz, sum.y * rz));
  }
  if (tid < 32 && in) {
    const int tok = tok0 + lane;
    const long long i = (long long)h * a.seqs.total + tok;
    a.alpha[i] = g.alpha;
    if (tok > p.t0) a.bias[i - 1] = g.log_rest;
    if (tok == p.t1 - 1) a.bias[i] = 0.f;
  }
  if (tid == 0) leave(a, before, launch);
}

// Chunks from the last to the first. A chunk passes on the sum over t of (its alphas up
// to t) u_t, and w_t alike.
template <typename T, int D>
__global__ void __launch_bounds__(D) states_backward_kernel(const StatesArgs a) {
  using P = Pair<T>;
  using Raw = typename P::Raw;
  constexpr int kH = kC / 2;  // tokens whose sums are held at a time
  __shared__ StatesShared<D> sh;
  extern __shared__ __align__(16) char chunk_rows[];  // k, v, then dk~, dv~
  T* rows = reinterpret_cast<T*>(chunk_rows);
  T* grads = rows + 2 * kC * D;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int index = take_turn(a, sh), chunks = gridDim.x / a.Hkv;
  const int h = index % a.Hkv, chunk = chunks - 1 - index / a.Hkv;
  const unsigned int launch = sh.launch;
  if (index == 0) check_seqs(a.seqs, a.error);
  const Piece p = find_piece(a.seqs, kC, chunk);
  if (!p.ok) {
    if (tid == 0) leave(a, gone(a), launch);
    return;
  }
  const int tok0 = p.t0 + p.at * kC, n = min(kC, p.t1 - tok0), tok = tok0 + lane;
  const int after = (p.t1 - p.t0 + kC - 1) / kC - 1 - p.at;  // chunks after this one
  const bool in_chunk = lane < n;
  GateIn gi;
  if (tid < 32) gi = gate_in<T, D>(a, h, tok, in_chunk);
  const long long row0 = ((long long)tok0 * a.Hkv + h) * D, step = (long long)a.Hkv * D;
  load_chunk<T, D>(reinterpret_cast<char*>(rows), a.k, a.v, row0, step, n);
  load_chunk<T, D>(reinterpret_cast<char*>(grads), a.dkt, a.dvt, row0, step, n);
  cp_async_commit();
  const float* saved = a.saved + ((long long)chunk * a.Hkv + h) * sums_row(D);
  float* own = a.sums + ((long long)chunk * a.Hkv + h) * sums_row(D);
  float2 sum0 = make_float2(0.f, 0.f);
  if (p.at > 0) sum0 = reinterpret_cast<const float2*>(saved)[tid];
  const float zbefore0 = p.at > 0 ? saved[2 * D] : 0.f;
  Gate g;
  float z = 0.f, prod = 0.f, dbias = 0.f, dalpha_out = 0.f;
  if (tid < 32) {
    if (in_chunk && tok > p.t0) {
      const long long i = (long long)h * a.seqs.total + tok;
      dbias = element<T>(a.dbias, i - 1);
      if (a.dalpha) dalpha_out = a.dalpha[i];
    }
    g = gate_of(a, gi, in_chunk, tok == p.t0);
    z = scan_z(g.alpha, g.omega, zbefore0);
    prod = g.alpha;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const float o = __shfl_up_sync(0xffffffffu, prod, off);
      if (lane >= off) prod *= o;
    }
    sh.alpha[lane] = g.alpha;
    sh.omega[lane] = g.omega;
    sh.rz[lane] = 1.f / z;
    sh.prod[lane] = prod;
  }
  // tokens from n on: zeros, and alpha 1, so that they change nothing
  for (int i = tid; i < 4 * (kC - n) * (D / 2); i += D) {
    const int w = i / ((kC - n) * (D / 2)), x = i % ((kC - n) * (D / 2));
    reinterpret_cast<Raw*>(rows + (w * kC + n) * D)[x] = P::from_f(make_float2(0.f, 0.f));
  }
  cp_async_wait<0>();
  __syncthreads();
  const int which = tid / (D / 2), e = tid % (D / 2) * 2;
  const bool gate_pair = which == 0 && e == 0;
  auto pair = [&](const T* of, int t) {
    float2 x = P::to_f(*reinterpret_cast<const Raw*>(of + (which * kC + t) * D + e));
    if (gate_pair) x.x = 0.f;
    return x;
  };
  // forward over the chunk: the sums, g . A, and what the chunk passes on
  float2 middle = sum0;  // the sums before the second half
  {
    float2 pass = make_float2(0.f, 0.f), sum = sum0;
    float dot[kC];
#pragma unroll
    for (int t = 0; t < kC; ++t) {
      const float2 x = pair(rows, t), gr = pair(grads, t);
      const float al = sh.alpha[t], om = sh.omega[t], w = sh.prod[t] * sh.rz[t];
      if (t == kH) middle = sum;
      sum.x = fmaf(al, sum.x, om * x.x);
      sum.y = fmaf(al, sum.y, om * x.y);
      dot[t] = fmaf(gr.x, sum.x, gr.y * sum.y);
      pass.x = fmaf(w, gr.x, pass.x);
      pass.y = fmaf(w, gr.y, pass.y);
    }
    if (p.at > 0) reinterpret_cast<float2*>(own)[tid] = pass;
    sh.dot[0][warp][lane] = transposed_sum(dot);
  }
  __syncthreads();
  float zeta = 0.f;
  if (tid < 32) {
    float d = 0.f;
#pragma unroll
    for (int w = 0; w < D / 32; ++w) d += sh.dot[0][w][lane];
    const float rz = sh.rz[lane];
    zeta = in_chunk ? -d * rz * rz : 0.f;
    float s = zeta * prod;
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    if (lane == 31) *reinterpret_cast<float2*>(own + 2 * D) = make_float2(s, prod);
  }
  unsigned int* flag = a.flags + (long long)chunk * a.Hkv + h;
  if (p.at > 0) publish(flag, launch, kOwn);
  float2 in = make_float2(0.f, 0.f);  // alpha L of the next token
  float zin = 0.f;
  if (after > 0) {
    in = come_in<D>(a, sh, a.sums, a.carry, chunk, h, after, 1, launch, zin);
    if (p.at > 0 && sh.prod[kC - 1] != 0.f) {  // (with a product of 0 nobody asks for what came in)
      float* carry = a.carry + ((long long)chunk * a.Hkv + h) * sums_row(D);
      reinterpret_cast<float2*>(carry)[tid] = in;
      if (tid == 0) carry[2 * D] = zin;
      publish(flag, launch, kIn);
    }
  }
  // from the last token to the first, half a chunk at a time: L, and its dots with the
  // values and with the sums before
  T* dst = static_cast<T*>(which ? a.dv : a.dk) + row0 + e;
#pragma unroll 1
  for (int half = 1; half >= 0; --half) {
    const int t0 = half * kH;
    float2 A[kH];  // the sums before token t0 + i
    float2 sum = half ? middle : sum0;
#pragma unroll
    for (int i = 0; i < kH; ++i) {
      const float2 x = pair(rows, t0 + i);
      const float al = sh.alpha[t0 + i], om = sh.omega[t0 + i];
      A[i] = sum;
      sum.x = fmaf(al, sum.x, om * x.x);
      sum.y = fmaf(al, sum.y, om * x.y);
    }
    float dots[kC];  // with the values, with the sums
#pragma unroll
    for (int i = kH - 1; i >= 0; --i) {
      const int t = t0 + i;
      const float2 x = pair(rows, t), gr = pair(grads, t);
      const float rz = sh.rz[t], om = sh.omega[t], al = sh.alpha[t];
      const float2 l = make_float2(fmaf(gr.x, rz, in.x), fmaf(gr.y, rz, in.y));
      dots[i] = fmaf(l.x, x.x, l.y * x.y);
      dots[kH + i] = fmaf(l.x, A[i].x, l.y * A[i].y);
      const float2 out = make_float2(om * l.x, om * l.y);
      if (gate_pair)
        sh.e1[t] = out.y;
      else if (t < n)
        *reinterpret_cast<Raw*>(dst + t * step) = P::from_f(out);
      in = make_float2(al * l.x, al * l.y);
    }
    sh.dot[1 + half][warp][lane] = transposed_sum(dots);
  }
  __syncthreads();
  unsigned int before = 0;
  if (tid == 0) before = gone(a);
  if (tid < 32) {
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
      float domega = zeta, dalpha = fmaf(zeta, zbefore, dalpha_out);
#pragma unroll
      for (int w = 0; w < D / 32; ++w) {
        domega += sh.dot[1 + lane / kH][w][lane % kH];
        dalpha += sh.dot[1 + lane / kH][w][kH + lane % kH];
      }
      float dx = 0.f;
      if (tok > p.t0) dx = (dalpha * g.alpha * g.rest - dbias * g.alpha) / a.temperature;
      *reinterpret_cast<Raw*>(static_cast<T*>(a.dk) + ((long long)tok * a.Hkv + h) * D) =
          P::from_f(make_float2(dx, sh.e1[lane]));
      const T dq = Elt<T>::from_f(domega * g.omega * (1.f - g.omega) / (float)a.G);
      for (int j = 0; j < a.G; ++j)
        static_cast<T*>(a.dq)[(long long)tok * a.dq_tok + (long long)(h * a.G + j) * a.dq_head] = dq;
    }
  }
  if (tid == 0) leave(a, before, launch);
}

template <typename T, int D>
cudaError_t forward(const StatesArgs& a, cudaStream_t stream) {
  states_kernel<T, D><<<(unsigned)(pieces(a.seqs.total, a.seqs.num, kC) * a.Hkv), D, 0, stream>>>(a);
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t backward(const StatesArgs& a, cudaStream_t stream) {
  constexpr int bytes = 4 * kC * D * sizeof(T);
  const cudaError_t e =
      cudaFuncSetAttribute(states_backward_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != cudaSuccess) return e;
  states_backward_kernel<T, D><<<(unsigned)(pieces(a.seqs.total, a.seqs.num, kC) * a.Hkv), D, bytes, stream>>>(a);
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
