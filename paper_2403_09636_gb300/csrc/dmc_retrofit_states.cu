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
// neighbouring elements of k or v per thread: each chunk's own sums, a scan over the
// chunks, and the chunks again with what comes in from before (after).
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

template <typename T, int D>
__device__ __forceinline__ Gate gate_of(const StatesArgs& a, int h, int tok, bool in, bool first) {
  Gate g;
  g.alpha = 1.f;
  g.rest = g.omega = g.log_rest = 0.f;
  if (!in) return g;
  float x = element<T>(a.k, ((long long)tok * a.Hkv + h) * D) - a.offset;
  if (a.noise) x += a.noise[(long long)h * a.seqs.total + tok];
  x /= a.temperature;
  float q = 0.f;
  for (int j = 0; j < a.G; ++j) q += element<T>(a.q, (long long)tok * a.q_tok + (long long)(h * a.G + j) * a.q_head);
  g.omega = 1.f / (1.f + expf(-q / (float)a.G));
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
  float zeta[kC];
  float dot[3][D / 32][kC];
  float e1[kC];         // second element of dk
};

// Forward. kApply false: the chunk's own sums and the product of its alphas into
// `saved`; true: its states, from the sums before it.
template <typename T, int D, bool kApply>
__global__ void __launch_bounds__(D) states_kernel(const StatesArgs a) {
  using P = Pair<T>;
  __shared__ StatesShared<D> sh;
  const int tid = threadIdx.x, lane = tid & 31, h = blockIdx.y;
  if (!kApply && blockIdx.x == 0 && h == 0) check_seqs(a.seqs, a.error);
  const Piece p = find_piece(a.seqs, kC, blockIdx.x);
  if (!p.ok) return;
  const int tok0 = p.t0 + p.at * kC, n = min(kC, p.t1 - tok0);
  float* row = a.saved + ((long long)blockIdx.x * a.Hkv + h) * sums_row(D);
  if (tid < 32) {
    const int tok = tok0 + lane;
    const bool in = lane < n;
    const Gate g = gate_of<T, D>(a, h, tok, in, tok == p.t0);
    const float z = scan_z(g.alpha, g.omega, kApply && p.at > 0 ? row[2 * D] : 0.f);
    sh.alpha[lane] = g.alpha;
    sh.omega[lane] = g.omega;
    sh.rz[lane] = 1.f / z;
    if (kApply && in) {
      const long long i = (long long)h * a.seqs.total + tok;
      a.alpha[i] = g.alpha;
      if (tok > p.t0) a.bias[i - 1] = g.log_rest;
      if (tok == p.t1 - 1) a.bias[i] = 0.f;
    }
    if (!kApply) {
      float prod = g.alpha;
#pragma unroll
      for (int off = 16; off >= 1; off >>= 1) prod *= __shfl_xor_sync(0xffffffffu, prod, off);
      if (lane == 31) {
        row[2 * D] = z;
        row[2 * D + 1] = prod;
      }
    }
  }
  __syncthreads();
  const int which = tid / (D / 2), e = tid % (D / 2) * 2;
  const long long at = ((long long)tok0 * a.Hkv + h) * D + e, step = (long long)a.Hkv * D;
  const T* src = static_cast<const T*>(which ? a.v : a.k) + at;
  T* dst = static_cast<T*>(which ? a.vt : a.kt) + at;
  const bool gate_pair = which == 0 && e == 0;
  float2 sum = make_float2(0.f, 0.f);
  if (kApply && p.at > 0) sum = *reinterpret_cast<const float2*>(row + which * D + e);
  typename P::Raw raw[kC];
#pragma unroll
  for (int t = 0; t < kC; ++t)
    if (t < n) raw[t] = *reinterpret_cast<const typename P::Raw*>(src + t * step);
#pragma unroll
  for (int t = 0; t < kC; ++t) {
    if (t >= n) break;
    float2 x = P::to_f(raw[t]);
    if (gate_pair) x.x = 0.f;
    const float al = sh.alpha[t], om = sh.omega[t];
    sum.x = fmaf(al, sum.x, om * x.x);
    sum.y = fmaf(al, sum.y, om * x.y);
    if (kApply)
      *reinterpret_cast<typename P::Raw*>(dst + t * step) = P::from_f(make_float2(sum.x * sh.rz[t], sum.y * sh.rz[t]));
  }
  if (!kApply) *reinterpret_cast<float2*>(row + which * D + e) = sum;
}

// The chunks' own sums into the sums before each chunk, in place; one block per
// sequence and head. kBack: from the last chunk to the first, what comes in from after.
template <int D, bool kBack>
__global__ void __launch_bounds__(2 * D + kPad) states_scan_kernel(const Seqs seqs, int Hkv, float* sums) {
  const int s = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
  const int t0 = seqs.cu[s], t1 = seqs.cu[s + 1];
  if (!seq_ok(seqs, t0, t1)) return;
  const int n = (t1 - t0 + kC - 1) / kC;
  const long long stride = (long long)Hkv * sums_row(D);
  float* base = sums + ((long long)(t0 / kC + s) * Hkv + h) * sums_row(D);
  float run = 0.f;
#pragma unroll 4
  for (int c = 0; c < n; ++c) {
    float* row = base + (kBack ? n - 1 - c : c) * stride;
    const float own = row[tid], prod = row[2 * D + 1];
    if (tid != 2 * D + 1) row[tid] = run;
    run = fmaf(prod, run, own);
  }
}

// Backward. kApply false: what the chunk passes on to the one before it of its own
// (sum over t of the alphas up to t times u_t, w_t) and the product of its alphas into
// `sums`; true: the gradients, from what comes in from after.
template <typename T, int D, bool kApply>
__global__ void __launch_bounds__(D) states_backward_kernel(const StatesArgs a) {
  using P = Pair<T>;
  using Raw = typename P::Raw;
  __shared__ StatesShared<D> sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, h = blockIdx.y;
  if (!kApply && blockIdx.x == 0 && h == 0) check_seqs(a.seqs, a.error);
  const Piece p = find_piece(a.seqs, kC, blockIdx.x);
  if (!p.ok) return;
  const int tok0 = p.t0 + p.at * kC, n = min(kC, p.t1 - tok0);
  const float* saved = a.saved + ((long long)blockIdx.x * a.Hkv + h) * sums_row(D);
  float* row = a.sums + ((long long)blockIdx.x * a.Hkv + h) * sums_row(D);
  const float zin = p.at > 0 ? saved[2 * D] : 0.f;
  Gate g;
  float z = 0.f;
  if (tid < 32) {
    const int tok = tok0 + lane;
    g = gate_of<T, D>(a, h, tok, lane < n, tok == p.t0);
    z = scan_z(g.alpha, g.omega, zin);
    float prod = g.alpha;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const float o = __shfl_up_sync(0xffffffffu, prod, off);
      if (lane >= off) prod *= o;
    }
    sh.alpha[lane] = g.alpha;
    sh.omega[lane] = g.omega;
    sh.rz[lane] = 1.f / z;
    sh.prod[lane] = prod;
    if (!kApply && lane == 31) row[2 * D + 1] = prod;
  }
  __syncthreads();
  const int which = tid / (D / 2), e = tid % (D / 2) * 2;
  const long long at = ((long long)tok0 * a.Hkv + h) * D + e, step = (long long)a.Hkv * D;
  const T* src = static_cast<const T*>(which ? a.v : a.k) + at;
  const T* gsrc = static_cast<const T*>(which ? a.dvt : a.dkt) + at;
  const bool gate_pair = which == 0 && e == 0;
  float2 sum = make_float2(0.f, 0.f);
  if (p.at > 0) sum = *reinterpret_cast<const float2*>(saved + which * D + e);
  const float2 sum0 = sum;
  auto value = [&](int t) {
    float2 x = P::to_f(*reinterpret_cast<const Raw*>(src + t * step));
    if (gate_pair) x.x = 0.f;
    return x;
  };
  auto grad = [&](int t) {
    float2 x = P::to_f(*reinterpret_cast<const Raw*>(gsrc + t * step));
    if (gate_pair) x.x = 0.f;
    return x;
  };
  // forward over the chunk: the sums, and g . A
  float2 A[kC];
  float2 own = make_float2(0.f, 0.f);
  {
    float dot[kC];
#pragma unroll
    for (int t = 0; t < kC; ++t) {
      dot[t] = 0.f;
      A[t] = sum;
      if (t >= n) continue;
      const float2 x = value(t), gr = grad(t);
      const float al = sh.alpha[t], om = sh.omega[t];
      sum.x = fmaf(al, sum.x, om * x.x);
      sum.y = fmaf(al, sum.y, om * x.y);
      A[t] = sum;
      dot[t] = fmaf(gr.x, sum.x, gr.y * sum.y);
      if (!kApply) {
        const float w = sh.prod[t] * sh.rz[t];
        own.x = fmaf(w, gr.x, own.x);
        own.y = fmaf(w, gr.y, own.y);
      }
    }
    sh.dot[0][warp][lane] = transposed_sum(dot);
  }
  __syncthreads();
  float zeta = 0.f;
  if (tid < 32) {
    float d = 0.f;
#pragma unroll
    for (int w = 0; w < D / 32; ++w) d += sh.dot[0][w][lane];
    const float rz = sh.rz[lane];
    zeta = lane < n ? -d * rz * rz : 0.f;
    if (!kApply) {
      float s = zeta * sh.prod[lane];
#pragma unroll
      for (int off = 16; off >= 1; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
      if (lane == 0) row[2 * D] = s;
    } else {
      // Z_t = w_t + alpha_{t+1} Z_{t+1}; what comes in has its alpha already
      float next = __shfl_down_sync(0xffffffffu, g.alpha, 1);
      if (lane == 31) {
        next = 0.f;
        zeta += row[2 * D];  // lanes from n on are the identity: alpha 1, w 0
      }
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const float on = __shfl_down_sync(0xffffffffu, next, off), oz = __shfl_down_sync(0xffffffffu, zeta, off);
        if (lane + off < 32) {
          zeta = fmaf(next, oz, zeta);
          next *= on;
        }
      }
    }
  }
  if (!kApply) {
    *reinterpret_cast<float2*>(row + which * D + e) = own;
    return;
  }
  // from the last token to the first: L, and its dots with the values and with the sums before
  T* dst = static_cast<T*>(which ? a.dv : a.dk) + at;
  float2 in = *reinterpret_cast<const float2*>(row + which * D + e);  // alpha L of the next token
  float dw[kC], da[kC];
#pragma unroll
  for (int t = kC - 1; t >= 0; --t) {
    dw[t] = da[t] = 0.f;
    if (t >= n) continue;
    const float2 x = value(t), gr = grad(t);
    const float rz = sh.rz[t], om = sh.omega[t], al = sh.alpha[t];
    const float2 l = make_float2(fmaf(gr.x, rz, in.x), fmaf(gr.y, rz, in.y));
    const float2 before = t > 0 ? A[t > 0 ? t - 1 : 0] : sum0;
    dw[t] = fmaf(l.x, x.x, l.y * x.y);
    da[t] = fmaf(l.x, before.x, l.y * before.y);
    const float2 out = make_float2(om * l.x, om * l.y);
    if (gate_pair)
      sh.e1[t] = out.y;
    else
      *reinterpret_cast<Raw*>(dst + t * step) = P::from_f(out);
    in = make_float2(al * l.x, al * l.y);
  }
  sh.dot[1][warp][lane] = transposed_sum(dw);
  sh.dot[2][warp][lane] = transposed_sum(da);
  __syncthreads();
  if (tid < 32) {
    float zbefore = __shfl_up_sync(0xffffffffu, z, 1);
    if (lane == 0) zbefore = zin;
    if (lane < n) {
      float domega = zeta, dalpha = zeta * zbefore;
#pragma unroll
      for (int w = 0; w < D / 32; ++w) {
        domega += sh.dot[1][w][lane];
        dalpha += sh.dot[2][w][lane];
      }
      const int tok = tok0 + lane;
      const long long i = (long long)h * a.seqs.total + tok;
      float dx = 0.f;
      if (tok > p.t0) {
        if (a.dalpha) dalpha += a.dalpha[i];
        dx = (dalpha * g.alpha * g.rest - element<T>(a.dbias, i - 1) * g.alpha) / a.temperature;
      }
      *reinterpret_cast<Raw*>(static_cast<T*>(a.dk) + ((long long)tok * a.Hkv + h) * D) =
          P::from_f(make_float2(dx, sh.e1[lane]));
      const T dq = Elt<T>::from_f(domega * g.omega * (1.f - g.omega) / (float)a.G);
      for (int j = 0; j < a.G; ++j)
        static_cast<T*>(a.dq)[(long long)tok * a.dq_tok + (long long)(h * a.G + j) * a.dq_head] = dq;
    }
  }
}

template <typename T, int D>
cudaError_t forward(const StatesArgs& a, cudaStream_t stream) {
  const dim3 grid((unsigned)pieces(a.seqs.total, a.seqs.num, kC), a.Hkv);
  states_kernel<T, D, false><<<grid, D, 0, stream>>>(a);
  states_scan_kernel<D, false><<<dim3(a.seqs.num, a.Hkv), sums_row(D), 0, stream>>>(a.seqs, a.Hkv, a.saved);
  states_kernel<T, D, true><<<grid, D, 0, stream>>>(a);
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t backward(const StatesArgs& a, cudaStream_t stream) {
  const dim3 grid((unsigned)pieces(a.seqs.total, a.seqs.num, kC), a.Hkv);
  states_backward_kernel<T, D, false><<<grid, D, 0, stream>>>(a);
  states_scan_kernel<D, true><<<dim3(a.seqs.num, a.Hkv), sums_row(D), 0, stream>>>(a.seqs, a.Hkv, a.sums);
  states_backward_kernel<T, D, true><<<grid, D, 0, stream>>>(a);
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
