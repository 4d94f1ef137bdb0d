// Appending to the cache with the position rotation on the way: what dmc_decode_step and dmc_prefill_compress do to a
// cache, for queries and keys that are not rotated yet, and without attention.
//
//  one token per sequence at most (a step of decoding): dmc_append_kernel, a warp per (sequence, KV head). It rotates
//    the key and the group's queries, applies Algorithm 1 to the head's last slot, or opens one, and writes the
//    queries back. All of it is a chain of trips to memory (slot count, page, old row and z), beside which the key, the
//    queries and their turns are on their way.
//  longer texts: the plan of dmc_prefill.cuh, dmc_rotate's kernel for the queries, and the scan with its rotation.
#include <math.h>

#include <type_traits>

#include "dmc_prefill.cuh"

namespace dmc {

cudaError_t prefill_launch(const Layout& L, int layer, int first_seq, int num_seqs, const void* q,
                           long long q_tok, long long q_head, const void* k, const void* v,
                           const int* cu, int total_tokens, int max_seqlen, float* carry,
                           float* weights, cudaStream_t stream);
cudaError_t rotate_prompt_launch(const Layout& L, int num_seqs, int total_tokens, const void* q, void* q_out, const int* cu,
                                 const int* at, const unsigned long long* turns, bool pairs, float* weights,
                                 cudaStream_t stream);

namespace {

constexpr int kAppendWarps = 4;

struct AppendArgs {
  Layout lay;
  int layer, first_seq, num_seqs, total_tokens;
  const char* q;
  const char* k;
  const char* v;
  char* q_out;
  const int* cu;  // null: one token each
  const int* at;
  const unsigned long long* turns;
  float* weights;  // room for the omegas of a prompt, or null
};

// A lane's share of a row: D / 64 elements of either half of it, or the same number twice in a row (kRotPairs).
template <typename T, int D, int kRot>
struct Share {
  static constexpr int N = D / 64, B = N * (int)sizeof(T);  // elements and bytes of one of the two pieces
  using Piece = typename std::conditional<B == 2, unsigned short,
                                          typename std::conditional<B == 4, unsigned int, uint2>::type>::type;
  static constexpr bool kHalves = kRot != kRotPairs;
  static __device__ __forceinline__ int off(int lane, int piece) {
    return kHalves ? piece * (D / 2) * (int)sizeof(T) + lane * B : (2 * lane + piece) * B;
  }
  Piece p[2];
  __device__ __forceinline__ void load(const char* row, int lane) {
    p[0] = *reinterpret_cast<const Piece*>(row + off(lane, 0));
    p[1] = *reinterpret_cast<const Piece*>(row + off(lane, 1));
  }
  __device__ __forceinline__ void store(char* row, int lane) const {
    *reinterpret_cast<Piece*>(row + off(lane, 0)) = p[0];
    *reinterpret_cast<Piece*>(row + off(lane, 1)) = p[1];
  }
  // floats x[0 .. N) of the first piece, x[N .. 2 N) of the second
  __device__ __forceinline__ void unpack(float* x) const {
    const T* e = reinterpret_cast<const T*>(p);
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) x[i] = Elt<T>::to_f(e[i]);
  }
  __device__ __forceinline__ void pack(const float* x) {
    T* e = reinterpret_cast<T*>(p);
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) e[i] = Elt<T>::from_f(x[i]);
  }
  // pair i of the lane turned by cs[i]
  static __device__ __forceinline__ void apply(const float2* cs, float* x) {
#pragma unroll
    for (int i = 0; i < N; ++i) turn(cs[i], x[kHalves ? i : 2 * i], x[kHalves ? i + N : 2 * i + 1]);
  }
};

template <typename T, int D, int kRot>
__global__ void __launch_bounds__(kAppendWarps * 32) dmc_append_kernel(const AppendArgs a) {
  using S = Share<T, D, kRot>;
  constexpr int N = S::N, ROW = D * (int)sizeof(T);
  const Layout& L = a.lay;
  const int lane = threadIdx.x & 31;
  const int unit = blockIdx.x * kAppendWarps + (threadIdx.x >> 5);
  if (unit >= a.num_seqs * L.Hkv) return;
  const int s = unit / L.Hkv, h = unit % L.Hkv, bh = a.first_seq * L.Hkv + unit;
  const int parity = *reinterpret_cast<const volatile int*>(&L.ctl[a.layer * 4]);
  int t = s;
  if (a.cu != nullptr) {
    t = a.cu[s];
    const int t1 = a.cu[s + 1];
    if (t < 0 || t1 < t || t1 - t > 1 || t1 > a.total_tokens) {
      if (lane == 0) atomicOr(L.error, DMC_FAULT_BAD_SEQLENS);
      return;
    }
    if (t1 == t) return;
  }
  int* len = L.lengths + ((size_t)a.layer * 2 + parity) * L.NH + bh;
  int* table = L.page_table + ((size_t)a.layer * L.NH + bh) * L.MPH;
  S k, v;
  const char* krow = a.k + ((size_t)t * L.Hkv + h) * ROW;
  const char* qrow = a.q + ((size_t)t * L.Hq + (size_t)h * L.G) * ROW;
  k.load(krow, lane);
  v.load(a.v + ((size_t)t * L.Hkv + h) * ROW, lane);
  const float k0 = Elt<T>::to_f(*reinterpret_cast<const T*>(krow));
  float y = lane < L.G ? Elt<T>::to_f(*reinterpret_cast<const T*>(qrow + (size_t)lane * ROW)) : 0.f;
  const int len_old = *len;
  float2 cs[N];
  if (kRot != kRotNone) {
#pragma unroll
    for (int i = 0; i < N; ++i) cs[i] = turn_of(turns_of_pair(a.turns, lane * N + i), a.at[s]);
  }
  // omega = sigmoid(mean of the group's q[0])
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) y += __shfl_xor_sync(0xffffffffu, y, off);
  const float omega = 1.f / (1.f + expf(-y / (float)L.G));
  // alpha = round(sigmoid(k[0])) = [k[0] >= 0]; an empty head always opens a slot
  const bool accum = k0 >= 0.f && len_old > 0;
  int page = -1;
  if (accum || len_old % kPage != 0) page = table[(len_old - 1) / kPage];
  const int slot = accum ? len_old - 1 : len_old;
  S ko, vo;
  float zold = 0.f;
  const int W = L.window;
  if (accum && W == 0) {
    const char* old = L.pages + (size_t)page * L.page_bytes + (size_t)(slot % kPage) * ROW;
    ko.load(old, lane);
    vo.load(old + (size_t)kPage * ROW, lane);
    zold = L.z[(size_t)page * kPage + slot % kPage];
  }
  float kf[2 * N], vf[2 * N];
  k.unpack(kf);
  v.unpack(vf);
  if (lane == 0) kf[0] = 0.f;  // k[0] <- 0 (Algorithm 1), a gate of any value
  if (kRot != kRotNone) S::apply(cs, kf);
  if (lane == 0) kf[0] = 0.f;  // (and where its partner, which keeps its value, is infinite)
  float znew = omega;
  int n_old = 0;
  if (W > 0) {
    // the mean of the open segment's last W tokens; the new one joins the head's ring at entry n_old % W
    char* ring = L.ring + ((size_t)a.layer * L.NH + bh) * W * 2 * ROW;
    float* ring_w = L.ring_w + ((size_t)a.layer * L.NH + bh) * W;
    int* seglen = L.seglen + ((size_t)a.layer * 2 + parity) * L.NH + bh;
    float sk[2 * N], sv[2 * N];
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) {
      sk[i] = omega * kf[i];
      sv[i] = omega * vf[i];
    }
    if (accum) {
      n_old = *seglen;
      for (int e = 0; e < min(n_old, W - 1); ++e) {
        const int pos = (n_old - 1 - e) % W;
        const float w = ring_w[pos];
        float ok[2 * N], ov[2 * N];
        ko.load(ring + (size_t)pos * 2 * ROW, lane);
        vo.load(ring + (size_t)pos * 2 * ROW + ROW, lane);
        ko.unpack(ok);
        vo.unpack(ov);
        znew += w;
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) {
          sk[i] = fmaf(w, ok[i], sk[i]);
          sv[i] = fmaf(w, ov[i], sv[i]);
        }
      }
    }
    k.pack(kf);
    k.store(ring + (size_t)(n_old % W) * 2 * ROW, lane);
    v.store(ring + (size_t)(n_old % W) * 2 * ROW + ROW, lane);
    __syncwarp();
    if (lane == 0) ring_w[n_old % W] = omega;
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) {
      kf[i] = sk[i] / znew;
      vf[i] = sv[i] / znew;
    }
  } else if (accum) {
    float ok[2 * N], ov[2 * N];
    ko.unpack(ok);
    vo.unpack(ov);
    znew = zold + omega;
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) {
      kf[i] = (ok[i] * zold + kf[i] * omega) / znew;
      vf[i] = (ov[i] * zold + vf[i] * omega) / znew;
    }
  }
  k.pack(kf);
  v.pack(vf);
  const bool fits = slot < L.max_slots;
  if (fits && page < 0) {
    if (lane == 0) {
      page = take_page(L);
      if (page >= 0) table[slot / kPage] = page;
    }
    page = __shfl_sync(0xffffffffu, page, 0);
  }
  if (fits && page >= 0) {
    char* row = L.pages + (size_t)page * L.page_bytes + (size_t)(slot % kPage) * ROW;
    k.store(row, lane);
    v.store(row + (size_t)kPage * ROW, lane);
  }
  if (lane == 0) {
    if (!fits) atomicOr(L.error, DMC_FAULT_SLOT_CAPACITY);
    if (k0 != k0) atomicOr(L.error, DMC_FAULT_NAN_GATE);
    if (fits && page >= 0) {
      L.z[(size_t)page * kPage + slot % kPage] = znew;
      *len = slot + 1;
      if (W > 0) L.seglen[((size_t)a.layer * 2 + parity) * L.NH + bh] = n_old + 1;
    }
  }
  if (kRot != kRotNone) {
    char* to = a.q_out + ((size_t)t * L.Hq + (size_t)h * L.G) * ROW;
    for (int g = 0; g < L.G; ++g) {
      S q;
      float qf[2 * N];
      q.load(qrow + (size_t)g * ROW, lane);
      q.unpack(qf);
      constexpr int kPartner = S::kHalves ? N : 1;
      const float gate = qf[0], partner = qf[kPartner];  // lane 0: they stay, whatever they are
      S::apply(cs, qf);
      if (lane == 0) {
        qf[0] = gate;
        qf[kPartner] = partner;
      }
      q.pack(qf);
      q.store(to + (size_t)g * ROW, lane);
    }
  }
}

template <typename T, int D, int kRot>
cudaError_t launch_step(const AppendArgs& a, cudaStream_t stream) {
  const int units = a.num_seqs * a.lay.Hkv;
  dmc_append_kernel<T, D, kRot><<<ceil_div(units, kAppendWarps), kAppendWarps * 32, 0, stream>>>(a);
  return cudaGetLastError();
}

template <typename T, int D, int kRot>
cudaError_t launch_text(const AppendArgs& a, int max_seqlen, cudaStream_t stream) {
  const Layout& L = a.lay;
  PrefillArgs p = {};
  p.lay = L;
  p.layer = a.layer;
  p.first_seq = a.first_seq;
  p.num_seqs = a.num_seqs;
  p.q = a.q;
  p.q_tok = (long long)L.Hq * D;
  p.q_head = D;
  p.k = a.k;
  p.v = a.v;
  p.cu = a.cu;
  p.total_tokens = a.total_tokens;
  p.max_seqlen = max_seqlen;
  p.at = a.at;
  p.turns = a.turns;
  // The queries' rotation runs beside the plan, which is all latency, and leaves the omegas for the scan where the cache
  // has room for them: a query's first component costs the scan a line of DRAM
  cudaError_t e = launch_plan<T, D>(p, stream);
  if (e != cudaSuccess) return e;
  e = rotate_prompt_launch(L, a.num_seqs, a.total_tokens, a.q, a.q_out, a.cu, a.at, a.turns, kRot == kRotPairs, a.weights,
                           stream);
  if (e != cudaSuccess) return e;
  p.omegas = a.weights;
  return launch_scan<T, D, kRot>(p, stream);
}

template <typename T, int D>
cudaError_t launch_append(const AppendArgs& a, int max_seqlen, int rot, cudaStream_t stream) {
  if (max_seqlen <= 1)
    return rot == kRotNone   ? launch_step<T, D, kRotNone>(a, stream)
           : rot == kRotHalf ? launch_step<T, D, kRotHalf>(a, stream)
                             : launch_step<T, D, kRotPairs>(a, stream);
  return rot == kRotHalf ? launch_text<T, D, kRotHalf>(a, max_seqlen, stream)
                         : launch_text<T, D, kRotPairs>(a, max_seqlen, stream);
}

}  // namespace

// One token per sequence (cu null) or texts of up to max_seqlen tokens. turns null: no rotation.
cudaError_t append_launch(const Layout& L, int layer, int first_seq, int num_seqs, const void* q, const void* k,
                          const void* v, const int* cu, int total_tokens, int max_seqlen, const int* at,
                          const unsigned long long* turns, bool pairs, void* q_out, float* weights,
                          cudaStream_t stream) {
  if (turns == nullptr && max_seqlen > 1)
    return prefill_launch(L, layer, first_seq, num_seqs, q, (long long)L.Hq * L.D, L.D, k, v, cu, total_tokens,
                          max_seqlen, nullptr, nullptr, stream);
  const AppendArgs a{L, layer, first_seq, num_seqs, total_tokens, static_cast<const char*>(q),
                     static_cast<const char*>(k), static_cast<const char*>(v), static_cast<char*>(q_out), cu, at, turns, weights};
  const int rot = turns == nullptr ? kRotNone : pairs ? kRotPairs : kRotHalf;
  cudaError_t e = cudaErrorInvalidValue;
  if (L.esize == 4 && L.D == 64) e = launch_append<float, 64>(a, max_seqlen, rot, stream);
  if (L.esize == 4 && L.D == 128) e = launch_append<float, 128>(a, max_seqlen, rot, stream);
  if (L.esize == 2 && L.D == 64) e = launch_append<__nv_bfloat16, 64>(a, max_seqlen, rot, stream);
  if (L.esize == 2 && L.D == 128) e = launch_append<__nv_bfloat16, 128>(a, max_seqlen, rot, stream);
  return e;
}

}  // namespace dmc
