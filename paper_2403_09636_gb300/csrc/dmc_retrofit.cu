// Host side of the retrofitting calls of include/dmc.h: checks of arguments, the
// layout of a handle's scratch in the caller's arena, and the join of the loss's
// shares of the vocabulary.
#include <math.h>
#include <string.h>

#include <new>

#include "dmc_retrofit.cuh"

namespace dmc {
cudaError_t states_forward(const StatesArgs& a, bool bf16, int D, cudaStream_t stream);
cudaError_t states_backward(const StatesArgs& a, bool bf16, int D, cudaStream_t stream);
cudaError_t attn_forward_f32(const AttnArgs& a, int D, cudaStream_t stream);
cudaError_t attn_backward_f32(const AttnArgs& a, int D, cudaStream_t stream);
cudaError_t attn_backward_bf16(const AttnArgs& a, int D, cudaStream_t stream);
cudaError_t attn_forward_bf16(const AttnArgs& a, int D, cudaStream_t stream);
cudaError_t loss_forward(const LossArgs& a, bool bf16, int* share, cudaStream_t stream);
cudaError_t loss_backward(const LossArgs& a, bool bf16, cudaStream_t stream);

namespace {

constexpr size_t kAlign = 256;
// The fault bits, from byte 128 the attention kernels' counter, from byte 256 the states' turns
constexpr size_t kControl = 768;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool given16(const void* p) { return p && aligned16(p); }
bool given4(const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
dmc_status cuda_status(cudaError_t e) { return e == cudaSuccess ? DMC_OK : DMC_ERR_CUDA; }

bool has_heads(const dmc_retrofit_config& c) { return c.num_q_heads > 0; }
bool has_loss(const dmc_retrofit_config& c) { return c.hidden > 0; }

// Elements of the largest tensor of a call that a handle may be made for, beyond any memory: so sizes of scratch
// stay far below 64 bits.
constexpr int64_t kMostElements = 1ll << 48;

bool valid(const dmc_retrofit_config* c) {
  if (!c) return false;
  if (c->dtype != DMC_F32 && c->dtype != DMC_BF16) return false;
  if (c->max_tokens < 1 || c->max_seqs < 1) return false;
  if (c->num_q_heads != 0 || c->num_kv_heads != 0 || c->head_dim != 0) {
    if (c->num_q_heads < 1 || c->num_kv_heads < 1 || c->num_q_heads % c->num_kv_heads != 0) return false;
    if (c->num_q_heads / c->num_kv_heads > 32 || c->num_q_heads > 65535) return false;
    if (c->head_dim != 64 && c->head_dim != 128) return false;
    if (((int64_t)c->max_tokens + c->max_seqs) * c->num_q_heads * c->head_dim > kMostElements) return false;
  }
  if (c->hidden != 0 || c->vocab != 0) {
    if (c->hidden < 1 || c->vocab < 1 || c->vocab > (1 << 30)) return false;
    if ((int64_t)c->hidden * (c->dtype == DMC_F32 ? 4 : 2) % 16 != 0) return false;
    if ((int64_t)c->hidden * c->max_tokens > kMostElements || (int64_t)c->hidden * c->vocab > kMostElements) return false;
  }
  return has_heads(*c) || has_loss(*c);
}

// Words of one piece of the vocabulary: the gradient of its logits is kept for all tokens
// (in fp32 the parts of its weights, too), in about 512 MB, but no fewer than 1024 words.
int loss_piece(const dmc_retrofit_config* c) {
  const int64_t per_word = c->dtype == DMC_F32 ? 6 * ((int64_t)c->max_tokens + loss_stride(c->hidden)) : 2ll * c->max_tokens;
  int64_t words = (512ll << 20) / per_word / kLossTile * kLossTile;
  const int64_t all = ((int64_t)c->vocab + kLossTile - 1) / kLossTile * kLossTile;
  if (words < 1024) words = 1024;
  return (int)(words < all ? words : all);
}

struct Offsets {
  size_t error, sums, carry, cleared, rows, shares, loss_sums, part_m, part_l, target_logit, dh, grad, hidden_parts, weight_parts, total;
  int piece;
};

Offsets offsets(const dmc_retrofit_config* c) {
  Offsets o = {};
  size_t at = 0;
  const size_t tokens = c->max_tokens;
  o.error = at; at = align_up(at + kControl);
  if (has_heads(*c)) {
    const size_t sums = (size_t)pieces(c->max_tokens, c->max_seqs, kStateChunk) * c->num_kv_heads * 2 * (c->head_dim + 2) * 8;
    o.sums = at; at = align_up(at + sums);
    o.carry = at; at = align_up(at + sums);
  }
  o.cleared = at;
  if (has_heads(*c)) {
    // the backward pass's two numbers per query, padded to tiles of 128 (one in fp32)
    o.rows = at;
    at = align_up(at + (c->dtype == DMC_F32 ? tokens * 4 : (size_t)pieces(c->max_tokens, c->max_seqs, 128) * 1024) *
                           c->num_q_heads);
    o.shares = at;
    at = align_up(at + attn_sums(c->max_tokens, c->num_kv_heads, c->num_q_heads / c->num_kv_heads, c->head_dim) * 4);
  }
  if (has_loss(*c)) {
    o.piece = loss_piece(c);
    const size_t parts = c->dtype == DMC_F32 ? 3 : 0, row = (size_t)loss_stride(c->hidden) * 2;
    const size_t shares = ceil_div(c->vocab, kLossTile / 4);  // of half a tile of half the columns at least
    o.part_m = at; at = align_up(at + tokens * shares * 4);
    o.part_l = at; at = align_up(at + tokens * shares * 4);
    o.target_logit = at; at = align_up(at + tokens * 4);
    o.dh = at; at = align_up(at + (!parts && o.piece < c->vocab ? tokens * c->hidden * 4 : 0));
    o.loss_sums = at; at = align_up(at + kSumTiles * kLossTile * kLossTile * 4);
    o.grad = at; at = align_up(at + tokens * o.piece * 2 * (parts ? parts : 1));
    o.hidden_parts = at; at = align_up(at + parts * tokens * row);
    o.weight_parts = at; at = align_up(at + parts * o.piece * row);
  }
  o.total = at;
  return o;
}

// The shares' maxima and sums into each token's log-sum and loss. One warp per token,
// the shares over its lanes, joined in an order that depends on their number alone.
__global__ void __launch_bounds__(256) loss_join_kernel(const LossArgs a, int shares) {
  const int t = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (t >= a.N) return;
  float m = -INFINITY, l = 0.f;  // of this lane's shares, the sum relative to the maximum
#pragma unroll 4
  for (int s = lane; s < shares; s += 32) {
    const float pm = a.part_m[(long long)s * a.N + t], pl = a.part_l[(long long)s * a.N + t];
    const float to = fmaxf(m, pm), ref = to == -INFINITY ? 0.f : to;
    l = fmaf(l, expf(m - ref), pl * expf(pm - ref));
    m = to;
  }
  const float own = m;
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
  l *= expf(own - (m == -INFINITY ? 0.f : m));
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
  if (lane) return;
  const float lse = m + logf(l);
  const int target = a.targets[t];
  if (target >= a.V) atomicOr(a.error, DMC_FAULT_BAD_TARGET);
  a.lse[t] = lse;
  a.loss[t] = target >= 0 && target < a.V ? lse - a.target_logit[t] : 0.f;
}

// The shares' sums of 128 rows of a KV head, in the shares' order: blockIdx.z / 2 is a quarter of
// the rows, its lowest bit dV or dK. Bound by the L2 cache, where the sums still are.
template <int D, typename T>
__global__ void __launch_bounds__(256) attn_join_kernel(const AttnArgs a) {
  constexpr int kLanes = D / 4, kPer = 256 / kLanes, kRows = 128 / 4;
  const int hk = blockIdx.y;
  const bool dk = blockIdx.z & 1;
  const Piece p = find_piece(a.seqs, 128, blockIdx.x);
  if (!p.ok) return;
  const int tok0 = p.t0 + p.at * 128 + (blockIdx.z >> 1) * kRows, rows = min(kRows, p.t1 - tok0);
  const int c = threadIdx.x % kLanes * 4;
  float4 x[kRows / kPer];
#pragma unroll
  for (int i = 0; i < kRows / kPer; ++i) x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s = 0; s < a.shares; ++s) {
#pragma unroll
    for (int i = 0; i < kRows / kPer; ++i) {
      const int r = threadIdx.x / kLanes + i * kPer;
      if (r >= rows) continue;
      const float4 y = *reinterpret_cast<const float4*>(share_rows(a, D, dk, s, hk, tok0 + r) + c);
      x[i].x += y.x;
      x[i].y += y.y;
      x[i].z += y.z;
      x[i].w += y.w;
    }
  }
#pragma unroll
  for (int i = 0; i < kRows / kPer; ++i) {
    const int r = threadIdx.x / kLanes + i * kPer;
    if (r >= rows) continue;
    typename Pair<T>::Raw* dst =
        reinterpret_cast<typename Pair<T>::Raw*>(static_cast<T*>(dk ? a.dk : a.dv) + ((long long)(tok0 + r) * a.Hkv + hk) * D + c);
    dst[0] = Pair<T>::from_f(make_float2(x[i].x, x[i].y));
    dst[1] = Pair<T>::from_f(make_float2(x[i].z, x[i].w));
  }
  if (!dk && a.dbias && (int)threadIdx.x < rows) {
    float b = 0.f;
    for (int s = 0; s < a.shares; ++s) b += share_dbias(a, D, s, hk)[tok0 + threadIdx.x];
    static_cast<T*>(a.dbias)[(long long)hk * a.seqs.total + tok0 + threadIdx.x] = (T)b;
  }
}

}  // namespace

cudaError_t attn_join(const AttnArgs& a, bool bf16, int D, cudaStream_t stream) {
  const dim3 grid((unsigned)pieces(a.seqs.total, a.seqs.num, 128), a.Hkv, 8);
  if (bf16 && D == 128)
    attn_join_kernel<128, __nv_bfloat16><<<grid, 256, 0, stream>>>(a);
  else if (bf16)
    attn_join_kernel<64, __nv_bfloat16><<<grid, 256, 0, stream>>>(a);
  else if (D == 128)
    attn_join_kernel<128, float><<<grid, 256, 0, stream>>>(a);
  else
    attn_join_kernel<64, float><<<grid, 256, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace dmc

struct dmc_retrofit {
  dmc_retrofit_config cfg;
  int device;
  dmc::Offsets at;
  char* base;
};

namespace {

// A handle whose device is the current one: kernels go there, whatever the stream's number means elsewhere.
bool usable(dmc_retrofit_t h) {
  int dev = 0;
  return h && cudaGetDevice(&dev) == cudaSuccess && dev == h->device;
}

// What every call on sequences checks. 1: go on, 0: nothing to do, -1: refused.
int seqs_arg(dmc_retrofit_t h, int32_t num_seqs, const int32_t* cu, int32_t total, int32_t longest) {
  if (!usable(h) || !dmc::has_heads(h->cfg)) return -1;
  if (num_seqs < 0 || num_seqs > h->cfg.max_seqs || total < 0 || total > h->cfg.max_tokens) return -1;
  if (longest < 0 || longest > total) return -1;
  if (num_seqs == 0 || total == 0) return 0;
  return dmc::given4(cu) ? 1 : -1;
}

dmc::StatesArgs states_args(dmc_retrofit_t h, int32_t num_seqs, const void* q, int64_t q_tok, int64_t q_head,
                            const void* k, const void* v, const float* noise, float offset, float temperature,
                            const int32_t* cu, int32_t total, int32_t longest, void* saved) {
  dmc::StatesArgs a = {};
  a.seqs = {cu, num_seqs, total, longest};
  a.Hq = h->cfg.num_q_heads;
  a.Hkv = h->cfg.num_kv_heads;
  a.G = a.Hq / a.Hkv;
  a.q = q;
  a.q_tok = q_tok;
  a.q_head = q_head;
  a.k = k;
  a.v = v;
  a.noise = noise;
  a.offset = offset;
  a.temperature = temperature;
  a.saved = static_cast<float*>(saved);
  a.error = reinterpret_cast<unsigned int*>(h->base + h->at.error);
  a.sums = reinterpret_cast<uint64_t*>(h->base + h->at.sums);
  a.carry = reinterpret_cast<uint64_t*>(h->base + h->at.carry);
  a.turns = reinterpret_cast<unsigned int*>(h->base + h->at.error + 256);
  return a;
}

dmc::AttnArgs attn_args(dmc_retrofit_t h, int32_t num_seqs, const void* q, const void* k, const void* v,
                        const float* bias, const int32_t* cu, int32_t total, int32_t longest) {
  dmc::AttnArgs a = {};
  a.seqs = {cu, num_seqs, total, longest};
  a.Hq = h->cfg.num_q_heads;
  a.Hkv = h->cfg.num_kv_heads;
  a.G = a.Hq / a.Hkv;
  a.q = q;
  a.k = k;
  a.v = v;
  a.bias = bias;
  a.rows = reinterpret_cast<float*>(h->base + h->at.rows);
  a.sums = reinterpret_cast<float*>(h->base + h->at.shares);
  a.counter = reinterpret_cast<int*>(h->base + h->at.error + 128);
  a.error = reinterpret_cast<unsigned int*>(h->base + h->at.error);
  return a;
}

dmc::LossArgs loss_args(dmc_retrofit_t h, int32_t n, const void* hidden, const void* weight, const int32_t* targets) {
  dmc::LossArgs a = {};
  a.N = n;
  a.H = h->cfg.hidden;
  a.V = h->cfg.vocab;
  a.hidden = hidden;
  a.weight = weight;
  a.targets = targets;
  a.piece = h->at.piece;
  a.grad = h->base + h->at.grad;
  a.hidden_parts = h->base + h->at.hidden_parts;
  a.weight_parts = h->base + h->at.weight_parts;
  a.dh = reinterpret_cast<float*>(h->base + h->at.dh);
  a.sums = reinterpret_cast<float*>(h->base + h->at.loss_sums);
  a.part_m = reinterpret_cast<float*>(h->base + h->at.part_m);
  a.part_l = reinterpret_cast<float*>(h->base + h->at.part_l);
  a.target_logit = reinterpret_cast<float*>(h->base + h->at.target_logit);
  a.error = reinterpret_cast<unsigned int*>(h->base + h->at.error);
  return a;
}

bool bf16(dmc_retrofit_t h) { return h->cfg.dtype == DMC_BF16; }
// an address of elements of the handle's type
bool given(dmc_retrofit_t h, const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & (bf16(h) ? 1u : 3u)) == 0; }

}  // namespace

extern "C" {

size_t dmc_retrofit_required_bytes(const dmc_retrofit_config* cfg) {
  return dmc::valid(cfg) ? dmc::offsets(cfg).total : 0;
}

dmc_status dmc_retrofit_create(const dmc_retrofit_config* cfg, void* arena_dev, size_t arena_bytes, cudaStream_t stream,
                               dmc_retrofit_t* out) {
  if (!out) return DMC_ERR_INVALID_ARG;
  *out = nullptr;
  if (!dmc::valid(cfg) || !arena_dev) return DMC_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(arena_dev) & (dmc::kAlign - 1)) != 0) return DMC_ERR_INVALID_ARG;
  const dmc::Offsets o = dmc::offsets(cfg);
  if (arena_bytes < o.total) return DMC_ERR_ARENA_TOO_SMALL;
  dmc_retrofit* h = new (std::nothrow) dmc_retrofit();
  if (!h) return DMC_ERR_INVALID_ARG;
  h->cfg = *cfg;
  h->at = o;
  h->base = static_cast<char*>(arena_dev);
  cudaPointerAttributes where;
  cudaError_t e = cudaGetDevice(&h->device);
  if (e == cudaSuccess) e = cudaPointerGetAttributes(&where, arena_dev);
  if (e == cudaSuccess && where.type == cudaMemoryTypeDevice && where.device != h->device) {
    delete h;
    return DMC_ERR_INVALID_ARG;  // another device's memory
  }
  if (e == cudaSuccess) e = cudaMemsetAsync(h->base + o.error, 0, o.cleared - o.error, stream);
  if (e != cudaSuccess) {
    delete h;
    return DMC_ERR_CUDA;
  }
  *out = h;
  return DMC_OK;
}

dmc_status dmc_retrofit_destroy(dmc_retrofit_t h) {
  delete h;
  return DMC_OK;
}

size_t dmc_retrofit_saved_bytes(dmc_retrofit_t h, int32_t num_seqs, int32_t total_tokens) {
  if (!h || !dmc::has_heads(h->cfg) || num_seqs < 0 || num_seqs > h->cfg.max_seqs || total_tokens < 0 ||
      total_tokens > h->cfg.max_tokens)
    return 0;
  return (size_t)dmc::pieces(total_tokens, num_seqs, dmc::kStateChunk) * h->cfg.num_kv_heads *
         (2 * h->cfg.head_dim + 4) * 4;
}

dmc_status dmc_retrofit_states(dmc_retrofit_t h, int32_t num_seqs, const void* q_dev, int64_t q_token_stride,
                               int64_t q_head_stride, const void* k_dev, const void* v_dev, const float* noise_dev,
                               float offset, float temperature, const int32_t* cu_seqlens_dev, int32_t total_tokens,
                               int32_t max_seqlen, void* kt_dev, void* vt_dev, float* alpha_dev, float* bias_dev,
                               void* saved_dev, cudaStream_t stream) {
  const int go = seqs_arg(h, num_seqs, cu_seqlens_dev, total_tokens, max_seqlen);
  if (go < 0 || !(temperature > 0.f) || !isfinite(temperature) || !isfinite(offset)) return DMC_ERR_INVALID_ARG;
  if (go == 0) return DMC_OK;
  if (!given(h, q_dev) || q_token_stride < 0 || q_head_stride < 0 || !dmc::given16(k_dev) || !dmc::given16(v_dev) ||
      !dmc::given16(kt_dev) || !dmc::given16(vt_dev) || !dmc::given4(alpha_dev) || !dmc::given4(bias_dev) ||
      !dmc::given16(saved_dev) || (noise_dev && !dmc::given4(noise_dev)))
    return DMC_ERR_INVALID_ARG;
  dmc::StatesArgs a = states_args(h, num_seqs, q_dev, q_token_stride, q_head_stride, k_dev, v_dev, noise_dev, offset,
                                  temperature, cu_seqlens_dev, total_tokens, max_seqlen, saved_dev);
  a.kt = kt_dev;
  a.vt = vt_dev;
  a.alpha = alpha_dev;
  a.bias = bias_dev;
  return dmc::cuda_status(dmc::states_forward(a, bf16(h), h->cfg.head_dim, stream));
}

dmc_status dmc_retrofit_states_backward(dmc_retrofit_t h, int32_t num_seqs, const void* q_dev, int64_t q_token_stride,
                                        int64_t q_head_stride, const void* k_dev, const void* v_dev,
                                        const float* noise_dev, float offset, float temperature,
                                        const int32_t* cu_seqlens_dev, int32_t total_tokens, int32_t max_seqlen,
                                        const void* saved_dev, const void* dkt_dev, const void* dvt_dev,
                                        const void* dbias_dev, const float* dalpha_dev, void* dq_dev,
                                        int64_t dq_token_stride, int64_t dq_head_stride, void* dk_dev, void* dv_dev,
                                        cudaStream_t stream) {
  const int go = seqs_arg(h, num_seqs, cu_seqlens_dev, total_tokens, max_seqlen);
  if (go < 0 || !(temperature > 0.f) || !isfinite(temperature) || !isfinite(offset)) return DMC_ERR_INVALID_ARG;
  if (go == 0) return DMC_OK;
  if (!given(h, q_dev) || q_token_stride < 0 || q_head_stride < 0 || !dmc::given16(k_dev) || !dmc::given16(v_dev) ||
      !dmc::given16(saved_dev) || (noise_dev && !dmc::given4(noise_dev)) || !dmc::given16(dkt_dev) ||
      !dmc::given16(dvt_dev) || !given(h, dbias_dev) || (dalpha_dev && !dmc::given4(dalpha_dev)) || !given(h, dq_dev) ||
      dq_token_stride < 0 || dq_head_stride < 0 || !dmc::given16(dk_dev) || !dmc::given16(dv_dev))
    return DMC_ERR_INVALID_ARG;
  // what is written may not lie in one place
  if ((dq_token_stride == 0 && total_tokens > 1) || (dq_head_stride == 0 && h->cfg.num_q_heads > 1)) return DMC_ERR_INVALID_ARG;
  dmc::StatesArgs a = states_args(h, num_seqs, q_dev, q_token_stride, q_head_stride, k_dev, v_dev, noise_dev, offset,
                                  temperature, cu_seqlens_dev, total_tokens, max_seqlen, const_cast<void*>(saved_dev));
  a.dkt = dkt_dev;
  a.dvt = dvt_dev;
  a.dbias = dbias_dev;
  a.dalpha = dalpha_dev;
  a.dq = dq_dev;
  a.dq_tok = dq_token_stride;
  a.dq_head = dq_head_stride;
  a.dk = dk_dev;
  a.dv = dv_dev;
  return dmc::cuda_status(dmc::states_backward(a, bf16(h), h->cfg.head_dim, stream));
}

dmc_status dmc_retrofit_attention(dmc_retrofit_t h, int32_t num_seqs, const void* q_dev, const void* k_dev,
                                  const void* v_dev, const float* bias_dev, const int32_t* cu_seqlens_dev,
                                  int32_t total_tokens, int32_t max_seqlen, void* out_dev, float* lse_dev,
                                  cudaStream_t stream) {
  const int go = seqs_arg(h, num_seqs, cu_seqlens_dev, total_tokens, max_seqlen);
  if (go < 0) return DMC_ERR_INVALID_ARG;
  if (go == 0) return DMC_OK;
  if (!dmc::given16(q_dev) || !dmc::given16(k_dev) || !dmc::given16(v_dev) || !dmc::given16(out_dev) ||
      !dmc::given4(lse_dev) || (bias_dev && !dmc::given4(bias_dev)))
    return DMC_ERR_INVALID_ARG;
  dmc::AttnArgs a = attn_args(h, num_seqs, q_dev, k_dev, v_dev, bias_dev, cu_seqlens_dev, total_tokens, max_seqlen);
  a.out = out_dev;
  a.lse = lse_dev;
  const int D = h->cfg.head_dim;
  return dmc::cuda_status(bf16(h) ? dmc::attn_forward_bf16(a, D, stream) : dmc::attn_forward_f32(a, D, stream));
}

dmc_status dmc_retrofit_attention_backward(dmc_retrofit_t h, int32_t num_seqs, const void* q_dev, const void* k_dev,
                                           const void* v_dev, const float* bias_dev, const void* out_dev,
                                           const float* lse_dev, const void* dout_dev, const int32_t* cu_seqlens_dev,
                                           int32_t total_tokens, int32_t max_seqlen, void* dq_dev, void* dk_dev,
                                           void* dv_dev, void* dbias_dev, cudaStream_t stream) {
  const int go = seqs_arg(h, num_seqs, cu_seqlens_dev, total_tokens, max_seqlen);
  if (go < 0) return DMC_ERR_INVALID_ARG;
  if (go == 0) return DMC_OK;
  if (!dmc::given16(q_dev) || !dmc::given16(k_dev) || !dmc::given16(v_dev) || !dmc::given16(out_dev) ||
      !dmc::given4(lse_dev) || (bias_dev && !dmc::given4(bias_dev)) || !dmc::given16(dout_dev) ||
      !dmc::given16(dq_dev) || !dmc::given16(dk_dev) || !dmc::given16(dv_dev) || (dbias_dev && !given(h, dbias_dev)))
    return DMC_ERR_INVALID_ARG;
  dmc::AttnArgs a = attn_args(h, num_seqs, q_dev, k_dev, v_dev, bias_dev, cu_seqlens_dev, total_tokens, max_seqlen);
  a.out = const_cast<void*>(out_dev);
  a.lse = const_cast<float*>(lse_dev);
  a.dout = dout_dev;
  a.dq = dq_dev;
  a.dk = dk_dev;
  a.dv = dv_dev;
  a.dbias = dbias_dev;
  const int D = h->cfg.head_dim;
  return dmc::cuda_status(bf16(h) ? dmc::attn_backward_bf16(a, D, stream) : dmc::attn_backward_f32(a, D, stream));
}

dmc_status dmc_retrofit_loss(dmc_retrofit_t h, int32_t num_tokens, const void* hidden_dev, const void* weight_dev,
                             const int32_t* targets_dev, float* loss_dev, float* lse_dev, cudaStream_t stream) {
  if (!usable(h) || !dmc::has_loss(h->cfg) || num_tokens < 0 || num_tokens > h->cfg.max_tokens) return DMC_ERR_INVALID_ARG;
  if (num_tokens == 0) return DMC_OK;
  if (!dmc::given16(hidden_dev) || !dmc::given16(weight_dev) || !dmc::given4(targets_dev) || !dmc::given4(loss_dev) ||
      !dmc::given4(lse_dev))
    return DMC_ERR_INVALID_ARG;
  dmc::LossArgs a = loss_args(h, num_tokens, hidden_dev, weight_dev, targets_dev);
  a.loss = loss_dev;
  a.lse = lse_dev;
  int share = 1;
  if (dmc::loss_forward(a, bf16(h), &share, stream) != cudaSuccess) return DMC_ERR_CUDA;
  dmc::loss_join_kernel<<<dmc::ceil_div(a.N, 8), 256, 0, stream>>>(a, dmc::ceil_div(a.V, share));
  return dmc::cuda_status(cudaGetLastError());
}

dmc_status dmc_retrofit_loss_backward(dmc_retrofit_t h, int32_t num_tokens, const void* hidden_dev,
                                      const void* weight_dev, const int32_t* targets_dev, const float* lse_dev,
                                      const float* dloss_dev, void* dhidden_dev, void* dweight_dev,
                                      cudaStream_t stream) {
  if (!usable(h) || !dmc::has_loss(h->cfg) || num_tokens < 0 || num_tokens > h->cfg.max_tokens) return DMC_ERR_INVALID_ARG;
  if (!dmc::given16(dweight_dev)) return DMC_ERR_INVALID_ARG;
  if (num_tokens == 0)  // no token: no gradient
    return dmc::cuda_status(cudaMemsetAsync(
        dweight_dev, 0, (size_t)h->cfg.vocab * h->cfg.hidden * (bf16(h) ? 2 : 4), stream));
  if (!dmc::given16(hidden_dev) || !dmc::given16(weight_dev) || !dmc::given4(targets_dev) || !dmc::given4(lse_dev) ||
      !dmc::given4(dloss_dev) || !dmc::given16(dhidden_dev))
    return DMC_ERR_INVALID_ARG;
  dmc::LossArgs a = loss_args(h, num_tokens, hidden_dev, weight_dev, targets_dev);
  a.lse = const_cast<float*>(lse_dev);
  a.dloss = dloss_dev;
  a.dhidden = dhidden_dev;
  a.dweight = dweight_dev;
  return dmc::cuda_status(dmc::loss_backward(a, bf16(h), stream));
}

dmc_status dmc_retrofit_status(dmc_retrofit_t h, cudaStream_t stream, uint32_t* bits) {
  if (!usable(h)) return DMC_ERR_INVALID_ARG;
  uint32_t b = 0;
  cudaError_t e = cudaStreamSynchronize(stream);
  if (e == cudaSuccess) e = cudaMemcpy(&b, h->base + h->at.error, 4, cudaMemcpyDeviceToHost);
  if (e != cudaSuccess) return DMC_ERR_CUDA;
  if (bits) *bits = b;
  return b ? DMC_ERR_DEVICE_FAULT : DMC_OK;
}

}  // extern "C"
