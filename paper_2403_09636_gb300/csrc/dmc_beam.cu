// Beam search's selection: the `keep` best continuations among a group's beams x words.
//
// score(b, w) = scores[b] + logits[b, w] - log sum_w' exp(logits[b, w']). Within a beam the order is that of the logits,
// so one pass over them gives both parts: the log-sum (running maximum and sum per lane) and the beam's own best `keep`.
// A row is cut into pieces, a block each, whose warps keep their lists sorted across their lanes: lane i holds the
// i-th best, as one 64-bit key (the logit's bits in an order that compares as whole numbers do, then the word's number
// turned round, so that equal logits go to the lower word). Few elements pass a list's last: with n seen about
// keep (1 + ln(n / keep)) of them. The group's last block (a counter, no waiting) joins the pieces: sums and lists of a
// row by a warp, then the rows' lists by score, in 64 bits.
//
// Bound by HBM (each logit is read once) where there are many, by the chain load - list - join otherwise.
#include <math.h>

#include <new>

#include "dmc_internal.cuh"

namespace dmc {

namespace {

typedef unsigned long long u64;

constexpr int kBeamWarps = 8;
constexpr int kBeamThreads = kBeamWarps * 32;
constexpr int kBeamMost = 32;             // beams of a group, and continuations kept: a lane each
constexpr int kVector = 8;                // words of a lane at a time
constexpr int kStep = 32 * kVector;       // and of a warp
constexpr int kBeamBlocks = 608;          // pieces that rows are cut into, in all: four blocks per SM
constexpr unsigned kFull = 0xffffffffu;

struct BeamArgs {
  int groups, beams, keep, vocab;
  int pieces, per;            // of a row; words of a piece, a multiple of kStep
  const char* logits;
  long long stride;           // bytes between rows
  const float* scores;
  const unsigned char* finished;
  int eos;
  u64* lists;                 // [rows][pieces][keep]
  float2* sums;               // [rows][pieces]: maximum, sum of exponentials
  int* counters;              // [groups]
  float* out_scores;
  int* out_tokens;
  int* out_parents;
  unsigned char* out_done;
};

// A logit's bits in an order that compares as whole numbers do; one that is not a number counts as -infinity.
__device__ __forceinline__ unsigned ordered(float x) {
  const unsigned u = __float_as_uint(x == x ? x : -INFINITY);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(unsigned u) {
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ u64 key_of(float x, int word) { return (u64)ordered(x) << 32 | (unsigned)~word; }

__device__ __forceinline__ u64 shfl64(u64 x, int src) { return __shfl_sync(kFull, x, src); }

// Takes the lanes' keys (0: none) into the warp's list, best first.
__device__ __forceinline__ void take(u64& list, u64& last, u64 key, int lane, int keep) {
  unsigned m = __ballot_sync(kFull, key > last);
  while (m) {
    const u64 x = shfl64(key, __ffs(m) - 1);
    m &= m - 1;
    const int at = __popc(__ballot_sync(kFull, list > x));
    const u64 up = __shfl_up_sync(kFull, list, 1);
    list = lane < at ? list : lane == at ? x : up;
    last = shfl64(list, keep - 1);
    m &= __ballot_sync(kFull, key > last);
  }
}

// Eight words from element i on. Rows may begin at any element: then the 16-byte blocks around them are read and
// shifted (a block that holds one of the row's elements is readable as a whole), so that sums are taken in the same
// order wherever a row lies.
template <typename T>
struct Words {
  static constexpr int N = kVector * (int)sizeof(T) / 16;  // 16-byte blocks
  uint4 u[N + 1];
  __device__ __forceinline__ void load(const char* p, int off, bool more) {  // p: aligned down by off bytes
    const uint4* q = reinterpret_cast<const uint4*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] = __ldg(q + i);
    if (off != 0 && more) u[N] = __ldg(q + N);
  }
  __device__ __forceinline__ void shift(int off) {
    if (off == 0) return;
    unsigned w[4 * N + 4];
#pragma unroll
    for (int i = 0; i <= N; ++i) {
      w[4 * i] = u[i].x;
      w[4 * i + 1] = u[i].y;
      w[4 * i + 2] = u[i].z;
      w[4 * i + 3] = u[i].w;
    }
#pragma unroll
    for (int s = 2; s > 0; s >>= 1)  // whole words
      if (off / 4 & s) {
#pragma unroll
        for (int i = 0; i < 4 * N + 4 - s; ++i) w[i] = w[i + s];
      }
    if (off & 2) {
#pragma unroll
      for (int i = 0; i < 4 * N; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
  __device__ __forceinline__ void unpack(float* x) const {
#pragma unroll
    for (int i = 0; i < N; ++i) Chunk<T>::unpack(u[i], x + i * Chunk<T>::N);
  }
};

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float2 join(float2 a, float2 b) {  // of (maximum, sum)
  const float m = fmaxf(a.x, b.x), r = m == -INFINITY ? 0.f : m;
  return make_float2(m, a.y * exp2f((a.x - r) * kLog2e) + b.y * exp2f((b.x - r) * kLog2e));
}

// A continuation: its score, and beam and word as one number, in order of which ties go.
struct Best {
  double score;
  u64 at;
  __device__ __forceinline__ bool before(const Best& o) const {
    return score > o.score || (score == o.score && at < o.at);
  }
};
__device__ __forceinline__ Best shfl_best(const Best& b, int src) {
  return Best{__shfl_sync(kFull, b.score, src), shfl64(b.at, src)};
}

template <typename T>
__global__ void __launch_bounds__(kBeamThreads) dmc_beam_kernel(const BeamArgs a) {
  __shared__ u64 s_lists[kBeamMost][kBeamMost];  // a list per warp, at the end per beam
  __shared__ float2 s_sums[kBeamWarps];
  __shared__ double s_lse[kBeamMost];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces, group = row / a.beams;
  const bool skip = a.finished != nullptr && a.finished[row];

  if (!skip) {
    const char* p = a.logits + (size_t)row * a.stride;
    const int off = (int)(reinterpret_cast<uintptr_t>(p) & 15);
    const int first = piece * a.per, end = min(first + a.per, a.vocab);
    u64 list = 0, last = 0;
    float m = -INFINITY, sum = 0.f;
    constexpr int U = 4 / Words<T>::N;  // vectors in flight
    for (int i0 = first + warp * kStep + lane * kVector; i0 - lane * kVector < end; i0 += U * kBeamWarps * kStep) {
      Words<T> w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * kBeamWarps * kStep;
        // whole blocks where the row has eight more words; else one word at a time, below
        if (i + kVector <= end) w[u].load(p - off + (size_t)i * sizeof(T), off, true);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * kBeamWarps * kStep;
        if (i - lane * kVector >= end) break;  // the whole warp
        float x[kVector];
        if (i + kVector <= end) {
          w[u].shift(off);
          w[u].unpack(x);
        } else {
#pragma unroll
          for (int e = 0; e < kVector; ++e)
            x[e] = i + e < end ? Elt<T>::to_f(reinterpret_cast<const T*>(p)[i + e]) : -INFINITY;
        }
        float top = x[0];
#pragma unroll
        for (int e = 1; e < kVector; ++e) top = fmaxf(top, x[e]);
        const float mn = fmaxf(m, top), r = mn == -INFINITY ? 0.f : mn;
        float s = sum * exp2f((m - r) * kLog2e);
#pragma unroll
        for (int e = 0; e < kVector; ++e) s += exp2f((x[e] - r) * kLog2e);
        sum = s;
        m = mn;
        if (__any_sync(kFull, ordered(top) >= (unsigned)(last >> 32) && i < end)) {
#pragma unroll
          for (int e = 0; e < kVector; ++e)
            take(list, last, i + e < end ? key_of(x[e], i + e) : 0ull, lane, a.keep);
        }
      }
    }
    float2 ms = make_float2(m, sum);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      ms = join(ms, make_float2(__shfl_xor_sync(kFull, ms.x, o), __shfl_xor_sync(kFull, ms.y, o)));
    s_lists[warp][lane] = list;
    if (lane == 0) s_sums[warp] = ms;
    __syncthreads();
    if (warp == 0) {
      for (int i = lane; i < (kBeamWarps - 1) * 32; i += 32) {
        const u64 key = (i & 31) < a.keep ? s_lists[1 + i / 32][i & 31] : 0ull;
        take(list, last, key, lane, a.keep);
      }
      const size_t at = (size_t)row * a.pieces + piece;
      if (lane < a.keep) a.lists[at * a.keep + lane] = list;
      float2 t = lane < kBeamWarps ? s_sums[lane] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int o = kBeamWarps / 2; o > 0; o >>= 1)
        t = join(t, make_float2(__shfl_xor_sync(kFull, t.x, o), __shfl_xor_sync(kFull, t.y, o)));
      if (lane == 0) a.sums[at] = t;
      __threadfence();
    }
  }
  __syncthreads();
  if (tid == 0) {
    const int all = a.beams * a.pieces;
    const int old = atomicAdd(a.counters + group, 1);
    s_last = old == all - 1;
    if (s_last) a.counters[group] = 0;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();

  // the group's last block: a warp per beam joins its pieces
  for (int b = warp; b < a.beams; b += kBeamWarps) {
    const size_t r = (size_t)group * a.beams + b;
    if (a.finished != nullptr && a.finished[r]) continue;
    float2 ms = make_float2(-INFINITY, 0.f);
    for (int i = lane; i < a.pieces; i += 32) ms = join(ms, __ldcg(a.sums + r * a.pieces + i));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      ms = join(ms, make_float2(__shfl_xor_sync(kFull, ms.x, o), __shfl_xor_sync(kFull, ms.y, o)));
    u64 list = 0, last = 0;
    const u64* from = a.lists + r * a.pieces * a.keep;
    for (int i = lane; i - lane < a.pieces * a.keep; i += 32)
      take(list, last, i < a.pieces * a.keep ? __ldcg(from + i) : 0ull, lane, a.keep);
    s_lists[b][lane] = list;
    if (lane == 0) s_lse[b] = (double)ms.x + log((double)ms.y);
  }
  __syncthreads();
  if (warp != 0) return;
  Best mine{-INFINITY, ~0ull}, worst = mine;
  for (int b = 0; b < a.beams; ++b) {
    const size_t r = (size_t)group * a.beams + b;
    const double base = a.scores[r];
    const bool ended = a.finished != nullptr && a.finished[r];
    Best c{-INFINITY, ~0ull};  // this lane's candidate of the beam
    if (lane < a.keep) {
      // a beam without a finite score (or without a finite log-sum) has nothing to offer: its words at -infinity
      int word = lane;
      double score = -INFINITY;
      if (ended && isfinite(base)) {  // its end word, the others at -infinity
        word = lane == 0 ? a.eos : lane - 1 < a.eos ? lane - 1 : lane;
        if (lane == 0) score = base;
      } else if (!ended && isfinite(base) && isfinite(s_lse[b])) {
        const u64 key = s_lists[b][lane];
        word = key ? (int)~(unsigned)key : a.vocab;
        score = base + ((double)unordered((unsigned)(key >> 32)) - s_lse[b]);
      }
      if (word < a.vocab) c = Best{score, (u64)b << 32 | (unsigned)word};
    }
    unsigned m = __ballot_sync(kFull, c.before(worst));
    while (m) {
      const Best x = shfl_best(c, __ffs(m) - 1);
      m &= m - 1;
      const int at = __popc(__ballot_sync(kFull, mine.before(x)));
      const Best up{__shfl_up_sync(kFull, mine.score, 1), __shfl_up_sync(kFull, mine.at, 1)};
      mine = lane < at ? mine : lane == at ? x : up;
      worst = shfl_best(mine, a.keep - 1);
      m &= __ballot_sync(kFull, c.before(worst));
    }
  }
  const size_t r = (size_t)group * a.beams + min((int)(mine.at >> 32), a.beams - 1);
  const bool ended = a.finished != nullptr && a.finished[r];
  __syncwarp();  // finished and out_done may be one
  if (lane < a.keep) {
    const size_t o = (size_t)group * a.keep + lane;
    const int word = (int)(unsigned)mine.at;
    a.out_scores[o] = (float)mine.score;
    a.out_tokens[o] = word;
    a.out_parents[o] = (int)r;
    a.out_done[o] = ended || word == a.eos;
  }
}

}  // namespace
}  // namespace dmc

struct dmc_beam {
  dmc_beam_config cfg;
  dmc::BeamArgs args;
  int device;
};

namespace {

size_t up(size_t x) { return (x + 255) / 256 * 256; }

bool valid(const dmc_beam_config* c) {
  return c && c->groups >= 1 && c->groups <= (1 << 20) && c->beams >= 1 && c->beams <= dmc::kBeamMost && c->keep >= 1 &&
         c->keep <= dmc::kBeamMost && c->vocab >= 1 && c->vocab <= (1 << 28) &&
         (long long)c->beams * c->vocab >= c->keep && (c->dtype == DMC_F32 || c->dtype == DMC_BF16);
}

// Pieces of a row and the words of one.
void cut(const dmc_beam_config* c, int* pieces, int* per) {
  const long long rows = (long long)c->groups * c->beams;
  const int most = dmc::ceil_div(c->vocab, dmc::kBeamWarps * dmc::kStep);
  const int want = (int)((dmc::kBeamBlocks + rows - 1) / rows);
  const int n = most < want ? most : want;
  *per = dmc::ceil_div(dmc::ceil_div(c->vocab, n), dmc::kStep) * dmc::kStep;
  *pieces = dmc::ceil_div(c->vocab, *per);
}

struct Places {
  size_t lists, sums, counters, total;
};

Places places(const dmc_beam_config* c) {
  int pieces, per;
  cut(c, &pieces, &per);
  const size_t n = (size_t)c->groups * c->beams * pieces;
  Places p;
  p.lists = 0;
  p.sums = up(n * c->keep * 8);
  p.counters = p.sums + up(n * 8);
  p.total = p.counters + up((size_t)c->groups * 4);
  return p;
}

bool aligned(const void* p, size_t n) { return p && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace

extern "C" {

size_t dmc_beam_required_bytes(const dmc_beam_config* cfg) { return valid(cfg) ? places(cfg).total : 0; }

dmc_status dmc_beam_create(const dmc_beam_config* cfg, void* arena_dev, size_t arena_bytes, cudaStream_t stream,
                           dmc_beam_t* out) {
  if (!out) return DMC_ERR_INVALID_ARG;
  *out = nullptr;
  if (!valid(cfg) || !aligned(arena_dev, 256)) return DMC_ERR_INVALID_ARG;
  const Places p = places(cfg);
  if (arena_bytes < p.total) return DMC_ERR_ARENA_TOO_SMALL;
  dmc_beam* h = new (std::nothrow) dmc_beam();
  if (!h) return DMC_ERR_INVALID_ARG;
  h->cfg = *cfg;
  char* base = static_cast<char*>(arena_dev);
  dmc::BeamArgs& a = h->args;
  a.groups = cfg->groups;
  a.beams = cfg->beams;
  a.keep = cfg->keep;
  a.vocab = cfg->vocab;
  cut(cfg, &a.pieces, &a.per);
  a.lists = reinterpret_cast<dmc::u64*>(base + p.lists);
  a.sums = reinterpret_cast<float2*>(base + p.sums);
  a.counters = reinterpret_cast<int*>(base + p.counters);
  cudaError_t e = cudaGetDevice(&h->device);
  if (e == cudaSuccess) e = cudaMemsetAsync(a.counters, 0, (size_t)cfg->groups * 4, stream);
  if (e != cudaSuccess) {
    delete h;
    return DMC_ERR_CUDA;
  }
  *out = h;
  return DMC_OK;
}

dmc_status dmc_beam_destroy(dmc_beam_t h) {
  delete h;
  return DMC_OK;
}

dmc_status dmc_beam_select(dmc_beam_t h, const void* logits_dev, int64_t logits_row_stride, const float* scores_dev,
                           const uint8_t* finished_dev, int32_t eos, float* out_scores_dev, int32_t* out_tokens_dev,
                           int32_t* out_parents_dev, uint8_t* out_done_dev, cudaStream_t stream) {
  if (!h) return DMC_ERR_INVALID_ARG;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return DMC_ERR_CUDA;
  const int es = h->cfg.dtype == DMC_F32 ? 4 : 2;
  if (dev != h->device || !aligned(logits_dev, es) || logits_row_stride < h->cfg.vocab ||
      logits_row_stride > ((int64_t)1 << 40) || !aligned(scores_dev, 4) || !aligned(out_scores_dev, 4) ||
      !aligned(out_tokens_dev, 4) || !aligned(out_parents_dev, 4) || !out_done_dev || eos >= h->cfg.vocab ||
      (finished_dev && eos < 0))
    return DMC_ERR_INVALID_ARG;
  // (in place a group would read what another wrote, unless each keeps as many as it had)
  if (h->cfg.keep != h->cfg.beams && (out_scores_dev == scores_dev || out_done_dev == finished_dev))
    return DMC_ERR_INVALID_ARG;
  dmc::BeamArgs a = h->args;
  a.logits = static_cast<const char*>(logits_dev);
  a.stride = logits_row_stride * es;
  a.scores = scores_dev;
  a.finished = finished_dev;
  a.eos = eos;
  a.out_scores = out_scores_dev;
  a.out_tokens = out_tokens_dev;
  a.out_parents = out_parents_dev;
  a.out_done = out_done_dev;
  const long long blocks = (long long)a.groups * a.beams * a.pieces;
  if (es == 4) dmc::dmc_beam_kernel<float><<<(unsigned)blocks, dmc::kBeamThreads, 0, stream>>>(a);
  else dmc::dmc_beam_kernel<__nv_bfloat16><<<(unsigned)blocks, dmc::kBeamThreads, 0, stream>>>(a);
  return cudaGetLastError() == cudaSuccess ? DMC_OK : DMC_ERR_CUDA;
}

}  // extern "C"
