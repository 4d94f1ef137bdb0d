// Beam search's selection: the `keep` best continuations among a group's beams x words.
//
// score(b, w) = scores[b] + logits[b, w] - log sum_w' exp(logits[b, w']). Within a beam the order is that of the logits,
// so one pass over them gives both parts: the log-sum (running maximum and sum per lane) and the beam's own best `keep`.
// A row is cut into pieces, a block each, whose warps keep their lists sorted across their lanes: lane i holds the
// i-th best, as one 64-bit key (the logit's bits in an order that compares as whole numbers do, then the word's number
// turned round, so that equal logits go to the lower word). Words are held to a bar that few more than `keep` of the
// words so far reach: at first the keep-th largest of the lanes' maxima over the block's first 8192 words, then also the
// least of the warps' ceil(keep / 8)-th best. The group's last block (a counter, no waiting) joins the pieces: sums and
// lists of a row by a warp, then the rows' lists by score, in 48 bits (the log-sum in them is that of fp32 exponentials, off
// by up to some 2^-20, but the same for all of a row's words and for rows that are alike); where sorted lists are joined,
// each entry looks up how many are before it.
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
constexpr int kWords = 32;                // words of a lane at a time
constexpr int kBlock = 32 * kWords;       // words of a warp at a time
// Pieces that rows are cut into, in all: two blocks per SM, as many as fit. 256 rows of 130,003 words, 16 kept, take 32.5 us
// in fp32 and 30 in bf16 with one piece each, 38.7 and 38 with two, 50.5 and 49 with four (one kept: 28 and 23, 30 and 26.5,
// 35 and 32). bf16 has half the bytes but the same instructions for a word, which bound it.
constexpr int kBeamBlocks = 304;
constexpr unsigned kFull = 0xffffffffu;

struct BeamArgs {
  int groups, beams, keep, vocab;
  int pieces, per;            // of a row; words of a piece, a multiple of kBlock
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

// A logit's bits in an order that compares as whole numbers do; one that is not a number counts as -infinity, and the
// zeros of both signs are one number.
__device__ __forceinline__ unsigned ordered(float x) {
  const unsigned u = __float_as_uint(x == x ? __fadd_rn(x, 0.f) : -INFINITY);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(unsigned u) {
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ u64 key_of(float x, int word) { return (u64)ordered(x) << 32 | (unsigned)~word; }

__device__ __forceinline__ u64 shfl64(u64 x, int src) { return __shfl_sync(kFull, x, src); }

// One compare-exchange of a warp's sorting network: lanes `j` apart, the larger key to the lower lane (or, rising, to
// the upper).
template <typename K>
__device__ __forceinline__ K exchange(K key, int lane, int j, bool rising) {
  const K other = __shfl_xor_sync(kFull, key, j);
  return ((lane & j) == 0) != rising ? max(key, other) : min(key, other);
}
template <typename K>
__device__ __forceinline__ K sorted(K key, int lane) {  // falling across the lanes
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int j = k / 2; j > 0; j >>= 1) key = exchange(key, lane, j, (lane & k) != 0);
  return key;
}

// The place of a key that has `before` others before it in its own list, `own`, among N lists of `keep` falling keys: larger
// ones are before it, and (kTies) its equals of lower lists. Places from keep on are not told from each other. A few keys
// are counted one by one, more are searched in five steps, the lists side by side. us of 64 groups of 8 beams over 32,000
// words (bf16) with counting / searching: keep 8 30.3 / 31.4, 32 48.7 / 36.0 (and 33.0 / 31.4 once the scores were no longer
// fp64); of one of 4 beams, keep 4, 10.2 / 11.2.
constexpr int kCountTo = 8;
template <int N, bool kTies, typename K>
__device__ __forceinline__ int place_of(const K (*lists)[32], int n, int own, int before, int keep, K key) {
  if (keep <= kCountTo) {
    for (int v = 0; v < n && before < keep; ++v) {
      if (v == own) continue;
      const bool ties = kTies && v < own;
      for (int j = 0; j < keep && (lists[v][j] > key || (ties && lists[v][j] == key)); ++j) ++before;
    }
    return before;
  }
#pragma unroll
  for (int v0 = 0; v0 < N; v0 += 8) {
    if (v0 >= n) break;
    int at[8] = {};
#pragma unroll
    for (int step = 16; step > 0; step >>= 1)
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int v = min(v0 + u, n - 1), i = at[u] + step - 1;
        const K x = lists[v][min(i, 31)];
        if (i < keep && (x > key || (kTies && v < own && x == key))) at[u] += step;
      }
#pragma unroll
    for (int u = 0; u < 8; ++u) {  // (31 of 32: the last one is still to be looked at)
      const int v = v0 + u;
      if (v >= n || v == own) continue;
      const K x = lists[v][31];
      before += at[u] + (at[u] == 31 && keep == 32 && (x > key || (kTies && v < own && x == key)) ? 1 : 0);
    }
  }
  return before;
}

// A warp's best keys, falling across its lanes, and the keep-th of them.
struct List {
  u64 key, last;
  // Takes the lanes' keys (0: none). A key or four go in one by one (some 150 cycles each), more are sorted and merged
  // (some 800).
  __device__ __forceinline__ void take(u64 x, int lane, int keep) {
    unsigned m = __ballot_sync(kFull, x > last);
    if (__popc(m) > 4) {
      x = sorted(x, lane);
      if (!__any_sync(kFull, key != 0)) {
        key = x;
        last = shfl64(key, keep - 1);
        return;
      }
      key = max(key, shfl64(x, 31 - lane));
#pragma unroll
      for (int j = 16; j > 0; j >>= 1) key = exchange(key, lane, j, false);
      last = shfl64(key, keep - 1);
      return;
    }
    while (m) {
      const u64 y = shfl64(x, __ffs(m) - 1);
      m &= m - 1;
      const int at = __popc(__ballot_sync(kFull, key > y));
      const u64 up = __shfl_up_sync(kFull, key, 1);
      key = lane < at ? key : lane == at ? y : up;
    }
    last = shfl64(key, keep - 1);
  }
};

// A warp's blocks of 1024 words pass through a ring of its own in shared memory, by copies of the 16-byte pieces that
// hold them: rows may begin at any element, pieces are whole (one that holds an element of the row can be read). A lane
// takes the fp32 words lane + 32 j, or the bf16 words 2 lane, 2 lane + 1 of each 64: which ones, and so the order of its
// sum, does not depend on where the row lies.
constexpr int kRing = 3;  // blocks, all but one on their way (one, by loads into registers that the compiler moves down to
                          // their use: 32 groups of 8 beams over 130,003 words 43.4 us, 39.0 so)
template <typename T>
struct Words {
  static constexpr int kBytes = kBlock * (int)sizeof(T), kSlot = kBytes + 16, kPieces = kBytes / 16 / 32;
  static __device__ __forceinline__ int word(int lane, int j) {
    return sizeof(T) == 4 ? lane + 32 * j : j / 2 * 64 + 2 * lane + (j & 1);
  }
  // from: the block's first word; left: the row's bytes from there on
  static __device__ __forceinline__ void copy(uint32_t to, const char* from, long long left, int lane) {
    const int off = (int)(reinterpret_cast<uintptr_t>(from) & 15);
    const char* at = from - off;
    left += off;
#pragma unroll
    for (int i = 0; i <= kPieces; ++i) {
      const int x = (lane + 32 * i) * 16;
      if (i < kPieces ? x < left : lane == 0 && off != 0 && x < left) cp_async16(to + x, at + x);
    }
  }
  static __device__ __forceinline__ void load(float* x, const unsigned char* slot, const char* from, int words, int lane) {
    const int off = (int)(reinterpret_cast<uintptr_t>(from) & 15);
    if constexpr (sizeof(T) == 4) {
      const float* w = reinterpret_cast<const float*>(slot + off) + lane;
#pragma unroll
      for (int j = 0; j < kWords; ++j) x[j] = w[32 * j];
    } else {
      const unsigned* w = reinterpret_cast<const unsigned*>(slot + (off & ~3)) + lane;
      const bool odd = (off & 2) != 0;
#pragma unroll
      for (int j = 0; j < kWords / 2; ++j) {
        unsigned u = w[32 * j];
        if (odd) u = __funnelshift_r(u, w[32 * j + 1], 16);
        Chunk<__nv_bfloat16>::unpack2(u, x[2 * j], x[2 * j + 1]);
      }
    }
    if (words < kBlock) {  // the row's last ones
#pragma unroll
      for (int j = 0; j < kWords; ++j)
        if (word(lane, j) >= words) x[j] = -INFINITY;
    }
  }
};

constexpr float kLog2e = 1.4426950408889634f;

// 2^x; what is below 2^-126 is 0 (a sum of exponentials of which one is 1 does not see it).
__device__ __forceinline__ float pow2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float2 join(float2 a, float2 b) {  // of (maximum, sum)
  const float m = fmaxf(a.x, b.x), r = m == -INFINITY ? 0.f : m;
  return make_float2(m, a.y * pow2((a.x - r) * kLog2e) + b.y * pow2((b.x - r) * kLog2e));
}
__device__ __forceinline__ float2 join_lanes(float2 x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = join(x, make_float2(__shfl_xor_sync(kFull, x.x, o), __shfl_xor_sync(kFull, x.y, o)));
  return x;
}

// Scores and log-sums as sums of two fp32 numbers, the second below half a step of the first: 48 bits. (In fp64 the log-sums
// and scores of eight beams kept a block's warps waiting for an SM's one slow fp64 unit: 3 us of a call's 11.)
struct Two {
  float hi, lo;
};
__device__ __forceinline__ Two two_sum(float a, float b) {  // exactly a + b
  const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
  return Two{s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Two normal(Two x) {
  const float s = __fadd_rn(x.hi, x.lo);
  return Two{s, __fsub_rn(x.lo, __fsub_rn(s, x.hi))};
}
// m + log(s) of s in fp32's normal range: s = 2^e (1 + f), 1 + f within sqrt(2) of 1; log(1 + f) = 2 atanh(q), q = f / (2 + f)
// with its rounding, as 2 q + 2 q (q^2 / 3 + q^4 / 5 + ...), |q| < 0.172: what the series leaves out is below 2^-32.
__device__ __forceinline__ Two log_sum(float m, float s) {
  const unsigned u = __float_as_uint(s);
  int e = (int)(u >> 23) - 127;
  float x = __uint_as_float((u & 0x7fffffu) | 0x3f800000u);
  if (x > 1.41421356f) {
    x *= 0.5f;
    ++e;
  }
  const float f = x - 1.f, d = __fadd_rn(2.f, f), dl = __fsub_rn(f, __fsub_rn(d, 2.f));
  const float q = __fdiv_rn(f, d), ql = __fdiv_rn(fmaf(-q, dl, fmaf(-q, d, f)), d), t = q * q;
  const float p = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.f / 11, 1.f / 9), 1.f / 7), 1.f / 5), 1.f / 3);
  constexpr float kLn2 = 2839.f / 4096, kLn2Rest = 3.19461849453e-5f;  // log 2: twelve bits, which e does not round, and the rest
  const Two a = two_sum((float)e * kLn2, 2.f * q), b = two_sum(m, a.hi);
  const float rest = fmaf(2.f * q, p, fmaf((float)e, kLn2Rest, 2.f * ql));
  // (not a number, infinite or zero: as log says)
  return s > 0.f && s < INFINITY ? normal(Two{b.hi, __fadd_rn(b.lo, __fadd_rn(a.lo, rest))}) : Two{m + logf(s), 0.f};
}
__device__ __forceinline__ Two score_of(float base, float x, Two lse) {
  const Two a = two_sum(base, x), b = two_sum(a.hi, -lse.hi);
  return normal(Two{b.hi, __fadd_rn(b.lo, __fsub_rn(a.lo, lse.lo))});
}

template <typename T>
__global__ void __launch_bounds__(kBeamThreads, 2) dmc_beam_kernel(const BeamArgs a) {
  __shared__ u64 s_keys[kBeamMost][kBeamMost];   // a list per warp, at the end the scores of one per beam
  __shared__ int s_words[kBeamMost][kBeamMost];  // and their words
  __shared__ unsigned s_tops[kBeamWarps][32];    // the warps' lanes' maxima, falling
  __shared__ float2 s_sums[kBeamWarps];
  __shared__ float s_bar;
  __shared__ volatile unsigned s_few[kBeamWarps];  // the warps' lists' ceil(keep / 8)-th best
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, keep = a.keep;
  const int row = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces, group = row / a.beams;
  const bool skip = a.finished != nullptr && a.finished[row];

  if (!skip) {
    using W = Words<T>;
    extern __shared__ __align__(16) unsigned char rings[];
    unsigned char* ring = rings + (size_t)warp * kRing * W::kSlot;
    const char* p = a.logits + (size_t)row * a.stride;
    const int first = piece * a.per, end = min(first + a.per, a.vocab);
    auto issue = [&](int i, int slot) {  // (always committed)
      if (i < end) W::copy(smem_u32(ring) + slot * W::kSlot, p + (size_t)i * sizeof(T), (long long)(end - i) * (int)sizeof(T), lane);
      cp_async_commit();
    };
#pragma unroll
    for (int u = 0; u < kRing - 1; ++u) issue(first + (u * kBeamWarps + warp) * kBlock, u);
    int slot = 0;
    List list{0, 0};
    float m = -INFINITY, sum = 0.f, rest = 0.f, bar = -INFINITY;  // rest: what rounding kept from the sum
    bool fresh = true;
    const int share = (keep + kBeamWarps - 1) / kBeamWarps;
    if (lane == 0) s_few[warp] = 0;
    for (int i0 = first + warp * kBlock; i0 - warp * kBlock < end; i0 += kBeamWarps * kBlock) {
      float x[kWords];
      cp_async_wait<kRing - 2>();
      __syncwarp();  // every lane's pieces of the block are there
      W::load(x, ring + slot * W::kSlot, p + (size_t)i0 * sizeof(T), end - i0, lane);
      issue(i0 + (kRing - 1) * kBeamWarps * kBlock, slot == 0 ? kRing - 1 : slot - 1);  // the one that was read before it
      slot = slot == kRing - 1 ? 0 : slot + 1;
      float tops[4] = {x[0], x[1], x[2], x[3]};  // (four chains: one is 32 dependent steps)
#pragma unroll
      for (int j = 4; j < kWords; ++j) tops[j & 3] = fmaxf(tops[j & 3], x[j]);
      const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(fmaxf(tops[2], tops[3]), -INFINITY));
      if (fresh) {  // a bar that `keep` words of the block's first ones reach: the keep-th of its lanes' maxima
        const unsigned mine = sorted(ordered(top), lane);
        s_tops[warp][lane] = mine;
        __syncthreads();
        if (lane < keep) {  // (a lane's place among all, as for the lists below)
          const int before = place_of<kBeamWarps, true>(s_tops, kBeamWarps, warp, lane, keep, mine);
          if (before == keep - 1) s_bar = unordered(mine);
        }
      }
      const float mn = fmaxf(m, top), r = mn == -INFINITY ? 0.f : mn;
      const float scale = pow2((m - r) * kLog2e);
      sum *= scale;
      rest *= scale;
      float2 s0 = make_float2(0.f, 0.f), s1 = s0, s2 = s0, s3 = s0;
      const float2 r2 = make_float2(-r, -r), l2 = make_float2(kLog2e, kLog2e);
#pragma unroll
      for (int j = 0; j < kWords; j += 8) {
        const float2 d = mul2(add2(make_float2(x[j], x[j + 1]), r2), l2);
        const float2 e = mul2(add2(make_float2(x[j + 2], x[j + 3]), r2), l2);
        const float2 f = mul2(add2(make_float2(x[j + 4], x[j + 5]), r2), l2);
        const float2 h = mul2(add2(make_float2(x[j + 6], x[j + 7]), r2), l2);
        s0 = add2(s0, make_float2(pow2(d.x), pow2(d.y)));
        s1 = add2(s1, make_float2(pow2(e.x), pow2(e.y)));
        s2 = add2(s2, make_float2(pow2(f.x), pow2(f.y)));
        s3 = add2(s3, make_float2(pow2(h.x), pow2(h.y)));
      }
      s0 = add2(add2(s0, s1), add2(s2, s3));
      // (added as they are, the words of a long row far below its largest would be lost one block after another: 4 M words
      // 22 below it took 4e-6 off the log-sum)
      const Two t = two_sum(sum, s0.x + s0.y);
      sum = t.hi;
      rest += t.lo;
      m = mn;
      if (fresh) {
        __syncthreads();
        bar = s_bar;
        fresh = false;
      }
      else {  // `keep` words or more reach the least of what each warp has a share of (later values of it are no less)
        const unsigned least = __reduce_min_sync(kFull, lane < kBeamWarps ? s_few[lane] : 0xffffffffu);
        if (least != 0) bar = fmaxf(bar, unordered(least));
      }
      if (!__any_sync(kFull, top >= bar)) continue;
      // Words that reach the bar, a word of each lane at a time. Where a lane has one it is its largest; where it has
      // more they are read again (which of its registers it wants is not known).
      unsigned masks[4] = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < kWords; ++j) masks[j & 3] |= x[j] >= bar ? 1u << j : 0u;
      unsigned mask = (masks[0] | masks[1]) | (masks[2] | masks[3]);
      const bool more = (mask & (mask - 1)) != 0;
      while (__any_sync(kFull, mask != 0)) {
        const int j = __ffs(mask) - 1, i = i0 + W::word(lane, max(j, 0));
        const bool in = j >= 0 && i < end;
        float v = top;
        if (in && more) v = Elt<T>::to_f(reinterpret_cast<const T*>(p)[i]);
        list.take(in ? key_of(v, i) : 0, lane, keep);
        mask &= mask - 1;
      }
      if (lane == share - 1) s_few[warp] = (unsigned)(list.key >> 32);
    }
    cp_async_wait<0>();
    const float2 ms = join_lanes(make_float2(m, sum + rest));
    // (an empty place's key is below every word's, and its own)
    u64 key = list.key ? list.key : (u64)tid + 1;
    s_keys[warp][lane] = key;
    if (lane == 0) s_sums[warp] = ms;
    __syncthreads();
    const size_t at = (size_t)row * a.pieces + piece;
    if (lane < keep) {
      const int before = place_of<kBeamWarps, false>(s_keys, kBeamWarps, warp, lane, keep, key);
      if (before < keep) a.lists[at * keep + before] = key;
    }
    if (warp == 0) {
      const float2 t = join_lanes(lane < kBeamWarps ? s_sums[lane] : make_float2(-INFINITY, 0.f));
      if (lane == 0) a.sums[at] = t;
    }
    __threadfence();
  }
  __syncthreads();
  if (tid == 0) {
    const int old = atomicAdd(a.counters + group, 1);
    s_last = old == a.beams * a.pieces - 1;
    if (s_last) a.counters[group] = 0;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();

  // the group's last block: a warp per beam joins its pieces and gives its words their scores
  for (int b = warp; b < a.beams; b += kBeamWarps) {
    const size_t r = (size_t)group * a.beams + b;
    const float base = a.scores[r];
    const bool ended = a.finished != nullptr && a.finished[r];
    // a beam without a finite score (or without a finite log-sum) has nothing to offer: its words at -infinity
    int word = lane;
    Two score{-INFINITY, 0.f};
    if (ended) {
      if (isfinite(base)) {  // its end word, the others at -infinity
        word = lane == 0 ? a.eos : lane - 1 < a.eos ? lane - 1 : lane;
        if (lane == 0) score.hi = base;
      }
    } else {
      const u64* from = a.lists + r * a.pieces * keep;
      const int n = a.pieces * keep;
      List list{0, 0};
      u64 next = lane < n ? __ldcg(from + lane) : 0;
      float2 ms = make_float2(-INFINITY, 0.f);
      for (int i = lane; i < a.pieces; i += 32) ms = join(ms, __ldcg(a.sums + r * a.pieces + i));
      if (a.pieces == 1) {
        list.key = next >> 32 ? next : 0;  // in order as it is
      } else {
        for (int i = lane; i - lane < n; i += 32) {
          const u64 x = next;
          next = i + 32 < n ? __ldcg(from + i + 32) : 0;
          list.take(x >> 32 ? x : 0, lane, keep);
        }
      }
      ms = join_lanes(ms);
      // (one lane's: where products are contracted with sums, the two lanes of a pair round different ones)
      const Two lse = log_sum(__shfl_sync(kFull, ms.x, 0), __shfl_sync(kFull, ms.y, 0));
      if (isfinite(base) && isfinite(lse.hi)) {
        word = list.key ? (int)~(unsigned)list.key : a.vocab;
        const float x = unordered((unsigned)(list.key >> 32));
        if (x != -INFINITY) score = score_of(base, x, lse);
      }
    }
    // 0: no word. Rounded to 48 bits, the score of a higher logit can come out a step below a lower one's (a beam at minus
    // its log-sum, logits around half a step of it): no score is above one before it, so that the list is in order.
    u64 key = word < a.vocab ? (u64)ordered(score.hi) << 32 | ordered(score.lo) : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 up = __shfl_up_sync(kFull, key, o);
      if (lane >= o) key = min(key, up);
    }
    s_keys[b][lane] = key;
    s_words[b][lane] = word;
  }
  __syncthreads();
  // a continuation's place is the number of those before it: of higher scores, of equal ones of lower beams (and of its
  // own beam's words before it, which its list has in order)
  constexpr int kMore = kBeamMost * kBeamMost / kBeamThreads;
  int place[kMore];
#pragma unroll
  for (int i = 0; i < kMore; ++i) {
    const int c = tid + i * kBeamThreads, b = c / kBeamMost, j = c % kBeamMost;
    place[i] = keep;
    if (b < a.beams && j < keep && s_keys[b][j] != 0) {
      const u64 key = s_keys[b][j];
      place[i] = place_of<kBeamMost, true>(s_keys, a.beams, b, j, keep, key);
    }
  }
  bool ended[kMore];
#pragma unroll
  for (int i = 0; i < kMore; ++i) {
    const size_t r = (size_t)group * a.beams + min((tid + i * kBeamThreads) / kBeamMost, a.beams - 1);
    ended[i] = a.finished != nullptr && a.finished[r];
  }
  __syncthreads();  // finished and out_done, scores and out_scores may be one
#pragma unroll
  for (int i = 0; i < kMore; ++i) {
    if (place[i] >= keep) continue;
    const int c = tid + i * kBeamThreads, b = c / kBeamMost, j = c % kBeamMost, word = s_words[b][j];
    const size_t o = (size_t)group * keep + place[i];
    a.out_scores[o] = unordered((unsigned)(s_keys[b][j] >> 32));
    a.out_tokens[o] = word;
    a.out_parents[o] = group * a.beams + b;
    a.out_done[o] = ended[i] || word == a.eos;
  }
}

template <typename T>
constexpr int beam_smem() { return kBeamWarps * kRing * Words<T>::kSlot; }

cudaError_t beam_setup(int dtype) {
  return dtype == DMC_F32 ? cudaFuncSetAttribute(dmc_beam_kernel<float>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 beam_smem<float>())
                          : cudaFuncSetAttribute(dmc_beam_kernel<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 beam_smem<__nv_bfloat16>());
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
  const int most = dmc::ceil_div(c->vocab, dmc::kBeamWarps * dmc::kBlock);
  const int want = (int)(rows < dmc::kBeamBlocks ? dmc::kBeamBlocks / rows : 1);
  const int n = most < want ? most : want;
  *per = dmc::ceil_div(dmc::ceil_div(c->vocab, n), dmc::kBlock) * dmc::kBlock;
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
  if (e == cudaSuccess) e = dmc::beam_setup(cfg->dtype);
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
  const unsigned blocks = (unsigned)((long long)a.groups * a.beams * a.pieces);
  if (es == 4) dmc::dmc_beam_kernel<float><<<blocks, dmc::kBeamThreads, dmc::beam_smem<float>(), stream>>>(a);
  else dmc::dmc_beam_kernel<__nv_bfloat16><<<blocks, dmc::kBeamThreads, dmc::beam_smem<__nv_bfloat16>(), stream>>>(a);
  return cudaGetLastError() == cudaSuccess ? DMC_OK : DMC_ERR_CUDA;
}

}  // extern "C"
