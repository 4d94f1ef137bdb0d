// Attention of packed sequences in bf16 on the tensor cores: causal, grouped heads, a
// bias per row of K that counts for all later queries.
//
// Forward. A work item is 256 queries of one head of one sequence, as two tiles of 128
// rows that share the K and V tiles; one persistent CTA per SM, its warps specialised:
//   warps 0-3, 4-7  softmax of query tile 0 / 1, one thread per row
//   warp 8          tensor-core work (one thread issues)
//   warp 9          TMA loads: the Q tiles, and a ring of K and V tiles
// and per query tile and 128 rows of K
//   S = Q K^T          into tensor memory
//   softmax            S / sqrt(d) + bias, the running maximum and sum, P = e^(score - max)
//                      in bf16 over the row's S columns
//   O += P V           P read from tensor memory
// P is rounded to bf16, the type of the tensor cores' operand; the sum is taken from the
// unrounded weights. The running maximum moves only when it grows by more than 8 (in log2
// units): P stays below 2^8, and O is rescaled rarely.
//
// Bound by the softmax warps' instructions beside the tensor cores, which are busy for about 70 % of a long
// sequence: 8192 tokens of 64 / 8 heads of 128 800 us, 1.37 PFLOP/s (767 us without biases, 1.43); four
// sequences of 2048, 32 heads, 133 us, 1.03. Heads of 64 do half the products per exponential and are bound by the
// chain of a query tile, S, softmax, P V and the next S over P's columns: tensor pipe 29 %, issue slots 43 %; seven ragged
// sequences of 40 / 8 heads 186 us, 0.58. Short sequences are chains of S, softmax, P V and epilogue, two
// at a time: 24 of 1 to 211 tokens, 32 / 8 heads, 32 us. Slower: the next item's first S before an item's last
// P V (133 -> 138, 800 -> 819; short ones 35 -> 33), the diagonal tile's biases by selects in one loop for
// all tiles (800 -> 915).
#include "dmc_retrofit_attn.cuh"

namespace dmc {

namespace {

constexpr int kItem = 2 * kR;    // queries of a work item
constexpr int kRing = 4;
constexpr float kFarShift = 65536.f;  // log2 units, whose rounding is below 2^-8

template <int D>
struct FwdShared {
  unsigned char q[2][kR * D * 2];       // [64 columns each][128 rows][128 bytes], swizzled
  unsigned char kv[kRing][kR * D * 2];
  unsigned char stage[8][32 * kStageRow];
  float bias[8][2][kR];                 // each softmax warp's copy, this step's and the next's
  uint64_t kv_full[kRing], kv_empty[kRing];
  uint64_t q_full[2], q_empty[2];
  uint64_t s_full[2], p_full[2][2], o_full[2];  // P in two halves
  WorkRing work;
  uint32_t tmem;
  int abort;
};

struct AttnMaps {
  CUtensorMap q, k, v;  // [token][head][D], box: 128 tokens x 64 columns
};

// A work item: queries [q0, q0 + 256) as the query tiles 0 and 1, or, where they all lie in one
// tile, the two tiles' places in turn, so that one such item's softmax runs beside the
// epilogue of the one before.
struct Item {
  int t0, t1;     // the sequence's tokens
  int q[2];       // first query of each tile
  int n[2];       // K tiles that it sees (0: it has no rows)
  int h;
};
__device__ __forceinline__ Item item_of(const Work& w, int& single) {
  Item it;
  it.t0 = w.t0;
  it.t1 = w.t1;
  it.h = w.head;
  it.q[0] = w.t0 + w.at * kItem;
  it.q[1] = it.q[0] + kR;
  it.n[0] = 2 * w.at + 1;
  it.n[1] = it.q[1] < w.t1 ? 2 * w.at + 2 : 0;
  if (it.n[1] == 0) {
    if (single & 1) {
      it.q[1] = it.q[0];
      it.n[1] = it.n[0];
      it.n[0] = 0;
    }
    ++single;
  }
  return it;
}

// multiplies the rows' O (one per lane) by corr
template <int D>
__device__ __forceinline__ void rescale(uint32_t tO, float corr) {
#pragma unroll 1
  for (int c0 = 0; c0 < D; c0 += 32) {
    float f[32];
    uint32_t u[32];
    tc_ld32(tO + c0, f);
    tc_wait_ld();
#pragma unroll
    for (int i = 0; i < 32; ++i) u[i] = __float_as_uint(f[i] * corr);
    tc_st32(tO + c0, u);
  }
}

template <int D, bool kBias>
__global__ void __launch_bounds__(kAttnThreads, 1)
attn_forward_kernel(const AttnArgs a, const __grid_constant__ AttnMaps maps, int items) {
  constexpr int kTile = kR * D * 2;
  extern __shared__ unsigned char smem_raw[];
  FwdShared<D>& sh =
      *reinterpret_cast<FwdShared<D>*>(smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  volatile int* s_abort = &sh.abort;
  if (blockIdx.x == 0) check_seqs(a.seqs, a.error);
  if (tid == 0) {
    for (int i = 0; i < kRing; ++i) {
      mbar_init(smem_u32(&sh.kv_full[i]), 1);
      mbar_init(smem_u32(&sh.kv_empty[i]), 1);
    }
    for (int w = 0; w < 2; ++w) {
      mbar_init(smem_u32(&sh.q_full[w]), 1);
      mbar_init(smem_u32(&sh.q_empty[w]), 1);
      mbar_init(smem_u32(&sh.s_full[w]), 1);
      for (int hf = 0; hf < 2; ++hf) mbar_init(smem_u32(&sh.p_full[w][hf]), 4);
      mbar_init(smem_u32(&sh.o_full[w]), 1);
    }
    work_init(sh.work);
    fence_mbar_init();
    sh.abort = 0;
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(512));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tc_uniform(sh.tmem);
  auto wait = [&](uint64_t* bar, uint32_t ph) -> bool { return warp_wait(smem_u32(bar), ph, s_abort, a.error); };
  auto arrive_warp = [&](uint64_t* bar) {
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(bar));
  };
  if (warp >= 8) {
    // A softmax thread holds a row of scores: 208 registers for those, 88 for the others
    // (256 x 208 + 128 x 88 of the 384 x 168 launched).
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 9) {
      // ---------------------------------------------------------------- loads
      uint32_t n = 0, q_par = 0, q_any = 0;  // bit t: parity of query tile t's next Q, whether there was one
      bool ok = true;
      WorkSource src = work_source(a.seqs);
      int single = 0;
      while (ok) {
        const Work work = take_work(sh.work, src, a.seqs, kItem, false, a.Hq, items, a.counter, wait);
        if (work.head < 0) break;
        const Item w = item_of(work, single);
        const int hk = w.h / a.G, steps = max(w.n[0], w.n[1]);
#pragma unroll 1
        for (int x = 0; x < 2 * steps; ++x, ++n) {
          const int s = n % kRing;
          ok = wait(&sh.kv_empty[s], ((n / kRing) & 1) ^ 1);
          if (!ok) break;
          if (tc_elect()) {
            const uint32_t bar = smem_u32(&sh.kv_full[s]);
            mbar_arrive_expect_tx(bar, kTile);
            load_tile<D>(smem_u32(sh.kv[s]), x & 1 ? &maps.v : &maps.k, bar, hk, w.t0 + (x >> 1) * kR);
          }
          __syncwarp();
          if (x == 0) {
#pragma unroll 1
            for (int t = 0; t < 2 && ok; ++t) {
              if (!w.n[t]) continue;
              ok = wait(&sh.q_empty[t], ~q_par >> t & 1);
              if (!ok) break;
              q_par ^= 1u << t;
              q_any |= 1u << t;
              if (tc_elect()) {
                const uint32_t bar = smem_u32(&sh.q_full[t]);
                mbar_arrive_expect_tx(bar, kTile);
                load_tile<D>(smem_u32(sh.q[t]), &maps.q, bar, w.h, w.q[t]);
              }
              __syncwarp();
            }
          }
          if (!ok) {
            ++n;  // the K tile is on its way
            break;
          }
        }
      }
      // every copy has landed before the CTA may end
      for (uint32_t i = n > kRing ? n - kRing : 0; i < n; ++i)
        mbar_wait(smem_u32(&sh.kv_full[i % kRing]), (i / kRing) & 1, a.error);
      for (int t = 0; t < 2; ++t)
        if (q_any >> t & 1) mbar_wait(smem_u32(&sh.q_full[t]), ~q_par >> t & 1, a.error);
    } else if (warp == 8) {
      // ---------------------------------------------------------------- tensor cores
      uint32_t n = 0;  // ring tiles passed
      uint32_t s_par = 0, v_par = 0, q_par = 0, s_any = 0, v_any = 0;
      bool ok = true;
      const uint64_t k_desc = tc_desc(0, 16, 1024), v_desc = tc_desc(0, kR * 128, 1024);
      const uint32_t kv0 = smem_u32(sh.kv[0]) >> 4, qa = smem_u32(sh.q[0]) >> 4;
      // O of query tile t += P V (ring tile rv)
      auto value = [&](int t, int rv, bool add, bool last) -> bool {
        const uint32_t tS = tmem + t * 128, tO = tmem + 256 + t * D;
        const uint64_t vd = v_desc + (kv0 + rv * (kTile / 16));
#pragma unroll 1
        for (int hf = 0; hf < 2; ++hf) {
          if (!wait(&sh.p_full[t][hf], v_par >> t & 1)) return false;
          if (tc_elect()) {
            tc_fence_after();
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              tc_mma_ts(tO, tS + (hf * 4 + kk) * 8, vd + (hf * 4 + kk) * (2048 / 16), tc_idesc(kR, D, false, true),
                        add || hf || kk > 0);
            if (hf) {
              tc_commit(smem_u32(&sh.o_full[t]));
              if (last) tc_commit(smem_u32(&sh.kv_empty[rv]));
            }
          }
          __syncwarp();
        }
        v_par ^= 1u << t;
        v_any |= 1u << t;
        return true;
      };
      // S of query tile t = Q K^T (ring tile rk). It overwrites P of the step before,
      // whose product has to be over.
      auto score = [&](int t, int rk, bool last, bool last_of_q) -> bool {
        const uint32_t tS = tmem + t * 128;
        const uint64_t qd = k_desc + (qa + t * (kTile / 16)), kd = k_desc + (kv0 + rk * (kTile / 16));
        if ((v_any >> t & 1) && !wait(&sh.o_full[t], ~v_par >> t & 1)) return false;
        if (tc_elect()) {
          tc_fence_after();
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint32_t off = ((kk >> 2) * (kR * 128) + (kk & 3) * 32) / 16;
            tc_mma(tS, qd + off, kd + off, tc_idesc(kR, kR, false, false), kk > 0);
          }
          tc_commit(smem_u32(&sh.s_full[t]));
          if (last) tc_commit(smem_u32(&sh.kv_empty[rk]));
          if (last_of_q) tc_commit(smem_u32(&sh.q_empty[t]));
        }
        __syncwarp();
        s_par ^= 1u << t;
        s_any |= 1u << t;
        return true;
      };
      int turn = 0, single = 0;
      while (ok) {
        const Work work = next_work(sh.work, turn, wait);
        if (work.head < 0) break;
        const Item it = item_of(work, single);
        const int n0 = it.n[0], n1 = it.n[1], steps = max(n0, n1);
        const int keys = it.t1 - it.t0 - (steps - 1) * kR;  // of the last K tile
        // step j: P V of K tile j - 1, then S of tile j, query tile by query tile
#pragma unroll 1
        for (int j = 0; j <= steps && ok; ++j) {
          const uint32_t kt = n + 2 * j, vt = n + 2 * j - 1;
          const int rk = kt % kRing, rv = vt % kRing;
#pragma unroll 1
          for (int t = 0; t < 2 && ok; ++t) {
            const int nt = t ? n1 : n0;
            if (j > 0 && j - 1 < nt) {
              ok = wait(&sh.kv_full[rv], (vt / kRing) & 1);
              if (!ok) break;
              if (j == steps && keys < kR) zero_rows<D>(sh.kv[rv], keys);
              ok = value(t, rv, j > 1, t == 1 || j - 1 >= n1);
              if (!ok) break;
            }
            if (j < nt) {
              if (j == 0) {
                ok = wait(&sh.q_full[t], q_par >> t & 1);
                if (!ok) break;
                q_par ^= 1u << t;
              }
              ok = wait(&sh.kv_full[rk], (kt / kRing) & 1) && score(t, rk, t == 1 || j >= n1, j == nt - 1);
            }
          }
        }
        n += 2 * steps;
      }
      // every product is over before the CTA may end
      for (int t = 0; t < 2; ++t) {
        if (s_any >> t & 1) mbar_wait(smem_u32(&sh.s_full[t]), ~s_par >> t & 1, a.error);
        if (v_any >> t & 1) mbar_wait(smem_u32(&sh.o_full[t]), ~v_par >> t & 1, a.error);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // ---------------------------------------------------------------- softmax
    const int t = warp >> 2, r = tid & (kR - 1), wq = warp & 3;
    const uint32_t lane_base = (uint32_t)(wq * 32) << 16;
    const uint32_t tS = tmem + t * 128 + lane_base, tO = tmem + 256 + t * D + lane_base;
    const float scale = 1.f / sqrtf((float)D);
    const float log2_unit = kBias ? kLog2e : kLog2e * scale;  // of a score as it is kept, in log2 units
    uint32_t steps = 0;
    bool ok = true;
    int turn = 0, single = 0;
    struct Mine {  // an item, for this query tile
      int t1, h, n, row0;  // the sequence's end, head (below 0: no more items), K tiles, the warp's first query
      const float* bias;   // of the first row of K
      int key;             // that row
    };
    // the biases of step j, to this warp's copy
    auto fetch = [&](const Mine& it, int j) {
      if (kBias) {
        const uint32_t dst = smem_u32(sh.bias[warp][j & 1]) + lane * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = j * kR + 32 * i + lane;
          const bool in = it.key + row < it.t1;
          cp_async4_zfill(dst + 128 * i, it.bias + (in ? row : 0), in);
        }
        cp_async_commit();
      }
    };
    // the next item that this query tile has rows of, its first biases on their way
    auto next = [&]() {
      Mine it;
      do {
        const Work work = next_work(sh.work, turn, wait);
        it.h = -1;
        if (work.head < 0) return it;
        const Item x = item_of(work, single);
        it.t1 = x.t1;
        it.h = x.h;
        it.n = t ? x.n[1] : x.n[0];
        it.row0 = (t ? x.q[1] : x.q[0]) + wq * 32;
        it.key = x.t0;
        if (kBias) it.bias = a.bias + (long long)(x.h / a.G) * a.seqs.total + it.key;
      } while (it.n == 0);
      fetch(it, 0);
      return it;
    };
    Mine it = next();
    while (it.h >= 0) {
      const int nt = it.n, row0 = it.row0;
      float m = -INFINITY, l = 0.f;
#pragma unroll 1
      for (int j = 0; j < nt; ++j, ++steps) {
        const float* b = sh.bias[warp][j & 1];
        if (kBias) {
          cp_async_wait<0>();
          __syncwarp();
          if (j + 1 < nt) fetch(it, j + 1);
        }
        if (!(ok = wait(&sh.s_full[t], steps & 1))) break;
        tc_fence_after();
        float s[kR];
#pragma unroll
        for (int c0 = 0; c0 < kR; c0 += 32) tc_ld32(tS + c0, s + c0);
        tc_wait_ld();
        if (kBias && j < nt - 1) {
          // scores in natural units
#pragma unroll
          for (int i = 0; i < kR; i += 4) {
            const float4 c = *reinterpret_cast<const float4*>(b + i);
            const float2 x = fma2(make_float2(s[i], s[i + 1]), make_float2(scale, scale), make_float2(c.x, c.y));
            const float2 y = fma2(make_float2(s[i + 2], s[i + 3]), make_float2(scale, scale), make_float2(c.z, c.w));
            s[i] = x.x; s[i + 1] = x.y; s[i + 2] = y.x; s[i + 3] = y.y;
          }
        } else if (kBias) {
          // the diagonal tile: rows up to the query's own, which has no bias
#pragma unroll
          for (int i = 0; i < kR; i += 4) {
            const float4 c = *reinterpret_cast<const float4*>(b + i);
            const float e[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
            for (int k = 0; k < 4; ++k)
              s[i + k] = i + k > r ? -INFINITY : fmaf(s[i + k], scale, i + k == r ? 0.f : e[k]);
          }
        } else if (j == nt - 1) {
#pragma unroll
          for (int i = 0; i < kR; ++i) s[i] = i > r ? -INFINITY : s[i];
        }
        float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int i = 4; i < kR; i += 8) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            mx[e] = i + e + 4 < kR ? fmaxf(fmaxf(mx[e], s[i + e]), s[i + e + 4]) : fmaxf(mx[e], s[i + e]);
        }
        const float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        {
          const bool grow = (mt - m) * log2_unit > 8.f || m == -INFINITY, resc = grow && m != -INFINITY;
          const float corr = resc ? ex2f((m - mt) * log2_unit) : 1.f;
          if (grow) m = mt;
          l *= corr;
          if (__any_sync(0xffffffffu, resc)) rescale<D>(tO, corr);
        }
        float nm = m == -INFINITY ? 0.f : -m * log2_unit;  // nothing seen yet: every score is -inf
        // A rounding of the shift is the same factor in all of a row's weights, so it may not be large: where the
        // maximum is (that of rows hidden by finite biases as low as the type's lowest, whose shift is not even
        // finite), it is taken off the scores themselves.
        // (8192 tokens of 64 / 8 heads: 801 us as without the test; where there are no biases it would cost 2 %.)
        const bool far = !(fabsf(nm) <= kFarShift);
        if (kBias && __any_sync(0xffffffffu, far)) {
          const float off = far ? m : 0.f;
          if (far) nm = 0.f;
#pragma unroll
          for (int i = 0; i < kR; ++i) s[i] -= off;
        }
        const float2 shift2 = make_float2(nm, nm), unit2 = make_float2(log2_unit, log2_unit);
        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
        for (int c0 = 0; c0 < kR; c0 += 32) {
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float2 x = fma2(make_float2(s[c0 + 2 * i], s[c0 + 2 * i + 1]), unit2, shift2);
            const float2 p = make_float2(ex2f(x.x), ex2f(x.y));
            sum[i & 1] = add2(sum[i & 1], p);
            pk[i] = Chunk<__nv_bfloat16>::pack2(p.x, p.y);
          }
          tc_st16(tS + c0 / 2, pk);
          if (c0 & 32) {
            tc_wait_st();
            tc_fence_before();
            arrive_warp(&sh.p_full[t][c0 / 64]);
          }
        }
        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
      }
      if (!ok) break;
      // ---- the row of O over the row's sum
      const Mine after = next();
      const float inv = 1.f / l;
      if (!(ok = wait(&sh.o_full[t], (steps - 1) & 1))) break;
      tc_fence_after();
      const int rows = it.t1 - row0;  // of the warp that count (may be over 32 or below 1)
      char* out = static_cast<char*>(a.out) + ((long long)row0 * a.Hq + it.h) * (D * 2);
#pragma unroll 1
      for (int c0 = 0; c0 < D; c0 += 32) {
        float o[32];
        tc_ld32(tO + c0, o);
        tc_wait_ld();
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] *= inv;
        write_rows(sh.stage[warp], o, out + c0 * 2, (long long)a.Hq * D * 2, rows);
      }
      if (lane < rows) a.lse[(long long)it.h * a.seqs.total + row0 + lane] = fmaf(m, log2_unit, log2f(l)) * kLn2;
      tc_fence_before();  // the loads of O are done before the next item's P is announced
      it = after;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
  }
  if (tid == 0) work_done(a.counter);
}

template <int D, bool kBias>
cudaError_t forward(const AttnArgs& a, cudaStream_t stream) {
  constexpr int bytes = sizeof(FwdShared<D>) + 1024;
  static_assert(bytes <= 227 * 1024, "one CTA's shared memory");
  AttnMaps maps;
  int sms = 0;
  cudaError_t e = allow_shared<attn_forward_kernel<D, kBias>>(bytes);
  if (e == cudaSuccess) e = sm_count(&sms);
  if (e == cudaSuccess) e = heads_map(&maps.q, a.q, D, a.Hq, a.seqs.total);
  if (e == cudaSuccess) e = heads_map(&maps.k, a.k, D, a.Hkv, a.seqs.total);
  if (e == cudaSuccess) e = heads_map(&maps.v, a.v, D, a.Hkv, a.seqs.total);
  if (e != cudaSuccess) return e;
  const long long items = pieces(a.seqs.total, a.seqs.num, kItem) * a.Hq;
  if (items > INT32_MAX) return cudaErrorInvalidValue;
  attn_forward_kernel<D, kBias><<<(unsigned)(items < sms ? items : sms), kAttnThreads, bytes, stream>>>(a, maps, (int)items);
  return cudaGetLastError();
}

}  // namespace

cudaError_t attn_forward_bf16(const AttnArgs& a, int D, cudaStream_t stream) {
  if (D == 128) return a.bias ? forward<128, true>(a, stream) : forward<128, false>(a, stream);
  return a.bias ? forward<64, true>(a, stream) : forward<64, false>(a, stream);
}

}  // namespace dmc
