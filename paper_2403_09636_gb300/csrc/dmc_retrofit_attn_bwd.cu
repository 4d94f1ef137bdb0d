// Gradients of attention over packed sequences in bf16, on the tensor cores.
//
// With P the softmax weights, delta_i = dO_i . out_i and dS = P (dO V^T - delta):
//   dV = P^T dO,  dK = dS^T Q / sqrt(d),  dQ = dS K / sqrt(d),  dbias_j = sum over i > j of dS_ij
// Two kernels, each with sums of its own rows only, so that nothing is added atomically
// and results do not depend on the order in which CTAs run; S and dO V^T are computed by
// both (7 products of 128 x 128 x D per pair of tiles instead of 5). P and dS are rounded to bf16 as
// operands; dbias is summed from the unrounded dS.
//
// dK, dV: a work item is 128 rows of K and V of one KV head; it walks over the query
// tiles that see them, for all queries of the group, so that a shared head's gradients are
// sums in tensor memory (where such items are few, for a share of the group's heads: attn_shares).
// Everything is transposed, S^T = K Q^T, so that a thread's row is a row of K: P^T and dS^T are
// written over S^T and dP^T and multiply dO and Q from tensor memory, and dbias is a sum within a
// thread. The order of products,
//   dV += P^T dO (step i), dK += dS^T Q (i), S^T (i + 1), dP^T (i + 1),
// leaves one between any two of which the second overwrites what the first reads.
// dQ: a work item is 128 queries of one head; it walks over the K and V tiles they see.
//   S (j + 1), dP (j + 1), dQ += dS K (j)
// with two dP buffers, so that a step's row work runs beside three products.
// delta from the rounded `out` is off by up to 2^-8 |dO| |out|, which in short sequences is the
// largest error of all. But the weights of a row add up to 1, so that the sum of its dS with
// an approximate delta is what delta lacks: dQ's kernel, which runs first, adds it up unrounded, puts
// delta right for dK, dV and dbias, and for its own dS in items of a single tile, whose rows
// see few others (in longer ones the sum over the row of P k, by which it enters, is small).
// In both, warps 0-7 do the row work, four warps for each half of the 128 columns.
//
// Bound by the tensor cores, busy for three quarters of the time, and the row work between two
// products: 8192 tokens of 64 / 8 heads of 128 rows 47, dQ 1138 and dK, dV 1515 us, 1.45 PFLOP/s of the seven
// products; four sequences of 2048, 32 heads, 25, 187 and 241 us. Five products in one kernel would need dQ's sums
// in memory, added atomically in whatever order tiles finish. The rows beyond a sequence's end are
// cleared by the product warp: two more warps that only wait for that slow the others (forward 770 ->
// 930), the row warps are busy (dK and dV of heads of 64 572 -> 600).
#include "dmc_retrofit_attn.cuh"

namespace dmc {
cudaError_t attn_join(const AttnArgs& a, bool bf16, int D, cudaStream_t stream);

namespace {

// Per query: -log-sum (log2 units) and delta, in tiles of 128 queries of one head:
// rows[head][tile][2][128]. Queries beyond a sequence's end get -inf and 0, so that
// their weights are zero.
__device__ __forceinline__ float* row_tile(const AttnArgs& a, int tiles, int head, int tile) {
  return a.rows + ((long long)head * tiles + tile) * (2 * kR);
}
inline int row_tiles(const AttnArgs& a) { return (int)pieces(a.seqs.total, a.seqs.num, kR); }

// Bound by HBM (out and dO read once). Half a warp (D = 64: a quarter) per query.
template <int D>
__global__ void __launch_bounds__(256) attn_rows_kernel(const AttnArgs a, int tiles) {
  constexpr int kLanes = D / 8, kPer = 256 / kLanes;
  const int h = blockIdx.y;
  griddep_launch_dependents();
  if (blockIdx.x == 0 && h == 0) check_seqs(a.seqs, a.error);
  const Piece p = find_piece(a.seqs, kR, blockIdx.x);
  if (!p.ok) return;
  const int tok0 = p.t0 + p.at * kR;
  float* rows = row_tile(a, tiles, h, blockIdx.x);
  const int c = threadIdx.x % kLanes;
#pragma unroll 4
  for (int r = threadIdx.x / kLanes; r < kR; r += kPer) {
    const int tok = tok0 + r;
    float d = 0.f;
    if (tok < p.t1) {
      const long long at = ((long long)tok * a.Hq + h) * D + c * 8;
      float x[8], y[8];
      Chunk<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.out) + at), x);
      Chunk<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.dout) + at), y);
#pragma unroll
      for (int i = 0; i < 8; ++i) d = fmaf(x[i], y[i], d);
    }
#pragma unroll
    for (int off = kLanes / 2; off >= 1; off >>= 1) d += __shfl_xor_sync(0xffffffffu, d, off);
    if (c == 0) {
      rows[r] = tok < p.t1 ? -a.lse[(long long)h * a.seqs.total + tok] * kLog2e : -INFINITY;
      rows[kR + r] = d;
    }
  }
}

// untiled copy of `bytes` (a multiple of 16) into shared memory
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}

struct BwdMaps {
  CUtensorMap q, k, v, o;  // o: dout
};

// ---------------------------------------------------------------- dK, dV, dbias

template <int D>
struct DkvShared {
  unsigned char k[kR * D * 2], v[kR * D * 2];
  unsigned char q[2][kR * D * 2], o[2][kR * D * 2];
  float rows[2][2 * kR];  // of the query tile: -log-sum, delta (with q)
  unsigned char stage[8][32 * kStageRow];
  uint64_t k_full, k_empty, v_full, v_empty;
  uint64_t q_full[2], q_empty[2], o_full[2], o_empty[2];
  uint64_t s_full, dp_full, p_ready, ds_ready, dv_done, dk_done, db_full;
  float db[kR];
  WorkRing work;
  uint32_t tmem;
  int abort;
};

struct DkvItem {
  int t1, j0;      // the sequence's end, the first row of K
  int hk, tile0;   // KV head, the row tile (attn_rows_kernel) of the query tile at j0
  int tiles;       // query tiles that see the rows
  int share, h0;   // share of the group's queries, its first head
  int heads;       // its heads
};
// The group's queries are split over `a.shares` items when there are few (see backward): whole heads,
// the same number in each but for one. KV heads fastest, so that neighbours in the order share tiles of Q and dO.
__device__ __forceinline__ DkvItem dkv_item(const AttnArgs& a, const Work& w) {
  DkvItem it;
  it.t1 = w.t1;
  it.j0 = w.t0 + w.at * kR;
  it.hk = w.head < 0 ? -1 : w.head % a.Hkv;
  it.share = w.head < 0 ? 0 : w.head / a.Hkv;
  const int g0 = it.share * a.G / a.shares;
  it.h0 = it.hk * a.G + g0;
  it.heads = (it.share + 1) * a.G / a.shares - g0;
  it.tile0 = w.t0 / kR + w.seq + w.at;
  it.tiles = (w.t1 - it.j0 + kR - 1) / kR;
  return it;
}

template <int D, bool kBias>
__global__ void __launch_bounds__(kAttnThreads, 1)
attn_dkv_kernel(const AttnArgs a, const __grid_constant__ BwdMaps maps, int items, int row_tiles) {
  constexpr int kTile = kR * D * 2;
  extern __shared__ unsigned char smem_raw[];
  DkvShared<D>& sh = *reinterpret_cast<DkvShared<D>*>(smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  volatile int* s_abort = &sh.abort;
  if (tid == 0) {
    uint64_t* one[] = {&sh.k_full, &sh.k_empty, &sh.v_full, &sh.v_empty, &sh.s_full, &sh.dp_full, &sh.dv_done, &sh.dk_done};
    for (auto* b : one) mbar_init(smem_u32(b), 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sh.q_full[i]), 1);
      mbar_init(smem_u32(&sh.q_empty[i]), 9);  // the product warp, and the row warps that read `rows`
      mbar_init(smem_u32(&sh.o_full[i]), 1);
      mbar_init(smem_u32(&sh.o_empty[i]), 1);
    }
    mbar_init(smem_u32(&sh.db_full), 4);
    mbar_init(smem_u32(&sh.p_ready), 8);
    mbar_init(smem_u32(&sh.ds_ready), 8);
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
  griddep_wait();  // what came before reads only arguments; dQ's kernel leaves delta and the work counter
  const uint32_t tmem = tc_uniform(sh.tmem);
  auto wait = [&](uint64_t* bar, uint32_t ph) -> bool { return warp_wait(smem_u32(bar), ph, s_abort, a.error); };
  auto arrive_warp = [&](uint64_t* bar) {
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(bar));
  };
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 9) {
      // ---------------------------------------------------------------- loads
      uint32_t n = 0, ni = 0;  // query tiles, items
      bool ok = true;
      WorkSource src = work_source(a.seqs);
      while (ok) {
        const Work work = take_work(sh.work, src, a.seqs, kR, true, a.Hkv * a.shares, items, a.counter, wait);
        if (work.head < 0) break;
        const DkvItem w = dkv_item(a, work);
        ok = wait(&sh.k_empty, (ni & 1) ^ 1) && wait(&sh.v_empty, (ni & 1) ^ 1);
        if (!ok) break;
        if (tc_elect()) {
          mbar_arrive_expect_tx(smem_u32(&sh.k_full), kTile);
          load_tile<D>(smem_u32(sh.k), &maps.k, smem_u32(&sh.k_full), w.hk, w.j0);
          mbar_arrive_expect_tx(smem_u32(&sh.v_full), kTile);
          load_tile<D>(smem_u32(sh.v), &maps.v, smem_u32(&sh.v_full), w.hk, w.j0);
        }
        __syncwarp();
        ++ni;
        const int steps = w.heads * w.tiles;
        int h = w.h0, i = 0;
#pragma unroll 1
        for (int x = 0; x < steps; ++x, ++n) {
          const int s = n & 1;
          ok = wait(&sh.q_empty[s], ((n >> 1) & 1) ^ 1);
          if (!ok) break;
          if (tc_elect()) {
            const uint32_t bar = smem_u32(&sh.q_full[s]);
            mbar_arrive_expect_tx(bar, kTile + 8 * kR);
            load_tile<D>(smem_u32(sh.q[s]), &maps.q, bar, h, w.j0 + i * kR);
            bulk_load(smem_u32(sh.rows[s]), row_tile(a, row_tiles, h, w.tile0 + i), 8 * kR, bar);
          }
          __syncwarp();
          ok = wait(&sh.o_empty[s], ((n >> 1) & 1) ^ 1);
          if (tc_elect()) {  // (also after a wait gave up: the drain below expects it)
            const uint32_t bar = smem_u32(&sh.o_full[s]);
            if (ok) {
              mbar_arrive_expect_tx(bar, kTile);
              load_tile<D>(smem_u32(sh.o[s]), &maps.o, bar, h, w.j0 + i * kR);
            } else {
              mbar_arrive(bar);
            }
          }
          __syncwarp();
          if (++i == w.tiles) {
            i = 0;
            ++h;
          }
          if (!ok) {
            ++n;
            break;
          }
        }
      }
      // every copy has landed before the CTA may end
      for (uint32_t x = n > 2 ? n - 2 : 0; x < n; ++x) {
        mbar_wait(smem_u32(&sh.q_full[x & 1]), (x >> 1) & 1, a.error);
        mbar_wait(smem_u32(&sh.o_full[x & 1]), (x >> 1) & 1, a.error);
      }
      if (ni > 0) {
        mbar_wait(smem_u32(&sh.k_full), (ni - 1) & 1, a.error);
        mbar_wait(smem_u32(&sh.v_full), (ni - 1) & 1, a.error);
      }
    } else if (warp == 8) {
      // ---------------------------------------------------------------- products
      const uint64_t kd = tc_desc(0, 16, 1024), md = tc_desc(0, kR * 128, 1024);  // K-major, MN-major
      const uint32_t ks = smem_u32(sh.k) >> 4, vs = smem_u32(sh.v) >> 4, qs = smem_u32(sh.q[0]) >> 4,
                     os = smem_u32(sh.o[0]) >> 4;
      constexpr uint32_t kT16 = kTile / 16;
      uint32_t n = 0, ni = 0;
      bool ok = true;
      // C (128 x 128) = X Y^T over the D columns of two tiles
      auto scores = [&](uint32_t tC, uint32_t x, uint32_t y) {
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t off = ((kk >> 2) * (kR * 128) + (kk & 3) * 32) / 16;
          tc_mma(tC, kd + (x + off), kd + (y + off), tc_idesc(kR, kR, false, false), kk > 0);
        }
      };
      // C (128 x D) += X Y, X in tensor memory: columns 0-63 from tX, 64-127 from tX + 64
      auto sums = [&](uint32_t tC, uint32_t tX, uint32_t y, bool add) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          tc_mma_ts(tC, tX + (kk >> 2) * 64 + (kk & 3) * 8, md + (y + kk * (2048 / 16)), tc_idesc(kR, D, false, true),
                    add || kk > 0);
      };
      int turn = 0;
      while (ok) {
        const Work work = next_work(sh.work, turn, wait);
        if (work.head < 0) break;
        const DkvItem w = dkv_item(a, work);
        const int tiles = w.tiles, steps = w.heads * tiles;
        const int last_rows = w.t1 - w.j0 - (tiles - 1) * kR;  // queries of the last tile
        ok = wait(&sh.k_full, ni & 1) && wait(&sh.v_full, ni & 1);
        int i = 0;  // query tile of step x
#pragma unroll 1
        for (int x = 0; x <= steps && ok; ++x, ++n) {
          // n: the step whose S and dP are due; n - 1 the one whose sums are
          if (x > 0) {
            const uint32_t s = (n - 1) & 1;
            if (!(ok = wait(&sh.p_ready, (n - 1) & 1))) break;
            if (tc_elect()) {
              tc_fence_after();
              sums(tmem + 256, tmem, os + s * kT16, x > 1);
              tc_commit(smem_u32(&sh.dv_done));
              tc_commit(smem_u32(&sh.o_empty[s]));
            }
            __syncwarp();
            if (!(ok = wait(&sh.ds_ready, (n - 1) & 1))) break;
            if (tc_elect()) {
              tc_fence_after();
              sums(tmem + 384, tmem + 128, qs + s * kT16, x > 1);
              tc_commit(smem_u32(&sh.dk_done));
              tc_commit(smem_u32(&sh.q_empty[s]));
            }
            __syncwarp();
          }
          if (x == steps) break;
          const uint32_t s = n & 1;
          const bool cut = i == tiles - 1 && last_rows < kR;
          if (!(ok = wait(&sh.q_full[s], (n >> 1) & 1))) break;
          if (cut) zero_rows<D>(sh.q[s], last_rows);
          if (n > 0 && !(ok = wait(&sh.dv_done, (n - 1) & 1))) break;  // P has been used
          if (tc_elect()) {
            tc_fence_after();
            scores(tmem, ks, qs + s * kT16);
            tc_commit(smem_u32(&sh.s_full));
            if (x == steps - 1) tc_commit(smem_u32(&sh.k_empty));
          }
          __syncwarp();
          if (!(ok = wait(&sh.o_full[s], (n >> 1) & 1))) break;
          if (cut) zero_rows<D>(sh.o[s], last_rows);
          if (n > 0 && !(ok = wait(&sh.dk_done, (n - 1) & 1))) break;  // dS has been used
          if (tc_elect()) {
            tc_fence_after();
            scores(tmem + 128, vs, os + s * kT16);
            tc_commit(smem_u32(&sh.dp_full));
            if (x == steps - 1) tc_commit(smem_u32(&sh.v_empty));
          }
          __syncwarp();
          if (++i == tiles) i = 0;
        }
        ++ni;
      }
      // every product is over before the CTA may end
      if (n > 0) {
        mbar_wait(smem_u32(&sh.dp_full), (n - 1) & 1, a.error);
        mbar_wait(smem_u32(&sh.dk_done), (n - 1) & 1, a.error);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // ---------------------------------------------------------------- rows of K
    const int half = warp >> 2, wq = warp & 3;
    const int r = wq * 32 + lane;            // row of the tile
    const uint32_t lane_base = (uint32_t)(wq * 32) << 16;
    const uint32_t tS = tmem + lane_base + half * 64, tP = tS + 128;  // this thread's columns of S^T, dP^T
    const float scale = 1.f / sqrtf((float)D), qscale = kLog2e * scale;
    const float2 scale2 = make_float2(qscale, qscale);
    uint32_t n = 0, ni = 0;
    bool ok = true;
    int turn = 0;
    float nb = 0.f;  // the next item's bias
    auto next = [&]() {
      const Work work = next_work(sh.work, turn, wait);
      const DkvItem w = dkv_item(a, work);
      nb = 0.f;
      if (kBias && work.head >= 0 && w.j0 + r < w.t1) nb = a.bias[(long long)w.hk * a.seqs.total + w.j0 + r] * kLog2e;
      return w;
    };
    DkvItem w = next();
    while (w.hk >= 0) {
      const int row = w.j0 + r;
      const float b = nb;
      const float2 b2 = make_float2(b, b);
      const int steps = w.heads * w.tiles;
      float2 db = make_float2(0.f, 0.f);
      int i = 0;
#pragma unroll 1
      for (int x = 0; x < steps; ++x, ++n) {
        const int s = n & 1;
        const float* nl = sh.rows[s] + half * 64;
        if (!(ok = wait(&sh.q_full[s], (n >> 1) & 1))) break;  // `rows` came with it
        if (!(ok = wait(&sh.s_full, n & 1))) break;
        tc_fence_after();
        float p[64];
        tc_ld32(tS, p);
        tc_ld32(tS + 32, p + 32);
        tc_wait_ld();
        const bool diag = i == 0;
        if (!diag) {
#pragma unroll
          for (int c = 0; c < 64; c += 4) {
            const float4 l = *reinterpret_cast<const float4*>(nl + c);
            float2 u = fma2(make_float2(p[c], p[c + 1]), scale2, make_float2(l.x, l.y));
            float2 v = fma2(make_float2(p[c + 2], p[c + 3]), scale2, make_float2(l.z, l.w));
            if (kBias) {
              u = add2(u, b2);
              v = add2(v, b2);
            }
            p[c] = ex2f(u.x); p[c + 1] = ex2f(u.y); p[c + 2] = ex2f(v.x); p[c + 3] = ex2f(v.y);
          }
        } else {
          const int own = r - half * 64;  // the column of the row's own query
#pragma unroll
          for (int c = 0; c < 64; ++c) {
            const float e = fmaf(p[c], qscale, nl[c]) + (c == own ? 0.f : b);
            p[c] = c < own ? 0.f : ex2f(e);
          }
        }
        {
          uint32_t pk[32];
#pragma unroll
          for (int c = 0; c < 32; ++c) pk[c] = Chunk<__nv_bfloat16>::pack2(p[2 * c], p[2 * c + 1]);
          tc_st32(tS, pk);
          tc_wait_st();
          tc_fence_before();
          arrive_warp(&sh.p_ready);
        }
        if (!(ok = wait(&sh.dp_full, n & 1))) break;
        tc_fence_after();
        {
          float d[64];
          tc_ld32(tP, d);
          tc_ld32(tP + 32, d + 32);
          tc_wait_ld();
          uint32_t pk[32];
#pragma unroll
          for (int c = 0; c < 64; c += 4) {
            const float4 e = *reinterpret_cast<const float4*>(nl + kR + c);
            const float2 u = mul2(make_float2(p[c], p[c + 1]), add2(make_float2(d[c], d[c + 1]), make_float2(-e.x, -e.y)));
            const float2 v = mul2(make_float2(p[c + 2], p[c + 3]), add2(make_float2(d[c + 2], d[c + 3]), make_float2(-e.z, -e.w)));
            p[c] = u.x; p[c + 1] = u.y; p[c + 2] = v.x; p[c + 3] = v.y;
          }
          if (diag) {
            const int own = r - half * 64;
#pragma unroll
            for (int c = 0; c < 64; ++c) {
              if (c < own) p[c] = 0.f;  // (0 times what need not be a number)
              if (kBias && c != own) db.x += p[c];
            }
          }
#pragma unroll
          for (int c = 0; c < 32; ++c) {
            if (kBias && !diag) db = add2(db, make_float2(p[2 * c], p[2 * c + 1]));
            pk[c] = Chunk<__nv_bfloat16>::pack2(p[2 * c], p[2 * c + 1]);
          }
          tc_st32(tP, pk);
          tc_wait_st();
          tc_fence_before();
          arrive_warp(&sh.q_empty[s]);  // `rows` has been read
          arrive_warp(&sh.ds_ready);
        }
        if (++i == w.tiles) i = 0;
      }
      if (!ok) break;
      // ---- the rows of dV (the first four warps) and dK
      const DkvItem after = next();
      if (!(ok = wait(half ? &sh.dk_done : &sh.dv_done, (n - 1) & 1))) break;
      tc_fence_after();
      const int row0 = w.j0 + wq * 32, rows = w.t1 - row0;
      char* dst = static_cast<char*>(half ? a.dk : a.dv) + ((long long)row0 * a.Hkv + w.hk) * (D * 2);
#pragma unroll 1
      for (int c0 = 0; c0 < D; c0 += 32) {
        float f[32];
        tc_ld32(tmem + lane_base + 256 + half * 128 + c0, f);
        tc_wait_ld();
        if (half)
#pragma unroll
          for (int c = 0; c < 32; ++c) f[c] *= scale;
        if (a.shares == 1) {
          write_rows(sh.stage[warp], f, dst + c0 * 2, (long long)a.Hkv * D * 2, rows);
        } else {
          char* sums = reinterpret_cast<char*>(share_rows(a, D, half, w.share, w.hk, row0) + c0);
#pragma unroll
          for (int c = 0; c < 32; c += 16) {
            uint4 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
              x[i] = make_uint4(__float_as_uint(f[c + 4 * i]), __float_as_uint(f[c + 4 * i + 1]),
                                __float_as_uint(f[c + 4 * i + 2]), __float_as_uint(f[c + 4 * i + 3]));
            write_rows(sh.stage[warp], x, sums + c * 4, D * 4, rows);
          }
        }
      }
      if (kBias && a.dbias) {
        // the sum of the two halves of the columns (the second half's next value is written
        // after the first half's warps have announced the next item's weights)
        const float own = db.x + db.y;
        if (half) sh.db[r] = own;
        if (half) {
          arrive_warp(&sh.db_full);
        } else {
          if (!(ok = wait(&sh.db_full, ni & 1))) break;
          const float all = own + sh.db[r];
          if (row < w.t1) {
            if (a.shares == 1)
              static_cast<__nv_bfloat16*>(a.dbias)[(long long)w.hk * a.seqs.total + row] = __float2bfloat16_rn(all);
            else
              share_dbias(a, D, w.share, w.hk)[row] = all;
          }
        }
      }
      ++ni;
      tc_fence_before();  // the loads of dV and dK are done before the next item's P is announced
      w = after;
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

// ---------------------------------------------------------------- dQ

template <int D>
struct DqShared {
  unsigned char q[kR * D * 2], o[kR * D * 2];
  unsigned char k[3][kR * D * 2];
  unsigned char v[3][kR * 128];  // 64 columns of a V tile each
  float bias[8][2][64];          // each row warp's copy, this step's and the next's
  uint64_t q_full, q_empty, o_full, o_empty;
  uint64_t k_full[3], k_empty[3], v_full[3], v_empty[3];
  uint64_t s_full, s_free, dp_full[2], ds_ready[2], dq_done[2], lack_full;
  float lack[2][2][kR];  // what delta lacks, by the two halves of the columns, of every other item
  WorkRing work;
  uint32_t tmem;
  int abort;
};

struct DqItem {
  int t0, t1, q0;  // the sequence's tokens, the first query
  int h, tile;     // head, row tile (attn_rows_kernel)
  int steps;       // K tiles
};
__device__ __forceinline__ DqItem dq_item(const Work& w) {
  DqItem it;
  it.t0 = w.t0;
  it.t1 = w.t1;
  it.q0 = w.t0 + w.at * kR;
  it.h = w.head;
  it.tile = w.t0 / kR + w.seq + w.at;
  it.steps = w.at + 1;
  return it;
}

template <int D, bool kBias>
__global__ void __launch_bounds__(kAttnThreads, 1)
attn_dq_kernel(const AttnArgs a, const __grid_constant__ BwdMaps maps, int items, int row_tiles) {
  constexpr int kTile = kR * D * 2, kHalves = D / 64;
  extern __shared__ unsigned char smem_raw[];
  DqShared<D>& sh = *reinterpret_cast<DqShared<D>*>(smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  volatile int* s_abort = &sh.abort;
  if (tid == 0) {
    uint64_t* one[] = {&sh.q_full, &sh.q_empty, &sh.o_full, &sh.o_empty, &sh.s_full};
    for (auto* b : one) mbar_init(smem_u32(b), 1);
    for (int i = 0; i < 3; ++i) {
      mbar_init(smem_u32(&sh.k_full[i]), 1);
      mbar_init(smem_u32(&sh.k_empty[i]), 1);
      mbar_init(smem_u32(&sh.v_full[i]), 1);
      mbar_init(smem_u32(&sh.v_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sh.dp_full[i]), 1);
      mbar_init(smem_u32(&sh.ds_ready[i]), 8);
      mbar_init(smem_u32(&sh.dq_done[i]), 1);
    }
    mbar_init(smem_u32(&sh.s_free), 8);
    mbar_init(smem_u32(&sh.lack_full), 8);
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
  griddep_launch_dependents();
  griddep_wait();  // what came before reads only arguments
  const uint32_t tmem = tc_uniform(sh.tmem);
  auto wait = [&](uint64_t* bar, uint32_t ph) -> bool { return warp_wait(smem_u32(bar), ph, s_abort, a.error); };
  auto arrive_warp = [&](uint64_t* bar) {
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(bar));
  };
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 9) {
      // ---------------------------------------------------------------- loads
      uint32_t nk = 0, nv = 0, nq = 0, ni = 0;  // K tiles, V halves, Q tiles and dO tiles requested
      bool ok = true;
      WorkSource src = work_source(a.seqs);
      while (ok) {
        const Work work = take_work(sh.work, src, a.seqs, kR, false, a.Hq, items, a.counter, wait);
        if (work.head < 0) break;
        const DqItem w = dq_item(work);
        const int hk = w.h / a.G;
#pragma unroll 1
        for (int j = 0; j < w.steps && ok; ++j) {
          const uint32_t s = nk % 3;
          if (!(ok = wait(&sh.k_empty[s], ((nk / 3) & 1) ^ 1))) break;
          if (tc_elect()) {
            const uint32_t bar = smem_u32(&sh.k_full[s]);
            mbar_arrive_expect_tx(bar, kTile);
            load_tile<D>(smem_u32(sh.k[s]), &maps.k, bar, hk, w.t0 + j * kR);
          }
          __syncwarp();
          ++nk;
          if (j == 0) {
            if (!(ok = wait(&sh.q_empty, (ni & 1) ^ 1))) break;
            if (tc_elect()) {
              mbar_arrive_expect_tx(smem_u32(&sh.q_full), kTile);
              load_tile<D>(smem_u32(sh.q), &maps.q, smem_u32(&sh.q_full), w.h, w.q0);
            }
            __syncwarp();
            ++nq;
            if (!(ok = wait(&sh.o_empty, (ni & 1) ^ 1))) break;
            if (tc_elect()) {
              mbar_arrive_expect_tx(smem_u32(&sh.o_full), kTile);
              load_tile<D>(smem_u32(sh.o), &maps.o, smem_u32(&sh.o_full), w.h, w.q0);
            }
            __syncwarp();
            ++ni;
          }
#pragma unroll 1
          for (int hf = 0; hf < kHalves; ++hf) {
            const uint32_t c = nv % 3;
            if (!(ok = wait(&sh.v_empty[c], ((nv / 3) & 1) ^ 1))) break;
            if (tc_elect()) {
              const uint32_t bar = smem_u32(&sh.v_full[c]);
              mbar_arrive_expect_tx(bar, kR * 128);
              tma_load(smem_u32(sh.v[c]), &maps.v, bar, hf * 64, hk, w.t0 + j * kR);
            }
            __syncwarp();
            ++nv;
          }
        }
      }
      // every copy has landed before the CTA may end
      for (uint32_t x = nk > 3 ? nk - 3 : 0; x < nk; ++x) mbar_wait(smem_u32(&sh.k_full[x % 3]), (x / 3) & 1, a.error);
      for (uint32_t x = nv > 3 ? nv - 3 : 0; x < nv; ++x) mbar_wait(smem_u32(&sh.v_full[x % 3]), (x / 3) & 1, a.error);
      if (nq > 0) mbar_wait(smem_u32(&sh.q_full), (nq - 1) & 1, a.error);
      if (ni > 0) mbar_wait(smem_u32(&sh.o_full), (ni - 1) & 1, a.error);
    } else if (warp == 8) {
      // ---------------------------------------------------------------- products
      const uint64_t kd = tc_desc(0, 16, 1024), md = tc_desc(0, kR * 128, 1024);
      const uint32_t qs = smem_u32(sh.q) >> 4, os = smem_u32(sh.o) >> 4, ks = smem_u32(sh.k[0]) >> 4,
                     vs = smem_u32(sh.v[0]) >> 4;
      uint32_t n = 0, ni = 0;  // steps, items
      bool ok = true;
      int turn = 0;
      while (ok) {
        const Work work = next_work(sh.work, turn, wait);
        if (work.head < 0) break;
        const DqItem w = dq_item(work);
        const int steps = w.steps;
        const int keys = w.t1 - w.q0;  // rows of the last K tile, the queries' own
        ok = wait(&sh.q_full, ni & 1);
#pragma unroll 1
        for (int x = 0; x <= steps && ok; ++x, ++n) {
          if (x < steps) {
            const uint32_t s = n % 3;
            if (!(ok = wait(&sh.k_full[s], (n / 3) & 1))) break;
            if (x == steps - 1 && keys < kR) zero_rows<D>(sh.k[s], keys);
            if (n > 0 && !(ok = wait(&sh.s_free, (n - 1) & 1))) break;
            if (tc_elect()) {
              tc_fence_after();
#pragma unroll
              for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t off = ((kk >> 2) * (kR * 128) + (kk & 3) * 32) / 16;
                tc_mma(tmem, kd + (qs + off), kd + (ks + s * (kTile / 16) + off), tc_idesc(kR, kR, false, false), kk > 0);
              }
              tc_commit(smem_u32(&sh.s_full));
              if (x == steps - 1) tc_commit(smem_u32(&sh.q_empty));
            }
            __syncwarp();
            if (x == 0 && !(ok = wait(&sh.o_full, ni & 1))) break;
            // the buffer's last dS has been used
            if (n > 1 && !(ok = wait(&sh.dq_done[n & 1], ((n - 2) >> 1) & 1))) break;
#pragma unroll 1
            for (int hf = 0; hf < kHalves; ++hf) {
              const uint32_t v = n * kHalves + hf, c = v % 3;
              if (!(ok = wait(&sh.v_full[c], (v / 3) & 1))) break;
              if (tc_elect()) {
                tc_fence_after();
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                  tc_mma(tmem + 128 + (n & 1) * 128, kd + (os + (hf * (kR * 128) + kk * 32) / 16),
                         kd + (vs + (c * (kR * 128) + kk * 32) / 16), tc_idesc(kR, kR, false, false), hf > 0 || kk > 0);
                tc_commit(smem_u32(&sh.v_empty[c]));
                if (hf == kHalves - 1) {
                  tc_commit(smem_u32(&sh.dp_full[n & 1]));
                  if (x == steps - 1) tc_commit(smem_u32(&sh.o_empty));
                }
              }
              __syncwarp();
            }
            if (!ok) break;
          }
          if (x > 0) {
            const uint32_t y = n - 1, s = y % 3;
            if (!(ok = wait(&sh.ds_ready[y & 1], (y >> 1) & 1))) break;
            if (tc_elect()) {
              tc_fence_after();
#pragma unroll
              for (int kk = 0; kk < 8; ++kk)
                tc_mma_ts(tmem + 384, tmem + 128 + (y & 1) * 128 + (kk >> 2) * 64 + (kk & 3) * 8,
                          md + (ks + s * (kTile / 16) + kk * (2048 / 16)), tc_idesc(kR, D, false, true), x > 1 || kk > 0);
              tc_commit(smem_u32(&sh.dq_done[y & 1]));
              tc_commit(smem_u32(&sh.k_empty[s]));
            }
            __syncwarp();
          }
          if (x == steps) break;
        }
        ++ni;
      }
      // every product is over before the CTA may end
      if (n > 0) {
        mbar_wait(smem_u32(&sh.dp_full[(n - 1) & 1]), ((n - 1) >> 1) & 1, a.error);
        mbar_wait(smem_u32(&sh.dq_done[(n - 1) & 1]), ((n - 1) >> 1) & 1, a.error);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // ---------------------------------------------------------------- rows of Q
    const int half = warp >> 2, wq = warp & 3;
    const int r = wq * 32 + lane;
    const uint32_t lane_base = (uint32_t)(wq * 32) << 16;
    const uint32_t tS = tmem + lane_base + half * 64;
    const float scale = 1.f / sqrtf((float)D), qscale = kLog2e * scale;
    const float2 scale2 = make_float2(qscale, qscale);
    uint32_t n = 0, ni = 0;
    bool ok = true;
    int turn = 0;
    float nrow[2] = {0.f, 0.f};   // the next item's row
    const float* bias = nullptr;  // of the item's first row of K
    // the biases of step j, to this warp's copy
    auto fetch = [&](const DqItem& w, int j) {
      if (kBias) {
        const uint32_t dst = smem_u32(sh.bias[warp][j & 1]) + lane * 4;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int row = j * kR + half * 64 + 32 * i + lane;
          const bool in = w.t0 + row < w.t1;
          cp_async4_zfill(dst + 128 * i, bias + (in ? row : 0), in);
        }
        cp_async_commit();
      }
    };
    auto next = [&]() {  // its numbers on their way
      const Work work = next_work(sh.work, turn, wait);
      const DqItem w = dq_item(work);
      if (work.head >= 0) {
        if (kBias) bias = a.bias + (long long)(w.h / a.G) * a.seqs.total + w.t0;
        fetch(w, 0);
        const float* rows = row_tile(a, row_tiles, w.h, w.tile);
        nrow[0] = rows[r];
        nrow[1] = rows[kR + r];
      }
      return w;
    };
    DqItem w = next();
    while (w.h >= 0) {
      const float nl = nrow[0], delta = nrow[1];
      const float2 nl2 = make_float2(nl, nl), nd2 = make_float2(-delta, -delta);
      float2 lack = make_float2(0.f, 0.f);
      // the row's, from both halves of its columns; by all row warps, once per item
      auto whole = [&](float& sum) {
        float(&l)[2][kR] = sh.lack[ni & 1];
        l[half][r] = lack.x + lack.y;
        arrive_warp(&sh.lack_full);
        if (!wait(&sh.lack_full, ni & 1)) return false;
        sum = l[0][r] + l[1][r];
        return true;
      };
      float sum = 0.f;
#pragma unroll 1
      for (int j = 0; j < w.steps; ++j, ++n) {
        const float* b = sh.bias[warp][j & 1];
        if (kBias) {
          cp_async_wait<0>();
          __syncwarp();
          if (j + 1 < w.steps) fetch(w, j + 1);
        }
        if (!(ok = wait(&sh.s_full, n & 1))) break;
        tc_fence_after();
        float p[64];
        tc_ld32(tS, p);
        tc_ld32(tS + 32, p + 32);
        tc_wait_ld();
        tc_fence_before();
        arrive_warp(&sh.s_free);
        const bool diag = j == w.steps - 1;
        if (!diag) {
#pragma unroll
          for (int c = 0; c < 64; c += 4) {
            float2 u = make_float2(p[c], p[c + 1]), v = make_float2(p[c + 2], p[c + 3]);
            if (kBias) {
              const float4 e = *reinterpret_cast<const float4*>(b + c);
              u = fma2(fma2(u, make_float2(scale, scale), make_float2(e.x, e.y)), make_float2(kLog2e, kLog2e), nl2);
              v = fma2(fma2(v, make_float2(scale, scale), make_float2(e.z, e.w)), make_float2(kLog2e, kLog2e), nl2);
            } else {
              u = fma2(u, scale2, nl2);
              v = fma2(v, scale2, nl2);
            }
            p[c] = ex2f(u.x); p[c + 1] = ex2f(u.y); p[c + 2] = ex2f(v.x); p[c + 3] = ex2f(v.y);
          }
        } else {
          const int own = r - half * 64;
#pragma unroll
          for (int c = 0; c < 64; ++c) {
            const float e = fmaf(fmaf(p[c], scale, kBias && c < own ? b[c] : 0.f), kLog2e, nl);
            p[c] = c > own ? 0.f : ex2f(e);
          }
        }
        if (!(ok = wait(&sh.dp_full[n & 1], (n >> 1) & 1))) break;
        tc_fence_after();
        const uint32_t tP = tmem + 128 + (n & 1) * 128 + lane_base + half * 64;
        float d[64];
        tc_ld32(tP, d);
        tc_ld32(tP + 32, d + 32);
        tc_wait_ld();
#pragma unroll
        for (int c = 0; c < 32; ++c) {
          float2 u = mul2(make_float2(p[2 * c], p[2 * c + 1]), add2(make_float2(d[2 * c], d[2 * c + 1]), nd2));
          if (diag) {  // (0 times what need not be a number)
            if (2 * c > r - half * 64) u.x = 0.f;
            if (2 * c + 1 > r - half * 64) u.y = 0.f;
          }
          lack = add2(lack, u);
          d[2 * c] = u.x;
          d[2 * c + 1] = u.y;
        }
        if (w.steps == 1) {
          if (!(ok = whole(sum))) break;
#pragma unroll
          for (int c = 0; c < 32; ++c) {
            const float2 u = fma2(make_float2(p[2 * c], p[2 * c + 1]), make_float2(-sum, -sum), make_float2(d[2 * c], d[2 * c + 1]));
            d[2 * c] = u.x;
            d[2 * c + 1] = u.y;
          }
        }
        uint32_t pk[32];
#pragma unroll
        for (int c = 0; c < 32; ++c) pk[c] = Chunk<__nv_bfloat16>::pack2(d[2 * c], d[2 * c + 1]);
        tc_st32(tP, pk);
        tc_wait_st();
        tc_fence_before();
        arrive_warp(&sh.ds_ready[n & 1]);
      }
      if (!ok) break;
      // ---- delta as it should be, and this thread's half of its row of dQ
      if (w.steps > 1 && !(ok = whole(sum))) break;
      ++ni;
      if (half == 0 && w.q0 + r < w.t1) row_tile(a, row_tiles, w.h, w.tile)[kR + r] = delta + sum;
      const DqItem after = next();
      if (!(ok = wait(&sh.dq_done[(n - 1) & 1], ((n - 1) >> 1) & 1))) break;
      tc_fence_after();
      constexpr int kCols = D / 2;
      const int tok = w.q0 + r;
      uint4* dst = reinterpret_cast<uint4*>(static_cast<char*>(a.dq) + ((long long)tok * a.Hq + w.h) * (D * 2) + half * (kCols * 2));
#pragma unroll 1
      for (int c0 = 0; c0 < kCols; c0 += 32) {
        float f[32];
        tc_ld32(tmem + lane_base + 384 + half * kCols + c0, f);
        tc_wait_ld();
#pragma unroll
        for (int c = 0; c < 32; ++c) f[c] *= scale;
        if (tok < w.t1)
#pragma unroll
          for (int c = 0; c < 4; ++c) dst[c0 / 8 + c] = Chunk<__nv_bfloat16>::pack(f + 8 * c);
      }
      tc_fence_before();  // the loads of dQ are done before the next item's dS is announced
      w = after;
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

using BwdKernel = void(AttnArgs, BwdMaps, int, int);
cudaError_t dependent(BwdKernel* kernel, int grid, int bytes, cudaStream_t stream, const AttnArgs& a, const BwdMaps& maps,
                      int items, int tiles) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kAttnThreads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, maps, items, tiles);
}

template <int D, bool kBias>
cudaError_t backward(AttnArgs a, cudaStream_t stream) {
  constexpr int dkv_bytes = sizeof(DkvShared<D>) + 1024, dq_bytes = sizeof(DqShared<D>) + 1024;
  static_assert(dkv_bytes <= 227 * 1024 && dq_bytes <= 227 * 1024, "one CTA's shared memory");
  auto* dkv = attn_dkv_kernel<D, kBias>;
  auto* dq = attn_dq_kernel<D, kBias>;
  BwdMaps maps;
  int sms = 0;
  cudaError_t e = allow_shared<attn_dkv_kernel<D, kBias>>(dkv_bytes);
  if (e == cudaSuccess) e = allow_shared<attn_dq_kernel<D, kBias>>(dq_bytes);
  if (e == cudaSuccess) e = sm_count(&sms);
  if (e == cudaSuccess) e = heads_map(&maps.q, a.q, D, a.Hq, a.seqs.total);
  if (e == cudaSuccess) e = heads_map(&maps.k, a.k, D, a.Hkv, a.seqs.total);
  if (e == cudaSuccess) e = heads_map(&maps.v, a.v, D, a.Hkv, a.seqs.total);
  if (e == cudaSuccess) e = heads_map(&maps.o, a.dout, D, a.Hq, a.seqs.total);
  if (e != cudaSuccess) return e;
  const int tiles = row_tiles(a);
  long long dkv_items = (long long)tiles * a.Hkv, dq_items = (long long)tiles * a.Hq;
  if (dq_items > INT_MAX / 2) return cudaErrorInvalidValue;
  // Calls of sequences of up to three tiles (by their max_seqlen) are not split: there a sequence has the same
  // gradients to the bit alone and in any company, a long pack among them. Shares would save up to a quarter (two of
  // 300 tokens, 64 / 8 heads, 82 us, 59 in shares). Whole groups for the short sequences of any other call would hold
  // for those, too, but set its time (300 and 700 tokens, 64 / 8 heads: 96 us, 121 so; 385 and 384, 7 / 1: 45, 74).
  a.shares = a.seqs.longest > 3 * kR ? attn_shares(dkv_items, a.G) : 1;
  if (!kBias) a.dbias = nullptr;
  dkv_items *= a.shares;
  attn_rows_kernel<D><<<dim3(tiles, a.Hq), 256, 0, stream>>>(a, tiles);
  // Each sets itself up while the one before it ends (backward of 256 tokens of 32 heads 31 us, 27 so;
  // of four sequences of 2048, 470 and 461).
  e = cudaGetLastError();
  if (e == cudaSuccess)
    e = dependent(dq, dq_items < sms ? (int)dq_items : sms, dq_bytes, stream, a, maps, (int)dq_items, tiles);
  if (e == cudaSuccess)
    e = dependent(dkv, dkv_items < sms ? (int)dkv_items : sms, dkv_bytes, stream, a, maps, (int)dkv_items, tiles);
  return e == cudaSuccess && a.shares > 1 ? attn_join(a, true, D, stream) : e;
}

}  // namespace

cudaError_t attn_backward_bf16(const AttnArgs& a, int D, cudaStream_t stream) {
  if (D == 128) return a.bias ? backward<128, true>(a, stream) : backward<128, false>(a, stream);
  return a.bias ? backward<64, true>(a, stream) : backward<64, false>(a, stream);
}

}  // namespace dmc
