// Reordering of a cache's sequences: sequence first + j continues from the cache of sequence first + parents[j], as
// beam search has it after each selection (and as sampling several continuations of one prompt has it once).
//
// A slot is never written again once the head has opened a slot on a later page (Algorithm 1 changes the last slot
// alone), so copies of a sequence share every page but the last: only the page table's entries are copied, and a
// count beside the pool says how many heads hold a page beside the first. The page of the last slot has one holder:
// the first of a sequence's heirs (itself, where it stays) keeps it, every other heir gets a page of its own with the
// rows copied. There are as many of those as sequences that nobody continues, whose last pages they take; where such
// a sequence was empty, they take one from the pool. Pages that nobody holds any more go back to the pool.
//
// Two kernels. The first, a block per (layer, KV head), does the tables and the counts, alone for its pages: sequences
// only ever share pages of one layer and head. It leaves a list of the pages to copy (in the scratch of the layer's
// split attention), which the second spreads over the GPU. Bound by latency: parents, lengths, last entries and the
// table's shares are trips to memory one after the other, then the pages. 64 sequences of 50 pages in 8 layers of 8
// heads, parents drawn afresh each time: 14.7 us (16.8 with one entry of the table in flight per thread instead of
// 8); 4 layers of 32 heads, 4 sequences of 16 pages: 7.6; nobody moved: 3. Blocks of 512 threads take 12.3 and 8.3,
// and 18.4 instead of 13.8 where 1024 heads of 4 sequences are more than one block per SM; eight counts taken down
// together changed nothing.
#include "dmc_internal.cuh"
#include "dmc_reorder.h"

namespace dmc {

namespace {

constexpr int kReorderThreads = 256;
constexpr int kStage = 4096;  // entries of the page table that a block holds at a time
constexpr int kNobody = 0x7fffffff;
constexpr int kCopyBlocks = 1216;  // of the copying kernel, where the heads leave room for more than one each

struct ReorderArgs {
  Layout lay;
  int first, n;
  const int* parents;
};

// Row j's numbers in shared memory.
struct Row {
  int parent;    // who it continues
  int heir;      // of row j: its first heir, j itself as -1; kNobody where nobody continues it
  int len, len_new;
  int last;      // its last page
  int last_new;
};

// A layer's lists of copies: the number of each KV head's, then n places of each head: (from, to, rows).
__device__ __forceinline__ int* copy_counts(const Layout& L, int layer) {
  return reinterpret_cast<int*>(L.partials + (size_t)layer * L.partials_layer_stride);
}
__device__ __forceinline__ int4* copies(const Layout& L, int layer, int h, int n) {
  return reinterpret_cast<int4*>(copy_counts(L, layer) + (L.Hkv + 3) / 4 * 4) + (size_t)h * n;
}

__device__ __forceinline__ void give_back(const Layout& L, int page) {
  const unsigned long long at = atomicAdd(L.pool_top + 2, 1ull);
  L.page_use[at % (unsigned long long)L.num_pages].y = page;
}

// The window's tokens (window grouping), `per` pieces of T for each row: row j gets its parent's. All rows' pieces
// [x0, x0 + w) pass through shared memory together.
template <typename T>
__device__ void move_pieces(T* stage, const Row* rows, int n, T* base, size_t row_stride, int per) {
  const int w = max(1, min(per, (int)(kStage * sizeof(int) / sizeof(T)) / n));
  for (int x0 = 0; x0 < per; x0 += w) {
    const int m = min(w, per - x0);
    for (int i = threadIdx.x; i < n * m; i += kReorderThreads)
      stage[i] = base[(size_t)(i / m) * row_stride + x0 + i % m];
    __syncthreads();
    for (int i = threadIdx.x; i < n * m; i += kReorderThreads) {
      const int j = i / m;
      if (rows[j].parent != j) base[(size_t)j * row_stride + x0 + i % m] = stage[rows[j].parent * m + i % m];
    }
    __syncthreads();
  }
}

__global__ void __launch_bounds__(kReorderThreads) dmc_reorder_kernel(const ReorderArgs a) {
  __shared__ Row rows[kReorderRows];
  __shared__ int extra[kReorderRows], dead[kReorderRows];  // rows that need a last page, rows that give theirs
  __shared__ __align__(16) int stage[kStage];
  __shared__ int s_extras, s_deads, s_pages;
  const Layout& L = a.lay;
  const int n = a.n, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int layer = blockIdx.y, h = blockIdx.x;
  const int parity = *reinterpret_cast<const volatile int*>(&L.ctl[layer * 4]);
  const size_t head0 = (size_t)a.first * L.Hkv + h;  // row j's head of the layer: head0 + j * Hkv
  int* len = L.lengths + ((size_t)layer * 2 + parity) * L.NH + head0;
  int* table = L.page_table + ((size_t)layer * L.NH + head0) * L.MPH;
  const size_t table_row = (size_t)L.Hkv * L.MPH;

  bool moved = false;
  for (int j = tid; j < n; j += kReorderThreads) {
    int p = a.parents[j];
    if (p < 0 || p >= n) {
      atomicOr(L.error, DMC_FAULT_BAD_PARENT);
      p = j;
    }
    const int l = len[(size_t)j * L.Hkv];
    rows[j] = Row{p, kNobody, l, l, -1, -1};
    moved |= p != j;
  }
  griddep_launch_dependents();  // the copying kernel may start its blocks
  if (!__syncthreads_or(moved)) {
    if (tid == 0) copy_counts(L, layer)[h] = 0;
    return;
  }
  for (int j = tid; j < n; j += kReorderThreads) {
    const int p = rows[j].parent, l = rows[j].len;
    atomicMin(&rows[p].heir, p == j ? -1 : j);
    if (l > 0) rows[j].last = table[(size_t)j * table_row + (l - 1) / kPage];
  }
  __syncthreads();
  if (warp == 0) {  // the lists, in the rows' order
    int extras = 0, deads = 0, pages = 0;
    for (int j0 = 0; j0 < n; j0 += 32) {
      const int j = j0 + lane;
      bool ex = false, de = false;
      if (j < n) {
        const Row r = rows[j];
        ex = rows[r.parent].heir != (r.parent == j ? -1 : j) && rows[r.parent].len > 0;
        de = r.heir == kNobody && r.len > 0;
        pages = max(pages, ceil_div(r.len, kPage));
      }
      const unsigned eb = __ballot_sync(0xffffffffu, ex), db = __ballot_sync(0xffffffffu, de);
      const unsigned below = (1u << lane) - 1u;
      if (ex) extra[extras + __popc(eb & below)] = j;
      if (de) dead[deads + __popc(db & below)] = j;
      extras += __popc(eb);
      deads += __popc(db);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) pages = max(pages, __shfl_xor_sync(0xffffffffu, pages, off));
    if (lane == 0) {
      s_extras = extras;
      s_deads = deads;
      s_pages = pages;
    }
  }
  for (int j = tid; j < n; j += kReorderThreads) {
    const int p = rows[j].parent;
    rows[j].len_new = rows[p].len;
    rows[j].last_new = rows[p].last;  // its heir's; the others' below
  }
  __syncthreads();
  const int extras = s_extras, deads = s_deads, pages = s_pages;
  for (int i = tid; i < max(extras, deads); i += kReorderThreads) {
    if (i >= extras) {
      give_back(L, rows[dead[i]].last);
      continue;
    }
    const int page = i < deads ? rows[dead[i]].last : take_page(L);
    Row& r = rows[extra[i]];
    r.last_new = page;
    if (page < 0) r.len_new = 0;  // the pool is empty: so is the sequence (the fault bit is set)
    copies(L, layer, h, n)[i] = make_int4(rows[r.parent].last, page, page < 0 ? 0 : (r.len_new - 1) % kPage + 1, 0);
  }
  if (tid == 0) copy_counts(L, layer)[h] = extras;
  __syncthreads();

  // the pages before the last: holders first come, then go, so that no page that stays in use is given back
  const int w = max(1, min(pages, kStage / n));
  for (int i0 = 0; i0 < pages - 1; i0 += w) {
    const int m = min(w, pages - 1 - i0);
    constexpr int U = 8;  // entries of a thread in flight
    for (int x0 = tid; x0 < n * m; x0 += U * kReorderThreads) {
      int page[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int x = x0 + u * kReorderThreads, j = x / m, i = i0 + x % m;
        page[u] = x < n * m && i < ceil_div(rows[j].len, kPage) - 1 ? table[(size_t)j * table_row + i] : -1;
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (x0 + u * kReorderThreads < n * m) stage[x0 + u * kReorderThreads] = page[u];
    }
    __syncthreads();
    for (int x = tid; x < n * m; x += kReorderThreads) {
      const int j = x / m, i = i0 + x % m, p = rows[j].parent;
      if (p == j || i >= ceil_div(rows[j].len_new, kPage) - 1) continue;
      const int page = stage[p * m + x % m];
      if (page == stage[x]) continue;  // shared already
      atomicAdd(&L.page_use[page].x, 1);
      table[(size_t)j * table_row + i] = page;
    }
    __threadfence();
    __syncthreads();
    for (int x = tid; x < n * m; x += kReorderThreads) {
      const int j = x / m, i = i0 + x % m, p = rows[j].parent;
      const int page = stage[x];
      if (p == j || page < 0) continue;
      if (i < ceil_div(rows[j].len_new, kPage) - 1 && stage[p * m + x % m] == page) continue;
      if (atomicSub(&L.page_use[page].x, 1) == 0) {  // the last holder
        atomicExch(&L.page_use[page].x, 0);
        give_back(L, page);
      }
    }
    __syncthreads();
  }
  for (int j = tid; j < n; j += kReorderThreads) {
    const Row r = rows[j];
    if (r.parent == j) continue;
    if (r.len_new > 0) table[(size_t)j * table_row + (r.len_new - 1) / kPage] = r.last_new;
    len[(size_t)j * L.Hkv] = r.len_new;
  }
  if (L.window > 0) {
    __syncthreads();
    const size_t head = (size_t)layer * L.NH + head0;
    move_pieces(stage, rows, n, L.seglen + ((size_t)layer * 2 + parity) * L.NH + head0, L.Hkv, 1);
    move_pieces(reinterpret_cast<float*>(stage), rows, n, L.ring_w + head * L.window, (size_t)L.Hkv * L.window, L.window);
    const int pieces = L.window * 2 * L.row_bytes / 16;
    move_pieces(reinterpret_cast<uint4*>(stage), rows, n, reinterpret_cast<uint4*>(L.ring) + head * pieces,
                (size_t)L.Hkv * pieces, pieces);
  }
}

// Copies rows [0, rows) of K and V and their z from page to page; what the launch before gave back can be taken from
// here on, and places that failed requests have asked for are there again.
constexpr int kCopyThreads = 256;
__global__ void __launch_bounds__(kCopyThreads) dmc_reorder_copy_kernel(const ReorderArgs a) {
  const Layout& L = a.lay;
  const int tid = threadIdx.x, h = blockIdx.y, layer = blockIdx.z;
  griddep_wait();
  if (tid == 0 && (blockIdx.x | blockIdx.y | blockIdx.z) == 0) {  // (nothing else takes pages now)
    L.pool_top[0] = places_taken(L.pool_top, L.num_pages);
    L.pool_top[3] = 0;
    L.pool_top[1] = L.pool_top[2];
  }
  const int count = copy_counts(L, layer)[h], half = kPage * L.row_bytes;
  for (int i = blockIdx.x; i < count; i += gridDim.x) {
    const int4 c = copies(L, layer, h, a.n)[i];
    const char* from = L.pages + (size_t)c.x * L.page_bytes;
    char* to = L.pages + (size_t)c.y * L.page_bytes;
    const int all = c.z * L.row_bytes;
    if (tid < c.z) L.z[(size_t)c.y * kPage + tid] = L.z[(size_t)c.x * kPage + tid];
    constexpr int U = 2;  // of each half in flight: a page of 256-byte rows in one go
    for (int x0 = tid * 16; x0 < all; x0 += U * kCopyThreads * 16) {
      uint4 k[U], v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int x = x0 + u * kCopyThreads * 16;
        if (x < all) {
          k[u] = *reinterpret_cast<const uint4*>(from + x);
          v[u] = *reinterpret_cast<const uint4*>(from + half + x);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int x = x0 + u * kCopyThreads * 16;
        if (x < all) {
          *reinterpret_cast<uint4*>(to + x) = k[u];
          *reinterpret_cast<uint4*>(to + half + x) = v[u];
        }
      }
    }
  }
}

}  // namespace

cudaError_t reorder_launch(const Layout& L, int first, int n, const int* parents, cudaStream_t stream) {
  const ReorderArgs a{L, first, n, parents};
  dmc_reorder_kernel<<<dim3(L.Hkv, L.L), kReorderThreads, 0, stream>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(max(1, min(n, kCopyBlocks / (L.Hkv * L.L))), L.Hkv, L.L);
  cfg.blockDim = dim3(kCopyThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, dmc_reorder_copy_kernel, a);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace dmc
