// Prompt-phase compression of keys that are already rotated (or have no rotation): the kernels of dmc_prefill.cuh
// without one.
#include "dmc_prefill.cuh"

namespace dmc {

template <typename T, int D>
static cudaError_t launch_prefill(const PrefillArgs& a, cudaStream_t stream) {
  const cudaError_t e = launch_plan<T, D>(a, stream);
  return e != cudaSuccess ? e : launch_scan<T, D, kRotNone>(a, stream);
}

cudaError_t prefill_launch(const Layout& L, int layer, int first_seq, int num_seqs, const void* q,
                           long long q_tok, long long q_head, const void* k, const void* v,
                           const int* cu, int total_tokens, int max_seqlen, float* carry,
                           float* weights, cudaStream_t stream) {
  PrefillArgs a;
  a.lay = L;
  a.layer = layer;
  a.first_seq = first_seq;
  a.num_seqs = num_seqs;
  a.q = static_cast<const char*>(q);
  a.q_tok = q_tok;
  a.q_head = q_head;
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.cu = cu;
  a.total_tokens = total_tokens;
  a.max_seqlen = max_seqlen;
  a.carry = carry;
  a.weights = weights;
  a.at = nullptr;
  a.turns = nullptr;
  a.omegas = nullptr;
  if (L.esize == 4 && L.D == 64) return launch_prefill<float, 64>(a, stream);
  if (L.esize == 4 && L.D == 128) return launch_prefill<float, 128>(a, stream);
  if (L.esize == 2 && L.D == 64) return launch_prefill<__nv_bfloat16, 64>(a, stream);
  if (L.esize == 2 && L.D == 128) return launch_prefill<__nv_bfloat16, 128>(a, stream);
  return cudaErrorInvalidValue;
}

}  // namespace dmc
