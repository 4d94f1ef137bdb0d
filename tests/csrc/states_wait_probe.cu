// Test-only kernel for the waits between chunks of the states' kernels (come_in in dmc_retrofit_states.cu). The test
// builds it with a shortened DMC_WAIT_LIMIT_NS. Even blocks wait for the one neighbour that the odd block after them
// publishes, `delay_ns` after it began, if its number is below `published`.
#include "dmc_retrofit_states.cu"

namespace dmc {
namespace {

constexpr int kD = 64, kRow = kD + 2;

__global__ void __launch_bounds__(32) states_wait_kernel(const StatesArgs a, unsigned int tag, int published,
                                                         unsigned long long delay_ns, float* got, unsigned long long* ns) {
  const int lane = threadIdx.x, pair = blockIdx.x / 2;
  uint64_t* row = a.sums + (long long)pair * 2 * kRow;  // the chunk's own; its neighbour's is the next
  const uint64_t t0 = globaltimer_ns();
  if (blockIdx.x & 1) {
    if (pair >= published) return;
    for (int i = 0; i < 100000 && globaltimer_ns() - t0 < delay_ns; ++i) __nanosleep(1000);
    const float2 x[1] = {make_float2(lane + 0.25f, lane + 0.5f)};
    publish<2>(row + kRow, x, tag);
    if (lane == 0) publish_zp<kD>(row + kRow, 3.f, 0.5f, tag);
    return;
  }
  float2 x[1];
  const float z = come_in<kD>(a, row, a.carry, 1, kRow, tag, x);
  float* to = got + (pair * 32 + lane) * 3;
  to[0] = x[0].x;
  to[1] = x[0].y;
  to[2] = z;
  ns[pair * 32 + lane] = globaltimer_ns() - t0;
}

}  // namespace
}  // namespace dmc

extern "C" int dmc_states_wait_probe(int pairs, unsigned int tag, int published, unsigned long long delay_ns, uint64_t* rows_dev,
                                     unsigned int* turns_dev, unsigned int* err_dev, float* got_dev, unsigned long long* ns_dev,
                                     cudaStream_t stream) {
  if (pairs < 1 || pairs > 64) return (int)cudaErrorInvalidValue;
  dmc::StatesArgs a = {};
  a.sums = a.carry = rows_dev;
  a.turns = turns_dev;
  a.error = err_dev;
  dmc::states_wait_kernel<<<2 * pairs, 32, 0, stream>>>(a, tag, published, delay_ns, got_dev, ns_dev);
  return (int)cudaGetLastError();
}
