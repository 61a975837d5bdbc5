// rgc_parts.hip -- sums of what workgroups left of gradients that many of them have a part in: [count][columns] numbers, added up over `count`.
//
// A workgroup takes 64 columns.  Each wave adds up neighbouring rows in their order, then the waves' sums are added in theirs: the result depends on the sizes alone.
// It is bound by the parts' reading, which mostly comes from the caches, and by the launch.
#include <hip/hip_runtime.h>

#include "rgc_lm.h"
#include "rgc_sequence.h"

namespace rgc {
namespace {

constexpr uint32_t kWaves = 8;

__global__ void __launch_bounds__(64 * kWaves) sum_parts_kernel(PartsArgs P, uint64_t begin) {
  __shared__ float sums[kWaves][64];
  const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6);
  const uint64_t column = (begin + blockIdx.x) * 64u + lane, each = (P.count + kWaves - 1u) / kWaves;
  const uint64_t upto = min(P.count, (wave + 1u) * each);
  float sum = 0.0f;
  if (column < P.columns) {
#pragma unroll 8
    for (uint64_t p = wave * each; p < upto; ++p) sum += P.parts[p * P.columns + column];
  }
  sums[wave][lane] = sum;
  __syncthreads();
  if (wave > 0u || column >= P.columns) return;
  for (uint32_t w = 1; w < kWaves; ++w) sum += sums[w][lane];
  uint64_t first = 0;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    if (column >= first && column < P.ends[i] && P.to[i]) P.to[i][column - first] = sum;
    first = P.ends[i];
  }
}

}  // namespace

hipError_t launch_sum_parts(const PartsArgs& a, hipStream_t s) {
  in_grids((a.columns + 63u) / 64u, [&](uint64_t begin, dim3 grid) { sum_parts_kernel<<<grid, dim3(64 * kWaves), 0, s>>>(a, begin); });
  return hipGetLastError();
}

}  // namespace rgc
