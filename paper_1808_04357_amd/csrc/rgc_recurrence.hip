// rgc_recurrence.hip -- the gated linear recurrence, forward and backward (include/rgc.h has the formulas).
//
// 1 - sigmoid(v) is computed as sigmoid(-v), which keeps its precision where the gate is nearly open.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rgc_lm.h"

namespace rgc {
namespace {

constexpr uint32_t kChunk = 256;       // steps between kept states (RGC_RECURRENCE_CHUNK)
constexpr uint32_t kThreads = 64;
constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float sigmoid(float v) { return 1.0f / (1.0f + __builtin_amdgcn_exp2f(-kLog2e * v)); }

template <typename T>
__device__ __forceinline__ float read(const SequenceView& v, uint32_t b, uint32_t t, uint32_t c) {
  return static_cast<float>(static_cast<const T*>(v.data)[b * v.batch_stride + t * v.step_stride + c]);
}
template <typename T>
__device__ __forceinline__ void write(const SequenceView& v, uint32_t b, uint32_t t, uint32_t c, float value) {
  static_cast<T*>(v.data)[b * v.batch_stride + t * v.step_stride + c] = static_cast<T>(value);
}

__device__ __forceinline__ uint32_t length_of(const RecurrenceArgs& A, uint32_t b) {
  if (!A.lengths) return A.steps;
  const int32_t n = A.lengths[b];
  return n < 0 ? 0u : min(static_cast<uint32_t>(n), A.steps);
}

__device__ __forceinline__ bool starts_anew(const RecurrenceArgs& A, uint32_t b, uint32_t t) {
  return A.resets && A.resets[static_cast<uint64_t>(b) * A.steps + t] != 0;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) recurrence_kernel(RecurrenceArgs A) {
  const uint32_t across = (A.width + kThreads - 1u) / kThreads;      // workgroups a sequence takes
  const uint32_t b = blockIdx.x / across, c = (blockIdx.x - b * across) * kThreads + threadIdx.x;
  if (c >= A.width) return;
  const uint32_t n = length_of(A, b), chunks = (A.steps + kChunk - 1u) / kChunk;
  const uint64_t at = static_cast<uint64_t>(b) * A.width + c;
  float h = A.h0 ? A.h0[at] : 0.0f;
  for (uint32_t t = 0; t < A.steps; ++t) {
    if (A.states && t % kChunk == 0u) A.states[(static_cast<uint64_t>(b) * chunks + t / kChunk) * A.width + c] = h;
    if (t >= n) {
      write<T>(A.y, b, t, c, 0.0f);
      continue;
    }
    const float v = read<T>(A.gate, b, t, c);
    const float before = starts_anew(A, b, t) ? 0.0f : h;
    h = sigmoid(v) * before + sigmoid(-v) * read<T>(A.x, b, t, c);
    write<T>(A.y, b, t, c, A.out_gate.data ? sigmoid(read<T>(A.out_gate, b, t, c)) * h : h);
  }
  if (A.h_last) A.h_last[at] = h;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) recurrence_backward_kernel(RecurrenceArgs A, RecurrenceGradArgs G) {
  __shared__ float states[kChunk][kThreads];      // the state before every step of the chunk
  const uint32_t across = (A.width + kThreads - 1u) / kThreads;      // workgroups a sequence takes
  const uint32_t b = blockIdx.x / across, c = (blockIdx.x - b * across) * kThreads + threadIdx.x;
  if (c >= A.width) return;
  const uint32_t n = length_of(A, b), chunks = (A.steps + kChunk - 1u) / kChunk;
  const uint64_t at = static_cast<uint64_t>(b) * A.width + c;
  float d = G.dh_last ? G.dh_last[at] : 0.0f;     // of the loss, by the state after the step at hand
  for (uint32_t chunk = chunks; chunk-- > 0u;) {
    const uint32_t first = chunk * kChunk, end = min(first + kChunk, A.steps);
    float h = A.states[(static_cast<uint64_t>(b) * chunks + chunk) * A.width + c];
    for (uint32_t t = first; t < end && t < n; ++t) {
      const float v = read<T>(A.gate, b, t, c);
      const float before = starts_anew(A, b, t) ? 0.0f : h;
      states[t - first][threadIdx.x] = before;
      h = sigmoid(v) * before + sigmoid(-v) * read<T>(A.x, b, t, c);
    }
    for (uint32_t t = end; t-- > first;) {
      if (t >= n) {
        write<T>(G.dx, b, t, c, 0.0f);
        write<T>(G.dgate, b, t, c, 0.0f);
        if (A.out_gate.data) write<T>(G.dout_gate, b, t, c, 0.0f);
        continue;
      }
      const float v = read<T>(A.gate, b, t, c), x = read<T>(A.x, b, t, c), dy = read<T>(G.dy, b, t, c);
      const float keep = sigmoid(v), take = sigmoid(-v), before = states[t - first][threadIdx.x];
      if (A.out_gate.data) {
        const float w = read<T>(A.out_gate, b, t, c), open = sigmoid(w);
        write<T>(G.dout_gate, b, t, c, dy * (keep * before + take * x) * open * sigmoid(-w));
        d += dy * open;
      } else {
        d += dy;
      }
      write<T>(G.dx, b, t, c, d * take);
      write<T>(G.dgate, b, t, c, d * (before - x) * keep * take);
      d = starts_anew(A, b, t) ? 0.0f : keep * d;
    }
  }
  if (G.dh0) G.dh0[at] = d;
}

}  // namespace

#define RGC_BY_TYPE(dtype, launch)                      \
  do {                                                  \
    if ((dtype) == 0) { using T = float; launch; }      \
    else if ((dtype) == 1) { using T = __bf16; launch; } \
    else { using T = _Float16; launch; }                \
  } while (0)

hipError_t launch_recurrence(const RecurrenceArgs& a, int dtype, hipStream_t s) {
  const dim3 grid((a.width + kThreads - 1u) / kThreads * a.batch);
  RGC_BY_TYPE(dtype, (recurrence_kernel<T><<<grid, dim3(kThreads), 0, s>>>(a)));
  return hipGetLastError();
}

hipError_t launch_recurrence_backward(const RecurrenceArgs& a, const RecurrenceGradArgs& g, int dtype, hipStream_t s) {
  const dim3 grid((a.width + kThreads - 1u) / kThreads * a.batch);
  RGC_BY_TYPE(dtype, (recurrence_backward_kernel<T><<<grid, dim3(kThreads), 0, s>>>(a, g)));
  return hipGetLastError();
}

}  // namespace rgc
