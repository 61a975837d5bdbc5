// rgc_vocab.hip -- operators over rows of logits: log probabilities of given tokens with entropy and top alternatives, their
// gradient, and the distillation loss with its gradient (include/rgc.h has the formulas).
//
// A softmax is computed in powers of two: with c = log2(e) / T and M the row's largest logit, a_j = (z_j - M) c, S = sum 2^a_j,
//   log p_j = ln 2 * (a_j - log2 S),   entropy = ln 2 * (log2 S - sum 2^a_j a_j / S).
// The difference is taken before the scaling: z_j c overflows for logits near the type's lowest value, with which masks are written.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rgc_lm.h"

namespace rgc {
namespace {

constexpr uint32_t kThreads = 256, kWaves = kThreads / 64u;
constexpr float kLn2 = 0.693147180559945309f;
constexpr uint32_t kTopMost = 128;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }   // 1 ulp; a result below 2^-126 is 0
__device__ __forceinline__ float log2_of(float x) { return __builtin_amdgcn_logf(x); }    // 1 ulp; log2(0) = -inf

// (z - m) c; a row of nothing but -inf has m = -inf, and every element has probability 0.
__device__ __forceinline__ float exponent(float z, float m, float c) { return m == -INFINITY ? -INFINITY : (z - m) * c; }

// ln of a logit's probability, given ln S; -inf for every logit of a row of nothing but -inf.
__device__ __forceinline__ float log_probability(float z, float m, float inv_t, float log_sum) {
  return m == -INFINITY ? m : (z - m) * inv_t - log_sum;
}

// Sums over the elements seen so far: m the largest, s = sum 2^a, e = sum 2^a a.
struct Sums {
  float m, s, e;
};

__device__ __forceinline__ float finite_or_zero_weight(float a) { return fmaxf(a, -200.0f); }   // 2^-200 is 0 in fp32, and 0 * -inf is not

// The two sets of elements as one: the one with the smaller maximum is scaled down.
__device__ __forceinline__ Sums join(const Sums& x, const Sums& y, float c) {
  const float m = fmaxf(x.m, y.m);
  if (m == -INFINITY) return Sums{m, x.s + y.s, x.e + y.e};        // (nothing but -inf on either side: zeros, or NaN)
  const float ax = finite_or_zero_weight((x.m - m) * c), ay = finite_or_zero_weight((y.m - m) * c);
  const float wx = exp2_of((x.m - m) * c), wy = exp2_of((y.m - m) * c);
  return Sums{m, x.s * wx + y.s * wy, wx * (x.e + x.s * ax) + wy * (y.e + y.s * ay)};
}

__device__ __forceinline__ void add(Sums& t, float z, float c) {
  t = join(t, Sums{z, z == -INFINITY ? 0.0f : 1.0f + (z - z), 0.0f}, c);      // z - z: NaN for a NaN or an infinity
}

__device__ __forceinline__ Sums wave_join(Sums t, float c) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Sums o{__shfl_xor(t.m, d), __shfl_xor(t.s, d), __shfl_xor(t.e, d)};
    t = join(t, o, c);
  }
  return t;
}

// The same value in all threads of the workgroup; lds: 3 * kWaves floats.
__device__ __forceinline__ Sums block_join(Sums t, float c, float* lds) {
  t = wave_join(t, c);
  const uint32_t wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63u) == 0u) {
    lds[3u * wave] = t.m;
    lds[3u * wave + 1u] = t.s;
    lds[3u * wave + 2u] = t.e;
  }
  __syncthreads();
  Sums r{lds[0], lds[1], lds[2]};
  for (uint32_t w = 1; w < kWaves; ++w) r = join(r, Sums{lds[3u * w], lds[3u * w + 1u], lds[3u * w + 2u]}, c);
  if (r.s != r.s) r.m = r.s;       // a NaN or +inf: everything that is made of the row is NaN (fmaxf passes NaN over)
  return r;
}

__device__ __forceinline__ bool is_token(int32_t t, uint32_t vocab) { return static_cast<uint32_t>(t) < vocab; }

// Larger for a larger logit, the same for +0 and -0, largest for a NaN.
__device__ __forceinline__ uint32_t order_of(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  if (z != z) return 0xFFFFFFFFu;
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ uint64_t block_max(uint64_t v, uint64_t* lds) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t o = __shfl_xor(v, d);
    v = o > v ? o : v;
  }
  __syncthreads();
  if ((threadIdx.x & 63u) == 0u) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  uint64_t r = lds[0];
  for (uint32_t w = 1; w < kWaves; ++w) r = lds[w] > r ? lds[w] : r;
  return r;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) score_kernel(ScoreArgs A) {
  __shared__ float lds[3 * kWaves];
  __shared__ uint64_t lds_key[kWaves];
  const uint32_t r = blockIdx.x;
  const T* z = static_cast<const T*>(A.logits) + static_cast<int64_t>(r) * A.row_stride;
  const int32_t target = A.targets ? A.targets[r] : 0;
  if (!is_token(target, A.vocab)) {
    if (threadIdx.x == 0u) {
      if (A.logprob) A.logprob[r] = 0.0f;
      if (A.entropy) A.entropy[r] = 0.0f;
      if (A.stats) A.stats[2ull * r] = A.stats[2ull * r + 1u] = 0.0f;
    }
    for (uint32_t i = threadIdx.x; i < A.top; i += kThreads) {
      A.top_idx[static_cast<uint64_t>(r) * A.top + i] = -1;
      A.top_logprob[static_cast<uint64_t>(r) * A.top + i] = -INFINITY;
    }
    return;
  }
  Sums t{-INFINITY, 0.0f, 0.0f};
  for (uint64_t i = threadIdx.x; i < A.vocab; i += kThreads) add(t, static_cast<float>(z[i]), A.scale);
  t = block_join(t, A.scale, lds);
  const float log2s = log2_of(t.s);
  if (threadIdx.x == 0u) {
    if (A.logprob) A.logprob[r] = log_probability(static_cast<float>(z[target]), t.m, A.inv_t, kLn2 * log2s);
    if (A.entropy) A.entropy[r] = t.s == 0.0f ? 0.0f : kLn2 * (log2s - t.e / t.s);
    if (A.stats) {
      A.stats[2ull * r] = t.m;
      A.stats[2ull * r + 1u] = kLn2 * log2s;
    }
  }
  uint64_t last = ~0ull;
  for (uint32_t i = 0; i < A.top; ++i) {
    uint64_t best = 0;
    for (uint64_t j = threadIdx.x; j < A.vocab; j += kThreads) {
      const uint64_t key = (static_cast<uint64_t>(order_of(static_cast<float>(z[j]))) << 32) | (0xFFFFFFFFu - static_cast<uint32_t>(j));
      if (key < last && key > best) best = key;
    }
    last = block_max(best, lds_key);
    if (threadIdx.x == 0u) {
      const uint32_t j = 0xFFFFFFFFu - static_cast<uint32_t>(last);
      A.top_idx[static_cast<uint64_t>(r) * A.top + i] = static_cast<int32_t>(j);
      A.top_logprob[static_cast<uint64_t>(r) * A.top + i] =
          log_probability(static_cast<float>(z[j]), t.m, A.inv_t, kLn2 * log2s);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) score_grad_kernel(ScoreGradArgs A) {
  const uint32_t r = blockIdx.x;
  const T* z = static_cast<const T*>(A.logits) + static_cast<int64_t>(r) * A.row_stride;
  T* dz = static_cast<T*>(A.grad_logits) + static_cast<int64_t>(r) * A.grad_row_stride;
  const int32_t target = A.targets ? A.targets[r] : 0;
  const float m = A.stats[2ull * r], log2s = A.stats[2ull * r + 1u] * (1.0f / kLn2);
  const bool nothing = !is_token(target, A.vocab) || m == -INFINITY;
  const float g = A.grad_logprob ? A.grad_logprob[r] * A.inv_t : 0.0f;
  const float h = A.grad_entropy ? A.grad_entropy[r] * A.inv_t : 0.0f;
  const float entropy = A.grad_entropy ? A.entropy[r] : 0.0f;
  for (uint64_t j = threadIdx.x; j < A.vocab; j += kThreads) {
    if (nothing) {
      dz[j] = static_cast<T>(0.0f);
      continue;
    }
    const float a = (static_cast<float>(z[j]) - m) * A.scale - log2s;
    const float p = exp2_of(a);
    const float one = A.targets && j == static_cast<uint64_t>(target) ? g : 0.0f;
    dz[j] = static_cast<T>(one - p * (g + h * (kLn2 * finite_or_zero_weight(a) + entropy)));
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) distill_kernel(DistillArgs A) {
  __shared__ float lds[3 * kWaves];
  __shared__ float q[kTopMost], q_log[kTopMost], z_at[kTopMost + 1];
  __shared__ int32_t at[kTopMost + 1];
  const uint32_t r = blockIdx.x;
  const T* z = static_cast<const T*>(A.logits) + static_cast<int64_t>(r) * A.row_stride;
  T* dz = static_cast<T*>(A.grad_logits) + static_cast<int64_t>(r) * A.grad_row_stride;
  const int32_t target = A.targets ? A.targets[r] : -1;
  const bool labelled = A.label_weight > 0.0f && is_token(target, A.vocab);
  // the teacher's softmax, by the first wave (two entries a lane)
  if (threadIdx.x < 64u) {
    float t[2], largest = -INFINITY;
    for (uint32_t u = 0; u < 2u; ++u) {
      const uint32_t i = threadIdx.x + 64u * u;
      int32_t index = -1;
      t[u] = -INFINITY;
      if (i < A.k && A.soft_weight > 0.0f) {
        index = A.teacher_idx[static_cast<uint64_t>(r) * A.k + i];
        if (!is_token(index, A.vocab)) index = -1;
        if (index >= 0) t[u] = A.teacher_logits[static_cast<uint64_t>(r) * A.k + i];
      }
      at[i] = index;
      largest = fmaxf(largest, t[u]);
    }
    for (int d = 1; d < 64; d <<= 1) largest = fmaxf(largest, __shfl_xor(largest, d));
    float w[2], sum = 0.0f;
    for (uint32_t u = 0; u < 2u; ++u) {
      w[u] = t[u] != t[u] ? t[u] : exp2_of(exponent(t[u], largest, A.scale));
      sum += w[u];
    }
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    for (uint32_t u = 0; u < 2u; ++u) {
      const uint32_t i = threadIdx.x + 64u * u;
      q[i] = sum == 0.0f ? 0.0f : w[u] / sum;
      q_log[i] = log_probability(t[u], largest, A.inv_t, kLn2 * log2_of(sum));
      z_at[i] = at[i] >= 0 ? static_cast<float>(z[at[i]]) : 0.0f;
    }
    if (threadIdx.x == 0u) {
      at[kTopMost] = labelled ? target : -1;
      z_at[kTopMost] = labelled ? static_cast<float>(z[target]) : 0.0f;
      lds[0] = sum;
    }
  }
  __syncthreads();
  const bool softened = A.soft_weight > 0.0f && !(lds[0] == 0.0f);
  if (!softened && !labelled) {
    if (threadIdx.x == 0u && A.loss) A.loss[r] = 0.0f;
    if (A.grad_logits)
      for (uint64_t j = threadIdx.x; j < A.vocab; j += kThreads) dz[j] = static_cast<T>(0.0f);
    return;
  }
  const float c1 = A.scale * A.temperature;                      // the label's softmax has T = 1
  Sums t{-INFINITY, 0.0f, 0.0f}, t1{-INFINITY, 0.0f, 0.0f};
  for (uint64_t i = threadIdx.x; i < A.vocab; i += kThreads) {
    add(t, static_cast<float>(z[i]), A.scale);
    add(t1, static_cast<float>(z[i]), c1);
  }
  t = block_join(t, A.scale, lds);
  t1 = block_join(t1, c1, lds);
  const float m = t.m, log2s = m == -INFINITY ? 0.0f : log2_of(t.s), log2s1 = m == -INFINITY ? 0.0f : log2_of(t1.s);
  const float T1 = A.temperature;
  if (threadIdx.x < 64u && A.loss) {
    float part = 0.0f;
    if (softened)
      for (uint32_t i = threadIdx.x; i < A.k; i += 64u)
        if (!(q[i] == 0.0f)) part += q[i] * (q_log[i] - log_probability(z_at[i], m, A.inv_t, kLn2 * log2s));
    for (int d = 1; d < 64; d <<= 1) part += __shfl_xor(part, d);
    if (threadIdx.x == 0u) {
      float loss = softened ? A.soft_weight * T1 * T1 * part : 0.0f;
      if (labelled) loss -= A.label_weight * log_probability(z_at[kTopMost], m, 1.0f, kLn2 * log2s1);
      A.loss[r] = loss;
    }
  }
  if (!A.grad_logits) return;
  const float g = A.grad_loss ? A.grad_loss[r] : 1.0f;
  const float gs = softened ? A.soft_weight * T1 : 0.0f, gl = labelled ? A.label_weight : 0.0f;
  auto smooth = [&](float v) {
    float d = 0.0f;
    if (softened) d += gs * exp2_of(exponent(v, m, A.scale) - log2s);
    if (labelled) d += gl * exp2_of(exponent(v, m, c1) - log2s1);
    return d;
  };
  for (uint64_t j = threadIdx.x; j < A.vocab; j += kThreads) dz[j] = static_cast<T>(g * smooth(static_cast<float>(z[j])));
  __syncthreads();
  // the teacher's entries and the label, over what was stored for them
  for (uint32_t i = threadIdx.x; i <= kTopMost; i += kThreads) {
    if (at[i] < 0) continue;
    float off = labelled && at[i] == target ? gl : 0.0f;
    if (softened)
      for (uint32_t j = 0; j < A.k; ++j)
        if (at[j] == at[i]) off += gs * q[j];
    dz[at[i]] = static_cast<T>(g * (smooth(z_at[i]) - off));
  }
}

}  // namespace

#define RGC_BY_TYPE(dtype, launch)                      \
  do {                                                  \
    if ((dtype) == 0) { using T = float; launch; }      \
    else if ((dtype) == 1) { using T = __bf16; launch; } \
    else { using T = _Float16; launch; }                \
  } while (0)

hipError_t launch_token_logprobs(const ScoreArgs& a, int dtype, hipStream_t s) {
  RGC_BY_TYPE(dtype, (score_kernel<T><<<dim3(a.rows), dim3(kThreads), 0, s>>>(a)));
  return hipGetLastError();
}

hipError_t launch_token_logprobs_backward(const ScoreGradArgs& a, int dtype, hipStream_t s) {
  RGC_BY_TYPE(dtype, (score_grad_kernel<T><<<dim3(a.rows), dim3(kThreads), 0, s>>>(a)));
  return hipGetLastError();
}

hipError_t launch_distill(const DistillArgs& a, int dtype, hipStream_t s) {
  RGC_BY_TYPE(dtype, (distill_kernel<T><<<dim3(a.rows), dim3(kThreads), 0, s>>>(a)));
  return hipGetLastError();
}

}  // namespace rgc
