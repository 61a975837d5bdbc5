// rgc_convolution.hip -- the short causal convolution along a sequence's steps, forward and backward (include/rgc.h has the formulas).
//
// Every channel is by itself.  A wave takes neighbouring channels, kVec a lane, and walks along some steps of a sequence with the last taps - 1 inputs in registers;
// those before its first step it reads again (the caches have them).  Where a text begins the inputs in registers become zeros: nothing of what was before them is ever
// used again, so that no tap has to know how far its text reaches back.
//
// Backward the same walk recomputes s, has ds = dy silu'(s), and adds w ds to the gradients of the last `taps` inputs, of which the oldest then is whole.  For the steps
// it calls its own, a wave also walks the taps - 1 behind them, whose ds its inputs have a part in.  ds u and ds are added up over a wave's steps, its workgroup's
// waves, and by a second launch over the workgroups, in an order made of the sizes alone.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "rgc_lm.h"
#include "rgc_sequence.h"

namespace rgc {
namespace {

constexpr uint32_t kWaves = 4;         // of a workgroup
constexpr uint32_t kOwn = 64;          // steps of a wave's walk backward
constexpr uint32_t kMostParts = 2048;  // workgroups of the backward pass, beyond which one takes several walks

template <typename T>
__device__ __forceinline__ const T* row_of(const SequenceView& v, uint32_t b, uint32_t t) {
  return static_cast<const T*>(v.data) + (b * v.batch_stride + t * v.step_stride);
}

template <int kTaps, int kVec>
struct Weights {
  float w[kTaps][kVec], bias[kVec];
  __device__ Weights(const ConvArgs& A, uint32_t c) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
#pragma unroll
      for (int j = 0; j < kTaps; ++j) w[j][i] = A.weight[static_cast<uint64_t>(c + i) * kTaps + j];
      bias[i] = A.bias ? A.bias[c + i] : 0.0f;
    }
  }
};

// Bit i: a text begins at step first + i (of those that the row has).
__device__ __forceinline__ uint64_t starts_from(const uint8_t* resets, uint32_t steps, uint32_t b, int64_t first, uint32_t n) {
  if (!resets) return 0u;
  const int64_t t = first + (threadIdx.x & 63u);
  return __ballot(t >= 0 && t < static_cast<int64_t>(n) && resets[static_cast<uint64_t>(b) * steps + static_cast<uint64_t>(t)] != 0);
}

// The inputs before step `first`, oldest first: the sequence's, or before its beginning the kept ones; zeros before the text's beginning.
template <typename T, int kTaps, int kVec>
__device__ __forceinline__ void inputs_before(const ConvArgs& A, uint32_t b, uint32_t first, uint32_t c, uint64_t starts, float (&u)[kTaps][kVec]) {
#pragma unroll
  for (int j = 0; j < kTaps - 1; ++j) {
    const int64_t t = static_cast<int64_t>(first) - (kTaps - 1) + j;
    Raw<T, kVec> r = {};
    if (t >= 0) r = read_at<T, kVec>(row_of<T>(A.x, b, static_cast<uint32_t>(t)) + c);
    else if (A.before) r = read_at<T, kVec>(static_cast<const T*>(A.before) + (static_cast<uint64_t>(b) * (kTaps - 1) + static_cast<uint32_t>(t + kTaps - 1)) * A.width + c);
    const bool anew = ((starts >> j) & 1u) != 0u;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
#pragma unroll
      for (int k = 0; k < j; ++k) u[k][i] = anew ? 0.0f : u[k][i];
      u[j][i] = static_cast<float>(r.v[i]);
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------------------------- forward

// us, where the caches are warm (the same call again and again; with others in between 4 x 16 takes 53 and 62: 3.7 and 4.3 TB/s), 1 x 32768 x 1500 and 8 x 4096 x 2048 bf16, four taps, by channels a lane and steps: 4 x 16 43 and 62, 4 x 8 44 and 64, 2 x 16 48 and 68, 2 x 32 54 and 79, 8 x 8 62 and 81 (registers, two
// waves a SIMD): 4.6 and 4.3 TB/s.  fp32, two channels a lane: 85 and 105, 4.6 and 5.1 TB/s with others in between.
template <typename T, int kTaps, int kVec, int kSteps>
__global__ void __launch_bounds__(64 * kWaves) convolution_kernel(ConvArgs A, uint32_t across, uint32_t tiles, uint64_t begin, uint64_t waves) {
  const uint64_t at = (begin + blockIdx.x) * kWaves + uniform(threadIdx.x >> 6);
  if (at >= waves) return;
  const uint32_t block = uniform(static_cast<uint32_t>(at % across)), tile = uniform(static_cast<uint32_t>(at / across % tiles)), b = uniform(static_cast<uint32_t>(at / across / tiles));
  const Channels<kVec> lane(block, A.width);
  const uint32_t first = tile * kSteps, n = steps_of(A.lengths, b, A.steps), valid = n > first ? min(n - first, static_cast<uint32_t>(kSteps)) : 0u;
  const uint32_t behind = A.steps > first ? min(A.steps - first, static_cast<uint32_t>(kSteps)) : 0u;
  const bool ends = tile == (max(n, 1u) - 1u) / kSteps;                               // the row's last step is one of these (a row without steps ends in the first tile)
  float u[kTaps][kVec] = {};                                                          // the inputs that enter a step, oldest first
  Raw<T, kVec> x[kSteps];
  if (valid > 0u || ends) {
    if (valid > 0u) {
      const T* p = row_of<T>(A.x, b, first) + lane.c;
#pragma unroll
      for (uint32_t r = 0; r < kSteps; ++r) {                                         // (steps behind the row's end: its last one, again)
        x[r] = read_at<T, kVec>(p);
        if (r + 1u < valid) p += A.x.step_stride;
      }
    }
    const uint64_t starts = starts_from(A.resets, A.steps, b, static_cast<int64_t>(first) - (kTaps - 1), n);
    const Weights<kTaps, kVec> W(A, lane.c);
    inputs_before<T, kTaps, kVec>(A, b, first, lane.c, starts, u);
    T* to = const_cast<T*>(row_of<T>(A.y, b, first));
    auto walk = [&](auto with_starts) __attribute__((always_inline)) {
#pragma unroll
      for (uint32_t r = 0; r < kSteps; ++r, to += A.y.step_stride) {
        if (r >= valid) continue;
        const bool anew = with_starts && ((starts >> (kTaps - 1 + r)) & 1u) != 0u;
        float y[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          if (anew) {
#pragma unroll
            for (int j = 0; j < kTaps - 1; ++j) u[j][i] = 0.0f;
          }
          u[kTaps - 1][i] = static_cast<float>(x[r].v[i]);
          y[i] = W.bias[i];
#pragma unroll
          for (int j = 0; j < kTaps; ++j) y[i] = __fmaf_rn(W.w[j][i], u[j][i], y[i]);
          if (A.silu) {
            float open, shut;
            gate_of(y[i], open, shut);
            y[i] *= open;
          }
#pragma unroll
          for (int j = 0; j + 1 < kTaps; ++j) u[j][i] = u[j + 1][i];                  // the next step's
        }
        write_own<T, kVec>(to, lane, y);
      }
    };
    if (starts == 0u) walk(No{}); else walk(Yes{});
    if (ends && A.last) {
#pragma unroll
      for (int j = 0; j < kTaps - 1; ++j) write_own<T, kVec>(static_cast<T*>(A.last) + (static_cast<uint64_t>(b) * (kTaps - 1) + j) * A.width, lane, u[j]);
    }
  }
  const float zero[kVec] = {};
  for (uint32_t r = valid; r < behind; ++r) write_own<T, kVec>(const_cast<T*>(row_of<T>(A.y, b, first + r)), lane, zero);
}

// ---------------------------------------------------------------------------------------------------------------------------------- backward

struct Walks {
  uint32_t across, ranges;             // stretches of channels; walks of a sequence
  uint64_t walks, parts;               // batch * ranges, and the workgroups that share them
  float* sums;                         // [parts][width * taps + width]
};

// (Four waves a SIMD: what it waits for is memory.  us, 8 x 4096 x 2048 bf16, four taps: 109; as the compiler likes it, 137 registers and three waves, 126; five waves, which spill 47, 196; the next
// batch asked for early, 175 registers, 157; walks of 32 steps 121, of 128 138; one channel a lane 164.  More taps have more weights to hold than that leaves room for.
// fp32: 179, 1 x 32768 x 1500 166; bf16 there 104.)
template <typename T, int kTaps, int kVec>
__global__ void __launch_bounds__(64 * kWaves, kTaps <= 4 ? 4 : 1) convolution_backward_kernel(ConvArgs A, ConvGradArgs G, Walks K, uint64_t begin) {
  constexpr uint32_t kBatch = 8;                                                      // steps read at once
  __shared__ float sums[kWaves][kTaps + 1][64 * kVec];
  const uint64_t at = begin + blockIdx.x;
  const uint32_t block = uniform(static_cast<uint32_t>(at % K.across)), wave = uniform(threadIdx.x >> 6), l = threadIdx.x & 63u;
  const uint64_t part = at / K.across;
  const Channels<kVec> lane(block, A.width);
  const Weights<kTaps, kVec> W(A, lane.c);
  float dw[kTaps + 1][kVec] = {};                                                     // the last: the bias's
  for (uint64_t walk = part * kWaves + wave; walk < K.walks; walk += K.parts * kWaves) {
    const uint32_t b = uniform(static_cast<uint32_t>(walk / K.ranges)), first = uniform(static_cast<uint32_t>(walk % K.ranges)) * kOwn;
    const uint32_t n = steps_of(A.lengths, b, A.steps), end = min(first + kOwn, A.steps);   // its own steps
    const uint32_t upto = end + kTaps - 1;                                            // and those behind them (there or not)
    float u[kTaps][kVec] = {}, du[kTaps][kVec] = {};                                  // inputs of a step, oldest first, and their gradients so far
    uint32_t reach = kTaps - 1;                                                       // how many inputs back the step's text goes
    if (n > first) {
      const uint64_t starts = starts_from(A.resets, A.steps, b, static_cast<int64_t>(first) - (kTaps - 1), n) & ((1ull << (kTaps - 1)) - 1ull);
      inputs_before<T, kTaps, kVec>(A, b, first, lane.c, starts, u);
      if (starts != 0u) reach = kTaps - 1 - (63u - static_cast<uint32_t>(__clzll(starts)));
    } else if (n == 0u && first == 0u && G.dlast) {                                   // (a row without steps hands the kept inputs on)
#pragma unroll
      for (int j = 0; j < kTaps - 1; ++j) {
        const Raw<T, kVec> r = read_at<T, kVec>(static_cast<const T*>(G.dlast) + (static_cast<uint64_t>(b) * (kTaps - 1) + j) * A.width + lane.c);
#pragma unroll
        for (int i = 0; i < kVec; ++i) du[j][i] = static_cast<float>(r.v[i]);
      }
    }
    for (uint32_t t0 = first; t0 < upto; t0 += kBatch) {
      Raw<T, kVec> x[kBatch], dy[kBatch];
      if (t0 < n) {
        const T *px = row_of<T>(A.x, b, t0) + lane.c, *pd = row_of<T>(G.dy, b, t0) + lane.c;
#pragma unroll
        for (uint32_t r = 0; r < kBatch; ++r) {
          x[r] = read_at<T, kVec>(px);
          dy[r] = read_at<T, kVec>(pd);
          if (t0 + r + 1u < n) px += A.x.step_stride, pd += G.dy.step_stride;
        }
      }
      const uint64_t starts = starts_from(A.resets, A.steps, b, t0, n) & ((1ull << kBatch) - 1ull);
      // kPlain: all of the batch's steps are there and the wave's own, no text begins, none is the row's last
      auto go = [&](auto plain) __attribute__((always_inline)) {
        constexpr bool kPlain = decltype(plain){};
#pragma unroll
        for (uint32_t r = 0; r < kBatch; ++r) {
          const uint32_t t = t0 + r;
          if (!kPlain && t >= upto) continue;
          if (!kPlain && ((starts >> r) & 1u) != 0u) {
            reach = 0u;
#pragma unroll
            for (int j = 0; j < kTaps - 1; ++j) {
#pragma unroll
              for (int i = 0; i < kVec; ++i) u[j][i] = 0.0f;
            }
          }
          if (kPlain || t < n) {
            const bool own = kPlain || t < end;
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
              u[kTaps - 1][i] = static_cast<float>(x[r].v[i]);
              float ds = static_cast<float>(dy[r].v[i]);
              if (A.silu) {
                float s = W.bias[i], open, shut;
#pragma unroll
                for (int j = 0; j < kTaps; ++j) s = __fmaf_rn(W.w[j][i], u[j][i], s);
                gate_of(s, open, shut);
                ds *= open * __fmaf_rn(s, shut, 1.0f);
              }
#pragma unroll
              for (int j = 0; j < kTaps; ++j) {
                if (kPlain || kTaps - 1u - j <= reach) du[j][i] = __fmaf_rn(W.w[j][i], ds, du[j][i]);
                if (own) dw[j][i] = __fmaf_rn(ds, u[j][i], dw[j][i]);
              }
              if (own) dw[kTaps][i] += ds;
            }
            if (!kPlain && t + 1u == n && G.dlast) {
#pragma unroll
              for (int j = 1; j < kTaps; ++j) {
                if (kTaps - 1u - j > reach) continue;
                const Raw<T, kVec> d = read_at<T, kVec>(static_cast<const T*>(G.dlast) + (static_cast<uint64_t>(b) * (kTaps - 1) + j - 1) * A.width + lane.c);
#pragma unroll
                for (int i = 0; i < kVec; ++i) du[j][i] += static_cast<float>(d.v[i]);
              }
            }
          }
          // the oldest input's gradient is whole
          const int64_t oldest = static_cast<int64_t>(t) - (kTaps - 1);
          if (kPlain ? oldest >= static_cast<int64_t>(first) : oldest >= static_cast<int64_t>(first) && oldest < static_cast<int64_t>(end))
            write_own<T, kVec>(const_cast<T*>(row_of<T>(G.dx, b, static_cast<uint32_t>(oldest))), lane, du[0]);
          else if (oldest < 0 && G.dbefore)
            write_own<T, kVec>(static_cast<T*>(G.dbefore) + (static_cast<uint64_t>(b) * (kTaps - 1) + t) * A.width, lane, du[0]);
          if (!kPlain && reach < kTaps - 1) ++reach;
#pragma unroll
          for (int j = 0; j + 1 < kTaps; ++j) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) u[j][i] = u[j + 1][i], du[j][i] = du[j + 1][i];
          }
#pragma unroll
          for (int i = 0; i < kVec; ++i) du[kTaps - 1][i] = 0.0f;
        }
      };
      if (starts == 0u && reach == kTaps - 1 && t0 + kBatch <= end && t0 + kBatch < n) go(Yes{}); else go(No{});
    }
  }
#pragma unroll
  for (int j = 0; j <= kTaps; ++j) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) sums[wave][j][i * 64 + l] = dw[j][i];
  }
  __syncthreads();
  // the lanes of the first wave know which channels they are
  if (wave > 0u || !lane.mine) return;
  float* to = K.sums + part * (static_cast<uint64_t>(A.width) * (kTaps + 1));
#pragma unroll
  for (int j = 0; j <= kTaps; ++j) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      float sum = dw[j][i];
      for (uint32_t w = 1; w < kWaves; ++w) sum += sums[w][j][i * 64 + l];
      if (lane.c + i < lane.own) continue;
      if (j < kTaps) to[static_cast<uint64_t>(lane.c + i) * kTaps + j] = sum;
      else to[static_cast<uint64_t>(A.width) * kTaps + lane.c + i] = sum;
    }
  }
}

uint32_t stretches(uint32_t width, uint32_t vec) { return (width + 64u * vec - 1u) / (64u * vec); }

uint32_t lane_channels(uint32_t width, int dtype, bool backward) { return width < 4u ? 1u : dtype == 0 || backward ? 2u : 4u; }

Walks walks_of(const ConvArgs& a, int dtype) {
  Walks K{};
  K.across = stretches(a.width, lane_channels(a.width, dtype, true));
  K.ranges = a.steps == 0u ? 1u : (a.steps + kOwn - 1u) / kOwn;
  K.walks = static_cast<uint64_t>(a.batch) * K.ranges;
  const uint64_t most = kMostParts / K.across + 1u, all = (K.walks + kWaves - 1u) / kWaves;
  K.parts = all < most ? all : most;
  return K;
}

// Calls f with the type, the taps and the channels a lane as constants.
template <bool kBackward, typename F>
hipError_t chosen(uint32_t taps, int dtype, uint32_t vec, F&& f) {
  auto by_vec = [&](auto type, auto k) {
    constexpr int kMost = sizeof(type) == 4 || kBackward ? 2 : 4;
    return vec == 1u ? f(type, k, std::integral_constant<int, 1>{}) : f(type, k, std::integral_constant<int, kMost>{});
  };
  auto by_type = [&](auto k) {
    if (dtype == 0) return by_vec(float{}, k);
    if (dtype == 1) return by_vec(__bf16{}, k);
    return by_vec(_Float16{}, k);
  };
  switch (taps) {
    case 1: return by_type(std::integral_constant<int, 1>{});
    case 2: return by_type(std::integral_constant<int, 2>{});
    case 3: return by_type(std::integral_constant<int, 3>{});
    case 4: return by_type(std::integral_constant<int, 4>{});
    case 5: return by_type(std::integral_constant<int, 5>{});
    case 6: return by_type(std::integral_constant<int, 6>{});
    case 7: return by_type(std::integral_constant<int, 7>{});
    default: return by_type(std::integral_constant<int, 8>{});
  }
}

}  // namespace

hipError_t launch_convolution(const ConvArgs& a, uint32_t taps, int dtype, hipStream_t s) {
  return chosen<false>(taps, dtype, lane_channels(a.width, dtype, false), [&](auto type, auto k, auto vec) {
    using T = decltype(type);
    constexpr int kTaps = decltype(k)::value, kVec = decltype(vec)::value;
    auto go = [&](auto steps) {
      constexpr int kSteps = decltype(steps)::value;
      const uint32_t across = stretches(a.width, kVec), tiles = a.steps == 0u ? 1u : (a.steps + kSteps - 1u) / kSteps;
      const uint64_t waves = static_cast<uint64_t>(a.batch) * tiles * across;
      in_grids((waves + kWaves - 1u) / kWaves, [&](uint64_t begin, dim3 grid) {
        convolution_kernel<T, kTaps, kVec, kSteps><<<grid, dim3(64 * kWaves), 0, s>>>(a, across, tiles, begin, waves);
      });
      return hipGetLastError();
    };
    return a.steps <= 1u ? go(std::integral_constant<int, 1>{}) : go(std::integral_constant<int, 16>{});
  });
}

uint64_t convolution_scratch_words(const ConvArgs& a, uint32_t taps, int dtype) {
  return (walks_of(a, dtype).parts * a.width * (taps + 1u) + 1u) / 2u;
}

hipError_t launch_convolution_backward(const ConvArgs& a, const ConvGradArgs& g, uint32_t taps, int dtype, unsigned long long* scratch, hipStream_t s) {
  Walks K = walks_of(a, dtype);
  K.sums = reinterpret_cast<float*>(scratch);
  const hipError_t e = chosen<true>(taps, dtype, lane_channels(a.width, dtype, true), [&](auto type, auto k, auto vec) {
    in_grids(K.parts * K.across, [&](uint64_t begin, dim3 grid) {
      convolution_backward_kernel<decltype(type), decltype(k)::value, decltype(vec)::value><<<grid, dim3(64 * kWaves), 0, s>>>(a, g, K, begin);
    });
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  const uint64_t weights = static_cast<uint64_t>(a.width) * taps;
  return launch_sum_parts(PartsArgs{K.sums, K.parts, weights + a.width, {g.dweight, g.dbias, nullptr}, {weights, weights + a.width, weights + a.width}}, s);
}

}  // namespace rgc
