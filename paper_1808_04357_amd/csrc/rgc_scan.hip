// rgc_scan.hip -- the selective scan, forward (include/rgc.h has the formulas; rgc_scan.h how a wave is laid out).
//
// A step of a state is two products, a power and two fused steps; the tensors are read and written once.  It is bound by that arithmetic.  Each wave walks along its steps with its
// channels' states in registers.  Where sequences and channels alone are too few waves, a sequence is cut into stretches of whole chunks: one launch takes every stretch from
// a state of zero to the state H that it ends with and adds up its steps' sizes, the next one makes the states that stretches begin with of those, h -> exp(rate sum) h + H, and the last one is
// the walk from there.  What a state was before it starts anew is not used: not even multiplied by 0.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "rgc_scan.h"

namespace rgc {
namespace {

constexpr uint32_t kWaves = 4;         // of a workgroup
constexpr uint32_t kTile = 8;          // steps of a wave at a time

// kSummary: what a stretch does to a state, instead of its results.
// What memory gives is asked for early: x, delta and the gate of kTiles tiles while those before are walked, B and C of a chunk during the chunk before.
template <typename T, int kS, int kQ, bool kSummary>
__global__ void __launch_bounds__(64 * kWaves) scan_kernel(ScanArgs A, ScanCut K, uint64_t begin) {
  typedef Spot<kS, kQ, kTile> At;
  constexpr uint32_t kOwn = At::kOwn, kStates = At::kStates, kChannels = At::kChannels;
  constexpr uint32_t kTiles = kOwn == 1 ? 4 : kOwn == 2 ? 2 : 1, kSteps = kTiles * kTile, kApart = kTiles > 1 ? kSteps + 4 : kSteps;   // (apart: lanes of neighbouring channels in other banks)
  __shared__ __attribute__((aligned(16))) float rows_b[2][kChunk * kStates], rows_c[2][kSummary ? 4 : kChunk * kStates];
  __shared__ __attribute__((aligned(16))) float sizes[kWaves][kChannels * kApart], feeds[kWaves][kChannels * kApart];
  uint64_t rest = begin + blockIdx.x;
  const uint32_t wave = uniform(threadIdx.x >> 6);
  const uint32_t across = kSummary ? K.across_summary : K.across;
  const uint32_t block = uniform(static_cast<uint32_t>(rest % across)) * kWaves + wave;
  rest /= across;
  const uint32_t g = uniform(static_cast<uint32_t>(rest % A.groups));
  rest /= A.groups;
  const uint32_t walked = kSummary ? K.stretches - 1u : K.stretches;                  // (what the last stretch ends with, the walk itself knows)
  const uint32_t stretch = uniform(static_cast<uint32_t>(rest % walked)), b = uniform(static_cast<uint32_t>(rest / walked));
  const At at(A, g, block);
  const uint32_t n = steps_of(A.lengths, b, A.steps);
  const uint64_t states_of_row = static_cast<uint64_t>(A.width) * A.states;
  const uint32_t first_chunk = stretch * K.stretch, last_chunk = min(first_chunk + K.stretch, K.chunks);
  const bool gate = !kSummary && A.gate.data != nullptr;
  float rate[kS], h[kS] = {};
  Staged<T, kStates, 64 * kWaves> next_b, next_c;
  auto ask_rows = [&](uint32_t chunk) {
    const uint32_t count = steps_in(chunk * kChunk, kChunk, n);
    next_b.ask(A.b, A, b, g, chunk * kChunk, count);
    if constexpr (!kSummary) next_c.ask(A.c, A, b, g, chunk * kChunk, count);
  };
  auto put_rows = [&](uint32_t chunk) {
    next_b.put(rows_b[chunk & 1u]);
    if constexpr (!kSummary) next_c.put(rows_c[chunk & 1u]);
  };
  T x[kTiles][kOwn], v[kTiles][kOwn], z[kTiles][kOwn];
  Column<T> from_x(A.x, b, first_chunk * kChunk, at.own, at.c), from_v(A.delta, b, first_chunk * kChunk, at.own, at.c), from_z(gate ? A.gate : A.x, b, first_chunk * kChunk, at.own, at.c);
  auto ask = [&](uint32_t t0) {                                                       // the next steps; those behind the row's end are not looked at
    auto each = [&](auto whole) __attribute__((always_inline)) {
#pragma unroll
      for (uint32_t m = 0; m < kTiles; ++m) {
#pragma unroll
        for (uint32_t j = 0; j < kOwn; ++j) {
          x[m][j] = v[m][j] = z[m][j] = static_cast<T>(0.0f);
          if (decltype(whole){} || t0 + m * kTile + at.own + j < n) {
            x[m][j] = from_x.at(m * kTile + j);
            v[m][j] = from_v.at(m * kTile + j);
            if (gate) z[m][j] = from_z.at(m * kTile + j);
          }
        }
      }
    };
    if (t0 + kSteps <= n) each(Yes{}); else each(No{});
    from_x.row += kSteps * from_x.step, from_v.row += kSteps * from_v.step, from_z.row += kSteps * from_z.step;
  };
  const uint32_t first_step = first_chunk * kChunk, end = min(n, last_chunk * kChunk);      // of the stretch's walk
  if (first_step < end) {
    ask_rows(first_chunk);
    ask(first_step);
  }
  rates_of(A, at, rate);
  const float through = !kSummary && A.d ? A.d[at.c] : 0.0f, bias = A.delta_bias ? A.delta_bias[at.c] : 0.0f;
  if constexpr (!kSummary) {
    if (K.stretches > 1u) read_states(K.starts + (static_cast<uint64_t>(b) * K.stretches + stretch) * states_of_row, A, at, h);
    else if (A.h0) read_states(A.h0 + b * states_of_row, A, at, h);
  }
  if (first_step < end) {
    put_rows(first_chunk);
    __syncthreads();
  }
  float total = 0.0f;                  // of the owner's steps' sizes
  uint64_t cut = 0u;
  Column<T> to_y(kSummary ? A.x : A.y, b, first_step, at.own, at.c);
  for (uint32_t chunk = first_chunk; chunk < last_chunk; ++chunk) {
    const uint32_t first = chunk * kChunk, count = steps_in(first, kChunk, n);
    if (!kSummary && A.kept) write_states(A.kept + (static_cast<uint64_t>(b) * K.chunks + chunk) * states_of_row, A, at, h);
    const bool more = chunk + 1u < last_chunk && first + kChunk < n;
    if (more) ask_rows(chunk + 1u);
    const uint64_t anew = anew_from(A, b, first, kChunk, n);
    cut |= anew;
    const float *const in_b = rows_b[chunk & 1u] + at.q * kS, *const in_c = rows_c[chunk & 1u] + (kSummary ? 0u : at.q * kS);
    for (uint32_t part = 0; part < count; part += kSteps) {
      const uint32_t t0 = first + part;
      float input[kTiles][kOwn], shown[kTiles][kOwn];
#pragma unroll
      for (uint32_t m = 0; m < kTiles; ++m) {
#pragma unroll
        for (uint32_t j = 0; j < kOwn; ++j) {
          float grow, size = size_of(A, static_cast<float>(v[m][j]), bias, grow);
          if (t0 + m * kTile + at.own + j >= n) size = 0.0f;                         // (what is not there was read as 0)
          input[m][j] = static_cast<float>(x[m][j]);
          sizes[wave][at.channel * kApart + m * kTile + at.own + j] = size;
          feeds[wave][at.channel * kApart + m * kTile + at.own + j] = size * input[m][j];
          if constexpr (kSummary) {
            total += size;
          } else {
            shown[m][j] = 1.0f;
            if (gate) {
              const float zj = static_cast<float>(z[m][j]);
              float open, shut;
              gate_of(zj, open, shut);
              shown[m][j] = zj * open;
            }
          }
        }
      }
      if (t0 + kSteps < end) ask(t0 + kSteps);
      wave_sync();
      const uint32_t all_starts = static_cast<uint32_t>(anew >> part), left = count - part;
      // (a step that is not there has the size 0 and brings nothing: it leaves the states as they are)
      auto walk = [&](uint32_t m, auto with_starts) __attribute__((always_inline)) {
        const uint32_t tile = part + m * kTile;
        float size[kTile], fed[kTile], y[kTile] = {};
        read_tile(&sizes[wave][at.channel * kApart + m * kTile], size);
        read_tile(&feeds[wave][at.channel * kApart + m * kTile], fed);
        const uint32_t starts = all_starts >> (m * kTile);
#pragma unroll
        for (uint32_t t = 0; t < kTile; ++t) {
          float in[kS], out[kS];
          read_shared<kS>(in_b + (tile + t) * kStates, in);
          if constexpr (!kSummary) read_shared<kS>(in_c + (tile + t) * kStates, out);
#pragma unroll
          for (uint32_t s = 0; s < kS; ++s) {
            if (with_starts && ((starts >> t) & 1u) != 0u) h[s] = 0.0f;
            h[s] = __fmaf_rn(__builtin_amdgcn_exp2f(size[t] * rate[s]), h[s], fed[t] * in[s]);
            if constexpr (!kSummary) y[t] = __fmaf_rn(h[s], out[s], y[t]);
          }
        }
        if constexpr (!kSummary) {
          sum_for_owners<kQ, kTile>(y, at.lane);
#pragma unroll
          for (uint32_t j = 0; j < kOwn; ++j)
            if (at.owner && (!with_starts || m * kTile + at.own + j < left)) to_y.at(m * kTile + j) = static_cast<T>(__fmaf_rn(through, input[m][j], y[j]) * shown[m][j]);
        }
      };
      // where all steps are there and none starts anew, without a branch between the tiles: one tile's sums go on beside the next one's steps
      if (left >= kSteps && (all_starts & static_cast<uint32_t>((1ull << kSteps) - 1ull)) == 0u) {
#pragma unroll
        for (uint32_t m = 0; m < kTiles; ++m) walk(m, No{});
      } else {
#pragma unroll
        for (uint32_t m = 0; m < kTiles; ++m)
          if (m * kTile < left) walk(m, Yes{});
      }
      wave_sync();                     // (before the next tiles' sizes take their place)
      to_y.row += kSteps * to_y.step;
    }
    if constexpr (!kSummary) {
      const uint32_t behind = steps_in(first, kChunk, A.steps);
      for (uint32_t t = count + at.q; t < behind; t += kQ)
        if (at.mine) *element<T>(A.y, b, first + t, at.c) = static_cast<T>(0.0f);
    }
    if (more) {
      put_rows(chunk + 1u);
      __syncthreads();
    }
  }
  if constexpr (kSummary) {
    const uint64_t slot = static_cast<uint64_t>(b) * K.stretches + stretch;
    write_states(K.starts + slot * states_of_row, A, at, h);
    if (!at.first) total = 0.0f;
    total = sum_lanes<kQ>(total);
    if (at.mine && at.q == 0u) K.sums[slot * A.width + at.c] = total;
    if (g == 0u && block == 0u && at.lane == 0u) K.cuts[slot] = cut != 0u ? 1u : 0u;
  } else {
    if (A.h_last && stretch + 1u == K.stretches) write_states(A.h_last + b * states_of_row, A, at, h);
  }
}

// The states that stretches begin with, in the place of those that they end with from 0.
__global__ void __launch_bounds__(256) scan_join_kernel(ScanArgs A, ScanCut K, uint64_t begin) {
  constexpr uint32_t kAtOnce = 8;
  const uint64_t row = static_cast<uint64_t>(A.width) * A.states, i = (begin + blockIdx.x) * 256u + threadIdx.x;
  if (i >= row * A.batch) return;
  const uint64_t b = i / row, at = i % row, c = at / A.states;
  const float r0 = A.a[at] * kLog2e, r1 = r0 > 3.0e38f ? 3.0e38f : r0, rate = r1 < -3.0e38f ? -3.0e38f : r1;
  float h = A.h0 ? A.h0[i] : 0.0f;
  float* to = K.starts + b * K.stretches * row + at;
  const float* sums = K.sums + b * K.stretches * A.width + c;
  const uint32_t* cuts = K.cuts + b * K.stretches;
  for (uint32_t k0 = 0; k0 < K.stretches; k0 += kAtOnce) {
    float ends[kAtOnce], half[kAtOnce];
#pragma unroll
    for (uint32_t j = 0; j < kAtOnce; ++j) {
      const uint32_t k = min(k0 + j, K.stretches - 1u);                              // (the last one's slot is unset memory, and not used)
      ends[j] = to[k * row];
      half[j] = half_decay(rate, sums[static_cast<uint64_t>(k) * A.width]);
    }
#pragma unroll
    for (uint32_t j = 0; j < kAtOnce; ++j) {
      const uint32_t k = k0 + j;
      if (k >= K.stretches) continue;
      to[k * row] = h;
      if (k + 1u < K.stretches) h = cuts[k] != 0u ? ends[j] : past(half[j], h, ends[j]);
    }
  }
}

// One step: a lane for kS states of a channel, whose kQ lanes are neighbours.  Bound by the states, read and written once.
template <typename T, int kS, int kQ>
__global__ void __launch_bounds__(64 * kWaves) scan_step_kernel(ScanArgs A, uint32_t blocks, uint64_t begin, uint64_t waves) {
  constexpr uint32_t kChannels = 64 / kQ;
  const uint64_t wave = (begin + blockIdx.x) * kWaves + uniform(threadIdx.x >> 6);
  if (wave >= waves) return;
  const uint32_t b = uniform(static_cast<uint32_t>(wave / blocks)), block = uniform(static_cast<uint32_t>(wave % blocks));
  const uint32_t lane = threadIdx.x & 63u, q = lane % kQ, want = block * kChannels + lane / kQ, c = min(want, A.width - 1u), g = c / (A.width / A.groups);
  const bool mine = want < A.width, there = steps_of(A.lengths, b, 1u) > 0u;
  const uint64_t row = b * (static_cast<uint64_t>(A.width) * A.states);
  const uint32_t at = (c * A.states + q * kS) * 4u;
  float h[kS] = {}, rate[kS];
  if (A.h0) read_states<kS, kQ>(A.h0 + row, A, q, at, h);
  auto put = [&](float* to) {
    float* p = reinterpret_cast<float*>(reinterpret_cast<char*>(to + row) + at);
    if (!mine) return;
    if (kS == 4 && A.states == kS * kQ) {
      write_at<float, kS>(p, h);
    } else {
#pragma unroll
      for (uint32_t s = 0; s < kS; ++s)
        if (q * kS + s < A.states) p[s] = h[s];
    }
  };
  if (A.kept) put(A.kept);
  float y = 0.0f;
  if (there) {
    float grow, shown = 1.0f;
    const float x = static_cast<float>(*element<T>(A.x, b, 0u, c)), size = size_of(A, static_cast<float>(*element<T>(A.delta, b, 0u, c)), A.delta_bias ? A.delta_bias[c] : 0.0f, grow);
    if (A.gate.data) {
      const float z = static_cast<float>(*element<T>(A.gate, b, 0u, c));
      float open, shut;
      gate_of(z, open, shut);
      shown = z * open;
    }
    const T *in = element<T>(A.b, b, 0u, g * A.states), *out = element<T>(A.c, b, 0u, g * A.states);
    read_states<kS, kQ>(A.a, A, q, at, rate);
    finite_rates(rate);
    const bool anew = A.resets && A.resets[b] != 0;
#pragma unroll
    for (uint32_t s = 0; s < kS; ++s) {
      const uint32_t n = min(q * kS + s, A.states - 1u);
      if (anew) h[s] = 0.0f;
      h[s] = __fmaf_rn(__builtin_amdgcn_exp2f(size * rate[s]), h[s], size * x * static_cast<float>(in[n]));
      if (q * kS + s < A.states) y = __fmaf_rn(h[s], static_cast<float>(out[n]), y);
    }
    y = sum_lanes<kQ>(y);
    y = __fmaf_rn(A.d ? A.d[c] : 0.0f, x, y) * shown;
  }
  if (mine && q == 0u) *element<T>(A.y, b, 0u, c) = static_cast<T>(y);
  if (A.h_last) put(A.h_last);
}

template <typename T, int kS, int kQ>
hipError_t launch_step(const ScanArgs& a, hipStream_t s) {
  const uint32_t blocks = (a.width + 64u / kQ - 1u) / (64u / kQ);
  const uint64_t waves = static_cast<uint64_t>(a.batch) * blocks;
  in_grids((waves + kWaves - 1u) / kWaves, [&](uint64_t begin, dim3 grid) { scan_step_kernel<T, kS, kQ><<<grid, dim3(64 * kWaves), 0, s>>>(a, blocks, begin, waves); });
  return hipGetLastError();
}
template <typename T>
hipError_t launch_step(const ScanArgs& a, hipStream_t s) {
  if (a.states == 1u) return launch_step<T, 1, 1>(a, s);
  if (a.states <= 4u) return launch_step<T, 4, 1>(a, s);
  if (a.states <= 8u) return launch_step<T, 4, 2>(a, s);
  if (a.states <= 16u) return launch_step<T, 4, 4>(a, s);
  if (a.states <= 32u) return launch_step<T, 4, 8>(a, s);
  return launch_step<T, 4, 16>(a, s);
}

uint64_t workgroups(const ScanArgs& a, uint32_t stretches, uint32_t across) { return static_cast<uint64_t>(a.batch) * stretches * a.groups * across; }

}  // namespace

// Stretches where sequences and channels are fewer waves than kFew: so many that there are kEnough.
// us, 16 states, bf16, sequences of 1024 channels (128 waves), whole / cut, with kEnough 4096, 8192, 16384, 32768:
//   waves    1024 steps                     8192 steps
//     128     83 /  27  27  26  26          647 /   97   98  109  142
//     512     83 /  50  50  56  55          657 /  317  287  274  280
//     768     83 /  75  66  66  74          683 /  501  451  422  414
//    1024     83 /  84  80  81  94          686 /  626  572  548  549
//    1536    102 / 123 114 111 114          859 /  950  829  803  802
//    2048    103 / 139 133 135 144          880 / 1093 1029 1018 1032
// and 1 x 32768 x 1500 (188 waves) 2720 / 525 458 439 444.  With 4, 8, 32 and 64 states, and in fp32, cut and whole meet at 1024 waves of 1024 steps too (4 states 252 / 250 244 253 277).  Left as they
// are: a few chunks would rather be whole whatever the waves (4 x 128 x 1024 13 / 16), long sequences rather cut at 768 and 1024 waves.
ScanCut scan_cut(const ScanArgs& a) {
  constexpr uint64_t kFew = 768, kEnough = 16384;
  ScanCut K{};
  K.chunks = (a.steps + kChunk - 1u) / kChunk;
  const uint32_t channels = kWaves * wave_channels<Kind::kWalk>(a.states), summary = kWaves * wave_channels<Kind::kSummary>(a.states), each = a.width / a.groups;
  K.across = (each + channels - 1u) / channels;
  K.across_summary = (each + summary - 1u) / summary;
  const uint64_t waves = static_cast<uint64_t>(a.batch) * a.groups * ((each + channels / kWaves - 1u) / (channels / kWaves));
  K.stretches = 1u;
  K.stretch = K.chunks > 0u ? K.chunks : 1u;
  if (waves < kFew && K.chunks > 1u) {
    const uint64_t want = kEnough / waves;
    K.stretch = static_cast<uint32_t>((K.chunks + want - 1u) / want);
    K.stretches = (K.chunks + K.stretch - 1u) / K.stretch;
  }
  return K;
}

uint64_t scan_scratch_words(const ScanArgs& a) {
  const ScanCut K = scan_cut(a);
  if (K.stretches <= 1u) return 0u;
  return (static_cast<uint64_t>(a.batch) * K.stretches * (static_cast<uint64_t>(a.width) * (a.states + 1u) + 1u) + 1u) / 2u;
}

hipError_t launch_scan(const ScanArgs& a, int dtype, unsigned long long* scratch, hipStream_t s) {
  if (a.steps == 1u) return dtype == 0 ? launch_step<float>(a, s) : dtype == 1 ? launch_step<__bf16>(a, s) : launch_step<_Float16>(a, s);
  ScanCut K = scan_cut(a);
  if (K.stretches > 1u) {
    const uint64_t slots = static_cast<uint64_t>(a.batch) * K.stretches;
    K.starts = reinterpret_cast<float*>(scratch);
    K.sums = K.starts + slots * a.width * a.states;
    K.cuts = reinterpret_cast<uint32_t*>(K.sums + slots * a.width);
  }
  if (K.stretches > 1u) {
    const hipError_t e = by_states<Kind::kSummary>(a.states, dtype, [&](auto type, auto layout) {
      in_grids(workgroups(a, K.stretches - 1u, K.across_summary), [&](uint64_t begin, dim3 grid) {
        scan_kernel<decltype(type), decltype(layout)::kS, decltype(layout)::kQ, true><<<grid, dim3(64 * kWaves), 0, s>>>(a, K, begin);
      });
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    const uint64_t all = static_cast<uint64_t>(a.batch) * a.width * a.states;
    in_grids((all + 255u) / 256u, [&](uint64_t begin, dim3 grid) { scan_join_kernel<<<grid, dim3(256), 0, s>>>(a, K, begin); });
  }
  return by_states<Kind::kWalk>(a.states, dtype, [&](auto type, auto layout) {
    in_grids(workgroups(a, K.stretches, K.across), [&](uint64_t begin, dim3 grid) {
      scan_kernel<decltype(type), decltype(layout)::kS, decltype(layout)::kQ, false><<<grid, dim3(64 * kWaves), 0, s>>>(a, K, begin);
    });
    return hipGetLastError();
  });
}

}  // namespace rgc
