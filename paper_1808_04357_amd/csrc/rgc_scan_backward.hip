// rgc_scan_backward.hip -- the selective scan's gradients (include/rgc.h has the formulas; rgc_scan.h how a wave is laid out).
//
// With g the gradient that leaves a step towards the state before it and e = the step's output gradient times C, a state's gradient is d = e + g' (g' of the step behind it), and g = a d.
// So the gradients go through the steps as the states do, the other way.
//  1. Every chunk but the first from a gradient of zero behind it: what it hands on, and the sum of its steps' sizes (scan_rear_kernel).
//  2. What comes in behind each chunk, from the last one to the first (scan_rear_join_kernel).  With one chunk neither is needed.
//  3. A workgroup for each chunk and group of channels (scan_backward_kernel).  Its waves take eight steps each, of as many channels as a wave has at a time: each makes its powers,
//     what its steps do to a state and to a gradient (both from zero), hears from the others what state it begins and what gradient it ends with, and walks its steps in both directions out of
//     registers: B's and C's gradients, sums over channels, stay in registers over all of the workgroup's channels; those of A, D and delta's bias, sums over steps, are added up over the waves.
//  4. The workgroups' parts of both are added up in an order made of the sizes alone (scan_rows_kernel, launch_sum_parts).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "rgc_scan.h"

namespace rgc {
namespace {

constexpr uint32_t kRearWaves = 4;     // of a workgroup of the first launch
constexpr uint32_t kRearTile = 8;      // steps of a wave at a time in the first launch
// A sequence of a few steps more than a chunk has is taken as one, by workgroups of more waves: no launch but the third is needed for it, and no workgroups with next to nothing to do.
// us, the backward call, as one / in two chunks, 33 to 48 steps (the same to 2 us): 20 x 1500 fp32 56 / 63, with 4 states 31 / 37, 24 states 73 / 79, 32 states 95 / 111, 64 x 2048 bf16 171 / 197,
// 256 x 512 171 / 193, 2 x 4096 36 / 34.  (With layouts whose waves walk eight steps.)
constexpr uint32_t kWholeWaves = 6, kWholeTile = 8, kWholeStates = 32;

struct RearCut {
  uint32_t chunks, kept, across;       // chunks of a sequence, states kept of it, workgroups of the first launch for a group's channels
  uint32_t splits, blocks;             // workgroups of the third for them, stretches of a wave's channels
  bool whole;                          // a sequence is one chunk, and longer than others
  float* ends;                         // [batch][chunks][width][states]: what a chunk hands on from 0, then what comes in behind it
  float* sums;                         // [batch][chunks][width]
  uint32_t* cuts;                      // [batch][chunks]
  float* parts;                        // [batch][chunks][width * states + width + width]: gradients of A, D and delta's bias
  float* rows;                         // [splits][batch][steps][2][groups * states]: of B and C
};

// Gradients that reach the states of a step through its output: the output's, before the gate.
__device__ __forceinline__ float shown_of(bool gate, float z, float& slope) {
  if (!gate) {
    slope = 0.0f;
    return 1.0f;
  }
  float open, shut;
  gate_of(z, open, shut);
  slope = open * __fmaf_rn(z, shut, 1.0f);
  return z * open;
}

template <typename T, int kS, int kQ>
__global__ void __launch_bounds__(64 * kRearWaves) scan_rear_kernel(ScanArgs A, ScanGradArgs G, RearCut K, uint64_t begin) {
  typedef Spot<kS, kQ, kRearTile> At;
  constexpr uint32_t kTile = kRearTile;
  constexpr uint32_t kOwn = At::kOwn, kStates = At::kStates, kChannels = At::kChannels;
  __shared__ __attribute__((aligned(16))) float rows_c[kChunk * kStates], sizes[kRearWaves][kChannels * kTile], grads[kRearWaves][kChannels * kTile];
  uint64_t rest = begin + blockIdx.x;
  const uint32_t wave = uniform(threadIdx.x >> 6);
  const uint32_t block = uniform(static_cast<uint32_t>(rest % K.across)) * kRearWaves + wave;
  rest /= K.across;
  const uint32_t group = uniform(static_cast<uint32_t>(rest % A.groups));
  rest /= A.groups;
  const uint32_t chunk = 1u + uniform(static_cast<uint32_t>(rest % (K.chunks - 1u))), b = uniform(static_cast<uint32_t>(rest / (K.chunks - 1u)));
  const At at(A, group, block);
  const uint32_t n = steps_of(A.lengths, b, A.steps), first = chunk * kChunk, count = steps_in(first, kChunk, n);
  const bool gate = A.gate.data != nullptr;
  float rate[kS], g[kS] = {};
  rates_of(A, at, rate);
  const float bias = A.delta_bias ? A.delta_bias[at.c] : 0.0f;
  stage<T, kChunk, kStates>(rows_c, A.c, A, b, group, first, count, 64u * kRearWaves);
  __syncthreads();
  const uint64_t anew = anew_from(A, b, first, kChunk, n);
  float total = 0.0f;
  const uint32_t tiles = (count + kTile - 1u) / kTile;
  T v[kOwn], z[kOwn], dy[kOwn];
  const Column<T> v_at(A.delta, b, first, at.own, at.c), z_at(gate ? A.gate : A.delta, b, first, at.own, at.c), dy_at(G.dy, b, first, at.own, at.c);
  auto ask = [&](uint32_t tile) {
#pragma unroll
    for (uint32_t j = 0; j < kOwn; ++j) {
      v[j] = z[j] = dy[j] = static_cast<T>(0.0f);
      if (tile + kTile <= count || tile + at.own + j < count) {
        v[j] = v_at.at(tile + j), dy[j] = dy_at.at(tile + j);
        if (gate) z[j] = z_at.at(tile + j);
      }
    }
  };
  if (tiles > 0u) ask((tiles - 1u) * kTile);
  for (uint32_t i = tiles; i-- > 0u;) {
    const uint32_t tile = i * kTile, t0 = first + tile;
#pragma unroll
    for (uint32_t j = 0; j < kOwn; ++j) {
      float grow, slope, size = size_of(A, static_cast<float>(v[j]), bias, grow);
      if (t0 + at.own + j >= n) size = 0.0f;
      total += size;
      sizes[wave][at.channel * kTile + at.own + j] = size;
      grads[wave][at.channel * kTile + at.own + j] = static_cast<float>(dy[j]) * shown_of(gate, gate ? static_cast<float>(z[j]) : 0.0f, slope);
    }
    if (i > 0u) ask(tile - kTile);
    wave_sync();
    float size[kTile], dinner[kTile];
    read_tile(&sizes[wave][at.channel * kTile], size);
    read_tile(&grads[wave][at.channel * kTile], dinner);
    const uint32_t starts = static_cast<uint32_t>(anew >> tile) & ((1u << kTile) - 1u);
    auto walk = [&](auto with_starts) __attribute__((always_inline)) {
#pragma unroll
      for (uint32_t t = kTile; t-- > 0u;) {
        float out[kS];
        read_shared<kS>(&rows_c[(tile + t) * kStates + at.q * kS], out);
#pragma unroll
        for (uint32_t s = 0; s < kS; ++s) {
          g[s] = __builtin_amdgcn_exp2f(size[t] * rate[s]) * __fmaf_rn(dinner[t], out[s], g[s]);
          if (with_starts && ((starts >> t) & 1u) != 0u) g[s] = 0.0f;
        }
      }
    };
    if (starts == 0u) walk(No{}); else walk(Yes{});
    wave_sync();
  }
  const uint64_t slot = static_cast<uint64_t>(b) * K.chunks + chunk;
  write_states(K.ends + slot * (static_cast<uint64_t>(A.width) * A.states), A, at, g);
  if (!at.first) total = 0.0f;
  total = sum_lanes<kQ>(total);
  if (at.mine && at.q == 0u) K.sums[slot * A.width + at.c] = total;
  if (group == 0u && block == 0u && at.lane == 0u) K.cuts[slot] = anew != 0u ? 1u : 0u;
}

__global__ void __launch_bounds__(256) scan_rear_join_kernel(ScanArgs A, ScanGradArgs G, RearCut K, uint64_t begin) {
  constexpr uint32_t kAtOnce = 8;
  const uint64_t row = static_cast<uint64_t>(A.width) * A.states, i = (begin + blockIdx.x) * 256u + threadIdx.x;
  if (i >= row * A.batch) return;
  const uint64_t b = i / row, at = i % row, c = at / A.states;
  const float r0 = A.a[at] * kLog2e, r1 = r0 > 3.0e38f ? 3.0e38f : r0, rate = r1 < -3.0e38f ? -3.0e38f : r1;
  float g = G.dh_last ? G.dh_last[i] : 0.0f;
  float* to = K.ends + b * K.chunks * row + at;
  const float* sums = K.sums + b * K.chunks * A.width + c;
  const uint32_t* cuts = K.cuts + b * K.chunks;
  for (uint32_t done = 0; done < K.chunks; done += kAtOnce) {
    const uint32_t upto = K.chunks - done;                                           // chunks left, the last of them first
    float ends[kAtOnce], half[kAtOnce];
#pragma unroll
    for (uint32_t j = 0; j < kAtOnce; ++j) {
      const uint32_t k = max(upto, j + 1u) - j - 1u;                                 // (the first one's slot is unset memory, and not used)
      ends[j] = to[k * row];
      half[j] = half_decay(rate, sums[static_cast<uint64_t>(k) * A.width]);
    }
#pragma unroll
    for (uint32_t j = 0; j < kAtOnce; ++j) {
      if (j >= upto) continue;
      const uint32_t k = upto - j - 1u;
      to[k * row] = g;
      if (k > 0u) g = cuts[k] != 0u ? ends[j] : past(half[j], g, ends[j]);
    }
  }
}

// Sums over the channels of a wave of kCount numbers a lane: lanes that differ in kBit and above are different channels of the same states.  Every lane is left with some of the sums, those
// from `base` on; how many, is returned.
template <int kBit, int kLeast, int kCount>
__device__ __forceinline__ constexpr int left_of() {
  if constexpr (kBit < kLeast) return kCount;
  else return left_of<kBit / 2, kLeast, kCount % 2 == 0 ? kCount / 2 : kCount>();
}
template <int kBit, int kLeast, int kCount, int kAll>
__device__ __forceinline__ void sum_channels(float (&v)[kAll], uint32_t lane, uint32_t& base) {
  if constexpr (kBit >= kLeast) {
    if constexpr (kCount % 2 == 0) {
      const bool upper = (lane & kBit) != 0u;
#pragma unroll
      for (int i = 0; i < kCount / 2; ++i) {
        const float keep = upper ? v[i + kCount / 2] : v[i], give = upper ? v[i] : v[i + kCount / 2];
        v[i] = keep + __shfl_xor(give, kBit);
      }
      base += upper ? kCount / 2 : 0u;
      sum_channels<kBit / 2, kLeast, kCount / 2>(v, lane, base);
    } else {
#pragma unroll
      for (int i = 0; i < kCount; ++i) v[i] += __shfl_xor(v[i], kBit);
      sum_channels<kBit / 2, kLeast, kCount>(v, lane, base);
    }
  }
}

// Which of a tile's steps a lane owns, where their sums are made for four steps at a time: the exchange leaves lane q the sum of step q / (kQ / 4) of the four, or of several.
template <int kQ, int kT>
struct Owned {
  static constexpr uint32_t kFours = kT / 4, kPer = kQ >= 4 ? 1 : 4 / kQ, kOwn = kQ > 4 ? (kFours * 4 + kQ - 1) / kQ : kFours * kPer, kLanes = kQ >= 4 ? kQ / 4 : 1;   // kLanes get the same sum
  static_assert(kFours == 1 || kFours == 2, "one or two times four steps");
  uint32_t q;
  // the lane's first step, and the others' distance from it
  __device__ uint32_t first() const { return kQ > 4 ? (kFours == 2 ? (q & 1u) * 4u : 0u) + q / kLanes : q * kPer; }
  static constexpr uint32_t apart(uint32_t j) { return kQ > 4 ? 0u : j / kPer * 4u + j % kPer; }
  // of the lanes that own the same step, the one that stores its results
  __device__ bool stores() const { return kQ <= 4 || (kFours == 2 ? q / 2u % (kLanes / 2u > 0u ? kLanes / 2u : 1u) == 0u : q % kLanes == 0u); }
  // takes its sums of the four-th four steps
  __device__ void take(uint32_t four, const float (&v)[4], float (&own)[kOwn]) const {
    if constexpr (kQ > 4) {
      own[0] = kFours == 1 || (q & 1u) == four ? v[0] : own[0];
    } else {
#pragma unroll
      for (uint32_t j = 0; j < kPer; ++j) own[four * kPer + j] = v[j];
    }
  }
};

template <int kS, int kQ, int kT, uint32_t kWaves>
struct SharedBackward {
  static constexpr uint32_t kStates = kS * kQ, kChannels = 64 / kQ, kTile = kT;
  float rows_b[kWaves * kTile * kStates], rows_c[kWaves * kTile * kStates];
  float of_step[kWaves][3][kChannels * kTile];     // sizes, size * input, gradient before the gate
  float parts[2][kWaves][3][64 * kS];              // what a wave's steps do: half of the decay's exponent, as a factor, state, gradient
  float da[2][kWaves][64 * kS], own[2][kWaves][2][kChannels];
};

// Two waves a SIMD, of workgroups that wait for different barriers. With 16 states it has 190 registers (the sums of B's and C's gradients are 32 of them); where they are made to be 168, for three
// waves, they spill, and 8 x 4096 x 2048 bf16 takes 3700 to 4300 us instead of 1520; with the states behind the steps in shared memory instead, which leaves eleven to spill, 2680, and 1720 with two
// waves. Sums over a channel's states are made for four steps at a time: for eight 206 registers, 1600 (24 states, 6 x 1001 x 1502 f16: 152 instead of 281, as two waves find room).
template <typename T, int kS, int kQ, int kT, uint32_t kWaves>
__global__ void __launch_bounds__(64 * kWaves) scan_backward_kernel(ScanArgs A, ScanGradArgs G, RearCut K, uint64_t begin) {
  typedef Spot<kS, kQ, kT> At;
  typedef Owned<kQ, kT> Mine;
  constexpr uint32_t kTile = kT, kWalked = kWaves * kTile, kOwn = Mine::kOwn, kStates = At::kStates, kChannels = At::kChannels;
  __shared__ __attribute__((aligned(16))) SharedBackward<kS, kQ, kT, kWaves> lds;
  uint64_t rest = begin + blockIdx.x;
  const uint32_t split = uniform(static_cast<uint32_t>(rest % K.splits));
  rest /= K.splits;
  const uint32_t group = uniform(static_cast<uint32_t>(rest % A.groups));
  rest /= A.groups;
  const uint32_t chunk = uniform(static_cast<uint32_t>(rest % K.chunks)), b = uniform(static_cast<uint32_t>(rest / K.chunks));
  const uint32_t wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63u, each = A.width / A.groups;
  const uint32_t n = steps_of(A.lengths, b, A.steps), first = chunk * kChunk, count = steps_in(first, kWalked, n);
  const uint32_t t0 = first + wave * kTile, valid = steps_in(t0, kTile, n), behind = steps_in(t0, kTile, A.steps);
  const bool gate = A.gate.data != nullptr;
  const uint64_t row = static_cast<uint64_t>(A.width) * A.states, slot = static_cast<uint64_t>(b) * K.chunks + chunk;
  const uint32_t per = (K.blocks + K.splits - 1u) / K.splits, from = split * per, upto = min(from + per, K.blocks);
  if (count == 0u) {                   // (the same for the whole workgroup) nothing of the row is here: zeros, and what comes in behind the chunk goes on before it
    const uint32_t first_channel = min(from * kChannels, each), channels = min(upto * kChannels, each) - min(first_channel, min(upto * kChannels, each));
    const uint32_t length = steps_in(first, kWalked, A.steps), both = A.groups * A.states;
    for (uint32_t i = threadIdx.x; i < channels; i += 64u * kWaves) {
      const uint32_t c = group * each + first_channel + i;
      for (uint32_t t = 0; t < length; ++t) {
        *element<T>(G.dx, b, first + t, c) = static_cast<T>(0.0f);
        *element<T>(G.ddelta, b, first + t, c) = static_cast<T>(0.0f);
        if (gate) *element<T>(G.dgate, b, first + t, c) = static_cast<T>(0.0f);
      }
      float* to = K.parts + slot * (row + 2u * A.width);
      to[row + c] = to[row + A.width + c] = 0.0f;
    }
    for (uint32_t i = threadIdx.x; i < channels * A.states; i += 64u * kWaves) {
      const uint64_t at = static_cast<uint64_t>(group * each + first_channel) * A.states + i;
      K.parts[slot * (row + 2u * A.width) + at] = 0.0f;
      if (G.dh0 && chunk == 0u) G.dh0[b * row + at] = K.chunks > 1u ? K.ends[slot * row + at] : G.dh_last ? G.dh_last[b * row + at] : 0.0f;
    }
    for (uint32_t i = threadIdx.x; i < length * 2u * A.states; i += 64u * kWaves) {
      const uint32_t t = i / (2u * A.states), which = i / A.states % 2u, state = i % A.states;
      K.rows[(((static_cast<uint64_t>(split) * A.batch + b) * A.steps + first + t) * 2u + which) * both + group * A.states + state] = 0.0f;
    }
    return;
  }
  stage<T, kWalked, kStates>(lds.rows_b, A.b, A, b, group, first, count, 64u * kWaves);
  stage<T, kWalked, kStates>(lds.rows_c, A.c, A, b, group, first, count, 64u * kWaves);
  const uint64_t anew = anew_from(A, b, first, kWalked, n);
  constexpr uint32_t kBits = (1u << kTile) - 1u;
  const uint32_t starts = static_cast<uint32_t>(anew >> (wave * kTile)) & kBits;
  float sums[2 * kTile * kS] = {};     // of the gradients of B and C
  // the sums over the waves of what an earlier turn left
  auto finish = [&](uint32_t block, uint32_t turn) __attribute__((always_inline)) {
    float* to = K.parts + slot * (row + 2u * A.width);
    for (uint32_t id = here(threadIdx.x); id < 64u * kS + 2u * kChannels; id += 64u * kWaves) {
      float sum = 0.0f;
      if (id < 64u * kS) {
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) sum += lds.da[turn][w][id];
        const uint32_t l = id / kS, state = l % kQ * kS + id % kS, c = block * kChannels + l / kQ;
        if (c < each && state < A.states) to[(group * each + c) * A.states + state] = sum;
      } else {
        const uint32_t which = (id - 64u * kS) / kChannels, channel = (id - 64u * kS) % kChannels, c = block * kChannels + channel;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) sum += lds.own[turn][w][which][channel];
        if (c < each) to[static_cast<uint32_t>(row) + which * A.width + group * each + c] = sum;
      }
    }
  };
  const uint32_t own_step = Mine{lane % kQ}.first();
  const Column<T> x_at(A.x, b, t0, own_step, group * each), v_at(A.delta, b, t0, own_step, group * each), z_at(gate ? A.gate : A.x, b, t0, own_step, group * each),
      dy_at(G.dy, b, t0, own_step, group * each), dx_at(G.dx, b, t0, own_step, group * each), dv_at(G.ddelta, b, t0, own_step, group * each),
      dz_at(gate ? G.dgate : G.dx, b, t0, own_step, group * each);
  T x[kOwn], v[kOwn], z[kOwn], dy[kOwn];
  float rate_in[kS], h_in[kS], g_in[kS] = {}, through_in, bias_in;
  // what a stretch of channels needs from memory, asked for while the one before is worked on; steps that are not there are not looked at
  auto ask = [&](uint32_t block) __attribute__((always_inline)) {
    const At at(A, group, block, here(lane));
    const uint32_t along = (at.c - group * each) * static_cast<uint32_t>(sizeof(T));
    if (valid == kTile) {
#pragma unroll
      for (uint32_t j = 0; j < kOwn; ++j) {
        x[j] = x_at.at(Mine::apart(j), along), v[j] = v_at.at(Mine::apart(j), along), dy[j] = dy_at.at(Mine::apart(j), along);
        z[j] = gate ? z_at.at(Mine::apart(j), along) : static_cast<T>(0.0f);
      }
    } else {
#pragma unroll
      for (uint32_t j = 0; j < kOwn; ++j) {
        x[j] = v[j] = z[j] = dy[j] = static_cast<T>(0.0f);
        if (own_step + Mine::apart(j) < valid) {
          x[j] = x_at.at(Mine::apart(j), along), v[j] = v_at.at(Mine::apart(j), along), dy[j] = dy_at.at(Mine::apart(j), along);
          if (gate) z[j] = z_at.at(Mine::apart(j), along);
        }
      }
    }
    read_states(A.a, A, at, rate_in);
    read_states(A.kept + (static_cast<uint64_t>(b) * K.kept + chunk) * row, A, at, h_in);
    if (K.chunks > 1u) read_states(K.ends + slot * row, A, at, g_in);
    else if (G.dh_last) read_states(G.dh_last + b * row, A, at, g_in);
    through_in = A.d ? A.d[at.c] : 0.0f;
    bias_in = A.delta_bias ? A.delta_bias[at.c] : 0.0f;
  };
  if (from < upto) ask(from);
  __syncthreads();
  auto turns = [&](auto with_starts) __attribute__((always_inline)) {
    for (uint32_t block = from; block < upto; ++block) {
      const uint32_t turn = (block - from) & 1u;
      const At at(A, group, block, here(lane));
      const uint32_t along = (at.c - group * each) * static_cast<uint32_t>(sizeof(T));
      const Mine mine{at.q};
      const uint32_t own = mine.first();
      float input[kOwn], grow[kOwn], size_own[kOwn], dinner_own[kOwn], dgate_by[kOwn];      // dgate_by: the gate's gradient, without its factor `inner`
      float h[kS], g[kS], rate[kS];
      const float through = through_in;
      float *const of_size = lds.of_step[wave][0] + at.channel * kTile, *const of_fed = lds.of_step[wave][1] + at.channel * kTile, *const of_grad = lds.of_step[wave][2] + at.channel * kTile;
#pragma unroll
      for (uint32_t j = 0; j < kOwn; ++j) {
        float slope;
        const bool there = at.mine && own + Mine::apart(j) < valid;           // (lanes behind the group have no part in its sums)
        input[j] = there ? static_cast<float>(x[j]) : 0.0f;
        const float size = size_of(A, static_cast<float>(v[j]), bias_in, grow[j]), given = there ? static_cast<float>(dy[j]) : 0.0f;
        size_own[j] = there ? size : 0.0f;
        dinner_own[j] = given * shown_of(gate, static_cast<float>(z[j]), slope);
        dgate_by[j] = given * slope;
        if (!there) dinner_own[j] = dgate_by[j] = 0.0f;
        held(input[j]), held(size_own[j]), held(grow[j]), held(dinner_own[j]), held(dgate_by[j]);
        of_size[own + Mine::apart(j)] = size_own[j];
        of_fed[own + Mine::apart(j)] = size_own[j] * input[j];
        of_grad[own + Mine::apart(j)] = dinner_own[j];
      }
#pragma unroll
      for (uint32_t s = 0; s < kS; ++s) rate[s] = rate_in[s], h[s] = at.mine ? h_in[s] : 0.0f, g[s] = at.mine ? g_in[s] : 0.0f;
      finite_rates(rate);
      if (block + 1u < upto) ask(block + 1u);
      wave_sync();
      float size[kTile], fed[kTile], dinner[kTile];
      read_tile(of_size, size);
      read_tile(of_fed, fed);
      read_tile(of_grad, dinner);
      wave_sync();
      const float *const row_b = lds.rows_b + (wave * kTile * kStates + at.q * kS), *const row_c = lds.rows_c + (wave * kTile * kStates + at.q * kS);
      // (a step that is not there has the size 0 and brings nothing: it leaves states and gradients as they are)
      float a[kTile][kS], own_h[kS] = {}, own_g[kS] = {}, half[kS];
#pragma unroll
      for (uint32_t t = 0; t < kTile; ++t) {
        float in[kS];
        read_shared<kS>(row_b + t * kStates, in);
#pragma unroll
        for (uint32_t s = 0; s < kS; ++s) {
          a[t][s] = __builtin_amdgcn_exp2f(size[t] * rate[s]);
          if (with_starts && ((starts >> t) & 1u) != 0u) own_h[s] = 0.0f;
          own_h[s] = t == 0u ? fed[t] * in[s] : __fmaf_rn(a[t][s], own_h[s], fed[t] * in[s]);
        }
      }
#pragma unroll
      for (uint32_t t = kTile; t-- > 0u;) {
        float out[kS];
        read_shared<kS>(row_c + t * kStates, out);
#pragma unroll
        for (uint32_t s = 0; s < kS; ++s) {
          own_g[s] = a[t][s] * (t + 1u == kTile ? dinner[t] * out[s] : __fmaf_rn(dinner[t], out[s], own_g[s]));
          if (with_starts && ((starts >> t) & 1u) != 0u) own_g[s] = 0.0f;
        }
      }
      float total = 0.0f;
#pragma unroll
      for (uint32_t t = 0; t < kTile; ++t) total += size[t];
#pragma unroll
      for (uint32_t s = 0; s < kS; ++s) half[s] = half_decay(rate[s], total);
      write_shared<kS>(&lds.parts[turn][wave][0][at.lane * kS], half);
      write_shared<kS>(&lds.parts[turn][wave][1][at.lane * kS], own_h);
      write_shared<kS>(&lds.parts[turn][wave][2][at.lane * kS], own_g);
      __syncthreads();
      // the state before the wave's steps and the gradient behind them, from the other waves' stretches
#pragma unroll
      for (uint32_t w = 0; w + 1u < kWaves; ++w) {
        if (w >= wave) break;
        float p[kS], own[kS];
        read_shared<kS>(&lds.parts[turn][w][0][at.lane * kS], p);
        read_shared<kS>(&lds.parts[turn][w][1][at.lane * kS], own);
        const bool cut = with_starts && (static_cast<uint32_t>(anew >> (w * kTile)) & kBits) != 0u;
#pragma unroll
        for (uint32_t s = 0; s < kS; ++s) h[s] = cut ? own[s] : past(p[s], h[s], own[s]);
      }
#pragma unroll
      for (uint32_t w = kWaves - 1u; w > 0u; --w) {
        if (w <= wave) break;
        float p[kS], own[kS];
        read_shared<kS>(&lds.parts[turn][w][0][at.lane * kS], p);
        read_shared<kS>(&lds.parts[turn][w][2][at.lane * kS], own);
        const bool cut = with_starts && (static_cast<uint32_t>(anew >> (w * kTile)) & kBits) != 0u;
#pragma unroll
        for (uint32_t s = 0; s < kS; ++s) g[s] = cut ? own[s] : past(p[s], g[s], own[s]);
      }
      if (block > from) finish(block - 1u, turn ^ 1u);
      float inner[kOwn] = {}, came[kOwn] = {}, slower[kOwn] = {}, da[kS] = {};      // of the lane's own steps, sums over the channel's states; da of its states, over the steps
      float after[kTile][kS];
#pragma unroll
      for (uint32_t t = 0; t < kTile; ++t) {
        float in[kS];
        read_shared<kS>(row_b + t * kStates, in);
#pragma unroll
        for (uint32_t s = 0; s < kS; ++s) {
          const float prior = t == 0u ? h[s] : after[t > 0u ? t - 1u : 0u][s];
          after[t][s] = __fmaf_rn(a[t][s], with_starts && ((starts >> t) & 1u) != 0u ? 0.0f : prior, fed[t] * in[s]);
        }
      }
#pragma unroll
      for (uint32_t four = Mine::kFours; four-- > 0u;) {
        float inner4[4] = {}, came4[4] = {}, slower4[4] = {};
#pragma unroll
        for (uint32_t i = 4; i-- > 0u;) {
          const uint32_t t = four * 4u + i;
          float in[kS], out[kS];
          read_shared<kS>(row_b + t * kStates, in);
          read_shared<kS>(row_c + t * kStates, out);
          const bool anew_here = with_starts && ((starts >> t) & 1u) != 0u;
#pragma unroll
          for (uint32_t s = 0; s < kS; ++s) {
            float prior = t == 0u ? h[s] : after[t > 0u ? t - 1u : 0u][s];
            if (anew_here) prior = 0.0f;
            inner4[i] = __fmaf_rn(after[t][s], out[s], inner4[i]);
            sums[(kTile + t) * kS + s] = __fmaf_rn(dinner[t], after[t][s], sums[(kTile + t) * kS + s]);
            const float d = __fmaf_rn(dinner[t], out[s], g[s]);
            came4[i] = __fmaf_rn(d, in[s], came4[i]);
            sums[t * kS + s] = __fmaf_rn(fed[t], d, sums[t * kS + s]);
            g[s] = a[t][s] * d;
            const float lost = g[s] * prior;                         // the gradient of the decay's exponent
            slower4[i] = __fmaf_rn(lost, rate[s], slower4[i]);
            da[s] = __fmaf_rn(lost, size[t], da[s]);
            if (anew_here) g[s] = 0.0f;
          }
        }
        sum_for_owners<kQ, 4>(inner4, lane);
        sum_for_owners<kQ, 4>(came4, lane);
        sum_for_owners<kQ, 4>(slower4, lane);
        mine.take(four, inner4, inner), mine.take(four, came4, came), mine.take(four, slower4, slower);
      }
      if (G.dh0 && chunk == 0u && wave == 0u) write_states(G.dh0 + b * row, A, at, g);
      float dd = 0.0f, dbias = 0.0f;
#pragma unroll
      for (uint32_t j = 0; j < kOwn; ++j) {
        const bool there = own + Mine::apart(j) < valid;
        const float dv = there ? __fmaf_rn(came[j], input[j], slower[j] * kLn2) * grow[j] : 0.0f;
        const float dx = there ? __fmaf_rn(came[j], size_own[j], dinner_own[j] * through) : 0.0f;
        const float dgate = there ? __fmaf_rn(through, input[j], inner[j]) * dgate_by[j] : 0.0f;
        dd += there ? dinner_own[j] * input[j] : 0.0f;
        dbias += dv;
        if (at.mine && mine.stores() && own + Mine::apart(j) < behind) {
          dx_at.at(Mine::apart(j), along) = static_cast<T>(dx);
          dv_at.at(Mine::apart(j), along) = static_cast<T>(dv);
          if (gate) dz_at.at(Mine::apart(j), along) = static_cast<T>(dgate);
        }
      }
      dd = sum_lanes<kQ>(mine.stores() ? dd : 0.0f);
      dbias = sum_lanes<kQ>(mine.stores() ? dbias : 0.0f);
      write_shared<kS>(&lds.da[turn][wave][at.lane * kS], da);
      if (at.q == 0u) lds.own[turn][wave][0][at.channel] = dd, lds.own[turn][wave][1][at.channel] = dbias;
    }
  };
  // (in a chunk where nothing starts anew nothing has to be looked at for it; the same for the whole workgroup)
  if (anew == 0u) turns(No{}); else turns(Yes{});
  __syncthreads();
  if (from < upto) finish(upto - 1u, (upto - 1u - from) & 1u);
  uint32_t base = 0u;
  sum_channels<32, kQ, 2 * kTile * kS>(sums, lane, base);
  constexpr int kLeft = left_of<32, kQ, 2 * kTile * kS>();
  const uint32_t both = A.groups * A.states;
#pragma unroll
  for (int i = 0; i < kLeft; ++i) {
    const uint32_t id = base + i, which = id / (kTile * kS), t = id / kS % kTile, state = lane % kQ * kS + id % kS;
    if (t0 + t < A.steps && state < A.states)
      K.rows[(((static_cast<uint64_t>(split) * A.batch + b) * A.steps + t0 + t) * 2u + which) * both + group * A.states + state] = first + wave * kTile + t < n ? sums[i] : 0.0f;
  }
}

// Gradients of B and C from the splits' parts.
template <typename T>
__global__ void __launch_bounds__(256) scan_rows_kernel(ScanArgs A, ScanGradArgs G, RearCut K, uint64_t begin) {
  const uint64_t both = static_cast<uint64_t>(A.groups) * A.states, all = static_cast<uint64_t>(A.batch) * A.steps * 2u * both, i = (begin + blockIdx.x) * 256u + threadIdx.x;
  if (i >= all) return;
  float sum = 0.0f;
#pragma unroll 8
  for (uint32_t k = 0; k < K.splits; ++k) sum += K.rows[k * all + i];
  const uint64_t step = i / (2u * both), in_step = i % (2u * both);
  const uint32_t j = static_cast<uint32_t>(in_step % both), b = static_cast<uint32_t>(step / A.steps), t = static_cast<uint32_t>(step % A.steps);
  *element<T>(in_step < both ? G.db : G.dc, b, t, j) = static_cast<T>(sum);
}

// Sequences without steps hand on what comes in.
__global__ void __launch_bounds__(256) scan_hand_on_kernel(const float* dh_last, float* dh0, uint64_t count, uint64_t begin) {
  const uint64_t i = (begin + blockIdx.x) * 256u + threadIdx.x;
  if (i < count) dh0[i] = dh_last ? dh_last[i] : 0.0f;
}

RearCut rear_cut(const ScanArgs& a) {
  // Workgroups of the third launch: each has a start of its own (rows to stage), so no more of them than fill the device (kFill).  Where rows may end early, a few times as many (kSpare), as all of a
  // chunk's workgroups behind a row's end have nothing to do; not so for sequences of one chunk, which all rows with steps have, nor down to fewer than kLeast stretches of channels each.
  // us, the backward call with lengths that are all full / of every size, with kFill, with kSpare and no least, and as it is (without lengths a call takes what all full ones do with kFill):
  //   20 x 35 x 1500 fp32              56 / 55    84 / 81    56 / 55
  //   32 x 48 x 4096 bf16             176 / 174  203 / 198  176 / 174
  //   2 x 500 x 768 fp32               43 / 42    61 / 50    43 / 42
  //   8 x 100 x 2048 bf16              68 / 66    78 / 60    70 / 51
  //   8 x 200 x 1024 bf16, 64 states  234 / 222  279 / 175  260 / 170
  //   8 x 200 x 1024 bf16, 32 states  113 / 108  130 / 90   125 / 86
  //   128 x 64 x 512 bf16             114 / 111  122 / 118  122 / 118
  //   1 x 4096 x 1024 bf16            146 / 127  154 / 106  154 / 106
  //   6 x 1001 x 1502 bf16            298 / 279  257 / 181  257 / 181
  //   6 x 1001 x 1502 f16, 24 states  386 / 365  336 / 232  337 / 232
  //   4 x 2048 x 2048 bf16            450 / 395  437 / 256  437 / 257
  //   16 x 300 x 4096 bf16            567 / 509  549 / 387  549 / 385
  constexpr uint64_t kFill = 512, kSpare = 2048, kLeast = 8;
  RearCut K{};
  const uint32_t channels = wave_channels<Kind::kBackward>(a.states), rear = kRearWaves * wave_channels<Kind::kSummary>(a.states), each = a.width / a.groups;
  K.kept = (a.steps + kChunk - 1u) / kChunk;
  K.whole = a.steps > kChunk && a.steps <= kWholeWaves * kWholeTile && a.states <= kWholeStates;
  K.chunks = K.whole ? 1u : K.kept;
  K.across = (each + rear - 1u) / rear;
  K.blocks = (each + channels - 1u) / channels;
  const uint64_t apart = static_cast<uint64_t>(a.batch) * K.chunks * a.groups;
  auto splits_of = [&](uint64_t enough) { return std::min<uint64_t>(apart > 0u && apart < enough ? enough / apart : 1u, K.blocks); };
  K.splits = static_cast<uint32_t>(splits_of(kFill));
  if (a.lengths && K.chunks > 1u) K.splits = std::max(K.splits, static_cast<uint32_t>(std::min<uint64_t>(splits_of(kSpare), K.blocks / kLeast)));
  return K;
}

struct RearWords {
  uint64_t ends, sums, cuts, parts, rows;                                             // 32-bit words of each
  uint64_t all() const { return ends + sums + cuts + parts + rows; }
};
RearWords rear_words(const ScanArgs& a, const RearCut& k) {
  const uint64_t slots = static_cast<uint64_t>(a.batch) * k.chunks, joined = k.chunks > 1u ? slots : 0u;
  return RearWords{joined * a.width * a.states, joined * a.width, joined, slots * a.width * (a.states + 2u),
                   static_cast<uint64_t>(k.splits) * a.batch * a.steps * 2u * a.groups * a.states};
}

}  // namespace

uint64_t scan_backward_scratch_words(const ScanArgs& a) { return (rear_words(a, rear_cut(a)).all() + 1u) / 2u; }

hipError_t launch_scan_backward(const ScanArgs& a, const ScanGradArgs& g, int dtype, unsigned long long* scratch, hipStream_t s) {
  RearCut K = rear_cut(a);
  const RearWords W = rear_words(a, K);
  K.ends = reinterpret_cast<float*>(scratch);
  K.sums = K.ends + W.ends;
  K.cuts = reinterpret_cast<uint32_t*>(K.sums + W.sums);
  K.parts = reinterpret_cast<float*>(K.cuts + W.cuts);
  K.rows = K.parts + W.parts;
  const uint64_t slots = static_cast<uint64_t>(a.batch) * K.chunks, weights = static_cast<uint64_t>(a.width) * a.states;
  if (slots > 0u) {
    if (K.chunks > 1u) {
      const hipError_t e = by_states<Kind::kSummary>(a.states, dtype, [&](auto type, auto layout) {
        in_grids((slots - a.batch) * a.groups * K.across, [&](uint64_t begin, dim3 grid) {
          scan_rear_kernel<decltype(type), decltype(layout)::kS, decltype(layout)::kQ><<<grid, dim3(64 * kRearWaves), 0, s>>>(a, g, K, begin);
        });
        return hipGetLastError();
      });
      if (e != hipSuccess) return e;
      in_grids((a.batch * weights + 255u) / 256u, [&](uint64_t begin, dim3 grid) { scan_rear_join_kernel<<<grid, dim3(256), 0, s>>>(a, g, K, begin); });
    }
    const hipError_t e = by_states<Kind::kBackward>(a.states, dtype, [&](auto type, auto layout) {
      using T = decltype(type);
      constexpr int kS = decltype(layout)::kS, kQ = decltype(layout)::kQ, kT = decltype(layout)::kT;
      in_grids(slots * a.groups * K.splits, [&](uint64_t begin, dim3 grid) {
        if (K.whole) {
          if constexpr (kT == kWholeTile) scan_backward_kernel<T, kS, kQ, kT, kWholeWaves><<<grid, dim3(64 * kWholeWaves), 0, s>>>(a, g, K, begin);
        } else {
          scan_backward_kernel<T, kS, kQ, kT, kChunk / kT><<<grid, dim3(64 * (kChunk / kT)), 0, s>>>(a, g, K, begin);
        }
      });
      const uint64_t all = static_cast<uint64_t>(a.batch) * a.steps * 2u * a.groups * a.states;
      in_grids((all + 255u) / 256u, [&](uint64_t begin, dim3 grid) { scan_rows_kernel<T><<<grid, dim3(256), 0, s>>>(a, g, K, begin); });
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  } else if (g.dh0) {
    const uint64_t count = a.batch * weights;
    in_grids((count + 255u) / 256u, [&](uint64_t begin, dim3 grid) { scan_hand_on_kernel<<<grid, dim3(256), 0, s>>>(g.dh_last, g.dh0, count, begin); });
  }
  return launch_sum_parts(PartsArgs{K.parts, slots, weights + 2u * a.width, {g.da, g.dd, g.ddelta_bias}, {weights, weights + a.width, weights + 2u * a.width}}, s);
}

}  // namespace rgc
