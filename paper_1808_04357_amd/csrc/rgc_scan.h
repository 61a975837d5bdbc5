// What the kernels of the selective scan share (rgc_scan.hip, rgc_scan_backward.hip).
//
// A wave takes 64 / kQ channels of a sequence: kQ lanes have a channel's states, kS each, and kTile steps at a time. What a step has once for all of a channel's states (its size,
// its input, ...) is computed by one of the channel's lanes, its owner, and handed to the others through shared memory; sums over a channel's states go the other way, by exchanges
// between neighbouring lanes that leave every owner its steps' sums.  B and C, which all channels of a group share, lie in shared memory in 32 bits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "rgc_lm.h"
#include "rgc_sequence.h"

namespace rgc {
namespace {

constexpr uint32_t kChunk = 64;        // steps between kept states (RGC_SCAN_CHUNK)
constexpr uint32_t kTile = 8;          // steps of a wave at a time
constexpr float kLn2 = 0.693147180559945309f;

template <int kCtrl>
__device__ __forceinline__ float from_lane(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kCtrl, 0xF, 0xF, true));
}
// One level of the exchange: lanes whose number has kBit keep the upper half of their sums, the others the lower, and get what the lane across has for it.
template <int kCtrl, int kBit, int kCount>
__device__ __forceinline__ void exchange(float (&v)[kTile], uint32_t lane) {
  if constexpr (kCount >= 2) {
    const bool upper = (lane & kBit) != 0u;
#pragma unroll
    for (int i = 0; i < kCount / 2; ++i) {
      const float keep = upper ? v[i + kCount / 2] : v[i], give = upper ? v[i] : v[i + kCount / 2];
      v[i] = keep + from_lane<kCtrl>(give);
    }
  } else {
    v[0] += from_lane<kCtrl>(v[0]);
  }
}
// v[t]: a lane's part of step t's sum over the channel's states; afterwards v[0 .. steps it owns) are its steps' sums.
template <int kQ>
__device__ __forceinline__ void sum_for_owners(float (&v)[kTile], uint32_t lane) {
  static_assert(kQ == 1 || kQ == 2 || kQ == 4 || kQ == 8 || kQ == 16, "lanes of a channel");
  if constexpr (kQ >= 16) exchange<0x140, 8, kTile>(v, lane);                         // row_mirror
  if constexpr (kQ >= 8) exchange<0x141, 4, kQ >= 16 ? kTile / 2 : kTile>(v, lane);   // row_half_mirror
  if constexpr (kQ >= 4) exchange<0x4E, 2, kQ >= 16 ? kTile / 4 : kQ >= 8 ? kTile / 2 : kTile>(v, lane);                            // quad_perm 2 3 0 1
  if constexpr (kQ >= 2) exchange<0xB1, 1, kQ >= 16 ? kTile / 8 : kQ >= 8 ? kTile / 4 : kQ >= 4 ? kTile / 2 : kTile>(v, lane);      // quad_perm 1 0 3 2
}

// Where a lane is: its channel, its states, its steps of a tile.
template <int kS, int kQ>
struct Spot {
  static constexpr uint32_t kChannels = 64 / kQ, kStates = kS * kQ, kOwn = kQ >= 8 ? 1 : kTile / kQ;
  uint32_t lane, channel, q, own;      // within the wave; the first of its steps
  uint32_t c;                          // of the sequence (the group's last one in a lane behind it)
  bool mine, owner;                    // it is a channel of the group; the lane stores its steps' results
  // block: how many waves' channels of the group come before
  __device__ Spot(const ScanArgs& A, uint32_t group, uint32_t block) {
    const uint32_t each = A.width / A.groups;
    lane = threadIdx.x & 63u;
    channel = lane / kQ;
    q = lane % kQ;
    own = kQ == 16 ? q / 2u : q * kOwn;
    const uint32_t at = block * kChannels + channel;
    mine = at < each;
    owner = mine && (kQ < 16 || q % 2u == 0u);
    c = group * each + min(at, each - 1u);
  }
};

// A channel's rates for the lane's states, in powers of two.  Finite, so that a step that is not there (its size 0) has the decay 1.
template <int kS, int kQ>
__device__ __forceinline__ void rates_of(const ScanArgs& A, const Spot<kS, kQ>& at, float (&rate)[kS]) {
#pragma unroll
  for (uint32_t s = 0; s < kS; ++s) {
    const uint32_t n = at.q * kS + s;
    float r = n < A.states ? A.a[static_cast<uint64_t>(at.c) * A.states + n] * kLog2e : 0.0f;
    r = r > 3.0e38f ? 3.0e38f : r;
    rate[s] = r < -3.0e38f ? -3.0e38f : r;
  }
}

// The lane's states of a [.., width, states] tensor whose row for the sequence (and chunk) begins at `from`.
template <int kS, int kQ>
__device__ __forceinline__ void read_states(const float* from, const ScanArgs& A, const Spot<kS, kQ>& at, float (&h)[kS]) {
  const float* p = from + static_cast<uint64_t>(at.c) * A.states + at.q * kS;
  if (kS == 4 && A.states == kS * kQ) {
    const Raw<float, 4> r = read_at<float, 4>(p);
#pragma unroll
    for (uint32_t s = 0; s < kS; ++s) h[s] = r.v[s & 3u];
  } else {
#pragma unroll
    for (uint32_t s = 0; s < kS; ++s) h[s] = at.q * kS + s < A.states ? p[s] : 0.0f;
  }
}
template <int kS, int kQ>
__device__ __forceinline__ void write_states(float* to, const ScanArgs& A, const Spot<kS, kQ>& at, const float (&h)[kS]) {
  if (!at.mine) return;
  float* p = to + static_cast<uint64_t>(at.c) * A.states + at.q * kS;
#pragma unroll
  for (uint32_t s = 0; s < kS; ++s)
    if (at.q * kS + s < A.states) p[s] = h[s];
}

// ln(1 + exp(v)), with what it is beside exp(v) where that is small: the power is corrected by what its exponent lost in rounding, the sum 1 + e by what it lost.
// grow: sigmoid(v), its slope.
__device__ __forceinline__ float softplus(float v, float& grow) {
  const float low = v < -150.0f ? -150.0f : v;                     // (exp is 0 there; keeps the correction finite)
  const float x = low * kLog2e;
  const float lost = __fmaf_rn(low, 1.925963033500e-8f, __fmaf_rn(low, kLog2e, -x));      // log2(e) has more digits
  const float p = __builtin_amdgcn_exp2f(x), e = __fmaf_rn(p, lost * kLn2, p);
  const float w = 1.0f + e, c = e - (w - 1.0f), r = __builtin_amdgcn_rcpf(w);
  const bool large = v > 20.0f;                                    // (there ln(1 + exp(v)) - v is below v's last digit)
  grow = large ? 1.0f - __builtin_amdgcn_exp2f(-v * kLog2e) : e * r;
  return large ? v : __fmaf_rn(c, r, __builtin_amdgcn_logf(w) * kLn2);
}

// What a step does: its size and the slope of the softplus (1 without one).
__device__ __forceinline__ float size_of(const ScanArgs& A, float v, float bias, float& grow) {
  v += bias;
  if (A.softplus) return softplus(v, grow);
  grow = 1.0f;
  return v;
}

template <typename T>
__device__ __forceinline__ T* element(const SequenceView& v, uint32_t b, uint32_t t, uint32_t c) {
  return static_cast<T*>(v.data) + (b * v.batch_stride + t * v.step_stride + c);
}

// An owner's steps of one tensor, from step `first` on; those at `end` and beyond are not looked at and read as 0.
template <typename T, uint32_t kOwn>
struct Own {
  T v[kOwn];
  __device__ void read(const SequenceView& s, uint32_t b, uint32_t first, uint32_t end, uint32_t c) {
    const T* p = element<T>(s, b, first, c);
#pragma unroll
    for (uint32_t j = 0; j < kOwn; ++j, p += s.step_stride) v[j] = first + j < end ? *p : static_cast<T>(0.0f);
  }
  // all of them are there
  __device__ void read(const SequenceView& s, uint32_t b, uint32_t first, uint32_t c) {
    const T* p = element<T>(s, b, first, c);
#pragma unroll
    for (uint32_t j = 0; j < kOwn; ++j, p += s.step_stride) v[j] = *p;
  }
};

// Rows of B or C in 32 bits: steps [first, first + count) of group g, kStates apart (zeros behind the group's states), by the workgroup's kThreads threads.
template <typename T, uint32_t kStates, uint32_t kThreads>
__device__ __forceinline__ void stage(float* to, const SequenceView& from, const ScanArgs& A, uint32_t b, uint32_t g, uint32_t first, uint32_t count) {
  for (uint32_t i = threadIdx.x; i < count * kStates; i += kThreads) {
    const uint32_t t = i / kStates, n = i % kStates;
    to[i] = n < A.states ? static_cast<float>(*element<T>(from, b, first + t, g * A.states + n)) : 0.0f;
  }
}

// kS neighbouring numbers of shared memory.
template <int kS>
__device__ __forceinline__ void read_shared(const float* p, float (&v)[kS]) {
  if constexpr (kS == 4) {
    typedef float four __attribute__((ext_vector_type(4)));
    const four r = *reinterpret_cast<const four*>(p);
    v[0] = r.x, v[1] = r.y, v[2] = r.z, v[3] = r.w;
  } else {
#pragma unroll
    for (int s = 0; s < kS; ++s) v[s] = p[s];
  }
}
__device__ __forceinline__ void read_tile(const float* p, float (&v)[kTile]) {
  float low[4], high[4];
  read_shared<4>(p, low);
  read_shared<4>(p + 4, high);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = low[i], v[i + 4] = high[i];
}

// What lanes of one wave have written to shared memory is there for the others of it.  (The wave's accesses are carried out in their order; the compiler keeps it.)
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Bit i: the state starts anew at step first + i (of those the row has).
__device__ __forceinline__ uint64_t anew_from(const ScanArgs& A, uint32_t b, uint32_t first, uint32_t n) {
  if (!A.resets) return 0u;
  const uint32_t t = first + (threadIdx.x & 63u);
  return __ballot(t < n && A.resets[static_cast<uint64_t>(b) * A.steps + t] != 0);
}

// Steps of [first, first + most) that are before `end`.
__device__ __forceinline__ uint32_t steps_in(uint32_t first, uint32_t most, uint32_t end) { return min(max(end, first) - first, most); }

// Calls f with the type, the states a lane and the lanes a channel as constants.  Fewer lanes a channel mean fewer exchanges, more of them fewer registers.
template <typename F>
hipError_t by_states(uint32_t states, int dtype, F&& f) {
  auto with = [&](auto s, auto q) {
    if (dtype == 0) return f(float{}, s, q);
    if (dtype == 1) return f(__bf16{}, s, q);
    return f(_Float16{}, s, q);
  };
  typedef std::integral_constant<int, 1> One;
  typedef std::integral_constant<int, 4> Four;
  if (states == 1u) return with(One{}, One{});
  if (states <= 4u) return with(Four{}, One{});
  if (states <= 8u) return with(Four{}, std::integral_constant<int, 2>{});
  if (states <= 16u) return with(Four{}, Four{});
  if (states <= 24u) return with(std::integral_constant<int, 3>{}, std::integral_constant<int, 8>{});
  if (states <= 32u) return with(Four{}, std::integral_constant<int, 8>{});
  return with(Four{}, std::integral_constant<int, 16>{});
}
// The same choice for the host: channels of a wave.
inline uint32_t wave_channels(uint32_t states) { return states <= 4u ? 64u : states <= 8u ? 32u : states <= 16u ? 16u : states <= 32u ? 8u : 4u; }

}  // namespace
}  // namespace rgc
