// What the kernels of the selective scan share (rgc_scan.hip, rgc_scan_backward.hip).
//
// A wave takes 64 / kQ channels of a sequence: kQ lanes have a channel's states, kS each, and kT steps at a time. What a step has once for all of a channel's states (its size,
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

constexpr uint32_t kChunk = 32;        // steps between kept states (RGC_SCAN_CHUNK)
constexpr float kLn2 = 0.693147180559945309f;

template <int kCtrl>
__device__ __forceinline__ float from_lane(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kCtrl, 0xF, 0xF, true));
}
// One level of the exchange: lanes whose number has kBit keep the upper half of their kCount sums, the others the lower, and get what the lane across has for it.
template <int kCtrl, int kBit, int kCount, int kAll>
__device__ __forceinline__ void exchange(float (&v)[kAll], uint32_t lane) {
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
// The sum over a channel's lanes, in all of them.
template <int kQ>
__device__ __forceinline__ float sum_lanes(float v) {
  if constexpr (kQ >= 16) v += from_lane<0x140>(v);
  if constexpr (kQ >= 8) v += from_lane<0x141>(v);
  if constexpr (kQ >= 4) v += from_lane<0x4E>(v);
  if constexpr (kQ >= 2) v += from_lane<0xB1>(v);
  return v;
}
// v[t]: a lane's part of step t's sum over the channel's states; afterwards v[0 .. steps it owns) are its steps' sums.
template <int kQ, int kT>
__device__ __forceinline__ void sum_for_owners(float (&v)[kT], uint32_t lane) {
  static_assert(kQ == 1 || kQ == 2 || kQ == 4 || kQ == 8 || kQ == 16, "lanes of a channel");
  constexpr int k8 = kQ >= 16 ? kT / 2 : kT, k4 = kQ >= 8 ? k8 / 2 : k8, k2 = kQ >= 4 ? k4 / 2 : k4;      // sums left before a level (0 as one)
  if constexpr (kQ >= 16) exchange<0x140, 8, kT>(v, lane);       // row_mirror
  if constexpr (kQ >= 8) exchange<0x141, 4, k8>(v, lane);        // row_half_mirror
  if constexpr (kQ >= 4) exchange<0x4E, 2, k4>(v, lane);         // quad_perm 2 3 0 1
  if constexpr (kQ >= 2) exchange<0xB1, 1, k2>(v, lane);         // quad_perm 1 0 3 2
}

// Where a lane is: its channel, its states, its steps of a tile.
template <int kS, int kQ, int kT>
struct Spot {
  static constexpr uint32_t kChannels = 64 / kQ, kStates = kS * kQ, kOwn = kQ >= kT ? 1 : kT / kQ, kShare = kQ > kT ? kQ / kT : 1;      // kShare lanes own the same step
  uint32_t lane, channel, q, own;      // within the wave; the first of its steps
  uint32_t c;                          // of the sequence (the group's last one in a lane behind it)
  bool mine, first, owner;             // it is a channel of the group; the first lane that owns its step; the lane stores its steps' results
  // block: how many waves' channels of the group come before
  __device__ Spot(const ScanArgs& A, uint32_t group, uint32_t block) : Spot(A, group, block, threadIdx.x & 63u) {}
  __device__ Spot(const ScanArgs& A, uint32_t group, uint32_t block, uint32_t in_wave) {
    const uint32_t each = A.width / A.groups;
    lane = in_wave;
    channel = lane / kQ;
    q = lane % kQ;
    own = q * kOwn / kShare;
    const uint32_t at = block * kChannels + channel;
    mine = at < each;
    first = q % kShare == 0u;
    owner = mine && first;
    c = group * each + min(at, each - 1u);
  }
};

// Where a lane's states lie in a [.., width, states] tensor: bytes from its row for the sequence (and chunk), which is the same for the whole wave.
template <int kS, int kQ, int kT>
__device__ __forceinline__ uint32_t states_at(const ScanArgs& A, const Spot<kS, kQ, kT>& at) {
  return (at.c * A.states + at.q * kS) * static_cast<uint32_t>(sizeof(float));
}
// The states that lie there; zeros for those that a channel does not have.  (No branch but one that the whole wave takes.)
template <int kS, int kQ>
__device__ __forceinline__ void read_states(const float* row, const ScanArgs& A, uint32_t q, uint32_t offset, float (&h)[kS]) {
  const char* base = reinterpret_cast<const char*>(row);
  if (A.states == kS * kQ) {
    constexpr int kVec = kS % 4 == 0 ? 4 : kS % 2 == 0 ? 2 : 1;
#pragma unroll
    for (int s = 0; s < kS; s += kVec) {
      const Raw<float, kVec> r = read_at<float, kVec>(reinterpret_cast<const float*>(base + (offset + s * 4u)));
#pragma unroll
      for (int i = 0; i < kVec; ++i) h[s + i] = r.v[i];
    }
  } else {
    const uint32_t first = offset - q * kS * 4u;
#pragma unroll
    for (uint32_t s = 0; s < kS; ++s) {
      const float v = *reinterpret_cast<const float*>(base + (first + min(q * kS + s, A.states - 1u) * 4u));
      h[s] = q * kS + s < A.states ? v : 0.0f;
    }
  }
}
template <int kS, int kQ, int kT>
__device__ __forceinline__ void write_states(float* row, const ScanArgs& A, const Spot<kS, kQ, kT>& at, const float (&h)[kS]) {
  if (!at.mine) return;
  float* p = reinterpret_cast<float*>(reinterpret_cast<char*>(row) + states_at(A, at));
  constexpr int kVec = kS % 4 == 0 ? 4 : kS % 2 == 0 ? 2 : 1;
  if (kVec > 1 && A.states == kS * kQ) {
#pragma unroll
    for (int s = 0; s < kS; s += kVec) write_at<float, kVec>(p + s, *reinterpret_cast<const float(*)[kVec]>(&h[s]));
  } else {
#pragma unroll
    for (uint32_t s = 0; s < kS; ++s)
      if (at.q * kS + s < A.states) p[s] = h[s];
  }
}

// A channel's rates for the lane's states, in powers of two.  Finite, so that a step that is not there (its size 0) has the decay 1.
template <int kS>
__device__ __forceinline__ void finite_rates(float (&rate)[kS]) {
#pragma unroll
  for (uint32_t s = 0; s < kS; ++s) {
    float r = rate[s] * kLog2e;
    r = r > 3.0e38f ? 3.0e38f : r;
    rate[s] = r < -3.0e38f ? -3.0e38f : r;
  }
}
template <int kS, int kQ, int kT>
__device__ __forceinline__ void rates_of(const ScanArgs& A, const Spot<kS, kQ, kT>& at, float (&rate)[kS]) {
  read_states<kS, kQ>(A.a, A, at.q, states_at(A, at), rate);
  finite_rates(rate);
}
template <int kS, int kQ, int kT>
__device__ __forceinline__ void read_states(const float* row, const ScanArgs& A, const Spot<kS, kQ, kT>& at, float (&h)[kS]) {
  read_states<kS, kQ>(row, A, at.q, states_at(A, at), h);
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

// A lane's elements of one tensor: a row's address, the same for the whole wave, and the lane's own steps and channel as 32 bits of offset from it.  (A tile's steps span less than
// 2^32 bytes: the host refuses strides beyond.)
template <typename T>
struct Column {
  char* row;
  int64_t step;
  uint32_t offset;
  __device__ Column(const SequenceView& v, uint32_t b, uint32_t first, uint32_t own, uint32_t c)
      : row(reinterpret_cast<char*>(element<T>(v, b, first, 0u))), step(v.step_stride * static_cast<int64_t>(sizeof(T))),
        offset((own * static_cast<uint32_t>(v.step_stride) + c) * static_cast<uint32_t>(sizeof(T))) {}
  // the j-th step behind the lane's first, a uniform number of bytes along the row
  __device__ T& at(uint32_t j, uint32_t along = 0u) const { return *reinterpret_cast<T*>(row + static_cast<int64_t>(j) * step + (offset + along)); }
};

// A chunk's rows of B or C on their way to shared memory in 32 bits, kStates a step (zeros behind the group's states), by the workgroup's kThreads threads: asked for well before they are needed.
template <typename T, uint32_t kStates, uint32_t kThreads>
struct Staged {
  static constexpr uint32_t kEach = (kChunk * kStates + kThreads - 1u) / kThreads;
  T v[kEach];
  __device__ void ask(const SequenceView& from, const ScanArgs& A, uint32_t b, uint32_t g, uint32_t first, uint32_t count) {
    const char* row = reinterpret_cast<const char*>(element<T>(from, b, first, g * A.states));
    const int64_t step = from.step_stride * static_cast<int64_t>(sizeof(T));
#pragma unroll
    for (uint32_t r = 0; r < kEach; ++r) {
      const uint32_t i = threadIdx.x + r * kThreads, t = i / kStates, n = i % kStates;
      v[r] = t < count && n < A.states ? *reinterpret_cast<const T*>(row + t * step + n * sizeof(T)) : static_cast<T>(0.0f);
    }
  }
  __device__ void put(float* to) const {
#pragma unroll
    for (uint32_t r = 0; r < kEach; ++r) {
      const uint32_t i = threadIdx.x + r * kThreads;
      if (kChunk * kStates % kThreads == 0u || i < kChunk * kStates) to[i] = static_cast<float>(v[r]);
    }
  }
};

// kRows rows of B or C in 32 bits, `count` of them from memory and zeros behind, kStates a step, by so many threads.
template <typename T, uint32_t kRows, uint32_t kStates>
__device__ __forceinline__ void stage(float* to, const SequenceView& from, const ScanArgs& A, uint32_t b, uint32_t g, uint32_t first, uint32_t count, uint32_t threads) {
  const char* row = reinterpret_cast<const char*>(element<T>(from, b, first, g * A.states));
  const int64_t step = from.step_stride * static_cast<int64_t>(sizeof(T));
#pragma unroll 2
  for (uint32_t i = threadIdx.x; i < kRows * kStates; i += threads) {
    const uint32_t t = i / kStates, n = i % kStates;
    to[i] = t < count && n < A.states ? static_cast<float>(*reinterpret_cast<const T*>(row + t * step + n * sizeof(T))) : 0.0f;
  }
}

// kS neighbouring numbers of shared memory, four or two at a time.
typedef float Two __attribute__((ext_vector_type(2)));
typedef float Four __attribute__((ext_vector_type(4)));
template <int kS>
__device__ __forceinline__ void read_shared(const float* p, float (&v)[kS]) {
#pragma unroll
  for (int s = 0; s < kS; s += kS % 4 == 0 ? 4 : kS % 2 == 0 ? 2 : 1) {
    if constexpr (kS % 4 == 0) {
      const Four r = *reinterpret_cast<const Four*>(p + s);
      v[s] = r.x, v[s + 1] = r.y, v[s + 2] = r.z, v[s + 3] = r.w;
    } else if constexpr (kS % 2 == 0) {
      const Two r = *reinterpret_cast<const Two*>(p + s);
      v[s] = r.x, v[s + 1] = r.y;
    } else {
      v[s] = p[s];
    }
  }
}
template <int kS>
__device__ __forceinline__ void write_shared(float* p, const float (&v)[kS]) {
#pragma unroll
  for (int s = 0; s < kS; s += kS % 4 == 0 ? 4 : kS % 2 == 0 ? 2 : 1) {
    if constexpr (kS % 4 == 0) *reinterpret_cast<Four*>(p + s) = Four{v[s], v[s + 1], v[s + 2], v[s + 3]};
    else if constexpr (kS % 2 == 0) *reinterpret_cast<Two*>(p + s) = Two{v[s], v[s + 1]};
    else p[s] = v[s];
  }
}
template <int kT>
__device__ __forceinline__ void read_tile(const float* p, float (&v)[kT]) {
#pragma unroll
  for (int t = 0; t < kT; t += 4) {
    float part[4];
    read_shared<4>(p + t, part);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[t + i] = part[i];
  }
}

// A number that the compiler takes for a new one here: it does not compute what follows from it earlier, to hold it in registers all the way to its use.
__device__ __forceinline__ uint32_t here(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}
// A number that is computed here, and not where it is used, from the several that it is made of.
__device__ __forceinline__ void held(float& v) { asm volatile("" : "+v"(v)); }

// What lanes of one wave have written to shared memory is there for the others of it.  (The wave's accesses are carried out in their order; the compiler keeps it.)
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// What comes out of a stretch of steps, of what goes in and of what it makes of 0.  Its decay comes in two equal factors: where states grow their product may be beyond all numbers though no state
// is, and a 0 stays 0.
__device__ __forceinline__ float half_decay(float rate, float size) { return __builtin_amdgcn_exp2f(0.5f * rate * size); }
__device__ __forceinline__ float past(float half, float in, float made) { return in == 0.0f ? made : __fmaf_rn(half, half * in, made); }

// Bit i: the state starts anew at step first + i (of the next `most`, and of those the row has).
__device__ __forceinline__ uint64_t anew_from(const ScanArgs& A, uint32_t b, uint32_t first, uint32_t most, uint32_t n) {
  if (!A.resets) return 0u;
  const uint32_t i = threadIdx.x & 63u, t = first + i;
  return __ballot(i < most && t < n && A.resets[static_cast<uint64_t>(b) * A.steps + t] != 0);
}

// Steps of [first, first + most) that are before `end`.
__device__ __forceinline__ uint32_t steps_in(uint32_t first, uint32_t most, uint32_t end) { return min(max(end, first) - first, most); }

// How many states a lane has and how many lanes a channel: fewer lanes mean fewer exchanges and less to be done once a channel, more of them more waves and fewer registers.
template <int kStatesOfLane, int kLanes, int kStepsAtOnce>
struct Layout {
  static constexpr int kS = kStatesOfLane, kQ = kLanes, kT = kStepsAtOnce;
};
enum class Kind { kWalk, kSummary, kBackward };      // a walk along the steps for results, for what a stretch does to a state (or a gradient) alone, the backward walk
// Calls f with the type and the layout.  us, 8 x 4096 x 2048 bf16 with 16 states (20 x 35 x 1500 fp32): backward two states a lane, eight steps, four waves a workgroup 1520 (53), four states, four
// steps, eight waves 1711 (63; all of a compute unit's waves wait at one barrier), four states and eight steps do not fit into registers; the walk by two states a lane 550, by four 1013 (half
// the waves: one a SIMD), by one 998; a summary, which has little to do once a channel and waves enough, by four 262, by two 311.
// What that makes of other numbers of states, us, 8 x 1024 x 2048, forward and backward call: 1 state bf16 66 and 129 (fp32 92 and 170), 4 85 and 190 (108 and 233), 8 115 and 268 (125 and 288),
// 16 126 and 432 (126 and 461), 24 153 and 559 (149 and 582), 32 171 and 850 (168 and 873), 64 335 and 1997 (337 and 2017): above 32 the backward pass has 84 KB of shared memory a workgroup, one a
// compute unit, and twice the time a state's step.
template <Kind kKind, typename F>
hipError_t by_states(uint32_t states, int dtype, F&& f) {
  auto with = [&](auto layout) {
    if (dtype == 0) return f(float{}, layout);
    if (dtype == 1) return f(__bf16{}, layout);
    return f(_Float16{}, layout);
  };
  if (states == 1u) return with(Layout<1, 1, 8>{});
  if constexpr (kKind == Kind::kBackward) {
    if (states <= 4u) return with(Layout<2, 2, 8>{});
    if (states <= 8u) return with(Layout<2, 4, 8>{});
    if (states <= 16u) return with(Layout<2, 8, 8>{});
    if (states <= 24u) return with(Layout<3, 8, 8>{});
    if (states <= 32u) return with(Layout<2, 16, 8>{});
    return with(Layout<4, 16, 4>{});
  } else {
    if (states <= 4u) return with(Layout<4, 1, 8>{});
    if (states <= 8u) return with(Layout<4, 2, 8>{});
    if constexpr (kKind == Kind::kSummary) {
      if (states <= 16u) return with(Layout<4, 4, 8>{});
    } else {
      if (states <= 16u) return with(Layout<2, 8, 8>{});
    }
    if (states <= 24u) return with(Layout<3, 8, 8>{});
    if (states <= 32u) return with(Layout<4, 8, 8>{});
    return with(Layout<4, 16, 8>{});
  }
}
// The same choice for the host: channels of a wave.
template <Kind kKind>
uint32_t wave_channels(uint32_t states) {
  uint32_t channels = 0u;
  (void)by_states<kKind>(states, 0, [&](auto, auto layout) {
    channels = 64u / decltype(layout)::kQ;
    return hipSuccess;
  });
  return channels;
}

}  // namespace
}  // namespace rgc
