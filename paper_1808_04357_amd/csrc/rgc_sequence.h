// What the kernels over sequences share: sigmoids, channels read and written where they lie, a lane's channels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rgc_lm.h"

namespace rgc {
namespace {

constexpr float kLog2e = 1.44269504088896341f;

// sigmoid(v) and sigmoid(-v) with one power and one reciprocal.  Below -87 the power may be infinite, and infinity times 0 is not 1.
// (Written so that a NaN passes.)
__device__ __forceinline__ void gate_of(float v, float& keep, float& take) {
  const float x = -kLog2e * v;
  const float e = __builtin_amdgcn_exp2f(x);
  keep = __builtin_amdgcn_rcpf(1.0f + e);
  take = x > 126.0f ? 1.0f : e * keep;
}

// kVec neighbouring channels as they lie in memory (aligned to an element only: rows may start anywhere, and gfx950 reads and
// writes words at any address).
typedef uint32_t __attribute__((aligned(2))) word;

template <typename T, int kVec>
struct alignas(sizeof(T)) Raw {
  T v[kVec];
};

// A tensor's rows from a step on: an address that is the same for the whole wave, which a step moves on, and a lane's offset from it.
template <typename T>
struct Rows {
  char* p;
  int64_t step;                       // bytes
  __device__ Rows(const SequenceView& v, uint32_t b, uint32_t t)
      : p(reinterpret_cast<char*>(static_cast<T*>(v.data) + (b * v.batch_stride + t * v.step_stride))), step(v.step_stride * static_cast<int64_t>(sizeof(T))) {}
};

template <typename T, int kVec>
__device__ __forceinline__ Raw<T, kVec> read(const char* row, uint32_t offset) {
  Raw<T, kVec> r;
  if constexpr (sizeof(T) * kVec == 4) {
    const uint32_t w = *reinterpret_cast<const word*>(row + offset);
    __builtin_memcpy(&r, &w, 4);
  } else {
    r = *reinterpret_cast<const Raw<T, kVec>*>(row + offset);
  }
  return r;
}

template <typename T, int kVec>
__device__ __forceinline__ void write(char* row, uint32_t offset, const float (&v)[kVec]) {
  Raw<T, kVec> r;
#pragma unroll
  for (int i = 0; i < kVec; ++i) r.v[i] = static_cast<T>(v[i]);
  if constexpr (sizeof(T) * kVec == 4) {
    uint32_t w;
    __builtin_memcpy(&w, &r, 4);
    *reinterpret_cast<word*>(row + offset) = w;
  } else {
    *reinterpret_cast<Raw<T, kVec>*>(row + offset) = r;
  }
}

struct Yes {
  constexpr operator bool() const { return true; }
};
struct No {
  constexpr operator bool() const { return false; }
};

// Where a lane's channels lie.  The last lane of a row with an odd number of channels takes the two last ones and stores the second only; lanes
// behind the row's end work on the last channels too, so that all lanes do the same, and store nothing.
template <int kVec>
struct Lane {
  uint32_t c;                 // first channel
  bool all, last;             // stores all its channels / its last one only
  __device__ Lane(uint32_t block, uint32_t width) {
    const uint32_t want = (block * 64u + (threadIdx.x & 63u)) * kVec;
    all = want + kVec <= width;
    last = kVec > 1 && !all && want < width;
    c = all ? want : width - kVec;
  }
};

template <typename T, int kVec, bool kWhole>
__device__ __forceinline__ void store(char* row, const Lane<kVec>& lane, const float (&v)[kVec]) {
  if (kWhole || lane.all) write<T, kVec>(row, lane.c * static_cast<uint32_t>(sizeof(T)), v);
  else if (lane.last) reinterpret_cast<T*>(row)[lane.c + kVec - 1] = static_cast<T>(v[kVec - 1]);
}

// kVec neighbouring elements in one access of up to 16 bytes, at any address that is a multiple of the element's size.
template <uint32_t kBytes>
struct Bits;
template <>
struct Bits<2> {
  typedef uint16_t type;
};
template <>
struct Bits<4> {
  typedef uint32_t __attribute__((aligned(2))) type;
};
template <>
struct Bits<8> {
  typedef uint32_t __attribute__((ext_vector_type(2), aligned(2))) type;
};
template <>
struct Bits<16> {
  typedef uint32_t __attribute__((ext_vector_type(4), aligned(2))) type;
};
template <typename T, int kVec>
__device__ __forceinline__ Raw<T, kVec> read_at(const T* p) {
  Raw<T, kVec> r;
  if constexpr (sizeof(T) * kVec > 16) {
    constexpr int kPart = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < kVec; i += kPart) {
      const Raw<T, kPart> part = read_at<T, kPart>(p + i);
      __builtin_memcpy(&r.v[i], &part, 16);
    }
  } else {
    const auto w = *reinterpret_cast<const typename Bits<sizeof(T) * kVec>::type*>(p);
    __builtin_memcpy(&r, &w, sizeof(T) * kVec);
  }
  return r;
}
template <typename T, int kVec>
__device__ __forceinline__ void write_at(T* p, const float (&v)[kVec]) {
  if constexpr (sizeof(T) * kVec > 16) {
    constexpr int kPart = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < kVec; i += kPart) write_at<T, kPart>(p + i, *reinterpret_cast<const float(*)[kPart]>(&v[i]));
  } else {
    Raw<T, kVec> r;
#pragma unroll
    for (int i = 0; i < kVec; ++i) r.v[i] = static_cast<T>(v[i]);
    typename Bits<sizeof(T) * kVec>::type w;
    __builtin_memcpy(&w, &r, sizeof(T) * kVec);
    *reinterpret_cast<typename Bits<sizeof(T) * kVec>::type*>(p) = w;
  }
}

// Where a lane's kVec channels lie in a row that has at least kVec.  The last lane of a row whose width is no multiple takes the row's last ones, some of which
// the lane before has too, and stores those only that no other lane has (another one's may have been replaced already where a call works in place).  Lanes behind
// it do as it does, so that all lanes do the same, and store nothing.
template <int kVec>
struct Channels {
  uint32_t c, own;             // the first one; the first that no lane before has
  bool mine;
  __device__ Channels(uint32_t block, uint32_t width) {
    own = (block * 64u + (threadIdx.x & 63u)) * kVec;
    mine = own < width;
    c = own + kVec <= width ? own : width - kVec;
  }
};

template <typename T, int kVec>
__device__ __forceinline__ void write_own(T* row, const Channels<kVec>& lane, const float (&v)[kVec]) {
  if (lane.c == lane.own) {
    write_at<T, kVec>(row + lane.c, v);
  } else if (lane.mine) {
#pragma unroll
    for (int i = 1; i < kVec; ++i)
      if (lane.c + i >= lane.own) row[lane.c + i] = static_cast<T>(v[i]);
  }
}

// Steps that a row has.
__device__ __forceinline__ uint32_t steps_of(const int32_t* lengths, uint32_t b, uint32_t steps) {
  if (!lengths) return steps;
  const int32_t n = __builtin_amdgcn_readfirstlane(lengths[b]);
  return n < 0 ? 0u : min(static_cast<uint32_t>(n), steps);
}

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }

// A grid has fewer than 2^32 threads: more workgroups (of up to 512 threads) than that take several launches, each told which its first one is.
template <typename F>
void in_grids(uint64_t workgroups, F&& launch) {
  constexpr uint64_t kMost = uint64_t(1) << 22;
  for (uint64_t begin = 0; begin < workgroups; begin += kMost) launch(begin, dim3(static_cast<uint32_t>(workgroups - begin < kMost ? workgroups - begin : kMost)));
}

}  // namespace
}  // namespace rgc
