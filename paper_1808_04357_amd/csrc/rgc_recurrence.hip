// rgc_recurrence.hip -- the gated linear recurrence, forward and backward (include/rgc.h has the formulas).
//
// A stretch of steps takes the state h before it to P h + H after it: P is the product of its gates, H the state it ends with from 0.
// Two stretches (P1, H1), (P2, H2) in a row make (P1 P2, P2 H1 + H2).  That is all a parallel scan needs: a workgroup takes a tile of
// kWaves * kSteps steps by one wave's channels, every wave reads its kSteps steps into registers (each tensor is read once), makes its (P, H) of them,
// learns from the others' what state it begins with, and runs through its steps again from that state, out of the registers.
// Backward the same is done twice, for the state in the order of the steps and for its gradient against it:
// with g the gradient that leaves a step towards the one before it, d = e + g', g = f d.
//
// Tiles of one chain (a sequence's 64 kVec channels) follow each other in time, and a tile needs the state that the one before it ends with.
// Tiles are handed out by a ticket, all chains' first tiles, then all second ones: a tile publishes its (P, H) as soon as it has it, the last one of a group of
// tiles the group's, and the state behind the group (which is a stretch with P = 0) when it knows that; and a tile looks back over the published ones until it has come to
// a state.  It waits for tiles of smaller tickets only, and a ticket is taken by a workgroup that runs, so the smallest ticket not done
// waits for nothing: every wait ends, however few workgroups run at a time.
//
// Which words were states already when a tile looked is a matter of time, what it makes of them is not: stretches are joined in the same order whatever
// was met, to the last bit (rgc_stretch.h).
//
// 1 - sigmoid(v) is computed as sigmoid(-v), which keeps its precision where the gate is nearly open.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "rgc_lm.h"
#include "rgc_sequence.h"
#include "rgc_stretch.h"

namespace rgc {
namespace {

constexpr uint32_t kChunk = 256;       // steps between kept states (RGC_RECURRENCE_CHUNK)
constexpr uint32_t kOneTile = 128;     // steps of the sequences that are one tile (kMiddle below)

// How a sequence is cut: the same constants make the tiles and choose the kernel.  What it is bound by: a forward pass moves 4 tensors, a backward one 7, and
// with 29 and 61 instructions an element the arithmetic takes half of that time.  Forward and backward, us, bf16: 20 x 35 x 1500 with waves of eight steps 5.9 and 8.8, of sixteen
// 11.4 and 11.1, of four 6.7 and 11.1; 64 x 100 x 1024 in one tile of sixteen waves 17 and 28.5, in tiles as for long ones 22 and 42.  Long ones forward, one prompt
// of 32768 x 1500 and 8 x 4096 x 2048, by waves and steps: 8 x 16 129 and 124, 4 x 16 135 and 134, 16 x 8 142 and 154, 8 x 8 149 and 138, 16 x 16 143 and 147 (one or two channels a
// lane as the registers allow; four channels a lane 240 and 174), all with the stretches joined as come_in says of earlier; 8 x 16 now 123 and 122.  Backward, 16 x 16 (a kept
// state begins every tile): 235, 4.0 TB/s.
// With an output gate the long kernels of 16 bits have no registers left: of 128 a lane the forward one spills 12 to 14, the backward one 11 (7 in fp32); without a gate
// they have 115 and 114, in fp32 forward 75.
struct Shape {
  uint32_t waves, steps;           // waves a workgroup, steps a wave
  constexpr uint32_t tile() const { return waves * steps; }
};
constexpr Shape kOneWave{1, 4}, kShort{8, 8}, kMiddle{16, 8}, kLong{8, 16}, kLongBackward{16, 16};
static_assert(kMiddle.tile() == kOneTile && kLongBackward.tile() == kChunk, "as backward_tile takes its states");
enum class Kind { kOneWave, kShort, kMiddle, kLong };
// Whether tiles of this shape wait for each other (a shorter sequence than those is one tile).
constexpr bool chained(uint32_t waves, uint32_t steps) {
  return (waves == kLong.waves && steps == kLong.steps) || (waves == kLongBackward.waves && steps == kLongBackward.steps);
}

// A wave's steps of one tensor, all asked for at once.  Steps at `end` and beyond are read as the last one before: a branch around every
// read makes the compiler wait for one before it asks for the next.
template <typename T, int kVec, int kSteps, bool kWhole>
__device__ __forceinline__ void read_steps(Raw<T, kVec> (&to)[kSteps], const SequenceView& v, uint32_t b, uint32_t first, uint32_t end, uint32_t offset) {
  Rows<T> rows(v, b, first);
#pragma unroll
  for (uint32_t r = 0; r < kSteps; ++r) {
    to[r] = read<T, kVec>(rows.p, offset);
    if (kWhole || first + r + 1u < end) rows.p += rows.step;
  }
}

template <int kVec>
__device__ __forceinline__ void store_state(float* row, const Lane<kVec>& lane, const float (&v)[kVec]) {
#pragma unroll
  for (int i = 0; i < kVec; ++i)
    if (lane.all || (lane.last && i == kVec - 1)) row[lane.c + i] = v[i];
}

__device__ __forceinline__ uint32_t length_of(const RecurrenceArgs& A, uint32_t b) {
  if (!A.lengths) return A.steps;
  const int32_t n = A.lengths[b];
  return uniform(n < 0 ? 0u : min(static_cast<uint32_t>(n), A.steps));
}

// Bit r: the state starts anew at step first + r.
template <int kSteps>
__device__ __forceinline__ uint32_t resets_of(const RecurrenceArgs& A, uint32_t b, uint32_t first, uint32_t end) {
  if (!A.resets) return 0u;
  const uint32_t t = first + (threadIdx.x & 63u);
  const bool anew = (threadIdx.x & 63u) < kSteps && t < end && A.resets[static_cast<uint64_t>(b) * A.steps + t] != 0;
  return static_cast<uint32_t>(__ballot(anew));
}

// Which tile this workgroup works on: by ticket where tiles wait for each other.  (Stretches of channels side by side share cache lines where rows do not
// begin on one.  Handing them to workgroups of one die, eight tiles of each chain side by side, took longer: one prompt 135 instead of 129 us, the backward
// kernel of 8 x 4096 x 2048 246 instead of 234: tiles that begin together wait for each other.)
struct Place {
  uint32_t chain, b, block, order;      // order: how many tiles of the chain come before it
};
template <bool kChained>
__device__ __forceinline__ Place take_place(const RecurrenceArgs& A, const TileArgs& G, uint32_t* lds) {
  uint32_t ticket = blockIdx.x;
  if (kChained && G.tiles > 1u) {
    if (threadIdx.x == 0u) *lds = atomicAdd(G.ticket, 1u);
    __syncthreads();
    ticket = uniform(*lds);
  }
  const uint32_t chains = A.batch * G.across;
  Place p;
  p.order = ticket / chains;
  p.chain = ticket - p.order * chains;
  if (kChained) p.order = min(p.order, G.tiles - 1u);                // (a ticket may be anything where another call has written over it, see settle)
  p.b = p.chain / G.across;
  p.block = p.chain - p.b * G.across;
  return p;
}

template <int kVec>
__device__ __forceinline__ unsigned long long* words_of(const TileArgs& G, uint32_t chain, uint32_t at) {
  return G.words + (static_cast<uint64_t>(chain) * (G.tiles + G.groups) + at) * (64u * kVec) + (threadIdx.x & 63u) * kVec;
}

template <int kVec>
__device__ __forceinline__ void publish(unsigned long long* w, const Stretch (&s)[kVec]) {
#pragma unroll
  for (int i = 0; i < kVec; ++i) __hip_atomic_store(w + i, word_of(s[i]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int kVec>
struct Words {
  unsigned long long v[kVec];
};
template <int kVec>
__device__ __forceinline__ Words<kVec> ask(const unsigned long long* w) {
  Words<kVec> r;
#pragma unroll
  for (int i = 0; i < kVec; ++i) r.v[i] = __hip_atomic_load(w + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return r;
}
template <int kVec>
__device__ __forceinline__ Words<kVec> lost_words() {
  Words<kVec> r;
#pragma unroll
  for (int i = 0; i < kVec; ++i) r.v[i] = kLost;
  return r;
}
// Asks again until they are published.  They are, unless another call on the same context runs at the same time, which the caller is to rule out, and clears them; then
// the kernel ends all the same, with NaN.
template <int kVec>
__device__ __forceinline__ void settle(const TileArgs& G, Words<kVec>& r, const unsigned long long* w, Stretch* to) {
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    for (uint32_t looks = 1u; __any(r.v[i] == kUnset) && looks < G.looks; ++looks) {
      __builtin_amdgcn_s_sleep(1);
      if (r.v[i] == kUnset) r.v[i] = __hip_atomic_load(w + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (r.v[i] == kUnset) r.v[i] = kLost;
    to[i] = stretch_of(r.v[i]);
  }
}

// The state that comes into the tile, from published words.  (A word carries all there is to know, so no other memory needs ordering.)  kGroup tiles that follow each other
// are a group; what is told:
//  - every tile's stretch, to the later ones of its group;
//  - by the group's last tile, the group's stretch, joined from those; and in its place, as soon as that tile knows what came before, the state behind the group.
// A tile goes back over the earlier groups' words until it comes to a state, kWaves of them at a time, one by each wave, applies the groups' stretches behind it one after the
// other, and then its own group's tiles'.  It waits for tiles that wait for nothing themselves, or for the stretches of their group alone; only where none of kKept
// groups' words is a state, it asks for the oldest of them again until one is.
// In us, one prompt of 32768 x 1500, 8 x 4096 x 2048 forward and backward, 1 x 32768 x 64 forward: groups of 16 123, 121, 238, 13.6; of 8 126, 122, 246, 13.5;
// no groups, but every tile's state in the place of its stretch, 133, 125, 234, 23.  (The stretches joined to one on the way back, whichever were met as
// states, 127, 120, 234, 16.4: its last bits were a matter of time.)
constexpr uint32_t kGroup = 16, kKept = 16;

template <int kVec, int kWaves>
struct Before {
  Stretch tiles[kGroup][64 * kVec], groups[kKept][64 * kVec];      // groups[j]: the group j + 1 before this one
  uint32_t is_state[kKept];
  float group_state[64 * kVec], state[64 * kVec];                  // what comes into the group, and into the tile (with two channels a lane)
};
struct Nothing {};

// `whole`: the tile's own stretch, in wave 0; carry: what comes into the first tile.
template <int kVec, int kWaves>
__device__ __forceinline__ void come_in(const TileArgs& G, const Place& at, uint32_t wave, Stretch (&whole)[kVec], Before<kVec, kWaves>& lds, float (&carry)[kVec]) {
  constexpr uint32_t kEach = (kGroup + kWaves - 1u) / kWaves, kMine = 64u * kVec / kWaves;
  static_assert(kKept % kWaves == 0u, "whole rounds");
  const uint32_t lane = threadIdx.x & 63u, group = at.order / kGroup, place = at.order % kGroup;
  const bool followed = at.order + 1u < G.tiles, ends = followed && place + 1u == kGroup;
  if (wave == 0u && followed && !ends) {
    if (at.order == 0u) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) whole[i] = state_of(after(whole[i], carry[i]));
    }
    publish<kVec>(words_of<kVec>(G, at.chain, at.order), whole);
  }
  if (at.order == 0u) return;
  // the nearest groups' words are asked for together with the tiles'; the group's last tile tells the group's stretch before it waits for them
  const unsigned long long *const from = words_of<kVec>(G, at.chain, group * kGroup), *const groups = words_of<kVec>(G, at.chain, G.tiles);
  auto group_at = [&](uint32_t first) { return groups + static_cast<uint64_t>(group - 1u - (first + wave)) * (64u * kVec); };
  Words<kVec> near = {}, tile[kEach] = {};
  if (wave < group) near = ask<kVec>(group_at(0u));
#pragma unroll
  for (uint32_t j = 0; j < kEach; ++j)
    if (wave + j * kWaves < place) tile[j] = ask<kVec>(from + (wave + j * kWaves) * (64u * kVec));
#pragma unroll
  for (uint32_t j = 0; j < kEach; ++j)
    if (wave + j * kWaves < place) settle<kVec>(G, tile[j], from + (wave + j * kWaves) * (64u * kVec), &lds.tiles[wave + j * kWaves][lane * kVec]);
  if (ends) {
    __syncthreads();
    if (wave == 0u) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        Stretch s = lds.tiles[0][lane * kVec + i];
#pragma unroll 4
        for (uint32_t j = 1; j + 1u < kGroup; ++j) s = both(s, lds.tiles[j][lane * kVec + i]);
        whole[i] = both(s, whole[i]);
      }
      publish<kVec>(words_of<kVec>(G, at.chain, G.tiles + group), whole);
    }
  }
  uint32_t n = 0u;                                                   // groups back to the nearest state
  for (uint32_t first = 0, looks = 1u;; ++looks) {
    if (first + wave < group) {
      Stretch* to = &lds.groups[first + wave][lane * kVec];
      settle<kVec>(G, near, group_at(first), to);
      bool open = false;
#pragma unroll
      for (int i = 0; i < kVec; ++i) open |= !cut(stretch_of(near.v[i]).p);
      const bool state = !__any(open);                               // (of all lanes)
      if (lane == 0u) lds.is_state[first + wave] = state ? 1u : 0u;
    }
    __syncthreads();
    if (group == 0u) break;
    const uint32_t seen = min(group - first, static_cast<uint32_t>(kWaves));
    const unsigned long long states = __ballot(lane < seen && lds.is_state[first + min(lane, seen - 1u)] != 0u);
    if (states != 0ull) {
      n = first + static_cast<uint32_t>(__ffsll(states));
      break;
    }
    if (first + kWaves < kKept) first += kWaves;
    else __syncthreads();                                            // (before the same words are replaced)
    if (first + wave < group) near = looks < G.looks ? ask<kVec>(group_at(first)) : lost_words<kVec>();
  }
  auto into_group = [&](uint32_t c) { return state_behind<4>(n, [&](uint32_t j) { return lds.groups[j][c]; }); };
  auto into_tile = [&](uint32_t c, float h) { return state_behind<4>(place, [&](uint32_t j) { return lds.tiles[place - 1u - j][c]; }, h); };
  float into[kVec];
  if constexpr (kVec == 1) {
    into[0] = into_group(lane);
    carry[0] = into_tile(lane, into[0]);
  } else {
    // each wave for some of the channels: eight waves that read all words for all of them keep the shared memory busy for half a microsecond
    const uint32_t c = wave * kMine + min(lane, kMine - 1u);
    const float of_group = into_group(c), of_tile = into_tile(c, of_group);
    if (lane < kMine) {
      lds.group_state[c] = of_group;
      lds.state[c] = of_tile;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kVec; ++i) into[i] = lds.group_state[lane * kVec + i], carry[i] = lds.state[lane * kVec + i];
  }
  if (ends && wave == 0u && group > 0u) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) whole[i] = state_of(after(whole[i], into[i]));
    publish<kVec>(words_of<kVec>(G, at.chain, G.tiles + group), whole);
  }
}

template <int kVec, int kWaves, bool kChained>
struct Shared {
  Stretch parts[kWaves][64 * kVec];
  std::conditional_t<kChained, Before<kVec, kWaves>, Nothing> before;
  uint32_t ticket;
};

// kWhole: all the tile's steps are there, and all its channels.  Otherwise steps behind the row's end become steps that change nothing (f = 1, u = 0).
// What depends on a state starting anew stands in loops of its own, in two forms: the one without is taken by the waves that have none.
template <typename T, int kVec, int kWaves, int kSteps, bool kGated, bool kWhole>
__device__ __forceinline__ void forward_tile(const RecurrenceArgs& A, const TileArgs& G, const Place& at, uint32_t n, Shared<kVec, kWaves, chained(kWaves, kSteps)>& lds) {
  constexpr uint32_t kTile = kWaves * kSteps;
  auto& parts = lds.parts;
  const uint32_t wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63u, b = at.b;
  const Lane<kVec> mine(at.block, A.width);
  const uint32_t offset = mine.c * static_cast<uint32_t>(sizeof(T));
  const uint32_t first = at.order * kTile + wave * kSteps;           // this wave's steps
  const uint32_t valid = kWhole ? kSteps : n > first ? min(n - first, static_cast<uint32_t>(kSteps)) : 0u;
  Raw<T, kVec> x[kSteps], v[kSteps], w[kSteps];
  if (kWhole || valid > 0u) {
    read_steps<T, kVec, kSteps, kWhole>(v, A.gate, b, first, n, offset);
    read_steps<T, kVec, kSteps, kWhole>(x, A.x, b, first, n, offset);
    if constexpr (kGated) read_steps<T, kVec, kSteps, kWhole>(w, A.out_gate, b, first, n, offset);
  }
  const uint32_t anew = resets_of<kSteps>(A, b, first, n);
  float carry[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) carry[i] = at.order == 0u && A.h0 ? A.h0[static_cast<uint64_t>(b) * A.width + mine.c + i] : 0.0f;
  float f[kSteps][kVec], u[kSteps][kVec];
#pragma unroll
  for (uint32_t r = 0; r < kSteps; ++r) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      float take;
      gate_of(static_cast<float>(v[r].v[i]), f[r][i], take);
      u[r][i] = take * static_cast<float>(x[r].v[i]);
      if (!kWhole && r >= valid) f[r][i] = 1.0f, u[r][i] = 0.0f;
    }
  }
  Stretch own[kVec];
  auto scan = [&](auto with_resets) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) own[i] = Stretch{1.0f, 0.0f};
#pragma unroll
    for (uint32_t r = 0; r < kSteps; ++r) {
      const bool starts = with_resets && ((anew >> r) & 1u) != 0u;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        if (starts) own[i] = Stretch{-0.0f, 0.0f};
        own[i].h = __fmaf_rn(f[r][i], own[i].h, u[r][i]);
        own[i].p *= f[r][i];
      }
    }
  };
  if constexpr (kWaves > 1) {
    if (anew == 0u) scan(No{}); else scan(Yes{});
#pragma unroll
    for (int i = 0; i < kVec; ++i) parts[wave][lane * kVec + i] = own[i];
    __syncthreads();
  }
  if constexpr (chained(kWaves, kSteps)) {
    if (G.tiles > 1u) {
      Stretch whole[kVec];
      if (wave == 0u) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          whole[i] = own[i];
#pragma unroll 4
          for (uint32_t j = 1; j < kWaves; ++j) whole[i] = both(whole[i], parts[j][lane * kVec + i]);
        }
      }
      come_in<kVec, kWaves>(G, at, wave, whole, lds.before, carry);
    }
  }
  if (A.states && wave == 0u && at.order * kTile < A.steps && (at.order * kTile) % kChunk == 0u) {
    const uint32_t chunks = (A.steps + kChunk - 1u) / kChunk;
    store_state<kVec>(A.states + (static_cast<uint64_t>(b) * chunks + at.order * kTile / kChunk) * A.width, mine, carry);
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
#pragma unroll 4
    for (uint32_t j = 0; j < wave; ++j) carry[i] = after(parts[j][lane * kVec + i], carry[i]);
  }
  // the states take the place of u, step by step
  auto run = [&](auto with_resets) __attribute__((always_inline)) {
#pragma unroll
    for (uint32_t r = 0; r < kSteps; ++r) {
      const bool starts = with_resets && ((anew >> r) & 1u) != 0u;
#pragma unroll
      for (int i = 0; i < kVec; ++i) u[r][i] = carry[i] = __fmaf_rn(f[r][i], starts ? 0.0f : carry[i], u[r][i]);
    }
  };
  if (anew == 0u) run(No{}); else run(Yes{});
  const uint32_t behind = kWhole ? kSteps : A.steps > first ? min(A.steps - first, static_cast<uint32_t>(kSteps)) : 0u;
  Rows<T> to(A.y, b, first);
#pragma unroll
  for (uint32_t r = 0; r < kSteps; ++r, to.p += to.step) {
    if (!kWhole && r >= behind) continue;
    float y[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      y[i] = u[r][i];
      if constexpr (kGated) {
        float open, shut;
        gate_of(static_cast<float>(w[r].v[i]), open, shut);
        y[i] *= open;
      }
      if (!kWhole && r >= valid) y[i] = 0.0f;
    }
    store<T, kVec, kWhole>(to.p, mine, y);
  }
  if (A.h_last && at.order + 1u == G.tiles && wave + 1u == kWaves) store_state<kVec>(A.h_last + static_cast<uint64_t>(b) * A.width, mine, carry);
}

template <typename T, int kVec, int kWaves, int kSteps, bool kGated>
__global__ void __launch_bounds__(64 * kWaves, 4) recurrence_kernel(RecurrenceArgs A, TileArgs G) {
  __shared__ Shared<kVec, kWaves, chained(kWaves, kSteps)> lds;
  const Place at = take_place<chained(kWaves, kSteps)>(A, G, &lds.ticket);
  const uint32_t n = length_of(A, at.b);
  if ((at.order + 1u) * (kWaves * kSteps) <= n && (at.block + 1u) * 64u * kVec <= A.width)
    forward_tile<T, kVec, kWaves, kSteps, kGated, true>(A, G, at, n, lds);
  else
    forward_tile<T, kVec, kWaves, kSteps, kGated, false>(A, G, at, n, lds);
}

template <int kWaves, bool kChained>
struct SharedBackward {
  Stretch parts[kWaves][64], back[kWaves][64];
  std::conditional_t<kChained, Before<1, kWaves>, Nothing> before;
  uint32_t ticket;
};

template <typename T, int kWaves, int kSteps, bool kGated, bool kWhole>
__device__ __forceinline__ void backward_tile(const RecurrenceArgs& A, const RecurrenceGradArgs& D, const TileArgs& G, const Place& at, uint32_t n,
                                              SharedBackward<kWaves, chained(kWaves, kSteps)>& lds) {
  constexpr uint32_t kTile = kWaves * kSteps;
  static_assert(kTile == kChunk || kTile <= kOneTile, "a tile begins with a kept state, the only one of a short sequence with the first");
  auto& parts = lds.parts;
  auto& back = lds.back;
  const uint32_t wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63u, b = at.b;
  const Lane<1> mine(at.block, A.width);
  const uint32_t offset = mine.c * static_cast<uint32_t>(sizeof(T));
  const uint32_t tile = G.tiles - 1u - at.order;                     // the last tile first
  const uint32_t first = tile * kTile + wave * kSteps;
  const uint32_t valid = kWhole ? kSteps : n > first ? min(n - first, static_cast<uint32_t>(kSteps)) : 0u;
  const uint64_t state_at = static_cast<uint64_t>(b) * A.width + mine.c;
  Raw<T, 1> read_x[kSteps], v[kSteps], w[kSteps], dy[kSteps];
  if (kWhole || valid > 0u) {
    read_steps<T, 1, kSteps, kWhole>(v, A.gate, b, first, n, offset);
    read_steps<T, 1, kSteps, kWhole>(read_x, A.x, b, first, n, offset);
    if constexpr (kGated) read_steps<T, 1, kSteps, kWhole>(w, A.out_gate, b, first, n, offset);
    read_steps<T, 1, kSteps, kWhole>(dy, D.dy, b, first, n, offset);
  }
  const uint32_t anew = resets_of<kSteps>(A, b, first, n);
  const uint32_t chunks = (A.steps + kChunk - 1u) / kChunk;
  float h = chunks > 0u ? A.states[(static_cast<uint64_t>(b) * chunks + tile) * A.width + mine.c] : 0.0f;
  float carry[1] = {at.order == 0u && D.dh_last ? D.dh_last[state_at] : 0.0f};

  // e: the gradient that y brings to the state; shut: 1 - o
  float f[kSteps], take[kSteps], x[kSteps], e[kSteps], shut[kSteps];
#pragma unroll
  for (uint32_t r = 0; r < kSteps; ++r) {
    gate_of(static_cast<float>(v[r].v[0]), f[r], take[r]);
    x[r] = static_cast<float>(read_x[r].v[0]);
    if (!kWhole && r >= valid) f[r] = 1.0f, take[r] = 0.0f, x[r] = 0.0f;
  }
#pragma unroll
  for (uint32_t r = 0; r < kSteps; ++r) {
    e[r] = static_cast<float>(dy[r].v[0]);
    if constexpr (kGated) {
      float open;
      gate_of(static_cast<float>(w[r].v[0]), open, shut[r]);
      e[r] *= open;
    }
    if (!kWhole && r >= valid) e[r] = 0.0f;
  }
  // (Held as they are: the compiler would rather keep each one's power and reciprocal for later, which is twice the registers.)
#pragma unroll
  for (uint32_t r = 0; r < kSteps; ++r) {
    asm volatile("" : "+v"(f[r]), "+v"(take[r]), "+v"(x[r]), "+v"(e[r]));
    if constexpr (kGated) asm volatile("" : "+v"(shut[r]));
  }
  Stretch own, rear;                 // rear: from the gradient that comes in behind the steps to the one that leaves before them
  auto scan = [&](auto with_resets) __attribute__((always_inline)) {
    own = rear = Stretch{1.0f, 0.0f};
#pragma unroll
    for (uint32_t r = 0; r < kSteps; ++r) {
      if (with_resets && ((anew >> r) & 1u) != 0u) own = Stretch{-0.0f, 0.0f};
      own.h = __fmaf_rn(f[r], own.h, take[r] * x[r]);
      own.p *= f[r];
    }
#pragma unroll
    for (uint32_t r = kSteps; r-- > 0u;) {
      rear.h = f[r] * (e[r] + rear.h);
      rear.p *= f[r];
      if (with_resets && ((anew >> r) & 1u) != 0u) rear = Stretch{-0.0f, 0.0f};
    }
  };
  if constexpr (kWaves > 1) {
    if (anew == 0u) scan(No{}); else scan(Yes{});
    parts[wave][lane] = own;
    back[wave][lane] = rear;
    __syncthreads();
  }
  if constexpr (chained(kWaves, kSteps)) {
    if (G.tiles > 1u) {
      Stretch whole[1];
      if (wave == 0u) {
        whole[0] = back[kWaves - 1][lane];
#pragma unroll 4
        for (uint32_t j = kWaves - 1u; j-- > 0u;) whole[0] = both(whole[0], back[j][lane]);
      }
      come_in<1, kWaves>(G, at, wave, whole, lds.before, carry);
    }
  }
#pragma unroll 4
  for (uint32_t j = 0; j < wave; ++j) h = after(parts[j][lane], h);
  float g = carry[0];
#pragma unroll 4
  for (uint32_t j = kWaves - 1u; j > wave; --j) g = after(back[j][lane], g);
  float before[kSteps];              // the state before the step
  const uint32_t behind = kWhole ? kSteps : A.steps > first ? min(A.steps - first, static_cast<uint32_t>(kSteps)) : 0u;
  Rows<T> to_out(D.dout_gate, b, first), to_x(D.dx, b, first + kSteps - 1u), to_gate(D.dgate, b, first + kSteps - 1u);
#pragma unroll
  for (uint32_t r = 0; r < kSteps; ++r) asm volatile("" : "+v"(x[r]));      // (keeps take * x from being held in sixteen more registers)
  auto finish = [&](auto with_resets) __attribute__((always_inline)) {
#pragma unroll
    for (uint32_t r = 0; r < kSteps; ++r, to_out.p += to_out.step) {
      if (with_resets && ((anew >> r) & 1u) != 0u) h = 0.0f;
      before[r] = h;
      h = __fmaf_rn(f[r], h, take[r] * x[r]);
      if constexpr (kGated) {
        const float dout[1] = {kWhole || r < valid ? shut[r] * e[r] * h : 0.0f};
        if (kWhole || r < behind) store<T, 1, kWhole>(to_out.p, mine, dout);
      }
    }
#pragma unroll
    for (uint32_t r = kSteps; r-- > 0u; to_x.p -= to_x.step, to_gate.p -= to_gate.step) {
      const float d = e[r] + g;      // the gradient of the state after the step
      float dx[1] = {d * take[r]}, dgate[1] = {d * take[r] * (before[r] - x[r]) * f[r]};
      if (!kWhole && r >= valid) dx[0] = dgate[0] = 0.0f;
      g = f[r] * d;
      if (with_resets && ((anew >> r) & 1u) != 0u) g = 0.0f;
      if (kWhole || r < behind) {
        store<T, 1, kWhole>(to_x.p, mine, dx);
        store<T, 1, kWhole>(to_gate.p, mine, dgate);
      }
    }
  };
  if (anew == 0u) finish(No{}); else finish(Yes{});
  if (D.dh0 && tile == 0u && wave == 0u && mine.all) D.dh0[state_at] = g;
}

template <typename T, int kWaves, int kSteps, bool kGated>
__global__ void __launch_bounds__(64 * kWaves) recurrence_backward_kernel(RecurrenceArgs A, RecurrenceGradArgs D, TileArgs G) {
  __shared__ SharedBackward<kWaves, chained(kWaves, kSteps)> lds;
  const Place at = take_place<chained(kWaves, kSteps)>(A, G, &lds.ticket);
  const uint32_t n = length_of(A, at.b);
  if ((G.tiles - at.order) * (kWaves * kSteps) <= n && (at.block + 1u) * 64u <= A.width)
    backward_tile<T, kWaves, kSteps, kGated, true>(A, D, G, at, n, lds);
  else
    backward_tile<T, kWaves, kSteps, kGated, false>(A, D, G, at, n, lds);
}

__global__ void __launch_bounds__(256) clear_words_kernel(TileArgs G, uint64_t words) {
  typedef unsigned long long two __attribute__((ext_vector_type(2)));
  two* to = reinterpret_cast<two*>(G.words);                         // (scratch begins on 256 bytes, and a chain has an even number of words)
  const uint64_t pairs = words / 2u, threads = static_cast<uint64_t>(gridDim.x) * 256u;
  for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256u + threadIdx.x; i < pairs; i += threads) to[i] = two{kUnset, kUnset};
  if (blockIdx.x == 0u && threadIdx.x == 0u) *G.ticket = 0u;
}

struct Cut {
  Kind kind;
  uint32_t vec;                    // channels a lane
};

constexpr Shape shape_of(Kind kind, bool backward) {
  return kind == Kind::kOneWave ? kOneWave : kind == Kind::kShort ? kShort : kind == Kind::kMiddle ? kMiddle : backward ? kLongBackward : kLong;
}

Cut cut_of(const RecurrenceArgs& a, int dtype, bool backward) {
  Cut c;
  c.vec = !backward && dtype != 0 && a.width > 64u ? 2u : 1u;
  c.kind = a.steps <= kOneWave.tile() ? Kind::kOneWave : a.steps <= kShort.tile() ? Kind::kShort : a.steps <= kMiddle.tile() ? Kind::kMiddle : Kind::kLong;
  return c;
}

TileArgs tiles_of(const RecurrenceArgs& a, const Cut& c, bool backward) {
  TileArgs G{};
  G.across = (a.width + 64u * c.vec - 1u) / (64u * c.vec);
  const uint32_t tile = shape_of(c.kind, backward).tile();
  G.tiles = a.steps == 0u ? 1u : (a.steps + tile - 1u) / tile;
  G.groups = (G.tiles - 1u) / kGroup;
  return G;
}

uint64_t words_for(const RecurrenceArgs& a, const Cut& c, const TileArgs& G) {
  return G.tiles > 1u ? static_cast<uint64_t>(a.batch) * G.across * (uint64_t(G.tiles) + G.groups) * 64u * c.vec : 0u;
}

uint64_t workgroups(const RecurrenceArgs& a, const TileArgs& G) { return static_cast<uint64_t>(a.batch) * G.across * G.tiles; }

hipError_t clear_words(TileArgs& G, uint64_t words, unsigned long long* scratch, hipStream_t s) {
  if (words == 0u) return hipSuccess;
  G.words = scratch;
  G.ticket = reinterpret_cast<uint32_t*>(scratch + words);
  const uint64_t wgs = (words / 2u + 1023u) / 1024u;                  // four pairs a thread, up to a grid that fills the device twice over
  clear_words_kernel<<<dim3(static_cast<uint32_t>(wgs < 2048u ? wgs : 2048u)), dim3(256), 0, s>>>(G, words);
  return hipGetLastError();
}

template <typename T, int kVec, bool kGated, uint32_t kWaves, uint32_t kSteps>
void launch_forward(const RecurrenceArgs& a, const TileArgs& G, uint32_t wgs, hipStream_t s) {
  recurrence_kernel<T, kVec, kWaves, kSteps, kGated><<<dim3(wgs), dim3(64u * kWaves), 0, s>>>(a, G);
}
template <typename T, int kVec, bool kGated>
void launch_forward(const RecurrenceArgs& a, const Cut& c, const TileArgs& G, uint32_t wgs, hipStream_t s) {
  if (c.kind == Kind::kOneWave) launch_forward<T, kVec, kGated, kOneWave.waves, kOneWave.steps>(a, G, wgs, s);
  else if (c.kind == Kind::kShort) launch_forward<T, kVec, kGated, kShort.waves, kShort.steps>(a, G, wgs, s);
  else if (c.kind == Kind::kMiddle) launch_forward<T, kVec, kGated, kMiddle.waves, kMiddle.steps>(a, G, wgs, s);
  else launch_forward<T, kVec, kGated, kLong.waves, kLong.steps>(a, G, wgs, s);
}

template <typename T, bool kGated, uint32_t kWaves, uint32_t kSteps>
void launch_backward(const RecurrenceArgs& a, const RecurrenceGradArgs& d, const TileArgs& G, uint32_t wgs, hipStream_t s) {
  recurrence_backward_kernel<T, kWaves, kSteps, kGated><<<dim3(wgs), dim3(64u * kWaves), 0, s>>>(a, d, G);
}
template <typename T, bool kGated>
void launch_backward(const RecurrenceArgs& a, const RecurrenceGradArgs& d, const Cut& c, const TileArgs& G, uint32_t wgs, hipStream_t s) {
  if (c.kind == Kind::kOneWave) launch_backward<T, kGated, kOneWave.waves, kOneWave.steps>(a, d, G, wgs, s);
  else if (c.kind == Kind::kShort) launch_backward<T, kGated, kShort.waves, kShort.steps>(a, d, G, wgs, s);
  else if (c.kind == Kind::kMiddle) launch_backward<T, kGated, kMiddle.waves, kMiddle.steps>(a, d, G, wgs, s);
  else launch_backward<T, kGated, kLongBackward.waves, kLongBackward.steps>(a, d, G, wgs, s);
}

// One of the two template arguments a run decides.
template <typename T, typename F>
void by_gate(const RecurrenceArgs& a, F&& f) {
  if (a.out_gate.data) f(T{}, Yes{}); else f(T{}, No{});
}

}  // namespace

// A grid has fewer than 2^32 threads (and tickets are 32 bits).
bool recurrence_fits_grid(const RecurrenceArgs& a, int dtype, bool backward) {
  const Cut c = cut_of(a, dtype, backward);
  return workgroups(a, tiles_of(a, c, backward)) <= 0xFFFFFFFFull / (64u * shape_of(c.kind, backward).waves);
}

uint64_t recurrence_scratch_words(const RecurrenceArgs& a, int dtype, bool backward) {
  const Cut c = cut_of(a, dtype, backward);
  const uint64_t words = words_for(a, c, tiles_of(a, c, backward));
  return words ? words + 1u : 0u;
}

hipError_t launch_recurrence(const RecurrenceArgs& a, int dtype, unsigned long long* scratch, uint32_t looks, hipStream_t s) {
  const Cut c = cut_of(a, dtype, false);
  TileArgs G = tiles_of(a, c, false);
  G.looks = looks;
  const uint32_t wgs = static_cast<uint32_t>(workgroups(a, G));
  const hipError_t e = clear_words(G, words_for(a, c, G), scratch, s);
  if (e != hipSuccess) return e;
  auto launch = [&](auto type, auto gated) {
    using T = decltype(type);
    constexpr bool kGated = decltype(gated){};
    if constexpr (sizeof(T) == 2) {
      if (c.vec == 2u) return launch_forward<T, 2, kGated>(a, c, G, wgs, s);
    }
    launch_forward<T, 1, kGated>(a, c, G, wgs, s);
  };
  if (dtype == 0) by_gate<float>(a, launch);
  else if (dtype == 1) by_gate<__bf16>(a, launch);
  else by_gate<_Float16>(a, launch);
  return hipGetLastError();
}

hipError_t launch_recurrence_backward(const RecurrenceArgs& a, const RecurrenceGradArgs& g, int dtype, unsigned long long* scratch, uint32_t looks, hipStream_t s) {
  const Cut c = cut_of(a, dtype, true);
  TileArgs G = tiles_of(a, c, true);
  G.looks = looks;
  const uint32_t wgs = static_cast<uint32_t>(workgroups(a, G));
  const hipError_t e = clear_words(G, words_for(a, c, G), scratch, s);
  if (e != hipSuccess) return e;
  auto launch = [&](auto type, auto gated) { launch_backward<decltype(type), bool(decltype(gated){})>(a, g, c, G, wgs, s); };
  if (dtype == 0) by_gate<float>(a, launch);
  else if (dtype == 1) by_gate<__bf16>(a, launch);
  else by_gate<_Float16>(a, launch);
  return hipGetLastError();
}

}  // namespace rgc
