// What the tiles of a long recurrence tell each other, and how a tile makes of it the state that it begins with.  No HIP in here: the host tests
// compile it by itself.
//
// A stretch of steps takes the state h before it to P h + H after it.  The sign bit of P says that nothing from before enters at all (a state that
// started anew, a published state): P h is not even formed there, h may be NaN.
#pragma once

#include <stdint.h>

namespace rgc {

struct Stretch {
  float p, h;
};

constexpr bool cut(float p) { return (__builtin_bit_cast(uint32_t, p) & 0x80000000u) != 0u; }
constexpr float after(const Stretch& s, float h) { return cut(s.p) ? s.h : __builtin_fmaf(s.p, h, s.h); }
// `first`, then `second`.
constexpr Stretch both(const Stretch& first, const Stretch& second) {
  return Stretch{cut(first.p) || cut(second.p) ? -0.0f : first.p * second.p, after(second, first.h)};
}
// A state: what comes before it no longer matters.
constexpr Stretch state_of(float h) { return Stretch{-0.0f, h}; }

constexpr uint64_t kUnset = ~0ull;      // a word that is not published yet (its upper half would be a NaN as P, which is never published)
constexpr uint64_t kLost = 0x800000007FC00000ull;       // in the place of one that never came: the state is a NaN

// A NaN among the gates or states: NaN whatever comes before, and one NaN as good as another.
constexpr uint64_t word_of(const Stretch& s) {
  const bool broken = s.p != s.p || s.h != s.h;
  const uint32_t p = broken ? 0x80000000u : __builtin_bit_cast(uint32_t, s.p), h = broken ? 0x7FC00000u : __builtin_bit_cast(uint32_t, s.h);
  return (static_cast<uint64_t>(p) << 32) | h;
}
constexpr Stretch stretch_of(uint64_t word) {
  return Stretch{__builtin_bit_cast(float, static_cast<uint32_t>(word >> 32)), __builtin_bit_cast(float, static_cast<uint32_t>(word))};
}

// The state behind n stretches that follow each other, the first of them a state; back(j): the j-th from the end.
// A group's word is the stretch of its tiles first and the state behind them later, and which of the two is met is a matter of time.  It makes no difference here:
// from a state on, each stretch is applied to the state before it, just as the tile that published it does to come to the state that it publishes.  (Joining the
// stretches to one on the way would round otherwise: (P2 P1) c + (P2 H1 + H2) is not P2 (P1 c + H1) + H2 to the last bit.)
// h: the state before them, where the first is none.  (kAtOnce of them are asked for before one is needed.)
template <uint32_t kAtOnce, typename Back>
constexpr float state_behind(uint32_t n, Back&& back, float h = 0.0f) {
  for (; n % kAtOnce != 0u; --n) h = after(back(n - 1u), h);
  for (; n > 0u; n -= kAtOnce) {
    Stretch s[kAtOnce] = {};
    for (uint32_t i = 0; i < kAtOnce; ++i) s[i] = back(n - 1u - i);
    for (uint32_t i = 0; i < kAtOnce; ++i) h = after(s[i], h);
  }
  return h;
}

}  // namespace rgc
