// Host check of rgc_stretch.h: the state that follows from published words has the same bits whichever of them were states already when
// they were met, and those of the states one after the other.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <random>
#include <vector>

#include "../paper_1808_04357_amd/csrc/rgc_stretch.h"

using namespace rgc;

namespace {

uint32_t bits(float f) {
  if (f != f) return 0x7FC00000u;
  uint32_t b;
  std::memcpy(&b, &f, 4);
  return b;
}

int faults = 0;

// `steps` steps a stretch; slope: the gates' (the larger, the longer a state is kept); odd: which unusual things occur.
void check(uint32_t stretches, uint32_t steps, double slope, int odd, uint32_t seed) {
  std::mt19937 rng(seed);
  std::normal_distribution<double> normal;
  std::vector<uint64_t> own(stretches), states(stretches);
  float c = static_cast<float>(normal(rng));
  for (uint32_t t = 0; t < stretches; ++t) {
    Stretch s{1.0f, 0.0f};
    for (uint32_t i = 0; i < steps; ++i) {
      float f = static_cast<float>(1.0 / (1.0 + std::exp(-(slope + normal(rng))))), x = static_cast<float>(normal(rng));
      const uint32_t what = odd ? rng() % (steps * 6u) : 9u;
      if (odd == 1 && what == 0u) s = Stretch{-0.0f, 0.0f};                                   // starts anew
      if (odd == 2 && what == 0u) x = std::numeric_limits<float>::quiet_NaN();
      if (odd == 2 && what == 1u) f = -std::numeric_limits<float>::quiet_NaN();
      if (odd == 3 && what == 0u) x = std::numeric_limits<float>::infinity();
      if (odd == 3 && what == 1u) f = 0.0f;
      s.h = std::fmaf(f, s.h, (1.0f - f) * x);
      s.p *= f;
    }
    own[t] = word_of(s);
    c = after(s, c);
    states[t] = word_of(state_of(c));
    if (own[t] == kUnset || states[t] == kUnset) ++faults;
  }
  for (uint32_t order = 1; order < stretches; ++order) {
    const float want = stretch_of(states[order - 1]).h;
    for (int mix = 0; mix < 64; ++mix) {
      // words from the first state met on; the first one is a state at once
      const uint32_t n = 1u + rng() % order;
      auto back = [&](uint32_t j) {
        const uint32_t t = order - 1u - j;
        const bool state = t == 0u || j == n - 1u || (mix > 0 && (mix == 1 || rng() % 3u == 0u));
        return stretch_of(state ? states[t] : own[t]);
      };
      const float got = mix % 2 ? state_behind<1>(n, back) : state_behind<4>(n, back);
      if (bits(got) != bits(want)) ++faults;
    }
  }
}

}  // namespace

int main() {
  for (uint32_t seed = 0; seed < 300; ++seed)
    for (double slope : {-2.0, 0.0, 4.0, 7.5})
      for (int odd = 0; odd < 4; ++odd) check(24, 16, slope, odd, seed * 97u + static_cast<uint32_t>(odd));
  for (uint32_t seed = 0; seed < 200; ++seed) check(60, 128, 7.5, 0, 100000u + seed);
  // a stretch and its word
  const Stretch s{0.25f, -3.0f};
  if (stretch_of(word_of(s)).p != s.p || stretch_of(word_of(s)).h != s.h || !cut(state_of(1.0f).p) || cut(0.0f)) ++faults;
  if (faults) {
    std::printf("%d faults\n", faults);
    return 1;
  }
  std::printf("stretches_check ok\n");
  return 0;
}
