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
// Tiles are handed out by a ticket, all chains' first tiles, then all second ones: a tile publishes its (P, H) as soon as it has it, and the
// state it ends with (which is a stretch with P = 0) when it knows that, and looks back over the published ones until it has come to such a
// state.  It waits for tiles of smaller tickets only, and a ticket is taken by a workgroup that runs, so the smallest ticket not done
// waits for nothing: every wait ends, however few workgroups run at a time.
//
// The sign bit of P says that nothing from before enters at all (a state that started anew, a published state): P h is not even formed there, h may be NaN.
//
// 1 - sigmoid(v) is computed as sigmoid(-v), which keeps its precision where the gate is nearly open.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rgc_lm.h"

namespace rgc {
namespace {

constexpr uint32_t kChunk = 256;       // steps between kept states (RGC_RECURRENCE_CHUNK)
constexpr float kLog2e = 1.44269504088896341f;
constexpr unsigned long long kUnset = ~0ull;      // a word that is not published yet (its upper half would be a NaN as P, which is never published)

struct Stretch {
  float p, h;
};

__device__ __forceinline__ bool cut(float p) { return __float_as_int(p) < 0; }
__device__ __forceinline__ float after(const Stretch& s, float h) { return cut(s.p) ? s.h : __fmaf_rn(s.p, h, s.h); }
// `first`, then `second`.
__device__ __forceinline__ Stretch both(const Stretch& first, const Stretch& second) {
  return Stretch{cut(first.p) || cut(second.p) ? -0.0f : first.p * second.p, after(second, first.h)};
}

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

template <typename T, int kVec>
__device__ __forceinline__ Raw<T, kVec> read(const T* p) {
  if constexpr (sizeof(T) * kVec == 4) {
    const uint32_t w = *reinterpret_cast<const word*>(p);
    Raw<T, kVec> r;
    __builtin_memcpy(&r, &w, 4);
    return r;
  } else {
    return *reinterpret_cast<const Raw<T, kVec>*>(p);
  }
}

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

template <typename T, int kVec>
__device__ __forceinline__ void store(T* row, const Lane<kVec>& lane, const float (&v)[kVec]) {
  if (lane.all) {
    Raw<T, kVec> r;
#pragma unroll
    for (int i = 0; i < kVec; ++i) r.v[i] = static_cast<T>(v[i]);
    if constexpr (sizeof(T) * kVec == 4) {
      uint32_t w;
      __builtin_memcpy(&w, &r, 4);
      *reinterpret_cast<word*>(row + lane.c) = w;
    } else {
      *reinterpret_cast<Raw<T, kVec>*>(row + lane.c) = r;
    }
  } else if (lane.last) {
    row[lane.c + kVec - 1] = static_cast<T>(v[kVec - 1]);
  }
}
template <int kVec>
__device__ __forceinline__ void store_state(float* row, const Lane<kVec>& lane, const float (&v)[kVec]) {
#pragma unroll
  for (int i = 0; i < kVec; ++i)
    if (lane.all || (lane.last && i == kVec - 1)) row[lane.c + i] = v[i];
}

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }

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

template <typename T>
__device__ __forceinline__ T* row_at(const SequenceView& v, uint32_t b, uint32_t t) {
  return static_cast<T*>(v.data) + (b * v.batch_stride + t * v.step_stride);
}

// Which tile this workgroup works on: by ticket where tiles wait for each other.
struct Place {
  uint32_t chain, b, block, order;      // order: how many tiles of the chain come before it
};
__device__ __forceinline__ Place take_place(const RecurrenceArgs& A, const TileArgs& G, uint32_t* lds) {
  uint32_t ticket = blockIdx.x;
  if (G.tiles > 1u) {
    if (threadIdx.x == 0u) *lds = atomicAdd(G.ticket, 1u);
    __syncthreads();
    ticket = uniform(*lds);
  }
  const uint32_t chains = A.batch * G.across;
  Place p;
  p.order = ticket / chains;
  p.chain = ticket - p.order * chains;
  p.b = p.chain / G.across;
  p.block = p.chain - p.b * G.across;
  return p;
}

template <int kVec>
__device__ __forceinline__ unsigned long long* words_of(const TileArgs& G, uint32_t chain, uint32_t order) {
  return G.words + (static_cast<uint64_t>(chain) * G.tiles + order) * (64u * kVec) + (threadIdx.x & 63u) * kVec;
}

template <int kVec>
__device__ __forceinline__ void publish(unsigned long long* w, const Stretch (&s)[kVec]) {
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const bool broken = s[i].p != s[i].p;                            // a NaN among the gates: NaN whatever comes before
    const uint32_t p = __float_as_uint(broken ? -0.0f : s[i].p), h = __float_as_uint(broken ? s[i].p : s[i].h);
    __hip_atomic_store(w + i, (static_cast<unsigned long long>(p) << 32) | h, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

// What comes into the tile, from the published words of the chain's earlier tiles: kWaves of them at a time, a wave each.
// (A word carries all there is to know, so no other memory needs ordering.)  lds: as `parts` of the kernels.
template <int kVec, int kWaves>
__device__ __forceinline__ void look_back(const TileArgs& G, const Place& at, uint32_t wave, Stretch (*lds)[64 * kVec], float (&carry)[kVec]) {
  const uint32_t lane = threadIdx.x & 63u;
  Stretch seen[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) seen[i] = Stretch{1.0f, 0.0f};
  for (uint32_t next = at.order; next > 0u;) {                       // tiles next - 1, next - 2, ..
    if (wave < next) {
      const unsigned long long* w = words_of<kVec>(G, at.chain, next - 1u - wave);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        unsigned long long v = __hip_atomic_load(w + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        while (v == kUnset) {
          __builtin_amdgcn_s_sleep(1);
          v = __hip_atomic_load(w + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        lds[wave][lane * kVec + i] = Stretch{__uint_as_float(static_cast<uint32_t>(v >> 32)), __uint_as_float(static_cast<uint32_t>(v))};
      }
    }
    __syncthreads();
    bool open = false;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      for (uint32_t j = 0; j < kWaves && j < next; ++j) seen[i] = both(lds[j][lane * kVec + i], seen[i]);
      open |= !cut(seen[i].p);
    }
    // the same in every wave, which all have the same words (the first tile's word is a state, so it ends there at the latest)
    if (!__any(open)) break;
    next = next > kWaves ? next - kWaves : 0u;
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i) carry[i] = seen[i].h;
}

template <typename T, int kVec, int kWaves, int kSteps>
__global__ void __launch_bounds__(64 * kWaves) recurrence_kernel(RecurrenceArgs A, TileArgs G) {
  constexpr uint32_t kTile = kWaves * kSteps;
  __shared__ Stretch parts[kWaves][64 * kVec];
  __shared__ Stretch earlier[kWaves][64 * kVec];
  __shared__ uint32_t lds_ticket;
  const Place at = take_place(A, G, &lds_ticket);
  const uint32_t wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63u, b = at.b;
  const Lane<kVec> mine(at.block, A.width);
  const uint32_t n = length_of(A, b);
  const uint32_t first = at.order * kTile + wave * kSteps;           // this wave's steps
  const uint32_t valid = n > first ? min(n - first, static_cast<uint32_t>(kSteps)) : 0u;
  const uint32_t anew = resets_of<kSteps>(A, b, first, n);

  Raw<T, kVec> x[kSteps], v[kSteps], w[kSteps];
#pragma unroll
  for (uint32_t r = 0; r < kSteps; ++r)
    if (r < valid) {
      v[r] = read<T, kVec>(row_at<T>(A.gate, b, first + r) + mine.c);
      x[r] = read<T, kVec>(row_at<T>(A.x, b, first + r) + mine.c);
    }
  if (A.out_gate.data) {
#pragma unroll
    for (uint32_t r = 0; r < kSteps; ++r)
      if (r < valid) w[r] = read<T, kVec>(row_at<T>(A.out_gate, b, first + r) + mine.c);
  }
  float carry[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) carry[i] = at.order == 0u && A.h0 ? A.h0[static_cast<uint64_t>(b) * A.width + mine.c + i] : 0.0f;

  float f[kSteps][kVec], u[kSteps][kVec];
  Stretch own[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) own[i] = Stretch{1.0f, 0.0f};
#pragma unroll
  for (uint32_t r = 0; r < kSteps; ++r)
    if (r < valid) {
      const bool starts = (anew >> r) & 1u;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        float take;
        gate_of(static_cast<float>(v[r].v[i]), f[r][i], take);
        u[r][i] = take * static_cast<float>(x[r].v[i]);
        if (starts) own[i] = Stretch{-0.0f, 0.0f};
        own[i].h = __fmaf_rn(f[r][i], own[i].h, u[r][i]);
        own[i].p *= f[r][i];
      }
    }
  if constexpr (kWaves > 1) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) parts[wave][lane * kVec + i] = own[i];
    __syncthreads();
  }
  if (G.tiles > 1u) {
    Stretch whole[kVec];
    if (wave == 0u) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        whole[i] = own[i];
        for (uint32_t j = 1; j < kWaves; ++j) whole[i] = both(whole[i], parts[j][lane * kVec + i]);
      }
      if (at.order > 0u && at.order + 1u < G.tiles) publish<kVec>(words_of<kVec>(G, at.chain, at.order), whole);
    }
    if (at.order > 0u) look_back<kVec, kWaves>(G, at, wave, earlier, carry);
    if (wave == 0u && at.order + 1u < G.tiles) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) whole[i] = Stretch{-0.0f, after(whole[i], carry[i])};
      publish<kVec>(words_of<kVec>(G, at.chain, at.order), whole);
    }
  }
  if (A.states && A.steps > 0u && wave == 0u && (at.order * kTile) % kChunk == 0u) {
    const uint32_t chunks = (A.steps + kChunk - 1u) / kChunk;
    store_state<kVec>(A.states + (static_cast<uint64_t>(b) * chunks + at.order * kTile / kChunk) * A.width, mine, carry);
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i)
    for (uint32_t j = 0; j < wave; ++j) carry[i] = after(parts[j][lane * kVec + i], carry[i]);
#pragma unroll
  for (uint32_t r = 0; r < kSteps; ++r) {
    if (r < valid) {
      float y[kVec];
      const bool starts = (anew >> r) & 1u;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        if (starts) carry[i] = 0.0f;
        carry[i] = __fmaf_rn(f[r][i], carry[i], u[r][i]);
        y[i] = carry[i];
        if (A.out_gate.data) {
          float open, shut;
          gate_of(static_cast<float>(w[r].v[i]), open, shut);
          y[i] *= open;
        }
      }
      store<T, kVec>(row_at<T>(A.y, b, first + r), mine, y);
    } else if (first + r < A.steps) {
      const float zero[kVec] = {};
      store<T, kVec>(row_at<T>(A.y, b, first + r), mine, zero);
    }
  }
  if (A.h_last && at.order + 1u == G.tiles && wave + 1u == kWaves) store_state<kVec>(A.h_last + static_cast<uint64_t>(b) * A.width, mine, carry);
}

template <typename T, int kWaves, int kSteps>
__global__ void __launch_bounds__(64 * kWaves) recurrence_backward_kernel(RecurrenceArgs A, RecurrenceGradArgs D, TileArgs G) {
  constexpr uint32_t kTile = kWaves * kSteps;
  static_assert(kTile <= kChunk, "a tile begins with a kept state");
  __shared__ Stretch parts[kWaves][64], back[kWaves][64];
  __shared__ Stretch earlier[kWaves][64];
  __shared__ uint32_t lds_ticket;
  const Place at = take_place(A, G, &lds_ticket);
  const uint32_t wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63u, b = at.b;
  const Lane<1> mine(at.block, A.width);
  const uint32_t n = length_of(A, b);
  const uint32_t tile = G.tiles - 1u - at.order;                     // the last tile first
  const uint32_t first = tile * kTile + wave * kSteps;
  const uint32_t valid = n > first ? min(n - first, static_cast<uint32_t>(kSteps)) : 0u;
  const uint32_t anew = resets_of<kSteps>(A, b, first, n);
  const uint64_t state_at = static_cast<uint64_t>(b) * A.width + mine.c;

  T x[kSteps], v[kSteps], w[kSteps], dy[kSteps];
#pragma unroll
  for (uint32_t r = 0; r < kSteps; ++r)
    if (r < valid) {
      v[r] = row_at<T>(A.gate, b, first + r)[mine.c];
      x[r] = row_at<T>(A.x, b, first + r)[mine.c];
    }
#pragma unroll
  for (uint32_t r = 0; r < kSteps; ++r)
    if (r < valid) dy[r] = row_at<T>(D.dy, b, first + r)[mine.c];
  if (A.out_gate.data) {
#pragma unroll
    for (uint32_t r = 0; r < kSteps; ++r)
      if (r < valid) w[r] = row_at<T>(A.out_gate, b, first + r)[mine.c];
  }
  const uint32_t chunks = (A.steps + kChunk - 1u) / kChunk;
  float h = chunks > 0u ? A.states[(static_cast<uint64_t>(b) * chunks + tile) * A.width + mine.c] : 0.0f;
  float carry[1] = {at.order == 0u && D.dh_last ? D.dh_last[state_at] : 0.0f};

  // e: the gradient that y brings to the state; shut: 1 - o
  float f[kSteps], take[kSteps], e[kSteps], shut[kSteps];
  Stretch own{1.0f, 0.0f};
#pragma unroll
  for (uint32_t r = 0; r < kSteps; ++r)
    if (r < valid) {
      gate_of(static_cast<float>(v[r]), f[r], take[r]);
      if ((anew >> r) & 1u) own = Stretch{-0.0f, 0.0f};
      own.h = __fmaf_rn(f[r], own.h, take[r] * static_cast<float>(x[r]));
      own.p *= f[r];
      e[r] = static_cast<float>(dy[r]);
      if (A.out_gate.data) {
        float open;
        gate_of(static_cast<float>(w[r]), open, shut[r]);
        e[r] *= open;
      }
    }
  Stretch rear{1.0f, 0.0f};                                          // from the gradient that comes in behind the steps to the one that leaves before them
#pragma unroll
  for (uint32_t r = kSteps; r-- > 0u;)
    if (r < valid) {
      rear.h = f[r] * (e[r] + rear.h);
      rear.p *= f[r];
      if ((anew >> r) & 1u) rear = Stretch{-0.0f, 0.0f};
    }
  if constexpr (kWaves > 1) {
    parts[wave][lane] = own;
    back[wave][lane] = rear;
    __syncthreads();
  }
  if (G.tiles > 1u) {
    Stretch whole[1];
    if (wave == 0u) {
      whole[0] = back[kWaves - 1][lane];
      for (uint32_t j = kWaves - 1u; j-- > 0u;) whole[0] = both(whole[0], back[j][lane]);
      if (at.order > 0u && at.order + 1u < G.tiles) publish<1>(words_of<1>(G, at.chain, at.order), whole);
    }
    if (at.order > 0u) look_back<1, kWaves>(G, at, wave, earlier, carry);
    if (wave == 0u && at.order + 1u < G.tiles) {
      whole[0] = Stretch{-0.0f, after(whole[0], carry[0])};
      publish<1>(words_of<1>(G, at.chain, at.order), whole);
    }
  }
  for (uint32_t j = 0; j < wave; ++j) h = after(parts[j][lane], h);
  float g = carry[0];
  for (uint32_t j = kWaves - 1u; j > wave; --j) g = after(back[j][lane], g);
  float before[kSteps];
#pragma unroll
  for (uint32_t r = 0; r < kSteps; ++r)
    if (r < valid) {
      if ((anew >> r) & 1u) h = 0.0f;
      before[r] = h;
      h = __fmaf_rn(f[r], h, take[r] * static_cast<float>(x[r]));
    }
#pragma unroll
  for (uint32_t r = kSteps; r-- > 0u;) {
    float dx[1] = {0.0f}, dgate[1] = {0.0f}, dout[1] = {0.0f};
    if (r < valid) {
      const float d = e[r] + g, xr = static_cast<float>(x[r]);
      dx[0] = d * take[r];
      dgate[0] = dx[0] * (before[r] - xr) * f[r];
      if (A.out_gate.data) dout[0] = e[r] * shut[r] * __fmaf_rn(f[r], before[r], take[r] * xr);
      g = (anew >> r) & 1u ? 0.0f : f[r] * d;
    }
    if (first + r < A.steps) {
      store<T, 1>(row_at<T>(D.dx, b, first + r), mine, dx);
      store<T, 1>(row_at<T>(D.dgate, b, first + r), mine, dgate);
      if (A.out_gate.data) store<T, 1>(row_at<T>(D.dout_gate, b, first + r), mine, dout);
    }
  }
  if (D.dh0 && tile == 0u && wave == 0u && mine.all) D.dh0[state_at] = g;
}

__global__ void __launch_bounds__(256) clear_words_kernel(TileArgs G, uint64_t words) {
  const uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256u + threadIdx.x;
  if (i < words) G.words[i] = kUnset;
  if (i == 0u) *G.ticket = 0u;
}

struct Cut {
  uint32_t vec, waves, steps;      // channels a lane, waves a workgroup, steps a wave
};

Cut cut_of(const RecurrenceArgs& a, int dtype, bool backward) {
  Cut c;
  c.vec = !backward && dtype != 0 && a.width > 64u ? 2u : 1u;
  c.waves = a.steps <= 4u ? 1u : a.steps <= 64u ? 4u : backward ? 16u : 8u;
  c.steps = a.steps <= 16u ? 4u : 16u;
  return c;
}

TileArgs tiles_of(const RecurrenceArgs& a, const Cut& c) {
  TileArgs G{};
  G.across = (a.width + 64u * c.vec - 1u) / (64u * c.vec);
  const uint32_t tile = c.waves * c.steps;
  G.tiles = a.steps == 0u ? 1u : (a.steps + tile - 1u) / tile;
  return G;
}

uint64_t words_for(const RecurrenceArgs& a, const Cut& c, const TileArgs& G) {
  return G.tiles > 1u ? static_cast<uint64_t>(a.batch) * G.across * G.tiles * 64u * c.vec : 0u;
}

// Workgroups, or 0 if there are more than a grid has.
uint32_t workgroups(const RecurrenceArgs& a, const TileArgs& G) {
  const uint64_t n = static_cast<uint64_t>(a.batch) * G.across * G.tiles;
  return n <= 0x7FFFFFFFull ? static_cast<uint32_t>(n) : 0u;
}

hipError_t clear_words(TileArgs& G, uint64_t words, unsigned long long* scratch, hipStream_t s) {
  if (words == 0u) return hipSuccess;
  G.words = scratch + 1;
  G.ticket = reinterpret_cast<uint32_t*>(scratch);
  clear_words_kernel<<<dim3(static_cast<uint32_t>((words + 255u) / 256u)), dim3(256), 0, s>>>(G, words);
  return hipGetLastError();
}

template <typename T, int kVec>
void launch_forward(const RecurrenceArgs& a, const Cut& c, const TileArgs& G, uint32_t wgs, hipStream_t s) {
  if (c.waves == 1u) recurrence_kernel<T, kVec, 1, 4><<<dim3(wgs), dim3(64), 0, s>>>(a, G);
  else if (c.steps == 4u) recurrence_kernel<T, kVec, 4, 4><<<dim3(wgs), dim3(256), 0, s>>>(a, G);
  else if (c.waves == 4u) recurrence_kernel<T, kVec, 4, 16><<<dim3(wgs), dim3(256), 0, s>>>(a, G);
  else recurrence_kernel<T, kVec, 8, 16><<<dim3(wgs), dim3(512), 0, s>>>(a, G);
}

template <typename T>
void launch_backward(const RecurrenceArgs& a, const RecurrenceGradArgs& d, const Cut& c, const TileArgs& G, uint32_t wgs, hipStream_t s) {
  if (c.waves == 1u) recurrence_backward_kernel<T, 1, 4><<<dim3(wgs), dim3(64), 0, s>>>(a, d, G);
  else if (c.steps == 4u) recurrence_backward_kernel<T, 4, 4><<<dim3(wgs), dim3(256), 0, s>>>(a, d, G);
  else if (c.waves == 4u) recurrence_backward_kernel<T, 4, 16><<<dim3(wgs), dim3(256), 0, s>>>(a, d, G);
  else recurrence_backward_kernel<T, 16, 16><<<dim3(wgs), dim3(1024), 0, s>>>(a, d, G);
}

}  // namespace

uint64_t recurrence_scratch_words(const RecurrenceArgs& a, int dtype, bool backward) {
  const Cut c = cut_of(a, dtype, backward);
  const uint64_t words = words_for(a, c, tiles_of(a, c));
  return words ? words + 1u : 0u;
}

hipError_t launch_recurrence(const RecurrenceArgs& a, int dtype, unsigned long long* scratch, hipStream_t s) {
  const Cut c = cut_of(a, dtype, false);
  TileArgs G = tiles_of(a, c);
  const uint32_t wgs = workgroups(a, G);
  if (wgs == 0u) return hipErrorInvalidValue;
  const hipError_t e = clear_words(G, words_for(a, c, G), scratch, s);
  if (e != hipSuccess) return e;
  if (dtype == 0) launch_forward<float, 1>(a, c, G, wgs, s);
  else if (dtype == 1 && c.vec == 2u) launch_forward<__bf16, 2>(a, c, G, wgs, s);
  else if (dtype == 1) launch_forward<__bf16, 1>(a, c, G, wgs, s);
  else if (c.vec == 2u) launch_forward<_Float16, 2>(a, c, G, wgs, s);
  else launch_forward<_Float16, 1>(a, c, G, wgs, s);
  return hipGetLastError();
}

hipError_t launch_recurrence_backward(const RecurrenceArgs& a, const RecurrenceGradArgs& g, int dtype, unsigned long long* scratch, hipStream_t s) {
  const Cut c = cut_of(a, dtype, true);
  TileArgs G = tiles_of(a, c);
  const uint32_t wgs = workgroups(a, G);
  if (wgs == 0u) return hipErrorInvalidValue;
  const hipError_t e = clear_words(G, words_for(a, c, G), scratch, s);
  if (e != hipSuccess) return e;
  if (dtype == 0) launch_backward<float>(a, g, c, G, wgs, s);
  else if (dtype == 1) launch_backward<__bf16>(a, g, c, G, wgs, s);
  else launch_backward<_Float16>(a, g, c, G, wgs, s);
  return hipGetLastError();
}

}  // namespace rgc
