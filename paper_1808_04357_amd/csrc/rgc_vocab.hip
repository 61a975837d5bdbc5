// rgc_vocab.hip -- operators over rows of logits: log probabilities of given tokens with entropy and top alternatives, their
// gradient, and the distillation loss with its gradient (include/rgc.h has the formulas).
//
// A softmax is computed in powers of two: with c = log2(e) / T and M the row's largest logit, a_j = (z_j - M) c, S = sum 2^a_j,
//   p_j = 2^a_j / S,   ln p_j = (z_j - M) / T - ln S,   entropy = ln S - ln 2 * sum 2^a_j a_j / S.
// The difference is taken before the scaling: z_j c overflows for logits near the type's lowest value, with which masks are written.
//
// All of it is bound by reading (and, for gradients, writing) the logits once.  A workgroup holds a row, or a segment of one, in registers as it
// lies in memory: all its 16-byte reads are in flight at once, and the later passes (exponentials again for the gradient, a look for
// the top alternatives) cost no traffic.  Several such workgroups share a compute unit, so that one's reads overlap another's arithmetic.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "rgc_device.h"
#include "rgc_lm.h"

namespace rgc {
namespace {

constexpr float kLn2 = 0.693147180559945309f;
constexpr uint32_t kTopMost = 128;         // RGC_TOP_MAX

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }   // 1 ulp; a result below 2^-126 is 0
__device__ __forceinline__ float log2_of(float x) { return __builtin_amdgcn_logf(x); }    // 1 ulp; log2(0) = -inf

// What is subtracted from the logits: their largest, but 0 where that is -inf (a row of nothing else, whose weights are all 0 then).
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }

// ln of a logit's probability, given ln S; -inf for every logit of a row of nothing but -inf.
__device__ __forceinline__ float log_probability(float z, float m, float inv_t, float log_sum) {
  return m == -INFINITY ? m : (z - m) * inv_t - log_sum;
}

// An exponent as a factor beside its power: 2^-200 is 0 in fp32, and 0 * -inf is not.
__device__ __forceinline__ float as_factor(float a) { return fmaxf(a, -200.0f); }

__device__ __forceinline__ bool is_token(int32_t t, uint32_t vocab) { return static_cast<uint32_t>(t) < vocab; }
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }

template <int kCtrl, int kRowMask>
__device__ __forceinline__ float dpp(float old, float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(x), kCtrl, kRowMask, 0xF, false));
}
__device__ __forceinline__ float last_lane(float x) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63)); }
__device__ __forceinline__ float wave_sum(float x) {
  x += dpp<0x111, 0xF>(0.0f, x);
  x += dpp<0x112, 0xF>(0.0f, x);
  x += dpp<0x114, 0xF>(0.0f, x);
  x += dpp<0x118, 0xF>(0.0f, x);
  x += dpp<0x142, 0xA>(0.0f, x);
  x += dpp<0x143, 0xC>(0.0f, x);
  return last_lane(x);
}
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, dpp<0x111, 0xF>(x, x));
  x = fmaxf(x, dpp<0x112, 0xF>(x, x));
  x = fmaxf(x, dpp<0x114, 0xF>(x, x));
  x = fmaxf(x, dpp<0x118, 0xF>(x, x));
  x = fmaxf(x, dpp<0x142, 0xA>(x, x));
  x = fmaxf(x, dpp<0x143, 0xC>(x, x));
  return last_lane(x);
}

// What a softmax needs of a set of logits: m the largest (NaN passed over), s = sum 2^a with a = (z - m) c, and a third sum that
// goes along: of 2^a a (scores) or of the weights at another temperature (distillation).  A NaN or +inf among the logits makes s a NaN.
enum class Third { kNone, kEntropy, kOther };      // kOther: of 2^((z - m) c1)
struct Sums {
  float m, s, e;
};
constexpr Sums kNothing{-INFINITY, 0.0f, 0.0f};

template <Third kThird>
__device__ __forceinline__ Sums rebased(const Sums& t, float m, float c, float c1) {
  const float d = t.m - base_of(m), a = d * c, w = exp2_of(a);
  Sums r{m, t.s * w, 0.0f};
  if constexpr (kThird == Third::kEntropy) r.e = w * (t.e + t.s * as_factor(a));
  if constexpr (kThird == Third::kOther) r.e = t.e * exp2_of(d * c1);
  return r;
}

// The same in every lane.
template <Third kThird>
__device__ __forceinline__ Sums wave_join(const Sums& t, float c, float c1) {
  Sums r = rebased<kThird>(t, wave_max(t.m), c, c1);
  r.s = wave_sum(r.s);
  if constexpr (kThird != Third::kNone) r.e = wave_sum(r.e);
  return r;
}

// Everything that is made of a row with a NaN or +inf is NaN.
__device__ __forceinline__ Sums spoiled(Sums t) {
  if (t.s != t.s) t.m = t.s;
  return t;
}

// ---------------------------------------------------------------- a row's segment in registers

template <typename T>
struct Vector {
  static constexpr uint32_t kElems = 16u / sizeof(T);
  typedef uint32_t Words __attribute__((ext_vector_type(4)));
  // aligned to an element only: gfx950 reads and writes 16 bytes at any address
  typedef uint32_t Unaligned __attribute__((ext_vector_type(4), aligned(2)));

  static __device__ __forceinline__ Words load(const T* p) { return *reinterpret_cast<const Words*>(p); }
  template <bool kStream = false>
  static __device__ __forceinline__ void store(T* p, const float (&v)[kElems]) {
    T t[kElems];
#pragma unroll
    for (uint32_t i = 0; i < kElems; ++i) t[i] = static_cast<T>(v[i]);
    Words w;
    __builtin_memcpy(&w, t, 16);
    if constexpr (kStream) __builtin_nontemporal_store(static_cast<Unaligned>(w), reinterpret_cast<Unaligned*>(p));
    else *reinterpret_cast<Unaligned*>(p) = w;
  }
  static __device__ __forceinline__ void unpack(const Words& w, float (&v)[kElems]) {
    T t[kElems];
    __builtin_memcpy(t, &w, 16);
#pragma unroll
    for (uint32_t i = 0; i < kElems; ++i) v[i] = static_cast<float>(t[i]);
  }
};

// n elements from z on, by a workgroup of kThreads: vector i * kThreads + thread in raw[i].  Vectors begin on 16 bytes (an odd vocabulary's rows read at two bytes
// off took 42 us more of 104); the few elements before the first and behind the last are held one each by the first threads.  What is beyond the segment
// reads as -inf.
template <typename T, uint32_t kThreads, uint32_t kVectors>
struct Held {
  using V = Vector<T>;
  static constexpr uint32_t kElems = V::kElems, kCapacity = kThreads * kVectors * kElems;
  mutable typename V::Words raw[kVectors];
  float single;
  uint32_t n, head, vectors, wave0;      // wave0: the wave's first thread

  __device__ __forceinline__ Held(const T* z, uint32_t n_) : n(n_), wave0(uniform(threadIdx.x & ~63u)) {
    head = min((16u - (static_cast<uint32_t>(reinterpret_cast<uintptr_t>(z)) & 15u)) % 16u / static_cast<uint32_t>(sizeof(T)), n);
    vectors = (n - head) / kElems;
    if (vectors > 0u) {
      const T* from = z + head;
      // (no branches between the reads, or the compiler waits for each: behind the end, the last vector again)
#pragma unroll
      for (uint32_t i = 0; i < kVectors; ++i) raw[i] = V::load(from + static_cast<uint64_t>(min(i * kThreads + threadIdx.x, vectors - 1u)) * kElems);
    }
    single = has_single() ? static_cast<float>(z[single_index()]) : -INFINITY;
  }
  __device__ __forceinline__ bool has_single() const { return threadIdx.x < n - vectors * kElems; }
  __device__ __forceinline__ uint32_t single_index() const { return threadIdx.x < head ? threadIdx.x : threadIdx.x + vectors * kElems; }
  __device__ __forceinline__ uint32_t index(uint32_t i) const { return head + (i * kThreads + threadIdx.x) * kElems; }
  __device__ __forceinline__ bool mine(uint32_t i) const { return i * kThreads + threadIdx.x < vectors; }
  // f(i, values): for the vectors of which the wave has any
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
#pragma unroll
    for (uint32_t i = 0; i < kVectors; ++i) {
      if (i * kThreads + wave0 >= vectors) break;
      // (Another pass's unpacked values are not to be kept for this one: they take two registers where the packed ones take one.)
      asm volatile("" : "+v"(raw[i]));
      float v[kElems];
      V::unpack(raw[i], v);
      if (i * kThreads + wave0 + 64u > vectors) {
#pragma unroll
        for (uint32_t j = 0; j < kElems; ++j) v[j] = mine(i) ? v[j] : -INFINITY;
      }
      f(i, v);
    }
  }
  // Which thread holds element `at` of the segment.
  __device__ __forceinline__ uint32_t owner(uint32_t at) const {
    if (at < head) return at;
    const uint32_t vector = (at - head) / kElems;
    return vector < vectors ? vector % kThreads : at - vectors * kElems;
  }
};

__device__ __forceinline__ float weigh(float z, float base, float c) { return exp2_of((z - base) * c); }

// Sums of what a thread holds, the largest rescaling those before it, vector by vector as they arrive.  kSquared: the other temperature's weights are the squares
// of these (T = 2).
template <Third kThird, bool kSquared, typename H>
__device__ __forceinline__ Sums sums_of(const H& held, float c, float c1) {
  Sums t{held.single, 0.0f, 0.0f};
  {
    const float base = base_of(t.m), w = weigh(held.single, base, c);      // 1, 0 for -inf, NaN for NaN and +inf
    t.s = w;
    if constexpr (kThird == Third::kOther) t.e = w;
  }
  held.each([&](uint32_t, const float (&v)[H::kElems]) __attribute__((always_inline)) {
    float m = t.m;
#pragma unroll
    for (uint32_t j = 0; j < H::kElems; ++j) m = fmaxf(m, v[j]);
    const float base = base_of(m);
    {
      const float d = t.m - base, a = d * c, w = exp2_of(a);
      if constexpr (kThird == Third::kEntropy) t.e = w * (t.e + t.s * as_factor(a));
      if constexpr (kThird == Third::kOther) t.e *= kSquared ? w * w : exp2_of(d * c1);
      t.s *= w;
    }
    t.m = m;
#pragma unroll
    for (uint32_t j = 0; j < H::kElems; ++j) {
      const float d = v[j] - base, a = d * c, w = exp2_of(a);
      t.s += w;
      if constexpr (kThird == Third::kEntropy) t.e = __fmaf_rn(w, as_factor(a), t.e);
      if constexpr (kThird == Third::kOther) t.e = kSquared ? __fmaf_rn(w, w, t.e) : t.e + exp2_of(d * c1);
    }
  });
  return t;
}

// A row whose largest logit has nearly all the weight has S = 1 + x with a small x, of which fp32 keeps little beside the 1, and its log probability is
// -ln(1 + x).  Up to this S, x is added up by itself.
constexpr float kNearlyOne = 1.25f;
__device__ __forceinline__ bool nearly_one(float s) { return s >= 1.0f && s < kNearlyOne; }
// ln(1 + x) for -1 + 1 / kNearlyOne <= x <= kNearlyOne - 1: 2 artanh(t) with t = x / (2 + x), |t| <= 1/9, by its series up to t^9 (the next term is below 2^-34 of it).
__device__ __forceinline__ float log1p_of(float x) {
  const float t = x * __builtin_amdgcn_rcpf(2.0f + x), t2 = t * t;
  return 2.0f * t * __fmaf_rn(t2, __fmaf_rn(t2, __fmaf_rn(t2, __fmaf_rn(t2, 1.0f / 9.0f, 1.0f / 7.0f), 1.0f / 5.0f), 1.0f / 3.0f), 1.0f);
}
__device__ __forceinline__ float log_of_sum(float s, float x) { return nearly_one(s) ? log1p_of(x) : kLn2 * log2_of(s); }

// The weights of all logits but one of the largest, and the same at the other temperature (kOther).
struct Others {
  float x, x1;
};
template <Third kThird>
__device__ __forceinline__ bool others_wanted(const Sums& t) { return nearly_one(t.s) || (kThird == Third::kOther && nearly_one(t.e)); }

// Of several sets (a row's waves or segments) joined to t: own and x are the lane's set's.
template <Third kThird>
__device__ __forceinline__ Others others_join(const Sums& own, const Others& x, const Sums& t, float c, float c1) {
  // the first set that has the largest logit counts without it
  const unsigned long long holders = __ballot(own.m == t.m);
  const bool holds = holders != 0ull && (threadIdx.x & 63u) == static_cast<uint32_t>(__ffsll(holders) - 1);
  const Sums moved = rebased<kThird == Third::kOther ? Third::kOther : Third::kNone>(own, t.m, c, c1);
  Others o{wave_sum(holds ? x.x : moved.s), 0.0f};
  if constexpr (kThird == Third::kOther) o.x1 = wave_sum(holds ? x.x1 : moved.e);
  return o;
}

template <uint32_t kThreads, uint32_t kVectors>
struct JoinShared {
  float sums[kThreads / 64u][5];
  uint4 raw[kThreads / 64u][kVectors];                               // of one thread of each wave
};

// What a wave holds; t: its sums.  Only the lane that holds the one left out has the loss: what it holds is added up again, by the whole wave (by that
// lane alone it took 3 us of 17, 700 rows of 10000 in fp32).
template <Third kThird, bool kSquared, typename T, uint32_t kThreads, uint32_t kVectors>
__device__ __forceinline__ Others others_of(const Held<T, kThreads, kVectors>& held, const Sums& own, const Sums& t, float c, float c1, uint4 (&raw)[kVectors]) {
  constexpr bool kTwo = kThird == Third::kOther;
  const uint32_t lane = threadIdx.x & 63u, first = static_cast<uint32_t>(__ffsll(__ballot(own.m == t.m)) - 1), thread = held.wave0 + first;
  if (lane == first) {
#pragma unroll
    for (uint32_t i = 0; i < kVectors; ++i) __builtin_memcpy(&raw[i], &held.raw[i], 16);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const uint32_t n = thread < held.vectors ? ((held.vectors - 1u - thread) / kThreads + 1u) * Vector<T>::kElems : 0u;
  // (element n: the single one)
  const float single = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(held.single), static_cast<int>(first)));
  const Sums moved = rebased<kTwo ? Third::kOther : Third::kNone>(own, t.m, c, c1);
  Others x{lane == first ? 0.0f : moved.s, lane == first ? 0.0f : moved.e};
  uint32_t equal = 0u;
  for (uint32_t from = 0; from <= n; from += 64u) {
    const uint32_t i = from + lane;
    const float v = i < n ? static_cast<float>(reinterpret_cast<const T*>(raw)[i]) : i == n ? single : -INFINITY;
    const bool largest = v == t.m;
    const float w = largest ? 0.0f : weigh(v, t.m, c);
    x.x += w;
    if constexpr (kTwo) x.x1 += kSquared ? w * w : largest ? 0.0f : weigh(v, t.m, c1);
    equal += static_cast<uint32_t>(__popcll(__ballot(largest)));
  }
  x.x = wave_sum(x.x) + static_cast<float>(equal - 1u);
  if constexpr (kTwo) x.x1 = wave_sum(x.x1) + static_cast<float>(equal - 1u);
  return x;
}

// The same in every thread.  Holds one barrier, which callers rely on.
struct Joined {
  Sums t;
  Others x;
};
template <Third kThird, bool kSquared, typename T, uint32_t kThreads, uint32_t kVectors>
__device__ __forceinline__ Joined block_join(const Held<T, kThreads, kVectors>& held, const Sums& own, float c, float c1, JoinShared<kThreads, kVectors>& lds) {
  constexpr uint32_t kWaves = kThreads / 64u;
  const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6);
  auto others = [](const Sums& t) { return Others{t.s - 1.0f, t.e - 1.0f}; };
  Joined j;
  j.t = wave_join<kThird>(own, c, c1);
  j.x = others_wanted<kThird>(j.t) ? others_of<kThird, kSquared>(held, own, j.t, c, c1, lds.raw[wave]) : others(j.t);
  if (kWaves > 1 && lane == 0u) {
    float(&to)[5] = lds.sums[wave];
    to[0] = j.t.m, to[1] = j.t.s, to[2] = j.t.e, to[3] = j.x.x, to[4] = j.x.x1;
  }
  __syncthreads();
  if constexpr (kWaves > 1) {
    Sums of = kNothing;
    Others x{};
    if (lane < kWaves) {
      const float(&from)[5] = lds.sums[lane];
      of = Sums{from[0], from[1], from[2]};
      x = Others{from[3], from[4]};
    }
    j.t = wave_join<kThird>(of, c, c1);
    j.x = others_wanted<kThird>(j.t) ? others_join<kThird>(of, x, j.t, c, c1) : others(j.t);
  }
  return j;
}

// ---------------------------------------------------------------- the top alternatives of a segment

// Larger for a larger logit, the same for +0 and -0, largest for a NaN; 0 is no logit's.
__device__ __forceinline__ uint32_t order_of(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  if (z != z) return 0xFFFFFFFFu;
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t order) {
  if (order == 0xFFFFFFFFu) return NAN;
  return __uint_as_float((order & 0x80000000u) ? order & 0x7FFFFFFFu : ~order);
}
// Orders entries: larger logits first, then lower indices.
__device__ __forceinline__ uint64_t entry_of(float z, uint32_t index) { return (static_cast<uint64_t>(order_of(z)) << 32) | (0xFFFFFFFFu - index); }

constexpr uint32_t kListed = 1024;      // candidates a workgroup can list

template <uint32_t kThreads>
struct TopShared {
  uint64_t list[kListed];
  uint32_t line[kThreads / 64u];        // of every wave
  uint32_t count, scan[kThreads / 64u];
};

// The largest number, looked for from bit `from` down to bit `to`, that at least k of the wave's lanes reach.
__device__ __forceinline__ uint32_t reached_by(uint32_t v, uint32_t k, uint32_t line, int from, int to) {
  for (int bit = from; bit >= to; --bit) {
    const uint32_t higher = line | (1u << bit);
    if (popc64(__ballot(v >= higher)) >= k) line = higher;
  }
  return line;
}

// How many of n entries come before e.
__device__ __forceinline__ uint32_t rank_in(const uint64_t* list, uint32_t n, uint64_t e) {
  uint32_t rank = 0, j = 0;
  for (; j + 8u <= n; j += 8u) {      // (eight reads in flight)
    uint64_t v[8];
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) v[i] = list[j + i];
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) rank += v[i] > e ? 1u : 0u;
  }
  for (; j < n; ++j) rank += list[j] > e ? 1u : 0u;
  return rank;
}

// f(index, logit) for every logit of a segment, read again from memory.  (One at a time: with vectors the whole kernel has a quarter more registers, and fewer
// workgroups share a compute unit.)
template <typename T, uint32_t kThreads, typename F>
__device__ __forceinline__ void read_again(const T* z, uint32_t n, F&& f) {
#pragma unroll 4
  for (uint32_t i = threadIdx.x; i < n; i += kThreads) f(i, static_cast<float>(z[i]));
}

// How many of the segment's logits have an order above `line`; the same in every thread.  Holds barriers.
template <typename T, uint32_t kThreads>
__device__ __forceinline__ uint32_t count_above(const T* z, uint32_t n, uint32_t line, TopShared<kThreads>& lds) {
  uint32_t mine = 0, total = 0;
  read_again<T, kThreads>(z, n, [&](uint32_t, float v) { mine += order_of(v) > line ? 1u : 0u; });
  (void)block_excl_scan<kThreads / 64u>(mine, lds.scan, total);
  return total;
}

// lds.list: the k largest, where more logits than it holds reach a line, `line` not above the k-th largest.  Those above the k-th largest, and
// then those equal to it in the order of their indices.
template <typename T, uint32_t kThreads>
__device__ __forceinline__ void list_exactly(const T* z, uint32_t n, uint32_t line, uint32_t k, uint32_t first, TopShared<kThreads>& lds) {
  uint32_t above = count_above<T, kThreads>(z, n, line, lds);
  if (above >= k) {                                        // the k-th largest is higher: bit by bit
    uint32_t found = 0u;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t higher = found | (1u << bit);
      if (count_above<T, kThreads>(z, n, higher - 1u, lds) >= k) found = higher;
    }
    line = found;
    above = count_above<T, kThreads>(z, n, line, lds);
  }
  if (threadIdx.x == 0u) lds.count = 0u;
  __syncthreads();
  read_again<T, kThreads>(z, n, [&](uint32_t i, float v) {
    if (order_of(v) > line) lds.list[atomicAdd(&lds.count, 1u)] = entry_of(v, first + i);
  });
  constexpr uint32_t kElems = Vector<T>::kElems;
  const uint32_t vectors = n / kElems;
  uint32_t before = above;
  for (uint32_t from = 0; from < n && before < k;) {
    // a vector a thread, at last the elements behind the last whole one
    const bool whole = from < vectors * kElems;
    const uint32_t at = from + (whole ? threadIdx.x * kElems : threadIdx.x), each = whole ? kElems : 1u, end = whole ? vectors * kElems : n;
    uint32_t equal = 0;
    if (at < end)
      for (uint32_t j = 0; j < each; ++j) equal |= order_of(static_cast<float>(z[at + j])) == line ? 1u << j : 0u;
    uint32_t total = 0;
    uint32_t place = before + block_excl_scan<kThreads / 64u>(static_cast<uint32_t>(__popc(equal)), lds.scan, total);
    for (; equal != 0u && place < k; equal &= equal - 1u) lds.list[place++] = entry_of(logit_of(line), first + at + static_cast<uint32_t>(__ffs(static_cast<int>(equal)) - 1));
    before += total;
    from = whole ? min(from + kThreads * kElems, end) : n;
  }
  __syncthreads();
}

// A line under the k-th largest of a segment comes cheap: with q = ceil(k / waves), every wave's q-th largest of its lanes' largest is reached by q logits
// of that wave, so the lowest of these is reached by k.  (Of the waves all of whose lanes have a vector, that is; without one all logits reach it.)  Few more
// reach it (where the logits lie anywhere: some 20 with four waves and k = 8, 100 with k = 64, 55 with sixteen waves and k = 8); they are listed and ranked.
// Where more do than the list holds, as with many equal ones (a mask that leaves fewer than k), list_exactly reads the segment again.
template <uint32_t kThreads, typename H>
__device__ __forceinline__ uint32_t line_of(const H& held, float t, uint32_t k, uint32_t line, int from, int to) {
  const uint32_t full = min(kThreads, held.vectors) / 64u;
  if (full == 0u) return 0u;
  if (threadIdx.x / 64u >= full) return 0xFFFFFFFFu;
  return reached_by(order_of(t), (k + full - 1u) / full, line, from, to);
}
// Before the barrier of the sums' join; t: the thread's largest.
template <uint32_t kThreads, typename H>
__device__ __forceinline__ uint32_t put_line(const H& held, float t, uint32_t k, TopShared<kThreads>& lds) {
  // (sixteen bits of it will do: a line a little lower lets a few more through)
  const uint32_t line = line_of<kThreads>(held, t, k, 0u, 31, 16);
  if ((threadIdx.x & 63u) == 0u) lds.line[threadIdx.x >> 6] = line;
  if (threadIdx.x == 0u) lds.count = 0u;
  return line;
}
template <uint32_t kThreads>
__device__ __forceinline__ uint32_t lowest_line(const TopShared<kThreads>& lds) {
  uint32_t line = lds.line[0];
#pragma unroll
  for (uint32_t w = 1; w < kThreads / 64u; ++w) line = min(line, lds.line[w]);
  return uniform(line);
}

// Behind that barrier: the k largest (k <= the segment's length), put(rank, entry) each.  `own`: what put_line gave; `spoilt`: there is a NaN or +inf among them.
template <typename T, uint32_t kThreads, typename H, typename Put>
__device__ __forceinline__ void top_of(const H& held, const T* z, float t, uint32_t own, bool spoilt, uint32_t k, uint32_t first, TopShared<kThreads>& lds, Put&& put) {
  if (!spoilt) {
    const uint32_t line = lowest_line<kThreads>(lds);
    const float least = line <= 0x007FFFFFu ? -INFINITY : logit_of(line);      // (below the order of -inf all are taken)
    // Eight bits a vector, then places in the list for all of a thread's: their indices alone, the few logits are read again below.  (With 8192 rows of 32000, 91 us
    // without alternatives: 108 with k = 8, 122 with k = 64.  When these were 96, 121 and 139: writing each where it is met 128 and 177, asking the whole wave about
    // every element of a vector that has one 135 and 190; what needs the packed registers a second time takes 50 more registers a thread, and a third of the workgroups.)
    constexpr uint32_t kVectors = sizeof(held.raw) / sizeof(held.raw[0]), kHitWords = (kVectors + 3u) / 4u;
    uint32_t hits[kHitWords] = {}, n = held.has_single() && held.single >= least ? 1u : 0u;
    held.each([&](uint32_t i, const float (&v)[H::kElems]) __attribute__((always_inline)) {
      float most = v[0];
#pragma unroll
      for (uint32_t j = 1; j < H::kElems; ++j) most = fmaxf(most, v[j]);
      if (most >= least && held.mine(i)) {
        uint32_t bits = 0;
#pragma unroll
        for (uint32_t j = 0; j < H::kElems; ++j) bits |= v[j] >= least ? 1u << j : 0u;
        hits[i / 4u] |= bits << (8u * (i % 4u));
      }
    });
#pragma unroll
    for (uint32_t w = 0; w < kHitWords; ++w) n += static_cast<uint32_t>(__popc(hits[w]));
    if (n > 0u) {
      uint32_t at = atomicAdd(&lds.count, n);
      if (held.has_single() && held.single >= least && at < kListed) lds.list[at++] = held.single_index();
#pragma unroll
      for (uint32_t w = 0; w < kHitWords; ++w)
        for (uint32_t bits = hits[w]; bits != 0u && at < kListed; bits &= bits - 1u) {
          const uint32_t bit = static_cast<uint32_t>(__ffs(static_cast<int>(bits)) - 1);
          lds.list[at++] = held.index(4u * w + bit / 8u) + bit % 8u;
        }
    }
  }
  __syncthreads();
  uint32_t listed = uniform(lds.count);
  if (spoilt || listed > kListed) {
    const uint32_t exact = line_of<kThreads>(held, t, k, own, 15, 0);
    if ((threadIdx.x & 63u) == 0u) lds.line[threadIdx.x >> 6] = spoilt ? 0u : exact;
    __syncthreads();
    list_exactly<T, kThreads>(z, held.n, lowest_line<kThreads>(lds), k, first, lds);
    listed = k;
  } else {
    for (uint32_t i = threadIdx.x; i < listed; i += kThreads) {
      const uint32_t index = static_cast<uint32_t>(lds.list[i]);
      lds.list[i] = entry_of(static_cast<float>(z[index]), first + index);
    }
    __syncthreads();
  }
  for (uint32_t i = threadIdx.x; i < listed; i += kThreads) {
    const uint64_t e = lds.list[i];
    const uint32_t rank = rank_in(lds.list, listed, e);
    if (rank < k) put(rank, e);
  }
}

// ---------------------------------------------------------------- scores

__device__ __forceinline__ void put_alternative(const ScoreArgs& A, uint32_t r, uint32_t rank, uint64_t entry, const Sums& t, float log_sum) {
  const uint64_t at = static_cast<uint64_t>(r) * A.top + rank;
  A.top_idx[at] = static_cast<int32_t>(0xFFFFFFFFu - static_cast<uint32_t>(entry));
  A.top_logprob[at] = log_probability(logit_of(static_cast<uint32_t>(entry >> 32)), t.m, A.inv_t, log_sum);
}

__device__ __forceinline__ void put_left_out(const ScoreArgs& A, uint32_t r) {
  if (threadIdx.x == 0u) {
    if (A.logprob) A.logprob[r] = 0.0f;
    if (A.entropy) A.entropy[r] = 0.0f;
    if (A.stats) A.stats[2ull * r] = A.stats[2ull * r + 1u] = 0.0f;
  }
  for (uint32_t i = threadIdx.x; i < A.top; i += blockDim.x) {
    A.top_idx[static_cast<uint64_t>(r) * A.top + i] = -1;
    A.top_logprob[static_cast<uint64_t>(r) * A.top + i] = -INFINITY;
  }
}

// By one thread; at_target: the target's logit.
__device__ __forceinline__ void put_scores(const ScoreArgs& A, uint32_t r, const Sums& t, float log_sum, float at_target) {
  if (A.logprob) A.logprob[r] = log_probability(at_target, t.m, A.inv_t, log_sum);
  if (A.entropy) A.entropy[r] = t.s == 0.0f ? 0.0f : log_sum - kLn2 * (t.e / t.s);
  if (A.stats) {
    A.stats[2ull * r] = t.m;
    A.stats[2ull * r + 1u] = log_sum;
  }
}

template <typename T>
__device__ __forceinline__ const T* row_of(const void* p, int64_t stride, uint32_t r) {
  return static_cast<const T*>(p) + static_cast<int64_t>(r) * stride;
}

// A workgroup a segment.  One segment a row: its results; several: its sums and its top entries for score_join_kernel.
template <typename T, uint32_t kThreads, uint32_t kVectors>
__global__ void __launch_bounds__(kThreads) score_kernel(ScoreArgs A, SplitArgs P) {
  __shared__ JoinShared<kThreads, kVectors> lds;
  __shared__ TopShared<kThreads> top;
  const uint32_t r = blockIdx.x / P.segments, segment = blockIdx.x - r * P.segments;
  const uint32_t first = segment * P.length, n = min(A.vocab - first, P.length);
  const int32_t target = A.targets ? A.targets[r] : 0;
  const T* z = row_of<T>(A.logits, A.row_stride, r);
  if (!is_token(target, A.vocab)) {
    if (P.segments == 1u) put_left_out(A, r);
    return;
  }
  const Held<T, kThreads, kVectors> held(z + first, n);
  const float at_target = P.segments == 1u && threadIdx.x == 0u ? static_cast<float>(z[target]) : 0.0f;
  const Sums own = sums_of<Third::kEntropy, false>(held, A.scale, 0.0f);
  const uint32_t k = min(A.top, n), line = k > 0u ? put_line<kThreads>(held, own.m, k, top) : 0u;
  const Joined raw = block_join<Third::kEntropy, false>(held, own, A.scale, 0.0f, lds);
  const Sums t = spoiled(raw.t);
  if (P.segments == 1u) {
    const float log_sum = log_of_sum(t.s, raw.x.x);
    if (threadIdx.x == 0u) put_scores(A, r, t, log_sum, at_target);
    if (k > 0u)
      top_of<T, kThreads>(held, z, own.m, line, t.s != t.s, k, 0u, top, [&](uint32_t rank, uint64_t e) { put_alternative(A, r, rank, e, t, log_sum); });
  } else {
    if (threadIdx.x == 0u) {
      float* to = P.sums + 4ull * blockIdx.x;
      to[0] = raw.t.m;
      to[1] = raw.t.s;
      to[2] = raw.t.e;
      to[3] = raw.x.x;
    }
    if (k > 0u)
      top_of<T, kThreads>(held, z + first, own.m, line, t.s != t.s, k, first, top,
                          [&](uint32_t rank, uint64_t e) { P.entries[static_cast<uint64_t>(blockIdx.x) * A.top + rank] = e; });
  }
}

// A row of several segments (64 at most): their sums joined, their entries, which stand in order, merged.
constexpr uint32_t kJoinThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) score_join_kernel(ScoreArgs A, SplitArgs P) {
  extern __shared__ uint64_t entries[];                    // [segments][top]
  const uint32_t r = blockIdx.x, lane = threadIdx.x & 63u, last = A.vocab - (P.segments - 1u) * P.length;
  const int32_t target = A.targets ? A.targets[r] : 0;
  if (!is_token(target, A.vocab)) {
    put_left_out(A, r);
    return;
  }
  const float at_target = static_cast<float>(row_of<T>(A.logits, A.row_stride, r)[target]);
  Sums own = kNothing;
  float x = 0.0f;                                          // of the segment's weights, without one of its largest
  if (lane < P.segments) {
    const float* from = P.sums + 4ull * (static_cast<uint64_t>(r) * P.segments + lane);
    own = Sums{from[0], from[1], from[2]};
    x = from[3];
  }
  // (every segment but the last has more than RGC_TOP_MAX logits)
  const uint32_t all = (P.segments - 1u) * A.top + min(A.top, last);
  for (uint32_t i = threadIdx.x; i < all; i += kJoinThreads) entries[i] = P.entries[static_cast<uint64_t>(r) * P.segments * A.top + i];
  const Sums t = spoiled(wave_join<Third::kEntropy>(own, A.scale, 0.0f));
  const float log_sum = log_of_sum(t.s, others_join<Third::kEntropy>(own, Others{x, 0.0f}, t, A.scale, 0.0f).x);
  if (threadIdx.x == 0u) put_scores(A, r, t, log_sum, at_target);
  __syncthreads();
  if (all <= 2u * kJoinThreads) {
    for (uint32_t i = threadIdx.x; i < all; i += kJoinThreads) {
      const uint32_t rank = rank_in(entries, all, entries[i]);
      if (rank < A.top) put_alternative(A, r, rank, entries[i], t, log_sum);
    }
    return;
  }
  for (uint32_t i = threadIdx.x; i < all; i += kJoinThreads) {
    const uint32_t segment = i / A.top;
    const uint64_t e = entries[i];
    uint32_t rank = i - segment * A.top;
    for (uint32_t s = 0; s < P.segments && rank < A.top; ++s) {
      if (s == segment) continue;
      uint32_t low = 0, high = s + 1u == P.segments ? min(A.top, last) : A.top;      // how many of that segment's entries come before e
      while (low < high) {
        const uint32_t mid = (low + high) / 2u;
        if (entries[s * A.top + mid] > e) low = mid + 1u; else high = mid;
      }
      rank += low;
    }
    if (rank < A.top) put_alternative(A, r, rank, e, t, log_sum);
  }
}

// dz_j = g (1{j = target} - p_j) - h p_j (log p_j + entropy), g and h divided by T: no sums, so any part of a row by any workgroup.
// A gradient of more than kStreamFrom bytes is stored past the caches (kStream).  Stored the common way, what of it was still in them was written out while
// the next pass read its logits.  Loss and gradient of 4096 x 32000 bf16 in turn, common -> past the caches: 165 -> 140 us, and 258 -> 240 with a copy of the
// gradient right behind them; 2000 x 50257 bf16 124 -> 109 and 199 -> 186; 4000 x 10000 bf16 (80 MB) 58 -> 52 and 82 -> 81.  Under the bound a reader finds
// the gradient in the caches, and loses more than the call gains: 1300 x 10000 f32 (52 MB) 32.0 -> 31.5 and 49.7 -> 52.1.  (The distillation's gradient has no
// second reading of the logits to disturb; past the caches its reader lost all that it gained: 2048 x 128000 213 -> 207 and 412 -> 420.)
constexpr uint32_t kGradThreads = 256, kGradVectors = 4;
constexpr uint64_t kStreamFrom = 64ull << 20;
template <typename T, bool kStream>
__global__ void __launch_bounds__(kGradThreads) score_grad_kernel(ScoreGradArgs A, uint32_t parts) {
  using V = Vector<T>;
  constexpr uint32_t kPart = kGradThreads * kGradVectors * V::kElems;
  const uint32_t r = blockIdx.x / parts, first = (blockIdx.x - r * parts) * kPart, n = min(A.vocab - first, kPart);
  const T* z = row_of<T>(A.logits, A.row_stride, r) + first;
  T* dz = static_cast<T*>(A.grad_logits) + static_cast<int64_t>(r) * A.grad_row_stride + first;
  const int32_t target = A.targets ? A.targets[r] : -1;
  const float m = A.stats[2ull * r], log_sum = A.stats[2ull * r + 1u];
  const bool nothing = (A.targets && !is_token(target, A.vocab)) || log_sum == -INFINITY;
  const Held<T, kGradThreads, kGradVectors> held(z, n);
  if (nothing) {
    held.each([&](uint32_t i, const float (&)[V::kElems]) __attribute__((always_inline)) {
      const float zeros[V::kElems] = {};
      if (held.mine(i)) V::template store<kStream>(dz + held.index(i), zeros);
    });
    if (held.has_single()) dz[held.single_index()] = static_cast<T>(0.0f);
    return;
  }
  const float g = A.grad_logprob ? A.grad_logprob[r] * A.inv_t : 0.0f, h = A.grad_entropy ? A.grad_entropy[r] * A.inv_t : 0.0f;
  const float entropy = A.grad_entropy ? A.entropy[r] : 0.0f, log2s = log_sum * (1.0f / kLn2);
  // p (g + h (ln p + entropy)) = p (u + w a), a = log2 p
  const float hh = h * entropy, u = g + hh, w = h * kLn2;
  auto slope = [&](float v) {
    const float a = __fmaf_rn(v - m, A.scale, -log2s);
    return -exp2_of(a) * __fmaf_rn(w, as_factor(a), u);
  };
  const uint32_t at = static_cast<uint32_t>(target) - first;       // of the target in this part, if it is
  const bool here = target >= 0 && at < n && held.owner(at) == threadIdx.x;
  // there g (1 - p) - h p (ln p + entropy); 1 - p is made of ln p, for of a probability near 1 fp32 keeps little beside the 1
  float at_target = 0.0f;
  if (here) {
    const float v = static_cast<float>(z[at]), a = __fmaf_rn(v - m, A.scale, -log2s);
    at_target = -g * expm1f(log_probability(v, m, A.inv_t, log_sum)) - exp2_of(a) * __fmaf_rn(w, as_factor(a), hh);
  }
  held.each([&](uint32_t i, const float (&v)[V::kElems]) __attribute__((always_inline)) {
    float d[V::kElems];
#pragma unroll
    for (uint32_t j = 0; j < V::kElems; ++j) d[j] = slope(v[j]);
    if (held.mine(i)) V::template store<kStream>(dz + held.index(i), d);
  });
  if (held.has_single()) dz[held.single_index()] = static_cast<T>(slope(held.single));
  if (here) dz[at] = static_cast<T>(at_target);                    // over what the same thread has just stored
}

// ---------------------------------------------------------------- distillation

// A row's teacher entries and label, made by the first wave.
constexpr uint32_t kSeenBits = 65536;
struct Teacher {
  int32_t at[kTopMost + 1];             // k entries, an index once, and the label's unless it is one of them; -1: none
  float q[kTopMost + 1], z[kTopMost + 1];        // the teacher's probability there, and the student's logit
  float soft;                           // sum of the weights: 0 if there are none
  int32_t heavy;                        // the index of nearly all of the teacher's probability, -1: none; and the others' probability
  float rest;
  alignas(16) uint32_t seen[kSeenBits / 32u];
};

// Two entries a lane.
struct TeacherLane {
  float q[2], log_q[2], z[2];
  int32_t at[2];
  float at_label;
};

__device__ __forceinline__ float lane_of(float x, uint32_t lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), static_cast<int>(lane))); }

// gather(index): the student's logit.
template <typename Gather>
__device__ __forceinline__ TeacherLane teach(const DistillArgs& A, uint32_t r, int32_t label, Gather&& gather, Teacher& to) {
  const uint32_t lane = threadIdx.x;
  TeacherLane t;
  float z[2], largest = -INFINITY;
  t.at_label = label >= 0 ? gather(kTopMost, label) : 0.0f;
#pragma unroll
  for (uint32_t u = 0; u < 2u; ++u) {
    const uint32_t i = lane + 64u * u;
    t.at[u] = i < A.k ? A.teacher_idx[static_cast<uint64_t>(r) * A.k + i] : -1;
    if (!is_token(t.at[u], A.vocab)) t.at[u] = -1;
    z[u] = t.at[u] >= 0 ? A.teacher_logits[static_cast<uint64_t>(r) * A.k + i] : -INFINITY;
    t.z[u] = t.at[u] >= 0 ? gather(i, t.at[u]) : 0.0f;
    largest = fmaxf(largest, z[u]);
  }
  largest = wave_max(largest);
  float w[2], sum = 0.0f;
#pragma unroll
  for (uint32_t u = 0; u < 2u; ++u) {
    w[u] = weigh(z[u], base_of(largest), A.scale);
    sum += w[u];
  }
  sum = wave_sum(sum);
  const float log_sum = kLn2 * log2_of(sum);
  bool again[2] = {false, false};
#pragma unroll
  for (uint32_t u = 0; u < 2u; ++u) {
    t.q[u] = sum == 0.0f ? 0.0f : w[u] / sum;
    t.log_q[u] = log_probability(z[u], largest, A.inv_t, log_sum);
  }
  // An index that comes twice has both weights, at its first place, in the loss as in the gradient (q ln q of a sum is not the sum of its parts').  Few
  // rows have any: whether one may come twice is told by a bit for every index (one of kSeenBits), and those that find theirs set are looked for among
  // all.  (A loop over all entries took 20 us of 108, 2048 rows of 64.)
#pragma unroll
  for (uint32_t i = 0; i < kSeenBits / 32u / 256u; ++i) reinterpret_cast<uint4*>(to.seen)[i * 64u + lane] = uint4{0u, 0u, 0u, 0u};
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (uint32_t u = 0; u < 2u; ++u) {
    const uint32_t h = (static_cast<uint32_t>(t.at[u]) * 2654435761u) >> 16;
    unsigned long long met = __ballot(t.at[u] >= 0 && ((atomicOr(&to.seen[h / 32u], t.at[u] >= 0 ? 1u << (h & 31u) : 0u) >> (h & 31u)) & 1u) != 0u);
    for (; met != 0ull; met &= met - 1ull) {
      const int32_t at = __builtin_amdgcn_readlane(t.at[u], __ffsll(met) - 1);
      const unsigned long long in0 = __ballot(t.at[0] == at), in1 = __ballot(t.at[1] == at);
      if (__popcll(in0) + __popcll(in1) < 2) continue;
      const uint32_t place = in0 != 0ull ? static_cast<uint32_t>(__ffsll(in0) - 1) : 64u + static_cast<uint32_t>(__ffsll(in1) - 1);
      float both = 0.0f;
      for (unsigned long long m = in0; m != 0ull; m &= m - 1ull) both += lane_of(w[0], static_cast<uint32_t>(__ffsll(m) - 1));
      for (unsigned long long m = in1; m != 0ull; m &= m - 1ull) both += lane_of(w[1], static_cast<uint32_t>(__ffsll(m) - 1));
#pragma unroll
      for (uint32_t v = 0; v < 2u; ++v) {
        if (t.at[v] != at) continue;
        const bool here = lane + 64u * v == place;
        t.q[v] = here && sum != 0.0f ? both / sum : 0.0f;
        t.log_q[v] = kLn2 * log2_of(both) - log_sum;
        again[v] = !here;
      }
    }
  }
  // What is made of 1 - q where q is nearly one is made of the others' weights.
  int32_t heavy = -1;
  float rest = 0.0f;
  const unsigned long long heavy0 = __ballot(t.q[0] > 1.0f / kNearlyOne), heavy1 = __ballot(t.q[1] > 1.0f / kNearlyOne);
  if ((heavy0 | heavy1) != 0ull) {
    heavy = heavy0 != 0ull ? __builtin_amdgcn_readlane(t.at[0], __ffsll(heavy0) - 1) : __builtin_amdgcn_readlane(t.at[1], __ffsll(heavy1) - 1);
    rest = wave_sum((t.at[0] == heavy ? 0.0f : w[0]) + (t.at[1] == heavy ? 0.0f : w[1])) / sum;
#pragma unroll
    for (uint32_t u = 0; u < 2u; ++u)
      if (t.at[u] == heavy) t.log_q[u] = log1p_of(-rest);
  }
  const bool label_listed = label >= 0 && __any(t.at[0] == label || t.at[1] == label);
#pragma unroll
  for (uint32_t u = 0; u < 2u; ++u) {
    const uint32_t i = lane + 64u * u;
    if (i >= A.k) continue;
    to.at[i] = again[u] ? -1 : t.at[u];
    to.q[i] = t.q[u];
    to.z[i] = t.z[u];
  }
  if (lane == 0u) {
    to.at[A.k] = label_listed ? -1 : label;
    to.q[A.k] = 0.0f;
    to.z[A.k] = t.at_label;
    to.soft = sum;
    to.heavy = heavy;
    to.rest = rest;
  }
  return t;
}

// A row's sums as loss and gradient need them, at temperature T and at 1.
struct Softmaxes {
  float m, s, s1;
  Others others;
  __device__ __forceinline__ float log_s() const { return log_of_sum(s, others.x); }
  __device__ __forceinline__ float log_s1() const { return log_of_sum(s1, others.x1); }
};
template <Temperatures kTemps>
__device__ __forceinline__ Softmaxes softmaxes_of(const Sums& t, const Others& x) {
  if constexpr (kTemps == Temperatures::kOne) return Softmaxes{t.m, t.s, t.s, Others{x.x, x.x}};
  return Softmaxes{t.m, t.s, t.e, x};
}

// The row's loss, by the first wave.
__device__ __forceinline__ void put_loss(const DistillArgs& A, uint32_t r, const TeacherLane& l, bool softened, bool labelled, const Softmaxes& t) {
  float part = 0.0f;
  const float log_s = t.log_s();
#pragma unroll
  for (uint32_t u = 0; u < 2u; ++u)
    if (softened && l.at[u] >= 0 && !(l.q[u] == 0.0f)) part += l.q[u] * (l.log_q[u] - log_probability(l.z[u], t.m, A.inv_t, log_s));
  part = wave_sum(part);
  if (threadIdx.x == 0u) {
    float loss = softened ? A.soft_weight * A.temperature * A.temperature * part : 0.0f;
    if (labelled) loss -= A.label_weight * log_probability(l.at_label, t.m, 1.0f, t.log_s1());
    A.loss[r] = loss;
  }
}

// g [soft part of p^T + label part of p]: w = 2^((z - M) c) times (a + b w), or a w + b 2^((z - M) c1).
template <Temperatures kTemps>
struct Slope {
  float base, c, c1, a, b;
  __device__ __forceinline__ Slope(const DistillArgs& A, const Softmaxes& t, bool softened, bool labelled, float g) : base(base_of(t.m)), c(A.scale), c1(A.other_scale) {
    const float soft = softened && !(t.s == 0.0f) ? g * A.soft_weight * A.temperature / t.s : 0.0f;
    const float label = labelled && !(t.s1 == 0.0f) ? g * A.label_weight / t.s1 : 0.0f;
    a = kTemps == Temperatures::kOne ? soft + label : soft;
    b = label;
  }
  __device__ __forceinline__ float operator()(float z) const {
    const float d = z - base, w = exp2_of(d * c);
    if constexpr (kTemps == Temperatures::kOne) return a * w;
    if constexpr (kTemps == Temperatures::kSquared) return w * __fmaf_rn(b, w, a);
    return __fmaf_rn(b, exp2_of(d * c1), a * w);
  }
};

// The whole gradient at the label, and where the teacher has nearly all of its probability.  Of a probability near 1 fp32 keeps little beside the 1:
// 1 - p of a largest logit is the others' weights over the sum (of any other p is a half at most), and p^T - q is (1 - q) - (1 - p^T).
template <Temperatures kTemps>
__device__ __forceinline__ float slope_at(const DistillArgs& A, const Softmaxes& t, const Teacher& teacher, uint32_t i, int32_t label, bool softened, float g) {
  const float z = teacher.z[i], d = z - base_of(t.m), w = exp2_of(d * A.scale);
  const float w1 = kTemps == Temperatures::kOne ? w : kTemps == Temperatures::kSquared ? w * w : exp2_of(d * A.other_scale);
  const bool largest = z == t.m && !(t.s == 0.0f);
  const float of_s = t.s == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(t.s), of_s1 = t.s1 == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(t.s1);
  const float p = w * of_s, p1 = w1 * of_s1, not_p = largest ? t.others.x * of_s : 1.0f - p, not_p1 = largest ? t.others.x1 * of_s1 : 1.0f - p1;
  const float soft = teacher.at[i] == teacher.heavy ? teacher.rest - not_p : p - teacher.q[i], hard = teacher.at[i] == label ? -not_p1 : p1;
  return (softened ? g * A.soft_weight * A.temperature * soft : 0.0f) + (label >= 0 ? g * A.label_weight * hard : 0.0f);
}

template <typename T, uint32_t kThreads, uint32_t kVectors>
__device__ __forceinline__ void fill_zeros(T* dz, uint32_t n) {
  using V = Vector<T>;
  const uint32_t whole = n / V::kElems;
  const float zeros[V::kElems] = {};
  for (uint32_t i = threadIdx.x; i < whole; i += kThreads) V::store(dz + i * V::kElems, zeros);
  if (threadIdx.x < n - whole * V::kElems) dz[whole * V::kElems + threadIdx.x] = static_cast<T>(0.0f);
}

// The gradient of a held segment; then the entries of the teacher and the label over what was stored for them, each by the wave that
// stored it (a wave's stores to one address are done in order).
template <Temperatures kTemps, typename T, uint32_t kThreads, uint32_t kVectors>
__device__ __forceinline__ void put_gradient(const DistillArgs& A, const Held<T, kThreads, kVectors>& held, T* dz, uint32_t first, const Teacher& teacher, const Softmaxes& t,
                                             int32_t label, bool softened, float g) {
  const Slope<kTemps> slope(A, t, softened, label >= 0, g);
  const float of_teacher = softened ? g * A.soft_weight * A.temperature : 0.0f;
  using V = Vector<T>;
  held.each([&](uint32_t i, const float (&v)[V::kElems]) __attribute__((always_inline)) {
    float d[V::kElems];
#pragma unroll
    for (uint32_t j = 0; j < V::kElems; ++j) d[j] = slope(v[j]);
    if (held.mine(i)) V::store(dz + held.index(i), d);
  });
  if (held.has_single()) dz[held.single_index()] = static_cast<T>(slope(held.single));
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  for (uint32_t i = threadIdx.x & 63u; i <= A.k; i += 64u) {
    const uint32_t at = static_cast<uint32_t>(teacher.at[i]) - first;
    if (teacher.at[i] < 0 || at >= held.n) continue;
    if (held.owner(at) / 64u != threadIdx.x / 64u) continue;
    float d;
    if (teacher.at[i] == label || teacher.at[i] == teacher.heavy) d = slope_at<kTemps>(A, t, teacher, i, label, softened, g);
    else d = slope(teacher.z[i]) - of_teacher * teacher.q[i];
    dz[at] = static_cast<T>(d);
  }
}

// The row's label, -1: none.
__device__ __forceinline__ int32_t label_of(const DistillArgs& A, uint32_t r) {
  const int32_t target = A.targets ? A.targets[r] : -1;
  return is_token(target, A.vocab) ? target : -1;
}

template <Temperatures kTemps, typename H>
__device__ __forceinline__ Sums distill_sums(const H& held, const DistillArgs& A) {
  if constexpr (kTemps == Temperatures::kOne) return sums_of<Third::kNone, false>(held, A.scale, 0.0f);
  return sums_of<Third::kOther, kTemps == Temperatures::kSquared>(held, A.scale, A.other_scale);
}
template <Temperatures kTemps>
constexpr Third third_of() { return kTemps == Temperatures::kOne ? Third::kNone : Third::kOther; }

// A workgroup a row: loss and gradient.
template <typename T, uint32_t kThreads, uint32_t kVectors, Temperatures kTemps>
__global__ void __launch_bounds__(kThreads) distill_kernel(DistillArgs A) {
  __shared__ JoinShared<kThreads, kVectors> lds;
  __shared__ Teacher teacher;
  const uint32_t r = blockIdx.x;
  const T* z = row_of<T>(A.logits, A.row_stride, r);
  T* dz = static_cast<T*>(A.grad_logits) + static_cast<int64_t>(r) * A.grad_row_stride;
  const int32_t label = label_of(A, r);
  const bool labelled = label >= 0;
  if (!labelled && A.k == 0u) {
    if (threadIdx.x == 0u && A.loss) A.loss[r] = 0.0f;
    if (A.grad_logits) fill_zeros<T, kThreads, kVectors>(dz, A.vocab);
    return;
  }
  const Held<T, kThreads, kVectors> held(z, A.vocab);
  const float g = A.grad_loss ? A.grad_loss[r] : 1.0f;
  TeacherLane lane{};
  if (threadIdx.x < 64u) lane = teach(A, r, label, [&](uint32_t, int32_t i) { return static_cast<float>(z[i]); }, teacher);
  const Joined raw = block_join<third_of<kTemps>(), kTemps == Temperatures::kSquared>(held, distill_sums<kTemps>(held, A), A.scale, A.other_scale, lds);
  const Softmaxes t = softmaxes_of<kTemps>(spoiled(raw.t), raw.x);
  const bool softened = A.k > 0u && !(teacher.soft == 0.0f);
  if (A.loss && threadIdx.x < 64u) put_loss(A, r, lane, softened, labelled, t);
  if (!A.grad_logits) return;
  if (!softened && !labelled) fill_zeros<T, kThreads, kVectors>(dz, A.vocab);
  else put_gradient<kTemps>(A, held, dz, 0u, teacher, t, label, softened, g);
}

// Rows of several segments: the sums of each (and, by a row's first, the student's logits that the loss and the entries need, before
// a gradient can take their place), then the gradient of each with all of them.
template <typename T, uint32_t kThreads, uint32_t kVectors, Temperatures kTemps>
__global__ void __launch_bounds__(kThreads) distill_sums_kernel(DistillArgs A, SplitArgs P) {
  __shared__ JoinShared<kThreads, kVectors> lds;
  const uint32_t r = blockIdx.x / P.segments, segment = blockIdx.x - r * P.segments;
  const uint32_t first = segment * P.length, n = min(A.vocab - first, P.length);
  const T* z = row_of<T>(A.logits, A.row_stride, r);
  const int32_t label = label_of(A, r);
  const Held<T, kThreads, kVectors> held(z + first, n);
  if (segment == 0u && threadIdx.x < 64u) {
    float* to = P.logits + static_cast<uint64_t>(r) * (kTopMost + 1u);
    for (uint32_t i = threadIdx.x; i < A.k; i += 64u) {
      const int32_t at = A.teacher_idx[static_cast<uint64_t>(r) * A.k + i];
      if (is_token(at, A.vocab)) to[i] = static_cast<float>(z[at]);
    }
    if (threadIdx.x == 0u && label >= 0) to[kTopMost] = static_cast<float>(z[label]);
  }
  const Joined raw = block_join<third_of<kTemps>(), kTemps == Temperatures::kSquared>(held, distill_sums<kTemps>(held, A), A.scale, A.other_scale, lds);
  if (threadIdx.x == 0u) {
    float* to = P.sums + kDistillSums * blockIdx.x;
    to[0] = raw.t.m;
    to[1] = raw.t.s;
    to[2] = raw.t.e;
    to[3] = raw.x.x;
    to[4] = raw.x.x1;
  }
}

template <typename T, uint32_t kThreads, uint32_t kVectors, Temperatures kTemps>
__global__ void __launch_bounds__(kThreads) distill_gradient_kernel(DistillArgs A, SplitArgs P) {
  __shared__ Teacher teacher;
  const uint32_t r = blockIdx.x / P.segments, segment = blockIdx.x - r * P.segments, lane_id = threadIdx.x & 63u;
  const uint32_t first = segment * P.length, n = min(A.vocab - first, P.length);
  const T* z = row_of<T>(A.logits, A.row_stride, r) + first;
  T* dz = static_cast<T*>(A.grad_logits) + static_cast<int64_t>(r) * A.grad_row_stride + first;
  const int32_t label = label_of(A, r);
  const bool labelled = label >= 0;
  const Held<T, kThreads, kVectors> held(z, A.grad_logits ? n : 0u);
  const float g = A.grad_loss ? A.grad_loss[r] : 1.0f;
  Sums own = kNothing;
  Others x{};
  if (lane_id < P.segments) {
    const float* from = P.sums + kDistillSums * (static_cast<uint64_t>(r) * P.segments + lane_id);
    own = Sums{from[0], from[1], from[2]};
    x = Others{from[3], from[4]};
  }
  const Sums raw = wave_join<third_of<kTemps>()>(own, A.scale, A.other_scale);
  x = others_wanted<third_of<kTemps>()>(raw) ? others_join<third_of<kTemps>()>(own, x, raw, A.scale, A.other_scale) : Others{raw.s - 1.0f, raw.e - 1.0f};
  const Softmaxes t = softmaxes_of<kTemps>(spoiled(raw), x);
  TeacherLane lane{};
  const float* kept = P.logits + static_cast<uint64_t>(r) * (kTopMost + 1u);
  if (threadIdx.x < 64u) lane = teach(A, r, label, [&](uint32_t i, int32_t) { return kept[i]; }, teacher);
  __syncthreads();
  const bool softened = A.k > 0u && !(teacher.soft == 0.0f);
  if (A.loss && segment == 0u && threadIdx.x < 64u) put_loss(A, r, lane, softened, labelled, t);
  if (!A.grad_logits) return;
  if (!softened && !labelled) fill_zeros<T, kThreads, kVectors>(dz, n);
  else put_gradient<kTemps>(A, held, dz, first, teacher, t, label, softened, g);
}

// ---------------------------------------------------------------- launches

template <typename T, uint32_t kThreads_, uint32_t kVectors_>
struct Shape {
  using Type = T;
  static constexpr uint32_t kThreads = kThreads_, kVectors = kVectors_, kCapacity = Held<T, kThreads_, kVectors_>::kCapacity;
};

constexpr uint32_t kFewRows = 128, kFewSegments = 2, kWanted = 512, kManyRows = 2048, kFewWorkgroups = 256;

// f(shape): of the workgroups that hold `length` logits, the one of fewest threads.  (More alternatives than threads make a poor line: see top_of.)
// With fewer workgroups than compute units, of sixteen waves: one workgroup's time is all there is.
// kSegments: for segments as split_of cuts them, of which none is so short or just of that length; the last one holds any.
template <typename T, bool kSegments = false, typename F>
void by_length(uint32_t length, uint32_t top, uint64_t workgroups, F&& f) {
  if constexpr (!kSegments) {
    if (length <= Shape<T, 64, 4>::kCapacity && top <= 64u) return f(Shape<T, 64, 4>{});
  }
  if (length <= Shape<T, 256, 4>::kCapacity) return f(Shape<T, 256, 4>{});
  if (length <= Shape<T, 1024, 4>::kCapacity && workgroups <= kFewWorkgroups) return f(Shape<T, 1024, 4>{});
  if (length <= Shape<T, 256, 8>::kCapacity) return f(Shape<T, 256, 8>{});
  if (length <= Shape<T, 256, 16>::kCapacity) return f(Shape<T, 256, 16>{});
  if constexpr (!kSegments) {
    if (length <= Shape<T, 512, 16>::kCapacity) return f(Shape<T, 512, 16>{});
  }
  f(Shape<T, 1024, 16>{});
}

template <typename F>
void by_type(int dtype, F&& f) {
  if (dtype == 0) f(float{});
  else if (dtype == 1) f(__bf16{});
  else f(_Float16{});
}

}  // namespace

// How rows are cut, by what was measured (us; one segment / several).  The launch that joins them takes 3.
//  - Few rows of many logits: as many segments as give every compute unit two workgroups.  48 rows of 131072 with 20 alternatives 20.3 / 15.7, 4 such 18.9 / 18.3,
//    64 of 50257 few of whose words are allowed 43.3 / 22.3; 200 of 50257 take 14.2, in two 16.5, and stay whole.
//  - Scores of rows of three workgroups of four waves and more: these, for five of them share a compute unit and one's selection is hidden behind the others' reads.
//    1000 rows of 100003 with 20 alternatives 76.2 / 53.8, without 50.7 / 41.4, 300 of 131072 42.4 / 28.6.  Of two, where there are alternatives and many rows: 6001 of
//    50257 140 / 123, 4096 of 32000 in fp32 108 / 99 (without alternatives 87 / 95), but 700 of 33278 19.8 / 21.0.
//  - A gradient after the sums reads its row again if it does not hold it: one segment, as long as a workgroup holds the row.  (2048 rows of 131072 bf16 220, of 151936, which
//    none holds, 357; the floors are 211 and 245.)
SplitArgs split_of(uint32_t rows, uint32_t vocab, int dtype, Use use, uint32_t top) {
  SplitArgs P{};
  const uint32_t of = dtype == 0 ? 1u : 2u;                          // capacities: Shape<T, 256, 8>, <T, 256, 16> and <T, 1024, 16>
  const uint32_t small = Shape<float, 256, 8>::kCapacity * of, unit = Shape<float, 256, 16>::kCapacity * of, most = Shape<float, 1024, 16>::kCapacity * of;
  const uint32_t many = (vocab + small - 1u) / small, units = (vocab + unit - 1u) / unit, big = (vocab + most - 1u) / most;
  uint32_t segments = big;
  if (static_cast<uint64_t>(rows) * big < kFewRows && vocab > kFewSegments * small && many <= 64u)
    segments = min(64u, max(many, min((kWanted + rows - 1u) / rows, 2u * many)));
  else if (units <= 64u && (use == Use::kScores ? units >= 3u || (units == 2u && top > 0u && rows >= kManyRows) : big > 1u))
    segments = units;
  P.length = segments == 1u ? vocab : ((vocab + segments - 1u) / segments + 7u) / 8u * 8u;
  P.segments = (vocab + P.length - 1u) / P.length;
  return P;
}

namespace {

// f(first, rows): stretches of rows whose grids have fewer than 2^32 threads each.
template <typename F>
void by_rows(uint32_t rows, uint64_t threads_a_row, F&& f) {
  const uint64_t most = 0xFFFFFFFFull / threads_a_row;
  for (uint64_t first = 0; first < rows; first += most) f(first, static_cast<uint32_t>(rows - first < most ? rows - first : most));
}
template <typename P>
P* shifted(P* p, uint64_t by) { return p ? p + by : p; }
// A tensor of rows, by its type's size.
const void* shifted(const void* p, uint64_t rows, int64_t stride, int dtype) {
  return p ? static_cast<const char*>(p) + static_cast<int64_t>(rows) * stride * (dtype == 0 ? 4 : 2) : p;
}
void* shifted(void* p, uint64_t rows, int64_t stride, int dtype) { return const_cast<void*>(shifted(static_cast<const void*>(p), rows, stride, dtype)); }

}  // namespace

hipError_t launch_token_logprobs(const ScoreArgs& all, int dtype, const SplitArgs& P, hipStream_t s) {
  by_type(dtype, [&](auto type) {
    using T = decltype(type);
    by_length<T>(P.length, all.top, uint64_t(all.rows) * P.segments, [&](auto shape) {
      using S = decltype(shape);
      by_rows(all.rows, static_cast<uint64_t>(S::kThreads) * P.segments, [&](uint64_t first, uint32_t rows) {
        ScoreArgs a = all;
        a.rows = rows;
        a.logits = shifted(a.logits, first, a.row_stride, dtype);
        a.targets = shifted(a.targets, first);
        a.logprob = shifted(a.logprob, first);
        a.entropy = shifted(a.entropy, first);
        a.stats = shifted(a.stats, 2u * first);
        a.top_idx = shifted(a.top_idx, first * a.top);
        a.top_logprob = shifted(a.top_logprob, first * a.top);
        score_kernel<T, S::kThreads, S::kVectors><<<dim3(rows * P.segments), dim3(S::kThreads), 0, s>>>(a, P);
        if (P.segments > 1u) score_join_kernel<T><<<dim3(rows), dim3(kJoinThreads), P.segments * a.top * sizeof(uint64_t), s>>>(a, P);
      });
    });
  });
  return hipGetLastError();
}

hipError_t launch_token_logprobs_backward(const ScoreGradArgs& all, int dtype, hipStream_t s) {
  by_type(dtype, [&](auto type) {
    using T = decltype(type);
    const uint32_t part = kGradThreads * kGradVectors * Vector<T>::kElems, parts = (all.vocab + part - 1u) / part;
    const bool stream = uint64_t(all.rows) * all.vocab * sizeof(T) > kStreamFrom;
    by_rows(all.rows, static_cast<uint64_t>(kGradThreads) * parts, [&](uint64_t first, uint32_t rows) {
      ScoreGradArgs a = all;
      a.rows = rows;
      a.logits = shifted(a.logits, first, a.row_stride, dtype);
      a.grad_logits = shifted(a.grad_logits, first, a.grad_row_stride, dtype);
      a.targets = shifted(a.targets, first);
      a.stats = shifted(a.stats, 2u * first);
      a.entropy = shifted(a.entropy, first);
      a.grad_logprob = shifted(a.grad_logprob, first);
      a.grad_entropy = shifted(a.grad_entropy, first);
      if (stream) score_grad_kernel<T, true><<<dim3(rows * parts), dim3(kGradThreads), 0, s>>>(a, parts);
      else score_grad_kernel<T, false><<<dim3(rows * parts), dim3(kGradThreads), 0, s>>>(a, parts);
    });
  });
  return hipGetLastError();
}

hipError_t launch_distill(const DistillArgs& all, int dtype, const SplitArgs& P, hipStream_t s) {
  auto launch = [&](auto temps) {
    constexpr Temperatures kTemps = decltype(temps)::value;
    by_type(dtype, [&](auto type) {
      using T = decltype(type);
      auto run = [&](auto shape, auto split) {
        using S = decltype(shape);
        const dim3 threads(S::kThreads);
        by_rows(all.rows, static_cast<uint64_t>(S::kThreads) * P.segments, [&](uint64_t first, uint32_t rows) {
          DistillArgs a = all;
          a.rows = rows;
          a.logits = shifted(a.logits, first, a.row_stride, dtype);
          a.grad_logits = shifted(a.grad_logits, first, a.grad_row_stride, dtype);
          a.teacher_idx = shifted(a.teacher_idx, first * a.k);
          a.teacher_logits = shifted(a.teacher_logits, first * a.k);
          a.targets = shifted(a.targets, first);
          a.grad_loss = shifted(a.grad_loss, first);
          a.loss = shifted(a.loss, first);
          if constexpr (!decltype(split)::value) {
            distill_kernel<T, S::kThreads, S::kVectors, kTemps><<<dim3(rows), threads, 0, s>>>(a);
          } else {
            distill_sums_kernel<T, S::kThreads, S::kVectors, kTemps><<<dim3(rows * P.segments), threads, 0, s>>>(a, P);
            distill_gradient_kernel<T, S::kThreads, S::kVectors, kTemps><<<dim3(rows * P.segments), threads, 0, s>>>(a, P);
          }
        });
      };
      const uint64_t workgroups = uint64_t(all.rows) * P.segments;
      if (P.segments == 1u) by_length<T>(P.length, 0u, workgroups, [&](auto shape) { run(shape, std::false_type{}); });
      else by_length<T, true>(P.length, 0u, workgroups, [&](auto shape) { run(shape, std::true_type{}); });
    });
  };
  switch (all.temperatures) {
    case Temperatures::kOne: launch(std::integral_constant<Temperatures, Temperatures::kOne>{}); break;
    case Temperatures::kSquared: launch(std::integral_constant<Temperatures, Temperatures::kSquared>{}); break;
    default: launch(std::integral_constant<Temperatures, Temperatures::kTwo>{}); break;
  }
  return hipGetLastError();
}

}  // namespace rgc
