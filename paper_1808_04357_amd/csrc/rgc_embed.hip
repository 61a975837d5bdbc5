// rgc_embed.hip -- rows of an embedding table, and the table's gradient (include/rgc.h has the formulas).
//
// Forward a wave takes a stretch of a row's channels: it is bound by the rows it reads and writes.
//
// Backward, dtable[v] = scale * sum of dout[r] over the rows r whose token is v, in an order that the tokens alone decide, without atomics.
//  1. The (token, row) pairs are put in order of the token, equal tokens in order of the row: few rows by counting, for each, the pairs that come before
//     it (rows^2 comparisons spread over the device, one launch), more of them by a radix sort of 8 bits a pass, whose blocks rank their rows with ballots.
//  2. The sorted pairs are cut into segments of kSegment, whatever runs of one token they hold.  A wave adds up a segment's runs for a stretch of channels; a run
//     that lies in one segment is stored at its place in the table, the part of one that goes on before or behind the segment into scratch.  The
//     same launch writes zeros where a token of the table does not occur, which it learns from the sorted pairs.
//  3. A workgroup for each run of several segments joins its parts: every wave adds up neighbouring ones in their order, then the waves' sums are added.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "rgc_lm.h"
#include "rgc_sequence.h"

namespace rgc {
namespace {

typedef unsigned long long Pair;       // token << 32 | row; tokens outside the vocabulary have `vocab`, behind all others

constexpr uint32_t kCounted = 4096;    // rows up to which pairs are ranked by counting
constexpr uint32_t kBlock = 1024;      // rows of a workgroup of the radix sort
constexpr uint32_t kFewBlocks = 64;    // of those, up to which each adds up the others' counts by itself
constexpr uint32_t kDigit = 8, kBins = 1u << kDigit;
constexpr uint32_t kSegment = 32;      // pairs of a segment
constexpr uint32_t kJoinWaves = 4;
constexpr uint32_t kFillRows = 8;      // rows of the table that a wave looks after

__device__ __forceinline__ uint32_t known(int32_t token, uint32_t vocab) {
  return static_cast<uint32_t>(token) < vocab ? static_cast<uint32_t>(token) : vocab;
}

// ---------------------------------------------------------------------------------------------------------------------------------- forward

// One wave: kBlocks stretches of 64 kVec channels of one row.
template <typename S, typename T, int kVec, int kBlocks>
__global__ void __launch_bounds__(256) embed_kernel(EmbedArgs A, uint32_t across, uint64_t begin, uint64_t waves) {
  const uint64_t at = (begin + blockIdx.x) * 4u + (threadIdx.x >> 6);
  if (at >= waves) return;
  const uint32_t row = uniform(static_cast<uint32_t>(at / across)), first = uniform(static_cast<uint32_t>(at % across)) * kBlocks;
  const uint32_t token = uniform(known(A.tokens[row], A.vocab));
  const S* from = static_cast<const S*>(A.table) + static_cast<int64_t>(token) * A.table_stride;
  T* to = static_cast<T*>(A.out) + static_cast<int64_t>(row) * A.out_stride;
  Raw<S, kVec> r[kBlocks];
  if (token < A.vocab) {
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) r[j] = read_at<S, kVec>(from + Channels<kVec>(first + j, A.width).c);
  }
#pragma unroll
  for (int j = 0; j < kBlocks; ++j) {
    const Channels<kVec> lane(first + j, A.width);
    float v[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = token < A.vocab ? static_cast<float>(r[j].v[i]) * A.scale : 0.0f;
    write_own<T, kVec>(to, lane, v);
  }
}

// ---------------------------------------------------------------------------------------------------------------------------------- order

// One wave a row: how many pairs come before its own.
__global__ void __launch_bounds__(256) rank_kernel(const int32_t* tokens, uint32_t rows, uint32_t vocab, Pair* sorted) {
  const uint32_t row = blockIdx.x * 4u + (threadIdx.x >> 6), lane = threadIdx.x & 63u;
  if (row >= rows) return;
  const uint32_t mine = uniform(known(tokens[row], vocab));
  uint32_t before = 0u;
#pragma unroll 4
  for (uint32_t i = lane; i < rows; i += 64u) {
    const uint32_t other = known(tokens[i], vocab);
    before += other < mine || (other == mine && i < row) ? 1u : 0u;
  }
  for (uint32_t m = 32u; m > 0u; m >>= 1) before += __shfl_xor(before, m);
  if (lane == 0u) sorted[before] = (static_cast<Pair>(mine) << 32) | row;
}

// The pairs of a radix pass: the first one makes them of the tokens.
__device__ __forceinline__ Pair pair_at(const Pair* from, const int32_t* tokens, uint32_t vocab, uint32_t i) {
  return from ? from[i] : (static_cast<Pair>(known(tokens[i], vocab)) << 32) | i;
}

// counts[digit][block]: how many of a block's pairs have the digit.
__global__ void __launch_bounds__(1024) count_kernel(const Pair* from, const int32_t* tokens, uint32_t rows, uint32_t vocab, uint32_t shift, uint32_t* counts) {
  __shared__ uint32_t bins[kBins];
  if (threadIdx.x < kBins) bins[threadIdx.x] = 0u;
  __syncthreads();
  for (uint32_t j = 0; j < kBlock / 1024u; ++j) {
    const uint64_t i = static_cast<uint64_t>(blockIdx.x) * kBlock + j * 1024u + threadIdx.x;
    if (i < rows) atomicAdd(&bins[(pair_at(from, tokens, vocab, static_cast<uint32_t>(i)) >> (32u + shift)) & (kBins - 1u)], 1u);
  }
  __syncthreads();
  if (threadIdx.x < kBins) counts[static_cast<uint64_t>(threadIdx.x) * gridDim.x + blockIdx.x] = bins[threadIdx.x];
}

// Counts become what comes before them: within their digit here (one workgroup a digit), over the digits in the next kernel.
__global__ void __launch_bounds__(1024) prefix_kernel(uint32_t* counts, uint32_t blocks, uint32_t* totals) {
  __shared__ uint32_t waves[16];
  uint32_t* const mine = counts + static_cast<uint64_t>(blockIdx.x) * blocks;
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
  uint32_t carry = 0u;
  for (uint32_t first = 0; first < blocks; first += 1024u) {
    const uint32_t i = first + threadIdx.x, n = i < blocks ? mine[i] : 0u;
    uint32_t sum = n;
    for (uint32_t d = 1u; d < 64u; d <<= 1) {
      const uint32_t other = __shfl_up(sum, d);
      if (lane >= d) sum += other;
    }
    if (lane == 63u) waves[wave] = sum;
    __syncthreads();
    uint32_t before = carry, all = 0u;
    for (uint32_t w = 0; w < 16u; ++w) {
      if (w < wave) before += waves[w];
      all += waves[w];
    }
    if (i < blocks) mine[i] = before + sum - n;
    carry += all;
    __syncthreads();
  }
  if (threadIdx.x == 0u) totals[blockIdx.x] = carry;
}

// Puts a block's pairs where their digit's come, in their order (totals == null: `before` holds the counts themselves): ranks within a wave by ballots, between waves by their counts.
__global__ void __launch_bounds__(1024) place_kernel(const Pair* from, const int32_t* tokens, uint32_t rows, uint32_t vocab, uint32_t shift, const uint32_t* before,
                                                     const uint32_t* totals, Pair* to) {
  constexpr uint32_t kRounds = kBlock / 1024u;
  __shared__ uint32_t bins[16][kBins], start[kBins];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
  for (uint32_t i = threadIdx.x; i < 16u * kBins; i += 1024u) (&bins[0][0])[i] = 0u;
  uint32_t here = 0u;                                 // of the digit, in the blocks before
  if (threadIdx.x < kBins) {
    const uint32_t* mine = before + static_cast<uint64_t>(threadIdx.x) * gridDim.x;
    if (totals) {
      here = mine[blockIdx.x];
      start[threadIdx.x] = totals[threadIdx.x];
    } else {
      uint32_t all = 0u;
#pragma unroll 8
      for (uint32_t i = 0; i < gridDim.x; ++i) {
        const uint32_t n = mine[i];
        all += n;
        here += i < blockIdx.x ? n : 0u;
      }
      start[threadIdx.x] = all;
    }
  }
  __syncthreads();
  if (wave == 0u) {                                   // where each digit begins
    uint32_t n[kBins / 64u], sum = 0u;
    for (uint32_t j = 0; j < kBins / 64u; ++j) n[j] = start[lane * (kBins / 64u) + j], sum += n[j];
    uint32_t upto = sum;
    for (uint32_t d = 1u; d < 64u; d <<= 1) {
      const uint32_t other = __shfl_up(upto, d);
      if (lane >= d) upto += other;
    }
    uint32_t at = upto - sum;
    for (uint32_t j = 0; j < kBins / 64u; ++j) start[lane * (kBins / 64u) + j] = at, at += n[j];
  }
  const uint64_t first = static_cast<uint64_t>(blockIdx.x) * kBlock + wave * (64u * kRounds);
  Pair pair[kRounds];
  uint32_t rank[kRounds];
#pragma unroll
  for (uint32_t j = 0; j < kRounds; ++j) {
    const uint64_t i = first + j * 64u + lane;
    const bool there = i < rows;
    pair[j] = there ? pair_at(from, tokens, vocab, static_cast<uint32_t>(i)) : 0ull;
    const uint32_t digit = static_cast<uint32_t>(pair[j] >> (32u + shift)) & (kBins - 1u);
    unsigned long long same = __ballot(there);
#pragma unroll
    for (uint32_t b = 0; b < kDigit; ++b) {
      const unsigned long long ones = __ballot(((digit >> b) & 1u) != 0u);
      same &= ((digit >> b) & 1u) != 0u ? ones : ~ones;
    }
    const uint32_t ahead = static_cast<uint32_t>(__popcll(same & ((1ull << lane) - 1ull)));
    if (there) {
      rank[j] = bins[wave][digit] + ahead;
      __builtin_amdgcn_wave_barrier();
      if (ahead == 0u) bins[wave][digit] = rank[j] + static_cast<uint32_t>(__popcll(same));
    }
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  if (threadIdx.x < kBins) {
    uint32_t at = start[threadIdx.x] + here;
    for (uint32_t w = 0; w < 16u; ++w) {
      const uint32_t n = bins[w][threadIdx.x];
      bins[w][threadIdx.x] = at;
      at += n;
    }
  }
  __syncthreads();
#pragma unroll
  for (uint32_t j = 0; j < kRounds; ++j) {
    const uint64_t i = first + j * 64u + lane;
    if (i < rows) to[bins[wave][static_cast<uint32_t>(pair[j] >> (32u + shift)) & (kBins - 1u)] + rank[j]] = pair[j];
  }
}

// ---------------------------------------------------------------------------------------------------------------------------------- sums

struct Sums {
  const Pair* sorted;
  float* parts;                        // [segments][2][width]: of the run that began before the segment (or is all of it), of the one that goes on behind it
  uint32_t segments, across;           // stretches of 64 kVec channels
};

__device__ __forceinline__ uint32_t token_of(Pair p) { return static_cast<uint32_t>(p >> 32); }

// The first pair whose token is at least `token`: a wave looks at 64 places at a time.
__device__ __forceinline__ uint32_t lower_bound(const Pair* sorted, uint32_t rows, uint32_t token) {
  uint32_t first = 0u, n = rows;                      // it lies in [first, first + n]
  while (n > 0u) {
    const uint32_t step = (n + 63u) / 64u, i = (threadIdx.x & 63u) * step;
    const bool less = i < n && token_of(sorted[first + i]) < token;
    const uint32_t smaller = static_cast<uint32_t>(__popcll(__ballot(less)));      // of the places looked at
    if (smaller == 0u) return first;
    const uint32_t from = (smaller - 1u) * step + 1u, to = min(smaller * step, n);
    first += from;
    n = to - from;
  }
  return first;
}

// A row's sums to their place.
template <int kVec>
__device__ __forceinline__ void put(float* row, const Channels<kVec>& lane, float (&v)[kVec], float scale, uint32_t add) {
#pragma unroll
  for (int i = 0; i < kVec; ++i) v[i] *= scale;
  if (add) {
    const Raw<float, kVec> old = read_at<float, kVec>(row + lane.c);
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] += old.v[i];
  }
  write_own<float, kVec>(row, lane, v);
}

// Zeros where the table has tokens that do not occur.
template <int kVec>
__device__ __forceinline__ void fill(const EmbedArgs& A, const EmbedGradArgs& G, const Sums& S, uint64_t at) {
  const uint32_t group = static_cast<uint32_t>(at), first = uniform(group * kFillRows), end = min(first + kFillRows, A.vocab);
  uint32_t p = lower_bound(S.sorted, A.rows, first);
  uint32_t there = 0u;                                // bit: the token occurs
  while (true) {
    // (one load a round; a run longer than a wave is left by another search)
    const uint32_t i = p + (threadIdx.x & 63u);
    const uint32_t token = i < A.rows ? token_of(S.sorted[i]) : A.vocab;
    const bool inside = token < end;
    uint32_t bits = inside ? 1u << (token - first) : 0u;
    for (uint32_t m = 32u; m > 0u; m >>= 1) bits |= __shfl_xor(bits, m);
    there |= bits;
    if (!__all(inside)) break;
    const uint32_t last = uniform(__shfl(token, 63));
    if (last + 1u >= end) break;
    p = lower_bound(S.sorted, A.rows, last + 1u);
  }
  there = uniform(there);
  for (uint32_t j = 0; first + j < end; ++j) {
    if ((there >> j) & 1u) continue;
    float* to = G.dtable + static_cast<uint64_t>(first + j) * A.width;
    for (uint32_t b = 0; b < S.across; ++b) {
      const Channels<kVec> lane(b, A.width);
      const float zero[kVec] = {};
      write_own<float, kVec>(to, lane, zero);
    }
  }
}

template <typename T, int kVec>
__global__ void __launch_bounds__(256) sum_kernel(EmbedArgs A, EmbedGradArgs G, Sums S, uint64_t fills, uint64_t begin, uint64_t waves) {
  constexpr uint32_t kAtOnce = 8;
  uint64_t at = (begin + blockIdx.x) * 4u + (threadIdx.x >> 6);
  if (at >= waves) return;
  const uint64_t sums = waves - fills;
  if (at >= sums) return fill<kVec>(A, G, S, at - sums);
  const uint32_t segment = uniform(static_cast<uint32_t>(at / S.across)), block = uniform(static_cast<uint32_t>(at % S.across));
  const Channels<kVec> lane(block, A.width);
  const uint32_t first = segment * kSegment, n = min(kSegment, A.rows - first);
  const uint32_t l = threadIdx.x & 63u;
  // the segment's pairs, the one before and the one behind it
  const int64_t place = static_cast<int64_t>(first) - 1 + l;
  const Pair pair = place >= 0 && place < static_cast<int64_t>(A.rows) && l <= n + 1u ? S.sorted[place] : ~0ull;
  const uint32_t token = token_of(pair), row = static_cast<uint32_t>(pair);
  const bool entered = first > 0u;                    // (there is a pair before)
  float sum[kVec] = {};
  uint32_t now = uniform(__shfl(token, 1));
  bool from_before = entered && uniform(__shfl(token, 0)) == now;
  auto leave = [&](bool goes_on) {
    if (now >= A.vocab) return;                       // (uniform)
    if (from_before || goes_on) {
      write_own<float, kVec>(S.parts + (static_cast<uint64_t>(segment) * 2u + (from_before ? 0u : 1u)) * A.width, lane, sum);
    } else {
      put<kVec>(G.dtable + static_cast<uint64_t>(now) * A.width, lane, sum, A.scale, G.add);
    }
  };
  for (uint32_t i = 0; i < n; i += kAtOnce) {
    Raw<T, kVec> v[kAtOnce];
#pragma unroll
    for (uint32_t j = 0; j < kAtOnce; ++j) {          // (behind the segment's end the last row again; what a left out row holds is not used)
      const uint32_t r = uniform(__shfl(row, min(i + j, n - 1u) + 1u));
      v[j] = read_at<T, kVec>(static_cast<const T*>(G.dout) + static_cast<int64_t>(r) * G.dout_stride + lane.c);
    }
#pragma unroll
    for (uint32_t j = 0; j < kAtOnce; ++j) {
      if (i + j >= n) continue;
      const uint32_t t = uniform(__shfl(token, i + j + 1u));
      if (t != now) {
        leave(false);
        now = t;
        from_before = false;
#pragma unroll
        for (int c = 0; c < kVec; ++c) sum[c] = 0.0f;
      }
      if (t < A.vocab) {
#pragma unroll
        for (int c = 0; c < kVec; ++c) sum[c] += static_cast<float>(v[j].v[c]);
      }
    }
  }
  leave(first + n < A.rows && uniform(__shfl(token, n + 1u)) == now);
}

// A run of several segments that begins in this one: its parts are this segment's second and the first of those after it.
// One workgroup joins a run however long.  us, the whole call, bf16: 32768 rows x 2048 of 50257 words, tokens all over / one token in half / in all of the rows 139 / 149 / 155; 1048577 x 64, where a
// run has up to 32769 parts, 160 / 334 / 539.
template <int kVec>
__global__ void __launch_bounds__(64 * kJoinWaves) join_kernel(EmbedArgs A, EmbedGradArgs G, Sums S, uint64_t begin) {
  __shared__ float sums[kJoinWaves][64 * kVec];
  const uint64_t at = begin + blockIdx.x;
  const uint32_t segment = static_cast<uint32_t>(at / S.across), block = static_cast<uint32_t>(at % S.across), wave = uniform(threadIdx.x >> 6), l = threadIdx.x & 63u;
  const uint32_t first = segment * kSegment, next = first + kSegment;
  if (next >= A.rows) return;
  // (asked for at once: most runs do not span segments, and their workgroups are gone with that)
  const Pair behind = S.sorted[next], last = S.sorted[next - 1u], before = S.sorted[first > 0u ? first - 1u : 0u];
  const uint32_t token = uniform(token_of(behind));
  if (token >= A.vocab || uniform(token_of(last)) != token || (first > 0u && uniform(token_of(before)) == token)) return;     // (the last: it began before)
  const uint32_t end = lower_bound(S.sorted, A.rows, token + 1u);
  const uint32_t parts = (end - 1u) / kSegment - segment + 1u, each = (parts + kJoinWaves - 1u) / kJoinWaves;
  const Channels<kVec> lane(block, A.width);
  float sum[kVec] = {};
  const uint32_t upto = min(parts, (wave + 1u) * each);
#pragma unroll 8
  for (uint32_t p = wave * each; p < upto; ++p) {
    const Raw<float, kVec> v = read_at<float, kVec>(S.parts + (static_cast<uint64_t>(segment + p) * 2u + (p == 0u ? 1u : 0u)) * A.width + lane.c);
#pragma unroll
    for (int i = 0; i < kVec; ++i) sum[i] += v.v[i];
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i) sums[wave][i * 64 + l] = sum[i];
  __syncthreads();
  if (wave > 0u) return;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    for (uint32_t w = 1; w < kJoinWaves; ++w) sum[i] += sums[w][i * 64 + l];
  }
  put<kVec>(G.dtable + static_cast<uint64_t>(token) * A.width, lane, sum, A.scale, G.add);
}

// ---------------------------------------------------------------------------------------------------------------------------------- launches

uint32_t stretches(uint32_t width, uint32_t vec) { return (width + 64u * vec - 1u) / (64u * vec); }
uint32_t blocks_of(uint32_t rows) { return static_cast<uint32_t>((static_cast<uint64_t>(rows) + kBlock - 1u) / kBlock); }
uint32_t segments_of(uint32_t rows) { return static_cast<uint32_t>((static_cast<uint64_t>(rows) + kSegment - 1u) / kSegment); }

template <typename S, typename T>
void launch_forward(const EmbedArgs& a, hipStream_t s) {
  // 16 bytes of the narrower type a lane, fewer where a row has not that many channels
  constexpr int kMost = sizeof(S) == 4 && sizeof(T) == 4 ? 4 : 8;
  auto go = [&](auto vec, auto blocks) {
    constexpr int kVec = decltype(vec)::value, kBlocks = decltype(blocks)::value;
    const uint32_t across = (stretches(a.width, kVec) + kBlocks - 1u) / kBlocks;
    const uint64_t waves = static_cast<uint64_t>(a.rows) * across;
    in_grids((waves + 3u) / 4u, [&](uint64_t begin, dim3 grid) { embed_kernel<S, T, kVec, kBlocks><<<grid, dim3(256), 0, s>>>(a, across, begin, waves); });
  };
  if (a.width < kMost) go(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{});
  else if (a.width <= 64u * kMost) go(std::integral_constant<int, kMost>{}, std::integral_constant<int, 1>{});
  else go(std::integral_constant<int, kMost>{}, std::integral_constant<int, 2>{});
}

template <typename S>
void launch_forward(const EmbedArgs& a, int dtype, hipStream_t s) {
  if (dtype == 0) launch_forward<S, float>(a, s);
  else if (dtype == 1) launch_forward<S, __bf16>(a, s);
  else launch_forward<S, _Float16>(a, s);
}

template <typename T, int kVec>
hipError_t launch_sums(const EmbedArgs& a, const EmbedGradArgs& g, Sums S, hipStream_t s) {
  S.across = stretches(a.width, kVec);
  const uint64_t fills = g.add ? 0u : (static_cast<uint64_t>(a.vocab) + kFillRows - 1u) / kFillRows;
  const uint64_t waves = static_cast<uint64_t>(S.segments) * S.across + fills;
  in_grids((waves + 3u) / 4u, [&](uint64_t begin, dim3 grid) { sum_kernel<T, kVec><<<grid, dim3(256), 0, s>>>(a, g, S, fills, begin, waves); });
  if (S.segments > 1u) {
    in_grids(static_cast<uint64_t>(S.segments) * S.across, [&](uint64_t begin, dim3 grid) { join_kernel<kVec><<<grid, dim3(64 * kJoinWaves), 0, s>>>(a, g, S, begin); });
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(const EmbedArgs& a, int table_dtype, int dtype, hipStream_t s) {
  if (table_dtype == 0) launch_forward<float>(a, dtype, s);
  else if (table_dtype == 1) launch_forward<__bf16>(a, dtype, s);
  else launch_forward<_Float16>(a, dtype, s);
  return hipGetLastError();
}

// Sorted pairs, the other half of the radix sort's, its counts, and the parts of runs.
uint64_t embed_scratch_words(const EmbedArgs& a) {
  if (a.rows == 0u) return 0u;
  uint64_t words = a.rows;
  if (a.rows > kCounted) words += a.rows + (static_cast<uint64_t>(blocks_of(a.rows)) * kBins + kBins + 1u) / 2u;
  return words + static_cast<uint64_t>(segments_of(a.rows)) * a.width;
}

hipError_t launch_embed_backward(const EmbedArgs& a, const EmbedGradArgs& g, int dtype, unsigned long long* scratch, hipStream_t s) {
  Sums S{};
  S.segments = segments_of(a.rows);
  Pair* sorted = scratch;
  unsigned long long* behind = scratch + a.rows;
  if (a.rows > kCounted) {
    Pair* other = behind;
    uint32_t* counts = reinterpret_cast<uint32_t*>(other + a.rows);
    const uint32_t blocks = blocks_of(a.rows);
    uint32_t* totals = counts + static_cast<uint64_t>(blocks) * kBins;
    behind = other + a.rows + (static_cast<uint64_t>(blocks) * kBins + kBins + 1u) / 2u;
    uint32_t passes = 1u;
    while (passes < 4u && (a.vocab >> (kDigit * passes)) != 0u) ++passes;
    const Pair* from = nullptr;
    for (uint32_t p = 0; p < passes; ++p) {
      Pair* to = (passes - 1u - p) % 2u == 0u ? sorted : other;      // the last pass into `sorted`
      count_kernel<<<dim3(blocks), dim3(1024), 0, s>>>(from, a.tokens, a.rows, a.vocab, p * kDigit, counts);
      if (blocks > kFewBlocks) prefix_kernel<<<dim3(kBins), dim3(1024), 0, s>>>(counts, blocks, totals);
      place_kernel<<<dim3(blocks), dim3(1024), 0, s>>>(from, a.tokens, a.rows, a.vocab, p * kDigit, counts, blocks > kFewBlocks ? totals : nullptr, to);
      from = to;
    }
  } else if (a.rows > 0u) {
    rank_kernel<<<dim3((a.rows + 3u) / 4u), dim3(256), 0, s>>>(a.tokens, a.rows, a.vocab, sorted);
  }
  S.sorted = sorted;
  S.parts = reinterpret_cast<float*>(behind);
  auto go = [&](auto type) {
    using T = decltype(type);
    return a.width < 4u ? launch_sums<T, 1>(a, g, S, s) : launch_sums<T, 4>(a, g, S, s);
  };
  return dtype == 0 ? go(float{}) : dtype == 1 ? go(__bf16{}) : go(_Float16{});
}

}  // namespace rgc
