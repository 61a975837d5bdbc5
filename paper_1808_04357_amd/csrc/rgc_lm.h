// Arguments of the language-model operators' kernels (rgc_vocab.hip, rgc_recurrence.hip), as the host side fills them.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace rgc {

struct ScoreArgs {
  const void* logits;
  int64_t row_stride;
  uint32_t rows, vocab;
  const int32_t* targets;
  float scale, inv_t;        // log2(e) / T: what turns a difference of logits into an exponent of two; 1 / T
  uint32_t top;
  float* logprob;
  float* entropy;
  float* stats;
  int32_t* top_idx;
  float* top_logprob;
};

struct ScoreGradArgs {
  const void* logits;
  int64_t row_stride;
  uint32_t rows, vocab;
  const int32_t* targets;
  float scale, inv_t;
  const float* stats;
  const float* entropy;
  const float* grad_logprob;
  const float* grad_entropy;
  void* grad_logits;
  int64_t grad_row_stride;
};

// Which softmaxes of a row a distillation needs: one (T = 1, or only one of the two parts is on); at T = 2 and 1, the weights of the second being the squares of
// the first's; at another T and 1.
enum class Temperatures { kOne, kSquared, kTwo };

struct DistillArgs {
  const void* logits;
  int64_t row_stride;
  uint32_t rows, vocab;
  const int32_t* teacher_idx;
  const float* teacher_logits;
  uint32_t k;                // 0: no soft part
  const int32_t* targets;    // null: no labels
  float temperature, inv_t;
  float scale, other_scale;  // of the first softmax, log2(e) / T or log2(e), and of the second
  Temperatures temperatures;
  float soft_weight, label_weight;
  const float* grad_loss;
  float* loss;
  void* grad_logits;
  int64_t grad_row_stride;
};

// How rows are cut into segments (workgroups), and what those leave for each other where there are several.
struct SplitArgs {
  uint32_t segments, length;
  float* sums;               // [rows][segments][4], distillation [rows][segments][kDistillSums]
  uint64_t* entries;         // [rows][segments][top]: scores
  float* logits;             // [rows][RGC_TOP_MAX + 1]: distillation
};
constexpr uint64_t kDistillSums = 6;
enum class Use { kScores, kDistillation };
SplitArgs split_of(uint32_t rows, uint32_t vocab, int dtype, Use use, uint32_t top);

struct SequenceView {
  void* data;
  int64_t batch_stride, step_stride;
};

struct RecurrenceArgs {
  uint32_t batch, steps, width;
  SequenceView x, gate, out_gate, y;
  const int32_t* lengths;
  const uint8_t* resets;
  const float* h0;
  float* h_last;
  float* states;
};

struct RecurrenceGradArgs {
  SequenceView dy, dx, dgate, dout_gate;
  const float* dh_last;
  float* dh0;
};

// Looks of a few hundred nanoseconds each: seconds, where a tile in its turn waits for microseconds.
constexpr uint32_t kMostLooks = 1u << 23;

// How a recurrence is cut into tiles (workgroups), and what they tell each other.
struct TileArgs {
  uint32_t across, tiles;        // chains a sequence has (stretches of channels), tiles a chain has
  uint32_t groups;               // groups of tiles with another behind them
  unsigned long long* words;     // [chains][tiles, then groups][channels of a tile]
  uint32_t looks;                // how many times a tile looks for a word at most
  uint32_t* ticket;
};

hipError_t launch_token_logprobs(const ScoreArgs& a, int dtype, const SplitArgs& p, hipStream_t s);
hipError_t launch_token_logprobs_backward(const ScoreGradArgs& a, int dtype, hipStream_t s);
hipError_t launch_distill(const DistillArgs& a, int dtype, const SplitArgs& p, hipStream_t s);
bool recurrence_fits_grid(const RecurrenceArgs& a, int dtype, bool backward);
uint64_t recurrence_scratch_words(const RecurrenceArgs& a, int dtype, bool backward);      // 64-bit words of `scratch`
hipError_t launch_recurrence(const RecurrenceArgs& a, int dtype, unsigned long long* scratch, uint32_t looks, hipStream_t s);
hipError_t launch_recurrence_backward(const RecurrenceArgs& a, const RecurrenceGradArgs& g, int dtype, unsigned long long* scratch, uint32_t looks, hipStream_t s);

}  // namespace rgc
