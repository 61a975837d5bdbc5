// Arguments of the language-model operators' kernels (rgc_vocab.hip, rgc_recurrence.hip, rgc_embed.hip, rgc_convolution.hip, rgc_scan.hip,
// rgc_scan_backward.hip, rgc_parts.hip), as the host side fills them.
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

struct EmbedArgs {
  const void* table;
  int64_t table_stride;
  uint32_t vocab, width;
  const int32_t* tokens;
  uint32_t rows;
  float scale;
  void* out;
  int64_t out_stride;
};

struct EmbedGradArgs {
  const void* dout;
  int64_t dout_stride;
  float* dtable;
  uint32_t add;              // dtable += instead of =
};

struct SequenceView {
  void* data;
  int64_t batch_stride, step_stride;
};

struct ConvArgs {
  uint32_t batch, steps, width;
  SequenceView x, y;
  const float* weight;       // [width][taps]
  const float* bias;
  uint32_t silu;
  const int32_t* lengths;
  const uint8_t* resets;
  const void* before;        // [batch][taps - 1][width]
  void* last;
};

struct ConvGradArgs {
  SequenceView dy, dx;
  float* dweight;
  float* dbias;
  const void* dlast;
  void* dbefore;
};

struct ScanArgs {
  uint32_t batch, steps, width, states, groups;
  uint32_t softplus;
  SequenceView x, delta, gate, b, c, y;
  const float* a;            // [width][states]
  const float* d;
  const float* delta_bias;
  const int32_t* lengths;
  const uint8_t* resets;
  const float* h0;           // [batch][width][states]
  float* h_last;
  float* kept;               // [batch][chunks][width][states]
};

struct ScanGradArgs {
  SequenceView dy, dx, ddelta, dgate, db, dc;
  float* da;
  float* dd;
  float* ddelta_bias;
  const float* dh_last;
  float* dh0;
};

// How a scan is cut along its steps, and what the pieces tell each other.
struct ScanCut {
  uint32_t chunks, stretch, stretches;   // chunks of a sequence, chunks of a stretch, stretches of a sequence
  uint32_t across, across_summary;       // workgroups for a group's channels, of the walk and of the summary
  float* starts;                         // [batch][stretches][width][states]
  float* sums;                           // [batch][stretches][width]
  uint32_t* cuts;                        // [batch][stretches]: a text begins in it
};

// Sums of [count][columns] parts over their rows; the columns are those of up to three outputs, one behind the other (a null one is left out).
struct PartsArgs {
  const float* parts;
  uint64_t count, columns;
  float* to[3];
  uint64_t ends[3];          // the column behind each one's last
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
hipError_t launch_embed(const EmbedArgs& a, int table_dtype, int dtype, hipStream_t s);
uint64_t embed_scratch_words(const EmbedArgs& a);
hipError_t launch_embed_backward(const EmbedArgs& a, const EmbedGradArgs& g, int dtype, unsigned long long* scratch, hipStream_t s);
hipError_t launch_sum_parts(const PartsArgs& a, hipStream_t s);
hipError_t launch_convolution(const ConvArgs& a, uint32_t taps, int dtype, hipStream_t s);
uint64_t convolution_scratch_words(const ConvArgs& a, uint32_t taps, int dtype);
hipError_t launch_convolution_backward(const ConvArgs& a, const ConvGradArgs& g, uint32_t taps, int dtype, unsigned long long* scratch, hipStream_t s);
hipError_t launch_scan(const ScanArgs& a, int dtype, unsigned long long* scratch, hipStream_t s);
uint64_t scan_scratch_words(const ScanArgs& a);
hipError_t launch_scan_backward(const ScanArgs& a, const ScanGradArgs& g, int dtype, unsigned long long* scratch, hipStream_t s);
uint64_t scan_backward_scratch_words(const ScanArgs& a);
bool recurrence_fits_grid(const RecurrenceArgs& a, int dtype, bool backward);
uint64_t recurrence_scratch_words(const RecurrenceArgs& a, int dtype, bool backward);      // 64-bit words of `scratch`
hipError_t launch_recurrence(const RecurrenceArgs& a, int dtype, unsigned long long* scratch, uint32_t looks, hipStream_t s);
hipError_t launch_recurrence_backward(const RecurrenceArgs& a, const RecurrenceGradArgs& g, int dtype, unsigned long long* scratch, uint32_t looks, hipStream_t s);

}  // namespace rgc
