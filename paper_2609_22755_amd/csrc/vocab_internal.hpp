// Internal host/device interface of the vocabulary's operators (embedding, log
// probabilities from hidden rows, distillation): arguments of the launchers.
#pragma once

#include "nsp_internal.hpp"
#include "vocab_plans.hpp"

namespace nsp {

// ----------------------------------- log probabilities from hidden rows --

struct LinearArgs {
  const char *x, *w;           // bf16
  int64_t x_stride, w_stride;  // elements
  const int64_t *targets;
  int64_t n_tokens;
  int32_t dim, vocab;
  float scale;
  // forward
  float *logp, *lse, *entropy;
  // backward
  const float *lse_in, *entropy_in, *g_logp, *g_lse, *g_entropy;
  char *dx, *dw;
  int64_t dx_stride, dw_stride;
  bool g_f32;
  char *ws;
};
hipError_t launch_linear_logp_fwd(const LinearArgs &a, hipStream_t s);
hipError_t launch_linear_logp_bwd(const LinearArgs &a, hipStream_t s);

// ------------------------------------------------------------ distillation --

constexpr int kDistillMaxTop = 256;
struct DistillArgs {
  const char *logits;
  int64_t row_stride, d_row_stride;
  const int64_t *index;        // [n_tokens][top]
  const float *teacher;
  int32_t n_tokens, vocab, top;
  bool normalized;
  float scale;
  float *loss, *lse;
  int32_t parts, part_len;     // parts a row, elements a part
  FastDiv by_parts;
  float4 *part_sums;
  const float *lse_in, *g_loss;
  char *dlogits;
};
hipError_t launch_distill_fwd(bool f32, const DistillArgs &a, hipStream_t s);
hipError_t launch_distill_bwd(bool f32, const DistillArgs &a, hipStream_t s);

// --------------------------------------------------------------- embedding --

struct EmbedArgs {
  const int64_t *tokens;
  int32_t n_tokens, vocab, dim;
  float scale;
  RowView w, y;                // backward: dw, dy
  plan::EmbedBwd f;
  char *ws;
};
hipError_t launch_embedding_fwd(bool w_f32, bool y_f32, const EmbedArgs &a, hipStream_t s);
hipError_t launch_embedding_bwd(bool w_f32, bool y_f32, const EmbedArgs &a, hipStream_t s);

}  // namespace nsp
