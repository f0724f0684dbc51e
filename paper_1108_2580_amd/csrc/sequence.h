// Internal declarations of the sequence operators: norm and rotation of queries and keys
// (rotate.hip), attention with a decay for each head (attention.hip), attention over gaps of time (gap.hip,
// gap_back.hip, gap_step.hip), tokens of no row (unheld.hip) and beam selection (beam.hip). Host entries:
// sequence.hip.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "als.h"

namespace als {

// Records the message of a failing call that has no context (api.hip); returns st.
als_status fail_without_context(als_status st, const char *fmt, ...);

using f32x4 = float __attribute__((ext_vector_type(4)));
using bf16 = __bf16;
using bf16x4 = bf16 __attribute__((ext_vector_type(4)));
using bf16x8 = bf16 __attribute__((ext_vector_type(8)));

// Whether rows of `width` elements of `size` bytes at this base and these strides (elements) can
// be read 16 bytes at a time.
inline bool aligned16(const void *p, int64_t token_stride, int64_t head_stride, int width,
                      int size) {
  return ((uintptr_t)p | (uint64_t)(token_stride * size) | (uint64_t)(head_stride * size) |
          (uint64_t)(width * size)) % 16 == 0;
}

// The largest stride of attention's tokens (values): a chunk is addressed with 32-bit offsets.
constexpr int64_t kMaxTokenStride = 1 << 22;

// One pass of decayed attention over packed rows of tokens; the gradients are passes of the same
// form (attention.hip).
struct AttentionPass {
  int64_t n_tokens, n_rows;
  int32_t heads, group;   // heads of q, and how many of them share one head of k and v
  int32_t k_width, v_width;
  als_heads q, k, v;      // data null in q: states only
  int32_t q_group = 1;    // heads that share one head of q (a gradient pass reads k there)
  int32_t v_group = 1;    // and of v
  const float *log_decay;
  const int64_t *row_ptr;
  float weight_scale;     // of the products of tokens
  float update_scale;     // of what a token adds to the state
  float read_scale;       // of what is read from the state
  bool reverse;           // from each row's last token to its first
  const float *first_state;  // nullable, [n_rows, heads, ...]; element (i, j) at i * first_ld[0] + j * first_ld[1]
  int64_t first_ld[2];
  float *last_state;         // nullable, the same
  int64_t last_ld[2];
  void *out;              // [n_tokens, heads, v_width], packed
  bool out_f32;           // out is fp32 whatever the type of the inputs
  // workspace (attention_space), each null where its size is 0
  void *places;           // of the segments, written by launch_places
  int32_t *entries;
  float *segments;        // states of the segments
  bool shares_segments;   // they are another pass's, whose state is this one's transposed
  // set by launch_attention
  int64_t segment_ld[2];
  bool vec_in;            // q, k and v are read 16 bytes at a time
};

// Bytes of a pass's workspace, by part, each a multiple of 16.
struct AttentionSpace {
  int64_t places, entries, states;
  int64_t total() const { return places + entries + states; }
};

// log2 of the tokens a segment: longer rows are cut and their segments run side by side.
int attention_shift(als_dtype dtype, int64_t n_tokens, int32_t heads);
AttentionSpace attention_space(als_dtype dtype, int64_t n_tokens, int64_t n_rows, int32_t heads,
                               int k_width, int v_width);
// Fills p.places and p.entries, which all passes over the same rows and heads share.
hipError_t launch_places(als_dtype dtype, const AttentionPass &p, hipStream_t s);
// Up to three passes over the same rows and heads. One that shares segments comes after its owner.
hipError_t launch_attention(als_dtype dtype, const AttentionPass *p, int n, hipStream_t s);
// dk[t, h, d] = sum over the head's group of of_k[t, h * group + i, d], in order; dv likewise.
hipError_t launch_sum_groups(als_dtype dtype, const float *of_k, const float *of_v, int64_t n_tokens,
                             int32_t heads, int32_t group, int32_t k_width, int32_t v_width, void *dk,
                             void *dv, hipStream_t s);
hipError_t launch_attention_step(als_dtype dtype, int64_t n_rows, int32_t heads, int32_t group,
                                 int32_t k_width, int32_t v_width, const als_heads &q,
                                 const als_heads &k, const als_heads &v, const float *log_decay,
                                 float scale, const float *state, const int32_t *source,
                                 int64_t n_sources, float *state_out, void *out, hipStream_t s);

// Attention over gaps of time (gap.hip, gap_back.hip, gap_step.hip): what all its calls share.
struct GapShape {
  int64_t n_tokens, n_rows;
  const int64_t *row_ptr;
  const int32_t *positions;
  const float *bias;       // [heads, buckets]
  int32_t heads, group;    // heads of q, and how many of them share one head of k and v
  int32_t width, buckets;
  float scale;
  bool clear_unheld;       // whether tokens of no row get zeros
  int32_t last_bound;      // bounds[buckets - 2], 0 where there is one bucket
  int32_t bounds[63];
};
// Bytes of the table of the tokens' rows, which calls over more than a few rows need.
int64_t gap_spans_bytes(int64_t n_tokens, int64_t n_rows);
hipError_t launch_gap_spans(const GapShape &g, void *spans, hipStream_t s);
// stats: nullable, fp32 [2, heads, n_tokens], the largest score (times log2 e) and one over the sum;
// rest: nullable, like out, what its rounding to bf16 left out.
hipError_t launch_gap_read(als_dtype dtype, const GapShape &g, const als_heads &q, const als_heads &k,
                           const als_heads &v, const void *spans, void *out, float *stats, int16_t *rest,
                           hipStream_t s);

// Bytes of the gradients' workspace, by part, each a multiple of 16.
struct GapBackSpace {
  int64_t spans, delta, dbias, heads;
  int64_t total() const { return spans + delta + dbias + 2 * heads; }
};
GapBackSpace gap_back_space(int64_t n_tokens, int64_t n_rows, int32_t heads, int32_t k_heads, int32_t width,
                            int32_t buckets);
hipError_t launch_gap_back(als_dtype dtype, const GapShape &g, const als_heads &d_out, const als_heads &q,
                           const als_heads &k, const als_heads &v, const void *out, const float *stats,
                           const int16_t *rest, void *dq, void *dk, void *dv, float *dbias, void *workspace,
                           hipStream_t s);

// One token of each beam: what it reads besides its list's row of the history.
struct GapPath {
  int32_t beams, steps;
  const int32_t *q_positions;  // [lists * beams]
  als_heads k, v;              // [steps, lists * beams, heads, width]
  int64_t k_step, v_step;      // values from step to step
  const int32_t *positions;    // [steps, lists * beams]
  const int32_t *path;         // [lists * beams, steps], rows path_stride apart: the beam that holds each step
  int64_t path_stride;
};
int64_t gap_step_space(int64_t n_tokens, int64_t n_lists, int32_t heads, int32_t k_heads, int32_t beams,
                       int32_t width);
hipError_t launch_gap_step(als_dtype dtype, const GapShape &g, const GapPath &p, const als_heads &q,
                           const als_heads &k, const als_heads &v, void *out, void *workspace, hipStream_t s);

// Packed tensors to clear at the tokens that no row holds (unheld.hip).
struct Unheld {
  int32_t n;
  char *data[3];
  int64_t token_bytes[3];
};
hipError_t launch_clear_unheld(int64_t n_tokens, int64_t n_rows, const int64_t *row_ptr, const Unheld &u,
                               hipStream_t s);

// Blocks of a pass of norm and rotation: partial sums of the weights' gradients (rotate.hip).
int64_t rotate_blocks(int64_t n_tokens);
// x, dy, out, weight, dweight: two each, queries and keys. partial: 2 * rotate_blocks * width floats.
hipError_t launch_rotate(als_dtype dtype, bool back, const als_rotation &shape, const als_heads *x,
                         const als_heads *dy, const als_heads *out, const float *const *weight,
                         float *const *dweight, float *partial, hipStream_t s);

constexpr int kMaxBeams = 32;
int64_t beam_workspace(int64_t lists, int beams, int width, int64_t n_items);
hipError_t launch_beam_select(als_dtype dtype, int64_t lists, int beams, int width, int64_t n_items,
                              const void *logits, int64_t row_stride, const float *scores,
                              const uint8_t *finished, int32_t end, int32_t *parents,
                              int32_t *tokens, float *scores_out, uint8_t *finished_out,
                              void *workspace, hipStream_t s);
hipError_t launch_reorder(const void *src, void *dst, int64_t lists, int beams, int width,
                          int64_t bytes, const int32_t *parents, hipStream_t s);

}  // namespace als
