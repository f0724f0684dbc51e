// Internal declarations of the sequence operators: norm and rotation of queries and keys
// (rotate.hip), attention with a decay for each head (attention.hip) and beam selection
// (beam.hip). Host entries: sequence.hip.
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
