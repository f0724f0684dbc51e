// Host side of the sequence operators of include/als.h: checks of the arguments, the workspaces'
// layout, and the passes that make up a call.
#include <cmath>

#include "internal.h"
#include "sequence.h"

using als::AttentionPass;
using als::fail_without_context;

namespace {

constexpr int64_t kMax31 = (1LL << 31) - 1;
constexpr int64_t kMaxRows = 1LL << 30;  // of attention: with its segments below 2^31

#define REQUIRE(cond, ...) \
  if (!(cond)) return fail_without_context(ALS_ERR_INVALID_ARG, __VA_ARGS__)

als_status launched(hipError_t e, const char *what) {
  if (e == hipSuccess) return ALS_OK;
  return fail_without_context(e == hipErrorOutOfMemory ? ALS_ERR_OUT_OF_MEMORY : ALS_ERR_HIP,
                              "%s: %s", what, hipGetErrorString(e));
}

// The bytes [first, last) that n tokens of a tensor lie in.
struct Span {
  uintptr_t first, last;
};
Span span(const void *p, int64_t bytes) {
  return {(uintptr_t)p, (uintptr_t)p + (uintptr_t)(bytes > 0 ? bytes : 0)};
}
Span span(const als_heads &x, int64_t n, int32_t heads, int32_t width, int size) {
  if (n == 0) return span(x.data, 0);
  return span(x.data,
              ((n - 1) * x.token_stride + (heads - 1) * x.head_stride + width) * (int64_t)size);
}
bool overlap(Span a, Span b) {
  return a.first < a.last && b.first < b.last && a.first < b.last && b.first < a.last;
}
Span optional(const void *p, int64_t bytes) { return p ? span(p, bytes) : Span{0, 0}; }
bool same(const als_heads &a, const als_heads &b) {
  return a.data == b.data && a.token_stride == b.token_stride && a.head_stride == b.head_stride;
}

// nullptr, or what is wrong with one tensor
const char *wrong(const als_heads &x, int64_t n, int size) {
  if (n == 0) return nullptr;
  if (!x.data) return "NULL data";
  if (x.token_stride < 0 || x.head_stride < 0) return "a negative stride";
  // the last value's offset stays far inside 64 bits
  if (x.token_stride > (1LL << 56) / n || x.head_stride > (1LL << 40)) return "a stride out of range";
  if ((uintptr_t)x.data % size) return "data not aligned to its type";
  return nullptr;
}
// Rows of an output must not fall onto each other.
const char *wrong_out(const als_heads &x, int64_t n, int32_t heads, int32_t width, int size) {
  if (const char *w = wrong(x, n, size)) return w;
  if (n == 0) return nullptr;
  const bool by_token = x.head_stride >= width && x.token_stride >= (heads - 1) * x.head_stride + width;
  const bool by_head = x.token_stride >= width && x.head_stride >= (n - 1) * x.token_stride + width;
  if ((heads > 1 || n > 1) && !by_token && !by_head &&
      !(heads == 1 && x.token_stride >= width) && !(n == 1 && x.head_stride >= width))
    return "overlapping rows";
  return nullptr;
}

int size_of(als_dtype t) { return t == ALS_F32 ? 4 : 2; }
int64_t rounded16(int64_t x) { return (x + 15) / 16 * 16; }

als_status check_dtype(als_dtype t) {
  REQUIRE(t == ALS_F32 || t == ALS_BF16, "dtype %d is neither ALS_F32 nor ALS_BF16", (int)t);
  return ALS_OK;
}

als_status check_workspace(const void *p, int64_t bytes, int64_t needed) {
  REQUIRE(bytes >= needed, "workspace of %lld bytes, %lld needed", (long long)bytes,
          (long long)needed);
  REQUIRE(needed == 0 || p, "workspace is NULL");
  REQUIRE((uintptr_t)p % 16 == 0, "workspace is not 16-byte aligned");
  return ALS_OK;
}

// ---- norm and rotation ---------------------------------------------------------------------------

als_status check_rotation(const als_rotation *s, als_dtype dtype) {
  REQUIRE(s, "shape is NULL");
  if (als_status st = check_dtype(dtype)) return st;
  REQUIRE(s->n_tokens >= 0 && s->n_tokens <= kMax31, "n_tokens %lld out of range",
          (long long)s->n_tokens);
  REQUIRE(s->q_heads >= 1 && s->q_heads <= 1024 && s->k_heads >= 1 && s->k_heads <= 1024,
          "q_heads %d or k_heads %d outside [1, 1024]", s->q_heads, s->k_heads);
  REQUIRE(s->width >= 1 && s->width <= 256, "width %d outside [1, 256]", s->width);
  REQUIRE(s->rotated >= 0 && s->rotated <= s->width && s->rotated % 2 == 0,
          "rotated %d is not even in [0, width]", s->rotated);
  REQUIRE(s->neighbours == 0 || s->neighbours == 1, "neighbours %d is not 0 or 1", s->neighbours);
  REQUIRE(std::isfinite(s->eps) && s->eps >= 0.f, "eps %g is negative or not finite", s->eps);
  REQUIRE(s->n_positions >= (s->n_tokens > 0 ? 1 : 0) && s->n_positions <= kMax31,
          "n_positions %lld out of range", (long long)s->n_positions);
  REQUIRE(s->n_tokens == 0 || s->positions, "positions is NULL");
  REQUIRE(s->n_tokens == 0 || s->rotated == 0 || (s->cos_table && s->sin_table),
          "a NULL table of cosines or sines");
  return ALS_OK;
}

// The tensors of one side: x and dy read, out written.
als_status check_side(const als_rotation *s, als_dtype dtype, const char *side, int32_t heads,
                      const als_heads &x, const als_heads *dy, const als_heads &out,
                      const float *weight) {
  const int size = size_of(dtype);
  const int64_t n = s->n_tokens;
  REQUIRE(weight, "the weight of %s is NULL", side);
  if (const char *w = wrong(x, n, size))
    return fail_without_context(ALS_ERR_INVALID_ARG, "%s has %s", side, w);
  if (const char *w = dy ? wrong(*dy, n, size) : nullptr)
    return fail_without_context(ALS_ERR_INVALID_ARG, "the gradient of %s has %s", side, w);
  if (const char *w = wrong_out(out, n, heads, s->width, size))
    return fail_without_context(ALS_ERR_INVALID_ARG, "the output of %s has %s", side, w);
  const Span o = span(out, n, heads, s->width, size);
  REQUIRE(same(out, x) || !overlap(o, span(x, n, heads, s->width, size)),
          "the output of %s overlaps it in part", side);
  REQUIRE(!dy || same(out, *dy) || !overlap(o, span(*dy, n, heads, s->width, size)),
          "the output of %s overlaps its gradient in part", side);
  return ALS_OK;
}

als_status check_both(const als_rotation *s, als_dtype dtype, const als_heads *x,
                      const als_heads *dy, const als_heads *out, const float *const *weight) {
  const int size = size_of(dtype);
  const int32_t heads[2] = {s->q_heads, s->k_heads};
  for (int i = 0; i < 2; ++i)
    if (als_status st = check_side(s, dtype, i ? "k" : "q", heads[i], x[i], dy ? dy + i : nullptr,
                                   out[i], weight[i]))
      return st;
  for (int i = 0; i < 2; ++i) {  // one side's output on the other side's tensors
    // (heads of one projection lie between each other's rows: only whole packed outputs are compared)
    const Span o = span(out[i], s->n_tokens, heads[i], s->width, size);
    const bool packed = out[i].token_stride == (int64_t)heads[i] * out[i].head_stride;
    const Span other = span(out[1 - i], s->n_tokens, heads[1 - i], s->width, size);
    REQUIRE(out[0].data != out[1].data || s->n_tokens == 0, "q_out and k_out are the same");
    REQUIRE(!packed || !overlap(o, other), "q_out and k_out overlap");
    REQUIRE(!packed || (!overlap(o, span(x[1 - i], s->n_tokens, heads[1 - i], s->width, size)) &&
                        !(dy && overlap(o, span(dy[1 - i], s->n_tokens, heads[1 - i], s->width, size)))),
            "the output of %s overlaps %s or its gradient", i ? "k" : "q", i ? "q" : "k");
  }
  return ALS_OK;
}

// ---- attention -------------------------------------------------------------------------------------

als_status check_attention(const als_attention *s, als_dtype dtype, bool step) {
  REQUIRE(s, "shape is NULL");
  if (als_status st = check_dtype(dtype)) return st;
  REQUIRE(s->n_rows >= 0 && s->n_rows <= kMaxRows, "n_rows %lld out of range", (long long)s->n_rows);
  REQUIRE(s->q_heads >= 1 && s->q_heads <= 1024 && s->k_heads >= 1 &&
              s->q_heads % (s->k_heads > 0 ? s->k_heads : 1) == 0,
          "q_heads %d is not in [1, 1024] and a multiple of k_heads %d", s->q_heads, s->k_heads);
  REQUIRE(s->k_width >= 1 && s->k_width <= 128 && s->v_width >= 1 && s->v_width <= 128,
          "k_width %d or v_width %d outside [1, 128]", s->k_width, s->v_width);
  REQUIRE(std::isfinite(s->scale), "scale %g is not finite", s->scale);
  REQUIRE(s->log_decay, "log_decay is NULL");
  if (step) return ALS_OK;
  REQUIRE(s->n_tokens >= 0 && s->n_tokens <= kMax31, "n_tokens %lld out of range",
          (long long)s->n_tokens);
  REQUIRE(s->row_ptr, "row_ptr is NULL");
  REQUIRE(s->n_rows > 0 || s->n_tokens == 0, "tokens without rows");
  REQUIRE(s->clear_unheld == 0 || s->clear_unheld == 1, "clear_unheld %d is not 0 or 1", s->clear_unheld);
  return ALS_OK;
}

// One token's stride means nothing and may be anything (a slice of a large tensor has its own): it is taken
// out, since a pass from the last token to the first addresses its rows from those that would lie below.
// A step addresses its rows in 64 bits, at any stride.
als_status check_input(const char *name, als_heads &x, int64_t n, int size, bool step = false) {
  if (n <= 1) x.token_stride = 0;
  const char *w = wrong(x, n, size);
  if (!w && !step && x.token_stride > als::kMaxTokenStride) w = "a token_stride above 2^22";
  return w ? fail_without_context(ALS_ERR_INVALID_ARG, "%s has %s", name, w) : ALS_OK;
}

bool sane(const als_attention *s) {
  return s && s->n_tokens >= 0 && s->n_tokens <= kMax31 && s->n_rows >= 0 && s->n_rows <= kMaxRows &&
         s->q_heads >= 1 && s->q_heads <= 1024 && s->k_heads >= 1 && s->k_width >= 1 &&
         s->k_width <= 128 && s->v_width >= 1 && s->v_width <= 128;
}

als::AttentionSpace space_of(const als_attention *s, als_dtype dtype) {
  return als::attention_space(dtype, s->n_tokens, s->n_rows, s->q_heads, s->k_width, s->v_width);
}
// Of passes over a state and its transpose.
als::AttentionSpace backward_space(const als_attention *s, als_dtype dtype) {
  const int32_t w = s->k_width > s->v_width ? s->k_width : s->v_width;
  return als::attention_space(dtype, s->n_tokens, s->n_rows, s->q_heads, w, w);
}
// Of either type.
int64_t space_bytes(const als_attention *s) {
  const int64_t a = space_of(s, ALS_F32).total(), b = space_of(s, ALS_BF16).total();
  return a > b ? a : b;
}
// Gradients of shared heads, one per query head, before their sum: of k, then of v.
int64_t shared_bytes(const als_attention *s, int width) {
  return s->q_heads == s->k_heads ? 0 : rounded16(4 * s->n_tokens * s->q_heads * width);
}
int64_t backward_bytes(const als_attention *s) {  // the segments of two passes
  int64_t states = 0;
  for (als_dtype t : {ALS_F32, ALS_BF16}) {
    const als::AttentionSpace x = backward_space(s, t);
    states = x.total() + x.states > states ? x.total() + x.states : states;
  }
  return states + shared_bytes(s, s->k_width) + shared_bytes(s, s->v_width);
}

AttentionPass pass_of(const als_attention *s, als_dtype dtype, void *workspace) {
  AttentionPass p{};
  p.n_tokens = s->n_tokens;
  p.n_rows = s->n_rows;
  p.heads = s->q_heads;
  p.group = p.q_group = p.v_group = 1;
  p.log_decay = s->log_decay;
  p.row_ptr = s->row_ptr;
  p.weight_scale = s->scale;
  p.update_scale = p.read_scale = 1.f;
  const als::AttentionSpace x = space_of(s, dtype);
  char *w = (char *)workspace;
  p.places = x.places ? w : nullptr;
  p.entries = x.places ? (int32_t *)(w + x.places) : nullptr;
  p.segments = x.states ? (float *)(w + x.places + x.entries) : nullptr;
  return p;
}

// ---- attention over gaps of time -------------------------------------------------------------------

constexpr int64_t kMaxGapTokens = kMax31 - 255;  // a block's tokens are counted in 32 bits

bool sane(const als_gaps *s) {
  return s && s->n_tokens >= 0 && s->n_tokens <= kMaxGapTokens && s->n_rows >= 0 && s->n_rows <= kMaxRows &&
         s->q_heads >= 1 && s->q_heads <= 1024 && s->k_heads >= 1 && s->q_heads % s->k_heads == 0 &&
         s->width >= 1 && s->width <= 128 && s->buckets >= 1 && s->buckets <= 64;
}

als_status check_gaps(const als_gaps *s, als_dtype dtype) {
  REQUIRE(s, "shape is NULL");
  if (als_status st = check_dtype(dtype)) return st;
  REQUIRE(s->n_tokens >= 0 && s->n_tokens <= kMaxGapTokens, "n_tokens %lld out of range",
          (long long)s->n_tokens);
  REQUIRE(s->n_rows >= 0 && s->n_rows <= kMaxRows, "n_rows %lld out of range", (long long)s->n_rows);
  REQUIRE(s->q_heads >= 1 && s->q_heads <= 1024 && s->k_heads >= 1 && s->q_heads % s->k_heads == 0,
          "q_heads %d is not in [1, 1024] and a multiple of k_heads %d", s->q_heads, s->k_heads);
  REQUIRE(s->width >= 1 && s->width <= 128, "width %d outside [1, 128]", s->width);
  REQUIRE(s->buckets >= 1 && s->buckets <= 64, "buckets %d outside [1, 64]", s->buckets);
  REQUIRE(s->buckets == 1 || s->bounds, "bounds is NULL");
  for (int b = 0; b + 1 < s->buckets; ++b)
    REQUIRE(s->bounds[b] >= 1 && (b == 0 || s->bounds[b] > s->bounds[b - 1]),
            "bounds[%d] = %d is below 1 or not above the one before it", b, s->bounds[b]);
  REQUIRE(std::isfinite(s->scale), "scale %g is not finite", s->scale);
  REQUIRE(s->bias, "bias is NULL");
  REQUIRE(s->row_ptr, "row_ptr is NULL");
  REQUIRE(s->n_tokens == 0 || s->positions, "positions is NULL");
  REQUIRE(s->n_rows > 0 || s->n_tokens == 0, "tokens without rows");
  REQUIRE(s->clear_unheld == 0 || s->clear_unheld == 1, "clear_unheld %d is not 0 or 1", s->clear_unheld);
  return ALS_OK;
}

als::GapShape gap_shape(const als_gaps *s) {
  als::GapShape g{};
  g.n_tokens = s->n_tokens;
  g.n_rows = s->n_rows;
  g.row_ptr = s->row_ptr;
  g.positions = s->positions;
  g.bias = s->bias;
  g.heads = s->q_heads;
  g.group = s->q_heads / s->k_heads;
  g.width = s->width;
  g.buckets = s->buckets;
  g.scale = s->scale;
  g.clear_unheld = s->clear_unheld != 0;
  for (int b = 0; b + 1 < s->buckets; ++b) g.last_bound = g.bounds[b] = s->bounds[b];
  return g;
}

// A tensor of a call, by name.
struct Named {
  const char *name;
  Span at;
};
// What a call writes lies on nothing else of it.
als_status check_apart(const Named *written, int n_written, const Named *read, int n_read) {
  for (int i = 0; i < n_written; ++i) {
    for (int j = 0; j < i; ++j)
      REQUIRE(!overlap(written[i].at, written[j].at), "%s overlaps %s", written[i].name, written[j].name);
    for (int j = 0; j < n_read; ++j)
      REQUIRE(!overlap(written[i].at, read[j].at), "%s overlaps %s", written[i].name, read[j].name);
  }
  return ALS_OK;
}
als_status check_packed(const char *name, const void *p, int64_t n, int size) {
  REQUIRE(n == 0 || p, "%s is NULL", name);
  REQUIRE((uintptr_t)p % size == 0, "%s is not aligned to its type", name);
  return ALS_OK;
}

}  // namespace

extern "C" {

als_status als_norm_rotate(const als_rotation *shape, als_dtype dtype, als_heads q, als_heads k,
                           const float *q_weight, const float *k_weight, als_heads q_out,
                           als_heads k_out, void *hip_stream) {
  if (als_status st = check_rotation(shape, dtype)) return st;
  const als_heads x[2] = {q, k}, out[2] = {q_out, k_out};
  const float *const weight[2] = {q_weight, k_weight};
  if (als_status st = check_both(shape, dtype, x, nullptr, out, weight)) return st;
  if (shape->n_tokens == 0) return ALS_OK;
  return launched(als::launch_rotate(dtype, false, *shape, x, nullptr, out, weight, nullptr, nullptr,
                                     (hipStream_t)hip_stream),
                  "als_norm_rotate");
}

int64_t als_norm_rotate_workspace(const als_rotation *shape) {
  if (!shape || shape->n_tokens < 0 || shape->n_tokens > kMax31 || shape->width < 1 ||
      shape->width > 256)
    return -1;
  return 2 * als::rotate_blocks(shape->n_tokens) * shape->width * 4;
}

als_status als_norm_rotate_backward(const als_rotation *shape, als_dtype dtype, als_heads dq,
                                    als_heads dk, als_heads q, als_heads k, const float *q_weight,
                                    const float *k_weight, als_heads q_out, als_heads k_out,
                                    float *dq_weight, float *dk_weight, void *workspace,
                                    int64_t workspace_bytes, void *hip_stream) {
  if (als_status st = check_rotation(shape, dtype)) return st;
  const als_heads x[2] = {q, k}, dy[2] = {dq, dk}, out[2] = {q_out, k_out};
  const float *const weight[2] = {q_weight, k_weight};
  float *const dweight[2] = {dq_weight, dk_weight};
  if (als_status st = check_both(shape, dtype, x, dy, out, weight)) return st;
  REQUIRE(dq_weight && dk_weight, "a NULL gradient of a weight");
  REQUIRE(dq_weight != dk_weight, "the weights' gradients are the same");
  const Span dw[2] = {span(dq_weight, 4 * shape->width), span(dk_weight, 4 * shape->width)};
  REQUIRE(!overlap(dw[0], dw[1]), "the weights' gradients overlap");
  for (int i = 0; i < 2; ++i) {
    const Span o = span(out[i], shape->n_tokens, i ? shape->k_heads : shape->q_heads, shape->width,
                        size_of(dtype));
    REQUIRE(!overlap(o, dw[0]) && !overlap(o, dw[1]), "a weight's gradient overlaps the output of %s",
            i ? "k" : "q");
  }
  if (als_status st = check_workspace(workspace, workspace_bytes, als_norm_rotate_workspace(shape)))
    return st;
  return launched(als::launch_rotate(dtype, true, *shape, x, dy, out, weight, dweight,
                                     (float *)workspace, (hipStream_t)hip_stream),
                  "als_norm_rotate_backward");
}

int64_t als_decay_attention_workspace(const als_attention *shape) {
  return sane(shape) ? space_bytes(shape) : -1;
}

als_status als_decay_attention(const als_attention *shape, als_dtype dtype, als_heads q, als_heads k,
                               als_heads v, const float *initial_state, void *out,
                               float *final_state, void *workspace, int64_t workspace_bytes,
                               void *hip_stream) {
  if (als_status st = check_attention(shape, dtype, false)) return st;
  const als_attention *s = shape;
  const int size = size_of(dtype);
  if (als_status st = check_input("q", q, s->n_tokens, size)) return st;
  if (als_status st = check_input("k", k, s->n_tokens, size)) return st;
  if (als_status st = check_input("v", v, s->n_tokens, size)) return st;
  REQUIRE(s->n_tokens == 0 || out, "out is NULL");
  REQUIRE((uintptr_t)out % size == 0, "out is not aligned to its type");
  const Span o = span(out, s->n_tokens * s->q_heads * s->v_width * size);
  REQUIRE(!overlap(o, span(q, s->n_tokens, s->q_heads, s->k_width, size)) &&
              !overlap(o, span(k, s->n_tokens, s->k_heads, s->k_width, size)) &&
              !overlap(o, span(v, s->n_tokens, s->k_heads, s->v_width, size)),
          "out overlaps an input");
  const int64_t states = 4 * s->n_rows * s->q_heads * s->k_width * s->v_width;
  const Span first = optional(initial_state, states), last = optional(final_state, states);
  REQUIRE(!overlap(first, last), "final_state overlaps initial_state");
  REQUIRE(!overlap(o, first) && !overlap(o, last), "out overlaps a state");
  REQUIRE(!overlap(last, span(q, s->n_tokens, s->q_heads, s->k_width, size)) &&
              !overlap(last, span(k, s->n_tokens, s->k_heads, s->k_width, size)) &&
              !overlap(last, span(v, s->n_tokens, s->k_heads, s->v_width, size)),
          "final_state overlaps an input");
  if (als_status st = check_workspace(workspace, workspace_bytes, space_bytes(s))) return st;
  AttentionPass p = pass_of(s, dtype, workspace);
  p.group = p.v_group = s->q_heads / s->k_heads;
  p.k_width = s->k_width;
  p.v_width = s->v_width;
  p.q = q;
  p.k = k;
  p.v = v;
  p.read_scale = s->scale;
  p.first_state = initial_state;
  p.last_state = final_state;
  p.first_ld[0] = p.last_ld[0] = s->v_width;
  p.first_ld[1] = p.last_ld[1] = 1;
  p.out = out;
  hipError_t e = als::launch_places(dtype, p, (hipStream_t)hip_stream);
  if (e == hipSuccess) e = als::launch_attention(dtype, &p, 1, (hipStream_t)hip_stream);
  if (e == hipSuccess && s->clear_unheld) {
    const als::Unheld u{1, {(char *)out}, {(int64_t)s->q_heads * s->v_width * size}};
    e = als::launch_clear_unheld(s->n_tokens, s->n_rows, s->row_ptr, u, (hipStream_t)hip_stream);
  }
  return launched(e, "als_decay_attention");
}

int64_t als_decay_attention_backward_workspace(const als_attention *shape) {
  return sane(shape) ? backward_bytes(shape) : -1;
}

als_status als_decay_attention_backward(const als_attention *shape, als_dtype dtype, als_heads d_out,
                                        als_heads q, als_heads k, als_heads v,
                                        const float *initial_state, const float *d_final_state,
                                        void *dq, void *dk, void *dv, float *d_initial_state,
                                        void *workspace, int64_t workspace_bytes, void *hip_stream) {
  if (als_status st = check_attention(shape, dtype, false)) return st;
  const als_attention *s = shape;
  const int size = size_of(dtype), group = s->q_heads / s->k_heads;
  const int64_t n = s->n_tokens;
  if (als_status st = check_input("d_out", d_out, n, size)) return st;
  if (als_status st = check_input("q", q, n, size)) return st;
  if (als_status st = check_input("k", k, n, size)) return st;
  if (als_status st = check_input("v", v, n, size)) return st;
  REQUIRE(n == 0 || (dq && dk && dv), "a NULL gradient");
  REQUIRE(((uintptr_t)dq | (uintptr_t)dk | (uintptr_t)dv) % size == 0,
          "a gradient is not aligned to its type");
  const Span outs[3] = {span(dq, n * s->q_heads * s->k_width * size),
                        span(dk, n * s->k_heads * s->k_width * size),
                        span(dv, n * s->k_heads * s->v_width * size)};
  const Span ins[4] = {span(d_out, n, s->q_heads, s->v_width, size),
                       span(q, n, s->q_heads, s->k_width, size),
                       span(k, n, s->k_heads, s->k_width, size),
                       span(v, n, s->k_heads, s->v_width, size)};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 4; ++j) REQUIRE(!overlap(outs[i], ins[j]), "a gradient overlaps an input");
    REQUIRE(!overlap(outs[i], outs[(i + 1) % 3]), "two gradients overlap");
  }
  const int64_t states = 4 * s->n_rows * s->q_heads * s->k_width * s->v_width;
  const Span first = optional(initial_state, states), last = optional(d_final_state, states),
             d_first = optional(d_initial_state, states);
  REQUIRE(!overlap(first, d_first) && !overlap(last, d_first), "d_initial_state overlaps another state");
  for (const Span &x : outs)
    REQUIRE(!overlap(x, first) && !overlap(x, last) && !overlap(x, d_first), "a gradient overlaps a state");
  for (const Span &x : ins) REQUIRE(!overlap(d_first, x), "d_initial_state overlaps an input");
  if (als_status st = check_workspace(workspace, workspace_bytes,
                                      als_decay_attention_backward_workspace(s)))
    return st;
  const hipStream_t stream = (hipStream_t)hip_stream;
  const als::AttentionSpace space = backward_space(s, dtype);
  char *rest = (char *)workspace + space.total() + space.states;
  float *shared_k = group > 1 ? (float *)rest : nullptr;
  float *shared_v = group > 1 ? (float *)(rest + shared_bytes(s, s->k_width)) : nullptr;

  AttentionPass p[3] = {pass_of(s, dtype, workspace), pass_of(s, dtype, workspace),
                        pass_of(s, dtype, workspace)};
  // dq: the pass over (d_out, v, k), with the state transposed
  p[0].group = p[0].v_group = group;
  p[0].k_width = s->v_width;
  p[0].v_width = s->k_width;
  p[0].q = d_out;
  p[0].k = v;
  p[0].v = k;
  p[0].read_scale = s->scale;
  p[0].first_state = initial_state;
  p[0].first_ld[0] = 1;
  p[0].first_ld[1] = s->v_width;
  p[0].out = dq;
  // dv: the reversed pass over (k, q, d_out); its last state is the initial state's gradient
  p[1].reverse = true;
  p[1].update_scale = s->scale;
  p[1].q_group = group;
  p[1].k_width = s->k_width;
  p[1].v_width = s->v_width;
  p[1].q = k;
  p[1].k = q;
  p[1].v = d_out;
  p[1].first_state = d_final_state;
  p[1].last_state = d_initial_state;
  p[1].first_ld[0] = p[1].last_ld[0] = s->v_width;
  p[1].first_ld[1] = p[1].last_ld[1] = 1;
  p[1].out = shared_v ? (void *)shared_v : dv;
  p[1].out_f32 = shared_v || dtype == ALS_F32;
  if (space.states) p[1].segments = (float *)((char *)workspace + space.total());
  // dk: the reversed pass over (v, d_out, q), with dv's state transposed
  p[2] = p[1];
  p[2].k_width = s->v_width;
  p[2].v_width = s->k_width;
  p[2].q = v;
  p[2].k = d_out;
  p[2].v = q;
  p[2].last_state = nullptr;
  p[2].first_ld[0] = 1;
  p[2].first_ld[1] = s->v_width;
  p[2].shares_segments = true;
  p[2].out = shared_k ? (void *)shared_k : dk;
  hipError_t e = als::launch_places(dtype, p[0], stream);
  if (e == hipSuccess) e = als::launch_attention(dtype, p, 3, stream);
  if (e == hipSuccess && shared_k)
    e = als::launch_sum_groups(dtype, shared_k, shared_v, n, s->q_heads, group, s->k_width, s->v_width,
                               dk, dv, stream);
  if (e == hipSuccess && s->clear_unheld) {
    const als::Unheld u{3,
                        {(char *)dq, (char *)dk, (char *)dv},
                        {(int64_t)s->q_heads * s->k_width * size, (int64_t)s->k_heads * s->k_width * size,
                         (int64_t)s->k_heads * s->v_width * size}};
    e = als::launch_clear_unheld(n, s->n_rows, s->row_ptr, u, stream);
  }
  return launched(e, "als_decay_attention_backward");
}

als_status als_decay_attention_step(const als_attention *shape, als_dtype dtype, als_heads q,
                                    als_heads k, als_heads v, const float *state, int64_t n_sources,
                                    const int32_t *source, float *state_out, void *out,
                                    void *hip_stream) {
  if (als_status st = check_attention(shape, dtype, true)) return st;
  const als_attention *s = shape;
  const int size = size_of(dtype);
  if (als_status st = check_input("q", q, s->n_rows, size, true)) return st;
  if (als_status st = check_input("k", k, s->n_rows, size, true)) return st;
  if (als_status st = check_input("v", v, s->n_rows, size, true)) return st;
  REQUIRE(n_sources >= 0 && n_sources <= kMax31, "n_sources %lld out of range", (long long)n_sources);
  REQUIRE(source || n_sources == s->n_rows, "%lld states for %lld rows without source",
          (long long)n_sources, (long long)s->n_rows);
  if (s->n_rows == 0) return ALS_OK;
  REQUIRE(n_sources > 0, "rows without a state");
  REQUIRE(state && state_out && out, "state, state_out or out is NULL");
  REQUIRE(((uintptr_t)state | (uintptr_t)state_out) % 4 == 0 && (uintptr_t)out % size == 0,
          "a tensor is not aligned to its type");
  const int64_t one = 4LL * s->q_heads * s->k_width * s->v_width;
  REQUIRE((!source && state == state_out) ||
              !overlap(span(state, n_sources * one), span(state_out, s->n_rows * one)),
          "state_out overlaps state");
  const Span o = span(out, s->n_rows * s->q_heads * s->v_width * size);
  REQUIRE(!overlap(o, span(state, n_sources * one)) && !overlap(o, span(state_out, s->n_rows * one)),
          "out overlaps a state");
  REQUIRE(!overlap(o, span(q, s->n_rows, s->q_heads, s->k_width, size)) &&
              !overlap(o, span(k, s->n_rows, s->k_heads, s->k_width, size)) &&
              !overlap(o, span(v, s->n_rows, s->k_heads, s->v_width, size)),
          "out overlaps an input");
  const Span to = span(state_out, s->n_rows * one);
  REQUIRE(!overlap(to, span(q, s->n_rows, s->q_heads, s->k_width, size)) &&
              !overlap(to, span(k, s->n_rows, s->k_heads, s->k_width, size)) &&
              !overlap(to, span(v, s->n_rows, s->k_heads, s->v_width, size)),
          "state_out overlaps an input");
  return launched(als::launch_attention_step(dtype, s->n_rows, s->q_heads, s->q_heads / s->k_heads,
                                             s->k_width, s->v_width, q, k, v, s->log_decay, s->scale,
                                             state, source, n_sources, state_out, out,
                                             (hipStream_t)hip_stream),
                  "als_decay_attention_step");
}

static als_status check_beams(const als_beams *s) {
  REQUIRE(s, "shape is NULL");
  REQUIRE(s->n_lists >= 0 && s->n_lists <= kMax31, "n_lists %lld out of range",
          (long long)s->n_lists);
  REQUIRE(s->beams >= 1 && s->beams <= als::kMaxBeams && s->width >= 1 && s->width <= als::kMaxBeams,
          "beams %d or width %d outside [1, %d]", s->beams, s->width, als::kMaxBeams);
  REQUIRE(s->n_items >= 1 && s->n_items <= kMax31, "n_items %lld out of range",
          (long long)s->n_items);
  REQUIRE(s->row_stride >= s->n_items && s->row_stride <= (1LL << 56) / (s->n_lists * s->beams + 1),
          "row_stride %lld below n_items or out of range", (long long)s->row_stride);
  REQUIRE(s->end_token >= -1 && s->end_token < s->n_items, "end_token %d outside [-1, n_items)",
          s->end_token);
  return ALS_OK;
}

int64_t als_gap_attention_workspace(const als_gaps *shape) {
  return sane(shape) ? als::gap_spans_bytes(shape->n_tokens, shape->n_rows) : -1;
}

als_status als_gap_attention(const als_gaps *shape, als_dtype dtype, als_heads q, als_heads k, als_heads v,
                             void *out, float *stats, int16_t *rest, void *workspace, int64_t workspace_bytes,
                             void *hip_stream) {
  if (als_status st = check_gaps(shape, dtype)) return st;
  const als_gaps *s = shape;
  const int size = size_of(dtype);
  const int64_t n = s->n_tokens, values = n * s->q_heads * s->width;
  if (als_status st = check_input("q", q, n, size)) return st;
  if (als_status st = check_input("k", k, n, size)) return st;
  if (als_status st = check_input("v", v, n, size)) return st;
  if (als_status st = check_packed("out", out, n, size)) return st;
  if (als_status st = check_packed("stats", stats, 0, 4)) return st;
  if (als_status st = check_packed("rest", rest, 0, size)) return st;
  REQUIRE(!rest || dtype == ALS_BF16, "rest is for bf16 outputs");
  const int64_t needed = als::gap_spans_bytes(n, s->n_rows);
  if (als_status st = check_workspace(workspace, workspace_bytes, needed)) return st;
  const Named written[] = {{"out", span(out, values * size)},
                           {"stats", optional(stats, 8 * n * s->q_heads)},
                           {"rest", optional(rest, values * size)},
                           {"the workspace", span(workspace, needed)}};
  const Named read[] = {{"q", span(q, n, s->q_heads, s->width, size)},
                        {"k", span(k, n, s->k_heads, s->width, size)},
                        {"v", span(v, n, s->k_heads, s->width, size)},
                        {"bias", span(s->bias, 4LL * s->q_heads * s->buckets)},
                        {"positions", span(s->positions, 4 * n)},
                        {"row_ptr", span(s->row_ptr, 8 * (s->n_rows + 1))}};
  if (als_status st = check_apart(written, 4, read, 6)) return st;
  const als::GapShape g = gap_shape(s);
  void *spans = needed ? workspace : nullptr;
  hipError_t e = als::launch_gap_spans(g, spans, (hipStream_t)hip_stream);
  if (e == hipSuccess)
    e = als::launch_gap_read(dtype, g, q, k, v, spans, out, stats, rest, (hipStream_t)hip_stream);
  return launched(e, "als_gap_attention");
}

int64_t als_gap_attention_backward_workspace(const als_gaps *shape) {
  return sane(shape)
             ? als::gap_back_space(shape->n_tokens, shape->n_rows, shape->q_heads, shape->k_heads, shape->width,
                                   shape->buckets).total()
             : -1;
}

als_status als_gap_attention_backward(const als_gaps *shape, als_dtype dtype, als_heads d_out, als_heads q,
                                      als_heads k, als_heads v, const void *out, const float *stats,
                                      const int16_t *rest, void *dq, void *dk, void *dv, float *dbias,
                                      void *workspace, int64_t workspace_bytes, void *hip_stream) {
  if (als_status st = check_gaps(shape, dtype)) return st;
  const als_gaps *s = shape;
  const int size = size_of(dtype);
  const int64_t n = s->n_tokens, q_bytes = n * s->q_heads * s->width * size,
                k_bytes = n * s->k_heads * s->width * size;
  if (als_status st = check_input("d_out", d_out, n, size)) return st;
  if (als_status st = check_input("q", q, n, size)) return st;
  if (als_status st = check_input("k", k, n, size)) return st;
  if (als_status st = check_input("v", v, n, size)) return st;
  if (als_status st = check_packed("out", out, n, size)) return st;
  if (als_status st = check_packed("stats", stats, n, 4)) return st;
  if (als_status st = check_packed("rest", rest, 0, size)) return st;
  REQUIRE(!rest || dtype == ALS_BF16, "rest is for bf16 outputs");
  if (als_status st = check_packed("dq", dq, n, size)) return st;
  if (als_status st = check_packed("dk", dk, n, size)) return st;
  if (als_status st = check_packed("dv", dv, n, size)) return st;
  if (als_status st = check_packed("dbias", dbias, 1, 4)) return st;
  const int64_t needed = als_gap_attention_backward_workspace(s);
  if (als_status st = check_workspace(workspace, workspace_bytes, needed)) return st;
  const int64_t bias_bytes = 4LL * s->q_heads * s->buckets;
  const Named written[] = {{"dq", span(dq, q_bytes)},
                           {"dk", span(dk, k_bytes)},
                           {"dv", span(dv, k_bytes)},
                           {"dbias", span(dbias, bias_bytes)},
                           {"the workspace", span(workspace, needed)}};
  const Named read[] = {{"d_out", span(d_out, n, s->q_heads, s->width, size)},
                        {"q", span(q, n, s->q_heads, s->width, size)},
                        {"k", span(k, n, s->k_heads, s->width, size)},
                        {"v", span(v, n, s->k_heads, s->width, size)},
                        {"out", span(out, q_bytes)},
                        {"stats", span(stats, 8 * n * s->q_heads)},
                        {"rest", optional(rest, q_bytes)},
                        {"bias", span(s->bias, bias_bytes)},
                        {"positions", span(s->positions, 4 * n)},
                        {"row_ptr", span(s->row_ptr, 8 * (s->n_rows + 1))}};
  if (als_status st = check_apart(written, 5, read, 10)) return st;
  return launched(als::launch_gap_back(dtype, gap_shape(s), d_out, q, k, v, out, stats, rest, dq, dk, dv, dbias,
                                       workspace, (hipStream_t)hip_stream),
                  "als_gap_attention_backward");
}

int64_t als_gap_attention_step_workspace(const als_gaps *shape, const als_gap_path *path) {
  return sane(shape) && path && path->beams >= 1 && path->beams <= als::kMaxBeams
             ? als::gap_step_space(shape->n_tokens, shape->n_rows, shape->q_heads, shape->k_heads, path->beams,
                                   shape->width)
             : -1;
}

als_status als_gap_attention_step(const als_gaps *shape, const als_gap_path *path, als_dtype dtype, als_heads q,
                                  als_heads k, als_heads v, void *out, void *workspace,
                                  int64_t workspace_bytes, void *hip_stream) {
  const als_gaps *s = shape;
  if (als_status st = check_gaps(s, dtype)) return st;
  REQUIRE(path, "path is NULL");
  const als_gap_path *p = path;
  REQUIRE(p->beams >= 1 && p->beams <= als::kMaxBeams, "beams %d outside [1, %d]", p->beams, als::kMaxBeams);
  REQUIRE(p->steps >= 0 && p->steps <= 1 << 20, "steps %d out of range", p->steps);
  const int64_t rows = s->n_rows * p->beams;
  REQUIRE(rows <= kMax31, "%lld lists of %d beams", (long long)s->n_rows, p->beams);
  const int size = size_of(dtype);
  const int64_t n = s->n_tokens, path_rows = p->steps > 0 ? rows : 0;
  REQUIRE(rows == 0 || p->q_positions, "q_positions is NULL");
  if (als_status st = check_input("q", q, rows, size, true)) return st;
  if (als_status st = check_input("k", k, n, size, true)) return st;
  if (als_status st = check_input("v", v, n, size, true)) return st;
  als::GapPath g{p->beams, p->steps, p->q_positions, p->k, p->v, p->k_step, p->v_step, p->positions, p->path,
                 p->path_stride};
  if (als_status st = check_input("the path's k", g.k, path_rows, size, true)) return st;
  if (als_status st = check_input("the path's v", g.v, path_rows, size, true)) return st;
  if (path_rows > 0) {
    REQUIRE(p->k_step >= 0 && p->v_step >= 0 && p->k_step <= (1LL << 56) / p->steps &&
                p->v_step <= (1LL << 56) / p->steps,
            "a step's stride of the path's k or v is negative or out of range");
    REQUIRE(p->positions, "the path's positions are NULL");
    REQUIRE(p->path, "path is NULL");
    REQUIRE(p->path_stride >= p->steps && p->path_stride <= 1LL << 24, "path_stride %lld out of range",
            (long long)p->path_stride);
  }
  if (als_status st = check_packed("out", out, rows, size)) return st;
  const int64_t needed = als::gap_step_space(n, s->n_rows, s->q_heads, s->k_heads, p->beams, s->width);
  if (als_status st = check_workspace(workspace, workspace_bytes, needed)) return st;
  const auto path_span = [&](const als_heads &x, int64_t step) {
    if (path_rows == 0) return Span{0, 0};
    return span(x.data, ((p->steps - 1) * step + (rows - 1) * x.token_stride +
                         (s->k_heads - 1) * x.head_stride + s->width) * (int64_t)size);
  };
  const Named written[] = {{"out", span(out, rows * s->q_heads * s->width * size)},
                           {"the workspace", span(workspace, needed)}};
  const Named read[] = {{"q", span(q, rows, s->q_heads, s->width, size)},
                        {"k", span(k, n, s->k_heads, s->width, size)},
                        {"v", span(v, n, s->k_heads, s->width, size)},
                        {"bias", span(s->bias, 4LL * s->q_heads * s->buckets)},
                        {"positions", span(s->positions, 4 * n)},
                        {"row_ptr", span(s->row_ptr, 8 * (s->n_rows + 1))},
                        {"q_positions", span(p->q_positions, 4 * rows)},
                        {"the path's k", path_span(g.k, p->k_step)},
                        {"the path's v", path_span(g.v, p->v_step)},
                        {"the path's positions", span(p->positions, 4 * p->steps * path_rows)},
                        {"path", path_rows ? span(p->path, 4 * ((rows - 1) * p->path_stride + p->steps))
                                           : Span{0, 0}}};
  if (als_status st = check_apart(written, 2, read, 11)) return st;
  return launched(als::launch_gap_step(dtype, gap_shape(s), g, q, k, v, out, workspace,
                                       (hipStream_t)hip_stream),
                  "als_gap_attention_step");
}

int64_t als_beam_select_workspace(const als_beams *shape) {
  if (check_beams(shape) != ALS_OK) return -1;
  return als::beam_workspace(shape->n_lists, shape->beams, shape->width, shape->n_items);
}

als_status als_beam_select(const als_beams *shape, als_dtype dtype, const void *logits,
                           const float *scores, const uint8_t *finished, int32_t *parents,
                           int32_t *tokens, float *scores_out, uint8_t *finished_out,
                           void *workspace, int64_t workspace_bytes, void *hip_stream) {
  if (als_status st = check_beams(shape)) return st;
  if (als_status st = check_dtype(dtype)) return st;
  const als_beams *s = shape;
  REQUIRE(!finished || s->end_token >= 0, "finished beams need an end_token");
  if (s->n_lists == 0) return ALS_OK;
  REQUIRE(logits && scores && parents && tokens && scores_out && finished_out, "a NULL tensor");
  REQUIRE((uintptr_t)logits % size_of(dtype) == 0, "logits are not aligned to their type");
  const int64_t before = s->n_lists * s->beams, after = s->n_lists * s->width;
  REQUIRE((uintptr_t)scores % 4 == 0 && (uintptr_t)scores_out % 4 == 0 && (uintptr_t)parents % 4 == 0 &&
              (uintptr_t)tokens % 4 == 0,
          "a tensor is not aligned to its type");
  const Span ins[3] = {
      span(logits, ((before - 1) * s->row_stride + s->n_items) * size_of(dtype)),
      span(scores, 4 * before), span(finished, finished ? before : 0)};
  const Span outs[4] = {span(parents, 4 * after), span(tokens, 4 * after), span(scores_out, 4 * after),
                        span(finished_out, after)};
  for (int i = 0; i < 4; ++i) {
    for (const Span &x : ins) REQUIRE(!overlap(outs[i], x), "an output overlaps an input");
    for (int j = 0; j < i; ++j) REQUIRE(!overlap(outs[i], outs[j]), "two outputs overlap");
  }
  if (als_status st = check_workspace(
          workspace, workspace_bytes,
          als::beam_workspace(s->n_lists, s->beams, s->width, s->n_items)))
    return st;
  return launched(als::launch_beam_select(dtype, s->n_lists, s->beams, s->width, s->n_items, logits,
                                          s->row_stride, scores, finished, s->end_token, parents,
                                          tokens, scores_out, finished_out, workspace,
                                          (hipStream_t)hip_stream),
                  "als_beam_select");
}

als_status als_reorder_states(int64_t n_lists, int32_t beams, int32_t width, int64_t row_bytes,
                              const void *src, void *dst, const int32_t *parents, void *hip_stream) {
  REQUIRE(n_lists >= 0 && n_lists <= kMax31, "n_lists %lld out of range", (long long)n_lists);
  REQUIRE(beams >= 1 && beams <= als::kMaxBeams && width >= 1 && width <= als::kMaxBeams,
          "beams %d or width %d outside [1, %d]", beams, width, als::kMaxBeams);
  REQUIRE(row_bytes >= 0 && row_bytes <= (1LL << 56) / (32 * (n_lists + 1)), "row_bytes %lld out of range",
          (long long)row_bytes);
  if (n_lists == 0 || row_bytes == 0) return ALS_OK;
  REQUIRE(src && dst && parents, "a NULL tensor");
  REQUIRE((src == dst && beams == width) ||
              !overlap(span(src, n_lists * beams * row_bytes), span(dst, n_lists * width * row_bytes)),
          "dst overlaps src");
  return launched(als::launch_reorder(src, dst, n_lists, beams, width, row_bytes, parents,
                                      (hipStream_t)hip_stream),
                  "als_reorder_states");
}

}  // extern "C"
