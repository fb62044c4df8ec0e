/* taw_model.h -- what stands around the decoder layers in a training step, on one GPU: the embedding and its gradient, the
 * loss over the vocabulary with its gradient, and the global gradient norm with clipping.
 *
 *   ids -> taw_embed_fwd -> layers (taw_layer_fwd) -> norm (taw_op_rmsnorm_fwd) -> logits (taw_op_gemm) -> taw_loss_fwd_bwd
 *       -> taw_op_linear_bwd -> taw_op_rmsnorm_bwd -> layers (taw_layer_bwd) -> taw_embed_bwd
 *       -> taw_grad_norm over every shard -> taw_optimizer_step_clipped, shard by shard
 *
 * The general rules of taw.h hold: int status, device pointers unless a parameter says "host", nothing allocated, everything
 * enqueued on `stream` (the stream's device is the current one), no synchronisation, all validation on the host before the first
 * launch, device pointers 16-byte aligned (token ids and labels: aligned to their type).  Every call can be captured into a graph.
 * Calls, and captured graphs, that may run at the same time need workspaces (and clip states) of their own.  A call repeated gives
 * the same bits: the order of every sum follows from the arguments, and there are no floating-point atomics.
 */
#ifndef TAW_MODEL_H
#define TAW_MODEL_H

#include "../taw.h"

#ifdef __cplusplus
extern "C" {
#endif

/* type of token ids and labels */
enum { TAW_I32 = 0, TAW_I64 = 1 };

/* ---------------------------------------------------------------------------------------------- embedding
 * table [V, H] of dtype with row stride ld_table; x, dx [T, H] of dtype with row stride ld_x; G fp32 [V, H] with the table's row
 * stride (the table's gradient shard: same element offsets).  An id outside [0, V), negative ones among them, names no row: it
 * gives a row of zeros forward and takes no part backward (padding). */
typedef struct {
  int32_t dtype;      /* taw_dtype */
  int32_t T;          /* tokens, 0 .. 2^24 */
  int32_t H, V;       /* row length and rows of the table, V <= 2^24 */
  int64_t ld_table;   /* row strides in elements, >= H; 0 stands for H */
  int64_t ld_x;
  float scale;        /* x = scale * row (1, or the square root of H) */
  uint32_t flags;     /* TAW_ACCUMULATE: taw_embed_bwd adds into G; without it every row of G is overwritten */
} taw_embed_desc;

/* x[t] = scale * table[ids[t]], rounded once. */
int taw_embed_fwd(const taw_embed_desc* desc, const void* ids, int32_t id_type, const void* table, void* x, void* stream);

/* G[v] (=|+=) scale * sum over t with ids[t] == v of dx[t], summed in fp32 in an order that T and the ids decide.  Rows that no
 * id names are zeroed, or left alone with TAW_ACCUMULATE; the padding between rows (ld_table > H) is left alone.
 * workspace: taw_embed_bwd_workspace_bytes() bytes (0 for an invalid descriptor); holds nothing between calls. */
size_t taw_embed_bwd_workspace_bytes(const taw_embed_desc* desc);
int taw_embed_bwd(const taw_embed_desc* desc, const void* ids, int32_t id_type, const void* dx, float* G, void* workspace,
                  size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------- loss over the vocabulary
 * logits [T, V] of dtype with row stride ld.  For a row l with label y in [0, V), eps = label_smoothing, z = z_loss:
 *   lse  = log sum_v exp l_v
 *   row  = lse - (1 - eps) l_y - eps/V sum_v l_v + z lse^2
 *   dl_v = up ((1 + 2 z lse) exp(l_v - lse) - (1 - eps) [v = y] - eps/V)
 * with up = grad_scale, divided by the number of counted rows with TAW_LOSS_MEAN (taw_loss_fwd_bwd), or dloss_rows[t] (taw_loss_bwd).
 * A row whose label is outside [0, V) (-100 and its like) is not counted: its logits are not looked at, its loss, lse and gradient
 * are 0.  Logits of -inf are masked classes of probability 0, which leaves them the rest of the formulas: the loss is +inf where
 * such a class is the label or has a share eps/V of it, and its gradient -up times what it has of the label (0 without smoothing).
 * (The type's lowest value is a finite logit like any other.)  A counted row with nothing but -inf has lse -inf, loss +inf and a gradient of 0;
 * +inf or NaN in a counted row make all of its results NaN.
 * Everything is computed in fp32 (sums over rows in fp64) from the logits as stored, and dlogits is rounded once.  Only differences of
 * logits count: a row's loss and probabilities are no less exact far from zero (the sum of logits of a smoothed label, the z-loss and
 * lse itself have the precision of numbers of their size).
 * dlogits [T, V_pad] of grad_dtype with row stride ld_grad: columns V .. V_pad-1 (a vocabulary padded for the products around
 * this call) are written as zeros; columns of logits beyond V are not read.  dlogits may be logits itself where types and strides
 * are equal. */
#define TAW_LOSS_MEAN 1u /* loss and gradient are divided by the number of counted rows (none counted: both are 0) */
typedef struct {
  int32_t dtype;          /* taw_dtype of the logits */
  int32_t grad_dtype;     /* taw_dtype of dlogits: dtype, or TAW_BF16 */
  int32_t T;              /* rows, 0 .. 2^24 */
  int32_t V, V_pad;       /* classes, 1 .. 2^24, and columns of dlogits to write, >= V; 0 stands for V */
  int64_t ld, ld_grad;    /* row strides in elements, >= V and >= V_pad; 0 stands for V and V_pad */
  float label_smoothing;  /* [0, 1) */
  float z_loss;           /* >= 0 */
  float grad_scale;
  uint32_t flags;
} taw_loss_desc;

/* Bytes of scratch taw_loss_fwd and taw_loss_fwd_bwd need (0 for an invalid descriptor); holds nothing between calls. */
size_t taw_loss_workspace_bytes(const taw_loss_desc* desc);

/* The loss alone (evaluation).  loss (fp32 [2]): sum of the counted rows' losses, or their mean, and the number of counted rows.
 * loss_rows, lse (fp32 [T]): may be NULL. */
int taw_loss_fwd(const taw_loss_desc* desc, const void* logits, const void* labels, int32_t label_type, float* loss,
                 float* loss_rows, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* Loss and gradient in one call (training): what taw_loss_fwd gives, and dlogits. */
int taw_loss_fwd_bwd(const taw_loss_desc* desc, const void* logits, const void* labels, int32_t label_type, float* loss,
                     float* loss_rows, float* lse, void* dlogits, void* workspace, size_t workspace_bytes, void* stream);

/* The gradient from lse (as taw_loss_fwd wrote it) and the gradient of every row's loss (fp32 [T]); grad_scale and TAW_LOSS_MEAN
 * play no part.  exp(l - lse) is formed with the lse that is given, which fp32 holds to 2^-24 of its size: around 1e4 the probabilities
 * of a row have a common factor of up to 1 +- 5e-4, which those of taw_loss_fwd_bwd have not. */
int taw_loss_bwd(const taw_loss_desc* desc, const void* logits, const void* labels, int32_t label_type, const float* lse,
                 const float* dloss_rows, void* dlogits, void* stream);

/* ---------------------------------------------------------------------------------------------- gradient norm and clipping
 * The norm is taken over a list of tensors (host array; its entries are copied at the call, so the list may go away).  The result
 * stays on the device, in a taw_clip_state that the clipping and the optimizer step read there: no call waits for it. */
typedef struct {
  void* data;         /* device, fp32 or bf16; may be NULL where n is 0 */
  size_t n;           /* elements */
  int32_t dtype;      /* taw_dtype */
} taw_tensor;

typedef struct {      /* device, 32 bytes */
  double sumsq;       /* sum of squares of the unscaled gradients */
  float norm;         /* |grad_scale| sqrt(sumsq): infinite or NaN where a gradient is, or where fp32 cannot hold it */
  float coef;         /* max_norm / norm where norm > max_norm, else 1; 0 where norm is not finite */
  int32_t nonfinite;  /* 1 where norm is not finite */
  int32_t reserved[3];
} taw_clip_state;

/* Bytes of scratch taw_grad_sumsq and taw_grad_norm need for such a list (0 for an invalid one). */
size_t taw_grad_norm_workspace_bytes(const taw_tensor* tensors, int32_t count);

/* Fills *state for the gradients grad_scale * g of the list.  Squares and sums are taken in fp64.  max_norm > 0 (infinity: measure
 * only). */
int taw_grad_norm(const taw_tensor* tensors, int32_t count, float max_norm, float grad_scale, taw_clip_state* state,
                  void* workspace, size_t workspace_bytes, void* stream);

/* The two halves, for shards that live on several devices: state->sumsq (=|+= with accumulate) the list's sum of squares; the
 * owners add up their state->sumsq (an all-reduce of one double), and taw_clip_coef fills in the rest. */
int taw_grad_sumsq(const taw_tensor* tensors, int32_t count, int32_t accumulate, taw_clip_state* state, void* workspace,
                   size_t workspace_bytes, void* stream);
int taw_clip_coef(taw_clip_state* state, float max_norm, float grad_scale, void* stream);

/* g *= state->coef for every tensor of the list, in place.  Nothing is touched where coef is 1 or the norm is not finite. */
int taw_grad_clip(const taw_tensor* tensors, int32_t count, const taw_clip_state* state, void* stream);

/* taw_optimizer_step on clipped gradients: opt->grad_scale * state->coef in the place of grad_scale (taw_grad_norm is given the
 * same grad_scale).  Where state->nonfinite is set the step is skipped: the chunk, master, m and v stay as they are, and G_shard
 * is zeroed where opt->zero_grad asks for it.  state must not overlap the arrays. */
int taw_optimizer_step_clipped(const taw_adamw_desc* opt, const taw_clip_state* state, void* W_chunk, int32_t chunk_dtype,
                               float* master, float* m, float* v, float* G_shard, size_t n_elems, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TAW_MODEL_H */
