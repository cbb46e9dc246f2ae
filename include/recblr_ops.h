/*
 * recblr_ops.h - C ABI of librecblr.so next to the BD-LRU layer (recblr.h): a
 * recurrence with a matrix state (the gated delta rule), AdamW over many
 * tensors, and the choice of an item from logits.
 *
 * The conventions of recblr.h hold: dense row-major device tensors aligned to
 * their element size, `io` (RECBLR_F32 or RECBLR_BF16) for the type of the
 * sequence tensors, float states, a hipStream_t that a call only enqueues on,
 * a caller's workspace (256-byte aligned, NULL where its size is 0, not shared
 * by two calls in flight), validation on the host before anything is enqueued,
 * no allocation on the device, no synchronisation and no state kept between
 * calls.  Outputs must not overlap inputs or each other unless stated.  The
 * tensors and the stream belong to the current device.  Results repeat bit for
 * bit.
 */
#ifndef RECBLR_OPS_H_
#define RECBLR_OPS_H_

#include "recblr.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Gated delta rule: a linear recurrence whose state is a matrix S [Dk][Dv] for
 * each value head (Yang, Kautz and Hatamizadeh, "Gated Delta Networks").  For
 * every row b and value head j, with the query and key of head j / (HV / H):
 *     S_t = a_t (I - beta_t k_t k_t^T) S_{t-1} + beta_t k_t v_t^T,  a_t = e^{g_t}
 *     o_t = scale S_t^T q_t
 *   q, k : [B][L][H][Dk] io;  v, o : [B][L][HV][Dv] io;  g, beta : [B][L][HV] io
 *   h0, hT and every other state : [B][HV][Dk][Dv] float
 * 1 <= Dk, Dv <= 128, HV <= 4096, B HV ceil(Dv / 32) and B HV ceil(L / 64) below 2^24
 * (else UNSUPPORTED), HV a multiple of H (else INVALID_ARGUMENT).  g is the
 * logarithm of the decay, usually <= 0; below -100 it counts as -100, so -inf
 * leaves e^-100 of the (finite) state, nothing next to float's rounding.  Where g is
 * positive, its sums over successive steps of a group of 64 stay below 88, since
 * their powers of e are formed.  A step with g = 0 and beta = 0 leaves the state
 * as it is (padding); queries and keys are taken as given (they are usually
 * brought to length one by the caller).  Inputs are finite, in
 * padding too (g may be -inf): steps are worked on 64 at a time, and a NaN or an
 * infinity reaches the outputs of its whole group of 64 steps, those before it
 * among them, and what follows; other rows and heads are not touched by it.
 */
enum { RECBLR_OP_DELTA_FORWARD = 16, RECBLR_OP_DELTA_BACKWARD = 17 };

/* Steps between two kept states (below), and the bytes of workspace that `op` needs
 * (0: none, ws may be NULL; 0 for invalid arguments too). */
enum { RECBLR_DELTA_CHUNK = 64 };
size_t recblr_delta_workspace_size(int op, int64_t B, int64_t L, int64_t H, int64_t HV,
                                   int64_t Dk, int64_t Dv, int io);

/*
 * Forward from h0 (NULL: zero) to o and the final state hT (may be NULL).
 *   states : [B][HV][ceil(L / 64)][Dk][Dv] float or NULL, the states before the
 *            steps 0, 64, 128, ..., which the backward reads
 * L == 0 writes hT := h0 only.
 */
int recblr_delta_forward(const void* q, const void* k, const void* v, const void* g,
                         const void* beta, const float* h0, void* o, float* hT, float* states,
                         int64_t B, int64_t L, int64_t H, int64_t HV, int64_t Dk, int64_t Dv,
                         float scale, int io, void* ws, size_t ws_bytes, void* stream);

/*
 * Backward of recblr_delta_forward: the exact adjoint of the recurrence.
 *   states : the forward's (the initial state is the first of them)
 *   d_o : [B][L][HV][Dv] io;  dhT : [B][HV][Dk][Dv] float or NULL
 * Outputs: dq, dk [B][L][H][Dk], dv [B][L][HV][Dv], dg, dbeta [B][L][HV] io, dq and dk
 * summed over the value heads that share a query head; dh0 [B][HV][Dk][Dv] float
 * or NULL.  L == 0 writes dh0 := dhT (0 for NULL) only.
 */
int recblr_delta_backward(const void* q, const void* k, const void* v, const void* g,
                          const void* beta, const float* states, const void* d_o,
                          const float* dhT, void* dq, void* dk, void* dv, void* dg, void* dbeta,
                          float* dh0, int64_t B, int64_t L, int64_t H, int64_t HV, int64_t Dk,
                          int64_t Dv, float scale, int io, void* ws, size_t ws_bytes,
                          void* stream);

/* One token: q, k [B][H][Dk], v, o [B][HV][Dv], g, beta [B][HV];
 * h_prev, h_next [B][HV][Dk][Dv] float (h_next may == h_prev).  No workspace. */
int recblr_delta_step(const void* q, const void* k, const void* v, const void* g,
                      const void* beta, const float* h_prev, void* o, float* h_next, int64_t B,
                      int64_t H, int64_t HV, int64_t Dk, int64_t Dv, float scale, int io,
                      void* stream);

/*
 * AdamW (Loshchilov and Hutter: Adam with decoupled weight decay) over a list
 * of tensors, in place.  With m, v the moments, t the 1-based update count:
 *     m = beta1 m + (1 - beta1) grad,   v = beta2 v + (1 - beta2) grad^2
 *     param = param (1 - lr wd) - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 * param and grad are of type `io` (arithmetic in fp32, bf16 parameters rounded
 * to nearest even).
 *   state_bits = 32: m1, m2 are float [n]; scale1, scale2 are not read.
 *   state_bits = 8: m1 is int8 [n], m2 uint8 [n], with one float scale for each
 *     block of RECBLR_ADAMW_BLOCK elements of the tensor (the last one may be
 *     short), scale1, scale2 [ceil(n / block)].  A code c stands for
 *         m = scale1 sign(c) (c / 127)^2,    v = scale2 ((c + 1) / 256)^4,
 *     the scale is the block's largest |m| (or v) rounded to float, and a value
 *     takes the code nearest to it on the root's scale, i.e. 127 sqrt(|m| / s)
 *     and 256 (v / s)^(1/4) rounded.  Moments are updated and compared with the
 *     borders between codes in 64 bits, the step is taken with the moments
 *     before they are rounded to codes.  Zeroed codes and scales are the state
 *     before the first step.
 * Tensors of n = 0 are passed over.  NaN and Inf gradients propagate; with 8
 * bits they spread to the block, whose scale they become.
 * Errors: INVALID_ARGUMENT for a NULL list or pointer, misalignment, n < 0,
 * step < 1, or a tensor that is written and overlaps another one of the call
 * (the same tensor listed twice is one case); UNSUPPORTED for other state_bits
 * or io, or n > 2^36 - 4096.  `tensors` is host memory, read before the call returns.
 */
enum { RECBLR_ADAMW_BLOCK = 256 };

typedef struct {
    void* param;         /* [n] io */
    const void* grad;    /* [n] io */
    void* m1;            /* [n] float, or int8 codes */
    void* m2;            /* [n] float, or uint8 codes */
    float* scale1;       /* [ceil(n / 256)], 8-bit states only */
    float* scale2;
    int64_t n;
    double weight_decay; /* wd of this tensor */
} recblr_adamw_tensor;

int recblr_adamw_update(const recblr_adamw_tensor* tensors, int64_t count, int state_bits, int io,
                        int64_t step, double lr, double beta1, double beta2, double eps,
                        void* stream);

/* The values that 8-bit moments stand for: m1_out[i], m2_out[i] (float [n], either
 * list may be NULL) from tensors[i].m1, m2 and scales; param and grad are not read.
 * Errors as above: an output may overlap no other output and no moment or scale of the call. */
int recblr_adamw_moments(const recblr_adamw_tensor* tensors, int64_t count,
                         float* const* m1_out, float* const* m2_out, void* stream);

/*
 * One item a row from logits, by one given uniform number a row.
 *   logits : [B][V] io;  u : [B] float in [0, 1)
 *   temperature, top_p, min_p : [B] float or NULL (1, 1 and 0)
 *   top_k : [B] int32 or NULL (no limit)
 *   ids : [B] int32;  prob : [B] float or NULL
 * With w_i = exp((l_i - max l) / temperature), items in falling order of l_i
 * (equal ones in rising order of i):
 *   top_k: the first top_k stay (all of them where top_k <= 0);
 *   top_p: of these, the shortest run from the first whose w reach top_p of the
 *          sum of these (at least the first; all of them where top_p >= 1);
 *   min_p: of these, those with w_i >= min_p (1 is the largest w).
 * ids is the least i whose running sum of the w that stay, in order of i,
 * exceeds u times their sum (the last item with w > 0 for u >= 1), and prob is
 * w_ids over that sum.  temperature <= 0 takes the first item, prob 1.  A top_p or
 * min_p that is NaN sets no limit, and a NaN u counts as 1.
 * Masked items have the logit -inf, or any value far below the rest (the
 * type's lowest, say).  A row with no item (V = 0, all -inf) or none to be
 * chosen by its values (a NaN or +inf among logits, a NaN temperature) gives
 * id -1 and prob 0.
 * w are formed in 64 bits and summed as integers of 2^-F, F = 62 - ceil(log2 V), at
 * most 51: sums are exact whatever their order, and a w below half of that is 0.
 * Errors: INVALID_ARGUMENT, UNSUPPORTED (io, V > 2^24, B max(1, ceil(V / 4096)) >= 2^24),
 * WORKSPACE.
 */
size_t recblr_sample_workspace_size(int64_t B, int64_t V, int io);
int recblr_sample(const void* logits, const float* u, const float* temperature,
                  const int32_t* top_k, const float* top_p, const float* min_p, int32_t* ids,
                  float* prob, int64_t B, int64_t V, int io, void* ws, size_t ws_bytes,
                  void* stream);

#ifdef __cplusplus
}
#endif

#endif /* RECBLR_OPS_H_ */
