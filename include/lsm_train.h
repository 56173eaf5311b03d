/*
 * lsm_train.h -- operators that training a Linear-MoE model needs around the token mixer of lsm.h: routing tokens to experts,
 * the experts' products for many tokens, and the losses over a large vocabulary, each with its backward pass.
 *
 * Conventions of lsm.h: device pointers, 16-byte aligned; the caller owns every buffer; nothing is allocated, kept between
 * calls or synchronised; all work is enqueued on `stream`; outputs are overwritten and alias neither inputs nor each other;
 * results are bitwise reproducible (no floating-point atomics); every argument check comes before the first HIP call.  Sizes of
 * which a launch would need 2^32 threads are refused (LSM_ERR_SHAPE).
 */
#ifndef LSM_TRAIN_H
#define LSM_TRAIN_H

#include "lsm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- routing ------------------------------------------------------------------------------------------------------- */

typedef struct {
    uint32_t struct_size; /* = sizeof(lsm_route_params)                                                        */
    int32_t  n, E, top_k; /* tokens, experts (1..256), how many of them a token goes to (1..16, at most E); n * top_k at most 2^24 */
    int32_t  dtype;       /* lsm_dtype of the logits and of their gradient                                    */
    int32_t  renormalise; /* 1: a token's weights sum to 1; 0: they are the softmax over all experts           */
} lsm_route_params;

/*
 * For every token:   S = the top_k experts of largest logit, by falling logit, equal ones by rising index,
 *     w_e = exp(l_e) / sum_S exp(l)   (renormalise)   or   exp(l_e) / sum over all experts   for e in S.
 *   logits     [n, E] dtype                                                                          in
 *   weights    [n, top_k] fp32                                                                       out
 *   chosen     [n, top_k] int32                                                                      out
 * A logit that is NaN counts as -inf and +inf as the largest finite number of its type.  An expert of -inf is never chosen:
 * where fewer than top_k are left the other places hold the expert -1 and the weight 0, and a token of none (padding) goes to
 * no expert at all.
 */
int lsm_moe_route(const lsm_route_params* p, const void* logits, float* weights, int32_t* chosen, void* stream);

/*
 * Backward of L = <weights, d_weights>, from the logits and the experts chosen by the forward call.
 *   chosen     [n, top_k] int32; outside [0, E): no expert; one that stands twice counts once in S, its gradients add   in
 *   d_weights  [n, top_k] fp32; not used where there is no expert                                    in
 *   d_logits   [n, E] dtype                                                                          out
 */
int lsm_moe_route_bwd(const lsm_route_params* p, const void* logits, const int32_t* chosen, const float* d_weights,
                      void* d_logits, void* stream);

/*
 * The (token, expert) pairs sorted by expert, those of an expert by rising pair t * top_k + j.
 *   chosen     [n, top_k] int32; outside [0, E): the pair is left out                                 in
 *   offsets    [E + 1] int32: the pairs of expert e are at offsets[e] .. offsets[e + 1] - 1            out
 *   order      [n top_k] int32: the pair at each place; -1 behind offsets[E]                          out
 *   place      [n, top_k] int32: the place of each pair, -1 where it is left out                       out
 *   workspace  at least lsm_moe_plan_workspace_bytes(p) (0 for invalid params, and where none is needed: up to 8192 pairs)
 * Of p only n, E and top_k count.
 */
size_t lsm_moe_plan_workspace_bytes(const lsm_route_params* p);
int lsm_moe_plan(const lsm_route_params* p, const int32_t* chosen, int32_t* offsets, int32_t* order, int32_t* place,
                 void* workspace, size_t workspace_bytes, void* stream);

/* ---- the experts of many tokens ---------------------------------------------------------------------------------------- */

typedef struct {
    uint32_t struct_size; /* = sizeof(lsm_experts_params)                                                     */
    int32_t  n, D, F;     /* tokens, their width and the experts' (multiples of 8, at most 65536; 2 F D * element size below 2^32 - 4096) */
    int32_t  E, top_k;    /* experts (1..256), pairs of a token (1..16); n * top_k at most 2^24                */
    int32_t  dtype;       /* lsm_dtype of x, weights of the experts, y and all their gradients                */
    int32_t  reserved;    /* 0                                                                               */
    int64_t  x_stride;    /* elements between rows of x, >= D, a multiple of 8; n * x_stride * element size below 2^32 - 4096 */
    int64_t  dy_stride;   /* the same of d_y (backward only)                                                  */
} lsm_experts_params;

/*
 * (Up to about 100 tokens forward alone lsm_moe_step of lsm_block.h is the faster form.)
 * For every token t:   y_t = residual_t + sum_j weights[t, j] Wd_e (silu(Wg_e x_t) * (Wu_e x_t)) ,   e the expert of pair (t, j),
 * over the pairs that the plan of lsm_moe_plan holds (offsets, order, place).
 *   x          [n, D], rows x_stride apart                                                          in
 *   weights    [n, top_k] fp32                                                                       in
 *   offsets, order, place   as lsm_moe_plan leaves them for the same n, E and top_k                    in
 *   w_gate_up  [E, 2 F, D]: F rows of Wg_e, then F rows of Wu_e                                       in
 *   w_down     [E, D, F]: Wd_e                                                                       in
 *   residual   [n, D] or NULL (= 0)                                                                 in
 *   y          [n, D]                                                                               out
 *   workspace  at least lsm_moe_experts_workspace_bytes(p) (0 for invalid params)
 * Products of the elements as they are, sums in fp32, over a token's pairs too; with bf16 elements the result is rounded to bf16, and in
 * calls of more than 16 tokens the hidden activations as well (in smaller calls what their rounding leaves goes along).  A number that is
 * not finite in x reaches the rows of its token alone.
 */
size_t lsm_moe_experts_workspace_bytes(const lsm_experts_params* p);
int lsm_moe_experts(const lsm_experts_params* p, const void* x, const float* weights, const int32_t* offsets, const int32_t* order,
                    const int32_t* place, const void* w_gate_up, const void* w_down, const void* residual, void* y,
                    void* workspace, size_t workspace_bytes, void* stream);

/*
 * Backward of L = <y, d_y>; nothing is saved by the forward call, the hidden activations are formed again.  (The residual's
 * gradient is d_y.)
 *   d_y          [n, D], rows dy_stride apart                                                       in
 *   dx           [n, D] through the experts                                                         out
 *   d_weights    [n, top_k] fp32; 0 for a pair that is left out                                      out
 *   d_w_gate_up  [E, 2 F, D], d_w_down [E, D, F]; 0 for an expert without tokens                      out
 *   workspace    at least lsm_moe_experts_bwd_workspace_bytes(p) (0 for invalid params)
 * With bf16 elements the hidden activations' gradients, and the activations times their weight, are rounded to bf16 on their way
 * into the next product (for dx in calls of up to 16 tokens: with what the rounding leaves).
 * d_w_gate_up and d_w_down: both or neither (NULL: not wanted, as in a layer whose experts are frozen).
 */
size_t lsm_moe_experts_bwd_workspace_bytes(const lsm_experts_params* p);
int lsm_moe_experts_bwd(const lsm_experts_params* p, const void* x, const float* weights, const int32_t* offsets,
                        const int32_t* order, const int32_t* place, const void* w_gate_up, const void* w_down, const void* d_y,
                        void* dx, float* d_weights, void* d_w_gate_up, void* d_w_down,
                        void* workspace, size_t workspace_bytes, void* stream);

/* ---- losses over a vocabulary ------------------------------------------------------------------------------------------- */

typedef struct {
    uint32_t struct_size; /* = sizeof(lsm_vocab_params)                                                       */
    int32_t  n, D, V;     /* tokens (1..2^24), their width (a multiple of 8, at most 65536), vocabulary (1..2^24)  */
    int32_t  K;           /* 0: one target a token; 1..256: so many logits of a teacher, n * K at most 2^28       */
    int32_t  dtype;       /* lsm_dtype of x, w and their gradients                                            */
    float    temperature; /* 2^-127 or more: divides the logits, the teacher's too                            */
    int32_t  reserved;    /* 0                                                                               */
    int64_t  x_stride;    /* elements between rows of x, >= D, a multiple of 8; n * x_stride * element size below 2^32 - 4096 */
} lsm_vocab_params;

/*
 * For every token:   z_v = <x, w_v> / temperature ,   lse = log sum_v exp(z_v) ,
 *     K = 0:   loss = lse - z_target ,
 *     K > 0:   loss = sum_j p_j (log p_j - (z_{index_j} - lse)) ,   p = softmax(teacher / temperature) over the token's entries
 * (the divergence of the model from the teacher, whose other tokens count as impossible).  The logits are never kept; of every 32 to
 * 128 of a token's the workspace holds a maximum and a sum, 8 bytes (16384 tokens, 131072 columns, bf16: 134 MB).
 *   x          [n, D], rows x_stride apart                                                          in
 *   w          [V, D]                                                                               in
 *   index      [n] (K = 0: the target) or [n, K] int32                                               in
 *   teacher    [n, K] fp32; NULL exactly when K = 0                                                  in
 *   loss, lse  [n] fp32                                                                             out
 *   workspace  at least lsm_vocab_loss_workspace_bytes(p) (0 for invalid params)
 * An index outside [0, V) is no target and no entry, nor is a teacher's logit of -inf or NaN (+inf counts as the largest finite
 * number).  Entries of the same index each count with their own p: their gradients add up, and the loss is the sum as it stands, which is
 * less than the divergence from the teacher with such entries made one, by what their p log p differ.
 * A token without target or entries is left out: its row of x is not read, loss and lse are 0.  Sums are fp32.  A token with a logit of
 * 2^127 or more (or NaN) gets a loss that is not finite.
 */
size_t lsm_vocab_loss_workspace_bytes(const lsm_vocab_params* p);
int lsm_vocab_loss(const lsm_vocab_params* p, const void* x, const void* w, const int32_t* index, const float* teacher,
                   float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Backward of L = <loss, d_loss>, with lse from the forward call; the logits are formed again, a piece of the vocabulary at a time.
 *   d_loss     [n] fp32; not used for tokens that are left out                                        in
 *   dx         [n, D]; 0 for tokens that are left out                                               out
 *   dw         [V, D], or NULL (not wanted)                                                        out
 *   workspace  at least lsm_vocab_loss_bwd_workspace_bytes(p) (0 for invalid params)
 * With bf16 elements the gradient of the logits is rounded to bf16 on its way into the next products (of up to 16 tokens: with what
 * the rounding leaves).
 */
size_t lsm_vocab_loss_bwd_workspace_bytes(const lsm_vocab_params* p);
int lsm_vocab_loss_bwd(const lsm_vocab_params* p, const void* x, const void* w, const int32_t* index, const float* teacher,
                       const float* lse, const float* d_loss, void* dx, void* dw,
                       void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LSM_TRAIN_H */
