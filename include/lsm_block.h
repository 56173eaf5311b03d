/*
 * lsm_block.h -- operators around the token mixer of lsm.h in one block of a model: the norm and rotation of the queries
 * and keys that go into it (forward and backward), the mixture-of-experts layer behind it for a few tokens, and one step
 * of a beam search with the recurrent states rearranged.
 *
 * Conventions of lsm.h: device pointers, 16-byte aligned; the caller owns every buffer; nothing is allocated, kept between
 * calls or synchronised; all work is enqueued on `stream`; outputs are overwritten and alias neither inputs nor each other
 * (but the results of lsm_qk_norm_rope may take its inputs' place, and lsm_state_reorder works in place); results are
 * bitwise reproducible (no floating-point atomics); every argument check comes before the first HIP call.
 */
#ifndef LSM_BLOCK_H
#define LSM_BLOCK_H

#include "lsm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- per-head norm of queries and keys with the rotation by position ------------------------------------------------ */

typedef enum {
    LSM_NORM_NONE = 0, /* r = 1                                                                     */
    LSM_NORM_RMS  = 1, /* r = (mean of x_i^2 + eps)^(-1/2)                                            */
    LSM_NORM_L2   = 2  /* r = (sum of x_i^2 + eps)^(-1/2): rows of unit length (the delta rule's keys)   */
} lsm_norm_kind;

/* Which features a rotation takes together, of the first rot_dim. */
typedef enum {
    LSM_ROT_HALVES = 0, /* i and i + rot_dim/2 */
    LSM_ROT_PAIRS  = 1  /* 2i and 2i + 1       */
} lsm_rotation;

/* Element (b, h, t, i) of a tensor is at b*batch + h*head + t*token + i, in elements. */
typedef struct { int64_t batch, head, token; } lsm_strides;

typedef struct {
    uint32_t struct_size;     /* = sizeof(lsm_qk_params)                                                            */
    int32_t  B, T;            /* sequences and tokens of each (packed input: B = 1), B * T at most 2^30 and, forward,
                                 the rows of one head at most 2^36 - 4096 bytes (LSM_ERR_SHAPE beyond)               */
    int32_t  H_q, H_k, d;     /* heads of q and of k (H_k = 0: no k), d in {64,128,256}                               */
    int32_t  dtype;           /* lsm_dtype of q, k, their outputs and gradients                                     */
    int32_t  norm, rotation;  /* lsm_norm_kind, lsm_rotation                                                        */
    int32_t  rot_dim, n_pos;  /* rotated features (0: none; a multiple of 16, at most d) and rows of the table      */
    float    eps;             /* > 0 where there is a norm                                                          */
    float    q_scale, k_scale;/* factor of the outputs (the 1/sqrt(d) that lsm.h leaves to its callers)             */
    int32_t  reserved;        /* 0                                                                                  */
    lsm_strides q, k;         /* inputs: slices of a fused projection as they stand                                  */
    lsm_strides q_out, k_out; /* outputs, and their gradients in the backward call                                   */
    lsm_strides dq, dk;       /* gradients of the inputs (backward only)                                             */
} lsm_qk_params;

/*
 * For every row x (one head of one token of q or k):   y = scale * R_p (w * (r x)) ,
 * R_p the rotation of the token's position p: (a, b) -> (a cos - b sin, b cos + a sin) for the feature pairs of the first
 * rot_dim features, the others as they are.
 *   q, k        dtype, by strides; strides of axes longer than 1 in whole 16-byte pieces                       in
 *   q_weight, k_weight   [d] fp32 or NULL (= 1)                                                                in
 *   cos_sin     [n_pos, rot_dim] fp32: rot_dim/2 cosines, then rot_dim/2 sines; NULL exactly when rot_dim = 0      in
 *   positions   [B, T] int32 or NULL (= 0..T-1 in every sequence, T <= n_pos then); not read when rot_dim = 0.
 *               A position outside [0, n_pos) makes that token's rows NaN (the table is not read for it)       in
 *   q_out, k_out   dtype, by strides with which no two rows share an element (nor with those of dq, dk; rows of
 *               inputs and of d_q_out, d_k_out may repeat); may be q, k themselves, with their strides            out
 * Squares, sums and the rotation are computed in fp32; a row's elements that are not finite reach that row alone.
 */
int lsm_qk_norm_rope(const lsm_qk_params* p, const void* q, const void* k, const float* q_weight, const float* k_weight,
                     const float* cos_sin, const int32_t* positions, void* q_out, void* k_out, void* stream);

/*
 * Backward of L = <q_out, d_q_out> + <k_out, d_k_out>; only the inputs are needed, nothing saved by the forward call.
 *   d_q_out, d_k_out   dtype, by the strides q_out, k_out                                                      in
 *   dq, dk             dtype, by the strides dq, dk                                                            out
 *   d_q_weight, d_k_weight   [d] fp32; given only where the weight was given, NULL skips it                     out
 *   workspace          at least lsm_qk_norm_rope_bwd_workspace_bytes(p) (0 for invalid params)
 */
size_t lsm_qk_norm_rope_bwd_workspace_bytes(const lsm_qk_params* p);
int lsm_qk_norm_rope_bwd(const lsm_qk_params* p, const void* q, const void* k, const float* q_weight, const float* k_weight,
                         const float* cos_sin, const int32_t* positions, const void* d_q_out, const void* d_k_out,
                         void* dq, void* dk, float* d_q_weight, float* d_k_weight,
                         void* workspace, size_t workspace_bytes, void* stream);

/* ---- a mixture-of-experts layer for a few tokens ----------------------------------------------------------------------- */

typedef struct {
    uint32_t struct_size; /* = sizeof(lsm_moe_params)                                                         */
    int32_t  n, D, F;     /* tokens (1..128), their width and the experts' (multiples of 8, at most 65536)     */
    int32_t  E, top_k;    /* experts (1..256) and how many of them a token goes to (1..16, at most E)         */
    int32_t  dtype;       /* lsm_dtype of everything below                                                    */
    int32_t  renormalise; /* 1: the chosen experts' weights sum to 1; 0: they are the softmax over all experts */
} lsm_moe_params;

/*
 * For every token x:   p = softmax(router x) over the E experts,  S = the top_k experts of largest router output (equal
 * ones by rising index),  w_e = p_e or p_e / sum_S p,
 *     y = residual + sum_{e in S} w_e Wd_e (silu(Wg_e x) * (Wu_e x)) ,      silu(z) = z / (1 + exp(-z)) .
 *   x          [n, D]                                                                               in
 *   router     [E, D]                                                                               in
 *   w_gate_up  [E, 2 F, D]: F rows of Wg_e, then F rows of Wu_e                                       in
 *   w_down     [E, D, F]: Wd_e                                                                       in
 *   residual   [n, D] or NULL (= 0)                                                                 in
 *   y          [n, D]                                                                               out
 *   workspace  at least lsm_moe_step_workspace_bytes(p) (0 for invalid params)
 * The form for decoding: the active experts' weights are read once, whatever the tokens that share them.  Beside lsm_moe_route,
 * lsm_moe_plan and lsm_moe_experts of lsm_train.h it is the faster one up to about 100 tokens, and as fast at 128 (64 experts of 1024 x
 * 1024, 8 a token, bf16: one token 23 us against 59, 32 tokens 92 against 101, 128 tokens 106 against 104); they are the form for more tokens,
 * and for training.  Sums are fp32; with bf16 elements the hidden activations are kept as a bf16 head and a bf16 remainder, so that the one
 * rounding to bf16 is the result's.  A token with a router output of NaN or +inf, or with none above -inf, gets a row of NaN (beside
 * finite ones an expert of -inf has the weight 0); other tokens are not affected.
 */
size_t lsm_moe_step_workspace_bytes(const lsm_moe_params* p);
int lsm_moe_step(const lsm_moe_params* p, const void* x, const void* router, const void* w_gate_up, const void* w_down,
                 const void* residual, void* y, void* workspace, size_t workspace_bytes, void* stream);

/* ---- one step of a beam search --------------------------------------------------------------------------------------- */

typedef struct {
    uint32_t struct_size; /* = sizeof(lsm_beam_params)                                                       */
    int32_t  B, K, V;     /* sequences (below 2^23), beams of each (at most 32), vocabulary; K * V at most 2^25;
                             B * K * ceil(V / 4096) below 2^24 will do always (LSM_ERR_SHAPE beyond a launch) */
    int32_t  n_out;       /* candidates wanted of each sequence: 1..32, at most K * V                        */
    int32_t  dtype;       /* lsm_dtype of the logits                                                         */
    int32_t  eos;         /* the token that ends a beam, or -1                                               */
    int32_t  reserved;    /* 0                                                                               */
    int64_t  row_stride;  /* elements between the logits of consecutive beams, >= V                          */
} lsm_beam_params;

/*
 * The n_out best candidates (beam k, token t) of every sequence by
 *     score(k, t) = scores[k] + ((x_t - m) - log(sum_t exp(x_t - m))) ,   m = max_t x_t ,   x = logits of beam k,
 * in fp32; a finished beam offers (k, eos) at scores[k] and nothing else (its logits are not read).
 *   logits     [B, K, V] dtype, rows row_stride apart (what lies between them is read but not used)             in
 *   scores     [B, K] fp32: the beams' log-probabilities so far (-inf: no such beam)                        in
 *   finished   [B, K] bytes (0 or not), or NULL; needs eos >= 0                                             in
 *   out_scores, parent, token   [B, n_out] fp32, int32, int32                                              out
 *   out_finished   [B, n_out] bytes 0 / 1: the parent was finished or the token is eos; NULL skips it, must be NULL
 *              where eos < 0                                                                               out
 *   workspace  at least lsm_beam_select_workspace_bytes(p) (0 for invalid params); contents undefined after the call
 * Candidates come by falling score, equal ones by rising k * V + t (all K V of them take part, those at -inf too).
 * A logit that is NaN counts as -inf and +inf as the largest finite number of its type; a score that comes out NaN is -inf.
 */
size_t lsm_beam_select_workspace_bytes(const lsm_beam_params* p);
int lsm_beam_select(const lsm_beam_params* p, const void* logits, const float* scores, const uint8_t* finished,
                    float* out_scores, int32_t* parent, int32_t* token, uint8_t* out_finished,
                    void* workspace, size_t workspace_bytes, void* stream);

/*
 * The states that belong to the beams follow them, in place: row b K + i of every tensor becomes what row b K + parent[b, i]
 * was before the call.
 *   states     HOST array of n_states (1..64) device pointers to [B * K] rows, no two tensors sharing memory  in/out
 *   row_bytes  HOST array: bytes of a row of each, a multiple of 4
 *   parent     [B, K] int32; a value outside [0, K) fills its row with 0xff bytes (NaN)                      in
 * Rows that stay where they are (parent[b, i] = i) are not touched.  B at most 65535, K at most 32.
 */
int lsm_state_reorder(void* const* states, const size_t* row_bytes, int n_states, const int32_t* parent, int B, int K,
                      void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LSM_BLOCK_H */
