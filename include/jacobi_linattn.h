/*
 * jacobi_linattn.h -- C ABI of the linear-attention part of libjacobi_made.so: a recurrent layer whose state is a
 * matrix that decays at a rate of its head's,
 *
 *     S_t = lambda S_{t-1} + k_t v_t^T,      o_t = scale * S_t^T q_t,      lambda = exp(log_decay),   t = 1..T,
 *
 * for whole sequences (forward and gradients) and for single steps.  Like the recurrence of jacobi_rnn.h it is a
 * triangular system, here a linear one: a block of steps is solved at once from the state that enters it.
 *
 * Heads: `heads` query heads read `kv_heads` states; query head h reads state h / (heads / kv_heads).  A state, its
 * decay, k and v belong to a state head; heads must be a multiple of kv_heads.
 *
 * Arrays (DEVICE memory, owned by the caller; in the type `dtype` unless said otherwise):
 *   q, o, and their gradients [B, T, heads, Dk] and [B, T, heads, Dv];   k, v [B, T, kv_heads, Dk], [B, T, kv_heads, Dv]
 *   log_decay [kv_heads], states [B, kv_heads, Dk, Dv]: fp32 always.  log_decay is 0 (no decay) or below, -infinity
 *   included (no memory); it is a constant of the layer and gets no gradient.
 *   Packed sequences (offsets != NULL): the arrays over steps are [T, ...]; sequence b has the rows offsets[b] ..
 *   offsets[b+1] - 1 (int32, [B+1], not decreasing, within 0..T); rows outside every sequence are neither read nor written.
 *   A sequence without rows hands its state on unchanged.
 *   ld_*: elements from one row (all heads of a step) to the next, 0 = heads * D (no gap); the heads of a row lie side by
 *   side.  q, k and v may so be parts of one wider array.  Gradients have the strides of what they are gradients of.
 * Outputs and the workspace must not overlap anything else a call reads or writes, except that a state may be replaced in
 * place (state_out == state_in); one at another array's own address is refused.
 *
 * Calls are enqueued on `stream` (a hipStream_t, NULL = default stream) and return without waiting for the device; they
 * may be recorded into a graph.  The return value is MADE_OK or a negative made_status (jacobi_made.h),
 * made_last_error() has the message.  No call allocates memory.
 * Limits: 1 <= Dk, Dv <= 128; B >= 0, 0 <= T <= 2^30, and a launch's workgroups have fewer than 2^32 threads together
 * (bf16, a width above 64: 8 million states, 2.7 million for gradients; a step: 16 million parts of 32 or 128 values).
 * Inputs are finite: the steps of a block of 64 (fp32: 32) are products of the whole block, and a NaN or infinity in it
 * can reach every output row of its block, earlier ones too.
 *
 * Arithmetic: states, decays and sums are fp32.  MADE_F32: products are fp32.  MADE_BF16: products of bf16 values with
 * fp32 sums; scores, states and decayed values enter them as sums of two bf16 parts (2^-17 of each; three parts, 2^-25,
 * where a state is asked for), and only the outputs are rounded to bf16.  States beyond 2^117 may overflow.
 */
#ifndef JACOBI_LINATTN_H
#define JACOBI_LINATTN_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct linattn_config {
  int32_t B;              /* sequences                                                        */
  int32_t T;              /* steps of each sequence; packed: rows of the arrays               */
  int32_t heads;          /* query heads                                                      */
  int32_t kv_heads;       /* states, a divisor of heads                                       */
  int32_t Dk, Dv;         /* widths of a key and of a value, 1..128                           */
  int32_t dtype;          /* MADE_F32 or MADE_BF16                                            */
  float scale;
  int64_t ld_q, ld_k, ld_v, ld_o; /* elements between rows, 0 = no gap                        */
  const int32_t* offsets; /* device, [B+1], or NULL: B sequences of T steps                   */
} linattn_config;

/*
 * linattn_workspace_bytes -- size of the workspace linattn_forward (backward = 0) or linattn_backward (backward = 1) takes
 * to split long sequences over the device; offsets is only looked at for being NULL or not (packed sequences: any one may
 * have all T rows, and there is room for a state of each beside those of the segments).  A workspace serves one call at a
 * time: calls that may run at once (other streams, other graphs) need one each.  *bytes may be 0.
 */
int linattn_workspace_bytes(const linattn_config* cfg, int32_t backward, int64_t* bytes);

/*
 * linattn_forward -- o for every step.
 *   state_in : [B, kv_heads, Dk, Dv] state before the first step, or NULL (zeros)
 *   state_out: the state after the last step, or NULL; may be state_in
 *   workspace: workspace_bytes of device memory, 256-byte aligned.  With fewer bytes than linattn_workspace_bytes says
 *              (or NULL) every sequence is computed from its first step to its last by one workgroup a head: the same
 *              result up to the order of sums, later.
 */
int linattn_forward(const linattn_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
                    const float* state_in, void* o, float* state_out, void* workspace, int64_t workspace_bytes, void* stream);

/*
 * linattn_backward -- gradients of a loss from d_o = dL/do and, where the last state is used further, d_state_out:
 *     dq_t = scale (S_t do_t),   dk_t = R_t v_t,   dv_t = R_t^T k_t,   R_t = lambda R_{t+1} + scale q_t do_t^T
 * (R_T+1 = d_state_out / lambda), sums over the query heads of a state for dk and dv.
 *   state_in   : as given to linattn_forward, or NULL;   d_state_out: [B, kv_heads, Dk, Dv] or NULL (zeros)
 *   dq, dk, dv : like q, k, v (outputs);   d_state_in: [B, kv_heads, Dk, Dv] gradient of state_in, or NULL; not
 *                d_state_out itself
 * Sums are taken in an order that depends on the sizes alone: equal calls give equal bits.
 */
int linattn_backward(const linattn_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
                     const float* state_in, const void* d_o, const float* d_state_out, void* dq, void* dk, void* dv,
                     float* d_state_in, void* workspace, int64_t workspace_bytes, void* stream);

/*
 * linattn_step -- one step of cfg->B sequences (cfg->T and offsets are not looked at): arrays over steps are [B, ...],
 * states are replaced in place.
 *   state: [n_slots, kv_heads, Dk, Dv];   slots: device int32 [B], the place of each row's state, or NULL: row b has
 *   place b (then n_slots >= B).  A row whose slot is negative or not below n_slots is left out: its o is not written.
 *   Rows that name the same slot are taken one after the other in the order of the rows; to find them every workgroup reads
 *   all of slots, so that very many rows cost time with the square of B (2 heads of 64 x 64: 4096 rows 86 us, 59 without
 *   slots; 32768 rows 1.8 ms and 0.5).
 */
int linattn_step(const linattn_config* cfg, const void* q, const void* k, const void* v, const float* log_decay, float* state,
                 int32_t n_slots, const int32_t* slots, void* o, void* stream);

#ifdef __cplusplus
}
#endif
#endif
