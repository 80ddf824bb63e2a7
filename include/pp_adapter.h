/* pp_adapter.h -- C ABI of low-rank adapters beside the block-pruned matrix product, for AMD MI355X (gfx950).
 *
 * A pruned layer's weights are packed once (pp_block_gemm.h) and shared; what a user or a task adds to them is a
 * product of two thin matrices.  A bank holds the adapters of one layer in numbered slots: slot s has A_s [rank][k],
 * B_s [m][rank] and a factor c_s, each slot with a rank of its own.  Every column of x -- a token -- names its slot:
 *
 *   u[:, t] = A_s x[:, t]                                    s = slot_of[t]
 *   y[:, t] = act( Wd x[:, t] + bias + c_s B_s u[:, t] )     without the last term where the token has no adapter
 *
 * and the gradients that train the adapters, Wd staying as it is, for dy = the gradient with respect to y:
 *
 *   g = dy where act let through, 0 elsewhere;      v[:, t] = B_s^T g[:, t]
 *   dx[:, t] = Wd^T g[:, t] + c_s A_s^T v[:, t]
 *   dA_s = c_s sum_t v[:, t] x[:, t]^T,   dB_s = c_s sum_t g[:, t] u[:, t]^T      over the tokens of slot s
 *
 * slot_of_dev is int32 [n] in device memory, read when the kernels run (a captured graph can be replayed with other
 * contents).  A value outside 0 .. slots - 1 (-1 by convention) and a slot that nothing is loaded into are "no adapter".  Tokens may
 * name slots in any order; tokens of one slot next to each other are fastest.  What an infinity or a NaN in one token's column or in one
 * slot's matrices does stays with that token, with that slot's tokens and with that slot's gradients.
 * Two things bound that.  Where x was held in 8 bits, 128 neighbouring tokens share a step, whatever their slots: one value that is not finite
 * makes its row's whole block NaN, and with it that column of dA for every slot with a token in the block; a large one makes the others'
 * steps coarse.  Columns of padding tokens are set to zero before pp_act8_pack, then they do neither.  And in a PP_F16 bank
 * products that the formulas make infinite may come out as NaN (an infinity meets both parts of u or v, one of which may be 0), which a
 * ReLU stores as 0.
 *
 * Storage is the bank's dtype for x, y, dy, g, dx, A and B; sums, u, v and the gradients of A and B are binary32.  In a
 * PP_F16 bank u and v enter products as two binary16 parts with a power of two taken out, which leaves them 20 bits or more,
 * and 2^-38 of the largest of what shares the power: 16 ranks of a token for y and dx, 128 tokens of a rank for dA and dB.
 *
 * Pointers named *_dev are device pointers to the device the bank was made on, which has to be current, and the plan's
 * (PP_ERR_DEVICE otherwise).  Matrices are row-major without gaps and 16-byte aligned, lists of
 * slots 4-byte aligned.  Runs only read the bank and the plan: any number may be in flight at
 * once, each with buffers of its own.  A load of a slot is ordered against its uses by the caller (one stream does).
 * Status codes, dtypes and flags are those of pp_conv.h.  Validation comes before any device call.  No call throws; none but plan and destroy
 * synchronises or allocates, so all others can be captured into a graph.
 */
#ifndef PP_ADAPTER_H
#define PP_ADAPTER_H

#include <stdint.h>

#include "pp_act8.h"
#include "pp_block_gemm.h"
#include "pp_conv.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pp_adapter_bank pp_adapter_bank_t; /* opaque; owned by the library */

typedef struct {
    int32_t m, k;        /* rows (outputs) and columns (inputs) of the layer, 1 .. 4194304, m * k at most 2^31 - 1 */
    int32_t slots;       /* 1 .. 65536 */
    int32_t max_rank;    /* the largest rank a slot can take, 1 .. 128 */
    int32_t dtype;       /* pp_dtype_t */
    uint32_t flags;      /* PP_FLAG_HOST_ONLY: sizes and checks only, touches no device */
} pp_adapter_desc_t;

/* Allocate a bank with empty slots on the current device.  PP_ERR_SHAPE: a size out of range.  PP_ERR_UNSUPPORTED: an
 * unknown dtype or flag.  PP_ERR_DEVICE: no device, or not enough of its memory (each slot takes about
 * 4 (m + k) max_rank bytes, twice that with PP_F32). */
pp_status_t pp_adapter_plan(const pp_adapter_desc_t *desc, pp_adapter_bank_t **out_bank);

/* Enqueue the loading of a slot: a_dev [rank][k], b_dev [m][rank] are copied into the orders that the kernels read, for
 * both directions.  rank 0 empties the slot (a_dev and b_dev are not read).  PP_ERR_SHAPE: a slot or rank out of
 * range.  PP_ERR_UNSUPPORTED: a scale that is not finite. */
pp_status_t pp_adapter_load(pp_adapter_bank_t *bank, int32_t slot, int32_t rank, float scale, const void *a_dev, const void *b_dev, void *hip_stream);

/* Enqueue the loading of count slots, as count calls of pp_adapter_load in their order would, in a launch for each 64 of them
 * (fewer where a slot is listed twice: the last of its entries stays).  The five arrays are host memory, count entries each, read before
 * the call returns; a_dev and b_dev list device pointers, not read where rank is 0.  If one entry is refused, nothing is loaded.
 * Refusals as pp_adapter_load; PP_ERR_SHAPE also: count < 1. */
pp_status_t pp_adapter_load_many(pp_adapter_bank_t *bank, int32_t count, const int32_t *slot, const int32_t *rank, const float *scale,
                                 const void *const *a_dev, const void *const *b_dev, void *hip_stream);

/* Sizes of what a run leaves for the backward pass, for n tokens: u (of A x) and v (of B^T g), opaque, 16-byte aligned.
 * A buffer belongs to the n it was made for.  0 if n is out of range. */
int64_t pp_adapter_u_bytes(const pp_adapter_bank_t *bank, int32_t n);
int64_t pp_adapter_v_bytes(const pp_adapter_bank_t *bank, int32_t n);
/* Scratch memory of pp_adapter_grad_weights for n tokens and count slots (at least 16): about 8 n max_rank bytes a slot up to 256 MB, over
 * which longer lists are gone through in parts. */
int64_t pp_adapter_work_bytes(const pp_adapter_bank_t *bank, int32_t n, int32_t count);

/* Enqueue u = A x alone: x_dev [k][n].  What pp_adapter_run leaves in u_dev. */
pp_status_t pp_adapter_project(const pp_adapter_bank_t *bank, const void *x_dev, const int32_t *slot_of_dev, void *u_dev, int32_t n, void *hip_stream);

/* Enqueue y = act(Wd x + bias + c B (A x)): x_dev [k][n], y_dev [m][n]; u_dev is scratch that a later
 * pp_adapter_grad_weights can be given.  plan is the layer's pp_block_gemm plan (m, k, dtype equal to the bank's; bias and act
 * are the plan's).  The adapters' part is added before act and before y is rounded.  PP_ERR_SHAPE: n < 1 or above 4194304, k * n or m * n beyond
 * 2^31 - 1, or a plan of another size or of the transposed weights.  PP_ERR_UNSUPPORTED: another dtype, a host-only bank or plan, a PP_F16 plan with a forced
 * variant (variant 1 has no adapters; variant 2 takes n that are multiples of 8 only).  PP_ERR_ALIGN: misaligned, or an output that overlaps another buffer. */
pp_status_t pp_adapter_run(const pp_adapter_bank_t *bank, const pp_block_gemm_plan_t *plan, const void *x_dev, const int32_t *slot_of_dev, void *u_dev,
                           void *y_dev, int32_t n, void *hip_stream);

/* Enqueue the first half of the backward pass, from dy_dev [m][n]:
 *   gate_dev   the layer's output y in 8 bits (pp_act8_pack of [m][n]) if the layer has a ReLU: g = dy where y > 0, written to
 *              g_dev [m][n] (dy_dev itself is allowed).  NULL: g = dy, and g_dev is not used.
 *   v_dev      receives v = B^T g
 *   dx_dev     [k][n], from plan_t, the plan of the layer's transposed weights that pp_block_gemm_plan_transposed makes (one of
 *              pp_block_gemm_plan: PP_ERR_SHAPE, so that a square layer's own plan is not taken for it).  NULL (plan_t is not
 *              used then): no gradient with respect to x is wanted.
 * Refusals as pp_adapter_run. */
pp_status_t pp_adapter_grad_input(const pp_adapter_bank_t *bank, const pp_block_gemm_plan_t *plan_t, const void *dy_dev, const void *gate_dev, void *g_dev,
                                  const int32_t *slot_of_dev, void *v_dev, void *dx_dev, int32_t n, void *hip_stream);

/* Enqueue the second half: the gradients of the count slots that which_dev (int32, device memory) lists.
 *   x_dev      the layer's input [k][n]; with x_is_act8 non-zero its 8-bit form (pp_act8_pack)
 *   u_dev, v_dev, g_dev   of pp_adapter_run or pp_adapter_project, of pp_adapter_grad_input, and g (dy if there was no gate)
 *   da_dev     binary32 [count][max_rank][k], rows from the slot's rank on are zeros
 *   db_dev     binary32 [count][m][max_rank], columns from the slot's rank on are zeros
 *   work_dev   pp_adapter_work_bytes bytes of scratch
 * An entry of which_dev outside 0 .. slots - 1, an empty slot and one that no token names get zeros; a slot may be listed twice.
 * u and v say with which rank and factor they were made, and dB takes those of u, dA those of v: what has been loaded into a slot since
 * changes nothing.  slot_of_dev has to be as it was then; a token that it names another slot for than u (v) does counts for neither.
 * Sums are taken in an order that follows from the sizes and the tokens' slots: equal calls give equal bits.  PP_ERR_SHAPE also: count < 1 or above 65535. */
pp_status_t pp_adapter_grad_weights(const pp_adapter_bank_t *bank, const void *x_dev, int32_t x_is_act8, const void *u_dev, const void *g_dev,
                                    const void *v_dev, const int32_t *slot_of_dev, const int32_t *which_dev, int32_t count, float *da_dev, float *db_dev,
                                    void *work_dev, int32_t n, void *hip_stream);

/* Free the bank.  NULL is a no-op returning PP_OK.  No call on the bank may still be executing. */
pp_status_t pp_adapter_destroy(pp_adapter_bank_t *bank);

#ifdef __cplusplus
}
#endif

#endif /* PP_ADAPTER_H */
