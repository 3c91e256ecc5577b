/*
 * fbx_train.h — C ABI of the trainer's operators in libfbx.so.
 *
 * Extraction (fbx.h) ends with slots of 64-bit signs in device memory; the next stage of the
 * paper's pipeline trains a model on them (Section 2.1: a sparse input of wide ids, an embedding
 * layer, a dense network).  These are the operators such a trainer runs first, in the middle and
 * last: rows of a table pooled per record, with the table's gradient; a gated feed-forward block,
 * with its gradient; an AdamW step over many tensors at once.
 *
 * Conventions, beside those of fbx.h
 *   - "HOST" / "DEVICE" on a pointer says which memory it must point to.  HOST arrays and structs are
 *     read before the call returns; DEVICE memory is the caller's and must stay until the work that
 *     was enqueued on hip_stream is done.
 *   - Calls only enqueue work on hip_stream (a hipStream_t, 0 = default stream): no wait, no device
 *     allocation, no copy to the host, so they can be captured into a graph.
 *   - Scratch is the caller's: 256-byte aligned, of the size the *_scratch function gives, unspecified
 *     afterwards.  A size of 0 means that NULL is fine.
 *   - Strides ("ld", "stride") are in elements, from one row to the next; elements of a row are adjacent.
 *   - Outputs may not overlap inputs or each other.
 *   - Sums are held in 32-bit floating point and rounded once, to nearest, where a result is stored.
 *     Results do not depend on the order in which workgroups run: the same inputs give the same bits.
 *   - On an error nothing is enqueued (FBX_E_HIP: unspecified).  fbx_train_last_error says why.
 */
#ifndef FBX_TRAIN_H
#define FBX_TRAIN_H

#include "fbx.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { FBX_F32 = 0, FBX_F16 = 1, FBX_BF16 = 2 } fbx_dtype;

/* Why the last call of this thread to a function of this header failed. */
const char* fbx_train_last_error(void);

/*
 * fbx_embed_forward — rows of a table, pooled per (record, slot).
 *
 *   row(sign)     = floor(mix64(sign) * rows / 2^64)      (mix64: the mixer of the extraction path; it is
 *                   applied because neither end of an FNV sign's bits is mixed well enough by itself)
 *   out[r][s][:]  = sum over the signs of slot s in record r of table[row(sign)][:], or their mean;
 *                   zeros for a record without signs in that slot
 *
 *   slots      : HOST, n_slots entries: fbx_result.slots, or entries made by the caller (slot_id is ignored;
 *                n_values must be fixed_arity * n_records for fixed arity, at least offsets[n_records] for lists.
 *                A list slot's values before offsets[0] or from offsets[n_records] on belong to no record and are
 *                left out: offsets + k of a slot of more records are the offsets of the records from k on)
 *   arrival_tile_records : fbx_result.arrival_tile_records, 0 for slots in record order
 *   d_table    : DEVICE, rows x dim, table_stride elements from row to row
 *   d_out      : DEVICE, n_records x (n_slots * dim), record_stride elements from record to record
 * Signs of a record are added in their order.  Limits: rows < 2^31, 1 <= dim <= 65536, n_records < 2^32, fewer than 2^32
 * signs a slot.
 * Errors: FBX_E_ARG, FBX_E_HIP.
 */
fbx_status fbx_embed_forward(const fbx_slot_view* slots, uint32_t n_slots, uint64_t n_records,
                             uint32_t arrival_tile_records, const void* d_table, uint64_t rows, uint32_t dim,
                             uint64_t table_stride, fbx_dtype dtype, int mean, void* d_out,
                             uint64_t record_stride, void* hip_stream);

/*
 * fbx_embed_backward — the gradient of fbx_embed_forward with respect to the table:
 *   dtable[v][:] = sum over all signs with row(sign) = v of w * dout[record][slot][:]
 * w = 1, or 1 / (signs of that record in that slot) where mean is set.  All of dtable is written,
 * zeros where no sign leads.  A row's terms are ordered by slot, record and position; stretches of them are
 * added up in that order, and then the stretches' sums in theirs.
 * Arguments as above.  Limits also: fewer than 2^32 values in all (those of no record count, for scratch and time
 * too), n_records * n_slots <= 2^32 - 256.
 * Errors: FBX_E_ARG, FBX_E_NOMEM (scratch too small), FBX_E_HIP.
 */
fbx_status fbx_embed_backward_scratch(const fbx_slot_view* slots, uint32_t n_slots, uint64_t n_records,
                                      uint64_t rows, uint32_t dim, int mean, uint64_t* bytes);
fbx_status fbx_embed_backward(const fbx_slot_view* slots, uint32_t n_slots, uint64_t n_records,
                              uint32_t arrival_tile_records, const void* d_dout, uint64_t record_stride,
                              uint64_t rows, uint32_t dim, uint64_t table_stride, fbx_dtype dtype, int mean,
                              void* d_dtable, void* d_scratch, uint64_t scratch_bytes, void* hip_stream);

/*
 * The gated feed-forward block: h = act(x Wg^T) * (x Wu^T), the two projections, the activation and the
 * product in one kernel.  x: records x inputs; Wg, Wu: hidden x inputs; h: records x hidden; all of
 * one type.  No value between x and h is rounded to fewer than 32 bits.
 *   act: silu a / (1 + e^-a); gelu a Phi(a), Phi by erf; relu max(a, 0), slope 0 at 0; sigmoid 1 / (1 + e^-a)
 * Limits: records < 2^31, 1 <= inputs, hidden <= 2^20, strides < 2^22; and so few tiles of 256 x 256 elements in each product
 * (records x 2 hidden; of the gradient also records x inputs and 2 hidden x inputs) that a launch holds them: below 2^23 - 4096.
 */
typedef enum { FBX_ACT_SILU = 0, FBX_ACT_GELU = 1, FBX_ACT_RELU = 2, FBX_ACT_SIGMOID = 3 } fbx_act;
typedef struct {
  uint64_t records;
  uint32_t inputs, hidden;
  fbx_dtype dtype;
  fbx_act act;
  const void* d_x;      /* DEVICE */
  const void* d_w_gate; /* DEVICE */
  const void* d_w_up;   /* DEVICE */
  uint64_t ld_x, ld_w_gate, ld_w_up;
} fbx_gated;

/* Scratch of fbx_gated_forward (backward = 0) or fbx_gated_backward (backward = 1) for these arguments. */
fbx_status fbx_gated_scratch(const fbx_gated* g, int backward, uint64_t* bytes);
/* Errors: FBX_E_ARG, FBX_E_NOMEM, FBX_E_HIP. */
fbx_status fbx_gated_forward(const fbx_gated* g, void* d_h, uint64_t ld_h, void* d_scratch,
                             uint64_t scratch_bytes, void* hip_stream);
/*
 * fbx_gated_backward — gradients with respect to x, Wg and Wu, given dh = d_dh:
 *   a = x Wg^T and u = x Wu^T are computed again;  da = dh * u * act'(a),  du = dh * act(a)
 *   dx = da Wg + du Wu,   dWg = da^T x,   dWu = du^T x
 * da and du are kept in the block's type between the products (rounded to nearest; in f16 a value
 * beyond its range becomes infinite there: scale the loss).  d_dx, or d_dw_gate and d_dw_up together, may
 * be NULL: not computed.
 */
fbx_status fbx_gated_backward(const fbx_gated* g, const void* d_dh, uint64_t ld_dh, void* d_dx,
                              uint64_t ld_dx, void* d_dw_gate, uint64_t ld_dw_gate, void* d_dw_up,
                              uint64_t ld_dw_up, void* d_scratch, uint64_t scratch_bytes, void* hip_stream);

/*
 * fbx_adamw_step — one step of AdamW (decoupled weight decay) over all tensors of a list, in place:
 *   g  = grad_scale * grad
 *   m  = beta1 m + (1 - beta1) g            v = beta2 v + (1 - beta2) g^2
 *   p  = p (1 - lr weight_decay) - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * in 32-bit arithmetic without contraction; p rounded to its type.
 *
 * state_bits = 32: m and v are arrays of floats.
 * state_bits = 8:  m and v are arrays of bytes: e4m3 codes (4 bits of exponent, 3 of mantissa, no infinity) of m
 *   and of sqrt(v), and one byte e8m0 (the power of two 2^(b - 127), 255 = NaN) per 32 elements that scales them
 *   and puts the block's largest magnitude into [128, 256).  After the step codes are rounded at random, up with
 *   the probability of the rest cut off, so that averages over many steps do not stick: element i of
 *   tensor t takes 16 bits (m: from bit 0, sqrt(v): from bit 16; 32 higher for odd i) of
 *   mix64(mix64(mix64(seed + step) + t) + i / 2).  A value that is not finite makes its block NaN.
 *   All zero bytes are the state before the first step.
 *   m and sqrt(v) are rounded independently of each other, so sqrt(v) can become 0 beside an m that does not; a gradient of 0
 *   then moves that weight by lr * m / eps, thousands of times lr.  With FBX_ADAMW_KEEP_ROOTS a sqrt(v) above 0
 *   that would be coded as 0 is coded as 1, the smallest code above it, and nothing else changes.
 * state_bits = 8 | FBX_ADAMW_KEEP_ROOTS: what a training run is to use, from its first step on.
 *
 *   tensors    : HOST, n_tensors entries; elements of a tensor are adjacent; at most FBX_ADAMW_MOST of them in one
 *   copy       : DEVICE or NULL: receives the new weights in copy_dtype as well (for weights kept in f32)
 * Errors: FBX_E_ARG, FBX_E_HIP.
 */
#define FBX_ADAMW_KEEP_ROOTS 0x100u
#define FBX_ADAMW_MOST 34359736320ull /* 2^35 - 2048 */
typedef struct {
  void* d_param;
  const void* d_grad;
  void* d_m;
  void* d_v;
  uint8_t* d_m_scale; /* state_bits = 8: ceil(n / 32) bytes */
  uint8_t* d_v_scale;
  void* d_copy;
  uint64_t n;
} fbx_adamw_tensor;
typedef struct {
  fbx_dtype param_dtype, grad_dtype, copy_dtype;
  uint32_t state_bits;
  uint64_t step; /* 1 for the first */
  double lr, beta1, beta2, eps, weight_decay, grad_scale;
  uint64_t seed;
} fbx_adamw;
fbx_status fbx_adamw_step(const fbx_adamw* h, const fbx_adamw_tensor* tensors, uint32_t n_tensors,
                          void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* FBX_TRAIN_H */
