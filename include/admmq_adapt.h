/*
 * admmq_adapt.h -- running and adapting the layers that admmq.h quantizes (B200, sm_100a).
 *
 * A quantized layer holds W[j][i] = z0 + Delta k with one (Delta, z0) per output channel j and group of input
 * channels.  These calls multiply by W and by W^T straight from its codes, add the low-rank adapters of many requests
 * to the same rows, form the adapters' gradients, keep activations in 8 bits for the backward pass, and norm and
 * rotate the query and key heads that such a projection produces.
 *
 * Conventions shared by every call
 *  - d_* are DEVICE pointers; the caller owns every buffer, the library allocates nothing on the device.  The device
 *    that owns the pointers and the stream must be the calling thread's current device.  cuda_stream: a cudaStream_t
 *    (NULL = the default stream).  Every call is asynchronous, can be captured into a CUDA graph after a first call
 *    outside a capture, and neither throws, aborts nor traps.
 *  - Argument and shape errors are returned at once with nothing enqueued.  d_status: one device int the caller has
 *    zeroed; a kernel that meets an error raises it there (the first one stays).  Outputs are unspecified after that.
 *  - bf16 and fp32 pointers must be 16-byte aligned and row strides (ld*, in elements) keep every row so aligned,
 *    except where a call says otherwise.
 *  - Rows are tokens.  n_rows == 0 is a no-op (gradients that are sums over rows are set to zero).
 *  - Sums run in fp32.  Outputs may not overlap inputs unless a call says so.
 */
#ifndef ADMMQ_ADAPT_H_
#define ADMMQ_ADAPT_H_

#include "admmq.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ADMMQ_ADAPT_MAX_BITS 4
#define ADMMQ_ADAPT_MAX_RANK 128
#define ADMMQ_ADAPT_MAX_ROWS (1LL << 30)
#define ADMMQ_ADAPT_MAX_ADAPTERS 65535
#define ADMMQ_CHECKPOINT_BLOCK 128

/* ---- Packed layer ------------------------------------------------------------------------------------
 * d_codes: [d_out][d_in] uint8 in [0, 2^bits), d_scale / d_zero: [d_out][d_in/group] fp32, as
 * admmq_quantize_layer and admmq_local_search return them.  Limits: bits 2..4 (more: ADMMQ_ERR_UNSUPPORTED),
 * d_in and d_out multiples of 8, the group a multiple of 64 that divides d_in, or 0 / d_in (one group).
 * d_packed (admmq_packed_bytes) receives 4 bits a code in blocks of 64 input channels, d_grid (admmq_grid_bytes) the
 * pairs (Delta, z0) group by group.  A code of 2^bits or more raises ADMMQ_ERR_INVALID_ARG in d_status.  Done once;
 * both buffers describe the layer from then on. */
size_t admmq_packed_bytes(int d_in, int d_out);
size_t admmq_grid_bytes(int d_in, int d_out, int group_size);
admmq_status admmq_pack_layer(const unsigned char* d_codes, const float* d_scale, const float* d_zero, int d_in,
                              int d_out, int bits, int group_size, void* d_packed, void* d_grid, int* d_status,
                              void* cuda_stream);

typedef struct {
  size_t struct_size;     /* sizeof(admmq_packed_layer) */
  int d_in, d_out;
  int group_size;         /* as given to admmq_pack_layer */
  const void* d_packed;
  const void* d_grid;
} admmq_packed_layer;

/* ---- Adapters ----------------------------------------------------------------------------------------
 * A bank of n_adapters low-rank pairs for one layer, bf16, rank a multiple of 8 up to ADMMQ_ADAPT_MAX_RANK (an adapter
 * of a smaller rank is filled up with zero rows):
 *   d_down [n_adapters][rank][d_in], d_up [n_adapters][rank][d_out] (rank-major, like down), d_scale [n_adapters].
 * Adapter a adds scale_a up_a^T (down_a x) to the layer's output.  Entries must be finite: rows of different requests
 * share tensor-core tiles, where a non-finite entry of one adapter would reach its neighbours' rows.
 * admmq_adapters_check raises ADMMQ_ERR_NONFINITE in d_status if one is not; run it when a bank is loaded. */
typedef struct {
  size_t struct_size;     /* sizeof(admmq_adapters) */
  int n_adapters, rank;
  const void* d_down;
  const void* d_up;
  const float* d_scale;
} admmq_adapters;
admmq_status admmq_adapters_check(const admmq_adapters* bank, int d_in, int d_out, int* d_status, void* cuda_stream);

/* ---- The projection and its input gradient ------------------------------------------------------------
 * forward:    h_t = scale_a down_a x_t,   y_t  = W   x_t  + up_a^T   h_t      x [n_rows][ldx], y [n_rows][ldy]  bf16
 * grad_input: u_t = scale_a up_a   dy_t,  dx_t = W^T dy_t + down_a^T u_t      dy [n_rows][lddy], dx [n_rows][lddx] bf16
 * a = d_row_adapter[t]; a value outside [0, n_adapters) means none (h_t = u_t = 0).  bank NULL: no adapters, and
 * d_row_adapter and d_h / d_u are ignored.  d_h, d_u: [n_rows][rank] fp32, outputs (the backward pass reads them).
 * One launch without adapters, two with them, of which the second overlaps the first.
 * Roundings.  Up to 16 rows the forward call multiplies the codes themselves, and y carries the rounding of its 32-bit sum
 * to bf16 alone.  Above, and in grad_input always, the tensor cores take W (once z0 + Delta k is formed in fp32) and h or
 * u as bf16 operands; so a row's last bits may change when its batch passes 16 rows, and the W of the gradient is the
 * rounded one. */
admmq_status admmq_linear_forward(const admmq_packed_layer* layer, const admmq_adapters* bank, long long n_rows,
                                  const int* d_row_adapter, const void* d_x, long long ldx, void* d_y, long long ldy,
                                  float* d_h, int* d_status, void* cuda_stream);
admmq_status admmq_linear_grad_input(const admmq_packed_layer* layer, const admmq_adapters* bank, long long n_rows,
                                     const int* d_row_adapter, const void* d_dy, long long lddy, void* d_dx,
                                     long long lddx, float* d_u, int* d_status, void* cuda_stream);

/* ---- Adapter gradients --------------------------------------------------------------------------------
 * d_down_a = sum over the rows t of adapter a of u_t x_t^T,  d_up_a = sum of h_t dy_t^T   (bf16, the bank's layout),
 * in a fixed order of the rows.  rows of adapter a: d_order[d_offsets[a] .. d_offsets[a + 1]); d_order: row numbers
 * sorted by adapter, d_offsets: [n_adapters + 1].  A row number outside [0, n_rows) adds nothing, offsets are cut to
 * [0, n_rows].  An adapter without rows gets zeros.  The gradient of scale is not formed.
 * x is given either in bf16 (d_x, ldx) or as an 8-bit checkpoint (d_x_codes, d_x_scale; d_x NULL). */
typedef struct {
  size_t struct_size;     /* sizeof(admmq_adapter_grad_args) */
  int d_in, d_out, n_adapters, rank;
  long long n_rows;
  const int* d_order;
  const int* d_offsets;
  const float* d_h;       /* [n_rows][rank] */
  const float* d_u;       /* [n_rows][rank] */
  const void* d_x;
  long long ldx;
  const signed char* d_x_codes;   /* [n_rows][d_in] */
  const float* d_x_scale;         /* [n_rows][ceil(d_in / 128)] */
  const void* d_dy;
  long long lddy;
  void* d_grad_down;      /* [n_adapters][rank][d_in] */
  void* d_grad_up;        /* [n_adapters][rank][d_out] */
} admmq_adapter_grad_args;
admmq_status admmq_adapter_grad(const admmq_adapter_grad_args* args, void* cuda_stream);

/* ---- Activation checkpoints in 8 bits -------------------------------------------------------------------
 * save: for every row and block of ADMMQ_CHECKPOINT_BLOCK channels (the last may be shorter)
 *   scale = max |x| / 127,  code = round(x / scale) to nearest, ties to even, in [-127, 127]
 * (code 0 where scale is 0; a block that holds a non-finite value gets scale NaN and is restored as NaN).
 * x: [n_rows][ldx] fp32 or bf16, width a multiple of 8; codes [n_rows][width] int8, scale
 * [n_rows][ceil(width / 128)], at most 2^31 - 1 of them.  restore writes scale * code as out [n_rows][ldo] of the given type. */
admmq_status admmq_checkpoint_save(const void* d_x, admmq_dtype dtype, long long n_rows, int width, long long ldx,
                                   signed char* d_codes, float* d_scale, void* cuda_stream);
admmq_status admmq_checkpoint_restore(const signed char* d_codes, const float* d_scale, long long n_rows, int width,
                                      void* d_out, admmq_dtype dtype, long long ldo, void* cuda_stream);

/* ---- Per-head norm of queries and keys with the position rotation ---------------------------------------
 * For every head vector x of head_dim values at position pos:  n = x / sqrt(mean(x^2) + eps), z = w n, and for
 * i < rot_dim / 2:  y_i = z_i cos - z_{i + rot/2} sin,  y_{i + rot/2} = z_{i + rot/2} cos + z_i sin,  with cos and sin
 * at [pos][i]; the values from rot_dim on pass unrotated.  Queries and keys have a weight each.
 * A tensor [n_rows][heads][head_dim] is given by its row and head strides (elements; inner stride 1).  head_dim and
 * rot_dim: multiples of 16, rot_dim <= head_dim <= 256.  d_cos, d_sin: [n_positions][rot_dim / 2] fp32; a position
 * outside [0, n_positions) raises ADMMQ_ERR_SHAPE in d_status.  k_heads may be 0.  fp32 or bf16 throughout, the
 * arithmetic in fp32.  The forward call may work in place (out = in, same strides).
 * backward: dq, dk [n_rows][heads][head_dim] from dy of the same layouts, and the weights' gradients [head_dim], summed
 * over rows and heads in a fixed order; d_workspace: admmq_qk_workspace_bytes(head_dim) bytes. */
typedef struct {
  size_t struct_size;     /* sizeof(admmq_qk_args) */
  admmq_dtype dtype;
  int q_heads, k_heads, head_dim, rot_dim;
  long long n_rows;
  double eps;
  const void *d_q, *d_k;  /* inputs of the norm */
  long long q_row, q_head, k_row, k_head;
  const void *d_wq, *d_wk;
  const float *d_cos, *d_sin;
  long long n_positions;
  const int* d_pos;       /* [n_rows] */
  void *d_out_q, *d_out_k;              /* forward: y;  backward: gradients of q and k */
  long long out_q_row, out_q_head, out_k_row, out_k_head;
  const void *d_dy_q, *d_dy_k;          /* backward only */
  long long dy_q_row, dy_q_head, dy_k_row, dy_k_head;
  void *d_grad_wq, *d_grad_wk;          /* backward only: [head_dim], of dtype */
  void* d_workspace;                    /* backward only */
  size_t workspace_bytes;
  int* d_status;
} admmq_qk_args;
size_t admmq_qk_workspace_bytes(int head_dim);
admmq_status admmq_qk_norm_rope(const admmq_qk_args* args, void* cuda_stream);
admmq_status admmq_qk_norm_rope_backward(const admmq_qk_args* args, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* ADMMQ_ADAPT_H_ */
