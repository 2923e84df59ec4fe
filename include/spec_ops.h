/*
 * spec_ops.h - single-kernel entry points of the verify step, for checking
 * each kernel on its own at full workload sizes, and operators beside it (page
 * copies; a 4-bit cache, which no context holds) for callers that run them one
 * by one.  Same conventions as spec.h:
 * "device" pointers are HIP device addresses, "host" pointers CPU memory,
 * stream is a hipStream_t as void*, errors are spec_status codes and the
 * caller owns every buffer.
 */
#ifndef SPEC_OPS_H_
#define SPEC_OPS_H_

#include "spec.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { SPEC_EPI_STORE_F32 = 0, SPEC_EPI_ADD_F32 = 1, SPEC_EPI_SWIGLU = 2 };

/* One bf16 weight [rows, K] (device) from row-major to the tiled layout, in
 * place (the per-matrix step of spec_pack_model; K % 128 == 0, else
 * SPEC_E_UNSUPPORTED).  rot_rows > 0 marks the first rot_rows rows as rotary
 * heads of head_dim rows (head_dim % 16 == 0, rot_rows % head_dim == 0),
 * reordered as wqkv's q and k heads are.  Asynchronous. */
SPEC_API spec_status spec_pack_weight(void* w, int32_t rows, int32_t K, int32_t rot_rows,
                                      int32_t head_dim, void* stream);

/* Decoder projection Y = X W^T (the QKV, O, gate/up, down and LM-head
 * products of the Llama layer).  X device [R, K] row-major, W device [N, K]
 * (SwiGLU: [2N, K], gate rows then up rows), element type dtype; fp32
 * accumulation.  fp32 W is row-major; bf16 W is in the tiled layout
 * (spec_pack_weight; for SwiGLU the gate and up halves packed separately).
 *   SPEC_EPI_STORE_F32: Y fp32 [R, N] = X W^T
 *   SPEC_EPI_ADD_F32:   Y fp32 [R, N] += X W^T   (residual add)
 *   SPEC_EPI_SWIGLU:    Y dtype [R, N] = silu(X Wg^T) * (X Wu^T)
 * bf16 needs K % 128 == 0 (else SPEC_E_UNSUPPORTED).  workspace (device,
 * optional, NULL allowed): fp32 split-K partials for R > 64 when the output
 * grid is small; size it with spec_op_gemm_workspace_bytes(R, N_w). */
SPEC_API size_t spec_op_gemm_workspace_bytes(int32_t R, int32_t Nw);
SPEC_API spec_status spec_op_gemm(int32_t dtype, int32_t R, int32_t N, int32_t K, const void* X,
                                  const void* W, void* Y, int32_t epilogue, void* workspace,
                                  size_t workspace_bytes, void* stream);

/* RMSNorm: y[r] (dtype) = h[r] / sqrt(mean(h[r]^2) + eps) * w, h fp32 [R, d]. */
SPEC_API spec_status spec_op_rmsnorm(int32_t dtype, int32_t R, int32_t d, const float* h,
                                     const void* w, float eps, void* y, void* stream);

/* Rotary embedding + paged KV append for one layer.  qkv device fp32
 * [R, (Hq + 2 Hkv) hd]; pos and slot device int32 [R] (slot = page * 16 + offset);
 * q_out device [R, Hq, hd]; k_pages [pages][Hkv][16][hd]; v_pages [pages][Hkv][hd][16].
 * head_dim even and at most 256 (SPEC_E_INVALID otherwise). */
SPEC_API spec_status spec_op_rope_kv(int32_t dtype, int32_t R, int32_t n_heads, int32_t n_kv_heads,
                                     int32_t head_dim, float theta, const float* qkv,
                                     const int32_t* pos, const int32_t* slot, void* q_out,
                                     void* k_pages, void* v_pages, void* stream);

/* Paged causal attention of n_seqs row groups: group i has rows[i] query rows
 * (packed in order in q, device [sum rows, Hq, hd]) at positions pos0[i]..,
 * attending keys 0..position through page table row i of page_table (host
 * int32 [n_seqs, max_pages]).  out device [sum rows, Hq * hd], dtype.
 * workspace: device, >= spec_op_attention_workspace_bytes(...). */
SPEC_API size_t spec_op_attention_workspace_bytes(int32_t n_seqs, int32_t total_rows,
                                                  int32_t max_pages, int32_t n_kv_heads,
                                                  int32_t head_dim);
SPEC_API spec_status spec_op_attention(int32_t dtype, int32_t n_seqs, const int32_t* rows,
                                       const int32_t* pos0, const int32_t* page_table,
                                       int32_t max_pages, int32_t n_heads, int32_t n_kv_heads,
                                       int32_t head_dim, const void* q, const void* k_pages,
                                       const void* v_pages, void* out, void* workspace,
                                       size_t workspace_bytes, void* stream);

/* Copies of cache pages in every plane of a pool: page dst_pages[i] of each of
 * the n_planes planes <- page src_pages[i] of that plane (host int32 [n]).
 * pool: device, 16-byte aligned, [n_planes][num_pages][page_bytes] (a context's
 * pool is one: K and V pages of every layer; page_bytes % 16 == 0, whatever the
 * pages hold).  One source may have several copies; a page that is a
 * destination twice, or a destination and a source, is refused
 * (SPEC_E_INVALID), as is one outside the pool.  workspace: device, 16-byte
 * aligned, >= spec_op_kv_copy_pages_workspace_bytes(n), not shared by calls that
 * overlap in time.  A captured call takes at most 384 pairs
 * (SPEC_E_UNSUPPORTED beyond).  Asynchronous; host arrays are consumed before
 * return (more pairs are staged as the larger tables of spec_op_attention_kv4). */
SPEC_API size_t spec_op_kv_copy_pages_workspace_bytes(int32_t n);
SPEC_API spec_status spec_op_kv_copy_pages(int32_t n_planes, int32_t num_pages, size_t page_bytes, void* pool,
                                           int32_t n, const int32_t* src_pages, const int32_t* dst_pages,
                                           void* workspace, size_t workspace_bytes, void* stream);

/* The KV cache in 4 bits, for one layer: 17/64 of the bytes of a bf16 cache.
 * k_pages and v_pages (device, 16-byte aligned): [num_pages][Hkv] blocks of 16
 * tokens x hd dims, spec_kv4_page_bytes(Hkv, hd) bytes a page, hd 64 or 128 (0
 * bytes, and SPEC_E_UNSUPPORTED from the calls, for another).  A token's head
 * vector is held in blocks of 32 consecutive dims: a scale 2^E, E the smallest
 * integer >= -126 with max |x| <= 6 2^E, and for every x the nearest of 0, 0.5,
 * 1, 1.5, 2, 3, 4, 6 times 2^E with its sign (ties to the one of even code 0, 2,
 * 4, 6 in that order).  A block with an infinity or a NaN reads back as NaN.
 * Every value held is a bf16 number, but for magnitudes from 1.75 2^127 on, which
 * are held as 2^128 and read back as infinities.  The library alone writes the
 * pages (kv4_layout.h has the byte order). */
SPEC_API size_t spec_kv4_page_bytes(int32_t n_kv_heads, int32_t head_dim);

/* spec_op_rope_kv into a 4-bit cache: q_out <- the rotated q (dtype), the
 * rotated k and the v of row r into slot[r].  A row with a slot outside 0 ..
 * 16 num_pages - 1 (padding: -1) has its q written and no K / V.  Two rows of
 * one call must not have one slot.  qkv and q_out 16-byte aligned. */
SPEC_API spec_status spec_op_rope_kv4(int32_t dtype, int32_t R, int32_t n_heads, int32_t n_kv_heads,
                                      int32_t head_dim, float theta, const float* qkv, const int32_t* pos,
                                      const int32_t* slot, int32_t num_pages, void* q_out, void* k_pages,
                                      void* v_pages, void* stream);

/* The values held in the slots of a 4-bit cache: k_out, v_out (device, dtype,
 * [R, Hkv, hd], 16-byte aligned) row r <- slot[r] (device int32); rows with a
 * slot outside the pool are left as they were. */
SPEC_API spec_status spec_op_kv4_read(int32_t dtype, int32_t R, int32_t n_kv_heads, int32_t head_dim,
                                      const int32_t* slot, int32_t num_pages, const void* k_pages,
                                      const void* v_pages, void* k_out, void* v_out, void* stream);

/* spec_op_attention over a 4-bit cache, of at most 2^30 positions a sequence and
 * 65535 heads (SPEC_E_INVALID beyond; 65535 in the other 4-bit calls too).
 * rows[i] may be 0 (a sequence without rows in this call).  num_pages: pages of
 * the pool; a page id outside it is refused (SPEC_E_INVALID).  q, out: dtype,
 * 16-byte aligned.  n_heads / n_kv_heads <= 64 (bf16) or 32 (fp32), else
 * SPEC_E_UNSUPPORTED.  Scores and sums are fp32; the probabilities' product with
 * V takes them to 24 bits in fp32, and rounded to bf16's 8 in bf16, as
 * spec_op_attention does.  A NaN or an infinity in the cache reaches the rows
 * that see its key only.
 * workspace: device, 256-byte aligned, >= spec_op_attention_kv4_workspace_bytes
 * of the same rows and positions (0 for arguments the call refuses), not shared
 * by calls that overlap in time.  A captured call takes tables of at most 3 KB
 * (SPEC_E_UNSUPPORTED beyond).  Asynchronous, host arrays are consumed before
 * return; but larger tables go through four staging buffers that the context-free
 * calls of a process share, and with four such calls in flight the host waits for
 * the oldest one's tables to be taken. */
SPEC_API size_t spec_op_attention_kv4_workspace_bytes(int32_t dtype, int32_t n_seqs, const int32_t* rows,
                                                      const int32_t* pos0, int32_t max_pages, int32_t n_heads,
                                                      int32_t n_kv_heads, int32_t head_dim);
SPEC_API spec_status spec_op_attention_kv4(int32_t dtype, int32_t n_seqs, const int32_t* rows,
                                           const int32_t* pos0, const int32_t* page_table, int32_t max_pages,
                                           int32_t num_pages, int32_t n_heads, int32_t n_kv_heads,
                                           int32_t head_dim, const void* q, const void* k_pages,
                                           const void* v_pages, void* out, void* workspace,
                                           size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SPEC_OPS_H_ */
