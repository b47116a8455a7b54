/*
 * dg4 - serving calls in 4 bits, beside those of dg4_serving.h: the historical K|V rows in microscaled
 * 4-bit floating point with the attention that reads them, and projection and feed-forward sub-block with
 * rows and weights in it. The conventions of dg4.h hold; nothing here allocates but a dg4_graph's neighbour
 * tables.
 */
#ifndef DG4_MX4_H
#define DG4_MX4_H

#include "dg4.h"
#include "dg4_serving.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Blocks in microscaled 4-bit floating point, of the calls below: 32 numbers, each 1 sign, 2 exponent and
 * 1 mantissa bits (codes 0 .. 7: 0, 0.5, 1, 1.5, 2, 3, 4, 6; code + 8: the same, negative), and one scale
 * byte b for the power of two 2^(b - 127) that multiplies them. A block is quantised with the smallest
 * power of two (not below 2^-127) with which its largest magnitude is at most 7 times it; a value divided
 * by it goes to the nearest code, ties to even, from 6 on to 6. Nothing else is rounded. The error of a
 * value is at most a fifth of it, or a fourteenth of the block's largest magnitude where that is more (or
 * 2^-129); over a block of normal numbers it is a ninth in the 2-norm. A block that holds an infinity or
 * a NaN gets byte 255 and stands for NaN. Magnitudes above 1.75 * 2^127, an eighth below float's largest, go to
 * 4 * 2^126 = 2^128, which the products take as it is and float and bfloat16 read as an infinity.
 *
 * The K|V store in 4 bits: the historical K and V rows (Section 3.4) in 272 bytes where hidden is 256, a
 * quarter of bfloat16's. A head (32 features) of K or V is a block. Store row u, n_store rows, device memory of
 * the caller:
 *   codes  uint8 [n_store, hidden]       K of all heads | V of all heads, two codes to a byte, the first
 *                                        in the low half
 *   scales uint8 [n_store, heads, 2]     for K and V of each head
 * dg4_kv4_write, dg4_kv4_read and dg4_sparse_attn_kv4_fwd are dg4_kv8_write, dg4_kv8_read and
 * dg4_sparse_attn_kv8_fwd on such a store, without the format: what stands there of ids, ranges, rows
 * that are named twice, overlaps, masks and rounding holds here. Values read back are exact in float and
 * bfloat16 as far as the type reaches.
 */
int dg4_kv4_write(const dg4_layer_cfg* cfg, const void* K, const void* V,
                  int64_t row_begin, int64_t row_end, const int32_t* ids /* nullable, device */,
                  uint8_t* codes, uint8_t* scales, int64_t n_store, void* stream);
int dg4_kv4_read(const dg4_layer_cfg* cfg, const uint8_t* codes, const uint8_t* scales,
                 int64_t n_store, const int32_t* ids /* nullable, device */,
                 int64_t row_begin, int64_t row_end, void* K, void* V, void* stream);
int dg4_sparse_attn_kv4_fwd(const dg4_layer_cfg* cfg, dg4_graph* g,
                            int64_t row_begin, int64_t row_end, const int32_t* ids /* nullable, device */,
                            const void* Q, const uint8_t* codes, const uint8_t* scales,
                            const float* rel_bias, void* A, void* stream);

/*
 * Products of rows and weights that are both in such blocks, q(.) below; blocks run along the summed axis.
 * dg4_mx4_pack lays a weight matrix W [k, n] (device, row-major, cfg->dtype) out once in matrix-core
 * operand order, 17/32 of a byte an element; (k, n) is (hidden, 3*hidden) for Wqkv, (hidden, 4*hidden)
 * for W1 or (4*hidden, hidden) for W2 of cfg (EUNSUPPORTED otherwise). packed: dg4_mx4_packed_bytes,
 * 256-byte aligned (EWORKSPACE otherwise). The calls below read it as a dg4_mx4_pack of the same cfg and of
 * the matrix that they ask for left it; any number of calls and streams at once may share it. They allocate nothing, one
 * launch, no workspace. Sums are in fp32, with one rounding at the end: to cfg->dtype, or to the store's
 * codes. A row's result depends on nothing but the row and the weights. A block of a row or of W that is
 * not finite makes what it is summed into NaN. cfg: hidden, heads, dtype (dg4_ffn_mx4_fwd: ln_eps) are used.
 *   dg4_qkv_proj_mx4: [Q | K | V][r] = q(S[r]) q(Wqkv) for rows [row_begin, row_end), as dg4_qkv_proj.
 *   S, Q, K and V may not overlap (EINVAL).
 *   dg4_qkv_proj_kv4: the same, with Q to rows and K and V into the store in 4 bits: row r goes to store
 *   row ids[r], or to row r without ids, as in dg4_kv4_write. (Every row of Q is written, also those whose
 *   id names no store row.) The store holds the sums themselves, rounded once. S and Q may not overlap.
 *   dg4_ffn_mx4_fwd: Out[r] = LayerNorm(S[r] + q(max(q(S[r]) q(W1), 0)) q(W2)) for rows [row_begin,
 *   row_end), as dg4_ffn_fwd; S as it is in the first sum. S and Out may not overlap (EINVAL).
 */
int64_t dg4_mx4_packed_bytes(const dg4_layer_cfg* cfg, int32_t k, int32_t n);
int dg4_mx4_pack(const dg4_layer_cfg* cfg, const void* W, int32_t k, int32_t n,
                 void* packed, int64_t packed_bytes, void* stream);
int dg4_qkv_proj_mx4(const dg4_layer_cfg* cfg, const void* packed, int64_t packed_bytes,
                     const void* S, int64_t row_begin, int64_t row_end, void* Q, void* K, void* V, void* stream);
int dg4_qkv_proj_kv4(const dg4_layer_cfg* cfg, const void* packed, int64_t packed_bytes,
                     const void* S, int64_t row_begin, int64_t row_end, const int32_t* ids /* nullable, device */,
                     void* Q, uint8_t* codes, uint8_t* scales, int64_t n_store, void* stream);
int dg4_ffn_mx4_fwd(const dg4_layer_cfg* cfg, const void* packed_W1, int64_t packed_W1_bytes,
                    const void* packed_W2, int64_t packed_W2_bytes,
                    const void* S, int64_t row_begin, int64_t row_end, void* Out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DG4_MX4_H */
