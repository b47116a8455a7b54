/*
 * dg4 - serving calls beside the layer: the historical K|V rows held in 8 bits with the attention that
 * reads them, and the projection of rows of many circuits, each with its own low-rank adapter.
 * The conventions of dg4.h hold; nothing here allocates but a dg4_graph's neighbour tables.
 */
#ifndef DG4_SERVING_H
#define DG4_SERVING_H

#include "dg4.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element format of a K|V store in 8 bits (dg4_kv8_write) */
typedef enum {
    DG4_KV_E4M3 = 0,        /* floating: 4 exponent and 3 mantissa bits, largest 448; relative  */
                            /* error of a value at most 2^-4 down to 2^-13 of its block's       */
                            /* largest magnitude, below that at most 2^-17 of the latter        */
                            /* (2^-137 where scales end)                                        */
    DG4_KV_INT8 = 1         /* whole numbers -127 .. 127; error at most 1/127 of the block's    */
                            /* largest magnitude (or 2^-128), four times less on average than   */
                            /* e4m3's                                                           */
} dg4_kv_format;

/*
 * The K|V store in 8 bits: the historical K and V rows (Section 3.4) at half the bytes of bfloat16, a
 * quarter of float. Store row u, n_store rows, both arrays device memory of the caller:
 *   codes  uint8 [n_store, 2*hidden]     K of all heads | V of all heads, in the element format
 *   scales uint8 [n_store, heads, 2]     for K and V of each head a power of two, as exponent + 127
 * A value is code * 2^(scale - 127). Writing quantises by blocks of one head (32 features): the scale
 * is the smallest power of two with which the block's largest magnitude stays within the format's
 * largest code (448 or 127; not below 2^-127), a value divided by it is rounded to the nearest code,
 * ties to even. Nothing else is rounded. A block that holds an infinity or a NaN gets scale 255 and
 * reads as NaN.
 *   dg4_kv8_write: rows [row_begin, row_end) of K and V [*, hidden] (cfg->dtype) into the store; row r
 *   goes to store row ids[r], or to row r without ids (then row_end <= n_store). Entries of ids outside
 *   [0, n_store) are skipped (-1: a padded row). The others are to be distinct: a store row that is named
 *   twice holds parts of both rows afterwards, codes of one under scales of the other among them, and
 *   has to be written again. Store rows that are not named stay as they are.
 */
int dg4_kv8_write(const dg4_layer_cfg* cfg, int32_t format, const void* K, const void* V,
                  int64_t row_begin, int64_t row_end, const int32_t* ids /* nullable, device */,
                  uint8_t* codes, uint8_t* scales, int64_t n_store, void* stream);

/*
 * Rows [row_begin, row_end) of K and V [*, hidden] from the store: row r is store row ids[r] (any
 * number of times the same), or row r without ids. Rows whose id is outside [0, n_store) stay as they
 * are. K and V may not overlap (EINVAL). Exact in float and bfloat16 (a code has at most 8 significant
 * bits) as far as the type reaches.
 */
int dg4_kv8_read(const dg4_layer_cfg* cfg, int32_t format, const uint8_t* codes, const uint8_t* scales,
                 int64_t n_store, const int32_t* ids /* nullable, device */,
                 int64_t row_begin, int64_t row_end, void* K, void* V, void* stream);

/*
 * dg4_sparse_attn_fwd over a store in 8 bits (graph's n_nodes rows, row = node id; the gate's own row
 * among them): rows [row_begin, row_end) of Q and A, row r the gate ids[r] (rows with an id outside
 * [0, n_nodes) stay as they are), or gate r without ids (then row_end <= n_nodes). Scores, softmax and
 * sums in fp32, one rounding to cfg->dtype. rel_bias = -infinity leaves a head's sources of that
 * relation out: what the store holds for them is not looked at, and a head whose sources are all left
 * out gives zeros. A may be Q itself, but not overlap it otherwise (EINVAL). The result of a row does
 * not depend on which rows a call covers. The graph's neighbour tables must be on the current device
 * (EINVAL otherwise).
 */
int dg4_sparse_attn_kv8_fwd(const dg4_layer_cfg* cfg, int32_t format, dg4_graph* g,
                            int64_t row_begin, int64_t row_end, const int32_t* ids /* nullable, device */,
                            const void* Q, const uint8_t* codes, const uint8_t* scales,
                            const float* rel_bias, void* A, void* stream);

/*
 * The projection (dg4_qkv_proj) with low-rank adapters beside it, for rows of many circuits at once:
 *   [Q | K | V][r] = S[r] Wqkv + gain[a] (S[r] Down_a) Up_a,  a = adapter[r]
 * Down_a [hidden, rank], Up_a [rank, 3*hidden], rank 1..DG4_MAX_RANK (adapters of smaller rank are
 * padded with zeros). dg4_lora_pack lays the weights out once in matrix-core operand order:
 *   Wqkv as in dg4_qkv_proj; Down [n_adapters, hidden, rank], Up [n_adapters, rank, 3*hidden] device,
 *   row-major, cfg->dtype; gain device float [n_adapters], null: 1 for all. n_adapters = 0 is allowed
 *   (rank, Down, Up, gain are not looked at then). packed: dg4_lora_packed_bytes, 256-byte aligned
 *   (EWORKSPACE otherwise). cfg: hidden, heads, dtype are used.
 * dg4_qkv_proj_lora reads `packed` as a dg4_lora_pack of the same cfg, n_adapters and rank left it (any
 * number of calls and streams at once may share it) for rows [row_begin, row_end) of S; adapter: device
 * int32, one of every row of S, in any order (runs of equal ones cost least); a row whose adapter is
 * outside [0, n_adapters), or any row where adapter is null, gets S[r] Wqkv alone. Q, K, V as in
 * dg4_qkv_proj; S, Q, K and V may not overlap (EINVAL). fp32 accumulation, one rounding to cfg->dtype
 * at the end (S Down is carried in at least 16 significant bits in bfloat16). A row's result depends on
 * nothing but the row, its adapter and Wqkv. Allocates nothing, one launch.
 */
#define DG4_MAX_RANK 64
int64_t dg4_lora_packed_bytes(const dg4_layer_cfg* cfg, int32_t n_adapters, int32_t rank);
int dg4_lora_pack(const dg4_layer_cfg* cfg, const void* Wqkv, int32_t n_adapters, int32_t rank,
                  const void* Down, const void* Up, const float* gain /* nullable */,
                  void* packed, int64_t packed_bytes, void* stream);
int dg4_qkv_proj_lora(const dg4_layer_cfg* cfg, const void* packed, int64_t packed_bytes,
                      int32_t n_adapters, int32_t rank, const void* S, int64_t row_begin, int64_t row_end,
                      const int32_t* adapter /* nullable */, void* Q, void* K, void* V, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DG4_SERVING_H */
