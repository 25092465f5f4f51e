/*
 * vpp_block_attn.h -- attention of a chunk's tokens to selected blocks of a paged KV cache.
 *
 * Beside the dense attention of vpp_chunk_attn.h, whose cost grows with the prefix: the
 * cached keys of a request are cut into blocks of block_size, a cheap score selects a
 * list of blocks for each query block (query_block consecutive tokens of one segment) and
 * kv head, and the tokens attend to the keys of their listed blocks alone. Per layer
 * and chunk, with the chunk's keys and values in the cache:
 *
 *   vpp_block_summarize_paged   one vector for each block of keys that the chunk completed
 *   vpp_block_select_paged      the lists
 *   vpp_block_attn_run_paged    the attention
 *
 * Positions, segments, causality, page layout, strides, alignment and status codes are
 * those of vpp_chunk_attn_run_paged; the stride of a dimension of size 1 is not used. All
 * calls but the host helpers are asynchronous on `stream` (a hipStream_t of the current
 * device; NULL is the default stream), allocate nothing, keep nothing between calls and
 * may be captured. Page indices, block indices and query blocks come from device memory:
 * values out of range are clamped or skipped there, so they give wrong or no results, never
 * an access outside the buffers described by the arguments.
 */
#ifndef VPP_BLOCK_ATTN_H
#define VPP_BLOCK_ATTN_H

#include "vpp_chunk_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Heads, blocks and lists, passed by pointer (copied). */
typedef struct {
    int32_t num_q_heads;   /* Hq > 0                                                     */
    int32_t num_kv_heads;  /* Hkv > 0, Hq % Hkv == 0, Hq / Hkv <= 128                    */
    int32_t head_dim_qk;   /* dqk                                                        */
    int32_t head_dim_v;    /* dv; (dqk, dv) in {(64,64), (128,128), (192,128)}           */
    float softmax_scale;   /* 0 => 1/sqrt(dqk)                                           */
    int32_t block_size;    /* keys of a block: 64, 128 or 256, at most a page            */
    int32_t query_block;   /* tokens of a query block, 1 .. 128                          */
    int32_t max_blocks;    /* length of a list, 1 .. 2048, at least sink_blocks +
                              local_blocks + ceil((query_block - 1) / block_size)        */
    int32_t sink_blocks;   /* first blocks of a request that are on every list, >= 0     */
    int32_t local_blocks;  /* last blocks up to that of a query block's first token that
                              are on its list, >= 1                                      */
} vpp_block_attn_config_t;

/* A query block: rows row0 .. row0 + rows - 1 of the chunk, of one segment; their first
 * token's position; the cache row of the request's position 0 (kv_start). */
typedef struct {
    int32_t row0, rows, segment, pos0, kv_start, reserved[3];
} vpp_query_block_t;

/*
 * Host helper: the query blocks of a chunk (segment metadata as for vpp_chunk_attn_plan;
 * kv_start[s] a multiple of block_size), in row order, each segment cut from its first row
 * on. *count receives their number; at most `capacity` are written (blocks may be NULL
 * with capacity 0). Copy them to the device for the calls below. Errors:
 * VPP_ERR_INVALID_ARG for malformed metadata or cache rows past 2^31 - 1.
 */
vpp_status_t vpp_query_blocks(int32_t num_segments, const int32_t* cu_q, const int64_t* kv_start,
                              const int64_t* prefix_len, int32_t query_block, int32_t block_size,
                              vpp_query_block_t* blocks, int32_t capacity, int32_t* count);

/*
 * Host helper: the blocks that a chunk completes, those with at least one of the chunk's
 * rows whose last row is cached with it, as indices page * (page_size / block_size) + block
 * of the page. Metadata and block table as for vpp_paged_slot_mapping, kv_start[s] a
 * multiple of block_size. *count and capacity as above. Errors: VPP_ERR_INVALID_ARG.
 */
vpp_status_t vpp_completed_blocks(int32_t num_segments, const int32_t* cu_q, const int64_t* kv_start,
                                  const int64_t* prefix_len, const int32_t* block_table,
                                  int64_t block_table_stride, int32_t pages_per_row, int32_t page_size,
                                  int32_t block_size, int64_t* blocks, int32_t capacity, int32_t* count);

/*
 * The summary of each listed block (device array of num_blocks indices as above; those
 * outside the cache are skipped): per kv head the mean of the block's keys, summed in 64 bits,
 * on the grid of its dqk values: multiples of 2^(e-8), where 2^e is the power of two above
 * the largest magnitude (at least 2^-54), rounded to nearest even. Values count at most
 * 2^60 in magnitude, a mean that is NaN counts as 0. That is 8 bits a value, exact in bf16.
 * Written to summaries, bf16 [num_pages][page_size / block_size][Hkv][dqk], contiguous,
 * 16-byte aligned; the others stay as they are. A block listed twice is written twice with
 * the same values. Errors: VPP_ERR_INVALID_ARG, VPP_ERR_UNSUPPORTED, VPP_ERR_HIP.
 */
vpp_status_t vpp_block_summarize_paged(const vpp_block_attn_config_t* cfg,
                                       const void* k_pages, int64_t k_stride_page, int64_t k_stride_tok,
                                       int64_t k_stride_head, int32_t page_size, int32_t num_pages,
                                       const int64_t* blocks, int32_t num_blocks, void* summaries, void* stream);

/*
 * Bytes of device workspace that vpp_block_select_paged needs (0: none): the scores of a slab of
 * the query blocks, at most 256 MiB or those of 64 of them. Errors: VPP_ERR_INVALID_ARG,
 * VPP_ERR_UNSUPPORTED (head dims; more than 32768 blocks up to max_kv_len).
 */
vpp_status_t vpp_block_select_workspace(const vpp_block_attn_config_t* cfg, int32_t num_query_blocks,
                                        int64_t max_kv_len, size_t* bytes);

/*
 * The lists: blocks[i][kv head][0 .. max_blocks - 1] (int32, contiguous) of query block i.
 * Of blocks 0 .. c, c that of the query block's last token, with f that of its first:
 *   - always on the list: b < sink_blocks, and b > f - local_blocks;
 *   - of the others, those with the largest scores, the lowest ones of equal scores.
 * The score of a block is the largest product of its summary with a query row of the kv
 * head's group and of the query block's tokens, the row taken on the grid of its values as a
 * summary is (NaN counts as 0). Products of such vectors are multiples of one step below
 * 2^24 steps: fp32 sums of them are exact, so lists do not depend on how they are computed.
 * Lists ascend; unused places at the end are -1 (fewer than max_blocks blocks up to c).
 * query_blocks: device array; q as for the attention; summaries as above (those of blocks
 * without a written summary are read as they are; only complete blocks before f are
 * read). max_kv_len: an upper bound on kv positions of the chunk (its longest prefix + len);
 * blocks past it are not seen. block_table [num_segments][pages_per_row]. workspace:
 * 256-byte aligned, may be NULL if the size is 0; not to be used by other work in flight.
 * Errors: VPP_ERR_INVALID_ARG; VPP_ERR_UNSUPPORTED (head dims; more than 32768 blocks up
 * to max_kv_len); VPP_ERR_WORKSPACE; VPP_ERR_HIP.
 */
vpp_status_t vpp_block_select_paged(const vpp_block_attn_config_t* cfg,
                                    const vpp_query_block_t* query_blocks, int32_t num_query_blocks,
                                    const void* q, int64_t q_stride_tok, int64_t q_stride_head, int32_t num_tokens,
                                    const void* summaries, int32_t page_size, int32_t num_pages,
                                    const int32_t* block_table, int64_t block_table_stride, int32_t num_segments,
                                    int32_t pages_per_row, int64_t max_kv_len, int32_t* blocks,
                                    void* workspace, size_t workspace_bytes, void* stream);

/*
 * Bytes of device workspace that vpp_block_attn_run_paged needs for a chunk of num_tokens
 * tokens in num_query_blocks query blocks (0: none; partial results where few query
 * blocks have their lists split over several workgroups).
 */
vpp_status_t vpp_block_attn_workspace(const vpp_block_attn_config_t* cfg, int32_t num_query_blocks,
                                      int32_t num_tokens, size_t* bytes);

/*
 * Attention of each query block's tokens to the keys of its listed blocks: a token at
 * position i sees the keys j <= i of the blocks blocks[query block][kv head][*]. Entries that
 * are negative or past the query block's last token count for nothing, a block listed
 * twice counts twice. out [num_tokens][Hq][dv] bf16, lse (NULL or fp32, element
 * h * lse_stride_head + row) as for vpp_chunk_attn_run_paged; a row that sees no key gets
 * zeros and lse -infinity; rows of no query block stay as they are. Values of keys that a
 * token does not see do not reach its results, not as infinities or NaN either. The rows
 * of out share no memory with each other or with an input.
 * Arithmetic as for vpp_chunk_attn_run. workspace: 256-byte aligned, may be NULL if the
 * size is 0; not to be used by other work in flight.
 * Errors: VPP_ERR_INVALID_ARG, VPP_ERR_UNSUPPORTED, VPP_ERR_WORKSPACE, VPP_ERR_HIP.
 */
vpp_status_t vpp_block_attn_run_paged(const vpp_block_attn_config_t* cfg,
                                      const vpp_query_block_t* query_blocks, int32_t num_query_blocks,
                                      const void* q, int64_t q_stride_tok, int64_t q_stride_head, int32_t num_tokens,
                                      const void* k_pages, int64_t k_stride_page, int64_t k_stride_tok,
                                      int64_t k_stride_head,
                                      const void* v_pages, int64_t v_stride_page, int64_t v_stride_tok,
                                      int64_t v_stride_head, int32_t page_size, int32_t num_pages,
                                      const int32_t* block_table, int64_t block_table_stride, int32_t num_segments,
                                      int32_t pages_per_row, const int32_t* blocks,
                                      void* out, int64_t o_stride_tok, int64_t o_stride_head,
                                      float* lse, int64_t lse_stride_head,
                                      void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* VPP_BLOCK_ATTN_H */
