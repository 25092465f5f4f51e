/*
 * vpp_rope.h -- rotary positions for the rows that chunked-prefill attention reads
 * (vpp_chunk_attn.h), alone and on the way into a paged KV cache.
 *
 * A pair (a, b) of a head's dims is rotated by the angle position * frequency:
 *   a' = scale * (a cos t - b sin t),   b' = scale * (b cos t + a sin t).
 * Of head_dim dims, rotary_dim from `offset` on are rotated; the others are copied.
 * Pair i of them is dims (i, i + rotary_dim / 2) of the rotated part, or, interleaved,
 * dims (2i, 2i + 1).
 *
 * Angles are held in turns as 64-bit fixed-point numbers: turns[i] is the double quotient
 * of frequency i and 2 pi, times 2^64 and modulo that, rounded (vpp_rope_turns), and
 * position * turns[i] modulo 2^64 is the angle's fraction of a turn, without a rounding
 * however far the position. Positions are any 64-bit integers, negative ones too.
 *
 * Types: rows bf16, arithmetic fp32 with cos and sin within 2e-7, results rounded once
 * (nearest even). Layouts, strides (elements, last dimension contiguous), alignment (16-byte
 * pointers, strides multiples of 8; the stride of a dimension of size 1 is not used) and
 * status codes are those of vpp_chunk_attn.h. Strides of x, q, out and q_out are below 2^31;
 * the rows of out and of q_out share no memory. Calls are asynchronous on `stream` (a
 * hipStream_t of the current device; NULL is the default stream), allocate nothing, need no
 * workspace and may be captured.
 */
#ifndef VPP_ROPE_H
#define VPP_ROPE_H

#include "vpp_chunk_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* How the dims of a head are rotated, passed by value (copied). */
typedef struct {
    int32_t head_dim;    /* a multiple of 8, at most 1024                           */
    int32_t rotary_dim;  /* a multiple of 16, 16 .. head_dim - offset               */
    int32_t offset;      /* first rotated dim, a multiple of 8                      */
    int32_t interleaved; /* 0: pairs (i, i + rotary_dim / 2); 1: pairs (2i, 2i + 1) */
    float scale;         /* factor on the rotated dims (1 unless the frequencies'
                            scaling asks for another); finite                       */
} vpp_rope_config_t;

/*
 * Host helper: turns[i] (rotary_dim / 2 entries, host) of the angles per position
 * frequency[i] (radians, rotary_dim / 2 entries, host). Errors: VPP_ERR_INVALID_ARG for
 * a bad rotary_dim, a null pointer or a frequency that is not finite.
 */
vpp_status_t vpp_rope_turns(int32_t rotary_dim, const double* frequency, uint64_t* turns);

/*
 * Rotate the rows x [tokens][heads][head_dim] of tokens at positions[t] into out (the
 * same shape, its own strides). out may be x itself, with the same strides; any other
 * overlap of the two is refused. `inverse` rotates back by the same angles (with the same
 * scale): for scale 1 the inverse, for any scale the transpose, which is the gradient
 * of the rotation. turns is a device array of vpp_rope_turns, positions a device array;
 * both are read on `stream`.
 * Errors: VPP_ERR_INVALID_ARG, VPP_ERR_HIP (launch failure).
 */
vpp_status_t vpp_rope(const vpp_rope_config_t* cfg,
                      const void* x, int64_t x_stride_tok, int64_t x_stride_head,
                      void* out, int64_t o_stride_tok, int64_t o_stride_head,
                      int32_t num_tokens, int32_t num_heads,
                      const uint64_t* turns, const int64_t* positions, int32_t inverse, void* stream);

/*
 * vpp_kv_append_paged with the rotation on the way, and that of the chunk's queries in
 * the same launch: token t's k_new rows are rotated by positions[t] and written, with its
 * v_new rows as they are, to slot slot_mapping[t] of k_pages / v_pages; its q rows
 * [num_q_heads][head_dim] are rotated into q_out (which may be q itself, with the same
 * strides; any other overlap of the two is refused). cfg->head_dim is the dim of queries
 * and keys. num_q_heads = 0 leaves the queries out (q and q_out may be NULL). Slots
 * outside [0, num_pages * page_size) skip the token's cache rows, not its queries. Two
 * tokens mapped to one slot race; q_out must not overlap k_new or v_new, nor the
 * pages any input.
 * Errors: VPP_ERR_INVALID_ARG, VPP_ERR_HIP (launch failure).
 */
vpp_status_t vpp_rope_append_paged(const vpp_rope_config_t* cfg,
                                   const void* q, int64_t q_stride_tok, int64_t q_stride_head,
                                   void* q_out, int64_t qo_stride_tok, int64_t qo_stride_head,
                                   const void* k_new, int64_t kn_stride_tok, int64_t kn_stride_head,
                                   const void* v_new, int64_t vn_stride_tok, int64_t vn_stride_head,
                                   void* k_pages, int64_t k_stride_page, int64_t k_stride_tok,
                                   int64_t k_stride_head,
                                   void* v_pages, int64_t v_stride_page, int64_t v_stride_tok,
                                   int64_t v_stride_head,
                                   int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads,
                                   int32_t head_dim_v, int32_t page_size, int32_t num_pages,
                                   const uint64_t* turns, const int64_t* positions,
                                   const int64_t* slot_mapping, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* VPP_ROPE_H */
