// vpp_block_common.h -- what the sources of block-sparse attention share: query blocks and pages as
// the device reads them, wave operations, and the checks of arguments.
#ifndef VPP_BLOCK_COMMON_H
#define VPP_BLOCK_COMMON_H

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#include "vpp_block_attn.h"

namespace {

typedef uint16_t u16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void_t;

constexpr int NWAVES = 4;
constexpr int NTHREADS = 64 * NWAVES;
constexpr int BN = 64;               // keys of a tile
constexpr int MAX_LIST = 2048;       // entries of a list
constexpr int MAX_CANDIDATES = 32768;  // blocks that a selection looks at
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// Values of a vector count at most 2^60, and its grid's step is at least 2^-62: the product of
// two steps is a normal number and a sum of 192 products below 2^128.
constexpr float GRID_MOST = 0x1p60f;
constexpr int GRID_MIN_EXP = -54;

__device__ __forceinline__ int count(uint64_t mask) { return (int)__popcll(mask); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The value and its neighbour's 16 or 32 lanes further, combined.
// Of finite numbers (or -infinity): one v_med3_f32, where fmaxf would first make both operands
// canonical. (Not asm: the compiler keeps the distance between a matrix instruction and what
// reads its result.)
__device__ __forceinline__ float max_finite(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, 3.402823466e38f); }
template <bool FINITE = false>
__device__ __forceinline__ float max2(float a, float b) {
    if constexpr (FINITE) return max_finite(a, b);
    else return fmaxf(a, b);
}
template <bool FINITE = false>
__device__ __forceinline__ float max_xor16(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return max2<FINITE>(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <bool FINITE = false>
__device__ __forceinline__ float max_xor32(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return max2<FINITE>(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_groups(float x) {  // over the four 16-lane groups
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The page of a cache row, whatever the table holds.
struct Pages {
    const int32_t* table;
    int64_t table_st;
    int32_t pages_per_row, num_pages, page_shift;
    __device__ __forceinline__ int page(int segment, int row) const {
        const int i = min(row >> page_shift, pages_per_row - 1);
        return (int)min((uint32_t)table[(int64_t)segment * table_st + i], (uint32_t)(num_pages - 1));
    }
};

// A query block as the device reads it; rows = 0 if it is none of this chunk's.
struct Entry {
    int row0, rows, segment, pos0, kv_start;
};
__device__ __forceinline__ Entry checked_entry(const vpp_query_block_t& b, int query_block, int tokens, int segments) {
    Entry e{b.row0, min(b.rows, query_block), b.segment, b.pos0, b.kv_start};
    const bool bad = e.rows < 0 || e.row0 < 0 || e.row0 > tokens - e.rows || e.segment < 0 || e.segment >= segments ||
                     e.pos0 < 0 || e.kv_start < 0 || e.pos0 > INT32_MAX - e.kv_start - 256;
    if (bad) e = Entry{0, 0, 0, 0, 0};
    e.kv_start &= ~(BN - 1);  // so that no tile of keys leaves its page
    return e;
}
__device__ __forceinline__ Entry uniform(const Entry& e) {
    return Entry{uniform(e.row0), uniform(e.rows), uniform(e.segment), uniform(e.pos0), uniform(e.kv_start)};
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
[[maybe_unused]] bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
[[maybe_unused]] bool stride_ok(int64_t s) { return s > 0 && s % 8 == 0; }
[[maybe_unused]] int log2_of(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

[[maybe_unused]] vpp_status_t check_config(const vpp_block_attn_config_t* c) {
    if (!c) return VPP_ERR_INVALID_ARG;
    if (c->num_q_heads < 1 || c->num_kv_heads < 1 || c->num_q_heads % c->num_kv_heads) return VPP_ERR_INVALID_ARG;
    if (c->num_q_heads / c->num_kv_heads > 128) return VPP_ERR_INVALID_ARG;
    if (!isfinite(c->softmax_scale) || c->softmax_scale < 0) return VPP_ERR_INVALID_ARG;
    if (c->block_size != 64 && c->block_size != 128 && c->block_size != 256) return VPP_ERR_INVALID_ARG;
    if (c->query_block < 1 || c->query_block > 128) return VPP_ERR_INVALID_ARG;
    if (c->sink_blocks < 0 || c->local_blocks < 1 || c->max_blocks < 1 || c->max_blocks > MAX_LIST) return VPP_ERR_INVALID_ARG;
    const int64_t sure = (int64_t)c->sink_blocks + c->local_blocks + (c->query_block - 1 + c->block_size - 1) / c->block_size;
    if (c->max_blocks < sure) return VPP_ERR_INVALID_ARG;
    const int d = c->head_dim_qk, v = c->head_dim_v;
    if (!((d == 64 && v == 64) || (d == 128 && v == 128) || (d == 192 && v == 128))) return VPP_ERR_UNSUPPORTED;
    return VPP_OK;
}

[[maybe_unused]] bool page_ok(int32_t page_size, int32_t num_pages, int32_t block_size) {
    return page_size >= block_size && page_size <= (1 << 20) && (page_size & (page_size - 1)) == 0 && num_pages >= 1;
}

[[maybe_unused]] bool table_ok(const int32_t* table, int64_t st, int32_t segments, int32_t pages_per_row) {
    return table && ((uintptr_t)table & 3u) == 0 && segments >= 1 && pages_per_row >= 1 && (segments == 1 || st >= 0);
}

// [rows][heads][dim] strides in elements; the stride of a size of 1 is not used
[[maybe_unused]] bool strides_ok(int64_t st, int64_t rows, int64_t st_most, int64_t sh, int64_t heads, int64_t dim) {
    return (rows == 1 || (stride_ok(st) && st >= dim && st < st_most)) &&
           (heads == 1 || (stride_ok(sh) && sh >= dim && sh < ((int64_t)1 << 31)));
}

// Whether no two of [rows][heads] vectors of dim elements share memory, rows or heads outermost.
[[maybe_unused]] bool rows_apart(int64_t st, int64_t rows, int64_t sh, int64_t heads, int64_t dim) {
    if (rows == 1 || heads == 1) return (rows == 1 || st >= dim) && (heads == 1 || sh >= dim);
    const int64_t lo = st < sh ? st : sh, hi = st < sh ? sh : st, inner = st < sh ? rows : heads;
    return lo >= dim && hi / lo >= inner - 1 && hi >= (inner - 1) * lo + dim;
}

}  // namespace

#endif  // VPP_BLOCK_COMMON_H
