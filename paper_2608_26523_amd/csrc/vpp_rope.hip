// vpp_rope.hip -- rotary positions for MI355X (gfx950): rows rotated alone, and a chunk's
// queries and new keys rotated while the keys and values go to a paged cache.
//
// The angle of pair i at a position is position * turns[i] modulo 2^64, a fraction of a
// turn in 64-bit fixed point: one integer multiplication, exact for any position, where a
// product of floats has lost 0.03 radians by position 500000. The top 32 bits become the
// float that v_sin_f32 and v_cos_f32 take, which count in turns (within 1.8e-7 of the
// 64-bit values over 2^20 random phases).
//
// Bound by HBM: rows are read and written once. A workgroup takes the rows of one token, or
// of several that have few; its threads first put the tokens' cos and sin into LDS, once for
// all heads, and then move units of two 16-byte granules: the two that hold the partners of 8
// pairs, or two of the same distance that hold 4 pairs each or are only copied.
// 8192 rows of 128 heads, dims 128..191 of 192 rotated into another tensor, 805 MB: 166 us, 4.85 TB/s;
// 8192 tokens of 64/4 heads into a paged cache, 302 MB: 61 us, 5.0 TB/s; 32 tokens of 32 heads, a chain of
// launch, angles and rows: 3.8 us.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "vpp_rope.h"

namespace {

typedef uint16_t u16;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int NTHREADS = 256;
constexpr int MAX_PAIRS = 512;   // of a head: dims are at most 1024
constexpr int LDS_PAIRS = 2048;  // cos and sin of a workgroup's tokens (16 KB)

struct Divisor {  // x / d for x < 2^31: the high half of x * mul, shifted; mul 0: d = 1
    uint32_t mul;
    int32_t shift;
};
Divisor divisor(uint32_t d) {
    if (d <= 1) return {0, 0};
    int s = 1;  // 2^s >= d
    while (((uint64_t)1 << s) < d) ++s;
    return {(uint32_t)((((uint64_t)1 << (31 + s)) + d - 1) / d), s - 1};
}
__device__ __forceinline__ int divide(int x, Divisor d) {
    return d.mul ? (int)(__umulhi((uint32_t)x, d.mul) >> d.shift) : x;
}

// Rows of one kind (queries, keys or values) of every token.
struct Rows {
    const u16* from;
    u16* to;
    int64_t from_st, from_sh, to_st, to_sh;  // element strides
    int32_t units;                           // of a row
    int32_t turned;                          // of them, rotated (the first ones)
    Divisor by_units;
};

struct RopeArgs {
    Rows q, k, v;
    const uint64_t* turns;
    const int64_t* positions;
    const int64_t* slots;  // null: no cache rows
    int64_t k_sp, v_sp;    // page strides
    int32_t tokens, wg_tokens;
    int32_t q_units, qk_units, units;  // of a token: its queries', with its keys', all
    int32_t pairs;                     // rotary_dim / 2
    int32_t off_gr, rot_gr;            // first rotated granule, rotated granules
    int32_t gran_qk, gran_v;           // granules of a row
    int32_t page_shift, num_pages;
    float scale, sign;                 // sign: of the sine (-1 rotates back)
    Divisor by_token, by_pairs;
};

// One unit of a row: two granules (null: there is no second one, or none at all), and cos and sin of the
// pairs that they hold (c0, c1), or of the pairs that they hold halves of (c0); null: only copied.
struct Unit {
    const u32x4 *f0, *f1;
    u32x4 *t0, *t1;
    const float2 *c0, *c1;
    u32x4 x, y;
};

template <bool INTERLEAVED>
__device__ __forceinline__ void turn(Unit& u) {
    const bf16x8 a = __builtin_bit_cast(bf16x8, u.x), b = __builtin_bit_cast(bf16x8, u.y);
    bf16x8 c, d;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 w = INTERLEAVED ? (i < 4 ? u.c0[i] : u.c1[i - 4]) : u.c0[i];  // cos, sin
        if constexpr (INTERLEAVED) {
            const bf16x8& s = i < 4 ? a : b;
            bf16x8& r = i < 4 ? c : d;
            const float p = (float)s[i % 4 * 2], q = (float)s[i % 4 * 2 + 1];
            r[i % 4 * 2] = (__bf16)(p * w.x - q * w.y);
            r[i % 4 * 2 + 1] = (__bf16)(q * w.x + p * w.y);
        } else {
            const float p = (float)a[i], q = (float)b[i];
            c[i] = (__bf16)(p * w.x - q * w.y);
            d[i] = (__bf16)(q * w.x + p * w.y);
        }
    }
    u.x = __builtin_bit_cast(u32x4, c);
    u.y = __builtin_bit_cast(u32x4, d);
}

template <bool INTERLEAVED, bool NT>
__global__ __launch_bounds__(NTHREADS) void rope_kernel(RopeArgs a) {
    __shared__ float2 cs[LDS_PAIRS];
    const int t0 = (int)blockIdx.x * a.wg_tokens;
    const int tokens = min(a.wg_tokens, a.tokens - t0);
    for (int i = threadIdx.x; i < tokens * a.pairs; i += NTHREADS) {
        const int t = divide(i, a.by_pairs);
        const uint64_t angle = (uint64_t)a.positions[t0 + t] * a.turns[i - t * a.pairs];
        const float turn = (float)(int32_t)(angle >> 32) * 0x1p-32f;
        cs[i] = make_float2(__builtin_amdgcn_cosf(turn) * a.scale, __builtin_amdgcn_sinf(turn) * a.scale * a.sign);
    }
    auto unit = [&](int i) {
        Unit m{};
        if (i >= tokens * a.units) return m;
        const int tl = divide(i, a.by_token), t = t0 + tl;
        int r = i - tl * a.units;
        const bool is_q = r < a.q_units, is_v = r >= a.qk_units;
        const Rows& rows = is_q ? a.q : is_v ? a.v : a.k;
        r -= is_q ? 0 : is_v ? a.qk_units : a.q_units;
        const int h = divide(r, rows.by_units), u = r - h * rows.units;
        const u16* from = rows.from + (int64_t)t * rows.from_st + (int64_t)h * rows.from_sh;
        u16* to = rows.to + (int64_t)h * rows.to_sh;
        if (is_q) {
            to += (int64_t)t * rows.to_st;
        } else {
            const int64_t slot = a.slots[t];
            if (slot < 0 || slot >= ((int64_t)a.num_pages << a.page_shift)) return m;
            to += (slot >> a.page_shift) * (is_v ? a.v_sp : a.k_sp) + (slot & (((int64_t)1 << a.page_shift) - 1)) * rows.to_st;
        }
        // neighbouring threads move neighbouring granules, in both of a thread's
        int g0, g1;
        if (u < rows.turned) {
            g0 = a.off_gr + u;
            g1 = g0 + a.rot_gr / 2;
            m.c0 = cs + tl * a.pairs + u * (INTERLEAVED ? 4 : 8);
            m.c1 = m.c0 + a.rot_gr / 2 * 4;
        } else {  // granules that are only copied: those around the rotated ones
            const int skip = rows.turned ? a.rot_gr : 0, n = (is_v ? a.gran_v : a.gran_qk) - skip;
            const int x = u - rows.turned, y = x + (n + 1) / 2;
            g0 = x < a.off_gr || !skip ? x : x + skip;
            g1 = y >= n ? -1 : y < a.off_gr || !skip ? y : y + skip;
        }
        m.f0 = (const u32x4*)from + g0;
        m.t0 = (u32x4*)to + g0;
        m.f1 = g1 < 0 ? nullptr : (const u32x4*)from + g1;
        m.t1 = (u32x4*)to + g1;
        return m;
    };
    auto load = [](const u32x4* p) { return NT ? __builtin_nontemporal_load(p) : *p; };
    auto store = [](u32x4 x, u32x4* p) {
        if constexpr (NT) __builtin_nontemporal_store(x, p);
        else *p = x;
    };
    // AHEAD units of a thread are loaded before the first is stored: the first ones travel while cos and sin
    // are worked out
    constexpr int AHEAD = 2;
    for (int i0 = 0; i0 < tokens * a.units; i0 += AHEAD * NTHREADS) {
        Unit m[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            m[j] = unit(i0 + j * NTHREADS + (int)threadIdx.x);
            if (m[j].f0) m[j].x = load(m[j].f0);
            if (m[j].f1) m[j].y = load(m[j].f1);
        }
        if (i0 == 0) __syncthreads();
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (m[j].c0) turn<INTERLEAVED>(m[j]);
            if (m[j].f0) store(m[j].x, m[j].t0);
            if (m[j].f1) store(m[j].y, m[j].t1);
        }
    }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
bool stride_ok(int64_t s) { return s > 0 && s % 8 == 0; }
// Token and head strides; that of a single token or head is not used.
bool strides_ok(int64_t st, int64_t tokens, int64_t sh, int64_t heads) {
    return (tokens == 1 || stride_ok(st)) && (heads == 1 || stride_ok(sh));
}
// Whether no two of [tokens][heads] rows of dim elements share memory, tokens or heads outermost.
bool rows_apart(int64_t st, int64_t tokens, int64_t sh, int64_t heads, int64_t dim) {
    if (tokens == 1 || heads == 1) return (tokens == 1 || st >= dim) && (heads == 1 || sh >= dim);
    const int64_t lo = st < sh ? st : sh, hi = st < sh ? sh : st, inner = st < sh ? tokens : heads;
    return lo >= dim && hi / lo >= inner - 1 && hi >= (inner - 1) * lo + dim;
}

vpp_status_t check_config(const vpp_rope_config_t* c) {
    if (!c) return VPP_ERR_INVALID_ARG;
    if (c->head_dim < 16 || c->head_dim > 2 * MAX_PAIRS || c->head_dim % 8) return VPP_ERR_INVALID_ARG;
    if (c->offset < 0 || c->offset % 8 || c->offset > c->head_dim) return VPP_ERR_INVALID_ARG;
    if (c->rotary_dim < 16 || c->rotary_dim % 16 || c->rotary_dim > c->head_dim - c->offset) return VPP_ERR_INVALID_ARG;
    if (c->interleaved != 0 && c->interleaved != 1) return VPP_ERR_INVALID_ARG;
    if (!isfinite(c->scale)) return VPP_ERR_INVALID_ARG;
    return VPP_OK;
}

// Whether [tokens][heads][dim] rows of two buffers are the same memory or share none of it.
bool same_or_apart(const void* x, int64_t x_st, int64_t x_sh, const void* y, int64_t y_st, int64_t y_sh, int64_t tokens,
                   int64_t heads, int64_t dim) {
    // (strides below 2^31, so that the rows' ends below do not wrap)
    for (const int64_t s : {tokens == 1 ? 0 : x_st, heads == 1 ? 0 : x_sh, tokens == 1 ? 0 : y_st, heads == 1 ? 0 : y_sh})
        if (s >= ((int64_t)1 << 31)) return false;
    if (tokens == 1) x_st = y_st = 0;
    if (heads == 1) x_sh = y_sh = 0;
    if (x == y) return x_st == y_st && x_sh == y_sh;
    const uint64_t xb = (uint64_t)(uintptr_t)x, yb = (uint64_t)(uintptr_t)y;
    const uint64_t xe = xb + 2 * (uint64_t)((tokens - 1) * x_st + (heads - 1) * x_sh + dim);
    const uint64_t ye = yb + 2 * (uint64_t)((tokens - 1) * y_st + (heads - 1) * y_sh + dim);
    return xe <= yb || ye <= xb;
}

// The rows' units: `turned` rotated ones, and the other granules two by two.
void set_units(Rows& r, int turned, int copied_granules) {
    r.turned = turned;
    r.units = turned + (copied_granules + 1) / 2;
    r.by_units = divisor((uint32_t)r.units);
}

vpp_status_t launch(const vpp_rope_config_t& c, RopeArgs& a, int32_t hq, int32_t hkv, bool in_place, void* stream) {
    const int copied = (c.head_dim - c.rotary_dim) / 8;
    a.pairs = c.rotary_dim / 2;
    a.off_gr = c.offset / 8;
    a.rot_gr = c.rotary_dim / 8;
    a.gran_qk = c.head_dim / 8;
    a.scale = c.scale;
    set_units(a.q, c.rotary_dim / 16, in_place ? 0 : copied);  // in place, the other dims stay
    set_units(a.k, c.rotary_dim / 16, copied);
    set_units(a.v, 0, a.gran_v);
    const int64_t q_units = (int64_t)hq * a.q.units, units = q_units + (int64_t)hkv * (a.k.units + a.v.units);
    if (units * a.tokens >= ((int64_t)1 << 31) - NTHREADS) return VPP_ERR_INVALID_ARG;
    a.q_units = (int32_t)q_units;
    a.qk_units = (int32_t)(q_units + (int64_t)hkv * a.k.units);
    a.units = (int32_t)units;
    a.by_token = divisor((uint32_t)units);
    a.by_pairs = divisor((uint32_t)a.pairs);
    // Tokens of few rows share a workgroup, up to two units a thread, while four workgroups a CU are left.
    int64_t share = 2 * NTHREADS / units;
    for (const int64_t most : {(int64_t)a.tokens / 1024, (int64_t)LDS_PAIRS / a.pairs})
        if (share > most) share = most;
    a.wg_tokens = share < 1 ? 1 : (int32_t)share;
    const unsigned grid = (unsigned)((a.tokens + a.wg_tokens - 1) / a.wg_tokens);
    // Non-temporal past 64 MB of rows on the way into a cache, twice the L2s: 8192 tokens of 64/4 heads (302 MB
    // moved) 60.8 us, 65.4 without. Rows that are only rotated, 805 MB: 167 and 166.
    const bool nt = a.slots && units * a.tokens * 32 > ((int64_t)64 << 20);
    auto* kernel = c.interleaved ? (nt ? rope_kernel<true, true> : rope_kernel<true, false>)
                                 : (nt ? rope_kernel<false, true> : rope_kernel<false, false>);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(NTHREADS), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? VPP_OK : VPP_ERR_HIP;
}

}  // namespace

extern "C" vpp_status_t vpp_rope_turns(int32_t rotary_dim, const double* frequency, uint64_t* turns) {
    if (rotary_dim < 16 || rotary_dim % 16 || rotary_dim > 2 * MAX_PAIRS || !frequency || !turns) return VPP_ERR_INVALID_ARG;
    for (int i = 0; i < rotary_dim / 2; ++i)
        if (!isfinite(frequency[i])) return VPP_ERR_INVALID_ARG;
    for (int i = 0; i < rotary_dim / 2; ++i) {
        const double t = frequency[i] / 6.283185307179586476925286766559005768;  // turns, 53 bits
        const long double f = ((long double)t - floorl((long double)t)) * 0x1p64L;  // in [0, 2^64]
        const long double r = rintl(f);
        turns[i] = r >= 0x1p64L ? 0 : (uint64_t)r;
    }
    return VPP_OK;
}

extern "C" vpp_status_t vpp_rope(const vpp_rope_config_t* cfg, const void* x, int64_t x_st, int64_t x_sh, void* out,
                                 int64_t o_st, int64_t o_sh, int32_t num_tokens, int32_t num_heads,
                                 const uint64_t* turns, const int64_t* positions, int32_t inverse, void* stream) {
    const vpp_status_t st = check_config(cfg);
    if (st != VPP_OK) return st;
    if (num_tokens < 0 || num_heads < 1) return VPP_ERR_INVALID_ARG;
    if (num_tokens == 0) return VPP_OK;
    if (!x || !out || !turns || !positions) return VPP_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(out) || ((uintptr_t)turns & 7u) || ((uintptr_t)positions & 7u)) return VPP_ERR_INVALID_ARG;
    if (!strides_ok(x_st, num_tokens, x_sh, num_heads) || !strides_ok(o_st, num_tokens, o_sh, num_heads) ||
        !rows_apart(o_st, num_tokens, o_sh, num_heads, cfg->head_dim))
        return VPP_ERR_INVALID_ARG;
    if (!same_or_apart(x, x_st, x_sh, out, o_st, o_sh, num_tokens, num_heads, cfg->head_dim)) return VPP_ERR_INVALID_ARG;
    RopeArgs a{};
    a.q.from = (const u16*)x;
    a.q.to = (u16*)out;
    a.q.from_st = x_st; a.q.from_sh = x_sh; a.q.to_st = o_st; a.q.to_sh = o_sh;
    a.turns = turns;
    a.positions = positions;
    a.tokens = num_tokens;
    a.sign = inverse ? -1.f : 1.f;
    return launch(*cfg, a, num_heads, 0, x == out, stream);
}

extern "C" vpp_status_t vpp_rope_append_paged(
    const vpp_rope_config_t* cfg, const void* q, int64_t q_st, int64_t q_sh, void* q_out, int64_t qo_st, int64_t qo_sh,
    const void* k_new, int64_t kn_st, int64_t kn_sh, const void* v_new, int64_t vn_st, int64_t vn_sh, void* k_pages,
    int64_t k_sp, int64_t k_st, int64_t k_sh, void* v_pages, int64_t v_sp, int64_t v_st, int64_t v_sh, int32_t num_tokens,
    int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim_v, int32_t page_size, int32_t num_pages,
    const uint64_t* turns, const int64_t* positions, const int64_t* slot_mapping, void* stream) {
    const vpp_status_t st = check_config(cfg);
    if (st != VPP_OK) return st;
    if (num_tokens < 0 || num_q_heads < 0 || num_kv_heads < 1 || num_pages < 1) return VPP_ERR_INVALID_ARG;
    if (head_dim_v < 8 || head_dim_v % 8 || head_dim_v > 1024) return VPP_ERR_INVALID_ARG;
    if (page_size < 64 || page_size > (1 << 20) || (page_size & (page_size - 1)) != 0) return VPP_ERR_INVALID_ARG;
    if (num_tokens == 0) return VPP_OK;
    if (!k_new || !v_new || !k_pages || !v_pages || !turns || !positions || !slot_mapping) return VPP_ERR_INVALID_ARG;
    if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(k_pages) || !aligned16(v_pages) || ((uintptr_t)turns & 7u) ||
        ((uintptr_t)positions & 7u) || ((uintptr_t)slot_mapping & 7u))
        return VPP_ERR_INVALID_ARG;
    if (!strides_ok(kn_st, num_tokens, kn_sh, num_kv_heads) || !strides_ok(vn_st, num_tokens, vn_sh, num_kv_heads) ||
        !strides_ok(k_st, page_size, k_sh, num_kv_heads) || !strides_ok(v_st, page_size, v_sh, num_kv_heads) ||
        (num_pages > 1 && (!stride_ok(k_sp) || !stride_ok(v_sp))))
        return VPP_ERR_INVALID_ARG;
    if (num_q_heads > 0) {
        if (!q || !q_out || !aligned16(q) || !aligned16(q_out)) return VPP_ERR_INVALID_ARG;
        if (!strides_ok(q_st, num_tokens, q_sh, num_q_heads) || !strides_ok(qo_st, num_tokens, qo_sh, num_q_heads) ||
            !rows_apart(qo_st, num_tokens, qo_sh, num_q_heads, cfg->head_dim))
            return VPP_ERR_INVALID_ARG;
        if (!same_or_apart(q, q_st, q_sh, q_out, qo_st, qo_sh, num_tokens, num_q_heads, cfg->head_dim))
            return VPP_ERR_INVALID_ARG;
    }
    RopeArgs a{};
    a.q.from = (const u16*)q;
    a.q.to = (u16*)q_out;
    a.q.from_st = q_st; a.q.from_sh = q_sh; a.q.to_st = qo_st; a.q.to_sh = qo_sh;
    a.k.from = (const u16*)k_new;
    a.k.to = (u16*)k_pages;
    a.k.from_st = kn_st; a.k.from_sh = kn_sh; a.k.to_st = k_st; a.k.to_sh = k_sh;
    a.v.from = (const u16*)v_new;
    a.v.to = (u16*)v_pages;
    a.v.from_st = vn_st; a.v.from_sh = vn_sh; a.v.to_st = v_st; a.v.to_sh = v_sh;
    a.turns = turns;
    a.positions = positions;
    a.slots = slot_mapping;
    a.k_sp = k_sp;
    a.v_sp = v_sp;
    a.gran_v = head_dim_v / 8;
    int shift = 0;
    while ((1 << shift) < page_size) ++shift;
    a.page_shift = shift;
    a.num_pages = num_pages;
    a.tokens = num_tokens;
    a.sign = 1.f;
    return launch(*cfg, a, num_q_heads, num_kv_heads, num_q_heads > 0 && q == q_out, stream);
}
