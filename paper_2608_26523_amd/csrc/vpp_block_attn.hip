// vpp_block_attn.hip -- attention to selected blocks of a paged KV cache for MI355X (gfx950).
#include "vpp_block_common.h"

namespace {

// ---------------------------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------------------------
struct AttendArgs {
    const u16* q;
    const u16* k;
    const u16* v;
    u16* out;
    float* lse;
    const vpp_query_block_t* entries;
    const int32_t* lists;
    int64_t q_st, q_sh, k_sp, v_sp, o_st, o_sh, lse_sh;
    int32_t k_st, k_sh, v_st, v_sh;
    Pages pages;
    int32_t num_entries, tokens, segments, query_block, group, hkv;
    int32_t block_shift, max_blocks, chunks;  // chunks: workgroups that share a query block's rows
    float scale_log2;
};

// Raw buffer resource over [base, base + bytes): reads past the end return 0.
__device__ __forceinline__ i32x4 make_rsrc(const void* base, int32_t bytes) {
    const uint64_t b = (uint64_t)(uintptr_t)base;
    i32x4 r;
    r[0] = uniform((int32_t)(uint32_t)b);
    r[1] = uniform((int32_t)((uint32_t)(b >> 32) & 0xffffu));
    r[2] = uniform(bytes);
    r[3] = 0x00020000;
    return r;
}

// 16 bytes per lane from global memory to LDS at base + OFF + 16 * lane. Asm, so that the
// compiler does not wait for it before other LDS reads; the kernel waits itself. The scalar add
// that sets M0 writes SCC.
template <int OFF>
__device__ __forceinline__ void copy16_to_lds(const i32x4& rsrc, uint32_t lds_base, uint32_t voff) {
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(lds_base), "v"(voff), "s"(rsrc), "i"(OFF)
                 : "memory", "scc");
}

template <typename F, int... I>
__device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>()), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
    static_for_impl(f, std::make_integer_sequence<int, N>());
}

// Granule of a V row that sits at granule g of its LDS row. ds_read_b64_tr_b16 serves 32 lanes at
// once, here 8 consecutive keys x 32 bytes: those 8 must fall on different 32-byte parts of the
// 256 bytes that the banks serve.
template <int VGR>
__device__ __forceinline__ int vswz(int key, int g) {
    if constexpr (VGR == 16) return g ^ ((key & 7) << 1);
    else return g ^ (((key >> 1) & 3) << 1);
}

// One workgroup takes up to 16 * RB rows -- (token, head) pairs of a query block and a kv head --
// and each of its waves every fourth tile of 64 listed keys, with all rows: keys and values
// are read once a workgroup and no wave waits for another until the end, where the four
// partial results are joined through LDS.
//   S^T = K Q^T on v_mfma_f32_16x16x32_bf16, K straight from memory (16 bytes a lane), Q held in
//   registers: a lane has one row (column) and 16 of the 64 scores. Softmax in fp32 with exp2.
//   O^T = V^T P^T: P leaves the scores already as the B operand; V^T is read from an LDS copy of
//   the row-major tile by ds_read_b64_tr_b16.
template <int DQK, int DV, int RB>
__global__ __launch_bounds__(NTHREADS) void attend_kernel(AttendArgs a) {
    constexpr int KS = DQK / 32, DB = DV / 16, VGR = DV / 8;
    constexpr int V_BYTES = BN * DV * 2, V_LOADS = V_BYTES / 1024;
    constexpr int ROWS = 16 * RB, OST = DV + 4;  // row stride of a partial result, floats
    constexpr int BYTES = NWAVES * (2 * V_BYTES > ROWS * OST * 4 ? 2 * V_BYTES : ROWS * OST * 4);
    __shared__ __attribute__((aligned(1024))) char smem[BYTES];
    __shared__ int2 list[MAX_LIST];  // first position and page of the listed blocks
    __shared__ float part_m[NWAVES][ROWS], part_l[NWAVES][ROWS];
    __shared__ int list_len;
    const int lane = (int)threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;

    const int head = (int)blockIdx.x % a.hkv, item = (int)blockIdx.x / a.hkv;
    const int chunk = item % a.chunks, ei = item / a.chunks;
    const Entry e = uniform(checked_entry(a.entries[ei], a.query_block, a.tokens, a.segments));
    const int row0 = chunk * ROWS, rows = min(e.rows * a.group - row0, ROWS);  // of the query block's rows
    if (rows <= 0) return;
    const int end = e.pos0 + e.rows;  // cached positions of the segment so far

    if (wave == 0) {
        const int32_t* const from = a.lists + ((int64_t)ei * a.hkv + head) * a.max_blocks;
        int n = 0;
        for (int i0 = 0; i0 < a.max_blocks; i0 += 64) {
            const int b = i0 + lane < a.max_blocks ? from[i0 + lane] : -1;
            const bool use = b >= 0 && b <= (end - 1) >> a.block_shift;
            const uint64_t all = __ballot(use);
            if (use)
                list[n + count(all & (((uint64_t)1 << lane) - 1))] =
                    make_int2(b << a.block_shift, a.pages.page(e.segment, e.kv_start + (b << a.block_shift)));
            n += count(all);
        }
        if (lane == 0) list_len = n;
    }

    // this lane's row of each 16: its token's position, and Q as B operands
    bf16x8 qf[RB][KS];
    int lim[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = row0 + min(rb * 16 + col, rows - 1);
        const int token = r / a.group, h = head * a.group + r - token * a.group;
        lim[rb] = e.pos0 + token;
        const u16* const p = a.q + (int64_t)(e.row0 + token) * a.q_st + (int64_t)h * a.q_sh + grp * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[rb][s] = *(const bf16x8*)(p + s * 32);
    }
    __syncthreads();
    const int shift = a.block_shift - 6;  // tiles of a block
    const int tiles = uniform(list_len) << shift;

    const u16* const kbase = a.k + (int64_t)head * a.k_sh;
    const u16* const vbase = a.v + (int64_t)head * a.v_sh;
    const int pmask = (1 << a.pages.page_shift) - 1;
    uint32_t k_off[4], v_src[V_LOADS];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) k_off[kb] = (uint32_t)((kb * 16 + col) * a.k_st + grp * 8) * 2u;
#pragma unroll
    for (int t = 0; t < V_LOADS; ++t) {
        const int key = (t * 64 + lane) / VGR, g = (t * 64 + lane) % VGR;
        v_src[t] = (uint32_t)(key * a.v_st + vswz<VGR>(key, g) * 8) * 2u;
    }
    char* const vbuf = smem + wave * 2 * V_BYTES;
    const uint32_t vbuf_lds = (uint32_t)(uintptr_t)(lds_void_t*)vbuf;
    // V^T: lane group grp reads keys grp * 4 .. + 3 (and 16 further) of 16 columns
    const int tr_key = grp * 4 + (col >> 2);
    uint32_t v_at[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
        v_at[d] = vbuf_lds + tr_key * (DV * 2) + vswz<VGR>(tr_key, d * 2 + ((col & 3) >> 1)) * 16 + (col & 1) * 8;

    // where tile t's keys are: position of the first, rows of it that are cached, first row's place
    auto tile = [&](int t, int& key0, int& n, int64_t& page, int& row) {
        const int2 b = list[t >> shift];
        key0 = uniform(b.x) + ((t & ((1 << shift) - 1)) << 6);
        n = max(0, min(BN, end - key0));
        page = uniform(b.y);
        row = (e.kv_start + key0) & pmask;
    };
    bf16x8 kf[4][KS];
    auto load_k = [&](int t) {
        int key0, n, row;
        int64_t page;
        tile(t, key0, n, page, row);
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(kbase + page * a.k_sp + (int64_t)row * a.k_st), 0, (int32_t)((uint32_t)n * (uint32_t)a.k_st * 2u), 0x00020000);
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int s = 0; s < KS; ++s)
                kf[kb][s] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(r, (int)k_off[kb] + s * 64, 0, 0));
    };
    auto copy_v = [&](int t, int buf) {
        int key0, n, row;
        int64_t page;
        tile(t, key0, n, page, row);
        const i32x4 r = make_rsrc(vbase + page * a.v_sp + (int64_t)row * a.v_st, (int32_t)((uint32_t)n * (uint32_t)a.v_st * 2u));
        static_for<V_LOADS>([&](auto T) { copy16_to_lds<decltype(T)::value * 1024>(r, vbuf_lds + buf * V_BYTES, v_src[decltype(T)::value]); });
    };

    float m_run[RB], l_run[RB];  // the row's reference maximum; this lane's share of its sum
    f32x4 o[RB][DB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m_run[rb] = -INFINITY;
        l_run[rb] = 0;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[rb][d] = f32x4{0, 0, 0, 0};
    }
    if (wave < tiles) {
        copy_v(wave, 0);
        load_k(wave);
    }
    int buf = 0;
    for (int t = wave; t < tiles; t += NWAVES, buf ^= 1) {
        int key0, n, row;
        int64_t page;
        tile(t, key0, n, page, row);
        f32x4 s[RB][4];
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                s[rb][kb] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < KS; ++k)
                    s[rb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kb][k], qf[rb][k], s[rb][kb], 0, 0, 0);
            }
        // this tile's values are in LDS once the loads up to here are done, and the other buffer is
        // free once the last tile's reads of it are
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        if (t + NWAVES < tiles) {
            copy_v(t + NWAVES, buf ^ 1);
            load_k(t + NWAVES);
        }
        const bool masked = key0 + BN - 1 > e.pos0;
        // Values of keys that not every row sees would reach the others as 0 * inf: here they
        // count as 0, and the rows that see them get them after the product.
        uint64_t wild = 0;
        if (masked && e.rows > 1) {
            bool any = false;
#pragma unroll 1
            for (int i = 0; i < V_LOADS; ++i) {
                const int key = (i * 64 + lane) / VGR;
                if (key0 + key <= e.pos0) continue;
                u32x4* const at = (u32x4*)(vbuf + buf * V_BYTES + (i * 64 + lane) * 16);
                u32x4 x = *at;
                bool bad = false;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if ((x[j] & 0x7f80u) == 0x7f80u) x[j] &= 0xffff0000u, bad = true;
                    if ((x[j] & 0x7f800000u) == 0x7f800000u) x[j] &= 0xffffu, bad = true;
                }
                if (bad) *at = x;
                any = any || bad;
            }
            wild = __ballot(any);
        }
        bf16x8 p[RB][2];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            if (masked) {
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (key0 + kb * 16 + grp * 4 + i > lim[rb]) s[rb][kb][i] = -INFINITY;
            }
            float top = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 4; ++kb)
                top = fmaxf(top, fmaxf(fmaxf(s[rb][kb][0], s[rb][kb][1]), fmaxf(s[rb][kb][2], s[rb][kb][3])));
            top = max_xor32(max_xor16(top)) * a.scale_log2;
            const float m = fmaxf(m_run[rb], top);
            const float use = m == -INFINITY ? 0.f : m;
            const float alpha = __builtin_amdgcn_exp2f(m_run[rb] - use);
            m_run[rb] = m;
            float sum = 0;
#pragma unroll
            for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][kb][i], a.scale_log2, -use));
                    sum += x;
                    p[rb][kb / 2][kb % 2 * 4 + i] = (__bf16)x;
                }
            l_run[rb] = l_run[rb] * alpha + sum;
#pragma unroll
            for (int d = 0; d < DB; ++d) o[rb][d] *= alpha;
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const uint32_t at = v_at[d] + buf * V_BYTES + kk * 32 * DV * 2;
                const i16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(uintptr_t)at);
                const i16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(uintptr_t)(at + 16 * DV * 2));
                bf16x8 vf;
                __builtin_memcpy(&vf, &x, 8);
                __builtin_memcpy((char*)&vf + 8, &y, 8);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) o[rb][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[rb][kk], o[rb][d], 0, 0, 0);
            }
        if (wild) {
            const u16* const v0 = vbase + page * a.v_sp + (int64_t)row * a.v_st + grp * 4;
#pragma unroll 1
            for (int key = max(0, e.pos0 + 1 - key0); key < n; ++key)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const u32x2 x = *(const u32x2*)(v0 + (int64_t)key * a.v_st + d * 16);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float v = __uint_as_float(i % 2 ? x[i / 2] & 0xffff0000u : x[i / 2] << 16);
#pragma unroll
                        for (int rb = 0; rb < RB; ++rb)
                            if (!(fabsf(v) < INFINITY) && key0 + key <= lim[rb]) o[rb][d][i] += v;
                    }
                }
        }
    }

    // join the waves' partial results
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const float l = sum_groups(l_run[rb]);
        if (grp == 0) {
            part_m[wave][rb * 16 + col] = m_run[rb];
            part_l[wave][rb * 16 + col] = l;
        }
    }
    __syncthreads();  // every wave is past its last tile: smem is free
    float* const part = (float*)smem;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int d = 0; d < DB; ++d)
            *(f32x4*)(part + (wave * ROWS + rb * 16 + col) * OST + d * 16 + grp * 4) = o[rb][d];
    __syncthreads();
    for (int i = threadIdx.x; i < rows * (DV / 8); i += NTHREADS) {
        const int r = i / (DV / 8), g = i % (DV / 8);
        float m = part_m[0][r];
#pragma unroll
        for (int w = 1; w < NWAVES; ++w) m = fmaxf(m, part_m[w][r]);
        const float use = m == -INFINITY ? 0.f : m;
        float l = 0, x[8] = {};
#pragma unroll
        for (int w = 0; w < NWAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(part_m[w][r] - use);
            l += part_l[w][r] * f;
            const float* const y = part + (w * ROWS + r) * OST + g * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] += y[j] * f;
        }
        const float inv = l > 0 ? 1 / l : l;  // no key: zeros
        bf16x8 res;
#pragma unroll
        for (int j = 0; j < 8; ++j) res[j] = (__bf16)(x[j] * inv);
        const int tl = (row0 + r) / a.group, h = head * a.group + (row0 + r) % a.group;
        *(bf16x8*)(a.out + (int64_t)(e.row0 + tl) * a.o_st + (int64_t)h * a.o_sh + g * 8) = res;
        if (g == 0 && a.lse) a.lse[(int64_t)h * a.lse_sh + e.row0 + tl] = l > 0 ? (m + __builtin_amdgcn_logf(l)) * LN2 : l == 0 ? -INFINITY : l;
    }
}

}  // namespace

extern "C" vpp_status_t vpp_block_attn_workspace(const vpp_block_attn_config_t* cfg, int32_t num_query_blocks,
                                                 int32_t num_tokens, size_t* bytes) {
    const vpp_status_t st = check_config(cfg);
    if (st != VPP_OK) return st;
    if (num_query_blocks < 0 || num_tokens < 0 || !bytes) return VPP_ERR_INVALID_ARG;
    *bytes = 0;
    return VPP_OK;
}

namespace {
template <int DQK, int DV>
auto pick_attend(int rb) {
    return rb == 1 ? attend_kernel<DQK, DV, 1> : rb == 2 ? attend_kernel<DQK, DV, 2> : attend_kernel<DQK, DV, 4>;
}
}  // namespace

extern "C" vpp_status_t vpp_block_attn_run_paged(
    const vpp_block_attn_config_t* cfg, const vpp_query_block_t* query_blocks, int32_t num_query_blocks, const void* q,
    int64_t q_st, int64_t q_sh, int32_t num_tokens, const void* k_pages, int64_t k_sp, int64_t k_st, int64_t k_sh,
    const void* v_pages, int64_t v_sp, int64_t v_st, int64_t v_sh, int32_t page_size, int32_t num_pages,
    const int32_t* block_table, int64_t bt_st, int32_t num_segments, int32_t pages_per_row, const int32_t* blocks, void* out,
    int64_t o_st, int64_t o_sh, float* lse, int64_t lse_sh, void* workspace, size_t workspace_bytes, void* stream) {
    const vpp_status_t st = check_config(cfg);
    if (st != VPP_OK) return st;
    if (num_query_blocks < 0 || num_tokens < 0 || !page_ok(page_size, num_pages, cfg->block_size)) return VPP_ERR_INVALID_ARG;
    if (num_query_blocks == 0 || num_tokens == 0) return VPP_OK;
    if (!query_blocks || !q || !k_pages || !v_pages || !blocks || !out || !aligned16(query_blocks) || !aligned16(q) ||
        !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out) || ((uintptr_t)blocks & 3u) || ((uintptr_t)lse & 3u) ||
        !table_ok(block_table, bt_st, num_segments, pages_per_row))
        return VPP_ERR_INVALID_ARG;
    const int hq = cfg->num_q_heads, hkv = cfg->num_kv_heads;
    // a tile of 64 cache rows spans less than 2^31 bytes, the range of a buffer resource
    const int64_t row_most = ((int64_t)1 << 31) / (2 * BN);
    const int64_t most = (int64_t)1 << 31;
    const int dqk = cfg->head_dim_qk, dv = cfg->head_dim_v;
    if (!strides_ok(q_st, num_tokens, most, q_sh, hq, dqk) || !strides_ok(o_st, num_tokens, most, o_sh, hq, dv) ||
        !strides_ok(k_st, page_size, row_most, k_sh, hkv, dqk) || !strides_ok(v_st, page_size, row_most, v_sh, hkv, dv) ||
        (num_pages > 1 && (!stride_ok(k_sp) || !stride_ok(v_sp))) || (lse && hq > 1 && lse_sh < num_tokens))
        return VPP_ERR_INVALID_ARG;
    AttendArgs a{};
    a.q = (const u16*)q;
    a.k = (const u16*)k_pages;
    a.v = (const u16*)v_pages;
    a.out = (u16*)out;
    a.lse = lse;
    a.entries = query_blocks;
    a.lists = blocks;
    a.q_st = q_st; a.q_sh = q_sh; a.k_sp = k_sp; a.v_sp = v_sp; a.o_st = o_st; a.o_sh = o_sh; a.lse_sh = lse_sh;
    a.k_st = (int32_t)k_st; a.k_sh = hkv == 1 ? 0 : (int32_t)k_sh;
    a.v_st = (int32_t)v_st; a.v_sh = hkv == 1 ? 0 : (int32_t)v_sh;
    a.pages = Pages{block_table, bt_st, pages_per_row, num_pages, log2_of(page_size)};
    a.num_entries = num_query_blocks;
    a.tokens = num_tokens;
    a.segments = num_segments;
    a.query_block = cfg->query_block;
    a.group = hq / hkv;
    a.hkv = hkv;
    a.block_shift = log2_of(cfg->block_size);
    a.max_blocks = cfg->max_blocks;
    a.scale_log2 = (cfg->softmax_scale > 0 ? cfg->softmax_scale : 1 / sqrtf((float)cfg->head_dim_qk)) * LOG2E;
    const int rows = a.group * a.query_block, rb = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    a.chunks = (rows + 16 * rb - 1) / (16 * rb);
    const int64_t grid = (int64_t)num_query_blocks * a.chunks * hkv;
    if (grid >= ((int64_t)1 << 31)) return VPP_ERR_INVALID_ARG;
    (void)workspace;
    (void)workspace_bytes;
    auto* kernel = cfg->head_dim_qk == 64 ? pick_attend<64, 64>(rb)
                   : cfg->head_dim_qk == 128 ? pick_attend<128, 128>(rb) : pick_attend<192, 128>(rb);
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(NTHREADS), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? VPP_OK : VPP_ERR_HIP;
}
