// vpp_block_attn.hip -- attention to selected blocks of a paged KV cache for MI355X (gfx950).
#include "vpp_block_common.h"

namespace {

// ---------------------------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------------------------
constexpr int BT = 32;                 // keys of a tile
constexpr int MAX_PACK = 16;           // query blocks of a workgroup
constexpr int MAX_ELEMENTS = 2048;     // listed blocks of a workgroup that packs several
constexpr int MAX_SPLITS = 16;
// A row's reference maximum moves only when a score passes it by more than 2^LAZY: sums and
// products share the reference, so quotients do not change, and P stays below 2^LAZY.
constexpr float LAZY = 8.f;

struct AttendArgs {
    const u16* q;
    const u16* k;
    const u16* v;
    u16* out;
    float* lse;
    float* part_o;    // [splits][tokens][hq][dv], where the lists are split
    float* part_lse;  // [splits][tokens][hq], of powers of two
    const vpp_query_block_t* entries;
    const int32_t* lists;
    int64_t q_st, q_sh, k_sp, v_sp, o_st, o_sh, lse_sh;
    int32_t k_st, k_sh, v_st, v_sh;
    Pages pages;
    int32_t num_entries, tokens, segments, query_block, group, hkv;
    int32_t block_shift, max_blocks;
    int32_t heads, items;                // kv heads whose workgroups run at one time; workgroups of a head
    int32_t generation;                  // of those, at one time
    int32_t pack, rows, chunks, splits;  // query blocks of a workgroup, rows of one; workgroups of their rows, of their lists
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
__device__ __forceinline__ void copy16_to_lds(const i32x4& rsrc, uint32_t lds_base, uint32_t voff, uint32_t soff) {
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %4 offen lds"
                 :
                 : "s"(lds_base), "v"(voff), "s"(rsrc), "i"(OFF), "s"(soff)
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

// Granule of a K row that sits at granule g of its LDS row. ds_read_b128 serves 16 lanes at once, here one
// granule of 16 rows: they must fall on different 16-byte parts of the banks' 256 bytes.
template <int KGR>
__device__ __forceinline__ int kswz(int row, int g) {
    if constexpr (KGR % 16 == 0) return g ^ (row & 15);
    else return g ^ ((row >> 1) & 7);
}

// Granule of a V row that sits at granule g of its LDS row. ds_read_b64_tr_b16 serves 32 lanes at
// once, here 8 consecutive keys x 32 bytes: those 8 must fall on different 32-byte parts of the
// 256 bytes that the banks serve.
template <int VGR>
__device__ __forceinline__ int vswz(int key, int g) {
    if constexpr (VGR == 16) return g ^ ((key & 7) << 1);
    else return g ^ (((key >> 1) & 3) << 1);
}

// O of 64 columns fills the accumulation registers. In rarely taken branches it is read from there by asm: for
// ordinary operands the compiler copies all of it out every tile (8192 tokens in query blocks of 64: 606 us,
// so 563). The asm does not wait for matrix products: products_done() first.
template <bool ASM>
__device__ __forceinline__ void products_done() {
    if constexpr (ASM) asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
}
template <bool ASM>
__device__ __forceinline__ float out_of_agprs(float x) {
    if constexpr (ASM) {
        float y;
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(y) : "a"(x));
        return y;
    }
    return x;
}
template <bool ASM>
__device__ __forceinline__ f32x4 out_of_agprs(f32x4 x) {
    return f32x4{out_of_agprs<ASM>(x[0]), out_of_agprs<ASM>(x[1]), out_of_agprs<ASM>(x[2]), out_of_agprs<ASM>(x[3])};
}

// A listed block, once for all query blocks of a workgroup that list it.
struct Element {
    int key0, page, row;  // position of its first key; its page and first row of it
    int rows_mask;        // cached rows of it << 16 | query blocks that list it
};

// The workgroup's list of blocks. A block that several of its query blocks list becomes one element,
// with all their bits, if every list ascends (as a selection's do): each block is looked up in the
// other lists of the same request by bisection, is left to the first list that has it, and takes
// the place that its order gives it among all. Else every entry is an element of its own, so that
// a block listed twice counts twice. Either way the order is the same every time.
// raw and ranks: [entries * max_blocks + 1], shared: two numbers. Returns the elements' number.
__device__ __forceinline__ int list_elements(const AttendArgs& a, const Entry* ents, int entries, int entry0, int head, int* raw,
                                             int* ranks, Element* elements, int* shared) {
    const int lane = (int)threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), most = a.max_blocks, total = entries * most;
    for (int i = threadIdx.x; i < total; i += NTHREADS) {
        const int t = i / most, j = i - t * most;
        const Entry e = ents[t];
        const int b = a.lists[((int64_t)(entry0 + t) * a.hkv + head) * most + j];
        raw[i] = e.rows > 0 && b >= 0 && b <= (e.pos0 + e.rows - 1) >> a.block_shift ? b : INT32_MAX;
    }
    if (threadIdx.x == 0) shared[0] = 0;
    __syncthreads();
    auto element = [&](int b, const Entry& e, int end, int mask) {
        Element x;
        x.key0 = b << a.block_shift;
        const int row = e.kv_start + x.key0;
        x.page = a.pages.page(e.segment, row);
        x.row = row & ((1 << a.pages.page_shift) - 1);
        x.rows_mask = min(1 << a.block_shift, end - x.key0) << 16 | mask;
        return x;
    };
    if (entries == 1) {  // a list as it is, without its holes; ranks are not used
        int n = 0;
        for (int i0 = 0; i0 < most && wave == 0; i0 += 64) {
            const int b = i0 + lane < most ? raw[i0 + lane] : INT32_MAX;
            const uint64_t all = __ballot(b != INT32_MAX);
            if (b != INT32_MAX) elements[n + count(all & (((uint64_t)1 << lane) - 1))] = element(b, ents[0], ents[0].pos0 + ents[0].rows, 1);
            n += count(all);
        }
        if (threadIdx.x == 0) shared[1] = n;
        __syncthreads();
        return uniform(shared[1]);
    }
    {
        bool bad = false;
        for (int i = threadIdx.x; i < total; i += NTHREADS)
            bad = bad || (i % most && (raw[i - 1] == INT32_MAX ? raw[i] != INT32_MAX : raw[i] <= raw[i - 1]));
        if (__ballot(bad) && lane == 0) shared[0] = 1;
        __syncthreads();
    }
    const bool merge = uniform(shared[0]) == 0;
    auto bisect = [&](int o, int b) {  // first place of list o with a block >= b
        const int* const r = raw + o * most;
        int l = 0, h = most;
        while (l < h) {
            const int m = (l + h) >> 1;
            if (r[m] < b) l = m + 1;
            else h = m;
        }
        return l;
    };
    auto apart = [&](const Entry& x, const Entry& y) { return x.segment != y.segment || x.kv_start != y.kv_start; };
    // which entries become elements, and how many before each
    for (int i = threadIdx.x; i < total; i += NTHREADS) {
        const int b = raw[i], t = i / most;
        bool mine = b != INT32_MAX;
        if (merge && mine)
            for (int o = 0; o < t && mine; ++o) {
                if (apart(ents[o], ents[t])) continue;
                const int l = bisect(o, b);
                mine = l == most || raw[o * most + l] != b;
            }
        ranks[i] = mine;
    }
    __syncthreads();
    if (wave == 0) {
        int n = 0;
        for (int i0 = 0; i0 < total; i0 += 64) {
            const bool mine = i0 + lane < total && ranks[i0 + lane];
            const uint64_t all = __ballot(mine);
            if (i0 + lane < total) ranks[i0 + lane] = (n + count(all & (((uint64_t)1 << lane) - 1))) * 2 + mine;
            n += count(all);
        }
        if (lane == 0) ranks[total] = n * 2, shared[1] = n;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < total; i += NTHREADS) {
        if (!(ranks[i] & 1)) continue;
        const int b = raw[i], t = i / most;
        const Entry e = ents[t];
        int mask = 1 << t, end = e.pos0 + e.rows, at = ranks[i] >> 1;
        if (merge) {
            at = 0;
            for (int o = 0; o < entries; ++o) {
                const Entry f = ents[o];
                const int l = bisect(o, b);
                at += (ranks[o * most + l] >> 1) - (ranks[o * most] >> 1);  // of list o's elements, those before b
                // an equal block of another request: by the order of the lists
                if (l < most && raw[o * most + l] == b) {
                    if (!apart(e, f)) mask |= 1 << o, end = max(end, f.pos0 + f.rows);
                    else if (o < t) at += ranks[o * most + l] & 1;
                }
            }
        }
        elements[at] = element(b, e, end, mask);
    }
    __syncthreads();
    return uniform(shared[1]);
}

// One workgroup takes up to 16 * RB rows -- (token, head) pairs of a kv head, of one query block or
// of several short ones -- and each of its waves every fourth tile of 32 listed keys, with all rows:
// keys and values are read once a workgroup and no wave waits for another until the end, where
// the four partial results are joined through LDS.
//   S^T = K Q^T on v_mfma_f32_16x16x32_bf16, Q held in registers: a lane has one row (column) and 8
//   of the 32 scores. Softmax in fp32 with exp2.
//   O^T = V^T P^T: P, rounded to bf16 as the matrix instruction takes it, leaves the scores
//   already as the B operand; V^T is read from the row-major tile by ds_read_b64_tr_b16.
// Keys and values come into a wave's own LDS, so it waits for its copies alone: keys read
// from memory in the operand's layout are 64-byte pieces of 16 rows (query blocks of 64 tokens, 16 heads,
// 64 blocks a list behind 120K: 975 us, through LDS 620).
// Infinities and NaN among values that only some rows see would reach the others as 0 * inf. They
// are not looked for: only if a result is not finite the workgroup does its tiles again, carefully.
// SKIP: several query blocks, and tiles that none of a 16 rows' lists pass them by.
//
// What bounds it:
//   single tokens of many requests: HBM (32 of 32/8 heads, 32 blocks each, 254 MB: 49 us, 5.2 TB/s);
//   every token its own list: the blocks that few rows share, out of the caches (4096 tokens of 32/8
//   heads, 16 blocks each, 14 GB of tiles: 640 us, 22 TB/s);
//   long query blocks: the instructions that one wave a SIMD issues, scores, softmax and products in turn
//   (8192 tokens in query blocks of 64: 563 us, 606 TFLOP/s). More in flight does not help, nor the next
//   scores beside this softmax: two key buffers 663 us against 641 on one card, scores ahead 651 to 627.
template <int DQK, int DV, int RB, bool SKIP>
__global__ __attribute__((amdgpu_flat_work_group_size(NTHREADS, NTHREADS), amdgpu_waves_per_eu(RB == 4 || DQK == 192 ? 1 : 2)))
void attend_kernel(AttendArgs a) {
    constexpr int KS = DQK / 32, DB = DV / 16, KGR = DQK / 8, VGR = DV / 8;
    constexpr int K_BYTES = BT * DQK * 2, K_LOADS = K_BYTES / 1024, V_BYTES = BT * DV * 2, V_LOADS = V_BYTES / 1024;
    constexpr int VB = RB == 4 ? 2 : 1;                    // V buffers of a wave
    constexpr int WAVE_BYTES = K_BYTES + VB * V_BYTES;
    // copies of a tile after which the swizzle repeats
    constexpr int K_PERIOD = KGR == 16 ? 4 : KGR == 24 ? 6 : 2;
    constexpr int ROWS = 16 * RB, JP = RB == 4 ? 2 : 1;    // joined in JP parts of the columns
    constexpr int OST = DV / JP + 4;                       // row stride of a partial result, floats
    constexpr int JOIN = NWAVES * ROWS * OST * 4, BYTES = NWAVES * WAVE_BYTES > JOIN ? NWAVES * WAVE_BYTES : JOIN;
    __shared__ __attribute__((aligned(1024))) char smem[BYTES];
    __shared__ float part_m[NWAVES][ROWS], part_l[NWAVES][ROWS];
    __shared__ Entry ents[MAX_PACK];
    __shared__ int shared[4];
    extern __shared__ Element elements[];  // [pack * max_blocks], and behind them the lists and the ranks
    const int lane = (int)threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;

    // Workgroups go to the 8 XCDs in turn: with 8 heads at a time those of one head share an XCD's L2.
    const int turn = (int)blockIdx.x / (a.items * a.heads), in_turn = (int)blockIdx.x - turn * a.items * a.heads;
    const int head = turn * a.heads + in_turn % a.heads;
    int item = in_turn / a.heads;
    const int split = item % a.splits;
    item /= a.splits;
    const int chunk = item % a.chunks, entry0 = item / a.chunks * a.pack;
    const int entries = min(a.pack, a.num_entries - entry0);
    if ((int)threadIdx.x < entries)
        ents[threadIdx.x] = checked_entry(a.entries[entry0 + threadIdx.x], a.query_block, a.tokens, a.segments);
    __syncthreads();
    const int row0 = chunk * ROWS;  // (one query block) of its rows
    if (entries == 1 && uniform(ents[0].rows) * a.group <= row0) return;

    // this lane's rows: their place, and Q as B operands
    bf16x8 qf[RB][KS];
    int lim[RB], bit[RB];  // last position that the row sees; its query block's bit
    int bits[RB];          // of the query blocks of these 16 rows
    int first_pos = INT32_MAX;
    for (int t = 0; t < entries; ++t) first_pos = min(first_pos, uniform(ents[t].pos0));
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int c = row0 + rb * 16 + col, t = entries > 1 ? min(c / a.rows, entries - 1) : 0;
        const Entry e = ents[t];
        const int r = max(0, min(c - t * a.rows, e.rows * a.group - 1));  // past the last row: that one again
        const int token = r / a.group, h = head * a.group + r - token * a.group;
        lim[rb] = e.pos0 + token;
        bit[rb] = 1 << t;
        // (none of its own: those of the last, which the tiles do anyway)
        const int t0 = entries > 1 ? min(rb * 16 / a.rows, entries - 1) : 0, t1 = entries > 1 ? min((rb * 16 + 15) / a.rows, entries - 1) : 0;
        bits[rb] = (2 << t1) - (1 << t0);
        const u16* const p = a.q + (int64_t)(e.row0 + token) * a.q_st + (int64_t)h * a.q_sh + grp * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[rb][s] = *(const bf16x8*)(p + s * 32);
    }
    int* const raw = (int*)(elements + a.pack * a.max_blocks);
    const int listed = list_elements(a, ents, entries, entry0, head, raw, raw + a.pack * a.max_blocks, elements, shared);
    const int shift = a.block_shift - 5;  // tiles of a block
    const int tiles = listed << shift;
    const int tile_end = (int)((int64_t)tiles * (split + 1) / a.splits), tile0 = (int)((int64_t)tiles * split / a.splits) + wave;
    // The workgroups that run at one time read the same blocks at about one time, out of their XCD's L2, if the
    // next ones begin where these end: every other generation of them goes down its list (4096 tokens of 32/8
    // heads, 16 blocks each: 640 us, always up 660).
    const bool down = (uint32_t)item / (uint32_t)a.generation & 1;
    const int all_bits = (1 << entries) - 1;

    const u16* const kbase = a.k + (int64_t)head * a.k_sh;
    const u16* const vbase = a.v + (int64_t)head * a.v_sh;
    // sources of a tile's copies, less what the scalar offset adds
    uint32_t k_src[K_PERIOD], v_src[2];
#pragma unroll
    for (int i = 0; i < K_PERIOD; ++i) {
        const int slot = i * 64 + lane, key = slot / KGR, g = slot % KGR;
        k_src[i] = (uint32_t)(key * a.k_st + kswz<KGR>(key, g) * 8) * 2u;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int slot = i * 64 + lane, key = slot / VGR, g = slot % VGR;
        v_src[i] = (uint32_t)(key * a.v_st + vswz<VGR>(key, g) * 8) * 2u;
    }
    char* const vbuf = smem + wave * WAVE_BYTES;
    const uint32_t vbuf_lds = (uint32_t)(uintptr_t)(lds_void_t*)vbuf, kbuf_lds = vbuf_lds + VB * V_BYTES;
    // K: lane group grp reads granule 4 s + grp of row col (and of the row 16 further)
    const u32x4* k_at[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) k_at[s] = (const u32x4*)(vbuf + VB * V_BYTES + col * (DQK * 2) + kswz<KGR>(col, s * 4 + grp) * 16);
    // V^T: lane group grp reads keys grp * 4 .. + 3 (and 16 further) of 16 columns
    const int tr_key = grp * 4 + (col >> 2);
    uint32_t v_at[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
        v_at[d] = vbuf_lds + tr_key * (DV * 2) + vswz<VGR>(tr_key, d * 2 + ((col & 3) >> 1)) * 16 + (col & 1) * 8;

    struct Tile {
        int key0, n, page, row, mask;  // n: cached keys of it
    };
    auto tile = [&](int t) {
        if (down) t = tiles - 1 - t;
        const Element x = elements[t >> shift];
        const int sub = (t & ((1 << shift) - 1)) * BT, rm = uniform(x.rows_mask);
        return Tile{uniform(x.key0) + sub, max(0, min(BT, (rm >> 16) - sub)), uniform(x.page), uniform(x.row) + sub, rm & 0xffff};
    };
    auto copy_k = [&](const Tile& x) {
        const i32x4 r = make_rsrc(kbase + x.page * a.k_sp + (int64_t)x.row * a.k_st, (int32_t)((uint32_t)x.n * (uint32_t)a.k_st * 2u));
        static_for<K_LOADS>([&](auto T) {
            constexpr int t = decltype(T)::value, rows = t / K_PERIOD * K_PERIOD * 64 / KGR;
            copy16_to_lds<t * 1024>(r, kbuf_lds, k_src[t % K_PERIOD], (uint32_t)(rows * 2) * (uint32_t)a.k_st);
        });
    };
    auto copy_v = [&](const Tile& x, int buf) {
        const i32x4 r = make_rsrc(vbase + x.page * a.v_sp + (int64_t)x.row * a.v_st, (int32_t)((uint32_t)x.n * (uint32_t)a.v_st * 2u));
        static_for<V_LOADS>([&](auto T) {
            constexpr int t = decltype(T)::value, rows = t / 2 * 2 * 64 / VGR;
            copy16_to_lds<t * 1024>(r, vbuf_lds + buf * V_BYTES, v_src[t % 2], (uint32_t)(rows * 2) * (uint32_t)a.v_st);
        });
    };

    float m_run[RB], l_run[RB];  // the row's reference maximum; this lane's share of its sum
    f32x4 o[RB][DB];
    for (bool careful = false;; careful = true) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            m_run[rb] = -INFINITY;
            l_run[rb] = 0;
#pragma unroll
            for (int d = 0; d < DB; ++d) o[rb][d] = f32x4{0, 0, 0, 0};
        }
        int buf = 0;
        Tile now{}, next{};
        // Copies are in flight in this order: K(t), V(t) | K(t + 1), V(t + 1), a tile's K after the scores of the
        // one before, its V after the values of the one before (with two V buffers with its K), and waits
        // count the younger ones. No other load of the loop is waited for by number.
        if (tile0 < tile_end) {
            now = tile(tile0);
            copy_k(now);
            copy_v(now, 0);
        }
        for (int t = tile0; t < tile_end; t += NWAVES, now = next) {
            const bool more = t + NWAVES < tile_end;
            if (more) next = tile(t + NWAVES);
            asm volatile("s_waitcnt vmcnt(%0)" ::"i"(V_LOADS) : "memory");
            f32x4 s[RB][2];
            bf16x8 kf[2][KS];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int k = 0; k < KS; ++k) kf[kb][k] = __builtin_bit_cast(bf16x8, k_at[k][kb * 16 * KGR]);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                if (SKIP && !(now.mask & bits[rb])) continue;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    s[rb][kb] = f32x4{0, 0, 0, 0};
#pragma unroll
                    for (int k = 0; k < KS; ++k)
                        s[rb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kb][k], qf[rb][k], s[rb][kb], 0, 0, 0);
                }
            }
            if (more) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // K is read (and V of the tile before)
                copy_k(next);
                if constexpr (VB == 2) copy_v(next, buf ^ 1);
            }
            const bool masked = now.key0 + BT - 1 > first_pos, partial = now.mask != all_bits;
            if (__builtin_expect(masked || partial, SKIP)) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    if (SKIP && !(now.mask & bits[rb])) continue;
                    const int last = now.mask & bit[rb] ? lim[rb] : -1;
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (now.key0 + kb * 16 + grp * 4 + i > last) s[rb][kb][i] = -INFINITY;
                }
            }
            bool above = false;
            float top[RB];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                top[rb] = -INFINITY;
                if (SKIP && !(now.mask & bits[rb])) continue;
                top[rb] = fmaxf(fmaxf(fmaxf(s[rb][0][0], s[rb][0][1]), fmaxf(s[rb][0][2], s[rb][0][3])),
                                fmaxf(fmaxf(s[rb][1][0], s[rb][1][1]), fmaxf(s[rb][1][2], s[rb][1][3]))) * a.scale_log2;
                above = above || top[rb] > m_run[rb] + LAZY;
            }
            if (__builtin_expect(__ballot(above) != 0, 0)) {
                products_done<RB == 4>();
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    const float m = fmaxf(m_run[rb], max_xor32(max_xor16(top[rb])));
                    const float alpha = __builtin_amdgcn_exp2f(m_run[rb] - (m == -INFINITY ? 0.f : m));
                    m_run[rb] = m;
                    l_run[rb] *= alpha;
#pragma unroll
                    for (int d = 0; d < DB; ++d) o[rb][d] = out_of_agprs<RB == 4>(o[rb][d]) * alpha;
                }
            }
            bf16x8 p[RB];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                if (SKIP && !(now.mask & bits[rb])) continue;
                const float use = m_run[rb] == -INFINITY ? 0.f : m_run[rb];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][kb][i], a.scale_log2, -use));
                        l_run[rb] += x;
                        p[rb][kb * 4 + i] = (__bf16)x;
                    }
            }
            // this tile's values are in LDS: only what belongs to the next one is younger
            if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"i"(K_LOADS + (VB == 2 ? V_LOADS : 0)) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            bool wild = false;
            if (__builtin_expect(careful && (masked || partial), 0)) {
                // values that are not finite count as 0 here; the rows that see them get them after the product
#pragma unroll 1
                for (int i = 0; i < V_LOADS; ++i) {
                    u32x4* const at = (u32x4*)(vbuf + buf * V_BYTES + (i * 64 + lane) * 16);
                    u32x4 x = *at;
                    bool bad = false;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if ((x[j] & 0x7f80u) == 0x7f80u) x[j] &= 0xffff0000u, bad = true;
                        if ((x[j] & 0x7f800000u) == 0x7f800000u) x[j] &= 0xffffu, bad = true;
                    }
                    if (bad) *at = x;
                    wild = wild || bad;
                }
                wild = __ballot(wild) != 0;
            }
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const uint32_t at = v_at[d] + buf * V_BYTES;
                const i16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(uintptr_t)at);
                const i16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(uintptr_t)(at + 16 * DV * 2));
                bf16x8 vf;
                __builtin_memcpy(&vf, &x, 8);
                __builtin_memcpy((char*)&vf + 8, &y, 8);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
                    if (!SKIP || now.mask & bits[rb]) o[rb][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[rb], o[rb][d], 0, 0, 0);
            }
            if (__builtin_expect(wild, 0)) {
                products_done<RB == 4>();
                const u16* const v0 = vbase + now.page * a.v_sp + (int64_t)now.row * a.v_st + grp * 4;
#pragma unroll 1
                for (int key = 0; key < now.n; ++key)
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        const u32x2 x = *(const u32x2*)(v0 + (int64_t)key * a.v_st + d * 16);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float v = __uint_as_float(i % 2 ? x[i / 2] & 0xffff0000u : x[i / 2] << 16);
#pragma unroll
                            for (int rb = 0; rb < RB; ++rb)
                                if (!(fabsf(v) < INFINITY) && now.key0 + key <= (now.mask & bit[rb] ? lim[rb] : -1)) o[rb][d][i] = out_of_agprs<RB == 4>(o[rb][d][i]) + v;
                        }
                    }
            }
            if constexpr (VB == 1) {
                // the buffer is free once the reads above are done
                if (more) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    copy_v(next, 0);
                }
            } else {
                buf ^= 1;
            }
        }
        // 0 * inf is NaN
        float probe = 0;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) probe = __builtin_fmaf(o[rb][d][i], 0.f, probe);
        if (threadIdx.x == 0) shared[2] = 0;
        __syncthreads();  // every wave is past its last tile: smem is free
        if (__ballot(probe != 0) && lane == 0) shared[2] = 1;
        __syncthreads();
        if (careful || uniform(shared[2]) == 0) break;
        __syncthreads();
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
    float* const part = (float*)smem;
#pragma unroll
    for (int jp = 0; jp < JP; ++jp) {
        if (jp > 0) __syncthreads();
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int d = 0; d < DB / JP; ++d)
                *(f32x4*)(part + (wave * ROWS + rb * 16 + col) * OST + d * 16 + grp * 4) = o[rb][jp * (DB / JP) + d];
        __syncthreads();
        constexpr int GR = DV / 8 / JP;  // granules of a row of this part
        for (int i = threadIdx.x; i < ROWS * GR; i += NTHREADS) {
            const int c = i / GR, g = i % GR;
            const int t = entries > 1 ? min((row0 + c) / a.rows, entries - 1) : 0;
            const Entry e = ents[t];
            const int r = row0 + c - t * a.rows;
            if (r >= e.rows * a.group) continue;
            float m = part_m[0][c];
#pragma unroll
            for (int w = 1; w < NWAVES; ++w) m = fmaxf(m, part_m[w][c]);
            const float use = m == -INFINITY ? 0.f : m;
            float l = 0, x[8] = {};
#pragma unroll
            for (int w = 0; w < NWAVES; ++w) {
                const float f = __builtin_amdgcn_exp2f(part_m[w][c] - use);
                l += part_l[w][c] * f;
                const float* const y = part + (w * ROWS + c) * OST + g * 8;
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] += y[j] * f;
            }
            const float inv = l > 0 ? 1 / l : l;  // no key: zeros
            const int token = e.row0 + r / a.group, h = head * a.group + r % a.group, at = (jp * GR + g) * 8;
            const float lse = l > 0 ? m + __builtin_amdgcn_logf(l) : l == 0 ? -INFINITY : l;
            if (a.splits > 1) {
                const int64_t i0 = ((int64_t)split * a.tokens + token) * (a.group * a.hkv) + h;
#pragma unroll
                for (int j = 0; j < 8; ++j) a.part_o[i0 * DV + at + j] = x[j] * inv;
                if (at == 0) a.part_lse[i0] = lse;
                continue;
            }
            bf16x8 res;
#pragma unroll
            for (int j = 0; j < 8; ++j) res[j] = (__bf16)(x[j] * inv);
            *(bf16x8*)(a.out + (int64_t)token * a.o_st + (int64_t)h * a.o_sh + at) = res;
            if (at == 0 && a.lse) a.lse[(int64_t)h * a.lse_sh + token] = lse * LN2;
        }
    }
}

// The parts of split lists, weighted by their sums: a thread 8 values of a row. Rows of no query
// block stay as they are.
template <int DV>
__global__ __launch_bounds__(NTHREADS) void merge_kernel(AttendArgs a) {
    constexpr int GR = DV / 8;
    const int hq = a.group * a.hkv;
    const Entry e = uniform(checked_entry(a.entries[blockIdx.x], a.query_block, a.tokens, a.segments));
    for (int i = (int)blockIdx.y * NTHREADS + (int)threadIdx.x; i < e.rows * hq * GR; i += (int)gridDim.y * NTHREADS) {
        const int g = i % GR, h = i / GR % hq, token = e.row0 + i / GR / hq;
        const int64_t i0 = (int64_t)token * hq + h, st = (int64_t)a.tokens * hq;
        // all parts' sums at once, then four parts' values at a time: one after the other, a token's 16 parts
        // take 16 latencies
        float part[MAX_SPLITS], m = -INFINITY;
#pragma unroll
        for (int s = 0; s < MAX_SPLITS; ++s) {
            const float v = a.part_lse[i0 + min(s, a.splits - 1) * st];
            part[s] = s < a.splits ? v : -INFINITY;
        }
#pragma unroll
        for (int s = 0; s < MAX_SPLITS; ++s) m = fmaxf(m, part[s]);
        const float use = m == -INFINITY ? 0.f : m;
        float l = 0, x[8] = {};
#pragma unroll
        for (int s0 = 0; s0 < MAX_SPLITS; s0 += 4) {
            if (s0 >= a.splits) break;
            f32x4 y[4][2];
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    y[s][j] = *(const f32x4*)(a.part_o + (i0 + min(s0 + s, a.splits - 1) * st) * DV + g * 8 + j * 4);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const float f = __builtin_amdgcn_exp2f(part[s0 + s] - use);
                l += f;
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] += f == 0 ? 0 : y[s][j / 4][j % 4] * f;
            }
        }
        const float inv = l > 0 ? 1 / l : l;
        bf16x8 res;
#pragma unroll
        for (int j = 0; j < 8; ++j) res[j] = (__bf16)(x[j] * inv);
        *(bf16x8*)(a.out + (int64_t)token * a.o_st + (int64_t)h * a.o_sh + g * 8) = res;
        if (g == 0 && a.lse) a.lse[(int64_t)h * a.lse_sh + token] = (l > 0 ? m + __builtin_amdgcn_logf(l) : l == 0 ? -INFINITY : l) * LN2;
    }
}

// How a launch is cut up: query blocks of a workgroup, workgroups of a query block's rows, parts of the lists.
struct Cut {
    int rb, rows, pack, chunks, splits;
};
Cut cut_of(const vpp_block_attn_config_t& c, int64_t num_query_blocks) {
    Cut u;
    u.rows = c.num_q_heads / c.num_kv_heads * c.query_block;
    u.rb = u.rows <= 16 ? 1 : u.rows <= 32 ? 2 : 4;
    u.pack = 1;
    // Several short query blocks share a workgroup, and the blocks that they list in common, while there are
    // two workgroups a CU left.
    // (32 columns: two workgroups run on a CU. 4096 tokens of 32/8 heads, 16 blocks each: 640 us, in 16 columns
    // 744, in 64, which read the least but run one a CU, 1097.)
    for (int rb = 2; rb >= 1 && u.rows <= 16; rb /= 2) {
        const int pack = 16 * rb / u.rows < MAX_PACK ? 16 * rb / u.rows : MAX_PACK;
        if (pack < 2 || pack * c.max_blocks > MAX_ELEMENTS || num_query_blocks * c.num_kv_heads / pack < 512) continue;
        u.pack = pack;
        u.rb = (pack * u.rows + 15) / 16;
        break;
    }
    u.chunks = u.pack > 1 ? 1 : (u.rows + 16 * u.rb - 1) / (16 * u.rb);
    // Few workgroups split their lists, down to two tiles a wave (a token of 32/8 heads, 64 blocks: 12 us with
    // the merge, one workgroup a head alone goes through 32 tiles a wave).
    const int64_t wgs = (num_query_blocks + u.pack - 1) / u.pack * u.chunks * c.num_kv_heads;
    const int64_t tiles = (int64_t)c.max_blocks * (c.block_size / BT), most = tiles / (2 * NWAVES);
    int64_t s = wgs > 0 && wgs < 256 ? (512 + wgs - 1) / wgs : 1;
    if (s > most) s = most;
    u.splits = (int)(s < 1 ? 1 : s > MAX_SPLITS ? MAX_SPLITS : s);
    return u;
}

}  // namespace

extern "C" vpp_status_t vpp_block_attn_workspace(const vpp_block_attn_config_t* cfg, int32_t num_query_blocks,
                                                 int32_t num_tokens, size_t* bytes) {
    const vpp_status_t st = check_config(cfg);
    if (st != VPP_OK) return st;
    if (num_query_blocks < 0 || num_tokens < 0 || !bytes) return VPP_ERR_INVALID_ARG;
    const int splits = cut_of(*cfg, num_query_blocks).splits;
    *bytes = splits > 1 ? (size_t)splits * num_tokens * cfg->num_q_heads * (cfg->head_dim_v + 1) * 4 : 0;
    return VPP_OK;
}

namespace {
template <int DQK, int DV>
auto pick_attend(int rb, bool pack) {
    return rb == 1 ? attend_kernel<DQK, DV, 1, false> : rb == 4 ? attend_kernel<DQK, DV, 4, false>
           : pack ? attend_kernel<DQK, DV, 2, true> : attend_kernel<DQK, DV, 2, false>;
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
        !rows_apart(o_st, num_tokens, o_sh, hq, dv) ||
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
    const Cut cut = cut_of(*cfg, num_query_blocks);
    a.pack = cut.pack;
    a.rows = cut.rows;
    a.chunks = cut.chunks;
    a.splits = cut.splits;
    if (a.splits > 1) {
        const size_t need = (size_t)a.splits * num_tokens * hq * (dv + 1) * 4;
        if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need) return VPP_ERR_WORKSPACE;
        a.part_o = (float*)workspace;
        a.part_lse = a.part_o + (size_t)a.splits * num_tokens * hq * dv;
    }
    const int64_t items = (int64_t)((num_query_blocks + a.pack - 1) / a.pack) * a.chunks * a.splits, grid = items * hkv;
    if (grid >= ((int64_t)1 << 31)) return VPP_ERR_INVALID_ARG;
    // (8 of 16 heads at a time: query blocks of 64, 64 blocks each 606 us, all at once 617; 1024 tokens, 32 blocks
    // each 551, all at once 584.)
    a.heads = hkv % 8 == 0 ? 8 : hkv;
    a.items = (int32_t)items;
    const int resident = cut.rb == 4 || dqk == 192 ? 256 : 512;  // one or two workgroups a CU
    a.generation = resident > a.heads ? resident / a.heads : 1;
    const size_t lds = (size_t)a.pack * a.max_blocks * (sizeof(Element) + (a.pack > 1 ? 8 : 4)) + 8;
    auto* kernel = dqk == 64 ? pick_attend<64, 64>(cut.rb, a.pack > 1) : dqk == 128 ? pick_attend<128, 128>(cut.rb, a.pack > 1) : pick_attend<192, 128>(cut.rb, a.pack > 1);
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(NTHREADS), lds, (hipStream_t)stream, a);
    if (hipGetLastError() != hipSuccess) return VPP_ERR_HIP;
    if (a.splits > 1) {
        const int per = cfg->query_block * hq * (dv / 8), y = (per + NTHREADS - 1) / NTHREADS;
        auto* merge = dv == 64 ? merge_kernel<64> : merge_kernel<128>;
        hipLaunchKernelGGL(merge, dim3((unsigned)num_query_blocks, (unsigned)(y < 256 ? y : 256)), dim3(NTHREADS), 0, (hipStream_t)stream, a);
        if (hipGetLastError() != hipSuccess) return VPP_ERR_HIP;
    }
    return VPP_OK;
}
