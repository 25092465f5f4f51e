// vpp_block_select.hip -- block summaries and block selection for MI355X (gfx950): what precedes the
// attention of vpp_block_attn.hip.
#include "vpp_block_common.h"

namespace {

// ---------------------------------------------------------------------------------------------
// summaries
// ---------------------------------------------------------------------------------------------
struct SummarizeArgs {
    const u16* k;
    u16* summaries;
    const int64_t* blocks;
    int64_t k_sp, k_st, k_sh;
    int64_t total;  // blocks of the cache
    int32_t hkv, block, per_page_shift;
};

// One workgroup a (block, kv head). Bound by HBM: the keys are read once, 16 bytes a load; a
// thread sums 8 dims of every RS-th row in 64 bits, which is exact for keys within 2^37 of the
// largest, so the order of the sum does not show. 8192 new rows of 128 heads, dqk 192, 409 MB: 77 us,
// 5.3 TB/s; few blocks are one latency of the rows after the launch (64 of 8 heads: 4 us).
template <int DQK>
__global__ __launch_bounds__(NTHREADS) void summarize_kernel(SummarizeArgs a) {
    constexpr int GR = DQK / 8, RS = NTHREADS / GR;  // granules of a row, rows at a time
    __shared__ double part[RS][DQK];
    __shared__ float top[NWAVES];
    const int head = (int)blockIdx.x % a.hkv, n = (int)blockIdx.x / a.hkv;
    const int64_t block = a.blocks[n];
    if (block < 0 || block >= a.total) return;
    const int64_t page = block >> a.per_page_shift;
    const int row0 = (int)(block & ((1 << a.per_page_shift) - 1)) * a.block;
    const u16* const base = a.k + page * a.k_sp + (int64_t)row0 * a.k_st + (int64_t)head * a.k_sh;
    const int g = (int)threadIdx.x % GR, r0 = (int)threadIdx.x / GR;
    if (r0 < RS) {
        double sum[8] = {};
        for (int r = r0; r < a.block; r += RS) {
            const bf16x8 x = *(const bf16x8*)(base + (int64_t)r * a.k_st + g * 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += (double)(float)x[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) part[r0][g * 8 + i] = sum[i];
    }
    __syncthreads();
    const int d = (int)threadIdx.x;
    double mean = 0;
    if (d < DQK) {
#pragma unroll
        for (int r = 0; r < RS; ++r) mean += part[r][d];
        mean /= a.block;
        mean = mean == mean ? fmin(fmax(mean, -(double)GRID_MOST), (double)GRID_MOST) : 0;
    }
    // the exponent of the largest: of the mean as it is, or (rounded up to fp32) no smaller
    float m = __double2float_rz(fabs(mean));  // the same power of two below
#pragma unroll
    for (int s = 1; s < 64; s *= 2) m = fmaxf(m, __shfl_xor(m, s));
    if (d % 64 == 0) top[d / 64] = m;
    __syncthreads();
    m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    const int e = max(m > 0 ? ilogbf(m) + 1 : GRID_MIN_EXP, GRID_MIN_EXP);
    if (d < DQK) {
        const double v = ldexp(rint(ldexp(mean, 8 - e)), e - 8);
        const __bf16 r = (__bf16)(float)v;  // exact: 8 bits
        a.summaries[(block * a.hkv + head) * DQK + d] = __builtin_bit_cast(u16, r);
    }
}

// ---------------------------------------------------------------------------------------------
// selection
// ---------------------------------------------------------------------------------------------
constexpr int MAX_ENTRIES = 64;                // query blocks of a workgroup
constexpr int64_t SCORE_BYTES = 256ll << 20;  // scores of one slab of query blocks: what the last-level cache holds
constexpr int LISTS = 4;                       // lists of a workgroup, where a wave takes one

struct SelectArgs {
    const u16* q;
    const u16* summaries;
    const vpp_query_block_t* entries;  // of the slab
    float* scores;                     // [query blocks][hkv][cap]
    int32_t* lists;
    int64_t q_st, q_sh;
    Pages pages;
    int32_t num_entries, tokens, segments, query_block, group, hkv;
    int32_t block_shift, sink, local, max_blocks, cap;  // cap: blocks that the scores have room for
    int32_t wg_entries, rows;                           // query blocks of a workgroup; MFMA rows of one
    int32_t wgs, splits;                                // workgroups of a kv head; that share the blocks
};

// Blocks [lo, hi) of a query block compete for its list; last: that of its last token. Returns how
// many of them are wanted (0: none compete).
__device__ __forceinline__ int contest(const SelectArgs& a, const Entry& e, int& lo, int& hi, int& last) {
    lo = hi = 0, last = -1;
    if (e.rows == 0) return 0;
    last = min((e.pos0 + e.rows - 1) >> a.block_shift, a.cap - 1);
    const int l = a.sink, h = min((e.pos0 >> a.block_shift) - a.local + 1, last + 1);
    if (h <= l || last + 1 <= a.max_blocks) return 0;  // nothing to choose
    lo = l, hi = h;
    return a.max_blocks - (last + 1 - (hi - lo));
}

// A score as an unsigned number of the same order, at least 1.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);  // -0 becomes 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Workgroup -> (kv head, workgroup of that head). Workgroups go to the 8 XCDs in turn: those of a head
// stay on one XCD, one head after the other, so that the summaries they share stay in its L2.
__device__ __forceinline__ void place(int wg, int hkv, int wgs, int& head, int& index) {
    if (hkv % 8 == 0) {
        const int i = wg / 8;
        head = wg % 8 + 8 * (i / wgs);
        index = i % wgs;
    } else {
        head = wg % hkv;
        index = wg / hkv;
    }
}

// The largest over a wave's lanes, in all of them.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    auto dpp = [&](auto ctrl) {
        x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, decltype(ctrl)::value, 0xf, 0xf, true));
    };
    dpp(std::integral_constant<int, 0xB1>());   // pairs
    dpp(std::integral_constant<int, 0x4E>());   // quads
    dpp(std::integral_constant<int, 0x141>());  // halves of a row of 16, mirrored
    dpp(std::integral_constant<int, 0x140>());  // rows, mirrored
    auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(r[0], r[1]);
    r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return max(r[0], r[1]);
}

// A list, from the scores x of its blocks: the blocks before the contested ones, the wanted ones of
// those, of equal scores the first, and the blocks behind them. The smallest key that is in is
// found bit by bit: first down the exponents from the largest key's (the wanted ones are few of many, so
// nearly always within a few), then the mantissa, and no further than until as many keys as wanted are
// at least that large: about 10 counts where 32 are needed bit by bit. The keys are held in
// registers, KR a lane, of one wave, or of the NW waves of a workgroup, which add up their counts in LDS.
// Bound by the counts, a compare and a ballot a register each: 32768 lists of up to 512 blocks 32 us.
template <int NW, int KR>
struct ListShared {
    int counts[48], above[NW], same[NW];
};
template <int NW, int KR>
__device__ __forceinline__ void make_list(const SelectArgs& a, const Entry& e, const float* x, int32_t* list, ListShared<NW, KR>& sh) {
    const int lane = (int)threadIdx.x & 63, wave = NW == 1 ? 0 : uniform((int)threadIdx.x >> 6);
    int lo, hi, last;
    const int want = contest(a, e, lo, hi, last);
    const int n = last + 1 - (hi - lo) + want;  // entries of the list
    for (int i = wave * 64 + lane; i < a.max_blocks; i += NW * 64)
        if (i < lo || i >= lo + want) list[i] = i >= n ? -1 : i < lo ? i : i - lo - want + hi;
    if (want <= 0) return;
    if constexpr (NW > 1) {
        if (threadIdx.x < 48) sh.counts[threadIdx.x] = 0;
        __syncthreads();
    }
    const int base = lo + wave * KR * 64 + lane;
    uint32_t key[KR];
#pragma unroll
    for (int r = 0; r < KR; ++r) {
        const float v = x[min(base + r * 64, hi - 1)];
        key[r] = base + r * 64 < hi ? order_key(v) : 0;  // 0: in no count
    }
    const int regs = NW == 1 ? (hi - lo + 63) / 64 : KR;
    int turn = 0;
    auto of_all = [&](int c) {  // a count over the waves
        if constexpr (NW == 1) return c;
        if (lane == 0 && c) atomicAdd(&sh.counts[turn], c);
        __syncthreads();
        return uniform(sh.counts[turn++]);
    };
    auto at_least = [&](uint32_t t) {
        int c = 0;
#pragma unroll
        for (int r = 0; r < KR; ++r) c += count(__ballot(key[r] >= t));
        return of_all(c);
    };
    uint32_t least = 1;
    bool exact = true;  // all keys from `least` on are in
    int equal = 0;      // else: how many of those equal to it
    if (hi - lo > want) {
        uint32_t top = 0;
#pragma unroll
        for (int r = 0; r < KR; ++r) top = max(top, key[r]);
        top = (uint32_t)uniform((int)wave_max(top));
        if constexpr (NW > 1) {
            if (lane == 0) atomicMax((uint32_t*)&sh.counts[47], top);
            __syncthreads();
            top = (uint32_t)uniform(sh.counts[47]);
        }
        top &= ~0x7fffffu;
        int bit = 31, c = 0;
        least = 0;
        for (int i = 0; i < 4 && top >= 0x800000u; ++i, top -= 0x800000u) {
            c = at_least(top);
            if (c < want) continue;
            least = top;
            bit = 22;
            break;
        }
        if (c != want)
            for (; bit >= 0; --bit) {
                const uint32_t t = least | 1u << bit;
                c = at_least(t);
                if (c >= want) least = t;
                if (c == want) break;
            }
        exact = c == want;
        if (!exact) equal = want - (least == ~0u ? 0 : at_least(least + 1));
    }
    auto before = [](uint64_t mask) {  // lanes of it below this one
        return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
    };
    int rank = lo;
    if constexpr (NW > 1) {  // the entries and the equal keys of the waves before
        int c = 0, s = 0;
#pragma unroll
        for (int r = 0; r < KR; ++r) {
            c += count(__ballot(exact ? key[r] >= least : key[r] > least));
            s += count(__ballot(key[r] == least));
        }
        if (lane == 0) sh.above[wave] = c, sh.same[wave] = s;
        __syncthreads();
        for (int w = 0; w < wave; ++w) {
            rank += sh.above[w] + (exact ? 0 : min(sh.same[w], max(equal, 0)));
            equal -= sh.same[w];
        }
        rank = uniform(rank);
        equal = uniform(equal);
    }
#pragma unroll
    for (int r = 0; r < KR; ++r) {
        if (NW == 1 && r >= regs) continue;
        const uint32_t k = key[r];
        bool in = k >= least && k != 0;
        if (!exact) {
            const uint64_t ties = __ballot(k == least);
            in = k > least || (k == least && before(ties) < equal);
            equal -= count(ties);
        }
        const uint64_t all = __ballot(in);
        if (in) list[rank + before(all)] = base + r * 64;
        rank += count(all);
    }
}

// NW = 1: a wave a list, LISTS of them a workgroup.
template <int NW, int KR>
__global__ __launch_bounds__(64 * (NW == 1 ? LISTS : NW)) void list_kernel(SelectArgs a) {
    __shared__ ListShared<NW, KR> sh;
    const int64_t item = NW == 1 ? (int64_t)blockIdx.x * LISTS + uniform((int)threadIdx.x >> 6) : blockIdx.x;
    if (item >= (int64_t)a.num_entries * a.hkv) return;  // (NW > 1: never)
    const Entry e = uniform(checked_entry(a.entries[item / a.hkv], a.query_block, a.tokens, a.segments));
    make_list<NW, KR>(a, e, a.scores + item * a.cap, a.lists + item * a.max_blocks, sh);
}

// Scores of a workgroup's query blocks: MFMA tiles of 16 query rows x 16 blocks. MT row tiles are held
// in registers as A operands, on their grid; the waves share the blocks, whose summaries come
// straight from memory as B operands, NT tiles ahead. Rows of a query block start on a power of two
// up to 16 or a multiple of 16, and those past its last repeat it. RM: rows of a query block, 1
// (one or two), 4 (or 8), 16, 32, 64, 128 (with eight tiles), 48 (any other above 16, or 128 with four). WHOLE: one query block a workgroup, its scores go to LDS, and
// the workgroup makes its list.
// Products of two 8-bit grids are whole multiples of a step and their sums stay below 2^24 of them, so fp32
// holds every sum exactly, whatever the order: lists do not depend on tiles, splits or slabs.
// Bound by the matrix unit and, one or two waves a SIMD, by what runs beside it: maxima, and moves of scalars
// that do not fit the registers. 16384 rows in query blocks of 64, 16 heads, dqk 192, behind 508K: 1.2
// ms, 674 TFLOP/s; 4096 tokens of 32/8 heads behind 28672, a list each: 73 us.
constexpr int WHOLE_BLOCKS = 2048;
template <int DQK, int MT, int NT, int RM, bool WHOLE>
__global__ __launch_bounds__(NTHREADS) void score_kernel(SelectArgs a) {
    constexpr int KS = DQK / 32;  // MFMA steps of a product
    constexpr bool PACKED = RM == 16 && MT % 4 == 0;
    __shared__ Entry ents[WHOLE ? 1 : MAX_ENTRIES];
    __shared__ float own[WHOLE ? WHOLE_BLOCKS : 1];
    __shared__ ListShared<NWAVES, WHOLE_BLOCKS / NTHREADS> sh;
    const int lane = (int)threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    int head, wg;
    place((int)blockIdx.x, a.hkv, a.wgs * a.splits, head, wg);
    const int split = wg % a.splits, entry0 = wg / a.splits * a.wg_entries;
    const int entries = min(a.wg_entries, a.num_entries - entry0);
    const int col = lane & 15, grp = lane >> 4;
    if ((int)threadIdx.x < entries)
        ents[threadIdx.x] = checked_entry(a.entries[entry0 + threadIdx.x], a.query_block, a.tokens, a.segments);
    __syncthreads();
    const Entry mine = ents[min(lane, entries - 1)];  // lane i: query block i
    const int tiles = (entries * a.rows + 15) / 16;
    const int64_t entry_st = (int64_t)a.hkv * a.cap;
    float* const scores = WHOLE ? own : a.scores + (int64_t)entry0 * entry_st + (int64_t)head * a.cap;
    for (int done = 0; done < entries;) {
        // the next query blocks of one segment, [first, done), and the blocks that compete for their lists
        const int first = done;
        const int segment = __builtin_amdgcn_readlane(mine.segment, first);
        const uint64_t other = __ballot(lane >= first && mine.segment != segment);
        done = min(other ? (int)__builtin_ctzll(other) : 64, entries);
        int l = 0, h = 0, last;
        if (lane >= first && lane < done) contest(a, mine, l, h, last);
        const int all = uniform((int)wave_max((uint32_t)h));  // (none compete: 0)
        if (all <= a.sink) continue;
        const int kv_start = __builtin_amdgcn_readlane(mine.kv_start, (int)__builtin_ctzll(__ballot(h > l)));
        constexpr int STEP = NWAVES * NT * 16;  // blocks of the workgroup's waves at a time
        // this workgroup's share of them, whole steps
        const int steps = (all - a.sink + STEP - 1) / STEP, share = (steps + a.splits - 1) / a.splits * STEP;
        const int lo = a.sink + split * share, hi = min(all, lo + share);
        if (hi <= lo) continue;
        const u16* const sums = a.summaries + (int64_t)head * DQK + grp * 8;
        const int in_page = (1 << (a.pages.page_shift - a.block_shift)) - 1, block0 = kv_start >> a.block_shift;
        auto page_of = [&](int b) { return a.pages.page(segment, (block0 + min(b, hi - 1)) << a.block_shift); };
        auto load = [&](bf16x8 (&to)[KS], int b, int page) {
            const int at = (block0 + min(b, hi - 1)) & in_page;
            const u16* const p = sums + (((int64_t)page << (a.pages.page_shift - a.block_shift)) + at) * (a.hkv * DQK);
#pragma unroll
            for (int s = 0; s < KS; ++s) to[s] = *(const bf16x8*)(p + s * 32);
        };
        const int mt_begin = first * a.rows / 16, mt_end = min((done * a.rows + 15) / 16, tiles);
        for (int mt0 = mt_begin; mt0 < mt_end; mt0 += MT) {
            // the first blocks' pages and summaries travel with the query rows
            const int b0 = lo + wave * NT * 16 + col;
            int page[NT];
            bf16x8 kf[2][NT][KS], qf[MT][KS];
#pragma unroll
            for (int n = 0; n < NT; ++n) page[n] = page_of(b0 + n * 16);
            // Where a lane's score of row tile m goes (< 0: nowhere): to its rows' query block, or, where
            // the maxima of four tiles are taken together, lane group g has those of tile 4 (m / 4) + g.
            int entry[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int slot = (mt0 + m) * 16 + col;
                const Entry e = ents[min(slot / a.rows, entries - 1)];
                const int r = min(slot % a.rows, max(e.rows * a.group - 1, 0));  // rows past the last repeat it
                const int token = min(e.row0 + r / a.group, a.tokens - 1);
                const u16* const p = a.q + (int64_t)token * a.q_st + (int64_t)(head * a.group + r % a.group) * a.q_sh + grp * 8;
#pragma unroll
                for (int s = 0; s < KS; ++s) qf[m][s] = *(const bf16x8*)(p + s * 32);
                entry[m] = (PACKED ? (mt0 + m / 4 * 4 + grp) * 16 : (mt0 + m) * 16 + grp * 4) / a.rows;
                if (entry[m] < first || entry[m] >= done) entry[m] = -1;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) load(kf[0][n], b0 + n * 16, page[n]);
#pragma unroll
            for (int n = 0; n < NT; ++n) page[n] = page_of(b0 + STEP + n * 16);
            // query rows on their grid, as A operands
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                float top = 0;
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float v = fabsf((float)qf[m][s][i]);
                        top = v == v ? fmaxf(top, v) : top;
                    }
                top = fminf(max_xor32(max_xor16(top)), GRID_MOST);
                const int e = max(top > 0 ? ilogbf(top) + 1 : GRID_MIN_EXP, GRID_MIN_EXP);
                const float up = ldexpf(1.f, 8 - e), down = ldexpf(1.f, e - 8);
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float v = (float)qf[m][s][i];
                        qf[m][s][i] = (__bf16)(v == v ? rintf(fminf(fmaxf(v, -GRID_MOST), GRID_MOST) * up) * down : 0.f);
                        if (i == 7) __builtin_amdgcn_sched_barrier(0);  // few values at a time: registers
                    }
            }
            // A tile's largest scores are taken while the products of the next one run.
            auto put = [&](int ei, int block, float v) { scores[ei * entry_st + block] = v; };
            auto take = [&](const f32x4 (&d)[MT], int block) {  // d[m][i]: row (mt0 + m) * 16 + grp * 4 + i
                if constexpr (RM == 1) {
                    const int apart = a.rows == 1 ? 1 : 2;
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int i = 0; i < 4; i += 1) {
                            const int ei = ((mt0 + m) * 16 + grp * 4 + i) / apart;
                            const float v = apart == 1 ? d[m][i] : max_finite(d[m][i], d[m][i ^ 1]);
                            if (ei >= first && ei < done && i % apart == 0) put(ei, block, v);
                        }
                    return;
                }
                float v[MT];
#pragma unroll
                for (int m = 0; m < MT; ++m) v[m] = max_finite(max_finite(d[m][0], d[m][1]), max_finite(d[m][2], d[m][3]));
                if constexpr (PACKED) {
                    // maxima over the lane groups of four tiles at once: swapping rows of 16 lanes between two
                    // tiles' values, then halves of the wave, leaves tile g's maximum in lane group g
                    auto both = [](float x, float y, auto swap) {
                        const auto r = swap(__float_as_uint(x), __float_as_uint(y));
                        return max_finite(__uint_as_float(r[0]), __uint_as_float(r[1]));
                    };
                    auto swap16 = [](uint32_t x, uint32_t y) { return __builtin_amdgcn_permlane16_swap(x, y, false, false); };
                    auto swap32 = [](uint32_t x, uint32_t y) { return __builtin_amdgcn_permlane32_swap(x, y, false, false); };
#pragma unroll
                    for (int m = 0; m < MT; m += 4) {
                        const float x = both(both(v[m], v[m + 1], swap16), both(v[m + 2], v[m + 3], swap16), swap32);
                        if (entry[m] >= 0) put(entry[m], block, x);
                    }
                } else if constexpr (RM > 16 && RM != 48) {
                    // RM / 16 tiles, which are always of one pass: no branch on their number beside the products
                    // (16384 rows in query blocks of 64: 1341 us with the one below, so 1291)
                    constexpr int per = RM / 16;
#pragma unroll
                    for (int m = 0; m < MT; m += per) {
                        float x = v[m];
#pragma unroll
                        for (int i = 1; i < per; ++i) x = max_finite(x, v[m + i]);
                        x = max_xor32<true>(max_xor16<true>(x));
                        if (grp == 0 && entry[m] >= 0) put(entry[m], block, x);
                    }
                } else if constexpr (RM == 48) {
                    // several tiles to a query block; what its earlier ones left in memory counts (only the lane
                    // whose block it is reads and writes it: the waves are not at the same tiles)
                    const int per = a.rows / 16;
                    float x = -INFINITY;
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        x = max_finite(x, v[m]);
                        if (m + 1 < MT && (mt0 + m + 1) % per != 0) continue;
                        x = max_xor32<true>(max_xor16<true>(x));
                        if (grp == 0 && entry[m] >= 0 && block < hi) {
                            if (mt0 / per == (mt0 + m) / per && mt0 % per != 0) x = max_finite(x, scores[entry[m] * entry_st + block]);
                            put(entry[m], block, x);
                        }
                        x = -INFINITY;
                    }
                } else {
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        const float x = max_xor16<true>(v[m]);
                        v[m] = a.rows >= 8 ? x : v[m];
                        if constexpr (RM == 16) v[m] = max_xor32<true>(v[m]);
                    }
                    if (RM == 16 ? grp == 0 : a.rows == 4 || grp % 2 == 0)
#pragma unroll
                        for (int m = 0; m < MT; ++m)
                            if (entry[m] >= 0) put(entry[m], block, v[m]);
                }
            };
            f32x4 d[2][MT];
            int block[2] = {-1, -1};
            auto tile = [&](const bf16x8 (&k)[KS], f32x4 (&now)[MT], const f32x4 (&then)[MT], int then_block) {
#pragma unroll
                for (int m = 0; m < MT; ++m) now[m] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int m = 0; m < MT; ++m) now[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[m][s], k[s], now[m], 0, 0, 0);
                if (then_block >= 0) take(then, then_block);
                if constexpr (PACKED || RM > 16) {
#pragma unroll
                    for (int i = 0; i < KS * MT; ++i) {  // a product, then 2 of the maxima's operations
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
                    }
                }
            };
            // NT tiles at blocks b, from one buffer, while the next ones come into the other: their pages are
            // here; the pages of those behind them are asked for after, so that the wait for a page is
            // not one for a load issued just before. D: which of d the first tile writes.
            auto step = [&](auto BUF, auto D, int b) {
                constexpr int buf = decltype(BUF)::value, d0 = decltype(D)::value;
#pragma unroll
                for (int n = 0; n < NT; ++n) load(kf[1 - buf][n], b + STEP + n * 16, page[n]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int n = 0; n < NT; ++n) page[n] = page_of(b + 2 * STEP + n * 16);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int now = (d0 + n) % 2;
                    tile(kf[buf][n], d[now], d[1 - now], block[1 - now]);
                    // past the last: its score again, the same (but RM = 48, which leaves them out)
                    block[now] = RM == 48 ? b + n * 16 : min(b + n * 16, hi - 1);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            typedef std::integral_constant<int, 0> zero;
            typedef std::integral_constant<int, 1> one;
            bool odd = false;  // the last scores are in d[0]
#pragma unroll 1
            for (int b = b0;; b += 2 * STEP) {
                step(zero(), zero(), b);
                odd = NT % 2 == 1;
                if (b + STEP - col >= hi) break;
                step(one(), std::integral_constant<int, NT % 2>(), b + STEP);
                odd = false;
                if (b + 2 * STEP - col >= hi) break;
            }
            if (odd) take(d[0], block[0]);
            else take(d[1], block[1]);
        }
    }
    if constexpr (WHOLE) {
        __syncthreads();
        const Entry e = uniform(ents[0]);
        int32_t* const list = a.lists + ((int64_t)entry0 * a.hkv + head) * a.max_blocks;
        if (a.cap > 1024) {
            make_list<NWAVES, WHOLE_BLOCKS / NTHREADS>(a, e, own, list, sh);
        } else if (wave == 0) {  // one wave alone needs no barriers: 2.5 us less at 513 blocks
            ListShared<1, 16> none;
            make_list<1, 16>(a, e, own, list, none);
        }
    }
}

}  // namespace

extern "C" vpp_status_t vpp_query_blocks(int32_t num_segments, const int32_t* cu_q, const int64_t* kv_start,
                                         const int64_t* prefix_len, int32_t query_block, int32_t block_size,
                                         vpp_query_block_t* blocks, int32_t capacity, int32_t* count) {
    if (num_segments < 0 || !cu_q || !count || capacity < 0 || (capacity > 0 && !blocks)) return VPP_ERR_INVALID_ARG;
    if (query_block < 1 || query_block > 128 || (block_size != 64 && block_size != 128 && block_size != 256))
        return VPP_ERR_INVALID_ARG;
    if (num_segments > 0 && (!kv_start || !prefix_len)) return VPP_ERR_INVALID_ARG;
    if (cu_q[0] != 0) return VPP_ERR_INVALID_ARG;
    int32_t n = 0;
    for (int s = 0; s < num_segments; ++s) {
        const int64_t len = (int64_t)cu_q[s + 1] - cu_q[s];
        if (len < 0 || kv_start[s] < 0 || prefix_len[s] < 0 || kv_start[s] % block_size) return VPP_ERR_INVALID_ARG;
        const int64_t most = INT32_MAX - 256;
        if (kv_start[s] > most || prefix_len[s] > most || kv_start[s] + prefix_len[s] + len > most) return VPP_ERR_INVALID_ARG;
        for (int64_t r = 0; r < len; r += query_block, ++n)
            if (n < capacity)
                blocks[n] = vpp_query_block_t{(int32_t)(cu_q[s] + r), (int32_t)(len - r < query_block ? len - r : query_block), s,
                                              (int32_t)(prefix_len[s] + r), (int32_t)kv_start[s], {0, 0, 0}};
    }
    *count = n;
    return VPP_OK;
}

extern "C" vpp_status_t vpp_completed_blocks(int32_t num_segments, const int32_t* cu_q, const int64_t* kv_start,
                                             const int64_t* prefix_len, const int32_t* block_table,
                                             int64_t block_table_stride, int32_t pages_per_row, int32_t page_size,
                                             int32_t block_size, int64_t* blocks, int32_t capacity, int32_t* count) {
    if (num_segments < 0 || !cu_q || !count || capacity < 0 || (capacity > 0 && !blocks)) return VPP_ERR_INVALID_ARG;
    if ((block_size != 64 && block_size != 128 && block_size != 256) || !page_ok(page_size, 1, block_size))
        return VPP_ERR_INVALID_ARG;
    if (num_segments > 0 && (!kv_start || !prefix_len || !block_table)) return VPP_ERR_INVALID_ARG;
    if (pages_per_row < 0 || block_table_stride < 0 || cu_q[0] != 0) return VPP_ERR_INVALID_ARG;
    int32_t n = 0;
    for (int s = 0; s < num_segments; ++s) {
        const int64_t len = (int64_t)cu_q[s + 1] - cu_q[s];
        if (len < 0 || kv_start[s] < 0 || prefix_len[s] < 0 || kv_start[s] % block_size) return VPP_ERR_INVALID_ARG;
        const int64_t most = INT32_MAX - 256;
        if (kv_start[s] > most || prefix_len[s] > most || kv_start[s] + prefix_len[s] + len > most) return VPP_ERR_INVALID_ARG;
        const int64_t first = prefix_len[s] / block_size, last = (prefix_len[s] + len) / block_size;
        for (int64_t b = first; b < last; ++b, ++n) {
            const int64_t row = kv_start[s] + b * block_size, idx = row / page_size;
            if (idx >= pages_per_row) return VPP_ERR_INVALID_ARG;
            const int32_t page = block_table[(int64_t)s * block_table_stride + idx];
            if (page < 0) return VPP_ERR_INVALID_ARG;
            if (n < capacity) blocks[n] = (int64_t)page * (page_size / block_size) + row % page_size / block_size;
        }
    }
    *count = n;
    return VPP_OK;
}

extern "C" vpp_status_t vpp_block_summarize_paged(const vpp_block_attn_config_t* cfg, const void* k_pages, int64_t k_sp,
                                                  int64_t k_st, int64_t k_sh, int32_t page_size, int32_t num_pages,
                                                  const int64_t* blocks, int32_t num_blocks, void* summaries, void* stream) {
    const vpp_status_t st = check_config(cfg);
    if (st != VPP_OK) return st;
    if (num_blocks < 0 || !page_ok(page_size, num_pages, cfg->block_size)) return VPP_ERR_INVALID_ARG;
    if (num_blocks == 0) return VPP_OK;
    if (!k_pages || !blocks || !summaries || !aligned16(k_pages) || !aligned16(summaries) || ((uintptr_t)blocks & 7u))
        return VPP_ERR_INVALID_ARG;
    const int hkv = cfg->num_kv_heads;
    if (!strides_ok(k_st, page_size, (int64_t)1 << 31, k_sh, hkv, cfg->head_dim_qk) || (num_pages > 1 && !stride_ok(k_sp))) return VPP_ERR_INVALID_ARG;
    if ((int64_t)num_blocks * hkv >= ((int64_t)1 << 31)) return VPP_ERR_INVALID_ARG;
    SummarizeArgs a{};
    a.k = (const u16*)k_pages;
    a.summaries = (u16*)summaries;
    a.blocks = blocks;
    a.k_sp = k_sp; a.k_st = k_st; a.k_sh = k_sh;
    a.per_page_shift = log2_of(page_size / cfg->block_size);
    a.total = (int64_t)num_pages << a.per_page_shift;
    a.hkv = hkv;
    a.block = cfg->block_size;
    auto* kernel = cfg->head_dim_qk == 64 ? summarize_kernel<64> : cfg->head_dim_qk == 128 ? summarize_kernel<128> : summarize_kernel<192>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(num_blocks * hkv)), dim3(NTHREADS), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? VPP_OK : VPP_ERR_HIP;
}

namespace {
template <int DQK, int RM>
auto pick_rows(int mt) {  // 0: the whole selection
    auto* four = score_kernel<DQK, 4, 1, RM <= 64 ? RM : 48, false>;
    if constexpr (DQK == 192)
        if (mt == 8) return score_kernel<DQK, 8, 1, RM, false>;
    if constexpr (RM <= 16) {  // more rows than a tile has: never one tile
        if (mt == 1) return score_kernel<DQK, 1, 4, RM, false>;
        if (mt == 0) return score_kernel<DQK, 1, 4, RM, true>;
    }
    return four;
}
template <int DQK>
auto pick_score(int mt, int rows) {
    return rows < 4 ? pick_rows<DQK, 1>(mt) : rows < 16 ? pick_rows<DQK, 4>(mt) : rows == 16 ? pick_rows<DQK, 16>(mt)
           : rows == 32 ? pick_rows<DQK, 32>(mt) : rows == 64 ? pick_rows<DQK, 64>(mt)
           : rows == 128 && mt == 8 ? pick_rows<DQK, 128>(mt) : pick_rows<DQK, 48>(mt);
}

// Blocks that the scores of a chunk up to max_kv_len have room for, and the query blocks of a slab.
int64_t score_room(const vpp_block_attn_config_t& c, int64_t max_kv_len) {
    const int64_t cap = (max_kv_len + c.block_size - 1) / c.block_size;
    return cap < 1 ? 1 : cap;
}
int64_t slab_entries(const vpp_block_attn_config_t& c, int64_t cap, int64_t num_query_blocks) {
    int64_t n = SCORE_BYTES / (cap * c.num_kv_heads * 4);
    n = n < MAX_ENTRIES ? MAX_ENTRIES : n / MAX_ENTRIES * MAX_ENTRIES;
    return n < num_query_blocks ? n : num_query_blocks;
}
}  // namespace

extern "C" vpp_status_t vpp_block_select_workspace(const vpp_block_attn_config_t* cfg, int32_t num_query_blocks,
                                                   int64_t max_kv_len, size_t* bytes) {
    const vpp_status_t st = check_config(cfg);
    if (st != VPP_OK) return st;
    if (num_query_blocks < 0 || max_kv_len < 0 || !bytes) return VPP_ERR_INVALID_ARG;
    if (max_kv_len > (int64_t)MAX_CANDIDATES * cfg->block_size) return VPP_ERR_UNSUPPORTED;
    const int64_t cap = score_room(*cfg, max_kv_len);
    // every block fits the lists: no scores
    *bytes = cap <= cfg->max_blocks ? 0 : (size_t)(slab_entries(*cfg, cap, num_query_blocks) * cfg->num_kv_heads * cap * 4);
    return VPP_OK;
}

extern "C" vpp_status_t vpp_block_select_paged(const vpp_block_attn_config_t* cfg, const vpp_query_block_t* query_blocks,
                                               int32_t num_query_blocks, const void* q, int64_t q_st, int64_t q_sh,
                                               int32_t num_tokens, const void* summaries, int32_t page_size,
                                               int32_t num_pages, const int32_t* block_table, int64_t bt_st,
                                               int32_t num_segments, int32_t pages_per_row, int64_t max_kv_len,
                                               int32_t* blocks, void* workspace, size_t workspace_bytes, void* stream) {
    const vpp_status_t st = check_config(cfg);
    if (st != VPP_OK) return st;
    if (num_query_blocks < 0 || num_tokens < 0 || max_kv_len < 0 || !page_ok(page_size, num_pages, cfg->block_size))
        return VPP_ERR_INVALID_ARG;
    if (num_query_blocks == 0 || num_tokens == 0) return VPP_OK;
    if (!query_blocks || !q || !summaries || !blocks || !aligned16(query_blocks) || !aligned16(q) || !aligned16(summaries) ||
        ((uintptr_t)blocks & 3u) || !table_ok(block_table, bt_st, num_segments, pages_per_row))
        return VPP_ERR_INVALID_ARG;
    if (!strides_ok(q_st, num_tokens, (int64_t)1 << 31, q_sh, cfg->num_q_heads, cfg->head_dim_qk)) return VPP_ERR_INVALID_ARG;
    size_t need = 0;
    const vpp_status_t ws = vpp_block_select_workspace(cfg, num_query_blocks, max_kv_len, &need);
    if (ws != VPP_OK) return ws;
    if (need && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need)) return VPP_ERR_WORKSPACE;
    const int64_t cap = score_room(*cfg, max_kv_len);
    SelectArgs a{};
    a.q = (const u16*)q;
    a.summaries = (const u16*)summaries;
    a.scores = (float*)workspace;
    a.q_st = q_st;
    a.q_sh = q_sh;
    a.pages = Pages{block_table, bt_st, pages_per_row, num_pages, log2_of(page_size)};
    a.tokens = num_tokens;
    a.segments = num_segments;
    a.query_block = cfg->query_block;
    a.group = cfg->num_q_heads / cfg->num_kv_heads;
    a.hkv = cfg->num_kv_heads;
    a.block_shift = log2_of(cfg->block_size);
    a.sink = cfg->sink_blocks;
    a.local = cfg->local_blocks;
    a.max_blocks = cfg->max_blocks;
    a.cap = (int32_t)cap;
    const int rows = a.group * a.query_block;
    a.rows = rows <= 16 ? 1 << log2_of(rows) : (rows + 15) / 16 * 16;
    const int64_t slab = slab_entries(*cfg, cap, num_query_blocks);
    for (int64_t e0 = 0; e0 < num_query_blocks; e0 += slab) {
        a.num_entries = (int32_t)(num_query_blocks - e0 < slab ? num_query_blocks - e0 : slab);
        a.entries = query_blocks + e0;
        a.lists = blocks + e0 * a.hkv * a.max_blocks;
        if (need) {
            // Row tiles held at a time and query blocks of a workgroup: as many as fill the tiles, while the
            // launch still has two workgroups a CU; then the blocks are split, to four of them.
            // Eight tiles need a SIMD's registers for one wave. At dqk 192, where the products outweigh the
            // maxima, they are faster for the summaries that they read half as often (16384 rows of 16 heads
            // behind 508K: 1323 us, four tiles 1548); below, two waves of four tiles are (4096 rows of 32/8 heads
            // behind 28672: 98 us, one wave of eight 114).
            const int most = cfg->head_dim_qk == 192 ? 8 : 4;
            int mt = a.rows > 64 ? most : a.rows > 16 ? 4 : 1;
            a.wg_entries = 1;
            for (int m = most; m >= 4; m /= 2) {
                const int n = m * 16 / a.rows;
                if (n < 1 || n > MAX_ENTRIES || (int64_t)a.num_entries * a.hkv / n < 512) continue;
                mt = m;
                a.wg_entries = n;
                break;
            }
            a.wgs = (a.num_entries + a.wg_entries - 1) / a.wg_entries;
            const int64_t wgs = (int64_t)a.wgs * a.hkv, step = NWAVES * (mt == 1 ? 4 : 1) * 16, steps = (cap + step - 1) / step;
            const int64_t splits = wgs >= 1024 ? 1 : (1024 + wgs - 1) / wgs;
            a.splits = (int32_t)(splits < steps ? splits : steps);
            // Few lists of few blocks are made where their scores are (256 lists up to 513 blocks 12.8 us, in two
            // kernels 18.9), unless they are so few that the blocks are better split (8 of 1563 20.6, split 13.3).
            const bool whole = mt == 1 && cap <= WHOLE_BLOCKS && wgs >= 64;
            if (whole) mt = 0, a.splits = 1;
            if (wgs * a.splits >= ((int64_t)1 << 31)) return VPP_ERR_INVALID_ARG;
            auto* kernel = cfg->head_dim_qk == 64 ? pick_score<64>(mt, a.rows) : cfg->head_dim_qk == 128 ? pick_score<128>(mt, a.rows)
                                                                                                           : pick_score<192>(mt, a.rows);
            hipLaunchKernelGGL(kernel, dim3((unsigned)(wgs * a.splits)), dim3(NTHREADS), 0, (hipStream_t)stream, a);
            if (hipGetLastError() != hipSuccess) return VPP_ERR_HIP;
            if (whole) continue;
        }
        const int64_t lists = (int64_t)a.num_entries * a.hkv;
        if (lists >= ((int64_t)1 << 31)) return VPP_ERR_INVALID_ARG;
        if (cap <= 512)
            hipLaunchKernelGGL((list_kernel<1, 8>), dim3((unsigned)((lists + LISTS - 1) / LISTS)), dim3(64 * LISTS), 0, (hipStream_t)stream, a);
        else if (cap <= 2048)
            hipLaunchKernelGGL((list_kernel<4, 8>), dim3((unsigned)lists), dim3(256), 0, (hipStream_t)stream, a);
        else if (cap <= 8192)
            hipLaunchKernelGGL((list_kernel<4, 32>), dim3((unsigned)lists), dim3(256), 0, (hipStream_t)stream, a);
        else
            hipLaunchKernelGGL((list_kernel<16, 32>), dim3((unsigned)lists), dim3(1024), 0, (hipStream_t)stream, a);
        if (hipGetLastError() != hipSuccess) return VPP_ERR_HIP;
    }
    return VPP_OK;
}
