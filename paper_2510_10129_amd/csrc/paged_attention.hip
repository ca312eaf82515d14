// Causal grouped-query attention of new rows over a paged cache, optionally under a sliding window with sinks.
//
// Few rows (few_attn_kernel).  A sequence's new rows are a handful of (row, query head) columns per kv head, every key and
// value is read once, and what bounds the call is how fast HBM delivers them: 512 bytes a key and head at d_h = 128
// against 4 d_h flops a column, 16 or 32 columns.  So the chip is filled along the keys: the key tiles of all
// (sequence, kv head) blocks form one sequence of units that is cut into equal ranges, a workgroup each (one per CU), and a
// block that a cut goes through is put together from its pieces by the workgroup that finishes it last.  Within a workgroup the
// tiles of a block are dealt to four waves that run on their own: a wave keeps a ring of tiles of its own in LDS, filled by
// 16-byte global->LDS loads, and waits for nothing but its own loads, so that 16 to 32 KB per wave, up to 128 KB per CU,
// are always on their way.
//
// A wave computes S^T = K Q^T and O^T = V^T P^T with 16x16x32 MFMAs, columns on the N side: a lane then owns one
// column, its scores are laid out as the second product's operand needs them, and the rescale factor is one number per
// lane.  The running maximum moves only when a score exceeds it by more than 2^8 (in base 2), so most tiles need neither an
// exchange between lanes nor a rescale; probabilities up to 2^8 and sums in fp32 cancel in the final division.  Probabilities
// meet the values in two bf16 parts, what the first one's rounding left is the second, so that 2^-16 of them is lost: the matrix pipe
// has the time (one token of 32 ragged sequences of up to 16577, 32 heads of 8, us with one part / two: d_h 128 236 / 234, d_h 64
// 136 / 140).
//
// Many rows (chunk_attn_kernel): the loop of the contiguous cache's attention (attend.h), 256 columns a workgroup, with the
// key tiles of all (sequence, row tile, kv head) blocks in equal ranges, and pieces put together as above.  Probabilities are
// rounded to bf16, 2^-8 of each at most, as there.  Two parts would take half as many matrix operations again and some
// more vector ones, on pipes that bound these calls (us with one part / two: 1024 rows over 66560, 64 heads of 8, 2003 / 2697; 2 times
// 1024 under a window of 4096, 28 of 4, 150 / 195; 6 times up to 512 over 4224, 32 of 8, d_h 64, 104 / 121; 5 drafted
// tokens of 16 sequences of up to 16581, 32 of 8, where one wave of a workgroup has columns, 133 / 153).
#include "attend.h"
#include "paged.h"

namespace {

constexpr int KEYS = 32;                      // of a tile of few_attn_kernel
constexpr int WAVES = 4;
constexpr int START = 4;                      // units that a block costs besides its tiles: its queries, first loads and result
// Blocks of up to so many tiles are not cut where every block can have a workgroup: 512 tokens take 8.3 us either way, 256
// take 6.2 whole and 7.3 in pieces (one sequence, 4 query heads of 2, d_h 64), 7.0 and 8.6 (32 of 8, d_h 128).
constexpr int WHOLE = 16;
// Longer ones are cut at multiples of the shortest range from their start on, if there are workgroups for it: one with the end
// of a block and the start of another takes 3 us more (8 sequences of 1073 tokens, 4 heads of 2: 13.0 us in equal ranges, 10.4 so).

// 16 bytes per lane from global memory into LDS at wave base + OFF + 16 * lane; OFF is added to the global address too.
// Non-temporal: what few rows read is read once.
template <int OFF>
__device__ __forceinline__ void stream16(const char* gsrc_minus_off, char* lds_wave_base) {
    static_assert(OFF >= 0 && OFF < 4096, "the instruction offset is 13 bits signed");
    __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)gsrc_minus_off,
                                     (void __attribute__((address_space(3)))*)lds_wave_base, 16, OFF, 2);
}
// At most N of this wave's loads and stores still on their way.
template <int N>
__device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
    asm volatile("" ::: "memory");
}

// The blocks of a many-rows launch that leaves its pieces to another: entry (kv head, e) has the units
// kvh * head_units + first[e] .., in ranges of `per`.
constexpr int CUT_SHARE = 4;                  // of the workgroups: up to so many blocks leave their pieces to another launch
constexpr int CUT_BLOCKS = CC_PAGED_WGS / 2;
struct cut_table {
    int64_t per;
    int32_t head_units, blocks;
    int32_t first[CUT_BLOCKS], tiles[CUT_BLOCKS], seq[CUT_BLOCKS], row_tile[CUT_BLOCKS];
};
static_assert(sizeof(cut_table) <= CC_PAGED_CUT_BYTES, "room for it in a pool's scratch");

struct paged_args {
    const bf16_t* q;
    bf16_t* o;
    const int32_t* start;
    const int32_t* seq;
    int32_t n, rows;
    cc_pool_view p;
    const bf16_t* K;
    const bf16_t* V;
    int64_t st_page, st_tok, st_head;
    int32_t window, sinks, H_q, H_kv, g;
    float scale_log2;
    const bf16_t* zeros;        // d_h of them
    float* part;                // pieces: two slots a workgroup
    int32_t* arrived;           // [workgroups], zero between calls
    struct cut_table* cuts;     // many rows: where the pieces are, for a launch that adds them; NULL: the last workgroup does
};

struct batch_seq {
    int row0, n, s, L;          // first row, rows, row of the table, tokens
};
__device__ __forceinline__ batch_seq seq_of(const paged_args& a, int b) {
    batch_seq r;
    const int r0 = max(0, a.start[b]), r1 = min(a.rows, a.start[b + 1]);
    r.row0 = r0;
    r.n = max(0, r1 - r0);
    r.s = a.seq ? a.seq[b] : b;
    r.L = cc_seq_len(a.p, r.s);
    if ((unsigned)r.s >= (unsigned)a.p.n_seqs) r.s = 0;
    return r;
}

__device__ __forceinline__ int64_t of_lane(int64_t v, int l) {
    return ((int64_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)v, l);
}
// x / y of whole numbers, 0 <= x < 2^52: the quotient in 64-bit floating point is exact enough to be cut off, and takes a
// tenth of the instructions of a 64-bit integer division.
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) { return (int64_t)((double)x / (double)y); }

// NC: blocks of 16 columns that a wave multiplies a tile with.  Compiled for workgroups of eight waves, two a SIMD: with 512 registers the
// compiler keeps the sums in accumulation registers and copies them out and in for every rescale.
template <int D_H, int NC>
__global__ __launch_bounds__(512, 2) void few_attn_kernel(paged_args a, int per_min) {
    constexpr int KS = D_H / 32;              // k-steps of the scores
    constexpr int DT = D_H / 16;              // 16-row tiles of O^T
    constexpr int CPR = D_H / 8;              // 16-byte chunks of a row
    constexpr int RPI = 64 / CPR;             // rows moved by one load
    constexpr int NL = KEYS / RPI;            // loads of a K or V tile
    constexpr int HL = NL / 2;                // of 16 keys: within one page
    constexpr int ROW = D_H * 2;              // bytes
    constexpr int TILE = KEYS * ROW;
    constexpr int NS = D_H == 128 ? 2 : 4;    // tiles in a wave's ring
    constexpr int RING = 2 * NS * TILE;
    constexpr int COLS = 16 * NC;
    __shared__ __align__(1024) char ring[WAVES][RING];
    __shared__ int64_t pre[CC_PAGED_MAX_N + 1];
    __shared__ int64_t wave_sum[WAVES];
    __shared__ float2 ml[WAVES][COLS];
    __shared__ int last_here;
    static_assert(COLS * D_H * 4 <= RING, "a wave's sums fit its ring");
    const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);

    // ---- units in front of every sequence of the batch: up to 64 sequences a lane each, in every wave; more in LDS ----
    auto blocks_of = [&](const batch_seq& s) -> int { return (s.n * a.g + COLS - 1) / COLS * a.H_kv; };
    auto block_len = [&](const batch_seq& s) -> int {
        return s.n > 0 ? visible_tiles(s.L - s.n, s.L, a.window, a.sinks, KEYS).count + START : 0;
    };
    // over the first `lanes` lanes: an exchange between lanes is a trip through LDS, and one sequence needs none
    auto wave_scan = [&](int64_t v, int lanes) -> int64_t {
        for (int off = 1; off < lanes; off <<= 1) {
            const int64_t x = __shfl_up(v, off);
            if (lane >= off) v += x;
        }
        return v;
    };
    const bool small = a.n <= 64;
    batch_seq mine = {0, 0, 0, 0};
    int64_t my_end = 0, my_units = 0, total;
    // > 0: no workgroup has two blocks: every block starts a range of so many units and is as long as whole ranges
    int aligned = 0;
    if (small) {
        mine = seq_of(a, min(lane, a.n - 1));
        if (lane >= a.n) mine.n = 0;
        int len = block_len(mine), longest = len, blocks = blocks_of(mine);
        for (int off = 1; off < a.n; off <<= 1) {
            longest = max(longest, __shfl_xor(longest, off));
            blocks += __shfl_xor(blocks, off);
        }
        longest = uniform(longest);
        blocks = uniform(blocks);
        if (blocks > 0 && blocks <= (int)gridDim.x) {
            if (longest <= WHOLE + START) aligned = longest;
            else if ((longest + per_min - 1) / per_min <= (int)gridDim.x / blocks) aligned = per_min;
        }
        if (aligned > 0) len = (len + aligned - 1) / aligned * aligned;
        my_units = (int64_t)blocks_of(mine) * len;
        my_end = wave_scan(my_units, a.n);
        total = of_lane(my_end, a.n - 1);
    } else {
        int64_t carry = 0;
        for (int i0 = 0; i0 < a.n; i0 += 64 * WAVES) {
            const int i = i0 + tid;
            const batch_seq s = seq_of(a, min(i, a.n - 1));
            const int64_t v = i < a.n ? (int64_t)blocks_of(s) * block_len(s) : 0, inc = wave_scan(v, 64);
            if (lane == 63) wave_sum[w] = inc;
            __syncthreads();
            int64_t base = carry;
            for (int j = 0; j < WAVES; ++j) {
                if (j < w) base += wave_sum[j];
                carry += wave_sum[j];
            }
            if (i < a.n) pre[i] = base + inc - v;
            __syncthreads();
        }
        if (tid == 0) pre[a.n] = carry;
        __syncthreads();
        total = uniform(pre[a.n]);
    }
    const int64_t per = aligned > 0 ? aligned : max((int64_t)per_min, quotient(total + gridDim.x - 1, gridDim.x));
    const int range = blockIdx.x;
    int64_t u = range * per;
    const int64_t stop = min(u + per, total);

    while (u < stop) {
        // ---- the block that unit u lies in ----
        int row0, n_new, s, L;
        int64_t seq0;
        if (small) {
            const int b = __popcll(__ballot(lane < a.n && my_end <= u));
            row0 = __builtin_amdgcn_readlane(mine.row0, b);
            n_new = __builtin_amdgcn_readlane(mine.n, b);
            s = __builtin_amdgcn_readlane(mine.s, b);
            L = __builtin_amdgcn_readlane(mine.L, b);
            seq0 = of_lane(my_end - my_units, b);
        } else {
            int b = 0;
            for (int i = lane; i - lane < a.n; i += 64) b += __popcll(__ballot(i < a.n && pre[min(i, a.n - 1) + 1] <= u));
            b = uniform(b);
            const batch_seq sq = seq_of(a, b);
            row0 = uniform(sq.row0), n_new = uniform(sq.n), s = uniform(sq.s), L = uniform(sq.L);
            seq0 = uniform(pre[b]);
        }
        const int first = L - n_new;
        const tile_span span = visible_tiles(first, L, a.window, a.sinks, KEYS);
        const int real = span.count + START, len = aligned > 0 ? (real + aligned - 1) / aligned * aligned : real;
        const int which = (int)quotient(u - seq0, len), blk = which / a.H_kv, h = which - blk * a.H_kv;
        const int64_t u0 = seq0 + (int64_t)which * len, u1 = u0 + len;
        const int ta = (int)max((int64_t)0, u - u0 - START), te = min((int)(min(u1, stop) - u0) - START, span.count);
        u = u1;
        if (te <= ta) continue;

        // ---- lane constants of the block: loads (row and swizzled chunk) and fragment addresses ----
        // K: chunk c of row r at slot c ^ kswz(r); V: the 32-byte pair of chunks dt at pair dt ^ vswz(r).
        auto kswz = [](int r) { return D_H == 128 ? (r & 15) : ((r >> 1) & 7); };
        auto vswz = [](int r) { return D_H == 128 ? (r & 7) : ((r >> 1) & 3); };
        const int ln0 = here(lane), c16 = ln0 & 15, kg = ln0 >> 4, l_row = ln0 / CPR, l_c = ln0 % CPR;
        // Both swizzles and the places they act on are bit fields: what a load's index, a k-step or a tile of O^T adds to an address
        // is one exclusive or with a constant.
        const uint32_t st_b = (uint32_t)a.st_tok * 2;
        const uint32_t k_col = (l_c ^ kswz(l_row)) * 16, v_col = (l_c ^ (2 * vswz(l_row))) * 16;
        char* const my_ring = ring[w];
        const uint32_t ring_at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)my_ring;
        const uint32_t k_base = ring_at + c16 * ROW + ((kg ^ kswz(c16)) << 4);
        const int v_row = 4 * kg + (c16 >> 2);
        const uint32_t v_base = ring_at + TILE + v_row * ROW + ((((c16 & 3) >> 1) ^ (2 * vswz(v_row))) << 4) + (c16 & 1) * 8;

        // ---- queries: B operand of the scores ----
        bf16x8 qf[NC][KS];
        int limit[NC];                                     // the newest key a column sees
        // positions of the block's last and first row
        const int most = max(first + min(n_new - 1, (blk * COLS + COLS - 1) / a.g), -1), least = max(first + blk * COLS / a.g, -1);
#pragma unroll
        for (int nc = 0; nc < NC; ++nc) {
            const int col = blk * COLS + nc * 16 + c16, i = col / a.g, hg = col - i * a.g;
            const bool valid = i < n_new;
            limit[nc] = valid ? max(first + i, -1) : -1;
            const bf16_t* qp = a.q + ((int64_t)(row0 + (valid ? i : 0)) * a.H_q + h * a.g + (valid ? hg : 0)) * D_H + 8 * kg;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) qf[nc][ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 32);
        }
        f32x4 acc[DT][NC];
        float m_run[NC], l_run[NC];
#pragma unroll
        for (int nc = 0; nc < NC; ++nc) {
            m_run[nc] = -INFINITY;
            l_run[nc] = 0.0f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) acc[dt][nc] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        // ---- loads of the wave's k-th tile ----
        const int nt = te - ta > w ? (te - ta - w + WAVES - 1) / WAVES : 0;
        auto tile_key = [&](int k) { return span.tile(ta + w + k * WAVES) * KEYS; };
        // (scalar loads do not count among the loads that the waits below count)
        const scalar_table row_table = (scalar_table)(a.p.table + s * a.p.st_table);
        const int64_t head_off = (int64_t)h * a.st_head;
        // The two pages of a tile (16 keys each, in one page): those of the first NS tiles together, the others' a tile ahead.
        struct pages { int a, b; };
        auto pages_of = [&](int k) __attribute__((always_inline)) -> pages {
            const int key0 = tile_key(min(k, max(nt - 1, 0))), end = max(L - 1, 0);
            return {row_table[min(key0, end) >> a.p.shift], row_table[min(key0 + 16, end) >> a.p.shift]};
        };
        // First row of 16 keys as an offset into K and V, and its last one: rows behind the last token repeat it (they are
        // masked); rmax < 0: zeros, for what no page holds.
        struct rows16 { int64_t at; int rmax; };
        auto rows_of = [&](int key0, int page) __attribute__((always_inline)) -> rows16 {
            const bool there = key0 < L && (unsigned)page < (unsigned)a.p.n_pages;
            return {(page * a.st_page + (int64_t)(key0 & ((1 << a.p.shift) - 1)) * a.st_tok + head_off) * 2,
                    there ? min(15, L - 1 - key0) : -1};
        };
        // (a scalar base and a 32-bit lane offset: 64-bit vector addresses cost more to make than the loads to issue)
        auto load = [&](const bf16_t* base, rows16 r, uint32_t col, auto swz, char* dst) __attribute__((always_inline)) {
            const char* src = r.rmax < 0 ? (const char*)a.zeros : (const char*)base + r.at;
            const int last = max(r.rmax, 0);
            static_for<HL>([&](auto ic) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value;
                uint32_t off = __umul24(min(i * RPI + l_row, last), st_b) + (col ^ (swz(i * RPI) << 4));
                asm volatile("" : "+v"(off));
                stream16<i * 1024>(scalar_base(src - i * 1024) + off, dst);
            });
        };
        auto kswz_of = [&](int r) { return kswz(r); };
        auto vswz_of = [&](int r) { return 2 * vswz(r); };
        auto stage_of = [&](int k) { return my_ring + ((k + NS) % NS) * 2 * TILE; };
        pages ahead[NS];
#pragma unroll
        for (int k = 0; k < NS; ++k) ahead[k] = pages_of(k);
        // The queries are waited for here, where the page numbers are: left to the compiler the wait would stand in the loop, for
        // every load on its way (one token of 32 ragged sequences, 32 heads of 8, d_h 128, us with the wait in the loop / here: up to 300
        // tokens 11.0 / 10.6, up to 16577 233 / 237).
        asm volatile("" :: "s"(ahead[0].a), "s"(ahead[0].b));
        wait_loads<0>();
        // Loads younger than K(k): V(k) and the pairs of up to NS - 1 later tiles; than V(k): those and K(k + NS).
        auto wait_k = [&](int rem) __attribute__((always_inline)) {
            static_for<NS>([&](auto jc) __attribute__((always_inline)) {
                constexpr int j = decltype(jc)::value;
                if (j == NS - 1 ? rem >= j : rem == j) wait_loads<NL * (1 + 2 * j)>();
            });
        };
        auto wait_v = [&](int rem) __attribute__((always_inline)) {
            static_for<NS>([&](auto jc) __attribute__((always_inline)) {
                constexpr int j = decltype(jc)::value;
                if (rem == j) wait_loads<NL * 2 * j>();
            });
            if (rem >= NS) wait_loads<NL * (2 * (NS - 1) + 1)>();
        };

        // Iterations -NS .. -1 only fill the ring.
#pragma unroll 1
        for (int k = -NS; k < nt; ++k) {
            const int key0 = tile_key(k), rem = nt - 1 - k, key_in = tile_key(k + NS);
            const uint32_t stage = (uint32_t)((k + NS) % NS) * 2 * TILE;
            bf16x8 kf[2][KS];
            if (k >= 0) {
                wait_k(rem);
                static_for<KS>([&](auto kc) __attribute__((always_inline)) {
                    constexpr int ks = decltype(kc)::value;
                    const uint32_t at = (k_base + stage) ^ (ks << 6);
                    kf[0][ks] = lds_read_b128_at<0>(at);
                    kf[1][ks] = lds_read_b128_at<16 * ROW>(at);
                });
                if constexpr (KS == 4)
                    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(kf[0][0]), "+v"(kf[1][0]), "+v"(kf[0][1]), "+v"(kf[1][1]), "+v"(kf[0][2]),
                                 "+v"(kf[1][2]), "+v"(kf[0][3]), "+v"(kf[1][3])
                                 :: "memory");
                else
                    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(kf[0][0]), "+v"(kf[1][0]), "+v"(kf[0][1]), "+v"(kf[1][1])::"memory");
            }
            const rows16 x = rows_of(key_in, ahead[0].a), y = rows_of(key_in + 16, ahead[0].b);
            if (rem >= NS) {
                load(a.K, x, k_col, kswz_of, stage_of(k));
                load(a.K, y, k_col, kswz_of, stage_of(k) + TILE / 2);
            }
#pragma unroll
            for (int i = 0; i + 1 < NS; ++i) ahead[i] = ahead[i + 1];
            if (k < 0) {
                if (k == -1) ahead[0] = pages_of(NS);
                if (rem >= NS) {
                    load(a.V, x, v_col, vswz_of, stage_of(k) + TILE);
                    load(a.V, y, v_col, vswz_of, stage_of(k) + TILE + TILE / 2);
                }
                continue;
            }
            // a block of columns at a time: scores, mask, softmax in base 2 with the scale folded into the exponent
            const bool masked = key0 + KEYS - 1 > least || (a.window > 0 && key0 <= most - a.window && key0 + KEYS > a.sinks);
            bf16x8 pf[NC], pr[NC];                         // probabilities: bf16, and what that left of them
#pragma unroll
            for (int nc = 0; nc < NC; ++nc) {
                f32x4 sc[2];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
                        sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t][ks], qf[nc][ks], sc[t], 0, 0, 0);
                }
                if (masked) {                              // keys behind a row, or in front of its window and no sink
                    const int under = a.window > 0 ? limit[nc] - a.window : (int)0x80000000;
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            const int key = key0 + t * 16 + 4 * kg + v;
                            // (no short circuits: selects, not branches)
                            const bool out = (key > limit[nc]) | ((key <= under) & (key >= a.sinks));
                            sc[t][v] = out ? -INFINITY : sc[t][v];
                        }
                }
                float mx = -INFINITY;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int v = 0; v < 4; ++v) mx = fmaxf(mx, sc[t][v]);
                mx *= a.scale_log2;
                if (__any(mx > m_run[nc] + 8.0f)) {
                    mx = fmaxf(mx, __shfl_xor(mx, 16));
                    mx = fmaxf(mx, __shfl_xor(mx, 32));
                    const float m_new = mx > m_run[nc] + 8.0f ? mx : m_run[nc];
                    const float alpha = __builtin_amdgcn_exp2f(m_run[nc] - (m_new == -INFINITY ? 0.0f : m_new));
                    l_run[nc] *= alpha;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) acc[dt][nc] *= alpha;
                    m_run[nc] = m_new;
                }
                const float ref = m_run[nc] == -INFINITY ? 0.0f : m_run[nc];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(sc[t][v], a.scale_log2, -ref));
                        l_run[nc] += p;
                        pf[nc][t * 4 + v] = (bf16_t)p;
                        pr[nc][t * 4 + v] = (bf16_t)(p - (float)pf[nc][t * 4 + v]);
                    }
            }
            // ---- O^T += V^T P^T: the 32 keys in the order in which a lane holds its scores ----
            wait_v(rem);
            bf16x4 va[DT], vb[DT];
            static_for<DT>([&](auto dc) __attribute__((always_inline)) {
                constexpr int dt = decltype(dc)::value;
                const uint32_t at = (v_base + stage) ^ (dt << 5);
                va[dt] = lds_read_tr_at<0>(at);
                vb[dt] = lds_read_tr_at<16 * ROW>(at);
            });
            asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(va[0]), "+v"(vb[0]), "+v"(va[1]), "+v"(vb[1]), "+v"(va[2]), "+v"(vb[2]),
                         "+v"(va[3]), "+v"(vb[3])
                         :: "memory");
            if constexpr (DT == 8)
                asm volatile("" : "+v"(va[4]), "+v"(vb[4]), "+v"(va[5]), "+v"(vb[5]), "+v"(va[6]), "+v"(vb[6]), "+v"(va[7]), "+v"(vb[7])::"memory");
            if (rem >= NS) {
                load(a.V, x, v_col, vswz_of, stage_of(k) + TILE);
                load(a.V, y, v_col, vswz_of, stage_of(k) + TILE + TILE / 2);
            }
            ahead[0] = pages_of(k + 1 + NS);
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const bf16x8 vf = __builtin_shufflevector(va[dt], vb[dt], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                    for (int nc = 0; nc < NC; ++nc)
                        acc[dt][nc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, part ? pr[nc] : pf[nc], acc[dt][nc], 0, 0, 0);
                }
        }

        // ---- the four waves' sums together, as the registers lie: [dt][nc][lane]; to the output or to a piece (two lots of
        // eight bytes a lane, then (maximum, sum) a column).  Ends with the rings free again ----
        auto together = [&](float* piece) __attribute__((always_inline)) {
            const int ln = here(lane), c = ln & 15, quad = ln >> 4;
#pragma unroll
            for (int nc = 0; nc < NC; ++nc) {
                float l = l_run[nc];
                l += __shfl_xor(l, 16);
                l += __shfl_xor(l, 32);
                if (quad == 0) ml[w][nc * 16 + c] = make_float2(m_run[nc], l);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
                    *reinterpret_cast<f32x4*>(my_ring + ((dt * NC + nc) * 64 + ln) * 16) = acc[dt][nc];
            }
            __syncthreads();
#pragma unroll
            for (int nc = 0; nc < NC; ++nc) {
                float2 x[WAVES];
                float m = -INFINITY, l = 0.0f;
#pragma unroll
                for (int j = 0; j < WAVES; ++j) {
                    x[j] = ml[j][nc * 16 + c];
                    m = fmaxf(m, x[j].x);
                }
                const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
                for (int j = 0; j < WAVES; ++j) {
                    x[j].x = __builtin_amdgcn_exp2f(x[j].x - ref);
                    l += x[j].x * x[j].y;
                }
                const int col = blk * COLS + nc * 16 + c, i = col / a.g, hg = col - i * a.g;
                const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
                for (int d = 0; d < DT / WAVES; ++d) {
                    const int dt = d * WAVES + w;
                    f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < WAVES; ++j)
                        r += x[j].x * *reinterpret_cast<const f32x4*>(ring[j] + ((dt * NC + nc) * 64 + ln) * 16);
                    if (piece) {
                        put(piece + (dt * NC + nc) * 256 + ln * 2, r[0], r[1]);
                        put(piece + (dt * NC + nc) * 256 + 128 + ln * 2, r[2], r[3]);
                    } else if (i < n_new) {
                        bf16x4 out;
#pragma unroll
                        for (int e = 0; e < 4; ++e) out[e] = (bf16_t)(r[e] * inv);
                        *reinterpret_cast<bf16x4*>(a.o + ((int64_t)(row0 + i) * a.H_q + h * a.g + hg) * D_H + dt * 16 + 4 * quad) = out;
                    }
                }
                if (piece && w == 0 && quad == 0) put(piece + COLS * D_H + nc * 32 + c * 2, m, l);
            }
            if (piece) wait_loads<0>();                    // it is written
            __syncthreads();
        };
        // ---- A cut block: a range leaves at most two pieces, of the block it starts in and of a later one.  The workgroup
        // that comes last adds them: a wave takes every fourth, then as above.  (Stores past the L2 have been
        // acknowledged before the count is raised, and loads past it follow the count: no fence is needed.) ----
        const int w0 = (int)quotient(u0 + START, per), w1 = (int)quotient(u0 + real - 1, per);
        auto piece_of = [&](int j) { return a.part + (int64_t)(2 * j + (j == w0 ? 1 : 0)) * COLS * (D_H + 2); };
        wait_loads<0>();
        float* piece = ta == 0 && te == span.count ? nullptr : piece_of(range);
        while (true) {
            together(piece);
            if (!piece) break;
            if (tid == 0) {
                const int before = __hip_atomic_fetch_add(&a.arrived[w0], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                last_here = before == w1 - w0;
                if (last_here) __hip_atomic_store(&a.arrived[w0], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (!last_here) break;
            piece = nullptr;
            const int ln = here(lane), c = ln & 15, quad = ln >> 4;
#pragma unroll
            for (int nc = 0; nc < NC; ++nc) {
                m_run[nc] = -INFINITY;
                l_run[nc] = 0.0f;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) acc[dt][nc] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            constexpr int AT_ONCE = NC == 1 ? 2 : 1;
            for (int j = w0 + w; j <= w1; j += WAVES * AT_ONCE) {
#pragma unroll
                for (int nc = 0; nc < NC; ++nc) {
                    float2 x[AT_ONCE], v[AT_ONCE][DT][2];
                    float m = m_run[nc];
#pragma unroll
                    for (int k = 0; k < AT_ONCE; ++k) {
                        const float* pc = piece_of(min(j + k * WAVES, w1));   // past the end: the last one, with weight 0
                        x[k] = get(pc + COLS * D_H + nc * 32 + c * 2);
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) {
                            v[k][dt][0] = get(pc + (dt * NC + nc) * 256 + ln * 2);
                            v[k][dt][1] = get(pc + (dt * NC + nc) * 256 + 128 + ln * 2);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < AT_ONCE; ++k) m = fmaxf(m, j + k * WAVES <= w1 ? x[k].x : -INFINITY);
                    const float ref = m == -INFINITY ? 0.0f : m, keep = __builtin_amdgcn_exp2f(m_run[nc] - ref);
                    l_run[nc] *= keep;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) acc[dt][nc] *= keep;
#pragma unroll
                    for (int k = 0; k < AT_ONCE; ++k) {
                        const float f = j + k * WAVES <= w1 ? __builtin_amdgcn_exp2f(x[k].x - ref) : 0.0f;
                        if (quad == 0) l_run[nc] += x[k].y * f;
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) acc[dt][nc] += f * f32x4{v[k][dt][0].x, v[k][dt][0].y, v[k][dt][1].x, v[k][dt][1].y};
                    }
                    m_run[nc] = m;
                }
            }
        }
    }
}

constexpr int CHUNK_START = 5;                // units of a block besides its key tiles, as in the even grids of attention.hip
constexpr int MAX_BLOCKS = CC_PAGED_MAX_COLUMNS / 256 + CC_PAGED_MAX_N;

// Key tiles that row tile rt of a sequence of n new rows from position `first` on sees.
__device__ __forceinline__ tile_span row_tile_span(const paged_args& a, int first, int n, int rt) {
    const int end = first + min(n - 1, (rt * 256 + 255) / a.g) + 1;
    return visible_tiles(first + rt * 256 / a.g, max(end, 0), a.window, a.sinks, BN_KEYS);
}

// A workgroup of eight waves per range.  Blocks are numbered e0(b) + row tile with e0(b) = floor(columns in front of b / 256) + b:
// at least as many numbers as sequence b has row tiles, the unused ones of length 0, and no scan is needed to find one.
template <int D_H, bool WIDE_PAGES, bool ONCE>
__global__ __launch_bounds__(512, 1) void chunk_attn_kernel(paged_args a, int per_min) {
    __shared__ __align__(16) bf16_t smem[LDS_TILES * BN_KEYS * D_H];
    __shared__ int simd_waves[4], group_waves[2], wave_units[8], last_here;
    __shared__ struct { int longest, count; float sum; } of_wave[8];
    __shared__ int pre[MAX_BLOCKS + 1];
    __shared__ int e0[CC_PAGED_MAX_N + 1], rows_of[CC_PAGED_MAX_N], len_of[CC_PAGED_MAX_N];
    const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
    int grp, widx;
    wave_role(simd_waves, group_waves, grp, widx);

    auto sequence_of = [&](int e) -> int {                // the last one with e0 <= e
        int b = 0;
        for (int hi = a.n - 1; b < hi;) {
            const int mid = (b + hi + 1) >> 1;
            if (e0[mid] <= e) b = mid; else hi = mid - 1;
        }
        return b;
    };
    // ---- units in front of every block of a head ----
    int aligned;
    {
        const int base = max(0, min(a.start[0], a.rows));
        for (int b = tid; b <= a.n; b += 512) {
            const int r = max(base, min(a.start[b], a.rows));
            e0[b] = (int)((int64_t)(r - base) * a.g / 256) + b;
            if (b < a.n) {
                const batch_seq s = seq_of(a, b);
                rows_of[b] = s.n;
                len_of[b] = s.L;
            }
        }
        __syncthreads();
        const int blocks = min(e0[a.n], MAX_BLOCKS);
        int longest = 0, count = 0;
        float sum = 0.0f;
        for (int e = tid; e < blocks; e += 512) {
            const int b = sequence_of(e), c0 = (e - e0[b]) * 256, n = rows_of[b], first = len_of[b] - n;
            int len = 0;
            if (c0 >= 0 && c0 < n * a.g) {
                len = row_tile_span(a, first, n, e - e0[b]).count + CHUNK_START;
                longest = max(longest, len);
                sum += len;
                ++count;
            }
            pre[e] = len;
        }
        for (int off = 32; off > 0; off >>= 1) {
            longest = max(longest, __shfl_xor(longest, off));
            count += __shfl_xor(count, off);
            sum += __shfl_xor(sum, off);
        }
        if (lane == 0) of_wave[w] = {longest, count, sum};
        __syncthreads();
        longest = count = 0;
        sum = 0.0f;
        for (int j = 0; j < 8; ++j) {
            longest = max(longest, of_wave[j].longest);
            count += of_wave[j].count;
            sum += of_wave[j].sum;
        }
        // Ranges start with a block where equal ones would not be much shorter: one with the end of a block and the start of
        // another leaves two pieces (two chunks of 1024 rows under a window of 4096, 28 heads of 4: 170 us in equal ranges, 163
        // so; 16 of 100 rows over 500 to 1500 tokens 60 and 56; 700 rows over 20000 238 and 225).  Without any cut they may be longer.
        const int in_all = count * a.H_kv, n_wg = gridDim.x;
        aligned = 0;
        if (count > 0 && in_all <= n_wg) {
            const int cuts = n_wg / in_all, each = max(per_min, (longest + cuts - 1) / cuts);
            if ((float)each <= 1.1f * sum * a.H_kv / n_wg + (cuts == 1 ? 10.0f : 2.0f)) aligned = each;
        }
        int carry = 0;
        for (int i0 = 0; i0 < blocks; i0 += 512) {
            const int e = i0 + tid;
            int len = e < blocks ? pre[e] : 0;
            if (aligned > 0) len = (len + aligned - 1) / aligned * aligned;
            int inc = len;
            for (int off = 1; off < 64; off <<= 1) {
                const int v = __shfl_up(inc, off);
                if (lane >= off) inc += v;
            }
            if (lane == 63) wave_units[w] = inc;
            __syncthreads();
            int before = carry;
            for (int j = 0; j < 8; ++j) {
                if (j < w) before += wave_units[j];
                carry += wave_units[j];
            }
            if (e < blocks) pre[e] = before + inc - len;
            __syncthreads();
        }
        if (tid == 0) pre[blocks] = carry;
        __syncthreads();
        aligned = uniform(aligned);
    }
    const int blocks = uniform(min(e0[a.n], MAX_BLOCKS)), head_units = uniform(pre[blocks]);
    const int64_t total = (int64_t)head_units * a.H_kv;
    const int n_wg = gridDim.x;
    const int64_t per = aligned > 0 ? aligned : max((int64_t)per_min, (total + n_wg - 1) / n_wg);
    if (a.cuts && blockIdx.x == 0) {
        if (tid == 0) a.cuts->per = per, a.cuts->head_units = head_units, a.cuts->blocks = blocks;
        for (int e = tid; e < min(blocks, CUT_BLOCKS); e += 512) {
            const int b = sequence_of(e), rt = e - e0[b], n = rows_of[b], first = len_of[b] - n;
            a.cuts->first[e] = pre[e];
            a.cuts->seq[e] = b;
            a.cuts->row_tile[e] = rt;
            a.cuts->tiles[e] = pre[e + 1] == pre[e] ? 0 : row_tile_span(a, first, n, rt).count;
        }
    }
    // workgroup ids go round-robin to the 8 XCDs: each gets consecutive ranges
    const int x = blockIdx.x & 7, xq = n_wg >> 3, xr = n_wg & 7;
    const int range = x * xq + min(x, xr) + (int)(blockIdx.x >> 3);
    int64_t u = range * per;
    const int64_t stop = min(u + per, total);
    while (u < stop) {
        const int kvh = (int)quotient(u, head_units), uh = (int)(u - (int64_t)kvh * head_units);
        int e = 0;
        for (int i = lane; i - lane < blocks; i += 64) e += __popcll(__ballot(i < blocks && pre[min(i, blocks - 1) + 1] <= uh));
        e = uniform(e);
        const int b = uniform(sequence_of(e));
        const int b0 = uniform(pre[e]), padded = uniform(pre[e + 1]) - b0, rt = e - uniform(e0[b]);
        const batch_seq sq = seq_of(a, b);
        const int n_new = uniform(sq.n), L = uniform(sq.L), first = L - n_new;
        const tile_span span = row_tile_span(a, first, n_new, rt);
        const int ta = max(0, uh - b0 - CHUNK_START), te = min((int)min((int64_t)padded, uh - b0 + (stop - u)) - CHUNK_START, span.count);
        const int64_t u0 = (int64_t)kvh * head_units + b0;
        u = u0 + padded;
        if (te <= ta) continue;
        in_pages<WIDE_PAGES, ONCE> keys;
        keys.table = (scalar_table)(a.p.table + uniform(sq.s) * a.p.st_table);
        keys.K = a.K, keys.V = a.V, keys.zeros = a.zeros;
        keys.st_page = a.st_page, keys.st_tok = a.st_tok, keys.sh = a.st_head;
        keys.shift = a.p.shift, keys.n_pages = a.p.n_pages, keys.L = L, keys.first = first, keys.row0 = uniform(sq.row0);
        keys.window = a.window, keys.sinks = a.sinks;
        keys.span = span;
        const bool whole = ta == 0 && te == span.count;
        const int w0 = (int)quotient(u0 + CHUNK_START, per), w1 = (int)quotient(u0 + CHUNK_START + span.count - 1, per);
        attend<D_H, true, uint32_t>(keys, a.q, n_new, a.H_q, a.g, a.o, a.scale_log2, a.part, smem, grp, widx, kvh, rt, ta, te - ta,
                                    whole ? -1 : 2 * range + (w0 == range ? 1 : 0));
        if (whole || a.cuts) continue;
        // ---- a cut block: the workgroup that comes last adds the pieces, in the order of their keys ----
        wait_loads<0>();                                   // the piece is written
        __syncthreads();
        if (tid == 0) {
            const int before = __hip_atomic_fetch_add(&a.arrived[w0], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            last_here = before == w1 - w0;
            if (last_here) __hip_atomic_store(&a.arrived[w0], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!last_here) continue;
        // A thread holds what the lane that left it did: half of a column's sums, in two passes; up to four
        // pieces are asked for together (one after the other they took 1.9 us each).
        constexpr int NG = D_H / 16;
        const int col = rt * 256 + w * 32 + (lane & 31), mi = col / a.g, hg = col - mi * a.g;
        if (mi >= n_new) continue;
        for (int k0 = 0; k0 < D_H / 8; k0 += NG) {
            f32x4 acc[NG];
            float m = -INFINITY, l = 0.0f;
#pragma unroll
            for (int k = 0; k < NG; ++k) acc[k] = f32x4{0.f, 0.f, 0.f, 0.f};
            auto take = [&](auto nc, int j0) __attribute__((always_inline)) {
                constexpr int NP = decltype(nc)::value;
                float2 ml[NP], v[NP][NG][2];
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const int j = min(j0 + i, w1);         // past the end: the last piece again, with weight 0
                    const float* pp = a.part + (int64_t)(2 * j + (j == w0 ? 1 : 0)) * 256 * (D_H + 4) + w * 32 * (D_H + 4);
                    ml[i] = get(pp + 32 * D_H + lane * 2);
#pragma unroll
                    for (int k = 0; k < NG; ++k) {
                        v[i][k][0] = get(pp + (k0 + k) * 256 + lane * 2);
                        v[i][k][1] = get(pp + (k0 + k) * 256 + 128 + lane * 2);
                    }
                }
                float mn = m;
#pragma unroll
                for (int i = 0; i < NP; ++i) mn = fmaxf(mn, ml[i].x);
                const float ref = mn == -INFINITY ? 0.0f : mn, keep = __builtin_amdgcn_exp2f(m - ref);
                l *= keep;
                m = mn;
#pragma unroll
                for (int k = 0; k < NG; ++k) acc[k] *= keep;
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const float f = j0 + i <= w1 ? __builtin_amdgcn_exp2f(ml[i].x - ref) : 0.0f;
                    l += ml[i].y * f;
#pragma unroll
                    for (int k = 0; k < NG; ++k) acc[k] += f * f32x4{v[i][k][0].x, v[i][k][0].y, v[i][k][1].x, v[i][k][1].y};
                }
            };
            for (int j = w0; j <= w1;) {
                if (w1 - j >= 2) take(std::integral_constant<int, 4>{}, j), j += 4;
                else take(std::integral_constant<int, 2>{}, j), j += 2;
            }
            const float inv = l > 0.0f ? 1.0f / l : 0.0f;
            bf16_t* op = a.o + ((int64_t)(keys.row0 + mi) * a.H_q + kvh * a.g + hg) * D_H + 4 * (lane >> 5);
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                bf16x4 r;
#pragma unroll
                for (int i = 0; i < 4; ++i) r[i] = (bf16_t)(acc[k][i] * inv);
                *reinterpret_cast<bf16x4*>(op + 8 * (k0 + k)) = r;
            }
        }
    }
}

// Adds the pieces of a many-rows launch: o = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s, in the order of their keys.  A workgroup takes
// 32 columns (a wave of the kernel that left them) and 32 of their d's of a block; a thread four sums of a column,
// of eight pieces at a time.  For few blocks in many pieces, which one workgroup a block reads at 75 GB/s (64 rows over 32768
// tokens, 8 blocks in 32 pieces: 116 us with the last workgroup adding them, 60 so).  From a quarter as many blocks as workgroups on each
// has four pieces at most, and the second launch costs more than it saves.
template <int D_H>
__global__ __launch_bounds__(256) void add_pieces_kernel(paged_args a) {
    const cut_table& c = *a.cuts;
    const int kvh = blockIdx.x % a.H_kv, e = blockIdx.x / a.H_kv;
    if (e >= min(c.blocks, CUT_BLOCKS) || c.tiles[e] == 0) return;
    const int64_t u0 = (int64_t)kvh * c.head_units + c.first[e] + CHUNK_START;
    const int w0 = (int)quotient(u0, c.per), w1 = (int)quotient(u0 + c.tiles[e] - 1, c.per);
    if (w0 == w1) return;
    const batch_seq s = seq_of(a, c.seq[e]);
    const int lane = threadIdx.x & 63, k = blockIdx.z * 4 + (threadIdx.x >> 6);
    const int col = c.row_tile[e] * 256 + blockIdx.y * 32 + (lane & 31), mi = col / a.g, hg = col - mi * a.g;
    if (mi >= s.n) return;
    float m = -INFINITY, l = 0.0f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    constexpr int NP = 8;
    for (int j0 = w0; j0 <= w1; j0 += NP) {
        float2 ml[NP], v[NP][2];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int j = min(j0 + i, w1);                 // past the end: the last piece again, with weight 0
            const float* pp = a.part + (int64_t)(2 * j + (j == w0 ? 1 : 0)) * 256 * (D_H + 4) + blockIdx.y * 32 * (D_H + 4);
            ml[i] = *reinterpret_cast<const float2*>(pp + 32 * D_H + lane * 2);
            v[i][0] = *reinterpret_cast<const float2*>(pp + k * 256 + lane * 2);
            v[i][1] = *reinterpret_cast<const float2*>(pp + k * 256 + 128 + lane * 2);
        }
        float mn = m;
#pragma unroll
        for (int i = 0; i < NP; ++i) mn = fmaxf(mn, ml[i].x);
        const float ref = mn == -INFINITY ? 0.0f : mn, keep = __builtin_amdgcn_exp2f(m - ref);
        l *= keep;
        acc *= keep;
        m = mn;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const float f = j0 + i <= w1 ? __builtin_amdgcn_exp2f(ml[i].x - ref) : 0.0f;
            l += ml[i].y * f;
            acc += f * f32x4{v[i][0].x, v[i][0].y, v[i][1].x, v[i][1].y};
        }
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    bf16x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (bf16_t)(acc[i] * inv);
    *reinterpret_cast<bf16x4*>(a.o + ((int64_t)(s.row0 + mi) * a.H_q + kvh * a.g + hg) * D_H + 8 * k + 4 * (lane >> 5)) = r;
}

}  // namespace

void cc_launch_paged_attention(const bf16_t* q, const cc_new_rows& r, const cc_page_pool& p, const cc_paged_kv& kv, int window,
                               int sinks, const cc_model_desc& m, const cc_paged_scratch& ws, bf16_t* o, hipStream_t s) {
    if (r.rows <= 0 || r.n <= 0) return;
    const int g = m.H_q / m.H_kv;
    paged_args a = {q, o, r.start, r.seq, r.n, r.rows, cc_view(p), (const bf16_t*)kv.K, (const bf16_t*)kv.V, kv.stride_page,
                    kv.stride_token, kv.stride_head, window, sinks, m.H_q, m.H_kv, g,
                    1.4426950408889634f / sqrtf((float)m.d_h), ws.zeros,
                    (float*)((char*)((int32_t*)p.work + cc_page_work_layout(p.n_pages, p.n_seqs).attn) + CC_PAGED_CUT_BYTES), ws.arrived, nullptr};
    const int grid = std::min(cc_device_cus(), CC_PAGED_WGS);
    const int64_t columns = (int64_t)std::min(r.max_new, r.rows) * g;
    const int per_min = WAVES + START;                     // a tile for each wave
    if (!cc_few_rows(columns, m.d_h)) {
        const int chunk_min = 3 + CHUNK_START;
#define CC_CHUNK(D, WIDE, ONCE) hipLaunchKernelGGL((chunk_attn_kernel<D, WIDE, ONCE>), dim3(grid), dim3(512), 0, s, a, chunk_min)
        // Keys that few rows read, and no other workgroup, go past the caches: 4 tokens over 4 times 65000, 64 heads of 8, 202 -> 173 us,
        // 5 over 16 ragged sequences of up to 16581, 32 of 8, 141 -> 125, 8 over 4 of 8000 38.6 -> 38.3.  More columns leave less of
        // the time to the loads and gain only where the last cache is too small, 64 over 16 of up to 16000 212 -> 207, 16 over
        // 8 of 8000 58 -> 60.
        const bool once = columns <= 32;
        const bool wide = p.page_size >= BN_KEYS;          // a tile of keys lies in one page
        // few blocks are cut into many pieces each: a launch of its own adds them
        const int64_t blocks = ((int64_t)r.rows * g / 256 + r.n) * m.H_kv;
        if (blocks <= CUT_BLOCKS && blocks <= grid / CUT_SHARE)
            a.cuts = (cut_table*)((int32_t*)p.work + cc_page_work_layout(p.n_pages, p.n_seqs).attn);
        if (m.d_h == 128) {
            if (wide && once) CC_CHUNK(128, true, true);
            else if (wide) CC_CHUNK(128, true, false);
            else if (once) CC_CHUNK(128, false, true);
            else CC_CHUNK(128, false, false);
        } else {
            if (wide) CC_CHUNK(64, true, false);           // (so few are the other kernel's)
            else CC_CHUNK(64, false, false);
        }
#undef CC_CHUNK
        if (a.cuts) {
            const dim3 mg((unsigned)blocks, 8, m.d_h / 32);
            if (m.d_h == 128) hipLaunchKernelGGL(add_pieces_kernel<128>, mg, dim3(256), 0, s, a);
            else hipLaunchKernelGGL(add_pieces_kernel<64>, mg, dim3(256), 0, s, a);
        }
        return;
    }
#define CC_FEW(D, NC) hipLaunchKernelGGL((few_attn_kernel<D, NC>), dim3(grid), dim3(64 * WAVES), 0, s, a, per_min)
    if (m.d_h == 128) CC_FEW(128, 1);
    else if (columns <= 16) CC_FEW(64, 1);
    else CC_FEW(64, 2);
#undef CC_FEW
}
