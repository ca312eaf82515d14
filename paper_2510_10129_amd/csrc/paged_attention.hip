// Causal grouped-query attention of new rows over a paged cache, optionally under a sliding window with sinks.
//
// Few rows (few_attn_kernel).  A sequence's new rows are a handful of (row, query head) columns per kv head, every key and
// value is read once, and what bounds the call is how fast HBM delivers them: 512 bytes a key and head at d_h = 128
// against 4 d_h flops a column, 16 to 64 columns.  So the chip is filled along the keys: the key tiles of all
// (sequence, kv head) blocks form one sequence of units that is cut into equal ranges, a workgroup each (one per CU), and a
// block that a cut goes through is put together from its pieces by the workgroup that finishes it last.  Within a workgroup the
// tiles of a block are dealt to four waves that run on their own: a wave keeps a ring of tiles of its own in LDS, filled by
// 16-byte global->LDS loads, and waits for nothing but its own loads, so that 16 to 32 KB per wave, up to 128 KB per CU,
// are always on their way.
//
// A wave computes S^T = K Q^T and O^T = V^T P^T with 16x16x32 MFMAs, columns on the N side: a lane then owns one
// column, its scores are laid out as the second product's operand needs them, and the rescale factor is one number per
// lane.  The running maximum moves only when a score exceeds it by more than 2^8 (in base 2), so most tiles need neither an
// exchange between lanes nor a rescale; probabilities up to 2^8 in bf16 and sums in fp32 cancel in the final division.
//
// Many rows (chunk_attn_kernel): the loop of the contiguous cache's attention (attend.h), 256 columns a workgroup, with the
// key tiles of all (sequence, row tile, kv head) blocks in equal ranges, and pieces put together as above.
#include "attend.h"
#include "paged.h"

namespace {

constexpr int KEYS = 32;                      // of a tile of few_attn_kernel
constexpr int WAVES = 4;
constexpr int START = 4;                      // units that a block costs besides its tiles: its queries, first loads and result

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
__device__ __forceinline__ const char* scalar_ptr(const char* p) {
    return (const char*)uniform((int64_t)(uintptr_t)p);
}

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
    constexpr bool Q_LDS = NC * KS > 8;       // the queries' fragments do not fit the registers
    __shared__ __align__(1024) char ring[WAVES][RING];
    __shared__ int64_t pre[CC_PAGED_MAX_N + 1];
    __shared__ int64_t wave_sum[WAVES];
    __shared__ float2 ml[WAVES][COLS];
    __shared__ bf16x8 qs[Q_LDS ? NC : 1][Q_LDS ? KS : 1][64];
    __shared__ int last_here;
    static_assert(COLS * D_H * 4 <= RING, "a wave's sums fit its ring");
    const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
    const int c16 = lane & 15, kg = lane >> 4;

    // ---- units before every sequence of the batch ----
    {
        int64_t carry = 0;
        for (int i0 = 0; i0 < a.n; i0 += 64 * WAVES) {
            const int i = i0 + tid;
            int64_t u = 0;
            if (i < a.n) {
                const batch_seq s = seq_of(a, i);
                if (s.n > 0) {
                    const tile_span v = visible_tiles(s.L - s.n, s.L, a.window, a.sinks, KEYS);
                    u = (int64_t)((s.n * a.g + COLS - 1) / COLS) * a.H_kv * (v.count + START);
                }
            }
            int64_t inc = u;
            for (int off = 1; off < 64; off <<= 1) {
                const int64_t v = __shfl_up(inc, off);
                if (lane >= off) inc += v;
            }
            if (lane == 63) wave_sum[w] = inc;
            __syncthreads();
            int64_t base = carry;
            for (int j = 0; j < WAVES; ++j) {
                if (j < w) base += wave_sum[j];
                carry += wave_sum[j];
            }
            if (i < a.n) pre[i] = base + inc - u;
            __syncthreads();
        }
        if (tid == 0) pre[a.n] = carry;
        __syncthreads();
    }
    const int64_t total = uniform(pre[a.n]);
    const int64_t per = max((int64_t)per_min, (total + gridDim.x - 1) / gridDim.x);
    const int range = blockIdx.x;
    int64_t u = range * per;
    const int64_t stop = min(u + per, total);

    // ---- lane constants: loads (row and swizzled chunk) and fragment addresses ----
    // K: chunk c of row r at slot c ^ kswz(r); V: the 32-byte pair of chunks dt at pair dt ^ vswz(r).
    auto kswz = [](int r) { return D_H == 128 ? (r & 15) : ((r >> 1) & 7); };
    auto vswz = [](int r) { return D_H == 128 ? (r & 7) : ((r >> 1) & 3); };
    const int l_row = lane / CPR, l_c = lane % CPR;
    const uint32_t st_b = (uint32_t)a.st_tok * 2;
    uint32_t k_off[HL], v_off[HL];                        // from the first of 16 rows, of the lane's 16 bytes of load i
#pragma unroll
    for (int i = 0; i < HL; ++i) {
        const int r = i * RPI + l_row;
        k_off[i] = r * st_b + (l_c ^ kswz(r)) * 16;
        v_off[i] = r * st_b + (l_c ^ (2 * vswz(r))) * 16;
    }
    char* const my_ring = ring[w];
    const uint32_t ring_at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)my_ring;
    uint32_t kaddr[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kaddr[ks] = ring_at + c16 * ROW + (((ks * 4 + kg) ^ kswz(c16)) << 4);
    const int v_row = 4 * kg + (c16 >> 2);
    const uint32_t v_base = ring_at + TILE + v_row * ROW + ((((c16 & 3) >> 1) ^ (2 * vswz(v_row))) << 4) + (c16 & 1) * 8;
    uint32_t vaddr[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) vaddr[dt] = v_base ^ (dt << 5);

    const uint32_t q_at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)&qs[0][0][lane];

    while (u < stop) {
        // ---- the block that unit u lies in ----
        int b = 0;
        for (int i = lane; i - lane < a.n; i += 64) b += __popcll(__ballot(i < a.n && pre[min(i, a.n - 1) + 1] <= u));
        b = uniform(b);
        const batch_seq sq = seq_of(a, b);
        const int row0 = uniform(sq.row0), n_new = uniform(sq.n), s = uniform(sq.s), L = uniform(sq.L);
        const int first = L - n_new;
        const tile_span span = visible_tiles(first, L, a.window, a.sinks, KEYS);
        const int64_t seq0 = uniform(pre[b]);
        const int len = span.count + START;
        const int which = (int)((u - seq0) / len), blk = which / a.H_kv, h = which - blk * a.H_kv;
        const int64_t u0 = seq0 + (int64_t)which * len, u1 = u0 + len;
        const int ta = (int)max((int64_t)0, u - u0 - START), te = (int)(min(u1, stop) - u0 - START);
        const bool opened_here = u0 + START >= range * per;
        u = u1;
        if (te <= ta) continue;

        // ---- queries: B operand of the scores ----
        bf16x8 qf[Q_LDS ? 1 : NC][KS];
        int limit[NC], under[NC];                          // the newest key a column sees; keys up to `under` left its window
        int most = -1, least = 0x7fffffff;                 // positions of the block's rows
#pragma unroll
        for (int nc = 0; nc < NC; ++nc) {
            const int col = blk * COLS + nc * 16 + c16, i = col / a.g, hg = col - i * a.g;
            const bool valid = i < n_new;
            limit[nc] = valid ? max(first + i, -1) : -1;
            under[nc] = a.window > 0 ? limit[nc] - a.window : (int)0x80000000;
            most = max(most, limit[nc]);
            if (valid) least = min(least, limit[nc]);
            const bf16_t* qp = a.q + ((int64_t)(row0 + (valid ? i : 0)) * a.H_q + h * a.g + (valid ? hg : 0)) * D_H + 8 * kg;
            if constexpr (Q_LDS) {
                if (nc == w) {
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) qs[nc][ks][lane] = *reinterpret_cast<const bf16x8*>(qp + ks * 32);
                }
            } else {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) qf[nc][ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 32);
            }
        }
        if constexpr (Q_LDS) __syncthreads();
        for (int off = 8; off > 0; off >>= 1) {
            most = max(most, __shfl_xor(most, off));
            least = min(least, __shfl_xor(least, off));
        }
        most = uniform(most);
        least = uniform(least);

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
        const in_pages::table_t row_table = (in_pages::table_t)(a.p.table + s * a.p.st_table);
        const int64_t head_off = (int64_t)h * a.st_head;
        // The two pages of a tile (16 keys each, in one page), asked for a tile ahead of the loads that need them.
        struct pages { int a, b; };
        auto pages_of = [&](int k) __attribute__((always_inline)) -> pages {
            const int key0 = tile_key(k), end = max(L - 1, 0);
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
        auto load = [&](const bf16_t* base, rows16 r, const uint32_t* off16, char* dst) __attribute__((always_inline)) {
            const char* src = (const char*)base + r.at;
            if (r.rmax == 15) {
                static_for<HL>([&](auto ic) __attribute__((always_inline)) {
                    constexpr int i = decltype(ic)::value;
                    uint32_t off = off16[i];
                    asm volatile("" : "+v"(off));
                    stream16<i * 1024>(scalar_ptr(src - i * 1024) + off, dst);
                });
            } else {
                if (r.rmax < 0) src = (const char*)a.zeros;
                static_for<HL>([&](auto ic) __attribute__((always_inline)) {
                    constexpr int i = decltype(ic)::value;
                    const int row = i * RPI + l_row;
                    uint32_t off = off16[i] - (uint32_t)(row - min(row, max(r.rmax, 0))) * st_b;
                    asm volatile("" : "+v"(off));
                    stream16<i * 1024>(scalar_ptr(src - i * 1024) + off, dst);
                });
            }
        };
        auto stage_of = [&](int k) { return my_ring + (k % NS) * 2 * TILE; };
        {
            pages pg[NS];
#pragma unroll
            for (int k = 0; k < NS; ++k) pg[k] = pages_of(min(k, max(nt - 1, 0)));
#pragma unroll
            for (int k = 0; k < NS; ++k)
                if (k < nt) {
                    const int key0 = tile_key(k);
                    const rows16 x = rows_of(key0, pg[k].a), y = rows_of(key0 + 16, pg[k].b);
                    load(a.K, x, k_off, stage_of(k));
                    load(a.K, y, k_off, stage_of(k) + TILE / 2);
                    load(a.V, x, v_off, stage_of(k) + TILE);
                    load(a.V, y, v_off, stage_of(k) + TILE + TILE / 2);
                }
        }
        pages pg_next = pages_of(max(0, min(NS, nt - 1)));
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

        for (int k = 0; k < nt; ++k) {
            const int key0 = tile_key(k), rem = nt - 1 - k;
            const uint32_t stage = (uint32_t)(k % NS) * 2 * TILE;
            wait_k(rem);
            bf16x8 kf[2][KS];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                kf[0][ks] = lds_read_b128_at<0>(kaddr[ks] + stage);
                kf[1][ks] = lds_read_b128_at<16 * ROW>(kaddr[ks] + stage);
            }
            if constexpr (KS == 4)
                asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(kf[0][0]), "+v"(kf[1][0]), "+v"(kf[0][1]), "+v"(kf[1][1]), "+v"(kf[0][2]),
                             "+v"(kf[1][2]), "+v"(kf[0][3]), "+v"(kf[1][3])
                             :: "memory");
            else
                asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(kf[0][0]), "+v"(kf[1][0]), "+v"(kf[0][1]), "+v"(kf[1][1])::"memory");
            const rows16 x = rows_of(tile_key(k + NS), pg_next.a), y = rows_of(tile_key(k + NS) + 16, pg_next.b);
            if (rem >= NS) {
                load(a.K, x, k_off, stage_of(k));
                load(a.K, y, k_off, stage_of(k) + TILE / 2);
            }
            f32x4 sc[NC][2];
#pragma unroll
            for (int nc = 0; nc < NC; ++nc) {
                if constexpr (Q_LDS) {
                    static_assert(!Q_LDS || KS == 4, "four fragments a column block");
                    const uint32_t at = q_at + nc * KS * 1024;
                    qf[0][0] = lds_read_b128_at<0>(at);
                    qf[0][1] = lds_read_b128_at<1024>(at);
                    qf[0][KS - 2] = lds_read_b128_at<(KS - 2) * 1024>(at);
                    qf[0][KS - 1] = lds_read_b128_at<(KS - 1) * 1024>(at);
                    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(qf[0][0]), "+v"(qf[0][1]), "+v"(qf[0][KS - 2]), "+v"(qf[0][KS - 1]));
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    sc[nc][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
                        sc[nc][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t][ks], qf[Q_LDS ? 0 : nc][ks], sc[nc][t], 0, 0, 0);
                }
            }
            // ---- mask: keys behind a row, or in front of its window and no sink ----
            if (key0 + KEYS - 1 > least || (a.window > 0 && key0 <= most - a.window && key0 + KEYS > a.sinks)) {
#pragma unroll
                for (int nc = 0; nc < NC; ++nc)
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            const int key = key0 + t * 16 + 4 * kg + v;
                            // (no short circuits: selects, not branches)
                            const bool out = (key > limit[nc]) | ((key <= under[nc]) & (key >= a.sinks));
                            sc[nc][t][v] = out ? -INFINITY : sc[nc][t][v];
                        }
            }
            // ---- softmax in base 2, the scale folded into the exponent ----
            bf16x8 pf[NC];
#pragma unroll
            for (int nc = 0; nc < NC; ++nc) {
                float mx = -INFINITY;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int v = 0; v < 4; ++v) mx = fmaxf(mx, sc[nc][t][v]);
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
                        const float p = __builtin_amdgcn_exp2f(fmaf(sc[nc][t][v], a.scale_log2, -ref));
                        l_run[nc] += p;
                        pf[nc][t * 4 + v] = (bf16_t)p;
                    }
            }
            // ---- O^T += V^T P^T: the 32 keys in the order in which a lane holds its scores ----
            wait_v(rem);
            bf16x4 va[DT], vb[DT];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                va[dt] = lds_read_tr_at<0>(vaddr[dt] + stage);
                vb[dt] = lds_read_tr_at<16 * ROW>(vaddr[dt] + stage);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(va[0]), "+v"(vb[0]), "+v"(va[1]), "+v"(vb[1]), "+v"(va[2]), "+v"(vb[2]),
                         "+v"(va[3]), "+v"(vb[3])
                         :: "memory");
            if constexpr (DT == 8)
                asm volatile("" : "+v"(va[4]), "+v"(vb[4]), "+v"(va[5]), "+v"(vb[5]), "+v"(va[6]), "+v"(vb[6]), "+v"(va[7]), "+v"(vb[7])::"memory");
            if (rem >= NS) {
                load(a.V, x, v_off, stage_of(k) + TILE);
                load(a.V, y, v_off, stage_of(k) + TILE + TILE / 2);
            }
            pg_next = pages_of(min(k + 1 + NS, nt - 1));
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const bf16x8 vf = __builtin_shufflevector(va[dt], vb[dt], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int nc = 0; nc < NC; ++nc)
                    acc[dt][nc] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[nc], acc[dt][nc], 0, 0, 0);
            }
        }

        // ---- the four waves' sums together: as the registers lie, [dt][nc][lane] ----
        wait_loads<0>();
#pragma unroll
        for (int nc = 0; nc < NC; ++nc) {
            float l = l_run[nc];
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            if (kg == 0) ml[w][nc * 16 + c16] = make_float2(m_run[nc], l);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
                *reinterpret_cast<f32x4*>(my_ring + ((dt * NC + nc) * 64 + lane) * 16) = acc[dt][nc];
        }
        __syncthreads();
        const bool whole = ta == 0 && te == span.count;
        // pieces: a range leaves at most two, of the block it starts in and of a later one
        float* const piece = a.part + (int64_t)(2 * range + (opened_here ? 1 : 0)) * COLS * (D_H + 2);
#pragma unroll
        for (int nc = 0; nc < NC; ++nc) {
            float2 x[WAVES];
            float m = -INFINITY, l = 0.0f;
#pragma unroll
            for (int j = 0; j < WAVES; ++j) {
                x[j] = ml[j][nc * 16 + c16];
                m = fmaxf(m, x[j].x);
            }
            const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int j = 0; j < WAVES; ++j) {
                x[j].x = __builtin_amdgcn_exp2f(x[j].x - ref);
                l += x[j].x * x[j].y;
            }
            const int col = blk * COLS + nc * 16 + c16, i = col / a.g, hg = col - i * a.g;
            const float inv = l > 0.0f ? 1.0f / l : 0.0f;
            for (int dt = w; dt < DT; dt += WAVES) {
                f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < WAVES; ++j)
                    r += x[j].x * *reinterpret_cast<const f32x4*>(ring[j] + ((dt * NC + nc) * 64 + lane) * 16);
                if (!whole) {
                    put(piece + ((dt * NC + nc) * 128 + lane) * 2, r[0], r[1]);
                    put(piece + ((dt * NC + nc) * 128 + 64 + lane) * 2, r[2], r[3]);
                } else if (i < n_new) {
                    bf16x4 out;
#pragma unroll
                    for (int e = 0; e < 4; ++e) out[e] = (bf16_t)(r[e] * inv);
                    *reinterpret_cast<bf16x4*>(a.o + ((int64_t)(row0 + i) * a.H_q + h * a.g + hg) * D_H + dt * 16 + 4 * kg) = out;
                }
            }
            if (!whole && w == 0 && kg == 0) put(piece + COLS * D_H + (nc * 16 + c16) * 2, m, l);
        }
        if (whole) {
            __syncthreads();                               // the rings are free again
            continue;
        }
        // ---- a cut block: the workgroup that comes last adds the pieces, in the order of their keys ----
        const int w0 = (int)((u0 + START) / per), w1 = (int)((u1 - 1) / per);
        wait_loads<0>();                                   // the piece is written
        __syncthreads();
        if (tid == 0) {
            const int before = __hip_atomic_fetch_add(&a.arrived[w0], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            last_here = before == w1 - w0;
            if (last_here) __hip_atomic_store(&a.arrived[w0], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!last_here) continue;
        for (int e = tid; e < DT * NC * 64; e += 64 * WAVES) {
            const int ln = e & 63, dn = e >> 6, nc = dn % NC, dt = dn / NC;
            const int cc = nc * 16 + (ln & 15), col = blk * COLS + cc, i = col / a.g, hg = col - i * a.g;
            if (i >= n_new) continue;
            float m = -INFINITY, l = 0.0f;
            f32x4 r = {0.f, 0.f, 0.f, 0.f};
            for (int j = w0; j <= w1; ++j) {
                const float* pc = a.part + (int64_t)(2 * j + (j == w0 ? 1 : 0)) * COLS * (D_H + 2);
                const float2 x = get(pc + COLS * D_H + cc * 2), va = get(pc + (dn * 128 + ln) * 2), vb = get(pc + (dn * 128 + 64 + ln) * 2);
                const f32x4 v = {va.x, va.y, vb.x, vb.y};
                const float mn = fmaxf(m, x.x), ref = mn == -INFINITY ? 0.0f : mn;
                const float keep = __builtin_amdgcn_exp2f(m - ref), f = __builtin_amdgcn_exp2f(x.x - ref);
                l = l * keep + x.y * f;
                r = r * keep + v * f;
                m = mn;
            }
            const float inv = l > 0.0f ? 1.0f / l : 0.0f;
            bf16x4 out;
#pragma unroll
            for (int k = 0; k < 4; ++k) out[k] = (bf16_t)(r[k] * inv);
            *reinterpret_cast<bf16x4*>(a.o + ((int64_t)(row0 + i) * a.H_q + h * a.g + hg) * D_H + dt * 16 + 4 * (ln >> 4)) = out;
        }
    }
}

constexpr int CHUNK_START = 5;                // units of a block besides its key tiles, as in the even grids of attention.hip
constexpr int MAX_BLOCKS = CC_PAGED_MAX_COLUMNS / 256 + CC_PAGED_MAX_N;

// A workgroup of eight waves per range.  Blocks are numbered e0(b) + row tile with e0(b) = floor(columns in front of b / 256) + b:
// at least as many numbers as sequence b has row tiles, the unused ones of length 0, and no scan is needed to find one.
template <int D_H>
__global__ __launch_bounds__(512, 1) void chunk_attn_kernel(paged_args a, int per_min) {
    __shared__ __align__(16) bf16_t smem[LDS_TILES * BN_KEYS * D_H];
    __shared__ int simd_waves[4], group_waves[2], wave_units[8], last_here;
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
        int carry = 0;
        for (int i0 = 0; i0 < blocks; i0 += 512) {
            const int e = i0 + tid;
            int len = 0;
            if (e < blocks) {
                const int b = sequence_of(e);
                const int c0 = (e - e0[b]) * 256, n = rows_of[b], first = len_of[b] - n;
                if (c0 >= 0 && c0 < n * a.g) {
                    const int end = first + min(n - 1, (c0 + 255) / a.g) + 1;
                    len = visible_tiles(first + c0 / a.g, max(end, 0), a.window, a.sinks, BN_KEYS).count + CHUNK_START;
                }
            }
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
    }
    const int blocks = uniform(min(e0[a.n], MAX_BLOCKS)), head_units = uniform(pre[blocks]);
    const int64_t total = (int64_t)head_units * a.H_kv;
    const int n_wg = gridDim.x;
    const int64_t per = max((int64_t)per_min, (total + n_wg - 1) / n_wg);
    // workgroup ids go round-robin to the 8 XCDs: each gets consecutive ranges
    const int x = blockIdx.x & 7, xq = n_wg >> 3, xr = n_wg & 7;
    const int range = x * xq + min(x, xr) + (int)(blockIdx.x >> 3);
    int64_t u = range * per;
    const int64_t stop = min(u + per, total);
    while (u < stop) {
        const int kvh = (int)(u / head_units), uh = (int)(u - (int64_t)kvh * head_units);
        int e = 0;
        for (int i = lane; i - lane < blocks; i += 64) e += __popcll(__ballot(i < blocks && pre[min(i, blocks - 1) + 1] <= uh));
        e = uniform(e);
        const int b = uniform(sequence_of(e));
        const int b0 = uniform(pre[e]), len = uniform(pre[e + 1]) - b0, rt = e - uniform(e0[b]);
        const batch_seq sq = seq_of(a, b);
        const int n_new = uniform(sq.n), L = uniform(sq.L), first = L - n_new;
        const int ta = max(0, uh - b0 - CHUNK_START), te = (int)min((int64_t)len, uh - b0 + (stop - u)) - CHUNK_START;
        const int64_t u0 = (int64_t)kvh * head_units + b0;
        u = u0 + len;
        if (te <= ta) continue;
        in_pages keys;
        keys.table = (in_pages::table_t)(a.p.table + uniform(sq.s) * a.p.st_table);
        keys.K = a.K, keys.V = a.V, keys.zeros = a.zeros;
        keys.st_page = a.st_page, keys.st_tok = a.st_tok, keys.sh = a.st_head;
        keys.shift = a.p.shift, keys.n_pages = a.p.n_pages, keys.L = L, keys.first = first, keys.row0 = uniform(sq.row0);
        keys.window = a.window, keys.sinks = a.sinks;
        const int end = first + min(n_new - 1, (rt * 256 + 255) / a.g) + 1;
        keys.span = visible_tiles(first + rt * 256 / a.g, max(end, 0), a.window, a.sinks, BN_KEYS);
        const bool whole = ta == 0 && te == keys.span.count;
        const int w0 = (int)((u0 + CHUNK_START) / per), w1 = (int)((u0 + len - 1) / per);
        attend<D_H, true, uint32_t>(keys, a.q, n_new, a.H_q, a.g, a.o, a.scale_log2, a.part, smem, grp, widx, kvh, rt, ta, te - ta,
                                    whole ? -1 : 2 * range + (w0 == range ? 1 : 0));
        if (whole) continue;
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
        // a thread holds what the lane that left it did: half of a column's sums
        constexpr int NG = D_H / 8;
        const int col = rt * 256 + w * 32 + (lane & 31), mi = col / a.g, hg = col - mi * a.g;
        if (mi < n_new) {
            f32x4 acc[NG];
            float m = -INFINITY, l = 0.0f;
#pragma unroll
            for (int k = 0; k < NG; ++k) acc[k] = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int j = w0; j <= w1; ++j) {
                const float* pp = a.part + (int64_t)(2 * j + (j == w0 ? 1 : 0)) * 256 * (D_H + 4) + w * 32 * (D_H + 4);
                const float2 ml = get(pp + 32 * D_H + lane * 2);
                float2 v[NG][2];
#pragma unroll
                for (int k = 0; k < NG; ++k) {
                    v[k][0] = get(pp + k * 256 + lane * 2);
                    v[k][1] = get(pp + k * 256 + 128 + lane * 2);
                }
                const float mn = fmaxf(m, ml.x), ref = mn == -INFINITY ? 0.0f : mn;
                const float keep = __builtin_amdgcn_exp2f(m - ref), f = __builtin_amdgcn_exp2f(ml.x - ref);
                l = l * keep + ml.y * f;
                m = mn;
#pragma unroll
                for (int k = 0; k < NG; ++k) acc[k] = acc[k] * keep + f32x4{v[k][0].x, v[k][0].y, v[k][1].x, v[k][1].y} * f;
            }
            const float inv = l > 0.0f ? 1.0f / l : 0.0f;
            bf16_t* op = a.o + ((int64_t)(keys.row0 + mi) * a.H_q + kvh * a.g + hg) * D_H + 4 * (lane >> 5);
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                bf16x4 r;
#pragma unroll
                for (int i = 0; i < 4; ++i) r[i] = (bf16_t)(acc[k][i] * inv);
                *reinterpret_cast<bf16x4*>(op + 8 * k) = r;
            }
        }
    }
}

}  // namespace

void cc_launch_paged_attention(const bf16_t* q, const cc_new_rows& r, const cc_page_pool& p, const cc_paged_kv& kv, int window,
                               int sinks, const cc_model_desc& m, const cc_paged_scratch& ws, bf16_t* o, hipStream_t s) {
    if (r.rows <= 0 || r.n <= 0) return;
    const int g = m.H_q / m.H_kv;
    paged_args a = {q, o, r.start, r.seq, r.n, r.rows, cc_view(p), (const bf16_t*)kv.K, (const bf16_t*)kv.V, kv.stride_page,
                    kv.stride_token, kv.stride_head, window, sinks, m.H_q, m.H_kv, g,
                    1.4426950408889634f / sqrtf((float)m.d_h), ws.zeros,
                    (float*)p.work + cc_page_work_layout(p.n_pages, p.n_seqs).attn, ws.arrived};
    const int grid = std::min(cc_device_cus(), CC_PAGED_WGS);
    const int64_t columns = (int64_t)std::min(r.max_new, r.rows) * g;
    const int per_min = 2 * WAVES + START;
    if (columns > 64) {
        const int chunk_min = 3 + CHUNK_START;
        if (m.d_h == 128) hipLaunchKernelGGL(chunk_attn_kernel<128>, dim3(grid), dim3(512), 0, s, a, chunk_min);
        else hipLaunchKernelGGL(chunk_attn_kernel<64>, dim3(grid), dim3(512), 0, s, a, chunk_min);
        return;
    }
#define CC_FEW(D, NC) hipLaunchKernelGGL((few_attn_kernel<D, NC>), dim3(grid), dim3(64 * WAVES), 0, s, a, per_min)
    if (m.d_h == 128) {
        if (columns <= 16) CC_FEW(128, 1);
        else if (columns <= 32) CC_FEW(128, 2);
        else CC_FEW(128, 4);
    } else {
        if (columns <= 16) CC_FEW(64, 1);
        else if (columns <= 32) CC_FEW(64, 2);
        else CC_FEW(64, 4);
    }
#undef CC_FEW
}
