// Pages of the answer phase: growing, forking, freeing and compacting what sequences hold, the copies this
// takes in every layer, and the rotary step that writes new keys and values into pages.
//
// The bookkeeping of a call is one workgroup's: its lists are short, every decision depends on a scan over them, and
// what it costs is the latency of a few dependent passes.  Free pages are handed out lowest first in the order of the
// list, so results do not depend on the order in which threads run; the only atomics add to counts.
// The copies are left as a list in the pool's scratch and made by a second launch over all layers.
#include "paged.h"

namespace {

constexpr int NT = 1024;
typedef int quad __attribute__((ext_vector_type(4), aligned(4)));   // of a list that is aligned to its entries only
constexpr int ROWS = 8;                      // entries of a table row that a lane loads before it stores the first

// Inclusive scan over the workgroup; every thread comes here.  part: NT / 64 entries of LDS.
template <class T>
__device__ __forceinline__ T block_scan(T v, T* part, T& total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int off = 1; off < 64; off <<= 1) {
        const T u = __shfl_up(v, off);
        if (lane >= off) v += u;
    }
    __syncthreads();                                  // the last scan's part has been read
    if (lane == 63) part[w] = v;
    __syncthreads();
    T base = 0, sum = 0;
    for (int i = 0; i < NT / 64; ++i) {
        if (i < w) base += part[i];
        sum += part[i];
    }
    total = sum;
    return base + v;
}

enum { BAD_INDEX = 1, BAD_LENGTH = 2, NO_PAGES = 4 };
__device__ __forceinline__ int status_of(int bad) {
    return bad & BAD_INDEX ? CC_ERR_IDX : bad & BAD_LENGTH ? CC_ERR_SHAPE : bad & NO_PAGES ? CC_ERR_WORKSPACE : CC_OK;
}
__device__ __forceinline__ void finish(int32_t* status, int32_t* host, int bad) {
    if (threadIdx.x) return;
    const int st = status_of(bad);
    *status = st;
    if (host) *host = st;
}

// Sequences that a list has named: a bit each.
struct seen_bits {
    uint32_t word[65536 / 32];
    __device__ __forceinline__ void clear() {
        for (int i = threadIdx.x; i < 65536 / 32; i += NT) word[i] = 0;
    }
    // whether s is a sequence and named for the first time
    __device__ __forceinline__ bool first(int s, int n_seqs) {
        return (unsigned)s < (unsigned)n_seqs && !(atomicOr(&word[s >> 5], 1u << (s & 31)) >> (s & 31) & 1);
    }
};

// A decode loop's every step comes here, and what it costs is its chain of round trips to memory.  So a thread keeps its entry
// of the list in registers from its checks to its writes, the counts of the first pages are asked for before they are needed, and the pages
// found wait in LDS; only lists of more than NT entries go through the pool's scratch.  36 entries with a copy each: 8.2 us (9.6 with
// everything in scratch and a wave per entry); 1000 entries of three pages, a launch's 6 us among them, 25 (64).
__global__ __launch_bounds__(NT) void grow_kernel(cc_pool_view p, const int32_t* __restrict__ seq,
                                                  const int32_t* __restrict__ n_new, int n, int32_t* work, cc_page_work w,
                                                  int32_t* status, int32_t* host) {
    constexpr int PER = 32;                           // pages a thread looks at in a step
    constexpr int LIST = 4096;                        // pages found that LDS holds
    constexpr int FEW = 5;                            // pages that a thread hands to its entry by itself
    __shared__ seen_bits seen;
    __shared__ int bad, big, list[LIST];
    __shared__ int64_t part[NT / 64];
    __shared__ int part32[NT / 64];
    __shared__ struct { int64_t row; int at, all; } hand[NT];
    const int tid = threadIdx.x, lane = tid & 63, page = 1 << p.shift;
    // nothing changes but what the append looks at: who asked for tokens and got none
    auto refuse = [&](int why) {
        if (p.refused)
            for (int i = tid; i < n; i += NT)
                if ((unsigned)seq[i] < (unsigned)p.n_seqs && n_new[i] != 0) p.refused[seq[i]] = status_of(why);
        finish(status, host, why);
    };
    // the free ones among the thread's pages from p0 on
    auto look = [&](int64_t p0) -> unsigned {
        const int64_t a = p0 + (int64_t)tid * PER;
        unsigned free = 0;
        if (a + PER <= p.n_pages) {
            quad x[PER / 4];
#pragma unroll
            for (int k = 0; k < PER / 4; ++k) x[k] = *reinterpret_cast<const quad*>(p.refs + a + 4 * k);
#pragma unroll
            for (int k = 0; k < PER; ++k) free |= (unsigned)(x[k / 4][k % 4] == 0) << k;
        } else if (a < p.n_pages) {
#pragma unroll
            for (int k = 0; k < PER; ++k) free |= (unsigned)(p.refs[min(a + k, (int64_t)p.n_pages - 1)] == 0 && a + k < p.n_pages) << k;
        }
        return free;
    };
    const int s0 = tid < n ? seq[tid] : 0, c0 = tid < n ? n_new[tid] : 0;
    const unsigned free0 = look(0);
    seen.clear();
    if (tid == 0) bad = big = 0, work[0] = 0;
    __syncthreads();

    // t: twice the pages that an entry takes, plus one if one of them is for a copy; before: pages and copies (the upper part) of
    // the entries in front of it
    struct entry { int s, c, L, t, old; int64_t before; };
    auto entry_of = [&](int i) -> entry {
        entry e = {};
        if (i < n) e.s = seq[i], e.c = n_new[i], e.L = p.len[e.s], e.t = work[w.take + i];
        return e;
    };
    constexpr int64_t COPY = (int64_t)1 << 40;
    entry mine = {};
    for (int i0 = 0; i0 < n; i0 += NT) {
        const int i = i0 + tid;
        entry e = {};
        int wrong = 0;
        if (i < n) {
            e.s = i0 == 0 ? s0 : seq[i], e.c = i0 == 0 ? c0 : n_new[i];
            if (!seen.first(e.s, p.n_seqs)) {
                wrong = BAD_INDEX;
            } else {
                e.L = p.len[e.s];
                const int64_t to = (int64_t)e.L + e.c;
                if (e.c < 0 || e.L < 0) wrong = BAD_INDEX;
                else if (to > (int64_t)p.max_pages << p.shift) wrong = BAD_LENGTH;
                else {
                    const int have = (e.L + page - 1) >> p.shift;
                    int copy = 0;
                    if (e.c > 0 && (e.L & (page - 1))) {
                        e.old = p.table[e.s * p.st_table + have - 1];
                        if ((unsigned)e.old >= (unsigned)p.n_pages) wrong = BAD_INDEX;
                        else copy = p.refs[e.old] > 1;
                    }
                    e.t = 2 * ((int)((to + page - 1) >> p.shift) - have + copy) + copy;
                }
            }
        }
        if (wrong) atomicOr(&bad, wrong);
        if (i0 == 0) mine = e;
        else if (i < n) work[w.take + i] = e.t;
    }
    __syncthreads();
    if (bad) return refuse(bad);

    int64_t carry = 0;
    for (int i0 = 0; i0 < n; i0 += NT) {
        const int i = i0 + tid, t = i0 == 0 ? mine.t : i < n ? work[w.take + i] : 0;
        const int64_t own = (t >> 1) + (t & 1) * COPY;
        int64_t sum;
        const int64_t before = carry + block_scan(own, part, sum) - own;
        if (i0 == 0) {
            mine.before = before;
        } else if (i < n) {
            work[w.first + i] = (int)min(before & (COPY - 1), (int64_t)1 << 30);
            work[w.copy_at + i] = (int)(before >> 40);
        }
        carry += sum;
    }
    const int64_t total = carry & (COPY - 1);
    const int copies = (int)(carry >> 40);

    // the lowest free pages until there are enough (a step is a round trip and a scan whatever it looks at: behind 150000 pages
    // in use 97 us with 8 a thread, 33 with 32)
    int found = 0;
    for (int64_t p0 = 0; p0 < p.n_pages && found < total; p0 += NT * PER) {
        unsigned free = p0 == 0 ? free0 : look(p0);
        int sum, at = found + block_scan((int)__popc(free), part32, sum) - (int)__popc(free);
#pragma unroll 1
        for (; free; free &= free - 1, ++at) {
            const int q = (int)(p0 + (int64_t)tid * PER + __ffs(free) - 1);
            if (at < LIST) list[at] = q;
            else if (at < total) work[w.list + at] = q;
        }
        found += sum;
    }
    __syncthreads();
    if (found < total) return refuse(NO_PAGES);
    auto page_at = [&](int k) -> int { return k < LIST ? list[k] : work[w.list + k]; };

    for (int i0 = 0; i0 < n; i0 += NT) {
        const int i = i0 + tid;
        entry e = mine;
        if (i0 > 0) {
            e = entry_of(i);
            if (i < n) e.before = work[w.first + i] + work[w.copy_at + i] * COPY;
        }
        const int copy = e.t & 1, all = e.t >> 1, have = (e.L + page - 1) >> p.shift, at = (int)(e.before & (COPY - 1));
        int32_t* row = p.table + e.s * p.st_table + have - copy;
        if (copy) {
            const int k = (int)(e.before >> 40), old = i0 == 0 ? e.old : row[0];
            work[w.src + k] = old;
            work[w.dst + k] = page_at(at);
            work[w.rows + k] = e.L & (page - 1);
            atomicSub(&p.refs[old], 1);
        }
#pragma unroll 1
        for (int k = 0; k < min(all, FEW); ++k) {
            const int q = page_at(at + k);
            row[k] = q;
            p.refs[q] = 1;
        }
        if (i < n) {
            p.len[e.s] = e.L + e.c;
            if (p.refused && e.c > 0) p.refused[e.s] = 0;
        }
        // more than a few: by whole waves
        hand[tid] = {e.s * p.st_table + have - copy, at, all};
        if (all > FEW) big = 1;
        __syncthreads();
        if (big)
            for (int j = tid >> 6; j < min(NT, n - i0); j += NT / 64)
                for (int k = FEW + lane; k < hand[j].all; k += 64) {
                    const int q = page_at(hand[j].at + k);
                    p.table[hand[j].row + k] = q;
                    p.refs[q] = 1;
                }
        __syncthreads();
    }
    if (tid == 0) work[0] = copies;
    finish(status, host, 0);
}

// A source that is listed many times is counted first: its pages' counts are raised once, by the entry that was the first to
// count it (eight answers from each of four contexts: 13.3 us with every entry adding for itself).
__global__ __launch_bounds__(NT) void fork_kernel(cc_pool_view p, const int32_t* __restrict__ src,
                                                  const int32_t* __restrict__ dst, int n, int32_t* work, cc_page_work w,
                                                  int32_t* status, int32_t* host) {
    __shared__ seen_bits seen;
    __shared__ int bad;
    const int tid = threadIdx.x, page = 1 << p.shift;
    int32_t *copies = work + w.first, *len = work + w.take, *leads = work + w.copy_at;
    seen.clear();
    if (tid == 0) bad = 0;
    __syncthreads();
    for (int i = tid; i < n; i += NT) {
        const int s = src[i], d = dst[i];
        if ((unsigned)s >= (unsigned)p.n_seqs || !seen.first(d, p.n_seqs) || p.len[d] != 0) {
            atomicOr(&bad, BAD_INDEX);
        } else {
            copies[s] = 0;
            len[i] = cc_seq_len(p, s);                        // as it is at the call
        }
    }
    __syncthreads();
    if (bad) return finish(status, host, bad);
    for (int i = tid; i < n; i += NT) leads[i] = atomicAdd(&copies[src[i]], 1) == 0;
    __syncthreads();
    const int lane = tid & 63;
    for (int i = tid >> 6; i < n; i += NT / 64) {
        const int s = src[i], d = dst[i], L = len[i], held = (L + page - 1) >> p.shift, more = leads[i] ? copies[s] : 0;
        const int32_t* from = p.table + s * p.st_table;
        int32_t* to = p.table + d * p.st_table;
        for (int c0 = lane; c0 < held; c0 += 64 * ROWS) {
            int q[ROWS];
#pragma unroll
            for (int k = 0; k < ROWS; ++k) q[k] = from[min(c0 + 64 * k, held - 1)];
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                if (c0 + 64 * k >= held) break;
                to[c0 + 64 * k] = q[k];
                if (more && (unsigned)q[k] < (unsigned)p.n_pages) atomicAdd(&p.refs[q[k]], more);
            }
        }
        if (lane == 0) p.len[d] = L;
    }
    finish(status, host, 0);
}

__global__ __launch_bounds__(NT) void free_kernel(cc_pool_view p, const int32_t* __restrict__ seq, int n, int32_t* status,
                                                  int32_t* host) {
    __shared__ seen_bits seen;
    __shared__ int bad;
    const int tid = threadIdx.x, page = 1 << p.shift;
    seen.clear();
    if (tid == 0) bad = 0;
    __syncthreads();
    for (int i = tid; i < n; i += NT)
        if (!seen.first(seq[i], p.n_seqs)) atomicOr(&bad, BAD_INDEX);
    __syncthreads();
    if (bad) return finish(status, host, bad);
    const int lane = tid & 63;
    for (int i = tid >> 6; i < n; i += NT / 64) {
        const int s = seq[i], held = (cc_seq_len(p, s) + page - 1) >> p.shift;
        int32_t* row = p.table + s * p.st_table;
        for (int c0 = lane; c0 < held; c0 += 64 * ROWS) {
            int q[ROWS];
#pragma unroll
            for (int k = 0; k < ROWS; ++k) q[k] = row[min(c0 + 64 * k, held - 1)];
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                if (c0 + 64 * k >= held) break;
                row[c0 + 64 * k] = -1;
                if ((unsigned)q[k] < (unsigned)p.n_pages) atomicSub(&p.refs[q[k]], 1);
            }
        }
        if (lane == 0) {
            p.len[s] = 0;
            if (p.refused) p.refused[s] = 0;
        }
    }
    finish(status, host, 0);
}

// Which page goes where: the i-th used page at L or behind to the i-th free one in front of L.
__global__ __launch_bounds__(NT) void compact_plan_kernel(cc_pool_view p, int32_t* work, cc_page_work w, int32_t* status,
                                                          int32_t* host) {
    __shared__ int part[NT / 64];
    constexpr int PER = 8;
    const int tid = threadIdx.x;
    int mine = 0, live;
    for (int64_t a = tid; a < p.n_pages; a += NT) mine += p.refs[a] != 0;
    block_scan(mine, part, live);
    int holes = 0, movers = 0;
    for (int64_t p0 = 0; p0 < p.n_pages; p0 += NT * PER) {
        const int64_t a = p0 + (int64_t)tid * PER;
        unsigned hole = 0, move = 0;
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if (a + k < p.n_pages) {
                const bool used = p.refs[a + k] != 0;
                if (a + k < live ? !used : used) (a + k < live ? hole : move) |= 1u << k;
            }
        int sum;
        // holes in the low half of the sum, movers in the high one (at most 8192 of each a step)
        const int cnt = __popc(hole) + (__popc(move) << 16);
        const int before = block_scan(cnt, part, sum) - cnt;
        int h = holes + (before & 0xffff), m = movers + (before >> 16);
        for (; hole; hole &= hole - 1) work[w.dst + h++] = (int)(a + __ffs(hole) - 1);
        for (; move; move &= move - 1) work[w.src + m++] = (int)(a + __ffs(move) - 1);
        holes += sum & 0xffff;
        movers += sum >> 16;
    }
    __syncthreads();
    for (int i = tid; i < movers; i += NT) {
        const int from = work[w.src + i], to = work[w.dst + i];
        work[w.map + from] = to;
        work[w.rows + i] = 1 << p.shift;
        p.refs[to] = p.refs[from];
        p.refs[from] = 0;
    }
    if (tid == 0) {
        work[0] = movers;
        work[1] = live;
    }
    finish(status, host, 0);
}

// Entries of every sequence that name a moved page; a wave per sequence.
__global__ __launch_bounds__(256) void compact_table_kernel(cc_pool_view p, const int32_t* __restrict__ work, cc_page_work w) {
    const int s = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, live = work[1];
    if (s >= p.n_seqs) return;
    const int held = (cc_seq_len(p, s) + (1 << p.shift) - 1) >> p.shift;
    int32_t* row = p.table + s * p.st_table;
    for (int c = lane; c < held; c += 64) {
        const int q = row[c];
        if (q >= live && q < p.n_pages) row[c] = work[w.map + q];
    }
}

struct copy_args {
    void* ptr[2 * CC_PAGE_LAYERS];
    int32_t n_ptr;
};
// A workgroup takes a (copy, tensor) at a time: the copy's rows of all heads, eight pieces of 16 bytes a thread loaded before
// the first is stored, all past the caches.  Bound by HBM.
template <int D_H>
__global__ __launch_bounds__(256) void page_copy_kernel(copy_args a, const int32_t* __restrict__ work, cc_page_work w,
                                                        int H_kv, int page, int64_t st_page, int64_t st_tok, int64_t st_head) {
    constexpr int CPH = D_H / 8, NB = 8;
    const bool by_token = st_tok > st_head || H_kv == 1;
    const bool gapless = by_token ? st_tok == (int64_t)H_kv * D_H && (H_kv == 1 || st_head == D_H)
                                  : st_head == (int64_t)page * D_H && st_tok == D_H;
    const int64_t items = (int64_t)work[0] * a.n_ptr;
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
        const int i = (int)(it / a.n_ptr), t = (int)(it - (int64_t)i * a.n_ptr);
        const int rows = work[w.rows + i], units = rows * H_kv * CPH;
        bf16_t* base = (bf16_t*)a.ptr[t];
        const bf16_t* from = base + work[w.src + i] * st_page;
        bf16_t* to = base + work[w.dst + i] * st_page;
        const bool flat = gapless && (by_token || rows == page);
        auto place = [&](int u) -> int64_t {
            if (flat) return (int64_t)u * 8;
            const int c = u % CPH, r = u / CPH;
            const int tok = by_token ? r / H_kv : r % rows, h = by_token ? r % H_kv : r / rows;
            return tok * st_tok + h * st_head + c * 8;
        };
        for (int u0 = threadIdx.x; u0 < units; u0 += 256 * NB) {
            u32x4 x[NB];
            int64_t at[NB];
#pragma unroll
            for (int k = 0; k < NB; ++k) {
                at[k] = place(min(u0 + k * 256, units - 1));
                x[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from + at[k]));
            }
#pragma unroll
            for (int k = 0; k < NB; ++k)
                if (u0 + k * 256 < units) __builtin_nontemporal_store(x[k], reinterpret_cast<u32x4*>(to + at[k]));
        }
    }
}

__global__ __launch_bounds__(64) void check_rows_kernel(const int32_t* __restrict__ start, const int32_t* __restrict__ seq, int rows,
                                                        cc_pool_view p, int window, int sinks, int append, int32_t* flag) {
    const int b = blockIdx.x, lane = threadIdx.x, r0 = start[b], r1 = start[b + 1], s = seq ? seq[b] : b;
    bool bad = r0 < 0 || r1 < r0 || r1 > rows || (unsigned)s >= (unsigned)p.n_seqs;
    if (!bad) {
        const int n = r1 - r0, L = p.len[s];
        bad = L < n || L > (int64_t)p.max_pages << p.shift || (append && n > 0 && p.refused && p.refused[s] != 0);
        if (!bad && n > 0) {
            // a sequence's last places belong to one set of rows
            if (append && seq)
                for (int i = lane; i < b; i += 64) bad |= seq[i] == s && start[i + 1] > start[i];
            const int first = L - n;
            const int low = append ? first : window > 0 ? max(0, first - window + 1) : 0;
            const int seen = append ? 0 : min(low, sinks);
            for (int c = lane; c <= (L - 1) >> p.shift; c += 64)
                if ((c >= low >> p.shift || c << p.shift < seen) && (unsigned)p.table[s * p.st_table + c] >= (unsigned)p.n_pages) bad = true;
        }
    }
    if (__any(bad) && lane == 0) *flag = 1;
}

struct rope_args {
    double turns[64];           // of pair j per position
    int32_t rot, interleaved;
    float mscale;
};
enum { ROPE_HALVES = 0, ROPE_NEIGHBOURS = 1, ROPE_ODD_HALVES = 2 };
// A wave per row and slice of its heads.  The row's (cos, sin) are computed once: the angle in turns in 64 bits (a far position's
// angle keeps its fraction), its fraction's sine and cosine in 32.
// A lane owns the same place of every head it comes to, so that its (cos, sin) stay in registers: where pairs lie half
// of `rot` apart, 16 bytes of the low half and the 16 of the high half that belong to them (or 16 bytes that pass
// through), so that a pair meets in one lane and queries may be turned in place; where they are neighbours, 16 bytes.  Halves that
// are no multiple of 16 bytes take the pairs' other members one by one; a head is then read by one wave before it is written.
// Up to four passes over heads are loaded before the first is stored, the first of them before the row's place is looked up: a
// chain of start, length and page.  A chunk's rows are bound by HBM, a few rows by that chain.  Loads are non-temporal (what is
// written is read next, what is read is not): rows from HBM, 4096 of 64 heads of 8 44 -> 37 us (4.5 TB/s read and written), 1024 of 32 of 8 12.4 -> 10.3,
// 32 6.8 -> 6.6.
template <int D_H, int MODE>
__global__ __launch_bounds__(256) void rope_append_kernel(rope_args a, const bf16_t* q, int64_t st_q, const bf16_t* __restrict__ k,
                                                          int64_t st_k, const bf16_t* __restrict__ v, int64_t st_v,
                                                          const int32_t* __restrict__ start, const int32_t* __restrict__ seq, int n,
                                                          int rows, const int32_t* __restrict__ pos, cc_pool_view p, bf16_t* Kp,
                                                          bf16_t* Vp, int64_t st_page, int64_t st_tok, int64_t st_head, int H_q,
                                                          int H_kv, bf16_t* q_out, int passes_per_slice) {
    constexpr int CPH = D_H / 8;
    constexpr int NB = MODE == ROPE_ODD_HALVES ? 1 : 4;
    __shared__ float2 cs[4][64];
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int r = blockIdx.x * 4 + w, row = min(r, rows - 1);
    const int half = a.rot / 2, heads = H_q + 2 * H_kv;
    const int units = MODE == ROPE_HALVES ? CPH - half / 8 : CPH;      // of a head
    const int per_pass = 64 / units, my_head = lane / units, unit = lane - my_head * units;
    const bool paired = MODE == ROPE_HALVES && unit < half / 8;
    const int e0 = (MODE == ROPE_HALVES && !paired ? unit + half / 8 : unit) * 8;
    const int h0 = (blockIdx.y * passes_per_slice) * per_pass + my_head;
    const int h_end = min(heads, (int)(blockIdx.y + 1) * passes_per_slice * per_pass);
    auto source = [&](int h) -> const bf16_t* {
        const int hk = h - H_q, hv = hk - H_kv;
        return hk < 0 ? q + row * st_q + h * D_H : hv < 0 ? k + row * st_k + hk * D_H : v + row * st_v + hv * D_H;
    };
    bf16x8 x[NB], y[NB];
    auto load = [&](int hb) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int h = hb + i * per_pass;
            if (my_head >= per_pass || h >= h_end) continue;
            const bf16_t* src = source(h) + e0;
            x[i] = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(src));
            if (MODE == ROPE_HALVES && paired) y[i] = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(src + half));
            if (MODE == ROPE_ODD_HALVES && h < H_q + H_kv) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int j = e0 + e;
                    y[i][e] = source(h)[j >= a.rot ? j : j < half ? j + half : j - half];
                }
            }
        }
    };
    load(h0);

    const int b = r < rows ? cc_row_owner(start, n, r) : -1;
    int at = -1, page = -1;
    if (b >= 0) {
        const int s = seq ? seq[b] : b;
        const int L = cc_append_len(p, s);
        at = L - start[b + 1] + r;
        if (at >= 0 && at < L) page = p.table[s * p.st_table + (at >> p.shift)];
        else at = -1;
    }
    if (at >= 0 && lane < half) {
        const double t = (double)(pos ? pos[r] : at) * a.turns[lane];
        float sn, c;
        sincospif(2.0f * (float)(t - rint(t)), &sn, &c);
        cs[w][lane] = make_float2(c * a.mscale, sn * a.mscale);
    }
    __syncthreads();
    if (at < 0 || my_head >= per_pass) return;
    const bool stored = (unsigned)page < (unsigned)p.n_pages;
    const int64_t slot = stored ? page * st_page + (int64_t)(at & ((1 << p.shift) - 1)) * st_tok : 0;
    constexpr int NC = MODE == ROPE_NEIGHBOURS ? 4 : 8;
    float2 c[NC];
#pragma unroll
    for (int e = 0; e < NC; ++e) {
        const int j = MODE == ROPE_NEIGHBOURS ? e0 / 2 + e : MODE == ROPE_HALVES ? e0 + e : (e0 + e) % half;
        c[e] = cs[w][min(j, half - 1)];
    }
    for (int hb = h0; hb < h_end; hb += NB * per_pass) {
        if (hb != h0) load(hb);
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int h = hb + i * per_pass, hk = h - H_q, hv = hk - H_kv;
            if (h >= h_end || (hk >= 0 && !stored)) continue;
            bf16_t* dst = (hk < 0 ? q_out + ((int64_t)r * H_q + h) * D_H : hv < 0 ? Kp + slot + hk * st_head : Vp + slot + hv * st_head) + e0;
            if (hv < 0) {
                if (MODE == ROPE_HALVES && paired) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float lo = (float)x[i][e], hi = (float)y[i][e];
                        x[i][e] = (bf16_t)(lo * c[e].x - hi * c[e].y);
                        y[i][e] = (bf16_t)(hi * c[e].x + lo * c[e].y);
                    }
                } else if (MODE == ROPE_NEIGHBOURS) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float lo = (float)x[i][2 * e], hi = (float)x[i][2 * e + 1];
                        if (e0 + 2 * e < a.rot) {
                            x[i][2 * e] = (bf16_t)(lo * c[e].x - hi * c[e].y);
                            x[i][2 * e + 1] = (bf16_t)(hi * c[e].x + lo * c[e].y);
                        }
                    }
                } else if (MODE == ROPE_ODD_HALVES) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int j = e0 + e;
                        const float m = (float)x[i][e] * c[e].x, o = (float)y[i][e] * c[e].y;
                        if (j < a.rot) x[i][e] = (bf16_t)(j < half ? m - o : m + o);
                    }
                }
            }
            *reinterpret_cast<bf16x8*>(dst) = x[i];
            if (MODE == ROPE_HALVES && paired) *reinterpret_cast<bf16x8*>(dst + half) = y[i];
        }
    }
}

}  // namespace

void cc_launch_grow(const cc_page_pool& p, const int32_t* seq, const int32_t* n_new, int n, int32_t* host, hipStream_t s) {
    hipLaunchKernelGGL(grow_kernel, dim3(1), dim3(NT), 0, s, cc_view(p), seq, n_new, n, (int32_t*)p.work,
                       cc_page_work_layout(p.n_pages, p.n_seqs), p.status, host);
}
void cc_launch_fork(const cc_page_pool& p, const int32_t* src, const int32_t* dst, int n, int32_t* host, hipStream_t s) {
    hipLaunchKernelGGL(fork_kernel, dim3(1), dim3(NT), 0, s, cc_view(p), src, dst, n, (int32_t*)p.work,
                       cc_page_work_layout(p.n_pages, p.n_seqs), p.status, host);
}
void cc_launch_free(const cc_page_pool& p, const int32_t* seq, int n, int32_t* host, hipStream_t s) {
    hipLaunchKernelGGL(free_kernel, dim3(1), dim3(NT), 0, s, cc_view(p), seq, n, p.status, host);
}
void cc_launch_compact(const cc_page_pool& p, int32_t* host, hipStream_t s) {
    const cc_page_work w = cc_page_work_layout(p.n_pages, p.n_seqs);
    hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(NT), 0, s, cc_view(p), (int32_t*)p.work, w, p.status, host);
    hipLaunchKernelGGL(compact_table_kernel, dim3((p.n_seqs + 3) / 4), dim3(256), 0, s, cc_view(p), (const int32_t*)p.work, w);
}

void cc_launch_page_copies(const cc_page_pool& p, const cc_paged_kv* kv, int n_layers, int most, int H_kv, int d_h, hipStream_t s) {
    const cc_page_work w = cc_page_work_layout(p.n_pages, p.n_seqs);
    for (int l0 = 0; l0 < n_layers; l0 += CC_PAGE_LAYERS) {
        copy_args a;
        a.n_ptr = 2 * std::min(CC_PAGE_LAYERS, n_layers - l0);
        for (int i = 0; i < a.n_ptr; ++i) a.ptr[i] = i & 1 ? kv[l0 + i / 2].V : kv[l0 + i / 2].K;
        const dim3 grid((unsigned)std::min<int64_t>((int64_t)most * a.n_ptr, 64 * cc_device_cus()));
        if (grid.x == 0) return;
        if (d_h == 128)
            hipLaunchKernelGGL(page_copy_kernel<128>, grid, dim3(256), 0, s, a, (const int32_t*)p.work, w, H_kv, p.page_size,
                               kv[0].stride_page,
                               kv[0].stride_token, kv[0].stride_head);
        else
            hipLaunchKernelGGL(page_copy_kernel<64>, grid, dim3(256), 0, s, a, (const int32_t*)p.work, w, H_kv, p.page_size,
                               kv[0].stride_page,
                               kv[0].stride_token, kv[0].stride_head);
    }
}

void cc_launch_check_rows(const cc_new_rows& r, const cc_page_pool& p, int window, int sinks, int append, int32_t* flag, hipStream_t s) {
    if (r.n > 0)
        hipLaunchKernelGGL(check_rows_kernel, dim3(r.n), dim3(64), 0, s, r.start, r.seq, r.rows, cc_view(p), window, sinks, append, flag);
}

void cc_launch_rope_append(const bf16_t* q, int64_t st_q, const bf16_t* k, int64_t st_k, const bf16_t* v, int64_t st_v,
                           const cc_new_rows& r, const int32_t* pos, const cc_page_pool& p, const cc_paged_kv& kv,
                           const cc_rope& rope, const cc_model_desc& m, bf16_t* q_out, hipStream_t s) {
    if (r.rows <= 0 || r.n <= 0) return;
    rope_args a;
    cc_rope_turns(rope, a.turns);
    a.rot = rope.rot;
    a.interleaved = rope.interleaved != 0;
    a.mscale = (float)rope.mscale;
    // slices of a row until there are sixteen waves a CU or every pass has a wave of its own
    const int mode = a.interleaved ? ROPE_NEIGHBOURS : a.rot % 16 ? ROPE_ODD_HALVES : ROPE_HALVES;
    const int units = mode == ROPE_HALVES ? m.d_h / 8 - a.rot / 16 : m.d_h / 8, per_pass = 64 / units;
    const int passes = (m.H_q + 2 * m.H_kv + per_pass - 1) / per_pass;
    const int slices = std::max(1, std::min(passes, 16 * cc_device_cus() / r.rows));
    const int per_slice = (passes + slices - 1) / slices;
    const dim3 grid((r.rows + 3) / 4, (passes + per_slice - 1) / per_slice);
#define CC_ROPE(D, MODE)                                                                                                   \
    hipLaunchKernelGGL((rope_append_kernel<D, MODE>), grid, dim3(256), 0, s, a, q, st_q, k, st_k, v, st_v, r.start, r.seq, r.n, r.rows, \
                       pos, cc_view(p), (bf16_t*)kv.K, (bf16_t*)kv.V, kv.stride_page, kv.stride_token, kv.stride_head, m.H_q,  \
                       m.H_kv, q_out, per_slice)
    if (m.d_h == 128) {
        if (mode == ROPE_HALVES) CC_ROPE(128, ROPE_HALVES);
        else if (mode == ROPE_NEIGHBOURS) CC_ROPE(128, ROPE_NEIGHBOURS);
        else CC_ROPE(128, ROPE_ODD_HALVES);
    } else {
        if (mode == ROPE_HALVES) CC_ROPE(64, ROPE_HALVES);
        else if (mode == ROPE_NEIGHBOURS) CC_ROPE(64, ROPE_NEIGHBOURS);
        else CC_ROPE(64, ROPE_ODD_HALVES);
    }
#undef CC_ROPE
}
