// The tile loop of the attention kernels: 256 (row, query head) columns against a run of key tiles, for keys that lie
// in one cache or in pages.  The design is described where its first kernels are, in attention.hip.
#pragma once

#include "cc_internal.h"

#include <type_traits>

namespace {

constexpr int BN_KEYS = 64;

// 16 bytes per lane from global memory straight into LDS.  The LDS address is
// wave base (M0) + OFF + 16 * lane and OFF is also added to the global address.
// Rewriting M0 between loads is expensive while MFMAs are in flight (measured:
// several hundred cycles per rewrite with two MFMA-bound waves on a SIMD), so
// the loads of one tile and tensor share one base and differ in OFF only.
// STREAM: non-temporal.
template <int OFF, bool STREAM = false>
__device__ __forceinline__ void dma16(const bf16_t* gsrc_minus_off, bf16_t* lds_wave_base) {
    static_assert(OFF >= 0 && OFF < 4096, "the instruction offset is 13 bits signed; a larger value wraps silently");
    __builtin_amdgcn_global_load_lds(
        (const void __attribute__((address_space(1)))*)gsrc_minus_off,
        (void __attribute__((address_space(3)))*)lds_wave_base, 16, OFF, STREAM ? 2 : 0);
}
// LDS reads whose place in the instruction stream is fixed by the source order (the
// compiler's scheduler, short of registers, would issue every read right before its use).
// The waits for them are written by hand: LDS operations of a wave return in order, so
// "at most N outstanding" after N younger reads means this one has arrived.
// Transposing LDS read: within each group of 16 lanes, lane i receives, as element e, element (i % 4) of
// the 8-byte row addressed by lane (i / 4 + 4 e).
template <int IMM>
__device__ __forceinline__ bf16x4 lds_read_tr_at(uint32_t addr) {
    bf16x4 v;
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(IMM));
    return v;
}
template <int IMM>
__device__ __forceinline__ bf16x8 lds_read_b128_at(uint32_t addr) {
    bf16x8 v;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(IMM));
    return v;
}
template <int N>
__device__ __forceinline__ void lds_wait_all_but(bf16x8& x) {
    asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(x) : "n"(N));
}

template <int NI, int I = 0, class F>
__device__ __forceinline__ void static_for(F&& f) {
    if constexpr (I < NI) {
        f(std::integral_constant<int, I>{});
        static_for<NI, I + 1>(f);
    }
}

constexpr int LDS_TILES = 7;              // K tile t lives in stage t % 3, V tile t in stage 3 + t % 4

// Group (0: A, 1: B) and slot of this wave.  The two waves that share a SIMD must land in different
// groups: the SIMD id comes from the hardware id register (HW_ID bits 5:4), the first
// wave to register on a SIMD joins group A (0), the second group B (1).  Should the
// eight waves not sit two per SIMD, the split falls back to wave index order (correct,
// but the phases of a SIMD's waves then no longer alternate).
__device__ __forceinline__ void wave_role(int* simd_waves, int* group_waves, int& grp, int& widx) {
    const int tid = threadIdx.x, lane = tid & 63;
    if (tid < 4) simd_waves[tid] = 0;
    if (tid < 2) group_waves[tid] = 0;
    __syncthreads();
    int a = 0, b = 0;
    if (lane == 0) {
        const int simd = __builtin_amdgcn_s_getreg(((2 - 1) << 11) | (4 << 6) | 4);
        a = atomicAdd(&simd_waves[simd & 3], 1) & 1;
        b = atomicAdd(&group_waves[a], 1);
    }
    grp = __builtin_amdgcn_readfirstlane(a);
    widx = __builtin_amdgcn_readfirstlane(b);
    __syncthreads();
    if (group_waves[0] != 4) {
        const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
        grp = w >> 2;
        widx = w & 3;
    }
}

// last position that the 256 columns of row tile rt see (rows are sorted)
__device__ __forceinline__ int last_key(const int32_t* idx, int M, int g, int rt) {
    return idx[min(M - 1, (rt * 256 + 255) / g)];
}

// Keys and values in one cache: row i of the recomputed rows sees every slot up to idx[i].
struct one_cache {
    static constexpr bool paged = false, wide_pages = true;
    const int32_t* idx;
    const bf16_t* K;
    const bf16_t* V;
    int64_t st, sh;
    int N;
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
    return ((int64_t)uniform((int)(v >> 32)) << 32) | (uint32_t)uniform((int)v);
}

// The value, where it is asked for: what is made of it is not made ahead and kept through code in front of it.
__device__ __forceinline__ int here(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// Eight bytes of a piece, past the L2 and read past it: pieces go from one XCD to another within a launch.  A fence over the whole
// L2 instead (every workgroup's write-back and invalidation, 32 workgroups an L2) cost 70 to 110 us a call.
__device__ __forceinline__ void put(float* p, float x, float y) {
    const uint64_t v = (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x);
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get(const float* p) {
    const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}
// A pointer that is the same in all lanes, in scalar registers.
__device__ __forceinline__ const char* scalar_base(const char* p) {
    return (const char*)uniform((int64_t)(uintptr_t)p);
}

// Key tiles of `keys` keys that the rows of a sequence see: the first `sink` tiles, then those from `from` to the end.
struct tile_span {
    int sink, from, count;
    __device__ __forceinline__ int tile(int t) const { return t < sink ? t : t - sink + from; }
    // tiles in front of key tile `k`'s successor
    __device__ __forceinline__ int up_to(int k) const { return k < sink ? k + 1 : max(sink, k - from + sink + 1); }
};
// Rows at positions first .. end - 1.
__device__ __forceinline__ tile_span visible_tiles(int first, int end, int window, int sinks, int keys) {
    tile_span s;
    const int low = window > 0 ? (int)max((int64_t)0, (int64_t)first - window + 1) : 0;
    s.from = low / keys;
    s.sink = window > 0 ? min((int)(((int64_t)sinks + keys - 1) / keys), s.from) : 0;
    s.count = max(1, s.sink + (end + keys - 1) / keys - s.from);     // a row that sees nothing still has its zeros to write
    return s;
}

// Keys and values in pages: row i of a sequence's new rows sits at position first + i.  The visible key tiles of a
// row tile are `span`'s; within them a row sees key j up to its position, if it is within its window or a sink.
// WIDE_PAGES: pages of 64 tokens and more, so that a tile lies in one; else every 16 keys have a page of their own.
// ONCE: no other workgroup reads the same keys, so that they go past the caches.
typedef const __attribute__((address_space(4))) int32_t* scalar_table;   // constant for the launch: scalar loads
template <bool WIDE_PAGES, bool ONCE>
struct in_pages {
    static constexpr bool paged = true, wide_pages = WIDE_PAGES, once = ONCE;
    scalar_table table;             // of the sequence
    const bf16_t* K;
    const bf16_t* V;
    const bf16_t* zeros;            // a row of them, for what no page holds
    int64_t st_page, st_tok, sh;
    int shift, n_pages, L, first, row0, window, sinks;
    tile_span span;
};

// Key tiles ta .. ta + n_tiles - 1 (n_tiles >= 1) of the 256 columns of row tile rt and kv head kvh, of M rows.
// PIECE and slot >= 0: the sums stay unnormalised and go to part's slot.  Off: type
// of the lane offsets of the global -> LDS loads.  Can be called again by the same
// workgroup: every wave's reads of LDS lie before its last barrier, and a wave only loads
// into rows that it has loaded (and waited for) itself.
template <int D_H, bool PIECE, class Off, class Keys>
__device__ __forceinline__ void attend(
    const Keys& keys, const bf16_t* __restrict__ q, int M, int H_q, int g, bf16_t* __restrict__ o, float scale_log2, float* __restrict__ part, bf16_t* smem, int grp, int widx,
    int kvh, int rt, int ta, int n_tiles, int slot) {
    constexpr int KS = D_H / 16;          // k-steps of the QK^T contraction
    constexpr int DT = D_H / 32;          // 32-row tiles of O^T
    constexpr int CPRW = D_H / 8;         // 16-byte chunks per cache row
    constexpr int RPI = 64 / CPRW;        // rows moved by one global->LDS instruction
    constexpr int NI = BN_KEYS / RPI / 4; // such instructions per wave, tile and tensor

    constexpr int TILE = BN_KEYS * D_H;   // elements of one K or V tile
    auto k_stage = [&](int t) __attribute__((always_inline)) { return smem + (t % 3) * TILE; };
    auto v_stage = [&](int t) __attribute__((always_inline)) { return smem + (3 + t % 4) * TILE; };

    const int lane = Keys::paged ? here(threadIdx.x & 63) : threadIdx.x & 63;
    const int wave = widx;                              // role in the cooperative tile loads
    const int qr = lane & 31, hf = lane >> 5;
    const int col_in = (grp * 4 + widx) * 32 + qr;      // column within the row tile
    const int col = rt * 256 + col_in;                  // flat (token, head) column
    const int mi = col / g, hg = col - mi * g;
    const bool valid = mi < M;
    int limit = -1, under = (int)0x80000000;            // the newest key a row sees; keys up to `under` left its window
    int row = mi;                                       // of q and o
    if constexpr (Keys::paged) {
        if (valid) limit = max(keys.first + mi, -1);
        if (keys.window > 0) under = limit - keys.window;
        row += keys.row0;
    } else {
        if (valid) limit = keys.idx[mi];
    }
    // first key of the piece's t-th tile
    auto key_of = [&](int t) __attribute__((always_inline)) -> int {
        if constexpr (Keys::paged) return keys.span.tile(ta + t) * BN_KEYS;
        else return ta * BN_KEYS + t * BN_KEYS;
    };

    // wave-wide largest limit (tiles beyond it are skipped by this wave) and smallest
    // limit of a valid row (tiles that end at or below it need no mask)
    int wave_limit = limit;
    for (int off = 32; off > 0; off >>= 1) wave_limit = max(wave_limit, __shfl_xor(wave_limit, off));
    int wave_min = valid ? limit : 0x7fffffff;
    for (int off = 32; off > 0; off >>= 1) wave_min = min(wave_min, __shfl_xor(wave_min, off));

    // ---- Q fragments (B operand of S^T = K Q^T): lane = query row, 8 d's per k-step ----
    bf16x8 qf[KS];
    {
        const bf16_t* qp = q + ((int64_t)(valid ? row : 0) * H_q + kvh * g + hg) * D_H + 8 * hf;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if (valid) {
                qf[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16);
            } else {
#pragma unroll
                for (int u = 0; u < 8; ++u) qf[ks][u] = (bf16_t)0.0f;
            }
        }
    }

    // ---- global -> LDS: instruction i of this wave moves the RPI logical rows
    //      (i*4 + wave)*RPI ..; lane L fills physical chunk L % CPRW of row L / CPRW and
    //      fetches the logical chunk that the swizzle maps there.  In LDS the rows of one
    //      wave's NI instructions are adjacent (physical row rho(r) below), so they are
    //      reached from one base with immediate offsets of 1 KB ----
    //   K rows: chunk c sits at slot c ^ kswz(row)           (16-byte fragment reads)
    //   V rows: the 64-byte group dt sits at group dt ^ vswz(row)  (transposing 8-byte reads)
    // The swizzles use row bits that the instruction index does not touch, so one lane
    // offset per tensor serves every instruction.
    auto kswz = [](int r) { return D_H == 128 ? (r & 15) : ((r >> 1) & 7); };
    auto vswz = [](int r) { return D_H == 128 ? (r & 3) : ((r >> 1) & 1); };
    constexpr auto rho = [](int r) constexpr { return (((r / RPI) % 4) * NI + r / (4 * RPI)) * RPI + r % RPI; };
    static_assert((4 * RPI) % 16 == 0 && NI * 1024 <= 4096, "row bits of the swizzle / immediate offset range");
    const bf16_t* kbase = keys.K + (int64_t)kvh * keys.sh;
    const bf16_t* vbase = keys.V + (int64_t)kvh * keys.sh;
    const int l_row = lane / CPRW, l_p = lane % CPRW;
    const int r0 = wave * RPI + l_row;                 // logical row of instruction 0
    const int k_col = (l_p ^ kswz(r0)) * 8;
    const int v_col = ((((l_p >> 2) ^ vswz(r0)) << 2) | (l_p & 3)) * 8;
    const int wave_slot = wave * NI * RPI * D_H;
    // Group A loads V tiles, group B K tiles: a wave-uniform base per tile (scalar registers) plus
    // 32-bit lane offsets that are the same for every tile; from the tile on that reaches past the
    // cache (only a workgroup's last one can) rows past N-1 are clamped (they are masked anyway).
    const char* const lbase = reinterpret_cast<const char*>(grp == 0 ? vbase : kbase);
    const int l_col = grp == 0 ? v_col : k_col;
    auto scalar_ptr = [](const char* p) -> const char* {   // keeps the base in scalar registers
        const uint64_t u = reinterpret_cast<uint64_t>(p);
        const uint64_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)u);
        const uint64_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(u >> 32));
        return reinterpret_cast<const char*>((hi << 32) | lo);
    };
    // In pages a tile has one base, or every instruction one of its own: its rows (4 or 8, aligned) lie in one page.  The
    // pages of a tile are asked for a tile ahead.  Rows behind the last token repeat it (only the last tile's can be); what
    // no page holds is read from a row of zeros.
    constexpr int NB = Keys::wide_pages ? 1 : NI;      // bases of a tile
    Off loff[NI];
    struct tile_src { const char* at[NB]; bool there[NB]; };
    int next_page[NB];
    // first key of the 16 that instruction i takes its rows of, and its first row within them (narrow pages)
    auto group = [&](int i) __attribute__((always_inline)) -> int { return (i * 4 + wave) * RPI & ~15; };
    const int group_row = wave * RPI & 15;
    auto ask_pages = [&](int t) __attribute__((always_inline)) {
        if constexpr (Keys::paged) {
#pragma unroll
            for (int i = 0; i < NB; ++i)
                next_page[i] = keys.table[min(key_of(t) + (NB == 1 ? 0 : group(i)), max(keys.L - 1, 0)) >> keys.shift];
        }
    };
    auto set_loff = [&](int rmax) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            if constexpr (!Keys::paged) loff[i] = ((Off)min(r0 + i * 4 * RPI, rmax) * (Off)keys.st + (Off)l_col) * 2;
            else if constexpr (NB == 1) loff[i] = ((Off)max(min(r0 + i * 4 * RPI, rmax), 0) * (Off)keys.st_tok + (Off)l_col) * 2;
            else loff[i] = ((Off)max(min(group_row + l_row, rmax - group(i)), 0) * (Off)keys.st_tok + (Off)l_col) * 2;
        }
    };
    set_loff(BN_KEYS);
    auto tile_at = [&](int t) __attribute__((always_inline)) -> tile_src {
        const int j0 = key_of(t);
        tile_src src;
        if constexpr (Keys::paged) {
            if (j0 + BN_KEYS > keys.L) set_loff(keys.L - 1 - j0);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int key = j0 + (NB == 1 ? 0 : group(i));
                src.there[i] = key < keys.L && (unsigned)next_page[i] < (unsigned)keys.n_pages;
                // (a page is smaller than 2^32 bytes)
                src.at[i] = lbase + (next_page[i] * keys.st_page * 2 + (uint32_t)(key & ((1 << keys.shift) - 1)) * (uint32_t)(keys.st_tok * 2));
                if (!src.there[i]) src.at[i] = (const char*)keys.zeros;
            }
        } else {
            if (j0 + BN_KEYS > keys.N) set_loff(keys.N - 1 - j0);
            src.at[0] = lbase + (int64_t)j0 * keys.st * 2;
        }
        return src;
    };
    auto load_part = [&](const tile_src& tile, bf16_t* stage, auto ic) __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value;
        const char* b = scalar_ptr(tile.at[NB == 1 ? 0 : i] - i * 1024);   // the immediate adds it back
        if constexpr (Keys::paged) {
            Off off = tile.there[NB == 1 ? 0 : i] ? loff[i] : (Off)(l_col * 2);
            asm volatile("" : "+v"(off));
            dma16<i * 1024, Keys::once>(reinterpret_cast<const bf16_t*>(b + off), stage + wave_slot);
        } else {
            asm volatile("" : "+v"(loff[i]));   // keeps the (32-bit) offset a register operand of the load
            dma16<i * 1024>(reinterpret_cast<const bf16_t*>(b + loff[i]), stage + wave_slot);
        }
    };
    auto load_tile = [&](const tile_src& tile, bf16_t* stage) __attribute__((always_inline)) {
        static_for<NI>([&](auto i) __attribute__((always_inline)) { load_part(tile, stage, i); });
    };

    // ---- fragment addresses: LDS byte addresses in the stage this wave reads next (they
    //      move on after every matrix phase); key block and half are immediate offsets ----
    const uint32_t smem_base = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)smem;
    // K: logical row kt*32 + qr (physical rho(qr) + 8 kt), logical chunk 2 ks + hf
    const int k_sw = kswz(qr);
    uint32_t kaddr[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
        kaddr[ks] = smem_base + 2 * (rho(qr) * D_H + (((ks * 2 + hf) ^ k_sw) << 3));
    // V^T through the transposing read: lane s of a 16-lane group addresses key
    // (4 hf + s/4) and the 4 d's starting at 16*(group%2) + 4*(s%4); the lane then
    // holds 4 consecutive keys of column d = 32 dt + lane%32.  Key 16 ss + 8 e + v_key sits
    // in physical row rho(16 ss + 8 e) + rho(v_key) (the two parts use different row bits).
    const int s16 = lane & 15, dsub = (lane >> 4) & 1;
    const int v_key = 4 * hf + (s16 >> 2);
    const int v_sw = vswz(v_key);
    const int v_lane = (2 * dsub + ((s16 & 3) >> 1)) * 8 + (s16 & 1) * 4;
    uint32_t vaddr[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
        vaddr[dt] = smem_base + 2 * (3 * TILE + rho(v_key) * D_H + v_lane + ((dt ^ v_sw) << 5));

    f32x16 acc_o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc_o[dt][v] = 0.0f;
    float m_run = -INFINITY, l_run = 0.0f;
    f32x16 s[2];       // S^T tile: 64 keys x 32 query rows
    bf16x8 pf[4];      // its probabilities as B operand of the second contraction

    // `load`: the four loads of this wave's next tile go between the exponentials, evenly apart
    auto softmax = [&](int j0, auto load) __attribute__((always_inline)) {
        // ---- causal mask (only in tiles that reach past the wave's first row),
        //      online softmax in base 2 with the 1/sqrt(d_h) scale folded into the exponent ----
        if constexpr (Keys::paged) {
            if (j0 + BN_KEYS - 1 > wave_min || (keys.window > 0 && j0 <= wave_limit - keys.window && j0 + BN_KEYS > keys.sinks)) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int key = j0 + kt * 32 + 8 * (v >> 2) + 4 * hf + (v & 3);
                        // (no short circuits: selects, not branches)
                        const bool out = (key > limit) | ((key <= under) & (key >= keys.sinks));
                        s[kt][v] = out ? -INFINITY : s[kt][v];
                    }
            }
        } else if (j0 + BN_KEYS - 1 > wave_min) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    int key = j0 + kt * 32 + 8 * (v >> 2) + 4 * hf + (v & 3);
                    if (key > limit) s[kt][v] = -INFINITY;
                }
        }
        float mx = -INFINITY;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[kt][v]);
        {   // the other half-wave's maximum of the same query row: lanes i and i + 32 exchange by a
            // register swap (no LDS round trip)
            const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * scale_log2;
        }
        // The reference point m_run of the exponent is only moved when a row's maximum
        // grew by more than 2^8: until then probabilities up to 256 are accumulated
        // (harmless in fp32 / bf16, and the final division by the row sum cancels it),
        // which keeps the 64-element rescale of O out of most tiles.
        const bool grow = mx > m_run + 8.0f;
        if (__any(grow)) {
            const float m_new = grow ? mx : m_run;
            const float alpha = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.0f : m_new));
            l_run *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc_o[dt][v] *= alpha;
            m_run = m_new;
        }
        const float m_use = m_run == -INFINITY ? 0.0f : m_run;
        float psum = 0.0f;
        // four scores at a time: exponentials, their sum and their bf16 pair conversions are
        // finished before the next four start (keeps only four probabilities live)
        static_for<8>([&](auto chunk) __attribute__((always_inline)) {
            constexpr int c = decltype(chunk)::value;
            constexpr int kt = c >> 2, v0 = (c & 3) * 4;
            if constexpr (c * NI % 8 == 0) {
                __builtin_amdgcn_sched_barrier(0);
                load(std::integral_constant<int, c * NI / 8>{});
                __builtin_amdgcn_sched_barrier(0);
            }
            float pv[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) pv[u] = __builtin_amdgcn_exp2f(fmaf(s[kt][v0 + u], scale_log2, -m_use));
            psum += (pv[0] + pv[1]) + (pv[2] + pv[3]);
            typedef float f32x2 __attribute__((ext_vector_type(2)));
            typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));
            bf16x2 lo = __builtin_convertvector(f32x2{pv[0], pv[1]}, bf16x2);
            bf16x2 hi = __builtin_convertvector(f32x2{pv[2], pv[3]}, bf16x2);
            asm volatile("" : "+v"(lo), "+v"(hi));   // converted here, not gathered at the end
            bf16x8& dst = pf[kt * 2 + (v0 >> 3)];
            dst[(v0 & 7) + 0] = lo[0];
            dst[(v0 & 7) + 1] = lo[1];
            dst[(v0 & 7) + 2] = hi[0];
            dst[(v0 & 7) + 3] = hi[1];
            });
        l_run += psum;
    };
    // End of a phase: all of this wave's global -> LDS loads but the newest tile's
    // (`pending`) have landed, then the workgroup barrier.  The tile
    // reads are written by hand, so no compiler-made wait is needed around the barrier.
    auto phase_end = [&](bool pending) __attribute__((always_inline)) {
        if (pending) __builtin_amdgcn_s_waitcnt((NI & 0xF) | ((NI >> 4) << 14) | (0x7 << 4) | (0xF << 8));
        else __builtin_amdgcn_s_waitcnt((0x7 << 4) | (0xF << 8));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // Matrix phase of one wave: O^T += V^T P^T for the V tile at vaddr (with_pv), then
    // S^T = K Q^T for the K tile at kaddr.  The other wave of the SIMD is in
    // its softmax, so this wave alone has to keep the matrix pipe fed: the LDS reads of MFMA
    // j + PD are issued before MFMA j.  P V: MFMA j = (ss, dt) = (j / DT, j % DT), DT
    // independent accumulation chains; A slots 0..3 <- keys 16ss+4hf.., 4..7 <- keys
    // 16ss+8+4hf..  Scores: MFMA n = (ks, kt) = (n / 2, n % 2), two chains.
    constexpr int PD = 4;
    auto matrix_phase = [&](auto with_pv) __attribute__((always_inline)) {
        constexpr int NPV = decltype(with_pv)::value ? 4 * DT : 0, NQK = 2 * KS, NALL = NPV + NQK;
        const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        bf16x8 opnd[NALL];
        // Order of the MFMAs when both contractions run: two of P V, two of Q K^T, and so on, so
        // that an MFMA follows the one whose accumulator it continues four issue slots later, not
        // two (the score tile has only two accumulation chains; back to back they wait for each
        // other's result).
        constexpr auto is_pv = [](int j) constexpr { return NPV != 0 && (j & 3) < 2; };
        constexpr auto pv_of = [](int j) constexpr { return (j >> 2) * 2 + (j & 3); };
        constexpr auto qk_of = [](int j) constexpr { return NPV != 0 ? (j >> 2) * 2 + (j & 3) - 2 : j; };
        static_assert(NPV == 0 || NPV == NQK, "the interleaved order pairs the two contractions one to one");
        // reads of the operands j+1 .. last (a P V operand is two reads)
        constexpr auto reads_after = [](int j, int last) constexpr {
            int n = 0;
            for (int i = j + 1; i <= last; ++i) n += (NPV != 0 && (i & 3) < 2) ? 2 : 1;
            return n;
        };
        auto issue = [&](auto jc) __attribute__((always_inline)) {
            constexpr int j = decltype(jc)::value;
            if constexpr (j < NALL) {
                if constexpr (is_pv(j)) {
                    constexpr int p = pv_of(j), ss = p / DT, dt = p % DT;
                    constexpr int at = 2 * rho(16 * ss) * D_H;
                    constexpr int at8 = 2 * rho(16 * ss + 8) * D_H;
                    const bf16x4 a0 = lds_read_tr_at<at>(vaddr[dt]);
                    const bf16x4 a1 = lds_read_tr_at<at8>(vaddr[dt]);
                    opnd[j] = __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7);
                } else {
                    constexpr int n = qk_of(j), ks = n / 2, kt = n % 2;
                    opnd[j] = lds_read_b128_at<2 * kt * 8 * D_H>(kaddr[ks]);
                }
            }
        };
        static_for<PD>(issue);
        static_for<NALL>([&](auto jc) __attribute__((always_inline)) {
            constexpr int j = decltype(jc)::value;
            issue(std::integral_constant<int, j + PD>{});
            constexpr int last = j + PD < NALL ? j + PD : NALL - 1;
            lds_wait_all_but<reads_after(j, last)>(opnd[j]);
            if constexpr (is_pv(j)) {
                constexpr int p = pv_of(j), ss = p / DT, dt = p % DT;
                acc_o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(opnd[j], pf[ss], acc_o[dt], 0, 0, 0);
            } else {
                constexpr int n = qk_of(j), ks = n / 2, kt = n % 2;
                s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(opnd[j], qf[ks], ks == 0 ? zero : s[kt], 0, 0, 0);
            }
        });
    };

    // ---- phases.  P0: A scores(0).  P(2t+1): A softmax(t) | B values(t-1), scores(t).
    //      P(2t+2): A values(t), scores(t+1) | B softmax(t).  A wave issues its loads in its
    //      softmax phase, between the exponentials.  Group A loads V(t+2) in P(2t+1) into the
    //      stage of V(t-2), which group B left in P(2t-1); first read in P(2t+6).  Group A lets
    //      only its newest tile stay in flight at the end of P(2t+1): V(t+1) has landed, and is
    //      first read in P(2t+4).  Group B loads K(t+3) in P(2t+2) into the stage of K(t), which it
    //      left in P(2t+1); at the end of P(2t+2) K(t+2) has landed, first read in P(2t+4).
    //      Every wave passes 2 n_tiles + 3 barriers; tiles past a wave's own last key only cost it
    //      the barriers and its loads.  The scores of tile my_tiles (computed from whatever its
    //      stage holds) are never used.
    int my_tiles = 0;
    if constexpr (Keys::paged) {
        if (wave_limit >= 0) my_tiles = max(0, min(keys.span.up_to(wave_limit / BN_KEYS) - ta, n_tiles));
    } else {
        if (wave_limit >= 0) my_tiles = max(0, min(wave_limit / BN_KEYS + 1 - ta, n_tiles));
    }
    using yes = std::integral_constant<int, 1>;
    using no = std::integral_constant<int, 0>;
    int k_at = 0, v_at = 0;           // stages the address registers point at
    auto advance = [&](bool also_v) __attribute__((always_inline)) {
        const int kd = k_at == 2 ? -4 * TILE : 2 * TILE;
        k_at = k_at == 2 ? 0 : k_at + 1;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kaddr[ks] += kd;
        if (also_v) {
            const int vd = v_at == 3 ? -6 * TILE : 2 * TILE;
            v_at = v_at == 3 ? 0 : v_at + 1;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) vaddr[dt] += vd;
        }
    };
    if (grp == 0) {
        ask_pages(0);
        load_tile(tile_at(0), v_stage(0));
        ask_pages(min(1, n_tiles - 1));
        if (n_tiles > 1) load_tile(tile_at(1), v_stage(1));
        ask_pages(min(2, n_tiles - 1));
        phase_end(n_tiles > 1);                            // K(0), V(0) are in place
        if (my_tiles > 0) {                                // P0
            matrix_phase(no{});
            advance(false);
        }
        phase_end(n_tiles > 1);
        for (int t = 0; t < n_tiles; ++t) {
            const tile_src next = tile_at(min(t + 2, n_tiles - 1));   // past the end: the last tile again, unused
            ask_pages(min(t + 3, n_tiles - 1));
            if (t < my_tiles)
                softmax(key_of(t), [&](auto i) __attribute__((always_inline)) { load_part(next, v_stage(t + 2), i); });
            else
                load_tile(next, v_stage(t + 2));
            phase_end(true);                               // V(t), V(t+1) have landed
            if (t < my_tiles) {
                matrix_phase(yes{});
                advance(true);
            }
            phase_end(true);
        }
        phase_end(false);
    } else {
        ask_pages(0);
        load_tile(tile_at(0), k_stage(0));
        ask_pages(min(1, n_tiles - 1));
        if (n_tiles > 1) load_tile(tile_at(1), k_stage(1));
        ask_pages(min(2, n_tiles - 1));
        if (n_tiles > 2) load_tile(tile_at(2), k_stage(2));
        ask_pages(min(3, n_tiles - 1));
        if (n_tiles > 2) __builtin_amdgcn_s_waitcnt(((2 * NI) & 0xF) | (((2 * NI) >> 4) << 14) | (0x7 << 4) | (0xF << 8));
        phase_end(n_tiles > 1);                            // K(0), V(0) are in place
        phase_end(true);                                   // P0
        if (my_tiles > 0) {                                // P1
            matrix_phase(no{});
            advance(false);
        }
        phase_end(n_tiles > 2);                            // K(1) has landed
        for (int t = 0; t < n_tiles; ++t) {
            const tile_src next = tile_at(min(t + 3, n_tiles - 1));   // past the end: the last tile again, unused
            ask_pages(min(t + 4, n_tiles - 1));
            if (t < my_tiles)
                softmax(key_of(t), [&](auto i) __attribute__((always_inline)) { load_part(next, k_stage(t), i); });
            else
                load_tile(next, k_stage(t));
            phase_end(true);                               // K(t+2) has landed
            if (t < my_tiles) {
                matrix_phase(yes{});
                advance(true);
            }
            phase_end(true);
        }
    }

    __builtin_amdgcn_s_waitcnt((0x7 << 4) | (0xF << 8));   // the unused loads of the last tiles have landed

    // ---- normalise and write: lane holds 4 consecutive d per (dt, v/4) ----
    float l_tot = l_run + __shfl_xor(l_run, 32);
    if (!valid) return;
    if (!PIECE || slot < 0) {
        const float inv = Keys::paged && !(l_tot > 0.0f) ? 0.0f : 1.0f / l_tot;
        bf16_t* op = o + ((int64_t)row * H_q + kvh * g + hg) * D_H;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int vq = 0; vq < 4; ++vq) {
                bf16x4 w;
#pragma unroll
                for (int u = 0; u < 4; ++u) w[u] = (bf16_t)(acc_o[dt][vq * 4 + u] * inv);
                *reinterpret_cast<bf16x4*>(op + dt * 32 + 8 * vq + 4 * hf) = w;
            }
    } else {
        // as the registers lie, so that every store is one contiguous KB: [wave][D_H / 8][lane] four
        // unnormalised sums, then [lane] the exponent's reference point and the row sum
        float* pp = part + (int64_t)slot * 256 * (D_H + 4) + (grp * 4 + widx) * 32 * (D_H + 4);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int vq = 0; vq < 4; ++vq) {
                f32x4 w;
#pragma unroll
                for (int u = 0; u < 4; ++u) w[u] = acc_o[dt][vq * 4 + u];
                if constexpr (Keys::paged) {               // [wave][D_H / 8][2][lane] two sums: put together within the launch
                    put(pp + (dt * 4 + vq) * 256 + lane * 2, w[0], w[1]);
                    put(pp + (dt * 4 + vq) * 256 + 128 + lane * 2, w[2], w[3]);
                } else {
                    *reinterpret_cast<f32x4*>(pp + (dt * 4 + vq) * 256 + lane * 4) = w;
                }
            }
        if constexpr (Keys::paged) put(pp + 32 * D_H + lane * 2, m_run, l_tot);
        else *reinterpret_cast<float2*>(pp + 32 * D_H + lane * 2) = make_float2(m_run, l_tot);
    }
}

}  // namespace
