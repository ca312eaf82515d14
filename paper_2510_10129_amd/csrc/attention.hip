// Sparse-query causal GQA attention over the updated KV cache: recomputed row i
// (global position idx[i]) attends to every cache slot j <= idx[i].  This is
// the kernel Section 5.6 of the paper describes as flash attention with sparse
// query indices; the design below is for gfx950.
//
// Work split: the (recomputed token, query head of the group) pairs of one kv
// head form one flat column sequence c = i*g + h (g = H_q/H_kv); a workgroup of
// eight waves owns 256 consecutive columns, a wave 32 of them on the N side of
// the MFMA tile, so a K/V tile read from LDS serves the whole query group and
// no column is padding when g does not divide 32.
//
// Each wave computes S^T = K Q^T (keys on the MFMA row side, query rows on the
// column side).  In the 32x32 accumulator layout a lane then owns ONE query row
// and 16 keys per tile, so the online-softmax maximum and sum are in-lane
// reductions plus one exchange with lane^32, the rescale factor is a per-lane
// scalar, and the probabilities are already laid out as the B operand of
// O^T = V^T P^T: no shuffle between the two contractions.
//
// Two wave groups alternate between the matrix pipe and the vector ALU.  Per
// 64-key tile a wave issues 32 MFMAs and about as many cycles of exponentials,
// sums and conversions, one after the other; two independent waves on a SIMD
// drift into the same phase (both contend for the matrix pipe, then both for
// the vector ALU) and each pipe idles half of the time.  Here the two waves of a
// SIMD belong to the same workgroup, one to group A and one to group B, and
// the workgroup barrier separates phases: while A runs the softmax of tile t, B
// runs P V of tile t-1 and Q K^T of tile t, and the other way round in the next
// phase.  A wave issues its global -> LDS loads in its softmax phase, one after every
// second group of four exponentials (group A the V tiles, group B the K tiles): the four of
// them back to back at the end of the matrix phase queue up behind each other and lengthen
// the phase that the matrix pipe is busy in.  The form of the load decides: scalar base plus
// 32-bit lane offset and one LDS base for the four.  With 64-bit vector addresses and the LDS
// base rewritten between them the same placement ran 18 % slower.  At 64k context, 64 query
// heads and M = 13363: 12.05 -> 11.72 ms; M = 16576 at 16k: 2.05 -> 1.99 ms.
//
// K and V tiles (64 keys) go from the cache straight into LDS with 16-byte
// global->LDS loads, row-major as they are stored, three stages of K, four of V.  K
// fragments are plain 16-byte LDS reads; the V^T fragments (contraction index =
// key) come from the row-major V tile through the transposing LDS read
// ds_read_b64_tr_b16, so V is never transposed in registers.  Both tiles are
// XOR-swizzled (by choosing which global chunk a lane fetches) so that the
// fragment reads spread over the 64 LDS banks.
//
// Causality with sorted idx: the key loop of a workgroup ends at the position
// of its last row; the per-row mask only bites between the positions of the
// first and last row of the tile.  Workgroups are issued longest-first and
// workgroup id modulo H_kv picks the kv head, so the workgroups resident on
// one XCD walk the same K/V stream through that XCD's L2.
#include "attend.h"
#include "launch_plan.h"
#include <algorithm>

namespace {

// One block of 256 columns per workgroup, longest first.  Off: 64 bits only for token strides that
// a 32-bit lane offset cannot hold.
#define CC_ATTN_ARGS                                                                                        \
    const bf16_t *__restrict__ q, int M, const int32_t *__restrict__ idx, int H_q, int H_kv,                \
        const bf16_t *__restrict__ Kc, const bf16_t *__restrict__ Vc, int64_t st, int64_t sh, int N,        \
        bf16_t *__restrict__ o, int n_row_tiles, float scale_log2
template <int D_H, class Off>
__device__ __forceinline__ void attend_block(CC_ATTN_ARGS) {
    __shared__ __align__(16) bf16_t smem[LDS_TILES * BN_KEYS * D_H];
    __shared__ int simd_waves[4], group_waves[2];
    int grp, widx;
    wave_role(simd_waves, group_waves, grp, widx);
    const int g = H_q / H_kv, kvh = blockIdx.x % H_kv, rt = n_row_tiles - 1 - blockIdx.x / H_kv;
    attend<D_H, false, Off>(one_cache{idx, Kc, Vc, st, sh, N}, q, M, H_q, g, o, scale_log2, nullptr, smem, grp, widx, kvh, rt, 0,
                            last_key(idx, M, g, rt) / BN_KEYS + 1, -1);
}
template <int D_H>
__global__ __launch_bounds__(512, 1) void sparse_attn_kernel(CC_ATTN_ARGS) {
    attend_block<D_H, uint32_t>(q, M, idx, H_q, H_kv, Kc, Vc, st, sh, N, o, n_row_tiles, scale_log2);
}
template <int D_H>
__global__ __launch_bounds__(512, 1) void wide_stride_attn_kernel(CC_ATTN_ARGS) {
    attend_block<D_H, uint64_t>(q, M, idx, H_q, H_kv, Kc, Vc, st, sh, N, o, n_row_tiles, scale_log2);
}

// Even grid.  A block costs as many key tiles as its last row can see, so a grid of a few hundred
// blocks ends unevenly: its makespan is the longest block or one more round.  Here every workgroup (one
// per CU) takes the same number of units of one long sequence: the blocks of kv head 0 by row
// tile, those of head 1, ...; a block of L key tiles is L + EVEN_START units long, the first of
// them for what a block costs besides its tiles (query loads, first tiles, output).  A range
// covers some whole blocks and, at its ends, pieces of two; the pieces go to slots 2 w and 2 w + 1
// of range w (a piece of the block that the range starts in, of a later one) and
// attn_merge_kernel combines the pieces of a block.  Consecutive ranges run on one XCD, so that its
// L2 serves one kv head when H_kv = 8.
constexpr int EVEN_START = CC_ATTN_EVEN_START;          // 3 and 5 units measured: 5 is 1 % of the layer faster
constexpr int EVEN_MAX_TILES = CC_ATTN_EVEN_MAX_TILES;
// table: [n_row_tiles + 2] the first unit of every row tile within a head, their sum, units per range
template <int D_H>
__global__ __launch_bounds__(512, 1) void even_attn_kernel(CC_ATTN_ARGS, int per_min, float* __restrict__ part,
                                                           int* __restrict__ table) {
    __shared__ __align__(16) bf16_t smem[LDS_TILES * BN_KEYS * D_H];
    __shared__ int simd_waves[4], group_waves[2], wave_units[8];
    __shared__ int pre[EVEN_MAX_TILES + 1];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int g = H_q / H_kv;
    int grp, widx;
    wave_role(simd_waves, group_waves, grp, widx);

    // first unit of every row tile: exclusive scan, two row tiles a thread
    int len[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        len[i] = 2 * tid + i < n_row_tiles ? last_key(idx, M, g, 2 * tid + i) / BN_KEYS + 1 + EVEN_START : 0;
    int inc = len[0] + len[1];
    for (int off = 1; off < 64; off <<= 1) {
        const int v = __shfl_up(inc, off);
        if (lane >= off) inc += v;
    }
    if (lane == 63) wave_units[w] = inc;
    __syncthreads();
    int base = inc - len[0] - len[1];
    for (int i = 0; i < w; ++i) base += wave_units[i];
    pre[2 * tid] = base;
    pre[2 * tid + 1] = base + len[0];
    if (tid == 511) pre[EVEN_MAX_TILES] = base + len[0] + len[1];
    __syncthreads();
    const int head_units = __builtin_amdgcn_readfirstlane(pre[n_row_tiles]);   // tiles past the last have no units
    const int total = head_units * H_kv, n_wg = gridDim.x;
    const int per = max(per_min, (total + n_wg - 1) / n_wg);
    if (blockIdx.x == 0) {
        for (int t = tid; t <= n_row_tiles; t += 512) table[t] = pre[t];
        if (tid == 0) table[n_row_tiles + 1] = per;
    }
    // workgroup ids go round-robin to the 8 XCDs: each gets consecutive ranges
    const int x = blockIdx.x & 7, xq = n_wg >> 3, xr = n_wg & 7;
    const int range = x * xq + min(x, xr) + (int)(blockIdx.x >> 3);
    int u = range * per, stop = min(u + per, total);     // units of the whole sequence, then of head kvh
    if (u < total) {
        int kvh = u / head_units;
        u -= kvh * head_units;
        stop -= kvh * head_units;
        int rt = 0;                                      // last row tile whose first unit is <= u
        for (int hi = n_row_tiles - 1; rt < hi;) {
            const int mid = (rt + hi + 1) >> 1;
            if (pre[mid] <= u) rt = mid; else hi = mid - 1;
        }
        rt = __builtin_amdgcn_readfirstlane(rt);
        for (int later = 0; u < stop; later = 1) {
            const int b0 = __builtin_amdgcn_readfirstlane(pre[rt]), b1 = __builtin_amdgcn_readfirstlane(pre[rt + 1]);
            const int ta = max(0, u - b0 - EVEN_START), te = min(b1, stop) - b0 - EVEN_START;
            if (te > ta) {
                const bool whole = ta == 0 && te == b1 - b0 - EVEN_START;
                attend<D_H, true, uint32_t>(one_cache{idx, Kc, Vc, st, sh, N}, q, M, H_q, g, o, scale_log2, part, smem, grp, widx,
                                            kvh, rt, ta, te - ta, whole ? -1 : 2 * range + later);
            }
            u = b1;
            if (++rt == n_row_tiles) {
                rt = 0;
                ++kvh;
                u = 0;
                stop -= head_units;
            }
        }
    }
}

// Whole blocks cut S ways: workgroup (block, s) takes the s-th of S equal runs of the block's key tiles
// and leaves its piece in slot block * S + s; attn_merge_kernel combines them.
template <int D_H, class Off>
__device__ __forceinline__ void attend_cut(CC_ATTN_ARGS, float* __restrict__ part) {
    __shared__ __align__(16) bf16_t smem[LDS_TILES * BN_KEYS * D_H];
    __shared__ int simd_waves[4], group_waves[2];
    int grp, widx;
    wave_role(simd_waves, group_waves, grp, widx);
    const int g = H_q / H_kv, kvh = blockIdx.x % H_kv, rt = n_row_tiles - 1 - blockIdx.x / H_kv, S = gridDim.y;
    const int L = last_key(idx, M, g, rt) / BN_KEYS + 1, per = (L + S - 1) / S;
    const int ta = blockIdx.y * per, n = min(per, L - ta);
    const int slot = (kvh * n_row_tiles + rt) * S + blockIdx.y;
    if (n <= 0) {                                        // a short block: no keys for this piece
        float* pp = part + (int64_t)slot * 256 * (D_H + 4) + (threadIdx.x >> 6) * 32 * (D_H + 4);
        *reinterpret_cast<float2*>(pp + 32 * D_H + (threadIdx.x & 63) * 2) = make_float2(-INFINITY, 0.0f);
        return;
    }
    attend<D_H, true, Off>(one_cache{idx, Kc, Vc, st, sh, N}, q, M, H_q, g, o, scale_log2, part, smem, grp, widx, kvh, rt, ta, n,
                           slot);
}
template <int D_H>
__global__ __launch_bounds__(512, 1) void cut_attn_kernel(CC_ATTN_ARGS, float* __restrict__ part) {
    attend_cut<D_H, uint32_t>(q, M, idx, H_q, H_kv, Kc, Vc, st, sh, N, o, n_row_tiles, scale_log2, part);
}

template <int D_H>
__global__ __launch_bounds__(512, 1) void wide_stride_cut_attn_kernel(CC_ATTN_ARGS, float* __restrict__ part) {
    attend_cut<D_H, uint64_t>(q, M, idx, H_q, H_kv, Kc, Vc, st, sh, N, o, n_row_tiles, scale_log2, part);
}

// Combines the pieces of the blocks that an even grid (S = 0) or a cut one (S pieces) has left:
// o = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s with m = max m_s, pieces in the order of their keys.
// Workgroup (block, 32 of its columns = one wave of the attention kernel, 32 of their d's); a
// thread holds the same elements as the lane that wrote them, four of a column.  Up to eight pieces at
// a time, so that their loads are out together.  Workgroup id modulo H_kv is the kv head, as in the attention
// kernels, so that a piece is read through the L2 that it was written to: with the heads one after
// the other 64 blocks of 3 pieces took 34 us in both launches, so 25 (64 query heads of 8, N = 850,
// M = 256).  32 d's a workgroup instead of all: 1 to 2 us of a few blocks' merge.
template <int D_H>
__global__ __launch_bounds__(256) void attn_merge_kernel(const float* __restrict__ part, const int* __restrict__ table,
                                                         int S, int M, int H_q, int H_kv, int n_row_tiles,
                                                         bf16_t* __restrict__ o) {
    const int g = H_q / H_kv, kvh = blockIdx.x % H_kv, rt = blockIdx.x / H_kv;
    int w0 = 0, w1 = S - 1, per = 1, first = 0;
    if (S == 0) {                                        // even grid: the ranges that hold the block's key tiles
        per = table[n_row_tiles + 1];
        const int head = kvh * table[n_row_tiles], end = head + table[rt + 1];
        first = head + table[rt];
        w0 = (first + EVEN_START) / per;
        w1 = (end - 1) / per;
        if (w0 == w1) return;
    }
    const int lane = threadIdx.x & 63, v0 = blockIdx.z * 4 + (threadIdx.x >> 6);     // 16-byte group of a column
    const int col = rt * 256 + blockIdx.y * 32 + (lane & 31), mi = col / g, hg = col - mi * g;
    if (mi >= M) return;
    float m = -INFINITY, l = 0.0f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    auto take = [&](auto nc, int wb) __attribute__((always_inline)) {
        constexpr int NP = decltype(nc)::value;
        f32x4 v[NP];
        float2 ml[NP];
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            const int w = min(wb + k, w1);               // past the end: the last piece again, with weight 0
            const int slot = S ? (kvh * n_row_tiles + rt) * S + w : 2 * w + (w * per < first ? 1 : 0);
            const float* pp = part + (int64_t)slot * 256 * (D_H + 4) + blockIdx.y * 32 * (D_H + 4);
            ml[k] = *reinterpret_cast<const float2*>(pp + 32 * D_H + lane * 2);
            v[k] = *reinterpret_cast<const f32x4*>(pp + v0 * 256 + lane * 4);
        }
        float mn = m;
#pragma unroll
        for (int k = 0; k < NP; ++k) mn = fmaxf(mn, ml[k].x);
        const float ref = mn == -INFINITY ? 0.0f : mn;   // no key of this column so far
        const float keep = __builtin_amdgcn_exp2f(m - ref);
        l *= keep;
        acc *= keep;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            // a piece without keys of this column: a cut grid's empty piece leaves no sums at all
            const bool on = wb + k <= w1 && ml[k].x != -INFINITY;
            const float f = on ? __builtin_amdgcn_exp2f(ml[k].x - ref) : 0.0f;
            l += ml[k].y * f;
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += on ? v[k][e] * f : 0.0f;
        }
        m = mn;
    };
    for (int wb = w0; wb <= w1;) {
        const int left = w1 - wb + 1;
        if (left > 4) take(std::integral_constant<int, 8>{}, wb), wb += 8;
        else if (left > 2) take(std::integral_constant<int, 4>{}, wb), wb += 4;
        else take(std::integral_constant<int, 2>{}, wb), wb += 2;
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    bf16_t* op = o + ((int64_t)mi * H_q + kvh * g + hg) * D_H + 4 * (lane >> 5);
    bf16x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = (bf16_t)(acc[e] * inv);
    *reinterpret_cast<bf16x4*>(op + 8 * v0) = r;
}

}  // namespace

int cc_attn_piece_workgroups(const cc_model_desc& m, int64_t M, int64_t N) {
    return cc_plan_attn_workgroups(cc_device_cus(), (M * (m.H_q / m.H_kv) + 255) / 256 * m.H_kv, (N + BN_KEYS - 1) / BN_KEYS);
}

void cc_launch_attention(const bf16_t* q, int M, const int32_t* idx, const cc_model_desc& m,
                         const cc_kv_layer& kv, bf16_t* o, float* part, int slots, int* table,
                         const cc_launch_override& ovr, hipStream_t s) {
    if (M <= 0) return;
    const int g = m.H_q / m.H_kv;
    const int n_row_tiles = (int)(((int64_t)M * g + 255) / 256);   // 256 (token, head) columns each
    const float scale_log2 = 1.4426950408889634f / sqrtf((float)m.d_h);
    const int n_wg = n_row_tiles * m.H_kv;
    const int t_max = (kv.N + BN_KEYS - 1) / BN_KEYS;
#define CC_ATTN_LAUNCH(KERN, GRID, ...)                                                                       \
    do {                                                                                                      \
        if (m.d_h == 128)                                                                                     \
            hipLaunchKernelGGL(KERN<128>, dim3(GRID), dim3(512), 0, s, q, M, idx, m.H_q, m.H_kv,              \
                               (const bf16_t*)kv.K, (const bf16_t*)kv.V, kv.stride_token, kv.stride_head,     \
                               kv.N, o, n_row_tiles, scale_log2, ##__VA_ARGS__);                              \
        else                                                                                                  \
            hipLaunchKernelGGL(KERN<64>, dim3(GRID), dim3(512), 0, s, q, M, idx, m.H_q, m.H_kv,               \
                               (const bf16_t*)kv.K, (const bf16_t*)kv.V, kv.stride_token, kv.stride_head,     \
                               kv.N, o, n_row_tiles, scale_log2, ##__VA_ARGS__);                              \
    } while (0)
    // 64 rows of a tile, 2 bytes an element, in an unsigned 32-bit lane offset
    const bool wide = kv.stride_token >= (1ll << 32) / (2 * (BN_KEYS + 1));
    const cc_attn_plan p = cc_plan_attention(cc_device_cus(), n_row_tiles, m.H_kv, m.d_h, t_max, slots, wide, ovr.attn_splits);
    if (p.kind == CC_ATTN_EVEN) {
        CC_ATTN_LAUNCH(even_attn_kernel, p.ranges, p.per_min, part, table);
    } else if (p.kind == CC_ATTN_CUT) {
        const dim3 cg(n_wg, p.pieces);
        if (wide) CC_ATTN_LAUNCH(wide_stride_cut_attn_kernel, cg, part);
        else CC_ATTN_LAUNCH(cut_attn_kernel, cg, part);
    } else if (wide) {
        CC_ATTN_LAUNCH(wide_stride_attn_kernel, n_wg);
    } else {
        CC_ATTN_LAUNCH(sparse_attn_kernel, n_wg);
    }
    if (p.kind != CC_ATTN_WHOLE) {
        const int S = p.kind == CC_ATTN_CUT ? p.pieces : 0;
        const dim3 mg(n_wg, 8, m.d_h / 32);
        if (m.d_h == 128)
            hipLaunchKernelGGL(attn_merge_kernel<128>, mg, dim3(256), 0, s, part, table, S, M, m.H_q, m.H_kv, n_row_tiles, o);
        else
            hipLaunchKernelGGL(attn_merge_kernel<64>, mg, dim3(256), 0, s, part, table, S, M, m.H_q, m.H_kv, n_row_tiles, o);
    }
#undef CC_ATTN_LAUNCH
}
