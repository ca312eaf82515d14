// Causal grouped-query attention of new rows over a paged cache, optionally under a sliding window with sinks.
#include "paged.h"

namespace {

// A wave per (row, query head): 64 keys at a time, a lane per key for the scores, a lane per D_H / 64 elements for the
// values, with the running maximum and sum of an online softmax.
template <int D_H>
__global__ __launch_bounds__(64) void row_attn_kernel(const bf16_t* __restrict__ q, const int32_t* __restrict__ start,
                                                      const int32_t* __restrict__ seq, int n, int rows, cc_pool_view p,
                                                      const bf16_t* __restrict__ Kp, const bf16_t* __restrict__ Vp, int64_t st_page,
                                                      int64_t st_tok, int64_t st_head, int window, int sinks, int H_q, int H_kv,
                                                      float scale_log2, bf16_t* __restrict__ o) {
    constexpr int DL = D_H / 64;
    __shared__ float qs[D_H], ps[64];
    __shared__ int64_t slot[64];
    const int lane = threadIdx.x, r = blockIdx.x, h = blockIdx.y, kvh = h / (H_q / H_kv);
    const int b = cc_row_owner(start, n, r);
    if (b < 0) return;
    const int s = seq ? seq[b] : b, L = cc_seq_len(p, s), at = L - start[b + 1] + r;
    const int64_t row = ((int64_t)r * H_q + h) * D_H;
#pragma unroll
    for (int e = 0; e < DL; ++e) qs[lane * DL + e] = (float)q[row + lane * DL + e];
    __syncthreads();
    float m = -INFINITY, l = 0.0f, acc[DL] = {};
    const int low = window > 0 ? max(0, at - window + 1) : 0;
    for (int j0 = 0; j0 <= at; j0 += 64) {
        if (j0 + 63 < low && j0 >= sinks) continue;
        const int j = j0 + lane;
        bool on = j <= at && (j >= low || j < sinks);
        int64_t a = -1;
        float z = on ? 0.0f : -INFINITY;
        if (on) {
            const int page = p.table[s * p.st_table + (j >> p.shift)];
            if ((unsigned)page < (unsigned)p.n_pages) {
                a = page * st_page + (int64_t)(j & ((1 << p.shift) - 1)) * st_tok + kvh * st_head;
                for (int e = 0; e < D_H; ++e) z += qs[e] * (float)Kp[a + e];
                z *= scale_log2;
            }
        }
        float mx = z;
        for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
        const float m_new = fmaxf(m, mx), ref = m_new == -INFINITY ? 0.0f : m_new;
        const float pr = exp2f(z - ref), keep = exp2f(m - ref);
        float sum = pr;
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
        l = l * keep + sum;
        m = m_new;
        ps[lane] = pr;
        slot[lane] = a;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < DL; ++e) acc[e] *= keep;
        for (int i = 0; i < 64; ++i)
            if (slot[i] >= 0)
#pragma unroll
                for (int e = 0; e < DL; ++e) acc[e] += ps[i] * (float)Vp[slot[i] + lane * DL + e];
        __syncthreads();
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
    for (int e = 0; e < DL; ++e) o[row + lane * DL + e] = (bf16_t)(acc[e] * inv);
}

}  // namespace

void cc_launch_paged_attention(const bf16_t* q, const cc_new_rows& r, const cc_page_pool& p, const cc_paged_kv& kv, int window,
                               int sinks, const cc_model_desc& m, bf16_t* o, hipStream_t s) {
    if (r.rows <= 0 || r.n <= 0) return;
    const float scale_log2 = 1.4426950408889634f / sqrtf((float)m.d_h);
    const dim3 grid(r.rows, m.H_q);
#define CC_ROW_ATTN(D)                                                                                                     \
    hipLaunchKernelGGL(row_attn_kernel<D>, grid, dim3(64), 0, s, q, r.start, r.seq, r.n, r.rows, cc_view(p),               \
                       (const bf16_t*)kv.K, (const bf16_t*)kv.V, kv.stride_page, kv.stride_token, kv.stride_head, window, \
                       sinks, m.H_q, m.H_kv, scale_log2, o)
    if (m.d_h == 128) CC_ROW_ATTN(128);
    else CC_ROW_ATTN(64);
#undef CC_ROW_ATTN
}
