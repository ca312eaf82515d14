// Device view of a page pool and of a batch of new rows, shared by the kernels of the paged cache.
#pragma once

#include "cc_internal.h"
#include "paged_plan.h"

struct cc_pool_view {
    int32_t* refs;
    int32_t* table;
    int32_t* len;
    int32_t* refused;               // or NULL
    int64_t st_table;
    int32_t n_pages, n_seqs, max_pages;
    int32_t shift;                  // log2(page_size)
};
inline cc_pool_view cc_view(const cc_page_pool& p) {
    return {p.refs, p.table, p.len, p.refused, p.stride_table, p.n_pages, p.n_seqs, p.max_pages, __builtin_ctz(p.page_size)};
}

// Tokens of sequence s as far as its table can hold them; 0 for an index that is none.
__device__ __forceinline__ int cc_seq_len(const cc_pool_view& p, int s) {
    if ((unsigned)s >= (unsigned)p.n_seqs) return 0;
    return max(0, min(p.len[s], p.max_pages << p.shift));
}

// The same for rows that are to be written: none where the sequence's last grow was refused, as its last places hold other
// tokens then.
__device__ __forceinline__ int cc_append_len(const cc_pool_view& p, int s) {
    if ((unsigned)s >= (unsigned)p.n_seqs) return 0;
    const int refused = p.refused ? p.refused[s] : 0, len = cc_seq_len(p, s);
    return refused ? 0 : len;
}

// Sequence of the batch that row r belongs to (uniform in the wave; all lanes come here), -1: none.
__device__ __forceinline__ int cc_row_owner(const int32_t* start, int n, int r) {
    const int lane = threadIdx.x & 63;
    int b = 0;
    for (int i = lane; i - lane < n; i += 64) b += __popcll(__ballot(i < n && start[min(i, n - 1) + 1] <= r));
    return b < n && start[b] <= r ? b : -1;
}

void cc_launch_grow(const cc_page_pool& p, const int32_t* seq, const int32_t* n_new, int n, int32_t* host, hipStream_t s);
void cc_launch_fork(const cc_page_pool& p, const int32_t* src, const int32_t* dst, int n, int32_t* host, hipStream_t s);
void cc_launch_free(const cc_page_pool& p, const int32_t* seq, int n, int32_t* host, hipStream_t s);
void cc_launch_compact(const cc_page_pool& p, int32_t* host, hipStream_t s);
// The copies that a grow or compact left in the pool's scratch, at most `most` of them, in every layer.
void cc_launch_page_copies(const cc_page_pool& p, const cc_paged_kv* kv, int n_layers, int most, int H_kv, int d_h, hipStream_t s);
// Sets *flag where a batch does not fit its pool.  Of its pages it looks at those that rows see (window, sinks), or with append at
// those that they are written to.
void cc_launch_check_rows(const cc_new_rows& r, const cc_page_pool& p, int window, int sinks, int append, int32_t* flag, hipStream_t s);
void cc_launch_rope_append(const bf16_t* q, int64_t st_q, const bf16_t* k, int64_t st_k, const bf16_t* v, int64_t st_v,
                           const cc_new_rows& r, const int32_t* pos, const cc_page_pool& p, const cc_paged_kv& kv,
                           const cc_rope& rope, const cc_model_desc& m, bf16_t* q_out, hipStream_t s);
// Of the context: d_h zeros for keys that no page holds, and a count per workgroup that is zero between calls.
struct cc_paged_scratch {
    const bf16_t* zeros;
    int32_t* arrived;
};
void cc_launch_paged_attention(const bf16_t* q, const cc_new_rows& r, const cc_page_pool& p, const cc_paged_kv& kv, int window,
                               int sinks, const cc_model_desc& m, const cc_paged_scratch& ws, bf16_t* o, hipStream_t s);
