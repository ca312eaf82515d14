// Argument checks and host-side arithmetic of the paged cache: plain functions without HIP, so that they can be
// read and tested where there is no GPU.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "cacheclip.h"

#define CC_PAGED_MAX_N 1024        // sequences of a batch of new rows
#define CC_PAGED_MAX_COLUMNS (1 << 20)   // (row, query head of a group) columns of one call
#define CC_PAGED_WGS 256           // most workgroups of an attention launch that leave pieces, two slots each
#define CC_PAGED_SLOT (256 * (128 + 4))  // floats of the largest piece
#define CC_PAGED_CUT_BYTES 4096     // the table of a launch that leaves its pieces to another
#define CC_PAGED_CTX_INTS (CC_PAGED_WGS + 64)   // of a context: a count per workgroup, and 128 bf16 zeros
#define CC_PAGE_LAYERS 128         // layers whose pages one copy launch takes (their addresses are kernel arguments)

// Scratch of a pool, in ints: a header, per sequence (takes, offsets), per page (a list, a map), and the copies
// that a call leaves for the copy kernel; behind it what an attention launch leaves (the table of its cuts, the pieces).
struct cc_page_work {
    int64_t take, first, copy_at, list, map, src, dst, rows, attn, ints;
};
inline cc_page_work cc_page_work_layout(int64_t n_pages, int64_t n_seqs) {
    cc_page_work w;
    int64_t at = 64;                              // [0]: copies to make
    auto take = [&](int64_t n) { const int64_t a = at; at += (n + 63) / 64 * 64; return a; };
    w.take = take(n_seqs), w.first = take(n_seqs), w.copy_at = take(n_seqs);
    w.list = take(n_pages), w.map = take(n_pages);
    const int64_t n = std::max(n_pages, n_seqs);
    w.src = take(n), w.dst = take(n), w.rows = take(n);
    w.attn = at;
    w.ints = at + CC_PAGED_CUT_BYTES / 4 + (int64_t)2 * CC_PAGED_WGS * CC_PAGED_SLOT;
    return w;
}

// Which attention kernel takes a batch whose sequences have up to so many (row, query head of a group) columns: few rows read
// every key once per 16 columns (32 at d_h = 64) from a ring a wave, many rows multiply 256 columns a workgroup.  16 sequences of 4000
// to 12000 tokens, us few / many:  d_h = 128, 32 heads of 8, 4 columns 97 / 98, 16 columns 98 / 98, 20 columns (two blocks of 16 a
// wave) 147 / 106;  d_h = 64, 32 of 8, 4 columns 58 / 72, 32 columns 59 / 72, 64 columns (four blocks) 114 / 88.  So a single token
// of more than 16 query heads a kv head is a call of many rows at d_h = 128: 32 ragged sequences of up to 16577 tokens, 32 heads of 1
// 46 us (176 MB) and 64 of 2 73 (351 MB), where 16 of 1 and 32 of 2 take 37 and 66.
inline bool cc_few_rows(int64_t columns, int32_t d_h) { return columns <= (d_h == 128 ? 16 : 32); }

struct cc_refusal {
    cc_status code;
    const char* why;
};
#define CC_REFUSE_IF(cond, code, why) do { if (cond) return cc_refusal{code, why}; } while (0)

inline bool cc_aligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Whether runs of so many bf16 from a and b on share memory.
inline bool cc_overlap(const void* a, int64_t n_a, const void* b, int64_t n_b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return n_a > 0 && n_b > 0 && x < y + (uintptr_t)n_b * 2 && y < x + (uintptr_t)n_a * 2;
}

inline int64_t cc_page_work_size(int32_t n_pages, int32_t n_seqs) { return 4 * cc_page_work_layout(n_pages, n_seqs).ints; }

inline cc_refusal cc_check_pool(const cc_page_pool* p) {
    CC_REFUSE_IF(!p, CC_ERR_NULL, "pool must not be NULL");
    CC_REFUSE_IF(!p->refs || !p->table || !p->len || !p->status || !p->work, CC_ERR_NULL,
                 "refs, table, len, status and work must not be NULL");
    CC_REFUSE_IF(p->page_size < 16 || p->page_size > 1024 || (p->page_size & (p->page_size - 1)), CC_ERR_SHAPE,
                 "page_size must be a power of two in [16, 1024]");
    CC_REFUSE_IF(p->n_pages < 1 || p->n_seqs < 1 || p->n_seqs > 65536 || p->max_pages < 1, CC_ERR_SHAPE,
                 "need n_pages >= 1, max_pages >= 1 and n_seqs in [1, 65536]");
    CC_REFUSE_IF((int64_t)p->n_pages * p->page_size >= (1ll << 31) || (int64_t)p->max_pages * p->page_size >= (1ll << 30),
                 CC_ERR_SHAPE, "n_pages * page_size must be below 2^31, max_pages * page_size below 2^30");
    CC_REFUSE_IF(p->stride_table < p->max_pages, CC_ERR_SHAPE, "stride_table must be at least max_pages");
    CC_REFUSE_IF(!cc_aligned(p->refs, 4) || !cc_aligned(p->table, 4) || !cc_aligned(p->len, 4) || !cc_aligned(p->status, 4) ||
                     !cc_aligned(p->refused, 4) || !cc_aligned(p->work, 256), CC_ERR_SHAPE, "tables must be 4-byte aligned and work 256-byte aligned");
    CC_REFUSE_IF(p->work_bytes < cc_page_work_size(p->n_pages, p->n_seqs), CC_ERR_WORKSPACE,
                 "work holds less than cc_page_work_bytes(n_pages, n_seqs)");
    return {CC_OK, ""};
}

// A grow that nobody waits for says what it refused to the append behind it.
inline cc_refusal cc_check_grow(const cc_page_pool& p, const int32_t* status_host) {
    CC_REFUSE_IF(!status_host && !p.refused, CC_ERR_NULL, "a grow without status_host needs pool->refused");
    return {CC_OK, ""};
}

// Tokens or heads outermost, pages behind each other: every element of a page at an address of its own.
inline cc_refusal cc_check_paged_kv(const cc_paged_kv* kv, int32_t page_size, int32_t H_kv, int32_t d_h) {
    CC_REFUSE_IF(!kv || !kv->K || !kv->V, CC_ERR_NULL, "kv, kv->K and kv->V must not be NULL");
    CC_REFUSE_IF(kv->stride_page % 8 || kv->stride_token % 8 || kv->stride_head % 8, CC_ERR_SHAPE,
                 "page, token and head strides must be multiples of 8");
    CC_REFUSE_IF(kv->stride_page < 1 || kv->stride_token < d_h || kv->stride_head < (H_kv > 1 ? d_h : 0), CC_ERR_SHAPE,
                 "strides must be positive and cover d_h");
    const bool tokens_out = kv->stride_token >= (H_kv - 1) * kv->stride_head + d_h;
    const bool heads_out = kv->stride_head >= (page_size - 1) * kv->stride_token + d_h;
    CC_REFUSE_IF(H_kv > 1 && !tokens_out && !heads_out, CC_ERR_SHAPE, "tokens or heads must be outermost in a page");
    CC_REFUSE_IF(kv->stride_page < (page_size - 1) * kv->stride_token + (H_kv - 1) * kv->stride_head + d_h, CC_ERR_SHAPE,
                 "stride_page must cover a page");
    CC_REFUSE_IF(kv->stride_token >= (1ll << 23) || kv->stride_token * page_size >= (1ll << 31), CC_ERR_SHAPE,
                 "stride_token must be below 2^23, and times page_size below 2^31");
    CC_REFUSE_IF(!cc_aligned(kv->K, 16) || !cc_aligned(kv->V, 16), CC_ERR_SHAPE, "K and V must be 16-byte aligned");
    return {CC_OK, ""};
}

inline cc_refusal cc_check_layers(const cc_paged_kv* kv, int32_t n_layers, int32_t page_size, int32_t H_kv, int32_t d_h) {
    CC_REFUSE_IF(n_layers < 0, CC_ERR_SHAPE, "n_layers must be >= 0");
    CC_REFUSE_IF(n_layers > 0 && !kv, CC_ERR_NULL, "kv must not be NULL");
    for (int i = 0; i < n_layers; ++i) {
        const cc_refusal r = cc_check_paged_kv(kv + i, page_size, H_kv, d_h);
        if (r.code != CC_OK) return r;
        CC_REFUSE_IF(kv[i].stride_page != kv[0].stride_page || kv[i].stride_token != kv[0].stride_token ||
                         kv[i].stride_head != kv[0].stride_head, CC_ERR_SHAPE, "all layers must have the same strides");
    }
    return {CC_OK, ""};
}

// Lists of sequences, each at most once.
inline cc_refusal cc_check_list(int32_t n, int32_t n_seqs, const int32_t* a, const int32_t* b) {
    CC_REFUSE_IF(n < 0 || n > n_seqs, CC_ERR_SHAPE, "n must be in [0, n_seqs]");
    CC_REFUSE_IF(n > 0 && (!a || !b), CC_ERR_NULL, "the lists must not be NULL");
    CC_REFUSE_IF(!cc_aligned(a, 4) || !cc_aligned(b, 4), CC_ERR_SHAPE, "the lists must be 4-byte aligned");
    return {CC_OK, ""};
}

inline cc_refusal cc_check_new_rows(const cc_new_rows* r, int32_t n_seqs, int32_t g) {
    CC_REFUSE_IF(!r, CC_ERR_NULL, "rows must not be NULL");
    CC_REFUSE_IF(r->n < 0 || r->n > CC_PAGED_MAX_N, CC_ERR_SHAPE, "n must be in [0, 1024]");
    CC_REFUSE_IF(r->rows < 0 || r->max_new < 0 || (int64_t)r->rows * g > CC_PAGED_MAX_COLUMNS, CC_ERR_SHAPE,
                 "need rows >= 0, max_new >= 0 and at most 2^20 rows times query heads of a group");
    CC_REFUSE_IF(r->n > 0 && !r->start, CC_ERR_NULL, "start must not be NULL");
    CC_REFUSE_IF(!r->seq && r->n > n_seqs, CC_ERR_SHAPE, "without seq, n must be at most n_seqs");
    CC_REFUSE_IF(!cc_aligned(r->start, 4) || !cc_aligned(r->seq, 4), CC_ERR_SHAPE, "start and seq must be 4-byte aligned");
    return {CC_OK, ""};
}

// Key tiles that the blocks of a head can add up to are counted in 32 bits.
inline cc_refusal cc_check_attend(const cc_new_rows& r, const cc_page_pool& p, int32_t g, int32_t window, int32_t sinks) {
    CC_REFUSE_IF(window < 0 || sinks < 0, CC_ERR_SHAPE, "window and sinks must be >= 0");
    const int64_t blocks = (int64_t)r.rows * g / 256 + r.n, tiles = ((int64_t)p.max_pages * p.page_size + 63) / 64 + 8;
    CC_REFUSE_IF(blocks * tiles >= (1ll << 31), CC_ERR_SHAPE, "rows of the batch times columns of the table are too many for one call");
    return {CC_OK, ""};
}

inline cc_refusal cc_check_rope(const cc_rope* r, int32_t d_h) {
    CC_REFUSE_IF(!r, CC_ERR_NULL, "rope must not be NULL");
    CC_REFUSE_IF(!(r->base > 1.0) || !std::isfinite(r->base), CC_ERR_SHAPE, "base must be finite and > 1");
    CC_REFUSE_IF(r->rot < 2 || r->rot > d_h || r->rot % 2, CC_ERR_SHAPE, "rot must be even and in [2, d_h]");
    CC_REFUSE_IF(r->scaling < CC_ROPE_PLAIN || r->scaling > CC_ROPE_INDEX, CC_ERR_SHAPE, "unknown scaling");
    CC_REFUSE_IF(!(std::fabs(r->mscale) <= 3.4e38), CC_ERR_SHAPE, "mscale must be finite in 32 bits");
    CC_REFUSE_IF(r->scaling != CC_ROPE_PLAIN && (!(r->factor >= 1.0) || !std::isfinite(r->factor)), CC_ERR_SHAPE,
                 "factor must be finite and >= 1");
    CC_REFUSE_IF(r->scaling >= CC_ROPE_TURNS && (r->orig_len < 1 || !(r->low > 0.0) || !(r->high > r->low) || !std::isfinite(r->high)),
                 CC_ERR_SHAPE, "need orig_len >= 1 and 0 < low < high");
    return {CC_OK, ""};
}

// Turns (of 2 pi) that pair j moves by per position.
inline void cc_rope_turns(const cc_rope& r, double* turns) {
    const double two_pi = 6.283185307179586476925286766559;
    double lo = 0.0, hi = 0.0;
    if (r.scaling == CC_ROPE_INDEX) {
        auto index_at = [&](double t) { return r.rot * std::log(r.orig_len / (two_pi * t)) / (2.0 * std::log(r.base)); };
        lo = std::max(std::floor(index_at(r.high)), 0.0);
        hi = std::min(std::ceil(index_at(r.low)), (double)r.rot - 1.0);
    }
    // base^(-2j/rot) as a product of two powers: 16 of them for 64 pairs, 1.1 us a call for 3.4
    double fine[8], coarse = 1.0;
    for (int b = 0; b < 8; ++b) fine[b] = std::pow(r.base, -2.0 * b / r.rot);
    for (int j = 0; j < r.rot / 2; ++j) {
        if (j % 8 == 0) coarse = std::pow(r.base, -2.0 * j / r.rot);
        const double w = coarse * fine[j % 8];
        double keep = 1.0;                        // share of the unscaled frequency
        if (r.scaling == CC_ROPE_LINEAR) keep = 0.0;
        if (r.scaling == CC_ROPE_TURNS) keep = std::min(1.0, std::max(0.0, (r.orig_len * w / two_pi - r.low) / (r.high - r.low)));
        if (r.scaling == CC_ROPE_INDEX) keep = 1.0 - std::min(1.0, std::max(0.0, (j - lo) / std::max(hi - lo, 0.001)));
        turns[j] = (keep == 1.0 ? w : w * ((1.0 - keep) / r.factor + keep)) / two_pi;
    }
}
