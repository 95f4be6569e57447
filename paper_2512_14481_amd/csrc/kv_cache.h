// The paged key/value cache and a step's sequences as the kernels see them, and the host's checks of both (gfx950 only).
#pragma once

#include "sasq_device.h"

namespace sasq {

struct KvPages {
    uint8_t* k;
    uint8_t* v;
    const float* k_scale;
    const float* v_scale;
    int64_t page_stride, token_stride, head_stride;      // bytes
    int pages, page_shift, heads;
};

struct KvSteps {
    const int* __restrict__ cu_q;
    const int* __restrict__ kv_len;
    const int* __restrict__ table;
    int batch, max_pages, tokens, max_q;
};

// A sequence's rows and keys, bounded whatever the device arrays hold.  (Places in the workspace are for max_q rows of it: one with more has none.)
struct KvSeq {
    int row0, rows, keys, past;                           // first new token's row, new tokens, keys that the table has places for, position of the first new token
};
__device__ __forceinline__ KvSeq kv_seq(const KvSteps& s, int b, int page_shift)
{
    const int first = min(max(s.cu_q[b], 0), s.tokens), end = min(max(s.cu_q[b + 1], first), s.tokens);
    const int rows = end - first <= s.max_q ? end - first : 0, keys = max(s.kv_len[b], 0), places = s.max_pages << page_shift;
    return {first, rows, min(keys, places), min(keys - rows, places)};
}
// The last key that new token i of the sequence sees, -1 (or less) if there is none.  A length past the table leaves the tokens where they
// are: those past the table see all of it.
__device__ __forceinline__ int kv_last(const KvSeq& seq, int i) { return min(seq.past + i, seq.keys - 1); }

// Page of a sequence's position, -1 if it is not there; at >= 0 and inside the table's row is the caller's part.
__device__ __forceinline__ int kv_page(const KvPages& c, const KvSteps& s, int b, int index)
{
    const int page = s.table[(int64_t)b * s.max_pages + index];
    return page >= 0 && page < c.pages ? page : -1;
}

constexpr int64_t kKvMost = INT64_C(1) << 30;             // positions of a sequence, rows of a step

inline int kv_check(const sasq_kv_cache* c, const sasq_kv_batch* b, int64_t q_heads, sasq_dtype dt)
{
    if (!c || !b) return SASQ_ERR_NULL;
    if (!c->k || !c->v || !b->cu_q || !b->kv_len || !b->block_table) return SASQ_ERR_NULL;
    if (c->fmt != SASQ_KV_16 && c->fmt != SASQ_KV_INT8) return SASQ_ERR_UNSUPPORTED;
    if (dt != SASQ_F16 && dt != SASQ_BF16) return SASQ_ERR_UNSUPPORTED;
    if (c->fmt == SASQ_KV_INT8 && (!c->k_scale || !c->v_scale)) return SASQ_ERR_NULL;
    if (c->dim != 64 && c->dim != 128) return SASQ_ERR_SHAPE;
    if (c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1))) return SASQ_ERR_SHAPE;
    if (c->pages <= 0 || c->pages > INT32_MAX || c->heads <= 0 || c->heads > 65535) return SASQ_ERR_SHAPE;
    const int64_t e = c->fmt == SASQ_KV_16 ? 2 : 1, most = INT64_C(1) << 60;
    for (int64_t stride : {c->page_stride, c->token_stride, c->head_stride})
        if (stride < c->dim || stride > most / (2 * c->pages) || (stride * e) % 16) return SASQ_ERR_SHAPE;
    if (c->token_stride > INT64_C(1) << 26) return SASQ_ERR_SHAPE;          // sixteen places in a 32-bit offset
    if (b->batch <= 0 || b->batch >= kKvMost || b->tokens <= 0 || b->tokens > kKvMost || b->max_q <= 0 || b->max_kv <= 0) return SASQ_ERR_SHAPE;
    if (b->max_pages <= 0 || b->max_pages > kKvMost / c->page_size) return SASQ_ERR_SHAPE;
    if (q_heads <= 0 || q_heads > 65535 || q_heads % c->heads) return SASQ_ERR_SHAPE;
    if (!aligned16(c->k) || !aligned16(c->v)) return SASQ_ERR_ALIGN;
    return SASQ_OK;
}

// (The factors are an int8 cache's: what another's fields hold does not count.)
inline KvPages kv_pages(const sasq_kv_cache* c)
{
    const bool codes = c->fmt == SASQ_KV_INT8;
    const int64_t e = codes ? 1 : 2;
    return {static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), codes ? c->k_scale : nullptr, codes ? c->v_scale : nullptr, c->page_stride * e, c->token_stride * e,
            c->head_stride * e, (int)c->pages, __builtin_ctz((unsigned)c->page_size), (int)c->heads};
}

inline KvSteps kv_steps(const sasq_kv_batch* b)
{
    return {b->cu_q, b->kv_len, b->block_table, (int)b->batch, (int)b->max_pages, (int)b->tokens, (int)(b->max_q < b->tokens ? b->max_q : b->tokens)};
}

}  // namespace sasq
