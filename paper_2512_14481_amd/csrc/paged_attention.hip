// Causal attention of a step's new tokens over the paged key/value cache (sasq_paged_attention): entry points and host logic.
#include "attention.h"

#include <algorithm>

namespace sasq {

struct Plan {
    AttnSplit few, many;
    bool tiled;                                           // some sequences may have more than kFewRows rows
    int64_t few_blocks, many_blocks, few_slots, many_slots;
};

// Runs of `keys` keys, of whole tiles: `runs` of them, but no more than one for every `least` keys begun (all but the last then have three quarters of that
// at least) and, up to 256, no fewer than one for every `most`.
static void cut(AttnSplit& s, int64_t keys, int64_t runs, int64_t least, int64_t most)
{
    runs = std::min(runs, (keys + least - 1) / least);
    runs = std::min<int64_t>(std::max(runs, (keys + most - 1) / most), 256);
    const int64_t chunk = ((keys + runs - 1) / runs + 127) / 128 * 128;
    s.chunk = (int)chunk;
    s.splits = (int)((keys + chunk - 1) / chunk);
}

static Plan plan_of(const sasq_kv_cache* c, const sasq_kv_batch* b, int64_t q_heads)
{
    Plan p{};
    const int64_t group = q_heads / c->heads, rows = std::min(b->max_q, b->tokens) * group;
    const int64_t keys = std::min(b->max_kv, b->max_pages * c->page_size);
    p.tiled = rows > kFewRows;
    // Few rows: about 1024 workgroups, four or two rounds of what the chip holds at a time (512: chunks beside single tokens 107 us against
    // 99), one for 512 keys begun at most (up to 512 no join: 9.2 us for 301 keys of 7B; with 256 two runs, 10.5), and of 2048 keys at most,
    // so that sequences of very different lengths end at about the same time (48 of 70B with 200 to 8190 keys: 109 us, with 4096 116).
    const int64_t heads = b->batch * c->heads;
    p.few.tile_rows = kFewRows;
    p.few.rows = (int)std::min<int64_t>(rows, kFewRows);
    cut(p.few, keys, (1024 + heads - 1) / heads, 512, 2048);
    p.few_blocks = group <= kFewRows ? p.few.splits * heads : 0;
    p.few_slots = p.few.splits > 1 ? p.few_blocks * p.few.rows : 0;
    if (p.tiled) {
        // Many rows: runs only where the tiles (about so many: a sequence's last one may be part empty) would leave the chip half empty: about
        // 768 workgroups, one and a half times what it holds at a time (five tokens for each of 16 of 70B: 39 us, with 1024 47; in tiles of
        // 128 rows 43, with 512 54, with 1024 52).
        p.many.tile_rows = rows <= kTileRows / 2 ? kTileRows / 2 : kTileRows;
        const int64_t full = b->tokens * group / p.many.tile_rows, other = std::min(b->batch, b->tokens);
        p.many.rows = (int)rows;
        cut(p.many, keys, 768 / (std::max(full, other) * c->heads), 512, INT64_C(1) << 30);
        p.many_blocks = p.many.splits * (full + other) * c->heads;
        p.many_slots = p.many.splits > 1 ? p.many.splits * b->tokens * q_heads : 0;
    }
    return p;
}

// Rows, and workgroups, are numbered in 32 bits.
static bool numbered(const Plan& p, const sasq_kv_cache* c, const sasq_kv_batch* b, int64_t q_heads)
{
    return b->tokens * q_heads < INT64_C(1) << 31 && p.few_blocks + p.many_blocks < INT64_C(1) << 31 && b->batch * c->heads * kFewRows < INT64_C(1) << 30;
}

}  // namespace sasq

using namespace sasq;

extern "C" size_t sasq_paged_attention_workspace(const sasq_kv_cache* cache, const sasq_kv_batch* batch, int64_t q_heads)
{
    if (kv_check(cache, batch, q_heads, SASQ_F16) != SASQ_OK) return 0;
    const Plan p = plan_of(cache, batch, q_heads);
    if (!numbered(p, cache, batch, q_heads)) return 0;
    return (size_t)(p.few_slots + p.many_slots) * (sizeof(float2) + sizeof(float) * cache->dim);
}

extern "C" int sasq_paged_attention(const void* q, void* out, float* lse, int64_t q_stride, int64_t out_stride, int64_t q_heads, float scale,
                                    const sasq_kv_cache* cache, const sasq_kv_batch* batch, sasq_dtype dt,
                                    void* workspace, size_t workspace_bytes, void* stream)
{
    if (!q || !out) return SASQ_ERR_NULL;
    if (const int rc = kv_check(cache, batch, q_heads, dt)) return rc;
    if (!(scale > 0.0f && scale <= 0x1p127f)) return SASQ_ERR_UNSUPPORTED;      // scale / ln 2 has to be finite too
    const int64_t dim = cache->dim, most = INT64_C(1) << 40;
    if (q_stride < q_heads * dim || out_stride < q_heads * dim || q_stride % 8 || out_stride % 8 || q_stride > most || out_stride > most) return SASQ_ERR_SHAPE;
    Plan plan = plan_of(cache, batch, q_heads);
    if (!numbered(plan, cache, batch, q_heads)) return SASQ_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(out)) return SASQ_ERR_ALIGN;
    const size_t need = sasq_paged_attention_workspace(cache, batch, q_heads);
    if (need && (!workspace || workspace_bytes < need)) return SASQ_ERR_WORKSPACE;
    if (need && !aligned16(workspace)) return SASQ_ERR_ALIGN;

    float* o = static_cast<float*>(workspace);                             // the sums of both kinds, then the maxima
    float2* ml = reinterpret_cast<float2*>(o + (plan.few_slots + plan.many_slots) * dim);
    plan.few.o = o;
    plan.few.ml = ml;
    plan.many.o = o + plan.few_slots * dim;
    plan.many.ml = ml + plan.few_slots;
    const AttnArgs a{static_cast<const uint16_t*>(q), static_cast<uint16_t*>(out), lse, q_stride, out_stride, (int)q_heads, (int)(q_heads / cache->heads), scale};
    const KvPages pages = kv_pages(cache);
    const KvSteps steps = kv_steps(batch);
    const bool int8 = cache->fmt == SASQ_KV_INT8;
    hipStream_t st = as_stream(stream);
    int rc = plan.tiled ? attention_tiles_launch(a, pages, steps, plan.few, plan.many, plan.many_blocks, plan.few_blocks, (int)dim, int8, dt, st)
                        : attention_rows_launch(a, pages, steps, plan.few, (int)dim, int8, dt, st);
    if (rc == SASQ_OK && plan.few_slots + plan.many_slots)
        rc = attention_join_launch(a, pages, steps, plan.few, plan.many, plan.few_slots > 0, plan.many_slots > 0, (int)dim, dt, st);
    return rc;
}
