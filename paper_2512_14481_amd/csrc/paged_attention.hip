// Causal attention of a step's new tokens over the paged key/value cache (sasq_paged_attention): entry points and host logic.
#include "attention.h"

#include <algorithm>
#include <cmath>

#ifndef SASQ_HEIGHT
#define SASQ_HEIGHT 128
#endif
namespace sasq {

constexpr int kFew = 64;                                 // rows of a kv head up to which a sequence is the rows kernel's

struct Plan {
    AttnSplit rows, tiles;
    bool tiled;                                           // some sequences may have more than kFew rows
    int64_t rows_slots, tiles_slots, most_blocks;
};

// Runs of `keys` keys: `runs` of them where possible, of whole tiles, at least `least` keys each and, unless that takes more than 256 runs, at most `most`.
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
    p.tiled = rows > kFew;
    // Few rows: enough workgroups to fill the chip a few times over, and runs short enough that sequences of very different lengths end
    // at about the same time.
    const int64_t tile = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
    p.rows.tile_rows = (int)tile;
    p.rows.tiles = 1;
    cut(p.rows, keys, (1024 + b->batch * c->heads - 1) / (b->batch * c->heads), 256, 2048);
    p.rows_slots = p.rows.splits > 1 ? p.rows.splits * b->batch * c->heads * tile : 0;
    p.most_blocks = p.rows.splits * b->batch * c->heads;
    if (p.tiled) {
        // Many rows: runs only where the tiles would leave the chip half empty.
        const int64_t height = SASQ_HEIGHT, about = std::max<int64_t>(1, b->tokens * group / height) * c->heads;
        p.tiles.tile_rows = (int)height;
        p.tiles.tiles = (int)((rows + height - 1) / height);
        cut(p.tiles, keys, 512 / about, 1024, INT64_C(1) << 30);
        p.tiles_slots = p.tiles.splits > 1 ? p.tiles.splits * b->tokens * q_heads : 0;
        p.most_blocks = std::max(p.most_blocks, p.tiles.splits * b->batch * p.tiles.tiles * c->heads);
    }
    return p;
}

}  // namespace sasq

using namespace sasq;

extern "C" size_t sasq_paged_attention_workspace(const sasq_kv_cache* cache, const sasq_kv_batch* batch, int64_t q_heads)
{
    if (kv_check(cache, batch, q_heads, SASQ_F16) != SASQ_OK) return 0;
    const Plan p = plan_of(cache, batch, q_heads);
    return (size_t)(p.rows_slots + p.tiles_slots) * (sizeof(float2) + sizeof(float) * cache->dim);
}

extern "C" int sasq_paged_attention(const void* q, void* out, float* lse, int64_t q_stride, int64_t out_stride, int64_t q_heads, float scale,
                                    const sasq_kv_cache* cache, const sasq_kv_batch* batch, sasq_dtype dt,
                                    void* workspace, size_t workspace_bytes, void* stream)
{
    if (!q || !out) return SASQ_ERR_NULL;
    if (const int rc = kv_check(cache, batch, q_heads, dt)) return rc;
    if (!std::isfinite(scale) || scale <= 0.0f) return SASQ_ERR_UNSUPPORTED;
    const int64_t dim = cache->dim, most = INT64_C(1) << 40;
    if (q_stride < q_heads * dim || out_stride < q_heads * dim || q_stride % 8 || out_stride % 8 || q_stride > most || out_stride > most) return SASQ_ERR_SHAPE;
    if (batch->tokens * q_heads >= INT64_C(1) << 31) return SASQ_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(out)) return SASQ_ERR_ALIGN;
    const size_t need = sasq_paged_attention_workspace(cache, batch, q_heads);
    if (need && (!workspace || workspace_bytes < need)) return SASQ_ERR_WORKSPACE;
    if (need && !aligned16(workspace)) return SASQ_ERR_ALIGN;

    Plan plan = plan_of(cache, batch, q_heads);
    if (plan.most_blocks >= INT64_C(1) << 31) return SASQ_ERR_SHAPE;
    float* o = static_cast<float*>(workspace);                             // the sums of both, then the maxima
    float2* ml = reinterpret_cast<float2*>(o + (plan.rows_slots + plan.tiles_slots) * dim);
    plan.rows.o = o;
    plan.rows.ml = ml;
    plan.tiles.o = o + plan.rows_slots * dim;
    plan.tiles.ml = ml + plan.rows_slots;
    const AttnArgs a{static_cast<const uint16_t*>(q), static_cast<uint16_t*>(out), lse, q_stride, out_stride, (int)q_heads, (int)(q_heads / cache->heads), scale};
    const KvPages pages = kv_pages(cache);
    const KvSteps steps = kv_steps(batch);
    const bool int8 = cache->fmt == SASQ_KV_INT8;
    const int few = plan.tiled ? kFew : INT32_MAX;
    hipStream_t st = as_stream(stream);
    int rc = SASQ_OK;
    if (plan.tiled) rc = attention_tiles_launch(a, pages, steps, plan.tiles, few, (int)dim, int8, dt, st);
    if (rc == SASQ_OK) rc = attention_rows_launch(a, pages, steps, plan.rows, few, (int)dim, int8, dt, st);
    if (rc == SASQ_OK && plan.tiles_slots) rc = attention_join_launch(a, pages, steps, plan.tiles, true, few, (int)dim, dt, st);
    if (rc == SASQ_OK && plan.rows_slots) rc = attention_join_launch(a, pages, steps, plan.rows, false, few, (int)dim, dt, st);
    return rc;
}
