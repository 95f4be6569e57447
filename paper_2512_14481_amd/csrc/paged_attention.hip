// Causal attention of a step's new tokens over the paged key/value cache (sasq_paged_attention): entry points and host logic.
#include "attention.h"

#include <algorithm>
#include <cmath>

namespace sasq {

struct Plan {
    AttnSplit split;
    int64_t blocks, slots;                                // workgroups; rows of partial results
};

// Rows to a tile, and runs of keys: enough workgroups to fill the chip a few times over, of at least 256 keys each, and of at most 2048 keys
// where that does not take more than 256 runs, so that sequences of very different lengths end at about the same time.
static Plan plan_of(const sasq_kv_cache* c, const sasq_kv_batch* b, int64_t q_heads)
{
    Plan p{};
    const int64_t group = q_heads / c->heads, rows = std::min(b->max_q, b->tokens) * group;
    const int64_t keys = std::min(b->max_kv, b->max_pages * c->page_size);
    const int64_t tile = rows <= 16 ? 16 : rows <= 32 ? 32 : 64, tiles = (rows + tile - 1) / tile;
    const int64_t base = b->batch * c->heads * tiles;
    int64_t runs = std::min((1024 + base - 1) / base, (keys + 255) / 256);
    runs = std::min<int64_t>(std::max(runs, (keys + 2047) / 2048), 256);
    const int64_t chunk = ((keys + runs - 1) / runs + 127) / 128 * 128;
    runs = (keys + chunk - 1) / chunk;
    p.split = {(int)tile, (int)tiles, (int)chunk, (int)runs, nullptr, nullptr};
    p.blocks = runs * base;
    p.slots = runs > 1 ? runs * base * tile : 0;
    return p;
}

}  // namespace sasq

using namespace sasq;

extern "C" size_t sasq_paged_attention_workspace(const sasq_kv_cache* cache, const sasq_kv_batch* batch, int64_t q_heads)
{
    if (kv_check(cache, batch, q_heads, SASQ_F16) != SASQ_OK) return 0;
    return (size_t)plan_of(cache, batch, q_heads).slots * (sizeof(float2) + sizeof(float) * cache->dim);
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
    if (plan.blocks >= INT64_C(1) << 31) return SASQ_ERR_SHAPE;
    plan.split.ml = static_cast<float2*>(workspace);
    plan.split.o = reinterpret_cast<float*>(plan.split.ml + plan.slots);
    const AttnArgs a{static_cast<const uint16_t*>(q), static_cast<uint16_t*>(out), lse, q_stride, out_stride, (int)q_heads, (int)(q_heads / cache->heads), scale};
    return attention_rows_launch(a, kv_pages(cache), kv_steps(batch), plan.split, (int)dim, cache->fmt == SASQ_KV_INT8, dt, as_stream(stream));
}
