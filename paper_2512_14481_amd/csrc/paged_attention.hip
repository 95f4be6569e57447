// Causal attention of a step's new tokens over the paged key/value cache (sasq_paged_attention): entry points and host logic.
#include "kv_cache.h"

#include <cmath>

namespace sasq {

struct AttnArgs {
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    int64_t q_stride, out_stride;
    int q_heads;
    float scale;
};

// One wave for each new token and head, two (or one) channels a lane, one key after the other with the running maximum and sum of
// the softmax.
template <int DT, int D, bool I8>
__global__ __launch_bounds__(64) void attention_plain_kernel(AttnArgs a, KvPages cache, KvSteps steps, int first)
{
    constexpr int E = D / 64;
    const int block = (int)blockIdx.x + first, t = block / a.q_heads, h = block % a.q_heads, lane = (int)threadIdx.x;
    int before = 0;
    for (int i = 0; i <= steps.batch; i += kWave) {
        const bool starts = i + lane <= steps.batch && steps.cu_q[min(i + lane, steps.batch)] <= t;
        before += __popcll(__ballot(starts));
    }
    const int b = before - 1;
    if (b < 0 || b >= steps.batch) return;
    const KvSeq seq = kv_seq(steps, b, cache.page_shift);
    const int last = seq.keys - seq.rows + (t - seq.row0);                 // the token's own position
    const int hk = h / (a.q_heads / cache.heads);
    const float ks = I8 ? cache.k_scale[hk] : 1.0f, vs = I8 ? cache.v_scale[hk] : 1.0f;
    float qf[E], o[E], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) { qf[e] = Store16<DT>::one(a.q[t * a.q_stride + (int64_t)h * D + lane * E + e]); o[e] = 0.0f; }
    for (int j = 0; j <= last; ++j) {
        const int page = kv_page(cache, steps, b, j >> cache.page_shift);
        if (page < 0) continue;
        const int64_t at = page * cache.page_stride + (j & ((1 << cache.page_shift) - 1)) * cache.token_stride + hk * cache.head_stride;
        float k[E], v[E], s = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if constexpr (I8) {
                k[e] = (float)reinterpret_cast<const int8_t*>(cache.k + at)[lane * E + e] * ks;
                v[e] = (float)reinterpret_cast<const int8_t*>(cache.v + at)[lane * E + e] * vs;
            } else {
                k[e] = Store16<DT>::one(reinterpret_cast<const uint16_t*>(cache.k + at)[lane * E + e]);
                v[e] = Store16<DT>::one(reinterpret_cast<const uint16_t*>(cache.v + at)[lane * E + e]);
            }
            s = __builtin_fmaf(qf[e], k[e], s);
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, kWave);
        s *= a.scale;
        const float top = fmaxf(m, s), keep = top == -INFINITY ? 1.0f : __expf(m - top), p = top == -INFINITY ? 0.0f : __expf(s - top);
        l = l * keep + p;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * keep + p * v[e];
        m = top;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) a.out[t * a.out_stride + (int64_t)h * D + lane * E + e] = Store16<DT>::enc(l > 0.0f || l != l ? o[e] / l : 0.0f);
    if (a.lse && lane == 0) a.lse[(int64_t)t * a.q_heads + h] = l > 0.0f || l != l ? m + logf(l) : -INFINITY;
}

}  // namespace sasq

using namespace sasq;

extern "C" size_t sasq_paged_attention_workspace(const sasq_kv_cache* cache, const sasq_kv_batch* batch, int64_t q_heads)
{
    return 0;
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

    const AttnArgs a{static_cast<const uint16_t*>(q), static_cast<uint16_t*>(out), lse, q_stride, out_stride, (int)q_heads, scale};
    const KvPages pages = kv_pages(cache);
    const KvSteps steps = kv_steps(batch);
    hipStream_t st = as_stream(stream);
    auto go = [&](auto kernel) {
        launch_in_parts(batch->tokens * q_heads, 64, [&](unsigned blocks, int first) {
            hipLaunchKernelGGL(kernel, dim3(blocks), dim3(64), 0, st, a, pages, steps, first);
        });
    };
    auto by_format = [&](auto dtv, auto dimv) {
        if (cache->fmt == SASQ_KV_INT8) go(attention_plain_kernel<decltype(dtv)::value, decltype(dimv)::value, true>);
        else                            go(attention_plain_kernel<decltype(dtv)::value, decltype(dimv)::value, false>);
    };
    auto by_dim = [&](auto dtv) {
        if (dim == 64) by_format(dtv, std::integral_constant<int, 64>{});
        else           by_format(dtv, std::integral_constant<int, 128>{});
    };
    if (dt == SASQ_F16) by_dim(std::integral_constant<int, SASQ_F16>{});
    else                by_dim(std::integral_constant<int, SASQ_BF16>{});
    return hipGetLastError() == hipSuccess ? SASQ_OK : SASQ_ERR_LAUNCH;
}
