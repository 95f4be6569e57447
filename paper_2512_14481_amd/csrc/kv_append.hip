// Append to the paged key/value cache: the new tokens' queries and keys rotated by position, keys and values stored (sasq_kv_append).
#include "kv_cache.h"

namespace sasq {

struct AppendArgs {
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    uint16_t* q_out;
    int64_t q_stride, k_stride, v_stride, q_out_stride;
    const float* __restrict__ cos;
    const float* __restrict__ sin;
    const int* __restrict__ positions;
    int table_rows, rot, q_heads;                        // rot 0: no rotation; q_heads 0: keys and values only
};

// Sixteen channels of a head as two pieces of eight.  Where the pairs that are turned together are halves apart, the pieces are too,
// so that a unit holds whole pairs; the lanes of a head then read whole lines with each of the two loads.
struct Unit {
    int at0, at1;
};
template <int STYLE>
__device__ __forceinline__ Unit unit_of(int u, int dim, int rot)
{
    if (rot == 0) return {8 * u, 8 * u + dim / 2};
    if (STYLE == SASQ_ROPE_HALVES && 16 * u < rot) return {8 * u, 8 * u + rot / 2};
    return {16 * u, 16 * u + 8};
}

template <int DT>
__device__ __forceinline__ void widen(const u32x4& w, float* f)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = Store16<DT>::lo(w[i]); f[2 * i + 1] = Store16<DT>::hi(w[i]); }
}
template <int DT>
__device__ __forceinline__ u32x4 narrow(const float* f)
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = Store16<DT>::pack(f[2 * i], f[2 * i + 1]);
    return w;
}

// Every product and sum is rounded by itself (the contract): no fused multiply-add.
template <int DT, int STYLE>
__device__ __forceinline__ void rotate(u32x4& w0, u32x4& w1, const float* c, const float* s)
{
    float a[8], b[8], x[8], y[8];
    widen<DT>(w0, a);
    widen<DT>(w1, b);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if constexpr (STYLE == SASQ_ROPE_HALVES) {
            x[j] = a[j] * c[j] - b[j] * s[j];
            y[j] = b[j] * c[j] + a[j] * s[j];
        } else {
            float* to = j < 4 ? x + 2 * j : y + 2 * (j - 4);
            const float* from = j < 4 ? a + 2 * j : b + 2 * (j - 4);
            to[0] = from[0] * c[j] - from[1] * s[j];
            to[1] = from[1] * c[j] + from[0] * s[j];
        }
    }
    w0 = narrow<DT>(x);
    w1 = narrow<DT>(y);
}

template <int DT>
__device__ __forceinline__ u32x2 codes8(const u32x4& w, const QConst& k)
{
    float f[8];
    widen<DT>(w, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = quantize(f[i], k).c;
    return {pack_codes4(f[0], f[1], f[2], f[3]), pack_codes4(f[4], f[5], f[6], f[7])};
}

// A workgroup takes 256 units of one token: its queries, then its keys, then its values; a lane reads, turns and writes 32 bytes, so that
// nothing passes through LDS and a token's units are read and written in whole lines.  The sequence is found by the wave (64 of cu_q at a time,
// from the cache) rather than by a list that a step before would have to make.  Bound by the bytes of long steps (4 x 2048 tokens of 70B: 60 us,
// 5.6 TB/s; 2649 of 13B into int8 33 us) and by launch and waits of short ones (one token of 7B 4.2 us, 200 of 70B the same).
template <int DT, int STYLE, bool I8>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a, KvPages cache, KvSteps steps, int dim, int parts, int first)
{
    const int block = (int)blockIdx.x + first, t = block / parts, lane = (int)threadIdx.x & 63;
    // The token's sequence: the last that starts at or before it, counted by the wave.
    int before = 0;
    for (int i = 0; i <= steps.batch; i += kWave) {
        const bool starts = i + lane <= steps.batch && steps.cu_q[min(i + lane, steps.batch)] <= t;
        before += __popcll(__ballot(starts));
    }
    const int b = before - 1;
    if (b < 0 || b >= steps.batch) return;
    const int per_head = dim / 16, units = (a.q_heads + 2 * cache.heads) * per_head;
    const int n = (block % parts) * 256 + (int)threadIdx.x;
    if (n >= units) return;
    const int head = n / per_head, u = n % per_head;
    const int part = head < a.q_heads ? 0 : head < a.q_heads + cache.heads ? 1 : 2;
    const int h = head - (part == 0 ? 0 : part == 1 ? a.q_heads : a.q_heads + cache.heads);
    const int64_t p = (int64_t)steps.kv_len[b] - steps.cu_q[b + 1] + t;
    const int64_t row = a.positions ? (int64_t)a.positions[t] : p;
    const bool in_table = a.rot == 0 || (row >= 0 && row < a.table_rows);

    const uint16_t* src = part == 0 ? a.q + t * a.q_stride : part == 1 ? a.k + t * a.k_stride : a.v + t * a.v_stride;
    src += (int64_t)h * dim;
    const Unit at = unit_of<STYLE>(u, dim, part == 2 ? 0 : a.rot);
    u32x4 w0 = *reinterpret_cast<const u32x4*>(src + at.at0), w1 = *reinterpret_cast<const u32x4*>(src + at.at1);
    if (part != 2 && 16 * u < a.rot && in_table) {
        const f32x4* cp = reinterpret_cast<const f32x4*>(a.cos + row * (a.rot / 2) + 8 * u);
        const f32x4* sp = reinterpret_cast<const f32x4*>(a.sin + row * (a.rot / 2) + 8 * u);
        const f32x4 c[2] = {cp[0], cp[1]}, s[2] = {sp[0], sp[1]};
        rotate<DT, STYLE>(w0, w1, reinterpret_cast<const float*>(c), reinterpret_cast<const float*>(s));
    }
    if (part == 0) {
        if (!in_table) w0 = w1 = u32x4{0, 0, 0, 0};
        uint16_t* dst = a.q_out + t * a.q_out_stride + (int64_t)h * dim;
        *reinterpret_cast<u32x4*>(dst + at.at0) = w0;
        *reinterpret_cast<u32x4*>(dst + at.at1) = w1;
        return;
    }
    if (!in_table || p < 0 || (p >> cache.page_shift) >= steps.max_pages) return;
    const int page = kv_page(cache, steps, b, (int)(p >> cache.page_shift));
    if (page < 0) return;
    uint8_t* dst = (part == 1 ? cache.k : cache.v) + page * cache.page_stride + (p & ((1 << cache.page_shift) - 1)) * cache.token_stride + h * cache.head_stride;
    if constexpr (I8) {
        const QConst k = make_qconst(part == 1 ? cache.k_scale[h] : cache.v_scale[h], 8);
        *reinterpret_cast<u32x2*>(dst + at.at0) = codes8<DT>(w0, k);
        *reinterpret_cast<u32x2*>(dst + at.at1) = codes8<DT>(w1, k);
    } else {
        *reinterpret_cast<u32x4*>(dst + 2 * at.at0) = w0;
        *reinterpret_cast<u32x4*>(dst + 2 * at.at1) = w1;
    }
}

}  // namespace sasq

using namespace sasq;

extern "C" int sasq_kv_append(const void* q, const void* k, const void* v, void* q_out, int64_t q_stride, int64_t k_stride,
                              int64_t v_stride, int64_t q_out_stride, int64_t q_heads, const float* cos, const float* sin,
                              const int32_t* positions, int64_t table_rows, int64_t rot_dim, sasq_rope style,
                              const sasq_kv_cache* cache, const sasq_kv_batch* batch, sasq_dtype dt, void* stream)
{
    if (!k || !v || !q != !q_out || !cos != !sin) return SASQ_ERR_NULL;
    if (const int rc = kv_check(cache, batch, q_heads, dt)) return rc;
    if (style != SASQ_ROPE_HALVES && style != SASQ_ROPE_PAIRS) return SASQ_ERR_UNSUPPORTED;
    const int64_t dim = cache->dim, most = INT64_C(1) << 40;
    if (cos && (rot_dim <= 0 || rot_dim > dim || rot_dim % 16 || table_rows <= 0 || table_rows > kKvMost)) return SASQ_ERR_SHAPE;
    if (q && (q_stride < q_heads * dim || q_out_stride < q_heads * dim || q_stride % 8 || q_out_stride % 8 || q_stride > most || q_out_stride > most)) return SASQ_ERR_SHAPE;
    if (k_stride < cache->heads * dim || v_stride < cache->heads * dim || k_stride % 8 || v_stride % 8 || k_stride > most || v_stride > most) return SASQ_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(cos) || !aligned16(sin)) return SASQ_ERR_ALIGN;

    const AppendArgs a{static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v),
                       static_cast<uint16_t*>(q_out), q_stride, k_stride, v_stride, q_out_stride, cos, sin, positions,
                       (int)table_rows, cos ? (int)rot_dim : 0, q ? (int)q_heads : 0};
    const int64_t units = (a.q_heads + 2 * cache->heads) * dim / 16, parts = (units + 255) / 256;
    if (batch->tokens * parts >= INT64_C(1) << 31) return SASQ_ERR_SHAPE;
    const KvPages pages = kv_pages(cache);
    const KvSteps steps = kv_steps(batch);
    hipStream_t st = as_stream(stream);
    auto go = [&](auto kernel) {
        launch_in_parts(batch->tokens * parts, 256, [&](unsigned blocks, int first) {
            hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, st, a, pages, steps, (int)dim, (int)parts, first);
        });
    };
    auto by_format = [&](auto dtv, auto stylev) {
        if (cache->fmt == SASQ_KV_INT8) go(kv_append_kernel<decltype(dtv)::value, decltype(stylev)::value, true>);
        else                            go(kv_append_kernel<decltype(dtv)::value, decltype(stylev)::value, false>);
    };
    auto by_style = [&](auto dtv) {
        if (style == SASQ_ROPE_HALVES) by_format(dtv, std::integral_constant<int, SASQ_ROPE_HALVES>{});
        else                           by_format(dtv, std::integral_constant<int, SASQ_ROPE_PAIRS>{});
    };
    if (dt == SASQ_F16) by_style(std::integral_constant<int, SASQ_F16>{});
    else                by_style(std::integral_constant<int, SASQ_BF16>{});
    return hipGetLastError() == hipSuccess ? SASQ_OK : SASQ_ERR_LAUNCH;
}
