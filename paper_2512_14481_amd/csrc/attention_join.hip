// Joins the partial results that runs of keys have left of a row (sasq_paged_attention).
#include "attention.h"

#include <algorithm>

namespace sasq {

// out = sum over runs of o 2^(m - top) / sum over runs of l 2^(m - top), D / 64 channels a lane.  First the sequences of many rows, a wave for
// each token and head, where these have runs; then those of few, whose runs may be many: a workgroup for a row, its four waves take every
// fourth run.  How many rows a sequence has is known here only; where places for all of them would make more than some 2048 workgroups,
// there are that many and each goes round (LOOP): ten single tokens beside two chunks of 13B, where 480 of 7680 would have had work, 93.6 us
// against 101 for the whole call.  Without LOOP there is one pass (two documents of 70B 95 us, going round 97).
// Bound by its waits, one after another (lengths, maxima, sums, output): 4 to 8 us.
constexpr int kJoinBlocks = 2048;
template <int DTQ, int D, bool LOOP>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a, KvPages cache, KvSteps steps, AttnSplit few, AttnSplit all_of_many, int many_blocks, int few_parts, int first)
{
    constexpr int E = D / 64;
    const int lane = (int)threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int block = (int)blockIdx.x + first;
    const bool many = block < many_blocks;
    const AttnSplit split = many ? all_of_many : few;
    __shared__ float parts[4][D + 1];
    int b, hk, r;
    if (many) {
        const int64_t row = (int64_t)block * 4 + wave;
        const int t = (int)(row / a.q_heads), head = (int)(row % a.q_heads);
        if (t >= steps.tokens) return;
        int before = 0;
        for (int i = 0; i <= steps.batch; i += kWave)
            before += __popcll(__ballot(i + lane <= steps.batch && steps.cu_q[min(i + lane, steps.batch)] <= t));
        b = before - 1;
        if (b < 0 || b >= steps.batch) return;
        hk = head / a.group;
        r = (t - kv_seq(steps, b, cache.page_shift).row0) * a.group + head % a.group;
    } else {
        const int at = block - many_blocks;
        r = at % few_parts;
        hk = at / few_parts % cache.heads;
        b = at / few_parts / cache.heads;
    }
    const KvSeq seq = kv_seq(steps, b, cache.page_shift);
    const int rows = seq.rows * a.group;
    if (r < 0 || (rows > kFewRows) != many) return;
    if (r >= rows || attn_runs(split, attn_end(seq, a.group, split, r / split.tile_rows)) == 1) return;      // nothing to do, or written already
    do {                                                                   // (a workgroup of the second kind goes through this as one)
        const int token = r / a.group, t = seq.row0 + token, head = hk * a.group + r % a.group;
        const int sees = kv_last(seq, token);
        const int runs = sees < 0 ? 0 : min(split.splits, sees / split.chunk + 1);            // later ones have no key of this row
        auto slot = [&](int i) -> int64_t { return many ? token_slot(steps.tokens, a.q_heads, i, t, head) : few_slot(split, steps.batch, cache.heads, i, b, hk, r); };
        float top = -INFINITY;
        for (int i = lane; i < runs; i += kWave) top = fmaxf(top, split.ml[slot(i)].x);
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
        float sum = 0.0f, x[E];
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = 0.0f;
#pragma unroll 8
        for (int i = many ? 0 : wave; i < runs; i += many ? 1 : 4) {
            const int64_t at = slot(i);
            const float2 f = split.ml[at];
            const float weight = part_weight(f, top);
            sum += f.y * weight;
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = __builtin_fmaf(split.o[at * D + lane * E + e], weight, x[e]);
        }
        if (!many) {
#pragma unroll
            for (int e = 0; e < E; ++e) parts[wave][lane * E + e] = x[e];
            if (lane == 0) parts[wave][D] = sum;
            __syncthreads();
            if (!LOOP && wave != 0) return;
            sum = (parts[0][D] + parts[1][D]) + (parts[2][D] + parts[3][D]);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = (parts[0][lane * E + e] + parts[1][lane * E + e]) + (parts[2][lane * E + e] + parts[3][lane * E + e]);
            if (LOOP) __syncthreads();
        }
        if (many || wave == 0) {
            const bool none = sum == 0.0f;
            const float f = none ? 0.0f : 1.0f / sum, v = cache.v_scale ? cache.v_scale[hk] : 1.0f;      // (apart, as in attention_rows.hip)
            uint16_t* dst = a.out + (int64_t)t * a.out_stride + (int64_t)head * D + lane * E;
#pragma unroll
            for (int e = 0; e < E; ++e) dst[e] = none ? (uint16_t)0 : Store16<DTQ>::enc(x[e] * f * v);
            if (a.lse && lane == 0) a.lse[(int64_t)t * a.q_heads + head] = none ? -INFINITY : (top + log2f(sum)) * 0.693147180559945f;
        }
        r += few_parts;
    } while (LOOP && !many && r < rows);
}

int attention_join_launch(const AttnArgs& a, const KvPages& c, const KvSteps& s, const AttnSplit& few, const AttnSplit& many, bool join_few, bool join_many, int dim,
                          sasq_dtype dt, hipStream_t st)
{
    const int64_t many_blocks = join_many ? ((int64_t)s.tokens * a.q_heads + 3) / 4 : 0, heads = (int64_t)s.batch * c.heads;
    const int64_t few_parts = std::min<int64_t>(few.rows, (kJoinBlocks + heads - 1) / heads), few_blocks = join_few ? heads * few_parts : 0;
    auto go = [&](auto kernel) {
        launch_in_parts(many_blocks + few_blocks, 256,
                        [&](unsigned n, int first) { hipLaunchKernelGGL(kernel, dim3(n), dim3(256), 0, st, a, c, s, few, many, (int)many_blocks, (int)few_parts, first); });
    };
    auto by_dim = [&](auto dtv) {
        constexpr int DTQ = decltype(dtv)::value;
        if (few_parts < few.rows) dim == 64 ? go(attention_join_kernel<DTQ, 64, true>) : go(attention_join_kernel<DTQ, 128, true>);
        else                      dim == 64 ? go(attention_join_kernel<DTQ, 64, false>) : go(attention_join_kernel<DTQ, 128, false>);
    };
    if (dt == SASQ_F16) by_dim(std::integral_constant<int, SASQ_F16>{});
    else                by_dim(std::integral_constant<int, SASQ_BF16>{});
    return hipGetLastError() == hipSuccess ? SASQ_OK : SASQ_ERR_LAUNCH;
}

}  // namespace sasq
