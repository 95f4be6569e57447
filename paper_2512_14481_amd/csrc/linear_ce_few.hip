// sasq_linear_ce for at most 64 rows (linear_ce.h): both products read the head once, from memory into registers, and are bound by that.
//
// A workgroup has 64 rows of a head's layout (64 vocabulary entries for the logits, 64 channels for the gradient) and its eight waves an eighth of the
// contraction each: a wave loads four 1 KB blocks at a time, which are four operands of v_mfma_f32_16x16x32 as they lie, and the rows of x (or their
// exponentials) beside them from L2.  The waves' sums meet in LDS.  There are as many waves as fill the chip twice from 32000 entries on, each with 8 to 16 KB
// requested ahead.  No rows are packed: left-out ones are computed along and dropped.
#include "sasq_device.h"
#include "gemm_tile.h"
#include "gemm_k64_body.h"
#include "linear_ce.h"
#include <limits.h>

namespace sasq {

constexpr int kFewBlocks = kFewCols / 16, kFewPitch = kFewCols + 4, kFewWaves = 8, kFewThreads = kFewWaves * kWave;

// Sums of a wave's share of the K steps [k0, k1), of 32 each and an even number, of W (row blocks at `w`, `w_kt` KB apart, of which `there` are there: the
// last one stands in for others) times 16 MB rows that `load` brings: lane (fq, frow) holds acc[nb][b][e], of row 16 b + frow and column 16 nb + 4 fq + e.
// The waves take the steps in turn, so that what a workgroup reads at a time lies together.
template <int DT, int MB, typename Load>
__device__ __forceinline__ void few_product(const uint8_t* __restrict__ w, int64_t w_kt, int there, int k0, int k1, f32x4 (&acc)[kFewBlocks][MB], Load&& load)
{
    constexpr int kStep = MB == 1 ? 2 : 1;                     // K steps requested at once: what leaves room for the waves of two workgroups on a CU
    constexpr int kTurn = kStep * kFewWaves;
#pragma unroll
    for (int nb = 0; nb < kFewBlocks; ++nb)
#pragma unroll
        for (int b = 0; b < MB; ++b) acc[nb][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int lane = threadIdx.x & 63, r = lane & 15, c = lane >> 4;
    const uint32_t at = (uint32_t)(4 * r + (c ^ swz64(r))) << 4;
    i32x4 wf[2][kStep][kFewBlocks], xf[2][kStep][MB];
    auto fetch = [&](int set, int k) {
#pragma unroll
        for (int s = 0; s < kStep; ++s) {
#pragma unroll
            for (int nb = 0; nb < kFewBlocks; ++nb)
                wf[set][s][nb] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(w + (min(nb, there - 1) * w_kt + k + s) * 1024 + at));
#pragma unroll
            for (int b = 0; b < MB; ++b) xf[set][s][b] = load(b, k + s);
        }
    };
    auto multiply = [&](int set) {
#pragma unroll
        for (int s = 0; s < kStep; ++s)
#pragma unroll
            for (int nb = 0; nb < kFewBlocks; ++nb)
#pragma unroll
                for (int b = 0; b < MB; ++b) acc[nb][b] = Mfma16x16<DT>::mma(wf[set][s][nb], xf[set][s][b], acc[nb][b]);
    };
    int k = k0 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * kStep;         // uniform: block addresses stay scalar
    if (k < k1) fetch(0, k);
    for (; k < k1; k += 2 * kTurn) {
        if (k + kTurn < k1) fetch(1, k + kTurn);
        multiply(0);
        if (k + 2 * kTurn < k1) fetch(0, k + 2 * kTurn);
        if (k + kTurn < k1) multiply(1);
    }
}

template <int N>
__device__ __forceinline__ float few_turn(float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x120 + N, 0xf, 0xf, true)); }
// Over sixteen lanes next to each other, for all of them.
__device__ __forceinline__ float few_max(float v)
{
    v = fmaxf(v, few_turn<8>(v));
    v = fmaxf(v, few_turn<4>(v));
    v = fmaxf(v, few_turn<2>(v));
    return fmaxf(v, few_turn<1>(v));
}
__device__ __forceinline__ float few_sum(float v)
{
    v += few_turn<8>(v);
    v += few_turn<4>(v);
    v += few_turn<2>(v);
    return v + few_turn<1>(v);
}

// The waves' sums: thread t of the first 256 then has, of row 16 b + t / 16, the columns 4 (t % 16) .. + 3.
template <int MB>
__device__ __forceinline__ void few_meet(const f32x4 (&acc)[kFewBlocks][MB], float (&lds)[kFewWaves][16][kFewPitch], f32x4 (&out)[MB])
{
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, frow = lane & 15, fq = lane >> 4;
#pragma unroll
    for (int b = 0; b < MB; ++b) {
        if (b) __syncthreads();
#pragma unroll
        for (int nb = 0; nb < kFewBlocks; ++nb) *reinterpret_cast<f32x4*>(&lds[wave][frow][16 * nb + 4 * fq]) = acc[nb][b];
        __syncthreads();
        out[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) out[b] += *reinterpret_cast<const f32x4*>(&lds[w][(t >> 4) & 15][4 * (t & 15)]);
    }
}

template <int DT, int MB, bool VEC, bool GRAD>
__global__ __launch_bounds__(kFewThreads) __attribute__((amdgpu_waves_per_eu(MB == 4 ? 2 : 4))) void ce_few_logits_kernel(const uint16_t* __restrict__ x, int64_t stride, const uint8_t* __restrict__ head,
                                                           const int32_t* __restrict__ targets, int T, int V, int H, int Hp, RowStat* __restrict__ stats,
                                                           float* __restrict__ zt, uint16_t* __restrict__ a, int a_kt, int32_t* __restrict__ count,
                                                           uint32_t* __restrict__ ticket)
{
    using S = Store16<DT>;
    __shared__ __attribute__((aligned(16))) float lds[kFewWaves][16][kFewPitch];
    const int t = threadIdx.x, lane = t & 63, frow = lane & 15, fq = lane >> 4;
    const int v0 = (int)blockIdx.x * kFewCols;
    if (blockIdx.x == 0 && t < 64) {                           // how many rows count, for the kernels behind this one
        const int v = t < T ? targets[t] : -1;
        const uint64_t mask = __builtin_amdgcn_ballot_w64(v >= 0 && v < V);
        if (t == 0) {
            *count = __popcll(mask);
            *ticket = 0;
        }
    }
    const int64_t w_kt = row_blocks(Hp);
    f32x4 acc[kFewBlocks][MB];
    int tgt[MB];                                               // of the rows that this thread reduces at the end
#pragma unroll
    for (int b = 0; b < MB; ++b) tgt[b] = targets[min(16 * b + ((t >> 4) & 15), T - 1)];
    const uint16_t* row[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) row[b] = x + (int64_t)min(16 * b + frow, T - 1) * stride;
    auto load = [&](int b, int k) {
        const int h = k * 32 + 8 * fq;
        u32x4 o = {0u, 0u, 0u, 0u};
        if (VEC) {
            if (h < H) o = *reinterpret_cast<const u32x4*>(row[b] + h);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t lo = h + 2 * e < H ? row[b][h + 2 * e] : 0u, hi = h + 2 * e + 1 < H ? row[b][h + 2 * e + 1] : 0u;
                o[e] = lo | hi << 16;
            }
        }
        return __builtin_bit_cast(i32x4, o);
    };
    // columns past the vocabulary's end are dropped below
    few_product<DT, MB>(head + (int64_t)(v0 >> 4) * w_kt * 1024, w_kt, ((V - 1) >> 4) - (v0 >> 4) + 1, 0, Hp / 32, acc, load);
    f32x4 z[MB];
    few_meet<MB>(acc, lds, z);
    if (t >= 256) return;
    const int r16 = t >> 4, v = v0 + 4 * (t & 15);
#pragma unroll
    for (int b = 0; b < MB; ++b) {
        const int m = 16 * b + r16;
        const int target = tgt[b];
        float top = -__builtin_inff();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (v + e == target && v + e < V && m < T) zt[m] = z[b][e];
            if (v + e >= V || v + e == target) z[b][e] = -__builtin_inff();
            top = fmaxf(top, z[b][e]);
        }
        top = few_max(top);
        const float mm = top == -__builtin_inff() ? 0.0f : ceilf(top * kLog2e) - (float)kTopExp<DT>;
        float av[4], sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            av[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][e], kLog2e, -mm));
            sum += av[e];
        }
        sum = few_sum(sum);
        if ((t & 15) == 0 && m < T) stats[(int64_t)blockIdx.x * T + m] = RowStat{mm, sum};
        if (GRAD) *reinterpret_cast<u32x2*>(a + block_at(m, v, a_kt)) = u32x2{S::pack(av[0], av[1]), S::pack(av[2], av[3])};
    }
}

// The gradient's sums over a part of the vocabulary; exponentials are brought to their row's M on the way.
template <int DT, int MB, bool JOIN>
__global__ __launch_bounds__(kFewThreads) __attribute__((amdgpu_waves_per_eu(MB == 4 ? 2 : 4))) void ce_few_grad_kernel(const uint16_t* __restrict__ a, int a_kt, const uint8_t* __restrict__ head_grad, int T, int H, int Hp, int Vp,
                                                         const RowStat* __restrict__ stats, const RowStat* __restrict__ run, float* __restrict__ acc_out, int parts)
{
    using S = Store16<DT>;
    __shared__ __attribute__((aligned(16))) float lds[kFewWaves][16][kFewPitch];
    const int t = threadIdx.x, lane = t & 63, frow = lane & 15, fq = lane >> 4;
    const int cols = (Hp + kFewCols - 1) / kFewCols, part = (int)blockIdx.x / cols, h0 = (int)blockIdx.x % cols * kFewCols;
    // K steps in pairs: 64 columns share M and S
    const int pairs = Vp / 64, p0 = (int)((int64_t)pairs * part / parts), p1 = (int)((int64_t)pairs * (part + 1) / parts);
    f32x4 acc[kFewBlocks][MB];
    float m[MB];
    if constexpr (JOIN) {                                      // the rows' M, whole numbers, from their groups' (no kernel has joined them)
        __shared__ int top[64];
        if (t < 64) top[t] = INT_MIN;
        __syncthreads();
        const int all = (Vp / kFewCols) * T;
        for (int i = t; i < all; i += kFewThreads) {
            const RowStat s = stats[i];
            if (s.s != 0.0f) atomicMax(&top[i % T], (int)s.m);
        }
        __syncthreads();
#pragma unroll
        for (int b = 0; b < MB; ++b) {
            const int at = top[min(16 * b + frow, T - 1)];
            m[b] = at == INT_MIN ? 0.0f : (float)at;
        }
    } else {
#pragma unroll
        for (int b = 0; b < MB; ++b) m[b] = run[min(16 * b + frow, T - 1)].m;
    }
    auto load = [&](int b, int k) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(a + block_at(16 * b + frow, k * 32 + 8 * fq, a_kt));
        const float f = exp2f(fminf(stats[(int64_t)(k >> 1) * T + min(16 * b + frow, T - 1)].m - m[b], 0.0f));     // (a group of nothing but the target has no M)
        u32x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = S::pack(S::lo(v[e]) * f, S::hi(v[e]) * f);
        return __builtin_bit_cast(i32x4, o);
    };
    const int64_t w_kt = row_blocks(Vp);
    // sums of channels past the end are not used
    few_product<DT, MB>(head_grad + (int64_t)(h0 >> 4) * w_kt * 1024, w_kt, ((H - 1) >> 4) - (h0 >> 4) + 1, 2 * p0, 2 * p1, acc, load);
    f32x4 out[MB];
    few_meet<MB>(acc, lds, out);
    if (t >= 256) return;
#pragma unroll
    for (int b = 0; b < MB; ++b) {
        const int row = 16 * b + (t >> 4), h = h0 + 4 * (t & 15);
        if (row < T) *reinterpret_cast<f32x4*>(acc_out + ((int64_t)part * T + row) * Hp + h) = out[b];
    }
}

void launch_ce_few_logits(const CeArgs& c, sasq_dtype dt, hipStream_t st)
{
    const int grid = (int)((c.V + kFewCols - 1) / kFewCols), mb = (int)((c.T + 15) / 16);
    const bool vec = c.x_stride % 8 == 0 && c.H % 8 == 0;
    auto go = [&](auto d, auto m, auto v, auto g) {
        ce_few_logits_kernel<decltype(d)::value, decltype(m)::value, decltype(v)::value, decltype(g)::value><<<grid, kFewThreads, 0, st>>>(
            static_cast<const uint16_t*>(c.x), c.x_stride, c.head, c.targets, (int)c.T, (int)c.V, (int)c.H, c.Hp, c.stats, c.zt, c.a, row_blocks(c.piece),
            c.count, c.ticket);
    };
    auto by_grad = [&](auto d, auto m, auto v) { if (c.grad) go(d, m, v, std::true_type{}); else go(d, m, v, std::false_type{}); };
    auto by_vec = [&](auto d, auto m) { if (vec) by_grad(d, m, std::true_type{}); else by_grad(d, m, std::false_type{}); };
    auto by_rows = [&](auto d) {
        if (mb == 1)      by_vec(d, std::integral_constant<int, 1>{});
        else if (mb == 2) by_vec(d, std::integral_constant<int, 2>{});
        else              by_vec(d, std::integral_constant<int, 4>{});
    };
    if (dt == SASQ_F16) by_rows(std::integral_constant<int, SASQ_F16>{});
    else                by_rows(std::integral_constant<int, SASQ_BF16>{});
}

void launch_ce_few_grad(const CeArgs& c, sasq_dtype dt, hipStream_t st)
{
    const int mb = (int)((c.T + 15) / 16), grid = (c.Hp + kFewCols - 1) / kFewCols * c.few_parts;
    auto go = [&](auto d, auto m) {
        if (c.few_own_join)
            ce_few_grad_kernel<decltype(d)::value, decltype(m)::value, true><<<grid, kFewThreads, 0, st>>>(
                c.a, row_blocks(c.piece), c.head_grad, (int)c.T, (int)c.H, c.Hp, c.Vp, c.stats, c.run, c.acc, c.few_parts);
        else
            ce_few_grad_kernel<decltype(d)::value, decltype(m)::value, false><<<grid, kFewThreads, 0, st>>>(c.a, row_blocks(c.piece), c.head_grad, (int)c.T, (int)c.H, c.Hp, c.Vp,
                                                                                        c.stats, c.run, c.acc, c.few_parts);
    };
    auto by_rows = [&](auto d) {
        if (mb == 1)      go(d, std::integral_constant<int, 1>{});
        else if (mb == 2) go(d, std::integral_constant<int, 2>{});
        else              go(d, std::integral_constant<int, 4>{});
    };
    if (dt == SASQ_F16) by_rows(std::integral_constant<int, SASQ_F16>{});
    else                by_rows(std::integral_constant<int, SASQ_BF16>{});
}

}  // namespace sasq
