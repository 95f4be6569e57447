// sasq_linear_ce for at most 64 rows, or more of a small head, 64 at a time (linear_ce.h): both products read the head once, from memory into registers, and are bound by that.
//
// A workgroup has 16 to 64 rows of a head's layout (vocabulary entries for the logits, channels for the gradient) and its eight waves an eighth of the
// contraction each: a wave loads 1 KB blocks, which are operands of v_mfma_f32_16x16x32 as they lie, and the rows of x (or their exponentials) beside them
// from L2.  The waves' sums meet in LDS.  4 to 8 blocks of the head are requested ahead by each wave, and 16 waves of a CU keep 64 to 128 KB in flight: one row of
// 4096 -> 32000 reads its 262 MB in 41 us, 6.4 TB/s (a large copy 5.2).  With 64 rows it is the rows of x that bind, 512 KB for every workgroup: 66 us.  No
// rows are packed: left-out ones are computed along and dropped.  33 to 48 rows go as 64 (with the gradient 32 | 33 | 48 | 64 rows 107 | 126 | 131 | 138 us).  The
// gradient's kernel reads the head again, in its other layout: one row takes 93 us with it.
#include "sasq_device.h"
#include "gemm_tile.h"
#include "gemm_k64_body.h"
#include "linear_ce.h"
#include <limits.h>

namespace sasq {

constexpr int kFewWaves = 8, kFewThreads = kFewWaves * kWave;
// Blocks of 16 rows whose sums meet at a time.
constexpr int few_at_once(int nb, int mb) { return nb == 1 ? mb : mb < 2 ? mb : 2; }
template <int NB, int MB>
using FewLds = float[kFewWaves][16 * few_at_once(NB, MB)][16 * NB + 4];

// Sums of a wave's share of the K steps [k0, k1), of 32 each and an even number, of W (row blocks at `w`, `w_kt` KB apart, of which `there` are there: the
// last one stands in for others) times 16 MB rows that `load` brings: lane (fq, frow) holds acc[nb][b][e], of row 16 b + frow and column 16 nb + 4 fq + e.
// The waves take the steps in turn, so that what a workgroup reads at a time lies together.
template <int DT, int NB, int MB, typename Load>
__device__ __forceinline__ void few_product(const uint8_t* __restrict__ w, int64_t w_kt, int there, int k0, int k1, f32x4 (&acc)[NB][MB], Load&& load)
{
    constexpr int kStep = NB + MB <= 5 ? 2 : 1;                   // K steps requested at once: what leaves room for the waves of two workgroups on a CU
    constexpr int kTurn = kStep * kFewWaves;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int b = 0; b < MB; ++b) acc[nb][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int lane = threadIdx.x & 63, r = lane & 15, c = lane >> 4;
    const uint32_t at = (uint32_t)(4 * r + (c ^ swz64(r))) << 4;
    i32x4 wf[2][kStep][NB], xf[2][kStep][MB];
    auto fetch = [&](int set, int k) {
#pragma unroll
        for (int s = 0; s < kStep; ++s) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
                wf[set][s][nb] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(w + (min(nb, there - 1) * w_kt + k + s) * 1024 + at));
#pragma unroll
            for (int b = 0; b < MB; ++b) xf[set][s][b] = load(b, k + s);
        }
    };
    auto multiply = [&](int set) {
#pragma unroll
        for (int s = 0; s < kStep; ++s)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
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

// Over EACH lanes next to each other (4, 8 or 16), for all of them.
template <int CTRL>
__device__ __forceinline__ float few_lane(float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true)); }
template <int EACH, typename Op>
__device__ __forceinline__ float few_fold(float v, Op&& op)
{
    v = op(v, few_lane<0xB1>(v));                              // neighbours,
    v = op(v, few_lane<0x4E>(v));                              // pairs in a four,
    if (EACH >= 8) v = op(v, few_lane<0x141>(v));              // the eight back to front,
    if (EACH == 16) v = op(v, few_lane<0x140>(v));             // the sixteen back to front
    return v;
}

// The waves' sums: in out[q] thread t has, of row 16 (few_at_once q) + t / (4 NB), the columns 4 (t % (4 NB)) .. + 3; threads past the rows of a pass have nothing.
template <int NB, int MB>
struct FewMeet {
    static constexpr int kAtOnce = few_at_once(NB, MB), kPasses = MB / kAtOnce, kEach = 4 * NB, kUsed = 16 * kAtOnce * kEach;
    static __device__ __forceinline__ int row(int q) { return 16 * kAtOnce * q + (int)threadIdx.x / kEach; }
    static __device__ __forceinline__ int col() { return 4 * ((int)threadIdx.x % kEach); }
    static __device__ __forceinline__ void run(const f32x4 (&acc)[NB][MB], FewLds<NB, MB>& lds, f32x4 (&out)[kPasses])
    {
        const int t = threadIdx.x, lane = t & 63, wave = t >> 6, frow = lane & 15, fq = lane >> 4;
#pragma unroll
        for (int q = 0; q < kPasses; ++q) {
            if (q) __syncthreads();
#pragma unroll
            for (int b = 0; b < kAtOnce; ++b)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) *reinterpret_cast<f32x4*>(&lds[wave][16 * b + frow][16 * nb + 4 * fq]) = acc[nb][q * kAtOnce + b];
            __syncthreads();
            out[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (t < kUsed) {
#pragma unroll
                for (int w = 0; w < kFewWaves; ++w) out[q] += *reinterpret_cast<const f32x4*>(&lds[w][t / kEach][col()]);
            }
        }
    }
};

// 16 NB columns a workgroup.
template <int DT, int NB, int MB, bool VEC, bool GRAD>
__global__ __launch_bounds__(kFewThreads) __attribute__((amdgpu_waves_per_eu(NB * MB == 16 || (MB == 4 && !VEC) ? 2 : 4))) void ce_few_logits_kernel(const uint16_t* __restrict__ x, int64_t stride, const uint8_t* __restrict__ head,
                                                           const int32_t* __restrict__ targets, int T, int V, int H, int Hp, RowStat* __restrict__ stats,
                                                           float* __restrict__ zt, uint16_t* __restrict__ a, int a_kt, int32_t* __restrict__ count,
                                                           uint32_t* __restrict__ ticket)
{
    using S = Store16<DT>;
    using Meet = FewMeet<NB, MB>;
    __shared__ __attribute__((aligned(16))) FewLds<NB, MB> lds;
    const int t = threadIdx.x, lane = t & 63, frow = lane & 15, fq = lane >> 4;
    const int v0 = (int)blockIdx.x * 16 * NB;
    const int r0 = (int)blockIdx.y * kFewRows;
    if (blockIdx.x + blockIdx.y == 0 && t < 64) {              // how many rows count, for the kernels behind this one
        constexpr int kAhead = 8;
        int all = 0;
        for (int i0 = t; i0 - t < T; i0 += 64 * kAhead) {
            int v[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) v[j] = targets[min(i0 + 64 * j, T - 1)];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) all += __popcll(__builtin_amdgcn_ballot_w64(i0 + 64 * j < T && v[j] >= 0 && v[j] < V));
        }
        if (t == 0) {
            *count = all;
            *ticket = 0;
        }
    }
    const int64_t w_kt = row_blocks(Hp);
    f32x4 acc[NB][MB];
    int tgt[Meet::kPasses];                                    // of the rows that this thread reduces at the end
#pragma unroll
    for (int q = 0; q < Meet::kPasses; ++q) tgt[q] = targets[min(r0 + Meet::row(q), T - 1)];
    const uint16_t* row[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) row[b] = x + (int64_t)min(r0 + 16 * b + frow, T - 1) * stride;
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
    // columns past the vocabulary's end, whole workgroups of them up to the next 64, are dropped below
    const int w0 = min(v0 >> 4, (V - 1) >> 4);
    few_product<DT, NB, MB>(head + (int64_t)w0 * w_kt * 1024, w_kt, ((V - 1) >> 4) - w0 + 1, 0, Hp / 32, acc, load);
    f32x4 z[Meet::kPasses];
    Meet::run(acc, lds, z);
    if (t >= Meet::kUsed) return;
    const int v = v0 + Meet::col();
#pragma unroll
    for (int q = 0; q < Meet::kPasses; ++q) {
        const int m = r0 + Meet::row(q);
        const int target = tgt[q];
        float top = -__builtin_inff();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (v + e == target && v + e < V && m < T) zt[m] = z[q][e];
            if (v + e >= V || v + e == target) z[q][e] = -__builtin_inff();
            top = fmaxf(top, z[q][e]);
        }
        top = few_fold<Meet::kEach>(top, [](float x, float y) { return fmaxf(x, y); });
        const float mm = top == -__builtin_inff() ? 0.0f : ceilf(top * kLog2e) - (float)kTopExp<DT>;
        float av[4], sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            av[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[q][e], kLog2e, -mm));
            sum += av[e];
        }
        sum = few_fold<Meet::kEach>(sum, [](float x, float y) { return x + y; });
        if (Meet::col() == 0 && m < T) stats[(int64_t)blockIdx.x * T + m] = RowStat{mm, sum};
        if (GRAD) *reinterpret_cast<u32x2*>(a + block_at(m, v & ~7, a_kt) + (v & 4)) = u32x2{S::pack(av[0], av[1]), S::pack(av[2], av[3])};
    }
}

// The gradient's sums over a part of the vocabulary; exponentials are brought to their row's M on the way.
template <int DT, int MB, bool JOIN>
__global__ __launch_bounds__(kFewThreads) __attribute__((amdgpu_waves_per_eu(MB == 4 ? 2 : 4))) void ce_few_grad_kernel(const uint16_t* __restrict__ a, int a_kt, const uint8_t* __restrict__ head_grad, int T, int H, int Hp, int Vp,
                                                         const RowStat* __restrict__ stats, int stat_shift, const RowStat* __restrict__ run, float* __restrict__ acc_out, int parts)
{
    using S = Store16<DT>;
    constexpr int NB = kFewCols / 16;
    using Meet = FewMeet<NB, MB>;
    __shared__ __attribute__((aligned(16))) FewLds<NB, MB> lds;
    const int t = threadIdx.x, lane = t & 63, frow = lane & 15, fq = lane >> 4;
    const int cols = (Hp + kFewCols - 1) / kFewCols, part = (int)blockIdx.x / cols, h0 = (int)blockIdx.x % cols * kFewCols;
    const int r0 = (int)blockIdx.y * kFewRows;
    // in pairs of K steps
    const int pairs = Vp / 64, p0 = (int)((int64_t)pairs * part / parts), p1 = (int)((int64_t)pairs * (part + 1) / parts);
    f32x4 acc[NB][MB];
    float m[MB];
    if constexpr (JOIN) {                                      // the rows' M, whole numbers, from their groups' (no kernel has joined them)
        __shared__ int top[64];
        if (t < 64) top[t] = INT_MIN;
        __syncthreads();
        const int all = (Vp >> stat_shift) * T;
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
        for (int b = 0; b < MB; ++b) m[b] = run[min(r0 + 16 * b + frow, T - 1)].m;
    }
    auto load = [&](int b, int k) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(a + block_at(r0 + 16 * b + frow, k * 32 + 8 * fq, a_kt));
        const float f = exp2f(fminf(stats[(int64_t)((k * 32 + 8 * fq) >> stat_shift) * T + min(r0 + 16 * b + frow, T - 1)].m - m[b], 0.0f));     // (a group of nothing but the target has no M)
        u32x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = S::pack(S::lo(v[e]) * f, S::hi(v[e]) * f);
        return __builtin_bit_cast(i32x4, o);
    };
    const int64_t w_kt = row_blocks(Vp);
    // sums of channels past the end are not used
    few_product<DT, NB, MB>(head_grad + (int64_t)(h0 >> 4) * w_kt * 1024, w_kt, ((H - 1) >> 4) - (h0 >> 4) + 1, 2 * p0, 2 * p1, acc, load);
    f32x4 out[Meet::kPasses];
    Meet::run(acc, lds, out);
    if (t >= Meet::kUsed) return;
#pragma unroll
    for (int q = 0; q < Meet::kPasses; ++q) {
        const int row = r0 + Meet::row(q), h = h0 + Meet::col();
        if (row < T) *reinterpret_cast<f32x4*>(acc_out + ((int64_t)part * T + row) * Hp + h) = out[q];
    }
}

void launch_ce_few_logits(const CeArgs& c, sasq_dtype dt, hipStream_t st)
{
    const dim3 grid(c.Vp / c.few_cols, (unsigned)((c.T + kFewRows - 1) / kFewRows));
    const int mb = (int)((c.T + 15) / 16);
    const bool vec = c.x_stride % 8 == 0 && c.H % 8 == 0;
    auto launch = [&](auto d, auto nb, auto m, auto v, auto g) {
        ce_few_logits_kernel<decltype(d)::value, decltype(nb)::value, decltype(m)::value, decltype(v)::value, decltype(g)::value><<<grid, kFewThreads, 0, st>>>(
            static_cast<const uint16_t*>(c.x), c.x_stride, c.head, c.targets, (int)c.T, (int)c.V, (int)c.H, c.Hp, c.stats, c.zt, c.a, row_blocks(c.piece),
            c.count, c.ticket);
    };
    auto go = [&](auto d, auto m, auto v, auto g) {
        if (c.few_cols == 16)      launch(d, std::integral_constant<int, 1>{}, m, v, g);
        else if (c.few_cols == 32) launch(d, std::integral_constant<int, 2>{}, m, v, g);
        else                       launch(d, std::integral_constant<int, 4>{}, m, v, g);
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
    const dim3 grid((c.Hp + kFewCols - 1) / kFewCols * c.few_parts, (unsigned)((c.T + kFewRows - 1) / kFewRows));
    const int mb = (int)((c.T + 15) / 16), stat_shift = c.few_cols == 16 ? 4 : c.few_cols == 32 ? 5 : 6;
    auto go = [&](auto d, auto m) {
        if (c.few_own_join)
            ce_few_grad_kernel<decltype(d)::value, decltype(m)::value, true><<<grid, kFewThreads, 0, st>>>(
                c.a, row_blocks(c.piece), c.head_grad, (int)c.T, (int)c.H, c.Hp, c.Vp, c.stats, stat_shift, c.run, c.acc, c.few_parts);
        else
            ce_few_grad_kernel<decltype(d)::value, decltype(m)::value, false><<<grid, kFewThreads, 0, st>>>(c.a, row_blocks(c.piece), c.head_grad, (int)c.T, (int)c.H, c.Hp, c.Vp,
                                                                                        c.stats, stat_shift, c.run, c.acc, c.few_parts);
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
