// The two products of sasq_linear_ce (linear_ce.h) on the tile body of the 16-bit GEMMs (gemm_k64_body.h).
#include "sasq_device.h"
#include "gemm_tile.h"
#include "gemm_k64_body.h"
#include "linear_ce.h"

namespace sasq {

// The tile of a workgroup among those of the rows that count, whose number only the device knows: the mapping of tile_of_block, ids past the
// last tile have nothing to do.
__device__ __forceinline__ bool tile_of_counted(int tiles_m, int tiles_n, int& tm, int& tn)
{
    const int per = (tiles_m * tiles_n + 7) >> 3;
    return (int)(blockIdx.x >> 3) < per && tile_of_block((int)blockIdx.x, tiles_m, tiles_n, tm, tn);
}

// Lanes l and l ^ 16, or l ^ 32, with the results of both.
__device__ __forceinline__ float max16(float v)
{
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float max32(float v)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float add16(float v)
{
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
__device__ __forceinline__ float add32(float v)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// ---- logits: z of a tile, reduced and stored as a_v ----
// 2 T V H operations; the epilogue (one exponential, four vector operations an element) is not overlapped with another tile's products: 4096 x 4096 -> 32000 in
// three pieces 809 us, 1.33 PFLOP/s (a library product of that size alone 845 us); 8192 x 8192 -> 32000 in bf16 2876 us, 1.49.  Matrix pipe busy 62 to 81 % under a
// tracer, the longer the contraction the more, at the 1.6 to 1.9 GHz that the power limit leaves.  In a row of 1376 the tiles' starts and ends are 40 % of them.
template <int DT, bool GRAD>
struct LogitsExt {
    static constexpr bool kOn = true;
    int x_kt, w_kt;
    const int32_t* tgt;
    float* zt;
    const RowStat* run;                         // of the pieces before, or NULL
    RowStat* stats;
    int64_t T;                                  // rows of `stats`
    uint16_t* a;
    int a_kt;                                   // blocks a row of blocks
    int col0;                                   // first column of the piece

    // Lane (fq, frow) of a wave holds, for each of its MF rows b * 16 + frow, the columns 16 g + 4 fq + e: a row's columns lie in the four lanes
    // of equal frow, which meet without LDS.  A 16-byte chunk of a_v is in two lanes; one exchange between neighbouring groups of sixteen
    // lanes gives each a whole one, and a wave's store is a whole 1 KB block.
    template <int BM, int BN, class ACC>
    __device__ __forceinline__ void finish(ACC& acc, int m0, int n0, int M, int N, char*) const
    {
        using S = Store16<DT>;
        constexpr int MF = BM / 32, NF = BN / 32;
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wm = wave & 1, wn = wave >> 1, frow = lane & 15, fq = lane >> 4;
        const int wn0 = n0 + wn * (BN / 2), wm0 = m0 + wm * (BM / 2);
        const bool edge = wn0 + BN / 2 > N;                    // columns past the vocabulary
        RowStat* stat = stats + (int64_t)((wn0 - col0) / (BN / 2)) * T;
        const int chunk = ((fq & 1) << 1) | (fq >> 1);         // of its row's four in a block
        uint16_t* dst = a + ((int64_t)(wm0 >> 4) * a_kt + ((wn0 - col0) >> 5)) * 512 + ((4 * frow + (chunk ^ swz64(frow))) << 3);
#pragma unroll
        for (int b = 0; b < MF; ++b) {
            __builtin_amdgcn_sched_barrier(0);                 // a row of tiles at a time: all of them at once need more registers than there are
            if (wm0 + b * 16 >= M) break;
            const int m = wm0 + b * 16 + frow;
            const int t = tgt[min(m, M - 1)] - wn0;            // the target's place among the wave's columns
            const bool here = t >= 0 && t < BN / 2 && ((t >> 2) & 3) == fq;
            const RowStat before = run ? run[min(m, M - 1)] : RowStat{0.0f, 0.0f};
            // Two copies of the rest: with the target or an edge among the columns, and without, where no element is looked at for them.
            auto rows = [&](auto special) {
                constexpr bool SPECIAL = decltype(special)::value;
                float zv[NF][4];
#pragma unroll
                for (int g = 0; g < NF; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) zv[g][e] = acc[g][b][e];
                if constexpr (SPECIAL) {
                    float z = 0.0f;
#pragma unroll
                    for (int g = 0; g < NF; ++g)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (here && t == 16 * g + 4 * fq + e) { z = zv[g][e]; zv[g][e] = -__builtin_inff(); }
                            if (edge && wn0 + 16 * g + 4 * fq + e >= N) zv[g][e] = -__builtin_inff();
                        }
                    if (here && m < M) zt[m] = z;
                }
                float top = zv[0][0];
#pragma unroll
                for (int g = 0; g < NF; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, zv[g][e]);
                top = max32(max16(top));
                // whole numbers, so that one M takes another's place by an exact factor
                float mm = ceilf(top * kLog2e) - (float)kTopExp<DT>;
                if (SPECIAL) mm = top == -__builtin_inff() ? 0.0f : mm;
                if (before.s != 0.0f && mm <= before.m + (float)kRoom<DT>) mm = before.m;
                float sum = 0.0f;
                u32x2 pk[NF];
#pragma unroll
                for (int g = 0; g < NF; ++g) {
                    float av[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        av[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(zv[g][e], kLog2e, -mm));
                        sum += av[e];
                    }
                    pk[g] = u32x2{S::pack(av[0], av[1]), S::pack(av[2], av[3])};
                }
                sum = add32(add16(sum));
                if (fq == 0 && m < M) stat[m] = RowStat{mm, sum};
                if constexpr (GRAD) {
#pragma unroll
                    for (int g = 0; g < NF; g += 2) {
                        const auto lo = __builtin_amdgcn_permlane16_swap(pk[g][0], pk[g + 1][0], false, false);
                        const auto hi = __builtin_amdgcn_permlane16_swap(pk[g][1], pk[g + 1][1], false, false);
                        *reinterpret_cast<u32x4*>(dst + (int64_t)b * a_kt * 512 + (g >> 1) * 512) = u32x4{lo[0], hi[0], lo[1], hi[1]};
                    }
                }
            };
            if (edge || __builtin_amdgcn_ballot_w64(here)) rows(std::true_type{});
            else                                           rows(std::false_type{});
        }
    }
};

// The tile of number `logical` in the order of tile_of_block.
__device__ __forceinline__ void tile_at(int logical, int tiles_m, int tiles_n, int& tm, int& tn)
{
    constexpr int PN = 4;
    const int panel = logical / (tiles_m * PN), in = logical - panel * tiles_m * PN, width = min(PN, tiles_n - panel * PN);
    tm = in / width;
    tn = panel * PN + in % width;
}

// Tiles of 256x256 come in rounds of 256 workgroups; a last round of at most 128 goes as twice as many tiles of 128 rows, which take 0.65 of a round, and so does
// a last row of tiles of at most 128 rows.
constexpr int kHalvesTo = 128;

template <int DT, int BM, int BN, bool GRAD>
__global__ __launch_bounds__(kGemmThreads)
__attribute__((amdgpu_waves_per_eu(Tile<BM, BN>::kWavesPerSimd, Tile<BM, BN>::kWavesPerSimd)))
void ce_logits_kernel(const uint16_t* __restrict__ xs, const uint8_t* __restrict__ head, const int32_t* __restrict__ count, int V, int Hp,
                      int tiles_n, LogitsExt<DT, GRAD> ext)
{
    __shared__ __attribute__((aligned(1024))) char lds[kStages * Tile<BM, BN>::kStageBytes];
    const int M = *count, tiles_m = (M + BM - 1) / BM;
    int tm, tn;
    if constexpr (BM == 256) {
        const int total = tiles_m * tiles_n, last = total % 256, tail = last <= kHalvesTo ? last : 0, whole = total - tail;
        const int id = tail ? (int)blockIdx.x - whole : -1, per = ((id < 0 ? whole : 2 * tail) + 7) >> 3, at = id < 0 ? (int)blockIdx.x : id;
        const int logical = (at & 7) * per + (at >> 3);
        if (at >> 3 >= per || logical >= (id < 0 ? whole : 2 * tail)) return;
        tile_at(id < 0 ? logical : whole + logical / 2, tiles_m, tiles_n, tm, tn);
        int half = 2 * tm + (id < 0 ? 0 : logical & 1);
        if (id >= 0 || M - tm * 256 <= 128) {
            if (half * 128 < M)
                gemm_k64_body<DT, KW_I8B, 128, BN, false, GR_NONE, 1, LogitsExt<DT, GRAD>>(
                    reinterpret_cast<const int8_t*>(xs), head, nullptr, nullptr, nullptr, nullptr, nullptr, M, V, Hp * 2, half, ext.col0 / BN + tn, lds, 0, ext);
            return;
        }
    } else if (!tile_of_counted(tiles_m, tiles_n, tm, tn)) {
        return;
    }
    gemm_k64_body<DT, KW_I8B, BM, BN, false, GR_NONE, 1, LogitsExt<DT, GRAD>>(
        reinterpret_cast<const int8_t*>(xs), head, nullptr, nullptr, nullptr, nullptr, nullptr, M, V, Hp * 2, tm, ext.col0 / BN + tn, lds, 0, ext);
}

// ---- gradient: running sums over v of a_v W_v ----
// 2 T V H operations; 4096 x 4096 x 32000 in three pieces 760 us, 1.41 PFLOP/s, 8192 x 8192 x 32000 in bf16 2944 us, 1.46 (under a tracer 866 and 3720 us at 1.7 to
// 1.8 GHz, the matrix pipe 74 and 79 % busy).  The sums stay in fp32 between pieces: read, multiplied by a power of two and added to in the epilogue.
struct SumsExt {
    static constexpr bool kOn = true;
    int x_kt, w_kt;
    float* acc;                                 // [T][Hp]
    const float* beta;                          // NULL: the first piece
    int Hp;

    template <int BM, int BN, class ACC>
    __device__ __forceinline__ void finish(ACC& sums, int m0, int n0, int M, int N, char*) const
    {
        constexpr int MF = BM / 32, NF = BN / 32;
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wm = wave & 1, wn = wave >> 1, frow = lane & 15, fq = lane >> 4;
        const int wn0 = n0 + wn * (BN / 2), wm0 = m0 + wm * (BM / 2);
        // The next row of tiles' old sums are requested before this one's are needed.
        f32x4 old[2][NF];
        float f[2] = {0.0f, 0.0f};
        auto fetch = [&](int b) {
            const int m = min(wm0 + b * 16 + frow, M - 1);
            f[b & 1] = beta[m];
#pragma unroll
            for (int g = 0; g < NF; ++g) old[b & 1][g] = *reinterpret_cast<const f32x4*>(acc + (int64_t)m * Hp + min(wn0 + 16 * g, Hp - 16) + 4 * fq);
        };
        if (beta) fetch(0);
#pragma unroll
        for (int b = 0; b < MF; ++b) {
            __builtin_amdgcn_sched_barrier(0);
            const int m = wm0 + b * 16 + frow;
            if (beta && b + 1 < MF) fetch(b + 1);
            __builtin_amdgcn_sched_barrier(0);
            float* row = acc + (int64_t)m * Hp + wn0 + 4 * fq;
#pragma unroll
            for (int g = 0; g < NF; ++g) {
                f32x4 v = sums[g][b];
                if (beta) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(old[b & 1][g][e], f[b & 1], v[e]);
                }
                if (m < M && wn0 + 16 * g < Hp) *reinterpret_cast<f32x4*>(row + 16 * g) = v;
            }
        }
    }
};

// Part `part` of `splits` of the contraction over the piece's columns, whole 64 columns each, with running sums of its own.
template <int DT, int BM, int BN>
__device__ __forceinline__ void grad_part(const uint16_t* a, const uint8_t* head_grad, int M, int H, int Hp, int cols64, int kt0, int part, int splits, int tm, int tn,
                                          char* lds, SumsExt ext)
{
    const int c0 = (int)((int64_t)cols64 * part / splits), c1 = (int)((int64_t)cols64 * (part + 1) / splits);
    ext.acc += (int64_t)part * M * Hp;
    if (c0 == c1) {                             // a last piece of fewer columns than parts
        for (int i = threadIdx.x; i < BM * (BN / 4); i += kGemmThreads) {
            const int m = tm * BM + i / (BN / 4), n = tn * BN + i % (BN / 4) * 4;
            if (m >= M || n >= Hp) continue;
            f32x4* at = reinterpret_cast<f32x4*>(ext.acc + (int64_t)m * Hp + n);
            f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
            if (ext.beta) {
                const float f = ext.beta[m];
                v = *at;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] *= f;
            }
            *at = v;
        }
        return;
    }
    gemm_k64_body<DT, KW_I8B, BM, BN, false, GR_NONE, 1, SumsExt>(
        reinterpret_cast<const int8_t*>(a) + (int64_t)c0 * 2048, head_grad + (int64_t)(kt0 + 2 * c0) * 1024, nullptr, nullptr, nullptr, nullptr, nullptr,
        M, H, (c1 - c0) * 128, tm, tn, lds, 0, ext);
}

template <int DT, int BM, int BN>
__global__ __launch_bounds__(kGemmThreads)
__attribute__((amdgpu_waves_per_eu(Tile<BM, BN>::kWavesPerSimd, Tile<BM, BN>::kWavesPerSimd)))
void ce_grad_kernel(const uint16_t* __restrict__ a, const uint8_t* __restrict__ head_grad, const int32_t* __restrict__ count, int H, int Hp,
                    int cols64, int kt0, int tiles_n, int slots, int max_splits, SumsExt ext)
{
    __shared__ __attribute__((aligned(1024))) char lds[kStages * Tile<BM, BN>::kStageBytes];
    const int M = *count;
    const GradParts parts = grad_parts(M, BM, tiles_n, slots, max_splits);
    const int whole = (parts.tiles * tiles_n * parts.full + 7) & ~7;
    int tm, tn;
    if ((int)blockIdx.x < whole) {
        if (!tile_of_block((int)blockIdx.x, parts.tiles, tiles_n * parts.full, tm, tn)) return;
        const int part = tn / tiles_n;
        grad_part<DT, BM, BN>(a, head_grad, M, H, Hp, cols64, kt0, part, parts.full, tm, tn - part * tiles_n, lds, ext);
        return;
    }
    if constexpr (BM == 256) {
        const int id = (int)blockIdx.x - whole;
        if (id >= ((tiles_n * parts.half + 7) & ~7) || !tile_of_block(id, 1, tiles_n * parts.half, tm, tn)) return;
        const int part = tn / tiles_n;
        grad_part<DT, 128, BN>(a, head_grad, M, H, Hp, cols64, kt0, part, parts.half, 2 * parts.tiles, tn - part * tiles_n, lds, ext);
    }
}

template <int DT, int BM, int BN>
static void launch_logits(const CeArgs& c, int64_t col0, int64_t cols, hipStream_t st)
{
    const int tiles_m = (int)((c.T + BM - 1) / BM), tiles_n = (int)((cols + BN - 1) / BN);
    const int grid = ((tiles_m * tiles_n + 7) / 8) * 8 + (BM == 256 ? kHalvesTo + 8 : 0);
    auto go = [&](auto grad_tag) {
        constexpr bool GRAD = decltype(grad_tag)::value;
        const LogitsExt<DT, GRAD> ext{row_blocks(c.Hp), row_blocks(c.Hp), c.tgt, c.zt, GRAD && col0 ? c.run : nullptr, c.stats, c.T, c.a, row_blocks(c.piece), (int)col0};
        ce_logits_kernel<DT, BM, BN, GRAD><<<grid, kGemmThreads, 0, st>>>(c.xs, c.head, c.count, (int)c.V, c.Hp, tiles_n, ext);
    };
    if (c.grad) go(std::true_type{});
    else        go(std::false_type{});
}

template <int DT, int BM, int BN>
static void launch_grad(const CeArgs& c, int64_t col0, int64_t cols, hipStream_t st)
{
    const int tiles_n = (int)((c.H + BN - 1) / BN);
    const int64_t tiles = (c.T + BM - 1) / BM * tiles_n, all = tiles * c.max_splits;
    // for any number of counted rows: a part a tile, or as many as there are slots, and a row of halves and what rounds up to whole eights
    const int64_t most = (tiles > c.slots ? tiles : all < c.slots ? all : c.slots) + tiles_n + 16;
    const SumsExt ext{row_blocks(c.piece), row_blocks(c.Vp), c.acc, col0 ? c.beta : nullptr, c.Hp};
    ce_grad_kernel<DT, BM, BN><<<(unsigned)most, kGemmThreads, 0, st>>>(
        c.a, c.head_grad, c.count, (int)c.H, c.Hp, (int)((cols + 63) / 64), (int)(col0 / 32), tiles_n, c.slots, c.max_splits, ext);
}

template <typename Go>
static void by_type_and_tile(sasq_dtype dt, int tile, Go&& go)
{
    auto by_tile = [&](auto d) {
        if (tile == 0) go(d, std::integral_constant<int, 256>{});
        else           go(d, std::integral_constant<int, 128>{});
    };
    if (dt == SASQ_F16) by_tile(std::integral_constant<int, SASQ_F16>{});
    else                by_tile(std::integral_constant<int, SASQ_BF16>{});
}

void launch_ce_logits(const CeArgs& c, sasq_dtype dt, int64_t col0, int64_t cols, hipStream_t st)
{
    by_type_and_tile(dt, c.tile, [&](auto d, auto b) { launch_logits<decltype(d)::value, decltype(b)::value, decltype(b)::value>(c, col0, cols, st); });
}

void launch_ce_grad(const CeArgs& c, sasq_dtype dt, int64_t col0, int64_t cols, hipStream_t st)
{
    by_type_and_tile(dt, c.grad_tile, [&](auto d, auto b) { launch_grad<decltype(d)::value, decltype(b)::value, decltype(b)::value>(c, col0, cols, st); });
}

}  // namespace sasq
