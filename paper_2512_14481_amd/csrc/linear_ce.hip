// Cross entropy of a frozen output head (linear_ce.h): laying the head out, the rows that count, the steps between the two products, entry points.
#include "sasq_device.h"
#include "gemm_tile.h"
#include "linear_ce.h"
#include <math.h>

namespace sasq {

constexpr int64_t kCeMaxTokens = INT64_C(1) << 23, kCeMaxVocab = INT64_C(1) << 22, kCeMaxHidden = INT64_C(1) << 20;
constexpr int64_t kCeMaxProduct = INT64_C(1) << 37;                 // elements of x, of the head, and of a piece of the logits
constexpr int kPieceStep = 256;

static int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }

// ---- the head's two layouts: 1 KB blocks of 16 rows x 32 columns, chunks swizzled as in every operand of the GEMMs ----
// Once a head, bound by bytes: 32000 x 4096, 524 MB in and out, 96 us (5.5 TB/s) for the logits, 111 us (4.8) turned for the gradient.
__device__ __forceinline__ uint16_t head_at(const uint16_t* w, int64_t stride, int64_t v, int64_t h, int64_t V, int64_t H)
{
    return v < V && h < H ? w[v * stride + h] : (uint16_t)0;
}

// Rows v, columns h.  A thread takes one 16-byte chunk.
__global__ __launch_bounds__(256) void head_logits_kernel(const uint16_t* __restrict__ w, int64_t stride, u32x4* __restrict__ out, int64_t V, int64_t H,
                                                         int64_t kt, int64_t chunks, bool vec)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (int64_t)gridDim.x * 256) {
        const int64_t block = i >> 6;
        const int r = (int)(i & 63) >> 2, c = ((int)i & 3) ^ swz64(r);
        const int64_t v = block / kt * 16 + r, h = block % kt * 32 + 8 * c;
        u32x4 o = {0u, 0u, 0u, 0u};
        if (vec && v < V && h + 8 <= H) {
            o = *reinterpret_cast<const u32x4*>(w + v * stride + h);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                o[e] = head_at(w, stride, v, h + 2 * e, V, H) | (uint32_t)head_at(w, stride, v, h + 2 * e + 1, V, H) << 16;
        }
        out[i] = o;
    }
}

// Rows h, columns v: 64 x 64 elements at a time through LDS.
__global__ __launch_bounds__(256) void head_grad_kernel(const uint16_t* __restrict__ w, int64_t stride, u32x4* __restrict__ out, int64_t V, int64_t H,
                                                       int64_t hb, int64_t kt, int64_t tiles, bool vec)
{
    __shared__ uint16_t tile[64][64 + 8];
    const int64_t tiles_h = (H + 63) / 64;
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int64_t v0 = t / tiles_h * 64, h0 = t % tiles_h * 64;
        __syncthreads();
        for (int i = threadIdx.x; i < 64 * 8; i += 256) {
            const int r = i >> 3, c = (i & 7) * 8;
            const int64_t v = v0 + r, h = h0 + c;
            u32x4 o = {0u, 0u, 0u, 0u};
            if (vec && v < V && h + 8 <= H) {
                o = *reinterpret_cast<const u32x4*>(w + v * stride + h);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    o[e] = head_at(w, stride, v, h + 2 * e, V, H) | (uint32_t)head_at(w, stride, v, h + 2 * e + 1, V, H) << 16;
            }
            *reinterpret_cast<u32x4*>(&tile[r][c]) = o;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 8 * 64; i += 256) {                      // 4 x 2 blocks of 64 chunks
            const int b = i >> 6, r = (i & 63) >> 2, c = (i & 3) ^ swz64(r);
            const int h = (b >> 1) * 16 + r, v = (b & 1) * 32 + 8 * c;
            const int64_t hblock = (h0 >> 4) + (b >> 1);
            if (hblock >= hb) continue;
            u32x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = tile[v + 2 * e][h] | (uint32_t)tile[v + 2 * e + 1][h] << 16;
            out[(hblock * kt + (v0 >> 5) + (b & 1)) * 64 + (i & 63)] = o;
        }
    }
}

// ---- the rows that count, packed together: the tiles of the two products then hold no row that is left out (711 of 1777 rows count,
// 5120 -> 32000: 420 us, at 2.5 times the products more than 900) ----
constexpr int kPackThreads = 1024;
__global__ __launch_bounds__(kPackThreads) void ce_pack_kernel(const int32_t* __restrict__ targets, int T, int V, int32_t* __restrict__ count,
                                                              int32_t* __restrict__ pos, int32_t* __restrict__ row, int32_t* __restrict__ tgt,
                                                              float* __restrict__ loss, float* __restrict__ lse, uint32_t* __restrict__ ticket,
                                                              float* __restrict__ mean)
{
    __shared__ int wave_count[kPackThreads / kWave];
    constexpr int kEach = 4;                                   // rows of a thread, next to each other
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    int base = 0;
    for (int r0 = 0; r0 < T; r0 += kPackThreads * kEach) {
        int v[kEach];
        bool counts[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int r = r0 + t * kEach + j;
            v[j] = r < T ? targets[r] : -1;
        }
        int below = 0, all = 0;                                // counted rows of the lanes before this one, and of the wave
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            counts[j] = v[j] >= 0 && v[j] < V;
            const uint64_t mask = __builtin_amdgcn_ballot_w64(counts[j]);
            below += __popcll(mask & ((UINT64_C(1) << lane) - 1));
            all += __popcll(mask);
        }
        if (lane == 0) wave_count[wave] = all;
        __syncthreads();
        int before = 0, round = 0;
#pragma unroll
        for (int w = 0; w < kPackThreads / kWave; ++w) {
            before += w < wave ? wave_count[w] : 0;
            round += wave_count[w];
        }
        __syncthreads();
        int p = base + before + below;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int r = r0 + t * kEach + j;
            if (counts[j]) {
                pos[r] = p;
                row[p] = r;
                tgt[p] = v[j];
                ++p;
            } else if (r < T) {
                pos[r] = -1;
                loss[r] = 0.0f;
                if (lse) lse[r] = 0.0f;
            }
        }
        base += round;
    }
    if (t == 0) {
        *count = base;
        *ticket = 0;
        if (mean && base == 0) *mean = 0.0f;
    }
}

// A wave copies one counted row of x to its packed place, with zeros past H, four loads of 1 KB ahead.  Bytes: 4096 x 4096 (and the counting) 16.9 us, 4.0 TB/s.
template <bool VEC>
__device__ __forceinline__ void ce_stage_row(const uint16_t* __restrict__ src, uint16_t* __restrict__ xs, int p, int H, int Hp)
{
    constexpr int kAhead = 4;
    for (int h0 = (int)(threadIdx.x & 63) * 8; h0 < Hp; h0 += 512 * kAhead) {
        u32x4 o[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int h = h0 + 512 * j;
            o[j] = u32x4{0u, 0u, 0u, 0u};
            if (VEC) {
                if (h < H) o[j] = *reinterpret_cast<const u32x4*>(src + h);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t lo = h + 2 * e < H ? src[h + 2 * e] : 0u, hi = h + 2 * e + 1 < H ? src[h + 2 * e + 1] : 0u;
                    o[j][e] = lo | hi << 16;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (h0 + 512 * j < Hp) *reinterpret_cast<u32x4*>(xs + block_at(p, h0 + 512 * j, row_blocks(Hp))) = o[j];
    }
}
template <bool VEC>
__global__ __launch_bounds__(256) void ce_stage_kernel(const uint16_t* __restrict__ x, int64_t stride, uint16_t* __restrict__ xs, const int32_t* __restrict__ count,
                                                      const int32_t* __restrict__ row, int H, int Hp)
{
    const int p = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6);
    if (p < *count) ce_stage_row<VEC>(x + (int64_t)row[p] * stride, xs, p, H, Hp);
}

// Both at once: a workgroup counts the rows before its four by itself, up to kPackedTo rows (a launch and its wait less, 4 us; the counting takes T^2 / 2 bytes
// of L2 reads, 32 MB at most).
constexpr int kPackedTo = 8192;
template <bool VEC>
__global__ __launch_bounds__(256) void ce_pack_stage_kernel(const uint16_t* __restrict__ x, int64_t stride, uint16_t* __restrict__ xs,
                                                           const int32_t* __restrict__ targets, int T, int V, int32_t* __restrict__ count,
                                                           int32_t* __restrict__ pos, int32_t* __restrict__ row, int32_t* __restrict__ tgt,
                                                           float* __restrict__ loss, float* __restrict__ lse, uint32_t* __restrict__ ticket,
                                                           float* __restrict__ mean, int H, int Hp)
{
    constexpr int kAhead = 8;
    __shared__ int wave_count[4];
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), r0 = (int)blockIdx.x * 4;
    int mine[4], before = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) mine[j] = r0 + j < T ? targets[r0 + j] : -1;
    for (int i = t; i - t < r0; i += 256 * kAhead) {
        int v[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) v[j] = targets[min(i + 256 * j, T - 1)];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) before += __popcll(__builtin_amdgcn_ballot_w64(i + 256 * j < r0 && v[j] >= 0 && v[j] < V));
    }
    if ((t & 63) == 0) wave_count[wave] = before;
    __syncthreads();
    int p = wave_count[0] + wave_count[1] + wave_count[2] + wave_count[3], own = -1, target = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bool counts = mine[j] >= 0 && mine[j] < V;
        if (j == wave && counts) { own = p; target = mine[j]; }
        p += counts;
    }
    const int r = r0 + wave;
    if (t == 0 && r0 + 4 >= T) {                               // the last four rows
        *count = p;
        *ticket = 0;
        if (mean && p == 0) *mean = 0.0f;
    }
    if (r >= T) return;
    if ((t & 63) == 0) {
        pos[r] = own;
        if (own >= 0) {
            row[own] = r;
            tgt[own] = target;
        } else {
            loss[r] = 0.0f;
            if (lse) lse[r] = 0.0f;
        }
    }
    if (own >= 0) ce_stage_row<VEC>(x + (int64_t)r * stride, xs, own, H, Hp);
}

// ---- between the products: M and S of each row so far ----
// ROWS rows a workgroup, 1024 / ROWS threads a row, eight groups of columns requested at a time by each.  16 rows, whose M and S are whole cache lines, or 4
// where a row has many groups (333 x 1376 -> 100003, 1564 groups, 16 | 4 rows: 15.0 | 10.8 us).  Otherwise 6 to 9 us, its waits one after another.  All factors are exact powers of two.
// targets: rows are not packed, and some of the T may be left out; NULL: they are, and *count of them are there.
constexpr int kJoinThreads = 1024, kJoinAhead = 8, kJoinManyGroups = 512;

struct RowEnd { float loss, lse, u, coef; };
// What M and S over the others and z of the target make of a row, in fp64: a small loss is the exponential of a difference.
__device__ __forceinline__ RowEnd row_end(float m, float s, float zt)
{
    const double z = (double)zt;
    const double d = s == 0.0f ? -(double)__builtin_inff() : ((double)m + log2((double)s)) * 0.69314718055994530942 - z;
    const double ex = exp(-fabs(d)), over = 1.0 / (1.0 + ex);
    const double l = fmax(d, 0.0) + log1p(ex), u = d > 0.0 ? over : ex * over;
    return RowEnd{(float)l, (float)(z + l), (float)u, s == 0.0f ? 0.0f : (float)(u / (double)s)};
}

template <int ROWS>
__global__ __launch_bounds__(kJoinThreads) void ce_join_kernel(const RowStat* __restrict__ stats, int groups, int64_t T, const int32_t* __restrict__ count,
                                                              RowStat* __restrict__ run, float* __restrict__ beta, uint8_t* __restrict__ scale_rows,
                                                              const float* __restrict__ zt, const int32_t* __restrict__ row, float* __restrict__ coef,
                                                              float* __restrict__ u_out, float* __restrict__ loss, float* __restrict__ lse,
                                                              float* __restrict__ mean, double* __restrict__ part_loss, uint32_t* __restrict__ ticket,
                                                              const int32_t* __restrict__ targets, int V, int first, int last)
{
    constexpr int kJoinRows = ROWS, kJoinLanes = kJoinThreads / ROWS, kWaves = kJoinThreads / kWave;
    __shared__ float part[kWaves][kJoinRows];
    __shared__ double row_loss[kJoinRows];
    __shared__ bool is_last;
    const int r = threadIdx.x % kJoinRows, k = threadIdx.x / kJoinRows, p = (int)blockIdx.x * kJoinRows + r;
    const RowStat* mine = stats + min((int64_t)p, T - 1);      // (rows past the counted ones hold anything)
    const RowStat old = first ? RowStat{0.0f, 0.0f} : run[min((int64_t)p, T - 1)];
    const int target = targets ? targets[min((int64_t)p, T - 1)] : 0;
    const float target_z = zt[min((int64_t)p, T - 1)];
    const int to = row ? row[min((int64_t)p, T - 1)] : p;
    RowStat s[kJoinAhead];
    auto fetch = [&](int g0) {
#pragma unroll
        for (int j = 0; j < kJoinAhead; ++j) {
            const int g = g0 + j * kJoinLanes;
            s[j] = mine[(int64_t)min(g, groups - 1) * T];
            if (g >= groups) s[j].s = 0.0f;
        }
    };
    float top = -__builtin_inff();
    fetch(k);
    const int counted = *count, n = targets ? (int)T : counted;
    if ((int)blockIdx.x * kJoinRows >= n) return;
    for (int g0 = k; g0 < groups; g0 += kJoinLanes * kJoinAhead) {
        if (g0 != k) fetch(g0);
#pragma unroll
        for (int j = 0; j < kJoinAhead; ++j)
            if (s[j].s != 0.0f) top = fmaxf(top, s[j].m);
    }
    // a row's threads in a wave meet by shuffles, the waves in LDS
    const int wave = threadIdx.x / kWave;
    auto share = [&](float v) {
        if (threadIdx.x % kWave < kJoinRows) part[wave][r] = v;
    };
#pragma unroll
    for (int o = ROWS; o < kWave; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
    share(top);
    __syncthreads();
    float m = old.s != 0.0f ? old.m : -__builtin_inff();
#pragma unroll
    for (int j = 0; j < kWaves; ++j) m = fmaxf(m, part[j][r]);
    if (m == -__builtin_inff()) m = 0.0f;
    __syncthreads();
    float sum = 0.0f;
    bool other = false;
    for (int g0 = k; g0 < groups; g0 += kJoinLanes * kJoinAhead) {
        if (groups > kJoinLanes * kJoinAhead) fetch(g0);
#pragma unroll
        for (int j = 0; j < kJoinAhead; ++j) {
            if (s[j].s != 0.0f) sum += s[j].s * exp2f(s[j].m - m);
            other = other || (s[j].s != 0.0f && s[j].m != m);
        }
    }
#pragma unroll
    for (int o = ROWS; o < kWave; o <<= 1) sum += __shfl_xor(sum, o, kWave);
    share(sum);
    const int any = __syncthreads_or(other && p < n);
    if (scale_rows && threadIdx.x == 0) scale_rows[blockIdx.x] = any != 0;
    if (k == 0 && p < n) {
        const float f = old.s != 0.0f ? exp2f(old.m - m) : 0.0f;
        float all = old.s * f;
#pragma unroll
        for (int j = 0; j < kWaves; ++j) all += part[j][r];
        run[p] = RowStat{m, all};
        beta[p] = f;
        if (last) {
            const bool counts = !targets || (target >= 0 && target < V);
            const RowEnd end = row_end(m, all, target_z);
            loss[to] = counts ? end.loss : 0.0f;
            if (lse) lse[to] = counts ? end.lse : 0.0f;
            u_out[p] = end.u;
            coef[p] = end.coef;
            row_loss[r] = counts ? (double)end.loss : 0.0;
        }
    } else if (k == 0) {
        row_loss[r] = 0.0;
    }
    if (!last || !mean) return;
    // the mean, where no kernel follows: every workgroup's sum is published, the last to arrive adds them in their order
    __syncthreads();
    const int blocks = (n + kJoinRows - 1) / kJoinRows;
    if (threadIdx.x == 0) {
        double all = 0.0;
        for (int j = 0; j < kJoinRows; ++j) all += row_loss[j];
        if (blocks == 1) {
            *mean = counted ? (float)(all / (double)counted) : 0.0f;
            is_last = false;
        } else is_last = publish_then_ticket(&part_loss[blockIdx.x], all, ticket) == (uint32_t)blocks - 1;
    }
    __syncthreads();
    if (!is_last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    __shared__ double wave_part[kJoinThreads / kWave];
    double all = 0.0;
    for (int i = threadIdx.x; i < blocks; i += kJoinThreads) all += __hip_atomic_load(&part_loss[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    all = wave_sum(all);
    if (threadIdx.x % kWave == 0) wave_part[threadIdx.x / kWave] = all;
    __syncthreads();
    if (threadIdx.x) return;
    all = 0.0;
    for (int j = 0; j < kJoinThreads / kWave; ++j) all += wave_part[j];
    *mean = counted ? (float)(all / (double)counted) : 0.0f;
}

// a_v of groups of columns with another M than their row's, in place: sixteen rows and `each` blocks a workgroup, a 1 KB block a wave and access.
// Bytes: 333 x 100003, all of them, 134 MB in 24 us, 5.5 TB/s (64 blocks a workgroup 28); where no row has to be touched 4.6 us, a launch and its wait.  Doing it on the fragments in the
// gradient GEMM instead costs that kernel more: 256x256 tiles 386 -> 448 us (their registers move), 128x128 123 -> 130.
template <int DT>
__global__ __launch_bounds__(256) void ce_scale_kernel(uint16_t* __restrict__ a, int a_kt, int kt, int stat_blocks, const RowStat* __restrict__ stats,
                                                      const RowStat* __restrict__ run, const uint8_t* __restrict__ scale_rows, int flags, int64_t T,
                                                      const int32_t* __restrict__ count, int each)
{
    using S = Store16<DT>;
    const int n = *count, r16 = (int)blockIdx.x;
    if (r16 * 16 >= n) return;
    int any = 0;                                              // `flags` of the join's workgroups tell for sixteen rows
    for (int f = r16 * flags; f < (r16 + 1) * flags && f * (16 / flags) < n; ++f) any |= scale_rows[f];
    if (!any) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int p = min(r16 * 16 + (lane >> 2), n - 1);
    const float m = run[p].m;
    const int k1 = min(kt, ((int)blockIdx.y + 1) * each);
    u32x4* at = reinterpret_cast<u32x4*>(a) + (int64_t)r16 * a_kt * 64 + lane;
    constexpr int kAhead = 4;
    for (int k = (int)blockIdx.y * each + wave; k < k1; k += 4 * kAhead) {
        u32x4 v[kAhead];
        float f[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int kk = min(k + 4 * j, k1 - 1);
            v[j] = at[(int64_t)kk * 64];
            f[j] = stats[(int64_t)(kk / stat_blocks) * T + p].m;
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (k + 4 * j >= k1) break;
            const float s = exp2f(fminf(f[j] - m, 0.0f));      // (a group of nothing but the target has no M, and zeros)
            u32x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = S::pack(S::lo(v[j][e]) * s, S::hi(v[j][e]) * s);
            at[(int64_t)(k + 4 * j) * 64] = o;
        }
    }
}

// M, S and what follows of row r from the groups of columns of a single piece, by `each` threads of a wave next to each other (a power of two), of which this is
// number i.
__device__ __forceinline__ RowEnd few_row_end(const RowStat* __restrict__ stats, int groups, int T, int r, float zt, int i, int each)
{
    constexpr int kAhead = 4;
    RowStat s[kAhead];
    auto fetch = [&](int g0) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            s[j] = stats[(int64_t)min(g0 + j * each, groups - 1) * T + r];
            if (g0 + j * each >= groups) s[j].s = 0.0f;
        }
    };
    float m = -__builtin_inff(), sum = 0.0f;
    for (int g0 = i; g0 < groups; g0 += each * kAhead) {
        fetch(g0);
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (s[j].s != 0.0f) m = fmaxf(m, s[j].m);
    }
    for (int o = 1; o < each; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
    if (m == -__builtin_inff()) m = 0.0f;
    for (int g0 = i; g0 < groups; g0 += each * kAhead) {
        if (groups > each * kAhead) fetch(g0);
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (s[j].s != 0.0f) sum += s[j].s * exp2f(s[j].m - m);
    }
    for (int o = 1; o < each; o <<= 1) sum += __shfl_xor(sum, o, kWave);
    return row_end(m, sum, zt);
}

// ---- the end: dx of every row, kDxCols channels a workgroup; left-out ones are 0 ----
// Bytes: the sums, W of the targets and dx, 4096 x 4096 169 MB in 28.6 us, 5.9 TB/s; a lane adds four parts' sums of eight channels at a time.
constexpr int kDxCols = 256 * 8;
// JOIN: few rows of few groups of columns, which no other kernel has joined: a workgroup does so for its row, the one more for all.
template <int DT, bool VEC, bool JOIN>
__global__ __launch_bounds__(256) void ce_dx_kernel(const float* __restrict__ acc, int bm, int tiles_n, int slots, int max_splits, int few_parts, const int32_t* __restrict__ count,
                                                   const int32_t* __restrict__ pos, const int32_t* __restrict__ tgt, const float* __restrict__ coef,
                                                   const float* __restrict__ u, const uint8_t* __restrict__ head, const float* __restrict__ row_weight,
                                                   float scale, uint16_t* __restrict__ dx, int64_t stride, int H, int Hp, const float* __restrict__ loss,
                                                   float* __restrict__ mean, int T, int V, const RowStat* __restrict__ stats, int groups,
                                                   const float* __restrict__ zt, float* __restrict__ loss_out, float* __restrict__ lse)
{
    using S = Store16<DT>;
    const int r = (int)blockIdx.x, h = (int)blockIdx.y * kDxCols + (int)threadIdx.x * 8;
    if (r == T) {                                 // a workgroup more: the mean, in fp64 and a fixed order
        if (blockIdx.y) return;
        __shared__ double part[4];
        double sum = 0.0;
        if constexpr (JOIN) {
            // (few rows: as many threads for each as there are)
            const int each = T <= 4 ? 64 : T <= 8 ? 32 : T <= 16 ? 16 : T <= 32 ? 8 : 4, i = (int)threadIdx.x / each;
            const int t = tgt[min(i, T - 1)];
            const RowEnd end = few_row_end(stats, groups, T, min(i, T - 1), zt[min(i, T - 1)], (int)threadIdx.x % each, each);
            if (i < T && t >= 0 && t < V && threadIdx.x % each == 0) sum = (double)end.loss;
        } else {
            for (int i = threadIdx.x; i < T; i += 256) sum += (double)loss[i];
        }
        sum = wave_sum(sum);
        if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = sum;
        __syncthreads();
        if (threadIdx.x == 0) *mean = *count ? (float)((part[0] + part[1] + part[2] + part[3]) / (double)*count) : 0.0f;
        return;
    }
    // few_parts: rows are not packed, and their targets tell which count
    int p = few_parts ? r : pos[r];
    float g = 0.0f, cf = 0.0f, uu = 0.0f;
    int t = 0;
    const int n = *count, splits = few_parts ? few_parts : grad_parts(n, bm, tiles_n, slots, max_splits).of_row(p, bm), rows = few_parts ? T : n;
    if (p >= 0) {
        t = tgt[p];
        if (few_parts && (t < 0 || t >= V)) p = -1;
    }
    if (p >= 0) g = scale * (row_weight ? row_weight[r] : 1.0f / (float)n);
    if constexpr (JOIN) {
        const RowEnd end = few_row_end(stats, groups, T, r, zt[r], (int)threadIdx.x % kWave, kWave);
        if (h == 0) {
            loss_out[r] = p >= 0 ? end.loss : 0.0f;
            if (lse) lse[r] = p >= 0 ? end.lse : 0.0f;
        }
        cf = end.coef;
        uu = end.u;
    } else if (p >= 0) {
        cf = coef[p];
        uu = u[p];
    }
    if (h >= H) return;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (p >= 0) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(head) + block_at(t, h, row_blocks(Hp)));
        constexpr int kAhead = 4;
        for (int s = 0; s < splits; s += kAhead) {
            f32x4 at[kAhead][2];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const f32x4* from = reinterpret_cast<const f32x4*>(acc + ((int64_t)min(s + j, splits - 1) * rows + p) * Hp + h);
                at[j][0] = from[0];
                at[j][1] = from[1];
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (s + j >= splits) break;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += at[j][e >> 2][e & 3];
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = g * __builtin_fmaf(cf, v[e], -uu * ((e & 1) ? S::hi(w[e >> 1]) : S::lo(w[e >> 1])));
    }
    uint16_t* dst = dx + (int64_t)r * stride + h;
    if (VEC) {
        *reinterpret_cast<u32x4*>(dst) = u32x4{S::pack(v[0], v[1]), S::pack(v[2], v[3]), S::pack(v[4], v[5]), S::pack(v[6], v[7])};
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (h + e < H) dst[e] = S::enc(v[e]);
    }
}

// ---- plan ----
// Columns of a piece and of the first.  All of them while a_v takes 128 MB at most; without the gradient, while M and S of the waves take 256 MB (512 in
// groups of 64 columns).  Otherwise the first piece, all of whose a_v are read and written once more, has as many tiles of 256x256 as the chip has CUs, and the others a multiple
// of them (a launch of 880 takes four rounds as one of 1024 does: 7B's logits 951 us in such pieces, 850 so), with 256 MB (512, 1024) and about half of the
// vocabulary, but for the rounding to whole rounds, and 256 columns at least.
constexpr int64_t kRoomGrad = INT64_C(1) << 26, kRoomAlone = INT64_C(1) << 32;      // rows times columns of a single piece
static void ce_pieces(int64_t T, int64_t V, int64_t piece, bool grad, int& cols, int& first)
{
    const int64_t all = up(V, kPieceStep), room = grad ? kRoomGrad : kRoomAlone;
    if (piece || T <= room / all) {
        cols = first = (int)(piece && piece < all ? piece : all);
        return;
    }
    const int64_t tiles_m = (T + 255) / 256, round = (tiles_m >= 256 ? 1 : 256 / tiles_m) * 256;
    int64_t most = 2 * room / T;
    if (most > (V + 1) / 2) most = (V + 1) / 2;
    first = (int)(round < all ? round : all);
    cols = (int)(most > round ? up(most, round) : round);
    if (cols > all) cols = (int)all;
    if (!grad) first = cols;
}

// The logits' tile, by the time of its rounds of 256 workgroups (of 128x128 tiles a CU holds two): what a tile takes to start and for its epilogue, and its K
// tiles.  us, whole call without the gradient, 256x256 | 128x128, T x H -> V (a last round of few as halves): 128 x 4096 -> 32000 90 | 71, 200 rows 88 | 92,
// 333 112 | 120, 512 118 | 157, 2048 415 | 507, 711 x 5120 -> 32000 211 | 261, 333 x 1376 -> 100003 130 | 128, 1500 x 1024 -> 50000 172 | 158, 3000 x
// 512 -> 8000 55 | 45.  Tiles of 128x256 throughout were in front nowhere but where halves are them.
static int ce_tile(int64_t M, int64_t N, int64_t K)
{
    auto tiles = [&](int64_t bm, int64_t bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
    const double kt = (double)(K / 32);
    const int64_t halves = M % 256 > 0 && M % 256 <= 128 ? tiles(1 << 30, 256) : 0, t256 = tiles(256, 256) - halves, tail = t256 % 256;
    const int64_t t128 = tiles(128, 128), rest = t128 % 512;
    const double two = 1.5 + 0.55 * kt, one = 1.5 + 0.31 * kt;
    const double last = tail == 0 ? 0.0 : tail <= 128 ? 0.65 : 1.0;
    double rounds = (double)(t256 / 256) + last;
    if (halves) rounds = fmax(t256 ? 1.0 : 0.65, ((double)t256 + 0.65 * (double)halves) / 256.0 + 0.2);
    const double c0 = rounds * (8.5 + 0.77 * kt);
    const double c2 = (double)(t128 / 512) * two + (rest == 0 ? 0.0 : rest <= 256 ? one : two);
    return c0 <= c2 ? 0 : 2;
}
// The gradient's tile: its contraction is cut until the chip is full, so what counts is the part of a tile that is used, with 0.65 of a tile for a half where
// rows are of 2048 and more and the piece has more than 8192 columns.  In short rows parts of 256x256 tiles are many, and their sums cost what the halves save; of
// short pieces there are too few parts to fill the chip with such tiles.  us, whole call, 128x128 | 256x256 and halves, T x H -> V: 333 x 1376 -> 100003 289 | 291,
// 300 x 1000 -> 60000 163 | 169, 350 x 2048 -> 100003 389 | 377, 384 x 4096 -> 20000 184 | 179; 300 x 4096 -> 1000 55 | 70, -> 2000 62 | 73, -> 4000 68 | 78,
// -> 8000 97 | 102.
int ce_grad_tile(int64_t M, int64_t N, int64_t columns)
{
    const int64_t rest = M % 256;
    const double rows = (double)(M / 256) + (rest == 0 ? 0.0 : rest <= 128 && N >= 2048 && columns > 8192 ? 0.65 : 1.0);
    const double used256 = (double)(M * N) / (rows * 256.0 * (double)up(N, 256)), used128 = (double)(M * N) / (double)(up(M, 128) * up(N, 128));
    return 0.8 * used128 > used256 ? 2 : 0;
}

// Whether the kernels of few rows do the call: up to 64 rows, and where all of it is so small that it is launches that count (four in place of six, and none of
// their workgroups waits for another's), 64 rows a workgroup.  us, whole call with the gradient, tiles | these, T x H -> V: 100 x 100 -> 600 33.0 | 21.4, 1000 x 512
// -> 1000 50 | 24, 500 x 512 -> 4000 51 | 40, 500 x 4096 -> 500 70 | 44, 200 x 1024 -> 4000 52 | 37; but 300 x 4096 -> 1000 56 | 61, 100 x 512 -> 16000 45 | 50,
// 512 x 128 -> 8000 39.4 | 40.3; rows that are not whole 16 bytes, 400 x 300 -> 700 34.8 | 29.1 but 700 x 700 -> 2000 54 | 62.
static bool ce_few(const CeArgs& c)
{
    if (c.piece < c.V) return false;
    if (c.T <= kFewRows) return true;
    return c.T <= kFewMost && c.V <= 8192 && up(c.T, kFewRows) / kFewRows * (c.Vp / kFewCols) <= 512 && c.T * c.V * c.H <= (c.H % 8 ? INT64_C(1) << 27 : INT64_C(1) << 30);
}

// Columns of a workgroup of few rows' logits: fewer where 64 would leave CUs without one, and where a row or four cost nothing beside the head; each workgroup
// reads all of x, so more rows want more columns.  us, whole call without the gradient, 64 | 32 | 16 columns, T x H -> V: 1 x 4096 -> 2000 17.3 | 13.4 | 12.4,
// -> 8000 20.8 | 17.7 | 18.2, -> 32000 51.2 | 47.0 | 45.5 (with the gradient 97 | 93 | 96); 16 x 4096 -> 2000 20.5 | 16.6 | 14.8, -> 8000 23.5 | 19.3 | 22.0,
// -> 32000 52.3 | 54.5 | 64.6; 64 x 4096 -> 2000 36.1 | 31.4 | 29.5, -> 8000 38.1 | 33.0 | 47.5, -> 32000 72 | 95 | 154; 1 x 1024 -> 128000 45.3 | 49.8 | 52.2.
static int ce_few_cols(const CeArgs& c)
{
    if (c.H < 2048) return kFewCols;
    if (c.Vp / 16 <= 256) return 16;
    if (c.Vp / 32 <= 256) return 32;
    return c.T <= 4 && c.H >= 4096 ? c.grad ? 32 : 16 : kFewCols;
}
static int ce_few_groups(const CeArgs& c) { return c.Vp / c.few_cols; }

// Sizes of the parts that do not simply grow with the number of rows: for T rows what any number up to T needs, so that a program may size its workspace for its
// longest batch.  Each is a bound that grows with T, over both kinds of kernels and of tiles.
struct CeRoom { int64_t rows, a, stats, sums; };                    // rows staged, bytes of a_v, number of M and S, rows of running sums
static CeRoom ce_room(const CeArgs& c, int64_t piece)
{
    const int64_t T = c.T, all = piece && piece < up(c.V, kPieceStep) ? piece : up(c.V, kPieceStep), room = c.grad ? kRoomGrad : kRoomAlone;
    CeRoom r;
    r.rows = T > 32 ? up(T, 64) : up(T, 16);
    int64_t cells = T * all;
    r.a = r.rows * row_blocks(all) * 64;
    if (!piece) {
        // ce_pieces: one piece of T * cols <= room, or T * cols <= 2 room + T * round, where T * round is 2^16 a tile's rows or 256 T at most; T > room / all there.
        // a_v has up to 63 rows more (15 in several pieces), and a block a row of blocks.
        const int64_t rounds = 256 * (T + 63) > (INT64_C(5) << 22) ? 256 * (T + 63) : INT64_C(5) << 22, most = 4 * room + 128 * all + 2 * rounds + 64 * (T + 63);
        if (r.a > most) r.a = most;
        if (cells > 2 * room + rounds) cells = 2 * room + rounds;
    }
    r.stats = (cells + 63) / 64;
    if (c.piece >= c.V) {
        CeArgs few = c;
        auto groups = [&](int64_t rows) { few.T = rows; return (int64_t)(c.Vp / ce_few_cols(few)); };
        const int64_t to = c.V <= 8192 ? kFewMost : kFewRows, four = groups(4) * (T < 4 ? T : 4), more = groups(kFewRows) * (T < to ? T : to);
        if (r.stats < four) r.stats = four;
        if (r.stats < more) r.stats = more;
    }
    // one part of all, or as many parts as there are slots for
    r.sums = 64 * (512 / (c.Hp / 64));
    for (const int tile : {0, 2}) {
        const int64_t filled = (tile == 2 ? 512 : 256) / ((c.H + tile_cols(tile) - 1) / tile_cols(tile)) * tile_rows(tile);
        if (r.sums < filled) r.sums = filled;
    }
    const int64_t splits = all / 512 > 1 ? all / 512 : 1;
    if (r.sums > T * splits) r.sums = T * splits;
    if (r.sums < T) r.sums = T;
    return r;
}

// Sizes and the workspace's parts, from `base` (0: only how long they are).
static size_t ce_plan(CeArgs& c, int64_t piece, char* base)
{
    c.Hp = (int)up(c.H, 64);
    c.Vp = (int)up(c.V, 64);
    ce_pieces(c.T, c.V, piece, c.grad, c.piece, c.first_piece);
    c.few_parts = 0;
    c.few_own_join = false;
    c.few_cols = kFewCols;
    if (ce_few(c)) {
        // as many workgroups as fill the chip twice, of 64 columns a wave at least
        int64_t parts = 512 / ((c.Hp + kFewCols - 1) / kFewCols * ((c.T + kFewRows - 1) / kFewRows));
        if (parts > c.Vp / 512) parts = c.Vp / 512;
        c.few_parts = (int)(parts < 1 ? 1 : parts);
        c.few_cols = ce_few_cols(c);
        c.few_own_join = c.grad && c.T <= kFewRows && c.T * ce_few_groups(c) <= kFewOwnJoin;
    }
    c.tile = ce_tile(c.T, c.piece, c.Hp);
    c.grad_tile = ce_grad_tile(c.T, c.H, c.piece);
    c.slots = c.grad_tile == 2 ? 512 : 256;
    c.max_splits = c.piece / 512 > 1 ? c.piece / 512 : 1;
    const CeRoom room = ce_room(c, piece);
    size_t at = kWsHeaderBytes;                                        // the tickets of other calls on this workspace stay as they are
    auto part = [&](auto*& p, size_t bytes) {
        p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(base + at);
        at += (bytes + 255) / 256 * 256;
    };
    const size_t T = (size_t)c.T;
    part(c.count, 4);
    part(c.ticket, 4);
    part(c.pos, T * 4);
    part(c.row, T * 4);
    part(c.tgt, T * 4);
    part(c.zt, T * 4);
    part(c.run, T * 8);
    part(c.beta, T * 4);
    part(c.coef, T * 4);
    part(c.u, T * 4);
    part(c.part, (T + 3) / 4 * 8);
    part(c.stats, (size_t)room.stats * 8);
    part(c.xs, (size_t)room.rows * row_blocks(c.Hp) * 64);
    if (c.grad) {
        part(c.scale_rows, (T + 3) / 4);
        part(c.a, (size_t)room.a);
        part(c.acc, (size_t)room.sums * (size_t)c.Hp * 4);
    }
    return at;
}

static bool ce_sizes_ok(int64_t T, int64_t V, int64_t H, int64_t piece)
{
    return T > 0 && V > 0 && H > 0 && T <= kCeMaxTokens && V <= kCeMaxVocab && H <= kCeMaxHidden && up(H, 64) <= kCeMaxProduct / T &&
           up(H, 64) <= kCeMaxProduct / V && piece >= 0 && piece % kPieceStep == 0 && (piece < V ? piece : V) <= kCeMaxProduct / T;
}

template <int DT>
static void launch_dx(const CeArgs& c, hipStream_t st)
{
    const int T = (int)c.T, H = (int)c.H, chunks = (H + kDxCols - 1) / kDxCols, bm = tile_rows(c.grad_tile), tiles_n = (int)((c.H + tile_cols(c.grad_tile) - 1) / tile_cols(c.grad_tile));
    const bool vec = c.dx_stride % 8 == 0 && H % 8 == 0;
    auto go = [&](auto v, auto join) {
        ce_dx_kernel<DT, decltype(v)::value, decltype(join)::value><<<dim3(T + (c.mean ? 1 : 0), chunks), 256, 0, st>>>(
            c.acc, bm, tiles_n, c.slots, c.max_splits, c.few_parts, c.count, c.pos, c.few_parts ? c.targets : c.tgt, c.coef, c.u, c.head, c.row_weight, c.scale,
            static_cast<uint16_t*>(c.dx), c.dx_stride, H, c.Hp, c.loss, c.mean, T, (int)c.V, c.stats, ce_few_groups(c), c.zt, c.loss, c.lse);
    };
    auto by_join = [&](auto v) {
        if (c.few_own_join) go(v, std::true_type{});
        else                go(v, std::false_type{});
    };
    if (vec) by_join(std::true_type{});
    else     by_join(std::false_type{});
}

static int join_rows(int groups) { return groups > kJoinManyGroups ? 4 : 16; }

static void launch_join(const CeArgs& c, int groups, bool first, bool last, hipStream_t st)
{
    auto go = [&](auto rows) {
        constexpr int ROWS = decltype(rows)::value;
        ce_join_kernel<ROWS><<<(unsigned)((c.T + ROWS - 1) / ROWS), kJoinThreads, 0, st>>>(
            c.stats, groups, c.T, c.count, c.run, c.beta, c.grad && !c.few_parts ? c.scale_rows : nullptr, c.zt, c.few_parts ? nullptr : c.row, c.coef, c.u, c.loss,
            c.lse, c.grad ? nullptr : c.mean, c.part, c.ticket, c.few_parts ? c.targets : nullptr, (int)c.V, first, last);
    };
    if (join_rows(groups) == 4) go(std::integral_constant<int, 4>{});
    else                        go(std::integral_constant<int, 16>{});
}

template <int DT>
static void ce_run(const CeArgs& c, sasq_dtype dt, hipStream_t st)
{
    const int T = (int)c.T, H = (int)c.H;
    if (c.few_parts) {
        launch_ce_few_logits(c, dt, st);
        if (!c.few_own_join) launch_join(c, ce_few_groups(c), true, true, st);
        if (c.grad) {
            launch_ce_few_grad(c, dt, st);
            launch_dx<DT>(c, st);
        }
        return;
    }
    auto stage = [&](auto v) {
        constexpr bool VEC = decltype(v)::value;
        const auto x = static_cast<const uint16_t*>(c.x);
        if (T <= kPackedTo) {
            ce_pack_stage_kernel<VEC><<<(T + 3) / 4, 256, 0, st>>>(x, c.x_stride, c.xs, c.targets, T, (int)c.V, c.count, c.pos, c.row, c.tgt, c.loss, c.lse, c.ticket,
                                                                   c.mean, H, c.Hp);
            return;
        }
        ce_pack_kernel<<<1, kPackThreads, 0, st>>>(c.targets, T, (int)c.V, c.count, c.pos, c.row, c.tgt, c.loss, c.lse, c.ticket, c.mean);
        ce_stage_kernel<VEC><<<(T + 3) / 4, 256, 0, st>>>(x, c.x_stride, c.xs, c.count, c.row, H, c.Hp);
    };
    if (c.x_stride % 8 == 0 && H % 8 == 0) stage(std::true_type{});
    else                                   stage(std::false_type{});
    const int sc = stat_cols(c.tile), bn = 2 * sc;
    for (int64_t col0 = 0; col0 < c.V;) {
        const int64_t piece = col0 ? c.piece : c.first_piece, cols = c.V - col0 < piece ? c.V - col0 : piece;
        const int groups = (int)((cols + bn - 1) / bn) * 2;
        launch_ce_logits(c, dt, col0, cols, st);
        launch_join(c, groups, col0 == 0, col0 + cols >= c.V, st);
        if (c.grad) {
            const int kt = (int)(up(cols, 64) / 32);
            const int rows16 = (T + 15) / 16, each = col0 ? 64 : 16;          // (of later pieces few rows have any: larger workgroups leave sooner)
            ce_scale_kernel<DT><<<dim3(rows16, (kt + each - 1) / each), 256, 0, st>>>(c.a, row_blocks(c.piece), kt, sc / 32, c.stats, c.run, c.scale_rows,
                                                                                      16 / join_rows(groups), c.T, c.count, each);
            launch_ce_grad(c, dt, col0, cols, st);
        }
        col0 += cols;
    }
    if (c.grad) launch_dx<DT>(c, st);
}

}  // namespace sasq

using namespace sasq;

extern "C" size_t sasq_head_bytes(int64_t V, int64_t H, sasq_head_form form)
{
    if (V <= 0 || H <= 0 || V > kCeMaxVocab || H > kCeMaxHidden || up(H, 64) > kCeMaxProduct / V) return 0;
    if (form == SASQ_HEAD_LOGITS) return (size_t)up(V, 16) * row_blocks(up(H, 64)) * 64;
    if (form == SASQ_HEAD_GRAD) return (size_t)up(H, 16) * row_blocks(up(V, 64)) * 64;
    return 0;
}

extern "C" int sasq_prepare_head(const void* w, int64_t w_stride, void* head, int64_t V, int64_t H, sasq_head_form form, sasq_dtype dt, void* stream)
{
    if (!w || !head) return SASQ_ERR_NULL;
    if (form != SASQ_HEAD_LOGITS && form != SASQ_HEAD_GRAD) return SASQ_ERR_UNSUPPORTED;
    if (dt != SASQ_F16 && dt != SASQ_BF16) return SASQ_ERR_UNSUPPORTED;
    if (sasq_head_bytes(V, H, form) == 0 || w_stride < H) return SASQ_ERR_SHAPE;
    if (!aligned16(w) || !aligned16(head)) return SASQ_ERR_ALIGN;
    hipStream_t st = as_stream(stream);
    auto W = static_cast<const uint16_t*>(w);
    auto O = static_cast<u32x4*>(head);
    const bool vec = w_stride % 8 == 0;
    if (form == SASQ_HEAD_LOGITS) {
        const int64_t kt = row_blocks(up(H, 64)), chunks = up(V, 16) / 16 * kt * 64, blocks = (chunks + 255) / 256;
        head_logits_kernel<<<(int)(blocks < 8192 ? blocks : 8192), 256, 0, st>>>(W, w_stride, O, V, H, kt, chunks, vec);
    } else {
        const int64_t tiles = up(V, 64) / 64 * (up(H, 64) / 64);
        head_grad_kernel<<<(int)(tiles < 8192 ? tiles : 8192), 256, 0, st>>>(W, w_stride, O, V, H, up(H, 16) / 16, row_blocks(up(V, 64)), tiles, vec);
    }
    return hipGetLastError() == hipSuccess ? SASQ_OK : SASQ_ERR_LAUNCH;
}

extern "C" size_t sasq_linear_ce_workspace(int64_t T, int64_t V, int64_t H, int grad, int64_t piece)
{
    if (!ce_sizes_ok(T, V, H, piece)) return 0;
    CeArgs c{};
    c.T = T; c.V = V; c.H = H; c.grad = grad != 0;
    return ce_plan(c, piece, nullptr);
}

extern "C" int sasq_linear_ce(const void* x, int64_t x_stride, const void* head, const void* head_grad, const int32_t* targets,
                              const float* row_weight, float scale, float* loss, float* lse, float* mean, void* dx, int64_t dx_stride,
                              int64_t T, int64_t V, int64_t H, int64_t piece, sasq_dtype dt, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!x || !head || !targets || !loss || (dx && !head_grad)) return SASQ_ERR_NULL;
    if (!ce_sizes_ok(T, V, H, piece) || x_stride < H || (dx && dx_stride < H)) return SASQ_ERR_SHAPE;
    if (dt != SASQ_F16 && dt != SASQ_BF16) return SASQ_ERR_UNSUPPORTED;
    if (!aligned16(x) || !aligned16(head) || (dx && (!aligned16(dx) || !aligned16(head_grad)))) return SASQ_ERR_ALIGN;
    if (!workspace || workspace_bytes < sasq_linear_ce_workspace(T, V, H, dx != nullptr, piece)) return SASQ_ERR_WORKSPACE;
    if (!aligned16(workspace)) return SASQ_ERR_ALIGN;
    CeArgs c{};
    c.T = T; c.V = V; c.H = H; c.grad = dx != nullptr;
    c.x = x; c.x_stride = x_stride;
    c.head = static_cast<const uint8_t*>(head); c.head_grad = static_cast<const uint8_t*>(head_grad);
    c.targets = targets; c.row_weight = row_weight; c.scale = scale;
    c.loss = loss; c.lse = lse; c.mean = mean;
    c.dx = dx; c.dx_stride = dx_stride;
    ce_plan(c, piece, static_cast<char*>(workspace));
    hipStream_t st = as_stream(stream);
    if (dt == SASQ_F16) ce_run<SASQ_F16>(c, dt, st);
    else                ce_run<SASQ_BF16>(c, dt, st);
    return hipGetLastError() == hipSuccess ? SASQ_OK : SASQ_ERR_LAUNCH;
}
