// Fake quantization that keeps one byte an element for its backward, in place of the 16-bit x (sasq_fakequant_*_ckpt).
//
// The backward (Sec. 4.2, Eq. 4 and the chain rule) needs of x only whether it was clamped, and to which end, or else the rounding residual:
//     dx = dy * m,   ds = sum dy * (m ? e : q),   e = q - x/s in [-1/2, 1/2]
// The byte c is that residual in units of 1/252, or a mark: 127 above the range, -128 below it.  e is one fused product and difference (exact but for
// its rounding to fp32), c the nearest whole number of the exact 252 e.  ds then is sum dy * t / 252 with t = c, or 252 q at the ends.  The product of a 16-bit
// dy and t (7 bits, 13 at the ends) is exact in fp32; bf16 has fp32's exponents, and there t goes by 2^-18, so that neither a product nor the sum of four
// passes fp32 (what falls below its normal numbers loses 2^-139 of ds at most).  x itself in 8 bits would not do, as the residual is what 8 bits of x leave out.
//
// Bound by memory: forward x in, y and the byte out, 5 bytes an element; backward the byte and dy in, dx out, 5 bytes, where the form that keeps x has 6.
#include "sasq_device.h"
#include <type_traits>

namespace sasq {

constexpr int kCkThreads = 256, kCkWaves = kCkThreads / kWave, kCkUnroll = 4;
constexpr float kCkSteps = 252.0f;
template <int DT> constexpr float kCkUnit = DT == SASQ_BF16 ? 0x1p-18f : 1.0f;       // terms of ds are kCkSteps * kCkUnit times as large
constexpr int kCkHigh = 127, kCkLow = -128;
constexpr int kCkCols = kWave * 8;               // columns of a block of the per-channel kernels
constexpr int kCkMaxBatch = SASQ_MAX_BATCH;
constexpr int kCkBlocks = 2048;                  // eight workgroups a CU
constexpr int kCkSmallThreads = 1024, kCkSmallUnroll = 3;
constexpr int64_t kCkSmall = (int64_t)kCkSmallThreads * kCkSmallUnroll * 8;

struct CkItem {
    const uint16_t* x;
    const float* s;
    uint16_t* out;
    int8_t* kept;
    const uint16_t* dy;
    float* ds;
    void* partial;                                // backward: of this tensor
    int64_t rows, cols, n;
    int64_t chunk_rows;                           // per channel: rows of a block,
    int chunks;                                   // and blocks of a column block
};
struct CkBatch {
    CkItem it[kCkMaxBatch];
    int first[kCkMaxBatch + 1];
    int count;
};

__device__ __forceinline__ int ck_item_of(const CkBatch& b, int block)
{
    int k = 0;
#pragma unroll
    for (int i = 1; i < kCkMaxBatch; ++i)
        if (i < b.count && block >= b.first[i]) k = i;
    return k;
}

// q * s and the byte, in the low bits of a float as pack_codes4 wants it.
__device__ __forceinline__ float ck_fwd(float x, float inv_s, float s, float lo, float hi, float& byte)
{
    const float f = __builtin_fmaf(x, inv_s, kMagic);
    const float c = __builtin_amdgcn_fmed3f(f, lo, hi);
    const float q = c - kMagic;
    const float e = __builtin_fmaf(-x, inv_s, q);
    byte = __builtin_fmaf(e, kCkSteps, kMagic);
    byte = f > c ? kMagic + (float)kCkHigh : byte;
    byte = f < c ? kMagic + (float)kCkLow : byte;
    return rounded_f32(q * s);                    // elements stored one by one would be multiplied and converted at once
}

template <int DT>
__device__ __forceinline__ u32x4 ck_fwd_vec(const u32x4& in, const float (&inv_s)[8], const float (&s)[8], float lo, float hi, u32x2& kept)
{
    using S = Store16<DT>;
    u32x4 out;
    float b[8];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float y0 = ck_fwd(S::lo(in[w]), inv_s[2 * w], s[2 * w], lo, hi, b[2 * w]);
        const float y1 = ck_fwd(S::hi(in[w]), inv_s[2 * w + 1], s[2 * w + 1], lo, hi, b[2 * w + 1]);
        out[w] = S::pack(y0, y1);
    }
    kept[0] = pack_codes4(b[0], b[1], b[2], b[3]);
    kept[1] = pack_codes4(b[4], b[5], b[6], b[7]);
    return out;
}

// 252 units times what the byte stands for; m: inside the range.
template <int DT>
__device__ __forceinline__ float ck_value(int c, float lo252, float hi252, bool& m)
{
    const bool high = c == kCkHigh, low = c == kCkLow;
    m = !high && !low;
    return high ? hi252 : low ? lo252 : (float)c * kCkUnit<DT>;
}

// dx and the eight terms of ds times 252 units.
template <int DT>
__device__ __forceinline__ u32x4 ck_bwd_vec(const u32x2& kept, const u32x4& g, float lo252, float hi252, float (&term)[8])
{
    using S = Store16<DT>;
    u32x4 out;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        bool ma, mb;
        const int c0 = (int)(kept[w >> 1] << (24 - 16 * (w & 1))) >> 24, c1 = (int)(kept[w >> 1] << (16 - 16 * (w & 1))) >> 24;
        term[2 * w] = S::lo(g[w]) * ck_value<DT>(c0, lo252, hi252, ma);
        term[2 * w + 1] = S::hi(g[w]) * ck_value<DT>(c1, lo252, hi252, mb);
        out[w] = g[w] & ((ma ? 0x0000FFFFu : 0u) | (mb ? 0xFFFF0000u : 0u));
    }
    return out;
}

__device__ __forceinline__ float ck_low(int bits) { return -(float)(1 << (bits - 1)); }
__device__ __forceinline__ float ck_high(int bits) { return (float)((1 << (bits - 1)) - 1); }

// ---- one factor per tensor: a flat array, eight elements a lane and access ----
// 2048 x 4096 four times (q, k, v share x): forward 22.0 us, 134 MB, 6.1 TB/s; backward 30.6 us, 168 MB, 5.5; a large copy 5.2.
template <int DT>
__global__ __launch_bounds__(kCkThreads) void ck_fwd_kernel(const CkBatch b, int bits)
{
    using S = Store16<DT>;
    const int k = ck_item_of(b, (int)blockIdx.x);
    const CkItem& it = b.it[k];
    const int64_t block = (int)blockIdx.x - b.first[k], blocks = b.first[k + 1] - b.first[k];
    const float f = *it.s, lo = kMagic + ck_low(bits), hi = kMagic + ck_high(bits);
    float s[8], inv_s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { s[e] = f; inv_s[e] = 1.0f / f; }
    const u32x4* x = reinterpret_cast<const u32x4*>(it.x);
    u32x4* y = reinterpret_cast<u32x4*>(it.out);
    u32x2* kept = reinterpret_cast<u32x2*>(it.kept);
    const int64_t nvec = it.n / 8;
    constexpr int64_t kChunk = (int64_t)kCkThreads * kCkUnroll;
    for (int64_t base = block * kChunk; base < nvec; base += blocks * kChunk) {
        u32x4 in[kCkUnroll];
#pragma unroll
        for (int u = 0; u < kCkUnroll; ++u) in[u] = x[min(base + u * kCkThreads + (int64_t)threadIdx.x, nvec - 1)];
#pragma unroll
        for (int u = 0; u < kCkUnroll; ++u) {
            const int64_t i = base + u * kCkThreads + threadIdx.x;
            u32x2 kp;
            const u32x4 out = ck_fwd_vec<DT>(in[u], inv_s, s, lo, hi, kp);
            if (i < nvec) {
                __builtin_nontemporal_store(out, &y[i]);
                __builtin_nontemporal_store(kp, &kept[i]);
            }
        }
    }
    if (block == blocks - 1 && threadIdx.x < (unsigned)(it.n - nvec * 8)) {
        const int64_t i = nvec * 8 + threadIdx.x;
        float byte;
        const float v = ck_fwd(S::one(it.x[i]), inv_s[0], f, lo, hi, byte);
        it.out[i] = S::enc(v);
        it.kept[i] = (int8_t)(__float_as_int(byte) - kMagicBits);
    }
}

// SMALL: a workgroup of 1024 threads takes a whole tensor, and its ds needs no join (64 x 256, with the forward, 23 -> 8.6 us, two launches).  The products are exact in fp32 and added in fp64: sums over many
// elements that nearly cancel keep their digits.
template <int DT, bool SMALL>
__global__ __launch_bounds__(SMALL ? kCkSmallThreads : kCkThreads) void ck_bwd_kernel(const CkBatch b, int bits)
{
    using S = Store16<DT>;
    constexpr int kThreads = SMALL ? kCkSmallThreads : kCkThreads, kWaves = kThreads / kWave, kUnroll = SMALL ? kCkSmallUnroll : kCkUnroll;
    const int k = SMALL ? (int)blockIdx.x : ck_item_of(b, (int)blockIdx.x);
    const CkItem& it = b.it[k];
    const int64_t block = SMALL ? 0 : (int)blockIdx.x - b.first[k], blocks = SMALL ? 1 : b.first[k + 1] - b.first[k];
    constexpr float kPer = kCkSteps * kCkUnit<DT>;
    const float lo = ck_low(bits) * kPer, hi = ck_high(bits) * kPer;
    const u32x2* kept = reinterpret_cast<const u32x2*>(it.kept);
    const u32x4* dy = reinterpret_cast<const u32x4*>(it.dy);
    u32x4* dx = reinterpret_cast<u32x4*>(it.out);
    const int64_t nvec = it.n / 8;
    constexpr int64_t kChunk = (int64_t)kThreads * kUnroll;
    double acc = 0.0;
    for (int64_t base = block * kChunk; base < nvec; base += blocks * kChunk) {
        u32x2 kp[kUnroll];
        u32x4 g[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t i = min(base + u * kThreads + (int64_t)threadIdx.x, nvec - 1);
            kp[u] = __builtin_nontemporal_load(&kept[i]);
            g[u] = __builtin_nontemporal_load(&dy[i]);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t i = base + u * kThreads + threadIdx.x;
            float term[8];
            double sum = 0.0;
            const u32x4 out = ck_bwd_vec<DT>(kp[u], g[u], lo, hi, term);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += (double)term[e];
            if (i < nvec) {
                acc += sum;
                if (dx) __builtin_nontemporal_store(out, &dx[i]);
            }
        }
    }
    if (block == blocks - 1 && threadIdx.x < (unsigned)(it.n - nvec * 8)) {
        const int64_t i = nvec * 8 + threadIdx.x;
        bool m;
        const uint16_t g = it.dy[i];
        acc += (double)(S::one(g) * ck_value<DT>(it.kept[i], lo, hi, m));
        if (dx) it.out[i] = m ? g : (uint16_t)0;
    }
    __shared__ double part[kWaves];
    const double w = wave_sum(acc);
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = w;
    __syncthreads();
    if (threadIdx.x < kWave) {
        const double all = wave_sum(threadIdx.x < kWaves ? part[threadIdx.x] : 0.0);
        if (threadIdx.x == 0) {
            if (blocks == 1) *it.ds = (float)(all / (double)kPer);
            else             static_cast<double*>(it.partial)[block] = all;
        }
    }
}

// ds of a tensor from its blocks' sums, in a fixed order.
template <int DT>
__global__ __launch_bounds__(kCkThreads) void ck_join_kernel(const CkBatch b)
{
    const CkItem& it = b.it[blockIdx.x];
    const int n = b.first[blockIdx.x + 1] - b.first[blockIdx.x];
    if (n == 1) return;
    const double* p = static_cast<const double*>(it.partial);
    double acc = 0.0;
    for (int i = threadIdx.x; i < n; i += kCkThreads) acc += p[i];
    __shared__ double part[kCkWaves];
    const double w = wave_sum(acc);
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = w;
    __syncthreads();
    if (threadIdx.x == 0) {
        double all = 0.0;
        for (int i = 0; i < kCkWaves; ++i) all += part[i];
        *it.ds = (float)(all / (double)(kCkSteps * kCkUnit<DT>));
    }
}

// ---- one factor per column ----
// Bytes: a 13B layer's seven, forward 56.7 us, 343 MB, 6.1 TB/s, backward 75.5 us, 404 MB, 5.4.  Blocks next to each other take columns next to each other (rows
// below each other 153 us for both, so 149), and what the backward reads, once, passes the caches by (145).
// A block takes 512 columns of a run of rows, each of its waves every fourth of them.  VEC: a lane has eight columns next to each other and a row's
// elements in one access; otherwise (rows that are no multiple of eight) every 64th column, an access of 2 bytes or 1 each: 4096 x 4097 forward 44 us, backward 26,
// where 4104 columns take 21 and 25 (4096 15 and 21), 1777 x 13825 45 and 32 where 13824 take 22 and 26.
template <bool VEC>
__device__ __forceinline__ int64_t ck_col(int64_t col_block, int lane, int e) { return col_block * kCkCols + (VEC ? lane * 8 + e : e * kWave + lane); }

template <int DT, bool VEC, bool ONCE>
__device__ __forceinline__ u32x4 ck_load_row(const uint16_t* at, int64_t col_block, int lane, int64_t cols)
{
    if (VEC) {
        const auto from = reinterpret_cast<const u32x4*>(at + ck_col<VEC>(col_block, lane, 0));
        return ONCE ? __builtin_nontemporal_load(from) : *from;
    }
    u32x4 v;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int64_t c0 = ck_col<VEC>(col_block, lane, 2 * w), c1 = ck_col<VEC>(col_block, lane, 2 * w + 1);
        v[w] = (uint32_t)at[min(c0, cols - 1)] | (uint32_t)at[min(c1, cols - 1)] << 16;
    }
    return v;
}
template <bool VEC>
__device__ __forceinline__ u32x2 ck_load_kept(const int8_t* at, int64_t col_block, int lane, int64_t cols)
{
    if (VEC) return __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(at + ck_col<VEC>(col_block, lane, 0)));
    u32x2 v = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e >> 2] |= (uint32_t)(uint8_t)at[min(ck_col<VEC>(col_block, lane, e), cols - 1)] << (8 * (e & 3));
    return v;
}
template <bool VEC>
__device__ __forceinline__ void ck_store_row(uint16_t* at, const u32x4& v, int64_t col_block, int lane, int64_t cols)
{
    if (VEC) {
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(at + ck_col<VEC>(col_block, lane, 0)));
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (ck_col<VEC>(col_block, lane, e) < cols) at[ck_col<VEC>(col_block, lane, e)] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
}
template <bool VEC>
__device__ __forceinline__ void ck_store_kept(int8_t* at, const u32x2& v, int64_t col_block, int lane, int64_t cols)
{
    if (VEC) {
        __builtin_nontemporal_store(v, reinterpret_cast<u32x2*>(at + ck_col<VEC>(col_block, lane, 0)));
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (ck_col<VEC>(col_block, lane, e) < cols) at[ck_col<VEC>(col_block, lane, e)] = (int8_t)(v[e >> 2] >> (8 * (e & 3)));
}

template <int DT, bool VEC>
__device__ __forceinline__ void ck_fwd_pc_body(const CkItem& it, int block, int bits)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t cols = it.cols, across = (cols + kCkCols - 1) / kCkCols, cb = block % across, chunk = block / across;
    const int64_t r0 = chunk * it.chunk_rows, r1 = min(it.rows, r0 + it.chunk_rows);
    if (VEC && ck_col<VEC>(cb, lane, 0) >= cols) return;
    const float lo = kMagic + ck_low(bits), hi = kMagic + ck_high(bits);
    u32x4 in[2][kCkUnroll];
    auto fetch = [&](int set, int64_t base) {
#pragma unroll
        for (int u = 0; u < kCkUnroll; ++u) in[set][u] = ck_load_row<DT, VEC, false>(it.x + min(base + u * kCkWaves, r1 - 1) * cols, cb, lane, cols);
    };
    fetch(0, r0 + wave);
    float s[8], inv_s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        s[e] = it.s[min(ck_col<VEC>(cb, lane, e), cols - 1)];
        inv_s[e] = 1.0f / s[e];
    }
    auto rows = [&](int set, int64_t base) {
#pragma unroll
        for (int u = 0; u < kCkUnroll; ++u) {
            const int64_t r = base + u * kCkWaves;
            if (r >= r1) break;
            u32x2 kp;
            const u32x4 out = ck_fwd_vec<DT>(in[set][u], inv_s, s, lo, hi, kp);
            ck_store_row<VEC>(it.out + r * cols, out, cb, lane, cols);
            ck_store_kept<VEC>(it.kept + r * cols, kp, cb, lane, cols);
        }
    };
    constexpr int kStep = kCkWaves * kCkUnroll;
    for (int64_t base = r0 + wave; base < r1; base += 2 * kStep) {
        if (base + kStep < r1) fetch(1, base + kStep);
        rows(0, base);
        if (base + 2 * kStep < r1) fetch(0, base + 2 * kStep);
        if (base + kStep < r1) rows(1, base + kStep);
    }
}

// ANY: some tensor of the launch has rows that are no multiple of eight (a kernel with both bodies needs more registers).
template <int DT, bool ANY>
__global__ __launch_bounds__(kCkThreads) void ck_fwd_pc_kernel(const CkBatch b, int bits)
{
    const int k = ck_item_of(b, (int)blockIdx.x);
    const CkItem& it = b.it[k];
    const int block = (int)blockIdx.x - b.first[k];
    if (!ANY || it.cols % 8 == 0) ck_fwd_pc_body<DT, true>(it, block, bits);
    else                          ck_fwd_pc_body<DT, false>(it, block, bits);
}

template <int DT, bool VEC>
__device__ __forceinline__ void ck_bwd_pc_body(const CkItem& it, int block, int bits, float (&red)[kCkWaves][kCkCols])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t cols = it.cols, across = (cols + kCkCols - 1) / kCkCols, cb = block % across, chunk = block / across;
    const int64_t r0 = chunk * it.chunk_rows, r1 = min(it.rows, r0 + it.chunk_rows);
    constexpr float kPer = kCkSteps * kCkUnit<DT>;
    const float lo = ck_low(bits) * kPer, hi = ck_high(bits) * kPer;
    double acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};      // four rows in fp32; a wave's sum and a block's are rounded to fp32 on their way, all else is added in fp64
    if (!VEC || ck_col<VEC>(cb, lane, 0) < cols) {
        for (int64_t base = r0 + wave; base < r1; base += kCkWaves * kCkUnroll) {
            u32x2 kp[kCkUnroll];
            u32x4 g[kCkUnroll];
#pragma unroll
            for (int u = 0; u < kCkUnroll; ++u) {
                const int64_t at = min(base + u * kCkWaves, r1 - 1) * cols;
                kp[u] = ck_load_kept<VEC>(it.kept + at, cb, lane, cols);
                g[u] = ck_load_row<DT, VEC, true>(it.dy + at, cb, lane, cols);
            }
            float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int u = 0; u < kCkUnroll; ++u) {
                const int64_t r = base + u * kCkWaves;
                float term[8];
                const u32x4 out = ck_bwd_vec<DT>(kp[u], g[u], lo, hi, term);
                if (r >= r1) break;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += term[e];
                if (it.out) ck_store_row<VEC>(it.out + r * cols, out, cb, lane, cols);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] += (double)sum[e];
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) red[wave][ck_col<VEC>(0, lane, e)] = (float)acc[e];
    __syncthreads();
    for (int c = threadIdx.x; c < kCkCols; c += kCkThreads) {
        if (cb * kCkCols + c >= cols) continue;
        double all = 0.0;
#pragma unroll
        for (int w = 0; w < kCkWaves; ++w) all += (double)red[w][c];
        if (it.chunks == 1) it.ds[cb * kCkCols + c] = (float)(all / (double)kPer);
        else                static_cast<float*>(it.partial)[chunk * cols + cb * kCkCols + c] = (float)all;
    }
}

template <int DT, bool ANY>
__global__ __launch_bounds__(kCkThreads) void ck_bwd_pc_kernel(const CkBatch b, int bits)
{
    __shared__ float red[kCkWaves][kCkCols];
    const int k = ck_item_of(b, (int)blockIdx.x);
    const CkItem& it = b.it[k];
    const int block = (int)blockIdx.x - b.first[k];
    if (!ANY || it.cols % 8 == 0) ck_bwd_pc_body<DT, true>(it, block, bits, red);
    else                          ck_bwd_pc_body<DT, false>(it, block, bits, red);
}

// 64 columns a workgroup, a quarter of the row blocks a wave, eight loads in flight; the order of the sum follows from the sizes.
constexpr int kCkJoinAhead = 8;
template <int DT>
__global__ __launch_bounds__(kCkThreads) void ck_join_pc_kernel(const CkBatch b)
{
    __shared__ double part[kCkWaves][kWave];
    const CkItem& it = b.it[blockIdx.y];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * kWave + lane;
    if (it.chunks == 1 || (int64_t)blockIdx.x * kWave >= it.cols) return;
    const float* p = static_cast<const float*>(it.partial) + min(c, it.cols - 1);
    double all = 0.0;
    for (int i0 = wave; i0 < it.chunks; i0 += kCkWaves * kCkJoinAhead) {
        float v[kCkJoinAhead];
#pragma unroll
        for (int j = 0; j < kCkJoinAhead; ++j) v[j] = p[min(i0 + j * kCkWaves, it.chunks - 1) * it.cols];
#pragma unroll
        for (int j = 0; j < kCkJoinAhead; ++j) all += i0 + j * kCkWaves < it.chunks ? (double)v[j] : 0.0;
    }
    part[wave][lane] = all;
    __syncthreads();
    if (wave || c >= it.cols) return;
    all = 0.0;
#pragma unroll
    for (int w = 0; w < kCkWaves; ++w) all += part[w][lane];
    it.ds[c] = (float)(all / (double)(kCkSteps * kCkUnit<DT>));
}

// ---- plan ----
static int ck_blocks(int64_t n, int most)
{
    const int64_t need = (n / 8 + (int64_t)kCkThreads * kCkUnroll - 1) / ((int64_t)kCkThreads * kCkUnroll);
    return (int)(need < 1 ? 1 : need < most ? need : most);
}
static int64_t ck_col_blocks(int64_t cols) { return (cols + kCkCols - 1) / kCkCols; }
// Rows of a block: they follow from the tensor alone, so that a batch gives the bits of the single calls.
static int64_t ck_chunk_rows(int64_t rows, int64_t cols)
{
    if (rows <= 64) return 64;                      // one block of all: no join
    int64_t r = 16;
    while (r < 64 && (rows + 2 * r - 1) / (2 * r) * ck_col_blocks(cols) >= 512) r *= 2;
    while ((rows + r - 1) / r > 256) r *= 2;
    return r;
}
// Most row blocks of a tensor of at most so many rows and any columns: ck_chunk_rows has 16 rows in a block at least, and 256 blocks at most.
static int64_t ck_most_chunks(int64_t rows)
{
    if (rows <= 64) return 1;
    const int64_t n = (rows + 15) / 16;
    return n < 256 ? n : 256;
}
constexpr int64_t kCkMaxElements = INT64_C(1) << 40, kCkMaxCols = INT64_C(1) << 24;
constexpr int64_t kCkMaxBlocks = INT64_C(1) << 23;       // a launch holds fewer than 2^32 threads

// Workgroups of a tensor in the backward, a power of two, by the number of tensors (what a small one does not fill it does not launch): one of 8192 x 8192 66.8 us
// with 512, 63.3 with 2048; three of an 8192-row 70B MLP 327 with 512 each, 344 with 682, 337 with 1024, 370 with 256.  Of others the choice is within 3 % of the best:
// 512 | 1024 | 2048 for two of 8192 x 8192 117.0 | 118.3 | 117.6, two of 2048 x 4096 18.5 | 19.0 | 18.8; 256 | 512 | 1024 for four of 2048 x 4096 33.0 | 31.7 | 32.1,
// five 39.6 | 40.2 | 38.8, seven 53.9 | 53.6 | 52.0, eight 60.0 | 59.1 | 58.5.
static int ck_partials(int count) { return count == 1 ? 2048 : count == 2 ? 1024 : 512; }
// What a tensor's partial sums take; in a batch of so many.  A workspace serves fewer tensors, rows and columns too.
static size_t ck_partial_bytes(int64_t rows, int64_t cols, bool pc, int count)
{
    if (!pc) return (size_t)ck_partials(count) * sizeof(double);
    return ((size_t)(ck_most_chunks(rows) * cols) * sizeof(float) + 255) / 256 * 256;
}

static int ck_check(const sasq_ckpt_item* items, int count, bool pc, bool backward, int bits, int dt)
{
    if (!items) return SASQ_ERR_NULL;
    if (count <= 0 || count > kCkMaxBatch) return SASQ_ERR_SHAPE;
    if (bits < 2 || bits > 8) return SASQ_ERR_UNSUPPORTED;
    if (dt != SASQ_F16 && dt != SASQ_BF16) return SASQ_ERR_UNSUPPORTED;
    int64_t blocks = 0;
    for (int i = 0; i < count; ++i) {
        const sasq_ckpt_item& it = items[i];
        if (!it.kept || (backward ? (!it.dy || !it.ds) : (!it.x || !it.s || !it.out))) return SASQ_ERR_NULL;
        if (it.rows <= 0 || it.cols <= 0 || it.rows > kCkMaxElements / it.cols || (pc && it.cols > kCkMaxCols)) return SASQ_ERR_SHAPE;
        if (!aligned16(it.kept) || !aligned16(it.out) || (backward ? !aligned16(it.dy) : !aligned16(it.x))) return SASQ_ERR_ALIGN;
        if (pc) blocks += (it.rows + ck_chunk_rows(it.rows, it.cols) - 1) / ck_chunk_rows(it.rows, it.cols) * ck_col_blocks(it.cols);
    }
    return blocks > kCkMaxBlocks ? SASQ_ERR_SHAPE : SASQ_OK;
}

static void ck_plan(const sasq_ckpt_item* items, int count, bool pc, bool backward, char* workspace, CkBatch& b)
{
    b.count = count;
    b.first[0] = 0;
    size_t at = kWsHeaderBytes;                      // the tickets of other calls on this workspace stay as they are
    for (int i = 0; i < count; ++i) {
        const sasq_ckpt_item& it = items[i];
        CkItem& k = b.it[i];
        k.x = static_cast<const uint16_t*>(it.x);
        k.s = it.s;
        k.out = static_cast<uint16_t*>(it.out);
        k.kept = it.kept;
        k.dy = static_cast<const uint16_t*>(it.dy);
        k.ds = it.ds;
        k.rows = it.rows; k.cols = it.cols; k.n = it.rows * it.cols;
        k.partial = workspace + at;
        int blocks;
        if (pc) {
            const int64_t r = ck_chunk_rows(it.rows, it.cols);
            k.chunk_rows = r;
            k.chunks = (int)((it.rows + r - 1) / r);
            blocks = (int)(k.chunks * ck_col_blocks(it.cols));
        } else {
            blocks = ck_blocks(k.n, backward ? ck_partials(count) : kCkBlocks);
        }
        if (backward) at += ck_partial_bytes(it.rows, it.cols, pc, count);
        b.first[i + 1] = b.first[i] + blocks;
    }
    for (int i = count; i < kCkMaxBatch; ++i) b.first[i + 1] = b.first[count];
}

static size_t ck_workspace(const sasq_ckpt_item* items, int count, bool pc)
{
    if (!items || count <= 0 || count > kCkMaxBatch) return 0;
    size_t bytes = kWsHeaderBytes;
    for (int i = 0; i < count; ++i) {
        if (items[i].rows <= 0 || items[i].cols <= 0 || items[i].rows > kCkMaxElements / items[i].cols || (pc && items[i].cols > kCkMaxCols)) return 0;
        bytes += ck_partial_bytes(items[i].rows, items[i].cols, pc, count);
    }
    const size_t one = kWsHeaderBytes + ck_partial_bytes(1, 1, false, 1);       // (one tensor has as many workgroups as four have)
    return pc || bytes > one ? bytes : one;
}

static bool ck_odd_rows(const CkBatch& b)
{
    for (int i = 0; i < b.count; ++i)
        if (b.it[i].cols % 8) return true;
    return false;
}

static int ck_fwd(const sasq_ckpt_item* items, int count, bool pc, int bits, sasq_dtype dt, void* stream)
{
    const int rc = ck_check(items, count, pc, false, bits, (int)dt);
    if (rc) return rc;
    CkBatch b{};
    ck_plan(items, count, pc, false, nullptr, b);
    hipStream_t st = as_stream(stream);
    const int grid = b.first[count];
    auto go = [&](auto dt_tag) {
        constexpr int DT = decltype(dt_tag)::value;
        if (!pc)                     ck_fwd_kernel<DT><<<grid, kCkThreads, 0, st>>>(b, bits);
        else if (ck_odd_rows(b))     ck_fwd_pc_kernel<DT, true><<<grid, kCkThreads, 0, st>>>(b, bits);
        else                         ck_fwd_pc_kernel<DT, false><<<grid, kCkThreads, 0, st>>>(b, bits);
    };
    if (dt == SASQ_F16) go(std::integral_constant<int, SASQ_F16>{});
    else                go(std::integral_constant<int, SASQ_BF16>{});
    return hipGetLastError() == hipSuccess ? SASQ_OK : SASQ_ERR_LAUNCH;
}

static int ck_bwd(const sasq_ckpt_item* items, int count, bool pc, int bits, sasq_dtype dt, void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = ck_check(items, count, pc, true, bits, (int)dt);
    if (rc) return rc;
    if (!workspace || workspace_bytes < ck_workspace(items, count, pc)) return SASQ_ERR_WORKSPACE;
    if (!aligned16(workspace)) return SASQ_ERR_ALIGN;
    CkBatch b{};
    ck_plan(items, count, pc, true, static_cast<char*>(workspace), b);
    hipStream_t st = as_stream(stream);
    const int grid = b.first[count];
    bool small = !pc, join = false;
    int64_t widest = 0;
    for (int i = 0; i < count; ++i) {
        if (b.it[i].n > kCkSmall) small = false;
        if (pc ? b.it[i].chunks > 1 : b.first[i + 1] - b.first[i] > 1) join = true;
        if (b.it[i].cols > widest) widest = b.it[i].cols;
    }
    auto go = [&](auto dt_tag) {
        constexpr int DT = decltype(dt_tag)::value;
        if (small)                   ck_bwd_kernel<DT, true><<<count, kCkSmallThreads, 0, st>>>(b, bits);
        else if (!pc)                ck_bwd_kernel<DT, false><<<grid, kCkThreads, 0, st>>>(b, bits);
        else if (ck_odd_rows(b))     ck_bwd_pc_kernel<DT, true><<<grid, kCkThreads, 0, st>>>(b, bits);
        else                         ck_bwd_pc_kernel<DT, false><<<grid, kCkThreads, 0, st>>>(b, bits);
        if (join && pc)              ck_join_pc_kernel<DT><<<dim3((unsigned)((widest + kWave - 1) / kWave), (unsigned)count), kCkThreads, 0, st>>>(b);
        else if (join && !small)     ck_join_kernel<DT><<<count, kCkThreads, 0, st>>>(b);
    };
    if (dt == SASQ_F16) go(std::integral_constant<int, SASQ_F16>{});
    else                go(std::integral_constant<int, SASQ_BF16>{});
    return hipGetLastError() == hipSuccess ? SASQ_OK : SASQ_ERR_LAUNCH;
}

}  // namespace sasq

using namespace sasq;

extern "C" int sasq_fakequant_fwd_ckpt_batch(const sasq_ckpt_item* items, int count, int bits, sasq_dtype dt, void* stream)
{
    return ck_fwd(items, count, false, bits, dt, stream);
}
extern "C" int sasq_fakequant_fwd_pc_ckpt_batch(const sasq_ckpt_item* items, int count, int bits, sasq_dtype dt, void* stream)
{
    return ck_fwd(items, count, true, bits, dt, stream);
}
extern "C" size_t sasq_fakequant_bwd_ckpt_batch_workspace(const sasq_ckpt_item* items, int count) { return ck_workspace(items, count, false); }
extern "C" size_t sasq_fakequant_bwd_pc_ckpt_batch_workspace(const sasq_ckpt_item* items, int count) { return ck_workspace(items, count, true); }
extern "C" int sasq_fakequant_bwd_ckpt_batch(const sasq_ckpt_item* items, int count, int bits, sasq_dtype dt, void* workspace, size_t workspace_bytes, void* stream)
{
    return ck_bwd(items, count, false, bits, dt, workspace, workspace_bytes, stream);
}
extern "C" int sasq_fakequant_bwd_pc_ckpt_batch(const sasq_ckpt_item* items, int count, int bits, sasq_dtype dt, void* workspace, size_t workspace_bytes, void* stream)
{
    return ck_bwd(items, count, true, bits, dt, workspace, workspace_bytes, stream);
}

extern "C" int sasq_fakequant_fwd_ckpt(const void* x, const float* s, void* y, int8_t* kept, int64_t rows, int64_t cols, int bits, sasq_dtype dt, void* stream)
{
    const sasq_ckpt_item it{x, s, y, kept, nullptr, nullptr, rows, cols};
    return ck_fwd(&it, 1, false, bits, dt, stream);
}
extern "C" int sasq_fakequant_fwd_pc_ckpt(const void* x, const float* s, void* y, int8_t* kept, int64_t rows, int64_t cols, int bits, sasq_dtype dt, void* stream)
{
    const sasq_ckpt_item it{x, s, y, kept, nullptr, nullptr, rows, cols};
    return ck_fwd(&it, 1, true, bits, dt, stream);
}
extern "C" size_t sasq_fakequant_bwd_ckpt_workspace(int64_t rows, int64_t cols)
{
    const sasq_ckpt_item it{nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, rows, cols};
    return ck_workspace(&it, 1, false);
}
extern "C" size_t sasq_fakequant_bwd_pc_ckpt_workspace(int64_t rows, int64_t cols)
{
    const sasq_ckpt_item it{nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, rows, cols};
    return ck_workspace(&it, 1, true);
}
extern "C" int sasq_fakequant_bwd_ckpt(const int8_t* kept, const void* dy, void* dx, float* ds, int64_t rows, int64_t cols, int bits, sasq_dtype dt,
                                       void* workspace, size_t workspace_bytes, void* stream)
{
    const sasq_ckpt_item it{nullptr, nullptr, dx, const_cast<int8_t*>(kept), dy, ds, rows, cols};
    return ck_bwd(&it, 1, false, bits, dt, workspace, workspace_bytes, stream);
}
extern "C" int sasq_fakequant_bwd_pc_ckpt(const int8_t* kept, const void* dy, void* dx, float* ds, int64_t rows, int64_t cols, int bits, sasq_dtype dt,
                                          void* workspace, size_t workspace_bytes, void* stream)
{
    const sasq_ckpt_item it{nullptr, nullptr, dx, const_cast<int8_t*>(kept), dy, ds, rows, cols};
    return ck_bwd(&it, 1, true, bits, dt, workspace, workspace_bytes, stream);
}
