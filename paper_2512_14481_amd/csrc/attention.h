// Attention over the paged key/value cache: what its kernels and host logic share (gfx950 only).
#pragma once

#include "gemm_tile.h"
#include "kv_cache.h"

namespace sasq {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i16x4* lds_i16x4;
typedef __attribute__((address_space(3))) i32x2* lds_i32x2;

struct AttnArgs {
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    int64_t q_stride, out_stride;
    int q_heads, group;                                   // group: query heads of a kv head
    float scale;
};

// A kv head's rows of a sequence are its new tokens times the query heads that share it: row r is token r / group, head r % group of
// the group.  A sequence with up to kFewRows of them is worked on in one piece, another in tiles of kTileRows (of half as many where no
// sequence has more), each over `splits` runs of `chunk` keys (the last one open-ended).  Where there is more than one run each leaves fp32
// partial results in the workspace, joined by a kernel of their own.  The two kinds of sequences have runs and places of their own: single
// tokens are split finely.
constexpr int kFewRows = 16, kTileRows = 128;
struct AttnSplit {
    int tile_rows, rows, chunk, splits;                   // rows: the most that a sequence has (kFewRows at most, or any number)
    float2* ml;                                           // running maximum (of log2-scaled scores) and sum
    float* o;                                             // unnormalized sums of values
};
// Places of the partial results of row r of a sequence of few rows, and of token t and a head of the others.
__device__ __forceinline__ int64_t few_slot(const AttnSplit& s, int batch, int heads, int run, int b, int hk, int r)
{
    return (((int64_t)run * batch + b) * heads + hk) * s.rows + r;
}
__device__ __forceinline__ int64_t token_slot(int tokens, int q_heads, int run, int t, int head) { return ((int64_t)run * tokens + t) * q_heads + head; }
// Keys that a tile's last row sees, and how many runs they make.
__device__ __forceinline__ int attn_end(const KvSeq& seq, int group, const AttnSplit& s, int tile)
{
    const int last = min(seq.rows * group, (tile + 1) * s.tile_rows) - 1;
    return max(kv_last(seq, last / group) + 1, 0);
}
__device__ __forceinline__ int attn_runs(const AttnSplit& s, int end) { return min(s.splits, max(1, (end + s.chunk - 1) / s.chunk)); }

// 16 bytes a lane straight from global memory to LDS: lane i's go to lds_addr + 16 i.  The compiler does not know of the write: the
// callers order it with s_waitcnt vmcnt.  Non-temporal, for what is read once (48 sequences of 70B 109 us without, 100 with).
__device__ __forceinline__ void load_to_lds_once(uint32_t lds_addr, const void* base, uint32_t lane_off)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" :: "s"(lds_addr), "v"(lane_off), "s"(base) : "memory");
}
// The same with the ordinary policy, or nothing where `on` is 0 (all ones otherwise): no branch, which would part the products that the
// load stands among.
__device__ __forceinline__ void load_to_lds_if(int on, uint32_t lds_addr, const void* base, uint32_t lane_off)
{
    uint64_t lanes;
    asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, exec\n\ts_and_b32 exec_lo, exec_lo, %4\n\ts_and_b32 exec_hi, exec_hi, %4\n\t"
                 "global_load_lds_dwordx4 %2, %3\n\ts_mov_b64 exec, %0"
                 : "=&s"(lanes) : "s"(lds_addr), "v"(lane_off), "s"(base), "s"(__builtin_amdgcn_readfirstlane(on)) : "memory", "scc");
}

// Four int8 codes as fp16, exactly: a byte c + 128 in the low half of 0x6400 is 1152 + c.
__device__ __forceinline__ u32x2 codes_to_f16(uint32_t c)
{
    const f16x2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    const uint32_t u = c ^ 0x80808080u;
    const f16x2 lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - bias;
    const f16x2 hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - bias;
    return {__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

template <int DT>
__device__ __forceinline__ f32x4 mfma16(const u32x4& a, const u32x4& b, const f32x4& c)
{
    if constexpr (DT == SASQ_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Which of a dword's two 16-bit values are infinite or NaN.
template <int DT>
__device__ __forceinline__ bool any_special(uint32_t w)
{
    constexpr uint32_t e = DT == SASQ_F16 ? 0x7C00u : 0x7F80u;
    return (w & e) == e || (w >> 16 & e) == e;
}
// The dword with its infinite and NaN values at 0.
template <int DT>
__device__ __forceinline__ uint32_t finite_of(uint32_t w)
{
    constexpr uint32_t e = DT == SASQ_F16 ? 0x7C00u : 0x7F80u;
    return ((w & e) == e ? 0u : w & 0xFFFFu) | ((w >> 16 & e) == e ? 0u : w & 0xFFFF0000u);
}
// Adds +inf, or -inf, to the output of the rows that see an infinite value of that sign, and both for a NaN: as a product of the largest
// bf16 value by itself, which overflows, so that the rows that do not see it (a factor of 0) stay as they are.  v: eight values of the
// first operand, seen: kSeen (else 0) for the eight keys of the second.
constexpr uint32_t kSeen = 0x7F7Fu;
template <int DT>
__device__ __forceinline__ f32x4 add_specials(const u32x4& v, const u32x4& seen, f32x4 o)
{
    constexpr uint32_t e = DT == SASQ_F16 ? 0x7C00u : 0x7F80u;
#pragma unroll
    for (int sign = 0; sign < 2; ++sign) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = 0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t h = v[j] >> (16 * i) & 0xFFFFu;
                const bool mine = (h & 0x7FFFu) > e || h == (e | (uint32_t)sign << 15);
                w[j] |= (mine ? kSeen | (uint32_t)sign << 15 : 0u) << (16 * i);
            }
        }
        o = mfma16<SASQ_BF16>(w, seen, o);
    }
    return o;
}

template <int N>
__device__ __forceinline__ void wait_loads()
{
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(N));
    asm volatile("" ::: "memory");
}

// A probability is 2^(score - m).  m is moved only when a score would pass `most`, and then to `below` under the row's largest: the common step
// needs no reduction over lanes and no rescaling of the output, and rounding is relative all the same.  fp16 ends at 2^-24, so probabilities go as
// high as it reaches with room for a score in between (the largest 2^7 to 2^15): what is rounded to 0 is under 2^-32 of the row's largest, 2^-15 of
// the row for 131072 such keys (at 2^0 to 2^8 it was 2^-25 of each, 0.4 % of the row).  bf16 has room below but values as large as fp32's:
// probabilities of 1 at most (the largest 2^-8 to 2^0) times them stay in it.
template <int DT>
struct Lazy {
    static constexpr float below = DT == SASQ_F16 ? 7.0f : -8.0f, most = below + 8.0f;
};
// m before any score: finite, so that a row whose scores are all masked gets probabilities of 0, and the lowest that is, so that any other
// score moves it (or is that value, with a probability of 1).
constexpr float kNoMax = -0x1.fffffep127f;
// m is a product of a score and c, rounded; from here on the exact product that a fused multiply-add subtracts it from is more than half a
// power of two away (2^128 from about 2^32 on: probabilities of 0 or infinity for the largest score itself), and is to be rounded alike.
constexpr float kExact = 0x1p24f;
// What sums over an older maximum are multiplied by.  Never 0, which would make NaN of an infinite sum, but the least there is: of a sum of 2^120
// (bf16 values) 1e-37 would be 0.1 of what has no weight.
__device__ __forceinline__ float kept(float before, float now) { return fmaxf(__builtin_amdgcn_exp2f(before - now), 0x1p-149f); }
// The same for a part of a row's keys, f = (maximum, sum), joined with others under `top`: a part without keys has nothing to add, one whose
// maximum is infinite or whose sum is NaN hands that on.
__device__ __forceinline__ float part_weight(const float2& f, float top)
{
    return f.x == -INFINITY && f.y == 0.0f ? 0.0f : f.x == top ? 1.0f : kept(f.x, top);
}

// Keys or values of one head in LDS.  A wave-wide load brings whole rows, 1 KB of them, and puts them down as a block: four of a row's
// 16-byte chunks together (neighbouring lanes read neighbouring bytes: loads whose lanes took turns among the rows took 150 cycles each
// to issue), the rows' fours after each other, blocks 16 bytes apart, and the chunks of a four swapped in pairs in every other four rows of a
// block.  The eight rows that a wave reads at a time at one chunk then lie in different banks, and so does what a transposing read of 16 lanes
// takes (16 bits: two chunks of four rows; codes: a chunk of four rows of both halves of 32); and every place is a lane's own plus
// a constant.
template <int D, bool I8>
struct KvRow {
    static constexpr int kRow = D * (I8 ? 1 : 2);         // bytes of a key
    static constexpr int kPerLoad = 1024 / kRow;          // rows of a block
    static constexpr int kLoads = 16 / kPerLoad;          // blocks of 16 rows
    static constexpr int kBlock = 1024 + 16;
    static constexpr int k16 = kLoads * kBlock;           // bytes of 16 rows
    static constexpr int kFour = kPerLoad * 64;           // from a chunk to the fourth after it
    static __device__ __forceinline__ int swapped(int row) { return (row % kPerLoad >> 2 ^ row % kPerLoad >> 3) & 1; }
    static __device__ __forceinline__ int place(int row, int chunk)
    {
        return row / kPerLoad * kBlock + (chunk >> 2) * kFour + row % kPerLoad * 64 + ((chunk & 3) ^ swapped(row)) * 16;
    }
    // Chunks 0..3 of a four, where the lane's own is 0 or 1 and `chunk` is even: the swap is in the lane's part already.
    static constexpr int step(int chunk) { return (chunk >> 2) * kFour + (chunk & 3) * 16; }
    // Where lane's 16 bytes of block j of 16 rows come from.
    static __device__ __forceinline__ uint32_t source(int j, int lane, int64_t token_stride)
    {
        const int row = lane / 4 % kPerLoad, chunk = lane / 4 / kPerLoad * 4 + ((lane & 3) ^ swapped(row));
        return (uint32_t)((j * kPerLoad + row) * token_stride) + 16 * chunk;
    }
    // First operands of 16x16x32; a lane is (l16 = lane % 16, g = lane / 16).
    // K Q^T: 16 bytes of row l16, from chunk 4 t + g on.  at: the 16 keys + key_lane.
    static __device__ __forceinline__ int key_lane(int lane) { return place(lane & 15, lane >> 4); }
    static __device__ __forceinline__ u32x4 key(const char* at, int t) { return *reinterpret_cast<const u32x4*>(at + t * kFour); }
    // V^T P^T: channel 16 n + l16 of the eight keys that a lane has scores of, in 16 bits: rows 4g..4g+3 of both halves of 32 keys.
    // at: the 32 keys + value_lane.
    static __device__ __forceinline__ int value_lane(int lane)
    {
        const int l16 = lane & 15, g = lane >> 4;
        if constexpr (I8) return place((l16 < 8 ? 0 : 16) + 4 * g + (l16 >> 1 & 3), 0) + 8 * (l16 & 1);
        else              return place(4 * g + (l16 >> 2), l16 >> 1 & 1) + 8 * (l16 & 1);
    }
    // (Codes of 16 channels are one chunk: of the odd ones the lane's part has the swap the wrong way round; this is what is to be added.)
    static __device__ __forceinline__ int value_odd(int lane) { return 16 - 32 * swapped(4 * (lane >> 4)); }
    static __device__ __forceinline__ u32x4 value(const char* at, int n, int odd)
    {
        if constexpr (I8) {
            const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2)(at + step(n & ~1) + (n & 1 ? odd : 0)));
            const u32x2 x = codes_to_f16((uint32_t)w[0]), y = codes_to_f16((uint32_t)w[1]);
            return u32x4{x[0], x[1], y[0], y[1]};
        } else {
            const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(at + step(2 * n))));
            const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(at + k16 + step(2 * n))));
            return u32x4{x[0], x[1], y[0], y[1]};
        }
    }
};

// Q as the second operand of K Q^T: eight channels of the lane's row for each step of 32.  c: from a score to a power of two.
template <int DTQ, int D, bool I8>
__device__ __forceinline__ void load_q(const AttnArgs& a, const uint16_t* src, bool there, int g, float k_scale, u32x4 (&q)[D / 32], float& c)
{
    constexpr int DS = D / 32;
#pragma unroll
    for (int t = 0; t < DS; ++t) {
        const int d = I8 ? 64 * (t >> 1) + 16 * g + 8 * (t & 1) : 32 * t + 8 * g;          // sixteen codes of one load serve two steps
        q[t] = *reinterpret_cast<const u32x4*>(src + d);
        if (!there) q[t] = u32x4{0, 0, 0, 0};
    }
    c = a.scale * 1.44269504088896f;
    if constexpr (I8) {
        int e = 0;
        // fp16 products: a bf16 row is brought to at most 2 by a power of two (exact but for values 2^-14 and more below its largest),
        // and the sign of the factor goes into Q, so that larger products stay larger scores.
        const uint32_t flip = k_scale < 0.0f ? 0x80008000u : 0u;
        if constexpr (DTQ == SASQ_BF16) {
            float top = 0.0f;
#pragma unroll
            for (int t = 0; t < DS; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(Store16<DTQ>::lo(q[t][i])), fabsf(Store16<DTQ>::hi(q[t][i]))));
            top = fmaxf(top, __shfl_xor(top, 16, kWave));
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            e = top > 0.0f && top < INFINITY ? __builtin_amdgcn_frexp_expf(top) - 1 : 0;      // -133 to 127: no single factor reaches both ends
#pragma unroll
            for (int t = 0; t < DS; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) q[t][i] = Store16<SASQ_F16>::pack(__builtin_ldexpf(Store16<DTQ>::lo(q[t][i]), -e), __builtin_ldexpf(Store16<DTQ>::hi(q[t][i]), -e));
        }
#pragma unroll
        for (int t = 0; t < DS; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) q[t][i] ^= flip;
        // The three are multiplied with their powers of two apart: two of them may leave fp32 where all three do not.  Where these do, scores
        // are infinite, but a score of 0 stays that.
        c = __builtin_ldexpf(__builtin_amdgcn_frexp_mantf(c) * __builtin_amdgcn_frexp_mantf(fabsf(k_scale)),
                             __builtin_amdgcn_frexp_expf(c) + __builtin_amdgcn_frexp_expf(k_scale) + e);
        c = fminf(c, 0x1.fffffep127f);
    }
    c = fmaxf(c, 0x1p-149f);                              // a scale and a factor whose product is 0 in fp32: a masked score times it stays -inf
}

// Calls whose sequences all have few rows are the rows kernel's, any others the tiles kernel's.
int attention_rows_launch(const AttnArgs& a, const KvPages& c, const KvSteps& s, const AttnSplit& few, int dim, bool int8, sasq_dtype dt, hipStream_t st);
int attention_tiles_launch(const AttnArgs& a, const KvPages& c, const KvSteps& s, const AttnSplit& few, const AttnSplit& many, int64_t many_blocks, int64_t few_blocks,
                           int dim, bool int8, sasq_dtype dt, hipStream_t st);
int attention_join_launch(const AttnArgs& a, const KvPages& c, const KvSteps& s, const AttnSplit& few, const AttnSplit& many, bool join_few, bool join_many, int dim, sasq_dtype dt, hipStream_t st);

}  // namespace sasq
