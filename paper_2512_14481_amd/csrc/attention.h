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
// the group.  They are worked on in tiles of `tile_rows`, each over `splits` runs of `chunk` keys (the last one open-ended).  A tile
// of more than one run leaves fp32 partial results in the workspace, joined by a kernel of their own.
struct AttnSplit {
    int tile_rows, tiles, chunk, splits;
    float2* ml;                                           // running maximum (of log2-scaled scores) and sum
    float* o;                                             // unnormalized sums of values
};
__device__ __forceinline__ int64_t attn_slot(const AttnSplit& s, int batch, int heads, int split, int b, int hk, int r)
{
    return (((int64_t)split * batch + b) * heads + hk) * ((int64_t)s.tiles * s.tile_rows) + r;
}
// Keys that a tile's last row sees, and how many runs they make.
__device__ __forceinline__ int attn_end(const KvSeq& seq, int group, const AttnSplit& s, int tile)
{
    const int last = min(seq.rows * group, (tile + 1) * s.tile_rows) - 1;
    return max(seq.keys - seq.rows + last / group + 1, 0);
}
__device__ __forceinline__ int attn_runs(const AttnSplit& s, int end) { return min(s.splits, max(1, (end + s.chunk - 1) / s.chunk)); }

// 16 bytes a lane straight from global memory to LDS: lane i's go to lds_addr + 16 i.  The compiler does not know of the write: the
// callers order it with s_waitcnt vmcnt.
__device__ __forceinline__ void load_to_lds(uint32_t lds_addr, const void* base, uint32_t lane_off)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(lds_addr), "v"(lane_off), "s"(base) : "memory");
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
// The dword with 1 where a value is of the kind asked for (0: +inf, 1: -inf, 2: NaN) and 0 elsewhere; kind 3: the finite values.
template <int DT>
__device__ __forceinline__ uint32_t special_mask(uint32_t w, int kind)
{
    constexpr uint32_t e = DT == SASQ_F16 ? 0x7C00u : 0x7F80u, one = DT == SASQ_F16 ? 0x3C00u : 0x3F80u;
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t h = w >> (16 * i) & 0xFFFFu;
        const bool special = (h & e) == e, nan = (h & 0x7FFFu) > e;
        const int is = !special ? 3 : nan ? 2 : (int)(h >> 15);
        r |= (is != kind ? 0u : kind == 3 ? h : one) << (16 * i);
    }
    return r;
}

int attention_rows_launch(const AttnArgs& a, const KvPages& c, const KvSteps& s, const AttnSplit& split, int dim, bool int8, sasq_dtype dt, hipStream_t st);

}  // namespace sasq
