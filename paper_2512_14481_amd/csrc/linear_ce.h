// Cross entropy of a frozen output head (sasq_linear_ce): what its kernels share.
//
// Row i (of the counted ones, packed together), vocabulary entry v, target t:  z_v = x . W_v.  With lg = log2(e) and any number M of the row
//     a_v = 2^(z_v lg - M) for v != t,   S = sum a_v,   d = ln(sum_{v != t} e^{z_v}) - z_t = (M + log2 S - z_t lg) / lg
//     loss = ln(1 + e^d)     lse = z_t + loss     u = 1 - p_t = 1 / (1 + e^-d)
//     dx = g u (sum a_v W_v / S - W_t)
// The target is kept out of the sums, so that nothing cancels in a row whose target is all but certain.  The vocabulary goes by in pieces:
//     logits GEMM   z of a piece; each wave reduces its rows over its columns to (M, S) and stores a_v in 16 bits.  M is the row's so far, if
//                   there is one and a_v can be held so, else a whole number from the wave's own columns
//     join          M of the row so far, 2^(M_old - M) for its sums, and which rows have columns with another M
//     scale         these rows' a_v, by powers of two: those of the first piece, which is made small, and few in others
//     gradient GEMM the running sums over v of a_v W_v, fp32
// and at last one kernel divides, subtracts W_t and rounds.  A pass costs the two products that the formulas have and no third; the logits
// themselves are never stored.
#pragma once

#include "gemm_tile.h"

namespace sasq {

// (off by 2^-26 of itself: of a logit z, its exponential is off by 2^-26 |z|, less than the product that z is)
constexpr float kLog2e = 1.44269504088896340736f;

// 16-bit a_v of a wave's own M are at most 2^kTopExp; those of the row's M so far may be 2^kRoom times as much.  fp16 has 2^-24 .. 2^15 to offer.  bf16 has the
// exponents of fp32, but the fp32 sums of a_v W_v have to hold them too: 2^22 terms of at most 2^8 max |W| stay below 2^128 for entries below 2^98 (room for 2^64
// in its place left 2^42).  5.5 nats are what a row's largest logit may grow by from piece to piece before its columns are multiplied once more.
template <int DT> constexpr int kTopExp = DT == SASQ_F16 ? 11 : 0;
template <int DT> constexpr int kRoom = DT == SASQ_F16 ? 4 : 8;

struct RowStat { float m, s; };                 // M (a whole number; -inf: no column yet) and S

struct CeArgs {
    // sizes
    int64_t T, V, H;
    int Hp, Vp;                                 // H and V in whole multiples of 64
    int piece, first_piece;                     // columns of a piece, and of the first
    int slots, max_splits;                      // parts that its contraction is cut into: as many as fill the slots of the chip (grad_parts)
    int tile, grad_tile;                        // 0: 256x256, 2: 128x128
    bool grad;
    int few_parts;                              // few rows (linear_ce_few.hip): parts of the gradient's contraction, 0: the tiles
    int few_cols;                               // columns of a workgroup of its logits, and of an M and S
    bool few_own_join;                          // and so few groups of columns that the gradient's kernels join them by themselves
    // operands
    const void* x; int64_t x_stride;
    const uint8_t* head; const uint8_t* head_grad;
    const int32_t* targets;
    const float* row_weight; float scale;
    float* loss; float* lse; float* mean;
    void* dx; int64_t dx_stride;
    // workspace
    int32_t* count;                             // counted rows
    int32_t* pos;                               // [T] place of a row among them, -1: left out
    int32_t* row;                               // [T] packed: the row
    int32_t* tgt;                               // [T] packed: target
    float* zt;                                  // [T] packed: z_t
    RowStat* run;                               // [T] packed: M and S of the pieces so far
    float* beta;                                // [T] packed: 2^(M_old - M)
    uint8_t* scale_rows;                        // [T / 16] packed: whether any of sixteen rows has columns with another M
    uint32_t* ticket; double* part;             // of the mean: workgroups of the join that are done, their sums
    float* coef;                                // [T] packed: u / S
    float* u;                                   // [T] packed: u
    RowStat* stats;                             // [columns of a piece / stat_cols][T]
    uint16_t* xs;                               // packed rows of x, zeros past H, in the 1 KB blocks of the GEMMs' operands (block_at)
    uint16_t* a;                                // a_v of a piece, rows and columns in the same blocks
    float* acc;                                 // [parts][counted rows][Hp]
};
// Parts of the gradient's contraction for so many counted rows: as many as fill the slots of the chip.  A last row of 256x256 tiles of at most 128 rows is of
// halves, which take 0.65 of the time, and has fewer and longer parts.
struct GradParts {
    int tiles;                                  // rows of whole tiles, with `full` parts each
    int full, half;                             // half: parts of the halves behind them, 0: there are none
    __host__ __device__ int of_row(int64_t row, int bm) const { return row < (int64_t)tiles * bm ? full : half; }
};
__host__ __device__ inline GradParts grad_parts(int64_t rows, int bm, int tiles_n, int slots, int max_splits)
{
    const int rest = (int)(rows % bm);
    const bool halves = bm == 256 && rest > 0 && rest <= 128;
    const int64_t tiles = rows / bm + (rest > 0 && !halves);
    auto clamp = [&](int64_t s, int64_t most) { return (int)(s > most ? most : s < 1 ? 1 : s); };
    GradParts p{(int)tiles, 0, 0};
    if (tiles) p.full = clamp(100 * (int64_t)slots / (tiles_n * (100 * tiles + (halves ? 65 : 0))), max_splits);
    if (halves) p.half = clamp((slots - tiles * p.full * tiles_n) / tiles_n, tiles ? p.full : max_splits);
    return p;
}
constexpr int tile_rows(int tile) { return tile == 0 ? 256 : 128; }
constexpr int tile_cols(int tile) { return tile_rows(tile); }
constexpr int stat_cols(int tile) { return tile == 2 ? 64 : 128; }     // half a tile's columns: what a wave has

// Blocks from one row of blocks to the next, of `cols` columns (a multiple of 64): an odd number.
__host__ __device__ constexpr int row_blocks(int64_t cols) { return (int)(cols / 32) | 1; }
// Element (row, col) of an operand in 1 KB blocks of 16 rows x 32 columns, `kt` blocks a row of blocks; col a multiple of 8: a chunk of 16 bytes.
__device__ __forceinline__ int64_t block_at(int64_t row, int col, int kt)
{
    const int r = (int)(row & 15), c = (col >> 3) & 3;
    return ((row >> 4) * kt + (col >> 5)) * 512 + ((4 * r + (c ^ swz64(r))) << 3) + (col & 7);
}

void launch_ce_logits(const CeArgs& c, sasq_dtype dt, int64_t col0, int64_t cols, hipStream_t st);
void launch_ce_grad(const CeArgs& c, sasq_dtype dt, int64_t col0, int64_t cols, hipStream_t st);

// At most kFewRows rows, or kFewMost where the head is small (ce_few), the whole vocabulary in one piece (linear_ce_few.hip).  M and S are of few_cols columns (16, 32 or 64); rows are not packed.
// kFewOwnJoin: up to so many M and S in all, every workgroup of the gradient reads them and the join is no kernel of its own (64 x 256 -> 1000 22.8 -> 18.8 us).
// kFewCols: most columns of a workgroup of the logits, and channels of one of the gradient.
constexpr int kFewMost = 2048, kFewRows = 64, kFewCols = 64, kFewOwnJoin = 4096;
void launch_ce_few_logits(const CeArgs& c, sasq_dtype dt, hipStream_t st);
void launch_ce_few_grad(const CeArgs& c, sasq_dtype dt, hipStream_t st);

}  // namespace sasq
