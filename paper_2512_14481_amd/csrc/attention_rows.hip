// Attention of few rows over the paged cache (single tokens, drafts): bound by the bytes of the cache.
//
// A workgroup has one kv head of one sequence, up to 16 RB rows of it (RB blocks of 16), and one run of keys; its four waves take
// slabs of 32 keys in turn, each with its own running maximum, sum and output, joined at the end.  A wave streams its slabs through a
// ring of two stages of its own in LDS (direct global-to-LDS loads, no barrier in the loop): one stage is always in flight.
//
// Products are taken transposed, so that a lane keeps one row from the scores to the output:
//   S^T[key, row] = K Q^T     16x16x32: lane (row = l % 16, g = l / 16) gets keys 4g..4g+3 of each 16
//   O^T[d, row]  += V^T P^T   the eight keys of a lane's slots are then the ones it has scores of (4g + j of both halves of the slab):
//                             the probabilities go into the second product as they come out of the first, and V is read
//                             transposed by ds_read_tr with the same order of keys.
// The running maximum is moved only when a score passes it by more than 8 (in powers of two): probabilities then reach 2^8 at most, and
// the common slab needs no reduction over lanes and no rescaling.
#include "attention.h"

namespace sasq {

constexpr int kSlab = 32, kRing = 2, kRowWaves = 4;
constexpr int kSegment = 2048;                            // keys whose pages are listed in LDS at a time

template <int D, bool I8>
struct RowsGeo : KvRow<D, I8> {
    using K = KvRow<D, I8>;
    static constexpr int kPart = 2 * K::k16;              // a slab's keys, or its values
    static constexpr int kStage = 2 * kPart;
    static constexpr int kRingBytes = kRowWaves * kRing * kStage;
    static constexpr int kJoin = kRowWaves * 16 * (D + 4) * 4;
    static constexpr int kBody = kRingBytes > kJoin ? kRingBytes : kJoin;
    static constexpr int kLds = kBody + kRowWaves * 16 * 8 + kSegment / 16 * 4;
};

template <int DTQ, int D, bool I8, int RB>
__global__ __launch_bounds__(kRowWaves * 64, 1) void attention_rows_kernel(AttnArgs a, KvPages cache, KvSteps steps, AttnSplit split, int few, int first)
{
    using G = RowsGeo<D, I8>;
    constexpr int DT = I8 ? SASQ_F16 : DTQ;               // of the products
    constexpr int DS = D / 32, DO = D / 16;               // steps over d of the first product, blocks of d of the second
    __shared__ __attribute__((aligned(1024))) char lds[G::kLds];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int l16 = lane & 15, g = lane >> 4;

    int rest = (int)blockIdx.x + first;
    const int hk = rest % cache.heads; rest /= cache.heads;
    const int tile = rest % split.tiles; rest /= split.tiles;
    const int b = rest % steps.batch, run = rest / steps.batch;
    const KvSeq seq = kv_seq(steps, b, cache.page_shift);
    const int rows = seq.rows * a.group, row0 = tile * 16 * RB;
    if (rows > few || row0 >= rows) return;
    const int end = attn_end(seq, a.group, split, tile), runs = attn_runs(split, end);
    if (run >= runs) return;
    const int from = run * split.chunk, to = run == runs - 1 ? end : min(end, from + split.chunk);
    const int sees_first = seq.keys - seq.rows + row0 / a.group;           // last key of the tile's first row: masks begin after it

    // The lane's rows: their last key, and Q as the second operand (8 channels of row l16 for each step).
    int sees[RB];
    float c[RB];                                                           // from a score to a power of two
    u32x4 q[RB][DS];
    const float k_scale = I8 ? cache.k_scale[hk] : 1.0f;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = row0 + 16 * rb + l16;
        const bool there = r < rows;
        const int token = (there ? r : row0) / a.group, head = (there ? r : row0) % a.group;
        sees[rb] = seq.keys - seq.rows + token;
        load_q<DTQ, D, I8, 16>(a, a.q + (int64_t)(seq.row0 + token) * a.q_stride + (int64_t)(hk * a.group + head) * D, there, g, k_scale, q[rb], c[rb]);
    }

    uint32_t off[G::kLoads];
#pragma unroll
    for (int j = 0; j < G::kLoads; ++j) off[j] = G::source(j, lane, cache.token_stride);
    char* const ring = lds + wave * kRing * G::kStage;
    const uint32_t ring_at = (uint32_t)(uintptr_t)(lds_ptr_t)ring;
    int* const pages = reinterpret_cast<int*>(lds + G::kBody + kRowWaves * 16 * 8);

    f32x4 o[RB][DO];
    float m[RB], l[RB];                                                    // maximum of the log2-scaled scores, sum
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m[rb] = kNoMax; l[rb] = 0.0f;
#pragma unroll
        for (int i = 0; i < DO; ++i) o[rb][i] = f32x4{0, 0, 0, 0};
    }

    for (int seg = from; seg < to; seg += kSegment) {
        const int seg_end = min(to, seg + kSegment);
        if (seg != from) __syncthreads();
        for (int u = (int)threadIdx.x; u < kSegment / 16 && seg + 16 * u < seg_end; u += kRowWaves * 64) {
            const int index = (seg + 16 * u) >> cache.page_shift;
            pages[u] = index < steps.max_pages ? kv_page(cache, steps, b, index) : -1;
        }
        __syncthreads();
        const int units = (seg_end - seg + 15) / 16, slabs = (units + 1) / 2;
        const int mine = (slabs - wave + kRowWaves - 1) / kRowWaves;       // slabs wave, wave + 4, ...
        auto page_of = [&](int i, int h) -> int {                          // -1: nothing there
            const int u = 2 * (wave + i * kRowWaves) + h;
            return u < units ? __builtin_amdgcn_readfirstlane(pages[u]) : -1;
        };
        auto fetch = [&](int i, const uint8_t* plane, int part) {
            const int k0 = seg + kSlab * (wave + i * kRowWaves);
            const uint32_t at = ring_at + (i % kRing) * G::kStage + part * G::kPart;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int page = page_of(i, h), place = (k0 + 16 * h) & ((1 << cache.page_shift) - 1);
                const uint8_t* base = plane + (int64_t)hk * cache.head_stride + (page < 0 ? 0 : page * cache.page_stride + place * cache.token_stride);
#pragma unroll
                for (int j = 0; j < G::kLoads; ++j) load_to_lds(at + (h * G::kLoads + j) * G::kBlock, base, off[j]);
            }
        };
        wait_loads<0>();                                                   // Q has landed: the loop's waits count the ring's loads alone
        constexpr int NL = 2 * G::kLoads;                                  // loads of a slab's keys, or of its values
        for (int i = 0; i < kRing && i < mine; ++i) { fetch(i, cache.k, 0); fetch(i, cache.v, 1); }
        for (int i = 0; i < mine; ++i) {
            const char* stage = ring + (i % kRing) * G::kStage;
            const char* kp = stage + G::template key_lane<16>(lane);
            const char* vp = stage + G::kPart + G::template value_lane<16>(lane);
            const int k0 = seg + kSlab * (wave + i * kRowWaves);
            if (i + 1 < mine) wait_loads<3 * NL>();
            else              wait_loads<NL>();
            f32x4 s[RB][2];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) s[rb][0] = s[rb][1] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < (I8 ? DS / 2 : DS); ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const u32x4 w = G::template key<16>(kp + h * G::k16, t);
                    if constexpr (I8) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const u32x2 x = codes_to_f16(w[2 * e]), y = codes_to_f16(w[2 * e + 1]);
                            const u32x4 k = {x[0], x[1], y[0], y[1]};
#pragma unroll
                            for (int rb = 0; rb < RB; ++rb) s[rb][h] = mfma16<DT>(k, q[rb][2 * t + e], s[rb][h]);
                        }
                    } else {
#pragma unroll
                        for (int rb = 0; rb < RB; ++rb) s[rb][h] = mfma16<DT>(w, q[rb][t], s[rb][h]);
                    }
                }
            const int page0 = page_of(i, 0), page1 = page_of(i, 1);
            __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
            asm volatile("" ::: "memory");
            if (i + kRing < mine) fetch(i + kRing, cache.k, 0);

            const bool masked = k0 + kSlab - 1 > sees_first || page0 < 0 || page1 < 0;
            if (masked) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (page0 < 0 || k0 + 4 * g + j > sees[rb]) s[rb][0][j] = -INFINITY;
                        if (page1 < 0 || k0 + 16 + 4 * g + j > sees[rb]) s[rb][1][j] = -INFINITY;
                    }
            }
            u32x4 p[RB];
            float top[RB];
            bool above = false;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                top[rb] = fmaxf(fmaxf(fmaxf(s[rb][0][0], s[rb][0][1]), fmaxf(s[rb][0][2], s[rb][0][3])),
                                fmaxf(fmaxf(s[rb][1][0], s[rb][1][1]), fmaxf(s[rb][1][2], s[rb][1][3])));
                above |= __builtin_fmaf(top[rb], c[rb], -m[rb]) > kLazy;
            }
            if (__any(above)) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    float t = fmaxf(top[rb], __shfl_xor(top[rb], 16, kWave));
                    t = fmaxf(t, __shfl_xor(t, 32, kWave));
                    t = fmaxf(t * c[rb], m[rb]);
                    const float keep = kept(m[rb], t);
                    m[rb] = t;
                    l[rb] *= keep;
#pragma unroll
                    for (int i2 = 0; i2 < DO; ++i2) o[rb][i2] *= keep;
                }
            }
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                float e[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][j >> 2][j & 3], c[rb], -m[rb]));
                l[rb] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
#pragma unroll
                for (int j = 0; j < 4; ++j) p[rb][j] = Store16<DT>::pack(e[2 * j], e[2 * j + 1]);
            }

            if (i + kRing < mine)    wait_loads<3 * NL>();
            else if (i + 1 < mine)   wait_loads<2 * NL>();
            else                     wait_loads<0>();
            u32x4 v[DO];
#pragma unroll
            for (int n = 0; n < DO; ++n) v[n] = G::template value<16>(vp, n, G::value_odd(lane));
            if constexpr (!I8) {
                // A masked place may hold anything, and 0 times infinity is not 0: infinities and NaN are taken out of the product and
                // put in by hand for the rows that see them.
                if (masked) {
                    bool special = false;
#pragma unroll
                    for (int n = 0; n < DO; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j) special |= any_special<DT>(v[n][j]);
                    if (__any(special)) {
#pragma unroll
                        for (int rb = 0; rb < RB; ++rb) {
                            u32x4 seen;
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const int key = k0 + (j < 2 ? 0 : 16) + 4 * g + 2 * (j & 1);
                                const bool there = (j < 2 ? page0 : page1) >= 0;
                                seen[j] = (there && key <= sees[rb] ? kSeen : 0u) | (there && key + 1 <= sees[rb] ? kSeen << 16 : 0u);
                            }
#pragma unroll
                            for (int n = 0; n < DO; ++n) o[rb][n] = add_specials<DT>(v[n], seen, o[rb][n]);
                        }
#pragma unroll
                        for (int n = 0; n < DO; ++n)
#pragma unroll
                            for (int j = 0; j < 4; ++j) v[n][j] = finite_of<DT>(v[n][j]);
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < DO; ++n)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) o[rb][n] = mfma16<DT>(v[n], p[rb], o[rb][n]);
            __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
            asm volatile("" ::: "memory");
            if (i + kRing < mine) fetch(i + kRing, cache.v, 1);
        }
    }

    // Join the waves, one block of 16 rows at a time: thread (row, eight channels or four).
    constexpr int E = D / 16;
    float* const part = reinterpret_cast<float*>(lds);                     // [wave][row][D + 4]
    float2* const ml = reinterpret_cast<float2*>(lds + G::kBody);          // [wave][row]
    const float v_scale = I8 ? cache.v_scale[hk] : 1.0f;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        __syncthreads();
        l[rb] += __shfl_xor(l[rb], 16, kWave);
        l[rb] += __shfl_xor(l[rb], 32, kWave);
        if (g == 0) ml[wave * 16 + l16] = make_float2(m[rb] == kNoMax ? -INFINITY : m[rb], l[rb]);
#pragma unroll
        for (int n = 0; n < DO; ++n) *reinterpret_cast<f32x4*>(part + (wave * 16 + l16) * (D + 4) + 16 * n + 4 * g) = o[rb][n];
        __syncthreads();
        const int rr = (int)threadIdx.x >> 4, d = ((int)threadIdx.x & 15) * E, r = row0 + 16 * rb + rr;
        float top = -INFINITY, sum = 0.0f, x[E];
#pragma unroll
        for (int w = 0; w < kRowWaves; ++w) top = fmaxf(top, ml[w * 16 + rr].x);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = 0.0f;
#pragma unroll
        for (int w = 0; w < kRowWaves; ++w) {
            const float2 f = ml[w * 16 + rr];
            const float weight = part_weight(f, top);
            sum += f.y * weight;
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = __builtin_fmaf(part[(w * 16 + rr) * (D + 4) + d + e], weight, x[e]);
        }
        if (r >= rows) continue;
        const int token = r / a.group, head = hk * a.group + r % a.group;
        if (runs == 1) {
            const bool none = sum == 0.0f;
            const float f = none ? 0.0f : v_scale / sum;
            uint16_t* dst = a.out + (int64_t)(seq.row0 + token) * a.out_stride + (int64_t)head * D + d;
            uint32_t w[E / 2];
#pragma unroll
            for (int e = 0; e < E / 2; ++e) w[e] = none ? 0u : Store16<DTQ>::pack(x[2 * e] * f, x[2 * e + 1] * f);
            __builtin_memcpy(dst, w, sizeof(w));
            if (a.lse && d == 0) a.lse[(int64_t)(seq.row0 + token) * a.q_heads + head] = none ? -INFINITY : (top + log2f(sum)) * 0.693147180559945f;
        } else {
            const int64_t slot = rows_slot(split, steps.batch, cache.heads, run, b, hk, r);
            float* dst = split.o + slot * D + d;
#pragma unroll
            for (int e = 0; e < E; e += 4) *reinterpret_cast<f32x4*>(dst + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
            if (d == 0) split.ml[slot] = make_float2(top, sum);
        }
    }
}

int attention_rows_launch(const AttnArgs& a, const KvPages& c, const KvSteps& s, const AttnSplit& split, int few, int dim, bool int8, sasq_dtype dt, hipStream_t st)
{
    auto go = [&](auto kernel) {
        launch_in_parts((int64_t)split.splits * s.batch * split.tiles * c.heads, 256,
                        [&](unsigned n, int first) { hipLaunchKernelGGL(kernel, dim3(n), dim3(256), 0, st, a, c, s, split, few, first); });
    };
    auto with = [&](auto dtv, auto dimv, auto i8v) {
        constexpr int DT = decltype(dtv)::value, D = decltype(dimv)::value;
        constexpr bool I8 = decltype(i8v)::value;
        if (split.tile_rows == 16)      go(attention_rows_kernel<DT, D, I8, 1>);
        else if (split.tile_rows == 32) go(attention_rows_kernel<DT, D, I8, 2>);
        else                            go(attention_rows_kernel<DT, D, I8, 4>);
    };
    auto by_format = [&](auto dtv, auto dimv) {
        if (int8) with(dtv, dimv, std::true_type{});
        else      with(dtv, dimv, std::false_type{});
    };
    auto by_dim = [&](auto dtv) {
        if (dim == 64) by_format(dtv, std::integral_constant<int, 64>{});
        else           by_format(dtv, std::integral_constant<int, 128>{});
    };
    if (dt == SASQ_F16) by_dim(std::integral_constant<int, SASQ_F16>{});
    else                by_dim(std::integral_constant<int, SASQ_BF16>{});
    return hipGetLastError() == hipSuccess ? SASQ_OK : SASQ_ERR_LAUNCH;
}

}  // namespace sasq
