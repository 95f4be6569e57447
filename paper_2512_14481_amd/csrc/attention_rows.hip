// Attention of few rows over the paged cache (single tokens, drafts): bound by the bytes of the cache.
//
// A workgroup has one kv head of one sequence, up to 16 rows of it (its new tokens times the query heads that share the kv head), and one run
// of keys; its four waves take slabs of 32 keys in turn, each with its own running maximum, sum and output, joined at the end.  A wave
// streams its slabs through a ring of two stages of its own in LDS (direct global-to-LDS loads, no barrier in the loop): while one slab is
// worked on the other is under way, and each half of a stage is asked for again as soon as its last reader is done.
//
// Products are taken transposed, so that a lane keeps one row from the scores to the output:
//   S^T[key, row] = K Q^T     16x16x32: lane (row = l % 16, g = l / 16) gets keys 4g..4g+3 of each 16
//   O^T[d, row]  += V^T P^T   the eight keys of a lane's slots are then the ones it has scores of (4g + j of both halves of the slab):
//                             the probabilities go into the second product as they come out of the first, and V is read
//                             transposed by ds_read_tr with the same order of keys.
// Fifteen of sixteen rows of the matrix units' work are idle with one row; they still have it done long before the next slab is there.
//
// Measured, with the join where there is one: 48 sequences of 70B with 200 to 8190 keys 101 us (4.3 TB/s; a large copy reaches 4.8), 32 of 13B in
// int8 142 us (4.5), two of 120000 to 131000 keys of 70B in int8 95 us (5.5); one of 301 keys of 7B 9.2 us, the time of its waits one after
// another (lengths, pages, keys, join).  Three blocks of 16 rows a wave in place of the other kernel for 17 to 48 rows: no better in int8
// (45 us against 44 for 16 times five tokens), 64 against 41 in 16 bits.
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

template <int DTQ, int D, bool I8>
__global__ __launch_bounds__(kRowWaves * 64, I8 ? 2 : 1) void attention_rows_kernel(AttnArgs a, KvPages cache, KvSteps steps, AttnSplit split, int first)
{
    using G = RowsGeo<D, I8>;
    constexpr int DT = I8 ? SASQ_F16 : DTQ;               // of the products
    constexpr int DS = D / 32, DO = D / 16;               // steps over d of the first product, blocks of d of the second
    __shared__ __attribute__((aligned(1024))) char lds[G::kLds];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int l16 = lane & 15, g = lane >> 4;

    int rest = (int)blockIdx.x + first;
    const int hk = rest % cache.heads; rest /= cache.heads;
    const int b = rest % steps.batch, run = rest / steps.batch;
    // The first segment's pages, asked for together with the lengths that say how many of them count.
    const int from = run * split.chunk, unit = (int)threadIdx.x;
    auto page_of_unit = [&](int seg) -> int {
        const int index = (int)(((int64_t)seg + 16 * unit) >> cache.page_shift);
        return unit < kSegment / 16 && index < steps.max_pages ? kv_page(cache, steps, b, index) : -1;
    };
    int listed = page_of_unit(from);
    const KvSeq seq = kv_seq(steps, b, cache.page_shift);
    const int rows = seq.rows * a.group;
    if (rows == 0 || rows > kFewRows) return;
    const int end = attn_end(seq, a.group, split, 0), runs = attn_runs(split, end);
    if (run >= runs) return;
    const int to = run == runs - 1 ? end : min(end, from + split.chunk);
    const int past = kv_last(seq, 0);                                      // the first row's last key: masks begin after it

    const bool row_there = l16 < rows;
    const int my_token = (row_there ? l16 : 0) / a.group, my_head = hk * a.group + (row_there ? l16 : 0) % a.group;
    const int sees = kv_last(seq, my_token);
    float c;
    u32x4 q[DS];
    load_q<DTQ, D, I8>(a, a.q + (int64_t)(seq.row0 + my_token) * a.q_stride + (int64_t)my_head * D, row_there, g, I8 ? cache.k_scale[hk] : 1.0f, q, c);

    uint32_t off[G::kLoads];
#pragma unroll
    for (int j = 0; j < G::kLoads; ++j) off[j] = G::source(j, lane, cache.token_stride);
    char* const ring = lds + wave * kRing * G::kStage;
    const uint32_t ring_at = (uint32_t)(uintptr_t)(lds_ptr_t)ring;
    int* const pages = reinterpret_cast<int*>(lds + G::kBody + kRowWaves * 16 * 8);

    f32x4 o[DO];
    float m = kNoMax, l = 0.0f;                                            // maximum of the log2-scaled scores, sum
#pragma unroll
    for (int n = 0; n < DO; ++n) o[n] = f32x4{0, 0, 0, 0};

    for (int seg = from; seg < to; seg += kSegment) {
        const int seg_end = min(to, seg + kSegment);
        if (seg != from) {
            __syncthreads();
            listed = page_of_unit(seg);
        }
        if (unit < kSegment / 16) pages[unit] = listed;
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
                for (int j = 0; j < G::kLoads; ++j) load_to_lds_once(at + (h * G::kLoads + j) * G::kBlock, base, off[j]);
            }
        };
        wait_loads<0>();                                                   // Q has landed: the loop's waits count the ring's loads alone
        constexpr int NL = 2 * G::kLoads;                                  // loads of a slab's keys, or of its values
        for (int i = 0; i < kRing && i < mine; ++i) { fetch(i, cache.k, 0); fetch(i, cache.v, 1); }
        for (int i = 0; i < mine; ++i) {
            const char* stage = ring + (i % kRing) * G::kStage;
            const char* kp = stage + G::key_lane(lane);
            const char* vp = stage + G::kPart + G::value_lane(lane);
            const int k0 = seg + kSlab * (wave + i * kRowWaves);
            if (i + 1 < mine) wait_loads<3 * NL>();
            else              wait_loads<NL>();
            f32x4 s[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
#pragma unroll
            for (int t = 0; t < (I8 ? DS / 2 : DS); ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const u32x4 w = G::key(kp + h * G::k16, t);
                    if constexpr (I8) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const u32x2 lo = codes_to_f16(w[2 * e]), hi = codes_to_f16(w[2 * e + 1]);
                            s[h] = mfma16<DT>(u32x4{lo[0], lo[1], hi[0], hi[1]}, q[2 * t + e], s[h]);
                        }
                    } else {
                        s[h] = mfma16<DT>(w, q[t], s[h]);
                    }
                }
            const int page0 = page_of(i, 0), page1 = page_of(i, 1);
            __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
            asm volatile("" ::: "memory");
            if (i + kRing < mine) fetch(i + kRing, cache.k, 0);

            const bool masked = k0 + kSlab - 1 > past || page0 < 0 || page1 < 0;
            if (masked) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (page0 < 0 || k0 + 4 * g + j > sees) s[0][j] = -INFINITY;
                    if (page1 < 0 || k0 + 16 + 4 * g + j > sees) s[1][j] = -INFINITY;
                }
            }
            float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
            if (__any(top * c - m > Lazy<DT>::most)) {
                top = fmaxf(top, __shfl_xor(top, 16, kWave));
                top = fmaxf(top, __shfl_xor(top, 32, kWave));
                const float now = fmaxf(top * c - Lazy<DT>::below, m), keep = kept(m, now);
                m = now;
                l *= keep;
#pragma unroll
                for (int n = 0; n < DO; ++n) o[n] *= keep;
            }
            float e[8];
            u32x4 p;
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = __builtin_amdgcn_exp2f(s[j >> 2][j & 3] * c - m);      // the product rounded as in m (kExact); bound by bytes
            l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
#pragma unroll
            for (int j = 0; j < 4; ++j) p[j] = Store16<DT>::pack(e[2 * j], e[2 * j + 1]);

            if (i + kRing < mine)    wait_loads<3 * NL>();
            else if (i + 1 < mine)   wait_loads<2 * NL>();
            else                     wait_loads<0>();
            u32x4 v[DO];
#pragma unroll
            for (int n = 0; n < DO; ++n) v[n] = G::value(vp, n, G::value_odd(lane));
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
                        u32x4 seen;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int key = k0 + (j < 2 ? 0 : 16) + 4 * g + 2 * (j & 1);
                            const bool there = (j < 2 ? page0 : page1) >= 0;
                            seen[j] = (there && key <= sees ? kSeen : 0u) | (there && key + 1 <= sees ? kSeen << 16 : 0u);
                        }
#pragma unroll
                        for (int n = 0; n < DO; ++n) o[n] = add_specials<DT>(v[n], seen, o[n]);
#pragma unroll
                        for (int n = 0; n < DO; ++n)
#pragma unroll
                            for (int j = 0; j < 4; ++j) v[n][j] = finite_of<DT>(v[n][j]);
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < DO; ++n) o[n] = mfma16<DT>(v[n], p, o[n]);
            __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
            asm volatile("" ::: "memory");
            if (i + kRing < mine) fetch(i + kRing, cache.v, 1);
        }
    }

    // Join the waves: sixteen threads for a row.
    constexpr int E = D / 16;
    float* const part = reinterpret_cast<float*>(lds);                     // [wave][row][D + 4]
    float2* const ml = reinterpret_cast<float2*>(lds + G::kBody);          // [wave][row]
    __syncthreads();
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    if (g == 0) ml[wave * 16 + l16] = make_float2(l == 0.0f ? -INFINITY : m, l);
#pragma unroll
    for (int n = 0; n < DO; ++n) *reinterpret_cast<f32x4*>(part + (wave * 16 + l16) * (D + 4) + 16 * n + 4 * g) = o[n];
    __syncthreads();
    const int r = (int)threadIdx.x / 16, d = (int)threadIdx.x % 16 * E;
    if (r >= rows) return;
    float top = -INFINITY, sum = 0.0f, x[E];
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) top = fmaxf(top, ml[w * 16 + r].x);
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = 0.0f;
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) {
        const float2 f = ml[w * 16 + r];
        const float weight = part_weight(f, top);
        sum += f.y * weight;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = __builtin_fmaf(part[(w * 16 + r) * (D + 4) + d + e], weight, x[e]);
    }
    const int token = r / a.group, head = hk * a.group + r % a.group;
    if (runs == 1) {
        const bool none = sum == 0.0f;
        const float f = none ? 0.0f : 1.0f / sum, v = I8 ? cache.v_scale[hk] : 1.0f;       // (apart: a small factor over a large sum may be no number of fp32's)
        uint16_t* dst = a.out + (int64_t)(seq.row0 + token) * a.out_stride + (int64_t)head * D + d;
        uint32_t w[E / 2];
#pragma unroll
        for (int e = 0; e < E / 2; ++e) w[e] = none ? 0u : Store16<DTQ>::pack(x[2 * e] * f * v, x[2 * e + 1] * f * v);
        __builtin_memcpy(dst, w, sizeof(w));
        if (a.lse && d == 0) a.lse[(int64_t)(seq.row0 + token) * a.q_heads + head] = none ? -INFINITY : (top + log2f(sum)) * 0.693147180559945f;
    } else {
        const int64_t slot = few_slot(split, steps.batch, cache.heads, run, b, hk, r);
        float* dst = split.o + slot * D + d;
#pragma unroll
        for (int e = 0; e < E; e += 4) *reinterpret_cast<f32x4*>(dst + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
        if (d == 0) split.ml[slot] = make_float2(top, sum);
    }
}

int attention_rows_launch(const AttnArgs& a, const KvPages& c, const KvSteps& s, const AttnSplit& split, int dim, bool int8, sasq_dtype dt, hipStream_t st)
{
    auto go = [&](auto kernel) {
        launch_in_parts((int64_t)split.splits * s.batch * c.heads, kRowWaves * 64,
                        [&](unsigned n, int first) { hipLaunchKernelGGL(kernel, dim3(n), dim3(kRowWaves * 64), 0, st, a, c, s, split, first); });
    };
    auto by_format = [&](auto dtv, auto dimv) {
        if (int8) go(attention_rows_kernel<decltype(dtv)::value, decltype(dimv)::value, true>);
        else      go(attention_rows_kernel<decltype(dtv)::value, decltype(dimv)::value, false>);
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
