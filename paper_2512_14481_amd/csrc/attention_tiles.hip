// Attention of many rows over the paged cache (chunks and prompts): bound by the matrix units and the exponentials beside them.
//
// A workgroup has one kv head of one sequence, 64 RB rows of it (its four waves 16 RB each, the heads that share the kv head packed into
// the rows) and one run of keys, which it takes in tiles of 64 through rings of four stages in LDS for K and for V.
//
// Both products are taken transposed on 16x16x32 (see attention_rows.hip), a lane keeps one row of each block of 16 from the scores to the
// output, and each fragment of K or V that a wave reads from LDS serves RB products.  The scores of the next tile take the registers of
// this one's as these become probabilities, 16 keys after 16, so that products and exponentials stand side by side.
#include "attention.h"

#ifndef SCHED_A
#define SCHED_A 4
#endif
#ifndef SASQ_RB
#define SASQ_RB 2
#endif
namespace sasq {

constexpr int kTileKeys = 64, kTileRing = 4;

template <int D, bool I8, int W>
struct TilesGeo : KvRow<D, I8> {
    using K = KvRow<D, I8>;
    static constexpr int kTile = 4 * K::k16;     // bytes of a tile's keys, or of its values
    static constexpr int kKeysAt = 0, kValuesAt = kTileRing * kTile, kPagesAt = 2 * kTileRing * kTile;
    static constexpr int kFlagsAt = kPagesAt + W * 2 * 64 * 4;
    static constexpr int kLds = kFlagsAt + 64;
};

template <int DTQ, int D, bool I8, int RB, int W>
__global__ __launch_bounds__(W * 64, W / 4) void attention_tiles_kernel(AttnArgs a, KvPages cache, KvSteps steps, AttnSplit split, int few, int first)
{
    using G = TilesGeo<D, I8, W>;
    constexpr int DT = I8 ? SASQ_F16 : DTQ;
    constexpr int DS = D / 32, DO = D / 16, KT = kTileKeys / 16;
    constexpr int L = G::kLoads;
    __shared__ __attribute__((aligned(1024))) char lds[G::kLds];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int l16 = lane & 15, g = lane >> 4;

    // The tiles of a sequence's last rows see the most keys: they come first.
    int rest = (int)blockIdx.x + first;
    const int hk = rest % cache.heads; rest /= cache.heads;
    const int b = rest % steps.batch; rest /= steps.batch;
    const int run = rest % split.splits, tile = split.tiles - 1 - rest / split.splits;
    const KvSeq seq = kv_seq(steps, b, cache.page_shift);
    const int rows = seq.rows * a.group, row0 = tile * 16 * RB * W;
    if (rows <= few || row0 >= rows) return;
    const int end = attn_end(seq, a.group, split, tile), runs = attn_runs(split, end);
    if (run >= runs) return;
    const int from = run * split.chunk, to = run == runs - 1 ? end : min(end, from + split.chunk);
    const int tiles = (to - from + kTileKeys - 1) / kTileKeys;
    const int past = seq.keys - seq.rows;
    const int sees_group = past + row0 / a.group;                          // last key of the workgroup's first row, of the wave's, of the wave's last row
    const int wave_row = row0 + 16 * RB * wave;
    const int sees_wave = past + wave_row / a.group;
    const int wave_end = past + (min(rows, wave_row + 16 * RB) - 1) / a.group + 1;
    const int wave_tiles = wave_row < rows ? min(tiles, max(0, (wave_end - from + kTileKeys - 1) / kTileKeys)) : 0;

    int sees[RB];
    float c[RB];
    u32x4 q[RB][DS];
    const float k_scale = I8 ? cache.k_scale[hk] : 1.0f;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = wave_row + 16 * rb + l16;
        const bool there = r < rows;
        const int token = (there ? r : row0) / a.group, head = (there ? r : row0) % a.group;
        sees[rb] = past + token;
        load_q<DTQ, D, I8>(a, a.q + (int64_t)(seq.row0 + token) * a.q_stride + (int64_t)(hk * a.group + head) * D, there, g, k_scale, q[rb], c[rb]);
    }

    // A page that is not there makes every tile of the run a masked one (a rare thing: no list of which).
    const int* const table = steps.table + (int64_t)b * steps.max_pages;
    bool hole = false;
    for (int u = (from >> cache.page_shift) + (int)threadIdx.x; u <= (to - 1) >> cache.page_shift; u += W * 64)
        hole |= u >= steps.max_pages || kv_page(cache, steps, b, u) < 0;
    const bool holes = __builtin_amdgcn_readfirstlane(__syncthreads_or(hole));
    auto there_is = [&](int i, int unit) -> bool {                         // keys 16 unit .. of tile i
        const int key = from + kTileKeys * i + 16 * unit;
        if (key >= to) return false;
        if (!holes) return true;
        const int index = key >> cache.page_shift;
        return index < steps.max_pages && kv_page(cache, steps, b, index) >= 0;
    };

    // Wave w brings unit w % 4 (16 keys) of every tile, of eight waves the first four of K and the others of V.  The pages of its next 64 tiles lie in a list of its own, the ones after them in another;
    // loads return in order, so a list has long landed when its first entry is read.
    const int unit = wave & 3;
    const bool brings_k = W == 4 || wave < 4, brings_v = W == 4 || wave >= 4;
    int* const list = reinterpret_cast<int*>(lds + G::kPagesAt) + wave * 128;
    const uint32_t lds_at = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
    const uint32_t list_at = lds_at + G::kPagesAt + wave * 512;
    auto fetch_list = [&](int n) {                                         // of tiles 64 n and on
        const int64_t key = (int64_t)from + kTileKeys * (64 * (int64_t)n + lane) + 16 * unit;
        const int64_t index = min(key >> cache.page_shift, (int64_t)steps.max_pages - 1);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" :: "s"(list_at + (n & 1) * 256), "v"((uint32_t)(4 * index)), "s"(table) : "memory");
    };
    uint32_t off[L];
#pragma unroll
    for (int j = 0; j < L; ++j) off[j] = G::source(j, lane, cache.token_stride);
    auto page_of = [&](int i) -> int { return list[i & 127]; };
    auto fetch = [&](int i, int page, const uint8_t* plane, int at) {       // the wave's unit of tile i, which lies on `page`
        page = __builtin_amdgcn_readfirstlane(page);
        const int place = (from + kTileKeys * i + 16 * unit) & ((1 << cache.page_shift) - 1);
        const uint8_t* base = plane + (int64_t)hk * cache.head_stride + (page < 0 || page >= cache.pages ? 0 : page * cache.page_stride + place * cache.token_stride);
        const uint32_t to_lds = lds_at + at + unit * G::k16;
#pragma unroll
        for (int j = 0; j < L; ++j) load_to_lds(to_lds + G::kBlock * j, base, off[j]);
    };
    auto fetch_keys = [&](int i, int page) { fetch(i, page, cache.k, G::kKeysAt + i % kTileRing * G::kTile); };
    auto fetch_values = [&](int i, int page) { fetch(i, page, cache.v, G::kValuesAt + i % kTileRing * G::kTile); };
    auto keys_at = [&](int i) -> const char* { return lds + G::kKeysAt + i % kTileRing * G::kTile; };
    auto values_at = [&](int i) -> char* { return lds + G::kValuesAt + i % kTileRing * G::kTile; };

    f32x4 o[RB][DO];
    float m[RB], l[RB];                                                    // maximum of the log2-scaled scores, sum
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m[rb] = kNoMax; l[rb] = 0.0f;
#pragma unroll
        for (int n = 0; n < DO; ++n) o[rb][n] = f32x4{0, 0, 0, 0};
    }
    f32x4 s[RB][KT];
    u32x4 p[RB][KT / 2];
    constexpr int KF = I8 ? DS / 2 : DS;                                   // fragments of 16 keys
    typedef u32x4 KeyFrags[KF];
    typedef u32x4 ValueFrags[4];
    auto read_keys = [&](int i, int k, KeyFrags& w) {                      // keys 16 k .. of tile i
        const char* at = keys_at(i) + G::key_lane(lane) + k * G::k16;
#pragma unroll
        for (int t = 0; t < KF; ++t) w[t] = G::key(at, t);
    };
    auto scores = [&](int k, const KeyFrags& w) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) s[rb][k] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < KF; ++t) {
            if constexpr (I8) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const u32x2 x = codes_to_f16(w[t][2 * e]), y = codes_to_f16(w[t][2 * e + 1]);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) s[rb][k] = mfma16<DT>(u32x4{x[0], x[1], y[0], y[1]}, q[rb][2 * t + e], s[rb][k]);
                }
            } else {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) s[rb][k] = mfma16<DT>(w[t], q[rb][t], s[rb][k]);
            }
        }
    };
    auto unmasked = [&](int i) -> bool { return !holes && from + kTileKeys * i + kTileKeys - 1 <= sees_wave; };
    auto mask = [&](int i) {
        const int k0 = from + kTileKeys * i;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int last = sees[rb] - k0 - 4 * g;                        // of the lane's keys, 0 being its first
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (16 * k + j > last) s[rb][k][j] = -INFINITY;
        }
        if (holes) {
#pragma unroll
            for (int k = 0; k < KT; ++k)
                if (!there_is(i, k)) {
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) s[rb][k] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                }
        }
    };
    float top[RB];
    auto maxima = [&]() -> bool {                                          // whether a score passes the running maximum by too much
        bool above = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            top[rb] = s[rb][0][0];
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) top[rb] = fmaxf(top[rb], s[rb][k][j]);
            above |= __builtin_fmaf(top[rb], c[rb], -m[rb]) > kLazy;
        }
        return __any(above);
    };
    auto raise = [&]() {                                                   // moves the maxima, and the sums with them
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float t = fmaxf(top[rb], __shfl_xor(top[rb], 16, kWave));
            t = fmaxf(t, __shfl_xor(t, 32, kWave));
            t = fmaxf(t * c[rb], m[rb]);
            const float keep = kept(m[rb], t);
            m[rb] = t;
            l[rb] *= keep;
#pragma unroll
            for (int n = 0; n < DO; ++n) o[rb][n] *= keep;
        }
    };
    auto probabilities = [&](int k) {                                      // of keys 16 k ..
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][k][j], c[rb], -m[rb]));
            l[rb] += (e[0] + e[1]) + (e[2] + e[3]);
            p[rb][k / 2][2 * (k & 1)] = Store16<DT>::pack(e[0], e[1]);
            p[rb][k / 2][2 * (k & 1) + 1] = Store16<DT>::pack(e[2], e[3]);
        }
    };
    constexpr int VG = KT / 2 * DO / 4;                                    // groups of four fragments of a tile's values: 64 channels of 32 keys
    auto read_values = [&](int i, int x, ValueFrags& w) {
        const char* at = values_at(i) + G::value_lane(lane) + 2 * (x / (DO / 4)) * G::k16;
#pragma unroll
        for (int n = 0; n < 4; ++n) w[n] = G::value(at, 4 * (x % (DO / 4)) + n);
    };
    auto add_values = [&](int x, const ValueFrags& w) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) o[rb][4 * (x % (DO / 4)) + n] = mfma16<DT>(w[n], p[rb][x / (DO / 4)], o[rb][4 * (x % (DO / 4)) + n]);
    };
    // A masked place may hold anything, and 0 times infinity is not 0: in a masked tile with infinities or NaN among its values these are
    // put into the rows that see them by hand, and taken out of the tile.
    int* const flags = reinterpret_cast<int*>(lds + G::kFlagsAt);
    auto masked_group = [&](int i) -> bool { return holes || from + kTileKeys * i + kTileKeys - 1 > sees_group; };
    auto own_values = [&](int i) -> u32x4* { return reinterpret_cast<u32x4*>(values_at(i) + unit * G::k16); };
    auto look_for_specials = [&](int i) {
        bool special = false;
#pragma unroll
        for (int j = 0; j < L; ++j) {
            const u32x4 w = own_values(i)[G::kBlock / 16 * j + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) special |= any_special<DT>(w[e]);
        }
        const bool any = __any(special);
        if (lane == 0) flags[(i & 1) * 4 + unit] = any;
    };
    auto take_specials_out = [&](int i) {
        const int k0 = from + kTileKeys * i;
        if (i < wave_tiles) {
#pragma unroll
            for (int k = 0; k < KT / 2; ++k) {
                const bool there[2] = {there_is(i, 2 * k), there_is(i, 2 * k + 1)};
                u32x4 seen[RB];
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int key = k0 + 32 * k + (j < 2 ? 0 : 16) + 4 * g + 2 * (j & 1);
                        seen[rb][j] = (there[j >> 1] && key <= sees[rb] ? kSeen : 0u) | (there[j >> 1] && key + 1 <= sees[rb] ? kSeen << 16 : 0u);
                    }
#pragma unroll
                for (int n = 0; n < DO; ++n) {
                    const u32x4 v = G::value(values_at(i) + G::value_lane(lane) + 2 * k * G::k16, n);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) o[rb][n] = add_specials<DT>(v, seen[rb], o[rb][n]);
                }
            }
        }
        __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (brings_v) {
#pragma unroll
            for (int j = 0; j < L; ++j) {
                u32x4 w = own_values(i)[G::kBlock / 16 * j + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = finite_of<DT>(w[e]);
                own_values(i)[G::kBlock / 16 * j + lane] = w;
            }
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    int ahead_k = 0, ahead_v = 0;                                          // pages of tiles i + 4 (keys) and i + 3 (values), read a tile before
    auto enter = [&](int i) {                                              // the workgroup goes on to tile i
        // In order: of four waves, K(i+2) V(i+1) have landed when at most V(i+2) and K(i+3) are still under way; of eight each has one of them.
        if (i + 3 < tiles) wait_loads<(W == 4 ? 2 : 1) * L>();
        else               wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (i + 4 < tiles && ((i + 4) & 63) == 0) fetch_list((i + 4) / 64 + 1);
        if (brings_k && i + 4 < tiles) fetch_keys(i + 4, ahead_k);
        if (brings_v && i + 3 < tiles) fetch_values(i + 3, ahead_v);
        ahead_v = W == 4 ? ahead_k : page_of(i + 4);
        ahead_k = page_of(i + 5);
        if (!I8 && masked_group(i)) {
            if (brings_v) look_for_specials(i);
            __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            const int* f = flags + (i & 1) * 4;
            if (__builtin_amdgcn_readfirstlane(f[0] | f[1] | f[2] | f[3])) take_specials_out(i);
        }
    };
    constexpr int kMfma = 0x8, kValu = 0x2;
    KeyFrags kf;                                                           // of the first 16 keys of the next tile, read ahead of the barrier
    bool above = false;
    auto work = [&](int i) {
        if (above) raise();
        probabilities(0);
        ValueFrags vf;
        if (i + 1 < wave_tiles) {
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                KeyFrags next;
                if (k + 1 < KT) read_keys(i + 1, k + 1, next);
                else            read_values(i, 0, vf);
                __builtin_amdgcn_sched_barrier(0);                         // the reads of the next products stand ahead of these
                scores(k, kf);
                if (k + 1 < KT) {
                    probabilities(k + 1);
#pragma unroll
                    for (int x = 0; x < RB * DS; ++x) {
                        __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(kValu, SCHED_A, 0);
                    }
#pragma unroll
                    for (int t = 0; t < KF; ++t) kf[t] = next[t];
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (!unmasked(i + 1)) mask(i + 1);
        } else {
#pragma unroll
            for (int k = 1; k < KT; ++k) probabilities(k);
            read_values(i, 0, vf);
        }
#pragma unroll
        for (int x = 0; x < VG; ++x) {
            ValueFrags next;
            if (x + 1 < VG) read_values(i, x + 1, next);
            else            read_keys(i + 2, 0, kf);
            __builtin_amdgcn_sched_barrier(0);
            add_values(x, vf);
            if (x == 0) above = maxima();                                  // (of the last tile's scores again after the last tile: never above)
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < 4; ++n) vf[n] = next[n];
        }
    };

    if (tiles > 0) {
        fetch_list(0);
        fetch_list(1);
        wait_loads<0>();                                                   // Q too: the loop's waits count the rings' loads alone
        for (int i = 0; i < 4 && i < tiles; ++i) {
            if (brings_k) fetch_keys(i, page_of(i));
            if (brings_v && i < 3) fetch_values(i, page_of(i));
        }
        ahead_k = page_of(4);
        ahead_v = page_of(3);
        if (tiles > 3) wait_loads<(W == 4 ? 4 : 2) * L>();
        else           wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (wave_tiles > 0) {
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                read_keys(0, k, kf);
                scores(k, kf);
            }
            if (!unmasked(0)) mask(0);
            if (maxima()) raise();
            read_keys(1, 0, kf);
        }
        for (int i = 0; i < tiles; ++i) {
            enter(i);
            if (i < wave_tiles) work(i);
        }
    }

    const float v_scale = I8 ? cache.v_scale[hk] : 1.0f;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float sum = l[rb];
        sum += __shfl_xor(sum, 16, kWave);
        sum += __shfl_xor(sum, 32, kWave);
        const int r = wave_row + 16 * rb + l16;
        if (r >= rows) continue;
        const int64_t t = seq.row0 + r / a.group, head = hk * a.group + r % a.group;
        const float top = m[rb] == kNoMax ? -INFINITY : m[rb];
        if (runs == 1) {
            const bool none = sum == 0.0f;
            const float f = none ? 0.0f : v_scale / sum;
            uint16_t* dst = a.out + t * a.out_stride + head * D + 4 * g;
#pragma unroll
            for (int n = 0; n < DO; ++n) {
                const f32x4 x = o[rb][n];
                const u32x2 w = {none ? 0u : Store16<DTQ>::pack(x[0] * f, x[1] * f), none ? 0u : Store16<DTQ>::pack(x[2] * f, x[3] * f)};
                *reinterpret_cast<u32x2*>(dst + 16 * n) = w;
            }
            if (a.lse && g == 0) a.lse[t * a.q_heads + head] = none ? -INFINITY : (top + log2f(sum)) * 0.693147180559945f;
        } else {
            const int64_t slot = tiles_slot(steps.tokens, a.q_heads, run, (int)t, (int)head);
            float* dst = split.o + slot * D + 4 * g;
#pragma unroll
            for (int n = 0; n < DO; ++n) *reinterpret_cast<f32x4*>(dst + 16 * n) = o[rb][n];
            if (g == 0) split.ml[slot] = make_float2(top, sum);
        }
    }
}

int attention_tiles_launch(const AttnArgs& a, const KvPages& c, const KvSteps& s, const AttnSplit& split, int few, int dim, bool int8, sasq_dtype dt, hipStream_t st)
{
    auto go = [&](auto kernel, int threads) {
        launch_in_parts((int64_t)split.splits * s.batch * split.tiles * c.heads, threads,
                        [&](unsigned n, int first) { hipLaunchKernelGGL(kernel, dim3(n), dim3(threads), 0, st, a, c, s, split, few, first); });
    };
    auto with = [&](auto dtv, auto dimv, auto i8v) {
        constexpr int DT = decltype(dtv)::value, D = decltype(dimv)::value;
        constexpr bool I8 = decltype(i8v)::value;
        if (split.tile_rows == 128) go(attention_tiles_kernel<DT, D, I8, 2, 4>, 256);
        else                        go(attention_tiles_kernel<DT, D, I8, SASQ_RB, 16 / SASQ_RB>, 1024 / SASQ_RB);
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
