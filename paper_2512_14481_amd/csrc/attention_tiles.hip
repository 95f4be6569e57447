// Attention of many rows over the paged cache (chunks and prompts): bound by the matrix units and the exponentials beside them.
//
// A workgroup has one kv head of one sequence, 128 rows of it (RB = 2 blocks of 16 for each of its four waves, the heads that share the kv head
// packed into the rows) and one run of keys, which it takes in tiles of 64 through two stages in LDS for K and two for V.  Two workgroups
// share a CU: one's waves have products for the matrix units while the other's wait.  Where no sequence of the call has more than 64 rows
// (drafts, short prompts) a tile has 64 and a wave one block: five tokens for each of 16 of 70B on 500 to 4000 keys in int8 37 us, with
// 128 rows, of which two waves have none, 44; one prompt of 40 tokens on 300 of 7B 11.4 and 14.3.
//
// Both products are taken transposed (see attention_rows.hip), a lane keeps one row of each block of 16 from the scores to the output, and what a
// wave reads of K or V from LDS serves RB products.  The scores of the next tile take the registers of this one's, 16 keys after 16, as these
// become probabilities; what a product reads from LDS is read before the products ahead of it, the loads of the tiles to come are dealt out
// among them, and a tile is one block of instructions without a branch (but for masks, which only a run's last tiles have), so that products,
// exponentials, reads and loads stand side by side.
//
// Measured: a chunk of 4096 tokens on 12281 of 70B 1.69 to 1.81 ms by card (1.14 to 1.06 PFLOP/s; the library's largest product reaches 1.59); on the
// card with 1.69, 1.79 on 32x32x16, 1.74 with eight waves and 256 rows a workgroup on it: the card is at its power limit (1.8 to 2.1 GHz of 2.4),
// where the 16x16 form gives more.  On an int8 cache 2.27 where it is 1.74 in 16 bits: each wave turns the codes of the whole tile to fp16.
#include "attention.h"

namespace sasq {

constexpr int kTileKeys = 64, kTileWaves = 4;

template <int D, bool I8>
struct TilesGeo : KvRow<D, I8> {
    using K = KvRow<D, I8>;
    static constexpr int kTile = 4 * K::k16;     // bytes of a tile's keys, or of its values
    static constexpr int kKeysAt = 0, kValuesAt = 2 * kTile, kFlagsAt = 4 * kTile;
    static constexpr int kLds = kFlagsAt + 64;
};

template <int DTQ, int D, bool I8, int RB>
__global__ __launch_bounds__(kTileWaves * 64, RB == 1 && I8 ? 3 : 2) void attention_tiles_kernel(AttnArgs a, KvPages cache, KvSteps steps, AttnSplit few, AttnSplit many, int many_blocks, int first)
{
    using G = TilesGeo<D, I8>;
    constexpr int DT = I8 ? SASQ_F16 : DTQ;
    constexpr int R = 16, Rows = R * RB * kTileWaves, DS = D / 32, DO = D / 16, KB = kTileKeys / 16;   // blocks of 16 rows of a wave; steps of the first product; blocks of 16 channels, of 16 keys
    constexpr int L = G::kLoads;
    __shared__ __attribute__((aligned(1024))) char lds[G::kLds];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int l16 = lane & 15, g = lane >> 4;

    // First the tiles of sequences of many rows, the last rows (which see the most keys) first, then the sequences of few rows.
    int rest = (int)blockIdx.x + first;
    const bool is_few = rest >= many_blocks;
    if (is_few) rest -= many_blocks;
    const AttnSplit split = is_few ? few : many;
    const int hk = rest % cache.heads; rest /= cache.heads;
    int b, run, tile;
    if (is_few) {
        b = rest % steps.batch;
        run = rest / steps.batch;
        tile = 0;
    } else {
        run = rest % split.splits;
        rest /= split.splits;
        // Tile `rest` from the end: the wave adds up the tiles of 64 sequences at a time, from the last one on.
        bool found = false;
        for (int i = 0; i < steps.batch && !found; i += kWave) {
            const int at = steps.batch - 1 - i - lane;
            int n = 0;
            if (at >= 0) {
                const int of = kv_seq(steps, at, cache.page_shift).rows * a.group;
                n = of > kFewRows ? (of + Rows - 1) / Rows : 0;
            }
            int sum = n;
#pragma unroll
            for (int d = 1; d < kWave; d <<= 1) {
                const int below = __shfl_up(sum, d, kWave);
                if (lane >= d) sum += below;
            }
            const uint64_t past_it = __ballot(rest < sum);
            if (past_it) {
                const int where = __ffsll((unsigned long long)past_it) - 1;
                found = true;
                b = steps.batch - 1 - i - where;
                tile = __builtin_amdgcn_readlane(sum, where) - 1 - rest;
            } else {
                rest -= __builtin_amdgcn_readlane(sum, kWave - 1);
            }
        }
        if (!found) return;
        b = __builtin_amdgcn_readfirstlane(b);
        tile = __builtin_amdgcn_readfirstlane(tile);
    }
    const KvSeq seq = kv_seq(steps, b, cache.page_shift);
    const int rows = seq.rows * a.group, row0 = tile * Rows;
    if (rows == 0 || (rows <= kFewRows) != is_few) return;
    const int end = attn_end(seq, a.group, split, tile), runs = attn_runs(split, end);
    if (run >= runs) return;
    const int from = run * split.chunk, to = run == runs - 1 ? end : min(end, from + split.chunk);
    const int tiles = (to - from + kTileKeys - 1) / kTileKeys;
    const int sees_group = kv_last(seq, row0 / a.group);                        // last key of the workgroup's first row, of the wave's, of the wave's last row
    const int wave_row = row0 + R * RB * wave;
    const int sees_wave = kv_last(seq, wave_row / a.group);
    const int wave_end = kv_last(seq, (min(rows, wave_row + R * RB) - 1) / a.group) + 1;
    const int wave_tiles = wave_row < rows ? min(tiles, max(0, (wave_end - from + kTileKeys - 1) / kTileKeys)) : 0;

    // The lane's rows.
    int sees[RB];
    float c[RB];
    u32x4 q[RB][DS];
    auto token_of = [&](int rb) -> int { return (wave_row + R * rb + l16) / a.group; };
    auto head_of = [&](int rb) -> int { return hk * a.group + (wave_row + R * rb + l16) % a.group; };
    auto row_there = [&](int rb) -> bool { return wave_row + R * rb + l16 < rows; };
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const bool there = row_there(rb);
        const int token = there ? token_of(rb) : row0 / a.group, head = there ? head_of(rb) : hk * a.group;
        sees[rb] = kv_last(seq, token);
        load_q<DTQ, D, I8>(a, a.q + (int64_t)(seq.row0 + token) * a.q_stride + (int64_t)head * D, there, g, I8 ? cache.k_scale[hk] : 1.0f, q[rb], c[rb]);
    }

    // A page that is not there makes every tile of the run a masked one (a rare thing: no list of which).
    bool holes = false;
    auto missing = [&]() -> bool {
        bool any = false;
        for (int u = (from >> cache.page_shift) + (int)threadIdx.x; u <= (to - 1) >> cache.page_shift; u += kTileWaves * 64)
            any |= u >= steps.max_pages || kv_page(cache, steps, b, u) < 0;
        return any;
    };
    auto there_is = [&](int i, int unit) -> bool {                         // keys 16 unit .. of tile i
        const int key = from + kTileKeys * i + 16 * unit;
        if (key >= to) return false;
        if (!holes) return true;
        const int index = key >> cache.page_shift;
        return index < steps.max_pages && kv_page(cache, steps, b, index) >= 0;
    };

    // Wave w brings unit w (16 keys) of every tile.  Where the unit of tile 64 n + t lies in either plane is lane t's to know.
    const int unit = wave;
    const uint32_t lds_at = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
    uint32_t off[L];
#pragma unroll
    for (int j = 0; j < L; ++j) off[j] = G::source(j, lane, cache.token_stride);
    int64_t lies;
    auto look_up = [&](int n) {
        const int64_t key = (int64_t)from + kTileKeys * (64 * (int64_t)n + lane) + 16 * unit;
        const int page = kv_page(cache, steps, b, (int)min(key >> cache.page_shift, (int64_t)steps.max_pages - 1));
        const int place = (int)key & ((1 << cache.page_shift) - 1);
        lies = hk * cache.head_stride + (page < 0 ? 0 : page * cache.page_stride + place * cache.token_stride);
    };
    auto lies_at = [&](int i) -> int64_t {
        const uint32_t lo = __builtin_amdgcn_readlane((int)lies, i & 63), hi = __builtin_amdgcn_readlane((int)(lies >> 32), i & 63);
        return (int64_t)((uint64_t)hi << 32 | lo);
    };
    struct Source {                                                        // the wave's unit of a tile: where it comes from and where it goes, if it is asked for
        const uint8_t* base;
        uint32_t to;
        int on;
    };
    auto source = [&](int i, int64_t at, const uint8_t* plane, int to) -> Source {
        return {plane + at, lds_at + to + (i & 1) * G::kTile + unit * G::k16, i < tiles ? -1 : 0};
    };
    auto fetch = [&](const Source& f, int j) { load_to_lds_if(f.on, f.to + G::kBlock * j, f.base, off[j]); };
    auto keys_at = [&](int i) -> const char* { return lds + G::kKeysAt + (i & 1) * G::kTile; };
    auto values_at = [&](int i) -> char* { return lds + G::kValuesAt + (i & 1) * G::kTile; };

    f32x4 o[RB][DO], s[RB][KB];
    float m[RB], l[RB];                                                    // maximum of the log2-scaled scores, sum
    u32x4 p[RB][KB / 2];                                                   // of 32 keys each
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m[rb] = kNoMax; l[rb] = 0.0f;
#pragma unroll
        for (int n = 0; n < DO; ++n) o[rb][n] = f32x4{0, 0, 0, 0};
    }

    // What is read from LDS goes in groups: the fragments of 16 keys; four fragments of 32 keys' values.
    constexpr int KF = I8 ? DS / 2 : DS, VG = KB / 2 * DO / 4;
    typedef u32x4 KeyFrags[KF];
    typedef u32x4 ValueFrags[4];
    auto read_keys = [&](int i, int k, KeyFrags& w) {                      // block k of tile i
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
                    const u32x2 lo = codes_to_f16(w[t][2 * e]), hi = codes_to_f16(w[t][2 * e + 1]);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) s[rb][k] = mfma16<DT>(u32x4{lo[0], lo[1], hi[0], hi[1]}, q[rb][2 * t + e], s[rb][k]);
                }
            } else {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) s[rb][k] = mfma16<DT>(w[t], q[rb][t], s[rb][k]);
            }
        }
    };
    // A wave that has met a score of kExact or more multiplies its scores by c ahead of everything else, and c is 1 from then on.  (Products rounded
    // in every tile: a chunk of 4096 on 12281 tokens 1846 us against 1803.)
    bool coarse = false;
    float by[RB];
    auto multiply = [&]() {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[rb][k][j] *= by[rb];
    };
    // Score j of block k is of key 16 k + 4 g + j.
    auto unmasked = [&](int i) -> bool { return !coarse && !holes && from + kTileKeys * i + kTileKeys - 1 <= sees_wave; };
    auto mask = [&](int i) {
        if (coarse) multiply();
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int last = sees[rb] - (from + kTileKeys * i) - 4 * g;    // of the lane's keys, 0 being its first
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (16 * k + j > last) s[rb][k][j] = -INFINITY;
        }
        if (holes) {
#pragma unroll
            for (int k = 0; k < KB; ++k)
                if (!there_is(i, k)) {
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) s[rb][k] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                }
        }
    };
    float top[RB];
    auto maxima = [&]() -> bool {                                          // whether a score passes the running maximum by too much
        bool passes = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            top[rb] = s[rb][0][0];
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) top[rb] = fmaxf(top[rb], s[rb][k][j]);
            passes |= __builtin_fmaf(top[rb], c[rb], -m[rb]) > Lazy<DT>::most;
        }
        return __any(passes);
    };
    auto raise = [&]() {                                                   // moves the maxima, and the sums with them
        bool large = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            top[rb] = fmaxf(top[rb], __shfl_xor(top[rb], 16, kWave));
            top[rb] = fmaxf(top[rb], __shfl_xor(top[rb], 32, kWave));
            large |= top[rb] > -INFINITY && fabsf(top[rb] * c[rb]) >= kExact;
        }
        if (!coarse && __any(large)) {
            coarse = true;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                by[rb] = c[rb];
                c[rb] = 1.0f;
                top[rb] *= by[rb];
            }
            multiply();
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const float t = fmaxf(top[rb] * c[rb] - Lazy<DT>::below, m[rb]);
            const float keep = kept(m[rb], t);
            m[rb] = t;
            l[rb] *= keep;
#pragma unroll
            for (int n = 0; n < DO; ++n) o[rb][n] *= keep;
        }
    };
    auto probabilities = [&](int k, float (&sum)[RB]) {                    // of block k, and their sums
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][k][j], c[rb], -m[rb]));
            sum[rb] = (e[0] + e[1]) + (e[2] + e[3]);
            p[rb][k / 2][2 * (k & 1)] = Store16<DT>::pack(e[0], e[1]);
            p[rb][k / 2][2 * (k & 1) + 1] = Store16<DT>::pack(e[2], e[3]);
        }
    };
    auto read_values = [&](int i, int x, ValueFrags& w) {
        const char* at = values_at(i) + G::value_lane(lane) + 2 * (x / (DO / 4)) * G::k16;
#pragma unroll
        for (int f = 0; f < 4; ++f) w[f] = G::value(at, 4 * (x % (DO / 4)) + f, G::value_odd(lane));
    };
    auto add_values = [&](int x, const ValueFrags& w) {
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) o[rb][4 * (x % (DO / 4)) + f] = mfma16<DT>(w[f], p[rb][x / (DO / 4)], o[rb][4 * (x % (DO / 4)) + f]);
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
            for (int k = 0; k < KB / 2; ++k) {
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
                    const u32x4 v = G::value(values_at(i) + G::value_lane(lane) + 2 * k * G::k16, n, G::value_odd(lane));
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) o[rb][n] = add_specials<DT>(v, seen[rb], o[rb][n]);
                }
            }
        }
        __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int j = 0; j < L; ++j) {
            u32x4 w = own_values(i)[G::kBlock / 16 * j + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = finite_of<DT>(w[e]);
            own_values(i)[G::kBlock / 16 * j + lane] = w;
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    Source next_keys, next_values;                                         // of tiles i + 2 and i + 1, requested while tile i is worked on
    int64_t next_at;                                                       // where tile i + 1's unit lies
    auto enter = [&](int i) {                                              // the workgroup goes on to tile i: K(i+1) and V(i), all that is under way, have to be there
        wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        next_values = source(i + 1, next_at, cache.v, G::kValuesAt);
        if (((i + 2) & 63) == 0) look_up((i + 2) / 64);
        next_at = lies_at(i + 2);
        next_keys = source(i + 2, next_at, cache.k, G::kKeysAt);
        if (!I8 && masked_group(i)) {
            look_for_specials(i);
            __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            const int* f = flags + (i & 1) * 4;
            if (__builtin_amdgcn_readfirstlane(f[0] | f[1] | f[2] | f[3])) take_specials_out(i);
        }
    };
    // Tile i.  The probabilities of its first block are there already.  After the last tile the scores are of whatever lies in LDS, and not
    // used: one block of instructions without a branch lets the compiler keep the order written here.
    KeyFrags kf;
    auto work = [&](int i) {
        ValueFrags vf;
#pragma unroll
        for (int k = 0; k < KB; ++k) {
            KeyFrags next;
            if (k + 1 < KB) read_keys(i + 1, k + 1, next);
            else            read_values(i, 0, vf);
#pragma unroll
            for (int j = k * 2 * L / KB; j < (k + 1) * 2 * L / KB; ++j) fetch(j < L ? next_values : next_keys, j % L);
            __builtin_amdgcn_sched_barrier(0);                             // what is read for the next products stands ahead of these
            scores(k, kf);
            if (k + 1 < KB) {
                float sum[RB];
                probabilities(k + 1, sum);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) l[rb] += sum[rb];
#pragma unroll
                for (int t = 0; t < KF; ++t) kf[t] = next[t];
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        // (Used here, so that the compiler does not put off their sums and roundings.)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) asm volatile("" : "+v"(l[rb]), "+v"(p[rb][0]), "+v"(p[rb][1]));
        if (i + 1 < wave_tiles && !unmasked(i + 1)) mask(i + 1);
        bool passes = false;
        float sum0[RB];
#pragma unroll
        for (int x = 0; x < VG; ++x) {
            ValueFrags next;
            if (x + 1 < VG) read_values(i, x + 1, next);
            __builtin_amdgcn_sched_barrier(0);
            add_values(x, vf);
            if (x == 0) passes = maxima();
            if (x == VG / 2) probabilities(0, sum0);                       // with the maximum as it is: of the next tile, whose first blocks' have gone in
            __builtin_amdgcn_sched_barrier(0);
            if (x + 1 < VG) {
#pragma unroll
                for (int n = 0; n < 4; ++n) vf[n] = next[n];
            }
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) asm volatile("" : "+v"(sum0[rb]), "+v"(p[rb][0]));
        if (i + 1 >= wave_tiles) return;
        if (passes) {
            raise();
            probabilities(0, sum0);
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) l[rb] += sum0[rb];
    };

    if (tiles > 0) {
        const bool any_missing = missing();                                // (asked for beside the places, seen to while the first tiles are under way)
        look_up(0);
        next_at = lies_at(1);
        const Source k0 = source(0, lies_at(0), cache.k, G::kKeysAt), v0 = source(0, lies_at(0), cache.v, G::kValuesAt), k1 = source(1, next_at, cache.k, G::kKeysAt);
#pragma unroll
        for (int j = 0; j < L; ++j) fetch(k0, j);
#pragma unroll
        for (int j = 0; j < L; ++j) fetch(v0, j);
#pragma unroll
        for (int j = 0; j < L; ++j) fetch(k1, j);
        wait_loads<0>();                                                   // Q too: from here on what is waited for is the loop's own
        holes = __builtin_amdgcn_readfirstlane(__syncthreads_or(any_missing));
        if (wave_tiles > 0) {
#pragma unroll
            for (int k = 0; k < KB; ++k) {
                read_keys(0, k, kf);
                scores(k, kf);
            }
            if (!unmasked(0)) mask(0);
            if (maxima()) raise();
            probabilities(0, l);
        }
        for (int i = 0; i < tiles; ++i) {
            enter(i);
            if (i < wave_tiles) {
                read_keys(i + 1, 0, kf);
                work(i);
            } else {
#pragma unroll
                for (int j = 0; j < L; ++j) { fetch(next_values, j); fetch(next_keys, j); }
            }
        }
        wait_loads<0>();
    }

#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float sum = l[rb];
        sum += __shfl_xor(sum, 16, kWave);
        sum += __shfl_xor(sum, 32, kWave);
        if (!row_there(rb)) continue;
        const int64_t t = seq.row0 + token_of(rb);
        const int head = head_of(rb);
        const float last = sum == 0.0f ? -INFINITY : m[rb];
        if (runs == 1) {
            const bool none = sum == 0.0f;
            const float f = none ? 0.0f : 1.0f / sum, v = I8 ? cache.v_scale[hk] : 1.0f;       // (apart, as in attention_rows.hip)
            uint16_t* dst = a.out + t * a.out_stride + (int64_t)head * D + 4 * g;
#pragma unroll
            for (int n = 0; n < DO; ++n) {
                const f32x4 x = o[rb][n];
                const u32x2 w = {none ? 0u : Store16<DTQ>::pack(x[0] * f * v, x[1] * f * v), none ? 0u : Store16<DTQ>::pack(x[2] * f * v, x[3] * f * v)};
                *reinterpret_cast<u32x2*>(dst + 16 * n) = w;
            }
            if (a.lse && g == 0) a.lse[t * a.q_heads + head] = none ? -INFINITY : (last + log2f(sum)) * 0.693147180559945f;
        } else {
            const int64_t slot = is_few ? few_slot(split, steps.batch, cache.heads, run, b, hk, wave_row + R * rb + l16) : token_slot(steps.tokens, a.q_heads, run, (int)t, head);
            float* dst = split.o + slot * D + 4 * g;
#pragma unroll
            for (int n = 0; n < DO; ++n) *reinterpret_cast<f32x4*>(dst + 16 * n) = o[rb][n];
            if (g == 0) split.ml[slot] = make_float2(last, sum);
        }
    }
}

int attention_tiles_launch(const AttnArgs& a, const KvPages& c, const KvSteps& s, const AttnSplit& few, const AttnSplit& many, int64_t many_blocks, int64_t few_blocks,
                           int dim, bool int8, sasq_dtype dt, hipStream_t st)
{
    auto go = [&](auto kernel) {
        launch_in_parts(many_blocks + few_blocks, kTileWaves * 64, [&](unsigned n, int first) {
            hipLaunchKernelGGL(kernel, dim3(n), dim3(kTileWaves * 64), 0, st, a, c, s, few, many, (int)many_blocks, first);
        });
    };
    auto by_format = [&](auto dtv, auto dimv) {
        constexpr int DTQ = decltype(dtv)::value, D = decltype(dimv)::value;
        const bool half = many.tile_rows == kTileRows / 2;
        if (int8) half ? go(attention_tiles_kernel<DTQ, D, true, 1>) : go(attention_tiles_kernel<DTQ, D, true, 2>);
        else      half ? go(attention_tiles_kernel<DTQ, D, false, 1>) : go(attention_tiles_kernel<DTQ, D, false, 2>);
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
