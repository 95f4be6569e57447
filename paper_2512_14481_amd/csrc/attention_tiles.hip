// Attention of many rows over the paged cache (chunks and prompts): bound by the matrix units and the exponentials beside them.
//
// A workgroup has one kv head of one sequence, up to 256 rows of it (32 for each of four or eight waves, the heads that share the kv head packed
// into the rows) and one run of keys, which it takes in tiles of 64 through rings of four stages in LDS for K and for V.
//
// Both products are taken transposed (see attention_rows.hip) on 32x32x16: a lane keeps one row from the scores to the output.  The scores of
// the next tile take the registers of this one's as these become probabilities, and what a product reads from LDS is
// read before the products ahead of it, so that products, exponentials and reads stand side by side.
#include "attention.h"

namespace sasq {

constexpr int kTileKeys = 64;

template <int D, bool I8, int W>
struct TilesGeo : KvRow<D, I8> {
    using K = KvRow<D, I8>;
    static constexpr int kTileRing = W == 4 ? 2 : 4;
    static constexpr int kTile = 4 * K::k16;     // bytes of a tile's keys, or of its values
    static constexpr int kKeysAt = 0, kValuesAt = kTileRing * kTile, kPagesAt = 2 * kTileRing * kTile;
    static constexpr int kFlagsAt = kPagesAt + W * 2 * 64 * 4;
    static constexpr int kLds = kFlagsAt + 64;
};

template <int DTQ, int D, bool I8, int W>
__global__ __launch_bounds__(W * 64, 2) void attention_tiles_kernel(AttnArgs a, KvPages cache, KvSteps steps, AttnSplit split, int few, int first)
{
    using G = TilesGeo<D, I8, W>;
    constexpr int DT = I8 ? SASQ_F16 : DTQ;
    constexpr int R = 32, DS = D / 16, DO = D / 32, KB = kTileKeys / 32;   // steps of the first product, blocks of 32 channels, of 32 keys
    constexpr int L = G::kLoads;
    __shared__ __attribute__((aligned(1024))) char lds[G::kLds];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int l32 = lane & 31, g = lane >> 5;

    // The tiles of a sequence's last rows see the most keys: they come first.
    int rest = (int)blockIdx.x + first;
    const int hk = rest % cache.heads; rest /= cache.heads;
    const int b = rest % steps.batch; rest /= steps.batch;
    const int run = rest % split.splits, tile = split.tiles - 1 - rest / split.splits;
    const KvSeq seq = kv_seq(steps, b, cache.page_shift);
    const int rows = seq.rows * a.group, row0 = tile * R * W;
    if (rows <= few || row0 >= rows) return;
    const int end = attn_end(seq, a.group, split, tile), runs = attn_runs(split, end);
    if (run >= runs) return;
    const int from = run * split.chunk, to = run == runs - 1 ? end : min(end, from + split.chunk);
    const int tiles = (to - from + kTileKeys - 1) / kTileKeys;
    const int past = seq.keys - seq.rows;
    const int sees_group = past + row0 / a.group;                          // last key of the workgroup's first row, of the wave's, of the wave's last row
    const int wave_row = row0 + R * wave;
    const int sees_wave = past + wave_row / a.group;
    const int wave_end = past + (min(rows, wave_row + R) - 1) / a.group + 1;
    const int wave_tiles = wave_row < rows ? min(tiles, max(0, (wave_end - from + kTileKeys - 1) / kTileKeys)) : 0;

    const int r = wave_row + l32;                                          // the lane's row
    const bool row_there = r < rows;
    const int token = (row_there ? r : row0) / a.group, head = hk * a.group + (row_there ? r : row0) % a.group;
    const int sees = past + token;
    float c;
    u32x4 q[DS];
    load_q<DTQ, D, I8, R>(a, a.q + (int64_t)(seq.row0 + token) * a.q_stride + (int64_t)head * D, row_there, g, I8 ? cache.k_scale[hk] : 1.0f, q, c);

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
    auto fetch_keys = [&](int i, int page) { fetch(i, page, cache.k, G::kKeysAt + i % G::kTileRing * G::kTile); };
    auto fetch_values = [&](int i, int page) { fetch(i, page, cache.v, G::kValuesAt + i % G::kTileRing * G::kTile); };
    auto keys_at = [&](int i) -> const char* { return lds + G::kKeysAt + i % G::kTileRing * G::kTile; };
    auto values_at = [&](int i) -> char* { return lds + G::kValuesAt + i % G::kTileRing * G::kTile; };

    f32x16 o[DO], s[KB];
    float m = kNoMax, l = 0.0f;                                            // maximum of the log2-scaled scores, sum
    u32x4 p[2 * KB];                                                       // of 16 keys each
#pragma unroll
    for (int n = 0; n < DO; ++n)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[n][j] = 0.0f;

    // The steps of both products go in groups of four.
    constexpr int KG = DS / 4, KF = I8 ? 2 : 4;                            // groups for 32 keys, 16-byte pieces of a group
    constexpr int VG = DO;                                                 // groups of a tile's values
    typedef u32x4 KeyFrags[KF];
    typedef u32x4 ValueFrags[4];
    auto read_keys = [&](int i, int x, KeyFrags& w) {                      // group x of tile i
        const char* at = keys_at(i) + G::template key_lane<R>(lane) + 2 * (x / KG) * G::k16;
#pragma unroll
        for (int t = 0; t < KF; ++t) w[t] = G::template key<R>(at, KF * (x % KG) + t);
    };
    auto scores = [&](int x, const KeyFrags& w) {
        f32x16& to = s[x / KG];
        if (x % KG == 0) {
#pragma unroll
            for (int j = 0; j < 16; ++j) to[j] = 0.0f;
        }
#pragma unroll
        for (int t = 0; t < KF; ++t) {
            if constexpr (I8) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const u32x2 lo = codes_to_f16(w[t][2 * e]), hi = codes_to_f16(w[t][2 * e + 1]);
                    to = mfma32<DT>(u32x4{lo[0], lo[1], hi[0], hi[1]}, q[4 * (x % KG) + 2 * t + e], to);
                }
            } else {
                to = mfma32<DT>(w[t], q[4 * (x % KG) + t], to);
            }
        }
    };
    // Score j of block k is of key 32 k + 8 (j / 4) + 4 g + j % 4.
    auto unmasked = [&](int i) -> bool { return !holes && from + kTileKeys * i + kTileKeys - 1 <= sees_wave; };
    auto mask = [&](int i) {
        const int last = sees - (from + kTileKeys * i) - 4 * g;            // of the lane's keys, 0 being its first
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (32 * k + 8 * (j / 4) + j % 4 > last) s[k][j] = -INFINITY;
        if (holes) {
#pragma unroll
            for (int u = 0; u < 2 * KB; ++u)
                if (!there_is(i, u)) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) s[u / 2][8 * (u & 1) + j] = -INFINITY;
                }
        }
    };
    float top;
    auto maxima = [&]() -> bool {                                          // whether a score passes the running maximum by too much
        top = s[0][0];
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, s[k][j]);
        return __any(__builtin_fmaf(top, c, -m) > kLazy);
    };
    auto raise = [&]() {                                                   // moves the maxima, and the sums with them
        const float t = fmaxf(fmaxf(top, __shfl_xor(top, 32, kWave)) * c, m);
        const float keep = kept(m, t);
        m = t;
        l *= keep;
#pragma unroll
        for (int n = 0; n < DO; ++n) o[n] *= keep;
    };
    auto probabilities = [&](int k) {                                      // of block k
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k][8 * h + j], c, -m));
            l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
#pragma unroll
            for (int j = 0; j < 4; ++j) p[2 * k + h][j] = Store16<DT>::pack(e[2 * j], e[2 * j + 1]);
        }
    };
    auto read_values = [&](int i, int x, ValueFrags& w) {
        const char* at = values_at(i) + G::template value_lane<R>(lane);
#pragma unroll
        for (int f = 0; f < 4; ++f) w[f] = G::template value<R>(at + (4 * x + f) / DO * G::k16, (4 * x + f) % DO);
    };
    auto add_values = [&](int x, const ValueFrags& w) {
#pragma unroll
        for (int f = 0; f < 4; ++f) o[(4 * x + f) % DO] = mfma32<DT>(w[f], p[(4 * x + f) / DO], o[(4 * x + f) % DO]);
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
            for (int u = 0; u < 2 * KB; ++u) {
                const bool there = there_is(i, u);
                u32x4 seen;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = k0 + 16 * u + (j < 2 ? 0 : 8) + 4 * g + 2 * (j & 1);
                    seen[j] = (there && key <= sees ? kSeen : 0u) | (there && key + 1 <= sees ? kSeen << 16 : 0u);
                }
#pragma unroll
                for (int n = 0; n < DO; ++n)
                    o[n] = add_specials<DT>(G::template value<R>(values_at(i) + G::template value_lane<R>(lane) + u * G::k16, n), seen, o[n]);
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

    constexpr int LEAD = G::kTileRing;                                     // tile i + LEAD's keys are requested at tile i, and i + LEAD - 1's values
    constexpr bool AHEAD = LEAD == 4;
    int ahead_k = 0, ahead_v = 0;                                          // their pages, read a tile before
    auto enter = [&](int i) {                                              // the workgroup goes on to tile i
        // LEAD 2: K(i+1) and V(i) have to be there, all that is under way.  LEAD 4: K(i+2) V(i+1), of four waves all but V(i+2) and K(i+3), of
        // eight all but one of these.
        if (AHEAD && i + 3 < tiles) wait_loads<L>();
        else                        wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (i + LEAD < tiles && ((i + LEAD) & 63) == 0) fetch_list((i + LEAD) / 64 + 1);
        if (brings_k && i + LEAD < tiles) fetch_keys(i + LEAD, ahead_k);
        if (brings_v && i + LEAD - 1 < tiles) fetch_values(i + LEAD - 1, ahead_v);
        ahead_v = W == 4 ? ahead_k : page_of(i + LEAD);
        ahead_k = page_of(i + LEAD + 1);
        if (!I8 && masked_group(i)) {
            if (brings_v) look_for_specials(i);
            __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            const int* f = flags + (i & 1) * 4;
            if (__builtin_amdgcn_readfirstlane(f[0] | f[1] | f[2] | f[3])) take_specials_out(i);
        }
    };
    KeyFrags kf;                                                           // the first group of the next tile; with a longer lead read ahead of the barrier
    auto work = [&](int i) {
        if (!AHEAD) read_keys(i + 1, 0, kf);
        if (!unmasked(i)) mask(i);
        if (maxima()) raise();
        probabilities(0);
        // (After the last tile the scores are of whatever lies in the ring, and not used: one block of instructions without a branch lets
        // the compiler keep the order below.)
        ValueFrags vf;
#pragma unroll
        for (int x = 0; x < KB * KG; ++x) {
            KeyFrags next;
            if (x + 1 < KB * KG) read_keys(i + 1, x + 1, next);
            else                 read_values(i, 0, vf);
            __builtin_amdgcn_sched_barrier(0);                             // the reads of the next products stand ahead of these
            scores(x, kf);
            if (x == 0) probabilities(1);
            if (x + 1 < KB * KG) {
#pragma unroll
                for (int t = 0; t < KF; ++t) kf[t] = next[t];
            }
            if (x >= KG - 1) __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int x = 0; x < VG; ++x) {
            ValueFrags next;
            if (x + 1 < VG) read_values(i, x + 1, next);
            else if (AHEAD) read_keys(i + 2, 0, kf);
            __builtin_amdgcn_sched_barrier(0);
            add_values(x, vf);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < 4; ++n) vf[n] = next[n];
        }
    };

    if (tiles > 0) {
        fetch_list(0);
        fetch_list(1);
        wait_loads<0>();                                                   // Q too: the loop's waits count the rings' loads alone
        for (int i = 0; i < LEAD && i < tiles; ++i) {
            if (brings_k) fetch_keys(i, page_of(i));
            if (brings_v && i < LEAD - 1) fetch_values(i, page_of(i));
        }
        ahead_k = page_of(LEAD);
        ahead_v = page_of(LEAD - 1);
        if (AHEAD && tiles > 3)       wait_loads<2 * L>();                 // K(0), K(1)
        else if (!AHEAD && tiles > 1) wait_loads<2 * L>();                 // K(0)
        else                          wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (wave_tiles > 0) {
#pragma unroll
            for (int x = 0; x < KB * KG; ++x) {
                read_keys(0, x, kf);
                scores(x, kf);
            }
            if (AHEAD) read_keys(1, 0, kf);
        }
        for (int i = 0; i < tiles; ++i) {
            enter(i);
            if (i < wave_tiles) work(i);
        }
    }

    float sum = l;
    sum += __shfl_xor(sum, 32, kWave);
    if (!row_there) return;
    const int64_t t = seq.row0 + token;
    top = m == kNoMax ? -INFINITY : m;
    if (runs == 1) {
        const bool none = sum == 0.0f;
        const float f = none ? 0.0f : (I8 ? cache.v_scale[hk] : 1.0f) / sum;
        uint16_t* dst = a.out + t * a.out_stride + (int64_t)head * D + 4 * g;
#pragma unroll
        for (int n = 0; n < DO; ++n)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const u32x2 w = {none ? 0u : Store16<DTQ>::pack(o[n][j] * f, o[n][j + 1] * f), none ? 0u : Store16<DTQ>::pack(o[n][j + 2] * f, o[n][j + 3] * f)};
                *reinterpret_cast<u32x2*>(dst + 32 * n + 2 * j) = w;
            }
        if (a.lse && g == 0) a.lse[t * a.q_heads + head] = none ? -INFINITY : (top + log2f(sum)) * 0.693147180559945f;
    } else {
        const int64_t slot = tiles_slot(steps.tokens, a.q_heads, run, (int)t, head);
        float* dst = split.o + slot * D + 4 * g;
#pragma unroll
        for (int n = 0; n < DO; ++n)
#pragma unroll
            for (int j = 0; j < 16; j += 4) *reinterpret_cast<f32x4*>(dst + 32 * n + 2 * j) = f32x4{o[n][j], o[n][j + 1], o[n][j + 2], o[n][j + 3]};
        if (g == 0) split.ml[slot] = make_float2(top, sum);
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
        if (split.tile_rows == 128) go(attention_tiles_kernel<DT, D, I8, 4>, 256);
        else                        go(attention_tiles_kernel<DT, D, I8, 8>, 512);
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
