// What the kernels of the paged cache and of packed sequences share: which sequence a row belongs to, where a token lies in
// the cache, and the attention of one row by one wavefront.
#pragma once
#include "lss_common.h"
#include "lss_kernels.h"
#include "lss_starts.h"

#include <type_traits>

namespace lss {

// The sequence of packed row t: the last b in [0, B) with cu[b] <= t, if t < cu[b + 1] too, else -1.  By the whole wavefront, 64 starts at a
// time: as many dependent loads as B has digits to the base 64.  (cu ascending; whatever it holds, only its B + 1 entries are read.)
__device__ __forceinline__ int find_sequence(const int32_t *__restrict__ cu, int B, int t, int lane, int &begin, int &end)
{
    int lo = 0, n = B + 1;
    while (n > 1) {
        const int step = (n + 63) / 64, at = lane * step;
        const uint64_t below = __ballot(at < n && cu[lo + min(at, n - 1)] <= t);
        if (below == 0) return -1;
        const int last = 63 - __clzll((long long)below);
        lo += last * step;
        n = min(step, n - last * step);
    }
    if (lo >= B) return -1;
    begin = cu[lo];
    end = cu[lo + 1];
    return begin <= t && t < end ? lo : -1;
}

// Index of the cache row that holds token `position` of sequence b, in units of H_kv * d elements; -1 where the table names no page.
__device__ __forceinline__ int64_t cache_row(const PageTable &pt, int b, int position)
{
    const int nth = position >> pt.page_shift;
    if (position < 0 || nth >= pt.max_pages) return -1;
    const int page = pt.table[(int64_t)b * pt.max_pages + nth];
    if ((uint32_t)page >= (uint32_t)pt.n_pages) return -1;
    return ((int64_t)page << pt.page_shift) + (position & ((1 << pt.page_shift) - 1));
}

// ---- tiles of packed sequences: BR rows each, a row being one of a token's G heads
__device__ __forceinline__ int lane_sum_scan(int x)     // inclusive over the wavefront; all lanes active
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}
struct PackedTile { int q_begin, n_q, k_begin, n_k, tile, b; };
// Tile `rank` of a head of keys and values; false: there are fewer.  Up to 64 sequences, a lane each: tiles in the order of the keys they see (in
// steps of 64), most first, so that no long one starts last.  More sequences: in the sequences' order, sequence b's tiles from number
// floor(cu[b] G / BR) + b on -- room for all of them, one at most too much --, which is found like a row's sequence.
__device__ __forceinline__ void sequence_rows(const int32_t *cu, int b, int rows, int &begin, int &n)
{
    const int start = cu[b];
    begin = start_within(start, rows);
    n = rows_between(start, cu[b + 1], rows);
}
__device__ __forceinline__ void queries_of(const PackedArgs &a, int b, int &begin, int &n) { sequence_rows(a.cu_q, b, a.rows_q, begin, n); }
__device__ __forceinline__ void keys_of(const PackedArgs &a, int b, int &begin, int &n) { sequence_rows(a.cu_k, b, a.rows_k, begin, n); }
__device__ __forceinline__ int first_query(const PackedArgs &a, int b) { return start_within(a.cu_q[b], a.rows_q); }
__device__ __forceinline__ int most_keys(const PackedArgs &a) { return a.rows_k; }
__device__ __forceinline__ bool is_causal(const PackedArgs &a) { return a.causal; }
// ... of drafted tokens, whose keys are in the cache (their number; they begin nowhere)
__device__ __forceinline__ void queries_of(const TreeArgs &a, int b, int &begin, int &n) { sequence_rows(a.cu, b, a.rows, begin, n); }
__device__ __forceinline__ void keys_of(const TreeArgs &a, int b, int &begin, int &n) { begin = 0, n = max(0, min(a.lengths[b], a.max_len)); }
__device__ __forceinline__ int first_query(const TreeArgs &a, int b) { return start_within(a.cu[b], a.rows); }
__device__ __forceinline__ int most_keys(const TreeArgs &a) { return a.max_len; }
__device__ __forceinline__ bool is_causal(const TreeArgs &a) { return a.tree == nullptr; }
template <int BR, typename Args>
__device__ __forceinline__ bool packed_tile(const Args &a, int G, int rank, int lane, PackedTile &t)
{
    int b, begin = 0, n_q = 0, k_begin = 0, n_k = 0, tile;
    if (a.B <= 64) {
        if (lane < a.B) {
            queries_of(a, lane, begin, n_q);
            keys_of(a, lane, k_begin, n_k);
        }
        const int tiles = (n_q * G + BR - 1) / BR;
        // its tiles that see keys from number 64 (x - 1) on: tile j's last row is of token ((j + 1) BR - 1) / G
        const auto count = [&](int x) {
            if (x <= 1) return tiles;
            const int last = 64 * (x - 1);              // some row's position must reach it
            if (last >= n_k) return 0;
            return is_causal(a) ? max(0, tiles - max(0, last - (n_k - n_q)) * G / BR) : tiles;
        };
        const auto total = [&](int x) { return __builtin_amdgcn_readlane(lane_sum_scan(count(x)), 63); };
        int lo = 1, hi = (most_keys(a) + 63) / 64 + 1;      // total(lo) > rank >= total(hi)
        if (rank >= total(1)) return false;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (total(mid) > rank) lo = mid;
            else hi = mid;
        }
        const int above = count(lo + 1), mine = count(lo) - above, scan = lane_sum_scan(mine), in = rank - total(lo + 1);
        b = __ffsll((long long)__ballot(scan > in)) - 1;
        tile = tiles - count(lo) + in - (scan - mine);
        const auto of = [&](int x) { return __builtin_amdgcn_readlane(x, b); };
        t = {of(begin), of(n_q), of(k_begin), of(n_k), of(tile), b};
        return true;
    }
    const auto first = [&](int i) { return (int)((int64_t)first_query(a, i) * G / BR) + i; };
    int lo = 0, n = a.B;
    while (n > 1) {
        const int step = (n + 63) / 64, at = lane * step;
        const uint64_t below = __ballot(at < n && first(lo + min(at, n - 1)) <= rank);
        if (below == 0) return false;
        const int last = 63 - __clzll((long long)below);
        lo += last * step;
        n = min(step, n - last * step);
    }
    b = __builtin_amdgcn_readfirstlane(lo);
    queries_of(a, b, begin, n_q);
    keys_of(a, b, k_begin, n_k);
    t = {__builtin_amdgcn_readfirstlane(begin), __builtin_amdgcn_readfirstlane(n_q), __builtin_amdgcn_readfirstlane(k_begin),
         __builtin_amdgcn_readfirstlane(n_k), __builtin_amdgcn_readfirstlane(rank - first(b)), b};
    return t.tile >= 0 && t.tile < (t.n_q * G + BR - 1) / BR;
}

template <typename T> struct Vec16;
template <> struct Vec16<bf16_t> { typedef bf16x8 type; };
template <> struct Vec16<float> { typedef f32x4 type; };

__device__ __forceinline__ float wave_max(float x)      // all lanes active
{
    const auto step = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
        const int other = __builtin_amdgcn_update_dpp((int)0xff800000, __builtin_bit_cast(int, x), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        x = fmaxf(x, __builtin_bit_cast(float, other));
    };
    step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ __forceinline__ float wave_total(float x)
{
#pragma unroll
    for (int sh = 32; sh >= 1; sh >>= 1) x += __shfl_xor(x, sh);
    return x;
}

// Attention of one query row against the first n_keys keys by one wavefront, everything in fp32, for rows whose log-sum-exp is known and whose result was spoilt by
// a value that the row does not see: a value is multiplied only where its key is seen here.  64 keys at a time, a lane each for the scores; then each lane's 16 bytes
// of every (64 / CHUNKS)th value, LOADS loads on their way at once.  The weights' own sum divides them, so that the log-sum-exp's rounding does not matter.
// (Keys and values one by one, a broadcast each: 1000 cycles a key.)
template <typename T, int D, int LOADS>
__device__ __forceinline__ void row_attention(const T *q, const T *k, int64_t k_stride, const T *v, int64_t v_stride, int n_keys, float lse, int lane, T *out)
{
    typedef typename Vec16<T>::type Vec;
    constexpr int VEC = 16 / sizeof(T), CHUNKS = D / VEC, KEYS = 64 / CHUNKS;
    const float c = kLog2e / sqrtf((float)D), top = lse * kLog2e;
    if (lse == -INFINITY) n_keys = 0;                   // no key, or none with a weight: zeros
    const int mine = lane / CHUNKS, column = lane % CHUNKS * VEC;
    float acc[VEC], l = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
    for (int j0 = 0; j0 < n_keys; j0 += 64) {
        const T *const key = k + min(j0 + lane, n_keys - 1) * k_stride;
        float s = 0.f;
#pragma unroll (LOADS < 4 ? LOADS : 4)
        for (int i = 0; i < D; i += VEC) {
            const Vec a = *reinterpret_cast<const Vec *>(q + i), b = *reinterpret_cast<const Vec *>(key + i);
#pragma unroll
            for (int e = 0; e < VEC; ++e) s = fmaf((float)a[e], (float)b[e], s);
        }
        const float p = j0 + lane < n_keys ? fast_exp2(s * c - top) : 0.f;
        l += p;
#pragma unroll LOADS
        for (int i = 0; i < CHUNKS; ++i) {
            const int at = j0 + i * KEYS + mine;
            const Vec x = *reinterpret_cast<const Vec *>(v + min(at, n_keys - 1) * v_stride + column);
            const float w = __shfl(p, i * KEYS + mine);
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[e] = fmaf(w, at < n_keys ? (float)x[e] : 0.f, acc[e]);
        }
    }
    l = wave_total(l);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    Vec r;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
#pragma unroll
        for (int sh = CHUNKS; sh < 64; sh *= 2) acc[e] += __shfl_xor(acc[e], sh);
        r[e] = (T)(acc[e] * inv);
    }
    if (lane < CHUNKS) *reinterpret_cast<Vec *>(out + column) = r;
}

// a / b in 32 bits where both fit (a fifth of the instructions); wavefront-uniform
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b)
{
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// ---- drafted tokens (lss_paged_attn_tree).  Sequence b has n_b G rows per head of keys and values, row r of them query head r % G of its drafted token r / G: tiles
// of BR rows.  The rounds of a tile (ROUND keys each) are cut into parts of as many as it takes to have about `target` of all sequences together, at least `least`; a
// workgroup has one.
// Only tiles that are cut need scratch memory and joining.  Their parts are of S rounds, S >= (all rounds) / target: a tile of R > S rounds has c < R / S + 1 < 2 R / S of them, so that all cut
// tiles together have fewer than 2 target parts, and there are fewer than target of those tiles, whatever the number of rows, sequences and heads.
struct TreePart {
    int b, h_kv, tile, tiles, begin, n, length;         // n: drafted tokens, from row `begin` on
    int r0, r1, count, slot;                            // rounds; parts of the tile of rows, of several this one's number among those of all cut tiles: a tile's are `tiles` apart
    int item, items;                                    // of several parts: which cut tile of rows of any head, of how many
    int64_t all;                                        // parts of all tiles.  (This and items are set in any case)
};
__device__ __forceinline__ int64_t lane64(int64_t x, int lane)        // of that lane, wavefront-uniform
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)x, lane) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32);
}
// inclusive sums over the wavefront of numbers from 0 to 2^50: two 32-bit ones (by shuffles of 64 bits: 1 us for the three of tree_part)
__device__ __forceinline__ int64_t lanes_upto(int64_t x)
{
    const int low = lane_sum_scan((int)(x & 0xffffff)), high = lane_sum_scan((int)(x >> 24));
    return ((int64_t)high << 24) + low;
}
// A sequence's tiles of BR rows and rounds of ROUND keys; none from number B on
struct TreeSequence { int length, begin, n, tiles, R; };
__device__ __forceinline__ TreeSequence tree_sequence(const TreeArgs &a, int G, int round, int rows, int b)
{
    TreeSequence s{0, 0, 0, 0, 0};
    if (b < a.B) {
        s.length = max(0, min(a.lengths[b], a.max_len));
        queries_of(a, b, s.begin, s.n);
    }
    s.tiles = (s.n * G + rows - 1) / rows;              // (rows * H <= 2^24)
    s.R = (max(1, s.length) + round - 1) / round;
    return s;
}
__device__ __forceinline__ int64_t parts_of_tiles(const TreeSequence &s, int S) { return (int64_t)s.tiles * ((s.R + S - 1) / S); }
__device__ __forceinline__ int cut_tiles(const TreeSequence &s, int S) { return s.R > S ? s.tiles : 0; }
// Rounds of a part.  parts(S): how many parts of S rounds there are per head.  (A part too many for the workgroups that there is room for at once waits for all of another: a few sizes are
// tried, where one part a tile fits.)
template <typename F> __device__ __forceinline__ int part_rounds(int64_t rounds, int64_t all_tiles, int H_kv, int target, int least, F &&parts)
{
    const int64_t wanted = divide(rounds * H_kv + target - 1, target);
    int S = wanted < least ? least : wanted < 1 << 30 ? (int)wanted : 1 << 30;
    for (int tries = 0;; ++tries) {
        const int64_t all = parts(S);
        if (all * H_kv <= target || all_tiles * H_kv > target || tries == 4 || S >= 1 << 24) return S;
        const int64_t more = divide((all * H_kv - target) * S, target);
        S += more < 1 ? 1 : more < S ? (int)more : S;
    }
}
// Are parts of S_most rounds, `most` of them, worth it where `target` of S rounds are the rule?  Where as many more are resident at once, each of them slower, and parts become so much shorter.
// d = 64, two and three workgroups a compute unit: a round takes 17 twelfths as long, and a part some three rounds of its own (its start, its share of the joining launch).  24 sequences of 6000
// tokens, 64 drafted: 85.4 us by 512, 69.1 by 768; 48 137.9 and 121.5; one of 36,000 with a chain of 256, whose tiles fill either: 64.4 and 68.6.
__device__ __forceinline__ bool worth_more(int S, int S_most) { return (int64_t)17 * S_most + 36 < (int64_t)12 * S; }
// Many sequences: every workgroup would go over all of them to find its part -- 2048 of one token, 8 heads of keys, 1.3 ms, 4096 4.4 --, so that a launch in front does it once
// (tree_count_kernel) and says per 64 sequences what is in front of them.
struct TreeCount { int64_t all; int S, cut; };          // per head of keys: parts, rounds of one, cut tiles
struct TreeBatch { int64_t before; int cut, slots; };   // per head of keys, of the sequences in front: parts, cut tiles, parts of these
inline size_t tree_count_bytes(int B) { return sizeof(TreeCount) + (size_t)((B + 63) / 64) * sizeof(TreeBatch); }

// Workgroup `id`'s part; false: there is none.  Parts are numbered by sequence, head, part of the keys and tile of rows, and each XCD (workgroups go to them in turn) has a run
// of them: tiles of rows that read the same keys do so at the same time from one L2.  All lanes active; wavefront-uniform.
// `room`: workgroups, target and a part for every tile of rows at least.
template <int ROUND, int BR>
__device__ __forceinline__ bool tree_part(const TreeArgs &a, int lane, int id, int target, int most, int least, int room, TreePart &p)
{
    const int G = a.H / a.H_kv;
    const auto load = [&](int b0) __attribute__((always_inline)) { return tree_sequence(a, G, ROUND, BR, b0 + lane); };
    const auto last_of = [](int x) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(x, 63); };
    TreeSequence s;
    int S, cut, cut_upto = 0, b0 = 0, cut_before = 0, slots_before = 0;
    int64_t mine, upto, before = 0, at, nth;
    bool some_cut;                                      // (where none is, nothing needs their numbers)
    const auto find = [&](int64_t all) __attribute__((always_inline)) {
        p.all = all * a.H_kv;
        if (p.all > room) return false;                 // (more than there can be: cu does not ascend)
        const int64_t per_xcd = (p.all + 7) / 8;
        at = id % 8 * per_xcd + id / 8;
        nth = divide(at, a.H_kv);                       // (some sequence has it)
        return id / 8 < per_xcd && at < p.all;
    };
    if (a.count) {
        const TreeCount c = *a.count;
        const TreeBatch *const batches = reinterpret_cast<const TreeBatch *>(a.count + 1);
        S = c.S;
        some_cut = c.cut > 0;
        p.items = c.cut * a.H_kv;
        if (!find(c.all)) return false;
        int lo = 0, n = (a.B + 63) / 64;                // the last batch that begins with part nth or in front of it: 64 tried at a time
        while (n > 1) {
            const int step = (n + 63) / 64, i = lane * step;
            const uint64_t below = __ballot(i < n && batches[lo + min(i, n - 1)].before <= nth);
            const int last = 63 - __clzll((long long)(below | 1));
            lo += last * step;
            n = min(step, n - last * step);
        }
        const TreeBatch batch = batches[lo];
        b0 = 64 * lo, before = batch.before, cut_before = batch.cut, slots_before = batch.slots;
        s = load(b0);
        mine = parts_of_tiles(s, S), upto = lanes_upto(mine), cut = cut_tiles(s, S);
        if (some_cut) cut_upto = lane_sum_scan(cut);
    } else {
        s = load(0);
        int64_t rounds = lane64(lanes_upto((int64_t)s.tiles * s.R), 63);
        int all_tiles = last_of(lane_sum_scan(s.tiles));
        for (int i = 64; i < a.B; i += 64) {
            const TreeSequence t = load(i);
            rounds += lane64(lanes_upto((int64_t)t.tiles * t.R), 63);
            all_tiles += last_of(lane_sum_scan(t.tiles));
        }
        int64_t all;
        int behind;                                     // cut tiles of the sequences from number 64 on
        const auto parts = [&](int S) __attribute__((always_inline)) {
            mine = parts_of_tiles(s, S), upto = lanes_upto(mine), all = lane64(upto, 63), behind = 0;
            for (int i = 64; i < a.B; i += 64) {
                const TreeSequence t = load(i);
                all += lane64(lanes_upto(parts_of_tiles(t, S)), 63);
                behind += last_of(lane_sum_scan(cut_tiles(t, S)));
            }
            return all;
        };
        S = part_rounds(rounds, all_tiles, a.H_kv, target, least, parts);
        if (most > target && rounds * a.H_kv >= (int64_t)20 * most) {
            const int64_t mine_of = mine, upto_of = upto, all_of = all;
            const int behind_of = behind, S_most = part_rounds(rounds, all_tiles, a.H_kv, most, least, parts);
            if (worth_more(S, S_most)) S = S_most;
            else mine = mine_of, upto = upto_of, all = all_of, behind = behind_of;
        }
        cut = cut_tiles(s, S);
        some_cut = __any(cut != 0) || behind > 0;
        if (some_cut) cut_upto = lane_sum_scan(cut);
        p.items = (last_of(cut_upto) + behind) * a.H_kv;
        if (!find(all)) return false;
    }
    const auto slots_of = [](int64_t mine, int cut) __attribute__((always_inline)) { return cut ? (int)mine : 0; };
    while (before + lane64(upto, 63) <= nth) {
        before += lane64(upto, 63);
        if (some_cut) cut_before += last_of(cut_upto), slots_before += last_of(lane_sum_scan(slots_of(mine, cut)));
        b0 += 64;
        if (b0 >= a.B) return false;
        s = load(b0);
        mine = parts_of_tiles(s, S), upto = lanes_upto(mine);
        if (some_cut) cut = cut_tiles(s, S), cut_upto = lane_sum_scan(cut);
    }
    const int l = __ffsll((long long)__ballot(before + upto > nth)) - 1;
    const auto of = [&](int x) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(x, l); };
    const int R = of(s.R), tiles = of(s.tiles), c = (R + S - 1) / S, within = (int)(at - (before + lane64(upto - mine, l)) * a.H_kv), rest = within % (tiles * c);
    p.b = b0 + l, p.begin = of(s.begin), p.n = of(s.n), p.length = of(s.length);
    p.h_kv = within / (tiles * c), p.tiles = tiles, p.tile = rest % tiles;
    const int part = rest / tiles, even = R / c, more_of = R - even * c;       // (as equal as they can be)
    p.count = c, p.r0 = part * even + min(part, more_of), p.r1 = p.r0 + even + (part < more_of);
    p.slot = p.item = 0;
    if (c > 1) {
        const int slots = slots_of(mine, cut);
        p.slot = (slots_before + of(lane_sum_scan(slots) - slots)) * a.H_kv + within;
        p.item = (cut_before + of(cut_upto - cut)) * a.H_kv + p.h_kv * tiles + p.tile;
    }
    return true;
}
// row of out and lse of row r of a sequence that begins with drafted token `begin`
__device__ __forceinline__ int64_t tree_row(const TreeArgs &a, int begin, int G, int h_kv, int r) { return (int64_t)(begin + r / G) * a.H + h_kv * G + r % G; }
// Scratch memory of `slots` parts, for those of tiles that are cut: of each row sum of weight * value [d], maximum (log2 domain) and sum; and for the joining launch
// how many such tiles of rows there are, `chains` at most, and where the parts of each begin (its first part says so).
struct TreeChain { int b, h_kv, tile, first, count, tiles, unused[2]; };
struct TreeScratch {
    float *base;
    int rows, d, slots, chains;
    __device__ __forceinline__ int *items() const { return reinterpret_cast<int *>(base); }
    __device__ __forceinline__ TreeChain *chain(int i) const { return reinterpret_cast<TreeChain *>(base) + 1 + i; }
    __device__ __forceinline__ float *sums(int part, int n) const { return base + 8 * (chains + 1) + ((int64_t)part * rows + n) * 2; }
    __device__ __forceinline__ float *values(int part, int n) const { return base + 8 * (chains + 1) + (int64_t)slots * rows * 2 + ((int64_t)part * rows + n) * d; }
    // by one thread of each workgroup
    __device__ __forceinline__ void enter(const TreePart &p, bool some) const
    {
        if (blockIdx.x == 0) *items() = p.all > gridDim.x ? 0 : p.items;
        if (some && p.count > 1 && p.r0 == 0) *chain(p.item) = {p.b, p.h_kv, p.tile, p.slot, p.count, p.tiles, {0, 0}};
    }
};
// sum + factor * x, x a sum of weights times values and the factor what those weights are off by: above 0, but 0 in 32 bits where x's scores lie 2^7 or more (in powers of 2) below others.
// 0 times a sum that is infinite would be NaN: such a one stays what it is.
__device__ __forceinline__ float add_scaled(float factor, float x, float sum) { return fmaf(fabsf(x) < INFINITY ? factor : 1.f, x, sum); }
inline size_t tree_scratch_bytes(int rows, int d, int slots, int chains) { return sizeof(float) * (8 * ((size_t)chains + 1) + (size_t)slots * rows * (d + 2)); }
// Which of the 32 keys from drafted number c0 on (below 0: the tokens in front of them) drafted token i of its sequence sees; `bits`: its words
__device__ __forceinline__ uint32_t keys_seen(const TreeArgs &a, const uint64_t *bits, int i, int c0)
{
    if (a.tree == nullptr) {
        const int last = i - c0;
        return last < 0 ? 0u : last >= 31 ? ~0u : (2u << last) - 1;
    }
    if (c0 <= -32) return ~0u;
    const int from = max(c0, 0), word = from >> 6, sh = from & 63;
    uint64_t seen = word < a.words ? bits[word] >> sh : 0;
    if (sh > 32 && word + 1 < a.words) seen |= bits[word + 1] << (64 - sh);
    return c0 >= 0 ? (uint32_t)seen : (uint32_t)seen << -c0 | ((1u << -c0) - 1);
}

} // namespace lss
