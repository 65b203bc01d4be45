// Tuned bf16 forward of Eq. 2 (Section 3, Principle 3) for gfx950.
//
// S^T = K Q^T with one query per lane, then O^T += V^T P^T with P^T fed straight from the S^T registers.  The keys are
// walked in blocks of 32 (two per 64-key K/V tile).  Per block g three stages:
//     A(g): S^T product (matrix),  B(g): weights P^T (vector: exp, row sum, bf16 packing),
//     C(g): O^T product (matrix).
// A wavefront issues in order, and vector work costs it several times the issue time of a matrix
// instruction, so the stages are software-pipelined: step g issues the matrix instructions of
// A(g+1) and C(g-1) with the vector work of B(g) spread between them.  K/V tiles travel
// global -> LDS directly (no registers in between), a full loop iteration ahead, into two unpadded, swizzled
// slots each; V is read transposed by DS_READ_B64_TR_B16.
//
// A workgroup is RB wavefronts of 32 query rows, or KG such groups that have a part of the keys each and tiles of their own
// in LDS, and meet there at the end: what fills the chip in launches of few rows without partial results in memory and
// a launch to merge them, and shortens the walk that each wavefront is alone with.  Between backward passes, 8 x 2 heads of 1024
// rows behind 0, 2048 and 4096 others: 128-row workgroups with the best split and its merge 21.1, 29.6 and 38.2 us, 64 rows in two
// groups 14.9, 27.4 and 38.2, 128 rows in two groups 18.4, 28.5 and 35.9; 4 heads of 256 rows behind 512: 11.3, 9.7 and 12.4.  Four groups
// of one or two row blocks (d = 64) go on where that leaves off (figures: pick_fwd_plan).  Large
// launches keep one group (64 heads of 4096 rows: 1692 us, in two groups
// 1829): three workgroups per compute unit hide each other's waits.  The form is chosen per launch (pick_fwd_plan).
//
// Softmax: B subtracts the running maximum m as it stands (no pass over the block first).  Only
// when the block's weights of some row add up to more than 2^8 -- so no weight can be larger
// without this being noticed: a score well above m, or a row seeing its first key -- does a rare,
// wavefront-uniform fix-up raise m to the exact maximum, rescale the row sum and the accumulator,
// and redo the block's weights.  The final division by the row sum, which uses the same m, makes
// the result independent of when m was raised.
#include "lss_bf16.h"
#include <type_traits>
#include "lss_kernels.h"
#include "lss_serve.h"

namespace lss {

template <int D, int RB_, int KG_>
struct FwdBf16Cfg {
    // KG groups of RB wavefronts share the query rows (32 per wavefront of a group) and have a part of the keys each.
    static constexpr int RB = RB_, KG = KG_, WAVES = RB * KG, RW = 32, BR = RB * RW, BC = 64, NT = 64 * WAVES;
    static constexpr int NU = D / 16;                   // operand steps of the S^T product; same for O^T
    using Tile = DirectTile<D, BC, RB>;
    // A group's LDS: two pair slots, slot p a K tile (number p mod 2) and after it a V tile (number p + 1 mod 2): K is
    // loaded one tile further ahead than V and done with one tile earlier, so that two tiles of each are enough.
    static constexpr int OFF_V = Tile::BYTES, PAIR = 2 * Tile::BYTES, RING = 2 * PAIR;
    // (dropout: behind them, the column keys of the last four tiles issued, 64 each)
    static constexpr int group_lds(bool drop) { return RING + (drop ? 4 * BC * 4 : 0); }
    // what the groups hand each other at the end: accumulators in chunks of 16 bytes per lane; maximum and row sum
    static constexpr int UNITS = D / 8, HAND_ML = WAVES * UNITS * 1024, HAND = KG > 1 ? HAND_ML + WAVES * 512 : 0;
    static constexpr int lds(bool drop) { return KG * group_lds(drop) > HAND ? KG * group_lds(drop) : HAND; }
    static constexpr float kMaxBlockSum = 256.0f;       // 2^8: largest sum of a lane's weights of one block without a fix-up
};

// What a workgroup's rows are and what they read, in elements: row r is head r % G (D columns further on) of token r / G, whose position is s0 + r / G.
struct FwdView {
    const bf16_t *q, *k, *v;    // first rows
    int64_t q_ld, k_ld, v_ld;   // from a token to the next
    int64_t s0;
    int l_s, l_x, causal, G;    // rows, keys
};

// ... and drafted tokens over a paged cache (FwdView's k, v and their distances are not used; s0 and causal where there is no tree): tiles t0 .. t1 - 1 of the sequence's keys
struct PagedView : FwdView {
    const TreeArgs *a;
    const int32_t *table;       // the sequence's
    const char *k_head, *v_head;        // of the head, page 0
    const uint64_t *bits;       // of the sequence's first row
    int first, t0, t1;          // key of the first drafted token
    int *spoilt;                // LDS, 0: has some value among the drafted ones' been found that is not finite
};
// v with 0 in the place of what is not finite
__device__ __forceinline__ bf16x8 finite_part(bf16x8 v)
{
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (!(fabsf((float)v[e]) < INFINITY)) v[e] = (bf16_t)0.f;
    return v;
}

// DROP: dropout on the weights (Section 2.2): the weight that multiplies V is dropped or (the finished sum) scaled by
// 1 / (1 - p) according to drop_keep() of (seed, batch*head, global row, key); row sum and lse are
// those of the softmax.
// The rows r0 .. of a workgroup: put(u, values) takes columns 8 u + 4 (lane / 32) .. + 3 of row r0 + 32 (wavefront) + lane % 32, normalised,
// put_lse its lse.  `bh`: batch * head for the dropout's decisions.  PACKED: G heads of a token, K's and V's rows each with a distance of their own,
// perhaps more rows than keys (a segment has none of that, and what is not there costs its kernels nothing: 1.2 % of lx24k's last segment).
template <int D, bool DROP, int RB, int KG, bool PACKED, typename View, typename Put, typename PutLse>
__device__ __forceinline__ void fwd_bf16_body(char *smem, const View &s, const DropArgs &dr, int bh, int r0, int split, int n_splits, Put &&put,
                                              PutLse &&put_lse)
{
    using C = FwdBf16Cfg<D, RB, KG>;
    using Tile = typename C::Tile;
    constexpr int NU = C::NU;
    constexpr bool PAGED = std::is_same<View, PagedView>::value;
    static_assert(!PAGED || (PACKED && KG == 1), "");

    const int tid = threadIdx.x, lane = tid & 63, lq = lane & 31, hh = lane >> 5;
    const int all_waves = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = KG > 1 ? all_waves / RB : 0, wave = KG > 1 ? all_waves % RB : all_waves;      // wave: within the group
    char *const ring = smem + group * C::group_lds(DROP);
    const int rw0 = r0 + wave * C::RW;                  // first row of this wavefront

    const int r_last = min(r0 + C::BR, s.l_s) - 1;
    const int G = PACKED ? s.G : 1;
    int kv_end = s.causal ? (int)min<int64_t>(s.l_x, s.s0 + r_last / G + 1) : s.l_x;
    if (PACKED) kv_end = max(kv_end, 0);                // (more rows than keys: the first ones see none)
    const int n_tiles = (kv_end + C::BC - 1) / C::BC;
    const int per = (n_tiles + n_splits - 1) / n_splits;
    int s_begin = split * per, s_tiles = max(min(n_tiles, s_begin + per) - s_begin, 0);
    if constexpr (PAGED) s_begin = s.t0, s_tiles = max(min(n_tiles, s.t1) - s.t0, 0);
    // this group's tiles; the first group has `iters` of them, the last ones fewer or none
    const int iters = KG > 1 ? (s_tiles + KG - 1) / KG : s_tiles;
    const int t_begin = s_begin + group * iters, T = KG > 1 ? max(min(s_tiles - group * iters, iters), 0) : s_tiles;

    // this lane's query row (column of the S^T tile); rows past the segment re-read its last row
    // (unconditional loads), are computed like any other and never stored
    const int r = rw0 + lq;
    const bool row_ok = r < s.l_s;
    const int position = (int)s.s0 + r / G;
    Frag<bf16_t> qf[NU];
    {
        const int rr = min(r, s.l_s - 1);
        const bf16_t *qp = s.q + (int64_t)(rr / G) * s.q_ld + (rr % G) * D + hh * 8;
#pragma unroll
        for (int kb = 0; kb < NU; ++kb) qf[kb] = load_frag<bf16_t>(qp + kb * 16);
    }
    const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    f32x16 o[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) o[db] = zero16;
    float m = -INFINITY, l = 0.f;                       // running maximum (log2 domain); this lane's half of the row sum
    float m_sub = -1e30f;                               // what B subtracts: m, or as long as the row has seen no key a huge negative number
    const float c = kLog2e / sqrtf((float)D);

    if (s_tiles > 0) {
        // dropout: this lane's row key; the column seed; the column keys of tile t (global tile index)
        // are computed once, by one wavefront when the tile's loads are issued, into quarter t % 4 of
        // a small ring behind the tiles -- published by the same barrier as the tile
        uint32_t drop_rk = 0u, drop_cs = 0u;
        if (DROP) { drop_rk = drop_row_key(dr.seed_lo, (uint32_t)bh, (uint32_t)position); drop_cs = drop_col_seed(dr.seed_hi); }
        char *const ck_ring = ring + C::RING;

        // ---- tile loads, by all wavefronts of the group.  No branch and few scalar instructions on purpose: a branch inside a
        // pipeline step splits it into basic blocks, and the vector work that was meant to sit between the step's matrix
        // instructions is then moved behind the branch in one lump; addresses move on between the iterations instead.
        uint32_t offK[Tile::NI], offV[Tile::NI], offD[Tile::NI];    // this lane's global offsets within the next K and V tile; and
        Tile::pair_offsets(offK, s.k_ld, C::BC, wave, lane);        // what must be added to them in the sequence's last, partial
        const int t_part = s.l_x % C::BC ? s.l_x / C::BC : -1;     // tile (rows past the end re-read the last row)
        uint32_t offDV[PACKED ? Tile::NI : 1];                      // ... V's, where its rows are not as far apart as K's
        {
            uint32_t offL[Tile::NI];
            Tile::pair_offsets(offL, s.k_ld, t_part >= 0 ? s.l_x % C::BC : C::BC, wave, lane);
#pragma unroll
            for (int i = 0; i < Tile::NI; ++i) { offD[i] = offL[i] - offK[i]; offV[i] = offK[i]; }
            if constexpr (PACKED) {
                Tile::pair_offsets(offV, s.v_ld, C::BC, wave, lane);
                Tile::pair_offsets(offL, s.v_ld, t_part >= 0 ? s.l_x % C::BC : C::BC, wave, lane);
#pragma unroll
                for (int i = 0; i < Tile::NI; ++i) offDV[i] = offL[i] - offV[i];
            }
        }
        const uint32_t k_bytes = (uint32_t)(C::BC * s.k_ld * 2), v_bytes = PACKED ? (uint32_t)(C::BC * s.v_ld * 2) : k_bytes;
        // the next tile of K to load, and of V, one behind; past the group's last one that one again
        const int t_last = t_begin + max(T, 1) - 1;
        int k_tile_next = t_begin, v_tile_next = t_begin;
        const char *k_next = tile_ptr(Tile::pair_base(s.k), t_begin, k_bytes), *v_next = tile_ptr(Tile::pair_base(s.v), t_begin, v_bytes);
        auto to_part = [&](int t, uint32_t (&off)[Tile::NI], bool of_v) __attribute__((always_inline)) {
            if (t == t_part)
#pragma unroll
                for (int i = 0; i < Tile::NI; ++i) off[i] += PACKED && of_v ? offDV[PACKED ? i : 0] : offD[i];
        };
        to_part(k_tile_next, offK, false);
        to_part(v_tile_next, offV, true);
        // Pages: this lane's place in a part of 16 rows; buffers of the next K tile's part and, one tile behind, of V's; 64 pages' numbers, a lane each, and the 64 behind
        // them (page numbers wait for nothing when a tile's turn comes).  `holes`: some number so far was none
        uint32_t off_page[PAGED ? Tile::NI : 1];
        u32x4 k_buffer, v_buffer;
        int window = 0, window_behind = 0, window_at = 0, row_bytes = 0;
        bool holes = false;
        int64_t k_row = 0;              // bytes from page 0, and how many
        uint32_t k_ok = 0;
        const auto numbers = [&](int from) {
            if constexpr (PAGED) return s.table[min(from + lane, s.a->pt.max_pages - 1)];
            else return 0;
        };
        const auto look_for_holes = [&] {
            if constexpr (PAGED) holes = holes || __any(((window_at + lane) << s.a->pt.page_shift) < s.l_x && (uint32_t)window >= (uint32_t)s.a->pt.n_pages);
        };
        const auto find_page = [&](int t) __attribute__((always_inline)) {
            if constexpr (PAGED) {
                const int key = t * C::BC + wave * 16 / (RB / 4) / 16 * 16, shift = s.a->pt.page_shift;
                if ((key >> shift) - window_at >= 64) {
                    window_at += 64;
                    window = window_behind;
                    window_behind = numbers(window_at + 64);
                    look_for_holes();
                }
                const int page = __builtin_amdgcn_readlane(window, (key >> shift) - window_at & 63);
                const bool there = (uint32_t)page < (uint32_t)s.a->pt.n_pages && key < s.l_x;
                k_row = (((int64_t)(there ? page : 0) << shift) + (key & ((1 << shift) - 1))) * row_bytes;
                k_ok = there ? (uint32_t)(min(s.l_x - key, 16) - 1) * (uint32_t)row_bytes + D * 2 : 0;
            }
        };
        const auto buffer_of = [&](const char *head) __attribute__((always_inline)) {
            const uint64_t p = (uint64_t)(head + k_row);
            const auto uniform = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
            return u32x4{uniform((uint32_t)p), uniform((uint32_t)(p >> 32) & 0xffffu), uniform(k_ok), 0x00020000u};
        };
        if constexpr (PAGED) {
            static_assert(RB == 4 || RB == 8, "");
            row_bytes = s.a->H_kv * D * 2;
            Tile::page_offsets(off_page, (uint32_t)row_bytes, wave, lane);
            window_at = t_begin * C::BC >> s.a->pt.page_shift;
            window = numbers(window_at);
            window_behind = numbers(window_at + 64);
            look_for_holes();
            find_page(t_begin);
            k_buffer = buffer_of(s.k_head);
            v_buffer = buffer_of(s.v_head);
        }
        auto advance_k = [&] {
            if constexpr (PAGED) {
                // (V's next tile is the one that was K's)
                v_buffer = buffer_of(s.v_head);
                if (k_tile_next < t_last) {
                    find_page(++k_tile_next);
                    k_buffer = buffer_of(s.k_head);
                }
                return;
            }
            if (k_tile_next < t_last) { ++k_tile_next; k_next += k_bytes; to_part(k_tile_next, offK, false); }
        };
        auto advance_v = [&] {
            if (!PAGED && v_tile_next < t_last) { ++v_tile_next; v_next += v_bytes; to_part(v_tile_next, offV, true); }
        };
        // Iteration t's loads, behind its barrier: K of tile t + 2 in the place of tile t's, whose last rows have been read
        // by then, and V of tile t + 1 in the place of tile t - 1's.  (Past the end a tile is loaded once more: K where it
        // lies already or where nobody reads any more, V where nobody reads any more.)
        auto issue_next = [&](char *pair_slot) __attribute__((always_inline)) {
            static_assert(C::OFF_V == Tile::BYTES, "V tile follows K tile");
            if constexpr (PAGED) Tile::issue_pages(k_buffer, v_buffer, off_page, pair_slot, wave);
            else Tile::issue_pair(k_next, v_next, offK, offV, pair_slot, wave);
            if (DROP && wave == 0)
                reinterpret_cast<uint32_t *>(ck_ring)[(k_tile_next & 3) * C::BC + lane] = drop_col_key(drop_cs, (uint32_t)(k_tile_next * C::BC + lane));
        };

        // ---- this lane's LDS addresses (bytes from smem) in the K tile that A and in the V tile that C reads next; they move to
        // the next tile once per iteration, to the other pair slot and back
        const int ring_at = group * C::group_lds(DROP);
        int a_at[NU];                                   // A-operand chunk of row lq for operand step kb
#pragma unroll
        for (int kb = 0; kb < NU; ++kb) a_at[kb] = ring_at + Tile::chunk_offset(lq, 2 * kb + hh);
        int t_at[D / 32][2];                            // transposed reads, column block db: either read's
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
            const int off = tr_lane_offset_sw<D>(lane, db);
            t_at[db][0] = ring_at + C::OFF_V + off;
            t_at[db][1] = ring_at + C::OFF_V + (off ^ 48);
        }

        // ---- stage pieces.  `kb2`: which half of the tile, a block of 32 keys.
        auto load_a = [&](int kb2, int kb, Frag<bf16_t> &fk) __attribute__((always_inline)) {
            fk = load_frag<bf16_t>(reinterpret_cast<const bf16_t *>(smem + a_at[kb] + kb2 * 32 * (D * 2)));
        };
        auto load_c = [&](int kb2, int u, Frag<bf16_t> &fv) __attribute__((always_inline)) {
            const int half = u / (D / 32), db = u % (D / 32);
            fv = load_frag_tr_sw<D>(smem, (kb2 * 2 + half) * 16, t_at[db][0], t_at[db][1]);
        };
        // Where the causal diagonal or the end of the sequence crosses a block (first key jb), the
        // masked elements of its finished S^T accumulator are set to -inf, which B turns into weight
        // 0: keys after the lane's row, and keys past the sequence (whose loads re-read its last
        // row).  C-tile element e of this lane is key 8*(e/4) + 4*hh + e%4 of the block.
        // (positions are below 2^30, checked on the host: one 32-bit scalar compare, no vector work per step)
        int last_whole = min(s.causal ? (int)s.s0 + rw0 / G - 31 : s.l_x, s.l_x - 32);       // blocks from here on need no mask
        if constexpr (PAGED)
            if (!s.causal) last_whole = min(last_whole, s.first - 32);
        auto mask_s = [&](int jb, f32x16 &sc) __attribute__((always_inline)) {
            if constexpr (PAGED) {
                if (jb > last_whole || holes) {
                    const int token = min(r, s.l_s - 1) / G, left = s.l_x - jb;
                    uint32_t seen = keys_seen(*s.a, s.bits + (int64_t)token * s.a->words, token, jb - s.first);
                    if (left < 32) seen &= left <= 0 ? 0u : (1u << left) - 1;
                    if (holes)
                        for (int i = 0; i < 2; ++i) {
                            const int nth = (jb + 16 * i) >> s.a->pt.page_shift;
                            if (jb + 16 * i < s.l_x && (uint32_t)s.table[nth] >= (uint32_t)s.a->pt.n_pages) seen &= ~(0xffffu << 16 * i);
                        }
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (!(seen >> (8 * (e >> 2) + 4 * hh + (e & 3)) & 1)) sc[e] = -INFINITY;
                }
                return;
            }
            if (jb > last_whole) {
                const int last = s.causal ? min(position, s.l_x - 1) : s.l_x - 1;
                const int rel = max(min(last - jb - 4 * hh, 64), -1);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (8 * (e >> 2) + (e & 3) > rel) sc[e] = -INFINITY;
            }
        };
        // B for the pairs [n0, n1) of elements 2 n, 2 n + 1: weight = 2^(c * S - m); the pair is added to the row sum
        // and rounded to bf16 into the operand fragment of C.  What a pair's instructions wait for was made with the pair before:
        // its exponents come a pair ahead of its exponentials, sum and rounding a pair behind.
        // A row that has seen no key yet (m = -inf) subtracts a huge negative number instead (m_sub), so that
        // any real score gives weight +inf and forces the fix-up, while masked scores still give 0.
        // Dropout: a decision is a chain of eight instructions, which goes over three pairs' slots: first round a pair ahead of the exponential,
        // second beside it, the rest a pair behind.  (All in one slot, with two conversions and a permutation per pair and the keys read when they
        // were due: 16 heads x 2 of 4096 rows behind 16384, 1212 us; 1134 so.)
        u32x4 ck4;      // the column keys of four consecutive elements: element e of this lane is key jb + 8 (e / 4) + 4 hh + e % 4
        uint32_t r1_0, r1_1, r2_0, r2_1;
        float x0, x1, p0, p1;
        auto load_keys = [&](int jb, int e) __attribute__((always_inline)) {
            if (DROP) ck4 = *reinterpret_cast<const u32x4 *>(ck_ring + (((jb >> 6) & 3) * C::BC + (jb & 63) + 8 * (e >> 2) + 4 * hh) * 4);
        };
        auto round1 = [&](int e) __attribute__((always_inline)) {
            r1_0 = drop_round1(drop_rk, ck4[e & 3]);
            r1_1 = drop_round1(drop_rk, ck4[(e & 3) + 1]);
        };
        auto b_pairs = [&](const f32x16 &sc, int jb, int n0, int n1, float &psum, Frag<bf16_t> (&pf)[2])
            __attribute__((always_inline)) {
            auto finish = [&](int e) __attribute__((always_inline)) {       // p0, p1: the weights of elements e, e + 1
                psum += p0;
                psum += p1;
                if (DROP) {
                    p0 = drop_decide(r2_0, dr.thr) ? p0 : 0.f;
                    p1 = drop_decide(r2_1, dr.thr) ? p1 : 0.f;
                    asm("" : "+v"(p0), "+v"(p1));       // (or each is rounded by itself ahead of the choice: five instructions for three)
                }
                pf[e >> 3].v[e & 7] = (bf16_t)p0; pf[e >> 3].v[(e & 7) + 1] = (bf16_t)p1;
            };
#pragma unroll
            for (int n = n0; n < n1; ++n) {
                if (n == 0) {
                    x0 = sc[0] * c - m_sub; x1 = sc[1] * c - m_sub;
                    if (DROP) round1(0);
                }
                const float e0 = fast_exp2(x0), e1 = fast_exp2(x1);
                if (n < 7) { x0 = sc[2 * n + 2] * c - m_sub; x1 = sc[2 * n + 3] * c - m_sub; }
                if (n > 0) finish(2 * n - 2);
                if (DROP) {
                    r2_0 = drop_round2(r1_0);
                    r2_1 = drop_round2(r1_1);
                    if (n < 7) round1(2 * n + 2);
                    if (n % 2 == 0 && n < 6) load_keys(jb, 2 * n + 4);     // (the four before are done with)
                }
                p0 = e0, p1 = e1;
                if (n == 7) finish(14);
            }
        };
        // The fix-up: raise m to the exact maximum over what the row has seen including this block,
        // rescale what was accumulated under the old m (row sum l0 before this block; accumulator,
        // to which this block has not been added yet) and redo the block's weights.
        auto fixup = [&](const f32x16 &sc, int jb, float l0, Frag<bf16_t> (&pf)[2]) __attribute__((always_inline)) {
            float mx = -INFINITY;
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[e]);
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float m_new = fmaxf(m, mx * c);
            const float alpha = (m == -INFINITY) ? 0.f : fast_exp2(m - m_new);
            m = m_new;
            m_sub = m == -INFINITY ? -1e30f : m;
            l = l0 * alpha;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[db][e] *= alpha;
            load_keys(jb, 0);
            b_pairs(sc, jb, 0, 8, l, pf);
        };

        // One pipeline step.  A: half kb2_a of its tile into sc_a.  B: sc_b, first key jb_b, packing
        // into pf_b.  C: half kb2_c of its tile from pf_c into o.  Per unit the matrix instructions
        // go C, A (A, C in the last unit); after each one come the B elements that fall to its slot.  Operand fragments are
        // read from LDS one unit ahead of their use; those of the first unit by the step before
        // (ak[0], cv[0] on entry), and this step leaves there those of the next step: halves kb2_an and kb2_cn.  `mid` runs
        // before those last reads: the even steps put the loop's barrier there, because the next step's blocks may lie in the
        // tile that the barrier publishes, and move the addresses on.
        // Pages: V of a tile that drafted tokens are in, once it has landed and ahead of the barrier that shows it to the others: 0 in the place of values that are not
        // finite, of the rows that this wavefront loaded.  0 times such a value is NaN, and not all rows see it; those that do get it at the end.
        const auto clean = [&](char *pair_slot, int t) __attribute__((always_inline)) {
            if constexpr (PAGED) {
                if ((t + 1) * C::BC <= s.first) return;
                bool some = false;
#pragma unroll
                for (int i = 0; i < Tile::NI; ++i) {
                    bf16x8 *const at = reinterpret_cast<bf16x8 *>(pair_slot + C::OFF_V + (wave * Tile::NI + i) * 1024 + lane * 16);
                    const bf16x8 v = *at, kept = finite_part(v);
                    const u32x4 x = __builtin_bit_cast(u32x4, v), y = __builtin_bit_cast(u32x4, kept);
                    some = some || x[0] != y[0] || x[1] != y[1] || x[2] != y[2] || x[3] != y[3];
                    *at = kept;
                }
                if (__any(some) && lane == 0) *s.spoilt = 1;
                wait_lds_reads();
            }
        };
        Frag<bf16_t> ak[2], cv[2];
        auto step = [&](auto has_a, auto has_b, auto has_c, int kb2_a, f32x16 &sc_a, f32x16 &sc_b,
                        int jb_b, Frag<bf16_t> (&pf_b)[2], int kb2_c, Frag<bf16_t> (&pf_c)[2], int kb2_an, int kb2_cn, auto &&mid)
            __attribute__((always_inline)) {
            constexpr bool HA = decltype(has_a)::value, HB = decltype(has_b)::value, HC = decltype(has_c)::value;
            constexpr int NS = 2 * NU;                  // slots; the 8 element pairs of B spread over them
            static_assert(NU % 2 == 0, "fragment double buffers assume an even number of units");
            const float l0 = l;
            auto b_slot = [&](int slot) __attribute__((always_inline)) {
                if (HB) {
                    __builtin_amdgcn_sched_barrier(0);
                    b_pairs(sc_b, jb_b, slot * 8 / NS, (slot + 1) * 8 / NS, l, pf_b);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            if (HB) {
                load_keys(jb_b, 0);
                mask_s(jb_b, sc_b);
                // B's inputs pass through an empty asm here: its arithmetic depends on nothing else in
                // this step, and the compiler would otherwise move all of it out of the step, in one lump
                asm volatile("" : "+v"(sc_b));
            }
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                const int half = u / (D / 32), db = u % (D / 32);
                if (u + 1 < NU) {
                    if (HC) load_c(kb2_c, u + 1, cv[(u + 1) & 1]);
                    if (HA) load_a(kb2_a, u + 1, ak[(u + 1) & 1]);
                    __builtin_amdgcn_sched_barrier(0);
                    wait_lds<(HC ? 2 : 0) + (HA ? 1 : 0)>();        // this unit's are there
                    __builtin_amdgcn_sched_barrier(0);
                    if (HC) o[db] = mma(cv[u & 1], pf_c[half], o[db]);
                    b_slot(2 * u);
                    if (HA) sc_a = mma(ak[u & 1], qf[u], u == 0 ? zero16 : sc_a);
                    b_slot(2 * u + 1);
                } else {
                    // last unit: A first, so that its result is there when the next step's B wants it
                    if (HA) sc_a = mma(ak[u & 1], qf[u], sc_a);
                    b_slot(2 * u);
                    mid();
                    load_c(kb2_cn, 0, cv[0]);
                    load_a(kb2_an, 0, ak[0]);
                    __builtin_amdgcn_sched_barrier(0);
                    if (HC) o[db] = mma(cv[u & 1], pf_c[half], o[db]);
                    b_slot(2 * u + 1);
                }
            }
            if (HB) {
                // ... and its results through another one, so that it is not sunk below the step either
                asm volatile("" : "+v"(pf_b[0].v), "+v"(pf_b[1].v), "+v"(l));
                if (__any(!(l - l0 <= C::kMaxBlockSum))) fixup(sc_b, jb_b, l0, pf_b);
            }
        };
        using std::true_type;
        using std::false_type;

        // ---- pipeline.  Block g = keys (t_begin + g/2) * 64 + (g%2) * 32 ..; tile t = blocks 2t, 2t+1.
        if (T > 0) {
            issue_next(ring);                           // (K of tile 0; its V here is overwritten before anybody reads it)
            advance_k();
            issue_next(ring + C::PAIR);
            advance_k();
            advance_v();
        }
        wait_vmem_all();
        __syncthreads();

        if (rw0 >= s.l_s) {
            // None of this wavefront's rows exists (a partly filled last query tile): it only keeps moving
            // tiles and meeting the loop's barriers.
            for (int t = 0; t < T; ++t) {
                wait_vmem_all();
                clean(ring + ((t & 1) ^ 1) * C::PAIR, t_begin + t);
                __syncthreads();
                issue_next(ring + (t & 1) * C::PAIR);
                advance_k();
                advance_v();
            }
        } else if (T > 0) {
            f32x16 sc0, sc1;                            // even / odd blocks
            Frag<bf16_t> pf0[2], pf1[2];
            // step -1: A(0) alone.  The first loop step has no C(-1): it multiplies zeros with tile 0 instead.
            load_a(0, 0, ak[0]);
            auto nothing = [] {};
            step(true_type{}, false_type{}, false_type{}, 0, sc0, sc1, 0, pf0, 0, pf1, 1, 1, nothing);
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int e = 0; e < 8; ++e) pf1[half].v[e] = (bf16_t)0.f;

            // the pair slot (bytes) of K of tile t and V of tile t - 1, and the way to that of K of t + 1 and V of t
            int slot = 0, other = C::PAIR;
            int j0 = t_begin * C::BC;
            for (int t = 0; t < T; ++t) {
                // even step g = 2t: A(2t+1) [tile t, second half], B(2t), C(2t-1) [tile t-1, second half;
                // for t = 0 V of tile 0, which lies in both slots, times zero]
                // Before its last reads (which may touch tile t+1): K of tile t+1 and V of tile t, issued one iteration
                // ago, have landed for this wavefront; after the barrier for all, and every wavefront has
                // requested its last operands from K of tile t and V of tile t-1.
                step(true_type{}, true_type{}, true_type{}, 1, sc1, sc0, j0, pf0, 1, pf1, 0, 0, [&] {
                    wait_vmem_all();
                    clean(ring + slot + other, t_begin + t);
                    __syncthreads();
                    issue_next(ring + slot);
#pragma unroll
                    for (int kb = 0; kb < NU; ++kb) a_at[kb] += other;
#pragma unroll
                    for (int db = 0; db < D / 32; ++db) { t_at[db][0] += other; t_at[db][1] += other; }
                });
                if constexpr (PAGED)                    // (zeros times a first value that is not finite)
                    if (t == 0)
#pragma unroll
                        for (int db = 0; db < D / 32; ++db) o[db] = zero16;
                // odd step g = 2t+1: A(2t+2) [tile t+1, first half; past the end of whatever its slot holds, result unused],
                // B(2t+1), C(2t) [tile t, first half]
                step(true_type{}, true_type{}, true_type{}, 0, sc0, sc1, j0 + 32, pf1, 0, pf0, 1, 1, nothing);
                advance_k();
                advance_v();
                slot += other, other = -other;
                j0 += C::BC;
            }
            // step 2T: C(2T-1) [tile T-1, second half] alone
            step(false_type{}, false_type{}, true_type{}, 0, sc0, sc0, 0, pf0, 1, pf1, 0, 1, nothing);
        }
        if (KG > 1)
            for (int t = T; t < iters; ++t) __syncthreads();           // the barriers of the groups that have more tiles
        wait_vmem_all();                                // the last, redundant prefetches must land before the workgroup's LDS is given away
    }
    if constexpr (PAGED) {
        // values that are not finite in the tiles that drafted tokens are in, to the rows that see them: their weights are above 0, whatever they are (what joins parts keeps that: add_scaled)
        if (s_tiles > 0 && *s.spoilt && rw0 < s.l_s) {
            const int token = min(r, s.l_s - 1) / G;
            for (int key = max(max(s.first, 0) / C::BC, s_begin) * C::BC; key < min(s.l_x, (s_begin + s_tiles) * C::BC); ++key) {
                const uint32_t page = (uint32_t)s.table[key >> s.a->pt.page_shift];
                const bool sees = page < (uint32_t)s.a->pt.n_pages && (keys_seen(*s.a, s.bits + (int64_t)token * s.a->words, token, key - s.first) & 1);
                if (!sees) continue;
                const int64_t row = ((int64_t)page << s.a->pt.page_shift) + (key & ((1 << s.a->pt.page_shift) - 1));
                const bf16_t *const value = reinterpret_cast<const bf16_t *>(s.v_head + row * (s.a->H_kv * D * 2)) + 4 * hh;
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int e4 = 0; e4 < 4; ++e4) {
                        const bf16x4 x = *reinterpret_cast<const bf16x4 *>(value + 32 * db + 8 * e4);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!(fabsf((float)x[e]) < INFINITY)) o[db][4 * e4 + e] += (float)x[e];
                    }
            }
        }
    }

    const float l_own = l + __shfl_xor(l, 32);
    const float kept = DROP ? dr.scale : 1.f;           // of the kept weights: applied to their sum
    const auto has_sum = [](float sum) { return PACKED ? sum != 0.f : sum > 0.f; };    // (packed: a NaN among the scores is one in lse)
    if constexpr (KG == 1) {
        const float inv = l_own > 0.f ? kept / l_own : 0.f;
        if (!row_ok) return;
        if (hh == 0) put_lse(has_sum(l_own) ? (m + log2f(l_own)) * kLn2 : -INFINITY);
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4)
                put(db * 4 + e4, f32x4{o[db][4 * e4] * inv, o[db][4 * e4 + 1] * inv, o[db][4 * e4 + 2] * inv, o[db][4 * e4 + 3] * inv});
    } else {
        // The groups' results meet in LDS, where the tiles were: group g adds up its share of the columns, in group order,
        // weighted to the rows' maximum over all groups.
        auto hand = [&](int g, int u) { return reinterpret_cast<f32x4 *>(smem + ((g * RB + wave) * C::UNITS + u) * 1024 + lane * 16); };
        auto hand_ml = [&](int g) { return reinterpret_cast<float *>(smem + C::HAND_ML + (g * RB + wave) * 512 + lane * 8); };
        __syncthreads();
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4)
                *hand(group, db * 4 + e4) = f32x4{o[db][4 * e4], o[db][4 * e4 + 1], o[db][4 * e4 + 2], o[db][4 * e4 + 3]};
        hand_ml(group)[0] = m;
        hand_ml(group)[1] = l_own;
        __syncthreads();
        if (!row_ok) return;
        float mg[KG], m_all = -INFINITY, l_all = 0.f;
#pragma unroll
        for (int g = 0; g < KG; ++g) { mg[g] = hand_ml(g)[0]; m_all = fmaxf(m_all, mg[g]); }
#pragma unroll
        for (int g = 0; g < KG; ++g) {
            mg[g] = mg[g] == -INFINITY ? 0.f : fast_exp2(mg[g] - m_all);       // from here on: its weight
            l_all += mg[g] * hand_ml(g)[1];
        }
        const float inv = l_all > 0.f ? kept / l_all : 0.f;
        if (group == 0 && hh == 0) put_lse(has_sum(l_all) ? (m_all + log2f(l_all)) * kLn2 : -INFINITY);
        constexpr int PER = C::UNITS / KG;
        static_assert(C::UNITS % KG == 0, "");
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int u = group * PER + i;
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < KG; ++g) {
                const f32x4 v = *hand(g, u);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += mg[g] * v[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] *= inv;
            put(u, sum);
        }
    }
}

template <int D, bool DROP, int RB, int KG>
__global__ __launch_bounds__(64 * RB * KG, D == 64 ? 2 : 1) void fwd_bf16_kernel(SegShape s, DropArgs dr, const bf16_t *__restrict__ q,
                                                                       const bf16_t *__restrict__ k,
                                                                       const bf16_t *__restrict__ v,
                                                                       bf16_t *__restrict__ out, float *__restrict__ lse,
                                                                       float *__restrict__ o_part,
                                                                       float *__restrict__ lse_part, int n_splits, int n_q_tiles)
{
    using C = FwdBf16Cfg<D, RB, KG>;
    __shared__ __attribute__((aligned(1024))) char smem[C::lds(DROP)];
    // 1-D grid in XCD order (xcd_item): one head at a time per XCD, whose workgroups share its K and
    // V in that XCD's L2.  Within a head: query tiles, last first -- under the causal mask the last
    // tiles see the most keys, and starting the longest workgroups first shortens the tail of the
    // launch -- then key splits.
    const int bhs = s.B * s.H;
    int bh, inner;
    if (!xcd_item(blockIdx.x, bhs, n_q_tiles * n_splits, s.causal && s.s0 < s.l_s, bh, inner)) return;
    const int b = bh / s.H, h = bh % s.H;
    const int q_tile = inner % n_q_tiles, split = inner / n_q_tiles;
    const int r0 = (n_q_tiles - 1 - q_tile) * C::BR;
    const int64_t ld = (int64_t)s.H * D, head = (int64_t)h * D;
    const FwdView view{q + (int64_t)b * s.l_s * ld + head, k + (int64_t)b * s.l_x * ld + head, v + (int64_t)b * s.l_x * ld + head, ld, ld, ld, s.s0, s.l_s,
                       s.l_x, s.causal, 1};
    // this lane's row of the result (a split's normalised output travels to the merge kernel in fp32: rounded to bf16 once, there)
    const int lane = threadIdx.x & 63, r = r0 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % RB * C::RW + (lane & 31), hh = lane >> 5;
    const int64_t part_row = ((int64_t)split * bhs + bh) * s.l_s + r;
    fwd_bf16_body<D, DROP, RB, KG, false>(
        smem, view, dr, bh, r0, split, n_splits,
        [&](int u, const f32x4 &val) __attribute__((always_inline)) {
            if (n_splits == 1)
                *reinterpret_cast<bf16x4 *>(out + ((int64_t)b * s.l_s + r) * ld + (int64_t)h * D + 8 * u + 4 * hh) = pack4(val[0], val[1], val[2], val[3]);
            else *reinterpret_cast<f32x4 *>(o_part + part_row * D + 8 * u + 4 * hh) = val;
        },
        [&](float v) {
            if (n_splits == 1) lse[(int64_t)bh * s.l_s + r] = v;
            else lse_part[part_row] = v;
        });
}

// Packed sequences (lss_packed_attn_fwd).  A row of a workgroup is a query head of a token: the G heads that share a head of keys and values are
// neighbours, so that a tile of keys serves 128 / G tokens of all of them, the causal diagonal crosses fewer of a wavefront's blocks,
// and short prompts fill the rows.  Matrix and vector work bound it, as in a segment: 24,576 rows, 16 heads of 64, 4 of keys 1.21 ms (1020 TFLOP/s, matrix units
// busy 60 % of the cycles, vector ALU 86 %); nine prompts of 205 to 4108 rows, 32 heads of 128, 8 of keys 248 us (911; 49 and 48 %: one in ten of a tile's
// cycles is its start and end, and short prompts' last tiles of keys are half masked).  Weights are rounded to bf16 before they multiply the values (off by at most 2^-8
// of each): two parts, as for single tokens, would be half as much matrix work again.
template <int D, int RB, int KG, bool SPLIT>
__global__ __launch_bounds__(64 * RB * KG, D == 64 ? 2 : 1) void packed_bf16_kernel(PackedArgs a, const bf16_t *__restrict__ q, const bf16_t *__restrict__ k,
                                                                                   const bf16_t *__restrict__ v, bf16_t *__restrict__ out,
                                                                                   float *__restrict__ lse, PackedParts parts, int n_tiles)
{
    using C = FwdBf16Cfg<D, RB, KG>;
    __shared__ __attribute__((aligned(1024))) char smem[C::lds(false)];
    const int lane = threadIdx.x & 63, lq = lane & 31, hh = lane >> 5, G = a.H / a.H_kv;
    int h_kv, rank;
    if (!xcd_item(blockIdx.x, a.H_kv, SPLIT ? n_tiles * parts.splits : n_tiles, a.causal != 0, h_kv, rank)) return;
    const int split = SPLIT ? rank % parts.splits : 0;
    if (SPLIT) rank /= parts.splits;
    PackedTile t;
    if (!packed_tile<C::BR>(a, G, rank, lane, t)) return;
    const FwdView view{q + (int64_t)t.q_begin * a.q_stride + (int64_t)h_kv * G * D, k + (int64_t)t.k_begin * a.k_stride + (int64_t)h_kv * D,
                       v + (int64_t)t.k_begin * a.v_stride + (int64_t)h_kv * D, a.q_stride, a.k_stride, a.v_stride, t.n_k - t.n_q, t.n_q * G, t.n_k, a.causal, G};
    const int r0 = t.tile * C::BR, rw0 = r0 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % RB * C::RW, r = rw0 + lq;
    const int token = t.q_begin + r / G, h = h_kv * G + r % G;
    bf16_t *const row = out + ((int64_t)token * a.H + h) * D;
    bool finite = true;
    fwd_bf16_body<D, false, RB, KG, true>(
        smem, view, DropArgs{}, 0, r0, split, SPLIT ? parts.splits : 1,
        [&](int u, const f32x4 &val) __attribute__((always_inline)) {
            if (SPLIT) {
                *reinterpret_cast<f32x4 *>(parts.values(a, split, token, h) + 8 * u + 4 * hh) = val;
                return;
            }
            *reinterpret_cast<bf16x4 *>(row + 8 * u + 4 * hh) = pack4(val[0], val[1], val[2], val[3]);
            finite = finite && fabsf(val[0]) < INFINITY && fabsf(val[1]) < INFINITY && fabsf(val[2]) < INFINITY && fabsf(val[3]) < INFINITY;
        },
        [&](float v) {
            if (SPLIT) *parts.lse(a, split, token, h) = v;
            else lse[(int64_t)h * a.rows_q + token] = v;
        });
    // A key's weight is 0 for the rows of its block that do not see it, but 0 times a value that is not finite is NaN: rows with such a result are done over,
    // over the keys that they see alone (of a tile whose keys are split: by packed_merge_kernel).  Not where lse is NaN: lse is made of the scores of seen keys alone.
    if (SPLIT) return;
    if (KG > 1) __syncthreads();                // (the groups have written parts of one row)
    const uint64_t bad = __ballot(!finite);
    for (uint32_t rows = (uint32_t)bad | (uint32_t)(bad >> 32); rows != 0; rows &= rows - 1) {
        const int again = rw0 + __builtin_ctz(rows), at = again / G, head = h_kv * G + again % G;
        const int seen = a.causal ? max(0, min(t.n_k, t.n_k - t.n_q + at + 1)) : t.n_k;
        const float row_lse = lse[(int64_t)head * a.rows_q + t.q_begin + at];
        if (row_lse != row_lse) continue;
        row_attention<bf16_t, D, 8>(view.q + (int64_t)at * a.q_stride + again % G * D, view.k, a.k_stride, view.v, a.v_stride, seen, row_lse, lane,
                                 out + ((int64_t)(t.q_begin + at) * a.H + head) * D);
    }
}

// Drafted tokens over a paged cache (lss_paged_attn_tree): rows as above, keys and values from pages.
// WHOLE: a workgroup per tile of 128 rows, those with the most keys first; else per part of a tile's keys (tree_part), joined by a second launch.
//   48 sequences of 2048 to 6500 tokens, 64 drafted, 32 heads of 128, 8 of keys, 917 MB, 2.1e11 flop: 266 to 284 us by box, 780 TFLOP/s, matrix units busy 45 % and vector ALU 41 % of the cycles: a SIMD's two
// wavefronts take turns, as over contiguous keys (261).  1001 rows of a chain behind 23,000 tokens, 16 heads of 64, 4 of keys: 128 to 131 us, vector ALU 68 %.  24 sequences of up to 8192, trees of 4 to 12,
// 112 MB: 30.7 us, 3.9 TB/s, 9 of them until the first tile is there.  Weights are rounded to bf16 (off by at most 2^-8 of each), as for packed prompts.
template <int D, bool WHOLE>
__global__ __launch_bounds__(256, 2) void tree_bf16_kernel(TreeArgs a, const bf16_t *__restrict__ q, const bf16_t *__restrict__ k_cache,
                                                          const bf16_t *__restrict__ v_cache, bf16_t *__restrict__ out, float *__restrict__ lse,
                                                          float *__restrict__ scratch, int n_tiles, int target, int most, int least, int slots, int chains)
{
    using C = FwdBf16Cfg<D, 4, 1>;
    __shared__ __attribute__((aligned(1024))) char smem[C::lds(false)];
    __shared__ int spoilt;
    const int lane = threadIdx.x & 63, lq = lane & 31, hh = lane >> 5, G = a.H / a.H_kv;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const TreeScratch parts{scratch, C::BR, D, slots, chains};
    TreePart p;
    if constexpr (WHOLE) {
        int rank;
        if (!xcd_item(blockIdx.x, a.H_kv, n_tiles, true, p.h_kv, rank)) return;
        PackedTile t;
        if (!packed_tile<C::BR>(a, G, rank, lane, t)) return;
        p.b = t.b, p.tile = t.tile, p.begin = t.q_begin, p.n = t.n_q, p.length = t.n_k, p.r0 = 0, p.r1 = (t.n_k + C::BC - 1) / C::BC, p.count = 1, p.slot = 0;
    } else {
        static_assert(C::BC == tree_round(2, true), "");
        const bool some = tree_part<C::BC, C::BR>(a, lane, blockIdx.x, target, most, least, gridDim.x, p);
        if (threadIdx.x == 0) parts.enter(p, some);
        if (!some) return;
    }
    if (threadIdx.x == 0) spoilt = 0;
    __syncthreads();
    PagedView view;
    view.q = q + (int64_t)p.begin * a.q_stride + (int64_t)p.h_kv * G * D;
    view.q_ld = a.q_stride;
    view.k = view.v = nullptr;
    view.k_ld = view.v_ld = 0;
    view.s0 = view.first = p.length - p.n;
    view.l_s = p.n * G;
    view.l_x = p.length;
    view.causal = a.tree == nullptr;
    view.G = G;
    view.a = &a;
    view.table = a.pt.table + (int64_t)p.b * a.pt.max_pages;
    view.k_head = reinterpret_cast<const char *>(k_cache + (int64_t)p.h_kv * D);
    view.v_head = reinterpret_cast<const char *>(v_cache + (int64_t)p.h_kv * D);
    view.bits = a.tree + (int64_t)p.begin * a.words;
    view.t0 = p.r0;
    view.t1 = p.r1;
    view.spoilt = &spoilt;
    const int in_tile = wave * C::RW + lq, r = p.tile * C::BR + in_tile, token = p.begin + r / G, h = p.h_kv * G + r % G;
    const bool all = WHOLE || p.count == 1;
    fwd_bf16_body<D, false, 4, 1, true>(
        smem, view, DropArgs{}, 0, p.tile * C::BR, 0, 1,
        [&](int u, const f32x4 &val) __attribute__((always_inline)) {
            if (all) *reinterpret_cast<bf16x4 *>(out + ((int64_t)token * a.H + h) * D + 8 * u + 4 * hh) = pack4(val[0], val[1], val[2], val[3]);
            else *reinterpret_cast<f32x4 *>(parts.values(p.slot, in_tile) + 8 * u + 4 * hh) = val;
        },
        [&](float v) {
            if (all) {
                lse[(int64_t)token * a.H + h] = v;
                return;
            }
            parts.sums(p.slot, in_tile)[0] = v * kLog2e;
            parts.sums(p.slot, in_tile)[1] = v == -INFINITY ? 0.f : 1.f;
        });
}

hipError_t launch_tree_bf16_main(const TreeArgs &a, const TreePlan &p, const bf16_t *q, const bf16_t *k_cache, const bf16_t *v_cache, bf16_t *out, float *lse, float *scratch,
                                 hipStream_t st)
{
    const int n_tiles = (int)((int64_t)a.rows * (a.H / a.H_kv) / 128) + (a.B <= 64 && a.rows < a.B ? a.rows : a.B);
    TimedLaunch tl(K_TREE_BF16, st);
    const dim3 grid((unsigned)(p.slots == 0 ? xcd_grid(a.H_kv, n_tiles) : (p.most + p.tiles + 7) / 8 * 8)), block(256);
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a, q, k_cache, v_cache, out, lse, scratch, n_tiles, p.target, p.most, p.least, p.slots, p.chains); };
    if (a.d == 64) p.slots == 0 ? go(tree_bf16_kernel<64, true>) : go(tree_bf16_kernel<64, false>);
    else p.slots == 0 ? go(tree_bf16_kernel<128, true>) : go(tree_bf16_kernel<128, false>);
    return hipGetLastError();
}

int fwd_bf16_rows_per_workgroup(int d) { return d == 64 ? 128 : 256; }

template <int D, int RB, int KG>
static hipError_t launch_fwd_main(const SegShape &s, const DropArgs &drop, const bf16_t *q, const bf16_t *k,
                                  const bf16_t *v, bf16_t *out, float *lse, const Workspace &ws, int n_splits, hipStream_t st)
{
    using C = FwdBf16Cfg<D, RB, KG>;
    const int n_q_tiles = (s.l_s + C::BR - 1) / C::BR;
    dim3 grid((unsigned)xcd_grid(s.B * s.H, n_q_tiles * n_splits));
    auto kernel = fwd_bf16_kernel<D, false, RB, KG>;
    if (drop.thr != 0) {
        if constexpr (D == 64 && RB == 4 && KG == 2) return hipErrorInvalidConfiguration;      // (pick_fwd_plan: never with dropout)
        else kernel = fwd_bf16_kernel<D, true, RB, KG>;
    }
    TimedLaunch tl(K_FWD_BF16, st);
    hipLaunchKernelGGL(kernel, grid, dim3(C::NT), 0, st, s, drop, q, k, v, out, lse, ws.o_part, ws.lse_part, n_splits, n_q_tiles);
    return hipGetLastError();
}

hipError_t launch_fwd_bf16_main(const SegShape &s, const DropArgs &drop, const bf16_t *q, const bf16_t *k,
                                const bf16_t *v, bf16_t *out, float *lse, const Workspace &ws, const FwdPlan &plan, hipStream_t st)
{
    if (s.d == 64) {
        switch (plan.form) {
        case FWD_2x2: return launch_fwd_main<64, 2, 2>(s, drop, q, k, v, out, lse, ws, plan.splits, st);
        case FWD_4x2: return launch_fwd_main<64, 4, 2>(s, drop, q, k, v, out, lse, ws, plan.splits, st);
        case FWD_2x4: return launch_fwd_main<64, 2, 4>(s, drop, q, k, v, out, lse, ws, plan.splits, st);
        case FWD_1x4: return launch_fwd_main<64, 1, 4>(s, drop, q, k, v, out, lse, ws, plan.splits, st);
        default: return launch_fwd_main<64, 4, 1>(s, drop, q, k, v, out, lse, ws, plan.splits, st);
        }
    }
    if (plan.form == FWD_4x2) return launch_fwd_main<128, 4, 2>(s, drop, q, k, v, out, lse, ws, plan.splits, st);
    return launch_fwd_main<128, 8, 1>(s, drop, q, k, v, out, lse, ws, plan.splits, st);
}

template <int D, int RB, int KG, bool SPLIT = false>
static hipError_t launch_packed(const PackedArgs &a, const bf16_t *q, const bf16_t *k, const bf16_t *v, bf16_t *out, float *lse, const PackedParts &parts,
                                hipStream_t st)
{
    using C = FwdBf16Cfg<D, RB, KG>;
    const int n_tiles = packed_tiles(a, C::BR);
    TimedLaunch tl(K_PACKED_BF16, st);
    hipLaunchKernelGGL((packed_bf16_kernel<D, RB, KG, SPLIT>), dim3((unsigned)xcd_grid(a.H_kv, n_tiles * parts.splits)), dim3(C::NT), 0, st, a, q, k, v, out, lse,
                       parts, n_tiles);
    return hipGetLastError();
}

hipError_t launch_packed_bf16_main(const PackedArgs &a, const PackedPlan &f, const bf16_t *q, const bf16_t *k, const bf16_t *v, bf16_t *out, float *lse,
                                   const PackedParts &parts, hipStream_t st)
{
    const auto is = [&](int row_blocks, int groups) { return f.row_blocks == row_blocks && f.groups == groups; };
    if (parts.splits > 1)        // (with splits: always this form)
        return a.d == 64 ? launch_packed<64, 2, 2, true>(a, q, k, v, out, lse, parts, st) : launch_packed<128, 2, 2, true>(a, q, k, v, out, lse, parts, st);
    if (a.d == 64) {
        if (is(2, 1)) return launch_packed<64, 2, 1>(a, q, k, v, out, lse, parts, st);
        if (is(2, 2)) return launch_packed<64, 2, 2>(a, q, k, v, out, lse, parts, st);
        if (is(4, 2)) return launch_packed<64, 4, 2>(a, q, k, v, out, lse, parts, st);
        if (is(2, 4)) return launch_packed<64, 2, 4>(a, q, k, v, out, lse, parts, st);
        if (is(1, 4)) return launch_packed<64, 1, 4>(a, q, k, v, out, lse, parts, st);
        return launch_packed<64, 4, 1>(a, q, k, v, out, lse, parts, st);
    }
    if (is(2, 2)) return launch_packed<128, 2, 2>(a, q, k, v, out, lse, parts, st);
    if (is(4, 2)) return launch_packed<128, 4, 2>(a, q, k, v, out, lse, parts, st);
    if (is(8, 1)) return launch_packed<128, 8, 1>(a, q, k, v, out, lse, parts, st);
    return launch_packed<128, 4, 1>(a, q, k, v, out, lse, parts, st);
}

} // namespace lss
