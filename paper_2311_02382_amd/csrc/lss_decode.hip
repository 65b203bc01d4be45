// Attention of one token per sequence over a paged cache of keys and values.
//
// A sequence's keys and values are read once by every group of up to 32 query heads that share their head (so once, but for more than 32 of them): what bounds it is
// those bytes.  Work is counted in rounds of one tile per wavefront (4 x 32 keys in bf16, 4 x 16 in float); the
// rounds of all sequences and heads, one behind the other, are dealt out in equal parts to as many workgroups as the chip holds at once, so that
// sequences of any lengths fill it evenly.  A part that is not all of its sequence goes to scratch memory, two at most per
// workgroup (its first and its last), and a second launch of 4 to 5 us joins those (decode_merge_kernel).  Where no sequence is long
// (kWholeLen), a workgroup takes all of one and there is no second launch.
//
// Within a round each wavefront is by itself: a tile's keys go from memory to the registers that the matrix instructions
// S^T = K Q^T read, its values through registers to LDS (wavefront's own: no barrier), from where O^T += V^T P^T reads them
// transposed.  The next tile's loads are issued as soon as the registers are free, and are on their way while the weights are
// computed; the other wavefronts of the compute unit hide what is left.
//
// Softmax: one query per lane (four lanes share it, with the keys among them); the running maximum is raised only where a score exceeds it by more than 2^8
// in weight.  A bf16 weight would lose 16 bits before it multiplies a value; the matrix cores have time to spare here (busy for 7 % of a large call), so that
// weights go in as two bf16 parts (error 2^-16) and the only rounding to bf16 is the result's.  The first part is cut off, not rounded, and the second is not 0 where the weight is not:
// both are positive, so that an infinite value gives infinity as the definition has it, not the NaN of parts of either sign or of 0 times it.
//
// 128 sequences of 2048 to 6500 tokens, 8 heads of 128 for 32, 2.07 GB: 336 us, 6.2 TB/s (plain reads of as much: 7.06; with one head of keys, whose rows
// lie one behind the other, 6.5); 76 MB in 24 ragged sequences 21.0 us, of which the first loads of a workgroup take 5 and the second launch 4,
// and whole rounds: 1296 of them for 512 workgroups, 432 of which take three and 80 none.
// Built, measured and longer: the heads of a sequence side by side in neighbouring workgroups (the same tokens at the same time: 357 us against
// 338 for the large one); at d = 64 two tiles on their way and three workgroups a compute unit instead of four (98 sequences in float 172 us, 153); at d = 128 three
// workgroups (registers to memory: 490) -- or two tiles on their way, likewise.
#include "lss_bf16.h"
#include "lss_serve.h"

#include <algorithm>

namespace lss {

namespace {

constexpr int kWaves = 4, kWholeLen = 512;

// Large calls' keys and values pass the last-level cache (256 MB) by, with non-temporal loads: 2.07 GB 378 -> 347 us, 268 MB 58.6 -> 53.1 with the first kernel that
// had them.  From where?  Read again right away, calls gain from it up to its size (76 MB: 21.9 us, past it 23.3); after three or more others
// of their size, as in a model of many layers, from 40 MB on they gain from staying out (41 MB: 18.2 -> 17.5, 111 MB: 30.6 -> 29.0, 196 MB: 54.6 -> 50.8).
constexpr int64_t kStreamBytes = (int64_t)96 << 20;
// Buffer loads: a lane past the end of the `bytes` from `first` on gets zeros and moves nothing -- the rows of a tile behind a sequence's last token, and those
// of a page that is none.
template <bool STREAM, typename V>
__device__ __forceinline__ V load16(__amdgpu_buffer_rsrc_t buffer, uint32_t offset)
{
    return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(buffer, (int)offset, 0, STREAM ? 2 : 0));       // (2: non-temporal)
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const char *first, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(first), 0, (int)bytes, 0x00020000);       // (raw, 32-bit data)
}

// how a tile's keys and values meet the matrix cores
template <typename T, int D> struct Step;

template <int D> struct Step<bf16_t, D> {
    static constexpr int TILE = 32, NQ_FRAGS = D / 32, V_LOADS = TILE * D * 2 / 1024, CHUNKS = D / 8;
    typedef bf16x8 Vec;
    struct Queries { Frag<bf16_t> f[NQ_FRAGS]; };       // 16 of them: lane's is l % 16, columns 32 i + 8 (l / 16) ..
    struct Keys { Frag<bf16_t> f[2][NQ_FRAGS]; };
    static __device__ __forceinline__ void load_query(Queries &q, const bf16_t *row, int g, bool there)
    {
#pragma unroll
        for (int i = 0; i < NQ_FRAGS; ++i) {
            q.f[i].v = bf16x8{};
            if (there) q.f[i] = load_frag<bf16_t>(row + 32 * i + 8 * g);
        }
    }
    // half i of a tile: 16 keys, this lane's 16 bytes of the first step at lane_offset
    template <bool STREAM>
    static __device__ __forceinline__ void load_keys(Keys &k, int i, __amdgpu_buffer_rsrc_t half, uint32_t lane_offset)
    {
#pragma unroll
        for (int j = 0; j < NQ_FRAGS; ++j) k.f[i][j].v = load16<STREAM, Vec>(half, lane_offset + 64 * j);
    }
    // element e of half i: key 16 i + 4 (l / 16) + e, query l % 16
    static __device__ __forceinline__ f32x4 scores(const Keys &k, int i, const Queries &q)
    {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NQ_FRAGS; ++j) s = mma16(k.f[i][j], q.f[j], s);
        return s;
    }
    static __device__ __forceinline__ void store_value(char *tile, int row, int chunk, const Vec &v)
    {
        *reinterpret_cast<Vec *>(tile + DirectTile<D, 64>::chunk_offset(row, chunk)) = v;
    }
    static __device__ __forceinline__ f32x4 values4(const char *tile, int row, int column)     // four neighbouring columns
    {
        const bf16x4 v = *reinterpret_cast<const bf16x4 *>(tile + DirectTile<D, 64>::chunk_offset(row, column / 8) + column % 8 * 2);
        return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
    }
    // o[n][db] += V^T P^T, element v of o[n][db]: column 16 db + 4 (l / 16) + v of query l % 16
    template <int NQ>
    static __device__ __forceinline__ void add_values(const char *tile, const f32x4 (&p)[NQ][2], f32x4 (&o)[NQ][D / 16], int lane)
    {
        Frag<bf16_t> hi[NQ], lo[NQ];
        const float smallest = 0x1p-126f;               // (of a weight that is not 0; the median is max(w - cut, min(w, smallest)))
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float w = p[n][e >> 2][e & 3], cut = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, w) & 0xffff0000u);
                hi[n].v[e] = (bf16_t)cut;
                lo[n].v[e] = (bf16_t)__builtin_amdgcn_fmed3f(w - cut, w, smallest);
            }
#pragma unroll
        for (int db = 0; db < D / 16; ++db) {
            const Frag<bf16_t> v = load_frag_tr16_sw<D>(tile, 0, tr16_lane_offset_sw<D>(lane, db));
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                o[n][db] = mma16(v, lo[n], o[n][db]);
                o[n][db] = mma16(v, hi[n], o[n][db]);
            }
        }
    }
};

template <int D> struct Step<float, D> {
    static constexpr int TILE = 16, NQ_FRAGS = D / 16, V_LOADS = TILE * D * 4 / 1024, CHUNKS = D / 4;
    typedef f32x4 Vec;
    struct Queries { f32x4 f[NQ_FRAGS]; };
    struct Keys { f32x4 f[1][NQ_FRAGS]; };
    static __device__ __forceinline__ void load_query(Queries &q, const float *row, int g, bool there)
    {
#pragma unroll
        for (int i = 0; i < NQ_FRAGS; ++i) {
            q.f[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (there) q.f[i] = *reinterpret_cast<const f32x4 *>(row + 16 * i + 4 * g);
        }
    }
    template <bool STREAM>
    static __device__ __forceinline__ void load_keys(Keys &k, int i, __amdgpu_buffer_rsrc_t half, uint32_t lane_offset)
    {
#pragma unroll
        for (int j = 0; j < NQ_FRAGS; ++j) k.f[i][j] = load16<STREAM, Vec>(half, lane_offset + 64 * j);
    }
    static __device__ __forceinline__ f32x4 scores(const Keys &k, int i, const Queries &q)
    {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NQ_FRAGS; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k.f[i][j][e], q.f[j][e], s, 0, 0, 0);
        return s;
    }
    // rows of D floats; every fourth one begins 16 banks further on, so that the four rows that one read takes a float of are apart
    static __device__ __forceinline__ int at(int row, int column) { return (row * D + (column ^ ((row >> 2 & 3) << 4))) * 4; }
    static __device__ __forceinline__ void store_value(char *tile, int row, int chunk, const Vec &v)
    {
        *reinterpret_cast<Vec *>(tile + at(row, 4 * chunk)) = v;
    }
    static __device__ __forceinline__ f32x4 values4(const char *tile, int row, int column) { return *reinterpret_cast<const f32x4 *>(tile + at(row, column)); }
    template <int NQ>
    static __device__ __forceinline__ void add_values(const char *tile, const f32x4 (&p)[NQ][1], f32x4 (&o)[NQ][D / 16], int lane)
    {
        const int g = lane >> 4, c = lane & 15;
#pragma unroll
        for (int db = 0; db < D / 16; ++db)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = *reinterpret_cast<const float *>(tile + at(4 * g + e, 16 * db + c));
#pragma unroll
                for (int n = 0; n < NQ; ++n) o[n][db] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[n][0][e], o[n][db], 0, 0, 0);
            }
    }
};

template <typename Vec> __device__ __forceinline__ bool all_finite(const Vec &v)
{
    bool all = true;
#pragma unroll
    for (int e = 0; e < (int)(16 / sizeof(v[0])); ++e) all = all && fabsf((float)v[e]) < INFINITY;
    return all;
}
// v with 0 in the place of the elements that are finite, or of those that are not
template <typename Vec> __device__ __forceinline__ Vec without(Vec v, bool finite)
{
#pragma unroll
    for (int e = 0; e < (int)(16 / sizeof(v[0])); ++e)
        if ((fabsf((float)v[e]) < INFINITY) == finite) v[e] = 0.f;
    return v;
}

// ---- which rounds a workgroup takes.  Sequence b has R_b = ceil(length / round) of them per virtual head (a head of keys and values and up to 16 NQ
// query heads), at least one; the virtual heads of a sequence lie one behind the other, then the next sequence's.
template <int ROUND, typename Args>
__device__ __forceinline__ int rounds_of(const Args &a, int length) { return (max(1, min(length, a.max_len)) + ROUND - 1) / ROUND; }
// 64 sequences' rounds by a wavefront, a lane each, and the sums up to each (a round is 64 tokens at least: 64 sequences have fewer than 2^31)
template <int ROUND> struct Rounds {
    int length, mine, upto;
    __device__ __forceinline__ Rounds(const DecodeArgs &a, int b0, int lane)
    {
        length = b0 + lane < a.B ? a.lengths[b0 + lane] : 0;
        mine = b0 + lane < a.B ? rounds_of<ROUND>(a, length) : 0;
        upto = lane_sum_scan(mine);
    }
    __device__ __forceinline__ int all() const { return __builtin_amdgcn_readlane(upto, 63); }
};

// Scratch memory.  What a part of a sequence leaves there for its query n of `rows`: sum of weight * value [d], maximum (log2 domain) and sum.  A
// workgroup has room for two parts: 2 w for its first and, if it begins there, 2 w + 1 for its last.  And for the joining launch, the sequences that
// more than one workgroup has: by sequence and virtual head where those are not more than the workgroups, else by the workgroup that one begins in (as
// its last: there is one at most).
struct Chain { int b, v_head, w, count; };              // b < 0: none; it begins in part w and has `count` parts, one per workgroup
struct Scratch {
    float *base;
    int rows, d, parts;     // workgroups
    __device__ __forceinline__ Chain *chain(int i) const { return reinterpret_cast<Chain *>(base) + i; }
    __device__ __forceinline__ float *sums(int part, int n) const { return base + 4 * parts + ((int64_t)part * rows + n) * 2; }
    __device__ __forceinline__ float *values(int part, int n) const { return base + 4 * parts + (int64_t)2 * parts * rows * 2 + ((int64_t)part * rows + n) * d; }
};
size_t scratch_bytes(int rows, int d, int parts) { return sizeof(float) * (4 * parts + (size_t)2 * parts * rows * (d + 2)); }

// workgroups that share the rounds: as many as there is room for at once
constexpr int parts_of(int elem_bytes, int d, int nq) { return 256 * (d == 64 ? (nq == 1 ? 4 : 3) : nq == 1 || elem_bytes == 2 ? 2 : 1); }
template <typename T, int D> struct Decode {
    static constexpr int ROUND = kWaves * Step<T, D>::TILE, ROW_STRIDE = D + 4;       // (16 bytes more: rows of the joining start in other banks)
    static constexpr int TILE_BYTES = Step<T, D>::TILE * D * (int)sizeof(T), JOIN_BYTES = 16 * ROW_STRIDE * 4;
    static constexpr int REGION = TILE_BYTES > JOIN_BYTES ? TILE_BYTES : JOIN_BYTES;
};

// Rounds at .. end - 1, the first of which is of sequence b, of `length` tokens, and virtual head v_head; `base`: the first of (b, virtual head 0).  WHOLE: all of (b, v_head).
// Args: DecodeArgs, or TreeArgs where the queries are drafted tokens' and every row sees keys of its own among the last n_b: then a part of one tile of rows, `tp`, only.
template <typename T, int D, int NQ, bool STREAM, typename Args>
__device__ __forceinline__ void decode_rounds(const Args &a, char *smem, float (&sums)[kWaves][2][16], const T *__restrict__ q,
                                              const T *__restrict__ k_cache, const T *__restrict__ v_cache, T *__restrict__ out, float *__restrict__ lse,
                                              float *__restrict__ scratch, bool whole, int64_t at, int64_t end, int64_t share, int64_t base, int b, int v_head, int length,
                                              const TreePart &tp = TreePart{}, int slots = 0, int chains = 0)
{
    typedef Decode<T, D> C;
    typedef Step<T, D> S;
    typedef typename S::Vec Vec;
    constexpr int TILE = S::TILE, HALVES = TILE / 16, ROUND = C::ROUND, ROW_STRIDE = C::ROW_STRIDE, REGION = C::REGION;
    const int tid = threadIdx.x, lane = tid & 63, lq = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    char *const mine = smem + wave * REGION;
    constexpr bool TREE = std::is_same<Args, TreeArgs>::value;
    const int G = a.H / a.H_kv, n_rows = TREE ? tp.n * G : G, groups = TREE ? tp.tiles : (G + 16 * NQ - 1) / (16 * NQ), v_heads = a.H_kv * groups;
    constexpr int PARTS = parts_of(sizeof(T), D, NQ);
    const Scratch parts{scratch, min(G, 16 * NQ), D, PARTS};
    const TreeScratch tree_parts{scratch, 16 * NQ, D, slots, chains};
    const bool by_item = (int64_t)a.B * v_heads <= PARTS;
    // (a page is at most 2^29 elements: what lies within 16 rows of one is 32 bits away)
    const int64_t row_bytes = (int64_t)a.H_kv * D * (int)sizeof(T);
    const uint32_t k_lane = (uint32_t)lq * (uint32_t)row_bytes + 16 * g, v_lane = (uint32_t)(lane / S::CHUNKS) * (uint32_t)row_bytes + lane % S::CHUNKS * 16;
    const float c = kLog2e / sqrtf((float)D);
    const int64_t start = at;
    while (at < end) {
        const int R = rounds_of<ROUND>(a, length), n = max(0, min(length, a.max_len));
        const int64_t first = base + (int64_t)v_head * R;           // of this sequence and head
        const int r0 = TREE ? tp.r0 : whole ? 0 : (int)(at - first), r1 = TREE ? tp.r1 : whole ? R : (int)min<int64_t>(R, end - first);
        const int h_kv = TREE ? tp.h_kv : v_head / groups, sub = TREE ? tp.tile : v_head % groups, n_q = min(16 * NQ, n_rows - sub * 16 * NQ), h0 = h_kv * G + sub * 16 * NQ;

        typename S::Queries qf[NQ];
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if constexpr (TREE) {
                const int r = sub * 16 * NQ + min(16 * i + lq, n_q - 1), token = r / G;
                S::load_query(qf[i], q + (int64_t)(tp.begin + token) * a.q_stride + (int64_t)(h_kv * G + r - token * G) * D, g, 16 * i + lq < n_q);
            } else {
                S::load_query(qf[i], q + b * a.q_stride + (int64_t)(h0 + min(16 * i + lq, n_q - 1)) * D, g, 16 * i + lq < n_q);
            }
        }
        f32x4 o[NQ][D / 16];
        float m[NQ], l[NQ];
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            m[i] = -INFINITY;
            l[i] = 0.f;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) o[i][db] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const int j_end = min(n, r1 * ROUND);
        int j0 = r0 * ROUND + wave * TILE;
        // 64 pages' numbers, a lane each, from window_at on, and the 64 behind them
        const int32_t *const table = a.pt.table + (int64_t)b * a.pt.max_pages;
        int window_at = j0 >> a.pt.page_shift;
        const auto numbers = [&](int from) { return table[min(from + lane, a.pt.max_pages - 1)]; };
        int window = numbers(window_at), next_window = numbers(window_at + 64);
        const char *const k_head = reinterpret_cast<const char *>(k_cache + (int64_t)h_kv * D), *const v_head_base = reinterpret_cast<const char *>(v_cache + (int64_t)h_kv * D);

        typename S::Keys keys;
        Vec values[S::V_LOADS];
        bool ok[HALVES];                                // is there a page
        const auto load = [&](int j) __attribute__((always_inline)) {
            if ((j >> a.pt.page_shift) - window_at >= 64 && j < j_end) {
                window_at += 64;
                window = next_window;
                next_window = numbers(window_at + 64);
            }
            __amdgpu_buffer_rsrc_t k_half[HALVES], v_half[HALVES];
#pragma unroll
            for (int i = 0; i < HALVES; ++i) {
                const int nth = (j + 16 * i) >> a.pt.page_shift;
                // (the second half of the window's last tile may lie in a page of the next)
                int page = __builtin_amdgcn_readlane(window, (nth - window_at) & 63);
                if (nth - window_at >= 64) page = __builtin_amdgcn_readlane(next_window, 0);
                ok[i] = (uint32_t)page < (uint32_t)a.pt.n_pages && j + 16 * i < j_end;
                const int64_t row = ((int64_t)(ok[i] ? page : 0) << a.pt.page_shift) + ((j + 16 * i) & ((1 << a.pt.page_shift) - 1));
                const uint32_t bytes = ok[i] ? (uint32_t)(min(j_end - j - 16 * i, 16) - 1) * (uint32_t)row_bytes + D * (int)sizeof(T) : 0;
                k_half[i] = buffer_of(k_head + row * row_bytes, bytes);
                v_half[i] = buffer_of(v_head_base + row * row_bytes, bytes);
            }
#pragma unroll
            for (int i = 0; i < HALVES; ++i) S::template load_keys<STREAM>(keys, i, k_half[i], k_lane);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < S::V_LOADS; ++i) {
                const int row = i * 64 / S::CHUNKS;        // (of lane 0)
                values[i] = load16<STREAM, Vec>(v_half[row / 16], v_lane + (uint32_t)(row & 15) * (uint32_t)row_bytes);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        f32x4 p[NQ][HALVES];
        // scores of a tile, its values to LDS ...
        const auto scores = [&](int j) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < NQ; ++i)
#pragma unroll
                for (int hf = 0; hf < HALVES; ++hf) p[i][hf] = S::scores(keys, hf, qf[i]);
            bool all_there = j + TILE <= j_end;
#pragma unroll
            for (int hf = 0; hf < HALVES; ++hf) all_there = all_there && ok[hf];
            if (!all_there) {
                // keys that are not there have weight 0 (and their values were loaded as 0)
#pragma unroll
                for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!ok[hf] || j + 16 * hf + 4 * g + e >= j_end)
#pragma unroll
                            for (int i = 0; i < NQ; ++i) p[i][hf][e] = -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < S::V_LOADS; ++i) S::store_value(mine, (i * 64 + lane) / S::CHUNKS, lane % S::CHUNKS, values[i]);
        };
        // ... and their weights and sums; `drafted`: sums so far may hold an infinite value of a drafted token's
        const auto weights = [&](auto drafted) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                float top = -INFINITY;
#pragma unroll
                for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, p[i][hf][e]);
                if (__any(top * c > m[i] + 8.f)) {
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(top, __shfl_xor(top, 32));
                    const float m_new = fmaxf(m[i], top * c), alpha = m_new > m[i] ? fast_exp2(m[i] - m_new) : 1.f;
                    l[i] *= alpha;
                    if (decltype(drafted)::value && __any(alpha == 0.f && m[i] > -INFINITY)) {
#pragma unroll
                        for (int db = 0; db < D / 16; ++db)
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[i][db][e] = add_scaled(alpha, o[i][db][e], 0.f);
                    } else {
#pragma unroll
                        for (int db = 0; db < D / 16; ++db)
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[i][db][e] *= alpha;
                    }
                    m[i] = m_new;
                }
                const float m_use = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
                for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[i][hf][e] = fast_exp2(p[i][hf][e] * c - m_use);
                        l[i] += p[i][hf][e];
                    }
            }
        };
        if (j0 < j_end) load(j0);
        const int first_drafted = TREE ? n - n_rows / G : n;      // its key; tiles that it or a later one is in come last
        for (; j0 < j_end && (!TREE || j0 + TILE <= first_drafted); j0 += ROUND) {
            scores(j0);
            if (j0 + ROUND < j_end) load(j0 + ROUND);
            weights(std::false_type{});
            S::template add_values<NQ>(mine, p, o, lane);
        }
        if constexpr (TREE)
            for (; j0 < j_end; j0 += ROUND) {            // (the next tile's loads wait for this one's end: registers)
                uint32_t seen[NQ];
#pragma unroll
                for (int i = 0; i < NQ; ++i) {
                    const int token = (sub * 16 * NQ + min(16 * i + lq, n_q - 1)) / G;
                    seen[i] = keys_seen(a, a.tree + (int64_t)(tp.begin + token) * a.words, token, j0 - first_drafted);
                }
                scores(j0);
                bool finite = true;
                uint32_t there = 0;                     // keys
#pragma unroll
                for (int i = 0; i < S::V_LOADS; ++i) finite = finite && all_finite(values[i]);
#pragma unroll
                for (int hf = 0; hf < HALVES; ++hf)
                    if (ok[hf]) there |= (min(j_end - j0 - 16 * hf, 16) >= 16 ? 0xffffu : (1u << max(j_end - j0 - 16 * hf, 0)) - 1) << 16 * hf;
#pragma unroll
                for (int i = 0; i < NQ; ++i)
#pragma unroll
                    for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!(seen[i] >> (16 * hf + 4 * g + e) & 1)) p[i][hf][e] = -INFINITY;
                weights(std::true_type{});
                // 0 times a value that is not finite is NaN: such values are taken out of the tile, and added by themselves where their key is seen, with a weight
                // that is not 0 then
                const bool plain = !__any(!finite);
                const auto values_to_lds = [&](bool finite_out) __attribute__((always_inline)) {
#pragma unroll
                    for (int i = 0; i < S::V_LOADS; ++i) S::store_value(mine, (i * 64 + lane) / S::CHUNKS, lane % S::CHUNKS, without(values[i], finite_out));
                };
                if (!plain) values_to_lds(false);
                S::template add_values<NQ>(mine, p, o, lane);
                if (!plain) values_to_lds(true);
                const float smallest = 0x1p-126f;
#pragma unroll 1
                for (int key = plain ? TILE : 0; key < TILE; ++key) {
                    if (!(there >> key & 1)) continue;
#pragma unroll
                    for (int i = 0; i < NQ; ++i) {
                        float w = 0.f;
#pragma unroll
                        for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (key >> 4 == hf && (key & 3) == e) w = p[i][hf][e];
                        w = fmaxf(__shfl(w, 16 * (key >> 2 & 3) + lq), smallest);
                        if (seen[i] >> key & 1)
#pragma unroll
                            for (int db = 0; db < D / 16; ++db) {
                                const f32x4 x = S::values4(mine, key, 16 * db + 4 * g);
#pragma unroll
                                for (int v = 0; v < 4; ++v) o[i][db][v] = fmaf(w, x[v], o[i][db][v]);
                            }
                    }
                }
                if (j0 + ROUND < j_end) load(j0 + ROUND);
            }
        // the wavefronts' sums meet in LDS, in their order; 16 queries at a time
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            l[i] += __shfl_xor(l[i], 16);
            l[i] += __shfl_xor(l[i], 32);
            if (g == 0) { sums[wave][0][lq] = m[i]; sums[wave][1][lq] = l[i]; }
#pragma unroll
            for (int db = 0; db < D / 16; ++db) *reinterpret_cast<f32x4 *>(mine + (lq * ROW_STRIDE + 16 * db + 4 * g) * 4) = o[i][db];
            __syncthreads();
            const int row = tid >> 4, col = (tid & 15) * (D / 16), nth = 16 * i + row;
            if (nth < n_q) {
                float top = -INFINITY, total = 0.f, weight[kWaves];
#pragma unroll
                for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sums[w][0][row]);
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float mw = sums[w][0][row];
                    weight[w] = mw == -INFINITY ? 0.f : fast_exp2(mw - top);
                    total += weight[w] * sums[w][1][row];
                }
                float r[D / 16];
                const auto join = [&](auto add) __attribute__((always_inline)) {
#pragma unroll
                    for (int e = 0; e < D / 16; ++e) r[e] = 0.f;
#pragma unroll
                    for (int w = 0; w < kWaves; ++w)
#pragma unroll
                        for (int e = 0; e < D / 16; ++e)
                            r[e] = add(weight[w], *reinterpret_cast<const float *>(smem + w * REGION + (row * ROW_STRIDE + col + e) * 4), r[e]);
                };
                join([](float w, float x, float sum) { return fmaf(w, x, sum); });
                if constexpr (TREE) {
                    // (0 times infinity, or a NaN of its own: seldom)
                    bool some = false;
#pragma unroll
                    for (int e = 0; e < D / 16; ++e) some = some || r[e] != r[e];
                    if (some) join([](float w, float x, float sum) { return add_scaled(w, x, sum); });
                }
                if (TREE ? tp.count == 1 : r0 == 0 && r1 == R) {
                    const float inv = total == 0.f ? 0.f : 1.f / total;
                    int64_t row_out = (int64_t)b * a.H + h0 + nth;
                    if constexpr (TREE) row_out = tree_row(a, tp.begin, G, h_kv, sub * 16 * NQ + nth);
                    T *dst = out + row_out * D + col;
#pragma unroll
                    for (int e = 0; e < D / 16; ++e) dst[e] = (T)(r[e] * inv);
                    if (col == 0) lse[row_out] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
                } else if constexpr (TREE) {
#pragma unroll
                    for (int e = 0; e < D / 16; e += 4) *reinterpret_cast<f32x4 *>(tree_parts.values(tp.slot, nth) + col + e) = f32x4{r[e], r[e + 1], r[e + 2], r[e + 3]};
                    if (col == 0) { tree_parts.sums(tp.slot, nth)[0] = top; tree_parts.sums(tp.slot, nth)[1] = total; }
                } else {
                    const int part = 2 * blockIdx.x + (at == start ? 0 : 1);
#pragma unroll
                    for (int e = 0; e < D / 16; e += 4) *reinterpret_cast<f32x4 *>(parts.values(part, nth) + col + e) = f32x4{r[e], r[e + 1], r[e + 2], r[e + 3]};
                    if (col == 0) { parts.sums(part, nth)[0] = top; parts.sums(part, nth)[1] = total; }
                }
            }
            __syncthreads();
        }
        if (TREE || whole) return;
        if (r0 == 0 && tid == 0 && (by_item || r1 < R))
            *parts.chain(by_item ? b * v_heads + v_head : blockIdx.x) = {r1 < R ? b : -1, v_head, 2 * (int)blockIdx.x + (at == start ? 0 : 1),
                                                                         1 + (int)divide(R - r1 + share - 1, share)};
        at = first + r1;
        if (r1 == R && ++v_head == v_heads) {
            base += (int64_t)R * v_heads;
            v_head = 0;
            ++b;
            if (at < end) length = a.lengths[b];
        }
    }
}

template <typename T, int D, int NQ>
__global__ __launch_bounds__(64 * kWaves, parts_of(sizeof(T), D, NQ) / 256) void paged_decode_kernel(DecodeArgs a, const T *__restrict__ q, const T *__restrict__ k_cache,
                                                                      const T *__restrict__ v_cache, T *__restrict__ out, float *__restrict__ lse,
                                                                      float *__restrict__ scratch, int whole)
{
    typedef Decode<T, D> C;
    constexpr int PARTS = parts_of(sizeof(T), D, NQ);
    __shared__ __attribute__((aligned(1024))) char smem[kWaves * C::REGION];
    __shared__ float sums[kWaves][2][16];               // maximum, sum
    const int lane = threadIdx.x & 63;
    const int G = a.H / a.H_kv, groups = (G + 16 * NQ - 1) / (16 * NQ), v_heads = a.H_kv * groups;
    int64_t at = 0, end = 1, share = 0, base = 0, bytes;
    int b, v_head, n;                                   // (n: of b's tokens)
    if (whole) {
        b = blockIdx.x / v_heads;
        n = a.lengths[b];
        v_head = blockIdx.x % v_heads;
        bytes = (int64_t)a.B * a.max_len * a.H_kv * (2 * D * (int)sizeof(T));
    } else {
        // rounds of all sequences, per virtual head
        Rounds<C::ROUND> group(a, 0, lane);
        int64_t rounds = group.all();
        for (int b0 = 64; b0 < a.B; b0 += 64) rounds += Rounds<C::ROUND>(a, b0, lane).all();
        const int64_t all = rounds * v_heads;
        bytes = rounds * a.H_kv * (C::ROUND * 2 * D * (int)sizeof(T));
        share = (all + PARTS - 1) / PARTS;
        at = blockIdx.x * share;
        end = min(at + share, all);
        if (threadIdx.x == 0 && (int64_t)a.B * v_heads > PARTS) Scratch{scratch, 0, D, PARTS}.chain(blockIdx.x)->b = -1;
        if (at >= end) return;
        // the sequence that this workgroup's first round belongs to, and the rounds in front of it
        const int64_t nth = divide(at, v_heads);
        int64_t before = 0;
        int b0 = 0;
        while (before + group.all() <= nth) {           // (nth < rounds: some sequence has it)
            before += group.all();
            b0 += 64;
            group = Rounds<C::ROUND>(a, b0, lane);
        }
        const int l = __ffsll((long long)__ballot(before + group.upto > nth)) - 1;
        b = b0 + l;
        n = __builtin_amdgcn_readlane(group.length, l);
        base = (before + __builtin_amdgcn_readlane(group.upto - group.mine, l)) * v_heads;
        v_head = (int)divide(at - base, rounds_of<C::ROUND>(a, n));
    }
    if (bytes >= kStreamBytes) decode_rounds<T, D, NQ, true>(a, smem, sums, q, k_cache, v_cache, out, lse, scratch, whole, at, end, share, base, b, v_head, n);
    else decode_rounds<T, D, NQ, false>(a, smem, sums, q, k_cache, v_cache, out, lse, scratch, whole, at, end, share, base, b, v_head, n);
}

// Drafted tokens: the same rounds of a part of a tile of rows (tree_part); slots = 0: of all of it.  Weights enter in two parts, as above.  Bound by latency and by memory: 5 rows behind 77 tokens
// 5.7 us, one round; float, 8 heads of 64, 35 MB: 12.0 to 12.6 (2.9 TB/s) and 4.8 of joining; bf16, 24 sequences of 2 drafted tokens, 32 heads of 128, 8 of keys, 112 MB: 27 (4.1 TB/s).
template <typename T, int D, int NQ>
__global__ __launch_bounds__(64 * kWaves, tree_per_cu(sizeof(T), D, NQ)) void paged_tree_kernel(TreeArgs a, const T *__restrict__ q, const T *__restrict__ k_cache,
                                                                    const T *__restrict__ v_cache, T *__restrict__ out, float *__restrict__ lse,
                                                                    float *__restrict__ scratch, int target, int least, int slots, int chains)
{
    typedef Decode<T, D> C;
    __shared__ __attribute__((aligned(1024))) char smem[kWaves * C::REGION];
    __shared__ float sums[kWaves][2][16];
    static_assert(C::ROUND == tree_round(sizeof(T), false), "");
    const int lane = threadIdx.x & 63, G = a.H / a.H_kv;
    TreePart p;
    if (slots == 0 && a.B > 64) {
        // no tile is cut: found like a packed one
        int rank;
        PackedTile t;
        if (!xcd_item(blockIdx.x, a.H_kv, (int)((int64_t)a.rows * G / (16 * NQ)) + a.B, true, p.h_kv, rank) || !packed_tile<16 * NQ>(a, G, rank, lane, t)) return;
        p.b = t.b, p.tile = t.tile, p.tiles = 1, p.begin = t.q_begin, p.n = t.n_q, p.length = t.n_k, p.r0 = 0, p.r1 = (max(1, t.n_k) + C::ROUND - 1) / C::ROUND, p.count = 1, p.slot = 0;
    } else {
        const bool some = tree_part<C::ROUND, 16 * NQ>(a, lane, blockIdx.x, target, target, least, gridDim.x, p);
        if (slots && threadIdx.x == 0) TreeScratch{scratch, 16 * NQ, D, slots, chains}.enter(p, some);
        if (!some) return;
    }
    decode_rounds<T, D, NQ, false>(a, smem, sums, q, k_cache, v_cache, out, lse, scratch, true, 0, 1, 0, 0, p.b, 0, p.length, p, slots, chains);
}

// Joins the parts of the sequences that more than one workgroup had rounds of, in their order: workgroup x those of chain x, queries y, y + gridDim.y ..
// Thread: four columns of every (THREADS / (D / 4))th part.
template <typename T, int D, int THREADS>
__global__ __launch_bounds__(THREADS) void decode_merge_kernel(DecodeArgs a, const float *__restrict__ scratch, int nq, int n_parts, T *__restrict__ out,
                                                               float *__restrict__ lse)
{
    constexpr int LANES = D / 4, GROUPS = THREADS / LANES;
    __shared__ f32x4 acc[GROUPS][LANES];
    __shared__ float totals[GROUPS];
    const int tid = threadIdx.x, lane = tid & 63;
    const int G = a.H / a.H_kv, groups = (G + 16 * nq - 1) / (16 * nq);
    const Scratch parts{const_cast<float *>(scratch), min(G, 16 * nq), D, n_parts};
    const Chain chain = *parts.chain(blockIdx.x);
    if (chain.b < 0) return;
    const int sub = chain.v_head % groups, n_q = min(16 * nq, G - sub * 16 * nq), h0 = chain.v_head / groups * G + sub * 16 * nq;
    const auto part_of = [&](int i) { return i == 0 ? chain.w : (chain.w & ~1) + 2 * i; };
    const int grp = tid / LANES, col = tid % LANES * 4;
    for (int n = blockIdx.y; n < n_q; n += gridDim.y) {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        float v_top = -INFINITY, v_sum = 0.f, top = -INFINITY;
        if (grp < chain.count) {                        // (a thread's first part is on its way while the maximum is found)
            v = *reinterpret_cast<const f32x4 *>(parts.values(part_of(grp), n) + col);
            v_top = parts.sums(part_of(grp), n)[0];
            v_sum = parts.sums(part_of(grp), n)[1];
        }
        for (int i = lane; i < chain.count; i += 64) top = fmaxf(top, parts.sums(part_of(i), n)[0]);
        top = wave_max(top);
        const float top_use = top == -INFINITY ? 0.f : top;
        const float first = fast_exp2(v_top - top_use);
        f32x4 sum = {first * v[0], first * v[1], first * v[2], first * v[3]};
        float total = first * v_sum;
#pragma unroll 4
        for (int i = grp + GROUPS; i < chain.count; i += GROUPS) {
            const int part = part_of(i);
            const float weight = fast_exp2(parts.sums(part, n)[0] - top_use);
            const f32x4 w = *reinterpret_cast<const f32x4 *>(parts.values(part, n) + col);
            total += weight * parts.sums(part, n)[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = fmaf(weight, w[e], sum[e]);
        }
        acc[grp][tid % LANES] = sum;
        if (tid % LANES == 0) totals[grp] = total;
        __syncthreads();
        if (tid < D) {
            const int64_t row = (int64_t)chain.b * a.H + h0 + n;
            float value = 0.f;
            total = 0.f;
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) {
                value += reinterpret_cast<const float *>(&acc[i][0])[tid];
                total += totals[i];
            }
            out[row * D + tid] = (T)(total == 0.f ? 0.f : value / total);
            if (tid == 0) lse[row] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
        }
        __syncthreads();
    }
}

int queries_per_wave(int H, int H_kv) { return H / H_kv > 16 ? 2 : 1; }       // in sixteens

template <typename T, int D, int NQ>
hipError_t launch(const DecodeArgs &a, const T *q, const T *k_cache, const T *v_cache, T *out, float *lse, float *scratch, hipStream_t st)
{
    const int G = a.H / a.H_kv, v_heads = a.H_kv * ((G + 16 * NQ - 1) / (16 * NQ));
    const bool whole = a.max_len <= kWholeLen;
    constexpr int parts = parts_of(sizeof(T), D, NQ);
    {
        TimedLaunch tl(K_PAGED_DECODE, st);
        hipLaunchKernelGGL((paged_decode_kernel<T, D, NQ>), dim3((unsigned)(whole ? a.B * v_heads : parts)), dim3(64 * kWaves), 0, st, a, q, k_cache, v_cache,
                           out, lse, scratch, whole ? 1 : 0);
    }
    if (whole) return hipGetLastError();
    // (few chains may be long: more threads each)
    const int chains = (int)std::min<int64_t>((int64_t)a.B * v_heads, parts), y = std::min(G, 8);
    TimedLaunch tl(K_DECODE_MERGE, st);
    if (chains * y <= 256) hipLaunchKernelGGL((decode_merge_kernel<T, D, 1024>), dim3((unsigned)chains, (unsigned)y), dim3(1024), 0, st, a, scratch, NQ, parts, out, lse);
    else hipLaunchKernelGGL((decode_merge_kernel<T, D, 256>), dim3((unsigned)chains, (unsigned)y), dim3(256), 0, st, a, scratch, NQ, parts, out, lse);
    return hipGetLastError();
}

} // namespace

size_t paged_decode_workspace_bytes(int H, int H_kv, int d, int max_len)
{
    if (max_len <= kWholeLen) return 0;
    const int nq = queries_per_wave(H, H_kv);
    return scratch_bytes(std::min(H / H_kv, 16 * nq), d, parts_of(2, d, nq));       // (no fewer for bf16)
}

template <typename T>
hipError_t launch_paged_decode(const DecodeArgs &a, const T *q, const T *k_cache, const T *v_cache, T *out, float *lse, float *scratch, hipStream_t st)
{
    const bool two = queries_per_wave(a.H, a.H_kv) == 2;
    if (a.d == 64) return two ? launch<T, 64, 2>(a, q, k_cache, v_cache, out, lse, scratch, st) : launch<T, 64, 1>(a, q, k_cache, v_cache, out, lse, scratch, st);
    return two ? launch<T, 128, 2>(a, q, k_cache, v_cache, out, lse, scratch, st) : launch<T, 128, 1>(a, q, k_cache, v_cache, out, lse, scratch, st);
}

template <typename T>
hipError_t launch_tree_narrow(const TreeArgs &a, const TreePlan &p, const T *q, const T *k_cache, const T *v_cache, T *out, float *lse, float *scratch, hipStream_t st)
{
    const int in_order = (int)((int64_t)a.rows * (a.H / a.H_kv) / p.rows) + a.B;       // (tiles that packed_tile numbers)
    const dim3 grid((unsigned)(p.slots ? (p.most + p.tiles + 7) / 8 * 8 : a.B > 64 ? xcd_grid(a.H_kv, in_order) : (p.tiles + 7) / 8 * 8)), block(64 * kWaves);
    TimedLaunch tl(K_PAGED_TREE, st);
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a, q, k_cache, v_cache, out, lse, scratch, p.target, p.least, p.slots, p.chains); };
    if (a.d == 64) p.rows == 16 ? go(paged_tree_kernel<T, 64, 1>) : go(paged_tree_kernel<T, 64, 2>);
    else p.rows == 16 ? go(paged_tree_kernel<T, 128, 1>) : go(paged_tree_kernel<T, 128, 2>);
    return hipGetLastError();
}

template hipError_t launch_tree_narrow<bf16_t>(const TreeArgs &, const TreePlan &, const bf16_t *, const bf16_t *, const bf16_t *, bf16_t *, float *, float *, hipStream_t);
template hipError_t launch_tree_narrow<float>(const TreeArgs &, const TreePlan &, const float *, const float *, const float *, float *, float *, float *, hipStream_t);

template hipError_t launch_paged_decode<bf16_t>(const DecodeArgs &, const bf16_t *, const bf16_t *, const bf16_t *, bf16_t *, float *, float *, hipStream_t);
template hipError_t launch_paged_decode<float>(const DecodeArgs &, const float *, const float *, const float *, float *, float *, float *, hipStream_t);

} // namespace lss
