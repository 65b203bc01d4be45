// Attention of one token per sequence over a paged cache of keys and values.
//
// A sequence's keys and values are read once, by groups of up to 16 or 32 query heads that share their head: what bounds it is
// those bytes.  Work is counted in rounds of one tile per wavefront (4 x 32 keys in bf16, 4 x 16 in float); the
// rounds of all sequences and heads, one behind the other, are dealt out in equal parts to as many workgroups as the chip holds at once, so that
// sequences of any lengths fill it evenly.  A part that is not all of its sequence goes to scratch memory, two at most per
// workgroup (its first and its last), and a second launch joins those (decode_merge_kernel).  Where no sequence is long
// (kWholeLen), a workgroup takes all of one and there is no second launch.
//
// Within a round each wavefront is by itself: a tile's keys go from memory to the registers that the matrix instructions
// S^T = K Q^T read, its values through registers to LDS (wavefront's own: no barrier), from where O^T += V^T P^T reads them
// transposed.  The next tile's loads are issued as soon as the registers are free, and are on their way while the weights are
// computed; the other wavefronts of the compute unit hide what is left.
//
// Softmax: one query per lane (four lanes share it, with the keys among them); the running maximum is raised only where a score exceeds it by more than 2^8
// in weight.  A bf16 weight would lose 16 bits before it multiplies a value; the matrix cores have time to spare here, so that
// weights go in as two bf16 parts (error 2^-17) and the only rounding to bf16 is the result's.
#include "lss_bf16.h"
#include "lss_serve.h"

#include <algorithm>

namespace lss {

namespace {

constexpr int kWaves = 4, kParts = 512;                 // workgroups that share the rounds
constexpr int kWholeLen = 512;

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
    // half i of a tile: 16 keys from `row` (this lane's key's row)
    static __device__ __forceinline__ void load_keys(Keys &k, int i, const bf16_t *row, int g)
    {
#pragma unroll
        for (int j = 0; j < NQ_FRAGS; ++j) k.f[i][j] = load_frag<bf16_t>(row + 32 * j + 8 * g);
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
    // o[n][db] += V^T P^T, element v of o[n][db]: column 16 db + 4 (l / 16) + v of query l % 16
    template <int NQ>
    static __device__ __forceinline__ void add_values(const char *tile, const f32x4 (&p)[NQ][2], f32x4 (&o)[NQ][D / 16], int lane)
    {
        Frag<bf16_t> hi[NQ], lo[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float w = p[n][e >> 2][e & 3];
                hi[n].v[e] = (bf16_t)w;
                lo[n].v[e] = (bf16_t)(w - (float)hi[n].v[e]);
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
    static __device__ __forceinline__ void load_keys(Keys &k, int i, const float *row, int g)
    {
#pragma unroll
        for (int j = 0; j < NQ_FRAGS; ++j) k.f[i][j] = *reinterpret_cast<const f32x4 *>(row + 16 * j + 4 * g);
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

// ---- which rounds a workgroup takes.  Sequence b has R_b = ceil(length / round) of them per virtual head (a head of keys and values and up to 16 NQ
// query heads), at least one; the virtual heads of a sequence lie one behind the other, then the next sequence's.
template <int ROUND>
__device__ __forceinline__ int rounds_of(const DecodeArgs &a, int b)
{
    return (max(1, min(a.lengths[b], a.max_len)) + ROUND - 1) / ROUND;
}
__device__ __forceinline__ int64_t wave_sum_i64(int64_t x)
{
#pragma unroll
    for (int sh = 32; sh >= 1; sh >>= 1) x += __shfl_xor(x, sh);
    return x;
}
// rounds of all sequences, per virtual head; by a whole wavefront
template <int ROUND>
__device__ __forceinline__ int64_t all_rounds(const DecodeArgs &a, int lane)
{
    int64_t sum = 0;
    for (int b = lane; b < a.B; b += 64) sum += rounds_of<ROUND>(a, b);
    return wave_sum_i64(sum);
}
// the sequence that round `at` belongs to (rounds counted per virtual head: at < all_rounds), and the rounds in front of it
template <int ROUND>
__device__ __forceinline__ int sequence_at(const DecodeArgs &a, int64_t at, int lane, int64_t &before)
{
    before = 0;
    for (int b0 = 0;; b0 += 64) {
        int64_t upto = b0 + lane < a.B ? rounds_of<ROUND>(a, b0 + lane) : 0;
        const int64_t mine = upto;
#pragma unroll
        for (int sh = 1; sh < 64; sh <<= 1) {
            const int64_t other = __shfl_up(upto, sh);
            if (lane >= sh) upto += other;
        }
        const uint64_t past = __ballot(before + upto > at);
        if (past != 0) {
            const int l = __ffsll((long long)past) - 1;
            before += __shfl(upto - mine, l);
            return b0 + l;
        }
        before += __shfl(upto, 63);
        if (b0 + 64 >= a.B) return a.B - 1;
    }
}
__device__ __forceinline__ int64_t scalar(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)x) | (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32);
}

// What a part of a sequence leaves in scratch memory, for its query n of `rows`: sum of weight * value [d], then maximum (log2 domain) and sum
struct Scratch {
    float *base;
    int rows, d;
    __device__ __forceinline__ float *values(int part, int n) const { return base + ((int64_t)part * rows + n) * d; }
    __device__ __forceinline__ float *sums(int part, int n) const { return base + (int64_t)2 * kParts * rows * d + ((int64_t)part * rows + n) * 2; }
};

template <typename T, int D, int NQ>
__global__ __launch_bounds__(64 * kWaves, 2) void paged_decode_kernel(DecodeArgs a, const T *__restrict__ q, const T *__restrict__ k_cache,
                                                                      const T *__restrict__ v_cache, T *__restrict__ out, float *__restrict__ lse,
                                                                      float *__restrict__ scratch, int whole)
{
    typedef Step<T, D> S;
    typedef typename S::Vec Vec;
    constexpr int TILE = S::TILE, HALVES = TILE / 16, ROUND = kWaves * TILE, ROW_STRIDE = D + 4;       // (16 bytes more: rows of the joining start in other banks)
    constexpr int REGION = 16 * ROW_STRIDE * 4 > TILE * D * (int)sizeof(T) ? 16 * ROW_STRIDE * 4 : TILE * D * (int)sizeof(T);
    __shared__ __attribute__((aligned(1024))) char smem[kWaves * REGION];
    __shared__ float sums[kWaves][2][16];               // maximum, sum
    const int tid = threadIdx.x, lane = tid & 63, lq = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    char *const mine = smem + wave * REGION;
    const int G = a.H / a.H_kv, groups = (G + 16 * NQ - 1) / (16 * NQ), v_heads = a.H_kv * groups;
    const Scratch parts{scratch, min(G, 16 * NQ), D};
    const int64_t ld = (int64_t)a.H_kv * D;
    const float c = kLog2e / sqrtf((float)D);

    int64_t at, end, share = 0;                         // rounds of all sequences and virtual heads
    int b, v_head;
    int64_t base = 0;                                   // first round of (b, virtual head 0)
    if (whole) {
        b = blockIdx.x / v_heads;
        v_head = blockIdx.x % v_heads;
        at = 0;
        end = 1;                                        // (one piece)
    } else {
        const int64_t all = scalar(all_rounds<ROUND>(a, lane)) * v_heads;
        share = (all + kParts - 1) / kParts;
        at = blockIdx.x * share;
        end = min(at + share, all);
        if (at >= end) return;
        int64_t before;
        b = __builtin_amdgcn_readfirstlane(sequence_at<ROUND>(a, at / v_heads, lane, before));
        base = scalar(before) * v_heads;
        v_head = (int)((at - base) / rounds_of<ROUND>(a, b));
    }
    const int64_t start = at;
    while (at < end) {
        const int n = max(0, min(a.lengths[b], a.max_len)), R = rounds_of<ROUND>(a, b);
        const int64_t first = base + (int64_t)v_head * R;           // of this sequence and head
        const int r0 = whole ? 0 : (int)(at - first), r1 = whole ? R : (int)min<int64_t>(R, end - first);
        const int h_kv = v_head / groups, sub = v_head % groups, n_q = min(16 * NQ, G - sub * 16 * NQ), h0 = h_kv * G + sub * 16 * NQ;

        typename S::Queries qf[NQ];
#pragma unroll
        for (int i = 0; i < NQ; ++i)
            S::load_query(qf[i], q + b * a.q_stride + (int64_t)(h0 + min(16 * i + lq, n_q - 1)) * D, g, 16 * i + lq < n_q);
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
        const T *const k_head = k_cache + (int64_t)h_kv * D, *const v_head_base = v_cache + (int64_t)h_kv * D;

        typename S::Keys keys;
        Vec values[S::V_LOADS];
        bool ok[HALVES];                                // is there a page
        const auto load = [&](int j) __attribute__((always_inline)) {
            if ((j >> a.pt.page_shift) - window_at >= 64) {
                window_at += 64;
                window = next_window;
                next_window = numbers(window_at + 64);
            }
            const T *k_row[HALVES], *v_row[HALVES];
#pragma unroll
            for (int i = 0; i < HALVES; ++i) {
                const int nth = (j + 16 * i) >> a.pt.page_shift;
                // (the second half of the window's last tile may lie in a page of the next)
                int page = __builtin_amdgcn_readlane(window, (nth - window_at) & 63);
                if (nth - window_at >= 64) page = __builtin_amdgcn_readlane(next_window, 0);
                ok[i] = (uint32_t)page < (uint32_t)a.pt.n_pages && j + 16 * i < j_end;
                const int64_t row = ((int64_t)(ok[i] ? page : 0) << a.pt.page_shift) + ((j + 16 * i) & ((1 << a.pt.page_shift) - 1));
                k_row[i] = k_head + row * ld;
                v_row[i] = v_head_base + row * ld;
            }
#pragma unroll
            for (int i = 0; i < HALVES; ++i) S::load_keys(keys, i, k_row[i] + lq * (int)ld, g);
#pragma unroll
            for (int i = 0; i < S::V_LOADS; ++i) {
                const int row = (i * 64 + lane) / S::CHUNKS, half = i * 64 / S::CHUNKS / 16;
                values[i] = *reinterpret_cast<const Vec *>(v_row[half] + (row & 15) * (int)ld + (lane % S::CHUNKS) * (16 / (int)sizeof(T)));
            }
        };
        if (j0 < j_end) load(j0);
        for (; j0 < j_end; j0 += ROUND) {
            f32x4 p[NQ][HALVES];
#pragma unroll
            for (int i = 0; i < NQ; ++i)
#pragma unroll
                for (int hf = 0; hf < HALVES; ++hf) p[i][hf] = S::scores(keys, hf, qf[i]);
            bool all_there = j0 + TILE <= j_end;
#pragma unroll
            for (int hf = 0; hf < HALVES; ++hf) all_there = all_there && ok[hf];
            if (!all_there) {
                // keys that are not there have weight 0, and their values, which may be anything, are taken as 0
#pragma unroll
                for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!ok[hf] || j0 + 16 * hf + 4 * g + e >= j_end)
#pragma unroll
                            for (int i = 0; i < NQ; ++i) p[i][hf][e] = -INFINITY;
#pragma unroll
                for (int i = 0; i < S::V_LOADS; ++i)
                    if (!ok[i * 64 / S::CHUNKS / 16] || j0 + (i * 64 + lane) / S::CHUNKS >= j_end) values[i] = Vec{};
            }
#pragma unroll
            for (int i = 0; i < S::V_LOADS; ++i) S::store_value(mine, (i * 64 + lane) / S::CHUNKS, lane % S::CHUNKS, values[i]);
            if (j0 + ROUND < j_end) load(j0 + ROUND);
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
#pragma unroll
                    for (int db = 0; db < D / 16; ++db)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[i][db][e] *= alpha;
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
            S::template add_values<NQ>(mine, p, o, lane);
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
#pragma unroll
                for (int e = 0; e < D / 16; ++e) r[e] = 0.f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w)
#pragma unroll
                    for (int e = 0; e < D / 16; ++e)
                        r[e] = fmaf(weight[w], *reinterpret_cast<const float *>(smem + w * REGION + (row * ROW_STRIDE + col + e) * 4), r[e]);
                if (r0 == 0 && r1 == R) {
                    const float inv = total == 0.f ? 0.f : 1.f / total;
                    T *dst = out + ((int64_t)b * a.H + h0 + nth) * D + col;
#pragma unroll
                    for (int e = 0; e < D / 16; ++e) dst[e] = (T)(r[e] * inv);
                    if (col == 0) lse[(int64_t)b * a.H + h0 + nth] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
                } else {
                    const int part = 2 * blockIdx.x + (at == start ? 0 : 1);
#pragma unroll
                    for (int e = 0; e < D / 16; e += 4) *reinterpret_cast<f32x4 *>(parts.values(part, nth) + col + e) = f32x4{r[e], r[e + 1], r[e + 2], r[e + 3]};
                    if (col == 0) { parts.sums(part, nth)[0] = top; parts.sums(part, nth)[1] = total; }
                }
            }
            __syncthreads();
        }
        if (whole) return;
        at = first + r1;
        if (r1 == R && ++v_head == v_heads) {
            base += (int64_t)R * v_heads;
            v_head = 0;
            ++b;
        }
    }
}

// Joins the parts of the sequences that more than one workgroup had rounds of, in their order; a workgroup per sequence and query head.  Thread: four
// columns of every eighth (sixteenth at d = 64) part.
template <typename T, int D, int ROUND>
__global__ __launch_bounds__(256) void decode_merge_kernel(DecodeArgs a, const float *__restrict__ scratch, int nq, T *__restrict__ out, float *__restrict__ lse)
{
    constexpr int LANES = D / 4, GROUPS = 256 / LANES;
    __shared__ float4 acc[GROUPS][LANES];
    __shared__ float totals[GROUPS];
    const int tid = threadIdx.x, lane = tid & 63, b = blockIdx.x / a.H, h = blockIdx.x % a.H;
    const int G = a.H / a.H_kv, groups = (G + 16 * nq - 1) / (16 * nq), v_heads = a.H_kv * groups;
    const Scratch parts{const_cast<float *>(scratch), min(G, 16 * nq), D};
    const int v_head = h / G * groups + h % G / (16 * nq), n = h % G % (16 * nq);
    const int64_t all = all_rounds<ROUND>(a, lane) * v_heads, share = (all + kParts - 1) / kParts;
    int64_t before = 0;
    for (int i = lane; i < b; i += 64) before += rounds_of<ROUND>(a, i);
    before = wave_sum_i64(before);
    const int R = rounds_of<ROUND>(a, b);
    const int64_t first = before * v_heads + (int64_t)v_head * R, last = first + R - 1;
    const int w0 = (int)(first / share), w1 = (int)(last / share);
    if (w0 == w1) return;
    const auto part_of = [&](int w) { return 2 * w + (w == w0 && first > w0 * share ? 1 : 0); };
    float top = -INFINITY;
    for (int w = w0 + lane; w <= w1; w += 64) top = fmaxf(top, parts.sums(part_of(w), n)[0]);
    top = wave_max(top);
    const float top_use = top == -INFINITY ? 0.f : top;
    const int grp = tid / LANES, col = tid % LANES * 4;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
#pragma unroll 4
    for (int w = w0 + grp; w <= w1; w += GROUPS) {
        const int part = part_of(w);
        const float weight = fast_exp2(parts.sums(part, n)[0] - top_use);
        const f32x4 v = *reinterpret_cast<const f32x4 *>(parts.values(part, n) + col);
        total += weight * parts.sums(part, n)[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = fmaf(weight, v[e], sum[e]);
    }
    acc[grp][tid % LANES] = float4{sum[0], sum[1], sum[2], sum[3]};
    if (tid % LANES == 0) totals[grp] = total;
    __syncthreads();
    if (tid >= D) return;
    float value = 0.f;
    total = 0.f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
        value += reinterpret_cast<const float *>(&acc[i][0])[tid];
        total += totals[i];
    }
    out[((int64_t)b * a.H + h) * D + tid] = (T)(total == 0.f ? 0.f : value / total);
    if (tid == 0) lse[(int64_t)b * a.H + h] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
}

int queries_per_wave(int H, int H_kv) { return H / H_kv > 16 ? 2 : 1; }       // in sixteens

template <typename T, int D, int NQ>
hipError_t launch(const DecodeArgs &a, const T *q, const T *k_cache, const T *v_cache, T *out, float *lse, float *scratch, hipStream_t st)
{
    const int G = a.H / a.H_kv, v_heads = a.H_kv * ((G + 16 * NQ - 1) / (16 * NQ));
    const bool whole = a.max_len <= kWholeLen;
    {
        TimedLaunch tl(K_PAGED_DECODE, st);
        hipLaunchKernelGGL((paged_decode_kernel<T, D, NQ>), dim3((unsigned)(whole ? a.B * v_heads : kParts)), dim3(64 * kWaves), 0, st, a, q, k_cache, v_cache,
                           out, lse, scratch, whole ? 1 : 0);
    }
    if (whole) return hipGetLastError();
    TimedLaunch tl(K_DECODE_MERGE, st);
    hipLaunchKernelGGL((decode_merge_kernel<T, D, kWaves * Step<T, D>::TILE>), dim3((unsigned)(a.B * a.H)), dim3(256), 0, st, a, scratch, NQ, out, lse);
    return hipGetLastError();
}

} // namespace

size_t paged_decode_workspace_bytes(int H, int H_kv, int d, int max_len)
{
    if (max_len <= kWholeLen) return 0;
    const int G = H / H_kv, rows = std::min(G, 16 * queries_per_wave(H, H_kv));
    return (size_t)2 * kParts * rows * (d + 2) * sizeof(float);
}

template <typename T>
hipError_t launch_paged_decode(const DecodeArgs &a, const T *q, const T *k_cache, const T *v_cache, T *out, float *lse, float *scratch, hipStream_t st)
{
    const bool two = queries_per_wave(a.H, a.H_kv) == 2;
    if (a.d == 64) return two ? launch<T, 64, 2>(a, q, k_cache, v_cache, out, lse, scratch, st) : launch<T, 64, 1>(a, q, k_cache, v_cache, out, lse, scratch, st);
    return two ? launch<T, 128, 2>(a, q, k_cache, v_cache, out, lse, scratch, st) : launch<T, 128, 1>(a, q, k_cache, v_cache, out, lse, scratch, st);
}

template hipError_t launch_paged_decode<bf16_t>(const DecodeArgs &, const bf16_t *, const bf16_t *, const bf16_t *, bf16_t *, float *, float *, hipStream_t);
template hipError_t launch_paged_decode<float>(const DecodeArgs &, const float *, const float *, const float *, float *, float *, float *, hipStream_t);

} // namespace lss
