// Attention of drafted tokens over a paged cache (lss_paged_attn_tree): which kernel a call takes, and what joins the parts of a tile of rows.
#include "lss_serve.h"

#include <algorithm>

namespace lss {

namespace {

// Many sequences, by one workgroup: the size of a part, and what is in front of every 64 of them.  What bounds it is latency, four or five passes over the sequences, each loads and a sum over the
// workgroup: of 320 7.3 us, 1024 8.5, 4096 18, 65,536 209 (where the main launch takes 73, 216, 822 and 12,950).
constexpr int kCountThreads = 1024, kCountWaves = kCountThreads / 64;
__global__ __launch_bounds__(kCountThreads) void tree_count_kernel(TreeArgs a, int round, int rows, int target, int most, int least, TreeCount *__restrict__ count)
{
    __shared__ int64_t sums[kCountWaves];
    __shared__ int cuts[kCountWaves], slots[kCountWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, G = a.H / a.H_kv;
    const int64_t limit = (int64_t)1 << 46;             // (no sum of rows that there are comes near it; starts that do not ascend may)
    const auto sum_of = [&](auto &&of) __attribute__((always_inline)) {
        int64_t sum = 0;
        for (int b = tid; b < a.B; b += kCountThreads) sum = min(sum + of(tree_sequence(a, G, round, rows, b)), limit);
        sum = lane64(lanes_upto(sum), 63);
        __syncthreads();
        if (lane == 0) sums[wave] = sum;
        __syncthreads();
        sum = 0;
        for (int w = 0; w < kCountWaves; ++w) sum = min(sum + sums[w], limit);
        return sum;
    };
    const int64_t rounds = sum_of([](const TreeSequence &s) { return (int64_t)s.tiles * s.R; }), all_tiles = sum_of([](const TreeSequence &s) { return (int64_t)s.tiles; });
    const auto parts = [&](int S) { return sum_of([&](const TreeSequence &s) { return parts_of_tiles(s, S); }); };
    int S = part_rounds(rounds, all_tiles, a.H_kv, target, least, parts);
    if (most > target && rounds * a.H_kv >= (int64_t)20 * most) {
        const int S_most = part_rounds(rounds, all_tiles, a.H_kv, most, least, parts);
        if (worth_more(S, S_most)) S = S_most;
    }
    TreeBatch *const batches = reinterpret_cast<TreeBatch *>(count + 1);
    TreeBatch before{0, 0, 0};
    for (int b0 = 0; b0 < a.B; b0 += kCountThreads) {
        const TreeSequence s = tree_sequence(a, G, round, rows, b0 + tid);
        const int64_t mine = parts_of_tiles(s, S);
        const int cut = cut_tiles(s, S);
        const int64_t all = lane64(lanes_upto(mine), 63);
        const int all_cut = __builtin_amdgcn_readlane(lane_sum_scan(cut), 63), all_slots = __builtin_amdgcn_readlane(lane_sum_scan(cut ? (int)mine : 0), 63);
        __syncthreads();
        if (lane == 0) sums[wave] = all, cuts[wave] = all_cut, slots[wave] = all_slots;
        __syncthreads();
        for (int w = 0; w < kCountWaves; ++w) {
            if (w == wave && lane == 0 && b0 + 64 * w < a.B) batches[b0 / 64 + w] = before;
            before.before += sums[w], before.cut += cuts[w], before.slots += slots[w];
        }
    }
    if (tid == 0) *count = {before.before, S, before.cut};
}

// Joins the parts of cut tile of rows blockIdx.x, in their order: LANES lanes have a row, or in long chains S such groups with a part each, which meet in LDS.  What bounds it is a chain of
// loads (where the parts are, whose rows, their sums and values): 5.7 us for 7 MB, 8.2 for 26 (16,016 rows of 6 parts of 64; there two groups, four took 11.6).
template <typename T, int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a, const float *__restrict__ scratch, int rows, int slots, int chains, T *__restrict__ out,
                                                         float *__restrict__ lse)
{
    constexpr int LANES = D / 4, GROUPS = 256 / LANES, AHEAD = 4;
    __shared__ f32x4 acc[GROUPS][LANES];
    __shared__ float tops[GROUPS], totals[GROUPS];
    const TreeScratch parts{const_cast<float *>(scratch), rows, D, slots, chains};
    const TreeChain chain = *parts.chain(blockIdx.x);   // (there is room for one of each workgroup)
    if ((int)blockIdx.x >= *parts.items()) return;
    const int G = a.H / a.H_kv, grp = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    int begin, n_rows;
    queries_of(a, chain.b, begin, n_rows);
    n_rows *= G;
    const int n_q = min(rows, n_rows - chain.tile * rows);
    const int S = chain.count <= 4 ? 1 : chain.count <= 8 ? 2 : chain.count <= 16 ? 4 : GROUPS, at_once = GROUPS / S, share = grp % S;
    for (int n0 = blockIdx.y * at_once; n0 < n_q; n0 += gridDim.y * at_once) {
        const int n = min(n0 + grp / S, n_q - 1);
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        float top = -INFINITY, total = 0.f;
        for (int i0 = share; i0 < chain.count; i0 += AHEAD * S) {
            float m[AHEAD], l[AHEAD];
            f32x4 v[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int i = i0 + j * S, part = chain.first + min(i, chain.count - 1) * chain.tiles;
                m[j] = parts.sums(part, n)[0];
                l[j] = i < chain.count ? parts.sums(part, n)[1] : 0.f;
                v[j] = *reinterpret_cast<const f32x4 *>(parts.values(part, n) + 4 * lane);
            }
            float higher = top;
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) higher = fmaxf(higher, m[j]);
            const float use = higher == -INFINITY ? 0.f : higher, alpha = fast_exp2(top - use);
            top = higher;
            total *= alpha;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] *= alpha;
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const float weight = i0 + j * S < chain.count ? fast_exp2(m[j] - use) : 0.f;
                total += weight * l[j];
                if (i0 + j * S < chain.count)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[e] = fmaf(weight, v[j][e], sum[e]);
            }
        }
        if (S > 1) {
            __syncthreads();
            acc[grp][lane] = sum;
            if (lane == 0) tops[grp] = top, totals[grp] = total;
            __syncthreads();
            const int first = grp / S * S;
            for (int i = 0; i < S; ++i) top = fmaxf(top, tops[first + i]);
            const float use = top == -INFINITY ? 0.f : top;
            total = 0.f;
            sum = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int i = 0; i < S; ++i) {
                const f32x4 v = acc[first + i][lane];
                const float weight = fast_exp2(tops[first + i] - use);
                total += weight * totals[first + i];
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] = fmaf(weight, v[e], sum[e]);
            }
        }
        if (share != 0 || n0 + grp / S >= n_q) continue;
        if (sum[0] != sum[0] || sum[1] != sum[1] || sum[2] != sum[2] || sum[3] != sum[3]) {
            // (0 times infinity, or a NaN of its own: seldom; once more from the parts)
            sum = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int i = 0; i < chain.count; ++i) {
                const int part = chain.first + i * chain.tiles;
                const float weight = fast_exp2(parts.sums(part, n)[0] - (top == -INFINITY ? 0.f : top));
                const f32x4 v = *reinterpret_cast<const f32x4 *>(parts.values(part, n) + 4 * lane);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] = add_scaled(weight, v[e], sum[e]);
            }
        }
        const int64_t row = tree_row(a, begin, G, chain.h_kv, chain.tile * rows + n);
        T *const to = out + row * D + 4 * lane;
#pragma unroll
        for (int e = 0; e < 4; ++e) to[e] = (T)(total == 0.f ? 0.f : sum[e] / total);
        if (lane == 0) lse[row] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
    }
}

// The form of a launch, from what the host knows: rows, sequences and a bound on their lengths, not the lengths.
//   * bf16, more than 16 rows to a head of keys of an average sequence: wide, all sequences of the call (400 single tokens behind 1000 and a piece of 1000 behind 8000 are not: 1683 us in one call, 313 and
//     174 in two).  24 sequences of 1 to 8192 tokens, 32 heads, 8 of keys, d = 128: 2 drafted tokens (8 rows)
//     37.7 us, narrow 33.6; 4 39.8 and 35.3; 8 37.3 and 49.5; 32 53 and 93; 48 sequences of 2048 to 6500 with 64: 268 and 1736.  Float is always narrow.
//   * Parts: as many as are resident at once (wide: two workgroups a compute unit, or at d = 64 three, see tree_part), of 384 keys at least.  One sequence of 30,000 tokens, 16 drafted: 39.5 us, with half
//     as many again 52; d = 64, 24 sequences with 8: 17.7, parts of 512 keys 18.7, of 768 21, of 1024 24.
//   * Lengths up to 512, or many tiles of up to 64 sequences (which then start with the longest): a tile each and no joining launch.  48 x 64 drafted tokens over 2048 to 6500, 768 tiles: 287,
//     in parts 338; a chain of 8000 behind 8000 1550 and 1662.  The host does not know the lengths, and there are some that would have it otherwise: 48 x 64 over 1 to 8192 137 and 84, 47 x 64 behind
//     500 and one behind 100,000 2060 and 340.
//   * Counted in front from 257 sequences on.  Of one token, 8 heads of keys, 20 to 700 tokens: 192 sequences 55.7 us without that launch and 59.0 with it, 256 70.0 and 71.1, 320 89.2 and 84.3,
//     2048 1365 and 436.  (Where no tile is cut, sequences past the 64th are found among their starts, and nothing is counted: 65 21.6 -> 16.9.)
constexpr int kListed = 256;
TreePlan pick(int64_t rows, int B, int H, int H_kv, int d, int max_len, int elem_bytes)
{
    const int64_t in_a_head = rows * (H / H_kv);
    const bool some = in_a_head > (int64_t)16 * B, wide = elem_bytes == 2 && some;
    TreePlan p;
    p.wide = wide;
    p.rows = wide ? 128 : some ? 32 : 16;
    p.target = wide ? 512 : 256 * tree_per_cu(elem_bytes, d, p.rows / 16);
    p.most = wide && d == 64 ? 768 : p.target;
    p.least = wide ? 6 : 2;
    p.tiles = (int)((in_a_head / p.rows + std::min<int64_t>(rows, B)) * H_kv);
    p.counted = false;
    p.slots = p.chains = 0;
    if (max_len > 512 && !(wide && p.tiles >= 768 && B <= 64)) p.slots = 2 * p.most, p.chains = p.most, p.counted = B > kListed;
    else p.least = 1 << 30;
    return p;
}

} // namespace

size_t paged_tree_workspace_bytes(int64_t rows, int B, int H, int H_kv, int d, int max_len, int elem_bytes)
{
    const TreePlan p = pick(rows, B, H, H_kv, d, max_len, elem_bytes);
    return (p.counted ? tree_count_bytes(B) : 0) + (p.slots ? tree_scratch_bytes(p.rows, d, p.slots, p.chains) : 0);
}

template <typename T>
hipError_t launch_paged_tree(const TreeArgs &args, const T *q, const T *k_cache, const T *v_cache, T *out, float *lse, float *scratch, hipStream_t st)
{
    TreeArgs a = args;
    const TreePlan p = pick(a.rows, a.B, a.H, a.H_kv, a.d, a.max_len, sizeof(T));
    if (p.counted) {
        TreeCount *const count = reinterpret_cast<TreeCount *>(scratch);
        TimedLaunch tl(K_TREE_COUNT, st);
        hipLaunchKernelGGL(tree_count_kernel, dim3(1), dim3(kCountThreads), 0, st, a, tree_round(sizeof(T), p.wide), p.rows, p.target, p.most, p.least, count);
        a.count = count;
        scratch += tree_count_bytes(a.B) / sizeof(float);
    }
    hipError_t e = hipSuccess;
    if constexpr (sizeof(T) == 2) {
        if (p.wide) e = launch_tree_bf16_main(a, p, q, k_cache, v_cache, out, lse, scratch, st);
        else e = launch_tree_narrow<T>(a, p, q, k_cache, v_cache, out, lse, scratch, st);
    } else {
        e = launch_tree_narrow<T>(a, p, q, k_cache, v_cache, out, lse, scratch, st);
    }
    if (e != hipSuccess || p.slots == 0) return e;
    TimedLaunch tl(K_TREE_MERGE, st);
    const dim3 grid((unsigned)std::min(p.tiles, p.chains), (unsigned)std::min(p.rows, 32)), block(256);
    if (a.d == 64) hipLaunchKernelGGL((tree_merge_kernel<T, 64>), grid, block, 0, st, a, scratch, p.rows, p.slots, p.chains, out, lse);
    else hipLaunchKernelGGL((tree_merge_kernel<T, 128>), grid, block, 0, st, a, scratch, p.rows, p.slots, p.chains, out, lse);
    return hipGetLastError();
}

template hipError_t launch_paged_tree<bf16_t>(const TreeArgs &, const bf16_t *, const bf16_t *, const bf16_t *, bf16_t *, float *, float *, hipStream_t);
template hipError_t launch_paged_tree<float>(const TreeArgs &, const float *, const float *, const float *, float *, float *, float *, hipStream_t);

} // namespace lss
