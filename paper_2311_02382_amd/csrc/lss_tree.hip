// Attention of drafted tokens over a paged cache (lss_paged_attn_tree): which kernel a call takes, and what joins the parts of a tile of rows.
#include "lss_serve.h"

#include <algorithm>

namespace lss {

namespace {

// Joins the parts of the tile of rows that begins in part blockIdx.x, in their order: LANES lanes have a row, or in long chains S such groups, which meet in LDS
template <typename T, int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a, const float *__restrict__ scratch, int rows, int slots, T *__restrict__ out, float *__restrict__ lse)
{
    constexpr int LANES = D / 4, GROUPS = 256 / LANES;
    __shared__ f32x4 acc[GROUPS][LANES];
    __shared__ float totals[GROUPS];
    const TreeScratch parts{const_cast<float *>(scratch), rows, D, slots};
    if ((int)blockIdx.x >= *parts.parts()) return;
    const TreeChain chain = *parts.chain(blockIdx.x);
    if (chain.count <= 1) return;
    const int G = a.H / a.H_kv, grp = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    int begin, n_rows;
    queries_of(a, chain.b, begin, n_rows);
    n_rows *= G;
    const int tiles = (n_rows + rows - 1) / rows, n_q = min(rows, n_rows - chain.tile * rows);
    const int S = chain.count <= 8 ? 1 : chain.count <= 32 ? 4 : GROUPS, at_once = GROUPS / S, share = grp % S;
    const auto part_of = [&](int i) { return (int)min((int64_t)blockIdx.x + (int64_t)i * tiles, (int64_t)slots - 1); };
    for (int n0 = blockIdx.y * at_once; n0 < n_q; n0 += gridDim.y * at_once) {
        const int n = min(n0 + grp / S, n_q - 1);
        float top = -INFINITY;
        for (int i = lane; i < chain.count; i += LANES) top = fmaxf(top, parts.sums(part_of(i), n)[0]);
#pragma unroll
        for (int sh = LANES / 2; sh >= 1; sh >>= 1) top = fmaxf(top, __shfl_xor(top, sh));
        const float use = top == -INFINITY ? 0.f : top;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        float total = 0.f;
#pragma unroll 4
        for (int i = share; i < chain.count; i += S) {
            const int part = part_of(i);
            const float weight = fast_exp2(parts.sums(part, n)[0] - use);
            const f32x4 v = *reinterpret_cast<const f32x4 *>(parts.values(part, n) + 4 * lane);
            total += weight * parts.sums(part, n)[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = fmaf(weight, v[e], sum[e]);
        }
        if (S > 1) {
            __syncthreads();
            acc[grp][lane] = sum;
            if (lane == 0) totals[grp] = total;
            __syncthreads();
            total = 0.f;
            sum = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int i = 0; i < S; ++i) {
                const f32x4 v = acc[grp / S * S + i][lane];
                total += totals[grp / S * S + i];
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += v[e];
            }
        }
        if (share != 0 || n0 + grp / S >= n_q) continue;
        const int64_t row = tree_row(a, begin, G, chain.h_kv, chain.tile * rows + n);
        T *const to = out + row * D + 4 * lane;
#pragma unroll
        for (int e = 0; e < 4; ++e) to[e] = (T)(total == 0.f ? 0.f : sum[e] / total);
        if (lane == 0) lse[row] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
    }
}

// The form of a launch, from what the host knows: rows, sequences and a bound on their lengths, not the lengths
TreePlan pick(int64_t rows, int B, int H, int H_kv, int d, int max_len, int elem_bytes)
{
    const int G = H / H_kv;
    TreePlan p{elem_bytes == 2 && rows * G > (int64_t)16 * B, 128, 0, 0};
    if (!p.wide) p.rows = rows * G > (int64_t)16 * B ? 32 : 16;
    const int64_t tiles = (rows * G / p.rows + std::min<int64_t>(rows, B)) * H_kv;
    if (p.wide) {
        p.target = 1024;
        if (tiles < 768 && max_len > 512) p.slots = (int)(p.target + tiles);
    } else {
        p.target = 1024;
        if (max_len > 512) p.slots = (int)(p.target + tiles);
    }
    return p;
}

} // namespace

size_t paged_tree_workspace_bytes(int64_t rows, int B, int H, int H_kv, int d, int max_len, int elem_bytes)
{
    const TreePlan p = pick(rows, B, H, H_kv, d, max_len, elem_bytes);
    return p.slots ? tree_scratch_bytes(p.rows, d, p.slots) : 0;
}

template <typename T>
hipError_t launch_paged_tree(const TreeArgs &a, const T *q, const T *k_cache, const T *v_cache, T *out, float *lse, float *scratch, hipStream_t st)
{
    const TreePlan p = pick(a.rows, a.B, a.H, a.H_kv, a.d, a.max_len, sizeof(T));
    hipError_t e = hipSuccess;
    if constexpr (sizeof(T) == 2) {
        if (p.wide) e = launch_tree_bf16_main(a, p, q, k_cache, v_cache, out, lse, scratch, st);
        else e = launch_tree_narrow<T>(a, p, q, k_cache, v_cache, out, lse, scratch, st);
    } else {
        e = launch_tree_narrow<T>(a, p, q, k_cache, v_cache, out, lse, scratch, st);
    }
    if (e != hipSuccess || p.slots == 0) return e;
    TimedLaunch tl(K_TREE_MERGE, st);
    const dim3 grid((unsigned)p.slots, (unsigned)std::max(1, p.rows * a.d / 4096)), block(256);
    if (a.d == 64) hipLaunchKernelGGL((tree_merge_kernel<T, 64>), grid, block, 0, st, a, scratch, p.rows, p.slots, out, lse);
    else hipLaunchKernelGGL((tree_merge_kernel<T, 128>), grid, block, 0, st, a, scratch, p.rows, p.slots, out, lse);
    return hipGetLastError();
}

template hipError_t launch_paged_tree<bf16_t>(const TreeArgs &, const bf16_t *, const bf16_t *, const bf16_t *, bf16_t *, float *, float *, hipStream_t);
template hipError_t launch_paged_tree<float>(const TreeArgs &, const float *, const float *, const float *, float *, float *, float *, hipStream_t);

} // namespace lss
