// Attention of packed sequences: the main kernels' launches (lss_fwd_bf16.hip, lss_f32.hip) and what joins the splits of the keys.
#include "lss_serve.h"

namespace lss {

namespace {

// D / 4 lanes per row and head, four columns each: lse = log sum_s exp(lse_s), out = sum_s exp(lse_s - lse) out_s, in the splits' order (16 at most: a lane
// of the row's each).  A row whose result is not finite is done over by the wavefront, over the keys that it sees alone (packed_bf16_kernel).  4155 rows of 8
// heads of 64 in float, 2 splits, 25 MB: 8 us (a wavefront per row 14).
template <typename T, int D>
__global__ __launch_bounds__(256) void packed_merge_kernel(PackedArgs a, PackedParts parts, const T *__restrict__ q, const T *__restrict__ k,
                                                           const T *__restrict__ v, T *__restrict__ out, float *__restrict__ lse)
{
    constexpr int LANES = D / 4, ROWS = 64 / LANES;
    const int lane = threadIdx.x & 63, mine = lane % LANES;
    const int items = a.rows_q * a.H, item = ((int)blockIdx.x * 4 + (int)(threadIdx.x >> 6)) * ROWS + lane / LANES;     // (2^30 at most)
    const int t = min(item, items - 1) / a.H, h = min(item, items - 1) - t * a.H;
    // the row's sequence: a wavefront's rows are of one token or of neighbours
    int b = -1, end = 0;
    for (int i = 0; i < ROWS; ++i) {
        const int ti = __builtin_amdgcn_readlane(t, i * LANES);
        int begin_i, end_i;
        const int bi = find_sequence(a.cu_q, a.B, ti, lane, begin_i, end_i);
        for (; i < ROWS && __builtin_amdgcn_readlane(t, i * LANES) == ti; ++i)
            if (lane / LANES == i) { b = bi; end = end_i; }
        --i;
    }
    const bool there = item < items && b >= 0;
    const float part_lse = there && mine < parts.splits ? *parts.lse(a, mine, t, h) : -INFINITY;
    float top = part_lse;
#pragma unroll
    for (int sh = LANES / 2; sh >= 1; sh >>= 1) top = fmaxf(top, __shfl_xor(top, sh));
    const float weight = fast_exp2((part_lse - (top == -INFINITY ? 0.f : top)) * kLog2e);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
#pragma unroll 4
    for (int s = 0; s < parts.splits; ++s) {
        const float w = __shfl(weight, lane / LANES * LANES + s);
        const f32x4 part = there ? *reinterpret_cast<const f32x4 *>(parts.values(a, s, t, h) + 4 * mine) : f32x4{0.f, 0.f, 0.f, 0.f};
        total += w;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = fmaf(w, part[e], sum[e]);
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const float row_lse = total == 0.f ? -INFINITY : top + log2f(total) * kLn2;
    bool finite = true;
    if (there) {
        T *const to = out + (int64_t)item * D + 4 * mine;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float r = sum[e] * inv;
            to[e] = (T)r;
            finite = finite && fabsf(r) < INFINITY;
        }
        if (mine == 0) lse[(int64_t)h * a.rows_q + t] = row_lse;
    }
    const uint64_t bad = __ballot(!finite && row_lse == row_lse);
    for (int i = 0; i < ROWS; ++i) {
        if ((bad >> (i * LANES) & ((uint64_t)1 << (LANES - 1) << 1) - 1) == 0) continue;
        const auto of = [&](int x) { return __builtin_amdgcn_readlane(x, i * LANES); };
        const int ti = of(t), hi = of(h), bi = of(b), h_kv = hi / (a.H / a.H_kv);
        int k_begin, n_k;
        keys_of(a, bi, k_begin, n_k);
        const int seen = a.causal ? max(0, min(n_k, n_k - (min(of(end), a.rows_q) - ti) + 1)) : n_k;
        row_attention<T, D, 2>(q + ti * a.q_stride + (int64_t)hi * D, k + k_begin * a.k_stride + (int64_t)h_kv * D, a.k_stride,
                            v + k_begin * a.v_stride + (int64_t)h_kv * D, a.v_stride, seen, __builtin_bit_cast(float, of(__builtin_bit_cast(int, row_lse))), lane,
                            out + ((int64_t)ti * a.H + hi) * D);
    }
}

} // namespace

template <typename T>
hipError_t launch_packed(const PackedArgs &a, const T *q, const T *k, const T *v, T *out, float *lse, float *scratch, hipStream_t st)
{
    const PackedPlan plan = pick_packed_plan(a.rows_q, a.rows_k, a.B, a.H, a.H_kv, a.d, sizeof(T));
    const PackedParts parts{scratch, plan.splits};
    hipError_t e;
    if constexpr (sizeof(T) == 2) e = launch_packed_bf16_main(a, plan, q, k, v, out, lse, parts, st);
    else e = launch_packed_f32_main(a, q, k, v, out, lse, parts, st);
    if (e != hipSuccess || plan.splits == 1) return e;
    const int64_t rows_per_wg = 256 / (a.d / 4);
    const dim3 grid((unsigned)(((int64_t)a.rows_q * a.H + rows_per_wg - 1) / rows_per_wg)), block(256);
    TimedLaunch tl(K_PACKED_MERGE, st);
    if (a.d == 64) hipLaunchKernelGGL((packed_merge_kernel<T, 64>), grid, block, 0, st, a, parts, q, k, v, out, lse);
    else hipLaunchKernelGGL((packed_merge_kernel<T, 128>), grid, block, 0, st, a, parts, q, k, v, out, lse);
    return hipGetLastError();
}

template hipError_t launch_packed<bf16_t>(const PackedArgs &, const bf16_t *, const bf16_t *, const bf16_t *, bf16_t *, float *, float *, hipStream_t);
template hipError_t launch_packed<float>(const PackedArgs &, const float *, const float *, const float *, float *, float *, float *, hipStream_t);

} // namespace lss
