// Attention of packed sequences: the main kernels' launches (lss_fwd_bf16.hip, lss_f32.hip) and what joins the splits of the keys.
#include "lss_serve.h"

namespace lss {

namespace {

// A wavefront per row and head: lse = log sum_s exp(lse_s), out = sum_s exp(lse_s - lse) out_s, in the splits' order.  A row whose result is not finite is
// done over, over the keys that it sees alone (packed_bf16_kernel).
template <typename T, int D>
__global__ __launch_bounds__(256) void packed_merge_kernel(PackedArgs a, PackedParts parts, const T *__restrict__ q, const T *__restrict__ k,
                                                           const T *__restrict__ v, T *__restrict__ out, float *__restrict__ lse)
{
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (item >= (int64_t)a.rows_q * a.H) return;
    const int t = (int)(item / a.H), h = (int)(item % a.H);
    int begin, end;
    const int b = find_sequence(a.cu_q, a.B, t, lane, begin, end);
    if (b < 0) return;
    const float mine = lane < parts.splits ? *parts.lse(a, lane, t, h) : -INFINITY, top = wave_max(mine), top_use = top == -INFINITY ? 0.f : top;
    const float weight = fast_exp2((mine - top_use) * kLog2e), total = wave_total(lane < parts.splits ? weight : 0.f);
    float sum[D / 64];
#pragma unroll
    for (int i = 0; i < D / 64; ++i) sum[i] = 0.f;
    for (int s = 0; s < parts.splits; ++s) {
        const float *const from = parts.values(a, s, t, h);
        const float w = __shfl(weight, s);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) sum[i] = fmaf(w, from[lane + 64 * i], sum[i]);
    }
    bool finite = true;
    T *const row = out + item * D;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        const float r = total == 0.f ? 0.f : sum[i] / total;
        row[lane + 64 * i] = (T)r;
        finite = finite && fabsf(r) < INFINITY;
    }
    float *const to = lse + (int64_t)h * a.rows_q + t;
    if (lane == 0) *to = total == 0.f ? -INFINITY : top + log2f(total) * kLn2;
    if (__any(!finite)) {
        const int h_kv = h / (a.H / a.H_kv), k_begin = max(0, min(a.cu_k[b], a.rows_k)), n_k = max(0, min(a.cu_k[b + 1], a.rows_k) - k_begin);
        const int seen = a.causal ? max(0, min(n_k, n_k - (min(end, a.rows_q) - t) + 1)) : n_k;
        row_attention<T, D>(q + t * a.q_stride + (int64_t)h * D, k + k_begin * a.k_stride + (int64_t)h_kv * D, a.k_stride,
                            v + k_begin * a.v_stride + (int64_t)h_kv * D, a.v_stride, seen, lane, [](int j) { return (int64_t)j; }, row, to);
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
    const dim3 grid((unsigned)(((int64_t)a.rows_q * a.H + 3) / 4)), block(256);
    TimedLaunch tl(K_PACKED_MERGE, st);
    if (a.d == 64) hipLaunchKernelGGL((packed_merge_kernel<T, 64>), grid, block, 0, st, a, parts, q, k, v, out, lse);
    else hipLaunchKernelGGL((packed_merge_kernel<T, 128>), grid, block, 0, st, a, parts, q, k, v, out, lse);
    return hipGetLastError();
}

template hipError_t launch_packed<bf16_t>(const PackedArgs &, const bf16_t *, const bf16_t *, const bf16_t *, bf16_t *, float *, float *, hipStream_t);
template hipError_t launch_packed<float>(const PackedArgs &, const float *, const float *, const float *, float *, float *, float *, hipStream_t);

} // namespace lss
