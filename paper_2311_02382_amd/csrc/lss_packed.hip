// Attention of whole prompts of different lengths, packed one behind the other, with groups of query heads that share a head of keys
// and values.
#include "lss_serve.h"

namespace lss {

namespace {

// A wavefront per row and head.  Row r of sequence b's n_q rows stands at position n_k - n_q + r of its n_k keys.
template <typename T, int D>
__global__ __launch_bounds__(256) void packed_attn_kernel(PackedArgs a, const T *__restrict__ q, const T *__restrict__ k, const T *__restrict__ v,
                                                         T *__restrict__ out, float *__restrict__ lse)
{
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (item >= (int64_t)a.rows_q * a.H) return;
    const int t = (int)(item / a.H), h = (int)(item % a.H), h_kv = h / (a.H / a.H_kv);
    int begin, end;
    const int b = find_sequence(a.cu_q, a.B, t, lane, begin, end);
    if (b < 0) return;
    const int k_begin = max(0, min(a.cu_k[b], a.rows_k)), k_end = max(k_begin, min(a.cu_k[b + 1], a.rows_k)), n_k = k_end - k_begin;
    const int seen = a.causal ? max(0, min(n_k, n_k - (end - t) + 1)) : n_k;
    row_attention<T, D>(q + t * a.q_stride + (int64_t)h * D, k + k_begin * a.k_stride + (int64_t)h_kv * D, a.k_stride,
                        v + k_begin * a.v_stride + (int64_t)h_kv * D, a.v_stride, seen, lane, [&](int j) { return (int64_t)j; }, out + item * D, lse + (int64_t)h * a.rows_q + t);
}

} // namespace

template <typename T>
hipError_t launch_packed_attn(const PackedArgs &a, const T *q, const T *k, const T *v, T *out, float *lse, hipStream_t st)
{
    const dim3 grid((unsigned)(((int64_t)a.rows_q * a.H + 3) / 4)), block(256);
    TimedLaunch tl(K_PACKED_ATTN, st);
    if (a.d == 64) hipLaunchKernelGGL((packed_attn_kernel<T, 64>), grid, block, 0, st, a, q, k, v, out, lse);
    else hipLaunchKernelGGL((packed_attn_kernel<T, 128>), grid, block, 0, st, a, q, k, v, out, lse);
    return hipGetLastError();
}

template <>
hipError_t launch_packed_attn<bf16_t>(const PackedArgs &a, const bf16_t *q, const bf16_t *k, const bf16_t *v, bf16_t *out, float *lse, hipStream_t st)
{
    return launch_packed_bf16(a, q, k, v, out, lse, st);
}
template hipError_t launch_packed_attn<float>(const PackedArgs &, const float *, const float *, const float *, float *, float *, hipStream_t);

} // namespace lss
