// Attention of drafted tokens over a paged cache (lss_paged_attn_tree).
//
// A wavefront per row and head: 64 keys at a time, a lane each for the scores; then each lane's 16 bytes of every (64 / CHUNKS)th value.
#include "lss_serve.h"

namespace lss {

namespace {

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_tree_kernel(TreeArgs a, const T *__restrict__ q, const T *__restrict__ k_cache, const T *__restrict__ v_cache,
                                                         T *__restrict__ out, float *__restrict__ lse)
{
    typedef typename Vec16<T>::type Vec;
    constexpr int VEC = 16 / sizeof(T), CHUNKS = D / VEC, KEYS = 64 / CHUNKS;
    const int lane = threadIdx.x & 63, item = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6);
    if (item >= a.rows * a.H) return;
    const int t = item / a.H, h = item % a.H, h_kv = h / (a.H / a.H_kv);
    int begin, end;
    const int b = find_sequence(a.cu, a.B, t, lane, begin, end);
    if (b < 0) return;
    const int L = max(0, min(a.lengths[b], a.max_len)), first = L - (end - begin);      // the key of the first drafted token
    const T *const mine = q + t * a.q_stride + (int64_t)h * D;
    const float c = kLog2e / sqrtf((float)D);
    const int nth = lane / CHUNKS, column = lane % CHUNKS * VEC;
    float acc[VEC], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
    for (int j0 = 0; j0 < L; j0 += 64) {
        const int j = j0 + lane, drafted = j - first;
        const int64_t row = j < L ? cache_row(a.pt, b, j) : -1;
        bool seen = row >= 0;
        if (drafted >= 0) {
            if (a.tree == nullptr) seen = seen && drafted <= t - begin;
            else seen = seen && drafted < 64 * a.words && (a.tree[(int64_t)t * a.words + drafted / 64] >> (drafted % 64) & 1);
        }
        const int64_t at = (max(row, (int64_t)0) * a.H_kv + h_kv) * D;
        float s = 0.f;
        if (seen)
            for (int i = 0; i < D; i += VEC) {
                const Vec x = *reinterpret_cast<const Vec *>(mine + i), y = *reinterpret_cast<const Vec *>(k_cache + at + i);
#pragma unroll
                for (int e = 0; e < VEC; ++e) s = fmaf((float)x[e], (float)y[e], s);
            }
        s = seen ? s * c : -INFINITY;
        const float higher = fmaxf(m, wave_max(s)), use = higher == -INFINITY ? 0.f : higher, alpha = fast_exp2(m - use), p = fast_exp2(s - use);
        m = higher;
        l = l * alpha + p;
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] *= alpha;
        for (int i = 0; i < CHUNKS; ++i) {
            const int who = i * KEYS + nth;
            const float w = __shfl(p, who);
            const int64_t from = __shfl(at, who);
            if (!__shfl((int)seen, who)) continue;
            const Vec x = *reinterpret_cast<const Vec *>(v_cache + from + column);
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[e] = fmaf(w, (float)x[e], acc[e]);
        }
    }
    l = wave_total(l);
    Vec r;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
#pragma unroll
        for (int sh = CHUNKS; sh < 64; sh *= 2) acc[e] += __shfl_xor(acc[e], sh);
        r[e] = (T)(l == 0.f ? 0.f : acc[e] / l);
    }
    if (lane < CHUNKS) *reinterpret_cast<Vec *>(out + ((int64_t)t * a.H + h) * D + column) = r;
    if (lane == 0) lse[(int64_t)t * a.H + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

} // namespace

size_t paged_tree_workspace_bytes(int64_t, int, int, int, int, int, int) { return 0; }

template <typename T>
hipError_t launch_paged_tree(const TreeArgs &a, const T *q, const T *k_cache, const T *v_cache, T *out, float *lse, float *, hipStream_t st)
{
    const dim3 grid((unsigned)(((int64_t)a.rows * a.H + 3) / 4)), block(256);
    TimedLaunch tl(K_PAGED_TREE, st);
    if (a.d == 64) hipLaunchKernelGGL((paged_tree_kernel<T, 64>), grid, block, 0, st, a, q, k_cache, v_cache, out, lse);
    else hipLaunchKernelGGL((paged_tree_kernel<T, 128>), grid, block, 0, st, a, q, k_cache, v_cache, out, lse);
    return hipGetLastError();
}

template hipError_t launch_paged_tree<bf16_t>(const TreeArgs &, const bf16_t *, const bf16_t *, const bf16_t *, bf16_t *, float *, float *, hipStream_t);
template hipError_t launch_paged_tree<float>(const TreeArgs &, const float *, const float *, const float *, float *, float *, float *, hipStream_t);

} // namespace lss
