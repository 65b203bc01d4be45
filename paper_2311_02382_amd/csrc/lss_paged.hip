// A paged cache of keys and values: what puts new tokens into it.
//
// Token `position` of sequence b lies in page table[b, position / page_size], slot position % page_size, of both caches,
// [n_pages, page_size, H_kv, d] each.  A number outside [0, n_pages) is no page: nothing is written there and nobody sees its tokens.
#include "lss_serve.h"

#include <climits>

namespace lss {

namespace {

constexpr int kAppendThreads = 256;

// ---- append.  Row t of the packed rows has position lengths[b] - (rows of b) + (t - cu[b]).  A workgroup takes up to four rows, one per wavefront
// for the way from row to cache row; then one thread per angle turns positions into cosines and sines, which serve all heads of a
// row through LDS; then 32 bytes per thread and step are rotated and stored.
//   Angle: position * inv_freq in 64 bits, taken to within half a turn there -- a position of 2^20 is off by 0.06 radians in 32 bits -- and its
// cosine and sine in 32 bits.
//   A thread's 32 bytes are two 16-byte chunks of a head that rotate with one another: chunks c and c + rot / 2 of it, or neighbours where pairs
// are neighbours (and behind the rotated columns).
template <typename T>
__global__ __launch_bounds__(kAppendThreads) void paged_append_kernel(AppendArgs a, const T *k, const T *v, const T *q, T *__restrict__ k_cache,
                                                                     T *__restrict__ v_cache, T *q_rot, T *k_rot)
{
    typedef typename Vec16<T>::type Vec;
    constexpr int VEC = 16 / sizeof(T);
    __shared__ int position[4];
    __shared__ int64_t target[4];                       // cache row, -1: none
    __shared__ float turn[2][4][64];                    // cosine, sine
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row0 = blockIdx.x * a.rows_per_wg, n_rows = min(a.rows_per_wg, a.rows - row0);
    if (wave < n_rows) {
        const int t = row0 + wave;
        int b = -1, begin = t, end = t + 1;
        if (a.cu == nullptr) b = t < a.B ? t : -1;
        else b = find_sequence(a.cu, a.B, t, lane, begin, end);
        const int p = b < 0 ? -1 : a.lengths[b] - (end - t);
        const int64_t at = b < 0 ? -1 : cache_row(a.pt, b, p);
        if (lane == 0) {
            position[wave] = b < 0 ? INT_MIN : p;       // (no sequence's row: not touched at all)
            target[wave] = at;
        }
    }
    __syncthreads();
    const int half = a.rot / 2;
    for (int i = tid; i < n_rows * half; i += kAppendThreads) {
        const int r = i / half, pair = i - r * half;
        if (position[r] == INT_MIN) continue;
        const double turns = (double)position[r] * (a.inv_freq[pair] * 0.15915494309189535);
        float sn, cs;
        sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
        turn[0][r][pair] = cs;
        turn[1][r][pair] = sn;
    }
    __syncthreads();
    const int upr = a.d / (2 * VEC);                    // units of a head: 2, 4 or 8 .. 16
    const int heads = 2 * a.H_kv + (q_rot ? a.H : 0), per_row = heads * upr, rot_units = a.rot / (2 * VEC);
    for (int i = tid; i < n_rows * per_row; i += kAppendThreads) {
        const int r = i / per_row, u = i - r * per_row, hd = u / upr, c = u - hd * upr;
        if (position[r] == INT_MIN) continue;
        const int64_t t = row0 + r;
        const bool is_k = hd < a.H_kv, is_v = !is_k && hd < 2 * a.H_kv;
        const int h = is_k ? hd : is_v ? hd - a.H_kv : hd - 2 * a.H_kv;
        const bool turned = !is_v && c < rot_units;
        const int first = turned && !a.interleaved ? c * VEC : 2 * c * VEC, second = turned && !a.interleaved ? first + half : first + VEC;
        const T *src = (is_k ? k + t * a.k_stride : is_v ? v + t * a.v_stride : q + t * a.q_stride) + (int64_t)h * a.d;
        Vec x = *reinterpret_cast<const Vec *>(src + first), y = *reinterpret_cast<const Vec *>(src + second);
        if (turned) {
            const float *cs = &turn[0][r][c * VEC], *sn = &turn[1][r][c * VEC];
            Vec x1, y1;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                if (a.interleaved) {
                    const int pe = e & ~1;
                    const float cx = cs[pe / 2], sx = sn[pe / 2], cy = cs[VEC / 2 + pe / 2], sy = sn[VEC / 2 + pe / 2];
                    x1[e] = (T)((e & 1) == 0 ? (float)x[pe] * cx - (float)x[pe + 1] * sx : (float)x[pe] * sx + (float)x[pe + 1] * cx);
                    y1[e] = (T)((e & 1) == 0 ? (float)y[pe] * cy - (float)y[pe + 1] * sy : (float)y[pe] * sy + (float)y[pe + 1] * cy);
                } else {
                    x1[e] = (T)((float)x[e] * cs[e] - (float)y[e] * sn[e]);
                    y1[e] = (T)((float)x[e] * sn[e] + (float)y[e] * cs[e]);
                }
            }
            x = x1;
            y = y1;
        }
        const auto put = [&](T *row) {
            *reinterpret_cast<Vec *>(row + first) = x;
            *reinterpret_cast<Vec *>(row + second) = y;
        };
        if (is_k || is_v) {
            if (target[r] >= 0) put((is_k ? k_cache : v_cache) + (target[r] * a.H_kv + h) * a.d);
            if (is_k && k_rot) put(k_rot + (t * a.H_kv + h) * a.d);
        } else {
            put(q_rot + (t * a.H + h) * a.d);
        }
    }
}

} // namespace

template <typename T>
hipError_t launch_paged_append(const AppendArgs &args, const T *k, const T *v, const T *q, T *k_cache, T *v_cache, T *q_rot, T *k_rot, hipStream_t st)
{
    AppendArgs a = args;
    a.rows_per_wg = a.rows >= 1024 ? 4 : 1;
    TimedLaunch tl(K_PAGED_APPEND, st);
    hipLaunchKernelGGL(paged_append_kernel<T>, dim3((unsigned)((a.rows + a.rows_per_wg - 1) / a.rows_per_wg)), dim3(kAppendThreads), 0, st, a, k, v, q,
                       k_cache, v_cache, q_rot, k_rot);
    return hipGetLastError();
}

template hipError_t launch_paged_append<bf16_t>(const AppendArgs &, const bf16_t *, const bf16_t *, const bf16_t *, bf16_t *, bf16_t *, bf16_t *, bf16_t *,
                                                hipStream_t);
template hipError_t launch_paged_append<float>(const AppendArgs &, const float *, const float *, const float *, float *, float *, float *, float *,
                                               hipStream_t);

} // namespace lss
