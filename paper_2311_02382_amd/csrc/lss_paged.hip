// A paged cache of keys and values: what puts new tokens into it.
//
// Token `position` of sequence b lies in page table[b, position / page_size], slot position % page_size, of both caches,
// [n_pages, page_size, H_kv, d] each.  A number outside [0, n_pages) is no page: nothing is written there and nobody sees its tokens.
#include "lss_serve.h"

#include <climits>

namespace lss {

namespace {

constexpr int kAppendThreads = 256, kAppendRows = 2, kAppendUnits = 3;

// ---- append.  Row t of the packed rows has position lengths[b] - (rows of b) + (t - cu[b]).  What bounds it is the bytes it moves, or in a step of single tokens
// its launch and two loads that wait for one another, length and page number (of rows that are found in the starts, two more), and inv_freq's, which waits for nothing
// but is issued behind the first barrier.  A workgroup takes two rows (one of few): one wavefront each finds the way from row to cache row; then one thread per angle
// turns positions into cosines and sines, which serve all heads of a row through LDS; then 32 bytes per thread and unit are rotated and stored.  A thread's first
// three units are loaded before all that: where they lie does not depend on it.  6904 rows of 32 + 8 + 8 heads of 128, keys also
// to a tensor of their own, 184 MB: 32.7 us, 5.6 TB/s (a copy of as much: 29.4); loaded behind the angles, four rows, 46.6; with loads that stay in the caches 40.4.
//   Angle: position * inv_freq in 64 bits, taken to within half a turn there -- a position of 2^20 is off by 0.06 radians in 32 bits -- and its
// cosine and sine in 32 bits; products in 32 bits, rounded to the type once.
//   A unit is two 16-byte chunks of a head, which has `units` of them: where pairs are rot / 2 columns apart the two that rotate with one another, chunks c and
// c + rot_units, elsewhere and behind the rotated columns c and c + units.  So neighbouring lanes have neighbouring chunks (a unit of two neighbours, one row in two
// stores: 36.3 us).
template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kAppendThreads) void paged_append_kernel(AppendArgs a, const T *k, const T *v, const T *q, T *__restrict__ k_cache,
                                                                     T *__restrict__ v_cache, T *q_rot, T *k_rot)
{
    typedef typename Vec16<T>::type Vec;
    constexpr int VEC = 16 / sizeof(T);
    __shared__ int position[kAppendRows];                         // INT_MIN: no sequence's row, not touched at all
    __shared__ int64_t target[kAppendRows];                       // cache row, -1: none
    __shared__ float turn[2][kAppendRows][64];                    // cosine, sine
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row0 = blockIdx.x * a.rows_per_wg, n_rows = min(a.rows_per_wg, a.rows - row0);
    // this thread's units: number c of every slots-th head, over the rows' heads (k's, v's, then q's)
    const int half = a.rot / 2, units = 1 << a.unit_shift, rot_units = half / VEC, c = tid & (units - 1), slots = kAppendThreads >> a.unit_shift;
    const int heads = 2 * a.H_kv + (q_rot ? a.H : 0), n_items = n_rows * heads;
    struct Unit {
        int row, head;
        bool is_k, is_v;
        int first, second;
    };
    const auto unit = [&](int item) {
        Unit u;
        static_assert(kAppendRows == 2, "");
        u.row = item >= heads;
        u.head = item - (u.row ? heads : 0);
        u.is_k = u.head < a.H_kv;
        u.is_v = !u.is_k && u.head < 2 * a.H_kv;
        u.head -= u.is_k ? 0 : u.is_v ? a.H_kv : 2 * a.H_kv;
        const bool halves = !INTERLEAVED && !u.is_v;
        u.first = (halves && c >= rot_units ? c + rot_units : c) * VEC;
        u.second = (halves && c < rot_units ? c + rot_units : c + units) * VEC;
        return u;
    };
    Vec x[kAppendUnits], y[kAppendUnits];
    const auto load = [&](int item0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kAppendUnits; ++i) {
            const Unit u = unit(min(item0 + i * slots, n_items - 1));
            const int64_t t = row0 + u.row;
            const T *src = (u.is_k ? k + t * a.k_stride : u.is_v ? v + t * a.v_stride : q + t * a.q_stride) + (int64_t)u.head * a.d;
            x[i] = __builtin_nontemporal_load(reinterpret_cast<const Vec *>(src + u.first));
            y[i] = __builtin_nontemporal_load(reinterpret_cast<const Vec *>(src + u.second));
        }
    };
    int item0 = tid >> a.unit_shift;
    load(item0);
    if (wave < n_rows) {
        const int t = row0 + wave;
        int b = -1, begin = t, end = t + 1;
        if (a.cu == nullptr) b = t < a.B ? t : -1;
        else b = find_sequence(a.cu, a.B, t, lane, begin, end);
        const int p = b < 0 ? -1 : a.lengths[b] - (end - t);
        const int64_t at = b < 0 ? -1 : cache_row(a.pt, b, p);
        if (lane == 0) {
            position[wave] = b < 0 ? INT_MIN : p;
            target[wave] = at;
        }
    }
    __syncthreads();
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
    for (; item0 < n_items; item0 += slots * kAppendUnits) {
#pragma unroll
        for (int i = 0; i < kAppendUnits; ++i) {
            const int item = item0 + i * slots;
            if (item >= n_items) continue;
            const Unit u = unit(item);
            if (position[u.row] == INT_MIN) continue;
            const float *const cosine = turn[0][u.row], *const sine = turn[1][u.row];
            if constexpr (INTERLEAVED) {
                const auto rotate = [&](Vec &z, int first) __attribute__((always_inline)) {
                    Vec r;
#pragma unroll
                    for (int e = 0; e < VEC; e += 2) {
                        const float cs = cosine[first / 2 + e / 2], sn = sine[first / 2 + e / 2], z0 = (float)z[e], z1 = (float)z[e + 1];
                        r[e] = (T)(z0 * cs - z1 * sn);
                        r[e + 1] = (T)(z0 * sn + z1 * cs);
                    }
                    z = r;
                };
                if (!u.is_v && u.first < a.rot) rotate(x[i], u.first);
                if (!u.is_v && u.second < a.rot) rotate(y[i], u.second);
            } else if (!u.is_v && c < rot_units) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float cs = cosine[c * VEC + e], sn = sine[c * VEC + e], x0 = (float)x[i][e], y0 = (float)y[i][e];
                    x[i][e] = (T)(x0 * cs - y0 * sn);
                    y[i][e] = (T)(x0 * sn + y0 * cs);
                }
            }
            const int64_t t = row0 + u.row, at = target[u.row];
            const auto put = [&](T *to) __attribute__((always_inline)) {
                *reinterpret_cast<Vec *>(to + u.first) = x[i];
                *reinterpret_cast<Vec *>(to + u.second) = y[i];
            };
            if (u.is_k || u.is_v) {
                if (at >= 0) put((u.is_k ? k_cache : v_cache) + (at * a.H_kv + u.head) * a.d);
                if (u.is_k && k_rot) put(k_rot + (t * a.H_kv + u.head) * a.d);
            } else {
                put(q_rot + (t * a.H + u.head) * a.d);
            }
        }
        if (item0 + slots * kAppendUnits < n_items) load(item0 + slots * kAppendUnits);
    }
}

} // namespace

template <typename T>
hipError_t launch_paged_append(const AppendArgs &args, const T *k, const T *v, const T *q, T *k_cache, T *v_cache, T *q_rot, T *k_rot, hipStream_t st)
{
    AppendArgs a = args;
    a.rows_per_wg = a.rows >= 1024 ? kAppendRows : 1;
    a.unit_shift = (a.d == 64 ? 2 : 3) + (sizeof(T) == 4);      // units of a head: d / 16 in bf16, d / 8 in float
    const dim3 grid((unsigned)((a.rows + a.rows_per_wg - 1) / a.rows_per_wg)), block(kAppendThreads);
    TimedLaunch tl(K_PAGED_APPEND, st);
    if (a.interleaved) hipLaunchKernelGGL((paged_append_kernel<T, true>), grid, block, 0, st, a, k, v, q, k_cache, v_cache, q_rot, k_rot);
    else hipLaunchKernelGGL((paged_append_kernel<T, false>), grid, block, 0, st, a, k, v, q, k_cache, v_cache, q_rot, k_rot);
    return hipGetLastError();
}

template hipError_t launch_paged_append<bf16_t>(const AppendArgs &, const bf16_t *, const bf16_t *, const bf16_t *, bf16_t *, bf16_t *, bf16_t *, bf16_t *,
                                                hipStream_t);
template hipError_t launch_paged_append<float>(const AppendArgs &, const float *, const float *, const float *, float *, float *, float *, float *,
                                               hipStream_t);

} // namespace lss
