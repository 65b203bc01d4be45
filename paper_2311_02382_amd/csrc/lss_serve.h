// What the kernels of the paged cache and of packed sequences share: which sequence a row belongs to, where a token lies in
// the cache, and the attention of one row by one wavefront.
#pragma once
#include "lss_common.h"
#include "lss_kernels.h"

#include <type_traits>

namespace lss {

// The sequence of packed row t: the last b in [0, B) with cu[b] <= t, if t < cu[b + 1] too, else -1.  By the whole wavefront, 64 starts at a
// time: as many dependent loads as B has digits to the base 64.  (cu ascending; whatever it holds, only its B + 1 entries are read.)
__device__ __forceinline__ int find_sequence(const int32_t *__restrict__ cu, int B, int t, int lane, int &begin, int &end)
{
    int lo = 0, n = B + 1;
    while (n > 1) {
        const int step = (n + 63) / 64, at = lane * step;
        const uint64_t below = __ballot(at < n && cu[lo + min(at, n - 1)] <= t);
        if (below == 0) return -1;
        const int last = 63 - __clzll((long long)below);
        lo += last * step;
        n = min(step, n - last * step);
    }
    if (lo >= B) return -1;
    begin = cu[lo];
    end = cu[lo + 1];
    return begin <= t && t < end ? lo : -1;
}

// Index of the cache row that holds token `position` of sequence b, in units of H_kv * d elements; -1 where the table names no page.
__device__ __forceinline__ int64_t cache_row(const PageTable &pt, int b, int position)
{
    const int nth = position >> pt.page_shift;
    if (position < 0 || nth >= pt.max_pages) return -1;
    const int page = pt.table[(int64_t)b * pt.max_pages + nth];
    if ((uint32_t)page >= (uint32_t)pt.n_pages) return -1;
    return ((int64_t)page << pt.page_shift) + (position & ((1 << pt.page_shift) - 1));
}

// ---- tiles of packed sequences: BR rows each, a row being one of a token's G heads
__device__ __forceinline__ int lane_sum_scan(int x)     // inclusive over the wavefront; all lanes active
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}
struct PackedTile { int q_begin, n_q, k_begin, n_k, tile; };
// Tile `rank` of a head of keys and values; false: there are fewer.  Up to 64 sequences, a lane each: tiles in the order of the keys they see (in
// steps of 64), most first, so that no long one starts last.  More sequences: in the sequences' order, sequence b's tiles from number
// floor(cu[b] G / BR) + b on -- room for all of them, one at most too much --, which is found like a row's sequence.
template <int BR>
__device__ __forceinline__ bool packed_tile(const PackedArgs &a, int G, int rank, int lane, PackedTile &t)
{
    const auto ends = [](const int32_t *cu, int b, int rows, int &begin, int &n) {
        begin = max(0, min(cu[b], rows));
        n = max(0, min(cu[b + 1], rows) - begin);
    };
    int b, begin = 0, n_q = 0, k_begin = 0, n_k = 0, tile;
    if (a.B <= 64) {
        if (lane < a.B) {
            ends(a.cu_q, lane, a.rows_q, begin, n_q);
            ends(a.cu_k, lane, a.rows_k, k_begin, n_k);
        }
        const int tiles = (n_q * G + BR - 1) / BR;
        // its tiles that see keys from number 64 (x - 1) on: tile j's last row is of token ((j + 1) BR - 1) / G
        const auto count = [&](int x) {
            if (x <= 1) return tiles;
            const int last = 64 * (x - 1);              // some row's position must reach it
            if (last >= n_k) return 0;
            return a.causal ? max(0, tiles - max(0, last - (n_k - n_q)) * G / BR) : tiles;
        };
        const auto total = [&](int x) { return __builtin_amdgcn_readlane(lane_sum_scan(count(x)), 63); };
        int lo = 1, hi = (a.rows_k + 63) / 64 + 1;      // total(lo) > rank >= total(hi)
        if (rank >= total(1)) return false;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (total(mid) > rank) lo = mid;
            else hi = mid;
        }
        const int above = count(lo + 1), mine = count(lo) - above, scan = lane_sum_scan(mine), in = rank - total(lo + 1);
        b = __ffsll((long long)__ballot(scan > in)) - 1;
        tile = tiles - count(lo) + in - (scan - mine);
        const auto of = [&](int x) { return __builtin_amdgcn_readlane(x, b); };
        t = {of(begin), of(n_q), of(k_begin), of(n_k), of(tile)};
        return true;
    }
    const auto first = [&](int i) { return (int)((int64_t)max(0, min(a.cu_q[i], a.rows_q)) * G / BR) + i; };
    int lo = 0, n = a.B;
    while (n > 1) {
        const int step = (n + 63) / 64, at = lane * step;
        const uint64_t below = __ballot(at < n && first(lo + min(at, n - 1)) <= rank);
        if (below == 0) return false;
        const int last = 63 - __clzll((long long)below);
        lo += last * step;
        n = min(step, n - last * step);
    }
    b = __builtin_amdgcn_readfirstlane(lo);
    ends(a.cu_q, b, a.rows_q, begin, n_q);
    ends(a.cu_k, b, a.rows_k, k_begin, n_k);
    t = {__builtin_amdgcn_readfirstlane(begin), __builtin_amdgcn_readfirstlane(n_q), __builtin_amdgcn_readfirstlane(k_begin),
         __builtin_amdgcn_readfirstlane(n_k), __builtin_amdgcn_readfirstlane(rank - first(b))};
    return t.tile >= 0 && t.tile < (t.n_q * G + BR - 1) / BR;
}

template <typename T> struct Vec16;
template <> struct Vec16<bf16_t> { typedef bf16x8 type; };
template <> struct Vec16<float> { typedef f32x4 type; };

__device__ __forceinline__ float wave_max(float x)      // all lanes active
{
    const auto step = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
        const int other = __builtin_amdgcn_update_dpp((int)0xff800000, __builtin_bit_cast(int, x), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        x = fmaxf(x, __builtin_bit_cast(float, other));
    };
    step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ __forceinline__ float wave_total(float x)
{
#pragma unroll
    for (int sh = 32; sh >= 1; sh >>= 1) x += __shfl_xor(x, sh);
    return x;
}

// Attention of one query row against the first n_keys keys by one wavefront, everything in fp32, for rows whose log-sum-exp is known and whose result was spoilt by
// a value that the row does not see: a value is multiplied only where its key is seen here.  64 keys at a time, a lane each for the scores; then each lane's 16 bytes
// of every (64 / CHUNKS)th value, LOADS loads on their way at once.  The weights' own sum divides them, so that the log-sum-exp's rounding does not matter.
// (Keys and values one by one, a broadcast each: 1000 cycles a key.)
template <typename T, int D, int LOADS>
__device__ __forceinline__ void row_attention(const T *q, const T *k, int64_t k_stride, const T *v, int64_t v_stride, int n_keys, float lse, int lane, T *out)
{
    typedef typename Vec16<T>::type Vec;
    constexpr int VEC = 16 / sizeof(T), CHUNKS = D / VEC, KEYS = 64 / CHUNKS;
    const float c = kLog2e / sqrtf((float)D), top = lse * kLog2e;
    if (lse == -INFINITY) n_keys = 0;                   // no key, or none with a weight: zeros
    const int mine = lane / CHUNKS, column = lane % CHUNKS * VEC;
    float acc[VEC], l = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
    for (int j0 = 0; j0 < n_keys; j0 += 64) {
        const T *const key = k + min(j0 + lane, n_keys - 1) * k_stride;
        float s = 0.f;
#pragma unroll (LOADS < 4 ? LOADS : 4)
        for (int i = 0; i < D; i += VEC) {
            const Vec a = *reinterpret_cast<const Vec *>(q + i), b = *reinterpret_cast<const Vec *>(key + i);
#pragma unroll
            for (int e = 0; e < VEC; ++e) s = fmaf((float)a[e], (float)b[e], s);
        }
        const float p = j0 + lane < n_keys ? fast_exp2(s * c - top) : 0.f;
        l += p;
#pragma unroll LOADS
        for (int i = 0; i < CHUNKS; ++i) {
            const int at = j0 + i * KEYS + mine;
            const Vec x = *reinterpret_cast<const Vec *>(v + min(at, n_keys - 1) * v_stride + column);
            const float w = __shfl(p, i * KEYS + mine);
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[e] = fmaf(w, at < n_keys ? (float)x[e] : 0.f, acc[e]);
        }
    }
    l = wave_total(l);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    Vec r;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
#pragma unroll
        for (int sh = CHUNKS; sh < 64; sh *= 2) acc[e] += __shfl_xor(acc[e], sh);
        r[e] = (T)(acc[e] * inv);
    }
    if (lane < CHUNKS) *reinterpret_cast<Vec *>(out + column) = r;
}

} // namespace lss
