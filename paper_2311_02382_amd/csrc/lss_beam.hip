// Beam search's choice over beams and vocabulary (lss_beam_select).
//
// total(k, v) = score_k + x_kv - log sum_v exp x_kv.  Within a beam the order of the totals is that of the logits, so a beam's candidates are found by their
// logits alone, in one pass over them that also keeps a running maximum and sum per lane; only n_out of each beam's get a total, in 64 bits.  Where these may be alike though a
// beam's logits are not (next to 0, or beside a large score), equal ones of a beam are compared by their logits once more.
//
// Rows are cut into chunks, a wavefront each (beam_rows_kernel), so that few rows fill the chip; a second launch, a workgroup per prompt, joins a row's chunks and
// its beams (beam_select_kernel).  Where rows are short (kDirect) and few the second kernel goes over them itself and there is no first one.
//
// What bounds them: long rows by vector issue (an exponential, a conversion, a product, a sum and half a maximum a logit): 256 rows of 128,256 in bf16, 66 MB, 18 to 19 us, 3.5 TB/s,
// the vector ALU busy 59 % of the cycles, loads alone 12.1; short ones by latency (64 rows of 32,001: 6 us).  The second launch is 7 to 10 us of steps one behind the other: lists, a bound, totals,
// ranking.  All of it, 32 prompts x 8 beams of 128,256: 25.9 us; 8 x 8 of 32,001, 16 chosen, 15.0; 4 beams of 256 6.4.
#include "lss_serve.h"

#include <algorithm>

namespace lss {

namespace {

constexpr int kLoads = 32;          // logits of a lane in one batch
constexpr int kBatch = 64 * kLoads;
constexpr int kCap = 256;           // candidates that a wavefront keeps before it drops all but the best
constexpr int kDirect = 2 * kBatch;
constexpr int kHeld = 12;           // floats of eight logits in LDS, behind which stands whose they are; neighbours in other banks
constexpr int kWaveLds = kCap * 8 + 64 * kHeld * 4;     // a wavefront's: its list, and 64 of those
constexpr int kFew = 16;            // lanes' largest suffice to find a bound that little more than so many reach
constexpr int kAtOnce = 6;          // candidates of a row that a lane of the second launch looks at at once
constexpr int kUnbounded = 128;     // totals of a prompt's candidates that are ranked as they are; of more those at or above a bound
constexpr int kRanked = 320;        // of those, at most, that are compared with one another only; room for them in one wavefront's list

struct Candidate { uint32_t value, index; };            // value: a float as an ascending whole number; 0: none
struct ChunkStats { double sum; float top, unused; };   // sum of exp(x - top)

__device__ __forceinline__ uint32_t ascending(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);        // (-0 equals 0)
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float descend(uint32_t a) { return __builtin_bit_cast(float, a & 0x80000000u ? a ^ 0x80000000u : ~a); }
constexpr uint32_t kLeast = 0x00800000u;                // of the lowest finite value: -infinity is no candidate
__device__ __forceinline__ int count_of(bool x) { return __popcll(__ballot(x)); }
// a wavefront's own LDS: what one lane wrote is there for the others
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

typedef __attribute__((address_space(3))) Candidate LdsCandidate;
__device__ __forceinline__ uint32_t wave_max_of(uint32_t x)      // all lanes active
{
    const auto step = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
        x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
    };
    step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
// A number that from n to `limit` values are at or above, or if there is none (values alike) the n-th largest value.  count(t): how many are at or above t, at least n for
// `low`; none is above `most`.  (Halving ends after a few steps; the n-th largest itself, bit by bit, took 32.)
template <typename F> __device__ __forceinline__ uint32_t at_least(uint32_t low, uint32_t most, int n, int limit, F &&count)
{
    uint32_t lo = low, hi = max(most, low);             // the n-th largest is lo .. hi
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        const int c = count(mid);
        if (c < n) hi = mid - 1;
        else lo = mid;
        if (c >= n && c <= limit) break;
    }
    return lo;
}
struct Bound { uint32_t value, index; int count; };     // what is below (value, index) has been beaten; candidates in the list
// The list is cut down to the n best and at most `limit`: those at or above a bound, and where too many equal it those with the lowest indices.  (A function of its own: it
// is called from several places, and seldom.)
template <int R>                                        // 64 R of them at most
__device__ __attribute__((noinline)) Bound prune(LdsCandidate *list, int count, int n_, int limit_, int lane, uint32_t low_)
{
    const auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    const int n = uniform(n_), limit = uniform(limit_);
    wave_sync();
    Candidate c[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        c[r] = {0u, 0u};
        if (r * 64 + lane < count) c[r].value = list[r * 64 + lane].value, c[r].index = list[r * 64 + lane].index;
    }
    const auto all = [&](auto &&test) __attribute__((always_inline)) {
        int sum = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) sum += count_of(test(c[r]));
        return sum;
    };
    uint32_t most = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) most = max(most, c[r].value);
    const uint32_t t = at_least((uint32_t)uniform((int)low_), wave_max_of(most), n, limit, [&](uint32_t least) __attribute__((always_inline)) {
        return all([&](const Candidate &x) __attribute__((always_inline)) { return x.value >= least; });
    });
    uint32_t last = ~0u;
    if (all([&](const Candidate &x) __attribute__((always_inline)) { return x.value >= t; }) > limit) {
        const int wanted = n - all([&](const Candidate &x) __attribute__((always_inline)) { return x.value > t; });
        last = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t upto = last | ((1u << bit) - 1);
            if (all([&](const Candidate &x) __attribute__((always_inline)) { return x.value == t && x.index <= upto; }) < wanted) last |= 1u << bit;
        }
    }
    wave_sync();
    count = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool stays = c[r].value > t || (c[r].value == t && c[r].index <= last);
        const uint64_t who = __ballot(stays);
        const int at = count + __popcll(who & (((uint64_t)1 << lane) - 1));
        if (stays) list[at].value = c[r].value, list[at].index = c[r].index;
        count += __popcll(who);
    }
    wave_sync();
    return {t, last, count};
}

// The `n` best of the candidates that a wavefront has seen, by value, then by the lower index, in kCap places of LDS.  Whatever is below the bound (value, index) has
// been beaten by n others.
struct Best {
    LdsCandidate *list;
    __attribute__((address_space(3))) float *held;
    int n, lane;
    Bound bound{kLeast, ~0u, 0};                        // wavefront-uniform
    float value_f = -3.402823466e38f;

    __device__ __forceinline__ Best(char *lds, int n_, int lane_)
        : list((LdsCandidate *)lds), held((__attribute__((address_space(3))) float *)(lds + kCap * sizeof(Candidate))), n(n_), lane(lane_) {}
    __device__ __forceinline__ int count() const { return bound.count; }
    // of 64 R values, R a lane, at least n of which are at or above the bound's, at least n are at or above what this returns
    template <int R> __device__ __forceinline__ uint32_t nth(const uint32_t (&v)[R]) const
    {
        uint32_t most = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) most = max(most, v[r]);
        return at_least(bound.value, wave_max_of(most), n, n + n / 4, [&](uint32_t least) __attribute__((always_inline)) {
            int c = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) c += count_of(v[r] >= least);
            return c;
        });
    }
    __device__ __forceinline__ void raise(uint32_t v)
    {
        bound.value = v, bound.index = ~0u;
        value_f = descend(v);
    }
    __device__ __forceinline__ void cut(int limit)      // (n or more)
    {
        if (bound.count <= limit) return;
        const Bound b = bound.count <= 64 ? prune<1>(list, bound.count, n, limit, lane, bound.value) : prune<kCap / 64>(list, bound.count, n, limit, lane, bound.value);
        const auto uniform = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
        bound = {uniform(b.value), uniform(b.index), (int)uniform((uint32_t)b.count)};
        value_f = descend(bound.value);
    }
    // a candidate a lane
    __device__ __forceinline__ void offer(uint32_t v, uint32_t i)
    {
        const bool in = v > bound.value || (v == bound.value && i <= bound.index);
        const uint64_t who = __ballot(in);
        if (who == 0) return;
        const int at = bound.count + __popcll(who & (((uint64_t)1 << lane) - 1));
        if (in) list[at].value = v, list[at].index = i;
        bound.count += __popcll(who);
        if (bound.count > kCap - 64) cut(96);
    }
};

__device__ __forceinline__ double lanes_total(double x)
{
#pragma unroll
    for (int sh = 32; sh >= 1; sh >>= 1) x += __shfl_xor(x, sh);
    return x;
}

// exp(x), log2 e in two parts: one rounding of it would shift a row's weights all the same way, and the row's sum with them
constexpr float kLog2eUp = 1.44269502f;
__device__ __forceinline__ float exp_of(float x) { return fast_exp2(fmaf(x, 1.9259629e-8f, x * kLog2eUp)); }

// Tokens v0 .. v1 - 1 of a row (v0 a multiple of kBatch): the best of them go to `best`.  Which lane has which token does not depend on where the row lies (rows of an
// odd number of logits are not 16-byte aligned, and loads need not be): rows alike have sums alike to the last bit, and equal totals then go to the lower beam.
template <typename T>
__device__ __forceinline__ ChunkStats scan_row(const T *row, int64_t v0, int64_t v1, Best &best)
{
    constexpr int VEC = 16 / sizeof(T), N = kLoads / VEC;
    struct __attribute__((packed, aligned(sizeof(T)))) Anywhere { typename Vec16<T>::type v; };
    const int lane = best.lane;
    float top = -INFINITY;
    double sum = 0.0;
    typename Vec16<T>::type ahead[N];                   // the next batch is on its way while one is worked on
    const auto load = [&](int64_t v) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t at = v + (i * 64 + lane) * VEC;
            if (at + VEC <= v1) ahead[i] = reinterpret_cast<const Anywhere *>(row + at)->v;
            else
#pragma unroll
                for (int e = 0; e < VEC; ++e) ahead[i][e] = at + e < v1 ? row[at + e] : (T)-INFINITY;
        }
    };
    load(v0);
    for (int64_t v = v0; v < v1; v += kBatch) {
        float x[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) x[i] = (float)ahead[i / VEC][i % VEC];
        if (v + kBatch < v1) load(v + kBatch);
        float most = -INFINITY, of_eight[kLoads / 8];
#pragma unroll
        for (int g = 0; g < kLoads / 8; ++g) {
            of_eight[g] = x[8 * g];
#pragma unroll
            for (int i = 1; i < 8; ++i) of_eight[g] = fmaxf(of_eight[g], x[8 * g + i]);
            most = fmaxf(most, of_eight[g]);
        }
        const float higher = fmaxf(top, most), use = higher == -INFINITY ? 0.f : higher;
        float part[2] = {0.f, 0.f};
        if (__all(fabsf(use) <= 16384.f)) {
            // exp(x - use) = 2^(x c - m) 2^(m - use c), c log2 e rounded, m use c rounded: one instruction a logit ahead of its exponential, and what m is off by is made up for
            // in the sum.  (Off by x - use times 1.3e-8 and half a step of the exponent.)
            const float m = use * kLog2eUp;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) part[i & 1] += fast_exp2(fmaf(x[i], kLog2eUp, -m));
            part[0] = (part[0] + part[1]) * fast_exp2(-fmaf(use, kLog2eUp, -m));
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) part[i & 1] += exp_of(x[i] - use);
            part[0] += part[1];
        }
        sum = sum * (double)exp_of(top - use) + (double)part[0];
        top = higher;
        // the bound from the largest of the lanes, or where they would be too few of their eights: n of them are candidates themselves
        if (best.n <= kFew) {
            if (count_of(most >= best.value_f) >= best.n) best.raise(max(best.bound.value, best.nth<1>({ascending(most)})));
        } else {
            int candidates = 0;
#pragma unroll
            for (int g = 0; g < kLoads / 8; ++g) candidates += count_of(of_eight[g] >= best.value_f);
            if (candidates >= best.n) {
                uint32_t largest[kLoads / 8];
#pragma unroll
                for (int g = 0; g < kLoads / 8; ++g) largest[g] = ascending(of_eight[g]);
                const uint32_t t = best.nth(largest);
                if (t > best.bound.value) best.raise(t);
            }
        }
        // Few eights of a lane's logits have a candidate: they go through LDS, up to 64 of them at a time, to all lanes.  (Slot by slot, 32 tests and an offer for each
        // candidate: 8 of 23 us for 256 rows of 128,256; lane by lane 6.5.)
        if (!__any(most >= best.value_f)) continue;
        int n = 0;
        const auto offer_held = [&] __attribute__((always_inline)) {
            wave_sync();
            for (int i0 = 0; i0 < 8 * n; i0 += 64) {
                const int at = min(i0 + lane, 8 * n - 1), from = at / 8 * kHeld;
                const float y = best.held[from + at % 8];
                const int first = __builtin_bit_cast(int, best.held[from + 8]), i = (first & 63) * 8 + at % 8;      // of the eight's lane
                best.offer(i0 + lane < 8 * n && y >= best.value_f ? ascending(y) : 0u, (uint32_t)(v + (i / VEC * 64 + (first >> 6)) * VEC + i % VEC));
            }
            wave_sync();
            n = 0;
        };
#pragma unroll
        for (int g = 0; g < kLoads / 8; ++g) {
            const bool mine = of_eight[g] >= best.value_f;
            const uint64_t who = __ballot(mine);
            if (who == 0) continue;
            if (n + __popcll(who) > 64) offer_held();
            if (mine) {
                const auto to = best.held + (n + __popcll(who & (((uint64_t)1 << lane) - 1))) * kHeld;
                *(__attribute__((address_space(3))) f32x4 *)to = f32x4{x[8 * g], x[8 * g + 1], x[8 * g + 2], x[8 * g + 3]};
                *(__attribute__((address_space(3))) f32x4 *)(to + 4) = f32x4{x[8 * g + 4], x[8 * g + 5], x[8 * g + 6], x[8 * g + 7]};
                to[8] = __builtin_bit_cast(float, lane << 6 | g);
            }
            n += __popcll(who);
        }
        if (n > 0) offer_held();
    }
    const float all = wave_max(top);
    return {lanes_total(sum * (double)exp_of(all == -INFINITY ? 0.f : top - all)), all, 0.f};
}

struct BeamArgs {
    int64_t stride;
    int B, K, V, N, end_token, chunks, kept;    // candidates that a chunk hands on: a few more than are needed, so that it seldom has to look for the best
    int64_t chunk;          // tokens of one, a multiple of kBatch
};

template <typename T>
__global__ __launch_bounds__(256) void beam_rows_kernel(BeamArgs a, const T *__restrict__ logits, const uint8_t *__restrict__ finished, Candidate *__restrict__ lists,
                                                        ChunkStats *__restrict__ stats)
{
    __shared__ __attribute__((aligned(16))) char lds[4][kWaveLds];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)blockIdx.x * 4 + wave;
    const int row = (int)(item / a.chunks), chunk = (int)(item % a.chunks);
    if (row >= a.B * a.K || (finished && finished[row])) return;
    Best best(lds[wave], a.N, lane);
    const ChunkStats s = scan_row<T>(logits + row * a.stride, chunk * a.chunk, min((int64_t)a.V, (chunk + 1) * a.chunk), best);
    best.cut(a.kept);
    wave_sync();
    if (lane < a.kept) lists[item * a.kept + lane] = lane < best.count() ? Candidate{best.list[lane].value, best.list[lane].index} : Candidate{0u, 0u};
    if (lane == 0) stats[item] = s;
}

// A workgroup per prompt, of up to 16 wavefronts that take a beam each.  A beam's candidates -- the n_out best, or a few more where that saves looking for them -- go to LDS
// with their totals; a candidate's place in the result is the number of those that are better.  Where there are many, those below a bound on the n_out-th largest
// are passed over.  DIRECT: from the logits.
template <typename T, bool DIRECT>
__global__ __launch_bounds__(1024) void beam_select_kernel(BeamArgs a, const T *__restrict__ logits, const float *__restrict__ scores,
                                                           const uint8_t *__restrict__ finished, const Candidate *__restrict__ lists,
                                                           const ChunkStats *__restrict__ stats, int per_beam, float *__restrict__ scores_out,
                                                           int32_t *__restrict__ parents, int32_t *__restrict__ tokens, uint8_t *__restrict__ finished_out)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ int n_candidates, n_above, alike, above[32];
    double *const total = reinterpret_cast<double *>(smem);                        // [K per_beam]
    uint32_t *const flat = reinterpret_cast<uint32_t *>(total + a.K * per_beam);    // beam * V + token
    char *const lds = smem + ((a.K * per_beam * 12 + 15) & ~15);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6, b = blockIdx.x;
    if (tid == 0) n_candidates = n_above = alike = 0;
    if (tid < 32) above[tid] = 0;
    __syncthreads();
    for (int k = wave; k < a.K; k += waves) {
        const int64_t row = (int64_t)b * a.K + k;
        const int n_list = a.chunks * a.kept;
        const Candidate *const list = lists + row * n_list;
        const ChunkStats *const mine = stats + row * a.chunks;
        // (all that a row of up to 64 chunks needs first is on its way at once)
        const float score = scores[row];
        const bool ended = finished && finished[row];
        Candidate c[kAtOnce];
        ChunkStats chunk{0.0, -INFINITY, 0.f};
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) c[i] = list[min(i * 64 + lane, n_list - 1)];
            if (lane < a.chunks) chunk = mine[lane];
        }
        if (!(fabsf(score) < INFINITY)) continue;
        if (ended) {
            if (lane == 0) {
                const int at = atomicAdd(&n_candidates, 1);
                total[at] = score;
                flat[at] = (uint32_t)k * a.V + a.end_token;
            }
            continue;
        }
        Best best(lds + wave * kWaveLds, a.N, lane);
        ChunkStats s;
        if constexpr (DIRECT) {
            s = scan_row<T>(logits + row * a.stride, 0, a.V, best);
        } else {
            float top = chunk.top;
            for (int i = 64 + lane; i < a.chunks; i += 64) top = fmaxf(top, mine[i].top);
            top = wave_max(top);
            const auto weight = [&](float x) { return (double)exp_of(top == -INFINITY ? 0.f : x - top); };
            double sum = lane < a.chunks ? chunk.sum * weight(chunk.top) : 0.0;
            for (int i = 64 + lane; i < a.chunks; i += 64) sum += mine[i].sum * weight(mine[i].top);
            s = {lanes_total(sum), top, 0.f};
            for (int i0 = 0; i0 < n_list; i0 += 64 * kAtOnce) {
                if (i0 > 0)
#pragma unroll
                    for (int i = 0; i < kAtOnce; ++i) c[i] = list[min(i0 + i * 64 + lane, n_list - 1)];
                uint32_t values[kAtOnce], most = 0;
                int candidates = 0;
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    values[i] = i0 + i * 64 + lane < n_list ? c[i].value : 0u;
                    most = max(most, values[i]);
                }
                if (a.N <= kFew) {
                    if (count_of(most > best.bound.value) >= a.N) best.raise(max(best.bound.value, best.nth<1>({most})));
                } else {
#pragma unroll
                    for (int i = 0; i < kAtOnce; ++i) candidates += count_of(values[i] > best.bound.value);
                    if (candidates >= a.N) best.raise(max(best.bound.value, best.nth(values)));
                }
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) best.offer(values[i], c[i].index);
            }
        }
        best.cut(per_beam);
        wave_sync();
        const double lse = (double)s.top + log(s.sum);
        if (!(fabs(lse) < (double)INFINITY)) continue;
        int first = __builtin_amdgcn_readfirstlane(best.count());
        if (lane == 0) first = atomicAdd(&n_candidates, first);
        first = __builtin_amdgcn_readfirstlane(first);
        // Two of its logits differ by 2^-24 of either at least, their totals' roundings by less than 2^-51 of |logit| + |lse| + |score|: totals may be alike where the logits are not only where
        // a logit that is not 0 is below 2^-26 of |lse| + |score|
        const float beside = (float)(fabs(lse) + fabs((double)score));
        bool next_to_0 = false;
        for (int i = lane; i < best.count(); i += 64) {
            const float x = descend(best.list[i].value);
            total[first + i] = (double)score + ((double)x - lse);
            flat[first + i] = (uint32_t)k * a.V + best.list[i].index;
            next_to_0 = next_to_0 || (x != 0.f && fabsf(x) * 0x1p26f < beside);
        }
        if (next_to_0) alike = 1;
    }
    __syncthreads();
    const int n = n_candidates;
    // a bound of the totals in 32 bits, as ascending whole numbers: n_out are at or above it
    uint32_t bound = 0;
    if (n > kUnbounded) {
        int step = 0;
        bound = at_least(0, ascending(3.402823466e38f), a.N, max(kUnbounded / 2, 2 * a.N), [&](uint32_t least) {
            int mine = 0;
            for (int i = tid; i < n; i += blockDim.x) mine += ascending((float)total[i]) >= least;
            mine = lane_sum_scan(mine);
            if (lane == 63) atomicAdd(&above[step], mine);
            __syncthreads();
            return __builtin_amdgcn_readfirstlane(above[step++]);       // (32 steps at most)
        });
    }
    const auto put = [&](int better, double x, uint32_t place) {
        if (better >= a.N) return;
        const int k = (int)(place / (uint32_t)a.V), token = (int)(place - (uint32_t)k * a.V);
        const int64_t to = (int64_t)b * a.N + better;
        scores_out[to] = (float)x;
        parents[to] = b * a.K + k;
        tokens[to] = token;
        if (finished_out) finished_out[to] = token == a.end_token;          // (what a beam that has ended goes on with, too)
    };
    const auto better_than = [&](const double *totals, const uint32_t *places, double x, uint32_t place, int from, int to) __attribute__((always_inline)) {
        int better = 0;
        if (alike) {
            // of equal totals of one beam the larger logit, as it is
            const uint32_t V = (uint32_t)a.V, k = place / V;
            const T *const row = logits + ((int64_t)b * a.K + k) * a.stride;
#pragma unroll 1
            for (int j = from; j < to; ++j) {
                const double y = totals[j];
                const uint32_t at = places[j];
                bool before = at < place;
                if (y == x && at != place && at / V == k) {
                    const float theirs = (float)row[at - k * V], mine = (float)row[place - k * V];
                    before = theirs > mine || (theirs == mine && before);
                }
                better += (int)(y > x) | ((int)(y == x) & (int)before);
            }
            return better;
        }
#pragma unroll 8
        for (int j = from; j < to; ++j) {               // (no branch: reads ahead of one another)
            const double y = totals[j];
            const uint32_t at = places[j];
            better += (int)(y > x) | ((int)(y == x) & (int)(at < place));
        }
        return better;
    };
    // (The lists are done with: there go those at or above the bound, and how many are better than each.  Whoever is better than one of them is one of them.)
    double *const high = n <= kUnbounded ? total : reinterpret_cast<double *>(lds);
    uint32_t *const high_flat = n <= kUnbounded ? flat : reinterpret_cast<uint32_t *>(lds + 8 * kRanked);
    int *const better = reinterpret_cast<int *>(lds + 12 * kRanked);
    static_assert(kRanked * 16 <= kWaveLds, "");
    if (n <= kUnbounded) {
        for (int i = tid; i < n; i += blockDim.x) better[i] = 0;
    } else {
        for (int i = tid; i < n; i += blockDim.x) {
            const double x = total[i];
            if (ascending((float)x) < bound) continue;
            const int at = atomicAdd(&n_above, 1);
            if (at < kRanked) high[at] = x, high_flat[at] = flat[i], better[at] = 0;
        }
    }
    __syncthreads();
    const int m = n <= kUnbounded ? n : n_above;
    if (m <= kRanked) {
        // the others are shared out among as many groups of wavefronts as there are
        const int in_a_group = (m + 63) & ~63, groups = max(1, (int)blockDim.x / max(in_a_group, 1)), each = (m + groups - 1) / groups;
        for (int s = tid; s < in_a_group * groups; s += blockDim.x) {
            const int i = s % in_a_group, group = s / in_a_group;
            if (i >= m) continue;
            const int count = better_than(high, high_flat, high[i], high_flat[i], min(m, group * each), min(m, (group + 1) * each));
            if (count > 0) atomicAdd(&better[i], count);
        }
        __syncthreads();
        for (int i = tid; i < m; i += blockDim.x) put(better[i], high[i], high_flat[i]);
    } else {
        // (more than that alike)
        for (int i = tid; i < n; i += blockDim.x) put(better_than(total, flat, total[i], flat[i], 0, n), total[i], flat[i]);
    }
    for (int i = n + tid; i < a.N; i += blockDim.x) {
        const int64_t to = (int64_t)b * a.N + i;
        scores_out[to] = -INFINITY;
        parents[to] = tokens[to] = -1;
        if (finished_out) finished_out[to] = 1;
    }
}

// Chunks of a row: a batch at least, and as many as it takes to have 4096 wavefronts, but no more than 16384 candidates for the workgroup that joins them (32 beams of
// 128,256 logits, 64 from each, one prompt: 74 us, 87 without that; 16 of 50,000, 32 from each: 24.4, with 4096 candidates 30.7).
BeamArgs chunked(int64_t stride, int B, int K, int V, int N, int end_token)
{
    BeamArgs a{stride, B, K, V, N, end_token, 0, std::min(N + N / 4 + 4, 64), 0};
    const int64_t batches = ((int64_t)V + kBatch - 1) / kBatch, wanted = std::max<int64_t>(1, std::min<int64_t>(4096 / ((int64_t)B * K), 16384 / (K * a.kept)));
    const int64_t each = (batches + wanted - 1) / wanted;
    a.chunk = each * kBatch;
    a.chunks = (int)((batches + each - 1) / each);
    return a;
}
// (32 beams of 206 logits, 64 prompts: two rows by each wavefront one after the other would take longer than a launch)
bool is_direct(int K, int V) { return V <= kDirect && K <= 16; }
size_t lists_bytes(const BeamArgs &a) { return ((size_t)a.B * a.K * a.chunks * a.kept * sizeof(Candidate) + 15) & ~(size_t)15; }

} // namespace

size_t beam_select_workspace_bytes(int B, int K, int V, int N)
{
    if (is_direct(K, V)) return 0;
    const BeamArgs a = chunked(0, B, K, V, N, 0);
    return lists_bytes(a) + (size_t)B * K * a.chunks * sizeof(ChunkStats);
}

template <typename T>
hipError_t launch_beam_select(const T *logits, int64_t stride, const float *scores, const uint8_t *finished, int end_token, int B, int K, int V, int N, void *workspace,
                              float *scores_out, int32_t *parents, int32_t *tokens, uint8_t *finished_out, hipStream_t st)
{
    const BeamArgs a = chunked(stride, B, K, V, N, end_token);
    Candidate *const lists = static_cast<Candidate *>(workspace);
    ChunkStats *const stats = reinterpret_cast<ChunkStats *>(static_cast<char *>(workspace) + (is_direct(K, V) ? 0 : lists_bytes(a)));
    // (12 bytes of LDS a candidate, of 4096 at most, and 5 KB a wavefront: more than the 64 KB that a launch may have without asking)
    const int per_beam = K * N <= 1024 ? 2 * N : N, waves = std::min(K, 16);
    const size_t lds = (((size_t)K * per_beam * 12 + 15) & ~(size_t)15) + (size_t)waves * kWaveLds;
    const bool direct = is_direct(K, V);
    if (lds > 65536 - 1024) {
        static DeviceOnce once[2];
        const hipError_t e = allow_lds(direct ? beam_select_kernel<T, true> : beam_select_kernel<T, false>, 4096 * 12 + 16 * kWaveLds, once[direct]);
        if (e != hipSuccess) return e;
    }
    if (direct) {
        TimedLaunch tl(K_BEAM_SELECT, st);
        hipLaunchKernelGGL((beam_select_kernel<T, true>), dim3((unsigned)B), dim3(64 * waves), lds, st, a, logits, scores, finished, lists, stats, per_beam, scores_out,
                           parents, tokens, finished_out);
        return hipGetLastError();
    }
    {
        TimedLaunch tl(K_BEAM_ROWS, st);
        hipLaunchKernelGGL((beam_rows_kernel<T>), dim3((unsigned)(((int64_t)B * K * a.chunks + 3) / 4)), dim3(256), 0, st, a, logits, finished, lists, stats);
    }
    TimedLaunch tl(K_BEAM_SELECT, st);
    hipLaunchKernelGGL((beam_select_kernel<T, false>), dim3((unsigned)B), dim3(64 * waves), lds, st, a, logits, scores, finished, lists, stats, per_beam, scores_out, parents,
                       tokens, finished_out);
    return hipGetLastError();
}

template hipError_t launch_beam_select<bf16_t>(const bf16_t *, int64_t, const float *, const uint8_t *, int, int, int, int, int, void *, float *, int32_t *, int32_t *,
                                               uint8_t *, hipStream_t);
template hipError_t launch_beam_select<float>(const float *, int64_t, const float *, const uint8_t *, int, int, int, int, int, void *, float *, int32_t *, int32_t *,
                                              uint8_t *, hipStream_t);

} // namespace lss
