// Beam search's choice over beams and vocabulary (lss_beam_select).
//
// total(k, v) = score_k + x_kv - log sum_v exp x_kv.  Within a beam the order of the totals is that of the logits, so a beam's candidates are found by their
// logits alone, in one pass over them that also keeps a running maximum and sum per lane; only n_out of each beam's get a total, in 64 bits.
//
// Rows are cut into chunks, a wavefront each (beam_rows_kernel), so that few rows fill the chip; a second launch, a workgroup per prompt, joins a row's chunks and
// its beams (beam_select_kernel).  Where rows are short (kDirect) the second kernel goes over them itself and there is no first one.
#include "lss_serve.h"

#include <algorithm>

namespace lss {

namespace {

constexpr int kLoads = 32;          // logits of a lane in one batch
constexpr int kBatch = 64 * kLoads;
constexpr int kCap = 256;           // candidates that a wavefront keeps before it drops all but the best
constexpr int kDirect = 2 * kBatch;

struct Candidate { uint32_t value, index; };            // value: a float as an ascending whole number; 0: none
struct ChunkStats { double sum; float top, unused; };    // sum of exp(x - top)

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

// The `n` best of the candidates that a wavefront has seen, by value, then by the lower index, in kCap places of LDS.  Whatever is below the bound (value, index) has
// been beaten by n others.
struct Best {
    Candidate *list;
    int n, lane, count = 0;
    uint32_t value = kLeast, index = ~0u;               // the bound; wavefront-uniform
    float value_f = -3.402823466e38f;

    __device__ __forceinline__ Best(Candidate *list_, int n_, int lane_) : list(list_), n(n_), lane(lane_) {}
    __device__ __forceinline__ void raise(uint32_t v, uint32_t i)
    {
        value = v, index = i;
        value_f = descend(v);
    }
    // n-th largest of `v`, a value a lane; 0 where there are fewer that are not
    __device__ __forceinline__ uint32_t nth(uint32_t v) const
    {
        uint32_t t = 0;
        for (int bit = 31; bit >= 0; --bit)
            if (count_of(v >= (t | 1u << bit)) >= n) t |= 1u << bit;
        return t;
    }
    // all but the best go: the n-th largest value, bit by bit, and the lowest indices of those that equal it
    __device__ void prune()
    {
        constexpr int R = kCap / 64;
        wave_sync();
        Candidate c[R];
#pragma unroll
        for (int r = 0; r < R; ++r) c[r] = r * 64 + lane < count ? list[r * 64 + lane] : Candidate{0u, 0u};
        const auto all = [&](auto &&test) {
            int sum = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) sum += count_of(test(c[r]));
            return sum;
        };
        if (count <= n) return;
        uint32_t t = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t higher = t | 1u << bit;
            if (all([&](const Candidate &x) { return x.value >= higher; }) >= n) t = higher;
        }
        const int wanted = n - all([&](const Candidate &x) { return x.value > t; });
        uint32_t last = ~0u;
        if (all([&](const Candidate &x) { return x.value == t; }) > wanted) {
            last = 0;
            for (int bit = 31; bit >= 0; --bit) {
                const uint32_t most = last | ((1u << bit) - 1);
                if (all([&](const Candidate &x) { return x.value == t && x.index <= most; }) < wanted) last |= 1u << bit;
            }
        }
        wave_sync();
        count = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool stays = c[r].value > t || (c[r].value == t && c[r].index <= last);
            const uint64_t who = __ballot(stays);
            if (stays) list[count + __popcll(who & (((uint64_t)1 << lane) - 1))] = c[r];
            count += __popcll(who);
        }
        wave_sync();
        raise(t, last);
    }
    // a candidate a lane
    __device__ __forceinline__ void offer(uint32_t v, uint32_t i)
    {
        const bool in = v > value || (v == value && i <= index);
        const uint64_t who = __ballot(in);
        if (who == 0) return;
        if (in) list[count + __popcll(who & (((uint64_t)1 << lane) - 1))] = {v, i};
        count += __popcll(who);
        if (count > kCap - 64) prune();
    }
};

__device__ __forceinline__ double lanes_total(double x)
{
#pragma unroll
    for (int sh = 32; sh >= 1; sh >>= 1) x += __shfl_xor(x, sh);
    return x;
}

// exp(x) with log2 e in two parts: one rounding of it would shift every weight of a row the same way, and the row's sum with it
__device__ __forceinline__ float exp_of(float x) { return fast_exp2(fmaf(x, 1.9259629e-8f, x * 1.44269502f)); }

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
    for (int64_t v = v0; v < v1; v += kBatch) {
        float x[kLoads];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t at = v + (i * 64 + lane) * VEC;
            if (at + VEC <= v1) {
                const typename Vec16<T>::type some = reinterpret_cast<const Anywhere *>(row + at)->v;
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[i * VEC + e] = (float)some[e];
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[i * VEC + e] = at + e < v1 ? (float)row[at + e] : -INFINITY;
            }
        }
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) most = fmaxf(most, x[i]);
        const float higher = fmaxf(top, most), use = higher == -INFINITY ? 0.f : higher;
        float part = 0.f;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) part += exp_of(x[i] - use);
        sum = sum * (double)exp_of(top - use) + (double)part;
        top = higher;
        // the bound from the lanes' largest: n of them are candidates themselves
        if (count_of(most >= best.value_f) >= best.n) {
            const uint32_t t = best.nth(ascending(most));
            if (t > best.value) best.raise(t, ~0u);
        }
        if (!__any(most >= best.value_f)) continue;
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            if (__any(x[i] >= best.value_f))
                best.offer(x[i] >= best.value_f ? ascending(x[i]) : 0u, (uint32_t)(v + (i / VEC * 64 + lane) * VEC + i % VEC));
    }
    const float all = wave_max(top);
    return {lanes_total(sum * (double)exp_of(all == -INFINITY ? 0.f : top - all)), all, 0.f};
}

struct BeamArgs {
    int64_t stride;
    int B, K, V, N, end_token, chunks;
    int64_t chunk;          // tokens of one, a multiple of kBatch
};

template <typename T>
__global__ __launch_bounds__(256) void beam_rows_kernel(BeamArgs a, const T *__restrict__ logits, const uint8_t *__restrict__ finished, Candidate *__restrict__ lists,
                                                        ChunkStats *__restrict__ stats)
{
    __shared__ Candidate lds[4][kCap];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)blockIdx.x * 4 + wave;
    const int row = (int)(item / a.chunks), chunk = (int)(item % a.chunks);
    if (row >= a.B * a.K || (finished && finished[row])) return;
    Best best(lds[wave], a.N, lane);
    const ChunkStats s = scan_row<T>(logits + row * a.stride, chunk * a.chunk, min((int64_t)a.V, (chunk + 1) * a.chunk), best);
    best.prune();
    if (lane < a.N) lists[item * a.N + lane] = lane < best.count ? best.list[lane] : Candidate{0u, 0u};
    if (lane == 0) stats[item] = s;
}

// A workgroup per prompt, of up to 16 wavefronts that take a beam each; then its beams' candidates, K N of them in LDS, are sorted by their totals (in 64 bits), the
// lower (beam, token) first.  DIRECT: from the logits.
template <typename T, bool DIRECT>
__global__ __launch_bounds__(1024) void beam_select_kernel(BeamArgs a, const T *__restrict__ logits, const float *__restrict__ scores,
                                                           const uint8_t *__restrict__ finished, const Candidate *__restrict__ lists,
                                                           const ChunkStats *__restrict__ stats, int places, float *__restrict__ scores_out,
                                                           int32_t *__restrict__ parents, int32_t *__restrict__ tokens, uint8_t *__restrict__ finished_out)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    double *const total = reinterpret_cast<double *>(smem);                        // [places]
    uint32_t *const flat = reinterpret_cast<uint32_t *>(total + places);           // [places]: beam * V + token
    Candidate *const lds = reinterpret_cast<Candidate *>(flat + places);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6, b = blockIdx.x;
    for (int i = tid; i < places; i += blockDim.x) {
        total[i] = -INFINITY;
        flat[i] = ~0u;
    }
    __syncthreads();
    for (int k = wave; k < a.K; k += waves) {
        const int64_t row = (int64_t)b * a.K + k;
        const float score = scores[row];
        if (!(fabsf(score) < INFINITY)) continue;
        if (finished && finished[row]) {
            if (lane == 0) {
                total[k * a.N] = score;
                flat[k * a.N] = (uint32_t)k * a.V + a.end_token;
            }
            continue;
        }
        Best best(lds + wave * kCap, a.N, lane);
        ChunkStats s;
        if constexpr (DIRECT) {
            s = scan_row<T>(logits + row * a.stride, 0, a.V, best);
        } else {
            float top = -INFINITY;
            double sum = 0.0;
            const ChunkStats *const mine = stats + row * a.chunks;
            for (int i = lane; i < a.chunks; i += 64) top = fmaxf(top, mine[i].top);
            top = wave_max(top);
            for (int i = lane; i < a.chunks; i += 64) sum += mine[i].sum * (double)exp_of(top == -INFINITY ? 0.f : mine[i].top - top);
            s = {lanes_total(sum), top, 0.f};
            const Candidate *const list = lists + row * a.chunks * a.N;
            const int n = a.chunks * a.N;
            for (int i = 0; i < n; i += 64) {
                const Candidate c = i + lane < n ? list[i + lane] : Candidate{0u, 0u};
                best.offer(c.value, c.index);
            }
        }
        best.prune();
        wave_sync();
        const double lse = (double)s.top + log(s.sum);
        if (!(fabs(lse) < (double)INFINITY)) continue;
        if (lane < best.count) {
            total[k * a.N + lane] = (double)score + ((double)descend(best.list[lane].value) - lse);
            flat[k * a.N + lane] = (uint32_t)k * a.V + best.list[lane].index;
        }
    }
    __syncthreads();
    for (int size = 2; size <= places; size *= 2)
        for (int step = size / 2; step > 0; step /= 2) {
            for (int i = tid; i < places / 2; i += blockDim.x) {
                const int one = 2 * i - (i & (step - 1)), two = one + step;
                const double x = total[one], y = total[two];
                const uint32_t p = flat[one], q = flat[two];
                const bool before = x > y || (x == y && p < q);            // one is the better
                if (before != ((one & size) == 0)) {
                    total[one] = y, total[two] = x;
                    flat[one] = q, flat[two] = p;
                }
            }
            __syncthreads();
        }
    for (int i = tid; i < a.N; i += blockDim.x) {
        const bool some = flat[i] != ~0u;
        const int k = some ? (int)(flat[i] / (uint32_t)a.V) : 0, token = some ? (int)(flat[i] - (uint32_t)k * a.V) : -1;
        const int64_t to = (int64_t)b * a.N + i;
        scores_out[to] = (float)total[i];
        parents[to] = some ? b * a.K + k : -1;
        tokens[to] = token;
        if (finished_out) finished_out[to] = !some || token == a.end_token || (finished && finished[(int64_t)b * a.K + k]);
    }
}

// Chunks of a row: a batch at least, and as many as it takes to have 4096 wavefronts
BeamArgs chunked(int64_t stride, int B, int K, int V, int N, int end_token)
{
    BeamArgs a{stride, B, K, V, N, end_token, 0, 0};
    const int64_t batches = ((int64_t)V + kBatch - 1) / kBatch, wanted = std::max<int64_t>(1, 4096 / ((int64_t)B * K));
    const int64_t each = (batches + wanted - 1) / wanted;
    a.chunk = each * kBatch;
    a.chunks = (int)((batches + each - 1) / each);
    return a;
}
size_t lists_bytes(const BeamArgs &a) { return ((size_t)a.B * a.K * a.chunks * a.N * sizeof(Candidate) + 15) & ~(size_t)15; }

} // namespace

size_t beam_select_workspace_bytes(int B, int K, int V, int N)
{
    if (V <= kDirect) return 0;
    const BeamArgs a = chunked(0, B, K, V, N, 0);
    return lists_bytes(a) + (size_t)B * K * a.chunks * sizeof(ChunkStats);
}

template <typename T>
hipError_t launch_beam_select(const T *logits, int64_t stride, const float *scores, const uint8_t *finished, int end_token, int B, int K, int V, int N, void *workspace,
                              float *scores_out, int32_t *parents, int32_t *tokens, uint8_t *finished_out, hipStream_t st)
{
    const BeamArgs a = chunked(stride, B, K, V, N, end_token);
    Candidate *const lists = static_cast<Candidate *>(workspace);
    ChunkStats *const stats = reinterpret_cast<ChunkStats *>(static_cast<char *>(workspace) + (V <= kDirect ? 0 : lists_bytes(a)));
    int places = 2;
    while (places < K * N) places *= 2;
    // (64 KB of LDS at most: 12 bytes a place, of 4096 at most, and 2 KB a wavefront)
    const int waves = std::min({K, 16, (65536 - 12 * places) / (int)(kCap * sizeof(Candidate))});
    const size_t lds = (size_t)places * 12 + (size_t)waves * kCap * sizeof(Candidate);
    if (V <= kDirect) {
        TimedLaunch tl(K_BEAM_SELECT, st);
        hipLaunchKernelGGL((beam_select_kernel<T, true>), dim3((unsigned)B), dim3(64 * waves), lds, st, a, logits, scores, finished, lists, stats, places, scores_out,
                           parents, tokens, finished_out);
        return hipGetLastError();
    }
    {
        TimedLaunch tl(K_BEAM_ROWS, st);
        hipLaunchKernelGGL((beam_rows_kernel<T>), dim3((unsigned)(((int64_t)B * K * a.chunks + 3) / 4)), dim3(256), 0, st, a, logits, finished, lists, stats);
    }
    TimedLaunch tl(K_BEAM_SELECT, st);
    hipLaunchKernelGGL((beam_select_kernel<T, false>), dim3((unsigned)B), dim3(64 * waves), lds, st, a, logits, scores, finished, lists, stats, places, scores_out, parents,
                       tokens, finished_out);
    return hipGetLastError();
}

template hipError_t launch_beam_select<bf16_t>(const bf16_t *, int64_t, const float *, const uint8_t *, int, int, int, int, int, void *, float *, int32_t *, int32_t *,
                                               uint8_t *, hipStream_t);
template hipError_t launch_beam_select<float>(const float *, int64_t, const float *, const uint8_t *, int, int, int, int, int, void *, float *, int32_t *, int32_t *,
                                              uint8_t *, hipStream_t);

} // namespace lss
