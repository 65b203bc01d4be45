// Pages of a cache from step to step: sequences that take on their parents' (lss_paged_fork), accepted ones of drafted tokens (lss_paged_compact).
//
// Fork.  Nothing is kept between calls but the table: a page is free if no sequence of the result names it and nobody else holds it.  So a word per page in
// scratch memory says who has it: -1 a reader (a sequence that has all of it, or has no room in it, or another holder), else the lowest sequence that will write
// into it.  Marks commute, so the order in which they arrive does not matter.  A sequence whose partly filled page is not its own by that takes a new one and the
// tokens in it.  New pages are the lowest free numbers, in the order of (sequence, page).
//   What bounds it is latency: four launches, each of which needs all that the one before wrote.  384 sequences of 48 prompts of 300 to 6000 tokens, 21.5 MB copied (8 heads of 128): 21.9 us, the
// marks' array cleared in 1.3 to 2.1, tables 6.1, plan 6.3, copies 7.0 to 7.5 (3 TB/s).  Few sequences, pages and entries take one workgroup and LDS for the first three: four beams 7.7 us, by all four
// launches 15.5.
#include "lss_serve.h"

#include <algorithm>
#include <climits>

namespace lss {

namespace {

constexpr int kNobody = INT_MAX, kReader = -1, kPlanThreads = 1024, kPerThread = 16;
constexpr int kSmallSequences = 256, kSmallPages = 4096, kSmallEntries = 16384;        // what one workgroup goes over at once

// what sequence s of the result has from its parent, and what it will need
struct Heir {
    int parent, length, full, part, room, table_pages;
    int64_t wanted;         // pages
};
__device__ __forceinline__ Heir heir_of(const ForkArgs &a, int s)
{
    Heir h;
    const int p = a.parents[s], page = 1 << a.pt.page_shift;
    const bool some = (uint32_t)p < (uint32_t)a.B;
    h.parent = some ? p : -1;
    h.length = some ? max(0, min(a.lengths[p], a.pt.max_pages << a.pt.page_shift)) : 0;
    h.room = a.room ? max(a.room[s], 0) : some ? 1 : 0;
    h.full = h.length >> a.pt.page_shift;
    h.part = h.length & (page - 1);
    h.wanted = ((int64_t)h.length + h.room + page - 1) >> a.pt.page_shift;
    h.table_pages = (int)min(h.wanted, (int64_t)a.pt.max_pages);
    return h;
}
__device__ __forceinline__ int pages_before(const Heir &h) { return h.full + (h.part > 0); }
__device__ __forceinline__ int page_at(const ForkArgs &a, int parent, int nth)        // -1: none
{
    const int page = a.pt.table[(int64_t)parent * a.pt.max_pages + nth];
    return (uint32_t)page < (uint32_t)a.pt.n_pages ? page : -1;
}

// What a sequence does to its partly filled page: the page if it is to write into it, else -1; and the pages that it takes besides one to move out of that into
struct alignas(16) Wish {
    int tail, taken;
    int past;               // pages that its table has no entry for (2^31 tokens are 2^27 pages)
    int part, before;       // tokens in its partly filled page; pages that it has from its parent
};
__device__ __forceinline__ Wish wish_of(const ForkArgs &a, const Heir &h)
{
    const int tail = h.part > 0 && h.room > 0 ? page_at(a, h.parent, h.full) : -1;
    return {tail, max(0, h.table_pages - pages_before(h)), (int)(h.wanted - h.table_pages), h.part, pages_before(h)};
}

__global__ __launch_bounds__(256) void fork_clear_kernel(ForkArgs a, int32_t *__restrict__ owner)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < a.pt.n_pages) owner[i] = a.held && a.held[i] ? kReader : kNobody;
}

// The entries of sequence blockIdx.x's table, 256 at a time
__global__ __launch_bounds__(256) void fork_table_kernel(ForkArgs a, int32_t *__restrict__ owner, Wish *__restrict__ wishes, int32_t *__restrict__ table_out,
                                                         int32_t *__restrict__ lengths_out)
{
    const int s = blockIdx.x;
    int nth = blockIdx.y * 256 + threadIdx.x;
    // (an entry is on its way with the length that says whether it counts)
    const int p = a.parents[s];
    int entry = nth < a.pt.max_pages && (uint32_t)p < (uint32_t)a.B ? page_at(a, p, nth) : -1;
    const Heir h = heir_of(a, s);
    while (nth < a.pt.max_pages) {
        const int page = nth < pages_before(h) ? entry : -1;
        if (page >= 0) {
            if (nth == h.full && h.room > 0) atomicMin(owner + page, s);
            else __hip_atomic_store(owner + page, kReader, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        table_out[(int64_t)s * a.pt.max_pages + nth] = page;
        nth += gridDim.y * 256;
        entry = nth < min(pages_before(h), a.pt.max_pages) ? page_at(a, h.parent, nth) : -1;
    }
    if (blockIdx.y == 0 && threadIdx.x == 0) {
        lengths_out[s] = (int)min((int64_t)h.length + h.room, (int64_t)a.pt.max_pages << a.pt.page_shift);
        wishes[s] = wish_of(a, h);
    }
}

// inclusive sums over a workgroup of kPlanThreads, and of all
__device__ __forceinline__ int64_t group_scan(int64_t x, int64_t *waves, int64_t &all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    x = lanes_upto(x);
    __syncthreads();
    if (lane == 63) waves[wave] = x;
    __syncthreads();
    int64_t before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        if (w < wave) before += waves[w];
        all += waves[w];
    }
    return x + before;
}

// By one workgroup: of each sequence its first page in the list of the lowest free ones, ~ where it moves out of its partly filled one; that list, as long as is taken.
// wish(s), owner(page): of sequence s, of a page
template <typename WishOf, typename OwnerOf>
__device__ __forceinline__ void plan(const ForkArgs &a, int64_t *waves, WishOf &&wish, OwnerOf &&owner, int32_t *first, int32_t *free_pages, int32_t *n_free, int32_t *missing)
{
    const int tid = threadIdx.x;
    int64_t need = 0, past = 0, all;
    int of_page[kPerThread];                            // the first kPlanThreads * kPerThread pages', on their way while the sequences are gone over
    const auto load = [&](int p) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) of_page[i] = owner(min(p + i, a.pt.n_pages - 1));
    };
    load(tid * kPerThread);
    for (int s0 = 0; s0 < a.B_out; s0 += kPlanThreads) {
        const int s = s0 + tid;
        Wish w{-1, 0, 0, 0, 0};
        if (s < a.B_out) w = wish(s);
        const bool moves = w.tail >= 0 && owner(w.tail) != s;
        const int64_t mine = (int64_t)moves + w.taken, upto = group_scan(mine, waves, all);
        // (a place in the list of free pages past its end is as good as any other)
        const int at = (int)min(need + upto - mine, (int64_t)a.pt.n_pages);
        if (s < a.B_out) first[s] = moves ? ~at : at;
        need += all;
        past += w.past;
    }
    group_scan(past, waves, past);
    const int wanted = (int)min(need, (int64_t)a.pt.n_pages);
    int found = 0;
    for (int p0 = 0; p0 < a.pt.n_pages && found < wanted; p0 += kPlanThreads * kPerThread) {
        const int p = p0 + tid * kPerThread;
        uint32_t mine = 0;
        if (p0 > 0) load(p);
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) mine |= (uint32_t)(p + i < a.pt.n_pages && of_page[i] == kNobody) << i;
        int at = found + (int)group_scan(__popc(mine), waves, all) - __popc(mine);
        for (; mine != 0 && at < wanted; mine &= mine - 1, ++at) free_pages[at] = p + __ffs(mine) - 1;
        found += (int)all;
    }
    found = min(found, wanted);
    if (tid == 0) {
        *n_free = found;
        *missing = (int)min(need - found + past, (int64_t)INT_MAX);
    }
}

__global__ __launch_bounds__(kPlanThreads) void fork_plan_kernel(ForkArgs a, const int32_t *__restrict__ owner, const Wish *__restrict__ wishes, int32_t *__restrict__ first,
                                                                 int32_t *__restrict__ free_pages, int32_t *__restrict__ n_free, int32_t *__restrict__ missing)
{
    __shared__ int64_t waves[kPlanThreads / 64];
    plan(a, waves, [&](int s) { return wishes[s]; }, [&](int page) { return owner[page]; }, first, free_pages, n_free, missing);
}

// Few sequences, short tables and few pages: the three launches above by one workgroup, who has what in LDS
__global__ __launch_bounds__(kPlanThreads) void fork_small_kernel(ForkArgs a, Wish *__restrict__ wishes, int32_t *__restrict__ first, int32_t *__restrict__ free_pages, int32_t *__restrict__ n_free,
                                                                  int32_t *__restrict__ missing, int32_t *__restrict__ table_out, int32_t *__restrict__ lengths_out)
{
    __shared__ int64_t waves[kPlanThreads / 64];
    __shared__ int owner[kSmallPages];
    __shared__ Heir heirs[kSmallSequences];
    const int tid = threadIdx.x;
    Heir mine{};
    Wish w{-1, 0, 0, 0, 0};
    if (tid < a.B_out) mine = heir_of(a, tid);
    for (int i = tid; i < a.pt.n_pages; i += kPlanThreads) owner[i] = a.held && a.held[i] ? kReader : kNobody;
    if (tid < a.B_out) {
        heirs[tid] = mine;
        wishes[tid] = w = wish_of(a, mine);
        lengths_out[tid] = (int)min((int64_t)mine.length + mine.room, (int64_t)a.pt.max_pages << a.pt.page_shift);
    }
    __syncthreads();
    const int entries = a.B_out * a.pt.max_pages;
#pragma unroll 4
    for (int i = tid; i < entries; i += kPlanThreads) {
        const int s = i / a.pt.max_pages, nth = i - s * a.pt.max_pages;
        const Heir &h = heirs[s];
        const int page = nth < pages_before(h) ? page_at(a, h.parent, nth) : -1;
        if (page >= 0) atomicMin(owner + page, nth == h.full && h.room > 0 ? s : kReader);
        table_out[i] = page;
    }
    __syncthreads();
    plan(a, waves, [&](int) { return w; }, [&](int page) { return owner[page]; }, first, free_pages, n_free, missing);
}

// Sequence blockIdx.x: its new pages into its table (blockIdx.y = 0), what its partly filled page holds into a new one (all of them)
template <typename Vec>
__global__ __launch_bounds__(256) void fork_copy_kernel(ForkArgs a, const Wish *__restrict__ wishes, const int32_t *__restrict__ first,
                                                        const int32_t *__restrict__ free_pages, const int32_t *__restrict__ n_free, int row_vecs,
                                                        Vec *__restrict__ k_cache, Vec *__restrict__ v_cache, int32_t *__restrict__ table_out)
{
    const int s = blockIdx.x, found = *n_free, of_list = first[s];
    const Wish w = wishes[s];
    const bool moves = of_list < 0;
    const int at = moves ? ~of_list : of_list, begin = w.before - moves, n = moves + w.taken;
    if (blockIdx.y == 0)
        for (int i = threadIdx.x; i < n; i += 256)
            table_out[(int64_t)s * a.pt.max_pages + begin + i] = at + i < found ? free_pages[at + i] : -1;
    if (!moves || at >= found) return;
    const int64_t from = ((int64_t)w.tail << a.pt.page_shift) * row_vecs, to = ((int64_t)free_pages[at] << a.pt.page_shift) * row_vecs;
    const int64_t vecs = (int64_t)w.part * row_vecs;
    for (int64_t i = blockIdx.y * 256 + threadIdx.x; i < vecs; i += gridDim.y * 256) {
        k_cache[to + i] = k_cache[from + i];
        v_cache[to + i] = v_cache[from + i];
    }
}

__device__ __forceinline__ int64_t of_lane(int64_t x, int lane)       // wavefront-uniform, whichever lanes are active
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)x, lane) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32);
}

// Compact.  What bounds it is latency: 192 sequences, 1 to 12 of 16 to 64 drafted tokens of 8 heads of 128 kept, 9.3 MB: 7.8 us; one sequence 4.3.  Sequence blockIdx.x, 16-byte columns blockIdx.y * 256 + (thread) of a row of both caches; kept rows 64 at a time, a lane each for the way to them, then
// eight at a time from memory to registers and back.  Kept numbers ascend, so that a row is never overwritten before it has been read: row i comes from i or later.
template <typename Vec>
__global__ __launch_bounds__(256) void paged_compact_kernel(CompactArgs a, int row_vecs, Vec *__restrict__ k_cache, Vec *__restrict__ v_cache,
                                                            int32_t *__restrict__ lengths_out)
{
    constexpr int AHEAD = 8;
    const int b = blockIdx.x, lane = threadIdx.x & 63, column = blockIdx.y * 256 + threadIdx.x;
    const int n = max(0, a.cu[b + 1] - a.cu[b]), length = max(0, min(a.lengths[b], a.pt.max_pages << a.pt.page_shift));
    const int m = max(0, min(a.n_kept[b], min(a.max_kept, n))), base = length - n;
    if (blockIdx.y == 0 && threadIdx.x == 0) lengths_out[b] = max(0, base + m);
    Vec *const cache = column < row_vecs ? k_cache : v_cache;
    const int mine = column < row_vecs ? column : column - row_vecs;
    for (int i0 = 0; i0 < m; i0 += 64) {
        int64_t from = -1, to = -1;
        if (i0 + lane < m) {
            const int at = a.kept[(int64_t)b * a.max_kept + i0 + lane];
            if (at > i0 + lane && at < n) {              // (where it is already, or not a number of such a list: nothing moves)
                from = cache_row(a.pt, b, base + at);
                to = cache_row(a.pt, b, base + i0 + lane);
            }
        }
        const uint64_t moved = __ballot(from >= 0 && to >= 0);
        if (moved == 0) continue;
        for (int i = 0; i < 64; i += AHEAD) {
            if ((moved >> i & ((1u << AHEAD) - 1)) == 0) continue;
            Vec x[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
                if (moved >> (i + j) & 1) {
                    const Vec *const row = cache + of_lane(from, i + j) * row_vecs;
                    if (column < 2 * row_vecs) x[j] = row[mine];
                }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
                if (moved >> (i + j) & 1) {
                    Vec *const row = cache + of_lane(to, i + j) * row_vecs;
                    if (column < 2 * row_vecs) row[mine] = x[j];
                }
        }
    }
}

} // namespace

size_t paged_fork_workspace_bytes(int64_t n_pages, int64_t B_out) { return sizeof(Wish) * (size_t)B_out + sizeof(int32_t) * (size_t)(2 * n_pages + B_out + 4); }

hipError_t launch_paged_fork(const ForkArgs &a, int row_bytes, void *k_cache, void *v_cache, int32_t *scratch, int32_t *table_out, int32_t *lengths_out, int32_t *missing,
                             hipStream_t st)
{
    // (a launch has fewer than 2^32 threads)
    const auto shared = [&](int64_t workgroups) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(workgroups, ((int64_t)1 << 22) / std::max(a.B_out, 1))); };
    Wish *const wishes = reinterpret_cast<Wish *>(scratch);
    int32_t *const owner = reinterpret_cast<int32_t *>(wishes + a.B_out), *const free_pages = owner + a.pt.n_pages, *const first = free_pages + a.pt.n_pages, *const n_free = first + a.B_out;
    if (a.B_out <= kSmallSequences && a.pt.n_pages <= kSmallPages && (int64_t)a.B_out * a.pt.max_pages <= kSmallEntries) {
        TimedLaunch tl(K_FORK_SMALL, st);
        hipLaunchKernelGGL(fork_small_kernel, dim3(1), dim3(kPlanThreads), 0, st, a, wishes, first, free_pages, n_free, missing, table_out, lengths_out);
    } else {
        {
            TimedLaunch tl(K_FORK_CLEAR, st);
            hipLaunchKernelGGL(fork_clear_kernel, dim3((unsigned)((a.pt.n_pages + 255ll) / 256)), dim3(256), 0, st, a, owner);
        }
        if (a.B_out > 0) {
            TimedLaunch tl(K_FORK_TABLE, st);
            hipLaunchKernelGGL(fork_table_kernel, dim3((unsigned)a.B_out, shared((a.pt.max_pages + 255) / 256)), dim3(256), 0, st, a, owner, wishes, table_out, lengths_out);
        }
        TimedLaunch tl(K_FORK_PLAN, st);
        hipLaunchKernelGGL(fork_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, a, owner, wishes, first, free_pages, n_free, missing);
    }
    if (a.B_out > 0) {
        const int64_t bytes = 2 * ((int64_t)row_bytes << a.pt.page_shift);
        TimedLaunch tl(K_FORK_COPY, st);
        hipLaunchKernelGGL(fork_copy_kernel<f32x4>, dim3((unsigned)a.B_out, shared(std::min<int64_t>(64, bytes / 32768))), dim3(256), 0, st, a, wishes,
                           first, free_pages, n_free, row_bytes / 16, static_cast<f32x4 *>(k_cache), static_cast<f32x4 *>(v_cache), table_out);
    }
    return hipGetLastError();
}

hipError_t launch_paged_compact(const CompactArgs &a, int row_bytes, void *k_cache, void *v_cache, int32_t *lengths_out, hipStream_t st)
{
    TimedLaunch tl(K_PAGED_COMPACT, st);
    hipLaunchKernelGGL(paged_compact_kernel<f32x4>, dim3((unsigned)a.B, (unsigned)((2 * (row_bytes / 16) + 255) / 256)), dim3(256), 0, st, a, row_bytes / 16,
                       static_cast<f32x4 *>(k_cache), static_cast<f32x4 *>(v_cache), lengths_out);
    return hipGetLastError();
}

} // namespace lss
