// Pages of a cache that are forked, copied, freed and moved together, for
// gfx950.  refs[p] counts the page-table entries that hold page p (and whatever
// else the caller counts there); a page with none is free.  Everything is
// integers: counts change by atomic additions, whose order does not matter, and
// pages are given out by rank (the lowest free ones, in the order of sequences
// and entries), so that results do not depend on which workgroup is first.
//
// The tables are small: what they cost is a chain of loads and the launches.
// Copies of pages are bound by the bytes, read once and written once.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "rr_internal.hpp"
#include "rr_pages.hpp"

namespace rr {
namespace {

// ------------------------------------------------------------------- fork

constexpr int kForkThreads = 256;
constexpr int kForkLds = 65536;  // bytes of parents, children and columns

// Row b becomes what row parent[b] was; no such row: empty.  A workgroup takes
// some columns of all rows, through LDS, so that rows change in place.  A row
// that k others become and that itself changes (m = 1) or not (0) adds k - m
// holders to each of its pages.
__global__ __launch_bounds__(kForkThreads) void fork_kernel(ForkArgs a)
{
    extern __shared__ int32_t lds[];
    int32_t *s_parent = lds, *s_kids = lds + a.n_seqs, *s_tile = lds + 2 * a.n_seqs;
    const int tid = threadIdx.x, C = a.columns;
    const int c0 = blockIdx.x * C;
    for (int b = tid; b < a.n_seqs; b += kForkThreads) s_kids[b] = 0;
    __syncthreads();
    for (int b = tid; b < a.n_seqs; b += kForkThreads) {
        int s = a.parent[b];
        if ((uint32_t)s >= (uint32_t)a.n_seqs) s = -1;
        s_parent[b] = s;
        if (s >= 0 && s != b) atomicAdd(s_kids + s, 1);
    }
    __syncthreads();
    for (int x = tid; x < a.n_seqs * C; x += kForkThreads) {
        const int b = x / C, c = c0 + x - b * C, more = s_kids[b] - (s_parent[b] != b);
        if (c >= a.max_pages || (s_kids[b] == 0 && s_parent[b] == b)) continue;
        const int e = a.table[(int64_t)b * a.max_pages + c];
        s_tile[x] = e;
        if (more && (uint32_t)e < (uint32_t)a.n_pages) atomicAdd(a.refs + e, more);
    }
    __syncthreads();
    for (int x = tid; x < a.n_seqs * C; x += kForkThreads) {
        const int b = x / C, k = x - b * C, c = c0 + k, s = s_parent[b];
        if (c >= a.max_pages || s == b) continue;
        a.table[(int64_t)b * a.max_pages + c] = s >= 0 ? s_tile[s * C + k] : -1;
    }
    if (blockIdx.x > 0) return;
    __syncthreads();
    for (int b = tid; b < a.n_seqs; b += kForkThreads) s_tile[b] = a.lengths[b];
    __syncthreads();
    for (int b = tid; b < a.n_seqs; b += kForkThreads)
        if (s_parent[b] != b) a.lengths[b] = s_parent[b] >= 0 ? s_tile[s_parent[b]] : 0;
}

// ----------------------------------------------------------------- resize

constexpr int kReleaseThreads = 256, kReleaseColumns = 1024;
constexpr int kBookThreads = 1024, kBookWaves = kBookThreads / 64;
constexpr int kScan = 4;  // blocks of four pages a thread that are looked at together

typedef int32_t i32x4_t __attribute__((ext_vector_type(4), aligned(4)));

// Entries past a sequence's last page let go of theirs.
__global__ __launch_bounds__(kReleaseThreads) void release_kernel(PagesArgs a)
{
    const int tiles = (a.max_pages + kReleaseColumns - 1) / kReleaseColumns;
    const int b = blockIdx.x / tiles, c0 = (blockIdx.x - b * tiles) * kReleaseColumns;
    const int length = held_tokens(a.lengths[b], a.capacity);
    const int end = a.pd.div(length + a.pd.page - 1);
#pragma unroll
    for (int k = 0; k < kReleaseColumns; k += kReleaseThreads) {
        const int c = c0 + k + threadIdx.x;
        if (c < end || c >= a.max_pages) continue;
        int32_t *entry = a.table + (int64_t)b * a.max_pages + c;
        const int e = pool_page(*entry, a.n_pages);
        if (e < 0) continue;
        atomicSub(a.refs + e, 1);
        *entry = -1;
    }
}

// Sums of x over the threads before this one, and over all of them.
template <typename T>
__device__ __forceinline__ T before_of(T x, T *s_wave, T *all)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    T to = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T y = __shfl_up(to, o, 64);
        if (lane >= o) to += y;
    }
    __syncthreads();
    if (lane == 63) s_wave[w] = to;
    __syncthreads();
    T base = 0, sum = 0;
#pragma unroll
    for (int i = 0; i < kBookWaves; ++i) {
        if (i < w) base += s_wave[i];
        sum += s_wave[i];
    }
    *all = sum;
    return base + to - x;
}

__device__ __forceinline__ void wait_vm() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// What other waves of this workgroup may have changed a moment ago.
__device__ __forceinline__ int32_t now(const int32_t *p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// refs of the four pages from p on (1 past the pools).
__device__ __forceinline__ i32x4_t four_refs(const PagesArgs &a, int p)
{
    if (p + 4 <= a.n_pages) return *reinterpret_cast<const i32x4_t *>(a.refs + p);
    i32x4_t r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = p + e < a.n_pages ? a.refs[p + e] : 1;
    return r;
}

// The entries of the newest tokens, a thread each, in the order of sequences
// and entries: those without a page get one, and those whose page others hold
// too get a copy of it.  One workgroup.
__global__ __launch_bounds__(kBookThreads) void provide_kernel(PagesArgs a)
{
    __shared__ int s_first[kBookThreads], s_begin[kBookThreads], s_to[kBookThreads + 1], s_missing[kBookThreads];
    __shared__ int s_page[kBookThreads], s_free[kBookThreads];
    __shared__ int s_wave[kBookWaves];
    __shared__ uint64_t s_wave64[kBookWaves];
    __shared__ int s_cursor, s_copies, s_stop;
    const int tid = threadIdx.x;
    if (tid == 0) s_cursor = s_copies = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += kBookThreads) {
        // the sequences' new entries
        const int b = b0 + tid;
        int first = 0, n = 0, begin = 0;
        if (b < a.n_seqs) {
            const int length = a.lengths[b], end = held_tokens(length, a.capacity);
            begin = max(0, length - max(0, a.new_tokens ? a.new_tokens[b] : a.n_new));
            if (begin < end) {
                first = a.pd.div(begin);
                n = a.pd.div(end - 1) + 1 - first;
            }
        }
        int items;
        const int at = before_of(n, s_wave, &items);
        s_first[tid] = first;
        s_begin[tid] = begin;
        s_to[tid] = at;
        s_missing[tid] = 0;
        if (tid == 0) s_to[kBookThreads] = items;
        __syncthreads();
        for (int i0 = 0; i0 < items; i0 += kBookThreads) {
            const int i = i0 + tid;
            const bool live = i < items;
            int q = 0, c = 0, e = -1, holders = 0;
            if (live) {
                // the last sequence that begins at or before item i
                int lo = 0, hi = kBookThreads;
                while (hi - lo > 1) {
                    const int mid = (lo + hi) / 2;
                    if (s_to[mid] <= i)
                        lo = mid;
                    else
                        hi = mid;
                }
                q = lo;
                c = s_first[q] + i - s_to[q];
                e = pool_page(now(a.table + (int64_t)(b0 + q) * a.max_pages + c), a.n_pages);
                if (e >= 0) holders = now(a.refs + e);
            }
            // A page that several hold is copied as long as that is so: each
            // item of this round before this one takes its own copy.
            const bool shared = holders > 1;
            int rank = 0;
            if (__syncthreads_or(shared)) {
                s_page[tid] = shared ? e : -1;
                __syncthreads();
                if (shared)
                    for (int j = 0; j < tid; ++j) rank += s_page[j] == e;
            }
            bool need = live && (e < 0 || holders - rank > 1);
            int wanted;
            const int order = before_of((int)need, s_wave, &wanted);
            // the lowest free pages
            int have = 0;
            for (int from = s_cursor; have < wanted && from < a.n_pages; from += 4 * kScan * kBookThreads) {
                i32x4_t r[kScan];
#pragma unroll
                for (int k = 0; k < kScan; ++k) r[k] = four_refs(a, min(from + 4 * (k * kBookThreads + tid), a.n_pages));
                uint64_t mine = 0, all;  // free pages of each block, 16 bits each
#pragma unroll
                for (int k = 0; k < kScan; ++k)
                    mine |= (uint64_t)((r[k][0] == 0) + (r[k][1] == 0) + (r[k][2] == 0) + (r[k][3] == 0)) << (16 * k);
                const uint64_t before = before_of(mine, s_wave64, &all);
#pragma unroll
                for (int k = 0; k < kScan; ++k) {
                    int at_free = have + (int)(before >> (16 * k) & 0xffff);
                    const int p = from + 4 * (k * kBookThreads + tid);
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        if (r[k][x] == 0) {
                            if (at_free < wanted) s_free[at_free] = p + x;
                            if (at_free == wanted - 1) s_cursor = p + x + 1;
                            ++at_free;
                        }
                    have += (int)(all >> (16 * k) & 0xffff);
                }
            }
            if (tid == 0) s_stop = kBookThreads;
            __syncthreads();
            if (have < wanted) {
                // not enough: who comes after the last page that is left sees
                // pages as shared as they then are
                if (need && order == have) s_stop = tid;
                if (tid == 0) s_cursor = a.n_pages;
                __syncthreads();
                if (shared && tid > s_stop) {
                    rank = 0;
                    for (int j = 0; j < s_stop; ++j) rank += s_page[j] == e;
                    need = holders - rank > 1;
                }
            }
            if (need && tid < s_stop) {
                const int id = s_free[order];
                a.table[(int64_t)(b0 + q) * a.max_pages + c] = id;
                a.refs[id] = 1;
                if (e >= 0) {
                    atomicSub(a.refs + e, 1);
                    const int places = min(a.pd.page, s_begin[q] - c * a.pd.page);
                    if (places > 0) a.copies[atomicAdd(&s_copies, 1)] = PageCopy{e, id, places};
                }
            } else if (need) {
                atomicAdd(s_missing + q, 1);
            }
            wait_vm();  // (the pages' counts, for the next round)
            __syncthreads();
        }
        __syncthreads();
        if (a.missing && b < a.n_seqs) a.missing[b] = s_missing[tid];
        __syncthreads();
    }
    if (tid == 0) *a.n_copies = s_copies;
}

// ---------------------------------------------------------------- compact

// The n used pages that lie past page n - 1 take the free ones before it, in
// order.  One workgroup: the pages are counted, then listed, then the counts
// of holders move.
__global__ __launch_bounds__(kBookThreads) void compact_kernel(PagesArgs a)
{
    __shared__ int s_wave[kBookWaves];
    __shared__ uint64_t s_wave64[kBookWaves];
    const int tid = threadIdx.x;
    int mine = 0, used;
    for (int p = 4 * tid; p < a.n_pages; p += 4 * kBookThreads) {
        const i32x4_t r = four_refs(a, p);
#pragma unroll
        for (int x = 0; x < 4; ++x) mine += p + x < a.n_pages && r[x] != 0;
    }
    before_of(mine, s_wave, &used);
    int low = 0, high = 0;  // free pages before page `used`, used ones from it on
    for (int p0 = 0; p0 < a.n_pages; p0 += 4 * kBookThreads) {
        const int p = p0 + 4 * tid;
        i32x4_t r = {0, 0, 0, 0};
        if (p < a.n_pages) r = four_refs(a, p);
        uint64_t n = 0, all;
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (p + x < a.n_pages) n += p + x < used ? (uint64_t)(r[x] == 0) : (uint64_t)(r[x] != 0) << 32;
        const uint64_t before = before_of(n, s_wave64, &all);
        int at_low = low + (int)(uint32_t)before, at_high = high + (int)(before >> 32);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if (p + x >= a.n_pages) continue;
            const bool is_used = r[x] != 0;
            if (p + x < used || !is_used) a.new_ids[p + x] = is_used ? p + x : -1;
            if (p + x < used && !is_used) a.copies[at_low++].dst = p + x;
            if (p + x >= used && is_used) {
                a.copies[at_high].src = p + x;
                a.copies[at_high++].places = a.pd.page;
            }
        }
        low += (int)(uint32_t)all;
        high += (int)(all >> 32);
    }
    wait_vm();
    __syncthreads();
    for (int k = tid; k < high; k += kBookThreads) {
        const int src = now(&a.copies[k].src), dst = now(&a.copies[k].dst);
        a.refs[dst] = a.refs[src];
        a.refs[src] = 0;
        a.new_ids[src] = dst;
    }
    if (tid == 0) {
        *a.n_copies = high;
        *a.n_used = used;
    }
}

__global__ __launch_bounds__(256) void rename_kernel(PagesArgs a)
{
    const int64_t n = (int64_t)a.n_seqs * a.max_pages;
    for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int e = pool_page(a.table[i], a.n_pages);
        if (e >= 0) a.table[i] = a.new_ids[e];
    }
}

// ------------------------------------------------------------------ copies

constexpr int kCopyThreads = 256, kCopyEach = 8;  // pieces of a thread's turn
constexpr int kCopyGroups = 2048;

// Pages of all pools, a piece of P bytes at a time: a unit is the same stretch
// of the pieces of one page in one pool.
template <typename P>
__global__ __launch_bounds__(kCopyThreads) void copies_kernel(PagesArgs a, Pools pools, int n_pools)
{
    const int n = *a.n_copies;
    const int row = a.row_bytes / (int)sizeof(P), whole = a.pd.page * row;  // pieces of a token of a head, of a page of a head
    constexpr int kStretch = kCopyThreads * kCopyEach;
    const int64_t stretches = ((int64_t)a.heads * whole + kStretch - 1) / kStretch;
    const int64_t units = (int64_t)n * n_pools * stretches;
    for (int64_t t = blockIdx.x; t < units; t += gridDim.x) {
        const int64_t pair = t / stretches, x0 = (t - pair * stretches) * kStretch;
        const int k = (int)(pair / n_pools), pool = (int)(pair - (int64_t)k * n_pools);
        const PageCopy c = a.copies[k];
        const int seg = c.places * row;  // pieces that move of a head
        const int64_t all = (int64_t)a.heads * seg;
        P *base = static_cast<P *>(pools.p[pool]);
        const P *src = base + (int64_t)c.src * a.heads * whole;
        P *dst = base + (int64_t)c.dst * a.heads * whole;
        P v[kCopyEach];
        int64_t at[kCopyEach];
#pragma unroll
        for (int j = 0; j < kCopyEach; ++j) {
            const int64_t x = x0 + j * kCopyThreads + threadIdx.x;
            at[j] = -1;
            if (x < all) {
                const int g = (int)((uint32_t)x / (uint32_t)seg);
                at[j] = (int64_t)g * whole + ((int)x - g * seg);
                v[j] = src[at[j]];
            }
        }
#pragma unroll
        for (int j = 0; j < kCopyEach; ++j)
            if (at[j] >= 0) dst[at[j]] = v[j];
    }
}

}  // namespace

int64_t release_groups(int32_t n_seqs, int32_t max_pages)
{
    return (int64_t)n_seqs * ((max_pages + kReleaseColumns - 1) / kReleaseColumns);
}

hipError_t launch_fork(const ForkArgs &args, hipStream_t stream)
{
    ForkArgs a = args;
    // as many columns as LDS holds, up to 8
    a.columns = 8;
    while (a.columns > 1 && a.n_seqs * (2 + a.columns) * (int)sizeof(int32_t) > kForkLds) a.columns /= 2;
    const unsigned lds = (unsigned)(a.n_seqs * (2 + a.columns) * sizeof(int32_t));
    hipLaunchKernelGGL(fork_kernel, dim3((unsigned)((a.max_pages + a.columns - 1) / a.columns)), dim3(kForkThreads), lds,
                       stream, a);
    return hipGetLastError();
}

hipError_t launch_resize(const PagesArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL(release_kernel, dim3((unsigned)release_groups(a.n_seqs, a.max_pages)), dim3(kReleaseThreads), 0, stream,
                       a);
    hipLaunchKernelGGL(provide_kernel, dim3(1), dim3(kBookThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_compact(const PagesArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL(compact_kernel, dim3(1), dim3(kBookThreads), 0, stream, a);
    const int64_t groups = ((int64_t)a.n_seqs * a.max_pages + 255) / 256;
    hipLaunchKernelGGL(rename_kernel, dim3((unsigned)(groups < 1024 ? groups : 1024)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_copies(const PagesArgs &a, const Pools &pools, int n_pools, hipStream_t stream)
{
    auto go = [&](auto piece) {
        typedef decltype(piece) P;
        hipLaunchKernelGGL(copies_kernel<P>, dim3(kCopyGroups), dim3(kCopyThreads), 0, stream, a, pools, n_pools);
    };
    // (rows of 8 features are 8 bytes in e4m3)
    a.row_bytes % 16 == 0 ? go(uint4()) : go(uint2());
    return hipGetLastError();
}

}  // namespace rr
