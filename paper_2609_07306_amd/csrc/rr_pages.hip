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

#include "rr_device.hpp"
#include "rr_internal.hpp"
#include "rr_pages.hpp"

namespace rr {
namespace {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------- fork

constexpr int kForkThreads = 512, kForkAtOnce = 4;
constexpr int kForkLds = 65536;  // bytes of parents, children and columns
static_assert(kForkSeqs * (2 + 2) * sizeof(int32_t) <= kForkLds, "two columns of any call");

// Row b becomes what row parent[b] was; no such row: empty.  A workgroup takes
// C columns of all rows, through LDS, so that rows change in place.  A row that
// k others become and that itself changes (m = 1) or not (0) adds k - m holders
// to each of its pages.
//
// Bound by those additions where many rows change: sequences that hold the same
// page mostly follow each other, so neighbouring rows' are summed in a wave
// before one of them adds (beams of 512 sequences, in groups of 8 that share all
// but the last page of up to 1000: 12.2 -> 9.2 us), and
// neighbouring columns, which share lines of memory, are one XCD's (-> 5.1).
template <int C>
__global__ __launch_bounds__(kForkThreads) void fork_kernel(ForkArgs a)
{
    extern __shared__ int32_t lds[];
    int32_t *s_parent = lds, *s_kids = lds + a.n_seqs, *s_tile = lds + 2 * a.n_seqs;
    // (workgroups are dealt to the eight XCDs in turn)
    const int tid = threadIdx.x, n = a.n_seqs * C, c0 = ((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3)) * C;
    if (c0 >= a.max_pages) return;
    for (int b = tid; b < a.n_seqs; b += kForkThreads) s_kids[b] = 0;
    __syncthreads();
    for (int b = tid; b < a.n_seqs; b += kForkThreads) {
        int s = a.parent[b];
        if ((uint32_t)s >= (uint32_t)a.n_seqs) s = -1;
        s_parent[b] = s;
        if (s >= 0 && s != b) atomicAdd(s_kids + s, 1);
    }
    __syncthreads();
    const int lane = tid & 63;
    uint64_t column = 0;  // lanes of this one's column
#pragma unroll
    for (int l = 0; l < 64; l += C) column |= (uint64_t)1 << l;
    column <<= lane % C;
    // (entries that wait for nothing but themselves: some at a time)
    for (int x0 = tid; x0 - tid < n; x0 += kForkAtOnce * kForkThreads) {
        int e[kForkAtOnce], more[kForkAtOnce];
#pragma unroll
        for (int j = 0; j < kForkAtOnce; ++j) {
            const int x = x0 + j * kForkThreads, b = x / C, c = c0 + x % C;
            more[j] = 0;
            e[j] = -1;
            if (x >= n || c >= a.max_pages) continue;
            const int kids = s_kids[b];
            const bool stays = s_parent[b] == b;
            more[j] = kids - !stays;
            if (kids || !stays) e[j] = a.table[(int64_t)b * a.max_pages + c];
        }
#pragma unroll
        for (int j = 0; j < kForkAtOnce; ++j) {
            if (x0 + j * kForkThreads < n) s_tile[x0 + j * kForkThreads] = e[j];
            // runs of rows with the same page, numbered; the sum of each, in its first row
            const int above = __shfl_up(e[j], C, 64);
            const bool first = lane < C || above != e[j] || e[j] < 0;
            const int run = __popcll(__ballot(first) & column & (~(uint64_t)0 >> (63 - lane)));
            int sum = more[j];
            if (__ballot(!first)) {
#pragma unroll
                for (int step = C; step < 64; step *= 2) {
                    const int other = __shfl_down(run, step, 64), y = __shfl_down(sum, step, 64);
                    if (lane + step < 64 && other == run) sum += y;
                }
            }
            if (first && sum && (uint32_t)e[j] < (uint32_t)a.n_pages) atomicAdd(a.refs + e[j], sum);
        }
    }
    __syncthreads();
    for (int x = tid; x < n; x += kForkThreads) {
        const int b = x / C, c = c0 + x % C, s = s_parent[b];
        if (c < a.max_pages && s != b) a.table[(int64_t)b * a.max_pages + c] = s >= 0 ? s_tile[s * C + x % C] : -1;
    }
    if (blockIdx.x > 0) return;
    __syncthreads();
    for (int b = tid; b < a.n_seqs; b += kForkThreads) s_tile[b] = a.lengths[b];
    __syncthreads();
    for (int b = tid; b < a.n_seqs; b += kForkThreads)
        if (s_parent[b] != b) a.lengths[b] = s_parent[b] >= 0 ? s_tile[s_parent[b]] : 0;
}

// ------------------------------------------------- sums over a workgroup

constexpr int kBookThreads = 1024, kBookWaves = kBookThreads / 64;
constexpr int kDeviceScope = 16;  // sc1 of a buffer instruction

typedef int32_t i32x4_t __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ void wait_vm() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// What other waves may have changed a moment ago.
__device__ __forceinline__ int32_t now(const int32_t *p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int x)
{
    return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, true);
}

// Sums over lanes 0 .. this one of its row of 16, and of the wave.
__device__ __forceinline__ int row_up_to(int x)
{
    x += moved<0x111, 0xf>(x);  // from 1, 2, 4 and 8 lanes before
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    return x + moved<0x118, 0xf>(x);
}

__device__ __forceinline__ int wave_up_to(int x)
{
    x = row_up_to(x);
    x += moved<0x142, 0xa>(x);         // row 0 to row 1, row 2 to row 3
    return x + moved<0x143, 0xc>(x);   // the first two rows to the others
}

// Sums over the waves before this one of what each one has (`mine`, in its lane
// 63), and over all of them, in one barrier; s_wave is one of two that calls
// take in turn.  One workgroup's time goes into instructions (its 16 waves share
// four SIMDs: 16 cycles each), so sums are few and by data-parallel moves.
__device__ __forceinline__ int waves_before(int mine, int *s_wave, int *all)
{
    static_assert(kBookWaves == 16, "a row of lanes");
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (lane == 63) s_wave[w] = mine;
    __syncthreads();
    const int to = row_up_to(s_wave[lane & 15]);
    *all = __builtin_amdgcn_readlane(to, 15);
    return w ? __builtin_amdgcn_readlane(to, w - 1) : 0;
}

// Sums of x over the threads before this one, and over all of them.
__device__ __forceinline__ int before_of(int x, int *s_wave, int *all)
{
    const int to = wave_up_to(x);
    return waves_before(to, s_wave, all) + to - x;
}

// The largest x of the threads up to this one (x >= 0).
__device__ __forceinline__ int up_to_last(int x, int *s_wave)
{
    auto row = [](int x) {
        x = max(x, moved<0x111, 0xf>(x));
        x = max(x, moved<0x112, 0xf>(x));
        x = max(x, moved<0x114, 0xf>(x));
        return max(x, moved<0x118, 0xf>(x));
    };
    x = row(x);
    x = max(x, moved<0x142, 0xa>(x));
    x = max(x, moved<0x143, 0xc>(x));
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (lane == 63) s_wave[w] = x;
    __syncthreads();
    const int to = row(s_wave[lane & 15]);
    return w ? max(x, __builtin_amdgcn_readlane(to, w - 1)) : x;
}

// A round's pages: kScan times 256 of each wave, four a lane, wave after wave.
constexpr int kScan = 4, kWavePages = kScan * 256;
static_assert(kRoundPages == kBookWaves * kWavePages, "a round of pages");

// ----------------------------------------------------------------- resize

constexpr int kEntriesEach = 4;  // of the table, a thread of a resize

constexpr int kFreeHeld = 4096;    // free pages that are found ahead
constexpr int kSlots = 2 * kBookThreads;  // of the table of shared pages

// Entries past a sequence's last page let go of theirs, all workgroups; then
// the one that comes last goes through the entries of the newest tokens, a
// thread each, in the order of sequences and entries: those without a page get
// one, and those whose page others hold too get a copy of it.
//
// Bound by the chain of a round of 1024 entries (count, table, holders, free
// pages, each a load and a sum over the workgroup): 8.0 us for a decode step's 64
// sequences, 9.2 for 128 just forked, 45 for prompts of 16800 pages.
__global__ __launch_bounds__(kBookThreads) void resize_kernel(PagesArgs a)
{
    __shared__ int s_first[kBookThreads], s_begin[kBookThreads], s_to[kBookThreads], s_missing[kBookThreads];
    __shared__ int s_mark[kBookThreads];
    __shared__ int s_page[kSlots], s_times[kSlots], s_last[kSlots];  // shared pages of a round, by a hash
    __shared__ int s_free[kFreeHeld];                                // a ring
    __shared__ int s_wave[2][kBookWaves];
    __shared__ int s_cursor, s_copies, s_stop, s_any;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // The new entries of sequences b0 .. b0 + 1023, one after the other: how many.
    int own_at = 0, own_n = 0;  // of this thread's sequence
    auto lay_out = [&](int b0) {
        const int b = b0 + tid;
        int first = 0, n = 0, begin = 0, items;
        if (b < a.n_seqs) {
            const int length = a.lengths[b], end = held_tokens(length, a.capacity);
            begin = max(0, length - max(0, a.new_tokens ? a.new_tokens[b] : a.n_new));
            if (begin < end) {
                first = a.pd.div(begin);
                n = a.pd.div(end - 1) + 1 - first;
            }
        }
        own_n = n;
        s_to[tid] = own_at = before_of(n, s_wave[1], &items);
        s_first[tid] = first;
        s_begin[tid] = begin;
        s_missing[tid] = 0;
        __syncthreads();
        return items;
    };
    // Entries i0 .. i0 + 1023 of them, one a thread: its sequence (less b0), its
    // entry, and the page there.  A sequence marks where it begins; the last mark
    // up to a thread is its sequence.  (A search of ten steps takes longer.)
    struct Item {
        int q, c, e;
    };
    auto look_up = [&](int b0, int i0, int items) {
        s_mark[tid] = 0;
        __syncthreads();
        if (own_n && own_at < i0 + kBookThreads && own_at + own_n > i0) s_mark[max(own_at - i0, 0)] = tid + 1;
        __syncthreads();
        const int mark = up_to_last(s_mark[tid], s_wave[0]), i = i0 + tid;
        Item it{0, 0, -1};
        if (i < items) {
            it.q = mark - 1;
            it.c = s_first[it.q] + i - s_to[it.q];
            it.e = pool_page(a.table[(int64_t)(b0 + it.q) * a.max_pages + it.c], a.n_pages);
        }
        return it;
    };

#pragma unroll
    for (int j = 0; j < kEntriesEach; ++j) {
        const uint32_t x = (blockIdx.x * kEntriesEach + j) * kBookThreads + tid;  // (a table has less than 2^30 entries)
        if (x >= (uint32_t)(a.n_seqs * a.max_pages)) continue;
        const int b = a.row.div((int)x), c = (int)x - b * a.max_pages;
        const int e = pool_page(a.table[x], a.n_pages);
        const int end = a.pd.div(held_tokens(a.lengths[b], a.capacity) + a.pd.page - 1);
        if (c < end || e < 0) continue;
        atomicSub(a.refs + e, 1);
        a.table[x] = -1;
    }
    // (Any workgroup may be the last, so each prepares the first round while its
    // changes are on their way: entries of new tokens are not among them.  Where
    // they do not all run at once, only the last does.)
    const bool early = gridDim.x <= 256;
    int items = 0;
    Item it{0, 0, -1};
    if (early) {
        items = lay_out(0);
        it = look_up(0, 0, items);
    }
    wait_vm();        // this wave's changes are there for all ...
    __syncthreads();  // ... and the other waves'
    if (tid == 0) {
        s_stop = 1;
        if (gridDim.x > 1) {
            const uint32_t before = __hip_atomic_fetch_add(a.counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_stop = before == gridDim.x - 1;
            if (s_stop) __hip_atomic_store(a.counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        s_cursor = s_copies = 0;
        s_any = 0;
    }
    __syncthreads();
    if (!s_stop) return;

    // A round of counts, from page `from` on.  The first is asked for now: between
    // here and its use no count falls to 0, and none leaves 0 unseen.
    const __amdgpu_buffer_rsrc_t refs =
        __builtin_amdgcn_make_buffer_rsrc(a.refs, 0, a.n_pages * (int)sizeof(int32_t), 0x00020000);
    i32x4_t r[kScan];
    auto ask = [&](int from) {
        const int p0 = from + wave * kWavePages;
        if (p0 >= a.n_pages) return;
#pragma unroll
        for (int k = 0; k < kScan; ++k)
            r[k] = __builtin_bit_cast(i32x4_t, __builtin_amdgcn_raw_buffer_load_b128(refs, 4 * (p0 + 4 * lane + 256 * k), 0,
                                                                                    kDeviceScope));
    };
    ask(0);
    int round = 0, head = 0, held = 0, cursor = 0;  // (head, held) of s_free; pages before `cursor` have been looked at
    for (int b0 = 0; b0 < a.n_seqs; b0 += kBookThreads) {
        if (b0 || !early) {
            items = lay_out(b0);
            it = look_up(b0, 0, items);
        }
        for (int i0 = 0; i0 < items; i0 += kBookThreads) {
            const int i = i0 + tid, q = it.q, c = it.c, e = it.e, holders = e >= 0 ? now(a.refs + e) : 0;
            if (i0 + kBookThreads < items) it = look_up(b0, i0 + kBookThreads, items);  // (asked for a round ahead)
            // A page that several hold is copied as long as that is so: by each of
            // this round's, but for the last one where no one else holds it.
            const bool shared = holders > 1;
            ++round;
            if (shared) s_any = round;
            __syncthreads();
            const bool any_shared = s_any == round;
            int slot = 0;
            bool keeps = true;
            if (any_shared) {
                for (int x = tid; x < kSlots; x += kBookThreads) {
                    s_page[x] = s_last[x] = -1;
                    s_times[x] = 0;
                }
                __syncthreads();
                if (shared) {
                    slot = (int)((uint32_t)e * 2654435761u >> 21);
                    for (int was; (was = atomicCAS(s_page + slot, -1, e)) != -1 && was != e;) slot = (slot + 1) % kSlots;
                    atomicAdd(s_times + slot, 1);
                    atomicMax(s_last + slot, tid);
                }
                __syncthreads();
                keeps = !shared || (s_last[slot] == tid && s_times[slot] >= holders);
            }
            bool need = i < items && (e < 0 || !keeps);
            int wanted;
            const int order = before_of((int)need, s_wave[1], &wanted);
            // the lowest free pages, as many ahead as the ring takes
            while (held < wanted && cursor < a.n_pages) {
                const int p0 = cursor + wave * kWavePages + 4 * lane, room = kFreeHeld - held;
                int free = 0, at[kScan];
                if (cursor) ask(cursor);
                if (p0 - 4 * lane < a.n_pages) {
#pragma unroll
                    for (int k = 0; k < kScan; ++k) {
                        int mine = 0;
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            if (p0 + 256 * k + x >= a.n_pages) r[k][x] = 1;  // (past the pools zeros are read)
                            mine += r[k][x] == 0;
                        }
                        const int to = wave_up_to(mine);
                        at[k] = free + to - mine;
                        free += __builtin_amdgcn_readlane(to, 63);
                    }
                }
                int all;
                const int before = waves_before(free, s_wave[0], &all);  // (others may still read s_wave[1])
                if (free) {
#pragma unroll
                    for (int k = 0; k < kScan; ++k) {
                        int to = before + at[k];
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            if (r[k][x] == 0) {
                                if (to < room) s_free[(head + held + to) % kFreeHeld] = p0 + 256 * k + x;
                                if (to == room - 1) s_cursor = p0 + 256 * k + x + 1;
                                ++to;
                            }
                    }
                }
                __syncthreads();
                cursor = all < room ? cursor + kRoundPages : s_cursor;
                held += min(all, room);
            }
            if (tid == 0) s_stop = kBookThreads;
            __syncthreads();
            const int have = min(held, wanted);
            if (have < wanted) {
                // Not enough: who comes after the last page that is left sees pages
                // as shared as they then are.
                if (need && order == have) s_stop = tid;
                if (shared) s_times[slot] = 0;
                __syncthreads();
                if (shared && tid < s_stop) atomicAdd(s_times + slot, 1);
                __syncthreads();
                if (shared && tid > s_stop) need = holders - s_times[slot] > 1;
            }
            if (need && tid < s_stop) {
                const int id = s_free[(head + order) % kFreeHeld];
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
            head = (head + have) % kFreeHeld;
            held -= have;
            if (any_shared) wait_vm();  // (their holders, for the next round)
            __syncthreads();
        }
        if (a.missing && b0 + tid < a.n_seqs) a.missing[b0 + tid] = s_missing[tid];
        __syncthreads();
    }
    if (tid == 0) *a.n_copies = s_copies;
}

// ---------------------------------------------------------------- compact

// refs of the four pages from p on, as far as there are any.
__device__ __forceinline__ i32x4_t four_refs(const PagesArgs &a, int p)
{
    if (p + 4 <= a.n_pages) return *reinterpret_cast<const i32x4_t *>(a.refs + p);
    i32x4_t r = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (p + e < a.n_pages) r[e] = a.refs[p + e];
    return r;
}

// A thread's pages of a round from page `from` on, and sums over them in the
// order of pages: of the wave's before the thread's first page of each block, and
// of the wave's.
struct Round {
    i32x4_t r[kScan];
    int p0, before[kScan], sum;
    bool any;  // the wave has pages

    __device__ __forceinline__ void load(const PagesArgs &a, int from)
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        p0 = from + wave * kWavePages + 4 * lane;
        any = p0 - 4 * lane < a.n_pages;
        if (any) {
#pragma unroll
            for (int k = 0; k < kScan; ++k) r[k] = four_refs(a, min(p0 + 256 * k, a.n_pages));
        }
    }

    template <typename F>
    __device__ __forceinline__ void add_up(F value)
    {
        sum = 0;
        if (!any) return;
#pragma unroll
        for (int k = 0; k < kScan; ++k) {
            int n = 0;
#pragma unroll
            for (int x = 0; x < 4; ++x) n += value(p0 + 256 * k + x, r[k][x]);
            const int to = wave_up_to(n);
            before[k] = sum + to - n;
            sum += __builtin_amdgcn_readlane(to, 63);
        }
    }

    // Writes down where pages go: low free ones from index `low` on (the waves
    // before counted), high used ones from `high` on; both 16 bits of `before`.
    __device__ __forceinline__ void list(const PagesArgs &a, int used, int low, int high, int32_t *rank) const
    {
        if (!any) return;
#pragma unroll
        for (int k = 0; k < kScan; ++k) {
            int at_low = low + (before[k] & 0xffff), at_high = high + (before[k] >> 16);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int p = p0 + 256 * k + x;
                if (p >= a.n_pages) continue;
                const bool is_used = r[k][x] != 0;
                if (p < used || !is_used) a.new_ids[p] = is_used ? p : -1;
                if (p < used && !is_used) a.copies[at_low++].dst = p;
                if (p >= used && rank) rank[p] = is_used ? at_high : -1;
                if (p >= used && is_used) {
                    a.copies[at_high].src = p;
                    a.copies[at_high++].places = a.pd.page;
                }
            }
        }
    }
};

// The holders of a page that moves, and its new name.
__device__ __forceinline__ void settle(const PagesArgs &a, int src, int dst)
{
    a.refs[dst] = a.refs[src];
    a.refs[src] = 0;
    a.new_ids[src] = dst;
}

// The n used pages that lie past page n - 1 take the free ones before it, in
// order: a round of pages, by one workgroup, which counts them, lists them and
// moves the counts of holders.
__global__ __launch_bounds__(kBookThreads) void compact_kernel(PagesArgs a)
{
    __shared__ int s_wave[2][kBookWaves];
    const int tid = threadIdx.x;
    Round t;
    t.load(a, 0);
    int used, all;
    t.add_up([](int, int r) { return (int)(r != 0); });
    waves_before(t.sum, s_wave[0], &used);
    t.add_up([&](int p, int r) { return p < used ? (int)(r == 0) : (int)(r != 0) << 16; });
    const int before = waves_before(t.sum, s_wave[1], &all);
    t.list(a, used, before & 0xffff, before >> 16, nullptr);
    const int moves = all >> 16;
    wait_vm();
    __syncthreads();
    for (int k = tid; k < moves; k += kBookThreads) settle(a, now(&a.copies[k].src), now(&a.copies[k].dst));
    if (tid == 0) {
        *a.n_copies = moves;
        *a.n_used = used;
    }
}

// The same for more pages, a round by each workgroup, in three launches: used
// pages are counted; listed; and settled beside the copies.  (100000 pages, half
// of them used: one workgroup 70 us, these 20
// before the copies.)
__global__ __launch_bounds__(kBookThreads) void count_kernel(PagesArgs a)
{
    __shared__ int s_wave[kBookWaves];
    Round t;
    t.load(a, blockIdx.x * kRoundPages);
    t.add_up([](int, int r) { return (int)(r != 0); });
    int all;
    waves_before(t.sum, s_wave, &all);
    if (threadIdx.x == 0) a.spans[blockIdx.x] = all;
}

__global__ __launch_bounds__(kBookThreads) void list_kernel(PagesArgs a)
{
    __shared__ int s_wave[2][kBookWaves];
    const int tid = threadIdx.x, n = gridDim.x, own = blockIdx.x, from = own * kRoundPages;
    // used pages in all rounds, and in those before this one
    int mine = 0, mine_before = 0, used, used_before, low_used, below;
    for (int i = tid; i < n; i += kBookThreads) {
        const int x = a.spans[i];
        mine += x;
        if (i < own) mine_before += x;
    }
    before_of(mine, s_wave[0], &used);
    before_of(mine_before, s_wave[1], &used_before);
    // used pages below page `used`: in the rounds before its own, and in that one
    const int middle = used / kRoundPages;
    mine = 0;
    for (int i = tid; i < middle; i += kBookThreads) mine += a.spans[i];
    before_of(mine, s_wave[0], &below);
    Round t;
    t.load(a, middle * kRoundPages);
    t.add_up([&](int p, int r) { return (int)(r != 0 && p < used); });
    waves_before(t.sum, s_wave[1], &low_used);
    low_used += below;
    t.load(a, from);
    t.add_up([&](int p, int r) { return p < used ? (int)(r == 0) : (int)(r != 0) << 16; });
    int all;
    const int before = waves_before(t.sum, s_wave[0], &all);
    // free pages below `used` in rounds before this one, and used ones from it on
    const int low = min(from, used) - min(used_before, low_used), high = max(used_before - low_used, 0);
    t.list(a, used, low + (before & 0xffff), high + (before >> 16), a.rank);
    if (own == 0 && tid == 0) {
        *a.n_copies = used - low_used;
        *a.n_used = used;
    }
}

// ------------------------------------------------------------------ copies

constexpr int kCopyThreads = 256;

// How pages are copied.  Compaction reads every page once and leaves little to
// other calls, so both ways go past the caches, and workgroups are many: 600
// pages of 128 KB in four pools (629 MB) in 111 us, 5.6 TB/s (116 in a trace); four
// pieces a thread and 8192 workgroups 117, with stores alone past the caches 120,
// none 125.  Copies of a page that several sequences share read it again, from the
// caches; most calls have none to make, and fewer workgroups are sooner through
// (an empty launch of 4096 takes 2.3 us, of 8192 3.9): half a page of 16 pools,
// three times each for 32 groups (31 MB read, 92 written), in 23.5 us, 5.2 TB/s;
// with stores through the caches 30, and the attention that follows is no faster
// (eight layers 828 us, 837 so).  Units of a page are an odd number
// (kOdd): where a page is copied in part, the units of its end have nothing to do,
// and an even number would leave them to the same XCDs page after page (four
// units 27.7 us).  Small pages take fewer pieces a thread, which need no more
// registers than leave five waves (2 KB in 8 pools: 4.5 us, eight pieces 7.5).
struct Moved {
    static constexpr int kEach = 2, kEachSmall = 2, kGroups = 16384;  // pieces of a thread's turn
    static constexpr bool kOnce = true;
    static constexpr uint32_t kOdd = 0;
};
struct Shared {
    static constexpr int kEach = 8, kEachSmall = 4, kGroups = 4096;
    static constexpr bool kOnce = false;
    static constexpr uint32_t kOdd = 1;
};

// Pages of all pools, a piece (a vector P) at a time.  A unit of a workgroup's
// work is a stretch of the pieces of one page in one pool, or (SMALL) as many
// pages as it has room for.  units < 2^31.
//
// Before that, after a compaction (in the first of its launches), the entries
// of the table take their pages' new names.
template <typename P, bool SMALL, typename How>
__global__ __launch_bounds__(kCopyThreads) void copies_kernel(PagesArgs a, Pools pools, uint32_t n_pools, int64_t n_entries)
{
    if constexpr (How::kOnce) {
        const int32_t all = gridDim.x * kCopyThreads, first = blockIdx.x * kCopyThreads + threadIdx.x;
        const int used = *a.n_used;
        for (int64_t i = first; i < n_entries; i += all) {
            const int e = pool_page(a.table[i], a.n_pages);
            if (e < 0) continue;
            const int k = a.rank && e >= used ? a.rank[e] : -1;
            a.table[i] = k >= 0 ? a.copies[k].dst : a.rank && e >= used ? -1 : a.new_ids[e];
        }
        if (a.rank && n_entries)
            for (int k = first; k < *a.n_copies; k += all) settle(a, a.copies[k].src, a.copies[k].dst);
    }
    constexpr int kEach = SMALL ? How::kEachSmall : How::kEach, kCopyUnit = kEach * kCopyThreads;
    const uint32_t pairs = (uint32_t)*a.n_copies * n_pools;
    const uint32_t row = a.row_bytes / sizeof(P), head = a.pd.page * row;  // pieces of a token of a head, of a head's page
    const uint32_t page = a.heads * head;
    const uint32_t each = SMALL ? kCopyUnit / page : (page + kCopyUnit - 1) / kCopyUnit | How::kOdd;  // pages a unit; units a page
    const uint32_t units = SMALL ? (pairs + each - 1) / each : pairs * each;
    for (uint32_t t = blockIdx.x; t < units; t += gridDim.x) {
        P v[kEach], *to[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            uint32_t x = j * kCopyThreads + threadIdx.x, pair;
            if (SMALL) {
                pair = t * each + x / page;
                x %= page;
            } else {
                pair = t / each;
                x += (t - pair * each) * kCopyUnit;
            }
            to[j] = nullptr;
            if (SMALL && (pair >= pairs || pair >= (t + 1) * each)) continue;
            const uint32_t k = pair / n_pools;
            const PageCopy c = a.copies[k];
            const uint32_t part = c.places * row;  // pieces that move of a head
            if (x >= a.heads * part) continue;
            const uint32_t at = part == head ? x : x / part * head + x % part;
            P *base = static_cast<P *>(pools.p[pair - k * n_pools]);
            const P *from = base + (int64_t)c.src * page + at;
            v[j] = How::kOnce ? __builtin_nontemporal_load(from) : *from;
            to[j] = base + (int64_t)c.dst * page + at;
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (to[j]) __builtin_nontemporal_store(v[j], to[j]);
    }
}

}  // namespace

hipError_t launch_fork(const ForkArgs &a, hipStream_t stream)
{
    auto lds = [&](int columns) { return a.n_seqs * (2 + columns) * (int)sizeof(int32_t); };
    auto go = [&](auto kern, int columns) {
        const int groups = (a.max_pages + columns - 1) / columns;
        hipLaunchKernelGGL(kern, dim3((unsigned)((groups + 7) / 8 * 8)), dim3(kForkThreads), (unsigned)lds(columns), stream, a);
    };
    // as many columns as LDS holds, up to 8, and to 4 where that leaves compute units idle
    if (lds(8) <= kForkLds && a.max_pages >= 8 * 256)
        go(fork_kernel<8>, 8);
    else if (lds(4) <= kForkLds)
        go(fork_kernel<4>, 4);
    else
        go(fork_kernel<2>, 2);
    return hipGetLastError();
}

hipError_t launch_resize(const PagesArgs &a, hipStream_t stream)
{
    constexpr int kEntries = kEntriesEach * kBookThreads;
    const int64_t groups = ((int64_t)a.n_seqs * a.max_pages + kEntries - 1) / kEntries;
    hipLaunchKernelGGL(resize_kernel, dim3((unsigned)groups), dim3(kBookThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_compact(const PagesArgs &a, hipStream_t stream)
{
    if (a.n_pages <= kRoundPages) {
        hipLaunchKernelGGL(compact_kernel, dim3(1), dim3(kBookThreads), 0, stream, a);
        return hipGetLastError();
    }
    const int rounds = (a.n_pages + kRoundPages - 1) / kRoundPages;
    hipLaunchKernelGGL(count_kernel, dim3((unsigned)rounds), dim3(kBookThreads), 0, stream, a);
    hipLaunchKernelGGL(list_kernel, dim3((unsigned)rounds), dim3(kBookThreads), 0, stream, a);
    return hipGetLastError();
}

template <typename How>
hipError_t copy_pages(const PagesArgs &a, void *const *list, int n, int64_t most_copies, hipStream_t stream)
{
    // (rows of 8 features are 8 bytes in e4m3)
    const int piece = a.row_bytes % 16 == 0 ? 16 : 8;
    const int64_t page = (int64_t)a.heads * a.pd.page * (a.row_bytes / piece);
    const bool small = page <= How::kEachSmall * kCopyThreads / 2;
    const int unit = (small ? How::kEachSmall : How::kEach) * kCopyThreads;
    const int64_t each = small ? unit / page : (page + unit - 1) / unit | How::kOdd;  // as in the kernel
    const int64_t most = (int64_t)INT32_MAX / (a.n_pages * (small ? 1 : each));
    const int at_once = (int)(most < 1 ? 1 : most < kPoolsAtOnce ? most : kPoolsAtOnce);
    for (int i0 = 0; i0 < n; i0 += at_once) {
        const int some = n - i0 < at_once ? n - i0 : at_once;
        Pools pools{};
        for (int i = 0; i < some; ++i) pools.p[i] = list[i0 + i];
        const int64_t units = small ? most_copies * some / each + 1 : most_copies * some * each;
        const int64_t entries = How::kOnce && i0 == 0 ? (int64_t)a.n_seqs * a.max_pages : 0, turns = entries / kCopyThreads + 1;
        const int64_t wanted = units > turns ? units : turns;
        const int groups = (int)(wanted < How::kGroups ? wanted : How::kGroups);
        auto go = [&](auto kern) {
            hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(kCopyThreads), 0, stream, a, pools, (uint32_t)some, entries);
        };
        if (piece == 16)
            small ? go(copies_kernel<u32x4_t, true, How>) : go(copies_kernel<u32x4_t, false, How>);
        else
            small ? go(copies_kernel<u32x2_t, true, How>) : go(copies_kernel<u32x2_t, false, How>);
    }
    return hipGetLastError();
}

hipError_t launch_copies(const PagesArgs &a, void *const *list, int n, bool compacted, hipStream_t stream)
{
    if (compacted) return copy_pages<Moved>(a, list, n, a.n_pages / 2, stream);
    const int64_t entries = a.new_tokens ? a.max_pages : (int64_t)a.n_new / a.pd.page + 2;
    const int64_t most = a.n_seqs * (entries < a.max_pages ? entries : a.max_pages);
    return copy_pages<Shared>(a, list, n, most < a.n_pages ? most : a.n_pages, stream);
}

}  // namespace rr
