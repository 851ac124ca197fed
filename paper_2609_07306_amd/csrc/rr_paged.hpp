// The paged cache: where a token lies, and the argument blocks of the append
// and attention kernels (rr_append.hip, rr_paged.hip).
//
// Pools are [n_pages, H_kv, page, D]; sequence b's token u lies in page
// table[b][u / page] at place u % page.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rr {

// Quotients by the page length for 0 <= n < 2^31: with s the bits of
// page - 1 and mul = ceil(2^(31+s) / page), n / page = (n * mul) >> (31 + s):
// mul exceeds 2^(31+s) / page by less than 1, so the product's excess over
// the quotient is below n / 2^(31+s) <= 1 / page, and mul < 2^32.
struct PageDiv {
    uint32_t mul;
    int32_t shift;
    int32_t page;

    __host__ __device__ __forceinline__ int32_t div(int32_t n) const
    {
        return (int32_t)(((uint64_t)(uint32_t)n * mul) >> shift);
    }
};

inline PageDiv page_div(int32_t page)
{
    int s = 0;
    while (((int64_t)1 << s) < page) ++s;
    const uint64_t num = (uint64_t)1 << (31 + s);
    return PageDiv{(uint32_t)((num + (uint32_t)page - 1) / (uint32_t)page), 31 + s, page};
}

// A page number as the pools take it: -1 for one outside them.
__host__ __device__ __forceinline__ int32_t pool_page(int32_t id, int32_t n_pages)
{
    return (uint32_t)id < (uint32_t)n_pages ? id : -1;
}

// First element of row (page, key head g, place) of a pool.
__host__ __device__ __forceinline__ int64_t pool_row(int32_t phys, int32_t n_kv, int32_t g, int32_t page, int32_t place,
                                                     int32_t d)
{
    return (((int64_t)phys * n_kv + g) * page + place) * d;
}

// A sequence's length as the page table can hold it.
__host__ __device__ __forceinline__ int32_t held_tokens(int32_t length, int32_t capacity)
{
    return length < 0 ? 0 : (length < capacity ? length : capacity);
}

// Sequence of new token i: the largest b with start[b] <= i < start[b + 1],
// -1 past the last sequence's tokens.  start ascends; whatever it holds, the
// answer lies in [-1, n_seqs).
__host__ __device__ __forceinline__ int32_t sequence_of(const int32_t *start, int32_t n_seqs, int32_t i)
{
    int32_t lo = 0, hi = n_seqs;  // start[lo] <= i (or lo = 0), i < start[hi] (or hi = n_seqs)
    while (hi - lo > 1) {
        const int32_t mid = lo + (hi - lo) / 2;
        if (start[mid] <= i)
            lo = mid;
        else
            hi = mid;
    }
    return start[lo] <= i && i < start[lo + 1] ? lo : -1;
}

constexpr int kPagedUnit = 128;  // keys of a unit of the attention's work
constexpr int kPagedGrid = 512;  // workgroups of an attention launch: two a compute unit

enum CacheType : int32_t { CACHE_F32 = 0, CACHE_BF16 = 1, CACHE_E4M3 = 2 };

struct AppendArgs {
    const void *Q, *K, *V;  // [n_tokens, heads, d] with rows of ldq / ldk / ldv elements; Q or null
    void *Kc, *Vc;          // pools
    void *Q_out;            // [n_tokens, H, d]
    const int32_t *seq_start, *lengths, *table;
    const double *freqs;    // [rot / 2] radians per position
    const float *k_scale, *v_scale;
    int64_t ldq, ldk, ldv;
    int32_t n_heads, n_kv_heads, d, n_pages, max_pages, n_seqs, n_tokens, rot;
    int32_t per_seq;   // new tokens of each sequence where seq_start is null
    PageDiv pd;
};

struct PagedArgs {
    const void *Q;  // [B, n_q, H, D]
    const void *K, *V;
    void *O;
    float *lse;  // [B, n_q, H] or null
    const int32_t *table, *lengths, *routes, *prefix_pages;
    const float *k_scale, *v_scale;  // [H_kv] or null
    int32_t n_heads, n_kv_heads, group, n_pages, max_pages, n_seqs, n_q;
    int32_t capacity;             // tokens a page-table row can hold
    int32_t k, n_sink, n_recent;  // routes: slots, first and last pages
    int32_t n_prefix;             // tokens of the shared prefix (0: none)
    PageDiv pd;
    float scale;
    // schedule (paged_schedule)
    int32_t rows;           // query rows of a (sequence, key head): n_q * group; routes: 1
    int32_t own_tile, row_tiles;  // ... in tiles of so many
    int32_t items_per_seq;  // H_kv * row_tiles; routes: H * n_q
    int32_t route_units;    // routes: units of every item
    int32_t item_cost;      // units that stand for what an item of a sequence costs besides its keys
    int32_t prefix_rows, prefix_tile, prefix_tiles, prefix_items, prefix_units;  // of the batch against the prefix
    bool own_wide, prefix_wide;        // which body takes them
    bool two_weights;  // in the wide body a weight is two bf16 numbers
    int32_t prefix_splits, prefix_slots;  // of the wide body: key splits, (key head, split, row tile) slots
    int32_t grid;
    bool join_apart;     // without a prefix: the parts are joined by a second launch
    int32_t batch_keys;  // keys whose page numbers a workgroup holds at a time
    // workspace
    uint32_t *counters;  // [kPagedGrid] finished parts of the item that begins in a workgroup, 0 between calls
    float *parts;        // [2 * grid] parts of items that several workgroups share
    float *prefix_parts; // [prefix_slots] parts
    float *whole;        // with a prefix: [2][rows of the call] parts of items that one workgroup held
    int4 *heads;         // with a second launch: per item its first part, its first workgroup, its parts, 0
};

size_t paged_workspace_bytes(const PagedArgs &a, int d);
// Fills in the schedule of a call whose shape is set; cache: CacheType.  False
// where it may have more than 2^31 - 1 - kPagedGrid units of work.
bool paged_schedule(PagedArgs &a, int cache, int d);
// Lays the workspace out from its first byte.
void paged_layout(PagedArgs &a, int d, void *workspace);
bool paged_supported(int dtype, int cache, int d);
hipError_t launch_paged(const PagedArgs &a, int cache, int d, hipStream_t stream);
hipError_t launch_paged_join(const PagedArgs &a, int cache, int d, hipStream_t stream);
hipError_t launch_append(const AppendArgs &a, int dtype, int cache, bool interleaved, hipStream_t stream);

}  // namespace rr
