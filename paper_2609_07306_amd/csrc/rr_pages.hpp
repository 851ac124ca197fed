// Arguments of the calls that change which pages sequences hold (rr_pages.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "rr_paged.hpp"

namespace rr {

constexpr int kForkSeqs = 4096;    // sequences of a fork: a workgroup holds a column of all of them in LDS
constexpr int kPoolsAtOnce = 64;   // pools that a launch copies pages of

struct ForkArgs {
    const int32_t *parent;
    int32_t *table, *lengths, *refs;
    int32_t n_seqs, max_pages, n_pages;
};

// A page's first `places` places go from page src to page dst.
struct PageCopy {
    int32_t src, dst, places;
};

struct PagesArgs {
    const int32_t *lengths, *new_tokens;  // new_tokens: [n_seqs], or null: n_new
    int32_t *table, *refs;
    int32_t *missing;           // [n_seqs] or null
    int32_t *new_ids, *n_used;  // compaction: [n_pages], [1]
    int32_t n_seqs, max_pages, n_pages, n_new;
    int32_t capacity;  // tokens a page-table row can hold
    int32_t heads;     // of a page
    int32_t row_bytes; // of a token of a head
    PageDiv pd;
    PageDiv row;  // quotients by max_pages
    uint32_t *counter;  // workspace: finished workgroups, 0 between calls;
    int32_t *n_copies;  // copies to make ...
    PageCopy *copies;   // ... [n_pages]
    int32_t *spans;     // compaction of more than a round of pages: used ones of each round,
    int32_t *rank;      // which of the pages that move a used page past the others is; else null
};

constexpr int kRoundPages = 16384;  // pages that a workgroup counts at once

// The workspace holds the counter and the number of copies, the copies, and
// numbers of rounds.  No more than half of the pages move: the ranks take the
// copies' second half.
constexpr size_t kPagesHeadBytes = 256;
inline size_t pages_workspace_bytes(int32_t n_pages)
{
    return kPagesHeadBytes + (size_t)n_pages * sizeof(PageCopy) + ((size_t)n_pages / kRoundPages + 1) * sizeof(int32_t);
}

inline void pages_layout(PagesArgs &a, void *workspace)
{
    a.counter = static_cast<uint32_t *>(workspace);
    a.n_copies = static_cast<int32_t *>(workspace) + 1;
    a.copies = reinterpret_cast<PageCopy *>(static_cast<char *>(workspace) + kPagesHeadBytes);
    a.spans = reinterpret_cast<int32_t *>(a.copies + a.n_pages);
    a.rank = a.n_pages > kRoundPages ? reinterpret_cast<int32_t *>(a.copies + (a.n_pages + 1) / 2) : nullptr;
}

struct Pools {
    void *p[kPoolsAtOnce];
};

hipError_t launch_fork(const ForkArgs &a, hipStream_t stream);
hipError_t launch_resize(const PagesArgs &a, hipStream_t stream);   // the tables; copies to make
hipError_t launch_compact(const PagesArgs &a, hipStream_t stream);  // the same
hipError_t launch_copies(const PagesArgs &a, void *const *list, int n, bool compacted, hipStream_t stream);  // in n pools

}  // namespace rr
