// The paged attention's schedule and launches, and the join of the parts that
// its workgroups leave (the attention itself is in rr_paged_impl.hpp).
#include <type_traits>

#include "rr_paged_impl.hpp"

namespace rr {
namespace {

using paged::add_part;
using paged::f32x4_t;
using paged::inverse_sum;
using paged::log_sum;

constexpr int kT = 256;  // threads of a joining workgroup
constexpr int kAtOnce = 4;  // parts of a thread in flight

// -------------------------------------------------------------------- join
//
// Where a call takes a second launch: a query row's parts -- of its own item,
// and of the prefix item that holds it -- are added with weights 2^(m_i - m), by
// a workgroup or (ROWS = 4) a wave of one.  Bound by the parts, which it reads
// once (2048 rows of 33 parts, 36 MB: 4.5 TB/s), with four parts of a thread
// asked for before the first is used (the whole call 56.9 us, without 58.5, as
// long with eight).

template <int D, bool F32, int ROWS>
__global__ __launch_bounds__(kT) void paged_join_kernel(PagedArgs a)
{
    constexpr int PL = D / 4;          // lanes of a part, four features each
    constexpr int T = kT / ROWS;       // threads of a row
    constexpr int NP = T / PL;         // its parts in flight
    __shared__ float s_m[ROWS][NP], s_l[ROWS][NP];
    __shared__ float s_acc[ROWS][NP][D];
    const int tid = threadIdx.x % T, w = threadIdx.x / T;
    const int64_t n_rows = (int64_t)a.n_seqs * a.n_q * a.n_heads;
    const int64_t orow = min((int64_t)blockIdx.x * ROWS + w, n_rows - 1);  // (b, t, h)
    bool live = (int64_t)blockIdx.x * ROWS + w < n_rows;
    const int h = (int)(orow % a.n_heads);
    const int64_t bt = orow / a.n_heads;
    const int t = (int)(bt % a.n_q), b = (int)(bt / a.n_q);
    const int g = h / a.group, j = h - g * a.group;

    const int r = t * a.group + j, own_row = r % a.own_tile;  // row within its item's tile
    const int4 own = a.heads[a.prefix_items + (int64_t)b * a.items_per_seq + g * a.row_tiles + r / a.own_tile];
    int4 pre = {0, 0, 0, 0};
    const float *pre_part = nullptr;  // of a wide prefix: its splits lie a.prefix_tiles slots apart
    const int q = b * a.rows + t * a.group + j, x_tile = q / a.prefix_tile, pre_row = q - x_tile * a.prefix_tile;
    if (a.prefix_items == 0) {
        live = live && own.z != 1;  // (else its workgroup wrote the output itself)
    } else if (a.prefix_wide) {
        pre.z = a.prefix_splits;
        const int slot = g * a.prefix_splits * a.prefix_tiles + x_tile;
        pre_part = a.prefix_parts + ((int64_t)slot * a.prefix_tile + pre_row) * (D + 4);
    } else {
        pre = a.heads[g * a.prefix_tiles + x_tile];
    }
    const int n_own = own.z, n = live ? n_own + pre.z : 0;
    auto part_of = [&](int i) -> const float * {
        const bool p = i >= n_own;
        const int4 &hd = p ? pre : own;
        i = p ? i - n_own : i;
        if (p && pre_part) return pre_part + (int64_t)i * a.prefix_tiles * a.prefix_tile * (D + 4);
        if (hd.z == 1) return a.whole + ((p ? 0 : n_rows) + orow) * (D + 4);
        const int64_t slot = i == 0 ? hd.x : 2 * (int64_t)(hd.y + i);
        return a.parts + (slot * a.own_tile + (p ? pre_row : own_row)) * (D + 4);
    };
    // PL lanes a part, NP parts at once, kept with a running maximum like the
    // attention's own: sums and statistics are asked for together
    const int pl = tid % PL, pg = tid / PL;
    f32x4_t x = {0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    for (int i0 = pg; i0 < n; i0 += kAtOnce * NP) {
        f32x4_t y[kAtOnce];
        float mi[kAtOnce], li[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const float *p = part_of(min(i0 + k * NP, n - 1));
            y[k] = *reinterpret_cast<const f32x4_t *>(p + 4 * pl);
            mi[k] = p[D];
            li[k] = p[D + 1];
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (i0 + k * NP < n) add_part(y[k], mi[k], li[k], x, m, l);
    }
    *reinterpret_cast<f32x4_t *>(&s_acc[w][pg][4 * pl]) = x;
    if (pl == 0) {
        s_m[w][pg] = m;
        s_l[w][pg] = l;
    }
    __syncthreads();
    if (!live) return;
    m = -INFINITY;
    l = 0.f;
    float wt[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) m = fmaxf(m, s_m[w][i]);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        wt[i] = s_m[w][i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[w][i] - m);
        l += wt[i] * s_l[w][i];
    }
    const float inv = inverse_sum(l, a.v_scale ? a.v_scale[g] : 1.f);
    for (int f = tid; f < D; f += T) {
        float y = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) y = __builtin_fmaf(wt[i], s_acc[w][i][f], y);
        y *= inv;
        if constexpr (F32)
            static_cast<float *>(a.O)[orow * D + f] = y;
        else
            static_cast<__bf16 *>(a.O)[orow * D + f] = (__bf16)y;
    }
    if (tid == 0 && a.lse) a.lse[orow] = log_sum(m, l);
}

}  // namespace

bool paged_supported(int dtype, int cache, int d)
{
    if (dtype == 0) return cache == CACHE_F32 && (d == 64 || d == 128);
    return (cache == CACHE_BF16 || cache == CACHE_E4M3) && (d == 64 || d == 128 || d == 256);
}

bool paged_schedule(PagedArgs &a, int cache, int d)
{
    const int per_b = a.n_q * a.group;
    const bool routed = a.k + a.n_sink + a.n_recent > 0, f32 = cache == CACHE_F32;
    a.rows = routed ? 1 : per_b;
    a.prefix_rows = a.n_prefix ? a.n_seqs * per_b : 0;
    // more than 16 rows go to the wide body; binary32 has the narrow one alone,
    // with tiles of 32 rows (such tiles for bf16 too, of which a compute unit
    // holds one workgroup: 32 rows on 8192 tokens 23.4 us against 25.4, but on 8
    // times 32768 in an 8-bit cache 164 against 129)
    a.own_wide = !f32 && a.rows > 16;
    a.prefix_wide = !f32 && a.prefix_rows > 16;
    // (of a narrow prefix and the sequences behind it the tiles are alike)
    const int narrow = f32 && (a.rows > 16 || a.prefix_rows > 16) ? 32 : 16;
    const auto tile = [&](bool wide, int rows) { return !wide ? narrow : rows <= 32 ? 32 : rows <= 64 ? 64 : 128; };
    a.own_tile = tile(a.own_wide, a.rows);
    a.prefix_tile = tile(a.prefix_wide, a.prefix_rows);
    // Rounded to one bf16 number, a weight is 2^-8 off, as much as the output; as
    // two, 2^-16.  Where tiles hold up to 64 rows the reads of keys take the time
    // and the second product costs little: 8192 tokens, 32 and 64 rows 24.1 and
    // 27.0 us with one, 25.0 and 28.1 with two; 32 sequences of 1000 to 4000, 64
    // rows 84.0 and 85.6; 64 of 100 to 1000, 32 rows 43.7 and 47.0; six behind
    // 2000 tokens 14.2 and 14.8.  With more the products do: 8192 tokens, 128 rows
    // 44.2 and 49.0; 2048 new ones behind 6144 305 and 384; 1280 rows on 32768
    // tokens 241 and 302
    a.two_weights = (a.prefix_rows ? a.prefix_rows : a.rows) <= 64;
    a.row_tiles = 1 + (a.rows - 1) / a.own_tile;  // (there may be 2^31 - 1 rows)
    a.items_per_seq = routed ? a.n_heads * a.n_q : a.n_kv_heads * a.row_tiles;
    // (kernels of 32-row narrow tiles and of 256 features take a compute unit
    // for one workgroup)
    const int most_wg = d == 256 || narrow == 32 ? kPagedGrid / 2 : kPagedGrid;
    // Without a prefix the workgroup that finishes an item's last part joins
    // its parts alone, row after row; a second launch has all of the card for
    // it, but costs some 3 us and a little more with the rows of the batch.  It
    // is taken where an item may have that many rows of parts (they count by
    // their features).  32 heads on 8, d = 128, one launch and two:
    //   1 sequence of 8192 tokens, 4 rows: 15.6 and 17.9 us; 16 rows: 21.4 and
    //   19.0; 128 rows: 86 and 34; 8 sequences of 1000 to 8000, 32 rows: 58.7
    //   and 42; 32 of 1000 to 4000, 64 rows: 93 and 81 (both with a weight in one
    //   number, two add 1.5 us); 1 of 2048, all of them new: 83 and 99
    // (So a call that takes two has less than 2^25 rows.)
    const int64_t items = (int64_t)a.n_seqs * a.items_per_seq;
    const int64_t parts = (items <= kPagedGrid / 8 ? kPagedGrid / 2 : most_wg) / items + 1;  // (as the runs are cut, find_run)
    a.join_apart = a.n_prefix == 0 && !routed && parts * (a.rows < a.own_tile ? a.rows : a.own_tile) * d / 128 >=
                                          (a.own_wide ? 80 : 140) + (int64_t)a.n_seqs * a.n_q * a.n_heads / 256;
    a.route_units = 0;
    if (routed) {
        const int64_t slots = (int64_t)a.k + a.n_sink + a.n_recent;
        const int64_t pages = slots < a.max_pages ? slots : a.max_pages;
        a.route_units = (int32_t)((pages * a.pd.page + kPagedUnit - 1) / kPagedUnit);
    }
    a.prefix_tiles = (a.prefix_rows + a.prefix_tile - 1) / a.prefix_tile;
    a.prefix_items = a.n_kv_heads * a.prefix_tiles;
    a.prefix_units = (a.n_prefix + kPagedUnit - 1) / kPagedUnit;
    const int64_t keys = (int64_t)(paged::kStagedPages - 1) * a.pd.page / kPagedUnit * kPagedUnit;
    a.batch_keys = (int32_t)(keys < (1 << 30) ? keys : (1 << 30));
    // an item's rows, page numbers and result take about as long as 128 keys: it
    // counts where workgroups take several items, whose lengths may differ (160
    // sequences of 64 to 2048 tokens: 110 us without, 92 with; behind a prefix of
    // 32768 tokens in runs, 4 of 1 to 400: 40.7 and 37.1)
    const bool several = (int64_t)a.items_per_seq * a.n_seqs >= kPagedGrid || (a.n_prefix && !a.prefix_wide);
    a.item_cost = !routed && several ? 1 : 0;
    // units of the longest sequences that the page table can hold
    const double longest = routed ? a.route_units : (a.capacity + kPagedUnit - 1) / kPagedUnit + a.item_cost;
    const double most_own = longest * a.items_per_seq * a.n_seqs;
    const double most = most_own + (double)a.prefix_items * a.prefix_units;
    // (rounded up to the grid's runs they still have to be a 32-bit number)
    if (most > (double)(INT32_MAX - kPagedGrid)) return false;
    // splits of a wide prefix: the fewest that leave at most a tenth more of
    // the card idle than the best number does
    a.prefix_splits = a.prefix_slots = 0;
    if (a.prefix_wide) {
        const auto used = [&](int splits) {
            const int64_t n = (int64_t)a.prefix_items * splits, rounds = (n + most_wg - 1) / most_wg;
            return (double)n / ((double)rounds * most_wg);
        };
        const int most_splits = a.prefix_units < most_wg ? a.prefix_units : most_wg;
        double best = 0.;
        for (int n = 1; n <= most_splits; ++n) best = used(n) > best ? used(n) : best;
        a.prefix_splits = 1;
        while (used(a.prefix_splits) < 0.9 * best) ++a.prefix_splits;
        a.prefix_slots = a.prefix_items * a.prefix_splits;
    }
    const double need = a.prefix_wide ? (most_own > a.prefix_slots ? most_own : a.prefix_slots) : most;
    a.grid = need < most_wg ? (int32_t)need : most_wg;
    return true;
}

static int64_t align256(int64_t n) { return (n + 255) / 256 * 256; }

static int64_t parts_bytes(const PagedArgs &a, int d)
{
    return align256((int64_t)2 * a.grid * a.own_tile * (d + 4) * 4);
}

static int64_t prefix_bytes(const PagedArgs &a, int d) { return align256((int64_t)a.prefix_slots * a.prefix_tile * (d + 4) * 4); }

static int64_t whole_bytes(const PagedArgs &a, int d)
{
    return a.n_prefix ? align256((int64_t)2 * a.n_seqs * a.n_q * a.n_heads * (d + 4) * 4) : 0;
}

// The counters come first, at the same place for calls of every shape, which
// may follow each other in one workspace; heads serve calls that take a second
// launch, whole parts those with a prefix.
constexpr int64_t kCounterBytes = (int64_t)kPagedGrid * sizeof(uint32_t);

static int64_t heads_bytes(const PagedArgs &a)
{
    const int64_t items = a.prefix_items + (int64_t)a.n_seqs * a.items_per_seq;
    return a.n_prefix || a.join_apart ? align256(items * (int64_t)sizeof(int4)) : 0;
}

size_t paged_workspace_bytes(const PagedArgs &a, int d)
{
    return (size_t)(kCounterBytes + parts_bytes(a, d) + prefix_bytes(a, d) + whole_bytes(a, d) + heads_bytes(a));
}

void paged_layout(PagedArgs &a, int d, void *workspace)
{
    unsigned char *p = static_cast<unsigned char *>(workspace);
    a.counters = reinterpret_cast<uint32_t *>(p);
    p += kCounterBytes;
    a.parts = reinterpret_cast<float *>(p);
    p += parts_bytes(a, d);
    a.prefix_parts = reinterpret_cast<float *>(p);
    p += prefix_bytes(a, d);
    a.whole = reinterpret_cast<float *>(p);
    p += whole_bytes(a, d);
    a.heads = reinterpret_cast<int4 *>(p);
}

hipError_t launch_paged_CACHE_F32_64(const PagedArgs &a, hipStream_t stream);
hipError_t launch_paged_CACHE_F32_128(const PagedArgs &a, hipStream_t stream);
hipError_t launch_paged_CACHE_BF16_64(const PagedArgs &a, hipStream_t stream);
hipError_t launch_paged_CACHE_BF16_128(const PagedArgs &a, hipStream_t stream);
hipError_t launch_paged_CACHE_BF16_256(const PagedArgs &a, hipStream_t stream);
hipError_t launch_paged_CACHE_E4M3_64(const PagedArgs &a, hipStream_t stream);
hipError_t launch_paged_CACHE_E4M3_128(const PagedArgs &a, hipStream_t stream);
hipError_t launch_paged_CACHE_E4M3_256(const PagedArgs &a, hipStream_t stream);

hipError_t launch_paged(const PagedArgs &a, int cache, int d, hipStream_t stream)
{
    if (cache == CACHE_F32) return d == 64 ? launch_paged_CACHE_F32_64(a, stream) : launch_paged_CACHE_F32_128(a, stream);
    if (cache == CACHE_BF16)
        return d == 64    ? launch_paged_CACHE_BF16_64(a, stream)
               : d == 128 ? launch_paged_CACHE_BF16_128(a, stream)
                          : launch_paged_CACHE_BF16_256(a, stream);
    return d == 64    ? launch_paged_CACHE_E4M3_64(a, stream)
           : d == 128 ? launch_paged_CACHE_E4M3_128(a, stream)
                      : launch_paged_CACHE_E4M3_256(a, stream);
}

hipError_t launch_paged_join(const PagedArgs &a, int cache, int d, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.n_seqs * a.n_q * a.n_heads;
    auto go = [&](auto kern, int at_once) {
        hipLaunchKernelGGL(kern, dim3((unsigned)((rows + at_once - 1) / at_once)), dim3(kT), 0, stream, a);
    };
    // four rows a workgroup where that leaves one for each half of a compute unit
    // (10240 rows of 7 to 9 parts: 11 us against 23; 2048 of 33: 8.2 against 9; but
    // one sequence of 8192 tokens, 16 rows of one key head: the call 20.1 against
    // 14.9)
    const bool many = rows >= 4 * kPagedGrid;
    auto width = [&](auto f32, auto width) {
        constexpr bool F32 = decltype(f32)::value;
        constexpr int D = decltype(width)::value;
        many ? go(paged_join_kernel<D, F32, 4>, 4) : go(paged_join_kernel<D, F32, 1>, 1);
    };
    if (cache == CACHE_F32)
        d == 64 ? width(std::true_type(), std::integral_constant<int, 64>())
                : width(std::true_type(), std::integral_constant<int, 128>());
    else
        d == 64    ? width(std::false_type(), std::integral_constant<int, 64>())
        : d == 128 ? width(std::false_type(), std::integral_constant<int, 128>())
                   : width(std::false_type(), std::integral_constant<int, 256>());
    return hipGetLastError();
}

}  // namespace rr
