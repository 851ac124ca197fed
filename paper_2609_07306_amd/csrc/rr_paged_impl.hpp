// Attention of the newest tokens of a batch of sequences over a paged cache
// (all of it, along routes of pages, or behind a shared prefix), for gfx950.
//
//   o = sum_u 2^(c q.k_u - m) v_u / l,  l = sum_u 2^(c q.k_u - m),  c = scale log2 e
//
// One pass over the keys with a running maximum m per query.  A call's work
// is cut into items: the query rows of one (sequence, key head) -- n_q tokens
// times the heads that share the key head -- in tiles of rows; with routes one
// query head's row, which has its own pages; with a shared prefix also tiles
// over the rows of the whole batch against the prefix, which is so read once a
// tile (up to 128 rows; 32 in binary32) in place of once a sequence.  Every
// item is a number of units of 128 keys, and the units of all items, in order,
// are cut into equal runs, one per workgroup: lengths that differ a hundredfold
// leave no compute unit idle, and one long sequence is spread over the card.
// (Not so along routes, where every item counts the units that its slots can
// name, so that workgroups of short sequences end early; and of many new tokens,
// whose row tiles all count the whole sequence.)  Lengths live on the device, so
// every workgroup sums them to find its run.  An item that lies in several
// runs leaves a part (m, l, sum) per run in the workspace, and the workgroup
// that finishes the last of them joins them.  A second launch does where that
// is faster (paged_schedule), and with a prefix, whose items share rows with
// the sequences'.
//
// Two bodies share this.  The narrow one is for items of up to 16 rows (in
// binary32 of any number, 32 at a time), where memory is the bound: each of four waves takes its own 32-key tiles of
// the run, so that no barrier stands between loads and products, and a tile's
// keys and values are requested while the tile before it is still in its
// softmax.  The wide one is for items of more rows, where the products are:
// a wave holds 32 rows, and the four share tiles of 64 keys through LDS.
#pragma once

#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>

#include "rr_device.hpp"
#include "rr_internal.hpp"
#include "rr_paged.hpp"

namespace rr {
namespace paged {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef short short8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));

constexpr int kMostWaves = 4;       // waves of a workgroup at most
constexpr int kStagedPages = 512;   // page numbers held in LDS at a time
constexpr int kJoin = 8;            // parts in flight of a thread that joins them
constexpr float kLazy = 8.f;        // log2 headroom of the running softmax maximum
constexpr float kLn2 = 0.6931471805599453f;
constexpr int32_t kNoToken = INT_MAX;

// Four bf16 of a transposed LDS read (ds_read_b64_tr_b16): lane i of each
// 16-lane group receives column i of the four rows that its lanes address,
// lane j the 8 bytes of row j / 4 at columns 4 (j % 4).
__device__ __forceinline__ short4_t lds_read_tr16(const unsigned char *p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t *)p);
}

__device__ __forceinline__ bf16x8_t as_bf16x8(u32x4_t x) { return __builtin_bit_cast(bf16x8_t, x); }

__device__ __forceinline__ bf16x8_t join8(short4_t x, short4_t y)
{
    return __builtin_bit_cast(bf16x8_t, (short8_t){x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]});
}

// Eight e4m3 values, exactly, as bf16.
__device__ __forceinline__ bf16x8_t e4m3_to_bf16(uint32_t lo, uint32_t hi)
{
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
    const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
    const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight weights as sums of two bf16 numbers each, 2^-16 off: rounded to one,
// they would add as much error as the rounding of the output.  The first
// number is the weight cut off after its eighth bit (a mask, no rounding), the
// second what that leaves, rounded.
__device__ __forceinline__ void split_weights(const float (&x)[8], bf16x8_t &hi, bf16x8_t &lo)
{
    u32x4_t h;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t a = __float_as_uint(x[2 * q]), b = __float_as_uint(x[2 * q + 1]);
        h[q] = __builtin_amdgcn_perm(b, a, 0x07060302u);  // the upper halves of b and a
        lo[2 * q] = (__bf16)(x[2 * q] - __uint_as_float(a & 0xFFFF0000u));
        lo[2 * q + 1] = (__bf16)(x[2 * q + 1] - __uint_as_float(b & 0xFFFF0000u));
    }
    hi = as_bf16x8(h);
}

// Where some rows of a product see a token and others don't, a value that is
// not finite would reach the others as 0 * inf.  It is taken out of the
// operand, and `odd` marks it: a product of the marks with "the row sees the
// token" then tells which outputs it belongs to.  Only where there is one: the
// marks of every mixed tile took 128 sequences of 20 to 400 tokens, 32 rows,
// from 47.7 to 52.9 us, 256 of 10 to 500, 12 rows, from 49.6 to 54.3.
__device__ __forceinline__ void take_odd(bf16x8_t &v, bf16x8_t &odd)
{
    // (bits of the whole vector: a bit cast of one of its elements takes the first one's)
    const short8_t bits = __builtin_bit_cast(short8_t, v);
    short8_t kept, marks;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const bool is = (bits[e] & 0x7F80) == 0x7F80;
        marks[e] = is ? (short)0x3F80 : (short)0;  // 1
        kept[e] = is ? (short)0 : bits[e];
    }
    v = __builtin_bit_cast(bf16x8_t, kept);
    odd = __builtin_bit_cast(bf16x8_t, marks);
}

// Adds to `found` whether one of the values in x (a cache's bits) is not finite:
// an exponent of ones (e4m3: NaN, all ones) and one more reaches the sign's bit.
template <int TY>
__device__ __forceinline__ void find_odd(uint32_t x, uint32_t &found)
{
    constexpr uint32_t ones = TY == CACHE_F32 ? 0x7F800000u : TY == CACHE_BF16 ? 0x7F807F80u : 0x7F7F7F7Fu;
    constexpr uint32_t one = TY == CACHE_F32 ? 0x00800000u : TY == CACHE_BF16 ? 0x00800080u : 0x01010101u;
    constexpr uint32_t sign = TY == CACHE_F32 ? 0x80000000u : TY == CACHE_BF16 ? 0x80008000u : 0x80808080u;
    found |= ((x & ones) + one) & sign;
}

// ------------------------------------------------------------- the runs

struct Item {
    bool prefix;
    int32_t b;      // sequence
    int32_t j;      // item within the sequence (or within the prefix)
    int32_t units;  // its units
    int32_t first;  // its first unit
    int32_t index;  // its number (of its head)
};

struct Run {
    int32_t me;               // its number
    int32_t at, end, per_wg;  // units [at, end) of the body's
    Item it;
};

// A value that is the same in all lanes, as the scalar that it is.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// LDS that both bodies use.
struct Common {
    int32_t phys[kStagedPages];
    int32_t chunk[kMaxAttnSlots];
    int32_t sum[kMostWaves];
    int32_t at, b;
    int32_t count[kMostWaves];
    int32_t lo[kMostWaves], hi[kMostWaves], bad[kMostWaves];
    int32_t lim[32 * kMostWaves];
    float m[kMostWaves][32], l[kMostWaves][32];
    float jm[16], jl[16];
};

__device__ __forceinline__ int32_t seq_units(const PagedArgs &a, int32_t b)
{
    if (a.route_units) return a.route_units;
    const int32_t n = held_tokens(a.lengths[b], a.capacity) - a.n_prefix, units = n <= 0 ? 0 : (n + kPagedUnit - 1) / kPagedUnit;
    return max(units + a.item_cost, 1);
}

// Run `me` of the items that a body takes: the prefix's, the sequences', or
// one after the other.  False where there is none.
template <int NW>
__device__ __forceinline__ bool find_run(const PagedArgs &a, Common &sh, int me, bool pre, bool own, Run &r)
{
    r.me = me;
    constexpr int T = 64 * NW;
    const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
    // (a call has less than 2^31 - kPagedGrid units)
    const int prefix_total = pre ? a.prefix_items * a.prefix_units : 0;
    // per thread: its sequences, their units and those of all before them
    const bool few = a.n_seqs <= 64;
    const int per = few ? 1 : (a.n_seqs + T - 1) / T;
    const int b0 = own ? min((few ? lane : tid) * per, a.n_seqs) : 0, b1 = own ? min(b0 + per, a.n_seqs) : 0;
    int sum = 0;
    for (int b = b0; b < b1; ++b) sum += seq_units(a, b);
    int before = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(before, o, 64);
        before += lane >= o ? v : 0;
    }
    int all = __builtin_amdgcn_readlane(before, 63);
    before -= sum;
    if (!few) {  // (else each wave for itself, without a barrier)
        __syncthreads();  // (an earlier body's readers of LDS are done)
        if (lane == 0) sh.sum[w] = all;
        __syncthreads();
        all = 0;
        for (int v = 0; v < NW; ++v) {
            before += v < w ? sh.sum[v] : 0;
            all += sh.sum[v];
        }
        all = uniform(all);
    }
    const int total = prefix_total + all * a.items_per_seq;
    // two workgroups a compute unit; but one of up to eight units where few
    // items are cut into many parts and one workgroup joins them, of which
    // there are then half as many (one sequence of 8192 tokens: 15.5 us
    // against 20.5; of 32768: 29.8 against 34.9; eight of 1000 to 8000: 31.0
    // against 31.9)
    r.per_wg = (total + a.grid - 1) / a.grid;
    if (!pre && !a.join_apart && a.n_seqs * a.items_per_seq <= kPagedGrid / 8)
        r.per_wg = max(r.per_wg, min(8, (total + kPagedGrid / 2 - 1) / (kPagedGrid / 2)));
    if ((int64_t)me * r.per_wg >= total) return false;
    r.at = me * r.per_wg;
    r.end = total - r.at < r.per_wg ? total : r.at + r.per_wg;
    // the sequence that the run begins in, and the units before it
    int b_at = 0, b_before = 0, b_units = 0;
    if (own && r.at >= prefix_total) {
        const int u = (r.at - prefix_total) / a.items_per_seq;
        const bool mine = u >= before && u < before + sum;
        if (few) {
            b_at = __ffsll((unsigned long long)__ballot(mine)) - 1;
            b_before = __builtin_amdgcn_readlane(before, b_at);
            b_units = __builtin_amdgcn_readlane(sum, b_at);
        } else {
            if (mine) {
                int b = b0, base = before;
                for (;;) {
                    const int n = seq_units(a, b);
                    if (u < base + n) break;
                    base += n;
                    ++b;
                }
                sh.b = b;
                sh.at = base;
            }
            __syncthreads();
            b_at = uniform(sh.b);
            b_before = uniform(sh.at);
            b_units = uniform(seq_units(a, b_at));
        }
    }
    Item &it = r.it;
    it.b = b_at;
    it.prefix = r.at < prefix_total;
    if (it.prefix) {
        it.units = a.prefix_units;
        it.j = r.at / it.units;
        it.index = it.j;
        it.first = it.j * it.units;
    } else {
        const int base = prefix_total + b_before * a.items_per_seq;
        it.units = b_units;
        it.j = (r.at - base) / it.units;
        it.index = a.prefix_items + b_at * a.items_per_seq + it.j;
        it.first = base + it.j * it.units;
    }
    return true;
}

__device__ __forceinline__ void next_item(const PagedArgs &a, Item &it)
{
    it.first += it.units;
    ++it.index;
    ++it.j;
    if (it.prefix) {
        if (it.j == a.prefix_items) {
            it.prefix = false;
            it.j = it.b = 0;
            it.units = uniform(seq_units(a, 0));
        }
    } else if (it.j == a.items_per_seq) {
        it.j = 0;
        ++it.b;
        it.units = uniform(seq_units(a, it.b));
    }
}

// The query rows of an item: of key head g, from row0 on.
struct Rows {
    bool prefix;
    int b, g, row0, n;

    // sequence, query token and head of row r
    __device__ __forceinline__ void of(const PagedArgs &a, int r, int &b_, int &t, int &h) const
    {
        int x = row0 + r;
        b_ = b;
        if (prefix) {
            b_ = x / a.rows;
            x -= b_ * a.rows;
        }
        t = x / a.group;
        h = g * a.group + (x - t * a.group);
    }
    // the last token that row r sees, -1 for none
    __device__ __forceinline__ int last(const PagedArgs &a, int r) const
    {
        int b_, t, h;
        of(a, r, b_, t, h);
        const int p = held_tokens(a.lengths[b_], a.capacity) - a.n_q + t;
        return max(prefix ? min(p, a.n_prefix - 1) : p, -1);
    }
};

__device__ __forceinline__ Rows rows_of(const PagedArgs &a, const Item &it)
{
    Rows r;
    r.prefix = it.prefix;
    r.b = it.b;
    if (it.prefix) {
        r.g = it.j / a.prefix_tiles;
        r.row0 = (it.j - r.g * a.prefix_tiles) * a.prefix_tile;
        r.n = min(a.prefix_tile, a.prefix_rows - r.row0);
    } else if (a.route_units) {
        // item = head * n_q + query token: row t * group + j of its key head
        const int h = it.j / a.n_q, t = it.j - h * a.n_q;
        r.g = h / a.group;
        r.row0 = t * a.group + (h - r.g * a.group);
        r.n = 1;
    } else {
        r.g = it.j / a.row_tiles;
        r.row0 = (it.j - r.g * a.row_tiles) * a.own_tile;
        r.n = min(a.own_tile, a.rows - r.row0);
    }
    return r;
}

// Where a body writes an item's result: the output itself where no other item
// or workgroup has a part in its rows, else a part of D sums, the maximum and
// the sum of weights: D + 4 floats a row.
struct Sink {
    bool last_word;
    float *by_row;  // parts by row of the call, or null:
    float *cut;     // parts by row of the item

    __device__ __forceinline__ float *part(int D, int r, int64_t orow) const
    {
        return by_row ? by_row + orow * (D + 4) : cut + (int64_t)r * (D + 4);
    }
};

// The part of an item that run wg leaves: a run's first item has its slot
// 2 wg, the one that it ends in slot 2 wg + 1.
__device__ __forceinline__ int part_slot(const Run &r, int wg) { return 2 * wg + (wg * r.per_wg >= r.it.first ? 0 : 1); }

__device__ __forceinline__ Sink sink_of(const PagedArgs &a, int D, const Run &r, int u0, int u1, int tile)
{
    const bool entire = u0 == 0 && u1 == r.it.units;
    const int slot = part_slot(r, r.me);
    Sink s;
    s.last_word = entire && a.prefix_items == 0;
    s.by_row = entire ? a.whole + (r.it.prefix ? 0 : (int64_t)a.n_seqs * a.n_q * a.n_heads) * (D + 4) : nullptr;
    s.cut = a.parts + (int64_t)slot * tile * (D + 4);
    if ((a.prefix_items || a.join_apart) && u0 == 0 && threadIdx.x == 0) {
        // the item's head, for a second launch: its first part, its first workgroup, its parts
        const int last_wg = (r.it.first + r.it.units - 1) / r.per_wg;
        a.heads[r.it.index] = int4{slot, r.me, last_wg - r.me + 1, 0};
    }
    return s;
}

__device__ __forceinline__ float inverse_sum(float sum, float scale)
{
    return sum > 0.f ? scale / sum : sum == 0.f ? 0.f : sum;  // (a sum that is NaN stays)
}

__device__ __forceinline__ float log_sum(float m, float sum) { return m == -INFINITY ? -INFINITY : (m + log2f(sum)) * kLn2; }

// Adds a part (four features y, maximum mi, sum of weights li) to sums x with
// maximum m and sum of weights l.  A part of weight 0 is added too: its sums are
// NaN or infinite where its rows see a value that is, and stay so.  (A part whose
// row sees nothing holds zeros.)
__device__ __forceinline__ void add_part(const f32x4_t y, float mi, float li, f32x4_t &x, float &m, float &l)
{
    const float m_new = fmaxf(m, mi);
    const float w0 = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
    const float w1 = mi == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mi - m_new);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(w1, y[e], w0 * x[e]);
    l = w0 * l + w1 * li;
    m = m_new;
}

template <bool F32>
__device__ __forceinline__ void write_four(void *O, int64_t at, f32x4_t x)
{
    if constexpr (F32) {
        *reinterpret_cast<f32x4_t *>(static_cast<float *>(O) + at) = x;
    } else {
        bf16x4_t y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (__bf16)x[i];
        *reinterpret_cast<bf16x4_t *>(static_cast<__bf16 *>(O) + at) = y;
    }
}

// Waits for all of the wave's loads from memory and stores to it.
__device__ __forceinline__ void wait_vm() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Parts pass between workgroups on different XCDs, whose L2 caches do not
// see each other's lines.  They are stored and loaded at device scope (sc1, as
// a device-scope atomic is), which goes past the L2, so a part is there once
// its stores have returned, which the storing wave waits for (vmcnt) before its
// workgroup's relaxed atomic counts the part; the loads follow the atomic whose
// value says that all are there.  That is what these instructions do on gfx950,
// not what the memory model of the language promises, which asks for a release
// and an acquire: a release fence would write the whole L2 back, from every
// workgroup (measured: one sequence's decode 17 -> 72 us).
// (Where a second launch reads them they are plain stores.)
constexpr int kDeviceScope = 16;  // sc1 of a buffer instruction

template <int D>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t parts_of(const PagedArgs &a)
{
    return __builtin_amdgcn_make_buffer_rsrc(a.parts, 0, 2 * a.grid * a.own_tile * (D + 4) * (int)sizeof(float), 0x00020000);
}

// Four sums (or the maximum and the sum of weights, and two that nothing
// reads) at p, which lies in a.parts where they are joined within the launch.
template <int D>
__device__ __forceinline__ void store_part(const PagedArgs &a, float *p, f32x4_t x, bool within)
{
    if (within)
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, x), parts_of<D>(a),
                                               (int)((p - a.parts) * sizeof(float)), 0, kDeviceScope);
    else
        *reinterpret_cast<f32x4_t *>(p) = x;
}

// After a part of a cut item was stored: the workgroup that comes last of the
// item's joins them, in the order of the keys whoever comes last.  The counter
// (one per workgroup that an item may begin in) is left at zero.
template <int D, bool F32, int NW>
__device__ __forceinline__ void join_cut(const PagedArgs &a, Common &sh, unsigned char *smem, const Run &run, const Rows &rows,
                                         int tile)
{
    constexpr int T = 64 * NW, PL = D / 4, NP = T / PL;  // lanes of a part, parts in flight
    const int tid = threadIdx.x;
    const int wg0 = run.it.first / run.per_wg, n = (run.it.first + run.it.units - 1) / run.per_wg - wg0 + 1;
    wait_vm();        // this wave's stores have returned ...
    __syncthreads();  // ... and the other waves'
    if (tid == 0) {
        const uint32_t before = __hip_atomic_fetch_add(a.counters + wg0, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (before == (uint32_t)(n - 1)) __hip_atomic_store(a.counters + wg0, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        sh.at = before == (uint32_t)(n - 1);
    }
    __syncthreads();
    if (!uniform(sh.at)) return;
    // (bytes; at most 2 * 512 parts of 128 rows)
    constexpr int ROW = (D + 4) * (int)sizeof(float);
    const int stride = 2 * tile * ROW, first = part_slot(run, wg0) * tile * ROW, rest = wg0 * stride;
    const __amdgpu_buffer_rsrc_t parts = parts_of<D>(a);
    // groups of a row: a power of two, all of them for one row
    int per_row = NP;
    while (per_row > 1 && per_row * rows.n > NP) per_row >>= 1;
    const int pl = tid % PL, pg = tid / PL, sub = pg & (per_row - 1);
    float *s_acc = reinterpret_cast<float *>(smem);
    const float vs = a.v_scale ? a.v_scale[rows.g] : 1.f;
    for (int r = pg / per_row; r < rows.n || per_row > 1; r += NP / per_row) {
        f32x4_t x = {0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        if (r < rows.n) {
            // (kJoin parts are asked for before the first is used)
            for (int i0 = sub; i0 < n; i0 += kJoin * per_row) {
                u32x4_t y[kJoin];
                u32x2_t ml[kJoin];
#pragma unroll
                for (int k = 0; k < kJoin; ++k) {
                    const int i = min(i0 + k * per_row, n - 1), at = (i == 0 ? first : rest + i * stride) + r * ROW;
                    y[k] = __builtin_amdgcn_raw_buffer_load_b128(parts, at + 16 * pl, 0, kDeviceScope);
                    ml[k] = __builtin_amdgcn_raw_buffer_load_b64(parts, at + 4 * D, 0, kDeviceScope);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int k = 0; k < kJoin; ++k)
                    if (i0 + k * per_row < n)
                        add_part(__builtin_bit_cast(f32x4_t, y[k]), __uint_as_float(ml[k][0]), __uint_as_float(ml[k][1]),
                                 x, m, l);
            }
        }
        if (per_row > 1) {  // (uniform; one round, every thread)
            *reinterpret_cast<f32x4_t *>(s_acc + pg * D + 4 * pl) = x;
            if (pl == 0) {
                sh.jm[pg] = m;
                sh.jl[pg] = l;
            }
            __syncthreads();
            if (sub == 0)
                for (int i = 1; i < per_row; ++i)
                    add_part(*reinterpret_cast<const f32x4_t *>(s_acc + (pg + i) * D + 4 * pl), sh.jm[pg + i],
                             sh.jl[pg + i], x, m, l);
        }
        if (r < rows.n && sub == 0) {
            int b, t, h;
            rows.of(a, r, b, t, h);
            const int64_t orow = ((int64_t)b * a.n_q + t) * a.n_heads + h;
            write_four<F32>(a.O, orow * D + 4 * pl, x * inverse_sum(l, vs));
            if (a.lse && pl == 0) a.lse[orow] = log_sum(m, l);
        }
        if (per_row > 1) break;
    }
}

// ------------------------------------------------------------- narrow body
//
// S^T = K Q^T on 16x16 MFMA tiles with the keys as rows, so K goes from memory
// to the operand registers as it lies (a lane holds 16 bytes of one key); a
// lane then has four scores of one query per tile, which are just the keys
// that its part of the operand of O^T = V^T P^T takes.  V is transposed on the
// way: row-major into a buffer of the wave's own in LDS, read with the LDS
// transpose read; in binary32, where an operand holds one key per lane,
// straight from memory.
//
// Bound by the reads of K and V: 64 sequences of 300 to 32768 tokens (32 heads
// on 8, d = 128) 342 us, 5.75 TB/s; 128 of 100 to 16384 in an 8-bit cache 174
// us, 4.9 TB/s (each item begins with a chain of loads; 64 of 8192: 5.7); along
// routes 187 us, 5.6 TB/s.  One sequence of 8192 tokens
// (33 MB, 6.6 us of reads) takes 15.7 us: the chain length, page, tile before
// the reads, and after them the parts that pass between workgroups.

// What a cache type's tiles look like.
//   KT  keys of a wave's tile
//   KR  rows (keys) of a tile that a lane loads 16-byte pieces of
//   PK  such pieces of a row and lane: piece c of lane group kg holds the
//       row's elements from (4 c + kg) * (16 / SIZE) on
template <int TY, int D>
struct Shape {
    static constexpr int SIZE = TY == CACHE_F32 ? 4 : TY == CACHE_BF16 ? 2 : 1;
    static constexpr int KT = TY == CACHE_F32 ? 16 : 32;
    static constexpr int KR = KT / 16;
    static constexpr int PK = D * SIZE / 64;
    // bytes of a row of the V buffer: 8 banks from one row to the next; rows 8 ..
    // 15 of 16 hold their 16-byte pieces in swapped pairs.  (Laid out so that the
    // transposed reads, 8 rows x 32 bytes at a time, and the writes, 16 rows x 16
    // bytes, spread over the banks; the counters show conflicts in three eighths
    // of the cycles that LDS works all the same, which is not what these bodies
    // wait for)
    static constexpr int VRS = 2 * D + 32;
    static constexpr int ORS = D + 4;       // floats of a row of the output buffer
    static constexpr int VBYTES = TY == CACHE_F32 ? 0 : KT * VRS;
    static constexpr int OBYTES = 16 * ORS * 4;
    static constexpr int WAVE = VBYTES > OBYTES ? VBYTES : OBYTES;
};

// The feature that element i of value accumulator v belongs to, for lane
// group kg.
template <int TY>
__device__ __forceinline__ int feature_of(int v, int i, int kg)
{
    if constexpr (TY == CACHE_F32)
        return 64 * (v >> 2) + 16 * kg + 4 * i + (v & 3);  // (rows of V^T are 4 features apart)
    else
        return 16 * v + 4 * kg + i;
}

template <int TY, int D, int NR, int NW>
__device__ __forceinline__ void narrow_body(const PagedArgs &a, Common &sh, unsigned char *smem, int me, bool pre, bool own)
{
    using S = Shape<TY, D>;
    constexpr bool F32 = TY == CACHE_F32;
    static_assert(F32 || NR == 1, "bf16 items of more than 16 rows are the wide body's");
    constexpr int NV = D / 16;  // value accumulators of a row block
    constexpr int T = 64 * NW;
    Run run;
    if (!find_run<NW>(a, sh, me, pre, own, run)) return;
    const int tid = threadIdx.x, w = uniform(tid >> 6), lane = tid & 63, l16 = lane & 15, kg = lane >> 4;
    unsigned char *vbuf = smem + w * S::WAVE;

    for (;;) {
        const Item &it = run.it;
        const int u0 = run.at - it.first, u1 = min(it.units, run.end - it.first);
        const Rows rows = rows_of(a, it);
        const int g = rows.g, blocks = (rows.n + 15) >> 4;

        // (a sequence's first item_cost units stand for what an item costs besides its keys)
        const int cost = it.prefix || a.route_units ? 0 : a.item_cost, k0 = max(u0 - cost, 0), k1 = max(u1 - cost, 0);
        // key positions: tokens from `base` on, or, along routes, the places
        // of the listed pages one after the other.  The run's first pages (or
        // the row's routes) are asked for here, before the lengths are there
        const int base = it.prefix ? 0 : a.n_prefix, slots = a.n_sink + a.n_recent + a.k;
        const int32_t *pages = it.prefix ? a.prefix_pages : a.table + (int64_t)it.b * a.max_pages;
        const int last_page = it.prefix ? a.pd.div(a.n_prefix - 1) : a.max_pages - 1;
        int asked = -1;
        if (a.route_units) {
            const int64_t row = ((int64_t)it.b * a.items_per_seq + it.j) * a.k;
            if (tid >= a.n_sink + a.n_recent && tid < slots) asked = a.routes[row + tid - a.n_sink - a.n_recent];
        } else {
            asked = pages[min(a.pd.div(base + min(k0 * kPagedUnit, a.capacity)) + tid, last_page)];
        }

        // query operands; lim: the last token that a row sees (-1: none);
        // lo and hi: the least and the largest of them that is one
        bf16x8_t fq[F32 ? 1 : D / 32];
        f32x4_t fqf[F32 ? NR : 1][F32 ? D / 16 : 1];
        int lim[NR], lo = kNoToken, hi = -1;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            int b, t, h;
            const int r = min(16 * n + l16, rows.n - 1);
            rows.of(a, r, b, t, h);
            lim[n] = rows.last(a, r);
            if (lim[n] >= 0) {
                lo = min(lo, lim[n]);
                hi = max(hi, lim[n]);
            }
            const int64_t q = (((int64_t)b * a.n_q + t) * a.n_heads + h) * D;
            if constexpr (F32) {
#pragma unroll
                for (int c = 0; c < D / 16; ++c)
                    fqf[n][c] = *reinterpret_cast<const f32x4_t *>(static_cast<const float *>(a.Q) + q + 16 * c + 4 * kg);
            } else {
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    // (e4m3 keys come 16 to a piece, two operands of 8)
                    const int f = TY == CACHE_E4M3 ? 64 * (c >> 1) + 16 * kg + 8 * (c & 1) : 32 * c + 8 * kg;
                    fq[c] = as_bf16x8(*reinterpret_cast<const u32x4_t *>(static_cast<const bf16_t *>(a.Q) + q + f));
                }
            }
        }
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) {
            lo = min(lo, __shfl_xor(lo, o, 64));
            hi = max(hi, __shfl_xor(hi, o, 64));
        }
        lo = uniform(lo);
        hi = uniform(hi);

        float m_run[NR], l_run[NR];
        f32x4_t acc[NR][NV];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            m_run[n] = -INFINITY;
            l_run[n] = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v) acc[n][v] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        const float c2 = a.scale * 1.4426950408889634f * (a.k_scale ? a.k_scale[g] : 1.f);

        int n_pos;
        __syncthreads();  // (the last item's readers of LDS are done)
        if (a.route_units) {
            // the pages that the row sees, each once: a slot is dropped if an
            // earlier one names its page
            const int here = hi >= 0 ? a.pd.div(hi) : -1;
            static_assert(kMaxAttnSlots <= T, "a slot per thread");
            int id = -1;
            if (tid < a.n_sink)
                id = tid;
            else if (tid < a.n_sink + a.n_recent)
                id = here - (tid - a.n_sink);
            else if (tid < slots)
                id = asked;
            bool ok = tid < slots && id >= 0 && id <= here;
            if (tid < kMaxAttnSlots) sh.phys[tid] = ok ? id : -1;
            __syncthreads();
            if (ok)
                for (int s = 0; s < tid; ++s) ok = ok && sh.phys[s] != id;
            const uint64_t mk = __ballot(ok);
            if (lane == 0) sh.count[w] = __popcll(mk);
            __syncthreads();
            int before = __popcll(mk & ((1ull << lane) - 1ull)), all = 0;
            for (int v = 0; v < NW; ++v) {
                before += v < w ? sh.count[v] : 0;
                all += sh.count[v];
            }
            if (ok) {
                sh.chunk[before] = id;
                sh.phys[before] = pool_page(a.table[(int64_t)it.b * a.max_pages + id], a.n_pages);
            }
            n_pos = uniform(all) * a.pd.page;
        } else {
            n_pos = hi < base ? 0 : hi - base + 1;
        }
        const int p0 = (int)min((int64_t)k0 * kPagedUnit, (int64_t)n_pos);
        const int p1 = (int)min((int64_t)k1 * kPagedUnit, (int64_t)n_pos);

        for (int pa = p0; pa < p1; pa += a.batch_keys) {
            const int pb = min(p1 - pa, a.batch_keys) + pa;
            const int ch0 = a.route_units ? 0 : a.pd.div(base + pa);
            if (!a.route_units) {  // (routes: a list of at most 256 pages is there whole)
                if (pa != p0) __syncthreads();
                const int n = a.pd.div(base + pb - 1) - ch0 + 1;
                for (int c = tid; c < n; c += T)
                    sh.phys[c] = pool_page(pa == p0 && c < T ? asked : pages[ch0 + c], a.n_pages);
            }
            __syncthreads();

            // where position p lies: its token and page, kNoToken where the
            // page is none or p is past the run
            auto locate = [&](int p, int &phys, int &place) -> int32_t {
                const bool in = p < pb;
                p = min(p, pb - 1);
                int tok;
                if (a.route_units) {
                    const int s = a.pd.div(p);
                    place = p - s * a.pd.page;
                    phys = sh.phys[s];
                    tok = sh.chunk[s] * a.pd.page + place;
                } else {
                    tok = base + p;
                    const int c = a.pd.div(tok);
                    place = tok - c * a.pd.page;
                    phys = sh.phys[c - ch0];
                }
                const bool ok = in && phys >= 0 && tok <= hi;
                if (!ok) phys = place = 0;  // (row 0 of the pool is there)
                return ok ? tok : kNoToken;
            };

            u32x4_t kr[S::KR][S::PK], vr[S::KR][S::PK];
            int32_t tok[S::KR];
            const unsigned char *Kb = static_cast<const unsigned char *>(a.K);
            const unsigned char *Vb = static_cast<const unsigned char *>(a.V);
            auto load = [&](int p) {
                int64_t off[S::KR];
#pragma unroll
                for (int r = 0; r < S::KR; ++r) {
                    int phys, place;
                    tok[r] = locate(p + 16 * r + l16, phys, place);
                    off[r] = pool_row(phys, a.n_kv_heads, g, a.pd.page, place, D) * S::SIZE;
                }
#pragma unroll
                for (int r = 0; r < S::KR; ++r)
#pragma unroll
                    for (int c = 0; c < S::PK; ++c)
                        kr[r][c] = *reinterpret_cast<const u32x4_t *>(Kb + off[r] + 64 * c + 16 * kg);
                if constexpr (F32) {
                    // V^T operands: lane (l16, kg) takes features 64 c + 4 l16 ..
                    // of key 4 kg + s: vr[0][4 c + s]
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        const int64_t o = (int64_t)shfl_u64((uint64_t)off[0], 4 * kg + s);
#pragma unroll
                        for (int c = 0; c < D / 64; ++c)
                            vr[0][4 * c + s] = *reinterpret_cast<const u32x4_t *>(Vb + o + 256 * c + 16 * l16);
                    }
                } else {
#pragma unroll
                    for (int r = 0; r < S::KR; ++r)
#pragma unroll
                        for (int c = 0; c < S::PK; ++c)
                            vr[r][c] = *reinterpret_cast<const u32x4_t *>(Vb + off[r] + 64 * c + 16 * kg);
                }
            };

            int p = pa + w * S::KT;
            if (p < pb) load(p);
            for (; p < pb; p += NW * S::KT) {
                // (wave-uniform) all_seen: every key of the tile is seen by
                // every row; mixed: some key by some rows and not by others
                bool all_seen = true, mixed = false;
#pragma unroll
                for (int r = 0; r < S::KR; ++r) {
                    all_seen = all_seen && tok[r] <= lo;
                    mixed = mixed || (tok[r] > lo && tok[r] != kNoToken);
                }
                all_seen = __ballot(all_seen) == ~0ull;
                mixed = __ballot(mixed) != 0ull;

                // rows that no query sees become zeros: their weights are 0,
                // but memory that was never written may hold NaN.  Of a mixed
                // tile's other rows it matters whether all are finite
                uint32_t found = 0;
                if constexpr (F32) {
                    if (!all_seen) {
#pragma unroll
                        for (int s = 0; s < 4; ++s) {
                            const bool keep = __shfl(tok[0], 4 * kg + s, 64) != kNoToken;
#pragma unroll
                            for (int c = 0; c < D / 64; ++c)
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    vr[0][4 * c + s][e] = keep ? vr[0][4 * c + s][e] : 0u;
                                    find_odd<TY>(vr[0][4 * c + s][e], found);
                                }
                        }
                    }
                } else {
                    __builtin_amdgcn_wave_barrier();  // (the buffer's readers are this wave's, and in order)
#pragma unroll
                    for (int r = 0; r < S::KR; ++r) {
                        const bool keep = tok[r] != kNoToken;
#pragma unroll
                        for (int c = 0; c < S::PK; ++c) {
                            if (!all_seen) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    vr[r][c][e] = keep ? vr[r][c][e] : 0u;
                                    find_odd<TY>(vr[r][c][e], found);
                                }
                            }
                            unsigned char *dst = vbuf + (16 * r + l16) * S::VRS;
                            const int swap = (l16 & 8) << 1;
                            if constexpr (TY == CACHE_BF16) {
                                *reinterpret_cast<u32x4_t *>(dst + ((64 * c + 16 * kg) ^ swap)) = vr[r][c];
                            } else {
                                const int at = 128 * c + 32 * kg;
                                *reinterpret_cast<bf16x8_t *>(dst + (at ^ swap)) = e4m3_to_bf16(vr[r][c][0], vr[r][c][1]);
                                *reinterpret_cast<bf16x8_t *>(dst + ((at + 16) ^ swap)) = e4m3_to_bf16(vr[r][c][2], vr[r][c][3]);
                            }
                        }
                    }
                    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
                    __builtin_amdgcn_wave_barrier();
                }

                mixed = mixed && __ballot(found != 0) != 0ull;

                // S^T = K Q^T: s[n][r] of lane (l16, kg): keys 16 r + 4 kg + i
                // of the tile, query row 16 n + l16
                f32x4_t s[NR][S::KR];
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int r = 0; r < S::KR; ++r) s[n][r] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int r = 0; r < S::KR; ++r) {
#pragma unroll
                    for (int c = 0; c < S::PK; ++c) {
                        if constexpr (F32) {
                            const f32x4_t k4 = __builtin_bit_cast(f32x4_t, kr[r][c]);
#pragma unroll
                            for (int n = 0; n < NR; ++n)
                                if (NR == 1 || n < blocks)
#pragma unroll
                                    for (int e = 0; e < 4; ++e)
                                        s[n][r] = __builtin_amdgcn_mfma_f32_16x16x4f32(k4[e], fqf[n][c][e], s[n][r], 0, 0, 0);
                        } else if constexpr (TY == CACHE_BF16) {
                            s[0][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kr[r][c]), fq[c], s[0][r], 0, 0, 0);
                        } else {
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                const bf16x8_t kf = e4m3_to_bf16(kr[r][c][2 * q], kr[r][c][2 * q + 1]);
                                s[0][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, fq[2 * c + q], s[0][r], 0, 0, 0);
                            }
                        }
                    }
                }
                int32_t of_key[S::KR][4];  // token of key 16 r + 4 kg + i
                if (!all_seen) {
#pragma unroll
                    for (int r = 0; r < S::KR; ++r)
#pragma unroll
                        for (int i = 0; i < 4; ++i) of_key[r][i] = __shfl(tok[r], 4 * kg + i, 64);
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        const int last = lim[n] < 0 ? hi : lim[n];
#pragma unroll
                        for (int r = 0; r < S::KR; ++r)
#pragma unroll
                            for (int i = 0; i < 4; ++i) s[n][r][i] = of_key[r][i] <= last ? s[n][r][i] : -INFINITY;
                    }
                }
                f32x4_t vf[F32 ? D / 16 : 1];
                if constexpr (F32) {
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) vf[c] = __builtin_bit_cast(f32x4_t, vr[0][c]);
                }
                if (p + NW * S::KT < pb) load(p + NW * S::KT);

                // the running maximum moves only when a score exceeds it by
                // more than kLazy (weights are then at most 2^kLazy), so that
                // lanes compare notes and rescale rarely
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    if (NR > 1 && n >= blocks) continue;
                    float mx = s[n][0][0];
#pragma unroll
                    for (int r = 0; r < S::KR; ++r)
#pragma unroll
                        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[n][r][i]);
                    mx *= c2;
                    if (__ballot(mx > m_run[n] + kLazy) != 0ull) {
                        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
                        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                        const float m_new = fmaxf(m_run[n], mx);
                        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[n] - m_new);
                        l_run[n] *= alpha;
#pragma unroll
                        for (int v = 0; v < NV; ++v)
#pragma unroll
                            for (int i = 0; i < 4; ++i) acc[n][v][i] *= alpha;
                        m_run[n] = m_new;
                    }
                    const float m_use = m_run[n] == -INFINITY ? 0.f : m_run[n];
#pragma unroll
                    for (int r = 0; r < S::KR; ++r)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            s[n][r][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][r][i], c2, -m_use));
                            l_run[n] += s[n][r][i];
                        }
                }

                // O^T += V^T P^T
                if constexpr (F32) {
                    auto values = [&](auto odd_tile) {
#pragma unroll
                        for (int c = 0; c < D / 64; ++c)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    float x = vf[4 * c + i][e], odd = 0.f;
                                    if constexpr (decltype(odd_tile)::value) {
                                        const bool is = (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u;
                                        odd = is ? 1.f : 0.f;
                                        x = is ? 0.f : x;
                                    }
#pragma unroll
                                    for (int n = 0; n < NR; ++n) {
                                        if (NR > 1 && n >= blocks) continue;
                                        f32x4_t &o = acc[n][4 * c + e];
                                        o = __builtin_amdgcn_mfma_f32_16x16x4f32(x, s[n][0][i], o, 0, 0, 0);
                                        if constexpr (decltype(odd_tile)::value) {
                                            const float sees = of_key[0][i] <= (lim[n] < 0 ? hi : lim[n]) ? 1.f : 0.f;
                                            const f32x4_t z = {0.f, 0.f, 0.f, 0.f};
                                            const f32x4_t k = __builtin_amdgcn_mfma_f32_16x16x4f32(odd, sees, z, 0, 0, 0);
#pragma unroll
                                            for (int y = 0; y < 4; ++y) o[y] = k[y] > 0.f ? NAN : o[y];
                                        }
                                    }
                                }
                    };
                    if (mixed)
                        values(std::true_type());
                    else
                        values(std::false_type());
                } else {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = s[0][e >> 2][e & 3];
                    bf16x8_t ph, pl;
                    split_weights(x, ph, pl);
                    // (rows 4 kg + 0..3 of 16: swapped pieces where kg & 2)
                    const unsigned char *vp = vbuf + (4 * kg + (l16 >> 2)) * S::VRS;
                    const int piece = (8 * (l16 & 3)) ^ ((kg & 2) << 3);
                    auto values = [&](auto odd_tile) {
#pragma unroll
                        for (int v = 0; v < NV; ++v) {
                            const unsigned char *x = vp + 32 * v + piece;
                            bf16x8_t vt = join8(lds_read_tr16(x), lds_read_tr16(x + 16 * S::VRS)), odd;
                            if constexpr (decltype(odd_tile)::value) take_odd(vt, odd);
                            f32x4_t &o = acc[0][v];
                            o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, ph, o, 0, 0, 0);
                            o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pl, o, 0, 0, 0);
                            if constexpr (decltype(odd_tile)::value) {
                                bf16x8_t sees;
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    sees[e] = of_key[e >> 2][e & 3] <= (lim[0] < 0 ? hi : lim[0]) ? (__bf16)1.f : (__bf16)0.f;
                                const f32x4_t z = {0.f, 0.f, 0.f, 0.f};
                                const f32x4_t c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, sees, z, 0, 0, 0);
#pragma unroll
                                for (int y = 0; y < 4; ++y) o[y] = c[y] > 0.f ? NAN : o[y];
                            }
                        }
                    };
                    if (mixed)
                        values(std::true_type());
                    else
                        values(std::false_type());
                }
            }
        }

        // ------------------------- the waves' sums joined, the result written
        const Sink sink = sink_of(a, D, run, u0, u1, a.own_tile);
        const bool within = a.prefix_items == 0 && !a.join_apart;  // the parts are joined within this launch
        const float vs = a.v_scale ? a.v_scale[g] : 1.f;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            if (n >= blocks) continue;  // (uniform)
            __syncthreads();
            float *ob = reinterpret_cast<float *>(smem + w * S::WAVE);
            const bool none = lim[n] < 0;
            // (it went along as a row that sees all of the item's tokens, of which
            // some may not be finite)
            if (__ballot(none) != 0ull) {
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[n][v][i] = none ? 0.f : acc[n][v][i];
            }
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if constexpr (F32) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) ob[l16 * S::ORS + feature_of<TY>(v, i, kg)] = acc[n][v][i];
                } else {
                    *reinterpret_cast<f32x4_t *>(ob + l16 * S::ORS + feature_of<TY>(v, 0, kg)) = acc[n][v];
                }
            }
            float l = l_run[n];
            l += __shfl_xor(l, 16, 64);
            l += __shfl_xor(l, 32, 64);
            if (kg == 0) {
                // (scores that are all NaN leave no maximum, but their sum counts)
                sh.m[w][l16] = none ? -INFINITY : l != l ? 0.f : m_run[n];
                sh.l[w][l16] = none ? 0.f : l;
            }
            __syncthreads();
            // 16 threads a row, D / 16 features each in pieces of four
            const int q = tid >> 4, r = 16 * n + q;
            if (q < 16 && r < rows.n) {
                float m = -INFINITY, sum = 0.f, wt[NW];
#pragma unroll
                for (int v = 0; v < NW; ++v) m = fmaxf(m, sh.m[v][q]);
#pragma unroll
                for (int v = 0; v < NW; ++v) {
                    wt[v] = sh.m[v][q] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sh.m[v][q] - m);
                    sum += wt[v] * sh.l[v][q];
                }
                int b, t, h;
                rows.of(a, r, b, t, h);
                const int64_t orow = ((int64_t)b * a.n_q + t) * a.n_heads + h;
                const float inv = inverse_sum(sum, vs);
                float *part = sink.part(D, r, orow);
#pragma unroll
                for (int f0 = 0; f0 < D / 64; ++f0) {
                    const int f = 64 * f0 + 4 * (tid & 15);
                    f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int v = 0; v < NW; ++v) {
                        const float *ov = reinterpret_cast<const float *>(smem + v * S::WAVE);
                        const f32x4_t y = *reinterpret_cast<const f32x4_t *>(ov + q * S::ORS + f);
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[i] = __builtin_fmaf(wt[v], y[i], x[i]);  // (0 * NaN stays, see add_part)
                    }
                    if (sink.last_word)
                        write_four<F32>(a.O, orow * D + f, x * inv);
                    else
                        store_part<D>(a, part + f, x, within);
                }
                if ((tid & 15) == 0) {
                    if (!sink.last_word) {
                        store_part<D>(a, part + D, f32x4_t{m, sum, 0.f, 0.f}, within);
                    } else if (a.lse) {
                        a.lse[orow] = log_sum(m, sum);
                    }
                }
            }
        }
        if (within && (u0 != 0 || u1 != it.units)) join_cut<D, F32, NW>(a, sh, smem, run, rows, a.own_tile);
        run.at = it.first + u1;
        if (run.at >= run.end) return;
        next_item(a, run.it);
    }
}

// --------------------------------------------------------------- wide body
//
// S^T = K Q^T on 32x32 MFMA tiles: a lane owns one query row and 16 keys of a
// 32-key block, which is the order in which O^T = V^T P^T takes them.  A row
// block is one wave's; items of half as many rows as the waves could hold, or
// less, give two waves to a row block, each with every other key block.
//
// Bound by the products and the softmax's vector instructions, which overlap
// little, and by the tiles' way from the L2 to LDS: 2048 new tokens behind
// 6144 (d = 128, 32 heads on 8) 306 us, 1280 rows a key head on a prefix of
// 32768 tokens 240 us, 715 TFLOP/s.  Without the loads it would take 195 us.
// TWO: a weight enters the value product as two bf16 numbers, as in the narrow
// body, else rounded to one (paged_schedule says which, with the times of both).
// Measured and not kept: which of them decided at run time (the rows of 128-row
// tiles then take 4 to 10 % longer, the others 2 to 13 %); the next tile's loads between the products (274 us
// for the call where this takes 267), the softmax of one block between the
// products of the next one (291 against 262), eight waves that share tiles in
// three stages (257 against 268 there, but 69 against 59 for 256 rows on 8192
// tokens, 27 against 23 for 32 rows on 4096).

template <int TY, int D>
struct WideShape {
    static constexpr int NW = 4;
    static constexpr int T = 64 * NW;
    static constexpr int ROWS = 32 * NW;           // rows of an item at most
    static constexpr int SIZE = TY == CACHE_BF16 ? 2 : 1;
    static constexpr int KB = D <= 128 ? 64 : 32;  // keys of a staged tile
    static constexpr int NB = KB / 32;
    // bf16 tiles go from memory to LDS without passing through registers, which
    // leaves no room between rows: a row's 16-byte chunk c lies at place c ^
    // key_swap(row), c ^ value_swap(row) instead, so that the rows that are
    // read together (16 at one chunk; 4 at four chunks) meet different banks.
    // e4m3 tiles are widened on the way and have padded rows
    static constexpr bool DIRECT = TY == CACHE_BF16;
    static constexpr int KRS = DIRECT ? 2 * D : 2 * D + 16;  // bytes of a row of the K tile
    static constexpr int VRS = DIRECT ? 2 * D : 2 * D + 64;  // ... of the V tile
    static constexpr int BUF = KB * (KRS + VRS);
    __device__ __forceinline__ static int key_swap(int row) { return !DIRECT ? 0 : D == 64 ? (row >> 1) & 7 : row & 15; }
    __device__ __forceinline__ static int value_swap(int row) { return !DIRECT ? 0 : D == 64 ? (row & 2) << 1 : (row & 3) << 2; }
    static constexpr int LDS = 2 * BUF;
    static constexpr int PPR = D * SIZE / 16;          // 16-byte pieces of a row
    static constexpr int PIECES = KB * PPR;            // ... of a tile
    static constexpr int PT = PIECES / T;              // ... of a thread
    static_assert(PIECES % T == 0, "");
    static constexpr int KPW = 64 / PPR;               // keys that a wave's 64 pieces hold
    // (half the waves' sums pass through the tiles' memory)
    static_assert(NB == 1 || NW / 2 * 64 * (D / 32) * 16 * 4 <= LDS, "");
};

// 16 bytes from each lane's address to lane * 16 bytes from `lds` on, without
// a register in between.  The wave waits for them by vmcnt; the compiler does
// not know of them, and would wait for all of them before any read of LDS if
// it did.  (M0 is set where it is used, and nothing else in these kernels
// reads it.)
__device__ __forceinline__ void load_to_lds(const unsigned char *from, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "memory");
}

template <int TY, int D, bool TWO>
__device__ __forceinline__ void wide_body(const PagedArgs &a, Common &sh, unsigned char *smem, int slot, int me, bool own)
{
    using S = WideShape<TY, D>;
    constexpr int NMB = D / 32;
    const int tid = threadIdx.x, w = uniform(tid >> 6), lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    Run run;
    run.at = run.end = -1;

    for (;;) {
        Rows rows;
        int u0, u1;
        Sink sink;
        if (slot < a.prefix_slots) {
            const int tile = slot % a.prefix_tiles, gs = slot / a.prefix_tiles, split = gs % a.prefix_splits;
            rows.prefix = true;
            rows.b = 0;
            rows.g = gs / a.prefix_splits;
            rows.row0 = tile * a.prefix_tile;
            rows.n = min(a.prefix_tile, a.prefix_rows - rows.row0);
            u0 = (int)((int64_t)split * a.prefix_units / a.prefix_splits);
            u1 = (int)((int64_t)(split + 1) * a.prefix_units / a.prefix_splits);
            sink = Sink{false, nullptr, a.prefix_parts + (int64_t)slot * a.prefix_tile * (D + 4)};
            slot += a.grid;
        } else {
            if (run.at < 0) {
                if (!own || !find_run<S::NW>(a, sh, me, false, true, run)) return;
            } else {
                if (run.at >= run.end) return;
                next_item(a, run.it);
            }
            u0 = run.at - run.it.first;
            u1 = min(run.it.units, run.end - run.it.first);
            rows = rows_of(a, run.it);
            sink = sink_of(a, D, run, u0, u1, a.own_tile);
            run.at = run.it.first + u1;
        }
        const int g = rows.g, cost = rows.prefix ? 0 : a.item_cost;
        // row blocks (a power of two), waves of a row block, this wave's of each
        const int wr = rows.n <= 32 ? 1 : rows.n <= 64 ? 2 : 4, wk = min(S::NB, S::NW / wr);
        const int rb = w & (wr - 1), kp = w / wr;
        const bool on = kp < wk && 32 * rb < rows.n;

        __syncthreads();  // (the last item's readers of LDS are done)
        {
            const int last = tid < rows.n ? rows.last(a, tid) : -1;
            if (tid < S::ROWS) sh.lim[tid] = last;
            int lo = last < 0 ? kNoToken : last, hi = last;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                lo = min(lo, __shfl_xor(lo, o, 64));
                hi = max(hi, __shfl_xor(hi, o, 64));
            }
            if (lane == 0) {
                sh.lo[w] = lo;
                sh.hi[w] = hi;
            }
        }
        Frag<bf16_t, D> fq;
        {
            int b, t, h;
            rows.of(a, min(32 * rb + l32, rows.n - 1), b, t, h);
            fq.load(static_cast<const bf16_t *>(a.Q) + (((int64_t)b * a.n_q + t) * a.n_heads + h) * D, hh);
        }
        __syncthreads();
        int lo = sh.lo[0], hi = sh.hi[0];
#pragma unroll
        for (int v = 1; v < S::ROWS / 64; ++v) {
            lo = min(lo, sh.lo[v]);
            hi = max(hi, sh.hi[v]);
        }
        lo = uniform(lo);
        hi = uniform(hi);
        const int lim = sh.lim[32 * rb + l32], last = lim < 0 ? hi : lim;

        float m_run = -INFINITY, l_run = 0.f;
        f32x16_t acc[NMB];
#pragma unroll
        for (int mb = 0; mb < NMB; ++mb) acc[mb] = f32x16_t{};
        const float c2 = a.scale * 1.4426950408889634f * (a.k_scale ? a.k_scale[g] : 1.f);

        const int base = rows.prefix ? 0 : a.n_prefix;
        const int n_pos = hi < base ? 0 : hi - base + 1;
        const int p0 = (int)min((int64_t)max(u0 - cost, 0) * kPagedUnit, (int64_t)n_pos);
        const int p1 = (int)min((int64_t)max(u1 - cost, 0) * kPagedUnit, (int64_t)n_pos);

        for (int pa = p0; pa < p1; pa += a.batch_keys) {
            const int pb = min(p1 - pa, a.batch_keys) + pa;
            const int ch0 = a.pd.div(base + pa), ch1 = a.pd.div(base + pb - 1);
            __syncthreads();
            {
                const int32_t *src = rows.prefix ? a.prefix_pages : a.table + (int64_t)rows.b * a.max_pages;
                bool bad = false;
                for (int c = ch0 + tid; c <= ch1; c += S::T) {
                    const int x = pool_page(src[c], a.n_pages);
                    sh.phys[c - ch0] = x;
                    bad = bad || x < 0;
                }
                const uint64_t any = __ballot(bad);
                if (lane == 0) sh.bad[w] = any != 0ull;
            }
            __syncthreads();
            int bad = 0;
#pragma unroll
            for (int v = 0; v < S::NW; ++v) bad |= sh.bad[v];
            const bool holes = uniform(bad) != 0;
            auto there = [&](int tok) { return sh.phys[a.pd.div(tok) - ch0] >= 0; };

            // The keys of a wave's pieces (KPW of them at a time) lie in one
            // page where pages and the first token are multiples of KPW: then
            // a page is looked up once a wave, and a lane adds its own constant
            const bool together = a.pd.page % S::KPW == 0 && base % S::KPW == 0;
            const unsigned char *Kb = static_cast<const unsigned char *>(a.K), *Vb = static_cast<const unsigned char *>(a.V);
            // each(q, first byte of the piece's row, its row in the tile, its
            // chunk, whether some row sees it) for this thread's pieces
            auto pieces = [&](int p, auto each) __attribute__((always_inline)) {
#pragma unroll
                for (int q = 0; q < S::PT; ++q) {
                    const int x = tid + q * S::T, key = x / S::PPR, c = x % S::PPR;
                    int64_t row;
                    bool seen;
                    if (together) {
                        const int key0 = (w * 64 + q * S::T) / S::PPR;  // (the wave's first)
                        const int tok = base + min(p + key0, pb - 1), ch = a.pd.div(tok), phys = uniform(sh.phys[ch - ch0]);
                        const int place = tok - ch * a.pd.page & ~(S::KPW - 1);
                        row = pool_row(max(phys, 0), a.n_kv_heads, g, a.pd.page, place, D) * S::SIZE +
                              lane / S::PPR * (D * S::SIZE);
                        seen = p + key < pb && phys >= 0;
                    } else {
                        const int tok = base + min(p + key, pb - 1), ch = a.pd.div(tok);
                        int phys = sh.phys[ch - ch0], place = tok - ch * a.pd.page;
                        seen = p + key < pb && phys >= 0;
                        if (phys < 0) phys = place = 0;  // (row 0 of the pool is there)
                        row = pool_row(phys, a.n_kv_heads, g, a.pd.page, place, D) * S::SIZE;
                    }
                    each(q, row, key, c, seen);
                }
            };
            u32x4_t kr[S::DIRECT ? 1 : S::PT], vr[S::DIRECT ? 1 : S::PT];
            uint32_t keep = 0;  // bit q: some row sees this thread's piece q
            const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
            auto load = [&](int p, int buf) __attribute__((always_inline)) {
                keep = 0;
                pieces(p, [&](int q, int64_t row, int key, int c, bool seen) __attribute__((always_inline)) {
                    if constexpr (S::DIRECT) {
                        const uint32_t at = lds0 + buf * S::BUF + (w * 64 + q * S::T) * 16;
                        load_to_lds(Kb + row + 16 * (c ^ S::key_swap(key)), at);
                        load_to_lds(Vb + row + 16 * (c ^ S::value_swap(key)), at + S::KB * S::KRS);
                    } else {
                        keep |= (uint32_t)seen << q;
                        kr[q] = *reinterpret_cast<const u32x4_t *>(Kb + row + 16 * c);
                        vr[q] = *reinterpret_cast<const u32x4_t *>(Vb + row + 16 * c);
                    }
                });
            };
            auto store = [&](int buf) __attribute__((always_inline)) {
                if constexpr (S::DIRECT) {
                    wait_vm();
                } else {
#pragma unroll
                    for (int q = 0; q < S::PT; ++q) {
                        const int x = tid + q * S::T, key = x / S::PPR, c = x % S::PPR;
                        unsigned char *kd = smem + buf * S::BUF + key * S::KRS;
                        unsigned char *vd = smem + buf * S::BUF + S::KB * S::KRS + key * S::VRS;
                        // (a value that no row sees is 0: memory that was never written may hold NaN)
#pragma unroll
                        for (int e = 0; e < 4; ++e) vr[q][e] = (keep >> q) & 1u ? vr[q][e] : 0u;
                        *reinterpret_cast<bf16x8_t *>(kd + 32 * c) = e4m3_to_bf16(kr[q][0], kr[q][1]);
                        *reinterpret_cast<bf16x8_t *>(kd + 32 * c + 16) = e4m3_to_bf16(kr[q][2], kr[q][3]);
                        *reinterpret_cast<bf16x8_t *>(vd + 32 * c) = e4m3_to_bf16(vr[q][0], vr[q][1]);
                        *reinterpret_cast<bf16x8_t *>(vd + 32 * c + 16) = e4m3_to_bf16(vr[q][2], vr[q][3]);
                    }
                }
            };
            // ... the same where the rows are in LDS already
            auto clear = [&](int p, int buf) {
                const u32x4_t z = {0u, 0u, 0u, 0u};
                unsigned char *vt = smem + buf * S::BUF + S::KB * S::KRS;
                for (int x = tid; x < S::KB * (D / 8); x += S::T) {
                    const int key = x / (D / 8);
                    if (p + key >= pb || (holes && !there(base + p + key)))
                        *reinterpret_cast<u32x4_t *>(vt + key * S::VRS + 16 * (x % (D / 8))) = z;
                }
            };
            // one 32-key block of a staged tile; MASKED: some row does not see
            // some key of it
            auto block = [&](auto masked, const unsigned char *kt, int p, int kb) __attribute__((always_inline)) {
                constexpr bool MASKED = decltype(masked)::value;
                // (what follows from the lane is worked out again for masked
                // blocks, where it would cost registers from before the loop)
                int own_lane = threadIdx.x & 63;
                if constexpr (MASKED) asm volatile("" : "+v"(own_lane));
                const int lane = own_lane, l32 = lane & 31, hh = lane >> 5;
                const unsigned char *vt = kt + S::KB * S::KRS;
                // (operands are read two products ahead, in this order: left alone
                // the compiler reads each right before its product, which then
                // waits the LDS latency every time)
                const unsigned char *krow = kt + (32 * kb + l32) * S::KRS;
                auto key = [&](int q) {
                    return *reinterpret_cast<const bf16x8_t *>(krow + 16 * ((hh * (D / 16) + q) ^ S::key_swap(l32)));
                };
                f32x16_t s = {};
                bf16x8_t kf[3];
#pragma unroll
                for (int q = 0; q < 2; ++q) kf[q] = key(q);
#pragma unroll
                for (int q = 0; q < D / 16; ++q) {
                    if (q + 2 < D / 16) kf[(q + 2) % 3] = key(q + 2);
                    __builtin_amdgcn_sched_barrier(0);
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[q % 3], fq.v[q], s, 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
                // V^T operand i = NMB s2 + mb of the block: keys 16 s2 + 4 hh + 0..3
                // and + 8..11, the order of the score accumulator
                const int j = lane & 15;
                const unsigned char *vrow = vt + (32 * kb + 4 * hh + (j >> 2)) * S::VRS + 8 * (j & 1);
                auto value = [&](int i) {
                    const int c = (4 * (i % NMB) + 2 * (l32 >> 4) + ((j & 3) >> 1)) ^ S::value_swap(j >> 2);
                    const unsigned char *x = vrow + 16 * (i / NMB) * S::VRS + 16 * c;
                    return join8(lds_read_tr16(x), lds_read_tr16(x + 8 * S::VRS));
                };
                bf16x8_t vf[3];
                vf[0] = value(0);
                vf[1] = value(1);
                __builtin_amdgcn_sched_barrier(0);
                uint32_t seen = 0u;  // bit r: this lane's row sees key acc_row(r, hh)
                if constexpr (MASKED) {
#pragma unroll 1
                    for (int r = 0; r < 16; ++r) {
                        const int x = p + 32 * kb + acc_row(r, hh), tok = base + x;
                        const bool is = x < pb && tok <= last && (!holes || there(tok));
                        seen |= (uint32_t)is << r;
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = (seen >> r) & 1u ? s[r] : -INFINITY;
                }
                float mx = s[0];
#pragma unroll
                for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
                mx *= c2;
                if (__ballot(mx > m_run + kLazy) != 0ull) {  // (the maximum moves rarely, as in the narrow body)
                    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                    const float m_new = fmaxf(m_run, mx);
                    const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
                    l_run *= alpha;
#pragma unroll
                    for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[mb][r] *= alpha;
                    m_run = m_new;
                }
                const float m_use = m_run == -INFINITY ? 0.f : m_run;
                bf16x8_t pw[2], rest[2];
                float l = 0.f;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * q + e], c2, -m_use));
                        l += x[e];
                        if constexpr (!TWO) pw[q][e] = (__bf16)x[e];
                    }
                    if constexpr (TWO) split_weights(x, pw[q], rest[q]);
                }
                l_run += l;
#pragma unroll
                for (int i = 0; i < 2 * NMB; ++i) {
                    if (i + 2 < 2 * NMB) vf[(i + 2) % 3] = value(i + 2);
                    __builtin_amdgcn_sched_barrier(0);
                    bf16x8_t v = vf[i % 3], odd;
                    bool any_odd = false;  // (uniform)
                    if constexpr (MASKED) {
                        uint32_t found = 0;
#pragma unroll
                        for (int e = 0; e < 4; ++e) find_odd<CACHE_BF16>(__builtin_bit_cast(u32x4_t, v)[e], found);
                        any_odd = __ballot(found != 0) != 0ull;
                        if (any_odd) take_odd(v, odd);
                    }
                    f32x16_t &o = acc[i % NMB];
                    o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pw[i / NMB], o, 0, 0, 0);
                    if constexpr (TWO) o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, rest[i / NMB], o, 0, 0, 0);
                    if (MASKED && any_odd) {
                        bf16x8_t see;
#pragma unroll
                        for (int e = 0; e < 8; ++e) see[e] = (seen >> (8 * (i / NMB) + e)) & 1u ? (__bf16)1.f : (__bf16)0.f;
                        const f32x16_t z = {};
                        const f32x16_t k = __builtin_amdgcn_mfma_f32_32x32x16_bf16(odd, see, z, 0, 0, 0);
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[r] = k[r] > 0.f ? NAN : o[r];
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            // tiles that every row sees whole, then the others
            const int open = holes ? pa : max(pa, min(pb, lo - base + 1) - (min(pb, lo - base + 1) - pa) % S::KB);
            load(pa, 0);
            store(0);
            __syncthreads();
            int cur = 0, p = pa;
            auto tiles = [&](auto masked, int end) __attribute__((always_inline)) {
                for (; p < end; p += S::KB, cur ^= 1) {
                    const bool more = p + S::KB < pb;
                    if (more) load(p + S::KB, cur ^ 1);
                    if (S::DIRECT && decltype(masked)::value && (holes || p + S::KB > pb)) {  // (uniform)
                        clear(p, cur);
                        __syncthreads();
                    }
                    if (on) {
                        const unsigned char *kt = smem + cur * S::BUF;
                        for (int kb = kp; kb < S::NB && p + 32 * kb < pb; kb += wk) block(masked, kt, p, kb);
                    }
                    if (more) store(cur ^ 1);
                    __syncthreads();
                }
            };
            tiles(std::false_type(), open);
            tiles(std::true_type(), pb);
        }

        // ------------------------------------------------- the result written
        const bool within = a.prefix_items == 0 && !a.join_apart;  // the parts are joined within this launch
        l_run += __shfl_xor(l_run, 32, 64);
        // (scores that are all NaN leave no maximum, but their sum counts)
        m_run = lim < 0 ? -INFINITY : l_run != l_run ? 0.f : m_run;
        l_run = lim < 0 ? 0.f : l_run;
        // a row that sees no token went along as one that sees all of the item's,
        // of which some may not be finite: 0 times those would not be 0
        if (__ballot(lim < 0) != 0ull) {
#pragma unroll
            for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[mb][r] = lim < 0 ? 0.f : acc[mb][r];
        }
        __syncthreads();
        if (wk == 2) {  // (uniform) the second wave of a row block hands its sums to the first
            f32x4_t *ob = reinterpret_cast<f32x4_t *>(smem) + rb * (64 * NMB * 4) + lane;
            if (on && kp == 1) {
#pragma unroll
                for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        ob[(4 * mb + q) * 64] =
                            f32x4_t{acc[mb][4 * q], acc[mb][4 * q + 1], acc[mb][4 * q + 2], acc[mb][4 * q + 3]};
                if (hh == 0) {
                    sh.m[rb][l32] = m_run;
                    sh.l[rb][l32] = l_run;
                }
            }
            __syncthreads();
            if (on && kp == 0) {
                const float m1 = sh.m[rb][l32], m = fmaxf(m_run, m1);
                const float w0 = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m);
                const float w1 = m1 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m1 - m);
#pragma unroll
                for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x4_t y = ob[(4 * mb + q) * 64];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            acc[mb][4 * q + i] = __builtin_fmaf(w1, y[i], w0 * acc[mb][4 * q + i]);
                    }
                l_run = w0 * l_run + w1 * sh.l[rb][l32];
                m_run = m;
            }
        }
        const int r = 32 * rb + l32;
        if (on && kp == 0 && r < rows.n) {
            int b, t, h;
            rows.of(a, r, b, t, h);
            const int64_t orow = ((int64_t)b * a.n_q + t) * a.n_heads + h;
            const float inv = inverse_sum(l_run, a.v_scale ? a.v_scale[g] : 1.f);
            float *part = sink.part(D, r, orow);
#pragma unroll
            for (int mb = 0; mb < NMB; ++mb) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int f = 32 * mb + 8 * q + 4 * hh;
                    const f32x4_t x = {acc[mb][4 * q], acc[mb][4 * q + 1], acc[mb][4 * q + 2], acc[mb][4 * q + 3]};
                    if (sink.last_word)
                        write_four<false>(a.O, orow * D + f, x * inv);
                    else
                        store_part<D>(a, part + f, x, within);
                }
            }
            if (hh == 0) {
                if (!sink.last_word) {
                    store_part<D>(a, part + D, f32x4_t{m_run, l_run, 0.f, 0.f}, within);
                } else if (a.lse) {
                    a.lse[orow] = log_sum(m_run, l_run);
                }
            }
        }
        if (within && (u0 != 0 || u1 != run.it.units))
            join_cut<D, false, S::NW>(a, sh, smem, run, rows, a.own_tile);
    }
}

// The bodies of a launch one after the other: WIDE for the items of many
// rows (TWO: with two numbers a weight), NR > 0 (16-row blocks) for the others.
template <int TY, int D, bool WIDE, int NR>
struct Launch {
    static constexpr int NW = WIDE ? WideShape<TY == CACHE_F32 ? CACHE_BF16 : TY, D>::NW : 4;
    static constexpr int NARROW = NR > 0 ? NW * Shape<TY, D>::WAVE : 0;
    static constexpr int WIDTH = WIDE ? WideShape<TY == CACHE_F32 ? CACHE_BF16 : TY, D>::LDS : 0;
    static constexpr int LDS = NARROW > WIDTH ? NARROW : WIDTH;
};

template <int TY, int D, bool WIDE, int NR, bool TWO>
__global__ __launch_bounds__((64 * Launch<TY, D, WIDE, NR>::NW), (D <= 128 && NR <= 1 ? 2 : 1)) void paged_kernel(PagedArgs a)
{
    constexpr int NW = Launch<TY, D, WIDE, NR>::NW;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ Common sh;
    // A wide prefix's length is known to the host, which cuts it into splits:
    // slot (key head, split, row tile), the tiles of a split next to each
    // other and so on one XCD (workgroups are dealt to the eight round-robin),
    // where they read the same keys at about the same time from its L2.  Runs
    // begin at the workgroups that the slots leave free.
    int slot = blockIdx.x, me = blockIdx.x;
    if constexpr (WIDE) {
        if ((a.grid & 7) == 0) slot = (blockIdx.x & 7) * (a.grid >> 3) + (blockIdx.x >> 3);
        me = slot - a.prefix_slots % a.grid;
        me += me < 0 ? a.grid : 0;
    }
    if constexpr (WIDE) wide_body<TY, D, TWO>(a, sh, smem, slot, me, NR == 0);
    if constexpr (NR > 0) narrow_body<TY, D, NR, NW>(a, sh, smem, me, !WIDE && a.prefix_items > 0, true);
}

template <int TY, int D, bool WIDE, int NR, bool TWO>
hipError_t launch_one(const PagedArgs &a, hipStream_t stream)
{
    using L = Launch<TY, D, WIDE, NR>;
    static LdsLimit seen;
    const void *fn = reinterpret_cast<const void *>(&paged_kernel<TY, D, WIDE, NR, TWO>);
    hipError_t e = raise_lds_limit(fn, L::LDS + sizeof(Common), seen);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((paged_kernel<TY, D, WIDE, NR, TWO>), dim3((unsigned)a.grid), dim3(64 * L::NW), L::LDS, stream, a);
    return hipGetLastError();
}

template <int TY, int D>
hipError_t launch_d(const PagedArgs &a, hipStream_t stream)
{
    if constexpr (TY == CACHE_F32) {
        return a.own_tile == 16 ? launch_one<TY, D, false, 1, false>(a, stream) : launch_one<TY, D, false, 2, false>(a, stream);
    } else {
        if (!a.own_wide && !a.prefix_wide) return launch_one<TY, D, false, 1, false>(a, stream);
        if (a.own_wide)
            return a.two_weights ? launch_one<TY, D, true, 0, true>(a, stream) : launch_one<TY, D, true, 0, false>(a, stream);
        return a.two_weights ? launch_one<TY, D, true, 1, true>(a, stream) : launch_one<TY, D, true, 1, false>(a, stream);
    }
}

}  // namespace paged
}  // namespace rr
