// Attention of the newest tokens of a batch of sequences over a paged cache
// (all of it, along routes of pages, or behind a shared prefix), for gfx950.
//
//   o = sum_u 2^(c q.k_u - m) v_u / l,  l = sum_u 2^(c q.k_u - m),  c = scale log2 e
//
// One pass over the keys with a running maximum m per query.  A call's work
// is cut into items: the query rows of one (sequence, key head) -- n_q tokens
// times the heads that share the key head -- in tiles of 16 * NR rows; with
// routes one query head's row, which has its own pages; with a shared prefix
// also tiles over the rows of the whole batch against the prefix, which is
// what reads it once for many sequences.  Every item is a number of units of
// 128 keys, and the units of all items, in order, are cut into equal runs,
// one per workgroup: lengths that differ a hundredfold leave no compute unit
// idle, and one long sequence is spread over the card.  Lengths live on the
// device, so every workgroup sums them to find its run.  An item that lies in
// several runs leaves a part (m, l, sum) per run in the workspace; a second
// launch joins them.
//
// Within a workgroup each of four waves takes its own 32-key tiles (16 in
// binary32) of the run: no barrier stands between loads and products, and a
// tile's 16 KB of keys and values is requested while the tile before it is
// still in its softmax.  S^T = K Q^T on 16x16 MFMA tiles with the keys as
// rows, so K goes from memory to the operand registers as it lies (a lane
// holds 16 bytes of one key); a lane then has four scores of one query per
// tile, which are just the keys that its part of the operand of O^T = V^T P^T
// takes.  V is transposed on the way: row-major into a buffer of the wave's
// own in LDS, read with the LDS transpose read; in binary32, where an operand
// holds one key per lane, straight from memory.
#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>

#include "rr_device.hpp"
#include "rr_internal.hpp"
#include "rr_paged.hpp"

namespace rr {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short short4_t __attribute__((ext_vector_type(4)));

constexpr int kT = 256;             // threads of a workgroup
constexpr int kW = kT / 64;         // waves
constexpr int kUnit = 128;          // keys of a unit of work
constexpr int kStagedPages = 1024;  // page numbers held in LDS at a time
constexpr float kLazy = 8.f;        // log2 headroom of the running softmax maximum
constexpr int kMostGrid = 1024;     // workgroups of a launch at most
constexpr int32_t kNoToken = INT_MAX;

// Four bf16 of a transposed LDS read (ds_read_b64_tr_b16): lane i of each
// 16-lane group receives column i of the four rows that its lanes address,
// lane j the 8 bytes of row j / 4 at columns 4 (j % 4).
__device__ __forceinline__ short4_t lds_read_tr16(const unsigned char *p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t *)p);
}

__device__ __forceinline__ bf16x8_t as_bf16x8(u32x4_t x) { return __builtin_bit_cast(bf16x8_t, x); }

// Eight e4m3 values, exactly, as bf16.
__device__ __forceinline__ bf16x8_t e4m3_to_bf16(uint32_t lo, uint32_t hi)
{
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
    const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
    const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u; }

// What a cache type's tiles look like.
//   KT     keys of a wave's tile
//   KR     rows (keys) of a tile that a lane loads 16-byte pieces of
//   PK     such pieces of a row and lane: piece c, lane group kg holds the
//          row's elements from (c * 4 + kg) * (16 / size)
template <int TY, int D>
struct Shape {
    static constexpr int SIZE = TY == CACHE_F32 ? 4 : TY == CACHE_BF16 ? 2 : 1;
    static constexpr int KT = TY == CACHE_F32 ? 16 : 32;
    static constexpr int KR = KT / 16;
    static constexpr int PK = D * SIZE / 64;
    static constexpr int VRS = 2 * D + 64;   // bytes of a row of the V buffer
    static constexpr int ORS = D + 4;        // floats of a row of the output buffer
    static constexpr int VBYTES = TY == CACHE_F32 ? 0 : KT * VRS;
    static constexpr int OBYTES = 16 * ORS * 4;
    static constexpr int WAVE = VBYTES > OBYTES ? VBYTES : OBYTES;
    static constexpr int LDS = kW * WAVE;
};

// A run's position: the item that unit `at` falls into.
struct Item {
    bool prefix;
    int32_t b;          // sequence
    int32_t j;          // item within the sequence (or within the prefix)
    int32_t units;      // its units
    int64_t first;      // its first unit
    int64_t index;      // its number
};

__device__ __forceinline__ int32_t seq_units(const PagedArgs &a, int32_t b)
{
    if (a.route_units) return a.route_units;
    const int32_t n = held_tokens(a.lengths[b], a.capacity) - a.n_prefix;
    return n <= kUnit ? 1 : (n + kUnit - 1) / kUnit;
}

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

template <int TY, int D, int NR>
__global__ __launch_bounds__(kT, NR == 1 && D <= 128 ? 2 : 1) void paged_kernel(PagedArgs a)
{
    using S = Shape<TY, D>;
    constexpr bool F32 = TY == CACHE_F32;
    constexpr int NV = D / 16;  // value accumulators of a row block
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int32_t s_phys[kStagedPages];
    __shared__ int32_t s_chunk[kMaxAttnSlots];
    __shared__ int64_t s_sum[kW];
    __shared__ int64_t s_at[3];
    __shared__ int32_t s_b;
    __shared__ int32_t s_wn[kW];
    __shared__ float s_m[kW][16], s_l[kW][16];

    const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, l16 = lane & 15, kg = lane >> 4;
    unsigned char *vbuf = smem + w * S::WAVE;

    // ---- the run of this workgroup: units [at, end) of all items'
    const int64_t prefix_total = (int64_t)a.prefix_items * a.prefix_units;
    {
        const int per = (a.n_seqs + kT - 1) / kT;
        const int b0 = min(tid * per, a.n_seqs), b1 = min(b0 + per, a.n_seqs);
        int64_t sum = 0;
        for (int b = b0; b < b1; ++b) sum += seq_units(a, b);
        int64_t inc = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t v = (int64_t)shfl_u64((uint64_t)inc, max(lane - o, 0));
            inc += lane >= o ? v : 0;
        }
        if (lane == 63) s_sum[w] = inc;
        __syncthreads();
        int64_t before = inc - sum, all = 0;
        for (int v = 0; v < kW; ++v) {
            before += v < w ? s_sum[v] : 0;
            all += s_sum[v];
        }
        const int64_t total = prefix_total + all * a.items_per_seq;
        const int64_t share = (total + a.grid - 1) / a.grid, per_wg = share > a.min_units ? share : a.min_units;
        const int64_t at = blockIdx.x * per_wg, end = min(at + per_wg, total);
        if (at >= end) return;  // (uniform)
        if (tid == 0) {
            s_at[0] = per_wg;
            s_at[1] = total;
        }
        // the sequence that the run begins in (0 where it begins in the prefix)
        const int64_t u = max(at - prefix_total, (int64_t)0) / a.items_per_seq;
        if (u >= before && u < before + sum) {
            int b = b0;
            int64_t base = before;
            for (;;) {
                const int32_t n = seq_units(a, b);
                if (u < base + n) break;
                base += n;
                ++b;
            }
            s_b = b;
            s_at[2] = base;
        }
    }
    __syncthreads();
    const int64_t per_wg = s_at[0];
    int64_t at = blockIdx.x * per_wg;
    const int64_t end = min(at + per_wg, s_at[1]);
    Item it;
    it.prefix = at < prefix_total;
    it.b = s_b;
    if (it.prefix) {
        it.units = a.prefix_units;
        it.j = (int32_t)(at / it.units);
        it.index = it.j;
        it.first = it.index * it.units;
    } else {
        const int64_t base = prefix_total + s_at[2] * a.items_per_seq;
        it.units = seq_units(a, it.b);
        it.j = (int32_t)((at - base) / it.units);
        it.index = a.prefix_items + (int64_t)it.b * a.items_per_seq + it.j;
        it.first = base + (int64_t)it.j * it.units;
    }
    const int64_t run0 = at;

    while (at < end) {
        // ---------------------------------------------- the item and its rows
        const int u0 = (int)(at - it.first), u1 = (int)min((int64_t)it.units, end - it.first);
        const int group = a.group, per_b = a.n_q * group;
        int g, row0, rows, b_item = it.b;
        if (it.prefix) {
            g = it.j / a.prefix_tiles;
            row0 = (it.j - g * a.prefix_tiles) * 16 * NR;
            rows = min(16 * NR, a.prefix_rows - row0);
        } else if (a.route_units) {
            // item = head * n_q + query token: row t * group + j of its key head
            const int h = it.j / a.n_q, t = it.j - h * a.n_q;
            g = h / group;
            row0 = t * group + (h - g * group);
            rows = 1;
        } else {
            g = it.j / a.row_tiles;
            row0 = (it.j - g * a.row_tiles) * 16 * NR;
            rows = min(16 * NR, a.rows - row0);
        }
        const int blocks = (rows + 15) >> 4;
        // row r of the item: sequence, query token and head
        auto row_of = [&](int r, int &b, int &t, int &h) {
            int x = row0 + r;
            b = b_item;
            if (it.prefix) {
                b = x / per_b;
                x -= b * per_b;
            }
            t = x / group;
            h = g * group + (x - t * group);
        };

        // query operands; lim: the last token that a row sees (-1: none);
        // rows that see nothing, and rows past the item's, take no part in
        // lo and hi, the least and the largest of them
        bf16x8_t fq[F32 ? 1 : NR][F32 ? 1 : D / 32];
        f32x4_t fqf[F32 ? NR : 1][F32 ? D / 16 : 1];
        int lim[NR], lo = kNoToken, hi = -1;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            int b, t, h;
            const int r = 16 * n + l16;
            row_of(min(r, rows - 1), b, t, h);
            const int last = held_tokens(a.lengths[b], a.capacity) - a.n_q + t;
            lim[n] = r < rows ? (it.prefix ? min(last, a.n_prefix - 1) : last) : -1;
            if (lim[n] >= 0) {
                lo = min(lo, lim[n]);
                hi = max(hi, lim[n]);
            }
            const int64_t q = (((int64_t)b * a.n_q + t) * a.n_heads + h) * D;
            const bool on = r < rows;
            if constexpr (F32) {
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    const f32x4_t x = *reinterpret_cast<const f32x4_t *>(static_cast<const float *>(a.Q) + q + 16 * c + 4 * kg);
                    fqf[n][c] = on ? x : f32x4_t{0.f, 0.f, 0.f, 0.f};
                }
            } else {
                const u32x4_t z = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    // (e4m3 keys come 16 to a piece, two operands of 8)
                    const int f = TY == CACHE_E4M3 ? 64 * (c >> 1) + 16 * kg + 8 * (c & 1) : 32 * c + 8 * kg;
                    const u32x4_t x = *reinterpret_cast<const u32x4_t *>(static_cast<const bf16_t *>(a.Q) + q + f);
                    fq[n][c] = as_bf16x8(on ? x : z);
                }
            }
        }
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) {
            lo = min(lo, __shfl_xor(lo, o, 64));
            hi = max(hi, __shfl_xor(hi, o, 64));
        }

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

        // ------------------------------------------------ the keys of the run
        // Positions: tokens from `base` on, or, along routes, the places of
        // the listed pages one after the other.
        const int base = it.prefix ? 0 : a.n_prefix;
        int n_pos;
        __syncthreads();  // (the last item's readers of LDS are done)
        if (a.route_units) {
            // the pages that the row sees, each once: a slot is dropped if an
            // earlier one names its page
            const int64_t row = ((int64_t)it.b * a.items_per_seq + it.j) * a.k;
            const int here = hi >= 0 ? a.pd.div(hi) : -1, slots = a.n_sink + a.n_recent + a.k;
            static_assert(kMaxAttnSlots <= kT, "a slot per thread");
            int id = -1;
            if (tid < a.n_sink)
                id = tid;
            else if (tid < a.n_sink + a.n_recent)
                id = here - (tid - a.n_sink);
            else if (tid < slots)
                id = a.routes[row + tid - a.n_sink - a.n_recent];
            bool ok = tid < slots && id >= 0 && id <= here;
            if (tid < kMaxAttnSlots) s_phys[tid] = ok ? id : -1;
            __syncthreads();
            if (ok)
                for (int s = 0; s < tid; ++s) ok = ok && s_phys[s] != id;
            const uint64_t mk = __ballot(ok);
            if (lane == 0) s_wn[w] = __popcll(mk);
            __syncthreads();
            int pre = __popcll(mk & ((1ull << lane) - 1ull)), all = 0;
            for (int v = 0; v < kW; ++v) {
                pre += v < w ? s_wn[v] : 0;
                all += s_wn[v];
            }
            if (ok) {
                s_chunk[pre] = id;
                s_phys[pre] = pool_page(a.table[(int64_t)it.b * a.max_pages + id], a.n_pages);
            }
            n_pos = all * a.pd.page;
        } else {
            n_pos = hi < base ? 0 : hi - base + 1;
        }
        const int p0 = (int)min((int64_t)u0 * kUnit, (int64_t)n_pos), p1 = (int)min((int64_t)u1 * kUnit, (int64_t)n_pos);

        for (int pa = p0; pa < p1 || (a.route_units && pa == p0); pa += a.batch_keys) {
            // (routes: the page list is staged whole, in one batch)
            const int pb = a.route_units ? p1 : min(p1 - pa, a.batch_keys) + pa;
            const int ch0 = a.route_units ? 0 : a.pd.div(base + pa);
            if (!a.route_units) {
                if (pa != p0) __syncthreads();
                const int ch1 = a.pd.div(base + pb - 1);
                const int32_t *src = it.prefix ? a.prefix_pages : a.table + (int64_t)it.b * a.max_pages;
                for (int c = ch0 + tid; c <= ch1; c += kT) s_phys[c - ch0] = pool_page(src[c], a.n_pages);
            }
            __syncthreads();
            if (pa >= pb) break;

            // where position p lies: its token and page, kNoToken where the
            // page is none or p is past the run
            auto locate = [&](int p, int &phys, int &place) -> int32_t {
                const bool in = p < pb;
                p = min(p, pb - 1);
                int tok;
                if (a.route_units) {
                    const int s = a.pd.div(p);
                    place = p - s * a.pd.page;
                    phys = s_phys[s];
                    tok = s_chunk[s] * a.pd.page + place;
                } else {
                    tok = base + p;
                    const int c = a.pd.div(tok);
                    place = tok - c * a.pd.page;
                    phys = s_phys[c - ch0];
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
            for (; p < pb; p += kW * S::KT) {
                // (wave-uniform) every key of the tile is seen by every row
                bool all_seen = true, mixed = false;
#pragma unroll
                for (int r = 0; r < S::KR; ++r) {
                    all_seen = all_seen && tok[r] <= lo;
                    mixed = mixed || (tok[r] > lo && tok[r] != kNoToken);
                }
                all_seen = __ballot(all_seen) == ~0ull;
                mixed = __ballot(mixed) != 0ull;

                // rows that no query sees become zeros: 0 weights them, but
                // memory that was never written may hold infinities and NaN.
                // In a tile that some rows see and others don't, values that
                // are not finite would come into the others as 0 * inf
                bool odd = false;
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
                                    odd = odd || not_finite(__uint_as_float(vr[0][4 * c + s][e]));
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
                                    const uint32_t x = keep ? vr[r][c][e] : 0u;
                                    vr[r][c][e] = x;
                                    if constexpr (TY == CACHE_BF16)
                                        odd = odd || (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u;
                                    else {
#pragma unroll
                                        for (int q = 0; q < 4; ++q) odd = odd || ((x >> 8 * q) & 0x7Fu) == 0x7Fu;
                                    }
                                }
                            }
                            unsigned char *dst = vbuf + (16 * r + l16) * S::VRS + (TY == CACHE_BF16 ? 64 * c + 16 * kg : 128 * c + 32 * kg);
                            if constexpr (TY == CACHE_BF16) {
                                *reinterpret_cast<u32x4_t *>(dst) = vr[r][c];
                            } else {
                                *reinterpret_cast<bf16x8_t *>(dst) = e4m3_to_bf16(vr[r][c][0], vr[r][c][1]);
                                *reinterpret_cast<bf16x8_t *>(dst + 16) = e4m3_to_bf16(vr[r][c][2], vr[r][c][3]);
                            }
                        }
                    }
                    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
                    __builtin_amdgcn_wave_barrier();
                }
                odd = mixed && __ballot(odd) != 0ull;

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
                            const bf16x8_t kf = as_bf16x8(kr[r][c]);
#pragma unroll
                            for (int n = 0; n < NR; ++n)
                                if (NR == 1 || n < blocks)
                                    s[n][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, fq[n][c], s[n][r], 0, 0, 0);
                        } else {
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                const bf16x8_t kf = e4m3_to_bf16(kr[r][c][2 * q], kr[r][c][2 * q + 1]);
#pragma unroll
                                for (int n = 0; n < NR; ++n)
                                    if (NR == 1 || n < blocks)
                                        s[n][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, fq[n][2 * c + q], s[n][r], 0, 0, 0);
                            }
                        }
                    }
                }
                int32_t seen_tok[S::KR][4];  // token of key 16 r + 4 kg + i
                if (!all_seen) {
#pragma unroll
                    for (int r = 0; r < S::KR; ++r)
#pragma unroll
                        for (int i = 0; i < 4; ++i) seen_tok[r][i] = __shfl(tok[r], 4 * kg + i, 64);
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        const int last = lim[n] < 0 ? hi : lim[n];
#pragma unroll
                        for (int r = 0; r < S::KR; ++r)
#pragma unroll
                            for (int i = 0; i < 4; ++i) s[n][r][i] = seen_tok[r][i] <= last ? s[n][r][i] : -INFINITY;
                    }
                }
                f32x4_t vf[F32 ? D / 16 : 1];
                if constexpr (F32) {
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) vf[c] = __builtin_bit_cast(f32x4_t, vr[0][c]);
                }
                if (p + kW * S::KT < pb) load(p + kW * S::KT);

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
                if (odd) {
                    // a value that is not finite stands where some rows see it
                    // and others don't: key by key, for the rows that see it
                    for (int key = 0; key < S::KT; ++key) {
                        int phys, place;
                        const int32_t t = locate(p + key, phys, place);
                        if (t == kNoToken) continue;  // (uniform)
                        const int64_t o = pool_row(phys, a.n_kv_heads, g, a.pd.page, place, D);
#pragma unroll
                        for (int n = 0; n < NR; ++n) {
                            if (NR > 1 && n >= blocks) continue;
                            float pk = 0.f;
#pragma unroll
                            for (int r = 0; r < S::KR; ++r)
#pragma unroll
                                for (int i = 0; i < 4; ++i) pk = (key >> 4) == r && (key & 3) == i ? s[n][r][i] : pk;
                            pk = __shfl(pk, (((key & 15) >> 2) << 4) + l16, 64);
                            const bool sees = t <= (lim[n] < 0 ? hi : lim[n]);
#pragma unroll
                            for (int v = 0; v < NV; ++v)
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const int64_t e = o + feature_of<TY>(v, i, kg);
                                    float x;
                                    if constexpr (F32)
                                        x = reinterpret_cast<const float *>(Vb)[e];
                                    else if constexpr (TY == CACHE_BF16)
                                        x = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(Vb)[e] << 16);
                                    else
                                        x = (float)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)Vb[e], 1.f, false)[0];
                                    acc[n][v][i] = sees ? __builtin_fmaf(pk, x, acc[n][v][i]) : acc[n][v][i];
                                }
                        }
                    }
                } else if constexpr (F32) {
#pragma unroll
                    for (int c = 0; c < D / 64; ++c)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
#pragma unroll
                                for (int n = 0; n < NR; ++n)
                                    if (NR == 1 || n < blocks)
                                        acc[n][4 * c + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[4 * c + i][e], s[n][0][i],
                                                                                                acc[n][4 * c + e], 0, 0, 0);
                } else {
                    // a weight rounded to one bf16 would add as much error as
                    // the rounding of the output: the rest of it goes through
                    // a second product
                    bf16x8_t ph[NR], pl[NR];
#pragma unroll
                    for (int n = 0; n < NR; ++n)
#pragma unroll
                        for (int r = 0; r < 2; ++r)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float x = s[n][r % S::KR][i];
                                const __bf16 h = (__bf16)x;
                                ph[n][4 * r + i] = h;
                                pl[n][4 * r + i] = (__bf16)(x - (float)h);
                            }
#pragma unroll
                    for (int v = 0; v < NV; ++v) {
                        const unsigned char *vp = vbuf + (4 * kg + (l16 >> 2)) * S::VRS + 2 * (16 * v + 4 * (l16 & 3));
                        const short4_t x = lds_read_tr16(vp), y = lds_read_tr16(vp + 16 * S::VRS);
                        const bf16x8_t vt = __builtin_bit_cast(
                            bf16x8_t, (short __attribute__((ext_vector_type(8)))){x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]});
#pragma unroll
                        for (int n = 0; n < NR; ++n)
                            if (NR == 1 || n < blocks) {
                                acc[n][v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, ph[n], acc[n][v], 0, 0, 0);
                                acc[n][v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pl[n], acc[n][v], 0, 0, 0);
                            }
                    }
                }
            }
        }

        // ------------------------- the waves' sums joined, the result written
        const bool entire = u0 == 0 && u1 == it.units;
        const bool last_word = entire && a.prefix_items == 0;  // no other item has a part in these rows
        const int64_t slot = 2 * (int64_t)blockIdx.x + (at == run0 ? 0 : 1);
        const float vs = a.v_scale ? a.v_scale[g] : 1.f;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            if (n >= blocks) continue;  // (uniform)
            __syncthreads();
            float *ob = reinterpret_cast<float *>(smem + w * S::WAVE);
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
                const bool none = lim[n] < 0;
                // (scores that are all NaN leave no maximum, but their sum counts)
                s_m[w][l16] = none ? -INFINITY : l != l ? 0.f : m_run[n];
                s_l[w][l16] = none ? 0.f : l;
            }
            __syncthreads();
            // 16 threads a row, D / 16 features each in pieces of four
            const int q = tid >> 4, r = 16 * n + q;
            if (r < rows) {
                float m = -INFINITY, sum = 0.f, wt[kW];
#pragma unroll
                for (int v = 0; v < kW; ++v) m = fmaxf(m, s_m[v][q]);
#pragma unroll
                for (int v = 0; v < kW; ++v) {
                    wt[v] = s_m[v][q] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[v][q] - m);
                    sum += wt[v] * s_l[v][q];
                }
                int b, t, h;
                row_of(r, b, t, h);
                const int64_t orow = ((int64_t)b * a.n_q + t) * a.n_heads + h;
                const float inv = sum > 0.f ? vs / sum : sum == 0.f ? 0.f : sum;
                float *part = entire ? a.whole + ((it.prefix ? 0 : (int64_t)a.n_seqs * a.n_q * a.n_heads) + orow) * (D + 4)
                                     : a.parts + (slot * 16 * NR + r) * (D + 4);
#pragma unroll
                for (int f0 = 0; f0 < D / 64; ++f0) {
                    const int f = 64 * f0 + 4 * (tid & 15);
                    f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int v = 0; v < kW; ++v) {
                        const f32x4_t y = *reinterpret_cast<const f32x4_t *>(reinterpret_cast<float *>(smem + v * S::WAVE) + q * S::ORS + f);
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[i] = wt[v] != 0.f ? __builtin_fmaf(wt[v], y[i], x[i]) : x[i];
                    }
                    if (last_word) {
                        if constexpr (F32) {
                            *reinterpret_cast<f32x4_t *>(static_cast<float *>(a.O) + orow * D + f) = x * inv;
                        } else {
                            __bf16 __attribute__((ext_vector_type(4))) y;
#pragma unroll
                            for (int i = 0; i < 4; ++i) y[i] = (__bf16)(x[i] * inv);
                            *reinterpret_cast<uint2 *>(static_cast<bf16_t *>(a.O) + orow * D + f) = __builtin_bit_cast(uint2, y);
                        }
                    } else {
                        *reinterpret_cast<f32x4_t *>(part + f) = x;
                    }
                }
                if ((tid & 15) == 0) {
                    if (!last_word) {
                        part[D] = m;
                        part[D + 1] = sum;
                    } else if (a.lse) {
                        a.lse[orow] = m == -INFINITY ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
                    }
                }
            }
        }
        // the item's head, by the workgroup that holds its first unit
        if (u0 == 0 && tid == 0) {
            const int64_t first_wg = blockIdx.x, last_wg = (it.first + it.units - 1) / per_wg;
            a.heads[it.index] = int4{(int)slot, (int)first_wg, (int)(last_wg - first_wg) + 1, 0};
        }

        // -------------------------------------------------------- the next item
        at = it.first + u1;
        if (at >= end) break;
        it.first += it.units;
        ++it.index;
        ++it.j;
        if (it.prefix) {
            if (it.j == a.prefix_items) {
                it.prefix = false;
                it.j = 0;
                it.b = 0;
                it.units = seq_units(a, 0);
            }
        } else if (it.j == a.items_per_seq) {
            it.j = 0;
            ++it.b;
            it.units = seq_units(a, it.b);
        }
    }
}

// -------------------------------------------------------------------- join
//
// One workgroup per query row.  The row's parts -- of its own item, and of
// the prefix item that holds it -- are added with weights 2^(m_i - m).

template <int D, bool F32>
__global__ __launch_bounds__(kT) void paged_join_kernel(PagedArgs a, bool e4m3)
{
    constexpr int PL = D / 4;      // lanes of a part, four features each
    constexpr int NP = kT / PL;    // parts in flight
    __shared__ float s_w[2 * kMostGrid + 2];
    __shared__ float s_red[kW];
    __shared__ float s_acc[NP][D];
    const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
    const int64_t orow = blockIdx.x;  // (b, t, h)
    const int h = (int)(orow % a.n_heads);
    const int64_t bt = orow / a.n_heads;
    const int t = (int)(bt % a.n_q), b = (int)(bt / a.n_q);
    const int g = h / a.group, j = h - g * a.group;
    const int tile = 16 * a.row_blocks;

    int own_row, item;  // row within its item's tile, item within the sequence
    if (a.route_units) {
        own_row = 0;
        item = h * a.n_q + t;
    } else {
        const int r = t * a.group + j;
        item = g * a.row_tiles + r / tile;
        own_row = r % tile;
    }
    const int4 own = a.heads[a.prefix_items + (int64_t)b * a.items_per_seq + item];
    int n_own = own.z, n_pre = 0, pre_row = 0;
    int4 pre = {0, 0, 0, 0};
    if (a.prefix_items) {
        const int r = b * a.rows + t * a.group + j;
        pre = a.heads[g * a.prefix_tiles + r / tile];
        pre_row = r % tile;
        n_pre = pre.z;
    } else if (n_own == 1) {
        return;  // (uniform) its workgroup wrote the result
    }
    const int64_t n_rows = (int64_t)a.n_seqs * a.n_q * a.n_heads;
    auto part_of = [&](int i) -> const float * {
        const bool p = i >= n_own;
        const int4 &hd = p ? pre : own;
        i = p ? i - n_own : i;
        if (hd.z == 1) return a.whole + ((p ? 0 : n_rows) + orow) * (D + 4);
        const int64_t slot = i == 0 ? hd.x : 2 * (int64_t)(hd.y + i);
        return a.parts + (slot * tile + (p ? pre_row : own_row)) * (D + 4);
    };
    const int n = n_own + n_pre;

    float m = -INFINITY;
    for (int i = tid; i < n; i += kT) {
        const float x = part_of(i)[D];
        s_w[i] = x;
        m = fmaxf(m, x);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    if (lane == 0) s_red[w] = m;
    __syncthreads();
    m = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
    __syncthreads();
    float l = 0.f;
    for (int i = tid; i < n; i += kT) {
        const float x = s_w[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_w[i] - m);
        l += x * part_of(i)[D + 1];
        s_w[i] = x;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) l += __shfl_xor(l, o, 64);
    if (lane == 0) s_red[w] = l;
    __syncthreads();
    l = (s_red[0] + s_red[1]) + (s_red[2] + s_red[3]);

    const int pl = tid % PL, pg = tid / PL;
    f32x4_t x = {0.f, 0.f, 0.f, 0.f};
    for (int i = pg; i < n; i += NP) {
        const float wt = s_w[i];
        const f32x4_t y = *reinterpret_cast<const f32x4_t *>(part_of(i) + 4 * pl);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = wt != 0.f ? __builtin_fmaf(wt, y[e], x[e]) : x[e];
    }
    *reinterpret_cast<f32x4_t *>(&s_acc[pg][4 * pl]) = x;
    __syncthreads();
    const float vs = a.v_scale ? a.v_scale[g] : 1.f, inv = l > 0.f ? vs / l : l == 0.f ? 0.f : l;
    for (int f = tid; f < D; f += kT) {
        float y = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) y += s_acc[i][f];
        y *= inv;
        if constexpr (F32)
            static_cast<float *>(a.O)[orow * D + f] = y;
        else
            static_cast<__bf16 *>(a.O)[orow * D + f] = (__bf16)y;
    }
    if (tid == 0 && a.lse) a.lse[orow] = m == -INFINITY ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

template <int TY, int D, int NR>
hipError_t launch_one(const PagedArgs &a, hipStream_t stream)
{
    static LdsLimit seen;
    const void *fn = reinterpret_cast<const void *>(&paged_kernel<TY, D, NR>);
    hipError_t e = raise_lds_limit(fn, Shape<TY, D>::LDS, seen);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((paged_kernel<TY, D, NR>), dim3((unsigned)a.grid), dim3(kT), (Shape<TY, D>::LDS), stream, a);
    return hipGetLastError();
}

template <int TY, int D>
hipError_t launch_blocks(const PagedArgs &a, hipStream_t stream)
{
    if (a.row_blocks == 1) return launch_one<TY, D, 1>(a, stream);
    if constexpr (D <= 128 && TY != CACHE_F32) {
        if (a.row_blocks == 4) return launch_one<TY, D, 4>(a, stream);
    }
    return launch_one<TY, D, 2>(a, stream);
}

}  // namespace

bool paged_supported(int dtype, int cache, int d)
{
    if (dtype == 0) return cache == CACHE_F32 && (d == 64 || d == 128);
    return (cache == CACHE_BF16 || cache == CACHE_E4M3) && (d == 64 || d == 128 || d == 256);
}

void paged_schedule(PagedArgs &a, int cache, int d)
{
    const int per_b = a.n_q * a.group;
    const bool routed = a.k + a.n_sink + a.n_recent > 0;
    a.rows = routed ? 1 : per_b;
    const int64_t most_rows = a.n_prefix ? (int64_t)a.n_seqs * per_b : a.rows;
    a.row_blocks = most_rows <= 16 ? 1 : most_rows <= 32 || d == 256 || cache == CACHE_F32 ? 2 : 4;
    const int tile = 16 * a.row_blocks;
    a.row_tiles = (a.rows + tile - 1) / tile;
    a.items_per_seq = routed ? a.n_heads * a.n_q : a.n_kv_heads * a.row_tiles;
    a.route_units = 0;
    if (routed) {
        const int64_t slots = (int64_t)a.k + a.n_sink + a.n_recent;
        const int64_t pages = slots < a.max_pages ? slots : a.max_pages;
        a.route_units = (int32_t)((pages * a.pd.page + kUnit - 1) / kUnit);
    }
    a.prefix_rows = a.n_prefix ? (int32_t)most_rows : 0;
    a.prefix_tiles = (a.prefix_rows + tile - 1) / tile;
    a.prefix_items = a.n_kv_heads * a.prefix_tiles;
    a.prefix_units = (a.n_prefix + kUnit - 1) / kUnit;
    const int64_t keys = (int64_t)(kStagedPages - 1) * a.pd.page / kUnit * kUnit;
    a.batch_keys = (int32_t)(keys < (1 << 30) ? keys : (1 << 30));
    a.min_units = 1;
    // units of the longest sequences that the page table can hold
    int64_t most = routed ? a.route_units : (a.capacity + kUnit - 1) / kUnit;
    most = most * a.items_per_seq * a.n_seqs + (int64_t)a.prefix_items * a.prefix_units;
    const int64_t full = 512;
    const int64_t need = (most + a.min_units - 1) / a.min_units;
    a.grid = (int32_t)(need < full ? need : full);
}

static int64_t align256(int64_t n) { return (n + 255) / 256 * 256; }

static int64_t parts_bytes(const PagedArgs &a, int d) { return align256((int64_t)2 * a.grid * 16 * a.row_blocks * (d + 4) * 4); }

static int64_t whole_bytes(const PagedArgs &a, int d)
{
    return a.n_prefix ? align256((int64_t)2 * a.n_seqs * a.n_q * a.n_heads * (d + 4) * 4) : 0;
}

size_t paged_workspace_bytes(const PagedArgs &a, int d)
{
    const int64_t items = a.prefix_items + (int64_t)a.n_seqs * a.items_per_seq;
    return (size_t)(parts_bytes(a, d) + whole_bytes(a, d) + align256(items * 16));
}

void paged_layout(PagedArgs &a, int d, void *workspace)
{
    unsigned char *p = static_cast<unsigned char *>(workspace);
    a.parts = reinterpret_cast<float *>(p);
    p += parts_bytes(a, d);
    a.whole = reinterpret_cast<float *>(p);
    p += whole_bytes(a, d);
    a.heads = reinterpret_cast<int4 *>(p);
}

hipError_t launch_paged(const PagedArgs &a, int cache, int d, hipStream_t stream)
{
    if (cache == CACHE_F32) return d == 64 ? launch_blocks<CACHE_F32, 64>(a, stream) : launch_blocks<CACHE_F32, 128>(a, stream);
    if (cache == CACHE_BF16) {
        if (d == 64) return launch_blocks<CACHE_BF16, 64>(a, stream);
        if (d == 128) return launch_blocks<CACHE_BF16, 128>(a, stream);
        return launch_blocks<CACHE_BF16, 256>(a, stream);
    }
    if (d == 64) return launch_blocks<CACHE_E4M3, 64>(a, stream);
    if (d == 128) return launch_blocks<CACHE_E4M3, 128>(a, stream);
    return launch_blocks<CACHE_E4M3, 256>(a, stream);
}

hipError_t launch_paged_join(const PagedArgs &a, int cache, int d, hipStream_t stream)
{
    const dim3 grid((unsigned)((int64_t)a.n_seqs * a.n_q * a.n_heads)), th(kT);
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, th, 0, stream, a, cache == CACHE_E4M3); };
    if (cache == CACHE_F32)
        d == 64 ? go(paged_join_kernel<64, true>) : go(paged_join_kernel<128, true>);
    else
        d == 64 ? go(paged_join_kernel<64, false>) : d == 128 ? go(paged_join_kernel<128, false>) : go(paged_join_kernel<256, false>);
    return hipGetLastError();
}

}  // namespace rr
