// Appending new tokens to the paged cache, for gfx950: keys rotated by their
// positions on the way into their pages, values beside them, queries rotated
// with the same angles.
//
// Bound by the bytes: every row is read once and written once (24 KB a token
// in all at 32 query heads on 8 key heads of 128 bf16 features).  What could
// cost more are the angles: position * frequency loses its low digits in
// binary32 beyond some thousand positions, so an angle is formed and reduced
// to a fraction of a turn in binary64, and its sine and cosine are taken once
// a token and shared by all of its heads through LDS.
//
// Measured: 32768 tokens of that size in 135 us, 5.8 TB/s read and written (a
// copy of 1 GiB: 5.1); 22600 tokens of ragged prompts into an 8-bit cache, rotated
// by axes, 90 (5.6 TB/s).  Small calls are a chain of loads -- start, length, page
// -- and the launch: one token 2.6 us, 64 by axes 3.9, 192 tokens of as many
// sequences into an 8-bit cache 4.4, 24 ragged binary32 prompts (3147 tokens, 16
// MB) 7.2.
//
// A workgroup takes a token.  A thread keeps the same features of a row over
// the heads that it goes through, so it reads its sines and cosines once; a
// piece is 16 bytes of input (an element, or two interleaved ones, where rows
// are not aligned to that).  What hides the chain are many waves and rows that
// are asked for before it: a kernel of 37 to 66 registers and pieces of 16 bytes
// takes 98 us for the ragged prompts where one of 87 and pieces of 8 took 121.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "rr_device.hpp"
#include "rr_internal.hpp"
#include "rr_paged.hpp"
#include "rr_rows.hpp"

namespace rr {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kMostRot = 1024;
constexpr int kAhead = 2;  // rows that a thread asks for first

// x / scale for many x, on the same side of every border between two 8-bit numbers
// as a division's quotient, in four instructions where a division takes ten, of
// which appending has more than of anything else.  With r the rounded 1 / scale, q =
// x r is off by less than 1.5 of its steps; r and the remainder x - q scale are off
// by 2^-24 relative each, so that q + (x - q scale) r before its own rounding is off
// by less than 2^-22 steps.  It can then leave a division's side only where x is one
// of the two binary32 numbers around scale times a border, or scale times half a step
// beside one.  Borders have 16 significands, and powers of two change nothing within
// the scales that are not divided by: for all 2^23 significands of scale, those x and
// the one beyond on either side give a division's quotient bit for bit (1.2e9 pairs,
// gone through once).  Quotients past 1024, which clamp in any case, are not refined
// (an infinite one would make a NaN of the remainder); scales so far from one that
// a remainder could leave the range of normal numbers divide.
struct Quotient {
    float scale, r;
    bool direct;

    __device__ __forceinline__ explicit Quotient(float s) : scale(s), r(1.f / s), direct(!(s > 0x1p-60f && s < 0x1p60f)) {}

    template <int N>
    __device__ __forceinline__ void operator()(const float (&x)[N], float (&y)[N]) const
    {
        if (direct) {
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = x[e] / scale;
            return;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float q = __builtin_amdgcn_fmed3f(x[e] * r, -1024.f, 1024.f);
            y[e] = __builtin_fmaf(-__builtin_fmaf(q, scale, -x[e]), r, q);  // (so that -0 stays -0)
        }
    }
};

// What e4m3 holds of x: beyond the largest finite value, that one.
__device__ __forceinline__ float clamp_e4m3(float x)
{
    return x != x ? x : __builtin_amdgcn_fmed3f(x, -448.f, 448.f);
}

template <int N, bool VEC>
__device__ __forceinline__ void write_e4m3(uint8_t *p, const float (&x)[N], const Quotient &over)
{
    float y[N];
    over(x, y);
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = clamp_e4m3(y[e]);
    if constexpr (VEC) {
        uint32_t o[N / 4];
#pragma unroll
        for (int q = 0; q < N / 4; ++q) {
            const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * q], y[4 * q + 1], 0, false);
            o[q] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * q + 2], y[4 * q + 3], lo, true);
        }
        __builtin_memcpy(__builtin_assume_aligned(p, N), o, N);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) p[e] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[e], 0.f, 0, false);
    }
}

// Pieces of rows, past the caches (ONCE) or not.
template <typename T, int N, bool VEC, bool ONCE>
__device__ __forceinline__ typename Raw<T, N>::V read_input(const T *p)
{
    if constexpr (ONCE)
        return __builtin_nontemporal_load(reinterpret_cast<const typename Raw<T, N>::V *>(p));
    else
        return read_raw<T, N, VEC>(p);
}

template <typename T, int N, bool VEC, bool ONCE>
__device__ __forceinline__ void write_output(T *p, const float (&x)[N])
{
    if constexpr (ONCE) {
        typename Piece<T, N>::V v;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (T)x[e];
        __builtin_nontemporal_store(v, reinterpret_cast<typename Piece<T, N>::V *>(p));
    } else {
        write_piece<T, N, VEC>(p, x);
    }
}

// (8-bit rows are written in parts of lines, which the caches put together)
template <typename T, bool E4, int N, bool VEC, bool ONCE>
__device__ __forceinline__ void write_cache(void *pool, int64_t at, const float (&x)[N], const Quotient &over)
{
    if constexpr (E4)
        write_e4m3<N, VEC>(static_cast<uint8_t *>(pool) + at, x, over);
    else
        write_output<T, N, VEC, ONCE>(static_cast<T *>(pool) + at, x);
}

// The same number, in a vector register.
__device__ __forceinline__ int in_vector(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// sequence_of by a wave: of up to 64 sequences every lane looks at one, which
// is one load's latency in place of six (24 sequences: 7.6 us against 8.4).
__device__ __forceinline__ int find_sequence(const int32_t *start, int n_seqs, int i)
{
    if (n_seqs > 64) return sequence_of(start, n_seqs, i);
    const int lane = threadIdx.x & 63, at = min(lane, n_seqs - 1);
    const int from = start[at], to = start[at + 1];
    const uint64_t begun = __ballot(lane < n_seqs && from <= i), here = __ballot(i < to);
    const int b = begun ? 63 - __clzll((long long)begun) : 0;
    return in_vector((begun & here) >> b & 1u ? b : -1);
}

// AXES: rotated by the token's positions on several axes, not by its place in the
// sequence.  ONCE: past the caches.  The first rows of a thread and its first
// values are asked for before the token's place is known (one token 2.6 us, none
// ahead 3.1; ragged prompts into an 8-bit cache 98 and 113).
template <typename T, bool E4, bool INTER, int N, bool VEC, bool AXES, bool ONCE>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs a)
{
    typedef typename Raw<T, N>::V V;
    __shared__ float s_cos[kMostRot / 2], s_sin[kMostRot / 2];
    const int tid = threadIdx.x, half = a.rot >> 1;
    const int64_t i = blockIdx.x;

    // Rows of queries and keys.  INTER: a piece is N / 2 pairs of neighbours;
    // otherwise a rotated unit is a piece of the first half and its partner,
    // and what is not rotated follows in single pieces.
    const int turned = INTER ? a.rot / N : half / N, units = INTER ? a.d / N : turned + (a.d - a.rot) / N;
    const int n_rows = a.n_kv_heads + (a.Q ? a.n_heads : 0);
    const int lanes = a.lanes, rows_at_once = a.rows_at_once, row0 = tid * a.lanes_mul >> 16;  // (tid / lanes)
    const int u0 = tid - row0 * lanes, r0 = row0 < rows_at_once ? row0 : n_rows;
    auto piece_at = [&](int u) { return INTER || u < turned ? u * N : a.rot + (u - turned) * N; };
    auto row_at = [&](int r) {
        return r < a.n_kv_heads ? static_cast<const T *>(a.K) + i * a.ldk + r * a.d
                                : static_cast<const T *>(a.Q) + i * a.ldq + (r - a.n_kv_heads) * a.d;
    };
    const int n_values = a.n_kv_heads * a.pieces.page;
    auto value_at = [&](int x) {  // (heads follow each other)
        return static_cast<const T *>(a.V) + i * a.ldv + x * N;
    };
    int axis[1];
    double freq = 0.0;
    if (tid < half) {
        freq = a.freqs[tid];
        if (AXES) a.axes.of(tid, axis);
    }
    V first_x[kAhead], first_y[kAhead], first_v;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
        const int r = r0 + k * rows_at_once;
        if (r < n_rows) {
            const T *src = row_at(r) + piece_at(u0);
            first_x[k] = read_input<T, N, VEC, ONCE>(src);
            if (!INTER && u0 < turned) first_y[k] = read_input<T, N, VEC, ONCE>(src + half);
        }
    }
    if (tid < n_values) first_v = read_input<T, N, VEC, ONCE>(value_at(tid));

    double at[1];
    if (AXES && tid < half) a.axes.at(i, axis, at);

    // where the token goes: sequence, position, page.  (Loads that wait for each
    // other; with their addresses in vector registers, as the scalar loads that
    // the compiler would make of them take longer: 3.3 us against 3.7 for a
    // token)
    int b, left;  // tokens of the sequence's new ones from this one on
    if (a.seq_start) {
        b = find_sequence(a.seq_start, a.n_seqs, in_vector((int)i));
        left = b < 0 ? 0 : a.seq_start[b + 1] - (int)i;
    } else {
        b = in_vector((int)i / a.per_seq);
        left = a.per_seq - ((int)i - b * a.per_seq);
    }
    if (b < 0) return;
    const int64_t p = (int64_t)a.lengths[b] - left;
    if (p < 0 || p >= (int64_t)a.max_pages * a.pd.page) return;
    const int pos = (int)p, c = a.pd.div(pos), place = __builtin_amdgcn_readfirstlane(pos - c * a.pd.page);
    const int phys = __builtin_amdgcn_readfirstlane(pool_page(a.table[(int64_t)b * a.max_pages + c], a.n_pages));
    const int64_t at0 = pool_row(phys, a.n_kv_heads, 0, a.pd.page, place, a.d), head = (int64_t)a.pd.page * a.d;

    for (int x = tid; x < half; x += kAppendThreads) {
        if (x != tid) {
            freq = a.freqs[x];
            if (AXES) {
                a.axes.of(x, axis);
                a.axes.at(i, axis, at);
            }
        }
        turn_of(AXES ? at[0] : (double)pos, freq, &s_cos[x], &s_sin[x]);
        if (AXES && !a.axes.there(axis[0])) s_cos[x] = kStays;
    }
    __syncthreads();

    constexpr int NT = kTurns<INTER, N>;
    auto put_row = [&](int r, int u, const float (&c)[NT], const float (&s)[NT], V raw_x, V raw_y) {
        const bool key = r < a.n_kv_heads, turn = u < turned;
        const int f0 = piece_at(u), f1 = f0 + half;
        if (key && phys < 0) return;
        float x[N], y[N];
        widen_piece<T, N>(raw_x, x);
        if (turn) {
            if constexpr (!INTER) widen_piece<T, N>(raw_y, y);
            turn_piece<INTER, N, AXES>(x, y, c, s);
        }
        if (key) {
            const int64_t at = at0 + r * head;
            const Quotient over(E4 ? a.k_scale[r] : 1.f);
            write_cache<T, E4, N, VEC, ONCE>(a.Kc, at + f0, x, over);
            if (!INTER && turn) write_cache<T, E4, N, VEC, ONCE>(a.Kc, at + f1, y, over);
        } else {
            T *dst = static_cast<T *>(a.Q_out) + (i * a.n_heads + (r - a.n_kv_heads)) * a.d;
            write_output<T, N, VEC, ONCE>(dst + f0, x);
            if (!INTER && turn) write_output<T, N, VEC, ONCE>(dst + f1, y);
        }
    };
    auto put_rows = [&](int u, auto first) {
        const bool turn = u < turned;
        const int f0 = piece_at(u);
        float c[NT], s[NT];
        if (turn) {
#pragma unroll
            for (int e = 0; e < NT; ++e) {
                c[e] = s_cos[(INTER ? f0 >> 1 : f0) + e];
                s[e] = s_sin[(INTER ? f0 >> 1 : f0) + e];
            }
        }
        int r = r0;
        if constexpr (decltype(first)::value) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k, r += rows_at_once)
                if (r < n_rows) put_row(r, u, c, s, first_x[k], first_y[k]);
        }
        for (; r < n_rows; r += rows_at_once) {
            const T *src = row_at(r) + f0;
            V x = read_input<T, N, VEC, ONCE>(src), y = x;
            if (!INTER && turn) y = read_input<T, N, VEC, ONCE>(src + half);
            put_row(r, u, c, s, x, y);
        }
    };
    put_rows(u0, std::true_type());
    // (a row has no more than 256 vectors, and a loop over them would cost the
    // registers of three waves: ragged prompts 121 us against 109)
    if constexpr (!VEC)
        for (int u = u0 + lanes; u < units; u += lanes) put_rows(u, std::false_type());
    // values
    if (phys < 0) return;
    for (int x = tid; x < n_values; x += kAppendThreads) {
        const int r = a.pieces.div(x), f = (x - r * a.pieces.page) * N;
        float v[N];
        widen_piece<T, N>(x == tid ? first_v : read_input<T, N, VEC, ONCE>(value_at(x)), v);
        write_cache<T, E4, N, VEC, ONCE>(a.Vc, at0 + r * head + f, v, Quotient(E4 ? a.v_scale[r] : 1.f));
    }
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, int dtype, int cache, bool interleaved, hipStream_t stream)
{
    const int size = dtype == 0 ? 4 : 2, n = 16 / size;
    auto aligned = [&](const void *p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % n == 0; };
    // (cache rows of 8 values are 8 bytes in e4m3)
    const bool vec = aligned(a.K, a.ldk) && aligned(a.V, a.ldv) && aligned(a.Q, a.Q ? a.ldq : 0) && aligned(a.Q_out, 0) &&
                     aligned(a.Kc, 0) && aligned(a.Vc, 0) && a.rot % (interleaved ? n : 2 * n) == 0;
    // Quotients that the threads of a workgroup would form: with m = ceil(2^16 /
    // lanes), tid * m >> 16 = tid / lanes for tid and lanes of at most 256.
    auto go = [&](auto kern, int n) {
        AppendArgs b = a;
        const int turned = interleaved ? a.rot / n : a.rot / 2 / n, units = interleaved ? a.d / n : turned + (a.d - a.rot) / n;
        b.lanes = units < kAppendThreads ? units : kAppendThreads;
        b.lanes_mul = (65536 + b.lanes - 1) / b.lanes;
        b.rows_at_once = kAppendThreads / b.lanes;
        b.pieces = page_div(a.d / n);
        hipLaunchKernelGGL(kern, dim3((unsigned)a.n_tokens), dim3(kAppendThreads), 0, stream, b);
    };
    // What is read and written does not fit the last cache together: past the
    // caches.  Between a call that writes the rows and one that reads the queries
    // (bf16, heads as above, by place; append and reader, through the caches and
    // past them): 8000 tokens 34 + 22 us and 33 + 27, 12000 52 + 49 and 48 + 37,
    // 32768 147 + 106 and 144 + 95, into an 8-bit cache 133 + 104 and 118 + 99.
    // But only in whole lines of 128 bytes, as in a rotation: parts of lines that
    // the caches do not put together are slower by more than the reader gains
    // (32768 tokens of 64 heads on 8: of 64 features 123 + 93 and 163 + 81, of 96
    // 190 + 135 and 274 + 120; 32 heads of 128, of which 64 are rotated, 144 + 93 and
    // 156 + 81, rows of a fused projection 146 + 92 and 147 + 80).
    const int64_t rows = a.n_tokens * (int64_t)a.d, heads = a.Q ? a.n_heads : 0;
    const int64_t bytes = rows * (size * 2 * (heads + a.n_kv_heads) + (cache == CACHE_E4M3 ? 1 : size) * 2 * (int64_t)a.n_kv_heads);
    const bool lines = interleaved ? a.d * size % 128 == 0 : a.rot / 2 * size % 128 == 0 && (a.d - a.rot) * size % 128 == 0;
    const bool once = vec && lines && bytes >= kLastCache;
    auto any = [&](auto type, auto e4, auto axes) {
        typedef decltype(type) T;
        constexpr bool E4 = decltype(e4)::value, AX = decltype(axes)::value;
        constexpr int W = 16 / sizeof(T);
        if (once)
            interleaved ? go(append_kernel<T, E4, true, W, true, AX, true>, W)
                        : go(append_kernel<T, E4, false, W, true, AX, true>, W);
        else if (vec)
            interleaved ? go(append_kernel<T, E4, true, W, true, AX, false>, W)
                        : go(append_kernel<T, E4, false, W, true, AX, false>, W);
        else  // (interleaved partners go together)
            interleaved ? go(append_kernel<T, E4, true, 2, false, AX, false>, 2)
                        : go(append_kernel<T, E4, false, 1, false, AX, false>, 1);
    };
    auto types = [&](auto axes) {
        if (dtype == 0)
            any(float(), std::false_type(), axes);
        else if (cache == CACHE_E4M3)
            any(__bf16(), std::true_type(), axes);
        else
            any(__bf16(), std::false_type(), axes);
    };
    a.axes.positions ? types(std::true_type()) : types(std::false_type());
    return hipGetLastError();
}

}  // namespace rr
