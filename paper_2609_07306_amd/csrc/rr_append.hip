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
// Measured: 32768 tokens of that size in 143 us, 5.6 TB/s read and written (a
// copy of 1 GiB: 5.1).  Small calls are a chain of loads -- length, page,
// rows -- and the launch: one token 3.3 us, 192 tokens of as many sequences
// into an 8-bit cache 5.4, 24 ragged binary32 prompts (3147 tokens, 16 MB) 7.4.
//
// A workgroup takes a token.  A thread keeps the same features of a row over
// the heads that it goes through, so it reads its sines and cosines once; a
// vector piece is 16 bytes of input (one element where rows are not aligned to
// that).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "rr_device.hpp"
#include "rr_internal.hpp"
#include "rr_paged.hpp"

namespace rr {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kMostRot = 1024;

template <typename T, int N>
struct Piece {
    typedef T V __attribute__((ext_vector_type(N)));
};

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__bf16 x) { return (float)x; }

// N consecutive elements of a row as binary32: one vector, or (VEC = false,
// where rows are not aligned to one) element by element.
template <typename T, int N, bool VEC>
__device__ __forceinline__ void read_piece(const T *p, float (&x)[N])
{
    if constexpr (VEC) {
        const auto v = *reinterpret_cast<const typename Piece<T, N>::V *>(p);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = widen(v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = widen(p[e]);
    }
}

template <typename T, int N, bool VEC>
__device__ __forceinline__ void write_piece(T *p, const float (&x)[N])
{
    if constexpr (VEC) {
        typename Piece<T, N>::V v;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (T)x[e];
        *reinterpret_cast<typename Piece<T, N>::V *>(p) = v;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) p[e] = (T)x[e];
    }
}

// What e4m3 holds of x: beyond the largest finite value, that one.
__device__ __forceinline__ float clamp_e4m3(float x)
{
    return x != x ? x : __builtin_amdgcn_fmed3f(x, -448.f, 448.f);
}

template <int N, bool VEC>
__device__ __forceinline__ void write_e4m3(uint8_t *p, const float (&x)[N], float scale)
{
    if constexpr (VEC) {
        uint32_t o[N / 4];
#pragma unroll
        for (int q = 0; q < N / 4; ++q) {
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = clamp_e4m3(x[4 * q + e] / scale);
            const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
            o[q] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
        }
        __builtin_memcpy(__builtin_assume_aligned(p, N), o, N);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            p[e] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(x[e] / scale), 0.f, 0, false);
    }
}

template <typename T, bool E4, int N, bool VEC>
__device__ __forceinline__ void write_cache(void *pool, int64_t at, const float (&x)[N], float scale)
{
    if constexpr (E4)
        write_e4m3<N, VEC>(static_cast<uint8_t *>(pool) + at, x, scale);
    else
        write_piece<T, N, VEC>(static_cast<T *>(pool) + at, x);
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

template <typename T, bool E4, bool INTER, int N, bool VEC>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs a)
{
    __shared__ float s_cos[kMostRot / 2], s_sin[kMostRot / 2];
    const int tid = threadIdx.x, half = a.rot >> 1;

    // where the token goes: sequence, position, page.  (Loads that wait for each
    // other; with their addresses in vector registers, as the scalar loads that
    // the compiler would make of them take longer: 3.3 us against 3.7 for a
    // token)
    const int64_t i = blockIdx.x;
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
    const int pos = (int)p, c = a.pd.div(pos), place = pos - c * a.pd.page;
    const int phys = pool_page(a.table[(int64_t)b * a.max_pages + c], a.n_pages);

    // angles in turns: position * frequency / 2 pi, less its nearest integer
    for (int x = tid; x < half; x += kAppendThreads) {
        const double turn = (double)pos * a.freqs[x] * 0.15915494309189533577;
        sincospif(2.f * (float)(turn - rint(turn)), &s_sin[x], &s_cos[x]);
    }
    __syncthreads();

    // Rows of queries and keys.  INTER: a piece is N / 2 pairs of neighbours;
    // otherwise a rotated unit is a piece of the first half and its partner,
    // and what is not rotated follows in single pieces.
    const int turned = INTER ? a.rot / N : half / N, units = INTER ? a.d / N : turned + (a.d - a.rot) / N;
    const int n_rows = a.n_kv_heads + (a.Q ? a.n_heads : 0);
    const int lanes = min(units, kAppendThreads), rows_at_once = kAppendThreads / lanes;
    if (tid < lanes * rows_at_once) {
        for (int u = tid % lanes; u < units; u += lanes) {
            const bool turn = u < turned;
            // first element of the piece, and of its partner
            const int f0 = INTER ? u * N : turn ? u * N : a.rot + (u - turned) * N, f1 = f0 + half;
            float c[N], s[N];
            if (turn) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    c[e] = s_cos[INTER ? (f0 + e) >> 1 : f0 + e];
                    s[e] = s_sin[INTER ? (f0 + e) >> 1 : f0 + e];
                }
            }
            for (int r = tid / lanes; r < n_rows; r += rows_at_once) {
                const bool key = r < a.n_kv_heads;
                if (key && phys < 0) continue;
                const T *src = key ? static_cast<const T *>(a.K) + i * a.ldk + r * a.d
                                   : static_cast<const T *>(a.Q) + i * a.ldq + (r - a.n_kv_heads) * a.d;
                float x[N], y[N];
                read_piece<T, N, VEC>(src + f0, x);
                if (turn) {
                    if constexpr (INTER) {
#pragma unroll
                        for (int e = 0; e < N; e += 2) {
                            const float p = x[e], q = x[e + 1];
                            x[e] = p * c[e] - q * s[e];
                            x[e + 1] = q * c[e] + p * s[e];
                        }
                    } else {
                        read_piece<T, N, VEC>(src + f1, y);
#pragma unroll
                        for (int e = 0; e < N; ++e) {
                            const float p = x[e], q = y[e];
                            x[e] = p * c[e] - q * s[e];
                            y[e] = q * c[e] + p * s[e];
                        }
                    }
                }
                if (key) {
                    const int64_t at = pool_row(phys, a.n_kv_heads, r, a.pd.page, place, a.d);
                    const float scale = E4 ? a.k_scale[r] : 1.f;
                    write_cache<T, E4, N, VEC>(a.Kc, at + f0, x, scale);
                    if (!INTER && turn) write_cache<T, E4, N, VEC>(a.Kc, at + f1, y, scale);
                } else {
                    T *dst = static_cast<T *>(a.Q_out) + (i * a.n_heads + (r - a.n_kv_heads)) * a.d;
                    write_piece<T, N, VEC>(dst + f0, x);
                    if (!INTER && turn) write_piece<T, N, VEC>(dst + f1, y);
                }
            }
        }
    }
    // values
    if (phys >= 0) {
        const int pieces = a.d / N;
        for (int x = tid; x < a.n_kv_heads * pieces; x += kAppendThreads) {
            const int r = x / pieces, f = (x - r * pieces) * N;
            float v[N];
            read_piece<T, N, VEC>(static_cast<const T *>(a.V) + i * a.ldv + r * a.d + f, v);
            write_cache<T, E4, N, VEC>(a.Vc, pool_row(phys, a.n_kv_heads, r, a.pd.page, place, a.d) + f, v,
                                  E4 ? a.v_scale[r] : 1.f);
        }
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
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)a.n_tokens), dim3(kAppendThreads), 0, stream, a); };
    auto any = [&](auto type, auto e4, auto width) {
        typedef decltype(type) T;
        constexpr bool E4 = decltype(e4)::value;
        constexpr int W = decltype(width)::value;
        if (vec)
            interleaved ? go(append_kernel<T, E4, true, W, true>) : go(append_kernel<T, E4, false, W, true>);
        else  // (interleaved partners go together)
            interleaved ? go(append_kernel<T, E4, true, 2, false>) : go(append_kernel<T, E4, false, 1, false>);
    };
    if (dtype == 0)
        any(float(), std::false_type(), std::integral_constant<int, 4>());
    else if (cache == CACHE_BF16)
        any(__bf16(), std::false_type(), std::integral_constant<int, 8>());
    else
        any(__bf16(), std::true_type(), std::integral_constant<int, 8>());
    return hipGetLastError();
}

}  // namespace rr
