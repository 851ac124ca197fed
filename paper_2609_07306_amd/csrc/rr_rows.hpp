// Rows of keys and queries in pieces of vectors, their positions on several
// axes, and the arguments of the rotation (rr_append.hip, rr_rotate.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rr {

template <typename T, int N>
struct Piece {
    typedef T V __attribute__((ext_vector_type(N)));
};

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__bf16 x) { return (float)x; }

// N consecutive elements of a row as they lie in memory, in as many registers as
// they have words (a vector of __bf16 would take one an element).
template <typename T, int N>
struct Raw {
    static constexpr int kWords = (N * (int)sizeof(T) + 3) / 4;
    typedef uint32_t V __attribute__((ext_vector_type(kWords)));
};

// One vector, or (VEC = false, where rows are not aligned to one) element by
// element.
template <typename T, int N, bool VEC>
__device__ __forceinline__ typename Raw<T, N>::V read_raw(const T *p)
{
    typedef typename Raw<T, N>::V V;
    if constexpr (VEC) return *reinterpret_cast<const V *>(p);
    V v;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = reinterpret_cast<const uint32_t *>(p)[e];
    } else {
        const uint16_t *q = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
        for (int e = 0; e < N; e += 2) v[e / 2] = q[e] | (e + 1 < N ? (uint32_t)q[e + 1] << 16 : 0u);
    }
    return v;
}

template <typename T, int N>
__device__ __forceinline__ void widen_piece(typename Raw<T, N>::V v, float (&x)[N])
{
#pragma unroll
    for (int e = 0; e < N; ++e)
        x[e] = sizeof(T) == 4 ? __uint_as_float(v[e / (4 / (int)sizeof(T))])
                              : __uint_as_float(e % 2 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
}

template <typename T, int N, bool VEC>
__device__ __forceinline__ void read_piece(const T *p, float (&x)[N])
{
    widen_piece<T, N>(read_raw<T, N, VEC>(p), x);
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

// Frequencies of a piece.
template <bool INTER, int N>
constexpr int kTurns = INTER ? N / 2 : N;

// The cosine, which no angle has, of a frequency whose axis is not there: its
// partners stay as they are.  (Turned by an angle of 0, an infinite one would make
// the other a NaN, and a -0 could lose its sign.)
constexpr float kStays = 2.f;

// Rotates a piece: neighbours are partners (INTER), or x's element e and y's.
// SOME: but for those that kStays stands for.  Of two products one is rounded before
// they are added; which one is written down, as the compiler would choose it kernel
// by kernel: every call gives a row the same bits.
template <bool INTER, int N, bool SOME>
__device__ __forceinline__ void turn_piece(float (&x)[N], float (&y)[N], const float (&c)[kTurns<INTER, N>],
                                           const float (&s)[kTurns<INTER, N>])
{
    auto turn = [](float &x, float &y, float c, float s) {
        const float p = x, q = y;
        const bool stays = SOME && c == kStays;
        x = stays ? p : __builtin_fmaf(p, c, -(q * s));
        y = stays ? q : INTER ? __builtin_fmaf(p, s, q * c) : __builtin_fmaf(q, c, p * s);
    };
    if constexpr (INTER) {
#pragma unroll
        for (int e = 0; e < N; e += 2) turn(x[e], x[e + 1], c[e / 2], s[e / 2]);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) turn(x[e], y[e], c[e], s[e]);
    }
}

// Cosine and sine of position * frequency.  The product loses its low digits in
// binary32 beyond some thousand positions, so the angle is formed and reduced
// to a fraction of a turn in binary64.
__device__ __forceinline__ void turn_of(double pos, double freq, float *c, float *s)
{
    const double turn = pos * freq * 0.15915494309189533577;
    sincospif(2.f * (float)(turn - rint(turn)), s, c);
}

// Positions of tokens on several axes.
struct Axes {
    const void *positions;  // [n_axes, n] int32, or binary32 where real
    const int32_t *axis;    // [rot / 2] axis of each frequency; null: the first one's
    int64_t n;              // tokens
    int32_t n_axes, real;

    // The axes of frequencies j .. j + N - 1.  (Their loads are a stage of their
    // own, so that loads wait for each other only where they must.)
    template <int N>
    __device__ __forceinline__ void of(int j, int (&t)[N]) const
    {
#pragma unroll
        for (int e = 0; e < N; ++e) t[e] = 0;
        if (axis) {
#pragma unroll
            for (int e = 0; e < N; ++e) t[e] = axis[j + e];
        }
    }

    __device__ __forceinline__ bool there(int t) const { return (uint32_t)t < (uint32_t)n_axes; }

    // Token i's positions on axes t; the first one's for an axis that is not there.
    template <int N>
    __device__ __forceinline__ void at(int64_t i, const int (&t)[N], double (&p)[N]) const
    {
        int32_t bits[N];
#pragma unroll
        for (int e = 0; e < N; ++e) bits[e] = static_cast<const int32_t *>(positions)[(there(t[e]) ? t[e] : 0) * n + i];
#pragma unroll
        for (int e = 0; e < N; ++e) p[e] = real ? (double)__int_as_float(bits[e]) : (double)bits[e];
    }
};

// Cosines (or kStays) and sines of token i for frequencies j .. j + N - 1.
template <int N>
__device__ __forceinline__ void turns_of(const Axes &axes, const double *freqs, int64_t i, int j, float (&c)[N], float (&s)[N])
{
    double p[N], f[N];
    int t[N];
    axes.of(j, t);
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = freqs[j + e];
    axes.at(i, t, p);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        turn_of(p[e], f[e], &c[e], &s[e]);
        if (!axes.there(t[e])) c[e] = kStays;
    }
}

struct RotateArgs {
    const void *X;
    void *Y;
    const double *freqs;  // [rot / 2]
    Axes axes;
    int64_t x_token, x_head, y_token, y_head;  // elements between rows
    int32_t n_heads, n_tokens, d, rot;
    int32_t each, heads;  // heads, or tokens and heads, of a workgroup (set by the launcher)
    float sign;           // -1: back
};

hipError_t launch_rotate(const RotateArgs &a, int dtype, bool interleaved, hipStream_t stream);

}  // namespace rr
