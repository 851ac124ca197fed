// Rotation of queries or keys by positions of several axes, for gfx950: rows of
// any two layouts, in place or not, forward or back (the transposed rotation,
// which is its inverse and its gradient).
//
// Bound by the bytes, every row read once and written once; how near to that it
// comes goes by the order: workgroups that follow each other in memory, each
// with a short stretch of its own, move 32768 tokens of 32 heads (128 bf16
// features, 268 MB each way) in 92 us heads first and 90 tokens first, 5.8 and
// 6.0 TB/s; a workgroup that takes 32 tokens of every head in turn in 122.  So
// there is a kernel for each layout.  Loads and stores of such calls go past the
// caches.  A small call (196 tokens, 6 heads) is a launch and a chain, 3.1 us.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "rr_device.hpp"
#include "rr_internal.hpp"
#include "rr_rows.hpp"

namespace rr {
namespace {

constexpr int kRotateThreads = 256;
constexpr int kManyGroups = 1024;  // workgroups that fill the card

// Units of a row that a thread takes.  INTER: pieces of N / 2 pairs of
// neighbours; otherwise a rotated unit is a piece of the first half and its
// partner.  What is not rotated follows in single pieces.
struct Units {
    int turned, all;
};

template <bool INTER, int N>
__host__ __device__ __forceinline__ Units units_of(int d, int rot)
{
    const int turned = INTER ? rot / N : rot / (2 * N);
    return Units{turned, turned + (d - rot) / N};
}

// First element of unit u.
template <bool INTER, int N>
__device__ __forceinline__ int unit_at(const RotateArgs &a, const Units &un, int u)
{
    return INTER || u < un.turned ? u * N : a.rot + (u - un.turned) * N;
}

// How rows are read and written: element by element, in vectors, or in vectors
// past the caches.
enum Way : int { WAY_EACH, WAY_VEC, WAY_ONCE };

template <typename T, int N, Way W>
__device__ __forceinline__ void read_row(const T *p, float (&x)[N])
{
    if constexpr (W == WAY_ONCE) {
        const auto v = __builtin_nontemporal_load(reinterpret_cast<const typename Piece<T, N>::V *>(p));
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = widen(v[e]);
    } else {
        read_piece<T, N, W == WAY_VEC>(p, x);
    }
}

template <typename T, int N, Way W>
__device__ __forceinline__ void write_row(T *p, const float (&x)[N])
{
    if constexpr (W == WAY_ONCE) {
        typename Piece<T, N>::V v;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (T)x[e];
        __builtin_nontemporal_store(v, reinterpret_cast<typename Piece<T, N>::V *>(p));
    } else {
        write_piece<T, N, W == WAY_VEC>(p, x);
    }
}

// Tokens of a head follow each other: a thread takes the same unit of one token
// over a few heads and keeps its angles.
template <typename T, bool INTER, int N, Way W>
__global__ __launch_bounds__(kRotateThreads) void rotate_heads_kernel(RotateArgs a)
{
    const Units un = units_of<INTER, N>(a.d, a.rot);
    const int half = a.rot >> 1, tid = threadIdx.x;
    // (in place, what is not rotated stays where it is)
    const int units = a.X == a.Y ? un.turned : un.all;
    const int lanes = min(un.all, kRotateThreads), tokens = kRotateThreads / lanes;
    const int64_t i = (int64_t)blockIdx.x * tokens + tid / lanes;
    if (tid >= lanes * tokens || i >= a.n_tokens) return;
    const int h0 = blockIdx.y * a.each, h1 = min(h0 + a.each, a.n_heads);
    for (int u = tid % lanes; u < units; u += lanes) {
        const bool turn = u < un.turned;
        const int f0 = unit_at<INTER, N>(a, un, u);
        const T *src = static_cast<const T *>(a.X) + i * a.x_token + h0 * a.x_head + f0;
        T *dst = static_cast<T *>(a.Y) + i * a.y_token + h0 * a.y_head + f0;
        constexpr int NT = kTurns<INTER, N>;
        float c[NT], s[NT], x[N], y[N], next_x[N], next_y[N];
        read_row<T, N, W>(src, next_x);
        if (!INTER && turn) read_row<T, N, W>(src + half, next_y);
        if (turn) {
            turns_of(a.axes, a.freqs, i, INTER ? f0 >> 1 : f0, c, s);
#pragma unroll
            for (int e = 0; e < NT; ++e) s[e] *= a.sign;
        }
        for (int h = h0; h < h1; ++h, dst += a.y_head) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                x[e] = next_x[e];
                y[e] = next_y[e];
            }
            if (h + 1 < h1) {
                src += a.x_head;
                read_row<T, N, W>(src, next_x);
                if (!INTER && turn) read_row<T, N, W>(src + half, next_y);
            }
            if (turn) turn_piece<INTER, N, true>(x, y, c, s);
            write_row<T, N, W>(dst, x);
            if (!INTER && turn) write_row<T, N, W>(dst + half, y);
        }
    }
}

// Heads of a token follow each other: a workgroup takes the heads of a few
// tokens in the order of memory, and its threads share the angles in LDS.
constexpr int kMostAngles = 2048;  // of a workgroup

template <typename T, bool INTER, int N, Way W>
__global__ __launch_bounds__(kRotateThreads) void rotate_tokens_kernel(RotateArgs a)
{
    __shared__ float s_cos[kMostAngles], s_sin[kMostAngles];
    const Units un = units_of<INTER, N>(a.d, a.rot);
    const int half = a.rot >> 1, tid = threadIdx.x;
    const int units = a.X == a.Y ? un.turned : un.all;
    const int64_t i0 = (int64_t)blockIdx.x * a.each;
    const int tokens = (int)min((int64_t)a.each, a.n_tokens - i0);
    const int h0 = blockIdx.y * a.heads, heads = min(a.heads, a.n_heads - h0);
#pragma unroll 4
    for (int x = tid; x < tokens * half; x += kRotateThreads) {
        const int t = x / half;
        float c[1], s[1];
        turns_of(a.axes, a.freqs, i0 + t, x - t * half, c, s);
        s_cos[x] = c[0];
        s_sin[x] = s[0] * a.sign;
    }
    __syncthreads();
    const int lanes = min(un.all, kRotateThreads), rows = kRotateThreads / lanes;
    if (tid >= lanes * rows) return;
    for (int u = tid % lanes; u < units; u += lanes) {
        const bool turn = u < un.turned;
        const int f0 = unit_at<INTER, N>(a, un, u);
        int t = 0, h = tid / lanes;
        while (h >= heads) {
            h -= heads;
            ++t;
        }
        while (t < tokens) {
            const int64_t i = i0 + t;
            const T *src = static_cast<const T *>(a.X) + i * a.x_token + (h0 + h) * a.x_head + f0;
            T *dst = static_cast<T *>(a.Y) + i * a.y_token + (h0 + h) * a.y_head + f0;
            float x[N], y[N];
            read_row<T, N, W>(src, x);
            if (!INTER && turn) read_row<T, N, W>(src + half, y);
            if (turn) {
                constexpr int NT = kTurns<INTER, N>;
                float c[NT], s[NT];
                const int at = t * half + (INTER ? f0 >> 1 : f0);
#pragma unroll
                for (int e = 0; e < NT; ++e) {
                    c[e] = s_cos[at + e];
                    s[e] = s_sin[at + e];
                }
                turn_piece<INTER, N, true>(x, y, c, s);
            }
            write_row<T, N, W>(dst, x);
            if (!INTER && turn) write_row<T, N, W>(dst + half, y);
            h += rows;
            while (h >= heads) {
                h -= heads;
                ++t;
            }
        }
    }
}

}  // namespace

hipError_t launch_rotate(const RotateArgs &args, int dtype, bool interleaved, hipStream_t stream)
{
    RotateArgs a = args;
    const int n = dtype == 0 ? 4 : 8;
    const bool vec = ((reinterpret_cast<uintptr_t>(a.X) | reinterpret_cast<uintptr_t>(a.Y)) & 15) == 0 && a.x_token % n == 0 &&
                     a.x_head % n == 0 && a.y_token % n == 0 && a.y_head % n == 0 && a.rot % (interleaved ? n : 2 * n) == 0;
    // Past the caches what does not fit the last one, input and output together, so
    // that a reader finds what is left there (between a call that writes the rows and
    // one that reads them, bf16, 32 heads of 128, out of place, through the caches and
    // past them: 12000 tokens 33 + 33 us and 33 + 37, 16384 46 + 57 and 44 + 49,
    // 32768 99 + 103 and 100 + 95; in place 16384 44 + 40 and 43 + 49, 32768 86 + 113
    // and 95 + 95), and only in whole lines of 128 bytes: a row of pairs of
    // neighbours, or halves of that size.
    const int size = dtype == 0 ? 4 : 2;
    const bool lines = interleaved ? a.d * size % 128 == 0 : a.rot / 2 * size % 128 == 0 && (a.d - a.rot) * size % 128 == 0;
    const bool once = lines && (int64_t)a.n_tokens * a.n_heads * a.d * size >= kLastCache / (a.X == a.Y ? 1 : 2);
    // which rows follow each other
    const bool by_token = a.n_heads > 1 && (a.n_tokens == 1 || a.y_head < a.y_token);
    auto go = [&](auto by_heads, auto by_tokens, Units un) {
        if (by_token) {
            // Tokens a workgroup: two turns of its threads (32768 tokens of 32 heads:
            // two tokens 90 us, four 91, eight 103; of 2 heads of 64: 16 tokens 9 us,
            // four 18), as long as there are workgroups for the card; then heads are
            // shared out too.
            const int lanes = un.all < kRotateThreads ? un.all : kRotateThreads, rows = kRotateThreads / lanes;
            const int half = a.rot / 2 > 0 ? a.rot / 2 : 1;
            int each = 2 * rows / (a.n_heads < rows ? a.n_heads : rows);
            if (each > kMostAngles / half) each = kMostAngles / half;
            while (each > 1 && (a.n_tokens + each - 1) / each < kManyGroups) each /= 2;
            const int tiles = (a.n_tokens + each - 1) / each, parts = tiles >= kManyGroups ? 1 : kManyGroups / tiles;
            int heads = (a.n_heads + parts - 1) / parts;
            if (heads < rows) heads = rows;
            if (heads > a.n_heads) heads = a.n_heads;
            a.each = each;
            a.heads = heads;
            hipLaunchKernelGGL(by_tokens, dim3((unsigned)tiles, (unsigned)((a.n_heads + heads - 1) / heads)),
                               dim3(kRotateThreads), 0, stream, a);
            return;
        }
        const int tokens = kRotateThreads / (un.all < kRotateThreads ? un.all : kRotateThreads);
        const int tiles = (a.n_tokens + tokens - 1) / tokens;
        // heads a workgroup: 4, fewer where the workgroups would not fill the card,
        // more where a launch would not hold them
        int each = 4;
        while (each > 1 && (int64_t)tiles * ((a.n_heads + each - 1) / each) < kManyGroups) each /= 2;
        while ((a.n_heads + each - 1) / each > 65535) each *= 2;
        a.each = each;
        hipLaunchKernelGGL(by_heads, dim3((unsigned)tiles, (unsigned)((a.n_heads + each - 1) / each)), dim3(kRotateThreads), 0,
                           stream, a);
    };
    auto ways = [&](auto type, auto inter, auto width, auto way) {
        typedef decltype(type) T;
        constexpr bool I = decltype(inter)::value;
        constexpr int N = decltype(width)::value;
        constexpr Way W = decltype(way)::value;
        go(rotate_heads_kernel<T, I, N, W>, rotate_tokens_kernel<T, I, N, W>, units_of<I, N>(a.d, a.rot));
    };
    auto any = [&](auto type, auto width) {
        typedef std::integral_constant<Way, WAY_EACH> Each;
        typedef std::integral_constant<Way, WAY_VEC> Vec;
        typedef std::integral_constant<Way, WAY_ONCE> Once;
        if (!vec)  // (interleaved partners go together)
            interleaved ? ways(type, std::true_type(), std::integral_constant<int, 2>(), Each())
                        : ways(type, std::false_type(), std::integral_constant<int, 1>(), Each());
        else if (once)
            interleaved ? ways(type, std::true_type(), width, Once()) : ways(type, std::false_type(), width, Once());
        else
            interleaved ? ways(type, std::true_type(), width, Vec()) : ways(type, std::false_type(), width, Vec());
    };
    if (dtype == 0)
        any(float(), std::integral_constant<int, 4>());
    else
        any(__bf16(), std::integral_constant<int, 8>());
    return hipGetLastError();
}

}  // namespace rr
