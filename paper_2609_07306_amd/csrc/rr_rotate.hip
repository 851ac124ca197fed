// Rotation of queries or keys by positions of several axes, for gfx950: rows of
// any two layouts, in place or not, forward or back (the transposed rotation,
// which is its inverse and its gradient).
//
// Bound by the bytes: every row is read once and written once.  A thread takes
// the same features of one token over the heads, so it forms its few angles
// once, in registers, and shares nothing with other threads; a wave's threads
// take neighbouring pieces of a token and neighbouring tokens.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "rr_device.hpp"
#include "rr_internal.hpp"
#include "rr_rows.hpp"

namespace rr {
namespace {

constexpr int kRotateThreads = 256;
constexpr int kRotateGroups = 2048;  // workgroups that a launch is cut into, if its heads allow

// Pieces of a row: INTER: N / 2 pairs of neighbours each; otherwise a rotated
// unit is a piece of the first half and its partner.  What is not rotated
// follows in single pieces.
struct Units {
    int turned, all;
};

template <bool INTER, int N>
__host__ __device__ __forceinline__ Units units_of(int d, int rot)
{
    const int turned = INTER ? rot / N : rot / (2 * N);
    return Units{turned, INTER ? d / N : turned + (d - rot) / N};
}

template <typename T, bool INTER, int N, bool VEC>
__global__ __launch_bounds__(kRotateThreads) void rotate_kernel(RotateArgs a)
{
    const Units un = units_of<INTER, N>(a.d, a.rot);
    const int half = a.rot >> 1, tid = threadIdx.x;
    // (in place, what is not rotated stays where it is)
    const int units = a.X == a.Y ? un.turned : un.all;
    const int lanes = min(un.all, kRotateThreads), tokens = kRotateThreads / lanes;
    const int64_t i = (int64_t)blockIdx.x * tokens + tid / lanes;
    if (tid >= lanes * tokens || i >= a.n_tokens) return;
    const int h0 = blockIdx.y * a.heads_each, h1 = min(h0 + a.heads_each, a.n_heads);
    for (int u = tid % lanes; u < units; u += lanes) {
        const bool turn = u < un.turned;
        // first element of the piece, and of its partner
        const int f0 = INTER ? u * N : turn ? u * N : a.rot + (u - un.turned) * N, f1 = f0 + half;
        float c[N], s[N];
        if (turn) {
#pragma unroll
            for (int e = 0; e < N; e += INTER ? 2 : 1) {
                const int j = INTER ? (f0 + e) >> 1 : f0 + e;
                turn_of(a.axes.at(i, j), a.freqs[j], &c[e], &s[e]);
                s[e] *= a.sign;
            }
        }
        const T *src = static_cast<const T *>(a.X) + i * a.x_token + h0 * a.x_head + f0;
        T *dst = static_cast<T *>(a.Y) + i * a.y_token + h0 * a.y_head + f0;
        for (int h = h0; h < h1; ++h, src += a.x_head, dst += a.y_head) {
            float x[N], y[N];
            read_piece<T, N, VEC>(src, x);
            if (turn) {
                if constexpr (!INTER) read_piece<T, N, VEC>(src + half, y);
                turn_piece<INTER, N>(x, y, c, s);
            }
            write_piece<T, N, VEC>(dst, x);
            if (!INTER && turn) write_piece<T, N, VEC>(dst + half, y);
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
    auto go = [&](auto kern, Units un) {
        const int tokens = kRotateThreads / (un.all < kRotateThreads ? un.all : kRotateThreads);
        const int tiles = (a.n_tokens + tokens - 1) / tokens;
        // heads a workgroup: all of them where the tokens fill the card
        const int parts = tiles >= kRotateGroups ? 1 : (kRotateGroups + tiles - 1) / tiles;
        a.heads_each = (a.n_heads + parts - 1) / parts;
        const dim3 grid((unsigned)tiles, (unsigned)((a.n_heads + a.heads_each - 1) / a.heads_each));
        hipLaunchKernelGGL(kern, grid, dim3(kRotateThreads), 0, stream, a);
    };
    auto any = [&](auto type, auto width) {
        typedef decltype(type) T;
        constexpr int W = decltype(width)::value;
        if (vec)
            interleaved ? go(rotate_kernel<T, true, W, true>, units_of<true, W>(a.d, a.rot))
                        : go(rotate_kernel<T, false, W, true>, units_of<false, W>(a.d, a.rot));
        else  // (interleaved partners go together)
            interleaved ? go(rotate_kernel<T, true, 2, false>, units_of<true, 2>(a.d, a.rot))
                        : go(rotate_kernel<T, false, 1, false>, units_of<false, 1>(a.d, a.rot));
    };
    if (dtype == 0)
        any(float(), std::integral_constant<int, 4>());
    else
        any(__bf16(), std::integral_constant<int, 8>());
    return hipGetLastError();
}

}  // namespace rr
