// Verification of drafted tokens against the target's probabilities, for
// gfx950: which drafts are taken, and the token that follows them, drawn from
// what the target has left beside the drafts (or from the target where all were
// taken), all from given uniform numbers.
//
// Draft i is taken iff u_i q_i(x_i) < p_i(x_i).  With a the first one that is
// not, the rest is r = max(p_a - q_a, 0), and the token the first v whose sum
// of r up to it exceeds u_n times the whole sum.  Everything is formed in
// binary64: a product of two binary32 numbers is exact there, and sums of a
// vocabulary are off by 2^-53 of the whole a term, so that the order of the
// additions moves a border by less than the uniform numbers' own steps.
//
// Bound by the bytes of one row of each of the two (the rows of taken drafts
// are not read).  A row is split into parts, one or several a wave, that sum r;
// the workgroup of a sequence that comes last finds the part in which the border
// lies and reads that part again.  192 sequences of five drafts over 131072
// tokens, binary32 (182 MB): 37 us, 4.9 TB/s; bf16 23.  What is missing to the 6.5
// that reads reach are a chain of loads before the first sum (draft, probability, row:
// about 4 us) and one after the last (counter, sums, part: about 5), which all
// sequences meet at once; one sequence over 32000 tokens is these chains, 6.1 us.
#include <hip/hip_runtime.h>

#include "rr_device.hpp"
#include "rr_verify.hpp"

namespace rr {
namespace {

constexpr int kVerifyThreads = 256, kVerifyWaves = kVerifyThreads / 64;
constexpr int kManyWaves = 4096;

__device__ __forceinline__ void wait_vm() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ double value(float x) { return (double)x; }
__device__ __forceinline__ double value(__bf16 x) { return (double)(float)x; }

// Sixteen bytes of a row, from an address that is a multiple of an element's
// size; a wave's step takes 64 of them.
template <typename T>
struct Some {
    static constexpr int N = 16 / sizeof(T), STEP = 64 * N;
    typedef T V __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

enum Rest : int { REST_TARGET, REST_DIFFERENCE, REST_WITHOUT };  // p; max(p - q, 0); p but for the draft

// What is drawn from.
template <typename T>
struct Row {
    const T *p, *q;
    int kind, draft, vocab;
    bool once;  // read past the caches

    // Of v, which is in the vocabulary.  Not a positive finite number: nothing.
    __device__ __forceinline__ double weight(int v) const
    {
        const double x = value(p[v]);
        const double r = kind == REST_DIFFERENCE ? x - value(q[v]) : (kind == REST_WITHOUT && v == draft) ? 0.0 : x;
        return r > 0.0 && r < (double)INFINITY ? r : 0.0;
    }
};

// By data-parallel moves; a lane that nothing comes to gets 0.
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double x)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xf, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Sums over lanes 0 .. this one.
__device__ __forceinline__ double wave_up_to(double x)
{
    x += moved<0x111, 0xf>(x);  // from 1, 2, 4 and 8 lanes before, of the row of 16
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    x += moved<0x118, 0xf>(x);
    x += moved<0x142, 0xa>(x);         // row 0 to row 1, row 2 to row 3
    return x + moved<0x143, 0xc>(x);   // the first two rows to the others
}

__device__ __forceinline__ double wave_sum(double x)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, wave_up_to(x));
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, 63), hi = __builtin_amdgcn_readlane((int)(b >> 32), 63);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Sums of x over the threads before this one, and over all of them; s_wave is
// one of two that calls take in turn.
__device__ __forceinline__ double block_before(double x, double *s_wave, double *all)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const double to = wave_up_to(x), before = moved<0x138, 0xf>(to);  // (the lane before's)
    if (lane == 63) s_wave[w] = to;
    __syncthreads();
    double base = 0.0, sum = 0.0;
#pragma unroll
    for (int i = 0; i < kVerifyWaves; ++i) {
        if (i < w) base += s_wave[i];
        sum += s_wave[i];
    }
    *all = sum;
    return base + before;
}

// A lane's elements of a part of STEPS steps, as they lie in memory.
template <typename T, int STEPS>
struct Held {
    typename Some<T>::V x[STEPS], y[STEPS];
};

template <int STEPS, typename T>
__device__ __forceinline__ void ask(const Row<T> &row, int from, Held<T, STEPS> &h)
{
    typedef typename Some<T>::V V;
    if (from + STEPS * Some<T>::STEP > row.vocab) return;  // (the last part is read element by element)
    const int v = from + Some<T>::N * (threadIdx.x & 63);
    auto read = [&](auto get) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            h.x[i] = get(reinterpret_cast<const V *>(row.p + v + i * Some<T>::STEP));
            if (row.kind == REST_DIFFERENCE) h.y[i] = get(reinterpret_cast<const V *>(row.q + v + i * Some<T>::STEP));
        }
    };
    if (row.once)
        read([](const V *p) { return __builtin_nontemporal_load(p); });
    else
        read([](const V *p) { return *p; });
}

// The sum of a part, of which `ask` has asked.  max(r, 0) is 0 for a NaN, and an
// infinite r shows in the sum: a part that has one is read again, as are those
// with the draft to leave out and the end of the vocabulary.
template <int STEPS, typename T>
__device__ __forceinline__ double part_sum(const Row<T> &row, int from, const Held<T, STEPS> &h)
{
    const int to = from + STEPS * Some<T>::STEP, lane = threadIdx.x & 63;
    double sum = 0.0;
    if (to <= row.vocab && !(row.kind == REST_WITHOUT && row.draft >= from && row.draft < to)) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int e = 0; e < Some<T>::N; ++e) {
                const double x = value(h.x[i][e]);
                sum += fmax(row.kind == REST_DIFFERENCE ? x - value(h.y[i][e]) : x, 0.0);
            }
        sum = wave_sum(sum);
        if (sum < (double)INFINITY) return sum;
        sum = 0.0;
    }
    for (int v = from + lane; v < min(to, row.vocab); v += 64) sum += row.weight(v);
    return wave_sum(sum);
}

__device__ __forceinline__ double load_sum(const double *p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ void store_sum(double *p, double x)
{
    __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// What the search for a border has found so far.
struct Found {
    int at;         // where it lies; before it is known, the last place that has any weight; -1
    int known;
    double before;  // the sum before that place
};

// Of one place a thread, in order (`any`: it has some weight, `here`: the
// border lies in it), the first that has the border, or else the last that has
// any weight, into `f` where it is not known yet; s_found is one of two that
// calls take in turn.
__device__ __forceinline__ void look(Found &f, bool any, bool here, int at, double before, Found *s_found)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t some = __ballot(any), border = __ballot(here);
    if (some ? lane == (border ? __builtin_ctzll(border) : 63 - __builtin_clzll(some)) : lane == 0)
        s_found[wave] = Found{some ? at : -1, border != 0, before};
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kVerifyWaves; ++w)
        if (!f.known && s_found[w].at >= 0) f = s_found[w];
}

template <typename T, int STEPS>
__global__ __launch_bounds__(kVerifyThreads) void verify_kernel(VerifyArgs a)
{
    __shared__ double s_wave[2][kVerifyWaves];
    __shared__ Found s_found[2][kVerifyWaves];
    __shared__ int s_last;
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T *P = static_cast<const T *>(a.P) + b * a.p_seq, *Q = a.Q ? static_cast<const T *>(a.Q) + b * a.q_seq : nullptr;
    const int32_t *drafts = a.drafts + (int64_t)b * a.n;
    const float *u = a.uniforms + (int64_t)b * (a.n + 1);

    // the first draft that is not taken: every wave looks for itself
    const int count = a.n_drafts ? max(0, min(a.n_drafts[b], a.n)) : a.n;
    int took = count, draft = -1;
    for (int i0 = 0; i0 < count; i0 += 64) {
        const int i = i0 + lane;
        int x = -1;
        bool taken = false;
        if (i < count) {
            x = drafts[i];
            if ((uint32_t)x < (uint32_t)a.vocab) {
                const double p = value(P[i * a.p_row + x]), q = Q ? value(Q[i * a.q_row + x]) : 1.0;
                taken = (double)u[i] * q < p;
            }
        }
        const uint64_t missed = __ballot(i < count && !taken);
        if (missed) {
            const int first = __builtin_ctzll(missed);
            took = i0 + first;
            draft = __shfl(x, first, 64);
            break;
        }
    }
    Row<T> row{P + took * a.p_row, Q, took == count ? REST_TARGET : Q ? REST_DIFFERENCE : REST_WITHOUT, draft, a.vocab, a.once};
    if (row.kind == REST_DIFFERENCE) row.q += took * a.q_row;

    // this wave's parts, of which the next is asked for before one is summed
    constexpr int kPart = STEPS * Some<T>::STEP, kEach = kPart / kVerifyThreads;
    double *sums = a.sums + (int64_t)b * a.n_parts;
    uint32_t *counter = a.counters + b * kVerifyApart;
    const int own = (blockIdx.x * kVerifyWaves + wave) * a.each, end = min(own + a.each, a.n_parts);
    Held<T, STEPS> held, next;
    if (own < end) ask(row, own * kPart, held);
    for (int i = own; i < end; ++i) {
        if (i + 1 < end) ask(row, (i + 1) * kPart, next);
        const double sum = part_sum(row, i * kPart, held);
        if (lane == 0) store_sum(sums + i, sum);
        held = next;
    }
    wait_vm();        // this wave's sums have been stored ...
    __syncthreads();  // ... and the other waves'
    if (tid == 0) {
        const uint32_t before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = before == gridDim.x - 1;
        if (s_last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) return;

    // The workgroup that comes last: the whole sum, and the part in which the
    // border lies (past all of them, the last one) ...
    Found found{-1, 0, 0.0};
    double border = 0.0;
    const double at_border = (double)u[a.n];
    for (int again = 0;; ++again) {
        double x = tid < a.n_parts ? load_sum(sums + tid) : 0.0, total;
        double from = block_before(x, s_wave[0], &total);
        if (a.n_parts > kVerifyThreads) {
            double more = 0.0, rest;
            for (int i = tid + kVerifyThreads; i < a.n_parts; i += kVerifyThreads) more += load_sum(sums + i);
            block_before(more, s_wave[1], &rest);
            double first = total;
            total += rest;
            border = at_border * total;
            look(found, x > 0.0, x > 0.0 && from + x > border, tid, from, s_found[0]);
            for (int i0 = kVerifyThreads, turn = 0; i0 < a.n_parts && !found.known; i0 += kVerifyThreads, turn ^= 1) {
                x = i0 + tid < a.n_parts ? load_sum(sums + i0 + tid) : 0.0;
                from = first + block_before(x, s_wave[turn], &rest);
                look(found, x > 0.0, x > 0.0 && from + x > border, i0 + tid, from, s_found[turn ^ 1]);
                first += rest;
            }
        } else {
            border = at_border * total;
            look(found, x > 0.0, x > 0.0 && from + x > border, tid, from, s_found[0]);
        }
        if (total > 0.0 || again || row.kind == REST_TARGET) break;
        // (the drafts cover all that the target has: drawn from the target)
        row.kind = REST_TARGET;
        for (int i = wave; i < a.n_parts; i += kVerifyWaves) {
            ask(row, i * kPart, held);
            const double sum = part_sum(row, i * kPart, held);
            if (lane == 0) store_sum(sums + i, sum);
        }
        wait_vm();
        __syncthreads();
    }
    // ... and in it the token, in the same way
    Found token{-1, 0, 0.0};
    if (found.at >= 0) {
        const int first = found.at * kPart + tid * kEach;
        double r[kEach], all, sum = 0.0;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            r[e] = first + e < a.vocab ? row.weight(first + e) : 0.0;
            sum += r[e];
        }
        double to = found.before + block_before(sum, s_wave[1], &all);
        int here = -1, any = -1;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            to += r[e];
            if (r[e] > 0.0) any = first + e;
            if (r[e] > 0.0 && here < 0 && to > border) here = first + e;
        }
        look(token, any >= 0, here >= 0, here >= 0 ? here : any, 0.0, s_found[1]);
    }
    for (int i = tid; i <= a.n; i += kVerifyThreads)
        a.tokens[(int64_t)b * (a.n + 1) + i] = i < took ? drafts[i] : i == took ? token.at : -1;
    if (tid == 0) {
        a.accepted[b] = took;
        if (a.lengths) a.lengths[b] -= count - took;
    }
}

}  // namespace

void verify_schedule(VerifyArgs &a, int dtype)
{
    // Parts of one, two or four steps, so that the last workgroup finds the
    // border's with one sum a thread; a wave takes as many, a power of two, as
    // leave some 4096 waves, four a SIMD.  (Fewer parts a wave are more chains of
    // loads -- draft, probability, row -- before the first sum, and more counters
    // to add to; four steps take registers that leave five waves.  192 sequences,
    // 131072 tokens, two steps: binary32 in 8 parts a wave 38.7 us, 4 37.7, 16 38.9;
    // bf16 in 4 25.2, 2 27.5, 8 26.5; one step 41.2 and 25.2.)
    const int step = dtype == 0 ? Some<float>::STEP : Some<__bf16>::STEP;
    a.steps = 1;
    while (a.steps < 4 && a.vocab > kVerifyThreads * a.steps * step) a.steps *= 2;
    a.n_parts = (a.vocab + a.steps * step - 1) / (a.steps * step);
    a.each = 1;
    while (a.each < 16 && (int64_t)a.n_seqs * a.n_parts >= 2 * a.each * kManyWaves) a.each *= 2;
}

size_t verify_workspace_bytes(const VerifyArgs &a)
{
    // Rows of two or four steps a part have fewer parts than some shorter ones (65536
    // tokens 256, 65537 129): for as many as any row up to this one's length has.
    const int seqs = a.n_seqs < kVerifySeqs ? a.n_seqs : kVerifySeqs, step = Some<float>::STEP;
    const int shorter = (a.vocab + step - 1) / step < kVerifyThreads ? (a.vocab + step - 1) / step : kVerifyThreads;
    return kVerifyCounterBytes + (size_t)seqs * (a.n_parts > shorter ? a.n_parts : shorter) * sizeof(double);
}

hipError_t launch_verify(const VerifyArgs &args, int dtype, void *workspace, hipStream_t stream)
{
    VerifyArgs a = args;
    a.counters = static_cast<uint32_t *>(workspace);
    a.sums = reinterpret_cast<double *>(static_cast<char *>(workspace) + kVerifyCounterBytes);
    const size_t size = dtype == 0 ? 4 : 2;
    // Past the caches what the last one has not kept of the call that wrote it (right
    // behind that call, three drafts, binary32, 128 sequences of 64000: 21.0 us through
    // the caches, 22.7 past them; 192 of 131072 and five drafts 42 and 37).
    a.once = (double)a.n_seqs * (a.Q ? 2 * a.n + 1 : a.n + 1) * a.vocab * size >= (double)kLastCache;
    const int each = kVerifyWaves * a.each;
    const unsigned groups = (unsigned)((a.n_parts + each - 1) / each);
    // (as many sequences at a time as there are counters)
    for (int left = a.n_seqs; left > 0; left -= kVerifySeqs) {
        const int n = left < kVerifySeqs ? left : kVerifySeqs;
        auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(groups, (unsigned)n), dim3(kVerifyThreads), 0, stream, a); };
        if (a.steps == 1)
            dtype == 0 ? go(verify_kernel<float, 1>) : go(verify_kernel<__bf16, 1>);
        else if (a.steps == 2)
            dtype == 0 ? go(verify_kernel<float, 2>) : go(verify_kernel<__bf16, 2>);
        else
            dtype == 0 ? go(verify_kernel<float, 4>) : go(verify_kernel<__bf16, 4>);
        a.P = static_cast<const char *>(a.P) + (int64_t)n * a.p_seq * size;
        if (a.Q) a.Q = static_cast<const char *>(a.Q) + (int64_t)n * a.q_seq * size;
        a.drafts += (int64_t)n * a.n;
        if (a.n_drafts) a.n_drafts += n;
        a.uniforms += (int64_t)n * (a.n + 1);
        if (a.lengths) a.lengths += n;
        a.accepted += n;
        a.tokens += (int64_t)n * (a.n + 1);
    }
    return hipGetLastError();
}

}  // namespace rr
