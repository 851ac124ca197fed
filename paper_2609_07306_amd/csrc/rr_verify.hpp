// Arguments of the verification of drafted tokens (rr_verify.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace rr {

// Sequences of a launch: each has a counter, in 64 bytes of its own (those of one
// line are added to one after the other: 32 sequences in 32 workgroups each 15.7
// us side by side, 7.9 so).
constexpr int kVerifySeqs = 1024, kVerifyApart = 16;
constexpr size_t kVerifyCounterBytes = kVerifySeqs * kVerifyApart * sizeof(uint32_t);

struct VerifyArgs {
    const void *P, *Q;  // [B, n + 1, V] and [B, n, V] with strides; Q or null
    const int32_t *drafts, *n_drafts;  // [B, n]; [B] or null
    const float *uniforms;             // [B, n + 1]
    int32_t *lengths;                  // [B] or null
    int32_t *accepted, *tokens;        // [B], [B, n + 1]
    int64_t p_seq, p_row, q_seq, q_row;  // elements between rows
    int32_t n_seqs, n, vocab;
    int32_t steps;    // of a part of a row
    int32_t n_parts;  // of a row
    int32_t each;     // parts of a wave
    bool once;        // rows are read past the caches
    uint32_t *counters;  // [n_seqs] kVerifyApart apart, finished workgroups, 0 between calls
    double *sums;        // [n_seqs, n_parts]
};

// Fills in the split of a row, from n_seqs and vocab.
void verify_schedule(VerifyArgs &a, int dtype);
size_t verify_workspace_bytes(const VerifyArgs &a);
hipError_t launch_verify(const VerifyArgs &a, int dtype, void *workspace, hipStream_t stream);

}  // namespace rr
