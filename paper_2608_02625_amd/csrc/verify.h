// Host-side launcher of the verification of drafted tokens (verify.hip); the entry
// point that checks its arguments is in cache.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/dlm.h"

constexpr int kVerifyMaxRows = 1024;     // a sequence's rows stand in one workgroup's LDS
constexpr int kVerifyRowWords = kVerifyMaxRows / 32;

struct VerifyArgs {
    int n_seqs, total_rows, max_rows, vocab;
    const int32_t *row_start, *tokens, *parent;
    const void *target, *draft;
    int64_t target_stride, draft_stride;
    double c;                            // log2(e) / temperature; 0: the largest logit decides
    float cf;
    const float *u, *u_next;
    int32_t *next, *keep, *keep_start;
    // workspace
    void* parts;
    uint32_t *kept, *removed;            // a bit per row of a window, kVerifyRowWords per sequence
    void* verdicts;
    double *sums, *rest, *inverse;
};
// A grid for n workgroups, counted along x first, the last ones idle: an axis takes fewer
// than 2^32 threads, the second one at most 65535 workgroups.
constexpr int kVerifyThreads = 256;
struct VerifyGrid {
    unsigned x, y;
};
constexpr VerifyGrid verify_grid(int64_t n) {
    constexpr int64_t across = 1 << 16;
    return {(unsigned)(n < across ? n : across), (unsigned)((n + across - 1) / across)};
}
constexpr int64_t kVerifyMaxWorkgroups = 0x7fffffff;
static_assert((int64_t)verify_grid(kVerifyMaxWorkgroups).x * kVerifyThreads < (int64_t)1 << 32 &&
              verify_grid(kVerifyMaxWorkgroups).y <= 65535, "every size that is taken can be launched");
int64_t verify_workgroups(int total_rows, int vocab);
size_t verify_workspace_bytes(int n_seqs, int total_rows, int vocab, bool draft);
hipError_t launch_verify(VerifyArgs a, int dtype, void* ws, hipStream_t st);
