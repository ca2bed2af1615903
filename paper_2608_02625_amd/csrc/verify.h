// Host-side launcher of the verification of drafted tokens (verify.hip); the entry
// point that checks its arguments is in cache.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/dlm.h"

constexpr int kVerifyMaxRows = 1024;     // a sequence's rows stand in one workgroup's LDS

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
    int32_t *path, *removed;
    void* verdicts;
    double *sums, *rest, *inverse;
};
int64_t verify_workgroups(int total_rows, int vocab);
size_t verify_workspace_bytes(int n_seqs, int total_rows, int vocab, bool draft);
hipError_t launch_verify(VerifyArgs a, int dtype, void* ws, hipStream_t st);
