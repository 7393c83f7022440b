// Sampling: arguments handed from the host layer to the kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

struct FcSampleArgs {
    const void *logits;
    int64_t ld;  // elements from row to row
    int32_t M, V, top_k;
    float top_p, min_p;
    double inv_t;  // 1 / temperature (1 where that is 0)
    int32_t greedy;
    double log_min_p;  // set by the launch, as are the next two
    double bin_width;  // in units of a logit
    int32_t last_bin;  // the last bin that can matter
    const float *u;
    int32_t *tok;
    float *conf;
    void *workspace;
};
size_t fc_sample_workspace(int M, int V);
hipError_t fc_launch_sample(const FcSampleArgs &p, int dtype, hipStream_t s);
