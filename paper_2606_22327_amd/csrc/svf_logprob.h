// svf_logprob.h -- internal interface between the host checks and the gfx950
// kernels of include/svflogprob.h (not part of the public ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "svflogprob.h"

namespace svfp {

struct Args {
    const char* logits;
    const char* token;
    float* logprob;
    float* entropy;
    int32_t* rank;
    float* top_logprob;
    int32_t* top_index;
    char* ws;
    int64_t row_stride;  // bytes
    float scale, scale2;  // scale2: times log2(e)
    int32_t rows, vocab, top, token_wide;
};

int64_t workspace(int32_t rows, int32_t vocab, int32_t top, int32_t dtype);
// Threads of the largest launch.
int64_t threads(int32_t rows, int32_t vocab, int32_t top, int32_t dtype);
hipError_t launch(const Args& a, int32_t dtype, hipStream_t s);

}  // namespace svfp
