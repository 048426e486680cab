// svf_logprob.h -- internal interface between the host checks and the gfx950
// kernels of include/svflogprob.h (not part of the public ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "svflogprob.h"

namespace svfp {

// No lane's reference lies below this in log2 terms: it would be rounded by more than 2^-4, and from some -2^31 on powers relative to it would
// be infinite.  A lane with lower logits alone (a mask's finite number) adds 0, as it should, where the row has larger ones;
// where it has none, and where references are as far above 0, all is summed again.
constexpr float kFarthest = -1048576.f;

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
    float scale, scale2, low;  // scale2: times log2(e); low: the logit that comes to kFarthest
    int32_t rows, vocab, top, token_wide;
};

int64_t workspace(int32_t rows, int32_t vocab, int32_t top, int32_t dtype);
// Threads of the largest launch.
int64_t threads(int32_t rows, int32_t vocab, int32_t top, int32_t dtype);
hipError_t launch(const Args& a, int32_t dtype, hipStream_t s);

}  // namespace svfp
