// svf_logprob_host.cpp -- host side of include/svflogprob.h: the checks, and the struct that the kernels take.
#include "svf_logprob.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "svfsim.h"

namespace {

// message of the calling thread's last failure
thread_local char g_err[256];

int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int fail(int code, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof g_err, fmt, ap);
    va_end(ap);
    return code;
}

constexpr int64_t kLimit31 = int64_t(1) << 31;
constexpr int64_t kStrideLimit = int64_t(1) << 40;  // elements: products with a row stay in 64 bits
constexpr int64_t kThreadLimit = int64_t(1) << 32;  // of a launch: what HIP supports is below

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int64_t item(const svf_logprob_args* a) { return a->dtype == SVF_LOGITS_F32 ? 4 : 2; }

int check(const svf_logprob_args* a) {
    if (!a) return fail(SVF_EINVAL, "args must not be NULL");
    if (a->rows < 0 || a->vocab < 1 || a->vocab > SVF_LOGPROB_MOST_VOCAB)
        return fail(SVF_EINVAL, "rows must be >= 0 and vocab in 1 .. %d (%d, %d)", SVF_LOGPROB_MOST_VOCAB, a->rows, a->vocab);
    if (a->top < 0 || a->top > SVF_LOGPROB_MOST_TOP || a->top > a->vocab)
        return fail(SVF_EINVAL, "top must be in 0 .. %d and no more than vocab (%d, %d)", SVF_LOGPROB_MOST_TOP, a->top, a->vocab);
    if (a->dtype != SVF_LOGITS_BF16 && a->dtype != SVF_LOGITS_F16 && a->dtype != SVF_LOGITS_F32)
        return fail(SVF_EINVAL, "unknown dtype %d", a->dtype);
    if ((int64_t)a->rows * a->top >= kLimit31) return fail(SVF_EINVAL, "rows * top must be below 2^31");
    if (svfp::threads(a->rows, a->vocab, a->top, a->dtype) >= kThreadLimit) return fail(SVF_EINVAL, "rows is too large (%d)", a->rows);
    return SVF_OK;
}

}  // namespace

extern "C" {

const char* svf_logprob_last_error(void) { return g_err; }

int64_t svf_logprob_workspace(const svf_logprob_args* a) {
    if (int rc = check(a)) return rc;
    return svfp::workspace(a->rows, a->vocab, a->top, a->dtype);
}

int svf_logprob(const svf_logprob_args* a, void* hip_stream) {
    if (int rc = check(a)) return rc;
    if (a->row_stride < 0 || a->row_stride >= kStrideLimit) return fail(SVF_EINVAL, "row_stride must be in 0 .. 2^40");
    if (a->token_bytes != 4 && a->token_bytes != 8) return fail(SVF_EINVAL, "token_bytes must be 4 or 8 (%d)", a->token_bytes);
    const float scale = a->scale * 1.4426950408889634f;  // for powers of two; twice that is a number too
    if (!(scale > 0.f) || !(a->scale < 0x1p126f)) return fail(SVF_EINVAL, "scale must be above 0 and below 2^126");
    if (a->rows == 0) return SVF_OK;
    if (!a->logits || !a->token || !a->logprob || !a->entropy || !a->rank || (a->top > 0 && (!a->top_logprob || !a->top_index)))
        return fail(SVF_EINVAL, "logits, token and outputs must not be NULL");
    if (!aligned(a->logits, item(a)) || !aligned(a->token, a->token_bytes))
        return fail(SVF_EINVAL, "logits and token must be aligned to their type");
    const int64_t need = svfp::workspace(a->rows, a->vocab, a->top, a->dtype);
    if (a->workspace_bytes < need || (need > 0 && !a->workspace) || !aligned(a->workspace, 256))
        return fail(SVF_EINVAL, "workspace must have %lld bytes, aligned to 256", (long long)need);
    svfp::Args k;
    k.logits = static_cast<const char*>(a->logits);
    k.token = static_cast<const char*>(a->token);
    k.logprob = a->logprob;
    k.entropy = a->entropy;
    k.rank = a->rank;
    k.top_logprob = a->top_logprob;
    k.top_index = a->top_index;
    k.ws = static_cast<char*>(a->workspace);
    k.row_stride = a->row_stride * item(a);
    k.scale = a->scale, k.scale2 = scale;
    k.low = svfp::kFarthest / scale;
    k.rows = a->rows;
    k.vocab = a->vocab;
    k.top = a->top;
    k.token_wide = a->token_bytes == 8;
    const hipError_t e = svfp::launch(k, a->dtype, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? SVF_OK : fail(SVF_EHIP, "kernel launch: %s", hipGetErrorString(e));
}

}  // extern "C"
