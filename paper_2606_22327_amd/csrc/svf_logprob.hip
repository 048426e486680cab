// svf_logprob.hip -- log probabilities of given tokens, entropies and the best alternatives of rows of logits.
#include "svf_kv_device.h"
#include "svf_logprob.h"

namespace svfp {
namespace {

constexpr float kLn2 = 0.69314718055994531f;

// A logit's place in the order as a whole number, larger first: -0 as 0, NaN below all.
__device__ inline uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return x != x ? 0u : u >> 31 ? ~u : u | 0x80000000u;
}
// With the index behind it, so that no two are equal.
__device__ inline uint64_t key_of(float x, int i) { return (uint64_t)order_of(x) << 32 | (uint32_t)~i; }

__device__ inline int64_t token_of(const Args& p, int row) {
    return p.token_wide ? ((const int64_t*)p.token)[row] : ((const int32_t*)p.token)[row];
}

template <class V, class Op>
__device__ inline V over_group(V x, Op op) {
    __shared__ V part[4];
    for (int d = 32; d; d >>= 1) x = op(x, __shfl_xor(x, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    return op(op(part[0], part[1]), op(part[2], part[3]));
}

// A row by a workgroup, one sum after another.
template <class T>
__global__ __launch_bounds__(256) void k_logprob(Args p) {
    const int row = blockIdx.x, tid = threadIdx.x, V = p.vocab;
    const T* x = (const T*)(p.logits + row * p.row_stride);
    auto add = [](auto a, auto b) { return a + b; };
    const int64_t token = token_of(p, row);
    const bool known = token >= 0 && token < V;
    const uint64_t mine = known ? key_of((float)x[token], (int)token) : 0;
    float m = -INFINITY, bad = 0.f;
    int before = 0;
    for (int i = tid; i < V; i += 256) {
        const float y = (float)x[i];
        m = fmaxf(m, y);
        bad += y == INFINITY || y != y ? 1.f : 0.f;
        before += key_of(y, i) > mine;
    }
    m = over_group(m, [](float a, float b) { return fmaxf(a, b); });
    bad = over_group(bad, add);
    before = over_group(before, add);
    const bool none = m == -INFINITY;
    float s = 0.f, sx = 0.f;
    for (int i = tid; i < V && !none; i += 256) {
        const float y = (0.5f * (float)x[i] - 0.5f * m) * (2.f * p.scale2), e = __builtin_amdgcn_exp2f(y);
        s += e;
        sx += e * fmaxf(y, -200.f);  // 0 times -infinity is 0
    }
    s = over_group(s, add);
    sx = over_group(sx, add);
    // (halves, and in natural terms: no difference of two numbers passes what 32 bits hold on the way)
    const float total = __builtin_amdgcn_logf(s) * kLn2, nan = __builtin_nanf("");
    auto lp = [&](float y) { return bad != 0.f ? nan : none ? -INFINITY : (0.5f * y - 0.5f * m) * (2.f * p.scale) - total; };
    if (tid == 0) {
        p.logprob[row] = known ? lp((float)x[token]) : nan;
        p.entropy[row] = bad != 0.f ? nan : none ? 0.f : total - sx / s * kLn2;
        p.rank[row] = known ? before : -1;
    }
    uint64_t last = ~0ull;
    for (int k = 0; k < p.top; k++) {
        uint64_t best = 0;
        for (int i = tid; i < V; i += 256) {
            const uint64_t key = key_of((float)x[i], i);
            if (key < last && key > best) best = key;
        }
        last = over_group(best, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
        if (tid == 0) {
            const int at = (int)~(uint32_t)last;
            p.top_index[row * p.top + k] = at;
            p.top_logprob[row * p.top + k] = lp((float)x[at]);
        }
    }
}

}  // namespace

int64_t workspace(int32_t, int32_t, int32_t, int32_t) { return 0; }

int64_t threads(int32_t rows, int32_t, int32_t, int32_t) { return (int64_t)rows * 256; }

hipError_t launch(const Args& a, int32_t dtype, hipStream_t s) {
    const dim3 grid(a.rows);
    return dtype == SVF_LOGITS_BF16  ? svfk::run(k_logprob<__bf16>, grid, 256, s, a)
           : dtype == SVF_LOGITS_F16 ? svfk::run(k_logprob<_Float16>, grid, 256, s, a)
                                     : svfk::run(k_logprob<float>, grid, 256, s, a);
}

}  // namespace svfp
