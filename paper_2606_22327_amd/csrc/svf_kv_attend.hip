// svf_kv_attend.hip -- attention of new tokens over the paged cache.
#include "svf_kv_attend.h"

namespace svfk {
namespace {

// Whether these kernels take the sequence, and not those of few rows.
__device__ inline bool ours(const AttendArgs& p, const Seq& s) {
    if (s.n > p.kv.max_q) return p.few == 0;
    return (int64_t)s.n * (p.heads / p.kv.kv_heads) > p.few;
}

// Row (t, h): one wave; a lane scores one slot at a time, then the wave adds
// up the values of 64 slots, a lane for D / 64 dimensions.
template <class E, int D>
__global__ __launch_bounds__(64) void k_attend(AttendArgs p) {
    using T = typename E::T;
    const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
    const int seq = find_seq(p.kv, t);
    const Seq s = seq_of(p.kv, seq);
    if (t < s.q0 || t >= s.q0 + s.n || !ours(p, s)) return;
    const int head = h / (p.heads / p.kv.kv_heads);
    const int r = s.len - s.n + (t - s.q0);
    const int hi = p.causal ? r + 1 : s.len, lo = p.window > 0 ? max(0, r - p.window + 1) : 0;
    __shared__ float q[D];
    __shared__ float prob[64];
    __shared__ int rows[64];
    const T* qp = (const T*)(p.q + t * p.q_tok + h * p.q_head);
    for (int d = lane; d < D; d += 64) q[d] = (float)qp[d] * p.scale;
    __syncthreads();
    float m = -INFINITY, l = 0.f, acc[D / 64];
    for (int i = 0; i < D / 64; i++) acc[i] = 0.f;
    for (int j0 = lo; j0 < hi; j0 += 64) {
        const int j = j0 + lane;
        const int row = j < hi ? pool_row(p.kv, seq, j) : -1;
        float sc = -INFINITY;
        if (row >= 0) {
            const T* k = (const T*)(p.kv.k + head * p.kv.k_head + row_offset(row, p.kv.shift, p.kv.k_page, p.kv.k_row));
            sc = 0.f;
            for (int d = 0; d < D; d++) sc += q[d] * (float)k[d];
        }
        float top = sc;
        for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
        const float nm = fmaxf(m, top), base = nm == -INFINITY ? 0.f : nm;
        const float e = exp2f(sc - base), old = exp2f(m - base);
        float sum = e;
        for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
        l = l * old + sum;
        m = nm;
        prob[lane] = e;
        rows[lane] = row;
        __syncthreads();
        for (int i = 0; i < D / 64; i++) acc[i] *= old;
        for (int x = 0; x < 64; x++) {
            if (rows[x] < 0) continue;
            const T* v = (const T*)(p.kv.v + head * p.kv.v_head + row_offset(rows[x], p.kv.shift, p.kv.v_page, p.kv.v_row));
            for (int i = 0; i < D / 64; i++) acc[i] += prob[x] * (float)v[lane + 64 * i];
        }
        __syncthreads();
    }
    T* o = (T*)(p.out + t * p.o_tok + h * p.o_head);
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    const bool over = s.n > p.kv.max_q;
    for (int i = 0; i < D / 64; i++) o[lane + 64 * i] = (T)(over ? __builtin_nanf("") : acc[i] * inv);
    if (lane == 0) p.lse[(int64_t)t * p.heads + h] = over ? __builtin_nanf("") : (m + log2f(l)) * 0.69314718055994531f;
}

// A thread has one slot: its softmax summed over the rows in order.
template <class E, int D>
__global__ __launch_bounds__(256) void k_weight(AttendArgs p) {
    using T = typename E::T;
    const int j = blockIdx.x * 256 + threadIdx.x, head = blockIdx.y, seq = blockIdx.z;
    const Seq s = seq_of(p.kv, seq);
    if (j >= s.len || s.n > p.kv.max_q || !ours(p, s)) return;
    const int row = pool_row(p.kv, seq, j);
    if (row < 0) return;
    const T* k = (const T*)(p.kv.k + head * p.kv.k_head + row_offset(row, p.kv.shift, p.kv.k_page, p.kv.k_row));
    const int G = p.heads / p.kv.kv_heads;
    float sum = 0.f;
    for (int t = s.q0; t < s.q0 + s.n; t++) {
        const int r = s.len - s.n + (t - s.q0);
        if ((p.causal && j > r) || (p.window > 0 && j <= r - p.window)) continue;
        for (int g = 0; g < G; g++) {
            const int h = head * G + g;
            const float lse = p.lse[(int64_t)t * p.heads + h] * 1.4426950408889634f;
            const T* qp = (const T*)(p.q + t * p.q_tok + h * p.q_head);
            float sc = 0.f;
            for (int d = 0; d < D; d++) sc += (float)qp[d] * p.scale * (float)k[d];
            if (lse != -INFINITY) sum += exp2f(sc - lse);
        }
    }
    p.kv.weight[stat_index(p.kv, row, head)] += sum;
}

template <class E, int D>
hipError_t launch(const AttendArgs& a, hipStream_t s) {
    if (a.kv.tokens > 0) {
        k_attend<E, D><<<dim3(a.kv.tokens, a.heads), 64, 0, s>>>(a);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.add_weight && a.kv.width > 0) {
        const unsigned blocks = (unsigned)((((int64_t)a.kv.width << a.kv.shift) + 255) / 256);
        k_weight<E, D><<<dim3(blocks, a.kv.kv_heads, a.kv.seqs), 256, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

int64_t attend_workspace(const AttendSizes& z) { return rows_workspace(z); }

hipError_t launch_attend(AttendArgs a, const AttendSizes& z, hipStream_t s) {
    a.few = few_rows(z);
    if (a.few) {
        hipError_t e = launch_rows(a, z, a.ws, s);
        if (e != hipSuccess || (int64_t)z.max_q * (z.heads / z.kv_heads) <= a.few) return e;
    }
    if (z.dtype == SVF_KV_BF16)
        return z.dim == 64 ? launch<BF16, 64>(a, s) : z.dim == 128 ? launch<BF16, 128>(a, s) : launch<BF16, 256>(a, s);
    return z.dim == 64 ? launch<F16, 64>(a, s) : z.dim == 128 ? launch<F16, 128>(a, s) : launch<F16, 256>(a, s);
}

}  // namespace svfk
