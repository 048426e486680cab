// svf_kv_device.h -- what the kernels of the paged key-value cache share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "svf_kv.h"

namespace svfk {

// A launch with its own error: hipGetLastError would also report one that a call before has left.
template <class X>
struct As {
    typedef X Type;
};
template <class... P>
inline hipError_t run(void (*kernel)(P...), dim3 grid, unsigned threads, hipStream_t s, typename As<P>::Type... args) {
    void* at[] = {&args...};
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), at, 0, s);
    if (e != hipSuccess) (void)hipGetLastError();  // reported here
    return e;
}

// A load that the compiler knows to be of global memory, whatever the address was chosen from.
template <class V>
__device__ inline V load_global(uint64_t at) {
    typedef const __attribute__((address_space(1))) V* G;
    return *(G)at;
}

// A sequence of the batch: its new tokens are q rows [q0, q0 + n), its slots [0, len).
struct Seq {
    int q0, n, len;
};

__device__ inline int clampi(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

__device__ inline int seq_len(const KvView& kv, int i) {
    return clampi(kv.kv_len[i], 0, kv.width << kv.shift);
}

__device__ inline Seq seq_of(const KvView& kv, int i) {
    Seq s;
    s.q0 = clampi(kv.q_offsets[i], 0, kv.tokens);
    s.n = clampi(kv.q_offsets[i + 1], s.q0, kv.tokens) - s.q0;
    s.len = seq_len(kv, i);
    return s;
}

// The last sequence whose new tokens begin at or before ``token``: 64 offsets
// are compared at a time, so the search takes one load for 64 sequences, two for 4096.
// Called by whole waves with the same token in every lane.
__device__ inline int find_seq(const KvView& kv, int token) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = kv.seqs;  // the answer lies in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 63) >> 6;
        const int at = lane * step;
        const bool le = at < n && kv.q_offsets[lo + at] <= token;
        const int hits = __popcll(__ballot(le));
        const int k = hits > 0 ? hits - 1 : 0;
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

// The pool row (page << shift | row) of slot j, or -1 where there is none.
__device__ inline int pool_row(const KvView& kv, int seq, int j) {
    const int page = kv.table[(int64_t)seq * kv.table_stride + (j >> kv.shift)];
    const bool there = (unsigned)page < (unsigned)kv.num_pages;
    return there ? (page << kv.shift) | (j & ((1 << kv.shift) - 1)) : -1;
}

// The same in two steps, so that the load can be on its way while the row before it is used: the
// table's entry, of the nearest slot that the sequence has (there is no branch in it: at its end the
// compiler would wait for every load on its way; entries behind its length are not read, and where it has no slot
// ``zero`` is read instead) ...
struct Table {
    uint64_t base;
    int last;
};
__host__ __device__ inline Table table_of(const KvView& kv, int seq, int len, const void* zero) {
    Table t;
    t.last = len > 0 ? (len - 1) >> kv.shift : 0;
    t.base = len > 0 ? (uint64_t)(kv.table + (int64_t)seq * kv.table_stride) : (uint64_t)zero;
    return t;
}
__device__ inline int table_entry(const KvView& kv, const Table& t, int j) {
    return load_global<int32_t>(t.base + (uint64_t)(uint32_t)clampi(j >> kv.shift, 0, t.last) * 4);
}
// ... and its row, -1 unless the slot is ``in`` range and the page there.
__device__ inline int entry_row(const KvView& kv, int page, int j, bool in) {
    const int row = page << kv.shift | (j & ((1 << kv.shift) - 1));
    return in && (unsigned)page < (unsigned)kv.num_pages ? row : -1;
}

// Where a pool's rows lie: the address of a row of a page (strides are below 2^32 bytes).
__device__ inline uint64_t row_address(uint64_t base, int page, int row, int64_t page_stride, int64_t row_stride) {
    return base + (uint64_t)(uint32_t)page * (uint32_t)page_stride + (uint64_t)(uint32_t)row * (uint32_t)row_stride;
}

__device__ inline int64_t row_offset(int row, int shift, int64_t page_stride, int64_t row_stride) {
    return (int64_t)(row >> shift) * page_stride + (int64_t)(row & ((1 << shift) - 1)) * row_stride;
}

// Index of a pool row's entry in weight and position.
__device__ inline int64_t stat_index(const KvView& kv, int row, int head) {
    const int64_t page = row >> kv.shift;
    return ((page * kv.kv_heads + head) << kv.shift) + (row & ((1 << kv.shift) - 1));
}

struct BF16 {
    using T = __bf16;
    typedef __bf16 V8 __attribute__((ext_vector_type(8)));
};
struct F16 {
    using T = _Float16;
    typedef _Float16 V8 __attribute__((ext_vector_type(8)));
};

}  // namespace svfk
