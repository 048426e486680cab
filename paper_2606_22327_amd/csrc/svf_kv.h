// svf_kv.h -- internal interface between the host checks and the gfx950
// kernels of the paged key-value cache (not part of the public ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "svfkv.h"

namespace svfk {

// A layer's cache and a call's sequences as the kernels see them.
struct KvView {
    const char* k;
    const char* v;
    float* weight;      // or null
    int32_t* position;  // or null
    int64_t k_page, k_head, k_row, v_page, v_head, v_row;  // bytes
    const int32_t* q_offsets;
    const int32_t* kv_len;
    const int32_t* table;
    int64_t table_stride;
    int32_t num_pages, shift, kv_heads;  // page_size == 1 << shift
    int32_t seqs, tokens, width, max_q;
};

struct AppendArgs {
    KvView kv;
    const char *q, *kn, *vn;
    char* q_out;
    const int32_t* positions;
    const float* rope;
    int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head;  // bytes
    int32_t heads, rot, half_layout, rope_rows, dim;
};

// Positions with several axes.
struct AxesArgs {
    const int32_t* kept;  // or null: axis 0's
    int64_t token, axis;  // strides of the positions, elements
    int32_t axes;
    uint32_t of_pair[8];  // two bits a pair
};

struct AttendArgs {
    KvView kv;
    const char* q;
    char* out;
    float* lse;
    char* ws;
    int64_t q_tok, q_head, o_tok, o_head;  // bytes
    float scale;  // times log2(e)
    int32_t heads, causal, window, add_weight;
    int32_t first;   // slots that stay visible before the window
    int32_t q_wide;  // q can be read 16 bytes at a time
    int32_t few;     // rows of a key head up to which the kernels of few rows take a sequence
};

// The sizes that an attention call's workspace and launches go by.
struct AttendSizes {
    int32_t num_pages, page_size, kv_heads, heads, dim, dtype, tokens, seqs, width, max_q, add_weight, first;
    int64_t places;  // slots of a sequence that its rows see at most, with what rounding to pieces of up to 256 adds
};

struct EvictArgs {
    KvView kv;
    const int32_t* next;
    int32_t* new_len;
    char* ws;
    int32_t budget, recent, first, row_bytes;
};

hipError_t launch_append(const AppendArgs& a, int32_t dtype, bool wide, hipStream_t s);
hipError_t launch_append_axes(const AppendArgs& a, const AxesArgs& x, int32_t dtype, hipStream_t s);
hipError_t launch_attend(AttendArgs a, const AttendSizes& z, hipStream_t s);
hipError_t launch_evict(const EvictArgs& a, hipStream_t s);
int64_t attend_workspace(const AttendSizes& z);
// Threads of the largest launch.
int64_t append_threads(const AppendArgs& a, bool wide);
int64_t append_axes_threads(const AppendArgs& a);
int64_t attend_threads(const AttendSizes& z);
int64_t evict_threads(const EvictArgs& a);

// The kernels of few rows (svf_kv_rows.hip).
int32_t few_rows(const AttendSizes& z);
int64_t rows_workspace(const AttendSizes& z);
int64_t rows_blocks(const AttendSizes& z);
hipError_t launch_rows(const AttendArgs& a, const AttendSizes& z, char* ws, hipStream_t s);

// Pairs (hole, mover) that one sequence's key head can have.
inline int64_t evict_pairs(int64_t capacity, int64_t budget) {
    return capacity <= budget ? 0 : (capacity - budget < budget ? capacity - budget : budget);
}

}  // namespace svfk
