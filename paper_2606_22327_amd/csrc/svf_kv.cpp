// svf_kv.cpp -- host side of include/svfkv.h: the checks of sizes, strides and
// alignment, and the structs that the kernels take.
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>

#include "svf_kv.h"
#include "svfsim.h"

using namespace svfk;

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
constexpr int64_t kStrideLimit = int64_t(1) << 40;  // elements: products with an index stay in 64 bits
constexpr int64_t kGridLimit = kLimit31 - 1;
constexpr int64_t kThreadLimit = int64_t(1) << 32;  // of a launch: what HIP supports is below

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool stride_ok(int64_t s) { return s >= 0 && s < kStrideLimit; }

int check_sizes(const svf_kv_cache* c, const svf_kv_batch* b) {
    if (!c || !b) return fail(SVF_EINVAL, "cache and batch must not be NULL");
    if (c->num_pages < 0 || c->kv_heads < 1 || c->kv_heads > 65535)
        return fail(SVF_EINVAL, "num_pages must be >= 0 and kv_heads in 1 .. 65535 (%d, %d)", c->num_pages, c->kv_heads);
    if (c->page_size < 1 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)))
        return fail(SVF_EINVAL, "page_size must be a power of two, 1 .. 65536 (%d)", c->page_size);
    if ((int64_t)c->num_pages * c->page_size >= kLimit31)
        return fail(SVF_EINVAL, "num_pages * page_size must be below 2^31");
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
        return fail(SVF_EINVAL, "head_dim must be 64, 128 or 256 (%d)", c->head_dim);
    if (c->dtype != SVF_KV_BF16 && c->dtype != SVF_KV_F16) return fail(SVF_EINVAL, "unknown dtype %d", c->dtype);
    if (b->num_seqs < 0 || b->num_tokens < 0 || b->table_width < 0 || b->max_q < 0)
        return fail(SVF_EINVAL, "num_seqs, num_tokens, table_width and max_q must be >= 0");
    if ((int64_t)b->num_seqs * c->kv_heads > kGridLimit) return fail(SVF_EINVAL, "num_seqs * kv_heads is too large");
    if ((int64_t)b->table_width * c->page_size >= kLimit31 - 65536)  // a tile past the last slot is still an int
        return fail(SVF_EINVAL, "table_width * page_size must be below 2^31 - 2^16");
    if (b->table_stride < b->table_width || b->table_stride >= kStrideLimit)
        return fail(SVF_EINVAL, "table_stride must be at least table_width");
    return SVF_OK;
}

int check_buffers(const svf_kv_cache* c, const svf_kv_batch* b) {
    if (c->num_pages > 0 && (!c->k || !c->v)) return fail(SVF_EINVAL, "k and v must not be NULL");
    if (!aligned(c->k, 16) || !aligned(c->v, 16)) return fail(SVF_EINVAL, "k and v must be aligned to 16 bytes");
    const int64_t strides[6] = {c->k_head_stride, c->v_head_stride, c->k_page_stride,
                                c->k_row_stride,  c->v_page_stride, c->v_row_stride};
    for (int i = 0; i < 6; i++)
        if (!stride_ok(strides[i]) || strides[i] % 8 || (i >= 2 && strides[i] >= kLimit31))
            return fail(SVF_EINVAL, "strides of k and v must be multiples of 8, from 0, of pages and rows below 2^31");
    if (b->num_seqs > 0 && (!b->kv_len || (b->table_width > 0 && !b->page_table)))
        return fail(SVF_EINVAL, "kv_len and page_table must not be NULL");
    return SVF_OK;
}

KvView view(const svf_kv_cache* c, const svf_kv_batch* b) {
    KvView v;
    v.k = static_cast<const char*>(c->k);
    v.v = static_cast<const char*>(c->v);
    v.weight = c->weight;
    v.position = c->position;
    v.k_page = c->k_page_stride * 2, v.k_head = c->k_head_stride * 2, v.k_row = c->k_row_stride * 2;
    v.v_page = c->v_page_stride * 2, v.v_head = c->v_head_stride * 2, v.v_row = c->v_row_stride * 2;
    v.q_offsets = b->q_offsets;
    v.kv_len = b->kv_len;
    v.table = b->page_table;
    v.table_stride = b->table_stride;
    v.num_pages = c->num_pages;
    v.shift = __builtin_ctz((unsigned)c->page_size);
    v.kv_heads = c->kv_heads;
    v.seqs = b->num_seqs;
    v.tokens = b->num_tokens;
    v.width = b->table_width;
    v.max_q = b->max_q;
    return v;
}

int check_heads(const svf_kv_cache* c, int32_t heads) {
    if (heads < 1 || heads > 65535 || heads % c->kv_heads)
        return fail(SVF_EINVAL, "heads must be a multiple of kv_heads, at most 65535 (%d, %d)", heads, c->kv_heads);
    return SVF_OK;
}

// A tensor [tokens][heads][dim] of 16-bit elements, strides in elements.
struct Rows {
    const void* at;
    int64_t token, head;
};

// Whether two tensors of one shape share an element: exactly where their strides are equal and rows lie side by side, so that
// parts of one buffer are apart; else by the first and the last address.
bool overlap(Rows a, Rows b, int64_t tokens, int64_t heads, int64_t dim) {
    typedef __int128 Wide;
    if (tokens == 1) a.token = b.token = 0;
    if (heads == 1) a.head = b.head = 0;
    const Wide row = dim * 2, delta = (Wide)reinterpret_cast<uintptr_t>(b.at) - (Wide)reinterpret_cast<uintptr_t>(a.at);
    auto span = [&](const Rows& x) { return ((Wide)x.token * (tokens - 1) + (Wide)x.head * (heads - 1)) * 2 + row; };
    if (delta >= span(a) || -delta >= span(b)) return false;
    const bool outer_token = a.token >= a.head;
    const Wide so = (outer_token ? a.token : a.head) * (Wide)2, si = (outer_token ? a.head : a.token) * (Wide)2;
    const int64_t no = outer_token ? tokens : heads, ni = outer_token ? heads : tokens;
    const bool apart = (ni == 1 || si >= row) && (no == 1 || so >= si * (ni - 1) + row);
    if (a.token != b.token || a.head != b.head || !apart) return true;
    // delta = x so + y si + less than a row either way
    auto below = [](Wide n, Wide d) { return n >= 0 ? n / d : -((-n + d - 1) / d); };
    for (Wide x = no > 1 ? below(delta, so) : 0, x1 = no > 1 ? x + 1 : 0; x <= x1; x++) {
        if (x <= -no || x >= no) continue;
        const Wide rest = delta - x * so;
        for (Wide y = ni > 1 ? below(rest, si) : 0, y1 = ni > 1 ? y + 1 : 0; y <= y1; y++) {
            const Wide off = rest - y * si;
            if (y > -ni && y < ni && off > -row && off < row) return true;
        }
    }
    return false;
}

int launched(hipError_t e) {
    return e == hipSuccess ? SVF_OK : fail(SVF_EHIP, "kernel launch: %s", hipGetErrorString(e));
}

AttendSizes sizes(const svf_kv_cache* c, const svf_kv_batch* b, const svf_kv_attend_args* a, int32_t first = 0) {
    // With first tokens: those, and the windows of max_q rows; else all.
    const int64_t cap = (int64_t)b->table_width * c->page_size, seen = (int64_t)first + a->window + b->max_q + 512;
    const int64_t places = first > 0 && a->window > 0 && seen < cap ? seen : cap;
    return {c->num_pages,  c->page_size, c->kv_heads,    a->heads, c->head_dim, c->dtype,
            b->num_tokens, b->num_seqs,  b->table_width, b->max_q, a->add_weight != 0, first, places};
}

int check_attend(const svf_kv_cache* c, const svf_kv_batch* b, const svf_kv_attend_args* a, int32_t first = 0) {
    if (int rc = check_sizes(c, b)) return rc;
    if (!a) return fail(SVF_EINVAL, "args must not be NULL");
    if (int rc = check_heads(c, a->heads)) return rc;
    if (a->window < 0) return fail(SVF_EINVAL, "window must be >= 0");
    if (first < 0) return fail(SVF_EINVAL, "first must be >= 0");
    if ((int64_t)b->num_tokens * a->heads > kGridLimit) return fail(SVF_EINVAL, "num_tokens * heads is too large");
    if (attend_threads(sizes(c, b, a, first)) >= kThreadLimit)
        return fail(SVF_EINVAL, "num_tokens * heads, num_seqs * kv_heads or the pool is too large for one launch");
    return SVF_OK;
}

int check_evict(const svf_kv_cache* c, const svf_kv_batch* b, const svf_kv_evict_args* a) {
    if (int rc = check_sizes(c, b)) return rc;
    if (!a) return fail(SVF_EINVAL, "args must not be NULL");
    if (a->budget < 1 || a->recent < 0 || a->first < 0 || (int64_t)a->recent + a->first > a->budget)
        return fail(SVF_EINVAL, "budget must be >= 1, recent and first >= 0 and no more than it together (%d, %d, %d)",
                    a->budget, a->recent, a->first);
    return SVF_OK;
}

int64_t evict_bytes(const svf_kv_cache* c, const svf_kv_batch* b, const svf_kv_evict_args* a) {
    const int64_t segs = (int64_t)b->num_seqs * c->kv_heads;
    return ((segs * 4 + 255) & ~int64_t(255)) +
           segs * evict_pairs((int64_t)b->table_width * c->page_size, a->budget) * 8;
}

// svf_kv_append, and svf_kv_append_axes with ``axes``.
int append(const svf_kv_cache* c, const svf_kv_batch* b, const svf_kv_append_args* a, const svf_kv_axes* axes, hipStream_t stream) {
    if (int rc = check_sizes(c, b)) return rc;
    if (!a) return fail(SVF_EINVAL, "args must not be NULL");
    if (int rc = check_buffers(c, b)) return rc;
    if (int rc = check_heads(c, a->heads)) return rc;
    if (a->rot < 0 || a->rot > c->head_dim || a->rot % 2)
        return fail(SVF_EINVAL, "rot must be even, 0 .. head_dim (%d)", a->rot);
    if (a->layout != SVF_KV_ROPE_HALF && a->layout != SVF_KV_ROPE_INTERLEAVED)
        return fail(SVF_EINVAL, "unknown layout %d", a->layout);
    const int64_t strides[8] = {a->q_token_stride, a->q_head_stride, a->k_token_stride, a->k_head_stride,
                                a->v_token_stride, a->v_head_stride, a->out_token_stride, a->out_head_stride};
    bool wide = a->rot % 16 == 0;
    for (int64_t s : strides) {
        if (!stride_ok(s)) return fail(SVF_EINVAL, "strides must be in 0 .. 2^40");
        wide = wide && s % 8 == 0;
    }
    AxesArgs x = {};
    if (axes) {
        if (axes->axes < 1 || axes->axes > SVF_KV_MOST_AXES)
            return fail(SVF_EINVAL, "axes must be in 1 .. %d (%d)", SVF_KV_MOST_AXES, axes->axes);
        if (!stride_ok(axes->token_stride) || !stride_ok(axes->axis_stride))
            return fail(SVF_EINVAL, "strides of positions must be in 0 .. 2^40");
        for (int i = 0; i < a->rot / 2; i++) {
            if (axes->of_pair[i] >= axes->axes)
                return fail(SVF_EINVAL, "of_pair must be below axes (pair %d: %d)", i, axes->of_pair[i]);
            x.of_pair[i / 16] |= (uint32_t)axes->of_pair[i] << 2 * (i % 16);
        }
        x.kept = axes->kept;
        x.token = axes->token_stride, x.axis = axes->axis_stride;
        x.axes = axes->axes;
    }
    if (b->num_tokens == 0 || b->num_seqs == 0) return SVF_OK;
    if (!b->q_offsets || !a->q || !a->k || !a->v || !a->q_out || !a->positions)
        return fail(SVF_EINVAL, "q_offsets, q, k, v, q_out and positions must not be NULL");
    const Rows q = {a->q, a->q_token_stride, a->q_head_stride}, q_out = {a->q_out, a->out_token_stride, a->out_head_stride};
    if (a->q != a->q_out && overlap(q, q_out, b->num_tokens, a->heads, c->head_dim))
        return fail(SVF_EINVAL, "q_out must be q itself or apart from it");
    if (a->rot > 0 && (!a->rope || a->rope_rows < 1)) return fail(SVF_EINVAL, "the table of positions must not be empty");
    if ((int64_t)b->num_tokens * (a->heads + 2 * c->kv_heads) > kGridLimit)
        return fail(SVF_EINVAL, "num_tokens * heads is too large");
    if (a->q == a->q_out && (a->q_token_stride != a->out_token_stride || a->q_head_stride != a->out_head_stride))
        return fail(SVF_EINVAL, "q_out in place of q needs its strides");
    wide = wide && aligned(a->q, 16) && aligned(a->k, 16) && aligned(a->v, 16) && aligned(a->q_out, 16);
    AppendArgs k;
    k.kv = view(c, b);
    k.q = static_cast<const char*>(a->q);
    k.kn = static_cast<const char*>(a->k);
    k.vn = static_cast<const char*>(a->v);
    k.q_out = static_cast<char*>(a->q_out);
    k.positions = a->positions;
    k.rope = a->rope;
    k.q_tok = a->q_token_stride * 2, k.q_head = a->q_head_stride * 2;
    k.k_tok = a->k_token_stride * 2, k.k_head = a->k_head_stride * 2;
    k.v_tok = a->v_token_stride * 2, k.v_head = a->v_head_stride * 2;
    k.o_tok = a->out_token_stride * 2, k.o_head = a->out_head_stride * 2;
    k.heads = a->heads;
    k.rot = a->rot;
    k.half_layout = a->layout == SVF_KV_ROPE_HALF;
    k.rope_rows = a->rope_rows;
    k.dim = c->head_dim;
    if ((axes ? append_axes_threads(k) : append_threads(k, wide)) >= kThreadLimit)
        return fail(SVF_EINVAL, "num_tokens is too large (%d)", b->num_tokens);
    return launched(axes ? launch_append_axes(k, x, c->dtype, stream) : launch_append(k, c->dtype, wide, stream));
}

// svf_kv_attend, and svf_kv_attend_first.
int attend(const svf_kv_cache* c, const svf_kv_batch* b, const svf_kv_attend_args* a, int32_t first, hipStream_t stream) {
    if (int rc = check_attend(c, b, a, first)) return rc;
    if (int rc = check_buffers(c, b)) return rc;
    if (!stride_ok(a->q_token_stride) || !stride_ok(a->q_head_stride))
        return fail(SVF_EINVAL, "strides of q must be in 0 .. 2^40");
    if (!stride_ok(a->out_token_stride) || !stride_ok(a->out_head_stride) || a->out_token_stride % 8 ||
        a->out_head_stride % 8)
        return fail(SVF_EINVAL, "strides of out must be multiples of 8, 0 .. 2^40");
    const float scale = a->scale * 1.4426950408889634f;  // for powers of two
    if (!(scale - scale == 0.f)) return fail(SVF_EINVAL, "scale must be a finite number below 2^127");
    if (a->add_weight && !c->weight && c->num_pages > 0) return fail(SVF_EINVAL, "add_weight needs the cache's weight");
    if (b->num_tokens == 0 || b->num_seqs == 0) return SVF_OK;
    if (!b->q_offsets || !a->q || !a->out || !a->lse) return fail(SVF_EINVAL, "q_offsets, q, out and lse must not be NULL");
    if (!aligned(a->out, 16)) return fail(SVF_EINVAL, "out must be aligned to 16 bytes");
    const int64_t need = attend_workspace(sizes(c, b, a, first));
    if (a->workspace_bytes < need || (need > 0 && !a->workspace) || !aligned(a->workspace, 256))
        return fail(SVF_EINVAL, "workspace must have %lld bytes, aligned to 256", (long long)need);
    const Rows q = {a->q, a->q_token_stride, a->q_head_stride}, out = {a->out, a->out_token_stride, a->out_head_stride};
    if (overlap(q, out, b->num_tokens, a->heads, c->head_dim)) return fail(SVF_EINVAL, "out must be apart from q");
    AttendArgs k;
    k.kv = view(c, b);
    k.q = static_cast<const char*>(a->q);
    k.out = static_cast<char*>(a->out);
    k.lse = a->lse;
    k.ws = static_cast<char*>(a->workspace);
    k.q_tok = a->q_token_stride * 2, k.q_head = a->q_head_stride * 2;
    k.o_tok = a->out_token_stride * 2, k.o_head = a->out_head_stride * 2;
    k.scale = scale;
    k.heads = a->heads;
    k.causal = a->causal != 0;
    // a window as wide as the table hides nothing, and a slot less than it is still an int
    k.window = a->window < (int64_t)b->table_width * c->page_size ? a->window : 0;
    // without a window every token stays visible; the table has no more of them than this
    k.first = k.window == 0 ? 0 : first < (int64_t)b->table_width * c->page_size ? first : b->table_width * c->page_size;
    k.add_weight = a->add_weight != 0;
    k.q_wide = aligned(a->q, 16) && a->q_token_stride % 8 == 0 && a->q_head_stride % 8 == 0;
    return launched(launch_attend(k, sizes(c, b, a, k.first), stream));
}

}  // namespace

extern "C" {

const char* svf_kv_last_error(void) { return g_err; }

int svf_kv_append(const svf_kv_cache* c, const svf_kv_batch* b, const svf_kv_append_args* a, void* hip_stream) {
    return append(c, b, a, nullptr, static_cast<hipStream_t>(hip_stream));
}

int svf_kv_append_axes(const svf_kv_cache* c, const svf_kv_batch* b, const svf_kv_append_args* a, const svf_kv_axes* axes,
                       void* hip_stream) {
    if (!axes) return fail(SVF_EINVAL, "axes must not be NULL");
    return append(c, b, a, axes, static_cast<hipStream_t>(hip_stream));
}

int64_t svf_kv_attend_workspace(const svf_kv_cache* c, const svf_kv_batch* b, const svf_kv_attend_args* a) {
    if (int rc = check_attend(c, b, a)) return rc;
    return attend_workspace(sizes(c, b, a));
}

int svf_kv_attend(const svf_kv_cache* c, const svf_kv_batch* b, const svf_kv_attend_args* a, void* hip_stream) {
    return attend(c, b, a, 0, static_cast<hipStream_t>(hip_stream));
}

int64_t svf_kv_attend_first_workspace(const svf_kv_cache* c, const svf_kv_batch* b, const svf_kv_attend_args* a, int32_t first) {
    if (int rc = check_attend(c, b, a, first)) return rc;
    return attend_workspace(sizes(c, b, a, first));
}

int svf_kv_attend_first(const svf_kv_cache* c, const svf_kv_batch* b, const svf_kv_attend_args* a, int32_t first, void* hip_stream) {
    return attend(c, b, a, first, static_cast<hipStream_t>(hip_stream));
}

int64_t svf_kv_evict_workspace(const svf_kv_cache* c, const svf_kv_batch* b, const svf_kv_evict_args* a) {
    if (int rc = check_evict(c, b, a)) return rc;
    return evict_bytes(c, b, a);
}

int svf_kv_evict(const svf_kv_cache* c, const svf_kv_batch* b, const svf_kv_evict_args* a, void* hip_stream) {
    if (int rc = check_evict(c, b, a)) return rc;
    if (int rc = check_buffers(c, b)) return rc;
    if (b->num_seqs == 0) return SVF_OK;
    if (c->num_pages > 0 && (!c->weight || !c->position))
        return fail(SVF_EINVAL, "eviction needs the cache's weight and position");
    if (!a->next_position || !a->new_len) return fail(SVF_EINVAL, "next_position and new_len must not be NULL");
    if (a->new_len == b->kv_len) return fail(SVF_EINVAL, "new_len must not be kv_len");
    const int64_t need = evict_bytes(c, b, a);
    if (a->workspace_bytes < need || !a->workspace || !aligned(a->workspace, 256))
        return fail(SVF_EINVAL, "workspace must have %lld bytes, aligned to 256", (long long)need);
    EvictArgs k;
    k.kv = view(c, b);
    k.next = a->next_position;
    k.new_len = a->new_len;
    k.ws = static_cast<char*>(a->workspace);
    k.budget = a->budget;
    k.recent = a->recent;
    k.first = a->first;
    k.row_bytes = c->head_dim * 2;
    if (evict_threads(k) >= kThreadLimit) return fail(SVF_EINVAL, "num_seqs * kv_heads is too large");
    return launched(launch_evict(k, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
