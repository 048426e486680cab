// svf_kv_chunk.hip -- attention over the paged cache of sequences with many rows
// (new tokens times query heads of a key head): prompts and their pieces.
#include "svf_kv_attend.h"

namespace svfk {
namespace {

constexpr int kRows = 128;  // rows of a workgroup, 32 for each of its four waves
constexpr int kTile = 64;   // slots that it takes at a time

// Whether these kernels take the sequence, and not those of few rows.
__device__ inline bool ours(const AttendArgs& p, const Seq& s) {
    if (s.n > p.kv.max_q) return p.few == 0;
    return (int64_t)s.n * (p.heads / p.kv.kv_heads) > p.few;
}

__device__ inline int row_tiles(const AttendArgs& p, const Seq& s) {
    return s.n > 0 && ours(p, s) ? (int)(((int64_t)s.n * (p.heads / p.kv.kv_heads) + kRows - 1) / kRows) : 0;
}

// Finds what ``count`` numbers: the sequence that item ``at`` of all sequences' items
// belongs to, and the item's number in it. For a whole workgroup of 256; false where there are fewer items.
template <class Count>
__device__ inline bool find_item(const KvView& kv, int64_t at, Count count, int64_t* scan, int& seq, int& item) {
    __shared__ int sh_seq, sh_item;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (kv.seqs + 255) / 256;
    const int i0 = min(tid * per, kv.seqs), i1 = min(i0 + per, kv.seqs);
    int64_t mine = 0;
    for (int i = i0; i < i1; i++) mine += count(seq_of(kv, i));
    int64_t incl = mine;
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t x = __shfl_up(incl, d);
        if (lane >= d) incl += x;
    }
    if (lane == 63) scan[wave] = incl;
    if (tid == 0) sh_seq = -1;
    __syncthreads();
    int64_t before = incl - mine;
    for (int w = 0; w < wave; w++) before += scan[w];
    if (before <= at && at < before + mine) {
        for (int i = i0; i < i1; i++) {
            const int c = count(seq_of(kv, i));
            if (at < before + c) {
                sh_seq = i;
                sh_item = (int)(at - before);
                break;
            }
            before += c;
        }
    }
    __syncthreads();
    seq = sh_seq;
    item = sh_item;
    return seq >= 0;
}

// Rows of the tile in LDS lie one behind the other, their 16-byte pieces permuted so that the lanes of
// a read meet every bank alike: sixteen rows' same piece (keys), and eight rows' four neighbouring
// pieces (values, read transposed).
template <int D>
__device__ inline int swizzle(int row) {
    return D == 64 ? (row >> 1 & 1) << 2 | (row >> 2 & 3) : (row & 3) << 2 | (row >> 2 & 3);
}

// S^T = K Q^T and O^T = V^T P^T on 32x32x16 products. In both a lane has one row (l % 32), so a
// row's maximum and sum take one exchange between the wave's halves and its scaling none; the
// scores of a lane are, in order, the second product's operand for the slots 16 s + 4 h + {0..3, 8..11}
// (h the half), and the values of those slots come transposed out of LDS, four slots a read.
// Keys and values go from memory straight to LDS, the next tile's while this one is worked on.
template <class E, int D>
__global__ __launch_bounds__(256, (D <= 128 ? 2 : 1)) void k_attend_chunk(AttendArgs p) {
    using T = typename E::T;
    using V8 = typename E::V8;
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* Lds4;
    constexpr int KS = D / 16, DT = D / 32, CH = D / 8, BUF = kTile * D * 2;
    __shared__ __align__(16) char lds[4 * BUF];  // keys and values, twice
    __shared__ uint32_t odd_marks[kRows][D / 16];
    __shared__ int64_t scan[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 31, h = lane >> 5;
    const int G = p.heads / p.kv.kv_heads, hk = p.kv.kv_heads;
    const int head = blockIdx.x % hk;
    int seq, tile;
    if (!find_item(p.kv, blockIdx.x / hk, [&](const Seq& s) { return row_tiles(p, s); }, scan, seq, tile)) return;
    const Seq s = seq_of(p.kv, seq);
    if (s.n > p.kv.max_q) {
        if (tile == 0) fill_nan<T, D>(p, s, head, G, tid, 256);
        return;
    }
    tile = row_tiles(p, s) - 1 - tile;  // the longest first
    const int rows = s.n * G, r0 = s.len - s.n;
    const int first_row = tile * kRows, last_row = min(first_row + kRows, rows) - 1;
    const int lo = p.window > 0 ? max(0, r0 + first_row / G - p.window + 1) : 0;
    const int hi = p.causal ? min(s.len, r0 + last_row / G + 1) : s.len;
    const int tiles = hi > lo ? (hi - lo + kTile - 1) / kTile : 0;

    // this lane's row, and the slots that all and any of the wave's rows see
    const int row = first_row + wave * 32 + c;
    const int t = min(row, rows - 1) / G;
    const int last = p.causal ? r0 + t : s.len - 1, from = p.window > 0 ? r0 + t - p.window + 1 : 0;
    const int wrow0 = first_row + wave * 32, wt0 = min(wrow0, rows - 1) / G, wt1 = min(wrow0 + 31, rows - 1) / G;
    const int all_last = p.causal ? r0 + wt0 : s.len - 1, any_last = p.causal ? r0 + wt1 : s.len - 1;
    const int all_from = p.window > 0 ? r0 + wt1 - p.window + 1 : 0;
    const int any_from = p.window > 0 ? r0 + wt0 - p.window + 1 : 0;

    // Scores are compared before they are scaled: the queries take the scale's sign.
    const float sign = p.scale < 0.f ? -1.f : 1.f, scale = p.scale == 0.f ? 1.f : fabsf(p.scale);
    V8 q[KS];
    {
        const char* at = p.q + (s.q0 + t) * p.q_tok + (head * G + min(row, rows - 1) - t * G) * p.q_head;
#pragma unroll
        for (int k = 0; k < KS; k++) {
            if (p.q_wide) {
                q[k] = *(const V8*)(at + (k * 16 + h * 8) * 2);
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++) q[k][i] = *(const T*)(at + (k * 16 + h * 8 + i) * 2);
            }
            if (p.scale <= 0.f) {
#pragma unroll
                for (int i = 0; i < 8; i++) q[k][i] = (T)((float)q[k][i] * (p.scale == 0.f ? 0.f : sign));
            }
        }
    }
    for (int i = tid; i < kRows * (D / 16); i += 256) (&odd_marks[0][0])[i] = 0;
    __syncthreads();

    const char* kbase = p.kv.k + head * p.kv.k_head;
    const char* vbase = p.kv.v + head * p.kv.v_head;
    // a lane has the addresses of slot ``lane`` of a tile
    struct Where {
        uint64_t k, v;
        bool there;
    };
    auto lookup = [&](int it) {
        const int j = lo + it * kTile + lane;
        const int at = it < tiles && j < hi ? pool_row(p.kv, seq, j) : -1;
        Where w;
        w.there = at >= 0;
        w.k = w.v = (uint64_t)zero_row();
        if (w.there) {
            w.k = (uint64_t)kbase + row_offset(at, p.kv.shift, p.kv.k_page, p.kv.k_row);
            w.v = (uint64_t)vbase + row_offset(at, p.kv.shift, p.kv.v_page, p.kv.v_row);
        }
        return w;
    };
    auto from_lane = [](uint64_t x, int l) {
        const uint32_t a = __shfl((int)(uint32_t)x, l), b = __shfl((int)(x >> 32), l);
        return (uint64_t)b << 32 | a;
    };
    typedef const __attribute__((address_space(1))) void* Global;
    typedef __attribute__((address_space(3))) void* Lds;
    auto fetch = [&](const Where& w, int buf) {
#pragma unroll
        for (int i = 0; i < CH / 4; i++) {
            const int piece = (wave * (CH / 4) + i) * 64, at = piece + lane;
            const int r = at / CH, x = ((at % CH) ^ swizzle<D>(r)) * 16;
            __builtin_amdgcn_global_load_lds((Global)(from_lane(w.k, r) + x), (Lds)(lds + (2 * buf) * BUF + piece * 16), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((Global)(from_lane(w.v, r) + x), (Lds)(lds + (2 * buf + 1) * BUF + piece * 16), 16, 0, 0);
        }
    };

    float m = -INFINITY, l = 0.f;
    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) o[d][i] = 0.f;

    Where now = lookup(0), next = lookup(1);
    if (tiles > 0) fetch(now, 0);
    auto step = [&](int it, int buf) {
        // this tile is there once every wave's loads have arrived, and the other buffer free
        __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
        __syncthreads();
        const uint64_t there = __ballot(now.there);
        if (it + 1 < tiles) fetch(next, buf ^ 1);
        now = next;
        next = lookup(it + 2);
        const int base = lo + it * kTile;
        if (base > any_last || base + kTile - 1 < any_from) return;
        const char* kb = lds + 2 * buf * BUF;
        const char* vb = kb + BUF;
        f32x16 sc[2];
#pragma unroll
        for (int st = 0; st < 2; st++) {
#pragma unroll
            for (int i = 0; i < 16; i++) sc[st][i] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; k++) {
                const int r = st * 32 + c;
                const V8 a = *(const V8*)(kb + r * (D * 2) + ((2 * k + h) ^ swizzle<D>(c)) * 16);
                sc[st] = E::mfma32(a, q[k], sc[st]);
            }
        }
        const bool whole = base + kTile - 1 <= all_last && base >= all_from && ~there == 0;
        if (!whole) {
#pragma unroll
            for (int st = 0; st < 2; st++)
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const int off = st * 32 + (i >> 2) * 8 + h * 4 + (i & 3), j = base + off;
                    if (!(there >> off & 1) || j > last || j < from) sc[st][i] = -INFINITY;
                }
        }
        float top = sc[0][0];
#pragma unroll
        for (int i = 0; i < 16; i++) top = fmaxf(top, fmaxf(sc[0][i], sc[1][i]));
        top = fmaxf(top, __shfl_xor(top, 32)) * scale;
        if (__any(top > m + E::kSlack)) {
            const float peak = fmaxf(m, top);
            const float keep = peak == -INFINITY ? 1.f : exp2_fast(m - peak);
            m = peak;
            l *= keep;
#pragma unroll
            for (int d = 0; d < DT; d++)
#pragma unroll
                for (int i = 0; i < 16; i++) o[d][i] *= keep;
        }
        const float ref = (m == -INFINITY ? 0.f : m) - E::kShift;
        V8 pr[4];
#pragma unroll
        for (int st = 0; st < 2; st++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const float e = exp2_fast(fmaf(sc[st][i], scale, -ref));
                l += e;
                pr[st * 2 + (i >> 3)][i & 7] = (T)e;
            }
        // Where rows do not see the same slots, a value that is no finite number would reach those that
        // do not see it (0 times infinity): it counts as 0, and the rows that see it get it from its marks.
        bool odd = false;
        if (!whole) {
            u16x2 size = {0, 0};
            for (int r = lane & 1; r < kTile; r += 2)
                for (int x = lane >> 1; x < D / 2; x += 32)
                    size = __builtin_elementwise_max(size, __builtin_bit_cast(u16x2, *(const uint32_t*)(vb + r * (D * 2) + x * 4) & 0x7fff7fffu));
            odd = __any(max(size.x, size.y) >= E::kInf);
            if (odd) {
                for (int r = lane & 1; r < kTile; r += 2)
                    for (int x = lane >> 1; x < D / 2; x += 32) {
                        const uint32_t pair = *(const uint32_t*)(vb + r * (D * 2) + x * 4);
                        if (!odd_pair<E>(pair)) continue;
                        const int w = ((x >> 2) ^ swizzle<D>(r)) * 4 + (x & 3);  // the dimensions 2 w and 2 w + 1
                        const uint32_t marks = odd_marks_of<E>(pair) << 4 * (w & 7);
                        for (int y = 0; y < 32 && wrow0 + y < rows; y++) {
                            const int at = r0 + (wrow0 + y) / G;
                            if ((!p.causal || base + r <= at) && (p.window == 0 || base + r > at - p.window))
                                atomicOr(&odd_marks[wave * 32 + y][w >> 3], marks);
                        }
                    }
            }
        }
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
            for (int d = 0; d < DT; d++) {
                s16x4 part[2];
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    // 16 lanes give four slots' rows, four dimensions each, and get four slots of one dimension
                    const int r = k * 16 + i * 8 + h * 4 + (lane >> 2 & 3), dim = d * 32 + (lane >> 4 & 1) * 16 + (lane & 3) * 4;
                    part[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)(vb + r * (D * 2) + ((dim >> 3) ^ swizzle<D>(r)) * 16 + (dim & 7) * 2));
                }
                uint2 a = __builtin_bit_cast(uint2, part[0]), b = __builtin_bit_cast(uint2, part[1]);
                if (odd) a = make_uint2(finite_pair<E>(a.x), finite_pair<E>(a.y)), b = make_uint2(finite_pair<E>(b.x), finite_pair<E>(b.y));
                o[d] = E::mfma32(__builtin_bit_cast(V8, make_uint4(a.x, a.y, b.x, b.y)), pr[k], o[d]);
            }
    };
    for (int it = 0; it < tiles; it += 2) {
        step(it, 0);
        if (it + 1 < tiles) step(it + 1, 1);
    }

    if (row < rows) {
        l += __shfl_xor(l, 32);
        const int hq = head * G + row - t * G;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        char* out = p.out + (s.q0 + t) * p.o_tok + hq * p.o_head;
        typedef T V4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int d = 0; d < DT; d++)
#pragma unroll
            for (int b = 0; b < 4; b++) {
                const int dim = d * 32 + b * 8 + h * 4;
                float x[4] = {o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]};
                add_marks(odd_marks[wave * 32 + c][dim >> 4] >> 2 * (dim & 15), x, 4);
                *(V4*)(out + dim * 2) = V4{(T)(x[0] * inv), (T)(x[1] * inv), (T)(x[2] * inv), (T)(x[3] * inv)};
            }
        if (h == 0) p.lse[(int64_t)(s.q0 + t) * p.heads + hq] = (m - E::kShift + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
    }
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
hipError_t launch(const AttendArgs& a, const AttendSizes& z, hipStream_t s) {
    // Row tiles at most: the full ones of all tokens, and one more for each sequence that is long enough to come here.
    const int64_t rows = (int64_t)z.tokens * (z.heads / z.kv_heads), seqs = rows / (a.few + 1);
    const int64_t blocks = (rows / kRows + (seqs < z.seqs ? seqs : z.seqs)) * z.kv_heads;
    if (blocks > 0) k_attend_chunk<E, D><<<(unsigned)blocks, 256, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.add_weight && a.kv.width > 0) {
        const unsigned n = (unsigned)((((int64_t)a.kv.width << a.kv.shift) + 255) / 256);
        k_weight<E, D><<<dim3(n, a.kv.kv_heads, a.kv.seqs), 256, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk(const AttendArgs& a, const AttendSizes& z, hipStream_t s) {
    if (z.dtype == SVF_KV_BF16)
        return z.dim == 64 ? launch<BF16M, 64>(a, z, s) : z.dim == 128 ? launch<BF16M, 128>(a, z, s) : launch<BF16M, 256>(a, z, s);
    return z.dim == 64 ? launch<F16M, 64>(a, z, s) : z.dim == 128 ? launch<F16M, 128>(a, z, s) : launch<F16M, 256>(a, z, s);
}

// A call's launches: single tokens and short chunks, and, where a sequence may have more rows, chunks.
int64_t attend_workspace(const AttendSizes& z) { return rows_workspace(z); }

hipError_t launch_attend(AttendArgs a, const AttendSizes& z, hipStream_t s) {
    a.few = few_rows(z);
    if (a.few) {
        const hipError_t e = launch_rows(a, z, a.ws, s);
        if (e != hipSuccess || (int64_t)z.max_q * (z.heads / z.kv_heads) <= a.few) return e;
    }
    return launch_chunk(a, z, s);
}

}  // namespace svfk
