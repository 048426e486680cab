// svf_kv_chunk.hip -- attention over the paged cache of sequences with many rows
// (new tokens times query heads of a key head): prompts and their pieces.
#include "svf_kv_attend.h"

namespace svfk {
namespace {

constexpr int kRows = 128;  // rows of a workgroup, 32 for each of its four waves
constexpr int kTile = 64;   // slots that it takes at a time

// A row tile of a key head whose slots are split, and what its parts are joined by.
struct Item {
    int32_t q0, first_row, rows, parts;
};
constexpr int kMostParts = 64;

struct ChunkPlan {
    int32_t groups;  // workgroups that the GPU holds; 0: no tile is split
    int32_t* items;  // row tiles over all key heads, 0 where none is split
    Item* item;      // [groups / 2]
    float* part;     // [groups][kRows][D + 4]
};

// The arguments of k_attend_chunk as they lie in memory.
struct ChunkCall {
    AttendArgs p;
    ChunkPlan plan;
};

// Whether these kernels take the sequence, and not those of few rows.
__device__ inline bool ours(const AttendArgs& p, const Seq& s) {
    if (s.n > p.kv.max_q) return p.few == 0;
    return (int64_t)s.n * (p.heads / p.kv.kv_heads) > p.few;
}

__device__ inline int row_tiles(const AttendArgs& p, const Seq& s) {
    return s.n > 0 && ours(p, s) ? (int)(((int64_t)s.n * (p.heads / p.kv.kv_heads) + kRows - 1) / kRows) : 0;
}

// Finds what ``count`` numbers: the sequence that item ``at`` of all sequences' items
// belongs to, and the item's number in it; ``place`` makes ``at`` from the number of all items.
// For a whole workgroup of 256; false where there is no such item.
template <class Count, class Place>
__device__ inline bool find_item(const KvView& kv, Place place, Count count, int64_t* scan, int& seq, int& item) {
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
    int64_t before = incl - mine, total = 0;
    for (int w = 0; w < 4; w++) {
        if (w < wave) before += scan[w];
        total += scan[w];
    }
    const int64_t at = place(total);
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

// The bits from .. last, both included, of those that a word has.
__device__ inline uint64_t bits_between(int from, int last) {
    if (last < 0 || from > 63 || from > last) return 0;
    const uint64_t below = last >= 63 ? ~0ull : (2ull << last) - 1;
    return from <= 0 ? below : below & (~0ull << from);
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
//
// The probabilities enter the second product as the sum of two numbers of the type, as with few rows: in one, their rounding would be an
// error of the size of the output's own (2.3e-3 in place of 1.7e-3 of the outputs' norm in bfloat16, for 412 us in place of 512 of
// six prompts).  A row's maximum is followed only when it has grown by more than kSlack.
//
// Products and exponentials bound it together: 2,048 tokens behind 12,001 (32 query heads on 8 key heads of 128 dimensions, 437 GFLOP,
// 656 with the second product's two halves) take 590 us, six prompts of 1,084 to 3,930 tokens (348, 522 with both) 505 us in a row of
// calls and 549 under the profiler: 950 to 1,110 TFLOP/s of products carried out, where a large one of the library reaches 1,350.
// Counters of the prompts: the matrix units are busy for 0.48 of the cycles, other vector instructions take 0.36 at four cycles
// each, and exponentials, at sixteen, 0.12 more; two waves a SIMD do not fill the waits between.
// WIDE: pages of 16 slots or more, so that the sixteen slots that a wave fetches lie in one page: their address is the same for
// the whole wave but for an offset that stays the same all along (a tile costs a wave 8 loads and some scalar
// instructions, and 100 vector instructions otherwise).
template <class E, int D, bool WIDE>
__global__ __launch_bounds__(256, (D <= 128 ? 2 : 1)) void k_attend_chunk(AttendArgs p, ChunkPlan plan) {
    using T = typename E::T;
    using V8 = typename E::V8;
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* Lds4;
    constexpr int KS = D / 16, DT = D / 32, CH = D / 8, BUF = kTile * D * 2;
    // keys and values twice, each an object of its own: reads of one do not wait for loads into another
    __shared__ __align__(16) char k0[BUF], v0[BUF], k1[BUF], v1[BUF];
    __shared__ uint32_t odd_marks[kRows][D / 16];
    __shared__ int64_t scan[4];
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = p.heads / p.kv.kv_heads, hk = p.kv.kv_heads;
    int seq, tile, item = 0, part = 0, parts = 1;
    const bool found = find_item(
        p.kv,
        [&](int64_t total) {
            // Few row tiles: as many parts of each one's slots as there is room for, all first parts first.
            const int64_t all = total * hk;
            if (plan.groups > 0 && all > 0) parts = (int)min((int64_t)kMostParts, max((int64_t)1, plan.groups / all));
            if (plan.groups > 0 && blockIdx.x == 0 && threadIdx.x == 0) *plan.items = parts > 1 ? (int)all : 0;
            if (blockIdx.x >= all * parts) return total;
            part = (int)(blockIdx.x / all);
            item = (int)(blockIdx.x - part * all);
            return (int64_t)(item / hk);
        },
        [&](const Seq& s) { return row_tiles(p, s); }, scan, seq, tile);
    if (!found) return;
    const int head = item % hk;
    const Seq s = seq_of(p.kv, seq);
    if (s.n > p.kv.max_q) {
        if (tile == 0 && part == 0) fill_nan<T, D>(p, s, head, G, tid, 256);
        if (parts > 1 && part == 0 && tid == 0) plan.item[item] = Item{0, 0, 0, 0};
        return;
    }
    tile = row_tiles(p, s) - 1 - tile;  // the longest first
    const int rows = s.n * G, r0 = s.len - s.n;
    const int first_row = tile * kRows, last_row = min(first_row + kRows, rows) - 1;
    int lo = p.window > 0 ? max(0, r0 + first_row / G - p.window + 1) & ~15 : 0;
    int hi = p.causal ? min(s.len, r0 + last_row / G + 1) : s.len;
    int tiles = hi > lo ? (hi - lo + kTile - 1) / kTile : 0;
    if (parts > 1) {
        // No part of fewer than four tiles: it would cost more to join than it saves.  (40 tokens of 32 query heads on 8 key heads behind
        // 2,000 slots: parts of one tile and more 28.0 us, of two 23.0, of four 21.8, of eight 26.1; behind 4,000: 28.8, 30.2, 27.5,
        // 30.1; behind 500, where one is best: 17.6, 18.5, 21.2, 26.6.)
        parts = max(1, min(parts, tiles / 4));
        if (part >= parts) return;
        if (part == 0 && tid == 0) plan.item[item] = Item{s.q0, first_row, rows, parts};
        const int from = (int)((int64_t)tiles * part / parts), to = (int)((int64_t)tiles * (part + 1) / parts);
        hi = min(hi, lo + to * kTile);
        lo += from * kTile;
        tiles = to - from;
    }

    // this lane's row, and the slots that all and any of the wave's rows see
    const int row = first_row + wave * 32 + c;
    const int t = min(row, rows - 1) / G;
    const int last = p.causal ? r0 + t : s.len - 1, from = p.window > 0 ? r0 + t - p.window + 1 : 0;
    const int wrow0 = first_row + wave * 32, wt0 = min(wrow0, rows - 1) / G, wt1 = min(wrow0 + 31, rows - 1) / G;
    const int all_last = p.causal ? r0 + wt0 : s.len - 1, any_last = p.causal ? r0 + wt1 : s.len - 1;
    const int all_from = p.window > 0 ? r0 + wt1 - p.window + 1 : 0;
    const int any_from = p.window > 0 ? r0 + wt0 - p.window + 1 : 0;
    const int block_last = p.causal ? r0 + first_row / G : s.len - 1;
    const int block_from = p.window > 0 ? r0 + last_row / G - p.window + 1 : 0;

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

    const uint64_t kbase = (uint64_t)(p.kv.k + head * p.kv.k_head), vbase = (uint64_t)(p.kv.v + head * p.kv.v_head);
    const Table table = table_of(p.kv, seq, s.len, zero_row());
    const int mask = (1 << p.kv.shift) - 1;
    // A wave fetches sixteen of a tile's slots, 64 / CH of them with an instruction; a lane's
    // slot of instruction i is own + i * 64 / CH.
    constexpr int NI = CH / 4, PER = 64 / CH;
    const int own = wave * 16 + lane / CH;
    int page[NI], page_all;  // of the lane's slots (not WIDE), and of slot ``lane``
    uint32_t koff[NI], voff[NI];  // WIDE: of the lane's piece from the first of the sixteen slots
#pragma unroll
    for (int i = 0; i < NI; i++) {
        const int r = lane / CH + i * PER, x = ((lane % CH) ^ swizzle<D>(r)) * 16;
        koff[i] = (uint32_t)r * (uint32_t)p.kv.k_row + x;
        voff[i] = (uint32_t)r * (uint32_t)p.kv.v_row + x;
    }
    auto look = [&](int it) {
        page_all = table_entry(p.kv, table, lo + it * kTile + lane);
        if constexpr (!WIDE) {
#pragma unroll
            for (int i = 0; i < NI; i++) page[i] = table_entry(p.kv, table, lo + it * kTile + own + i * PER);
        }
    };
    typedef const __attribute__((address_space(1))) char* Global;
    typedef __attribute__((address_space(3))) void* Lds;
    auto load = [](Global from, char* to) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (Lds)to, 16, 0, 0);
    };
    uint64_t there, there_next;
    auto fetch = [&](int it, char* kto, char* vto) {
        const int j0 = lo + it * kTile;
        there_next = __ballot((unsigned)page_all < (unsigned)p.kv.num_pages && j0 + lane < hi);
        kto += wave * NI * 1024;
        vto += wave * NI * 1024;
        if constexpr (WIDE) {
            // Slots behind the last one are read with the others: they are there, and their values count as 0.
            if (there_next >> (wave * 16) & 1) {
                const int at = __builtin_amdgcn_readlane(page_all, wave * 16), row = (j0 + wave * 16) & mask;
                const Global k = (Global)row_address(kbase, at, row, p.kv.k_page, p.kv.k_row);
                const Global v = (Global)row_address(vbase, at, row, p.kv.v_page, p.kv.v_row);
#pragma unroll
                for (int i = 0; i < NI; i++) load(k + koff[i], kto + i * 1024), load(v + voff[i], vto + i * 1024);
            } else {
#pragma unroll
                for (int i = 0; i < NI; i++) {
                    const Global zero = (Global)(uint64_t)zero_row() + lane % CH * 16;
                    load(zero, kto + i * 1024), load(zero, vto + i * 1024);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < NI; i++) {
                const int r = own + i * PER, j = j0 + r, x = ((lane % CH) ^ swizzle<D>(r)) * 16;
                const bool in = (unsigned)page[i] < (unsigned)p.kv.num_pages && j < hi;
                const uint64_t k = in ? row_address(kbase, page[i], j & mask, p.kv.k_page, p.kv.k_row) : (uint64_t)zero_row();
                const uint64_t v = in ? row_address(vbase, page[i], j & mask, p.kv.v_page, p.kv.v_row) : (uint64_t)zero_row();
                load((Global)(k + x), kto + i * 1024), load((Global)(v + x), vto + i * 1024);
            }
        }
    };
    // Where the tile's rows do not all see the same slots, a value that is no finite number would reach those
    // that do not see it (0 times infinity): it counts as 0, and the rows that see it get it
    // from their marks.  Each wave looks through the values of sixteen slots.
    // A tile whose slots all rows see is not looked through: there such a value can make no number of a sum, but only of sums that
    // it decides, and those are found at the end by being no finite numbers.
    auto clean = [&](char* vb, int base) {
        u16x2 size = {0, 0};
        uint32_t* words = (uint32_t*)(vb + wave * 16 * D * 2) + lane;
        for (int x = 0; x < 8 * D; x += 64) size = __builtin_elementwise_max(size, __builtin_bit_cast(u16x2, words[x] & 0x7fff7fffu));
        if (!__any(max(size.x, size.y) >= E::kInf)) return;
        for (int x = 0; x < 8 * D; x += 64) {
            const uint32_t pair = words[x];
            if (!odd_pair<E>(pair)) continue;
            const int r = wave * 16 + (x + lane) / (D / 2), at = (x + lane) % (D / 2);
            const int w = ((at >> 2) ^ swizzle<D>(r)) * 4 + (at & 3);  // the dimensions 2 w and 2 w + 1
            const uint32_t marks = odd_marks_of<E>(pair) << 4 * (w & 7);
            for (int y = 0; y <= last_row - first_row; y++) {
                const int t = r0 + (first_row + y) / G;
                if ((there >> r & 1) && (!p.causal || base + r <= t) && (p.window == 0 || base + r > t - p.window))
                    atomicOr(&odd_marks[y][w >> 3], marks);
            }
            words[x] = finite_pair<E>(pair);
        }
    };

    // Where a lane reads in a tile: keys, 16 bytes of row c, and values, eight bytes of the rows that it gives for
    // the transposed read (16 lanes give four slots' rows, four dimensions each, and get four
    // slots of one dimension).  Kept in registers; what is constant goes into the reads' offsets.
    constexpr int KA = KS < 8 ? KS : 8, VA = DT < 4 ? DT : 4;
    int ka[KA], va[VA][2];
#pragma unroll
    for (int k = 0; k < KA; k++) {
        ka[k] = c * (D * 2) + ((2 * k + h) ^ swizzle<D>(c)) * 16;
        asm volatile("" : "+v"(ka[k]));
    }
#pragma unroll
    for (int d = 0; d < VA; d++)
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int r = i * 8 + h * 4 + (lane >> 2 & 3), dim = d * 32 + (lane >> 4 & 1) * 16 + (lane & 3) * 4;
            va[d][i] = r * (D * 2) + ((dim >> 3) ^ swizzle<D>(r)) * 16 + (dim & 7) * 2;
            asm volatile("" : "+v"(va[d][i]));
        }

    float m = -INFINITY, l = 0.f;
    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) o[d][i] = 0.f;

    if (tiles > 0) {
        look(0);
        fetch(0, k0, v0);
        look(1);
    }
    auto step = [&](int it, char* kb, char* vb, char* knext, char* vnext) {
        // this tile is there once every wave's loads have arrived, and the other buffers free
        __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
        __syncthreads();
        there = there_next;
        if (it + 1 < tiles) {
            fetch(it + 1, knext, vnext);
            look(it + 2);
        }
        const int base = lo + it * kTile;
        if (!(base + kTile - 1 <= block_last && base >= block_from && ~there == 0)) {
            clean(vb, base);
            __syncthreads();
        }
        if (base > any_last || base + kTile - 1 < any_from) return;
        f32x16 sc[2];
#pragma unroll
        for (int st = 0; st < 2; st++)
#pragma unroll
            for (int i = 0; i < 16; i++) sc[st][i] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; k++)
#pragma unroll
            for (int st = 0; st < 2; st++)
                sc[st] = E::mfma32(*(const V8*)(kb + ka[k % KA] + st * 32 * (D * 2) + k / KA * 256), q[k], sc[st]);
        // reads two products ahead of their use
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int i = 0; i < 2 * KS - 4; i++) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
        if (!(base + kTile - 1 <= all_last && base >= all_from && ~there == 0)) {
            // bit (i / 4) * 8 + i % 4 of a word: whether the lane's row sees the slot of score i
            const uint64_t seen = (there & bits_between(from - base, last - base)) >> (h * 4);
#pragma unroll
            for (int st = 0; st < 2; st++) {
                const uint32_t word = (uint32_t)(seen >> (st * 32));
#pragma unroll
                for (int i = 0; i < 16; i++)
                    if (!(word >> ((i >> 2) * 8 + (i & 3)) & 1)) sc[st][i] = -INFINITY;
            }
        }
        float top = max3(sc[0][0], sc[0][1], sc[0][2]);
#pragma unroll
        for (int i = 3; i < 15; i += 2) top = max3(top, sc[0][i], sc[0][i + 1]);
        top = max3(top, sc[0][15], sc[1][0]);
#pragma unroll
        for (int i = 1; i < 15; i += 2) top = max3(top, sc[1][i], sc[1][i + 1]);
        top = fmaxf(top, sc[1][15]);
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
        // Eight probabilities of a lane at a time, exponentials among the products of the eight before; values are read
        // two products ahead of their use.
        auto value = [&](int n) {
            const int k = n / DT, d = n % DT;
            s16x4 part[2];
#pragma unroll
            for (int i = 0; i < 2; i++)
                part[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)(vb + va[d % VA][i] + k * 16 * (D * 2) + d / VA * 256));
            const uint2 a = __builtin_bit_cast(uint2, part[0]), b = __builtin_bit_cast(uint2, part[1]);
            return __builtin_bit_cast(V8, make_uint4(a.x, a.y, b.x, b.y));
        };
        V8 v[3] = {value(0), value(1), value(2)};
#pragma unroll
        for (int k = 0; k < 4; k++) {
            uint4 hi, low;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int x = (k & 1) * 8 + 2 * i;
                const float a = exp2_fast(fmaf(sc[k >> 1][x], scale, -ref)), b = exp2_fast(fmaf(sc[k >> 1][x + 1], scale, -ref));
                l += a, l += b;
                E::split(a, b, (&hi.x)[i], (&low.x)[i]);
            }
#pragma unroll
            for (int d = 0; d < DT; d++) {
                const int n = k * DT + d;
                o[d] = E::mfma32(v[n % 3], __builtin_bit_cast(V8, hi), o[d]);
                o[d] = E::mfma32(v[n % 3], __builtin_bit_cast(V8, low), o[d]);
                if (n + 3 < 4 * DT) v[n % 3] = value(n + 3);
            }
        }
        // a product, then an even part of the vector instructions of the next eight probabilities
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 1);
        __builtin_amdgcn_sched_group_barrier(0x002, 48, 1);
#pragma unroll
        for (int i = 0; i < 4 * DT; i++) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
            __builtin_amdgcn_sched_group_barrier(0x002, 24 / DT, 1);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
            __builtin_amdgcn_sched_group_barrier(0x002, 24 / DT, 1);
        }
    };
    for (int it = 0; it < tiles; it += 2) {
        step(it, k0, v0, k1, v1);
        if (it + 1 < tiles) step(it + 1, k1, v1, k0, v0);
    }

    // What is needed from here on only is read from here on only: kept in registers through the loop, it costs the loop its schedule
    // (the arguments lie in memory in this order).
    typedef const __attribute__((address_space(4))) ChunkCall* Call;
    Call call = (Call)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(call));
    const AttendArgs& z = ((const ChunkCall*)call)->p;
    // Rows with a sum that is no finite number (0 times a finite one is 0), though the row's own sum of probabilities is one: a tile that
    // all rows see has a value that is none. Each thread looks through two dimensions of the slots that all rows see.
    float zero = 0.f;
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) zero = fmaf(o[d][i], 0.f, zero);
    if (__syncthreads_or(zero != 0.f && l * 0.f == 0.f)) {
        const int w = tid % (D / 2);  // the dimensions 2 w and 2 w + 1
        const int first = max(lo, block_from), end = min(hi - 1, block_last) + 1;
        uint32_t marks = 0;
#pragma unroll 8
        for (int j = first + tid / (D / 2); j < end; j += 256 / (D / 2)) {
            const int at = entry_row(z.kv, table_entry(z.kv, table, j), j, true);
            const uint64_t from = at < 0 ? (uint64_t)zero_row() : vbase + row_offset(at, z.kv.shift, z.kv.v_page, z.kv.v_row);
            marks |= odd_marks_of<E>(load_global<uint32_t>(from + w * 4));
        }
        if (marks)
            for (int y = 0; y < kRows; y++) atomicOr(&odd_marks[y][w >> 3], marks << 4 * (w & 7));
        __syncthreads();
    }

    l += __shfl_xor(l, 32);
    if (row >= rows) return;
    const int hq = head * G + row - t * G;
    const float inv = 1.f / l;
    char* out = z.out + (s.q0 + t) * z.o_tok + hq * z.o_head;
    float* to = nullptr;
    if (parts > 1) to = ((const ChunkCall*)call)->plan.part + ((int64_t)blockIdx.x * kRows + wave * 32 + c) * (D + 4);
    typedef T V4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
        for (int b = 0; b < 4; b++) {
            const int dim = d * 32 + b * 8 + h * 4;
            float x[4] = {o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]};
            set_marked(odd_marks[wave * 32 + c][dim >> 4] >> 2 * (dim & 15), x, 4);
            if (to) {
                *(f32x4*)(to + dim) = f32x4{x[0], x[1], x[2], x[3]};
            } else {
                V4 y;
#pragma unroll
                for (int i = 0; i < 4; i++) y[i] = (T)(l == 0.f ? 0.f : x[i] * inv);
                *(V4*)(out + dim * 2) = y;
            }
        }
    if (h == 0) {
        if (to)
            to[D] = m, to[D + 1] = l;
        else
            z.lse[(int64_t)(s.q0 + t) * z.heads + hq] = (m + __builtin_amdgcn_logf(l * E::kUnshift)) * 0.69314718055994531f;
    }
}

// The parts of row tiles that were split: eight rows of a tile at a time, 32 lanes a row.
template <class E, int D>
__global__ __launch_bounds__(256) void k_join_chunk(AttendArgs p, ChunkPlan plan) {
    constexpr int VD = D / 32;
    const int items = *plan.items, G = p.heads / p.kv.kv_heads;
    const int item = blockIdx.x / (kRows / 8), row = blockIdx.x % (kRows / 8) * 8 + (threadIdx.x >> 5);
    if (item >= items) return;
    const Item x = plan.item[item];
    const int head = item % p.kv.kv_heads, at = x.first_row + row, d0 = (threadIdx.x & 31) * VD;
    if (x.parts < 2 || at >= x.rows) return;
    float top = -INFINITY, den = 0.f, acc[VD];
#pragma unroll
    for (int j = 0; j < VD; j++) acc[j] = 0.f;
#pragma unroll 4
    for (int i = 0; i < x.parts; i++) {
        const float* from = plan.part + (((int64_t)i * items + item) * kRows + row) * (D + 4);
        const float now = fmaxf(top, from[D]), ref = now == -INFINITY ? 0.f : now;
        const float keep = exp2_fast(top - ref), f = exp2_fast(from[D] - ref);
        den = den * keep + from[D + 1] * f;
#pragma unroll
        for (int j = 0; j < VD; j++) acc[j] = scaled(acc[j], keep) + scaled(from[d0 + j], f);
        top = now;
    }
    const int t = at / G;
    write_row<E, VD>(p, x.q0 + t, head * G + at - t * G, d0, acc, den, top);
}

// The weights of these sequences' slots: scores once more, now against the rows' final statistics.
// A workgroup has 256 slots, 64 for each wave, whose keys stay in registers while the rows'
// queries pass through LDS, 64 at a time; a lane sums its own rows for 32 slots and the lanes
// are added at the end, so nothing is added atomically.  2,048 tokens over 14,049 slots of 8 key heads (32 query heads, 218
// GFLOP, 8.5e8 exponentials) take 326 us; nothing bounds it alone: the matrix units are busy for 0.27 of the cycles, other vector
// instructions take 0.33, exponentials 0.2 more, and products and exponentials of a tile follow each other.
constexpr int kWSlots = 256, kWRows = 64;

__device__ inline int slot_tiles(const AttendArgs& p, const Seq& s) {
    if (s.n <= 0 || s.n > p.kv.max_q || !ours(p, s)) return 0;
    return (s.len - first_slot(p, s) + kWSlots - 1) / kWSlots;
}

template <class E, int D>
__device__ inline void weigh_slots(const AttendArgs& p, const Seq& s, int seq, int tile, int head) {
    using T = typename E::T;
    using V8 = typename E::V8;
    constexpr int KS = D / 16, CH = D / 8, PER = kWRows * CH / 256;
    __shared__ __align__(16) char lds[2][kWRows * D * 2];
    __shared__ float stat[2][kWRows];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 31, h = lane >> 5;
    const int G = p.heads / p.kv.kv_heads;
    const int r0 = s.len - s.n;
    const int j0 = first_slot(p, s) + tile * kWSlots, j1 = min(j0 + kWSlots, s.len);
    // rows that see one of the slots: tokens t0 .. t1 - 1
    const int t0 = p.causal ? max(0, j0 - r0) : 0;
    const int t1 = p.window > 0 ? (int)max((int64_t)0, min((int64_t)s.n, (int64_t)j1 - 1 + p.window - r0)) : s.n;
    const int row0 = t0 * G, row1 = t1 * G;

    // this wave's slots and their keys
    const int base = j0 + wave * 64;
    int pool[2];
    V8 k[2][KS];
#pragma unroll
    for (int st = 0; st < 2; st++) {
        const int j = base + st * 32 + c;
        pool[st] = j < j1 ? pool_row(p.kv, seq, j) : -1;
        const uint64_t at = pool[st] < 0 ? (uint64_t)zero_row()
                                         : (uint64_t)(p.kv.k + head * p.kv.k_head) + row_offset(pool[st], p.kv.shift, p.kv.k_page, p.kv.k_row);
#pragma unroll
        for (int x = 0; x < KS; x++) k[st][x] = load_global<V8>(at + x * 32 + h * 16);
    }
    // The rows whose pieces this thread brings to LDS, as token and query head: a tile on is ``step_t`` tokens
    // and ``step_g`` heads on.
    int qt[PER], qg[PER];
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int row = row0 + (i * 256 + tid) / CH;
        qt[i] = row / G;
        qg[i] = row - qt[i] * G;
    }
    const int step_t = kWRows / G, step_g = kWRows - step_t * G;
    V8 staged[PER];
    float staged_stat = 0.f;
    auto take = [&](int at) {  // rows at .. at + 63 into registers
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const int piece = i * 256 + tid, x = piece % CH;
            // a row behind the last has the last one's query: its statistic takes it out
            const int t = min(qt[i], t1 - 1);
            const char* from = p.q + (s.q0 + t) * p.q_tok + (head * G + qg[i]) * p.q_head + x * 16;
            if (p.q_wide) {
                staged[i] = load_global<V8>((uint64_t)from);
            } else {
#pragma unroll
                for (int y = 0; y < 8; y++) staged[i][y] = load_global<T>((uint64_t)(from + y * 2));
            }
            qt[i] += step_t;
            qg[i] += step_g;
            if (qg[i] >= G) qg[i] -= G, qt[i]++;
        }
        if (tid < kWRows) {
            const int row = at + tid, t = row / G;
            // a row that saw nothing, or is none, adds exp2(-inf)
            float x = -INFINITY;
            if (row < row1) x = p.lse[(int64_t)(s.q0 + t) * p.heads + head * G + row - t * G];
            staged_stat = x == -INFINITY ? INFINITY : x * 1.4426950408889634f;
        }
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const int piece = i * 256 + tid, r = piece / CH, x = piece % CH;
            *(V8*)(lds[buf] + r * (D * 2) + (x ^ swizzle<D>(r)) * 16) = staged[i];
        }
        if (tid < kWRows) stat[buf][tid] = staged_stat;
    };
    f32x16 sum[2];
#pragma unroll
    for (int st = 0; st < 2; st++)
#pragma unroll
        for (int i = 0; i < 16; i++) sum[st][i] = 0.f;
    if (row0 < row1) {
        take(row0);
        put(0);
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);  // the keys are there: no wait for them in the loop
    __syncthreads();
    int buf = 0;
    for (int at = row0; at < row1; at += kWRows, buf ^= 1) {
        if (at + kWRows < row1) take(at + kWRows);
        // tokens of the first and the last row
        const int ta = at / G, tb = min(at + kWRows - 1, row1 - 1) / G;
        const bool whole = (!p.causal || base + 63 <= r0 + ta) && (p.window == 0 || base > r0 + tb - p.window) && base + 63 < j1;
        const bool none = (p.causal && base > r0 + tb) || (p.window > 0 && base + 63 <= r0 + ta - p.window) || base >= j1;
        if (!none) {
#pragma unroll
            for (int rt = 0; rt < kWRows / 32; rt++) {
                f32x16 sc[2];
#pragma unroll
                for (int st = 0; st < 2; st++)
#pragma unroll
                    for (int i = 0; i < 16; i++) sc[st][i] = 0.f;
#pragma unroll
                for (int x = 0; x < KS; x++) {
                    const int r = rt * 32 + c;
                    const V8 b = *(const V8*)(lds[buf] + r * (D * 2) + ((2 * x + h) ^ swizzle<D>(c)) * 16);
                    sc[0] = E::mfma32(k[0][x], b, sc[0]);
                    sc[1] = E::mfma32(k[1][x], b, sc[1]);
                }
                // reads two products ahead of their use
                __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
#pragma unroll
                for (int x = 0; x < KS - 2; x++) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
                const float lse = stat[buf][rt * 32 + c];
                if (whole) {
#pragma unroll
                    for (int st = 0; st < 2; st++)
#pragma unroll
                        for (int i = 0; i < 16; i++) sum[st][i] += exp2_fast(fmaf(sc[st][i], p.scale, -lse));
                } else {
                    const int r = r0 + (at + rt * 32 + c) / G;
                    const uint64_t seen = bits_between(p.window > 0 ? r - p.window + 1 - base : 0, p.causal ? r - base : 63) >> (h * 4);
#pragma unroll
                    for (int st = 0; st < 2; st++) {
                        const uint32_t word = (uint32_t)(seen >> (st * 32));
#pragma unroll
                        for (int i = 0; i < 16; i++) {
                            const float e = exp2_fast(fmaf(sc[st][i], p.scale, -lse));
                            sum[st][i] += word >> ((i >> 2) * 8 + (i & 3)) & 1 ? e : 0.f;
                        }
                    }
                }
            }
        }
        if (at + kWRows < row1) put(buf ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int st = 0; st < 2; st++)
#pragma unroll
        for (int i = 0; i < 16; i++) {
            float x = sum[st][i];
            for (int d = 16; d; d >>= 1) x += __shfl_xor(x, d);
            // the lane that looked this slot up has its row
            const int off = (i >> 2) * 8 + h * 4 + (i & 3);
            if (c == off && pool[st] >= 0) p.kv.weight[stat_index(p.kv, pool[st], head)] += x;
        }
}

// One tile a workgroup, of as many as the pool has slots for.
template <class E, int D>
__global__ __launch_bounds__(256, (D <= 128 ? 2 : 1)) void k_weight_chunk(AttendArgs p) {
    __shared__ int64_t scan[4];
    const int hk = p.kv.kv_heads;
    int seq, tile;
    if (!find_item(p.kv, [&](int64_t) { return (int64_t)(blockIdx.x / hk); }, [&](const Seq& s) { return slot_tiles(p, s); }, scan,
                   seq, tile))
        return;
    weigh_slots<E, D>(p, seq_of(p.kv, seq), seq, tile, blockIdx.x % hk);
}

// Sequences with slots that have no page can have more tiles than that: those from ``first`` on, in a loop (a kernel of its own,
// since the loop around it makes the one above spill registers).
template <class E, int D>
__global__ __launch_bounds__(256, (D <= 128 ? 2 : 1)) void k_weight_chunk_more(AttendArgs p, int64_t first) {
    __shared__ int64_t scan[4];
    const int hk = p.kv.kv_heads;
    const int64_t begin = first + blockIdx.x / hk;
    int64_t total = 0;
    for (int64_t at = begin; at == begin || at < total; at += gridDim.x / hk) {
        auto place = [&](int64_t all) {
            total = all;
            return at;
        };
        int seq, tile;
        if (!find_item(p.kv, place, [&](const Seq& s) { return slot_tiles(p, s); }, scan, seq, tile)) return;
        weigh_slots<E, D>(p, seq_of(p.kv, seq), seq, tile, blockIdx.x % hk);
    }
}

// Row tiles at least: those of the rows that sequences of few rows cannot have. With more than half as many as the
// GPU holds workgroups none is split.
int32_t split_groups(const AttendSizes& z, int32_t few) {
    const int32_t groups = z.dim <= 128 ? 512 : 256;
    const int64_t least = ((int64_t)z.tokens * (z.heads / z.kv_heads) - (int64_t)z.seqs * few) / kRows;
    return least * z.kv_heads > groups / 2 ? 0 : groups;
}

int64_t chunk_workspace(const AttendSizes& z, int32_t few) {
    const int32_t groups = split_groups(z, few);
    return groups ? 256 + groups / 2 * (int64_t)sizeof(Item) + (int64_t)groups * kRows * (z.dim + 4) * 4 : 0;
}

// Workgroups of the launches for these sizes.
struct ChunkGrids {
    int64_t blocks, tiles, more;
};

ChunkGrids grids(const AttendSizes& z, int32_t few) {
    ChunkGrids g;
    // Row tiles at most: the full ones of all tokens, and one more for each sequence that is long enough to come here.
    const int64_t rows = (int64_t)z.tokens * (z.heads / z.kv_heads), long_enough = rows / (few + 1);
    const int64_t seqs = long_enough < z.seqs ? long_enough : z.seqs;
    g.blocks = (rows / kRows + seqs) * z.kv_heads;
    if (g.blocks < split_groups(z, few)) g.blocks = split_groups(z, few);
    // slot tiles at most, and where every slot has a page: each page is in the batch once
    const int64_t cap = (int64_t)z.width * z.page_size, all = seqs * ((cap + kWSlots - 1) / kWSlots);
    const int64_t pool = (int64_t)z.num_pages * z.page_size / kWSlots + seqs;
    g.tiles = z.add_weight ? (all < pool ? all : pool) : 0;
    g.more = !z.add_weight ? 0 : all - g.tiles < 64 ? all - g.tiles : 64;
    g.tiles *= z.kv_heads, g.more *= z.kv_heads;
    return g;
}

template <class E, int D>
hipError_t launch(const AttendArgs& a, const AttendSizes& z, char* ws, hipStream_t s) {
    ChunkPlan plan{split_groups(z, a.few), nullptr, nullptr, nullptr};
    if (plan.groups) {
        plan.items = (int32_t*)ws;
        plan.item = (Item*)(ws + 256);
        plan.part = (float*)(ws + 256 + plan.groups / 2 * sizeof(Item));
    }
    const ChunkGrids g = grids(z, a.few);
    hipError_t e;
    if (g.blocks > 0) {
        // Offsets of sixteen rows are 32 bits.
        const int64_t far = 16 * (a.kv.k_row > a.kv.v_row ? a.kv.k_row : a.kv.v_row);
        const bool wide = z.page_size >= 16 && far < (int64_t(1) << 31);
        e = run(wide ? k_attend_chunk<E, D, true> : k_attend_chunk<E, D, false>, dim3((unsigned)g.blocks), 256, s, a, plan);
        if (e != hipSuccess) return e;
    }
    if (plan.groups) {
        e = run(k_join_chunk<E, D>, dim3(plan.groups / 2 * (kRows / 8)), 256, s, a, plan);
        if (e != hipSuccess) return e;
    }
    if (g.tiles > 0) {
        e = run(k_weight_chunk<E, D>, dim3((unsigned)g.tiles), 256, s, a);
        if (e != hipSuccess) return e;
    }
    return g.more > 0 ? run(k_weight_chunk_more<E, D>, dim3((unsigned)g.more), 256, s, a, g.tiles / z.kv_heads) : hipSuccess;
}

}  // namespace

// A call's launches: single tokens and short chunks, and, where a sequence may have more rows, chunks.
bool has_chunks(const AttendSizes& z) { return (int64_t)z.max_q * (z.heads / z.kv_heads) > few_rows(z); }

int64_t attend_workspace(const AttendSizes& z) {
    return ((rows_workspace(z) + 255) & ~int64_t(255)) + (has_chunks(z) ? chunk_workspace(z, few_rows(z)) : 0);
}

int64_t attend_threads(const AttendSizes& z) {
    int64_t most = rows_blocks(z);
    if (has_chunks(z)) {
        const ChunkGrids g = grids(z, few_rows(z));
        if (g.blocks > most) most = g.blocks;
        if (g.tiles > most) most = g.tiles;
        if (g.more > most) most = g.more;
    }
    return most * 256;
}

hipError_t launch_attend(AttendArgs a, const AttendSizes& z, hipStream_t s) {
    a.few = few_rows(z);
    if (a.few) {
        const hipError_t e = launch_rows(a, z, a.ws, s);
        if (e != hipSuccess) return e;
    }
    if (!has_chunks(z)) return hipSuccess;
    char* ws = a.ws + ((rows_workspace(z) + 255) & ~int64_t(255));
    if (z.dtype == SVF_KV_BF16)
        return z.dim == 64 ? launch<BF16M, 64>(a, z, ws, s) : z.dim == 128 ? launch<BF16M, 128>(a, z, ws, s) : launch<BF16M, 256>(a, z, ws, s);
    return z.dim == 64 ? launch<F16M, 64>(a, z, ws, s) : z.dim == 128 ? launch<F16M, 128>(a, z, ws, s) : launch<F16M, 256>(a, z, ws, s);
}

}  // namespace svfk
