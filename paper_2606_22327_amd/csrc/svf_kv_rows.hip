// svf_kv_rows.hip -- attention over the paged cache of sequences with few rows
// (new tokens times query heads of a key head): single tokens and short chunks.
#include "svf_kv_attend.h"

namespace svfk {
namespace {

// Slots that a workgroup takes at a time: 32 for each of its four waves.
constexpr int kUnit = 128;

// What the launches of one call share, in the workspace.
struct RowsPlan {
    int64_t* first_unit;  // [seqs + 1]: units of a key head before each sequence; null where no launch follows
    float* part;          // [2 * groups][rows * (D + 4)]: partial results
    float* scores;        // [units][rows][kUnit] (add_weight): scores in log2 terms
    int4* units;          // [units] (add_weight): sequence, index of the first row's statistic, first slot (place with first tokens), head | rows << 16
    int64_t score_units;  // units that scores has room for
    int32_t groups;       // workgroups over which the units are dealt out
    int32_t rows;         // rows of a sequence's key head at most
};

// Units of one key head of a sequence, 0 where this kernel leaves it to another.
// One without a slot still has its rows to write.
template <bool FIRST>
__device__ inline int units_of(const AttendArgs& p, const Seq& s, int rows) {
    if (s.n <= 0) return 0;
    const int G = p.heads / p.kv.kv_heads;
    if (s.n <= p.kv.max_q && (int64_t)s.n * G > rows) return 0;
    if (s.n > p.kv.max_q) return 1;
    const int u = (line_of<FIRST>(p, s, 16).places + kUnit - 1) / kUnit;
    return u > 0 ? u : 1;
}

// One pass with a running maximum m and sum l of each row: with the scores x_j of a tile, m' = max(m, max x_j),
// l' = l 2^(m - m') + sum 2^(x_j - m'), o' = o 2^(m - m') + sum 2^(x_j - m') v_j (scores in log2 terms).
//
// S^T = K Q^T and O^T = V^T P^T on 16x16x32 products, 32 slots at a time: a lane has the
// scores of one row (l % 16) in both, so maxima and sums need two shuffles, and
// the probabilities are the second product's operand where the first left them.
// The slots that a lane's four-by-two scores belong to are the slots
// whose values it loads: eight rows of a head, D / 16 dimensions each, put
// together by byte permutes. Keys and values go from memory to registers
// once and through no LDS, the next tile's keys while this one's are weighed, its
// values while the next one's are.
//
// Keys and values, read once, bound it: 127 sequences of up to 900 slots (32 query heads on 8 key heads of
// 128 dimensions, 249 MB) take 60 us, 4.1 TB/s where a kernel that only reads reaches 6.2; 64 sequences of 2,000 slots
// 5.7 TB/s with all launches, one sequence of 65,535 slots (134 MB) 27 us.  What is left is the start of each key head's run, two of
// them in a workgroup's seven units in the first case.  Not WIDE, pages of 8 slots 97 us where pages of 16 take 86, of one slot 105.
template <class E, int D>
struct Tile {
    typename E::V8 k[2][D / 32];
    uint32_t v[8][D / 32];  // two dimensions a word
};

// Where the slots of a wave's tile lie.
// WIDE: pages of 16 slots or more, so that each half of the tile lies in one page: two addresses for the whole wave, and what
// a lane adds to them stays the same all along.
// Else a lane has the addresses of slot lane % 32 and hands them to the lanes that load it.
// A slot that is not there is a row of zeros; behind the last slot of a page that is there, WIDE reads what
// the page holds, and nothing comes of it.
struct Where {
    uint64_t k[2], v[2];
    bool there;
};

__device__ inline uint64_t from_lane(uint64_t x, int lane) {
    const uint32_t lo = __shfl((int)(uint32_t)x, lane), hi = __shfl((int)(x >> 32), lane);
    return (uint64_t)hi << 32 | lo;
}

// Each is read once by its key head's rows: past the caches (256 sequences with weights: 278 us and 299 through them).
template <class E, int D, bool WIDE>
__device__ inline void load_k(Tile<E, D>& x, const Where& w, uint32_t row_bytes) {
    typedef const __attribute__((address_space(1))) char* Global;
    typedef const __attribute__((address_space(1))) typename E::V8* Global8;
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
#pragma unroll
    for (int t = 0; t < 2; t++) {
        if constexpr (WIDE) {
            const uint32_t off = (w.k[t] == (uint64_t)zero_row() ? 0 : c * row_bytes) + g * 16;
#pragma unroll
            for (int s = 0; s < D / 32; s++) x.k[t][s] = __builtin_nontemporal_load((Global8)((Global)w.k[t] + off + s * 64));
        } else {
            const uint64_t at = from_lane(w.k[0], t * 16 + c) + g * 16;
#pragma unroll
            for (int s = 0; s < D / 32; s++) x.k[t][s] = load_global<typename E::V8>(at + s * 64);
        }
    }
}

template <class E, int D, bool WIDE>
__device__ inline void load_v(Tile<E, D>& x, const Where& w, uint32_t row_bytes) {
    typedef uint32_t Row __attribute__((ext_vector_type(D / 32)));
    typedef const __attribute__((address_space(1))) char* Global;
    typedef const __attribute__((address_space(1))) Row* GlobalRow;
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
#pragma unroll
    for (int j = 0; j < 8; j++) {
        Row r;
        if constexpr (WIDE) {
            const uint32_t off = (w.v[j >> 2] == (uint64_t)zero_row() ? 0 : (g * 4 + (j & 3)) * row_bytes) + c * (D / 8);
            r = __builtin_nontemporal_load((GlobalRow)((Global)w.v[j >> 2] + off));
        } else {
            r = load_global<Row>(from_lane(w.v[0], (j >> 2) * 16 + g * 4 + (j & 3)) + c * (D / 8));
        }
#pragma unroll
        for (int i = 0; i < D / 32; i++) x.v[j][i] = r[i];
    }
}

// Waves of a SIMD that the registers of a tile leave room for.  (Squeezed into a third wave's, 128 dimensions spill
// 14 registers, though none that the loop needs, and take 78 us where they took 68.)
constexpr int waves_per_simd(int dim, int rt) { return dim * rt <= 64 ? 3 : dim * rt <= 128 ? 2 : 1; }

template <class E, int D, int RT, bool WIDE, bool FIRST>
__global__ __launch_bounds__(256, waves_per_simd(D, RT)) void k_attend_rows(AttendArgs p, RowsPlan plan) {
    using T = typename E::T;
    using V8 = typename E::V8;
    constexpr int KS = D / 32, VD = D / 16;
    __shared__ __align__(16) float red[4][16][D + 4];
    static_assert(__alignof__(red) >= alignof(f32x4) && D / 16 % 4 == 0, "four at a time are written at their boundary");
    __shared__ float red_m[4][16], red_l[4][16];
    __shared__ int64_t scan[4];
    __shared__ uint32_t odd_marks[16 * RT][16];  // a word for D / 16 dimensions of a row
    __shared__ int sh_seq;
    __shared__ int64_t sh_first;
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = p.heads / p.kv.kv_heads, hk = p.kv.kv_heads;

    // Deal the units out: sequences in order, key head by key head, an equal run of units for
    // every workgroup.
    const int per = (p.kv.seqs + 255) / 256;
    const int i0 = min(tid * per, p.kv.seqs), i1 = min(i0 + per, p.kv.seqs);
    int64_t mine = 0;
    for (int i = i0; i < i1; i++) mine += units_of<FIRST>(p, seq_of(p.kv, i), plan.rows);
    int64_t incl = mine;
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t x = __shfl_up(incl, d);
        if (lane >= d) incl += x;
    }
    if (lane == 63) scan[wave] = incl;
    __syncthreads();
    int64_t total = 0, before = incl - mine;
    for (int w = 0; w < 4; w++) {
        if (w < wave) before += scan[w];
        total += scan[w];
    }
    const int64_t all = total * hk;
    const int64_t groups = min((int64_t)plan.groups, all);  // of which each has a unit
    const bool idle = blockIdx.x >= groups;
    const int64_t a = idle ? 0 : all * blockIdx.x / groups, b = idle ? 0 : all * (blockIdx.x + 1) / groups;
    if (blockIdx.x == 0 && plan.first_unit) {
        int64_t at = before;
        for (int i = i0; i < i1; i++) {
            plan.first_unit[i] = at;
            at += units_of<FIRST>(p, seq_of(p.kv, i), plan.rows);
        }
        if (tid == 0) plan.first_unit[p.kv.seqs] = total;
    }
    if (idle) return;
    if (before * hk <= a && a < (before + mine) * hk) {
        int64_t at = before;
        int i = i0;
        for (; i < i1; i++) {
            const int u = units_of<FIRST>(p, seq_of(p.kv, i), plan.rows);
            if (a < (at + u) * hk) break;
            at += u;
        }
        sh_seq = i;
        sh_first = at;
    }
    __syncthreads();
    int seq = sh_seq;
    int64_t first = sh_first;  // units of a key head before seq

    for (int64_t pos = a; pos < b && seq < p.kv.seqs;) {
        const Seq s = seq_of(p.kv, seq);
        const int units = units_of<FIRST>(p, s, plan.rows);
        if (pos >= (first + units) * hk) {  // a sequence done, or one without units
            first += units;
            seq++;
            continue;
        }
        const int64_t rel = pos - first * hk;
        const int head = (int)(rel / units), u0 = (int)(rel - (int64_t)head * units);
        const int u1 = (int)min((int64_t)units, u0 + (b - pos));
        const int64_t unit0 = pos;
        pos += u1 - u0;
        const int rows = s.n * G;
        if (s.n > p.kv.max_q) {
            fill_nan<T, D>(p, s, head, G, tid, 256);
            if (plan.scores && unit0 < plan.score_units && tid == 0) plan.units[unit0] = make_int4(seq, 0, 0, head);
            continue;
        }
        const Line line = line_of<FIRST>(p, s, 16);
        const int r0 = s.len - s.n;  // the first new token's slot
        const uint64_t kbase = (uint64_t)(p.kv.k + head * p.kv.k_head), vbase = (uint64_t)(p.kv.v + head * p.kv.v_head);

        V8 q[RT][KS];
        int last[RT], from[RT];  // a lane's rows see slots from .. last
#pragma unroll
        for (int rt = 0; rt < RT; rt++) {
            const int row = rt * 16 + c;
            const int t = row < rows ? row / G : 0;
            const char* at = p.q + (s.q0 + t) * p.q_tok + (head * G + (row < rows ? row - t * G : 0)) * p.q_head;
            load_query<E, KS>(q[rt], at, g, row < rows, p.q_wide);
            last[rt] = p.causal ? r0 + t : s.len - 1;
            from[rt] = p.window > 0 ? r0 + t - p.window + 1 : 0;
        }
        float m[RT], l[RT];
        f32x4 o[RT][VD];
#pragma unroll
        for (int rt = 0; rt < RT; rt++) {
            m[rt] = -INFINITY, l[rt] = 0.f;
#pragma unroll
            for (int j = 0; j < VD; j++) o[rt][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const int place0 = wave * 32 + (lane & 31);
        const Table table = table_of(p.kv, seq, s.len, zero_row());
        auto entry = [&](int u) { return table_entry(p.kv, table, slot_of<FIRST>(line, place0 + u * kUnit)); };
        auto where = [&](int u, int page) {
            const int j = slot_of<FIRST>(line, place0 + u * kUnit), row = entry_row(p.kv, page, j, u < u1 && j < s.len);
            Where w;
            w.there = row >= 0;
            if constexpr (WIDE) {
#pragma unroll
                for (int t = 0; t < 2; t++) {
                    const int at = __builtin_amdgcn_readlane(row, t * 16);
                    const int pg = at >> p.kv.shift, r = at & ((1 << p.kv.shift) - 1);
                    w.k[t] = at < 0 ? (uint64_t)zero_row() : row_address(kbase, pg, r, p.kv.k_page, p.kv.k_row);
                    w.v[t] = at < 0 ? (uint64_t)zero_row() : row_address(vbase, pg, r, p.kv.v_page, p.kv.v_row);
                }
            } else {
                const int pg = row >> p.kv.shift, r = row & ((1 << p.kv.shift) - 1);
                const uint64_t k = row_address(kbase, pg, r, p.kv.k_page, p.kv.k_row);
                const uint64_t v = row_address(vbase, pg, r, p.kv.v_page, p.kv.v_row);
                w.k[0] = w.there ? k : (uint64_t)zero_row();
                w.v[0] = w.there ? v : (uint64_t)zero_row();
            }
            return w;
        };
        const uint32_t k_row = (uint32_t)p.kv.k_row, v_row = (uint32_t)p.kv.v_row;
        int page0 = entry(u0), page_next = entry(u0 + 1);
        for (int i = tid; i < 16 * RT * 16; i += 256) (&odd_marks[0][0])[i] = 0;
        __syncthreads();
        Tile<E, D> x;
        Where now = where(u0, page0);
        // In the loop's order: where the two meet, the compiler waits for the more careful of them.
        __builtin_amdgcn_sched_barrier(0);
        load_k<E, D, WIDE>(x, now, k_row);
        __builtin_amdgcn_sched_barrier(0);
        load_v<E, D, WIDE>(x, now, v_row);
        __builtin_amdgcn_sched_barrier(0);
        for (int u = u0; u < u1; u++) {
            const Where next = where(u + 1, page_next);
            page_next = entry(u + 2);
            // slot of place x of the tile, without x: its two halves may lie apart
            const int place = u * kUnit + wave * 32, base[2] = {slot_of<FIRST>(line, place), slot_of<FIRST>(line, place + 16) - 16};
            f32x4 sc[RT][2];
#pragma unroll
            for (int rt = 0; rt < RT; rt++)
#pragma unroll
                for (int t = 0; t < 2; t++) {
                    sc[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < KS; k++) sc[rt][t] = E::mfma16(x.k[t][k], q[rt][k], sc[rt][t]);
                }
            // which of the tile's slots are there: the same for every row
            const uint32_t there = (uint32_t)__ballot(now.there);
            bool all_seen = there == 0xffffffffu && (!p.causal || base[1] + 31 <= r0);
#pragma unroll
            for (int t = 0; t <= FIRST; t++)
                all_seen = all_seen && (p.window == 0 || base[t] + 16 * t > s.len - 1 - p.window || (FIRST && base[t] + 16 * t + 15 < p.first));
            __builtin_amdgcn_sched_barrier(0);
            load_k<E, D, WIDE>(x, next, k_row);
            __builtin_amdgcn_sched_barrier(0);
            V8 hi[RT], low[RT];
#pragma unroll
            for (int rt = 0; rt < RT; rt++) {
                float top = -INFINITY;
#pragma unroll
                for (int i = 0; i < 8; i++) sc[rt][i >> 2][i & 3] *= p.scale;
                if (!all_seen) {
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const int off = (i >> 2) * 16 + g * 4 + (i & 3), j = base[i >> 2] + off;
                        if (!(there >> off & 1) || j > last[rt] || (j < from[rt] && !(FIRST && j < p.first))) sc[rt][i >> 2][i & 3] = -INFINITY;
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; i++) top = fmaxf(top, sc[rt][i >> 2][i & 3]);
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float peak = fmaxf(m[rt], top);
                const float ref = (peak == -INFINITY ? 0.f : peak) - E::kShift;
                const float keep = exp2_fast(m[rt] - (peak == -INFINITY ? 0.f : peak));
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float e = exp2_fast(sc[rt][i >> 2][i & 3] - ref);
                    sum += e;
                    // the probability as the sum of two numbers of the type: twice its bits, for
                    // products that memory hides
                    hi[rt][i] = (T)e;
                    low[rt][i] = (T)(e - (float)hi[rt][i]);
                }
                l[rt] = l[rt] * keep + sum;  // of this lane's slots; the four lanes of a row are added at the end
                m[rt] = peak;
#pragma unroll
                for (int j = 0; j < VD; j++)
#pragma unroll
                    for (int r = 0; r < 4; r++) o[rt][j][r] *= keep;
            }
            // A value that is no finite number would reach rows that do not see it (0 times infinity), and
            // meet both halves of a probability.  It counts as 0 here, and the rows that see it
            // get it from its marks.
            {
                u16x2 size = {0, 0};
#pragma unroll
                for (int i = 0; i < 8; i++)
#pragma unroll
                    for (int w = 0; w < D / 32; w++)
                        size = __builtin_elementwise_max(size, __builtin_bit_cast(u16x2, x.v[i][w] & 0x7fff7fffu));
                const bool odd = max(size.x, size.y) >= E::kInf;
                if (__any(odd)) {
                    // through this wave's part of ``red``, a word at a time: rare, and registers are scarce
                    uint32_t* own = (uint32_t*)&red[wave][0][0] + lane;
#pragma unroll
                    for (int i = 0; i < 8 * (D / 32); i++) own[i * 64] = x.v[i / (D / 32)][i % (D / 32)];
#pragma unroll 1
                    for (int i = 0; i < 8 * (D / 32); i++) {
                        const uint32_t pair = own[i * 64];
                        if (!odd_pair<E>(pair)) continue;
                        const int at = i / (D / 32), off = (at >> 2) * 16 + g * 4 + (at & 3), j = base[at >> 2] + off;
                        const uint32_t marks = odd_marks_of<E>(pair) << 4 * (i % (D / 32));
                        for (int row = 0; row < rows && (there >> off & 1); row++) {
                            const int r = r0 + row / G;
                            if ((!p.causal || j <= r) && (p.window == 0 || j > r - p.window || (FIRST && j < p.first))) atomicOr(&odd_marks[row][c], marks);
                        }
                        own[i * 64] = finite_pair<E>(pair);
                    }
#pragma unroll
                    for (int i = 0; i < 8 * (D / 32); i++) x.v[i / (D / 32)][i % (D / 32)] = own[i * 64];
                }
            }
#pragma unroll
            for (int j = 0; j < VD; j++) {
                uint4 t;
                const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
                t.x = __builtin_amdgcn_perm(x.v[1][j / 2], x.v[0][j / 2], sel);
                t.y = __builtin_amdgcn_perm(x.v[3][j / 2], x.v[2][j / 2], sel);
                t.z = __builtin_amdgcn_perm(x.v[5][j / 2], x.v[4][j / 2], sel);
                t.w = __builtin_amdgcn_perm(x.v[7][j / 2], x.v[6][j / 2], sel);
                const V8 vt = __builtin_bit_cast(V8, t);
#pragma unroll
                for (int rt = 0; rt < RT; rt++) {
                    o[rt][j] = E::mfma16(vt, hi[rt], o[rt][j]);
                    o[rt][j] = E::mfma16(vt, low[rt], o[rt][j]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            load_v<E, D, WIDE>(x, next, v_row);
            __builtin_amdgcn_sched_barrier(0);
            // behind the loads: a wait for those is none for these
            const int64_t unit = unit0 + (u - u0);
            if (plan.scores && unit < plan.score_units) {
#pragma unroll
                for (int rt = 0; rt < RT; rt++)
                    if (rt * 16 + c < rows) {
                        float* to = plan.scores + (unit * plan.rows + rt * 16 + c) * kUnit + wave * 32 + g * 4;
                        *(f32x4*)to = sc[rt][0];
                        *(f32x4*)(to + 16) = sc[rt][1];
                    }
                if (tid == 0) plan.units[unit] = make_int4(seq, s.q0 * p.heads + head * G, FIRST ? u * kUnit : line.skip + u * kUnit, head | rows << 16);
            }
            now = next;
        }

        // The four waves' parts of a row, then the row: whole, or this workgroup's part of it.
        const bool whole = u0 == 0 && u1 == units;
        float* part = plan.part + (int64_t)(2 * blockIdx.x + (u0 == 0 ? 1 : 0)) * plan.rows * (D + 4);
#pragma unroll
        for (int rt = 0; rt < RT; rt++) {
            if (rt * 16 >= rows) break;
            float sum = l[rt];
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (g == 0) red_m[wave][c] = m[rt], red_l[wave][c] = sum;
#pragma unroll
            for (int r = 0; r < 4; r++)
#pragma unroll
                for (int j = 0; j < VD; j += 4)
                    *(f32x4*)&red[wave][c][(g * 4 + r) * VD + j] =
                        f32x4{o[rt][j][r], o[rt][j + 1][r], o[rt][j + 2][r], o[rt][j + 3][r]};
            __syncthreads();
            const int rr = tid >> 4, d0 = (tid & 15) * VD, row = rt * 16 + rr;
            if (row < rows) {
                float top = -INFINITY;
                for (int w = 0; w < 4; w++) top = fmaxf(top, red_m[w][rr]);
                const float ref = top == -INFINITY ? 0.f : top;
                float den = 0.f, acc[VD];
#pragma unroll
                for (int j = 0; j < VD; j++) acc[j] = 0.f;
                for (int w = 0; w < 4; w++) {
                    const float f = exp2_fast(red_m[w][rr] - ref);
                    den += red_l[w][rr] * f;
#pragma unroll
                    for (int j = 0; j < VD; j++) acc[j] += red[w][rr][d0 + j] * f;
                }
                set_marked(odd_marks[row][tid & 15], acc, VD);
                if (whole) {
                    const int t = row / G, h = head * G + row - t * G;
                    write_row<E, VD>(p, s.q0 + t, h, d0, acc, den, top);
                } else {
#pragma unroll
                    for (int j = 0; j < VD; j += 4) *(f32x4*)&part[row * D + d0 + j] = f32x4{acc[j], acc[j + 1], acc[j + 2], acc[j + 3]};
                    if (d0 == 0) {
                        part[plan.rows * D + 2 * row] = top;
                        part[plan.rows * D + 2 * row + 1] = den;
                    }
                }
            }
            __syncthreads();
        }
    }
}

// The sequence that a unit belongs to: the last that begins at or before it. For whole waves.
__device__ inline int seq_of_unit(const AttendArgs& p, const RowsPlan& plan, int64_t unit) {
    const int lane = threadIdx.x & 63, hk = p.kv.kv_heads;
    int lo = 0, n = p.kv.seqs;
    while (n > 1) {
        const int step = (n + 63) >> 6, at = lane * step;
        const bool le = at < n && plan.first_unit[lo + at] * hk <= unit;
        const int hits = __popcll(__ballot(le)), k = hits > 0 ? hits - 1 : 0;
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

// The parts of the rows that were split over workgroups, in the order of their units.  One workgroup for
// each key head, or for each boundary between two workgroups' runs: then it does its work if the
// boundary is the first inside a key head's units.  ``parts`` groups of 32 lanes share a row's parts.
template <class E, int D>
__global__ __launch_bounds__(256) void k_join_rows(AttendArgs p, RowsPlan plan, int parts, bool by_head) {
    constexpr int VD = D / 32;
    const int hk = p.kv.kv_heads, G = p.heads / hk;
    const int64_t all = plan.first_unit[p.kv.seqs] * hk, groups = min((int64_t)plan.groups, all);
    int seq, head;
    int64_t units, s0, w0;  // the key head's units, its first and the workgroup that has it
    if (by_head) {
        seq = blockIdx.x / hk;
        head = blockIdx.x - seq * hk;
        const int64_t first = plan.first_unit[seq];
        units = plan.first_unit[seq + 1] - first;
        if (units < 2) return;
        s0 = first * hk + head * units;
        w0 = s0 * groups / all;
        while (all * (w0 + 1) / groups <= s0) w0++;
        while (all * w0 / groups > s0) w0--;
        if (all * (w0 + 1) / groups >= s0 + units) return;
    } else {
        const int64_t w = (int64_t)blockIdx.x + 1;
        if (w >= groups) return;
        const int64_t cut = all * w / groups;
        seq = seq_of_unit(p, plan, cut);
        const int64_t first = plan.first_unit[seq];
        units = plan.first_unit[seq + 1] - first;
        head = (int)((cut - first * hk) / units);
        s0 = first * hk + head * units;
        w0 = w - 1;
        if (cut == s0 || all * w0 / groups > s0) return;
    }
    const int64_t s1 = s0 + units;
    int64_t w1 = (s1 - 1) * groups / all;  // and the one that has the last
    while (all * (w1 + 1) / groups <= s1 - 1) w1++;
    while (all * w1 / groups > s1 - 1) w1--;
    const Seq s = seq_of(p.kv, seq);
    const int tid = threadIdx.x, sub = (tid >> 5) % parts, d0 = (tid & 31) * VD;
    const int64_t stride = (int64_t)plan.rows * (D + 4);
    __shared__ float red[8][D], red_m[8], red_l[8];
    const int rows = s.n * G, here = 8 / parts;
    for (int row0 = blockIdx.y * here; row0 < rows; row0 += gridDim.y * here) {
        const int row = row0 + (tid >> 5) / parts;
        float top = -INFINITY, den = 0.f, acc[VD];
#pragma unroll
        for (int j = 0; j < VD; j++) acc[j] = 0.f;
        if (row < rows) {
            // eight parts at a time, all their loads before the first is used
            for (int64_t x0 = w0 + sub; x0 <= w1; x0 += 8 * parts) {
                float pm[8], pl[8], pv[8][VD];
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const int64_t x = min(x0 + i * parts, w1);
                    const float* q = plan.part + (2 * x + (x == w0 ? 1 : 0)) * stride;
                    pm[i] = x0 + i * parts <= w1 ? q[plan.rows * D + 2 * row] : -INFINITY;
                    pl[i] = q[plan.rows * D + 2 * row + 1];
#pragma unroll
                    for (int j = 0; j < VD; j++) pv[i][j] = q[row * D + d0 + j];
                }
                float now = top;
#pragma unroll
                for (int i = 0; i < 8; i++) now = fmaxf(now, pm[i]);
                const float ref = now == -INFINITY ? 0.f : now, keep = exp2_fast(top - ref);
                den *= keep;
#pragma unroll
                for (int j = 0; j < VD; j++) acc[j] = scaled(acc[j], keep);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    if (x0 + i * parts > w1) continue;
                    const float f = exp2_fast(pm[i] - ref);
                    den += pl[i] * f;
#pragma unroll
                    for (int j = 0; j < VD; j++) acc[j] += scaled(pv[i][j], f);
                }
                top = now;
            }
        }
        if (parts > 1) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < VD; j++) red[tid >> 5][d0 + j] = acc[j];
            if ((tid & 31) == 0) red_m[tid >> 5] = top, red_l[tid >> 5] = den;
            __syncthreads();
            if (sub == 0) {
                const int g0 = tid >> 5;
                for (int x = 1; x < parts; x++) top = fmaxf(top, red_m[g0 + x]);
                const float ref = top == -INFINITY ? 0.f : top;
                den = 0.f;
#pragma unroll
                for (int j = 0; j < VD; j++) acc[j] = 0.f;
                for (int x = 0; x < parts; x++) {
                    const float f = exp2_fast(red_m[g0 + x] - ref);
                    den += red_l[g0 + x] * f;
#pragma unroll
                    for (int j = 0; j < VD; j++) acc[j] += scaled(red[g0 + x][d0 + j], f);
                }
            }
        }
        if (sub == 0 && row < rows) {
            const int t = row / G;
            write_row<E, VD>(p, s.q0 + t, head * G + row - t * G, d0, acc, den, top);
        }
    }
}

// The weights of a unit whose scores were not kept: they are formed again, two slots a lane. Right, not fast.
template <class E, int D, bool FIRST>
__device__ void weigh_again(const AttendArgs& p, const RowsPlan& plan, int64_t unit) {
    using T = typename E::T;
    const int hk = p.kv.kv_heads, G = p.heads / hk, lane = threadIdx.x & 63;
    const int seq = seq_of_unit(p, plan, unit);
    const int64_t first = plan.first_unit[seq], units = plan.first_unit[seq + 1] - first, rel = unit - first * hk;
    const int head = (int)(rel / units), u = (int)(rel - head * units);
    const Seq s = seq_of(p.kv, seq);
    if (s.n > p.kv.max_q) return;
    const int r0 = s.len - s.n;
    for (int x = 0; x < 2; x++) {
        const int j = slot_of<FIRST>(line_of<FIRST>(p, s, 16), u * kUnit + 2 * lane + x);
        const int at = j < s.len ? pool_row(p.kv, seq, j) : -1;
        if (at < 0) continue;
        const T* k = (const T*)(p.kv.k + head * p.kv.k_head + row_offset(at, p.kv.shift, p.kv.k_page, p.kv.k_row));
        float sum = 0.f;
        for (int r = 0; r < s.n * G; r++) {
            const int t = r / G, h = head * G + r - t * G;
            if ((p.causal && j > r0 + t) || (p.window > 0 && j <= r0 + t - p.window && !(FIRST && j < p.first))) continue;
            const T* q = (const T*)(p.q + (s.q0 + t) * p.q_tok + h * p.q_head);
            float dot = 0.f;
#pragma unroll 8
            for (int d = 0; d < D; d++) dot = fmaf((float)q[d], (float)k[d], dot);
            const float lse = p.lse[(int64_t)(s.q0 + t) * p.heads + h] * 1.4426950408889634f;
            sum += exp2_fast(dot * p.scale - (lse == -INFINITY ? INFINITY : lse));
        }
        p.kv.weight[stat_index(p.kv, at, head)] += sum;
    }
}

// The weights of these sequences' slots from the scores and the rows' final statistics: a wave for a unit, two
// slots a lane, the rows in order. (256 sequences, 255,882 slots of 8 key heads: 15 us for 32 MB of scores and 16 MB of weights.)
// There is room for the scores of as many slots as the pool has; sequences with slots that have no page can have more units.
template <class E, int D, bool FIRST>
__global__ __launch_bounds__(256) void k_weight_rows(AttendArgs p, RowsPlan plan) {
    const int hk = p.kv.kv_heads, G = p.heads / hk, lane = threadIdx.x & 63;
    const int64_t wave = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), all = plan.first_unit[p.kv.seqs] * hk;
    for (int64_t unit = plan.score_units + wave; unit < all; unit += (int64_t)gridDim.x * 4) weigh_again<E, D, FIRST>(p, plan, unit);
    if (wave >= min(all, plan.score_units)) return;
    const int4 x = plan.units[wave];
    const int rows = x.w >> 16, head = x.w & 0xffff;
    const Seq s = seq_of(p.kv, x.x);
    const int j = FIRST ? slot_of<FIRST>(line_of<FIRST>(p, s, 16), x.z + 2 * lane) : x.z + 2 * lane;
    const Table table = table_of(p.kv, x.x, s.len, zero_row());
    const int page[2] = {table_entry(p.kv, table, j), table_entry(p.kv, table, j + 1)};
    const float2* sc = (const float2*)(plan.scores + wave * plan.rows * kUnit) + lane;
    float2 sum = {0.f, 0.f};
#pragma unroll 4
    for (int r = 0; r < rows; r++) {
        const int t = r / G;
        const float lse = p.lse[x.y + t * p.heads + r - t * G] * 1.4426950408889634f;
        const float2 y = sc[r * (kUnit / 2)];
        const float ref = lse == -INFINITY ? INFINITY : lse;  // a row that saw nothing adds nothing
        // only to slots that the row sees: a statistic that is no number makes one of every score, also of the -inf of the others
        const int own = s.len - s.n + t, last = p.causal ? own : s.len - 1, from = p.window > 0 ? own - p.window + 1 : 0;
        sum.x += j <= last && (j >= from || (FIRST && j < p.first)) ? exp2_fast(y.x - ref) : 0.f;
        sum.y += j < last && (j + 1 >= from || (FIRST && j + 1 < p.first)) ? exp2_fast(y.y - ref) : 0.f;
    }
    const int row0 = entry_row(p.kv, page[0], j, j < s.len && sum.x != 0.f), row1 = entry_row(p.kv, page[1], j + 1, j + 1 < s.len && sum.y != 0.f);
    if (row0 >= 0) p.kv.weight[stat_index(p.kv, row0, head)] += sum.x;
    if (row1 >= 0) p.kv.weight[stat_index(p.kv, row1, head)] += sum.y;
}

template <class E, int D, bool WIDE, bool FIRST>
hipError_t launch_tiles(const AttendArgs& a, const RowsPlan& plan, hipStream_t s) {
    if constexpr (D <= 128) {
        if (plan.rows > 16) return run(k_attend_rows<E, D, 2, WIDE, FIRST>, dim3(plan.groups), 256, s, a, plan);
    }
    return run(k_attend_rows<E, D, 1, WIDE, FIRST>, dim3(plan.groups), 256, s, a, plan);
}

template <class E, int D, bool FIRST>
hipError_t launch(const AttendArgs& a, const RowsPlan& plan, hipStream_t s) {
    // Offsets of sixteen rows are 32 bits.
    const int64_t far = 16 * (a.kv.k_row > a.kv.v_row ? a.kv.k_row : a.kv.v_row);
    const bool wide = a.kv.shift >= 4 && far < (int64_t(1) << 31);
    hipError_t e = wide ? launch_tiles<E, D, true, FIRST>(a, plan, s) : launch_tiles<E, D, false, FIRST>(a, plan, s);
    if (e != hipSuccess) return e;
    const int64_t cap = (int64_t)a.kv.width << a.kv.shift;
    if (cap > kUnit && plan.groups > 1) {  // else no row has a second unit
        // Few key heads are split over many workgroups: a row's parts over 8 groups of lanes, a workgroup for each
        // row (one sequence of 65,535 slots on 4 key heads: 32.4 us, the other way 39.3).  Many are split over two or three: a workgroup
        // for all rows, its groups on as many rows as there are (16 sequences of 4,000 slots with 8 new tokens: 56.9 us, the
        // other way 65.1; 127 sequences of up to 900 slots: 65.1 and 69.5).
        // A workgroup for each key head where those are fewer than the boundaries between workgroups, which need a search: 4 sequences of
        // 16,000 slots 53.1 us by key head and 54.8 by boundary, 127 sequences 66.4 and 65.2.
        const bool many = plan.groups >= 8 * (int64_t)a.kv.seqs * a.kv.kv_heads;
        int parts = 8;
        while (!many && parts > 1 && 8 / parts < plan.rows) parts >>= 1;
        const int64_t heads = (int64_t)a.kv.seqs * a.kv.kv_heads;
        const bool by_head = heads < plan.groups - 1;
        e = run(k_join_rows<E, D>, dim3((unsigned)(by_head ? heads : plan.groups - 1), many ? plan.rows : 1), 256, s, a, plan, parts, by_head);
        if (e != hipSuccess) return e;
    }
    return a.add_weight && plan.score_units > 0 ? run(k_weight_rows<E, D, FIRST>, dim3((unsigned)((plan.score_units + 3) / 4)), 256, s, a, plan)
                                                : hipSuccess;
}

template <bool FIRST>
hipError_t launch_kind(const AttendArgs& a, const RowsPlan& plan, const AttendSizes& z, hipStream_t s) {
    if (z.dtype == SVF_KV_BF16)
        return z.dim == 64    ? launch<BF16M, 64, FIRST>(a, plan, s)
               : z.dim == 128 ? launch<BF16M, 128, FIRST>(a, plan, s)
                              : launch<BF16M, 256, FIRST>(a, plan, s);
    return z.dim == 64    ? launch<F16M, 64, FIRST>(a, plan, s)
           : z.dim == 128 ? launch<F16M, 128, FIRST>(a, plan, s)
                          : launch<F16M, 256, FIRST>(a, plan, s);
}

int64_t round256(int64_t x) { return (x + 255) & ~int64_t(255); }

struct Layout {
    int64_t part, scores, descs, units, bytes;
    int32_t groups, rows;
};

Layout layout(const AttendSizes& z) {
    Layout y;
    const int64_t cap = z.places;
    const int64_t most = (int64_t)z.seqs * z.kv_heads * ((cap + kUnit - 1) / kUnit > 0 ? (cap + kUnit - 1) / kUnit : 1);
    y.rows = few_rows(z);
    // What the GPU holds at a time, but eight units each where that still is one for every CU: the fewer parts a row has,
    // the less there is to join (65,535 slots of one sequence: 512 workgroups 38 us, 256 34).
    y.groups = 256 * waves_per_simd(z.dim, y.rows <= 16 ? 1 : 2);
    if (most / 8 < y.groups) y.groups = (int32_t)(most / 8 > 256 ? most / 8 : 256);
    if (most < y.groups) y.groups = (int32_t)most;
    y.part = round256((int64_t)(z.seqs + 1) * 8);
    y.scores = y.part + round256((int64_t)2 * y.groups * y.rows * (z.dim + 4) * 4);
    // every page once at most: the pool's slots, and a unit that is not full for each sequence (more where slots have no
    // page: those units' scores are formed again)
    y.units = 0;
    if (z.add_weight) {
        y.units = ((int64_t)z.num_pages * z.page_size / kUnit + z.seqs) * z.kv_heads;
        if (y.units > most) y.units = most;
    }
    y.descs = y.scores + round256(y.units * y.rows * kUnit * 4);
    y.bytes = y.descs + y.units * 16;
    return y;
}

}  // namespace

// Rows that these kernels take: a whole batch's where no sequence has more than 32 (16 of 256 dimensions), else
// single tokens' (or 16, whichever is more).  8 sequences of 8,000 slots, here and as a tile of 128 rows: 32 query heads on 8 key heads
// of 128 dimensions, 20 rows 57 us and 75, 32 rows 58 and 68; of 64 dimensions, 20 rows 42 and 45, 32 rows 45 and 44; of 256
// dimensions, 16 rows 103 and 142.  More rows than that would need registers that a wave does not have.
int32_t few_rows(const AttendSizes& z) {
    const int32_t G = z.heads / z.kv_heads, most = z.dim <= 128 ? 32 : 16;
    const int64_t want = (int64_t)z.max_q * G;
    if (want <= most) return (int32_t)(want < 1 ? 1 : want);
    const int32_t single = G > 16 ? G : 16;
    // None, where every sequence must have more: what the others can leave of the tokens.
    if (((int64_t)z.tokens - (int64_t)(z.seqs - 1) * z.max_q) * G > single) return 0;
    return single <= most ? single : 0;
}

// One launch does where every row has its slots in one unit and no weights are kept.
bool one_launch(const AttendSizes& z) { return (int64_t)z.width * z.page_size <= kUnit && !z.add_weight; }

int64_t rows_blocks(const AttendSizes& z) {
    if (!few_rows(z)) return 0;
    const Layout y = layout(z);
    return (y.units + 3) / 4 > y.groups ? (y.units + 3) / 4 : y.groups;
}

int64_t rows_workspace(const AttendSizes& z) { return few_rows(z) && !one_launch(z) ? layout(z).bytes : 0; }

hipError_t launch_rows(const AttendArgs& a, const AttendSizes& z, char* ws, hipStream_t s) {
    const Layout y = layout(z);
    RowsPlan plan;
    plan.first_unit = one_launch(z) ? nullptr : (int64_t*)ws;
    plan.part = (float*)(ws + y.part);
    plan.scores = a.add_weight ? (float*)(ws + y.scores) : nullptr;
    plan.units = (int4*)(ws + y.descs);
    plan.score_units = y.units;
    plan.groups = y.groups;
    plan.rows = y.rows;
    return a.first > 0 ? launch_kind<true>(a, plan, z, s) : launch_kind<false>(a, plan, z, s);
}

}  // namespace svfk
