// svf_kv_evict.hip -- eviction from the paged cache by accumulated weight.
#include <type_traits>

#include "svf_kv_device.h"

namespace svfk {
namespace {

// A slot's rank key: unsigned order is the order of keeping.  Protected slots are the largest value,
// NaN and slots without a page the smallest; between them the order of the
// weights as numbers (-0 and 0 are equal).
__device__ inline uint32_t rank_key(bool there, int pos, float w, int first, int recent_from) {
    if (!there) return 0u;
    if (pos < first || pos >= recent_from) return 0xffffffffu;
    if (w != w) return 0u;
    const uint32_t b = w == 0.f ? 0u : __float_as_uint(w);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

constexpr int kCopies = 8;  // of a histogram's bin, for lanes that meet in one

constexpr int kMoveRows = 32;   // pairs moved at a time
constexpr int kOwnPairs = 128;  // pairs that a workgroup moves right after it has found them

// Copies n movers' rows into their holes: 16 bytes a lane, key rows and value rows side by side. For a whole workgroup.
template <int THREADS>
__device__ inline void move_pairs(const EvictArgs& p, int seq, int head, const int2* pairs, int n, int* to, int* from) {
    const int tid = threadIdx.x;
    if (tid < n) {
        const int2 pr = pairs[tid];
        const int a = pool_row(p.kv, seq, pr.x), b = pool_row(p.kv, seq, pr.y);
        to[tid] = b < 0 ? -1 : a;
        from[tid] = b;
        if (a >= 0 && b >= 0) {
            const int64_t x = stat_index(p.kv, a, head), y = stat_index(p.kv, b, head);
            p.kv.weight[x] = p.kv.weight[y];
            p.kv.position[x] = p.kv.position[y];
        }
    }
    __syncthreads();
    const int lanes = p.row_bytes >> 4;  // lanes of a row
    for (int i = tid; i < n * lanes; i += THREADS) {
        const int r = i / lanes, off = (i - r * lanes) * 16;
        if (to[r] < 0) continue;
        const int sh = p.kv.shift;
        char* k = const_cast<char*>(p.kv.k) + head * p.kv.k_head + off;
        char* v = const_cast<char*>(p.kv.v) + head * p.kv.v_head + off;
        const uint4 a = *(const uint4*)(k + row_offset(from[r], sh, p.kv.k_page, p.kv.k_row));
        const uint4 b = *(const uint4*)(v + row_offset(from[r], sh, p.kv.v_page, p.kv.v_row));
        *(uint4*)(k + row_offset(to[r], sh, p.kv.k_page, p.kv.k_row)) = a;
        *(uint4*)(v + row_offset(to[r], sh, p.kv.v_page, p.kv.v_row)) = b;
    }
    __syncthreads();
}

// One workgroup for a sequence's key head: the budget-th largest key by four
// passes of eight bits over a histogram, then the slots that stay and lie at or
// above the budget (movers) against those that go and lie below it (holes),
// both in rising order by ballots and one scan over the waves.  Each pair is
// one row to copy, so no more than min(budget, len - budget) rows move
// and none is both read and written: the copies need no order.
// What it reads is little (8 bytes a slot); its passes over LDS and their barriers bound it: 1,056 slots 16 us with 32 rows
// moved, 64 sequences of 1,033 to 4,068 slots on 8 key heads 22 us.
// CACHED: keys held in LDS (what does not fit is made again from the cache in every pass: 28,000 slots shrunk to 1,024 take 60 us,
// 60,000 slots 188).  MOVE: the rows are few and
// the workgroup moves them itself, for one launch fewer.
template <int THREADS, int CACHED, bool MOVE>
__global__ __launch_bounds__(THREADS) void k_evict_select(EvictArgs p, int64_t pairs_max, int2* pairs,
                                                           int* counts) {
    constexpr int WAVES = THREADS / 64;
    const int seq = blockIdx.x / p.kv.kv_heads, head = blockIdx.x - seq * p.kv.kv_heads;
    const int len = seq_len(p.kv, seq);
    if (head == 0 && threadIdx.x == 0) p.new_len[seq] = min(len, p.budget);
    if (len <= p.budget) {
        if (!MOVE && threadIdx.x == 0) counts[blockIdx.x] = 0;
        return;
    }
    __shared__ int2 own[MOVE ? kOwnPairs : 1];
    __shared__ uint32_t keys[CACHED];
    __shared__ int hist[256 * kCopies];
    __shared__ int wave_a[WAVES], wave_b[WAVES];
    __shared__ uint32_t found;
    __shared__ int found_rank;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int recent_from = (int)max((int64_t)p.next[seq] - p.recent, (int64_t)INT32_MIN);
    const Table table = table_of(p.kv, seq, len, p.next);
    // N slots THREADS apart: their loads go together, the table's first and then what it leads to
    auto keys_of = [&](int j0, auto count, uint32_t* out) {
        constexpr int N = decltype(count)::value;
        int row[N], pos[N];
        float w[N];
#pragma unroll
        for (int i = 0; i < N; i++) row[i] = table_entry(p.kv, table, min(j0 + i * THREADS, len - 1));
#pragma unroll
        for (int i = 0; i < N; i++) {
            row[i] = entry_row(p.kv, row[i], min(j0 + i * THREADS, len - 1), true);
            const int64_t at = stat_index(p.kv, row[i] < 0 ? 0 : row[i], head);
            pos[i] = p.kv.num_pages > 0 ? p.kv.position[at] : 0;
            w[i] = p.kv.num_pages > 0 ? p.kv.weight[at] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < N; i++) out[i] = rank_key(row[i] >= 0, pos[i], w[i], p.first, recent_from);
    };
    for (int j = tid; j < len && j < CACHED; j += 8 * THREADS) {
        uint32_t k[8];
        keys_of(j, std::integral_constant<int, 8>(), k);
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (j + i * THREADS < min(len, CACHED)) keys[j + i * THREADS] = k[i];
    }
    auto key_of = [&](int j) {
        uint32_t k;
        keys_of(j, std::integral_constant<int, 1>(), &k);
        return k;
    };
    auto key_at = [&](int j) { return j < CACHED ? keys[j] : key_of(j); };

    uint32_t prefix = 0;
    int rank = p.budget;  // the rank-th largest among the keys that agree with prefix
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256 * kCopies; i += THREADS) hist[i] = 0;
        __syncthreads();
        const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
        for (int j = tid; j < len; j += THREADS) {
            const uint32_t k = key_at(j);
            if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift & 255) * kCopies + lane % kCopies], 1);
        }
        __syncthreads();
        if (wave == 0) {
            // bins from the largest: lane l has 255 - 4 l and the three below
            int c[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                c[i] = 0;
#pragma unroll
                for (int x = 0; x < kCopies; x++) c[i] += hist[(255 - 4 * lane - i) * kCopies + (x + lane) % kCopies];
                sum += c[i];
            }
            int incl = sum;
            for (int d = 1; d < 64; d <<= 1) {
                const int x = __shfl_up(incl, d);
                if (lane >= d) incl += x;
            }
            int above = incl - sum;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if (above < rank && rank <= above + c[i]) {
                    found = prefix | (uint32_t)(255 - 4 * lane - i) << shift;
                    found_rank = rank - above;
                }
                above += c[i];
            }
        }
        __syncthreads();
        prefix = found;
        rank = found_rank;
    }
    // kept: keys above ``prefix``, and the first ``rank`` slots of those equal to it
    const uint32_t edge = prefix;
    const int room = rank;
    const int span = ((len + THREADS - 1) / THREADS) * 64;  // slots of a wave
    const int lo = min(wave * span, len), hi = min(lo + span, len);
    int ties = 0;
    for (int j0 = lo; j0 < hi; j0 += 64) {
        const int j = j0 + lane;
        ties += __popcll(__ballot(j < hi && key_at(j) == edge));
    }
    if (lane == 0) wave_a[wave] = ties;
    __syncthreads();
    int ties_before = 0;
    for (int w = 0; w < wave; w++) ties_before += wave_a[w];
    __syncthreads();
    const uint64_t below = (1ull << lane) - 1;
    int holes = 0, movers = 0;
    for (int sweep = 0; sweep < 2; sweep++) {
        int seen = ties_before;
        int hole_at = 0, mover_at = 0;
        if (sweep == 1) {
            if (lane == 0) wave_a[wave] = holes, wave_b[wave] = movers;
            __syncthreads();
            for (int w = 0; w < wave; w++) hole_at += wave_a[w], mover_at += wave_b[w];
        }
        int2* out = MOVE ? own : pairs + (int64_t)blockIdx.x * pairs_max;
        for (int j0 = lo; j0 < hi; j0 += 64) {
            const int j = j0 + lane;
            const bool in = j < hi;
            const uint32_t k = in ? key_at(j) : 0u;
            const bool tie = in && k == edge;
            const uint64_t tied = __ballot(tie);
            const bool kept = in && (k > edge || (tie && seen + __popcll(tied & below) < room));
            seen += __popcll(tied);
            const bool hole = in && !kept && j < p.budget, mover = kept && j >= p.budget;
            const uint64_t hb = __ballot(hole), mb = __ballot(mover);
            if (sweep == 0) {
                holes += __popcll(hb);
                movers += __popcll(mb);
            } else {
                if (hole) out[hole_at + __popcll(hb & below)].x = j;
                if (mover) out[mover_at + __popcll(mb & below)].y = j;
                hole_at += __popcll(hb);
                mover_at += __popcll(mb);
            }
        }
        if (!MOVE && sweep == 1 && wave == WAVES - 1 && lane == 0) counts[blockIdx.x] = hole_at;
    }
    if constexpr (MOVE) {
        __shared__ int to[kMoveRows], from[kMoveRows];
        int count = 0;
        for (int w = 0; w < WAVES; w++) count += wave_a[w];
        __syncthreads();
        for (int first = 0; first < count; first += kMoveRows)
            move_pairs<THREADS>(p, seq, head, own + first, min(kMoveRows, count - first), to, from);
    }
}

// Copies the movers' rows into the holes, a workgroup for kMoveRows pairs: its bytes bound it (64 prompts shrunk to
// 1,024 slots each move 285 MB, read and written, in 62 us).
__global__ __launch_bounds__(256) void k_evict_move(EvictArgs p, int64_t pairs_max, const int2* pairs,
                                                    const int* counts) {
    const int at = blockIdx.x, seq = at / p.kv.kv_heads, head = at - seq * p.kv.kv_heads;
    const int count = counts[at];
    __shared__ int to[kMoveRows], from[kMoveRows];
    for (int64_t first = (int64_t)blockIdx.y * kMoveRows; first < count; first += (int64_t)gridDim.y * kMoveRows)
        move_pairs<256>(p, seq, head, pairs + at * pairs_max + first, (int)min((int64_t)kMoveRows, count - first), to, from);
}

}  // namespace

int64_t evict_threads(const EvictArgs& a) {
    return (int64_t)a.kv.seqs * a.kv.kv_heads * (((int64_t)a.kv.width << a.kv.shift) <= 4096 ? 512 : 1024);
}

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
    const int segs = a.kv.seqs * a.kv.kv_heads;
    const int64_t cap = (int64_t)a.kv.width << a.kv.shift;
    const int64_t pairs_max = evict_pairs(cap, a.budget);
    int* counts = (int*)a.ws;
    int2* pairs = (int2*)(a.ws + (((int64_t)segs * 4 + 255) & ~int64_t(255)));
    // Up to 4,096 slots four workgroups of a CU side by side (64 prompts of 1,033 to 4,068 slots: 256 threads each 103 us,
    // 512 threads 95, 1,024 threads 99); longer ones one, with up to 28,672 keys in 112 KB of its LDS.
    const bool move = pairs_max <= kOwnPairs;
    const hipError_t e =
        cap <= 4096 ? run(move ? k_evict_select<512, 4096, true> : k_evict_select<512, 4096, false>, dim3(segs), 512, s, a, pairs_max, pairs, counts)
                    : run(move ? k_evict_select<1024, 28672, true> : k_evict_select<1024, 28672, false>, dim3(segs), 1024, s, a, pairs_max, pairs, counts);
    if (e != hipSuccess || move) return e;
    const int64_t blocks = (pairs_max + kMoveRows - 1) / kMoveRows;
    const unsigned y = (unsigned)(blocks < 1 ? 1 : blocks > 4096 ? 4096 : blocks);
    return run(k_evict_move, dim3(segs, y), 256, s, a, pairs_max, pairs, counts);
}

}  // namespace svfk
