// svf_logprob.hip -- log probabilities of given tokens, entropies and the best alternatives of rows of logits.
#include <type_traits>

#include "svf_kv_device.h"
#include "svf_logprob.h"

#pragma clang fp contract(off)  // a reference and a distance from it are rounded as they are written

namespace svfp {
namespace {

constexpr float kLn2 = 0.69314718055994531f;
constexpr int kListed = 512;  // pieces of a row that may hold one of the best
constexpr int kMostParts = 64, kJoined = 2048;  // parts of a row, and best of all of them
constexpr int kUsual = 512;  // threads of a workgroup

// Pieces of a row whose largest logits a workgroup keeps in LDS. (Logits that may be one of the best, in the pieces' place, are half as many.)
constexpr int entries_of(int threads) { return threads < kUsual ? 1024 : 4096; }

// What a part of a row found: its largest logit, the sum of 2^y and of y 2^y over its logits, y their distance from that in log2 terms, and how
// many come before the token.
struct Part {
    float m, s, sy;
    int32_t before;
};

// How a row is dealt out.
struct Plan {
    int32_t parts;   // workgroups of a row
    int32_t per;     // whole 16-byte vectors of a part, a multiple of 32
    int32_t group;   // log2 of the vectors of a piece: 0, 3 or 5, by the length of a part
    Part* part;      // [rows][parts] (parts > 1)
    uint64_t* keys;  // [rows][parts][top]
};

// A logit's place in the order as a whole number, larger first: -0 as 0, NaN below all.
__device__ inline uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return x != x ? 0u : u >> 31 ? ~u : u | 0x80000000u;
}
__device__ inline float logit_of(uint32_t order) {
    return order == 0 ? __builtin_nanf("") : __uint_as_float(order >> 31 ? order & 0x7fffffffu : ~order);
}
// With the index behind it, so that no two are equal; 0 is none.
__device__ inline uint64_t key_of(float x, int i) { return (uint64_t)order_of(x) << 32 | (uint32_t)~i; }

// The next number above (NaN above +infinity).
__device__ inline float above(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return __uint_as_float(u >> 31 ? u - 1 : u + 1);
}

template <class T>
struct Logits {
    static constexpr int W = 16 / sizeof(T);  // of a vector
    static __device__ inline float at(const uint4& w, int i) {
        const uint32_t x = (&w.x)[i * (int)sizeof(T) / 4];
        if constexpr (sizeof(T) == 4) return __uint_as_float(x);
        if constexpr (__is_same(T, __bf16)) return __uint_as_float(i & 1 ? x & 0xffff0000u : x << 16);
        if constexpr (__is_same(T, _Float16)) return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? x >> 16 : x));
    }
    static __device__ inline float largest(const uint4& w) {
        if constexpr (__is_same(T, _Float16)) {  // two at a time
            typedef _Float16 V2 __attribute__((ext_vector_type(2)));
            const V2 x = __builtin_elementwise_max(
                __builtin_elementwise_max(__builtin_bit_cast(V2, w.x), __builtin_bit_cast(V2, w.y)),
                __builtin_elementwise_max(__builtin_bit_cast(V2, w.z), __builtin_bit_cast(V2, w.w)));
            return fmaxf((float)x.x, (float)x.y);
        }
        float x = fmaxf(at(w, 0), at(w, 1));
#pragma unroll
        for (int i = 2; i < W; i += 2) x = fmaxf(x, fmaxf(at(w, i), at(w, i + 1)));
        return x;
    }
    // Of U vectors.  In bfloat16 a word as a 32-bit number is its upper logit with some bits behind it, or, if that is infinite, no number:
    // +infinity may be missed, which the row's sum then shows.
    template <int U>
    static __device__ inline float largest(const uint4 (&w)[U]) {
        float x = -INFINITY, upper = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; u++) {
            if constexpr (__is_same(T, __bf16)) {
                upper = fmaxf(fmaxf(upper, fmaxf(__uint_as_float(w[u].x), __uint_as_float(w[u].y))),
                              fmaxf(__uint_as_float(w[u].z), __uint_as_float(w[u].w)));
                x = fmaxf(fmaxf(x, fmaxf(at(w[u], 0), at(w[u], 2))), fmaxf(at(w[u], 4), at(w[u], 6)));
            } else {
                x = fmaxf(x, largest(w[u]));
            }
        }
        return fmaxf(x, __uint_as_float(__float_as_uint(upper) & 0xffff0000u));
    }
};

// What another lane of the same sixteen has.
template <int Ctrl, class V>
__device__ inline V from_near(V x) {
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), Ctrl, 0xf, 0xf, true));
}
template <class V, class Op>
__device__ inline V over_8(V x, Op op) {
    x = op(x, from_near<0xb1>(x));         // quad_perm 1 0 3 2
    x = op(x, from_near<0x4e>(x));         // quad_perm 2 3 0 1
    return op(x, from_near<0x141>(x));     // the eight lanes the other way round
}
template <class V, class Op>
__device__ inline V over_wave(V x, Op op) {
    if constexpr (sizeof(V) == 4) {
        x = over_8(x, op);
        x = op(x, from_near<0x140>(x));    // the sixteen the other way round
    } else {
        for (int d = 1; d < 16; d <<= 1) x = op(x, __shfl_xor(x, d));
    }
    x = op(x, __shfl_xor(x, 16));
    return op(x, __shfl_xor(x, 32));
}

template <int NT, class V, class Op>
__device__ inline V over_group(V x, Op op) {
    __shared__ V part[NT / 64];
    x = over_wave(x, op);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    x = part[0];
    for (int i = 1; i < NT / 64; i++) x = op(x, part[i]);
    return x;
}

// Each line of a row is read once, by eight lanes: past the caches (4,001 rows of 128,000, 1,024 MB: 174 us, and 183 through them; 203
// rows, eight waves each then, 23.4 and 24.0; 517 rows of 50,001 in 32 bits, whose lines do not begin with a row, 28 both ways, and 30 before the grid began at a line).
__device__ inline uint4 load_once(const uint4* at) {
    typedef uint32_t V4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(uint4, __builtin_nontemporal_load((const V4*)at));
}

// The distance of a logit from the largest of all in log2 terms (by halves, so that it does not pass what 32 bits hold on the way).
__device__ inline float distance(float x, float m, float scale2) { return (0.5f * x - 0.5f * m) * (2.f * scale2); }

// What a row's sums come to: whether it has no distribution, or nothing that is allowed, and the logarithm of its sum. The largest logit's own power is 1, so
// no sum is below that; rounded from a lane's reference and back it can be 1 - 2^-24, and a certain token would have a
// probability above 1.
struct Total {
    bool bad, none;
    float sum, log;
};
__device__ inline Total total_of(const Part& x) {
    Total t;
    t.bad = !(x.s * 0.f == 0.f) || x.m == INFINITY;
    t.none = x.m == -INFINITY && x.s == 0.f;
    t.sum = fmaxf(x.s, 1.f);
    t.log = __builtin_amdgcn_logf(t.sum) * kLn2;
    return t;
}
__device__ inline void write_row(const Args& p, int row, const Part& x, bool known, float mine) {
    const Total t = total_of(x);
    const float nan = __builtin_nanf("");
    p.logprob[row] = !known || t.bad ? nan : t.none ? -INFINITY : distance(mine, x.m, p.scale) - t.log;
    p.entropy[row] = t.bad ? nan : t.none ? 0.f : fmaxf(t.log - x.sy / t.sum * kLn2, 0.f);
    p.rank[row] = known ? x.before : -1;
}
__device__ inline void write_top(const Args& p, int row, int at, const Part& x, uint64_t key) {
    const Total t = total_of(x);
    p.top_index[(int64_t)row * p.top + at] = (int)~(uint32_t)key;
    p.top_logprob[(int64_t)row * p.top + at] =
        t.bad ? __builtin_nanf("") : t.none ? -INFINITY : distance(logit_of((uint32_t)(key >> 32)), x.m, p.scale) - t.log;
}

// The logits of one part: vectors [v0, v1) of the row's grid, and with the first part the up to 9 W - 2 logits before its first line
// and behind its last whole vector.  The grid begins at a line of 128 bytes; vector v holds the logits v * W - off and following.
template <class T>
struct Span {
    const T* x;
    int off, lead, tail, vocab;  // logits [0, lead) and [tail, vocab) lie outside whole vectors
    int v0, v1;
    bool edges;
    __device__ inline int edge_count() const { return edges ? lead + vocab - tail : 0; }
    __device__ inline int edge(int i) const { return i < lead ? i : tail + i - lead; }
    // all of the part, in rising order
    __device__ inline int body() const { return v0 * Logits<T>::W - off; }
    __device__ inline int count() const { return edge_count() + (v1 - v0) * Logits<T>::W; }
    __device__ inline int nth(int i) const {
        const int first = edges ? lead : 0, in = (v1 - v0) * Logits<T>::W;
        return i < first ? i : i - first < in ? body() + i - first : tail + i - first - in;
    }
};

template <class T>
__device__ inline Span<T> span_of(const Args& p, const Plan& plan, int row, int part) {
    constexpr int W = Logits<T>::W;
    Span<T> s;
    s.x = (const T*)(p.logits + row * p.row_stride);
    s.vocab = p.vocab;
    s.off = (int)((uint64_t)s.x & 127) / (int)sizeof(T);
    s.lead = min(s.vocab, s.off ? 8 * W - s.off : 0);
    const int first = s.off ? 8 : 0, end = max(first, (s.vocab + s.off) / W);
    s.tail = min(s.vocab, max(s.lead, end * W - s.off));
    s.v0 = (int)min((int64_t)end, first + (int64_t)part * plan.per);
    s.v1 = min(end, s.v0 + plan.per);
    s.edges = part == 0;
    return s;
}

// One pass over a row's logits, or a part of them, in 16-byte loads, 64 bytes a lane on their way while as many are worked on. Each lane
// keeps sums of 2^y and y 2^y, y the distance from a reference of its own that follows the largest logit it has met where that has
// grown by more than 2^8.  Logits that may come before the token are counted only where a vector has one: with likely tokens hardly anywhere.
//
// The best alternatives: the largest logit of every piece of the row (512 bytes, four vectors of eight lanes; 128 or 16 bytes
// where the row is short) goes to LDS.  Pieces in 64 (or 128) bins: the top-th largest of the bins' best is a bound that at
// least ``top`` logits reach, so only pieces whose largest reaches it are read again, some more than ``top``, and of their logits those that reach it
// are put in order by counting.  Where too few are larger than -infinity, the lowest indices follow.  Where too many reach it (pieces full
// of one logit: a mask's finite number, say), or a logit is no number, the row is read twice again for a bound that no two logits
// share: the top-th largest key of the best that each thread meets.  Where too many reach that (one thread meets them all), ``top`` rounds over the
// row find them one by one.  (203 rows of 128,000 in bfloat16, three tokens allowed and the others at the type's lowest number: 69 us with 20
// best and 77 with 64, 1,042 and 3,239 by rounds, 53 and 54 with the others at -infinity.)
template <class T, bool TOP, int NT>
__global__ __launch_bounds__(NT, NT == 1024 ? 4 : 6) void k_score(Args p, Plan plan) {
    using L = Logits<T>;
    constexpr int W = L::W, U = 4, kEntries = entries_of(NT), kCand = kEntries / 2;
    constexpr float kSlack = 8.f;
    static_assert(9 * W - 2 <= NT, "a thread an edge");
    // the pieces' largest logits, and in their place, once those are done with, keys of logits
    __shared__ __align__(16) char board[TOP ? kEntries * sizeof(float) : 16];
    float* const largest = (float*)board;
    uint64_t* const cand = (uint64_t*)board;
    static_assert(__alignof__(board) >= alignof(uint64_t) && kCand * sizeof(uint64_t) <= kEntries * sizeof(float), "the keys fit and lie at their boundary");
    __shared__ uint16_t listed[TOP ? kListed : 1];
    __shared__ int hits[NT / 64];
    __shared__ uint64_t sh_bound;
    __shared__ int sh_listed, sh_cand;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = blockIdx.x / plan.parts, part = blockIdx.x - row * plan.parts;
    const Span<T> s = span_of<T>(p, plan, row, part);
    const uint4* at = (const uint4*)((uint64_t)s.x & ~(uint64_t)127);
    // (the last vectors of a part by themselves: logits of -infinity in the place of those that are not there)
    constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : __is_same(T, __bf16) ? 0xff80ff80u : 0xfc00fc00u;
    const int whole = (s.v1 - s.v0) / (U * NT);
    int v = s.v0 + (tid >> 3) * (8 * U) + (tid & 7);  // eight lanes have U lines that follow each other
    uint4 next[U];
    auto fetch = [&](int v) {
        if (s.v0 == s.v1) return;
#pragma unroll
        for (int u = 0; u < U; u++) next[u] = load_once(at + min(v + u * 8, s.v1 - 1));
    };
    fetch(v);
    __builtin_amdgcn_sched_barrier(0);  // on their way before the token's
    const int64_t token = p.token_wide ? ((const int64_t*)p.token)[row] : ((const int32_t*)p.token)[row];
    const bool known = token >= 0 && token < p.vocab;
    const float mine = known ? (float)s.x[token] : __builtin_nanf("");
    const float over = mine == mine ? above(mine) : mine;
    const int vt = known ? ((int)token + s.off) / W : 0, vb = min(vt, s.v1);  // its vector, and the last one before it

    float m = -INFINITY, b = 3e38f, sum = 0.f, sumy = 0.f;
    int before = 0;  // of the whole wave
    bool masked = false;
    const float c = p.scale2;
    // the same vector, whose logits are taken out of it again: kept from one use to the next they would need more registers than there are
    auto again = [](uint4 w) {
        asm volatile("" : "+v"(w.x), "+v"(w.y), "+v"(w.z), "+v"(w.w));
        return w;
    };
    auto work = [&](const uint4(&w)[U], int v, bool all) {
        const float most = L::largest(w);
        if constexpr (TOP) {
            const auto more = [](float a, float b) { return fmaxf(a, b); };
            if (plan.group == 5) {
                const float x = over_8(most, more);
                if ((lane & 7) == 0 && (all || v < s.v1)) largest[(v - s.v0) >> 5] = x;
            } else if (plan.group == 3) {
#pragma unroll
                for (int u = 0; u < U; u++) {
                    const float x = over_8(L::largest(again(w[u])), more);
                    if ((lane & 7) == 0 && (all || v + u * 8 < s.v1)) largest[(v - s.v0 + u * 8) >> 3] = x;
                }
            } else {
#pragma unroll
                for (int u = 0; u < U; u++)
                    if (all || v + u * 8 < s.v1) largest[v - s.v0 + u * 8] = L::largest(again(w[u]));
            }
        }
        m = fmaxf(m, most);
        const float ref = fmaxf(most, p.low), far = fmaf(ref, c, b);
        if (__any(far > kSlack)) {
            const float now = far > kSlack ? -ref * c : b, step = now - b, keep = __builtin_amdgcn_exp2f(step);
            sumy = keep * fmaf(sum, step, sumy);
            sum *= keep;
            b = now;
        }
        if (__any(most >= mine)) {
#pragma unroll
            for (int u = 0; u < U; u++) {
                const float least = v + u * 8 < vb ? mine : over;
#pragma unroll
                for (int i = 0; i < W; i++) before += __popcll(__ballot(L::at(w[u], i) >= least));
            }
        }
        // A vector's powers by themselves, the vectors', then all that there were before: one after another, those of unlikely tokens would be
        // lost beside a likely one's 1.  0 times -infinity is 0: from the first such logit of a wave on, distances are kept above
        // what gives 0.
        auto powers = [&](auto low) {
            float more = 0.f, morey = 0.f;
#pragma unroll
            for (int u = 0; u < U; u++) {
                const uint4 x = low || __is_same(T, _Float16) ? again(w[u]) : w[u];
                float part = 0.f, party = 0.f;
#pragma unroll
                for (int i = 0; i < W; i++) {
                    const float y = fmaf(L::at(x, i), c, b), e = __builtin_amdgcn_exp2f(y), near = low ? fmaxf(y, -200.f) : y;
                    part = i ? part + e : e;
                    party = i ? fmaf(e, near, party) : e * near;
                }
                more = u ? more + part : part;
                morey = u ? morey + party : party;
            }
            if (!low && __any(morey != morey)) return false;
            sum += more;
            sumy += morey;
            return true;
        };
        if (!masked && powers(std::false_type())) return;
        powers(std::true_type());
        masked = true;
    };
    for (int it = 0; it < whole; it++, v += U * NT) {
        uint4 w[U];
#pragma unroll
        for (int u = 0; u < U; u++) w[u] = next[u];
        fetch(v + U * NT);
        work(w, v, true);
    }
    if (whole * U * NT < s.v1 - s.v0) {
#pragma unroll
        for (int u = 0; u < U; u++)
            if (v + u * 8 >= s.v1) next[u] = make_uint4(kNone, kNone, kNone, kNone);
        masked = masked || __any(v + (U - 1) * 8 >= s.v1);
        work(next, v, false);
    }
    const int edges = s.edge_count();
    const uint64_t mine_key = known ? key_of(mine, (int)token) : ~0ull;
    bool edge_before = false;
    if (tid < edges) {
        const int i = s.edge(tid);
        const float x = (float)s.x[i];
        m = fmaxf(m, x);
        const float ref = fmaxf(x, p.low), far = fmaf(ref, c, b);
        if (far > kSlack) {
            const float step = -ref * c - b, keep = __builtin_amdgcn_exp2f(step);
            sumy = keep * fmaf(sum, step, sumy);
            sum *= keep;
            b = -ref * c;
        }
        const float y = fmaf(x, c, b), e = __builtin_amdgcn_exp2f(y);
        sum += e;
        sumy = fmaf(e, fmaxf(y, -200.f), sumy);
        edge_before = mine == mine && key_of(x, i) > mine_key;
    }
    int equal = 0;
    if (known && tid == 0 && vt >= s.v0 && vt < s.v1)  // equal logits before the token in its own vector
        for (int i = vt * W - s.off; i < (int)token; i++) equal += (float)s.x[i] == mine;
    before += __popcll(__ballot(edge_before)) + __builtin_amdgcn_readfirstlane(equal);

    // The row's scalars: the largest logit, then the sums relative to it.
    auto add = [](auto a, auto b) { return a + b; };
    __shared__ float group_m[NT / 64];
    __shared__ Part group[NT / 64];
    Part x;
    x.m = over_wave(m, [](float a, float b) { return fmaxf(a, b); });
    if (lane == 0) group_m[wave] = x.m;
    if (TOP && tid == 0) sh_listed = 0, sh_cand = 0;
    __syncthreads();
    const int shift = plan.group, entries = (s.v1 - s.v0 + (1 << shift) - 1) >> shift;
    if (TOP && wave == 0) {
        // The bound, by the first wave while the others add up: the top-th largest of 64 bins' best pieces, or of 128.
        const bool two = p.top > 32;
        float most[2] = {-INFINITY, -INFINITY};
        int at[2] = {0, 0};
        auto take = [&](int e, int i) {
            const float y = e < entries ? largest[e] : -INFINITY;
            if (y > most[i]) most[i] = y, at[i] = e;
        };
        for (int e = lane; e < entries; e += 256) {
            take(e, 0), take(e + 128, 0);
            if (two)
                take(e + 64, 1), take(e + 192, 1);
            else
                take(e + 64, 0), take(e + 192, 0);
        }
        uint64_t best[2];
#pragma unroll
        for (int i = 0; i < 2; i++) best[i] = most[i] > -INFINITY ? key_of(most[i], at[i]) : 0;
        int larger[2] = {0, 0};
        auto count = [&](uint64_t x, auto both) {
#pragma unroll
            for (int i = 0; i < 64; i++) {
                const uint64_t y = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), i) << 32 |
                                   (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, i);
                larger[0] += y > best[0];
                if (both) larger[1] += y > best[1];
            }
        };
        if (two) {
            count(best[0], std::true_type());
            count(best[1], std::true_type());
        } else {
            count(best[0], std::false_type());
        }
        if (lane == 0) sh_bound = 0;
#pragma unroll
        for (int i = 0; i < 2; i++)
            if (larger[i] == p.top - 1 && best[i] != 0) sh_bound = best[i];
    }
    for (int i = 0; i < NT / 64; i++) x.m = fmaxf(x.m, group_m[i]);
    {
        // (a part without a logit above -infinity has no distances)
        const float d = x.m == -INFINITY ? 0.f : fmaf(x.m, c, b), f = __builtin_amdgcn_exp2f(-d), dc = fminf(d, 1000.f);
        sumy = over_wave(f * fmaf(sum, -dc, sumy), add);
        sum = over_wave(sum * f, add);
    }
    if (lane == 0) group[wave] = Part{0.f, sum, sumy, before};
    __syncthreads();
    x.s = x.sy = 0.f, x.before = 0;
    for (int i = 0; i < NT / 64; i++) x.s += group[i].s, x.sy += group[i].sy, x.before += group[i].before;
    // Logits so large that a reference in log2 terms is rounded by more than 2^-4, or none in 32 bits: once more, each distance by itself.
    if (x.m != -INFINITY && !(fabsf(x.m * c) < -kFarthest) && x.m != INFINITY) {
        sum = sumy = 0.f;
        for (int i = tid; i < s.count(); i += NT) {
            const float y = distance((float)s.x[s.nth(i)], x.m, c), e = __builtin_amdgcn_exp2f(y);
            sum += e;
            sumy = fmaf(e, fmaxf(y, -200.f), sumy);
        }
        x.s = over_group<NT>(sum, add);
        x.sy = over_group<NT>(sumy, add);
    }
    const bool bad = !(x.s * 0.f == 0.f);  // a logit that is no number, or +infinity
    if (known && (mine != mine || bad)) {  // a token that is no number comes behind all that are
        before = 0;
        for (int i = tid; i < s.count(); i += NT) before += key_of((float)s.x[s.nth(i)], s.nth(i)) > mine_key;
        x.before = over_group<NT>(before, add);
    }
    if (tid == 0) {
        if (plan.parts == 1)
            write_row(p, row, x, known, mine);
        else
            plan.part[blockIdx.x] = x;
    }
    if constexpr (TOP) {
        auto emit = [&](int at, uint64_t key) {
            if (plan.parts == 1)
                write_top(p, row, at, x, key);
            else
                plan.keys[(int64_t)blockIdx.x * p.top + at] = key;
        };
        // the pieces that reach the bound
        const uint64_t bound = sh_bound;
        const float bound_logit = bound ? logit_of((uint32_t)(bound >> 32)) : -INFINITY;
        for (int e = tid; e < entries; e += NT) {
            if (!(largest[e] >= bound_logit) || largest[e] == -INFINITY || key_of(largest[e], e) < bound) continue;
            const int to = atomicAdd(&sh_listed, 1);
            if (to < kListed) listed[to] = (uint16_t)e;
        }
        __syncthreads();
        // the logits that reach it, in the pieces' place
        const int pieces = min(sh_listed, kListed);
        for (int i0 = tid; i0 < pieces << shift; i0 += 2 * NT) {
            uint4 w[2];
            int e[2], v[2];
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const int i = i0 + k * NT;
                e[k] = listed[min(i >> shift, pieces - 1)];
                v[k] = i < pieces << shift ? s.v0 + (e[k] << shift) + (i & ((1 << shift) - 1)) : s.v1;
                if (v[k] < s.v1) w[k] = at[v[k]];
            }
#pragma unroll
            for (int k = 0; k < 2; k++) {
                if (v[k] >= s.v1 || !(L::largest(w[k]) >= bound_logit)) continue;
#pragma unroll
                for (int j = 0; j < W; j++) {
                    const float y = L::at(w[k], j);
                    if (!(y >= bound_logit) || y == -INFINITY || key_of(y, e[k]) < bound) continue;
                    const int to = atomicAdd(&sh_cand, 1);
                    if (to < kCand) cand[to] = key_of(y, v[k] * W - s.off + j);
                }
            }
        }
        if (tid < edges) {
            const float y = (float)s.x[s.edge(tid)];
            if (y > -INFINITY) {
                const int to = atomicAdd(&sh_cand, 1);
                if (to < kCand) cand[to] = key_of(y, s.edge(tid));
            }
        }
        __syncthreads();
        int n = sh_cand;
        auto order = [&](int n) {
            for (int i = tid; i < n; i += NT) {
                const uint64_t key = cand[i];
                int larger = 0;
#pragma unroll 8
                for (int j = 0; j < n; j++) larger += cand[j] > key;
                if (larger < p.top) emit(larger, key);
            }
            for (int i = n + tid; i < p.top; i += NT) emit(i, 0);  // a part with fewer logits
        };
        if (n <= kCand && sh_listed <= kListed && !bad) {
            // too few: the lowest indices of -infinity, then of NaN
            for (int kind = 0; kind < 2 && n < p.top; kind++)
                for (int i0 = 0; i0 < s.count() && n < p.top; i0 += NT) {
                    const int i = i0 + tid, j = i < s.count() ? s.nth(i) : 0;
                    const float y = i < s.count() ? (float)s.x[j] : 0.f;
                    const bool hit = kind ? y != y : y == -INFINITY;
                    const uint64_t mask = __ballot(hit);
                    __syncthreads();
                    if (lane == 0) hits[wave] = __popcll(mask);
                    __syncthreads();
                    int to = n + __popcll(mask & ((1ull << lane) - 1));
                    for (int w = 0; w < NT / 64; w++) {
                        if (w < wave) to += hits[w];
                        n += hits[w];
                    }
                    if (hit && to < kCand) cand[to] = key_of(y, j);
                }
            n = min(n, kCand);
            __syncthreads();
            order(n);
            return;
        }
        // every key of the part
        auto each = [&](auto take) {
            for (int v = s.v0 + tid; v < s.v1; v += NT) {
                const uint4 w = at[v];
#pragma unroll
                for (int j = 0; j < W; j++) take(key_of(L::at(w, j), v * W - s.off + j));
            }
            if (tid < edges) take(key_of((float)s.x[s.edge(tid)], s.edge(tid)));
        };
        static_assert(NT <= kCand, "a key a thread");
        uint64_t best = 0;
        each([&](uint64_t key) { best = max(best, key); });
        __syncthreads();  // all have read the counters
        cand[tid] = best;
        if (tid == 0) sh_bound = 0, sh_cand = 0;
        __syncthreads();
        if (best != 0) {
            int larger = 0;
#pragma unroll 8
            for (int j = 0; j < NT; j++) larger += cand[j] > best;
            if (larger == p.top - 1) sh_bound = best;
        }
        __syncthreads();
        const uint64_t least = sh_bound;
        each([&](uint64_t key) {
            if (key < least) return;
            const int to = atomicAdd(&sh_cand, 1);
            if (to < kCand) cand[to] = key;
        });
        __syncthreads();
        n = sh_cand;
        if (n <= kCand) {
            order(n);
        } else {
            uint64_t last = ~0ull;
            for (int k = 0; k < p.top; k++) {
                uint64_t best = 0;
                for (int i = tid; i < s.count() && last; i += NT) {
                    const uint64_t key = key_of((float)s.x[s.nth(i)], s.nth(i));
                    if (key < last) best = max(best, key);
                }
                last = over_group<NT>(best, [](uint64_t a, uint64_t b) { return max(a, b); });
                if (tid == 0) emit(k, last);
            }
        }
    }
}

// The parts of a row: its scalars, and of the parts' best the best.
template <class T>
__global__ __launch_bounds__(256) void k_join(Args p, Plan plan) {
    __shared__ uint64_t cand[kJoined];
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const int64_t token = p.token_wide ? ((const int64_t*)p.token)[row] : ((const int32_t*)p.token)[row];
    const bool known = token >= 0 && token < p.vocab;
    Part x = lane < plan.parts ? plan.part[(int64_t)row * plan.parts + lane] : Part{-INFINITY, 0.f, 0.f, 0};
    float m = x.m;
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    const float d = m == -INFINITY ? 0.f : x.m == -INFINITY ? -INFINITY : distance(x.m, m, p.scale2), f = __builtin_amdgcn_exp2f(d);
    x.sy = f * fmaf(x.s, fmaxf(d, -1000.f), x.sy);
    x.s *= f;
    for (int k = 32; k; k >>= 1) {
        x.s += __shfl_xor(x.s, k);
        x.sy += __shfl_xor(x.sy, k);
        x.before += __shfl_xor(x.before, k);
    }
    x.m = m;
    if (tid == 0) write_row(p, row, x, known, known ? (float)((const T*)(p.logits + row * p.row_stride))[token] : 0.f);
    const int n = plan.parts * p.top;
    for (int i = tid; i < n; i += 256) cand[i] = plan.keys[(int64_t)row * n + i];
    __syncthreads();
    for (int i = tid; i < n; i += 256) {
        const uint64_t key = cand[i];
        int larger = 0;
#pragma unroll 8
        for (int j = 0; j < n; j++) larger += cand[j] > key;
        if (key != 0 && larger < p.top) write_top(p, row, larger, x, key);
    }
}

struct Layout {
    int32_t parts, per, group, threads;
    int64_t keys, bytes;
};

Layout layout(int32_t rows, int32_t vocab, int32_t top, int32_t dtype) {
    Layout y;
    const int64_t vectors = (int64_t)vocab / (dtype == SVF_LOGITS_F32 ? 4 : 8) + 1;
    // Two waves a row where many rows are short, so that what follows a row's last logit is done for more rows at a time (bf16, best 20: 4,000
    // rows of 2,644 26.7 us, 65.8 with eight waves; 1,548 of 8,000 19.5 and 28.4; 600 of 1,229 11.4 and 13.5), and not where rows are few
    // (256 of 8,000 12.7, 10.6 with eight) or long (600 of 16,000 18.4 and 15.9).  With one wave 4,000 of 2,644 24.6, but 600 14.3 and 11.9.
    y.threads = rows > 512 && vectors <= 1024 ? 128 : kUsual;
    // as many parts as the GPU has CUs for and as a join can order candidates of, none of fewer vectors than eight a thread
    int64_t parts = 256 / (rows < 1 ? 1 : rows);
    if (parts > vectors / (8 * kUsual)) parts = vectors / (8 * kUsual);
    if (top > 0 && parts > kJoined / 4 / top) parts = kJoined / 4 / top;
    // a part's pieces have to fit
    const int64_t most = (int64_t)entries_of(kUsual) * 32, least = (vectors + most - 33) / (most - 32);
    if (parts < least) parts = least;
    if (parts > kMostParts) parts = kMostParts;
    if (parts < 1) parts = 1;
    // Sixteen waves where a CU has but one row and that is long, for twice the loads on their way (bf16: 203 rows of 128,000, 20 best, 21.5 us
    // and 23.8 with eight, 64 best 26.9 and 30.1, 150 of 151,000 25.3 and 27.7; but 203 of 64,000 18.4 and 18.1, 400 of 128,000 37.5 and 31.8,
    // and one in parts 17.8 and 17.4).
    if (parts == 1 && rows <= 256 && vectors > 12288) y.threads = 1024;
    y.parts = (int32_t)parts;
    y.per = (int32_t)(((vectors + parts - 1) / parts + 31) & ~int64_t(31));
    // some hundred pieces: few for the bound, many for 64 of them to be a small part
    y.group = y.per <= 1024 ? 0 : y.per <= 8192 ? 3 : 5;
    y.keys = ((int64_t)rows * parts * (int64_t)sizeof(Part) + 255) & ~int64_t(255);
    y.bytes = parts == 1 ? 0 : y.keys + (int64_t)rows * parts * top * 8;
    return y;
}

template <class T, int NT>
hipError_t launch_score(const Args& a, const Plan& plan, hipStream_t s) {
    return svfk::run(a.top ? k_score<T, true, NT> : k_score<T, false, NT>, dim3((unsigned)(a.rows * plan.parts)), NT, s, a, plan);
}

template <class T>
hipError_t launch_type(const Args& a, const Layout& y, hipStream_t s) {
    const Plan plan{y.parts, y.per, y.group, (Part*)a.ws, (uint64_t*)(a.ws + y.keys)};
    const hipError_t e = y.threads == 128    ? launch_score<T, 128>(a, plan, s)
                         : y.threads == 1024 ? launch_score<T, 1024>(a, plan, s)
                                             : launch_score<T, kUsual>(a, plan, s);
    if (e != hipSuccess || y.parts == 1) return e;
    return svfk::run(k_join<T>, dim3(a.rows), 256, s, a, plan);
}

}  // namespace

int64_t workspace(int32_t rows, int32_t vocab, int32_t top, int32_t dtype) { return layout(rows, vocab, top, dtype).bytes; }

int64_t threads(int32_t rows, int32_t vocab, int32_t top, int32_t dtype) {
    const Layout y = layout(rows, vocab, top, dtype);
    return (int64_t)rows * y.parts * (y.threads < kUsual ? kUsual : y.threads);  // as many rows of any vocabulary that is not split
}

hipError_t launch(const Args& a, int32_t dtype, hipStream_t s) {
    const Layout y = layout(a.rows, a.vocab, a.top, dtype);
    return dtype == SVF_LOGITS_BF16  ? launch_type<__bf16>(a, y, s)
           : dtype == SVF_LOGITS_F16 ? launch_type<_Float16>(a, y, s)
                                     : launch_type<float>(a, y, s);
}

}  // namespace svfp
