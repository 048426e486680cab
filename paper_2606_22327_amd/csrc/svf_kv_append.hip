// svf_kv_append.hip -- rotary positions on new queries and keys, and the
// write of new keys and values into their pages.
#include "svf_kv_device.h"

namespace svfk {
namespace {

// Every element is read once and written once (with the positions' rows of
// the table, which the heads of a token share): bytes bound it, and for a few
// tokens the launch.  A lane takes 16 elements of one head (the two halves of
// eight pairs, or sixteen elements in a row) in 16-byte accesses and keeps the
// pairs' cosines and sines in registers while it walks over the heads, so the
// table is read once for ``per`` heads and not with every one of them.
// 19,432 tokens of 32 query and 8 key heads of 128 dimensions (484 MB) take 100 us, 4.8 TB/s, which is what a
// copy of 4 GB reaches; one token 3.6 us.
template <class E>
__global__ __launch_bounds__(256) void k_append_wide(AppendArgs p, int units, int groups, int per) {
    using V8 = typename E::V8;
    const int wave = (blockIdx.x * 256 + threadIdx.x) >> 6;
    const int t = wave / groups, group = wave - t * groups;
    if (t >= p.kv.tokens) return;
    const int lane = threadIdx.x & 63;
    const int seq = find_seq(p.kv, t);
    const Seq s = seq_of(p.kv, seq);
    const int slot = s.len - s.n + (t - s.q0);
    const bool ours = t >= s.q0 && t < s.q0 + s.n;
    const int row = ours && slot >= 0 ? pool_row(p.kv, seq, slot) : -1;
    const int pos = p.positions[t];
    const bool known = (unsigned)pos < (unsigned)p.rope_rows;

    const int lanes = 64 / units;  // heads that the wave takes at a time
    const int u = lane % units, sub = lane / units;
    const bool turned = u * 16 < p.rot;
    const int half = p.rot >> 1;
    // elements [ea, ea + 8) and [eb, eb + 8)
    const int ea = turned && p.half_layout ? u * 8 : u * 16;
    const int eb = turned && p.half_layout ? half + u * 8 : u * 16 + 8;
    float c[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; i++) c[i] = 1.f, sn[i] = 0.f;
    if (turned) {
        const float* tab = p.rope + (int64_t)(known ? pos : 0) * p.rot + u * 8;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            c[i] = known ? tab[i] : __builtin_nanf("");
            sn[i] = known ? tab[half + i] : __builtin_nanf("");
        }
    }
    const int hk = p.kv.kv_heads;
    const int total = p.heads + 2 * hk;
    const int h0 = group * lanes * per + sub;
    for (int i = 0; i < per; i++) {
        const int h = h0 + i * lanes;
        if (h >= total) break;
        const char* src;
        char* dst;
        bool rotate = turned;
        if (h < p.heads) {
            src = p.q + t * p.q_tok + h * p.q_head;
            dst = p.q_out + t * p.o_tok + h * p.o_head;
        } else {
            if (row < 0) continue;
            const int g = h - p.heads;
            if (g < hk) {
                src = p.kn + t * p.k_tok + g * p.k_head;
                dst = const_cast<char*>(p.kv.k) + row_offset(row, p.kv.shift, p.kv.k_page, p.kv.k_row) +
                      g * p.kv.k_head;
            } else {
                src = p.vn + t * p.v_tok + (g - hk) * p.v_head;
                dst = const_cast<char*>(p.kv.v) + row_offset(row, p.kv.shift, p.kv.v_page, p.kv.v_row) +
                      (g - hk) * p.kv.v_head;
                rotate = false;
            }
        }
        V8 a = *(const V8*)(src + 2 * ea), b = *(const V8*)(src + 2 * eb);
        if (rotate) {
            if (p.half_layout) {
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const float x = a[j], y = b[j];
                    a[j] = (typename E::T)(x * c[j] - y * sn[j]);
                    b[j] = (typename E::T)(y * c[j] + x * sn[j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const float x = j < 4 ? a[2 * j] : b[2 * j - 8], y = j < 4 ? a[2 * j + 1] : b[2 * j - 7];
                    const typename E::T r = (typename E::T)(x * c[j] - y * sn[j]);
                    const typename E::T w = (typename E::T)(y * c[j] + x * sn[j]);
                    if (j < 4) {
                        a[2 * j] = r, a[2 * j + 1] = w;
                    } else {
                        b[2 * j - 8] = r, b[2 * j - 7] = w;
                    }
                }
            }
        }
        *(V8*)(dst + 2 * ea) = a;
        *(V8*)(dst + 2 * eb) = b;
    }
    if (group == 0 && row >= 0) {
        for (int g = lane; g < hk; g += 64) {
            const int64_t at = stat_index(p.kv, row, g);
            if (p.kv.weight) p.kv.weight[at] = 0.f;
            if (p.kv.position) p.kv.position[at] = pos;
        }
    }
}

// The same element by element, for rows that do not lie on 16 bytes and rotated
// parts that are no multiple of 16.  One wave for a token; an element's
// partner is read with it, so q_out may be q only if one lane does both: a
// lane takes whole pairs.  Its narrow accesses bound it: 19,432 tokens with 72 of 128 dimensions turned 274 us, 1.8 TB/s.
template <class E>
__global__ __launch_bounds__(64) void k_append_any(AppendArgs p) {
    using T = typename E::T;
    const int t = blockIdx.x, lane = threadIdx.x;
    const int seq = find_seq(p.kv, t);
    const Seq s = seq_of(p.kv, seq);
    const int slot = s.len - s.n + (t - s.q0);
    const bool ours = t >= s.q0 && t < s.q0 + s.n;
    const int row = ours && slot >= 0 ? pool_row(p.kv, seq, slot) : -1;
    const int pos = p.positions[t];
    const bool known = (unsigned)pos < (unsigned)p.rope_rows;
    const float* tab = p.rope + (int64_t)(known ? pos : 0) * p.rot;
    const int hk = p.kv.kv_heads, half = p.rot >> 1, pairs = p.dim >> 1;
    for (int i = lane; i < (p.heads + 2 * hk) * pairs; i += 64) {
        const int h = i / pairs, u = i - h * pairs;
        const T* src;
        T* dst;
        bool rotate = u < half;
        if (h < p.heads) {
            src = (const T*)(p.q + t * p.q_tok + h * p.q_head);
            dst = (T*)(p.q_out + t * p.o_tok + h * p.o_head);
        } else {
            if (row < 0) continue;
            const int g = h - p.heads;
            if (g < hk) {
                src = (const T*)(p.kn + t * p.k_tok + g * p.k_head);
                dst = (T*)(const_cast<char*>(p.kv.k) + row_offset(row, p.kv.shift, p.kv.k_page, p.kv.k_row) +
                           g * p.kv.k_head);
            } else {
                src = (const T*)(p.vn + t * p.v_tok + (g - hk) * p.v_head);
                dst = (T*)(const_cast<char*>(p.kv.v) + row_offset(row, p.kv.shift, p.kv.v_page, p.kv.v_row) +
                           (g - hk) * p.kv.v_head);
                rotate = false;
            }
        }
        const bool half_pair = u < half && p.half_layout;
        const int ea = half_pair ? u : 2 * u, eb = half_pair ? u + half : 2 * u + 1;
        const float x = (float)src[ea], y = (float)src[eb];
        if (rotate) {
            const float c = known ? tab[u] : __builtin_nanf(""), sn = known ? tab[half + u] : __builtin_nanf("");
            dst[ea] = (T)(x * c - y * sn);
            dst[eb] = (T)(y * c + x * sn);
        } else {
            dst[ea] = src[ea];
            dst[eb] = src[eb];
        }
    }
    if (row >= 0) {
        for (int g = lane; g < hk; g += 64) {
            const int64_t at = stat_index(p.kv, row, g);
            if (p.kv.weight) p.kv.weight[at] = 0.f;
            if (p.kv.position) p.kv.position[at] = pos;
        }
    }
}

// Positions with several axes: a pair turns by its axis' position.  The row of the table that it takes its cosine and sine
// from is another for each axis; an axis whose position is outside the table makes NaN of its own pairs alone.
__device__ inline int axis_of(const AxesArgs& x, int pair) { return x.of_pair[pair >> 4] >> 2 * (pair & 15) & 3; }

// As in k_append_wide, for rotated parts of any size from 16 on and rows at any address: a lane has eight elements of the part's first half
// and eight of its second (eight pairs, or twice four where pairs are neighbours), the last ones
// again from the end, so that two lanes may turn the same pair (both have read it before either writes: they are lanes of one
// wave), and a 16-byte access may lie across two lines.  The rest of a head is copied in the same way.
// Bytes bound it: 19,432 tokens of prompts with images (489 MB) take 96 us and 32,001 of a video (three quarters of a head turned, 801 MB)
// 167, what a copy reaches; 203 tokens 5.4.
struct Units {
    int turned, all;  // of a head: units of eight pairs, and with those that are copied
};
template <class E>
__global__ __launch_bounds__(256) void k_axes_wide(AppendArgs p, AxesArgs x, Units units, int groups, int per) {
    using T = typename E::T;
    typedef T V8 __attribute__((ext_vector_type(8), aligned(2)));
    typedef T V2 __attribute__((ext_vector_type(2), aligned(2)));
    typedef float F4 __attribute__((ext_vector_type(4), aligned(4)));
    const int wave = __builtin_amdgcn_readfirstlane((int)((blockIdx.x * 256 + threadIdx.x) >> 6));
    const int t = wave / groups, group = wave - t * groups;
    if (t >= p.kv.tokens) return;
    const int lane = threadIdx.x & 63;
    const int seq = find_seq(p.kv, t);
    const Seq s = seq_of(p.kv, seq);
    const int slot = s.len - s.n + (t - s.q0);
    const bool ours = t >= s.q0 && t < s.q0 + s.n;
    const int row = ours && slot >= 0 ? pool_row(p.kv, seq, slot) : -1;

    const int lanes = 64 / units.all;  // heads that the wave takes at a time
    const int sub = lane / units.all, unit = lane - sub * units.all;
    const bool turned = unit < units.turned;
    // elements [ea, ea + 8) and [eb, eb + 8): of the two halves of the rotated part (neighbours are not torn apart), or of the rest
    const int half = p.rot >> 1, cut = p.half_layout ? half : (half + 1) & ~1;
    const int copied = unit - units.turned, rest_half = (units.all - units.turned) * 8;
    const int ea = turned ? min(unit * 8, cut - 8) : min(p.rot + copied * 8, p.dim - 8);
    const int eb = turned ? min(cut + unit * 8, p.rot - 8) : min(p.rot + rest_half + copied * 8, p.dim - 8);
    // and their pairs: eight from pa on, or four from pa and four from pb
    const int pa = p.half_layout ? ea : ea >> 1, pb = p.half_layout ? ea + 4 : eb >> 1;
    const int few = p.dim - p.rot < 8 ? p.dim - p.rot : 0;  // elements behind the pairs, where no eight are
    float c[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; i++) c[i] = 1.f, sn[i] = 0.f;
    if (turned) {
        auto table = [&](int axis) {
            const int pos = p.positions[t * x.token + axis * x.axis];
            return (unsigned)pos < (unsigned)p.rope_rows ? p.rope + (int64_t)pos * p.rot : nullptr;
        };
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const int p0 = i ? pb : pa;
            const uint64_t words = (uint64_t)x.of_pair[min(7, (p0 >> 4) + 1)] << 32 | x.of_pair[p0 >> 4];
            const uint32_t mine = (uint32_t)(words >> 2 * (p0 & 15)) & 0xff;
            if (mine == (mine & 3) * 0x55u) {  // one axis for all four
                const float* tab = table(mine & 3);
                const F4 a = tab ? *(const F4*)(tab + p0) : F4(__builtin_nanf("")), b = tab ? *(const F4*)(tab + half + p0) : F4(__builtin_nanf(""));
#pragma unroll
                for (int j = 0; j < 4; j++) c[i + j] = a[j], sn[i + j] = b[j];
            } else {
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const float* tab = table(mine >> 2 * j & 3);
                    c[i + j] = tab ? tab[p0 + j] : __builtin_nanf("");
                    sn[i + j] = tab ? tab[half + p0 + j] : __builtin_nanf("");
                }
            }
        }
    }
    const int hk = p.kv.kv_heads;
    const int total = p.heads + 2 * hk;
    const int h0 = group * lanes * per + sub;
    for (int i = 0; i < per && sub < lanes; i++) {
        const int h = h0 + i * lanes;
        if (h >= total) break;
        const char* src;
        char* dst;
        bool rotate = turned;
        if (h < p.heads) {
            src = p.q + t * p.q_tok + h * p.q_head;
            dst = p.q_out + t * p.o_tok + h * p.o_head;
        } else {
            if (row < 0) continue;
            const int g = h - p.heads;
            if (g < hk) {
                src = p.kn + t * p.k_tok + g * p.k_head;
                dst = const_cast<char*>(p.kv.k) + row_offset(row, p.kv.shift, p.kv.k_page, p.kv.k_row) + g * p.kv.k_head;
            } else {
                src = p.vn + t * p.v_tok + (g - hk) * p.v_head;
                dst = const_cast<char*>(p.kv.v) + row_offset(row, p.kv.shift, p.kv.v_page, p.kv.v_row) + (g - hk) * p.kv.v_head;
                rotate = false;
            }
        }
        if (few && !turned) {
            for (int j = p.rot; j < p.dim; j += 2) *(V2*)(dst + 2 * j) = *(const V2*)(src + 2 * j);
            continue;
        }
        V8 a = *(const V8*)(src + 2 * ea), b = *(const V8*)(src + 2 * eb);
        if (rotate) {
            if (p.half_layout) {
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const float y = a[j], z = b[j];
                    a[j] = (T)(y * c[j] - z * sn[j]);
                    b[j] = (T)(z * c[j] + y * sn[j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    V8& v = j < 4 ? a : b;
                    const float y = v[2 * (j & 3)], z = v[2 * (j & 3) + 1];
                    v[2 * (j & 3)] = (T)(y * c[j] - z * sn[j]);
                    v[2 * (j & 3) + 1] = (T)(z * c[j] + y * sn[j]);
                }
            }
        }
        *(V8*)(dst + 2 * ea) = a;
        *(V8*)(dst + 2 * eb) = b;
    }
    if (group == 0 && row >= 0) {
        const int kept = x.kept ? x.kept[t] : p.positions[t * x.token];
        for (int g = lane; g < hk; g += 64) {
            const int64_t at = stat_index(p.kv, row, g);
            if (p.kv.weight) p.kv.weight[at] = 0.f;
            if (p.kv.position) p.kv.position[at] = kept;
        }
    }
}

// The same pair by pair, for rotated parts of fewer than eight pairs.
template <class E>
__global__ __launch_bounds__(64) void k_axes_any(AppendArgs p, AxesArgs x) {
    using T = typename E::T;
    const int t = blockIdx.x, lane = threadIdx.x;
    const int seq = find_seq(p.kv, t);
    const Seq s = seq_of(p.kv, seq);
    const int slot = s.len - s.n + (t - s.q0);
    const bool ours = t >= s.q0 && t < s.q0 + s.n;
    const int row = ours && slot >= 0 ? pool_row(p.kv, seq, slot) : -1;
    const int hk = p.kv.kv_heads, half = p.rot >> 1, pairs = p.dim >> 1;
    for (int i = lane; i < (p.heads + 2 * hk) * pairs; i += 64) {
        const int h = i / pairs, u = i - h * pairs;
        const T* src;
        T* dst;
        bool rotate = u < half;
        if (h < p.heads) {
            src = (const T*)(p.q + t * p.q_tok + h * p.q_head);
            dst = (T*)(p.q_out + t * p.o_tok + h * p.o_head);
        } else {
            if (row < 0) continue;
            const int g = h - p.heads;
            if (g < hk) {
                src = (const T*)(p.kn + t * p.k_tok + g * p.k_head);
                dst = (T*)(const_cast<char*>(p.kv.k) + row_offset(row, p.kv.shift, p.kv.k_page, p.kv.k_row) +
                           g * p.kv.k_head);
            } else {
                src = (const T*)(p.vn + t * p.v_tok + (g - hk) * p.v_head);
                dst = (T*)(const_cast<char*>(p.kv.v) + row_offset(row, p.kv.shift, p.kv.v_page, p.kv.v_row) +
                           (g - hk) * p.kv.v_head);
                rotate = false;
            }
        }
        const bool half_pair = u < half && p.half_layout;
        const int ea = half_pair ? u : 2 * u, eb = half_pair ? u + half : 2 * u + 1;
        const T a = src[ea], b = src[eb];
        if (rotate) {
            const int pos = p.positions[t * x.token + axis_of(x, u) * x.axis];
            const bool known = (unsigned)pos < (unsigned)p.rope_rows;
            const float* tab = p.rope + (int64_t)(known ? pos : 0) * p.rot + u;
            const float c = known ? tab[0] : __builtin_nanf(""), sn = known ? tab[half] : __builtin_nanf("");
            dst[ea] = (T)((float)a * c - (float)b * sn);
            dst[eb] = (T)((float)b * c + (float)a * sn);
        } else {
            dst[ea] = a;
            dst[eb] = b;
        }
    }
    if (row >= 0) {
        const int kept = x.kept ? x.kept[t] : p.positions[t * x.token];
        for (int g = lane; g < hk; g += 64) {
            const int64_t at = stat_index(p.kv, row, g);
            if (p.kv.weight) p.kv.weight[at] = 0.f;
            if (p.kv.position) p.kv.position[at] = kept;
        }
    }
}

// How the wide kernel's work is dealt out.
struct Wide {
    int units, groups, per;
    int64_t blocks;
};

Wide wide_grid(const AppendArgs& a, int units) {
    Wide w;
    w.units = units;
    const int lanes = 64 / w.units, steps = (a.heads + 2 * a.kv.kv_heads + lanes - 1) / lanes;
    // Heads that a lane walks over: all of a token's once 8,192 waves are there
    // without splitting a token, fewer for fewer tokens.
    const int64_t per = ((int64_t)a.kv.tokens * steps + 8191) / 8192;
    w.per = per < 1 ? 1 : per > steps ? steps : (int)per;
    w.groups = (steps + w.per - 1) / w.per;
    w.blocks = ((int64_t)a.kv.tokens * w.groups + 3) / 4;
    return w;
}

}  // namespace

int64_t append_threads(const AppendArgs& a, bool wide) { return wide ? wide_grid(a, a.dim / 16).blocks * 256 : (int64_t)a.kv.tokens * 64; }

hipError_t launch_append(const AppendArgs& a, int32_t dtype, bool wide, hipStream_t s) {
    if (wide) {
        const Wide w = wide_grid(a, a.dim / 16);
        const dim3 grid((unsigned)w.blocks);
        return run(dtype == SVF_KV_BF16 ? k_append_wide<BF16> : k_append_wide<F16>, grid, 256, s, a, w.units, w.groups, w.per);
    }
    return run(dtype == SVF_KV_BF16 ? k_append_any<BF16> : k_append_any<F16>, dim3(a.kv.tokens), 64, s, a);
}

namespace {

bool axes_wide(const AppendArgs& a) { return a.rot >= 16; }

Units axes_units(const AppendArgs& a) {
    const int half = a.rot / 2, turned = ((a.half_layout ? half : (half + 1) & ~1) + 7) / 8;
    return {turned, turned + (a.dim - a.rot + 15) / 16};
}

}  // namespace

int64_t append_axes_threads(const AppendArgs& a) {
    return axes_wide(a) ? wide_grid(a, axes_units(a).all).blocks * 256 : (int64_t)a.kv.tokens * 64;
}

hipError_t launch_append_axes(const AppendArgs& a, const AxesArgs& x, int32_t dtype, hipStream_t s) {
    if (axes_wide(a)) {
        const Units units = axes_units(a);
        const Wide w = wide_grid(a, units.all);
        return run(dtype == SVF_KV_BF16 ? k_axes_wide<BF16> : k_axes_wide<F16>, dim3((unsigned)w.blocks), 256, s, a, x, units, w.groups, w.per);
    }
    return run(dtype == SVF_KV_BF16 ? k_axes_any<BF16> : k_axes_any<F16>, dim3(a.kv.tokens), 64, s, a, x);
}

}  // namespace svfk
