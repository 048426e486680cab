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

// How the wide kernel's work is dealt out.
struct Wide {
    int units, groups, per;
    int64_t blocks;
};

Wide wide_grid(const AppendArgs& a) {
    Wide w;
    w.units = a.dim / 16;
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

int64_t append_threads(const AppendArgs& a, bool wide) { return wide ? wide_grid(a).blocks * 256 : (int64_t)a.kv.tokens * 64; }

hipError_t launch_append(const AppendArgs& a, int32_t dtype, bool wide, hipStream_t s) {
    if (wide) {
        const Wide w = wide_grid(a);
        const dim3 grid((unsigned)w.blocks);
        return run(dtype == SVF_KV_BF16 ? k_append_wide<BF16> : k_append_wide<F16>, grid, 256, s, a, w.units, w.groups, w.per);
    }
    return run(dtype == SVF_KV_BF16 ? k_append_any<BF16> : k_append_any<F16>, dim3(a.kv.tokens), 64, s, a);
}

}  // namespace svfk
