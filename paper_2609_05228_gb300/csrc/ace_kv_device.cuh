// ace_kv_device.cuh — device helpers of the speculative decode step: e4m3 rows, the division of
// the attention's work over CTAs, and the joining of partial results.
#pragma once

#include <cuda_fp16.h>

#include "ace_device.cuh"
#include "ace_kv.h"

namespace ace {

// ---------------------------------------------------------------- e4m3 rows

// Scale byte e + 127 of a row whose largest finite |x| is amax: e is the smallest integer >= -126 with
// amax <= 448 * 2^e. amax = f * 2^x with f in [1, 2) and 448 = 1.75 * 2^8, so e = x - 8, one more where f > 1.75.
__device__ __forceinline__ int e4m3_scale_byte(float amax) {
    const uint32_t b = __float_as_uint(amax);
    const int e127 = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e127 < 1 ? 1 : e127;
}

__device__ __forceinline__ float pow2_of_byte(int byte) { return __uint_as_float((uint32_t)byte << 23); }
__device__ __forceinline__ float pow2_of_minus_byte(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }

// Two floats to e4m3 codes, lo in the low byte; infinities must have been made NaN.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// Two codes to the halves they stand for (exact: 4 significant bits).
__device__ __forceinline__ uint32_t f16x2_of_e4m3x2(uint32_t codes) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)codes));
    return r;
}

__device__ __forceinline__ void e4m3x8_to_float(uint2 c, float (&f)[8]) {
    const uint32_t w[4] = {c.x & 0xffffu, c.x >> 16, c.y & 0xffffu, c.y >> 16};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t h = f16x2_of_e4m3x2(w[i]);
        const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h));
        f[2 * i] = v.x;
        f[2 * i + 1] = v.y;
    }
}

__device__ __forceinline__ void store8f(float* p, const float (&f)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

__device__ __forceinline__ float finite_or_nan(float x) {
    return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? __uint_as_float(0x7fffffffu) : x;
}

// ---------------------------------------------------------------- requests and their share of the work

struct Request {
    int len, n, node0;
};

// Shape of request b; what points outside its array is cut and noted.
__device__ __forceinline__ Request request_of(const AttnArgs& a, int b) {
    int len = a.lens[b], o0 = a.node_offsets[b], o1 = a.node_offsets[b + 1];
    const long long cap = (long long)a.max_pages * a.page_size;
    bool bad = false;
    if (o0 < 0 || o1 < o0 || o1 > a.T) o0 = o1 = 0, bad = true;
    int n = o1 - o0;
    if (n > a.max_nodes) n = 0, bad = true;
    if (len < 0 || (long long)len + n > cap) n = 0, len = 0, bad = true;
    if (bad) atomicOr(a.err, kErrIndex);
    return Request{len, n, o0};
}

// The work is a line of key tiles: request by request, in it unit by unit (head, then row block), in it tile by
// tile. CTA c of g takes the tiles [c W / g, (c + 1) W / g), whatever units they belong to, so ragged
// lengths load every SM alike; a unit cut by a boundary leaves partial results, joined by the CTA that finishes last.
// START places of the line come before each unit's tiles: the time of as many tiles that its start and end cost.
template <int ROWS, int KEYS, int START>
struct Work {
    __device__ static int tiles(const Request& r) { return r.n > 0 ? (r.len + r.n + KEYS - 1) / KEYS : 0; }
    __device__ static int blocks(const AttnArgs& a, const Request& r) { return (r.n * a.group + ROWS - 1) / ROWS; }
    __device__ static long long of(const AttnArgs& a, const Request& r) {
        return r.n > 0 ? (long long)(START + tiles(r)) * blocks(a, r) * a.kv_heads : 0;
    }
};

struct Segment {
    int b, head, row0, rows;        // request, kv head, first row of the unit (node * G + g) and its rows
    int node0, len, n;              // the request
    int tile0, tile1;               // key tiles of this CTA
    int part;                       // partial result slot, -1: the whole unit is here
    int first, last;                // CTAs that share the unit
};

struct Cursor {
    long long W, w, w_end, base;    // all work, this CTA's rest [w, w_end), work before request b
    int b, ctas;
};

__device__ __forceinline__ long long share_start(long long W, int c, int g) { return (long long)c * W / g; }
__device__ __forceinline__ int share_of(long long W, long long w, int g) { return (int)(((w + 1) * g - 1) / W); }

// By one converged warp: the CTA's share. False: nothing to do.
template <int ROWS, int KEYS, int START>
__device__ bool cursor_init(const AttnArgs& a, int cta, int max_ctas, Cursor& c) {
    const int lane = threadIdx.x & 31;
    long long total = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32)
        if (b0 + lane < a.B) total += Work<ROWS, KEYS, START>::of(a, request_of(a, b0 + lane));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    c.W = total;
    c.ctas = (int)(total < max_ctas ? total : max_ctas);
    if (cta >= c.ctas) return false;
    c.w = share_start(total, cta, c.ctas);
    c.w_end = share_start(total, cta + 1, c.ctas);
    long long base = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
        const long long mine = b0 + lane < a.B ? Work<ROWS, KEYS, START>::of(a, request_of(a, b0 + lane)) : 0;
        long long sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long up = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += up;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, base + sum > c.w);
        if (hit) {
            const int l = __ffs(hit) - 1;
            c.b = b0 + l;
            c.base = base + __shfl_sync(0xffffffffu, sum - mine, l);
            return true;
        }
        base += __shfl_sync(0xffffffffu, sum, 31);
    }
    return false;
}

// The next segment of the share. False: the share is done.
template <int ROWS, int KEYS, int START>
__device__ bool cursor_next(const AttnArgs& a, int cta, Cursor& c, Segment& s) {
    if (c.w >= c.w_end) return false;
    Request r = request_of(a, c.b);
    long long work = Work<ROWS, KEYS, START>::of(a, r);
    while (c.w >= c.base + work) {
        c.base += work;
        r = request_of(a, ++c.b);
        work = Work<ROWS, KEYS, START>::of(a, r);
    }
    const int tiles = Work<ROWS, KEYS, START>::tiles(r), blocks = Work<ROWS, KEYS, START>::blocks(a, r);
    const long long unit = (c.w - c.base) / (START + tiles);
    const long long u0 = c.base + unit * (START + tiles) + START;      // place of its first tile
    if (c.w < u0) c.w = u0;
    if (c.w >= c.w_end) return false;
    s.b = c.b;
    s.head = (int)(unit / blocks);
    s.row0 = (int)(unit % blocks) * ROWS;
    s.rows = min(ROWS, r.n * a.group - s.row0);
    s.node0 = r.node0;
    s.len = r.len;
    s.n = r.n;
    s.tile0 = (int)(c.w - u0);
    const long long left = c.w_end - c.w;
    s.tile1 = left < tiles - s.tile0 ? s.tile0 + (int)left : tiles;
    if (s.tile1 - s.tile0 == tiles) {
        s.part = -1;
        s.first = s.last = cta;
    } else {
        s.part = 2 * cta + (u0 < share_start(c.W, cta, c.ctas) ? 0 : 1);
        s.first = share_of(c.W, u0, c.ctas);
        s.last = share_of(c.W, u0 + tiles - 1, c.ctas);
    }
    c.w += s.tile1 - s.tile0;
    return true;
}

// Partial result slot of CTA c in a unit whose first CTA is `first`.
__device__ __forceinline__ int part_slot(int c, int first) { return 2 * c + (c == first ? 1 : 0); }

// Page of position tile `pos / page_size` of request b, or -1 (noted) where the table names none of the pool's.
__device__ __forceinline__ int page_of(const AttnArgs& a, int b, int pos) {
    const int page = a.page_table[(long long)b * a.max_pages + (pos >> a.page_shift)];
    if (page < 0 || page >= a.n_pages) {
        atomicOr(a.err, kErrIndex);
        return -1;
    }
    return page;
}

// Word `w` (64 nodes) of the nodes that node i of the request sees, cut to its n nodes.
__device__ __forceinline__ unsigned long long sees_word(const AttnArgs& a, int node0, int n, int i, int w) {
    if (w * 64 >= n || w < 0) return 0ull;
    unsigned long long m;
    if (a.mask) {
        m = w < a.words ? a.mask[(long long)(node0 + i) * a.words + w] : 0ull;
    } else {
        const int k = i - w * 64;       // bits 0 .. k
        m = k < 0 ? 0ull : k >= 63 ? ~0ull : (2ull << k) - 1ull;
    }
    const int left = n - w * 64;
    return left >= 64 ? m : m & ((1ull << left) - 1ull);
}

// Place of dimension d of row r in partial result `slot`: by rows, or (BY_DIMS) by 4 dimensions and then rows, for kernels
// in which a thread holds a row.
template <int ROWS, bool BY_DIMS>
__device__ __forceinline__ long long part_place(int D, long long slot, int r, int d) {
    return BY_DIMS ? ((slot * (D / 4) + d / 4) * ROWS + r) * 4 + d % 4 : (slot * ROWS + r) * D + d;
}

// 4 dimensions of an output row.
template <typename T>
__device__ __forceinline__ void store_joined(const AttnArgs& a, long long at, int d, float4 o, float inv) {
    T* out = static_cast<T*>(a.out) + at * a.head_dim + d;
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(out) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    } else {
        __nv_bfloat162 lo = __floats2bfloat162_rn(o.x * inv, o.y * inv), hi = __floats2bfloat162_rn(o.z * inv, o.w * inv);
        uint2 w;
        w.x = *reinterpret_cast<uint32_t*>(&lo);
        w.y = *reinterpret_cast<uint32_t*>(&hi);
        *reinterpret_cast<uint2*>(out) = w;
    }
}

// A row's partial results over parts c0 .. c0 + PARTS - 1 of a unit, 4 dimensions at each of ITEMS places, onto what came
// before: with the reference that they turn up with, rescaled as it grows.
template <int ROWS, bool BY_DIMS, int ITEMS, int PARTS>
__device__ __forceinline__ void join_parts(const AttnArgs& a, const Segment& s, int c0, int r, int d, float& M, float& L, float4 (&o)[ITEMS]) {
    float2 ml[PARTS];
    float4 v[ITEMS][PARTS];
#pragma unroll
    for (int j = 0; j < PARTS; ++j) {
        const int c = c0 + j;
        ml[j] = make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) v[k][j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c <= s.last) {
            const long long slot = part_slot(c, s.first);
            ml[j] = __ldcg(&a.ws.part_ml[slot * ROWS + r]);
#pragma unroll
            for (int k = 0; k < ITEMS; ++k)
                v[k][j] = __ldcg(reinterpret_cast<const float4*>(a.ws.part_o + part_place<ROWS, BY_DIMS>(a.head_dim, slot, r, d + 16 * k)));
        }
    }
    float top = M;
#pragma unroll
    for (int j = 0; j < PARTS; ++j) top = fmaxf(top, ml[j].x);
    const float ref = top == -INFINITY ? 0.f : top, back = exp2f(M - ref);
    M = top;
    L *= back;
    float f[PARTS];
#pragma unroll
    for (int j = 0; j < PARTS; ++j) {
        f[j] = exp2f(ml[j].x - ref);
        L = fmaf(ml[j].y, f[j], L);
    }
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        o[k].x *= back;
        o[k].y *= back;
        o[k].z *= back;
        o[k].w *= back;
#pragma unroll
        for (int j = 0; j < PARTS; ++j) {
            o[k].x = fmaf(v[k][j].x, f[j], o[k].x);
            o[k].y = fmaf(v[k][j].y, f[j], o[k].y);
            o[k].z = fmaf(v[k][j].z, f[j], o[k].z);
            o[k].w = fmaf(v[k][j].w, f[j], o[k].w);
        }
    }
}

// Joins a unit's partial results: row r of the unit from the slots of CTAs first .. last, in that order. Every thread of a
// CTA calls it; all partial results must be visible. What it costs is rounds of loads, each of which takes more than a
// microsecond. Few rows (which have many parts: a long context): 8 parts at a time, 4 dimensions a thread. Many rows (D
// given): two parts at a time, a warp takes 8 rows whole, so that it reads lines and writes sectors.
template <typename T, int ROWS, int D, bool BY_DIMS = false>
__device__ __forceinline__ void join_unit(const AttnArgs& a, const Segment& s, int tid, int threads) {
    const int quads = a.head_dim / 4;
    if constexpr (ROWS > 16) {
        if (s.rows * quads >= 2 * threads) {
#pragma unroll 1
            for (int r0 = tid / 32 * 8; r0 < s.rows; r0 += threads / 4) {
                const int r = min(r0 + tid % 8, s.rows - 1), d = tid / 8 % 4 * 4;
                float M = -INFINITY, L = 0.f;
                float4 o[D / 16] = {};
#pragma unroll 1
                for (int c = s.first; c <= s.last; c += 2) join_parts<ROWS, BY_DIMS, D / 16, 2>(a, s, c, r, d, M, L, o);
                const float inv = L == 0.f ? 0.f : 1.f / L;
                const int row = s.row0 + r, node = s.node0 + row / a.group, hq = s.head * a.group + row % a.group;
                const long long at = (long long)node * a.n_heads + hq;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) store_joined<T>(a, at, d + 16 * k, o[k], inv);
                if (d == 0 && a.lse) a.lse[at] = (M + log2f(L)) * 0.69314718055994530942f;
            }
            return;
        }
    }
#pragma unroll 1
    for (int i = tid; i < s.rows * quads; i += threads) {
        const int r = i / quads, d = (i - r * quads) * 4;
        float M = -INFINITY, L = 0.f;
        float4 o[1] = {};
#pragma unroll 1
        for (int c = s.first; c <= s.last; c += 8) join_parts<ROWS, BY_DIMS, 1, 8>(a, s, c, r, d, M, L, o);
        const float inv = L == 0.f ? 0.f : 1.f / L;
        const int row = s.row0 + r, node = s.node0 + row / a.group, hq = s.head * a.group + row % a.group;
        const long long at = (long long)node * a.n_heads + hq;
        store_joined<T>(a, at, d, o[0], inv);
        if (d == 0 && a.lse) a.lse[at] = (M + log2f(L)) * 0.69314718055994530942f;
    }
}

// One thread, after all of the CTA's partial results are visible on the device: true in the last CTA of the unit.
__device__ __forceinline__ bool last_of_unit(const AttnArgs& a, const Segment& s) {
    const int want = s.last - s.first;
    if (atomicAdd(a.ws.ticket + s.first, 1) != want) return false;
    a.ws.ticket[s.first] = 0;           // for the next call
    return true;
}

}  // namespace ace
