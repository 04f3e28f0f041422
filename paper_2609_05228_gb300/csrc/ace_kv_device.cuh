// ace_kv_device.cuh — device helpers of the speculative decode step: e4m3 rows, the division of
// the attention's work over CTAs, and where partial results lie.
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
// lengths load every SM alike; a unit cut by a boundary leaves partial results, which a kernel after this one joins.
// START places of the line come before each unit's tiles: the time of as many tiles that its start and end cost.
template <int ROWS, int KEYS, int START>
struct Work {
    __device__ static int tiles(const Request& r) { return r.n > 0 ? (r.len + r.n + KEYS - 1) / KEYS : 0; }
    __device__ static int blocks(const AttnArgs& a, const Request& r) { return (r.n * a.group + ROWS - 1) / ROWS; }
    __device__ static long long of(const AttnArgs& a, const Request& r) {
        return r.n > 0 ? (long long)(START + tiles(r)) * blocks(a, r) * a.kv_heads : 0;
    }
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

// Place of dimension d of row r in partial result `slot` (ROWS rows each): by rows, or (BY_DIMS) by 4 dimensions and then
// rows, for kernels in which a thread holds a row.
template <bool BY_DIMS>
__device__ __forceinline__ long long part_place(int rows, int D, long long slot, int r, int d) {
    return BY_DIMS ? ((slot * (D / 4) + d / 4) * rows + r) * 4 + d % 4 : (slot * rows + r) * D + d;
}

// By one thread: the CTA's note of the cut unit that begins in it, for the joining kernel (none, until there is one).
__device__ __forceinline__ void note_none(const AttnArgs& a) { a.ws.unit[blockIdx.x].rows = 0; }
__device__ __forceinline__ void note_unit(const AttnArgs& a, const Segment& s) {
    if (s.part >= 0 && s.first == (int)blockIdx.x) a.ws.unit[blockIdx.x] = s;
}

}  // namespace ace
