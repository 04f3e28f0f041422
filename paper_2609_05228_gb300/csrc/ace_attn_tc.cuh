// ace_attn_tc.cuh — what the tensor-core attention kernels share: the roles that schedule, load and stage scales,
// and the wrappers of their instructions.
#pragma once

#include "ace_kv_device.cuh"
#include "ace_tc.cuh"

namespace ace {
namespace {

constexpr int kTcKeys = 128, kTcThreads = 512, kSegRing = 4, kAuxRing = 4;
// A row's reference is its maximum less kPUp when it is set, and moves once the maximum is kLazy above that
// (base 2): weights are at most 2^(kLazy + kPUp), which fp16 holds, and normal in fp16 down to 2^-(14 + kPUp) of the largest.
constexpr int kLazy = 8, kPUp = 6;
constexpr int kVUp = 6;                 // fp16 rows of V are code * 2^(e - eref + kVUp): at most 448 * 2^6, eref >= e
constexpr int kConvThreads = 128;
// Every wait is on an mbarrier and bounded. A wait names a phase by its parity, so each waiter takes part in every phase
// of its barriers, or what it waits for in between implies the phases that it leaves out.

struct TcAttnArgs {
    AttnArgs a;
    CUtensorMap k, v;
    int box_rows;                       // positions of a page in one box
};

struct Ring {
    int i = 0;
    uint32_t phase = 0;
    template <int N>
    __device__ __forceinline__ void next() {
        if (++i == N) i = 0, phase ^= 1u;
    }
};

struct TcSegment {
    Segment s;
    int go, pad;
    unsigned long long bad[kMaxNodes / 64];     // nodes whose V row holds what is not finite
    unsigned long long far[kMaxNodes / 64];     // fp8: nodes whose V is left out of the products for its scale (Reference)
};

// Barriers and hand-overs of a CTA.
struct TcShared {
    uint64_t k_full[6], k_empty[6], v_full[6], v_empty[6], v_ready[6];
    uint64_t s_full[4], p_ready[4], o_done[4], q_full, q_free, drain[2];
    uint64_t seg_full[kSegRing], seg_empty[kSegRing], aux_full[kAuxRing], aux_empty[kAuxRing];
    uint32_t tmem;
    int abort_flag, pad[2];
    TcSegment seg[kSegRing];
    int eref[kAuxRing];
};

// Shared-memory descriptors by halves: the low word holds the address, to which a K step adds, and the leading byte
// offset; the high one the stride byte offset, the version and the swizzle (2: 128 bytes, 4: 64 bytes).
constexpr uint32_t desc_hi(uint32_t sbo, uint32_t swizzle) { return (sbo >> 4) | 1u << 14 | swizzle << 29; }
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lbo) { return addr >> 4 | (lbo >> 4) << 16; }
constexpr uint32_t kRows128 = desc_hi(1024, 2);     // K-major rows of 128 bytes, or V as stored (8 K indices to the next group)
constexpr uint32_t kRows64 = desc_hi(512, 4);       // K-major rows of 64 bytes
constexpr uint32_t kVBlock = 16384;                 // V: to the next 64 dimensions

// Instruction descriptor: fp32 accumulator; type codes of A and B (kind::f16: 0 fp16, 1 bf16; kind::f8f6f4: 0 e4m3).
__host__ __device__ constexpr uint32_t idesc_of(int type, int M, int N, bool b_mn) {
    return (1u << 4) | ((uint32_t)type << 7) | ((uint32_t)type << 10) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

template <bool F8>
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, bool acc) {
    if constexpr (F8)
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\t"
            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %4, p;\n\t}" ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc),
            "r"((uint32_t)acc));
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n\t}" ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc),
            "r"((uint32_t)acc));
}

// A from TMEM.
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t hi, uint32_t idesc, bool acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 b, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}" ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(hi), "r"(idesc),
        "r"((uint32_t)acc));
}

#define ACE_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define ACE_V8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
        "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : ACE_R8(r, 0), ACE_R8(r, 8), ACE_R8(r, 16), ACE_R8(r, 24)
        : "r"(taddr));
}

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
        "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::ACE_V8(r, 0),
        ACE_V8(r, 8), ACE_V8(r, 16), ACE_V8(r, 24), "r"(taddr)
        : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::ACE_V8(r, 0),
        ACE_V8(r, 8), "r"(taddr)
        : "memory");
}

__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}

// (a & b) | c
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}

__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two fp32 values in one operation each.
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// Two weights (>= 0, or NaN) as two bf16 terms each: their upper 16 bits, and what is left of them, rounded: 2^-17 of a weight at most.
__device__ __forceinline__ void two_terms(float a, float b, uint32_t& upper, uint32_t& lower) {
    const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
    upper = __byte_perm(x, y, 0x7632);
    float c, d;
    unpair(add2(pair(a, b), pair(__uint_as_float(x & 0xffff0000u | 0x80000000u), __uint_as_float(y & 0xffff0000u | 0x80000000u))), c, d);
    const __nv_bfloat162 z = __floats2bfloat162_rn(c, d);
    lower = *reinterpret_cast<const uint32_t*>(&z);
}

// Which of the 32 keys from position `pos` on row `node` sees: the prefix, and the nodes of its mask.
__device__ __forceinline__ uint32_t sees32(const AttnArgs& a, const Segment& s, int node, int pos) {
    const int m0 = pos - s.len;         // first node
    if (m0 <= -32) return 0xffffffffu;
    const int from = m0 < 0 ? 0 : m0;
    const int w = from >> 6, sh = from & 63;
    unsigned long long bits = sees_word(a, s.node0, s.n, node, w) >> sh;
    if (sh > 32) bits |= sees_word(a, s.node0, s.n, node, w + 1) << (64 - sh);
    uint32_t r = (uint32_t)bits;
    if (m0 < 0) r = r << -m0 | ((1u << -m0) - 1u);
    return r;
}

// Values of V that are not finite were left out of the products: row `urow` of the unit, written already, gets those of
// the nodes that it sees in dimensions d .. d + count - 1.
template <int FMT, int ROWS, bool BY_DIMS = false>
__device__ __forceinline__ void add_not_finite(const AttnArgs& a, const Segment& s, const unsigned long long* bad, int urow, int d,
                                               int count) {
    const int nd = (s.row0 + urow) / a.group, hq = s.head * a.group + (s.row0 + urow) % a.group;
#pragma unroll 1
    for (int m = 0; m < s.n; ++m) {
        if (!(bad[m >> 6] & sees_word(a, s.node0, s.n, nd, m >> 6) & 1ull << (m & 63))) continue;
        const int page = page_of(a, s.b, s.len + m);
        if (page < 0) continue;
        const long long row = ((long long)page * a.kv_heads + s.head) * a.page_size + ((s.len + m) & (a.page_size - 1));
#pragma unroll 1
        for (int i = d; i < d + count; ++i) {
            float v;
            if constexpr (FMT == ACE_KV_FP8) v = (static_cast<const uint8_t*>(a.v_pool)[row * a.head_dim + i] & 0x7f) == 0x7f ? __uint_as_float(0x7fffffffu) : 0.f;
            else if constexpr (FMT == ACE_KV_INT4) v = finite_or_nan(float_of_bf16(reinterpret_cast<const uint16_t*>(a.v_scale)[row * groups4(a.head_dim) + i / kGroup4]));
            else v = to_f32(static_cast<const __nv_bfloat16*>(a.v_pool)[row * a.head_dim + i]);
            if (fabsf(v) < INFINITY) continue;
            if (s.part < 0) {
                __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + ((long long)(s.node0 + nd) * a.n_heads + hq) * a.head_dim + i;
                *out = from_f32<__nv_bfloat16>(to_f32(*out) + v);
            } else {
                a.ws.part_o[part_place<BY_DIMS>(ROWS, a.head_dim, s.part, urow, i)] += v;
            }
        }
    }
}

// By one warp, over an fp8 cache: row `urow` of the unit, written already, gets its share of the V rows that were left out for
// their scale: weights 2^(score - ref) times `mult`, which the row's sum has in it. (A whole unit's output is rounded once more by it:
// 2^-9 of what the products gave, where a far V is 2^6 of the others' or more.)
template <int ROWS, bool BY_DIMS>
__device__ __noinline__ void add_far(const AttnArgs& a, const Segment& s, const unsigned long long* far, int urow, float ref, float mult) {
    constexpr int kMost = 4;            // dimensions a lane (head sizes 64 and 128)
    const int lane = threadIdx.x & 31, per = a.head_dim / 32, d0 = lane * per;
    const int nd = (s.row0 + urow) / a.group, hq = s.head * a.group + (s.row0 + urow) % a.group;
    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + (s.node0 + nd) * a.q_token_stride + hq * a.q_head_stride + d0;
    float sum[kMost] = {};
    bool any = false;
#pragma unroll 1
    for (int w = 0; w < kMaxNodes / 64; ++w) {
#pragma unroll 1
        for (unsigned long long bits = far[w] & sees_word(a, s.node0, s.n, nd, w); bits; bits &= bits - 1) {
            const int pos = s.len + w * 64 + __ffsll(bits) - 1, page = page_of(a, s.b, pos);
            if (page < 0) continue;
            const long long row = ((long long)page * a.kv_heads + s.head) * a.page_size + (pos & (a.page_size - 1));
            float x = 0.f, v[kMost];
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                v[i] = 0.f;
                if (i >= per) continue;
                const uint32_t codes = static_cast<const uint8_t*>(a.k_pool)[row * a.head_dim + d0 + i] |
                                       static_cast<const uint8_t*>(a.v_pool)[row * a.head_dim + d0 + i] << 8;
                const uint32_t h = f16x2_of_e4m3x2(codes);
                const float2 kv = __half22float2(*reinterpret_cast<const __half2*>(&h));
                x = fmaf(to_f32(q[i]), kv.x, x);
                v[i] = kv.y == kv.y ? kv.y : 0.f;       // (NaN: add_not_finite)
            }
            x = warp_sum(x) * pow2_of_byte(a.k_scale[row]) * a.scale_log2;
            const float p = exp2f(x - ref) * mult, up = pow2_of_byte(a.v_scale[row]);
#pragma unroll
            for (int i = 0; i < kMost; ++i) sum[i] = fmaf(p * v[i], up, sum[i]);
            any = true;
        }
    }
    if (!any) return;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        if (i >= per) break;
        if (s.part < 0) {
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + ((long long)(s.node0 + nd) * a.n_heads + hq) * a.head_dim + d0 + i;
            *out = from_f32<__nv_bfloat16>(to_f32(*out) + sum[i]);
        } else {
            a.ws.part_o[part_place<BY_DIMS>(ROWS, a.head_dim, s.part, urow, d0 + i)] += sum[i];
        }
    }
}

// The same for rows first, first + step, .. below `end`. ml: a row's maximum (base 2) and sum.
template <int ROWS, bool BY_DIMS>
__device__ __noinline__ void add_far_rows(const AttnArgs& a, const Segment& s, const unsigned long long* far, const float2* ml, int first, int end,
                                          int step) {
    if (end > s.rows) end = s.rows;
    for (int r = first; r < end; r += step) add_far<ROWS, BY_DIMS>(a, s, far, r, ml[r].x, s.part >= 0 ? 1.f : ml[r].y == 0.f ? 0.f : 1.f / ml[r].y);
}

// 8 elements of a unit's q row (bf16), from dimension d on.
__device__ __forceinline__ uint4 load_q(const AttnArgs& a, const Segment& s, int row, int d) {
    const int nd = row / a.group;
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q) + (s.node0 + nd) * a.q_token_stride +
                               (s.head * a.group + row - nd * a.group) * a.q_head_stride + d;
    if ((uintptr_t)src % 16 == 0) return __ldg(reinterpret_cast<const uint4*>(src));
    const uint16_t* u = reinterpret_cast<const uint16_t*>(src);
    return make_uint4(u[0] | (uint32_t)u[1] << 16, u[2] | (uint32_t)u[3] << 16, u[4] | (uint32_t)u[5] << 16, u[6] | (uint32_t)u[7] << 16);
}

// Place of codes 16 c .. 16 c + 15 of a row in a tile of V as TMA leaves it (rows of 128 or 64 bytes, swizzled).
template <int D>
__device__ __forceinline__ int raw_v_offset(int row, int c) {
    return D == 128 ? row * 128 + ((c ^ (row & 7)) << 4) : row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
}

// A tile of V codes with drafted rows: zeros past the end and in place of NaN (all bits of a code but the sign), whose
// nodes are noted. Each thread cleans the 16 codes that it reads afterwards (row0 and c0 of the first).
template <int D>
__device__ __forceinline__ void clean_codes(unsigned char* v, int row0, int c0, const Segment& s, int pos0, unsigned long long* bad) {
    const int total = s.len + s.n;
#pragma unroll 1
    for (int i = 0; i < D / 16; ++i) {
        const int row = row0 + (i & 3) * 32, pos = pos0 + row;
        if (pos < s.len) continue;
        uint4* at = reinterpret_cast<uint4*>(v + raw_v_offset<D>(row, c0 + (i >> 2) * 4));
        if (pos >= total) {
            *at = make_uint4(0, 0, 0, 0);
            continue;
        }
        const uint4 w = *at;
        uint32_t x[4] = {w.x, w.y, w.z, w.w}, any = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t nan = ((x[j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
            any |= nan;
            x[j] &= ~((nan >> 7) * 0xffu);
        }
        if (any) {
            *at = make_uint4(x[0], x[1], x[2], x[3]);
            atomicOr(&bad[(pos - s.len) >> 6], 1ull << ((pos - s.len) & 63));
        }
    }
}

// The same for bf16 rows (infinities and NaN).
template <int D>
__device__ __forceinline__ void clean_bf16(unsigned char* v, int tid, const Segment& s, int pos0, unsigned long long* bad) {
    constexpr int kChunks = D / 8;
    const int total = s.len + s.n;
#pragma unroll 1
    for (int u = tid; u < 128 * kChunks; u += kConvThreads) {
        const int row = u / kChunks, c = u % kChunks, pos = pos0 + row;
        if (pos < s.len) continue;
        uint4* at = reinterpret_cast<uint4*>(v + (c >> 3) * 16384 + row * 128 + (((c & 7) ^ (row & 7)) << 4));
        if (pos >= total) {
            *at = make_uint4(0, 0, 0, 0);
            continue;
        }
        const uint4 w = *at;
        uint32_t x[4] = {w.x, w.y, w.z, w.w};
        bool found = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if ((x[i] & 0x7f80u) == 0x7f80u) found = true, x[i] &= 0xffff0000u;
            if ((x[i] & 0x7f800000u) == 0x7f800000u) found = true, x[i] &= 0xffffu;
        }
        if (found) {
            *at = make_uint4(x[0], x[1], x[2], x[3]);
            atomicOr(&bad[(pos - s.len) >> 6], 1ull << ((pos - s.len) & 63));
        }
    }
}

// ---------------------------------------------------------------- roles

// A role's walk over the CTA's segments. A segment stays in shared memory until done().
struct Walk {
    TcShared& m;
    const AttnArgs& a;
    Ring seg;
    // False: no more, or given up.
    __device__ __forceinline__ bool next() {
        if (!mbar_wait_warp(&m.seg_full[seg.i], seg.phase, a.err, &m.abort_flag)) {
            *static_cast<volatile int*>(&m.abort_flag) = 1;
            return false;
        }
        return m.seg[seg.i].go != 0;
    }
    __device__ __forceinline__ const Segment& segment() const { return m.seg[seg.i].s; }
    __device__ __forceinline__ void done() {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(&m.seg_empty[seg.i]);
        seg.next<kSegRing>();
    }
};

// The CTA's segments, published by one warp ahead of the roles that work on them.
template <int ROWS, int START>
struct Scheduler {
    TcShared& m;
    const AttnArgs& a;
    Ring seg;
    Cursor cur;
    bool more, done;
    __device__ __forceinline__ Scheduler(TcShared& m_, const AttnArgs& a_) : m(m_), a(a_), seg{}, cur{}, done(false) {
        if ((threadIdx.x & 31) == 0) note_none(a);
        more = cursor_init<ROWS, kTcKeys, START>(a, blockIdx.x, gridDim.x, cur);
    }
    // The next segment, or that there is none. False: given up.
    __device__ __forceinline__ bool publish() {
        if (done) return true;
        if (!mbar_wait_warp(&m.seg_empty[seg.i], seg.phase ^ 1u, a.err, &m.abort_flag)) {
            *static_cast<volatile int*>(&m.abort_flag) = 1;
            return false;
        }
        Segment s{};
        more = more && cursor_next<ROWS, kTcKeys, START>(a, blockIdx.x, cur, s);
        if ((threadIdx.x & 31) == 0) {
            m.seg[seg.i].s = s;
            m.seg[seg.i].go = more;
            if (more) note_unit(a, s);
            for (int w = 0; w < kMaxNodes / 64; ++w) m.seg[seg.i].bad[w] = m.seg[seg.i].far[w] = 0;
            mbar_arrive(&m.seg_full[seg.i]);
        }
        seg.next<kSegRing>();
        done = !more;
        return true;
    }
};

template <int ROWS, int START>
__device__ __forceinline__ void role_schedule(TcShared& m, const AttnArgs& a) {
    Scheduler<ROWS, START> sched(m, a);
    while (!sched.done && sched.publish()) {}
}

// One warp: TMA loads of K and V tiles; lane x loads box x of a tile. started(): called when a segment's first tile is under
// way; false gives up.
template <bool FP8, int D, int NK, int NV, typename Started>
__device__ __forceinline__ void role_load(TcShared& m, const TcAttnArgs& p, unsigned char* k_smem, unsigned char* v_smem, Started started) {
    constexpr int kTile = 128 * D * (FP8 ? 1 : 2);
    const AttnArgs& a = p.a;
    volatile int* abort_flag = &m.abort_flag;
    const int lane = threadIdx.x & 31;
    Ring rk, rv;
    long long nk = 0, nv = 0;
    bool ok = true;
    const int boxes = kTcKeys / p.box_rows;
    Walk walk{m, a, {}};
    while (ok && walk.next()) {
        const Segment& s = walk.segment();
        const int total = s.len + s.n;
        // a tile's pages are looked up while the tile before it is loaded; -1: a page that does not exist, whose rows are read
        // from before the pool, where TMA fills in zeros (what the buffer held before may be another request's)
        auto look_up = [&](int t) {
            const int at = t * kTcKeys + lane * p.box_rows;
            return t < s.tile1 && lane < boxes && at < total ? page_of(a, s.b, at) : -2;
        };
        int next_page = look_up(s.tile0);
        for (int t = s.tile0; t < s.tile1; ++t) {
            const int pos = t * kTcKeys + lane * p.box_rows;
            const int page = next_page;
            next_page = look_up(t + 1);
            const int row = page < 0 ? -kTcKeys : a.row0 + (page * a.kv_heads + s.head) * a.page_size + (pos & (a.page_size - 1));
            const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, page >= -1)) * (uint32_t)(p.box_rows * (kTile / 128));
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                Ring& r = kv ? rv : rk;
                uint64_t* full = kv ? m.v_full : m.k_full;
                uint64_t* empty = kv ? m.v_empty : m.k_empty;
                if (!mbar_wait_warp(&empty[r.i], r.phase ^ 1u, a.err, abort_flag)) { ok = false; break; }
                if (lane == 0) mbar_expect_tx(&full[r.i], bytes);
                __syncwarp();
                if (page >= -1) {
                    unsigned char* dst = (kv ? v_smem : k_smem) + r.i * kTile;
                    const CUtensorMap* map = kv ? &p.v : &p.k;
                    if constexpr (FP8) {
                        tma_load_2d(dst + lane * p.box_rows * D, map, &full[r.i], 0, row);
                    } else {
#pragma unroll
                        for (int h = 0; h < D / 64; ++h)
                            tma_load_2d(dst + h * 16384 + lane * p.box_rows * 128, map, &full[r.i], h * 64, row);
                    }
                }
                if (kv) ++nv, rv.next<NV>(); else ++nk, rk.next<NK>();
            }
            if (ok && t == s.tile0) ok = started();
            if (!ok) break;
        }
        walk.done();
    }
    if (!ok) *abort_flag = 1;
    if (*abort_flag) {
        // let the copies already issued land before the CTA exits
        for (long long f = nk - 1; f >= 0 && f >= nk - NK; --f)
            if (!mbar_wait(&m.k_full[f % NK], (uint32_t)((f / NK) & 1), a.err)) break;
        for (long long f = nv - 1; f >= 0 && f >= nv - NV; --f)
            if (!mbar_wait(&m.v_full[f % NV], (uint32_t)((f / NV) & 1), a.err)) break;
    }
}

// fp8 caches: `eref`, the power of two that V's factors are relative to, is above the scales e of all positions that count in the
// products. It is the rows' common unit, so what some of them do not see may not raise it as it likes: `common` is two octaves
// above the scales so far that every row of the unit sees (where there are none, above the least of the request's nodes), and
// nodes that some rows do not see raise eref by at most ROOM from there. A node still higher is far: it counts in the softmax, but
// its V is left out of the products, and added to the rows that see it once they are done.
constexpr int kNoRef = -1000, kLeastRef = -125;
struct Reference {
    int eref, common;
};

// By one warp: the reference with nodes of the tile above it. vb: scale bytes of V at the lane's four positions from `pos` on
// (0: none).
template <int ROOM>
__device__ __noinline__ Reference raise_reference(const AttnArgs& a, const Segment& s, unsigned long long* far, uint32_t vb, int pos, Reference r) {
    const int lane = threadIdx.x & 31;
    int top = 0, low = 256;             // scale bytes of nodes: the largest (that all rows see), the least of any
    if (r.common == kNoRef) {
        const int tile = pos - 4 * lane;
        if (s.len >= tile && s.len + s.n <= tile + kTcKeys) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int byte = (int)(vb >> (8 * i) & 0xff);
                top = max(top, byte);
                if (byte) low = min(low, byte);
            }
        } else {
            for (int m = lane; m < s.n; m += 32) {
                const int page = page_of(a, s.b, s.len + m);
                if (page < 0) continue;
                const int byte = a.v_scale[((long long)page * a.kv_heads + s.head) * a.page_size + ((s.len + m) & (a.page_size - 1))];
                top = max(top, byte);
                if (byte) low = min(low, byte);
            }
        }
        top = __reduce_max_sync(0xffffffffu, top);
        low = __reduce_min_sync(0xffffffffu, low);
        // who sees what makes no difference while all are within ROOM
        if (top - low <= ROOM) {
            if (top) r.common = low - 127 + 2, r.eref = max(r.eref, max(r.common, top - 127));
            return r;
        }
        top = 0;
    }
    // nodes that every row's node sees
    const int first = s.row0 / a.group, last = (s.row0 + s.rows - 1) / a.group;
    unsigned long long all[kMaxNodes / 64];
#pragma unroll
    for (int w = 0; w < kMaxNodes / 64; ++w) {
        unsigned long long x = ~0ull;
        for (int i = first + lane; i <= last; i += 32) x &= sees_word(a, s.node0, s.n, i, w);
        all[w] = (unsigned long long)__reduce_and_sync(0xffffffffu, (unsigned)(x >> 32)) << 32 | __reduce_and_sync(0xffffffffu, (unsigned)x);
    }
    auto seen = [&](int m) {
        unsigned long long x = 0;
#pragma unroll
        for (int w = 0; w < kMaxNodes / 64; ++w)
            if (w == m >> 6) x = all[w];
        return (x >> (m & 63) & 1) != 0;
    };
    if (r.common == kNoRef) {
        for (int m = lane; m < s.n; m += 32) {
            const int page = seen(m) ? page_of(a, s.b, s.len + m) : -1;
            if (page < 0) continue;
            top = max(top, (int)a.v_scale[((long long)page * a.kv_heads + s.head) * a.page_size + ((s.len + m) & (a.page_size - 1))]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (pos + i >= s.len && seen(pos + i - s.len)) top = max(top, (int)(vb >> (8 * i) & 0xff));
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (r.common == kNoRef && top == 0) top = low;
    if (top - 127 > r.common) r.common = top - 127 + 2;
    int e_top = r.common;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int byte = (int)(vb >> (8 * i) & 0xff), m = pos + i - s.len;
        if (m < 0 || byte == 0) continue;
        if (byte - 127 <= r.common + ROOM) e_top = max(e_top, byte - 127);
        else atomicOr(&far[m >> 6], 1ull << (m & 63));
    }
    r.eref = max(r.eref, __reduce_max_sync(0xffffffffu, e_top));
    return r;
}

// One warp, fp8 caches: a tile's scales, 4 positions a lane. K's as factors 2^e; V's as 2^(e - eref + kVUp) with the tile's
// eref.
template <int ROOM, typename V4>
__device__ __forceinline__ void role_scales(TcShared& m, const AttnArgs& a, float4 (*kf_out)[32], V4 (*vf_out)[32]) {
    volatile int* abort_flag = &m.abort_flag;
    const int lane = threadIdx.x & 31;
    Ring r;
    bool ok = true;
    Walk walk{m, a, {}};
    while (ok && walk.next()) {
        const Segment& s = walk.segment();
        const int total = s.len + s.n;
        Reference ref{kLeastRef, kNoRef};
        // in batches of 4 tiles, pages two and scales one batch ahead: a load takes longer than a tile
        auto look_up = [&](int t, int (&page)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = (t + i) * kTcKeys + lane * 4;
                page[i] = t + i < s.tile1 && at < total ? page_of(a, s.b, at) : -1;
            }
        };
        auto load = [&](const int (&page)[4], int t, uint32_t (&kb)[4], uint32_t (&vb)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                kb[i] = vb[i] = 0;
                if (page[i] >= 0) {
                    const long long at = ((long long)page[i] * a.kv_heads + s.head) * a.page_size + (((t + i) * kTcKeys + lane * 4) & (a.page_size - 1));
                    kb[i] = __ldg(reinterpret_cast<const uint32_t*>(a.k_scale + at));
                    vb[i] = __ldg(reinterpret_cast<const uint32_t*>(a.v_scale + at));
                }
            }
        };
        int page[4];
        uint32_t kb_next[4], vb_next[4], kb4[4], vb4[4];
        look_up(s.tile0, page);
        load(page, s.tile0, kb_next, vb_next);
        look_up(s.tile0 + 4, page);
        for (int t = s.tile0; t < s.tile1; ++t) {
            const int j = (t - s.tile0) & 3, pos = t * kTcKeys + lane * 4;
            if (j == 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) kb4[i] = kb_next[i], vb4[i] = vb_next[i];
                load(page, t + 4, kb_next, vb_next);
                look_up(t + 8, page);
            }
            uint32_t kb = kb4[0], vb = vb4[0];
#pragma unroll
            for (int i = 0; i < 3; ++i) kb4[i] = kb4[i + 1], vb4[i] = vb4[i + 1];
            if (pos + 4 > total) {
                const int left = total - pos;       // positions of the four that exist
                const uint32_t have = left <= 0 ? 0u : 0xffffffffu >> (8 * (4 - left));
                kb &= have;
                vb &= have;
            }
            int top = 0, nodes_top = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int byte = (int)(vb >> (8 * i) & 0xff);
                if (pos + i < s.len) top = max(top, byte);
                else nodes_top = max(nodes_top, byte);
            }
            top = __reduce_max_sync(0xffffffffu, top);
            // two octaves of room, so that small differences between tiles do not move it
            if (top - 127 > ref.common && top != 0) ref.common = top - 127 + 2, ref.eref = max(ref.eref, ref.common);
            if (__any_sync(0xffffffffu, nodes_top - 127 > ref.eref)) ref = raise_reference<ROOM>(a, s, m.seg[walk.seg.i].far, vb, pos, ref);
            const int eref = ref.eref;
            float kf[4], vf[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int vbyte = (int)(vb >> (8 * i) & 0xff);
                kf[i] = pow2_of_byte((int)(kb >> (8 * i) & 0xff));
                const int e = vbyte - eref + kVUp;      // biased exponent
                vf[i] = vbyte == 0 || e <= 0 || vbyte - 127 > eref ? 0.f : pow2_of_byte(e);
            }
            if (!mbar_wait_warp(&m.aux_empty[r.i], r.phase ^ 1u, a.err, abort_flag)) { ok = false; break; }
            kf_out[r.i][lane] = make_float4(kf[0], kf[1], kf[2], kf[3]);
            if constexpr (sizeof(V4) == 16) {
                vf_out[r.i][lane] = make_float4(vf[0], vf[1], vf[2], vf[3]);
            } else {
                const __half2 lo = __floats2half2_rn(vf[0], vf[1]), hi = __floats2half2_rn(vf[2], vf[3]);
                vf_out[r.i][lane] = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
            }
            if (lane == 0) m.eref[r.i] = eref;
            __syncwarp();
            if (lane == 0) mbar_arrive(&m.aux_full[r.i]);
            r.next<kAuxRing>();
        }
        if (ok) walk.done();
    }
    if (!ok) *abort_flag = 1;
}

}  // namespace
}  // namespace ace
