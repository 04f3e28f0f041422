// ace_attn_q4.cu — attention for trees of drafted tokens over a cache in 4 bits where a unit has few query rows (nodes times query
// heads a kv head at most 32; bf16 activations, head sizes 64 and 128): bound by the cache's bytes, 72 a row of 128.
//   S^T = K Q^T       16 positions x 8 rows a product (m16n8k16); codes are exact in fp16, q too once its row is scaled by a power
//                     of two, so a group's product is exact but for fp32's sums, and its scale is one factor of 16 x 8 sums
//   P^T = 2^(S^T - ref)   bf16
//   O^T += V^T P^T    V's code * scale is exact in bf16 (3 significant bits times 4)
// At 4 bits a tile of 128 positions is 18 KB and takes HBM 750 cycles of an SM, in which its 32768 codes have to become operands: too
// little time for the hand-overs of tcgen05 (scores, softmax, weights and conversion through shared and tensor memory take 2000
// cycles a tile in ace_attn_few.cu, fp8 codes without any conversion). So the codes become operands in the registers of the warp
// that multiplies them (mma.sync; 1.3 operations a code), S^T turns into the second product's operand by movmatrix, and the warps of a
// CTA walk their 16 positions of each tile on their own, with their own running maxima, from rings of cp.async stages; they meet at
// a unit's end only.
#include <cfloat>

#include "ace_attn_tc.cuh"

namespace ace {
namespace {

constexpr int kWarps = 8, kThreads4 = 32 * kWarps, kStep = 16, kStages = 4;
constexpr int kStart4 = 2;              // a unit's start and end in tiles of the work line
constexpr float kNone4 = -FLT_MAX;      // reference of a row that has seen nothing: any score passes it

template <int D>
struct Q4 {
    static constexpr int ROW = D / 2, G = D / kGroup4;          // bytes and groups of a row
    static constexpr int CODES = kStep * ROW, SCALES = kStep * G * 2;
    static constexpr int STAGE = 2 * CODES + 2 * SCALES;
    static constexpr int RING = kWarps * kStages * STAGE;
    static constexpr int PITCH = D + 4;                         // floats of a row of a warp's O: lanes' stores in distinct banks
    static constexpr int PER = D / 8;                           // dimensions a lane has of a position's V
};

template <int D, int NT>
struct Q4Shared {
    unsigned char ring[Q4<D>::RING];
    float join[kWarps * 8 * Q4<D>::PITCH];
    uint4 q[NT * Q4<D>::G * 32];        // operand of S^T: [8 rows][group][lane]
    float f_row[NT * 8];                // q's scale times the softmax's
    int node[NT * 8];                   // row's node of the request
    float2 ml[kWarps][NT * 8];          // a warp's reference and sum
    unsigned long long bad[kMaxNodes / 64];     // nodes with a V that is not finite, left out of the products
    Segment seg[2];
    int go[2];
};

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const float (&c)[4]) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The transpose of an 8 x 8 matrix of 16-bit values, two of a row a lane.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t add_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
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

// Elements 0 and 4, 1 and 5, 2 and 6, 3 and 7 of a word of codes as fp16, less 8: 1024 + c is c in the last places of 1024, and
// 1024 + 16 c the same one nibble up.
__device__ __forceinline__ void f16_of_codes(uint32_t w, uint32_t (&h)[4]) {
    constexpr uint32_t k1024 = 0x64006400u, kMinus1032 = 0xe408e408u, k16th = 0x2c002c00u, kMinus72 = 0xd480d480u;
    const uint32_t u = w >> 8;
    h[0] = add_f16x2(and_or(w, 0x000f000fu, k1024), kMinus1032);
    h[1] = fma_f16x2(and_or(w, 0x00f000f0u, k1024), k16th, kMinus72);
    h[2] = add_f16x2(and_or(u, 0x000f000fu, k1024), kMinus1032);
    h[3] = fma_f16x2(and_or(u, 0x00f000f0u, k1024), k16th, kMinus72);
}

// Element I of two positions' four codes (16 bits each) as bf16 times their scales: 128 + c is c in the last places of 128, and
// s (128 + c) - 136 s is exact. LARGE: 136 s may be past bf16's largest, so the 136 goes before the product.
template <int I, bool LARGE>
__device__ __forceinline__ uint32_t bf16_of_codes(uint32_t x, uint32_t s2, uint32_t minus136s) {
    const uint32_t c = and_or(x >> (4 * I), 0x000f000fu, 0x43004300u);
    if constexpr (LARGE) return fma_bf16x2(fma_bf16x2(c, 0x3f803f80u, 0xc308c308u), s2, 0x80008000u);
    else return fma_bf16x2(c, s2, minus136s);
}

__device__ __forceinline__ void copy16(void* dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(bytes) : "memory");
}

// Place of 16-byte chunk c of a position's codes in a stage. D = 128: two positions a line of 128 bytes, D = 64: four; turned so
// that the 8 positions x 16 bytes of a K operand, and the 4 positions x 32 (64) of a V operand's half (whole), lie in distinct banks.
template <int D>
__device__ __forceinline__ int chunk_at(int r, int c) {
    if constexpr (D == 128) {
        const int line = r >> 1;
        return line * 128 + ((((r & 1) * 5) ^ c ^ ((line & 1) * 2) ^ ((line & 2) * 2)) << 4);
    } else {
        return (r >> 2) * 128 + ((((r & 3) * 2 + c) ^ (r >> 2 & 1)) << 4);
    }
}

// O += V^T P^T of a stage: the lane's dimensions PER g .. of positions t, t + 4, t + 8, t + 12.
template <int D, int NT, bool LARGE>
__device__ __forceinline__ void add_values(const unsigned char* v, const uint16_t (&s)[4], int g, int t, const uint32_t (&p)[NT][2], float (&o)[D / 16][NT][4]) {
    constexpr int W = D / 64;           // words of codes of a position a lane has
    uint32_t w[4][W];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = t + 4 * i;
        if constexpr (D == 128) {
            const uint2 x = *reinterpret_cast<const uint2*>(v + chunk_at<D>(r, g >> 1) + (g & 1) * 8);
            w[i][0] = x.x;
            w[i][1] = x.y;
        } else {
            w[i][0] = *reinterpret_cast<const uint32_t*>(v + chunk_at<D>(r, g >> 2) + (g & 3) * 4);
        }
    }
    uint32_t s2[2], m2[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        s2[i] = s[2 * i] | (uint32_t)s[2 * i + 1] << 16;
        m2[i] = fma_bf16x2(s2[i], 0xc308c308u, 0x80008000u);            // times -136
    }
#pragma unroll
    for (int k = 0; k < W; ++k) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint32_t sel = half ? 0x7632u : 0x5410u;
            const uint32_t x0 = __byte_perm(w[0][k], w[1][k], sel), x1 = __byte_perm(w[2][k], w[3][k], sel);
            uint32_t a[4] = {bf16_of_codes<0, LARGE>(x0, s2[0], m2[0]), bf16_of_codes<1, LARGE>(x0, s2[0], m2[0]),
                             bf16_of_codes<0, LARGE>(x1, s2[1], m2[1]), bf16_of_codes<1, LARGE>(x1, s2[1], m2[1])};
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_bf16(o[4 * k + 2 * half][n], a, p[n][0], p[n][1]);
            a[0] = bf16_of_codes<2, LARGE>(x0, s2[0], m2[0]), a[1] = bf16_of_codes<3, LARGE>(x0, s2[0], m2[0]);
            a[2] = bf16_of_codes<2, LARGE>(x1, s2[1], m2[1]), a[3] = bf16_of_codes<3, LARGE>(x1, s2[1], m2[1]);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_bf16(o[4 * k + 2 * half + 1][n], a, p[n][0], p[n][1]);
        }
    }
}

// Rows r = 8 n + 0 .. 7 of a unit, n < NT. Lane (g, t) = (lane / 4, lane % 4) holds rows 2 t and 2 t + 1 of each eight: scores of positions
// place(g) and place(g) + 8, and dimensions PER g .. PER g + PER - 1 of O, tile j of it dimensions 2 j and 2 j + 1 of those.
template <int D, int NT>
__global__ void __launch_bounds__(kThreads4, NT <= 2 ? 2 : 1) k_attn_q4(const __grid_constant__ AttnArgs a) {
    using C = Q4<D>;
    constexpr int ROWS = 8 * NT, TJ = D / 16, G = C::G;
    extern __shared__ __align__(128) unsigned char smem_raw[];
    Q4Shared<D, NT>& m = *reinterpret_cast<Q4Shared<D, NT>*>(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    unsigned char* ring = m.ring + warp * (kStages * C::STAGE);
    // position of row i of the product: those of a V operand's halves lie 4 apart
    const int place = (g >> 1) + 4 * (g & 1);

    Cursor cur{};
    bool more = false;
    if (warp == 0) {
        if (lane == 0) note_none(a);
        more = cursor_init<ROWS, kTcKeys, kStart4>(a, blockIdx.x, gridDim.x, cur);
    }
    // by warp 0: the segment after, into slot i
    auto schedule = [&](int i) {
        if (warp == 0) {
            Segment s{};
            more = more && cursor_next<ROWS, kTcKeys, kStart4>(a, blockIdx.x, cur, s);
            if (lane == 0) {
                m.go[i] = more;
                if (more) {
                    m.seg[i] = s;
                    note_unit(a, s);
                }
            }
        }
    };
    // stage of tile `tile`: the warp's 16 positions (of one page); what does not exist is zeros
    auto load = [&](const Segment& s, int tile, int stage, int page) {
        if (tile < s.tile1) {
            const int pos = tile * kTcKeys + warp * kStep, left = page < 0 ? 0 : min(s.len + s.n - pos, kStep);
            const long long row = left <= 0 ? 0 : ((long long)page * a.kv_heads + s.head) * a.page_size + (pos & (a.page_size - 1));
            unsigned char* at = ring + stage * C::STAGE;
            constexpr int CHUNKS = C::CODES / 16, PER_ROW = C::ROW / 16;
#pragma unroll
            for (int i = 0; i < CHUNKS; i += 32) {
                const int id = i + lane, r = id / PER_ROW, c = id % PER_ROW, bytes = r < left ? 16 : 0;
                copy16(at + chunk_at<D>(r, c), static_cast<const unsigned char*>(a.k_pool) + row * C::ROW + id * 16, bytes);
                copy16(at + C::CODES + chunk_at<D>(r, c), static_cast<const unsigned char*>(a.v_pool) + row * C::ROW + id * 16, bytes);
            }
            constexpr int SCALE_CHUNKS = C::SCALES / 16;
            if (lane < 2 * SCALE_CHUNKS) {
                const int i = lane % SCALE_CHUNKS, bytes = min(max(left * (2 * G) - i * 16, 0), 16);
                const uint8_t* pool = lane < SCALE_CHUNKS ? a.k_scale : a.v_scale;
                copy16(at + 2 * C::CODES + lane * 16, pool + row * (2 * G) + i * 16, bytes);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto look_up = [&](const Segment& s, int tile) {
        const int pos = tile * kTcKeys + warp * kStep;
        return tile < s.tile1 && pos < s.len + s.n ? page_of(a, s.b, pos) : -1;
    };
    // a segment's first stages; returns the page of the one after
    auto begin = [&](const Segment& s) {
        int page[kStages];
#pragma unroll
        for (int i = 0; i < kStages; ++i) page[i] = look_up(s, s.tile0 + i);
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i) load(s, s.tile0 + i, i, page[i]);
        return page[kStages - 1];
    };
    // q's operand, PER_Q lanes a row with 8 elements each; elements of a row in units of 2^(e - 14), where its largest is below
    // 2^(e + 1): all bits of elements down to 2^-31 of it
    constexpr int PER_Q = D / 8, Q_ROWS = kThreads4 / PER_Q, Q_TURNS = (ROWS + Q_ROWS - 1) / Q_ROWS;
    auto q_load = [&](const Segment& s, uint4 (&raw)[Q_TURNS]) {
#pragma unroll
        for (int i = 0; i < Q_TURNS; ++i) {
            const int r = i * Q_ROWS + tid / PER_Q;
            raw[i] = r < s.rows ? load_q(a, s, s.row0 + r, tid % PER_Q * 8) : make_uint4(0, 0, 0, 0);
        }
    };
    auto q_store = [&](const Segment& s, const uint4 (&raw)[Q_TURNS]) {
#pragma unroll
        for (int i = 0; i < Q_TURNS; ++i) {
            const int r = i * Q_ROWS + tid / PER_Q, c = tid % PER_Q;
            float f[8], amax = 0.f;
            Vec16<__nv_bfloat16>::to_float(raw[i], f);
#pragma unroll
            for (int x = 0; x < 8; ++x) f[x] = finite_or_nan(f[x]), amax = fmaxf(amax, fabsf(f[x]));
#pragma unroll
            for (int o = PER_Q / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
            if (r >= ROWS) continue;
            const int e = max((int)(__float_as_uint(amax) >> 23), 15);
            const float mul = __uint_as_float((uint32_t)(268 - e) << 23);
            uint32_t w[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const __half2 h = __floats2half2_rn(f[x] * mul, f[x + 4] * mul);
                w[x] = *reinterpret_cast<const uint32_t*>(&h);
            }
            m.q[((r >> 3) * G + c / 4) * 32 + (r & 7) * 4 + c % 4] = make_uint4(w[0], w[1], w[2], w[3]);
            if (c == 0) {
                m.f_row[r] = a.scale_log2 * pow2_of_byte(e - 14);
                m.node[r] = r < s.rows ? (s.row0 + r) / a.group : 0;
            }
        }
        if (tid < kMaxNodes / 64) m.bad[tid] = 0;
    };

    schedule(0);
    __syncthreads();
    if (!m.go[0]) return;
    int next_page;
    {
        next_page = begin(m.seg[0]);
        uint4 raw[Q_TURNS];
        q_load(m.seg[0], raw);
        q_store(m.seg[0], raw);
    }
    __syncthreads();
    for (int turn = 0;; turn ^= 1) {
        const Segment& s = m.seg[turn];
        schedule(turn ^ 1);
        const int total = s.len + s.n;
        float o[TJ][NT][4], ref[NT][2], l[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int j = 0; j < TJ; ++j) o[j][n][0] = o[j][n][1] = o[j][n][2] = o[j][n][3] = 0.f;
            ref[n][0] = ref[n][1] = kNone4;
            l[n][0] = l[n][1] = 0.f;
        }
        int stage = 0;
        for (int tile = s.tile0; tile < s.tile1; ++tile) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
            __syncwarp();               // all lanes' copies are there, and the stage before is read
            load(s, tile + kStages - 1, (stage + kStages - 1) % kStages, next_page);
            next_page = look_up(s, tile + kStages);
            const unsigned char* at = ring + stage * C::STAGE;
            stage = (stage + 1) % kStages;
            const int pos = tile * kTcKeys + warp * kStep;
            if (pos >= total) continue;
            // ---- scores
            uint64_t x01[NT], x23[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) x01[n] = x23[n] = 0ull;
            uint32_t k0[G / 2], k1[G / 2];          // scales of the two positions
            if constexpr (G == 4) {
                const uint2 u = *reinterpret_cast<const uint2*>(at + 2 * C::CODES + place * 8), w = *reinterpret_cast<const uint2*>(at + 2 * C::CODES + place * 8 + 64);
                k0[0] = u.x, k0[1] = u.y, k1[0] = w.x, k1[1] = w.y;
            } else {
                k0[0] = *reinterpret_cast<const uint32_t*>(at + 2 * C::CODES + place * 4);
                k1[0] = *reinterpret_cast<const uint32_t*>(at + 2 * C::CODES + place * 4 + 32);
            }
#pragma unroll
            for (int b = 0; b < G; ++b) {
                uint32_t h0[4], h1[4];
                f16_of_codes(*reinterpret_cast<const uint32_t*>(at + chunk_at<D>(place, b) + t * 4), h0);
                f16_of_codes(*reinterpret_cast<const uint32_t*>(at + chunk_at<D>(place + 8, b) + t * 4), h1);
                const uint32_t a0[4] = {h0[0], h1[0], h0[1], h1[1]}, a1[4] = {h0[2], h1[2], h0[3], h1[3]};
                const float f0 = __uint_as_float(b & 1 ? k0[b / 2] & 0xffff0000u : k0[b / 2] << 16);
                const float f1 = __uint_as_float(b & 1 ? k1[b / 2] & 0xffff0000u : k1[b / 2] << 16);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint4 q = m.q[(n * G + b) * 32 + lane];
                    float c[4];
                    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
                    mma_f16(c, a0, q.x, q.y, zero);
                    mma_f16(c, a1, q.z, q.w, c);
                    x01[n] = fma2(pair(c[0], c[1]), pair(f0, f0), x01[n]);
                    x23[n] = fma2(pair(c[2], c[3]), pair(f1, f1), x23[n]);
                }
            }
            float x[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float2 f = *reinterpret_cast<const float2*>(&m.f_row[8 * n + 2 * t]);
                unpair(mul2(x01[n], pair(f.x, f.y)), x[n][0], x[n][1]);
                unpair(mul2(x23[n], pair(f.x, f.y)), x[n][2], x[n][3]);
            }
            uint16_t vs[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                vs[i] = *reinterpret_cast<const uint16_t*>(at + 2 * C::CODES + C::SCALES + (t + 4 * i) * (2 * G) + g * G / 8 * 2);
            if (pos + kStep > s.len) {
                // drafted rows, which not every node sees, or past the end
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int nd = pos + place + 8 * i - s.len;
                    if (nd < 0) continue;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const bool sees = nd < s.n && (sees_word(a, s.node0, s.n, m.node[8 * n + 2 * t + r], nd >> 6) >> (nd & 63) & 1);
                            if (!sees) x[n][2 * i + r] = -INFINITY;
                        }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int nd = pos + t + 4 * i - s.len;
                    if (nd < 0 || (vs[i] & 0x7f80u) != 0x7f80u) continue;
                    vs[i] = 0;
                    atomicOr(&m.bad[nd >> 6], 1ull << (nd & 63));
                }
            }
            // ---- references: a row's moves where a score is 2^kLazy above it
            float over = -INFINITY;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int r = 0; r < 2; ++r) over = fmaxf(over, fmaxf(x[n][r], x[n][2 + r]) - ref[n][r]);
            if (__any_sync(0xffffffffu, over > (float)kLazy)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float top = fmaxf(x[n][r], x[n][2 + r]);
#pragma unroll
                        for (int w = 4; w < 32; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
                        const float now = top > ref[n][r] + (float)kLazy ? top : ref[n][r], f = exp2_approx(ref[n][r] - now);
                        ref[n][r] = now;
                        l[n][r] *= f;
#pragma unroll
                        for (int j = 0; j < TJ; ++j) o[j][n][r] *= f, o[j][n][2 + r] *= f;
                    }
            }
            // ---- weights
            uint32_t p[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i] = exp2_approx(x[n][i] - ref[n][i & 1]);
                l[n][0] += e[0] + e[2];
                l[n][1] += e[1] + e[3];
                const __nv_bfloat162 u = __floats2bfloat162_rn(e[0], e[1]), w = __floats2bfloat162_rn(e[2], e[3]);
                p[n][0] = transposed(*reinterpret_cast<const uint32_t*>(&u));
                p[n][1] = transposed(*reinterpret_cast<const uint32_t*>(&w));
            }
            // ---- values
            bool large = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) large = large || (vs[i] & 0x7fffu) >= 0x7b80u;      // 2^120
            if (__any_sync(0xffffffffu, large)) add_values<D, NT, true>(at + C::CODES, vs, g, t, p, o);
            else add_values<D, NT, false>(at + C::CODES, vs, g, t, p, o);
        }
        // ---------------- the unit's result, or this CTA's part of it
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
#pragma unroll
                for (int w = 4; w < 32; w <<= 1) l[n][r] += __shfl_xor_sync(0xffffffffu, l[n][r], w);
                if (g == 0) m.ml[warp][8 * n + 2 * t + r] = make_float2(ref[n][r], l[n][r]);
            }
        __syncthreads();                // all have read q; the next segment is known
        const bool go = m.go[turn ^ 1];
        uint4 raw[Q_TURNS];
        if (go) {
            next_page = begin(m.seg[turn ^ 1]);
            q_load(m.seg[turn ^ 1], raw);
        }
        const bool whole = s.part < 0;
        const unsigned long long bad[kMaxNodes / 64] = {m.bad[0], m.bad[1], m.bad[2], m.bad[3]};
        const bool any_bad = (bad[0] | bad[1] | bad[2] | bad[3]) != 0;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (n > 0) __syncthreads();
            if (8 * n >= s.rows) break;
            // this warp's share of its rows, relative to the rows' largest reference
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float top = kNone4;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) top = fmaxf(top, m.ml[w][8 * n + 2 * t + r].x);
                const float f = exp2_approx(ref[n][r] - top);
                float* to = m.join + (warp * 8 + 2 * t + r) * C::PITCH + g * 2;
#pragma unroll
                for (int j = 0; j < TJ; ++j) *reinterpret_cast<float2*>(to + j * 16) = make_float2(o[j][n][r] * f, o[j][n][2 + r] * f);
            }
            __syncthreads();
            // dimensions 2 u and 2 u + 1 of a row: lane group g = 2 u / PER, tile j = u % (PER / 2)
            for (int i = tid; i < 8 * (D / 2); i += kThreads4) {
                const int r8 = i / (D / 2), u = i % (D / 2), r = 8 * n + r8, at = u % (C::PER / 2) * 16 + u / (C::PER / 2) * 2;
                if (r >= s.rows) break;
                float top = kNone4, sum = 0.f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) top = fmaxf(top, m.ml[w][r].x);
                float2 v = make_float2(0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float2 e = m.ml[w][r], y = *reinterpret_cast<const float2*>(m.join + (w * 8 + r8) * C::PITCH + at);
                    sum = fmaf(e.y, exp2_approx(e.x - top), sum);
                    v.x += y.x;
                    v.y += y.y;
                }
                const int ur = s.row0 + r, nd = ur / a.group, hq = s.head * a.group + ur - nd * a.group;
                if (any_bad) {
                    // what is not finite in a V that the row sees
                    for (int k = 0; k < s.n; ++k) {
                        if (!(m.bad[k >> 6] & sees_word(a, s.node0, s.n, nd, k >> 6) & 1ull << (k & 63))) continue;
                        const int page = page_of(a, s.b, s.len + k);
                        if (page < 0) continue;
                        const long long row = ((long long)page * a.kv_heads + s.head) * a.page_size + ((s.len + k) & (a.page_size - 1));
                        const uint16_t scale = reinterpret_cast<const uint16_t*>(a.v_scale)[row * G + 2 * u / kGroup4];
                        if ((scale & 0x7f80u) == 0x7f80u) v.x = v.y = __uint_as_float(0x7fffffffu);
                    }
                }
                const long long out = (long long)(s.node0 + nd) * a.n_heads + hq;
                if (whole) {
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    const __nv_bfloat162 b = __floats2bfloat162_rn(v.x * inv, v.y * inv);
                    reinterpret_cast<__nv_bfloat162*>(static_cast<__nv_bfloat16*>(a.out) + out * D)[u] = b;
                    if (u == 0 && a.lse) a.lse[out] = ((top == kNone4 ? -INFINITY : top) + log2f(sum)) * 0.69314718055994530942f;
                } else {
                    *reinterpret_cast<float2*>(a.ws.part_o + ((long long)s.part * ROWS + r) * D + 2 * u) = v;
                    if (u == 0) a.ws.part_ml[(long long)s.part * ROWS + r] = make_float2(top == kNone4 ? -INFINITY : top, sum);
                }
            }
        }
        if (!go) break;
        __syncthreads();                // bad and q are free
        q_store(m.seg[turn ^ 1], raw);
        __syncthreads();
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

template <int D, int NT>
constexpr int q4_smem() { return (int)sizeof(Q4Shared<D, NT>); }

template <int D, int NT>
cudaError_t q4_attr() {
    const cudaError_t e = raise_smem_limit(k_attn_q4<D, NT>, q4_smem<D, NT>());
    return e == cudaSuccess ? prefer_shared(k_attn_q4<D, NT>) : e;
}

template <int D, int NT>
cudaError_t q4_run(const ace_kv* kv, const AttnArgs& a, cudaStream_t s) {
    const int ctas = kv->num_sms * (NT <= 2 ? 2 : 1);
    k_attn_q4<D, NT><<<ctas, kThreads4, q4_smem<D, NT>(), s>>>(a);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? launch_join(a, ACE_BF16, false, 8 * NT, ctas, s) : e;
}

template <int D>
cudaError_t q4_go(const ace_kv* kv, const AttnArgs& a, cudaStream_t s) {
    const long long rows = (long long)a.max_nodes * a.group;
    if (rows <= 8) return q4_run<D, 1>(kv, a, s);
    if (rows <= 16) return q4_run<D, 2>(kv, a, s);
    return q4_run<D, 4>(kv, a, s);
}

template <int D>
cudaError_t q4_attrs() {
    cudaError_t e = q4_attr<D, 1>();
    if (e == cudaSuccess) e = q4_attr<D, 2>();
    return e == cudaSuccess ? q4_attr<D, 4>() : e;
}

}  // namespace

cudaError_t attn_q4_init(const ace_kv* kv) { return kv->desc.head_dim == 128 ? q4_attrs<128>() : q4_attrs<64>(); }

cudaError_t launch_attn_q4(const ace_kv* kv, const AttnArgs& a, cudaStream_t s) {
    return a.head_dim == 128 ? q4_go<128>(kv, a, s) : q4_go<64>(kv, a, s);
}

}  // namespace ace
