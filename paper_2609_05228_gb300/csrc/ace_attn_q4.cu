// ace_attn_q4.cu — attention for trees of drafted tokens over a cache in 4 bits where a unit has few query rows (nodes times query
// heads a kv head at most 16; bf16 activations, head sizes 64 and 128): bound by the cache's bytes, 72 a row of 128.
//   S^T = K Q^T       16 positions x 8 rows a product (m16n8k16); codes are exact in fp16, q too once its row is scaled by a power
//                     of two, so a group's product is exact but for fp32's sums, and its scale is one factor of 16 x 8 sums
//   P^T = 2^(S^T - ref)   two bf16 terms (2^-16 of a weight)
//   O^T += V^T P^T    V's code * scale is exact in bf16 (3 significant bits times 4), whose range spares it a unit; so weights have to be
//                     bf16 as well, and one term (2^-8 of a weight) would be what the output loses most by: 0.0023 of its size against
//                     64 bits, of which the output's own rounding is 0.0017. The second term's products take 3 us of 60 at 8 rows, 8 of 90
//                     at 16.
// At 4 bits a tile of 128 positions is 18 KB and takes HBM 850 cycles of an SM (copy rate), in which its 32768 codes have to become operands: too
// little time for the hand-overs of tcgen05 (scores, softmax, weights and conversion through shared and tensor memory take 2000
// cycles a tile in ace_attn_few.cu, fp8 codes without any conversion). So the codes become operands in the registers of the warp
// that multiplies them (mma.sync; about one operation a code), S^T turns into the second product's operand by movmatrix, and the
// warps of a CTA walk their positions of each tile on their own, with their own running maxima, from rings of cp.async stages; they
// meet at a unit's end only.
// Measured (64 users of up to 8192 positions, 322,000 in all, 4 kv heads of 128): 8 rows a unit 60 us (3.1 TB/s, 0.45 of the copy rate;
// ace_attn_few.cu over an fp8 cache 73), 16 rows 90. With 8 times the positions 4.6 TB/s: the rest is starts and ends of units and the
// joining kernel. They issue 0.54 and 0.47 a cycle and scheduler, with no pipe above 41%: bound by the warps' dependent
// chains (12 warps of 168 registers had the same rate a position).
#include <cfloat>
#include <type_traits>

#include "ace_attn_tc.cuh"

namespace ace {
namespace {

constexpr int kStep = 16;
constexpr float kNone4 = -FLT_MAX;      // reference of a row that has seen nothing: any score passes it

// A warp takes runs of 16 positions, one or two at a time: two where its registers hold them (8 rows), so that the chains of one fill the
// other's waits.
template <int D, int NT>
struct Q4 {
    static constexpr int SUBS = NT == 1 ? 2 : 1, STAGES = NT == 1 ? 2 : 4;
    static constexpr int WARPS = NT == 1 ? 8 : 6, THREADS = 32 * WARPS, CTAS = 2;        // CTAS: an SM
    static constexpr int KEYS = WARPS * SUBS * kStep;          // positions of a tile
    static constexpr int START = NT == 1 ? 2 : 3;               // a unit's start and end in tiles of the work line
    static constexpr int ROW = D / 2, G = D / kGroup4;          // bytes and groups of a row
    static constexpr int CODES = kStep * ROW, SCALES = kStep * G * 2;
    static constexpr int SUB = 2 * CODES + 2 * SCALES, STAGE = SUBS * SUB;
    static constexpr int RING = WARPS * STAGES * STAGE;
    static constexpr int PITCH = D + 4;                         // floats of a row of a warp's O: lanes' stores in distinct banks
    static constexpr int PER = D / 8;                           // dimensions a lane has of a position's V
};

template <int D, int NT>
struct Q4Shared {
    unsigned char ring[Q4<D, NT>::RING];
    float join[Q4<D, NT>::WARPS * 8 * Q4<D, NT>::PITCH];
    uint4 q[NT * Q4<D, NT>::G * 32];        // operand of S^T: [8 rows][group][lane]
    float q8[NT * Q4<D, NT>::G * 8];        // -8 times the sum of a row's q over a group: [8 rows][group][row]
    float f_row[2][NT * 8];             // q's scale times the softmax's, in two factors
    int node[NT * 8];                   // row's node of the request
    float2 ml[Q4<D, NT>::WARPS][NT * 8];          // a warp's reference and sum
    unsigned long long bad[kMaxNodes / 64];     // nodes with a V that is not finite, left out of the products
    Segment seg[3];                     // the one at work, and two ahead
    int go[3];
    RequestTable requests;
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, float c0, float c1,
                                        float c2, float c3) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The transpose of an 8 x 8 matrix of 16-bit values, two of a row a lane.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// A position's scales as V's operands want them, two positions each: s, -136 s, 8 s.
struct Scales {
    uint32_t s, m136, x8;
};

// Elements I and I + 1 (I = 0 or 2) of two positions' four codes (16 bits each) as bf16 times their scales, exactly. Element I:
// 128 + c is c in the last places of 128, and s (128 + c) - 136 s. Element I + 1, four places up: 16 c in bf16's last places is
// 16 c 2^-133 without any exponent, and 8 s (c / 8 - 1); a shift less than to bring it down. LARGE: 136 s or 8 s may be past bf16's
// largest, so s is the last factor.
template <int I, bool LARGE>
__device__ __forceinline__ void bf16_of_codes(uint32_t x, const Scales& k, uint32_t& lower, uint32_t& upper) {
    constexpr uint32_t kMinus136 = 0xc308c308u, kOne = 0x3f803f80u, k2To126 = 0x7e807e80u, kMinus1 = 0xbf80bf80u, kMinus0 = 0x80008000u;
    if constexpr (I == 2) x >>= 8;
    const uint32_t c = and_or(x, 0x000f000fu, 0x43004300u);
    if constexpr (LARGE) {
        lower = fma_bf16x2(fma_bf16x2(c, kOne, kMinus136), k.s, kMinus0);
        upper = fma_bf16x2(fma_bf16x2(and_or(x >> 4, 0x000f000fu, 0x43004300u), kOne, kMinus136), k.s, kMinus0);
    } else {
        lower = fma_bf16x2(c, k.s, k.m136);
        upper = fma_bf16x2(fma_bf16x2(x & 0x00f000f0u, k2To126, kMinus1), k.x8, kMinus0);
    }
}

__device__ __forceinline__ void copy16(void* dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(bytes) : "memory");
}

__device__ __forceinline__ void copy16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
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

// O += V^T P^T of a run: the lane's dimensions PER g .. of positions t, t + 4, t + 8, t + 12, whose codes are w; p and z are the weights'
// upper and lower terms.
template <int D, int NT, bool LARGE>
__device__ __forceinline__ void add_values(const uint32_t (&w)[4][D / 64], const Scales (&k)[2], const uint32_t (&p)[NT][2], const uint32_t (&z)[NT][2], float (&o)[D / 16][NT][4]) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint32_t sel = half ? 0x7632u : 0x5410u;
            const uint32_t x0 = __byte_perm(w[0][i], w[1][i], sel), x1 = __byte_perm(w[2][i], w[3][i], sel);
            uint32_t a[2][4];
            bf16_of_codes<0, LARGE>(x0, k[0], a[0][0], a[0][1]);
            bf16_of_codes<0, LARGE>(x1, k[1], a[0][2], a[0][3]);
            bf16_of_codes<2, LARGE>(x0, k[0], a[1][0], a[1][1]);
            bf16_of_codes<2, LARGE>(x1, k[1], a[1][2], a[1][3]);
            // two tiles' products in turn, as those of one add to the same sums (one tile after the other: 59.4 for 57.4 us in a row of calls)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int n = 0; n < NT; ++n) mma_bf16(o[4 * i + 2 * half + j][n], a[j], p[n][0], p[n][1]);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int n = 0; n < NT; ++n) mma_bf16(o[4 * i + 2 * half + j][n], a[j], z[n][0], z[n][1]);
        }
    }
}

// Rows r = 8 n + 0 .. 7 of a unit, n < NT. Lane (g, t) = (lane / 4, lane % 4) holds rows 2 t and 2 t + 1 of each eight: scores of positions
// place(g) and place(g) + 8, and dimensions PER g .. PER g + PER - 1 of O, tile j of it dimensions 2 j and 2 j + 1 of those.
template <int D, int NT>
__global__ void __launch_bounds__(Q4<D, NT>::THREADS, Q4<D, NT>::CTAS) k_attn_q4(const __grid_constant__ AttnArgs a) {
    using C = Q4<D, NT>;
    constexpr int kSub = C::SUBS, kStages = C::STAGES, kKeys4 = C::KEYS, kStart4 = C::START, kWarps = C::WARPS, kThreads4 = C::THREADS;
    constexpr int ROWS = 8 * NT, TJ = D / 16, G = C::G;
    extern __shared__ __align__(128) unsigned char smem_raw[];
    Q4Shared<D, NT>& m = *reinterpret_cast<Q4Shared<D, NT>*>(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    unsigned char* ring = m.ring + warp * (kStages * C::STAGE);
    // position of row i of the product: those of a V operand's halves lie 4 apart
    const int place = (g >> 1) + 4 * (g & 1);

    // where the lane's operands lie in a run: the codes that it has of K's groups, its half of V's (the other half is turned)
    int k_at[G];
#pragma unroll
    for (int b = 0; b < G; ++b) k_at[b] = chunk_at<D>(place, b) + t * 4;
    const int v0 = C::CODES + (D == 128 ? chunk_at<D>(t, g >> 1) + (g & 1) * 8 : chunk_at<D>(t, g >> 2) + (g & 3) * 4);
    const int v_at[2] = {v0, v0 ^ (D == 128 ? 64 : 16)};
    const int k_scale_at = 2 * C::CODES + place * (2 * G), v_scale_at = 2 * C::CODES + C::SCALES + t * (2 * G) + g * G / 8 * 2;

    Cursor cur{};
    if (tid == 0) note_none(a);
    bool more = cursor_init_block<ROWS, kKeys4, kStart4, kThreads4>(a, blockIdx.x, gridDim.x, cur, m.requests);
    if (!more) return;
    // by warp 0: the segment after, into slot i
    auto schedule = [&](int i) {
        if (warp == 0) {
            Segment s{};
            more = more && cursor_next<ROWS, kKeys4, kStart4>(a, blockIdx.x, cur, s,
                                                              [&](int b) { return b < kTabled ? m.requests.request[b] : request_of(a, b); });
            if (lane == 0) {
                m.go[i] = more;
                if (more) {
                    m.seg[i] = s;
                    note_unit(a, s);
                }
            }
        }
    };
    // where the lane's 16-byte words of a run go, and its operands lie
    constexpr int PER_ROW = C::ROW / 16, SCALE_CHUNKS = C::SCALES / 16;
    const int to = chunk_at<D>(lane / PER_ROW, lane % PER_ROW);
    const int page_rows = a.kv_heads * a.page_size;
    const unsigned char *k_from = nullptr, *v_from = nullptr, *scale_from = nullptr;        // the lane's words of the head's first row
    // a warp's runs of a tile, each of one page; what does not exist is zeros
    auto load = [&](const Segment& s, int tile, int stage, const Entries<kSub>& entries) {
        if (tile < s.tile1) {
#pragma unroll
            for (int u = 0; u < kSub; ++u) {
                const int pos = tile * kKeys4 + (warp * kSub + u) * kStep, left = s.len + s.n - pos;
                unsigned char* at = ring + stage * C::STAGE + u * C::SUB;
                const int page = entries.page(s, tile, u), row = page * page_rows + (pos & (a.page_size - 1));
                if (__builtin_expect(left >= kStep && page >= 0, 1)) {
                    const unsigned char *k = k_from + (long long)row * C::ROW, *v = v_from + (long long)row * C::ROW;
#pragma unroll
                    for (int i = 0; i < C::CODES / 512; ++i) {      // 8 rows of 64 bytes further on lie as far in the stage
                        copy16(at + to + i * 512, k + i * 512);
                        copy16(at + C::CODES + to + i * 512, v + i * 512);
                    }
                    if (lane < 2 * SCALE_CHUNKS) copy16(at + 2 * C::CODES + lane * 16, scale_from + (long long)row * (2 * G));
                } else {
                    const int have = page < 0 ? 0 : left;
                    const long long from = have <= 0 ? 0 : row;
#pragma unroll
                    for (int i = 0; i < C::CODES / 512; ++i) {
                        const int bytes = lane / PER_ROW + 8 * i < have ? 16 : 0;
                        copy16(at + to + i * 512, k_from + from * C::ROW + i * 512, bytes);
                        copy16(at + C::CODES + to + i * 512, v_from + from * C::ROW + i * 512, bytes);
                    }
                    if (lane < 2 * SCALE_CHUNKS)
                        copy16(at + 2 * C::CODES + lane * 16, scale_from + from * (2 * G), min(max(have * (2 * G) - lane % SCALE_CHUNKS * 16, 0), 16));
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // a segment's first stages
    Entries<kSub> entries;
    auto first_of = [&](int tile) { return tile * kKeys4 + warp * (kSub * kStep); };
    auto begin = [&](const Segment& s) {
        const long long head = (long long)s.head * a.page_size;
        k_from = static_cast<const unsigned char*>(a.k_pool) + head * C::ROW + lane * 16;
        v_from = static_cast<const unsigned char*>(a.v_pool) + head * C::ROW + lane * 16;
        scale_from = (lane < SCALE_CHUNKS ? a.k_scale : a.v_scale) + head * (2 * G) + lane % SCALE_CHUNKS * 16;
        entries.begin(a, s, first_of);
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i) load(s, s.tile0 + i, i, entries);
    };
    // q's operand, PER_Q lanes a row with 8 elements each; elements of a row in units of 2^(e - 14), where its largest is below
    // 2^(e + 1): all bits of elements down to 2^-27 of it. Those that meet codes 16 times too large are a 16th.
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
            const int e = max((int)(__float_as_uint(amax) >> 23), 15);
            const float mul = __uint_as_float((uint32_t)(268 - e) << 23);
            uint32_t w[4];
            float sum = 0.f;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float up = x & 1 ? mul * 0.0625f : mul;
                const __half2 h = __floats2half2_rn(f[x] * up, f[x + 4] * up);
                w[x] = *reinterpret_cast<const uint32_t*>(&h);
                const float2 back = __half22float2(h);
                sum += (back.x + back.y) * (x & 1 ? 16.f : 1.f);
            }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (r >= ROWS) continue;
            if (c % 4 == 0) m.q8[((r >> 3) * G + c / 4) * 8 + (r & 7)] = sum * (-8.f * 0x1p-24f);
            m.q[((r >> 3) * G + c / 4) * 32 + (r & 7) * 4 + c % 4] = make_uint4(w[0], w[1], w[2], w[3]);
            if (c == 0) {
                // scale_log2 2^(e - 117) is infinite from q's of 2^121 on, where scores need not be: it is halved by exponents, so
                // that what one factor gives lies between the sum and the score. (Past 2^250 no score but 0 is finite.)
                const int k = min(max((int)(__float_as_uint(a.scale_log2) >> 23 & 255u), 1), 253) - 127, both = min(k + e - 117, 250), half = both >> 1;
                m.f_row[0][r] = a.scale_log2 * pow2_of_byte(127 - k) * pow2_of_byte(127 + half);
                m.f_row[1][r] = pow2_of_byte(127 + both - half);
                m.node[r] = r < s.rows ? (s.row0 + r) / a.group : 0;
            }
        }
        if (tid < kMaxNodes / 64) m.bad[tid] = 0;
    };

    schedule(0);
    __syncthreads();
    float o[TJ][NT][4], ref[NT][2], l[NT][2];
    // Round by round: the segment before (`turn`) is finished while the loads of the one at hand (`next`) are under way. One copy of the
    // code for the first segment and the later ones: code that runs for the first time waits for its instructions.
    int turn = 2, next = 0;
    for (bool first = true;; first = false) {
        if (!first) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) l[n][r] += __shfl_xor_sync(0xffffffffu, l[n][r], w);
                    if (g == 0) m.ml[warp][8 * n + 2 * t + r] = make_float2(ref[n][r], l[n][r]);
                }
            __syncthreads();            // all have read q
        }
        const bool go = m.go[next];
        uint4 raw[Q_TURNS];
        if (go) {
            begin(m.seg[next]);
            q_load(m.seg[next], raw);
        }
        if (!first) {
            // ---------------- the unit's result, or this CTA's part of it
            const Segment& s = m.seg[turn];
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
        }
        if (!go) break;
        schedule(next == 2 ? 0 : next + 1);
        if (!first) __syncthreads();    // bad and q are free
        q_store(m.seg[next], raw);
        __syncthreads();
        turn = next;
        next = next == 2 ? 0 : next + 1;
        const Segment& s = m.seg[turn];
        const int len = s.len, total = s.len + s.n, tile1 = s.tile1;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int j = 0; j < TJ; ++j) o[j][n][0] = o[j][n][1] = o[j][n][2] = o[j][n][3] = 0.f;
            ref[n][0] = ref[n][1] = kNone4;
            l[n][0] = l[n][1] = 0.f;
        }
        int stage = 0;
        for (int tile = s.tile0; tile < tile1; ++tile) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
            __syncwarp();               // all lanes' copies are there, and the stage before is read
            entries.move_to(a, s, tile + kStages - 1, first_of);
            load(s, tile + kStages - 1, stage == 0 ? kStages - 1 : stage - 1, entries);
            const unsigned char* at = ring + stage * C::STAGE;
            stage = stage == kStages - 1 ? 0 : stage + 1;
            const int pos = tile * kKeys4 + warp * (kSub * kStep);
            if (pos >= total) continue;
            // ---- scores
            float x[kSub][NT][4];
            {
                uint64_t x01[kSub][NT], x23[kSub][NT];
                uint32_t k0[kSub][G / 2], k1[kSub][G / 2];      // scales of the two positions
#pragma unroll
                for (int u = 0; u < kSub; ++u) {
                    const unsigned char* from = at + u * C::SUB + k_scale_at;
                    if constexpr (G == 4) {
                        const uint2 y = *reinterpret_cast<const uint2*>(from), w = *reinterpret_cast<const uint2*>(from + 64);
                        k0[u][0] = y.x, k0[u][1] = y.y, k1[u][0] = w.x, k1[u][1] = w.y;
                    } else {
                        k0[u][0] = *reinterpret_cast<const uint32_t*>(from);
                        k1[u][0] = *reinterpret_cast<const uint32_t*>(from + 32);
                    }
                }
#pragma unroll
                for (int b = 0; b < G; ++b) {
                    uint32_t w0[kSub], w1[kSub];
#pragma unroll
                    for (int u = 0; u < kSub; ++u) {            // 8 positions further on lie 512 (256) bytes further on
                        w0[u] = *reinterpret_cast<const uint32_t*>(at + u * C::SUB + k_at[b]);
                        w1[u] = *reinterpret_cast<const uint32_t*>(at + u * C::SUB + k_at[b] + 8 * C::ROW);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const uint4 q = m.q[(n * G + b) * 32 + lane];
                        const float2 less = *reinterpret_cast<const float2*>(&m.q8[(n * G + b) * 8 + 2 * t]);
#pragma unroll
                        for (int u = 0; u < kSub; ++u) {
                            // elements 0 and 4, 1 and 5, .. in place are codes times 2^-24 and 16 times that
                            const uint32_t y0 = w0[u] >> 8, y1 = w1[u] >> 8;
                            const float f0 = __uint_as_float(b & 1 ? k0[u][b / 2] & 0xffff0000u : k0[u][b / 2] << 16);
                            const float f1 = __uint_as_float(b & 1 ? k1[u][b / 2] & 0xffff0000u : k1[u][b / 2] << 16);
                            float c[4], d[4];
                            mma_f16(c, w0[u] & 0x000f000fu, w1[u] & 0x000f000fu, w0[u] & 0x00f000f0u, w1[u] & 0x00f000f0u, q.x, q.y, less.x, less.y, less.x, less.y);
                            mma_f16(d, y0 & 0x000f000fu, y1 & 0x000f000fu, y0 & 0x00f000f0u, y1 & 0x00f000f0u, q.z, q.w, c[0], c[1], c[2], c[3]);
                            x01[u][n] = b == 0 ? mul2(pair(d[0], d[1]), pair(f0, f0)) : fma2(pair(d[0], d[1]), pair(f0, f0), x01[u][n]);
                            x23[u][n] = b == 0 ? mul2(pair(d[2], d[3]), pair(f1, f1)) : fma2(pair(d[2], d[3]), pair(f1, f1), x23[u][n]);
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float2 f = *reinterpret_cast<const float2*>(&m.f_row[0][8 * n + 2 * t]), z = *reinterpret_cast<const float2*>(&m.f_row[1][8 * n + 2 * t]);
#pragma unroll
                    for (int u = 0; u < kSub; ++u) {
                        unpair(mul2(mul2(x01[u][n], pair(f.x, f.y)), pair(z.x, z.y)), x[u][n][0], x[u][n][1]);
                        unpair(mul2(mul2(x23[u][n], pair(f.x, f.y)), pair(z.x, z.y)), x[u][n][2], x[u][n][3]);
                    }
                }
            }
            const bool drafted = pos + kSub * kStep > len;      // rows that not every node sees, or past the end
            if (__builtin_expect(drafted, 0)) {
#pragma unroll
                for (int i = 0; i < 2 * kSub; ++i) {
                    const int nd = pos + place + 8 * i - len;
                    if (nd < 0) continue;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const bool sees = nd < total - len && (sees_word(a, s.node0, total - len, m.node[8 * n + 2 * t + r], nd >> 6) >> (nd & 63) & 1);
                            if (!sees) x[i / 2][n][i % 2 * 2 + r] = -INFINITY;
                        }
                }
            }
            // ---- V's scales; 0 times an infinity or a NaN is no zero
            Scales k[kSub][2];
            uint32_t fine = 0;
#pragma unroll
            for (int u = 0; u < kSub; ++u)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const unsigned char* from = at + u * C::SUB + v_scale_at + 16 * G * i;
                    uint32_t lo = *reinterpret_cast<const uint16_t*>(from), hi = *reinterpret_cast<const uint16_t*>(from + 8 * G);
                    if (__builtin_expect(drafted, 0)) {
                        // what is not finite in a drafted row is for those that see it: noted, and left out of the products
                        const int nd = pos + u * kStep + t + 8 * i - len;
                        if (nd >= 0 && (lo & 0x7f80u) == 0x7f80u) lo = 0, atomicOr(&m.bad[nd >> 6], 1ull << (nd & 63));
                        if (nd + 4 >= 0 && (hi & 0x7f80u) == 0x7f80u) hi = 0, atomicOr(&m.bad[(nd + 4) >> 6], 1ull << ((nd + 4) & 63));
                    }
                    k[u][i].s = lo | hi << 16;
                    k[u][i].m136 = fma_bf16x2(k[u][i].s, 0xc308c308u, 0x80008000u);
                    k[u][i].x8 = fma_bf16x2(k[u][i].s, 0x41004100u, 0x80008000u);
                    fine = fma_bf16x2(k[u][i].m136, 0u, fine);
                }
            const bool large = (fine & 0x7fff7fffu) != 0;
            // ---- references: a row's moves where a score is 2^kLazy above it
            float over = -INFINITY;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float top = fmaxf(x[0][n][r], x[0][n][2 + r]);
#pragma unroll
                    for (int u = 1; u < kSub; ++u) top = fmaxf(top, fmaxf(x[u][n][r], x[u][n][2 + r]));
                    over = fmaxf(over, top - ref[n][r]);
                }
            bool any_large = false;
            if (__builtin_expect(__any_sync(0xffffffffu, over > (float)kLazy || large), 0)) {
                any_large = __any_sync(0xffffffffu, large);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float top = fmaxf(x[0][n][r], x[0][n][2 + r]);
#pragma unroll
                        for (int u = 1; u < kSub; ++u) top = fmaxf(top, fmaxf(x[u][n][r], x[u][n][2 + r]));
#pragma unroll
                        for (int w = 4; w < 32; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
                        const float now = top > ref[n][r] + (float)kLazy ? top : ref[n][r], f = exp2_approx(ref[n][r] - now);
                        ref[n][r] = now;
                        l[n][r] *= f;
#pragma unroll
                        for (int j = 0; j < TJ; ++j) o[j][n][r] *= f, o[j][n][2 + r] *= f;
                    }
            }
            // ---- weights and values
            auto finish = [&](auto is_large) {
#pragma unroll
                for (int u = 0; u < kSub; ++u) {
                    uint32_t p[NT][2], lower[NT][2], w[4][D / 64];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const unsigned char* from = at + u * C::SUB + (i & 1 ? v_at[1] : v_at[0]) + i * 4 * C::ROW;
                        if constexpr (D == 128) {
                            const uint2 y = *reinterpret_cast<const uint2*>(from);
                            w[i][0] = y.x, w[i][1] = y.y;
                        } else {
                            w[i][0] = *reinterpret_cast<const uint32_t*>(from);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float e[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) e[i] = exp2_approx(x[u][n][i] - ref[n][i & 1]);
                        l[n][0] += e[0] + e[2];
                        l[n][1] += e[1] + e[3];
                        uint32_t up[2], low[2];
                        two_terms(e[0], e[1], up[0], low[0]);
                        two_terms(e[2], e[3], up[1], low[1]);
#pragma unroll
                        for (int i = 0; i < 2; ++i) p[n][i] = transposed(up[i]), lower[n][i] = transposed(low[i]);
                    }
                    add_values<D, NT, decltype(is_large)::value>(w, k[u], p, lower, o);
                }
            };
            if (__builtin_expect(any_large, 0)) finish(std::true_type{});
            else finish(std::false_type{});
        }
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
    const int ctas = kv->num_sms * Q4<D, NT>::CTAS;
    k_attn_q4<D, NT><<<ctas, Q4<D, NT>::THREADS, q4_smem<D, NT>(), s>>>(a);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? launch_join(a, ACE_BF16, false, 8 * NT, ctas, s) : e;
}

template <int D>
cudaError_t q4_go(const ace_kv* kv, const AttnArgs& a, cudaStream_t s) {
    const long long rows = (long long)a.max_nodes * a.group;
    if (rows <= 8) return q4_run<D, 1>(kv, a, s);
    return q4_run<D, 2>(kv, a, s);
}

template <int D>
cudaError_t q4_attrs() {
    const cudaError_t e = q4_attr<D, 1>();
    return e == cudaSuccess ? q4_attr<D, 2>() : e;
}

}  // namespace

cudaError_t attn_q4_init(const ace_kv* kv) { return kv->desc.head_dim == 128 ? q4_attrs<128>() : q4_attrs<64>(); }

cudaError_t launch_attn_q4(const ace_kv* kv, const AttnArgs& a, cudaStream_t s) {
    return a.head_dim == 128 ? q4_go<128>(kv, a, s) : q4_go<64>(kv, a, s);
}

}  // namespace ace
