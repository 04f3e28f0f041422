// ace_attn_few.cu — attention for trees of drafted tokens on the tensor cores where a unit has few query rows
// (nodes times query heads a kv head at most 32: decode steps and small trees, bound by the cache's bytes).
// The products are turned round, so that the 128 rows of a tcgen05.mma are positions of the cache and not mostly
// empty query rows:
//   S^T = K Q^T        128 positions x NR rows
//   P^T = 2^(S^T - ref)  a thread holds one position's scores of all rows; its cached row's scale is one factor
//   O^T += V^T P^T     D x NR, V as stored (M-major), P^T through shared memory
// With 128-row blocks of q a tile of 8 live rows costs 16 times the products and exponentials that it needs, and fp8 V has
// to become fp16.
// fp8 caches: both products take the cached codes as they are (kind::f8f6f4). q is split into two e4m3 terms as in
// ace_attn_tc.cu; a weight (at most 2^kLazy) times its V row's factor (at most 2^kVUp), rounded to fp16, into four e5m2
// terms: the upper byte of an fp16 is one, and so on with what is left, times 2^kTermUp a term. A byte takes an fp16's three
// leading bits, or what of them is not below e5m2's least, 2^-16; so what is left fits in fp16 times 2^3 and four terms hold
// all bits down to fp16's least, 2^-24. (Not scaled, all terms end at 2^-16, which weights of 2^-20 of the largest are: beside
// a key that takes nearly all of the weight without a value, thousands of others lose 1 to 100% of theirs.)
// The rows' references lie in shared memory and move only where a score passes them by 2^kLazy (one barrier with an
// "or" a tile). Two groups of four warps take even and odd tiles into accumulators of their own; a group's next
// scores are computed as soon as it has read the last ones.
// Measured (64 users of up to 8192 positions, 332,000 in all, 4 kv heads of 128; 8 query rows a unit): fp8 71 us (4.8 TB/s,
// 0.70 of the copy rate), bf16 113 us (6.0 TB/s, 0.88). 32 rows: 110 and 124. fp8 tiles are half as long to load, and
// then the chain of a tile bounds it: scores, barrier, weights in four terms, hand-over, product (2000 cycles a tile with two
// in turn); of a unit's 40 tiles' time its start and end take 4 more.
#include <cfloat>

#include "ace_attn_tc.cuh"

namespace ace {
namespace {

// A unit's start and end in tiles of the work line (64 users, at most 8192 positions, 8 and 32 fp8 rows a unit: 71 and 109 us
// with 4, 72 and 114 with 2; with joins still in this kernel 73 and 120 with 1, 75 and 122 without).
constexpr int kFewStart = 4;
constexpr int kTermUp = 3;
constexpr int kFewRoom = 4;             // a weight of one is then 2^0 or more in fp16, whose least is 2^-24
constexpr float kNone = -FLT_MAX;       // reference of a row that has seen nothing: any score passes it

template <bool FP8, int D, int NR, int RG>
struct FewCfg {
    static constexpr int ROW = D * (FP8 ? 1 : 2);               // bytes of a cached row
    static constexpr int TILE = 128 * ROW;
    static constexpr int ROWS = NR * RG;                        // of a unit
    static constexpr int Q = NR * D * 2;                        // a group's rows: bf16, or two e4m3 terms
    static constexpr int TERMS = FP8 ? 4 : 1;
    static constexpr int PIECES = TERMS * NR * (FP8 ? 1 : 2) / 16;      // 16-byte pieces of a position's row of P^T
    static constexpr int P = PIECES * 128 * 16;                 // one group's P^T
    static constexpr int NK = D == 64 ? 6 : FP8 ? 5 : 3, NV = !FP8 && D == 128 && RG == 2 ? 2 : NK;
    static constexpr int OFF_K = 0;
    static constexpr int OFF_V = OFF_K + NK * TILE;
    static constexpr int OFF_Q = OFF_V + NV * TILE;             // 1024-byte multiples up to here
    static constexpr int OFF_P = OFF_Q + RG * Q;
    static constexpr int OFF_MISC = OFF_P + 2 * P;
    // fp8: q's terms and the weights' terms lie side by side along N, so that a product reads K and V once; their results
    // are added when they are read
    static constexpr int SN = FP8 ? 2 * NR : NR, ON = TERMS * NR;
    static constexpr uint32_t S = 0, O = 2 * SN, COLS = FP8 ? 16 * NR : 4 * NR;     // TMEM: S^T of both groups, then O^T
    static_assert(2 * (SN + ON) <= (int)COLS && (COLS & (COLS - 1)) == 0, "a power of two");
};

template <bool FP8, int NR, int RG>
struct FewShared : TcShared {
    uint64_t s_free[2];
    float4 kf[FP8 ? kAuxRing : 1][32], vf[FP8 ? kAuxRing : 1][32];
    // by segments of the ring: the next q rows may come while a segment's end still reads these
    float f_row[kSegRing][NR * RG];     // q's scale times the softmax's
    int node[kSegRing][NR * RG];        // row's node of the request
    float ref[2][2][NR];                // [group][turn]
    float top[2][4][NR];                // [group][warp]: maxima of a tile's scores
    float sum[2][4][NR];                // end: sums of weights
    float ref_end[2][NR];
    float2 fac[8][NR];                  // [warp]: factors of both accumulators
    float2 end[FP8 ? NR * RG : 1];      // a row's reference and sum
    int eref_end[2];
};

template <bool FP8, int D, int NR, int RG>
constexpr int few_smem() { return 1024 + FewCfg<FP8, D, NR, RG>::OFF_MISC + (int)sizeof(FewShared<FP8, NR, RG>); }

static_assert(few_smem<false, 128, 16, 1>() <= 232448 && few_smem<true, 128, 16, 1>() <= 232448, "shared memory");
static_assert(few_smem<false, 128, 16, 2>() <= 232448 && few_smem<true, 128, 16, 2>() <= 232448, "shared memory");

// D = A B with A and B in shared memory, operands' descriptors apart.
template <bool F8>
__device__ __forceinline__ void mma_few(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, bool acc) {
    if constexpr (F8)
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %6, 0;\n\tmov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\t"
            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %5, p;\n\t}" ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi),
            "r"(idesc), "r"((uint32_t)acc));
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %6, 0;\n\tmov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;\n\t}" ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi),
            "r"(idesc), "r"((uint32_t)acc));
}

// Instruction descriptor, fp32 accumulator: types and M-/N-majorness of A and B.
constexpr uint32_t few_idesc(int type_a, int type_b, int M, int N, bool a_mn, bool b_mn) {
    return (1u << 4) | ((uint32_t)type_a << 7) | ((uint32_t)type_b << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// N columns of TMEM (4, 8 or 16), not waited for.
template <int N>
__device__ __forceinline__ void tmem_ld(uint32_t taddr, float (&x)[N]) {
    uint32_t* r = reinterpret_cast<uint32_t*>(x);
    if constexpr (N == 16) {
        tmem_ld16(taddr, *reinterpret_cast<uint32_t(*)[16]>(r));
    } else if constexpr (N == 8) {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];" : ACE_R8(r, 0) : "r"(taddr));
    } else {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr));
    }
}

// N columns of an accumulator whose TERMS parts lie STEP columns apart, each 2^kTermUp times the one before.
template <int TERMS, int STEP, int N>
__device__ __forceinline__ void sum_terms(uint32_t taddr, float (&x)[N]) {
    tmem_ld<N>(taddr + (TERMS - 1) * STEP, x);
    tmem_ld_wait();
#pragma unroll 1
    for (int t = TERMS - 2; t >= 0; --t) {
        float y[N];
        tmem_ld<N>(taddr + t * STEP, y);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = fmaf(x[i], 1.f / (1 << kTermUp), y[i]);
    }
}

// Maximum over a warp (NaN counts as -inf): floats in the order of integers.
__device__ __forceinline__ float warp_max(float x) {
    int i = __float_as_int(x == x ? x : -INFINITY);
    i ^= (i >> 31) & 0x7fffffff;
    i = __reduce_max_sync(0xffffffffu, i);
    return __int_as_float(i ^ ((i >> 31) & 0x7fffffff));
}

// Sums of v[r] over a warp by halving: each run of 32 / NR lanes returns the sum of its row.
template <int NR>
__device__ __forceinline__ float row_sums(float (&v)[NR], int lane) {
    int o = 16;
#pragma unroll
    for (int n = NR / 2; n >= 1; n >>= 1, o >>= 1) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float send = lane & o ? v[i] : v[i + n], keep = lane & o ? v[i + n] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
        }
    }
#pragma unroll
    for (; o >= 1; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    return v[0];
}

// Named barriers of the softmax warps; meet_or: whether `x` holds in any thread.
__device__ __forceinline__ void meet(int id, int threads) { asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ bool meet_or(int id, int threads, bool x) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %3, 0;\n\tbarrier.cta.red.or.pred p, %1, %2, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r)
        : "r"(id), "r"(threads), "r"((uint32_t)x)
        : "memory");
    return r != 0;
}

// RG = 1: the two groups take even and odd tiles of all NR rows; RG = 2: each takes half of 2 NR rows of every tile.
template <bool FP8, int D, int NR, int RG>
__global__ void __launch_bounds__(kTcThreads, 1) k_attn_few(const __grid_constant__ TcAttnArgs p) {
    using C = FewCfg<FP8, D, NR, RG>;
    constexpr int NK = C::NK, NV = C::NV;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    using M = FewShared<FP8, NR, RG>;
    M& m = *reinterpret_cast<M*>(smem + C::OFF_MISC);
    const AttnArgs& a = p.a;
    volatile int* abort_flag = &m.abort_flag;
    const int warp = warp_index(), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < NK; ++i) mbar_init(&m.k_full[i], 1), mbar_init(&m.k_empty[i], 1);
        for (int i = 0; i < NV; ++i) mbar_init(&m.v_full[i], 1), mbar_init(&m.v_empty[i], 1), mbar_init(&m.v_ready[i], 4);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&m.s_full[i], 1);
            mbar_init(&m.s_free[i], 4);
            mbar_init(&m.p_ready[i], 4);
            mbar_init(&m.o_done[i], 1);
        }
        mbar_init(&m.q_full, 4);
        mbar_init(&m.q_free, 1);
        mbar_init(&m.drain[0], 1);
        for (int i = 0; i < kSegRing; ++i) {
            mbar_init(&m.seg_full[i], 1);
            mbar_init(&m.seg_empty[i], FP8 ? 15 : 14);  // load, MMA, (scales,) 8 softmax and 4 other warps
        }
        for (int i = 0; i < kAuxRing; ++i) {
            mbar_init(&m.aux_full[i], 1);
            mbar_init(&m.aux_empty[i], 4 * RG);
        }
        m.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&m.tmem)), "r"(C::COLS));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = m.tmem;
    Walk walk{m, a, {}};

    if (warp == 3) {
        role_schedule<C::ROWS, kFewStart>(m, a);
    } else if (warp == 0) {
        role_load<FP8, D, NK, NV>(m, p, smem + C::OFF_K, smem + C::OFF_V, [] { return true; });
    } else if (warp == 2) {
        if constexpr (FP8) role_scales<kFewRoom>(m, a, m.kf, m.vf);
    } else if (warp == 1) {
        // ------------------------------------------------ MMA issuer
        if (elect_one()) {
            Ring rk, rv;
            uint32_t q_phase = 0, p_phase = 0, f_phase = 3;     // bit g: a group's barriers; its S^T is free at first
            const uint32_t q0 = desc_lo(smem_u32(smem + C::OFF_Q), 0), k0 = desc_lo(smem_u32(smem + C::OFF_K), 0);
            const uint32_t v0 = desc_lo(smem_u32(smem + C::OFF_V), kVBlock), p0 = desc_lo(smem_u32(smem + C::OFF_P), 128);
            constexpr uint32_t kHi = C::ROW == 64 ? kRows64 : kRows128;
            constexpr uint32_t kPHi = desc_hi(128 * 16, 0);     // P^T: 16-byte pieces of 8 positions together, pieces 2 KB apart
            bool ok = true;
            while (true) {
                if (!mbar_wait_or_abort(&m.seg_full[walk.seg.i], walk.seg.phase, a.err, abort_flag)) { ok = false; break; }
                if (!m.seg[walk.seg.i].go) break;
                const int items = (m.seg[walk.seg.i].s.tile1 - m.seg[walk.seg.i].s.tile0) * RG;
                mbar_arrive(&m.seg_empty[walk.seg.i]);
                walk.seg.next<kSegRing>();
                if (!mbar_wait_or_abort(&m.q_full, q_phase, a.err, abort_flag)) { ok = false; break; }
                q_phase ^= 1u;
                for (int i = 0; i < items + 2; ++i) {
                    if (i < items) {
                        const bool last = RG == 1 || (i & 1);
                        const uint32_t ql = q0 + (RG == 2 ? (uint32_t)((i & 1) * (C::Q >> 4)) : 0u);
                        // S^T of group i & 1, once the group has read its scores of two tiles ago
                        if (!mbar_wait_or_abort(&m.s_free[i & 1], f_phase >> (i & 1) & 1u, a.err, abort_flag)) { ok = false; break; }
                        f_phase ^= 1u << (i & 1);
                        if ((RG == 1 || !(i & 1)) && !mbar_wait_or_abort(&m.k_full[rk.i], rk.phase, a.err, abort_flag)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t d = tmem + C::S + (uint32_t)((i & 1) * C::SN), kl = k0 + (uint32_t)(rk.i * (C::TILE >> 4));
                        if constexpr (FP8) {
#pragma unroll
                            for (int kk = 0; kk < D / 32; ++kk)
                                mma_few<true>(d, kl + 2 * kk, kHi, ql + 2 * kk, kHi, few_idesc(0, 0, 128, C::SN, false, false), kk > 0);
                        } else {
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk)
                                mma_few<false>(d, kl + (kk >> 2) * (16384 >> 4) + (kk & 3) * 2, kHi, ql + (kk >> 2) * (NR * 128 >> 4) + (kk & 3) * 2,
                                               kHi, few_idesc(1, 1, 128, NR, false, false), kk > 0);
                        }
                        mma_commit(&m.s_full[i & 1]);
                        if (last) {
                            mma_commit(&m.k_empty[rk.i]);
                            rk.next<NK>();
                        }
                        if (i == items - 1) mma_commit(&m.q_free);
                    }
                    if (i > 1) {
                        const int j = i - 2, g = j & 1;
                        if (!mbar_wait_or_abort(&m.p_ready[g], p_phase >> g & 1u, a.err, abort_flag)) { ok = false; break; }
                        p_phase ^= 1u << g;
                        if ((RG == 1 || g == 0) && !mbar_wait_or_abort(&m.v_ready[rv.i], rv.phase, a.err, abort_flag)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t d = tmem + C::O + (uint32_t)(g * C::ON), vl = v0 + (uint32_t)(rv.i * (C::TILE >> 4));
                        const uint32_t pl = p0 + (uint32_t)(g * (C::P >> 4));
                        if constexpr (FP8) {
#pragma unroll
                            for (int kk = 0; kk < 4; ++kk)              // 32 positions a step
                                mma_few<true>(d, vl + kk * (32 * C::ROW >> 4), kHi, pl + kk * 32, kPHi, few_idesc(0, 1, D, C::ON, true, true), j >= 2 || kk > 0);
                        } else {
#pragma unroll
                            for (int kk = 0; kk < 8; ++kk)              // 16 positions a step
                                mma_few<false>(d, vl + kk * 128, kRows128, pl + kk * 16, kPHi, few_idesc(1, 1, D, NR, true, true), j >= 2 || kk > 0);
                        }
                        mma_commit(&m.o_done[g]);
                        if (RG == 1 || g == 1) {
                            mma_commit(&m.v_empty[rv.i]);
                            rv.next<NV>();
                        }
                    }
                }
                if (!ok) break;
            }
            if (!ok) *abort_flag = 1;
            if (*abort_flag) {
                // products in flight read shared memory and write TMEM
                mma_commit(&m.drain[0]);
                mbar_wait(&m.drain[0], 0, a.err);
            }
        }
        __syncwarp();
    } else if (warp >= 12) {
        // ------------------------------------------------ q rows; V tiles with drafted rows
        const int tid = threadIdx.x - 384;
        Ring rv;
        uint32_t q_phase = 1;           // the first segment's q buffer is free
        bool ok = true;
        while (ok && walk.next()) {
            const Segment& s = walk.segment();
            const float q_mul = a.scale_log2 > 0.f ? 1.f : a.scale_log2 < 0.f ? -1.f : 0.f;
            const float f_row0 = a.scale_log2 == 0.f ? 1.f : fabsf(a.scale_log2);
            constexpr int kChunks = D / 8, kStep = 128 / kChunks, kTurns = C::ROWS > kStep ? C::ROWS / kStep : 1;
            uint4 qv[kTurns];
#pragma unroll
            for (int j = 0; j < kTurns; ++j) {
                const int r = j * kStep + tid / kChunks;
                qv[j] = r < s.rows ? load_q(a, s, s.row0 + r, tid % kChunks * 8) : make_uint4(0, 0, 0, 0);
            }
            // the rows are under way while the last products with the segment before read its q
            if (!mbar_wait_warp(&m.q_free, q_phase, a.err, abort_flag)) { ok = false; break; }
            q_phase ^= 1u;
#pragma unroll 1
            for (int j = 0; j < kTurns; ++j) {
                const int r = j * kStep + tid / kChunks, c = tid % kChunks, rr = r % NR;
                unsigned char* tile = smem + C::OFF_Q + r / NR * C::Q;
                uint4 w0 = qv[0];
#pragma unroll
                for (int i = 1; i < kTurns; ++i)
                    if (i == j) w0 = qv[i];
                float f[8];
                Vec16<__nv_bfloat16>::to_float(w0, f);
                if constexpr (FP8) {
                    float amax = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] = finite_or_nan(f[i] * q_mul), amax = fmaxf(amax, fabsf(f[i]));
#pragma unroll
                    for (int o = kChunks / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
                    if (kStep > C::ROWS && r >= C::ROWS) continue;
                    const int byte = e4m3_scale_byte(amax);
                    const float mul = pow2_of_minus_byte(byte);
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = f[2 * i] * mul, y = f[2 * i + 1] * mul;
                        hi[i] = e4m3x2(x, y);
                        const uint32_t h = f16x2_of_e4m3x2(hi[i]);
                        const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&h));
                        lo[i] = e4m3x2(x - back.x, y - back.y);
                    }
                    const int off = raw_v_offset<D>(rr, c >> 1) + (c & 1) * 8;
                    *reinterpret_cast<uint2*>(tile + off) = make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
                    *reinterpret_cast<uint2*>(tile + C::Q / 2 + off) = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
                    if (c == 0) m.f_row[walk.seg.i][r] = fmaxf(f_row0 * pow2_of_byte(byte), 0x1p-126f);   // 0 times a masked -inf is no score
                } else {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i] * q_mul, f[2 * i + 1] * q_mul);
                        w[i] = *reinterpret_cast<const uint32_t*>(&v);
                    }
                    *reinterpret_cast<uint4*>(tile + (c >> 3) * (NR * 128) + rr * 128 + (((c & 7) ^ (rr & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                    if (c == 0) m.f_row[walk.seg.i][r] = f_row0;
                }
                if (c == 0) m.node[walk.seg.i][r] = r < s.rows ? (s.row0 + r) / a.group : 0;
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&m.q_full);
            unsigned long long* bad = m.seg[walk.seg.i].bad;
            for (int t = s.tile0; t < s.tile1; ++t) {
                const int pos0 = t * kTcKeys;
                if (!mbar_wait_warp(&m.v_full[rv.i], rv.phase, a.err, abort_flag)) { ok = false; break; }
                if (pos0 + kTcKeys > s.len) {   // rows that not every node sees, or past the end
                    unsigned char* v = smem + C::OFF_V + rv.i * C::TILE;
                    if constexpr (FP8) clean_codes<D>(v, (tid >> 5) * 8 + (lane & 7), lane >> 3, s, pos0, bad);
                    else clean_bf16<D>(v, tid, s, pos0, bad);
                    fence_async_smem();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&m.v_ready[rv.i]);
                rv.next<NV>();
            }
            if (ok) walk.done();
        }
        if (!ok) *abort_flag = 1;
    } else {
        // ------------------------------------------------ softmax: group g of 4 warps, a thread per position of a tile
        const int g = (warp - 4) >> 2, quad = warp & 3, key = quad * 32 + lane;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const uint32_t s_t = tmem + lanes + C::S + (uint32_t)(g * C::SN), o_t = tmem + lanes + C::O + (uint32_t)(g * C::ON);
        unsigned char* p_out = smem + C::OFF_P + g * C::P + key * 16;
        uint32_t s_phase = 0, o_phase = 0;
        // These warps also meet at hardware barriers, which wait without a limit: so a warp whose bounded wait has run out
        // goes on without waiting (its error is noted, its results are not valid), and all leave together.
        bool dead = false;
        auto wait = [&](uint64_t* bar, uint32_t phase) {
            if (!dead && !mbar_wait_warp(bar, phase, a.err, abort_flag)) dead = true, *abort_flag = 1;
        };
        Ring ra;
        while (true) {
            const bool none = !walk.next();
            if (meet_or(3, 256, none || dead)) break;
            const Segment& s = walk.segment();
            const int tiles = s.tile1 - s.tile0, total = s.len + s.n;
            constexpr int kPer = RG == 2 ? NR : 0;          // first row of group g: g * kPer
            const float* f_row = m.f_row[walk.seg.i] + g * kPer;
            const int* nodes = m.node[walk.seg.i] + g * kPer;
            float l[NR];
#pragma unroll
            for (int r = 0; r < NR; ++r) l[r] = 0.f;
            int eref = 0, turn = 0;     // turn: which half of ref and flag holds
            int mine = 0;
            for (int t = 0; t < tiles; ++t) {
                if (RG == 1 && (t & 1) != g) {
                    if (FP8) ra.next<kAuxRing>();
                    continue;
                }
                const int pos = (s.tile0 + t) * kTcKeys + key;
                float kf = 1.f, vf = 1.f;
                int e_new = eref;
                if (FP8) {
                    wait(&m.aux_full[ra.i], ra.phase);
                    kf = reinterpret_cast<const float*>(m.kf[ra.i])[key];
                    vf = reinterpret_cast<const float*>(m.vf[ra.i])[key];
                    e_new = m.eref[ra.i];
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&m.aux_empty[ra.i]);
                    ra.next<kAuxRing>();
                }
                wait(&m.s_full[g], s_phase);
                s_phase ^= 1u;
                tc_fence_after();
                float x[NR];
                tmem_ld<NR>(s_t, x);
                float lower[FP8 ? NR : 1];
                if constexpr (FP8) tmem_ld<NR>(s_t + NR, lower);
                tmem_ld_wait();
                if constexpr (FP8) {
#pragma unroll
                    for (int r = 0; r < NR; r += 2) unpair(add2(pair(x[r], x[r + 1]), pair(lower[r], lower[r + 1])), x[r], x[r + 1]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&m.s_free[g]);
                // scores in units of the softmax (base 2)
#pragma unroll
                for (int r = 0; r < NR; r += 4) {
                    const float4 f = *reinterpret_cast<const float4*>(f_row + r);
                    unpair(mul2(pair(x[r], x[r + 1]), mul2(pair(f.x, f.y), pair(kf, kf))), x[r], x[r + 1]);
                    unpair(mul2(pair(x[r + 2], x[r + 3]), mul2(pair(f.z, f.w), pair(kf, kf))), x[r + 2], x[r + 3]);
                }
                if (pos >= s.len) {
                    const int nd = pos - s.len;
#pragma unroll
                    for (int r = 0; r < NR; ++r) {
                        const bool sees = pos < total && (sees_word(a, s.node0, s.n, nodes[r], nd >> 6) >> (nd & 63) & 1);
                        if (!sees) x[r] = -INFINITY;
                    }
                }
                bool waited = !mine;
                const float* ref = m.ref[g][turn];
                bool move = !mine || e_new != eref;
                if (mine) {
                    float over = -INFINITY;
#pragma unroll
                    for (int r = 0; r < NR; r += 4) {
                        const float4 f = *reinterpret_cast<const float4*>(ref + r);
                        over = fmaxf(over, fmaxf(fmaxf(x[r] - f.x, x[r + 1] - f.y), fmaxf(x[r + 2] - f.z, x[r + 3] - f.w)));
                    }
                    move = meet_or(1 + g, 128, move || over > (float)kLazy);
                }
                if (move) {
                    // new references: the tile's maxima over the group's positions
#pragma unroll 1
                    for (int r0 = 0; r0 < NR; r0 += 4) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float v = x[i];
#pragma unroll
                            for (int r = 4; r < NR; r += 4)
                                if (r == r0) v = x[r + i];
                            v = warp_max(v);
                            if (lane == 0) m.top[g][quad][r0 + i] = v;
                        }
                    }
                    meet(1 + g, 128);
                    if (mine) {
                        // the group's previous product has left O
                        wait(&m.o_done[g], o_phase);
                        o_phase ^= 1u;
                        waited = true;
                        tc_fence_after();
                    }
                    const float units = FP8 && mine ? (e_new - eref > 126 ? 0.f : pow2_of_byte(127 - (e_new - eref))) : 1.f;
                    float f[NR];
#pragma unroll
                    for (int r = 0; r < NR; ++r) {
                        const float top = fmaxf(fmaxf(m.top[g][0][r], m.top[g][1][r]), fmaxf(m.top[g][2][r], m.top[g][3][r]));
                        const float old = mine ? ref[r] : kNone;
                        const float now = top > old + (float)kLazy ? top : old;
                        f[r] = exp2_approx(old - now);
                        l[r] *= f[r];
                        f[r] *= units;
                        if (key == r) m.ref[g][turn ^ 1][r] = now;
                    }
                    if (mine) {
#pragma unroll 1
                        for (int c = 0; c < C::ON; c += 16) {
                            uint32_t o[16];
                            tmem_ld16(o_t + c, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f[i % NR]);
                            tmem_st16(o_t + c, o);
                        }
                        tmem_st_wait();
                    }
                    turn ^= 1;
                    eref = e_new;
                    meet(1 + g, 128);
                    ref = m.ref[g][turn];
                }
                if (!waited) {
                    wait(&m.o_done[g], o_phase);    // the product has read the P^T before
                    o_phase ^= 1u;
                }
                // weights; a 16-byte piece of P^T holds 16 e5m2 or 8 bf16 values along N = term * NR + row
                uint32_t h[NR / 2];
#pragma unroll
                for (int r = 0; r < NR; r += 4) {
                    const float4 f = *reinterpret_cast<const float4*>(ref + r);
                    float e[4] = {x[r] - f.x, x[r + 1] - f.y, x[r + 2] - f.z, x[r + 3] - f.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) e[j] = exp2_approx(e[j]), l[r + j] += e[j];
                    if constexpr (FP8) {
                        const __half2 p0 = __floats2half2_rn(e[0] * vf, e[1] * vf), p1 = __floats2half2_rn(e[2] * vf, e[3] * vf);
                        h[r / 2] = *reinterpret_cast<const uint32_t*>(&p0);
                        h[r / 2 + 1] = *reinterpret_cast<const uint32_t*>(&p1);
                    } else {
                        const __nv_bfloat162 p0 = __floats2bfloat162_rn(e[0], e[1]), p1 = __floats2bfloat162_rn(e[2], e[3]);
                        h[r / 2] = *reinterpret_cast<const uint32_t*>(&p0);
                        h[r / 2 + 1] = *reinterpret_cast<const uint32_t*>(&p1);
                    }
                }
                if constexpr (FP8) {
                    uint32_t w[NR];             // NR / 4 words a term
#pragma unroll
                    for (int term = 0; term < 4; ++term) {
#pragma unroll
                        for (int i = 0; i < NR / 4; ++i) w[term * (NR / 4) + i] = __byte_perm(h[2 * i], h[2 * i + 1], 0x7531);
                        if (term < 3) {
#pragma unroll
                            for (int i = 0; i < NR / 2; ++i) {
                                const uint32_t top = h[i] & 0xff00ff00u;
                                const __half2 rest = __hmul2(__hsub2(*reinterpret_cast<const __half2*>(&h[i]), *reinterpret_cast<const __half2*>(&top)),
                                                             __float2half2_rn((float)(1 << kTermUp)));
                                h[i] = *reinterpret_cast<const uint32_t*>(&rest);
                            }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < NR; i += 4) *reinterpret_cast<uint4*>(p_out + i / 4 * 2048) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
                } else {
#pragma unroll
                    for (int i = 0; i < NR / 2; i += 4) *reinterpret_cast<uint4*>(p_out + i / 4 * 2048) = make_uint4(h[i], h[i + 1], h[i + 2], h[i + 3]);
                }
                fence_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&m.p_ready[g]);
                ++mine;
            }
            if (mine) {
                wait(&m.o_done[g], o_phase);
                o_phase ^= 1u;
            }
            tc_fence_after();
            // ---------------- the unit's result, or this CTA's part of it: group g finishes half of the rows
            {
                const float sum = row_sums<NR>(l, lane);
                if (lane % (32 / NR) == 0) m.sum[g][quad][lane / (32 / NR)] = sum;
                if (key < NR) m.ref_end[g][key] = mine ? m.ref[g][turn][key] : kNone;
                if (key == 0) m.eref_end[g] = eref;
            }
            if (RG == 1) meet(3, 256);
            else meet(1 + g, 128);
            const bool whole = s.part < 0;
            const unsigned long long* bad = m.seg[walk.seg.i].bad;
            const bool any_bad = bad[0] | bad[1] | bad[2] | bad[3];
            // RG = 1: half of the rows from both accumulators; RG = 2: the group's own rows from its own, half at a time
            constexpr int HALF = NR / 2;
            for (int pass = 0; pass < RG; ++pass) {
                const int c0 = (RG == 1 ? g : pass) * HALF, r0 = g * kPer + c0;        // first column, first row of the unit
                if (lane < HALF) {
                    const int c = c0 + lane, r = r0 + lane, ga = RG == 1 ? 0 : g;
                    const float x = m.ref_end[ga][c], y = RG == 1 ? m.ref_end[1][c] : kNone, top = fmaxf(x, y);
                    float u0 = exp2_approx(x - top), u1 = RG == 1 ? exp2_approx(y - top) : 0.f;
                    float sum = ((m.sum[ga][0][c] + m.sum[ga][1][c]) + (m.sum[ga][2][c] + m.sum[ga][3][c])) * u0;
                    if (RG == 1) sum += ((m.sum[1][0][c] + m.sum[1][1][c]) + (m.sum[1][2][c] + m.sum[1][3][c])) * u1;
                    if (FP8) {
                        u0 *= exp2f((float)(m.eref_end[ga] - kVUp));
                        if (RG == 1) u1 *= exp2f((float)(m.eref_end[1] - kVUp));
                    }
                    if (whole) {
                        const float inv = sum == 0.f ? 0.f : 1.f / sum;
                        u0 *= inv;
                        u1 *= inv;
                    }
                    m.fac[warp - 4][lane] = make_float2(u0, u1);
                    if (FP8 && quad == 0) m.end[r] = make_float2(top, sum);
                    if (quad == 0 && r < s.rows) {
                        const float ref = top == kNone ? -INFINITY : top;
                        const int ur = s.row0 + r, nd = ur / a.group;
                        if (!whole) a.ws.part_ml[(long long)s.part * C::ROWS + r] = make_float2(ref, sum);
                        else if (a.lse) a.lse[(long long)(s.node0 + nd) * a.n_heads + s.head * a.group + ur - nd * a.group] = (ref + log2f(sum)) * 0.69314718055994530942f;
                    }
                }
                __syncwarp();
                // D = 64: an accumulator of 64 rows lies in the first 16 lanes of each warp's 32
                const int d = D == 128 ? key : quad * 16 + lane;
                const bool in = D == 128 || lane < 16;
                const bool both = RG == 1 && tiles > 1;
                float o0[HALF], o1[HALF];
                sum_terms<C::TERMS, NR, HALF>(tmem + lanes + C::O + (uint32_t)((RG == 1 ? 0 : g * C::ON) + c0), o0);
                if (both) sum_terms<C::TERMS, NR, HALF>(tmem + lanes + C::O + (uint32_t)(C::ON + c0), o1);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < HALF; ++i) {
                    const int r = r0 + i;
                    if (r >= s.rows) break;
                    const float2 f = m.fac[warp - 4][i];
                    float o = f.x == 0.f ? 0.f : o0[i] * f.x;
                    if (both && f.y != 0.f) o += o1[i] * f.y;
                    if (in) {
                        const int nd = nodes[r - g * kPer], hq = s.head * a.group + (s.row0 + r) - nd * a.group;
                        if (whole) static_cast<__nv_bfloat16*>(a.out)[((long long)(s.node0 + nd) * a.n_heads + hq) * D + d] = from_f32<__nv_bfloat16>(o);
                        else a.ws.part_o[((long long)s.part * C::ROWS + r) * D + d] = o;
                    }
                }
                if (any_bad && in)
                    for (int r = r0; r < min(r0 + HALF, s.rows); ++r) add_not_finite<FP8, C::ROWS>(a, s, bad, r, d, 1);
                __syncwarp();
            }
            if constexpr (FP8) {
                const unsigned long long* far = m.seg[walk.seg.i].far;
                if (far[0] | far[1] | far[2] | far[3]) {
                    if (RG == 1) meet(3, 256);
                    else meet(1 + g, 128);
                    add_far_rows<C::ROWS, false>(a, s, far, m.end, RG == 1 ? warp - 4 : g * NR + quad, g * kPer + NR, RG == 1 ? 8 : 4);
                }
            }
            tc_fence_before();
            if (RG == 1) meet(3, 256);          // O may be overwritten
            walk.done();
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::COLS));
}

template <bool FP8, int D, int NR, int RG>
cudaError_t few_attr() {
    return raise_smem_limit(k_attn_few<FP8, D, NR, RG>, few_smem<FP8, D, NR, RG>());
}

template <bool FP8, int D>
cudaError_t few_attrs() {
    cudaError_t e = few_attr<FP8, D, 16, 1>();
    if constexpr (FP8)
        if (e == cudaSuccess) e = few_attr<FP8, D, 8, 1>();
    return e == cudaSuccess ? few_attr<FP8, D, 16, 2>() : e;
}

template <bool FP8, int D, int NR, int RG>
cudaError_t few_run(const TcAttnArgs& p, int ctas, cudaStream_t s) {
    k_attn_few<FP8, D, NR, RG><<<ctas, kTcThreads, few_smem<FP8, D, NR, RG>(), s>>>(p);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? launch_join(p.a, ACE_BF16, false, FewCfg<FP8, D, NR, RG>::ROWS, ctas, s) : e;
}

template <bool FP8, int D>
cudaError_t few_go(const TcAttnArgs& p, int ctas, cudaStream_t s) {
    // NR by the rows of the largest tree; 8 are too few for plain caches (M = 128 wants N a multiple of 16, which two terms of
    // an fp8 q make of them), whose larger tiles leave the softmax time enough. 32 rows a thread (and 64 a unit) were
    // slower than ace_attn_tc.cu: their code and registers spill over (a unit of 40 rows 266 us, there 181)
    const long long rows = (long long)p.a.max_nodes * p.a.group;
    if constexpr (FP8)
        if (rows <= 8) return few_run<FP8, D, 8, 1>(p, ctas, s);
    if (rows <= 16) return few_run<FP8, D, 16, 1>(p, ctas, s);
    return few_run<FP8, D, 16, 2>(p, ctas, s);
}

}  // namespace

cudaError_t attn_few_init(const ace_kv* kv) {
    const bool fp8 = kv->desc.format == ACE_KV_FP8;
    if (kv->desc.head_dim == 128) return fp8 ? few_attrs<true, 128>() : few_attrs<false, 128>();
    return fp8 ? few_attrs<true, 64>() : few_attrs<false, 64>();
}

cudaError_t launch_attn_few(const ace_kv* kv, const AttnArgs& a, cudaStream_t s) {
    TcAttnArgs p;
    p.a = a;
    p.k = kv->maps.k;
    p.v = kv->maps.v;
    p.box_rows = a.page_size < kTcKeys ? a.page_size : kTcKeys;
    if (kv->desc.format == ACE_KV_FP8)
        return a.head_dim == 128 ? few_go<true, 128>(p, kv->num_sms, s) : few_go<true, 64>(p, kv->num_sms, s);
    return a.head_dim == 128 ? few_go<false, 128>(p, kv->num_sms, s) : few_go<false, 64>(p, kv->num_sms, s);
}

}  // namespace ace
