// ace_attn_tc.cu — attention for trees of drafted tokens on the tensor cores (bf16 activations, head sizes 64 and
// 128, plain and fp8 caches): one pass over the cached rows with a softmax's running maximum and sum, the keys of a request
// split over CTAs by the work line of ace_kv_device.cuh.
//
// A unit is one request, kv head and block of query rows r = node * G + g (G query heads share a kv head, so
// they share its cached rows too). A CTA walks key tiles of 128 positions:
//   S = Q K^T              tcgen05.mma, 128 x 64 fp32 in TMEM an item
//   P = 2^(S - m), l += P  softmax warps, a thread per row; P goes back to TMEM as bf16 / fp16
//   O += P V               tcgen05.mma, A = P from TMEM, B = V as stored (its rows are K indices)
// In items of 64 positions, two groups of four softmax warps and two accumulators: with RT = 2 a group has a block of 128
// rows, and both halves of each tile; with RT = 1 both have the same rows, and a half of each tile, joined at the end. A
// group has two buffers of S, so that the products of one item run beside the softmax of the next, and a thread of its own
// that issues them: an item's twelve products, waits and hand-overs take it 1050 cycles, as long as the softmax. (With one
// such thread for both groups a chain of 5 nodes over 262144 positions took 154 us and not 161, but 64 users' 40 rows 132
// and not 123, bf16 168 and not 130.)
// fp8 caches: K's codes are the B operand as stored (kind::f8f6f4), against q split into two e4m3 terms, which
// hold 8 significant bits, all of a bf16 q (elements 2^-10 and more below the row's largest lose their last bits, a
// 2^-18 of it); a code's scale multiplies its column of S. V's codes become fp16 in shared memory with their scales, in units
// of 2^eref, a power of two above the scales so far (ace_attn_tc.cuh: Reference): exact but for rows whose scale is 2^-20 of the
// largest and less, whose codes' last bits fall under fp16's least.
// P is rounded to bf16 (2^-9 of a weight; plain caches) or fp16 (2^-12), as the products need; sums, maxima and O are fp32.
// Measured: 8 users of up to 16384 positions, 128 nodes of 64 heads (8 kv heads of 128), bf16: 304 us, 850 TFLOP/s. 64 users
// of up to 8192, 4 kv heads of 128: 64 rows a unit 114 us fp8, 128 bf16; 128 rows 139 and 135; 192 rows 213 and 162. Bound by
// the chain scores, softmax, product of two groups that share one tensor pipe (an item's products alone take 625 cycles:
// N = 64 makes scores read the q rows from shared memory at its full rate), fp8 also by the conversion of V.
#include <cudaTypedefs.h>

#include "ace_attn_tc.cuh"

namespace ace {
namespace {

constexpr int kHalf = 64;               // positions of an item
// A unit's start and end in tiles of the work line (64 users, at most 8192 positions, 64 and 128 fp8 rows a unit: 117 and 144
// us with 7, 119 and 148 with 4, before they took 114 and 139; with joins still in this kernel 121 and 159 with 4, 137 and 172 without).
constexpr int kTcStart = 7;
constexpr int kTcRoom = 16;             // V in fp16 is then off by 2^-20 of the largest that all rows see, or exact

template <bool FP8, int D, int RT, int CP>
struct Cfg {
    static constexpr int ROWS = 128 * RT;
    static constexpr int Q = 256 * D;                   // bytes of a row block: bf16, or two e4m3 terms
    static constexpr int TILE = 128 * D * (FP8 ? 1 : 2);
    static constexpr int CONV = FP8 ? 128 * D * 2 : 0;  // V as fp16
    static constexpr int NC = FP8 ? 2 : 0;
    static constexpr int NK = D == 64 ? (FP8 ? 6 : 4) : 3;
    static constexpr int NV = D == 64 ? (FP8 ? 6 : 4) : FP8 && RT == 1 ? 3 : 2;
    static constexpr int OFF_K = RT * Q;
    static constexpr int OFF_V = OFF_K + NK * TILE;
    static constexpr int OFF_C = OFF_V + NV * TILE;
    static constexpr int OFF_MERGE = OFF_C + NC * CONV;     // CP > 1: 16 dimensions of each group's 128 rows of O
    static constexpr int OFF_MISC = OFF_MERGE + (CP > 1 ? 2 * 128 * 16 * 4 : 0);
};

template <bool FP8, int RT>
struct Misc : TcShared {
    uint64_t c_empty[2], soft, group[2];
    float2 ml[RT == 1 || FP8 ? 256 : 1];        // RT = 1: both halves' running maximum and sum; else a row's
    int eref1[RT == 1 ? 2 : 1];
    float q_scale[kSegRing][FP8 ? 128 * RT : 1];        // by segments of the ring: softmax may be behind
    float4 kf[FP8 ? kAuxRing : 1][32];          // 128 factors a tile
    uint2 vf[FP8 ? kAuxRing : 1][32];           // the same as fp16
};

template <bool FP8, int D, int RT, int CP>
constexpr int tc_smem() { return 1024 + Cfg<FP8, D, RT, CP>::OFF_MISC + (int)sizeof(Misc<FP8, RT>); }

static_assert(tc_smem<false, 128, 2, 1>() <= 232448 && tc_smem<false, 128, 1, 2>() <= 232448, "shared memory");
static_assert(tc_smem<true, 128, 2, 1>() <= 232448 && tc_smem<true, 128, 1, 2>() <= 232448, "shared memory");
static_assert(tc_smem<false, 64, 2, 1>() <= 232448 && tc_smem<true, 64, 1, 2>() <= 232448, "shared memory");

// An item's 64 scores stay in registers, and its code is as long as the instruction cache bears beside the other roles': with
// 128 scores unrolled, and the conversion, warps of different roles stalled on fetches (no_instruction 2.7 an issue, now 0.6
// to 0.9); read twice from TMEM, 32 at a time, they took twice the cycles of the second pass.

// 32 of a row's scores with fp8 rows' scales, and -inf where the row does not see the position.
template <bool FP8>
__device__ __forceinline__ void finish_scores(float* x, const float4* kf, bool masked, uint32_t see) {
    if (FP8) {
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
            const float4 f = kf[i / 4];
            unpair(mul2(pair(x[i], x[i + 1]), pair(f.x, f.y)), x[i], x[i + 1]);
            unpair(mul2(pair(x[i + 2], x[i + 3]), pair(f.z, f.w)), x[i + 2], x[i + 3]);
        }
    }
    if (masked) {
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = see >> i & 1 ? x[i] : -INFINITY;
    }
}

__device__ __forceinline__ float max32(const float* x) {
    float top[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
    for (int i = 4; i < 28; i += 8) {
#pragma unroll
        for (int j = 0; j < 4; ++j) top[j] = fmaxf(top[j], fmaxf(x[i + j], x[i + 4 + j]));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) top[j] = fmaxf(top[j], x[28 + j]);
    return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
}

// 32 weights 2^(x f + shift) to TMEM; returns their sum.
template <bool FP8>
__device__ __forceinline__ float store_weights(uint32_t p_t, const float* x, float f, float shift) {
    const uint64_t f2 = pair(f, f), shift2 = pair(shift, shift);
    uint64_t sum[2] = {0ull, 0ull};
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
        float e[4];
        unpair(fma2(pair(x[i], x[i + 1]), f2, shift2), e[0], e[1]);
        unpair(fma2(pair(x[i + 2], x[i + 3]), f2, shift2), e[2], e[3]);
#pragma unroll
        for (int j = 0; j < 4; ++j) e[j] = exp2_approx(e[j]);
        sum[0] = add2(sum[0], pair(e[0], e[1]));
        sum[1] = add2(sum[1], pair(e[2], e[3]));
        if constexpr (FP8) {
            const __half2 p0 = __floats2half2_rn(e[0], e[1]), p1 = __floats2half2_rn(e[2], e[3]);
            w[i / 2] = *reinterpret_cast<const uint32_t*>(&p0);
            w[i / 2 + 1] = *reinterpret_cast<const uint32_t*>(&p1);
        } else {
            const __nv_bfloat162 p0 = __floats2bfloat162_rn(e[0], e[1]), p1 = __floats2bfloat162_rn(e[2], e[3]);
            w[i / 2] = *reinterpret_cast<const uint32_t*>(&p0);
            w[i / 2 + 1] = *reinterpret_cast<const uint32_t*>(&p1);
        }
    }
    tmem_st16(p_t, w);
    float a, b, c, d;
    unpair(sum[0], a, b);
    unpair(sum[1], c, d);
    return (a + b) + (c + d);
}

// A thread's row of the running softmax.
struct RowState {
    float ref, l, o_mul;                // reference, sum, what O has to be multiplied with
};

// One item of a row: N scores from column `col` on become weights, over the scores that are read already; the row's other
// columns of P (of the item's kHalf) are zero.
template <bool FP8, int N>
__device__ __forceinline__ void softmax_item(const AttnArgs& a, const Segment& s, uint32_t s_t, int col, const float4* kf, bool drafted,
                                             int node, int pos0, float f_row, bool first, RowState& st) {
    float x[N];
#pragma unroll
    for (int c = 0; c < N; c += 32) tmem_ld32(s_t + col + c, *reinterpret_cast<uint32_t(*)[32]>(x + c));
    tmem_ld_wait();
    float top = -INFINITY;
#pragma unroll
    for (int c = 0; c < N; c += 32) {
        finish_scores<FP8>(x + c, kf + (col + c) / 4, drafted, drafted ? sees32(a, s, node, pos0 + col + c) : 0u);
        top = fmaxf(top, max32(x + c));
    }
    top = top == -INFINITY ? top : top * f_row;
    constexpr float kUp = FP8 ? (float)kPUp : 0.f;
    if (top > st.ref + (float)kLazy + kUp || st.ref == -INFINITY) {
        const float ref = top - kUp;
        // (what it has summed before its first score is zero)
        const float f = st.ref == -INFINITY ? 1.f : exp2_approx(st.ref - ref);
        st.ref = ref;
        st.l *= f;
        if (!first) st.o_mul *= f;
    }
    const float shift = st.ref == -INFINITY ? 0.f : -st.ref;
    // x f + shift in one operation is off by what `ref` lost in its rounding, nothing below 2^20; past that x f is rounded
    // too (by rows: what a row gets must not depend on its neighbours)
    const bool large = fabsf(shift) > 0x1p20f, any_large = __any_sync(0xffffffffu, large);
    const float before = large ? f_row : 1.f, f = large ? 1.f : f_row;
    if (any_large) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= before;
    }
#pragma unroll
    for (int c = 0; c < N; c += 32) st.l += store_weights<FP8>(s_t + (col + c) / 2, x + c, f, shift);
    if constexpr (N < kHalf) {
        const uint32_t zero[16] = {};
        tmem_st16(s_t + 16 - col / 2, zero);
    }
    tmem_st_wait();
}

__device__ __forceinline__ uint32_t bf16x2(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Two codes as fp16 times `f`.
__device__ __forceinline__ uint32_t f16x2_scaled(uint32_t codes, __half2 f) {
    const uint32_t y = f16x2_of_e4m3x2(codes);
    const __half2 z = __hmul2(*reinterpret_cast<const __half2*>(&y), f);
    return *reinterpret_cast<const uint32_t*>(&z);
}

// CP = 2 (at most 64 rows): the block holds them twice, 64 lanes apart, and each copy's warps take half of a tile's
// columns: the tile's softmax takes half the time, and the copies' O are added at the end.
template <bool FP8, int D, int RT, int CP>
__global__ void __launch_bounds__(kTcThreads, 1) k_attn_tc(const __grid_constant__ TcAttnArgs p) {
    using C = Cfg<FP8, D, RT, CP>;
    constexpr int ROWS = C::ROWS, NK = C::NK, NV = C::NV, NC = C::NC;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    using M = Misc<FP8, RT>;
    M& m = *reinterpret_cast<M*>(smem + C::OFF_MISC);
    const AttnArgs& a = p.a;
    volatile int* abort_flag = &m.abort_flag;
    const int warp = warp_index(), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < NK; ++i) mbar_init(&m.k_full[i], 1), mbar_init(&m.k_empty[i], 2);
        for (int i = 0; i < NV; ++i) mbar_init(&m.v_full[i], 1), mbar_init(&m.v_empty[i], FP8 ? 4 : 2);
        for (int i = 0; i < (FP8 ? NC : NV); ++i) mbar_init(&m.v_ready[i], 4);
        for (int i = 0; i < 4; ++i) {
            mbar_init(&m.s_full[i], 1);
            mbar_init(&m.p_ready[i], 4);
            mbar_init(&m.o_done[i], 1);
        }
        mbar_init(&m.c_empty[0], 2), mbar_init(&m.c_empty[1], 2);
        mbar_init(&m.q_full, 4);
        mbar_init(&m.soft, 8);
        mbar_init(&m.group[0], 4), mbar_init(&m.group[1], 4);
        mbar_init(&m.q_free, 2);
        mbar_init(&m.drain[0], 1), mbar_init(&m.drain[1], 1);
        for (int i = 0; i < kSegRing; ++i) {
            mbar_init(&m.seg_full[i], 1);
            mbar_init(&m.seg_empty[i], FP8 ? 16 : 15);  // load, 2 MMA, (scales,) 8 softmax and 4 converting warps
        }
        for (int i = 0; i < kAuxRing; ++i) {
            mbar_init(&m.aux_full[i], 1);
            mbar_init(&m.aux_empty[i], 12);          // 8 softmax and 4 converting warps
        }
        m.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&m.tmem)), "r"(512u));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = m.tmem;                       // four buffers of S, O0, O1
    constexpr uint32_t kO = 256;
    Walk walk{m, a, {}};

    if (warp == 0) {
        Scheduler<ROWS, kTcStart> sched(m, a);                    // a segment ahead of the loads
        if (sched.publish()) role_load<FP8, D, NK, NV>(m, p, smem + C::OFF_K, smem + C::OFF_V, [&] { return sched.publish(); });
    } else if (warp == 2) {
        if constexpr (FP8) role_scales<kTcRoom>(m, a, m.kf, m.vf);
    } else if (warp == 1 || warp == 3) {
        // ------------------------------------------------ MMA issuers, one a softmax group
        if (elect_one()) {
            const int g = warp >> 1;
            Ring rk, rv;                        // rv: V's ring, as stored (plain) or as fp16 (fp8)
            constexpr int NP = FP8 ? NC : NV, kVTile = FP8 ? C::CONV : C::TILE;
            uint64_t* v_free = FP8 ? m.c_empty : m.v_empty;
            uint32_t q_phase = 0, p_phase = 0;  // p_phase: bit n & 1 of the group's two S buffers
            const uint32_t q0 = desc_lo(smem_u32(smem + (RT == 2 ? g * C::Q : 0)), 0), k0 = desc_lo(smem_u32(smem + C::OFF_K), 0);
            const uint32_t v0 = desc_lo(smem_u32(smem + (FP8 ? C::OFF_C : C::OFF_V)), kVBlock);
            const uint32_t o = tmem + kO + (uint32_t)(g * D);
            bool ok = true;
            while (true) {
                if (!mbar_wait_or_abort(&m.seg_full[walk.seg.i], walk.seg.phase, a.err, abort_flag)) { ok = false; break; }
                if (!m.seg[walk.seg.i].go) break;
                const int items = (m.seg[walk.seg.i].s.tile1 - m.seg[walk.seg.i].s.tile0) * RT;        // the group's
                mbar_arrive(&m.seg_empty[walk.seg.i]);
                walk.seg.next<kSegRing>();
                if (!mbar_wait_or_abort(&m.q_full, q_phase, a.err, abort_flag)) { ok = false; break; }
                q_phase ^= 1u;
                for (int n = 0; n <= items; ++n) {
                    if (n < items) {
                        // S of item n = Q K^T; the product that read P from this buffer (item n - 2) was issued before
                        const int half = RT == 2 ? n & 1 : g, buf = (n & 1) * 2 + g;
                        if (n % RT == 0 && !mbar_wait_or_abort(&m.k_full[rk.i], rk.phase, a.err, abort_flag)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t d = tmem + (uint32_t)(buf * kHalf);
                        const uint32_t kl = k0 + (uint32_t)(rk.i * (C::TILE >> 4) + half * (kHalf * (FP8 ? D : 128) >> 4));
                        if constexpr (FP8) {
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk) {       // q's upper terms, then its lower ones
                                const uint32_t st = kk % (D / 32) * 2;
                                mma_ss<true>(d, q0 + (kk < D / 32 ? 0 : C::Q >> 5) + st, kl + st, D == 128 ? kRows128 : kRows64,
                                             idesc_of(0, 128, kHalf, false), kk > 0);
                            }
                        } else {
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk) {
                                const uint32_t st = (kk >> 2) * (16384 >> 4) + (kk & 3) * 2;
                                mma_ss<false>(d, q0 + st, kl + st, kRows128, idesc_of(1, 128, kHalf, false), kk > 0);
                            }
                        }
                        mma_commit(&m.s_full[buf]);
                        if (n % RT == RT - 1) {
                            mma_commit(&m.k_empty[rk.i]);
                            rk.next<NK>();
                        }
                        if (n == items - 1) mma_commit(&m.q_free);
                    }
                    if (n > 0) {
                        // O += P V of item j = n - 1
                        const int j = n - 1, half = RT == 2 ? j & 1 : g, buf = (j & 1) * 2 + g;
                        if (!mbar_wait_or_abort(&m.p_ready[buf], p_phase >> (j & 1) & 1u, a.err, abort_flag)) { ok = false; break; }
                        p_phase ^= 1u << (j & 1);
                        if (j % RT == 0 && !mbar_wait_or_abort(&m.v_ready[rv.i], rv.phase, a.err, abort_flag)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t vl = v0 + (uint32_t)(rv.i * (kVTile >> 4) + half * (kHalf * 128 >> 4));
                        const uint32_t pa = tmem + (uint32_t)(buf * kHalf);
#pragma unroll
                        for (int kk = 0; kk < kHalf / 16; ++kk)
                            mma_ts(o, pa + 8 * kk, vl + 128 * kk, kRows128, idesc_of(FP8 ? 0 : 1, 128, D, true), j > 0 || kk > 0);
                        mma_commit(&m.o_done[buf]);
                        if (j % RT == RT - 1) {
                            mma_commit(&v_free[rv.i]);
                            rv.next<NP>();
                        }
                    }
                }
                if (!ok) break;
            }
            if (!ok) *abort_flag = 1;
            if (*abort_flag) {
                // products in flight read shared memory and TMEM
                mma_commit(&m.drain[g]);
                mbar_wait(&m.drain[g], 0, a.err);
            }
        }
        __syncwarp();
    } else if (warp >= 12) {
        // ------------------------------------------------ q rows, and V tiles made ready
        const int tid = threadIdx.x - 384;
        Ring rv, rc, ra;
        uint32_t q_phase = 1;           // the first segment's q buffer is free
        bool ok = true;
        while (ok && walk.next()) {
            const Segment& s = walk.segment();
            const float q_mul = a.scale_log2 > 0.f ? 1.f : a.scale_log2 < 0.f ? -1.f : 0.f;
            constexpr int kChunks = D / 8;              // 8 elements a thread, a row's threads side by side
            constexpr int kStep = 128 / kChunks, kBatch = 4;        // rows a pass; passes whose loads are under way together
            constexpr int apart = 128 / CP;
            // (rows of the block past the unit's keep what they hold: rows of S, P and O do not mix)
            for (int b0 = 0; b0 < s.rows; b0 += kStep * kBatch) {
                uint4 qv[kBatch];
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    const int r = b0 + j * kStep + tid / kChunks;
                    qv[j] = r < s.rows ? load_q(a, s, s.row0 + r, tid % kChunks * 8) : make_uint4(0, 0, 0, 0);
                }
                // the rows are under way while the last products with the segment before read its q
                if (b0 == 0) {
                    if (!mbar_wait_warp(&m.q_free, q_phase, a.err, abort_flag)) { ok = false; break; }
                    q_phase ^= 1u;
                }
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    const int r = b0 + j * kStep + tid / kChunks, c = tid % kChunks;
                    float f[8];
                    Vec16<__nv_bfloat16>::to_float(qv[j], f);
                    unsigned char* tile = smem + (r >> 7) * C::Q;
                    if constexpr (FP8) {
                        float amax = 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) f[i] = finite_or_nan(f[i] * q_mul), amax = fmaxf(amax, fabsf(f[i]));
#pragma unroll
                        for (int o = kChunks / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
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
                        if (r >= s.rows) continue;
                        // 8 bytes of a 16-byte chunk
                        const int ch = c >> 1;
                        for (int rr = r & 127, k = 0; k < CP; ++k, rr += apart) {
                            const uint32_t off = D == 128 ? (uint32_t)rr * 128u + (uint32_t)((ch ^ (rr & 7)) << 4)
                                                          : (uint32_t)rr * 64u + (uint32_t)((ch ^ ((rr >> 1) & 3)) << 4);
                            *reinterpret_cast<uint2*>(tile + off + (c & 1) * 8) = make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
                            *reinterpret_cast<uint2*>(tile + C::Q / 2 + off + (c & 1) * 8) = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
                        }
                        if (c == 0) m.q_scale[walk.seg.i][r] = pow2_of_byte(byte);
                    } else {
                        if (r >= s.rows) continue;
                        uint32_t w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i] * q_mul, f[2 * i + 1] * q_mul);
                            w[i] = *reinterpret_cast<const uint32_t*>(&v);
                        }
                        for (int rr = r & 127, k = 0; k < CP; ++k, rr += apart)
                            *reinterpret_cast<uint4*>(tile + (c >> 3) * 16384 + rr * 128 + (((c & 7) ^ (rr & 7)) << 4)) =
                                make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
            if (!ok) break;
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&m.q_full);
            unsigned long long* bad = m.seg[walk.seg.i].bad;
            for (int t = s.tile0; t < s.tile1; ++t) {
                const int pos0 = t * kTcKeys;
                const bool drafted = pos0 + kTcKeys > s.len;    // rows that not every node sees, or past the end
                if (!mbar_wait_warp(&m.v_full[rv.i], rv.phase, a.err, abort_flag)) { ok = false; break; }
                unsigned char* v = smem + C::OFF_V + rv.i * C::TILE;
                if constexpr (FP8) {
                    if (!mbar_wait_warp(&m.c_empty[rc.i], rc.phase ^ 1u, a.err, abort_flag)) { ok = false; break; }
                    if (!mbar_wait_warp(&m.aux_full[ra.i], ra.phase, a.err, abort_flag)) { ok = false; break; }
                    unsigned char* out = smem + C::OFF_C + rc.i * C::CONV;
                    if (drafted) clean_codes<D>(v, (tid >> 5) * 8 + (lane & 7), lane >> 3, s, pos0, bad);
                    // 16 codes become two 16-byte chunks; a warp takes 8 rows of 4 chunks a turn, which lie in distinct
                    // banks on both sides (alone, a tile takes 664 cycles this way, and 1013 where integer operations move
                    // the codes' bits to fp16's places)
                    const int row0 = (tid >> 5) * 8 + (lane & 7);
                    const unsigned char* src0 = v + raw_v_offset<D>(row0, lane >> 3);
                    unsigned char* dst0 = out + row0 * 128 + (((lane >> 3) * 2 ^ (lane & 7)) << 4);
                    unsigned char* dst1 = out + row0 * 128 + (((lane >> 3) * 2 ^ (lane & 7) ^ 1) << 4);
                    const __half* vf = reinterpret_cast<const __half*>(m.vf[ra.i]) + row0;
#pragma unroll 1
                    for (int i = 0; i < 4; ++i) {
                        // a turn's loads before its stores; rows 32 apart share their swizzle, and the other 64 codes of a
                        // row (D = 128) lie at chunk ^ 4
                        const __half2 f2 = __half2half2(vf[32 * i]);
                        uint4 w[D / 64];
#pragma unroll
                        for (int k = 0; k < D / 64; ++k)
                            w[k] = *reinterpret_cast<const uint4*>(reinterpret_cast<const unsigned char*>((uintptr_t)src0 ^ (64 * k)) + i * 32 * D);
#pragma unroll
                        for (int k = 0; k < D / 64; ++k) {
                            const uint32_t x[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
                            uint32_t h[8];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                h[2 * j] = f16x2_scaled(x[j], f2);
                                h[2 * j + 1] = f16x2_scaled(x[j] >> 16, f2);
                            }
                            *reinterpret_cast<uint4*>(dst0 + k * 16384 + i * 4096) = make_uint4(h[0], h[1], h[2], h[3]);
                            *reinterpret_cast<uint4*>(dst1 + k * 16384 + i * 4096) = make_uint4(h[4], h[5], h[6], h[7]);
                        }
                    }
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(&m.v_ready[rc.i]);
                        mbar_arrive(&m.v_empty[rv.i]);
                        mbar_arrive(&m.aux_empty[ra.i]);
                    }
                    ra.next<kAuxRing>();
                    rc.next<NC ? NC : 1>();
                } else {
                    if (drafted) {
                        clean_bf16<D>(v, tid, s, pos0, bad);
                        fence_async_smem();
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&m.v_ready[rv.i]);
                }
                rv.next<NV>();
            }
            if (ok) walk.done();
        }
        if (!ok) *abort_flag = 1;
    } else {
        // ------------------------------------------------ softmax: group g of 4 warps, a thread per row
        const int g = (warp - 4) >> 2, quad = warp & 3, r = quad * 32 + lane;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const uint32_t s_t = tmem + lanes, o_t = tmem + lanes + kO + (uint32_t)(g * D);
        uint32_t s_phase = 0, soft_phase = 0;         // s_phase: bit i of the group's two buffers, of S and of its product
        // the eight warps meet
        auto soft_sync = [&]() -> bool {
            __syncwarp();
            if (lane == 0) mbar_arrive(&m.soft);
            soft_phase ^= 1u;
            return mbar_wait_warp(&m.soft, soft_phase ^ 1u, a.err, abort_flag);
        };
        Ring ra;
        uint32_t group_phase = 0;
        // this group's four warps meet
        auto group_sync = [&]() -> bool {
            __syncwarp();
            if (lane == 0) mbar_arrive(&m.group[g]);
            group_phase ^= 1u;
            return mbar_wait_warp(&m.group[g], group_phase ^ 1u, a.err, abort_flag);
        };
        bool ok = true;
        while (ok && walk.next()) {
            const Segment& s = walk.segment();
            constexpr int apart = 128 / CP;
            const int row = RT == 2 ? g * 128 + r : r & (apart - 1);        // of the unit
            const int col = CP == 1 ? 0 : quad / 2 * (kHalf / CP);          // first column of this copy (as a warp's value)
            const bool live = row < s.rows;
            const bool warp_live = row - lane < s.rows;
            const int node = live ? (s.row0 + row) / a.group : 0;
            const int hq = s.head * a.group + (live ? (s.row0 + row) % a.group : 0);
            const float f_row0 = a.scale_log2 == 0.f ? 1.f : fabsf(a.scale_log2);
            float f_row = f_row0;
            RowState st{-INFINITY, 0.f, 1.f};
            int eref = 0;
            // this group's items: all of its rows (RT = 2), half of the tile's positions (RT = 1)
            const int items = (s.tile1 - s.tile0) * RT;
            for (int i = 0; i < items; ++i) {
                const int buf = (i & 1) * 2 + g, half = RT == 2 ? i & 1 : g, pos0 = (s.tile0 + i / RT) * kTcKeys + half * kHalf;
                const bool drafted = pos0 + kHalf > s.len, tile_first = i % RT == 0, tile_last = i % RT == RT - 1;
                if (FP8 && tile_first && !mbar_wait_warp(&m.aux_full[ra.i], ra.phase, a.err, abort_flag)) { ok = false; break; }
                if (!mbar_wait_warp(&m.s_full[buf], s_phase >> (i & 1) & 1u, a.err, abort_flag)) { ok = false; break; }
                s_phase ^= 1u << (i & 1);
                tc_fence_after();
                st.o_mul = 1.f;
                if (warp_live) {
                    const float4* kf = m.kf[FP8 ? ra.i : 0] + half * (kHalf / 4);
                    if (FP8 && tile_first) {
                        if (i == 0) f_row = fmaxf(f_row0 * m.q_scale[walk.seg.i][row], 0x1p-126f);     // 0 times a masked -inf is no score
                        const int e = m.eref[ra.i];
                        if (i > 0 && e > eref) st.o_mul = e - eref > 126 ? 0.f : pow2_of_byte(127 - (e - eref));
                        eref = e;
                    }
                    softmax_item<FP8, kHalf / CP>(a, s, s_t + buf * kHalf, col, kf, drafted, node, pos0, f_row, i == 0, st);
                }
                if (FP8 && tile_last) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&m.aux_empty[ra.i]);
                    ra.next<kAuxRing>();
                }
                if (i > 0 && __any_sync(0xffffffffu, live && st.o_mul != 1.f)) {
                    // once the group's product before has left O (which runs beside this item's softmax, and is not waited
                    // for otherwise); the scores of this item came after the one before that
                    if (!mbar_wait_warp(&m.o_done[buf ^ 2], (s_phase >> (~i & 1) & 1u) ^ 1u, a.err, abort_flag)) { ok = false; break; }
                    tc_fence_after();
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t x[32];
                        tmem_ld32(o_t + 32 * c, x);
                        tmem_ld_wait();
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * st.o_mul);
                        tmem_st32(o_t + 32 * c, x);
                    }
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&m.p_ready[buf]);
            }
            if (!ok) break;
            if (!mbar_wait_warp(&m.o_done[(~items & 1) * 2 + g], (s_phase >> (~items & 1) & 1u) ^ 1u, a.err, abort_flag)) { ok = false; break; }
            tc_fence_after();
            // ---------------- the unit's result, or this CTA's part of it
            const bool whole = s.part < 0;
            const long long at = (long long)(s.node0 + node) * a.n_heads + hq;
            float up0, up1 = 0.f;               // factors of O0 and O1 (RT = 1), of this group's O (RT = 2: up0)
            float m_all = st.ref, l_all = st.l;
            if constexpr (RT == 1) {
                m.ml[g * 128 + r] = make_float2(st.ref, st.l);
                if (r == 0) m.eref1[g] = eref;
                if (!soft_sync()) { ok = false; break; }
                // over both accumulators and all copies of the row
                m_all = -INFINITY;
                for (int k = row; k < 256; k += apart) m_all = fmaxf(m_all, m.ml[k].x);
                const float z = m_all == -INFINITY ? 0.f : m_all;
                l_all = 0.f;
                for (int k = row; k < 256; k += apart) l_all += m.ml[k].y * exp2f(m.ml[k].x - z);
                up0 = exp2f(m.ml[r].x - z);
                up1 = exp2f(m.ml[128 + r].x - z);
                if (FP8) {
                    up0 *= exp2f((float)(m.eref1[0] - kVUp));
                    up1 *= exp2f((float)(m.eref1[1] - kVUp));
                }
            } else {
                up0 = st.ref == -INFINITY ? 0.f : FP8 ? exp2f((float)(eref - kVUp)) : 1.f;
            }
            const unsigned long long* bad = m.seg[walk.seg.i].bad;
            const bool any_bad = bad[0] | bad[1] | bad[2] | bad[3];
            if (whole) {
                const float inv = l_all == 0.f ? 0.f : 1.f / l_all;
                up0 *= inv;
                up1 *= inv;
            }
            // group g takes half of the dimensions of both accumulators (RT = 1), or its own accumulator
            const int c0 = RT == 1 ? g * (D / 2) : 0, c1 = RT == 1 ? c0 + D / 2 : D;
            const uint32_t ta = tmem + lanes + kO + (uint32_t)(RT == 1 ? 0 : g * D), tb = ta + D;
            if constexpr (CP > 1) {
                // as many dimensions at a time as the buffer holds of the unit's rows and copies: 16 to D / 2
                float* buf = reinterpret_cast<float*>(smem + C::OFF_MERGE) + g * 128 * 16;
                const int held = s.rows * CP, fit = 128 * 16 / held & ~15, wide = fit < D / 2 ? fit : D / 2;
                const int mine_at = (r / apart * s.rows + row) * wide;
                for (int c = c0; c < c1; c += wide) {
                    const int w = min(wide, c1 - c);
                    if (warp_live) {
                        for (int d = 0; d < w; d += 16) {
                            uint32_t x[16], y[16];
                            tmem_ld16(ta + c + d, x);
                            tmem_ld16(tb + c + d, y);
                            tmem_ld_wait();
                            if (!live) continue;
#pragma unroll
                            for (int i = 0; i < 16; i += 4) {
                                float o[4];
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    o[j] = up0 == 0.f ? 0.f : __uint_as_float(x[i + j]) * up0;
                                    if (up1 != 0.f) o[j] += __uint_as_float(y[i + j]) * up1;
                                }
                                // 16-byte chunks turned by the row: rows' equal chunks lie in distinct banks
                                *reinterpret_cast<float4*>(buf + mine_at + ((d + i) / 4 + row) % (wide / 4) * 4) = make_float4(o[0], o[1], o[2], o[3]);
                            }
                        }
                    }
                    if (!group_sync()) { ok = false; break; }
                    for (int i = r; i < s.rows * (w / 4); i += 128) {
                        const int urow = i / (w / 4), q4 = i - urow * (w / 4);
                        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
                        for (int k = 0; k < CP; ++k) {
                            const float4 v = *reinterpret_cast<const float4*>(buf + (k * s.rows + urow) * wide + (q4 + urow) % (wide / 4) * 4);
                            o.x += v.x;
                            o.y += v.y;
                            o.z += v.z;
                            o.w += v.w;
                        }
                        const int ur = s.row0 + urow, nd = ur / a.group;
                        if (whole) {
                            const long long to = (long long)(s.node0 + nd) * a.n_heads + s.head * a.group + ur - nd * a.group;
                            *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + to * D + c + q4 * 4) = make_uint2(bf16x2(o.x, o.y), bf16x2(o.z, o.w));
                        } else {
                            *reinterpret_cast<float4*>(a.ws.part_o + ((long long)s.part * ROWS + urow) * D + c + q4 * 4) = o;
                        }
                    }
                    if (any_bad)
                        for (int i = r; i < s.rows * (w / 4); i += 128) add_not_finite<FP8, ROWS>(a, s, bad, i / (w / 4), c + i % (w / 4) * 4, 4);
                    if (c + wide < c1 && !group_sync()) { ok = false; break; }
                }
                if (!ok) break;
            } else if (warp_live) {
#pragma unroll 1
                for (int c = c0; c < c1; c += 16) {
                    uint32_t x[16], y[16];
                    tmem_ld16(ta + c, x);
                    if (RT == 1) tmem_ld16(tb + c, y);
                    tmem_ld_wait();
                    if (!live) continue;
                    float o[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        o[i] = up0 == 0.f ? 0.f : __uint_as_float(x[i]) * up0;
                        if (RT == 1 && up1 != 0.f) o[i] += __uint_as_float(y[i]) * up1;
                    }
                    if (whole) {
                        uint32_t w[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = bf16x2(o[2 * i], o[2 * i + 1]);
                        uint4* to = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + at * D + c);
                        to[0] = make_uint4(w[0], w[1], w[2], w[3]);
                        to[1] = make_uint4(w[4], w[5], w[6], w[7]);
                    } else {
                        // parts of these units lie by dimensions, then rows: a store of a warp is 512 bytes on end
                        float4* to = reinterpret_cast<float4*>(a.ws.part_o) + ((long long)s.part * (D / 4) + c / 4) * ROWS + row;
#pragma unroll
                        for (int i = 0; i < 4; ++i) to[i * ROWS] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                    }
                }
                if (any_bad && live)
                    for (int d = c0; d < c1; d += 4) add_not_finite<FP8, ROWS, true>(a, s, bad, row, d, 4);
            }
            if (live && c0 == 0 && r < apart) {
                if (!whole) a.ws.part_ml[(long long)s.part * ROWS + row] = make_float2(m_all, l_all);
                else if (a.lse) a.lse[at] = (m_all + log2f(l_all)) * 0.69314718055994530942f;
            }
            if constexpr (FP8) {
                const unsigned long long* far = m.seg[walk.seg.i].far;
                if (far[0] | far[1] | far[2] | far[3]) {
                    // (the calls as they are: one call of add_far_rows with RT = 1 moved the compiler to code that took 160 us
                    // for 128 fp8 rows and not 139, calls by rows with RT = 2 to spills and 220 us for 192 rows, not 213)
                    if constexpr (RT == 1) {
                        if (!soft_sync()) { ok = false; break; }
                        for (int k = warp - 4; k < min(s.rows, 128); k += 8) {
                            float2 e = make_float2(-INFINITY, 0.f);
                            for (int c = k; c < 256; c += apart) e.x = fmaxf(e.x, m.ml[c].x);
                            for (int c = k; c < 256; c += apart) e.y += e.x == -INFINITY ? 0.f : m.ml[c].y * exp2f(m.ml[c].x - e.x);
                            add_far<ROWS, CP == 1>(a, s, far, k, e.x, !whole ? 1.f : e.y == 0.f ? 0.f : 1.f / e.y);
                        }
                    } else {
                        m.ml[row] = make_float2(m_all, l_all);
                        if (!group_sync()) { ok = false; break; }
                        add_far_rows<ROWS, true>(a, s, far, m.ml, g * 128 + quad, g * 128 + 128, 4);
                    }
                }
            }
            tc_fence_before();
            if (RT == 1 && !soft_sync()) { ok = false; break; }         // O and ml may be overwritten
            walk.done();
        }
        if (!ok) *abort_flag = 1;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
}

template <bool FP8, int D, int RT, int CP>
cudaError_t tc_attr() {
    return raise_smem_limit(k_attn_tc<FP8, D, RT, CP>, tc_smem<FP8, D, RT, CP>());
}

template <bool FP8, int D>
cudaError_t tc_attrs() {
    cudaError_t e = tc_attr<FP8, D, 1, 2>();
    if (e == cudaSuccess) e = tc_attr<FP8, D, 1, 1>();
    return e == cudaSuccess ? tc_attr<FP8, D, 2, 1>() : e;
}

template <bool FP8, int D, int RT, int CP>
cudaError_t tc_go(const TcAttnArgs& p, int ctas, cudaStream_t s) {
    k_attn_tc<FP8, D, RT, CP><<<ctas, kTcThreads, tc_smem<FP8, D, RT, CP>(), s>>>(p);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? launch_join(p.a, ACE_BF16, CP == 1, Cfg<FP8, D, RT, CP>::ROWS, ctas, s) : e;
}

template <bool FP8, int D>
cudaError_t tc_launch(const TcAttnArgs& p, int ctas, cudaStream_t s) {
    // by the rows of the largest tree: one block of 128 rows a unit where that holds them (twice, if it can), else two that
    // share the loaded tiles
    const long long rows = (long long)p.a.max_nodes * p.a.group;
    if (rows <= 64) return tc_go<FP8, D, 1, 2>(p, ctas, s);
    if (rows <= 128) return tc_go<FP8, D, 1, 1>(p, ctas, s);
    return tc_go<FP8, D, 2, 1>(p, ctas, s);
}

}  // namespace

// 2-D map of a pool's rows of `row` bytes, boxes of box_rows x at most 128 bytes (plain rows: 64 bf16).
static cudaError_t row_map(CUtensorMap* m, const void* base, uint64_t rows, bool fp8, uint32_t head_dim, uint32_t box_rows) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q);
    if (e != cudaSuccess) return e;
    if (q != cudaDriverEntryPointSuccess || !fn) return cudaErrorNotSupported;
    const cuuint64_t dims[2] = {head_dim, rows};
    const cuuint64_t strides[1] = {head_dim * (fp8 ? 1u : 2u)};
    const cuuint32_t box[2] = {fp8 ? head_dim : 64u, box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn)(
        m, fp8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
        CU_TENSOR_MAP_INTERLEAVE_NONE, fp8 && head_dim == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

bool attn_tc_supported(const ace_kv* kv) {
    return kv->desc.dtype == ACE_BF16 && (kv->desc.head_dim == 64 || kv->desc.head_dim == 128);
}

cudaError_t attn_tc_init(ace_kv* kv) {
    const ace_kv_desc& D = kv->desc;
    const bool fp8 = D.format == ACE_KV_FP8;
    const uint64_t rows = (uint64_t)D.layers * D.n_pages * D.n_kv_heads * D.page_size;
    const uint32_t box = D.page_size < kTcKeys ? D.page_size : kTcKeys;
    cudaError_t e = attn_few_init(kv);
    if (e != cudaSuccess) return e;
    if ((e = row_map(&kv->maps.k, kv->k_pool, rows, fp8, D.head_dim, box)) != cudaSuccess) return e;
    if ((e = row_map(&kv->maps.v, kv->v_pool, rows, fp8, D.head_dim, box)) != cudaSuccess) return e;
    if (fp8) return D.head_dim == 128 ? tc_attrs<true, 128>() : tc_attrs<true, 64>();
    return D.head_dim == 128 ? tc_attrs<false, 128>() : tc_attrs<false, 64>();
}

cudaError_t launch_tree_attention_tc(const ace_kv* kv, const AttnArgs& a, cudaStream_t s) {
    if ((long long)a.max_nodes * a.group <= kFewRows) return launch_attn_few(kv, a, s);
    TcAttnArgs p;
    p.a = a;
    p.k = kv->maps.k;
    p.v = kv->maps.v;
    p.box_rows = a.page_size < kTcKeys ? a.page_size : kTcKeys;
    if (kv->desc.format == ACE_KV_FP8)
        return a.head_dim == 128 ? tc_launch<true, 128>(p, kv->num_sms, s) : tc_launch<true, 64>(p, kv->num_sms, s);
    return a.head_dim == 128 ? tc_launch<false, 128>(p, kv->num_sms, s) : tc_launch<false, 64>(p, kv->num_sms, s);
}

}  // namespace ace
