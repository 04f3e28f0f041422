// ace_rope.cu — rotary positions: q and k (or their gradients) turned by their tokens' positions, and the rows of new tokens
// turned and written into the paged cache in one pass.
//   (x, y) -> magnitude (x cos a - y sin a, x sin a + y cos a),  a = position * f_i for pair i
// The angle is kept as a fraction of a turn: F_i = f_i / 2 pi in units of 2^-64 of a turn, so that position * F_i modulo
// 2^64 (one integer product) is the angle without its whole turns, exact for F_i: off by 2^-65 |position| of a turn for F_i's
// rounding and by what f_i is (ace_angles.h), where an fp32 angle at position 10^6 is off by a thirtieth of a radian.
// Its nearest quarter turn picks sign and place, and sine and cosine are taken in fp32 of what is left, at most an eighth of a turn
// (to 2^-28 of a turn).
// LANES lanes take kRowTurns neighbouring heads of a token, 8 elements of a row each, so that a lane needs its pairs' sines and
// cosines once. They come from a table of the block's tokens in shared memory, made while the rows are under way. In layout
// "half" a pair's partner comes by shuffles where a row is a whole number of lanes' shares, from memory elsewhere. Bound by memory:
// 16384 tokens of 72 heads of 128, half of each turned, 100 us for 604 MB, 6.0 TB/s. With a look at the table a row,
// and blocks that mixed rows of q, k and v, it took 115. Rows of 8192 tokens (32 heads, 8 kv heads) into a 4-bit cache 52 us, by issue
// slots, fp8 46, plain 44 (all of each head in layout "half" 60, 52, 50).
#include <math.h>

#include <initializer_list>
#include <new>
#include <string>

#include "ace_angles.h"
#include "ace_kv_rows.cuh"
#include "ace_overlap.h"

struct ace_rope {
    ace_rope_desc desc;
    int device = 0;
    uint64_t* turns = nullptr;          // [rot_dim / 2] F_i
};

namespace {

using namespace ace;

constexpr int kNoCache = -1;            // FMT of a call that turns rows only
constexpr int kBlock = 256;

struct RopeArgs {
    RowArgs cache;                      // kNoCache: only D counts
    const void* src[3];                 // q, k, v
    long long src_token[3], src_head[3];
    void* dst[2];                       // q, k (kNoCache)
    long long dst_token[2], dst_head[2];
    int heads[3];
    int quads[3];                       // units of a token in each tensor: kRowTurns heads
    uint32_t blocks[3], T;              // blocks of k, v and q, in this order
    const int32_t* positions;
    const uint64_t* turns;
    int rot, interleaved;
    float magnitude, sin_mul;           // sin_mul: the magnitude, its sign turned for gradients
};

__device__ __forceinline__ float2 turned(uint64_t turn) {
    const int hi = (int)(turn >> 32);   // a fraction of a turn in [-1/2, 1/2)
    const unsigned quarter = ((unsigned)hi + 0x20000000u) >> 30;
    const int rest = (int)((unsigned)hi - (quarter << 30));
    float s, c;
    sincospif((float)rest * 0x1p-31f, &s, &c);
    const float x = quarter & 1 ? -s : c, y = quarter & 1 ? c : s;
    return quarter & 2 ? make_float2(-x, -y) : make_float2(x, y);
}

template <typename T>
__device__ __forceinline__ Raw8<T> round8(const float (&f)[8]) {
    Raw8<T> r;
    store8(reinterpret_cast<T*>(r.w), f);
    return r;
}

// VEC: rows, partners and results in 16-byte words.
template <typename T, int FMT, bool VEC, int LANES>
__global__ void __launch_bounds__(kBlock) k_rope(const __grid_constant__ RopeArgs p) {
    extern __shared__ float2 table[];
    constexpr uint32_t kUnits = kBlock / LANES;
    const int D = p.cache.D, R = p.rot, pairs = R / 2, sub = threadIdx.x % LANES, d0 = sub * 8;
    const bool in = d0 < D;
    // a block has units of one tensor: what is quantised first, as it takes longest
    const int which = blockIdx.x < p.blocks[0] ? 1 : blockIdx.x < p.blocks[0] + p.blocks[1] ? 2 : 0;
    const uint32_t block = blockIdx.x - (which == 1 ? 0 : which == 2 ? p.blocks[0] : p.blocks[0] + p.blocks[1]);
    const uint32_t per = p.quads[which], units = p.T * per;
    const uint32_t u_block = block * kUnits, u = u_block + threadIdx.x / LANES, token = u / per, token0 = u_block / per;
    const int h0 = (int)(u - token * per) * kRowTurns, live = u < units ? min(p.heads[which] - h0, kRowTurns) : 0;      // heads of the unit
    const long long head_stride = p.src_head[which];
    const T* src = static_cast<const T*>(p.src[which]) + token * p.src_token[which] + h0 * head_stride;
    Raw8<T> raw[kRowTurns];
    Raw8<T> other[VEC ? 1 : kRowTurns];
#pragma unroll
    for (int i = 0; i < kRowTurns; ++i) {
        raw[i] = Raw8<T>{};
        if constexpr (!VEC) other[i] = Raw8<T>{};
        if (i >= live || !in) continue;
        const T* row = src + i * head_stride;
        if constexpr (VEC) {
#pragma unroll
            for (int w = 0; w < (int)sizeof(T) / 2; ++w) raw[i].w[w] = reinterpret_cast<const uint4*>(row + d0)[w];
        } else {
            T* e = reinterpret_cast<T*>(raw[i].w);
            T* o = reinterpret_cast<T*>(other[i].w);
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const int d = d0 + x;
                e[x] = row[d];
                if (!p.interleaved && d < R) o[x] = row[d < pairs ? d + pairs : d - pairs];
            }
        }
    }
    // the table of the block's tokens; a lane's pairs, 4 or 8 on end, lie apart, so that lanes read neighbouring entries
    const int shift = p.interleaved ? 2 : 3, low = (1 << shift) - 1, apart = pairs & low ? 0 : pairs >> shift;
    const int entries = which == 2 ? 0 : (int)((min(u_block + kUnits, units) - 1) / per - token0 + 1) * pairs;
    for (int e = threadIdx.x; e < entries; e += kBlock) {
        const int t = e / pairs, i = e - t * pairs;
        const float2 c = turned((uint64_t)(int64_t)p.positions[token0 + t] * p.turns[i]);
        table[t * pairs + (apart ? (i & low) * apart + (i >> shift) : i)] = make_float2(c.x * p.magnitude, c.y * p.sin_mul);
    }
    __syncthreads();
    const bool turns = live > 0 && which < 2 && d0 < R;
    const bool second = !p.interleaved && d0 >= pairs;      // VEC: the lane has its pairs' second elements
    float2 cs[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        cs[x] = make_float2(1.f, 0.f);
        if (!turns || (p.interleaved && x >= 4)) continue;
        int i = p.interleaved ? d0 / 2 + x : d0 + x;
        if (!p.interleaved && i >= pairs) i -= pairs;
        if (i < pairs && (p.interleaved || d0 + x < R)) cs[x] = table[(token - token0) * pairs + (apart ? (i & low) * apart + (i >> shift) : i)];
    }
    long long slot = -1;
    if constexpr (FMT != kNoCache) {
        if (live > 0 && which > 0) slot = p.cache.slots[token];
        if (slot >= p.cache.n_slots) {
            if (sub == 0) atomicOr(p.cache.err, kErrIndex);
            slot = -1;
        }
    }
    const bool keeps = FMT != kNoCache && which > 0;
    const int out = which == 1;
    T* dst = static_cast<T*>(p.dst[out]) + token * p.dst_token[out] + h0 * p.dst_head[out];
#pragma unroll
    for (int i = 0; i < kRowTurns; ++i) {
        if (!__any_sync(0xffffffffu, i < live)) break;
        float f[8], y[8] = {};
        raw[i].to_float(f);
        if constexpr (VEC) {
            if (!p.interleaved) {
                // lanes of pairs' first elements are R / 16 below their partners'
                const int q = R / 16, from = sub >= 2 * q ? sub : sub < q ? sub + q : sub - q;
                Raw8<T> o;
#pragma unroll
                for (int w = 0; w < (int)sizeof(T) / 2; ++w) {
                    o.w[w].x = __shfl_sync(0xffffffffu, raw[i].w[w].x, from, LANES);
                    o.w[w].y = __shfl_sync(0xffffffffu, raw[i].w[w].y, from, LANES);
                    o.w[w].z = __shfl_sync(0xffffffffu, raw[i].w[w].z, from, LANES);
                    o.w[w].w = __shfl_sync(0xffffffffu, raw[i].w[w].w, from, LANES);
                }
                o.to_float(y);
            }
        } else {
            other[i].to_float(y);
        }
        Raw8<T> result = raw[i];
        if (turns) {
            if (p.interleaved) {
#pragma unroll
                for (int x = 0; x < 8; x += 2) {
                    const float a = f[x], b = f[x + 1];
                    f[x] = fmaf(a, cs[x / 2].x, -__fmul_rn(b, cs[x / 2].y));
                    f[x + 1] = fmaf(a, cs[x / 2].y, __fmul_rn(b, cs[x / 2].x));
                }
            } else {
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const bool upper = VEC ? second : d0 + x >= pairs;
                    f[x] = upper ? fmaf(y[x], cs[x].y, __fmul_rn(f[x], cs[x].x)) : fmaf(f[x], cs[x].x, -__fmul_rn(y[x], cs[x].y));
                }
            }
            const Raw8<T> z = round8<T>(f);
            if (d0 + 8 <= R) {
                result = z;
            } else {                    // what is not rotated stays as it came
                const T* e = reinterpret_cast<const T*>(z.w);
                T* o = reinterpret_cast<T*>(result.w);
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    if (d0 + x < R) o[x] = e[x];
            }
        }
        if (i < live && in && (FMT == kNoCache || which == 0)) {
            T* row = dst + i * p.dst_head[out];
            if constexpr (VEC) {
#pragma unroll
                for (int w = 0; w < (int)sizeof(T) / 2; ++w) reinterpret_cast<uint4*>(row + d0)[w] = result.w[w];
            } else {
                const T* e = reinterpret_cast<const T*>(result.w);
#pragma unroll
                for (int x = 0; x < 8; ++x) row[d0 + x] = e[x];
            }
        }
        if constexpr (FMT != kNoCache)
            if (keeps)
                put_row<T, FMT, LANES>(p.cache, which == 2, slot >= 0 && i < live ? pool_row(p.cache, slot, h0 + i) : 0, sub, in && slot >= 0 && i < live, result);
    }
}

template <typename T, int FMT, bool VEC, int LANES>
cudaError_t run(RopeArgs p, cudaStream_t s) {
    constexpr int kUnits = kBlock / LANES, kOrder[3] = {1, 2, 0};
    uint32_t blocks = 0;
    int least = INT32_MAX;
    for (int i = 0; i < 3; ++i) {
        p.quads[i] = (p.heads[i] + kRowTurns - 1) / kRowTurns;
        if (p.quads[i] && i < 2 && p.quads[i] < least) least = p.quads[i];
    }
    for (int i = 0; i < 3; ++i) blocks += p.blocks[i] = (uint32_t)(((long long)p.T * p.quads[kOrder[i]] + kUnits - 1) / kUnits);
    const size_t tokens = (kUnits - 1) / least + 2;              // that a block's units may belong to
    k_rope<T, FMT, VEC, LANES><<<blocks, kBlock, tokens * (p.rot / 2) * sizeof(float2), s>>>(p);
    return cudaGetLastError();
}

template <typename T, int FMT, bool VEC>
cudaError_t run_lanes(const RopeArgs& p, cudaStream_t s) {
    if (p.cache.D <= 64) return run<T, FMT, VEC, 8>(p, s);
    if (p.cache.D <= 128) return run<T, FMT, VEC, 16>(p, s);
    return run<T, FMT, VEC, 32>(p, s);
}

template <int FMT>
cudaError_t run_type(int dtype, bool vec, const RopeArgs& p, cudaStream_t s) {
    if (dtype == ACE_BF16) return vec ? run_lanes<__nv_bfloat16, FMT, true>(p, s) : run_lanes<__nv_bfloat16, FMT, false>(p, s);
    return vec ? run_lanes<float, FMT, true>(p, s) : run_lanes<float, FMT, false>(p, s);
}

// Whether the rows of [T, heads, D] at these strides lie apart: written by different threads, they may not share memory.
bool rows_apart(int T, long long token, int heads, long long head, int D) {
    const bool token_outside = token > head;
    const long long s1 = token_outside ? head : token, s2 = token_outside ? token : head;
    const int n1 = token_outside ? heads : T, n2 = token_outside ? T : heads;
    return n1 == 0 || n2 == 0 || ((n1 == 1 || s1 >= D) && (n2 == 1 || s2 >= (n1 - 1) * s1 + D));
}

// Results of one tensor: apart from one another, and in the rows' own place only with their strides.
const char* bad_out(const void* x, long long token, long long head, const void* out, long long out_token, long long out_head, int T, int heads,
                    int D) {
    if (!rows_apart(T, out_token, heads, out_head, D)) return "the rows of an output must lie apart";
    if (x == out && ((T > 1 && token != out_token) || (heads > 1 && head != out_head)))
        return "an output in the place of its input must have its strides";
    return nullptr;
}

// Rows of a tensor of the call; the bytes of an array. (Other threads read and write them while an output is written.)
RowSet rows_of(const void* x, long long token, long long head, int T, int heads, int D, int elem) {
    return RowSet{(uintptr_t)x, (Wide)token * elem, (Wide)head * elem, T, heads, D * elem};
}
RowSet bytes_of(const void* x, long long bytes) { return RowSet{(uintptr_t)x, 0, 0, 1, 1, bytes}; }

// Whether an output meets any of the others but the `own` input, when it lies in that one's place.
bool meets(const RowSet& out, const RowSet& own, std::initializer_list<RowSet> others) {
    if (out.at != own.at && rows_meet(out, own)) return true;
    for (const RowSet& x : others)
        if (rows_meet(out, x)) return true;
    return false;
}

constexpr char kOverlap[] = "an output must not overlap the other tensors";

ace_status rope_fail(const char* m) { return kv_fail(ACE_ERR_INVALID_ARG, m); }

// Rows of a call whose rows all begin on 16 bytes, with whole words of pairs.
bool words(const RopeArgs& p, int elem, bool with_k_out) {
    const long long vec = 16 / elem;
    bool ok = p.interleaved || p.rot % 16 == 0;
    for (int i = 0; i < 3; ++i)
        if (p.heads[i]) ok = ok && aligned16(p.src[i]) && p.src_token[i] % vec == 0 && p.src_head[i] % vec == 0;
    for (int i = 0; i < (with_k_out ? 2 : 1); ++i)
        if (p.heads[i]) ok = ok && aligned16(p.dst[i]) && p.dst_token[i] % vec == 0 && p.dst_head[i] % vec == 0;
    return ok;
}

void of_rope(const ace_rope* rope, int inverse, const int32_t* positions, RopeArgs& p) {
    p.positions = positions;
    p.turns = rope->turns;
    p.rot = rope->desc.rot_dim;
    p.interleaved = rope->desc.layout == ACE_ROPE_INTERLEAVED;
    p.magnitude = (float)rope->desc.magnitude;
    p.sin_mul = inverse ? -p.magnitude : p.magnitude;
}

}  // namespace

extern "C" {

ace_status ace_rope_create(const ace_rope_desc* desc, const double* divisors, void* stream, ace_rope** out_rope) {
    if (!desc || !out_rope) return rope_fail("desc and out_rope must be non-NULL");
    *out_rope = nullptr;
    const ace_rope_desc& D = *desc;
    if (D.head_dim <= 0 || D.head_dim % 8 || D.head_dim > kMaxHeadDim)
        return kv_fail(ACE_ERR_UNSUPPORTED, "head_dim must be a multiple of 8, at most 256");
    if (D.rot_dim < 2 || D.rot_dim % 2 || D.rot_dim > D.head_dim) return rope_fail("rot_dim must be even, from 2 to head_dim");
    if (D.layout != ACE_ROPE_HALF && D.layout != ACE_ROPE_INTERLEAVED) return rope_fail("unknown layout");
    if (D.dtype != ACE_BF16 && D.dtype != ACE_F32) return rope_fail("unknown dtype");
    if (D.scaling < ACE_ROPE_NONE || D.scaling > ACE_ROPE_BY_INDEX) return rope_fail("unknown scaling");
    if (!(D.base > 1.0) || !isfinite(D.base)) return rope_fail("base must be above 1 and finite");
    if (!(D.magnitude > 0.0) || !isfinite((float)D.magnitude)) return rope_fail("magnitude must be positive and finite");
    if (D.scaling != ACE_ROPE_NONE && (!(D.factor > 0.0) || !isfinite(D.factor))) return rope_fail("factor must be positive and finite");
    if (D.scaling >= ACE_ROPE_BY_TURNS && (!(D.original_len > 0.0) || !isfinite(D.original_len) || !(D.low > 0.0) || !(D.high > D.low) || !isfinite(D.high)))
        return rope_fail("scaling by turns or index needs original_len > 0 and 0 < low < high, all finite");
    uint64_t turns[kMaxHeadDim / 2];
    for (int i = 0; i < D.rot_dim / 2; ++i) {
        double f = rope_frequency(D, i);
        if (divisors) {
            if (!(divisors[i] > 0.0) || !isfinite(divisors[i])) return rope_fail("divisors must be positive and finite");
            f /= divisors[i];
        }
        if (!isfinite(f)) return rope_fail("a frequency is not finite");
        turns[i] = rope_turn(f);
    }
    ace_rope* rope = new (std::nothrow) ace_rope();
    if (!rope) return kv_fail(ACE_ERR_OOM, "out of host memory");
    rope->desc = D;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const size_t bytes = D.rot_dim / 2 * sizeof(uint64_t);
    cudaError_t e = cudaGetDevice(&rope->device);
    if (e == cudaSuccess) e = cudaMalloc(&rope->turns, bytes);
    if (e == cudaSuccess) e = cudaMemcpyAsync(rope->turns, turns, bytes, cudaMemcpyHostToDevice, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e != cudaSuccess) {
        ace_rope_destroy(rope);
        if (e == cudaErrorMemoryAllocation) {
            cudaGetLastError();
            return kv_fail(ACE_ERR_OOM, "cudaMalloc failed for the frequencies");
        }
        return kv_cuda(e, "ace_rope_create");
    }
    *out_rope = rope;
    return ACE_OK;
}

void ace_rope_destroy(ace_rope* rope) {
    if (!rope) return;
    if (rope->turns) cudaFree(rope->turns);         // waits for the device
    delete rope;
}

ace_status ace_rope_apply(const ace_rope* rope, int inverse, const int32_t* positions, int T, const void* q, long long q_token_stride,
                          long long q_head_stride, int n_heads, void* q_out, long long q_out_token_stride, long long q_out_head_stride,
                          const void* k, long long k_token_stride, long long k_head_stride, int n_kv_heads, void* k_out,
                          long long k_out_token_stride, long long k_out_head_stride, void* stream) {
    if (!rope) return rope_fail("rope is NULL");
    if (T < 0 || n_heads < 0 || n_kv_heads < 0) return rope_fail("T, n_heads and n_kv_heads must be >= 0");
    const long long strides[] = {q_token_stride, q_head_stride, q_out_token_stride, q_out_head_stride,
                                 k_token_stride, k_head_stride, k_out_token_stride, k_out_head_stride};
    for (const long long x : strides)
        if (x < 0) return rope_fail("strides must be >= 0");
    const int elem = rope->desc.dtype == ACE_BF16 ? 2 : 4, D = rope->desc.head_dim;
    const long long rows = ((long long)n_heads + n_kv_heads) * T;
    if (rows > 0) {
        if (!positions || (n_heads && (!q || !q_out)) || (n_kv_heads && (!k || !k_out)))
            return rope_fail("positions, and the tensors with heads, must be non-NULL");
        if ((uintptr_t)q % elem || (uintptr_t)q_out % elem || (uintptr_t)k % elem || (uintptr_t)k_out % elem)
            return rope_fail("q, k and their outputs must be aligned to their type");
        const char* bad = bad_out(q, q_token_stride, q_head_stride, q_out, q_out_token_stride, q_out_head_stride, T, n_heads, D);
        if (!bad) bad = bad_out(k, k_token_stride, k_head_stride, k_out, k_out_token_stride, k_out_head_stride, T, n_kv_heads, D);
        if (bad) return rope_fail(bad);
        const RowSet rq = rows_of(q, q_token_stride, q_head_stride, T, n_heads, D, elem), rk = rows_of(k, k_token_stride, k_head_stride, T, n_kv_heads, D, elem);
        const RowSet oq = rows_of(q_out, q_out_token_stride, q_out_head_stride, T, n_heads, D, elem);
        const RowSet ok = rows_of(k_out, k_out_token_stride, k_out_head_stride, T, n_kv_heads, D, elem), at = bytes_of(positions, 4LL * T);
        if (meets(oq, rq, {rk, ok, at}) || meets(ok, rk, {rq, at})) return rope_fail(kOverlap);
    }
    if (const ace_status st = on_device(rope->device, "rope")) return st;
    if (rows == 0) return ACE_OK;
    if (rows > kMaxRows) return kv_fail(ACE_ERR_UNSUPPORTED, "a call turns at most 2^30 rows");
    RopeArgs p{};
    p.cache.D = D;
    p.src[0] = q, p.src_token[0] = q_token_stride, p.src_head[0] = q_head_stride;
    p.src[1] = k, p.src_token[1] = k_token_stride, p.src_head[1] = k_head_stride;
    p.dst[0] = q_out, p.dst_token[0] = q_out_token_stride, p.dst_head[0] = q_out_head_stride;
    p.dst[1] = k_out, p.dst_token[1] = k_out_token_stride, p.dst_head[1] = k_out_head_stride;
    p.heads[0] = n_heads, p.heads[1] = n_kv_heads;
    p.T = (uint32_t)T;
    of_rope(rope, inverse, positions, p);
    const cudaError_t e = run_type<kNoCache>(rope->desc.dtype, words(p, elem, true), p, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? ACE_OK : kv_cuda(e, "rope launch");
}

ace_status ace_kv_write_rotated(ace_kv* kv, int layer, const ace_rope* rope, const int32_t* positions, const void* q,
                                long long q_token_stride, long long q_head_stride, int n_heads, void* q_out, long long q_out_token_stride,
                                long long q_out_head_stride, const void* k, long long k_token_stride, long long k_head_stride, const void* v,
                                long long v_token_stride, long long v_head_stride, const int64_t* slots, int T, void* stream) {
    if (!kv || !rope) return rope_fail("cache and rope must be non-NULL");
    const ace_kv_desc& D = kv->desc;
    if (layer < 0 || layer >= D.layers) return rope_fail("layer out of range");
    if (rope->desc.head_dim != D.head_dim || rope->desc.dtype != D.dtype) return rope_fail("rope and cache must have the same head_dim and dtype");
    if (T < 0 || n_heads < 0) return rope_fail("T and n_heads must be >= 0");
    const long long strides[] = {q_token_stride, q_head_stride, q_out_token_stride, q_out_head_stride,
                                 k_token_stride, k_head_stride, v_token_stride, v_head_stride};
    for (const long long x : strides)
        if (x < 0) return rope_fail("strides must be >= 0");
    if (T > 0 && (!positions || !k || !v || !slots || (n_heads && (!q || !q_out))))
        return rope_fail("positions, k, v, slots and (with heads) q and q_out must be non-NULL");
    const int elem = kv->elem;
    if ((uintptr_t)q % elem || (uintptr_t)q_out % elem || (uintptr_t)k % elem || (uintptr_t)v % elem)
        return rope_fail("q, q_out, k and v must be aligned to their type");
    if (T > 0 && n_heads > 0) {
        if (const char* bad = bad_out(q, q_token_stride, q_head_stride, q_out, q_out_token_stride, q_out_head_stride, T, n_heads, D.head_dim))
            return rope_fail(bad);
        const long long rows = (long long)D.layers * D.n_pages * D.n_kv_heads * D.page_size, pool = rows * row_bytes(D.format, D.head_dim, elem);
        const long long scales = rows * scale_bytes(D.format, D.head_dim);
        auto heads_of = [&](const void* x, long long token, long long head, int heads) { return rows_of(x, token, head, T, heads, D.head_dim, elem); };
        if (meets(heads_of(q_out, q_out_token_stride, q_out_head_stride, n_heads), heads_of(q, q_token_stride, q_head_stride, n_heads),
                  {heads_of(k, k_token_stride, k_head_stride, D.n_kv_heads), heads_of(v, v_token_stride, v_head_stride, D.n_kv_heads), bytes_of(positions, 4LL * T),
                   bytes_of(slots, 8LL * T), bytes_of(kv->k_pool, pool), bytes_of(kv->v_pool, pool), bytes_of(kv->k_scale, scales), bytes_of(kv->v_scale, scales)}))
            return rope_fail(kOverlap);
    }
    if (const ace_status st = on_device(kv->device, "cache")) return st;
    if (const ace_status st = on_device(rope->device, "rope")) return st;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    kv->last_stream = s;
    if (T == 0) return ACE_OK;
    const long long rows = ((long long)n_heads + 2 * D.n_kv_heads) * T;
    if (rows > kMaxRows) return kv_fail(ACE_ERR_UNSUPPORTED, "a call writes at most 2^30 rows (T (n_heads + 2 n_kv_heads))");
    RopeArgs p{};
    p.cache = row_args(kv, layer, slots, T);
    p.src[0] = q, p.src_token[0] = q_token_stride, p.src_head[0] = q_head_stride;
    p.src[1] = k, p.src_token[1] = k_token_stride, p.src_head[1] = k_head_stride;
    p.src[2] = v, p.src_token[2] = v_token_stride, p.src_head[2] = v_head_stride;
    p.dst[0] = q_out, p.dst_token[0] = q_out_token_stride, p.dst_head[0] = q_out_head_stride;
    p.heads[0] = n_heads, p.heads[1] = p.heads[2] = D.n_kv_heads;
    p.T = (uint32_t)T;
    of_rope(rope, 0, positions, p);
    const bool vec = words(p, elem, false);
    const cudaError_t e = D.format == ACE_KV_INT4  ? run_type<ACE_KV_INT4>(D.dtype, vec, p, s)
                          : D.format == ACE_KV_FP8 ? run_type<ACE_KV_FP8>(D.dtype, vec, p, s)
                                                   : run_type<ACE_KV_PLAIN>(D.dtype, vec, p, s);
    return e == cudaSuccess ? ACE_OK : kv_cuda(e, "rotating write launch");
}

}  // extern "C"
