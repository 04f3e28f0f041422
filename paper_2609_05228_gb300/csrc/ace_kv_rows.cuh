// ace_kv_rows.cuh — rows on their way into and out of the paged cache: where they lie, and how they are quantised.
#pragma once

#include "ace_kv_device.cuh"

namespace ace {

// Row (within the layer's pool) of head h at `slot`: [page][h][row].
__device__ __forceinline__ long long pool_row(const RowArgs& p, long long slot, int h) {
    return (((slot >> p.page_shift) * p.H + h) << p.page_shift) + (slot & (p.page_size - 1));
}

// 8 elements of a row as they lie in memory.
template <typename T>
struct Raw8 {
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void to_float(float (&f)[8]) const {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) Vec16<T>::to_float(w[i], f + i * Vec16<T>::N);
    }
};

template <typename T, bool ALIGNED>
__device__ __forceinline__ Raw8<T> load8(const T* p) {
    Raw8<T> r;
    if constexpr (ALIGNED) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = ld_stream(p + i * Vec16<T>::N);
    } else {
        T* e = reinterpret_cast<T*>(r.w);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = p[i];
    }
    return r;
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&f)[8]) {
    if constexpr (sizeof(T) == 4) {
        reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&v);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

constexpr int kRowTurns = 4;            // rows that a group of lanes has under way together

// By a whole warp, each LANES lanes (a power of two, at least D / 8) with a row, 8 elements a lane from sub * 8 on (zeros past the
// row's end): the row into the pool of K (kv 0) or V (1) where `put`.
template <typename T, int FMT, int LANES>
__device__ __forceinline__ void put_row(const RowArgs& p, int kv, long long row, int sub, bool put, const Raw8<T>& raw) {
    if constexpr (FMT == ACE_KV_INT4) {
        // four lanes hold a group; the order of |x| is that of its bits, NaN and infinities on top
        float f[8];
        raw.to_float(f);
        uint32_t top = 0;
        if constexpr (sizeof(T) == 2) {
            const uint32_t x = __vmaxu2(__vmaxu2(raw.w[0].x & 0x7fff7fffu, raw.w[0].y & 0x7fff7fffu), __vmaxu2(raw.w[0].z & 0x7fff7fffu, raw.w[0].w & 0x7fff7fffu));
            top = max(x & 0xffff0000u, x << 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const bool fine = top < 0x7f800000u;
        const float s = int4_scale(fine ? __uint_as_float(top) : 0.f), inv = reciprocal_approx(s);
        if (put) {
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) w |= int4_code(f[i], s, inv) << (4 * i);
            if (!fine) w = 0x88888888u;
            *reinterpret_cast<uint32_t*>(p.pool[kv] + row * (p.D / 2) + sub * 4) = w;
            if (sub % 4 == 0)
                reinterpret_cast<uint16_t*>(p.scale[kv])[row * groups4(p.D) + sub / 4] = fine ? (uint16_t)(__float_as_uint(s) >> 16) : (uint16_t)0x7fffu;
        }
    } else if constexpr (FMT == ACE_KV_FP8) {
        float f[8], amax = 0.f;
        raw.to_float(f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f[i] = finite_or_nan(f[i]);
            amax = fmaxf(amax, fabsf(f[i]));             // fmaxf drops NaN
        }
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        const int byte = e4m3_scale_byte(amax);
        const float m = pow2_of_minus_byte(byte);
        if (put) {
            uint2 w;
            w.x = e4m3x2(f[0] * m, f[1] * m) | e4m3x2(f[2] * m, f[3] * m) << 16;
            w.y = e4m3x2(f[4] * m, f[5] * m) | e4m3x2(f[6] * m, f[7] * m) << 16;
            *reinterpret_cast<uint2*>(p.pool[kv] + row * p.D + sub * 8) = w;
            if (sub == 0) p.scale[kv][row] = (uint8_t)byte;
        }
    } else if (put) {
        uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.pool[kv]) + row * p.D + sub * 8);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) dst[i] = raw.w[i];
    }
}

}  // namespace ace
