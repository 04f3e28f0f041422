// ace_attn.cu — attention for trees of drafted tokens on the CUDA cores: any dtype, format and head size
// (the tensor-core kernel takes bf16 with head sizes 64 and 128). With G query heads per kv head, a unit
// is 16 rows (node, head of the group) of one request and kv head; a CTA walks its share of 64-key tiles:
//   s_j = scale q.k_j,  m = max s,  p_j = 2^(s_j - m) (base 2),  l = sum p_j,  o = sum p_j v_j
// with m, l and o rescaled when m grows (one pass over the cache). fp32 throughout. 16 rows by 64 keys keep K, V, q and
// scores in shared memory for two CTAs an SM at D = 128; bound by shared-memory reads. For development and odd head sizes: 4
// users of up to 777 positions, 6 nodes of 8 heads of 80, fp32: 19 us a call (of which 11 the host's).
#include "ace_kv_device.cuh"

namespace ace {
namespace {

constexpr int kRows = 16, kKeys = 64, kThreads = 256, kJoinParts = 8;

__host__ __device__ constexpr int pitch(int D) { return D + 4; }   // floats a row: 16-byte chunks of 8 rows in distinct banks
int core_smem(int D) { return (2 * kKeys * pitch(D) + kRows * pitch(D) + kRows * kKeys) * 4; }

// 8 elements of a cached row as floats; `scale` is the layer's.
template <typename T, int FMT>
__device__ __forceinline__ void cached8(const void* pool, const uint8_t* scale, long long row, int D, int d, float (&f)[8]) {
    if constexpr (FMT == ACE_KV_INT4) {
        const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(pool) + row * (D / 2) + d / 2));
        int4x8_to_float(w, float_of_bf16(__ldg(reinterpret_cast<const uint16_t*>(scale) + row * groups4(D) + d / kGroup4)), f);
    } else if constexpr (FMT == ACE_KV_FP8) {
        e4m3x8_to_float(__ldg(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(pool) + row * D + d)), f);
        const float m = pow2_of_byte(scale[row]);
#pragma unroll
        for (int x = 0; x < 8; ++x) f[x] *= m;
    } else if constexpr (sizeof(T) == 2) {
        Vec16<T>::to_float(__ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(pool) + row * D + d)), f);
    } else {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const T*>(pool) + row * D + d);
        Vec16<T>::to_float(__ldg(p), f);
        Vec16<T>::to_float(__ldg(p + 1), f + 4);
    }
}

template <typename T, int FMT>
__global__ void __launch_bounds__(kThreads) k_attn_core(const __grid_constant__ AttnArgs a) {
    extern __shared__ __align__(16) float sm[];
    const int D = a.head_dim, P = pitch(D);
    float* sk = sm;
    float* sv = sk + kKeys * P;
    float* sq = sv + kKeys * P;
    float* sp = sq + kRows * P;
    __shared__ Segment seg;
    __shared__ int go;
    const int tid = threadIdx.x, row = tid >> 4, sub = tid & 15;
    Cursor cur{};
    bool more = false;
    if (tid == 0) note_none(a);
    if (tid < 32) more = cursor_init<kRows, kKeys, 0>(a, blockIdx.x, gridDim.x, cur);
    while (true) {
        if (tid < 32) {
            Segment s;
            const bool ok = more && cursor_next<kRows, kKeys, 0>(a, blockIdx.x, cur, s);
            if (tid == 0) {
                go = ok;
                if (ok) {
                    seg = s;
                    note_unit(a, s);
                }
            }
        }
        __syncthreads();
        if (!go) break;
        const Segment s = seg;
        const bool live = row < s.rows;
        const int node = live ? (s.row0 + row) / a.group : 0;          // of the request
        const int hq = s.head * a.group + (s.row0 + row) % a.group;
        // the unit's q rows, scaled to base 2
        for (int i = tid; i < kRows * D; i += kThreads) {
            const int r = i / D, d = i % D;
            float v = 0.f;
            if (r < s.rows) {
                const int t = s.node0 + (s.row0 + r) / a.group, h = s.head * a.group + (s.row0 + r) % a.group;
                v = to_f32(static_cast<const T*>(a.q)[t * a.q_token_stride + h * a.q_head_stride + d]) * a.scale_log2;
            }
            sq[r * P + d] = v;
        }
        float m = -INFINITY, l = 0.f;
        float4 o[kMaxHeadDim / 64];
#pragma unroll
        for (int i = 0; i < kMaxHeadDim / 64; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        const int total = s.len + s.n;
        for (int tile = s.tile0; tile < s.tile1; ++tile) {
            const int pos0 = tile * kKeys;
            // K and V rows of the tile; rows past the end are zeros
            const int chunks = D / 8;
            for (int i = tid; i < kKeys * chunks; i += kThreads) {
                const int j = i / chunks, d = i % chunks * 8, pos = pos0 + j;
                float fk[8] = {}, fv[8] = {};
                if (pos < total) {
                    const int page = page_of(a, s.b, pos);
                    if (page >= 0) {
                        const long long r = ((long long)page * a.kv_heads + s.head) * a.page_size + (pos & (a.page_size - 1));
                        cached8<T, FMT>(a.k_pool, a.k_scale, r, D, d, fk);
                        cached8<T, FMT>(a.v_pool, a.v_scale, r, D, d, fv);
                    }
                }
                store8f(sk + j * P + d, fk);
                store8f(sv + j * P + d, fv);
            }
            __syncthreads();
            // thread (row, sub): scores of keys sub, sub + 16, ..
            float sc[kKeys / 16] = {};
            for (int d = 0; d < D; d += 4) {
                const float4 q = *reinterpret_cast<const float4*>(sq + row * P + d);
#pragma unroll
                for (int i = 0; i < kKeys / 16; ++i) {
                    const float4 k = *reinterpret_cast<const float4*>(sk + (sub + 16 * i) * P + d);
                    sc[i] = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, fmaf(q.w, k.w, sc[i]))));
                }
            }
            const bool drafted = pos0 + kKeys > s.len;      // holds rows that not every node sees
            uint32_t masked = 0;
            if (drafted) {
#pragma unroll
                for (int i = 0; i < kKeys / 16; ++i) {
                    const int pos = pos0 + sub + 16 * i, mth = pos - s.len;
                    if (mth >= 0 && !(sees_word(a, s.node0, s.n, node, mth >> 6) >> (mth & 63) & 1)) sc[i] = -INFINITY, masked |= 1u << i;
                }
            }
            float top = sc[0];
#pragma unroll
            for (int i = 1; i < kKeys / 16; ++i) top = fmaxf(top, sc[i]);
#pragma unroll
            for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
            const float m_new = fmaxf(m, top), ref = m_new == -INFINITY ? 0.f : m_new;
            const float back = exp2f(m - ref);
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < kKeys / 16; ++i) {
                const float p = exp2f(sc[i] - ref);
                sum += p;
                sp[row * kKeys + sub + 16 * i] = masked >> i & 1 ? -0.f : p;
            }
#pragma unroll
            for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
            l = fmaf(l, back, sum);
            m = m_new;
#pragma unroll
            for (int i = 0; i < kMaxHeadDim / 64; ++i) {
                o[i].x *= back;
                o[i].y *= back;
                o[i].z *= back;
                o[i].w *= back;
            }
            __syncwarp();
            // thread (row, sub): dimensions 4 sub + 64 i; a weight of minus zero, which no exp2f is, leaves out whatever a masked
            // row holds
            for (int j = 0; j < kKeys; ++j) {
                const float p = sp[row * kKeys + j];
                if (drafted && __float_as_uint(p) == 0x80000000u) continue;
#pragma unroll
                for (int i = 0; i < kMaxHeadDim / 64; ++i) {
                    const int d = 4 * sub + 64 * i;
                    if (d < D) {
                        const float4 v = *reinterpret_cast<const float4*>(sv + j * P + d);
                        o[i].x = fmaf(p, v.x, o[i].x);
                        o[i].y = fmaf(p, v.y, o[i].y);
                        o[i].z = fmaf(p, v.z, o[i].z);
                        o[i].w = fmaf(p, v.w, o[i].w);
                    }
                }
            }
            __syncthreads();
        }
        if (s.part < 0) {
            if (live) {
                const float inv = l == 0.f ? 0.f : 1.f / l;
                const long long at = (long long)(s.node0 + node) * a.n_heads + hq;
#pragma unroll
                for (int i = 0; i < kMaxHeadDim / 64; ++i) {
                    const int d = 4 * sub + 64 * i;
                    if (d < D) {
                        T* out = static_cast<T*>(a.out) + at * D + d;
                        out[0] = from_f32<T>(o[i].x * inv);
                        out[1] = from_f32<T>(o[i].y * inv);
                        out[2] = from_f32<T>(o[i].z * inv);
                        out[3] = from_f32<T>(o[i].w * inv);
                    }
                }
                if (sub == 0 && a.lse) a.lse[at] = (m + log2f(l)) * 0.69314718055994530942f;
            }
            __syncthreads();
            continue;
        }
        if (live) {
            const long long slot = (long long)s.part * kRows + row;
#pragma unroll
            for (int i = 0; i < kMaxHeadDim / 64; ++i) {
                const int d = 4 * sub + 64 * i;
                if (d < D) *reinterpret_cast<float4*>(a.ws.part_o + slot * D + d) = o[i];
            }
            if (sub == 0) a.ws.part_ml[slot] = make_float2(m, l);
        }
        __syncthreads();
    }
}

// Joins the units that were cut: block (CTA, 8 rows), where the CTA's note names the unit that begins in it; parts in the
// line's order, 8 at a time (a round of loads takes more than a microsecond), 4 dimensions a thread, with the reference that they
// turn up with: what came before is rescaled as it grows. A kernel of its own, so that all SMs join: when the last CTA of
// a unit joined it, that took 10 us for 128 rows of two parts and 20 for 40 rows of 19. Bound by the launch and its loads.
template <typename T, bool BY_DIMS>
__global__ void __launch_bounds__(kThreads) k_attn_join(const __grid_constant__ AttnArgs a, int rows) {
    pdl_wait();
    const int r0 = blockIdx.y * 8;
    if (r0 >= a.ws.unit[blockIdx.x].rows) return;
    const Segment s = a.ws.unit[blockIdx.x];
    const int D = a.head_dim, quads = D / 4;
    for (int i = threadIdx.x; i < 8 * quads; i += kThreads) {
        // by dimensions: 8 rows of 4 quads a warp, lines of the parts and sectors of the output
        const int r = r0 + (BY_DIMS ? i % 8 : i / quads), d = (BY_DIMS ? i / 8 : i % quads) * 4;
        if (r >= s.rows) continue;
        float M = -INFINITY, L = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int c0 = s.first; c0 <= s.last; c0 += kJoinParts) {
            float2 ml[kJoinParts];
            float4 v[kJoinParts];
#pragma unroll
            for (int j = 0; j < kJoinParts; ++j) {
                ml[j] = make_float2(-INFINITY, 0.f);
                v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (c0 + j <= s.last) {
                    const long long slot = part_slot(c0 + j, s.first);
                    ml[j] = __ldcg(&a.ws.part_ml[slot * rows + r]);
                    v[j] = __ldcg(reinterpret_cast<const float4*>(a.ws.part_o + part_place<BY_DIMS>(rows, D, slot, r, d)));
                }
            }
            float top = M;
#pragma unroll
            for (int j = 0; j < kJoinParts; ++j) top = fmaxf(top, ml[j].x);
            const float ref = top == -INFINITY ? 0.f : top, back = exp2f(M - ref);
            M = top;
            L *= back;
            o = make_float4(o.x * back, o.y * back, o.z * back, o.w * back);
#pragma unroll
            for (int j = 0; j < kJoinParts; ++j) {
                const float f = exp2f(ml[j].x - ref);
                L = fmaf(ml[j].y, f, L);
                o.x = fmaf(v[j].x, f, o.x);
                o.y = fmaf(v[j].y, f, o.y);
                o.z = fmaf(v[j].z, f, o.z);
                o.w = fmaf(v[j].w, f, o.w);
            }
        }
        const float inv = L == 0.f ? 0.f : 1.f / L;
        const int row = s.row0 + r, node = s.node0 + row / a.group, hq = s.head * a.group + row % a.group;
        const long long at = (long long)node * a.n_heads + hq;
        T* out = static_cast<T*>(a.out) + at * D + d;
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(out) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        } else {
            const __nv_bfloat162 lo = __floats2bfloat162_rn(o.x * inv, o.y * inv), hi = __floats2bfloat162_rn(o.z * inv, o.w * inv);
            *reinterpret_cast<uint2*>(out) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
        }
        if (d == 0 && a.lse) a.lse[at] = (M + log2f(L)) * 0.69314718055994530942f;
    }
}

template <typename T, bool BY_DIMS>
cudaError_t join_of(const AttnArgs& a, int rows, int ctas, cudaStream_t s) {
    const long long most = (long long)a.max_nodes * a.group;       // rows of the largest request
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas, (unsigned)(((most < rows ? most : rows) + 7) / 8));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_attn_join<T, BY_DIMS>, a, rows);
}

using CoreKernel = void (*)(const AttnArgs);

template <typename T>
CoreKernel core_of(int format) {
    return format == ACE_KV_INT4 ? k_attn_core<T, ACE_KV_INT4> : format == ACE_KV_FP8 ? k_attn_core<T, ACE_KV_FP8> : k_attn_core<T, ACE_KV_PLAIN>;
}

CoreKernel core_kernel(const ace_kv_desc& D) { return D.dtype == ACE_BF16 ? core_of<__nv_bfloat16>(D.format) : core_of<float>(D.format); }

}  // namespace

cudaError_t attn_init(ace_kv* kv) {
    const ace_kv_desc& D = kv->desc;
    kv->tc = attn_tc_supported(kv);
    size_t ctas = kv->num_sms, rows = kTcMaxRows;
    cudaError_t e;
    if (kv->tc) {
        e = attn_tc_init(kv);
    } else {
        e = raise_smem_limit(core_kernel(D), core_smem(D.head_dim));
        const int fit = 220 * 1024 / (core_smem(D.head_dim) + 2048);
        kv->core_ctas_per_sm = fit < 1 ? 1 : fit > 4 ? 4 : fit;
        ctas *= kv->core_ctas_per_sm;
        rows = kRows;
    }
    if (e != cudaSuccess) return e;
    // error word and count of moves, notes of units, pages' marks, list and moves; maxima and sums, outputs
    const size_t units = D.format == ACE_KV_INT4 && kv->tc ? 2 * ctas : ctas;       // CTAs of a launch
    const size_t pages = 256 + (units * sizeof(Segment) + 255) / 256 * 256, n_pages = D.n_pages;
    const size_t head = pages + (n_pages * (3 * sizeof(int) + sizeof(int3)) + 255) / 256 * 256, ml = (2 * ctas * rows * sizeof(float2) + 255) / 256 * 256;
    if ((e = cudaMalloc(&kv->block, head + ml + 2 * ctas * rows * D.head_dim * sizeof(float))) != cudaSuccess) return e;
    char* at = static_cast<char*>(kv->block);
    kv->err = reinterpret_cast<int*>(at);
    kv->ws.unit = reinterpret_cast<Segment*>(at + 256);
    kv->pages.count = reinterpret_cast<int*>(at + 128);
    kv->pages.mark = reinterpret_cast<int*>(at + pages);
    kv->pages.list = kv->pages.mark + 2 * n_pages;
    kv->pages.move = reinterpret_cast<int3*>(kv->pages.list + n_pages);
    kv->ws.part_ml = reinterpret_cast<float2*>(at + head);
    kv->ws.part_o = reinterpret_cast<float*>(at + head + ml);
    return cudaMemsetAsync(at, 0, head, kv->last_stream);
}

cudaError_t launch_tree_attention(const ace_kv* kv, const AttnArgs& a, cudaStream_t s) {
    if (kv->tc) return launch_tree_attention_tc(kv, a, s);
    const int grid = kv->num_sms * kv->core_ctas_per_sm;
    core_kernel(kv->desc)<<<grid, kThreads, core_smem(a.head_dim), s>>>(a);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? launch_join(a, kv->desc.dtype, false, kRows, grid, s) : e;
}

cudaError_t launch_join(const AttnArgs& a, int dtype, bool by_dims, int rows, int ctas, cudaStream_t s) {
    if (dtype != ACE_BF16) return join_of<float, false>(a, rows, ctas, s);
    return by_dims ? join_of<__nv_bfloat16, true>(a, rows, ctas, s) : join_of<__nv_bfloat16, false>(a, rows, ctas, s);
}

}  // namespace ace
