// ace_verify.cu — ace_verify_tree: the walk down each request's tree of drafted tokens that accepts
// tokens by speculative sampling without replacement, and picks the next one.
//
// A thread-block cluster walks one request's tree: every visited node's row of logits is split over the
// cluster's CTAs, and the row's maximum, sum and argmax are joined through distributed shared memory, so all
// CTAs take the same branch from the same bits. Only the rows that the walk visits are read: one pass for
// the softmax's statistics; where a child is rejected and another follows, one for the residual's sum;
// one for the argmax at the end. Later passes hit L2. No element is stored: after k rejections the residual
// at v is k steps from its logit and draft probability,
//   r <- max(r - q, 0) / Z_j,   q <- q / (1 - q(x_j)), 0 at x_j.
#include <math.h>

#include <string>

#include "ace_kv_device.cuh"

namespace {

using namespace ace;

constexpr int kVerThreads = 512, kVerWarps = kVerThreads / 32, kMaxCluster = 8, kVerUnroll = 8;

struct VerifyArgs {
    const void* logits;
    long long logits_stride, draft_stride, noise_stride;
    const int32_t* tokens;
    const int32_t* parents;
    const int32_t* node_offsets;
    const float* draft;
    const float* temperature;
    const float* uniforms;
    const float* noise;
    int32_t* path;
    int32_t* n_keep;
    int32_t* next_token;
    int vocab, T, max_nodes;
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

// What a pass adds up: a maximum, a sum relative to it (or plain), an index, a flag.
struct Sums {
    float m, s;
    int at, bad;
};

// Softmax statistics (sums relative to their maxima, in temperature units) and the lowest index of the maximum.
__device__ __forceinline__ Sums join_stats(const Sums& a, const Sums& b, float inv_t) {
    Sums r;
    r.m = fmaxf(a.m, b.m);
    const float ref = r.m == -INFINITY ? 0.f : r.m;
    r.s = a.s * __expf((a.m - ref) * inv_t) + b.s * __expf((b.m - ref) * inv_t);
    r.at = a.m > b.m ? a.at : b.m > a.m ? b.at : min(a.at, b.at);
    r.bad = a.bad | b.bad;
    return r;
}

// Plain sum and maximum (with the lowest index).
__device__ __forceinline__ Sums join_plain(const Sums& a, const Sums& b, float) {
    return Sums{fmaxf(a.m, b.m), a.s + b.s, a.m > b.m ? a.at : b.m > a.m ? b.at : min(a.at, b.at), a.bad | b.bad};
}

struct Shared {
    Sums warp[kVerWarps];
    Sums cta[2][kMaxCluster];           // by turns, so that a fast CTA's next values find the other buffer
    int parent[kMaxNodes];
    int token[kMaxNodes];
    // rejected children of the current node: token, 1 / Z (0: the residual stayed), 1 / (1 - q)
    int x[kMaxNodes];
    float rz[kMaxNodes], rq[kMaxNodes];
};

// Joins every thread's value over the CTA, then over the cluster; all threads of all CTAs get the same bits.
template <Sums (*JOIN)(const Sums&, const Sums&, float)>
__device__ Sums join_all(Shared& sh, Sums v, float inv_t, int& turn, int ctas) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Sums u;
        u.m = __shfl_xor_sync(0xffffffffu, v.m, o);
        u.s = __shfl_xor_sync(0xffffffffu, v.s, o);
        u.at = __shfl_xor_sync(0xffffffffu, v.at, o);
        u.bad = __shfl_xor_sync(0xffffffffu, v.bad, o);
        // the lower lane first, so that both lanes of a pair get the same bits
        v = (threadIdx.x & o) ? JOIN(u, v, inv_t) : JOIN(v, u, inv_t);
    }
    if ((threadIdx.x & 31) == 0) sh.warp[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x < 32) {
        Sums t = sh.warp[threadIdx.x % kVerWarps];
#pragma unroll
        for (int o = kVerWarps / 2; o > 0; o >>= 1) {
            Sums u;
            u.m = __shfl_xor_sync(0xffffffffu, t.m, o);
            u.s = __shfl_xor_sync(0xffffffffu, t.s, o);
            u.at = __shfl_xor_sync(0xffffffffu, t.at, o);
            u.bad = __shfl_xor_sync(0xffffffffu, t.bad, o);
            t = (threadIdx.x & o) ? JOIN(u, t, inv_t) : JOIN(t, u, inv_t);
        }
        if ((int)threadIdx.x < ctas) {          // lane c hands it to CTA c
            const uint32_t mine = smem_u32(&sh.cta[turn][cluster_rank()]);
            uint32_t there;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(threadIdx.x));
            asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(there), "r"(__float_as_uint(t.m)),
                         "r"(__float_as_uint(t.s)), "r"(t.at), "r"(t.bad)
                         : "memory");
        }
    }
    cluster_sync();
    Sums r = sh.cta[turn][0];
    for (int c = 1; c < ctas; ++c) r = JOIN(r, sh.cta[turn][c], inv_t);
    turn ^= 1;
    return r;
}

struct Row {
    float m, inv_t, inv_s;
    int k;                              // rejections so far
};

// Residual at v after the row's first `k` rejections; the last one not yet applied is the caller's.
template <bool DRAFT>
__device__ __forceinline__ float residual(const Shared& sh, const Row& w, int k, int v, float z, float& q) {
    float r = __expf((z - w.m) * w.inv_t) * w.inv_s;
    for (int j = 0; j < k; ++j) {
        const float less = DRAFT ? fmaxf(r - q, 0.f) : (v == sh.x[j] ? 0.f : r);
        if (sh.rz[j] > 0.f) r = less * sh.rz[j];
        if (DRAFT) q = v == sh.x[j] ? 0.f : q * sh.rq[j];
    }
    return r;
}

template <typename T, bool DRAFT>
__global__ void __launch_bounds__(kVerThreads) k_verify(const __grid_constant__ VerifyArgs p) {
    __shared__ Shared sh;
    uint32_t n_ctas;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n_ctas));
    const int ctas = (int)n_ctas, rank = (int)cluster_rank(), b = blockIdx.x / ctas, tid = threadIdx.x;
    const int V = p.vocab, chunk = (V + ctas - 1) / ctas;
    const int lo = min(V, rank * chunk), hi = min(V, lo + chunk);
    int o0 = p.node_offsets[b], n = p.node_offsets[b + 1] - o0;
    if (o0 < 0 || n < 0 || n > p.max_nodes || o0 > p.T - n) n = 0;
    for (int i = tid; i < n; i += kVerThreads) {
        const int q = p.parents[o0 + i];
        sh.parent[i] = q >= 0 && q < i ? q : -1;
        sh.token[i] = p.tokens[o0 + i];
    }
    const float temp = p.temperature ? p.temperature[b] : 1.f;
    const bool greedy = !(temp > 0.f);
    Row w;
    w.inv_t = greedy ? 1.f : 1.f / temp;
    const float* noise = p.noise + b * p.noise_stride;
    int turn = 0, node = 0, keep = 0, token = -1;
    // every CTA of the cluster has started before another writes into its shared memory
    cluster_sync();
    while (n > 0) {
        if (rank == 0 && tid == 0) p.path[(long long)b * p.max_nodes + keep] = node;
        ++keep;
        const T* z = static_cast<const T*>(p.logits) + (o0 + node) * p.logits_stride;
        const float* qrow = DRAFT ? p.draft + (o0 + node) * p.draft_stride : nullptr;
        Sums v{-INFINITY, 0.f, V, 0};
        for (int i0 = lo + tid; i0 < hi; i0 += kVerThreads * kVerUnroll) {
            float f[kVerUnroll];
            float top = v.m;
#pragma unroll
            for (int u = 0; u < kVerUnroll; ++u) {
                const int i = i0 + u * kVerThreads;
                f[u] = i < hi ? to_f32(z[i]) : -INFINITY;
                if (!(f[u] < INFINITY)) v.bad = 1;
                if (f[u] > top) top = f[u], v.at = i;
            }
            const float ref = top == -INFINITY ? 0.f : top;
            v.s *= __expf((v.m - ref) * w.inv_t);
#pragma unroll
            for (int u = 0; u < kVerUnroll; ++u) v.s += __expf((f[u] - ref) * w.inv_t);
            v.m = top;
        }
        v = join_all<join_stats>(sh, v, w.inv_t, turn, ctas);
        if (v.bad || v.m == -INFINITY) break;               // token stays -1
        w.m = v.m;
        w.inv_s = 1.f / v.s;
        w.k = 0;
        int taken = -1;
        bool pending = false;               // the last rejection's residual has not been summed
        for (int c = node + 1; c < n && taken < 0; ++c) {
            if (sh.parent[c] != node) continue;
            const int x = sh.token[c];
            if (greedy) {
                if (x == v.at) taken = c;
                continue;
            }
            if (pending) {
                // the residual after the last rejection: its sum over the vocabulary
                Sums t{0.f, 0.f, 0, 0};
                for (int i0 = lo + tid; i0 < hi; i0 += kVerThreads * kVerUnroll) {
#pragma unroll
                    for (int u = 0; u < kVerUnroll; ++u) {
                        const int i = i0 + u * kVerThreads;
                        if (i < hi) {
                            float q = DRAFT ? qrow[i] : 0.f;
                            const float r = residual<DRAFT>(sh, w, w.k - 1, i, to_f32(z[i]), q);
                            t.s += DRAFT ? fmaxf(r - q, 0.f) : (i == sh.x[w.k - 1] ? 0.f : r);
                        }
                    }
                }
                t = join_all<join_plain>(sh, t, 0.f, turn, ctas);
                if (tid == 0) sh.rz[w.k - 1] = t.s > 0.f ? 1.f / t.s : 0.f;
                __syncthreads();
                pending = false;
            }
            if (x < 0 || x >= V) continue;  // never accepted, takes nothing from the residual
            float q = DRAFT ? qrow[x] : 1.f;
            const float r = residual<DRAFT>(sh, w, w.k, x, to_f32(z[x]), q);
            if (r > 0.f && p.uniforms[o0 + c] * q <= r) {
                taken = c;
            } else {
                __syncthreads();            // the lists are read above
                if (tid == 0) {
                    const float rest = 1.f - q;
                    sh.x[w.k] = x;
                    sh.rz[w.k] = 1.f;
                    sh.rq[w.k] = rest > 0.f ? 1.f / rest : 0.f;
                }
                __syncthreads();
                ++w.k;
                pending = true;
            }
        }
        if (taken >= 0) {
            __syncthreads();                // the lists are read above
            node = taken;
            continue;
        }
        if (greedy) {
            token = v.at;
            break;
        }
        // a sample of the residual: argmax of r / noise. It is not normalised after the last rejection, and
        // where that leaves nothing the residual before it counts.
        for (int k = w.k; ; --k) {
            Sums t{-1.f, 0.f, V, 0};
            for (int i0 = lo + tid; i0 < hi; i0 += kVerThreads * kVerUnroll) {
#pragma unroll
                for (int u = 0; u < kVerUnroll; ++u) {
                    const int i = i0 + u * kVerThreads;
                    if (i < hi) {
                        float q = DRAFT ? qrow[i] : 0.f;
                        const float r = residual<DRAFT>(sh, w, k, i, to_f32(z[i]), q);
                        const float g = r > 0.f ? r / noise[i] : -1.f;
                        if (g > t.m) t.m = g, t.at = i;
                    }
                }
            }
            t = join_all<join_plain>(sh, t, 0.f, turn, ctas);
            if (t.m >= 0.f) token = t.at;
            if (t.m >= 0.f || !pending || k < w.k) break;
        }
        break;
    }
    if (rank == 0) {
        for (int i = keep + tid; i < p.max_nodes; i += kVerThreads) p.path[(long long)b * p.max_nodes + i] = -1;
        if (tid == 0) {
            p.n_keep[b] = keep;
            p.next_token[b] = token;
        }
    }
    // no CTA leaves while another may still write into its shared memory
    cluster_sync();
}

ace_status ver_fail(ace_status st, const std::string& m) {
    set_last_error(m.c_str());
    return st;
}

template <typename T, bool DRAFT>
cudaError_t launch_verify(const VerifyArgs& p, int B, int ctas, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)B * ctas);
    cfg.blockDim = dim3(kVerThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_verify<T, DRAFT>, p);
}

}  // namespace

extern "C" ace_status ace_verify_tree(const void* logits, int dtype, long long logits_stride, int vocab,
                                      const int32_t* tokens, const int32_t* parents, const int32_t* node_offsets, int B,
                                      int T, int max_nodes, const float* draft_probs, long long draft_stride,
                                      const float* temperature, const float* uniforms, const float* noise,
                                      long long noise_stride, int32_t* path, int32_t* n_keep, int32_t* next_token,
                                      void* stream) {
    if (dtype != ACE_BF16 && dtype != ACE_F32) return ver_fail(ACE_ERR_INVALID_ARG, "unknown dtype");
    if (vocab < 1) return ver_fail(ACE_ERR_INVALID_ARG, "vocab must be positive");
    if (B < 0 || T < 0) return ver_fail(ACE_ERR_INVALID_ARG, "B and T must be >= 0");
    if (max_nodes < 1 || max_nodes > kMaxNodes) return ver_fail(ACE_ERR_INVALID_ARG, "max_nodes must be in [1, 256]");
    if (logits_stride < vocab || noise_stride < vocab || (draft_probs && draft_stride < vocab))
        return ver_fail(ACE_ERR_INVALID_ARG, "row strides must be at least vocab");
    if (B == 0) return ACE_OK;
    if (!node_offsets || !path || !n_keep || !next_token || !noise || (T > 0 && (!logits || !tokens || !parents || !uniforms)))
        return ver_fail(ACE_ERR_INVALID_ARG, "a pointer is NULL");
    if ((uintptr_t)logits % (dtype == ACE_BF16 ? 2 : 4)) return ver_fail(ACE_ERR_INVALID_ARG, "logits must be aligned to their type");
    int dev = 0, sms = 1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    // as many CTAs a request as the SMs hold for the batch, and no more than a row fills
    int ctas = 1;
    while (ctas < kMaxCluster && 2LL * ctas * B <= sms && vocab / (2 * ctas) >= kVerThreads) ctas *= 2;
    if (e == cudaSuccess) {
        const VerifyArgs p{logits, logits_stride, draft_stride, noise_stride, tokens, parents, node_offsets, draft_probs,
                           temperature, uniforms, noise, path, n_keep, next_token, vocab, T, max_nodes};
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        if (dtype == ACE_BF16)
            e = draft_probs ? launch_verify<__nv_bfloat16, true>(p, B, ctas, s) : launch_verify<__nv_bfloat16, false>(p, B, ctas, s);
        else
            e = draft_probs ? launch_verify<float, true>(p, B, ctas, s) : launch_verify<float, false>(p, B, ctas, s);
    }
    if (e != cudaSuccess)
        return ver_fail(ACE_ERR_CUDA, std::string("verify launch: ") + cudaGetErrorName(e) + " (" + cudaGetErrorString(e) + ")");
    return ACE_OK;
}
