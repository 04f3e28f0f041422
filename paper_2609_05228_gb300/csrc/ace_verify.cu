// ace_verify.cu — ace_verify_tree: the walk down each request's tree of drafted tokens that accepts
// tokens by speculative sampling without replacement, and picks the next one.
//
// A thread-block cluster walks one request's tree: every visited node's row of logits is split over the
// cluster's CTAs, and the row's maximum, sum and argmax are joined through distributed shared memory, so all
// CTAs take the same branch from the same bits. Only the rows that the walk visits are read: one pass for
// the softmax's statistics; where a child is rejected and another follows, one for the residual's sum;
// one for the argmax at the end. Later passes hit L2. No element is stored: with q's normalisations and the
// residuals' gathered in scalars, the residual at v after k rejections is nu rho_k with
//   rho_0 = 2^((z - m) a),   rho_j = max(rho_(j-1) - c_j q, 0),   q <- 0 at x_j,
// two operations a rejection and element (the passes of a request that rejects are bound by them). m is the row's maximum,
// taken off before the product with a = log2(e) / temperature as the softmax's sum has it: z a - m a in one operation would be
// off by the rounding of m a, a factor that all of the row shares and its sum does not. Sums are fp32.
// Measured: 64 requests of 16 nodes over 128000 tokens: 81 us (floor 19: the rows that are visited, once; the longest walk,
// of some ten passes that wait for one another, bounds it). One request's chain of 8 over 32000: 16 us.
#include <float.h>
#include <math.h>

#include <string>

#include "ace_kv_device.cuh"

namespace {

using namespace ace;

constexpr int kVerThreads = 512, kVerWarps = kVerThreads / 32, kMaxCluster = 8;
constexpr int kAheadVocab = 65536;
constexpr int kPassUnroll = 2;          // loads of four elements a thread, row and turn of a pass (twice as many without the noise)

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

// What a pass adds up: a maximum with its lowest index, a sum (relative to the maximum, for the softmax), a flag.
struct Sums {
    float m, s;
    int at, bad;
};

enum Join { kStats, kSum, kArgmax };

// Floats in the order of integers (NaN must not occur).
__device__ __forceinline__ float warp_top(float x) {
    int i = __float_as_int(x);
    i ^= (i >> 31) & 0x7fffffff;
    i = __reduce_max_sync(0xffffffffu, i);
    return __int_as_float(i ^ ((i >> 31) & 0x7fffffff));
}

// Joins a warp's values; every lane gets the same bits.
template <Join J>
__device__ __forceinline__ Sums join_warp(Sums v, float inv_t) {
    Sums r{0.f, 0.f, 0, 0};
    if (J != kSum) {
        r.m = warp_top(v.m);
        r.at = (int)__reduce_min_sync(0xffffffffu, v.m == r.m ? (unsigned)v.at : 0x7fffffffu);
    }
    if (J != kArgmax) {
        float x = v.s;
        if (J == kStats) x *= r.m == -INFINITY ? 0.f : __expf((v.m - r.m) * inv_t);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        r.s = x;
    }
    if (J == kStats) r.bad = __any_sync(0xffffffffu, v.bad);
    return r;
}

struct Shared {
    Sums warp[kVerWarps];
    Sums cta[2][kMaxCluster];           // by turns, so that a fast CTA's next values find the other buffer
    Sums node[kMaxCluster];             // AHEAD: every node's statistics
    int parent[kMaxNodes];
    int token[kMaxNodes];
    // the current node's children: logit and draft probability at their token, and u
    float zx[kMaxNodes], qx[kMaxNodes], u[kMaxNodes];
    // rejected children of the current node: factor c of the draft probability (0: the residual stayed), token
    float c[kMaxNodes];
    int x[kMaxNodes];
};

// Joins every thread's value over the CTA and writes it to `place` in the shared memory of all CTAs of the cluster.
template <Join J>
__device__ void hand_out(Shared& sh, Sums v, Sums* place, float inv_t, int ctas) {
    const int lane = threadIdx.x & 31;
    const Sums none{-INFINITY, 0.f, 0x7fffffff, 0};
    v = join_warp<J>(v, inv_t);
    if (lane == 0) sh.warp[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x < 32) {
        const Sums t = join_warp<J>(lane < kVerWarps ? sh.warp[lane % kVerWarps] : none, inv_t);
        if (lane < ctas) {                      // lane c hands it to CTA c
            const uint32_t mine = smem_u32(place);
            uint32_t there;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(lane));
            asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(there), "r"(__float_as_uint(t.m)),
                         "r"(__float_as_uint(t.s)), "r"(t.at), "r"(t.bad)
                         : "memory");
        }
        __syncwarp();
    }
}

// Joins every thread's value over the cluster; all threads of all CTAs get the same bits.
template <Join J>
__device__ Sums join_all(Shared& sh, Sums v, float inv_t, int& turn, int ctas) {
    const int lane = threadIdx.x & 31;
    const Sums none{-INFINITY, 0.f, 0x7fffffff, 0};
    hand_out<J>(sh, v, &sh.cta[turn][cluster_rank()], inv_t, ctas);
    cluster_sync();
    const Sums r = join_warp<J>(lane < ctas ? sh.cta[turn][lane % kMaxCluster] : none, inv_t);
    turn ^= 1;
    return r;
}

// A node's softmax as rho_0 = 2^((z - m) a), and what its rejections make of it.
struct Row {
    float a, m, nu, q_mul;              // residual = nu rho_k; draft probabilities of what is left: q_mul q
    int k;                              // rejections so far
};

__device__ __forceinline__ float exp2_of(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// rho_k of N elements from their indices, logits and draft probabilities; q becomes 0 at rejected tokens.
template <bool DRAFT, int N>
__device__ __forceinline__ void residuals(const Shared& sh, const Row& w, const int (&v)[N], const float (&z)[N], float (&q)[N], float (&rho)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) rho[i] = exp2_of((z[i] - w.m) * w.a);
    for (int j = 0; j < w.k; ++j) {
        const float c = sh.c[j];
        const int x = sh.x[j];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (DRAFT) {
                rho[i] = fmaxf(fmaf(-c, q[i], rho[i]), 0.f);
                if (v[i] == x) q[i] = 0.f;
            } else if (v[i] == x) {
                rho[i] = c > 0.f ? 0.f : rho[i];
            }
        }
    }
}

// A pass over elements lo <= i < hi of up to three rows: calls f(indices, z, q, noise) for batches of the thread's. With VEC a
// thread's elements come four at a time in one load a row (all rows 16-byte aligned), else one by one. All
// loads of a turn are under way together.
template <typename T, bool VEC, bool Q, bool NOISE, typename F>
__device__ __forceinline__ void pass(const T* z, const float* q, const float* noise, int lo, int hi, F f) {
    constexpr int U = NOISE ? kPassUnroll : 2 * kPassUnroll, N = 4 * U;
    for (int base = lo; base < hi; base += kVerThreads * N) {
        float zf[N], qf[N], nf[NOISE ? N : 1];
        int at[N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = base + 4 * ((int)threadIdx.x + kVerThreads * u);
            if (VEC && i + 4 <= hi) {
                if constexpr (sizeof(T) == 2) {
                    const uint2 w = __ldg(reinterpret_cast<const uint2*>(z + i));
                    zf[4 * u] = __uint_as_float(w.x << 16), zf[4 * u + 1] = __uint_as_float(w.x & 0xffff0000u);
                    zf[4 * u + 2] = __uint_as_float(w.y << 16), zf[4 * u + 3] = __uint_as_float(w.y & 0xffff0000u);
                } else {
                    *reinterpret_cast<float4*>(zf + 4 * u) = __ldg(reinterpret_cast<const float4*>(z + i));
                }
                if (Q) *reinterpret_cast<float4*>(qf + 4 * u) = __ldg(reinterpret_cast<const float4*>(q + i));
                if constexpr (NOISE) *reinterpret_cast<float4*>(nf + 4 * u) = __ldg(reinterpret_cast<const float4*>(noise + i));
#pragma unroll
                for (int j = 0; j < 4; ++j) at[4 * u + j] = i + j;
            } else {
                // (an element past the end: a logit of -inf, so a residual of zero)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int e = VEC ? i + j : base + (int)threadIdx.x + kVerThreads * (4 * u + j);
                    const bool in = e < hi;
                    at[4 * u + j] = e;
                    zf[4 * u + j] = in ? to_f32(z[e]) : -INFINITY;
                    qf[4 * u + j] = Q && in ? __ldg(q + e) : 0.f;
                    if constexpr (NOISE) nf[4 * u + j] = in ? __ldg(noise + e) : 1.f;
                }
            }
            if (!Q) qf[4 * u] = qf[4 * u + 1] = qf[4 * u + 2] = qf[4 * u + 3] = 0.f;
        }
        f(at, zf, qf, nf);
    }
}

// Asks for a row's elements lo .. hi in L2, a line a thread and turn.
template <typename T>
__device__ __forceinline__ void prefetch_row(const T* row, int lo, int hi) {
    const char* end = reinterpret_cast<const char*>(row + hi);
    for (const char* p = reinterpret_cast<const char*>(row + lo) + threadIdx.x * 128; p < end; p += kVerThreads * 128)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
}

// Softmax statistics of z[lo .. hi): 16-byte loads between the unaligned ends, 4 a thread under way together.
template <typename T>
__device__ Sums row_stats(const T* z, int lo, int hi, int none, float inv_t, bool find) {
    constexpr int N = Vec16<T>::N, U = 4;
    Sums v{-INFINITY, 0.f, none, 0};
    auto one = [&](int i) {
        const float f = to_f32(z[i]);
        if (!(f < INFINITY)) v.bad = 1;
        if (f > v.m) {
            v.s = v.s * __expf((v.m - f) * inv_t) + 1.f;
            v.m = f;
            v.at = i;
        } else if (f > -INFINITY) {
            v.s += __expf((f - v.m) * inv_t);
        }
    };
    const int skip = (int)((16 - (uintptr_t)(z + lo) % 16) % 16 / sizeof(T));
    const int a0 = min(hi, lo + skip), groups = (hi - a0) / N, a1 = a0 + groups * N;
    // the few elements before and after the aligned ones, in increasing order within a thread
    if (lo + (int)threadIdx.x < a0) one(lo + threadIdx.x);
    for (int g0 = threadIdx.x; g0 < groups; g0 += kVerThreads * U) {
        float f[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int g = g0 + u * kVerThreads;
            if (g < groups) {
                Vec16<T>::to_float(__ldg(reinterpret_cast<const uint4*>(z + a0 + g * N)), f[u]);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) f[u][i] = -INFINITY;
            }
        }
        float top = v.m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (!(f[u][i] < INFINITY)) v.bad = 1;
                top = fmaxf(top, f[u][i]);
            }
        }
        if (find && top > v.m) {            // greedy requests: where the maximum is first
#pragma unroll
            for (int u = U - 1; u >= 0; --u) {
#pragma unroll
                for (int i = N - 1; i >= 0; --i)
                    if (f[u][i] == top) v.at = a0 + (g0 + u * kVerThreads) * N + i;
            }
        }
        const float ref = top == -INFINITY ? 0.f : top;
        v.s *= __expf((v.m - ref) * inv_t);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int i = 0; i < N; ++i) v.s += __expf((f[u][i] - ref) * inv_t);
        }
        v.m = top;
    }
    if (a1 + (int)threadIdx.x < hi) one(a1 + threadIdx.x);
    return v;
}

// AHEAD: all nodes' statistics at once before the walk, a row a CTA (so no tree has more nodes than the cluster CTAs), and what
// the walk asks of their children: then a step down costs no pass.
template <typename T, bool DRAFT, bool VEC, bool AHEAD>
__global__ void __launch_bounds__(kVerThreads, 2) k_verify(const __grid_constant__ VerifyArgs p) {
    __shared__ Shared sh;
    uint32_t n_ctas;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n_ctas));
    const int ctas = (int)n_ctas, rank = (int)cluster_rank(), b = blockIdx.x / ctas, tid = threadIdx.x;
    const int V = p.vocab, chunk = ((V + ctas - 1) / ctas + 7) / 8 * 8;
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
    const float inv_t = greedy ? 1.f : fminf(1.f / temp, FLT_MAX);       // (finite: 0 times it is the maximum's exponent)
    const float* noise = p.noise + b * p.noise_stride;
    int turn = 0, node = 0, keep = 0, token = -1;
    if (n > 0 && !greedy) prefetch_row(noise, lo, hi);
    // every CTA of the cluster has started before another writes into its shared memory
    cluster_sync();
    if constexpr (AHEAD) {
        if (tid < n && sh.parent[tid] >= 0) {
            const int of = sh.parent[tid], x = sh.token[tid];
            if (x >= 0 && x < V) {
                sh.zx[tid] = to_f32(static_cast<const T*>(p.logits)[(o0 + of) * p.logits_stride + x]);
                sh.qx[tid] = DRAFT ? p.draft[(o0 + of) * p.draft_stride + x] : 1.f;
                sh.u[tid] = p.uniforms[o0 + tid];
            }
        }
        if (rank < n) {
            const Sums v = row_stats(static_cast<const T*>(p.logits) + (o0 + rank) * p.logits_stride, 0, V, V, inv_t, greedy);
            hand_out<kStats>(sh, v, &sh.node[rank], inv_t, ctas);
        }
        cluster_sync();
    }
    while (n > 0) {
        if (rank == 0 && tid == 0) p.path[(long long)b * p.max_nodes + keep] = node;
        ++keep;
        const T* z = static_cast<const T*>(p.logits) + (o0 + node) * p.logits_stride;
        const float* qrow = DRAFT ? p.draft + (o0 + node) * p.draft_stride : nullptr;
        // what this node's walk may need next: its draft row where it has a child, and the first child's logits
        int first = node + 1;
        while (first < n && sh.parent[first] != node) ++first;
        if (first < n) {
            if (DRAFT && !greedy) prefetch_row(qrow, lo, hi);
            if (!AHEAD) prefetch_row(static_cast<const T*>(p.logits) + (o0 + first) * p.logits_stride, lo, hi);
        }
        Sums v;
        if constexpr (AHEAD) {
            v = sh.node[node];
        } else {
            // (a later node's children may lie in the same places: the walk has passed a barrier since it read them)
            for (int c = node + 1 + tid; c < n; c += kVerThreads) {
                const int x = sh.token[c];
                if (sh.parent[c] != node || x < 0 || x >= V) continue;
                sh.zx[c] = to_f32(z[x]);
                sh.qx[c] = DRAFT ? qrow[x] : 1.f;
                sh.u[c] = p.uniforms[o0 + c];
            }
            v = row_stats(z, lo, hi, V, inv_t, greedy);
            v = join_all<kStats>(sh, v, inv_t, turn, ctas);
        }
        if (v.bad || v.m == -INFINITY) break;               // token stays -1
        w.a = fminf(inv_t * 1.4426950408889634f, FLT_MAX);
        w.m = v.m;
        w.nu = 1.f / v.s;
        w.q_mul = 1.f;
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
                pass<T, VEC, DRAFT, false>(z, qrow, nullptr, lo, hi, [&](const auto& at, const auto& zi, auto& q, const auto&) {
                    float rho[sizeof(zi) / 4];
                    residuals<DRAFT>(sh, w, at, zi, q, rho);
#pragma unroll
                    for (int i = 0; i < (int)(sizeof(zi) / 4); ++i) t.s += rho[i];
                });
                t = join_all<kSum>(sh, t, 0.f, turn, ctas);
                if (t.s > 0.f) {
                    w.nu = 1.f / t.s;
                } else {
                    __syncthreads();
                    if (tid == 0) sh.c[w.k - 1] = 0.f;
                    __syncthreads();
                }
                pending = false;
            }
            if (x < 0 || x >= V) continue;  // never accepted, takes nothing from the residual
            const int at[1] = {x};
            const float zx[1] = {sh.zx[c]};
            float q1[1] = {sh.qx[c]}, rho[1];
            residuals<DRAFT>(sh, w, at, zx, q1, rho);
            const float r = rho[0] * w.nu, q = DRAFT ? q1[0] * w.q_mul : 1.f;
            if (r > 0.f && sh.u[c] * q <= r) {
                taken = c;
            } else {
                __syncthreads();            // the lists are read above
                if (tid == 0) {
                    sh.x[w.k] = x;
                    sh.c[w.k] = DRAFT ? w.q_mul / w.nu : 1.f;
                }
                __syncthreads();
                const float rest = 1.f - q;
                w.q_mul = rest > 0.f ? w.q_mul / rest : 0.f;
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
        for (bool again = pending; ; again = false) {
            Sums t{-1.f, 0.f, V, 0};
            pass<T, VEC, DRAFT, true>(z, qrow, noise, lo, hi, [&](const auto& at, const auto& zi, auto& q, const auto& e) {
                float rho[sizeof(zi) / 4];
                residuals<DRAFT>(sh, w, at, zi, q, rho);
#pragma unroll
                for (int i = 0; i < (int)(sizeof(zi) / 4); ++i) {
                    const float g = rho[i] > 0.f ? rho[i] / e[i] : -1.f;
                    if (g > t.m || (g == t.m && at[i] < t.at)) t.m = g, t.at = at[i];
                }
            });
            t = join_all<kArgmax>(sh, t, 0.f, turn, ctas);
            if (t.m >= 0.f) token = t.at;
            if (t.m >= 0.f || !again) break;
            __syncthreads();
            if (tid == 0) sh.c[w.k - 1] = 0.f;
            __syncthreads();
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

template <typename T, bool DRAFT, bool VEC>
cudaError_t launch_verify(const VerifyArgs& p, int B, int ctas, cudaStream_t s) {
    // statistics ahead pay from the second node on that a walk visits, for what a whole row costs a CTA more than its share: a
    // chain of 8 over 32000 tokens 17 us and not 25; over 128000 25 to 29 and, as the walk goes, 19 to 38 without
    const bool ahead = p.max_nodes > 1 && p.max_nodes <= ctas && p.vocab <= kAheadVocab;
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
    return ahead ? cudaLaunchKernelEx(&cfg, k_verify<T, DRAFT, VEC, true>, p) : cudaLaunchKernelEx(&cfg, k_verify<T, DRAFT, VEC, false>, p);
}

template <typename T>
cudaError_t verify_of(const VerifyArgs& p, int B, int ctas, bool vec, cudaStream_t s) {
    if (p.draft) return vec ? launch_verify<T, true, true>(p, B, ctas, s) : launch_verify<T, true, false>(p, B, ctas, s);
    return vec ? launch_verify<T, false, true>(p, B, ctas, s) : launch_verify<T, false, false>(p, B, ctas, s);
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
    // as many CTAs a request as the SMs hold for the batch (two each), and no more than a row fills
    int ctas = 1;
    while (ctas < kMaxCluster && 2LL * ctas * B <= 2 * sms && vocab / (2 * ctas) >= 2 * kVerThreads) ctas *= 2;
    if (e == cudaSuccess) {
        const VerifyArgs p{logits, logits_stride, draft_stride, noise_stride, tokens, parents, node_offsets, draft_probs,
                           temperature, uniforms, noise, path, n_keep, next_token, vocab, T, max_nodes};
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        const bool vec = ((uintptr_t)logits | (uintptr_t)draft_probs | (uintptr_t)noise) % 16 == 0 && logits_stride % (dtype == ACE_BF16 ? 8 : 4) == 0 &&
                         (!draft_probs || draft_stride % 4 == 0) && noise_stride % 4 == 0;
        if (dtype == ACE_BF16) e = verify_of<__nv_bfloat16>(p, B, ctas, vec, s);
        else e = verify_of<float>(p, B, ctas, vec, s);
    }
    if (e != cudaSuccess)
        return ver_fail(ACE_ERR_CUDA, std::string("verify launch: ") + cudaGetErrorName(e) + " (" + cudaGetErrorString(e) + ")");
    return ACE_OK;
}
