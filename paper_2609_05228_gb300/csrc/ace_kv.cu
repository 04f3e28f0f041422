// ace_kv.cu — the paged key/value cache of the speculative decode step: handle, quantising write, read back,
// keeping of accepted rows; ancestor masks of trees; argument checks of the attention.
#include <math.h>

#include <string>

#include "ace_kv_device.cuh"

namespace {

using namespace ace;

ace_status kv_fail(ace_status st, const std::string& m) {
    set_last_error(m.c_str());
    return st;
}

ace_status kv_cuda(cudaError_t e, const char* where) {
    return kv_fail(ACE_ERR_CUDA, std::string(where) + ": " + cudaGetErrorName(e) + " (" + cudaGetErrorString(e) + ")");
}

// A launch goes to the current device: the cache's, or nothing is launched.
ace_status kv_here(const ace_kv* kv) {
    int dev = -1;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return kv_cuda(e, "cudaGetDevice");
    return dev == kv->device ? ACE_OK : kv_fail(ACE_ERR_INVALID_ARG, "the cache belongs to another device than the current one");
}

struct RowArgs {
    const void* src[2];                 // write: K and V
    long long token_stride[2], head_stride[2];
    void* dst[2];                       // read: K and V
    uint8_t* pool[2];
    uint8_t* scale[2];
    const int64_t* slots;
    uint32_t rows;                      // (layers *) T * 2 * H
    long long n_slots;                  // of a layer
    int T, H, D, page_size, page_shift;
    int* err;
};

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

// Write: e the least with amax 2^-e <= 448, scale byte e + 127, codes = the row's elements times 2^-e in e4m3 (the only
// rounding). LANES lanes (a power of two, at least D / 8) hold one row, 8 elements each: its largest magnitude is
// a shuffle reduction, nothing is read twice. Bound by memory: each group of lanes has kRowTurns neighbouring rows under way
// together, and the rows are not waited for by way of their slots. Write and read back of 16384 tokens (8 heads of 128, bf16
// to fp8): 51 us for 201 MB, 4.0 TB/s (46 with the rows in L2, 61 then with one row at a time).
constexpr int kRowTurns = 4;

// Row r of a call: (token, K or V, head), heads fastest.
struct RowAt {
    uint32_t th;                        // 2 * token + (V: 1)
    int h;
    __device__ __forceinline__ RowAt(uint32_t r, uint32_t H) : th(r / H), h((int)(r - r / H * H)) {}
    __device__ __forceinline__ void next(int H) {
        if (++h == H) h = 0, ++th;
    }
};

template <typename T, bool FP8, bool ALIGNED, int LANES>
__global__ void __launch_bounds__(256) k_kv_write(const __grid_constant__ RowArgs p) {
    const int sub = threadIdx.x % LANES;
    const bool in = sub * 8 < p.D;
    const uint32_t r0 = (blockIdx.x * (256 / LANES) + threadIdx.x / LANES) * kRowTurns;
    RowAt at(r0, p.H);
    long long slot[kRowTurns];
    Raw8<T> raw[kRowTurns];
#pragma unroll
    for (int j = 0; j < kRowTurns; ++j, at.next(p.H)) {
        const bool live = r0 + j < p.rows;
        const int kv = at.th & 1;
        const long long t = at.th >> 1;
        slot[j] = live ? p.slots[t] : -1;
        if (live && in) raw[j] = load8<T, ALIGNED>(static_cast<const T*>(p.src[kv]) + t * p.token_stride[kv] + at.h * p.head_stride[kv] + sub * 8);
        else raw[j] = Raw8<T>{};
    }
    at = RowAt(r0, p.H);
#pragma unroll
    for (int j = 0; j < kRowTurns; ++j, at.next(p.H)) {
        const int kv = at.th & 1;
        if (slot[j] >= p.n_slots) {
            if (sub == 0) atomicOr(p.err, kErrIndex);
            slot[j] = -1;
        }
        const long long row = slot[j] >= 0 ? pool_row(p, slot[j], at.h) : 0;
        const bool put = in && slot[j] >= 0;
        if constexpr (FP8) {
            float f[8], amax = 0.f;
            raw[j].to_float(f);
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
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) dst[i] = raw[j].w[i];
        }
    }
}

// Read: code times 2^e, rounded to the storage type; the same lanes and turns as the write.
template <typename T, bool FP8, int LANES>
__global__ void __launch_bounds__(256) k_kv_read(const __grid_constant__ RowArgs p) {
    const int sub = threadIdx.x % LANES;
    if (sub * 8 >= p.D) return;
    const uint32_t r0 = (blockIdx.x * (256 / LANES) + threadIdx.x / LANES) * kRowTurns;
    RowAt at(r0, p.H);
    long long row[kRowTurns];           // -1: zeros
#pragma unroll
    for (int j = 0; j < kRowTurns; ++j, at.next(p.H)) {
        row[j] = -1;
        if (r0 + j >= p.rows) continue;
        const uint32_t lt = at.th >> 1, layer = lt / (uint32_t)p.T;          // layer * T + token
        const long long slot = p.slots[lt - layer * p.T];
        if (slot >= p.n_slots) {
            if (sub == 0) atomicOr(p.err, kErrIndex);
        } else if (slot >= 0) {
            row[j] = layer * p.n_slots * p.H + pool_row(p, slot, at.h);
        }
    }
    Raw8<T> raw[FP8 ? 1 : kRowTurns];
    uint2 code[kRowTurns];
    uint8_t byte[kRowTurns];
    at = RowAt(r0, p.H);
#pragma unroll
    for (int j = 0; j < kRowTurns; ++j, at.next(p.H)) {
        const int kv = at.th & 1;
        if constexpr (FP8) {
            code[j] = make_uint2(0, 0);
            byte[j] = 1;
            if (row[j] >= 0) {
                code[j] = __ldg(reinterpret_cast<const uint2*>(p.pool[kv] + row[j] * p.D + sub * 8));
                byte[j] = __ldg(p.scale[kv] + row[j]);
            }
        } else {
            if (row[j] >= 0) raw[j] = load8<T, true>(reinterpret_cast<const T*>(p.pool[kv]) + row[j] * p.D + sub * 8);
            else raw[j] = Raw8<T>{};
        }
    }
    at = RowAt(r0, p.H);
#pragma unroll
    for (int j = 0; j < kRowTurns; ++j, at.next(p.H)) {
        if (r0 + j >= p.rows) break;
        T* dst = static_cast<T*>(p.dst[at.th & 1]) + ((long long)(at.th >> 1) * p.H + at.h) * p.D + sub * 8;
        if constexpr (FP8) {
            float f[8];
            e4m3x8_to_float(code[j], f);
            const float m = pow2_of_byte(byte[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= m;
            store8(dst, f);
        } else {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(dst)[i] = raw[j].w[i];
        }
    }
}

struct KeepArgs {
    uint8_t* pool[2];
    uint8_t* scale[2];                  // NULL: plain rows
    const int32_t* page_table;
    const int32_t* lens;
    const int32_t* path;
    const int32_t* n_keep;
    int32_t* new_lens;
    int max_pages, max_nodes, H, row_words, page_size, page_shift, n_pages, layers;   // row_words: 8- or 16-byte words of a row
    int* err;
};

constexpr int kKeepThreads = 256, kKeepWords = 4;

// Block (request, share of the layers and heads); W is a word of 8 or 16 bytes. The path is looked up once; then all rows'
// words, in the order (layer, head), node, move in passes. Rows move towards the front (path[i] >= i and
// increasing), so a pass that has read its words before it writes any never overwrites a word of a later pass. Bound by
// memory: 128 requests of up to 64 nodes, 48 layers of 8 heads of 128, bf16: 77 us for 352 MB, 4.6 TB/s (110 with a block a
// layer, which looked the path up again); 32 of 16, 16 layers of 4: 8.9 us on the device, most of it the path's chain of loads.
template <typename W>
__global__ void __launch_bounds__(kKeepThreads) k_kv_keep(const __grid_constant__ KeepArgs p) {
    __shared__ int src_row[kMaxNodes], dst_row[kMaxNodes];          // of head 0
    __shared__ int bad;
    const int b = blockIdx.x, tid = threadIdx.x;
    const int n = p.n_keep[b], len = p.lens[b];
    if (tid == 0) bad = n < 0 || n > p.max_nodes || len < 0;
    __syncthreads();
    if (!bad) {
        for (int i = tid; i < n; i += kKeepThreads) {
            const int32_t* path = p.path + (long long)b * p.max_nodes;
            const int at = path[i];
            bool ok = at >= 0 && at < kMaxNodes && (i == 0 || at > path[i - 1]);
            const long long sp = (long long)len + at, dp = (long long)len + i;
            ok = ok && sp < (long long)p.max_pages * p.page_size;
            if (ok) {
                const int32_t* table = p.page_table + (long long)b * p.max_pages;
                const int ps = table[sp >> p.page_shift], pd = table[dp >> p.page_shift];
                ok = ps >= 0 && ps < p.n_pages && pd >= 0 && pd < p.n_pages;
                src_row[i] = (ps * p.H << p.page_shift) + (int)(sp & (p.page_size - 1));
                dst_row[i] = (pd * p.H << p.page_shift) + (int)(dp & (p.page_size - 1));
            }
            if (!ok) bad = 1;
        }
    }
    __syncthreads();
    if (bad) {
        if (tid == 0) {
            atomicOr(p.err, kErrIndex);
            if (p.new_lens && blockIdx.y == 0) p.new_lens[b] = len;
        }
        return;
    }
    if (tid == 0 && p.new_lens && blockIdx.y == 0) p.new_lens[b] = len + n;
    if (n == 0) return;
    const int all = p.layers * p.H, lh0 = (int)((long long)all * blockIdx.y / gridDim.y), lh1 = (int)((long long)all * (blockIdx.y + 1) / gridDim.y);
    const long long layer_rows = (long long)p.n_pages * p.H << p.page_shift;
    // word `w` of the share: (layer, head), node, K or V, word of the row
    const uint32_t of_node = 2 * p.row_words, of_head = n * of_node;
    const uint64_t words = (uint64_t)(lh1 - lh0) * of_head;
    for (uint64_t w0 = 0; w0 < words; w0 += kKeepThreads * kKeepWords) {
        W v[kKeepWords];
        W* to[kKeepWords];
#pragma unroll
        for (int j = 0; j < kKeepWords; ++j) {
            const uint64_t w = w0 + j * kKeepThreads + tid;
            to[j] = nullptr;
            if (w < words) {
                const uint32_t lh = (uint32_t)w / of_head, rest = (uint32_t)w - lh * of_head, i = rest / of_node, u = rest - i * of_node;
                const int kv = u >= (uint32_t)p.row_words, layer = (lh0 + (int)lh) / p.H, h = lh0 + (int)lh - layer * p.H;
                if (src_row[i] != dst_row[i]) {
                    const long long head = layer * layer_rows + ((long long)h << p.page_shift);
                    W* pool = reinterpret_cast<W*>(p.pool[kv]) + (u - kv * p.row_words);
                    v[j] = pool[(head + src_row[i]) * p.row_words];
                    to[j] = pool + (head + dst_row[i]) * p.row_words;
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kKeepWords; ++j)
            if (to[j]) *to[j] = v[j];
    }
    if (p.scale[0]) {
        const uint32_t bytes = (uint32_t)(lh1 - lh0) * 2 * n;
        for (uint32_t w0 = 0; w0 < bytes; w0 += kKeepThreads) {
            const uint32_t w = w0 + tid, lh = w / (2 * n), rest = w - lh * 2 * n, i = rest >> 1;
            const int layer = (lh0 + (int)lh) / p.H, h = lh0 + (int)lh - layer * p.H;
            const long long head = layer * layer_rows + ((long long)h << p.page_shift);
            uint8_t v = 0;
            if (w < bytes) v = p.scale[rest & 1][head + src_row[i]];
            __syncthreads();
            if (w < bytes) p.scale[rest & 1][head + dst_row[i]] = v;
        }
    }
}

// Block per request: node i's chain of parents, walked in shared memory (a parent is below its node, so it ends). Bound by
// the launch and the deepest chain.
__global__ void __launch_bounds__(kMaxNodes) k_tree_mask(const int32_t* parents, const int32_t* node_offsets, int T,
                                                         int max_nodes, int words, unsigned long long* mask, int32_t* depth) {
    __shared__ int par[kMaxNodes];
    const int o0 = node_offsets[blockIdx.x], o1 = node_offsets[blockIdx.x + 1], i = threadIdx.x;
    if (o0 < 0 || o1 <= o0 || o1 > T || o1 - o0 > max_nodes) return;
    const int n = o1 - o0;
    if (i < n) {
        const int q = parents[o0 + i];
        par[i] = q >= 0 && q < i ? q : -1;
    }
    __syncthreads();
    if (i >= n) return;
    unsigned long long m[kMaxNodes / 64] = {};
    int d = -1;
    for (int j = i; j >= 0; j = par[j]) {
#pragma unroll
        for (int w = 0; w < kMaxNodes / 64; ++w)
            if (w == j >> 6) m[w] |= 1ull << (j & 63);
        ++d;
    }
#pragma unroll
    for (int w = 0; w < kMaxNodes / 64; ++w)
        if (w < words) mask[(long long)(o0 + i) * words + w] = m[w];
    if (depth) depth[o0 + i] = d;
}

int log2_of(int x) {
    int s = 0;
    while (1 << s < x) ++s;
    return s;
}

RowArgs row_args(const ace_kv* kv, int layer, const int64_t* slots, int T) {
    RowArgs p{};
    const ace_kv_desc& D = kv->desc;
    const long long rows = (long long)D.n_pages * D.n_kv_heads * D.page_size;
    const int row_bytes = D.head_dim * (D.format == ACE_KV_FP8 ? 1 : kv->elem);
    p.pool[0] = static_cast<uint8_t*>(kv->k_pool) + rows * row_bytes * layer;
    p.pool[1] = static_cast<uint8_t*>(kv->v_pool) + rows * row_bytes * layer;
    if (D.format == ACE_KV_FP8) {
        p.scale[0] = kv->k_scale + rows * layer;
        p.scale[1] = kv->v_scale + rows * layer;
    }
    p.slots = slots;
    p.n_slots = kv->slots;
    p.T = T;
    p.H = D.n_kv_heads;
    p.D = D.head_dim;
    p.page_size = D.page_size;
    p.page_shift = log2_of(D.page_size);
    p.err = kv->err;
    return p;
}

// Blocks for all rows, `groups` groups of lanes a block.
unsigned row_grid(uint32_t rows, int groups) { return (rows + groups * kRowTurns - 1) / (groups * kRowTurns); }

template <typename T, bool FP8, bool ALIGNED>
void write_rows(const RowArgs& p, cudaStream_t s) {
    if (p.D <= 64) k_kv_write<T, FP8, ALIGNED, 8><<<row_grid(p.rows, 32), 256, 0, s>>>(p);
    else if (p.D <= 128) k_kv_write<T, FP8, ALIGNED, 16><<<row_grid(p.rows, 16), 256, 0, s>>>(p);
    else k_kv_write<T, FP8, ALIGNED, 32><<<row_grid(p.rows, 8), 256, 0, s>>>(p);
}

template <typename T, bool FP8>
void read_rows(const RowArgs& p, cudaStream_t s) {
    if (p.D <= 64) k_kv_read<T, FP8, 8><<<row_grid(p.rows, 32), 256, 0, s>>>(p);
    else if (p.D <= 128) k_kv_read<T, FP8, 16><<<row_grid(p.rows, 16), 256, 0, s>>>(p);
    else k_kv_read<T, FP8, 32><<<row_grid(p.rows, 8), 256, 0, s>>>(p);
}

constexpr long long kMaxRows = 1LL << 30;       // of a write or read call: row numbers are 32-bit

bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }

}  // namespace

extern "C" {

ace_status ace_kv_create(const ace_kv_desc* desc, void* k_pool, void* v_pool, void* k_scale, void* v_scale,
                         void* stream, ace_kv** out_kv) {
    if (!desc || !out_kv) return kv_fail(ACE_ERR_INVALID_ARG, "desc and out_kv must be non-NULL");
    *out_kv = nullptr;
    const ace_kv_desc& D = *desc;
    if (D.layers <= 0 || D.n_pages <= 0 || D.page_size <= 0 || D.n_kv_heads <= 0 || D.head_dim <= 0)
        return kv_fail(ACE_ERR_INVALID_ARG, "layers, n_pages, page_size, n_kv_heads and head_dim must be positive");
    if (D.dtype != ACE_BF16 && D.dtype != ACE_F32) return kv_fail(ACE_ERR_INVALID_ARG, "unknown dtype");
    if (D.format != ACE_KV_PLAIN && D.format != ACE_KV_FP8) return kv_fail(ACE_ERR_INVALID_ARG, "unknown cache format");
    if (D.page_size < 16 || D.page_size > 256 || (D.page_size & (D.page_size - 1)))
        return kv_fail(ACE_ERR_UNSUPPORTED, "page_size must be 16, 32, 64, 128 or 256");
    if (D.head_dim % 8 || D.head_dim > kMaxHeadDim)
        return kv_fail(ACE_ERR_UNSUPPORTED, "head_dim must be a multiple of 8, at most 256");
    if (!k_pool || !v_pool) return kv_fail(ACE_ERR_INVALID_ARG, "k_pool and v_pool must be non-NULL");
    if (!aligned16(k_pool) || !aligned16(v_pool)) return kv_fail(ACE_ERR_INVALID_ARG, "the pools must be 16-byte aligned");
    if (D.format == ACE_KV_FP8 && (!k_scale || !v_scale))
        return kv_fail(ACE_ERR_INVALID_ARG, "an fp8 cache needs k_scale and v_scale");
    if (D.format == ACE_KV_FP8 && (!aligned16(k_scale) || !aligned16(v_scale)))     // the attention reads four at a time
        return kv_fail(ACE_ERR_INVALID_ARG, "the scales must be 16-byte aligned");
    // products one at a time, each below 2^31 before the next
    long long rows = (long long)D.n_pages * D.page_size;
    if (rows <= INT32_MAX) rows *= D.n_kv_heads;
    if (rows <= INT32_MAX) rows *= D.layers;
    if (rows > INT32_MAX) return kv_fail(ACE_ERR_UNSUPPORTED, "layers * n_pages * n_kv_heads * page_size must be below 2^31");

    ace_kv* kv = new ace_kv();
    kv->desc = D;
    kv->elem = D.dtype == ACE_BF16 ? 2 : 4;
    kv->k_pool = k_pool;
    kv->v_pool = v_pool;
    kv->k_scale = static_cast<uint8_t*>(D.format == ACE_KV_FP8 ? k_scale : nullptr);
    kv->v_scale = static_cast<uint8_t*>(D.format == ACE_KV_FP8 ? v_scale : nullptr);
    kv->slots = (long long)D.n_pages * D.page_size;
    kv->last_stream = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaGetDevice(&kv->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&kv->num_sms, cudaDevAttrMultiProcessorCount, kv->device);
    if (e == cudaSuccess) e = attn_init(kv);
    if (e == cudaSuccess) e = cudaStreamSynchronize(kv->last_stream);
    if (e != cudaSuccess) {
        ace_kv_destroy(kv);
        if (e == cudaErrorMemoryAllocation) {
            cudaGetLastError();
            return kv_fail(ACE_ERR_OOM, "cudaMalloc failed for the attention workspace");
        }
        return kv_cuda(e, "ace_kv_create");
    }
    *out_kv = kv;
    return ACE_OK;
}

void ace_kv_destroy(ace_kv* kv) {
    if (!kv) return;
    cudaDeviceSynchronize();
    if (kv->block) cudaFree(kv->block);
    delete kv;
}

ace_status ace_kv_sync(ace_kv* kv) {
    if (!kv) return kv_fail(ACE_ERR_INVALID_ARG, "cache is NULL");
    cudaError_t e = cudaStreamSynchronize(kv->last_stream);
    if (e != cudaSuccess) return kv_cuda(e, "synchronize");
    int err = 0;
    if ((e = cudaMemcpy(&err, kv->err, sizeof(int), cudaMemcpyDeviceToHost)) != cudaSuccess) return kv_cuda(e, "read device error word");
    if (!err) return ACE_OK;
    if ((e = cudaMemset(kv->err, 0, sizeof(int))) != cudaSuccess) return kv_cuda(e, "clear device error word");
    if (err & kErrTimeout) {
        return kv_fail(ACE_ERR_TIMEOUT, "a bounded device wait ran out");
    }
    return kv_fail(ACE_ERR_INVALID_ARG, "a slot, page, length, offset or path in device memory was out of range and left out");
}

ace_status ace_kv_write(ace_kv* kv, int layer, const void* k, long long k_token_stride, long long k_head_stride,
                        const void* v, long long v_token_stride, long long v_head_stride, const int64_t* slots, int T,
                        void* stream) {
    if (!kv) return kv_fail(ACE_ERR_INVALID_ARG, "cache is NULL");
    if (layer < 0 || layer >= kv->desc.layers) return kv_fail(ACE_ERR_INVALID_ARG, "layer out of range");
    if (T < 0) return kv_fail(ACE_ERR_INVALID_ARG, "T must be >= 0");
    if (T > 0 && (!k || !v || !slots)) return kv_fail(ACE_ERR_INVALID_ARG, "k, v and slots must be non-NULL");
    if (k_token_stride < 0 || k_head_stride < 0 || v_token_stride < 0 || v_head_stride < 0)
        return kv_fail(ACE_ERR_INVALID_ARG, "strides must be >= 0");
    if ((uintptr_t)k % kv->elem || (uintptr_t)v % kv->elem) return kv_fail(ACE_ERR_INVALID_ARG, "k and v must be aligned to their type");
    if (const ace_status st = kv_here(kv)) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    kv->last_stream = s;
    if (T == 0) return ACE_OK;
    RowArgs p = row_args(kv, layer, slots, T);
    if (2LL * T * p.H > kMaxRows) return kv_fail(ACE_ERR_UNSUPPORTED, "a call writes at most 2^30 rows (2 T n_kv_heads)");
    p.rows = 2u * T * p.H;
    p.src[0] = k;
    p.src[1] = v;
    p.token_stride[0] = k_token_stride;
    p.token_stride[1] = v_token_stride;
    p.head_stride[0] = k_head_stride;
    p.head_stride[1] = v_head_stride;
    // 16-byte loads where every row begins on 16 bytes, single elements elsewhere
    const long long vec = 16 / kv->elem;
    const bool al = aligned16(k) && aligned16(v) && k_token_stride % vec == 0 && k_head_stride % vec == 0 &&
                    v_token_stride % vec == 0 && v_head_stride % vec == 0;
    const bool fp8 = kv->desc.format == ACE_KV_FP8;
    if (kv->desc.dtype == ACE_BF16) {
        if (fp8) al ? write_rows<__nv_bfloat16, true, true>(p, s) : write_rows<__nv_bfloat16, true, false>(p, s);
        else al ? write_rows<__nv_bfloat16, false, true>(p, s) : write_rows<__nv_bfloat16, false, false>(p, s);
    } else {
        if (fp8) al ? write_rows<float, true, true>(p, s) : write_rows<float, true, false>(p, s);
        else al ? write_rows<float, false, true>(p, s) : write_rows<float, false, false>(p, s);
    }
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? ACE_OK : kv_cuda(e, "cache write launch");
}

ace_status ace_kv_read(ace_kv* kv, int layer, const int64_t* slots, int T, void* k_out, void* v_out, void* stream) {
    if (!kv) return kv_fail(ACE_ERR_INVALID_ARG, "cache is NULL");
    if (layer < -1 || layer >= kv->desc.layers) return kv_fail(ACE_ERR_INVALID_ARG, "layer out of range");
    if (T < 0) return kv_fail(ACE_ERR_INVALID_ARG, "T must be >= 0");
    if (T > 0 && (!k_out || !v_out || !slots)) return kv_fail(ACE_ERR_INVALID_ARG, "k_out, v_out and slots must be non-NULL");
    if (!aligned16(k_out) || !aligned16(v_out)) return kv_fail(ACE_ERR_INVALID_ARG, "k_out and v_out must be 16-byte aligned");
    if (const ace_status st = kv_here(kv)) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    kv->last_stream = s;
    if (T == 0) return ACE_OK;
    RowArgs p = row_args(kv, layer < 0 ? 0 : layer, slots, T);
    const long long rows = 2LL * T * p.H * (layer < 0 ? kv->desc.layers : 1);
    if (rows > kMaxRows) return kv_fail(ACE_ERR_UNSUPPORTED, "a call reads at most 2^30 rows (2 T n_kv_heads layers)");
    p.rows = (uint32_t)rows;
    p.dst[0] = k_out;
    p.dst[1] = v_out;
    const bool fp8 = kv->desc.format == ACE_KV_FP8;
    if (kv->desc.dtype == ACE_BF16) fp8 ? read_rows<__nv_bfloat16, true>(p, s) : read_rows<__nv_bfloat16, false>(p, s);
    else fp8 ? read_rows<float, true>(p, s) : read_rows<float, false>(p, s);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? ACE_OK : kv_cuda(e, "cache read launch");
}

ace_status ace_kv_keep(ace_kv* kv, const int32_t* page_table, int max_pages, const int32_t* lens, const int32_t* path,
                       int max_nodes, const int32_t* n_keep, int B, int32_t* new_lens, void* stream) {
    if (!kv) return kv_fail(ACE_ERR_INVALID_ARG, "cache is NULL");
    if (B < 0 || max_pages < 1) return kv_fail(ACE_ERR_INVALID_ARG, "B must be >= 0 and max_pages >= 1");
    if (max_nodes < 1 || max_nodes > kMaxNodes) return kv_fail(ACE_ERR_INVALID_ARG, "max_nodes must be in [1, 256]");
    if (B > 0 && (!page_table || !lens || !path || !n_keep))
        return kv_fail(ACE_ERR_INVALID_ARG, "page_table, lens, path and n_keep must be non-NULL");
    if (new_lens && new_lens == lens) return kv_fail(ACE_ERR_INVALID_ARG, "new_lens must not alias lens");
    if ((long long)kv->desc.layers * kv->desc.n_kv_heads > 65535)
        return kv_fail(ACE_ERR_UNSUPPORTED, "layers * n_kv_heads must be at most 65535");
    if (const ace_status st = kv_here(kv)) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    kv->last_stream = s;
    if (B == 0) return ACE_OK;
    const RowArgs r = row_args(kv, 0, nullptr, 0);
    const ace_kv_desc& D = kv->desc;
    KeepArgs p{};
    for (int i = 0; i < 2; ++i) p.pool[i] = r.pool[i], p.scale[i] = r.scale[i];
    p.page_table = page_table;
    p.lens = lens;
    p.path = path;
    p.n_keep = n_keep;
    p.max_pages = max_pages;
    p.max_nodes = max_nodes;
    p.H = D.n_kv_heads;
    const int row_bytes = D.head_dim * (D.format == ACE_KV_FP8 ? 1 : kv->elem), word = row_bytes % 16 ? 8 : 16;
    p.row_words = row_bytes / word;
    p.page_size = D.page_size;
    p.page_shift = r.page_shift;
    p.n_pages = D.n_pages;
    p.layers = D.layers;
    p.err = kv->err;
    p.new_lens = new_lens;
    // about eight blocks an SM, or a block for every layer and head
    const int all = D.layers * D.n_kv_heads;
    long long shares = (8LL * kv->num_sms + B - 1) / B;
    if (shares > all) shares = all;
    const dim3 grid(B, (unsigned)shares);
    if (word == 16) k_kv_keep<uint4><<<grid, kKeepThreads, 0, s>>>(p);
    else k_kv_keep<uint2><<<grid, kKeepThreads, 0, s>>>(p);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? ACE_OK : kv_cuda(e, "cache keep launch");
}

ace_status ace_tree_mask(const int32_t* parents, const int32_t* node_offsets, int B, int max_nodes, uint64_t* mask,
                         int32_t* depth, void* stream) {
    return ace_tree_mask_rows(parents, node_offsets, B, INT32_MAX, max_nodes, mask, depth, stream);
}

ace_status ace_tree_mask_rows(const int32_t* parents, const int32_t* node_offsets, int B, int T, int max_nodes,
                              uint64_t* mask, int32_t* depth, void* stream) {
    if (B < 0 || T < 0) return kv_fail(ACE_ERR_INVALID_ARG, "B and T must be >= 0");
    if (max_nodes < 1 || max_nodes > kMaxNodes) return kv_fail(ACE_ERR_INVALID_ARG, "max_nodes must be in [1, 256]");
    if (B == 0 || T == 0) return ACE_OK;
    if (!parents || !node_offsets || !mask) return kv_fail(ACE_ERR_INVALID_ARG, "parents, node_offsets and mask must be non-NULL");
    k_tree_mask<<<B, (max_nodes + 31) / 32 * 32, 0, static_cast<cudaStream_t>(stream)>>>(
        parents, node_offsets, T, max_nodes, (max_nodes + 63) / 64, reinterpret_cast<unsigned long long*>(mask), depth);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? ACE_OK : kv_cuda(e, "tree mask launch");
}

ace_status ace_tree_attention(ace_kv* kv, int layer, const void* q, long long q_token_stride, long long q_head_stride,
                              int n_heads, const int32_t* page_table, int max_pages, const int32_t* lens,
                              const int32_t* node_offsets, const uint64_t* mask, int B, int T, int max_nodes,
                              float scale, void* out, float* lse, void* stream) {
    if (!kv) return kv_fail(ACE_ERR_INVALID_ARG, "cache is NULL");
    const ace_kv_desc& D = kv->desc;
    if (layer < 0 || layer >= D.layers) return kv_fail(ACE_ERR_INVALID_ARG, "layer out of range");
    if (n_heads < 1 || n_heads % D.n_kv_heads) return kv_fail(ACE_ERR_INVALID_ARG, "n_heads must be a multiple of n_kv_heads");
    if (B < 0 || T < 0 || max_pages < 1) return kv_fail(ACE_ERR_INVALID_ARG, "B and T must be >= 0 and max_pages >= 1");
    if (max_nodes < 1 || max_nodes > kMaxNodes) return kv_fail(ACE_ERR_INVALID_ARG, "max_nodes must be in [1, 256]");
    if ((long long)max_nodes * (n_heads / D.n_kv_heads) > (1 << 24)) return kv_fail(ACE_ERR_INVALID_ARG, "n_heads too large");
    if (!isfinite(scale)) return kv_fail(ACE_ERR_INVALID_ARG, "scale must be finite");
    if (q_token_stride < 0 || q_head_stride < 0) return kv_fail(ACE_ERR_INVALID_ARG, "strides must be >= 0");
    if (B > 0 && T > 0 && (!q || !out || !page_table || !lens || !node_offsets))
        return kv_fail(ACE_ERR_INVALID_ARG, "q, out, page_table, lens and node_offsets must be non-NULL");
    if (!aligned16(out)) return kv_fail(ACE_ERR_INVALID_ARG, "out must be 16-byte aligned");
    if ((uintptr_t)q % kv->elem) return kv_fail(ACE_ERR_INVALID_ARG, "q must be aligned to its type");
    if (const ace_status st = kv_here(kv)) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    kv->last_stream = s;
    if (B == 0 || T == 0) return ACE_OK;
    const RowArgs r = row_args(kv, layer, nullptr, 0);
    AttnArgs a{};
    a.q = q;
    a.q_token_stride = q_token_stride;
    a.q_head_stride = q_head_stride;
    a.k_pool = r.pool[0];
    a.v_pool = r.pool[1];
    a.k_scale = r.scale[0];
    a.v_scale = r.scale[1];
    a.page_table = page_table;
    a.lens = lens;
    a.node_offsets = node_offsets;
    a.mask = reinterpret_cast<const unsigned long long*>(mask);
    a.out = out;
    a.lse = lse;
    a.B = B;
    a.T = T;
    a.max_nodes = max_nodes;
    a.words = (max_nodes + 63) / 64;
    a.max_pages = max_pages;
    a.n_heads = n_heads;
    a.kv_heads = D.n_kv_heads;
    a.group = n_heads / D.n_kv_heads;
    a.head_dim = D.head_dim;
    a.page_size = D.page_size;
    a.page_shift = r.page_shift;
    a.n_pages = D.n_pages;
    a.row0 = (int)((long long)layer * D.n_pages * D.n_kv_heads * D.page_size);
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.ws = kv->ws;
    a.err = kv->err;
    const cudaError_t e = launch_tree_attention(kv, a, s);
    return e == cudaSuccess ? ACE_OK : kv_cuda(e, "tree attention launch");
}

}  // extern "C"
