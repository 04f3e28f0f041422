// ace_kv.h — the cache handle and what the speculative decode step's kernels share.
#pragma once

#include <string>

#include "ace_internal.h"

namespace ace {

// Bit of ace_kv::err beside the layer's bits: a slot, page, length, offset or path in device memory
// points outside its array (what it names was left out).
constexpr int kErrIndex = 8;

constexpr int kMaxNodes = 256;          // nodes of a request's tree
constexpr int kMaxHeadDim = 256;
constexpr int kGroup4 = 32;             // elements that share a scale in ACE_KV_INT4

__host__ __device__ constexpr int groups4(int D) { return (D + kGroup4 - 1) / kGroup4; }
// Bytes of a cached row, and of its scale or scales.
__host__ __device__ constexpr int row_bytes(int format, int D, int elem) { return format == ACE_KV_INT4 ? D / 2 : format == ACE_KV_FP8 ? D : D * elem; }
__host__ __device__ constexpr int scale_bytes(int format, int D) { return format == ACE_KV_INT4 ? 2 * groups4(D) : format == ACE_KV_FP8 ? 1 : 0; }

// A CTA's part of a unit.
struct Segment {
    int b, head, row0, rows;        // request, kv head, first row of the unit (node * G + g) and its rows
    int node0, len, n;              // the request
    int tile0, tile1;               // key tiles of this CTA
    int part;                       // partial result slot, -1: the whole unit is here
    int first, last;                // CTAs that share the unit
};

// Workspace of the attention kernels: a CTA's share of the work begins and ends inside a unit (request, head,
// row block), so two partial results a CTA are enough for any batch.
struct AttnWorkspace {
    float* part_o = nullptr;            // [2 * ctas][rows of a unit, D] unnormalised outputs (part_place)
    float2* part_ml = nullptr;          // [2 * ctas][rows of a unit] running maximum (base 2) and sum
    Segment* unit = nullptr;            // [ctas] the cut unit that begins in a CTA (rows = 0: none)
};

// Workspace of the calls that plan on the device which pages move.
struct PageWorkspace {
    int* count = nullptr;               // moves of the last plan
    int3* move = nullptr;               // [n_pages] source, destination, rows of each head
    int* mark = nullptr;                // [2 * n_pages] zeros between calls
    int* list = nullptr;                // [n_pages]
};

struct KvMaps {                         // tensor-core attention (head sizes 64 and 128, bf16)
    CUtensorMap k, v;
};

}  // namespace ace

struct ace_kv {
    ace_kv_desc desc;
    int device = 0;
    int num_sms = 1;
    int elem = 2;                       // bytes of dtype
    void* k_pool = nullptr;
    void* v_pool = nullptr;
    uint8_t* k_scale = nullptr;
    uint8_t* v_scale = nullptr;
    long long slots = 0;                // n_pages * page_size, per layer
    void* block = nullptr;              // one allocation for what follows
    int* err = nullptr;
    ace::AttnWorkspace ws;
    ace::PageWorkspace pages;
    int core_ctas_per_sm = 1;           // CUDA-core attention
    bool tc = false;                    // tensor-core attention in use
    ace::KvMaps maps;
    cudaStream_t last_stream = nullptr;
};

namespace ace {

ace_status kv_fail(ace_status st, const std::string& message);
ace_status kv_cuda(cudaError_t e, const char* where);
// A launch goes to the current device: that of the `what`, or nothing is launched.
ace_status on_device(int device, const char* what);
inline bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }

constexpr long long kMaxRows = 1LL << 30;       // of a write or read call: row numbers are 32-bit

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

// What a call says of the layer and the tokens' slots; src, strides, dst and rows are left to it.
RowArgs row_args(const ace_kv* kv, int layer, const int64_t* slots, int T);

struct AttnArgs {
    const void* q;
    long long q_token_stride, q_head_stride;
    const void* k_pool;                 // of the layer
    const void* v_pool;
    const uint8_t* k_scale;
    const uint8_t* v_scale;
    const int32_t* page_table;
    const int32_t* lens;
    const int32_t* node_offsets;
    const unsigned long long* mask;     // NULL: a chain
    void* out;
    float* lse;
    int B, T, max_nodes, words, max_pages;
    int n_heads, kv_heads, group, head_dim, page_size, page_shift, n_pages;
    int row0;                           // the layer's first row in the tensor maps
    float scale_log2;                   // scale * log2(e)
    AttnWorkspace ws;
    int* err;
};

cudaError_t attn_init(ace_kv* kv);      // kernel attributes, workspace, tensor maps
cudaError_t launch_tree_attention(const ace_kv* kv, const AttnArgs& a, cudaStream_t s);
// Joins the partial results of the kernel before: units of `rows` rows, `ctas` CTAs.
cudaError_t launch_join(const AttnArgs& a, int dtype, bool by_dims, int rows, int ctas, cudaStream_t s);
// tensor-core kernel (ace_attn_tc.cu): bf16, head sizes 64 and 128
constexpr int kTcMaxRows = 256;         // rows of a unit
bool attn_tc_supported(const ace_kv* kv);
cudaError_t attn_tc_init(ace_kv* kv);
cudaError_t launch_tree_attention_tc(const ace_kv* kv, const AttnArgs& a, cudaStream_t s);
// the same for few rows a unit (ace_attn_few.cu)
constexpr int kFewRows = 32;
cudaError_t attn_few_init(const ace_kv* kv);
cudaError_t launch_attn_few(const ace_kv* kv, const AttnArgs& a, cudaStream_t s);
// caches in 4 bits (ace_attn_q4.cu): two CTAs an SM, up to 16 rows a unit 60 to 90 us for 64 users where the tcgen05 kernel (ace_attn_tc.cu)
// takes 119 for any up to 32. With 32 rows a warp it would have no registers left for the chains to overlap.
constexpr int kFewRows4 = 16;
cudaError_t attn_q4_init(const ace_kv* kv);
cudaError_t launch_attn_q4(const ace_kv* kv, const AttnArgs& a, cudaStream_t s);
}  // namespace ace
