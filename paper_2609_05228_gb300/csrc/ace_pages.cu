// ace_pages.cu — the life of the cache's pages: forking of requests that share them, room for new tokens (fresh pages, and copies
// of partly filled ones that others hold too), release, compaction, copies. Pages are counted: refs[page] entries of
// page tables name it, 0 is free, so that nothing has to be kept in order when requests go.
//
// A call plans on the device, in one block, which pages move (the tables are a few thousand words, and fresh pages are handed out in
// the pages' order, so that the same call gives the same tables); a kernel after it, over all SMs, moves their rows: a warp a
// (page, layer, K or V, head), whose rows lie on end. The plan is bound by its chain of loads and barriers (128 requests: 11 us, with
// nothing in L2), the moves by memory (1000 pages of 16 layers, 4 heads of 128 in 4 bits: 168 us for 1.1 GB, 6.7 TB/s).
#include "ace_kv_device.cuh"

namespace {

using namespace ace;

constexpr int kPlan = 1024;             // threads of a plan
constexpr int kPlanRows = 8192;         // requests of a reserve
constexpr int kScan = 16;               // pages a thread of a scan

// Exclusive sums over a block of kPlan threads of x, and the total in `all`. sums: kPlan / 32 + 1 ints of shared memory.
__device__ __forceinline__ int block_scan(int x, int* sums, int& all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int sum = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += up;
    }
    __syncthreads();                    // sums may be in use
    if (lane == 31) sums[warp] = sum;
    __syncthreads();
    if (warp == 0) {
        int s = sums[lane];
        const int mine = s;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += up;
        }
        sums[lane] = s - mine;
        if (lane == 31) sums[32] = s;
    }
    __syncthreads();
    all = sums[32];
    return sums[warp] + sum - x;
}

// Calls found(page, rank) for the pages from `page0` on, one round of kPlan * kScan, that `is` holds for, in their order; ranks
// begin at `rank`, which moves on. A warp has kScan words of 32 pages, read on end.
template <typename Is, typename Found>
__device__ __forceinline__ void scan_round(int page0, int n_pages, int* sums, int& rank, Is is, Found found) {
    const int lane = threadIdx.x & 31, first = page0 + (threadIdx.x >> 5) * (32 * kScan) + lane;
    bool has[kScan];
#pragma unroll
    for (int i = 0; i < kScan; ++i) has[i] = first + 32 * i < n_pages && is(first + 32 * i);
    int mine = 0;
    unsigned word[kScan];
#pragma unroll
    for (int i = 0; i < kScan; ++i) {
        word[i] = __ballot_sync(0xffffffffu, has[i]);
        mine += __popc(word[i]);
    }
    int all;
    const int before = block_scan(lane == 0 ? mine : 0, sums, all);
    int at = rank + __shfl_sync(0xffffffffu, before, 0);
#pragma unroll
    for (int i = 0; i < kScan; ++i) {
        if (has[i]) found(first + 32 * i, at + __popc(word[i] & lanemask_lt()));
        at += __popc(word[i]);
    }
    rank += all;
}

__device__ __forceinline__ bool exists(int page, int n_pages) { return page >= 0 && page < n_pages; }

struct ForkArgs {
    const int32_t* table;
    const int32_t* lens;
    const int32_t* parents;
    int32_t* refs;
    int32_t* new_table;
    int32_t* new_lens;
    int B, B_out, max_pages, page_shift, n_pages;
    int* err;
};

// Block per row of the old tables, whose pages lose a holder, and of the new ones, whose pages gain one.
__global__ void __launch_bounds__(128) k_fork(const __grid_constant__ ForkArgs p) {
    const int b = blockIdx.x;
    bool bad = false;
    if (b < p.B) {
        const int32_t* row = p.table + (long long)b * p.max_pages;
        for (int i = threadIdx.x; i < p.max_pages; i += blockDim.x) {
            const int page = row[i];
            if (exists(page, p.n_pages)) atomicSub(&p.refs[page], 1);
            else bad = bad || page >= 0;
        }
    }
    if (b < p.B_out) {
        const int parent = p.parents[b];
        int len = 0;
        if (parent >= p.B) bad = true;
        else if (parent >= 0) len = p.lens[parent];
        if (len < 0 || len > (long long)p.max_pages << p.page_shift) len = 0, bad = true;
        const int held = (int)(((long long)len + (1 << p.page_shift) - 1) >> p.page_shift);
        const int32_t* row = p.table + (long long)parent * p.max_pages;
        int32_t* out = p.new_table + (long long)b * p.max_pages;
        for (int i = threadIdx.x; i < p.max_pages; i += blockDim.x) {
            int page = i < held ? row[i] : -1;
            if (exists(page, p.n_pages)) atomicAdd(&p.refs[page], 1);
            else bad = bad || i < held, page = -1;
            out[i] = page;
        }
        if (threadIdx.x == 0) p.new_lens[b] = len;
    }
    if (bad) atomicOr(p.err, kErrIndex);
}

// Block per request that may have ended.
__global__ void __launch_bounds__(128) k_release(int32_t* table, int max_pages, int32_t* lens, const int32_t* ended, int32_t* refs, int n_pages,
                                                 int* err) {
    if (ended[blockIdx.x] == 0) return;
    int32_t* row = table + (long long)blockIdx.x * max_pages;
    bool bad = false;
    for (int i = threadIdx.x; i < max_pages; i += blockDim.x) {
        const int page = row[i];
        if (page < 0) continue;
        if (page < n_pages) atomicSub(&refs[page], 1);
        else bad = true;
        row[i] = -1;
    }
    if (threadIdx.x == 0) lens[blockIdx.x] = 0;
    if (bad) atomicOr(err, kErrIndex);
}

struct ReserveArgs {
    int32_t* table;
    const int32_t* lens;
    const int32_t* grow;
    int32_t* refs;
    int32_t* missing;
    int B, max_pages, page_shift, n_pages;
    PageWorkspace ws;
    int* err;
};

// What a request asks for: entries `first` .. `end` - 1 of its row are to name pages, and `part` is its partly filled page (-1:
// none), entry first - 1. False: it is left out.
struct Want {
    int first, end, part;
    __device__ __forceinline__ bool of(const ReserveArgs& p, int b) {
        const int len = p.lens[b], grow = p.grow[b];
        first = end = 0;
        part = -1;
        if (grow == 0) return true;
        if (len < 0 || grow < 0 || (long long)len + grow > (long long)p.max_pages << p.page_shift) return false;
        const int rows = 1 << p.page_shift;
        first = (int)(((long long)len + rows - 1) >> p.page_shift);
        end = (int)(((long long)len + grow + rows - 1) >> p.page_shift);
        if (len & (rows - 1)) {
            part = p.table[(long long)b * p.max_pages + first - 1];
            if (!exists(part, p.n_pages)) {
                part = -1;
                end = first;
                return false;
            }
        }
        return true;
    }
};

constexpr int kShort = 16;              // entries of a row that one thread looks through

// One block: a thread a request where few entries are asked for, a warp where they are many (a prompt's). Of a request that asks for n
// pages, need holds 2 n, and one more where the first of them is a copy; then, in place of n, its sum over the requests before it.
__global__ void __launch_bounds__(kPlan) k_reserve(const __grid_constant__ ReserveArgs p) {
    __shared__ int need[kPlanRows];
    __shared__ int sums[33], moves, any_long;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int* holders = p.ws.mark;           // requests that grow in a page
    int* last = p.ws.mark + p.n_pages;  // the last of them, + 1
    bool bad = false;
    if (tid == 0) moves = any_long = 0;
    __syncthreads();
    Want w;
    for (int b = tid; b < p.B; b += kPlan) {
        if (!w.of(p, b)) bad = true;
        if (w.part >= 0) {
            atomicAdd(&holders[w.part], 1);
            atomicMax(&last[w.part], b + 1);
        }
        int n = -1;
        if (w.end - w.first <= kShort) {
            n = 0;
            for (int i = w.first; i < w.end; ++i) {
                const int page = p.table[(long long)b * p.max_pages + i];
                n += page < 0;
                bad = bad || page >= p.n_pages;
            }
        } else {
            any_long = 1;
        }
        need[b] = n;
    }
    __syncthreads();
    if (any_long)
        for (int b = warp; b < p.B; b += kPlan / 32) {
            if (need[b] >= 0) continue;
            w.of(p, b);
            int n = 0;
            for (int i = w.first + lane; i < w.end; i += 32) {
                const int page = p.table[(long long)b * p.max_pages + i];
                n += page < 0;
                bad = bad || page >= p.n_pages;
            }
            n = warp_sum_int(n);
            __syncwarp();
            if (lane == 0) need[b] = n;
        }
    if (bad) atomicOr(p.err, kErrIndex);
    __syncthreads();
    for (int b = tid; b < p.B; b += kPlan) {
        w.of(p, b);
        int copy = 0;
        if (w.part >= 0) {
            const int refs = p.refs[w.part];
            copy = refs > 1 && !(__ldcg(&holders[w.part]) == refs && __ldcg(&last[w.part]) == b + 1);
        }
        need[b] = 2 * (need[b] + copy) + copy;
    }
    __syncthreads();
    int total = 0;
    for (int b0 = 0; b0 < p.B; b0 += kPlan) {
        const int b = b0 + tid, x = b < p.B ? need[b] : 0;
        int all;
        const int before = block_scan(x >> 1, sums, all);
        if (b < p.B) need[b] = 2 * (total + before) + (x & 1);
        total += all;
    }
    // the lowest free pages, as many as are asked for
    int found = 0;
    for (int page0 = 0; page0 < p.n_pages && found < total; page0 += kPlan * kScan)
        scan_round(page0, p.n_pages, sums, found, [&](int page) { return p.refs[page] == 0; },
                   [&](int page, int rank) {
                       if (rank < total) p.ws.list[rank] = page;
                   });
    __syncthreads();
    const bool enough = found >= total;
    if (tid == 0) *p.missing = enough ? 0 : total - found;
    // a request's fresh pages into its row; by one thread, or by a warp
    auto give = [&](int b, bool by_warp) {
        int32_t* row = p.table + (long long)b * p.max_pages;
        int at = need[b] >> 1;
        const bool copy = need[b] & 1;
        const int fresh = copy ? __ldcg(&p.ws.list[at++]) : -1;
        if (by_warp) {
            for (int i0 = w.first; i0 < w.end; i0 += 32) {
                const int i = i0 + lane;
                const bool none = i < w.end && row[i] < 0;
                const unsigned word = __ballot_sync(0xffffffffu, none);
                if (none) {
                    const int page = __ldcg(&p.ws.list[at + __popc(word & lanemask_lt())]);
                    row[i] = page;
                    p.refs[page] = 1;
                }
                at += __popc(word);
            }
            __syncwarp();               // all lanes have read the row's partly filled page
        } else {
            for (int i = w.first; i < w.end; ++i)
                if (row[i] < 0) {
                    const int page = __ldcg(&p.ws.list[at++]);
                    row[i] = page;
                    p.refs[page] = 1;
                }
        }
        if (copy && (!by_warp || lane == 0)) {
            row[w.first - 1] = fresh;
            p.refs[fresh] = 1;
            atomicSub(&p.refs[w.part], 1);
            p.ws.move[atomicAdd(&moves, 1)] = make_int3(w.part, fresh, p.lens[b] & ((1 << p.page_shift) - 1));
        }
    };
    for (int b = tid; b < p.B; b += kPlan) {
        w.of(p, b);
        if (w.part >= 0) holders[w.part] = last[w.part] = 0;
        if (enough && w.end - w.first <= kShort) give(b, false);
    }
    if (any_long && enough) {
        __syncthreads();                // marks are cleared by rows as they were
        for (int b = warp; b < p.B; b += kPlan / 32) {
            w.of(p, b);
            if (w.end - w.first > kShort) give(b, true);
        }
    }
    __syncthreads();
    if (tid == 0) *p.ws.count = moves;
}

struct CompactArgs {
    int32_t* refs;
    int32_t* used;
    int n_pages, page_size;
    PageWorkspace ws;
};

// One block. ws.list becomes the pages' new places. The i-th page in use from n on and the i-th free one below it meet in move i.
__global__ void __launch_bounds__(kPlan) k_compact(const __grid_constant__ CompactArgs p) {
    __shared__ int sums[33];
    int n = 0;
    for (int page0 = 0; page0 < p.n_pages; page0 += kPlan * kScan)
        scan_round(page0, p.n_pages, sums, n, [&](int page) { return p.refs[page] != 0; }, [](int, int) {});
    int high = 0, low = 0;
    for (int page0 = 0; page0 < p.n_pages; page0 += kPlan * kScan) {
        scan_round(page0, p.n_pages, sums, high, [&](int page) {
            const bool used = p.refs[page] != 0;
            p.ws.list[page] = used ? page : -1;
            return used && page >= n;
        }, [&](int page, int rank) { p.ws.move[rank].x = page; });
        if (page0 < n)
            scan_round(page0, n, sums, low, [&](int page) { return p.refs[page] == 0; }, [&](int page, int rank) { p.ws.move[rank].y = page; });
    }
    __syncthreads();
    for (int i = threadIdx.x; i < high; i += kPlan) {
        const int from = p.ws.move[i].x, to = p.ws.move[i].y;
        p.ws.move[i].z = p.page_size;
        p.ws.list[from] = to;
        p.refs[to] = p.refs[from];
        p.refs[from] = 0;
    }
    if (threadIdx.x == 0) *p.ws.count = high, *p.used = n;
}

struct CopyArgs {
    const int32_t* src;
    const int32_t* dst;
    int n, n_pages, page_size;
    PageWorkspace ws;
    int* err;
};

// One block: which of the copies can be made side by side.
__global__ void __launch_bounds__(kPlan) k_copy_plan(const __grid_constant__ CopyArgs p) {
    __shared__ int moves;
    int* as_dst = p.ws.mark;
    int* as_src = p.ws.mark + p.n_pages;
    if (threadIdx.x == 0) moves = 0;
    auto asked = [&](int i, int& s, int& d) {
        s = p.src[i], d = p.dst[i];
        return exists(s, p.n_pages) && exists(d, p.n_pages) && s != d;
    };
    int s, d;
    for (int i = threadIdx.x; i < p.n; i += kPlan)
        if (asked(i, s, d)) {
            atomicAdd(&as_dst[d], 1);
            as_src[s] = 1;
        }
    __syncthreads();
    bool bad = false;
    for (int i = threadIdx.x; i < p.n; i += kPlan) {
        if (!asked(i, s, d)) {
            bad = bad || !exists(s, p.n_pages) || !exists(d, p.n_pages);
        } else if (__ldcg(&as_dst[d]) > 1 || __ldcg(&as_src[d])) {
            bad = true;
        } else {
            p.ws.move[atomicAdd(&moves, 1)] = make_int3(s, d, p.page_size);
        }
    }
    if (bad) atomicOr(p.err, kErrIndex);
    __syncthreads();
    for (int i = threadIdx.x; i < p.n; i += kPlan)
        if (asked(i, s, d)) as_dst[d] = 0, as_src[s] = 0;
    if (threadIdx.x == 0) *p.ws.count = moves;
}

struct MoveArgs {
    uint8_t *pool[2], *scale[2];        // K and V
    int row, scale_row;                 // bytes of a row and its scales
    int layers, H, page_size, n_pages;
    PageWorkspace ws;
    // compaction: the tables follow
    int32_t* table;
    int32_t* new_page;
    long long entries;
    int* err;
};

constexpr int kMoveWords = 8;           // 16-byte words of a lane's rows that are under way together

// By one warp: what is left of `bytes` behind whole words of 16.
__device__ __forceinline__ void copy_tail(uint8_t* dst, const uint8_t* src, int bytes) {
    const int lane = threadIdx.x & 31, words = bytes >> 4;
    if (lane < (bytes & 15)) dst[words * 16 + lane] = src[words * 16 + lane];
}

// By one warp: `bytes` from src to dst, and `bytes2` from src2 to dst2 (all 16-byte aligned), the first words of both together.
__device__ __forceinline__ void copy_rows(uint8_t* dst, const uint8_t* src, int bytes, uint8_t* dst2, const uint8_t* src2, int bytes2) {
    const int lane = threadIdx.x & 31, words = bytes >> 4, words2 = bytes2 >> 4;
    uint4 u;
    if (lane < words2) u = __ldcs(reinterpret_cast<const uint4*>(src2) + lane);
    for (int w0 = 0; w0 < words; w0 += 32 * kMoveWords) {
        uint4 v[kMoveWords];
#pragma unroll
        for (int i = 0; i < kMoveWords; ++i) {
            const int w = w0 + 32 * i + lane;
            if (w < words) v[i] = __ldcs(reinterpret_cast<const uint4*>(src) + w);
        }
#pragma unroll
        for (int i = 0; i < kMoveWords; ++i) {
            const int w = w0 + 32 * i + lane;
            if (w < words) __stcs(reinterpret_cast<uint4*>(dst) + w, v[i]);
        }
    }
    if (lane < words2) __stcs(reinterpret_cast<uint4*>(dst2) + lane, u);
    for (int w = 32 + lane; w < words2; w += 32) __stcs(reinterpret_cast<uint4*>(dst2) + w, __ldcs(reinterpret_cast<const uint4*>(src2) + w));
    copy_tail(dst, src, bytes);
    copy_tail(dst2, src2, bytes2);
}

__global__ void __launch_bounds__(256) k_move(const __grid_constant__ MoveArgs p) {
    pdl_wait();
    const long long tid = (long long)blockIdx.x * 256 + threadIdx.x, threads = (long long)gridDim.x * 256;
    if (p.table) {
        bool bad = false;
        for (long long i = tid; i < p.entries; i += threads) {
            const int page = p.table[i];
            if (page < 0) continue;
            const int to = exists(page, p.n_pages) ? p.ws.list[page] : -1;
            bad = bad || to < 0;
            if (to != page) p.table[i] = to;
        }
        if (bad) atomicOr(p.err, kErrIndex);
        if (p.new_page)
            for (long long i = tid; i < p.n_pages; i += threads) p.new_page[i] = p.ws.list[i];
    }
    // a warp a (move, layer, K or V, head): its rows and their scales
    const int per_move = p.layers * 2 * p.H;
    const long long all = (long long)*p.ws.count * per_move;
    for (long long i = tid >> 5; i < all; i += threads >> 5) {
        const long long n = (i | per_move) >> 32 ? i / per_move : (uint32_t)i / (uint32_t)per_move;
        const int3 m = p.ws.move[n];
        const int rest = (int)(i - n * per_move), lk = rest / p.H, h = rest - lk * p.H;
        // first rows of the head in the two pages
        const long long to = (((lk >> 1) * (long long)p.n_pages + m.y) * p.H + h) * p.page_size, from = (((lk >> 1) * (long long)p.n_pages + m.x) * p.H + h) * p.page_size;
        uint8_t* pool = lk & 1 ? p.pool[1] : p.pool[0];
        uint8_t* scale = lk & 1 ? p.scale[1] : p.scale[0];
        copy_rows(pool + to * p.row, pool + from * p.row, m.z * p.row, scale + to * p.scale_row, scale + from * p.scale_row, m.z * p.scale_row);
    }
}

ace_status pages_fail(const char* m) { return kv_fail(ACE_ERR_INVALID_ARG, m); }

// Moves what the plan before on the stream lists.
ace_status launch_moves(const ace_kv* kv, MoveArgs p, cudaStream_t s) {
    const ace_kv_desc& D = kv->desc;
    p.row = row_bytes(D.format, D.head_dim, kv->elem);
    p.scale_row = scale_bytes(D.format, D.head_dim);
    p.pool[0] = static_cast<uint8_t*>(kv->k_pool), p.pool[1] = static_cast<uint8_t*>(kv->v_pool);
    p.scale[0] = kv->k_scale, p.scale[1] = kv->v_scale;
    p.layers = D.layers, p.H = D.n_kv_heads, p.page_size = D.page_size, p.n_pages = D.n_pages;
    p.ws = kv->pages;
    p.err = kv->err;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kv->num_sms * 6);
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k_move, p);
    return e == cudaSuccess ? ACE_OK : kv_cuda(e, "page move launch");
}

int shift_of(int page_size) {
    int s = 0;
    while (1 << s < page_size) ++s;
    return s;
}

bool meet(const int32_t* a, long long n, const int32_t* b, long long m) {
    return n > 0 && m > 0 && (uintptr_t)a < (uintptr_t)(b + m) && (uintptr_t)b < (uintptr_t)(a + n);
}

}  // namespace

extern "C" {

ace_status ace_kv_fork(ace_kv* kv, const int32_t* page_table, const int32_t* lens, int B, const int32_t* parents, int B_out, int max_pages,
                       int32_t* refs, int32_t* new_table, int32_t* new_lens, void* stream) {
    if (!kv) return pages_fail("cache is NULL");
    if (B < 0 || B_out < 0 || max_pages < 1) return pages_fail("B and B_out must be >= 0 and max_pages >= 1");
    if (!refs || (B > 0 && (!page_table || !lens)) || (B_out > 0 && (!parents || !new_table || !new_lens)))
        return pages_fail("page_table, lens, parents, refs, new_table and new_lens must be non-NULL");
    const long long in = (long long)B * max_pages, out = (long long)B_out * max_pages;
    const int32_t* const old[] = {page_table, lens, parents, refs};
    const long long olds[] = {in, B, B_out, kv->desc.n_pages};
    for (int i = 0; i < 4; ++i)
        if (meet(new_table, out, old[i], olds[i]) || meet(new_lens, B_out, old[i], olds[i]))
            return pages_fail("new_table and new_lens must not overlap the other arrays");
    if (meet(new_table, out, new_lens, B_out)) return pages_fail("new_table and new_lens must not overlap the other arrays");
    for (int i = 0; i < 3; ++i)
        if (meet(refs, kv->desc.n_pages, old[i], olds[i])) return pages_fail("refs must not overlap the other arrays");
    if (const ace_status st = on_device(kv->device, "cache")) return st;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    kv->last_stream = s;
    if (B == 0 && B_out == 0) return ACE_OK;
    const ForkArgs p{page_table, lens, parents, refs, new_table, new_lens, B, B_out, max_pages, shift_of(kv->desc.page_size), kv->desc.n_pages, kv->err};
    k_fork<<<B > B_out ? B : B_out, 128, 0, s>>>(p);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? ACE_OK : kv_cuda(e, "fork launch");
}

ace_status ace_kv_reserve(ace_kv* kv, int32_t* page_table, int max_pages, const int32_t* lens, const int32_t* grow, int B, int32_t* refs,
                          int32_t* missing, void* stream) {
    if (!kv) return pages_fail("cache is NULL");
    if (B < 0 || max_pages < 1) return pages_fail("B must be >= 0 and max_pages >= 1");
    if (!refs || !missing || (B > 0 && (!page_table || !lens || !grow)))
        return pages_fail("page_table, lens, grow, refs and missing must be non-NULL");
    if (B > kPlanRows) return kv_fail(ACE_ERR_UNSUPPORTED, "a call reserves for at most 8192 requests");
    const long long entries = (long long)B * max_pages;
    if (entries > 1 << 29) return kv_fail(ACE_ERR_UNSUPPORTED, "a call reserves in tables of at most 2^29 entries");
    if (meet(page_table, entries, lens, B) || meet(page_table, entries, grow, B) || meet(page_table, entries, refs, kv->desc.n_pages) ||
        meet(refs, kv->desc.n_pages, lens, B) || meet(refs, kv->desc.n_pages, grow, B) || meet(missing, 1, page_table, entries) ||
        meet(missing, 1, refs, kv->desc.n_pages) || meet(missing, 1, lens, B) || meet(missing, 1, grow, B))
        return pages_fail("page_table, refs and missing must not overlap the other arrays");
    if (const ace_status st = on_device(kv->device, "cache")) return st;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    kv->last_stream = s;
    const ReserveArgs p{page_table, lens, grow, refs, missing, B, max_pages, shift_of(kv->desc.page_size), kv->desc.n_pages, kv->pages, kv->err};
    k_reserve<<<1, kPlan, 0, s>>>(p);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? launch_moves(kv, MoveArgs{}, s) : kv_cuda(e, "reserve launch");
}

ace_status ace_kv_release(ace_kv* kv, int32_t* page_table, int max_pages, int32_t* lens, const int32_t* ended, int B, int32_t* refs, void* stream) {
    if (!kv) return pages_fail("cache is NULL");
    if (B < 0 || max_pages < 1) return pages_fail("B must be >= 0 and max_pages >= 1");
    if (!refs || (B > 0 && (!page_table || !lens || !ended))) return pages_fail("page_table, lens, ended and refs must be non-NULL");
    const long long entries = (long long)B * max_pages;
    if (meet(page_table, entries, lens, B) || meet(page_table, entries, ended, B) || meet(page_table, entries, refs, kv->desc.n_pages) ||
        meet(refs, kv->desc.n_pages, lens, B) || meet(refs, kv->desc.n_pages, ended, B) || meet(lens, B, ended, B))
        return pages_fail("page_table, lens, ended and refs must not overlap");
    if (const ace_status st = on_device(kv->device, "cache")) return st;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    kv->last_stream = s;
    if (B == 0) return ACE_OK;
    k_release<<<B, 128, 0, s>>>(page_table, max_pages, lens, ended, refs, kv->desc.n_pages, kv->err);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? ACE_OK : kv_cuda(e, "release launch");
}

ace_status ace_kv_compact(ace_kv* kv, int32_t* page_table, int max_pages, int B, int32_t* refs, int32_t* used, int32_t* new_page, void* stream) {
    if (!kv) return pages_fail("cache is NULL");
    if (B < 0 || max_pages < 1) return pages_fail("B must be >= 0 and max_pages >= 1");
    if (!refs || !used || (B > 0 && !page_table)) return pages_fail("page_table, refs and used must be non-NULL");
    const long long entries = (long long)B * max_pages, n = kv->desc.n_pages;
    if (meet(page_table, entries, refs, n) || meet(used, 1, page_table, entries) || meet(used, 1, refs, n) ||
        (new_page && (meet(new_page, n, page_table, entries) || meet(new_page, n, refs, n) || meet(new_page, n, used, 1))))
        return pages_fail("page_table, refs, used and new_page must not overlap");
    if (const ace_status st = on_device(kv->device, "cache")) return st;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    kv->last_stream = s;
    const CompactArgs p{refs, used, kv->desc.n_pages, kv->desc.page_size, kv->pages};
    k_compact<<<1, kPlan, 0, s>>>(p);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return kv_cuda(e, "compaction launch");
    MoveArgs m{};
    m.table = page_table ? page_table : refs;       // (with no requests, no entries: new_page follows all the same)
    m.entries = entries;
    m.new_page = new_page;
    return launch_moves(kv, m, s);
}

ace_status ace_kv_copy_pages(ace_kv* kv, const int32_t* src, const int32_t* dst, int n, void* stream) {
    if (!kv) return pages_fail("cache is NULL");
    if (n < 0) return pages_fail("n must be >= 0");
    if (n > 0 && (!src || !dst)) return pages_fail("src and dst must be non-NULL");
    if (const ace_status st = on_device(kv->device, "cache")) return st;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    kv->last_stream = s;
    if (n == 0) return ACE_OK;
    const CopyArgs p{src, dst, n, kv->desc.n_pages, kv->desc.page_size, kv->pages, kv->err};
    k_copy_plan<<<1, kPlan, 0, s>>>(p);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? launch_moves(kv, MoveArgs{}, s) : kv_cuda(e, "page copy launch");
}

}  // extern "C"
