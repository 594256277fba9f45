// Eviction from the paged cache by accumulated attention weight: which tokens stay, and their move to other pages.
//
// Selection, one to eight blocks (a cluster) for a sequence and head: the `need`-th largest weight among the tokens that are neither sinks nor
// recent, by a radix search over the weights' order-preserving integers (11, 11 and 10 bits: a histogram in every block's shared memory,
// summed over the cluster, then the digit in which the count is reached), and then one pass in token order that writes the indices above
// it and the first ones equal to it.  The weights are read once and stay in shared memory, except where a block's part is longer than it holds (EV_HELD:
// one block for each of 75 or more heads, beyond 40,960 tokens): then every pass reads them anew.  Bound by latency: three histograms and their
// sums follow one another; clusters are as large as the GPU has room for and a block has 2048 tokens left.
// 65,536 tokens x 8 heads: 120 -> 27 us against one block a head that reads its weights anew for every pass.
// Move: bound by HBM.  A warp takes 32 kept tokens: its lanes look up where they lie and go, then all of them copy row after row, sixteen bytes a
// lane, eight rows under way.
#include "cache.cuh"

namespace vitint {
namespace {

constexpr int EV_THREADS = 1024;
constexpr int EV_BINS = 2048;
constexpr int EV_HELD = 40960;                                        // weights that a block keeps

struct EvictParams {
    SequenceView seq;
    float* weights;
    int kv_heads, budget, sinks, recent;
    int* kept;
    int* counts;
};

// Larger weights have larger keys; -0 and 0 are equal.
__device__ __forceinline__ uint32_t weight_key(float w) {
    const uint32_t u = __float_as_uint(w + 0.0f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// Exclusive sums of counts over the block's threads.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* warp_sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += t;
    }
    if (lane == 31) warp_sums[warp] = s;
    __syncthreads();
    if (warp == 0) {
        uint32_t w = warp_sums[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t t = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += t;
        }
        warp_sums[lane] = w;
    }
    __syncthreads();
    return (warp ? warp_sums[warp - 1] : 0u) + s - v;
}

// ---- clusters of blocks --------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_size() { uint32_t v; asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(v)); return v; }
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t v; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(v)); return v; }
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t remote_address(const void* mine, uint32_t rank) {           // of the same variable of another block
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(ptx::smem_addr(mine)), "r"(rank));
    return at;
}
__device__ __forceinline__ uint32_t remote_word(const uint32_t* mine, uint32_t rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(remote_address(mine, rank)));      // (ordered by the barriers around)
    return v;
}
__device__ __forceinline__ uint4 remote_quad(const uint4* mine, uint32_t rank) {
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(remote_address(mine, rank)));
    return v;
}

// Block `rank` of a cluster takes the rank-th part of a sequence's tokens.  held: tokens whose weights fit the dynamic shared memory; a part
// that is longer is read from memory in every pass.
__global__ void __launch_bounds__(EV_THREADS)
evict_select_kernel(const __grid_constant__ EvictParams P, int held) {
    extern __shared__ uint32_t ev_keys[];
    __shared__ __align__(16) uint32_t bins[2][EV_BINS];                // the largest digit first
    __shared__ uint32_t warp_sums[32];
    __shared__ uint32_t found[3];                                      // the digit, how many are still wanted inside it, and how many it has
    __shared__ uint32_t larger_of[33], equal_of[33];                   // counts of the block's warps, then of the block
    const int blocks = (int)cluster_size(), rank = (int)cluster_rank();
    const int h = blockIdx.x / blocks, b = blockIdx.y, t = threadIdx.x, warp = t >> 5, lane = t & 31;
    for (int i = t; i < EV_BINS; i += EV_THREADS) bins[0][i] = 0u;
    grid_dependency_wait();
    grid_dependency_launch();
    bool ok = true;
    const int length = length_of(P.seq, b, ok);
    if (!ok && t == 0) report_bad_data();
    const int count = min(length, P.budget);
    int* const kept = P.kept + ((long long)b * P.kv_heads + h) * P.budget;
    const int t0 = rank * EV_THREADS + t, all = blocks * EV_THREADS;
    if (h == 0 && t0 == 0) P.counts[b] = count;
    for (int i = count + t0; i < P.budget; i += all) kept[i] = -1;
    const int first = P.sinks, last = length - P.recent, need = P.budget - P.sinks - P.recent;
    if (length <= P.budget) {                                          // (the same for all blocks of the cluster)
        for (int i = t0; i < length; i += all) kept[i] = i;
        return;
    }
    for (int i = t0; i < P.sinks; i += all) kept[i] = i;
    for (int i = t0; i < P.recent; i += all) kept[P.budget - P.recent + i] = last + i;
    if (need == 0) return;

    const int part = (last - first + blocks - 1) / blocks, begin = min(first + rank * part, last), n = min(part, last - begin);
    const int shift = P.seq.page_shift, mask = (1 << shift) - 1;
    auto read_key = [&](int i) {
        const int p = page_of(P.seq, b, begin + i);
        return weight_key(p < P.seq.pages ? P.weights[(((long long)p * P.kv_heads + h) << shift) + ((begin + i) & mask)] : 0.0f);
    };
    const bool in_shared = n <= held;
    auto barrier = [&] {
        if (blocks > 1) cluster_barrier();
        else __syncthreads();
    };
    auto key_of = [&](int i) { return in_shared ? ev_keys[i] : read_key(i); };
    if (in_shared) {
        for (int i0 = t; i0 < n; i0 += 8 * EV_THREADS) {               // eight tokens of a thread under way
            int page[8];
            float w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) page[k] = i0 + k * EV_THREADS < n ? page_entry(P.seq, b, begin + i0 + k * EV_THREADS) : 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int i = i0 + k * EV_THREADS, p = i < n ? checked_page(P.seq, page[k]) : P.seq.pages;
                w[k] = p < P.seq.pages ? P.weights[(((long long)p * P.kv_heads + h) << shift) + ((begin + i) & mask)] : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (i0 + k * EV_THREADS < n) ev_keys[i0 + k * EV_THREADS] = weight_key(w[k]);
        }
    }
    __syncthreads();
    uint32_t prefix = 0, known = 0;                                    // digits found so far, and their bits
    uint32_t want = (uint32_t)need;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int low = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t digits = pass == 2 ? 1023u : 2047u;
        uint32_t* const mine = bins[pass & 1];
        for (int i = t; i - lane < n; i += EV_THREADS) {
            const uint32_t k = i < n ? key_of(i) : 0u, digit = digits - ((k >> low) & digits);
            const bool counted = i < n && (k & known) == prefix;
            // (a warp whose tokens all have one weight, none as a rule, counts them together: their additions would queue up)
            const bool leads = digit == __shfl_sync(0xffffffffu, digit, 0);
            if (__all_sync(0xffffffffu, counted && leads)) {
                if (lane == 0) atomicAdd(&mine[digit], 32u);
            } else if (counted) {
                atomicAdd(&mine[digit], 1u);
            }
        }
        barrier();
        // (the other histogram was last read in front of this barrier)
        for (int i = t; i < EV_BINS; i += EV_THREADS) bins[(pass + 1) & 1][i] = 0u;
        // four digits a thread, over all blocks
        uint4 q = make_uint4(0u, 0u, 0u, 0u);
        if (t < EV_BINS / 4) {
            const uint4* const at = reinterpret_cast<const uint4*>(mine) + t;
            q = *at;
            if (blocks > 1) {
#pragma unroll
                for (int r = 0; r < 8; ++r)                             // (all of them under way at once)
                    if (r < blocks && r != rank) {
                        const uint4 o = remote_quad(at, r);
                        q.x += o.x; q.y += o.y; q.z += o.z; q.w += o.w;
                    }
            }
        }
        uint32_t above = block_scan(q.x + q.y + q.z + q.w, warp_sums);
        const uint32_t count_of[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (above < want && want <= above + count_of[k]) { found[0] = digits - (uint32_t)(4 * t + k); found[1] = want - above; found[2] = count_of[k]; }
            above += count_of[k];
        }
        __syncthreads();
        prefix |= found[0] << low;
        known |= digits << low;
        want = found[1];
        const bool all_stay = want == found[2];
        __syncthreads();
        if (all_stay) break;                                           // (the same for all blocks: further digits tell nothing)
    }
    // Of the digits known, `prefix` are the last to stay, and `want` of the tokens that have them do.  A warp has a run of the block's tokens, 32 at a time.
    const int run = ((n + 1023) / 1024) * 32, from = min(warp * run, n), to = min(from + run, n);
    uint32_t larger = 0, equal = 0;
    for (int i = from + lane; i < to; i += 32) {
        const uint32_t k = key_of(i) & known;
        larger += k > prefix;
        equal += k == prefix;
    }
    larger = __reduce_add_sync(0xffffffffu, larger);
    equal = __reduce_add_sync(0xffffffffu, equal);
    if (lane == 0) { larger_of[warp] = larger; equal_of[warp] = equal; }
    __syncthreads();
    if (warp == 0) {
        const uint32_t a = larger_of[lane], e = equal_of[lane];
        const uint32_t sa = (uint32_t)__reduce_add_sync(0xffffffffu, a), se = (uint32_t)__reduce_add_sync(0xffffffffu, e);
        uint32_t pa = a, pe = e;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, pa, o), y = __shfl_up_sync(0xffffffffu, pe, o);
            if (lane >= o) { pa += x; pe += y; }
        }
        larger_of[lane] = pa - a;
        equal_of[lane] = pe - e;
        if (lane == 0) { larger_of[32] = sa; equal_of[32] = se; }
    }
    barrier();
    uint32_t ahead_larger = larger_of[warp], ahead_equal = equal_of[warp];
    for (int r = 0; r < rank; ++r) {
        ahead_larger += remote_word(&larger_of[32], r);
        ahead_equal += remote_word(&equal_of[32], r);
    }
    for (int i0 = from; i0 < to; i0 += 32) {
        const int i = i0 + lane;
        const uint32_t k = i < to ? key_of(i) & known : 0u;
        const bool is_larger = i < to && k > prefix, is_equal = i < to && k == prefix;
        const uint32_t a = __ballot_sync(0xffffffffu, is_larger), e = __ballot_sync(0xffffffffu, is_equal), below = (1u << lane) - 1u;
        const uint32_t my_equal = ahead_equal + __popc(e & below);
        if (is_larger || (is_equal && my_equal < want)) kept[P.sinks + ahead_larger + __popc(a & below) + min(my_equal, want)] = begin + i;
        ahead_larger += __popc(a);
        ahead_equal += __popc(e);
    }
    if (blocks > 1) cluster_barrier();                                 // the others have read this block's counts
}

struct MoveParams {
    SequenceView seq;
    const int* new_table;
    long long new_stride;
    const int* kept;
    uint8_t *k, *v;
    float *k_steps, *v_steps, *weights;
    long long page_bytes, head_bytes, token_bytes;
    int kv_heads, budget;
};

// UNITS: 16-byte pieces of a key row.  Block y: a sequence and head; a warp takes 32 of its kept tokens.
template <int UNITS>
__global__ void __launch_bounds__(256)
evict_move_kernel(const __grid_constant__ MoveParams P) {
    constexpr int ROWS = 32 / (2 * UNITS) > 0 ? 32 / (2 * UNITS) : 1;   // rows that a warp copies at once
    constexpr int DEEP = 8;                                            // ... and how often before it stores them
    grid_dependency_wait();
    grid_dependency_launch();
    const int lane = threadIdx.x & 31, b = blockIdx.y / P.kv_heads, h = blockIdx.y - b * P.kv_heads, shift = P.seq.page_shift, mask = (1 << shift) - 1;
    const int to0 = (blockIdx.x * 8 + (threadIdx.x >> 5)) * 32, to = to0 + lane;
    // the lane's token: where its row lies and goes (-1: nowhere)
    const int from = to < P.budget ? P.kept[(long long)blockIdx.y * P.budget + to] : -1;
    long long src = -1, dst = -1, z = 0;
    float weight = 0.0f, k_step = 0.0f, v_step = 0.0f;
    if (from >= 0) {
        const int old_page = page_of(P.seq, b, from), new_page = P.new_table[b * P.new_stride + (to >> shift)];
        if ((unsigned)new_page >= (unsigned)P.seq.pages) {
            report_bad_data();
        } else if (old_page < P.seq.pages) {
            src = old_page * P.page_bytes + (from & mask) * P.token_bytes + h * P.head_bytes;
            dst = new_page * P.page_bytes + (to & mask) * P.token_bytes + h * P.head_bytes;
            const long long a = (((long long)old_page * P.kv_heads + h) << shift) + (from & mask);
            z = (((long long)new_page * P.kv_heads + h) << shift) + (to & mask);
            weight = P.weights[a];
            if (P.k_steps) {
                k_step = P.k_steps[a];
                v_step = P.v_steps[a];
            }
        }
    }
    const int piece = lane % (2 * UNITS), row0 = lane / (2 * UNITS);
    uint8_t* const base = piece < UNITS ? P.k : P.v;
    const int inside = (piece % UNITS) * 16;
#pragma unroll 1
    for (int r = 0; r < 32; r += ROWS * DEEP) {
        uint4 w[DEEP];
        long long at[DEEP];
#pragma unroll
        for (int k = 0; k < DEEP; ++k) {
            const int row = r + k * ROWS + row0;
            const long long s = __shfl_sync(0xffffffffu, src, row & 31);
            at[k] = __shfl_sync(0xffffffffu, dst, row & 31);
            if (s >= 0) w[k] = *reinterpret_cast<const uint4*>(base + s + inside);
        }
#pragma unroll
        for (int k = 0; k < DEEP; ++k)
            if (at[k] >= 0) *reinterpret_cast<uint4*>(base + at[k] + inside) = w[k];
    }
    if (dst >= 0) {
        P.weights[z] = weight;
        if (P.k_steps) {
            P.k_steps[z] = k_step;
            P.v_steps[z] = v_step;
        }
    }
}

// Blocks of a cluster: as many as the GPU has room for side by side, while a block has 2048 tokens left.
inline int evict_cluster(int64_t items, int64_t max_length) {
    int c = 1;
    while (c < 8 && items * (2 * c) <= sm_count() && max_length >= 4096 * c) c *= 2;
    return c;
}

inline cudaError_t launch_select(const EvictParams& E, int sequences, int cluster, int held, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(E.kv_heads * cluster), (unsigned)sequences);
    cfg.blockDim = dim3(EV_THREADS);
    // (blocks of a cluster do not share an SM, which two of them may when they are placed early: so much that only one fits)
    cfg.dynamicSmemBytes = (size_t)held * 4;
    if (cluster > 1 && cfg.dynamicSmemBytes < 116 * 1024) cfg.dynamicSmemBytes = 116 * 1024;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, evict_select_kernel, E, held);
}

}  // namespace
}  // namespace vitint

using namespace vitint;

extern "C" int vitint_cache_evict(const vitint_cache* cache, const vitint_cache_batch* batch, float* weights, int32_t budget, int32_t sinks,
                                  int32_t recent, const int32_t* new_table, int64_t new_table_stride, int32_t* kept, int32_t* counts,
                                  void* stream) {
    if (int rc = check_cache(cache)) return rc;
    if (int rc = check_batch(cache, batch, false)) return rc;
    if (!weights || !new_table || !kept || !counts || counts == batch->lengths || new_table == batch->page_table) return VITINT_ERR_INVALID_ARG;
    if (!aligned_to(weights, 4) || !aligned_to(new_table, 4) || !aligned_to(kept, 4) || !aligned_to(counts, 4)) return VITINT_ERR_ALIGNMENT;
    if (budget <= 0 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget) return VITINT_ERR_INVALID_ARG;
    if (new_table_stride <= 0 || ((int64_t)budget + cache->page_tokens - 1) / cache->page_tokens > new_table_stride) return VITINT_ERR_INVALID_ARG;
    if (budget > CACHE_MAX_LENGTH) return VITINT_ERR_UNSUPPORTED;
    EvictParams E{};
    E.seq = sequence_view(cache, batch, 0);
    E.weights = weights;
    E.kv_heads = cache->kv_heads; E.budget = budget; E.sinks = sinks; E.recent = recent;
    E.kept = kept; E.counts = counts;
    MoveParams M{};
    M.seq = E.seq;
    M.new_table = new_table; M.new_stride = new_table_stride;
    M.kept = kept;
    M.k = (uint8_t*)cache->k; M.v = (uint8_t*)cache->v; M.k_steps = cache->k_steps; M.v_steps = cache->v_steps; M.weights = weights;
    const int size = dtype_bytes(cache->type);
    M.page_bytes = cache->page_stride * size; M.head_bytes = cache->head_stride * size; M.token_bytes = cache->token_stride * size;
    M.kv_heads = cache->kv_heads; M.budget = budget;
    const long long items = (long long)batch->sequences * cache->kv_heads;
    if (items > 65535 || (long long)cache->kv_heads * 8 > 65535) return VITINT_ERR_UNSUPPORTED;      // (blocks along a grid's second dimension)
    const int cluster = evict_cluster(items, batch->max_length);
    const int64_t part = (batch->max_length + cluster - 1) / cluster;
    const int held = part <= EV_HELD ? (int)part : EV_HELD;
    const int dev = current_device();
    if (dev < 0) return VITINT_ERR_CUDA;
    static bool attr_set_dev[MAX_DEVICES] = {};
    if (!attr_set_dev[dev]) {
        if (cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, EV_HELD * 4) != cudaSuccess) return VITINT_ERR_CUDA;
        attr_set_dev[dev] = true;
    }
    cudaStream_t st = (cudaStream_t)stream;
    if (int rc = cuda_status(launch_select(E, batch->sequences, cluster, held, st))) return rc;
    const dim3 grid((unsigned)((budget + 255) / 256), (unsigned)items);
    switch (cache->head_dim * size / 16) {
        case 4: launch_kernel(evict_move_kernel<4>, grid, dim3(256), 0, st, M); break;
        case 8: launch_kernel(evict_move_kernel<8>, grid, dim3(256), 0, st, M); break;
        default: launch_kernel(evict_move_kernel<16>, grid, dim3(256), 0, st, M); break;
    }
    return cuda_status(cudaGetLastError());
}
