// Eviction from the paged cache by accumulated attention weight: which tokens stay, and their move to other pages.
//
// Selection, one block for a sequence and head: the `need`-th largest weight among the tokens that are neither sinks nor recent, by a radix
// search over the weights' order-preserving integers (11, 11 and 10 bits: a histogram in shared memory, then the digit in which the
// count is reached), and then one pass in token order that writes the indices above it and the first ones equal to it.  A thread has a
// run of consecutive tokens, so that one scan over the threads gives every kept token its rank.
// Move: bound by HBM, sixteen bytes a thread and access, rows of keys and values side by side.
#include "cache.cuh"

namespace vitint {
namespace {

constexpr int EV_THREADS = 1024;
constexpr int EV_BINS = 2048;

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

// Exclusive sums over the block's threads of two counts packed in one word (each below 2^31), and the total.
__device__ __forceinline__ unsigned long long block_scan(unsigned long long v, unsigned long long* warp_sums, unsigned long long& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long t = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += t;
    }
    if (lane == 31) warp_sums[warp] = s;
    __syncthreads();
    if (warp == 0) {
        unsigned long long w = warp_sums[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long t = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += t;
        }
        warp_sums[lane] = w;
    }
    __syncthreads();
    const unsigned long long base = warp ? warp_sums[warp - 1] : 0ull;
    total = warp_sums[31];
    return base + s - v;
}

__global__ void __launch_bounds__(EV_THREADS)
evict_select_kernel(const __grid_constant__ EvictParams P) {
    __shared__ uint32_t bins[EV_BINS];
    __shared__ unsigned long long warp_sums[32];
    __shared__ uint32_t found[2];                                      // the digit, and how many are still wanted inside it
    const int h = blockIdx.x, b = blockIdx.y, t = threadIdx.x;
    grid_dependency_wait();
    grid_dependency_launch();
    bool ok = true;
    const int length = length_of(P.seq, b, ok);
    if (!ok && t == 0) report_bad_data();
    const int count = min(length, P.budget);
    int* const kept = P.kept + ((long long)b * P.kv_heads + h) * P.budget;
    if (h == 0 && t == 0) P.counts[b] = count;
    for (int i = count + t; i < P.budget; i += EV_THREADS) kept[i] = -1;
    if (length <= P.budget) {
        for (int i = t; i < length; i += EV_THREADS) kept[i] = i;
        return;
    }
    const int first = P.sinks, last = length - P.recent, need = P.budget - P.sinks - P.recent;
    for (int i = t; i < P.sinks; i += EV_THREADS) kept[i] = i;
    for (int i = t; i < P.recent; i += EV_THREADS) kept[P.budget - P.recent + i] = last + i;
    if (need == 0) return;
    const int shift = P.seq.page_shift, mask = (1 << shift) - 1;
    auto key_of = [&](int i) {
        const int p = page_of(P.seq, b, i);
        return weight_key(p < P.seq.pages ? P.weights[(((long long)p * P.kv_heads + h) << shift) + (i & mask)] : 0.0f);
    };
    uint32_t prefix = 0, known = 0;                                    // digits found so far, and their bits
    uint32_t want = (uint32_t)need;
    for (int pass = 0; pass < 3; ++pass) {
        const int low = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
        for (int i = t; i < EV_BINS; i += EV_THREADS) bins[i] = 0u;
        __syncthreads();
        for (int i = first + t; i < last; i += EV_THREADS) {
            const uint32_t k = key_of(i);
            if ((k & known) == prefix) atomicAdd(&bins[(k >> low) & ((1u << width) - 1u)], 1u);
        }
        __syncthreads();
        // bins from the largest digit down: thread t has digits EV_BINS-1-2t and EV_BINS-2-2t
        const uint32_t d0 = EV_BINS - 1 - 2 * t, d1 = d0 - 1;
        const uint32_t n0 = bins[d0], n1 = bins[d1];
        unsigned long long total;
        const uint32_t above = (uint32_t)block_scan(n0 + n1, warp_sums, total);
        if (above < want && want <= above + n0) { found[0] = d0; found[1] = want - above; }
        else if (above + n0 < want && want <= above + n0 + n1) { found[0] = d1; found[1] = want - above - n0; }
        __syncthreads();
        prefix |= found[0] << low;
        known |= ((1u << width) - 1u) << low;
        want = found[1];
        __syncthreads();
    }
    // `prefix` is the last weight to stay, `want` of the tokens that have it do
    const int run = (last - first + EV_THREADS - 1) / EV_THREADS;
    const int begin = min(first + t * run, last), end = min(begin + run, last);
    uint32_t larger = 0, equal = 0;
    for (int i = begin; i < end; ++i) {
        const uint32_t k = key_of(i);
        larger += k > prefix;
        equal += k == prefix;
    }
    unsigned long long total;
    const unsigned long long before = block_scan(((unsigned long long)larger << 32) | equal, warp_sums, total);
    uint32_t ahead = (uint32_t)before;                                 // equal ones in front
    int* to = kept + P.sinks + (uint32_t)(before >> 32) + min(ahead, want);
    for (int i = begin; i < end; ++i) {
        const uint32_t k = key_of(i);
        if (k > prefix || (k == prefix && ahead < want)) *to++ = i;
        ahead += k == prefix;
    }
}

struct MoveParams {
    SequenceView seq;
    const int* new_table;
    long long new_stride;
    const int* kept;
    uint8_t *k, *v;
    float *k_steps, *v_steps, *weights;
    long long page_bytes, head_bytes, token_bytes;
    int kv_heads, budget, units;                                       // units: 16-byte pieces of a key row
};

// A thread moves one piece of a key or value row; the threads of a row's first piece take its step, and the weight.
__global__ void __launch_bounds__(256)
evict_move_kernel(const __grid_constant__ MoveParams P) {
    grid_dependency_wait();
    grid_dependency_launch();
    const long long index = (long long)blockIdx.x * 256 + threadIdx.x;
    const int per = 2 * P.units, shift = P.seq.page_shift, mask = (1 << shift) - 1;
    const long long row = index / per;
    if (row >= (long long)P.seq.sequences * P.kv_heads * P.budget) return;
    const int piece = (int)(index - row * per);
    const int from = P.kept[row];
    if (from < 0) return;
    const int to = (int)(row % P.budget), bh = (int)(row / P.budget), b = bh / P.kv_heads, h = bh - b * P.kv_heads;
    const int old_page = page_of(P.seq, b, from), new_page = P.new_table[b * P.new_stride + (to >> shift)];
    if ((unsigned)new_page >= (unsigned)P.seq.pages) { report_bad_data(); return; }
    if (old_page >= P.seq.pages) return;
    const bool is_v = piece >= P.units;
    const int unit = piece - (is_v ? P.units : 0);
    uint8_t* const base = is_v ? P.v : P.k;
    const long long inside = h * P.head_bytes + unit * 16;
    const uint4 w = *reinterpret_cast<const uint4*>(base + old_page * P.page_bytes + (from & mask) * P.token_bytes + inside);
    *reinterpret_cast<uint4*>(base + new_page * P.page_bytes + (to & mask) * P.token_bytes + inside) = w;
    if (unit == 0) {
        const long long a = (((long long)old_page * P.kv_heads + h) << shift) + (from & mask);
        const long long z = (((long long)new_page * P.kv_heads + h) << shift) + (to & mask);
        float* const steps = is_v ? P.v_steps : P.k_steps;
        if (steps) steps[z] = steps[a];
        if (!is_v) P.weights[z] = P.weights[a];
    }
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
    M.kv_heads = cache->kv_heads; M.budget = budget; M.units = cache->head_dim * size / 16;
    const long long rows = (long long)batch->sequences * cache->kv_heads * budget, blocks = (rows * 2 * M.units + 255) / 256;
    if (blocks > 0x7fffffffll) return VITINT_ERR_UNSUPPORTED;
    cudaStream_t st = (cudaStream_t)stream;
    launch_kernel(evict_select_kernel, dim3(cache->kv_heads, batch->sequences), dim3(EV_THREADS), 0, st, E);
    if (int rc = cuda_status(cudaGetLastError())) return rc;
    launch_kernel(evict_move_kernel, dim3((unsigned)blocks), dim3(256), 0, st, M);
    return cuda_status(cudaGetLastError());
}
