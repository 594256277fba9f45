// How the attention kernels over the paged cache share their work out.
//
// An item is, for the attention, a head of the cache and a run of a sequence's new tokens (tile_tokens of them, all query heads of the
// group); its work is a number of key tiles.  (For the weighing it is a run of keys, and its work the runs of queries.)  All items' tiles,
// sequence by sequence, head by head, run by run, form one line, and every CTA takes an equal stretch of it: whatever the lengths are, no CTA
// has more than one tile above the mean.  A stretch that ends inside an item leaves a partial result (row maxima, sums and unnormalised outputs)
// in the workspace, at most two a CTA, and a second kernel joins them.  Short items stay whole (whole_items): a CTA then has all tiles of the items
// that begin in its stretch, up to an item's less one above its share.  The plan is made on the device from the lengths, so a
// recorded graph may be replayed with others; it is a warp's work: lanes take sequences, or the runs of one long chunk.
#pragma once

#include "cache.cuh"

namespace vitint {

struct PlanParams {
    SequenceView seq;
    int kv_heads, group, tile_tokens;
    int causal, window;                   // window 0: none
    int whole;                            // items are not split: a CTA has those that begin in its stretch
};

// Whether items stay whole: a second launch to join parts costs about 1.5 us on the device (and 2.2 us of the host).  That is more than what splitting
// gains where the longest item has at most `few` tiles, and up to `most` tiles where the items alone fill a quarter of the grid.  Recorded calls,
// us whole / split:
//   one token, 12 heads of 64, tiles of 128 keys:    1 sequence   3 tiles 7.1 / 7.4,  4: 7.9 / 7.5,  7: 10.1 / 7.4;  16 sequences  4: 9.2 / 10.6,  7: 12.3 / 13.2
//   one token, 32/8 heads of 128, tiles of 64:       1 sequence   3: 7.4 / 7.7,  6: 9.1 / 7.7;  8 sequences  4: 8.9 / 9.6,  6: 10.2 / 9.9;  16  6: 11.0 / 11.2
//   the same over codes (a grid a third larger):     1 sequence   2: 7.7 / 8.2,  4: 9.5 / 8.4;  16 sequences  4: 12.4 / 11.4,  8: 18.0 / 13.2;  64  8: 21.5 / 26.1
//   twelve rows a head (two products), 16/4 of 128:  1 sequence   1: 8.4 / 9.3,  2: 9.3 / 8.6;  16 sequences  4: 11.8 / 10.8;  64  8: 17.0 / 19.9
//   60 new tokens, 12/4 heads of 64:                 1 sequence   3: 12.7 / 13.6,  4: 14.8 / 13.8;  16 sequences  4: 15.2 / 16.4
// A loop of calls from the host, which a launch more takes 2.2 us longer (10.7 -> 12.8 for one sequence at any of these lengths), is not what the rule
// goes by.
inline bool whole_items(long long items, long long tiles, int ctas, int few, int most) { return tiles <= few || (tiles <= most && 4 * items >= ctas); }

// What an item is.  runs(): the items of a sequence for one head; tiles(): the steps of work of run p, at least one, and where they
// begin; uniform(): the steps where every run has the same number, else 0.

// Attention: a run of tile_tokens new tokens, a step for every KT keys that they see (a run that sees none still writes its rows).
template <int KT>
struct QueryRuns {
    static __device__ __forceinline__ int runs(const PlanParams& A, const Sequence& s) { return (s.queries + A.tile_tokens - 1) / A.tile_tokens; }
    static __device__ __forceinline__ int tiles(const PlanParams& A, const Sequence& s, int p, int& first_key) {
        const int i0 = p * A.tile_tokens, i1 = min(s.queries, i0 + A.tile_tokens) - 1, base = s.length - s.queries;
        const int end = A.causal ? min(base + i1 + 1, s.length) : s.length;
        first_key = A.window ? max(base + i0 - A.window + 1, 0) / KT * KT : 0;
        return max((end - first_key + KT - 1) / KT, 1);
    }
    static __device__ __forceinline__ int uniform(const PlanParams& A, const Sequence& s) {
        int key;
        return runs(A, s) <= 1 || !A.causal ? tiles(A, s, 0, key) : 0;
    }
};

// Weighing: a run of KT keys, a step for every tile_tokens new tokens that see some of them (keys that none sees still get their sum).
template <int KT>
struct KeyRuns {
    static __device__ __forceinline__ int runs(const PlanParams&, const Sequence& s) { return (s.length + KT - 1) / KT; }
    static __device__ __forceinline__ int tiles(const PlanParams& A, const Sequence& s, int p, int& first_run) {
        const int base = s.length - s.queries;
        int from = 0, to = s.queries;
        if (A.causal) from = max(p * KT - base, 0);
        if (A.window) to = min(to, p * KT + KT - 1 - base + A.window);
        first_run = from / A.tile_tokens;
        return max((to + A.tile_tokens - 1) / A.tile_tokens - first_run, 1);
    }
    static __device__ __forceinline__ int uniform(const PlanParams& A, const Sequence& s) {
        return s.queries <= A.tile_tokens ? 1 : A.causal ? 0 : (s.queries + A.tile_tokens - 1) / A.tile_tokens;
    }
};

// Steps of one head of sequence `b` of every lane (0 where b is none).  Whole-warp.
template <typename Runs>
__device__ __forceinline__ int sequence_tiles(const PlanParams& A, int b, bool& ok) {
    Sequence s{};
    if (b < A.seq.sequences) s = sequence_of(A.seq, b, ok);
    const int runs = b < A.seq.sequences ? Runs::runs(A, s) : 0, same = runs ? Runs::uniform(A, s) : 1;
    int sum = runs * same, first;
    if (same == 0 && runs <= 16)
        for (int p = 0; p < runs; ++p) sum += Runs::tiles(A, s, p, first);
    uint32_t many = __ballot_sync(0xffffffffu, same == 0 && runs > 16);
    const int lane = threadIdx.x & 31;
    while (many) {                                                     // the warp's lanes take a sequence's runs
        const int from = __ffs(many) - 1;
        many &= many - 1;
        Sequence t;
        t.length = __shfl_sync(0xffffffffu, s.length, from);
        t.first = 0;
        t.queries = __shfl_sync(0xffffffffu, s.queries, from);
        int part = 0;
        for (int p = lane; p < Runs::runs(A, t); p += 32) part += Runs::tiles(A, t, p, first);
        part = __reduce_add_sync(0xffffffffu, part);
        if (lane == from) sum = part;
    }
    return sum;
}

template <typename V>
__device__ __forceinline__ V warp_inclusive_sum(V v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}

// Where a CTA's stretch begins: item (b, h, p), the tile inside it, how many tiles follow, and (for the join) the first and
// last CTA that work on that item.
struct Stretch {
    int b, h, p, tile;
    int count;
    int first_cta, last_cta;
};

// Whole-warp.  `bad`: whether the host's declarations do not hold.
template <typename Runs>
__device__ __forceinline__ Stretch plan_stretch(const PlanParams& A, int cta, int ctas, bool& bad) {
    const int lane = threadIdx.x & 31;
    bool ok = true;
    int total = 0;                                                     // (plan_fits)
    const int first32 = sequence_tiles<Runs>(A, lane, ok);               // kept: most calls have no more sequences
    {
        int sum = first32;
        for (int b0 = 32; b0 < A.seq.sequences; b0 += 32) sum += sequence_tiles<Runs>(A, b0 + lane, ok);
        total = __reduce_add_sync(0xffffffffu, sum) * A.kv_heads;
    }
    bad = __any_sync(0xffffffffu, !ok);
    const int per = max((total + ctas - 1) / ctas, 1);
    Stretch r{};
    const long long lo = (long long)cta * per;
    if (lo >= total) return r;
    r.count = min(per, total - (int)lo);
    int base = 0;                                                      // tiles in front of the block of 32 sequences
    for (int b0 = 0; b0 < A.seq.sequences; b0 += 32) {
        const int t = b0 ? sequence_tiles<Runs>(A, b0 + lane, ok) : first32;
        const int all = t * A.kv_heads, sum = warp_inclusive_sum(all);
        const uint32_t hit = __ballot_sync(0xffffffffu, base + sum > (int)lo);
        if (!hit) {
            base += __shfl_sync(0xffffffffu, sum, 31);
            continue;
        }
        const int at = __ffs(hit) - 1;
        const int tiles = __shfl_sync(0xffffffffu, t, at);
        int begin = base + __shfl_sync(0xffffffffu, sum - all, at);    // first tile of the sequence
        r.b = b0 + at;
        r.h = ((int)lo - begin) / tiles;
        begin += r.h * tiles;                                          // ... of its head
        const Sequence s = sequence_of(A.seq, r.b);
        const int runs = Runs::runs(A, s), same = Runs::uniform(A, s);
        int p0 = 0;
        if (same) {
            p0 = ((int)lo - begin) / same;
            begin += p0 * same;
        }
        for (;; p0 += 32) {
            int first, n = 0;
            if (p0 + lane < runs) n = Runs::tiles(A, s, p0 + lane, first);
            const int psum = warp_inclusive_sum(n);
            const uint32_t phit = __ballot_sync(0xffffffffu, begin + psum > (int)lo);
            if (!phit) {
                begin += __shfl_sync(0xffffffffu, psum, 31);
                continue;
            }
            const int pat = __ffs(phit) - 1, size = __shfl_sync(0xffffffffu, n, pat);
            begin += __shfl_sync(0xffffffffu, psum - n, pat);
            r.p = p0 + pat;
            r.tile = (int)lo - begin;
            r.first_cta = begin / per;
            r.last_cta = (begin + size - 1) / per;
            return r;
        }
    }
    r.count = 0;
    return r;
}

// The items of a stretch, one after the other.
template <typename Runs>
struct StretchWalk {
    int b, h, p, left;
    int tile, end;             // this stretch's tiles of the item
    int tiles, first;          // all of the item's tiles, and the first key (or run of queries) of them
    Sequence s;
    __device__ __forceinline__ void begin(const PlanParams& A, const Stretch& r) {
        b = r.b; h = r.h; p = r.p; left = r.count; tile = r.tile;
        if (left > 0) {
            s = sequence_of(A.seq, b);
            load(A);
            if (A.whole && tile > 0) next(A);                          // (the item began in front of this stretch)
        }
    }
    __device__ __forceinline__ bool more() const { return left > 0; }
    __device__ __forceinline__ void next(const PlanParams& A) {
        left -= end - tile;
        if (left <= 0) return;
        tile = 0;
        if (++p == Runs::runs(A, s)) {
            p = 0;
            if (++h == A.kv_heads) {
                h = 0;
                do s = sequence_of(A.seq, ++b); while (Runs::runs(A, s) == 0);      // (another item follows: some sequence has it)
            }
        }
        load(A);
    }
    __device__ __forceinline__ bool whole() const { return tile == 0 && end == tiles; }

private:
    __device__ __forceinline__ void load(const PlanParams& A) {
        tiles = Runs::tiles(A, s, p, first);
        end = A.whole ? tiles : min(tiles, tile + left);
    }
};

// What a CTA whose stretch begins inside an item tells the join: the item and the CTAs that have parts of it.  Partial results lie
// at slot 2c (CTA c began inside the item) and 2c + 1 (the item began in CTA c's stretch and did not end there).
struct JoinNote {
    int first_cta, last_cta;   // last_cta < 0: nothing to do
    int b, h, p;
    int length, first, queries;   // the sequence
};

// Written by every CTA: the CTA behind an item's first one names it.
__device__ __forceinline__ JoinNote join_note(const PlanParams& A, const Stretch& r, int cta) {
    JoinNote n{};
    n.last_cta = -1;
    if (r.count > 0 && r.tile > 0 && r.first_cta == cta - 1) {
        n.first_cta = r.first_cta;
        n.last_cta = r.last_cta;
        n.b = r.b; n.h = r.h; n.p = r.p;
        const Sequence s = sequence_of(A.seq, r.b);
        n.length = s.length; n.first = s.first; n.queries = s.queries;
    }
    return n;
}

// ---- host -------------------------------------------------------------------------------------------------------------

// Arguments that the attention and the weighing of the cache share.
inline int check_paged_queries(const void* q, int32_t q_type, int64_t tokens, int32_t q_heads, int64_t token_stride, int64_t head_stride,
                        const vitint_cache* cache, const vitint_cache_batch* batch, float scale, int32_t causal, int32_t window) {
    if (int rc = check_cache(cache)) return rc;
    if (int rc = check_batch(cache, batch, true)) return rc;
    if (!q || tokens <= 0 || q_heads <= 0 || q_heads % cache->kv_heads != 0) return VITINT_ERR_INVALID_ARG;
    if (q_type != VITINT_BF16 && q_type != VITINT_F16) return VITINT_ERR_INVALID_ARG;
    if (cache->type != VITINT_I8 && cache->type != q_type) return VITINT_ERR_INVALID_ARG;
    if (!(scale > 0.0f && scale < INFINITY) || (causal != 0 && causal != 1) || window < 0 || (window > 0 && !causal)) return VITINT_ERR_INVALID_ARG;
    if (q_heads / cache->kv_heads > 128 || tokens > 0x7fffffffll / 128) return VITINT_ERR_UNSUPPORTED;
    if (!aligned16(q) || token_stride % 8 != 0 || head_stride % 8 != 0) return VITINT_ERR_ALIGNMENT;
    if (token_stride <= 0 || head_stride < cache->head_dim) return VITINT_ERR_INVALID_ARG;
    return VITINT_OK;
}

inline PlanParams plan_params(const vitint_cache* cache, const vitint_cache_batch* batch, int64_t tokens, int32_t q_heads, int32_t causal,
                              int32_t window) {
    PlanParams a{};
    a.seq = sequence_view(cache, batch, tokens);
    a.kv_heads = cache->kv_heads;
    a.group = q_heads / cache->kv_heads;
    a.causal = causal;
    a.window = window >= batch->max_length ? 0 : window;
    return a;
}

// Items (heads of the cache times a sequence's runs) and all their tiles, for the host's bounds.  The device counts tiles in 32 bits, and rounds their number
// up to the CTAs' stretches: false where that does not hold them.
constexpr long long PLAN_MOST_TILES = 0x7fffffffll - (1 << 16);
inline bool plan_fits(const vitint_cache* cache, const vitint_cache_batch* batch, long long runs, long long tiles, long long& items) {
    items = (long long)batch->sequences * cache->kv_heads * runs;        // (each below 2^16, 2^16 and 2^25)
    return items <= PLAN_MOST_TILES && items * tiles <= PLAN_MOST_TILES;
}
// Runs of `tokens` new tokens each that a sequence may have: no more new tokens than the call has rows, whatever the host's bound.
inline long long most_runs(const vitint_cache_batch* batch, int64_t rows, int tokens) {
    const int64_t most = batch->max_queries < rows ? batch->max_queries : rows;
    return (most + tokens - 1) / tokens;
}

inline size_t notes_bytes(int ctas) { return ((size_t)ctas * sizeof(JoinNote) + 255) & ~(size_t)255; }

}  // namespace vitint
