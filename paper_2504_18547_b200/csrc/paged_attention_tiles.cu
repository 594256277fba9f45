// Attention of many new tokens over the paged cache: items of two tiles of up to 128 rows (new tokens x query heads of a group).
//
// Per tile of 128 keys:  S = Q K^T (tcgen05, fp32 in tensor memory),  P = 2^(S c - m) rounded to 16 bits (in tensor memory, over S),
// O += P V (tcgen05, P from tensor memory).  The row maximum m is one that is not far below the true one: it follows only when a score exceeds
// it by more than 2^8, so O is rescaled a few times at most; the outputs and the sum l refer to the same m, and O / l does not depend
// on it.
//
// Bound by the exponential and the tensor core alike: 128 x 128 scores of 128 channels take 1024 cycles of tcgen05 (S and P V) and 1024 of the
// special-function unit.  So two query tiles share the stream of keys and values: while the tensor core works on one, the other's four warps
// (a row a thread: no shuffles) compute its probabilities.  One warp copies (TMA, a page's piece a copy), one issues the products.  8-bit
// codes are expanded to 16-bit operands by four more warps (exact), their steps multiply scores and probabilities.
// Work is shared out evenly over one CTA an SM (paged_plan.cuh); items split between CTAs are joined by a second kernel.
//
// 2048 tokens over 18,432 (32 query heads on 8 of 128): 503 - 530 us in a burst (1110 - 1160 TFLOP/s), 615 in a long loop under the power cap; over codes
// 1102 us in a burst (530 TFLOP/s).  A half's
// probabilities (1.2 us) and its two products (0.9 us until the next scores are there, 0.55 of it work) follow one another, as the next scores take the
// columns of the probabilities: with two halves the tensor core is busy for three quarters of the time.  Several chunks of up to 701 tokens with a
// window (12 heads on 4 of 64): 39 us, ten tiles a CTA, where the plan (2 us), changes of items (2 to 4 us each) and the join (6 us) count as much.
#include "paged_tiles.cuh"

namespace vitint {
namespace {

constexpr int PT_KEYS = 128;
constexpr int PT_TMA = 8, PT_MMA = 9, PT_EXPAND = 10;                   // warps behind the two groups of four
constexpr int PT_MAX_SLOTS = 10;
constexpr int PT_STEP_SLOTS = 2;

template <int D, bool CODES>
struct TilesShape {
    static constexpr int LINES = D / 64;
    static constexpr int OPERAND = LINES * 16384;                       // a tile of 128 rows as an operand
    static constexpr int RAW = PT_KEYS * D;                             // ... of codes as they come
    static constexpr int Q_BUFFERS = D == 64 ? 2 : 1;                   // the next item's queries arrive beside this one's where there is room
    static constexpr int SLOTS = CODES ? (D == 128 ? 4 : 6) : (D == 128 ? 5 : 8);
    static constexpr int RAW_SLOTS = CODES ? (D == 128 ? 2 : 4) : 0;
    static constexpr int THREADS = (CODES ? 14 : 10) * 32;
    static constexpr int STEPS = (2 * Q_BUFFERS + SLOTS) * OPERAND + RAW_SLOTS * RAW;       // offsets: codes' steps, barriers
    static constexpr int TAIL = STEPS + (CODES ? PT_STEP_SLOTS * 2 * PT_KEYS * 4 : 0);
    static constexpr int SMEM = TAIL + 512;
    static constexpr int PART = 2 * (D + 2) * 128;                      // floats of a partial result: [half][output columns, maximum, sum][row]
};

// Operands' type of the second product, and the offset of the probabilities in it: they are at most 2^8, as the maximum lags.
template <typename T, bool CODES>
using TilesOperand = typename std::conditional<CODES, __half, T>::type;
template <typename T, bool CODES>
constexpr float TILES_OFFSET = probability_offset<TilesOperand<T, CODES>>(8);

struct TilesParams {
    PlanParams plan;                                                    // tile_tokens: of both halves
    int half_tokens;
    void* out;
    float* lse;
    const float *k_steps, *v_steps;
    long long out_token, out_head;
    int q_heads, page_rows, box_rows;
    float c;                                                            // scale * log2(e)
    float* partial;
    JoinNote* notes;
};

struct TilesBars {
    uint64_t q_full[2], q_empty[2], full[PT_MAX_SLOTS], empty[PT_MAX_SLOTS], raw_full[4], raw_empty[4], steps_full[PT_STEP_SLOTS], steps_empty[PT_STEP_SLOTS],
        s_full[2], p_full[2], pv_done[2], drained;
};

struct TilesTail {
    TilesBars bars;
    Stretch stretch;
    uint32_t tmem_slot;
    int abort_flag;
};
static_assert(sizeof(TilesTail) <= 512, "shared memory");

struct TileRing {
    int at = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void step(int n) {
        if (++at == n) { at = 0; phase ^= 1u; }
    }
};

// Half x of an item: its tokens, rows, and the key tiles of this stretch that some of them see.
struct Half {
    int i0, rows;                                                       // first token (in the sequence's new ones), live rows
    int from, to;                                                       // tiles, from >= to: none
    int low_last, high_first;                                           // first key that the last token sees, end of what the first one sees
    int low, high;                                                      // keys that some token sees
};
__device__ __forceinline__ Half half_of(const TilesParams& P, const StretchWalk<QueryRuns<PT_KEYS>>& w, int x) {
    Half h;
    h.i0 = w.p * P.plan.tile_tokens + x * P.half_tokens;
    const int tokens = min(P.half_tokens, w.s.queries - h.i0), base = w.s.length - w.s.queries + h.i0;
    h.rows = max(tokens, 0) * P.plan.group;
    const int end = P.plan.causal ? min(base + tokens, w.s.length) : w.s.length;
    const int begin = P.plan.window ? max(base - P.plan.window + 1, 0) : 0;
    h.low_last = P.plan.window ? base + tokens - P.plan.window : 0;
    h.high_first = P.plan.causal ? min(base + 1, w.s.length) : w.s.length;
    h.low = begin;
    h.high = end;
    h.from = max(w.tile, (begin - w.first) / PT_KEYS);
    h.to = min(w.end, (end - w.first + PT_KEYS - 1) / PT_KEYS);
    if (tokens <= 0 || end <= begin) h.to = h.from;
    return h;
}

// Scores of 32 keys (those of codes times the keys' steps): the maximum with what was there.
template <bool CODES, bool EDGE>
__device__ __forceinline__ void tile_max(const uint32_t (&v)[32], const float* steps, uint32_t seen, float (&top)[4]) {
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
        float4 f;
        if (CODES) f = *reinterpret_cast<const float4*>(steps + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float s = __uint_as_float(v[i + k]);
            if (CODES) s *= k == 0 ? f.x : k == 1 ? f.y : k == 2 ? f.z : f.w;
            if (EDGE && !(seen & (1u << (i + k)))) s = -INFINITY;
            top[k] = fmaxf(top[k], s);
        }
    }
}

// Probabilities of 32 keys: 2^(s c - base), their sum, and 16 bits of each (times the value's step) for the second product.  EDGE: some keys are
// hidden; what their scores and steps are, behind the length anything, does not matter.
template <typename T, bool CODES, bool EDGE>
__device__ __forceinline__ void tile_probabilities(const uint32_t (&v)[32], const float* steps, uint32_t seen, float up, f32x2 c2, f32x2 minus_base, f32x2 (&sum)[2],
                                                   uint32_t (&out)[16]) {
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
        float4 kf, vf;
        if (CODES) {
            kf = *reinterpret_cast<const float4*>(steps + i);
            vf = *reinterpret_cast<const float4*>(steps + PT_KEYS + i);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            f32x2 s = f2_pack(__uint_as_float(v[i + 2 * k]), __uint_as_float(v[i + 2 * k + 1]));
            if (CODES) s = f2_mul(s, k ? f2_pack(kf.z, kf.w) : f2_pack(kf.x, kf.y));
            s = f2_fma(s, c2, minus_base);
            float a, b;
            f2_unpack(s, a, b);
            const bool seen_a = !EDGE || (seen & (1u << (i + 2 * k))), seen_b = !EDGE || (seen & (2u << (i + 2 * k)));
            a = seen_a ? exp2_approx(a) : 0.0f;
            b = seen_b ? exp2_approx(b) : 0.0f;
            sum[k] = f2_add(sum[k], f2_pack(a, b));
            if (CODES) {
                a = seen_a ? a * ((k ? vf.z : vf.x) * up) : 0.0f;
                b = seen_b ? b * ((k ? vf.w : vf.y) * up) : 0.0f;
            }
            out[(i >> 1) + k] = pack16<T>(a, b);
        }
    }
}

template <int D, typename T, bool CODES>
__global__ void __launch_bounds__(TilesShape<D, CODES>::THREADS, 1)
paged_tiles_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                   const __grid_constant__ TilesParams P) {
    using S = TilesShape<D, CODES>;
    using Runs = QueryRuns<PT_KEYS>;
    constexpr int LINES = S::LINES;
    // Codes: probabilities times value steps enter the second product in fp16, relative to the largest step so far (its power of two).
    constexpr bool SCALED = CODES;
    using M = TilesOperand<T, CODES>;
    constexpr float OFFSET = TILES_OFFSET<T, CODES>;
    constexpr bool BF16 = std::is_same<T, __nv_bfloat16>::value;
    constexpr uint32_t O_COL = 256;                                     // tensor memory: S and P of the halves at 0 and 128, O at 256 and 256 + D
    extern __shared__ __align__(1024) uint8_t pt_smem[];
    // (no other shared memory: the operands begin at its start, on a swizzle atom)
    TilesTail& tail = *reinterpret_cast<TilesTail*>(pt_smem + S::TAIL);
    TilesBars& B = tail.bars;
    float(*const steps)[2 * PT_KEYS] = reinterpret_cast<float(*)[2 * PT_KEYS]>(pt_smem + S::STEPS);      // codes: key steps, value steps of a tile
    volatile int* const abort_ptr = &tail.abort_flag;
    const uint32_t smem = ptx::smem_addr(pt_smem);
    uint8_t* const gen = pt_smem;
    const uint32_t ring = smem + 2 * S::Q_BUFFERS * S::OPERAND, raw_ring = ring + S::SLOTS * S::OPERAND;
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        tail.abort_flag = 0;
        auto init = [&](uint64_t* b, int n, int count) { for (int i = 0; i < n; ++i) ptx::mbar_init(ptx::smem_addr(b + i), count); };
        init(B.q_full, 2, 1);
        init(B.q_empty, 2, 1);
        init(B.full, PT_MAX_SLOTS, CODES ? 4 : 1);
        init(B.empty, PT_MAX_SLOTS, 1);
        init(B.raw_full, 4, 1);
        init(B.raw_empty, 4, 4);
        init(B.steps_full, PT_STEP_SLOTS, 1);
        init(B.steps_empty, PT_STEP_SLOTS, 8);
        init(B.s_full, 2, 1);
        init(B.p_full, 2, 4);
        init(B.pv_done, 2, 1);
        init(&B.drained, 1, 1);
        ptx::fence_mbar_init();
        ptx::fence_proxy_async_smem();
    }
    if (warp == PT_MMA) {
        ptx::tmem_alloc(ptx::smem_addr(&tail.tmem_slot), 512);
        ptx::tmem_relinquish();
    }
    if (warp == PT_TMA && lane == 0) { ptx::prefetch_tensormap(&map_q); ptx::prefetch_tensormap(&map_k); ptx::prefetch_tensormap(&map_v); }
    grid_dependency_wait();
    grid_dependency_launch();
    if (warp == 0) {
        bool bad = false;
        const Stretch r = plan_stretch<Runs>(P.plan, blockIdx.x, gridDim.x, bad);
        if (lane == 0) {
            tail.stretch = r;
            if (bad && blockIdx.x == 0) report_bad_data();
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tail.tmem_slot, 0);
    StretchWalk<Runs> w;
    // (by a thread that waits for its first tile anyway)
    if (threadIdx.x == 32) P.notes[blockIdx.x] = join_note(P.plan, tail.stretch, blockIdx.x);
    w.begin(P.plan, tail.stretch);
    bool ok = true;

    if (warp == PT_TMA) {
        // ---- copies: per key tile the keys, then the values; lane r copies the r-th piece of page rows ------------------------
        TileRing slot, step_slot;
        int issued = 0, steps_issued = 0, items = 0;
        const int copies = PT_KEYS / P.page_rows, page_mask = (1 << P.plan.seq.page_shift) - 1;
        constexpr int RING = CODES ? S::RAW_SLOTS : S::SLOTS;
        uint64_t *const full = CODES ? B.raw_full : B.full, *const empty = CODES ? B.raw_empty : B.empty;
        for (; ok && w.more(); w.next(P.plan)) {
            auto key_at = [&](int t) { return w.first + t * PT_KEYS + lane * P.page_rows; };
            auto copied = [&](int t) { return lane < copies && t < w.end && key_at(t) < w.s.length; };
            int next = copied(w.tile) ? page_entry(P.plan.seq, w.b, key_at(w.tile)) : 0;
            for (int t = w.tile; ok && t < w.end; ++t) {
                const int key = key_at(t);
                const bool mine = copied(t);
                const int here = mine ? checked_page(P.plan.seq, next) : 0;
                const bool inside = mine && here < P.plan.seq.pages;
                const uint32_t n = __popc(__ballot_sync(0xffffffffu, mine));
                if (copied(t + 1)) next = page_entry(P.plan.seq, w.b, key_at(t + 1));
                if (CODES) {
                    const uint32_t n_steps = __popc(__ballot_sync(0xffffffffu, inside));
                    ok = mbar_wait_warp(ptx::smem_addr(&B.steps_empty[step_slot.at]), step_slot.phase ^ 1u, abort_ptr);
                    if (!ok) break;
                    const uint32_t bar = ptx::smem_addr(&B.steps_full[step_slot.at]), to = ptx::smem_addr(&steps[step_slot.at][0]) + lane * P.page_rows * 4;
                    if (mine && !inside) zero_steps(reinterpret_cast<uint8_t*>(&steps[step_slot.at][0]) + lane * P.page_rows * 4, PT_KEYS * 4, P.page_rows);
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive_expect_tx(bar, 2u * n_steps * P.page_rows * 4u);
                    __syncwarp();
                    if (inside) {
                        const long long at = (((long long)here * P.plan.kv_heads + w.h) << P.plan.seq.page_shift) + (key & page_mask);
                        bulk_copy(to, P.k_steps + at, P.page_rows * 4, bar);
                        bulk_copy(to + PT_KEYS * 4, P.v_steps + at, P.page_rows * 4, bar);
                    }
                    __syncwarp();
                    ++steps_issued;
                    step_slot.step(PT_STEP_SLOTS);
                }
                for (int kv = 0; kv < 2; ++kv) {
                    ok = mbar_wait_warp(ptx::smem_addr(&empty[slot.at]), slot.phase ^ 1u, abort_ptr);
                    if (!ok) break;
                    const CUtensorMap* const map = kv ? &map_v : &map_k;
                    const uint32_t bar = ptx::smem_addr(&full[slot.at]);
                    if (lane == 0) ptx::mbar_arrive_expect_tx(bar, n * P.page_rows * (CODES ? D : 2 * D));
                    __syncwarp();
                    if (mine) {
                        if (CODES) {
                            ptx::tma_load_5d(raw_ring + slot.at * S::RAW + lane * P.page_rows * D, map, bar, 0, key & page_mask, 0, w.h, here);
                        } else {
                            for (int i = 0; i < LINES; ++i)
                                ptx::tma_load_5d(ring + slot.at * S::OPERAND + i * 16384 + lane * P.page_rows * 128, map, bar, 0, key & page_mask, i, w.h, here);
                        }
                    }
                    __syncwarp();
                    ++issued;
                    slot.step(RING);
                }
                if (!ok || t > w.tile) continue;
                // queries, behind the first keys and values: those need not wait until the last item's have been read
                const int buffer = items % S::Q_BUFFERS;
                ok = mbar_wait_warp(ptx::smem_addr(&B.q_empty[buffer]), (uint32_t)(items / S::Q_BUFFERS & 1) ^ 1u, abort_ptr);
                if (!ok) break;
                ++items;
                if (ptx::elect_one()) {
                    const uint32_t bar = ptx::smem_addr(&B.q_full[buffer]);
                    const int second = w.p * P.plan.tile_tokens + P.half_tokens < w.s.queries ? 2 : 1;
                    ptx::mbar_arrive_expect_tx(bar, second * LINES * P.box_rows * 128);
                    for (int x = 0; x < second; ++x)
                        for (int i = 0; i < LINES; ++i)
                            ptx::tma_load_4d(smem + (2 * buffer + x) * S::OPERAND + i * 16384, &map_q, bar, 0, w.h * P.plan.group,
                                             w.s.first + w.p * P.plan.tile_tokens + x * P.half_tokens, i);
                }
                __syncwarp();
            }
        }
        if (!ok) {                                                      // copies in flight are given a bounded chance to land
            auto drain = [&](uint64_t* bars, TileRing r, int size, int count) {
                for (int i = 0; i < size && i < count; ++i) {
                    if (r.at == 0) { r.at = size; r.phase ^= 1u; }
                    --r.at;
                    for (int spin = 0; spin < (1 << 16) && !ptx::mbar_try_wait(ptx::smem_addr(&bars[r.at]), r.phase); ++spin) {}
                }
            };
            drain(full, slot, RING, issued);
            if (CODES) drain(B.steps_full, step_slot, PT_STEP_SLOTS, steps_issued);
            for (int k = 1; k <= S::Q_BUFFERS && k <= items; ++k)
                for (int spin = 0; spin < (1 << 16) && !ptx::mbar_try_wait(ptx::smem_addr(&B.q_full[(items - k) % S::Q_BUFFERS]),
                                                                           (uint32_t)((items - k) / S::Q_BUFFERS) & 1u); ++spin) {}
        }
    } else if (warp == PT_MMA) {
        // ---- products: P V of a tile and Q K^T of the next, one half after the other ------------------------------------------
        TileRing r;                                                     // the next entry of the ring: keys of the first tile, values, keys, ...
        uint32_t items = 0, n_p[2] = {0, 0};
        const uint32_t idesc_qk = ptx::idesc_f16(128, PT_KEYS, BF16, 0), idesc_pv = ptx::idesc_f16(128, D, std::is_same<M, __nv_bfloat16>::value, 1);
        uint32_t q_at = 0;                                              // this item's query buffer
        auto issue_qk = [&](int x, int at) {
            const uint64_t a = ptx::smem_desc(smem + (2 * q_at + x) * S::OPERAND, 16, 1024, ptx::SWIZZLE_128B);
            const uint64_t b = ptx::smem_desc(ring + at * S::OPERAND, 16, 1024, ptx::SWIZZLE_128B);
            if (ptx::elect_one()) {
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
                    ptx::mma_f16(tmem + x * 128, a + (uint64_t)((i >> 2) * 1024 + (i & 3) * 2), b + (uint64_t)((i >> 2) * 1024 + (i & 3) * 2), idesc_qk, i > 0);
                ptx::mma_commit(ptx::smem_addr(&B.s_full[x]));
            }
            __syncwarp();
        };
        for (; ok && w.more(); w.next(P.plan)) {
            const Half half[2] = {half_of(P, w, 0), half_of(P, w, 1)};
            q_at = items % S::Q_BUFFERS;
            ok = mbar_wait_warp(ptx::smem_addr(&B.q_full[q_at]), items / S::Q_BUFFERS & 1u, abort_ptr) && mbar_wait_warp(ptx::smem_addr(&B.full[r.at]), r.phase, abort_ptr);
            if (!ok) break;
            ++items;
            ptx::tc_fence_after();
            for (int x = 0; x < 2; ++x)
                if (w.tile >= half[x].from && w.tile < half[x].to) issue_qk(x, r.at);
            if (ptx::elect_one()) ptx::mma_commit(ptx::smem_addr(&B.empty[r.at]));
            __syncwarp();
            r.step(S::SLOTS);
            for (int t = w.tile; ok && t < w.end; ++t) {
                const bool more = t + 1 < w.end;
                TileRing next = r;                                      // r: this tile's values, next: the next one's keys
                next.step(S::SLOTS);
                ok = mbar_wait_warp(ptx::smem_addr(&B.full[r.at]), r.phase, abort_ptr);
                if (!ok) break;
                const int valid = w.s.length - (w.first + t * PT_KEYS);
                if (!CODES && valid < PT_KEYS) {
                    // places behind the length: zeros instead of whatever lies there (NaN times a probability of 0)
                    uint8_t* const v = gen + 2 * S::Q_BUFFERS * S::OPERAND + r.at * S::OPERAND;
                    for (int i = max(valid, 0) * 8 + lane; i < PT_KEYS * 8; i += 32)
#pragma unroll
                        for (int line = 0; line < LINES; ++line) *reinterpret_cast<uint4*>(v + line * 16384 + i * 16) = make_uint4(0u, 0u, 0u, 0u);
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                }
                bool have_keys = false;
                for (int x = 0; ok && x < 2; ++x) {
                    if (t >= half[x].from && t < half[x].to) {
                        const uint64_t b = ptx::smem_desc(ring + r.at * S::OPERAND, 16384, 1024, ptx::SWIZZLE_128B);
                        ok = mbar_wait_warp(ptx::smem_addr(&B.p_full[x]), n_p[x] & 1u, abort_ptr);
                        if (!ok) break;
                        ptx::tc_fence_after();
                        if (ptx::elect_one()) {
#pragma unroll
                            for (int i = 0; i < PT_KEYS / 16; ++i)
                                ptx::mma_f16_ta(tmem + O_COL + x * D, tmem + x * 128 + i * 8, b + (uint64_t)(i * 128), idesc_pv, t > half[x].from || i > 0);
                            ptx::mma_commit(ptx::smem_addr(&B.pv_done[x]));
                        }
                        __syncwarp();
                        ++n_p[x];
                    }
                    if (more && t + 1 >= half[x].from && t + 1 < half[x].to) {
                        if (!have_keys) ok = mbar_wait_warp(ptx::smem_addr(&B.full[next.at]), next.phase, abort_ptr);
                        if (!ok) break;
                        have_keys = true;
                        ptx::tc_fence_after();
                        issue_qk(x, next.at);
                    }
                }
                if (!ok) break;
                if (more && !have_keys) ok = mbar_wait_warp(ptx::smem_addr(&B.full[next.at]), next.phase, abort_ptr);
                if (ptx::elect_one()) {
                    ptx::mma_commit(ptx::smem_addr(&B.empty[r.at]));
                    if (more) ptx::mma_commit(ptx::smem_addr(&B.empty[next.at]));
                }
                __syncwarp();
                r.step(S::SLOTS);
                if (more) r.step(S::SLOTS);
            }
            if (ok && ptx::elect_one()) ptx::mma_commit(ptx::smem_addr(&B.q_empty[q_at]));
            __syncwarp();
        }
        // tensor memory is given back when nothing writes to it any more
        if (ptx::elect_one()) ptx::mma_commit(ptx::smem_addr(&B.drained));
        __syncwarp();
        for (int spin = 0; spin < (1 << 16) && !ptx::mbar_try_wait(ptx::smem_addr(&B.drained), 0u); ++spin) {}
    } else if (CODES && warp >= PT_EXPAND) {
        TileRing raw, slot;
        const int row = (warp - PT_EXPAND) * 32 + lane;
        for (; ok && w.more(); w.next(P.plan))
            for (int i = 2 * w.tile; ok && i < 2 * w.end; ++i) {
                ok = mbar_wait_warp(ptx::smem_addr(&B.raw_full[raw.at]), raw.phase, abort_ptr) &&
                     mbar_wait_warp(ptx::smem_addr(&B.empty[slot.at]), slot.phase ^ 1u, abort_ptr);
                if (!ok) break;
                const uint8_t* const from = gen + (raw_ring - smem) + raw.at * S::RAW;
                uint8_t* const to = gen + 2 * S::Q_BUFFERS * S::OPERAND + slot.at * S::OPERAND;
                if (i & 1) expand_code_row<D, __half>(from, to, row);   // values
                else expand_code_row<D, T>(from, to, row);
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    ptx::mbar_arrive(ptx::smem_addr(&B.full[slot.at]));
                    ptx::mbar_arrive(ptx::smem_addr(&B.raw_empty[raw.at]));
                }
                raw.step(S::RAW_SLOTS);
                slot.step(S::SLOTS);
            }
    } else if (warp < 8) {
        // ---- probabilities and outputs: half x, a row a thread -----------------------------------------------------------------
        const int x = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t t_row = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_s = t_row + x * 128, t_o = t_row + O_COL + x * D;
        TileRing step_slot;
        uint32_t n_s = 0;                                               // tiles done: phases of s_full and pv_done
        for (; w.more(); w.next(P.plan)) {
            const Half half = half_of(P, w, x);
            const int i = row / P.plan.group, base = w.s.length - w.s.queries + half.i0 + i;      // the row's token and its position
            const bool live = row < half.rows;
            const int high = P.plan.causal ? min(base + 1, w.s.length) : w.s.length, low = P.plan.window ? base - P.plan.window + 1 : 0;
            float m = -INFINITY;
            f32x2 sum[2] = {f2_dup(0.0f), f2_dup(0.0f)};
            uint32_t unit = 0x00800000u;
            const f32x2 c2 = f2_dup(P.c);
            for (int t = w.tile; t < w.end; ++t) {
                const bool active = t >= half.from && t < half.to;
                const float* const f = &steps[step_slot.at][0];
                if (CODES) ok = ok && mbar_wait_warp(ptx::smem_addr(&B.steps_full[step_slot.at]), step_slot.phase, abort_ptr);
                if (active) ok = ok && mbar_wait_warp(ptx::smem_addr(&B.s_full[x]), n_s & 1u, abort_ptr);
                if (active && ok) {
                    ptx::tc_fence_after();
                    const int key0 = w.first + t * PT_KEYS, lo = low - key0, hi = high - key0;
                    const bool edge = key0 < half.low_last || key0 + PT_KEYS > half.high_first;
                    // the tile's scores, two blocks of 32 at a time, and read twice (all 128 in registers: 4 % slower)
                    uint32_t v[2][32];
                    float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    ptx::tmem_ld32(t_s, v[0]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        ptx::tmem_ld_wait();
                        if (k < 3) ptx::tmem_ld32(t_s + 32 * (k + 1), v[(k + 1) & 1]);
                        if (edge) tile_max<CODES, true>(v[k & 1], f + 32 * k, seen_bits(lo - 32 * k, hi - 32 * k), top);
                        else tile_max<CODES, false>(v[k & 1], f + 32 * k, 0u, top);
                    }
                    const float mt = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * P.c;
                    uint32_t larger = unit;
                    if (SCALED) {
                        const uint4 s4 = *reinterpret_cast<const uint4*>(f + PT_KEYS + 4 * lane);
                        const uint32_t word[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (key0 + 4 * lane + k >= half.low && key0 + 4 * lane + k < half.high) larger = max(larger, word[k] & 0x7F800000u);
                        larger = min(__reduce_max_sync(0xffffffffu, larger), 0x7E800000u);      // 2^126: its reciprocal is a normal number
                    }
                    if (t == half.from) {
                        m = mt;
                        unit = larger;
                    } else {
                        // the maximum follows where a score is 2^8 times above it (or the first one comes); O with it
                        const bool grow = mt > m + 8.0f;
                        if (__any_sync(0xffffffffu, grow) || larger != unit) {
                            const float now = grow ? mt : m;
                            float factor = grow ? exp2_approx((m - OFFSET) - (now - OFFSET)) : 1.0f;
                            sum[0] = f2_mul(sum[0], f2_dup(factor));
                            sum[1] = f2_mul(sum[1], f2_dup(factor));
                            if (SCALED) factor *= __uint_as_float(0x3F800000u - min(larger - unit, 0x3F000000u));
                            m = now;
                            unit = larger;
                            ok = mbar_wait_warp(ptx::smem_addr(&B.pv_done[x]), (n_s - 1) & 1u, abort_ptr);
                            ptx::tc_fence_after();
#pragma unroll 1
                            for (int k = 0; k < D; k += 16) {
                                uint32_t old[16];
                                ptx::tmem_ld16(t_o + k, old);
                                ptx::tmem_ld_wait();
#pragma unroll
                                for (int e = 0; e < 16; ++e) old[e] = __float_as_uint(__uint_as_float(old[e]) * factor);
                                ptx::tmem_st16(t_o + k, old);
                            }
                            ptx::tmem_st_wait();
                        }
                    }
                    const f32x2 minus_base = f2_dup(m == -INFINITY ? 0.0f : OFFSET - m);
                    const float up = SCALED ? __uint_as_float(0x7F000000u - unit) : 1.0f;
                    ptx::tmem_ld32(t_s, v[0]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        ptx::tmem_ld_wait();
                        if (k < 3) ptx::tmem_ld32(t_s + 32 * (k + 1), v[(k + 1) & 1]);
                        uint32_t p[16];
                        if (edge) {
                            const uint32_t seen = seen_bits(lo - 32 * k, hi - 32 * k);
                            tile_probabilities<M, CODES, true>(v[k & 1], f + 32 * k, seen, up, c2, minus_base, sum, p);
                        } else {
                            tile_probabilities<M, CODES, false>(v[k & 1], f + 32 * k, 0u, up, c2, minus_base, sum, p);
                        }
                        ptx::tmem_st16(t_s + 16 * k, p);                // (columns whose scores have been read)
                    }
                    ptx::tmem_st_wait();
                    ptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(ptx::smem_addr(&B.p_full[x]));
                    ++n_s;
                }
                if (CODES) {
                    __syncwarp();
                    if (ok && lane == 0) ptx::mbar_arrive(ptx::smem_addr(&B.steps_empty[step_slot.at]));
                    step_slot.step(PT_STEP_SLOTS);
                }
            }
            if (half.rows == 0) continue;
            const bool some = half.from < half.to;
            if (some) ok = ok && mbar_wait_warp(ptx::smem_addr(&B.pv_done[x]), (n_s - 1) & 1u, abort_ptr);
            if (!ok) continue;
            ptx::tc_fence_after();
            float a, b, c, d;
            f2_unpack(sum[0], a, b);
            f2_unpack(sum[1], c, d);
            // (o and l without the offset, exactly; the maximum is what the exponentials were taken relative to)
            const float l = ((a + b) + (c + d)) * offset_back(OFFSET), scale = (SCALED ? __uint_as_float(unit) : 1.0f) * offset_back(OFFSET);
            const bool whole = w.whole();
            const long long token = w.s.first + half.i0 + i;
            const int head = w.h * P.plan.group + row - i * P.plan.group;
            float* const part = P.partial + (2ll * blockIdx.x + (w.tile > 0 ? 0 : 1)) * S::PART + x * (D + 2) * 128 + row;
            T* const to = (T*)P.out + token * P.out_token + head * P.out_head;
            const float inv = (l > 0.0f ? 1.0f / l : 0.0f) * scale;
#pragma unroll 1
            for (int k = 0; k < D; k += 32) {
                uint32_t v[32];
                if (some) {
                    ptx::tmem_ld32(t_o + k, v);
                    ptx::tmem_ld_wait();
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = 0u;
                }
                if (live && whole) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint32_t p[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) p[q] = pack16<T>(__uint_as_float(v[e + 2 * q]) * inv, __uint_as_float(v[e + 2 * q + 1]) * inv);
                        *reinterpret_cast<uint4*>(to + k + e) = make_uint4(p[0], p[1], p[2], p[3]);
                    }
                } else if (live) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) part[(k + e) * 128] = __uint_as_float(v[e]) * scale;
                }
                __syncwarp();                                           // (the loads above are the whole warp's)
            }
            if (live) {
                if (!whole) {
                    part[D * 128] = m - OFFSET;
                    part[(D + 1) * 128] = l;
                } else if (P.lse) {
                    P.lse[token * P.q_heads + head] = l > 0.0f ? (((m - OFFSET) + OFFSET) + log2f(l)) * 0.69314718055994531f : -INFINITY;
                }
            }
            ptx::tc_fence_before();
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == PT_MMA) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 512);
    }
}

// Joins the partial results of an item that several CTAs worked on.  Block (c, y): the item that began in front of CTA c + 1's stretch, half y / 4 of
// it, a quarter of the output columns; a row a thread.
template <int D, typename T, bool CODES>
__global__ void __launch_bounds__(128)
paged_tiles_join_kernel(const __grid_constant__ TilesParams P) {
    constexpr int PART = 2 * (D + 2) * 128, COLS = D / 4;
    grid_dependency_wait();
    grid_dependency_launch();
    const JoinNote n = P.notes[blockIdx.x + 1];
    if (n.last_cta < 0) return;
    const int x = blockIdx.y >> 2, col0 = (blockIdx.y & 3) * COLS, row = threadIdx.x;
    const Sequence s{n.length, n.first, n.queries};
    const int i0 = n.p * P.plan.tile_tokens + x * P.half_tokens, rows = min(P.half_tokens, s.queries - i0) * P.plan.group;
    if (row >= rows) return;
    float o[COLS], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int k = 0; k < COLS; ++k) o[k] = 0.0f;
    for (int cta = n.first_cta; cta <= n.last_cta; cta += 2) {           // two parts' loads under way at once
        float v[2][COLS], pm[2], pl[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            pm[i] = -INFINITY;
            pl[i] = 0.0f;
            const bool there = cta + i <= n.last_cta;
            const float* const part = P.partial + (2ll * (cta + i) + (cta + i == n.first_cta ? 1 : 0)) * PART + x * (D + 2) * 128 + row;
            if (there) { pm[i] = part[D * 128]; pl[i] = part[(D + 1) * 128]; }
#pragma unroll
            for (int k = 0; k < COLS; ++k) v[i][k] = there ? part[(col0 + k) * 128] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float top = fmaxf(m, pm[i]), base = top == -INFINITY ? 0.0f : top;
            const float mine = exp2_approx(m - base), theirs = exp2_approx(pm[i] - base);
            m = top;
            l = l * mine + pl[i] * theirs;
#pragma unroll
            for (int k = 0; k < COLS; ++k) o[k] = o[k] * mine + v[i][k] * theirs;
        }
    }
    const int i = row / P.plan.group, head = n.h * P.plan.group + row - i * P.plan.group;
    const long long token = s.first + i0 + i;
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    T* const to = (T*)P.out + token * P.out_token + head * P.out_head + col0;
#pragma unroll
    for (int k = 0; k < COLS; k += 8) {
        uint32_t p[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) p[q] = pack16<T>(o[k + 2 * q] * inv, o[k + 2 * q + 1] * inv);
        *reinterpret_cast<uint4*>(to + k) = make_uint4(p[0], p[1], p[2], p[3]);
    }
    if (P.lse && col0 == 0) P.lse[token * P.q_heads + head] = l > 0.0f ? ((m + TILES_OFFSET<T, CODES>) + log2f(l)) * 0.69314718055994531f : -INFINITY;
}

inline size_t tiles_partial_bytes(int ctas, int head_dim) { return (size_t)ctas * 2 * 2 * (head_dim + 2) * 128 * 4; }

template <int D, typename T, bool CODES>
int paged_tiles_launch(TilesParams& P, const void* q, int64_t tokens, int64_t q_token, int64_t q_head, const vitint_cache* cache, const vitint_cache_batch* batch,
                       void* workspace, cudaStream_t st) {
    using S = TilesShape<D, CODES>;
    static_assert(S::SMEM <= 227 * 1024 && S::SLOTS <= PT_MAX_SLOTS && S::RAW_SLOTS <= 4, "shared memory");
    const long long tiles = (batch->max_length + PT_KEYS - 1) / PT_KEYS;
    long long items;
    if (!plan_fits(cache, batch, most_runs(batch, tokens, P.plan.tile_tokens), tiles, items)) return VITINT_ERR_UNSUPPORTED;
    const int box_tokens = P.half_tokens < batch->max_queries ? P.half_tokens : batch->max_queries;
    P.box_rows = box_tokens * P.plan.group;
    P.page_rows = cache->page_tokens;
    CUtensorMap map_q, map_k, map_v;
    if (!encode_query_map(&map_q, q, std::is_same<T, __nv_bfloat16>::value ? VITINT_BF16 : VITINT_F16, D, tokens, P.q_heads, q_token, q_head, P.plan.group, box_tokens) ||
        !encode_cache_map(&map_k, cache, cache->k, P.page_rows, CODES) || !encode_cache_map(&map_v, cache, cache->v, P.page_rows, CODES))
        return VITINT_ERR_CUDA;
    int grid = sm_count();
    P.plan.whole = whole_items(items, tiles, grid, 3, 4);
    if (grid > items * tiles) grid = (int)(items * tiles);
    P.notes = (JoinNote*)workspace;
    P.partial = (float*)((uint8_t*)workspace + notes_bytes(sm_count()));
    const int dev = current_device();
    if (dev < 0) return VITINT_ERR_CUDA;
    static bool attr_set_dev[MAX_DEVICES] = {};
    if (!attr_set_dev[dev]) {
        if (cudaFuncSetAttribute(paged_tiles_kernel<D, T, CODES>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess) return VITINT_ERR_CUDA;
        attr_set_dev[dev] = true;
    }
    launch_kernel(paged_tiles_kernel<D, T, CODES>, dim3(grid), dim3(S::THREADS), S::SMEM, st, map_q, map_k, map_v, P);
    if (int rc = cuda_status(cudaGetLastError())) return rc;
    if (!P.plan.whole && grid > 1) launch_kernel(paged_tiles_join_kernel<D, T, CODES>, dim3(grid - 1, 8), dim3(128), 0, st, P);
    return cuda_status(cudaGetLastError());
}

}  // namespace
}  // namespace vitint
