// Attention of a few new tokens over the paged cache: at most sixteen rows (new tokens x query heads of a group) for a head of the cache.
//
//   s_rj = scale * step_j (q_r . k_j);  p = 2^(s log2 e - m);  o_r = sum_j (p_rj vstep_j) v_j / sum_j p_rj
//
// Bound by HBM: every key and value is read once for a handful of multiplications.  What the kernel has to do is to keep enough
// bytes in flight on every SM, few instructions behind them, and share the keys out evenly (paged_plan.cuh).  A producer warp copies key
// tiles (their pages' pieces, one TMA copy a page for keys and one for values) into a ring; four warps take a quarter of each tile's keys,
// each with a running maximum, sum and output of its own, so that they meet only at an item's end.
// The contractions are warp-level m16n8k16 products with the keys (then the channels of the values) as the sixteen rows and the queries
// as eight columns: S^T = K Q^T, O^T = V^T P^T.  A 128-row tcgen05 tile of queries would be empty at fifteen sixteenths, and queries as the
// sixteen rows would spend twice the products and registers on the up to eight there mostly are; up to sixteen take two products.
// 8-bit codes become fp16 operands in registers (exact): the order of the contraction's index is free as long as both sides agree, so a thread
// takes its codes as they lie, sixteen bytes at a time.
// Up to eight rows a probability is multiplied as the sum of two 16-bit numbers (the tensor core is idle otherwise), so that only the output is
// rounded.  With bf16 queries over codes it is one fp16 number: the output is rounded eight times as coarsely.
//
// One token each of 48 sequences with up to 8192 cached ones (32 query heads on 8 of 128, 680 MB): 116 us, 5.8 TB/s; 2 x 3 tokens over 131,072 (12
// rows a head): 98 us, 5.5 TB/s; 64 sequences of codes (346 MB): 85 us, 4.1 TB/s (queries as rows, bf16 operands: 123), where the ALU, which expands the
// codes, is busy for 57 % of the time and 59 % of the issue slots are taken.
#include "paged_tiles.cuh"
#include "paged_attention_tiles.cu"

namespace vitint {
namespace {

constexpr int PA_WARPS = 4;
constexpr int PA_THREADS = (PA_WARPS + 1) * 32;
constexpr int PA_ROWS = 16;

// NQ: products of eight query rows (1 or 2).
template <int D, bool CODES, int NQ>
struct RowsShape {
    static constexpr int SIZE = CODES ? 1 : 2;                         // bytes of an element
    static constexpr int ROW = D * SIZE;                               // bytes of a key
    static constexpr int LINE = ROW < 128 ? ROW : 128, LINES = ROW / LINE;
    static constexpr int KT = ROW == 256 || (CODES && D == 128) ? 64 : 128;      // keys of a tile
    static constexpr int NK = KT / PA_WARPS;                           // a warp's keys of a tile
    static constexpr int HALF = KT * ROW;                              // bytes of a tile's keys (or values)
    static constexpr int STEPS = CODES ? KT * 4 : 0;                   // bytes of a tile's key (or value) steps
    static constexpr int STAGE = 2 * HALF;
    // CTAs on an SM, and tiles in a CTA's ring.  Codes are bound by latency as much as by bytes (they are half of them, and expanded): more CTAs
    // with fewer tiles (64 sequences of up to 6001 tokens: three CTAs of four tiles 95 us, four of two 85).
    static constexpr int CTAS = NQ == 2 ? 2 : CODES ? 4 : 3;
    static constexpr int STAGES = CODES ? (NQ == 2 ? 5 : 2) : (NQ == 2 ? 3 : 2);
    static constexpr int NREG = NQ * D / 4;                            // a thread's outputs
    static constexpr int PART = NREG * 32 + NQ * 16;                   // floats of a partial result: a warp's output fragments, maxima and sums of the rows
    static constexpr int MERGE = 2 * PART * 4;
    static constexpr int SMEM = STAGES * (STAGE + 2 * STEPS) + MERGE + 256;
    static_assert(SMEM <= 233472 / CTAS - 1024, "shared memory");
};
// Operands' type of the second product, and the offset of the probabilities in it: they are at most 1.
template <typename T, bool CODES>
using RowsOperand = typename std::conditional<CODES, __half, T>::type;
template <typename T, bool CODES>
constexpr float ROWS_OFFSET = probability_offset<RowsOperand<T, CODES>>(0);

struct RowsParams {
    PlanParams plan;
    const void* q;
    void* out;
    float* lse;
    const float *k_steps, *v_steps;
    long long q_token, q_head, out_token, out_head;
    int q_heads, page_rows;                                            // rows of a copy
    float c;                                                           // scale * log2(e)
    float* partial;
    JoinNote* notes;
};

template <typename T>
__device__ __forceinline__ void mma16816(float* d, const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<__nv_bfloat16>(float* d, const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__half>(float* d, const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// An 8 x 8 matrix of 16-bit elements in fragment form (row lane / 4, columns 2 (lane % 4) and the next), transposed.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void consumer_barrier() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// Joins two partial results of the same rows: (m, l, o) <- both.  A maximum of -inf stands for no key yet.
__device__ __forceinline__ void join_scales(float m, float other, float& top, float& mine, float& theirs) {
    top = fmaxf(m, other);
    const float base = top == -INFINITY ? 0.0f : top;
    mine = exp2_approx(m - base);
    theirs = exp2_approx(other - base);
}

// Writes the finished columns (query rows 8 n + 2 (lane % 4) + e) of one product's outputs: o[4 * n + 2 * half + e] is channel 16 mt + lane / 4 + 8 half, with
// codes (D / 8) (lane / 4) + 2 mt + half.
template <int D, typename T, bool CODES, int NQ>
__device__ __forceinline__ void write_product(const RowsParams& P, const Sequence& s, int h, int p, int mt, const float* o, const float (&inv)[NQ][2]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3, i0 = p * P.plan.tile_tokens;
    const int rows = min(P.plan.tile_tokens, s.queries - i0) * P.plan.group;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        // transposed: row 8 n + g, the matrix rows 2c and 2c + 1 of both halves
        const uint32_t a = transpose8x8(pack16<T>(o[4 * n] * inv[n][0], o[4 * n + 1] * inv[n][1]));
        const uint32_t b = transpose8x8(pack16<T>(o[4 * n + 2] * inv[n][0], o[4 * n + 3] * inv[n][1]));
        const int row = 8 * n + g;
        if (row < rows) {
            const int i = row / P.plan.group, head = h * P.plan.group + row - i * P.plan.group;
            T* const to = (T*)P.out + (long long)(s.first + i0 + i) * P.out_token + head * P.out_head;
            if (CODES) {
                *reinterpret_cast<uint32_t*>(to + (D / 8) * (2 * c) + 2 * mt) = __byte_perm(a, b, 0x5410);
                *reinterpret_cast<uint32_t*>(to + (D / 8) * (2 * c + 1) + 2 * mt) = __byte_perm(a, b, 0x7632);
            } else {
                *reinterpret_cast<uint32_t*>(to + 16 * mt + 2 * c) = a;
                *reinterpret_cast<uint32_t*>(to + 16 * mt + 8 + 2 * c) = b;
            }
        }
        __syncwarp();
    }
}
// (m is lower than the maximum that l refers to by the offset, and loses nothing when that is added again)
template <int NQ>
__device__ __forceinline__ void write_lse(const RowsParams& P, const Sequence& s, int h, int p, const float (&m)[NQ][2], const float (&l)[NQ][2], float offset) {
    const int lane = threadIdx.x & 31, i0 = p * P.plan.tile_tokens, rows = min(P.plan.tile_tokens, s.queries - i0) * P.plan.group;
    if (!P.lse || lane >= 4) return;
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int row = 8 * n + 2 * lane + e;
            if (row >= rows) continue;
            const int i = row / P.plan.group, head = h * P.plan.group + row - i * P.plan.group;
            P.lse[(long long)(s.first + i0 + i) * P.q_heads + head] = l[n][e] > 0.0f ? ((m[n][e] + offset) + log2f(l[n][e])) * 0.69314718055994531f : -INFINITY;
        }
}

template <int D, typename T, bool CODES, int NQ>
__global__ void __launch_bounds__(PA_THREADS, RowsShape<D, CODES, NQ>::CTAS)
paged_rows_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ RowsParams P) {
    using S = RowsShape<D, CODES, NQ>;
    using Runs = QueryRuns<S::KT>;
    constexpr int KT = S::KT, NK = S::NK, STAGES = S::STAGES, NU = NK / 16;
    constexpr bool BF16 = std::is_same<T, __nv_bfloat16>::value;
    // Codes: queries in bf16 are brought to fp16 as multiples of a power of two for each row (exact for all that is within 2^-29 of the row's
    // largest).  Probabilities times value steps enter the second contraction in fp16 too, relative to the largest step so far (its power of two), so
    // that they do not run out of exponents.
    constexpr bool RESCALED_Q = CODES && BF16;
    using M = RowsOperand<T, CODES>;
    constexpr float OFFSET = ROWS_OFFSET<T, CODES>;
    // A second product with what the first one's rounding left, except where the output is rounded eight times as coarsely, and where the
    // products would set the pace (two columns of products: 2 x 131,072 keys, twelve rows, 101 -> 121 us).
    constexpr bool SPLIT = NQ == 1 && !(CODES && BF16);
    extern __shared__ __align__(1024) uint8_t pa_smem[];
    const uint32_t smem = ptx::smem_addr(pa_smem);
    const uint32_t steps0 = smem + STAGES * S::STAGE;                  // [stage][keys, values][KT]
    float* const merge = reinterpret_cast<float*>(pa_smem + STAGES * (S::STAGE + 2 * S::STEPS));
    uint8_t* const tail = pa_smem + S::SMEM - 256;
    const uint32_t bars = ptx::smem_addr(tail);                        // full[STAGES], empty[STAGES]
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(tail + 128);
    Stretch* const shared_stretch = reinterpret_cast<Stretch*>(tail + 160);
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int i = 0; i < STAGES; ++i) {
            ptx::mbar_init(bars + 8 * i, 1);
            ptx::mbar_init(bars + 8 * (STAGES + i), PA_WARPS);
        }
        ptx::fence_mbar_init();
        ptx::fence_proxy_async_smem();
    }
    grid_dependency_wait();
    grid_dependency_launch();
    if (warp == 0) {
        bool bad = false;
        const Stretch r = plan_stretch<Runs>(P.plan, blockIdx.x, gridDim.x, bad);
        if (lane == 0) {
            *shared_stretch = r;
            if (bad && blockIdx.x == 0) report_bad_data();
        }
    }
    __syncthreads();
    StretchWalk<Runs> w;
    // (by a thread that waits for its first tile anyway)
    if (threadIdx.x == 32) P.notes[blockIdx.x] = join_note(P.plan, *shared_stretch, blockIdx.x);
    w.begin(P.plan, *shared_stretch);
    bool ok = true;
    int stage = 0;
    uint32_t phase = 0;
    auto advance = [&] {
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
    };

    if (warp == PA_WARPS) {
        // ---- producer: lane r copies the tile's r-th run of page rows; its page is looked up a tile ahead ----------------------
        const int copies = KT / P.page_rows, copy_bytes = P.page_rows * S::ROW;
        const int page_mask = (1 << P.plan.seq.page_shift) - 1;
        int issued = 0;
        for (; ok && w.more(); w.next(P.plan)) {
            auto key_at = [&](int t) { return w.first + t * KT + lane * P.page_rows; };
            auto copied = [&](int t) { return lane < copies && t < w.end && key_at(t) < w.s.length; };
            int next = copied(w.tile) ? page_entry(P.plan.seq, w.b, key_at(w.tile)) : 0;
            for (int t = w.tile; t < w.end; ++t) {
                const int key = key_at(t);
                const bool mine = copied(t);
                const int page = mine ? checked_page(P.plan.seq, next) : 0;
                const bool inside = mine && page < P.plan.seq.pages;
                const uint32_t n = __popc(__ballot_sync(0xffffffffu, mine)), n_steps = __popc(__ballot_sync(0xffffffffu, inside));
                if (copied(t + 1)) next = page_entry(P.plan.seq, w.b, key_at(t + 1));
                ok = mbar_wait_warp(bars + 8 * (STAGES + stage), phase ^ 1u, abort_flag);
                if (!ok) break;
                const uint32_t full = bars + 8 * stage;
                if (CODES && mine && !inside) zero_steps(pa_smem + STAGES * S::STAGE + stage * 2 * S::STEPS + lane * P.page_rows * 4, S::STEPS, P.page_rows);
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive_expect_tx(full, 2u * n * copy_bytes + (CODES ? 2u * n_steps * P.page_rows * 4u : 0u));
                __syncwarp();
                if (mine) {
                    const uint32_t to = smem + stage * S::STAGE + lane * copy_bytes;
                    ptx::tma_load_5d(to, &map_k, full, 0, key & page_mask, 0, w.h, page);
                    ptx::tma_load_5d(to + S::HALF, &map_v, full, 0, key & page_mask, 0, w.h, page);
                    if (CODES && inside) {
                        const long long at = (((long long)page * P.plan.kv_heads + w.h) << P.plan.seq.page_shift) + (key & page_mask);
                        const uint32_t st = steps0 + stage * 2 * S::STEPS + lane * P.page_rows * 4;
                        bulk_copy(st, P.k_steps + at, P.page_rows * 4, full);
                        bulk_copy(st + S::STEPS, P.v_steps + at, P.page_rows * 4, full);
                    }
                }
                __syncwarp();
                ++issued;
                advance();
            }
        }
        // copies in flight when the CTA gives up are given a bounded chance to land
        if (!ok)
            for (int k = 0; k < STAGES && k < issued; ++k) {
                if (stage == 0) { stage = STAGES; phase ^= 1u; }
                --stage;
                for (int spin = 0; spin < (1 << 16) && !ptx::mbar_try_wait(bars + 8 * stage, phase); ++spin) {}
            }
        return;
    }

    // ---- four warps, a quarter of every tile's keys each ------------------------------------------------------------------
    const int g = lane >> 2, c = lane & 3, rows_shift = 31 - __clz(P.page_rows);
    // where the warp's sixteen keys lie in a tile (each in one page)
    uint32_t group_at[NU];
    int in_block[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        const int j = warp * NK + 16 * u;
        group_at[u] = (j >> rows_shift) * (P.page_rows * S::ROW);
        in_block[u] = j & (P.page_rows - 1);
    }
    while (w.more()) {
        const int i0 = w.p * P.plan.tile_tokens, tokens = min(P.plan.tile_tokens, w.s.queries - i0), rows = tokens * P.plan.group;
        const int base = w.s.length - w.s.queries + i0;                  // position of the item's first token
        // queries as the right operand: column 8 n + g
        uint32_t qb[NQ][D / 16][2];
        float sc[NQ][2];                                                 // scale of the thread's score columns 2c and 2c + 1
        int low[NQ][2], high[NQ][2];                                     // the keys that they see
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int row = 8 * n + g, i = row / P.plan.group;
            const bool live = row < rows;
            const T* const from = (const T*)P.q + (long long)(w.s.first + i0 + i) * P.q_token + (long long)(w.h * P.plan.group + row - i * P.plan.group) * P.q_head;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                if (CODES) {                                             // channels as the codes lie: 16 (c + 4 (k / 4)) + 4 (k % 4) + 0 .. 3
                    const uint2 v = live ? *reinterpret_cast<const uint2*>(from + 16 * (c + 4 * (k >> 2)) + 4 * (k & 3)) : make_uint2(0u, 0u);
                    qb[n][k][0] = v.x;
                    qb[n][k][1] = v.y;
                } else {
                    qb[n][k][0] = live ? *reinterpret_cast<const uint32_t*>(from + 16 * k + 2 * c) : 0u;
                    qb[n][k][1] = live ? *reinterpret_cast<const uint32_t*>(from + 16 * k + 8 + 2 * c) : 0u;
                }
            }
            float unscale = P.c;
            if (RESCALED_Q) {
                uint32_t largest = 0;
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
#pragma unroll
                    for (int e = 0; e < 2; ++e) largest = max(largest, max((qb[n][k][e] & 0x7FFFu) << 16, qb[n][k][e] & 0x7FFF0000u));
                largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, 1));
                largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, 2));
                // the largest becomes 2^14 .. 2^15; 2^x for x within the exponents' range on both sides
                const int shift = min(max(141 - (int)(largest >> 23), -110), 110);
                const float up = __uint_as_float((uint32_t)(127 + shift) << 23);
                unscale = P.c * __uint_as_float((uint32_t)(127 - shift) << 23);
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float2 f = unpack16<T>(qb[n][k][e]);
                        qb[n][k][e] = pack16<__half>(f.x * up, f.y * up);
                    }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                sc[n][e] = RESCALED_Q ? __shfl_sync(0xffffffffu, unscale, (2 * c + e) * 4) : P.c;
                const int mine = 8 * n + 2 * c + e, token = mine / P.plan.group;
                high[n][e] = mine >= rows ? 0 : P.plan.causal ? min(base + token + 1, w.s.length) : w.s.length;
                low[n][e] = P.plan.window ? base + token - P.plan.window + 1 : 0;
            }
        }
        const int all_low = P.plan.window ? base + tokens - P.plan.window : 0;                               // the last row's
        const int all_high = P.plan.causal ? min(base + 1, w.s.length) : w.s.length;                         // the first row's
        const int some_low = P.plan.window ? base - P.plan.window + 1 : 0;                                    // keys that some row sees
        const int some_high = P.plan.causal ? min(base + tokens, w.s.length) : w.s.length;
        float o[D / 16][4 * NQ], m[NQ][2], l[NQ][2];
        uint32_t unit = 0x00800000u;                                     // CODES: the power of two that o is a multiple of
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) { m[n][e] = -INFINITY; l[n][e] = 0.0f; }
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int e = 0; e < 4 * NQ; ++e) o[i][e] = 0.0f;

        for (int t = w.tile; t < w.end; ++t) {
            ok = ok && mbar_wait_warp(bars + 8 * stage, phase, abort_flag);
            if (ok) {
                const uint32_t kbase = smem + stage * S::STAGE;
                const int key0 = w.first + t * KT + warp * NK;
                const bool edge = key0 < all_low || key0 + NK > all_high;
                float s[NU][4 * NQ];
#pragma unroll
                for (int u = 0; u < NU; ++u) {                           // sixteen keys
                    const uint32_t at = kbase + group_at[u];
#pragma unroll
                    for (int e = 0; e < 4 * NQ; ++e) s[u][e] = 0.0f;
                    if (!CODES) {
                        const int row = in_block[u] + ((lane >> 3) & 1) * 8 + (lane & 7), odd = lane >> 4;
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const int chunk = 2 * k + odd;
                            uint32_t a[4];
                            ldmatrix4(at + (chunk >> 3) * (P.page_rows * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4), a);
#pragma unroll
                            for (int n = 0; n < NQ; ++n) mma16816<M>(&s[u][4 * n], a, qb[n][k][0], qb[n][k][1]);
                        }
                    } else {
                        const int row = in_block[u] + g;                 // and row + 8, whose swizzle is the same
#pragma unroll
                        for (int x = 0; x < D / 64; ++x) {
                            const uint32_t chunk = c + 4 * x;
                            const uint32_t from = at + row * S::LINE + ((S::LINE == 128 ? chunk ^ (row & 7) : chunk ^ ((row >> 1) & 3)) << 4);
                            const uint4 v0 = lds128(from), v1 = lds128(from + 8 * S::LINE);
                            const uint32_t w0[4] = {v0.x, v0.y, v0.z, v0.w}, w1[4] = {v1.x, v1.y, v1.z, v1.w};
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const uint2 e0 = codes_to_half4(w0[k]), e1 = codes_to_half4(w1[k]);
                                const uint32_t a[4] = {e0.x, e1.x, e0.y, e1.y};
#pragma unroll
                                for (int n = 0; n < NQ; ++n) mma16816<M>(&s[u][4 * n], a, qb[n][4 * x + k][0], qb[n][4 * x + k][1]);
                            }
                        }
                    }
                }
                // scores in units of log2, hidden ones -inf, and the columns' maxima.  s[u][4 n + 2 r + e]: key 16 u + g + 8 r, column 8 n + 2c + e
                const float* const ks = reinterpret_cast<const float*>(pa_smem + STAGES * S::STAGE + stage * 2 * S::STEPS) + warp * NK + g;
                const float* const vs = ks + KT;
                float top[NQ][2];
#pragma unroll
                for (int n = 0; n < NQ; ++n) { top[n][0] = m[n][0]; top[n][1] = m[n][1]; }
#pragma unroll
                for (int u = 0; u < NU; ++u)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float step = CODES ? ks[16 * u + 8 * r] : 1.0f;
#pragma unroll
                        for (int n = 0; n < NQ; ++n)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                float& x = s[u][4 * n + 2 * r + e];
                                x *= CODES ? sc[n][e] * step : sc[n][e];
                                if (edge) {
                                    const int key = key0 + 16 * u + 8 * r + g;
                                    if (key < low[n][e] || key >= high[n][e]) x = -INFINITY;
                                }
                                top[n][e] = fmaxf(top[n][e], x);
                            }
                    }
                bool grew = false;
                float from[NQ][2];
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) top[n][e] = fmaxf(top[n][e], __shfl_xor_sync(0xffffffffu, top[n][e], x));
                        from[n][e] = (top[n][e] == -INFINITY ? 0.0f : top[n][e]) - OFFSET;
                        grew = grew || top[n][e] != m[n][e];
                    }
                if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float factor = exp2_approx((m[n][e] - OFFSET) - from[n][e]);
                            l[n][e] *= factor;
                            m[n][e] = top[n][e];
#pragma unroll
                            for (int i = 0; i < D / 16; ++i) { o[i][4 * n + e] *= factor; o[i][4 * n + 2 + e] *= factor; }
                        }
                }
#pragma unroll
                for (int u = 0; u < NU; ++u)
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float& x = s[u][4 * n + e];
                            x = exp2_approx(x - from[n][e & 1]);
                            l[n][e & 1] += x;
                        }
                if (CODES) {
                    float step[NU][2];
                    uint32_t largest = unit;
#pragma unroll
                    for (int u = 0; u < NU; ++u)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            step[u][r] = vs[16 * u + 8 * r];
                            if (edge) {                                  // no row sees it: whatever lies there, and no part of the largest step
                                const int key = key0 + 16 * u + 8 * r + g;
                                if (key < some_low || key >= some_high) step[u][r] = 0.0f;
                            }
                            largest = max(largest, __float_as_uint(step[u][r]) & 0x7F800000u);
                        }
                    largest = min(__reduce_max_sync(0xffffffffu, largest), 0x7E800000u);      // 2^126: its reciprocal is a normal number
                    if (largest != unit) {
                        const float down = __uint_as_float(0x3F800000u - min(largest - unit, 0x3F000000u));
#pragma unroll
                        for (int i = 0; i < D / 16; ++i)
#pragma unroll
                            for (int e = 0; e < 4 * NQ; ++e) o[i][e] *= down;
                        unit = largest;
                    }
                    const float up = __uint_as_float(0x7F000000u - unit);                                   // 1 / unit
#pragma unroll
                    for (int u = 0; u < NU; ++u)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const float f = step[u][r] * up;
#pragma unroll
                            for (int n = 0; n < NQ; ++n) { s[u][4 * n + 2 * r] *= f; s[u][4 * n + 2 * r + 1] *= f; }
                        }
                }
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    // probabilities as the right operand: columns 8 n + g, keys 2c, 2c + 1 and 8 further
                    uint32_t pb[NQ][2], rest[NQ][2];
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const float a = s[u][4 * n + 2 * r], b = s[u][4 * n + 2 * r + 1];
                            const uint32_t first = pack16<M>(a, b);
                            pb[n][r] = transpose8x8(first);
                            if (SPLIT) {
                                const float2 f = unpack16<M>(first);
                                rest[n][r] = transpose8x8(pack16<M>(a - f.x, b - f.y));
                            }
                        }
                    const uint32_t at = kbase + S::HALF + group_at[u];
                    auto product = [&](int mt, const uint32_t (&a)[4]) {
#pragma unroll
                        for (int n = 0; n < NQ; ++n) {
                            mma16816<M>(&o[mt][4 * n], a, pb[n][0], pb[n][1]);
                            if (SPLIT) mma16816<M>(&o[mt][4 * n], a, rest[n][0], rest[n][1]);
                        }
                    };
                    if (!CODES) {
                        uint32_t mask0 = 0xFFFFFFFFu, mask1 = 0xFFFFFFFFu;     // values behind the length are not multiplied: NaN times 0
                        if (edge) {
                            const int key = key0 + 16 * u + 2 * c;
                            mask0 = (key < w.s.length ? 0xFFFFu : 0u) | (key + 1 < w.s.length ? 0xFFFF0000u : 0u);
                            mask1 = (key + 8 < w.s.length ? 0xFFFFu : 0u) | (key + 9 < w.s.length ? 0xFFFF0000u : 0u);
                        }
                        const int row = in_block[u] + (lane >> 4) * 8 + (lane & 7), odd = (lane >> 3) & 1;
#pragma unroll
                        for (int mt = 0; mt < D / 16; ++mt) {
                            const int chunk = 2 * mt + odd;
                            uint32_t a[4];
                            ldmatrix4_trans(at + (chunk >> 3) * (P.page_rows * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4), a);
                            if (edge) { a[0] &= mask0; a[1] &= mask0; a[2] &= mask1; a[3] &= mask1; }
                            product(mt, a);
                        }
                    } else {
                        // D/8 codes of four keys: the thread's channels (D/8) g + 0, 1, ...
                        uint32_t words[4][D / 32];
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int row = in_block[u] + 2 * c + (x & 1) + 8 * (x >> 1);
                            if (D == 128) {
                                const uint4 v = lds128(at + row * 128 + ((g ^ (row & 7)) << 4));
                                words[x][0] = v.x; words[x][1] = v.y; words[x][D / 32 - 2] = v.z; words[x][D / 32 - 1] = v.w;
                            } else {
                                const uint2 v = lds64(at + row * 64 + ((((uint32_t)g >> 1) ^ ((row >> 1) & 3)) << 4) + (g & 1) * 8);
                                words[x][0] = v.x; words[x][1] = v.y;
                            }
                        }
#pragma unroll
                        for (int mt = 0; mt < D / 16; ++mt) {
                            uint32_t a[4];
#pragma unroll
                            for (int r = 0; r < 4; ++r) {                // channel 2 mt + r % 2, keys (r / 2) * 8 + 2c and the next
                                const int j = 2 * mt + (r & 1), x = 2 * (r >> 1);
                                a[r] = codes_to_16<__half>(__byte_perm(words[x][j >> 2], words[x + 1][j >> 2], (j & 3) | ((4 + (j & 3)) << 8)));
                            }
                            product(mt, a);
                        }
                    }
                }
            }
            __syncwarp();
            if (ok && lane == 0) ptx::mbar_arrive(bars + 8 * (STAGES + stage));
            advance();
        }

        // o and l without the offset (exactly); m stays what the exponentials were taken relative to
        if (CODES || OFFSET != 0.0f) {
            const float back = (CODES ? __uint_as_float(unit) : 1.0f) * offset_back(OFFSET);
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4 * NQ; ++e) o[i][e] *= back;
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    l[n][e] *= offset_back(OFFSET);
                    m[n][e] -= OFFSET;
                }
        }
        // ---- the four warps' results become one (every warp passes these barriers, whatever became of its waits) -------------
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], x);
        auto put = [&](float* to) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4 * NQ; ++e) to[(i * 4 * NQ + e) * 32 + lane] = o[i][e];
            if (g == 0) {
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        to[S::NREG * 32 + 8 * n + 2 * c + e] = m[n][e];
                        to[S::NREG * 32 + 8 * (NQ + n) + 2 * c + e] = l[n][e];
                    }
            }
        };
        auto join = [&](const float* from) {
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top, mine, theirs;
                    join_scales(m[n][e], from[S::NREG * 32 + 8 * n + 2 * c + e], top, mine, theirs);
                    m[n][e] = top;
                    l[n][e] = l[n][e] * mine + from[S::NREG * 32 + 8 * (NQ + n) + 2 * c + e] * theirs;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            float& x = o[i][4 * n + 2 * r + e];
                            x = x * mine + from[(i * 4 * NQ + 4 * n + 2 * r + e) * 32 + lane] * theirs;
                        }
                }
        };
        consumer_barrier();                                              // the last item's results have been read
        if (warp >= 2) put(merge + (warp - 2) * S::PART);
        consumer_barrier();
        if (warp < 2) join(merge + warp * S::PART);
        __syncwarp();                                                    // (what is overwritten has been read by the whole warp)
        if (warp == 1) put(merge + S::PART);
        consumer_barrier();
        if (warp == 0) {
            join(merge + S::PART);
            if (ok && w.whole()) {
                float inv[NQ][2];
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) inv[n][e] = l[n][e] > 0.0f ? 1.0f / l[n][e] : 0.0f;
#pragma unroll
                for (int mt = 0; mt < D / 16; ++mt) write_product<D, T, CODES, NQ>(P, w.s, w.h, w.p, mt, o[mt], inv);
                write_lse<NQ>(P, w.s, w.h, w.p, m, l, OFFSET);
            } else if (ok) {
                put(P.partial + (2ll * blockIdx.x + (w.tile > 0 ? 0 : 1)) * S::PART);
            }
        }
        w.next(P.plan);
    }
}

// Joins the partial results of an item that several CTAs worked on: the block of the second of them does it, a warp for every product.
template <int D, typename T, bool CODES, int NQ>
__global__ void __launch_bounds__(D * 2)
paged_rows_join_kernel(const __grid_constant__ RowsParams P) {
    using S = RowsShape<D, CODES, NQ>;
    grid_dependency_wait();
    grid_dependency_launch();
    const JoinNote note = P.notes[blockIdx.x + 1];
    if (note.last_cta < 0) return;
    const int mt = threadIdx.x >> 5, lane = threadIdx.x & 31, c = lane & 3;
    float o[4 * NQ], m[NQ][2], l[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) { m[n][e] = -INFINITY; l[n][e] = 0.0f; }
#pragma unroll
    for (int e = 0; e < 4 * NQ; ++e) o[e] = 0.0f;
    constexpr int DEEP = 8 / NQ;                                       // parts whose loads are under way at once
    for (int cta0 = note.first_cta; cta0 <= note.last_cta; cta0 += DEEP) {
        float v[DEEP][4 * NQ], pm[DEEP][NQ][2], pl[DEEP][NQ][2];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) {
            const int cta = cta0 + i;
            const bool there = cta <= note.last_cta;
            const float* const at = P.partial + (2ll * cta + (cta == note.first_cta ? 1 : 0)) * S::PART;
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    pm[i][n][e] = there ? at[S::NREG * 32 + 8 * n + 2 * c + e] : -INFINITY;
                    pl[i][n][e] = there ? at[S::NREG * 32 + 8 * (NQ + n) + 2 * c + e] : 0.0f;
                }
#pragma unroll
            for (int e = 0; e < 4 * NQ; ++e) v[i][e] = there ? at[(mt * 4 * NQ + e) * 32 + lane] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < DEEP; ++i)
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top, mine, theirs;
                    join_scales(m[n][e], pm[i][n][e], top, mine, theirs);
                    m[n][e] = top;
                    l[n][e] = l[n][e] * mine + pl[i][n][e] * theirs;
#pragma unroll
                    for (int r = 0; r < 2; ++r) o[4 * n + 2 * r + e] = o[4 * n + 2 * r + e] * mine + v[i][4 * n + 2 * r + e] * theirs;
                }
    }
    const Sequence s{note.length, note.first, note.queries};
    float inv[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) inv[n][e] = l[n][e] > 0.0f ? 1.0f / l[n][e] : 0.0f;
    write_product<D, T, CODES, NQ>(P, s, note.h, note.p, mt, o, inv);
    if (mt == 0) write_lse<NQ>(P, s, note.h, note.p, m, l, ROWS_OFFSET<T, CODES>);
}

inline int rows_grid(int nq) { return (nq == 1 ? 4 : 2) * sm_count(); }      // at most
inline size_t rows_partial_bytes(int nq, int head_dim) { return (size_t)rows_grid(nq) * 2 * (nq * head_dim * 8 + nq * 16) * 4; }

template <int D, typename T, bool CODES, int NQ>
int paged_rows_launch(RowsParams& P, const vitint_cache* cache, const vitint_cache_batch* batch, void* workspace, cudaStream_t st) {
    using S = RowsShape<D, CODES, NQ>;
    CUtensorMap map_k, map_v;
    P.page_rows = cache->page_tokens < S::KT ? cache->page_tokens : S::KT;
    const long long tiles = (batch->max_length + S::KT - 1) / S::KT;
    long long items;
    if (!plan_fits(cache, batch, most_runs(batch, P.plan.seq.tokens, P.plan.tile_tokens), tiles, items)) return VITINT_ERR_UNSUPPORTED;
    if (!encode_cache_map(&map_k, cache, cache->k, P.page_rows, true) || !encode_cache_map(&map_v, cache, cache->v, P.page_rows, true)) return VITINT_ERR_CUDA;
    int grid = S::CTAS * sm_count();
    P.plan.whole = whole_items(items, tiles, grid, NQ == 1 ? 3 : 1, 8);
    if (grid > items * tiles) grid = (int)(items * tiles);
    P.notes = (JoinNote*)workspace;
    P.partial = (float*)((uint8_t*)workspace + notes_bytes(rows_grid(NQ)));
    const int dev = current_device();
    if (dev < 0) return VITINT_ERR_CUDA;
    static bool attr_set_dev[MAX_DEVICES] = {};
    if (!attr_set_dev[dev]) {
        if (cudaFuncSetAttribute(paged_rows_kernel<D, T, CODES, NQ>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess) return VITINT_ERR_CUDA;
        attr_set_dev[dev] = true;
    }
    launch_kernel(paged_rows_kernel<D, T, CODES, NQ>, dim3(grid), dim3(PA_THREADS), S::SMEM, st, map_k, map_v, P);
    if (int rc = cuda_status(cudaGetLastError())) return rc;
    if (!P.plan.whole && grid > 1) launch_kernel(paged_rows_join_kernel<D, T, CODES, NQ>, dim3(grid - 1), dim3(D * 2), 0, st, P);
    return cuda_status(cudaGetLastError());
}

// Whether a head of the cache has at most as many rows as one warp-level product: the kernel of this file, else that of
// paged_attention_tiles.cu.
inline bool few_rows(int q_heads, const vitint_cache* cache, const vitint_cache_batch* batch) {
    return (int64_t)batch->max_queries * (q_heads / cache->kv_heads) <= PA_ROWS;
}
inline int row_products(int q_heads, const vitint_cache* cache, const vitint_cache_batch* batch) {
    return batch->max_queries * (q_heads / cache->kv_heads) <= 8 ? 1 : 2;
}

}  // namespace
}  // namespace vitint

using namespace vitint;

extern "C" size_t vitint_paged_attention_workspace_bytes(int32_t q_heads, const vitint_cache* cache, const vitint_cache_batch* batch) {
    if (check_cache(cache) != VITINT_OK || check_batch(cache, batch, true) != VITINT_OK || q_heads <= 0 || q_heads % cache->kv_heads != 0) return 0;
    if (few_rows(q_heads, cache, batch)) {
        const int nq = row_products(q_heads, cache, batch);
        return notes_bytes(rows_grid(nq)) + rows_partial_bytes(nq, cache->head_dim);
    }
    return notes_bytes(sm_count()) + tiles_partial_bytes(sm_count(), cache->head_dim);
}

extern "C" int vitint_paged_attention(const void* q, int32_t q_type, int64_t tokens, int32_t q_heads, int64_t q_token_stride,
                                      int64_t q_head_stride, const vitint_cache* cache, const vitint_cache_batch* batch, float scale,
                                      int32_t causal, int32_t window, void* out, int64_t out_token_stride, int64_t out_head_stride,
                                      float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = check_paged_queries(q, q_type, tokens, q_heads, q_token_stride, q_head_stride, cache, batch, scale, causal, window)) return rc;
    if (!out) return VITINT_ERR_INVALID_ARG;
    if (!aligned16(out) || !aligned_to(lse, 4) || out_token_stride % 8 != 0 || out_head_stride % 8 != 0) return VITINT_ERR_ALIGNMENT;
    if (out_token_stride <= 0 || out_head_stride < cache->head_dim) return VITINT_ERR_INVALID_ARG;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) ||
        workspace_bytes < vitint_paged_attention_workspace_bytes(q_heads, cache, batch))
        return VITINT_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)stream;
    const bool codes = cache->type == VITINT_I8, bf16 = q_type == VITINT_BF16;
    if (!few_rows(q_heads, cache, batch)) {
        TilesParams P{};
        P.plan = plan_params(cache, batch, tokens, q_heads, causal, window);
        P.half_tokens = 128 / P.plan.group;
        P.plan.tile_tokens = 2 * P.half_tokens;
        P.out = out; P.lse = lse;
        P.k_steps = cache->k_steps; P.v_steps = cache->v_steps;
        P.out_token = out_token_stride; P.out_head = out_head_stride;
        P.q_heads = q_heads;
        P.c = (float)((double)scale * 1.4426950408889634);
        auto go = [&](auto launch) { return launch(P, q, tokens, q_token_stride, q_head_stride, cache, batch, workspace, st); };
        if (cache->head_dim == 64) {
            if (codes) return bf16 ? go(paged_tiles_launch<64, __nv_bfloat16, true>) : go(paged_tiles_launch<64, __half, true>);
            return bf16 ? go(paged_tiles_launch<64, __nv_bfloat16, false>) : go(paged_tiles_launch<64, __half, false>);
        }
        if (codes) return bf16 ? go(paged_tiles_launch<128, __nv_bfloat16, true>) : go(paged_tiles_launch<128, __half, true>);
        return bf16 ? go(paged_tiles_launch<128, __nv_bfloat16, false>) : go(paged_tiles_launch<128, __half, false>);
    }
    RowsParams P{};
    P.plan = plan_params(cache, batch, tokens, q_heads, causal, window);
    P.plan.tile_tokens = PA_ROWS / P.plan.group;
    P.q = q; P.out = out; P.lse = lse;
    P.k_steps = cache->k_steps; P.v_steps = cache->v_steps;
    P.q_token = q_token_stride; P.q_head = q_head_stride; P.out_token = out_token_stride; P.out_head = out_head_stride;
    P.q_heads = q_heads;
    P.c = (float)((double)scale * 1.4426950408889634);
    auto go = [&](auto one, auto two) {
        return row_products(q_heads, cache, batch) == 1 ? one(P, cache, batch, workspace, st) : two(P, cache, batch, workspace, st);
    };
    if (cache->head_dim == 64) {
        if (codes)
            return bf16 ? go(paged_rows_launch<64, __nv_bfloat16, true, 1>, paged_rows_launch<64, __nv_bfloat16, true, 2>)
                        : go(paged_rows_launch<64, __half, true, 1>, paged_rows_launch<64, __half, true, 2>);
        return bf16 ? go(paged_rows_launch<64, __nv_bfloat16, false, 1>, paged_rows_launch<64, __nv_bfloat16, false, 2>)
                    : go(paged_rows_launch<64, __half, false, 1>, paged_rows_launch<64, __half, false, 2>);
    }
    if (codes)
        return bf16 ? go(paged_rows_launch<128, __nv_bfloat16, true, 1>, paged_rows_launch<128, __nv_bfloat16, true, 2>)
                    : go(paged_rows_launch<128, __half, true, 1>, paged_rows_launch<128, __half, true, 2>);
    return bf16 ? go(paged_rows_launch<128, __nv_bfloat16, false, 1>, paged_rows_launch<128, __nv_bfloat16, false, 2>)
                : go(paged_rows_launch<128, __half, false, 1>, paged_rows_launch<128, __half, false, 2>);
}
