// Attention of a few new tokens over the paged cache: at most sixteen rows (new tokens x query heads of a group) for a head of the cache.
//
//   s_rj = scale * step_j (q_r . k_j);  p = 2^(s log2 e - m);  o_r = sum_j (p_rj vstep_j) v_j / sum_j p_rj
//
// Bound by HBM: every key and value is read once for a handful of multiplications.  What the kernel has to do is to keep enough
// bytes in flight on every SM and share the keys out evenly (paged_plan.cuh).  A producer warp copies key tiles (their pages'
// pieces, one TMA copy a page for keys and one for values) into a ring of about 96 KB a CTA, two CTAs an SM; four warps take a
// quarter of each tile's keys, each with a running maximum, sum and output of its own, so that they meet only at an item's end.
// The contractions are warp-level m16n8k16 products: sixteen rows are all there are, and a 128-row tcgen05 tile would be empty at
// seven eighths.  8-bit codes become 16-bit operands in registers (integers up to 128 are exact in both types): the order of the
// contraction's index is free as long as both sides agree, so a thread takes its codes as they lie, sixteen bytes at a time.
#include "paged_tiles.cuh"
#include "paged_attention_tiles.cu"

namespace vitint {
namespace {

constexpr int PA_WARPS = 4;
constexpr int PA_THREADS = (PA_WARPS + 1) * 32;
constexpr int PA_ROWS = 16;

template <int D, bool CODES>
struct RowsShape {
    static constexpr int SIZE = CODES ? 1 : 2;                         // bytes of an element
    static constexpr int ROW = D * SIZE;                               // bytes of a key
    static constexpr int LINE = ROW < 128 ? ROW : 128, LINES = ROW / LINE;
    static constexpr int KT = ROW == 256 || (CODES && D == 128) ? 64 : 128;      // keys of a tile
    static constexpr int NK = KT / PA_WARPS;                           // a warp's keys of a tile
    static constexpr int HALF = KT * ROW;                              // bytes of a tile's keys (or values)
    static constexpr int STEPS = CODES ? KT * 4 : 0;                   // bytes of a tile's key (or value) steps
    static constexpr int STAGE = 2 * HALF;
    static constexpr int STAGES = STAGE == 32768 ? 3 : 5;
    static constexpr int PART = 16 * D + 32;                           // floats of a partial result: a warp's output fragments [D/2][32], maxima [16], sums [16]
    static constexpr int MERGE = 2 * PART * 4;
    static constexpr int SMEM = STAGES * (STAGE + 2 * STEPS) + MERGE + 256;
};

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
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
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

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void consumer_barrier() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// Joins two partial results of the same rows: (m, l, o) <- both.  A maximum of -inf stands for no key yet.
__device__ __forceinline__ void join_scales(float m, float other, float& top, float& mine, float& theirs) {
    top = fmaxf(m, other);
    const float base = top == -INFINITY ? 0.0f : top;
    mine = exp2_approx(m - base);
    theirs = exp2_approx(other - base);
}

// Writes a finished item's rows from their fragments.  o[4 j + 2 r + e]: row lane / 4 + 8 r of product j.
template <int D, typename T, bool CODES>
__device__ __forceinline__ void write_rows(const RowsParams& P, const Sequence& s, int h, int p, const float (&o)[D / 2], const float (&m)[2],
                                           const float (&l)[2]) {
    const int lane = threadIdx.x & 31, c = lane & 3;
    const int tokens = min(P.plan.tile_tokens, s.queries - p * P.plan.tile_tokens), rows = tokens * P.plan.group;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = (lane >> 2) + 8 * r;
        if (row >= rows) continue;
        const int i = row / P.plan.group, head = h * P.plan.group + row - i * P.plan.group;
        const long long token = s.first + p * P.plan.tile_tokens + i;
        const float inv = l[r] > 0.0f ? 1.0f / l[r] : 0.0f;
        T* const to = (T*)P.out + token * P.out_token + head * P.out_head;
        if (CODES) {                                                    // columns 2c * (D/8) + j and (2c + 1) * (D/8) + j
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int j = 0; j < D / 8; j += 8) {
                    uint32_t w[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) w[k] = pack16<T>(o[4 * (j + 2 * k) + 2 * r + e] * inv, o[4 * (j + 2 * k + 1) + 2 * r + e] * inv);
                    *reinterpret_cast<uint4*>(to + (2 * c + e) * (D / 8) + j) = make_uint4(w[0], w[1], w[2], w[3]);
                }
        } else {                                                        // columns 8 j + 2c, 8 j + 2c + 1
#pragma unroll
            for (int j = 0; j < D / 8; ++j)
                *reinterpret_cast<uint32_t*>(to + 8 * j + 2 * c) = pack16<T>(o[4 * j + 2 * r] * inv, o[4 * j + 2 * r + 1] * inv);
        }
        if (P.lse && c == 0) P.lse[token * P.q_heads + head] = l[r] > 0.0f ? (m[r] + log2f(l[r])) * 0.69314718055994531f : -INFINITY;
    }
}

template <int D, typename T, bool CODES>
__global__ void __launch_bounds__(PA_THREADS, 2)
paged_rows_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ RowsParams P) {
    using S = RowsShape<D, CODES>;
    constexpr int KT = S::KT, NK = S::NK, STAGES = S::STAGES, NT = NK / 8;
    // Probabilities times steps enter the second contraction in the queries' type.  In fp16 they would run out of exponents, so they are
    // taken relative to the largest step so far (its power of two).
    constexpr bool SCALED = CODES && std::is_same<T, __half>::value;
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
        const Stretch r = plan_stretch<QueryRuns<KT>>(P.plan, blockIdx.x, gridDim.x, bad);
        if (lane == 0) {
            *shared_stretch = r;
            P.notes[blockIdx.x] = join_note(r, blockIdx.x);
            if (bad && blockIdx.x == 0) report_bad_data();
        }
    }
    __syncthreads();
    StretchWalk<QueryRuns<KT>> w;
    w.begin(P.plan, *shared_stretch);
    bool ok = true;
    int stage = 0;
    uint32_t phase = 0;
    auto advance = [&] {
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
    };

    if (warp == PA_WARPS) {
        // ---- producer: lane r copies the tile's r-th run of page rows ----------------------------------------------------
        const int copies = KT / P.page_rows, copy_bytes = P.page_rows * S::ROW;
        const int page_mask = (1 << P.plan.seq.page_shift) - 1;
        int issued = 0;
        for (; ok && w.more(); w.next(P.plan)) {
            for (int t = w.tile; t < w.end; ++t) {
                const int key = w.first + t * KT + lane * P.page_rows;
                const bool mine = lane < copies && key < w.s.length;
                const int page = mine ? page_of(P.plan.seq, w.b, key) : 0;
                const bool inside = mine && page < P.plan.seq.pages;
                const uint32_t n = __popc(__ballot_sync(0xffffffffu, mine)), n_steps = __popc(__ballot_sync(0xffffffffu, inside));
                ok = mbar_wait_warp(bars + 8 * (STAGES + stage), phase ^ 1u, abort_flag);
                if (!ok) break;
                const uint32_t full = bars + 8 * stage;
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
    const float sc = P.c;
    while (w.more()) {
        const int i0 = w.p * P.plan.tile_tokens, tokens = min(P.plan.tile_tokens, w.s.queries - i0), rows = tokens * P.plan.group;
        const int base = w.s.length - w.s.queries + i0;                  // position of the item's first token
        // queries as the left operand: rows g and g + 8
        uint32_t qa[D / 16][4];
        int low[2], high[2];                                             // the keys that the two rows see
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int row = g + 8 * r, i = row / P.plan.group;
            const bool live = row < rows;
            const T* const from = (const T*)P.q + (long long)(w.s.first + i0 + i) * P.q_token + (long long)(w.h * P.plan.group + row - i * P.plan.group) * P.q_head;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                if (CODES) {                                             // channels as the codes lie: 16 (c + 4 (k / 4)) + 4 (k % 4) + 0 .. 3
                    const uint2 v = live ? *reinterpret_cast<const uint2*>(from + 16 * (c + 4 * (k >> 2)) + 4 * (k & 3)) : make_uint2(0u, 0u);
                    qa[k][r] = v.x;
                    qa[k][2 + r] = v.y;
                } else {
                    qa[k][r] = live ? *reinterpret_cast<const uint32_t*>(from + 16 * k + 2 * c) : 0u;
                    qa[k][2 + r] = live ? *reinterpret_cast<const uint32_t*>(from + 16 * k + 8 + 2 * c) : 0u;
                }
            }
            high[r] = !live ? 0 : P.plan.causal ? min(base + i + 1, w.s.length) : w.s.length;
            low[r] = P.plan.window ? base + i - P.plan.window + 1 : 0;
        }
        const int all_low = P.plan.window ? base + tokens - P.plan.window : 0;                               // the last row's
        const int all_high = P.plan.causal ? min(base + 1, w.s.length) : w.s.length;                         // the first row's
        float o[D / 2], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
        uint32_t unit = 0x00800000u;                                     // SCALED: the power of two that o is a multiple of
#pragma unroll
        for (int i = 0; i < D / 2; ++i) o[i] = 0.0f;

        for (int t = w.tile; t < w.end; ++t) {
            ok = ok && mbar_wait_warp(bars + 8 * stage, phase, abort_flag);
            if (ok) {
                const uint32_t kbase = smem + stage * S::STAGE;
                const int key0 = w.first + t * KT + warp * NK;
                const bool edge = key0 < all_low || key0 + NK > all_high;
                float s[NT][4];
#pragma unroll
                for (int u = 0; u < NK / 16; ++u) {                      // sixteen keys, in one page
                    const int j = warp * NK + 16 * u, block = j >> rows_shift, in_block = j & (P.page_rows - 1);
                    const uint32_t at = kbase + block * (P.page_rows * S::ROW);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[2 * u][e] = s[2 * u + 1][e] = 0.0f;
                    if (!CODES) {
                        const int row = in_block + (lane >> 4) * 8 + (lane & 7), odd = (lane >> 3) & 1;
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const int chunk = 2 * k + odd;
                            uint32_t b[4];
                            ldmatrix4(at + (chunk >> 3) * (P.page_rows * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4), b);
                            mma16816<T>(s[2 * u], qa[k], b[0], b[1]);
                            mma16816<T>(s[2 * u + 1], qa[k], b[2], b[3]);
                        }
                    } else {
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const int row = in_block + 8 * half + g;
#pragma unroll
                            for (int x = 0; x < D / 64; ++x) {
                                const uint32_t chunk = c + 4 * x;
                                const uint4 v = lds128(at + row * S::LINE + ((S::LINE == 128 ? chunk ^ (row & 7) : chunk ^ ((row >> 1) & 3)) << 4));
                                const uint32_t words[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    mma16816<T>(s[2 * u + half], qa[4 * x + k], codes_to_16<T>(__byte_perm(words[k], 0u, 0x4140)),
                                                codes_to_16<T>(__byte_perm(words[k], 0u, 0x4342)));
                            }
                        }
                    }
                }
                // scores in units of log2, hidden ones -inf, and the rows' maxima
                const float* const ks = reinterpret_cast<const float*>(pa_smem + STAGES * S::STAGE + stage * 2 * S::STEPS) + warp * NK;
                const float* const vs = ks + KT;
                float top[2] = {m[0], m[1]};
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float2 f = make_float2(sc, sc);
                    if (CODES) {
                        f = *reinterpret_cast<const float2*>(ks + 8 * n + 2 * c);
                        f.x *= sc;
                        f.y *= sc;
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[n][e] *= (e & 1) ? f.y : f.x;
                        if (edge) {
                            const int key = key0 + 8 * n + 2 * c + (e & 1);
                            if (key < low[e >> 1] || key >= high[e >> 1]) s[n][e] = -INFINITY;
                        }
                        top[e >> 1] = fmaxf(top[e >> 1], s[n][e]);
                    }
                }
                float factor[2], from[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
                    top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
                    from[r] = top[r] == -INFINITY ? 0.0f : top[r];
                    factor[r] = exp2_approx(m[r] - from[r]);
                }
                if (__any_sync(0xffffffffu, top[0] != m[0] || top[1] != m[1])) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) { l[r] *= factor[r]; m[r] = top[r]; }
#pragma unroll
                    for (int i = 0; i < D / 2; ++i) o[i] *= factor[(i >> 1) & 1];
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[n][e] = exp2_approx(s[n][e] - from[e >> 1]);
                        l[e >> 1] += s[n][e];
                    }
                if (SCALED) {
                    uint32_t largest = unit;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const uint2 f = *reinterpret_cast<const uint2*>(vs + 8 * n + 2 * c);
                        const int key = key0 + 8 * n + 2 * c;
                        if (!edge || key < w.s.length) largest = max(largest, f.x & 0x7F800000u);
                        if (!edge || key + 1 < w.s.length) largest = max(largest, f.y & 0x7F800000u);
                    }
                    largest = min(__reduce_max_sync(0xffffffffu, largest), 0x7E000000u);
                    if (largest != unit) {
                        const float down = __uint_as_float(0x3F800000u - min(largest - unit, 0x3F000000u));
#pragma unroll
                        for (int i = 0; i < D / 2; ++i) o[i] *= down;
                        unit = largest;
                    }
                }
                // outputs: the probabilities of sixteen keys are the left operand as they are
#pragma unroll
                for (int u = 0; u < NK / 16; ++u) {
                    const int j = warp * NK + 16 * u, block = j >> rows_shift, in_block = j & (P.page_rows - 1);
                    const uint32_t at = kbase + S::HALF + block * (P.page_rows * S::ROW);
                    if (CODES) {
#pragma unroll
                        for (int n = 2 * u; n < 2 * u + 2; ++n) {
                            float2 f = *reinterpret_cast<const float2*>(vs + 8 * n + 2 * c);
                            if (edge) {                                  // (places behind the length: whatever lies there)
                                const int key = key0 + 8 * n + 2 * c;
                                if (key >= w.s.length) f.x = 0.0f;
                                if (key + 1 >= w.s.length) f.y = 0.0f;
                            }
                            if (SCALED) {
                                const float up = __uint_as_float(0x7F000000u - unit);      // 1 / unit
                                f.x *= up;
                                f.y *= up;
                            }
                            s[n][0] *= f.x; s[n][1] *= f.y; s[n][2] *= f.x; s[n][3] *= f.y;
                        }
                    }
                    uint32_t pa[4];
                    pa[0] = pack16<T>(s[2 * u][0], s[2 * u][1]);
                    pa[1] = pack16<T>(s[2 * u][2], s[2 * u][3]);
                    pa[2] = pack16<T>(s[2 * u + 1][0], s[2 * u + 1][1]);
                    pa[3] = pack16<T>(s[2 * u + 1][2], s[2 * u + 1][3]);
                    if (!CODES) {
                        uint32_t mask0 = 0xFFFFFFFFu, mask1 = 0xFFFFFFFFu;     // values behind the length are not multiplied: NaN times 0
                        if (edge) {
                            const int key = key0 + 16 * u + 2 * c;
                            mask0 = (key < w.s.length ? 0xFFFFu : 0u) | (key + 1 < w.s.length ? 0xFFFF0000u : 0u);
                            mask1 = (key + 8 < w.s.length ? 0xFFFFu : 0u) | (key + 9 < w.s.length ? 0xFFFF0000u : 0u);
                        }
                        const int row = in_block + ((lane >> 3) & 1) * 8 + (lane & 7), odd = lane >> 4;
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const int chunk = 2 * k + odd;
                            uint32_t b[4];
                            ldmatrix4_trans(at + (chunk >> 3) * (P.page_rows * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4), b);
                            if (edge) { b[0] &= mask0; b[1] &= mask1; b[2] &= mask0; b[3] &= mask1; }
                            mma16816<T>(*reinterpret_cast<float(*)[4]>(&o[8 * k]), pa, b[0], b[1]);
                            mma16816<T>(*reinterpret_cast<float(*)[4]>(&o[8 * k + 4]), pa, b[2], b[3]);
                        }
                    } else {
                        // a thread's columns: D/8 codes of its four keys, which are the right operand of D/8 products
                        uint32_t words[4][D / 32];
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int row = in_block + 2 * c + (x & 1) + 8 * (x >> 1);
                            if (D == 128) {
                                const uint4 v = lds128(at + row * 128 + ((g ^ (row & 7)) << 4));
                                words[x][0] = v.x; words[x][1] = v.y; words[x][D / 32 - 2] = v.z; words[x][D / 32 - 1] = v.w;
                            } else {
                                const uint2 v = lds64(at + row * 64 + ((((uint32_t)g >> 1) ^ ((row >> 1) & 3)) << 4) + (g & 1) * 8);
                                words[x][0] = v.x; words[x][1] = v.y;
                            }
                        }
#pragma unroll
                        for (int n = 0; n < D / 8; ++n) {
                            const uint32_t pick = (n & 3) | ((4 + (n & 3)) << 8);               // byte n % 4 of both words
                            const uint32_t b0 = codes_to_16<T>(__byte_perm(words[0][n >> 2], words[1][n >> 2], pick));
                            const uint32_t b1 = codes_to_16<T>(__byte_perm(words[2][n >> 2], words[3][n >> 2], pick));
                            mma16816<T>(*reinterpret_cast<float(*)[4]>(&o[4 * n]), pa, b0, b1);
                        }
                    }
                }
            }
            __syncwarp();
            if (ok && lane == 0) ptx::mbar_arrive(bars + 8 * (STAGES + stage));
            advance();
        }

        if (SCALED) {
#pragma unroll
            for (int i = 0; i < D / 2; ++i) o[i] *= __uint_as_float(unit);
        }
        // ---- the four warps' results become one (every warp passes these barriers, whatever became of its waits) -------------
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
        }
        auto put = [&](float* to) {
#pragma unroll
            for (int i = 0; i < D / 2; ++i) to[i * 32 + lane] = o[i];
#pragma unroll
            for (int r = 0; r < 2; ++r)
                if (c == 0) { to[16 * D + 8 * r + g] = m[r]; to[16 * D + 16 + 8 * r + g] = l[r]; }
        };
        auto join = [&](const float* from) {
            float mine[2], theirs[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float top;
                join_scales(m[r], from[16 * D + 8 * r + g], top, mine[r], theirs[r]);
                m[r] = top;
                l[r] = l[r] * mine[r] + from[16 * D + 16 + 8 * r + g] * theirs[r];
            }
#pragma unroll
            for (int i = 0; i < D / 2; ++i) o[i] = o[i] * mine[(i >> 1) & 1] + from[i * 32 + lane] * theirs[(i >> 1) & 1];
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
            if (ok) {
                if (w.whole()) write_rows<D, T, CODES>(P, w.s, w.h, w.p, o, m, l);
                else put(P.partial + (2ll * blockIdx.x + (w.tile > 0 ? 0 : 1)) * S::PART);
            }
        }
        w.next(P.plan);
    }
}

// Joins the partial results of an item that several CTAs worked on: the block of the second of them does it.  Eight warps
// take an eighth of the outputs each.
template <int D, typename T, bool CODES>
__global__ void __launch_bounds__(256)
paged_rows_join_kernel(const __grid_constant__ RowsParams P) {
    using S = RowsShape<D, CODES>;
    constexpr int SHARE = D / 16;
    grid_dependency_wait();
    grid_dependency_launch();
    const JoinNote n = P.notes[blockIdx.x + 1];
    if (n.last_cta < 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2;
    float o[SHARE], m[2], l[2];
    const float* at = P.partial + (2ll * n.first_cta + 1) * S::PART ;
#pragma unroll
    for (int i = 0; i < SHARE; ++i) o[i] = at[(warp * SHARE + i) * 32 + lane];
#pragma unroll
    for (int r = 0; r < 2; ++r) { m[r] = at[16 * D + 8 * r + g]; l[r] = at[16 * D + 16 + 8 * r + g]; }
#pragma unroll 4
    for (int cta = n.first_cta + 1; cta <= n.last_cta; ++cta) {
        at = P.partial + 2ll * cta * S::PART ;
        float mine[2], theirs[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float top;
            join_scales(m[r], at[16 * D + 8 * r + g], top, mine[r], theirs[r]);
            m[r] = top;
            l[r] = l[r] * mine[r] + at[16 * D + 16 + 8 * r + g] * theirs[r];
        }
#pragma unroll
        for (int i = 0; i < SHARE; ++i) o[i] = o[i] * mine[(i >> 1) & 1] + at[(warp * SHARE + i) * 32 + lane] * theirs[(i >> 1) & 1];
    }
    const Sequence s = sequence_of(P.plan.seq, n.b);
    const int c = lane & 3, i0 = n.p * P.plan.tile_tokens, rows = min(P.plan.tile_tokens, s.queries - i0) * P.plan.group;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = g + 8 * r;
        if (row >= rows) continue;
        const int i = row / P.plan.group, head = n.h * P.plan.group + row - i * P.plan.group;
        const long long token = s.first + i0 + i;
        const float inv = l[r] > 0.0f ? 1.0f / l[r] : 0.0f;
        T* const to = (T*)P.out + token * P.out_token + head * P.out_head;
#pragma unroll
        for (int k = 0; k < SHARE / 4; ++k) {                             // product j: columns as in write_rows
            const int j = warp * (SHARE / 4) + k;
            const float a = o[4 * k + 2 * r] * inv, b = o[4 * k + 2 * r + 1] * inv;
            if (CODES) {
                const uint32_t w = pack16<T>(a, b);
                reinterpret_cast<uint16_t*>(to)[2 * c * (D / 8) + j] = (uint16_t)w;
                reinterpret_cast<uint16_t*>(to)[(2 * c + 1) * (D / 8) + j] = (uint16_t)(w >> 16);
            } else {
                *reinterpret_cast<uint32_t*>(to + 8 * j + 2 * c) = pack16<T>(a, b);
            }
        }
        if (P.lse && c == 0 && warp == 0) P.lse[token * P.q_heads + head] = l[r] > 0.0f ? (m[r] + log2f(l[r])) * 0.69314718055994531f : -INFINITY;
    }
}

inline int rows_grid() { return 2 * sm_count(); }
inline size_t rows_partial_bytes(int ctas, int head_dim) { return (size_t)ctas * 2 * (16 * head_dim + 32) * 4; }

template <int D, typename T, bool CODES>
int paged_rows_launch(RowsParams& P, const vitint_cache* cache, const vitint_cache_batch* batch, void* workspace, cudaStream_t st) {
    using S = RowsShape<D, CODES>;
    CUtensorMap map_k, map_v;
    P.page_rows = cache->page_tokens < S::KT ? cache->page_tokens : S::KT;
    if (!encode_cache_map(&map_k, cache, cache->k, P.page_rows, true) || !encode_cache_map(&map_v, cache, cache->v, P.page_rows, true)) return VITINT_ERR_CUDA;
    const long long runs = (batch->max_queries + P.plan.tile_tokens - 1) / P.plan.tile_tokens, tiles = (batch->max_length + S::KT - 1) / S::KT;
    const long long items = (long long)batch->sequences * cache->kv_heads * runs;
    if (items > 0x7fffffffll || items * tiles > 0x7fffffffll) return VITINT_ERR_UNSUPPORTED;
    int grid = rows_grid();
    if (grid > items * tiles) grid = (int)(items * tiles);
    P.notes = (JoinNote*)workspace;
    P.partial = (float*)((uint8_t*)workspace + notes_bytes(rows_grid()));
    const int dev = current_device();
    if (dev < 0) return VITINT_ERR_CUDA;
    static bool attr_set_dev[MAX_DEVICES] = {};
    if (!attr_set_dev[dev]) {
        if (cudaFuncSetAttribute(paged_rows_kernel<D, T, CODES>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess) return VITINT_ERR_CUDA;
        attr_set_dev[dev] = true;
    }
    launch_kernel(paged_rows_kernel<D, T, CODES>, dim3(grid), dim3(PA_THREADS), S::SMEM, st, map_k, map_v, P);
    if (int rc = cuda_status(cudaGetLastError())) return rc;
    if (tiles > 1 && grid > 1) launch_kernel(paged_rows_join_kernel<D, T, CODES>, dim3(grid - 1), dim3(256), 0, st, P);
    return cuda_status(cudaGetLastError());
}

// Whether a head of the cache has at most as many rows as one warp-level product: the kernel of this file, else that of
// paged_attention_tiles.cu.
inline bool few_rows(int q_heads, const vitint_cache* cache, const vitint_cache_batch* batch) {
    return (int64_t)batch->max_queries * (q_heads / cache->kv_heads) <= PA_ROWS;
}

}  // namespace
}  // namespace vitint

using namespace vitint;

extern "C" size_t vitint_paged_attention_workspace_bytes(int32_t q_heads, const vitint_cache* cache, const vitint_cache_batch* batch) {
    if (check_cache(cache) != VITINT_OK || check_batch(cache, batch, true) != VITINT_OK || q_heads <= 0 || q_heads % cache->kv_heads != 0) return 0;
    if (few_rows(q_heads, cache, batch)) return notes_bytes(rows_grid()) + rows_partial_bytes(rows_grid(), cache->head_dim);
    return notes_bytes(sm_count()) + tiles_partial_bytes(sm_count(), cache->head_dim);
}

extern "C" int vitint_paged_attention(const void* q, int32_t q_type, int64_t tokens, int32_t q_heads, int64_t q_token_stride,
                                      int64_t q_head_stride, const vitint_cache* cache, const vitint_cache_batch* batch, float scale,
                                      int32_t causal, int32_t window, void* out, int64_t out_token_stride, int64_t out_head_stride,
                                      float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = check_paged_queries(q, q_type, tokens, q_heads, q_token_stride, q_head_stride, cache, batch, scale, causal, window)) return rc;
    if (!out) return VITINT_ERR_INVALID_ARG;
    if (!aligned16(out) || out_token_stride % 8 != 0 || out_head_stride % 8 != 0) return VITINT_ERR_ALIGNMENT;
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
    auto go = [&](auto launch) { return launch(P, cache, batch, workspace, st); };
    if (cache->head_dim == 64) {
        if (codes) return bf16 ? go(paged_rows_launch<64, __nv_bfloat16, true>) : go(paged_rows_launch<64, __half, true>);
        return bf16 ? go(paged_rows_launch<64, __nv_bfloat16, false>) : go(paged_rows_launch<64, __half, false>);
    }
    if (codes) return bf16 ? go(paged_rows_launch<128, __nv_bfloat16, true>) : go(paged_rows_launch<128, __half, true>);
    return bf16 ? go(paged_rows_launch<128, __nv_bfloat16, false>) : go(paged_rows_launch<128, __half, false>);
}
