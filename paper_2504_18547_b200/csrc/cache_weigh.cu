// The attention weight that cached tokens receive:  w_j += sum over new tokens i and heads of the group  2^(s_ij log2 e - lse_i log2 e).
//
// With keys as the rows of the product S^T = K Q^T (tcgen05, 128 keys x up to 128 query rows) a thread has a key: it sums over the columns that
// tensor memory gives it, and nothing crosses threads.  The rows' logarithms of sums come from the attention call, so one pass does.
//
// For prompts it is bound by shared memory: the product of 128 x 128 scores reads 64 KB of operands, which is what shared memory delivers in its
// 512 cycles, and every thread loads the rows' logarithms beside it (1023 tokens x 32 heads over 12,287 cached codes: 151 us, 660 TFLOP/s; without
// these loads 121, with a quarter of the products 140; loading them once for two keys of a thread costs registers: 167).  The exponentials, 16 a clock
// and SM, take 1024 cycles of the special-function unit; a part of them goes through the FMA pipe (all through the unit: 164 us).  Over 16-bit keys the same takes 134 us.  For single
// tokens it is bound by reading the keys and by a tile's latency (32 sequences of up to 4096 tokens: 27 us for 18 of bytes; over codes 38).  Two tiles of keys stay in shared memory while the query tiles that see them stream past (one would have 32 KB
// of queries come from L2 for every 128 x 128 scores); a group of four warps has the scores of one of them, in two buffers each.  Work is shared out
// evenly as for the attention (paged_plan.cuh), with keys and queries in each other's places; a run of keys whose queries are split between CTAs is
// summed by a second kernel in the CTAs' order.
#include "paged_tiles.cuh"

namespace vitint {
namespace {

constexpr int CW_KEYS = 256, CW_HALF = 128;                              // keys of an item, of a tile
constexpr int CW_MAX_STAGES = 4;
constexpr int CW_TMA = 8, CW_MMA = 9, CW_EXPAND = 10;                  // warps behind the two groups of four

struct WeighParams {
    PlanParams plan;
    const float* lse;
    const float* in;
    float* out;
    const float* k_steps;
    float c;                                                           // scale * log2(e)
    int q_heads, page_rows, box_rows, n_pad;                           // rows of a query copy, columns of a product
    int q_stages, k_stages, raw_stages;
    uint32_t q_slot, off_q, off_k, off_raw;
    float* partial;
    JoinNote* notes;
};

struct WeighBars {
    uint64_t q_full[CW_MAX_STAGES], q_empty[CW_MAX_STAGES], k_full[CW_MAX_STAGES], k_empty[CW_MAX_STAGES], raw_full[CW_MAX_STAGES],
        raw_empty[CW_MAX_STAGES], s_full[2][2], s_empty[2][2], drained;          // scores: [half][buffer]
};

// Position in a ring and the phase of its barriers.
struct Ring {
    int at = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void step(int n) {
        if (++at == n) { at = 0; phase ^= 1u; }
    }
};

// Sum over 32 columns of 2^(s c - l); hidden columns (outside [low, high)) count 0.  Where none is hidden, six of sixteen pairs go through the
// polynomial: special-function unit and FMA pipe then take five cycles each for a warp's column instead of eight and two.
template <bool MASKED>
__device__ __forceinline__ void weigh_block(const uint32_t (&v)[32], const float* minus_l, f32x2 c2, int low, int high, f32x2 (&acc)[2]) {
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
        const float4 l = *reinterpret_cast<const float4*>(minus_l + i);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const f32x2 x = f2_fma(f2_pack(__uint_as_float(v[i + 2 * k]), __uint_as_float(v[i + 2 * k + 1])), c2, k ? f2_pack(l.z, l.w) : f2_pack(l.x, l.y));
            float a, b;
            f2_unpack(x, a, b);
            if (MASKED) {
                a = i + 2 * k >= low && i + 2 * k < high ? a : -INFINITY;
                b = i + 2 * k + 1 >= low && i + 2 * k + 1 < high ? b : -INFINITY;
            }
            if (!MASKED && k == 1 && i % 16 != 12) {
                exp2_poly(f2_pack(max_or_nan(a, -127.0f), max_or_nan(b, -127.0f)), a, b);
            } else {
                a = exp2_approx(a);
                b = exp2_approx(b);
            }
            acc[k] = f2_add(acc[k], f2_pack(a, b));
        }
    }
}

// FEW: at most 32 query rows, so that several CTAs fit an SM: single tokens are bound by the latency of what a CTA does for a tile of keys.
template <int D, typename T, bool CODES, bool FEW>
__global__ void __launch_bounds__((CODES ? 14 : 10) * 32, FEW ? (CODES ? 2 : 3) : 1)
cache_weigh_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ WeighParams P) {
    using Runs = KeyRuns<CW_KEYS>;
    constexpr int LINES = D / 64;
    constexpr uint32_t K_SLOT = LINES * 16384, RAW_SLOT = CW_HALF * D;
    constexpr uint32_t COLS = FEW ? 32 : 128, TMEM_COLS = 4 * COLS;    // of a score tile, of all
    extern __shared__ __align__(1024) uint8_t cw_smem[];
    __shared__ WeighBars B;
    __shared__ __align__(16) float minus_lse[2][2][COLS];              // [half][buffer]: -lse log2 e of the tile's rows, read four at a time
    __shared__ Stretch shared_stretch;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    volatile int* const abort_ptr = &abort_flag;
    const uint32_t smem = (ptx::smem_addr(cw_smem) + 1023u) & ~1023u;
    uint8_t* const gen = cw_smem + (smem - ptx::smem_addr(cw_smem));
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int i = 0; i < CW_MAX_STAGES; ++i) {
            ptx::mbar_init(ptx::smem_addr(&B.q_full[i]), 1);
            ptx::mbar_init(ptx::smem_addr(&B.q_empty[i]), 1);
            ptx::mbar_init(ptx::smem_addr(&B.k_full[i]), CODES ? 4 : 1);
            ptx::mbar_init(ptx::smem_addr(&B.k_empty[i]), 1);
            ptx::mbar_init(ptx::smem_addr(&B.raw_full[i]), 1);
            ptx::mbar_init(ptx::smem_addr(&B.raw_empty[i]), 4);
            ptx::mbar_init(ptx::smem_addr(&B.s_full[i >> 1][i & 1]), 1);
            ptx::mbar_init(ptx::smem_addr(&B.s_empty[i >> 1][i & 1]), 4);
        }
        ptx::mbar_init(ptx::smem_addr(&B.drained), 1);
        ptx::fence_mbar_init();
        ptx::fence_proxy_async_smem();
    }
    if (warp == CW_MMA) {
        ptx::tmem_alloc(ptx::smem_addr(&tmem_slot), TMEM_COLS);
        ptx::tmem_relinquish();
    }
    if (warp == CW_TMA && lane == 0) { ptx::prefetch_tensormap(&map_q); ptx::prefetch_tensormap(&map_k); }
    grid_dependency_wait();
    grid_dependency_launch();
    if (warp == 0) {
        bool bad = false;
        const Stretch r = plan_stretch<Runs>(P.plan, blockIdx.x, gridDim.x, bad);
        if (lane == 0) {
            shared_stretch = r;
            if (bad && blockIdx.x == 0) report_bad_data();
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    StretchWalk<Runs> w;
    // (by a thread that waits for its first tile anyway)
    if (threadIdx.x == 32) P.notes[blockIdx.x] = join_note(P.plan, shared_stretch, blockIdx.x);
    w.begin(P.plan, shared_stretch);
    bool ok = true;
    auto halves = [](const StretchWalk<Runs>& at) { return at.s.length - at.p * CW_KEYS > CW_HALF ? 2 : 1; };

    if (warp == CW_TMA) {
        Ring q, k;
        int q_issued = 0, k_issued = 0;
        const int copies = CW_HALF / P.page_rows, page_mask = (1 << P.plan.seq.page_shift) - 1;
        uint64_t *const k_full = CODES ? B.raw_full : B.k_full, *const k_empty = CODES ? B.raw_empty : B.k_empty;
        const int k_ring = CODES ? P.raw_stages : P.k_stages;
        const uint32_t k_base = smem + (CODES ? P.off_raw : P.off_k), k_slot = CODES ? RAW_SLOT : K_SLOT;
        // lane r looks up the item's r-th run of page rows, an item ahead
        auto key_at = [&](const StretchWalk<Runs>& at) { return at.p * CW_KEYS + lane * P.page_rows; };
        auto copied = [&](const StretchWalk<Runs>& at) { return at.more() && lane < 2 * copies && key_at(at) < at.s.length; };
        StretchWalk<Runs> next = w;
        int entry = copied(w) ? page_entry(P.plan.seq, w.b, key_at(w)) : 0;
        for (; ok && w.more(); w = next) {
            const int page = copied(w) ? checked_page(P.plan.seq, entry) : -1;
            next.next(P.plan);
            if (copied(next)) entry = page_entry(P.plan.seq, next.b, key_at(next));
            for (int x = 0; x < halves(w); ++x) {
                const bool mine = page >= 0 && lane / copies == x;
                const uint32_t n = __popc(__ballot_sync(0xffffffffu, mine));
                ok = mbar_wait_warp(ptx::smem_addr(&k_empty[k.at]), k.phase ^ 1u, abort_ptr);
                if (!ok) break;
                const uint32_t full = ptx::smem_addr(&k_full[k.at]), to = k_base + k.at * k_slot;
                if (lane == 0) ptx::mbar_arrive_expect_tx(full, n * P.page_rows * (CODES ? D : 2 * D));
                __syncwarp();
                if (mine) {
                    const int r = lane - x * copies, place = (w.p * CW_KEYS + lane * P.page_rows) & page_mask;
                    if (CODES) {
                        ptx::tma_load_5d(to + r * P.page_rows * D, &map_k, full, 0, place, 0, w.h, page);
                    } else {
                        for (int i = 0; i < LINES; ++i) ptx::tma_load_5d(to + i * 16384 + r * P.page_rows * 128, &map_k, full, 0, place, i, w.h, page);
                    }
                }
                __syncwarp();
                ++k_issued;
                k.step(k_ring);
            }
            for (int t = w.tile; ok && t < w.end; ++t) {
                ok = mbar_wait_warp(ptx::smem_addr(&B.q_empty[q.at]), q.phase ^ 1u, abort_ptr);
                if (!ok) break;
                if (ptx::elect_one()) {
                    const uint32_t bar = ptx::smem_addr(&B.q_full[q.at]), at = smem + P.off_q + q.at * P.q_slot;
                    ptx::mbar_arrive_expect_tx(bar, LINES * P.box_rows * 128);
                    for (int i = 0; i < LINES; ++i)
                        ptx::tma_load_4d(at + i * (P.q_slot / LINES), &map_q, bar, 0, w.h * P.plan.group, w.s.first + (w.first + t) * P.plan.tile_tokens, i);
                }
                __syncwarp();
                ++q_issued;
                q.step(P.q_stages);
            }
        }
        if (!ok) {                                                     // copies in flight are given a bounded chance to land
            auto drain = [&](uint64_t* bars, Ring r, int ring, int issued) {
                for (int i = 0; i < ring && i < issued; ++i) {
                    if (r.at == 0) { r.at = ring; r.phase ^= 1u; }
                    --r.at;
                    for (int spin = 0; spin < (1 << 16) && !ptx::mbar_try_wait(ptx::smem_addr(&bars[r.at]), r.phase); ++spin) {}
                }
            };
            drain(k_full, k, k_ring, k_issued);
            drain(B.q_full, q, P.q_stages, q_issued);
        }
    } else if (warp == CW_MMA) {
        Ring q, k;
        uint32_t n_s[2] = {0, 0};                                      // products of each half: buffer and phase
        const uint32_t idesc = ptx::idesc_f16(CW_HALF, P.n_pad, std::is_same<T, __nv_bfloat16>::value, 0);
        const uint32_t q_line = P.q_slot / LINES;
        for (; ok && w.more(); w.next(P.plan)) {
            const int nh = halves(w);
            Ring slot[2] = {k, k};
            slot[1].step(P.k_stages);
            for (int t = w.tile; ok && t < w.end; ++t) {
                ok = mbar_wait_warp(ptx::smem_addr(&B.q_full[q.at]), q.phase, abort_ptr);
                if (!ok) break;
                const uint64_t b = ptx::smem_desc(smem + P.off_q + q.at * P.q_slot, 16, 1024, ptx::SWIZZLE_128B);
                for (int x = 0; x < nh; ++x) {
                    const uint32_t buffer = n_s[x] & 1u;
                    ok = (t > w.tile || mbar_wait_warp(ptx::smem_addr(&B.k_full[slot[x].at]), slot[x].phase, abort_ptr)) &&
                         mbar_wait_warp(ptx::smem_addr(&B.s_empty[x][buffer]), ((n_s[x] >> 1) & 1u) ^ 1u, abort_ptr);
                    if (!ok) break;
                    ++n_s[x];
                    ptx::tc_fence_after();
                    const uint64_t a = ptx::smem_desc(smem + P.off_k + slot[x].at * K_SLOT, 16, 1024, ptx::SWIZZLE_128B);
                    if (ptx::elect_one()) {
#pragma unroll
                        for (int i = 0; i < D / 16; ++i)
                            ptx::mma_f16(tmem + (2 * x + buffer) * COLS, a + (uint64_t)((i >> 2) * 1024 + (i & 3) * 2), b + (uint64_t)((i >> 2) * (q_line >> 4) + (i & 3) * 2),
                                         idesc, i > 0);
                        ptx::mma_commit(ptx::smem_addr(&B.s_full[x][buffer]));
                    }
                    __syncwarp();
                }
                if (ok && ptx::elect_one()) ptx::mma_commit(ptx::smem_addr(&B.q_empty[q.at]));
                __syncwarp();
                q.step(P.q_stages);
            }
            for (int x = 0; x < nh; ++x) {
                if (ok && ptx::elect_one()) ptx::mma_commit(ptx::smem_addr(&B.k_empty[k.at]));
                __syncwarp();
                k.step(P.k_stages);
            }
        }
        // tensor memory is given back when nothing writes to it any more
        if (ptx::elect_one()) ptx::mma_commit(ptx::smem_addr(&B.drained));
        __syncwarp();
        for (int spin = 0; spin < (1 << 16) && !ptx::mbar_try_wait(ptx::smem_addr(&B.drained), 0u); ++spin) {}
    } else if (CODES && warp >= CW_EXPAND) {
        Ring raw, k;
        const int row = (warp - CW_EXPAND) * 32 + lane;
        for (; ok && w.more(); w.next(P.plan))
            for (int x = 0; x < halves(w); ++x) {
                ok = mbar_wait_warp(ptx::smem_addr(&B.raw_full[raw.at]), raw.phase, abort_ptr) &&
                     mbar_wait_warp(ptx::smem_addr(&B.k_empty[k.at]), k.phase ^ 1u, abort_ptr);
                if (!ok) break;
                expand_code_row<D, T>(gen + P.off_raw + raw.at * RAW_SLOT, gen + P.off_k + k.at * K_SLOT, row);
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    ptx::mbar_arrive(ptx::smem_addr(&B.k_full[k.at]));
                    ptx::mbar_arrive(ptx::smem_addr(&B.raw_empty[raw.at]));
                }
                raw.step(P.raw_stages);
                k.step(P.k_stages);
            }
    } else if (warp < 8) {
        // ---- a group of four warps for each half, a key a thread; every thread passes all named barriers, whatever became of its waits ------
        const int x = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t t_row = tmem + ((uint32_t)((warp & 3) * 32) << 16) + x * 2 * COLS;
        uint32_t n_s = 0;
        for (; w.more(); w.next(P.plan)) {
            if (x >= halves(w)) continue;
            const int key = w.p * CW_KEYS + x * CW_HALF + row, base = w.s.length - w.s.queries;
            const bool live = key < w.s.length;
            const int page = live ? page_of(P.plan.seq, w.b, key) : P.plan.seq.pages;
            const bool inside = page < P.plan.seq.pages;
            const long long at = (((long long)page * P.plan.kv_heads + w.h) << P.plan.seq.page_shift) + (key & ((1 << P.plan.seq.page_shift) - 1));
            const float step = CODES && inside ? P.k_steps[at] : 1.0f;
            const float before = w.whole() && inside && P.in ? P.in[at] : 0.0f;
            const f32x2 c2 = f2_dup(P.c * step);
            f32x2 acc[2] = {f2_dup(0.0f), f2_dup(0.0f)};
            const int row_token = row / P.plan.group, row_head = w.h * P.plan.group + row - row_token * P.plan.group;
            auto rows_of = [&](int t) { return min(P.plan.tile_tokens, w.s.queries - (w.first + t) * P.plan.tile_tokens) * P.plan.group; };
            auto lse_of = [&](int t) {                                 // of this thread's row of tile t
                if (t >= w.end || row >= rows_of(t)) return INFINITY;
                return P.lse[(long long)(w.s.first + (w.first + t) * P.plan.tile_tokens + row_token) * P.q_heads + row_head];
            };
            float next = lse_of(w.tile);
            for (int t = w.tile; t < w.end; ++t, ++n_s) {
                const uint32_t buffer = n_s & 1u;
                float* const l = minus_lse[x][buffer];
                // (the value asked for a tile ahead; a row that saw nothing gives nothing)
                if (row < (int)COLS) l[row] = next == -INFINITY ? -INFINITY : next * -1.4426950408889634f;
                asm volatile("bar.sync %0, 128;" ::"r"(1 + x) : "memory");
                next = lse_of(t + 1);
                ok = ok && mbar_wait_warp(ptx::smem_addr(&B.s_full[x][buffer]), (n_s >> 1) & 1u, abort_ptr);
                if (!ok) continue;
                ptx::tc_fence_after();
                const int i0 = (w.first + t) * P.plan.tile_tokens, rows = rows_of(t);
                int low = 0, high = rows;
                if (P.plan.causal) low = min(max(key - base - i0, 0), P.plan.tile_tokens) * P.plan.group;
                if (P.plan.window) high = min(high, min(max(key - base + P.plan.window - i0, 0), P.plan.tile_tokens) * P.plan.group);
                const uint32_t from = t_row + buffer * COLS;
                if (FEW) {
                    uint32_t v[32];
                    ptx::tmem_ld32(from, v);
                    ptx::tmem_ld_wait();
                    weigh_block<true>(v, l, c2, low, high, acc);
                } else {
                    uint32_t v[2][32];
                    ptx::tmem_ld32(from, v[0]);
#pragma unroll
                    for (int block = 0; block < 4; ++block) {
                        if (block * 32 >= rows) break;
                        const bool masked = !__all_sync(0xffffffffu, low <= block * 32 && high >= block * 32 + 32);
                        ptx::tmem_ld_wait();
                        if (block < 3 && block * 32 + 32 < rows) ptx::tmem_ld32(from + block * 32 + 32, v[(block + 1) & 1]);
                        if (masked) weigh_block<true>(v[block & 1], l + block * 32, c2, low - block * 32, high - block * 32, acc);
                        else weigh_block<false>(v[block & 1], l + block * 32, c2, 0, 32, acc);
                    }
                }
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(ptx::smem_addr(&B.s_empty[x][buffer]));
            }
            float a, b, c, d;
            f2_unpack(acc[0], a, b);
            f2_unpack(acc[1], c, d);
            const float sum = (a + b) + (c + d);
            if (ok) {
                if (!w.whole()) P.partial[(2ll * blockIdx.x + (w.tile > 0 ? 0 : 1)) * CW_KEYS + x * CW_HALF + row] = sum;
                else if (inside) P.out[at] = before + sum;
            }
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == CW_MMA) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, TMEM_COLS);
    }
}

// Sums the parts of a run of keys that several CTAs worked on: the block of the second of them does it.
__global__ void __launch_bounds__(CW_KEYS)
cache_weigh_join_kernel(const __grid_constant__ WeighParams P) {
    grid_dependency_wait();
    grid_dependency_launch();
    const JoinNote n = P.notes[blockIdx.x + 1];
    if (n.last_cta < 0) return;
    const Sequence s{n.length, n.first, n.queries};
    const int key = n.p * CW_KEYS + (int)threadIdx.x;
    if (key >= s.length) return;
    const int page = page_of(P.plan.seq, n.b, key);
    if (page >= P.plan.seq.pages) return;
    const long long at = (((long long)page * P.plan.kv_heads + n.h) << P.plan.seq.page_shift) + (key & ((1 << P.plan.seq.page_shift) - 1));
    float sum = P.partial[(2ll * n.first_cta + 1) * CW_KEYS + threadIdx.x];
    for (int cta = n.first_cta + 1; cta <= n.last_cta; ++cta) sum += P.partial[2ll * cta * CW_KEYS + threadIdx.x];
    P.out[at] = (P.in ? P.in[at] : 0.0f) + sum;
}

inline int weigh_grid() { return 3 * sm_count(); }                     // (of few query rows; a CTA an SM otherwise)

template <int D, typename T, bool CODES, bool FEW>
int cache_weigh_go(WeighParams& P, const CUtensorMap& map_q, const CUtensorMap& map_k, size_t smem, long long steps, cudaStream_t st) {
    // CTAs that fit an SM beside one another (FEW: barriers and the like take less than 2 KB)
    const int fit = (int)(228 * 1024 / (smem + 3 * 1024));
    long long grid = (long long)(!FEW ? 1 : fit < (CODES ? 2 : 3) ? fit : (CODES ? 2 : 3)) * sm_count();
    if (grid > steps) grid = steps;
    const int dev = current_device();
    if (dev < 0) return VITINT_ERR_CUDA;
    static bool attr_set_dev[MAX_DEVICES] = {};
    if (!attr_set_dev[dev]) {
        if (cudaFuncSetAttribute(cache_weigh_kernel<D, T, CODES, FEW>, cudaFuncAttributeMaxDynamicSharedMemorySize, 214 * 1024) != cudaSuccess) return VITINT_ERR_CUDA;
        attr_set_dev[dev] = true;
    }
    launch_kernel(cache_weigh_kernel<D, T, CODES, FEW>, dim3((unsigned)grid), dim3((CODES ? 14 : 10) * 32), smem, st, map_q, map_k, P);
    if (int rc = cuda_status(cudaGetLastError())) return rc;
    // (few query rows are one step for every run of keys: nothing is split)
    if (!FEW && grid > 1) launch_kernel(cache_weigh_join_kernel, dim3((unsigned)grid - 1), dim3(CW_KEYS), 0, st, P);
    return cuda_status(cudaGetLastError());
}

template <int D, typename T, bool CODES>
int cache_weigh_launch(WeighParams& P, const void* q, int64_t tokens, int64_t q_token, int64_t q_head, const vitint_cache* cache,
                       const vitint_cache_batch* batch, void* workspace, cudaStream_t st) {
    constexpr int LINES = D / 64;
    const long long runs = (batch->max_length + CW_KEYS - 1) / CW_KEYS, tiles = most_runs(batch, tokens, P.plan.tile_tokens);
    long long items;
    if (!plan_fits(cache, batch, runs, tiles, items)) return VITINT_ERR_UNSUPPORTED;
    const int box_tokens = P.plan.tile_tokens < batch->max_queries ? P.plan.tile_tokens : batch->max_queries;
    P.box_rows = box_tokens * P.plan.group;
    P.n_pad = (P.box_rows + 15) / 16 * 16;
    P.q_slot = (uint32_t)(LINES * P.n_pad * 128);
    P.page_rows = cache->page_tokens;
    // At most 32 rows are all of a sequence's new tokens where a tile holds as many.
    const bool few = P.n_pad <= 32 && batch->max_queries <= P.plan.tile_tokens;
    P.q_stages = CODES || few ? 2 : 3;
    P.k_stages = few ? 2 : 3;
    P.raw_stages = CODES ? (few ? 1 : 2) : 0;
    P.off_q = 0;
    P.off_k = P.off_q + P.q_stages * P.q_slot;
    P.off_raw = P.off_k + P.k_stages * LINES * 16384;
    const size_t smem = P.off_raw + (size_t)P.raw_stages * CW_HALF * D + 1024;
    static_assert(6 * 32768 + 1024 <= 214 * 1024, "shared memory");
    CUtensorMap map_q, map_k;
    if (!encode_query_map(&map_q, q, std::is_same<T, __nv_bfloat16>::value ? VITINT_BF16 : VITINT_F16, D, tokens, P.q_heads, q_token, q_head, P.plan.group, box_tokens) ||
        !encode_cache_map(&map_k, cache, cache->k, P.page_rows, CODES))
        return VITINT_ERR_CUDA;
    P.notes = (JoinNote*)workspace;
    P.partial = (float*)((uint8_t*)workspace + notes_bytes(weigh_grid()));
    return few ? cache_weigh_go<D, T, CODES, true>(P, map_q, map_k, smem, items * tiles, st) : cache_weigh_go<D, T, CODES, false>(P, map_q, map_k, smem, items * tiles, st);
}

}  // namespace
}  // namespace vitint

using namespace vitint;

extern "C" size_t vitint_cache_weigh_workspace_bytes(const vitint_cache* cache, const vitint_cache_batch* batch) {
    if (check_cache(cache) != VITINT_OK || check_batch(cache, batch, true) != VITINT_OK) return 0;
    return notes_bytes(weigh_grid()) + (size_t)sm_count() * 2 * CW_KEYS * 4;
}

extern "C" int vitint_cache_weigh(const void* q, int32_t q_type, int64_t tokens, int32_t q_heads, int64_t q_token_stride, int64_t q_head_stride,
                                  const float* lse, const vitint_cache* cache, const vitint_cache_batch* batch, float scale, int32_t causal,
                                  int32_t window, const float* weights_in, float* weights_out, void* workspace, size_t workspace_bytes,
                                  void* stream) {
    if (int rc = check_paged_queries(q, q_type, tokens, q_heads, q_token_stride, q_head_stride, cache, batch, scale, causal, window)) return rc;
    if (!lse || !weights_out) return VITINT_ERR_INVALID_ARG;
    if (!aligned_to(lse, 4) || !aligned_to(weights_in, 4) || !aligned_to(weights_out, 4)) return VITINT_ERR_ALIGNMENT;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < vitint_cache_weigh_workspace_bytes(cache, batch))
        return VITINT_ERR_WORKSPACE;
    WeighParams P{};
    P.plan = plan_params(cache, batch, tokens, q_heads, causal, window);
    P.plan.tile_tokens = 128 / P.plan.group;
    P.lse = lse; P.in = weights_in; P.out = weights_out;
    P.k_steps = cache->k_steps;
    P.c = (float)((double)scale * 1.4426950408889634);
    P.q_heads = q_heads;
    cudaStream_t st = (cudaStream_t)stream;
    const bool codes = cache->type == VITINT_I8, bf16 = q_type == VITINT_BF16;
    auto go = [&](auto launch) { return launch(P, q, tokens, q_token_stride, q_head_stride, cache, batch, workspace, st); };
    if (cache->head_dim == 64) {
        if (codes) return bf16 ? go(cache_weigh_launch<64, __nv_bfloat16, true>) : go(cache_weigh_launch<64, __half, true>);
        return bf16 ? go(cache_weigh_launch<64, __nv_bfloat16, false>) : go(cache_weigh_launch<64, __half, false>);
    }
    if (codes) return bf16 ? go(cache_weigh_launch<128, __nv_bfloat16, true>) : go(cache_weigh_launch<128, __half, true>);
    return bf16 ? go(cache_weigh_launch<128, __nv_bfloat16, false>) : go(cache_weigh_launch<128, __half, false>);
}
