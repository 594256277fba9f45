// Norm of query and key heads, rotation by position and the store of keys and values in the paged cache, in one pass.
//
//   y = norm(x) per head (fp32), (y1, y2) -> (y1 cos a - y2 sin a, y2 cos a + y1 sin a) with a = position * frequency, one rounding.
//
// Every input is read once and every output written once; the arithmetic is some twenty operations an element, which with fp32 rows, a layer norm and
// codes is what bounds it (8190 tokens x 40 head rows of 128: 66 us, 66 % of the issue slots, against 36 for the bytes).  A head row
// is spread over D/8 threads, eight consecutive channels each (one 16-byte access, two for fp32), so that the norm's sums are a
// few shuffles, a pair of neighbours lies in one thread, and the partner half of a channel in another one of the row, the same
// number of threads away for all eight (rotary dimensions are multiples of 16).  The angles belong to the token, not to the head:
// a block computes them once (position * frequency in fp64 - an fp32 product at position 10^6 is off by 0.03 rad -, the whole
// turns taken off in fp64, then sine and cosine in fp32) and uses them for all heads that it walks.  Blocks take a token's heads
// together where there are tokens enough to fill the GPU, and share them out where there are not.
#include "cache.cuh"

namespace vitint {
namespace {

constexpr int QN_THREADS = 256;

struct RotateParams {
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride;
    int tokens, q_heads, kv_heads, rotary;
    int heads_per_block, blocks_per_token;
    float eps;
    const float *q_gain, *k_gain, *q_offset, *k_offset;
    const int* positions;
    const double* frequencies;
    void *q_out, *k_out;
    long long q_out_stride, k_out_stride;
    const long long* slots;
    float* weights;
    void *cache_k, *cache_v;
    float *k_steps, *v_steps;
    long long page_stride, head_stride, token_stride, places;
    int page_shift, cache_heads;
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack16<T>(u[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&x)[8]) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&y)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack16<T>(y[0], y[1]), pack16<T>(y[2], y[3]), pack16<T>(y[4], y[5]), pack16<T>(y[6], y[7]));
}

template <int LANES>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <int LANES>
__device__ __forceinline__ void row_sums(float& a, float& b) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
        const float x = __shfl_xor_sync(0xffffffffu, a, o), y = __shfl_xor_sync(0xffffffffu, b, o);
        a += x;
        b += y;
    }
}
template <int LANES>
__device__ __forceinline__ float row_max(float v) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// TI: input type, TO: type of q_out, k_out and of a 16-bit cache, CODES: the cache holds 8-bit codes.
template <int D, typename TI, typename TO, bool CODES>
__global__ void __launch_bounds__(QN_THREADS, 4)
qk_norm_rotate_kernel(const __grid_constant__ RotateParams P, int norm, int pairs) {
    constexpr int LANES = D / 8, ROWS = QN_THREADS / LANES;              // threads of a head row, rows that a block walks side by side
    __shared__ float2 turn[D / 2];                                       // (cos, sin) of the token's angles
    grid_dependency_wait();
    grid_dependency_launch();
    const int token = blockIdx.x / P.blocks_per_token, part = blockIdx.x - token * P.blocks_per_token;
    const int half = P.rotary >> 1;
    const int lane = threadIdx.x % LANES, c0 = lane * 8, sub = (threadIdx.x & 31) - lane;     // sub: the row's first lane in its warp
    const int heads = P.q_heads + P.kv_heads + (P.cache_v ? P.kv_heads : 0);
    const int end = min(heads, (part + 1) * P.heads_per_block);
    const TI* const q0 = (const TI*)P.q + token * P.q_stride + c0;
    const TI* const k0 = (const TI*)P.k + token * P.k_stride + c0 - P.q_heads * D;
    const TI* const v0 = (const TI*)P.v + token * P.v_stride + c0 - (P.q_heads + P.kv_heads) * D;
    auto load_row = [&](int h, float (&y)[8]) {
        if (h < end) load8<TI>((h < P.q_heads ? q0 : h < P.q_heads + P.kv_heads ? k0 : v0) + h * D, y);
    };
    // the first row is asked for in front of the angles, every other one while its predecessor is worked on
    int h = part * P.heads_per_block + (int)threadIdx.x / LANES;
    float ahead[8] = {};
    load_row(h, ahead);
    const long long slot = P.slots ? P.slots[token] : -1;
    if ((int)threadIdx.x < half) {
        const double turns = (double)P.positions[token] * P.frequencies[threadIdx.x] * 0.15915494309189533577;   // 1 / 2 pi
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        turn[threadIdx.x] = make_float2(c, s);
    }
    __syncthreads();
    const bool stored = slot >= 0 && slot < P.places;
    const long long page = slot >> P.page_shift;
    const int place = (int)(slot - (page << P.page_shift));
    TO* const qo = (TO*)P.q_out + token * P.q_out_stride + c0;
    TO* const ko = (TO*)P.k_out + token * P.k_out_stride + c0;
    const long long cache_at = page * P.page_stride + place * P.token_stride + c0, flat_at = ((page * P.cache_heads) << P.page_shift) + place;
    // every thread of a warp takes the same number of steps: the shuffles below need all of them
    for (int h0 = part * P.heads_per_block; h0 < end; h0 += ROWS, h += ROWS) {
        const bool live = h < end;
        const bool is_q = h < P.q_heads, is_v = h >= P.q_heads + P.kv_heads;
        const int hk = is_q ? h : (h - P.q_heads) - (is_v ? P.kv_heads : 0);
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = ahead[i];
        load_row(h + ROWS, ahead);
        if (__any_sync(0xffffffffu, live && !is_v)) {                     // (values are neither normed nor rotated)
            if (norm != VITINT_NORM_NONE) {
                const float* const gain = is_q ? P.q_gain : P.k_gain;
                const float* const offset = is_q ? P.q_offset : P.k_offset;
                float g[8], o[8] = {};
                if (live && !is_v) {
                    load8<float>(gain + c0, g);
                    if (offset) load8<float>(offset + c0, o);
                }
                // Mean and variance in one pass: sums of x - x0 and of its square, x0 the row's first channel.  The variance is the mean square less
                // the mean's, which x0 costs at most a factor D in precision: no channel is more than sqrt(D) deviations away from the mean.
                float mean = 0.0f, v;
                if (norm == VITINT_NORM_LAYER) {
                    const float x0 = __shfl_sync(0xffffffffu, y[0], sub);
                    float s = 0.0f, q = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) { const float d = y[i] - x0; s += d; q = fmaf(d, d, q); }
                    row_sums<LANES>(s, q);
                    s *= 1.0f / D;
                    mean = x0 + s;
                    v = fmaxf(fmaf(-s, s, q * (1.0f / D)), 0.0f) + P.eps;
                } else {
                    float q = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) q = fmaf(y[i], y[i], q);
                    v = fmaf(row_sum<LANES>(q), 1.0f / D, P.eps);
                }
                // 1 / sqrt by the hardware's approximation and a Newton step (0 and infinity stay what the approximation makes of them)
                float r;
                asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
                if (v > 1e-36f && v < 1e36f) r = r * fmaf(-0.5f * v * r, r, 1.5f);
                if (live && !is_v) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = fmaf((y[i] - mean) * r, g[i], o[i]);
                }
            }
            if (half) {
                const bool turned = !is_v && c0 < P.rotary;
                if (pairs) {
                    if (turned) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float2 t = turn[(c0 >> 1) + i];
                            const float a = y[2 * i], b = y[2 * i + 1];
                            y[2 * i] = fmaf(a, t.x, -b * t.y);
                            y[2 * i + 1] = fmaf(b, t.x, a * t.y);
                        }
                    }
                } else {
                    const bool low = c0 < half;
                    const int from = sub + (lane + (low ? half / 8 : LANES - half / 8)) % LANES;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float other = __shfl_sync(0xffffffffu, y[i], from);
                        if (turned) {
                            const float2 t = turn[(low ? c0 : c0 - half) + i];
                            y[i] = fmaf(y[i], t.x, low ? -other * t.y : other * t.y);
                        }
                    }
                }
            }
        }
        float step = 0.0f;
        if (CODES && __any_sync(0xffffffffu, live && !is_q)) {
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(y[i]));
            step = row_max<LANES>(m) * (1.0f / 127.0f);
        }
        if (!live) continue;
        if (is_q) {
            store8<TO>(qo + hk * D, y);
            continue;
        }
        if (!is_v && P.k_out) store8<TO>(ko + hk * D, y);
        if (!stored) continue;
        const long long at = cache_at + hk * P.head_stride;
        void* const base = is_v ? P.cache_v : P.cache_k;
        if (CODES) {
            uint32_t w[2] = {0u, 0u};
            // the quotient by the step's reciprocal; at most 127 (1 + 2^-21), which needs no clamp, unless the step is denormal
            if (step >= 1e-37f) {
                float r;
                asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(step));
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t u[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) u[k] = __float_as_uint(fmaf(y[4 * i + k], r, 12582912.0f));       // rounded to an integer in the low bits
                    w[i] = __byte_perm(__byte_perm(u[0], u[1], 0x0040), __byte_perm(u[2], u[3], 0x0040), 0x5410);
                }
            } else if (step > 0.0f) {
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i >> 2] |= (round_clamp_bits(__fdiv_rn(y[i], step), -127.0f, 127.0f) & 255u) << (8 * (i & 3));
            }
            *reinterpret_cast<uint2*>((int8_t*)base + at) = make_uint2(w[0], w[1]);
            if (lane == 0) (is_v ? P.v_steps : P.k_steps)[flat_at + ((long long)hk << P.page_shift)] = step;
        } else {
            store8<TO>((TO*)base + at, y);
        }
        if (lane == 0 && !is_v && P.weights) P.weights[flat_at + ((long long)hk << P.page_shift)] = 0.0f;
    }
}

template <int D, typename TI, typename TO>
void rotate_launch(const RotateParams& P, bool codes, int norm, int pairs, cudaStream_t st) {
    const dim3 grid((unsigned)(P.tokens * P.blocks_per_token));
    if (codes) launch_kernel(qk_norm_rotate_kernel<D, TI, TO, true>, grid, dim3(QN_THREADS), 0, st, P, norm, pairs);
    else launch_kernel(qk_norm_rotate_kernel<D, TI, TO, false>, grid, dim3(QN_THREADS), 0, st, P, norm, pairs);
}
template <int D, typename TI>
void rotate_launch(const RotateParams& P, int out_type, bool codes, int norm, int pairs, cudaStream_t st) {
    if (out_type == VITINT_BF16) rotate_launch<D, TI, __nv_bfloat16>(P, codes, norm, pairs, st);
    else rotate_launch<D, TI, __half>(P, codes, norm, pairs, st);
}
template <int D>
void rotate_launch(const RotateParams& P, int in_type, int out_type, bool codes, int norm, int pairs, cudaStream_t st) {
    if (in_type == VITINT_F32) rotate_launch<D, float>(P, out_type, codes, norm, pairs, st);
    else if (in_type == VITINT_BF16) rotate_launch<D, __nv_bfloat16>(P, out_type, codes, norm, pairs, st);
    else rotate_launch<D, __half>(P, out_type, codes, norm, pairs, st);
}

}  // namespace
}  // namespace vitint

using namespace vitint;

extern "C" int vitint_qk_norm_rotate(const vitint_qk_norm_rotate_desc* d, const vitint_cache* cache, void* stream) {
    if (!d || d->tokens <= 0 || d->q_heads < 0 || d->kv_heads <= 0 || d->q_heads > 65535 || d->kv_heads > 65535) return VITINT_ERR_INVALID_ARG;
    if (d->in_type != VITINT_F32 && d->in_type != VITINT_BF16 && d->in_type != VITINT_F16) return VITINT_ERR_INVALID_ARG;
    if (d->out_type != VITINT_BF16 && d->out_type != VITINT_F16) return VITINT_ERR_INVALID_ARG;
    if (d->norm < VITINT_NORM_NONE || d->norm > VITINT_NORM_LAYER || (d->pairs != 0 && d->pairs != 1)) return VITINT_ERR_INVALID_ARG;
    if (d->head_dim != 64 && d->head_dim != 128) return VITINT_ERR_UNSUPPORTED;
    if (d->rotary < 0 || d->rotary > d->head_dim) return VITINT_ERR_INVALID_ARG;
    if (d->rotary % 16 != 0) return VITINT_ERR_UNSUPPORTED;
    if (d->tokens > 0x1000000) return VITINT_ERR_UNSUPPORTED;
    if (!d->k || (d->q_heads > 0) != (d->q != nullptr) || (d->q_heads > 0) != (d->q_out != nullptr)) return VITINT_ERR_INVALID_ARG;
    if (d->rotary && (!d->positions || !d->frequencies)) return VITINT_ERR_INVALID_ARG;
    const bool normed = d->norm != VITINT_NORM_NONE;
    if (normed != (d->k_gain != nullptr) || (normed && d->q_heads > 0) != (d->q_gain != nullptr)) return VITINT_ERR_INVALID_ARG;
    if ((d->q_offset || d->k_offset) && d->norm != VITINT_NORM_LAYER) return VITINT_ERR_INVALID_ARG;
    if (normed && !(d->eps >= 0.0f && d->eps < INFINITY)) return VITINT_ERR_INVALID_ARG;
    if (cache) {
        if (int rc = check_cache(cache)) return rc;
        if (!d->v || !d->slots || cache->kv_heads != d->kv_heads || cache->head_dim != d->head_dim) return VITINT_ERR_INVALID_ARG;
        if (cache->type != VITINT_I8 && cache->type != d->out_type) return VITINT_ERR_INVALID_ARG;
    } else if (d->v || d->slots || d->weights || !d->k_out) {
        return VITINT_ERR_INVALID_ARG;
    }
    const int in = dtype_bytes(d->in_type);
    const void* pointers[7] = {d->q, d->k, d->v, d->q_gain, d->k_gain, d->q_offset, d->k_offset};
    for (const void* p : pointers) if (!aligned16(p)) return VITINT_ERR_ALIGNMENT;
    if (!aligned16(d->q_out) || !aligned16(d->k_out)) return VITINT_ERR_ALIGNMENT;
    if (!aligned_to(d->positions, 4) || !aligned_to(d->frequencies, 8) || !aligned_to(d->slots, 8) || !aligned_to(d->weights, 4)) return VITINT_ERR_ALIGNMENT;
    const int64_t q_width = (int64_t)d->q_heads * d->head_dim, k_width = (int64_t)d->kv_heads * d->head_dim;
    struct { bool used; int64_t stride, width; int size; } rows[5] = {
        {d->q != nullptr, d->q_stride, q_width, in}, {true, d->k_stride, k_width, in}, {d->v != nullptr, d->v_stride, k_width, in},
        {d->q_out != nullptr, d->q_out_stride, q_width, 2}, {d->k_out != nullptr, d->k_out_stride, k_width, 2}};
    for (auto& r : rows) {
        if (!r.used) continue;
        if (d->tokens > 1 && r.stride < r.width) return VITINT_ERR_INVALID_ARG;
        if (!aligned16_elements(r.stride, r.size)) return VITINT_ERR_ALIGNMENT;
    }
    // a row may be written over itself, by the threads that have read it
    if (d->q && d->q_out == d->q && (d->in_type != d->out_type || d->q_out_stride != d->q_stride)) return VITINT_ERR_INVALID_ARG;
    if (d->k_out == d->k && (d->in_type != d->out_type || d->k_out_stride != d->k_stride)) return VITINT_ERR_INVALID_ARG;
    RotateParams P{};
    P.q = d->q; P.k = d->k; P.v = d->v;
    P.q_stride = d->q_stride; P.k_stride = d->k_stride; P.v_stride = d->v_stride;
    P.tokens = (int)d->tokens; P.q_heads = d->q_heads; P.kv_heads = d->kv_heads; P.rotary = d->rotary;
    P.eps = d->eps;
    P.q_gain = d->q_gain; P.k_gain = d->k_gain; P.q_offset = d->q_offset; P.k_offset = d->k_offset;
    P.positions = d->positions; P.frequencies = d->frequencies;
    P.q_out = d->q_out; P.k_out = d->k_out;
    P.q_out_stride = d->q_out_stride; P.k_out_stride = d->k_out_stride;
    if (cache) {
        P.slots = (const long long*)d->slots;
        P.weights = d->weights;
        P.cache_k = cache->k; P.cache_v = cache->v; P.k_steps = cache->k_steps; P.v_steps = cache->v_steps;
        P.page_stride = cache->page_stride; P.head_stride = cache->head_stride; P.token_stride = cache->token_stride;
        P.places = cache->pages * cache->page_tokens;
        P.page_shift = page_shift_of(cache);
        P.cache_heads = cache->kv_heads;
    }
    // A block walks `rows` head rows side by side: all heads of a token where the tokens alone fill the GPU, else as few as that.
    const int heads = d->q_heads + (cache ? 2 : 1) * d->kv_heads, side = QN_THREADS * 8 / d->head_dim, steps = (heads + side - 1) / side;
    int blocks = (int)((8ll * sm_count() + d->tokens - 1) / d->tokens);
    blocks = blocks > steps ? steps : blocks;
    P.heads_per_block = (steps + blocks - 1) / blocks * side;
    P.blocks_per_token = (heads + P.heads_per_block - 1) / P.heads_per_block;
    if ((long long)P.tokens * P.blocks_per_token > 0x7fffffffll) return VITINT_ERR_UNSUPPORTED;
    const bool codes = cache && cache->type == VITINT_I8;
    cudaStream_t st = (cudaStream_t)stream;
    if (d->head_dim == 64) rotate_launch<64>(P, d->in_type, d->out_type, codes, d->norm, d->pairs, st);
    else rotate_launch<128>(P, d->in_type, d->out_type, codes, d->norm, d->pairs, st);
    return cuda_status(cudaGetLastError());
}
