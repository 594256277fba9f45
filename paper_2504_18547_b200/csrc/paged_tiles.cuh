// What the tensor-core kernels over the paged cache share: 16-bit products on tcgen05, query tiles, and 8-bit codes as 16-bit operands.
#pragma once

#include "paged_plan.cuh"

namespace vitint {
namespace ptx {

// Instruction descriptor of a 16-bit MMA with fp32 accumulators: accumulator format F32 (1) in bits [4,6), operand format in [7,10) and
// [10,13) (0 fp16, 1 bf16), B major-ness in bit 16 (1 = N contiguous), N >> 3 in [17,23), M >> 4 in [24,29).
__host__ __device__ inline uint32_t idesc_f16(int m, int n, bool bf16, int b_mn_major) {
    uint32_t d = 1u << 4;
    if (bf16) d |= (1u << 7) | (1u << 10);
    d |= (uint32_t)b_mn_major << 16;
    d |= (uint32_t)(n >> 3) << 17;
    d |= (uint32_t)(m >> 4) << 24;
    return d;
}
// D[tmem] (+)= A[smem] * B[smem], 16-bit operands.  One thread issues.
__device__ __forceinline__ void mma_f16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t"
        "}" ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// The same with A in tensor memory: its row in the lane, two elements in each 32-bit column.
__device__ __forceinline__ void mma_f16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
        "}" ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

}  // namespace ptx

// Two signed bytes, one in the low byte of each half of `two` (other bytes anything), as exact 16-bit floats.
// bf16: the seven low bits lie in the significand of 128 .. 255, and the sign bit turns the 128 that is taken off into 256.
// f16: all eight bits, offset by 128, lie in the significand of 1024 .. 1279.
template <typename T>
__device__ __forceinline__ uint32_t codes_to_16(uint32_t two);
template <>
__device__ __forceinline__ uint32_t codes_to_16<__nv_bfloat16>(uint32_t two) {
    const uint32_t low = (two & 0x007F007Fu) | 0x43004300u, off = (two & 0x00800080u) | 0x43004300u;
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(low), "r"(off));
    return r;
}
template <>
__device__ __forceinline__ uint32_t codes_to_16<__half>(uint32_t two) {
    const uint32_t u = ((two & 0x00FF00FFu) ^ 0x00800080u) | 0x64006400u;
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(u), "r"(0x64806480u));        // 1152
    return r;
}
// Four codes of a word, in order, as fp16: one byte permute puts two of them (offset by 128) under the exponent of 1024.
__device__ __forceinline__ uint2 codes_to_half4(uint32_t four) {
    const uint32_t u = four ^ 0x80808080u;
    uint2 r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r.x) : "r"(__byte_perm(u, 0x64646464u, 0x4140)), "r"(0x64806480u));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r.y) : "r"(__byte_perm(u, 0x64646464u, 0x4342)), "r"(0x64806480u));
    return r;
}
// Four codes of a word, in order.
template <typename T>
__device__ __forceinline__ uint2 codes_to_16x4(uint32_t four) {
    return make_uint2(codes_to_16<T>(__byte_perm(four, 0u, 0x4140)), codes_to_16<T>(__byte_perm(four, 0u, 0x4342)));
}

__device__ __forceinline__ float max_or_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// 2^x of a pair, -127 <= x < 128, without the special-function unit: x = n + f with n the nearest integer (the constant 1.5 * 2^23 rounds), 2^f on
// [-1/2, 1/2] by a polynomial of degree five (weighted least squares on Chebyshev nodes until the relative error is even: 7.5e-8, 2.2e-7 with fp32
// steps), times 2^n, which is 0 for n = -127.  What is no number stays none (an exponent added to the bits would make it finite).  Nine packed operations
// and two integer ones take as long on the FMA pipe as the special-function unit takes for two results, so a kernel that is bound by exponentials
// shares them between the two.
__device__ __forceinline__ void exp2_poly(f32x2 x, float& a, float& b) {
    const f32x2 t = f2_add(x, f2_dup(12582912.0f));
    const f32x2 f = f2_fma(f2_add(t, f2_dup(-12582912.0f)), f2_dup(-1.0f), x);
    f32x2 p = f2_fma(f2_dup(1.327647129e-03f), f, f2_dup(9.675540961e-03f));
    p = f2_fma(p, f, f2_dup(5.550713092e-02f));
    p = f2_fma(p, f, f2_dup(2.402212024e-01f));
    p = f2_fma(p, f, f2_dup(6.931469440e-01f));
    p = f2_fma(p, f, f2_dup(1.000000119e+00f));
    float ta, tb;
    f2_unpack(t, ta, tb);
    p = f2_mul(p, f2_pack(__uint_as_float((__float_as_uint(ta) << 23) + 0x3F800000u), __uint_as_float((__float_as_uint(tb) << 23) + 0x3F800000u)));
    f2_unpack(p, a, b);
}

// Bits of the columns of a block of 32 that a row sees: low <= column < high.
__device__ __forceinline__ uint32_t seen_bits(int low, int high) {
    const uint32_t below_high = high >= 32 ? 0xFFFFFFFFu : high <= 0 ? 0u : (1u << high) - 1u;
    return low >= 32 ? 0u : low <= 0 ? below_high : below_high & ~((1u << low) - 1u);
}

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

// fp16 holds 2^15 and more, but what lies below 2^-24 becomes 0: a probability enters the second product as the multiple 2^offset of itself, and so do
// the sum that it is divided by and the maximum that both refer to (lower by the offset), so that the offset cancels.  Without it all that lies 17.4 nats
// below the maximum would be lost from the output (not from the sum): behind one token, 131,072 of them at 17.5 nats hold 0.3 % of the weight.
// `room`: how far above 1 a probability (times a step that is below 4 relative to the unit of the steps) may lie, as a power of two.
template <typename M>
__host__ __device__ constexpr float probability_offset(int room) { return std::is_same<M, __half>::value ? (float)(13 - room) : 0.0f; }
__host__ __device__ constexpr float offset_back(float offset) { return 1.0f / (float)(1 << (int)offset); }

// Steps of a page that is not there: the TMA fills its codes with zeros, the steps are plain copies, so the thread that would have copied them writes
// zeros (what shared memory held could be NaN or huge).  Key steps at `to`, value steps `apart` bytes behind; in front of the thread's arrival.
__device__ __forceinline__ void zero_steps(uint8_t* to, int apart, int rows) {
    for (int i = 0; i < rows; i += 4) {
        *reinterpret_cast<uint4*>(to + i * 4) = make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4*>(to + apart + i * 4) = make_uint4(0u, 0u, 0u, 0u);
    }
    ptx::fence_proxy_async_smem();                                      // (the slot's next steps come by asynchronous copies)
}

// A tile of 128 rows of D 16-bit channels as the tensor core wants it: lines of 64 channels, row r of line i at i * 16384 + r * 128, its 16-byte
// chunk c at slot c ^ (r % 8).  A row of raw codes (as the TMA left them: chunks swizzled likewise) becomes a row of it.
template <int D, typename T>
__device__ __forceinline__ void expand_code_row(const uint8_t* raw, uint8_t* tile, int r) {
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
        const int from = D == 128 ? (j ^ (r & 7)) : (j ^ ((r >> 1) & 3));
        const uint4 w = *reinterpret_cast<const uint4*>(raw + r * D + from * 16);
        const uint2 a = codes_to_16x4<T>(w.x), b = codes_to_16x4<T>(w.y), c = codes_to_16x4<T>(w.z), d = codes_to_16x4<T>(w.w);
        uint8_t* const line = tile + (j >> 2) * 16384 + r * 128;
        const int chunk = 2 * (j & 3), sw = r & 7;
        *reinterpret_cast<uint4*>(line + ((chunk ^ sw) << 4)) = make_uint4(a.x, a.y, b.x, b.y);
        *reinterpret_cast<uint4*>(line + (((chunk + 1) ^ sw) << 4)) = make_uint4(c.x, c.y, d.x, d.y);
    }
}

// Queries as rows token by token, the group's heads of a token behind one another: (64 channels, heads, tokens, lines of a head), one line a
// copy.
inline bool encode_query_map(CUtensorMap* map, const void* q, int type, int dim, int64_t tokens, int heads, int64_t token_stride, int64_t head_stride,
                             int group, int box_tokens) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[4] = {64, (cuuint64_t)heads, (cuuint64_t)tokens, (cuuint64_t)(dim / 64)};
    const cuuint64_t strides[3] = {(cuuint64_t)(head_stride * 2), (cuuint64_t)(token_stride * 2), 128};
    const cuuint32_t box[4] = {64, (cuuint32_t)group, (cuuint32_t)box_tokens, 1}, estr[4] = {1, 1, 1, 1};
    return fn(map, type == VITINT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(q), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace vitint
