// The paged cache: host checks of its descriptors, and what its kernels share on the device.
#pragma once

#include <atomic>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "common.cuh"
#include "ptx.cuh"
#include "tile_ops.cuh"

namespace vitint {

constexpr int64_t CACHE_MAX_LENGTH = 1ll << 29;

inline bool aligned16_elements(int64_t n, int size) { return (n * size) % 16 == 0; }
inline bool aligned_to(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline int dtype_bytes(int type) { return type == VITINT_F32 ? 4 : type == VITINT_I8 ? 1 : 2; }

inline int check_cache(const vitint_cache* c) {
    if (!c || !c->k || !c->v || c->pages <= 0 || c->kv_heads <= 0) return VITINT_ERR_INVALID_ARG;
    if (c->type != VITINT_BF16 && c->type != VITINT_F16 && c->type != VITINT_I8) return VITINT_ERR_INVALID_ARG;
    if ((c->type == VITINT_I8) != (c->k_steps != nullptr) || (c->type == VITINT_I8) != (c->v_steps != nullptr)) return VITINT_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128) return VITINT_ERR_UNSUPPORTED;
    if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128) return VITINT_ERR_UNSUPPORTED;
    if (c->pages > 0x7fffffffll || c->kv_heads > 65535) return VITINT_ERR_UNSUPPORTED;
    const int size = dtype_bytes(c->type);
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_steps) || !aligned16(c->v_steps)) return VITINT_ERR_ALIGNMENT;
    const int64_t strides[3] = {c->page_stride, c->head_stride, c->token_stride};
    for (int64_t s : strides) {
        if (s <= 0) return VITINT_ERR_INVALID_ARG;
        if (!aligned16_elements(s, size)) return VITINT_ERR_ALIGNMENT;
        if (s * size >= (1ll << 40)) return VITINT_ERR_UNSUPPORTED;            // the tensor map's limit
    }
    if (c->token_stride < c->head_dim) return VITINT_ERR_INVALID_ARG;
    return VITINT_OK;
}

inline int check_batch(const vitint_cache* c, const vitint_cache_batch* b, bool queries) {
    if (!b || !b->page_table || !b->lengths || b->sequences <= 0 || b->table_stride <= 0) return VITINT_ERR_INVALID_ARG;
    if (queries && (!b->query_starts || b->max_queries <= 0)) return VITINT_ERR_INVALID_ARG;
    if (b->max_length <= 0) return VITINT_ERR_INVALID_ARG;
    if (!aligned_to(b->page_table, 4) || !aligned_to(b->lengths, 4) || !aligned_to(b->query_starts, 4)) return VITINT_ERR_ALIGNMENT;
    if (b->max_length > CACHE_MAX_LENGTH || b->sequences > 65535) return VITINT_ERR_UNSUPPORTED;
    if ((b->max_length + c->page_tokens - 1) / c->page_tokens > b->table_stride) return VITINT_ERR_INVALID_ARG;
    return VITINT_OK;
}

// A [heads of a page][tokens of a page] view of keys or values for the TMA: (channels of one 128-byte line, tokens, lines of a row, heads,
// pages).  `lines`: whether a copy takes all lines of a row (behind one another), or one.
inline bool encode_cache_map(CUtensorMap* map, const vitint_cache* c, const void* base, int rows, bool lines) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const int size = dtype_bytes(c->type), row = c->head_dim * size, line = row < 128 ? row : 128;
    const cuuint64_t dims[5] = {(cuuint64_t)(line / size), (cuuint64_t)c->page_tokens, (cuuint64_t)(row / line), (cuuint64_t)c->kv_heads,
                                (cuuint64_t)c->pages};
    const cuuint64_t strides[4] = {(cuuint64_t)(c->token_stride * size), (cuuint64_t)line, (cuuint64_t)(c->head_stride * size),
                                   (cuuint64_t)(c->page_stride * size)};
    const cuuint32_t box[5] = {(cuuint32_t)(line / size), (cuuint32_t)rows, (cuuint32_t)(lines ? row / line : 1), 1, 1};
    const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    const CUtensorMapDataType type = c->type == VITINT_I8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                                          : (c->type == VITINT_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16);
    return fn(map, type, 5, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              line == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// ---- device ---------------------------------------------------------------------------------------------------------

// What the caller declared does not hold: the call's result is meaningless where it does not, and the status word says so.
__device__ __forceinline__ void report_bad_data() { atomicExch(&g_device_status, (int)VITINT_ERR_INVALID_ARG); }

// Two fp32 values as a pair of the 16-bit type, the first in the low half.
template <typename T>
__device__ __forceinline__ uint32_t pack16(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack16<__nv_bfloat16>(float a, float b) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
template <>
__device__ __forceinline__ uint32_t pack16<__half>(float a, float b) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
template <typename T>
__device__ __forceinline__ float2 unpack16(uint32_t v);
template <>
__device__ __forceinline__ float2 unpack16<__nv_bfloat16>(uint32_t v) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}
template <>
__device__ __forceinline__ float2 unpack16<__half>(uint32_t v) {
    return __half22float2(*reinterpret_cast<__half2*>(&v));
}

__device__ __forceinline__ float exp2_approx(float x) {              // 2 ulp; results below 2^-126 are 0
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// The sequences of a call as the kernels see them.
struct SequenceView {
    const int* page_table;
    const int* lengths;
    const int* starts;
    long long table_stride;
    int sequences;
    int max_length, max_queries;
    int tokens;              // rows of q
    int pages, page_shift;
};

inline int page_shift_of(const vitint_cache* c) { return c->page_tokens == 16 ? 4 : c->page_tokens == 32 ? 5 : c->page_tokens == 64 ? 6 : 7; }

// Whether a kernel of this unit may have written its status word: those that do so take sequences.
static std::atomic<bool> g_cache_called{false};

inline SequenceView sequence_view(const vitint_cache* c, const vitint_cache_batch* b, int64_t tokens) {
    g_cache_called.store(true, std::memory_order_relaxed);
    SequenceView s{};
    s.page_table = b->page_table; s.lengths = b->lengths; s.starts = b->query_starts;
    s.table_stride = b->table_stride;
    s.sequences = b->sequences;
    s.max_length = (int)b->max_length;
    s.max_queries = b->max_queries;
    s.tokens = (int)tokens;
    s.pages = (int)c->pages;
    s.page_shift = page_shift_of(c);
    return s;
}

// Length and query rows of a sequence, brought inside what the host declared (`ok` is cleared where that changes them).
struct Sequence {
    int length, first, queries;
};
__device__ __forceinline__ int length_of(const SequenceView& s, int b, bool& ok) {
    const int l = s.lengths[b], m = min(max(l, 0), s.max_length);
    ok = ok && l == m;
    return m;
}
__device__ __forceinline__ Sequence sequence_of(const SequenceView& s, int b, bool& ok) {
    Sequence q;
    q.length = length_of(s, b, ok);
    const int a = s.starts[b], e = s.starts[b + 1];
    q.first = min(max(a, 0), s.tokens);
    const int end = min(max(e, q.first), s.tokens);
    q.queries = min(end - q.first, s.max_queries);
    ok = ok && a == q.first && e == q.first + q.queries;
    return q;
}
__device__ __forceinline__ Sequence sequence_of(const SequenceView& s, int b) {
    bool unused = true;
    return sequence_of(s, b, unused);
}

// Page table entry of a sequence's token.  An entry outside the cache is reported where it is used and counts as `pages` (nothing lies there: the
// TMA fills in zeros).  The two are apart so that a kernel can ask for entries ahead of their use: a check waits for what it checks.
__device__ __forceinline__ int page_entry(const SequenceView& s, int b, int token) {
    return s.page_table[(long long)b * s.table_stride + (token >> s.page_shift)];
}
__device__ __forceinline__ int checked_page(const SequenceView& s, int entry) {
    if ((unsigned)entry < (unsigned)s.pages) return entry;
    report_bad_data();
    return s.pages;
}
__device__ __forceinline__ int page_of(const SequenceView& s, int b, int token) { return checked_page(s, page_entry(s, b, token)); }

}  // namespace vitint
