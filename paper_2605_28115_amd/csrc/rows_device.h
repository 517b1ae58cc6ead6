// What the kernels over plain caches share: rows of fp32 or bf16 channels as operands of 16 x 16 matrix products, and softmax sums that
// are taken against whole powers of two.
//
// A product of 16 rows with 16 columns over the channels: lane l holds 16 bytes of row (column) l % 16 at byte 64 t + 16 (l / 16), t = 0,
// 1, ..., of both operands.  That is the layout of v_mfma_f32_16x16x32_bf16 for bf16 channels; of fp32 ones each of the four words is an
// operand of v_mfma_f32_16x16x4_f32, whose contraction then runs over the channels in an order that both operands share.  The result: lane
// l has rows 4 (l / 16) .. + 3 of column l % 16.
//
// A softmax weight is 2^(s c - base), s a logit before its scale and c the scale times log2 e, in one fused multiply-add and one exponential.
// base is the column's largest s c so far rounded to a whole number, and moves only when a logit outgrows it by more than kBaseSlack.
// Because base is whole, s c - base is rounded once however large both are, and what joins two parts of a row is an exact power of two.
// (Against a base that is itself rounded, parts taken against different ones are off by 2^(2^-24 |base|), 1e-3 at logits of 40000.)
#pragma once

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <utility>

#include "civic_internal.h"

namespace civic {

typedef __bf16 row_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 row_bf16x8 __attribute__((ext_vector_type(8)));
typedef float row_f32x4 __attribute__((ext_vector_type(4)));

constexpr float kBaseSlack = 8.f;
constexpr float kLog2E = 1.4426950408889634f;

// acc += (16 bytes a lane of 16 rows) x (16 bytes a lane of 16 columns)
template <bool BF16>
__device__ __forceinline__ row_f32x4 mma16(const u32x4& a, const u32x4& b, row_f32x4 acc)
{
    if constexpr (BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(row_bf16x8, a), __builtin_bit_cast(row_bf16x8, b), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x = a[e], y = b[e];
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x), __uint_as_float(y), acc, 0, 0, 0);
        }
        return acc;
    }
}

// A lane's maximum or sum over the four lanes of its column (lanes 16 apart), in all of them.
template <typename OP>
__device__ __forceinline__ float over_rows(float v, OP op)
{
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(p[0]), __uint_as_float(p[1]));
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float rows_max(float v) { return over_rows(v, [](float x, float y) { return fmaxf(x, y); }); }
__device__ __forceinline__ float rows_sum(float v) { return over_rows(v, [](float x, float y) { return x + y; }); }

// Sums taken against base b0 times this join those taken against b1 >= b0 (nothing seen: -infinity, and 0).
__device__ __forceinline__ float base_step(float b0, float b1) { return b0 == b1 ? 1.f : __builtin_amdgcn_exp2f(b0 - b1); }

// Two fp32 values rounded to one word of bf16; bf16_rest also leaves what the rounding took off.
__device__ __forceinline__ uint32_t bf16_word(float a, float b)
{
    const row_bf16x2 p = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
    return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ uint32_t bf16_rest(float& a, float& b)
{
    const uint32_t w = bf16_word(a, b);
    a -= __uint_as_float(w << 16);
    b -= __uint_as_float(w & 0xFFFF0000u);
    return w;
}

__device__ __forceinline__ int clamped(const int32_t* length, int at, int most) { return length ? min(max(length[at], 0), most) : most; }

// Rows [from, s_max) of the weights of all pairs of sample and KV head become base's (0 without one), by workgroup `at` of `count`: what lies behind
// n_ctx in a cache of much room, where a launch has one workgroup to a pair for the rows before.  A thread has eight loads in flight.  (By the pair's workgroup,
// four bytes a thread at a time, 469 rows of 65536 took 61 us for 9 without the rows behind, so 9.9.)
template <int THREADS>
__device__ __forceinline__ void weights_behind(const float* base, float* weights, int64_t pairs, int64_t s_max, int64_t from, uint32_t at, uint32_t count)
{
    constexpr int U = 8;
    const int64_t chunks = (s_max - from + U * THREADS - 1) / (U * THREADS);
    for (int64_t c = at; c < pairs * chunks; c += count) {
        const int64_t pair = c / chunks, key = from + (c - pair * chunks) * (U * THREADS) + threadIdx.x, row = pair * s_max;
        float x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = base != nullptr && key + u * THREADS < s_max ? base[row + key + u * THREADS] : 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (key + u * THREADS < s_max) weights[row + key + u * THREADS] = x[u];
    }
}

// Workgroups for the rows behind: none where they are few, or the pairs so many that theirs fill the chip.
static inline unsigned behind_blocks(int64_t pairs, int64_t s_max, int64_t from, int threads)
{
    if (pairs >= 4096 || s_max - from <= 1024) return 0;
    return static_cast<unsigned>(std::min<int64_t>(2048, (pairs * (s_max - from) + 8 * threads - 1) / (8 * threads)));
}

// The scale of the logits as the kernels take it: its size times log2 e, neither 0 nor infinite (a masked logit of -infinity, or a logit of
// 0, would become NaN), and its sign, which goes into the queries.
struct LogitScale { float log2; uint32_t flip; };
static inline LogitScale logit_scale(float softmax_scale, int32_t head_dim, bool bf16)
{
    const double scale = softmax_scale == 0.f ? 1.0 / std::sqrt(static_cast<double>(head_dim)) : softmax_scale;
    const double size = std::fmin(std::fmax(std::fabs(scale) * 1.4426950408889634, 1.1754944e-38), 3.4028234e38);
    return {static_cast<float>(size), scale < 0.0 ? (bf16 ? 0x80008000u : 0x80000000u) : 0u};
}

// Whether the rows of head_dim elements of a written tensor [n0, n1, n2, head_dim] lie apart: from the smallest stride to the largest, each
// passes over all that the smaller ones span.
static inline bool rows_apart(const int64_t* strides, int64_t n0, int64_t n1, int64_t n2, int32_t head_dim)
{
    std::pair<int64_t, int64_t> x[3] = {{strides[0], n0}, {strides[1], n1}, {strides[2], n2}};
    std::sort(x, x + 3);
    int64_t span = head_dim;
    for (const auto& [stride, n] : x) {
        if (n <= 1) continue;
        if (stride < span || stride > (INT64_MAX - span) / (n - 1)) return false;
        span += stride * (n - 1);
    }
    return true;
}

// Whether two arrays of `bytes` bytes are the same one, or one is missing, or they share no memory.
static inline bool same_or_apart(const void* x, const void* y, int64_t bytes)
{
    const uintptr_t p = reinterpret_cast<uintptr_t>(x), q = reinterpret_cast<uintptr_t>(y);
    return p == q || p == 0 || q == 0 || (p < q ? q - p : p - q) >= static_cast<uintptr_t>(bytes);
}

// Bytes from the first element of a strided tensor [n0, n1, n2, head_dim] to its last (memory has less than 2^53; none: 0).
static inline int64_t reach_bytes(const int64_t* strides, int64_t n0, int64_t n1, int64_t n2, int32_t head_dim, int elem)
{
    if (n0 <= 0 || n1 <= 0 || n2 <= 0) return 0;
    const double last = (n0 - 1.0) * strides[0] + (n1 - 1.0) * strides[1] + (n2 - 1.0) * strides[2] + head_dim;
    return static_cast<int64_t>(std::fmin(last * elem, 0x1p62));
}

// `bytes` bytes of memory, or none.
struct Memory {
    const void* at;
    int64_t bytes;
    bool apart(const Memory& o) const
    {
        const uintptr_t p = reinterpret_cast<uintptr_t>(at), q = reinterpret_cast<uintptr_t>(o.at);
        return !at || !o.at || bytes <= 0 || o.bytes <= 0 || p + static_cast<uintptr_t>(bytes) <= q || q + static_cast<uintptr_t>(o.bytes) <= p;
    }
};
// Whether what a call writes shares no memory with what else it writes or reads.
static inline bool writes_apart(std::initializer_list<Memory> written, std::initializer_list<Memory> read)
{
    for (const Memory* w = written.begin(); w != written.end(); ++w) {
        for (const Memory* x = w + 1; x != written.end(); ++x)
            if (!w->apart(*x)) return false;
        for (const Memory& r : read)
            if (!w->apart(r)) return false;
    }
    return true;
}

static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int64_t kCacheMaxRows = int64_t{1} << 22;           // rows of a head's cache, and of a prefix

// civic_attn_weights of up to kFewWeightRows query rows a KV head (attn_cache.hip); the arguments are checked.
constexpr int64_t kFewWeightRows = 16;
size_t few_weights_bytes(int dtype, int32_t batch, int64_t rows, int32_t n_kv_heads, int32_t head_dim, int64_t n_ctx);
int few_weights(const void* q, const void* k_cache, const float* base, float* weights, int dtype, int32_t batch, int32_t seq, int32_t n_q_heads,
                int32_t n_kv_heads, int32_t head_dim, const int64_t* qs, int64_t s_max, int64_t n_ctx, const int32_t* ctx, int32_t causal,
                float softmax_scale, void* workspace, void* stream);

}  // namespace civic
