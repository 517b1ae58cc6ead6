// civic_kv_write_mx, civic_kv_write_mx_ragged, civic_kv_read_mx: cache rows in 8 or 4 bits (OCP microscaling), written from rows of
// the inputs' type and read back into them.  HBM-bound both ways: every element is met once.
//
// Blocks of 32 channels of a head row share a scale 2^e.  With the block's largest magnitude amax, e is the least integer for which
// amax <= 7 * 2^e (e2m1, whose codes end at 6 and round down from 7) or 464 * 2^e (e4m3: 448), so that no element is off by more than
// half a step.  In amax's bits, 7 = 1.75 * 2^2: the exponent field less 2, and one more where the mantissa is above 0.75 - a carry out
// of the mantissa once 2^21 - 1 is added (464 = 1.8125 * 2^8: 0x17FFFF).  x * 2^-e is exact and rounded once, by the conversion.
//
// A thread takes 8 channels, four threads a block: the largest magnitude meets in two exchanges of neighbouring lanes.
#include "mx_device.h"

namespace civic {

constexpr int kMxThreads = 256;
constexpr int kMxUnroll = 4;                                  // chunks in flight per thread
constexpr int mx_write_unroll(bool rope) { return rope ? 2 : kMxUnroll; }
constexpr int kMxRaggedItems = 64;                            // samples of one ragged launch

struct MxRowsArgs {
    const void* src[2];                                       // rows of the inputs' type (write: read from; read: see dst)
    void* dst[2];
    uint8_t* codes[2];
    uint8_t* scales[2];
    const float2* cos_sin;                                    // or null
    const int32_t* pos;                                       // per sample, or null
    int64_t stride_b, stride_t, stride_h;                     // elements
    int64_t s_max, pos0;
    int32_t seq, n_kv_heads, head_dim, chunks;                // chunks of a head row, one a thread at a time
    int32_t batch0;                                           // sample of blockIdx.y == 0 (ragged groups)
};

// A ragged launch: the first packed row of every sample of the group, and where the last one ends.
struct MxTable {
    int32_t row[kMxRaggedItems + 1];
};
struct MxNoTable {};

__device__ __forceinline__ uint32_t max_of_quad(uint32_t v)
{
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0xB1, 0xF, 0xF, false)));   // quad_perm [1,0,3,2]
    return max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x4E, 0xF, 0xF, false))); // quad_perm [2,3,0,1]
}

// 8 channels as they lie, and as fp32.
template <bool BF16>
struct MxChunk {
    u32x4 w[BF16 ? 1 : 2];
    __device__ __forceinline__ void load(const char* p)
    {
#pragma unroll
        for (int i = 0; i < (BF16 ? 1 : 2); ++i) w[i] = load_streaming(reinterpret_cast<const u32x4*>(p) + i);
    }
    __device__ __forceinline__ void widen(float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) {
                const uint32_t pair = w[0][i];
                x[2 * i] = __uint_as_float(pair << 16);
                x[2 * i + 1] = __uint_as_float(pair & 0xFFFF0000u);
            } else {
                const uint32_t lo = w[0][i], hi = w[BF16 ? 0 : 1][i];
                x[i] = __uint_as_float(lo);
                x[4 + i] = __uint_as_float(hi);
            }
        }
    }
};

// grid: (chunks of a head's tokens, samples, 2 * head + (K or V))
template <int FMT, bool BF16, bool ROPE, typename TABLE>
__global__ __launch_bounds__(kMxThreads) void kv_write_mx_kernel(MxRowsArgs a, TABLE t)
{
    constexpr bool RAGGED = std::is_same<TABLE, MxTable>::value;
    constexpr int ESZ = BF16 ? 2 : 4;
    constexpr uint32_t CARRY = FMT == 4 ? 0x1FFFFFu : 0x17FFFFu, BELOW = FMT == 4 ? 2u : 8u, LAST = FMT == 4 ? 252u : 246u;
    const int which = blockIdx.z & 1, g = blockIdx.z >> 1, b = blockIdx.y;
    int64_t token0 = 0;
    int seq = a.seq;
    const char* src = static_cast<const char*>(a.src[which]) + g * a.stride_h * ESZ;
    if constexpr (RAGGED) { token0 = t.row[b]; seq = t.row[b + 1] - t.row[b]; }
    else src += b * a.stride_b * ESZ;
    const int64_t row0 = a.pos0 + (a.pos ? a.pos[a.batch0 + b] : 0);
    const int64_t head_row0 = (static_cast<int64_t>(a.batch0 + b) * a.n_kv_heads + g) * a.s_max;
    const uint32_t chunks = a.chunks, total = static_cast<uint32_t>(seq) * chunks;
    constexpr int UNROLL = mx_write_unroll(ROPE);
    const uint32_t base = blockIdx.x * (kMxThreads * UNROLL) + threadIdx.x;
    const int half = a.head_dim / 2;
    const bool turns = ROPE && which == 0;

    // all of a thread's loads first: the rotation's second half and its (cos, sin) with them
    MxChunk<BF16> own[UNROLL], other[ROPE ? UNROLL : 1];
    float4 cs[ROPE ? UNROLL : 1][4];
    uint32_t tok[UNROLL], chunk[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        // (a block's four threads are in or out together: chunks is a multiple of four)
        const uint32_t idx = base + u * kMxThreads;
        tok[u] = idx / chunks; chunk[u] = idx - tok[u] * chunks;
        if (idx >= total) continue;
        const char* const from = src + (token0 + tok[u]) * a.stride_t * ESZ;
        const int ch = chunk[u] * 8;
        own[u].load(from + ch * ESZ);
        if constexpr (ROPE) {
            if (turns) {                                      // K: pair (i, i + d / 2)
                other[u].load(from + (ch < half ? ch + half : ch - half) * ESZ);
                const int64_t at = RAGGED ? token0 + tok[u] : static_cast<int64_t>(b) * a.seq + tok[u];
                const float4* const table = reinterpret_cast<const float4*>(a.cos_sin + at * half + (ch < half ? ch : ch - half));
#pragma unroll
                for (int i = 0; i < 4; ++i) cs[u][i] = table[i];
            }
        }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        if (base + u * kMxThreads >= total) continue;
        float x[8];
        own[u].widen(x);
        if constexpr (ROPE) {
            if (turns) {
                const bool low = chunk[u] * 8 < static_cast<uint32_t>(half);
                float y[8];
                other[u].widen(y);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float c = i & 1 ? cs[u][i / 2].z : cs[u][i / 2].x, sn = i & 1 ? cs[u][i / 2].w : cs[u][i / 2].y;
                    float r0, r1;
                    rope_pair(low ? x[i] : y[i], low ? y[i] : x[i], c, sn, r0, r1);
                    x[i] = low ? r0 : r1;
                    if constexpr (BF16) x[i] = static_cast<float>(static_cast<__bf16>(x[i]));
                }
            }
        }
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(x[i]) & 0x7FFFFFFFu);
        amax = max_of_quad(amax);
        const uint32_t up = (amax + CARRY) >> 23;
        uint32_t s = min(max(up, 27u + BELOW) - BELOW, LAST);
        const bool odd = amax >= 0x7F800000u;                 // an infinity or a NaN: the block reads back as NaN
        const float scale = __uint_as_float(s << 23);
        const int64_t row = row0 + tok[u];
        if (row < 0 || row >= a.s_max) continue;
        uint8_t* const dst = a.codes[which] + (head_row0 + row) * (a.head_dim * FMT / 8) + chunk[u] * FMT;
        if constexpr (FMT == 4) {
            uint32_t w = 0;
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
            *reinterpret_cast<uint32_t*>(dst) = odd ? 0u : w;
        } else {
            // only where the scale is the last one can a magnitude be above 464 times it: held at 448
            const float most = __uint_as_float(0x7F600000u);  // 448 * 2^119
            mx_i16x2 w[2] = {{0, 0}, {0, 0}};
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = fminf(fmaxf(x[i], -most), most);
            w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w[0], x[0], x[1], scale, false);
            w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w[0], x[2], x[3], scale, true);
            w[1] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w[1], x[4], x[5], scale, false);
            w[1] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w[1], x[6], x[7], scale, true);
            const u32x2 v = {odd ? 0u : __builtin_bit_cast(uint32_t, w[0]), odd ? 0u : __builtin_bit_cast(uint32_t, w[1])};
            *reinterpret_cast<u32x2*>(dst) = v;
        }
        if ((chunk[u] & 3) == 0) a.scales[which][(head_row0 + row) * (a.head_dim / kMxBlock) + chunk[u] / 4] = static_cast<uint8_t>(odd ? 255u : s);
    }
}

// grid as above.  A thread writes 16 bytes, 8 channels of bf16 or 4 of fp32, so that a wavefront's stores are whole rows (32 bytes a thread
// in two stores: 16 x 4001 rows of 8 bits to fp32 316 us, so 162).
template <int FMT, bool BF16>
__global__ __launch_bounds__(kMxThreads) void kv_read_mx_kernel(MxRowsArgs a)
{
    constexpr int ESZ = BF16 ? 2 : 4, CH = 16 / ESZ, BYTES = CH * FMT / 8;
    const int which = blockIdx.z & 1, g = blockIdx.z >> 1, b = blockIdx.y;
    char* const dst = static_cast<char*>(a.dst[which]) + (b * a.stride_b + g * a.stride_h) * ESZ;
    const int64_t row0 = a.pos0 + (a.pos ? a.pos[b] : 0);
    const int64_t head_row0 = (static_cast<int64_t>(b) * a.n_kv_heads + g) * a.s_max;
    const uint32_t chunks = a.chunks, total = static_cast<uint32_t>(a.seq) * chunks;
    const uint32_t base = blockIdx.x * (kMxThreads * kMxUnroll) + threadIdx.x;

    uint32_t w[kMxUnroll][2], s[kMxUnroll];
    uint32_t tok[kMxUnroll], chunk[kMxUnroll];
    bool live[kMxUnroll];
#pragma unroll
    for (int u = 0; u < kMxUnroll; ++u) {
        const uint32_t idx = base + u * kMxThreads;
        tok[u] = idx / chunks; chunk[u] = idx - tok[u] * chunks;
        const int64_t row = row0 + tok[u];
        live[u] = idx < total && row >= 0 && row < a.s_max;
        if (!live[u]) continue;
        const uint8_t* src = a.codes[which] + (head_row0 + row) * (a.head_dim * FMT / 8) + chunk[u] * BYTES;
        if constexpr (BYTES == 2) w[u][0] = load_streaming(reinterpret_cast<const uint16_t*>(src));
        else if constexpr (BYTES == 4) w[u][0] = load_streaming(reinterpret_cast<const uint32_t*>(src));
        else {
            const u32x2 v = load_streaming(reinterpret_cast<const u32x2*>(src));
            w[u][0] = v[0]; w[u][1] = v[1];
        }
        s[u] = a.scales[which][(head_row0 + row) * (a.head_dim / kMxBlock) + chunk[u] * CH / kMxBlock];
    }
#pragma unroll
    for (int u = 0; u < kMxUnroll; ++u) {
        if (!live[u]) continue;
        const float scale = __uint_as_float(s[u] << 23);
        uint32_t p[CH / 2];
#pragma unroll
        for (int i = 0; i < CH / 2; ++i) p[i] = mx_pair_bf16<FMT>(w[u], i, scale);
        u32x4* out = reinterpret_cast<u32x4*>(dst + (static_cast<int64_t>(tok[u]) * a.stride_t + chunk[u] * CH) * ESZ);
        if constexpr (BF16) store_streaming(out, u32x4{p[0], p[1], p[2], p[3]});
        else store_streaming(out, u32x4{p[0] << 16, p[0] & 0xFFFF0000u, p[1] << 16, p[1] & 0xFFFF0000u});   // values that bf16 holds, widened
    }
}

// Checks of the arguments that write and read share.  CIVIC_OK with *some false: nothing to do.
static int mx_rows_check(const void* k, const void* v, const int64_t* strides, int dtype, int format, const void* k_codes, const void* k_scales,
                         const void* v_codes, const void* v_scales, int32_t batch, int64_t seq, bool any, int32_t n_kv_heads, int32_t head_dim,
                         int64_t s_max, int64_t pos0, const int32_t* pos, bool packed)
{
    const int esz = dtype_size(dtype);
    if (!esz || !strides || !mx_format_ok(format)) return CIVIC_ERR_INVALID_ARG;
    if (batch < 0 || seq < 0 || n_kv_heads <= 0 || head_dim <= 0 || head_dim % kMxBlock) return CIVIC_ERR_INVALID_ARG;
    if (s_max < 0 || s_max % kMxBlock || pos0 < 0 || pos0 > s_max) return CIVIC_ERR_INVALID_ARG;
    if (!pos && pos0 + seq > s_max) return CIVIC_ERR_INVALID_ARG;
    if (any && (!k || !v || !k_codes || !k_scales || !v_codes || !v_scales)) return CIVIC_ERR_INVALID_ARG;
    for (const void* p : {k, v, k_codes, k_scales, v_codes, v_scales})
        if (!aligned16(p)) return CIVIC_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(pos) & 3u) return CIVIC_ERR_INVALID_ARG;
    for (int i = packed ? 1 : 0; i < 3; ++i)
        if (strides[i] < 0 || (strides[i] * esz) % 16) return CIVIC_ERR_INVALID_ARG;
    if (strides[2] < head_dim && n_kv_heads > 1) return CIVIC_ERR_INVALID_ARG;
    if (head_dim > CIVIC_MAX_HEAD_DIM || batch > 65535 || n_kv_heads > 32767 || s_max > kMxMaxRows) return CIVIC_ERR_UNSUPPORTED;
    if (seq * (head_dim / 4) > INT32_MAX) return CIVIC_ERR_UNSUPPORTED;
    return CIVIC_OK;
}

static MxRowsArgs mx_rows_args(const int64_t* strides, const float* cos_sin, const void* k_codes, const void* k_scales, const void* v_codes,
                               const void* v_scales, int64_t seq, int32_t n_kv_heads, int32_t head_dim, int64_t s_max, int64_t pos0, const int32_t* pos)
{
    MxRowsArgs a{};
    a.codes[0] = static_cast<uint8_t*>(const_cast<void*>(k_codes)); a.codes[1] = static_cast<uint8_t*>(const_cast<void*>(v_codes));
    a.scales[0] = static_cast<uint8_t*>(const_cast<void*>(k_scales)); a.scales[1] = static_cast<uint8_t*>(const_cast<void*>(v_scales));
    a.cos_sin = reinterpret_cast<const float2*>(cos_sin);
    a.pos = pos;
    a.stride_b = strides[0]; a.stride_t = strides[1]; a.stride_h = strides[2];
    a.s_max = s_max; a.pos0 = pos0;
    a.seq = static_cast<int32_t>(seq); a.n_kv_heads = n_kv_heads; a.head_dim = head_dim; a.chunks = head_dim / 8;
    return a;
}

static dim3 mx_rows_grid(int64_t seq, int32_t chunks, int unroll, int32_t batch, int32_t n_kv_heads)
{
    const int64_t per_block = kMxThreads * unroll;
    return dim3(static_cast<unsigned>((seq * chunks + per_block - 1) / per_block), static_cast<unsigned>(batch),
                static_cast<unsigned>(2 * n_kv_heads));
}

template <typename TABLE>
static int mx_write_launch(const MxRowsArgs& a, const TABLE& t, dim3 grid, int dtype, int format, hipStream_t stream)
{
    auto go = [&](auto fmt, auto bf16) {
        constexpr int F = decltype(fmt)::value;
        constexpr bool B = decltype(bf16)::value;
        if (a.cos_sin) civic::launch(kv_write_mx_kernel<F, B, true, TABLE>, grid, dim3(kMxThreads), 0, stream, a, t);
        else civic::launch(kv_write_mx_kernel<F, B, false, TABLE>, grid, dim3(kMxThreads), 0, stream, a, t);
    };
    using std::integral_constant; using std::true_type; using std::false_type;
    if (format == CIVIC_MXFP4) { if (dtype == CIVIC_BF16) go(integral_constant<int, 4>{}, true_type{}); else go(integral_constant<int, 4>{}, false_type{}); }
    else if (dtype == CIVIC_BF16) go(integral_constant<int, 8>{}, true_type{});
    else go(integral_constant<int, 8>{}, false_type{});
    return check_launch();
}

}  // namespace civic

extern "C" int civic_kv_write_mx(const void* k, const void* v, const int64_t* kv_strides, int dtype, const float* cos_sin, int format,
                                 void* k_codes, void* k_scales, void* v_codes, void* v_scales, int32_t batch, int32_t seq,
                                 int32_t n_kv_heads, int32_t head_dim, int64_t s_max, int64_t pos0, const int32_t* pos, void* stream)
{
    using namespace civic;
    const bool any = batch > 0 && seq > 0;
    const int rc = mx_rows_check(k, v, kv_strides, dtype, format, k_codes, k_scales, v_codes, v_scales, batch, seq, any, n_kv_heads, head_dim,
                                 s_max, pos0, pos, false);
    if (rc != CIVIC_OK) return rc;
    if (!aligned16(cos_sin)) return CIVIC_ERR_INVALID_ARG;
    if (!any) return CIVIC_OK;
    MxRowsArgs a = mx_rows_args(kv_strides, cos_sin, k_codes, k_scales, v_codes, v_scales, seq, n_kv_heads, head_dim, s_max, pos0, pos);
    a.src[0] = k; a.src[1] = v;
    return mx_write_launch(a, MxNoTable{}, mx_rows_grid(seq, a.chunks, mx_write_unroll(cos_sin != nullptr), batch, n_kv_heads), dtype, format, static_cast<hipStream_t>(stream));
}

extern "C" int civic_kv_write_mx_ragged(const void* k, const void* v, const int64_t* kv_strides, int dtype, const float* cos_sin, int format,
                                        void* k_codes, void* k_scales, void* v_codes, void* v_scales, int32_t batch,
                                        const int64_t* row_offsets, int32_t n_kv_heads, int32_t head_dim, int64_t s_max, int64_t pos0,
                                        const int32_t* pos, void* stream)
{
    using namespace civic;
    if (batch < 0 || !row_offsets || row_offsets[0] != 0) return CIVIC_ERR_INVALID_ARG;
    int64_t longest = 0;
    for (int32_t b = 0; b < batch; ++b) {
        const int64_t n = row_offsets[b + 1] - row_offsets[b];
        if (n < 0) return CIVIC_ERR_INVALID_ARG;
        if (n > longest) longest = n;
    }
    const bool any = longest > 0;
    const int rc = mx_rows_check(k, v, kv_strides, dtype, format, k_codes, k_scales, v_codes, v_scales, batch, longest, any, n_kv_heads, head_dim,
                                 s_max, pos0, pos, true);
    if (rc != CIVIC_OK) return rc;
    if (!aligned16(cos_sin)) return CIVIC_ERR_INVALID_ARG;
    if (row_offsets[batch] > INT32_MAX) return CIVIC_ERR_UNSUPPORTED;
    if (!any) return CIVIC_OK;
    for (int32_t b0 = 0; b0 < batch; b0 += kMxRaggedItems) {
        const int32_t n = batch - b0 < kMxRaggedItems ? batch - b0 : kMxRaggedItems;
        MxTable t;
        int64_t most = 0;
        for (int32_t i = 0; i <= n; ++i) {
            t.row[i] = static_cast<int32_t>(row_offsets[b0 + i]);
            if (i && row_offsets[b0 + i] - row_offsets[b0 + i - 1] > most) most = row_offsets[b0 + i] - row_offsets[b0 + i - 1];
        }
        for (int32_t i = n + 1; i <= kMxRaggedItems; ++i) t.row[i] = t.row[n];
        if (!most) continue;
        MxRowsArgs a = mx_rows_args(kv_strides, cos_sin, k_codes, k_scales, v_codes, v_scales, most, n_kv_heads, head_dim, s_max, pos0, pos);
        a.src[0] = k; a.src[1] = v; a.batch0 = b0;
        const int e = mx_write_launch(a, t, mx_rows_grid(most, a.chunks, mx_write_unroll(cos_sin != nullptr), n, n_kv_heads), dtype, format, static_cast<hipStream_t>(stream));
        if (e != CIVIC_OK) return e;
    }
    return CIVIC_OK;
}

extern "C" int civic_kv_read_mx(const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales, int format, void* k, void* v,
                                const int64_t* kv_strides, int dtype, int32_t batch, int32_t seq, int32_t n_kv_heads, int32_t head_dim,
                                int64_t s_max, int64_t pos0, const int32_t* pos, void* stream)
{
    using namespace civic;
    const bool any = batch > 0 && seq > 0;
    const int rc = mx_rows_check(k, v, kv_strides, dtype, format, k_codes, k_scales, v_codes, v_scales, batch, seq, any, n_kv_heads, head_dim,
                                 s_max, pos0, pos, false);
    if (rc != CIVIC_OK) return rc;
    if (!any) return CIVIC_OK;
    MxRowsArgs a = mx_rows_args(kv_strides, nullptr, k_codes, k_scales, v_codes, v_scales, seq, n_kv_heads, head_dim, s_max, pos0, pos);
    a.dst[0] = k; a.dst[1] = v;
    if (dtype == CIVIC_F32) a.chunks = head_dim / 4;
    const dim3 grid = mx_rows_grid(seq, a.chunks, kMxUnroll, batch, n_kv_heads);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (format == CIVIC_MXFP4) {
        if (dtype == CIVIC_BF16) civic::launch((kv_read_mx_kernel<4, true>), grid, dim3(kMxThreads), 0, s, a);
        else civic::launch((kv_read_mx_kernel<4, false>), grid, dim3(kMxThreads), 0, s, a);
    } else {
        if (dtype == CIVIC_BF16) civic::launch((kv_read_mx_kernel<8, true>), grid, dim3(kMxThreads), 0, s, a);
        else civic::launch((kv_read_mx_kernel<8, false>), grid, dim3(kMxThreads), 0, s, a);
    }
    return check_launch();
}
