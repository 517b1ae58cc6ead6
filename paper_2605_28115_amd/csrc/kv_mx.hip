// civic_kv_write_mx, civic_kv_write_mx_ragged, civic_kv_read_mx: cache rows in 8 or 4 bits (OCP microscaling), written from rows of
// the inputs' type and read back into them.  HBM-bound both ways: every element is met once.
//
// Blocks of 32 channels of a head row share a scale 2^e.  With the block's largest magnitude amax, e is the least integer for which
// amax <= 7 * 2^e (e2m1, whose codes end at 6 and round down from 7) or 464 * 2^e (e4m3: 448), so that no element is off by more than
// half a step.  In amax's bits, 7 = 1.75 * 2^2: the exponent field less 2, and one more where the mantissa is above 0.75 - a carry out
// of the mantissa once 2^21 - 1 is added (464 = 1.8125 * 2^8: 0x17FFFF).  x * 2^-e is exact and rounded once, by the conversion.
//
// A thread has 8 channels of a token and goes through the heads (those of its workgroup's slice), four threads a block: the largest
// magnitude meets in two exchanges of neighbouring lanes.  Token, cache row and the rotation's (cos, sin) are the same for all heads:
// 4 x 938 rows, 8 heads of 128 in bf16, rotated, to 4 bits 7.2 us (9.6 with a head a workgroup); 16 x 4001 rows of fp32 to 8 bits 128 us, 5.1
// TB/s, and back 108, 6.1; 64 x 3550 rows of 4 bits to bf16 207 us, 5.7 TB/s.
#include "mx_device.h"

namespace civic {

constexpr int kMxThreads = 256;
constexpr int kMxUnroll = 4;                                  // heads in flight per thread
constexpr int kMxRaggedItems = 64;                            // samples of one ragged launch
// A workgroup has four tokens at least, and a launch fewer than 2^32 threads along an axis.
constexpr int64_t kMxMaxTokens = int64_t{1} << 25;

struct MxRowsArgs {
    const void* src[2];                                       // rows of the inputs' type (write: read from; read: see dst)
    void* dst[2];
    uint8_t* codes[2];
    uint8_t* scales[2];
    const float2* cos_sin;                                    // or null
    const int32_t* pos;                                       // per sample, or null
    int64_t stride_b, stride_t, stride_h;                     // elements
    int64_t s_max, pos0;
    int32_t seq, n_kv_heads, head_dim;
    int32_t chunks, tokens, slice;                            // chunks of a head row, one a thread; tokens of a workgroup; heads of a slice
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

// 8 fp32 values over the scale as codes, rounded to nearest even (e2m1 saturating).
template <int FMT>
__device__ __forceinline__ void mx_convert(const float (&x)[8], float scale, uint32_t (&w)[FMT / 4])
{
    if constexpr (FMT == 4) {
        w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], scale, 0);
        w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], x[2], x[3], scale, 1);
        w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], x[4], x[5], scale, 2);
        w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], x[6], x[7], scale, 3);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            mx_i16x2 v = {0, 0};
            v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, x[4 * i], x[4 * i + 1], scale, false);
            v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, x[4 * i + 2], x[4 * i + 3], scale, true);
            w[i] = __builtin_bit_cast(uint32_t, v);
        }
    }
}

// 8 channels as they lie, and as fp32.
template <bool BF16>
struct MxChunk {
    u32x4 w[BF16 ? 1 : 2];
    // The bits of the largest magnitude, as an fp32 number's.
    __device__ __forceinline__ uint32_t largest() const
    {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        if constexpr (BF16) {
            u16x2 m = {0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t pair = w[0][i] & 0x7FFF7FFFu;
                m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, pair));
            }
            return max(static_cast<uint32_t>(m[0]), static_cast<uint32_t>(m[1])) << 16;
        } else {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t bits = w[BF16 ? 0 : i / 4][i % 4];
                m = max(m, bits & 0x7FFFFFFFu);
            }
            return m;
        }
    }
    // x rounded to the type, in place of the chunk.
    __device__ __forceinline__ void narrow(const float (&x)[8])
    {
        if constexpr (BF16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const mx_bf16x2 p = {static_cast<__bf16>(x[2 * i]), static_cast<__bf16>(x[2 * i + 1])};
                w[0][i] = __builtin_bit_cast(uint32_t, p);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[BF16 ? 0 : i / 4][i % 4] = __float_as_uint(x[i]);
        }
    }
    // mx_convert of bf16 pairs.
    template <int FMT>
    __device__ __forceinline__ void convert(float scale, uint32_t (&c)[FMT / 4]) const
    {
        const uint32_t w0 = w[0][0], w1 = w[0][1], w2 = w[0][2], w3 = w[0][3];
        const mx_bf16x2 p0 = __builtin_bit_cast(mx_bf16x2, w0), p1 = __builtin_bit_cast(mx_bf16x2, w1), p2 = __builtin_bit_cast(mx_bf16x2, w2),
                        p3 = __builtin_bit_cast(mx_bf16x2, w3);
        if constexpr (FMT == 4) {
            c[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, p0, scale, 0);
            c[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c[0], p1, scale, 1);
            c[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c[0], p2, scale, 2);
            c[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c[0], p3, scale, 3);
        } else {
            mx_i16x2 v = {0, 0};
            v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, p0, scale, false);
            v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, p1, scale, true);
            c[0] = __builtin_bit_cast(uint32_t, v);
            v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, p2, scale, false);
            v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, p3, scale, true);
            c[1] = __builtin_bit_cast(uint32_t, v);
        }
    }
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

// grid: (tiles of tokens, samples, 2 * slice of heads + (K or V))
template <int FMT, bool BF16, bool ROPE, typename TABLE>
__global__ __launch_bounds__(kMxThreads) void kv_write_mx_kernel(MxRowsArgs a, TABLE t)
{
    constexpr bool RAGGED = std::is_same<TABLE, MxTable>::value;
    constexpr int ESZ = BF16 ? 2 : 4;
    constexpr uint32_t CARRY = FMT == 4 ? 0x1FFFFFu : 0x17FFFFu, BELOW = FMT == 4 ? 2u : 8u, LAST = FMT == 4 ? 252u : 246u;
    const int which = blockIdx.z & 1, b = blockIdx.y;
    const int g0 = (blockIdx.z >> 1) * a.slice, g1 = min(g0 + a.slice, a.n_kv_heads);
    int64_t token0 = 0;
    int seq = a.seq;
    const char* src = static_cast<const char*>(a.src[which]);
    if constexpr (RAGGED) { token0 = t.row[b]; seq = t.row[b + 1] - t.row[b]; }
    else src += b * a.stride_b * ESZ;
    const int in_tile = threadIdx.x / a.chunks, chunk = threadIdx.x - in_tile * a.chunks, tok = blockIdx.x * a.tokens + in_tile;
    // (a block's four threads stay or leave together: chunks is a multiple of four)
    if (in_tile >= a.tokens || tok >= seq) return;
    const int64_t row = a.pos0 + (a.pos ? a.pos[a.batch0 + b] : 0) + tok;
    if (row < 0 || row >= a.s_max) return;
    const int64_t code_bytes = a.head_dim * FMT / 8;
    const int blocks = a.head_dim / kMxBlock, half = a.head_dim / 2, ch = chunk * 8;
    const bool low = ch < half;
    src += ((token0 + tok) * a.stride_t + ch) * ESZ;
    const int64_t to_other = static_cast<int64_t>(low ? half : -half) * ESZ;
    const int64_t cache_row = (static_cast<int64_t>(a.batch0 + b) * a.n_kv_heads) * a.s_max + row;

    const bool turns = ROPE && which == 0;
    float4 cs[4];
    if constexpr (ROPE) {
        if (turns) {                                          // K: pair (i, i + d / 2)
            const int64_t at = RAGGED ? token0 + tok : static_cast<int64_t>(b) * a.seq + tok;
            const float4* const table = reinterpret_cast<const float4*>(a.cos_sin + at * half + (low ? ch : ch - half));
#pragma unroll
            for (int i = 0; i < 4; ++i) cs[i] = table[i];
        }
    }
#pragma unroll 1
    for (int g = g0; g < g1; g += kMxUnroll) {
        MxChunk<BF16> own[kMxUnroll], other[ROPE ? kMxUnroll : 1];
#pragma unroll
        for (int u = 0; u < kMxUnroll; ++u)
            if (g + u < g1) {
                const char* const from = src + (g + u) * a.stride_h * ESZ;
                own[u].load(from);
                if constexpr (ROPE) if (turns) other[u].load(from + to_other);
            }
#pragma unroll
        for (int u = 0; u < kMxUnroll; ++u) {
            if (g + u >= g1) break;
            // bf16 stays packed: magnitudes are compared as pairs of whole numbers, and the conversions take pairs
            float x[8];
            if constexpr (ROPE) {
                if (turns) {
                    // own * c -+ other * s, as rope_pair rounds it
                    const uint32_t sign = low ? 0x80000000u : 0u;
                    float y[8];
                    own[u].widen(x);
                    other[u].widen(y);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float c = i & 1 ? cs[i / 2].z : cs[i / 2].x, sn = i & 1 ? cs[i / 2].w : cs[i / 2].y;
                        x[i] = __builtin_fmaf(x[i], c, __uint_as_float(__float_as_uint(y[i] * sn) ^ sign));
                    }
                    own[u].narrow(x);
                }
            }
            const uint32_t amax = max_of_quad(own[u].largest());
            const uint32_t up = (amax + CARRY) >> 23;
            const uint32_t s = min(max(up, 27u + BELOW) - BELOW, LAST);
            const bool odd = amax >= 0x7F800000u;             // an infinity or a NaN: the block reads back as NaN
            const float scale = __uint_as_float(s << 23);
            uint32_t w[FMT / 4];
            if (BF16 && (FMT == 4 || s != LAST)) {
                own[u].template convert<FMT>(scale, w);
            } else {
                own[u].widen(x);
                if constexpr (FMT == 8) {
                    // only where the scale is the last one can a magnitude be above 464 times it: held at 448
                    const float most = __uint_as_float(0x7F600000u);   // 448 * 2^119
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = fminf(fmaxf(x[i], -most), most);
                }
                mx_convert<FMT>(x, scale, w);
            }
            const int64_t at = cache_row + (g + u) * a.s_max;
            uint8_t* const dst = a.codes[which] + at * code_bytes + chunk * FMT;
            if constexpr (FMT == 4) *reinterpret_cast<uint32_t*>(dst) = odd ? 0u : w[0];
            else *reinterpret_cast<u32x2*>(dst) = u32x2{odd ? 0u : w[0], odd ? 0u : w[1]};
            if ((chunk & 3) == 0) a.scales[which][at * blocks + chunk / 4] = static_cast<uint8_t>(odd ? 255u : s);
        }
    }
}

// grid as above.  A thread writes 16 bytes, 8 channels of bf16 or 4 of fp32, so that a wavefront's stores are whole rows (32 bytes a thread
// in two stores: 16 x 4001 rows of 8 bits to fp32 316 us, so 152, and 108 through the heads).
template <int FMT, bool BF16>
__global__ __launch_bounds__(kMxThreads) void kv_read_mx_kernel(MxRowsArgs a)
{
    constexpr int ESZ = BF16 ? 2 : 4, CH = 16 / ESZ, BYTES = CH * FMT / 8;
    const int which = blockIdx.z & 1, b = blockIdx.y;
    const int g0 = (blockIdx.z >> 1) * a.slice, g1 = min(g0 + a.slice, a.n_kv_heads);
    const int in_tile = threadIdx.x / a.chunks, chunk = threadIdx.x - in_tile * a.chunks, tok = blockIdx.x * a.tokens + in_tile;
    if (in_tile >= a.tokens || tok >= a.seq) return;
    const int64_t row = a.pos0 + (a.pos ? a.pos[b] : 0) + tok;
    if (row < 0 || row >= a.s_max) return;
    const int64_t code_bytes = a.head_dim * FMT / 8;
    const int blocks = a.head_dim / kMxBlock;
    const int64_t cache_row = (static_cast<int64_t>(b) * a.n_kv_heads) * a.s_max + row;
    const uint8_t* const codes = a.codes[which] + cache_row * code_bytes + chunk * BYTES;
    const uint8_t* const scales = a.scales[which] + cache_row * blocks + chunk * CH / kMxBlock;
    char* const dst = static_cast<char*>(a.dst[which]) + (b * a.stride_b + tok * a.stride_t + chunk * CH) * ESZ;
#pragma unroll 1
    for (int g = g0; g < g1; g += kMxUnroll) {
        uint32_t w[kMxUnroll][2], s[kMxUnroll];
#pragma unroll
        for (int u = 0; u < kMxUnroll; ++u) {
            if (g + u >= g1) break;
            const uint8_t* const src = codes + (g + u) * a.s_max * code_bytes;
            if constexpr (BYTES == 2) w[u][0] = load_streaming(reinterpret_cast<const uint16_t*>(src));
            else if constexpr (BYTES == 4) w[u][0] = load_streaming(reinterpret_cast<const uint32_t*>(src));
            else {
                const u32x2 v = load_streaming(reinterpret_cast<const u32x2*>(src));
                w[u][0] = v[0]; w[u][1] = v[1];
            }
            s[u] = scales[(g + u) * a.s_max * blocks];
        }
#pragma unroll
        for (int u = 0; u < kMxUnroll; ++u) {
            if (g + u >= g1) break;
            const float scale = __uint_as_float(s[u] << 23);
            uint32_t p[CH / 2];
#pragma unroll
            for (int i = 0; i < CH / 2; ++i) p[i] = mx_pair_bf16<FMT>(w[u], i, scale);
            u32x4* const out = reinterpret_cast<u32x4*>(dst + (g + u) * a.stride_h * ESZ);
            if constexpr (BF16) store_streaming(out, u32x4{p[0], p[1], p[2], p[3]});
            else store_streaming(out, u32x4{p[0] << 16, p[0] & 0xFFFF0000u, p[1] << 16, p[1] & 0xFFFF0000u});   // values that bf16 holds, widened
        }
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
    if (head_dim > CIVIC_MAX_HEAD_DIM || batch > 65535 || n_kv_heads > 32767 || s_max > kMxMaxRows || seq > kMxMaxTokens) return CIVIC_ERR_UNSUPPORTED;
    return CIVIC_OK;
}

// Threads, workgroups and slices of the heads for chunks of `channels`: all heads in a workgroup where the tokens fill the chip four times.
static dim3 mx_rows_grid(MxRowsArgs* a, int32_t channels, int32_t batch)
{
    a->chunks = a->head_dim / channels;
    a->tokens = kMxThreads / a->chunks;
    const int64_t tiles = (static_cast<int64_t>(a->seq) + a->tokens - 1) / a->tokens, units = 2 * tiles * batch;
    int64_t slices = units >= 1024 ? 1 : 1024 / units;
    if (slices > a->n_kv_heads) slices = a->n_kv_heads;
    a->slice = static_cast<int32_t>((a->n_kv_heads + slices - 1) / slices);
    slices = (a->n_kv_heads + a->slice - 1) / a->slice;
    return dim3(static_cast<unsigned>(tiles), static_cast<unsigned>(batch), static_cast<unsigned>(2 * slices));
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
    a.seq = static_cast<int32_t>(seq); a.n_kv_heads = n_kv_heads; a.head_dim = head_dim;
    return a;
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
    const dim3 grid = mx_rows_grid(&a, 8, batch);
    return mx_write_launch(a, MxNoTable{}, grid, dtype, format, static_cast<hipStream_t>(stream));
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
        const dim3 grid = mx_rows_grid(&a, 8, n);
        const int e = mx_write_launch(a, t, grid, dtype, format, static_cast<hipStream_t>(stream));
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
    if (!mx_rows_apart(kv_strides, batch, seq, n_kv_heads, head_dim)) return CIVIC_ERR_INVALID_ARG;
    MxRowsArgs a = mx_rows_args(kv_strides, nullptr, k_codes, k_scales, v_codes, v_scales, seq, n_kv_heads, head_dim, s_max, pos0, pos);
    a.dst[0] = k; a.dst[1] = v;
    const dim3 grid = mx_rows_grid(&a, dtype == CIVIC_F32 ? 4 : 8, batch);
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
