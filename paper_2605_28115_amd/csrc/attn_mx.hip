// civic_decode_attn_mx, civic_prefill_attn_mx: attention of new tokens over a cache in 8 or 4 bits (OCP microscaling).
//
//   out[b, i, h, :] = sum_j softmax_j(scale * <q[b, i, h, :], K[b, g, j, :]>) V[b, g, j, :],   j < ctx[b] - (seq - 1 - i) when causal
//
// The queries of a KV head are its rows r = token * group + head of the group, 16 of them the columns of one MFMA tile.
//   - A wavefront takes 32 keys a step.  Codes become bf16 in registers, exactly (mx_device.h), so the products are those of a bf16
//     cache.  A lane holds a piece of a key's row that is contiguous in memory (a quarter of the channels), in the order that Q
//     shares; the two 16-key tiles hold keys 8 a + r and 8 a + 4 + r in row 4 a + r, so that a lane then owns the logits of 8
//     consecutive keys of one query row: the second operand of O^T += V^T P^T as it stands.
//   - Of V a lane reads a sixteenth of the channels of its 8 keys and gathers, for each channel, the 8 keys out of them (v_perm).
//   - Weights enter as sums of two bf16 terms (bf16 rows: 16 bits, an eighth of a thousandth of what the output's rounding leaves) or
//     three (fp32 rows: all 24), and so do fp32 queries.
//   - Each wavefront runs its own online softmax in fp32.
// Few rows: the wavefronts of a workgroup take turns over the keys and meet in LDS, and the context is split over workgroups, whose
// partial results a second launch joins.  Many rows: every wavefront has row tiles of its own.
#include <cmath>

#include "mx_device.h"

namespace civic {

struct MxAttnArgs {
    const void* q; void* out; float* ws;
    const uint8_t* kc; const uint8_t* ks; const uint8_t* vc; const uint8_t* vs;
    const int32_t* ctx;                                       // per sample, or null
    int64_t qs[3], os[3];                                     // element strides: batch, token, head
    int64_t s_max;
    int32_t batch, seq, n_q_heads, n_kv_heads, group, head_dim, rows;   // rows = seq * group
    int32_t n_ctx, splits, keys_per_split, causal;
    float scale_log2;
};

// A lane's maximum or sum over the four lanes of its column (lanes 16 apart), in all of them.
template <typename OP>
__device__ __forceinline__ float over_column(float v, OP op)
{
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(p[0]), __uint_as_float(p[1]));
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Two fp32 values as one word of bf16, and what that leaves of them.
__device__ __forceinline__ uint32_t bf16_pair(float a, float b)
{
    const mx_bf16x2 p = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
    return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ uint32_t bf16_pair_rest(float& a, float& b)
{
    const uint32_t w = bf16_pair(a, b);
    a -= __uint_as_float(w << 16);
    b -= __uint_as_float(w & 0xFFFF0000u);
    return w;
}

__device__ __forceinline__ int context_of(const MxAttnArgs& a, int b) { return a.ctx ? min(max(a.ctx[b], 0), a.n_ctx) : a.n_ctx; }
// Keys that row r sees.
__device__ __forceinline__ int row_limit(const MxAttnArgs& a, int ctx, int r) { return a.causal ? max(ctx - (a.seq - 1 - r / a.group), 0) : ctx; }

// DP: head_dim rounded up to 64, 128 or 256.  FULL: head_dim == DP.  R: row tiles of a wavefront.  BYROWS: the wavefronts have rows of
// their own (else keys of their own).
template <int FMT, bool BF16, int DP, bool FULL, int R, int WAVES, bool BYROWS>
__global__ __launch_bounds__(WAVES * kWave) void attn_mx_kernel(MxAttnArgs a)
{
    constexpr int NQ = BF16 ? 1 : 3, NP = BF16 ? 2 : 3;       // bf16 terms of a query, of a weight
    constexpr int CH = DP / 4, KT = CH / 8, KW = CH * FMT / 32;        // of K per lane: channels, MFMA steps, words
    constexpr int CV = DP / 16, VB = CV * FMT / 8, VW = VB < 4 ? 1 : VB / 4;   // of V per lane and key: channels, bytes, words
    constexpr int KB = CH > kMxBlock ? CH / kMxBlock : 1;              // blocks of K per lane
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, kq = lane >> 4;
    const int g = blockIdx.x % a.n_kv_heads, b = blockIdx.x / a.n_kv_heads;
    const int split = blockIdx.z;
    const int d = a.head_dim, nb = d / kMxBlock;
    const int row0 = (BYROWS ? blockIdx.y * WAVES + w : blockIdx.y) * (16 * R);
    const int ctx = context_of(a, b);
    const int n_splits = BYROWS ? 1 : max((ctx + a.keys_per_split - 1) / a.keys_per_split, 1);
    if (!BYROWS && split >= n_splits) return;
    if (BYROWS && row0 >= a.rows) return;
    const int k0 = split * a.keys_per_split;
    const int ctx1 = BYROWS ? ctx : min(k0 + a.keys_per_split, ctx);
    const int k1 = min(ctx1, row_limit(a, ctx, min(row0 + 16 * R, a.rows) - 1));   // (limits grow along the rows)

    int limit[R];                                             // keys that the lane's rows see
#pragma unroll
    for (int x = 0; x < R; ++x) limit[x] = row_limit(a, ctx, min(row0 + 16 * x + l16, a.rows - 1));
    const int least = row_limit(a, ctx, row0);                // keys that all rows see

    // Q^T: channels CH * kq + 8 t .. + 7 of row l16 of every tile
    mx_bf16x8 qf[R][NQ][KT];
#pragma unroll
    for (int x = 0; x < R; ++x) {
        const int r = min(row0 + 16 * x + l16, a.rows - 1);
        const int token = r / a.group, head = g * a.group + (r - token * a.group);
        const int64_t at = b * a.qs[0] + token * a.qs[1] + head * a.qs[2] + CH * kq;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            const bool there = FULL || CH * kq + 8 * t < d;
            if constexpr (BF16) {
                u32x4 v = u32x4{0u, 0u, 0u, 0u};
                if (there) v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q) + at + 8 * t);
                qf[x][0][t] = __builtin_bit_cast(mx_bf16x8, v);
            } else {
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = 0.f;
                if (there) {
                    const float4* src = reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + at + 8 * t);
                    const float4 u = src[0], v = src[1];
                    f[0] = u.x; f[1] = u.y; f[2] = u.z; f[3] = u.w; f[4] = v.x; f[5] = v.y; f[6] = v.z; f[7] = v.w;
                }
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    u32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = bf16_pair_rest(f[2 * e], f[2 * e + 1]);
                    qf[x][n][t] = __builtin_bit_cast(mx_bf16x8, v);
                }
            }
        }
    }

    const int64_t head_row = (static_cast<int64_t>(b) * a.n_kv_heads + g) * a.s_max;
    const uint32_t code_bytes = static_cast<uint32_t>(d) * FMT / 8;
    const uint8_t* const kc = a.kc + head_row * code_bytes;
    const uint8_t* const vc = a.vc + head_row * code_bytes;
    const uint8_t* const ks = a.ks + head_row * nb;
    const uint8_t* const vs = a.vs + head_row * nb;
    // a lane past the row reads the row's front; K's codes are made zero then, V's results are not written
    const uint32_t k_at = FULL || CH * kq < d ? CH * kq * FMT / 8 : 0, v_at = FULL || CV * l16 < d ? CV * l16 * FMT / 8 : 0;
    const uint32_t v_block = FULL || CV * l16 < d ? CV * l16 / kMxBlock : 0;

    mx_f32x4 o[R][CV];
    float m[R], l[R];                                         // l: of the lane's own keys
    uint32_t bad[R];                                          // blocks of V that hold a NaN in a row that the lane's row sees

    // The keys from `at` on (a multiple of 32: s_max is one too, so all 32 rows are there).
    // careful: V's NaN blocks are kept out of the products, and noted for the rows that see them.
    auto step = [&](int at, bool careful) __attribute__((always_inline)) {
        uint32_t kw[2][KW], vw[8][VW];
        float ksc[2][KB], vsc[8];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint32_t key = at + 8 * (l16 >> 2) + 4 * x + (l16 & 3);
            const uint8_t* src = kc + (key * code_bytes + k_at);
            if constexpr (KW == 2) {
                const u32x2 v = load_streaming(reinterpret_cast<const u32x2*>(src));
                kw[x][0] = v[0]; kw[x][1] = v[1];
            } else {
#pragma unroll
                for (int i = 0; i < KW / 4; ++i) {
                    const u32x4 v = load_streaming(reinterpret_cast<const u32x4*>(src) + i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) kw[x][4 * i + e] = v[e];
                }
            }
#pragma unroll
            for (int i = 0; i < KB; ++i) {
                const uint32_t blk = CH * kq / kMxBlock + i;
                ksc[x][i] = __uint_as_float(static_cast<uint32_t>(ks[key * nb + (FULL || blk < static_cast<uint32_t>(nb) ? blk : 0)]) << 23);
            }
            if constexpr (!FULL) {
#pragma unroll
                for (int i = 0; i < KB; ++i)
                    if (CH * kq + kMxBlock * i >= d) {
                        ksc[x][i] = 1.f;
#pragma unroll
                        for (int e = 0; e < KW / KB; ++e) kw[x][i * (KW / KB) + e] = 0u;
                    }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t key = at + 8 * kq + e;
            const uint8_t* src = vc + (key * code_bytes + v_at);
            if constexpr (VB == 2) vw[e][0] = *reinterpret_cast<const uint16_t*>(src);
            else {
#pragma unroll
                for (int i = 0; i < VW; ++i) vw[e][i] = reinterpret_cast<const uint32_t*>(src)[i];
            }
            vsc[e] = __uint_as_float(static_cast<uint32_t>(vs[key * nb + v_block]) << 23);
        }
        if (at + 32 > ctx1) {                                 // rows past the end hold anything
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + 8 * kq + e >= ctx1) {
                    vsc[e] = 1.f;
#pragma unroll
                    for (int i = 0; i < VW; ++i) vw[e][i] = 0u;
                }
        }
        if (careful) {
            for (int e = 0; e < 8; ++e) {
                const int key = at + 8 * kq + e;
                if (key >= ctx1) continue;
                for (int i = 0; i < nb; ++i)
                    if (vs[static_cast<uint32_t>(key) * nb + i] == 255) {
#pragma unroll
                        for (int x = 0; x < R; ++x)
                            if (key < limit[x]) bad[x] |= 1u << i;
                    }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (__float_as_uint(vsc[e]) == 0x7F800000u) {
                    vsc[e] = 1.f;
#pragma unroll
                    for (int i = 0; i < VW; ++i) vw[e][i] = 0u;
                }
        }

        mx_f32x4 s[R][2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
#pragma unroll
            for (int x = 0; x < R; ++x) s[x][y] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                u32x4 kf;
#pragma unroll
                for (int i = 0; i < 4; ++i) kf[i] = mx_pair_bf16<FMT>(kw[y], 4 * t + i, ksc[y][KB == 1 ? 0 : 8 * t / kMxBlock]);
#pragma unroll
                for (int x = 0; x < R; ++x)
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
                        s[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(mx_bf16x8, kf), qf[x][n][t], s[x][y], 0, 0, 0);
            }
        }
        u32x4 pf[R][NP];
#pragma unroll
        for (int x = 0; x < R; ++x) {
            float z[8], m_new = m[x];
            const int lim = min(limit[x], ctx1) - at - 8 * kq;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                z[e] = s[x][e >> 2][e & 3] * a.scale_log2;
                if (at + 32 > min(least, ctx1)) z[e] = e < lim ? z[e] : -INFINITY;
                m_new = fmaxf(m_new, z[e]);
            }
            m_new = over_column(m_new, [](float p, float q) { return fmaxf(p, q); });
            const float m_use = m_new == -INFINITY ? 0.f : m_new;
            if (__any(m_new != m[x])) {
                const float alpha = __builtin_amdgcn_exp2f(m[x] - m_use);
                l[x] *= alpha;
#pragma unroll
                for (int j = 0; j < CV; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[x][j][i] *= alpha;
                m[x] = m_new;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float p0 = __builtin_amdgcn_exp2f(z[2 * e] - m_use), p1 = __builtin_amdgcn_exp2f(z[2 * e + 1] - m_use);
                l[x] += p0 + p1;
#pragma unroll
                for (int n = 0; n < NP; ++n) pf[x][n][e] = bf16_pair_rest(p0, p1);
            }
        }
#pragma unroll
        for (int h = 0; h < CV / 2; ++h) {
            uint32_t c[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) c[e] = mx_pair_bf16<FMT>(vw[e], h, vsc[e]);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                u32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = __builtin_amdgcn_perm(c[2 * e + 1], c[2 * e], y ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int x = 0; x < R; ++x)
#pragma unroll
                    for (int n = 0; n < NP; ++n)
                        o[x][2 * h + y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(mx_bf16x8, v), __builtin_bit_cast(mx_bf16x8, pf[x][n]), o[x][2 * h + y], 0, 0, 0);
            }
        }
    };
    const int key_step = BYROWS ? 32 : 32 * WAVES, first = k0 + (BYROWS ? 0 : 32 * w);
    auto pass = [&](bool careful) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < R; ++x) {
            m[x] = -INFINITY; l[x] = 0.f; bad[x] = 0;
#pragma unroll
            for (int j = 0; j < CV; ++j) o[x][j] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll 1
        for (int at = first; at < k1; at += key_step) step(at, careful);
        float odd = 0.f;
#pragma unroll
        for (int x = 0; x < R; ++x)
#pragma unroll
            for (int j = 0; j < CV; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) odd = fmaf(o[x][j][i], 0.f, odd);
        return __any(odd != 0.f);
    };
    // A NaN of V has met weights of 0 (0 x NaN), the rows' that do not see it: once more, with NaN blocks apart.
#pragma unroll 1
    for (int careful = 0; careful < 2; ++careful)
        if (!pass(careful != 0)) break;
#pragma unroll
    for (int x = 0; x < R; ++x) {
        l[x] = over_column(l[x], [](float p, float q) { return p + q; });
        if (__any(bad[x] != 0)) {
            uint32_t all = bad[x];
            all |= __shfl_xor(all, 16, kWave);
            all |= __shfl_xor(all, 32, kWave);
#pragma unroll
            for (int j = 0; j < CV; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (all >> ((CV * (4 * kq + i) + j) / kMxBlock) & 1) o[x][j][i] = __builtin_nanf("");
        }
    }

    auto out_at = [&](int r) {
        const int token = r / a.group, head = g * a.group + (r - token * a.group);
        return b * a.os[0] + token * a.os[1] + head * a.os[2];
    };
    // register i of o[x][j]: channel CV (4 kq + i) + j of row l16 of tile x
    if constexpr (BYROWS) {
#pragma unroll
        for (int x = 0; x < R; ++x) {
            const int r = row0 + 16 * x + l16;
            if (r >= a.rows) continue;
            const float inv = l[x] == 0.f ? 0.f : 1.0f / l[x];
            const int64_t at = out_at(r);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int ch = CV * (4 * kq + i);
                if (!FULL && ch >= d) continue;
#pragma unroll
                for (int j = 0; j < CV; j += 4) {
                    const float v[4] = {o[x][j][i] * inv, o[x][j + 1][i] * inv, o[x][j + 2][i] * inv, o[x][j + 3][i] * inv};
                    if constexpr (BF16) *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + at + ch + j) = u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
                    else *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at + ch + j) = make_float4(v[0], v[1], v[2], v[3]);
                }
            }
        }
    } else {
        static_assert(BYROWS || R == 1, "one tile where the wavefronts share it");
        extern __shared__ __attribute__((aligned(16))) float mx_lds[];
        const int cols = min(16, a.rows - row0);
        float* const sm_o = mx_lds;                           // [wavefront][column][d], then maxima, then sums
        float* const sm_m = mx_lds + WAVES * cols * d;
        float* const sm_l = sm_m + WAVES * cols;
        if (l16 < cols) {
            if (kq == 0) { sm_m[w * cols + l16] = m[0]; sm_l[w * cols + l16] = l[0]; }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int ch = CV * (4 * kq + i);
                if (!FULL && ch >= d) continue;
#pragma unroll
                for (int j = 0; j < CV; j += 4)
                    *reinterpret_cast<float4*>(sm_o + (w * cols + l16) * d + ch + j) = make_float4(o[0][j][i], o[0][j + 1][i], o[0][j + 2][i], o[0][j + 3][i]);
            }
        }
        __syncthreads();
        const int half_d = d / 2;
        for (int n = tid; n < cols * half_d; n += WAVES * kWave) {
            const int c = n / half_d, ch = (n - c * half_d) * 2;
            float mx = sm_m[c];
#pragma unroll
            for (int x = 1; x < WAVES; ++x) mx = fmaxf(mx, sm_m[x * cols + c]);
            float o0 = 0.f, o1 = 0.f, lt = 0.f;
#pragma unroll
            for (int x = 0; x < WAVES; ++x) {                 // (a wavefront without a key: m = -inf, its sums 0 or a NaN's)
                const float mw = sm_m[x * cols + c], f = mw == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mw - mx);
                const float2 v = *reinterpret_cast<const float2*>(sm_o + (x * cols + c) * d + ch);
                o0 = fmaf(f, v.x, o0); o1 = fmaf(f, v.y, o1);
                lt = fmaf(f, sm_l[x * cols + c], lt);
            }
            const int r = row0 + c;
            if (n_splits == 1) {
                const float inv = lt == 0.f ? 0.f : 1.0f / lt;
                const int64_t at = out_at(r) + ch;
                if constexpr (BF16) *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + at) = bf16_pair(o0 * inv, o1 * inv);
                else *reinterpret_cast<float2*>(static_cast<float*>(a.out) + at) = make_float2(o0 * inv, o1 * inv);
            } else {
                float* dst = a.ws + ((static_cast<int64_t>(blockIdx.x) * a.rows + r) * a.splits + split) * (d + 2);
                if (ch == 0) *reinterpret_cast<float2*>(dst) = make_float2(mx, lt);
                *reinterpret_cast<float2*>(dst + 2 + ch) = make_float2(o0, o1);
            }
        }
    }
}

// Joins the splits of one row: out = sum_s w_s o_s / sum_s w_s l_s, w_s = 2^(m_s - max m).  grid: (sample and KV head, row)
constexpr int kMxMaxSplits = 256;
template <bool BF16>
__global__ __launch_bounds__(128) void attn_mx_merge_kernel(MxAttnArgs a)
{
    const int r = blockIdx.y, g = blockIdx.x % a.n_kv_heads, b = blockIdx.x / a.n_kv_heads;
    const int ctx = context_of(a, b);
    const int splits = (ctx + a.keys_per_split - 1) / a.keys_per_split;
    if (splits <= 1) return;                                  // the row has its result already
    const int d = a.head_dim;
    const float* src = a.ws + (static_cast<int64_t>(blockIdx.x) * a.rows + r) * a.splits * (d + 2);
    float mx = -INFINITY;
    for (int s = 0; s < splits; ++s) mx = fmaxf(mx, src[s * (d + 2)]);
    const int token = r / a.group, head = g * a.group + (r - token * a.group);
    const int64_t at = b * a.os[0] + token * a.os[1] + head * a.os[2];
    for (int ch = 2 * threadIdx.x; ch < d; ch += 256) {
        float o0 = 0.f, o1 = 0.f, lt = 0.f;
        for (int s = 0; s < splits; ++s) {
            const float* p = src + s * (d + 2);
            const float f = p[0] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(p[0] - mx);
            o0 = fmaf(f, p[2 + ch], o0); o1 = fmaf(f, p[3 + ch], o1);
            lt = fmaf(f, p[1], lt);
        }
        const float inv = lt == 0.f ? 0.f : 1.0f / lt;
        if constexpr (BF16) *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + at + ch) = bf16_pair(o0 * inv, o1 * inv);
        else *reinterpret_cast<float2*>(static_cast<float*>(a.out) + at + ch) = make_float2(o0 * inv, o1 * inv);
    }
}

constexpr int kMxWaves = 4;

struct MxAttnPlan {
    bool by_rows;
    int32_t row_blocks, splits, keys_per_split;
    size_t ws_bytes, lds_bytes;
};

static MxAttnPlan mx_attn_plan(int32_t batch, int64_t rows, int32_t n_kv_heads, int32_t head_dim, int64_t n_ctx)
{
    MxAttnPlan p{};
    const int64_t pairs = static_cast<int64_t>(batch) * n_kv_heads, tiles = (rows + 15) / 16;
    p.by_rows = tiles >= 4 && pairs * tiles >= 512;
    p.row_blocks = static_cast<int32_t>(p.by_rows ? (tiles + kMxWaves - 1) / kMxWaves : tiles);
    p.splits = 1;
    p.keys_per_split = static_cast<int32_t>((n_ctx + 31) / 32 * 32);
    if (!p.by_rows) {
        const int64_t units = pairs * p.row_blocks, step = 32 * kMxWaves;
        int64_t want = units > 0 ? (1024 + units - 1) / units : 1;
        const int64_t most = (n_ctx + step - 1) / step;
        if (want > most) want = most;
        if (want > kMxMaxSplits) want = kMxMaxSplits;
        if (want < 1) want = 1;
        const int64_t steps = (most + want - 1) / want;
        p.keys_per_split = static_cast<int32_t>((steps > 0 ? steps : 1) * step);
        p.splits = static_cast<int32_t>(n_ctx > 0 ? (n_ctx + p.keys_per_split - 1) / p.keys_per_split : 1);
        const int64_t cols = rows < 16 ? rows : 16;
        p.lds_bytes = sizeof(float) * kMxWaves * static_cast<size_t>(cols) * (head_dim + 2);
    }
    if (p.keys_per_split < 32) p.keys_per_split = 32;
    p.ws_bytes = p.splits > 1 ? sizeof(float) * static_cast<size_t>(pairs) * rows * p.splits * (head_dim + 2) : 0;
    return p;
}

static bool mx_attn_sizes_ok(int dtype, int format, int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t n_ctx)
{
    return dtype_size(dtype) && mx_format_ok(format) && batch >= 0 && seq >= 0 && n_q_heads > 0 && n_kv_heads > 0 && n_q_heads % n_kv_heads == 0
        && head_dim > 0 && head_dim % kMxBlock == 0 && n_ctx >= 0;
}

static bool mx_attn_covered(int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t s_max)
{
    const int64_t rows = static_cast<int64_t>(seq) * (n_q_heads / n_kv_heads);
    return head_dim <= CIVIC_MAX_HEAD_DIM && batch <= 65535 && static_cast<int64_t>(batch) * n_kv_heads <= INT32_MAX && s_max <= kMxMaxRows
        && rows <= 16 * 65535;
}

template <int FMT, bool BF16, int DP, bool FULL>
static int mx_attn_launch(const MxAttnArgs& a, const MxAttnPlan& p, hipStream_t stream)
{
    const dim3 grid(static_cast<unsigned>(a.batch * a.n_kv_heads), static_cast<unsigned>(p.row_blocks), static_cast<unsigned>(p.splits));
    if (p.by_rows) {
        civic::launch(attn_mx_kernel<FMT, BF16, DP, FULL, 1, kMxWaves, true>, grid, dim3(kMxWaves * kWave), 0, stream, a);
    } else {
        if (p.lds_bytes > 65536) {
            static std::atomic<uint64_t> done{0};
            const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(&attn_mx_kernel<FMT, BF16, DP, FULL, 1, kMxWaves, false>), 160 * 1024, &done);
            if (rc != CIVIC_OK) return rc;
        }
        civic::launch(attn_mx_kernel<FMT, BF16, DP, FULL, 1, kMxWaves, false>, grid, dim3(kMxWaves * kWave), p.lds_bytes, stream, a);
    }
    if (p.splits > 1) {
        const int rc = check_launch();
        if (rc != CIVIC_OK) return rc;
        civic::launch(attn_mx_merge_kernel<BF16>, dim3(static_cast<unsigned>(a.batch * a.n_kv_heads), static_cast<unsigned>(a.rows)), dim3(128), 0, stream, a);
    }
    return check_launch();
}

template <int FMT, bool BF16>
static int mx_attn_launch_dim(const MxAttnArgs& a, const MxAttnPlan& p, hipStream_t s)
{
    const int d = a.head_dim;
    if (d == 64) return mx_attn_launch<FMT, BF16, 64, true>(a, p, s);
    if (d == 128) return mx_attn_launch<FMT, BF16, 128, true>(a, p, s);
    if (d == 256) return mx_attn_launch<FMT, BF16, 256, true>(a, p, s);
    if (d < 64) return mx_attn_launch<FMT, BF16, 64, false>(a, p, s);
    if (d < 128) return mx_attn_launch<FMT, BF16, 128, false>(a, p, s);
    return mx_attn_launch<FMT, BF16, 256, false>(a, p, s);
}

static int mx_attn(const void* q, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales, void* out, int dtype,
                   int format, int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const int64_t* qs,
                   const int64_t* os, int64_t s_max, int64_t n_ctx, const int32_t* ctx, int32_t causal, float softmax_scale, void* workspace,
                   size_t workspace_bytes, void* stream)
{
    if (!mx_attn_sizes_ok(dtype, format, batch, seq, n_q_heads, n_kv_heads, head_dim, n_ctx) || !qs || !os) return CIVIC_ERR_INVALID_ARG;
    if (s_max < 0 || s_max % kMxBlock || n_ctx > s_max || !std::isfinite(softmax_scale)) return CIVIC_ERR_INVALID_ARG;
    const int esz = dtype_size(dtype);
    const bool any = batch > 0 && seq > 0;
    if (any && (!q || !out)) return CIVIC_ERR_INVALID_ARG;
    if (any && n_ctx > 0 && (!k_codes || !k_scales || !v_codes || !v_scales)) return CIVIC_ERR_INVALID_ARG;
    for (const void* p : {q, k_codes, k_scales, v_codes, v_scales, static_cast<const void*>(out), static_cast<const void*>(workspace)})
        if (!aligned16(p)) return CIVIC_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(ctx) & 3u) return CIVIC_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i)
        if (qs[i] < 0 || os[i] < 0 || (qs[i] * esz) % 16 || (os[i] * esz) % 16) return CIVIC_ERR_INVALID_ARG;
    if (n_q_heads > 1 && (qs[2] < head_dim || os[2] < head_dim)) return CIVIC_ERR_INVALID_ARG;
    if (!mx_attn_covered(batch, seq, n_q_heads, n_kv_heads, head_dim, s_max)) return CIVIC_ERR_UNSUPPORTED;
    if (!any) return CIVIC_OK;
    MxAttnArgs a{};
    a.rows = seq * (n_q_heads / n_kv_heads);
    const MxAttnPlan p = mx_attn_plan(batch, a.rows, n_kv_heads, head_dim, n_ctx);
    if (p.ws_bytes && (!workspace || workspace_bytes < p.ws_bytes)) return CIVIC_ERR_WORKSPACE;
    a.q = q; a.out = out; a.ws = static_cast<float*>(workspace);
    a.kc = static_cast<const uint8_t*>(k_codes); a.ks = static_cast<const uint8_t*>(k_scales);
    a.vc = static_cast<const uint8_t*>(v_codes); a.vs = static_cast<const uint8_t*>(v_scales);
    a.ctx = ctx;
    for (int i = 0; i < 3; ++i) { a.qs[i] = qs[i]; a.os[i] = os[i]; }
    a.s_max = s_max; a.batch = batch; a.seq = seq; a.n_q_heads = n_q_heads; a.n_kv_heads = n_kv_heads; a.group = n_q_heads / n_kv_heads;
    a.head_dim = head_dim; a.n_ctx = static_cast<int32_t>(n_ctx); a.splits = p.splits; a.keys_per_split = p.keys_per_split; a.causal = causal != 0;
    const double scale = softmax_scale == 0.f ? 1.0 / std::sqrt(static_cast<double>(head_dim)) : softmax_scale;
    a.scale_log2 = static_cast<float>(scale * 1.4426950408889634);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (format == CIVIC_MXFP4) return dtype == CIVIC_BF16 ? mx_attn_launch_dim<4, true>(a, p, s) : mx_attn_launch_dim<4, false>(a, p, s);
    return dtype == CIVIC_BF16 ? mx_attn_launch_dim<8, true>(a, p, s) : mx_attn_launch_dim<8, false>(a, p, s);
}

}  // namespace civic

extern "C" size_t civic_attn_mx_workspace_bytes(int dtype, int format, int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads,
                                                int32_t head_dim, int64_t n_ctx)
{
    using namespace civic;
    if (!mx_attn_sizes_ok(dtype, format, batch, seq, n_q_heads, n_kv_heads, head_dim, n_ctx)
        || !mx_attn_covered(batch, seq, n_q_heads, n_kv_heads, head_dim, n_ctx) || batch == 0 || seq == 0) return 0;
    return mx_attn_plan(batch, static_cast<int64_t>(seq) * (n_q_heads / n_kv_heads), n_kv_heads, head_dim, n_ctx).ws_bytes;
}

extern "C" int civic_decode_attn_mx(const void* q, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales, void* out,
                                    int dtype, int format, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t s_max,
                                    int64_t n_ctx, const int32_t* ctx, float softmax_scale, void* workspace, size_t workspace_bytes, void* stream)
{
    const int64_t row = static_cast<int64_t>(n_q_heads) * head_dim;
    const int64_t strides[3] = {row, row, head_dim};
    return civic::mx_attn(q, k_codes, k_scales, v_codes, v_scales, out, dtype, format, batch, 1, n_q_heads, n_kv_heads, head_dim, strides, strides,
                          s_max, n_ctx, ctx, 0, softmax_scale, workspace, workspace_bytes, stream);
}

extern "C" int civic_prefill_attn_mx(const void* q, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales, void* out,
                                     int dtype, int format, int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                     const int64_t* q_strides, const int64_t* o_strides, int64_t s_max, int64_t n_ctx, const int32_t* ctx,
                                     int32_t causal, float softmax_scale, void* workspace, size_t workspace_bytes, void* stream)
{
    return civic::mx_attn(q, k_codes, k_scales, v_codes, v_scales, out, dtype, format, batch, seq, n_q_heads, n_kv_heads, head_dim, q_strides,
                          o_strides, s_max, n_ctx, ctx, causal, softmax_scale, workspace, workspace_bytes, stream);
}
