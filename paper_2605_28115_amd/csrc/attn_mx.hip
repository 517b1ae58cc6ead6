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
//   - Weights enter as sums of two bf16 terms (bf16 rows: 16 bits, 2^-16 against the output's rounding of 2^-8; memory hides the second
//     term's products) or three (fp32 rows: all 24 bits), and so do fp32 queries.
//   - Each wavefront runs its own online softmax in fp32.
// Up to 32 rows a KV head (attn_mx_kernel): bound by the cache's bytes.  The wavefronts of a workgroup take turns over the keys and meet in
// LDS; contexts are split over workgroups where there are few, and a second launch joins the splits.  8 x 65000 rows of 8 bits, 32 / 8 heads
// of 128: 163 us, 6.7 TB/s; 64 x 3584 rows of 4 bits 44 us, 5.6 TB/s (of 200 vector and 24 matrix instructions a step, half the vector
// units' time); 64 x 117..3584 33 us, of which 6 are a launch's beginning and end.
// More rows in bf16 (attn_mx_rows_kernel): bound by the products.  1024 tokens behind 9001 rows of 8 bits, 28 / 4 heads: 131 us back to back,
// 950 TFLOP/s (144 as a single launch under the profiler); 8 x 512 tokens over 2000 rows of 4 bits, 32 / 8 heads 122 to 127 us, 920 to 960.
#include <climits>
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
    float scale_log2, slack;                                  // |scale| * log2(e); logits by which m may be below the largest
    uint32_t q_sign;                                          // 0x80008000 where the scale is negative
};
// The workspace: of every (sample, KV head, row, split) head_dim unnormalised outputs, then of every one (m, sum).
__device__ __forceinline__ float* split_out(const MxAttnArgs& a, int64_t row) { return a.ws + row * a.splits * a.head_dim; }
__device__ __forceinline__ float2* split_state(const MxAttnArgs& a, int64_t row)
{
    const int64_t all = static_cast<int64_t>(a.batch) * a.n_kv_heads * a.rows * a.splits;
    return reinterpret_cast<float2*>(a.ws + all * a.head_dim) + row * a.splits;
}
// Weights are taken against a logit that is at most kMxSlack / log2(e) below the largest so far: results are scaled anew a few times in
// all, not whenever one of 16 or 32 rows meets a larger logit (with 1000 keys behind, every other step).
constexpr float kMxSlack = 6.f;
// A weight is exp2(fma(logit, scale, base)), base = -m * scale rounded: off by a factor that the keys taken against one m share, up to
// 2^(2^-24 |base|).  Parts of a row that were taken against different m (before and after a renewal, of other wavefronts, key groups or
// splits) have different ones, so what brings a part from m0 to m1 takes the roundings' difference along (from_to; without it rows with
// logits of 40000 were off by 1e-3).  Where base is beyond kMxFar the logits are taken from m first and base is 0.
constexpr float kMxFar = 65536.f;
// Nothing seen yet: 0, and weights of 2^-inf.
__device__ __forceinline__ float base_of(const MxAttnArgs& a, float m) { return m == -INFINITY ? 0.f : -m * a.scale_log2; }
__device__ __forceinline__ float base_rounding(const MxAttnArgs& a, float m)
{
    const float base = -m * a.scale_log2;
    return fabsf(base) > kMxFar ? 0.f : fmaf(m, a.scale_log2, base);   // (exact; nothing seen: beyond kMxFar)
}
// What sums taken against m0 are multiplied by to join those taken against m1.
__device__ __forceinline__ float from_to(const MxAttnArgs& a, float m0, float m1)
{
    return __builtin_amdgcn_exp2f(fmaf(m0 - m1, a.scale_log2, base_rounding(a, m1) - base_rounding(a, m0)));
}

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

// The same with the first 8 bits of each value as they are, so that a finite value's term is finite: three of them are all of an fp32 number.
__device__ __forceinline__ uint32_t bf16_pair_front(float& a, float& b)
{
    const uint32_t lo = __float_as_uint(a) & 0xFFFF0000u, hi = __float_as_uint(b) & 0xFFFF0000u;
    a -= __uint_as_float(lo);
    b -= __uint_as_float(hi);
    return lo >> 16 | hi;
}

__device__ __forceinline__ int context_of(const MxAttnArgs& a, int b) { return a.ctx ? min(max(a.ctx[b], 0), a.n_ctx) : a.n_ctx; }
// Keys that row r sees.
__device__ __forceinline__ int row_limit(const MxAttnArgs& a, int ctx, int r) { return a.causal ? max(ctx - (a.seq - 1 - r / a.group), 0) : ctx; }

// The blocks of V that are NaN in a key's row, if it is below `end`: the key to the first ones met (keys come in rising order).
template <int NB, bool FULL>
__device__ __forceinline__ void nan_blocks(const uint8_t* vs, int key, int end, int nb, int (&nan_at)[NB])
{
    uint8_t s[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) s[i] = key < end && (FULL || i < nb) ? vs[static_cast<int64_t>(key) * nb + i] : 0;
#pragma unroll
    for (int i = 0; i < NB; ++i)
        if (s[i] == 255) nan_at[i] = min(nan_at[i], key);
}

// 16 or 4 bytes per lane from global memory (scalar base, offset per lane) straight into LDS at lds + lane * size, lds the wavefront's.
// In assembly, because the compiler would wait for all of them ahead of any LDS read; who reads waits by count (wait_loads).  It counts
// no wait states into an asm statement either: m0 is read a state after it was written, and a base that a vector instruction wrote
// (v_readfirstlane) five later, which scalar_base sees to.  m0 is reserved, and nothing else here reads it.
template <int SIZE>
__device__ __forceinline__ void load_lds(const uint8_t* base, uint32_t offset, uint32_t lds)
{
    if constexpr (SIZE == 16) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" :: "s"(lds), "v"(offset), "s"(base) : "memory");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2 nt" :: "s"(lds), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ const uint8_t* scalar_base(const uint8_t* p)
{
    const uint64_t bits = reinterpret_cast<uint64_t>(p);
    const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(bits >> 32)));
    const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(bits)));
    uint64_t copy;
    asm("s_mov_b64 %0, %1" : "=s"(copy) : "s"(static_cast<uint64_t>(hi) << 32 | lo));   // a scalar instruction waits for the vector one
    return reinterpret_cast<const uint8_t*>(copy);
}
// Until at most N of the wavefront's loads are outstanding (they end in order).
template <int N>
__device__ __forceinline__ void wait_loads()
{
    static_assert(N >= 0 && N < 64, "a count of six bits");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
    asm volatile("" ::: "memory");
}

// A wavefront's ring in LDS: two steps of 32 keys, each K's codes, V's codes, K's scales, V's scales as they lie in the cache.  Rows of PC
// pieces of 16 bytes (of DP channels; a shorter row repeats its front), key 8 k + 4 x + r in place 16 x + 4 r + k, piece c in place
// c ^ (place * PC / 16): the 16 keys of an MFMA tile, and a piece of the keys 8 k + e of all k, are then on distinct banks.
template <int FMT, int DP>
struct MxRing {
    static constexpr int PC = DP * FMT / 128, CODES = 32 * PC * 16, SCALES = 256, STEP = 2 * CODES + 2 * SCALES, BYTES = 2 * STEP;
    static constexpr int LOADS = PC / 2 + 1;                  // of K, and of V, per step
    static constexpr int SHIFT = PC == 2 ? 3 : PC == 4 ? 2 : PC == 8 ? 1 : 0;
    static __device__ __forceinline__ int swizzle(int place) { return (place >> SHIFT) & (PC - 1); }
};

// Wavefronts of a SIMD that the registers are held to.  (In 4 bits and 128 channels 121 registers a lane and 37 KB of LDS a workgroup: four;
// codes held in registers over a step, instead of the ring, took 144 and left three, 58 us for 49 on 64 x 3584 rows.)
constexpr int mx_resident(int fmt, bool bf16, int dp, bool full, int r)
{
    if (dp == 64) return bf16 ? (r == 1 ? (full ? 4 : 3) : full ? 3 : 2) : full ? 3 : 2;
    if (dp == 128) return bf16 && r == 1 ? (fmt == 4 ? 4 : 2) : 2;
    return 1;
}

// LDS of a workgroup: the rings, or at the end the accumulators that are handed over (at most four of a taker at a time).
template <int FMT, int DP, int R, int WAVES>
constexpr int mx_attn_lds()
{
    const int acc = R * (DP / 16), share = acc >= WAVES ? acc / WAVES : 1, takers = acc / share, part = share > 4 ? 4 : share;
    const int rings = WAVES * MxRing<FMT, DP>::BYTES, states = takers * part * (WAVES - 1) * kWave * 16;
    return rings > states ? rings : states;
}

// DP: head_dim rounded up to 64, 128 or 256.  FULL: head_dim == DP.  R: row tiles of a workgroup.
template <int FMT, bool BF16, int DP, bool FULL, int R, int WAVES>
__global__ __launch_bounds__(WAVES * kWave, mx_resident(FMT, BF16, DP, FULL, R)) void attn_mx_kernel(MxAttnArgs a)
{
    using Ring = MxRing<FMT, DP>;
    constexpr int NQ = BF16 ? 1 : 3, NP = BF16 ? 2 : 3;       // bf16 terms of a query, of a weight
    constexpr int CH = DP / 4, KT = CH / 8, KW = CH * FMT / 32;       // of K per lane: channels, MFMA steps, words
    constexpr int CV = DP / 16, VB = CV * FMT / 8, VW = VB < 4 ? 1 : VB / 4;   // of V per lane and key: channels, bytes, words
    constexpr int KB = DP == 256 ? 2 : 1, NB = DP / kMxBlock;          // blocks of K per lane, and of a row
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, kq = lane >> 4;
    const int g = blockIdx.x % a.n_kv_heads, b = blockIdx.x / a.n_kv_heads;
    const int split = blockIdx.z;
    const int d = FULL ? DP : a.head_dim, nb = d / kMxBlock;
    const int row0 = blockIdx.y * (16 * R);
    const int ctx = context_of(a, b);
    const int n_splits = max((ctx + a.keys_per_split - 1) / a.keys_per_split, 1);
    if (split >= n_splits) return;
    const int k0 = split * a.keys_per_split;
    const int ctx1 = min(k0 + a.keys_per_split, ctx);
    const int k1 = min(ctx1, row_limit(a, ctx, min(row0 + 16 * R, a.rows) - 1));   // (limits grow along the rows)
    const int least = min(row_limit(a, ctx, row0), ctx1);     // keys that all rows see

    const int64_t head_row = (static_cast<int64_t>(b) * a.n_kv_heads + g) * a.s_max;
    const uint32_t code_bytes = static_cast<uint32_t>(d) * FMT / 8;
    const uint8_t* const kc = a.kc + head_row * code_bytes;
    const uint8_t* const vc = a.vc + head_row * code_bytes;
    const uint8_t* const ks = a.ks + head_row * nb;
    const uint8_t* const vs = a.vs + head_row * nb;
    extern __shared__ __attribute__((aligned(16))) uint8_t mx_lds[];
    uint8_t* const ring = mx_lds + w * Ring::BYTES;
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)ring)));
    // what the lane loads of a step: pieces 64 j + lane of the rings' places, and a word of scales
    uint32_t piece[Ring::PC / 2];
#pragma unroll
    for (int j = 0; j < Ring::PC / 2; ++j) {
        const int place = (64 * j + lane) / Ring::PC, c = ((64 * j + lane) & (Ring::PC - 1)) ^ Ring::swizzle(place);
        const uint32_t key = 8 * (place & 3) + 4 * (place >> 4) + ((place >> 2) & 3);
        piece[j] = key * code_bytes + (FULL || 16u * c < code_bytes ? 16 * c : 0);
    }
    const uint32_t scale_word = 4 * min(lane, 8 * nb - 1);
    // and reads of it
    const int k_place = 4 * (l16 & 3) + (l16 >> 2), k_piece = CH * FMT / 8 * kq / 16;
    const uint32_t k_read = (k_place * Ring::PC + (k_piece ^ Ring::swizzle(k_place))) * 16 + CH * FMT / 8 * kq % 16;
    const uint32_t k_block = FULL || CH * kq < d ? CH * kq / kMxBlock : 0, v_block = FULL || CV * l16 < d ? CV * l16 / kMxBlock : 0;
    const uint32_t k_scale = (8 * (l16 >> 2) + (l16 & 3)) * nb + k_block, v_scales = FULL ? 8 * kq * NB : 8 * kq * nb + v_block;
    uint32_t v_read[4];                                       // keys 8 kq + e, e % 4
#pragma unroll
    for (int r = 0; r < 4; ++r) v_read[r] = ((4 * r + kq) * Ring::PC + ((VB * l16 / 16) ^ Ring::swizzle(4 * r + kq))) * 16 + VB * l16 % 16;

    // Loads of the keys from `at` on (a multiple of 32: s_max is one too, so all 32 rows are there) into half `slot` of the ring.
    auto fetch = [&](int at, int slot, const uint8_t* codes, const uint8_t* scales, uint32_t codes_at, uint32_t scales_at) __attribute__((always_inline)) {
        const uint8_t* const cb = scalar_base(codes + static_cast<uint64_t>(at) * code_bytes);
        const uint32_t to = ring_at + slot * Ring::STEP;
#pragma unroll
        for (int j = 0; j < Ring::PC / 2; ++j) load_lds<16>(cb, piece[j], to + codes_at + j * 1024);
        load_lds<4>(scalar_base(scales + static_cast<uint64_t>(at) * nb), scale_word, to + scales_at);
    };
    auto fetch_k = [&](int at, int slot) __attribute__((always_inline)) { fetch(at, slot, kc, ks, 0, 2 * Ring::CODES); };
    auto fetch_v = [&](int at, int slot) __attribute__((always_inline)) { fetch(at, slot, vc, vs, Ring::CODES, 2 * Ring::CODES + Ring::SCALES); };

    const int first = k0 + 32 * w;
    constexpr int STEP = 32 * WAVES;
    const int steps = first < k1 ? (k1 - first + STEP - 1) / STEP : 0;
    auto start = [&]() __attribute__((always_inline)) {
        if (steps > 0) { fetch_k(first, 0); fetch_v(first, 0); }
        if (steps > 1) { fetch_k(first + STEP, 1); fetch_v(first + STEP, 1); }
    };
    start();

    int limit[R];                                             // keys that the lane's rows see
#pragma unroll
    for (int x = 0; x < R; ++x) limit[x] = min(row_limit(a, ctx, min(row0 + 16 * x + l16, a.rows - 1)), ctx1);
    // Q^T: channels CH * kq + 8 t .. + 7 of row l16 of every tile (negated if the scale is negative: logits enter by their size)
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
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] ^= a.q_sign;
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
                    for (int e = 0; e < 4; ++e) v[e] = bf16_pair_front(f[2 * e], f[2 * e + 1]) ^ a.q_sign;
                    qf[x][n][t] = __builtin_bit_cast(mx_bf16x8, v);
                }
            }
        }
    }

    mx_f32x4 o[R][CV];
    float m[R], l[R];                                         // m: what weights are taken against; l: of the lane's own keys

    // Step n, whose keys begin at `at`.  The ring's half is loaded anew as soon as it has been read, K's part after the logits and V's after
    // the products with V: up to two steps are in flight.  The loads in flight younger than those waited for are counted.
    // careful: V's NaN blocks are kept out of the products.
    auto step = [&](int n, int at, bool careful) __attribute__((always_inline)) {
        const uint8_t* const half = ring + (n & 1) * Ring::STEP;
        if (n + 1 < steps) wait_loads<3 * Ring::LOADS>();     // V, and the next step's
        else wait_loads<Ring::LOADS>();
        uint32_t kw[2][KW], ksc[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint32_t row = x * 16 * Ring::PC * 16;
            if constexpr (KW == 2) {
                const u32x2 v = *reinterpret_cast<const u32x2*>(half + k_read + row);
                kw[x][0] = v[0]; kw[x][1] = v[1];
            } else {
#pragma unroll
                for (int i = 0; i < KW / 4; ++i) {
                    const u32x4 v = *reinterpret_cast<const u32x4*>(half + (k_read ^ (16 * i)) + row);
#pragma unroll
                    for (int e = 0; e < 4; ++e) kw[x][4 * i + e] = v[e];
                }
            }
            const uint8_t* const sp = half + 2 * Ring::CODES + k_scale + x * 4 * nb;
            if constexpr (KB == 1) ksc[x] = *sp;
            else if constexpr (FULL) ksc[x] = *reinterpret_cast<const uint16_t*>(sp);
            else ksc[x] = sp[0] | static_cast<uint32_t>(sp[k_block + 1 < static_cast<uint32_t>(nb) ? 1 : 0]) << 8;
        }
        if constexpr (!FULL) {                                // channels past the row: zeros
#pragma unroll
            for (int i = 0; i < KB; ++i)
                if (CH * kq + kMxBlock * i >= d) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        ksc[x] = i ? (ksc[x] & 0xFF) | 0x7F00 : 0x7F7F;
#pragma unroll
                        for (int e = 0; e < KW / KB; ++e) kw[x][i * (KW / KB) + e] = 0u;
                    }
                }
        }
        mx_f32x4 z[R][2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
#pragma unroll
            for (int x = 0; x < R; ++x) z[x][y] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                const uint32_t byte = KB == 2 && t >= KT / 2 ? ksc[y] >> 8 : ksc[y];
                u32x4 kf;
#pragma unroll
                for (int i = 0; i < 4; ++i) kf[i] = mx_pair_bf16<FMT>(kw[y], 4 * t + i, __uint_as_float(byte << 23));
#pragma unroll
                for (int x = 0; x < R; ++x)
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
                        z[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(mx_bf16x8, kf), qf[x][n][t], z[x][y], 0, 0, 0);
            }
        }
        if (n + 2 < steps) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            fetch_k(at + 2 * STEP, n & 1);
        }

        u32x4 pf[R][NP];
#pragma unroll
        for (int x = 0; x < R; ++x) {
            if (at + 32 > least) {
                const int lim = limit[x] - at - 8 * kq;
#pragma unroll
                for (int e = 0; e < 8; ++e) z[x][e >> 2][e & 3] = e < lim ? z[x][e >> 2][e & 3] : -INFINITY;
            }
            float m_new = m[x];
#pragma unroll
            for (int e = 0; e < 8; e += 2) m_new = fmaxf(fmaxf(m_new, z[x][e >> 2][e & 3]), z[x][(e + 1) >> 2][(e + 1) & 3]);
            if (__any(m_new > m[x] + a.slack)) {
                m_new = over_column(m_new, [](float p, float q) { return fmaxf(p, q); });
                const float alpha = from_to(a, m[x], m_new == -INFINITY ? 0.f : m_new);
                l[x] *= alpha;
#pragma unroll
                for (int j = 0; j < CV; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[x][j][i] *= alpha;
                m[x] = m_new;
            }
            float base = base_of(a, m[x]);
            if (__builtin_expect(__any(fabsf(base) > kMxFar), 0)) {
                const bool far = fabsf(base) > kMxFar;
#pragma unroll
                for (int e = 0; e < 8; ++e) z[x][e >> 2][e & 3] -= far ? m[x] : 0.f;
                base = far ? 0.f : base;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float p0 = __builtin_amdgcn_exp2f(fmaf(z[x][(2 * e) >> 2][(2 * e) & 3], a.scale_log2, base));
                float p1 = __builtin_amdgcn_exp2f(fmaf(z[x][(2 * e + 1) >> 2][(2 * e + 1) & 3], a.scale_log2, base));
                l[x] += p0 + p1;
#pragma unroll
                for (int n = 0; n < NP; ++n) pf[x][n][e] = bf16_pair_rest(p0, p1);
            }
        }
        if (n + 2 < steps) wait_loads<3 * Ring::LOADS>();     // the next step's, and K of the one after it
        else if (n + 1 < steps) wait_loads<2 * Ring::LOADS>();
        else wait_loads<0>();
        uint32_t vw[8][VW], vsc[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint8_t* const src = half + Ring::CODES + v_read[e & 3] + (e >> 2) * 16 * Ring::PC * 16;
            if constexpr (VB == 2) vw[e][0] = *reinterpret_cast<const uint16_t*>(src);
            else if constexpr (VW == 1) vw[e][0] = *reinterpret_cast<const uint32_t*>(src);
            else if constexpr (VW == 2) {
                const u32x2 v = *reinterpret_cast<const u32x2*>(src);
                vw[e][0] = v[0]; vw[e][1] = v[1];
            } else {
                const u32x4 v = *reinterpret_cast<const u32x4*>(src);
#pragma unroll
                for (int i = 0; i < 4; ++i) vw[e][i] = v[i];
            }
        }
        // V's scales as the exponents of floats: turned there with whatever lies next to them, which the conversions do not look at
        const uint8_t* const sp = half + 2 * Ring::CODES + Ring::SCALES + v_scales;
        const uint32_t turn = (8 * (v_block & 3) + 9) & 31;
        if constexpr (!FULL) {
#pragma unroll
            for (int e = 0; e < 8; ++e) vsc[e] = static_cast<uint32_t>(sp[e * nb]) << 23;
        } else {
            uint32_t lies[2 * NB];
#pragma unroll
            for (int i = 0; i < NB / 2; ++i) {
                const u32x4 v = *(reinterpret_cast<const u32x4*>(sp) + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) lies[4 * i + e] = v[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                uint32_t x = lies[NB == 2 ? e >> 1 : NB == 4 ? e : 2 * e];
                if constexpr (NB == 8) {
                    const uint32_t high = lies[2 * e + 1];
                    x = v_block & 4 ? high : x;
                }
                vsc[e] = __builtin_amdgcn_alignbit(x, x, NB == 2 && (e & 1) ? turn + 16 : turn);
            }
        }
        if (at + 32 > ctx1) {                                 // rows past the end hold anything
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + 8 * kq + e >= ctx1) {
                    vsc[e] = 0x3F800000u;
#pragma unroll
                    for (int i = 0; i < VW; ++i) vw[e][i] = 0u;
                }
        }
        if (__builtin_expect(careful, 0)) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if ((vsc[e] & 0x7F800000u) == 0x7F800000u) {
                    vsc[e] = 0x3F800000u;
#pragma unroll
                    for (int i = 0; i < VW; ++i) vw[e][i] = 0u;
                }
        }
#pragma unroll
        for (int h = 0; h < CV / 2; ++h) {
            uint32_t cv[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) cv[e] = mx_pair_bf16<FMT>(vw[e], h, __uint_as_float(vsc[e]));
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                u32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = __builtin_amdgcn_perm(cv[2 * e + 1], cv[2 * e], y ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int x = 0; x < R; ++x)
#pragma unroll
                    for (int n = 0; n < NP; ++n)
                        o[x][2 * h + y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(mx_bf16x8, v), __builtin_bit_cast(mx_bf16x8, pf[x][n]), o[x][2 * h + y], 0, 0, 0);
            }
        }
        if (n + 2 < steps) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            fetch_v(at + 2 * STEP, n & 1);
        }
    };
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < R; ++x) {
            m[x] = -INFINITY; l[x] = 0.f;
#pragma unroll
            for (int j = 0; j < CV; ++j) o[x][j] = mx_f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    // A NaN of V meets weights of 0 (0 x NaN), the rows' that do not see it: where one shows, once more with NaN blocks apart.
    bool careful = false;
#pragma unroll 1
    for (;;) {
        clear();
#pragma unroll 1
        for (int n = 0; n < steps; ++n) step(n, first + n * STEP, careful);
        float odd = 0.f;
#pragma unroll
        for (int x = 0; x < R; ++x)
#pragma unroll
            for (int j = 0; j < CV; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) odd = fmaf(o[x][j][i], 0.f, odd);
        if (__builtin_expect(careful || !__any(odd != 0.f), 1)) break;
        careful = true;
        start();
    }
    if (__builtin_expect(careful, 0)) {
        // A row sees a NaN in block i exactly if it sees the first of the wavefront's keys that have one there.
        int nan_at[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) nan_at[i] = INT_MAX;
#pragma unroll 1
        for (int n = 0; n < steps; ++n) {
            const int key = first + n * STEP + (lane & 31);
            nan_blocks<NB, FULL>(vs, key, ctx1, nb, nan_at);
        }
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) nan_at[i] = min(nan_at[i], __shfl_xor(nan_at[i], off, kWave));
#pragma unroll
        for (int x = 0; x < R; ++x) {
            uint32_t bad = 0;
#pragma unroll
            for (int i = 0; i < NB; ++i) bad |= nan_at[i] < limit[x] ? 1u << i : 0u;
#pragma unroll
            for (int j = 0; j < CV; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (bad >> ((CV * (4 * kq + i) + j) / kMxBlock) & 1) o[x][j][i] = __builtin_nanf("");
        }
    }

    // The wavefronts' states meet: each takes a share of the R * CV accumulators, which the others hand over in LDS as they lie, in
    // rounds that bound the LDS.  Register i of accumulator (x, j): channel CV (4 kq + i) + j of row l16 of tile x.
    constexpr int ACC = R * CV, SHARE = ACC >= WAVES ? ACC / WAVES : 1, TAKERS = ACC / SHARE;
    constexpr int PART = SHARE > 4 ? 4 : SHARE, ROUNDS = SHARE / PART;                 // accumulators of a taker and round
    __shared__ float sm_m[WAVES][16 * R], sm_l[WAVES][16 * R];
    mx_f32x4* const sm_o = reinterpret_cast<mx_f32x4*>(mx_lds);       // in the rings, when all are done with them
    static_assert(mx_attn_lds<FMT, DP, R, WAVES>() >= TAKERS * PART * (WAVES - 1) * kWave * 16, "the handed over accumulators fit");
    float f[R][WAVES], total[R], top[R];
#pragma unroll
    for (int x = 0; x < R; ++x) {
        l[x] = over_column(l[x], [](float p, float q) { return p + q; });
        if (kq == 0) { sm_m[w][16 * x + l16] = m[x]; sm_l[w][16 * x + l16] = l[x]; }
    }
#pragma unroll
    for (int round = 0; round < ROUNDS; ++round) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < TAKERS; ++t)
#pragma unroll
            for (int p = 0; p < PART; ++p) {
                const int n = t * SHARE + round * PART + p;
                if (t != w) sm_o[((t * PART + p) * (WAVES - 1) + (w < t ? w : w - 1)) * kWave + lane] = o[n / CV][n % CV];
            }
        __syncthreads();
        if (round == 0) {
#pragma unroll
            for (int x = 0; x < R; ++x) {
                top[x] = -INFINITY; total[x] = 0.f;
#pragma unroll
                for (int v = 0; v < WAVES; ++v) top[x] = fmaxf(top[x], sm_m[v][16 * x + l16]);
#pragma unroll
                for (int v = 0; v < WAVES; ++v) {             // (a wavefront without a key: m = -inf, its sums 0 or a NaN's)
                    const float mv = sm_m[v][16 * x + l16];
                    f[x][v] = mv == -INFINITY ? 1.f : from_to(a, mv, top[x]);
                    total[x] = fmaf(f[x][v], sm_l[v][16 * x + l16], total[x]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < TAKERS; ++t) {
            if (t != w) continue;
#pragma unroll
            for (int p = 0; p < PART; ++p) {
                const int n = t * SHARE + round * PART + p, x = n / CV, j = n % CV;
                mx_f32x4 sum = o[x][j];
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] *= f[x][t];
#pragma unroll
                for (int v = 0; v < WAVES; ++v) {
                    if (v == t) continue;
                    const mx_f32x4 part = sm_o[((t * PART + p) * (WAVES - 1) + (v < t ? v : v - 1)) * kWave + lane];
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[i] = fmaf(f[x][v], part[i], sum[i]);
                }
                o[x][j] = sum;
            }
        }
    }
    // and are written: GROUP adjacent channels at a time
    constexpr int GROUP = SHARE >= 4 ? 4 : SHARE;
#pragma unroll
    for (int t = 0; t < TAKERS; ++t) {
        if (t != w) continue;
#pragma unroll
        for (int n = t * SHARE; n < (t + 1) * SHARE; n += GROUP) {
            const int x = n / CV, j = n % CV, r = row0 + 16 * x + l16;
            if (r >= a.rows) continue;
            if (n_splits == 1) {
                const int token = r / a.group, head = g * a.group + (r - token * a.group);
                const int64_t at = b * a.os[0] + token * a.os[1] + head * a.os[2];
                const float inv = total[x] == 0.f ? 0.f : 1.0f / total[x];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int ch = CV * (4 * kq + i) + j;
                    if (!FULL && ch >= d) continue;
                    float v[GROUP];
#pragma unroll
                    for (int c = 0; c < GROUP; ++c) v[c] = o[x][j + c][i] * inv;
                    if constexpr (BF16) {
                        uint16_t* dst = static_cast<uint16_t*>(a.out) + at + ch;
                        if constexpr (GROUP == 4) *reinterpret_cast<u32x2*>(dst) = u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
                        else if constexpr (GROUP == 2) *reinterpret_cast<uint32_t*>(dst) = bf16_pair(v[0], v[1]);
                        else *dst = static_cast<uint16_t>(bf16_pair(v[0], 0.f));
                    } else {
                        float* dst = static_cast<float*>(a.out) + at + ch;
#pragma unroll
                        for (int c = 0; c < GROUP; ++c) dst[c] = v[c];
                    }
                }
            } else {
                const int64_t at = static_cast<int64_t>(blockIdx.x) * a.rows + r;
                float* const dst = split_out(a, at) + split * d;
                if (j == 0 && kq == 0) split_state(a, at)[split] = make_float2(top[x], total[x]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int ch = CV * (4 * kq + i) + j;
                    if (!FULL && ch >= d) continue;
                    if constexpr (GROUP == 4) *reinterpret_cast<float4*>(dst + ch) = make_float4(o[x][j][i], o[x][j + 1][i], o[x][j + 2][i], o[x][j + 3][i]);
                    else if constexpr (GROUP == 2) *reinterpret_cast<float2*>(dst + ch) = make_float2(o[x][j][i], o[x][j + 1][i]);
                    else dst[ch] = o[x][j][i];
                }
            }
        }
    }
}

// Many rows (bf16): the products bound it, so a cache element becomes bf16 once for all rows of a workgroup.  It takes tiles of 64 keys:
// its threads convert the next tile from registers into LDS, each 32 channels of a key of K or 4 channels of 8 keys of V, laid down as
// the operands of v_mfma_f32_32x32x16_bf16 that read them (K: a lane's 8 channels of its key; V^T: a lane's 8 keys of its channel), so
// that all LDS accesses are whole wavefronts of consecutive 16 bytes; then they ask for the tile after it and compute the present one.
// A wavefront has 32 rows, one per pair of lanes; the keys of a 32-key half tile stand in the order that leaves a lane with the logits
// of two runs of 8 keys, the second operand of O^T += V^T P^T as it stands.
// KG: groups of wavefronts that share the rows and take turns over the tiles, each with buffers of its own; their states meet in LDS.
// Large chunks end at the clock that the chip keeps under them (2.2 GHz): 2048 tokens over 16000 rows, 32 / 8 heads run at 1010 to 1165
// TFLOP/s in all three shapes of a workgroup.
typedef float mx_f32x16 __attribute__((ext_vector_type(16)));
constexpr int kMxTile = 64;

template <int FMT, int DP, bool FULL, int WAVES, int KG>
__global__ __launch_bounds__(WAVES * kWave, DP == 256 ? 1 : 2) void attn_mx_rows_kernel(MxAttnArgs a)
{
    constexpr int ROW_WAVES = WAVES / KG, THREADS = ROW_WAVES * kWave;                 // of a key group
    constexpr int NB = DP / kMxBlock, T = DP / 16, CT = DP / 32;
    constexpr int K_UNITS = kMxTile * NB, UNITS = K_UNITS + 2 * DP, N = UNITS > THREADS ? UNITS / THREADS : 1;
    constexpr bool PHASED = KG == 2 && FMT == 8 && DP == 128 && FULL;                  // the key groups take turns at the units (vector_phase)
    constexpr int AHEAD = 6;                                  // LDS reads ahead of the products in a matrix phase
    constexpr int BUF = kMxTile * DP / 8;                     // 16-byte entries of K, and of V, in a buffer
    extern __shared__ __attribute__((aligned(16))) u32x4 mx_all_tiles[];   // [KG][2][K, V][BUF]
    __shared__ int again;
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int group = KG > 1 ? __builtin_amdgcn_readfirstlane(tid >> 6) / ROW_WAVES : 0;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6) - group * ROW_WAVES;         // in its group
    u32x4* const mx_tiles = mx_all_tiles + group * (4 * BUF);
    const int l32 = lane & 31, half = lane >> 5;
    const int g = blockIdx.x % a.n_kv_heads, b = blockIdx.x / a.n_kv_heads;
    const int split = blockIdx.z;
    const int d = FULL ? DP : a.head_dim, nb = d / kMxBlock;
    const int block0 = blockIdx.y * (32 * ROW_WAVES), row0 = block0 + 32 * w;
    const int ctx = context_of(a, b);
    const int n_splits = max((ctx + a.keys_per_split - 1) / a.keys_per_split, 1);
    if (split >= n_splits) return;
    const int k0 = split * a.keys_per_split;
    const int ctx1 = min(k0 + a.keys_per_split, ctx);
    const int k1 = min(ctx1, row_limit(a, ctx, min(block0 + 32 * ROW_WAVES, a.rows) - 1));      // of the workgroup (limits grow along the rows)
    const int row = min(row0 + l32, a.rows - 1);
    const int limit = min(row_limit(a, ctx, row), ctx1);
    const int least = min(row_limit(a, ctx, min(row0, a.rows - 1)), ctx1);                  // keys that all rows of the wavefront see

    const int64_t head_row = (static_cast<int64_t>(b) * a.n_kv_heads + g) * a.s_max;
    const uint32_t code_bytes = static_cast<uint32_t>(d) * FMT / 8;
    const uint8_t* const kc = a.kc + head_row * code_bytes;
    const uint8_t* const vc = a.vc + head_row * code_bytes;
    const uint8_t* const ks = a.ks + head_row * nb;
    const uint8_t* const vs = a.vs + head_row * nb;

    // A thread's share of a tile: N units, each 32 channels of a key of K, or 4 channels of 8 keys of V; a wavefront's are of one kind.
    constexpr bool WIDE = FULL && NB == 4;                    // the scales of 8 keys of V as two loads
    uint32_t raw[N][8], sc[N][8];
    auto each_unit = [&](auto of_k, auto of_v) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if constexpr (K_UNITS % THREADS == 0) {
                if (n < K_UNITS / THREADS) of_k(n, n * THREADS + w * kWave); else of_v(n, n * THREADS + w * kWave - K_UNITS);
            } else {
                const int u0 = n * THREADS + w * kWave;
                if (u0 < K_UNITS) of_k(n, u0); else if (u0 < UNITS) of_v(n, u0 - K_UNITS);
            }
        }
    };
    // (s_max is a multiple of 32: a key, or 8 keys from a multiple of 8 on, are moved back into the rows of the head where a tile ends past them)
    auto fetch_from = [&](int k_at, int v_at) __attribute__((always_inline)) {
        each_unit([&](int n, int u0) __attribute__((always_inline)) {
            const uint32_t key = min(k_at + lane, static_cast<int>(a.s_max) - 1), blk = FULL ? u0 / kMxTile : min(u0 / kMxTile, nb - 1);
            const u32x4* src = reinterpret_cast<const u32x4*>(kc + (key * code_bytes + blk * (4 * FMT)));
#pragma unroll
            for (int i = 0; i < FMT / 4; ++i) {
                const u32x4 v = src[i];
#pragma unroll
                for (int e = 0; e < 4; ++e) raw[n][4 * i + e] = v[e];
            }
            sc[n][0] = ks[key * nb + blk];
        }, [&](int n, int u0) __attribute__((always_inline)) {
            const int vu = u0 + lane, cq = vu % (DP / 4), kg = vu / (DP / 4);
            const uint32_t ch = FULL || 4 * cq < d ? 4 * cq : 0, key = min(v_at + 8 * kg, static_cast<int>(a.s_max) - 8);
            const uint8_t* const src = vc + (key * code_bytes + ch * FMT / 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (FMT == 4) raw[n][e] = *reinterpret_cast<const uint16_t*>(src + e * code_bytes);
                else raw[n][e] = *reinterpret_cast<const uint32_t*>(src + e * code_bytes);
            }
            if constexpr (WIDE) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const u32x4 v = *(reinterpret_cast<const u32x4*>(vs + key * nb) + i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[n][4 * i + e] = v[e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) sc[n][e] = vs[key * nb + ch / kMxBlock + e * nb];
            }
        });
    };
    auto fetch = [&](int at) __attribute__((always_inline)) { fetch_from(at, at); };
    // Of the fetched tile: V's rows past the end, which hold anything, as zeros; careful: V's NaN blocks too.
    auto amend = [&](int at, bool careful) __attribute__((always_inline)) {
        if (__builtin_expect(at + kMxTile <= ctx1 && !careful, 1)) return;
        each_unit([&](int, int) {}, [&](int n, int u0) {
            const int vu = u0 + lane, cq = vu % (DP / 4), kg = vu / (DP / 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t byte = WIDE ? sc[n][e] >> (8 * (cq * 4 / kMxBlock)) & 0xFF : sc[n][e];
                if (at + 8 * kg + e >= ctx1 || (careful && byte == 255)) { raw[n][e] = 0u; sc[n][e] = 0x7F7F7F7Fu; }
            }
        });
    };
    // A unit into LDS: K's channels 8 i .. 8 i + 7 of its 32; V's key e as bf16, then its channel i.
    auto convert_k = [&](u32x4* kb, int n, int u0, int i) __attribute__((always_inline)) {
        const int blk = u0 / kMxTile, kt = lane >> 5, k = lane & 31;
        const int m = 16 * (k >> 4) + 8 * ((k >> 2) & 1) + 4 * ((k >> 3) & 1) + (k & 3);
        const float scale = __uint_as_float(sc[n][0] << 23);
        u32x4 v;                                              // chunk 4 blk + i of the row: step 2 blk + i / 2, half i % 2
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = mx_pair_bf16<FMT>(raw[n], 4 * i + e, scale);
        if (!FULL && blk >= nb) v = u32x4{0u, 0u, 0u, 0u};
        kb[(kt * T + 2 * blk + (i >> 1)) * kWave + (i & 1) * 32 + m] = v;
    };
    auto convert_v = [&](int n, int u0, int e, uint32_t (&c)[2][8]) __attribute__((always_inline)) {
        const int cq = (u0 + lane) % (DP / 4);
        const uint32_t turn = (8 * (cq * 4 / kMxBlock) + 9) & 31;
        const uint32_t y = WIDE ? __builtin_amdgcn_alignbit(sc[n][e], sc[n][e], turn) : sc[n][e] << 23;   // (the exponent, whatever lies next to it)
#pragma unroll
        for (int h = 0; h < 2; ++h) c[h][e] = mx_pair_bf16<FMT>(&raw[n][e], h, __uint_as_float(y));
    };
    auto store_v = [&](u32x4* tile, int u0, int i, const uint32_t (&c)[2][8]) __attribute__((always_inline)) {
        const int vu = u0 + lane, cq = vu % (DP / 4), kg = vu / (DP / 4), ch = 4 * cq + i;           // channel CT * m + tile
        u32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __builtin_amdgcn_perm(c[i >> 1][2 * e + 1], c[i >> 1][2 * e], (i & 1) ? 0x07060302u : 0x05040100u);
        tile[BUF + ((kg >> 1) * CT + ch % CT) * kWave + (kg & 1) * 32 + ch / CT] = v;
    };
    auto convert = [&](int buffer) __attribute__((always_inline)) {
        u32x4* const to = mx_tiles + buffer * (2 * BUF);
        each_unit([&](int n, int u0) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) convert_k(to, n, u0, i);
        }, [&](int n, int u0) __attribute__((always_inline)) {
            uint32_t c[2][8];
#pragma unroll
            for (int e = 0; e < 8; ++e) convert_v(n, u0, e, c);
#pragma unroll
            for (int i = 0; i < 4; ++i) store_v(to, u0, i, c);
        });
    };

    if (tid == 0) again = 0;
    const int last_tile = k0 < k1 ? k0 + (k1 - 1 - k0) / kMxTile * kMxTile : k0;
    // the group's tiles: every KG-th; all groups go through as many (the last of some is past the end, and masked)
    const int first = k0 + group * kMxTile;
    constexpr int STEP = KG * kMxTile;
    if (k0 < k1) fetch(min(first, last_tile));
    // Q^T: channels 16 t + 8 half .. + 7 of row l32 (negated if the scale is negative: logits enter by their size)
    mx_bf16x8 qf[T];
    {
        const int token = row / a.group, head = g * a.group + (row - token * a.group);
        const int64_t at = b * a.qs[0] + token * a.qs[1] + head * a.qs[2] + 8 * half;
#pragma unroll
        for (int t = 0; t < T; ++t) {
            u32x4 v = u32x4{0u, 0u, 0u, 0u};
            if (FULL || 16 * t < d) v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q) + at + 16 * t);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] ^= a.q_sign;
            qf[t] = __builtin_bit_cast(mx_bf16x8, v);
        }
    }

    mx_f32x16 o[CT];
    float m, l;                                               // of the row; l: of the lane's own keys
    const mx_bf16x2 ones = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
    mx_f32x16 s[2];                                           // logits of a tile
    float base;                                               // see kMxFar
    // The largest logit of the tile from `at` on, and what is scaled anew where one is far above m.
    auto renew = [&](int at) __attribute__((always_inline)) {
        if (at + kMxTile > least) {
            const int lim = limit - at - 8 * half;
#pragma unroll
            for (int i = 0; i < 32; ++i) s[i >> 4][i & 15] = 16 * (i >> 3) + (i & 7) < lim ? s[i >> 4][i & 15] : -INFINITY;
        }
        float m_new = m;
#pragma unroll
        for (int i = 0; i < 32; i += 2) m_new = fmaxf(fmaxf(m_new, s[i >> 4][i & 15]), s[i >> 4][(i + 1) & 15]);
        if (__any(m_new > m + a.slack)) {
            const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(m_new), __float_as_uint(m_new), false, false);
            m_new = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
            const float alpha = from_to(a, m, m_new == -INFINITY ? 0.f : m_new);
            l *= alpha;
#pragma unroll
            for (int j = 0; j < CT; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[j][i] *= alpha;
            m = m_new;
        }
        base = base_of(a, m);
        if (__builtin_expect(__any(fabsf(base) > kMxFar), 0)) {
            const bool far = fabsf(base) > kMxFar;
#pragma unroll
            for (int i = 0; i < 32; ++i) s[i >> 4][i & 15] -= far ? m : 0.f;
            base = far ? 0.f : base;
        }
    };
    // Weights of the lane's keys 16 k .. 16 k + 15 of the tile (8 of them the lane's), rounded to bf16 once, in the products and in their sum,
    // as civic_prefill_attn rounds them.  A second term, as in attn_mx_kernel where memory hides it, is half as many products again: 1024
    // tokens behind 9001 rows of 8 bits 134 -> 184 us, in 4 bits 133 -> 178, 4 x 128 over 1066 rows 26 -> 30.5, for a 2-norm error against 64
    // bits of 1.66e-3, that of the output's rounding alone, instead of 2.25e-3.
    auto weights = [&](int k) __attribute__((always_inline)) {
        u32x4 pf;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 8 * k + 2 * e;
            const uint32_t pair = bf16_pair(__builtin_amdgcn_exp2f(fmaf(s[i >> 4][i & 15], a.scale_log2, base)),
                                            __builtin_amdgcn_exp2f(fmaf(s[i >> 4][(i + 1) & 15], a.scale_log2, base)));
            l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(mx_bf16x2, pair), ones, l, false);
            pf[e] = pair;
        }
        return pf;
    };
    auto add_logits = [&](const u32x4* kb, int t, int kt) __attribute__((always_inline)) {
        s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(mx_bf16x8, kb[(kt * T + t) * kWave]), qf[t], s[kt], 0, 0, 0);
    };
    auto no_logits = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[0][i] = s[1][i] = 0.f;
    };
    // Logits of a tile.  LDS reads stay four ahead of the products that use them (left to itself the compiler waits for each: 133 us for
    // 128 on 8 x 512 tokens over 2000 rows, 32 / 8 heads of 128).
    auto logits = [&](const u32x4* kb) __attribute__((always_inline)) {
        no_logits();
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) add_logits(kb, t, kt);
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);    // LDS reads
#pragma unroll
        for (int i = 0; i < 2 * T; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // a matrix instruction
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // One tile; the one after it, whose codes are in registers, goes into the other buffer meanwhile, and the one after that is asked for
    // (past the last tile: that one again, not used).
    auto tile = [&](int at, int buffer, bool careful) __attribute__((always_inline)) {
        const u32x4* const kb = mx_tiles + buffer * (2 * BUF) + lane;
        const u32x4* const vb = kb + BUF;
        amend(at + STEP, careful);
        // (two wavefronts of a workgroup share a SIMD: one's products go ahead of the other's vector work, 135.6 us for 132.5 there; two
        // workgroups of 4: 35.8 for 37.6 on 4 x 256 tokens over 2000 rows, heads of 64)
        if constexpr (WAVES == 8) __builtin_amdgcn_s_setprio(1);
        logits(kb);
        if constexpr (WAVES == 8) __builtin_amdgcn_s_setprio(0);
        convert(buffer ^ 1);
        fetch(min(at + 2 * STEP, last_tile));
        renew(at);
        u32x4 vf[CT];                                         // V of the next 16 keys
#pragma unroll
        for (int j = 0; j < CT; ++j) vf[j] = vb[j * kWave];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const u32x4 pf = weights(k);
#pragma unroll
            for (int j = 0; j < CT; ++j) {
                o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(mx_bf16x8, vf[j]), __builtin_bit_cast(mx_bf16x8, pf), o[j], 0, 0, 0);
                if (k < 3) vf[j] = vb[((k + 1) * CT + j) * kWave];
            }
        }
    };
    // Two key groups take turns at the units of a SIMD, which holds a wavefront of each: while one has its vector phase (a tile's weights
    // from its logits; K of the next tile but one and V of the next are asked for) the other has its matrix phase (the products of the
    // weights with V and the next tile's logits, 32 cycles each, and between them the conversion of what was asked for).  A barrier of all
    // wavefronts ends each phase; the second group is one phase behind.  For 8 bits, whose loads and conversions are the longer ones (us, so
    // and as one tile after another: 1024 tokens behind 9001 rows, 28 / 4 heads 134 140, in 4 bits 135 138; 4 x 128 over 1066, 32 / 8, in
    // 4 bits 26.5 26.1; rows of 96 channels, whose registers do not suffice, 32 28).
    static_assert(!PHASED || (N == 2 && K_UNITS == THREADS), "a unit of K and one of V a thread");
    constexpr int V_UNIT = N > 1 ? 1 : 0;
    u32x4 pf[PHASED ? 4 : 1];
    auto vector_phase = [&](int at, bool careful) __attribute__((always_inline)) {
        fetch_from(min(at + 2 * STEP, last_tile), min(at + STEP, last_tile));
        __builtin_amdgcn_sched_barrier(0);
        renew(at);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            u32x4 p = weights(k);
            asm volatile("" : "+v"(p));                       // (else the compiler moves them past the barrier, to the products)
            pf[PHASED ? k : 0] = p;
        }
        __builtin_amdgcn_sched_barrier(0);
        amend(at + STEP, careful);
    };
    // (past the last tile the logits are of what the buffer holds, and not used)
    auto matrix_phase = [&](int buffer) __attribute__((always_inline)) {
        u32x4* const now = mx_tiles + buffer * (2 * BUF);
        u32x4* const then = mx_tiles + (buffer ^ 1) * (2 * BUF);
        const u32x4* const vb = now + BUF + lane;
        const u32x4* const kb = then + lane;
        // product 2 i: of V, keys 16 (i / CT) .. + 15; 2 i + 1: of K, channels 16 (i / 2) .. + 15.  (4 CT is 2 T)
        auto operand = [&](int n) __attribute__((always_inline)) { return n & 1 ? kb[((n >> 1 & 1) * T + (n >> 2)) * kWave] : vb[(n >> 1) * kWave]; };
        u32x4 next[AHEAD];
        uint32_t c[2][8];
        __builtin_amdgcn_s_setprio(1);
        no_logits();
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) next[n] = operand(n);
#pragma unroll
        for (int n = 0; n < 4 * T; ++n) {
            const mx_bf16x8 x = __builtin_bit_cast(mx_bf16x8, next[n % AHEAD]);
            const int i = n >> 1;
            if (n & 1) s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, qf[i >> 1], s[i & 1], 0, 0, 0);
            else o[i % CT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, __builtin_bit_cast(mx_bf16x8, pf[PHASED ? i / CT : 0]), o[i % CT], 0, 0, 0);
            if (n + AHEAD < 4 * T) next[n % AHEAD] = operand(n + AHEAD);
            const int at = n - (4 * T - 16);                  // the last 16 products
            if (at >= 0 && at < 4) convert_k(now, 0, w * kWave, at);
            if (at >= 4 && at < 12) convert_v(V_UNIT, w * kWave, at - 4, c);
            if (at >= 12) store_v(then, w * kWave, at - 12, c);
            __builtin_amdgcn_sched_barrier(0);                // (as it stands: left to itself the compiler waits for each read)
        }
        __builtin_amdgcn_s_setprio(0);
    };
    // A NaN of V meets weights of 0 (0 x NaN), the rows' that do not see it: where one shows, once more with NaN blocks apart.
    bool careful = false;
#pragma unroll 1
    for (;;) {
        m = -INFINITY; l = 0.f;
#pragma unroll
        for (int j = 0; j < CT; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[j][i] = 0.f;
        if (k0 < k1) {
            amend(first, careful);
            convert(0);
            fetch(min(first + STEP, last_tile));
        }
        __syncthreads();
        int buffer = 0;
        if constexpr (PHASED) {
            if (k0 < k1) {
                logits(mx_tiles + lane);
#pragma unroll
                for (int i = 0; i < 4; ++i) convert_k(mx_tiles + 2 * BUF, 0, w * kWave, i);
            }
            if (group == 1) __syncthreads();
#pragma unroll 1
            for (int at = k0; at < k1; at += STEP, buffer ^= 1) {
                vector_phase(at + group * kMxTile, careful);
                __syncthreads();
                matrix_phase(buffer);
                __syncthreads();
            }
            if (group == 0) __syncthreads();
        } else {
#pragma unroll 1
            for (int at = k0; at < k1; at += STEP, buffer ^= 1) {
                tile(at + group * kMxTile, buffer, careful);
                __syncthreads();
            }
        }
        if (careful) break;
        float odd = 0.f;
#pragma unroll
        for (int j = 0; j < CT; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) odd = fmaf(o[j][i], 0.f, odd);
        if (odd != 0.f) again = 1;
        __syncthreads();
        if (__builtin_expect(!again, 1)) break;
        careful = true;
        if (k0 < k1) fetch(min(first, last_tile));
    }
    if (__builtin_expect(careful, 0)) {
        // A row sees a NaN in block i exactly if it sees the first key that has one there: the workgroup's threads look for it together
        // (1024 tokens behind 9001 rows of 8 bits, 28 / 4 heads: 149 us as it is, 349 with a NaN block in every head).
        __shared__ int first_nan[NB];
        if (tid < NB) first_nan[tid] = INT_MAX;
        __syncthreads();
        int nan_at[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) nan_at[i] = INT_MAX;
#pragma unroll 1
        for (int key = k0 + tid; key < k1; key += WAVES * kWave) nan_blocks<NB, FULL>(vs, key, k1, nb, nan_at);
#pragma unroll
        for (int i = 0; i < NB; ++i)
            if (nan_at[i] != INT_MAX) atomicMin(&first_nan[i], nan_at[i]);
        __syncthreads();
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < NB; ++i) bad |= first_nan[i] < limit ? 1u << i : 0u;
#pragma unroll
        for (int j = 0; j < CT; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (bad >> ((CT * (8 * (i >> 2) + 4 * half + (i & 3)) + j) / kMxBlock) & 1) o[j][i] = __builtin_nanf("");
    }

    if constexpr (KG > 1) {                                   // the second group's states join the first one's
        static_assert(KG == 2, "two key groups");
        __shared__ float2 sm_state[ROW_WAVES][kWave];
        mx_f32x4* const theirs = reinterpret_cast<mx_f32x4*>(mx_all_tiles + 4 * BUF) + w * (4 * CT * kWave) + lane;
        if (group == 1) {
            sm_state[w][lane] = make_float2(m, l);
#pragma unroll
            for (int j = 0; j < CT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) theirs[(4 * j + i) * kWave] = mx_f32x4{o[j][4 * i], o[j][4 * i + 1], o[j][4 * i + 2], o[j][4 * i + 3]};
        }
        __syncthreads();
        if (group == 1) return;
        const float2 state = sm_state[w][lane];
        const float top = fmaxf(m, state.x);
        const float f0 = m == -INFINITY ? 1.f : from_to(a, m, top);          // (its sums are 0 or NaN)
        const float f1 = state.x == -INFINITY ? 1.f : from_to(a, state.x, top);
        m = top;
        l = fmaf(f1, state.y, l * f0);
#pragma unroll
        for (int j = 0; j < CT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const mx_f32x4 v = theirs[(4 * j + i) * kWave];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][4 * i + e] = fmaf(f1, v[e], o[j][4 * i + e] * f0);
            }
    }

    // Register i of o[j]: channel CT (8 (i / 4) + 4 half + i % 4) + j of row l32.  Rows go through LDS (the tiles are done with), so that
    // they are stored as they lie: as four channels a lane, 32 rows at a stride of 256 bytes and more, a split's stores took 8 us of 24
    // (4 x 128 tokens over 1066 rows).  Four channels of row r are at place p ^ r % PLACES: reads and writes meet distinct banks.
    constexpr int PARTS = ROW_WAVES > 4 ? ROW_WAVES / 4 : 1, PLACES = DP / 4 / PARTS;          // of a row: parts in turn, places of four channels
    const auto sums = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(sums[0]) + __uint_as_float(sums[1]);
    const float inv = n_splits > 1 ? 1.f : l == 0.f ? 0.f : 1.0f / l;
    int64_t to;                                               // of the lane's row: its first element
    if (n_splits > 1) {
        const int64_t at = static_cast<int64_t>(blockIdx.x) * a.rows + row;
        if (half == 0 && row0 + l32 < a.rows) split_state(a, at)[split] = make_float2(m, l);
        to = (at * a.splits + split) * d;
    } else {
        const int token = row / a.group, head = g * a.group + (row - token * a.group);
        to = b * a.os[0] + token * a.os[1] + head * a.os[2];
    }
    mx_f32x4* const mine = reinterpret_cast<mx_f32x4*>(mx_tiles) + w * (32 * PLACES);
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
#pragma unroll
        for (int x = 0; x < 4; ++x)                           // 4 CT channels lie together
#pragma unroll
            for (int c = 0; c < 4 * CT; c += 4) {
                const int place = (CT * (8 * x + 4 * half) + c) / 4 - part * PLACES;   // (in or out of the part for both halves: PLACES is a multiple of 2 CT)
                if ((CT * 8 * x) / 4 / PLACES != part) continue;
                mx_f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = o[(c + e) % CT][4 * x + (c + e) / CT] * inv;
                mine[l32 * PLACES + (place ^ (l32 & (PLACES - 1)))] = v;
            }
        __builtin_amdgcn_wave_barrier();
        constexpr int AT_ONCE = kWave / PLACES > 0 ? kWave / PLACES : 1;               // rows
#pragma unroll 4
        for (int r0 = 0; r0 < 32; r0 += AT_ONCE) {
            const int r = r0 + lane / PLACES, place = lane & (PLACES - 1), ch = 4 * (place + part * PLACES);
            const int64_t first = __shfl(to, r, kWave);
            const mx_f32x4 v = mine[r * PLACES + (place ^ (r & (PLACES - 1)))];
            if (row0 + r >= a.rows || (!FULL && ch >= d)) continue;
            if (n_splits > 1) *reinterpret_cast<mx_f32x4*>(a.ws + first + ch) = v;
            else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + first + ch) = u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Joins the splits: out = sum_s f_s o_s / sum_s f_s l_s, f_s from m_s to max m.  A wavefront takes a row: its lanes hold the states of a
// split each (two for more than 64) and then four channels each of a split, eight loads in flight.
// grid: (sample and KV head, four rows)
constexpr int kMxMaxSplits = 128;
template <bool BF16>
__global__ __launch_bounds__(256) void attn_mx_merge_kernel(MxAttnArgs a)
{
    __shared__ float sm_f[4][kMxMaxSplits];
    const int lane = threadIdx.x & (kWave - 1), w = threadIdx.x >> 6;
    const int r = blockIdx.y * 4 + w, g = blockIdx.x % a.n_kv_heads, b = blockIdx.x / a.n_kv_heads;
    const int ctx = context_of(a, b), d = a.head_dim;
    const int splits = (ctx + a.keys_per_split - 1) / a.keys_per_split;
    if (splits <= 1 || r >= a.rows) return;                   // (one: the row has its result already)
    const int64_t row = static_cast<int64_t>(blockIdx.x) * a.rows + r;
    const float* const src = split_out(a, row);
    const float2* const state = split_state(a, row);
    const float2 none = make_float2(-INFINITY, 0.f);
    const float2 s0 = lane < splits ? state[lane] : none, s1 = lane + kWave < splits ? state[lane + kWave] : none;
    // lanes `wide` apart hold the same channels of different splits
    const int wide = d <= 32 ? 8 : d <= 64 ? 16 : d <= 128 ? 32 : 64;
    const int c = lane & (wide - 1), y = lane / wide, step = kWave / wide;
    const bool live = 4 * c < d;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int kAhead = 8;
    float4 v[kAhead];
    auto fetch = [&](int at) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int s = at + i * step + y;
            v[i] = s < splits && live ? *reinterpret_cast<const float4*>(src + static_cast<int64_t>(s) * d + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    };
    fetch(0);
    float mx = fmaxf(s0.x, s1.x);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off, kWave));
    auto factor = [&](float2 s) { return s.x == -INFINITY ? 1.f : from_to(a, s.x, mx); };   // (its sums are 0 or NaN)
    const float f0 = factor(s0), f1 = factor(s1);
    sm_f[w][lane] = f0;
    sm_f[w][lane + kWave] = f1;
    const float l = wave_sum(fmaf(f0, s0.y, f1 * s1.y));
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    __builtin_amdgcn_wave_barrier();
    for (int at = 0;;) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int s = at + i * step + y;
            const float f = s < splits ? sm_f[w][s] : 0.f;
            o.x = fmaf(f, v[i].x, o.x); o.y = fmaf(f, v[i].y, o.y); o.z = fmaf(f, v[i].z, o.z); o.w = fmaf(f, v[i].w, o.w);
        }
        at += kAhead * step;
        if (at >= splits) break;
        fetch(at);
    }
#pragma unroll
    for (int off = 32; off >= 8; off >>= 1)
        if (off >= wide) {
            o.x += __shfl_xor(o.x, off, kWave); o.y += __shfl_xor(o.y, off, kWave);
            o.z += __shfl_xor(o.z, off, kWave); o.w += __shfl_xor(o.w, off, kWave);
        }
    if (y > 0 || !live) return;
    const int token = r / a.group, head = g * a.group + (r - token * a.group);
    const int64_t at = b * a.os[0] + token * a.os[1] + head * a.os[2] + 4 * c;
    if constexpr (BF16) *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + at) = u32x2{bf16_pair(o.x * inv, o.y * inv), bf16_pair(o.z * inv, o.w * inv)};
    else *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
}

constexpr int kMxWaves = 4;                                   // of a workgroup of attn_mx_kernel

struct MxAttnPlan {
    int rows_waves, key_groups;                               // of a workgroup of attn_mx_rows_kernel; 0 wavefronts: the other kernel
    int tiles;                                                // of 16 rows, of a workgroup
    int32_t row_blocks, splits, keys_per_split;
    size_t ws_bytes;
};

// What attn_mx_rows_kernel and the merge take, to choose between its shapes and between splits: a turn over a tile a key group takes 1.7 us in
// a workgroup of 4 wavefronts that has its unit alone, 2.4 us where two share it, and 2.1 us in one of 8 (128 channels); a merge reads and
// the kernel before it writes `states` rows of fp32.  (us, 4 wavefronts of 128 rows, 8 of 256, 8 of 128 rows in two key groups, each whole and
// in two splits: 4 x 128 tokens over 1066 rows, 32 / 8 heads 32 32, 38 36, 28 31; 8 x 512 over 2000 128 189, 122 192, 138 222; 1024 behind 9001
// of 8 bits, 28 / 4 191 161, 226 145, 132 154; 4 x 256 over 2000, heads of 64 37 46, 45 45, 29 50; 2 x 60 over 500, 16 / 8 18 17, 22 18, 17 17;
// 2 x 512 over 2000, 16 / 4 of 96 56 43, 68 50, 43 38, and of 256, 4 wavefronts alone, 107 78.)
static double mx_rows_us(int waves, int groups, int64_t units, double turns, int32_t head_dim)
{
    const double width = head_dim <= 64 ? 0.6 : head_dim <= 128 ? 1.0 : 2.0;
    const int64_t at_once = waves == 4 && head_dim <= 128 ? 512 : 256;
    const int64_t full = units / at_once, rest = units % at_once;
    const double shared = waves == 8 ? 2.1 : 2.4, alone = waves == 8 ? 2.1 : 1.7;
    return (groups > 1 ? 2.0 : 0.0) + width * turns * (full * shared + (rest == 0 ? 0.0 : rest <= 256 ? alone : shared));
}
static double mx_merge_us(int64_t states, int32_t head_dim) { return 6.0 + states * (2.0 * 4.0 * head_dim) / 4.0e6; }

// Shapes of a workgroup of attn_mx_rows_kernel: wavefronts, key groups.  Its rows in tiles of 16; its keys a turn.
struct MxRowsShape {
    int waves, groups;
    int64_t row_tiles() const { return 2 * waves / groups; }
    int64_t keys() const { return kMxTile * groups; }
    bool fits(int32_t head_dim) const { return head_dim <= 128 || waves == 4; }
};
constexpr MxRowsShape kMxRowsShapes[] = {{4, 1}, {8, 1}, {8, 2}};
constexpr int64_t kMxRowsMaxSplits = 16;
static bool mx_rows_may_split(int64_t s, int64_t turns, int64_t rows) { return s == 1 || (2 * s <= turns && rows <= 4 * 65535); }   // (the merge's grid.y)

// Splits for a workgroup of `steps` steps of attn_mx_kernel.  Contexts are split where that leaves fewer than 256 workgroups, into pieces of 256 rows or
// more (us, whole and in 4: 1 x 469 rows, 16 / 8 heads of 128 7.9, 8.5; 4 x 938, 32 / 8 11.3, 9.5; 16 x 4000 28.8, 21.3; 64 x 3584 46, 50;
// 8 x 65000 of 8 bits in 8 for 16: 177, 182).
static int64_t mx_few_splits(int64_t units, int64_t steps)
{
    if (units <= 0 || units >= 256 || steps <= 5) return 1;
    int64_t want = (512 + units - 1) / units;
    if (want > steps / 2) want = steps / 2;
    return want < kMxMaxSplits ? want : kMxMaxSplits;
}

static int mx_few_tiles(bool bf16, int64_t tiles) { return bf16 && tiles > 1 ? 2 : 1; }
static size_t mx_splits_bytes(int64_t pairs, int64_t rows, int64_t splits, int32_t head_dim)
{
    return splits > 1 ? sizeof(float) * static_cast<size_t>(pairs) * rows * splits * (head_dim + 2) : 0;
}

static MxAttnPlan mx_attn_plan(bool bf16, int32_t batch, int64_t rows, int32_t n_kv_heads, int32_t head_dim, int64_t n_ctx)
{
    MxAttnPlan p{};
    const int64_t pairs = static_cast<int64_t>(batch) * n_kv_heads, tiles = (rows + 15) / 16;
    int64_t want = 1, step = 32 * kMxWaves, most = (n_ctx + step - 1) / step;
    if (bf16 && rows > 32) {
        double best = 0.0;
        for (const auto& shape : kMxRowsShapes) {
            if (!shape.fits(head_dim)) continue;
            const int64_t row_tiles = shape.row_tiles(), keys = shape.keys();
            const int64_t units = pairs * ((tiles + row_tiles - 1) / row_tiles), turns = (n_ctx + keys - 1) / keys;
            for (int64_t s = 1; s <= kMxRowsMaxSplits && mx_rows_may_split(s, turns, rows); ++s) {
                const double us = mx_rows_us(shape.waves, shape.groups, units * s, static_cast<double>((turns + s - 1) / s), head_dim)
                                + (s > 1 ? mx_merge_us(pairs * rows * s, head_dim) : 0.0);
                if (!p.rows_waves || us < best) {
                    best = us; p.rows_waves = shape.waves; p.key_groups = shape.groups; p.tiles = static_cast<int>(row_tiles);
                    want = s; step = keys; most = turns;
                }
            }
        }
    } else {
        p.tiles = mx_few_tiles(bf16, tiles);
        want = mx_few_splits(pairs * ((tiles + p.tiles - 1) / p.tiles), most);
    }
    p.row_blocks = static_cast<int32_t>((tiles + p.tiles - 1) / p.tiles);
    if (want > most) want = most;
    if (want < 1) want = 1;
    const int64_t steps = (most + want - 1) / want;
    p.keys_per_split = static_cast<int32_t>((steps > 0 ? steps : 1) * step);
    p.splits = static_cast<int32_t>(n_ctx > 0 ? (n_ctx + p.keys_per_split - 1) / p.keys_per_split : 1);
    p.ws_bytes = mx_splits_bytes(pairs, rows, p.splits, head_dim);
    return p;
}

// As many splits as mx_attn_plan takes at most for contexts of up to n_ctx rows, so that a workspace for n_ctx serves the shorter ones too.
// (The plan's own number falls where the pieces become a step longer: 32 steps in 16 pieces of two, 33 in 11 of three.)  attn_mx_kernel: the
// number aimed at, which does not fall.  attn_mx_rows_kernel: the largest s that is faster than every other choice at some context of up to
// n_ctx rows.  What s pieces of n rows gain over r pieces in another shape is at most us(r, n / (keys' r) + 1) - us(s, n / (keys s)), linear
// in n, so the ends decide: the shortest context that is cut so, and the longest.
static int64_t mx_most_splits(bool bf16, int64_t pairs, int64_t rows, int32_t head_dim, int64_t n_ctx)
{
    const int64_t tiles = (rows + 15) / 16;
    if (!bf16 || rows <= 32) {
        const int64_t at_once = mx_few_tiles(bf16, tiles), step = 32 * kMxWaves;
        return mx_few_splits(pairs * ((tiles + at_once - 1) / at_once), (n_ctx + step - 1) / step);
    }
    auto units = [&](const MxRowsShape& x) { return pairs * ((tiles + x.row_tiles() - 1) / x.row_tiles()); };
    auto merge = [&](int64_t s) { return s > 1 ? mx_merge_us(pairs * rows * s, head_dim) : 0.0; };
    int64_t most = 1;
    for (const auto& shape : kMxRowsShapes) {
        if (!shape.fits(head_dim)) continue;
        const int64_t turns = (n_ctx + shape.keys() - 1) / shape.keys();
        for (int64_t s = kMxRowsMaxSplits; s > most; --s) {
            const int64_t shortest = (2 * s - 1) * shape.keys() + 1;
            bool taken = mx_rows_may_split(s, turns, rows);
            for (const auto& other : kMxRowsShapes)
                for (int64_t r = 1; r <= kMxRowsMaxSplits && taken; ++r) {
                    if (!other.fits(head_dim) || !mx_rows_may_split(r, shortest / other.keys(), rows)) break;
                    if (r == s && &other == &shape) continue;
                    auto gain = [&](double n) {
                        return mx_rows_us(other.waves, other.groups, units(other) * r, n / (other.keys() * r) + 1.0, head_dim) + merge(r)
                             - mx_rows_us(shape.waves, shape.groups, units(shape) * s, n / (shape.keys() * s), head_dim) - merge(s);
                    };
                    taken = std::fmax(gain(shortest), gain(n_ctx)) > -1e-3;
                }
            if (taken) most = s;
        }
    }
    return most;
}

static bool mx_attn_sizes_ok(int dtype, int format, int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t n_ctx)
{
    return dtype_size(dtype) && mx_format_ok(format) && batch >= 0 && seq >= 0 && n_q_heads > 0 && n_kv_heads > 0 && n_q_heads % n_kv_heads == 0
        && head_dim > 0 && head_dim % kMxBlock == 0 && n_ctx >= 0;
}

constexpr int64_t kMxMaxPairs = int64_t{1} << 22;             // of a sample and a KV head: grid.x
static bool mx_attn_covered(int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t s_max)
{
    const int64_t rows = static_cast<int64_t>(seq) * (n_q_heads / n_kv_heads);
    return head_dim <= CIVIC_MAX_HEAD_DIM && batch <= 65535 && static_cast<int64_t>(batch) * n_kv_heads <= kMxMaxPairs && s_max <= kMxMaxRows
        && rows <= 16 * 65535;
}

template <int FMT, bool BF16, int DP, bool FULL, int R, int WAVES>
static int mx_attn_launch_few(const MxAttnArgs& a, dim3 grid, hipStream_t stream)
{
    constexpr size_t lds = mx_attn_lds<FMT, DP, R, WAVES>();
    const auto kernel = attn_mx_kernel<FMT, BF16, DP, FULL, R, WAVES>;
    static std::atomic<uint64_t> done{0};
    const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds, &done);
    if (rc != CIVIC_OK) return rc;
    civic::launch(kernel, grid, dim3(WAVES * kWave), lds, stream, a);
    return CIVIC_OK;
}

template <int FMT, int DP, bool FULL, int WAVES, int KG>
static int mx_attn_launch_rows(const MxAttnArgs& a, dim3 grid, hipStream_t stream)
{
    constexpr size_t lds = KG * 2 * 2 * kMxTile * DP * 2;     // two tiles of K and V a key group
    const auto kernel = attn_mx_rows_kernel<FMT, DP, FULL, WAVES, KG>;
    static std::atomic<uint64_t> done{0};
    const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds, &done);
    if (rc != CIVIC_OK) return rc;
    civic::launch(kernel, grid, dim3(WAVES * kWave), lds, stream, a);
    return CIVIC_OK;
}

template <int FMT, bool BF16, int DP, bool FULL>
static int mx_attn_launch(const MxAttnArgs& a, const MxAttnPlan& p, hipStream_t stream)
{
    const dim3 grid(static_cast<unsigned>(a.batch * a.n_kv_heads), static_cast<unsigned>(p.row_blocks), static_cast<unsigned>(p.splits));
    if constexpr (BF16) {
        int rc = CIVIC_OK;
        if (p.rows_waves == 4) rc = mx_attn_launch_rows<FMT, DP, FULL, 4, 1>(a, grid, stream);
        else if (p.rows_waves == 8) {
            if constexpr (DP <= 128) rc = p.key_groups == 1 ? mx_attn_launch_rows<FMT, DP, FULL, 8, 1>(a, grid, stream) : mx_attn_launch_rows<FMT, DP, FULL, 8, 2>(a, grid, stream);
        }
        else if (p.tiles == 2) rc = mx_attn_launch_few<FMT, BF16, DP, FULL, 2, kMxWaves>(a, grid, stream);
        if (rc != CIVIC_OK) return rc;
    }
    if (!p.rows_waves && p.tiles == 1) {
        const int rc = mx_attn_launch_few<FMT, BF16, DP, FULL, 1, kMxWaves>(a, grid, stream);
        if (rc != CIVIC_OK) return rc;
    }
    if (p.splits > 1) {
        const int rc = check_launch();
        if (rc != CIVIC_OK) return rc;
        civic::launch(attn_mx_merge_kernel<BF16>, dim3(static_cast<unsigned>(a.batch * a.n_kv_heads), static_cast<unsigned>((a.rows + 3) / 4)), dim3(256), 0, stream, a);
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
    if (!mx_rows_apart(os, batch, seq, n_q_heads, head_dim)) return CIVIC_ERR_INVALID_ARG;
    MxAttnArgs a{};
    a.rows = seq * (n_q_heads / n_kv_heads);
    const MxAttnPlan p = mx_attn_plan(dtype == CIVIC_BF16, batch, a.rows, n_kv_heads, head_dim, n_ctx);
    if (p.ws_bytes && (!workspace || workspace_bytes < p.ws_bytes)) return CIVIC_ERR_WORKSPACE;
    a.q = q; a.out = out; a.ws = static_cast<float*>(workspace);
    a.kc = static_cast<const uint8_t*>(k_codes); a.ks = static_cast<const uint8_t*>(k_scales);
    a.vc = static_cast<const uint8_t*>(v_codes); a.vs = static_cast<const uint8_t*>(v_scales);
    a.ctx = ctx;
    for (int i = 0; i < 3; ++i) { a.qs[i] = qs[i]; a.os[i] = os[i]; }
    a.s_max = s_max; a.batch = batch; a.seq = seq; a.n_q_heads = n_q_heads; a.n_kv_heads = n_kv_heads; a.group = n_q_heads / n_kv_heads;
    a.head_dim = head_dim; a.n_ctx = static_cast<int32_t>(n_ctx); a.splits = p.splits; a.keys_per_split = p.keys_per_split; a.causal = causal != 0;
    const double scale = softmax_scale == 0.f ? 1.0 / std::sqrt(static_cast<double>(head_dim)) : softmax_scale;
    // (neither 0 nor infinite: a masked logit of -infinity, or a logit of 0, would become NaN)
    a.scale_log2 = static_cast<float>(std::fmin(std::fmax(std::fabs(scale) * 1.4426950408889634, 1.1754944e-38), 3.4028234e38));
    a.slack = std::fmin(kMxSlack / a.scale_log2, 1e30f);
    a.q_sign = scale < 0.0 ? 0x80008000u : 0u;
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
    const int64_t pairs = static_cast<int64_t>(batch) * n_kv_heads, rows = static_cast<int64_t>(seq) * (n_q_heads / n_kv_heads);
    return mx_splits_bytes(pairs, rows, mx_most_splits(dtype == CIVIC_BF16, pairs, rows, head_dim, n_ctx), head_dim);
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
