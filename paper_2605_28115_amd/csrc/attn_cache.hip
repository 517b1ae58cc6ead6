// Attention of new tokens over plain caches (fp32 or bf16 rows): civic_decode_attn_shared and civic_prefill_attn_shared, whose batch
// shares a prefix; civic_decode_attn_weights, which also gives the weights away; and civic_attn_weights of few query rows, the weights alone.
//
//   out[b, i, h, :] = (sum_p e(p) V_prefix[g, p, :] + sum_j e(j) V[b, g, j, :]) / (sum_p e(p) + sum_j e(j)),   e = exp(scale <q, K>),
//   p < P, j < ctx[b] - (seq - 1 - i) when causal, j < ctx[b] else;   weights[b, g, j] = base[b, g, j] + sum_h e(j) / sum e.
//
// The queries of a KV head are rows r = token * group + head of the group; a workgroup takes tiles of 16 of them, the columns of its
// matrix products, through a run of 32-key steps, its wavefronts taking turns.
//   - K rows are read as they lie and are the first operand of S^T = K Q^T.  The two 16-key tiles of a step hold keys 8 a + r and
//     8 a + 4 + r in row 4 a + r: a lane then owns the logits of 8 consecutive keys of one row, the second operand of
//     O^T += V^T P^T as it stands (fp32: of eight products of four keys).
//   - Of V a lane reads a sixteenth of the channels of its 8 keys (any permutation of the channels may be the rows of V^T); for bf16 it
//     gathers, for each channel, the 8 keys out of them (v_perm).  No LDS before the wavefronts meet.
//   - bf16 weights enter as the sum of two bf16 terms: 2^-17 of a weight against the output's rounding of 2^-9.
//   - K is asked for again when its product is done and V when its is: a step's loads fly under the other product.
// Sources: where rows of a sample are few (at most kPackedRows) and the prefix is long or the samples many, the prefix is attended by the
// rows of all samples together, by workgroups of their own in the same launch; else a workgroup goes through the prefix and then through
// its sample's own rows.  Runs are cut into pieces where that leaves few workgroups;
// a second launch joins the pieces.
#include "rows_device.h"
#include "tile_device.h"

namespace civic {

constexpr int kStepKeys = 32, kFewWaves = 4, kFewThreads = kFewWaves * kWave;
constexpr int kPackedRows = 32;
constexpr int kMaxPieces = 128;                               // of a row

struct CacheAttnArgs {
    const void* q; void* out; float* ws;
    const void* kp; const void* vp;                           // the prefix [n_kv_heads, s_prefix, head_dim]
    const void* kc; const void* vc;                           // the caches [batch, n_kv_heads, s_max, head_dim]
    const int32_t* prefix_ctx; const int32_t* ctx;
    const float* base; float* weights;                        // civic_decode_attn_weights: [batch, n_kv_heads, s_max]
    int64_t qs[3], os[3];
    int64_t s_prefix, s_max;
    int32_t batch, seq, n_q_heads, n_kv_heads, head_dim, group, causal;
    int32_t n_prefix, n_ctx;
    int32_t rows;                                             // of a sample and KV head: seq * group
    int32_t packed;                                           // the prefix has workgroups of its own
    int32_t prefix_tiles, row_tiles;                          // of R * 16 rows: of all samples (packed), of one
    int32_t prefix_pieces, own_pieces;                        // of a row (not packed: own_pieces, the prefix among them)
    int32_t prefix_steps, own_steps;                          // of a piece
    int32_t prefix_keys, own_keys;                            // of a step
    int32_t pitch;                                            // of the logits [batch, n_q_heads, pitch]; 0: not kept
    int32_t logit_steps, logits_at, ends_at;                  // steps whose logits fit LDS; where those and the rows' ends are there (floats)
    int32_t fused;                                            // a pair's weights are added up by its one workgroup, out of LDS
    uint32_t items;                                           // fused: workgroups of pairs; those behind them write rows from `written` on
    int64_t written;                                          // fused: rows of a pair that its workgroup writes (its context's in any case)
    float scale;                                              // times log2 e
    uint32_t flip;
};

// The workspace: the logits of every (sample, KV head, row), if they are kept; of every (row, piece) one (base, sum), then head_dim
// unnormalised outputs.
__device__ __forceinline__ int64_t all_rows(const CacheAttnArgs& a) { return static_cast<int64_t>(a.batch) * a.n_kv_heads * a.rows; }
__device__ __forceinline__ float* logits_of(const CacheAttnArgs& a, int64_t row) { return a.ws + row * a.pitch; }
__device__ __forceinline__ float2* piece_state(const CacheAttnArgs& a, int64_t row)
{
    return reinterpret_cast<float2*>(logits_of(a, all_rows(a))) + row * (a.prefix_pieces + a.own_pieces);
}
__device__ __forceinline__ float* piece_out(const CacheAttnArgs& a, int64_t row)
{
    const int pieces = a.prefix_pieces + a.own_pieces;
    return logits_of(a, all_rows(a)) + (all_rows(a) * pieces + 1) / 2 * 4 + row * pieces * a.head_dim;   // (16-byte aligned)
}

// What a workgroup has: `n` rows from row0 on, of sample b or (b < 0) of all samples; steps [s0, s1) over `prefix` and then `own` rows.
struct CacheItem {
    int b, g, row0, n, prefix, own, s0, s1, piece;
};

struct RowAt { int b, token, head, r; };                      // r: the row of its sample
__device__ __forceinline__ RowAt row_at(const CacheAttnArgs& a, const CacheItem& it, int i)
{
    int r = it.row0 + i, b = it.b;
    if (b < 0) { b = r / a.rows; r -= b * a.rows; }
    const int token = r / a.group;
    return {b, token, it.g * a.group + (r - token * a.group), r};
}
// Own rows that a token sees.
__device__ __forceinline__ int own_limit(const CacheAttnArgs& a, int own, int token) { return a.causal ? max(own - (a.seq - 1 - token), 0) : own; }

__device__ __forceinline__ int steps_of(int rows, int keys = kStepKeys) { return (rows + keys - 1) / keys; }

// A row's base and the reciprocal of its sum, as its weights are made from its logits (nothing seen: 0), and the keys that it sees.
struct RowEnd { float base, inv; int seen, none; };
__device__ __forceinline__ RowEnd ended(float base, float sum, int seen) { return {base == -INFINITY ? 0.f : base, sum == 0.f ? 0.f : 1.f / sum, seen, 0}; }
// What the row gives to key `key`, whose logit is z.
__device__ __forceinline__ float weight_of(const CacheAttnArgs& a, const RowEnd& e, float z, int64_t key)
{
    return key < e.seen ? __builtin_amdgcn_exp2f(fmaf(z, a.scale, -e.base)) * e.inv : 0.f;
}
__device__ __forceinline__ void keep_end(const CacheAttnArgs& a, const CacheItem& it, float* lds, int i, float base, float sum)
{
    reinterpret_cast<RowEnd*>(lds + a.ends_at)[i] = ended(base, sum, own_limit(a, it.own, (it.row0 + i) / a.group));
}

// Floats of a row of outputs in LDS (against bank conflicts).
constexpr int out_pitch(int dp) { return dp + 4; }
constexpr size_t meet_bytes(int dp, int states, int rows) { return sizeof(float) * states * rows * (out_pitch(dp) + 2); }

// The ends of a workgroup's STATES runs over its ROWS rows, in LDS as [state][row] outputs, then bases, then sums: joined, and written as the
// rows' results where they have one piece, else as a piece of them.
template <bool BF16, int DP, bool FULL, int STATES, int THREADS, bool LOGITS>
__device__ __forceinline__ void meet(const CacheAttnArgs& a, const CacheItem& it, float* lds, int rows)
{
    float* const sm_b = lds + STATES * rows * out_pitch(DP);
    float* const sm_l = sm_b + STATES * rows;
    const int d = FULL ? DP : a.head_dim, pieces = a.prefix_pieces + a.own_pieces;
    for (int idx = threadIdx.x; idx < it.n * (d / 4); idx += THREADS) {
        const int i = idx / (d / 4), c = (idx - i * (d / 4)) * 4;
        float to = sm_b[i];
#pragma unroll
        for (int x = 1; x < STATES; ++x) to = fmaxf(to, sm_b[x * rows + i]);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        float sum = 0.f;
#pragma unroll
        for (int x = 0; x < STATES; ++x) {
            const float f = base_step(sm_b[x * rows + i], to);
            const float4 v = *reinterpret_cast<const float4*>(lds + (x * rows + i) * out_pitch(DP) + c);
            acc.x = fmaf(f, v.x, acc.x); acc.y = fmaf(f, v.y, acc.y); acc.z = fmaf(f, v.z, acc.z); acc.w = fmaf(f, v.w, acc.w);
            sum = fmaf(f, sm_l[x * rows + i], sum);
        }
        const RowAt at = row_at(a, it, i);
        const int64_t row = (static_cast<int64_t>(at.b) * a.n_kv_heads + it.g) * a.rows + at.r;
        if (pieces == 1) {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            const int64_t dst = at.b * a.os[0] + at.token * a.os[1] + at.head * a.os[2] + c;
            if constexpr (BF16) *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + dst) = u32x2{bf16_word(acc.x * inv, acc.y * inv), bf16_word(acc.z * inv, acc.w * inv)};
            else *reinterpret_cast<float4*>(static_cast<float*>(a.out) + dst) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
        } else {
            *reinterpret_cast<float4*>(piece_out(a, row) + static_cast<int64_t>(it.piece) * d + c) = acc;
        }
        if (c == 0) {
            if (LOGITS && a.fused) keep_end(a, it, lds, i, to, sum);
            else if (LOGITS ? a.n_ctx > 0 : pieces > 1) piece_state(a, row)[it.piece] = make_float2(to, sum);
        }
    }
}

// DP: head_dim rounded up to 64, 128 or 256.  FULL: head_dim == DP.  R: tiles of 16 rows.  MODE: the outputs; the logits as well, which are
// kept, and where a row has one piece its weights are added up here; these alone, without V.
enum { kOutputs, kBoth, kLogits };
// Steps whose loads fit the registers at a time (row bytes, row tiles), and wavefronts of a SIMD that these are held to.  (Where outputs and logits
// are made, one: with two some are spilled, and it is no faster.  fp32 rows of 256 channels spill 32 registers with one as well.)
constexpr int few_stages(int row_bytes, int r) { return row_bytes <= 128 || (row_bytes <= 256 && r == 1) ? 2 : 1; }
constexpr int few_resident(int row_bytes) { return row_bytes <= 256 ? 2 : 1; }

template <bool BF16, int DP, bool FULL, int R, int MODE>
__device__ __forceinline__ void few_rows(const CacheAttnArgs& a, const CacheItem& it, float* lds)
{
    constexpr bool LOGITS = MODE != kOutputs, VALUES = MODE != kLogits;
    constexpr int ESZ = BF16 ? 2 : 4;
    constexpr int KT = DP * ESZ / 64;                         // 64-byte chunks of a row
    constexpr int NJ = DP / 16;                               // tiles of 16 channels of O^T
    constexpr int PB = NJ * ESZ < 16 ? NJ * ESZ : 16;         // bytes of a piece of V that a lane reads, PN of them 16 lanes apart
    constexpr int PN = NJ * ESZ / PB, PW = PB / 4, PJ = PB / ESZ;   // its words, its channels
    // Loads ahead: of a whole step where the registers hold two of them, else K's under the second product and V's under the first.
    constexpr int STAGES = MODE == kBoth ? 1 : MODE == kLogits ? (DP * ESZ <= 512 ? 2 : 1) : few_stages(DP * ESZ, R);
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, kq = lane >> 4;
    const int d = FULL ? DP : a.head_dim;
    const uint32_t row_bytes = static_cast<uint32_t>(d) * ESZ;

    // the queries: 16 bytes at byte 64 t + 16 kq of rows l16 of the tiles; own rows that they see (rows past the last: zeros that see none)
    u32x4 qf[R][KT];
    int lim[R];
#pragma unroll
    for (int x = 0; x < R; ++x) {
        const int i = 16 * x + l16;
        lim[x] = 0;
#pragma unroll
        for (int t = 0; t < KT; ++t) qf[x][t] = u32x4{0u, 0u, 0u, 0u};
        if (i < it.n) {
            const RowAt at = row_at(a, it, i);
            lim[x] = own_limit(a, it.own, at.token);
            const char* const q = static_cast<const char*>(a.q) + (at.b * a.qs[0] + at.token * a.qs[1] + at.head * a.qs[2]) * ESZ;
#pragma unroll
            for (int t = 0; t < KT; ++t)
                if (FULL || 64 * t + 16 * kq < static_cast<int>(row_bytes)) {
                    u32x4 v = *reinterpret_cast<const u32x4*>(q + 64 * t + 16 * kq);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] ^= a.flip;
                    qf[x][t] = v;
                }
        }
    }

    const int prefix_steps = steps_of(it.prefix);
    const char* const kp = static_cast<const char*>(a.kp) + static_cast<int64_t>(it.g) * a.s_prefix * row_bytes;
    const char* const vp = static_cast<const char*>(a.vp) + static_cast<int64_t>(it.g) * a.s_prefix * row_bytes;
    const int64_t own0 = (static_cast<int64_t>(it.b < 0 ? 0 : it.b) * a.n_kv_heads + it.g) * a.s_max * row_bytes;
    const char* const kc = static_cast<const char*>(a.kc) + own0;
    const char* const vc = static_cast<const char*>(a.vc) + own0;

    // Step s: whether it is the prefix's, its first key there, and the rows from that key on
    struct Step { bool prefix; int key, rows; };
    auto step_at = [&](int s) __attribute__((always_inline)) {
        Step x;
        x.prefix = s < prefix_steps;
        x.key = kStepKeys * (x.prefix ? s : s - prefix_steps);
        x.rows = (x.prefix ? it.prefix : it.own) - x.key;
        return x;
    };
    u32x4 kb[STAGES][2][KT];
    uint32_t vb[STAGES][8][PN * PW];
    // (keys past the last re-read it: their logits are masked)
    auto fetch_k = [&](int s, u32x4 (&kf)[2][KT]) __attribute__((always_inline)) {
        const Step x = step_at(s);
        const char* const base = (x.prefix ? kp : kc) + static_cast<int64_t>(x.key) * row_bytes;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const uint32_t off = static_cast<uint32_t>(min(8 * (l16 >> 2) + 4 * y + (l16 & 3), x.rows - 1)) * row_bytes + 16 * kq;
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                if (FULL || 64 * t + 16 * kq < static_cast<int>(row_bytes)) kf[y][t] = load_streaming(reinterpret_cast<const u32x4*>(base + off + 64 * t));
                else kf[y][t] = u32x4{0u, 0u, 0u, 0u};
            }
        }
    };
    auto fetch_v = [&](int s, uint32_t (&vf)[8][PN * PW]) __attribute__((always_inline)) {
        if constexpr (!VALUES) return;
        const Step x = step_at(s);
        const char* const base = (x.prefix ? vp : vc) + static_cast<int64_t>(x.key) * row_bytes;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t off = static_cast<uint32_t>(min(8 * kq + e, x.rows - 1)) * row_bytes;
#pragma unroll
            for (int p = 0; p < PN; ++p) {
                uint32_t c = p * 16 * PB + l16 * PB;
                if (!FULL && c >= row_bytes) c = 0;             // (channels past the row: written nowhere)
                if constexpr (PB == 16) {
                    const u32x4 v = load_streaming(reinterpret_cast<const u32x4*>(base + off + c));
#pragma unroll
                    for (int i = 0; i < 4; ++i) vf[e][4 * p + i] = v[i];
                } else {
                    const u32x2 v = load_streaming(reinterpret_cast<const u32x2*>(base + off + c));
                    vf[e][0] = v[0]; vf[e][1] = v[1];
                }
            }
        }
    };
    // channel of row m of tile j of O^T
    auto channel = [&](int j, int m) __attribute__((always_inline)) { return (j / PJ) * 16 * PJ + m * PJ + j % PJ; };

    row_f32x4 o[R][NJ];
    float base[R], l[R];                                       // l: the lane's own keys
#pragma unroll
    for (int x = 0; x < R; ++x) {
        base[x] = -INFINITY; l[x] = 0.f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) o[x][j] = row_f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // logits (before the scale) of keys 8 kq .. + 7 of step s and row l16 of tile x; -infinity where the row sees no such key
    auto logits = [&](const Step& st, const u32x4 (&kf)[2][KT], int x, float (&z)[8]) __attribute__((always_inline)) {
        row_f32x4 s[2] = {row_f32x4{0.f, 0.f, 0.f, 0.f}, row_f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int y = 0; y < 2; ++y) s[y] = mma16<BF16>(kf[y][t], qf[x][t], s[y]);
        const int seen = (st.prefix ? st.rows : lim[x] - st.key) - 8 * kq;
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = e < seen ? s[e >> 2][e & 3] : -INFINITY;
    };
    const int logit_pitch = LOGITS ? kStepKeys * a.logit_steps + 4 : 0;
    int round0 = it.s0, round1 = it.s1;
    auto turn = [&](int s, u32x4 (&kf)[2][KT], uint32_t (&vf)[8][PN * PW]) __attribute__((always_inline)) {
        const Step st = step_at(s);
        float z[R][8];
#pragma unroll
        for (int x = 0; x < R; ++x) logits(st, kf, x, z[x]);
        if (STAGES == 1 && s + kFewWaves < round1) fetch_k(s + kFewWaves, kf);
        if constexpr (LOGITS) {
#pragma unroll
            for (int x = 0; x < R; ++x)
                if (16 * x + l16 < it.n) {
                    float* const dst = lds + a.logits_at + (16 * x + l16) * logit_pitch + kStepKeys * (s - round0) + 8 * kq;
                    *reinterpret_cast<float4*>(dst) = make_float4(z[x][0], z[x][1], z[x][2], z[x][3]);
                    *reinterpret_cast<float4*>(dst + 4) = make_float4(z[x][4], z[x][5], z[x][6], z[x][7]);
                }
        }
        float top[R];
        bool outgrown = false;
#pragma unroll
        for (int x = 0; x < R; ++x) {
            top[x] = z[x][0];
#pragma unroll
            for (int e = 1; e < 8; ++e) top[x] = fmaxf(top[x], z[x][e]);
            outgrown |= top[x] * a.scale > base[x] + kBaseSlack;
        }
        if (__any(outgrown)) {
#pragma unroll
            for (int x = 0; x < R; ++x) {
                const float t = rows_max(top[x]) * a.scale;
                const float to = t > base[x] + kBaseSlack ? rintf(t) : base[x];
                const float f = base_step(base[x], to);
                base[x] = to;
                l[x] *= f;
                if constexpr (VALUES) {
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[x][j][r] *= f;
                }
            }
        }
#pragma unroll
        for (int x = 0; x < R; ++x) {
            const float off = base[x] == -INFINITY ? 0.f : base[x];
#pragma unroll
            for (int e = 0; e < 8; ++e) { z[x][e] = __builtin_amdgcn_exp2f(fmaf(z[x][e], a.scale, -off)); l[x] += z[x][e]; }
        }
        if constexpr (!VALUES) {
        } else if constexpr (BF16) {
            u32x4 hi[R], lo[R];
#pragma unroll
            for (int x = 0; x < R; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float p0 = z[x][2 * e], p1 = z[x][2 * e + 1];
                    hi[x][e] = bf16_rest(p0, p1);
                    lo[x][e] = bf16_word(p0, p1);
                }
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                u32x4 v;                                       // of keys 8 kq .. + 7 the channel that row l16 of tile j is
                const int word = (j / PJ) * PW + (j % PJ) / 2;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = __builtin_amdgcn_perm(vf[2 * e + 1][word], vf[2 * e][word], (j & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int x = 0; x < R; ++x) {
                    o[x][j] = mma16<true>(v, hi[x], o[x][j]);
                    o[x][j] = mma16<true>(v, lo[x], o[x][j]);
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int x = 0; x < R; ++x)
                        o[x][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[e][j]), z[x][e], o[x][j], 0, 0, 0);
        }
        if (STAGES == 1 && s + kFewWaves < round1) fetch_v(s + kFewWaves, vf);
    };
    auto run = [&]() __attribute__((always_inline)) {
        int s = round0 + w;
        if (s < round1) { fetch_k(s, kb[0]); fetch_v(s, vb[0]); }
        for (; s < round1; s += STAGES * kFewWaves) {
            if constexpr (STAGES == 2) {
                constexpr int W = kFewWaves;
                if (s + W < round1) { fetch_k(s + W, kb[1]); fetch_v(s + W, vb[1]); }
                turn(s, kb[0], vb[0]);
                if (s + W >= round1) break;
                if (s + 2 * W < round1) { fetch_k(s + 2 * W, kb[0]); fetch_v(s + 2 * W, vb[0]); }
                turn(s + W, kb[1], vb[1]);
            } else {
                turn(s, kb[0], vb[0]);
            }
        }
    };
    if constexpr (!LOGITS) {
        run();
    } else {
        // The logits stay in LDS and are written a round of steps at a time, rows of kilobytes.  (Written step by step, between the loads, they
        // take a third as long again as the loads: 8 x 65000 rows 307 us without them, 440 so, whatever the stores' size and policy.)
        const int64_t row_first = (static_cast<int64_t>(it.b) * a.n_kv_heads + it.g) * a.rows + it.row0;
        for (; round0 < it.s1; round0 = round1) {
            round1 = min(round0 + a.logit_steps, it.s1);
            run();
            if (a.fused) break;                                // (one round: they are used where they are)
            __syncthreads();
            const int quads = kStepKeys / 4 * (round1 - round0);
            for (int i = 0; i < it.n; ++i) {                   // (the pitch has room for whole steps)
                float4* const dst = reinterpret_cast<float4*>(logits_of(a, row_first + i) + kStepKeys * round0);
                const float4* const src = reinterpret_cast<const float4*>(lds + a.logits_at + i * logit_pitch);
                for (int c = tid; c < quads; c += kFewThreads) dst[c] = src[c];
            }
            __syncthreads();
        }
    }
#pragma unroll
    for (int x = 0; x < R; ++x) l[x] = rows_sum(l[x]);

    // An infinity or NaN of V has met a weight of 0 (a key that its row does not see, or past the end) or the terms of one: the wavefront's
    // outputs are made again, one multiply-add for each key that its row sees.
    float odd = 0.f;
    if constexpr (VALUES) {
#pragma unroll
        for (int x = 0; x < R; ++x)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) odd = fmaf(o[x][j][r], 0.f, odd);
    }
    if (__builtin_expect(__any(odd != 0.f), 0)) {
#pragma unroll
        for (int x = 0; x < R; ++x)
#pragma unroll
            for (int j = 0; j < NJ; ++j) o[x][j] = row_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int t = it.s0 + w; t < it.s1; t += kFewWaves) {
            const Step st = step_at(t);
            fetch_k(t, kb[0]);
            const char* const vbase = (st.prefix ? vp : vc) + static_cast<int64_t>(st.key) * row_bytes;
#pragma unroll
            for (int x = 0; x < R; ++x) {
                float z[8];
                logits(st, kb[0], x, z);
                const float off = base[x] == -INFINITY ? 0.f : base[x];
                const int seen = st.prefix ? st.rows : lim[x] - st.key;
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = __builtin_amdgcn_exp2f(fmaf(z[e], a.scale, -off));
#pragma unroll 1
                for (int y = 0; y < 4; ++y)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float wgt = __shfl(z[e], 16 * y + l16, kWave);
                        const int key = 8 * y + e;
                        if (key >= seen) continue;
#pragma unroll
                        for (int j = 0; j < NJ; ++j)
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const int c = channel(j, 4 * kq + r);
                                if (!FULL && c >= d) continue;
                                const char* const v = vbase + static_cast<int64_t>(key) * row_bytes + c * ESZ;
                                const float value = BF16 ? bf16_bits_to_float(*reinterpret_cast<const uint16_t*>(v)) : *reinterpret_cast<const float*>(v);
                                o[x][j][r] = fmaf(wgt, value, o[x][j][r]);
                            }
                    }
            }
        }
    }

    // the wavefronts meet
    float* const sm_b = lds + (VALUES ? kFewWaves * it.n * out_pitch(DP) : 0);
    float* const sm_l = sm_b + kFewWaves * it.n;
#pragma unroll
    for (int x = 0; x < R; ++x) {
        const int i = 16 * x + l16;
        if (i < it.n) {
            if (kq == 0) { sm_b[w * it.n + i] = base[x]; sm_l[w * it.n + i] = l[x]; }
            if constexpr (VALUES) {
                float* const dst = lds + (w * it.n + i) * out_pitch(DP);
                static_assert(PJ % 4 == 0, "four consecutive channels of a lane");
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int j = 0; j < NJ; j += 4)
                        *reinterpret_cast<float4*>(dst + channel(j, 4 * kq + r)) = make_float4(o[x][j][r], o[x][j + 1][r], o[x][j + 2][r], o[x][j + 3][r]);
            }
        }
    }
    __syncthreads();
    if constexpr (VALUES) {
        meet<BF16, DP, FULL, kFewWaves, kFewThreads, LOGITS>(a, it, lds, it.n);
    } else if (tid < it.n) {
        float to = sm_b[tid], sum = 0.f;
#pragma unroll
        for (int x = 1; x < kFewWaves; ++x) to = fmaxf(to, sm_b[x * it.n + tid]);
#pragma unroll
        for (int x = 0; x < kFewWaves; ++x) sum = fmaf(base_step(sm_b[x * it.n + tid], to), sm_l[x * it.n + tid], sum);
        if (a.fused) keep_end(a, it, lds, tid, to, sum);
        else if (a.n_ctx > 0) piece_state(a, (static_cast<int64_t>(it.b) * a.n_kv_heads + it.g) * a.rows + it.row0 + tid)[it.piece] = make_float2(to, sum);
    }
    if (LOGITS && a.fused) {
        __syncthreads();
        const int64_t first = (static_cast<int64_t>(it.b) * a.n_kv_heads + it.g) * a.s_max;
        for (int64_t key = tid, end = max(static_cast<int64_t>(it.own), a.written); key < end; key += kFewThreads) {
            const float had = a.base ? a.base[first + key] : 0.f;
            if (key < it.own) {
                float sum = 0.f;
#pragma unroll 4
                for (int i = 0; i < it.n; ++i)
                    sum += weight_of(a, reinterpret_cast<const RowEnd*>(lds + a.ends_at)[i], lds[a.logits_at + i * logit_pitch + key], key);
                a.weights[first + key] = had + sum;
            } else {
                a.weights[first + key] = had;
            }
        }
    }
}

// The id-th workgroup of those of the prefix (packed), of tiles of TILE rows and steps of KEYS keys.
template <int TILE, int KEYS>
__device__ __forceinline__ CacheItem prefix_item(const CacheAttnArgs& a, uint32_t id, int prefix)
{
    CacheItem it;
    const uint32_t v = id / a.n_kv_heads, tile = v / a.prefix_pieces;
    it.g = id - v * a.n_kv_heads;
    it.piece = v - tile * a.prefix_pieces;
    it.b = -1;
    it.row0 = tile * TILE;
    it.n = min(TILE, a.batch * a.rows - it.row0);
    it.prefix = prefix; it.own = 0;
    it.s0 = it.piece * a.prefix_steps;
    it.s1 = min(it.s0 + a.prefix_steps, steps_of(prefix, KEYS));
    return it;
}
// The same of a sample's rows; the heaviest causal tiles come first.
template <int TILE, int KEYS>
__device__ __forceinline__ CacheItem own_item(const CacheAttnArgs& a, uint32_t id, int prefix)
{
    CacheItem it;
    const uint32_t pairs = static_cast<uint32_t>(a.batch) * a.n_kv_heads;
    const uint32_t v = id / pairs, pair = id - v * pairs, up = v / a.own_pieces, piece = v - up * a.own_pieces;
    it.b = pair / a.n_kv_heads; it.g = pair - it.b * a.n_kv_heads;
    it.row0 = (a.row_tiles - 1 - up) * TILE;
    it.n = min(TILE, a.rows - it.row0);
    it.prefix = a.packed ? 0 : prefix;
    it.own = clamped(a.ctx, it.b, a.n_ctx);
    it.s0 = piece * a.own_steps;
    // (a causal tile's last token sees the most)
    const int sees = own_limit(a, it.own, (it.row0 + it.n - 1) / a.group);
    it.s1 = min(it.s0 + a.own_steps, steps_of(it.prefix, KEYS) + steps_of(sees, KEYS));
    it.piece = piece + a.prefix_pieces;
    return it;
}
// (nothing there: the join knows; one piece: zeros)
__device__ __forceinline__ bool leaves(const CacheAttnArgs& a, const CacheItem& it) { return it.s0 >= it.s1 && a.prefix_pieces + a.own_pieces > 1; }

template <bool BF16, int DP, bool FULL, int R, int MODE>
__global__ __launch_bounds__(kFewThreads, few_resident(DP * (BF16 ? 2 : 4))) void attn_cache_kernel(CacheAttnArgs a)
{
    extern __shared__ __attribute__((aligned(16))) float cache_lds[];
    if (MODE != kOutputs && a.fused && blockIdx.x >= a.items) {
        weights_behind<kFewThreads>(a.base, a.weights, static_cast<int64_t>(a.batch) * a.n_kv_heads, a.s_max, a.written, blockIdx.x - a.items, gridDim.x - a.items);
        return;
    }
    const int prefix = clamped(a.prefix_ctx, 0, a.n_prefix);
    const uint32_t prefix_items = a.packed ? static_cast<uint32_t>(a.n_kv_heads) * a.prefix_tiles * a.prefix_pieces : 0;
    const CacheItem it = blockIdx.x < prefix_items ? prefix_item<16 * R, kStepKeys>(a, blockIdx.x, prefix) : own_item<16 * R, kStepKeys>(a, blockIdx.x - prefix_items, prefix);
    if (leaves(a, it)) return;
    few_rows<BF16, DP, FULL, R, MODE>(a, it, cache_lds);
}

// ------------------------------------------------------------------------------------------------------------- many rows
// bf16 heads of 64, 96, 128 and (much work) 256, more than 32 rows: bound by the products.  KG groups of four wavefronts have the same 128 rows, 32 a wavefront,
// and take turns over tiles of 64 keys.  A group's threads hold the next tile's K and V in registers while the present one is computed from
// LDS, and lay it down in the other buffer: rows as they are, their 16-byte chunks exchanged against bank conflicts (swz).  S^T = K Q^T by
// v_mfma_f32_32x32x16_bf16 leaves a lane with 16 keys' logits of one row, the second operand of O^T += V^T P^T as it stands; V^T comes out of
// the rows by transposing LDS reads.  Weights are rounded to bf16 once, in the products and in their sum alike: with hundreds of keys to a row
// that is half the output's own rounding, and a second term would double the second product.  A row's base moves when what a lane
// has of a tile's weights adds up to more than 2^9, which takes no search for the largest logit in any other tile, and no weight is larger: sums over V stay finite
// as the few rows' do.  (us, so and with 2^20, 16 x 61 tokens behind 4001 rows: 79.6, 80.4; logits three times as large 81.0, 80.0, ten times 92.6, 85.6.)
constexpr int kManyRows = 128, kManyKeys = 64, kManyThreads = 256;   // of a key group
constexpr float kManySlack = 512.f;

typedef float many_f32x16 __attribute__((ext_vector_type(16)));

// Wavefronts of a SIMD: 256 channels need all its registers.
constexpr int many_resident(int dp) { return dp <= 128 ? 2 : 1; }

template <int DP, int KG> constexpr size_t many_lds()
{
    constexpr size_t tiles = size_t{KG} * 2 * 2 * kManyKeys * DP * 2, ends = meet_bytes(DP, KG, kManyRows);
    return tiles > ends ? tiles : ends;
}

template <int DP, int KG>
__device__ __forceinline__ void many_rows(const CacheAttnArgs& a, const CacheItem& it, float* lds_f)
{
    constexpr int KS = DP / 16, DT = DP / 32, PC = DP / 8, PITCH = PC, ROWB = DP * 2, TILEB = kManyKeys * ROWB;
    constexpr int NL = kManyKeys * PC / kManyThreads;         // 16-byte pieces of a thread, of a K or V tile
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), kg = w >> 2, wr = w & 3, gt = tid & (kManyThreads - 1);
    const int col = lane & 31, half = lane >> 5;
    char* const lds = reinterpret_cast<char*>(lds_f) + kg * 4 * TILEB;   // K of two tiles, V of two tiles
    const int i_row = 32 * wr + col;

    // the queries: channels 16 s + 8 half .. + 7 of row col (rows past the last: zeros that see everything); own rows seen
    row_bf16x8 qf[KS];
    int lim = it.own, all_see = it.own;                       // of the lane's row; of all rows of the wavefront
    {
        u32x4 z = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[s] = __builtin_bit_cast(row_bf16x8, z);
        if (i_row < it.n) {
            const RowAt at = row_at(a, it, i_row);
            if (it.b >= 0) lim = own_limit(a, it.own, at.token);
            const char* const q = static_cast<const char*>(a.q) + (at.b * a.qs[0] + at.token * a.qs[1] + at.head * a.qs[2]) * 2 + 16 * half;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                u32x4 v = *reinterpret_cast<const u32x4*>(q + 32 * s);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] ^= a.flip;
                qf[s] = __builtin_bit_cast(row_bf16x8, v);
            }
        }
        if (it.b >= 0 && 32 * wr < it.n) all_see = own_limit(a, it.own, row_at(a, it, 32 * wr).token);
    }
    const int prefix_steps = steps_of(it.prefix, kManyKeys);
    const char* const kp = static_cast<const char*>(a.kp) + static_cast<int64_t>(it.g) * a.s_prefix * ROWB;
    const char* const vp = static_cast<const char*>(a.vp) + static_cast<int64_t>(it.g) * a.s_prefix * ROWB;
    const int64_t own0 = (static_cast<int64_t>(it.b < 0 ? 0 : it.b) * a.n_kv_heads + it.g) * a.s_max * ROWB;
    const char* const kc = static_cast<const char*>(a.kc) + own0;
    const char* const vc = static_cast<const char*>(a.vc) + own0;
    struct Step { const char* k; const char* v; bool prefix; int key, rows; };
    auto step_at = [&](int s) __attribute__((always_inline)) {
        Step x;
        x.prefix = s < prefix_steps;
        x.key = kManyKeys * (x.prefix ? s : s - prefix_steps);
        x.rows = (x.prefix ? it.prefix : it.own) - x.key;
        x.k = (x.prefix ? kp : kc) + static_cast<int64_t>(x.key) * ROWB;
        x.v = (x.prefix ? vp : vc) + static_cast<int64_t>(x.key) * ROWB;
        return x;
    };
    u32x4 kn[NL], vn[NL];
    auto fetch = [&](int s) __attribute__((always_inline)) {  // (keys past the last re-read it: their logits are masked)
        const Step x = step_at(s);
#pragma unroll
        for (int j = 0; j < NL; ++j) {
            const int slot = j * kManyThreads + gt, row = slot / PC;
            const uint32_t off = static_cast<uint32_t>(min(row, x.rows - 1)) * ROWB + (slot - row * PC) * 16;
            kn[j] = *reinterpret_cast<const u32x4*>(x.k + off);
            vn[j] = *reinterpret_cast<const u32x4*>(x.v + off);
        }
    };
    auto put = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NL; ++j) {
            const int slot = j * kManyThreads + gt, row = slot / PC, at = row * ROWB + (((slot - row * PC) ^ swz<PITCH>(row)) << 4);
            *reinterpret_cast<u32x4*>(lds + buf * TILEB + at) = kn[j];
            *reinterpret_cast<u32x4*>(lds + (2 + buf) * TILEB + at) = vn[j];
        }
    };
    many_f32x16 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
    float base = -INFINITY, l[2] = {0.f, 0.f};
    const row_bf16x2 ones = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
    const int l16 = lane & 15, g16 = (lane >> 4) & 1;

    // keys that the lane's row sees of a tile, from its register 0 on: register r of half tile t is key 32 t + 8 (r / 4) + r % 4 + 4 half
    auto seen = [&](const Step& st) __attribute__((always_inline)) { return (st.prefix ? st.rows : min(lim, it.own) - st.key) - 4 * half; };
    auto mask = [&](many_f32x16 (&s)[2], int thr) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[t][r] = 32 * t + 8 * (r >> 2) + (r & 3) < thr ? s[t][r] : -INFINITY;
    };
    auto compute = [&](const Step& st, int buf) __attribute__((always_inline)) {
        const char* const kt = lds + buf * TILEB;
        const char* const vt = lds + (2 + buf) * TILEB;
        many_f32x16 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
#pragma unroll
        for (int c = 0; c < KS; ++c)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const row_bf16x8 kf = *reinterpret_cast<const row_bf16x8*>(kt + (32 * t + col) * ROWB + (((2 * c + half) ^ swz<PITCH>(32 * t + col)) << 4));
                s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[c], s[t], 0, 0, 0);
            }
        if (st.rows < kManyKeys || (!st.prefix && st.key + kManyKeys > all_see)) mask(s, seen(st));
        u32x4 p[2][2];
        float sum[2];
        auto weigh = [&]() __attribute__((always_inline)) {
            const float off = base == -INFINITY ? 0.f : base;
            sum[0] = sum[1] = 0.f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[t][8 * u + 2 * e], a.scale, -off));
                        const float p1 = __builtin_amdgcn_exp2f(fmaf(s[t][8 * u + 2 * e + 1], a.scale, -off));
                        const row_bf16x2 pp = {static_cast<__bf16>(p0), static_cast<__bf16>(p1)};
                        p[t][u][e] = __builtin_bit_cast(uint32_t, pp);
                        sum[e & 1] = __builtin_amdgcn_fdot2_f32_bf16(pp, ones, sum[e & 1], false);
                    }
        };
        const bool unseen = __any(base == -INFINITY);         // (a row that has seen nothing has no base)
        if (!unseen) weigh();
        if (unseen || __any(!(sum[0] + sum[1] <= kManySlack))) {
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
            const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * a.scale;
            const float to = top > base ? rintf(top) : base, f = base_step(base, to);
            base = to;
            l[0] *= f; l[1] *= f;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[t][r] *= f;
            weigh();
        }
        l[0] += sum[0]; l[1] += sum[1];
        // k slot (half, e) of step (t, u) is key 32 t + 16 u + 8 (e / 4) + 4 half + e % 4
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int x = 0; x < DT; ++x) {
                    s16x4 v[2];
#pragma unroll
                    for (int hi = 0; hi < 2; ++hi) {
                        const int row = 32 * t + 16 * u + 8 * hi + 4 * half + (l16 >> 2), el = 32 * x + 16 * g16 + 4 * (l16 & 3);
                        v[hi] = lds_read_tr16(reinterpret_cast<const __bf16*>(vt + row * ROWB + (((el >> 3) ^ swz<PITCH>(row)) << 4) + (el & 7) * 2));
                    }
                    const s16x8 vf = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
                    o[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(row_bf16x8, vf), __builtin_bit_cast(row_bf16x8, p[t][u]), o[x], 0, 0, 0);
                }
    };
    const int turns = (it.s1 - it.s0 + KG - 1) / KG;          // of every key group (the last may have nothing in its own)
    int s = it.s0 + kg;
    if (s < it.s1) { fetch(s); put(0); }
    __syncthreads();
    for (int i = 0; i < turns; ++i, s += KG) {
        const bool more = s + KG < it.s1;
        if (more) fetch(s + KG);
        if (s < it.s1 && 32 * wr < it.n) compute(step_at(s), i & 1);
        if (more) put((i + 1) & 1);
        __syncthreads();
    }
    const auto sums = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[0] + l[1]), __float_as_uint(l[0] + l[1]), false, false);
    const float total = __uint_as_float(sums[0]) + __uint_as_float(sums[1]);

    // An infinity or NaN of V has met a weight of 0: the wavefront's outputs are made again, one multiply-add for each key that its row sees.
    float odd = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) odd = fmaf(o[t][r], 0.f, odd);
    if (__builtin_expect(__any(odd != 0.f), 0)) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
        const float off = base == -INFINITY ? 0.f : base;
#pragma unroll 1
        for (int y = it.s0 + kg; y < it.s1; y += KG) {
            const Step st = step_at(y);
            const int thr = seen(st);
#pragma unroll 1
            for (int t = 0; t < 2; ++t) {
                many_f32x16 z;
#pragma unroll
                for (int r = 0; r < 16; ++r) z[r] = 0.f;
#pragma unroll
                for (int c = 0; c < KS; ++c)
                    z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        *reinterpret_cast<const row_bf16x8*>(st.k + static_cast<int64_t>(min(32 * t + col, st.rows - 1)) * ROWB + 32 * c + 16 * half), qf[c], z, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int in = 32 * t + 8 * (r >> 2) + (r & 3);
                    // (rounded as in the products, whose sum is that of the rounded ones)
                    const float p = in < thr ? static_cast<float>(static_cast<__bf16>(__builtin_amdgcn_exp2f(fmaf(z[r], a.scale, -off)))) : 0.f;
#pragma unroll 1
                    for (int h = 0; h < 2; ++h) {
                        const float wgt = __shfl(p, 32 * h + col, kWave);
                        const int key = in + 4 * h;
                        if (key >= thr + 4 * half) continue;  // (thr + 4 half: what the row sees)
#pragma unroll
                        for (int x = 0; x < DT; ++x)
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                o[x][e] = fmaf(wgt, bf16_bits_to_float(*reinterpret_cast<const uint16_t*>(st.v + static_cast<int64_t>(key) * ROWB + (32 * x + 8 * (e >> 2) + (e & 3) + 4 * half) * 2)), o[x][e]);
                    }
                }
            }
        }
    }

    // the key groups meet (every wavefront is through with the tiles)
    float* const sm_b = lds_f + KG * kManyRows * out_pitch(DP);
    float* const sm_l = sm_b + KG * kManyRows;
    if (i_row < it.n) {
        if (half == 0) { sm_b[kg * kManyRows + i_row] = base; sm_l[kg * kManyRows + i_row] = total; }
        float* const dst = lds_f + (kg * kManyRows + i_row) * out_pitch(DP);
#pragma unroll
        for (int x = 0; x < DT; ++x)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<float4*>(dst + 32 * x + 2 * e + 4 * half) = make_float4(o[x][e], o[x][e + 1], o[x][e + 2], o[x][e + 3]);
    }
    __syncthreads();
    meet<true, DP, true, KG, KG * kManyThreads, false>(a, it, lds_f, kManyRows);
}

template <int DP, int KG>
__global__ __launch_bounds__(KG * kManyThreads, many_resident(DP)) void attn_cache_rows_kernel(CacheAttnArgs a)
{
    extern __shared__ __attribute__((aligned(16))) float cache_lds[];
    const CacheItem it = own_item<kManyRows, kManyKeys>(a, blockIdx.x, clamped(a.prefix_ctx, 0, a.n_prefix));
    if (leaves(a, it)) return;
    many_rows<DP, KG>(a, it, cache_lds);
}

// The prefix for all samples' rows by many_rows, every sample's own rows by few_rows, in one launch: the first are bound by products and the
// second by memory, so they alternate in the grid, eight at a time (an XCD each).
template <int DP, int R>
__global__ __launch_bounds__(kManyThreads, many_resident(DP)) void attn_cache_mixed_kernel(CacheAttnArgs a)
{
    extern __shared__ __attribute__((aligned(16))) float cache_lds[];
    const int prefix = clamped(a.prefix_ctx, 0, a.n_prefix);
    const uint32_t first = static_cast<uint32_t>(a.n_kv_heads) * a.prefix_tiles * a.prefix_pieces, second = gridDim.x - first;
    const uint32_t id = blockIdx.x, both = min(first, second) / 8 * 16;   // as far as they alternate
    const bool is_first = id < both ? (id & 8) == 0 : first > second ? id - both < first - both / 2 : id - both >= second - both / 2;
    uint32_t at;
    if (id < both) at = (id >> 4) * 8 + (id & 7);
    else if (first > second) at = is_first ? id - both / 2 : id - first;
    else at = is_first ? id - second : id - both / 2;
    if (is_first) {
        const CacheItem it = prefix_item<kManyRows, kManyKeys>(a, at, prefix);
        if (!leaves(a, it)) many_rows<DP, 1>(a, it, cache_lds);
    } else {
        const CacheItem it = own_item<16 * R, kStepKeys>(a, at, prefix);
        if (!leaves(a, it)) few_rows<true, DP == 96 ? 128 : DP, DP != 96, R, kOutputs>(a, it, cache_lds);
    }
}

// Pieces of a row that hold anything: the first `first` of the prefix's, the first `second` of the others, in the order of the workspace.
struct LivePieces { int first, second; };
__device__ __forceinline__ LivePieces live_pieces(const CacheAttnArgs& a, int own, int sees)
{
    const int prefix = clamped(a.prefix_ctx, 0, a.n_prefix);
    LivePieces x;
    x.first = a.packed ? (steps_of(prefix, a.prefix_keys) + a.prefix_steps - 1) / a.prefix_steps : 0;
    x.second = (steps_of(a.packed ? 0 : prefix, a.own_keys) + steps_of(sees, a.own_keys) + a.own_steps - 1) / a.own_steps;
    return x;
}

// Joins the pieces of a row: out = sum_s f_s o_s / sum_s f_s l_s.  A wavefront takes a row: its lanes hold a piece's state each (two of
// more than 64) and then four channels each of a piece, eight loads in flight.
template <bool BF16>
__device__ __forceinline__ void join_row(const CacheAttnArgs& a, int b, int g, int r, int tile_rows, float* sm_f)
{
    const int lane = threadIdx.x & (kWave - 1), d = a.head_dim;
    const int own = clamped(a.ctx, b, a.n_ctx);
    // what the row's tile went through: as far as its last row sees
    const int last = min((r / tile_rows + 1) * tile_rows, a.rows) - 1;
    const LivePieces live = live_pieces(a, own, own_limit(a, own, last / a.group));
    const int n = live.first + live.second;
    const int64_t row = (static_cast<int64_t>(b) * a.n_kv_heads + g) * a.rows + r;
    const float* const src = piece_out(a, row);
    const float2* const state = piece_state(a, row);
    auto place = [&](int i) { return i < live.first ? i : i - live.first + a.prefix_pieces; };
    const float2 none = make_float2(-INFINITY, 0.f);
    const float2 s0 = lane < n ? state[place(lane)] : none, s1 = lane + kWave < n ? state[place(lane + kWave)] : none;
    const int wide = d <= 32 ? 8 : d <= 64 ? 16 : d <= 128 ? 32 : 64;    // lanes of a row; lanes `wide` apart: other pieces
    const int c = lane & (wide - 1), y = lane / wide, step = kWave / wide;
    const bool there = 4 * c < d;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int kAhead = 8;
    float4 v[kAhead];
    auto fetch = [&](int at) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int p = at + i * step + y;
            v[i] = p < n && there ? *reinterpret_cast<const float4*>(src + static_cast<int64_t>(place(p)) * d + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    };
    fetch(0);
    float to = fmaxf(s0.x, s1.x);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) to = fmaxf(to, __shfl_xor(to, off, kWave));
    const float f0 = base_step(s0.x, to), f1 = base_step(s1.x, to);
    sm_f[lane] = f0;
    sm_f[lane + kWave] = f1;
    const float sum = wave_sum(fmaf(f0, s0.y, f1 * s1.y));
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    __builtin_amdgcn_wave_barrier();
    for (int at = 0; at < n;) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int p = at + i * step + y;
            const float f = p < n ? sm_f[p] : 0.f;
            o.x = fmaf(f, v[i].x, o.x); o.y = fmaf(f, v[i].y, o.y); o.z = fmaf(f, v[i].z, o.z); o.w = fmaf(f, v[i].w, o.w);
        }
        at += kAhead * step;
        if (at < n) fetch(at);
    }
#pragma unroll
    for (int off = 32; off >= 8; off >>= 1)
        if (off >= wide) {
            o.x += __shfl_xor(o.x, off, kWave); o.y += __shfl_xor(o.y, off, kWave);
            o.z += __shfl_xor(o.z, off, kWave); o.w += __shfl_xor(o.w, off, kWave);
        }
    if (y > 0 || !there) return;
    const int token = r / a.group, head = g * a.group + (r - token * a.group);
    const int64_t dst = b * a.os[0] + token * a.os[1] + head * a.os[2] + 4 * c;
    if constexpr (BF16) *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + dst) = u32x2{bf16_word(o.x * inv, o.y * inv), bf16_word(o.z * inv, o.w * inv)};
    else *reinterpret_cast<float4*>(static_cast<float*>(a.out) + dst) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
}

template <bool BF16>
__global__ __launch_bounds__(256) void attn_cache_join_kernel(CacheAttnArgs a, int32_t tile_rows)
{
    __shared__ float sm_f[4][kMaxPieces];
    const int w = threadIdx.x >> 6;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + w;
    const int64_t pair = row / a.rows;
    if (pair >= static_cast<int64_t>(a.batch) * a.n_kv_heads) return;
    const int b = static_cast<int>(pair / a.n_kv_heads);
    join_row<BF16>(a, b, static_cast<int>(pair - static_cast<int64_t>(b) * a.n_kv_heads), static_cast<int>(row - pair * a.rows), tile_rows, sm_f[w]);
}

// Where a pair's logits were kept in memory, the second launch: grid (pair of sample and KV head, keys / kSumKeys + 1).  y = 0 joins the
// pieces of the pair's rows, where they have outputs; every other workgroup takes kSumKeys cache rows and adds up what their logits give over
// the pair's rows, 64 rows at a time: their ends from the pieces into LDS, then four keys a thread.
constexpr int kSumKeys = 1024, kSumRows = 64;
template <bool BF16>
__global__ __launch_bounds__(256) void attn_cache_sums_kernel(CacheAttnArgs a, int32_t tile_rows)
{
    __shared__ float sm_f[4][kMaxPieces];
    __shared__ RowEnd sm_e[kSumRows];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = tid >> 6;
    const int64_t pair = blockIdx.x;
    const int b = static_cast<int>(pair / a.n_kv_heads), g = static_cast<int>(pair - static_cast<int64_t>(b) * a.n_kv_heads);
    if (blockIdx.y == 0) {
        if (a.own_pieces > 1 && a.out != nullptr)
            for (int r = w; r < a.rows; r += 4) join_row<BF16>(a, b, g, r, tile_rows, sm_f[w]);
        return;
    }
    const int own = clamped(a.ctx, b, a.n_ctx);
    const int64_t key = static_cast<int64_t>(blockIdx.y - 1) * kSumKeys + tid * 4;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    if (static_cast<int64_t>(blockIdx.y - 1) * kSumKeys < own)           // (uniform)
        for (int r0 = 0; r0 < a.rows; r0 += kSumRows) {
            const int rows = min(kSumRows, a.rows - r0);
            __syncthreads();
            for (int r = r0 + w; r < r0 + rows; r += 4) {
                const int last = min((r / tile_rows + 1) * tile_rows, a.rows) - 1;   // the row's tile went as far as its last row sees
                const int pieces = a.own_pieces == 1 ? 1 : live_pieces(a, own, own_limit(a, own, last / a.group)).second;
                const float2* const state = piece_state(a, pair * a.rows + r);
                const float2 none = make_float2(-INFINITY, 0.f);
                const float2 s0 = lane < pieces ? state[lane] : none, s1 = lane + kWave < pieces ? state[lane + kWave] : none;
                float to = fmaxf(s0.x, s1.x);
#pragma unroll
                for (int off = 32; off > 0; off >>= 1) to = fmaxf(to, __shfl_xor(to, off, kWave));
                const float l = wave_sum(fmaf(base_step(s0.x, to), s0.y, base_step(s1.x, to) * s1.y));
                if (lane == 0) sm_e[r - r0] = ended(to, l, own_limit(a, own, r / a.group));
            }
            __syncthreads();
            if (key < own)
#pragma unroll 4
                for (int r = 0; r < rows; ++r) {               // (what the row does not see is in the pitch, and has no weight)
                    const RowEnd e = sm_e[r];
                    const float4 z = *reinterpret_cast<const float4*>(logits_of(a, pair * a.rows + r0 + r) + key);
                    sum[0] += weight_of(a, e, z.x, key); sum[1] += weight_of(a, e, z.y, key + 1);
                    sum[2] += weight_of(a, e, z.z, key + 2); sum[3] += weight_of(a, e, z.w, key + 3);
                }
        }
    const int64_t at = pair * a.s_max + key;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (key + e < a.s_max) {
            const float had = a.base ? a.base[at + e] : 0.f;
            if (key + e < own) a.weights[at + e] = had + sum[e];
            else if (a.weights != a.base) a.weights[at + e] = had;
        }
}

// ------------------------------------------------------------------------------------------------------------- host
enum CacheKind { kFew, kRows, kMixed };
struct CachePlan {
    CacheKind kind;
    int tiles;                                                // R
    int groups;                                               // KG
    bool packed;
    int prefix_tile, own_tile, prefix_keys, own_keys;         // rows of a tile, keys of a step
    int64_t prefix_tiles, row_tiles, prefix_pieces, own_pieces, prefix_steps, own_steps;
    int64_t most_pieces;                                      // of a row, at these sizes or with fewer keys
    int64_t blocks;
};

// Pieces that a run of `steps` steps is cut into at most, with `units` runs: three workgroups to a unit, of 8 steps or more; and of 32 steps at most,
// so that samples of different length even out, as long as that makes no more than kEvenUnits workgroups.  A grid that is full without is not cut:
// pieces of every row of a long prompt are its outputs several times over, written and read again, and a workspace that grows with rows times
// keys.  (us, bound as it is, with 768, 6144 and without: 128 samples of 500..8000 rows, 32 / 8 heads of 128 382, 425, 373, 379; 96 of 30000 1722,
// 1704, 1744, 1906; 16 x 512 tokens of heads of 80 behind 1024 and 512 rows 430, 433, 431, 724, and 164 MiB; 4096 fp32 rows a head over 4096 keys
// 467, 468, 467, 801.)  Where the logits are kept, as few as fill the chip twice: a pair that is not cut adds up its
// weights in the same launch, and longer rounds of logits cost less between the loads (us, cut so and into pieces of 512 rows: 64 samples of
// 117..3584 rows, 32 / 8 heads of 128 101, 114; 64 x 3584 150, 197; 8 x 65000 384, 463).  Runs of up to kWholeSteps steps, five to a wavefront,
// are through before a second launch would be (4 x 469 rows behind a prefix 10.0 whole, 11.9 cut; 4 x 1000 15.1, 12.2).
constexpr int64_t kWholeSteps = 20, kEvenUnits = 3200;
static int64_t pieces_of(bool logits, int64_t units, int64_t steps)
{
    if (units <= 0 || steps <= kWholeSteps) return 1;
    const int64_t want = logits ? 512 / units : std::max(ceil_div(768, units), std::min(ceil_div(steps, 32), kEvenUnits / units));
    return std::max<int64_t>(1, std::min<int64_t>({want, steps / 8, kMaxPieces / 2}));
}
// The same for many_rows: 256 workgroups, of `least` steps or more.
static int64_t many_pieces_of(int64_t units, int64_t steps, int64_t least)
{
    return std::max<int64_t>(1, std::min<int64_t>({units > 0 ? 256 / units : 1, steps / least, kMaxPieces / 2}));
}
// Steps of a prefix piece beside the samples' own rows, at least: 8, and as many as a workgroup gets through (1.4 us a step) while the
// own rows, on average half of what they may be, come from memory at 5 TB/s; more pieces then only write more results.  (us in pieces of 4, 8, 16 and 32
// steps: 64 samples behind 8001 rows with 117..900 of their own, 32 / 8 heads 64.7, 55.9, 45.2, 64.2; behind 1000 rows 36.6, 36.1, 37; 16 samples
// behind 8001 30.8, 25.5, 33.7, 55.2.)
static int64_t prefix_least(int64_t pairs, int64_t n_ctx, int32_t head_dim)
{
    return std::max<int64_t>(8, pairs * n_ctx * head_dim * 2 / (int64_t{7} * 1000 * 1000));
}

// Tiles of 16 rows times keys from which 256 channels go with many_rows, which then has one wavefront to a SIMD and 3.5 us a step.  (us, so and with
// few_rows: 16 samples of 64 rows, 4 KV heads, behind 1000, 260000, 42, 47; of 128, 530000, 53, 76; 2 of 512, 290000, 49, 52, of 256, 140000, 44, 31; 4 of
// 256 behind 2000, 530000, 51, 69; the prefix of 32 x 8 rows, 8 heads, behind 4000, 510000, 65, 81, of 16 x 8, 260000, 62, 58; 28 samples of 368 behind
// 1000 190, 304; against it: 64 x 8 rows, 8 heads, behind 2500 111, 94, 4000 causal rows of 4 heads over their own 1000 keys 72, 61.)
constexpr int64_t kWideWork = 300000;

static CachePlan cache_plan(bool bf16, bool logits, int32_t batch, int64_t rows, int32_t n_kv_heads, int32_t head_dim, int64_t n_prefix, int64_t n_ctx)
{
    CachePlan p{};
    const int64_t pairs = static_cast<int64_t>(batch) * n_kv_heads;
    // (us, the prefix by workgroups of its own and by those of each sample, over again: 16 samples behind 469 / 1000 / 2000 rows, 32 / 8 heads of 128
    // 21.2 / 21.5 / 21.7, 12.2 / 14.9 / 21.4; 4 behind 4000, 16 / 8 13.8, 16.4; 64 of 117..900 rows behind 469 34.6, 48.2)
    const int64_t pair_units = pairs * ceil_div(rows, bf16 && head_dim <= 128 && rows > 16 ? 32 : 16);
    const bool over_again = n_prefix <= 2048 && pair_units <= 256;
    p.packed = n_prefix > 0 && batch > 1 && rows <= kPackedRows && !over_again;
    const int64_t few_tiles = p.packed ? n_kv_heads * ceil_div(batch * rows, 16) : pairs * ceil_div(rows, 16);
    const bool many = bf16 && !logits && (head_dim == 64 || head_dim == 96 || head_dim == 128
                                          || (head_dim == 256 && few_tiles * (n_prefix + (p.packed ? 0 : n_ctx)) > kWideWork));
    p.kind = many && !p.packed && rows > kPackedRows ? kRows : many && p.packed && batch * rows > kPackedRows ? kMixed : kFew;
    p.tiles = bf16 && head_dim <= 128 && (p.packed && p.kind == kFew ? batch * rows : rows) > 16 ? 2 : 1;
    p.prefix_tile = p.kind == kMixed ? kManyRows : 16 * p.tiles;
    p.own_tile = p.kind == kRows ? kManyRows : 16 * p.tiles;
    p.prefix_keys = p.kind == kMixed ? kManyKeys : kStepKeys;
    p.own_keys = p.kind == kRows ? kManyKeys : kStepKeys;
    p.row_tiles = ceil_div(rows, p.own_tile);
    const int64_t units = pairs * p.row_tiles;
    const int64_t prefix_steps = ceil_div(n_prefix, p.packed ? p.prefix_keys : p.own_keys), own_steps = ceil_div(n_ctx, p.own_keys) + (p.packed ? 0 : prefix_steps);
    p.prefix_tiles = p.packed ? ceil_div(batch * rows, p.prefix_tile) : 0;
    const int64_t prefix_units = n_kv_heads * p.prefix_tiles;
    const int64_t prefix_most = !p.packed ? 0 : p.kind == kMixed ? many_pieces_of(prefix_units, prefix_steps, 8) : pieces_of(logits, prefix_units, prefix_steps);
    p.groups = p.kind == kRows && head_dim <= 128 && units < 384 ? 2 : 1;
    const int64_t own_most = p.kind == kRows ? many_pieces_of(units, own_steps, 4) : pieces_of(logits, units, own_steps);
    p.most_pieces = prefix_most + own_most;
    if (p.packed)                                              // (with a shorter prefix)
        p.most_pieces = std::max(p.most_pieces, pieces_of(logits, pair_units, ceil_div(n_ctx, kStepKeys) + ceil_div(std::min<int64_t>(n_prefix, 2048), kStepKeys)));
    if (head_dim == 256 && p.kind != kFew)                     // (with fewer keys)
        p.most_pieces = std::max(p.most_pieces, (p.packed ? pieces_of(false, few_tiles, ceil_div(n_prefix, kStepKeys)) : 0)
                                                    + pieces_of(false, pairs * ceil_div(rows, 16), ceil_div(n_ctx, kStepKeys) + (p.packed ? 0 : ceil_div(n_prefix, kStepKeys))));
    p.own_steps = std::max<int64_t>(1, ceil_div(own_steps, own_most));
    p.own_pieces = std::max<int64_t>(1, ceil_div(own_steps, p.own_steps));
    p.prefix_steps = 1;
    if (p.packed) {
        const int64_t pieces = p.kind == kMixed ? many_pieces_of(prefix_units, prefix_steps, prefix_least(pairs, n_ctx, head_dim)) : prefix_most;
        p.prefix_steps = std::max<int64_t>(1, ceil_div(prefix_steps, pieces));
        p.prefix_pieces = ceil_div(prefix_steps, p.prefix_steps);
    }
    p.blocks = prefix_units * p.prefix_pieces + units * p.own_pieces;
    return p;
}

static size_t cache_ws_bytes(const CachePlan& p, int32_t batch, int64_t rows, int32_t n_kv_heads, int32_t head_dim)
{
    return p.most_pieces > 1 ? sizeof(float) * static_cast<size_t>(batch) * n_kv_heads * rows * p.most_pieces * (head_dim + 2) + 16 : 0;
}

static bool cache_sizes_ok(int dtype, int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t n_prefix, int64_t n_ctx)
{
    return dtype_size(dtype) && batch >= 0 && seq >= 0 && n_q_heads > 0 && n_kv_heads > 0 && n_q_heads % n_kv_heads == 0 && head_dim > 0
        && head_dim % 8 == 0 && n_prefix >= 0 && n_ctx >= 0;
}

// Tiles of 16 rows of all pairs: a launch has fewer than 2^32 threads (more than kEvenUnits of them are not cut, and fewer make no more than that
// and 768 workgroups).
constexpr int64_t kMaxUnits = int64_t{1} << 21;
static bool cache_covered(int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t s_prefix, int64_t s_max)
{
    const int64_t rows = static_cast<int64_t>(seq) * (n_q_heads / n_kv_heads), pairs = static_cast<int64_t>(batch) * n_kv_heads;
    return head_dim <= CIVIC_MAX_HEAD_DIM && s_prefix <= kCacheMaxRows && s_max <= kCacheMaxRows && pairs <= kMaxUnits && rows <= (int64_t{1} << 26)
        && pairs * ceil_div(rows, 16) <= kMaxUnits;
}

// Where a workgroup that keeps logits has what in LDS (floats): the ends of its runs, the rows' ends, the logits.
constexpr size_t kLdsBytes = 160 * 1024;                      // of a unit
struct LogitPlace {
    int rows, ends_at, logits_at;
    int most;                                                 // steps that fit, with two workgroups to a unit where the ends are small
    size_t bytes(int steps) const { return sizeof(float) * (logits_at + static_cast<size_t>(rows) * (kStepKeys * steps + 4)); }
};
static LogitPlace logit_place(int64_t rows, int dp, int tiles, bool values)
{
    LogitPlace p{};
    p.rows = static_cast<int>(std::min<int64_t>(rows, 16 * tiles));
    p.ends_at = static_cast<int>((values ? meet_bytes(dp, kFewWaves, p.rows) / sizeof(float) : 2 * kFewWaves * p.rows) + 3) / 4 * 4;
    p.logits_at = p.ends_at + 4 * p.rows;
    const int room = static_cast<int>((p.logits_at > 10000 ? kLdsBytes - 4096 : kLdsBytes / 2) / sizeof(float));
    p.most = (room - p.logits_at - 4 * p.rows) / (kStepKeys * p.rows);
    return p;
}
static int padded_dim(int32_t head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

template <bool BF16, int DP, bool FULL, int R, int MODE>
static int launch_cache(const CacheAttnArgs& a, int64_t blocks, hipStream_t s)
{
    const size_t lds = MODE != kOutputs ? logit_place(a.rows, DP, R, MODE == kBoth).bytes(a.logit_steps) : meet_bytes(DP, kFewWaves, 16 * R);
    const auto kernel = attn_cache_kernel<BF16, DP, FULL, R, MODE>;
    static std::atomic<uint64_t> done{0};
    const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), kLdsBytes, &done);
    if (rc != CIVIC_OK) return rc;
    civic::launch(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kFewThreads), lds, s, a);
    return check_launch();
}

template <bool BF16, int MODE>
static int launch_cache_dim(const CacheAttnArgs& a, int tiles, int64_t blocks, hipStream_t s)
{
    const int d = a.head_dim;
    if constexpr (BF16 && MODE != kLogits) {
        if (tiles == 2) {
            if (d == 64) return launch_cache<true, 64, true, 2, MODE>(a, blocks, s);
            if (d == 128) return launch_cache<true, 128, true, 2, MODE>(a, blocks, s);
            return d < 64 ? launch_cache<true, 64, false, 2, MODE>(a, blocks, s) : launch_cache<true, 128, false, 2, MODE>(a, blocks, s);
        }
    }
    if (d == 64) return launch_cache<BF16, 64, true, 1, MODE>(a, blocks, s);
    if (d == 128) return launch_cache<BF16, 128, true, 1, MODE>(a, blocks, s);
    if (d == 256) return launch_cache<BF16, 256, true, 1, MODE>(a, blocks, s);
    if (d < 64) return launch_cache<BF16, 64, false, 1, MODE>(a, blocks, s);
    return d < 128 ? launch_cache<BF16, 128, false, 1, MODE>(a, blocks, s) : launch_cache<BF16, 256, false, 1, MODE>(a, blocks, s);
}

template <int DP, int KG>
static int launch_rows(const CacheAttnArgs& a, int64_t blocks, hipStream_t s)
{
    const auto kernel = attn_cache_rows_kernel<DP, KG>;
    static std::atomic<uint64_t> done{0};
    const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), many_lds<DP, KG>(), &done);
    if (rc != CIVIC_OK) return rc;
    civic::launch(kernel, dim3(static_cast<unsigned>(blocks)), dim3(KG * kManyThreads), many_lds<DP, KG>(), s, a);
    return check_launch();
}
template <int DP, int R>
static int launch_mixed(const CacheAttnArgs& a, int64_t blocks, hipStream_t s)
{
    constexpr size_t few = meet_bytes(DP == 96 ? 128 : DP, kFewWaves, 16 * R), lds = std::max(many_lds<DP, 1>(), few);
    const auto kernel = attn_cache_mixed_kernel<DP, R>;
    static std::atomic<uint64_t> done{0};
    const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds, &done);
    if (rc != CIVIC_OK) return rc;
    civic::launch(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kManyThreads), lds, s, a);
    return check_launch();
}
template <int DP>
static int launch_many(const CacheAttnArgs& a, const CachePlan& p, hipStream_t s)
{
    if constexpr (DP <= 128) {
        if (p.kind == kRows && p.groups == 2) return launch_rows<DP, 2>(a, p.blocks, s);
        if (p.kind == kMixed && p.tiles == 2) return launch_mixed<DP, 2>(a, p.blocks, s);
    }
    return p.kind == kRows ? launch_rows<DP, 1>(a, p.blocks, s) : launch_mixed<DP, 1>(a, p.blocks, s);
}

// Logits of a row: whole steps, so that a step is stored without a check.
static int64_t logits_pitch(int64_t n_ctx) { return ceil_div(n_ctx, kStepKeys) * kStepKeys; }

static void fill_args(CacheAttnArgs& a, const CachePlan& p, const void* q, void* out, int dtype, int32_t batch, int32_t seq, int32_t n_q_heads,
                      int32_t n_kv_heads, int32_t head_dim, const int64_t* qs, const int64_t* os, int64_t s_max, int64_t n_prefix, int64_t n_ctx,
                      const int32_t* ctx, int32_t causal, float softmax_scale, void* workspace)
{
    a.q = q; a.out = out; a.ws = static_cast<float*>(workspace); a.ctx = ctx;
    for (int i = 0; i < 3; ++i) { a.qs[i] = qs[i]; a.os[i] = os[i]; }
    a.s_max = s_max;
    a.batch = batch; a.seq = seq; a.n_q_heads = n_q_heads; a.n_kv_heads = n_kv_heads; a.head_dim = head_dim; a.group = n_q_heads / n_kv_heads;
    a.causal = causal != 0;
    a.n_prefix = static_cast<int32_t>(n_prefix); a.n_ctx = static_cast<int32_t>(n_ctx);
    a.rows = seq * a.group;
    a.packed = p.packed;
    a.prefix_tiles = static_cast<int32_t>(p.prefix_tiles); a.row_tiles = static_cast<int32_t>(p.row_tiles);
    a.prefix_pieces = static_cast<int32_t>(p.prefix_pieces); a.own_pieces = static_cast<int32_t>(p.own_pieces);
    a.prefix_steps = static_cast<int32_t>(p.prefix_steps); a.own_steps = static_cast<int32_t>(p.own_steps);
    a.prefix_keys = p.prefix_keys; a.own_keys = p.own_keys;
    const LogitScale scale = logit_scale(softmax_scale, head_dim, dtype == CIVIC_BF16);
    a.scale = scale.log2; a.flip = scale.flip;
}

// Whether the strides of a q or out of these sizes are multiples of 16 bytes and hold whole heads.
static bool strides_ok(const int64_t* s, int32_t n_heads, int32_t head_dim, int esz)
{
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0 || (s[i] * esz) % 16) return false;
    return n_heads == 1 || s[2] >= head_dim;
}

static int shared_attn(const void* q, const void* k_prefix, const void* v_prefix, const void* k_cache, const void* v_cache, void* out, int dtype,
                       int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const int64_t* qs, const int64_t* os,
                       int64_t s_prefix, int64_t n_prefix, const int32_t* prefix_ctx, int64_t s_max, int64_t n_ctx, const int32_t* ctx,
                       int32_t causal, float softmax_scale, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!cache_sizes_ok(dtype, batch, seq, n_q_heads, n_kv_heads, head_dim, n_prefix, n_ctx) || !qs || !os) return CIVIC_ERR_INVALID_ARG;
    if (s_prefix < 0 || n_prefix > s_prefix || s_max < 0 || n_ctx > s_max || !std::isfinite(softmax_scale)) return CIVIC_ERR_INVALID_ARG;
    const bool any = batch > 0 && seq > 0;
    if (any && (!q || !out || (n_prefix > 0 && (!k_prefix || !v_prefix)) || (n_ctx > 0 && (!k_cache || !v_cache)))) return CIVIC_ERR_INVALID_ARG;
    for (const void* p : {q, k_prefix, v_prefix, k_cache, v_cache, static_cast<const void*>(out), static_cast<const void*>(workspace)})
        if (!aligned16(p)) return CIVIC_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(ctx) | reinterpret_cast<uintptr_t>(prefix_ctx)) & 3u) return CIVIC_ERR_INVALID_ARG;
    const int esz = dtype_size(dtype);
    if (!strides_ok(qs, n_q_heads, head_dim, esz) || !strides_ok(os, n_q_heads, head_dim, esz)) return CIVIC_ERR_INVALID_ARG;
    if (!cache_covered(batch, seq, n_q_heads, n_kv_heads, head_dim, s_prefix, s_max)) return CIVIC_ERR_UNSUPPORTED;
    if (!any) return CIVIC_OK;
    if (!rows_apart(os, batch, seq, n_q_heads, head_dim)) return CIVIC_ERR_INVALID_ARG;
    const int64_t rows = static_cast<int64_t>(seq) * (n_q_heads / n_kv_heads);
    const CachePlan p = cache_plan(dtype == CIVIC_BF16, false, batch, rows, n_kv_heads, head_dim, n_prefix, n_ctx);
    const size_t need = cache_ws_bytes(p, batch, rows, n_kv_heads, head_dim);
    if (need && (!workspace || workspace_bytes < need)) return CIVIC_ERR_WORKSPACE;
    // (a tile's workgroups have read its queries before its outputs are written: out may be q; and the rows of both may lie between each other's)
    const int64_t row_bytes = static_cast<int64_t>(n_kv_heads) * head_dim * esz, prefix_bytes = s_prefix * row_bytes, cache_bytes = batch * s_max * row_bytes;
    const Memory outputs{out, reach_bytes(os, batch, seq, n_q_heads, head_dim, esz)}, scratch{workspace, static_cast<int64_t>(need)};
    if (!writes_apart({outputs, scratch}, {{k_prefix, prefix_bytes}, {v_prefix, prefix_bytes}, {k_cache, cache_bytes}, {v_cache, cache_bytes},
                                           {ctx, batch * int64_t{4}}, {prefix_ctx, 4}})
        || !scratch.apart({q, reach_bytes(qs, batch, seq, n_q_heads, head_dim, esz)})) return CIVIC_ERR_INVALID_ARG;
    CacheAttnArgs a{};
    fill_args(a, p, q, out, dtype, batch, seq, n_q_heads, n_kv_heads, head_dim, qs, os, s_max, n_prefix, n_ctx, ctx, causal, softmax_scale, workspace);
    a.kp = k_prefix; a.vp = v_prefix; a.kc = k_cache; a.vc = v_cache; a.prefix_ctx = prefix_ctx; a.s_prefix = s_prefix;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int rc = p.kind != kFew ? head_dim == 64 ? launch_many<64>(a, p, s) : head_dim == 96 ? launch_many<96>(a, p, s)
                                   : head_dim == 128 ? launch_many<128>(a, p, s) : launch_many<256>(a, p, s)
                 : dtype == CIVIC_BF16 ? launch_cache_dim<true, kOutputs>(a, p.tiles, p.blocks, s) : launch_cache_dim<false, kOutputs>(a, p.tiles, p.blocks, s);
    if (rc != CIVIC_OK || a.prefix_pieces + a.own_pieces == 1) return rc;
    const int64_t all = static_cast<int64_t>(batch) * n_kv_heads * rows;
    const auto join = dtype == CIVIC_BF16 ? attn_cache_join_kernel<true> : attn_cache_join_kernel<false>;
    civic::launch(join, dim3(static_cast<unsigned>(ceil_div(all, 4))), dim3(256), 0, s, a, p.own_tile);
    return check_launch();
}

static size_t logits_ws_bytes(const CachePlan& p, int64_t pairs, int64_t rows, int64_t n_ctx, int32_t values)
{
    return n_ctx == 0 ? 0 : sizeof(float) * static_cast<size_t>(pairs) * rows * (p.most_pieces * (values + 2) + logits_pitch(n_ctx)) + 16;
}

// Attention that keeps its logits, in one launch or two; out = null: no outputs, V is not read.
static int logits_attn(CacheAttnArgs& a, const CachePlan& p, int dtype, hipStream_t s)
{
    const bool values = a.out != nullptr, bf16 = dtype == CIVIC_BF16;
    a.pitch = static_cast<int32_t>(logits_pitch(a.n_ctx));
    const LogitPlace at = logit_place(a.rows, padded_dim(a.head_dim), p.tiles, values);
    a.logit_steps = static_cast<int32_t>(std::min<int64_t>(at.most, p.own_steps));
    a.ends_at = at.ends_at; a.logits_at = at.logits_at;
    a.fused = p.own_pieces == 1 && p.row_tiles == 1 && p.own_steps <= at.most;
    const bool here = a.weights == a.base;                     // (rows behind a context stay as they are)
    const unsigned behind = a.fused && !here ? behind_blocks(p.blocks, a.s_max, a.n_ctx, kFewThreads) : 0;
    a.items = static_cast<uint32_t>(p.blocks);
    a.written = here ? 0 : behind ? a.n_ctx : a.s_max;
    const int64_t blocks = p.blocks + behind;
    const int rc = values ? bf16 ? launch_cache_dim<true, kBoth>(a, p.tiles, blocks, s) : launch_cache_dim<false, kBoth>(a, p.tiles, blocks, s)
                          : bf16 ? launch_cache_dim<true, kLogits>(a, p.tiles, blocks, s) : launch_cache_dim<false, kLogits>(a, p.tiles, blocks, s);
    if (rc != CIVIC_OK || a.fused) return rc;
    const auto sums = bf16 ? attn_cache_sums_kernel<true> : attn_cache_sums_kernel<false>;
    civic::launch(sums, dim3(static_cast<unsigned>(a.batch) * a.n_kv_heads, static_cast<unsigned>(1 + ceil_div(here ? a.n_ctx : a.s_max, kSumKeys))), dim3(256), 0, s, a, p.own_tile);
    return check_launch();
}

size_t few_weights_bytes(int dtype, int32_t batch, int64_t rows, int32_t n_kv_heads, int32_t head_dim, int64_t n_ctx)
{
    return logits_ws_bytes(cache_plan(dtype == CIVIC_BF16, true, batch, rows, n_kv_heads, head_dim, 0, n_ctx), static_cast<int64_t>(batch) * n_kv_heads, rows, n_ctx, 0);
}

int few_weights(const void* q, const void* k_cache, const float* base, float* weights, int dtype, int32_t batch, int32_t seq, int32_t n_q_heads,
                int32_t n_kv_heads, int32_t head_dim, const int64_t* qs, int64_t s_max, int64_t n_ctx, const int32_t* ctx, int32_t causal,
                float softmax_scale, void* workspace, void* stream)
{
    const CachePlan p = cache_plan(dtype == CIVIC_BF16, true, batch, static_cast<int64_t>(seq) * (n_q_heads / n_kv_heads), n_kv_heads, head_dim, 0, n_ctx);
    CacheAttnArgs a{};
    fill_args(a, p, q, nullptr, dtype, batch, seq, n_q_heads, n_kv_heads, head_dim, qs, qs, s_max, 0, n_ctx, ctx, causal, softmax_scale, workspace);
    a.kc = k_cache; a.base = base; a.weights = weights;
    return logits_attn(a, p, dtype, static_cast<hipStream_t>(stream));
}

}  // namespace civic

extern "C" size_t civic_attn_shared_workspace_bytes(int dtype, int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                                    int64_t n_prefix, int64_t n_ctx)
{
    using namespace civic;
    if (!cache_sizes_ok(dtype, batch, seq, n_q_heads, n_kv_heads, head_dim, n_prefix, n_ctx)
        || !cache_covered(batch, seq, n_q_heads, n_kv_heads, head_dim, n_prefix, n_ctx) || batch == 0 || seq == 0) return 0;
    const int64_t rows = static_cast<int64_t>(seq) * (n_q_heads / n_kv_heads);
    return cache_ws_bytes(cache_plan(dtype == CIVIC_BF16, false, batch, rows, n_kv_heads, head_dim, n_prefix, n_ctx), batch, rows, n_kv_heads, head_dim);
}

extern "C" int civic_decode_attn_shared(const void* q, const void* k_prefix, const void* v_prefix, const void* k_cache, const void* v_cache, void* out,
                                        int dtype, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t s_prefix,
                                        int64_t n_prefix, const int32_t* prefix_ctx, int64_t s_max, int64_t n_ctx, const int32_t* ctx,
                                        float softmax_scale, void* workspace, size_t workspace_bytes, void* stream)
{
    const int64_t row = static_cast<int64_t>(n_q_heads) * head_dim;
    const int64_t strides[3] = {row, row, head_dim};
    return civic::shared_attn(q, k_prefix, v_prefix, k_cache, v_cache, out, dtype, batch, 1, n_q_heads, n_kv_heads, head_dim, strides, strides, s_prefix,
                              n_prefix, prefix_ctx, s_max, n_ctx, ctx, 0, softmax_scale, workspace, workspace_bytes, stream);
}

extern "C" int civic_prefill_attn_shared(const void* q, const void* k_prefix, const void* v_prefix, const void* k_cache, const void* v_cache, void* out,
                                         int dtype, int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                         const int64_t* q_strides, const int64_t* o_strides, int64_t s_prefix, int64_t n_prefix,
                                         const int32_t* prefix_ctx, int64_t s_max, int64_t n_ctx, const int32_t* ctx, int32_t causal,
                                         float softmax_scale, void* workspace, size_t workspace_bytes, void* stream)
{
    return civic::shared_attn(q, k_prefix, v_prefix, k_cache, v_cache, out, dtype, batch, seq, n_q_heads, n_kv_heads, head_dim, q_strides, o_strides,
                              s_prefix, n_prefix, prefix_ctx, s_max, n_ctx, ctx, causal, softmax_scale, workspace, workspace_bytes, stream);
}

extern "C" size_t civic_decode_attn_weights_workspace_bytes(int dtype, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t n_ctx)
{
    using namespace civic;
    if (!cache_sizes_ok(dtype, batch, 1, n_q_heads, n_kv_heads, head_dim, 0, n_ctx)
        || !cache_covered(batch, 1, n_q_heads, n_kv_heads, head_dim, 0, n_ctx) || batch == 0 || n_ctx == 0) return 0;
    const int64_t rows = n_q_heads / n_kv_heads;
    const CachePlan p = cache_plan(dtype == CIVIC_BF16, true, batch, rows, n_kv_heads, head_dim, 0, n_ctx);
    return logits_ws_bytes(p, static_cast<int64_t>(batch) * n_kv_heads, rows, n_ctx, head_dim);
}

extern "C" int civic_decode_attn_weights(const void* q, const void* k_cache, const void* v_cache, void* out, const float* base, float* weights, int dtype,
                                         int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t s_max, int64_t n_ctx,
                                         const int32_t* ctx, float softmax_scale, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace civic;
    if (!cache_sizes_ok(dtype, batch, 1, n_q_heads, n_kv_heads, head_dim, 0, n_ctx)) return CIVIC_ERR_INVALID_ARG;
    if (s_max < 0 || n_ctx > s_max || !std::isfinite(softmax_scale)) return CIVIC_ERR_INVALID_ARG;
    if (batch > 0 && (!q || !out || (s_max > 0 && !weights) || (n_ctx > 0 && (!k_cache || !v_cache)))) return CIVIC_ERR_INVALID_ARG;
    for (const void* p : {q, k_cache, v_cache, static_cast<const void*>(out), static_cast<const void*>(workspace)})
        if (!aligned16(p)) return CIVIC_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(base), static_cast<const void*>(weights), static_cast<const void*>(ctx)})
        if (reinterpret_cast<uintptr_t>(p) & 3u) return CIVIC_ERR_INVALID_ARG;
    if (!cache_covered(batch, 1, n_q_heads, n_kv_heads, head_dim, 0, s_max)) return CIVIC_ERR_UNSUPPORTED;
    if (batch == 0) return CIVIC_OK;
    if (!same_or_apart(base, weights, static_cast<int64_t>(batch) * n_kv_heads * s_max * 4)) return CIVIC_ERR_INVALID_ARG;
    const int64_t rows = n_q_heads / n_kv_heads;
    const size_t need = civic_decode_attn_weights_workspace_bytes(dtype, batch, n_q_heads, n_kv_heads, head_dim, n_ctx);
    if (need && (!workspace || workspace_bytes < need)) return CIVIC_ERR_WORKSPACE;
    // (a tile's workgroups have read its queries before the outputs are written: out may be q)
    const int64_t esz = dtype_size(dtype), sums = static_cast<int64_t>(batch) * n_kv_heads * s_max * 4, cache = sums / 4 * head_dim * esz;
    const Memory queries{q, static_cast<int64_t>(batch) * n_q_heads * head_dim * esz}, outputs{out, queries.bytes}, scratch{workspace, static_cast<int64_t>(need)};
    if (!writes_apart({{weights, sums}, outputs, scratch}, {{k_cache, cache}, {v_cache, cache}, {ctx, batch * int64_t{4}}})
        || !writes_apart({{weights, sums}, scratch}, {queries}) || (out != q && !outputs.apart(queries))
        || !writes_apart({outputs, scratch}, {{base, sums}})) return CIVIC_ERR_INVALID_ARG;
    const CachePlan p = cache_plan(dtype == CIVIC_BF16, true, batch, rows, n_kv_heads, head_dim, 0, n_ctx);
    const int64_t row = static_cast<int64_t>(n_q_heads) * head_dim;
    const int64_t strides[3] = {row, row, head_dim};
    CacheAttnArgs a{};
    fill_args(a, p, q, out, dtype, batch, 1, n_q_heads, n_kv_heads, head_dim, strides, strides, s_max, 0, n_ctx, ctx, 0, softmax_scale, workspace);
    a.kc = k_cache; a.vc = v_cache; a.base = base; a.weights = weights;
    return logits_attn(a, p, dtype, static_cast<hipStream_t>(stream));
}
