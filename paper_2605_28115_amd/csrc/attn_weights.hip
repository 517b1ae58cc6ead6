// civic_attn_weights: how much attention each cache row has received from new tokens,
//
//   weights[b, g, j] = base[b, g, j] + sum_{i, h in g} e(i, h, j) / sum_k e(i, h, k),   e = exp(scale <q[b, i, h], K[b, g, j]>),
//   j, k < ctx[b] - (seq - 1 - i) when causal, < ctx[b] else.
//
// A row's weights need the row's sum first.  The queries of a KV head are rows r = token * group + head of the group; by their number, R:
//   - up to 16: the decode's kernel without V (attn_cache.hip), which keeps the logits: four bytes for a row and key.
//   - up to 64 over a short cache: one launch that holds the logits in registers.
//   - more: keeping the logits would write and read as much as K at 64 rows of 128 bf16 channels, and there are hundreds, so the product
//     Q K^T is made twice: once over the keys for every row's base and sum, once over the rows for every key's total.
// The plain pair of launches (fp32, wide heads, up to 96 rows) has one shape: a wavefront holds 16 G rows of one side in registers, as columns
// of its products, and reads the other side in tiles of 16 rows from memory as they lie; the lanes of a column add up what they see, four
// results of a tile each, so that nothing crosses lanes before the end.  The wavefronts of a workgroup have the same columns and take turns
// over the tiles; they meet in LDS.  No atomics: a total's order of summation is the same on every call.
// Vector work per result: a fused multiply-add, an exponential and an addition (a second multiply-add in the second launch).
#include "rows_device.h"
#include "tile_device.h"

namespace civic {

constexpr int kWgtWaves = 4, kWgtThreads = kWgtWaves * kWave;
constexpr int kWgtMaxPieces = 64;
constexpr int kWgtInline = 4;                                 // up to so many pieces the second launch joins them itself
constexpr int kWgtRows = 2048;                                // query rows whose sums are in LDS at a time

struct WeightsArgs {
    const void* q; const void* kc;
    const int32_t* ctx;
    const float* base; float* weights;
    float2* stats;                                            // [pairs, pieces, rows] (base, sum); joined, in piece 0: (base, 1 / sum)
    int64_t qs[3];
    int64_t s_max;
    int32_t batch, seq, n_q_heads, n_kv_heads, head_dim, group, causal, n_ctx;
    int32_t rows;                                             // of a pair of sample and KV head: seq * group
    int32_t row_tiles, pieces, piece_tiles;                   // first launch: tiles of 16 keys of a piece
    int32_t joined;                                           // whether the second launch finds the pieces joined
    float* parts;                                             // [pairs, row_pieces, pitch] totals of the second launch's pieces
    int32_t row_pieces, row_piece_tiles, key_tiles, pitch;               // its pieces, tiles of 64 query rows of each; row_pieces = 1: no parts
    uint32_t pairs;                                           // one launch: workgroups of pairs; those behind them write rows from `written` on
    int64_t written;                                          // rows of a pair that are written; one launch: by its workgroup (its context's in any case)
    float scale;                                              // times log2 e
    uint32_t flip;
};

__device__ __forceinline__ int keys_seen(const WeightsArgs& a, int own, int r)
{
    return r >= a.rows ? 0 : a.causal ? max(own - (a.seq - 1 - r / a.group), 0) : own;
}

// 16 bytes at byte 64 t + 16 kq of a row, zeros past its end
template <bool FULL, int KT>
__device__ __forceinline__ void load_row(const char* row, int kq, uint32_t row_bytes, u32x4 (&f)[KT])
{
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        f[t] = u32x4{0u, 0u, 0u, 0u};
        if (FULL || 64 * t + 16 * kq < static_cast<int>(row_bytes)) f[t] = *reinterpret_cast<const u32x4*>(row + 64 * t + 16 * kq);
    }
}

template <bool BF16, int DP> constexpr int wgt_chunks() { return DP * (BF16 ? 2 : 4) / 64; }
// Column tiles that the registers hold: 128 of a lane for the operands.
template <bool BF16, int DP> constexpr int wgt_most_columns() { return wgt_chunks<BF16, DP>() <= 4 ? 8 : 32 / wgt_chunks<BF16, DP>(); }

// Two pieces' (base, sum) as one.
__device__ __forceinline__ float2 with(float2 s, float2 y)
{
    const float to = fmaxf(s.x, y.x);
    return make_float2(to, fmaf(base_step(s.x, to), s.y, base_step(y.x, to) * y.y));
}
// A row's (base, sum) over its pieces, `stride` apart.
__device__ __forceinline__ float2 over_pieces(const float2* st, int stride, int n)
{
    constexpr int U = 8;
    float2 s = make_float2(-INFINITY, 0.f);
    for (int p0 = 0; p0 < n; p0 += U) {
        float2 y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) y[u] = p0 + u < n ? st[static_cast<int64_t>(p0 + u) * stride] : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int u = 0; u < U; ++u) s = with(s, y[u]);
    }
    return s;
}
// What the second launch takes of a row: its base and the reciprocal of its sum (nothing seen: 0, so that it adds nothing; NaN: in the base
// alone, so that a weight of 0 in its place, of a key that the row does not see, adds nothing).
__device__ __forceinline__ float2 joined(float2 s)
{
    if (s.y != s.y) return make_float2(s.y, 1.f);
    return make_float2(s.x == -INFINITY ? 0.f : s.x, s.y == 0.f ? 0.f : 1.f / s.y);
}

// The query rows' bases and sums.  Columns: query rows; tiles: keys.
template <bool BF16, int DP, bool FULL, int G>
__global__ __launch_bounds__(kWgtThreads, 2) void weights_stats_kernel(WeightsArgs a)
{
    constexpr int ESZ = BF16 ? 2 : 4, KT = wgt_chunks<BF16, DP>();
    __shared__ float sm_b[kWgtWaves][16 * G], sm_l[kWgtWaves][16 * G];
    const int lane = threadIdx.x & (kWave - 1), w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, kq = lane >> 4;
    const uint32_t pairs = static_cast<uint32_t>(a.batch) * a.n_kv_heads, v = blockIdx.x / pairs, pair = blockIdx.x - v * pairs;
    const int piece = v % a.pieces, tile = a.row_tiles - 1 - v / a.pieces;      // the heaviest causal tiles first
    const int b = pair / a.n_kv_heads, g = pair - b * a.n_kv_heads;
    const int own = clamped(a.ctx, b, a.n_ctx);
    const uint32_t row_bytes = static_cast<uint32_t>(FULL ? DP : a.head_dim) * ESZ;
    const int r0 = tile * 16 * G;
    const int sees = keys_seen(a, own, min(r0 + 16 * G, a.rows) - 1), all_see = keys_seen(a, own, r0);
    const int t1 = min((piece + 1) * a.piece_tiles, (sees + 15) / 16);
    u32x4 qf[G][KT];
    int lim[G];
    {
        int r = r0 + l16, token = r / a.group, head = r - token * a.group;
        const int token_step = 16 / a.group, head_step = 16 - token_step * a.group;
        const char* const q = static_cast<const char*>(a.q) + (b * a.qs[0] + g * a.group * a.qs[2]) * ESZ;
#pragma unroll
        for (int x = 0; x < G; ++x) {                          // (rows past the last: the last token's, that see nothing)
            lim[x] = r + 16 * x >= a.rows ? 0 : a.causal ? max(own - (a.seq - 1 - token), 0) : own;
            load_row<FULL>(q + (min(token, a.seq - 1) * a.qs[1] + head * a.qs[2]) * ESZ, kq, row_bytes, qf[x]);
            token += token_step; head += head_step;
            if (head >= a.group) { head -= a.group; ++token; }
        }
    }
    if (a.flip) {
#pragma unroll
        for (int x = 0; x < G; ++x)
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) qf[x][t][e] ^= a.flip;
    }
    const char* const keys = static_cast<const char*>(a.kc) + static_cast<int64_t>(pair) * a.s_max * row_bytes;
    auto fetch = [&](int t, u32x4 (&kf)[KT]) __attribute__((always_inline)) {   // (keys past the last re-read it)
        load_row<FULL>(keys + static_cast<int64_t>(min(16 * t + l16, own - 1)) * row_bytes, kq, row_bytes, kf);
    };
    // A column's weights are taken against its first tile's largest logit, and against a later one when they add up to more than 2^64.
    float base[G], l[G];
#pragma unroll
    for (int x = 0; x < G; ++x) { base[x] = -INFINITY; l[x] = 0.f; }
    auto turn = [&](int t, u32x4 (&kf)[KT]) __attribute__((always_inline)) {
        row_f32x4 s[G];
#pragma unroll
        for (int x = 0; x < G; ++x) s[x] = row_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KT; ++c)
#pragma unroll
            for (int x = 0; x < G; ++x) s[x] = mma16<BF16>(kf[c], qf[x][c], s[x]);
        if (t + 2 * kWgtWaves < t1) fetch(t + 2 * kWgtWaves, kf);
        if (16 * t + 16 > all_see) {
#pragma unroll
            for (int x = 0; x < G; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[x][r] = 16 * t + 4 * kq + r < lim[x] ? s[x][r] : -INFINITY;
        }
        float sum[G], most = 0.f;
#pragma unroll
        for (int x = 0; x < G; ++x) {                          // (no base yet: infinite or NaN)
            sum[x] = l[x];
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[x] += __builtin_amdgcn_exp2f(fmaf(s[x][r], a.scale, -base[x]));
            most = sum[x] <= 0x1p64f ? most : 1.f;
        }
        if (__any(most != 0.f)) {
#pragma unroll
            for (int x = 0; x < G; ++x) {
                const float top = fmaxf(fmaxf(s[x][0], s[x][1]), fmaxf(s[x][2], s[x][3])) * a.scale;
                const float to = top > base[x] ? rintf(top) : base[x], off = to == -INFINITY ? 0.f : to;
                sum[x] = l[x] * base_step(base[x], to);
                base[x] = to;
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[x] += __builtin_amdgcn_exp2f(fmaf(s[x][r], a.scale, -off));
            }
        }
#pragma unroll
        for (int x = 0; x < G; ++x) l[x] = sum[x];
    };
    u32x4 kf[2][KT];
    int t = piece * a.piece_tiles + w;
    if (t < t1) fetch(t, kf[0]);
    if (t + kWgtWaves < t1) fetch(t + kWgtWaves, kf[1]);
    for (; t < t1; t += 2 * kWgtWaves) {
        turn(t, kf[0]);
        if (t + kWgtWaves < t1) turn(t + kWgtWaves, kf[1]);
    }
#pragma unroll
    for (int x = 0; x < G; ++x) {
        const float to = rows_max(base[x]), sum = rows_sum(l[x] * base_step(base[x], to));
        if (kq == 0) { sm_b[w][16 * x + l16] = to; sm_l[w][16 * x + l16] = sum; }
    }
    __syncthreads();
    const int i = threadIdx.x;
    if (i < 16 * G && r0 + i < a.rows) {
        float to = sm_b[0][i], sum = 0.f;
#pragma unroll
        for (int x = 1; x < kWgtWaves; ++x) to = fmaxf(to, sm_b[x][i]);
#pragma unroll
        for (int x = 0; x < kWgtWaves; ++x) sum = fmaf(base_step(sm_b[x][i], to), sm_l[x][i], sum);
        a.stats[(static_cast<int64_t>(pair) * a.pieces + piece) * a.rows + r0 + i] = a.pieces == 1 ? joined(make_float2(to, sum)) : make_float2(to, sum);
    }
}

// Joins the pieces of the query rows, into the first.  A thread takes a row.
__global__ __launch_bounds__(256) void weights_join_kernel(WeightsArgs a)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, pair = i / a.rows;
    if (pair >= static_cast<int64_t>(a.batch) * a.n_kv_heads) return;
    float2* const st = a.stats + pair * a.pieces * a.rows + (i - pair * a.rows);
    st[0] = joined(over_pieces(st, a.rows, a.pieces));
}

// The keys' totals.  Columns: keys; tiles: query rows.  grid: pairs, then the column tiles along y and z
template <bool BF16, int DP, bool FULL, int G>
__global__ __launch_bounds__(kWgtThreads, 2) void weights_sums_kernel(WeightsArgs a)
{
    constexpr int ESZ = BF16 ? 2 : 4, KT = wgt_chunks<BF16, DP>();
    __shared__ __attribute__((aligned(16))) float2 sm_s[kWgtRows];              // of a query row: base, 1 / sum;
    __shared__ __attribute__((aligned(16))) int sm_lim[kWgtRows];               // keys from key0 on that it sees
    __shared__ float sm_a[kWgtWaves][16 * G];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, kq = lane >> 4;
    const uint32_t pair = blockIdx.x;
    const int b = pair / a.n_kv_heads, g = pair - b * a.n_kv_heads;
    const int own = clamped(a.ctx, b, a.n_ctx);
    const uint32_t row_bytes = static_cast<uint32_t>(FULL ? DP : a.head_dim) * ESZ;
    const int64_t key0 = (static_cast<int64_t>(blockIdx.z) * gridDim.y + blockIdx.y) * 16 * G;
    float acc[G];
#pragma unroll
    for (int x = 0; x < G; ++x) acc[x] = 0.f;
    if (key0 < own) {
        const int k0 = static_cast<int>(key0), keys = min(16 * G, own - k0);
        u32x4 kf[G][KT];
#pragma unroll
        for (int x = 0; x < G; ++x)
            load_row<FULL>(static_cast<const char*>(a.kc) + (static_cast<int64_t>(pair) * a.s_max + k0 + min(16 * x + l16, keys - 1)) * row_bytes, kq, row_bytes, kf[x]);
        if (a.flip) {
#pragma unroll
            for (int x = 0; x < G; ++x)
#pragma unroll
                for (int c = 0; c < KT; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) kf[x][c][e] ^= a.flip;
        }
        // tiles of query rows that see any of the keys: from the first token whose limit passes key0
        const int tiles = (a.rows + 15) / 16;
        const int64_t r_first = a.causal ? static_cast<int64_t>(max(k0 - own + a.seq, 0)) * a.group : 0;
        int first = static_cast<int>(r_first / 16);
        for (int r0 = first * 16 / kWgtRows * kWgtRows; r0 < a.rows; r0 += kWgtRows) {
            const int end = min(r0 + kWgtRows, a.rows);
            __syncthreads();
            const float2* const stats = a.stats + static_cast<int64_t>(pair) * a.pieces * a.rows;
            for (int r = max(r0, first * 16) + tid; r < r0 + kWgtRows && r < tiles * 16; r += kWgtThreads) {
                float2 s = make_float2(0.f, 0.f);
                if (r < end) s = a.joined ? stats[r] : joined(over_pieces(stats + r, a.rows, a.pieces));
                sm_s[r - r0] = s;
                sm_lim[r - r0] = keys_seen(a, own, r) - k0;
            }
            __syncthreads();
            const int t1 = (end + 15) / 16;
            int t = max(r0 / 16, first) + w;
            // the lane's query row: token and head of the group, a round of tiles further each time
            int r = 16 * t + l16, token = r / a.group, head = r - token * a.group;
            const int token_step = 16 * kWgtWaves / a.group, head_step = 16 * kWgtWaves - token_step * a.group;
            const char* const q = static_cast<const char*>(a.q) + (b * a.qs[0] + g * a.group * a.qs[2]) * ESZ;
            auto fetch = [&](u32x4 (&qf)[KT]) __attribute__((always_inline)) {  // (rows past the last re-read the last token's)
                load_row<FULL>(q + (min(token, a.seq - 1) * a.qs[1] + head * a.qs[2]) * ESZ, kq, row_bytes, qf);
                token += token_step; head += head_step;
                if (head >= a.group) { head -= a.group; ++token; }
            };
            auto turn = [&](int t, u32x4 (&qf)[KT]) __attribute__((always_inline)) {
                row_f32x4 s[G];
#pragma unroll
                for (int x = 0; x < G; ++x) s[x] = row_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < KT; ++c)
#pragma unroll
                    for (int x = 0; x < G; ++x) s[x] = mma16<BF16>(qf[c], kf[x][c], s[x]);
                if (t + 2 * kWgtWaves < t1) fetch(qf);
                float2 st[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) st[e] = sm_s[16 * t - r0 + 4 * kq + e];
                const int4 lim = *reinterpret_cast<const int4*>(sm_lim + 16 * t - r0 + 4 * kq);
#pragma unroll
                for (int x = 0; x < G; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[x][e] = __builtin_amdgcn_exp2f(fmaf(s[x][e], a.scale, -st[e].x));
                if (!__all(min(min(lim.x, lim.y), min(lim.z, lim.w)) >= 16 * G)) {
                    const int lims[4] = {lim.x, lim.y, lim.z, lim.w};
#pragma unroll
                    for (int x = 0; x < G; ++x)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[x][e] = 16 * x + l16 < lims[e] ? s[x][e] : 0.f;
                }
#pragma unroll
                for (int x = 0; x < G; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[x] = fmaf(s[x][e], st[e].y, acc[x]);
            };
            u32x4 qf[2][KT];
            if (t < t1) fetch(qf[0]);
            if (t + kWgtWaves < t1) fetch(qf[1]);
            for (; t < t1; t += 2 * kWgtWaves) {
                turn(t, qf[0]);
                if (t + kWgtWaves < t1) turn(t + kWgtWaves, qf[1]);
            }
        }
    }
#pragma unroll
    for (int x = 0; x < G; ++x) {
        const float sum = rows_sum(acc[x]);
        if (kq == 0) sm_a[w][16 * x + l16] = sum;
    }
    __syncthreads();
    if (tid < 16 * G && key0 + tid < a.s_max) {
        const int64_t at = static_cast<int64_t>(pair) * a.s_max + key0 + tid;
        const float had = a.base ? a.base[at] : 0.f;
        if (key0 + tid < own) {
            float sum = 0.f;
#pragma unroll
            for (int x = 0; x < kWgtWaves; ++x) sum += sm_a[x][tid];
            a.weights[at] = had + sum;
        }
        else if (a.weights != a.base) a.weights[at] = had;
    }
}

// ------------------------------------------------------------------------------------------------------------- short caches
// Query rows over a cache that a workgroup holds the logits of in registers, 16 G rows by 128 T keys: one launch, one product.  Here the two
// launches above are most of the time (64 rows over 469 keys, 16 / 8 heads of 128: 6.9 and 5.5 us).  Columns: query rows; tiles: keys.
constexpr int kShortWaves = 8, kShortThreads = kShortWaves * kWave;

template <int CTRL>
__device__ __forceinline__ float dpp(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false)); }

template <bool BF16, int DP, bool FULL, int G, int T>
__global__ __launch_bounds__(kShortThreads, 2) void weights_short_kernel(WeightsArgs a)
{
    constexpr int ESZ = BF16 ? 2 : 4, KT = wgt_chunks<BF16, DP>();
    __shared__ float sm_b[kShortWaves][16 * G], sm_l[kShortWaves][16 * G];
    if (blockIdx.x >= a.pairs) {
        weights_behind<kShortThreads>(a.base, a.weights, a.pairs, a.s_max, a.written, blockIdx.x - a.pairs, gridDim.x - a.pairs);
        return;
    }
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, kq = lane >> 4;
    const int pair = blockIdx.x, b = pair / a.n_kv_heads, g = pair - b * a.n_kv_heads;
    const int own = clamped(a.ctx, b, a.n_ctx);
    const uint32_t row_bytes = static_cast<uint32_t>(FULL ? DP : a.head_dim) * ESZ;
    const int tiles = (own + 15) / 16;
    const char* const keys = static_cast<const char*>(a.kc) + static_cast<int64_t>(pair) * a.s_max * row_bytes;
    // everything is asked for at once: the time is that of a few trips to memory one after the other
    u32x4 kf[T][KT];
#pragma unroll
    for (int t = 0; t < T; ++t) {                              // (keys past the last re-read it: their logits are masked)
        const int tile = w + kShortWaves * t;
        if (tile < tiles) load_row<FULL>(keys + static_cast<int64_t>(min(16 * tile + l16, own - 1)) * row_bytes, kq, row_bytes, kf[t]);
    }
    const int64_t first = static_cast<int64_t>(pair) * a.s_max;
    float had[T];                                              // of the key that the lane writes (l16 < 4)
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int key = 16 * (w + kShortWaves * t) + 4 * kq + l16;
        had[t] = a.base && l16 < 4 && key < own ? a.base[first + key] : 0.f;
    }
    u32x4 qf[G][KT];
    int lim[G];
#pragma unroll
    for (int x = 0; x < G; ++x) {                              // (rows past the last: the last, seeing nothing)
        const int r = 16 * x + l16, rr = min(r, a.rows - 1), token = rr / a.group, head = g * a.group + (rr - token * a.group);
        lim[x] = keys_seen(a, own, r);
        load_row<FULL>(static_cast<const char*>(a.q) + (b * a.qs[0] + token * a.qs[1] + head * a.qs[2]) * ESZ, kq, row_bytes, qf[x]);
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) qf[x][t][e] ^= a.flip;
    }
    row_f32x4 s[T][G];
    float base[G], sum[G];
#pragma unroll
    for (int x = 0; x < G; ++x) { base[x] = -INFINITY; sum[x] = 0.f; }
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int k0 = 16 * (w + kShortWaves * t) + 4 * kq;
#pragma unroll
        for (int x = 0; x < G; ++x) {
            s[t][x] = row_f32x4{0.f, 0.f, 0.f, 0.f};
            if (w + kShortWaves * t < tiles) {
#pragma unroll
                for (int c = 0; c < KT; ++c) s[t][x] = mma16<BF16>(kf[t][c], qf[x][c], s[t][x]);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[t][x][r] = k0 + r < lim[x] ? s[t][x][r] : -INFINITY;
                base[x] = fmaxf(base[x], s[t][x][r]);
            }
        }
    }
    // a column's base over the wavefronts, then its sum
#pragma unroll
    for (int x = 0; x < G; ++x) {
        const float top = rows_max(base[x]);
        if (kq == 0) sm_b[w][16 * x + l16] = top;
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < G; ++x) {
        float top = sm_b[0][16 * x + l16];
#pragma unroll
        for (int y = 1; y < kShortWaves; ++y) top = fmaxf(top, sm_b[y][16 * x + l16]);
        const float off = top == -INFINITY ? 0.f : rintf(top * a.scale);
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[t][x][r] = __builtin_amdgcn_exp2f(fmaf(s[t][x][r], a.scale, -off));
                sum[x] += s[t][x][r];
            }
        sum[x] = rows_sum(sum[x]);
        if (kq == 0) sm_l[w][16 * x + l16] = sum[x];
    }
    __syncthreads();
    bool odd = false;
#pragma unroll
    for (int x = 0; x < G; ++x) {
        float l = 0.f;
#pragma unroll
        for (int y = 0; y < kShortWaves; ++y) l += sm_l[y][16 * x + l16];
        sum[x] = l == 0.f ? 0.f : 1.f / l;
        odd |= l != l;
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int k0 = 16 * (w + kShortWaves * t) + 4 * kq;
        if (__any(odd)) {                                      // (a row that is NaN has a weight of 0 for a key that it does not see)
#pragma unroll
            for (int x = 0; x < G; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[t][x][r] = k0 + r < lim[x] ? s[t][x][r] * sum[x] : 0.f;
        } else {
#pragma unroll
            for (int x = 0; x < G; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[t][x][r] *= sum[x];
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float y = s[t][0][r];
#pragma unroll
            for (int x = 1; x < G; ++x) y += s[t][x][r];
            y += dpp<0xB1>(y);                                 // quad_perm [1,0,3,2]
            y += dpp<0x4E>(y);                                 // quad_perm [2,3,0,1]
            y += dpp<0x141>(y);                                // row_half_mirror
            y += dpp<0x140>(y);                                // row_mirror
            if (l16 == r && k0 + r < own) a.weights[first + k0 + r] = had[t] + y;
        }
    }
    for (int64_t key = own + tid; key < a.written; key += kShortThreads) a.weights[first + key] = a.base ? a.base[first + key] : 0.f;
}

// ------------------------------------------------------------------------------------------------------------- many rows
// bf16 heads of up to 128 channels and more than kWgtFewRows query rows a KV head: bound by the products and the exponentials.  A wavefront
// holds 64 rows of one side, a workgroup of four 256 different ones, and the other side goes through LDS in tiles of 64 rows, which all four
// read: a quarter of the fetches of the kernels above, and four times as many tiles to a wavefront, whose beginning (its rows, the first base)
// and end weigh less.  Threads hold the next tile in registers while the present one is computed, and lay it down in the other of two buffers.
// The lanes of v_mfma_f32_32x32x16_bf16's result are query rows in the first launch and keys in the second, its registers the other side, 8 (r / 4) +
// r % 4 + 4 (lane / 32): what a launch adds up stays in a lane but for one exchange at its end.  (The second with keys in the registers, 32 totals
// and a row's base and reciprocal sum in one register each: 288 vector instructions for 203 of the first, 44.6 us for 42.6 on 4 x 938 tokens.)
constexpr int kTileRows = 64, kTileCols = 256, kTileThreads = 256;
constexpr int kWgtFewRows = 96;
constexpr int64_t kUnits = 256;
typedef float tile_f32x16 __attribute__((ext_vector_type(16)));

// DP: 64 or 128 channels of a row in LDS; KS: 16-channel steps of the products
template <int DP> struct RowTile {
    static constexpr int PC = DP / 8, ROWB = DP * 2, BYTES = kTileRows * ROWB, NL = kTileRows * PC / kTileThreads, STEP = kTileThreads / PC;
};
// 16-byte piece `chunk` of row `row` of a tile
template <int DP>
__device__ __forceinline__ int tile_at(int row, int chunk) { return row * RowTile<DP>::ROWB + ((chunk ^ swz<RowTile<DP>::PC>(row)) << 4); }

// 64 rows in registers, as two operands of 32: channels 16 c + 8 half .. + 7 of row col
template <int KS>
__device__ __forceinline__ void load_rows32(const char* row, int half, int d, uint32_t flip, row_bf16x8 (&f)[KS])
{
#pragma unroll
    for (int c = 0; c < KS; ++c) {
        u32x4 v = u32x4{0u, 0u, 0u, 0u};
        if (16 * c + 8 * half < d) v = *reinterpret_cast<const u32x4*>(row + 32 * c + 16 * half);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] ^= flip;
        f[c] = __builtin_bit_cast(row_bf16x8, v);
    }
}

// The query rows' bases and sums: columns are query rows, tiles keys.
template <int DP, int KS>
__global__ __launch_bounds__(kTileThreads, 2) void weights_stats_tiles_kernel(WeightsArgs a)
{
    using T = RowTile<DP>;
    __shared__ __attribute__((aligned(16))) char lds[2 * T::BYTES];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
    const uint32_t pairs = static_cast<uint32_t>(a.batch) * a.n_kv_heads, v = blockIdx.x / pairs, pair = blockIdx.x - v * pairs;
    // (piece by piece, the heaviest causal tiles first: what a piece has nothing of is then a run of workgroups, not every n-th one, which would
    // leave the units that those are dealt out to without work)
    const int piece = v / a.row_tiles, tile = a.row_tiles - 1 - (v - piece * a.row_tiles);
    const int b = pair / a.n_kv_heads, g = pair - b * a.n_kv_heads, d = a.head_dim;
    const int own = clamped(a.ctx, b, a.n_ctx);
    const int r0 = tile * kTileCols, rw = r0 + 64 * w;
    const int t1 = min((piece + 1) * a.piece_tiles, (keys_seen(a, own, min(r0 + kTileCols, a.rows) - 1) + kTileRows - 1) / kTileRows);
    const int all_see = rw < a.rows ? keys_seen(a, own, rw) : own;              // of the wavefront's rows
    const int wave_sees = rw < a.rows ? keys_seen(a, own, min(rw + 64, a.rows) - 1) : 0;
    row_bf16x8 qf[2][KS];
    int lim[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {                              // (rows past the last repeat it)
        const int r = min(rw + 32 * u + col, a.rows - 1), token = r / a.group, head = g * a.group + (r - token * a.group);
        lim[u] = a.causal ? max(own - (a.seq - 1 - token), 0) : own;
        load_rows32<KS>(static_cast<const char*>(a.q) + (b * a.qs[0] + token * a.qs[1] + head * a.qs[2]) * 2, half, d, a.flip, qf[u]);
    }
    const char* const keys = static_cast<const char*>(a.kc) + static_cast<int64_t>(pair) * a.s_max * d * 2;
    const int row_t = tid / T::PC, chunk_t = tid - row_t * T::PC;
    u32x4 next[T::NL];
    auto fetch = [&](int t) __attribute__((always_inline)) {   // (keys past the last re-read it)
#pragma unroll
        for (int j = 0; j < T::NL; ++j) {
            const int key = min(t * kTileRows + j * T::STEP + row_t, own - 1);
            next[j] = u32x4{0u, 0u, 0u, 0u};
            if (chunk_t * 8 < d) next[j] = *reinterpret_cast<const u32x4*>(keys + static_cast<int64_t>(key) * d * 2 + chunk_t * 16);
        }
    };
    auto put = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < T::NL; ++j) *reinterpret_cast<u32x4*>(lds + buf * T::BYTES + tile_at<DP>(j * T::STEP + row_t, chunk_t)) = next[j];
    };
    float base[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    const char* at[KS];                                        // the lane's pieces of row col of a tile (row col + 32 lies 32 rows on)
#pragma unroll
    for (int c = 0; c < KS; ++c) at[c] = lds + tile_at<DP>(col, 2 * c + half);
    auto compute = [&](int t, auto buf) __attribute__((always_inline)) {
        constexpr int BUF = decltype(buf)::value * T::BYTES;
#pragma unroll
        for (int x = 0; x < 2; ++x) {                          // 32 keys
            tile_f32x16 s[2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[u][r] = 0.f;
#pragma unroll
            for (int c = 0; c < KS; ++c) {
                const row_bf16x8 kf = *reinterpret_cast<const row_bf16x8*>(at[c] + BUF + 32 * x * T::ROWB);
#pragma unroll
                for (int u = 0; u < 2; ++u) s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[u][c], s[u], 0, 0, 0);
            }
            const int k0 = t * kTileRows + 32 * x;
            if (k0 + 32 > all_see) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[u][r] = k0 + 8 * (r >> 2) + (r & 3) + 4 * half < lim[u] ? s[u][r] : -INFINITY;
            }
            // weights against the first keys' largest logit, and against a later one when they add up to more than 2^64 (no base yet: infinite
            // or NaN)
            float sum[2];
            bool outgrown = false;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float part[2] = {l[u], 0.f};
#pragma unroll
                for (int r = 0; r < 16; ++r) part[r & 1] += __builtin_amdgcn_exp2f(fmaf(s[u][r], a.scale, -base[u]));
                sum[u] = part[0] + part[1];
                outgrown |= !(sum[u] <= 0x1p64f);
            }
            if (__any(outgrown)) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float top = s[u][0];
#pragma unroll
                    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[u][r]);
                    top *= a.scale;
                    const float to = top > base[u] ? rintf(top) : base[u], off = to == -INFINITY ? 0.f : to;
                    float part[2] = {l[u] * base_step(base[u], to), 0.f};
                    base[u] = to;
#pragma unroll
                    for (int r = 0; r < 16; ++r) part[r & 1] += __builtin_amdgcn_exp2f(fmaf(s[u][r], a.scale, -off));
                    sum[u] = part[0] + part[1];
                }
            }
            l[0] = sum[0]; l[1] = sum[1];
        }
    };
    int t = piece * a.piece_tiles;
    if (t < t1) { fetch(t); put(0); }
    __syncthreads();
    auto turn = [&](auto buf) __attribute__((always_inline)) {
        if (t + 1 < t1) fetch(t + 1);
        if (t * kTileRows < wave_sees) compute(t, buf);
        if (t + 1 < t1) put(decltype(buf)::value ^ 1);
        __syncthreads();
        ++t;
    };
    while (t < t1) {
        turn(std::integral_constant<int, 0>{});
        if (t < t1) turn(std::integral_constant<int, 1>{});
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const auto bb = __builtin_amdgcn_permlane32_swap(__float_as_uint(base[u]), __float_as_uint(base[u]), false, false);
        const float b0 = __uint_as_float(bb[0]), b1 = __uint_as_float(bb[1]), to = fmaxf(b0, b1);
        const auto ll = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[u]), __float_as_uint(l[u]), false, false);
        const float sum = fmaf(base_step(b0, to), __uint_as_float(ll[0]), base_step(b1, to) * __uint_as_float(ll[1]));
        const int r = rw + 32 * u + col;
        if (half == 0 && r < a.rows)
            a.stats[(static_cast<int64_t>(pair) * a.pieces + piece) * a.rows + r] = a.pieces == 1 ? joined(make_float2(to, sum)) : make_float2(to, sum);
    }
}

// The keys' totals.  Registers are query rows, columns keys: a key's total needs no meeting but that of its two lanes.  A row's exponents lose its
// base, a whole number, and its weights are multiplied by 1 / sum as they are added up.  (One offset for both, base + log2 sum, saves 16 registers
// and is rounded at the logits' size: a row's weights would all be off by up to 1.4e-3 at logits of 40000, and the two-norm error is 1.6e-7 for 7.5e-8 at ordinary ones.
// us, 4 x 938 tokens of 32 / 8 heads, so and with it: 128 channels 69.6, 69.5, 96 61.0, 60.5, 64, a wavefront of a SIMD less, 53.3, 50.1; 2 x 61 over
// 41000..65000 keys in the kernel below 175, 174.)  grid: pairs; 256 keys, times pieces of the rows
template <int DP, int KS>
__global__ __launch_bounds__(kTileThreads, 2) void weights_sums_tiles_kernel(WeightsArgs a)
{
    using T = RowTile<DP>;
    __shared__ __attribute__((aligned(16))) char lds[2 * T::BYTES];
    __shared__ __attribute__((aligned(16))) float sm_base[2][kTileRows], sm_inv[2][kTileRows];   // of the tile's rows: base, 1 / sum
    __shared__ __attribute__((aligned(16))) int sm_lim[2][kTileRows];                       // keys from the wavefronts' first on that they see
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
    const uint32_t pair = blockIdx.x;
    const int b = pair / a.n_kv_heads, g = pair - b * a.n_kv_heads, d = a.head_dim;
    const int own = clamped(a.ctx, b, a.n_ctx);
    const int64_t block = static_cast<int64_t>(blockIdx.z) * gridDim.y + blockIdx.y;
    // (piece by piece as well, the last rows, which see the most, first)
    const int piece = a.row_pieces - 1 - static_cast<int>(block / a.key_tiles);
    const int64_t key_tile = block % a.key_tiles;
    const int64_t key0 = key_tile * kTileCols;
    float total[2][4];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) total[x][r] = 0.f;
    // query rows that see any of the keys: from the first token whose limit passes key0
    const int k0 = static_cast<int>(min(key0, static_cast<int64_t>(own)));
    const int64_t r_first = a.causal ? static_cast<int64_t>(max(k0 - own + a.seq, 0)) * a.group : 0;
    int t = max(static_cast<int>(r_first / kTileRows), piece * a.row_piece_tiles);
    const int t1 = key0 < own ? min((piece + 1) * a.row_piece_tiles, (a.rows + kTileRows - 1) / kTileRows) : 0;
    const bool any = t < t1;
    if (any) {
        const int kw = k0 + 64 * w;
        const char* const keys = static_cast<const char*>(a.kc) + static_cast<int64_t>(pair) * a.s_max * d * 2;
        row_bf16x8 kf[2][KS];
#pragma unroll
        for (int x = 0; x < 2; ++x) load_rows32<KS>(keys + static_cast<int64_t>(min(kw + 32 * x + col, own - 1)) * d * 2, half, d, a.flip, kf[x]);
        // the thread's rows of a tile, T::STEP rows further each time: the head of the group, and where the row begins
        const int row_t = tid / T::PC, chunk_t = tid - row_t * T::PC;
        int row = t * kTileRows + row_t, head = row % a.group;
        const int64_t token_bytes = a.qs[1] * 2, head_bytes = a.qs[2] * 2;
        const char* q = static_cast<const char*>(a.q) + (b * a.qs[0] + g * a.group * a.qs[2]) * 2 + (row / a.group) * token_bytes + head * head_bytes + chunk_t * 16;
        const int head_step = T::STEP % a.group;
        const int64_t step = T::STEP / a.group * token_bytes + head_step * head_bytes, wrap = token_bytes - a.group * head_bytes;
        const float2* const stats = a.stats + static_cast<int64_t>(pair) * a.pieces * a.rows;
        u32x4 next[T::NL];
        float2 next_s;
        int next_lim;
        auto fetch = [&](int t) __attribute__((always_inline)) {   // (rows past the last: zeros that add nothing)
#pragma unroll
            for (int j = 0; j < T::NL; ++j) {
                next[j] = u32x4{0u, 0u, 0u, 0u};
                if (chunk_t * 8 < d && row < a.rows) next[j] = *reinterpret_cast<const u32x4*>(q);
                row += T::STEP; head += head_step; q += step;
                if (head >= a.group) { head -= a.group; q += wrap; }
            }
            const int r = t * kTileRows + (tid >> 2), p = tid & 3;  // (four pieces of a row in neighbouring lanes)
            next_s = make_float2(-INFINITY, 0.f);
            if (r < a.rows && p < (a.joined ? 1 : a.pieces)) next_s = stats[static_cast<int64_t>(p) * a.rows + r];
            next_lim = keys_seen(a, own, r) - k0;
        };
        auto put = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < T::NL; ++j) *reinterpret_cast<u32x4*>(lds + buf * T::BYTES + tile_at<DP>(j * T::STEP + row_t, chunk_t)) = next[j];
            if (!a.joined) {
                next_s = with(next_s, make_float2(dpp<0xB1>(next_s.x), dpp<0xB1>(next_s.y)));
                next_s = joined(with(next_s, make_float2(dpp<0x4E>(next_s.x), dpp<0x4E>(next_s.y))));
            }
            if ((tid & 3) == 0) {
                sm_base[buf][tid >> 2] = next_s.x;
                sm_inv[buf][tid >> 2] = next_s.y;
                sm_lim[buf][tid >> 2] = next_lim;
            }
        };
        const char* at[KS];                                    // the lane's pieces of row col of a tile (row col + 32 lies 32 rows on)
#pragma unroll
        for (int c = 0; c < KS; ++c) at[c] = lds + tile_at<DP>(col, 2 * c + half);
        auto compute = [&](auto buf_c) __attribute__((always_inline)) {
            constexpr int buf = decltype(buf_c)::value;
#pragma unroll
            for (int u = 0; u < 2; ++u) {                      // 32 query rows
                float4 base[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) base[e] = *reinterpret_cast<const float4*>(&sm_base[buf][32 * u + 8 * e + 4 * half]);
                tile_f32x16 s[2];
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[x][r] = 0.f;
#pragma unroll
                for (int c = 0; c < KS; ++c) {
                    const row_bf16x8 qf = *reinterpret_cast<const row_bf16x8*>(at[c] + buf * T::BYTES + 32 * u * T::ROWB);
#pragma unroll
                    for (int x = 0; x < 2; ++x) s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[x][c], s[x], 0, 0, 0);
                }
                // (rows see the more the later they are; past the last row: nothing)
                const bool all = t * kTileRows + 32 * u + 32 <= a.rows && sm_lim[buf][32 * u] >= 64 * w + 64;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float bb[4] = {base[e].x, base[e].y, base[e].z, base[e].w};
                    const float4 inv = *reinterpret_cast<const float4*>(&sm_inv[buf][32 * u + 8 * e + 4 * half]);
                    const float ii[4] = {inv.x, inv.y, inv.z, inv.w};
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[x][4 * e + r] = __builtin_amdgcn_exp2f(fmaf(s[x][4 * e + r], a.scale, -bb[r]));
                    if (!__all(all)) {
                        const int4 lim = *reinterpret_cast<const int4*>(&sm_lim[buf][32 * u + 8 * e + 4 * half]);
                        const int ll[4] = {lim.x, lim.y, lim.z, lim.w};
#pragma unroll
                        for (int x = 0; x < 2; ++x)
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[x][4 * e + r] = 64 * w + 32 * x + col < ll[r] ? s[x][4 * e + r] : 0.f;
                    }
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int r = 0; r < 4; ++r) total[x][r] = fmaf(s[x][4 * e + r], ii[r], total[x][r]);
                }
            }
        };
        if (t < t1) { fetch(t); put(0); }
        __syncthreads();
        auto turn = [&](auto buf) __attribute__((always_inline)) {
            if (t + 1 < t1) fetch(t + 1);
            if (sm_lim[decltype(buf)::value][min(kTileRows, a.rows - t * kTileRows) - 1] > 64 * w) compute(buf);   // (the last row sees the most)
            if (t + 1 < t1) put(decltype(buf)::value ^ 1);
            __syncthreads();
            ++t;
        };
        while (t < t1) {
            turn(std::integral_constant<int, 0>{});
            if (t < t1) turn(std::integral_constant<int, 1>{});
        }
    }
    float sum[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        sum[x] = (total[x][0] + total[x][1]) + (total[x][2] + total[x][3]);
        sum[x] += __shfl_xor(sum[x], 32, kWave);
    }
    const float own_sum = half ? sum[1] : sum[0];              // (lane 32 x + col: the x-th 32 keys)
    const int64_t key = key0 + 64 * w + lane;
    if (a.row_pieces > 1) {
        if (key < a.pitch) a.parts[(static_cast<int64_t>(pair) * a.row_pieces + piece) * a.pitch + key] = own_sum;
    } else if (key < a.s_max) {
        const int64_t at = static_cast<int64_t>(pair) * a.s_max + key;
        const float had = a.base ? a.base[at] : 0.f;
        if (key < own) a.weights[at] = had + own_sum;
        else if (a.weights != a.base) a.weights[at] = had;
    }
}

// The keys' totals where the query rows fit LDS and there are many keys: the query rows stay there, a workgroup goes through every gridDim.y-th
// tile of 256 keys, 64 to a wavefront, which asks for the next tile's while it computes; no wavefront waits for another.  Over 41000..65000 keys matrix
// instructions take 22 us and vector ones 38, of which 7 at the same time (SQ_VALU_MFMA_BUSY_CYCLES, SQ_ACTIVE_INST_VALU, SQ_VALU_MFMA_COEXEC_CYCLES),
// of 96; the rest is waits and the shorter sample's units.  (Three wavefronts to a SIMD without the next tile's keys: 135 us; four: spills, 181.)
// grid: pairs; parts
constexpr int kStayBytes = 64 * 1024;                          // of query rows: two workgroups to a unit
constexpr int kStayThreads = 256, kStayKeys = kStayThreads;
template <int DP, int KS>
__global__ __launch_bounds__(kStayThreads, 2) void weights_sums_stay_kernel(WeightsArgs a)
{
    using T = RowTile<DP>;
    constexpr int MOST = kStayBytes / T::ROWB;
    extern __shared__ __attribute__((aligned(16))) char lds[];  // rows, whole tiles of 64; then of each row its base, 1 / its sum, its limit
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
    const uint32_t pair = blockIdx.x;
    const int b = pair / a.n_kv_heads, g = pair - b * a.n_kv_heads, d = a.head_dim;
    const int own = clamped(a.ctx, b, a.n_ctx);
    const int padded = (a.rows + kTileRows - 1) / kTileRows * kTileRows;
    float* const sm_base = reinterpret_cast<float*>(lds + padded * T::ROWB);
    float* const sm_inv = sm_base + padded;
    int* const sm_lim = reinterpret_cast<int*>(sm_inv + padded);
    static_assert(MOST % kTileRows == 0, "whole tiles");

    const char* const keys = static_cast<const char*>(a.kc) + static_cast<int64_t>(pair) * a.s_max * d * 2;
    row_bf16x8 next[2][KS];
    auto fetch = [&](int64_t key0) __attribute__((always_inline)) {   // (keys past the last re-read it)
#pragma unroll
        for (int x = 0; x < 2; ++x) load_rows32<KS>(keys + min(key0 + 32 * x + col, static_cast<int64_t>(own - 1)) * d * 2, half, d, a.flip, next[x]);
    };
    int64_t tile = blockIdx.y;
    if (tile * kStayKeys < own) {
        fetch(tile * kStayKeys + 64 * w);
        const int chunk_t = tid % T::PC;
        for (int r = tid / T::PC; r < padded; r += kStayThreads / T::PC) {
            u32x4 v = u32x4{0u, 0u, 0u, 0u};
            if (chunk_t * 8 < d && r < a.rows) {
                const int token = r / a.group, head = g * a.group + (r - token * a.group);
                v = *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.q) + (b * a.qs[0] + token * a.qs[1] + head * a.qs[2]) * 2 + chunk_t * 16);
            }
            *reinterpret_cast<u32x4*>(lds + tile_at<DP>(r, chunk_t)) = v;
        }
        const float2* const stats = a.stats + static_cast<int64_t>(pair) * a.pieces * a.rows;
        for (int r = tid; r < padded; r += kStayThreads) {
            float2 st = make_float2(0.f, 0.f);
            if (r < a.rows) {
                st = stats[r];
                if (!a.joined) {
                    for (int p = 1; p < a.pieces; ++p) st = with(st, stats[static_cast<int64_t>(p) * a.rows + r]);
                    st = joined(st);
                }
            }
            sm_base[r] = st.x;
            sm_inv[r] = st.y;
            sm_lim[r] = keys_seen(a, own, r);
        }
        __syncthreads();
    }
    const char* at[KS];                                        // the lane's pieces of row col of the first 32
#pragma unroll
    for (int c = 0; c < KS; ++c) at[c] = lds + tile_at<DP>(col, 2 * c + half);
    for (; tile < a.key_tiles; tile += gridDim.y) {
        const int64_t key0 = tile * kStayKeys + 64 * w;
        float total[2][4];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) total[x][e] = 0.f;
        if (key0 < own) {
            row_bf16x8 kf[2][KS];
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int c = 0; c < KS; ++c) kf[x][c] = next[x][c];
            fetch(key0 + static_cast<int64_t>(gridDim.y) * kStayKeys);
            // query rows that see any of the keys: from the first token whose limit passes the first key
            const int k0 = static_cast<int>(key0);
            const int64_t r_first = a.causal ? static_cast<int64_t>(max(k0 - own + a.seq, 0)) * a.group : 0;
            for (int u = static_cast<int>(r_first / 32); 32 * u < a.rows; ++u) {
                const int rows = 32 * u * T::ROWB;
                row_bf16x8 qf[KS];
#pragma unroll
                for (int c = 0; c < KS; ++c) qf[c] = *reinterpret_cast<const row_bf16x8*>(at[c] + rows);
                float4 base[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) base[e] = *reinterpret_cast<const float4*>(sm_base + 32 * u + 8 * e + 4 * half);
                tile_f32x16 s[2];
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[x][r] = 0.f;
#pragma unroll
                for (int c = 0; c < KS; ++c)
#pragma unroll
                    for (int x = 0; x < 2; ++x) s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[c], kf[x][c], s[x], 0, 0, 0);
                // (rows of a block see the more the later they are; past the last row: nothing)
                const bool all = 32 * u + 32 <= a.rows && sm_lim[32 * u] >= static_cast<int>(key0) + 64;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float bb[4] = {base[e].x, base[e].y, base[e].z, base[e].w};
                    const float4 inv = *reinterpret_cast<const float4*>(sm_inv + 32 * u + 8 * e + 4 * half);
                    const float ii[4] = {inv.x, inv.y, inv.z, inv.w};
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[x][4 * e + r] = __builtin_amdgcn_exp2f(fmaf(s[x][4 * e + r], a.scale, -bb[r]));
                    if (!__all(all)) {
                        const int4 lim = *reinterpret_cast<const int4*>(sm_lim + 32 * u + 8 * e + 4 * half);
                        const int ll[4] = {lim.x, lim.y, lim.z, lim.w};
#pragma unroll
                        for (int x = 0; x < 2; ++x)
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[x][4 * e + r] = static_cast<int>(key0) + 32 * x + col < ll[r] ? s[x][4 * e + r] : 0.f;
                    }
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int r = 0; r < 4; ++r) total[x][r] = fmaf(s[x][4 * e + r], ii[r], total[x][r]);
                }
            }
        }
        float sum[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            sum[x] = (total[x][0] + total[x][1]) + (total[x][2] + total[x][3]);
            sum[x] += __shfl_xor(sum[x], 32, kWave);
        }
        const int64_t key = key0 + lane;                       // (lane 32 x + col: the x-th 32)
        if (key < a.s_max) {
            const int64_t to = static_cast<int64_t>(pair) * a.s_max + key;
            const float had = a.base ? a.base[to] : 0.f;
            if (key < own) a.weights[to] = had + (half ? sum[1] : sum[0]);
            else if (a.weights != a.base) a.weights[to] = had;
        }
    }
}

// Adds up the pieces of the keys' totals.  grid: pairs; 256 keys along y
__global__ __launch_bounds__(256) void weights_totals_kernel(WeightsArgs a)
{
    const int64_t pair = blockIdx.x, key = static_cast<int64_t>(blockIdx.y) * 256 + threadIdx.x;
    if (key >= a.s_max) return;
    const int own = clamped(a.ctx, static_cast<int>(pair / a.n_kv_heads), a.n_ctx);
    const float* const part = a.parts + pair * a.row_pieces * a.pitch + key;
    const int64_t at = pair * a.s_max + key;
    const float had = a.base ? a.base[at] : 0.f;
    if (key < own) {
        float sum = 0.f;
#pragma unroll 4
        for (int p = 0; p < a.row_pieces; ++p) sum += part[static_cast<int64_t>(p) * a.pitch];
        a.weights[at] = had + sum;
    } else if (a.weights != a.base) {
        a.weights[at] = had;
    }
}

// ------------------------------------------------------------------------------------------------------------- host
struct WeightsPlan {
    bool short_cache;                                         // one launch
    bool tiles;                                               // the kernels of many rows
    int g_rows, g_keys;                                       // else: column tiles of the two launches
    int64_t row_tiles, key_tiles, pieces, piece_tiles;
    int64_t row_pieces, row_piece_tiles;                      // pieces of the second launch, tiles of 64 rows of each
    int64_t stay;                                             // workgroups of a pair in which the query rows stay; 0: none does
    size_t stats_bytes, parts_bytes;                          // at these sizes or with fewer keys, at most
};

static int wgt_columns_for(int64_t rows, int most) { int g = 1; while (g < most && 16 * g < rows) g *= 2; return g; }
static int wgt_most(bool bf16, int32_t head_dim)
{
    const int dp = head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256, chunks = dp * (bf16 ? 2 : 4) / 64;
    return chunks <= 4 ? 8 : 32 / chunks;
}
// Pieces of `tiles` tiles that fill the chip, `least` tiles or more each.
static int64_t wgt_pieces(int64_t fill, int64_t units, int64_t tiles, int64_t least, int64_t most)
{
    return std::max<int64_t>(1, std::min<int64_t>({units > 0 ? fill / units : 1, tiles / least, most}));
}

// What the registers of the one launch hold, of rows of up to 256 bytes: 64 rows over 512 keys or 32 over 1024; fp32 rows of up to 16 pairs, whose products
// take four times as long on the few units that they have, up to 384 keys.  (us, so and in two launches.  bf16, 64 rows, 32 / 8 heads of 128, over 117 / 250 /
// 469 / 512 keys of one sample 10.4 / 11.4 / 12.5 / 12.9, 11.6 / 11.8 / 12.1 / 12.0, of 4 12.8, 13.6 over 469, of 32 13.3, 34; 20 rows, 8 / 8 heads,
// over 469 / 700 / 1024 of one 10.9 / 12.3 / 14.5, 10.6 / 13.3 / 13.2, of 4 11.1 / 12.3 / 14.7, 11.5 / 14.5 / 15.3: with up to 16 pairs within 9 % either
// way.  64 channels, 64 rows over 469 of one 10.0, 11.2; 96 10.1, 11.2.  fp32 of 64 channels, 64 rows over 250 / 350 / 400 / 512 of one 12.6 / 15.1 /
// 16.0 / 17.1, 13.2 / 14.4 / 14.1 / 13.2, of 2 12.7 / 15.1 / 16.0 / 17.2, 13.3 / 14.7 / 14.3 / 13.5, of 3 12.9 / 15.3 / 16.0 / 17.1, 13.5 / 16.1 /
// 15.9 / 15.1, of 16 17.5, 29 over 512; 20 rows over 700 / 1024 of one 15.9 / 19.7, 13.8 / 13.5, of 16 16.3 / 20.2, 32 / 41.)
static bool short_cache(bool bf16, int64_t pairs, int64_t rows, int32_t head_dim, int64_t n_ctx)
{
    if (!bf16 && rows > kFewWeightRows && pairs <= 16 && n_ctx > 384) return false;
    return wgt_most(bf16, head_dim) == 8 && (rows <= 32 ? n_ctx <= 1024 : rows <= 64 && n_ctx <= 512) && pairs <= (int64_t{1} << 22);
}
// Few rows go with the decode's kernel, without V, which keeps their logits; more of them over a short cache are better off above: its workgroup
// takes their exponentials out of registers.  (us, with the decode's and above: 4 rows over 117 / 1000 keys of 64 samples, 32 / 8 heads of 128, 6.3 / 28.8,
// 11.2 / 29.8; 16 over 250 / 469 / 1000 of one 7.2 / 10.4 / 13.6, 7.4 / 9.0 / 12.6; and in two launches, 4 over 3584 of 64 samples 90, 382, 16 146, 379.)
static bool weigh_few(bool bf16, int64_t pairs, int64_t rows, int32_t head_dim, int64_t n_ctx)
{
    return rows > 0 && rows <= kFewWeightRows && !(short_cache(bf16, pairs, rows, head_dim, n_ctx) && rows * n_ctx > 4000);
}

static WeightsPlan weights_plan(bool bf16, int32_t batch, int32_t seq, int64_t rows, int32_t n_kv_heads, int32_t head_dim, int64_t s_max, int64_t n_ctx)
{
    WeightsPlan p{};
    const int64_t pairs = static_cast<int64_t>(batch) * n_kv_heads;
    p.tiles = bf16 && head_dim <= 128 && rows > kWgtFewRows;
    const int most = wgt_most(bf16, head_dim);
    p.g_rows = wgt_columns_for(rows, most);
    p.short_cache = short_cache(bf16, pairs, rows, head_dim, n_ctx);
    p.row_tiles = ceil_div(rows, p.tiles ? kTileCols : 16 * p.g_rows);
    const int64_t tiles = ceil_div(n_ctx, p.tiles ? kTileRows : 16), units = pairs * p.row_tiles;
    // (many rows: at least as many workgroups as fit the chip at once, three a unit; where there are that many anyway, and at a time behind each
    // other on a unit, a row tile's keys in four, so that the longest of a causal prompt is not what the launch takes)
    const int64_t most_pieces = !p.tiles ? wgt_pieces(512, units, tiles, 8, kWgtMaxPieces)
                              : units >= kUnits ? std::max<int64_t>(1, std::min<int64_t>({kWgtInline, tiles / 6, 8 * kUnits / units}))
                              : wgt_pieces(3 * kUnits, units, tiles, 4, kWgtMaxPieces);
    p.piece_tiles = std::max<int64_t>(1, ceil_div(tiles, most_pieces));
    p.pieces = std::max<int64_t>(1, ceil_div(tiles, p.piece_tiles));
    p.stats_bytes = sizeof(float2) * static_cast<size_t>(pairs) * rows * most_pieces;
    p.row_pieces = 1;
    if (p.tiles) {
        const int64_t row_tiles = ceil_div(rows, kTileRows), key_tiles = ceil_div(n_ctx, kTileCols);
        // tiles of query rows of a piece where there are k key tiles: what a causal prompt leaves of them, over four workgroups a unit, 4 or more
        auto piece = [&](int64_t k) {
            const int64_t keys = k * kTileCols, all = pairs * k * row_tiles, seen = seq >= keys ? all / 2 : all - all * seq / (2 * keys);
            return std::min(row_tiles, std::max<int64_t>({4, ceil_div(seen, 4 * kUnits), ceil_div(row_tiles, kWgtMaxPieces)}));
        };
        p.row_piece_tiles = piece(std::max<int64_t>(key_tiles, 1));
        p.row_pieces = ceil_div(row_tiles, p.row_piece_tiles);
        int64_t parts = 0;                                     // (fewer keys may be cut into more pieces)
        for (int64_t k = 1; k <= key_tiles; ++k) {
            const int64_t n = ceil_div(row_tiles, piece(k));
            if (n > 1) parts = std::max(parts, k * n);
            else if (pairs * k > 4 * kUnits) break;            // (more keys are not cut either)
        }
        p.parts_bytes = sizeof(float) * static_cast<size_t>(pairs) * parts * kTileCols;
        // (two workgroups to a unit, of two tiles of keys or more.  us, so and with the query rows in tiles: 244 rows over 65000 / 16384 keys of 2 / 8 samples,
        // 32 / 8 heads of 128, 209 / 196, 226 / 216; over 3584 of 64 359, 408, of 8, 896 tiles, 66.9, 64.3; 160 rows of 96 over 8200 of 8, 1056 tiles, 48.9, 52.5)
        p.stay = rows <= kStayBytes / (head_dim <= 64 ? 128 : 256) && pairs * key_tiles >= 1024 ? std::max<int64_t>(1, 512 / pairs) : 0;
        if (p.stay || key_tiles == 0) p.row_pieces = 1;
        p.key_tiles = p.stay ? ceil_div(s_max, kStayKeys) : p.row_pieces > 1 ? key_tiles : ceil_div(s_max, kTileCols);
    } else {
        p.g_keys = most;
        while (p.g_keys > 2 && pairs * ceil_div(n_ctx, 16 * p.g_keys) < 512) p.g_keys /= 2;
        p.key_tiles = ceil_div(s_max, 16 * p.g_keys);
    }
    return p;
}

static bool weights_sizes_ok(int dtype, int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t n_ctx)
{
    return dtype_size(dtype) && batch >= 0 && seq >= 0 && n_q_heads > 0 && n_kv_heads > 0 && n_q_heads % n_kv_heads == 0 && head_dim > 0
        && head_dim % 8 == 0 && n_ctx >= 0;
}

constexpr int64_t kWgtMaxTiles = int64_t{1} << 23;            // workgroups along x: fewer than 2^32 threads
constexpr int64_t kWgtGridY = 32768;
static bool weights_covered(int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t s_max)
{
    const int64_t rows = static_cast<int64_t>(seq) * (n_q_heads / n_kv_heads), pairs = static_cast<int64_t>(batch) * n_kv_heads;
    return head_dim <= CIVIC_MAX_HEAD_DIM && s_max <= kCacheMaxRows && rows <= (int64_t{1} << 26) && pairs <= kWgtMaxTiles
        && pairs * ceil_div(rows, 16) <= kWgtMaxTiles;
}

static dim3 wgt_grid(unsigned pairs, int64_t tiles)
{
    return dim3(pairs, static_cast<unsigned>(std::min<int64_t>(tiles, kWgtGridY)), static_cast<unsigned>(ceil_div(tiles, kWgtGridY)));
}

static void launch_join(const WeightsArgs& a, const WeightsPlan& p, unsigned pairs, hipStream_t s)
{
    if (a.rows > 0 && p.pieces > kWgtInline)
        civic::launch(weights_join_kernel, dim3(static_cast<unsigned>(ceil_div(static_cast<int64_t>(pairs) * a.rows, 256))), dim3(256), 0, s, a);
}

template <int DP, int KS>
static int launch_tiles(const WeightsArgs& a, const WeightsPlan& p, hipStream_t s)
{
    const unsigned pairs = static_cast<unsigned>(a.batch) * a.n_kv_heads;
    civic::launch(weights_stats_tiles_kernel<DP, KS>, dim3(static_cast<unsigned>(pairs * p.row_tiles * p.pieces)), dim3(kTileThreads), 0, s, a);
    launch_join(a, p, pairs, s);
    if (p.stay) {
        constexpr size_t most = kStayBytes + kStayBytes / RowTile<DP>::ROWB * 12;
        const size_t lds = static_cast<size_t>(ceil_div(a.rows, kTileRows)) * kTileRows * (RowTile<DP>::ROWB + 12);
        static std::atomic<uint64_t> done{0};
        const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(weights_sums_stay_kernel<DP, KS>), most, &done);
        if (rc != CIVIC_OK) return rc;
        civic::launch(weights_sums_stay_kernel<DP, KS>, dim3(pairs, static_cast<unsigned>(p.stay)), dim3(kStayThreads), lds, s, a);
        return check_launch();
    }
    civic::launch(weights_sums_tiles_kernel<DP, KS>, wgt_grid(pairs, p.key_tiles * p.row_pieces), dim3(kTileThreads), 0, s, a);
    if (p.row_pieces > 1) civic::launch(weights_totals_kernel, dim3(pairs, static_cast<unsigned>(ceil_div(a.written, 256))), dim3(256), 0, s, a);
    return check_launch();
}

template <bool BF16, int DP, bool FULL>
static void launch_weights(WeightsArgs& a, const WeightsPlan& p, hipStream_t s)
{
    const unsigned pairs = static_cast<unsigned>(a.batch) * a.n_kv_heads;
    if constexpr (wgt_chunks<BF16, DP>() <= 4) {
        if (p.short_cache && a.rows > 0) {
            const bool here = a.weights == a.base;             // (rows behind a context stay as they are)
            const unsigned behind = here ? 0 : behind_blocks(pairs, a.s_max, a.n_ctx, kShortThreads);
            a.pairs = pairs;
            a.written = here ? 0 : behind ? a.n_ctx : a.s_max;
            const dim3 grid(pairs + behind);
            if (p.g_rows == 1) civic::launch(weights_short_kernel<BF16, DP, FULL, 1, 8>, grid, dim3(kShortThreads), 0, s, a);
            else if (p.g_rows == 2) civic::launch(weights_short_kernel<BF16, DP, FULL, 2, 8>, grid, dim3(kShortThreads), 0, s, a);
            else civic::launch(weights_short_kernel<BF16, DP, FULL, 4, 4>, grid, dim3(kShortThreads), 0, s, a);
            return;
        }
    }
    const dim3 block(kWgtThreads), rows(static_cast<unsigned>(pairs * p.row_tiles * p.pieces)), keys = wgt_grid(pairs, p.key_tiles);
    constexpr int MOST = wgt_most_columns<BF16, DP>();
    if (a.rows == 0) {}                                       // (no tokens: the totals are what they were)
    else if (p.g_rows == 2) civic::launch(weights_stats_kernel<BF16, DP, FULL, 2>, rows, block, 0, s, a);
    else if (p.g_rows == 4) { if constexpr (MOST >= 4) civic::launch(weights_stats_kernel<BF16, DP, FULL, 4>, rows, block, 0, s, a); }
    else if constexpr (MOST >= 8) civic::launch(weights_stats_kernel<BF16, DP, FULL, 8>, rows, block, 0, s, a);
    launch_join(a, p, pairs, s);
    if (p.g_keys == 2) civic::launch(weights_sums_kernel<BF16, DP, FULL, 2>, keys, block, 0, s, a);
    else if (p.g_keys == 4) { if constexpr (MOST >= 4) civic::launch(weights_sums_kernel<BF16, DP, FULL, 4>, keys, block, 0, s, a); }
    else if constexpr (MOST >= 8) civic::launch(weights_sums_kernel<BF16, DP, FULL, 8>, keys, block, 0, s, a);
}

template <bool BF16>
static int launch_weights_dim(WeightsArgs& a, const WeightsPlan& p, hipStream_t s)
{
    const int d = a.head_dim;
    if (p.tiles) return d <= 64 ? launch_tiles<64, 4>(a, p, s) : d <= 96 ? launch_tiles<128, 6>(a, p, s) : launch_tiles<128, 8>(a, p, s);
    if (d == 64) launch_weights<BF16, 64, true>(a, p, s);
    else if (d == 128) launch_weights<BF16, 128, true>(a, p, s);
    else if (d == 256) launch_weights<BF16, 256, true>(a, p, s);
    else if (d < 64) launch_weights<BF16, 64, false>(a, p, s);
    else if (d < 128) launch_weights<BF16, 128, false>(a, p, s);
    else launch_weights<BF16, 256, false>(a, p, s);
    return check_launch();
}

}  // namespace civic

extern "C" size_t civic_attn_weights_workspace_bytes(int dtype, int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t n_ctx)
{
    using namespace civic;
    if (!weights_sizes_ok(dtype, batch, seq, n_q_heads, n_kv_heads, head_dim, n_ctx)
        || !weights_covered(batch, seq, n_q_heads, n_kv_heads, head_dim, n_ctx) || batch == 0 || seq == 0) return 0;
    const int64_t rows = static_cast<int64_t>(seq) * (n_q_heads / n_kv_heads);
    if (rows <= kFewWeightRows) return few_weights_bytes(dtype, batch, rows, n_kv_heads, head_dim, n_ctx);
    const WeightsPlan p = weights_plan(dtype == CIVIC_BF16, batch, seq, rows, n_kv_heads, head_dim, n_ctx, n_ctx);
    return p.stats_bytes + p.parts_bytes;
}

extern "C" int civic_attn_weights(const void* q, const void* k_cache, const float* base, float* weights, int dtype, int32_t batch, int32_t seq,
                                  int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const int64_t* q_strides, int64_t s_max, int64_t n_ctx,
                                  const int32_t* ctx, int32_t causal, float softmax_scale, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace civic;
    if (!weights_sizes_ok(dtype, batch, seq, n_q_heads, n_kv_heads, head_dim, n_ctx) || !q_strides) return CIVIC_ERR_INVALID_ARG;
    if (s_max < 0 || n_ctx > s_max || !std::isfinite(softmax_scale)) return CIVIC_ERR_INVALID_ARG;
    const bool any = batch > 0 && s_max > 0;
    if (any && (!weights || (seq > 0 && !q) || (n_ctx > 0 && !k_cache))) return CIVIC_ERR_INVALID_ARG;
    for (const void* p : {q, k_cache, static_cast<const void*>(workspace)})
        if (!aligned16(p)) return CIVIC_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(base), static_cast<const void*>(weights), static_cast<const void*>(ctx)})
        if (reinterpret_cast<uintptr_t>(p) & 3u) return CIVIC_ERR_INVALID_ARG;
    const int esz = dtype_size(dtype);
    for (int i = 0; i < 3; ++i)
        if (q_strides[i] < 0 || (q_strides[i] * esz) % 16) return CIVIC_ERR_INVALID_ARG;
    if (n_q_heads > 1 && q_strides[2] < head_dim) return CIVIC_ERR_INVALID_ARG;
    if (!weights_covered(batch, seq, n_q_heads, n_kv_heads, head_dim, s_max)) return CIVIC_ERR_UNSUPPORTED;
    if (!any) return CIVIC_OK;
    if (!same_or_apart(base, weights, static_cast<int64_t>(batch) * n_kv_heads * s_max * 4)) return CIVIC_ERR_INVALID_ARG;
    WeightsArgs a{};
    a.group = n_q_heads / n_kv_heads;
    a.rows = seq * a.group;
    const size_t need = civic_attn_weights_workspace_bytes(dtype, batch, seq, n_q_heads, n_kv_heads, head_dim, n_ctx);
    if (need && (!workspace || workspace_bytes < need)) return CIVIC_ERR_WORKSPACE;
    const int64_t pairs = static_cast<int64_t>(batch) * n_kv_heads, sums = pairs * s_max * 4;
    if (!writes_apart({{weights, sums}, {workspace, static_cast<int64_t>(need)}},
                      {{q, reach_bytes(q_strides, batch, seq, n_q_heads, head_dim, esz)}, {k_cache, pairs * s_max * head_dim * esz}, {ctx, batch * int64_t{4}}})
        || !Memory{base, sums}.apart({workspace, static_cast<int64_t>(need)})) return CIVIC_ERR_INVALID_ARG;
    if (weigh_few(dtype == CIVIC_BF16, static_cast<int64_t>(batch) * n_kv_heads, a.rows, head_dim, n_ctx))
        return few_weights(q, k_cache, base, weights, dtype, batch, seq, n_q_heads, n_kv_heads, head_dim, q_strides, s_max, n_ctx, ctx, causal, softmax_scale, workspace, stream);
    const int64_t written = weights == base ? std::max<int64_t>(n_ctx, 1) : s_max;   // (in place rows behind a context stay as they are)
    const WeightsPlan p = weights_plan(dtype == CIVIC_BF16, batch, seq, std::max(a.rows, 1), n_kv_heads, head_dim, written, n_ctx);
    a.q = q; a.kc = k_cache; a.ctx = ctx; a.base = base; a.weights = weights; a.stats = static_cast<float2*>(workspace);
    for (int i = 0; i < 3; ++i) a.qs[i] = q_strides[i];
    a.s_max = s_max; a.batch = batch; a.seq = seq; a.n_q_heads = n_q_heads; a.n_kv_heads = n_kv_heads; a.head_dim = head_dim;
    a.causal = causal != 0; a.n_ctx = static_cast<int32_t>(n_ctx);
    a.row_tiles = static_cast<int32_t>(p.row_tiles); a.pieces = static_cast<int32_t>(p.pieces); a.piece_tiles = static_cast<int32_t>(p.piece_tiles);
    a.joined = p.pieces == 1 || p.pieces > kWgtInline;
    a.row_pieces = static_cast<int32_t>(p.row_pieces); a.row_piece_tiles = static_cast<int32_t>(p.row_piece_tiles); a.key_tiles = static_cast<int32_t>(p.key_tiles);
    a.pitch = static_cast<int32_t>(kTileCols * ceil_div(n_ctx, kTileCols));
    a.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.stats_bytes);
    const LogitScale scale = logit_scale(softmax_scale, head_dim, dtype == CIVIC_BF16);
    a.scale = scale.log2; a.flip = scale.flip;
    a.written = written;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return dtype == CIVIC_BF16 ? launch_weights_dim<true>(a, p, s) : launch_weights_dim<false>(a, p, s);
}
