// civic_attn_weights: how much attention each cache row has received from new tokens,
//
//   weights[b, g, j] = base[b, g, j] + sum_{i, h in g} e(i, h, j) / sum_k e(i, h, k),   e = exp(scale <q[b, i, h], K[b, g, j]>),
//   j, k < ctx[b] - (seq - 1 - i) when causal, < ctx[b] else.
//
// A row's weights need the row's sum first, so the product Q K^T is made twice (keeping it instead would write and read four bytes for
// every query row and key: as much as K at 64 query rows of 128 bf16 channels, and there are hundreds): once over the keys for every
// query row's base and sum, once over the query rows for every key's total.  The queries of a KV head are rows r = token * group + head
// of the group.  Both launches have the same shape: a wavefront holds 16 G rows of one side in registers, as columns of its products,
// and reads the other side in tiles of 16 rows from memory as they lie; the lanes of a column add up what they see, four results of a
// tile each, so that nothing crosses lanes before the end.  The wavefronts of a workgroup have the same columns and take turns over
// the tiles; they meet in LDS.  No atomics: a total's order of summation is the same on every call.
// Vector work per result: a fused multiply-add, an exponential and an addition (a second multiply-add in the second launch).
#include "rows_device.h"

namespace civic {

constexpr int kWgtWaves = 4, kWgtThreads = kWgtWaves * kWave;
constexpr int kWgtMaxPieces = 64;
constexpr int kWgtRows = 2048;                                // query rows whose sums are in LDS at a time

struct WeightsArgs {
    const void* q; const void* kc;
    const int32_t* ctx;
    const float* base; float* weights;
    float2* stats;                                            // [pairs, rows, pieces] (base, sum)
    int64_t qs[3];
    int64_t s_max;
    int32_t batch, seq, n_q_heads, n_kv_heads, head_dim, group, causal, n_ctx;
    int32_t rows;                                             // of a pair of sample and KV head: seq * group
    int32_t row_tiles, pieces, piece_tiles;                   // first launch: tiles of 16 keys of a piece
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
#pragma unroll
    for (int x = 0; x < G; ++x) {
        const int r = r0 + 16 * x + l16;
        lim[x] = keys_seen(a, own, r);
        const int rr = min(r, a.rows - 1), token = rr / a.group, head = g * a.group + (rr - token * a.group);
        load_row<FULL>(static_cast<const char*>(a.q) + (b * a.qs[0] + token * a.qs[1] + head * a.qs[2]) * ESZ, kq, row_bytes, qf[x]);
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) qf[x][t][e] ^= a.flip;
    }
    const char* const keys = static_cast<const char*>(a.kc) + static_cast<int64_t>(pair) * a.s_max * row_bytes;
    auto fetch = [&](int t, u32x4 (&kf)[KT]) __attribute__((always_inline)) {   // (keys past the last re-read it)
        load_row<FULL>(keys + static_cast<int64_t>(min(16 * t + l16, own - 1)) * row_bytes, kq, row_bytes, kf);
    };
    float base[G], l[G];
#pragma unroll
    for (int x = 0; x < G; ++x) { base[x] = -INFINITY; l[x] = 0.f; }
    u32x4 kf[KT];
    int t = piece * a.piece_tiles + w;
    if (t < t1) fetch(t, kf);
    for (; t < t1; t += kWgtWaves) {
        row_f32x4 s[G];
#pragma unroll
        for (int x = 0; x < G; ++x) s[x] = row_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KT; ++c)
#pragma unroll
            for (int x = 0; x < G; ++x) s[x] = mma16<BF16>(kf[c], qf[x][c], s[x]);
        if (t + kWgtWaves < t1) fetch(t + kWgtWaves, kf);
        if (16 * t + 16 > all_see) {
#pragma unroll
            for (int x = 0; x < G; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[x][r] = 16 * t + 4 * kq + r < lim[x] ? s[x][r] : -INFINITY;
        }
        bool outgrown = false;
        float top[G];
#pragma unroll
        for (int x = 0; x < G; ++x) {
            top[x] = fmaxf(fmaxf(s[x][0], s[x][1]), fmaxf(s[x][2], s[x][3]));
            outgrown |= top[x] * a.scale > base[x] + kBaseSlack;
        }
        if (__any(outgrown)) {
#pragma unroll
            for (int x = 0; x < G; ++x) {
                const float z = top[x] * a.scale, to = z > base[x] + kBaseSlack ? rintf(z) : base[x];
                l[x] *= base_step(base[x], to);
                base[x] = to;
            }
        }
#pragma unroll
        for (int x = 0; x < G; ++x) {
            const float off = base[x] == -INFINITY ? 0.f : base[x];
#pragma unroll
            for (int r = 0; r < 4; ++r) l[x] += __builtin_amdgcn_exp2f(fmaf(s[x][r], a.scale, -off));
        }
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
        a.stats[(static_cast<int64_t>(pair) * a.rows + r0 + i) * a.pieces + piece] = make_float2(to, sum);
    }
}

// The keys' totals.  Columns: keys; tiles: query rows.  grid: pairs, then the column tiles along y and z
template <bool BF16, int DP, bool FULL, int G>
__global__ __launch_bounds__(kWgtThreads, 2) void weights_sums_kernel(WeightsArgs a)
{
    constexpr int ESZ = BF16 ? 2 : 4, KT = wgt_chunks<BF16, DP>();
    __shared__ __attribute__((aligned(16))) float2 sm_s[kWgtRows];              // base, 1 / sum
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
        // tiles of query rows that see any of the keys: from the first token whose limit passes key0
        const int tiles = (a.rows + 15) / 16;
        const int64_t r_first = a.causal ? static_cast<int64_t>(max(k0 - own + a.seq, 0)) * a.group : 0;
        int first = static_cast<int>(r_first / 16);
        for (int r0 = first * 16 / kWgtRows * kWgtRows; r0 < a.rows; r0 += kWgtRows) {
            const int end = min(r0 + kWgtRows, a.rows);
            __syncthreads();
            for (int r = max(r0, first * 16) + tid; r < r0 + kWgtRows && r < tiles * 16; r += kWgtThreads) {
                float2 s = make_float2(-INFINITY, 0.f);
                if (r < end) {
                    const float2* const st = a.stats + (static_cast<int64_t>(pair) * a.rows + r) * a.pieces;
                    const int n = min(a.pieces, (keys_seen(a, own, min(r | 15, a.rows - 1)) + 16 * a.piece_tiles - 1) / (16 * a.piece_tiles));
                    for (int p = 0; p < n; ++p) {
                        const float2 y = st[p];
                        const float to = fmaxf(s.x, y.x);
                        s = make_float2(to, fmaf(base_step(s.x, to), s.y, base_step(y.x, to) * y.y));
                    }
                }
                sm_s[r - r0] = make_float2(s.x == -INFINITY ? 0.f : s.x, s.y == 0.f ? 0.f : 1.f / s.y);
            }
            __syncthreads();
            const int t1 = (end + 15) / 16;
            int t = max(r0 / 16, first) + w;
            // the lane's query row: token and head of the group, 64 rows further each time
            int r = 16 * t + l16, token = r / a.group, head = r - token * a.group;
            const int token_step = 16 * kWgtWaves / a.group, head_step = 16 * kWgtWaves - token_step * a.group;
            const char* const q = static_cast<const char*>(a.q) + (b * a.qs[0] + g * a.group * a.qs[2]) * ESZ;
            u32x4 qf[KT];
            auto fetch = [&]() __attribute__((always_inline)) {                 // (rows past the last re-read the last token's)
                load_row<FULL>(q + (min(token, a.seq - 1) * a.qs[1] + head * a.qs[2]) * ESZ, kq, row_bytes, qf);
                token += token_step; head += head_step;
                if (head >= a.group) { head -= a.group; ++token; }
#pragma unroll
                for (int c = 0; c < KT; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) qf[c][e] ^= a.flip;
            };
            if (t < t1) fetch();
            for (; t < t1; t += kWgtWaves) {
                row_f32x4 s[G];
#pragma unroll
                for (int x = 0; x < G; ++x) s[x] = row_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < KT; ++c)
#pragma unroll
                    for (int x = 0; x < G; ++x) s[x] = mma16<BF16>(qf[c], kf[x][c], s[x]);
                if (t + kWgtWaves < t1) fetch();
                float2 st[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) st[e] = sm_s[16 * t - r0 + 4 * kq + e];
                const bool whole = 16 * t + 16 <= a.rows && keys_seen(a, own, 16 * t) >= k0 + 16 * G;
                if (whole) {
#pragma unroll
                    for (int x = 0; x < G; ++x)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[x] = fmaf(__builtin_amdgcn_exp2f(fmaf(s[x][e], a.scale, -st[e].x)), st[e].y, acc[x]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int lim = keys_seen(a, own, 16 * t + 4 * kq + e) - k0;
#pragma unroll
                        for (int x = 0; x < G; ++x)
                            if (16 * x + l16 < lim) acc[x] = fmaf(__builtin_amdgcn_exp2f(fmaf(s[x][e], a.scale, -st[e].x)), st[e].y, acc[x]);
                    }
                }
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
        if (key0 + tid < own) a.weights[at] = had + ((sm_a[0][tid] + sm_a[1][tid]) + (sm_a[2][tid] + sm_a[3][tid]));
        else if (a.weights != a.base) a.weights[at] = had;
    }
}

// ------------------------------------------------------------------------------------------------------------- host
struct WeightsPlan {
    int g_rows, g_keys;                                       // column tiles of the two launches
    int64_t row_tiles, key_tiles, pieces, piece_tiles, most_pieces;
};

static int wgt_columns_for(int64_t rows, int most) { int g = 1; while (g < most && 16 * g < rows) g *= 2; return g; }
static int wgt_most(bool bf16, int32_t head_dim)
{
    const int dp = head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256, chunks = dp * (bf16 ? 2 : 4) / 64;
    return chunks <= 4 ? 8 : 32 / chunks;
}

static WeightsPlan weights_plan(bool bf16, int32_t batch, int64_t rows, int32_t n_kv_heads, int32_t head_dim, int64_t s_max, int64_t n_ctx)
{
    WeightsPlan p{};
    const int most = wgt_most(bf16, head_dim);
    const int64_t pairs = static_cast<int64_t>(batch) * n_kv_heads;
    p.g_rows = wgt_columns_for(rows, most);
    p.row_tiles = ceil_div(rows, 16 * p.g_rows);
    const int64_t units = pairs * p.row_tiles, tiles = ceil_div(n_ctx, 16);
    p.most_pieces = std::max<int64_t>(1, std::min<int64_t>({ceil_div(1024, units), tiles / 8, kWgtMaxPieces}));
    p.piece_tiles = std::max<int64_t>(1, ceil_div(tiles, p.most_pieces));
    p.pieces = std::max<int64_t>(1, ceil_div(tiles, p.piece_tiles));
    p.g_keys = most;
    while (p.g_keys > 2 && pairs * ceil_div(n_ctx, 16 * p.g_keys) < 512) p.g_keys /= 2;
    p.key_tiles = ceil_div(s_max, 16 * p.g_keys);
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

template <bool BF16, int DP, bool FULL>
static void launch_weights(const WeightsArgs& a, const WeightsPlan& p, hipStream_t s)
{
    const unsigned pairs = static_cast<unsigned>(a.batch) * a.n_kv_heads;
    const dim3 block(kWgtThreads), rows(static_cast<unsigned>(pairs * p.row_tiles * p.pieces)), keys(pairs, static_cast<unsigned>(std::min<int64_t>(p.key_tiles, kWgtGridY)), static_cast<unsigned>(ceil_div(p.key_tiles, kWgtGridY)));
    constexpr int MOST = wgt_most_columns<BF16, DP>();
    if (a.rows == 0) {}                                       // (no tokens: the totals are what they were)
    else if (p.g_rows == 1) civic::launch(weights_stats_kernel<BF16, DP, FULL, 1>, rows, block, 0, s, a);
    else if (p.g_rows == 2) civic::launch(weights_stats_kernel<BF16, DP, FULL, 2>, rows, block, 0, s, a);
    else if (p.g_rows == 4) { if constexpr (MOST >= 4) civic::launch(weights_stats_kernel<BF16, DP, FULL, 4>, rows, block, 0, s, a); }
    else if constexpr (MOST >= 8) civic::launch(weights_stats_kernel<BF16, DP, FULL, 8>, rows, block, 0, s, a);
    if (p.g_keys == 2) civic::launch(weights_sums_kernel<BF16, DP, FULL, 2>, keys, block, 0, s, a);
    else if (p.g_keys == 4) { if constexpr (MOST >= 4) civic::launch(weights_sums_kernel<BF16, DP, FULL, 4>, keys, block, 0, s, a); }
    else if constexpr (MOST >= 8) civic::launch(weights_sums_kernel<BF16, DP, FULL, 8>, keys, block, 0, s, a);
}

template <bool BF16>
static void launch_weights_dim(const WeightsArgs& a, const WeightsPlan& p, hipStream_t s)
{
    const int d = a.head_dim;
    if (d == 64) launch_weights<BF16, 64, true>(a, p, s);
    else if (d == 128) launch_weights<BF16, 128, true>(a, p, s);
    else if (d == 256) launch_weights<BF16, 256, true>(a, p, s);
    else if (d < 64) launch_weights<BF16, 64, false>(a, p, s);
    else if (d < 128) launch_weights<BF16, 128, false>(a, p, s);
    else launch_weights<BF16, 256, false>(a, p, s);
}

static size_t weights_ws_bytes(const WeightsPlan& p, int32_t batch, int64_t rows, int32_t n_kv_heads)
{
    return sizeof(float2) * static_cast<size_t>(batch) * n_kv_heads * rows * p.most_pieces;
}

}  // namespace civic

extern "C" size_t civic_attn_weights_workspace_bytes(int dtype, int32_t batch, int32_t seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t n_ctx)
{
    using namespace civic;
    if (!weights_sizes_ok(dtype, batch, seq, n_q_heads, n_kv_heads, head_dim, n_ctx)
        || !weights_covered(batch, seq, n_q_heads, n_kv_heads, head_dim, n_ctx) || batch == 0 || seq == 0) return 0;
    const int64_t rows = static_cast<int64_t>(seq) * (n_q_heads / n_kv_heads);
    return weights_ws_bytes(weights_plan(dtype == CIVIC_BF16, batch, rows, n_kv_heads, head_dim, n_ctx, n_ctx), batch, rows, n_kv_heads);
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
    const WeightsPlan p = weights_plan(dtype == CIVIC_BF16, batch, std::max(a.rows, 1), n_kv_heads, head_dim, s_max, n_ctx);
    const size_t need = weights_ws_bytes(p, batch, a.rows, n_kv_heads);
    if (need && (!workspace || workspace_bytes < need)) return CIVIC_ERR_WORKSPACE;
    a.q = q; a.kc = k_cache; a.ctx = ctx; a.base = base; a.weights = weights; a.stats = static_cast<float2*>(workspace);
    for (int i = 0; i < 3; ++i) a.qs[i] = q_strides[i];
    a.s_max = s_max; a.batch = batch; a.seq = seq; a.n_q_heads = n_q_heads; a.n_kv_heads = n_kv_heads; a.head_dim = head_dim;
    a.causal = causal != 0; a.n_ctx = static_cast<int32_t>(n_ctx);
    a.row_tiles = static_cast<int32_t>(p.row_tiles); a.pieces = static_cast<int32_t>(p.pieces); a.piece_tiles = static_cast<int32_t>(p.piece_tiles);
    const LogitScale scale = logit_scale(softmax_scale, head_dim, dtype == CIVIC_BF16);
    a.scale = scale.log2; a.flip = scale.flip;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == CIVIC_BF16) launch_weights_dim<true>(a, p, s);
    else launch_weights_dim<false>(a, p, s);
    return check_launch();
}
