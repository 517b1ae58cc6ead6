// civic_kv_evict: a cache keeps, of every (sample, KV head), the rows that have received the most attention, with its first and its
// latest ones; they move together to rows [0, m) in their order, m = min(ctx, keep).
//
// The least weight that stays is found by counting the candidates' leading 11 bits in LDS, then the next 11, then the last 10 of those that
// share what is settled so far; equal weights stay from the lowest row on.  Each wavefront then goes through a run of consecutive rows, 64
// at a time, counts what stays and, when the counts before it are known, writes the rows' numbers.
//   - Up to kSelectRows rows a workgroup of 16 wavefronts does that for a pair of sample and KV head, its keys in registers, in one launch; it
//     moves K and V as well where they are few bytes.
//   - Longer caches are cut into pieces, and each of the four passes is a launch: a workgroup adds up the bins that the last one left for all
//     pieces (8 KB each, out of the second cache), settles the bits and counts what lies above them before its piece.  One workgroup to a pair
//     needed 68 us for 65000 keys, most of it the LDS's additions.
// Then K and V are moved, 16 bytes a thread: bound by memory.  In place a workgroup takes 128 or 64 bytes of every row of a pair's K or V from the
// first row to the last: a row's source lies at or behind it, so a run of rows is read before it is written, and what is read later lies
// behind all that is written.
#include "rows_device.h"

namespace civic {

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / kWave;
constexpr int kMoveThreads = 256, kMoveRows = 64;             // rows of a workgroup of the second launch
constexpr int kSelectRows = 16 * kEvictThreads;
constexpr int kSpreadThreads = 512, kSpreadWaves = kSpreadThreads / kWave, kSpreadU = 8;   // long caches: keys of a thread at a time
constexpr int kSpreadRows = kSpreadThreads * kSpreadU, kSpreadMost = 32;                   // of a piece, or a multiple; pieces of a pair
constexpr int kPlaceThreads = 1024, kPlaceU = 4;   // in place

struct EvictArgs {
    const void* k; const void* v; const float* weights; const int32_t* ctx;
    void* k_out; void* v_out; float* weights_out; int32_t* kept_idx; int32_t* ctx_out;
    int32_t* held;                                            // workspace: rows that every pair keeps
    int64_t s_max, s_out;
    int32_t n_kv_heads, n_ctx, keep, first, recent;
    int32_t pieces;                                           // of 16 bytes of a row
    uint32_t magic;                                           // ceil(2^32 / pieces)
    int32_t chunks;                                           // moving launch: workgroups of a pair
    int32_t spread, spread_rows;                              // pieces of a long cache, their rows
    int64_t pairs;
    uint2* state;                                             // workspace: [2, pairs] bits settled so far, how many of the candidates that share them stay
    uint32_t* before;                                         // [pairs, pieces] candidates above those bits in the pieces before
    uint32_t* hist;                                           // [3, pairs, pieces, kBins]
    float* stash;                                             // [pairs, n_ctx] the kept weights (they may be written over what is selected from)
    uint32_t items;                                           // workgroups of pairs of the launch that writes the weights; those behind them clear rows from `cleared` on
    int64_t cleared;                                          // rows of weights_out of a pair that its own workgroups write
};

// Weights as numbers whose order is theirs: -0 as 0, NaN below everything.
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = x == 0.f ? 0u : __float_as_uint(x);
    return x != x ? 0u : u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}

constexpr int kBins = 2048;
// The first pass has four copies of its bins, a lane's by its number: weights lie within some twenty powers of two, four bins to each, and
// lanes that add to one bin wait for each other.  Copies begin on different banks.
constexpr int kCopies = 4, kCopyPitch = kBins + 8;

// `count`: candidates in a thread's bins, consecutive ones from the top -> found: the bin in which the `need`-th largest lies, and the
// candidates above that bin.
template <int THREADS>
__device__ __forceinline__ void border_bin(const uint32_t (&count)[kBins / THREADS], uint32_t need, uint32_t* sums, uint32_t* found)
{
    constexpr int N = kBins / THREADS;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = tid >> 6;
    uint32_t own = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) own += count[j];
    uint32_t upto = own;
    for (int off = 1; off < kWave; off <<= 1) { const uint32_t y = __shfl_up(upto, off, kWave); if (lane >= off) upto += y; }
    if (lane == kWave - 1) sums[w] = upto;
    __syncthreads();
    uint32_t before = upto - own;
    for (int x = 0; x < w; ++x) before += sums[x];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (before < need && need <= before + count[j]) { found[0] = kBins - 1 - (N * tid + j); found[1] = before; }
        before += count[j];
    }
    __syncthreads();
}

// One more candidate in bin `bin` for every lane that is `in`.
__device__ __forceinline__ void count_in(uint32_t* mine, uint32_t bin, bool in, int lane)
{
    const uint64_t who = __ballot(in);
    if (who == 0) return;
    // (the same bin for all of them, as of weights that are all 0: one addition)
    const uint32_t one = __builtin_amdgcn_readlane(bin, __builtin_ctzll(who));
    if (__ballot(in && bin != one) == 0) { if (lane == 0) atomicAdd(&mine[one], static_cast<uint32_t>(__popcll(who))); }
    else if (in) atomicAdd(&mine[bin], 1u);
}

// KPT: keys that a thread holds in registers, rows [w * 64 KPT, ...) of the pair a wavefront's.
// MOVE: the rows are moved here as well, in runs that are read before they are written (the caches may be changed in place).
template <int KPT, bool MOVE>
__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(EvictArgs a)
{
    __shared__ uint32_t bins[kCopies * kCopyPitch];
    __shared__ uint32_t sums[kEvictWaves];
    __shared__ uint32_t found[2];                             // the bin of the border, candidates above it
    __shared__ uint32_t more[kEvictWaves], equal[kEvictWaves];
    if (blockIdx.x >= a.items) {
        weights_behind<kEvictThreads>(nullptr, a.weights_out, a.items, a.s_out, a.cleared, blockIdx.x - a.items, gridDim.x - a.items);
        return;
    }
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t pair = blockIdx.x;
    const int n = clamped(a.ctx, static_cast<int>(pair / a.n_kv_heads), a.n_ctx), m = min(n, a.keep);
    const float* const weights = a.weights + pair * a.s_max;
    int32_t* const idx = a.kept_idx + pair * a.keep;
    if (tid == 0) a.held[pair] = m;
    if (n <= a.keep) {
        for (int i = tid; i < n; i += kEvictThreads) idx[i] = i;
    } else {
        const int lo = a.first, hi = n - a.recent;            // the candidates
        // a wavefront's rows: a run of whole 64s
        const int r0 = min(w * KPT * kWave, n), r1 = min(r0 + KPT * kWave, n);
        uint32_t key[KPT];
#pragma unroll
        for (int u = 0; u < KPT; ++u) key[u] = ordered(weights[min(r0 + u * kWave + lane, n - 1)]);
        uint32_t need = static_cast<uint32_t>(a.keep - a.first - a.recent), border = 0xFFFFFFFFu;
        // The largest `need` candidates: those above `border` and `need` equal ones.  (need = 0: no number is above the border, and none
        // of those equal to it is taken.)
        if (need > 0) {
            uint32_t settled = 0;
#pragma unroll
            for (int pass = 0; pass < 3; ++pass) {
                const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11, copies = pass == 0 ? kCopies : 1;
                for (int i = tid; i < copies * kCopyPitch; i += kEvictThreads) bins[i] = 0;
                __syncthreads();
                uint32_t* const mine = bins + (pass == 0 ? (lane & (kCopies - 1)) * kCopyPitch : 0);
#pragma unroll
                for (int u = 0; u < KPT; ++u) {
                    const int row = r0 + u * kWave + lane;
                    const bool in = row >= lo && row < hi && row < r1 && (pass == 0 || (key[u] >> (shift + width)) == settled);
                    count_in(mine, (key[u] >> shift) & ((1u << width) - 1u), in, lane);
                }
                __syncthreads();
                // a thread's two bins, from the top; how many candidates lie above them
                uint32_t count[2] = {0, 0};
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    for (int c = 0; c < copies; ++c) count[j] += bins[c * kCopyPitch + kBins - 1 - (2 * tid + j)];
                border_bin<kEvictThreads>(count, need, sums, found);
                settled = settled << width | found[0];
                need -= found[1];
            }
            border = settled;
        }
        auto look = [&](int row, uint32_t o, bool& above, bool& tied) __attribute__((always_inline)) {
            const bool fixed = row < lo || row >= hi;
            above = row < r1 && (fixed || o > border);
            tied = row < r1 && !fixed && o == border;
        };
        uint32_t above_n = 0, tied_n = 0;
#pragma unroll
        for (int u = 0; u < KPT; ++u) {
            bool above, tied;
            look(r0 + u * kWave + lane, key[u], above, tied);
            above_n += __popcll(__ballot(above));
            tied_n += __popcll(__ballot(tied));
        }
        if (lane == 0) { more[w] = above_n; equal[w] = tied_n; }
        __syncthreads();
        uint32_t at = 0, ties = 0;                             // rows above the border, rows equal to it, before the wavefront's
        for (int x = 0; x < w; ++x) { at += more[x]; ties += equal[x]; }
        const uint64_t below = (uint64_t{1} << lane) - 1;
#pragma unroll
        for (int u = 0; u < KPT; ++u) {
            const int row = r0 + u * kWave + lane;
            bool above, tied;
            look(row, key[u], above, tied);
            const uint64_t all_above = __ballot(above), all_tied = __ballot(tied);
            const uint32_t my_above = at + __popcll(all_above & below), my_ties = ties + __popcll(all_tied & below);
            if (above || (tied && my_ties < need)) idx[my_above + min(my_ties, need)] = row;
            at += __popcll(all_above);
            ties += __popcll(all_tied);
        }
    }
    for (int i = m + tid; i < a.keep; i += kEvictThreads) idx[i] = -1;
    if constexpr (MOVE) {
        if (tid == 0 && a.ctx_out != nullptr && pair % a.n_kv_heads == 0) a.ctx_out[pair / a.n_kv_heads] = m;
        const u32x4* const k = static_cast<const u32x4*>(a.k) + pair * a.s_max * a.pieces;
        const u32x4* const v = static_cast<const u32x4*>(a.v) + pair * a.s_max * a.pieces;
        u32x4* const ko = static_cast<u32x4*>(a.k_out) + pair * a.s_out * a.pieces;
        u32x4* const vo = static_cast<u32x4*>(a.v_out) + pair * a.s_out * a.pieces;
        constexpr int MU = 2;
        const int total = m * a.pieces;
        __syncthreads();
        u32x4 x[MU], y[MU];
        auto fetch_rows = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < MU; ++u) {
                const int i = i0 + u * kEvictThreads + tid;
                if (i < total) {
                    const int r = a.pieces == 1 ? i : static_cast<int>(__umulhi(static_cast<uint32_t>(i), a.magic));
                    const int64_t src = static_cast<int64_t>(idx[r]) * a.pieces + (i - r * a.pieces);
                    x[u] = load_streaming(k + src);
                    y[u] = load_streaming(v + src);
                }
            }
        };
        fetch_rows(0);
        for (int i0 = 0; i0 < total; i0 += MU * kEvictThreads) {
            u32x4 xs[MU], ys[MU];
#pragma unroll
            for (int u = 0; u < MU; ++u) { xs[u] = x[u]; ys[u] = y[u]; }
            __syncthreads();                                  // the run has been read by all
            if (i0 + MU * kEvictThreads < total) fetch_rows(i0 + MU * kEvictThreads);
#pragma unroll
            for (int u = 0; u < MU; ++u) {
                const int i = i0 + u * kEvictThreads + tid;
                if (i < total) { store_streaming(ko + i, xs[u]); store_streaming(vo + i, ys[u]); }
            }
        }
    }
    if (a.weights_out == nullptr) return;
    // the kept weights: a run of them is read before it is written, and what is read later lies behind (the arrays may be one)
    float* const out = a.weights_out + pair * a.s_out;
    constexpr int RUN = 4;
    __syncthreads();
    for (int i0 = 0; i0 < m; i0 += RUN * kEvictThreads) {
        float x[RUN];
#pragma unroll
        for (int j = 0; j < RUN; ++j) { const int i = i0 + j * kEvictThreads + tid; x[j] = i < m ? weights[idx[i]] : 0.f; }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < RUN; ++j) { const int i = i0 + j * kEvictThreads + tid; if (i < m) out[i] = x[j]; }
    }
    __syncthreads();
    for (int64_t i = m + tid; i < a.cleared; i += kEvictThreads) out[i] = 0.f;
}

// A pass over long caches: counts the candidates that share the bits settled by the passes before (0, 1, 2), or numbers the rows that stay (3).
// grid: pairs * pieces
template <int PASS>
__global__ __launch_bounds__(kSpreadThreads) void evict_spread_kernel(EvictArgs a)
{
    constexpr int COPIES = PASS == 0 ? kCopies : 1, N = kBins / kSpreadThreads;
    static_assert(N == 4, "a thread's bins are one load");
    __shared__ __attribute__((aligned(16))) uint32_t bins[PASS < 3 ? COPIES * kCopyPitch : 4];
    __shared__ uint32_t sums[kSpreadWaves], found[2];
    __shared__ uint32_t more[kSpreadWaves], equal[kSpreadWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t pair = blockIdx.x / a.spread;
    const int piece = blockIdx.x - static_cast<uint32_t>(pair) * a.spread;
    const int n = clamped(a.ctx, static_cast<int>(pair / a.n_kv_heads), a.n_ctx), m = min(n, a.keep);
    const float* const weights = a.weights + pair * a.s_max;
    const int lo = a.first, hi = n - a.recent;                // the candidates
    const int r0 = static_cast<int>(min(static_cast<int64_t>(piece) * a.spread_rows, static_cast<int64_t>(n))), r1 = min(r0 + a.spread_rows, n);
    uint32_t need = static_cast<uint32_t>(a.keep - a.first - a.recent), settled = 0;
    uint32_t before = 0, ties = 0;                            // candidates of the pieces before: above the settled bits; that share them
    const bool chosen = n > a.keep && need > 0;
    if (PASS > 0 && chosen) {
        if constexpr (PASS > 1) {
            const uint2 state = a.state[(PASS - 2) * a.pairs + pair];
            settled = state.x; need = state.y;
            before = a.before[blockIdx.x];
        }
        const uint4* const of = reinterpret_cast<const uint4*>(a.hist + ((PASS - 1) * a.pairs + pair) * a.spread * kBins) + (kSpreadThreads - 1 - tid);
        uint32_t count[N] = {0, 0, 0, 0}, earlier[N] = {0, 0, 0, 0};   // of all pieces; of those before
#pragma unroll 8
        for (int p = 0; p < a.spread; ++p) {
            const uint4 c = of[p * kSpreadThreads];
            const uint32_t cc[N] = {c.w, c.z, c.y, c.x};
#pragma unroll
            for (int j = 0; j < N; ++j) { count[j] += cc[j]; earlier[j] += p < piece ? cc[j] : 0u; }
        }
        border_bin<kSpreadThreads>(count, need, sums, found);
        const int top = kBins - 1 - N * tid, bin = found[0];
        uint32_t over = 0, same = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) { over += top - j > bin ? earlier[j] : 0u; same += top - j == bin ? earlier[j] : 0u; }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) { over += __shfl_xor(over, off, kWave); same += __shfl_xor(same, off, kWave); }
        if (lane == 0) { more[w] = over; equal[w] = same; }
        __syncthreads();
        for (int x = 0; x < kSpreadWaves; ++x) { before += more[x]; ties += equal[x]; }
        settled = settled << (PASS == 3 ? 10 : 11) | bin;
        need -= found[1];
        if (PASS < 3 && tid == 0) {
            a.before[blockIdx.x] = before;
            if (piece == 0) a.state[(PASS - 1) * a.pairs + pair] = make_uint2(settled, need);
        }
        __syncthreads();
    }
    if constexpr (PASS < 3) {
        if (!chosen) return;
        constexpr int SHIFT = PASS == 0 ? 21 : PASS == 1 ? 10 : 0, WIDTH = PASS == 2 ? 10 : 11;
        for (int i = tid; i < COPIES * kCopyPitch; i += kSpreadThreads) bins[i] = 0;
        __syncthreads();
        uint32_t* const mine = bins + (lane & (COPIES - 1)) * kCopyPitch;
        for (int r = r0; r < r1; r += kSpreadRows) {
            uint32_t key[kSpreadU];
#pragma unroll
            for (int u = 0; u < kSpreadU; ++u) key[u] = ordered(weights[min(r + u * kSpreadThreads + tid, n - 1)]);
#pragma unroll
            for (int u = 0; u < kSpreadU; ++u) {
                const int row = r + u * kSpreadThreads + tid;
                const bool in = row >= lo && row < hi && row < r1 && (PASS == 0 || (key[u] >> ((SHIFT + WIDTH) & 31)) == settled);
                count_in(mine, (key[u] >> SHIFT) & ((1u << WIDTH) - 1u), in, lane);
            }
        }
        __syncthreads();
        uint4* const to = reinterpret_cast<uint4*>(a.hist + ((PASS * a.pairs + pair) * a.spread + piece) * kBins);
        uint4 c = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int x = 0; x < COPIES; ++x) {
            const uint4 y = *reinterpret_cast<const uint4*>(bins + x * kCopyPitch + N * tid);
            c.x += y.x; c.y += y.y; c.z += y.z; c.w += y.w;
        }
        to[tid] = c;
    } else {
        int32_t* const idx = a.kept_idx + pair * a.keep;
        float* const stash = a.stash + pair * a.n_ctx;
        if (piece == 0 && tid == 0) a.held[pair] = m;
        for (int i = m + piece * kSpreadThreads + tid; i < a.keep; i += a.spread * kSpreadThreads) idx[i] = -1;
        if (n <= a.keep) {
            for (int i = r0 + tid; i < r1; i += kSpreadThreads) { idx[i] = i; stash[i] = weights[i]; }
            return;
        }
        const uint32_t border = chosen ? settled : 0xFFFFFFFFu;
        uint32_t at = before + min(r0, lo) + max(r0 - hi, 0);  // rows above the border, or kept in any case, so far
        const uint64_t below = (uint64_t{1} << lane) - 1;
        for (int r = r0; r < r1; r += kSpreadRows) {
            const int rw = r + w * kSpreadU * kWave;           // (a wavefront's rows follow each other here)
            float x[kSpreadU];
            uint32_t above_n = 0, tied_n = 0;
            uint64_t above[kSpreadU], tied[kSpreadU];
#pragma unroll
            for (int u = 0; u < kSpreadU; ++u) x[u] = weights[min(rw + u * kWave + lane, n - 1)];
#pragma unroll
            for (int u = 0; u < kSpreadU; ++u) {
                const int row = rw + u * kWave + lane;
                const uint32_t o = ordered(x[u]);
                const bool fixed = row < lo || row >= hi;
                above[u] = __ballot(row < r1 && (fixed || o > border));
                tied[u] = __ballot(row < r1 && !fixed && o == border);
                above_n += __popcll(above[u]);
                tied_n += __popcll(tied[u]);
            }
            if (lane == 0) { more[w] = above_n; equal[w] = tied_n; }
            __syncthreads();
            uint32_t at_w = at, ties_w = ties;
            for (int y = 0; y < kSpreadWaves; ++y) {
                if (y < w) { at_w += more[y]; ties_w += equal[y]; }
                at += more[y]; ties += equal[y];
            }
#pragma unroll
            for (int u = 0; u < kSpreadU; ++u) {
                const uint32_t my_ties = ties_w + __popcll(tied[u] & below), to = at_w + __popcll(above[u] & below) + min(my_ties, need);
                if (above[u] >> lane & 1 || (tied[u] >> lane & 1 && my_ties < need)) { idx[to] = rw + u * kWave + lane; stash[to] = x[u]; }
                at_w += __popcll(above[u]);
                ties_w += __popcll(tied[u]);
            }
            __syncthreads();
        }
    }
}

// The kept weights of a pair of long caches, and zeros behind them, by workgroup `part` of `parts`.
template <int THREADS>
__device__ __forceinline__ void weights_of_long(const EvictArgs& a, int64_t pair, int m, int part, int parts)
{
    if (a.stash == nullptr || a.weights_out == nullptr) return;
    const float* const stash = a.stash + pair * a.n_ctx;
    float* const out = a.weights_out + pair * a.s_out;
    for (int64_t i = part * THREADS + static_cast<int>(threadIdx.x); i < a.cleared; i += parts * THREADS) out[i] = i < m ? stash[i] : 0.f;
}

// grid: pairs * chunks of kMoveRows rows
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a)
{
    const int64_t pair = blockIdx.x / a.chunks;
    const int chunk = blockIdx.x - static_cast<uint32_t>(pair) * a.chunks, r0 = chunk * kMoveRows, m = a.held[pair];
    if (chunk == 0 && threadIdx.x == 0 && a.ctx_out != nullptr && pair % a.n_kv_heads == 0) a.ctx_out[pair / a.n_kv_heads] = m;
    weights_of_long<kMoveThreads>(a, pair, m, chunk, a.chunks);
    const int rows = min(kMoveRows, m - r0);
    if (rows <= 0) return;
    const int32_t* const idx = a.kept_idx + pair * a.keep + r0;
    const u32x4* const k = static_cast<const u32x4*>(a.k) + pair * a.s_max * a.pieces;
    const u32x4* const v = static_cast<const u32x4*>(a.v) + pair * a.s_max * a.pieces;
    u32x4* const ko = static_cast<u32x4*>(a.k_out) + (pair * a.s_out + r0) * a.pieces;
    u32x4* const vo = static_cast<u32x4*>(a.v_out) + (pair * a.s_out + r0) * a.pieces;
    const int total = rows * a.pieces;
    constexpr int U = 4;
    for (int i0 = threadIdx.x; i0 < total; i0 += U * kMoveThreads) {
        u32x4 x[U], y[U];
        int64_t src[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = min(i0 + u * kMoveThreads, total - 1);
            const int r = a.pieces == 1 ? i : static_cast<int>(__umulhi(static_cast<uint32_t>(i), a.magic));
            src[u] = static_cast<int64_t>(idx[r]) * a.pieces + (i - r * a.pieces);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) { x[u] = load_streaming(k + src[u]); y[u] = load_streaming(v + src[u]); }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * kMoveThreads;
            if (i < total) { store_streaming(ko + i, x[u]); store_streaming(vo + i, y[u]); }
        }
    }
}

// In place.  grid: pairs * 2 (K, V) * slices of PIECES pieces of a row
template <int PIECES>
__global__ __launch_bounds__(kPlaceThreads) void evict_place_kernel(EvictArgs a)
{
    const int slices = (a.pieces + PIECES - 1) / PIECES;
    if (blockIdx.x >= a.items) {
        weights_behind<kPlaceThreads>(nullptr, a.weights_out, a.pairs, a.s_out, a.cleared, blockIdx.x - a.items, gridDim.x - a.items);
        return;
    }
    const uint32_t u0 = blockIdx.x / slices, slice = blockIdx.x - u0 * slices;
    const int64_t pair = u0 >> 1;
    const int m = a.held[pair];
    if (slice == 0 && (u0 & 1) == 0 && threadIdx.x == 0 && a.ctx_out != nullptr && pair % a.n_kv_heads == 0) a.ctx_out[pair / a.n_kv_heads] = m;
    weights_of_long<kPlaceThreads>(a, pair, m, static_cast<int>(2 * slice + (u0 & 1)), 2 * slices);
    if (m < a.keep) return;                                   // (all rows stay where they are; as many as are kept: they may)
    const int32_t* const idx = a.kept_idx + pair * a.keep;
    u32x4* const rows = static_cast<u32x4*>((u0 & 1) ? a.v_out : a.k_out) + pair * a.s_max * a.pieces;
    const int piece = slice * PIECES + threadIdx.x % PIECES, y = threadIdx.x / PIECES;
    constexpr int STEP = kPlaceThreads / PIECES, RUN = STEP * kPlaceU;
    const bool there = piece < a.pieces;
    u32x4 x[kPlaceU];
    auto fetch = [&](int r0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kPlaceU; ++u) {
            const int r = r0 + u * STEP + y;
            if (r < m && there) x[u] = rows[static_cast<int64_t>(idx[r]) * a.pieces + piece];
        }
    };
    fetch(0);
    for (int r0 = 0; r0 < m; r0 += RUN) {
        u32x4 z[kPlaceU];
#pragma unroll
        for (int u = 0; u < kPlaceU; ++u) z[u] = x[u];
        __syncthreads();                                      // the run has been read by all
        if (r0 + RUN < m) fetch(r0 + RUN);
#pragma unroll
        for (int u = 0; u < kPlaceU; ++u) {
            const int r = r0 + u * STEP + y;
            if (r < m && there) rows[static_cast<int64_t>(r) * a.pieces + piece] = z[u];
        }
    }
}

// Bytes of K and V of a pair that the workgroup which selects them moves as well: a launch less (us, so and in two launches: 156 of 469 rows of 128
// bf16 channels, 8 heads 9.9, 13.0; but 2048 of 8192 40.6, 20.2, and 1024 of 3584 of 512 pairs, more than there are units, 119.5, 106).
constexpr int64_t kSelectMoves = 256 * 1024;

constexpr int64_t kEvictMaxPairs = int64_t{1} << 21, kEvictMaxBlocks = int64_t{1} << 23;   // launches of fewer than 2^32 threads

// Pieces of a row of a workgroup that moves rows in place: 128 bytes, or 64 where that leaves more than three units of four without work.  (us of the call,
// with 128 and 64: 8 pairs of 256-byte rows, 8192 of 65000 kept 68, 56, 20000 of 200000 135, 102; 32 pairs, 8192 of 30000 76, 94; 64, 2048 of 8192 40, 50;
// 512, 1024 of 3584 102, 142.)
static int place_pieces(int64_t pairs, int pieces) { return pairs * 2 * ceil_div(pieces, 8) <= 64 ? 4 : 8; }

// Pieces of a pair: as many as fill the chip twice, of kSpreadRows rows or more.
static int64_t spread_pieces(int64_t pairs, int64_t n_ctx)
{
    return std::max<int64_t>(1, std::min<int64_t>({kSpreadMost, ceil_div(512, pairs), ceil_div(n_ctx, kSpreadRows)}));
}

}  // namespace civic

extern "C" size_t civic_kv_evict_workspace_bytes(int32_t batch, int32_t n_kv_heads, int64_t n_ctx)
{
    if (batch <= 0 || n_kv_heads <= 0 || n_ctx < 0 || static_cast<int64_t>(batch) * n_kv_heads > civic::kEvictMaxPairs) return 0;
    const size_t pairs = static_cast<size_t>(batch) * n_kv_heads;
    if (n_ctx <= civic::kSelectRows) return sizeof(int32_t) * pairs;
    // rows held, state, counts before the pieces, bins (16-byte aligned), kept weights
    return sizeof(int32_t) * (pairs * (1 + 4 + static_cast<size_t>(n_ctx)) + 8 + pairs * civic::spread_pieces(pairs, n_ctx) * (1 + 3 * civic::kBins));
}

extern "C" int civic_kv_evict(const void* k_cache, const void* v_cache, const float* weights, int dtype, int32_t batch, int32_t n_kv_heads,
                              int32_t head_dim, int64_t s_max, int64_t n_ctx, const int32_t* ctx, int64_t keep, int64_t first, int64_t recent,
                              void* k_out, void* v_out, float* weights_out, int32_t* kept_idx, int32_t* ctx_out, int64_t s_max_out,
                              void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace civic;
    const int esz = dtype_size(dtype);
    if (!esz || batch < 0 || n_kv_heads <= 0 || head_dim <= 0 || head_dim % 8 || s_max < 0 || n_ctx < 0 || n_ctx > s_max) return CIVIC_ERR_INVALID_ARG;
    if (first < 0 || recent < 0 || keep < 0 || first > keep || recent > keep - first || s_max_out < 0) return CIVIC_ERR_INVALID_ARG;
    if (std::min(keep, n_ctx) > s_max_out) return CIVIC_ERR_INVALID_ARG;
    const bool any = batch > 0, rows = any && n_ctx > 0 && keep > 0;
    if (rows && (!k_cache || !v_cache || !weights || !k_out || !v_out)) return CIVIC_ERR_INVALID_ARG;
    if (any && keep > 0 && !kept_idx) return CIVIC_ERR_INVALID_ARG;
    for (const void* p : {k_cache, v_cache, static_cast<const void*>(k_out), static_cast<const void*>(v_out)})
        if (!aligned16(p)) return CIVIC_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(weights), static_cast<const void*>(weights_out), static_cast<const void*>(kept_idx),
                          static_cast<const void*>(ctx), static_cast<const void*>(ctx_out), static_cast<const void*>(workspace)})
        if (reinterpret_cast<uintptr_t>(p) & 3u) return CIVIC_ERR_INVALID_ARG;
    if (head_dim > CIVIC_MAX_HEAD_DIM || s_max > kCacheMaxRows || s_max_out > kCacheMaxRows || keep > kCacheMaxRows
        || static_cast<int64_t>(batch) * n_kv_heads > kEvictMaxPairs) return CIVIC_ERR_UNSUPPORTED;
    const int64_t pairs = static_cast<int64_t>(batch) * n_kv_heads, most = std::min(keep, n_ctx);
    const int pieces = head_dim * esz / 16, place = place_pieces(pairs, pieces), slices = static_cast<int>(ceil_div(pieces, place));
    const int64_t chunks = std::max<int64_t>(1, ceil_div(most, kMoveRows));
    const bool in_place = rows && k_out == k_cache;
    if (in_place ? pairs * 2 * slices * kPlaceThreads >= (int64_t{1} << 32) : pairs * chunks > kEvictMaxBlocks) return CIVIC_ERR_UNSUPPORTED;
    if (!any) return CIVIC_OK;
    // written arrays share no memory with read ones or with each other, but for the caches, weights and lengths that are changed in place
    const int64_t in_bytes = rows ? pairs * s_max * head_dim * esz : 0, out_bytes = rows ? pairs * s_max_out * head_dim * esz : 0;
    if (in_place && (v_out != v_cache || s_max_out != s_max)) return CIVIC_ERR_INVALID_ARG;
    if (rows && weights_out && weights_out == weights && s_max_out != s_max) return CIVIC_ERR_INVALID_ARG;
    const Memory k_in{in_place ? nullptr : k_cache, in_bytes}, v_in{in_place ? nullptr : v_cache, in_bytes};
    const Memory sums_in{weights_out == weights ? nullptr : weights, rows ? pairs * s_max * 4 : 0}, lengths_in{ctx_out == ctx ? nullptr : ctx, batch * int64_t{4}};
    const Memory k_to{k_out, out_bytes}, v_to{v_out, out_bytes}, sums_to{weights_out, pairs * s_max_out * 4}, numbers{kept_idx, pairs * keep * 4},
                 lengths_to{ctx_out, batch * int64_t{4}};
    if (!writes_apart({k_to, v_to, sums_to, numbers, lengths_to}, {k_in, v_in, sums_in, lengths_in})) return CIVIC_ERR_INVALID_ARG;
    const size_t need = civic_kv_evict_workspace_bytes(batch, n_kv_heads, n_ctx);
    if (!workspace || workspace_bytes < need) return CIVIC_ERR_WORKSPACE;
    if (!writes_apart({{workspace, static_cast<int64_t>(need)}}, {k_in, v_in, sums_in, lengths_in, k_to, v_to, sums_to, numbers, lengths_to})) return CIVIC_ERR_INVALID_ARG;
    EvictArgs a{};
    a.k = k_cache; a.v = v_cache; a.weights = weights; a.ctx = ctx;
    a.k_out = k_out; a.v_out = v_out; a.weights_out = weights_out; a.kept_idx = kept_idx; a.ctx_out = ctx_out;
    a.held = static_cast<int32_t*>(workspace);
    a.s_max = s_max; a.s_out = s_max_out;
    a.n_kv_heads = n_kv_heads; a.n_ctx = static_cast<int32_t>(rows ? n_ctx : 0); a.keep = static_cast<int32_t>(keep);
    a.first = static_cast<int32_t>(first); a.recent = static_cast<int32_t>(recent);
    a.pieces = pieces;
    a.magic = static_cast<uint32_t>(((int64_t{1} << 32) + pieces - 1) / pieces);
    a.chunks = static_cast<int32_t>(chunks);
    hipStream_t s = static_cast<hipStream_t>(stream);
    // (not where the lengths are changed in place: pairs of a sample that begin later read them)
    const bool short_cache = a.n_ctx <= kSelectRows;
    // rows of weights_out behind n_ctx: by workgroups of their own in the launch of the selection, of the move in place (into others that has many to a pair)
    const unsigned behind = weights_out && (short_cache || in_place) ? behind_blocks(pairs, s_max_out, a.n_ctx, kEvictThreads) : 0;
    a.cleared = behind ? a.n_ctx : s_max_out;
    a.items = static_cast<uint32_t>(pairs);
    const bool one = rows && (ctx_out == nullptr || ctx_out != ctx) && n_ctx <= 16 * kEvictThreads && most * pieces * 32 <= kSelectMoves;
    const dim3 block(kEvictThreads);
    if (one) {
        const auto select = n_ctx <= kEvictThreads ? evict_select_kernel<1, true> : n_ctx <= 4 * kEvictThreads ? evict_select_kernel<4, true> : evict_select_kernel<16, true>;
        civic::launch(select, dim3(a.items + behind), block, 0, s, a);
        return check_launch();
    }
    if (short_cache) {
        const auto select = n_ctx <= kEvictThreads ? evict_select_kernel<1, false> : n_ctx <= 4 * kEvictThreads ? evict_select_kernel<4, false> : evict_select_kernel<16, false>;
        civic::launch(select, dim3(a.items + behind), block, 0, s, a);
    } else {
        a.pairs = pairs;
        a.spread = static_cast<int32_t>(spread_pieces(pairs, n_ctx));
        a.spread_rows = static_cast<int32_t>(ceil_div(ceil_div(n_ctx, a.spread), kSpreadRows) * kSpreadRows);
        uintptr_t at = reinterpret_cast<uintptr_t>(workspace) + pairs * sizeof(int32_t);
        at = (at + 15) & ~uintptr_t{15};
        a.hist = reinterpret_cast<uint32_t*>(at); at += sizeof(uint32_t) * 3 * pairs * a.spread * kBins;
        a.state = reinterpret_cast<uint2*>(at); at += sizeof(uint2) * 2 * pairs;
        a.before = reinterpret_cast<uint32_t*>(at); at += sizeof(uint32_t) * pairs * a.spread;
        a.stash = reinterpret_cast<float*>(at);
        const dim3 grid(static_cast<unsigned>(pairs * a.spread));
        for (const auto pass : {evict_spread_kernel<0>, evict_spread_kernel<1>, evict_spread_kernel<2>, evict_spread_kernel<3>})
            civic::launch(pass, grid, dim3(kSpreadThreads), 0, s, a);
    }
    const int rc = check_launch();
    if (rc != CIVIC_OK) return rc;
    const auto place_rows = place == 8 ? evict_place_kernel<8> : evict_place_kernel<4>;
    a.items = static_cast<uint32_t>(pairs * 2 * slices);
    if (in_place) civic::launch(place_rows, dim3(a.items + (short_cache ? 0 : behind)), dim3(kPlaceThreads), 0, s, a);
    else civic::launch(evict_move_kernel, dim3(static_cast<unsigned>(pairs * chunks)), dim3(kMoveThreads), 0, s, a);
    return check_launch();
}
