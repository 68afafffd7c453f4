// The attention weight that every cached token received (psa_accumulate_weights): for KV head h and the key at position j of a sample,
//     w[j] <- w[j] + sum over rows that see j, and the head's query heads, of 2^(c s_j - lse2),     s = q.k,  c = sm_scale log2 e,
// with the rows' finished log-sum-exp as given; the new tokens' own weights start from zero.
//
// The transpose of attention's scores: S^T = K Q^T puts a key on every tensor-memory lane and the rows along its columns, so a thread sums
// its own key's weights in a register -- no atomics, one order of summation whatever the scheduling.  Two key tiles (a PAIR
// of 128 keys each) stay in shared memory while the rows' tiles stream past both.  One exponential per key and row is the bound for
// chunks; for a few rows (a decode step) it is reading K once.
//
// Work units are (KV head, sample, key pair, row tile); a share is a run of them, as in chunk.h.  A pair's rows may be cut between shares:
// each then leaves 256 partial sums, which weights_merge_kernel adds in order.
//
// 20 warps: 0-15 sum (thread = key), a warpgroup for each of a pair's two key tiles and score buffers; 16 is the MMA issuer and owner of the
// tensor memory, 17 brings in the rows with their log-sum-exps, 18 and 19 the key tiles.  Two score buffers of 128 columns for each key tile.
// Every wait is bounded.
//
// 64 samples x 1 token over U[0,4096], 8 heads (268 MB of K): 55.5 us, 4.8 TB/s (one TMA warp for both key tiles 66); launch, schedule and
// merge are 10 of them.  17 to 127 rows take the products and sums of 128: 64 x 4 tokens, 64 / 8 heads, 78 us (64 x 16, 128 rows, 65).
// 2048 tokens over 8192, 32 / 8 heads, 604 M exponentials, a quarter by polynomial: 185 us (before NaN and large exponents were kept 180, to
// which the following compare); the special-function units'
// share is 100 us, the products 111 (two warpgroups 229 us; log-sum-exps loaded when needed 216; masked rows unrolled beside the whole ones,
// which is too much code, 205).  No polynomials 196, three eighths 181, half 208, a score buffer let go
// before its last 16 columns are summed 185; row tiles of 64 with four buffers 252, an issuer for each key
// tile 202, both against 203 at that time.
#include <algorithm>

#include "chunk.h"
#include "psa_internal.h"
#include "tensor_core.cuh"

namespace psa {
namespace {

constexpr int kWeightsThreads = 20 * 32, kPagesPerTile = 128 / kPageSize;
constexpr int kPairKeys = 256, kTileKeys = 128, kRowTile = 128, kFewRows = 16;
constexpr int kPairCost = 4, kRowCost = 2, kLeastShare = 8;
constexpr float kLog2e = 1.4426950408889634f;

// Consecutive pairs of one sample that the same row tiles see.
struct WeightsGroup {
    long long cum;
    int32_t q0, n;           // rows of q: first token, tokens
    int32_t pos0, len;
    int32_t list0, first_pair, pairs, first_tile;   // first_tile: the first row tile that sees them
};
static_assert(sizeof(WeightsGroup) == 40, "");
struct WeightsArgs {
    ChunkArgs c;             // q, samples, pages, status, shares
    WeightsGroup *groups;
    const float *lse, *weights;
    float *weights_out;
    float *partial;          // [2 * blocks, 256]
};

__device__ __forceinline__ int row_tiles(int n, int group) { return (n * group + kRowTile - 1) / kRowTile; }
__device__ __forceinline__ int pair_cost(const WeightsGroup &g, int group) { return kPairCost + kRowCost * (row_tiles(g.n, group) - g.first_tile); }

// ------------------------------------------------------------------------------------------------------------- schedule
struct Cut {
    int diagonal;            // first pair that some row does not see
    int pairs, tiles;
    long long cost;
};
__device__ __forceinline__ int first_tile_of(const ChunkSample &s, int pair, int group)   // first row tile that sees the pair's first key
{
    const long long i = max(0ll, (long long)pair * kPairKeys - (s.len - s.n));
    return int(i * group / kRowTile);
}
__device__ __forceinline__ Cut cut_of(const ChunkSample &s, int group)
{
    Cut c{};
    if (s.n == 0 || s.len == 0) return c;
    c.pairs = (s.len + kPairKeys - 1) / kPairKeys;
    c.tiles = row_tiles(s.n, group);
    c.diagonal = s.len < s.n ? 0 : min(c.pairs, (s.len - s.n) / kPairKeys + 1);
    c.cost = (long long)c.diagonal * (kPairCost + kRowCost * c.tiles);
    for (int p = c.diagonal; p < c.pairs; ++p) c.cost += kPairCost + kRowCost * (c.tiles - first_tile_of(s, p, group));
    return c;
}
__global__ void __launch_bounds__(kScheduleThreads)
weights_schedule_kernel(WeightsArgs w)
{
    __shared__ long long sum_cost[kScheduleThreads / 32];
    __shared__ int sum_groups[kScheduleThreads / 32];
    __shared__ long long cums[kKeptCums];
    __shared__ ChunkHeader made;
    grid_release();
    const ChunkArgs &a = w.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long carry_cost = 0;
    int carry_groups = 0;
    for (int s0 = 0; s0 < a.num_samples; s0 += kScheduleThreads) {
        const int s = s0 + int(threadIdx.x);
        ChunkSample cs{};
        Cut c{};
        if (s < a.num_samples) {
            cs = chunk_sample(a, s);
            c = cut_of(cs, a.group);
        }
        const int groups = (c.diagonal > 0) + c.pairs - c.diagonal;
        long long x = c.cost;
        int y = groups;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long ux = __shfl_up_sync(0xffffffffu, x, d);
            const int uy = __shfl_up_sync(0xffffffffu, y, d);
            if (lane >= d) { x += ux; y += uy; }
        }
        if (lane == 31) { sum_cost[warp] = x; sum_groups[warp] = y; }
        __syncthreads();
        long long at = carry_cost + x - c.cost;
        int to = carry_groups + y - groups;
        for (int k = 0; k < kScheduleThreads / 32; ++k) {
            if (k < warp) { at += sum_cost[k]; to += sum_groups[k]; }
            carry_cost += sum_cost[k];
            carry_groups += sum_groups[k];
        }
        __syncthreads();
        WeightsGroup g{};
        g.q0 = cs.q0; g.n = cs.n; g.pos0 = cs.len - cs.n; g.len = cs.len; g.list0 = cs.list0;
        auto put = [&](int first, int pairs, int first_tile) {
            g.cum = at; g.first_pair = first; g.pairs = pairs; g.first_tile = first_tile;
            if (to < a.max_groups) w.groups[to] = g;
            if (to < kKeptCums) cums[to] = at;
            ++to;
            at += (long long)pairs * pair_cost(g, a.group);
        };
        if (c.diagonal > 0) put(0, c.diagonal, 0);
        for (int p = c.diagonal; p < c.pairs; ++p) put(p, 1, first_tile_of(cs, p, a.group));
        // q_indptr that runs backwards: more rows than there are.  Counting on would pass 32 bits; a round adds 2^25 at most.
        if (carry_groups > a.max_groups) break;
    }
    if (threadIdx.x == 0) {
        if (carry_groups > a.max_groups) {
            raise(a.status, PSA_ERR_BOUNDS);
            carry_groups = 0;
            carry_cost = 0;
        }
        ChunkHeader h{};
        h.per_head = carry_cost;
        h.groups = carry_groups;
        h.blocks = int(max(1ll, min((long long)a.blocks, carry_cost * a.num_kv_heads / kLeastShare)));
        *a.header = made = h;
    }
    __syncthreads();
    if (made.groups > 0)
        write_starts(made, a.num_kv_heads, a.starts, [&](int i) { return made.groups <= kKeptCums ? cums[i] : w.groups[i].cum; });
}

// A place inside a group: the pair, and how many of its row tiles lie before it.
struct Place { int pair, rows; };
__device__ __forceinline__ Place place_of(const WeightsGroup &g, int group, long long y)   // y: cost from the group's begin
{
    const int cost = pair_cost(g, group);
    if (y <= 0) return {0, 0};
    if (y >= (long long)cost * g.pairs) return {g.pairs, 0};
    const int pair = int(y / cost), rest = int(y - (long long)pair * cost);
    const int rows = max(0, rest - kPairCost) / kRowCost;
    return {pair, rows};
}
struct WeightsPiece {
    WeightsGroup g;
    int head;
    Place from, to;          // [from, to)
};
struct WeightsWalk {
    const WeightsArgs &w;
    ChunkHeader h;
    long long x0 = 0, x1 = 0;
    int head, gi = 0;
    __device__ __forceinline__ WeightsWalk(const WeightsArgs &args, int block) : w(args), h(*args.c.header)
    {
        const ChunkStart s = args.c.starts[block];   // asked for together with the header
        head = w.c.num_kv_heads;
        if (block >= h.blocks || h.groups == 0) return;
        x0 = s.x0;
        x1 = s.x1;
        head = s.head;
        gi = s.group;
    }
    __device__ __forceinline__ bool next(WeightsPiece &p)
    {
        for (;;) {
            if (gi >= h.groups) {
                gi = 0;
                ++head;
            }
            if (head >= w.c.num_kv_heads) return false;
            p.g = w.groups[gi];
            const long long base = head * h.per_head + p.g.cum;
            if (base >= x1) {
                head = w.c.num_kv_heads;
                return false;
            }
            ++gi;
            p.head = head;
            p.from = place_of(p.g, w.c.group, x0 - base);
            p.to = place_of(p.g, w.c.group, x1 - base);
            if (p.from.pair < p.to.pair || p.from.rows < p.to.rows) return true;
        }
    }
};
// One key's finished sum to its cell: new tokens start from zero.
__device__ __forceinline__ void finish(const WeightsArgs &w, const WeightsGroup &g, int head, int pos, float sum)
{
    if (pos >= g.len) return;
    const int page = w.c.page_indices[g.list0 + pos / kPageSize];
    if (page < 0 || page >= w.c.num_pool_pages) return;   // reported by the load of its keys
    const size_t at = (size_t(page) * w.c.num_kv_heads + head) * kPageSize + pos % kPageSize;
    w.weights_out[at] = (pos < g.pos0 ? w.weights[at] : 0.f) + sum;
}
// The pairs of a piece, with the row tiles of each: pair, [r0, r1) counted from the row tiles that see it
template <class F>
__device__ __forceinline__ void each_pair(const WeightsPiece &p, int count, F f)
{
    for (int pair = p.from.pair; pair <= p.to.pair; ++pair) {
        const int r0 = pair == p.from.pair ? p.from.rows : 0, r1 = pair == p.to.pair ? p.to.rows : count;
        if (r0 < r1 && !f(pair, r0, r1)) return;
    }
}

// ------------------------------------------------------------------------------------------------------------- sums
template <int D>
struct WeightsSmem {
    static constexpr int kHalves = D / 64;
    static constexpr int kHalfBytes = 128 * 128;
    static constexpr int kTileBytes = kHalves * kHalfBytes;
    static constexpr int kKRing = D == 128 ? 4 : 8, kQRing = D == 128 ? 3 : 6;   // tiles; K comes in pairs
    static constexpr int kLseRing = 3;
    static constexpr int kBarKFull = 0, kBarKEmpty = kBarKFull + kKRing, kBarQFull = kBarKEmpty + kKRing, kBarQEmpty = kBarQFull + kQRing,
                         kBarLFull = kBarQEmpty + kQRing, kBarLEmpty = kBarLFull + kLseRing, kBarS = kBarLEmpty + kLseRing, kBarSFree = kBarS + 4,
                         kBarPassed = kBarSFree + 4, kBarTaken = kBarPassed + 2, kBarDrain = kBarTaken + 2, kNumBars = kBarDrain + 1;
    static constexpr int kTmemPtrOff = 8 * kNumBars, kAbortOff = kTmemPtrOff + 4;
    static constexpr int kPassOff = 512;                         // a sum for every key of a pair
    static constexpr int kLseOff = kPassOff + 1024;
    static constexpr int kQOff = 3 * 1024;
    static constexpr int kKOff = kQOff + kQRing * kTileBytes;
    static constexpr int kTotal = kKOff + kKRing * kTileBytes;
    static_assert(kAbortOff + 4 <= kPassOff && kLseOff + kLseRing * 512 <= kQOff && kTotal <= 227 * 1024, "shared memory plan");
};

template <int D>
__global__ void __launch_bounds__(kWeightsThreads, 1)
weights_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_few, const __grid_constant__ CUtensorMap map_k,
               const WeightsArgs w)
{
    using L = WeightsSmem<D>;
    constexpr int kMmaWarp = 16, kRowWarp = 17, kKeyWarp = 18, kKSteps = D / 16;
    const ChunkArgs &a = w.c;
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t sbase = smem_u32(smem);
    if (sbase & 1023u) {
        if (threadIdx.x == 0) raise(a.status, PSA_ERR_BOUNDS);
        return;
    }
    volatile uint32_t *tmem_ptr = reinterpret_cast<volatile uint32_t *>(smem + L::kTmemPtrOff);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + L::kAbortOff);
    auto bar = [&](int i) { return sbase + 8 * i; };
    auto warp_wait = [&](uint32_t b, uint32_t parity) {   // the whole warp goes on, or the whole warp gives up
        return __all_sync(0xffffffffu, mbar_wait(b, parity, abort_flag)) != 0;
    };
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int i = 0; i < L::kNumBars; ++i) {
            // a log-sum-exp slot is filled by 32 lanes and let go by 16 warps; a score buffer, a passed sum are four warps'
            const int count = i >= L::kBarLFull && i < L::kBarLEmpty ? 32 : i >= L::kBarLEmpty && i < L::kBarS ? 16 : i >= L::kBarSFree && i < L::kBarDrain ? 4 : 1;
            mbar_init(bar(i), count);
        }
        fence_barrier_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_ptr)), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_ptr;
    grid_wait();
    grid_release();

    WeightsWalk walk(w, blockIdx.x);
    WeightsPiece pc;
    bool ok = true;

    // The order of things, which every role follows: for each pair of a piece its K tiles, then its row tiles one by one.  A sample with
    // one row tile has it loaded once for all pairs of a piece.
    if (warp >= kKeyWarp) {
        const int t = warp - kKeyWarp;      // key tile of the pairs
        uint32_t ke = t;
        while (ok && walk.next(pc)) {
            const WeightsGroup &g = pc.g;
            each_pair(pc, row_tiles(g.n, a.group) - g.first_tile, [&](int pair, int, int) {
                const int key0 = (g.first_pair + pair) * kPairKeys + t * kTileKeys;
                const int pages = min(kPagesPerTile, max(0, (g.len - key0 + kPageSize - 1) / kPageSize));
                int id = 0;
                if (lane < pages) {
                    id = a.page_indices[g.list0 + key0 / kPageSize + lane];   // inside the list: the schedule saw to that
                    if (id < 0 || id >= a.num_pool_pages) {
                        raise(a.status, PSA_ERR_BOUNDS);
                        id = a.num_pool_pages;                                // outside the map: zeros
                    }
                }
                const int slot = ke % L::kKRing, use = ke / L::kKRing;
                ke += 2;
                if (use > 0 && !(ok = warp_wait(bar(L::kBarKEmpty + slot), (use - 1) & 1))) return false;
                const uint32_t full = bar(L::kBarKFull + slot), dst = sbase + L::kKOff + slot * L::kTileBytes;
                int ids[kPagesPerTile];
#pragma unroll
                for (int p = 0; p < kPagesPerTile; ++p) ids[p] = __shfl_sync(0xffffffffu, id, p);
                if (elect_one()) {
                    mbar_expect_tx(full, pages * kPageSize * D * 2);   // no page: the barrier completes at once
#pragma unroll
                    for (int p = 0; p < kPagesPerTile; ++p)
                        if (p < pages)
#pragma unroll
                            for (int h = 0; h < L::kHalves; ++h)
                                tma_load_4d(dst + h * L::kHalfBytes + p * kPageSize * 128, &map_k, full, h * 64, 0, pc.head, ids[p]);
                }
                __syncwarp();
                return true;
            });
        }
    } else if (warp == kRowWarp) {
        uint32_t qe = 0, le = 0;
        const int shift = __ffs(a.group) - 1;
        while (ok && walk.next(pc)) {
            const WeightsGroup &g = pc.g;
            const int tiles = row_tiles(g.n, a.group), count = tiles - g.first_tile;
            const bool few = g.n * a.group <= kFewRows;
            bool have_q = false;
            // four rows' log-sum-exps a lane; the next tile's are asked for before they are needed, or their way would be the pace of it all
            auto ask = [&](int tile, float (&x)[4]) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = tile * kRowTile + lane * 4 + i;
                    x[i] = r < g.n * a.group ? w.lse[size_t(g.q0 + (r >> shift)) * a.num_q_heads + pc.head * a.group + (r & (a.group - 1))] : -INFINITY;
                }
            };
            auto load_q = [&](int tile, const float (&x)[4]) {
                const int slot = qe % L::kQRing, use = qe / L::kQRing;
                if (use > 0 && !(ok = warp_wait(bar(L::kBarQEmpty + slot), (use - 1) & 1))) return;
                ++qe;
                if (elect_one()) {
                    const uint32_t full = bar(L::kBarQFull + slot), dst = sbase + L::kQOff + slot * L::kTileBytes;
                    mbar_expect_tx(full, (few ? kFewRows : kRowTile) * D * 2);
                    for (int h = 0; h < L::kHalves; ++h)
                        tma_load_4d(dst + h * L::kHalfBytes, few ? &map_few : &map_q, full, h * 64, 0, pc.head, g.q0 + tile * (kRowTile / a.group));
                }
                __syncwarp();
                const int ls = le % L::kLseRing, lu = le / L::kLseRing;
                if (lu > 0 && !(ok = warp_wait(bar(L::kBarLEmpty + ls), (lu - 1) & 1))) return;
                ++le;
                // minus the log-sum-exps, in log2; what does not exist or saw nothing gives no weight
                auto off = [](float v) { return v == -INFINITY ? -INFINITY : -v * kLog2e; };
                *reinterpret_cast<float4 *>(smem + L::kLseOff + ls * 512 + lane * 16) = make_float4(off(x[0]), off(x[1]), off(x[2]), off(x[3]));
                mbar_arrive(bar(L::kBarLFull + ls));
            };
            each_pair(pc, count, [&](int, int r0, int r1) {
                float x[2][4];
                if (tiles == 1) {
                    if (!have_q) {
                        ask(0, x[0]);
                        load_q(0, x[0]);
                    }
                    have_q = true;
                    return ok;
                }
                ask(g.first_tile + r0, x[0]);
                for (int r = r0; ok && r < r1; r += 2) {
                    if (r + 1 < r1) ask(g.first_tile + r + 1, x[1]);
                    load_q(g.first_tile + r, x[0]);
                    if (r + 2 < r1) ask(g.first_tile + r + 2, x[0]);
                    if (ok && r + 1 < r1) load_q(g.first_tile + r + 1, x[1]);
                }
                return ok;
            });
        }
    } else if (warp == kMmaWarp) {
        if (elect_one()) {
            constexpr uint64_t kHi = uint64_t(smem_desc_hi(1024)) << 32;
            const uint64_t q_desc = kHi | smem_desc_lo(sbase + L::kQOff, 16), k_desc = kHi | smem_desc_lo(sbase + L::kKOff, 16);
            constexpr uint32_t kIdesc = make_idesc(kRowTile, false), kIdescFew = make_idesc(kFewRows, false);
            uint32_t ke = 0, qe = 0, se = 0;
            while (ok && walk.next(pc)) {
                const int tiles = row_tiles(pc.g.n, a.group), count = tiles - pc.g.first_tile;
                const bool few = pc.g.n * a.group <= kFewRows;
                bool have_q = false;
                int q_slot = 0;
                each_pair(pc, count, [&](int pair, int r0, int r1) {
                    int k_slot[2];
                    for (int t = 0; t < 2; ++t, ++ke) {
                        k_slot[t] = ke % L::kKRing;
                        if (!(ok = mbar_wait(bar(L::kBarKFull + k_slot[t]), (ke / L::kKRing) & 1, abort_flag))) return false;
                    }
                    for (int r = r0; r < r1; ++r, ++se) {
                        if (tiles > 1 || !have_q) {
                            q_slot = qe % L::kQRing;
                            if (!(ok = mbar_wait(bar(L::kBarQFull + q_slot), (qe / L::kQRing) & 1, abort_flag))) return false;
                            ++qe;
                            have_q = true;
                        }
                        for (int t = 0; t < 2; ++t) {
                            const int b = 2 * t + int(se & 1);
                            if (se >= 2 && !(ok = mbar_wait(bar(L::kBarSFree + b), ((se >> 1) - 1) & 1, abort_flag))) return false;
                            tc_fence_after();
                            const uint64_t k = k_desc + uint32_t(k_slot[t]) * (L::kTileBytes >> 4), q = q_desc + uint32_t(q_slot) * (L::kTileBytes >> 4);
                            const uint32_t d = tmem_base + uint32_t(b) * 128, idesc = few ? kIdescFew : kIdesc;
#pragma unroll
                            for (int i = 0; i < kKSteps; ++i) {
                                const uint32_t off = ((i / 4) * L::kHalfBytes + (i % 4) * 32) >> 4;
                                if (i == 0) mma_ss<false>(d, k + off, q + off, idesc);
                                else mma_ss<true>(d, k + off, q + off, idesc);
                            }
                            tc_commit(bar(L::kBarS + b));
                            if (r + 1 == r1) tc_commit(bar(L::kBarKEmpty + k_slot[t]));
                        }
                        if (tiles > 1) tc_commit(bar(L::kBarQEmpty + q_slot));
                    }
                    return true;
                });
                if (ok && tiles == 1 && have_q) tc_commit(bar(L::kBarQEmpty + q_slot));
            }
        }
    } else {
        // Four warpgroups: key tile t of the pair, score buffer b.  Row tiles go to the buffers in turns, and with them to the warpgroups.
        const int t = (warp >> 2) & 1, b = warp >> 3, key = (warp & 3) * 32 + lane;
        const uint32_t s_addr = tmem_base + (uint32_t((warp & 3) * 32) << 16) + uint32_t(2 * t + b) * 128;
        float *const passed = reinterpret_cast<float *>(smem + L::kPassOff) + t * 128 + key;   // buffer 1's sum for buffer 0's warpgroup
        auto warp_arrive = [&](uint32_t x) {
            __syncwarp();
            if (lane == 0) mbar_arrive(x);
        };
        uint32_t se = 0, le = 0, passes = 0;
        while (ok && walk.next(pc)) {
            const WeightsGroup &g = pc.g;
            const int tiles = row_tiles(g.n, a.group), count = tiles - g.first_tile;
            const bool few = g.n * a.group <= kFewRows;
            bool have_q = false;
            int ls = 0;
            each_pair(pc, count, [&](int pair, int r0, int r1) {
                const int pos = (g.first_pair + pair) * kPairKeys + t * kTileKeys + key;
                const int first_row = max(0, min(pos - g.pos0, g.n)) * a.group, rows = g.n * a.group;   // below 2^28
                const bool alone = r1 - r0 == 1, first_mine = int(se & 1) == b;   // one row tile is one warpgroup's
                float total = 0.f;
                for (int r = r0; r < r1; ++r, ++se) {
                    if (tiles > 1 || !have_q) {
                        ls = le % L::kLseRing;
                        if (!(ok = warp_wait(bar(L::kBarLFull + ls), (le / L::kLseRing) & 1))) return false;
                        ++le;
                        have_q = true;
                    }
                    if (int(se & 1) == b) {
                        if (!(ok = warp_wait(bar(L::kBarS + 2 * t + b), (se >> 1) & 1))) return false;
                        tc_fence_after();
                        const float4 *off = reinterpret_cast<const float4 *>(smem + L::kLseOff + ls * 512);
                        const int row0 = (g.first_tile + r) * kRowTile;
                        const int lo = first_row - row0, hi = rows - row0;   // rows [lo, hi) give weight
                        const bool whole = __all_sync(0xffffffffu, lo <= 0 && hi >= 128);
                        float2 sum[2] = {{0.f, 0.f}, {0.f, 0.f}};
                        auto add = [&](const uint32_t (&s)[16], int c, bool masked) {
#pragma unroll
                            for (int i = 0; i < 16; i += 4) {
                                const float4 o = off[(c + i) / 4];
#pragma unroll
                                for (int k = 0; k < 4; k += 2) {
                                    float2 x = fma2(make_float2(__uint_as_float(s[i + k]), __uint_as_float(s[i + k + 1])), make_float2(a.scale_log2, a.scale_log2),
                                                    k == 0 ? make_float2(o.x, o.y) : make_float2(o.z, o.w));
                                    if (masked) {
                                        if (c + i + k < lo || c + i + k >= hi) x.x = -INFINITY;
                                        if (c + i + k + 1 < lo || c + i + k + 1 >= hi) x.y = -INFINITY;
                                    }
                                    // a quarter by polynomial: the special-function unit, an exponential a score, is the bound
                                    const bool poly = !masked && (i / 2 + k / 2) % 4 == 3;
                                    if (poly) x = make_float2(min_nan(x.x, kMostPolyExp2), min_nan(x.y, kMostPolyExp2));   // an lse may be smaller than it should
                                    const float2 e = poly ? poly_exp2_pair<5>(x) : make_float2(fast_exp2(x.x), fast_exp2(x.y));
                                    sum[k / 2] = add2(sum[k / 2], e);
                                }
                            }
                        };
                        uint32_t s[2][16];
                        if (whole) {
                            tmem_ld16(s_addr, s[0]);
                            tmem_wait_ld();
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                if (c < 7) tmem_ld16(s_addr + (c + 1) * 16, s[(c + 1) & 1]);
                                add(s[c & 1], c * 16, false);
                                tmem_wait_ld();
                            }
                        } else {
#pragma unroll 1
                            for (int c = 0; c < (few ? 16 : 128); c += 16) {
                                tmem_ld16(s_addr + c, s[0]);
                                tmem_wait_ld();
                                add(s[0], c, true);
                            }
                        }
                        tc_fence_before();
                        warp_arrive(bar(L::kBarSFree + 2 * t + b));
                        total += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                    }
                    if (tiles > 1) warp_arrive(bar(L::kBarLEmpty + ls));
                }
                if (alone ? !first_mine : b == 1) {
                    if (alone) return true;
                    if (passes > 0 && !(ok = warp_wait(bar(L::kBarTaken + t), (passes - 1) & 1))) return false;
                    ++passes;
                    *passed = total;
                    warp_arrive(bar(L::kBarPassed + t));
                    return true;
                }
                if (!alone) {
                    if (!(ok = warp_wait(bar(L::kBarPassed + t), passes++ & 1))) return false;
                    total += *passed;
                    warp_arrive(bar(L::kBarTaken + t));
                }
                const bool cut = r0 > 0 || r1 < count;
                if (cut) w.partial[size_t(2 * blockIdx.x + (r0 > 0 ? 0 : 1)) * kPairKeys + t * kTileKeys + key] = total;
                else finish(w, g, pc.head, pos, total);
                return true;
            });
            if (ok && tiles == 1 && have_q) warp_arrive(bar(L::kBarLEmpty + ls));
        }
        if (!ok) *abort_flag = 1;
    }

    // ---------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        if (threadIdx.x == 0) raise(a.status, PSA_ERR_TIMEOUT);
        // let copies that were already issued land before the block's shared memory is released
        if (warp >= kRowWarp && lane == 0) {
            const unsigned long long t0 = global_timer_ns();
            while (global_timer_ns() - t0 < 2000000ull) { }
        }
        if (warp == kMmaWarp && elect_one()) {   // products still queued
            tc_commit(bar(L::kBarDrain));
            const unsigned long long t0 = global_timer_ns();
            while (!mbar_try_wait(bar(L::kBarDrain), 0) && global_timer_ns() - t0 < 2000000ull) { }
        }
        __syncthreads();
    }
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem_base, 512);
    }
}

// ------------------------------------------------------------------------------------------------------------- merge
// Block `cut`: the pair that the end of share `cut` falls into, if that is the first cut inside it; a thread per key.
__global__ void __launch_bounds__(kPairKeys)
weights_merge_kernel(const WeightsArgs w)
{
    grid_wait();
    const ChunkHeader h = *w.c.header;
    const int cut = blockIdx.x;
    if (cut + 1 >= h.blocks || h.groups == 0) return;
    const ChunkStart *starts = w.c.starts, before = starts[cut], after = starts[cut + 1];
    const int head = after.head;
    const long long x = after.x0;
    if (head >= w.c.num_kv_heads) return;
    const WeightsGroup g = w.groups[after.group];
    const long long base = head * h.per_head + g.cum;
    const int count = row_tiles(g.n, w.c.group) - g.first_tile;
    const Place at = place_of(g, w.c.group, x - base);
    if (at.pair >= g.pairs || at.rows <= 0 || at.rows >= count) return;                 // nothing is cut here
    if (cut > 0) {
        const Place earlier = place_of(g, w.c.group, before.x0 - base);
        if (earlier.pair == at.pair && earlier.rows > 0) return;                          // an earlier cut's pair
    }
    float sum = 0.f;
    for (int b = cut; b < h.blocks; ++b) {
        const Place from = place_of(g, w.c.group, starts[b].x0 - base), to = place_of(g, w.c.group, starts[b].x1 - base);
        const int r0 = from.pair == at.pair ? from.rows : 0, r1 = to.pair == at.pair ? to.rows : count;
        if (r0 < r1) sum += w.partial[size_t(2 * b + (r0 > 0 ? 0 : 1)) * kPairKeys + threadIdx.x];
        if (r1 >= count) break;
    }
    finish(w, g, head, (g.first_pair + at.pair) * kPairKeys + int(threadIdx.x), sum);
}

template <int D>
cudaError_t launch(const WeightsArgs &w, const CUtensorMap *maps, cudaStream_t st)
{
    static PerDeviceOnce once;
    if (const int rc = once.ensure([] { return int(cudaFuncSetAttribute(weights_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, WeightsSmem<D>::kTotal)); }))
        return cudaError_t(rc);
    weights_schedule_kernel<<<1, kScheduleThreads, 0, st>>>(w);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) e = launch_dependent(weights_kernel<D>, dim3(w.c.blocks), kWeightsThreads, WeightsSmem<D>::kTotal, st, maps[0], maps[1], maps[2], w);
    if (e == cudaSuccess && w.c.blocks > 1) e = launch_dependent(weights_merge_kernel, dim3(w.c.blocks - 1), kPairKeys, 0, st, w);
    return e;
}

bool misaligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

size_t layout(WeightsArgs &w, void *scratch)
{
    ChunkArgs &a = w.c;
    a.max_groups = int(a.num_tokens / kPairKeys + 3 * int64_t(a.num_samples));
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off = (off + bytes + 255) / 256 * 256; return static_cast<unsigned char *>(scratch) + at; };
    a.header = reinterpret_cast<ChunkHeader *>(take(sizeof(ChunkHeader)));
    a.starts = reinterpret_cast<ChunkStart *>(take(sizeof(ChunkStart) * size_t(a.blocks)));
    w.groups = reinterpret_cast<WeightsGroup *>(take(sizeof(WeightsGroup) * size_t(a.max_groups)));
    w.partial = reinterpret_cast<float *>(take(4 * size_t(2 * a.blocks) * kPairKeys));
    return off;
}

}  // namespace
}  // namespace psa

extern "C" size_t psa_accumulate_weights_scratch_bytes(int64_t num_tokens, int32_t num_samples)
{
    if (num_tokens < 0 || num_samples < 0 || num_tokens > (1 << 24) || num_samples > (1 << 20)) return 0;
    psa::WeightsArgs w{};
    w.c.num_tokens = num_tokens; w.c.num_samples = num_samples; w.c.blocks = psa::kMostBlocks;
    return psa::layout(w, nullptr);
}

extern "C" psa_status_t psa_accumulate_weights(const void *q, const int64_t q_strides[2], const int32_t *q_indptr, int64_t num_tokens, int32_t num_samples,
                                               int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, float sm_scale, const float *lse,
                                               const void *k_pool, const int64_t pool_strides[3], int64_t num_pool_pages, const int32_t *page_indptr,
                                               const int32_t *page_indices, int64_t num_entries, const int32_t *kv_lens, const float *weights,
                                               float *weights_out, int32_t *status, void *scratch, size_t scratch_bytes, void *cuda_stream)
{
    using namespace psa;
    WeightsArgs w{};
    ChunkArgs &a = w.c;
    a.num_tokens = num_tokens; a.num_samples = num_samples; a.num_q_heads = num_q_heads; a.num_kv_heads = num_kv_heads;
    a.group = num_kv_heads > 0 ? num_q_heads / num_kv_heads : 0;
    a.num_pool_pages = int32_t(std::min<int64_t>(num_pool_pages, kMostChunkPages + 1)); a.num_entries = num_entries;
    a.q_indptr = q_indptr; a.kv_lens = kv_lens; a.page_indptr = page_indptr; a.page_indices = page_indices;
    a.status = status;
    a.scale_log2 = sm_scale * kLog2e;
    w.lse = lse; w.weights = weights; w.weights_out = weights_out;
    psa_status_t rc = chunk_check(a, q, q_strides, k_pool, pool_strides, head_dim);
    if (rc != PSA_OK) return rc;
    if (!(sm_scale > 0.f) || sm_scale > 1e30f) return set_last_error(PSA_ERR_INVALID_ARG, "sm_scale must be positive and finite");
    if (num_tokens == 0 || num_samples == 0) return PSA_OK;
    if (!lse || !weights || !weights_out) return set_last_error(PSA_ERR_INVALID_ARG, "null lse or weights");
    if (misaligned(lse, 4) || misaligned(weights, 4) || misaligned(weights_out, 4)) return set_last_error(PSA_ERR_INVALID_ARG, "lse and weights must be 4-byte aligned");
    if (num_pool_pages == 0) return set_last_error(PSA_ERR_INVALID_ARG, "the pool has no pages");
    if (!scratch || misaligned(scratch, 256) || scratch_bytes < psa_accumulate_weights_scratch_bytes(num_tokens, num_samples))
        return set_last_error(PSA_ERR_WORKSPACE, "scratch must be 256-byte aligned and hold psa_accumulate_weights_scratch_bytes");
    a.blocks = std::min(multiprocessors(), kMostBlocks);
    if (a.blocks <= 0) return set_last_error(PSA_ERR_CUDA, "no CUDA device");
    layout(w, scratch);
    CUtensorMap maps[3];
    rc = chunk_q_map(a, q, q_strides, head_dim, kRowTile, &maps[0]);
    if (rc == PSA_OK) rc = chunk_q_map(a, q, q_strides, head_dim, kFewRows, &maps[1]);
    if (rc == PSA_OK) rc = chunk_pool_map(a, k_pool, pool_strides, head_dim, &maps[2]);
    if (rc != PSA_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = head_dim == 128 ? launch<128>(w, maps, st) : launch<64>(w, maps, st);
    if (e != cudaSuccess) return set_last_error(PSA_ERR_CUDA, std::string("cached weights launch: ") + cudaGetErrorString(e));
    return PSA_OK;
}
