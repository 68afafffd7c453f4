// Attention of several new tokens per sample over a paged K/V cache (psa_attend_paged).
//
// Sample s holds S keys in its pages, the last n of them its new tokens; new token i stands at position S - n + i and sees the keys up to
// its own:   out = softmax_{j <= S - n + i}(sm_scale q.k_j) . v_j,   lse = ln sum exp.   Optionally an earlier partial result of the same
// rows over other keys (prior_out, prior_lse) is folded in:  L = ln(e^lse + e^prior_lse),  out = e^(lse - L) out + e^(prior_lse - L) prior_out.
//
// Three launches.  chunk_schedule_kernel cuts every sample's new tokens into GROUPS of up to 256 rows (256 / G tokens x G query heads) and
// writes their running costs (key tiles).  chunk_kernel is persistent: block i takes the i-th equal share of all (KV head, group, key
// tile) units, in order, so every SM has the same work whatever the lengths are, and a group is cut only where a share ends.  What is cut
// leaves partial results, two slots a block at most, which chunk_merge_kernel joins; groups that were not cut are finished in place.  A
// batch of few short samples has a block for every group instead, uncut; where the lists' length alone says so, it is one launch, and
// every block finds its group by itself.
//
// chunk_kernel, 12 warps: 0-3 and 4-7 softmax warpgroups (streams 0 and 1), 8 MMA issuer (one lane) and owner of the tensor memory, 9-11 TMA
// producers.  Key tiles of 128 keys arrive page by page (one TMA box of 16 tokens x 64 channels each) in a ring; S = Q K^T goes to
// tensor memory, a warpgroup (thread = row) turns it into P (bf16, over S), O += P V.  More than 128 rows: each stream has a row tile and
// both read every key tile, so a byte of K and V serves 256 rows.  Up to 128 rows: the streams take alternate key tiles of the one row tile,
// each with an accumulator of its own, joined at the end.  P is handed over in halves of 64 keys, so that the first half's products run
// under the second half's exponentials.  The reference maximum moves only when a half's exponents exceed it by 2^8 (which its
// sum tells, with the largest exponent that went to a polynomial: beyond 2^127 those are wrong; a three-way maximum a pair, +0.2 %, clamping each
// +1.3 % on the long case).
//
// What bounds it.  4096 new tokens over 12288 (64 / 8 heads of 128): 1.66 to 1.69 ms = 1.16 PFLOP/s, 0.83 of the measured sustained bf16
// rate; a key tile of two row tiles takes 1.9 us at the full clock, its products 1.5; the way from one score tile to the next (commit, softmax,
// hand-over, P V, Q K^T) is the rest.  64 x 4 tokens over U[0,4096] (549 MB): 113 us, 4.9 TB/s: the tiles come at 6.1 TB/s while they come, but a
// piece ends with 6.5 us of one warp's work (32 rows) that the ring's 160 KB cover half of, the first tile is 8 us on its way, the last shares
// end 10 us behind the median.  Eight short samples: 8.8 us (with a
// schedule and a merge 10.9), a chain of launch, lists, page ids, tiles, one unit and the epilogue.
// The instruction cache was the limit for long: masks and the careful way inlined in both halves cost the long case 7 %, the epilogue two
// thirds of its time.
// Tried and not kept (the long case, then the 64 x 4 tokens, against 1832 and 133 at that time): two warpgroups a stream, each half of the
// keys, with a shared reference 1875 / 139; the same with a score buffer for each half (64-key products) 2096 / 151; an issuer for each
// stream 2221 / 138; a watcher thread that folds the tiles' arrival into P's barrier 1860 / 134; K by TMA and V by cp.async 2236 / 182; all by
// cp.async 2411 / 166; prefetches into L2 6 tiles ahead 2204 / 162; one arrival a warp on the P barriers, polling without suspension: no
// change.  Against 1660 and 122: no polynomials 1720 / 121, an eighth 1682 / 121, three eighths 1728 / 131, the careful way as a function that is
// called (it spills) 1874 / 153, both halves in a rolled loop 1767 / 118.
//
// What does not exist is never used: products stop at the last page, rows of V behind the last key are zeroed in shared memory (they may
// hold anything), scores behind a row's last key become -inf.  Page ids outside the pool read as zeros (TMA bounds) and raise
// PSA_ERR_BOUNDS.  Every wait is bounded.
#include <cuda_bf16.h>

#include <algorithm>

#include "chunk.h"
#include "psa_internal.h"
#include "tensor_core.cuh"

namespace psa {
namespace {

constexpr int kTileKeys = 128;
constexpr int kRowTile = 128;
constexpr int kChunkThreads = 12 * 32;
constexpr int kPagesPerTile = kTileKeys / kPageSize;
constexpr float kThreshold = 8.f;                      // log2 units
constexpr float kHalfSumLimit = 64.f * 256.f * 1.01f;  // 64 exponentials of at most 2^8
constexpr uint32_t kPolyOf16 = 0x1111;                 // pairs of 32 scores whose exponentials are polynomials
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;


// ------------------------------------------------------------------------------------------------------------- schedule
// Running sums over the samples by one block, a thread a sample; a sample of many groups is its warp's.
__global__ void __launch_bounds__(kScheduleThreads)
chunk_schedule_kernel(ChunkArgs a)
{
    constexpr int kWarps = kScheduleThreads / 32, kAlone = 4;   // groups that a thread goes through by itself
    __shared__ long long sum_cost[kWarps];
    __shared__ int sum_groups[kWarps], longest;
    __shared__ long long cums[kKeptCums];
    __shared__ ChunkHeader made;
    grid_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per_group = kGroupRows / a.group;   // tokens
    long long carry_cost = 0;
    int carry_groups = 0, my_longest = 0;
    if (threadIdx.x == 0) longest = 0;
    for (int s0 = 0; s0 < a.num_samples; s0 += kScheduleThreads) {
        const int s = s0 + int(threadIdx.x);
        ChunkSample c{};
        if (s < a.num_samples) c = chunk_sample(a, s);
        const int groups = (c.n + per_group - 1) / per_group;
        if (c.n > 0) my_longest = max(my_longest, chunk_tiles(c.len));
        // put(place, group) for every group of the lane's sample, places from `to` on, costs from `at` on; returns the cost of all
        auto each = [&](long long at, int to, auto put) {
            const long long begin = at;
            if (groups <= kAlone)
                for (int i = 0; i < groups; ++i) {
                    ChunkGroup g = chunk_group(c, i, per_group);
                    g.cum = at;
                    put(to + i, g);
                    at += chunk_cost(g, a.group);
                }
            for (unsigned many = __ballot_sync(0xffffffffu, groups > kAlone); many; many &= many - 1) {
                const int owner = __ffs(many) - 1;
                const ChunkSample o{__shfl_sync(0xffffffffu, c.q0, owner), __shfl_sync(0xffffffffu, c.n, owner), __shfl_sync(0xffffffffu, c.len, owner),
                                    __shfl_sync(0xffffffffu, c.list0, owner)};
                const int its = __shfl_sync(0xffffffffu, groups, owner), first = __shfl_sync(0xffffffffu, to, owner);
                long long before = __shfl_sync(0xffffffffu, at, owner);
                for (int i0 = 0; i0 < its; i0 += 32) {
                    ChunkGroup g = chunk_group(o, min(i0 + lane, its - 1), per_group);
                    const long long cost = i0 + lane < its ? chunk_cost(g, a.group) : 0;
                    long long x = cost;
#pragma unroll
                    for (int d = 1; d < 32; d <<= 1) {
                        const long long u = __shfl_up_sync(0xffffffffu, x, d);
                        if (lane >= d) x += u;
                    }
                    g.cum = before + x - cost;
                    if (i0 + lane < its) put(first + i0 + lane, g);
                    before += __shfl_sync(0xffffffffu, x, 31);
                }
                if (lane == owner) at = before;
            }
            return at - begin;
        };
        const long long cost = each(0, 0, [](int, const ChunkGroup &) {});
        // exclusive scans over the block
        long long x = cost;
        int y = groups;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long ux = __shfl_up_sync(0xffffffffu, x, d);
            const int uy = __shfl_up_sync(0xffffffffu, y, d);
            if (lane >= d) { x += ux; y += uy; }
        }
        if (lane == 31) { sum_cost[warp] = x; sum_groups[warp] = y; }
        __syncthreads();
        long long at = carry_cost + x - cost;
        int to = carry_groups + y - groups;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) { at += sum_cost[w]; to += sum_groups[w]; }
            carry_cost += sum_cost[w];
            carry_groups += sum_groups[w];
        }
        __syncthreads();
        each(at, to, [&](int place, const ChunkGroup &g) {
            if (place < a.max_groups) a.groups[place] = g;
            if (place < kKeptCums) cums[place] = g.cum;
        });
        // q_indptr that runs backwards: more rows than there are.  Counting on would pass 32 bits; a round adds 2^27 at most.
        if (carry_groups > a.max_groups) break;
    }
    if (my_longest) atomicMax(&longest, my_longest);
    __syncthreads();
    if (threadIdx.x == 0) {
        if (carry_groups > a.max_groups) {
            raise(a.status, PSA_ERR_BOUNDS);
            carry_groups = 0;
            carry_cost = 0;
        }
        const long long total = carry_cost * a.num_kv_heads;
        ChunkHeader h{};
        h.per_head = carry_cost;
        h.groups = carry_groups;
        h.blocks = int(max(1ll, min((long long)a.blocks, total / kLeastCost)));
        // a block for every group, uncut, where there are enough of them and none is long: no results to join
        if ((long long)carry_groups * a.num_kv_heads <= a.blocks && longest <= kWholeTiles) {
            h.whole = 1;
            h.blocks = max(1, carry_groups * a.num_kv_heads);
        }
        *a.header = made = h;
    }
    __syncthreads();
    if (made.groups > 0 && !made.whole)
        write_starts(made, a.num_kv_heads, a.starts, [&](int i) { return made.groups <= kKeptCums ? cums[i] : a.groups[i].cum; });
}

// ------------------------------------------------------------------------------------------------------------- attention
template <int D>
struct ChunkSmem {
    static constexpr int kHalves = D / 64;
    static constexpr int kHalfBytes = 128 * 128;                 // 128 rows x 64 bf16
    static constexpr int kTileBytes = kHalves * kHalfBytes;      // a tile of Q, K or V
    static constexpr int kRing = D == 128 ? 5 : 10;
    static constexpr int kBarQFull = 0, kBarQEmpty = 2, kBarFull = 4, kBarEmpty = kBarFull + kRing, kBarS = kBarEmpty + kRing, kBarP = kBarS + 2,
                         kBarHalf = kBarP + 4, kBarDone = kBarHalf + 2, kBarMet = kBarDone + 2, kBarDrain = kBarMet + 1, kNumBars = kBarDrain + 1;
    static constexpr int kTmemPtrOff = 8 * kNumBars, kAbortOff = kTmemPtrOff + 4;
    static constexpr int kShareOff = 512;
    static constexpr int kExchangeOff = 1024;                    // (m, l) of both streams' rows
    static constexpr int kQOff = 3 * 1024;
    static constexpr int kRingOff = kQOff + 2 * kTileBytes;
    static constexpr int kTotal = kRingOff + kRing * kTileBytes;
    static_assert(kAbortOff + 4 <= kShareOff && kTotal <= 227 * 1024, "shared memory plan");
};

// Element m of the order in which K and V tiles travel: alternating with two row tiles, K two tiles ahead with one.
struct Travel { int tile; bool is_v; };
__device__ __forceinline__ Travel travel(int m, int n, bool two)
{
    if (two || n == 1) return {m >> 1, (m & 1) != 0};
    if (m < 2) return {m, false};
    const int r = m - 2, both = 2 * (n - 2);
    if (r < both) return {(r >> 1) + (r & 1) * 2, (r & 1) == 0};
    return {n - 2 + r - both, true};
}
// place of V tile i in that order
__device__ __forceinline__ int v_place(int i, int n, bool two) { return two ? 2 * i + 1 : i < n - 1 ? 2 * i + 2 : 2 * n - 1; }

// 8 columns of one row to global memory
__device__ __forceinline__ void store_row(const ChunkArgs &a, size_t at, const float (&v)[8])
{
    if (a.out_f32) {
        float *to = static_cast<float *>(a.out) + at;
        *reinterpret_cast<float4 *>(to) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(to + 4) = make_float4(v[4], v[5], v[6], v[7]);
        return;
    }
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
        w[k] = reinterpret_cast<const uint32_t &>(p);
    }
    *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) + at) = make_uint4(w[0], w[1], w[2], w[3]);
}
// Lane i of four has row i, v[j] its columns 8 j ..: afterwards v[j] is row j's columns 8 i ...
__device__ __forceinline__ void quad_transpose(float (&v)[4][8], int quad)
{
#pragma unroll
    for (int bit = 1; bit < 4; bit <<= 1)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (!(j & bit))
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const bool upper = quad & bit;
                    const float got = __shfl_xor_sync(0xffffffffu, upper ? v[j][k] : v[j | bit][k], bit);
                    v[j][k] = upper ? got : v[j][k];
                    v[j | bit][k] = upper ? v[j | bit][k] : got;
                }
}
// 8 columns of the earlier result added: in bf16, the usual type, they have been asked for before
__device__ __forceinline__ void add_earlier(const ChunkArgs &a, const uint4 &asked, size_t at, float w, float (&v)[8])
{
    if (w == 0.f) return;                          // not 0 x NaN
    if (a.prior_f32) {
        const float4 *from = reinterpret_cast<const float4 *>(static_cast<const float *>(a.prior_out) + at);
        const float4 x = from[0], y = from[1];
        v[0] = fmaf(w, x.x, v[0]); v[1] = fmaf(w, x.y, v[1]); v[2] = fmaf(w, x.z, v[2]); v[3] = fmaf(w, x.w, v[3]);
        v[4] = fmaf(w, y.x, v[4]); v[5] = fmaf(w, y.y, v[5]); v[6] = fmaf(w, y.z, v[6]); v[7] = fmaf(w, y.w, v[7]);
    } else {
        const uint32_t u[4] = {asked.x, asked.y, asked.z, asked.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = fmaf(w, __uint_as_float(u[k] << 16), v[2 * k]);
            v[2 * k + 1] = fmaf(w, __uint_as_float(u[k] & 0xffff0000u), v[2 * k + 1]);
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kChunkThreads, 1)
chunk_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
             const ChunkArgs a)
{
    using L = ChunkSmem<D>;
    constexpr int kMmaWarp = 8, kProducerWarp = 9, kProducers = 3;
    static_assert(kProducers <= L::kRing, "a slot's use before the last is over when a warp waits for it");
    constexpr int kKSteps = D / 16;
    constexpr uint32_t kIdescQK = make_idesc(kTileKeys, false), kIdescPV = make_idesc(D, true);
    constexpr uint32_t kColO = 256;                    // S[t] at 128 t, O[t] at 256 + t D

    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t sbase = smem_u32(smem);
    if (sbase & 1023u) {   // swizzled tiles need a 1024-byte aligned base; refuse to run rather than read garbage
        if (threadIdx.x == 0) raise(a.status, PSA_ERR_BOUNDS);
        return;
    }
    volatile uint32_t *tmem_ptr = reinterpret_cast<volatile uint32_t *>(smem + L::kTmemPtrOff);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + L::kAbortOff);
    auto bar = [&](int i) { return sbase + 8 * i; };
    auto bar_p = [&](int t, int h) { return bar(L::kBarP + 2 * t + h); };
    auto warp_wait = [&](uint32_t b, uint32_t parity) {   // the whole warp goes on, or the whole warp gives up
        return __all_sync(0xffffffffu, mbar_wait(b, parity, abort_flag)) != 0;
    };
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int i = 0; i < L::kNumBars; ++i) mbar_init(bar(i), i >= L::kBarP && i < L::kBarHalf ? 128 : i == L::kBarMet ? 256 : 1);
        fence_barrier_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_ptr)), 512);
        tmem_relinquish();
    }
    if (warp == kProducerWarp && elect_one()) { prefetch_tensormap(&map_q); prefetch_tensormap(&map_k); prefetch_tensormap(&map_v); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_ptr;
    grid_wait();
    grid_release();

    ChunkShare *share = reinterpret_cast<ChunkShare *>(smem + L::kShareOff);
    if (warp == 0) {
        const ChunkShare s = chunk_share(a, blockIdx.x, lane);
        if (lane == 0) *share = s;
    }
    __syncthreads();
    ChunkWalk walk(a, *share);
    ChunkPiece pc;

    if (warp >= kProducerWarp) {
        // ------------------------------------------------------------ TMA producers, which take the elements of the ring in turns: a box is one
        // page's 2 KB, and a single warp issues them too slowly for HBM.  Elements are freed in the order in which they are filled, so the use
        // of a slot before its last one was over when the warp's previous element, kProducers earlier, was let in: a parity cannot be that of
        // an older phase, although a warp sees only its own elements.
        const int part = warp - kProducerWarp;
        uint32_t e = 0, q_uses[2] = {0, 0}, q_sel = 0;
        bool ok = true;
        while (ok && walk.next(pc)) {
            const int n = pc.t1 - pc.t0;
            if (n == 0) continue;
            const bool two = pc.g.n_tok * a.group > kRowTile;
            auto page_of = [&](int m) {   // this lane's page of element m
                const int page = (pc.t0 + travel(m, n, two).tile) * kPagesPerTile + lane;
                if (m >= 2 * n || lane >= kPagesPerTile || page * kPageSize >= pc.g.keys) return 0;
                const int id = a.page_indices[pc.g.list0 + page];   // inside the list: the schedule saw to that
                if (id >= 0 && id < a.num_pool_pages) return id;
                raise(a.status, PSA_ERR_BOUNDS);
                return a.num_pool_pages;                              // outside the map: zeros
            };
            // Q is the first warp's, always: the others may be ahead of it by more pieces than there are buffers.  It goes before the warp's first
            // element where two buffers take turns, and behind it where the buffers are waited for until the last piece's scores are made.
            bool q_due = part == 0;
            auto load_q = [&]() {
                for (int t = 0; ok && q_due && t < (two ? 2 : 1); ++t) {
                    const int b = two ? t : int(q_sel);
                    if (q_uses[b] > 0 && !(ok = warp_wait(bar(L::kBarQEmpty + b), (q_uses[b] - 1) & 1))) break;
                    if (elect_one()) {
                        mbar_expect_tx(bar(L::kBarQFull + b), L::kTileBytes);
                        for (int h = 0; h < L::kHalves; ++h)
                            tma_load_4d(sbase + L::kQOff + b * L::kTileBytes + h * L::kHalfBytes, &map_q, bar(L::kBarQFull + b), h * 64, 0, pc.head,
                                        pc.g.q0 + t * (kRowTile / a.group));
                    }
                    __syncwarp();
                }
                q_due = false;
            };
            if (!two) load_q();
            int m = (part + kProducers - int(e % kProducers)) % kProducers;
            int id = page_of(m);
            for (; ok && m < 2 * n; m += kProducers) {
                const Travel tr = travel(m, n, two);
                const int next = page_of(m + kProducers);
                const int slot = (e + m) % L::kRing, use = (e + m) / L::kRing;
                if (use > 0 && !(ok = warp_wait(bar(L::kBarEmpty + slot), (use - 1) & 1))) break;
                const int left = pc.g.keys - (pc.t0 + tr.tile) * kTileKeys;
                const int pages = min(kPagesPerTile, (left + kPageSize - 1) / kPageSize);
                const uint32_t full = bar(L::kBarFull + slot), dst = sbase + L::kRingOff + slot * L::kTileBytes;
                int ids[kPagesPerTile];
#pragma unroll
                for (int p = 0; p < kPagesPerTile; ++p) ids[p] = __shfl_sync(0xffffffffu, id, p);
                if (elect_one()) {
                    mbar_expect_tx(full, pages * kPageSize * D * 2);
                    const CUtensorMap *map = tr.is_v ? &map_v : &map_k;
#pragma unroll
                    for (int p = 0; p < kPagesPerTile; ++p)
                        if (p < pages)
#pragma unroll
                            for (int h = 0; h < L::kHalves; ++h)
                                tma_load_4d(dst + h * L::kHalfBytes + p * kPageSize * 128, map, full, h * 64, 0, pc.head, ids[p]);
                }
                __syncwarp();
                id = next;
                load_q();
            }
            load_q();   // a piece may have no element of this warp's
            e += 2 * n;
            if (two) {
                ++q_uses[0];
                ++q_uses[1];
            } else {
                ++q_uses[q_sel];
                q_sel ^= 1;
            }
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------------------ MMA issuer.  Unit u of a piece: stream u & 1, key tile u / 2 (two row
        // tiles) or u (one).  QK^T runs two units ahead of PV.
        if (elect_one()) {
            constexpr uint64_t kHi = uint64_t(smem_desc_hi(1024)) << 32;
            const uint64_t q_desc = kHi | smem_desc_lo(sbase + L::kQOff, 16);
            const uint64_t k_desc = kHi | smem_desc_lo(sbase + L::kRingOff, 16);               // K-major
            const uint64_t v_desc = kHi | smem_desc_lo(sbase + L::kRingOff, L::kHalfBytes);    // MN-major, halves kHalfBytes apart
            uint32_t e = 0, q_uses[2] = {0, 0}, q_sel = 0, uses[2] = {0, 0};
            bool ok = true;
            auto landed = [&]() {   // waits for the next element; its slot
                const int slot = e % L::kRing;
                ok = mbar_wait(bar(L::kBarFull + slot), (e / L::kRing) & 1, abort_flag);
                ++e;
                return slot;
            };
            while (ok && walk.next(pc)) {
                const int n = pc.t1 - pc.t0;
                if (n == 0) continue;
                const bool two = pc.g.n_tok * a.group > kRowTile;
                const int units = two ? 2 * n : n;
                const int qb = two ? 0 : int(q_sel);
                for (int t = 0; ok && t < (two ? 2 : 1); ++t) {
                    ok = mbar_wait(bar(L::kBarQFull + qb + t), q_uses[qb + t] & 1, abort_flag);
                    ++q_uses[qb + t];
                }
                if (!two) q_sel ^= 1;
                int k_slot = 0, v_slot = 0;
                auto issue_qk = [&](int u) {
                    const int t = u & 1;
                    if (!two || t == 0) k_slot = landed();
                    if (!ok) return;
                    tc_fence_after();
                    const uint64_t q = q_desc + uint32_t(two ? t : qb) * (L::kTileBytes >> 4);
                    const uint64_t k = k_desc + uint32_t(k_slot) * (L::kTileBytes >> 4);
                    const uint32_t d = tmem_base + uint32_t(t) * 128;
#pragma unroll
                    for (int i = 0; i < kKSteps; ++i) {
                        const uint32_t off = ((i / 4) * L::kHalfBytes + (i % 4) * 32) >> 4;
                        if (i == 0) mma_ss<false>(d, q + off, k + off, kIdescQK);
                        else mma_ss<true>(d, q + off, k + off, kIdescQK);
                    }
                    tc_commit(bar(L::kBarS + t));
                    if (!two || t == 1) tc_commit(bar(L::kBarEmpty + k_slot));
                    if (two ? u + 2 >= units : u + 1 == units) tc_commit(bar(L::kBarQEmpty + (two ? t : qb)));
                };
                for (int u = 0; ok && u < 2 && u < units; ++u) issue_qk(u);
                for (int u = 0; ok && u < units; ++u) {
                    const int t = u & 1, tile = pc.t0 + (two ? u >> 1 : u);
                    if (!two || t == 0) v_slot = landed();
                    if (!ok) break;
                    const int steps = min(kPagesPerTile, (pc.g.keys - tile * kTileKeys + kPageSize - 1) / kPageSize);   // of 16 keys
                    const uint64_t v = v_desc + uint32_t(v_slot) * (L::kTileBytes >> 4);
                    const uint32_t p = tmem_base + uint32_t(t) * 128, o = tmem_base + kColO + t * D;
                    const bool first = u < 2;
                    if (!(ok = mbar_wait(bar_p(t, 0), uses[t] & 1, abort_flag))) break;
                    tc_fence_after();
                    mma_ts_p(o, p, v, kIdescPV, first ? 0u : 1u);
#pragma unroll
                    for (int i = 1; i < 4; ++i)
                        if (i < steps) mma_ts(o, p + i * 8, v + ((i * 2048) >> 4), kIdescPV);
                    tc_commit(bar(L::kBarHalf + t));
                    if (!(ok = mbar_wait(bar_p(t, 1), uses[t] & 1, abort_flag))) break;
                    tc_fence_after();
#pragma unroll
                    for (int i = 4; i < 8; ++i)
                        if (i < steps) mma_ts(o, p + i * 8, v + ((i * 2048) >> 4), kIdescPV);
                    if (!two || t == 1) tc_commit(bar(L::kBarEmpty + v_slot));
                    ++uses[t];
                    if (u + 2 < units) issue_qk(u + 2);   // over P of this unit: ordered behind the products just issued
                    else tc_commit(bar(L::kBarDone + t));
                }
            }
        }
    } else {
        // ------------------------------------------------------------ softmax warpgroups and epilogue
        const int t = warp >> 2;
        const int row = (warp & 3) * 32 + lane;        // TMEM lane
        const uint32_t lane_addr = uint32_t((warp & 3) * 32) << 16;
        const uint32_t s_addr = tmem_base + lane_addr + uint32_t(t) * 128;
        const uint32_t o_base = tmem_base + lane_addr + kColO;
        float *exchange = reinterpret_cast<float *>(smem + L::kExchangeOff);   // [stream][m, l][row]
        const int shift = __ffs(a.group) - 1;
        uint32_t e = 0, uses = 0, met = 0, done[2] = {0, 0};
        bool ok = true;
        while (ok && walk.next(pc)) {
            const int n = pc.t1 - pc.t0;
            const int rows = pc.g.n_tok * a.group;
            const bool two = rows > kRowTile;
            const int in_group = (two ? t * kRowTile : 0) + row;
            const bool mine = in_group < rows;
            const bool active = __any_sync(0xffffffffu, mine);
            const int token = in_group >> shift;
            const int sees = mine ? max(0, min(pc.g.keys, pc.g.pos0 + token + 1)) : pc.g.keys;   // keys the row sees
            const int my_uses = two ? n : (n - t + 1) / 2;
            const int tiles = (pc.g.keys + kTileKeys - 1) / kTileKeys;
            float m_ref = -INFINITY, l_sum = 0.f;

            for (int j = 0; j < my_uses; ++j, ++uses) {
                const int local = two ? j : 2 * j + t, tile = pc.t0 + local;
                if (!(ok = warp_wait(bar(L::kBarS + t), uses & 1))) break;
                tc_fence_after();
                const int keys_here = pc.g.keys - tile * kTileKeys;
                if (tile == tiles - 1 && keys_here % kPageSize) {
                    // rows of V behind the last key may hold anything, and 0 x NaN is NaN: zero what the products will read of them
                    const uint32_t at = e + v_place(local, n, two);
                    const int slot = at % L::kRing;
                    if (!(ok = warp_wait(bar(L::kBarFull + slot), (at / L::kRing) & 1))) break;
                    const int chunks = (kPageSize - keys_here % kPageSize) * 8;
                    for (int i = row; i < chunks * L::kHalves; i += 128) {
                        const int h = i / chunks, c = i % chunks;
                        *reinterpret_cast<uint4 *>(smem + L::kRingOff + slot * L::kTileBytes + h * L::kHalfBytes + keys_here * 128 + c * 16) = make_uint4(0, 0, 0, 0);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                if (!active) {   // no row of this warp exists: whatever stands in these lanes of P stays in their lanes of O
                    mbar_arrive(bar_p(t, 0));
                    mbar_arrive(bar_p(t, 1));
                    continue;
                }
                const int valid = sees - tile * kTileKeys;
                // A half is 64 scores, 32 at a time; S of the half stays in tensor memory until all of it is known to be in range, P in p.
                uint32_t p[32];
                auto mask = [&](int v, uint32_t (&r)[32]) {
                    if (__any_sync(0xffffffffu, v < 32)) {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i >= v) r[i] = 0xff800000u;
                    }
                };
                // 32 scores -> 16 words of bf16 P; adds them to `sum`.  A sum tells of exponents out of range, but for those of polynomials, which
                // go to `most`.
                auto exponentials = [&](const uint32_t (&r)[32], uint32_t *to, float2 (&sum)[2], float &most) {
                    const float off = m_ref == -INFINITY ? 0.f : -m_ref;
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        const float2 x = fma2(make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), make_float2(a.scale_log2, a.scale_log2), make_float2(off, off));
                        // part of them by polynomial: it relieves the special-function unit, which has an exponential a score
                        const bool poly = kPolyOf16 >> (i / 2) & 1;
                        if (poly) most = max3(most, x.x, x.y);
                        const float2 e = poly ? poly_exp2_pair<4>(x) : make_float2(fast_exp2(x.x), fast_exp2(x.y));
                        sum[i / 2 & 1] = add2(sum[i / 2 & 1], e);
                        // P is rounded to nearest: its products need 16 bits; truncating it takes as long
                        const __nv_bfloat162 both = __floats2bfloat162_rn(e.x, e.y);
                        to[i / 2] = reinterpret_cast<const uint32_t &>(both);
                    }
                };
                auto hand_over = [&](int h, float total) {
                    tmem_st32(s_addr + h * 32, p);
                    l_sum += total;
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(bar_p(t, h));
                };
                // The usual way: every score is seen and in range.  Else false, and nothing has happened.
                auto plain = [&](int h) -> bool {
                    uint32_t r[2][32];
                    float2 sum[2] = {{0.f, 0.f}, {0.f, 0.f}};
                    float most = 0.f;
                    tmem_ld32(s_addr + h * 64, r[0]);
                    tmem_wait_ld();
                    tmem_ld32(s_addr + h * 64 + 32, r[1]);
                    exponentials(r[0], p, sum, most);
                    tmem_wait_ld();
                    exponentials(r[1], p + 16, sum, most);
                    const float total = (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                    if (__any_sync(0xffffffffu, !(total <= kHalfSumLimit) || most > kMostPolyExp2)) return false;
                    hand_over(h, total);
                    return true;
                };
                // Scores to be masked, or a reference to be moved.  There is one copy of this code, and it goes on to the second half: what
                // the loop's code takes of the instruction cache is its speed.
                auto careful = [&](int h) -> bool {
                    const int v = valid - 64 * h;
                    uint32_t r[2][32];
                    tmem_ld32(s_addr + h * 64, r[0]);
                    tmem_ld32(s_addr + h * 64 + 32, r[1]);
                    tmem_wait_ld();
                    mask(v, r[0]);
                    mask(v - 32, r[1]);
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int i = 0; i < 64; ++i) mx[i & 3] = fmaxf(mx[i & 3], __uint_as_float(r[i / 32][i % 32]));
                    const float top = a.scale_log2 * fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                    const bool need = top > m_ref + kThreshold;
                    if (__any_sync(0xffffffffu, need)) {
                        const float alpha = need ? fast_exp2(m_ref - top) : 1.f;
                        if (j > 0 || h == 1) {
                            // O[t] is at rest: S of this unit was made behind the products before it; the first half's products of
                            // this very unit are waited for
                            if (h == 1) {
                                if (!warp_wait(bar(L::kBarHalf + t), uses & 1)) return false;
                                tc_fence_after();
                            }
#pragma unroll 1
                            for (int c = 0; c < D / 32; ++c) {
                                tmem_ld32(o_base + t * D + c * 32, p);
                                tmem_wait_ld();
#pragma unroll
                                for (int i = 0; i < 32; ++i) p[i] = __float_as_uint(__uint_as_float(p[i]) * alpha);
                                tmem_st32(o_base + t * D + c * 32, p);
                            }
                            tmem_wait_st();
                        }
                        l_sum *= alpha;
                        if (need) m_ref = top;
                    }
                    float2 sum[2] = {{0.f, 0.f}, {0.f, 0.f}};
                    float most = 0.f;                  // of exponents that are in range
                    exponentials(r[0], p, sum, most);
                    exponentials(r[1], p + 16, sum, most);
                    hand_over(h, (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y));
                    return true;
                };
                int h = 0;
                if (__all_sync(0xffffffffu, m_ref > -INFINITY && valid >= kTileKeys) && plain(0)) h = plain(1) ? 2 : 1;
#pragma unroll 1
                for (; ok && h < 2; ++h) ok = careful(h);
                if (!ok) break;
            }
            if (!ok) break;
            e += 2 * n;

            // ---- epilogue
            auto out_row = [&](int r) { return size_t(pc.g.q0 + (r >> shift)) * a.num_q_heads + pc.head * a.group + (r & (a.group - 1)); };
            const size_t part_row = size_t(pc.slot) * a.slot_rows + in_group;
            // this warpgroup's columns: all of its own row tile, or half of the shared one
            const int c0 = two ? 0 : t * (D / 2), c1 = two ? D : (t + 1) * (D / 2);
            // To memory four lanes go side by side: each has 8 of 32 columns of their four rows.  The earlier result comes that way, while the
            // last products are waited for.
            const int quad = lane & 3, quad_row = in_group - quad;
            const bool joins = !pc.split && a.prior_lse;
            const float prior2 = joins && mine ? a.prior_lse[out_row(in_group)] * kLog2e : -INFINITY;
            size_t at[4];
            uint4 earlier[4];
            auto ask = [&](int c) {
                if (!a.prior_f32)
#pragma unroll
                    for (int k = 0; k < 4; ++k) earlier[k] = *reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(a.prior_out) + at[k] + c);
            };
            if (active && !pc.split) {
#pragma unroll
                for (int k = 0; k < 4; ++k) at[k] = out_row(min(quad_row + k, rows - 1)) * D + quad * 8;
                if (joins) ask(c0);
            }
            const int streams = n == 0 ? 0 : two || n > 1 ? 2 : 1;
            if (two || n == 0) {
                if (n > 0) {
                    if (!(ok = warp_wait(bar(L::kBarDone + t), done[t]++ & 1))) break;
                    done[1 - t]++;
                }
            } else {
                for (int i = 0; ok && i < streams; ++i) ok = warp_wait(bar(L::kBarDone + i), done[i]++ & 1);
                if (!ok) break;
            }
            tc_fence_after();
            float share[2] = {0.f, 0.f};   // of each stream's accumulator in the result
            float lse2;
            if (two || n == 0) {
                share[t] = l_sum == 0.f ? 0.f : 1.f / l_sum;
                lse2 = l_sum == 0.f ? -INFINITY : m_ref + log2f(l_sum);
            } else {
                exchange[t * 256 + row] = m_ref;
                exchange[t * 256 + 128 + row] = l_sum;
                mbar_arrive(bar(L::kBarMet));
                if (!(ok = warp_wait(bar(L::kBarMet), met++ & 1))) break;
                const float m[2] = {exchange[row], exchange[256 + row]}, l[2] = {exchange[128 + row], exchange[384 + row]};
                const float top = fmaxf(m[0], m[1]);
                const float w0 = l[0] == 0.f ? 0.f : fast_exp2(m[0] - top), w1 = l[1] == 0.f ? 0.f : fast_exp2(m[1] - top);
                const float total = w0 * l[0] + w1 * l[1];
                share[0] = total == 0.f ? 0.f : w0 / total;
                share[1] = total == 0.f ? 0.f : w1 / total;
                lse2 = total == 0.f ? -INFINITY : top + log2f(total);
            }
            float from_prior = 0.f;
            if (joins) {
                const Joined jn = join(lse2, prior2);
                share[0] *= jn.first;
                share[1] *= jn.first;
                from_prior = jn.second;
                lse2 = jn.lse2;
            }
            float from[4];                         // the quad's rows'
#pragma unroll
            for (int k = 0; k < 4; ++k) from[k] = __shfl_sync(0xffffffffu, from_prior, (lane & ~3) + k);
#pragma unroll 1
            for (int c = c0; active && c < c1; c += 32) {
                __syncwarp();
                float v[4][8];
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i / 8][i % 8] = 0.f;
#pragma unroll 1
                for (int i = 0; i < 2; ++i) {
                    if (n == 0 || (two ? i != t : i >= streams)) continue;
                    uint32_t o[32];
                    tmem_ld32(o_base + i * D + c, o);
                    tmem_wait_ld();
                    const float w = i ? share[1] : share[0];
                    if (w != 0.f)
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[k / 8][k % 8] = fmaf(__uint_as_float(o[k]), w, v[k / 8][k % 8]);
                }
                if (pc.split) {
                    // four columns of all rows stand together: whole lines, although a thread has a row
                    if (mine)
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            reinterpret_cast<float4 *>(a.partial_o)[(size_t(pc.slot) * (D / 4) + c / 4 + i) * a.slot_rows + in_group] =
                                make_float4(v[i / 2][i % 2 * 4], v[i / 2][i % 2 * 4 + 1], v[i / 2][i % 2 * 4 + 2], v[i / 2][i % 2 * 4 + 3]);
                    continue;
                }
                quad_transpose(v, quad);
                if (joins) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) add_earlier(a, earlier[k], at[k] + c, from[k], v[k]);
                    if (c + 32 < c1) ask(c + 32);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (quad_row + k < rows) store_row(a, at[k] + c, v[k]);
            }
            tc_fence_before();
            if (!two) {
                // each warpgroup has read both accumulators, the exchanged sums and prior_lse (which lse may be): none of them is written
                // before both are done
                mbar_arrive(bar(L::kBarMet));
                if (!(ok = warp_wait(bar(L::kBarMet), met++ & 1))) break;
            }
            if (mine && (two || t == 0)) {
                if (pc.split) a.partial_lse[part_row] = lse2;
                else a.lse[out_row(in_group)] = lse2 * kLn2;
            }
        }
        if (!ok) *abort_flag = 1;
    }

    // ---------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        if (threadIdx.x == 0) raise(a.status, PSA_ERR_TIMEOUT);
        // let copies that were already issued land before the block's shared memory is released
        if (warp >= kProducerWarp && lane == 0) {
            const unsigned long long t0 = global_timer_ns();
            while (global_timer_ns() - t0 < 2000000ull) { }
        }
        // products queued before the issuing thread gave up may still run: one more commit completes when all of them have retired
        if (warp == kMmaWarp && elect_one()) {
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
// Block (cut, slice): the group that the end of share `cut` falls into, if that is the first cut inside it; a warp for 8 rows.
constexpr int kMergeWarps = 4;
template <int D>
__global__ void __launch_bounds__(kMergeWarps * 32)
chunk_merge_kernel(const ChunkArgs a)
{
    __shared__ int slots[2 * kMostBlocks];
    grid_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const ChunkHeader h = *a.header;
    const int cut = blockIdx.x;                 // between blocks cut and cut + 1
    if (cut + 1 >= h.blocks || h.groups == 0 || h.whole) return;
    const ChunkStart before = a.starts[cut], after = a.starts[cut + 1];
    const int head = after.head;
    const long long x = after.x0;
    if (head >= a.num_kv_heads) return;
    const ChunkGroup g = a.groups[after.group];
    const long long base = head * h.per_head + g.cum;
    const int tiles = chunk_tiles(g.keys), t_cut = tile_at(g, a.group, base, x);
    if (t_cut <= 0 || t_cut >= tiles) return;                                              // nothing is cut here
    if (cut > 0 && tile_at(g, a.group, base, before.x0) > 0) return;   // an earlier cut's group
    // pieces: blocks cut, cut + 1, ... until the group ends
    __shared__ int last;
    if (threadIdx.x == 0) last = h.blocks - 1;
    __syncthreads();
    for (int b = cut + threadIdx.x; b < h.blocks; b += blockDim.x) {
        const int t0 = tile_at(g, a.group, base, a.starts[b].x0), t1 = tile_at(g, a.group, base, a.starts[b].x1);
        slots[b - cut] = t1 > t0 ? 2 * b + (t0 > 0 ? 0 : 1) : -1;
        if (t1 >= tiles) atomicMin(&last, b);
    }
    __syncthreads();
    const int pieces = last - cut + 1;
    const int rows = g.n_tok * a.group, shift = __ffs(a.group) - 1;
    // a lane's part: a row, and four columns of every 16
    constexpr int kSteps = D / 16;
    const int quarter = lane >> 3;
    for (int r0 = (blockIdx.y * kMergeWarps + warp) * 8; r0 < rows; r0 += gridDim.y * kMergeWarps * 8) {
        const bool mine = r0 + (lane & 7) < rows;
        const int r = min(r0 + (lane & 7), rows - 1);
        const size_t row = size_t(g.q0 + (r >> shift)) * a.num_q_heads + head * a.group + (r & (a.group - 1));
        const float prior2 = a.prior_lse ? a.prior_lse[row] * kLog2e : -INFINITY;
        // the earlier result's columns are asked for at once, like the pieces' log-sum-exps and columns: there is little else to wait for
        uint4 earlier[kSteps];
        if (a.prior_lse)
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                const size_t at = row * D + (j * 4 + quarter) * 4;
                if (a.prior_f32) {
                    earlier[j] = *reinterpret_cast<const uint4 *>(static_cast<const float *>(a.prior_out) + at);
                } else {
                    const uint2 u = *reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(a.prior_out) + at);
                    earlier[j] = make_uint4(u.x << 16, u.x & 0xffff0000u, u.y << 16, u.y & 0xffff0000u);
                }
            }
        float top = -INFINITY, sum = 0.f;
        float acc[kSteps][4];
#pragma unroll
        for (int j = 0; j < kSteps; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
        constexpr int kAbreast = 4;
        for (int i0 = 0; i0 < pieces; i0 += kAbreast) {
            float lse2[kAbreast];
            int slot[kAbreast];
            float next = top;
#pragma unroll
            for (int i = 0; i < kAbreast; ++i) {
                slot[i] = i0 + i < pieces ? slots[i0 + i] : -1;
                lse2[i] = slot[i] >= 0 ? a.partial_lse[size_t(slot[i]) * a.slot_rows + r] : -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < kAbreast; ++i) next = fmaxf(next, lse2[i]);
            const float keep = top == -INFINITY ? 0.f : exp2f(top - next);
            top = next;
            sum *= keep;
#pragma unroll
            for (int j = 0; j < kSteps; ++j) { acc[j][0] *= keep; acc[j][1] *= keep; acc[j][2] *= keep; acc[j][3] *= keep; }
#pragma unroll
            for (int i = 0; i < kAbreast; ++i) {
                if (slot[i] < 0) continue;           // the same for all rows
                const float4 *from = reinterpret_cast<const float4 *>(a.partial_o) + (size_t(slot[i]) * (D / 4) + quarter) * a.slot_rows + r;
                float4 o[kSteps];
#pragma unroll
                for (int j = 0; j < kSteps; ++j) o[j] = from[size_t(4 * j) * a.slot_rows];
                const float w = lse2[i] == -INFINITY ? 0.f : exp2f(lse2[i] - top);
                if (w == 0.f) continue;
                sum += w;
#pragma unroll
                for (int j = 0; j < kSteps; ++j) {
                    acc[j][0] = fmaf(w, o[j].x, acc[j][0]); acc[j][1] = fmaf(w, o[j].y, acc[j][1]);
                    acc[j][2] = fmaf(w, o[j].z, acc[j][2]); acc[j][3] = fmaf(w, o[j].w, acc[j][3]);
                }
            }
        }
        float lse2 = sum == 0.f ? -INFINITY : top + log2f(sum);
        float share = sum == 0.f ? 0.f : 1.f / sum, from_prior = 0.f;
        if (a.prior_lse) {
            const Joined jn = join(lse2, prior2);
            share *= jn.first;
            from_prior = jn.second;
            lse2 = jn.lse2;
        }
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            const size_t at = row * D + (j * 4 + quarter) * 4;
            float4 v = make_float4(acc[j][0] * share, acc[j][1] * share, acc[j][2] * share, acc[j][3] * share);
            if (from_prior != 0.f)
                v = make_float4(fmaf(from_prior, __uint_as_float(earlier[j].x), v.x), fmaf(from_prior, __uint_as_float(earlier[j].y), v.y),
                                fmaf(from_prior, __uint_as_float(earlier[j].z), v.z), fmaf(from_prior, __uint_as_float(earlier[j].w), v.w));
            if (!mine) continue;
            if (a.out_f32) {
                *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) = v;
            } else {
                const __nv_bfloat162 x = __floats2bfloat162_rn(v.x, v.y), y = __floats2bfloat162_rn(v.z, v.w);
                *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(a.out) + at) = make_uint2(reinterpret_cast<const uint32_t &>(x), reinterpret_cast<const uint32_t &>(y));
            }
        }
        __syncwarp();   // lse may be prior_lse: every lane has read it
        if (quarter == 0 && mine) a.lse[row] = lse2 * kLn2;
    }
}

template <int D>
cudaError_t launch(const ChunkArgs &a, const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t st)
{
    static PerDeviceOnce once;
    if (const int rc = once.ensure([] { return int(cudaFuncSetAttribute(chunk_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, ChunkSmem<D>::kTotal)); }))
        return cudaError_t(rc);
    if (a.direct) {
        chunk_kernel<D><<<a.direct * a.num_kv_heads, kChunkThreads, ChunkSmem<D>::kTotal, st>>>(mq, mk, mv, a);
        return cudaGetLastError();
    }
    chunk_schedule_kernel<<<1, kScheduleThreads, 0, st>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) e = launch_dependent(chunk_kernel<D>, dim3(a.blocks), kChunkThreads, ChunkSmem<D>::kTotal, st, mq, mk, mv, a);
    if (e == cudaSuccess && a.blocks > 1) e = launch_dependent(chunk_merge_kernel<D>, dim3(a.blocks - 1, (a.slot_rows + 8 * kMergeWarps - 1) / (8 * kMergeWarps)), kMergeWarps * 32, 0, st, a);
    return e;
}

bool misaligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

}  // namespace

size_t chunk_layout(ChunkArgs &a, void *scratch, int head_dim)
{
    const int per_group = kGroupRows / a.group;
    a.max_groups = int(a.num_tokens / per_group + a.num_samples);
    a.slot_rows = int(std::min<int64_t>(kGroupRows, a.num_tokens * a.group));
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off = (off + bytes + 255) / 256 * 256; return static_cast<unsigned char *>(scratch) + at; };
    a.header = reinterpret_cast<ChunkHeader *>(take(sizeof(ChunkHeader)));
    a.starts = reinterpret_cast<ChunkStart *>(take(sizeof(ChunkStart) * size_t(a.blocks)));
    a.groups = reinterpret_cast<ChunkGroup *>(take(sizeof(ChunkGroup) * size_t(a.max_groups)));
    if (head_dim > 0) {
        a.partial_lse = reinterpret_cast<float *>(take(4 * size_t(2 * a.blocks) * a.slot_rows));
        a.partial_o = reinterpret_cast<float *>(take(4 * size_t(2 * a.blocks) * a.slot_rows * head_dim));
    }
    return off;
}

psa_status_t chunk_check(const ChunkArgs &a, const void *q, const int64_t q_strides[2], const void *pool, const int64_t pool_strides[3], int head_dim)
{
    if (a.num_tokens < 0 || a.num_samples < 0 || a.num_pool_pages < 0 || a.num_entries < 0 || a.num_kv_heads <= 0 || a.num_q_heads <= 0)
        return set_last_error(PSA_ERR_INVALID_ARG, "negative sizes or no heads");
    if (head_dim != 64 && head_dim != 128) return set_last_error(PSA_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
    if (a.num_q_heads % a.num_kv_heads || (a.group != 1 && a.group != 2 && a.group != 4 && a.group != 8))
        return set_last_error(PSA_ERR_UNSUPPORTED, "num_q_heads / num_kv_heads must be 1, 2, 4 or 8");
    if (a.num_q_heads > 65536) return set_last_error(PSA_ERR_UNSUPPORTED, "at most 2^16 query heads");
    if (a.num_samples > (1 << 20)) return set_last_error(PSA_ERR_UNSUPPORTED, "at most 2^20 samples per call");
    if (a.num_tokens > (1 << 24)) return set_last_error(PSA_ERR_UNSUPPORTED, "at most 2^24 new tokens per call");
    if (a.num_pool_pages > kMostChunkPages || a.num_entries > kMostChunkEntries)
        return set_last_error(PSA_ERR_UNSUPPORTED, "at most 2^27 pages and 2^31 - 256 list entries");
    if (misaligned(a.status, 4)) return set_last_error(PSA_ERR_INVALID_ARG, "the status word must be 4-byte aligned");
    if (a.num_tokens == 0 || a.num_samples == 0) return PSA_OK;
    if (!q || !q_strides || !pool_strides || !a.page_indptr || !a.kv_lens || (a.num_entries > 0 && !a.page_indices) || (a.num_pool_pages > 0 && !pool) ||
        (!a.q_indptr && a.num_samples != a.num_tokens))
        return set_last_error(PSA_ERR_INVALID_ARG, "null paged attention argument");
    if (misaligned(q, 16) || misaligned(pool, 16)) return set_last_error(PSA_ERR_INVALID_ARG, "q and the pools must be 16-byte aligned");
    for (int i = 0; i < 3; ++i) {
        if (pool_strides[i] <= 0 || pool_strides[i] % 8 || pool_strides[i] >= (int64_t(1) << 38))
            return set_last_error(PSA_ERR_INVALID_ARG, "pool strides must be positive multiples of 8 elements below 2^38");
        if (i < 2 && (q_strides[i] <= 0 || q_strides[i] % 8 || q_strides[i] >= (int64_t(1) << 38)))
            return set_last_error(PSA_ERR_INVALID_ARG, "q strides must be positive multiples of 8 elements below 2^38");
    }
    return PSA_OK;
}

psa_status_t chunk_q_map(const ChunkArgs &a, const void *q, const int64_t q_strides[2], int head_dim, int rows, CUtensorMap *map)
{
    // Q as (d, g, kv head, token): a box of (64, G, 1, rows / G) is one 64-wide half of a row tile, g fastest
    const cuuint64_t dims[4] = {cuuint64_t(head_dim), cuuint64_t(a.group), cuuint64_t(a.num_kv_heads), cuuint64_t(a.num_tokens)};
    const cuuint64_t strides[3] = {cuuint64_t(q_strides[1]) * 2, cuuint64_t(q_strides[1]) * a.group * 2, cuuint64_t(q_strides[0]) * 2};
    const cuuint32_t box[4] = {64, cuuint32_t(a.group), 1, cuuint32_t(rows / a.group)};
    std::string err;
    EncodeFn fn = get_encode_fn(&err);
    if (!fn || !encode(fn, map, q, 4, dims, strides, box, &err)) return set_last_error(PSA_ERR_CUDA, err);
    return PSA_OK;
}

psa_status_t chunk_pool_map(const ChunkArgs &a, const void *pool, const int64_t pool_strides[3], int head_dim, CUtensorMap *map)
{
    // a pool as (d, slot, kv head, page): a box is one 64-wide half of a page
    const cuuint64_t dims[4] = {cuuint64_t(head_dim), kPageSize, cuuint64_t(a.num_kv_heads), cuuint64_t(a.num_pool_pages)};
    const cuuint64_t strides[3] = {cuuint64_t(pool_strides[2]) * 2, cuuint64_t(pool_strides[1]) * 2, cuuint64_t(pool_strides[0]) * 2};
    const cuuint32_t box[4] = {64, kPageSize, 1, 1};
    std::string err;
    EncodeFn fn = get_encode_fn(&err);
    if (!fn || !encode(fn, map, pool, 4, dims, strides, box, &err)) return set_last_error(PSA_ERR_CUDA, err);
    return PSA_OK;
}

int multiprocessors()
{
    static std::atomic<int> known[PerDeviceOnce::kMaxDevices];
    int dev = 0;
    if (PerDeviceOnce::device_ordinal(&dev)) return 0;
    if (dev < 0 || dev >= PerDeviceOnce::kMaxDevices) return 0;
    int n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
        known[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

}  // namespace psa

extern "C" size_t psa_attend_paged_scratch_bytes(int64_t num_tokens, int32_t num_samples, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim)
{
    if (num_tokens < 0 || num_samples < 0 || num_kv_heads <= 0 || num_q_heads < num_kv_heads || num_tokens > (1 << 24) || head_dim < 0 || head_dim > 1024) return 0;
    psa::ChunkArgs a{};
    a.num_tokens = num_tokens; a.num_samples = num_samples;
    a.group = std::min(8, num_q_heads / num_kv_heads);
    a.blocks = psa::kMostBlocks;
    return psa::chunk_layout(a, nullptr, head_dim);
}

extern "C" psa_status_t psa_attend_paged(const void *q, const int64_t q_strides[2], const int32_t *q_indptr, int64_t num_tokens, int32_t num_samples,
                                         int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, float sm_scale, const void *k_pool,
                                         const void *v_pool, const int64_t pool_strides[3], int64_t num_pool_pages, const int32_t *page_indptr,
                                         const int32_t *page_indices, int64_t num_entries, const int32_t *kv_lens, const void *prior_out,
                                         int32_t prior_dtype, const float *prior_lse, void *out, int32_t out_dtype, float *lse, int32_t *status,
                                         void *scratch, size_t scratch_bytes, void *cuda_stream)
{
    using namespace psa;
    ChunkArgs a{};
    a.num_tokens = num_tokens; a.num_samples = num_samples; a.num_q_heads = num_q_heads; a.num_kv_heads = num_kv_heads;
    a.group = num_kv_heads > 0 ? num_q_heads / num_kv_heads : 0;
    a.num_pool_pages = int32_t(std::min<int64_t>(num_pool_pages, kMostChunkPages + 1)); a.num_entries = num_entries;
    a.q_indptr = q_indptr; a.kv_lens = kv_lens; a.page_indptr = page_indptr; a.page_indices = page_indices;
    a.status = status;
    a.scale_log2 = sm_scale * kLog2e;
    a.prior_out = prior_out; a.prior_lse = prior_lse; a.prior_f32 = prior_dtype == PSA_OUT_F32;
    a.out = out; a.lse = lse; a.out_f32 = out_dtype == PSA_OUT_F32;
    psa_status_t rc = chunk_check(a, q, q_strides, k_pool, pool_strides, head_dim);
    if (rc != PSA_OK) return rc;
    if ((out_dtype != PSA_OUT_BF16 && out_dtype != PSA_OUT_F32) || (prior_out && prior_dtype != PSA_OUT_BF16 && prior_dtype != PSA_OUT_F32))
        return set_last_error(PSA_ERR_UNSUPPORTED, "out and prior_out must be bf16 or f32");
    if (!(sm_scale > 0.f) || sm_scale > 1e30f) return set_last_error(PSA_ERR_INVALID_ARG, "sm_scale must be positive and finite");
    if ((prior_out == nullptr) != (prior_lse == nullptr)) return set_last_error(PSA_ERR_INVALID_ARG, "prior_out and prior_lse go together");
    if (num_tokens == 0 || num_samples == 0) return PSA_OK;
    if ((num_pool_pages > 0 && !v_pool) || !out || !lse) return set_last_error(PSA_ERR_INVALID_ARG, "null paged attention argument");
    if (misaligned(v_pool, 16) || misaligned(out, 16) || misaligned(prior_out, 16) || misaligned(lse, 4) || misaligned(prior_lse, 4))
        return set_last_error(PSA_ERR_INVALID_ARG, "pools, out and prior_out must be 16-byte aligned, lse 4-byte aligned");
    if (prior_out == out && prior_out && prior_dtype != out_dtype) return set_last_error(PSA_ERR_INVALID_ARG, "prior_out may be out only with the same type");
    if (num_pool_pages == 0) return set_last_error(PSA_ERR_INVALID_ARG, "the pool has no pages");
    if (!scratch || misaligned(scratch, 256) ||
        scratch_bytes < psa_attend_paged_scratch_bytes(num_tokens, num_samples, num_q_heads, num_kv_heads, head_dim))
        return set_last_error(PSA_ERR_WORKSPACE, "scratch must be 256-byte aligned and hold psa_attend_paged_scratch_bytes");
    a.blocks = std::min(multiprocessors(), kMostBlocks);
    if (a.blocks <= 0) return set_last_error(PSA_ERR_CUDA, "no CUDA device");
    chunk_layout(a, scratch, head_dim);
    // a few short lists: every group is a block's, which finds it by itself
    if (num_entries * kPageSize <= kDirectTiles * kTileKeys && int64_t(a.max_groups) * num_kv_heads <= a.blocks) a.direct = a.max_groups;
    CUtensorMap maps[3];
    rc = chunk_q_map(a, q, q_strides, head_dim, kRowTile, &maps[0]);
    if (rc == PSA_OK) rc = chunk_pool_map(a, k_pool, pool_strides, head_dim, &maps[1]);
    if (rc == PSA_OK) rc = chunk_pool_map(a, v_pool, pool_strides, head_dim, &maps[2]);
    if (rc != PSA_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = head_dim == 128 ? launch<128>(a, maps[0], maps[1], maps[2], st) : launch<64>(a, maps[0], maps[1], maps[2], st);
    if (e != cudaSuccess) return set_last_error(PSA_ERR_CUDA, std::string("paged attention launch: ") + cudaGetErrorString(e));
    return PSA_OK;
}
