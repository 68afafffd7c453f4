// What the kernels over chunks of new tokens share (attention: chunk_sm100.cu; weights of cached tokens: weights_sm100.cu): a call's
// arguments, the checks of a sample's entries, and how the work is cut into equal shares.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "psa_internal.h"

namespace psa {

constexpr int kScheduleThreads = 256;
constexpr int kGroupRows = 256;                              // rows of a group: two row tiles of 128
constexpr int kKeptCums = 1024;                              // groups whose costs the schedule keeps in shared memory
constexpr int kMostBlocks = 160;                             // persistent blocks, at most one per SM
constexpr int kMostTokens = 1 << 30;                         // of one sample
constexpr int64_t kMostChunkPages = int64_t(1) << 27, kMostChunkEntries = (int64_t(1) << 31) - 256;

struct ChunkHeader {
    long long per_head;    // cost of one KV head's groups
    int32_t groups, blocks;
    int32_t whole, pad;    // a block for every group, uncut
};
// Up to kGroupRows rows of one sample: consecutive new tokens and the group's query heads, head fastest.
struct ChunkGroup {
    long long cum;         // cost of the groups before it
    int32_t q0, n_tok;     // rows of q
    int32_t pos0, keys;    // position of the first token (negative: it sees nothing), keys that the last one sees
    int32_t list0, pad;    // where the sample's pages start in page_indices
};
static_assert(sizeof(ChunkGroup) == 32, "");
// A block's share [x0, x1) of the cost of all heads, and the head and group that it starts in.
struct ChunkStart {
    long long x0, x1;
    int32_t head, group;
};

struct ChunkArgs {
    int64_t num_tokens, num_entries;
    int32_t num_samples, num_q_heads, num_kv_heads, group, num_pool_pages;
    const int32_t *q_indptr, *kv_lens, *page_indptr, *page_indices;
    int32_t *status;
    float scale_log2;
    const void *prior_out;
    const float *prior_lse;
    void *out;
    float *lse;
    bool prior_f32, out_f32;
    // scratch
    int32_t blocks, max_groups, slot_rows;
    int32_t direct;        // not 0: no schedule, a block for each of so many groups a head
    ChunkHeader *header;
    ChunkStart *starts;    // [blocks]
    ChunkGroup *groups;
    float *partial_lse, *partial_o;    // [2 * blocks, slot_rows] log2, [2 * blocks, D / 4, slot_rows, 4] normalised
};

#ifdef __CUDACC__
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
// A launch whose set-up may overlap the tail of the one before; its kernel calls grid_wait before it touches memory.
template <class K, class... A>
cudaError_t launch_dependent(K kernel, dim3 grid, int threads, int smem, cudaStream_t st, A... args)
{
    cudaLaunchConfig_t lc{};
    lc.gridDim = grid;
    lc.blockDim = dim3(threads);
    lc.dynamicSmemBytes = smem;
    lc.stream = st;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = &attr;
    lc.numAttrs = 1;
    return cudaLaunchKernelEx(&lc, kernel, args...);
}

__device__ __forceinline__ void raise(int32_t *status, int code)
{
    if (status) atomicCAS(status, 0, code);
}

// A sample's entries, made safe: n new tokens from row q0 on, len keys in pages from list0 on.  What does not hold together raises
// PSA_ERR_BOUNDS; a sample whose keys do not fit its list counts as empty.
struct ChunkSample { int q0, n, len, list0; };
__device__ __forceinline__ ChunkSample chunk_sample(const ChunkArgs &a, int s)
{
    const int tokens = int(a.num_tokens);
    const int r0 = a.q_indptr ? a.q_indptr[s] : s, r1 = a.q_indptr ? a.q_indptr[s + 1] : s + 1;
    const int l0 = a.page_indptr[s], l1 = a.page_indptr[s + 1];
    int len = a.kv_lens[s];
    const int b0 = min(max(r0, 0), tokens), b1 = min(max(r1, b0), tokens);
    if (b0 != r0 || b1 != r1) raise(a.status, PSA_ERR_BOUNDS);
    if (b1 == b0) return {b0, 0, 0, 0};
    if (l0 < 0 || l1 < l0 || l1 > a.num_entries || len < 0 || len > kMostTokens || len > (long long)(l1 - l0) * kPageSize) {
        raise(a.status, PSA_ERR_BOUNDS);
        len = 0;
    }
    return {b0, b1 - b0, len, l0};
}
__device__ __forceinline__ ChunkGroup chunk_group(const ChunkSample &c, int i, int per_group)
{
    ChunkGroup g{};
    const int first = i * per_group;
    g.q0 = c.q0 + first;
    g.n_tok = min(per_group, c.n - first);
    g.pos0 = c.len - c.n + first;
    g.keys = max(0, g.pos0 + g.n_tok);
    g.list0 = c.list0;
    return g;
}

// Cost of a piece in quarters of a key tile of two row tiles (1.9 us).  A single row tile's key tile, 1.05 to 1.15 us, costs two, and a piece
// 14: the first tiles' way and the epilogue, 4.4 us with two row tiles, 6.5 with one, where other pieces' loads fill the gap less.  (14, 2)
// against (8, 3), (10, 2), (12, 3), (18, 2) and (18, 3): 116 us for 64 x 4 tokens over U[0,4096] against 122, 118, 119, 117 and 118; 4096 tokens over
// 12288 do not mind.
constexpr int kPieceCost = 14;
constexpr int kLeastCost = 8;     // a share is not made smaller than this: 4 x 4 tokens over 2000 21 us, with 14 23, with 20 26
constexpr int kWholeTiles = 6;    // key tiles of samples that are not worth cutting
// ... nor a schedule and a merge, where all lists together are known to be no longer: one sample of 2 / 6 / 10 / 12 tiles 10.2 / 14.0 / 17.5 /
// 19.3 us, cut and joined 12.1 / 15.9 / 18.0 / 18.5
constexpr int kDirectTiles = 10;
__device__ __forceinline__ int chunk_tiles(int keys) { return (keys + 127) >> 7; }
__device__ __forceinline__ int chunk_weight(const ChunkGroup &g, int group) { return g.n_tok * group > 128 ? 4 : 2; }
__device__ __forceinline__ long long chunk_cost(const ChunkGroup &g, int group)
{
    return kPieceCost + (long long)chunk_tiles(g.keys) * chunk_weight(g, group);
}
// shares of [0, total): share i of n starts here
__device__ __forceinline__ long long share_begin(long long total, int i, int n) { return total / n * i + total % n * i / n; }
// the first key tile of a group at `base` that belongs behind x
__device__ __forceinline__ int tile_at(const ChunkGroup &g, int group, long long base, long long x)
{
    const long long y = x - base - kPieceCost;
    if (y <= 0) return 0;
    const int tiles = chunk_tiles(g.keys), w = chunk_weight(g, group);
    return y >= (long long)tiles * w ? tiles : int(uint32_t(y) / uint32_t(w));
}
// Every block's share, by the block that made the groups; `cum(i)` is the cost before group i.
template <class Cum>
__device__ __forceinline__ void write_starts(const ChunkHeader &h, int heads, ChunkStart *starts, Cum cum)
{
    const long long total = h.per_head * heads;
    for (int b = threadIdx.x; b < h.blocks; b += blockDim.x) {
        ChunkStart s;
        s.x0 = share_begin(total, b, h.blocks);
        s.x1 = share_begin(total, b + 1, h.blocks);
        s.head = int(s.x0 / h.per_head);
        const long long y = s.x0 - s.head * h.per_head;
        int lo = 0, hi = h.groups;                 // cum(lo) <= y < cum(hi)
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            (cum(mid) <= y ? lo : hi) = mid;
        }
        s.group = lo;
        starts[b] = s;
    }
}

// Group number `want` of all, found by a whole warp, a lane a sample.  No tokens: there are fewer.
__device__ __forceinline__ ChunkGroup find_group(const ChunkArgs &a, int want, int lane)
{
    const int per_group = kGroupRows / a.group;
    for (int s0 = 0; s0 < a.num_samples; s0 += 32) {
        ChunkSample c{};
        if (s0 + lane < a.num_samples) c = chunk_sample(a, s0 + lane);
        const int groups = (c.n + per_group - 1) / per_group;
        int upto = groups;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += u;
        }
        const unsigned has = __ballot_sync(0xffffffffu, want < upto);
        if (has) {
            const int owner = __ffs(has) - 1;
            const ChunkSample o{__shfl_sync(0xffffffffu, c.q0, owner), __shfl_sync(0xffffffffu, c.n, owner), __shfl_sync(0xffffffffu, c.len, owner),
                                __shfl_sync(0xffffffffu, c.list0, owner)};
            return chunk_group(o, want - __shfl_sync(0xffffffffu, upto - groups, owner), per_group);
        }
        want -= __shfl_sync(0xffffffffu, upto, 31);
    }
    return {};
}

struct ChunkPiece {
    ChunkGroup g;
    int head, t0, t1;      // key tiles
    bool split;            // not the whole group: the result is partial and goes to `slot`
    int slot;
};
// What a block's warps have to know of its share, in shared memory: registers are scarce.
struct ChunkShare {
    long long per_head, x0, x1;
    int32_t groups, whole;     // whole: `own` is all there is
    int32_t head, group;       // where it starts; head num_kv_heads: nothing to do
    ChunkGroup own;
};
// by a whole warp
__device__ __forceinline__ ChunkShare chunk_share(const ChunkArgs &a, int block, int lane)
{
    ChunkShare s{};
    s.head = a.num_kv_heads;
    if (a.direct) {
        s.whole = 1;
        s.own = find_group(a, block % a.direct, lane);
        if (s.own.n_tok > 0) s.head = block / a.direct;
        return s;
    }
    const ChunkHeader h = *a.header;
    const ChunkStart start = a.starts[block];      // asked for together with the header
    if (block >= h.blocks || h.groups == 0) return s;
    s.whole = h.whole;
    s.groups = h.groups;
    if (h.whole) {
        s.head = block / h.groups;
        s.own = a.groups[block % h.groups];
        return s;
    }
    s.per_head = h.per_head;
    s.x0 = start.x0;
    s.x1 = start.x1;
    s.head = start.head;
    s.group = start.group;
    return s;
}
// The pieces of one block's share, in order.
struct ChunkWalk {
    const ChunkArgs &a;
    const ChunkShare &share;
    int head, gi;
    __device__ __forceinline__ ChunkWalk(const ChunkArgs &args, const ChunkShare &s) : a(args), share(s), head(s.head), gi(s.group) {}
    __device__ __forceinline__ bool next(ChunkPiece &p)
    {
        if (share.whole) {
            if (head >= a.num_kv_heads) return false;
            p.g = share.own;
            p.head = head;
            p.t0 = 0;
            p.t1 = chunk_tiles(p.g.keys);
            p.split = false;
            p.slot = 0;
            head = a.num_kv_heads;
            return true;
        }
        for (;;) {
            if (gi >= share.groups) {
                gi = 0;
                ++head;
            }
            if (head >= a.num_kv_heads) return false;
            p.g = a.groups[gi];
            const long long base = head * share.per_head + p.g.cum;
            if (base >= share.x1) {
                head = a.num_kv_heads;
                return false;
            }
            ++gi;
            p.head = head;
            const int tiles = chunk_tiles(p.g.keys);
            p.t0 = tile_at(p.g, a.group, base, share.x0);
            p.t1 = tile_at(p.g, a.group, base, share.x1);
            p.split = false;
            p.slot = 0;
            if (tiles == 0) {
                if (base < share.x0) continue;     // the share where it starts has it
                return true;
            }
            if (p.t1 <= p.t0) continue;
            p.split = p.t0 > 0 || p.t1 < tiles;
            p.slot = 2 * int(blockIdx.x) + (p.t0 > 0 ? 0 : 1);
            return true;
        }
    }
};

// Two partial results of a row joined: their shares and the joint log2-sum-exp.
struct Joined { float first, second, lse2; };
__device__ __forceinline__ Joined join(float a2, float b2)
{
    const float top = fmaxf(a2, b2);
    if (a2 == -INFINITY && b2 == -INFINITY) return {0.f, 0.f, -INFINITY};   // not where one is NaN, which `top` does not show
    const float wa = exp2f(a2 - top), wb = exp2f(b2 - top), sum = wa + wb;
    return {wa / sum, wb / sum, top + log2f(sum)};
}
#endif

// chunk_sm100.cu: places in a call's scratch memory (sets the pointers; returns the bytes), checks, tensor maps of q and the pools
size_t chunk_layout(ChunkArgs &a, void *scratch, int head_dim);
psa_status_t chunk_check(const ChunkArgs &a, const void *q, const int64_t q_strides[2], const void *pool, const int64_t pool_strides[3], int head_dim);
psa_status_t chunk_q_map(const ChunkArgs &a, const void *q, const int64_t q_strides[2], int head_dim, int rows, CUtensorMap *map);
psa_status_t chunk_pool_map(const ChunkArgs &a, const void *pool, const int64_t pool_strides[3], int head_dim, CUtensorMap *map);
int multiprocessors();   // of the current device; 0: there is none

}  // namespace psa
