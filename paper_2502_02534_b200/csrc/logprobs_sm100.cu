// Log probabilities of given tokens, with entropy and the likeliest tokens (psa_token_logprobs).  For a row of logits x at temperature T:
//     m = max x,  d_i = (x_i - m) / T,  l = sum e^(d_i):   log p_t = d_t - ln l,   H = ln l - (sum e^(d_i) d_i) / l,
// and the k largest logits (of equal ones the lower token).
//
// One pass over the logits, which is all there is to read: a thread keeps (m, l, sum e d) of the vectors it meets, rescaling when its
// maximum moves, and they are joined at the end.  A row is a block, or a cluster of 2 to 8 blocks where there are few rows; the blocks'
// results meet in the first one's shared memory.
//
// The likeliest tokens cost the pass next to nothing.  Every warp gives the four largest of its threads' maxima, and the k-th largest of those
// is the border: k logits reach it, so the k largest lie with the few threads whose maximum does.  Those find in
// shared memory which of their tiles do (16 bits of each tile's maximum, rounded down); these are read once more, a vector a thread, and what
// reaches the border is listed.
// A (logit, token) pair is ordered by a 64-bit key, equal logits by the lower token, so nothing depends on who comes first.  A list that
// is too short (many equal logits) gives a higher border, its own k-th largest, and is made again.  256 rows x 131072 bf16, k = 20:
// listing inside the pass, with a border kept by the block 64 us, by each warp 164 us; all tiles read again 31 us; this way 22 us, of which
// 5 are the tail, and 16.9 us without likeliest tokens (floor 10.3).  256 rows x 131072 f32 24.8 us (floor 20.5).
// What bounds it: 24 instructions a pair of logits and warp, selection included, are 11 us of all issue slots (58 % of them taken with four
// rows an SM, special-function units 43 %); the rest is the begin and the end, when SMs have nothing to do (23 % of the time with 256 rows), and
// 256 rows on 148 SMs (the busiest SM 1.11 of the mean).
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cfloat>
#include <string>

#include "psa_internal.h"
#include "tensor_core.cuh"

namespace psa {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kPer = 16;                          // logits of a thread in a tile
constexpr int kTile = kThreads * kPer;
constexpr int kList = 2048;
constexpr int kCells = 512;
constexpr int kMarks = 24;                        // tile maxima kept of a thread: longer rows keep those of runs of tiles
constexpr int kGiven = 4;                         // maxima that a warp gives
constexpr int kMostTop = 64, kMostCluster = 8;
static_assert(kGiven * kWarps == 64 && kMostTop <= kGiven * kWarps, "the border is the kMostTop-th of them at most; two a lane");
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct LogprobArgs {
    const void *logits;
    int64_t stride, top_stride;
    int32_t vocab, top, segment, run_tiles;       // segment: logits of a block, a multiple of 8; run_tiles: tiles that share a mark
    const int32_t *tokens;
    const float *temperature;
    float *logprobs, *entropy, *top_logprobs;
    int32_t *top_ids;
};

__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ unsigned long long key_of(float x, int token) { return (unsigned long long)ordered(x + 0.f) << 32 | uint32_t(~token); }

constexpr uint32_t kKeyOfNothing = 0x007fffffu;   // ordered(-inf)

// Running sums: l = sum 2^d, s = sum 2^d d, exponents d in log2 units against m, a logit at most 2^8 below the largest (-inf: nothing yet).
struct Sums { float m, l, s; };
// ... against another reference, above m or equal
__device__ __forceinline__ Sums moved(const Sums &a, float m, float c)
{
    if (a.m == -INFINITY) return {m, a.l, a.s};    // nothing, or NaN alone
    const float d = fmaxf((a.m - m) * c, -200.f);
    float w;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(d));
    return {m, a.l * w, w * fmaf(a.l, d, a.s)};
}
// of the lanes below `lanes` of a whole warp, to every lane
template <int kLanes>
__device__ __forceinline__ Sums joined(Sums a, float c)
{
    const uint32_t top = __reduce_max_sync(0xffffffffu, ordered(a.m));
    a = moved(a, from_ordered(top), c);
#pragma unroll
    for (int d = kLanes / 2; d; d >>= 1) {
        a.l += __shfl_xor_sync(0xffffffffu, a.l, d);
        a.s += __shfl_xor_sync(0xffffffffu, a.s, d);
    }
    return a;
}

template <class T>
struct Vec;
template <>
struct Vec<__nv_bfloat16> {
    static __device__ __forceinline__ void one(const uint4 &w, float (&x)[8])
    {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[2 * k] = __uint_as_float(u[k] << 16);
            x[2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
        }
    }
    static constexpr int kLoads = 2;              // of 16 bytes, for kPer logits
    static constexpr int kAhead = 2;              // tiles on their way
    // the largest of a thread's logits, in packed bf16 (NaN does not count)
    static __device__ __forceinline__ float most(const uint4 (&w)[2], const float (&)[kPer])
    {
        const uint32_t u[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
        uint32_t m[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("max.bf16x2 %0, %1, %2;" : "=r"(m[i]) : "r"(u[i]), "r"(u[i + 4]));
        asm("max.bf16x2 %0, %0, %1;" : "+r"(m[0]) : "r"(m[1]));
        asm("max.bf16x2 %0, %0, %1;" : "+r"(m[2]) : "r"(m[3]));
        asm("max.bf16x2 %0, %0, %1;" : "+r"(m[0]) : "r"(m[2]));
        return fmaxf(__uint_as_float(m[0] << 16), __uint_as_float(m[0] & 0xffff0000u));
    }
    static __device__ __forceinline__ void get(const uint4 (&w)[2], float (&x)[kPer])
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[i * 8 + 2 * k] = __uint_as_float(u[k] << 16);
                x[i * 8 + 2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
            }
        }
    }
};
template <>
struct Vec<float> {
    static __device__ __forceinline__ void one(const uint4 &w, float (&x)[4])
    {
        x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
    }
    static constexpr int kLoads = 4, kAhead = 1;
    static __device__ __forceinline__ float most(const uint4 (&)[4], const float (&x)[kPer])
    {
        float top[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
        for (int i = 4; i < kPer; ++i) top[i & 3] = fmaxf(top[i & 3], x[i]);
        return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    }
    static __device__ __forceinline__ void get(const uint4 (&w)[4], float (&x)[kPer])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[4 * i] = __uint_as_float(w[i].x); x[4 * i + 1] = __uint_as_float(w[i].y);
            x[4 * i + 2] = __uint_as_float(w[i].z); x[4 * i + 3] = __uint_as_float(w[i].w);
        }
    }
};

struct Shared {
    unsigned long long list[kList], best[kMostTop], gathered[kMostCluster * kMostTop];
    Sums warp_sums[kWarps], block, all[kMostCluster];
    uint32_t given[kGiven * kWarps], reached;
    int count, cells_found, listed[kMostCluster];
    uint16_t cells[kCells];
    uint16_t marks[kMarks][kThreads];
};

// The k-th largest of list[0 .. n), n >= k > 0, to every thread: bit by bit, counting what is at least that large.
__device__ unsigned long long kth(const Shared &sh, int n, int k)
{
    unsigned long long mine[kList / kThreads];
#pragma unroll
    for (int i = 0; i < kList / kThreads; ++i) mine[i] = i * kThreads + int(threadIdx.x) < n ? sh.list[i * kThreads + threadIdx.x] : 0;
    unsigned long long at = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const unsigned long long test = at | 1ull << bit;
        int total = 0;
#pragma unroll
        for (int i = 0; i < kList / kThreads; ++i) total += __syncthreads_count(mine[i] >= test);
        if (total >= k) at = test;
        if (total == k) break;
    }
    return at;
}

// The k largest of list[0 .. n) in order to `to` (fewer if there are fewer); returns how many.
__device__ int sorted_best(const unsigned long long *list, int n, int k, unsigned long long *to)
{
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const unsigned long long mine = list[i];
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j < n; ++j) rank += list[j] > mine;
        if (rank < k) to[rank] = mine;
    }
    __syncthreads();
    return min(n, k);
}

template <class T>
__global__ void __launch_bounds__(kThreads, 2)
logprobs_kernel(const LogprobArgs a)
{
    __shared__ Shared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = int(cluster.num_blocks()), part = int(cluster.block_rank());
    const int row = blockIdx.x / blocks;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T *x_row = static_cast<const T *>(a.logits) + row * a.stride;
    const int v0 = min(a.vocab, part * a.segment), v1 = min(a.vocab, v0 + a.segment);
    float t = a.temperature ? a.temperature[row] : 1.f;
    if (!(t > 0.f && t < INFINITY)) t = 1.f;
    const float inv_t = fminf(1.f / t, 1e38f), c = inv_t * kLog2e;   // finite: 0 / T is 0 for the smallest T too
    float asked = -INFINITY;                       // the given token's logit; its way is long, so it starts here
    if (part == 0 && threadIdx.x == 0 && a.logprobs) {
        const int token = a.tokens[row];
        if (token >= 0 && token < a.vocab) asked = float(x_row[token]);
    }

    constexpr int kLoads = Vec<T>::kLoads, kVec = 16 / int(sizeof(T));
    if (blocks > 1) cluster.barrier_arrive();      // nobody writes to a block that has not begun
    // load i of a thread in the tile at v: kVec logits from v + (i * kThreads + thread) * kVec on
    auto load = [&](int v, uint4 (&w)[kLoads]) {
        if (v + kTile <= v1) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) w[i] = __ldcs(reinterpret_cast<const uint4 *>(x_row + v + (i * kThreads + int(threadIdx.x)) * kVec));
            return;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int at = v + (i * kThreads + int(threadIdx.x)) * kVec;
            if (at + kVec <= v1) {
                w[i] = __ldcs(reinterpret_cast<const uint4 *>(x_row + at));
            } else {                               // the row's end, one by one; behind it -inf
                alignas(16) T e[kVec];
#pragma unroll
                for (int k = 0; k < kVec; ++k) e[k] = at + k < v1 ? x_row[at + k] : T(-INFINITY);
                w[i] = *reinterpret_cast<const uint4 *>(e);
            }
        }
    };
    Sums sum{-INFINITY, 0.f, 0.f};
    float most = -INFINITY, limit = -INFINITY;     // the thread's largest logit; what the reference holds for
    float run_top = -INFINITY;
    int run = 0, marks = 0;
    constexpr int kAhead = Vec<T>::kAhead;
    uint4 w[kAhead][kLoads];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (v0 + i * kTile < v1) load(v0 + i * kTile, w[i]);
    auto tile = [&](int v, uint4 (&now)[kLoads]) {
        float x[kPer];
        Vec<T>::get(now, x);
        const float top_here = Vec<T>::most(now, x);
        if (v + kAhead * kTile < v1) load(v + kAhead * kTile, now);
        most = fmaxf(most, top_here);
        if (a.top > 0) {
            run_top = fmaxf(run_top, top_here);
            if (++run == a.run_tiles) {
                sh.marks[marks++][threadIdx.x] = uint16_t(ordered(run_top + 0.f) >> 16);
                run = 0;
                run_top = -INFINITY;
            }
        }
        // the reference moves when an exponent would pass 2^8; the sums do not mind being taken against a smaller one
        if (top_here > limit) {
            if (sum.m != -INFINITY) {
                const float d = (sum.m - top_here) * c, r = exp2f(d);
                sum.s = r * (sum.s + sum.l * fmaxf(d, -200.f));
                sum.l *= r;
            }
            sum.m = top_here;
            limit = fminf(top_here + 8.f / c, FLT_MAX);    // which a logit of +inf passes whatever the temperature
        }
        const float off = sum.m == -INFINITY ? 0.f : -sum.m;
        float2 l = {0.f, 0.f}, s = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kPer; i += 2) {
            float2 d = add2(make_float2(x[i], x[i + 1]), make_float2(off, off)), e;      // exact where it matters: near the maximum
            d = fma2(d, make_float2(c, c), make_float2(0.f, 0.f));
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(d.x));
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(d.y));
            l = add2(l, e);
            s = fma2(e, make_float2(fmaxf(d.x, -200.f), fmaxf(d.y, -200.f)), s);         // not 0 x -inf: e is 0 there
        }
        sum.l += l.x + l.y;
        sum.s += s.x + s.y;
    };
    for (int v = v0; v < v1; v += kAhead * kTile) {
        tile(v, w[0]);
        if constexpr (kAhead > 1)
            if (v + kTile < v1) tile(v + kTile, w[kAhead - 1]);
    }

    // ---- the block's sums and best
    sum = joined<32>(sum, c);
    if (lane == 0) sh.warp_sums[warp] = sum;
    if (threadIdx.x == 0) sh.count = sh.cells_found = 0;
    const uint32_t top_key = ordered(most + 0.f);  // never NaN
    if (a.top > 0) {
        if (run > 0) sh.marks[marks++][threadIdx.x] = uint16_t(ordered(run_top + 0.f) >> 16);
        uint32_t left = top_key;
#pragma unroll
        for (int r = 0; r < kGiven; ++r) {
            const uint32_t one = __reduce_max_sync(0xffffffffu, left);
            if (lane == __ffs(__ballot_sync(0xffffffffu, left == one)) - 1) left = 0;
            if (lane == 0) sh.given[r * kWarps + warp] = one;
        }
    }
    __syncthreads();
    if (warp == kWarps - 1) {
        sum = joined<kWarps>(lane < kWarps ? sh.warp_sums[lane] : Sums{-INFINITY, 0.f, 0.f}, c);
        if (lane == 0) sh.block = sum;
    }
    int n = 0;
    if (a.top > 0) {
        // the a.top-th largest of what the warps gave
        if (threadIdx.x < kGiven * kWarps) {
            const uint32_t mine = sh.given[threadIdx.x];
            int larger = 0;
#pragma unroll
            for (int i = 0; i < kGiven * kWarps; ++i) {
                const uint32_t o = sh.given[i];
                larger += o > mine || (o == mine && i < int(threadIdx.x));
            }
            if (larger == a.top - 1) sh.reached = mine;
        }
        __syncthreads();
        const uint32_t reached = sh.reached;
        // which tiles reach it: (mark, thread)
        const bool again = top_key >= reached;
        if (again) {
            const uint16_t least = uint16_t(reached >> 16);
#pragma unroll 4
            for (int m = 0; m < marks; ++m)
                if (sh.marks[m][threadIdx.x] >= least) {
                    const int place = atomicAdd(&sh.cells_found, 1);
                    if (place < kCells) sh.cells[place] = uint16_t(m * kThreads + threadIdx.x);
                }
        }
        __syncthreads();
        const int cells = sh.cells_found;
        // Of masked tokens only those can be among the likeliest that have fewer than a.top others before them.  NaN ones do not count, so
        // where there are any, and masked tokens are needed, the others are counted.
        int masked_end = v0 + a.top;
        if (reached == kKeyOfNothing && sh.block.l != sh.block.l) {
            masked_end = v0;
            for (int others = 0; others < a.top && masked_end < v1; masked_end += kThreads) {
                const int at = masked_end + int(threadIdx.x);
                const float x = at < v1 ? float(x_row[at]) : -INFINITY;
                others += __syncthreads_count(at < v1 && x == x);
            }
        }
        unsigned long long border = (unsigned long long)reached << 32;      // keys from it on are listed
        for (;;) {
            const float least = from_ordered(max(uint32_t(border >> 32), kKeyOfNothing));     // at least -inf
            // `per` consecutive logits from x on, the first of which is token `id`
            auto list = [&](const float *x, int per, int id) {
#pragma unroll
                for (int i = 0; i < per; ++i)
                    if (x[i] >= least) {
                        const unsigned long long k = key_of(x[i], id + i);
                        if (k >= border && id + i < v1 && (x[i] > -INFINITY || id + i < masked_end)) {
                            const int place = atomicAdd(&sh.count, 1);
                            if (place < kList) sh.list[place] = k;
                        }
                    }
            };
            if (cells <= kCells) {
                // a vector a thread
                const int each = a.run_tiles * kLoads;
                for (int i = threadIdx.x; i < cells * each; i += kThreads) {
                    const int cell = sh.cells[i / each], which = i % each;
                    const int id = v0 + (cell / kThreads * a.run_tiles + which / kLoads) * kTile + (which % kLoads * kThreads + cell % kThreads) * kVec;
                    float x[kVec];
                    if (id + kVec <= v1) {
                        const uint4 u = __ldg(reinterpret_cast<const uint4 *>(x_row + id));
                        Vec<T>::one(u, x);
                    } else {
#pragma unroll
                        for (int k = 0; k < kVec; ++k) x[k] = id + k < v1 ? float(x_row[id + k]) : -INFINITY;
                    }
                    list(x, kVec, id);
                }
            } else if (again) {
                // too many for a list: everyone goes through their own
                for (int v = v0; v < v1; v += kTile) {
                    uint4 now[kLoads];
                    float x[kPer];
                    load(v, now);
                    Vec<T>::get(now, x);
                    if (!(Vec<T>::most(now, x) >= least)) continue;
#pragma unroll
                    for (int i = 0; i < kLoads; ++i) list(x + i * kVec, kVec, v + (i * kThreads + int(threadIdx.x)) * kVec);
                }
            }
            __syncthreads();
            n = sh.count;
            if (n <= kList) break;
            border = kth(sh, kList, a.top);        // k of what was listed reach it
            __syncthreads();
            if (threadIdx.x == 0) sh.count = 0;
            __syncthreads();
        }
        if (n > kThreads) {
            // few enough to be ranked against one another
            const unsigned long long least = kth(sh, n, a.top);
            unsigned long long kept[kList / kThreads];
#pragma unroll
            for (int i = 0; i < kList / kThreads; ++i) kept[i] = i * kThreads + int(threadIdx.x) < n ? sh.list[i * kThreads + threadIdx.x] : 0;
            __syncthreads();
            if (threadIdx.x == 0) sh.count = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kList / kThreads; ++i)
                if (kept[i] >= least && kept[i]) sh.list[atomicAdd(&sh.count, 1)] = kept[i];
            __syncthreads();
            n = sh.count;
        }
        n = sorted_best(sh.list, n, a.top, sh.best);
    }
    if (blocks > 1) {
        // every block sends its part to the first one
        Shared *const first = cluster.map_shared_rank(&sh, 0);
        __syncthreads();                           // sh.block
        cluster.barrier_wait();
        for (int i = threadIdx.x; i < n; i += kThreads) first->gathered[part * kMostTop + i] = sh.best[i];
        if (threadIdx.x == 0) {
            first->all[part] = sh.block;
            first->listed[part] = n;
        }
        cluster.sync();
        if (part != 0) return;
        if (a.top > 0) {
            // closed up (the list's memory is free), then ranked
            if (warp < blocks) {
                int to = 0;
                for (int b = 0; b < warp; ++b) to += sh.listed[b];
                for (int i = lane; i < sh.listed[warp]; i += 32) sh.list[to + i] = sh.gathered[warp * kMostTop + i];
            }
            int total = 0;
            for (int b = 0; b < blocks; ++b) total += sh.listed[b];
            __syncthreads();
            n = sorted_best(sh.list, total, a.top, sh.best);
        }
        if (warp == kWarps - 1) {
            sum = joined<kMostCluster>(lane < blocks ? sh.all[lane] : Sums{-INFINITY, 0.f, 0.f}, c);
            if (lane == 0) sh.block = sum;
        }
    }
    __syncthreads();
    const Sums all = sh.block;
    const float ln_l = logf(all.l);
    auto logprob = [&](float x) { return x == -INFINITY && !(all.l != all.l) ? -INFINITY : (x - all.m) * inv_t - ln_l; };
    if (threadIdx.x == 0) {
        if (a.logprobs) a.logprobs[row] = logprob(asked);
        if (a.entropy) a.entropy[row] = all.l == 0.f ? 0.f : fmaxf(ln_l - kLn2 * all.s / all.l, 0.f) + (all.l != all.l ? all.l : 0.f);
    }
    for (int i = threadIdx.x; i < a.top; i += kThreads) {
        const bool is = i < n;
        const unsigned long long k = is ? sh.best[i] : 0;
        if (a.top_ids) a.top_ids[row * a.top_stride + i] = is ? int(~uint32_t(k)) : -1;
        if (a.top_logprobs) a.top_logprobs[row * a.top_stride + i] = is ? logprob(from_ordered(uint32_t(k >> 32))) : -INFINITY;
    }
}

template <class T>
cudaError_t launch(const LogprobArgs &a, int rows, int blocks, cudaStream_t st)
{
    cudaLaunchConfig_t lc{};
    lc.gridDim = dim3(unsigned(rows) * unsigned(blocks));
    lc.blockDim = dim3(kThreads);
    lc.stream = st;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = unsigned(blocks);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    lc.attrs = &attr;
    lc.numAttrs = 1;
    return cudaLaunchKernelEx(&lc, logprobs_kernel<T>, a);
}

bool misaligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

}  // namespace
}  // namespace psa

extern "C" psa_status_t psa_token_logprobs(const void *logits, int32_t logits_dtype, int64_t row_stride, int32_t num_rows, int32_t vocab,
                                           const int32_t *tokens, const float *temperature, float *logprobs, float *entropy, int32_t top,
                                           int32_t *top_ids, float *top_logprobs, int64_t top_stride, void *cuda_stream)
{
    using namespace psa;
    if (num_rows < 0 || vocab < 1 || top < 0) return set_last_error(PSA_ERR_INVALID_ARG, "negative sizes or no vocabulary");
    if (logits_dtype != PSA_OUT_BF16 && logits_dtype != PSA_OUT_F32) return set_last_error(PSA_ERR_UNSUPPORTED, "logits must be bf16 or f32");
    if (num_rows > 65535 || vocab > (1 << 24)) return set_last_error(PSA_ERR_UNSUPPORTED, "at most 65535 rows and 2^24 tokens");
    if (top > kMostTop || top > vocab) return set_last_error(PSA_ERR_UNSUPPORTED, "at most 64 top tokens, and no more than there are");
    if (num_rows == 0) return PSA_OK;
    if (!logits || (logprobs && !tokens) || (top > 0 && top_stride < top)) return set_last_error(PSA_ERR_INVALID_ARG, "null logits, logprobs without tokens, or top_stride < top");
    if (misaligned(logits, 16) || row_stride < vocab || row_stride % 8) return set_last_error(PSA_ERR_INVALID_ARG, "logits must be 16-byte aligned, row_stride a multiple of 8, at least vocab");
    if (misaligned(tokens, 4) || misaligned(temperature, 4) || misaligned(logprobs, 4) || misaligned(entropy, 4) || misaligned(top_ids, 4) || misaligned(top_logprobs, 4))
        return set_last_error(PSA_ERR_INVALID_ARG, "arrays must be 4-byte aligned");
    LogprobArgs a{};
    a.logits = logits; a.stride = row_stride; a.vocab = vocab; a.tokens = tokens; a.temperature = temperature;
    a.logprobs = logprobs; a.entropy = entropy; a.top_ids = top_ids; a.top_logprobs = top_logprobs; a.top_stride = top_stride;
    a.top = top_ids || top_logprobs ? top : 0;
    // Blocks of a row: doubled while all of them still have an SM of the 148 each, and a tile of work.  x 131072 bf16, 20 likeliest: 8, 19, 38,
    // 74, 76, 148, 256 rows 9.5, 9.7, 11.7, 12.5, 14.8, 15.7, 21.5 us; with two blocks an SM 9.4, 10.9, 11.4, 17.7, 14.7, 16.2, 21.6.
    int blocks = 1;
    while (blocks < kMostCluster && int64_t(num_rows) * blocks * 2 <= 148 && int64_t(vocab) > int64_t(kTile) * blocks) blocks *= 2;
    a.segment = int32_t(((int64_t(vocab) + blocks - 1) / blocks + 7) / 8 * 8);
    a.run_tiles = ((a.segment + kTile - 1) / kTile + kMarks - 1) / kMarks;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = logits_dtype == PSA_OUT_BF16 ? launch<__nv_bfloat16>(a, num_rows, blocks, st) : launch<float>(a, num_rows, blocks, st);
    if (e != cudaSuccess) return set_last_error(PSA_ERR_CUDA, std::string("log probabilities launch: ") + cudaGetErrorString(e));
    return PSA_OK;
}
