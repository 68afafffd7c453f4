// Log probabilities of given tokens, with entropy and the likeliest tokens (psa_token_logprobs).  For a row of logits x at temperature T:
//     m = max x,  d_i = (x_i - m) / T,  l = sum e^(d_i):   log p_t = d_t - ln l,   H = ln l - (sum e^(d_i) d_i) / l,
// and the k largest logits (of equal ones the lower token).
//
// One pass over the logits, which is all there is to read: a thread keeps (m, l, sum e d) of the vectors it meets, rescaling when its
// maximum moves, and they are joined at the end.  A row is a block, or a cluster of 2 to 8 blocks where there are few rows; the blocks'
// results meet in the first one's shared memory.
//
// The likeliest tokens come out of the same pass.  A (logit, token) pair is ordered by a 64-bit key, equal logits by the lower token, so
// nothing depends on who comes first.  From the threads' maxima over the first tile every warp takes its r-th largest, r = ceil(k / warps):
// at least k logits are as large as the smallest of these, which is the first border.  What lies above the border is appended to a list;
// a list that is full is cut to its k largest, whose least one is the new border, and the tile is gone through again.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <string>

#include "psa_internal.h"

namespace psa {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kPer = 16;                          // logits of a thread in a tile
constexpr int kTile = kThreads * kPer;
constexpr int kList = 2048;
constexpr int kMostTop = 64, kMostCluster = 8;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct LogprobArgs {
    const void *logits;
    int64_t stride, top_stride;
    int32_t vocab, top, segment;                  // segment: logits of a block, a multiple of 8
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

// running (m, l, s = sum 2^d d), d in log2 units against m; m is -inf until something was seen
struct Sums { float m, l, s; };
__device__ __forceinline__ Sums joined(const Sums &a, const Sums &b, float c)
{
    const float m = fmaxf(a.m, b.m);
    if (m == -INFINITY) return {m, a.l + b.l, a.s + b.s};
    Sums r{m, 0.f, 0.f};
    const Sums both[2] = {a, b};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (both[i].m == -INFINITY) {             // nothing, or NaN alone
            r.l += both[i].l;
            r.s += both[i].s;
            continue;
        }
        const float d = (both[i].m - m) * c, w = exp2f(d);
        r.l += both[i].l * w;
        r.s += w * (both[i].s + both[i].l * (d < -200.f ? 0.f : d));
    }
    return r;
}

template <class T>
struct Vec;
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int kLoads = 2;              // of 16 bytes, for kPer logits
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
    static constexpr int kLoads = 4;
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
    uint32_t border[kWarps];
    int count, listed;
};

// The k-th largest of list[0 .. n), n > k > 0: bit by bit, counting what is at least that large.
__device__ unsigned long long kth(const unsigned long long *list, int n, int k)
{
    unsigned long long at = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const unsigned long long test = at | 1ull << bit;
        int mine = 0;
        for (int i = threadIdx.x; i < n; i += kThreads) mine += list[i] >= test;
        // a thread has at most kList / kThreads of them: sum by counting each
        int total = 0;
#pragma unroll
        for (int i = 1; i <= kList / kThreads; ++i) total += __syncthreads_count(mine >= i);
        if (total >= k) at = test;
    }
    return at;
}

// The k largest of list[0 .. n) in order to `to` (fewer if there are fewer); returns how many.
__device__ int sorted_best(const unsigned long long *list, int n, int k, unsigned long long *to)
{
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const unsigned long long mine = list[i];
        int rank = 0;
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
    const float inv_t = 1.f / t, c = inv_t * kLog2e;

    constexpr int kLoads = Vec<T>::kLoads, kVec = 16 / int(sizeof(T));
    // load i of a thread in the tile at v: kVec logits from v + (i * kThreads + thread) * kVec on
    auto load = [&](int v, uint4 (&w)[kLoads]) {
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
    if (threadIdx.x == 0) sh.count = 0;

    Sums sum{-INFINITY, 0.f, 0.f};
    unsigned long long border = 0;                 // keys above it are listed
    uint4 next[kLoads];
    if (v0 < v1) load(v0, next);
    for (int v = v0; v < v1; v += kTile) {
        float x[kPer];
        Vec<T>::get(next, x);
        if (v + kTile < v1) load(v + kTile, next);
        float top[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
        for (int i = 4; i < kPer; ++i) top[i & 3] = fmaxf(top[i & 3], x[i]);
        const float most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        if (most > sum.m) {
            if (sum.m != -INFINITY) {
                const float d = (sum.m - most) * c, w = exp2f(d);
                sum.s = w * (sum.s + sum.l * fmaxf(d, -200.f));
                sum.l *= w;
            }
            sum.m = most;
        }
        const float off = sum.m == -INFINITY ? 0.f : -sum.m;
        float l[2] = {0.f, 0.f}, s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const float d = (x[i] + off) * c;
            float e;
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(d));
            l[i & 1] += e;
            s[i & 1] = fmaf(e, fmaxf(d, -200.f), s[i & 1]);     // 0 x -inf; e is 0 there
        }
        sum.l += l[0] + l[1];
        sum.s += s[0] + s[1];

        if (a.top == 0) continue;
        auto token = [&](int i) { return v + (i / kVec * kThreads + int(threadIdx.x)) * kVec + i % kVec; };
        if (v == v0) {
            // the first border, from the threads' maxima: below the smallest of the warps' r-th largest
            const int full = min(kWarps, (min(v1 - v0, kThreads * kVec)) / (32 * kVec));    // warps all of whose threads have logits
            uint32_t rth = 0;
            if (full > 0) {
                uint32_t mine = most == most ? ordered(most + 0.f) : 0u;
                const int r = (a.top + full - 1) / full;
                for (int i = 0; i < r && i < 32; ++i) {
                    rth = __reduce_max_sync(0xffffffffu, mine);
                    const unsigned has = __ballot_sync(0xffffffffu, mine == rth);
                    if (lane == __ffs(has) - 1) mine = 0;
                }
                if (r > 32) rth = 0;
            }
            if (lane == 0) sh.border[warp] = rth;
            __syncthreads();
            uint32_t least = full > 0 ? 0xffffffffu : 0u;
            for (int w = 0; w < full; ++w) least = min(least, sh.border[w]);
            border = least == 0 ? 0 : ((unsigned long long)least << 32) - 1;    // keys of that value and above are listed
        }
        // what lies above the border; -inf only where its place alone can bring it among the first
        int before = v == v0 ? 0 : sh.count;       // listed by earlier tiles
        __syncthreads();
        const unsigned long long first_border = border;
        for (;;) {
            // -inf is ordered as 0x007fffff: a border down there keeps nothing out
            if (border < 0x00800000ull << 32 || most >= from_ordered(uint32_t(border >> 32))) {
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const int id = token(i);
                    const unsigned long long k = key_of(x[i], id);
                    if (k > border && id < v1 && (x[i] > -INFINITY || (x[i] == -INFINITY && id < v0 + a.top))) {
                        const int place = atomicAdd(&sh.count, 1);
                        if (place < kList) sh.list[place] = k;
                    }
                }
            }
            __syncthreads();
            if (sh.count <= kList) break;
            // full: its k-th largest is the border of what can still count, for this tile again and for those to come
            const unsigned long long least = kth(sh.list, kList, a.top);
            unsigned long long mine[kList / kThreads];
#pragma unroll
            for (int i = 0; i < kList / kThreads; ++i) mine[i] = sh.list[i * kThreads + threadIdx.x];
            __syncthreads();
            if (threadIdx.x == 0) sh.count = 0;
            __syncthreads();
            // of what earlier tiles listed, the part that still counts; the tile's own is listed again
#pragma unroll
            for (int i = 0; i < kList / kThreads; ++i)
                if (i * kThreads + int(threadIdx.x) < before && mine[i] >= least) sh.list[atomicAdd(&sh.count, 1)] = mine[i];
            border = least - 1;
            __syncthreads();
            before = sh.count;
            __syncthreads();
        }
        // as many as are wanted lie at or above the first border, at lower tokens than all to come: from here on only larger values count
        if (v == v0 && border == first_border && border != 0) border += 1ull << 32;
    }

    // ---- the block's sums and best
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        const Sums o{__shfl_xor_sync(0xffffffffu, sum.m, d), __shfl_xor_sync(0xffffffffu, sum.l, d), __shfl_xor_sync(0xffffffffu, sum.s, d)};
        sum = lane & d ? joined(o, sum, c) : joined(sum, o, c);
    }
    if (lane == 0) sh.warp_sums[warp] = sum;
    __syncthreads();
    int n = sh.count;
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWarps; ++w) sum = joined(sum, sh.warp_sums[w], c);
        sh.block = sum;
    }
    if (a.top > 0) {
        if (n > kThreads) {
            const unsigned long long least = kth(sh.list, n, a.top);
            unsigned long long mine[kList / kThreads];
#pragma unroll
            for (int i = 0; i < kList / kThreads; ++i) mine[i] = i * kThreads + int(threadIdx.x) < n ? sh.list[i * kThreads + threadIdx.x] : 0;
            __syncthreads();
            if (threadIdx.x == 0) sh.count = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kList / kThreads; ++i)
                if (mine[i] >= least && i * kThreads + int(threadIdx.x) < n) sh.list[atomicAdd(&sh.count, 1)] = mine[i];
            __syncthreads();
            n = sh.count;
        }
        n = sorted_best(sh.list, n, a.top, sh.best);
    }
    if (threadIdx.x == 0) sh.listed = n;
    if (blocks > 1) {
        cluster.sync();
        if (part == 0) {
            int total = 0;
            for (int b = 0; b < blocks; ++b) {
                const Shared *o = cluster.map_shared_rank(&sh, b);
                const int have = o->listed;
                for (int i = threadIdx.x; i < have; i += kThreads) sh.gathered[total + i] = o->best[i];
                total += have;
                if (threadIdx.x == 0) sh.all[b] = o->block;
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                Sums all = sh.all[0];
                for (int b = 1; b < blocks; ++b) all = joined(all, sh.all[b], c);
                sh.block = all;
            }
            if (a.top > 0) n = sorted_best(sh.gathered, total, a.top, sh.best);
        }
        cluster.sync();                            // nobody leaves while its shared memory is read
        if (part != 0) return;
    }
    __syncthreads();
    const Sums all = sh.block;
    const float ln_l = logf(all.l);
    auto logprob = [&](float x) { return x == -INFINITY && !(all.l != all.l) ? -INFINITY : (x - all.m) * inv_t - ln_l; };
    if (threadIdx.x == 0) {
        const int token = a.tokens ? a.tokens[row] : -1;
        if (a.logprobs) a.logprobs[row] = token >= 0 && token < a.vocab ? logprob(float(x_row[token])) : -INFINITY;
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
    // blocks of a row: as many as keep the SMs (two blocks each) busy, with a tile of work for every one
    int blocks = 1;
    while (blocks < kMostCluster && int64_t(num_rows) * blocks * 2 <= 2 * 148 && int64_t(vocab) > int64_t(kTile) * blocks) blocks *= 2;
    a.segment = int32_t(((int64_t(vocab) + blocks - 1) / blocks + 7) / 8 * 8);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = logits_dtype == PSA_OUT_BF16 ? launch<__nv_bfloat16>(a, num_rows, blocks, st) : launch<float>(a, num_rows, blocks, st);
    if (e != cudaSuccess) return set_last_error(PSA_ERR_CUDA, std::string("log probabilities launch: ") + cudaGetErrorString(e));
    return PSA_OK;
}
