// Eviction of whole pages by the attention weight their tokens received (psa_evict_pages).
//
// A page weighs as much as its heaviest cell, max over the KV heads and 16 slots of psa_accumulate_weights' array; the newest pages stay
// whatever they weigh, of the others the heaviest up to the budget (equal weights: the older page stays).  K and V do not move: the list
// closes up in order, and the ids that leave go onto the stack of free pages.
//
// A running sum of the pages that go gives every sample its place on the stack.  Where lengths and count are not updated in place each
// block runs it for itself, from all samples' lengths and budgets; otherwise, and for many samples, evict_plan_kernel (one block) does so
// before.  evict_kernel has a block per sample: weights are read once (all of the bytes that matter) by whole warps, one redux a page, and
// kept as ordered 32-bit keys in shared memory.  The border between what stays and goes: up to 512 pages bit by bit with a block-wide count
// (20 barriers or so), else by four histograms of 8 bits.  One scan closes up the list.  8 samples x 512 tokens 6.3 us (two launches and
// histograms alone 10.3); 256 samples of up to 8192 tokens, 33.5 MB, 14.9 us (8 lanes-a-page loops 26, floor 5.1): latency and uneven
// blocks.  Five warps wait for memory for every instruction that is issued, 22 % of the issue slots are taken, and an SM is busy 22 k
// cycles on average, 30 k at most.
#include <cuda_runtime.h>

#include <algorithm>
#include <string>

#include "chunk.h"
#include "psa_internal.h"

namespace psa {
namespace {

constexpr int kPlanThreads = 1024, kThreads = 512, kWarps = kThreads / 32;
constexpr int kAlone = 1024;        // samples up to which every block sums up the others for itself
constexpr int kSharedKeys = 8192;   // longer lists keep their keys in the scratch memory

struct EvictSample {
    int list0, room;       // list
    int pages, budget;     // held; stay at most (budget == pages: nothing goes)
    int recent, to;        // newest pages that stay in any case; place of its first page behind the stack's height
};
struct EvictArgs {
    const float *weights;
    const int32_t *page_indptr, *page_indices, *kv_lens, *budgets, *free_count;
    int32_t *indices_out, *lens_out, *free_pages, *free_count_out, *status;
    int64_t num_entries, free_capacity;
    int32_t num_samples, recent, num_pool_pages, cells;   // cells: Hkv * 16
    int32_t *height;       // scratch: the stack's height before the call
    EvictSample *plan;
    uint32_t *keys;        // [num_entries]
};

__device__ __forceinline__ EvictSample sample_of(const EvictArgs &a, int s)
{
    EvictSample e{};
    const int l0 = a.page_indptr[s], l1 = a.page_indptr[s + 1], len = a.kv_lens[s], budget = a.budgets[s];
    if (l0 < 0 || l1 < l0 || l1 > a.num_entries) {
        raise(a.status, PSA_ERR_BOUNDS);
        return e;
    }
    e.list0 = l0;
    e.room = l1 - l0;
    if (len < 0 || len > (long long)e.room * kPageSize || budget < 1) {
        raise(a.status, PSA_ERR_BOUNDS);
        return e;                                   // nothing held, nothing goes: the list is copied as it is
    }
    e.pages = int(((long long)len + kPageSize - 1) / kPageSize);
    e.budget = min(budget, e.pages);
    e.recent = min(a.recent, e.budget);
    return e;
}

// What every sample does, and whether anything leaves at all, by one block: of all samples (kAll; entry s goes to plan[s], outputs are
// written), or of sample `only` as every block of the other form needs it.
template <bool kAll, int kBlock>
__device__ __forceinline__ EvictSample plan(const EvictArgs &a, int only, int *height_out)
{
    __shared__ long long part[kBlock / 32];
    __shared__ EvictSample chosen;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int height = *a.free_count;
    *height_out = height;
    long long carry = 0;
    for (int s0 = 0; s0 < a.num_samples; s0 += kBlock) {
        const int s = s0 + int(threadIdx.x);
        EvictSample e{};
        if (s < a.num_samples) e = sample_of(a, s);
        const int go = e.pages - e.budget;
        long long x = go;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += u;
        }
        if (lane == 31) part[warp] = x;
        __syncthreads();
        long long before = carry + x - go;
#pragma unroll
        for (int k = 0; k < kBlock / 32; ++k) {
            if (k < warp) before += part[k];
            carry += part[k];
        }
        __syncthreads();
        e.to = int(min(before, 0x7fffffffll));
        if (kAll) {
            if (s < a.num_samples) a.plan[s] = e;
        } else if (s == only) {
            chosen = e;
        }
    }
    // a height that cannot be, or no room on the stack for all of them: nothing goes
    const bool none = height < 0 || height > a.free_capacity || carry > a.free_capacity - height;
    if (kAll) {
        for (int s = threadIdx.x; s < a.num_samples; s += kBlock) {   // the thread's own entries
            EvictSample &e = a.plan[s];
            if (none) e.budget = e.pages;
            const int len = a.kv_lens[s];
            if (a.lens_out) a.lens_out[s] = len - (e.pages - e.budget) * kPageSize;
        }
    } else {
        __syncthreads();
    }
    if (threadIdx.x == 0 && (kAll || only == 0)) {
        if (none) raise(a.status, PSA_ERR_BOUNDS);
        *a.free_count_out = none ? height : int(height + carry);
    }
    if (kAll) return {};
    EvictSample e = chosen;
    if (none) e.budget = e.pages;
    if (threadIdx.x == 0 && a.lens_out) a.lens_out[only] = a.kv_lens[only] - (e.pages - e.budget) * kPageSize;
    return e;
}

__global__ void __launch_bounds__(kPlanThreads)
evict_plan_kernel(EvictArgs a)
{
    grid_release();
    int height;
    plan<true, kPlanThreads>(a, 0, &height);
    if (threadIdx.x == 0) *a.height = height;
}

// larger weight, larger key; NaN never gets here
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <bool kPlanned>
__global__ void __launch_bounds__(kThreads, 2)
evict_kernel(EvictArgs a)
{
    __shared__ uint32_t shared_keys[kSharedKeys];
    __shared__ uint32_t bins[256];
    __shared__ uint32_t part[kWarps];
    __shared__ uint32_t found[2];
    if (kPlanned) grid_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // entries that belong to no list
    if (a.indices_out != a.page_indices) {
        const long long first = min(max(a.page_indptr[0], 0), int(a.num_entries)), end = min(max(a.page_indptr[a.num_samples], 0), int(a.num_entries));
        const long long step = (long long)gridDim.x * kThreads, at = (long long)blockIdx.x * kThreads + threadIdx.x;
        for (long long i = at; i < first; i += step) a.indices_out[i] = a.page_indices[i];
        for (long long i = end + at; i < a.num_entries; i += step) a.indices_out[i] = a.page_indices[i];
    }
    if (int(blockIdx.x) >= a.num_samples) return;   // no samples: all there is to do was above
    int height;
    EvictSample e;
    if (kPlanned) {
        e = a.plan[blockIdx.x];
        height = *a.height;
    } else {
        e = plan<false, kThreads>(a, int(blockIdx.x), &height);
    }
    const int32_t *list = a.page_indices + e.list0;
    int32_t *out = a.indices_out + e.list0;
    const int go = e.pages - e.budget;
    if (go == 0) {
        if (out != list)
            for (int i = threadIdx.x; i < e.room; i += kThreads) out[i] = list[i];
        return;
    }
    const int candidates = e.pages - e.recent, stay = e.budget - e.recent;   // of the candidates
    uint32_t *keys = candidates <= kSharedKeys ? shared_keys : a.keys + e.list0;
    const int newest = int(threadIdx.x) < e.recent ? list[candidates + threadIdx.x] : 0;

    // ---- weights: a warp takes runs of kRun pages, a lane knows one's id and in the end its key; all lanes read a page
    constexpr int kRun = 16, kAhead = 4;
    const int vectors = a.cells / 4;
    for (int c0 = warp * kRun; c0 < candidates; c0 += kWarps * kRun) {
        const int c = c0 + lane;
        int page = lane < kRun && c < candidates ? list[c] : -1;
        if (lane < kRun && c < candidates && (page < 0 || page >= a.num_pool_pages)) {
            raise(a.status, PSA_ERR_BOUNDS);
            page = -1;                            // weighs less than any other
        }
        uint32_t key = 0;
#pragma unroll
        for (int r = 0; r < kRun; r += kAhead) {
            float top[kAhead];
            int at[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                top[i] = -INFINITY;
                at[i] = __shfl_sync(0xffffffffu, page, r + i);
            }
            for (int v = lane; v < vectors; v += 32) {
                float4 x[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
                    if (at[i] >= 0) x[i] = __ldcs(reinterpret_cast<const float4 *>(a.weights + size_t(at[i]) * a.cells) + v);
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
                    if (at[i] >= 0) top[i] = fmaxf(top[i], fmaxf(fmaxf(x[i].x, x[i].y), fmaxf(x[i].z, x[i].w)));
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const uint32_t k = __reduce_max_sync(0xffffffffu, ordered(top[i] + 0.f));   // + 0: -0 weighs as much as 0
                if (lane == r + i && page >= 0) key = k;
            }
        }
        if (lane < kRun && c < candidates) keys[c] = key;
    }

    // ---- the key of the lightest candidate that stays, from its highest byte down
    uint32_t prefix = 0, wanted = uint32_t(stay);
    __syncthreads();
    if (stay > 0 && candidates <= kThreads) {
        // a key a thread: bit by bit, counting those at least that large, until as many as may stay are
        const uint32_t mine = int(threadIdx.x) < candidates ? keys[threadIdx.x] : 0;
        const bool is = int(threadIdx.x) < candidates;
        int above = 0;          // larger than every key that has `prefix`'s bits so far
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t test = prefix | 1u << bit;
            const int n = __syncthreads_count(is && mine >= test);
            if (n >= stay) prefix = test;
            else above = n;
            if (n == stay) break;
        }
        // a count that hit: everything at or above `prefix` stays
        wanted = uint32_t(stay - above);
        if (__syncthreads_count(is && mine >= prefix) == stay) {
            prefix -= 1;        // not 0: some bit was set
            wanted = 0;
        }
    } else if (stay > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = threadIdx.x; i < 256; i += kThreads) bins[i] = 0;
            __syncthreads();
            for (int c = threadIdx.x; c < candidates; c += kThreads) {
                const uint32_t k = keys[c];
                if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&bins[(k >> shift) & 255], 1u);
            }
            __syncthreads();
            if (warp == 0) {   // bins from the top, eight a lane
                uint32_t mine8 = 0;
                for (int i = 0; i < 8; ++i) mine8 += bins[255 - (lane * 8 + i)];
                uint32_t upto = mine8;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const uint32_t u = __shfl_up_sync(0xffffffffu, upto, d);
                    if (lane >= d) upto += u;
                }
                uint32_t above = upto - mine8;
                if (above < wanted && upto >= wanted) {
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t n = bins[255 - (lane * 8 + i)];
                        if (above + n >= wanted) {
                            found[0] = prefix | uint32_t(255 - (lane * 8 + i)) << shift;
                            found[1] = wanted - above;
                            break;
                        }
                        above += n;
                    }
                }
            }
            __syncthreads();
            prefix = found[0];
            wanted = found[1];
        }
    }
    // heavier than `prefix` stays, and the first `wanted` of those that weigh just that

    // ---- the list closes up
    int32_t *stack = a.free_pages + height + e.to;
    int stayed = 0, tied = 0;   // among the candidates before this round
    for (int c0 = 0; c0 < candidates; c0 += kThreads) {
        const int c = c0 + int(threadIdx.x);
        const bool here = c < candidates;
        const uint32_t k = here ? keys[c] : 0;
        const int page = here ? list[c] : 0;
        const bool more = here && stay > 0 && k > prefix, tie = here && stay > 0 && k == prefix;
        const unsigned more_mask = __ballot_sync(0xffffffffu, more), tie_mask = __ballot_sync(0xffffffffu, tie);
        if (lane == 0) part[warp] = uint32_t(__popc(more_mask)) | uint32_t(__popc(tie_mask)) << 16;
        __syncthreads();
        uint32_t before = 0, all = 0;
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += part[w];
            all += part[w];
        }
        __syncthreads();   // every entry of this round has been read: the list may be written in place
        const unsigned below = (1u << lane) - 1;
        const int more_before = int(before & 0xffff) + __popc(more_mask & below);
        const int ties_before = tied + int(before >> 16) + __popc(tie_mask & below);
        const int rank = stayed + more_before + min(ties_before, int(wanted)) - min(tied, int(wanted));
        const bool stays = more || (tie && ties_before < int(wanted));
        if (here) {
            if (stays) out[rank] = page;
            else stack[c - rank] = page < 0 || page >= a.num_pool_pages ? -1 : page;
        }
        const int ties = int(all >> 16);
        stayed += int(all & 0xffff) + min(tied + ties, int(wanted)) - min(tied, int(wanted));
        tied += ties;
    }
    // the newest pages follow; then nothing, up to what was held
    for (int c0 = 0; c0 < e.recent; c0 += kThreads) {
        const int c = c0 + int(threadIdx.x);
        const int page = c0 == 0 ? newest : c < e.recent ? list[candidates + c] : 0;
        __syncthreads();
        if (c < e.recent) out[stay + c] = page;
    }
    __syncthreads();
    for (int i = e.budget + int(threadIdx.x); i < e.room; i += kThreads) {
        if (i < e.pages) out[i] = -1;
        else if (out != list) out[i] = list[i];
    }
}

bool misaligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }
size_t layout(EvictArgs &a, void *scratch)
{
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off = (off + bytes + 15) / 16 * 16; return static_cast<unsigned char *>(scratch) + at; };
    a.height = reinterpret_cast<int32_t *>(take(4));
    a.plan = reinterpret_cast<EvictSample *>(take(sizeof(EvictSample) * size_t(a.num_samples)));
    a.keys = reinterpret_cast<uint32_t *>(take(4 * size_t(a.num_entries)));
    return off;
}

// Whether an output lies over an input or another output, but for the three that may be updated in place.
bool overlapping(const EvictArgs &a)
{
    struct Range { const void *p; int64_t bytes; };
    const int64_t lens = 4 * int64_t(a.num_samples), list = 4 * a.num_entries;
    const Range in[] = {{a.page_indices, list}, {a.kv_lens, lens}, {a.free_count, 4}, {a.budgets, lens}, {a.page_indptr, lens + 4},
                        {a.weights, 4 * int64_t(a.num_pool_pages) * a.cells}};
    const Range out[] = {{a.indices_out, list}, {a.lens_out, lens}, {a.free_count_out, 4}, {a.free_pages, 4 * a.free_capacity}};
    auto meet = [](const Range &x, const Range &y) {
        const uintptr_t u = reinterpret_cast<uintptr_t>(x.p), v = reinterpret_cast<uintptr_t>(y.p);
        return x.p && y.p && x.bytes > 0 && y.bytes > 0 && u < v + uintptr_t(y.bytes) && v < u + uintptr_t(x.bytes);
    };
    for (int o = 0; o < 4; ++o) {
        for (int i = 0; i < 6; ++i)
            if (meet(out[o], in[i]) && !(o == i && o < 3 && out[o].p == in[i].p)) return true;
        for (int p = 0; p < o; ++p)
            if (meet(out[o], out[p])) return true;
    }
    return false;
}

}  // namespace
}  // namespace psa

extern "C" size_t psa_evict_pages_scratch_bytes(int32_t num_samples, int64_t num_entries)
{
    if (num_samples < 0 || num_entries < 0 || num_entries > psa::kMostChunkEntries) return 0;
    psa::EvictArgs a{};
    a.num_samples = num_samples; a.num_entries = num_entries;
    return psa::layout(a, nullptr);
}

extern "C" psa_status_t psa_evict_pages(const float *weights, int64_t num_pool_pages, int32_t num_kv_heads, const int32_t *page_indptr,
                                        const int32_t *page_indices, int64_t num_entries, const int32_t *kv_lens, const int32_t *budgets,
                                        int32_t num_samples, int32_t recent, int32_t *free_pages, int64_t free_capacity, const int32_t *free_count,
                                        int32_t *page_indices_out, int32_t *lens_out, int32_t *free_count_out, int32_t *status, void *scratch,
                                        size_t scratch_bytes, void *cuda_stream)
{
    using namespace psa;
    if (num_pool_pages < 0 || num_kv_heads <= 0 || num_entries < 0 || num_samples < 0 || free_capacity < 0)
        return set_last_error(PSA_ERR_INVALID_ARG, "negative sizes or no KV head");
    if (recent < 1) return set_last_error(PSA_ERR_INVALID_ARG, "at least the newest page stays: recent >= 1");
    if (num_samples > (1 << 20) || num_kv_heads > 65536 || num_pool_pages > kMostChunkPages || num_entries > kMostChunkEntries || free_capacity > kMostChunkEntries)
        return set_last_error(PSA_ERR_UNSUPPORTED, "at most 2^20 samples, 2^16 heads, 2^27 pages, 2^31 - 256 list entries");
    if (misaligned(status, 4)) return set_last_error(PSA_ERR_INVALID_ARG, "the status word must be 4-byte aligned");
    if (!free_count || !free_count_out || !page_indptr || (num_entries > 0 && (!page_indices || !page_indices_out)) || (free_capacity > 0 && !free_pages) ||
        (num_samples > 0 && (!kv_lens || !budgets)) || (num_pool_pages > 0 && !weights))
        return set_last_error(PSA_ERR_INVALID_ARG, "null eviction argument");
    if (misaligned(weights, 16)) return set_last_error(PSA_ERR_INVALID_ARG, "weights must be 16-byte aligned");
    if (!scratch || misaligned(scratch, 16) || scratch_bytes < psa_evict_pages_scratch_bytes(num_samples, num_entries))
        return set_last_error(PSA_ERR_WORKSPACE, "scratch must be 16-byte aligned and hold psa_evict_pages_scratch_bytes");
    EvictArgs a{};
    a.weights = weights; a.page_indptr = page_indptr; a.page_indices = page_indices; a.kv_lens = kv_lens; a.budgets = budgets;
    a.free_count = free_count; a.indices_out = page_indices_out; a.lens_out = lens_out; a.free_pages = free_pages;
    a.free_count_out = free_count_out; a.status = status; a.num_entries = num_entries; a.free_capacity = free_capacity;
    a.num_samples = num_samples; a.recent = recent; a.num_pool_pages = int32_t(num_pool_pages); a.cells = num_kv_heads * kPageSize;
    if (overlapping(a)) return set_last_error(PSA_ERR_INVALID_ARG, "outputs must not overlap inputs or one another, but for the three updated in place");
    layout(a, scratch);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e;
    // one launch where no block writes what another one reads, and reading all samples' entries in every block is little
    if (num_samples > 0 && num_samples <= kAlone && lens_out != kv_lens && free_count_out != free_count) {
        evict_kernel<false><<<num_samples, kThreads, 0, st>>>(a);
        e = cudaGetLastError();
    } else {
        evict_plan_kernel<<<1, kPlanThreads, 0, st>>>(a);
        e = cudaGetLastError();
        if (e == cudaSuccess) e = launch_dependent(evict_kernel<true>, dim3(std::max(1, num_samples)), kThreads, 0, st, a);
    }
    if (e != cudaSuccess) return set_last_error(PSA_ERR_CUDA, std::string("eviction launch: ") + cudaGetErrorString(e));
    return PSA_OK;
}
