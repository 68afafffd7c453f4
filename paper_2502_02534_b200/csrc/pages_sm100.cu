// Page tables and slot maps built on the device from request lengths.
//
// A sample s that holds S_s tokens and gets N_s new ones needs the pages ceil(S_s / 16) .. ceil((S_s + N_s) / 16) - 1 of
// its list.  Pages come off a caller-owned stack in sample order: with need_s = the number of those pages and
// P_s = sum of need over the samples before s, list entry j of sample s receives free_pages[count - 1 - (P_s + j - j0)].
// Token i of sample s lands in slot page(pos / 16) * 16 + pos % 16, pos = S_s + i, and stands at token_indptr[s] + i of
// the packed batch.  Everything is therefore three exclusive scans over the samples (tokens, list entries, pages) and
// then one independent lookup per token and per list entry.
//
//   scan phase     one thread per sample, 1024 samples per block.  A block gets its starting sums by reducing the samples
//                  before its own itself: no block waits for another one, and at the sizes of a decode batch (one to a
//                  few blocks) that costs a few loads.
//   spread phase   a warp takes a run of pieces of up to kSpread tokens and finds the samples of a piece's first and last token
//                  by a 32-way search over the scanned offsets (two rounds for 1024 samples), the first one only where the
//                  sample of the piece before has ended.  A few long samples are walked one after the other with everything
//                  about them in registers, their pages one a lane; many short ones are looked up lane by lane.
//
// Bound: 8 bytes written per token of capacity once there are many, the latency of a few dependent loads when there are few.  The
// two phases are one launch of one block, with the offsets in shared memory, up to kOneBlockWork lookups; two launches above it.
// Measured: 256 samples x 1 token 5.5 us, an empty launch being about 2; 2048 samples x U[0, 4096] tokens, capacity 8.4 million, 19.5 us
// for 70 MB (3.6 TB/s; a plain fill of as many bytes takes 10.5, the scan before it 5).  Pieces dealt out in turn instead of in runs
// cost a search each: 22.4 us.  Every block scanning up to 2048 samples for itself, without the launch before it: 27 us, and 13.9
// instead of 10.7 us for 2048 samples x 1 token.
// Every scan block sums the samples before its own, so very many samples cost the square of their number: 16384 x 1 token 23 us, 65536 62,
// 262144 275, 2^20 2830.
#include <cuda_runtime.h>

#include <algorithm>
#include <string>
#include <type_traits>

#include "psa_internal.h"

namespace psa {
namespace {

constexpr int kScanThreads = 1024;
constexpr int kSpread = 256;                 // most tokens or list entries a warp handles at a time
static_assert(kSpread / kPageSize < 32, "a warp holds the pages of a piece, one a lane");
constexpr int64_t kMostEntries = 0x7fffff00; // 32-bit positions, with room for one more stride of a loop
constexpr int kWalk = 8;                     // samples in such a piece that are walked one after the other
constexpr int64_t kOneBlockWork = 4096;      // one block: 1024 samples x 4 tokens 8.7 us, 2048 x 4 15.1; two launches 9.7 and 10.8
constexpr int kOneBlockSamples = 1024;

struct PageTableArgs {
    const int32_t *held;       // null: nothing is held yet (a table built from scratch)
    const int32_t *new_lens;
    const int32_t *limits;     // reserve_lens (build) / max_lens (extend), may be null
    int32_t num_samples;
    const int32_t *free_pages, *free_count;
    int32_t *free_count_out;
    int32_t *page_indptr;      // written when `build`, read otherwise
    int32_t *page_indices;
    int64_t num_entries;       // capacity of page_indices
    int32_t *token_indptr;
    int64_t *slot_map;
    int64_t max_tokens;        // capacity of slot_map
    int32_t *lens_out;         // may be null, may alias held / new_lens
    int32_t *status;           // may be null
    // scratch: head[0] = {pages on the stack, -}; rec[s] = {held, first page's rank on the stack or -1 (refused)};
    // block_used[b] = pages handed out up to and including the last served sample of scan block b
    int2 *head;
    int2 *rec;
    int32_t *block_used;
    int32_t scan_blocks;
    bool build;
};

// Where the spread phase finds the scanned offsets and records: global memory, or shared memory in the one-block kernel.
struct Tables {
    const int32_t *token_indptr, *page_indptr;
    const int2 *rec;
};

struct Sums {
    long long tokens, entries, pages;
};

// What a sample asks for, apart from whether the arrays have room for it.
struct Ask {
    int32_t held, count;       // tokens it holds, tokens it gets (0 where the input is negative)
    int32_t entries;           // list entries it reserves (build)
    int32_t pages;             // pages it needs; 0 when it is refused already
    int32_t list;              // where its list starts (extend)
    bool ok;
};

__device__ __forceinline__ Ask ask(const PageTableArgs &a, int s)
{
    Ask r;
    const int32_t n = a.new_lens[s];
    r.held = a.held ? a.held[s] : 0;
    r.count = max(n, 0);
    r.list = 0;
    const long long end = (long long)(r.held) + r.count;
    r.ok = n >= 0 && r.held >= 0 && end <= 0x7fffffffll;
    if (a.build) {
        const int32_t reserve = a.limits ? max(a.limits[s], 0) : r.count;
        r.entries = int32_t(((long long)reserve + kPageSize - 1) / kPageSize);
        r.ok = r.ok && end <= reserve;
    } else {
        r.entries = 0;
        r.list = a.page_indptr[s];
        if (a.limits) r.ok = r.ok && (r.count == 0 || end <= a.limits[s]);
        const long long first = r.list, last = a.page_indptr[s + 1];
        r.ok = r.ok && (r.count == 0 || (first >= 0 && last <= a.num_entries && (end + kPageSize - 1) / kPageSize <= last - first));
        // a partly filled page must be in the list already (a negative id marks an entry without a page)
        if (r.ok && r.count > 0 && r.held % kPageSize != 0) r.ok = a.page_indices[first + r.held / kPageSize] >= 0;
    }
    r.pages = r.ok ? int32_t((end + kPageSize - 1) / kPageSize - ((long long)r.held + kPageSize - 1) / kPageSize) : 0;
    return r;
}

__device__ __forceinline__ long long warp_inclusive(long long v, int lane)
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    return v;
}
__device__ __forceinline__ long long warp_total(long long v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Samples [s0, s0 + 1024) with the sums of everything before them; returns the sums behind them.
// `copy` (shared memory, may be null) receives what the spread phase reads besides the output arrays.
struct TableCopy {
    int32_t *token_indptr, *page_indptr;
    int2 *rec;
};
__device__ Sums scan_chunk(const PageTableArgs &a, int s0, const Ask &q, const Sums &before, int avail, int *used_to, const TableCopy *copy)
{
    __shared__ long long warp_sums[3][32];
    __shared__ int block_used;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int s = s0 + int(threadIdx.x);
    const long long v[3] = {q.count, q.entries, q.pages};
    long long incl[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        incl[i] = warp_inclusive(v[i], lane);
        if (lane == 31) warp_sums[i][warp] = incl[i];
    }
    if (threadIdx.x == 0) block_used = 0;
    __syncthreads();
    if (warp < 3) warp_sums[warp][lane] = warp_inclusive(warp_sums[warp][lane], lane);
    __syncthreads();
    long long excl[3], total[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        excl[i] = (warp ? warp_sums[i][warp - 1] : 0) + incl[i] - v[i];
        total[i] = warp_sums[i][31];
    }
    if (s < a.num_samples) {
        const long long t0 = before.tokens + excl[0], e0 = before.entries + excl[1], p0 = before.pages + excl[2];
        bool ok = q.ok && t0 + q.count <= a.max_tokens;
        const int32_t e_cut = int32_t(min(e0, (long long)a.num_entries)), e_end = int32_t(min(e0 + q.entries, (long long)a.num_entries));
        const int32_t t_cut = int32_t(min(t0, (long long)a.max_tokens)), t_end = int32_t(min(t0 + q.count, (long long)a.max_tokens));
        ok = ok && (!a.build || e0 + q.entries <= a.num_entries) && (q.pages == 0 || p0 + q.pages <= avail);
        const int2 rec = make_int2(q.held, ok ? int32_t(min(p0, (long long)avail)) : -1);
        const bool end = s == a.num_samples - 1;
        a.token_indptr[s] = t_cut;
        if (end) a.token_indptr[s + 1] = t_end;
        if (a.build) {
            a.page_indptr[s] = e_cut;
            if (end) a.page_indptr[s + 1] = e_end;
        }
        if (copy) {
            copy->token_indptr[s] = t_cut;
            copy->page_indptr[s] = a.build ? e_cut : q.list;
            copy->rec[s] = rec;
            if (end) { copy->token_indptr[s + 1] = t_end; copy->page_indptr[s + 1] = a.build ? e_end : 0; }
        } else {
            a.rec[s] = rec;
        }
        if (ok && q.pages > 0) atomicMax(&block_used, int(p0 + q.pages));
        if (!ok && a.status) atomicCAS(a.status, 0, int(PSA_ERR_BOUNDS));
    }
    __syncthreads();
    *used_to = block_used;
    __syncthreads();
    return Sums{before.tokens + total[0], before.entries + total[1], before.pages + total[2]};
}

// Largest i in [lo, hi) with offsets[i] <= x; offsets ascend and offsets[lo] <= x.  All lanes of the warp search together.
__device__ __forceinline__ int warp_find(const int32_t *offsets, int lo, int hi, long long x, int lane)
{
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32;
        const int at = lo + lane * step;
        const bool below = at < hi && (lane == 0 || offsets[at] <= x);
        const int last = __popc(__ballot_sync(0xffffffffu, below)) - 1;
        lo += last * step;
        hi = min(hi, lo + step);
    }
    return lo;
}
__device__ __forceinline__ int lane_find(const int32_t *offsets, int lo, int hi, long long x)
{
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (offsets[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Pages of n >= 0 tokens; n may be the largest 32-bit number.
__device__ __forceinline__ int pages_of(int n) { return n / kPageSize + (n % kPageSize != 0); }

// Page of entry j of a sample's list (record rec, list at e_first); entries from `fresh` on come off the stack.
__device__ __forceinline__ int page_of(const PageTableArgs &a, int j, int fresh, int2 rec, int e_first, int avail)
{
    return j >= fresh ? a.free_pages[avail - 1 - (rec.y + j - fresh)] : a.page_indices[(long long)e_first + j];
}

// The sample that a warp's last token belonged to.  A warp takes its pieces in order, so a long sample is looked up once.
struct Here {
    int s = 0;
    int t_first = 0, t_next = -1;   // its tokens; an empty range before any other at first
    int e_first = 0;
    int2 rec{};
    __device__ __forceinline__ void load(const Tables &tab, int sample)
    {
        s = sample;
        t_first = tab.token_indptr[s];
        t_next = tab.token_indptr[s + 1];
        e_first = tab.page_indptr[s];
        rec = tab.rec[s];
    }
};

// Tokens [t0, t0 + piece) of the slot map, piece <= kSpread.
__device__ void spread_tokens(const PageTableArgs &a, const Tables &tab, long long t0, int piece, int avail, int lane, Here &at)
{
    const int n = a.num_samples;
    const int total = n > 0 ? tab.token_indptr[n] : 0;
    const int end = int(min(t0 + piece, (long long)a.max_tokens)), live = min(end, total);
    int t = int(t0);
    if (t < live) {
        if (t >= at.t_next) at.load(tab, warp_find(tab.token_indptr, at.s, n, t, lane));
        const int s_lo = at.s, s_hi = at.t_next >= live ? s_lo : warp_find(tab.token_indptr, s_lo, n, live - 1, lane);
        if (s_hi - s_lo < kWalk) {
            for (int s = s_lo; s <= s_hi; ++s) {
                if (s != s_lo) at.load(tab, s);
                const int2 rec = at.rec;
                const int t_first = at.t_first, stop = min(live, at.t_next), e_first = at.e_first;
                if (rec.y < 0) {
                    for (int i = t + lane; i < stop; i += 32) a.slot_map[i] = -1;
                } else if (t < stop) {
                    // the pages of up to kSpread tokens are fetched at once, one a lane, and go round by shuffles.  32 tokens further
                    // on are two pages further on, at the same place in the page.
                    const int len = stop - t, pos0 = rec.x + (t - t_first), j0 = pos0 / kPageSize, j1 = (pos0 + len - 1) / kPageSize;
                    const int fresh = pages_of(rec.x), j = j0 + lane;
                    const int page = j <= j1 ? page_of(a, j, fresh, rec, e_first, avail) : 0;
                    if (!a.build && j <= j1 && j >= fresh && j * kPageSize >= pos0)   // the piece that holds a fresh page's first token files it
                        a.page_indices[(long long)e_first + j] = page;
                    const int in_first = pos0 % kPageSize + lane, from = in_first / kPageSize, in_page = in_first % kPageSize;
                    int64_t *to = a.slot_map + t + lane;
                    if (len == kSpread && !__any_sync(0xffffffffu, page < 0)) {   // the middle of a long sample
#pragma unroll
                        for (int k = 0; k < kSpread / 32; ++k)
                            to[k * 32] = (long long)__shfl_sync(0xffffffffu, page, from + 2 * k) * kPageSize + in_page;
                    } else {
                        for (int k = 0; k * 32 < len; ++k) {
                            const int p = __shfl_sync(0xffffffffu, page, from + 2 * k);
                            if (k * 32 + lane < len) to[k * 32] = p >= 0 ? (long long)p * kPageSize + in_page : -1;
                        }
                    }
                }
                t = max(t, stop);
            }
        } else {
            for (int i0 = t; i0 < live; i0 += 4 * 32) {   // four lookups in flight per lane
                int page[4], in_page[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int i = i0 + k * 32 + lane;
                    page[k] = -1;
                    in_page[k] = 0;
                    if (i < live) {
                        const int s = lane_find(tab.token_indptr, s_lo, s_hi + 1, i);
                        const int2 rec = tab.rec[s];
                        if (rec.y >= 0) {
                            const int pos = rec.x + (i - tab.token_indptr[s]), j = pos / kPageSize, fresh = pages_of(rec.x);
                            const int e_first = tab.page_indptr[s];
                            in_page[k] = pos % kPageSize;
                            page[k] = page_of(a, j, fresh, rec, e_first, avail);
                            if (!a.build && j >= fresh && in_page[k] == 0) a.page_indices[(long long)e_first + j] = page[k];
                        }
                    }
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i0 + k * 32 + lane < live) a.slot_map[i0 + k * 32 + lane] = page[k] >= 0 ? (long long)page[k] * kPageSize + in_page[k] : -1;
            }
            t = live;
        }
    }
    int64_t *to = a.slot_map + t + lane;
    if (end - t == kSpread) {
#pragma unroll
        for (int k = 0; k < kSpread / 32; ++k) to[k * 32] = -1;
    } else {
        for (int i = t + lane; i < end; i += 32, to += 32) *to = -1;
    }
}

// Entries [e0, e0 + piece) of a list array built from scratch: the pages of the tokens held, -1 in the rest.
__device__ void spread_entries(const PageTableArgs &a, const Tables &tab, long long e0, int piece, int avail, int lane)
{
    const int n = a.num_samples;
    const int total = n > 0 ? tab.page_indptr[n] : 0;
    const int end = int(min(e0 + piece, (long long)a.num_entries)), live = min(end, total);
    auto entry = [&](int e, int s) {
        const int2 rec = tab.rec[s];
        const int j = e - tab.page_indptr[s], tokens = tab.token_indptr[s + 1] - tab.token_indptr[s];
        return rec.y >= 0 && j < pages_of(tokens) ? a.free_pages[avail - 1 - (rec.y + j)] : -1;
    };
    int e = int(e0);
    if (e < live) {
        const int s_lo = warp_find(tab.page_indptr, 0, n, e, lane), s_hi = warp_find(tab.page_indptr, s_lo, n, live - 1, lane);
        for (int i0 = e; i0 < live; i0 += 4 * 32) {   // four lookups in flight per lane
            int page[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = i0 + k * 32 + lane;
                page[k] = i < live ? entry(i, s_lo == s_hi ? s_lo : lane_find(tab.page_indptr, s_lo, s_hi + 1, i)) : -1;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i0 + k * 32 + lane < live) a.page_indices[i0 + k * 32 + lane] = page[k];
        }
        e = live;
    }
    for (int i = e + lane; i < end; i += 32) a.page_indices[i] = -1;
}

// Everything behind the scans, shared out over `warps` warps in pieces of `piece`.
__device__ void spread(const PageTableArgs &a, const Tables &tab, int piece, int avail, long long warp, long long warps, int lane)
{
    const long long token_pieces = (a.max_tokens + piece - 1) / piece, per_warp = (token_pieces + warps - 1) / warps;
    Here at;
    for (long long c = warp * per_warp, stop = min(c + per_warp, token_pieces); c < stop; ++c) spread_tokens(a, tab, c * piece, piece, avail, lane, at);
    // the last warps, whose tokens are the least likely to exist, begin with the list entries
    const long long entry_pieces = a.build ? (a.num_entries + piece - 1) / piece : 0;
    for (long long c = warps - 1 - warp; c < entry_pieces; c += warps) spread_entries(a, tab, c * piece, piece, avail, lane);
    if (a.lens_out)
        for (long long s = warp * 32 + lane; s < a.num_samples; s += warps * 32) {
            const int2 rec = tab.rec[s];
            a.lens_out[s] = rec.y >= 0 ? rec.x + (tab.token_indptr[s + 1] - tab.token_indptr[s]) : rec.x;
        }
}

// Small batches: both phases in one block.
__global__ void __launch_bounds__(kScanThreads)
page_table_one_block_kernel(PageTableArgs a)
{
    __shared__ int32_t tokens[kOneBlockSamples + 1], pages[kOneBlockSamples + 1];
    __shared__ int2 rec[kOneBlockSamples];
    const TableCopy copy{tokens, pages, rec};
    const int avail = max(*a.free_count, 0);
    Sums sums{0, 0, 0};
    int used = 0;
    for (int s0 = 0; s0 < a.num_samples; s0 += kScanThreads) {
        int u;
        const int s = s0 + int(threadIdx.x);
        sums = scan_chunk(a, s0, s < a.num_samples ? ask(a, s) : Ask{}, sums, avail, &u, &copy);
        used = max(used, u);
    }
    if (threadIdx.x == 0 && a.num_samples == 0) {
        a.token_indptr[0] = 0;
        if (a.build) a.page_indptr[0] = 0;
    }
    __syncthreads();   // also: every thread has read the stack's height before it is written, and the lengths before lens_out
    if (threadIdx.x == 0) *a.free_count_out = avail - used;
    const int piece = max(32, int((a.max_tokens + (a.build ? a.num_entries : 0)) / (kScanThreads / 32)));
    spread(a, Tables{tokens, pages, rec}, min(piece, kSpread), avail, threadIdx.x >> 5, kScanThreads / 32, threadIdx.x & 31);
}

__global__ void __launch_bounds__(kScanThreads)
page_table_scan_kernel(PageTableArgs a)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ long long part[3][32];
    const int avail = max(*a.free_count, 0);
    const int s0 = blockIdx.x * kScanThreads, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int own = s0 + int(threadIdx.x);
    const Ask asked = own < a.num_samples ? ask(a, own) : Ask{};   // under way together with the samples before
    Sums mine{0, 0, 0};
    for (int s = threadIdx.x; s < s0; s += kScanThreads) {
        const Ask q = ask(a, s);
        mine.tokens += q.count; mine.entries += q.entries; mine.pages += q.pages;
    }
    const long long w[3] = {warp_total(mine.tokens), warp_total(mine.entries), warp_total(mine.pages)};
    if (lane == 0) { part[0][warp] = w[0]; part[1][warp] = w[1]; part[2][warp] = w[2]; }
    __syncthreads();
    const Sums before{warp_total(part[0][lane]), warp_total(part[1][lane]), warp_total(part[2][lane])};
    int used;
    scan_chunk(a, s0, asked, before, avail, &used, nullptr);
    if (threadIdx.x == 0) {
        a.block_used[blockIdx.x] = used;
        if (blockIdx.x == 0) {
            a.head[0] = make_int2(avail, 0);
            if (a.num_samples == 0) {
                a.token_indptr[0] = 0;
                if (a.build) a.page_indptr[0] = 0;
            }
        }
    }
}

template <int kPiece>
__global__ void __launch_bounds__(256, 6)
page_table_spread_kernel(PageTableArgs a)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int avail = a.head[0].x;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        int used = 0;
        for (int b = 0; b < a.scan_blocks; ++b) used = max(used, a.block_used[b]);
        *a.free_count_out = avail - used;
    }
    spread(a, Tables{a.token_indptr, a.page_indptr, a.rec}, kPiece, avail, (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5), (long long)gridDim.x * (blockDim.x >> 5),
           threadIdx.x & 31);
}

int scan_blocks_of(int num_samples) { return std::max(1, (num_samples + kScanThreads - 1) / kScanThreads); }

psa_status_t run(PageTableArgs a, void *scratch, size_t scratch_bytes, void *cuda_stream)
{
    if (a.num_samples < 0 || a.max_tokens < 0 || a.num_entries < 0) return set_last_error(PSA_ERR_INVALID_ARG, "negative sizes");
    if (a.num_samples > (1 << 20)) return set_last_error(PSA_ERR_UNSUPPORTED, "at most 2^20 samples per call");
    if (a.max_tokens > kMostEntries || a.num_entries > kMostEntries)
        return set_last_error(PSA_ERR_UNSUPPORTED, "slot_map and page_indices hold at most 2^31 - 256 entries");
    if (!a.free_pages || !a.free_count || !a.free_count_out || !a.page_indptr || !a.token_indptr || (a.max_tokens > 0 && !a.slot_map) ||
        (a.num_entries > 0 && !a.page_indices) || (a.num_samples > 0 && !a.new_lens) || (!a.build && a.num_samples > 0 && !a.held))
        return set_last_error(PSA_ERR_INVALID_ARG, "null page table argument");
    if (reinterpret_cast<uintptr_t>(a.status) % 4) return set_last_error(PSA_ERR_INVALID_ARG, "the status word must be 4-byte aligned");
    if (!scratch || reinterpret_cast<uintptr_t>(scratch) % 8 || scratch_bytes < psa_page_table_scratch_bytes(a.num_samples))
        return set_last_error(PSA_ERR_WORKSPACE, "scratch must be 8-byte aligned and hold psa_page_table_scratch_bytes(num_samples)");
    a.head = static_cast<int2 *>(scratch);
    a.rec = a.head + 1;
    a.block_used = reinterpret_cast<int32_t *>(a.rec + a.num_samples);
    a.scan_blocks = scan_blocks_of(a.num_samples);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int64_t work = a.max_tokens + (a.build ? a.num_entries : 0);
    cudaError_t e;
    if (work <= kOneBlockWork && a.num_samples <= kOneBlockSamples) {
        page_table_one_block_kernel<<<1, kScanThreads, 0, st>>>(a);
        e = cudaGetLastError();
    } else {
        page_table_scan_kernel<<<a.scan_blocks, kScanThreads, 0, st>>>(a);
        e = cudaGetLastError();
        if (e == cudaSuccess) {
            // pieces small enough to keep the machine's warps busy: 8.9 million lookups take 19.5 us in pieces of 256 and 26 in 128,
            // 270 thousand 9.4 and 7.7, 8 thousand 15 and 12.4 (10.8 in 32)
            auto go = [&](auto piece) {
                const int64_t warps = (work + piece.value - 1) / piece.value;
                cudaLaunchConfig_t lc{};
                lc.gridDim = dim3(unsigned(std::max<int64_t>(1, std::min<int64_t>((warps + 7) / 8, 148 * 6))));
                lc.blockDim = dim3(256);
                lc.stream = st;
                cudaLaunchAttribute attr{};
                attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
                attr.val.programmaticStreamSerializationAllowed = 1;
                lc.attrs = &attr;
                lc.numAttrs = 1;
                return cudaLaunchKernelEx(&lc, page_table_spread_kernel<piece.value>, a);
            };
            if (work >= 2000000) e = go(std::integral_constant<int, kSpread>{});
            else if (work >= 65536) e = go(std::integral_constant<int, 128>{});
            else e = go(std::integral_constant<int, 32>{});
        }
    }
    if (e != cudaSuccess) return set_last_error(PSA_ERR_CUDA, std::string("page table launch: ") + cudaGetErrorString(e));
    return PSA_OK;
}

}  // namespace
}  // namespace psa

extern "C" size_t psa_page_table_scratch_bytes(int32_t num_samples)
{
    if (num_samples < 0) return 0;
    return 8 * (size_t(num_samples) + 1) + 4 * size_t(psa::scan_blocks_of(num_samples));
}

extern "C" psa_status_t psa_build_page_table(const int32_t *seq_lens, const int32_t *reserve_lens, int32_t num_samples,
                                             const int32_t *free_pages, const int32_t *free_count, int32_t *free_count_out,
                                             int32_t *page_indptr, int32_t *page_indices, int64_t num_entries, int32_t *token_indptr,
                                             int64_t *slot_map, int64_t max_tokens, int32_t *lens_out, int32_t *status, void *scratch,
                                             size_t scratch_bytes, void *cuda_stream)
{
    psa::PageTableArgs a{};
    a.new_lens = seq_lens; a.limits = reserve_lens; a.num_samples = num_samples;
    a.free_pages = free_pages; a.free_count = free_count; a.free_count_out = free_count_out;
    a.page_indptr = page_indptr; a.page_indices = page_indices; a.num_entries = num_entries;
    a.token_indptr = token_indptr; a.slot_map = slot_map; a.max_tokens = max_tokens;
    a.lens_out = lens_out; a.status = status; a.build = true;
    return psa::run(a, scratch, scratch_bytes, cuda_stream);
}

extern "C" psa_status_t psa_extend_page_table(const int32_t *held_lens, const int32_t *new_lens, const int32_t *max_lens,
                                              int32_t num_samples, const int32_t *free_pages, const int32_t *free_count,
                                              int32_t *free_count_out, const int32_t *page_indptr, int32_t *page_indices,
                                              int64_t num_entries, int32_t *token_indptr, int64_t *slot_map, int64_t max_tokens,
                                              int32_t *lens_out, int32_t *status, void *scratch, size_t scratch_bytes,
                                              void *cuda_stream)
{
    psa::PageTableArgs a{};
    a.held = held_lens; a.new_lens = new_lens; a.limits = max_lens; a.num_samples = num_samples;
    a.free_pages = free_pages; a.free_count = free_count; a.free_count_out = free_count_out;
    a.page_indptr = const_cast<int32_t *>(page_indptr); a.page_indices = page_indices; a.num_entries = num_entries;   // read only: build is false
    a.token_indptr = token_indptr; a.slot_map = slot_map; a.max_tokens = max_tokens;
    a.lens_out = lens_out; a.status = status; a.build = false;
    return psa::run(a, scratch, scratch_bytes, cuda_stream);
}
