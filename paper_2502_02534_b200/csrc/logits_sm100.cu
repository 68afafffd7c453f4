// Rules applied to logits before a token is drawn: penalties for repeated tokens, additive biases, grammar masks.
//
// For logit x of token i in row r, with c = how often i stands in the row's generated tokens:
//     x <- x > 0 ? x / repetition : x * repetition       if c > 0 or i is in the row's prompt set   (by 1 / repetition, rounded once)
//     x <- x - frequency * c - presence * [c > 0]
//     x <- x + (sum of the row's biases for i, added in list order)
//     x <- -inf                                          if the row's mask has bit i clear
// in fp32, rounded once to the output type.
//
// A row touches a few hundred of its many tokens through its lists (generated tokens, biases), all others only through the two
// bitmaps.  So the work is split:
//   lists    one block per row counts the generated tokens and adds up the biases in a hash table in shared memory, and works out the
//            logit of every token in it;
//   stream   every other logit: a thread takes eight consecutive ones, and one byte each of the prompt set and the mask tell what there
//            is to do.
// Three forms of it:
//   whole    vocabularies up to kWholeRow: the block that did a row's lists streams the row as well, before it writes the lists' logits.
//   two      the stream as a launch of its own, and the lists' launch behind it: that counts while the stream is still running and
//            writes its few logits over the stream's when that is done.
//   run      a block per row and run of 4 to 16 tiles picks the entries of its own tokens out of the row's lists, streams the run and writes
//            the lists' logits over it.  One launch, everything written where it was just read; but every block reads all the lists
//            and waits for them.  In place, for lists that the row's table does not take, and for many biases.
// Lists of more entries than the table takes are done tile by tile with a slot for every token (run), with a slot for every token of the row
// (whole), or in ranges of tokens whose entries the table takes (two).  The table of "two" is sized for the history and four times the mean
// number of biases, since its size costs every row; a row with more biases takes a few passes over its lists.
// Bound: HBM, one read and one write of every logit (and 2 bits).  Measured: 256 rows x 131072 bf16 logits, U[0, 1024] generated tokens and
// U[0, 64] biases each, 134.9 MB: two 28.2 us (31.3 over three sets of inputs in turn), run 40.0, in place 29.4; the stream alone 24.3, a
// plain copy 22.3.
// What the lists add is their latency, not their traffic: a table half full instead of a quarter 32.2 us, linear probing 38, 96 KB of
// table instead of 48 (fewer blocks beside the stream's) 33.9, stream blocks of 4 or 16 tiles instead of 8 33.7 and 34.5.
// 8 / 64 / 128 rows of that: two 6.9 / 10.0 / 14.2, run 6.6 / 10.5 / 18.2, in place 6.7 / 10.6 / 18.5; 256 rows with up to 3500 generated tokens
// each: two 52, run 79, in place 70.  8 rows x 3001: whole 3.9 us.
// Biases of one row alone, 256 rows, none / 1000 / 3000 / 8000 / 30000: two 20 / 54 / 100 / 318 / 2430, in place 16 / 18 / 30 / 257 / 795 us.  The
// same number in every row, no history, 128 / 256 / 512: two 23 / 28 / 36, run 31 / 29 / 32; 64 rows 7.2 / 10.7 / 16.4 and 8.6 / 8.1 / 9.2; 8 rows
// 5.8 / 9.2 / 14.8 and 4.9 / 4.5 / 4.9.  Whole rows of 8000 tokens, none / 1000 / 8000 biases in one row: 5 / 21 / 97.
// Tried for the largest case: lists by warps beside the streaming ones of a block 40-59 us; a resident stream of 5 blocks an SM with the
// lists beside it from the start 42; groups of rows streamed and followed by their lists 35-42; prefetching the lists into L2: no change.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <string>
#include <type_traits>

#include "psa_internal.h"

namespace psa {
namespace {

constexpr int kListThreads = 512;
constexpr int kStreamThreads = 256;
constexpr int kVec = 8;                                    // logits a thread handles together
constexpr int kStreamTile = kStreamThreads * kVec;         // logits a block of the stream takes at a time
constexpr int kStreamRun = 8, kStreamDepth = 4;            // tiles of a block; of them in flight
constexpr int kWholeRow = 8192;                            // vocabularies up to this are streamed by the row's own block
constexpr int kLog2Few = 11, kLog2Many = 13;                // sizes of the row's hash table
__host__ __device__ constexpr int64_t table_takes(int log2_slots) { return int64_t(1) << (log2_slots - 1); }   // entries: half full
constexpr int kFewBiases = 128;                            // more of them in a row are added up by the whole block, where it can
constexpr int kManyBiases = 256;                           // more of them a row on average: one launch
constexpr int kParts = 512;                                // of the vocabulary, whose entries are counted where there are too many for the table
constexpr int kOwn = 8;                                    // list entries a thread keeps in registers
constexpr int kLongHistory = kOwn * kListThreads;
constexpr int kThreads = 256, kTile = kThreads * kVec;     // one launch: threads of a block, logits it takes at a time,
constexpr int kLeastRun = 4, kMostRun = 16;                // tiles of it,
__host__ __device__ constexpr int run_depth(bool f32) { return f32 ? 3 : 4; }   // of them in flight
constexpr int run_bytes(bool f32) { return run_depth(f32) * kTile * (f32 ? 4 : 2); }
constexpr int kLog2RunSlots = 11, kRunSlots = 1 << kLog2RunSlots;   // its table, at most half full; also a slot for every token of a tile
constexpr int kHits = kRunSlots / 2 - 1;                   // list entries inside the run that the hash table takes
constexpr int kRunOwn = (kHits + kThreads - 1) / kThreads;
static_assert(kRunSlots == kTile && kMostRun * kTile <= 0x8000, "a slot for every token, 15 bits for a place in the run");
constexpr int kMarkTile = 131072;                          // tokens of one block's bitmap
constexpr int kMarkThreads = 1024;
constexpr int kMarkBatch = 8;

struct RulesArgs {
    psa_logits_rules_t r;
    const void *logits;
    void *out;
    int64_t row_stride, out_stride;
    int vocab;
    int log2_slots;       // of the largest table
    int run;              // tiles of a block
};

template <bool kF32>
struct Vec8;
template <>
struct Vec8<true> {
    float4 a, b;
    __device__ __forceinline__ void load(const void *base, int64_t i)
    {
        const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(base) + i);
        a = p[0]; b = p[1];
    }
    __device__ __forceinline__ void store(void *base, int64_t i) const
    {
        float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(base) + i);
        p[0] = a; p[1] = b;
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
        a = make_float4(x[0], x[1], x[2], x[3]); b = make_float4(x[4], x[5], x[6], x[7]);
    }
};
template <>
struct Vec8<false> {
    uint4 a;
    __device__ __forceinline__ void load(const void *base, int64_t i)
    {
        a = *reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(base) + i);
    }
    __device__ __forceinline__ void store(void *base, int64_t i) const
    {
        *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(base) + i) = a;
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<uint32_t *>(&v);
        }
        a = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <bool kF32>
__device__ __forceinline__ float load_one(const void *base, int64_t i)
{
    if constexpr (kF32) return static_cast<const float *>(base)[i];
    else return __bfloat162float(static_cast<const __nv_bfloat16 *>(base)[i]);
}
template <bool kF32>
__device__ __forceinline__ void store_one(void *base, int64_t i, float x)
{
    if constexpr (kF32) static_cast<float *>(base)[i] = x;
    else static_cast<__nv_bfloat16 *>(base)[i] = __float2bfloat16_rn(x);
}

// What a row needs besides its logits.
struct Row {
    float rep, inv_rep;
    const unsigned char *prompt, *mask;   // bitmaps, may be null
    __device__ Row(const RulesArgs &a, int row)
    {
        const float r = a.r.repetition ? a.r.repetition[row] : 1.f;
        rep = r > 0.f && r < INFINITY ? r : 1.f;   // not a penalty: off
        inv_rep = __fdiv_rn(1.f, rep);
        prompt = rep != 1.f ? bitmap(a.r.prompt_bits, a.r.prompt_row_words, a.r.num_prompt_bitmaps, a.r.prompt_rows, row) : nullptr;
        mask = bitmap(a.r.mask_bits, a.r.mask_row_words, a.r.num_mask_bitmaps, a.r.mask_rows, row);
    }
    static __device__ const unsigned char *bitmap(const uint32_t *bits, int64_t words, int count, const int32_t *rows, int row)
    {
        if (!bits) return nullptr;
        const int64_t p = rows ? rows[row] : row;
        return p >= 0 && p < count ? reinterpret_cast<const unsigned char *>(bits + p * words) : nullptr;
    }
    __device__ __forceinline__ static bool has(const unsigned char *bits, int i) { return (__ldg(bits + (i >> 3)) >> (i & 7)) & 1; }
    __device__ __forceinline__ float penalised(float x) const { return x * (x > 0.f ? inv_rep : rep); }
};

// two products at once
__device__ __forceinline__ void mul2(float &a, float &b, float x, float y, float f)
{
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %4};\n\tmul.rn.f32x2 p, p, q;\n\tmov.b64 {%0, %1}, p;\n\t}"
        : "=f"(a), "=f"(b) : "f"(x), "f"(y), "f"(f));
}
// The penalty for all eight logits.  With repetition above 1 both of its branches give the smaller one of x / repetition and
// x * repetition, below 1 the larger one: two products and a minimum, without a comparison.
template <bool kUp>
__device__ __forceinline__ void penalise8(float (&y)[8], const float (&x)[8], const Row &row)
{
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        float a0, a1, b0, b1;
        mul2(a0, a1, x[e], x[e + 1], row.inv_rep);
        mul2(b0, b1, x[e], x[e + 1], row.rep);
        y[e] = kUp ? fmaxf(a0, b0) : fminf(a0, b0);
        y[e + 1] = kUp ? fmaxf(a1, b1) : fminf(a1, b1);
    }
}
// Four bits to the top bits of the four bytes of a word: the shifted copies in the product do not overlap.
__device__ __forceinline__ uint32_t spread4(uint32_t nibble) { return nibble * 0x10204080u; }
// All ones in the 16-bit halves of a word whose bits among the eight of `lo` (bits 0-3) and `hi` (bits 4-7) are set: logits 2 p and
// 2 p + 1.  prmt with the top selector bit repeats a byte's sign.
template <int p>
__device__ __forceinline__ uint32_t halves(uint32_t lo, uint32_t hi)
{
    uint32_t m;
    asm("prmt.b32 %0, %1, 0, %2;" : "=r"(m) : "r"(p < 2 ? lo : hi), "n"(p % 2 ? 0xBBAA : 0x9988));
    return m;
}
__device__ __forceinline__ uint32_t blend(uint32_t mask, uint32_t set, uint32_t clear) { return (set & mask) | (clear & ~mask); }

// Eight consecutive logits that lie inside the row.  bf16 to bf16 stays packed: the selections are made on pairs.
template <bool kInF32, bool kOutF32, bool kUp>
__device__ __forceinline__ void stream8(const Row &row, void *out, int i, const Vec8<kInF32> &v, uint32_t seen, uint32_t allowed)
{
    float x[8];
    Vec8<kOutF32> o;
    if constexpr (!kInF32 && !kOutF32) {
        uint32_t w[4] = {v.a.x, v.a.y, v.a.z, v.a.w};
        if (row.prompt) {
            float y[8];
            v.get(x);
            penalise8<kUp>(y, x, row);
            o.set(y);
            const uint32_t lo = spread4(seen & 15u), hi = spread4(seen >> 4);
            w[0] = blend(halves<0>(lo, hi), o.a.x, w[0]);
            w[1] = blend(halves<1>(lo, hi), o.a.y, w[1]);
            w[2] = blend(halves<2>(lo, hi), o.a.z, w[2]);
            w[3] = blend(halves<3>(lo, hi), o.a.w, w[3]);
        }
        if (row.mask) {
            const uint32_t lo = spread4(allowed & 15u), hi = spread4(allowed >> 4), none = 0xFF80FF80u;   // - infinity twice
            w[0] = blend(halves<0>(lo, hi), w[0], none);
            w[1] = blend(halves<1>(lo, hi), w[1], none);
            w[2] = blend(halves<2>(lo, hi), w[2], none);
            w[3] = blend(halves<3>(lo, hi), w[3], none);
        }
        o.a = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        v.get(x);
        if (row.prompt) {
            float y[8];
            penalise8<kUp>(y, x, row);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = seen & (1u << e) ? y[e] : x[e];
        }
        if (row.mask) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = allowed & (1u << e) ? x[e] : -INFINITY;
        }
        o.set(x);
    }
    o.store(out, i);
}

// The last logits of a row whose vocabulary is not a multiple of eight, by one thread: neither read nor written beyond it.
template <bool kInF32, bool kOutF32>
__device__ __forceinline__ void stream_rest(const Row &row, const void *in, void *out, int vocab)
{
    for (int i = vocab & ~7; i < vocab; ++i) {
        float x = load_one<kInF32>(in, i);
        if (row.prompt && Row::has(row.prompt, i)) x = row.penalised(x);
        store_one<kOutF32>(out, i, row.mask && !Row::has(row.mask, i) ? -INFINITY : x);
    }
}

__device__ __forceinline__ const void *row_of(const void *p, int64_t stride, int row, bool f32)
{
    return static_cast<const unsigned char *>(p) + int64_t(row) * stride * (f32 ? 4 : 2);
}

// One block per (row, run of kStreamRun tiles).  A thread copies its own groups of the next kStreamDepth - 1 tiles ahead of itself into
// shared memory (cp.async), so that enough bytes are on their way without registers or barriers.
template <bool kInF32, bool kOutF32>
__global__ void __launch_bounds__(kStreamThreads)
rules_stream_kernel(RulesArgs a)
{
    constexpr int kBytes = kVec * (kInF32 ? 4 : 2);
    __shared__ __align__(16) unsigned char ring[kStreamDepth][kStreamThreads * kBytes];
    const int row = blockIdx.y;
    const int first = blockIdx.x * (kStreamRun * kStreamTile) + threadIdx.x * kVec;
    const int n = min(kStreamRun, ((a.vocab & ~7) - first + kStreamTile - 1) / kStreamTile);   // whole groups of this thread; may be <= 0
    const unsigned char *in = static_cast<const unsigned char *>(row_of(a.logits, a.row_stride, row, kInF32));
    void *out = const_cast<void *>(row_of(a.out, a.out_stride, row, kOutF32));
    asm volatile("griddepcontrol.wait;" ::: "memory");                // for whatever wrote the inputs
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the lists' launch may count beside this one
    auto request = [&](int t) {
        if (t < n) {
            const uint32_t to = uint32_t(__cvta_generic_to_shared(&ring[t % kStreamDepth][threadIdx.x * kBytes]));
            const unsigned char *from = in + int64_t(first + t * kStreamTile) * (kBytes / kVec);
#pragma unroll
            for (int c = 0; c < kBytes; c += 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + c), "l"(from + c) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int t = 0; t < kStreamDepth - 1; ++t) request(t);
    const Row r(a, row);
    uint32_t seen, allowed;
    auto bits = [&](int t) {
        const int at = (first + t * kStreamTile) >> 3;
        seen = r.prompt && t < n ? __ldg(r.prompt + at) : 0u;
        allowed = r.mask && t < n ? __ldg(r.mask + at) : 0u;
    };
    bits(0);
    auto work = [&](auto up) {
        for (int t = 0; t < n; ++t) {
            request(t + kStreamDepth - 1);
            const uint32_t s = seen, ok = allowed;
            bits(t + 1);
            asm volatile("cp.async.wait_group %0;" ::"n"(kStreamDepth - 1) : "memory");
            Vec8<kInF32> v;
            v.load(&ring[t % kStreamDepth][threadIdx.x * kBytes], 0);
            stream8<kInF32, kOutF32, up.value>(r, out, first + t * kStreamTile, v, s, ok);
        }
    };
    if (r.rep < 1.f) work(std::true_type{});
    else work(std::false_type{});
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) stream_rest<kInF32, kOutF32>(r, in, out, a.vocab);
}

// Where a token's counters are: hashed with linear probing (the table is never full), or directly at id - r0.
struct Table {
    int32_t *key, *count;
    float *value;
    int log2_slots, r0, r1;   // tokens [r0, r1) belong to the table
    bool hashed;
    __device__ __forceinline__ int slots() const { return 1 << log2_slots; }
    // slot of a token (-1: none of the table's); `mine`: the caller has brought it in
    __device__ __forceinline__ int add(int id, bool &mine) const
    {
        mine = false;
        if (id < r0 || id >= r1) return -1;
        if (!hashed) {
            key[id - r0] = id;
            return id - r0;
        }
        for (int h = int((uint32_t(id) * 2654435761u) >> (32 - log2_slots)), k = 1;; h = (h + k++) & (slots() - 1)) {
            const int old = atomicCAS(key + h, -1, id);
            mine = old == -1;
            if (mine || old == id) return h;
        }
    }
    __device__ __forceinline__ void clear(int tid, int threads) const   // slots() is a multiple of 4
    {
        for (int h = tid; h < slots() / 4; h += threads) {
            reinterpret_cast<int4 *>(key)[h] = make_int4(-1, -1, -1, -1);
            reinterpret_cast<int4 *>(count)[h] = make_int4(0, 0, 0, 0);
            reinterpret_cast<float4 *>(value)[h] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
    __device__ __forceinline__ int find(int id) const   // of a token that has been added
    {
        if (id < r0 || id >= r1) return -1;
        if (!hashed) return id - r0;
        int h = int((uint32_t(id) * 2654435761u) >> (32 - log2_slots));
        for (int k = 1; key[h] != id; ++k) h = (h + k) & (slots() - 1);
        return h;
    }
};

// Hands every id of a list to one of the block's threads, which has four reads in flight; -1 behind the list.
template <int kBlock, class Take>
__device__ __forceinline__ void for_all(const int32_t *ids, int n, Take take)
{
    for (int e0 = threadIdx.x; e0 < n; e0 += 4 * kBlock) {
        int id[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) id[k] = e0 + k * kBlock < n ? ids[e0 + k * kBlock] : -1;
#pragma unroll
        for (int k = 0; k < 4; ++k) take(id[k]);
    }
}

// Adds 32 biases to their tokens' values, by one warp; at: slot of a lane's token, -1 for none.  Equal tokens are summed by the first lane
// that has them, so the order of the additions is that of the lanes.
__device__ __forceinline__ void add_32(const Table &t, int at, float v, int lane)
{
    const uint32_t same = __match_any_sync(0xffffffffu, at);
    const bool leader = at >= 0 && (__ffs(same) - 1) == lane;
    float sum = leader ? t.value[at] : 0.f;
    // every lane takes part in the shuffles; at most 32 rounds, one without duplicates
    uint32_t rest = at >= 0 ? same : 0u;
    while (__any_sync(0xffffffffu, rest != 0u)) {
        const int from = rest ? __ffs(rest) - 1 : 0;
        const float u = __shfl_sync(0xffffffffu, v, from);
        if (rest) sum += u;
        rest &= rest - 1u;
    }
    if (leader) t.value[at] = sum;
    __syncwarp();
}
// Adds a row's biases to their tokens' values in list order, by one warp.
__device__ void add_biases(const int32_t *ids, const float *values, int n, const Table &t, int lane)
{
    for (int e0 = 0; e0 < n; e0 += 32) {
        const int e = e0 + lane;
        const int at = e < n ? t.find(ids[e]) : -1;
        const float v = e < n ? values[e] : 0.f;
        add_32(t, at, v, lane);
    }
}
// The same by a whole block, for long lists: the entries that concern the table are brought together in list order, so that the warp that
// adds them up meets no others and does not wait for memory.  The caller synchronises the block before and after it.
template <int kBlock>
struct Together {   // in shared memory that is free meanwhile
    float value[kBlock];
    uint16_t slot[kBlock];
    int32_t count[kBlock / 32];
};
template <int kBlock>
__device__ __forceinline__ void add_many_biases(const int32_t *ids, const float *values, int n, const Table &t, Together<kBlock> &to)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int id = tid < n ? ids[tid] : -1;
    float v = tid < n ? values[tid] : 0.f;
    for (int e0 = 0; e0 < n; e0 += kBlock) {
        const int at = t.find(id);
        const float mine = v;
        const int next = e0 + kBlock + tid;
        id = next < n ? ids[next] : -1;
        v = next < n ? values[next] : 0.f;
        const uint32_t have = __ballot_sync(0xffffffffu, at >= 0);
        if (lane == 0) to.count[warp] = __popc(have);
        __syncthreads();   // also: the warp that adds is done with the entries before
        int before = 0, total = 0;
        for (int w = 0; w < kBlock / 32; ++w) {
            before += w < warp ? to.count[w] : 0;
            total += to.count[w];
        }
        if (at >= 0) {
            const int i = before + __popc(have & ((1u << lane) - 1u));
            to.slot[i] = uint16_t(at);
            to.value[i] = mine;
        }
        __syncthreads();
        if (warp == 0)
            for (int i = lane; i - lane < total; i += 32) add_32(t, i < total ? int(to.slot[i]) : -1, i < total ? to.value[i] : 0.f, lane);
    }
}

template <bool kInF32, bool kOutF32, bool kWhole>
__global__ void __launch_bounds__(kListThreads, kWhole ? 2 : 3)
rules_lists_kernel(RulesArgs a)
{
    extern __shared__ __align__(16) int32_t table_smem[];
    const int row = blockIdx.x, tid = threadIdx.x;
    // Behind a stream: that has waited for the inputs and does not write them; only this kernel's writes have to wait for it.
    if (kWhole) asm volatile("griddepcontrol.wait;" ::: "memory");
    const void *in = row_of(a.logits, a.row_stride, row, kInF32);
    void *out = const_cast<void *>(row_of(a.out, a.out_stride, row, kOutF32));
    const int32_t *said = a.r.history ? a.r.history + int64_t(row) * a.r.history_stride : nullptr;
    const int n_said = said ? max(0, min(a.r.history_lens[row], a.r.history_capacity)) : 0;
    int b0 = 0, n_bias = 0;
    if (a.r.bias_indptr) {
        b0 = max(0, a.r.bias_indptr[row]);
        n_bias = max(0, min(a.r.num_biases, a.r.bias_indptr[row + 1]) - b0);
    }
    const Row r(a, row);
    const float freq = a.r.frequency ? a.r.frequency[row] : 0.f;
    const float pres = a.r.presence ? a.r.presence[row] : 0.f;
    Vec8<kInF32> v[kWhole ? kWholeRow / kVec / kListThreads : 1];
    if constexpr (kWhole) {
#pragma unroll
        for (int k = 0; k < kWholeRow / kVec / kListThreads; ++k) {
            const int i = (k * kListThreads + tid) * kVec;
            if (i + kVec <= a.vocab) v[k].load(in, i);
        }
    }
    // everything but the lists' tokens, whose logits have been read by then
    auto rest = [&] {
        if constexpr (kWhole) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kWholeRow / kVec / kListThreads; ++k) {
                const int i = (k * kListThreads + tid) * kVec;
                if (i + kVec > a.vocab) continue;
                const uint32_t seen = r.prompt ? __ldg(r.prompt + (i >> 3)) : 0u, allowed = r.mask ? __ldg(r.mask + (i >> 3)) : 0u;
                if (r.rep < 1.f) stream8<kInF32, kOutF32, true>(r, out, i, v[k], seen, allowed);
                else stream8<kInF32, kOutF32, false>(r, out, i, v[k], seen, allowed);
            }
            if (tid == 0) stream_rest<kInF32, kOutF32>(r, in, out, a.vocab);
            __syncthreads();
        } else {
            asm volatile("griddepcontrol.wait;" ::: "memory");
        }
    };

    // the smallest table that stays half empty, or all there is, indexed directly
    const uint32_t entries = uint32_t(n_said) + uint32_t(n_bias);
    Table t;
    t.log2_slots = max(9, entries > 1u ? 33 - __clz(entries - 1u) : 0);
    if (t.log2_slots < a.log2_slots) ++t.log2_slots;   // a quarter full, where there is room
    t.hashed = entries <= kLongHistory && t.log2_slots <= a.log2_slots;
    if (!t.hashed) t.log2_slots = a.log2_slots;
    t.key = table_smem; t.count = t.key + t.slots(); t.value = reinterpret_cast<float *>(t.count + t.slots());
    // logit x of a token that stands in the lists c times, apart from its biases
    auto ruled = [&](float x, int c, bool in_prompt) {
        if (c > 0 || in_prompt) x = r.penalised(x);
        return c > 0 ? x - freq * float(c) - pres : x;
    };
    if (t.hashed) {
        // At most kOwn entries a thread.  The thread that brings a token into the table reads its logit and bits at once and keeps
        // them in registers, with the other entries' reads and with the biases still under way.
        t.r0 = 0; t.r1 = a.vocab;
        int id[kOwn], at[kOwn];
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            const int e = tid + k * kListThreads;
            id[k] = -1;
            if (k * kListThreads < int(entries) && e < int(entries)) id[k] = e < n_said ? said[e] : a.r.bias_ids[b0 + e - n_said];
        }
        t.clear(tid, kListThreads);
        __syncthreads();
        float x[kOwn];
        uint32_t in_prompt = 0u, allowed = ~0u;   // a bit per k
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            at[k] = -1;
            if (k * kListThreads >= int(entries)) continue;
            bool mine;
            const int h = t.add(id[k], mine);
            if (h >= 0 && tid + k * kListThreads < n_said) atomicAdd(t.count + h, 1);
            if (mine) {
                at[k] = h;
                x[k] = load_one<kInF32>(in, id[k]);
                if (r.prompt && Row::has(r.prompt, id[k])) in_prompt |= 1u << k;
                if (r.mask && !Row::has(r.mask, id[k])) allowed &= ~(1u << k);
            }
        }
        __syncthreads();
        if (n_bias > 0) {   // the same for the whole block
            if (tid < 32) add_biases(a.r.bias_ids + b0, a.r.bias_values + b0, n_bias, t, tid);
            __syncthreads();
        }
        rest();
#pragma unroll
        for (int k = 0; k < kOwn; ++k)
            if (at[k] >= 0)
                store_one<kOutF32>(out, id[k], allowed & (1u << k) ? ruled(x[k], t.count[at[k]], in_prompt & (1u << k)) + t.value[at[k]] : -INFINITY);
    } else {
        // what the table has come to: its tokens' logits, written when the stream is done with theirs
        auto finish = [&] {
            for (int h = tid; h < t.slots(); h += kListThreads) {
                const int token = t.key[h];
                if (token < 0) continue;
                const float x = ruled(load_one<kInF32>(in, token), t.count[h], r.prompt && Row::has(r.prompt, token));
                t.value[h] = !r.mask || Row::has(r.mask, token) ? x + t.value[h] : -INFINITY;
            }
            rest();
            for (int h = tid; h < t.slots(); h += kListThreads)
                if (t.key[h] >= 0) store_one<kOutF32>(out, t.key[h], t.value[h]);
        };
        if constexpr (kWhole) {
            t.r0 = 0; t.r1 = a.vocab;
            t.clear(tid, kListThreads);
            __syncthreads();
            bool mine;
            for (int e = tid; e < n_said; e += kListThreads) {
                const int h = t.add(said[e], mine);
                if (h >= 0) atomicAdd(t.count + h, 1);
            }
            for (int e = tid; e < n_bias; e += kListThreads) t.add(a.r.bias_ids[b0 + e], mine);
            __syncthreads();
            if (n_bias > 0) {
                if (tid < 32) add_biases(a.r.bias_ids + b0, a.r.bias_values + b0, n_bias, t, tid);
                __syncthreads();
            }
            finish();
        } else {
            // Ranges of as many neighbouring parts of the vocabulary as the table takes the entries of, so about entries / most passes over
            // the lists, where a slot for every token would need vocab / slots of them.  Half of the table, three quarters full; the other half of
            // the memory holds what else is needed.
            --t.log2_slots;
            t.count = t.key + t.slots(); t.value = reinterpret_cast<float *>(t.count + t.slots());
            const int most = t.slots() / 4 * 3;
            int *in_part = reinterpret_cast<int *>(t.value + t.slots());
            auto &to = *reinterpret_cast<Together<kListThreads> *>(in_part + kParts);
            static_assert(4 * kParts + sizeof(to) <= (12 << kLog2Few) / 2 && kParts <= kListThreads, "in the other half");
            int log2_part = t.log2_slots;
            while ((a.vocab - 1) >> log2_part >= kParts) ++log2_part;
            const int parts = ((a.vocab - 1) >> log2_part) + 1;
            if (tid < kParts) in_part[tid] = 0;
            __syncthreads();
            auto tally = [&](int id) {
                if (id >= 0 && id < a.vocab) atomicAdd(in_part + (id >> log2_part), 1);
            };
            for_all<kListThreads>(said, n_said, tally);
            for_all<kListThreads>(a.r.bias_ids + b0, n_bias, tally);
            __syncthreads();
            // a part that alone has more entries gets a slot for every token, as many tokens at a time as there are slots
            for (int p = 0, q, r0 = 0, r1; p < parts; p = q, r0 = r1) {
                int sum = in_part[p];
                for (q = p + 1; q < parts && sum + in_part[q] <= most; ++q) sum += in_part[q];
                r0 = max(r0, p << log2_part);
                r1 = min(a.vocab, q << log2_part);
                if (sum > most && r1 - r0 > t.slots()) { r1 = r0 + t.slots(); q = p; }
                if (sum == 0) continue;
                t.r0 = r0; t.r1 = r1; t.hashed = sum <= most;
                t.clear(tid, kListThreads);
                __syncthreads();
                bool mine;
                for_all<kListThreads>(said, n_said, [&](int id) {
                    const int h = t.add(id, mine);
                    if (h >= 0) atomicAdd(t.count + h, 1);
                });
                for_all<kListThreads>(a.r.bias_ids + b0, n_bias, [&](int id) { t.add(id, mine); });
                __syncthreads();
                if (n_bias > 0) {
                    add_many_biases<kListThreads>(a.r.bias_ids + b0, a.r.bias_values + b0, n_bias, t, to);
                    __syncthreads();
                }
                finish();
                __syncthreads();
            }
            rest();   // where no entry is a token's: this grid must not end before the stream has
        }
    }
}

// One block per (row, run of a.run tiles).  A thread copies its own groups of the next kDepth - 1 tiles ahead of itself into shared memory
// (cp.async), so that enough bytes are on their way without registers or barriers.
template <bool kInF32, bool kOutF32>
__global__ void __launch_bounds__(kThreads, 4)
rules_run_kernel(RulesArgs a)
{
    constexpr int kBytes = kVec * (kInF32 ? 4 : 2), kDepth = run_depth(kInF32);
    extern __shared__ __align__(16) unsigned char ring[];   // [kDepth][kThreads * kBytes]
    __shared__ __align__(16) int32_t keys[kRunSlots], counts[kRunSlots];
    __shared__ __align__(16) float values[kRunSlots];
    __shared__ __align__(16) uint16_t hits[kHits];   // the run's list entries: token - c0, and whether it is a bias
    auto &to = *reinterpret_cast<Together<kThreads> *>(hits);   // once they have been read
    static_assert(sizeof(to) <= sizeof hits, "in its place");
    __shared__ int num_hits;
    const int row = blockIdx.y, tid = threadIdx.x;
    const int c0 = blockIdx.x * (a.run * kTile), c1 = min(a.vocab, c0 + a.run * kTile), tiles = (c1 - c0 + kTile - 1) / kTile;
    const int first = c0 + tid * kVec, whole = a.vocab & ~7;
    const void *in = row_of(a.logits, a.row_stride, row, kInF32);
    void *out = const_cast<void *>(row_of(a.out, a.out_stride, row, kOutF32));
    if (tid == 0) num_hits = 0;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    auto request = [&](int t) {
        const int i = first + t * kTile;
        if (t < tiles && i < whole) {
            const uint32_t to = uint32_t(__cvta_generic_to_shared(ring + (t % kDepth * kThreads + tid) * kBytes));
            const unsigned char *from = static_cast<const unsigned char *>(in) + int64_t(i) * (kBytes / kVec);
#pragma unroll
            for (int c = 0; c < kBytes; c += 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + c), "l"(from + c) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int t = 0; t < kDepth - 1; ++t) request(t);
    const Row r(a, row);
    const int32_t *said = a.r.history ? a.r.history + int64_t(row) * a.r.history_stride : nullptr;
    const int n_said = said ? max(0, min(a.r.history_lens[row], a.r.history_capacity)) : 0;
    int b0 = 0, n_bias = 0;
    if (a.r.bias_indptr) {
        b0 = max(0, a.r.bias_indptr[row]);
        n_bias = max(0, min(a.r.num_biases, a.r.bias_indptr[row + 1]) - b0);
    }
    uint32_t seen, allowed;
    auto bits = [&](int t) {
        const int i = first + t * kTile;
        const bool there = t < tiles && i < whole;
        seen = r.prompt && there ? __ldg(r.prompt + (i >> 3)) : 0u;
        allowed = r.mask && there ? __ldg(r.mask + (i >> 3)) : 0u;
    };
    bits(0);
    auto stream = [&](int t) {
        request(t + kDepth - 1);
        const uint32_t s = seen, ok = allowed;
        bits(t + 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
        const int i = first + t * kTile;
        if (i < whole) {
            Vec8<kInF32> v;
            v.load(ring + (t % kDepth * kThreads + tid) * kBytes, 0);
            if (r.rep < 1.f) stream8<kInF32, kOutF32, true>(r, out, i, v, s, ok);
            else stream8<kInF32, kOutF32, false>(r, out, i, v, s, ok);
        }
        if (t == tiles - 1 && c1 == a.vocab && tid == 0) stream_rest<kInF32, kOutF32>(r, in, out, a.vocab);
    };
    if (n_said + n_bias == 0) {   // the same for the whole block, as everything below
        for (int t = 0; t < tiles; ++t) stream(t);
        return;
    }

    const float freq = a.r.frequency ? a.r.frequency[row] : 0.f;
    const float pres = a.r.presence ? a.r.presence[row] : 0.f;
    // logit x of a token that stands in the lists c times, apart from its biases
    auto ruled = [&](float x, int c, bool in_prompt) {
        if (c > 0 || in_prompt) x = r.penalised(x);
        return c > 0 ? x - freq * float(c) - pres : x;
    };
    __syncthreads();   // num_hits
    bool biased = false;
    auto gather = [&](const int32_t *ids, int n, uint32_t flag) {
        for (int e0 = tid; e0 < n; e0 += 4 * kThreads) {
            int id[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) id[k] = e0 + k * kThreads < n ? ids[e0 + k * kThreads] : -1;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (id[k] >= c0 && id[k] < c1) {
                    const int at = atomicAdd(&num_hits, 1);
                    if (at < kHits) hits[at] = uint16_t(uint32_t(id[k] - c0) | flag);
                    biased = biased || flag != 0u;
                }
        }
    };
    gather(said, n_said, 0u);
    gather(a.r.bias_ids + b0, n_bias, 0x8000u);
    biased = __syncthreads_or(biased);
    const int n_hits = num_hits;
    Table t;
    t.key = keys; t.count = counts; t.value = values;
    if (n_hits <= kHits) {
        // The thread that brings a token into the table reads its logit and bits at once and keeps them in registers.
        t.hashed = true;
        t.log2_slots = min(kLog2RunSlots, max(6, 33 - __clz(2 * n_hits)));   // a quarter full, where there is room
        t.r0 = c0; t.r1 = c1;
        t.clear(tid, kThreads);
        __syncthreads();
        int id[kRunOwn], at[kRunOwn];
        float x[kRunOwn];
        uint32_t in_prompt = 0u, open = ~0u;   // a bit per k
#pragma unroll
        for (int k = 0; k < kRunOwn; ++k) {
            at[k] = -1;
            if (k * kThreads >= n_hits) continue;
            const int e = tid + k * kThreads;
            if (e < n_hits) {
                const uint32_t hit = hits[e];
                bool mine;
                id[k] = c0 + int(hit & 0x7FFFu);
                const int h = t.add(id[k], mine);
                if (!(hit & 0x8000u)) atomicAdd(t.count + h, 1);
                if (mine) {
                    at[k] = h;
                    x[k] = load_one<kInF32>(in, id[k]);
                    if (r.prompt && Row::has(r.prompt, id[k])) in_prompt |= 1u << k;
                    if (r.mask && !Row::has(r.mask, id[k])) open &= ~(1u << k);
                }
            }
        }
        __syncthreads();
        if (biased && n_bias > kFewBiases) add_many_biases<kThreads>(a.r.bias_ids + b0, a.r.bias_values + b0, n_bias, t, to);
        else if (biased && tid < 32) add_biases(a.r.bias_ids + b0, a.r.bias_values + b0, n_bias, t, tid);
        for (int g = 0; g < tiles; ++g) stream(g);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kRunOwn; ++k)
            if (at[k] >= 0)
                store_one<kOutF32>(out, id[k], open & (1u << k) ? ruled(x[k], t.count[at[k]], in_prompt & (1u << k)) + t.value[at[k]] : -INFINITY);
    } else {
        // tile by tile, with a counter for every token of it
        t.hashed = false;
        t.log2_slots = kLog2RunSlots;
        for (int g = 0; g < tiles; ++g) {
            t.r0 = c0 + g * kTile;
            t.r1 = min(c1, t.r0 + kTile);
            t.clear(tid, kThreads);
            __syncthreads();
            bool mine;
            for (int e = tid; e < n_said; e += kThreads) {
                const int h = t.add(said[e], mine);
                if (h >= 0) atomicAdd(t.count + h, 1);
            }
            for (int e = tid; e < n_bias; e += kThreads) t.add(a.r.bias_ids[b0 + e], mine);
            __syncthreads();
            if (biased) {
                if (n_bias > kFewBiases) add_many_biases<kThreads>(a.r.bias_ids + b0, a.r.bias_values + b0, n_bias, t, to);
                else if (tid < 32) add_biases(a.r.bias_ids + b0, a.r.bias_values + b0, n_bias, t, tid);
                __syncthreads();
            }
#pragma unroll 8
            for (int h = tid; h < kTile; h += kThreads) {
                const int token = t.key[h];
                if (token < 0) continue;
                const float x = ruled(load_one<kInF32>(in, token), t.count[h], r.prompt && Row::has(r.prompt, token));
                t.value[h] = !r.mask || Row::has(r.mask, token) ? x + t.value[h] : -INFINITY;
            }
            __syncthreads();   // in place: the logits have been read
            stream(g);
            __syncthreads();
#pragma unroll 8
            for (int h = tid; h < kTile; h += kThreads)
                if (t.key[h] >= 0) store_one<kOutF32>(out, t.key[h], t.value[h]);
            __syncthreads();
        }
    }
}

// Token sets as bitmaps: one block per (row, kMarkTile tokens) walks the row's list and sets bits in shared memory.  Bound by the shared
// atomics of one block, 16-byte loads change nothing: 64 rows x 32768 ids, vocabulary 131072, 5.4 us (floor 1.1); 256 rows 9.1, and 14.4
// with tiles of half the size, whose blocks read every list twice.  Larger vocabularies are where that begins (131073 / 151936 tokens): 64 rows x
// 32768 ids 6.2 -> 6.7 / 7.4 us as calls, 256 x 4096 6.2 -> 8.1 / 8.3.
__global__ void __launch_bounds__(kMarkThreads)
mark_kernel(const int32_t *__restrict__ ids, int num_ids, const int32_t *__restrict__ indptr, int vocab, uint32_t *__restrict__ bits, int64_t row_words)
{
    __shared__ uint32_t tile[kMarkTile / 32];
    const int row = blockIdx.y, base = blockIdx.x * kMarkTile;
    const int limit = min(vocab, base + kMarkTile);
    for (int w = threadIdx.x; w < kMarkTile / 32; w += kMarkThreads) tile[w] = 0u;
    __syncthreads();
    const int first = max(0, indptr[row]), last = min(num_ids, indptr[row + 1]);
    for (int64_t e0 = first; e0 < last; e0 += kMarkBatch * kMarkThreads) {
        int id[kMarkBatch];   // that many loads in flight per thread
#pragma unroll
        for (int j = 0; j < kMarkBatch; ++j) {
            const int64_t e = e0 + j * kMarkThreads + threadIdx.x;
            id[j] = e < last ? ids[e] : -1;
        }
#pragma unroll
        for (int j = 0; j < kMarkBatch; ++j)
            if (id[j] >= base && id[j] < limit) atomicOr(&tile[(id[j] - base) >> 5], 1u << ((id[j] - base) & 31));
    }
    __syncthreads();
    uint32_t *to = bits + int64_t(row) * row_words + base / 32;
    for (int w = threadIdx.x; w < (limit - base + 31) / 32; w += kMarkThreads) to[w] = tile[w];
}

bool misaligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }
// Whether rows of `width` bytes every `stride` bytes from p share memory with rows of `width2` every `stride2` from q.  Different strides
// count as sharing wherever the two ranges do.
bool rows_overlap(const void *p, int64_t stride, int64_t width, const void *q, int64_t stride2, int64_t width2, int64_t rows)
{
    const int64_t gap = int64_t(reinterpret_cast<uintptr_t>(q)) - int64_t(reinterpret_cast<uintptr_t>(p));
    if (gap >= (rows - 1) * stride + width || -gap >= (rows - 1) * stride2 + width2) return false;
    if (stride != stride2 || rows == 1) return true;
    const int64_t d = ((gap % stride) + stride) % stride;   // from a row of p to the next row of q
    return d < width || stride - d < width2;
}
bool known_dtype(int32_t d) { return d == PSA_OUT_BF16 || d == PSA_OUT_F32; }

// A launch that sets itself up under the tail of the one before it and waits there (griddepcontrol.wait) for its results.
template <class Kernel>
cudaError_t launch_behind(Kernel kernel, dim3 grid, int threads, size_t smem, cudaStream_t st, const RulesArgs &a)
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
    return cudaLaunchKernelEx(&lc, kernel, a);
}

template <bool kInF32, bool kOutF32>
cudaError_t launch_rules(const RulesArgs &a, int rows, bool lists, bool long_lists, cudaStream_t st)
{
    const auto whole = rules_lists_kernel<kInF32, kOutF32, true>, part = rules_lists_kernel<kInF32, kOutF32, false>;
    const auto stream = rules_stream_kernel<kInF32, kOutF32>;
    const auto run = rules_run_kernel<kInF32, kOutF32>;
    if (lists) {
        static PerDeviceOnce once;
        const int rc = once.ensure([&] {
            cudaError_t e = cudaFuncSetAttribute(whole, cudaFuncAttributeMaxDynamicSharedMemorySize, 12 << kLog2Many);
            if (e == cudaSuccess) e = cudaFuncSetAttribute(part, cudaFuncAttributeMaxDynamicSharedMemorySize, 12 << kLog2Many);
            if (e == cudaSuccess) e = cudaFuncSetAttribute(run, cudaFuncAttributeMaxDynamicSharedMemorySize, run_bytes(kInF32));
            return int(e);
        });
        if (rc != 0) return cudaError_t(rc);
    }
    const size_t table = size_t(12) << a.log2_slots;
    if (lists && a.vocab <= kWholeRow) return launch_behind(whole, dim3(rows), kListThreads, table, st, a);
    if (lists && (a.logits == a.out || long_lists || a.r.num_biases > int64_t(kManyBiases) * rows)) {
        // Long runs, since every block reads all of its row's lists: 256 rows x 131072 in place take 44.5 us in runs of 4 tiles, 34.7 in 8 and
        // 31.2 in 16 (three sets of inputs in turn).  But two or three blocks for every SM (64 rows: 14.0, 12.3, 13.2; 8 rows: 6.7, 8.2, 10.4),
        // and no more entries in a run than its table takes (8192 generated tokens: 87, 97, 132).
        RulesArgs b = a;
        const int64_t said = a.r.history ? a.r.history_capacity : 0;
        auto blocks = [&](int tiles) { return (a.vocab + tiles * kTile - 1) / (tiles * kTile); };
        b.run = kLeastRun;
        while (b.run < kMostRun && int64_t(blocks(2 * b.run)) * rows >= 3 * 148 && said * (2 * b.run * kTile) / a.vocab <= kHits / 2) b.run *= 2;
        return launch_behind(run, dim3(blocks(b.run), rows), kThreads, run_bytes(kInF32), st, b);
    }
    const dim3 tiles((a.vocab + kStreamRun * kStreamTile - 1) / (kStreamRun * kStreamTile), rows);
    cudaError_t e = launch_behind(stream, tiles, kStreamThreads, 0, st, a);
    if (e == cudaSuccess && lists) e = launch_behind(part, dim3(rows), kListThreads, table, st, a);
    return e;
}

}  // namespace
}  // namespace psa

extern "C" psa_status_t psa_process_logits(const void *logits, int32_t logits_dtype, int64_t row_stride, int32_t num_rows, int32_t vocab,
                                           const psa_logits_rules_t *rules, void *out, int32_t out_dtype, int64_t out_row_stride,
                                           void *cuda_stream)
{
    using psa::set_last_error;
    if (num_rows < 0 || vocab < 0) return set_last_error(PSA_ERR_INVALID_ARG, "negative num_rows or vocab");
    if (num_rows == 0) return PSA_OK;
    if (vocab == 0) return set_last_error(PSA_ERR_INVALID_ARG, "vocab must be positive");
    if (num_rows > 65535) return set_last_error(PSA_ERR_UNSUPPORTED, "at most 65535 rows per call");
    if (vocab > (1 << 24)) return set_last_error(PSA_ERR_UNSUPPORTED, "vocab must be at most 2^24");
    if (!psa::known_dtype(logits_dtype) || !psa::known_dtype(out_dtype))
        return set_last_error(PSA_ERR_UNSUPPORTED, "dtypes must be PSA_OUT_BF16 or PSA_OUT_F32");
    if (!logits || !out || !rules) return set_last_error(PSA_ERR_INVALID_ARG, "null argument");
    if (psa::misaligned(logits, 16) || row_stride < vocab || row_stride % 8 || psa::misaligned(out, 16) || out_row_stride < vocab || out_row_stride % 8)
        return set_last_error(PSA_ERR_INVALID_ARG, "logits and out must be 16-byte aligned with row strides >= vocab that are multiples of 8 elements");
    if (logits == out && (logits_dtype != out_dtype || row_stride != out_row_stride))
        return set_last_error(PSA_ERR_INVALID_ARG, "in place, input and output must have the same type and stride");
    const int64_t in_size = logits_dtype == PSA_OUT_F32 ? 4 : 2, out_size = out_dtype == PSA_OUT_F32 ? 4 : 2;
    if (logits != out && psa::rows_overlap(logits, row_stride * in_size, vocab * in_size, out, out_row_stride * out_size, vocab * out_size, num_rows))
        return set_last_error(PSA_ERR_INVALID_ARG, "logits and out must be the same array or not overlap");
    const psa_logits_rules_t &r = *rules;
    if ((r.history && !r.history_lens) || r.history_capacity < 0 || (r.history && r.history_stride < r.history_capacity))
        return set_last_error(PSA_ERR_INVALID_ARG, "history needs history_lens and a stride of at least its capacity");
    if (r.num_prompt_bitmaps < 0 || r.num_mask_bitmaps < 0 || r.num_biases < 0) return set_last_error(PSA_ERR_INVALID_ARG, "negative counts");
    if (r.bias_indptr && r.num_biases > 0 && (!r.bias_ids || !r.bias_values)) return set_last_error(PSA_ERR_INVALID_ARG, "bias_indptr needs bias_ids and bias_values");
    const int64_t words = (int64_t(vocab) + 31) / 32;
    if ((r.prompt_bits && r.prompt_row_words < words) || (r.mask_bits && r.mask_row_words < words))
        return set_last_error(PSA_ERR_INVALID_ARG, "bitmap rows must hold at least ceil(vocab / 32) words");
    const bool lists = (r.history && r.history_capacity > 0) || (r.bias_indptr && r.num_biases > 0);
    psa::RulesArgs a{r, logits, out, row_stride, out_row_stride, vocab, 0, 0};
    // A table as small as the lists allow, since it decides how many of their blocks fit beside the stream's (256 rows x 131072, up
    // to 1088 entries a row: 96 KB 33.9 us, 48 KB 31.2).  For whole rows it takes all entries there can be or has a slot for every token; else it
    // takes four times the mean number of biases, and rows with more are done in ranges.
    const int64_t said = r.history ? r.history_capacity : 0, biases = r.bias_indptr ? r.num_biases : 0;
    const int64_t most = said + (vocab <= psa::kWholeRow ? biases : std::min(biases, std::max<int64_t>(512, 4 * biases / num_rows)));
    a.log2_slots = psa::kLog2Few;
    while (a.log2_slots < psa::kLog2Many && most > psa::table_takes(a.log2_slots)) ++a.log2_slots;
    static_assert(psa::kWholeRow <= 1 << psa::kLog2Many, "a slot for every token");
    const bool long_lists = most > psa::table_takes(psa::kLog2Many);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e;
    if (logits_dtype == PSA_OUT_F32)
        e = out_dtype == PSA_OUT_F32 ? psa::launch_rules<true, true>(a, num_rows, lists, long_lists, st) : psa::launch_rules<true, false>(a, num_rows, lists, long_lists, st);
    else
        e = out_dtype == PSA_OUT_F32 ? psa::launch_rules<false, true>(a, num_rows, lists, long_lists, st) : psa::launch_rules<false, false>(a, num_rows, lists, long_lists, st);
    if (e != cudaSuccess) return set_last_error(PSA_ERR_CUDA, std::string("logits launch: ") + cudaGetErrorString(e));
    return PSA_OK;
}

extern "C" psa_status_t psa_mark_tokens(const int32_t *ids, int32_t num_ids, const int32_t *indptr, int32_t num_rows, int32_t vocab,
                                        uint32_t *bits, int64_t row_words, void *cuda_stream)
{
    using psa::set_last_error;
    if (num_rows < 0 || vocab < 0 || num_ids < 0) return set_last_error(PSA_ERR_INVALID_ARG, "negative num_rows, vocab or num_ids");
    if (num_rows == 0) return PSA_OK;
    if (vocab == 0) return set_last_error(PSA_ERR_INVALID_ARG, "vocab must be positive");
    if (num_rows > 65535) return set_last_error(PSA_ERR_UNSUPPORTED, "at most 65535 rows per call");
    if (vocab > (1 << 24)) return set_last_error(PSA_ERR_UNSUPPORTED, "vocab must be at most 2^24");
    if ((!ids && num_ids > 0) || !indptr || !bits) return set_last_error(PSA_ERR_INVALID_ARG, "null argument");
    if (row_words < (int64_t(vocab) + 31) / 32) return set_last_error(PSA_ERR_INVALID_ARG, "bitmap rows must hold at least ceil(vocab / 32) words");
    psa::mark_kernel<<<dim3((vocab + psa::kMarkTile - 1) / psa::kMarkTile, num_rows), psa::kMarkThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
        ids, num_ids, indptr, vocab, bits, row_words);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return set_last_error(PSA_ERR_CUDA, std::string("mark launch: ") + cudaGetErrorString(e));
    return PSA_OK;
}
