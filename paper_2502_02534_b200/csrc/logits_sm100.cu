// Rules applied to logits before a token is drawn: penalties for repeated tokens, additive biases, grammar masks.
//
// For logit x of token i in row r, with c = how often i stands in the row's generated tokens:
//     x <- x > 0 ? x / repetition : x * repetition       if c > 0 or i is in the row's prompt set   (by 1 / repetition, rounded once)
//     x <- x - frequency * c - presence * [c > 0]
//     x <- x + (sum of the row's biases for i, added in list order)
//     x <- -inf                                          if the row's mask has bit i clear
// in fp32, rounded once to the output type.
//
// One block per (row, tile of kTile logits).  The tile's logits and bitmaps are requested first, into registers; while they are on
// their way the block walks the row's generated tokens and biases twice: the first walk marks the tile's touched tokens in
// a bitmap and zeroes exactly their counters (nothing else of the counter arrays is ever read, so they need no clearing), the
// second adds up.  A thread then handles eight consecutive logits at a time: one byte each of the touched bitmap, the
// prompt set and the mask tell whether there is anything to do, and the common answer (no) costs a conversion.
// Each block reads and writes only its own tile, so the output may be the input.
// Bound: HBM, one read and one write of every logit; the walks read a few KB per block from L2.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <string>

#include "psa_internal.h"

namespace psa {
namespace {

constexpr int kRuleThreads = 256;
constexpr int kVec = 8;                                    // logits a thread handles together
constexpr int kRounds = 2;
constexpr int kKeep = 4;                                   // generated tokens a thread remembers between the two walks
constexpr int kTile = kRuleThreads * kVec * kRounds;       // 4096 logits
constexpr int kMarkTile = 32768;                           // tokens of one block's bitmap
constexpr int kMarkThreads = 1024;
constexpr int kMarkBatch = 8;

struct RulesArgs {
    psa_logits_rules_t r;
    const void *logits;
    void *out;
    int64_t row_stride, out_stride;
    int vocab;
};

struct RulesSmem {
    uint32_t touched[kTile / 32];
    int32_t count[kTile];
    float bias[kTile];
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

// Biases of one row that fall into [base, base + kTile): added to their cells in list order, by one warp.  Equal ids inside
// the 32 entries of a step are summed by the first lane that has them, so the order of the additions is that of the list.
__device__ void add_biases(const RulesArgs &a, RulesSmem &sm, int first, int last, int base, int limit, int lane)
{
    for (int e0 = first; e0 < last; e0 += 32) {
        const int e = e0 + lane;
        const int id = e < last ? a.r.bias_ids[e] : -1;
        const float v = e < last ? a.r.bias_values[e] : 0.f;
        const bool mine = id >= base && id < limit;
        const uint32_t same = __match_any_sync(0xffffffffu, mine ? id : -1);
        const bool leader = mine && (__ffs(same) - 1) == lane;
        float sum = leader ? sm.bias[id - base] : 0.f;
        // every lane takes part in the shuffles; at most 32 rounds, one without duplicates
        uint32_t rest = mine ? same : 0u;
        while (__any_sync(0xffffffffu, rest != 0u)) {
            const int from = rest ? __ffs(rest) - 1 : 0;
            const float u = __shfl_sync(0xffffffffu, v, from);
            if (rest) sum += u;
            rest &= rest - 1u;
        }
        if (leader) sm.bias[id - base] = sum;
        __syncwarp();
    }
}

template <bool kInF32, bool kOutF32>
__global__ void __launch_bounds__(kRuleThreads)
rules_kernel(RulesArgs a)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    RulesSmem &sm = *reinterpret_cast<RulesSmem *>(smem_raw);
    const int row = blockIdx.y, base = blockIdx.x * kTile, tid = threadIdx.x;
    const int limit = min(a.vocab, base + kTile);
    const void *in = static_cast<const unsigned char *>(a.logits) + int64_t(row) * a.row_stride * (kInF32 ? 4 : 2);
    void *out = static_cast<unsigned char *>(a.out) + int64_t(row) * a.out_stride * (kOutF32 ? 4 : 2);

    // ---- everything that does not depend on the lists is requested first: the row's numbers, its logits, its bitmaps
    const int32_t *said = a.r.history ? a.r.history + int64_t(row) * a.r.history_stride : nullptr;
    const int said_len = said ? a.r.history_lens[row] : 0;
    int b0 = 0, b1 = 0;
    if (a.r.bias_indptr) { b0 = a.r.bias_indptr[row]; b1 = a.r.bias_indptr[row + 1]; }
    const float rep_in = a.r.repetition ? a.r.repetition[row] : 1.f;
    const float freq = a.r.frequency ? a.r.frequency[row] : 0.f;
    const float pres = a.r.presence ? a.r.presence[row] : 0.f;
    const int64_t prompt_row = a.r.prompt_rows && a.r.prompt_bits ? a.r.prompt_rows[row] : row;
    const int64_t mask_row = a.r.mask_rows && a.r.mask_bits ? a.r.mask_rows[row] : row;
    Vec8<kInF32> v[kRounds];
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
        const int i = base + (k * kRuleThreads + tid) * kVec;
        if (i + kVec <= limit) v[k].load(in, i);
    }
    const unsigned char *prompt = nullptr, *mask = nullptr;
    if (a.r.prompt_bits && prompt_row >= 0 && prompt_row < a.r.num_prompt_bitmaps)
        prompt = reinterpret_cast<const unsigned char *>(a.r.prompt_bits + prompt_row * a.r.prompt_row_words);
    if (a.r.mask_bits && mask_row >= 0 && mask_row < a.r.num_mask_bitmaps)
        mask = reinterpret_cast<const unsigned char *>(a.r.mask_bits + mask_row * a.r.mask_row_words);
    uint32_t seen[kRounds], allowed[kRounds];   // one bit per logit
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
        const int i = base + (k * kRuleThreads + tid) * kVec;
        seen[k] = prompt && i < limit ? __ldg(prompt + (i >> 3)) : 0u;
        allowed[k] = mask && i < limit ? __ldg(mask + (i >> 3)) : 0xFFu;
    }

    // ---- the row's lists
    const int n_said = max(0, min(said_len, a.r.history_capacity));
    b0 = max(0, b0);
    b1 = min(a.r.num_biases, b1);
    const bool lists = n_said > 0 || b1 > b0;   // the same for the whole block
    if (lists) {
        int kept[kKeep];   // this thread's first generated tokens, as positions in the tile (-1: elsewhere)
        for (int w = tid; w < kTile / 32; w += kRuleThreads) sm.touched[w] = 0u;
        auto place = [&](const int32_t *list, int e, int n) {
            const int id = e < n ? list[e] : -1;
            return id >= base && id < limit ? id - base : -1;
        };
#pragma unroll
        for (int j = 0; j < kKeep; ++j) kept[j] = place(said, tid + j * kRuleThreads, n_said);
        __syncthreads();
        auto touch = [&](int at) {
            if (at >= 0) {
                sm.count[at] = 0; sm.bias[at] = 0.f;
                atomicOr(&sm.touched[at >> 5], 1u << (at & 31));
            }
        };
#pragma unroll
        for (int j = 0; j < kKeep; ++j) touch(kept[j]);
        for (int e = tid + kKeep * kRuleThreads; e < n_said; e += kRuleThreads) touch(place(said, e, n_said));
        for (int e = b0 + tid; e < b1; e += kRuleThreads) touch(place(a.r.bias_ids, e, b1));
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kKeep; ++j)
            if (kept[j] >= 0) atomicAdd(&sm.count[kept[j]], 1);
        for (int e = tid + kKeep * kRuleThreads; e < n_said; e += kRuleThreads) {
            const int at = place(said, e, n_said);
            if (at >= 0) atomicAdd(&sm.count[at], 1);
        }
        if (tid < 32 && b1 > b0) add_biases(a, sm, b0, b1, base, limit, tid);
        __syncthreads();
    }

    const float rep = rep_in > 0.f ? rep_in : 1.f;   // not a penalty: off
    const float inv_rep = __fdiv_rn(1.f, rep);
    const unsigned char *touched = reinterpret_cast<const unsigned char *>(sm.touched);
    // a logit whose token is in one of the row's lists
    auto listed = [&](float x, int local, bool in_prompt) {
        const int c = sm.count[local];
        if (c > 0 || in_prompt) x *= x > 0.f ? inv_rep : rep;
        if (c > 0) x = x - freq * float(c) - pres;
        return x + sm.bias[local];
    };

#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
        const int local0 = (k * kRuleThreads + tid) * kVec;
        const int i = base + local0;
        if (i >= limit) continue;
        const uint32_t hits = lists ? touched[local0 >> 3] : 0u;
        const uint32_t prompt_only = seen[k] & ~hits, ok = allowed[k];
        float x[8];
        const bool whole = i + kVec <= limit;
        if (whole) {
            v[k].get(x);
        } else {   // the ragged end of a row: neither read nor written beyond the vocabulary
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = i + e < limit ? load_one<kInF32>(in, i + e) : 0.f;
        }
        if (hits) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (hits & (1u << e)) x[e] = listed(x[e], local0 + e, seen[k] & (1u << e));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (prompt_only & (1u << e)) x[e] *= x[e] > 0.f ? inv_rep : rep;
            if (!(ok & (1u << e))) x[e] = -INFINITY;
        }
        if (whole) {
            Vec8<kOutF32> o;
            o.set(x);
            o.store(out, i);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (i + e < limit) store_one<kOutF32>(out, i + e, x[e]);
        }
    }
}

// Token sets as bitmaps: one block per (row, kMarkTile tokens) walks the row's list and sets bits in shared memory.
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
bool known_dtype(int32_t d) { return d == PSA_OUT_BF16 || d == PSA_OUT_F32; }

template <bool kInF32, bool kOutF32>
cudaError_t launch_rules(const RulesArgs &a, int rows, cudaStream_t st)
{
    static PerDeviceOnce once;
    const int rc = once.ensure([] {
        return int(cudaFuncSetAttribute(rules_kernel<kInF32, kOutF32>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(sizeof(RulesSmem))));
    });
    if (rc != 0) return cudaError_t(rc);
    rules_kernel<kInF32, kOutF32><<<dim3((a.vocab + kTile - 1) / kTile, rows), kRuleThreads, sizeof(RulesSmem), st>>>(a);
    return cudaGetLastError();
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
    if (vocab > (1 << 30)) return set_last_error(PSA_ERR_UNSUPPORTED, "vocab must be at most 2^30");
    if (!psa::known_dtype(logits_dtype) || !psa::known_dtype(out_dtype))
        return set_last_error(PSA_ERR_UNSUPPORTED, "dtypes must be PSA_OUT_BF16 or PSA_OUT_F32");
    if (!logits || !out || !rules) return set_last_error(PSA_ERR_INVALID_ARG, "null argument");
    if (psa::misaligned(logits, 16) || row_stride < vocab || row_stride % 8 || psa::misaligned(out, 16) || out_row_stride < vocab || out_row_stride % 8)
        return set_last_error(PSA_ERR_INVALID_ARG, "logits and out must be 16-byte aligned with row strides >= vocab that are multiples of 8 elements");
    if (logits == out && (logits_dtype != out_dtype || row_stride != out_row_stride))
        return set_last_error(PSA_ERR_INVALID_ARG, "in place, input and output must have the same type and stride");
    const psa_logits_rules_t &r = *rules;
    if ((r.history && !r.history_lens) || r.history_capacity < 0 || (r.history && r.history_stride < r.history_capacity))
        return set_last_error(PSA_ERR_INVALID_ARG, "history needs history_lens and a stride of at least its capacity");
    if (r.num_prompt_bitmaps < 0 || r.num_mask_bitmaps < 0 || r.num_biases < 0) return set_last_error(PSA_ERR_INVALID_ARG, "negative counts");
    if (r.bias_indptr && r.num_biases > 0 && (!r.bias_ids || !r.bias_values)) return set_last_error(PSA_ERR_INVALID_ARG, "bias_indptr needs bias_ids and bias_values");
    const int64_t words = (int64_t(vocab) + 31) / 32;
    if ((r.prompt_bits && r.prompt_row_words < words) || (r.mask_bits && r.mask_row_words < words))
        return set_last_error(PSA_ERR_INVALID_ARG, "bitmap rows must hold at least ceil(vocab / 32) words");
    psa::RulesArgs a{r, logits, out, row_stride, out_row_stride, vocab};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e;
    if (logits_dtype == PSA_OUT_F32)
        e = out_dtype == PSA_OUT_F32 ? psa::launch_rules<true, true>(a, num_rows, st) : psa::launch_rules<true, false>(a, num_rows, st);
    else
        e = out_dtype == PSA_OUT_F32 ? psa::launch_rules<false, true>(a, num_rows, st) : psa::launch_rules<false, false>(a, num_rows, st);
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
    if (vocab > (1 << 30)) return set_last_error(PSA_ERR_UNSUPPORTED, "vocab must be at most 2^30");
    if ((!ids && num_ids > 0) || !indptr || !bits) return set_last_error(PSA_ERR_INVALID_ARG, "null argument");
    if (row_words < (int64_t(vocab) + 31) / 32) return set_last_error(PSA_ERR_INVALID_ARG, "bitmap rows must hold at least ceil(vocab / 32) words");
    psa::mark_kernel<<<dim3((vocab + psa::kMarkTile - 1) / psa::kMarkTile, num_rows), psa::kMarkThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
        ids, num_ids, indptr, vocab, bits, row_words);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return set_last_error(PSA_ERR_CUDA, std::string("mark launch: ") + cudaGetErrorString(e));
    return PSA_OK;
}
