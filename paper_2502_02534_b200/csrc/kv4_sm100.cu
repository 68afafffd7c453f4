// The 4-bit K/V cache's writer and reader: quantise the K/V rows of new tokens into the cells of their slots, and turn
// cached tokens back into bf16 rows (the layout is described in kv4.h).
//
// Quantisation of a group of 32 channels: b = min, s = bf16((max - min) / 15), code = rint((x - b) / s), 0 where s = 0.
// b is one of the inputs, hence exact; s is rounded once, to the bf16 it is stored as (half a step of 2^-8, which moves the
// top level by at most 0.03 of a step), and the codes are chosen against the rounded s.  Differences, quotients and
// roundings are IEEE fp32, so the codes do not depend on who computes them.  A group whose range is not finite (a NaN, an
// infinity, or a range beyond fp32) gets s = NaN: it reads back as NaN.
//
// Work: a thread takes half a group (16 channels, 32 bytes of bf16) of K and of V of one row, so that the group's minimum and
// maximum need one shuffle and the indices are worked out once per 64 bytes.  The quotient is one multiplication by the correctly
// rounded 1 / s and one residual step, which rounds exactly like the division (Markstein) as long as nothing under- or overflows;
// groups of extreme range, and those that are not finite, take the division itself.  Both kernels are bound by HBM: 4 bytes read and
// 1.25 written per channel of K and V, or the reverse.
// Measured, 65536 tokens x 8 heads of 128 channels (353 MB): store 57 us (6.2 TB/s, 0.95 of the measured copy rate), load 63 us (5.6
// TB/s).  Store with 8 channels a thread 73-76 us (the indices twice), with grid-wide loops 85-102.
#include <cuda_runtime.h>

#include <algorithm>
#include <string>

#include "kv4.h"

namespace psa {
namespace {

constexpr int kKv4Threads = 128;
constexpr int kPer = 16, kStoreRows = 1;     // channels of a thread that quantises, and rows it has in flight
constexpr int kLoadPer = 8, kLoadRows = 2;   // channels of a thread that reads back, and rows it has in flight
constexpr float kFifteenth = 1.f / 15.f;

struct Kv4Args {
    const __nv_bfloat16 *in_k, *in_v;   // store: [T, Hkv, D]
    __nv_bfloat16 *out_k, *out_v;       // load
    int64_t stride_tok, stride_head;    // elements
    const int64_t *slot_map;
    int64_t num_tokens;
    int num_kv_heads;
    uint32_t heads_magic, heads_shift;  // row / num_kv_heads = mulhi(row, magic) >> shift for row < 2^31
    unsigned char *pool;
    int64_t stride_page, stride_cell;   // bytes: page to page, KV head to KV head
    int64_t num_pool_pages;
    int32_t *status;
};

__device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ float lo_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Two fp32 operations at once (each rounded like the single one).
struct F2 {
    float x, y;
};
__device__ __forceinline__ F2 add2(F2 a, F2 b)
{
    F2 d;
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tadd.rn.f32x2 p, p, q;\n\tmov.b64 {%0, %1}, p;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b)
{
    F2 d;
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tmul.rn.f32x2 p, p, q;\n\tmov.b64 {%0, %1}, p;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c)
{
    F2 d;
    asm("{\n\t.reg .b64 p, q, r;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tmov.b64 r, {%6, %7};\n\tfma.rn.f32x2 p, p, q, r;\n\t"
        "mov.b64 {%0, %1}, p;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}

struct Quantised {
    uint32_t codes[kPer / 8];  // nibbles
    uint16_t scale, offset;    // bf16 bits, the same in all threads of a group
};

// Any group, by IEEE divisions; `w` this thread's channels.
__device__ __forceinline__ void quantise_any(const uint32_t (&w)[kPer / 2], float range, float b, Quantised &q)
{
    const float s = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(range, 15.f)));
    const bool finite = s <= 3.0e38f;
    q.scale = finite ? uint16_t(__float_as_uint(s) >> 16) : uint16_t(0x7FC0);   // NaN or infinite: the group reads back as NaN
#pragma unroll
    for (int i = 0; i < kPer / 8; ++i) q.codes[i] = 0u;
    if (!finite || !(s > 0.f)) return;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i) {
        const float r = ((i & 1) ? hi_f32(w[i >> 1]) : lo_f32(w[i >> 1])) - b;
        q.codes[i >> 3] = q.codes[i >> 3] * 16u + uint32_t(fminf(rintf(__fdiv_rn(r, s)), 15.f));
    }
}

__device__ __forceinline__ Quantised quantise(const uint32_t (&w)[kPer / 2])
{
    uint32_t lo = w[0], hi = w[0];
#pragma unroll
    for (int i = 1; i < kPer / 2; ++i) { lo = min2_nan(lo, w[i]); hi = max2_nan(hi, w[i]); }
    lo = min2_nan(lo, __byte_perm(lo, 0u, 0x1032));
    hi = max2_nan(hi, __byte_perm(hi, 0u, 0x1032));
    // both halves alike: the minimum and minus the maximum go through one shuffle and one minimum a step
    uint32_t both = __byte_perm(lo, hi ^ 0x80008000u, 0x5410);
#pragma unroll
    for (int o = 1; o < kKv4Group / kPer; o <<= 1) both = min2_nan(both, __shfl_xor_sync(0xffffffffu, both, o));
    const float b = lo_f32(both), range = -hi_f32(both) - b;
    // range / 15, rounded like the division
    const float s0 = __fmul_rn(range, kFifteenth);
    const float s = __bfloat162float(__float2bfloat16_rn(__fmaf_rn(__fmaf_rn(-s0, 15.f, range), kFifteenth, s0)));
    Quantised q;
    q.offset = uint16_t(both);
    if (s > 1e-30f && s < 1e30f) {
        q.scale = uint16_t(__float_as_uint(s) >> 16);
        // 1 / s to the last bit: s has 8 significant bits, so its reciprocal lies at least 2^-33 from a rounding border, and one
        // Newton step from an approximation good to 2^-22 ends within 2^-43
        float inv;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
        inv = __fmaf_rn(__fmaf_rn(-s, inv, 1.f), inv, inv);
        // code + 1.5 * 2^23: adding that constant rounds to the nearest whole number, ties to even, into the low bits
        const F2 nb{-b, -b}, i2{inv, inv}, ns{-s, -s}, magic{12582912.f, 12582912.f};
#pragma unroll
        for (int h = 0; h < kPer / 8; ++h) {
            uint32_t c = 0u;
#pragma unroll
            for (int i = 4 * h + 3; i >= 4 * h; --i) {
                const F2 r = add2(F2{lo_f32(w[i]), hi_f32(w[i])}, nb);
                const F2 q0 = mul2(r, i2);
                const F2 code = add2(fma2(fma2(q0, ns, r), i2, q0), magic);
                c = (c * 16u + __float_as_uint(code.y)) * 16u + __float_as_uint(code.x);
            }
            constexpr uint32_t kBiasSum = 0x4B400000u * 0x11111111u;   // of the eight constants, each shifted by its nibble
            q.codes[h] = c - kBiasSum;
        }
    } else {
        quantise_any(w, range, b, q);
    }
    return q;
}

// The cell of a slot, or null: negative slots are skipped, slots beyond the pool are reported.
__device__ __forceinline__ unsigned char *cell_of(const Kv4Args &a, int64_t slot, int head)
{
    if (slot < 0) return nullptr;
    const int64_t page = slot / kPageSize;
    if (page >= a.num_pool_pages) {
        if (a.status) atomicCAS(a.status, 0, int(PSA_ERR_BOUNDS));
        return nullptr;
    }
    return a.pool + page * a.stride_page + int64_t(head) * a.stride_cell;
}

__device__ __forceinline__ uint32_t token_of(const Kv4Args &a, uint32_t row)
{
    return a.num_kv_heads == 1 ? row : __umulhi(row, a.heads_magic) >> a.heads_shift;
}

// Rows (token, KV head) are dealt out in order, `per` channels a thread; a row never straddles a warp.
template <int D, int per>
struct MyRow {
    static constexpr int kThreads = D / per;
    static constexpr int kPerBlock = kKv4Threads / kThreads;
    uint32_t token;
    int head;
    __device__ __forceinline__ MyRow(const Kv4Args &a, uint32_t row)
    {
        token = token_of(a, row);
        head = int(row - token * uint32_t(a.num_kv_heads));
    }
    __device__ __forceinline__ int64_t at(const Kv4Args &a) const
    {
        return int64_t(token) * a.stride_tok + head * a.stride_head + threadIdx.x % kThreads * per;
    }
};

template <int D>
__global__ void __launch_bounds__(kKv4Threads)
store_kv4_kernel(Kv4Args a)
{
    using C = Kv4Cell<D>;
    using R = MyRow<D, kPer>;
    constexpr int kWords = kPer / 2;
    const uint32_t rows = uint32_t(a.num_tokens) * uint32_t(a.num_kv_heads);     // below 2^31
    const uint32_t base = blockIdx.x * uint32_t(R::kPerBlock * kStoreRows) + threadIdx.x / R::kThreads;
    const int lane = threadIdx.x % R::kThreads, group = lane / (kKv4Group / kPer), part = lane % (kKv4Group / kPer);
    uint32_t k[kStoreRows][kWords], v[kStoreRows][kWords];
    int64_t slot[kStoreRows];
    int head[kStoreRows];
    // K and V are requested before the slots are known: a row that is skipped costs its bytes, every other one a round trip less
#pragma unroll
    for (int i = 0; i < kStoreRows; ++i) {
        const uint32_t row = base + i * R::kPerBlock;
        slot[i] = -1;
        head[i] = 0;
#pragma unroll
        for (int j = 0; j < kWords; ++j) k[i][j] = v[i][j] = 0u;
        if (row < rows) {
            const R r(a, row);
            head[i] = r.head;
            const uint4 *pk = reinterpret_cast<const uint4 *>(a.in_k + r.at(a)), *pv = reinterpret_cast<const uint4 *>(a.in_v + r.at(a));
#pragma unroll
            for (int j = 0; j < kWords / 4; ++j) {
                *reinterpret_cast<uint4 *>(&k[i][4 * j]) = __ldg(pk + j);
                *reinterpret_cast<uint4 *>(&v[i][4 * j]) = __ldg(pv + j);
            }
            slot[i] = a.slot_map[r.token];
        }
    }
#pragma unroll
    for (int i = 0; i < kStoreRows; ++i) {
        const Quantised qk = quantise(k[i]), qv = quantise(v[i]);
        unsigned char *cell = cell_of(a, slot[i], head[i]);
        if (!cell) continue;
        const int tok = int(slot[i] & (kPageSize - 1));
        uint32_t *codes = reinterpret_cast<uint32_t *>(cell + C::chunk(tok, group) + part * (kPer / 2));
        uint32_t *codes_v = reinterpret_cast<uint32_t *>(reinterpret_cast<unsigned char *>(codes) + C::kCodeBytes);
        if constexpr (kPer == 16) {
            *reinterpret_cast<uint2 *>(codes) = make_uint2(qk.codes[0], qk.codes[1]);
            *reinterpret_cast<uint2 *>(codes_v) = make_uint2(qv.codes[0], qv.codes[1]);
        } else {
            codes[0] = qk.codes[0];
            codes_v[0] = qv.codes[0];
        }
        // the first thread of a group files K's parameters, the second V's
        if (part < 2) {
            unsigned char *params = cell + C::params(part, tok) + 2 * group;
            *reinterpret_cast<uint16_t *>(params) = part ? qv.scale : qk.scale;
            *reinterpret_cast<uint16_t *>(params + 2 * C::kGroups) = part ? qv.offset : qk.offset;
        }
    }
}

// Eight channels: s * code + b, rounded once to bf16.  A nibble or'ed into the mantissa of 128 is 128 + code; subtracting 128 is exact.
__device__ __forceinline__ uint4 dequantise(uint32_t codes, uint32_t scale, uint32_t offset)
{
    const uint32_t s2 = scale * 0x10001u, b2 = offset * 0x10001u;
    const uint32_t even = codes & 0x0F0F0F0Fu, odd = (codes >> 4) & 0x0F0F0F0Fu;   // byte i: channels 2 i and 2 i + 1
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // byte i of each into the halves' low bytes; the high bytes are whatever, and replaced
        const uint32_t pair = (__byte_perm(even, odd, uint32_t(i | (i << 4) | ((4 + i) << 8) | ((4 + i) << 12))) & 0x000F000Fu) | 0x43004300u;
        uint32_t c;
        asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(pair), "r"(0x43004300u));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(w[i]) : "r"(c), "r"(s2), "r"(b2));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int D>
__global__ void __launch_bounds__(kKv4Threads)
load_kv4_kernel(Kv4Args a)
{
    using C = Kv4Cell<D>;
    using R = MyRow<D, kLoadPer>;
    const uint32_t rows = uint32_t(a.num_tokens) * uint32_t(a.num_kv_heads);
    const uint32_t base = blockIdx.x * uint32_t(R::kPerBlock * kLoadRows) + threadIdx.x / R::kThreads;
    const int lane = threadIdx.x % R::kThreads, group = lane >> 2;
    const unsigned char *cell[kLoadRows];
    int tok[kLoadRows];
    int64_t to[kLoadRows];
#pragma unroll
    for (int i = 0; i < kLoadRows; ++i) {
        const uint32_t row = base + i * R::kPerBlock;
        cell[i] = nullptr;
        if (row < rows) {
            const R r(a, row);
            const int64_t slot = a.slot_map[r.token];
            cell[i] = cell_of(a, slot, r.head);
            tok[i] = int(slot & (kPageSize - 1));
            to[i] = r.at(a);
        }
    }
    uint32_t ck[kLoadRows], cv[kLoadRows], sk[kLoadRows], sv[kLoadRows], bk[kLoadRows], bv[kLoadRows];
#pragma unroll
    for (int i = 0; i < kLoadRows; ++i) {
        if (!cell[i]) continue;
        const unsigned char *codes = cell[i] + C::chunk(tok[i], group) + (lane & 3) * 4;
        ck[i] = *reinterpret_cast<const uint32_t *>(codes);
        cv[i] = *reinterpret_cast<const uint32_t *>(codes + C::kCodeBytes);
        const uint16_t *pk = reinterpret_cast<const uint16_t *>(cell[i] + C::params(0, tok[i])) + group;
        const uint16_t *pv = reinterpret_cast<const uint16_t *>(cell[i] + C::params(1, tok[i])) + group;
        sk[i] = pk[0]; bk[i] = pk[C::kGroups]; sv[i] = pv[0]; bv[i] = pv[C::kGroups];
    }
#pragma unroll
    for (int i = 0; i < kLoadRows; ++i) {
        if (!cell[i]) continue;
        *reinterpret_cast<uint4 *>(a.out_k + to[i]) = dequantise(ck[i], sk[i], bk[i]);
        *reinterpret_cast<uint4 *>(a.out_v + to[i]) = dequantise(cv[i], sv[i], bv[i]);
    }
}

bool misaligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

psa_status_t check(const Kv4Args &a, const void *k, const void *v, const int64_t kv_strides[2], int head_dim, const int64_t pool_strides[2])
{
    if (a.num_tokens < 0 || a.num_kv_heads <= 0 || a.num_pool_pages < 0) return set_last_error(PSA_ERR_INVALID_ARG, "negative sizes or no KV head");
    if (head_dim != 64 && head_dim != 128) return set_last_error(PSA_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
    if (a.num_kv_heads > 65536 || a.num_tokens > 0x7fffffff / a.num_kv_heads)
        return set_last_error(PSA_ERR_UNSUPPORTED, "at most 2^31 - 1 rows (tokens x KV heads) per call");
    if (a.num_tokens == 0) return PSA_OK;
    if (!k || !v || !kv_strides || !a.slot_map || !pool_strides || (a.num_pool_pages > 0 && !a.pool))
        return set_last_error(PSA_ERR_INVALID_ARG, "null K/V cache argument");
    if (misaligned(k, 16) || misaligned(v, 16) || misaligned(a.pool, 16))
        return set_last_error(PSA_ERR_INVALID_ARG, "K, V and the pool must be 16-byte aligned");
    if (misaligned(a.status, 4)) return set_last_error(PSA_ERR_INVALID_ARG, "the status word must be 4-byte aligned");
    for (int i = 0; i < 2; ++i) {
        if (kv_strides[i] <= 0 || kv_strides[i] % 8) return set_last_error(PSA_ERR_INVALID_ARG, "K/V strides must be positive multiples of 8 elements");
        if (pool_strides[i] < 20 * head_dim || pool_strides[i] % 16)
            return set_last_error(PSA_ERR_INVALID_ARG, "pool strides must be multiples of 16 bytes, at least one cell");
    }
    return PSA_OK;
}

template <class K64, class K128>
psa_status_t launch(Kv4Args a, int head_dim, K64 k64, K128 k128, int64_t rows_per_block, void *cuda_stream, const char *what)
{
    const unsigned blocks = unsigned((a.num_tokens * a.num_kv_heads + rows_per_block - 1) / rows_per_block);
    // division by the head count (Granlund and Montgomery): magic = ceil(2^(32 + shift) / heads), 2^shift < heads <= 2^(shift + 1)
    while ((2u << a.heads_shift) < unsigned(a.num_kv_heads)) ++a.heads_shift;
    a.heads_magic = uint32_t(((uint64_t(1) << (32 + a.heads_shift)) + unsigned(a.num_kv_heads) - 1) / unsigned(a.num_kv_heads));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (head_dim == 64) k64<<<blocks, kKv4Threads, 0, st>>>(a);
    else k128<<<blocks, kKv4Threads, 0, st>>>(a);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return set_last_error(PSA_ERR_CUDA, std::string(what) + cudaGetErrorString(e));
    return PSA_OK;
}

}  // namespace
}  // namespace psa

extern "C" size_t psa_kv4_cell_bytes(int32_t head_dim) { return head_dim == 64 || head_dim == 128 ? size_t(20) * head_dim : 0; }

extern "C" psa_status_t psa_store_kv4(const void *new_k, const void *new_v, const int64_t kv_strides[2], const int64_t *slot_map,
                                      int64_t num_tokens, int32_t num_kv_heads, int32_t head_dim, void *pool,
                                      const int64_t pool_strides[2], int64_t num_pool_pages, int32_t *status, void *cuda_stream)
{
    psa::Kv4Args a{};
    a.slot_map = slot_map; a.num_tokens = num_tokens; a.num_kv_heads = num_kv_heads;
    a.pool = static_cast<unsigned char *>(pool); a.num_pool_pages = num_pool_pages; a.status = status;
    const psa_status_t st = psa::check(a, new_k, new_v, kv_strides, head_dim, pool_strides);
    if (st != PSA_OK || num_tokens == 0) return st;
    a.in_k = static_cast<const __nv_bfloat16 *>(new_k); a.in_v = static_cast<const __nv_bfloat16 *>(new_v);
    a.stride_tok = kv_strides[0]; a.stride_head = kv_strides[1];
    a.stride_page = pool_strides[0]; a.stride_cell = pool_strides[1];
    return psa::launch(a, head_dim, psa::store_kv4_kernel<64>, psa::store_kv4_kernel<128>, psa::kKv4Threads / (head_dim / psa::kPer) * psa::kStoreRows, cuda_stream, "store launch: ");
}

extern "C" psa_status_t psa_load_kv4(const void *pool, const int64_t pool_strides[2], int64_t num_pool_pages, const int64_t *slot_map,
                                     int64_t num_tokens, int32_t num_kv_heads, int32_t head_dim, void *out_k, void *out_v,
                                     const int64_t kv_strides[2], int32_t *status, void *cuda_stream)
{
    psa::Kv4Args a{};
    a.slot_map = slot_map; a.num_tokens = num_tokens; a.num_kv_heads = num_kv_heads;
    a.pool = static_cast<unsigned char *>(const_cast<void *>(pool)); a.num_pool_pages = num_pool_pages; a.status = status;   // read only here
    const psa_status_t st = psa::check(a, out_k, out_v, kv_strides, head_dim, pool_strides);
    if (st != PSA_OK || num_tokens == 0) return st;
    a.out_k = static_cast<__nv_bfloat16 *>(out_k); a.out_v = static_cast<__nv_bfloat16 *>(out_v);
    a.stride_tok = kv_strides[0]; a.stride_head = kv_strides[1];
    a.stride_page = pool_strides[0]; a.stride_cell = pool_strides[1];
    return psa::launch(a, head_dim, psa::load_kv4_kernel<64>, psa::load_kv4_kernel<128>,
                       psa::kKv4Threads / (head_dim / psa::kLoadPer) * psa::kLoadRows, cuda_stream, "load launch: ");
}
