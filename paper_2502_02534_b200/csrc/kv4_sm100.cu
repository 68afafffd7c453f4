// The 4-bit K/V cache's writer and reader: quantise the K/V rows of new tokens into the cells of their slots, and turn
// cached tokens back into bf16 rows (the layout is described in kv4.h).
//
// Quantisation of a group of 32 channels: b = min, s = bf16((max - min) / 15), code = rint((x - b) / s), 0 where s = 0.
// b is one of the inputs, hence exact; s is rounded once, to the bf16 it is stored as (half a step of 2^-8, which moves the
// top level by at most 0.03 of a step), and the codes are chosen against the rounded s.  Differences, quotients and
// roundings are IEEE fp32, so the codes do not depend on who computes them.  A group whose range is not finite (a NaN, an
// infinity, or a range beyond fp32) gets s = NaN: it reads back as NaN.
//
// Work: 16 bytes of bf16 (8 channels) per thread and row, four threads per group, K and V of kRows rows in the same thread;
// the group's minimum and maximum need two shuffles.  The quotient is one multiplication by the correctly rounded 1 / s and
// one residual step, which rounds exactly like the division (Markstein) as long as nothing under- or overflows; other
// groups take the division itself.  Both kernels are bound by HBM: 4 bytes read and 1.25 written per channel of K and V, or the
// reverse.
#include <cuda_runtime.h>

#include <algorithm>
#include <string>

#include "kv4.h"

namespace psa {
namespace {

constexpr int kKv4Threads = 256;
constexpr int kRows = 2;                     // rows a thread has in flight
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

struct Quantised {
    uint32_t codes;          // 8 nibbles
    uint16_t scale, offset;  // bf16 bits, the same in the four threads of a group
};

__device__ __forceinline__ Quantised quantise(uint4 x)
{
    uint32_t lo = min2_nan(min2_nan(x.x, x.y), min2_nan(x.z, x.w)), hi = max2_nan(max2_nan(x.x, x.y), max2_nan(x.z, x.w));
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        lo = min2_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = max2_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    lo = min2_nan(lo, (lo >> 16) | (lo << 16));
    hi = max2_nan(hi, (hi >> 16) | (hi << 16));
    const float b = lo_f32(lo);
    // (max - min) / 15, rounded like the division: a multiplication by 1 / 15 and one residual step, unless the range is extreme
    const float range = hi_f32(hi) - b;
    float s0 = __fmul_rn(range, kFifteenth);
    s0 = range > 1e-30f && range < 1e30f ? __fmaf_rn(__fmaf_rn(-s0, 15.f, range), kFifteenth, s0) : __fdiv_rn(range, 15.f);
    const float s = __bfloat162float(__float2bfloat16_rn(s0));
    Quantised q;
    q.offset = uint16_t(lo);
    if (!(s <= 3.0e38f)) {   // NaN or infinite
        q.scale = 0x7FC0;
        q.codes = 0;
        return q;
    }
    q.scale = uint16_t(__float_as_uint(s) >> 16);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    if (s > 1e-30f && s < 1e30f) {
        // 1 / s to the last bit: s has 8 significant bits, so its reciprocal lies at least 2^-33 from a rounding border, and one
        // Newton step from an approximation good to 2^-22 ends within 2^-43
        float inv;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
        inv = __fmaf_rn(__fmaf_rn(-s, inv, 1.f), inv, inv);
        // code + 1.5 * 2^23: adding that constant rounds to the nearest whole number, ties to even, into the low bits
        uint32_t acc = 0;
#pragma unroll
        for (int i = 7; i >= 0; --i) {
            const float r = ((i & 1) ? hi_f32(w[i >> 1]) : lo_f32(w[i >> 1])) - b;
            const float q0 = __fmul_rn(r, inv);
            const float q1 = __fmaf_rn(__fmaf_rn(-q0, s, r), inv, q0);
            acc = acc * 16u + __float_as_uint(__fadd_rn(q1, 12582912.f));
        }
        constexpr uint32_t kBias = 0x4B400000u;
        constexpr uint32_t kBiasSum = kBias * 0x11111111u;   // of the eight biases, each shifted by its nibble
        q.codes = acc - kBiasSum;
    } else {
        q.codes = 0;
        if (s > 0.f) {
#pragma unroll
            for (int i = 7; i >= 0; --i) {
                const float r = ((i & 1) ? hi_f32(w[i >> 1]) : lo_f32(w[i >> 1])) - b;
                q.codes = q.codes * 16u + uint32_t(fminf(rintf(__fdiv_rn(r, s)), 15.f));
            }
        }
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

template <int D>
__global__ void __launch_bounds__(kKv4Threads)
store_kv4_kernel(Kv4Args a)
{
    using C = Kv4Cell<D>;
    constexpr int kPerRow = D / 8;                       // threads of one (token, head) row; rows never straddle a warp
    const int lane = threadIdx.x % kPerRow, g = lane >> 2;
    const uint32_t rows = uint32_t(a.num_tokens) * uint32_t(a.num_kv_heads);     // below 2^31
    const uint32_t base = blockIdx.x * uint32_t(kKv4Threads / kPerRow * kRows) + threadIdx.x / kPerRow;
    uint4 k[kRows], v[kRows];
    int64_t slot[kRows];
    int head[kRows];
    // K and V are requested before the slots are known: a row that is skipped costs its bytes, every other one a round trip less
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const uint32_t row = base + i * (kKv4Threads / kPerRow);
        slot[i] = -1;
        head[i] = 0;
        k[i] = v[i] = uint4{};
        if (row < rows) {
            const uint32_t t = token_of(a, row);
            head[i] = int(row - t * uint32_t(a.num_kv_heads));
            const int64_t at = int64_t(t) * a.stride_tok + head[i] * a.stride_head + lane * 8;
            k[i] = __ldg(reinterpret_cast<const uint4 *>(a.in_k + at));
            v[i] = __ldg(reinterpret_cast<const uint4 *>(a.in_v + at));
            slot[i] = a.slot_map[t];
        }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const Quantised qk = quantise(k[i]), qv = quantise(v[i]);
        unsigned char *cell = cell_of(a, slot[i], head[i]);
        if (!cell) continue;
        const int tok = int(slot[i] % kPageSize);
        const int at = C::chunk(tok, g) + (lane & 3) * 4;
        *reinterpret_cast<uint32_t *>(cell + at) = qk.codes;
        *reinterpret_cast<uint32_t *>(cell + C::kCodeBytes + at) = qv.codes;
        // the four threads of a group file its four parameters
        const int which = (lane >> 1) & 1, offset = lane & 1;
        const uint16_t value = which ? (offset ? qv.offset : qv.scale) : (offset ? qk.offset : qk.scale);
        *reinterpret_cast<uint16_t *>(cell + C::params(which, tok) + 2 * (offset * C::kGroups + g)) = value;
    }
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&v);
}
// eight channels: s * code + b in fp32, rounded once to bf16
__device__ __forceinline__ uint4 dequantise(uint32_t codes, uint32_t scale, uint32_t offset)
{
    const float s = __uint_as_float(scale << 16), b = __uint_as_float(offset << 16);
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        f[i] = __fmaf_rn(__uint_as_float(((codes >> (4 * i)) & 15u) | 0x4B000000u) - 8388608.f, s, b);
    return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}

template <int D>
__global__ void __launch_bounds__(kKv4Threads)
load_kv4_kernel(Kv4Args a)
{
    using C = Kv4Cell<D>;
    constexpr int kPerRow = D / 8;
    const int lane = threadIdx.x % kPerRow, g = lane >> 2;
    const uint32_t rows = uint32_t(a.num_tokens) * uint32_t(a.num_kv_heads);
    const uint32_t base = blockIdx.x * uint32_t(kKv4Threads / kPerRow * kRows) + threadIdx.x / kPerRow;
    const unsigned char *cell[kRows];
    int tok[kRows];
    int64_t to[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const uint32_t row = base + i * (kKv4Threads / kPerRow);
        cell[i] = nullptr;
        if (row < rows) {
            const uint32_t t = token_of(a, row);
            const int head = int(row - t * uint32_t(a.num_kv_heads));
            const int64_t slot = a.slot_map[t];
            cell[i] = cell_of(a, slot, head);
            tok[i] = int(slot % kPageSize);
            to[i] = int64_t(t) * a.stride_tok + head * a.stride_head + lane * 8;
        }
    }
    uint32_t ck[kRows], cv[kRows], sk[kRows], sv[kRows], bk[kRows], bv[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        if (!cell[i]) continue;
        const int at = C::chunk(tok[i], g) + (lane & 3) * 4;
        ck[i] = *reinterpret_cast<const uint32_t *>(cell[i] + at);
        cv[i] = *reinterpret_cast<const uint32_t *>(cell[i] + C::kCodeBytes + at);
        const uint16_t *pk = reinterpret_cast<const uint16_t *>(cell[i] + C::params(0, tok[i])) + g;
        const uint16_t *pv = reinterpret_cast<const uint16_t *>(cell[i] + C::params(1, tok[i])) + g;
        sk[i] = pk[0]; bk[i] = pk[C::kGroups]; sv[i] = pv[0]; bv[i] = pv[C::kGroups];
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
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
    for (int i = 0; i < 2; ++i) {
        if (kv_strides[i] <= 0 || kv_strides[i] % 8) return set_last_error(PSA_ERR_INVALID_ARG, "K/V strides must be positive multiples of 8 elements");
        if (pool_strides[i] < 20 * head_dim || pool_strides[i] % 16)
            return set_last_error(PSA_ERR_INVALID_ARG, "pool strides must be multiples of 16 bytes, at least one cell");
    }
    return PSA_OK;
}

template <class K64, class K128>
psa_status_t launch(Kv4Args a, int head_dim, K64 k64, K128 k128, void *cuda_stream, const char *what)
{
    const int64_t rows_per_block = kKv4Threads / (head_dim / 8) * kRows;
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
    return psa::launch(a, head_dim, psa::store_kv4_kernel<64>, psa::store_kv4_kernel<128>, cuda_stream, "store launch: ");
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
    return psa::launch(a, head_dim, psa::load_kv4_kernel<64>, psa::load_kv4_kernel<128>, cuda_stream, "load launch: ");
}
