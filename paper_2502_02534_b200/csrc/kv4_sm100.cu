// The 4-bit K/V cache's writer and reader: quantise the K/V rows of new tokens into the cells of their slots, and turn
// cached tokens back into bf16 rows (the layout is described in kv4.h).
//
// Quantisation of a group of 32 channels: b = min, s = bf16((max - min) / 15), code = rint((x - b) / s), 0 where s = 0.
// b is one of the inputs, hence exact; s is rounded once, to the bf16 it is stored as (half a step of 2^-8, which moves the
// top level by at most 0.03 of a step), and the codes are chosen against the rounded s.  Differences, quotients and
// roundings are IEEE fp32, so the codes do not depend on who computes them.  A group whose range is not finite (a NaN, an
// infinity, or a range beyond fp32) gets s = NaN: it reads back as NaN.
//
// Work: 16 bytes of bf16 (8 channels) per thread and row, four threads per group, K and V of a row in the same thread;
// the group's minimum and maximum need two shuffles.  The quotient is one multiplication by the correctly rounded 1 / s and
// one residual step, which rounds exactly like the division (Markstein) as long as nothing under- or overflows; other
// groups take the division itself.  Both kernels are bound by HBM: 4 bytes read and 1.25 written per channel pair of K and
// V, or the reverse.
#include <cuda_runtime.h>

#include <algorithm>
#include <string>

#include "kv4.h"

namespace psa {
namespace {

constexpr int kKv4Threads = 256;

struct Kv4Args {
    const __nv_bfloat16 *in_k, *in_v;   // store: [T, Hkv, D]
    __nv_bfloat16 *out_k, *out_v;       // load
    int64_t stride_tok, stride_head;    // elements
    const int64_t *slot_map;
    int64_t num_tokens;
    int num_kv_heads;
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
    float s = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(hi_f32(hi) - b, 15.f)));
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
        const float inv = __frcp_rn(s);
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

template <int D>
__global__ void __launch_bounds__(kKv4Threads)
store_kv4_kernel(Kv4Args a)
{
    using C = Kv4Cell<D>;
    constexpr int kPerRow = D / 8;                       // threads of one (token, head) row; rows never straddle a warp
    const int lane = threadIdx.x % kPerRow, g = lane >> 2;
    const int64_t rows = a.num_tokens * a.num_kv_heads;
    const int64_t per_grid = int64_t(gridDim.x) * (kKv4Threads / kPerRow);
    const int64_t rounds = (rows + per_grid - 1) / per_grid;   // the same for all threads: the shuffles are warp-wide
    int64_t row = int64_t(blockIdx.x) * (kKv4Threads / kPerRow) + threadIdx.x / kPerRow;
    for (int64_t i = 0; i < rounds; ++i, row += per_grid) {
        const bool live = row < rows;
        const int64_t t = live ? row / a.num_kv_heads : 0;
        const int head = live ? int(row - t * a.num_kv_heads) : 0;
        const int64_t slot = live ? a.slot_map[t] : -1;
        uint4 k{}, v{};
        if (slot >= 0) {
            const int64_t at = t * a.stride_tok + head * a.stride_head + lane * 8;
            k = __ldg(reinterpret_cast<const uint4 *>(a.in_k + at));
            v = __ldg(reinterpret_cast<const uint4 *>(a.in_v + at));
        }
        const Quantised qk = quantise(k), qv = quantise(v);
        unsigned char *cell = cell_of(a, slot, head);
        if (!cell) continue;
        const int tok = int(slot % kPageSize);
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
    const int64_t rows = a.num_tokens * a.num_kv_heads;
    const int64_t per_grid = int64_t(gridDim.x) * (kKv4Threads / kPerRow);
    for (int64_t row = int64_t(blockIdx.x) * (kKv4Threads / kPerRow) + threadIdx.x / kPerRow; row < rows; row += per_grid) {
        const int64_t t = row / a.num_kv_heads;
        const int head = int(row - t * a.num_kv_heads);
        const int64_t slot = a.slot_map[t];
        const unsigned char *cell = cell_of(a, slot, head);
        if (!cell) continue;
        const int tok = int(slot % kPageSize);
        const int at = C::chunk(tok, g) + (lane & 3) * 4;
        const uint32_t ck = *reinterpret_cast<const uint32_t *>(cell + at), cv = *reinterpret_cast<const uint32_t *>(cell + C::kCodeBytes + at);
        const uint16_t *pk = reinterpret_cast<const uint16_t *>(cell + C::params(0, tok)) + g;
        const uint16_t *pv = reinterpret_cast<const uint16_t *>(cell + C::params(1, tok)) + g;
        const uint4 k = dequantise(ck, pk[0], pk[C::kGroups]), v = dequantise(cv, pv[0], pv[C::kGroups]);
        const int64_t to = t * a.stride_tok + head * a.stride_head + lane * 8;
        *reinterpret_cast<uint4 *>(a.out_k + to) = k;
        *reinterpret_cast<uint4 *>(a.out_v + to) = v;
    }
}

bool misaligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

psa_status_t check(const Kv4Args &a, const void *k, const void *v, const int64_t kv_strides[2], int head_dim, const int64_t pool_strides[2])
{
    if (a.num_tokens < 0 || a.num_kv_heads <= 0 || a.num_pool_pages < 0) return set_last_error(PSA_ERR_INVALID_ARG, "negative sizes or no KV head");
    if (head_dim != 64 && head_dim != 128) return set_last_error(PSA_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
    if (a.num_tokens > 0x7fffffff || a.num_kv_heads > 65536) return set_last_error(PSA_ERR_UNSUPPORTED, "problem too large");
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
psa_status_t launch(const Kv4Args &a, int head_dim, K64 k64, K128 k128, void *cuda_stream, const char *what)
{
    const int64_t threads = a.num_tokens * a.num_kv_heads * (head_dim / 8);
    const unsigned blocks = unsigned(std::min<int64_t>((threads + kKv4Threads - 1) / kKv4Threads, 148 * 64));
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
