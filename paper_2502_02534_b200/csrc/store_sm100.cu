// Rows of K and V written into the slots of a paged bf16 cache (psa_store_kv): pool[page(slot), head, slot % 16, :] <- row.
//
// A copy with scattered rows: every byte is read and written once, so memory is the bound.  A row of a token and head is D / 8 threads of
// 16 bytes; a thread moves the same piece of K and V of kRows rows, all loads of which are in flight before the first store.
#include <cuda_runtime.h>

#include <string>

#include "psa_internal.h"

namespace psa {
namespace {

constexpr int kThreads = 256, kRows = 4;

struct StoreArgs {
    const uint4 *k, *v;                    // strides in pieces of 16 bytes
    uint4 *pool_k, *pool_v;
    int64_t stride_tok, stride_head, pool_page, pool_head, pool_slot, num_pool_pages;
    const int64_t *slots;
    uint32_t rows, heads;                  // tokens x heads
    int32_t *status;
};

template <int kPieces>   // of 16 bytes in a row
__global__ void __launch_bounds__(kThreads)
store_kernel(StoreArgs a)
{
    constexpr uint32_t kAbreast = kThreads / kPieces;
    const uint32_t piece = threadIdx.x % kPieces;
    const uint32_t first = blockIdx.x * (kAbreast * kRows) + threadIdx.x / kPieces;
    uint4 k[kRows], v[kRows];
    int64_t to[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const uint32_t row = first + i * kAbreast;
        to[i] = -1;
        if (row < a.rows) {
            const uint32_t token = row / a.heads, head = row - token * a.heads;
            const int64_t slot = a.slots[token];
            const int64_t page = slot >> 4;
            if (slot >= 0) {
                if (page >= a.num_pool_pages) {
                    if (a.status) atomicCAS(a.status, 0, int(PSA_ERR_BOUNDS));
                } else {
                    const int64_t from = token * a.stride_tok + head * a.stride_head + piece;
                    k[i] = __ldcs(a.k + from);
                    v[i] = __ldcs(a.v + from);
                    to[i] = page * a.pool_page + head * a.pool_head + (slot & (kPageSize - 1)) * a.pool_slot + piece;
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i)
        if (to[i] >= 0) {
            a.pool_k[to[i]] = k[i];
            a.pool_v[to[i]] = v[i];
        }
}

bool misaligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

}  // namespace
}  // namespace psa

extern "C" psa_status_t psa_store_kv(const void *new_k, const void *new_v, const int64_t kv_strides[2], const int64_t *slot_map, int64_t num_tokens,
                                     int32_t num_kv_heads, int32_t head_dim, void *k_pool, void *v_pool, const int64_t pool_strides[3],
                                     int64_t num_pool_pages, int32_t *status, void *cuda_stream)
{
    using namespace psa;
    if (num_tokens < 0 || num_kv_heads <= 0 || num_pool_pages < 0) return set_last_error(PSA_ERR_INVALID_ARG, "negative sizes or no KV head");
    if (head_dim != 64 && head_dim != 128) return set_last_error(PSA_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
    if (num_kv_heads > 65536 || num_tokens > 0x7fffffff / num_kv_heads)
        return set_last_error(PSA_ERR_UNSUPPORTED, "at most 2^31 - 1 rows (tokens x KV heads) per call");
    if (misaligned(status, 4)) return set_last_error(PSA_ERR_INVALID_ARG, "the status word must be 4-byte aligned");
    if (num_tokens == 0) return PSA_OK;
    if (!new_k || !new_v || !kv_strides || !slot_map || !pool_strides || (num_pool_pages > 0 && (!k_pool || !v_pool)))
        return set_last_error(PSA_ERR_INVALID_ARG, "null K/V cache argument");
    if (misaligned(new_k, 16) || misaligned(new_v, 16) || misaligned(k_pool, 16) || misaligned(v_pool, 16) || misaligned(slot_map, 8))
        return set_last_error(PSA_ERR_INVALID_ARG, "K, V and the pools must be 16-byte aligned, slot_map 8-byte aligned");
    for (int i = 0; i < 2; ++i)
        if (kv_strides[i] <= 0 || kv_strides[i] % 8) return set_last_error(PSA_ERR_INVALID_ARG, "K/V strides must be positive multiples of 8 elements");
    for (int i = 0; i < 3; ++i)
        if (pool_strides[i] <= 0 || pool_strides[i] % 8) return set_last_error(PSA_ERR_INVALID_ARG, "pool strides must be positive multiples of 8 elements");
    StoreArgs a{};
    a.k = static_cast<const uint4 *>(new_k); a.v = static_cast<const uint4 *>(new_v);
    a.pool_k = static_cast<uint4 *>(k_pool); a.pool_v = static_cast<uint4 *>(v_pool);
    a.stride_tok = kv_strides[0] / 8; a.stride_head = kv_strides[1] / 8;
    a.pool_page = pool_strides[0] / 8; a.pool_head = pool_strides[1] / 8; a.pool_slot = pool_strides[2] / 8;
    a.num_pool_pages = num_pool_pages; a.slots = slot_map; a.status = status;
    a.heads = uint32_t(num_kv_heads); a.rows = uint32_t(num_tokens) * a.heads;
    const uint32_t per_block = kThreads / (head_dim / 8) * kRows;
    const unsigned blocks = unsigned((uint64_t(a.rows) + per_block - 1) / per_block);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (head_dim == 128) store_kernel<16><<<blocks, kThreads, 0, st>>>(a);
    else store_kernel<8><<<blocks, kThreads, 0, st>>>(a);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return set_last_error(PSA_ERR_CUDA, std::string("store launch: ") + cudaGetErrorString(e));
    return PSA_OK;
}
