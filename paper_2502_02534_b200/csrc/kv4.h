// Layout of the 4-bit K/V cache, shared by the kernels that write it, read it back and attend over it.
//
// A cell holds the 16 tokens of one page for one KV head, K and V, in 20 * D consecutive bytes:
//   [0, 8 D)      K codes     16-byte chunk (token t, group g of 32 channels) at chunk index t * NG + (g ^ swizzle(t));
//                             byte i of a chunk: channel 32 g + 2 i in the low nibble, 32 g + 2 i + 1 in the high one
//   [8 D, 16 D)   V codes     the same
//   [16 D, 20 D)  parameters  bf16, one scale and one offset per (token, group):
//                   D = 128   K: 16 rows of 16 bytes {s0 s1 s2 s3 b0 b1 b2 b3}, then V the same
//                   D =  64   16 rows of 16 bytes {K s0 s1 b0 b1, V s0 s1 b0 b1}
// value = s * code + b.  The swizzle spreads the chunks that one 8x8 matrix load of the attention kernel reads (one
// group, eight tokens) over all shared-memory banks; a page is copied to shared memory as it is.
#pragma once

#include <cuda_bf16.h>
#include <cstdint>

#include "psa_internal.h"

namespace psa {

constexpr int kKv4Group = 32;   // channels that share a scale and an offset

template <int D>
struct Kv4Cell {
    static constexpr int kGroups = D / kKv4Group;
    static constexpr int kCodeBytes = kPageSize * D / 2;      // K or V
    static constexpr int kParamOff = 2 * kCodeBytes;
    static constexpr int kBytes = 20 * D;
    static_assert(kParamOff + kPageSize * kGroups * 8 == kBytes, "two bf16 pairs per (token, group)");
    __host__ __device__ static constexpr int swizzle(int t) { return D == 128 ? (t >> 1) & 3 : (t >> 2) & 1; }
    // byte offset of chunk (token, group) inside the K codes or inside the V codes
    __host__ __device__ static constexpr int chunk(int t, int g) { return 16 * (t * kGroups + (g ^ swizzle(t))); }
    // byte offset of the parameters {s0 .. , b0 ..} of a token: which = 0 for K, 1 for V
    __host__ __device__ static constexpr int params(int which, int t)
    {
        return kParamOff + (D == 128 ? which * 16 * kPageSize + t * 16 : t * 16 + which * 8);
    }
};

}  // namespace psa
