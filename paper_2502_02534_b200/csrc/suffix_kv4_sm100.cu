// Suffix stage over a cache held in 4 bits (layout: kv4.h): each sample's G query rows of one KV head against its own
// generated tokens, in 16-token pages scattered through a pool of cells.  Same place in a step, same partial results
// and same online softmax (running maximum, row sum, un-normalised accumulator, one division at the end) as the bf16 stage.
//
// The cache is never expanded.  With value = s * code + b per (token, group of 32 channels),
//     S[t, row]   = sum_g s[t, g] * (q[row, g] . code[t, g])  +  sum_g b[t, g] * (sum of q[row] over the group)
//     O[row, ch]  = sum_t (p[row, t] * s[t, g]) * (code[t, ch] - 8)  +  sum_t p[row, t] * (b[t, g] + 8 s[t, g])
// so scales multiply scores and probabilities, of which there are 8 per token, instead of 2 D channels per token, and the
// matrix instructions run on the bare codes.  A code becomes a bf16 operand by ONE and-operation: the bit pattern of a small
// whole number n is the subnormal bf16 n * 2^-133, exactly, and a nibble left in place at bits 4-7 is 16 n * 2^-133; the other
// two nibbles of a 16-bit half need one shift for both.  2^64 on the other operand keeps the products in fp32's normal range,
// and the powers of two come out again in constants (scores) or once at the end (outputs).  5 instructions unpack 8 codes of K.
// That bounds the magnitudes: q * 2^64 and p * s * 2^64, with p up to 2^8 while the reference lags, are finite bf16 numbers for q below
// 2^64 and scales of V up to 2^55; p * s * 2^-69 is a normal fp32 number for p = 1 and scales of V from 2^-57 on.
//   * scores: K codes come out of shared memory through ldmatrix with two 16-bit units = 8 channels of one token per
//     register; the four masked forms of that register are A operands of two m16n8k16 products whose B operands hold q in the
//     matching channel order (loaded that way once per block), odd nibbles' q divided by 16.
//   * outputs: V codes come through ldmatrix.trans, so that a register holds one unit (4 channels) of two neighbouring tokens.
//     Rows 0-7 of a product take whole bytes (even code + 16 * odd code, still a subnormal whole number), rows 8-15 the upper
//     nibbles alone; the even channel is their difference, taken once at the end.  4 instructions per 8 codes.
//   * the offset term of the scores is one and a half more products (one for D = 64), parameters x (group sums of q, split into three bf16
//     numbers: 2^-24 relative); the offset term of the outputs is one more product, parameters^T x p.
//   * rounding: p * s and p are rounded to bf16 (2^-8 relative at most, zero mean) before they meet the codes and the offsets.  With
//     codes centred on 8 both terms stay as small as the values themselves; uncentred, their errors would not cancel as the
//     terms do.  The centring is a product with a constant -8 on the same rounded operand, hence exact.
// Bound: HBM at 1.25 * D bytes per (token, KV head) while the unpacking and the products keep up; one block per (sample, KV
// head, token chunk), 4 warps with a private ring of kStages cells each, filled by 16-byte cp.async.
// Measured: 256 samples x U[0, 4096] tokens x 8 heads of 128 channels, 671 MB: 118 us (5.7 TB/s, 0.87 of the measured copy rate) at
// 1965 MHz; the copies alone take 105, the arithmetic alone 110 (284 instructions per page and warp: issue slots 60 % busy, ALU 50 %,
// tensor pipe 45 %).  In long loops under the power limit the clock falls to 1630 MHz and the time follows it, to 141 us.
// The same with heads of 64 channels, 350 MB: 76 us (4.6 TB/s, 0.70 of the copy rate): a page has half the bytes and more than half the instructions.
// Four blocks an SM of 126 registers: five or six (96, 80 registers) spill, 137 and 184 us; two pages at a time 120-124; 2 or 8 warps a
// block 121-124; q re-read from shared memory 121-126; 3 or 5 stages 120-121; one bulk copy a page with a barrier of its own 126; packed
// two-wide fp32 operations 118-119.
// Slots of the last page beyond the sample's length hold whatever the pool held: their scores are set to -inf and their
// parameters to zero, so nothing of them (NaN bit patterns included) reaches a result.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "kv4.h"

namespace psa {
namespace {

constexpr int kWarps = 4;
constexpr int kStages = 4;                // 40 KB a block at D = 128, four blocks an SM
constexpr float kRescaleThreshold = 8.f;  // log2 units: the reference maximum may lag this far behind
constexpr float kTwo64 = 18446744073709551616.f;
constexpr float kUnscaleEven = 590295810358705651712.f;     // 2^69 = 2^133 / 2^64
constexpr float kUnscaleOdd = 36893488147419103232.f;       // 2^65: odd nibbles stand 4 bits higher

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void lds64(uint32_t addr, uint32_t &r0, uint32_t &r1)
{
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];\n" : "=r"(r0), "=r"(r1) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr)
{
    uint32_t r;
    asm volatile("ld.shared.u32 %0, [%1];\n" : "=r"(r) : "r"(addr) : "memory");
    return r;
}
// D(16x8, f32) = A(16x16, bf16, row) * B(16x8, bf16, col)
__device__ __forceinline__ void mma_bf16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// D = C + A * B
__device__ __forceinline__ void mma_bf16_from(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, const float (&c)[4])
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};\n"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
// D += A * B
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// D(16x8, f32) += A(16x8, bf16, row) * B(8x8, bf16, col)
__device__ __forceinline__ void mma_bf16_k8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t b0)
{
    asm("mma.sync.aligned.m16n8k8.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5}, {%6}, {%0,%1,%2,%3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(b0));
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t a)
{
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ float fast_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&v);
}
__device__ __forceinline__ float lo_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

template <int D>
struct Kv4Smem {
    static constexpr int kWarpBytes = kStages * Kv4Cell<D>::kBytes;
    static constexpr int kTotal = kWarps * kWarpBytes;
};

template <int D, int G>
__global__ void __launch_bounds__(kWarps * 32, 4)
suffix_kv4_kernel(const __nv_bfloat16 *__restrict__ q, const unsigned char *__restrict__ pool, int64_t stride_page,
                  int64_t stride_cell, const int32_t *__restrict__ page_indptr, const int32_t *__restrict__ page_indices,
                  const int32_t *__restrict__ suffix_lens, const SuffixItem *__restrict__ items,
                  const SampleInfo *__restrict__ sample_info, int num_q_heads, int chunk_tokens, float scale_log2,
                  float *__restrict__ partial_o, float *__restrict__ partial_lse, int first_of_step)
{
    using C = Kv4Cell<D>;
    using L = Kv4Smem<D>;
    constexpr int NG = C::kGroups;
    constexpr int kChunks = C::kBytes / 16;
    extern __shared__ __align__(128) unsigned char smem_raw[];

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int4 item = __ldg(reinterpret_cast<const int4 *>(items + blockIdx.x));   // plan data, bound long before
    const int s = item.x, kv = item.y, tok0 = item.z, prow0 = item.w;
    // Alone (or first) in its step this grid is a programmatic dependent of whatever precedes it and waits before it touches
    // anything that may have been written there; behind a prefix stage the prefix blocks have waited already.
    if (first_of_step) {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    }
    int S = __ldg(suffix_lens + s);
    S = min(S, __ldg(&sample_info[s].suf_len_bound));
    const int n_tok = min(S - tok0, chunk_tokens);
    if (n_tok <= 0) return;  // the merge stage derives the chunk count from the same length
    const int n_pages = (n_tok + kPageSize - 1) / kPageSize;
    const int my_pages = (n_pages - warp + kWarps - 1) / kWarps;  // pages warp, warp+4, ...
    const int32_t *my_page_ids = page_indices + __ldg(page_indptr + s) + tok0 / kPageSize;

    const uint32_t warp_smem = smem_u32(smem_raw) + warp * L::kWarpBytes;
    const unsigned char *head = pool + int64_t(kv) * stride_cell + lane * 16;

    // page ids 32 at a time per warp: lane l holds the id of page number 32 g + l, for the group in use and the next one
    auto load_ids = [&](int g) {
        const int i = g * 32 + lane;
        return i < my_pages ? __ldg(my_page_ids + warp + i * kWarps) : 0;
    };
    int ids_cur = load_ids(0), ids_nxt = load_ids(1);
    auto issue_page = [&](int i) {   // called with i = 0, 1, 2, ... in order
        if (i > 0 && (i & 31) == 0) {
            ids_cur = ids_nxt;
            ids_nxt = load_ids((i >> 5) + 1);
        }
        const int64_t page = __shfl_sync(0xffffffffu, ids_cur, i & 31);
        if (i < my_pages) {
            const uint32_t dst = warp_smem + (i % kStages) * C::kBytes + lane * 16;
            const unsigned char *src = head + page * stride_page;
#pragma unroll
            for (int c = 0; c < kChunks; c += 32)
                if (c + 32 <= kChunks || lane < kChunks - c) cp_async16(dst + c * 16, src + c * 16);
        }
        cp_async_commit();  // an empty group keeps the group count uniform
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) issue_page(i);

    // ---- Q as B operands (rows lane / 4; rows >= G stay zero).  c = lane % 4 owns channels 8 c .. 8 c + 7 of each group, in
    // the order in which the masked registers of K present them: (0, 4), (1, 5)/16, (2, 6), (3, 7)/16.
    const int qrow = lane >> 2, c4 = lane & 3;
    uint32_t qb[NG][4];
    uint32_t qs0 = 0u, qs1 = 0u, qs2 = 0u;   // group sums of q (times the softmax scale) as three bf16 parts, where the offsets stand
    {
        float gsum[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            uint4 w{};
            if (qrow < G) w = __ldg(reinterpret_cast<const uint4 *>(q + (size_t(s) * num_q_heads + size_t(kv) * G + qrow) * D + g * 32 + c4 * 8));
            const float f[8] = {lo_f32(w.x), hi_f32(w.x), lo_f32(w.y), hi_f32(w.y), lo_f32(w.z), hi_f32(w.z), lo_f32(w.w), hi_f32(w.w)};
            qb[g][0] = pack_bf16(f[0] * kTwo64, f[4] * kTwo64);
            qb[g][1] = pack_bf16(f[1] * (kTwo64 / 16), f[5] * (kTwo64 / 16));
            qb[g][2] = pack_bf16(f[2] * kTwo64, f[6] * kTwo64);
            qb[g][3] = pack_bf16(f[3] * (kTwo64 / 16), f[7] * (kTwo64 / 16));
            float t = ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
            t += __shfl_xor_sync(0xffffffffu, t, 1);
            t += __shfl_xor_sync(0xffffffffu, t, 2);
            gsum[g] = t * scale_log2;
        }
        // parameter row of a token, as pairs: D = 128: {s0 s1} {s2 s3} {b0 b1} {b2 b3};  D = 64: {s0 s1} {b0 b1} of K, then of V
#pragma unroll
        for (int i = 0; i < NG / 2; ++i) {
            const uint32_t part0 = pack_bf16(gsum[2 * i], gsum[2 * i + 1]);
            const float r0 = gsum[2 * i] - lo_f32(part0), r1 = gsum[2 * i + 1] - hi_f32(part0);
            const uint32_t part1 = pack_bf16(r0, r1), part2 = pack_bf16(r0 - lo_f32(part1), r1 - hi_f32(part1));
            if (D == 128 && c4 == 2 + i) { qs0 = part0; qs1 = part1; qs2 = part2; }
            // K's half of the row twice along k, and again in the second half of k: the three parts stand in one product
            if (D == 64 && c4 == 1) { qs0 = part0; qs1 = part2; }
            if (D == 64 && c4 == 3) qs0 = part1;
        }
    }
    const float score_scale = scale_log2 * kUnscaleEven;

    // A thread holds query rows r0 = 2 * (lane % 4) and r0 + 1: scores of tokens u and u + 8, outputs of channels 4 u .. 4 u + 3 of
    // each group, u = lane / 4.
    const int u = lane >> 2, r0 = c4 * 2;
    float o[NG][2][4];   // [group][channels 4u, 4u + 1 | 4u + 2, 4u + 3][rows r0, r0 + 1: even + 16 odd channel | 16 odd channel]
    float ob[4] = {0.f, 0.f, 0.f, 0.f};   // parameters^T p: row u of the parameter row
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int h = 0; h < 2; ++h) o[g][h][0] = o[g][h][1] = o[g][h][2] = o[g][h][3] = 0.f;
    // Minus the reference maximum of rows r0, r0 + 1: what the scores' accumulators start from, so that the products deliver scores
    // relative to it.
    float base[4] = {0.f, 0.f, 0.f, 0.f};   // [0], [1] of tokens u, again for tokens u + 8
    float limit = -INFINITY;   // scores above it move the reference; the first page's do in any case
    float l_part[2] = {0.f, 0.f};

    // row addresses of the matrix loads inside a cell: matrix lane / 8, row lane % 8; matrices = (tokens 0-7, 8-15) x two groups
    const int mat = lane >> 3, mrow = lane & 7;
    const int mtok = (mat & 1) * 8 + mrow;
    uint32_t code_at[NG / 2];
#pragma unroll
    for (int p = 0; p < NG / 2; ++p) code_at[p] = C::chunk(mtok, 2 * p + (mat >> 1));
    // parameter rows: K's as A rows (tokens 0-7, 8-15) with both halves of k alike; V's transposed, tokens 0-7 and 8-15 along k, the
    // second half of the rows a copy that nobody reads.  D = 64: V's half of a row must stay out of the scores, since a zero in q would not
    // keep a NaN among its parameters out; each thread reads its two registers of K's half.
    const uint32_t pk_at = C::kParamOff + (D == 128 ? (lane & 15) * 16 : u * 16 + (c4 & 1) * 4);
    const uint32_t pv_at = C::params(D == 128 ? 1 : 0, 0) + ((mat >> 1) * 8 + mrow) * 16;
    // the centring operand - (8 + 16 * 8) for bytes, - 16 * 8 for upper nibbles, kept in registers
    uint32_t centre[4];
    asm volatile("mov.b32 %0, 0x80888088;\n\tmov.b32 %1, 0x80808080;\n\tmov.b32 %2, 0x80888088;\n\tmov.b32 %3, 0x80808080;"
                 : "=r"(centre[0]), "=r"(centre[1]), "=r"(centre[2]), "=r"(centre[3]));

    // page i of the warp; `last`: some of its slots may lie beyond the length
    auto work = [&](int i, auto last) {
        __syncwarp();
        issue_page(i + kStages - 1);   // refills the slot read in the iteration before
        cp_async_wait<kStages - 1>();
        __syncwarp();

        const uint32_t cell = warp_smem + (i % kStages) * C::kBytes;
        const int valid = n_tok - (warp + i * kWarps) * kPageSize;   // at least 16 unless this is the last page
        if constexpr (last.value) {
            // slots beyond the length get zero as V's parameters
            if ((lane & 15) >= valid) {
                const uint32_t at = cell + C::params(1, 0) + (lane & 15) * 16;
                if (D == 128) asm volatile("st.shared.v2.u32 [%0], {%1, %1};" ::"r"(at + (lane >> 4) * 8), "r"(0) : "memory");
                else asm volatile("st.shared.u32 [%0], %1;" ::"r"(at + (lane >> 4) * 4), "r"(0) : "memory");
            }
            __syncwarp();
        }

        // ---- scores of 16 tokens x 8 rows, in log2 units relative to the row's reference
        float x[4];
        {
            {
                if constexpr (D == 128) {
                    uint32_t a[4];
                    ldmatrix_x4(cell + pk_at, a);
                    mma_bf16_from(x, a[0], a[1], a[2], a[3], qs0, qs1, base);
                    mma_bf16_k8(x, a[0], a[1], qs2);
                } else {
                    const uint32_t a0 = lds32(cell + pk_at), a1 = lds32(cell + pk_at + 128);
                    mma_bf16_from(x, a0, a1, a0, a1, qs0, qs1, base);
                }
            }
            float acc[NG][4];
#pragma unroll
            for (int p = 0; p < NG / 2; ++p) {
                uint32_t w[4];
                ldmatrix_x4(cell + code_at[p], w);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int g = 2 * p + h;
                    const uint32_t lo = w[2 * h], hi = w[2 * h + 1];
                    mma_bf16_first(acc[g], lo & 0x000F000Fu, hi & 0x000F000Fu, lo & 0x00F000F0u, hi & 0x00F000F0u, qb[g][0], qb[g][1]);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int g = 2 * p + h;
                    const uint32_t lo8 = w[2 * h] >> 8, hi8 = w[2 * h + 1] >> 8;
                    mma_bf16(acc[g], lo8 & 0x000F000Fu, hi8 & 0x000F000Fu, lo8 & 0x00F000F0u, hi8 & 0x00F000F0u, qb[g][2], qb[g][3]);
                }
            }
            float sum[4];
            uint32_t sl[2], sh[2];   // scales of tokens u and u + 8
            const uint32_t at = cell + C::params(0, 0) + u * 16;
            if constexpr (D == 128) {
                lds64(at, sl[0], sl[1]);
                lds64(at + 128, sh[0], sh[1]);
            } else {
                sl[0] = lds32(at);
                sh[0] = lds32(at + 128);
            }
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const float a = (g & 1) ? hi_f32(sl[g >> 1]) : lo_f32(sl[g >> 1]), b = (g & 1) ? hi_f32(sh[g >> 1]) : lo_f32(sh[g >> 1]);
#pragma unroll
                for (int t = 0; t < 4; ++t) sum[t] = g == 0 ? (t < 2 ? a : b) * acc[g][t] : fmaf(t < 2 ? a : b, acc[g][t], sum[t]);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) x[t] = fmaf(sum[t], score_scale, x[t]);
        }
        if constexpr (last.value) {
            if (u >= valid) x[0] = x[1] = -INFINITY;
            if (u + 8 >= valid) x[2] = x[3] = -INFINITY;
        }
        const float tmax0 = fmaxf(x[0], x[2]), tmax1 = fmaxf(x[1], x[3]);
        if (__any_sync(0xffffffffu, fmaxf(tmax0, tmax1) > limit)) {
            float rmax0 = tmax0, rmax1 = tmax1;   // over the 8 lanes that hold the same rows
#pragma unroll
            for (int sh = 4; sh < 32; sh <<= 1) {
                rmax0 = fmaxf(rmax0, __shfl_xor_sync(0xffffffffu, rmax0, sh));
                rmax1 = fmaxf(rmax1, __shfl_xor_sync(0xffffffffu, rmax1, sh));
            }
            // the reference moves to the row's maximum: down only the first time, when nothing has been summed yet
            const bool first = i == 0;
            const float d0 = first ? rmax0 : fmaxf(rmax0, 0.f), d1 = first ? rmax1 : fmaxf(rmax1, 0.f);
            if (!first) {
                const float alpha0 = fast_exp2(-d0), alpha1 = fast_exp2(-d1);
                l_part[0] *= alpha0; l_part[1] *= alpha1;
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int h = 0; h < 2; ++h) { o[g][h][0] *= alpha0; o[g][h][1] *= alpha1; o[g][h][2] *= alpha0; o[g][h][3] *= alpha1; }
                ob[0] *= alpha0; ob[1] *= alpha1;
            }
            x[0] -= d0; x[2] -= d0; x[1] -= d1; x[3] -= d1;
            base[0] -= d0; base[1] -= d1;
            base[2] = base[0]; base[3] = base[1];
            limit = kRescaleThreshold;
        }

        {
            float p[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) p[t] = fast_exp2(x[t]);  // masked slots: exp2(-inf) = 0
            l_part[0] += p[0] + p[2];
            l_part[1] += p[1] + p[3];

            // ---- outputs.  The offset term: parameters^T (rows: the 8 units of a parameter row) x p
            {
                uint32_t a[4];
                ldmatrix_x4_trans(cell + pv_at, a);
                mma_bf16(ob, a[0], a[1], a[2], a[3], movmatrix_trans(pack_bf16(p[0], p[1])), movmatrix_trans(pack_bf16(p[2], p[3])));
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) p[t] *= kTwo64;
            uint32_t sl[2], sh[2];
            const uint32_t at = cell + C::params(1, 0) + u * 16;
            if constexpr (D == 128) {
                lds64(at, sl[0], sl[1]);
                lds64(at + 128, sh[0], sh[1]);
            } else {
                sl[0] = lds32(at);
                sh[0] = lds32(at + 128);
            }
#pragma unroll
            for (int pr = 0; pr < NG / 2; ++pr) {
                uint32_t w[4], pb0[2], pb1[2];
                ldmatrix_x4_trans(cell + C::kCodeBytes + code_at[pr], w);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float a = h ? hi_f32(sl[pr]) : lo_f32(sl[pr]), b = h ? hi_f32(sh[pr]) : lo_f32(sh[pr]);
                    pb0[h] = movmatrix_trans(pack_bf16(p[0] * a, p[1] * a));
                    pb1[h] = movmatrix_trans(pack_bf16(p[2] * b, p[3] * b));
                }
                // rows 0-7: whole bytes (even code + 16 odd code), rows 8-15: their upper nibbles; bytes 0, 2 and bytes 1, 3
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t lo = w[2 * h], hi = w[2 * h + 1];
                    const uint32_t lo1 = __byte_perm(lo, 0u, 0x4341), hi1 = __byte_perm(hi, 0u, 0x4341);
                    mma_bf16(o[2 * pr + h][0], lo & 0x00FF00FFu, lo & 0x00F000F0u, hi & 0x00FF00FFu, hi & 0x00F000F0u, pb0[h], pb1[h]);
                    mma_bf16(o[2 * pr + h][1], lo1, lo1 & 0x00F000F0u, hi1, hi1 & 0x00F000F0u, pb0[h], pb1[h]);
                }
                // - 8 for every code, on the same rounded operand
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    mma_bf16(o[2 * pr + h][0], centre[0], centre[1], centre[2], centre[3], pb0[h], pb1[h]);
                    mma_bf16(o[2 * pr + h][1], centre[0], centre[1], centre[2], centre[3], pb0[h], pb1[h]);
                }
            }
        }
    };
    int i = 0;
    for (; i + 1 < my_pages; ++i) work(i, std::false_type{});
    if (i < my_pages) work(i, std::true_type{});
    cp_async_wait<0>();

    // ---- finish the row sums over the 8 lanes that share the rows, then combine the 4 warps through shared memory
    float l_row[2] = {l_part[0], l_part[1]};
#pragma unroll
    for (int sh = 4; sh < 32; sh <<= 1) {
        l_row[0] += __shfl_xor_sync(0xffffffffu, l_row[0], sh);
        l_row[1] += __shfl_xor_sync(0xffffffffu, l_row[1], sh);
    }
    __syncthreads();  // every warp is done with its ring: reuse the memory
    float *sm_o = reinterpret_cast<float *>(smem_raw);           // [kWarps][G][D]
    float *sm_m = sm_o + kWarps * G * D;                          // [kWarps][G]
    float *sm_l = sm_m + kWarps * G;                              // [kWarps][G]
    // unit of V's scale and of its offset of group g in the parameter row
    constexpr int kScaleUnit = D == 128 ? 0 : 4, kOffsetUnit = D == 128 ? 4 : 6;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float sum_s = __shfl_sync(0xffffffffu, ob[h], (kScaleUnit + g) * 4 + c4);
            const float sum_b = __shfl_sync(0xffffffffu, ob[h], (kOffsetUnit + g) * 4 + c4);
            const float offset = fmaf(8.f, sum_s, sum_b);
            if (r0 + h < G) {
                const float4 v = make_float4(fmaf(o[g][0][h] - o[g][0][2 + h], kUnscaleEven, offset), fmaf(o[g][0][2 + h], kUnscaleOdd, offset),
                                             fmaf(o[g][1][h] - o[g][1][2 + h], kUnscaleEven, offset), fmaf(o[g][1][2 + h], kUnscaleOdd, offset));
                *reinterpret_cast<float4 *>(sm_o + (warp * G + r0 + h) * D + g * 32 + u * 4) = v;
            }
        }
    }
    if (u == 0) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (r0 + h < G) {
                sm_m[warp * G + r0 + h] = my_pages > 0 ? -base[h] : -INFINITY;
                sm_l[warp * G + r0 + h] = l_row[h];
            }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < G * D / 4; e += kWarps * 32) {
        const int g = e / (D / 4), d = e % (D / 4) * 4;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sm_m[w * G + g]);
        float z = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float mw = sm_m[w * G + g];
            const float f = mw == -INFINITY ? 0.f : fast_exp2(mw - top);
            const float4 v = *reinterpret_cast<const float4 *>(sm_o + (w * G + g) * D + d);
            z += f * sm_l[w * G + g];
            acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
        }
        *reinterpret_cast<float4 *>(partial_o + size_t(prow0 + g) * D + d) = make_float4(acc.x / z, acc.y / z, acc.z / z, acc.w / z);
        if (d == 0) partial_lse[prow0 + g] = (top + log2f(z)) * 0.6931471805599453f;
    }
    if (!first_of_step) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

template <int D, int G>
int launch_one(const SuffixKv4Args &a, cudaStream_t st)
{
    using L = Kv4Smem<D>;
    static_assert(L::kTotal >= int(sizeof(float)) * kWarps * G * (D + 2), "combine buffer must fit in the ring");
    auto kern = suffix_kv4_kernel<D, G>;
    static PerDeviceOnce once;   // per instantiation
    const int cfg_rc = once.ensure([&] {
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kTotal);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
        return int(e);
    });
    if (cfg_rc != 0) return cfg_rc;
    cudaLaunchConfig_t lc{};
    lc.gridDim = dim3(a.num_items);
    lc.blockDim = dim3(kWarps * 32);
    lc.dynamicSmemBytes = L::kTotal;
    lc.stream = st;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = &attr;
    lc.numAttrs = 1;
    return int(cudaLaunchKernelEx(&lc, kern, static_cast<const __nv_bfloat16 *>(a.q), static_cast<const unsigned char *>(a.pool),
                                  a.stride_page, a.stride_cell, a.page_indptr, a.page_indices, a.suffix_lens, a.items, a.sample_info,
                                  a.num_q_heads, a.chunk_tokens, a.sm_scale * 1.4426950408889634f, a.partial_o, a.partial_lse,
                                  a.after_prefix ? 0 : 1));
}

}  // namespace

int launch_suffix_kv4(const SuffixKv4Args &a, void *stream, std::string *err)
{
    if (a.num_items == 0) return 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int G = a.num_q_heads / a.num_kv_heads;
    int rc = -1;
#define PSA_CASE(DD, GG) if (a.head_dim == DD && G == GG) rc = launch_one<DD, GG>(a, st);
    PSA_CASE(128, 1) PSA_CASE(128, 2) PSA_CASE(128, 4) PSA_CASE(128, 8)
    PSA_CASE(64, 1) PSA_CASE(64, 2) PSA_CASE(64, 4) PSA_CASE(64, 8)
#undef PSA_CASE
    if (rc != 0 && err) *err = rc < 0 ? "suffix (4-bit): unsupported shape" : std::string("suffix (4-bit) launch: ") + cudaGetErrorString(cudaError_t(rc));
    return rc;
}

}  // namespace psa
