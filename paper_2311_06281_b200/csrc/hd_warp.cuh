// Products of a warp for the delta rule: mma.sync with bf16 operands in shared memory or in registers, float32 accumulators.
//
// A float32 factor enters a product as bf16 terms (the first 8 bits, the next 8, ..); `products` forms all pairs of terms up to
// a level, the small ones first.  Two terms of either factor and level 1: 16 bits; three and level 2: float32's 24.
#pragma once
#include "ha_common.cuh"

namespace hd {

using ha::smem_addr;

// Accumulators of 16 x 8: lane l holds rows l / 4 and l / 4 + 8, columns 2 (l % 4) and the next, as {row, row, row + 8, row + 8}.
// Two of them side by side have the layout of a 16 x 16 A operand: sums become the next product's factor in registers.
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void load4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void load4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void store4_t(uint32_t addr, const uint32_t (&r)[4]) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}

// d[2 n], d[2 n + 1] += a * b[n] for `pairs` (a constant, at most kPairs) pairs of accumulators side by side; b[n]: for each term {the
// first one's first half of k, second half, the second one's, ..}.  Independent sums in turn: one warp alone on its scheduler keeps
// the pipe busy with four.
template <int kLevel, int kA, int kB, int kPairs>
__device__ __forceinline__ void products(float (*d)[4], const uint32_t (&a)[kA][4], const uint32_t (&b)[kPairs][kB][4], int pairs = kPairs) {
#pragma unroll
    for (int level = kLevel; level >= 0; --level)
#pragma unroll
        for (int i = 0; i < kA; ++i)
            if (level - i >= 0 && level - i < kB)
#pragma unroll
                for (int n = 0; n < kPairs; ++n)
                    if (n < pairs) {
                        mma(d[2 * n], a[i], b[n][level - i][0], b[n][level - i][1]);
                        mma(d[2 * n + 1], a[i], b[n][level - i][2], b[n][level - i][3]);
                    }
}
// The same where 24 bits are asked for.  The tensor core cuts its sums off instead of rounding them, always towards zero: here the
// terms' products are summed by themselves, the small ones first, and added once (float32 prompts with keys 128 wide: 1.1e-6 off
// without, 1.3e-7 with).
template <int kLevel, int kA, int kB, int kPairs>
__device__ __forceinline__ void rounded_products(float (*d)[4], const uint32_t (&a)[kA][4], const uint32_t (&b)[kPairs][kB][4], int pairs = kPairs) {
    float t[2 * kPairs][4] = {};
    products<kLevel>(t, a, b, pairs);
#pragma unroll
    for (int n = 0; n < 2 * kPairs; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n < 2 * pairs) d[n][e] += t[n][e];
}
template <bool kRounded, int kLevel, int kA, int kB, int kPairs>
__device__ __forceinline__ void sum(float (*d)[4], const uint32_t (&a)[kA][4], const uint32_t (&b)[kPairs][kB][4], int pairs = kPairs) {
    if constexpr (kRounded) rounded_products<kLevel>(d, a, b, pairs);
    else products<kLevel>(d, a, b, pairs);
}

// Two accumulators as the terms of an A operand
template <int kTerms>
__device__ __forceinline__ void as_operand(uint32_t (&a)[kTerms][4], const float (&d0)[4], const float (&d1)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float* d = i < 2 ? d0 : d1;
        uint32_t t[kTerms];
        ha::split<kTerms>(ha::make_pair2(d[2 * (i & 1)], d[2 * (i & 1) + 1]), t);
#pragma unroll
        for (int u = 0; u < kTerms; ++u) a[u][i] = t[u];
    }
}

// Tiles in shared memory hold 16-byte pieces, permuted within a row so that eight rows' pieces at one place lie in different
// banks: rows of 128 bytes (64 bf16, blocks of columns one behind the other; TMA's 128-byte swizzle), of 64 and of 32 bytes.
template <int kBytes> __device__ __forceinline__ uint32_t place(int row, int piece) {
    static_assert(kBytes == 128 || kBytes == 64 || kBytes == 32, "row");
    constexpr int kPieces = kBytes / 16, kShift = kBytes == 128 ? 0 : kBytes == 64 ? 1 : 2;
    return row * kBytes + ((piece ^ ((row >> kShift) & (kPieces - 1))) << 4);
}
// kRows x any columns of bf16, blocks of 64 columns
template <int kRows> __device__ __forceinline__ uint32_t wide(int row, int piece) { return (piece >> 3) * (kRows * 128) + place<128>(row, piece & 7); }

// Which row and piece a lane names for load4: four 8 x 8 matrices
struct Lane {
    int lane = threadIdx.x & 31, low = lane & 7, bit3 = (lane >> 3) & 1, bit4 = lane >> 4;
    __device__ __forceinline__ int b_row() const { return low + 8 * bit4; }   // B [n][k]: two n tiles, both halves of k; B^T of a V tile
    __device__ __forceinline__ int b_piece() const { return bit3; }
    __device__ __forceinline__ int bt_row() const { return low + 8 * bit3; }  // B [k][n], transposed by the load
    __device__ __forceinline__ int bt_piece() const { return bit4; }
    __device__ __forceinline__ int a_row() const { return low + 8 * bit3; }   // A [m][k]
    __device__ __forceinline__ int a_piece() const { return bit4; }
    __device__ __forceinline__ int at_row() const { return low + 8 * bit4; }  // A [k][m], transposed by the load
    __device__ __forceinline__ int at_piece() const { return bit3; }
};

// A linear copy from global memory (16-byte aligned, a multiple of 16 bytes)
__device__ __forceinline__ void bulk_load(uint32_t to, const void* from, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar)
                 : "memory");
}

}  // namespace hd
