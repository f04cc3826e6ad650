// scan_kernel and back_kernel (hd_scan.cuh, hd_grad.cuh) on tcgen05: bf16, keys up to 128 wide, chunks of 64 tokens.
//
// A CTA has 128 columns of the values and all of the state's rows for them, S^T in registers (two threads to a column of V), and
// walks the chunks.  Everything is formed transposed, columns of V as rows of the tensor core's tiles:
//     X = S^T K^T,   Y = V^T - X e^c,   E = Y + (-beta Y) N^T,   S^T <- e^{c_C} S^T + (e^{c_C-c} beta E) K
// Left factors go from registers to tensor memory as bf16 terms, three for what the state hangs on (24 bits), sums come back from there;
// V^T is brought there by products with an identity.  Backward likewise from D^T:
//     X = D^T K^T,   dV'^T = X e^{c_C-c} + dO^T P,   F = dV'^T + (-beta dV'^T) N,   Z = beta F
//     D^T <- e^{c_C} D^T + (-e^c Z) K + (scale e^c dO^T) Q
// Warps 0-7 have the state and the chain of dependent steps; warps 8-15 what hangs on it without the chain waiting: the output
// (backward: dV, F and the sums over V for the gates, and the terms of dO).  One warp loads, a chunk ahead, one issues the products.
//
// Bound by the chain: a chunk takes 8900 clocks (products of X 1290, their sums scaled and split 1150, the solution 1200, E 1600, the
// update's products 1370, the state read, decayed and split anew 2150), the tensor pipe is busy 29% of them, HBM 12%.  64 (batch, head)
// pairs of 2048 tokens, keys and values 128 wide: 172 us; 128 pairs: 180 us forward, 180 us for the states, 257 us backward.  Of that 4% are
// the waits and the sums in places of their own that the order of the products needs.  mma.sync against it: many_slices in hd_host.h.
#pragma once
#include "hd_scan.cuh"

namespace hd {

constexpr int kPassThreads = 640;
// Registers: 96 a thread at launch; 2 * 136 + 2 * 80 + 48 = 5 * 96.
constexpr int kPassState = 136, kPassSide = 80, kPassFeed = 48;
static_assert(2 * kPassState + 2 * kPassSide + kPassFeed <= 5 * 96, "registers");

constexpr uint32_t kRows32 = (256u >> 4) | (1u << 14) | (6u << 29);  // operands of 32-byte rows, swizzled so
template <uint32_t kA, uint32_t kB>
__device__ __forceinline__ void mma_tile(uint32_t d, uint32_t a, uint32_t b, uint32_t shape, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.u32 p, %6, 0;\n\tmov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;\n\t}" ::"r"(d), "r"(a), "r"(kA), "r"(b), "r"(kB), "r"(shape), "r"((uint32_t)add)
                 : "memory");
}
// The same with the left factor in tensor memory
template <uint32_t kB>
__device__ __forceinline__ void mma_left(uint32_t d, uint32_t a, uint32_t b, uint32_t shape, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 b, {%2, %3};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(kB), "r"(shape), "r"((uint32_t)add)
                 : "memory");
}

// Tensor memory, in columns.  The update shares columns with the state's terms, V' (backward: dO) with X, and the later of two
// factors with the earlier: each is written when the products that read the other are done, which a barrier says.  Products are in
// the order in which they are issued only where accumulator and shape are the same: sums in the same columns all have one shape, or a
// barrier between them.
template <int kMode> struct PassColumns {
    static constexpr uint32_t s = 0, x = 192, y = 256, o = 320, f = 384, g = 480, columns = 512;
    // What the solution adds to Y (dV'), by itself: the tensor core cuts off what it adds, and Y is the larger.  N is triangular: the block
    // of 16 factors that reaches all tokens adds to the 64 columns of `solved`, the next to 48 of `second` (from the block of
    // tokens that it starts with on), the other two to two blocks of 16 in `third`.  The first is where the state's last terms were, which X
    // alone reads; the others are where its first ones were, or, where those still meet Q, in X (each half of the warps then writes V'
    // where it alone has read) and in columns that only the backward pass has another use for.
    static constexpr uint32_t solved = s + 128, second = kMode == 0 ? x : s, third = kMode == 0 ? g : s + 64;
    // term t of sixteen rows q of a thread's half of the state: its first two terms lie where its own half of the update will
    static __device__ __forceinline__ constexpr uint32_t state(int half, int q, int t) { return t < 2 ? s + half * 64 + q * 16 + t * 8 : s + 128 + half * 32 + q * 8; }
    static __device__ __forceinline__ constexpr uint32_t factor(int jj, int t) { return f + 24 * jj + 8 * t; }
    static __device__ __forceinline__ constexpr uint32_t value(int jj, int t) { return x + 16 * jj + 8 * t; }
    static __device__ __forceinline__ constexpr uint32_t outer(int jj, int t) { return t < 2 ? value(jj, t) : g + 8 * jj; }
};

// kMode 0: the output; 1: the states before the chunks and E for the gradients; 2: backward
template <int KP, int kMode>
struct PassLayout {
    static constexpr int C = 64, kStages = 2;
    static constexpr int kTermsP = kMode == 0 ? 2 : 3;
    using I = Image<C, 3, kTermsP, kMode != 0>;
    static constexpr uint32_t block = C * 128, tile = KP / 64 * block;
    static constexpr uint32_t k = 0, q = tile, v = kMode == 1 ? tile : 2 * tile, image = v + 2 * block;  // V (backward: dO): 128 columns
    // backward N is wanted by rows
    static constexpr uint32_t n = image + I::n, p = n + 3 * I::plane, bytes = p + (kMode == 1 ? 0 : kTermsP * I::plane), stage = (bytes + 1023) / 1024 * 1024;  // (bytes: of a chunk)
    // backward E^T as well, eight times [token][16]
    static constexpr uint32_t errors = stage, whole = stage + (kMode == 2 ? 8 * C * 64 : 0);
    static constexpr uint32_t ident = kStages * whole, bars = ident + 512, end = bars + 256;
};

// Sixteen values as terms of a left factor
template <int kTerms>
__device__ __forceinline__ void put_left(const uint32_t (&x)[16], uint32_t (&t)[kTerms][8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        uint32_t w[kTerms];
        ha::split<kTerms>(ha::make_pair2(x[2 * e], x[2 * e + 1]), w);
#pragma unroll
        for (int u = 0; u < kTerms; ++u) t[u][e] = w[u];
    }
}
// x[e] = weight[e] * x[e] for sixteen of a chunk's tokens; kPlain: no weight is zero (a weight of zero forgets whatever it is that it weighs)
template <bool kPlain>
__device__ __forceinline__ void weigh(const float* weight, uint32_t (&x)[16]) {
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
        const float4 f = *reinterpret_cast<const float4*>(weight + e);
        const float w[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float y = __uint_as_float(x[e + u]);
            x[e + u] = __float_as_uint(kPlain ? w[u] * y : ha::decayed(w[u], y));
        }
    }
}
// 32 values of each lane, summed over the warp's lanes: lane l gets the sum of the l-th ones.
__device__ __forceinline__ float sum_across(float (&x)[32]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const bool upper = lane & o;
#pragma unroll
        for (int e = 0; e < o; ++e) {
            const float keep = upper ? x[e + o] : x[e], give = upper ? x[e] : x[e + o];
            x[e] = keep + __shfl_xor_sync(~0u, give, o);
        }
    }
    return x[0];
}

enum PassBar : int { kStateReady = 5, kScores, kFactor, kSolved, kWrites, kUpdated, kFar, kFarScaled, kOut, kOutRead, kOuter = kFar, kSolvedRead = kFarScaled,
                     kDrainPass = kOutRead + 1, kPassBars };

template <int KP, int kMode, class T>
__global__ void __launch_bounds__(kPassThreads, 1)
    pass_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, const Params p,
                int* gave_up) {
    using L = PassLayout<KP, kMode>;
    using I = typename L::I;
    using M = PassColumns<kMode>;
    using B = Blocks<64>;
    constexpr int C = 64, kOwn = KP / 2;
    constexpr bool kOutput = kMode == 0, kBack = kMode == 2;
    extern __shared__ __align__(1024) uint8_t sm8[];
    const uint32_t base = smem_addr(sm8), bars = base + L::bars;
    volatile int* const stop = reinterpret_cast<int*>(sm8 + L::bars + 192);
    uint32_t* const s_tmem = reinterpret_cast<uint32_t*>(sm8 + L::bars + 200);
    const Waiter wait{bars, stop, p.spin};
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int slabs = (p.dv + 127) / 128, bh = blockIdx.x / slabs, b = bh / p.heads, h = bh % p.heads, v0 = (blockIdx.x % slabs) * 128;
    const int slices = (p.dv + 15) / 16, here = min(8, slices - v0 / 16), live = live_tokens(p.lengths, b, p.tokens), count = (live + C - 1) / C;
    if (tid == 0) {
        if (blockIdx.x == 0) p.fault->started_id = p.call_id;
        for (int i = 0; i < kPassBars; ++i) {
            uint32_t arrivals = 1;
            if (i >= kEmpty && i < kPatched) arrivals = kMode == 1 ? 9 : 17;  // the warps that read vectors, and the products
            if (i == kStateReady || i == kFactor || i == kWrites) arrivals = 8;
            if (i == kFarScaled || i == kOutRead || (kBack && i == kOuter)) arrivals = 8;
            ha::bar_init(bars + 8 * i, arrivals);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *stop = 0;
    }
    if (tid < 256) {  // the identity, two 8 x 8 core matrices along each of k and n
        const int n = tid >> 4, k = tid & 15;
        *reinterpret_cast<__nv_bfloat16*>(sm8 + L::ident + (k >> 3) * 256 + (n >> 3) * 128 + (n & 7) * 16 + (k & 7) * 2) = __float2bfloat16(n == k ? 1.0f : 0.0f);
    }
    ha::fence_smem_to_async();
    if (warp == 16) ha::tmem_alloc(smem_addr(s_tmem), M::columns);
    ha::tmem_before_sync();
    __syncthreads();
    ha::tmem_after_sync();
    if (tid == 0 && *s_tmem != 0) *stop = 1 + kPassBars;  // all columns were asked for: they start at 0
    auto chunk_at = [&](int it) { return kBack ? count - 1 - it : it; };
    if (warp >= 16) {
        ha::give_registers<kPassFeed>();
        if (warp == 16) {
            // ------------------------------------------------------------------------------------------ loads
            load_chunks<C, L::kStages>(
                wait, sm8, L::whole, L::image, 0, count, live, p.tokens, L::bytes + (kBack ? here * C * 64 : 0), p.mute,
                [&](int n, int s, uint32_t bar) {
                    const uint32_t to = base + s * L::whole;
                    const uint8_t* const image = p.image + ((long long)bh * p.chunks + n) * I::end;
                    bulk_load(to + L::image, image, I::n, bar);
                    bulk_load(to + L::n, image + (kBack ? I::rows : I::n), 3 * I::plane, bar);
                    if (kBack) bulk_load(to + L::errors, p.errors + (((long long)bh * p.chunks + n) * slices + v0 / 16) * 16 * C, here * C * 64, bar);
                    if (kMode != 1) bulk_load(to + L::p, image + I::p, L::kTermsP * I::plane, bar);
                    for (int c = 0; c < KP / 64; ++c) {
                        ha::tma_load_4d(to + L::k + c * L::block, &mk, 64 * c, h / p.kdiv, n * C, b, bar);
                        if (kMode != 1) ha::tma_load_4d(to + L::q + c * L::block, &mq, 64 * c, h / p.qdiv, n * C, b, bar);
                    }
                    for (int c = 0; c < 2; ++c) ha::tma_load_4d(to + L::v + c * L::block, &mv, v0 + 64 * c, kBack ? h : h / p.vdiv, n * C, b, bar);
                },
                kBack);
        } else if (warp == 17) {
            // ------------------------------------------------------------------------------------------ products
            if (ha::elect_one()) {
                constexpr uint32_t shape64 = ha::mma_shape(C, 0), shape_t = ha::mma_shape(16, ha::kColMajorA), shape_u = ha::mma_shape(KP, ha::kColMajorB);
                constexpr uint32_t kN = kBack ? ha::kColMajorB : 0, shape48 = ha::mma_shape(48, kN), shape16 = ha::mma_shape(16, kN);
                const uint32_t ident = ha::operand(base + L::ident, 256);
                auto step = [](int kk) { return (uint32_t)((kk >> 2) * (L::block >> 4) + (kk & 3) * 2); };
                // left factors of KP/16 steps, three terms of the state, with a tile of rows of tokens
                auto with_state = [&](uint32_t d, uint32_t tile, int terms) {
#pragma unroll
                    for (int t = 2; t >= 0; --t)
                        if (t < terms)
#pragma unroll
                            for (int kk = 0; kk < KP / 16; ++kk)
                                mma_left<ha::kSwizzled>(d, M::state(kk / (KP / 32), kk % (KP / 32), t), tile + step(kk), shape64, !(t == terms - 1 && kk == 0));
                };
                auto update = [&](uint32_t tile, bool outer, bool add) {  // D += factor * tile of KP columns
#pragma unroll
                    for (int t = 2; t >= 0; --t)
#pragma unroll
                        for (int jj = 0; jj < 4; ++jj)
                            mma_left<ha::kSwizzled>(M::s, outer ? M::outer(jj, t) : M::factor(jj, t), tile + jj * 128, shape_u, add || t < 2 || jj > 0);
                };
                bool ok = true;
                for (int it = 0; it < count; ++it) {
                    const int st = it % L::kStages;
                    const uint32_t at = base + st * L::whole, K = ha::operand(at + L::k, L::block), Q = ha::operand(at + L::q, L::block),
                                   V = ha::operand(at + L::v, L::block), N = ha::operand(at + L::n, 512), P = ha::operand(at + L::p, 512);
                    if (!(ok = wait(kFull + st, it / L::kStages))) break;
                    ha::tmem_after_sync();
                    if constexpr (kBack) {  // dO^T P, while the state's terms are formed: sixteen tokens j of all ii >= j
#pragma unroll
                        for (int u = 2; u >= 0; --u)
#pragma unroll
                            for (int ii = 3; ii >= 0; --ii)
#pragma unroll
                                for (int j = 0; j <= ii; ++j)
                                    mma_tile<ha::kSwizzled, kRows32>(M::o + 16 * j, V + ii * 128, P + ((u * I::plane + B::by_rows(ii, j) * 512) >> 4),
                                                                     ha::mma_shape(16, ha::kColMajorA | ha::kColMajorB), u < 2 || ii < 3);
                    } else {
#pragma unroll
                        for (int q = 0; q < 4; ++q) ha::mma_ss<ha::plain_layout(128)>(M::y + 16 * q, V + q * 128, ident, shape_t, false);
                    }
                    if (!(ok = wait(kStateReady, it))) break;
                    if constexpr (kOutput)
                        if (it > 0 && !(ok = wait(kOut, it - 1))) break;  // P has met the V' in X's columns
                    ha::tmem_after_sync();
                    with_state(M::x, K, 3);
                    ha::mma_commit(bars + 8 * kScores);
                    if (!(ok = wait(kFactor, it))) break;
                    ha::tmem_after_sync();
#pragma unroll
                    for (int level = 2; level >= 0; --level)
#pragma unroll
                        for (int u = 0; u <= level; ++u) {
                            const bool more = level < 2 || u > 0;
                            // block `n` of the factors, counted from the one that reaches all tokens, with block `i` of the tokens
                            auto left = [&](int n) { return M::factor(kBack ? 3 - n : n, u); };
                            auto block = [&](int i, int n) {
                                return N + (((level - u) * I::plane + (kBack ? B::by_rows(3 - n, i) : B::by_columns(i, n)) * 512) >> 4);
                            };
                            mma_left<kRows32>(M::solved, left(0), block(0, 0), ha::mma_shape(C, kN), more);
                            mma_left<kRows32>(M::second + (kBack ? 0 : 16), left(1), block(kBack ? 0 : 1, 1), shape48, more);
#pragma unroll
                            for (int i = 0; i < 2; ++i) mma_left<kRows32>(M::third + 16 * i, left(2), block(kBack ? i : i + 2, 2), shape16, more);
                            mma_left<kRows32>(M::third + (kBack ? 0 : 16), left(3), block(kBack ? 0 : 3, 3), shape16, true);
                        }
                    ha::mma_commit(bars + 8 * kSolved);
                    if constexpr (kOutput) {  // while the threads work on E
                        if (it > 0 && !(ok = wait(kOutRead, it - 1))) break;
                        ha::tmem_after_sync();
                        with_state(M::o, Q, 2);
                        ha::mma_commit(bars + 8 * kFar);
                    }
                    if (!(ok = wait(kWrites, it))) break;
                    if constexpr (kOutput)
                        if (!(ok = wait(kFar, it))) break;  // Q has met the state's terms in the update's columns
                    ha::tmem_after_sync();
                    update(K, false, false);
                    if constexpr (kBack) {
                        if (!(ok = wait(kOuter, it))) break;
                        ha::tmem_after_sync();
                        update(Q, true, true);
                    }
                    ha::mma_commit(bars + 8 * kUpdated);
                    if constexpr (kOutput) {
                        if (!(ok = wait(kFarScaled, it))) break;
                        ha::tmem_after_sync();
#pragma unroll
                        for (int level = 1; level >= 0; --level)
#pragma unroll
                            for (int t = level; t >= 0; --t)
#pragma unroll
                                for (int jj = 0; jj < 4; ++jj)
#pragma unroll
                                    for (int i = jj; i < 4; ++i)
                                        mma_left<kRows32>(M::o + 16 * i, M::value(jj, t), P + (((level - t) * I::plane + B::by_columns(i, jj) * 512) >> 4), shape16, true);
                        ha::mma_commit(bars + 8 * kOut);
                    }
                    ha::mma_commit(bars + 8 * (kEmpty + st));
                }
                ha::mma_commit(bars + 8 * kDrainPass);  // what was issued ends before the CTA does
                wait.drain(kDrainPass, 0);
            }
            __syncwarp();
        }
    } else if (warp >= 8) {
        ha::give_registers<kPassSide>();
        // ---------------------------------------------------------------------------------------------- beside the chain
        if constexpr (kMode != 1) {
            // a column of V and half of the tokens
            const int row = (warp & 3) * 32 + lane, v = v0 + row, j0 = ((warp - 8) >> 2) * 32;
            const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
            T* const out = static_cast<T*>(p.out) + b * p.ob + h * p.oh + v;
            const bool mine = v < p.dv;
            bool ok = true;
            auto store = [&](int t, float x) {
                if (mine && t < p.tokens && ok) out[t * p.ot] = ha::from_f<T>(t < live ? x : 0.0f);
            };
            for (int it = 0; it < count; ++it) {
                const int st = it % L::kStages, n = chunk_at(it), t0 = n * C;
                const float* const vec = reinterpret_cast<const float*>(sm8 + st * L::whole + L::image) + j0;
                uint32_t x[2][16];
                if constexpr (kOutput) {
                    ok = ok && wait(kFull + st, it / L::kStages) && wait(kFar, it);
                    ha::tmem_after_sync();
#pragma unroll
                    for (int c = 0; c < 2; ++c) ha::tmem_ld16_early(x[c], lanes + M::o + j0 + 16 * c);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        ha::tmem_ready(x[c]);
                        weigh<false>(vec + I::early / 4 + 16 * c, x[c]);
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[c][e] = __float_as_uint(p.scale * __uint_as_float(x[c][e]));
                        ha::tmem_st16(lanes + M::o + j0 + 16 * c, x[c]);
                    }
                    ha::release_reads();
                    ha::tmem_wait_st();
                    ha::tmem_before_sync();
                    ok = __all_sync(~0u, ok);
                    if (lane == 0 && ok) {
                        ha::bar_arrive(bars + 8 * kFarScaled);
                        ha::bar_arrive(bars + 8 * (kEmpty + st));
                    }
                    ok = ok && wait(kOut, it);
                    ha::tmem_after_sync();
#pragma unroll
                    for (int c = 0; c < 2; ++c) ha::tmem_ld16_early(x[c], lanes + M::o + j0 + 16 * c);
#pragma unroll
                    for (int c = 0; c < 2; ++c) ha::tmem_ready(x[c]);
                    ha::tmem_before_sync();
                    ok = __all_sync(~0u, ok);
                    if (lane == 0 && ok) ha::bar_arrive(bars + 8 * kOutRead);
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int e = 0; e < 16; ++e) store(t0 + j0 + 16 * c + e, __uint_as_float(x[c][e]));
                } else {
                    const long long chunk = (long long)bh * p.chunks + n;
                    const long long at = ((chunk * slices + (v >> 4)) * C + j0) * 16 + (v & 15);  // of E and F: [sixteen columns][token][16]
                    const bool counts = (v0 >> 5) + (warp & 3) < p.parts;
                    float* const dots = p.dots + (chunk * 2 * p.parts + (v0 >> 5) + (warp & 3)) * C + j0 + lane;
                    ok = ok && wait(kFull + st, it / L::kStages);
                    const float* const e = reinterpret_cast<const float*>(sm8 + st * L::whole + L::errors) + (row >> 4) * (C * 16) + j0 * 16 + (row & 15);
                    const uint8_t* const go = sm8 + st * L::whole + L::v + (row >> 6) * L::block + j0 * 128;
                    // scale e^c dO^T as terms, where X was
                    auto outer = [&](int c) {
                        uint32_t w[3][8];
#pragma unroll
                        for (int u = 0; u < 16; ++u)
                            x[c][u] = (uint32_t)*reinterpret_cast<const uint16_t*>(go + place<128>(16 * c + u, (row & 63) >> 3) + 2 * (row & 7)) << 16;
                        weigh<true>(vec + I::early / 4 + 16 * c, x[c]);
#pragma unroll
                        for (int u = 0; u < 16; ++u) x[c][u] = __float_as_uint(p.scale * __uint_as_float(x[c][u]));
                        put_left<3>(x[c], w);
#pragma unroll
                        for (int u = 0; u < 3; ++u) ha::tmem_st8(lanes + M::outer(j0 / 16 + c, u), w[u]);
                    };
                    ok = ok && wait(kScores, it);
                    ha::tmem_after_sync();
#pragma unroll
                    for (int c = 0; c < 2; ++c) ha::tmem_ld16_early(x[c], lanes + M::x + j0 + 16 * c);
                    float y[32];  // e^{c_C-c} k^T D V', over this warp's columns
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        ha::tmem_ready(x[c]);
                        weigh<false>(vec + I::late / 4 + 16 * c, x[c]);
#pragma unroll
                        for (int u = 0; u < 16; ++u) y[16 * c + u] = (v >> 4) < slices ? __uint_as_float(x[c][u]) * e[(16 * c + u) * 16] : 0.0f;
                    }
                    ok = ok && wait(kFactor, it);  // X and dO^T P have been read
#pragma unroll
                    for (int c = 0; c < 2; ++c) outer(c);
                    ha::tmem_wait_st();
                    ha::tmem_before_sync();
                    ok = __all_sync(~0u, ok);
                    if (lane == 0 && ok) ha::bar_arrive(bars + 8 * kOuter);
                    const float beta = vec[I::beta / 4 + lane];
                    const float sum = beta * sum_across(y);
                    if (ok && counts) dots[p.parts * C] = sum;
                    ok = ok && wait(kWrites, it);  // F is there
                    ha::tmem_after_sync();
#pragma unroll
                    for (int c = 0; c < 2; ++c) ha::tmem_ld16_early(x[c], lanes + M::y + j0 + 16 * c);
#pragma unroll
                    for (int c = 0; c < 2; ++c) ha::tmem_ready(x[c]);
                    ha::tmem_before_sync();
                    ok = __all_sync(~0u, ok);
                    if (lane == 0 && ok) ha::bar_arrive(bars + 8 * kSolvedRead);
#pragma unroll
                    for (int t = 0; t < 32; ++t) {
                        const float f = __uint_as_float(x[t >> 4][t & 15]);
                        if (ok && (v >> 4) < slices) p.errors_back[at + t * 16] = f;
                        y[t] = (v >> 4) < slices ? f * e[t * 16] : 0.0f;
                    }
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        weigh<true>(vec + I::beta / 4 + 16 * c, x[c]);
#pragma unroll
                        for (int u = 0; u < 16; ++u) store(t0 + j0 + 16 * c + u, __uint_as_float(x[c][u]));
                    }
                    ha::release_reads();
                    __syncwarp();
                    if (lane == 0 && ok) ha::bar_arrive(bars + 8 * (kEmpty + st));
                    const float sum2 = sum_across(y);
                    if (ok && counts) dots[0] = sum2;
                }
            }
            for (long long t = (long long)count * C + (j0 ? 1 : 0); t < p.tokens; t += 2)  // chunks without a token of the sequence
                if (mine) out[t * p.ot] = ha::from_f<T>(0.0f);
        }
    } else {
        ha::take_registers<kPassState>();
        // ---------------------------------------------------------------------------------------------- the state
        const int half = warp >> 2, row = (warp & 3) * 32 + lane, v = v0 + row, k0 = half * kOwn;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const bool mine = v < p.dv;
        float s[kOwn];
        {
            const float* const from = p.s_in ? p.s_in + (long long)bh * p.dk * p.dv : nullptr;
#pragma unroll
            for (int k = 0; k < kOwn; ++k) s[k] = from && mine && k0 + k < p.dk ? from[(long long)(k0 + k) * p.dv + v] : 0.0f;
        }
        bool ok = true;
        auto arrive = [&](int bar) {
            ok = __all_sync(~0u, ok);
            if (lane == 0 && ok) ha::bar_arrive(bars + 8 * bar);
        };
        auto publish = [&]() {  // the state's terms
#pragma unroll
            for (int q = 0; q < kOwn / 16; ++q) {
                uint32_t x[16], w[3][8];
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = __float_as_uint(s[16 * q + e]);
                put_left<3>(x, w);
#pragma unroll
                for (int t = 0; t < 3; ++t) ha::tmem_st8(lanes + M::state(half, q, t), w[t]);
            }
            ha::tmem_wait_st();
            ha::tmem_before_sync();
            arrive(kStateReady);
        };
        if (count > 0) publish();
        for (int it = 0; it < count; ++it) {
            const int st = it % L::kStages, n = chunk_at(it), t0 = n * C;
            const float* const vec = reinterpret_cast<const float*>(sm8 + st * L::whole + L::image);
            const long long chunk = (long long)bh * p.chunks + n;
            ok = ok && wait(kFull + st, it / L::kStages);
            if (kBack && it > 0) ok = ok && wait(kSolvedRead, it - 1);  // F of the chunk before
            ok = ok && wait(kScores, it);
            ha::tmem_after_sync();
            const float whole = vec[I::whole / 4];
            auto factors = [&](auto plain) {  // plain: no weight is zero, and all tokens are the sequence's
                constexpr bool kPlain = decltype(plain)::value;
                uint32_t x[2][16], y[2][16];
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    ha::tmem_ld16_early(x[g], lanes + M::x + 32 * half + 16 * g);
                    ha::tmem_ld16_early(y[g], lanes + (kBack ? M::o : M::y) + 32 * half + 16 * g);
                }
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int jj = 2 * half + g, j = 16 * jj;
                    ha::tmem_ready(x[g]);
                    ha::tmem_ready(y[g]);
                    weigh<kPlain>(vec + (kBack ? I::late : I::early) / 4 + j, x[g]);
                    if constexpr (!kPlain && !kBack)
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (forgotten(vec[I::whole / 4 + 1], vec[I::hi / 4 + j + e])) x[g][e] = __float_as_uint(number(__uint_as_float(x[g][e])));
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float f = kBack ? __uint_as_float(y[g][e]) + __uint_as_float(x[g][e]) : __uint_as_float(y[g][e]) - __uint_as_float(x[g][e]);
                        y[g][e] = __float_as_uint(kPlain || t0 + j + e < live ? f : 0.0f);
                    }
                    ha::tmem_st16(lanes + M::y + j, y[g]);
                    weigh<true>(vec + I::beta / 4 + j, y[g]);
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[g][e] ^= 0x80000000u;
                    uint32_t w[3][8];
                    put_left<3>(y[g], w);
#pragma unroll
                    for (int t = 0; t < 3; ++t) ha::tmem_st8(lanes + M::factor(jj, t), w[t]);
                }
            };
            if (whole != 0.0f && t0 + C <= live) factors(Int<1>{});
            else factors(Int<0>{});
            ha::tmem_wait_st();
            ha::tmem_before_sync();
            arrive(kFactor);
            if constexpr (kMode != 0) {  // the state before the chunk (its gradient after it), while the system is solved: [sixteen columns][k / 4][16][4]
                if (ok && (v >> 4) < slices) {
                    float4* const to = reinterpret_cast<float4*>((kBack ? p.gradients : p.states) + (chunk * slices + (v >> 4)) * 16 * KP) + (k0 / 4) * 16 + (v & 15);
#pragma unroll
                    for (int k = 0; k < kOwn; k += 4) to[k * 4] = make_float4(s[k], s[k + 1], s[k + 2], s[k + 3]);
                }
            }
            ok = ok && wait(kSolved, it);
            ha::tmem_after_sync();
            {
                // whether `third` reaches this half's two blocks of tokens; `second` reaches those and one of the other half's
                const bool far = half == (kBack ? 0 : 1);
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int jj = 2 * half + g, j = 16 * jj;
                    uint32_t x[16], z[16], more[16];
                    auto plus = [](uint32_t (&to)[16], const uint32_t (&y)[16]) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) to[e] = __float_as_uint(__uint_as_float(to[e]) + __uint_as_float(y[e]));
                    };
                    ha::tmem_ld16_early(z, lanes + M::solved + j);
                    if (far || g == (kBack ? 0 : 1)) {
                        ha::tmem_ld16(more, lanes + M::second + j);
                        ha::tmem_ready(z);
                        plus(z, more);
                    }
                    ha::tmem_ld16_early(x, lanes + M::y + j);
                    if (far) {
                        ha::tmem_ld16(more, lanes + M::third + 16 * g);
                        plus(z, more);
                    }
                    ha::tmem_ready(z);
                    ha::tmem_ready(x);
                    plus(x, z);
                    if constexpr (kBack) ha::tmem_st16(lanes + M::y + j, x);  // F, for the warps beside
                    if constexpr (kMode == 1) {
                        if (ok && (v >> 4) < slices) {
                            float* const to = p.errors + ((chunk * slices + (v >> 4)) * C + j) * 16 + (v & 15);
#pragma unroll
                            for (int e = 0; e < 16; ++e) to[e * 16] = __uint_as_float(x[e]);
                        }
                    }
                    weigh<true>(vec + I::beta / 4 + j, x);
                    if constexpr (kOutput) {
                        uint32_t w[2][8];
                        put_left<2>(x, w);
#pragma unroll
                        for (int t = 0; t < 2; ++t) ha::tmem_st8(lanes + M::value(jj, t), w[t]);
                    }
                    weigh<true>(vec + (kBack ? I::early : I::late) / 4 + j, x);
                    if constexpr (kBack)
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] ^= 0x80000000u;
                    uint32_t w[3][8];
                    put_left<3>(x, w);
#pragma unroll
                    for (int t = 0; t < 3; ++t) ha::tmem_st8(lanes + M::factor(jj, t), w[t]);
                }
            }
            ha::release_reads();
            ha::tmem_wait_st();
            ha::tmem_before_sync();
            arrive(kWrites);
            if (lane == 0 && ok) ha::bar_arrive(bars + 8 * (kEmpty + st));
            ok = ok && wait(kUpdated, it);
            ha::tmem_after_sync();
#pragma unroll
            for (int k = 0; k < kOwn; k += 16) {
                uint32_t x[16];
                ha::tmem_ld16(x, lanes + M::s + k0 + k);
#pragma unroll
                for (int e = 0; e < 16; ++e) s[k + e] = whole == 0.0f ? __uint_as_float(x[e]) : fmaf(whole, s[k + e], __uint_as_float(x[e]));
            }
            if (it + 1 < count) publish();
        }
        if (p.s_out && mine && ok) {
            float* const to = p.s_out + (long long)bh * p.dk * p.dv;
#pragma unroll
            for (int k = 0; k < kOwn; ++k)
                if (k0 + k < p.dk) to[(long long)(k0 + k) * p.dv + v] = s[k];
        }
    }
    ha::tmem_before_sync();
    __syncthreads();
    if (warp == 16) ha::tmem_free(0, M::columns);
    if (tid == 0 && *stop) give_up(p, gave_up, 200 + *stop);
}

}  // namespace hd
