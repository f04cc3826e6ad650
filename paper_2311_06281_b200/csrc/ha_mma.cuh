// The passes of ha_simt.cuh on the tensor cores (tcgen05): bf16 tensors, head dimensions up to 128, chunks of 128 tokens.
//
// One CTA walks the chunks of one (batch, head), or of one segment of it, with the state S^T in registers.  Per chunk
//     P   = mask(e^{c_i-c_j}) o (X Y^T)         X, Y from shared memory; P goes back to tensor memory as the next A operand
//     out = scale (e^{c_i} X S + P Z)           the second product adds to the first, whose rows are scaled between them
//     S^T = e^{c_C} S^T + (w Z)^T Y             Z^T reaches tensor memory by sixteen-column products with an identity: the
//                                               tensor core transposes, the threads scale by the weights w_j and write the
//                                               A operand back, no shared memory is spent on it
// Warps 0-7 own the rows of P and out (two threads to a row), warps 8-15 the rows of S^T (likewise); the two chains meet only
// in S.  Of the last four warps one loads (TMA, two chunks ahead), one sums the decays, and one thread of each of the others
// issues the products of a chain.
//
// Rounding.  A float32 factor enters a product as bf16 terms: w Z (and so the state, which is float32 to its owner) as three,
// 24 bits, exact to float32's own rounding; P and the state in X S as one, where only the bf16 output depends on them (its own
// rounding is as large).
//
// Measured, [8 x 2048 tokens, 16 heads of 128] (128 CTAs): forward and dv 77 us each, 268 MB at 3.5 TB/s; with kDots 157 us
// (dk) and 172 us (dq), of which some is spills (64 to 96 bytes a thread; the other passes have none).  Neither memory (55% of
// a copy's rate) nor the tensor core (31% of its cycles) bounds it: a chunk's steps wait for each other, 7000 to 8000 clocks of
// them, and shared memory holds one CTA.  Of those the output's chain has: scores 520, P 2000, X S 1100, scaling its rows 600,
// P Z 900, the output 760; the state's: Z^T 500, its terms 2400, the update 2000, reading it 500, publishing it 500.  What did
// not help: the output from registers straight to memory (2200 clocks for 760), one warp that watches the barriers of both
// chains (600 clocks from a barrier to the last of eight products), fewer registers for the rows of the state (spills).
//
// kDots: the pass also forms what the decay gradients need of it, in float32: the row sums of W = P o (w Z^T), w the fourth
// tensor, from the unrounded P, and the dots w_i . (X S)_i, for which X S has the state in three terms.  Each W_ij comes out of
// the two passes that form it in the same bits (each exponential is taken of the same difference there, each product is rounded
// once before it is added to anything), and the sums keep what their additions round off: what cancels between them leaves at
// most 2^-44 of the sum of |W|, at tokens that forget everything too.  (Four products added in float32 first left 1e-5 to 1e-4
// where nothing belonged.  This costs 2% of a training step, sums in 64 bits cost 4%: conversions are slow.)  Row sums from the
// outputs instead, w_i . out_i, were 1e-6 off in a common direction (the tensor core's additions cut off), which sums over many
// tokens turn into 5e-5.
#pragma once
#include <cuda.h>

#include "ha_ptx.cuh"
#include "ha_simt.cuh"

namespace ha {

constexpr int kChunk = 128;
constexpr int kMmaThreads = 640;
// Registers of a thread: 96 at launch (65536 over 20 warps); those that the feeding warps and the rows of out can spare go to
// the rows of the state.  80 + 2 * 64 + 2 * 136 = 480 for a thread of each warpgroup, 5 * 96 as at launch.
constexpr int kFeedRegs = 80;
constexpr int kRowRegs = 64, kStateRegs = 136;
constexpr uint32_t kTile = 128 * 256;        // 128 rows of 128 bf16: two blocks of 64 columns, 128-byte swizzle
constexpr uint32_t kBlock = kTile / 2;

struct MmaPass {
    const float* log_a;
    long long ab, at, ah;
    const int* lengths;
    int tokens, heads, dx, dz;
    int xdiv, ydiv, zdiv;
    float scale;
    const float* s_in;
    float* s_out;
    int s_in_t;
    float s_in_mul, s_out_mul;
    void* out;
    long long ob, ot, oh;
    // A sequence cut into segments: each starts from seg_state[bh][segment] ([dx, dz], formed by two kernels before this one)
    int segments, seg_chunks, chunks;
    float* seg_state;
    float* seg_decay;
    // For the decay gradients (kDots), by token and for each half of the columns, [2][batch * heads][tokens]: the row sums of
    // W below (reversed: above) the diagonal, and w_i . (X S)_i.  The forward pass also leaves the state before every chunk in
    // `dump`, the reversed one multiplies it with its own: cross[batch * heads][chunks][8], one for each warp.
    int wdiv;
    double* dots;
    float* dots_far;
    float4* dump;
    float* cross;
    Fault* fault;
    unsigned long long call_id;
    uint32_t spin;  // polls of a barrier before a wait gives up (0.15 us each, measured)
    int mute;       // tests: the chunk whose decays are never announced, or -1
};

// A chunk whose decay is below 2^-60 passes nothing on from before it that float32 could see beside what is in it.
constexpr float kNothingCrosses = -60.0f;

// Where a bounded wait of any pass on this device has run out since the record was last read, plus one; 0: nowhere.
__device__ int g_gave_up;

template <bool kDots>
struct MmaLayout {
    static constexpr int kTerms = kDots ? 2 : 1;               // of the state in X S (kDots: a third in a Y tile)
    static constexpr int kWeightsAtOnce = kDots ? 2 : 3;       // terms of w Z in the first product; the third follows
    // Stages.  A chunk's output leaves by TMA from its Z tile, the one that the next chunk needs last, or from its Y tile where Z
    // has one stage.  (Stores of a thread's own row took 2200 clocks a chunk instead of 760.)
    static constexpr int kXs = kDots ? 1 : 2, kYs = 2, kZs = kDots ? 1 : 2, kWs = kDots ? 1 : 0;
    static constexpr uint32_t x = 0, y = x + kXs * kTile, z = y + kYs * kTile, w = z + kZs * kTile, s = w + kWs * kTile,
                              ident = s + kTerms * kTile, decays = ident + 512, whole = decays + 4 * kChunk * 4, bars = whole + 32,
                              end = bars + 8 * 40;
    // Tensor memory columns, all 512.  What is read out before the next product of its chain is due shares columns with it:
    // Z^T with the state's update, the scores with the output.
    static constexpr uint32_t tw = 0;                          // the terms of (w Z)^T: A operand
    static constexpr uint32_t tz = tw + 64 * kWeightsAtOnce;   // Z^T, then the state's update
    static constexpr uint32_t to = tz + 128;                   // X Y^T, then X S, then P Z
    static constexpr uint32_t tp = to + 128;                   // P: A operand
    static constexpr uint32_t tt = tp + 64;                    // half of w Z^T (kDots)
    static_assert(tt + (kDots ? 64 : 0) == 512, "tensor memory");
    static __device__ __forceinline__ uint32_t staged(uint32_t base, int it) {
        return base + (kDots ? y + it % kYs * kTile : z + it % kZs * kTile);
    }
    // where 16 tokens q, and term t of them, lie
    static __device__ __forceinline__ constexpr uint32_t prob(int q) { return tp + 8 * q; }
    static __device__ __forceinline__ constexpr uint32_t weighted(int q, int t) { return tw + 8 * kWeightsAtOnce * q + 8 * t; }
};

// Every barrier completes one phase per chunk (those with two entries: per chunk that uses the entry), and nobody who waits
// for a phase can be overtaken by the next: it needs something of the waiter's own.
enum Bar : int { kFullX = 0, kFullY = 2, kFullZ = 4, kFreeX = 6, kFreeY = 8, kFreeZ = 10, kPatchY = 12, kPatchZ, kDecays, kDecaysFree, kScores,
                 kTransposed, kProbs, kFar, kFarRead, kNear, kOutRead, kWeighted, kWeightedLast, kUpdateFirst, kUpdate, kUpdateRead,
                 kStateReady, kFullW, kFreeW, kHalfRead, kHalf, kTileDone, kSent = kTileDone + 2, kStateLast, kDrain,
                 kBars = kDrain + 2 };
static_assert(kBars <= 40, "barriers");

template <int kValue> struct Int { static constexpr int value = kValue; };

// sum + the products of sixteen float32 values and sixteen bf16
__device__ __forceinline__ pair add_dot(pair sum, const uint32_t (&v)[16], const uint4& lo, const uint4& hi) {
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fma2(make_pair2(w[i] << 16, w[i] & 0xffff0000u), make_pair2(v[2 * i], v[2 * i + 1]), sum);
    return sum;
}
// sum + rest + v with no rounding but that of rest: what the sum's addition rounds off, from the operands themselves (Knuth's
// two-sum, for v of any size).
__device__ __forceinline__ void add_exact(pair& sum, pair& rest, pair v) {
    const pair minus = make_pair2(-1.0f, -1.0f), all = add2(sum, v), own = fma2(sum, minus, all), other = fma2(own, minus, all);
    rest = add2(rest, add2(fma2(own, minus, v), fma2(other, minus, sum)));
    sum = all;
}
// Sixteen columns of one row, or the n (a multiple of 8) that are left of it
__device__ __forceinline__ void store16(float* to, const uint32_t (&v)[16], int n) {
#pragma unroll
    for (int i = 0; i < 16; i += 4)
        if (i < n) *reinterpret_cast<uint4*>(to + i) = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
}
__device__ __forceinline__ void store16(__nv_bfloat16* to, const uint32_t (&v)[16], int n) {
#pragma unroll
    for (int i = 0; i < 16; i += 8)
        if (i < n)
            *reinterpret_cast<uint4*>(to + i) =
                make_uint4(pack_bf16(make_pair2(v[i], v[i + 1])), pack_bf16(make_pair2(v[i + 2], v[i + 3])),
                           pack_bf16(make_pair2(v[i + 4], v[i + 5])), pack_bf16(make_pair2(v[i + 6], v[i + 7])));
}

template <bool kRev, bool kDots, class Out, bool kStateOnly>
__global__ void __launch_bounds__(kMmaThreads, 1) mma_pass_kernel(const __grid_constant__ CUtensorMap mx, const __grid_constant__ CUtensorMap my,
                                                                  const __grid_constant__ CUtensorMap mz, const __grid_constant__ CUtensorMap mo,
                                                                  const __grid_constant__ CUtensorMap mw,
                                                                  const MmaPass p) {
    using L = MmaLayout<kDots>;
    // a group that asks for more than the others gave up would wait for ever
    static_assert(kFeedRegs + 2 * kRowRegs + 2 * kStateRegs <= 5 * 96 && kRowRegs <= 96, "registers");
    constexpr int kTerms = L::kTerms;
    extern __shared__ __align__(1024) uint8_t sm8[];
    const uint32_t base = smem_addr(sm8);
    float* const c_hi = reinterpret_cast<float*>(sm8 + L::decays);
    float* const c_lo = c_hi + kChunk;
    float* const w_st = c_lo + kChunk;    // what a token's update still weighs at the chunk's end (reversed: its beginning)
    float* const w_bt = w_st + kChunk;    // ... at the edge of its batch of 32
    float* const s_whole = reinterpret_cast<float*>(sm8 + L::whole);  // the chunk's decay, and its logarithm in two parts
    volatile int* const stop = reinterpret_cast<int*>(sm8 + L::whole + 16);
    uint32_t* const s_tmem = reinterpret_cast<uint32_t*>(sm8 + L::whole + 20);
    const uint32_t bars = base + L::bars;
    const Waiter wait{bars, stop, p.spin};
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    const int cuts = kStateOnly ? p.segments - 1 : p.segments;  // the last segment's own state is not needed by another
    const int segment = blockIdx.x % cuts, bh = blockIdx.x / cuts, b = bh / p.heads, h = bh % p.heads;
    const int live = live_tokens(p.lengths, b, p.tokens);
    const int chunks = (live + kChunk - 1) / kChunk;                       // that hold tokens
    const int first = min(chunks, segment * p.seg_chunks), count = min(chunks, first + p.seg_chunks) - first;
    auto chunk_at = [&](int it) { return kRev ? chunks - 1 - (first + it) : first + it; };

    if (tid == 0) {
        for (int i = 0; i < kBars; ++i) {
            uint32_t arrivals = 1;
            if (i >= kFreeY && i < kFreeZ) arrivals = kStateOnly || kDots ? 1 : 2;
            if (i >= kFreeZ && i < kPatchY) arrivals = kDots ? 2 : 1;
            if (i == kDecays) arrivals = 32;
            if (i == kDecaysFree) arrivals = 512;
            if (i == kProbs || i == kFarRead || i == kOutRead || i == kWeighted || i == kWeightedLast || i == kHalfRead || i == kUpdateRead ||
                i == kStateReady || i == kStateLast)
                arrivals = kStateOnly && i == kWeighted ? 512 : 256;
            if (i == kFreeW) arrivals = 257;
            bar_init(bars + 8 * i, arrivals);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *stop = 0;
        if (blockIdx.x == 0) p.fault->started_id = p.call_id;
    }
    if (tid < 256) {  // the identity, two 8 x 8 core matrices along each of k and n
        const int n = tid >> 4, k = tid & 15;
        *reinterpret_cast<__nv_bfloat16*>(sm8 + L::ident + (k >> 3) * 256 + (n >> 3) * 128 + (n & 7) * 16 + (k & 7) * 2) =
            __float2bfloat16(n == k ? 1.0f : 0.0f);
    }
    fence_smem_to_async();
    if (warp == 16) tmem_alloc(smem_addr(s_tmem), 512);
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    if (tid == 0 && *s_tmem != 0) *stop = 1 + kBars;  // all columns were asked for: they start at 0
    constexpr uint32_t tmem = 0;
    // a pass without an output has its columns for Z^T: the next chunk's is formed behind this one's update
    constexpr uint32_t zt = kStateOnly ? L::to : L::tz;

    // (w Z)^T of tokens 16 q0 to 16 q1, for one z of it each thread: its terms, the smallest first
    auto weigh = [&](uint32_t at, int q0, int q1, uint32_t (&last)[L::kWeightsAtOnce == 2 ? 4 : 1][8]) {
        uint32_t v[16];
        if (q0 < q1) tmem_ld16_early(v, at + zt + 16 * q0);
#pragma unroll L::kWeightsAtOnce == 2 ? 4 : 1
        for (int i = 0; i < 4; ++i) {
            const int q = q0 + i;
            if (q >= q1) break;
            uint32_t w[3][8];
            tmem_ready(v);
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const float4 f = read4(w_st + 16 * q + j);
                uint32_t t[3];
                split<3>(mul2(make_pair2(v[j], v[j + 1]), make_pair2(f.x, f.y)), t);
#pragma unroll
                for (int u = 0; u < 3; ++u) w[u][j / 2] = t[u];
                split<3>(mul2(make_pair2(v[j + 2], v[j + 3]), make_pair2(f.z, f.w)), t);
#pragma unroll
                for (int u = 0; u < 3; ++u) w[u][j / 2 + 1] = t[u];
            }
            if (q + 1 < q1) tmem_ld16_early(v, at + zt + 16 * (q + 1));
#pragma unroll
            for (int u = 0; u < L::kWeightsAtOnce; ++u) tmem_st8(at + L::weighted(q, u), w[2 - u]);
            if constexpr (L::kWeightsAtOnce == 2)
#pragma unroll
                for (int u = 0; u < 8; ++u) last[i][u] = w[0][u];
        }
    };
    if (warp >= 16) {
        give_registers<kFeedRegs>();
        // The thread that issues the output's products shares a scheduler with the rows that have least to do: the first 32
        // (reversed: the last)
        constexpr int kOutIssuer = kRev ? 19 : 16, kStateIssuer = kRev ? 16 : 19, kLoader = 17, kDecayer = 18;
        if (warp == kLoader) {
            // ------------------------------------------------------------ loads
            auto load = [&](const CUtensorMap* m, uint32_t to, int dim, int head, int t0, int full) {
                bar_expect(bars + 8 * full, dim > 64 ? kTile : kBlock);
                tma_load_4d(to, m, 0, head, t0, b, bars + 8 * full);
                if (dim > 64) tma_load_4d(to + kBlock, m, 64, head, t0, b, bars + 8 * full);
            };
            bool ok = true;
            int loads_x = 0, loads_y = 0, loads_z = 0, loads_w = 0, patched = -1;
            for (int it = 0; it < count && ok; ++it) {
                const int t0 = chunk_at(it) * kChunk;
                // tokens behind the sequence's end are in memory and may hold anything: 0 * NaN must not reach a sum
                const bool patch = live < p.tokens && t0 + kChunk > live;
                const uint32_t Y = base + L::y + it % L::kYs * kTile, Z = base + L::z + it % L::kZs * kTile;
                if (lane == 0) {  // in the order in which tiles become free
                    if (kDots && it >= 1) ok = wait(kFreeY + it % L::kYs, (it - 1) / L::kYs);  // the state's last term was in it
                    if (!kDots && it >= L::kYs) ok = wait(kFreeY + it % L::kYs, it / L::kYs - 1);
                    if (ok && patch) patched = it;
                    if (ok) load(&my, Y, p.dx, h / p.ydiv, t0, patch ? kPatchY : kFullY + it % L::kYs);
                    if (ok) loads_y = it + 1;
                    if (!kStateOnly) {
                        if (ok && it >= L::kXs) ok = wait(kFreeX + it % L::kXs, it / L::kXs - 1);
                        if (ok) load(&mx, base + L::x + it % L::kXs * kTile, p.dx, h / p.xdiv, t0, kFullX + it % L::kXs);
                        if (ok) loads_x = it + 1;
                    }
                    if (kDots) {
                        if (ok && it >= 1) ok = wait(kFreeW, it - 1);
                        if (ok) load(&mw, base + L::w, p.dz, h / p.wdiv, t0, kFullW);
                        if (ok) loads_w = it + 1;
                    }
                    if (ok && it >= L::kZs) ok = wait(kFreeZ + it % L::kZs, it / L::kZs - 1);
                    if (ok) load(&mz, Z, p.dz, h / p.zdiv, t0, patch ? kPatchZ : kFullZ + it % L::kZs);
                    if (ok) loads_z = it + 1;
                }
                if (patch) {
                    ok = __shfl_sync(~0u, (int)ok, 0);
                    ok = ok && wait(kPatchY, 0) && wait(kPatchZ, 0);
                    ok = __all_sync(~0u, ok);
                    const int rows = t0 + kChunk - live;
                    for (int e = lane; ok && e < rows * 16; e += 32) {
                        const uint32_t at = (e & 8 ? kBlock : 0) + (live - t0 + (e >> 4)) * 128 + (e & 7) * 16;
                        if (!(e & 8) || p.dx > 64) *reinterpret_cast<uint4*>(sm8 + (Y - base) + at) = make_uint4(0, 0, 0, 0);
                        if (!(e & 8) || p.dz > 64) *reinterpret_cast<uint4*>(sm8 + (Z - base) + at) = make_uint4(0, 0, 0, 0);
                    }
                    fence_smem_to_async();
                    __syncwarp();
                    if (lane == 0 && ok) {
                        bar_arrive(bars + 8 * (kFullY + it % L::kYs));
                        bar_arrive(bars + 8 * (kFullZ + it % L::kZs));
                    }
                }
                ok = __shfl_sync(~0u, (int)ok, 0);
            }
            if (lane == 0) {  // nothing may land in shared memory after the CTA has left
                auto drain = [&](int full, int stages, int loads, int patch) {
                    for (int it = max(0, loads - stages); it < loads; ++it)
                        if (patch && it == patched) wait.drain(patch, 0);
                        else wait.drain(full + it % stages, it / stages);
                };
                drain(kFullY, L::kYs, loads_y, kPatchY);
                drain(kFullZ, L::kZs, loads_z, kPatchZ);
                if (kDots) drain(kFullW, 1, loads_w, 0);
                if (!kStateOnly) drain(kFullX, L::kXs, loads_x, 0);
            }
        } else if (warp == kDecayer) {
            // ------------------------------------------------------------ decays, a lane has four tokens
            const float* ga = p.log_a + b * p.ab + h * p.ah;
            float a[4];
            auto fetch = [&](int it) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = chunk_at(it) * kChunk + 4 * lane + i;
                    a[i] = it < count && t < live ? ga[t * p.at] : 0.0f;
                }
            };
            fetch(0);
            bool ok = true;
            double total = 0.0;
            for (int it = 0; it < count && ok; ++it) {
                double c[4], sum;
#pragma unroll
                for (int i = 0; i < 4; ++i) c[i] = (i ? c[i - 1] : 0.0) + (double)(a[i] < kReset ? kReset : a[i]) * 1.4426950408889634;
                fetch(it + 1);
                sum = c[3];
                for (int o = 1; o < 32; o *= 2) {
                    const double u = __shfl_up_sync(~0u, sum, o);
                    if (lane >= o) sum += u;
                }
                const double whole = __shfl_sync(~0u, sum, 31), before = sum - c[3];
#pragma unroll
                for (int i = 0; i < 4; ++i) c[i] += before;
                const double edge = kRev ? __shfl_sync(~0u, c[0], lane & ~7) : __shfl_sync(~0u, c[3], lane | 7);
                float4 hi, lo, st, bt;
                auto four = [&](int i, float& h4, float& l4, float& s4, float& b4) {
                    h4 = (float)c[i];
                    l4 = (float)(c[i] - (double)(float)c[i]);
                    s4 = ex2((float)(kRev ? c[i] : whole - c[i]));
                    b4 = ex2((float)(kRev ? c[i] - edge : edge - c[i]));
                };
                four(0, hi.x, lo.x, st.x, bt.x);
                four(1, hi.y, lo.y, st.y, bt.y);
                four(2, hi.z, lo.z, st.z, bt.z);
                four(3, hi.w, lo.w, st.w, bt.w);
                if (it > 0) ok = __all_sync(~0u, wait(kDecaysFree, it - 1));
                if (!ok || chunk_at(it) == p.mute) break;
                reinterpret_cast<float4*>(c_hi)[lane] = hi;
                reinterpret_cast<float4*>(c_lo)[lane] = lo;
                reinterpret_cast<float4*>(w_st)[lane] = st;
                reinterpret_cast<float4*>(w_bt)[lane] = bt;
                if (lane == 31) {
                    s_whole[0] = ex2((float)whole);
                    s_whole[1] = (float)whole;
                    s_whole[2] = (float)(whole - (double)(float)whole);
                }
                total += whole;
                bar_arrive(bars + 8 * kDecays);
            }
            if (kStateOnly && lane == 0) p.seg_decay[bh * p.segments + segment] = ex2((float)total);
        } else if (warp == kStateIssuer) {
            // ------------------------------------------------------------ the products of the state's chain: Z^T; its update
            // Two warps issue, one for each chain, and wait for one barrier at a time: a thread that watched both chains took
            // 600 clocks from a barrier to the last of eight products.  Nearly all that a product takes is a constant (measured:
            // 20 to 30 clocks for a product's issue so, 48 to 110 with every operand in a register; the tensor core needs 30
            // to 64).
            if (elect_one()) {
                const uint32_t shape_t = mma_shape(16, kColMajorA), shape_u = mma_shape((p.dx + 15) / 16 * 16, kColMajorB);
                auto transpose = [&](int it) {
                    const int steps = 2 * min(4, (live - chunk_at(it) * kChunk + 31) / 32), zs = it % L::kZs;
                    const uint32_t zo = operand(base + L::z + zs * kTile, kBlock), ident = operand(base + L::ident, 256);
                    if (!(wait(kFullZ + zs, it / L::kZs) && (kStateOnly || it == 0 || wait(kUpdateRead, it - 1)))) return false;
                    tmem_after_sync();
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (q < steps) mma_ss<plain_layout(128)>(tmem + zt + 16 * q, zo + q * 128, ident, shape_t, false);
                    mma_commit(bars + 8 * kTransposed);
                    if (kDots || kStateOnly) mma_commit(bars + 8 * (kFreeZ + zs));
                    else mma_commit(bars + 8 * (kTileDone + zs));
                    return true;
                };
                bool ok = !kStateOnly || count == 0 || transpose(0);
                for (int it = 0; it < count && ok; ++it) {
                    const int steps = 2 * min(4, (live - chunk_at(it) * kChunk + 31) / 32), ys = it % L::kYs;
                    const uint32_t yo = operand(base + L::y + ys * kTile, kBlock);
                    if (!kStateOnly && !(ok = transpose(it))) break;
                    if (kStateOnly && it > 0 && !(ok = wait(kUpdateRead, it - 1))) break;
                    if (!(ok = wait(kFullY + ys, it / L::kYs) && wait(kWeighted, it))) break;
                    tmem_after_sync();
#pragma unroll
                    for (int t = 0; t < L::kWeightsAtOnce; ++t)
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            if (q < steps) mma_ts(tmem + L::weighted(q, t), yo + q * 128, shape_u, q + t > 0, tmem + L::tz);
                    if (L::kWeightsAtOnce == 2) {
                        mma_commit(bars + 8 * kUpdateFirst);
                        if (!(ok = wait(kWeightedLast, it))) break;
                        tmem_after_sync();
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            if (q < steps) mma_ts(tmem + L::weighted(q, 0), yo + q * 128, shape_u, true, tmem + L::tz);
                    }
                    mma_commit(bars + 8 * kUpdate);
                    mma_commit(bars + 8 * ((kDots ? kTileDone : kFreeY) + ys));
                    if (kStateOnly && it + 1 < count) ok = transpose(it + 1);
                }
                mma_commit(bars + 8 * kDrain);
                wait.drain(kDrain, 0);
            }
            __syncwarp();
        } else if (!kStateOnly && warp == kOutIssuer) {
            // ------------------------------------------------------------ the products of the output's chain: X Y^T (w Z^T in
            // two halves); X S; P Z.  The output leaves in between.
            if (elect_one()) {
                const int kx = (p.dx + 15) / 16;
                const uint32_t nz = (p.dz + 15) / 16 * 16;
                const uint32_t shape_p = mma_shape(128, 0), shape_f = mma_shape(nz, 0), shape_n = mma_shape(nz, kColMajorB);
                const uint32_t so = operand(base + L::s, kBlock);
                auto k_step = [](int kk) { return (uint32_t)((kk >> 2) * (kBlock >> 4) + (kk & 3) * 2); };  // 32 bytes, then the next block
                auto half_scores = [&](int half) {  // w Z^T for 64 of the chunk's tokens as columns
                    const uint32_t wo = operand(base + L::w, kBlock), zo = operand(base + L::z, kBlock) + half * (64 * 128 >> 4);
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        if (16 * kk < p.dz) mma_ss(tmem + L::tt, wo + k_step(kk), zo + k_step(kk), mma_shape(64, 0), kk > 0);
                };
                auto send = [&](int it) {  // a chunk's output is in shared memory
                    if constexpr (sizeof(Out) == 2) {
                        const uint32_t from = L::staged(base, it);
                        tma_store_4d(&mo, 0, h, chunk_at(it) * kChunk, b, from);
                        if (p.dz > 64) tma_store_4d(&mo, 64, h, chunk_at(it) * kChunk, b, from + kBlock);
                        tma_store_commit();
                    }
                };
                auto sent = [&](int it) {  // ... and has been read from there
                    if constexpr (sizeof(Out) == 2) tma_store_wait_read();
                    bar_arrive(bars + 8 * (kDots ? kSent : kFreeZ + it % L::kZs));
                };
                auto chunk = [&](int it, auto odd) {  // a copy for each stage: their addresses are constants
                    constexpr int xs = odd.value % L::kXs, ys = odd.value % L::kYs, zs = odd.value % L::kZs;
                    const int steps = 2 * min(4, (live - chunk_at(it) * kChunk + 31) / 32);
                    const uint32_t xo = operand(base + L::x + xs * kTile, kBlock), yo = operand(base + L::y + ys * kTile, kBlock),
                                   zo = operand(base + L::z + zs * kTile, kBlock), last = operand(base + L::y + (ys ^ 1) * kTile, kBlock);
                    if (!(wait(kFullX + xs, it / L::kXs) && wait(kFullY + ys, it / L::kYs) &&
                          (!kDots || (wait(kFullZ, it) && wait(kFullW, it))) && (it == 0 || wait(kOutRead, it - 1))))
                        return false;
                    tmem_after_sync();
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        if (kk < kx) mma_ss(tmem + L::to, xo + k_step(kk), yo + k_step(kk), shape_p, kk > 0);
                    if (kDots) half_scores(0);
                    mma_commit(bars + 8 * kScores);
                    if (!kDots) mma_commit(bars + 8 * (kFreeY + ys));
                    if (it > 0) {
                        send(it - 1);
                        sent(it - 1);
                    }
                    if (kDots) {
                        if (!wait(kHalfRead, it)) return false;
                        tmem_after_sync();
                        half_scores(1);
                        mma_commit(bars + 8 * kHalf);
                        mma_commit(bars + 8 * kFreeW);
                    }
                    if (!(wait(kStateReady, it) && (!kDots || wait(kStateLast, it)) && wait(kProbs, it))) return false;
                    tmem_after_sync();
                    if (kDots)
#pragma unroll
                        for (int kk = 0; kk < 8; ++kk)
                            if (kk < kx) mma_ss(tmem + L::to, xo + k_step(kk), last + k_step(kk), shape_f, kk > 0);
#pragma unroll
                    for (int t = kTerms - 1; t >= 0; --t)  // small terms first: every addition rounds the sum so far
#pragma unroll
                        for (int kk = 0; kk < 8; ++kk)
                            if (kk < kx)
                                mma_ss(tmem + L::to, xo + k_step(kk), so + t * (kTile >> 4) + k_step(kk), shape_f, kDots || t < kTerms - 1 || kk > 0);
                    mma_commit(bars + 8 * kFar);
                    mma_commit(bars + 8 * (kFreeX + xs));
                    if (kDots) mma_commit(bars + 8 * (kFreeY + (ys ^ 1)));
                    if (!(wait(kFullZ + zs, it / L::kZs) && wait(kFarRead, it))) return false;
                    tmem_after_sync();
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (q < steps) mma_ts(tmem + L::prob(q), zo + q * 128, shape_n, true, tmem + L::to);
                    mma_commit(bars + 8 * kNear);
                    if (kDots) mma_commit(bars + 8 * (kFreeZ + zs));
                    return true;
                };
                bool ok = true;
                for (int it = 0; it < count && ok; it += 2) {
                    ok = chunk(it, Int<0>{});
                    if (ok && it + 1 < count) ok = chunk(it + 1, Int<1>{});
                }
                if (ok && count > 0 && (ok = wait(kOutRead, count - 1))) send(count - 1);
                mma_commit(bars + 8 * (kDrain + 1));
                wait.drain(kDrain + 1, 0);
                tma_store_wait_all();
            }
            __syncwarp();
        }
    } else if (warp < 8) {
        give_registers<kRowRegs>();
        // ---------------------------------------------------------------- P and the output: two threads have one token's row
        if (kStateOnly) {  // no output: half of the weighing
            const int side = warp >> 2;
            const uint32_t at = tmem + ((uint32_t)((warp & 3) * 32) << 16);
            bool ok = true;
            for (int it = 0; it < count; ++it) {
                const int steps = 2 * min(4, (live - chunk_at(it) * kChunk + 31) / 32);
                uint32_t none[L::kWeightsAtOnce == 2 ? 4 : 1][8];
                ok = ok && wait(kDecays, it) && wait(kTransposed, it) && (it == 0 || wait(kUpdate, it - 1));
                tmem_after_sync();
                weigh(at, 4 * side + 2, min(steps, 4 * side + 4), none);
                release_reads();
                if (ok) bar_arrive(bars + 8 * kDecaysFree);
                tmem_wait_st();
                tmem_before_sync();
                if (ok) bar_arrive(bars + 8 * kWeighted);
            }
        }
        if (!kStateOnly) {
            const int side = warp >> 2, quarter = warp & 3, row = quarter * 32 + lane;
            const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16);
            Out* go = static_cast<Out*>(p.out) + b * p.ob + h * p.oh;
            const bool columns = 64 * side < p.dz;
            {   // P starts as zeros
                const uint32_t zero[8] = {};
#pragma unroll
                for (int i = 0; i < 4; ++i) tmem_st8(at + L::tp + 32 * side + 8 * i, zero);
                tmem_wait_st();
            }
            bool ok = true;
            for (int it = 0; it < count; ++it) {
                const int t0 = chunk_at(it) * kChunk, t = t0 + row;
                const int batches = min(4, (live - t0 + 31) / 32);
                ok = ok && wait(kDecays, it);
                const float own_hi = read1(c_hi + row), own_lo = read1(c_lo + row);
                const float far1 = ex2(kRev ? (read1(s_whole + 1) - own_hi) + (read1(s_whole + 2) - own_lo) : own_hi + own_lo);
                const float far = p.scale * far1;
                const bool forgotten = far1 == 0.0f;  // a decay of zero forgets the state whatever it holds: no 0 * inf
                ok = ok && wait(kScores, it);
                tmem_after_sync();
                pair sum = 0, sum_rest = 0;  // of W's row, in two floats each, since two such sums will be subtracted
                pair sum_far = 0;
                const pair minus = make_pair2(-1.0f, -1.0f), scale2 = make_pair2(p.scale, p.scale);
                const float to_late = kRev ? 1.0f : -1.0f;
                // A side has 16 columns of every batch of 32; batches on the empty side of the diagonal stay zero from the start.
#pragma unroll 1
                for (int n = 0; n < 4; ++n) {
                    if (kDots && n == 2) {  // the first half of w Z^T has been read by this thread
                        tmem_before_sync();
                        if (ok) bar_arrive(bars + 8 * kHalfRead);
                        ok = ok && wait(kHalf, it);
                        tmem_after_sync();
                    }
                    if (n >= batches || (kRev ? n < quarter : n > quarter)) continue;
                    const int q = 2 * n + side;
                    uint32_t v[16], term[8];
                    tmem_ld16(v, at + L::to + 16 * q);
                    auto keep = [&](int j, pair w) {  // two columns of P
                        w = mul2(w, make_pair2(v[j], v[j + 1]));
                        term[j / 2] = pack_bf16(w);
                        if constexpr (kDots) parts(w, v[j], v[j + 1]);
                    };
                    if (!kDots && n != quarter) {
                        // e^{c_i-c_j} = e^{c_i-c_m} e^{c_m-c_j} with m at the batch's edge between j and i: both exponents keep
                        // their sign, and one exponential of the row serves the batch's columns
                        const int m = kRev ? 32 * n : 32 * n + 31;
                        const float f1 = p.scale * ex2(to_late * ((read1(c_hi + m) - own_hi) + (read1(c_lo + m) - own_lo)));
                        const pair f = make_pair2(f1, f1);
#pragma unroll
                        for (int j = 0; j < 16; j += 4) {
                            const float4 g = read4(w_bt + 16 * q + j);
                            keep(j, mul2(f, make_pair2(g.x, g.y)));
                            keep(j + 2, mul2(f, make_pair2(g.z, g.w)));
                        }
                    } else {
                        const pair own_h = make_pair2(own_hi, own_hi), own_l = make_pair2(own_lo, own_lo);
                        const int ahead = n == quarter ? row - 16 * q : kRev ? -1 : 16;  // columns up to the diagonal
                        auto weights = [&](int j, float h0, float h1, float l0, float l1) {
                            // differences of the two parts first, either way round the same bits
                            float d0, d1;
                            parts(add2(fma2(own_h, minus, make_pair2(h0, h1)), fma2(own_l, minus, make_pair2(l0, l1))), d0, d1);
                            d0 = (kRev ? j >= ahead : j <= ahead) ? ex2(to_late * d0) : 0.0f;
                            d1 = (kRev ? j + 1 >= ahead : j + 1 <= ahead) ? ex2(to_late * d1) : 0.0f;
                            keep(j, mul2(scale2, make_pair2(d0, d1)));
                        };
#pragma unroll
                        for (int j = 0; j < 16; j += 4) {
                            const float4 hi = read4(c_hi + 16 * q + j), lo = read4(c_lo + 16 * q + j);
                            weights(j, hi.x, hi.y, lo.x, lo.y);
                            weights(j + 2, hi.z, hi.w, lo.z, lo.w);
                        }
                    }
                    tmem_st8(at + L::prob(q), term);
                    if constexpr (kDots) {
                        uint32_t t16[16];
                        tmem_ld16(t16, at + L::tt + 16 * (q & 3));
                        const int own = row - 16 * q;  // without the token itself
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (j == own) t16[j] = 0u;
#pragma unroll
                        for (int j = 0; j < 16; j += 2)  // each W_ij rounded once, the same way in both passes, before any addition
                            add_exact(sum, sum_rest, mul2(make_pair2(v[j], v[j + 1]), make_pair2(t16[j], t16[j + 1])));
                    }
                }
                release_reads();
                if (ok) bar_arrive(bars + 8 * kDecaysFree);
                tmem_wait_st();
                tmem_before_sync();
                if (ok) bar_arrive(bars + 8 * kProbs);
                ok = ok && wait(kFar, it);
                tmem_after_sync();
                const int col0 = 64 * side, col1 = min(p.dz, col0 + 64);
                const pair far2 = make_pair2(far, far);
                const uint8_t* const own_w = sm8 + L::w + side * kBlock + row * 128;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {  // X S with its row's weight, for P Z to be added to
                    const int col = col0 + 16 * c;
                    if (col >= col1) break;
                    uint32_t v[16];
                    tmem_ld16(v, at + L::to + col);
#pragma unroll
                    for (int u = 0; u < 16; u += 2) parts(mul2(far2, make_pair2(v[u], v[u + 1])), v[u], v[u + 1]);
                    if (forgotten)
#pragma unroll
                        for (int u = 0; u < 16; ++u) v[u] = 0u;
                    tmem_st16(at + L::to + col, v);
                    if constexpr (kDots) {
                        const uint4 lo = read4(own_w + (((2 * c) ^ (row & 7)) << 4)), hi = read4(own_w + (((2 * c + 1) ^ (row & 7)) << 4));
                        sum_far = add_dot(sum_far, v, lo, hi);
                    }
                }
                if constexpr (kDots) {
                    release_reads();
                    if (ok) bar_arrive(bars + 8 * kFreeW);
                }
                tmem_wait_st();
                tmem_before_sync();
                if (ok) bar_arrive(bars + 8 * kFarRead);
                ok = ok && wait(kNear, it);
                tmem_after_sync();
                // products may still read the tile that the output leaves from
                ok = ok && wait(kTileDone + it % 2, it / 2);
                uint8_t* const stage = sm8 + L::staged(0, it) + side * kBlock + row * 128;
#pragma unroll 1
                for (int col = col0; col < col1; col += 16) {
                    uint32_t v[16];
                    tmem_ld16(v, at + L::to + col);
                    if (t >= live)
#pragma unroll
                        for (int u = 0; u < 16; ++u) v[u] = 0u;
                    if constexpr (sizeof(Out) == 2) {
#pragma unroll
                        for (int c = 0; c < 2; ++c)
                            *reinterpret_cast<uint4*>(stage + ((((col - col0) / 8 + c) ^ (row & 7)) << 4)) =
                                make_uint4(pack_bf16(make_pair2(v[8 * c], v[8 * c + 1])), pack_bf16(make_pair2(v[8 * c + 2], v[8 * c + 3])),
                                           pack_bf16(make_pair2(v[8 * c + 4], v[8 * c + 5])), pack_bf16(make_pair2(v[8 * c + 6], v[8 * c + 7])));
                    } else if (t < p.tokens) {
                        store16(go + t * p.ot + col, v, p.dz - col);
                    }
                }
                if (sizeof(Out) == 2) fence_smem_to_async();
                tmem_before_sync();
                if (ok) bar_arrive(bars + 8 * kOutRead);
                if constexpr (kDots) {
                    const long long to = ((long long)side * gridDim.x / p.segments + bh) * p.tokens + t;
                    float a, c, s0, s1, r0, r1;
                    parts(sum_far, a, c);
                    parts(sum, s0, s1);
                    parts(sum_rest, r0, r1);
                    if (t < live) {
                        p.dots[to] = ((double)s0 + (double)s1) + ((double)r0 + (double)r1);
                        p.dots_far[to] = columns ? a + c : 0.0f;
                    }
                }
            }
            // chunks without tokens
            if (columns)
                for (int c = max(chunks, segment * p.seg_chunks); c < (segment + 1) * p.seg_chunks; ++c) {
                    const int t = c * kChunk + row;
                    const uint32_t o[16] = {};
                    for (int col = 64 * side; col < min(p.dz, 64 * side + 64) && t < p.tokens; col += 16) store16(go + t * p.ot + col, o, p.dz - col);
                }
        }
    } else {
        take_registers<kStateRegs>();
        // ---------------------------------------------------------------- the state: two threads have one row of S^T
        const int side = (warp - 8) >> 2, quarter = warp & 3, z = quarter * 32 + lane, k0 = 64 * side;
        const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16);
        const bool columns = k0 < p.dx, mine = z < p.dz;
        pair s[32];
        const float* from = kStateOnly ? nullptr : p.segments > 1 ? p.seg_state + ((long long)bh * p.segments + segment) * p.dx * p.dz
                                                 : p.s_in ? p.s_in + (long long)bh * p.dx * p.dz : nullptr;
        const bool across = p.segments == 1 && p.s_in_t;
        const float mul = p.segments == 1 ? p.s_in_mul : 1.0f;
#pragma unroll
        for (int k = 0; k < 64; k += 2) {  // dimensions are even: TMA could not load others
            float s0 = 0.0f, s1 = 0.0f;
            if (from && mine && k0 + k < p.dx) {
                s0 = from[across ? z * p.dx + k0 + k : (k0 + k) * p.dz + z] * mul;
                s1 = from[across ? z * p.dx + k0 + k + 1 : (k0 + k + 1) * p.dz + z] * mul;
            }
            s[k / 2] = make_pair2(s0, s1);
        }
        bool ok = true;
        auto publish = [&]() {  // the state as the B operand of X S: row z, contiguous along k
            if (columns) {
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint32_t w[kTerms][4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t t[kTerms];
                        split<kTerms>(s[4 * c + j], t);
#pragma unroll
                        for (int i = 0; i < kTerms; ++i) w[i][j] = t[i];
                    }
#pragma unroll
                    for (int i = 0; i < kTerms; ++i)
                        *reinterpret_cast<uint4*>(sm8 + L::s + i * kTile + side * kBlock + z * 128 + ((c ^ (z & 7)) << 4)) =
                            make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
                }
                fence_smem_to_async();
            }
            if (ok) bar_arrive(bars + 8 * kStateReady);
        };
        // kDots: the state's third term goes where the output of the chunk before has left from
        auto publish_last = [&](int it) {
            if (columns) {
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint32_t w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t t[3];
                        split<3>(s[4 * c + j], t);
                        w[j] = t[2];
                    }
                    *reinterpret_cast<uint4*>(sm8 + L::y + (it + 1) % L::kYs * kTile + side * kBlock + z * 128 + ((c ^ (z & 7)) << 4)) =
                        make_uint4(w[0], w[1], w[2], w[3]);
                }
                fence_smem_to_async();
            }
            if (ok) bar_arrive(bars + 8 * kStateLast);
        };
        if (!kStateOnly && count > 0) publish();
        for (int it = 0; it < count; ++it) {
            const int t0 = chunk_at(it) * kChunk;
            const int steps = 2 * min(4, (live - t0 + 31) / 32);
            ok = ok && wait(kDecays, it);
            const float whole = read1(s_whole);
            const pair whole2 = make_pair2(whole, whole);
            const bool crosses = read1(s_whole + 1) > kNothingCrosses;
            ok = ok && wait(kTransposed, it);
            tmem_after_sync();
            uint32_t last[L::kWeightsAtOnce == 2 ? 4 : 1][8];  // first terms, where they have to wait
            const int q0 = 4 * side, q1 = min(steps, q0 + (kStateOnly ? 2 : 4));
            weigh(at, q0, q1, last);
            release_reads();
            if (ok) bar_arrive(bars + 8 * kDecaysFree);
            tmem_wait_st();
            tmem_before_sync();
            if (ok) bar_arrive(bars + 8 * kWeighted);
            if constexpr (kDots) {
                if (it > 0) ok = ok && wait(kSent, it - 1);
                publish_last(it);
            }
            if constexpr (L::kWeightsAtOnce == 2) {
                ok = ok && wait(kUpdateFirst, it);
                tmem_after_sync();
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (q0 + i < q1) tmem_st8(at + L::weighted(q0 + i, 0), last[i]);
                tmem_wait_st();
                tmem_before_sync();
                if (ok) bar_arrive(bars + 8 * kWeightedLast);
            }
            if constexpr (kDots && !kRev) {  // the state from before this chunk, while its update is formed
                if (crosses && columns && mine) {
                    float4* to = p.dump + ((long long)bh * p.chunks + t0 / kChunk) * 4096 + side * 2048 + z;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float4 f;
                        parts(s[2 * j], f.x, f.y);
                        parts(s[2 * j + 1], f.z, f.w);
                        to[j * 128] = f;
                    }
                }
            }
            if constexpr (kDots && kRev) {  // <S, D> of this chunk, while its update is formed
                pair sum = 0;
                if (crosses && columns && mine) {
                    const float4* from4 = p.dump + ((long long)bh * p.chunks + t0 / kChunk) * 4096 + side * 2048 + z;
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        float4 f[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) f[u] = from4[(j + u) * 128];
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            sum = fma2(make_pair2(f[u].x, f[u].y), s[2 * (j + u)], sum);
                            sum = fma2(make_pair2(f[u].z, f[u].w), s[2 * (j + u) + 1], sum);
                        }
                    }
                }
                float a, c;
                parts(sum, a, c);
                a += c;
                for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(~0u, a, o);
                if (lane == 0) p.cross[((long long)bh * p.chunks + t0 / kChunk) * 8 + warp - 8] = a;
            }
            if (whole == 0.0f)  // likewise
#pragma unroll
                for (int j = 0; j < 32; ++j) s[j] = 0;
            ok = ok && wait(kUpdate, it);
            tmem_after_sync();
#pragma unroll
            for (int j = 0; j < 64; j += 16)
                if (k0 + j < p.dx) {  // the product has no further columns
                    uint32_t v[16];
                    tmem_ld16(v, at + L::tz + k0 + j);
#pragma unroll
                    for (int u = 0; u < 16; u += 2) s[(j + u) / 2] = fma2(whole2, s[(j + u) / 2], make_pair2(v[u], v[u + 1]));
                }
            tmem_before_sync();
            if (ok) bar_arrive(bars + 8 * kUpdateRead);
            if (!kStateOnly && it + 1 < count) {
                ok = ok && wait(kFar, it);  // this chunk's X S has read the state it started from
                publish();
            }
        }
        float* to = kStateOnly ? p.seg_state + ((long long)bh * p.segments + segment) * p.dx * p.dz
                               : p.s_out && segment == p.segments - 1 ? p.s_out + (long long)bh * p.dx * p.dz : nullptr;
        const float out_mul = kStateOnly ? 1.0f : p.s_out_mul;
#pragma unroll
        for (int k = 0; k < 64; k += 2)
            if (to && mine && k0 + k < p.dx) {
                float s0, s1;
                parts(s[k / 2], s0, s1);
                to[(k0 + k) * p.dz + z] = s0 * out_mul;
                to[(k0 + k + 1) * p.dz + z] = s1 * out_mul;
            }
    }
    tmem_before_sync();
    __syncthreads();
    if (warp == 16) tmem_free(tmem, 512);
    if (tid == 0 && *stop) {
        p.fault->error_code = 6;  // HS_ERR_COPY_TIMEOUT
        p.fault->error_where = *stop;
        g_gave_up = *stop;
        __threadfence();
        p.fault->error_id = p.call_id;
    }
}

// dlog_a of one chunk from what the two passes left (the formulas at the head of ha_simt.cuh): with r and r', u and u' the row
// sums and the far dots of the dq and the dk pass,
//     dlog_a_t = sum_{i>=t} (r_i - u_i + r'_i) + sum_{j<t} u'_j + e^{c_C} scale <S, D>.
// Pairs inside the chunk that both lie behind t are in r and in u and cancel.  A thread has one token; sums in 64 bits.
// part (fixed decays): only the sum over the chunk's tokens.
__global__ void __launch_bounds__(kChunk) join_decay_grad_kernel(const double* r, const double* u, const float* rf, const float* uf, const float* cross,
                                                                 const float* log_a, long long ab, long long at, long long ah,
                                                                 const int* lengths, int tokens, int heads, int chunks, long long side,
                                                                 float scale, float* dlog_a, double* part) {
    __shared__ double sums[3][4];
    const int n = blockIdx.x % chunks, bh = blockIdx.x / chunks, b = bh / heads, h = bh % heads, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int t = n * kChunk + threadIdx.x, live = live_tokens(lengths, b, tokens);
    const long long e = (long long)bh * tokens + t;
    double x = 0.0, y = 0.0, c = 0.0;
    if (t < live) {
        x = (r[e] + r[side + e]) - (u[e] + u[side + e]) + ((double)rf[e] + (double)rf[side + e]);
        y = (double)uf[e] + (double)uf[side + e];
        const float a = log_a[b * ab + t * at + h * ah];
        c = (double)(a < kReset ? kReset : a) * 1.4426950408889634;
    }
    const double own_x = x;
    for (int o = 1; o < 32; o *= 2) {  // running sums within a warp
        const double p = __shfl_up_sync(~0u, x, o), q = __shfl_up_sync(~0u, y, o);
        if (lane >= o) { x += p; y += q; }
    }
    for (int o = 16; o > 0; o >>= 1) c += __shfl_xor_sync(~0u, c, o);
    if (lane == 31) { sums[0][warp] = x; sums[1][warp] = y; sums[2][warp] = c; }
    __syncthreads();
    double all = 0.0, whole = 0.0;
    for (int w = 0; w < 4; ++w) {
        if (w < warp) { x += sums[0][w]; y += sums[1][w]; }
        all += sums[0][w];
        whole += sums[2][w];
    }
    double g = all - (x - own_x);                     // sum_{i>=t}
    const double before = __shfl_up_sync(~0u, y, 1);  // sum_{j<t}
    double first = 0.0;
    for (int w = 0; w < warp; ++w) first += sums[1][w];
    g += lane ? before : first;
    if (whole > (double)kNothingCrosses && n * kChunk < live) {
        double s = 0.0;
        for (int w = 0; w < 8; ++w) s += (double)cross[((long long)bh * chunks + n) * 8 + w];
        g += s * (double)scale * exp2(whole);
    }
    if (t >= live) g = 0.0;
    if (!part) {
        if (t < tokens) dlog_a[((long long)b * tokens + t) * heads + h] = (float)g;
        return;
    }
    for (int o = 16; o > 0; o >>= 1) g += __shfl_xor_sync(~0u, g, o);
    __syncthreads();
    if (lane == 0) sums[0][warp] = g;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.x] = sums[0][0] + sums[0][1] + sums[0][2] + sums[0][3];
}

// A strided [batch, tokens, heads, dim] tensor laid out contiguously, for TMA.
__global__ void pack_rows_kernel(const Rows from, __nv_bfloat16* to, int tokens, int heads, int dim, long long total) {
    for (long long e = (long long)blockIdx.x * blockDim.x + threadIdx.x; e < total; e += (long long)gridDim.x * blockDim.x) {
        const int d = (int)(e % dim);
        const long long row = e / dim, bt = row / heads;
        to[e] = static_cast<const __nv_bfloat16*>(from.ptr)[bt / tokens * from.sb + bt % tokens * from.st + row % heads * from.sh + d];
    }
}

}  // namespace ha
