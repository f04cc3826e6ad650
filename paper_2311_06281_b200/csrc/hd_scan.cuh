// The delta rule with a decay,  S_t = a_t S_{t-1} + beta_t k_t (v_t - a_t S_{t-1}^T k_t)^T,  o_t = scale S_t^T q_t,  in chunks.
//
// With c_i the running sums of the log decays inside a chunk, D_ij = e^{c_i-c_j}, S the state before the chunk, and
//     M_ij = D_ij k_i.k_j (i > j),   P_ij = scale D_ij q_i.k_j (i >= j),   N = (I + M beta)^{-1} M
// (beta as a diagonal matrix; N is strictly lower like M), what each token finds wrong with the state's answer for its key is
//     E = Y - N (beta Y),   Y = V - e^c K S        because E_i = Y_i - sum_{j<i} M_ij beta_j E_j
// and with V' = beta E
//     O = scale e^c Q S + P V',    S' = e^{c_C} S + K^T (e^{c_C-c} V').
// Backward, from the gradient D of S':
//     dV' = P^T dO + e^{c_C-c} K D,   F = dV' - N^T (beta dV'),   Z = beta F = dV,   dbeta_j = E_j.F_j,
//     dS  = e^{c_C} D + Q^T (scale e^c dO) - K^T (e^c Z).
// The system is solved once, for N: the two directions and beta come in around it, and no division by beta is needed.
//
// Two kernels a direction.  chunk_kernel forms M, P and N of every chunk, all chunks at once.  scan_kernel (backward: back_kernel)
// walks a sequence's chunks; a warp has 16 columns of the values and all that belongs to them: 16 columns of S, transposed, as
// mma accumulators, so that every product of the chain has its left factor in the registers that the one before left it in
// (hd_warp.cuh) and its right one, K, Q, N or P, in shared memory, where all warps of the CTA read it.  Nothing is handed from
// thread to thread; the columns of V are independent, so warps wait for nothing but the loads of the next chunk.
//
// Why mma.sync: five dependent products a chunk.  On tcgen05 each of them ends with a trip through tensor memory (commit,
// barrier, load, convert, store, barrier), about 1000 clocks as measured in ha_mma.cuh, for 128 x 128 tiles that it would take
// 60 to 500 clocks to multiply; the accumulators of mma.sync are its next operands after a conversion.
#pragma once
#include <cuda.h>

#include "hd_warp.cuh"

namespace hd {

using ha::Fault;
using ha::Waiter;
using ha::ex2;
using ha::kLog2e;
using ha::kReset;
using ha::live_tokens;

// Tokens of a chunk, by the width of the keys (64, 128 or 256 after padding): the longer, the fewer trips of the state through its
// terms; with 256 the tiles of 64 tokens do not fit.
constexpr int chunk_tokens(int kp) { return kp == 256 ? 32 : 64; }

struct Params {
    const float* log_a;
    long long ab, at, ah;
    const float* beta;
    long long bb, bt, bh;
    const int* lengths;
    int batch, tokens, heads, chunks;
    int qdiv, kdiv, vdiv;
    int dk, dv;
    float scale;
    int warps;             // of a CTA of the scans that have columns of V
    uint8_t* image;        // what chunk_kernel leaves for each (batch, head) and chunk
    const float* s_in;     // [batch, heads, dk, dv] or NULL
    float* s_out;          // or NULL
    void* out;             // o (backward: dv) through its strides, where TMA does not store it
    long long ob, ot, oh;
    int out_tma;
    float* states;         // backward: before every chunk the state (after it, its gradient), [batch * heads][chunks][16 slices][KP]
    float* errors;         // E (F) of every chunk, [batch * heads][chunks][16 slices][C]
    float* errors_back;    // F likewise (layouts of the tensor-core passes: hd_scan_mma.cuh)
    int parts;             // of the sums over V in `dots`
    float* gradients;      // the gradient of the state after every chunk, as `states`
    float* dots;           // [batch * heads][chunks][2][parts][C]: by part of V, dbeta and e^{c_C-c_j} k_j^T D V'_j
    void *dq, *dk_out;       // contiguous [batch, tokens, heads, dk]; in float32 where each_ says so (heads to be summed)
    int each_q, each_k, dq_tma, dk_tma;
    float *dlog_a, *dbeta; // [batch, tokens, heads], or NULL
    double* part;          // fixed decays: their gradients' sums over each chunk, [batch * heads][chunks]
    Fault* fault;
    unsigned long long call_id;
    uint32_t spin;
    int mute;              // tests: the chunk that is never loaded, or -1
};

// Where a bounded wait has run out on this device since the record was last read, plus one.
__device__ __forceinline__ void give_up(const Params& p, int* gave_up, int where) {
    p.fault->error_code = 6;  // HS_ERR_COPY_TIMEOUT
    p.fault->error_where = where;
    *gave_up = where;
    __threadfence();
    p.fault->error_id = p.call_id;
}

template <int kValue> struct Int { static constexpr int value = kValue; };

// The blocks of 16 x 16 on and below the diagonal of a C x C matrix, each 16 rows of 32 bytes: row by row of them, or column by column
// (an operand whose sums run along its rows takes a column of blocks at a time, one whose sums run along its columns a row).
template <int C> struct Blocks {
    static constexpr int kAlong = C / 16, kCount = kAlong * (kAlong + 1) / 2;
    static __host__ __device__ constexpr int by_rows(int i, int j) { return i * (i + 1) / 2 + j; }
    static __host__ __device__ constexpr int by_columns(int i, int j) { return j * kAlong - j * (j - 1) / 2 + (i - j); }
};
__device__ __forceinline__ uint32_t in_block(int block, int row, int piece) { return block * 512 + place<32>(row, piece); }

// What chunk_kernel writes: six vectors over the tokens and the decay of the whole chunk; the blocks of N by columns, kBack by rows as
// well; those of P, by columns, kBack by rows; as bf16 terms.
template <int C, int kTermsN, int kTermsP, bool kBack> struct Image {
    // e^{c}, e^{c_C-c}, beta, c in two parts, e^{c_m-c} with m the last of the token's sixteen; the whole chunk's decay and its logarithm
    static constexpr uint32_t early = 0, late = C * 4, beta = 2 * C * 4, hi = 3 * C * 4, lo = 4 * C * 4, edge = 5 * C * 4, whole = 6 * C * 4;
    static constexpr uint32_t plane = Blocks<C>::kCount * 512, n = 6 * C * 4 + 256, rows = n + kTermsN * plane, p = rows + (kBack ? kTermsN * plane : 0),
                              end = p + kTermsP * plane;
    static_assert(n % 256 == 0 && plane % 256 == 0, "the swizzle of 32-byte rows repeats every 256 bytes");
    static __device__ __forceinline__ int p_block(int i, int j) { return kBack ? Blocks<C>::by_rows(i, j) : Blocks<C>::by_columns(i, j); }
};

template <int KP, int C, int TI, int TM, int TP, bool kBack>
struct ChunkLayout {
    using I = Image<C, TM, TP, kBack>;
    // for each term and block of 64 columns the rows of K, then those of Q; the tensor core reads 128 rows from the first of a block
    static constexpr uint32_t block = 2 * C * 128, tile = TI * (KP / 64) * block, reads = tile + 128 * 128 - block;
    // M in three terms, then N, where K and Q were
    static constexpr uint32_t m = 0, n = 3 * I::plane, solved = n + TM * I::plane, region = (reads > solved ? reads : solved + 1023) / 1024 * 1024;
    // M's diagonal blocks in float32; the inverses in three terms
    static constexpr uint32_t diag = region, inverse = diag + C * 64, vec = inverse + 3 * C * 32, bars = vec + I::n, end = bars + 64;
    static constexpr int columns = C * (TI == 1 ? 1 : 2);  // of tensor memory
};

// M, P and N of one chunk.  [K; Q] K^T is one product of 128 rows on the tensor core (tcgen05; float32: the leading terms' product and
// the sum of the small ones side by side); a thread has a row of it, the first C threads M's, the others P's.  Then each of C / 16 warps
// inverts a diagonal block of I + M beta, and solves for 16 columns of N, transposed, block by block of rows,
//     N_iw = (I + M_ii beta_i)^{-1} (M_iw - sum_{w<=s<i} M_is beta_s N_sw),
// every N^T_sw the next product's factor in its registers.  24 bits in all of it: a wrong N is wrong for every column of V.
template <int KP, int C, int TI, int TM, int TP, bool kBack>
__global__ void __launch_bounds__(2 * C) chunk_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const Params p,
                                                      int* gave_up) {
    using L = ChunkLayout<KP, C, TI, TM, TP, kBack>;
    using I = Image<C, TM, TP, kBack>;
    constexpr int NB = C / 16;
    extern __shared__ __align__(1024) uint8_t sm8[];
    const uint32_t base = smem_addr(sm8), bars = base + L::bars;
    float* const vec = reinterpret_cast<float*>(sm8 + L::vec);
    volatile int* const stop = reinterpret_cast<int*>(sm8 + L::bars + 48);
    uint32_t* const s_tmem = reinterpret_cast<uint32_t*>(sm8 + L::bars + 56);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int n = blockIdx.x % p.chunks, bh = blockIdx.x / p.chunks, b = bh / p.heads, h = bh % p.heads;
    const int live = live_tokens(p.lengths, b, p.tokens), t0 = n * C;
    if (blockIdx.x == 0 && tid == 0) p.fault->started_id = p.call_id;
    if (t0 >= live) return;
    if (tid == 0) {
        ha::bar_init(bars, 1);
        ha::bar_init(bars + 8, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *stop = 0;
        ha::fence_smem_to_async();
        if (n != p.mute) {
            ha::bar_expect(bars, L::tile);
            for (int u = 0; u < TI; ++u)
                for (int c = 0; c < KP / 64; ++c) {
                    const uint32_t to = base + (u * (KP / 64) + c) * L::block;
                    ha::tma_load_4d(to, &mk, 64 * c, h / p.kdiv, t0, u * p.batch + b, bars);
                    ha::tma_load_4d(to + C * 128, &mq, 64 * c, h / p.qdiv, t0, u * p.batch + b, bars);
                }
        }
    }
    if (warp == 0) {
        __syncwarp();
        ha::tmem_alloc(smem_addr(s_tmem), L::columns);
    }
    if (warp == 1) {  // the decays: a lane has C / 32 tokens, sums in 64 bits
        constexpr int kOwn = C / 32;
        double c[kOwn];
        float be[kOwn];
        const float *ga = p.log_a + b * p.ab + h * p.ah, *gb = p.beta + b * p.bb + h * p.bh;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const long long t = t0 + kOwn * lane + i;
            const float a = t < live ? ga[t * p.at] : 0.0f;
            be[i] = t < live ? gb[t * p.bt] : 0.0f;
            c[i] = (i ? c[i - 1] : 0.0) + (double)(a < kReset ? kReset : a) * 1.4426950408889634;
        }
        double sum = c[kOwn - 1];
        for (int o = 1; o < 32; o *= 2) {
            const double u = __shfl_up_sync(~0u, sum, o);
            if (lane >= o) sum += u;
        }
        const double all = __shfl_sync(~0u, sum, 31), before = sum - c[kOwn - 1];
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int t = kOwn * lane + i;
            const double x = c[i] + before;
            vec[I::early / 4 + t] = ex2((float)x);
            vec[I::late / 4 + t] = ex2((float)(all - x));
            vec[I::beta / 4 + t] = be[i];
            vec[I::hi / 4 + t] = (float)x;
            vec[I::lo / 4 + t] = (float)(x - (double)(float)x);
            const double edge = __shfl_sync(~0u, c[kOwn - 1] + before, lane | (16 / kOwn - 1));
            vec[I::edge / 4 + t] = ex2((float)(edge - x));
        }
        vec[I::whole / 4 + lane] = lane == 0 ? ex2((float)all) : lane == 1 ? (float)all : 0.0f;
    }
    ha::tmem_before_sync();
    __syncthreads();
    ha::tmem_after_sync();
    const uint32_t tmem = *s_tmem;
    const Waiter wait{bars, stop, p.spin};
    if (warp == 0) {
        const bool loaded = __all_sync(~0u, wait(0, 0));
        if (!loaded) wait.drain(0, 0);
        if (loaded && ha::elect_one()) {
            constexpr uint32_t shape = ha::mma_shape(C, 0);
            const uint32_t at = ha::operand(base, 0);
            auto term = [](int u, int kk) { return (uint32_t)((u * (KP / 64) + (kk >> 2)) * (L::block >> 4) + (kk & 3) * 2); };
#pragma unroll
            for (int level = TI - 1; level >= 0; --level)
#pragma unroll
                for (int u = 0; u < TI; ++u)
                    if (level - u >= 0)
#pragma unroll
                        for (int kk = 0; kk < KP / 16; ++kk)
                            ha::mma_ss(tmem + (level ? C : 0), at + term(u, kk), at + term(level - u, kk), shape, kk > 0 || (level && (level < TI - 1 || u > 0)));
            ha::mma_commit(bars + 8);
        }
        __syncwarp();
    }
    const bool ok = __syncthreads_and(wait(1, 0));
    if (!ok) {  // outputs are not valid; nothing of this CTA's is in flight, or was not within the limit
        if (warp == 0) {
            wait.drain(1, 0);
            ha::tmem_free(tmem, L::columns);
        }
        if (tid == 0) give_up(p, gave_up, 1);
        return;
    }
    ha::tmem_after_sync();
    uint8_t* const image = p.image + (long long)blockIdx.x * I::end;
    {   // weights of a row
        const bool mine_p = tid >= C;
        const int i = tid & (C - 1), ib = i >> 4;
        const float own_hi = vec[I::hi / 4 + i], own_lo = vec[I::lo / 4 + i];
        float* const diag = reinterpret_cast<float*>(sm8 + L::diag) + ib * 256 + (i & 15);
#pragma unroll 1
        for (int jb = 0; jb <= ((tid | 31) & (C - 1)) >> 4; ++jb) {  // the warp's last row says how far
            uint32_t v[16];
            float x[16];
            __syncwarp();
            ha::tmem_ld16(v, tmem + ((uint32_t)(tid & ~31) << 16) + 16 * jb);
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = __uint_as_float(v[e]);
            if constexpr (TI > 1) {
                ha::tmem_ld16(v, tmem + ((uint32_t)(tid & ~31) << 16) + C + 16 * jb);
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] += __uint_as_float(v[e]);
            }
            if (jb > ib) continue;
            if (16 * jb + 15 < (tid & (C - 32))) {
                // Sixteen columns before all rows of the warp: e^{c_i-c_j} = e^{c_i-c_m} e^{c_m-c_j} with m the last of them; both exponents
                // keep their sign, and one exponential of the row serves them all.
                const int m = 16 * jb + 15;
                float f = t0 + i < live ? ex2((own_hi - vec[I::hi / 4 + m]) + (own_lo - vec[I::lo / 4 + m])) : 0.0f;
                if (mine_p) f *= p.scale;
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const float4 g = *reinterpret_cast<const float4*>(vec + I::edge / 4 + 16 * jb + e);
                    x[e] = f == 0.0f ? 0.0f : f * g.x * x[e];
                    x[e + 1] = f == 0.0f ? 0.0f : f * g.y * x[e + 1];
                    x[e + 2] = f == 0.0f ? 0.0f : f * g.z * x[e + 2];
                    x[e + 3] = f == 0.0f ? 0.0f : f * g.w * x[e + 3];
                }
            } else {
                const int last = t0 + i < live ? (mine_p ? i : i - 1) - 16 * jb : -1;  // the last column that counts
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const float4 hi = *reinterpret_cast<const float4*>(vec + I::hi / 4 + 16 * jb + e), lo = *reinterpret_cast<const float4*>(vec + I::lo / 4 + 16 * jb + e);
                    const float d[4] = {(own_hi - hi.x) + (own_lo - lo.x), (own_hi - hi.y) + (own_lo - lo.y), (own_hi - hi.z) + (own_lo - lo.z), (own_hi - hi.w) + (own_lo - lo.w)};
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float w = e + u <= last ? ex2(d[u]) : 0.0f;
                        x[e + u] = w != 0.0f ? (mine_p ? p.scale * w : w) * x[e + u] : 0.0f;
                    }
                    if (!mine_p && jb == ib)  // transposed: the inverse reads columns
#pragma unroll
                        for (int u = 0; u < 4; ++u) diag[(e + u) * 16] = x[e + u];
                }
            }
            auto put = [&](auto terms, uint8_t* to, int block) {
                constexpr int kTerms = decltype(terms)::value;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t t[4][kTerms];
#pragma unroll
                    for (int u = 0; u < 4; ++u) ha::split<kTerms>(ha::make_pair2(x[8 * half + 2 * u], x[8 * half + 2 * u + 1]), t[u]);
#pragma unroll
                    for (int u = 0; u < kTerms; ++u)
                        *reinterpret_cast<uint4*>(to + u * I::plane + in_block(block, i & 15, half)) = make_uint4(t[0][u], t[1][u], t[2][u], t[3][u]);
                }
            };
            if (mine_p) put(Int<TP>{}, image + I::p, I::p_block(ib, jb));
            else put(Int<3>{}, sm8 + L::m, Blocks<C>::by_rows(ib, jb));
        }
    }
    ha::tmem_before_sync();
    __syncthreads();
    if (warp == 0) ha::tmem_free(tmem, L::columns);
    {   // the inverse of the warp's diagonal block, a column for each lane of either half
        const float* const diag = reinterpret_cast<const float*>(sm8 + L::diag) + warp * 256;
        const int c = lane & 15;
        float x[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = r == c ? 1.0f : 0.0f;
#pragma unroll
        for (int i = 0; i < 15; ++i) {
            const float y = vec[I::beta / 4 + 16 * warp + i] * x[i];
#pragma unroll
            for (int r = (i + 1) / 4 * 4; r < 16; r += 4) {
                const float4 f = *reinterpret_cast<const float4*>(diag + i * 16 + r);
                const float g[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (r + u > i) x[r + u] = fmaf(-g[u], y, x[r + u]);
            }
        }
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
            uint32_t t[3];
            ha::split<3>(ha::make_pair2(x[r], x[r + 1]), t);
            if (lane < 16)
#pragma unroll
                for (int u = 0; u < 3; ++u) {
                    uint8_t* const to = sm8 + L::inverse + u * (C * 32) + 2 * (c & 7);
                    *reinterpret_cast<uint16_t*>(to + place<32>(16 * warp + r, c >> 3)) = (uint16_t)t[u];
                    *reinterpret_cast<uint16_t*>(to + place<32>(16 * warp + r + 1, c >> 3)) = (uint16_t)(t[u] >> 16);
                }
        }
    }
    __syncthreads();
    const Lane at;
    const int j0 = 2 * (lane & 3);
    uint32_t done[NB][3][4];  // -(N^T_sw) beta_s as an operand
#pragma unroll
    for (int i = 0; i < NB; ++i)
        if (i >= warp) {
            float r[2][4] = {}, x[2][4] = {};
            {   // M^T_iw
                uint32_t m[4];
#pragma unroll
                for (int u = 2; u >= 0; --u) {
                    load4_t(m, base + L::m + u * I::plane + in_block(Blocks<C>::by_rows(i, warp), at.b_row(), at.b_piece()));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        r[e >> 1][2 * (e & 1)] += __uint_as_float(m[e] << 16);
                        r[e >> 1][2 * (e & 1) + 1] += __uint_as_float(m[e] & 0xffff0000u);
                    }
                }
            }
            float t[NB][2][4] = {};  // products that do not wait for each other
            uint32_t bf[NB][1][3][4], a[3][4];
#pragma unroll
            for (int s = 0; s < i; ++s)
                if (s >= warp)
#pragma unroll
                    for (int u = 0; u < 3; ++u) load4(bf[s][0][u], base + L::m + u * I::plane + in_block(Blocks<C>::by_rows(i, s), at.b_row(), at.b_piece()));
#pragma unroll
            for (int level = 2; level >= 0; --level)
#pragma unroll
                for (int u = 0; u <= level; ++u)
#pragma unroll
                    for (int s = 0; s < i; ++s)
                        if (s >= warp) {
                            mma(t[s][0], done[s][u], bf[s][0][level - u][0], bf[s][0][level - u][1]);
                            mma(t[s][1], done[s][u], bf[s][0][level - u][2], bf[s][0][level - u][3]);
                        }
#pragma unroll
            for (int s = 0; s < i; ++s)
                if (s >= warp)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        r[0][e] += t[s][0][e];
                        r[1][e] += t[s][1][e];
                    }
            as_operand<3>(a, r[0], r[1]);
            uint32_t bi[1][3][4];
#pragma unroll
            for (int u = 0; u < 3; ++u) load4(bi[0][u], base + L::inverse + u * (C * 32) + place<32>(16 * i + at.b_row(), at.b_piece()));
            products<2>(x, a, bi);
            float w[2][4];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const float2 be = *reinterpret_cast<const float2*>(vec + I::beta / 4 + 16 * i + 8 * y + j0);
#pragma unroll
                for (int e = 0; e < 4; ++e) w[y][e] = -(e & 1 ? be.y : be.x) * x[y][e];
            }
            if (i + 1 < NB) as_operand<3>(done[i], w[0], w[1]);
            as_operand<3>(a, x[0], x[1]);
#pragma unroll
            for (int u = 0; u < TM; ++u)  // in the order in which M^T was loaded
                store4_t(base + L::n + u * I::plane + in_block(Blocks<C>::by_columns(i, warp), at.b_row(), at.b_piece()), a[u]);
        }
    __syncthreads();
    uint4* to = reinterpret_cast<uint4*>(image);
    for (uint32_t e = tid; e < I::n / 16; e += 2 * C) to[e] = reinterpret_cast<const uint4*>(sm8 + L::vec)[e];
    for (uint32_t e = tid; e < (I::rows - I::n) / 16; e += 2 * C) {
        const uint4 f = reinterpret_cast<const uint4*>(sm8 + L::n)[e];
        to[I::n / 16 + e] = f;
        if constexpr (kBack) {
            const int block = e / 32 % Blocks<C>::kCount;
            int j = 0;
            while (j + 1 < NB && block >= Blocks<C>::by_columns(j + 1, j + 1)) ++j;
            const int i = block - Blocks<C>::by_columns(j, j) + j;
            to[I::rows / 16 + e + (Blocks<C>::by_rows(i, j) - block) * 32] = f;
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------- scan

constexpr int kMaxWarps = 8;
// Warps of a CTA: those with columns of V, in groups of four (the rest of a group idles), and a group of which one loads.  Registers
// move between groups: 168 a thread at launch, 3 * 168 = 2 * 224 + 56 (with one group of columns 2 * 168 > 224 + 56).
constexpr int kScanThreads = 32 * (kMaxWarps + 4), kColumnRegs = 224, kLoadRegs = 56;
static_assert(2 * kColumnRegs + kLoadRegs <= 3 * 168 && kScanThreads * 168 <= 65536, "registers");
__host__ __device__ constexpr int loader_of(int warps) { return (warps + 3) / 4 * 4; }

// kQ: a tile of Q and the weights P
template <int KP, int C, int TI, int TM, int TP, bool kQ, bool kBack>
struct ScanLayout {
    using I = Image<C, TM, TP, kBack>;
    static constexpr int kStages = TI == 1 ? 2 : 1;
    static constexpr uint32_t tile = KP * C * 2 * TI, k = 0, q = tile, v = q + (kQ ? tile : 0), own = C * 32;  // V: 16 columns for each warp
    static constexpr uint32_t image_bytes = kQ ? I::end : I::rows;
    static __host__ __device__ constexpr uint32_t image(int warps) { return v + warps * TI * own; }
    static __host__ __device__ constexpr uint32_t stage(int warps) { return (image(warps) + image_bytes + 1023) / 1024 * 1024; }
    // stages, the output's staging (16 columns for each warp, bf16), barriers
    static __host__ __device__ constexpr uint32_t out(int warps) { return kStages * stage(warps); }
    static __host__ __device__ constexpr uint32_t bars(int warps) { return out(warps) + (kQ && TI == 1 ? warps * own : 0); }
    static __host__ __device__ constexpr uint32_t end(int warps) { return bars(warps) + 128; }
};

enum ScanBar : int { kFull = 0, kEmpty = 2, kPatched = 4, kScanBars = 5 };

// The warp that loads.  `load` issues a chunk's copies for a barrier.  The rows behind the sequence's end are set to zero, since
// 0 * NaN must not reach a sum over tokens: those of the first `wide_bytes` of the stage (C tokens in blocks of 64 columns) and of
// `narrow_bytes` behind them (C tokens in tiles of 16 columns).
template <int C, int kStages, class Load>
__device__ __forceinline__ void load_chunks(const Waiter& wait, uint8_t* sm8, uint32_t stage_bytes, uint32_t wide_bytes, uint32_t narrow_bytes, int count,
                                            int live, int tokens, uint32_t bytes, int mute, Load load, bool backwards) {
    const int lane = threadIdx.x & 31;
    bool ok = true;
    int loads = 0, patched = -1;
    for (int it = 0; it < count && ok; ++it) {
        const int n = backwards ? count - 1 - it : it, s = it % kStages, t0 = n * C;
        const bool patch = live < tokens && t0 + C > live;
        if (lane == 0) {
            if (it >= kStages) ok = wait(kEmpty + s, it / kStages - 1);
            if (n == mute) ok = false;
            if (ok) {
                const int bar = patch ? kPatched : kFull + s;
                ha::bar_expect(wait.bars + 8 * bar, bytes);
                load(n, s, wait.bars + 8 * bar);
                loads = it + 1;
                if (patch) patched = it;
            }
        }
        ok = __shfl_sync(~0u, (int)ok, 0);
        if (patch && ok) {
            ok = __all_sync(~0u, wait(kPatched, 0));
            const int rows = t0 + C - live;
            uint8_t* const stage = sm8 + s * stage_bytes;
            for (uint32_t block = 0; ok && block < wide_bytes; block += C * 128)
                for (int e = lane; e < rows * 8; e += 32)
                    *reinterpret_cast<uint4*>(stage + block + (live - t0) * 128 + e * 16) = make_uint4(0, 0, 0, 0);
            for (uint32_t block = wide_bytes; ok && block < wide_bytes + narrow_bytes; block += C * 32)
                for (int e = lane; e < rows * 2; e += 32)
                    *reinterpret_cast<uint4*>(stage + block + (live - t0) * 32 + e * 16) = make_uint4(0, 0, 0, 0);
            ha::fence_smem_to_async();
            __syncwarp();
            if (lane == 0 && ok) ha::bar_arrive(wait.bars + 8 * (kFull + s));
        }
    }
    if (lane == 0)  // nothing may land in shared memory after the CTA has left
        for (int it = max(0, loads - kStages); it < loads; ++it) {
            if (it == patched) wait.drain(kPatched, 0);
            else wait.drain(kFull + it % kStages, it / kStages);
        }
}

// Sixteen columns of S^T as accumulators: lane l has columns v0 + l / 4 and the eighth after, entries 8 j + 2 (l % 4) and the next.
template <int KP>
__device__ __forceinline__ void read_state(float (&s)[KP / 8][4], const float* from, int dk, int dv, int v0) {
    const int lane = threadIdx.x & 31, v = v0 + (lane >> 2), k = 2 * (lane & 3);
#pragma unroll
    for (int j = 0; j < KP / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int kk = 8 * j + k + (e & 1), vv = v + (e >> 1) * 8;
            s[j][e] = from && kk < dk && vv < dv ? from[(long long)kk * dv + vv] : 0.0f;
        }
}
template <int KP>
__device__ __forceinline__ void write_state(const float (&s)[KP / 8][4], float* to, int dk, int dv, int v0) {
    const int lane = threadIdx.x & 31, v = v0 + (lane >> 2), k = 2 * (lane & 3);
#pragma unroll
    for (int j = 0; j < KP / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int kk = 8 * j + k + (e & 1), vv = v + (e >> 1) * 8;
            if (kk < dk && vv < dv) to[(long long)kk * dv + vv] = s[j][e];
        }
}
// Accumulators [16][8 n] to rows of `pitch` floats
template <int kTiles>
__device__ __forceinline__ void dump_rows(const float (&s)[kTiles][4], float* to, int pitch) {
    const int lane = threadIdx.x & 31;
    float* at = to + (lane >> 2) * pitch + 2 * (lane & 3);
#pragma unroll
    for (int j = 0; j < kTiles; ++j) {
        *reinterpret_cast<float2*>(at + 8 * j) = make_float2(s[j][0], s[j][1]);
        *reinterpret_cast<float2*>(at + 8 * pitch + 8 * j) = make_float2(s[j][2], s[j][3]);
    }
}

// Sixteen columns of the output of one chunk: o^T in accumulators, tokens as columns; tokens from `live` on are zero.
template <int C, class T>
__device__ __forceinline__ void write_out(const float (&o)[C / 8][4], const CUtensorMap* map, const Params& p, uint8_t* stage, int b, int h, int v0, int t0,
                                          int live) {
    const int lane = threadIdx.x & 31, j0 = 2 * (lane & 3);
    if (sizeof(T) == 2 && p.out_tma) {
        const Lane at;
        if (lane == 0) ha::tma_store_wait_read();
        __syncwarp();
#pragma unroll
        for (int np = 0; np < C / 16; ++np) {
            uint32_t r[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int nt = 2 * np + (u >> 1), t = t0 + 8 * nt + j0, e = 2 * (u & 1);
                r[u] = ha::pack_bf16(t < live ? o[nt][e] : 0.0f, t + 1 < live ? o[nt][e + 1] : 0.0f);
            }
            store4_t(smem_addr(stage) + place<32>(16 * np + at.b_row(), at.b_piece()), r);
        }
        ha::fence_smem_to_async();
        __syncwarp();
        if (lane == 0) {
            if (v0 < p.dv) ha::tma_store_4d(map, v0, h, t0, b, smem_addr(stage));
            ha::tma_store_commit();
        }
        return;
    }
    T* go = static_cast<T*>(p.out) + b * p.ob + h * p.oh;
#pragma unroll
    for (int nt = 0; nt < C / 8; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int t = t0 + 8 * nt + j0 + (e & 1), v = v0 + (lane >> 2) + 8 * (e >> 1);
            if (t < p.tokens && v < p.dv) go[t * p.ot + v] = ha::from_f<T>(t < live ? o[nt][e] : 0.0f);
        }
}
// Tokens of chunks that hold none of the sequence: zeros
template <class T>
__device__ __forceinline__ void zero_out(const Params& p, int b, int h, int v0, int from) {
    const int lane = threadIdx.x & 31, v = v0 + (lane & 15);
    T* go = static_cast<T*>(p.out) + b * p.ob + h * p.oh;
    for (long long t = from + (lane >> 4); t < p.tokens; t += 2)
        if (v < p.dv) go[t * p.ot + v] = ha::from_f<T>(0.0f);
}

// kOut: the output; else the state before every chunk and E, for the gradients.  TO: terms of S and V' in the output.
template <int KP, int C, int TI, int TM, int TP, bool kOut, class T>
__global__ void __launch_bounds__(kScanThreads, 1)
    scan_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                const __grid_constant__ CUtensorMap mo, const Params p, int* gave_up) {
    using L = ScanLayout<KP, C, TI, TM, TP, kOut, !kOut>;
    using I = typename L::I;
    constexpr int kLevel = TM - 1, TO = TI == 1 ? 2 : 3, kGroup = TI == 1 && C == 64 ? 4 : 2;
    constexpr bool kRounded = TI == 3;
    extern __shared__ __align__(1024) uint8_t sm8[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = p.warps;
    const uint32_t base = smem_addr(sm8), stage_bytes = L::stage(warps), bars = base + L::bars(warps);
    volatile int* const stop = reinterpret_cast<int*>(sm8 + L::bars(warps) + 64);
    const Waiter wait{bars, stop, p.spin};
    const int slices = (p.dv + 15) / 16, groups = (slices + warps - 1) / warps;
    const int bh = blockIdx.x / groups, b = bh / p.heads, h = bh % p.heads, slice0 = (blockIdx.x % groups) * warps;
    const int live = live_tokens(p.lengths, b, p.tokens), count = (live + C - 1) / C;
    if (tid == 0) {
        for (int i = 0; i < kScanBars; ++i) ha::bar_init(bars + 8 * i, i >= kEmpty && i < kPatched ? warps : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *stop = 0;
    }
    __syncthreads();
    if (warp >= loader_of(warps)) {
        ha::give_registers<kLoadRegs>();
        const uint32_t bytes = (kOut ? 2 : 1) * L::tile + warps * TI * L::own + L::image_bytes;
        if (warp == loader_of(warps)) load_chunks<C, L::kStages>(
            wait, sm8, stage_bytes, kOut ? 2 * L::tile : L::tile, 0, count, live, p.tokens, bytes, p.mute,
            [&](int n, int s, uint32_t bar) {
                const uint32_t to = base + s * stage_bytes;
                bulk_load(to + L::image(warps), p.image + ((long long)bh * p.chunks + n) * I::end, L::image_bytes, bar);
                for (int u = 0; u < TI; ++u) {
                    for (int c = 0; c < KP / 64; ++c) {
                        ha::tma_load_4d(to + L::k + (u * (KP / 64) + c) * C * 128, &mk, 64 * c, h / p.kdiv, n * C, u * p.batch + b, bar);
                        if (kOut) ha::tma_load_4d(to + L::q + (u * (KP / 64) + c) * C * 128, &mq, 64 * c, h / p.qdiv, n * C, u * p.batch + b, bar);
                    }
                    for (int w = 0; w < warps; ++w)
                        ha::tma_load_4d(to + L::v + (w * TI + u) * L::own, &mv, 16 * (slice0 + w), h / p.vdiv, n * C, u * p.batch + b, bar);
                }
            },
            false);
    } else {
        ha::take_registers<kColumnRegs>();
        const Lane at;
        const int v0 = 16 * (slice0 + warp), j0 = 2 * (lane & 3);
        float s[KP / 8][4];
        read_state<KP>(s, p.s_in ? p.s_in + (long long)bh * p.dk * p.dv : nullptr, p.dk, p.dv, v0);
        bool ok = warp < warps;
        for (int it = 0; ok && it < count; ++it) {
            const int st = it % L::kStages, t0 = it * C;
            ok = __all_sync(~0u, wait(kFull + st, it / L::kStages));
            if (!ok) break;
            const uint32_t to = base + st * stage_bytes, K = to + L::k, Q = to + L::q, V = to + L::v + warp * TI * L::own, N = to + L::image(warps) + I::n,
                           P = to + L::image(warps) + I::p;
            const float* const vec = reinterpret_cast<const float*>(sm8 + st * stage_bytes + L::image(warps));
            if constexpr (!kOut)
                if (v0 < p.dv) dump_rows(s, p.states + (((long long)bh * p.chunks + it) * slices * 16 + v0) * KP, KP);
            float y[C / 8][4] = {}, o[kOut ? C / 8 : 1][4] = {};
#pragma unroll
            for (int kk = 0; kk < KP / 16; ++kk) {  // (K S)^T and (Q S)^T
                uint32_t a[TM][4];
                as_operand<TM>(a, s[2 * kk], s[2 * kk + 1]);
#pragma unroll
                for (int np = 0; np < C / 16; np += kGroup) {
                    uint32_t bf[kGroup][TI][4];
#pragma unroll
                    for (int g = 0; g < kGroup; ++g)
#pragma unroll
                        for (int u = 0; u < TI; ++u)
                            load4(bf[g][u], K + u * (KP * C * 2) + wide<C>(16 * (np + g) + at.b_row(), 2 * kk + at.b_piece()));
                    sum<kRounded, kLevel>(y + 2 * np, a, bf);
                    if constexpr (kOut) {
#pragma unroll
                        for (int g = 0; g < kGroup; ++g)
#pragma unroll
                            for (int u = 0; u < TI; ++u)
                                load4(bf[g][u], Q + u * (KP * C * 2) + wide<C>(16 * (np + g) + at.b_row(), 2 * kk + at.b_piece()));
                        sum<kRounded, TO - 1>(o + 2 * np, a, bf);
                    }
                }
            }
#pragma unroll
            for (int np = 0; np < C / 16; ++np) {  // Y^T
                uint32_t vf[TI][4];
#pragma unroll
                for (int u = 0; u < TI; ++u) load4_t(vf[u], V + u * L::own + place<32>(16 * np + at.b_row(), at.b_piece()));
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int nt = 2 * np + x;
                    const float2 e = *reinterpret_cast<const float2*>(vec + I::early / 4 + 8 * nt + j0);
                    const bool on0 = t0 + 8 * nt + j0 < live, on1 = t0 + 8 * nt + j0 + 1 < live;
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float f0 = 0.0f, f1 = 0.0f;
#pragma unroll
                        for (int u = TI - 1; u >= 0; --u) {
                            f0 += __uint_as_float(vf[u][2 * x + r] << 16);
                            f1 += __uint_as_float(vf[u][2 * x + r] & 0xffff0000u);
                        }
                        y[nt][2 * r] = on0 ? f0 - ha::decayed(e.x, y[nt][2 * r]) : 0.0f;
                        y[nt][2 * r + 1] = on1 ? f1 - ha::decayed(e.y, y[nt][2 * r + 1]) : 0.0f;
                    }
                    if constexpr (kOut) {
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            o[nt][2 * r] = ha::decayed(e.x, p.scale * o[nt][2 * r]);
                            o[nt][2 * r + 1] = ha::decayed(e.y, p.scale * o[nt][2 * r + 1]);
                        }
                    }
                }
            }
            // E^T in place, from the last sixteen tokens on: theirs are needed by no other before they change
#pragma unroll
            for (int jj = C / 16 - 1; jj >= 0; --jj) {
                float w[2][4];
                uint32_t a[TM][4];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const float2 be = *reinterpret_cast<const float2*>(vec + I::beta / 4 + 16 * jj + 8 * x + j0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[x][e] = -(e & 1 ? be.y : be.x) * y[2 * jj + x][e];
                }
                as_operand<TM>(a, w[0], w[1]);
#pragma unroll
                for (int np = jj; np < C / 16; np += 2) {
                    const int pairs = np + 1 < C / 16 ? 2 : 1;
                    uint32_t bf[2][TM][4];
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int u = 0; u < TM; ++u)
                            if (g < pairs) load4(bf[g][u], N + u * I::plane + in_block(Blocks<C>::by_columns(np + g, jj), at.b_row(), at.b_piece()));
                    sum<kRounded, kLevel>(y + 2 * np, a, bf, pairs);
                }
            }
            if constexpr (!kOut)
                if (v0 < p.dv) dump_rows(y, p.errors + (((long long)bh * p.chunks + it) * slices * 16 + v0) * C, C);
#pragma unroll
            for (int nt = 0; nt < C / 8; ++nt) {  // V'^T
                const float2 be = *reinterpret_cast<const float2*>(vec + I::beta / 4 + 8 * nt + j0);
#pragma unroll
                for (int e = 0; e < 4; ++e) y[nt][e] *= e & 1 ? be.y : be.x;
            }
            if constexpr (kOut) {
#pragma unroll
                for (int jj = 0; jj < C / 16; ++jj) {
                    uint32_t a[TO][4];
                    as_operand<TO>(a, y[2 * jj], y[2 * jj + 1]);
#pragma unroll
                    for (int np = jj; np < C / 16; np += 2) {
                        const int pairs = np + 1 < C / 16 ? 2 : 1;
                        uint32_t bf[2][TP][4];
#pragma unroll
                        for (int g = 0; g < 2; ++g)
#pragma unroll
                            for (int u = 0; u < TP; ++u)
                                if (g < pairs) load4(bf[g][u], P + u * I::plane + in_block(I::p_block(np + g, jj), at.b_row(), at.b_piece()));
                        sum<kRounded, TO - 1>(o + 2 * np, a, bf, pairs);
                    }
                }
                write_out<C, T>(o, &mo, p, sm8 + L::out(warps) + warp * L::own, b, h, v0, t0, live);
            }
            const float whole = vec[I::whole / 4];
            uint32_t au[C / 16][TM][4];
#pragma unroll
            for (int jj = 0; jj < C / 16; ++jj) {
                float w[2][4];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const float2 la = *reinterpret_cast<const float2*>(vec + I::late / 4 + 16 * jj + 8 * x + j0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[x][e] = (e & 1 ? la.y : la.x) * y[2 * jj + x][e];
                }
                as_operand<TM>(au[jj], w[0], w[1]);
            }
#pragma unroll
            for (int kp = 0; kp < KP / 16; kp += kGroup) {  // the update by itself, added once: the old state is rounded, not cut off
                float up[2 * kGroup][4] = {};
#pragma unroll
                for (int jj = 0; jj < C / 16; ++jj) {
                    uint32_t bf[kGroup][TI][4];
#pragma unroll
                    for (int g = 0; g < kGroup; ++g)
#pragma unroll
                        for (int u = 0; u < TI; ++u)
                            load4_t(bf[g][u], K + u * (KP * C * 2) + wide<C>(16 * jj + at.bt_row(), 2 * (kp + g) + at.bt_piece()));
                    sum<kRounded, kLevel>(up, au[jj], bf);
                }
#pragma unroll
                for (int n = 0; n < 2 * kGroup; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[2 * kp + n][e] = whole == 0.0f ? up[n][e] : fmaf(whole, s[2 * kp + n][e], up[n][e]);
            }
            ha::release_reads();
            __syncwarp();
            if (lane == 0) ha::bar_arrive(bars + 8 * (kEmpty + st));
        }
        if (kOut && lane == 0) ha::tma_store_wait_all();
        if (kOut && warp < warps && v0 < p.dv) zero_out<T>(p, b, h, v0, count * C);
        if (ok && p.s_out && v0 < p.dv) write_state<KP>(s, p.s_out + (long long)bh * p.dk * p.dv, p.dk, p.dv, v0);
    }
    __syncthreads();
    if (tid == 0 && *stop) give_up(p, gave_up, 1 + *stop);
}

// ------------------------------------------------------------------------------------------------- tensors for TMA

// A [batch, tokens, heads, dim] tensor that TMA cannot load as it is (float32, odd sizes or strides) as bf16 terms,
// [term][batch][tokens][heads][width], columns from dim on zero.
template <int TI, class T>
__global__ void __launch_bounds__(256) terms_kernel(const ha::Rows from, __nv_bfloat16* to, int tokens, int heads, int dim, int width, long long total) {
    for (long long e = (long long)blockIdx.x * blockDim.x + threadIdx.x; e < total; e += (long long)gridDim.x * blockDim.x) {
        const int d = (int)(e % width);
        const long long row = e / width, bt = row / heads;
        float x = 0.0f;
        if (d < dim) x = ha::to_f(static_cast<const T*>(from.ptr)[bt / tokens * from.sb + bt % tokens * from.st + row % heads * from.sh + d]);
#pragma unroll
        for (int u = 0; u < TI; ++u) {
            const __nv_bfloat16 t = __float2bfloat16_rn(x);
            to[u * total + e] = t;
            x -= __bfloat162float(t);
        }
    }
}

}  // namespace hd
