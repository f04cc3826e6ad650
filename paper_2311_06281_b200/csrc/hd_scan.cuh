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
// Two kernels a direction.  chunk_kernel forms M, P and N of every chunk, all chunks at once.  The scans walk a sequence's chunks: on
// tcgen05 (hd_scan_mma.cuh), or here with mma.sync, which is for all that the other is not (float32, wide keys) and where there are
// few sequences and heads.  A slice of sixteen columns of V has four warps, one on each scheduler of an SM; each has a quarter of the
// state's rows for it, transposed, as accumulators, and a quarter of a chunk's tokens.  Products over the state's rows are added up
// between the four (one barrier), and each hands the others its tokens' Y and V' as factors (two more), so that the state never leaves
// its registers.  Against one warp for a slice with all of the state: 16385 tokens, 8 heads of 128, 1.23 ms -> 0.64 ms.
//
// What bounds it: chunks follow each other, and in a chunk the sums, the solution and the update.  A chunk takes a slice 2.4 us (keys
// 128 wide; four barriers, 120 to 250 products of a warp one behind the other's operands), with the tensor pipe busy 41% of the time
// and two slices on an SM.
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
    int slices;            // of sixteen columns of V, of a CTA of the scans
    uint8_t* image;        // what chunk_kernel leaves for each (batch, head) and chunk
    const float* s_in;     // [batch, heads, dk, dv] or NULL
    float* s_out;          // or NULL
    void* out;             // o (backward: dv) through its strides
    long long ob, ot, oh;
    float* states;         // backward: before every chunk the state (after it, its gradient), [batch * heads][chunks][16 slices][KP]
    float* errors;         // E (F) of every chunk, [batch * heads][chunks][16 slices][C]
    float* errors_back;    // F likewise (both as slabs where grad_mma_kernel reads them: dump_state, dump_errors)
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

// x[e] = factor e^{c_i-c_j} x[e] for sixteen tokens j up to the last one that counts, zero behind it (whatever x holds there)
__device__ __forceinline__ void between_tokens(float (&x)[16], const float* hi, const float* lo, float own_hi, float own_lo, float factor, int last) {
    const ha::pair minus = ha::make_pair2(-1.0f, -1.0f), h = ha::make_pair2(own_hi, own_hi), l = ha::make_pair2(own_lo, own_lo), f = ha::make_pair2(factor, factor);
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
        const float4 h4 = *reinterpret_cast<const float4*>(hi + e), l4 = *reinterpret_cast<const float4*>(lo + e);
#pragma unroll
        for (int u = 0; u < 4; u += 2) {
            float d0, d1;
            ha::parts(ha::add2(ha::fma2(u ? ha::make_pair2(h4.z, h4.w) : ha::make_pair2(h4.x, h4.y), minus, h),
                               ha::fma2(u ? ha::make_pair2(l4.z, l4.w) : ha::make_pair2(l4.x, l4.y), minus, l)), d0, d1);
            d0 = e + u <= last ? ex2(d0) : 0.0f;
            d1 = e + u + 1 <= last ? ex2(d1) : 0.0f;
            const ha::pair y = ha::make_pair2(e + u <= last ? x[e + u] : 0.0f, e + u + 1 <= last ? x[e + u + 1] : 0.0f);
            ha::parts(ha::mul2(ha::mul2(f, ha::make_pair2(d0, d1)), y), x[e + u], x[e + u + 1]);
        }
    }
}

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
// Bound by the instructions around the products (issue slots 47%, tensor pipe 21%): the weights between tokens, two to an instruction
// and with one exponential for a row of a block where the block lies before all of the warp's rows, the splitting into terms and the
// solution's chain.  2048 chunks of 64 tokens, keys 128 wide: 40 us (56 MB of images written), with five CTAs to an SM for four 45 us,
// with the weights one by one 54 us.
template <int KP, int C, int TI, int TM, int TP, bool kBack>
__global__ void __launch_bounds__(2 * C, C == 64 && TI == 1 ? 5 : 1) chunk_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const Params p,
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
                const bool on = t0 + i < live;
                float f = on ? ex2((own_hi - vec[I::hi / 4 + m]) + (own_lo - vec[I::lo / 4 + m])) : 0.0f;
                if (mine_p) f *= p.scale;
                const ha::pair f2 = ha::make_pair2(f, f);
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const float4 g = *reinterpret_cast<const float4*>(vec + I::edge / 4 + 16 * jb + e);
#pragma unroll
                    for (int u = 0; u < 4; u += 2)
                        ha::parts(ha::mul2(ha::mul2(f2, u ? ha::make_pair2(g.z, g.w) : ha::make_pair2(g.x, g.y)),
                                           ha::make_pair2(on ? x[e + u] : 0.0f, on ? x[e + u + 1] : 0.0f)), x[e + u], x[e + u + 1]);
                }
            } else {
                const int last = t0 + i < live ? (mine_p ? i : i - 1) - 16 * jb : -1;  // the last column that counts
                between_tokens(x, vec + I::hi / 4 + 16 * jb, vec + I::lo / 4 + 16 * jb, own_hi, own_lo, mine_p ? p.scale : 1.0f, last);
                if (!mine_p && jb == ib)  // transposed: the inverse reads columns
#pragma unroll
                    for (int e = 0; e < 16; ++e) diag[e * 16] = x[e];
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

// A CTA has one or two slices of sixteen columns of V, four warps each, and a warp that loads (in a group of its own).
constexpr int kMaxSlices = 2, kScanThreads = 128 * (kMaxSlices + 1);

// kQ: a tile of Q and the weights P
template <int KP, int C, int TI, int TM, int TP, bool kQ, bool kBack>
struct ScanLayout {
    using I = Image<C, TM, TP, kBack>;
    static constexpr int kStages = TI == 1 ? 2 : 1, NB = C / 16;
    static constexpr uint32_t tile = KP * C * 2 * TI, k = 0, q = tile, v = q + (kQ ? tile : 0), own = C * 32;  // V: 16 columns for each slice
    static constexpr uint32_t image_bytes = kQ ? I::end : I::rows;
    static __host__ __device__ constexpr uint32_t image(int slices) { return v + slices * TI * own; }
    static __host__ __device__ constexpr uint32_t stage(int slices) { return (image(slices) + image_bytes + 1023) / 1024 * 1024; }
    // what the warps of a slice hand each other: two sets of partial sums (three for each block of tokens, 1 KB each), whose place
    // factors of later products take, and three terms of a factor
    static constexpr uint32_t sums = NB * 3 * 1024, factors = NB * 3 * 512, slice = 2 * sums + factors;
    static_assert(2 * factors <= 2 * sums, "factors in the place of sums");
    static __host__ __device__ constexpr uint32_t shared(int slices) { return kStages * stage(slices); }
    static __host__ __device__ constexpr uint32_t bars(int slices) { return shared(slices) + slices * slice; }
    static __host__ __device__ constexpr uint32_t end(int slices) { return bars(slices) + 128; }
};

// The four warps of a slice
__device__ __forceinline__ void slice_sync(int slice) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(slice + 1) : "memory"); }

// Partial sums over a quarter of the state's rows, [16][C], added up: warp w gets the sixteen tokens of block w, in the order of the
// warps.  A barrier between the two halves.
template <int NB>
__device__ __forceinline__ void hand_out(const float (&y)[2 * NB][4], float (&own)[2][4], uint8_t* to, int w) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 0; d < NB; ++d) {
        if (d == w) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                own[0][e] = y[2 * d][e];
                own[1][e] = y[2 * d + 1][e];
            }
        } else {
            float4* const at = reinterpret_cast<float4*>(to + (d * 3 + (w < d ? w : w - 1)) * 1024) + lane;
            at[0] = make_float4(y[2 * d][0], y[2 * d][1], y[2 * d][2], y[2 * d][3]);
            at[32] = make_float4(y[2 * d + 1][0], y[2 * d + 1][1], y[2 * d + 1][2], y[2 * d + 1][3]);
        }
    }
}
__device__ __forceinline__ void add_up(float (&own)[2][4], const uint8_t* from, int w) {
    const int lane = threadIdx.x & 31;
    float sum[2][4] = {};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if (u == w) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sum[0][e] += own[0][e];
                sum[1][e] += own[1][e];
            }
        } else {
            const float4* const at = reinterpret_cast<const float4*>(from + (w * 3 + (u < w ? u : u - 1)) * 1024) + lane;
            const float4 a = at[0], b = at[32];
            sum[0][0] += a.x; sum[0][1] += a.y; sum[0][2] += a.z; sum[0][3] += a.w;
            sum[1][0] += b.x; sum[1][1] += b.y; sum[1][2] += b.z; sum[1][3] += b.w;
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        own[0][e] = sum[0][e];
        own[1][e] = sum[1][e];
    }
}
// Factors of one block of tokens, from warp to warp
template <int kTerms>
__device__ __forceinline__ void put_factor(uint8_t* to, int block, const uint32_t (&a)[kTerms][4]) {
#pragma unroll
    for (int u = 0; u < kTerms; ++u)
        reinterpret_cast<uint4*>(to + (block * 3 + u) * 512)[threadIdx.x & 31] = make_uint4(a[u][0], a[u][1], a[u][2], a[u][3]);
}
template <int kTerms>
__device__ __forceinline__ void get_factor(uint32_t (&a)[kTerms][4], const uint8_t* from, int block) {
#pragma unroll
    for (int u = 0; u < kTerms; ++u) {
        const uint4 f = reinterpret_cast<const uint4*>(from + (block * 3 + u) * 512)[threadIdx.x & 31];
        a[u][0] = f.x; a[u][1] = f.y; a[u][2] = f.z; a[u][3] = f.w;
    }
}

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

// Sixteen columns of kTiles * 8 rows of S, transposed, as accumulators: lane l has columns v0 + l / 4 and the eighth after, rows
// k0 + 8 j + 2 (l % 4) and the next.
template <int kTiles>
__device__ __forceinline__ void read_state(float (&s)[kTiles][4], const float* from, int dk, int dv, int v0, int k0) {
    const int lane = threadIdx.x & 31, v = v0 + (lane >> 2), k = k0 + 2 * (lane & 3);
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int kk = 8 * j + k + (e & 1), vv = v + (e >> 1) * 8;
            s[j][e] = from && kk < dk && vv < dv ? from[(long long)kk * dv + vv] : 0.0f;
        }
}
template <int kTiles>
__device__ __forceinline__ void write_state(const float (&s)[kTiles][4], float* to, int dk, int dv, int v0, int k0) {
    const int lane = threadIdx.x & 31, v = v0 + (lane >> 2), k = k0 + 2 * (lane & 3);
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int kk = 8 * j + k + (e & 1), vv = v + (e >> 1) * 8;
            if (kk < dk && vv < dv) to[(long long)kk * dv + vv] = s[j][e];
        }
}
// For the gradients: sixteen columns of the state before a chunk (its gradient behind it), and of E (F) of sixteen tokens.  kSlabs: as
// hd_grad_mma.cuh reads them, [sixteen columns][k / 4][16][4] and [sixteen columns][token][16]; else rows of KP and of C for each column.
template <int KP, bool kSlabs, int kTiles>
__device__ __forceinline__ void dump_state(const float (&s)[kTiles][4], float* to, int k0) {
    const int lane = threadIdx.x & 31, v = lane >> 2, k = k0 + 2 * (lane & 3);
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int vv = v + 8 * r, kk = k + 8 * j;
            float* const at = kSlabs ? to + (kk >> 2) * 64 + vv * 4 + (kk & 3) : to + vv * KP + kk;
            *reinterpret_cast<float2*>(at) = make_float2(s[j][2 * r], s[j][2 * r + 1]);
        }
}
template <int C, bool kSlabs>
__device__ __forceinline__ void dump_errors(const float (&y)[2][4], float* to, int block) {
    const int lane = threadIdx.x & 31, v = lane >> 2, t = 16 * block + 2 * (lane & 3);
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int vv = v + 8 * r, tt = t + 8 * x;
            if constexpr (kSlabs) {
                to[tt * 16 + vv] = y[x][2 * r];
                to[(tt + 1) * 16 + vv] = y[x][2 * r + 1];
            } else {
                *reinterpret_cast<float2*>(to + vv * C + tt) = make_float2(y[x][2 * r], y[x][2 * r + 1]);
            }
        }
}
template <int C, bool kSlabs>
__device__ __forceinline__ void read_errors(float (&y)[2][4], const float* from, int block) {
    const int lane = threadIdx.x & 31, v = lane >> 2, t = 16 * block + 2 * (lane & 3);
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int vv = v + 8 * r, tt = t + 8 * x;
            y[x][2 * r] = kSlabs ? from[tt * 16 + vv] : from[vv * C + tt];
            y[x][2 * r + 1] = kSlabs ? from[(tt + 1) * 16 + vv] : from[vv * C + tt + 1];
        }
}

// Sixteen columns of the output for sixteen tokens from t0 on: o^T in accumulators; tokens from `live` on are zero.
template <class T>
__device__ __forceinline__ void write_out(const float (&o)[2][4], const Params& p, int b, int h, int v0, int t0, int live) {
    const int lane = threadIdx.x & 31, j0 = 2 * (lane & 3);
    T* const go = static_cast<T*>(p.out) + b * p.ob + h * p.oh;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int t = t0 + 8 * x + j0 + (e & 1), v = v0 + (lane >> 2) + 8 * (e >> 1);
            if (t < p.tokens && v < p.dv) go[t * p.ot + v] = ha::from_f<T>(t < live ? o[x][e] : 0.0f);
        }
}
// Tokens of chunks that hold none of the sequence: zeros, from the four warps of a slice
template <class T>
__device__ __forceinline__ void zero_out(const Params& p, int b, int h, int v0, int from, int w) {
    const int lane = threadIdx.x & 31, v = v0 + (lane & 15);
    T* const go = static_cast<T*>(p.out) + b * p.ob + h * p.oh;
    for (long long t = from + 2 * w + (lane >> 4); t < p.tokens; t += 8)
        if (v < p.dv) go[t * p.ot + v] = ha::from_f<T>(0.0f);
}
// w * x for the accumulators of sixteen tokens, a weight for each; decayed: a weight of zero forgets
template <bool kDecay>
__device__ __forceinline__ void weigh_tokens(float (&x)[2][4], const float* weight) {
    const int j0 = 2 * (threadIdx.x & 3);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const float2 f = *reinterpret_cast<const float2*>(weight + 8 * u + j0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float y = e & 1 ? f.y : f.x;
            x[u][e] = kDecay ? ha::decayed(y, x[u][e]) : y * x[u][e];
        }
    }
}
// Is the state forgotten behind a token of its chunk, by a log decay of -inf (kReset) that follows?  What the state answers there then meets
// nothing but weights of zero, and has to be a number: 0 * NaN must not reach the tokens behind.  (A chunk's log decays sum up to less
// than kReset only where one of them is below -156, whose decay is zero too.)
__device__ __forceinline__ bool forgotten(float whole_log, float token_log) { return whole_log - token_log < 0.99f * kReset * kLog2e; }
__device__ __forceinline__ float number(float x) { return fabsf(x) < __int_as_float(0x7f800000) ? x : 0.0f; }

// Sixteen tokens of sixteen columns of a tile of V (dO), transposed, as float32
template <int TI>
__device__ __forceinline__ void read_values(float (&y)[2][4], uint32_t tile, uint32_t term, int block, const Lane& at) {
    uint32_t f[TI][4];
#pragma unroll
    for (int u = 0; u < TI; ++u) load4_t(f[u], tile + u * term + place<32>(16 * block + at.b_row(), at.b_piece()));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a = 0.0f, b = 0.0f;
#pragma unroll
        for (int u = TI - 1; u >= 0; --u) {
            a += __uint_as_float(f[u][e] << 16);
            b += __uint_as_float(f[u][e] & 0xffff0000u);
        }
        y[e >> 1][2 * (e & 1)] = a;
        y[e >> 1][2 * (e & 1) + 1] = b;
    }
}

// A quarter's part of the products of its rows of the state with all tokens of a tile: y += (tile S)^T, TI terms of the tile
template <int KP, int C, int kLevel, int TI, int TM>
__device__ __forceinline__ void quarter_scores(float (*y)[4], const uint32_t (&a)[KP / 64][TM][4], uint32_t tile, int piece, const Lane& at) {
#pragma unroll
    for (int kk = 0; kk < KP / 64; ++kk)
#pragma unroll
        for (int np = 0; np < C / 16; np += 2) {
            uint32_t bf[2][TI][4];
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int u = 0; u < TI; ++u) load4(bf[g][u], tile + u * (KP * C * 2) + wide<C>(16 * (np + g) + at.b_row(), piece + 2 * kk + at.b_piece()));
            sum<TI == 3, kLevel>(y + 2 * np, a[kk], bf);
        }
}

// kOut: the output; else the state before every chunk and E, for the gradients.  TO: terms of S, P and V' in the output.  Of bf16 tensors
// the state has three terms where a later state hangs on it, and all three two (16 bits) in the output, which is rounded to 8 itself.
template <int KP, int C, int TI, int TM, int TP, bool kOut, class T>
__global__ void __launch_bounds__(kScanThreads, 1)
    scan_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, const Params p,
                int* gave_up) {
    using L = ScanLayout<KP, C, TI, TM, TP, kOut, !kOut>;
    using I = typename L::I;
    using B = Blocks<C>;
    constexpr int kLevel = TM - 1, TO = TI == 1 ? 2 : 3, NB = C / 16, kTiles = KP / 32, kOwn = KP / 4;
    constexpr bool kRounded = TI == 3, kSlabs = TI == 1 && KP <= 128;
    extern __shared__ __align__(1024) uint8_t sm8[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, own_slices = p.slices;
    const uint32_t base = smem_addr(sm8), stage_bytes = L::stage(own_slices), bars = base + L::bars(own_slices);
    volatile int* const stop = reinterpret_cast<int*>(sm8 + L::bars(own_slices) + 64);
    const Waiter wait{bars, stop, p.spin};
    const int slices = (p.dv + 15) / 16, groups = (slices + own_slices - 1) / own_slices;
    const int bh = blockIdx.x / groups, b = bh / p.heads, h = bh % p.heads, slice0 = (blockIdx.x % groups) * own_slices;
    const int live = live_tokens(p.lengths, b, p.tokens), count = (live + C - 1) / C;
    if (tid == 0) {
        if (blockIdx.x == 0) p.fault->started_id = p.call_id;  // (without a token no chunk has said so)
        for (int i = 0; i < kScanBars; ++i) ha::bar_init(bars + 8 * i, i >= kEmpty && i < kPatched ? 4 * own_slices : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *stop = 0;
    }
    __syncthreads();
    if (warp >= 4 * own_slices) {
        const uint32_t bytes = (kOut ? 2 : 1) * L::tile + own_slices * TI * L::own + L::image_bytes;
        if (warp == 4 * own_slices) load_chunks<C, L::kStages>(
            wait, sm8, stage_bytes, kOut ? 2 * L::tile : L::tile, 0, count, live, p.tokens, bytes, p.mute,
            [&](int n, int s, uint32_t bar) {
                const uint32_t to = base + s * stage_bytes;
                bulk_load(to + L::image(own_slices), p.image + ((long long)bh * p.chunks + n) * I::end, L::image_bytes, bar);
                for (int u = 0; u < TI; ++u) {
                    for (int c = 0; c < KP / 64; ++c) {
                        ha::tma_load_4d(to + L::k + (u * (KP / 64) + c) * C * 128, &mk, 64 * c, h / p.kdiv, n * C, u * p.batch + b, bar);
                        if (kOut) ha::tma_load_4d(to + L::q + (u * (KP / 64) + c) * C * 128, &mq, 64 * c, h / p.qdiv, n * C, u * p.batch + b, bar);
                    }
                    for (int x = 0; x < own_slices; ++x)
                        ha::tma_load_4d(to + L::v + (x * TI + u) * L::own, &mv, 16 * (slice0 + x), h / p.vdiv, n * C, u * p.batch + b, bar);
                }
            },
            false);
    } else {
        const Lane at;
        const int slice = warp >> 2, w = warp & 3, v0 = 16 * (slice0 + slice), k0 = w * kOwn;
        uint8_t* const xs = sm8 + L::shared(own_slices) + slice * L::slice;  // partial sums of X, then factors of the update
        uint8_t* const os = xs + L::sums;                                    // ... of Q S, then V'
        uint8_t* const fs = os + L::sums;                                    // beta Y
        const bool mine = w < NB, inside = v0 < p.dv;                        // has tokens of a chunk; columns that there are
        float s[kTiles][4];
        read_state(s, p.s_in ? p.s_in + (long long)bh * p.dk * p.dv : nullptr, p.dk, p.dv, v0, k0);
        bool ok = true;
        for (int it = 0; it < count; ++it) {
            const int st = it % L::kStages, t0 = it * C;
            ok = __all_sync(~0u, ok && wait(kFull + st, it / L::kStages));
            const uint32_t to = base + st * stage_bytes, K = to + L::k, Q = to + L::q, V = to + L::v + slice * TI * L::own,
                           N = to + L::image(own_slices) + I::n, P = to + L::image(own_slices) + I::p;
            const float* const vec = reinterpret_cast<const float*>(sm8 + st * stage_bytes + L::image(own_slices));
            const long long rows = (((long long)bh * p.chunks + it) * slices * 16 + v0);
            if constexpr (!kOut)
                if (inside && ok) dump_state<KP, kSlabs>(s, p.states + rows * KP, k0);
            float x[2][4], far[2][4];
            {
                uint32_t a[kTiles / 2][TM][4];
#pragma unroll
                for (int kk = 0; kk < kTiles / 2; ++kk) as_operand<TM>(a[kk], s[2 * kk], s[2 * kk + 1]);
                float y[2 * NB][4] = {};
                quarter_scores<KP, C, kLevel, TI, TM>(y, a, K, k0 / 8, at);
                if (it > 0) slice_sync(slice);  // the factors of the update before have been read
                hand_out<NB>(y, x, xs, w);
                if constexpr (kOut) {
                    float z[2 * NB][4] = {};
                    quarter_scores<KP, C, TO - 1, TI, TM>(z, a, Q, k0 / 8, at);
                    hand_out<NB>(z, far, os, w);
                }
            }
            slice_sync(slice);
            if (mine) {
                float y[2][4];
                add_up(x, xs, w);
                weigh_tokens<true>(x, vec + I::early / 4 + 16 * w);
                if (vec[I::whole / 4] == 0.0f)
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (forgotten(vec[I::whole / 4 + 1], vec[I::hi / 4 + 16 * w + 8 * u + 2 * (lane & 3) + (e & 1)])) x[u][e] = number(x[u][e]);
                read_values<TI>(y, V, L::own, w, at);
                const int left = live - (t0 + 16 * w) - 2 * (lane & 3);  // of the sequence, from this lane's first token on
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[u][e] = 8 * u + (e & 1) < left ? y[u][e] - x[u][e] : 0.0f;  // Y^T
                if constexpr (kOut) {
                    add_up(far, os, w);
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int e = 0; e < 4; ++e) far[u][e] *= p.scale;
                    weigh_tokens<true>(far, vec + I::early / 4 + 16 * w);
                }
            }
            uint32_t own_f[TM][4];
            if (mine) {
                float y[2][4];
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[u][e] = -x[u][e];
                weigh_tokens<false>(y, vec + I::beta / 4 + 16 * w);
                as_operand<TM>(own_f, y[0], y[1]);
                put_factor(fs, w, own_f);
            }
            slice_sync(slice);
            if (mine) {  // E^T
                float d[NB][2][4] = {};
#pragma unroll
                for (int jj = 0; jj < NB; ++jj)
                    if (jj <= w) {
                        uint32_t a[TM][4], bf[1][TM][4];
                        if (jj == w) {
#pragma unroll
                            for (int u = 0; u < TM; ++u)
#pragma unroll
                                for (int e = 0; e < 4; ++e) a[u][e] = own_f[u][e];
                        } else {
                            get_factor(a, fs, jj);
                        }
#pragma unroll
                        for (int u = 0; u < TM; ++u) load4(bf[0][u], N + u * I::plane + in_block(B::by_columns(w, jj), at.b_row(), at.b_piece()));
                        products<kLevel>(d[jj], a, bf);
                    }
#pragma unroll
                for (int jj = 0; jj < NB; ++jj)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[0][e] += d[jj][0][e];
                        x[1][e] += d[jj][1][e];
                    }
                if constexpr (!kOut)
                    if (inside && ok) dump_errors<C, kSlabs>(x, p.errors + rows * C, w);
                weigh_tokens<false>(x, vec + I::beta / 4 + 16 * w);  // V'^T
                uint32_t a[TM][4];
                if constexpr (kOut) {
                    uint32_t a2[TO][4];
                    as_operand<TO>(a2, x[0], x[1]);
                    put_factor(os, w, a2);
                }
                weigh_tokens<false>(x, vec + I::late / 4 + 16 * w);
                as_operand<TM>(a, x[0], x[1]);
                put_factor(xs, w, a);
            }
            slice_sync(slice);
            const float whole = vec[I::whole / 4];
            {   // the update by itself, added once: the old state is rounded, not cut off
                float up[kTiles][4] = {};
#pragma unroll
                for (int jj = 0; jj < NB; ++jj) {
                    uint32_t a[TM][4];
                    get_factor(a, xs, jj);
#pragma unroll
                    for (int kp = 0; kp < kTiles / 2; ++kp) {
                        uint32_t bf[1][TI][4];
#pragma unroll
                        for (int u = 0; u < TI; ++u)
                            load4_t(bf[0][u], K + u * (KP * C * 2) + wide<C>(16 * jj + at.bt_row(), k0 / 8 + 2 * kp + at.bt_piece()));
                        sum<kRounded, kLevel>(up + 2 * kp, a, bf);
                    }
                }
#pragma unroll
                for (int j = 0; j < kTiles; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[j][e] = whole == 0.0f ? up[j][e] : fmaf(whole, s[j][e], up[j][e]);
            }
            if constexpr (kOut)
                if (mine) {
#pragma unroll
                    for (int jj = 0; jj < NB; ++jj)
                        if (jj <= w) {
                            uint32_t a[TO][4], bf[1][TP][4];
                            get_factor(a, os, jj);
#pragma unroll
                            for (int u = 0; u < TP; ++u) load4(bf[0][u], P + u * I::plane + in_block(I::p_block(w, jj), at.b_row(), at.b_piece()));
                            sum<kRounded, TO - 1>(far, a, bf);
                        }
                    if (ok) write_out<T>(far, p, b, h, v0, t0 + 16 * w, live);
                }
            ha::release_reads();
            __syncwarp();
            if (lane == 0 && ok) ha::bar_arrive(bars + 8 * (kEmpty + st));
        }
        if (kOut && inside) zero_out<T>(p, b, h, v0, count * C, w);
        if (ok && p.s_out && inside) write_state(s, p.s_out + (long long)bh * p.dk * p.dv, p.dk, p.dv, v0, k0);
    }
    __syncthreads();
    if (tid == 0 && *stop) give_up(p, gave_up, 1 + *stop);
}

// ------------------------------------------------------------------------------------------------- tensors for TMA

// [batch, tokens, heads, dim] tensors that TMA cannot load as they are (float32, odd sizes or strides) as bf16 terms,
// [term][batch][tokens][heads][width], columns from dim on zero: all of a call's in one launch, a row of the grid each.  A thread has
// eight columns of a row; `whole`: they are there, at addresses of 16 bytes.
struct Terms {
    static constexpr int kMost = 4;
    struct Tensor {
        ha::Rows from;
        __nv_bfloat16* to;
        long long pieces;
        uint32_t heads;
        int dim, width, whole;
    } tensors[kMost];
    uint32_t tokens;
    int count;
};
template <int TI, class T>
__global__ void __launch_bounds__(256) terms_kernel(const Terms p) {
    const Terms::Tensor& x = p.tensors[blockIdx.y];
    for (long long e = (long long)blockIdx.x * blockDim.x + threadIdx.x; e < x.pieces; e += (long long)gridDim.x * blockDim.x) {
        const uint32_t along = x.width / 8;
        const long long row = e / along, bt = row / x.heads;
        const int d = 8 * (int)(e - row * along);
        const T* const at = static_cast<const T*>(x.from.ptr) + bt / p.tokens * x.from.sb + bt % p.tokens * x.from.st + row % x.heads * x.from.sh + d;
        float f[8];
        if (sizeof(T) == 4 && x.whole) {
            const float4 a = reinterpret_cast<const float4*>(at)[0], b = reinterpret_cast<const float4*>(at)[1];
            f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = d + i < x.dim ? ha::to_f(at[i]) : 0.0f;
        }
        uint32_t t[4][TI];
#pragma unroll
        for (int i = 0; i < 4; ++i) ha::split<TI>(ha::make_pair2(f[2 * i], f[2 * i + 1]), t[i]);
#pragma unroll
        for (int u = 0; u < TI; ++u) reinterpret_cast<uint4*>(x.to)[u * x.pieces + e] = make_uint4(t[0][u], t[1][u], t[2][u], t[3][u]);
    }
}

}  // namespace hd
