// Gradients of the delta rule (formulas at the head of hd_scan.cuh).  Forward once more without the output, keeping the state
// before every chunk and E; back_kernel walks the chunks from the last, with D in registers as scan_kernel has S, and leaves dv, F,
// D after every chunk, and the sums over V that the gates' gradients need; grad_kernel then forms the rest of every chunk by itself:
//     Gd = dO V'^T,  Gz = Z V'^T,  Hd = scale D o Gd (i >= j),  Hz = D o Gz (i > j)
//     dQ = scale e^c dO S^T + Hd K,   dK = e^{c_C-c} V' D^T - e^c Z S^T + Hd^T Q - Hz K - Hz^T K
//     dlog a_t = sum_{i>=t>j} W_ij + sum_{i>=t} far_i + sum_{j<t} late_j + e^{c_C} <S, D>
//         W_ij = D_ij (scale q_i.k_j Gd_ij - k_i.k_j Gz_ij),  far_i = e^{c_i} (scale q_i^T S dO_i - k_i^T S Z_i),
//         late_j = e^{c_C-c_j} k_j^T D V'_j
// (`D_ij` with indices are the decays between tokens, D alone the gradient of the state).  The gradient of a log decay is the sum
// of all that passes over its token; every term of it has its own decay as a factor and none cancels another, so that it stays
// good where decays are strong and little passes at all.
#pragma once
#include "hd_scan.cuh"

namespace hd {

// Bound as scan_kernel is, by a chunk's chain: 3.4 us for a chunk and two slices (keys 128 wide); 24 pairs of nine chunks, keys 96 and
// values 64 wide: 26 us.
template <int KP, int C, int TI, int TM, class T>
__global__ void __launch_bounds__(kScanThreads, 1)
    back_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mg, const Params p,
                int* gave_up) {
    constexpr int TP = TM;
    using L = ScanLayout<KP, C, TI, TM, TP, true, true>;
    using I = typename L::I;
    using B = Blocks<C>;
    constexpr int kLevel = TM - 1, NB = C / 16, kTiles = KP / 32, kOwn = KP / 4;
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
        const uint32_t bytes = 2 * L::tile + own_slices * TI * L::own + L::image_bytes;
        if (warp == 4 * own_slices) load_chunks<C, L::kStages>(
            wait, sm8, stage_bytes, 2 * L::tile, own_slices * TI * L::own, count, live, p.tokens, bytes, p.mute,
            [&](int n, int s, uint32_t bar) {
                const uint32_t to = base + s * stage_bytes;
                bulk_load(to + L::image(own_slices), p.image + ((long long)bh * p.chunks + n) * I::end, L::image_bytes, bar);
                for (int u = 0; u < TI; ++u) {
                    for (int c = 0; c < KP / 64; ++c) {
                        ha::tma_load_4d(to + L::k + (u * (KP / 64) + c) * C * 128, &mk, 64 * c, h / p.kdiv, n * C, u * p.batch + b, bar);
                        ha::tma_load_4d(to + L::q + (u * (KP / 64) + c) * C * 128, &mq, 64 * c, h / p.qdiv, n * C, u * p.batch + b, bar);
                    }
                    for (int x = 0; x < own_slices; ++x)
                        ha::tma_load_4d(to + L::v + (x * TI + u) * L::own, &mg, 16 * (slice0 + x), h, n * C, u * p.batch + b, bar);
                }
            },
            true);
    } else {
        const Lane at;
        const int slice = warp >> 2, w = warp & 3, v0 = 16 * (slice0 + slice), k0 = w * kOwn, j0 = 2 * (lane & 3);
        uint8_t* const xs = sm8 + L::shared(own_slices) + slice * L::slice;  // partial sums of X, then factors of the update by K
        uint8_t* const os = xs + L::sums;                                    // factors of the update by Q
        uint8_t* const fs = os + L::sums;                                    // beta dV'
        const bool mine = w < NB, inside = v0 < p.dv;
        float s[kTiles][4];
        read_state(s, p.s_in ? p.s_in + (long long)bh * p.dk * p.dv : nullptr, p.dk, p.dv, v0, k0);
        bool ok = true;
        for (int it = 0; it < count; ++it) {
            const int st = it % L::kStages, n = count - 1 - it, t0 = n * C;
            const long long chunk = (long long)bh * p.chunks + n, rows = chunk * slices * 16 + v0;
            if (inside && ok) dump_state<KP, kSlabs>(s, p.gradients + rows * KP, k0);
            float e[2][4] = {};  // E^T
            if (mine && inside && ok) read_errors<C, kSlabs>(e, p.errors + rows * C, w);
            ok = __all_sync(~0u, ok && wait(kFull + st, it / L::kStages));
            const uint32_t to = base + st * stage_bytes, K = to + L::k, Q = to + L::q, G = to + L::v + slice * TI * L::own,
                           N = to + L::image(own_slices) + I::n, P = to + L::image(own_slices) + I::p;
            const float* const vec = reinterpret_cast<const float*>(sm8 + st * stage_bytes + L::image(own_slices));
            float x[2][4], near[2][4] = {};
            {
                float y[2 * NB][4] = {};
#pragma unroll
                for (int kk = 0; kk < kTiles / 2; ++kk) {  // this quarter's part of (K D)^T
                    uint32_t a[TM][4];
                    as_operand<TM>(a, s[2 * kk], s[2 * kk + 1]);
#pragma unroll
                    for (int np = 0; np < NB; np += 2) {
                        uint32_t bf[2][TI][4];
#pragma unroll
                        for (int g = 0; g < 2; ++g)
#pragma unroll
                            for (int u = 0; u < TI; ++u)
                                load4(bf[g][u], K + u * (KP * C * 2) + wide<C>(16 * (np + g) + at.b_row(), k0 / 8 + 2 * kk + at.b_piece()));
                        sum<kRounded, kLevel>(y + 2 * np, a, bf);
                    }
                }
                if (it > 0) slice_sync(slice);  // the factors of the update before have been read
                hand_out<NB>(y, x, xs, w);
            }
            if (mine) {
                // (P^T dO)^T of this warp's tokens
#pragma unroll
                for (int ii = 0; ii < NB; ++ii)
                    if (ii >= w) {
                        uint32_t a[TI][4], bf[1][TP][4];
#pragma unroll
                        for (int u = 0; u < TI; ++u) load4_t(a[u], G + u * L::own + place<32>(16 * ii + at.b_row(), at.b_piece()));
#pragma unroll
                        for (int u = 0; u < TP; ++u) load4_t(bf[0][u], P + u * I::plane + in_block(I::p_block(ii, w), at.bt_row(), at.bt_piece()));
                        sum<kRounded, kLevel>(near, a, bf);
                    }
                // scale e^c dO^T of this warp's tokens, a factor of the update
                float g[2][4];
                uint32_t a[TM][4];
                read_values<TI>(g, G, L::own, w, at);
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) g[u][r] *= p.scale;
                weigh_tokens<false>(g, vec + I::early / 4 + 16 * w);
                as_operand<TM>(a, g[0], g[1]);
                put_factor(os, w, a);
            }
            slice_sync(slice);
            // sums over the slice's columns for every token, to the lanes that have tokens 8 u + j0 of them
            float* const dots = p.dots + (chunk * 2 * p.parts + slice0 + slice) * C + 16 * w + j0;
            auto put = [&](float* where, int u, float y, float z) {
#pragma unroll
                for (int o = 4; o < 32; o *= 2) {
                    y += __shfl_xor_sync(~0u, y, o);
                    z += __shfl_xor_sync(~0u, z, o);
                }
                if (lane < 4 && inside && ok) *reinterpret_cast<float2*>(where + 8 * u) = make_float2(y, z);
            };
            uint32_t own_f[TM][4];
            if (mine) {
                add_up(x, xs, w);
                weigh_tokens<true>(x, vec + I::late / 4 + 16 * w);
                float y[2][4];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const float2 be = *reinterpret_cast<const float2*>(vec + I::beta / 4 + 16 * w + 8 * u + j0);
                    put(dots + p.parts * C, u, be.x * fmaf(x[u][0], e[u][0], x[u][2] * e[u][2]), be.y * fmaf(x[u][1], e[u][1], x[u][3] * e[u][3]));
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        x[u][r] += near[u][r];
                        y[u][r] = -(r & 1 ? be.y : be.x) * x[u][r];
                    }
                }
                as_operand<TM>(own_f, y[0], y[1]);
                put_factor(fs, w, own_f);
            }
            slice_sync(slice);
            if (mine) {  // F^T
                float d[NB][2][4] = {};
#pragma unroll
                for (int ii = 0; ii < NB; ++ii)
                    if (ii >= w) {
                        uint32_t a[TM][4], bf[1][TM][4];
                        if (ii == w) {
#pragma unroll
                            for (int u = 0; u < TM; ++u)
#pragma unroll
                                for (int r = 0; r < 4; ++r) a[u][r] = own_f[u][r];
                        } else {
                            get_factor(a, fs, ii);
                        }
#pragma unroll
                        for (int u = 0; u < TM; ++u) load4_t(bf[0][u], N + u * I::plane + in_block(B::by_columns(ii, w), at.bt_row(), at.bt_piece()));
                        products<kLevel>(d[ii], a, bf);
                    }
#pragma unroll
                for (int ii = 0; ii < NB; ++ii)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        x[0][r] += d[ii][0][r];
                        x[1][r] += d[ii][1][r];
                    }
                if (inside && ok) dump_errors<C, kSlabs>(x, p.errors_back + rows * C, w);
#pragma unroll
                for (int u = 0; u < 2; ++u) put(dots, u, fmaf(x[u][0], e[u][0], x[u][2] * e[u][2]), fmaf(x[u][1], e[u][1], x[u][3] * e[u][3]));
                weigh_tokens<false>(x, vec + I::beta / 4 + 16 * w);  // Z^T
                if (ok) write_out<T>(x, p, b, h, v0, t0 + 16 * w, live);
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[u][r] = -x[u][r];
                weigh_tokens<false>(x, vec + I::early / 4 + 16 * w);
                uint32_t a[TM][4];
                as_operand<TM>(a, x[0], x[1]);
                put_factor(xs, w, a);
            }
            slice_sync(slice);
            const float whole = vec[I::whole / 4];
            {
                float up[kTiles][4] = {};
#pragma unroll
                for (int part = 0; part < 2; ++part)  // - K^T (e^c Z); Q^T (scale e^c dO)
#pragma unroll
                    for (int jj = 0; jj < NB; ++jj) {
                        uint32_t a[TM][4];
                        get_factor(a, part ? os : xs, jj);
#pragma unroll
                        for (int kp = 0; kp < kTiles / 2; ++kp) {
                            uint32_t bf[1][TI][4];
#pragma unroll
                            for (int u = 0; u < TI; ++u)
                                load4_t(bf[0][u], (part ? Q : K) + u * (KP * C * 2) + wide<C>(16 * jj + at.bt_row(), k0 / 8 + 2 * kp + at.bt_piece()));
                            sum<kRounded, kLevel>(up + 2 * kp, a, bf);
                        }
                    }
#pragma unroll
                for (int j = 0; j < kTiles; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[j][r] = whole == 0.0f ? up[j][r] : fmaf(whole, s[j][r], up[j][r]);
            }
            ha::release_reads();
            __syncwarp();
            if (lane == 0 && ok) ha::bar_arrive(bars + 8 * (kEmpty + st));
        }
        if (inside) zero_out<T>(p, b, h, v0, count * C, w);
        if (ok && p.s_out && inside) write_state(s, p.s_out + (long long)bh * p.dk * p.dv, p.dk, p.dv, v0, k0);
    }
    __syncthreads();
    if (tid == 0 && *stop) give_up(p, gave_up, 1 + *stop);
}

// ------------------------------------------------------------------------------------------------------ every chunk by itself

constexpr int kGradThreads = 256;

// Terms of V', Z and S (TM), and of D and the H (TD, TH), which only the gradients of the tensors' own type depend on: 16 bits for those
// that are rounded to 8 themselves.
template <int KP, int C, int TI, int TM>
struct GradLayout {
    static constexpr int SL = TI == 1 ? 64 : 32;  // columns of V at a time
    static constexpr int TD = TI == 1 ? 2 : 3, TH = TD;
    static constexpr uint32_t tile = KP * C * 2 * TI, k = 0, q = tile;
    static constexpr uint32_t slab = 2 * tile, g = slab, own = C * 32, v = g + SL / 16 * TI * own, z = v + TM * SL * C * 2, s = z + TM * SL * C * 2,
                              d = s + TM * SL * KP * 2, slab_end = d + TD * SL * KP * 2;
    static constexpr uint32_t plane = C * C * 2, hd = slab, hz = hd + TH * plane, w = hz + TH * plane, h_end = w + C * (C + 1) * 4;
    static constexpr uint32_t vec = (slab_end > h_end ? slab_end : h_end), far = vec + 6 * C * 4 + 256, sums = far + 8 * C * 4, bars = sums + 64 * 4,
                              end = bars + 64;
};

// Columns c and c + 1 of a row of a gradient, of which `left` are left; float32 where the heads' rows are summed later.
template <class T>
__device__ __forceinline__ void put_pair(void* to, int each, long long at, int left, float x, float y) {
    if (each) {
        float* g = static_cast<float*>(to) + at;
        if (left > 0) g[0] = x;
        if (left > 1) g[1] = y;
    } else {
        T* g = static_cast<T*>(to) + at;
        if (left > 0) g[0] = ha::from_f<T>(x);
        if (left > 1) g[1] = ha::from_f<T>(y);
    }
}

// A chunk without a token of the sequence: zeros
template <int C, class T, int kThreads>
__device__ __forceinline__ void empty_chunk(const Params& p, long long row0, int t0, int chunk) {
    const int tid = threadIdx.x, pairs = (p.dk + 1) / 2;
    for (int e = tid; e < C * pairs; e += kThreads)
        if (t0 + e / pairs < p.tokens) {
            const int c = 2 * (e % pairs);
            const long long to = (row0 + (long long)(e / pairs) * p.heads) * p.dk + c;
            put_pair<T>(p.dq, p.each_q, to, p.dk - c, 0.0f, 0.0f);
            put_pair<T>(p.dk_out, p.each_k, to, p.dk - c, 0.0f, 0.0f);
        }
    if (tid < C && t0 + tid < p.tokens) {
        if (p.dlog_a) p.dlog_a[row0 + (long long)tid * p.heads] = 0.0f;
        if (p.dbeta) p.dbeta[row0 + (long long)tid * p.heads] = 0.0f;
    }
    if (tid == 0 && p.part) p.part[chunk] = 0.0;
}

// The gradients of beta and log a of a chunk.  `far`: kParts parts of far_i for each token, then room for C / 16 of as many; `sums`: the
// warps' parts of <S, D>; `wm`: W, C rows of C + 1.
template <int C, class I, int kParts>
__device__ __forceinline__ void gate_gradients(const Params& p, const float* vec, float* far, float* sums, float* wm, long long row0, int t0, int live, int slices) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const float* const dots = p.dots + (long long)blockIdx.x * 2 * slices * C;
    float db = 0.0f, dl = 0.0f;
    if (tid < C)
        for (int v = 0; v < slices; ++v) {
            db += dots[v * C + tid];
            dl += dots[(slices + v) * C + tid];
        }
    if (tid < C && p.dbeta && t0 + tid < p.tokens) p.dbeta[row0 + (long long)tid * p.heads] = t0 + tid < live ? db : 0.0f;
    if (!p.dlog_a && !p.part) return;
    __syncthreads();  // W is there
    // sum_{i>=t>j} W_ij: sums up each column by parts of 16 rows, then along the rows
    float* const tops = far + kParts * C;  // of each part and column (the rest of `far`)
    static_assert((kParts + C / 16) * C <= 8 * C, "scratch");
    for (int e = tid; e < C * (C / 16); e += kGradThreads) {
        const int j = e % C, part = e / C;
        float x = 0.0f;
#pragma unroll
        for (int i = 15; i >= 0; --i) {
            float& w = wm[(16 * part + i) * (C + 1) + j];
            x += 16 * part + i > j ? w : 0.0f;
            w = x;
        }
        tops[part * C + j] = x;
    }
    __syncthreads();
    float g = 0.0f;
    if (tid < 4 * C) {
        const int t = tid >> 2, quarter = tid & 3;  // a quarter of the columns before t
        for (int j = quarter; j < t; j += 4) {
            float x = wm[t * (C + 1) + j];
            for (int part = (t >> 4) + 1; part < C / 16; ++part) x += tops[part * C + j];
            g += x;
        }
        g += __shfl_xor_sync(~0u, g, 1);
        g += __shfl_xor_sync(~0u, g, 2);
    }
    __syncthreads();
    if (tid < 4 * C && (tid & 3) == 0) wm[tid >> 2] = g;
    if (tid < C) {
        float f = 0.0f;
#pragma unroll
        for (int c = 0; c < kParts; ++c) f += far[c * C + tid];
        wm[C + tid] = f;       // far
        wm[2 * C + tid] = dl;  // late
    }
    __syncthreads();
    if (tid < C) {
        float x = wm[tid], all = 0.0f;
        for (int i = C - 1; i >= tid; --i) x += wm[C + i];
        for (int j = 0; j < tid; ++j) x += wm[2 * C + j];
        for (int w = 0; w < kGradThreads / 32; ++w) all += sums[w];
        x += ha::decayed(vec[I::whole / 4], all);
        const bool on = t0 + tid < live;
        if (!on) x = 0.0f;
        if (p.dlog_a && t0 + tid < p.tokens) p.dlog_a[row0 + (long long)tid * p.heads] = x;
        if (p.part) {
            double total = x;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(~0u, total, o);
            if (lane == 0) reinterpret_cast<double*>(sums + 16)[warp] = total;
        }
    }
    if (p.part) {
        __syncthreads();
        if (tid == 0) {
            double total = 0.0;
            for (int w = 0; w < C / 32; ++w) total += reinterpret_cast<double*>(sums + 16)[w];
            p.part[blockIdx.x] = total;
        }
    }
}

// Rows of `width` floats in global memory as bf16 terms in shared memory; `weight` (for each column) or NULL.
template <int kTerms>
__device__ __forceinline__ void put_terms(uint8_t* to, uint32_t plane, const float4& f, uint32_t at) {
    uint32_t t0[kTerms], t1[kTerms];
    ha::split<kTerms>(ha::make_pair2(f.x, f.y), t0);
    ha::split<kTerms>(ha::make_pair2(f.z, f.w), t1);
#pragma unroll
    for (int u = 0; u < kTerms; ++u) *reinterpret_cast<uint2*>(to + u * plane + at) = make_uint2(t0[u], t1[u]);
}

template <int KP, int C, int TI, int TM, class T>
__global__ void __launch_bounds__(kGradThreads, 1)
    grad_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mg, const Params p,
                int* gave_up) {
    using L = GradLayout<KP, C, TI, TM>;
    using I = Image<C, TM, TM, true>;
    constexpr int kLevel = TM - 1, TD = L::TD, TH = L::TH, SL = L::SL;
    constexpr bool kRounded = TI == 3;
    constexpr int kRowBlocks = C / 16, kColumnBlocks = 8 / kRowBlocks, kCols = KP / kColumnBlocks, kPairs = kCols / 16;
    constexpr int kNear = C == 64 ? 2 : 1;  // pairs of a warp's part of the C x C products: of 64 columns half, of 32 sixteen (four warps)
    extern __shared__ __align__(1024) uint8_t sm8[];
    const uint32_t base = smem_addr(sm8), bars = base + L::bars;
    float* const vec = reinterpret_cast<float*>(sm8 + L::vec);
    float* const far = reinterpret_cast<float*>(sm8 + L::far);
    float* const sums = reinterpret_cast<float*>(sm8 + L::sums);
    volatile int* const stop = reinterpret_cast<int*>(sm8 + L::bars + 48);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rb = warp % kRowBlocks, cb = warp / kRowBlocks;
    const int n = blockIdx.x % p.chunks, bh = blockIdx.x / p.chunks, b = bh / p.heads, h = bh % p.heads;
    const int live = live_tokens(p.lengths, b, p.tokens), t0 = n * C, slices = (p.dv + 15) / 16;
    const long long row0 = ((long long)b * p.tokens + t0) * p.heads + h;  // of [batch, tokens, heads, ..]
    if (t0 >= live) {
        empty_chunk<C, T, kGradThreads>(p, row0, t0, blockIdx.x);
        return;
    }
    const Waiter wait{bars, stop, p.spin};
    if (tid == 0) {
        ha::bar_init(bars, 1);
        ha::bar_init(bars + 8, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *stop = 0;
        ha::fence_smem_to_async();
        if (n != p.mute) {
            ha::bar_expect(bars, 2 * L::tile);
            for (int u = 0; u < TI; ++u)
                for (int c = 0; c < KP / 64; ++c) {
                    ha::tma_load_4d(base + L::k + (u * (KP / 64) + c) * C * 128, &mk, 64 * c, h / p.kdiv, t0, u * p.batch + b, bars);
                    ha::tma_load_4d(base + L::q + (u * (KP / 64) + c) * C * 128, &mq, 64 * c, h / p.qdiv, t0, u * p.batch + b, bars);
                }
        }
    }
    const float* const image = reinterpret_cast<const float*>(p.image + (long long)blockIdx.x * I::end);
    for (int e = tid; e < (int)I::n / 4; e += kGradThreads) vec[e] = image[e];
    __syncthreads();
    bool ok = wait(0, 0);
    ok = __syncthreads_and(ok);
    if (!ok) {
        wait.drain(0, 0);
        if (tid == 0) give_up(p, gave_up, 100);
        return;
    }
    if (t0 + C > live) {  // tokens behind the end: 0 * NaN must not reach a sum
        const int rows = t0 + C - live;
        for (uint32_t block = 0; block < 2 * L::tile; block += C * 128)
            for (int e = tid; e < rows * 8; e += kGradThreads) *reinterpret_cast<uint4*>(sm8 + block + (live - t0) * 128 + e * 16) = make_uint4(0, 0, 0, 0);
    }
    const Lane at;
    const int i0 = 16 * rb + (lane >> 2), j0 = 2 * (lane & 3);
    const bool near = cb < C / (16 * kNear);
    float fq[2 * kPairs][4] = {}, fz[2 * kPairs][4] = {}, fl[2 * kPairs][4] = {}, gd[2 * kNear][4] = {}, gz[2 * kNear][4] = {};
    float cross = 0.0f;
    const float* const beta = vec + I::beta / 4;
    int turn = 0;
    for (int v0 = 0; v0 < p.dv; v0 += SL, ++turn) {
        const int rows = min(SL, 16 * slices - v0);  // of the dumps
        if (turn) __syncthreads();                   // the slab before has been read
        if (tid == 0) {
            ha::fence_smem_to_async();
            ha::bar_expect(bars + 8, SL / 16 * TI * L::own);
            for (int u = 0; u < TI; ++u)
                for (int c = 0; c < SL / 16; ++c)
                    ha::tma_load_4d(base + L::g + (u * (SL / 16) + c) * L::own, &mg, v0 + 16 * c, h, t0, u * p.batch + b, bars + 8);
        }
        const long long at0 = (long long)blockIdx.x * slices * 16 + v0;
        const float4 zero = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
        for (int e = tid; e < SL * C / 4; e += kGradThreads) {
            const int r = e / (C / 4), c = 4 * (e % (C / 4));
            const float4 w = *reinterpret_cast<const float4*>(beta + c);
            float4 x = r < rows ? *reinterpret_cast<const float4*>(p.errors + (at0 + r) * C + c) : zero;
            float4 y = r < rows ? *reinterpret_cast<const float4*>(p.errors_back + (at0 + r) * C + c) : zero;
            x = make_float4(w.x * x.x, w.y * x.y, w.z * x.z, w.w * x.w);
            y = make_float4(w.x * y.x, w.y * y.y, w.z * y.z, w.w * y.w);
            const uint32_t to = place<2 * C>(r, c >> 3) + 2 * (c & 7);
            put_terms<TM>(sm8 + L::v, SL * C * 2, x, to);
            put_terms<TM>(sm8 + L::z, SL * C * 2, y, to);
        }
#pragma unroll 4
        for (int e = tid; e < SL * KP / 4; e += kGradThreads) {
            const int r = e / (KP / 4), c = 4 * (e % (KP / 4));
            const float4 x = r < rows ? *reinterpret_cast<const float4*>(p.states + (at0 + r) * KP + c) : zero;
            const float4 y = r < rows ? *reinterpret_cast<const float4*>(p.gradients + (at0 + r) * KP + c) : zero;
            cross = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, cross))));
            const uint32_t to = wide<SL>(r, c >> 3) + 2 * (c & 7);
            put_terms<TM>(sm8 + L::s, SL * KP * 2, x, to);
            put_terms<TD>(sm8 + L::d, SL * KP * 2, y, to);
        }
        ok = wait(1, turn);
        ok = __syncthreads_and(ok);
        if (!ok) {
            wait.drain(1, turn);
            if (tid == 0) give_up(p, gave_up, 101);
            return;
        }
#pragma unroll 1
        for (int kk = 0; kk < SL / 16; ++kk) {
            uint32_t ag[TI][4], az[TM][4], av[TM][4];
#pragma unroll
            for (int u = 0; u < TI; ++u) load4(ag[u], base + L::g + (u * (SL / 16) + kk) * L::own + place<32>(16 * rb + at.a_row(), at.a_piece()));
#pragma unroll
            for (int u = 0; u < TM; ++u) {
                load4_t(az[u], base + L::z + u * (SL * C * 2) + place<2 * C>(16 * kk + at.at_row(), 2 * rb + at.at_piece()));
                load4_t(av[u], base + L::v + u * (SL * C * 2) + place<2 * C>(16 * kk + at.at_row(), 2 * rb + at.at_piece()));
            }
#pragma unroll
            for (int np = 0; np < kPairs; ++np) {
                uint32_t bs[1][TM][4], bd[1][TD][4];
#pragma unroll
                for (int u = 0; u < TM; ++u)
                    load4_t(bs[0][u], base + L::s + u * (SL * KP * 2) + wide<SL>(16 * kk + at.bt_row(), cb * (kCols / 8) + 2 * np + at.bt_piece()));
#pragma unroll
                for (int u = 0; u < TD; ++u)
                    load4_t(bd[0][u], base + L::d + u * (SL * KP * 2) + wide<SL>(16 * kk + at.bt_row(), cb * (kCols / 8) + 2 * np + at.bt_piece()));
                sum<kRounded, kLevel>(fq + 2 * np, ag, bs);
                sum<kRounded, kLevel>(fz + 2 * np, az, bs);
                sum<kRounded, TI == 1 ? 1 : kLevel>(fl + 2 * np, av, bd);
            }
            if (near) {
#pragma unroll
                for (int np = 0; np < kNear; ++np) {
                    const int c = kNear * cb + np;
                    if (c <= rb) {
                        uint32_t bv[1][TM][4];
#pragma unroll
                        for (int u = 0; u < TM; ++u)
                            load4_t(bv[0][u], base + L::v + u * (SL * C * 2) + place<2 * C>(16 * kk + at.bt_row(), 2 * c + at.bt_piece()));
                        sum<kRounded, kLevel>(gd + 2 * np, ag, bv);
                        sum<kRounded, kLevel>(gz + 2 * np, az, bv);
                    }
                }
            }
        }
    }
    // far_i; dq and dk as far as they are
    const float* const early = vec + I::early / 4;
    const float* const late = vec + I::late / 4;
    {
        float f[2] = {};
#pragma unroll
        for (int nt = 0; nt < 2 * kPairs; ++nt)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int i = i0 + 8 * r, piece = cb * (kCols / 8) + nt;
                float q0 = 0.0f, q1 = 0.0f, k0 = 0.0f, k1 = 0.0f;
#pragma unroll
                for (int u = TI - 1; u >= 0; --u) {
                    const uint32_t qq = *reinterpret_cast<const uint32_t*>(sm8 + L::q + u * (KP * C * 2) + wide<C>(i, piece) + 2 * j0);
                    const uint32_t kk = *reinterpret_cast<const uint32_t*>(sm8 + L::k + u * (KP * C * 2) + wide<C>(i, piece) + 2 * j0);
                    q0 += __uint_as_float(qq << 16); q1 += __uint_as_float(qq & 0xffff0000u);
                    k0 += __uint_as_float(kk << 16); k1 += __uint_as_float(kk & 0xffff0000u);
                }
                const float ea = early[i], la = late[i];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float x = ha::decayed(ea, p.scale * fq[nt][2 * r + e]), y = ha::decayed(ea, fz[nt][2 * r + e]);
                    f[r] += fmaf(e ? q1 : q0, x, -(e ? k1 : k0) * y);
                    fq[nt][2 * r + e] = x;
                    fz[nt][2 * r + e] = ha::decayed(la, fl[nt][2 * r + e]) - y;
                }
            }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            f[r] += __shfl_xor_sync(~0u, f[r], 1);
            f[r] += __shfl_xor_sync(~0u, f[r], 2);
            if ((lane & 3) == 0) far[cb * C + i0 + 8 * r] = t0 + i0 + 8 * r < live ? f[r] : 0.0f;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) cross += __shfl_xor_sync(~0u, cross, o);
    if (lane == 0) sums[warp] = cross;
    // the weights between tokens
    float kk2[2 * kNear][4] = {}, qk2[2 * kNear][4] = {};
    if (near) {
#pragma unroll 2
        for (int kk = 0; kk < KP / 16; ++kk) {
            uint32_t ak[TI][4], aq[TI][4];
#pragma unroll
            for (int u = 0; u < TI; ++u) {
                load4(ak[u], base + L::k + u * (KP * C * 2) + wide<C>(16 * rb + at.a_row(), 2 * kk + at.a_piece()));
                load4(aq[u], base + L::q + u * (KP * C * 2) + wide<C>(16 * rb + at.a_row(), 2 * kk + at.a_piece()));
            }
#pragma unroll
            for (int np = 0; np < kNear; ++np)
                if (kNear * cb + np <= rb) {
                    uint32_t bk[1][TI][4];
#pragma unroll
                    for (int u = 0; u < TI; ++u)
                        load4(bk[0][u], base + L::k + u * (KP * C * 2) + wide<C>(16 * (kNear * cb + np) + at.b_row(), 2 * kk + at.b_piece()));
                    sum<kRounded, TI - 1>(kk2 + 2 * np, ak, bk);
                    sum<kRounded, TI - 1>(qk2 + 2 * np, aq, bk);
                }
        }
    }
    __syncthreads();  // the slab has been read
    float* const wm = reinterpret_cast<float*>(sm8 + L::w);
    if (near) {
        const float* const hi = vec + I::hi / 4;
        const float* const lo = vec + I::lo / 4;
#pragma unroll
        for (int nt = 0; nt < 2 * kNear; ++nt)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int i = i0 + 8 * r, j = 16 * kNear * cb + 8 * nt + j0;
                const float hi_i = hi[i], lo_i = lo[i];
                float x[2], y[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float d = j + e <= i && t0 + i < live ? ex2((hi_i - hi[j + e]) + (lo_i - lo[j + e])) : 0.0f;
                    x[e] = d != 0.0f ? p.scale * d * gd[nt][2 * r + e] : 0.0f;
                    y[e] = j + e < i && d != 0.0f ? -d * gz[nt][2 * r + e] : 0.0f;
                    wm[i * (C + 1) + j + e] = j + e < i && d != 0.0f ? fmaf(qk2[nt][2 * r + e], x[e], kk2[nt][2 * r + e] * y[e]) : 0.0f;
                }
                uint32_t t[TH];
                ha::split<TH>(ha::make_pair2(x[0], x[1]), t);
#pragma unroll
                for (int u = 0; u < TH; ++u) *reinterpret_cast<uint32_t*>(sm8 + L::hd + u * L::plane + place<2 * C>(i, j >> 3) + 2 * (j & 7)) = t[u];
                ha::split<TH>(ha::make_pair2(y[0], y[1]), t);
#pragma unroll
                for (int u = 0; u < TH; ++u) *reinterpret_cast<uint32_t*>(sm8 + L::hz + u * L::plane + place<2 * C>(i, j >> 3) + 2 * (j & 7)) = t[u];
            }
    }
    __syncthreads();
#pragma unroll
    for (int jj = 0; jj < kRowBlocks; ++jj) {
        uint32_t a[TH][4], b2[TH][4];
        if (jj <= rb) {  // Hd K, - Hz K
#pragma unroll
            for (int u = 0; u < TH; ++u) {
                load4(a[u], base + L::hd + u * L::plane + place<2 * C>(16 * rb + at.a_row(), 2 * jj + at.a_piece()));
                load4(b2[u], base + L::hz + u * L::plane + place<2 * C>(16 * rb + at.a_row(), 2 * jj + at.a_piece()));
            }
#pragma unroll
            for (int np = 0; np < kPairs; ++np) {
                uint32_t bk[1][TI][4];
#pragma unroll
                for (int u = 0; u < TI; ++u)
                    load4_t(bk[0][u], base + L::k + u * (KP * C * 2) + wide<C>(16 * jj + at.bt_row(), cb * (kCols / 8) + 2 * np + at.bt_piece()));
                sum<kRounded, TH - 1>(fq + 2 * np, a, bk);
                sum<kRounded, TH - 1>(fz + 2 * np, b2, bk);
            }
        }
        if (jj >= rb) {  // Hd^T Q, - Hz^T K
#pragma unroll
            for (int u = 0; u < TH; ++u) {
                load4_t(a[u], base + L::hd + u * L::plane + place<2 * C>(16 * jj + at.at_row(), 2 * rb + at.at_piece()));
                load4_t(b2[u], base + L::hz + u * L::plane + place<2 * C>(16 * jj + at.at_row(), 2 * rb + at.at_piece()));
            }
#pragma unroll
            for (int np = 0; np < kPairs; ++np) {
                uint32_t bk[1][TI][4], bq[1][TI][4];
#pragma unroll
                for (int u = 0; u < TI; ++u) {
                    load4_t(bk[0][u], base + L::k + u * (KP * C * 2) + wide<C>(16 * jj + at.bt_row(), cb * (kCols / 8) + 2 * np + at.bt_piece()));
                    load4_t(bq[0][u], base + L::q + u * (KP * C * 2) + wide<C>(16 * jj + at.bt_row(), cb * (kCols / 8) + 2 * np + at.bt_piece()));
                }
                sum<kRounded, TH - 1>(fz + 2 * np, a, bq);
                sum<kRounded, TH - 1>(fz + 2 * np, b2, bk);
            }
        }
    }
#pragma unroll
    for (int nt = 0; nt < 2 * kPairs; ++nt)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int i = i0 + 8 * r, c = cb * kCols + 8 * nt + j0;
            if (t0 + i >= p.tokens) continue;
            const long long to = (row0 + (long long)i * p.heads) * p.dk + c;
            const bool on = t0 + i < live;
            put_pair<T>(p.dq, p.each_q, to, p.dk - c, on ? fq[nt][2 * r] : 0.0f, on ? fq[nt][2 * r + 1] : 0.0f);
            put_pair<T>(p.dk_out, p.each_k, to, p.dk - c, on ? fz[nt][2 * r] : 0.0f, on ? fz[nt][2 * r + 1] : 0.0f);
        }
    gate_gradients<C, I, kColumnBlocks>(p, vec, far, sums, wm, row0, t0, live, slices);
}

// dlog_a[h]: the sum of the chunks' parts over the batch, in 64 bits and in a fixed order; a warp for each head.
__global__ void __launch_bounds__(32) part_sum_kernel(const double* part, int batch, int heads, int chunks, float* dlog_a) {
    const int h = blockIdx.x, lane = threadIdx.x;
    double s = 0.0;
    for (int b = 0; b < batch; ++b)
        for (int n = lane; n < chunks; n += 32) s += part[((long long)b * heads + h) * chunks + n];
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    if (lane == 0) dlog_a[h] = (float)s;
}

// [batch, tokens, heads, dim] float32, a row for each head, summed over the `each` heads that share one; one or two tensors, a row of the
// grid each.  A thread has a unit of four columns (`whole`: dim and the result's address allow it), or of one.
struct Sums {
    struct Tensor {
        const float* from;
        void* to;
        long long units;
        int each, dim, whole;
    } tensors[2];
    int count;
};
template <class T>
__global__ void __launch_bounds__(256) shared_sum_kernel(const Sums p) {
    const Sums::Tensor& x = p.tensors[blockIdx.y];
    const uint32_t along = x.whole ? x.dim / 4 : x.dim;
    for (long long e = (long long)blockIdx.x * blockDim.x + threadIdx.x; e < x.units; e += (long long)gridDim.x * blockDim.x) {
        const long long row = e >> 32 ? e / along : (uint32_t)e / along;
        const float* const from = x.from + row * x.each * x.dim;
        const int d = (int)(e - row * along);
        if (x.whole) {
            float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
            for (int i = 0; i < x.each; ++i) {
                const float4 f = *reinterpret_cast<const float4*>(from + (long long)i * x.dim + 4 * d);
                s.x += f.x; s.y += f.y; s.z += f.z; s.w += f.w;
            }
            if constexpr (sizeof(T) == 2) static_cast<uint2*>(x.to)[e] = make_uint2(ha::pack_bf16(s.x, s.y), ha::pack_bf16(s.z, s.w));
            else static_cast<float4*>(x.to)[e] = s;
        } else {
            float s = 0.0f;
            for (int i = 0; i < x.each; ++i) s += from[(long long)i * x.dim + d];
            static_cast<T*>(x.to)[e] = ha::from_f<T>(s);
        }
    }
}

}  // namespace hd
