// grad_kernel (hd_grad.cuh) on tcgen05: bf16, keys up to 128 wide, chunks of 64 tokens.
//
// Rows are stacked to fill the tensor core: 0..63 belong to the queries, 64..127 to the keys.
//     A = [dO; Z] S       (128 x KP, sixteen columns of V a step)      its rows then times scale e^c, and -e^c
//     G = [dO; Z] V'^T    (128 x 64)
//     L = [ . ; V'] D^T   (128 x KP, the upper half unused)
//     R = [Q; K] K^T      (128 x 64)
//     A += [Hd; -Hz] K + [0; Hd^T] Q + [0; -Hz^T] K       dQ = A above, dK = A + e^{c_C-c} L below
// V', Z and S enter as three bf16 terms (24 bits: dlog a hangs on them), formed from the float32 dumps while the tensor core works on
// the sixteen columns before; dO is exact, its lower terms zero.  A CTA stays and takes chunk after chunk; one warp loads ahead, one
// issues the products, the others have a row of a product and a quarter of its columns each.
//
// 4096 chunks, keys and values 128 wide: 392 us, 1.1 GB read and 0.14 GB written (HBM alone: 190 us).  A chunk's 27000 clocks are eight
// steps over V (1200 to 1500 each, bound by the products of three terms) and what follows them, which waits for the last one and which
// the next chunk's steps wait for: far_i, H and W, the last products, the gates' sums, dq and dk (10000).  D and H enter the products for
// dq and dk with two terms (16 bits), since those are rounded to 8.
#pragma once
#include "hd_grad.cuh"
#include "hd_scan_mma.cuh"

namespace hd {

constexpr int kGradMmaThreads = 576;  // sixteen warps that compute, one that loads, one that issues the products
constexpr int kTeam = 512;

// The team's barrier; true where all of its threads say so.
__device__ __forceinline__ bool team_sync(bool mine) {
    uint32_t all;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbarrier.cta.red.and.pred p, 1, 512, q;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(all) : "r"((uint32_t)mine) : "memory");
    return all != 0;
}

template <int KP> struct GradMmaLayout {
    static constexpr int C = 64, kTiles = 2, kRaw = 3;
    using I = Image<C, 3, 3, true>;
    static constexpr uint32_t block = 2 * C * 128, tiles_bytes = KP / 64 * block;  // blocks of 64 columns: rows of Q, then of K
    // two operand buffers, of sixteen columns of V each: three terms of [dO; Z] (the lower terms of dO zero), of V', of S; two of D
    static constexpr uint32_t ops = kTiles * tiles_bytes;
    static constexpr uint32_t az = 0, az_term = 2 * C * 32, v = 3 * az_term, v_term = C * 32, s = v + 3 * v_term, s_term = 16 * KP * 2, d = s + 3 * s_term,
                              op = (d + 2 * s_term + 1023) / 1024 * 1024;
    // what arrives for them: S, D (16 x KP), E^T, F^T (16 x C) in float32, dO
    static constexpr uint32_t raw = ops + 2 * op, raw_d = 16 * KP * 4, raw_e = 2 * raw_d, raw_f = raw_e + 16 * C * 4, raw_g = raw_f + 16 * C * 4,
                              raw_bytes = raw_g + C * 32;
    // in the operand buffers once they are done with: zeros, [Hd; -Hz] in two terms, W; then dq and dk on their way out
    static constexpr uint32_t zero = ops, h = zero + C * 128, h_term = 2 * C * 128, w = h + 2 * h_term, w_end = w + C * (C + 1) * 4;
    static constexpr uint32_t out = ops + op;
    static constexpr uint32_t raw_at = raw > (w_end + 1023) / 1024 * 1024 ? raw : (w_end + 1023) / 1024 * 1024;
    static constexpr uint32_t vec = raw_at + kRaw * raw_bytes, far = vec + kTiles * I::n, sums = far + 16 * C * 4, bars = sums + 256, end = bars + 192;
    static constexpr uint32_t ta = 0, tl = KP, tg = 2 * KP, tr = 2 * KP + C, columns = 512;
    static_assert(tr + C <= columns && s % 1024 == 0 && s_term % 1024 == 0 && raw_bytes % 1024 == 0 && I::n % 256 == 0, "layout");
    static_assert(out + KP / 64 * 2 * C * 128 <= raw_at, "the way out");
};

template <int KP, class T>
__global__ void __launch_bounds__(kGradMmaThreads, 1)
    grad_mma_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mg,
                    const __grid_constant__ CUtensorMap mdq, const __grid_constant__ CUtensorMap mdk, const Params p, int total, int* gave_up) {
    using L = GradMmaLayout<KP>;
    using I = typename L::I;
    constexpr int C = 64, TM = 3;
    enum : int { kFullTiles = 0, kFreeTiles = 2, kFullRaw = 4, kFreeRaw = 7, kDone = 10, kReady = 12, kStep = 14, kNear, kOutFree, kAll };
    extern __shared__ __align__(1024) uint8_t sm8[];
    const uint32_t base = smem_addr(sm8), bars = base + L::bars;
    float* const far = reinterpret_cast<float*>(sm8 + L::far);
    float* const sums = reinterpret_cast<float*>(sm8 + L::sums);
    volatile int* const stop = reinterpret_cast<int*>(sm8 + L::bars + 160);
    uint32_t* const s_tmem = reinterpret_cast<uint32_t*>(sm8 + L::bars + 168);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, slices = (p.dv + 15) / 16;
    const Waiter wait{bars, stop, p.spin};
    if (tid == 0) {
        for (int i = 0; i < kAll; ++i) ha::bar_init(bars + 8 * i, (i >= kFreeRaw && i < kDone) || i == kReady || i == kReady + 1 || i == kNear ? 16 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *stop = 0;
    }
    if (warp == 0) {
        __syncwarp();
        ha::tmem_alloc(smem_addr(s_tmem), L::columns);
    }
    ha::tmem_before_sync();
    __syncthreads();
    ha::tmem_after_sync();
    if (tid == 0 && *s_tmem != 0) *stop = 1 + kAll;  // all columns were asked for: they start at 0
    struct Chunk {
        int n, b, h, live, t0;
    };
    auto chunk_at = [&](int at) {
        Chunk c;
        c.n = at % p.chunks;
        const int bh = at / p.chunks;
        c.b = bh / p.heads;
        c.h = bh % p.heads;
        c.live = live_tokens(p.lengths, c.b, p.tokens);
        c.t0 = c.n * C;
        return c;
    };
    if (warp == 16) {
        // ---------------------------------------------------------------------------------------------- loads
        if (lane == 0) {
            bool ok = true;
            int tiles = 0, raws = 0;
            for (int at = blockIdx.x; at < total && ok; at += gridDim.x) {
                const Chunk c = chunk_at(at);
                if (c.t0 >= c.live) continue;
                if (c.n == p.mute) break;
                const int ts = tiles % L::kTiles;
                if (tiles >= L::kTiles) ok = wait(kFreeTiles + ts, tiles / L::kTiles - 1);
                if (!ok) break;
                const uint32_t full = bars + 8 * (kFullTiles + ts), to = base + ts * L::tiles_bytes;
                ha::bar_expect(full, L::tiles_bytes + I::n);
                bulk_load(base + L::vec + ts * I::n, p.image + (long long)at * I::end, I::n, full);
                for (int x = 0; x < KP / 64; ++x) {
                    ha::tma_load_4d(to + x * L::block, &mq, 64 * x, c.h / p.qdiv, c.t0, c.b, full);
                    ha::tma_load_4d(to + x * L::block + C * 128, &mk, 64 * x, c.h / p.kdiv, c.t0, c.b, full);
                }
                ++tiles;
                for (int slab = 0; slab < slices && ok; ++slab, ++raws) {
                    const int rs = raws % L::kRaw;
                    if (raws >= L::kRaw) ok = wait(kFreeRaw + rs, raws / L::kRaw - 1);
                    if (!ok) break;
                    const uint32_t bar = bars + 8 * (kFullRaw + rs), raw = base + L::raw_at + rs * L::raw_bytes;
                    const long long row = ((long long)at * slices + slab) * 16;
                    ha::bar_expect(bar, L::raw_bytes);
                    bulk_load(raw, p.states + row * KP, L::raw_d, bar);
                    bulk_load(raw + L::raw_d, p.gradients + row * KP, L::raw_d, bar);
                    bulk_load(raw + L::raw_e, p.errors + row * C, 16 * C * 4, bar);
                    bulk_load(raw + L::raw_f, p.errors_back + row * C, 16 * C * 4, bar);
                    ha::tma_load_4d(raw + L::raw_g, &mg, 16 * slab, c.h, c.t0, c.b, bar);
                }
            }
            for (int i = max(0, tiles - L::kTiles); i < tiles; ++i) wait.drain(kFullTiles + i % L::kTiles, i / L::kTiles);
            for (int i = max(0, raws - L::kRaw); i < raws; ++i) wait.drain(kFullRaw + i % L::kRaw, i / L::kRaw);
        }
        __syncwarp();
    } else if (warp == 17) {
        // ---------------------------------------------------------------------------------------------- products
        if (ha::elect_one()) {
            constexpr uint32_t wide_shape = ha::mma_shape(KP, ha::kColMajorB), near_shape = ha::mma_shape(C, 0);
            constexpr uint32_t late_shape = ha::mma_shape(KP, ha::kColMajorA | ha::kColMajorB);
            bool ok = true;
            int tiles = 0, ready[2] = {0, 0};
            for (int at = blockIdx.x; at < total && ok; at += gridDim.x) {
                const Chunk c = chunk_at(at);
                if (c.t0 >= c.live) continue;
                const int ts = tiles % L::kTiles;
                for (int slab = 0; slab < slices && ok; ++slab) {
                    const int buf = slab & 1;
                    ok = wait(kReady + buf, ready[buf]);  // (the team has waited for what arrived)
                    if (!ok) break;
                    ready[buf] += 1;
                    const uint32_t from = base + L::ops + buf * L::op;
                    ha::tmem_after_sync();
                    const uint32_t az = ha::operand(from + L::az, 0), vo = ha::operand(from + L::v, 0), so = ha::operand(from + L::s, 2048),
                                   dd = ha::operand(from + L::d, 2048);
#pragma unroll
                    for (int level = TM - 1; level >= 0; --level)
#pragma unroll
                        for (int u = 0; u <= level; ++u) {
                            const bool more = slab > 0 || level < TM - 1 || u > 0;
                            mma_tile<kRows32, ha::kSwizzled>(L::ta, az + u * (L::az_term >> 4), so + (level - u) * (L::s_term >> 4), wide_shape, more);
                            mma_tile<kRows32, kRows32>(L::tg, az + u * (L::az_term >> 4), vo + (level - u) * (L::v_term >> 4), near_shape, more);
                        }
#pragma unroll
                    for (int level = 1; level >= 0; --level)  // rows 64..127 are V' (above them is what lies before it: those sums are not used)
#pragma unroll
                        for (int u = level; u >= 0; --u)
                            mma_tile<kRows32, ha::kSwizzled>(L::tl, vo + u * (L::v_term >> 4) - (C * 32 >> 4), dd + (level - u) * (L::s_term >> 4), wide_shape,
                                                             slab > 0 || level == 0 || u == 0);
                    if (slab == 0) {
                        const uint32_t rows = ha::operand(base + ts * L::tiles_bytes, 0);
#pragma unroll
                        for (int kk = 0; kk < KP / 16; ++kk) {
                            const uint32_t step = (kk >> 2) * (L::block >> 4) + (kk & 3) * 2;
                            mma_tile<ha::kSwizzled, ha::kSwizzled>(L::tr, rows + step, rows + step + (C * 128 >> 4), near_shape, kk > 0);
                        }
                    }
                    ha::mma_commit(bars + 8 * (kDone + buf));
                }
                if (!ok || !(ok = wait(kNear, tiles))) break;
                ha::tmem_after_sync();
                const uint32_t q = ha::operand(base + ts * L::tiles_bytes, L::block), k = ha::operand(base + ts * L::tiles_bytes + C * 128, L::block);
#pragma unroll
                for (int u = 1; u >= 0; --u)
#pragma unroll
                    for (int kk = 0; kk < C / 16; ++kk) {
                        mma_tile<ha::kSwizzled, ha::kSwizzled>(L::ta, ha::operand(base + L::h + u * L::h_term, 0) + kk * 2, k + kk * 128, wide_shape, true);
                        // [0; H^T]: from the zeros the second 64 rows lie as far as H does
                        mma_tile<ha::kSwizzled, ha::kSwizzled>(L::ta, ha::operand(base + L::zero, L::h - L::zero + u * L::h_term) + kk * 128, q + kk * 128, late_shape, true);
                        mma_tile<ha::kSwizzled, ha::kSwizzled>(L::ta, ha::operand(base + L::zero, L::h - L::zero + u * L::h_term + C * 128) + kk * 128, k + kk * 128, late_shape, true);
                    }
                ha::mma_commit(bars + 8 * kStep);
                ++tiles;
            }
            // what was issued may still run
            for (int buf = 0; buf < 2; ++buf)
                if (ready[buf]) wait.drain(kDone + buf, ready[buf] - 1);
            if (tiles) wait.drain(kStep, tiles - 1);
        }
        __syncwarp();
    } else {
        bool ok = true;
        int tiles = 0, used = 0, issued[2] = {0, 0};  // chunks with tokens, slabs, slabs of each buffer so far
        const int quarter = warp >> 2, row = (warp & 3) * 32 + lane, i = row & (C - 1);  // a row of the products, a quarter of their columns
        const bool key = row >= C;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        for (int at = blockIdx.x; at < total; at += gridDim.x) {
            const Chunk c = chunk_at(at);
            const long long row0 = ((long long)c.b * p.tokens + c.t0) * p.heads + c.h;  // of [batch, tokens, heads, ..]
            if (c.t0 >= c.live) {
                empty_chunk<C, T, kTeam>(p, row0, c.t0, at);
                continue;
            }
            const int ts = tiles % L::kTiles;
            const float* const vec = reinterpret_cast<const float*>(sm8 + L::vec + ts * I::n);
            uint8_t* const kq = sm8 + ts * L::tiles_bytes;
            ok = ok && wait(kFullTiles + ts, tiles / L::kTiles);
            ++tiles;
            if (ok && c.t0 + C > c.live) {  // tokens behind the end: 0 * NaN must not reach a sum
                const int rows = c.t0 + C - c.live;
                for (uint32_t block = 0; block < L::tiles_bytes; block += C * 128)
                    for (int e = tid; e < rows * 8; e += kTeam) *reinterpret_cast<uint4*>(kq + block + (c.live - c.t0) * 128 + e * 16) = make_uint4(0, 0, 0, 0);
            }
            // for the first 2 C threads: the slices' parts of dbeta, and of what crosses into later chunks
            const float* const dots = p.dots + (long long)at * 2 * p.parts * C + (tid >> 6) * (p.parts * C) + (tid & 63);
            float part[8], cross = 0.0f;
            for (int slab = 0; slab < slices; ++slab, ++used) {
                const int buf = slab & 1, rs = used % L::kRaw;
                uint8_t* const to = sm8 + L::ops + buf * L::op;
                const uint8_t* const raw = sm8 + L::raw_at + rs * L::raw_bytes;
                // (the buffers held other things since the chunk before: its last products are done)
                if (slab >= 2) ok = ok && wait(kDone + buf, issued[buf] - 1);
                if (slab == 1 && tiles > 1) ok = ok && wait(kOutFree, tiles - 2);  // what the chunk before sent from there has left
                ok = ok && wait(kFullRaw + rs, used / L::kRaw);
                if (ok) {
                    const int token = (tid >> 2) & 63, quad = tid & 3;
                    const uint32_t piece = place<32>(token, quad >> 1) + 8 * (quad & 1);
                    const float be = vec[I::beta / 4 + token];
                    const float4 f4 = *reinterpret_cast<const float4*>(raw + (tid < 256 ? L::raw_f : L::raw_e) + token * 64 + quad * 16);
                    const float4 x = make_float4(be * f4.x, be * f4.y, be * f4.z, be * f4.w);
                    if (tid < 256) put_terms<TM>(to + L::az + C * 32, L::az_term, x, piece);
                    else put_terms<TM>(to + L::v, L::v_term, x, piece);
                    if (KP == 128 || tid < 256) {
                        const int r = tid & 15, col = tid >> 4 << 2;
                        const float4 s4 = reinterpret_cast<const float4*>(raw)[tid], d4 = reinterpret_cast<const float4*>(raw + L::raw_d)[tid];
                        const uint32_t sat = wide<16>(r, col >> 3) + 2 * (col & 7);
                        put_terms<TM>(to + L::s, L::s_term, s4, sat);
                        put_terms<2>(to + L::d, L::s_term, d4, sat);
                        cross = fmaf(s4.x, d4.x, fmaf(s4.y, d4.y, fmaf(s4.z, d4.z, fmaf(s4.w, d4.w, cross))));
                    }
                    if (tid < 128) reinterpret_cast<uint4*>(to + L::az)[tid] = reinterpret_cast<const uint4*>(raw + L::raw_g)[tid];
                    if (slab < 2 && tid >= 256) {  // the lower terms of dO
                        const int e = tid - 256;
                        *reinterpret_cast<uint4*>(to + L::az + (1 + (e >> 7)) * L::az_term + (e & 127) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    ha::release_reads();
                    ha::fence_smem_to_async();
                }
                ok = __all_sync(~0u, ok);
                ha::tmem_before_sync();  // (slab 0: the chunk before has been read from tensor memory)
                if (lane == 0 && ok) {
                    ha::bar_arrive(bars + 8 * (kFreeRaw + rs));
                    ha::bar_arrive(bars + 8 * (kReady + buf));
                }
                if (tid == 0 && slab == 0 && tiles > 1) {
                    ha::tma_store_wait_read();
                    if (ok) ha::bar_arrive(bars + 8 * kOutFree);
                }
                __syncwarp();
                issued[buf] += 1;
                if (slab == 0 && tid < 2 * C)
#pragma unroll
                    for (int u = 0; u < 8; ++u) part[u] = u < p.parts ? dots[u * C] : 0.0f;
            }
            ok = ok && wait(kDone, issued[0] - 1) && (slices == 1 || wait(kDone + 1, issued[1] - 1));
            ok = team_sync(ok);
            if (!ok) break;
            ha::tmem_after_sync();
            const bool on = c.t0 + i < c.live;
            if (tid < C * 8) *reinterpret_cast<uint4*>(sm8 + L::zero + tid * 16) = make_uint4(0, 0, 0, 0);
            {   // far_i, and the rows' weights
                const float weight = (key ? -1.0f : p.scale) * vec[I::early / 4 + i];
                float f = 0.0f;
#pragma unroll
                for (int x = 0; x < KP / 64; ++x) {
                    const int col = quarter * (KP / 4) + 16 * x;
                    uint32_t v[16];
                    ha::tmem_ld16(v, lanes + L::ta + col);
                    const uint8_t* const own = kq + (col >> 6) * L::block;
                    const uint4 y0 = *reinterpret_cast<const uint4*>(own + place<128>(row, (col & 63) >> 3)), y1 = *reinterpret_cast<const uint4*>(own + place<128>(row, ((col & 63) >> 3) + 1));
                    const uint32_t y[8] = {y0.x, y0.y, y0.z, y0.w, y1.x, y1.y, y1.z, y1.w};
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float z = weight == 0.0f ? 0.0f : weight * __uint_as_float(v[e]);
                        f = fmaf(__uint_as_float(e & 1 ? y[e / 2] & 0xffff0000u : y[e / 2] << 16), z, f);
                        v[e] = __float_as_uint(z);
                    }
                    ha::tmem_st16(lanes + L::ta + col, v);
                }
                far[(2 * quarter + key) * C + i] = on ? f : 0.0f;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) cross += __shfl_xor_sync(~0u, cross, o);
            if (lane == 0) sums[warp] = cross;
            float* const wm = reinterpret_cast<float*>(sm8 + L::w);
            float own_w[16];
            {   // the weights between tokens; H and W
                const int col = 16 * quarter;
                const float hi = vec[I::hi / 4 + i], lo = vec[I::lo / 4 + i];
                float x[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = own_w[e] = 0.0f;
                if (col <= ((row & 32) | 31)) {  // as far as the warp's last row
                    uint32_t g[16], r[16];
                    ha::tmem_ld16_early(g, lanes + L::tg + col);
                    ha::tmem_ld16_early(r, lanes + L::tr + col);
                    ha::tmem_ready(g);
                    ha::tmem_ready(r);
                    if (col + 15 < (row & 32)) {  // before all rows of the warp: one exponential for a row (as in chunk_kernel)
                        const int m = col + 15;
                        const float f = on ? (key ? -1.0f : p.scale) * ex2((hi - vec[I::hi / 4 + m]) + (lo - vec[I::lo / 4 + m])) : 0.0f;
#pragma unroll
                        for (int e = 0; e < 16; e += 4) {
                            const float4 g4 = *reinterpret_cast<const float4*>(vec + I::edge / 4 + col + e);
                            const float w4[4] = {g4.x, g4.y, g4.z, g4.w};
#pragma unroll
                            for (int u = 0; u < 4; ++u) {
                                x[e + u] = f == 0.0f ? 0.0f : f * w4[u] * __uint_as_float(g[e + u]);
                                own_w[e + u] = f == 0.0f ? 0.0f : x[e + u] * __uint_as_float(r[e + u]);
                            }
                        }
                    } else {
                        const int last = on ? (key ? i - 1 : i) - col : -1;
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] = __uint_as_float(g[e]);
                        between_tokens(x, vec + I::hi / 4 + col, vec + I::lo / 4 + col, hi, lo, key ? -1.0f : p.scale, last);
#pragma unroll
                        for (int e = 0; e < 16; ++e) own_w[e] = e <= last && col + e < i ? x[e] * __uint_as_float(r[e]) : 0.0f;
                    }
                }
                __syncwarp();
#pragma unroll
                for (int e = 0; e < 16; e += 8) {
                    uint32_t t[4][2];
#pragma unroll
                    for (int u = 0; u < 4; ++u) ha::split<2>(ha::make_pair2(x[e + 2 * u], x[e + 2 * u + 1]), t[u]);
                    const uint32_t to = L::h + place<128>(row, (col + e) >> 3);
#pragma unroll
                    for (int u = 0; u < 2; ++u) *reinterpret_cast<uint4*>(sm8 + to + u * L::h_term) = make_uint4(t[0][u], t[1][u], t[2][u], t[3][u]);
                }
                if (!key)
#pragma unroll
                    for (int e = 0; e < 16; ++e) wm[i * (C + 1) + col + e] = own_w[e];
            }
            ha::tmem_wait_st();
            ha::fence_smem_to_async();
            ha::tmem_before_sync();
            __syncwarp();
            if (lane == 0) ha::bar_arrive(bars + 8 * kNear);
            team_sync(true);
            if (key)
#pragma unroll
                for (int e = 0; e < 16; ++e) wm[i * (C + 1) + 16 * quarter + e] += own_w[e];
            {   // the gates' gradients, while the last products run
                float sum = 0.0f;
                if (tid < 2 * C) {
#pragma unroll
                    for (int u = 0; u < 8; ++u) sum += part[u];
                    for (int u = 8; u < p.parts; ++u) sum += dots[u * C];
                }
                if (tid < C && p.dbeta && c.t0 + tid < p.tokens) p.dbeta[row0 + (long long)tid * p.heads] = c.t0 + tid < c.live ? sum : 0.0f;
                if (p.dlog_a || p.part) {
                    // sum_{i>=t>j} W_ij: sums up each column by parts of 16 rows, then along the rows
                    float* const tops = far + 8 * C;          // of each part and column
                    float* const tokens3 = far + 12 * C;      // three sums of every token, and the late ones
                    if (tid >= C && tid < 2 * C) tokens3[3 * C + tid - C] = sum;
                    team_sync(true);
                    if (tid < 4 * C) {
                        const int j = tid & 63, r0 = (tid >> 6) * 16;
                        float x[16], s = 0.0f;
#pragma unroll
                        for (int r = 0; r < 16; ++r) x[r] = wm[(r0 + r) * (C + 1) + j];
#pragma unroll
                        for (int r = 15; r >= 0; --r) {
                            s += r0 + r > j ? x[r] : 0.0f;
                            wm[(r0 + r) * (C + 1) + j] = s;
                        }
                        tops[(tid >> 6) * C + j] = s;
                    }
                    if (warp == 8 || warp == 9) {  // sum_{i>=t} far_i; sum_{j<t} late_j: a lane has two tokens
                        float a = 0.0f, d = 0.0f;
                        const int t = 2 * lane;
                        if (warp == 8) {
#pragma unroll
                            for (int u = 0; u < 8; ++u) {
                                a += far[u * C + t];
                                d += far[u * C + t + 1];
                            }
                            float s = a + d;
#pragma unroll
                            for (int o = 1; o < 32; o *= 2) {
                                const float y = __shfl_down_sync(~0u, s, o);
                                if (lane + o < 32) s += y;
                            }
                            const float next = __shfl_down_sync(~0u, s, 1), behind = lane < 31 ? next : 0.0f;
                            tokens3[t] = a + (d + behind);
                            tokens3[t + 1] = d + behind;
                        } else {
                            a = tokens3[3 * C + t];
                            d = tokens3[3 * C + t + 1];
                            float s = a + d;
#pragma unroll
                            for (int o = 1; o < 32; o *= 2) {
                                const float y = __shfl_up_sync(~0u, s, o);
                                if (lane >= o) s += y;
                            }
                            const float last = __shfl_up_sync(~0u, s, 1), before = lane ? last : 0.0f;
                            tokens3[C + t] = before;
                            tokens3[C + t + 1] = before + a;
                        }
                    }
                    team_sync(true);
                    {
                        const int t = tid >> 3, o = tid & 7, own = t >> 4;
                        float g = 0.0f;
#pragma unroll
                        for (int u = 0; u < 8; ++u) {
                            const int j = o + 8 * u;
                            float x = wm[t * (C + 1) + j];
#pragma unroll
                            for (int q = 1; q < 4; ++q) x += q > own ? tops[q * C + j] : 0.0f;
                            g += j < t ? x : 0.0f;
                        }
#pragma unroll
                        for (int d = 1; d < 8; d *= 2) g += __shfl_xor_sync(~0u, g, d);
                        if (o == 0) tokens3[2 * C + t] = g;
                    }
                    team_sync(true);
                    if (tid < C) {
                        float all = 0.0f;
#pragma unroll
                        for (int w = 0; w < 16; ++w) all += sums[w];
                        float x = tokens3[tid] + tokens3[C + tid] + tokens3[2 * C + tid] + ha::decayed(vec[I::whole / 4], all);
                        if (c.t0 + tid >= c.live) x = 0.0f;
                        if (p.dlog_a && c.t0 + tid < p.tokens) p.dlog_a[row0 + (long long)tid * p.heads] = x;
                        if (p.part) {
                            double total = x;
#pragma unroll
                            for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(~0u, total, o);
                            if (lane == 0) reinterpret_cast<double*>(sums + 16)[warp] = total;
                        }
                    }
                    if (p.part) {
                        team_sync(true);
                        if (tid == 0) p.part[at] = reinterpret_cast<double*>(sums + 16)[0] + reinterpret_cast<double*>(sums + 16)[1];
                    }
                }
            }
            ok = team_sync(wait(kStep, tiles - 1));
            if (!ok) break;
            ha::tmem_after_sync();
            {
                const float late = vec[I::late / 4 + i];
                const long long to = (row0 + (long long)i * p.heads) * p.dk;
                const int each = key ? p.each_k : p.each_q, tma = key ? p.dk_tma : p.dq_tma;
                void* const out = key ? p.dk_out : p.dq;
                const bool whole = p.dk % 4 == 0 && (reinterpret_cast<uintptr_t>(out) & 15u) == 0;
#pragma unroll
                for (int x = 0; x < KP / 64; ++x) {
                    const int col = quarter * (KP / 4) + 16 * x;
                    uint32_t v[16], l[16];
                    ha::tmem_ld16_early(v, lanes + L::ta + col);
                    if (key) ha::tmem_ld16_early(l, lanes + L::tl + col);
                    ha::tmem_ready(v);
                    if (key) ha::tmem_ready(l);
                    float y[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[e] = !on ? 0.0f : key && late != 0.0f ? fmaf(late, __uint_as_float(l[e]), __uint_as_float(v[e])) : __uint_as_float(v[e]);
                    if (tma) {
                        uint8_t* const stage = sm8 + L::out + ((key ? KP / 64 : 0) + (col >> 6)) * (C * 128);
#pragma unroll
                        for (int e = 0; e < 16; e += 8)
                            *reinterpret_cast<uint4*>(stage + place<128>(i, ((col & 63) + e) >> 3)) =
                                make_uint4(ha::pack_bf16(y[e], y[e + 1]), ha::pack_bf16(y[e + 2], y[e + 3]), ha::pack_bf16(y[e + 4], y[e + 5]), ha::pack_bf16(y[e + 6], y[e + 7]));
                    } else if (c.t0 + i < p.tokens) {
#pragma unroll
                        for (int e = 0; e < 16; e += 4) {
                            if (col + e >= p.dk) break;
                            if (whole && each) *reinterpret_cast<float4*>(static_cast<float*>(out) + to + col + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
                            else
#pragma unroll
                                for (int u = 0; u < 4; u += 2) put_pair<T>(out, each, to + col + e + u, p.dk - (col + e + u), y[e + u], y[e + u + 1]);
                        }
                    }
                    __syncwarp();
                }
            }
            ha::fence_smem_to_async();
            ha::tmem_before_sync();
            team_sync(true);
            if (tid == 0) {
                for (int x = 0; x < KP / 64; ++x) {
                    if (64 * x >= p.dk) break;
                    if (p.dq_tma) ha::tma_store_4d(&mdq, 64 * x, c.h, c.t0, c.b, base + L::out + x * (C * 128));
                    if (p.dk_tma) ha::tma_store_4d(&mdk, 64 * x, c.h, c.t0, c.b, base + L::out + (KP / 64 + x) * (C * 128));
                }
                ha::tma_store_commit();
                ha::bar_arrive(bars + 8 * (kFreeTiles + ts));
            }
        }
        if (tid == 0) ha::tma_store_wait_all();
    }
    ha::tmem_before_sync();
    __syncthreads();
    if (warp == 0) ha::tmem_free(0, L::columns);
    if (tid == 0 && *stop) give_up(p, gave_up, 100 + *stop);
}

}  // namespace hd
